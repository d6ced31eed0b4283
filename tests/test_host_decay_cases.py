"""The GPU tests' long calls are cut as they have to be: several segments of more than eight chunks, prompts past the caches; every head dimension
and type in both directions."""
import os
import subprocess

from tests import test_gpu_decay as gpu
from tests import test_gpu_decay_long as long

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _shares_lines(case):
    """Heads inside tokens, with rows that are no whole lines of 128 bytes."""
    return case[5] != "bhnd" and case[3] * (2 if case[4] == "bf16" else 4) % 128 != 0


def _cuts(tmp_path, cases, walks):
    exe = tmp_path / "host_decay_cut"
    if not exe.exists():
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", os.path.join(ROOT, "tests", "host_decay_cut.cpp"), "-o", str(exe)], check=True)
    args = [str(x) for c in cases for x in (c[0] * c[1], c[2], c[3], int(c[4] == "bf16"), walks, int(_shares_lines(c)))]
    out = subprocess.run([str(exe), *args], stdout=subprocess.PIPE, text=True, check=True).stdout.split()
    return [tuple(map(int, out[3 * i:3 * i + 3])) for i in range(len(cases))]


def test_long_calls(tmp_path):
    for c, (segments, chunks, past) in zip(long.PROMPTS, _cuts(tmp_path, long.PROMPTS, 1)):
        assert segments > 1 and chunks > 8 and past == (not _shares_lines(c)), c
    for c, (segments, chunks, past) in zip(long.BACKWARDS, _cuts(tmp_path, long.BACKWARDS, 3)):
        assert segments > 1 and chunks > 8 and not past, c
    # (fp32 of 32 features past the caches: test_gpu_decay.py, long memory)
    kinds = {(d, t) for d in (32, 64, 112, 128) for t in ("bf16", "f32")}
    assert {(c[3], c[4]) for c in long.PROMPTS if not _shares_lines(c)} | {(32, "f32")} == kinds and {(c[3], c[4]) for c in long.BACKWARDS} == kinds


def test_short_calls(tmp_path):
    """One segment and several, of one chunk each and of more, among the small calls; none of them past the caches."""
    for walks in (1, 3):
        cuts = _cuts(tmp_path, gpu.CASES, walks)
        assert not any(past for _, _, past in cuts)
        assert any(s == 1 and n > 1 for s, n, _ in cuts) and any(s > 1 and n == 1 for s, n, _ in cuts) and any(s > 1 and n > 1 for s, n, _ in cuts)
