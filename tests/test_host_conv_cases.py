"""The runs of tokens that the GPU tests of long convolutions are after (csrc/conv_plan.hpp)."""
import os
import subprocess

from tests import test_gpu_conv_runs as runs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_runs(tmp_path):
    exe = tmp_path / "cases"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", os.path.join(ROOT, "tests", "host_conv_cases.cpp"), "-o", str(exe)], check=True)
    lines = []
    for c, _ in runs.FORWARD + runs.BACKWARD:
        B, H, N, d, dtype = c[0], c[1], c[2], c[3], c[6]
        lines.append(f"{B} {H * d // (8 if dtype == 'bf16' else 4)} {H * d // 4} {N}")
    out = subprocess.run([str(exe)], input="\n".join(lines), check=True, capture_output=True, text=True).stdout.splitlines()
    got = [tuple(map(int, line.split())) for line in out]
    assert [f for f, _ in got[:len(runs.FORWARD)]] == [r for _, r in runs.FORWARD]
    assert [b for _, b in got[len(runs.FORWARD):]] == [r for _, r in runs.BACKWARD]
