"""The GPU tests' cases of many rows make workgroups walk several steps, in every form of several waves, and leave lanes without a row."""
import os
import subprocess

from tests import test_gpu_norm_rows as rows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rows(tmp_path):
    exe = tmp_path / "host_norm_cut"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", os.path.join(ROOT, "tests", "host_norm_cut.cpp"), "-o", str(exe)], check=True)
    for cases, backward, forms in ((rows.FORWARD, 0, {(128, 4), (256, 3), (512, 2), (1024, 2)}),
                                   (rows.BACKWARD, 1, {(128, 2), (128, 3), (128, 4), (256, 3), (512, 2), (1024, 2)})):
        args = [str(x) for d, dtype, n in cases for x in (d * (2 if dtype == "bf16" else 4) // 16, n, backward, d)]
        out = list(map(int, subprocess.run([str(exe), *args], stdout=subprocess.PIPE, text=True, check=True).stdout.split()))
        seen = {"bf16": set(), "f32": set()}
        for i, (d, dtype, n) in enumerate(cases):
            lanes, vecs, per, wgs = out[4 * i:4 * i + 4]
            seen[dtype].add((lanes, vecs))
            assert n > wgs * per and (n % (wgs * per) or n % per), (d, dtype, n)
        assert seen["f32"] == forms and seen["bf16"] == forms - {(1024, 2)}, seen
