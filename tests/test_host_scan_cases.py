"""How selective scans are cut (csrc/scan_plan.hpp): the cases that the GPU tests take for their segments have them."""
import os
import subprocess

import pytest

from tests import test_gpu_scan_growth, test_gpu_scan_long

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """(B, groups, channels of a group, tokens) of each call -> ((segments, tokens of a segment) forwards, the same backwards)."""
    exe = tmp_path_factory.mktemp("plan") / "cases"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", os.path.join(ROOT, "tests", "host_scan_cases.cpp"), "-o", str(exe)], check=True)

    def of(calls):
        out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in calls), check=True, capture_output=True, text=True).stdout
        return [((a, b), (c, d)) for a, b, c, d in (map(int, line.split()) for line in out.splitlines())]
    return of


def _call(c):
    B, H, N, d, G = c[:5]
    return B, G, H // G * d, N


def test_long_cases(plans):
    assert plans([_call(c) for c, _, _ in test_gpu_scan_long.PLANS]) == [(f, b) for _, f, b in test_gpu_scan_long.PLANS]


def test_growth_cases(plans):
    for (c, _, _, per, segments), (f, b) in zip(test_gpu_scan_growth.CASES, plans([_call(c[0]) for c in test_gpu_scan_growth.CASES])):
        assert per == max(f[1], b[1]) and segments >= max(f[0], b[0])


def test_sequences_that_fill_the_machine_are_not_cut(plans):
    """More than half of the waves that run at once without a cut (4 096 forwards, 2 048 backwards): the sums of a cut cost more than its waves bring."""
    sequences = list(range(1, 200))
    for N in (512, 1560, 32760):
        for B, (f, b) in zip(sequences, plans([(B, 1, 2240, N) for B in sequences])):
            waves = 35 * B
            assert (f[0] == 1) == (waves > 2048) and (b[0] == 1) == (waves > 1024), (B, N, f, b)
