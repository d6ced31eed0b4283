"""Which group norms are held by one workgroup (csrc/group_plan.hpp): the rule at the limit of a launch."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rule(tmp_path):
    exe = tmp_path / "form"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", os.path.join(ROOT, "tests", "host_held_form.cpp"), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)
