"""The launch plans of the paged cache's attention and its workspace, swept on the host: no GPU is
needed to show that what a call writes fits into what it checks."""
import os
import subprocess

import pytest

import paper_2606_10896_amd as gmm

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(gmm.__file__), "csrc")


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "kv_plan_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, "-o", exe,
                    os.path.join(HERE, "kv_plan_check.cpp")], check=True)

    def run(rule):
        res = subprocess.run([exe, rule], capture_output=True, text=True)
        assert res.returncode == 0, res.stdout + res.stderr
    return run


def test_a_call_fits_into_its_workspace(check):
    check("covers")
