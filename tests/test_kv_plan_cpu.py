"""The launch plans of the paged cache's attention and its workspace, swept on the host: no GPU is
needed to show that what a call writes fits into what it checks."""
import ctypes
import os
import subprocess

import pytest

import paper_2606_10896_amd as gmm
from paper_2606_10896_amd.kv import _CCache

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


def test_a_workspace_for_larger_sizes_serves_smaller_ones(check):
    check("grows")


def test_the_largest_calls_fit_into_a_launch(check):
    check("launches")


def test_the_workspace_of_no_tokens(check):
    """A server's empty step: a size, and not a division by its zero tiles."""
    cache = _CCache(1 << 20, 1 << 20, None, None, 10, 2, 64, 128, 1)
    size = gmm.load_library().gmm_kv_workspace_bytes
    assert 0 < size(ctypes.byref(cache), 0, 4, 3, 4) <= size(ctypes.byref(cache), 1, 4, 3, 4)
