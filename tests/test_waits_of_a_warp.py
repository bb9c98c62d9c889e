"""The bounded waits of the attention that reads shared tokens once (csrc/wait_together.h), as a model on the CPU (tests/wait_model.cpp): a warp passes a
wait or leaves it as a whole, whatever its lanes see of the phase and of the flag."""
import ctypes
import os
import re
import subprocess

import pytest

from tests.conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2109_04312_b200", "csrc")


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("waits") / "waits.so")
    subprocess.run(["g++", "-std=c++20", "-O1", "-Wno-unknown-pragmas", "-shared", "-fPIC", "-pthread", "-I", CSRC, os.path.join(ROOT, "tests", "wait_model.cpp"),
                    "-o", so], check=True)
    return ctypes.CDLL(so)


def run(model, together, tries, runs=60):
    out = (ctypes.c_int32 * 2)()
    model.run_waits(together, runs, tries, 5 + tries, out)
    return list(out)


@pytest.mark.parametrize("tries", [1, 3, 10])
def test_a_warp_leaves_as_a_whole(model, tries):
    assert run(model, 1, tries) == [0, 0]


def test_lanes_that_wait_for_themselves_go_apart(model):
    assert run(model, 0, 10)[0] > 0


def test_no_role_waits_otherwise():
    # tries at a barrier stand in the wait of a warp alone, and the first one of it is voted on too
    with open(os.path.join(CSRC, "mate_decode_shared.cu")) as f:
        text = f.read()
    tries = re.findall(r"[^\n]*mbar_try_wait[^\n]*", text)
    assert len(tries) == 2 and any("bool there()" in t for t in tries) and any("__all_sync(~0u, mbar_try_wait(" in t for t in tries), tries
