"""The barriers between the softmax teams and the warps that issue products in the attention that reads shared tokens once, as a model on the CPU
(tests/shared_teams_model.cpp): no wait passes for another phase, nothing is written that somebody uses, and no run stands still, whatever the order in which the
roles get on."""
import ctypes
import os
import subprocess

import pytest

from tests.conftest import ROOT


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("teams") / "teams.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", os.path.join(ROOT, "tests", "shared_teams_model.cpp"), "-o", so], check=True)
    return ctypes.CDLL(so)


def run(model, variant, most, runs=3000):
    out = (ctypes.c_int32 * 3)()
    model.run_teams(variant, runs, most, 3 + most, out)
    return list(out)


@pytest.mark.parametrize("most", [1, 2, 3, 9])
def test_as_built(model, most):
    assert run(model, 0, most) == [0, 0, 0]


def test_what_the_model_finds(model):
    assert run(model, 1, 3)[1] > 0      # O is made 0 while the other team reads it
    assert run(model, 2, 9)[1] > 0      # scores go where weights are that are still multiplied
    assert run(model, 3, 9)[0] > 0      # a parity that is that of the phase before the last
