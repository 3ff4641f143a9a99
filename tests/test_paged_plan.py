"""ppd_paged_attention's index arithmetic at the ends of its ranges, on the CPU (paged_plan.hip: the kernels' own functions, built for the host)."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "paged_plan.so")
    subprocess.check_call(["hipcc", "--offload-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC", "-shared", "-fsanitize=signed-integer-overflow",
                           "-fsanitize-trap=signed-integer-overflow", "-o", so, os.path.join(HERE, "paged_plan.hip")], stderr=subprocess.DEVNULL)
    return ctypes.CDLL(so)


@pytest.mark.parametrize("pos", [-2 ** 22, -3, -1, 0, 1, 63, 64, 1000, 2 ** 30, MOST - 1])
@pytest.mark.parametrize("window", [0, 1, 2, 64, 1000, 2 ** 30, MOST - 1, MOST])
def test_the_first_position_of_a_window(plan, pos, window):
    assert plan.t_first_seen(pos, window) == (max(pos - window + 1, 0) if window else 0)
