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


def spans(plan, pos0, n, tile, tile_rows, group, parts, room, window):
    lo, hi, found = ctypes.c_int(), ctypes.c_int(), []
    for part in range(parts):
        plan.t_span(pos0, n, tile, tile_rows, group, part, parts, room, window, ctypes.byref(lo), ctypes.byref(hi))
        found.append((lo.value, hi.value))
    return found


@pytest.mark.parametrize("tile_rows", [16, 128])
@pytest.mark.parametrize("n,group", [(1, 1), (5, 1), (70, 4), (3, 7), (300, 8)])
@pytest.mark.parametrize("parts", [1, 2, 5, 40])
@pytest.mark.parametrize("room", [1, 64, 1000, 4096, 2 ** 30])
def test_a_tiles_parts(plan, tile_rows, n, group, parts, room):
    """Together they are the positions that some row of the tile sees, from a multiple of 64 on, each once and in order; an empty one is at 0,
    also for lengths at the ends of their range, where the look-ups ahead of a loop (a few hundred positions) stay within 31 bits."""
    for kv in (0, 2, n, n + 63, 700, 2 ** 30 - 1, 2 ** 30 + 5, MOST - 100, MOST):
        for window in (0, 1, 100, MOST - 200, MOST):
            for tile in sorted({0, (n * group - 1) // tile_rows}):
                first, last = tile * tile_rows // group, min((tile * tile_rows + tile_rows - 1) // group, n - 1)
                lo = max(kv - n + first - window + 1, 0) // 64 * 64 if window else 0
                hi = min(kv - n + last + 1, room)
                at = lo
                for a, b in spans(plan, kv - n, n, tile, tile_rows, group, parts, room, window):
                    assert 0 <= a <= b <= room and a % 64 == 0 and a + 4096 <= MOST
                    if a < b:
                        assert a == at and (b % 64 == 0 or b == hi)
                        at = b
                    else:
                        assert a == b == 0
                assert at == (hi if hi > lo else lo)


def test_parts_without_places(plan):
    have = plan.t_have_places
    assert have(0, 1, 1) and have(5, 3, 8) and have(0, MOST, MOST)
    assert not have(5, 4, 8) and not have(8, 1, 8) and not have(-1, 1, 8) and not have(MOST, 1, 8) and not have(0, MOST, 8) and not have(7, MOST, 8)
