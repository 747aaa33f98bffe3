"""How hot_linear_forward works on a product, on the host: that the shapes of the GPU tests reach every way there is, and what
hot_debug_linear_plan refuses."""
import ctypes as C

import pytest
import torch

import paper_2503_21261_amd as hot
from test_block_ops_gpu import LINEAR_WAYS

F32, BF16 = torch.float32, torch.bfloat16


def parts(p):
    """Whether tiles have a workgroup each, or K is cut for all of them or for the last ones."""
    return "whole" if p["whole"] == p["tiles"] else "sliced" if p["whole"] == 0 else "last sliced"


def test_the_shapes_of_the_tests_take_every_way():
    taken = {}
    for t, L, O, I in LINEAR_WAYS:
        p = hot.hot_debug_linear_plan(t, L, O, I)
        taken.setdefault((t, p["way"], p["tile"], parts(p), p["masked"]), []).append((L, O, I))
    for t in (F32, BF16):
        for tile in ((16, 16), (16, 32), (32, 16), (32, 32), (64, 16), (64, 32)):
            for cut in ("whole", "sliced"):
                assert (t, "rows", tile, cut, False) in taken
        for tile in ((64, 64), (32, 128)):
            for cut in ("whole", "sliced"):
                assert (t, "direct", tile, cut, True) in taken
        for tile in ((128, 128), (256, 256)):
            assert (t, "packed", tile, "whole", False) in taken and (t, "packed", tile, "sliced", False) in taken
    assert (F32, "packed", (128, 128), "last sliced", False) in taken and (F32, "packed", (256, 256), "last sliced", False) in taken
    for tile in ((128, 128), (256, 256)):
        for cut in ("whole", "sliced", "last sliced"):
            for masked in (False, True):
                assert (BF16, "tiles", tile, cut, masked) in taken


@pytest.mark.parametrize("t", [F32, BF16])
def test_plans_are_whole(t):
    for L, O, I in [s[1:] for s in LINEAR_WAYS] + [(1, 1, 1), (2 ** 31 - 1, 1, 1), (2 ** 23, 300, 64), (12608, 2304, 768), (16384, 11008, 4096)]:
        p = hot.hot_debug_linear_plan(t, L, O, I)
        run = min(L, 2 ** 23)
        assert p["tiles"] == -(-run // p["tile"][0]) * -(-O // p["tile"][1]) and 0 <= p["whole"] <= p["tiles"]
        assert 1 <= p["slices"] <= 16 and (p["slices"] > 1) == (p["whole"] < p["tiles"])
        need = hot.hot_linear_forward_workspace_bytes(t, run, O, I)
        assert (need > 0) == (p["way"] == "packed" or p["slices"] > 1)
        assert p["streams"] == (run * O * (4 if t == F32 else 2) > 2 ** 25 and O * (4 if t == F32 else 2) % 128 == 0)
        kept = hot.hot_debug_linear_plan(t, L, O, I, ckpt=True)       # a checkpoint's groups of 32 outputs are one workgroup's
        assert kept["way"] == p["way"] and (kept["slices"] > 1 or kept["tile"][1] >= 32)


def test_linear_plan_refusals():
    f, p = hot.lib().hot_debug_linear_plan, hot.hot_linear_plan()
    assert f(0, 0, 4, 4, 4, 0, None) == hot.HOT_ERR_ARG
    assert f(2, 0, 4, 4, 4, 0, C.byref(p)) == hot.HOT_ERR_ARG and f(0, 1, 4, 4, 4, 0, C.byref(p)) == hot.HOT_ERR_ARG
    for bad in ((0, 4, 4), (4, 0, 4), (4, 4, 0), (1 << 31, 4, 4), (4, 1 << 24, 4), (4, 4, 1 << 24)):
        assert f(0, 0, *bad, 0, C.byref(p)) == hot.HOT_ERR_SHAPE
    assert f(1, 0, 4, 4, 4, 0, C.byref(p)) == hot.HOT_OK
