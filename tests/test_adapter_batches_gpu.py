"""Adapters in batches of more of them than the segments' sort has workgroups, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2503_21261_amd as hot
from test_tune_ops_gpu import check_pass, make, run_pass

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def batch(adapters, segments, longest, seed, used=None):
    rng = np.random.default_rng(seed)
    cuts = np.concatenate([[0], np.cumsum(rng.integers(0, longest + 1, segments))]).tolist()
    if used is None:
        index = rng.integers(-1, adapters + 1, segments)              # -1 and `adapters`: none
    else:
        index = rng.choice(used, segments)
    return cuts, index.tolist(), adapters


@pytest.mark.parametrize("adapters,segments,longest", [(255, 400, 3), (256, 300, 4), (257, 700, 3), (600, 257, 6), (1300, 3000, 1), (513, 1, 9), (300, 5, 40)])
def test_ranges_of_adapters(adapters, segments, longest):
    for dtype in (F32, BF16):
        cuts, index, K = batch(adapters, segments, longest, adapters + segments)
        t, kind = make(cuts[-1] + 2, 24, 40, 4, (cuts, index, K), dtype, seed=3)
        check_pass(t, kind, run_pass(t))


def test_all_segments_of_one_adapter_of_many():
    """A range whose waves all have the same adapter, beside ranges without a segment."""
    cuts, _, _ = batch(1, 900, 2, 5)
    for k in (0, 511, 512, 999):
        t, kind = make(cuts[-1], 24, 40, 4, (cuts, [k] * 900, 1000), F32, seed=4)
        check_pass(t, kind, run_pass(t))


def test_as_many_adapters_as_there_can_be():
    """65536 adapters, of which some hundred have rows: the bits of a batch that has these alone."""
    K, O, I, rank = 65536, 8, 16, 2
    rng = np.random.default_rng(9)
    used = np.sort(np.concatenate([[0, 1, 255, 256, 257, 65535], rng.choice(np.arange(300, 65000), 180, replace=False)]))
    cuts, index, _ = batch(K, 2000, 2, 10, used)
    few, kind = make(cuts[-1] + 1, O, I, rank, (cuts, np.searchsorted(used, index).tolist(), len(used)), F32, seed=6)
    got_few = run_pass(few)
    check_pass(few, kind, got_few)
    many = dict(few, a=torch.zeros(K, rank, I), b=torch.zeros(K, O, rank), scale=torch.ones(K), g_a=torch.full((K, rank, I), float("nan")),
                g_b=torch.full((K, O, rank), float("nan")), index=torch.tensor(index, dtype=torch.int32))
    for name in ("a", "b", "scale"):
        many[name][used] = few[name]
    got = run_pass(many)
    for name in ("y", "u", "g_x"):
        assert torch.equal(got[name], got_few[name]), name
    none = torch.ones(K, dtype=torch.bool)
    none[used] = False
    for name in ("g_a", "g_b"):
        assert torch.equal(got[name].cpu()[used], got_few[name].cpu()), name
        assert not got[name].cpu()[none].any()
