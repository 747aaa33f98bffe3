"""Calls at the ends of what the operators of a fine-tuning step take, on the GPU."""
import math

import pytest
import torch

import paper_2503_21261_amd as hot
import tune_oracle as ref
from test_tune_ops_gpu import check_pass, make, rand, run_logprobs, run_pass, within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V,top", [(524288, 20), (524289, 20), (600001, 32), ((1 << 24) - 1, 32)])
def test_vocabularies_whose_parts_are_read_again(V, top, dtype):
    """More than 64 parts of what a workgroup holds: the likeliest tokens of the rest of a part come from a second reading."""
    z = rand((1, V), 3.0, V % 1000)
    z[0, V - 1], z[0, V // 3], z[0, 9000] = 21.0, 22.0, 23.0
    z[0, 5:V:7] = -math.inf
    z[0, 9000] = 23.0
    z = z.to(dtype)
    targets, gl, ge = torch.tensor([V // 3]), rand((1,), 1.0, 2), rand((1,), 0.3, 3)
    want = ref.logprobs(z, targets, top, gl, ge)
    got = run_logprobs(z, targets, top, gl, ge)
    for name in ("logp", "entropy", "stats", "top_logp", "g_logits"):
        within(name, got[name], *want[name])
    assert torch.equal(got["top_ids"].cpu().long(), want["top_ids"])


def test_ties_and_rows_without_tokens_in_parts_that_are_read_again():
    V, top = 600001, 32
    z = torch.zeros(3, V)
    z[1] = -math.inf
    z[1, V - 3], z[1, 20000] = 1.0, 2.0
    z[2, 15000], z[2, V - 1] = math.nan, math.nan
    got = run_logprobs(z, torch.tensor([V - 1, V - 3, 0]), top)
    assert torch.equal(got["top_ids"][0].cpu(), torch.arange(top, dtype=torch.int32))
    assert got["top_ids"][1].tolist() == [20000, V - 3] + list(range(top - 2)) and (got["top_logp"][1, 2:] == -math.inf).all()
    assert got["top_ids"][2].tolist()[:2] == [15000, V - 1] and got["top_logp"][2].isnan().all() and got["logp"][2].isnan()
    # V / 256 + 24 additions, as the 64-bit form counts them
    within("logp", got["logp"][:1], torch.tensor([-math.log(V)], dtype=torch.float64), torch.tensor([(V / 256 + 24 + 5 * math.log(V)) * ref.U], dtype=torch.float64))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(5, 300), (70, 9000), (2100, 40)])
@pytest.mark.parametrize("std,shift", [(40.0, 0.0), (100.0, -300.0), (1e-3, 50.0)])
def test_logits_far_apart(std, shift, rows, V, dtype):
    """Probabilities down to where they are none: those below 2^-126 count as 0, which is 2^-126 |log p + H| of the entropy's gradient."""
    z = (rand((rows, V), std, rows + V) + shift).to(dtype)
    targets, gl, ge = torch.randint(0, V, (rows,), generator=torch.Generator().manual_seed(1)), rand((rows,), 1.0, 2), rand((rows,), 1.0, 3)
    want, got = ref.logprobs(z, targets, 0, gl, ge), run_logprobs(z, targets, 0, gl, ge)
    for name in ("logp", "entropy", "stats"):
        within(name, got[name], *want[name])
    lp = torch.log_softmax(z.double(), 1)
    none = torch.where(lp < -87, 2.0 ** -126 * ge.double().abs()[:, None] * torch.exp(lp + 126 * math.log(2)).clamp(max=1.0) * (lp.abs() + want["entropy"][0][:, None]), 0.0)
    within("g_logits", got["g_logits"], want["g_logits"][0], want["g_logits"][1] + none)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("L", [1, 3, 70, 300])
def test_rows_without_offsets_have_the_first_of_several_adapters(L, dtype):
    t, kind = make(L, 72, 100, 12, (None, None, 3), dtype, seed=9)
    got = run_pass(t)
    check_pass(t, kind, got)
    assert not got["g_a"][1:].any() and not got["g_b"][1:].any()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_widest_rows(dtype):
    """Rows of 2^24 - 1 columns on either side."""
    N = (1 << 24) - 1
    for O, I in ((N, 5), (5, N)):
        t, kind = make(3, O, I, 2, (None, None, 1), dtype, seed=12)
        check_pass(t, kind, run_pass(t))


@pytest.mark.parametrize("L,wide,rank", [(70, 4, 1), (70, 4, 20), (70, 4, 100), (70, 2000, 1), (70, 2000, 40), (2100, 4, 16), (1, 4, 1), (1, 2000, 3)])
def test_factors_enter_bfloat16_products_within_16_bits(L, wide, rank):
    """u = 1 + 2^-7 - 2^-23 beside a base of -(1 + 2^-7): two parts that are both cut off make 2^-15 of it."""
    parts = torch.tensor([1.0, 2.0 ** -7 - 2.0 ** -15, 2.0 ** -15 - 2.0 ** -23]).to(BF16)
    assert parts.double().sum() == 1 + 2.0 ** -7 - 2.0 ** -23
    t, kind = make(L, wide, wide, rank, (None, None, 1), BF16, seed=1)
    for name in ("x", "g_y", "a", "b"):
        t[name].zero_()
    t["x"][:, 0:3], t["g_y"][:, 0:3] = parts, parts
    t["a"][0, 0], t["b"][0, :, 0] = 1.0, 1.0
    t["scale"] = torch.ones(1)
    t["base"].fill_(-(1 + 2.0 ** -7))
    t["g_base"].fill_(-(1 + 2.0 ** -7))
    got = run_pass(t)
    check_pass(t, kind, got)
    for name in ("y", "g_x"):
        # 2^-16 of u, and the roundings of three sums
        assert (got[name].double() + 2.0 ** -23).abs().max() <= 2.0 ** -16 * 1.01 + 2.0 ** -22, name
