"""The operators around the linear backward on the GPU, on values where they can go wrong: infinities and NaN, rows of a wide range,
operands whose products are exact; each on the way of working that is meant."""
import pytest
import torch

import block_oracle as ref
import paper_2503_21261_amd as hot
from test_block_ops_gpu import BF16, F32, FNS, LINEAR_WAYS, close, rand

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("fn", FNS)
def test_gradient_of_a_group_that_held_an_infinity_or_a_nan(fn, dtype):
    """Such a group of a checkpoint reads as NaN, so its gradients are NaN, finite neighbours of the bad element among them, and so are
    the bias sums of its columns; all others are as ever."""
    rows, cols = 300, 100
    x, g = rand((rows, cols), 1, dtype, 2.0), rand((rows, cols), 2, dtype)
    x[3, 5], x[7, 40], x[299, 99] = INF, NAN, -INF          # the last one in a row's short last group
    lost = torch.zeros((rows, cols), dtype=torch.bool)
    lost[3, :32], lost[7, 32:64], lost[299, 96:] = True, True, True
    kept, y = hot.alloc_checkpoint(rows, cols), torch.empty((rows, cols), dtype=dtype, device="cuda")
    gx, gb = torch.empty_like(y), torch.empty(cols, device="cuda")
    hot.hot_activation_forward(hot.ACT_FNS[fn], x.cuda(), y, ckpt=kept)
    hot.hot_activation_backward(hot.ACT_FNS[fn], g.cuda(), gx, ckpt=kept, g_bias=gb, ws=hot.alloc_activation_workspace(rows, cols))
    values = ref.checkpoint(x)[2]
    want, tol, bias, btol = ref.act_grad(fn, ref.f64(g), values, dtype)
    close(gx, want.masked_fill(lost, NAN), tol, "g_x")
    close(gb, bias.masked_fill(lost.any(0), NAN), btol, "g_bias")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_relu_gradient_of_infinities_and_nan(dtype):
    x = torch.tensor([[INF, 1.0, -INF, -1.0, NAN, 0.0, -0.0, 2.0]], dtype=dtype)
    g = torch.full_like(x, 3.0).cuda()
    gx = hot.hot_activation_backward(hot.HOT_ACT_RELU, g, torch.empty_like(g), x=x.cuda())
    want = torch.tensor([[3.0, 3.0, 0.0, 0.0, NAN, 0.0, 0.0, 3.0]], dtype=torch.float64)
    close(gx, want, torch.zeros_like(want), "g_x")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 100, 200, 500, 771, 1500, 4096, 5000, 11008, 16384])
def test_layer_norm_mean_is_the_exact_one_rounded_once(cols, dtype):
    """Rows about zero, with columns that stand out, far from zero, and of the largest numbers.  In 64 bits a lane adds 16 columns and at
    most 25 more additions join the lanes and waves (2^-53 of mean |h| each, and the division), then the mean is rounded: half a step."""
    x = rand((24, cols), cols, dtype)
    x[6:12, ::100] *= 20
    x[12:18] += 300
    x[18:21] *= 1e-30
    x[21:] = x[21:].abs() * 1e37
    y, mean, rstd = torch.empty((24, cols), dtype=dtype, device="cuda"), torch.empty(24, device="cuda"), torch.empty(24, device="cuda")
    hot.hot_layer_norm_forward(x.cuda(), None, None, 1e-6, y, mean, rstd)
    want = ref.f64(x).mean(1)
    close(mean, want, want.abs() * (1 + 2.0 ** -20) * ref.U + 2.0 ** -47 * ref.f64(x).abs().mean(1), "mean")


# ---- forward product ------------------------------------------------------------------------------------------------------------

def product64(x, w):
    """x.w^T and |x|.|w|^T of device tensors in 64 bits."""
    x, w = x.double(), w.double()
    return (x @ w.t().contiguous()).cpu(), (x.abs() @ w.abs().t().contiguous()).cpu()


def held_to(y, z, size, I, what, units=26):
    """The product's error for terms of random signs, in units of 2^-24 |x|.|w|: operands to 22 bits and a product left out, each 2^-22
    at most (12), what the checks of a row's range let through (4), and the additions: partial sums of k terms are about sqrt(k) of
    them, so that I roundings of them add up to 1.2 standard deviations (10 for eight).  Of factors that are multiplied as they are: a
    rounding of each product at most and the additions (12).  No result is nearer than half the smallest number in each of its
    terms."""
    close(y, z, units * ref.U * size + (2 * I + 1) * 2.0 ** -150, what)


def call_linear(x, w, **kw):
    L, O, I, t = x.shape[0], w.shape[0], x.shape[1], x.dtype
    y = torch.full((L, O), NAN, dtype=kw.pop("y_type", F32), device="cuda")
    return hot.hot_linear_forward(x, w, y, hot.alloc_linear_workspace(t, L, O, I), **kw)


# The large tiles of packed fp32 operands: 128 x 128 and 256 x 256, whole, in slices, and with the last ones in slices
PACKED = [(3590, 3585, 33, (128, 128), "whole"), (2600, 1500, 1030, (128, 128), "whole"), (3500, 3600, 100, (256, 256), "whole"),
          (1200, 260, 9001, (128, 128), "sliced"), (7329, 162, 5528, (256, 256), "sliced"), (6742, 1245, 2568, (128, 128), "last sliced"),
          (5054, 3202, 528, (256, 256), "last sliced")]


def packed(L, O, I, tile, cut):
    p = hot.hot_debug_linear_plan(F32, L, O, I)
    assert p["way"] == "packed" and p["tile"] == tile
    assert cut == ("whole" if p["whole"] == p["tiles"] else "sliced" if p["whole"] == 0 else "last sliced")
    print(f"[packed] {L}x{O}x{I} {p}", flush=True)


@pytest.mark.parametrize("t,L,O,I", LINEAR_WAYS + [(F32, 500, 100, 64), (F32, 100, 500, 96), (BF16, 500, 100, 128), (BF16, 100, 500, 64)])
def test_linear_of_whole_numbers_is_exact(t, L, O, I):
    """Every product and sum is a whole number that fp32 holds (sums of I <= 40003 terms of +-4095 are within 4096 x 4095 by twenty
    standard deviations), so the result has one value: a part of an operand or a piece of K that is left out shows.  fp32: twelve
    bits, one more than an fp16 part has, against +-1, either way round."""
    print(f"[whole numbers] {L}x{O}x{I} {t} {hot.hot_debug_linear_plan(t, L, O, I)['way']}", flush=True)
    g = torch.Generator("cuda").manual_seed(L + O + I)

    def numbers(shape, wide):
        sign = torch.randint(0, 2, shape, generator=g, device="cuda", dtype=F32) * 2 - 1
        if not wide:
            return sign.to(t)
        n = 2049 + 2 * torch.randint(0, 1024, shape, generator=g, device="cuda", dtype=F32) if t == F32 else \
            torch.randint(1, 256, shape, generator=g, device="cuda", dtype=F32)
        return (sign * n).to(t)

    for wide_x in (True, False):
        x, w = numbers((L, I), wide_x), numbers((O, I), not wide_x)
        want = x.double() @ w.double().t().contiguous()
        assert float(want.abs().max()) < 2 ** 24
        assert torch.equal(call_linear(x, w, y_type=F32).double(), want)


@pytest.mark.parametrize("t,L,O,I", LINEAR_WAYS)
def test_every_way_near_the_exact_one(t, L, O, I):
    x, w = rand((L, I), 1, t).cuda(), rand((O, I), 2, t, I ** -0.5).cuda()
    in_parts = t == F32 and hot.hot_debug_linear_plan(t, L, O, I)["way"] == "packed"
    held_to(call_linear(x, w), *product64(x, w), I, "y", units=26 if in_parts else 12)


@pytest.mark.parametrize("L,O,I,tile,cut", PACKED)
def test_packed_product_near_the_exact_one(L, O, I, tile, cut):
    packed(L, O, I, tile, cut)
    x, w = rand((L, I), 1).cuda(), rand((O, I), 2, std=I ** -0.5).cuda()
    held_to(call_linear(x, w), *product64(x, w), I, "y")


@pytest.mark.parametrize("L,O,I,tile,cut", PACKED)
def test_packed_rows_of_any_magnitude(L, O, I, tile, cut):
    """Each row of either operand has a scale of its own; rows of zeros, a row with one subnormal element, and within every row
    values far below its largest."""
    packed(L, O, I, tile, cut)
    x, w = rand((L, I), 1), rand((O, I), 2, std=I ** -0.5)
    x *= (2.0 ** torch.linspace(-62, 60, L).round())[torch.randperm(L, generator=torch.Generator().manual_seed(3))][:, None]
    w *= (2.0 ** torch.linspace(-62, 60, O).round())[torch.randperm(O, generator=torch.Generator().manual_seed(4))][:, None]
    x[:, ::3] *= 2.0 ** -20
    x[3], w[5], x[4] = 0.0, 0.0, 0.0
    x[4, 7] = 1e-40
    x, w = x.cuda(), w.cuda()
    held_to(call_linear(x, w), *product64(x, w), I, "y")


@pytest.mark.parametrize("L,O,I,tile,cut", PACKED)
def test_packed_rows_with_an_infinity_or_nan_stay_alone(L, O, I, tile, cut):
    packed(L, O, I, tile, cut)
    x, w = rand((L, I), 1), rand((O, I), 2, std=I ** -0.5)
    x[2, 5], x[L - 2, I - 1], x[L - 1, 0], w[7, 1], w[O - 1, I - 2] = NAN, INF, -INF, NAN, INF
    y = call_linear(x.cuda(), w.cuda())
    bad = torch.zeros((L, O), dtype=torch.bool)
    bad[2], bad[L - 2], bad[L - 1], bad[:, 7], bad[:, O - 1] = (True,) * 5
    assert torch.equal(~torch.isfinite(y.cpu()), bad)
    x[~torch.isfinite(x)], w[~torch.isfinite(w)] = 0.0, 0.0       # the rows beside them are right
    x, w = x.cuda(), w.cuda()
    z, size = product64(x, w)
    held_to(y.masked_fill(bad.cuda(), 0.0), z.masked_fill(bad, 0.0), size, I, "y")


def test_packed_products_on_two_streams_at_once():
    """Operands packed, K in slices, epilogue and checkpoint, on two streams with workspaces of their own: as one after another."""
    L, O, I = 7329, 162, 5528
    packed(L, O, I, (256, 256), "sliced")
    w, b = rand((O, I), 1, std=I ** -0.5).cuda(), rand((O,), 2).cuda()
    x = [rand((L, I), 3 + k).cuda() for k in range(2)]
    ws = [hot.alloc_linear_workspace(F32, L, O, I) for _ in range(2)]
    kept = [torch.zeros_like(hot.alloc_checkpoint(L, O)) for _ in range(2)]
    y = [torch.zeros((L, O), device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]

    def step(k, s):
        hot.hot_linear_forward(x[k], w, y[k], ws[k], bias=b, fn=hot.HOT_ACT_GELU, ckpt=kept[k], stream=s)

    torch.cuda.synchronize()
    for k in range(2):
        step(k, streams[0])
        torch.cuda.synchronize()
    alone = [t.clone() for t in y + kept]
    for t in y + kept:
        t.zero_()
    torch.cuda.synchronize()
    for _ in range(4):
        for k in range(2):
            step(k, streams[k])
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(alone, y + kept))


def spread_columns(x, w):
    """Columns that are large in x are small in w: their products are alike, and every one counts."""
    x *= torch.logspace(-8, 0, x.shape[1], device="cuda")
    w *= torch.logspace(0, -8, w.shape[1], device="cuda")


def large_column(size):
    def scale(x, w):
        x[:, x.shape[1] // 2] *= size
        w[:, x.shape[1] // 2] = 0.0
    return scale


def large_against_small(x, w):
    x[:, 1] *= 1e6
    w[:, 1] *= 1e-7


def one_wide_row(x, w):
    x[-1] *= 10.0 ** torch.linspace(-30, 6, x.shape[1], device="cuda")


def one_wide_weight(x, w):
    w[w.shape[0] // 2] *= 10.0 ** torch.linspace(5, -25, x.shape[1], device="cuda")


def one_column_rows(x, w):
    """Rows with one element: each result is one product."""
    at = torch.arange(x.shape[0], device="cuda") % x.shape[1]
    kept = x[torch.arange(x.shape[0], device="cuda"), at].clone()
    x.zero_()
    x[torch.arange(x.shape[0], device="cuda"), at] = kept


def from_end_to_end(x, w):
    """Beside the row's largest the others vanish even as they are scaled."""
    x *= 2.0 ** -100
    w *= 2.0 ** 90
    x[:, 0], w[:, 0] = 2.0 ** 100, 0.0


RANGES = {"columns": spread_columns, "2^24": large_column(2.0 ** 24), "2^30": large_column(2.0 ** 30), "1e6 by 1e-7": large_against_small,
          "a row": one_wide_row, "a weight": one_wide_weight, "one column": one_column_rows,
          "2^200": from_end_to_end}


@pytest.mark.parametrize("name", RANGES)
@pytest.mark.parametrize("L,O,I,tile,cut", PACKED + [(3590, 3585, 3, (128, 128), "whole"), (3590, 3585, 2, (128, 128), "whole"),
                                                     (3590, 3585, 5, (128, 128), "whole")])
def test_packed_rows_of_a_wide_range(L, O, I, tile, cut, name):
    """A row's two 16-bit parts hold an element to 2^-39 of the row's largest.  Where that is not enough for the product, whatever w is,
    the result is no worse than on any other way."""
    packed(L, O, I, tile, cut)
    x, w = rand((L, I), 1).cuda(), rand((O, I), 2, std=I ** -0.5).cuda()
    RANGES[name](x, w)
    held_to(call_linear(x, w), *product64(x, w), I, "y")


@pytest.mark.parametrize("L,O,I,tile,cut", PACKED)
def test_packed_rows_of_a_wide_range_through_the_epilogue(L, O, I, tile, cut):
    packed(L, O, I, tile, cut)
    x, w, b, r = rand((L, I), 1).cuda(), rand((O, I), 2, std=I ** -0.5).cuda(), rand((O,), 3), rand((L, O), 4)
    x[L // 2:, 0] *= 2.0 ** 24
    w[:, 0] = 0.0
    kept = hot.alloc_checkpoint(L, O)
    y = call_linear(x, w, bias=b.cuda(), residual=r.cuda(), fn=hot.HOT_ACT_SILU, ckpt=kept)
    z, size = product64(x, w)
    z = z + ref.f64(b)
    dz = 27 * ref.U * size + ref.U * z.abs()
    want, dy = ref.act("silu", z)
    close(y, want + ref.f64(r), dy + 1.2 * dz + 2 * ref.U * (want.abs() + ref.f64(r).abs()), "y")
    back = ref.f64(hot.hot_checkpoint_read(kept, torch.empty((L, O), device="cuda")))
    pad = torch.zeros(L, -(-O // 32) * 32, dtype=torch.float64)
    pad[:, :O] = z.abs() + dz
    step = pad.view(L, -1, 32).amax(-1).clamp(min=2.0 ** -118) / 63.75      # the largest is 63.75 steps or more
    close(back, z, dz + step.repeat_interleave(32, 1)[:, :O] / 2, "z of the checkpoint")


@pytest.mark.parametrize("L,O,I,tile,cut", PACKED)
def test_packed_infinities_are_infinite(L, O, I, tile, cut):
    packed(L, O, I, tile, cut)
    x, w = rand((L, I), 1), rand((O, I), 2, std=I ** -0.5)
    x[5, 3], x[L - 1, I - 1] = INF, -INF
    y = call_linear(x.cuda(), w.cuda()).cpu()
    assert torch.equal(y[5], w[:, 3].sign() * INF) and torch.equal(y[L - 1], w[:, I - 1].sign() * -INF)
    y[5], y[L - 1] = 0.0, 0.0
    assert bool(torch.isfinite(y).all())


# ---- outputs stored with the streaming hint ---------------------------------------------------------------------------------------
# Those past 32 MB with rows of whole 128-byte lines.

def streams(rows, cols, size):
    return rows * cols * size > 2 ** 25 and cols * size % 128 == 0


def pieces(rows, cols, size):
    """Runs of rows that are not streamed."""
    step = 2 ** 25 // (cols * size)
    return [slice(a, min(a + step, rows)) for a in range(0, rows, step)]


def large_input(rows, cols, seed):
    """bfloat16 of unit spread; a group at the end of the type, whose values past 127 steps are held there, one past it, and a NaN."""
    x = torch.empty((rows, cols), device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(seed)).bfloat16()
    x[rows // 2, :32] = torch.linspace(-1.9921875, 1.9921875, 32).mul(2.0 ** 127).bfloat16().cuda()
    x[rows - 1, cols - 32] = 3.3e38
    x[1, 40], x[rows - 2, 5] = NAN, INF
    return x


def same(a, b):
    """Equal bits, or a NaN in both."""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7.0, 3.0e38, -3.0e38), b.nan_to_num(7.0, 3.0e38, -3.0e38))


@pytest.mark.parametrize("fn", FNS)
def test_streamed_activation(fn):
    """Value, checkpoint, its reading, gradient and bias sums of a large bfloat16 tensor: every row as in a call too small to be
    streamed, and rows from all over against 64 bits."""
    rows, cols, code = 8200, 2112, hot.ACT_FNS[fn]
    assert streams(rows, cols, 2) and not any(streams(p.stop - p.start, cols, 2) for p in pieces(rows, cols, 2))
    x, g = large_input(rows, cols, 1), torch.empty((rows, cols), device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(2)).bfloat16()
    y, back, gx, gx2, alone = (torch.full_like(x, 7.0) for _ in range(5))
    kept, gb, gb2, ws = hot.alloc_checkpoint(rows, cols), *(torch.empty(cols, device="cuda") for _ in range(2)), hot.alloc_activation_workspace(rows, cols)
    only = torch.zeros_like(kept)
    hot.hot_activation_forward(code, x, y, ckpt=kept)
    hot.hot_activation_forward(code, x, alone)
    hot.hot_checkpoint_write(x, only)
    hot.hot_checkpoint_read(kept, back)
    hot.hot_activation_backward(code, g, gx, ckpt=kept, g_bias=gb, ws=ws)
    hot.hot_activation_backward(code, g, gx2, x=x, g_bias=gb2, ws=ws)
    no_sums = hot.hot_activation_backward(code, g, torch.empty_like(g), ckpt=kept)
    assert torch.equal(only, kept) and same(alone, y) and same(no_sums, gx)
    sums, sums2 = torch.zeros(cols, dtype=torch.float64, device="cuda"), torch.zeros(cols, dtype=torch.float64, device="cuda")
    for p in pieces(rows, cols, 2):
        n = p.stop - p.start
        part, ckpt = torch.empty((n, cols), dtype=BF16, device="cuda"), hot.alloc_checkpoint(n, cols)
        xs, gs, half = x[p].contiguous(), g[p].contiguous(), torch.empty(cols, device="cuda")
        assert same(hot.hot_activation_forward(code, xs, part, ckpt=ckpt), y[p])
        assert same(hot.hot_checkpoint_read(ckpt, part), back[p])
        small = hot.alloc_activation_workspace(n, cols)
        assert same(hot.hot_activation_backward(code, gs, part, ckpt=ckpt, g_bias=half, ws=small), gx[p])
        sums += half.double()
        assert same(hot.hot_activation_backward(code, gs, part, x=xs, g_bias=half, ws=small), gx2[p])
        sums2 += half.double()
    # each side adds 8200 values of a column in fp32, at most 64 + 64 one after the other; |g_x| <= 1.13 |g_y|
    size = 1.13 * g.double().abs().sum(0).cpu()
    for got, want in ((gb, sums), (gb2, sums2)):
        close(got, want.cpu(), 2 * 128 * ref.U * size, "g_bias")
    at = torch.tensor([0, 1, 2, rows // 2, rows - 2, rows - 1] + list(range(17, rows, 400)))
    xs, gs = x[at.cuda()].cpu(), g[at.cuda()].cpu()
    values = ref.checkpoint(xs)[2]
    assert torch.equal(torch.isnan(ref.f64(back[at.cuda()])), torch.isnan(values))
    assert torch.equal(ref.f64(back[at.cuda()]).nan_to_num(7.0), values.nan_to_num(7.0))
    plain = (xs.float().abs() < 1e4).all(1)       # the formulas of the tolerances end far out
    want, tol = ref.act(fn, ref.f64(xs[plain]))
    close(y[at.cuda()][plain.cuda()], want, tol + 2.0 ** -8 * (want.abs() + tol), "y")
    want, tol, _, _ = ref.act_grad(fn, ref.f64(gs[plain]), values[plain], BF16)
    close(gx[at.cuda()][plain.cuda()], want, tol, "g_x")


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("rows,cols", [(140000, 128), (70000, 256), (33000, 512), (17000, 1024), (8200, 2112), (4200, 4096), (2100, 8192), (1600, 11008)])
def test_streamed_layer_norm_gradient(rows, cols, kept):
    """Every width of the kernel: rows as in calls too small to be streamed, sums and some rows against 64 bits."""
    assert streams(rows, cols, 2)
    g = torch.Generator("cuda").manual_seed(cols)
    make = lambda *s: torch.empty(s, device="cuda").normal_(generator=g)          # noqa: E731
    x, gy, gr, gamma, beta = make(rows, cols).bfloat16(), make(rows, cols).bfloat16(), make(rows, cols).bfloat16(), 1 + 0.2 * make(cols), make(cols)
    y, mean, rstd, buf = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), hot.alloc_checkpoint(rows, cols)
    hot.hot_layer_norm_forward(x, gamma, beta, 1e-6, y, mean, rstd, ckpt=buf)
    gx, gg, gb = torch.full_like(x, 7.0), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    args = dict(h=None if kept else x, ckpt=buf if kept else None)
    hot.hot_layer_norm_backward(gy, gamma, mean, rstd, gx, gg, gb, hot.alloc_layer_norm_workspace(rows, cols), g_residual=gr, **args)
    held = hot.hot_checkpoint_read(buf, torch.empty_like(x)) if kept else x
    n = (held.double() - mean.double()[:, None]) * rstd.double()[:, None]
    # at most 1024 rows one after the other in a workgroup's sum, 32 + 5 of those; three roundings an element
    for got, terms in ((gg, gy.double() * n), (gb, gy.double())):
        close(got, terms.sum(0).cpu(), 1100 * ref.U * terms.abs().sum(0).cpu(), "sums")
    for p in pieces(rows, cols, 2):
        m = p.stop - p.start
        some = dict(h=None if kept else x[p].contiguous(), ckpt=None)
        if kept:
            some["ckpt"] = hot.hot_checkpoint_write(x[p].contiguous(), hot.alloc_checkpoint(m, cols))
        part = hot.hot_layer_norm_backward(gy[p].contiguous(), gamma, mean[p].clone(), rstd[p].clone(), torch.empty((m, cols), dtype=BF16, device="cuda"),
                                           g_residual=gr[p].contiguous(), **some)
        assert torch.equal(part, gx[p])
    at = torch.arange(0, rows, rows // 13, device="cuda")
    wx, _, _ = ref.norm_grad(ref.f64(gy[at]), ref.f64(held[at]), ref.f64(gamma), ref.f64(mean[at]), ref.f64(rstd[at]), ref.f64(gr[at]), BF16)
    close(gx[at], *wx, "g_x")


STREAMED = [
    (BF16, "direct", 8344, 2048, 64), (BF16, "direct", 26637, 640, 8), (BF16, "direct", 267070, 64, 64), (BF16, "direct", 16570, 1024, 8),
    (BF16, "packed", 65757, 320, 773), (BF16, "packed", 2130, 8192, 9), (BF16, "packed", 33352, 512, 707), (BF16, "packed", 128623, 192, 79),
    (BF16, "tiles", 26606, 640, 1074), (BF16, "tiles", 177597, 128, 64), (BF16, "tiles", 195187, 128, 10), (BF16, "tiles", 22519, 768, 1088),
    (BF16, "tiles", 66646, 256, 712), (BF16, "tiles", 123516, 192, 256), (BF16, "tiles", 131018, 192, 186),
    (F32, "direct", 1051, 8192, 32), (F32, "direct", 11037, 768, 8), (F32, "direct", 265528, 32, 32), (F32, "direct", 16560, 512, 8),
    (F32, "packed", 16634, 512, 1663), (F32, "packed", 1541, 8192, 8), (F32, "packed", 65543, 192, 482), (F32, "packed", 64792, 192, 33)]


@pytest.mark.parametrize("t,way,L,O,I", STREAMED)
def test_streamed_linear(t, way, L, O, I):
    """Bias, activation, residual and checkpoint behind a large product, one row of which reaches the end of the type."""
    p = hot.hot_debug_linear_plan(t, L, O, I, ckpt=True)
    print(f"[streamed] {L}x{O}x{I} {t} {p}", flush=True)
    assert p["streams"] and p["way"] == way
    g = torch.Generator("cuda").manual_seed(L + O)
    make = lambda *s: torch.empty(s, device="cuda").normal_(generator=g)          # noqa: E731
    x, w, b, r = make(L, I).to(t), (make(O, I) * I ** -0.5).to(t), make(O), make(L, O).to(t)
    far = L - 3                              # its first 32 outputs are +-255 x 2^120, 127.5 steps; no other row has its column
    x[:, 0], x[far], w[:, 0] = 0.0, 0.0, 0.0
    x[far, 0] = 2.0 ** 64
    w[:32, 0] = (torch.arange(32, device="cuda") % 2 * 2.0 - 1).to(t) * 1.9921875 * 2.0 ** 63
    kept, y, y0 = hot.alloc_checkpoint(L, O), torch.full((L, O), NAN, dtype=t, device="cuda"), torch.full((L, O), NAN, dtype=t, device="cuda")
    ws = hot.alloc_linear_workspace(t, L, O, I)
    hot.hot_linear_forward(x, w, y, ws, bias=b, residual=r, fn=hot.HOT_ACT_SILU, ckpt=kept)
    hot.hot_linear_forward(x, w, y0, ws)
    z, size = product64(x, w)
    half = ref.HALF[t]
    d0 = 26 * ref.U * size + (2 * I + 1) * 2.0 ** -150
    close(y0, z, d0 + half * (z.abs() + d0), "bare y")
    z = z + ref.f64(b)
    dz = d0 + ref.U * z.abs()
    want, dy = ref.act("silu", z)
    dy = dy + 1.2 * dz
    want, dy = want + ref.f64(r), dy + 2 * ref.U * (want.abs() + ref.f64(r).abs())
    # far out the formula of the activation's error has infinity times zero: the value is z or 0 there
    far_out = z.abs() > 1e4
    dy = torch.where(far_out, dz + 4 * ref.U * z.abs(), dy)
    close(y, want, dy + half * (want.abs() + dy), "y")
    back = torch.empty((L, O), device="cuda")
    back = ref.f64(hot.hot_checkpoint_read(kept, back))
    step = (z.abs() + dz).view(L, -1, 32).amax(-1).clamp(min=2.0 ** -118) / 63.75
    close(back, z, dz + step.repeat_interleave(32, 1) / 2, "z of the checkpoint")
    assert torch.equal(back[far, :32], (torch.arange(32) % 2 * 2.0 - 1).double() * 127 * 2.0 ** 121)


def test_streamed_tensors_past_32_bits():
    """Elements past 2^32 in rows of whole lines: the last rows give what they give in a call of their own."""
    rows, cols = 2 ** 17 + 6, 2 ** 15 + 256
    assert streams(rows, cols, 2) and streams(rows * 4, cols // 4, 2) and rows * cols > 2 ** 32
    x = torch.empty((rows, cols), dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    tail = x[-7:].contiguous()
    y, kept, y7, kept7 = torch.empty_like(x), hot.alloc_checkpoint(rows, cols), torch.empty_like(tail), hot.alloc_checkpoint(7, cols)
    hot.hot_activation_forward(hot.HOT_ACT_GELU, x, y, ckpt=kept)
    hot.hot_activation_forward(hot.HOT_ACT_GELU, tail, y7, ckpt=kept7)
    assert torch.equal(y[-7:], y7)
    back, back7 = torch.empty_like(x), torch.empty_like(tail)
    hot.hot_checkpoint_read(kept, back)
    hot.hot_checkpoint_read(kept7, back7)
    assert torch.equal(back[-7:], back7)
    hot.hot_activation_backward(hot.HOT_ACT_GELU, y, back, ckpt=kept)
    hot.hot_activation_backward(hot.HOT_ACT_GELU, y7, back7, ckpt=kept7)
    assert torch.equal(back[-7:], back7)
    mean, rstd, mean7, rstd7 = (torch.empty(n, device="cuda") for n in (rows * 4, rows * 4, 28, 28))
    x, tail = x.view(rows * 4, cols // 4), tail.view(28, cols // 4)
    y, y7, gx, gx7 = y.view_as(x), y7.view_as(tail), back.view_as(x), back7.view_as(tail)
    hot.hot_layer_norm_forward(x, None, None, 1e-6, y, mean, rstd)
    hot.hot_layer_norm_forward(tail, None, None, 1e-6, y7, mean7, rstd7)
    hot.hot_layer_norm_backward(y, None, mean, rstd, gx, h=x)
    hot.hot_layer_norm_backward(y7, None, mean7, rstd7, gx7, h=tail)
    assert torch.equal(y[-28:], y7) and torch.equal(mean[-28:], mean7) and torch.equal(gx[-28:], gx7)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs a second device")
def test_large_tiles_on_a_second_device():
    """Kernels that take more LDS than a launch may by itself, on one device of a process after another."""
    x, w = rand((3500, 100), 1), rand((3600, 100), 2)
    for device in ("cuda:0", "cuda:1"):
        with torch.cuda.device(device):
            y = torch.empty((3500, 3600), device=device)
            hot.hot_linear_forward(x.to(device), w.to(device), y, hot.alloc_linear_workspace(F32, 3500, 3600, 100, device=device))
            held_to(y, *product64(x.to(device), w.to(device)), 100, device)


def test_gelu_tanh_slope_keeps_its_tail():
    """1 - sigmoid is small beside 1 from x = 3 on and meets a large factor.  In units u = 2^-24: the argument and its exponential are off by
    4 u |arg|, which the sigmoid s takes times s (1 - s), the product x s (1 - s) arg' relative to itself; three roundings of s (a reciprocal
    and a sum), eight of the product, one of each sum."""
    x = torch.linspace(-9.9, 9.9, 20000).view(20, 1000)
    got = hot.hot_activation_backward(hot.HOT_ACT_GELU_TANH, torch.ones_like(x).cuda(), torch.empty_like(x, device="cuda"), x=x.cuda())
    X = ref.f64(x)
    arg, up = ref._tanh_arg(X)
    s, r = torch.sigmoid(arg), torch.sigmoid(-arg)
    want, product = ref.act_slope("gelu_tanh", X)[0], (X * up * s * r).abs()
    close(got, want, ref.U * (4 * arg.abs() * s * r + 3 * s + product * (4 * arg.abs() + 8) + 2 * want.abs()) + 2.0 ** -100, "slope")


@pytest.mark.parametrize("L,O,I,tile,cut", PACKED)
def test_packed_product_recorded_on_rows_of_other_ranges(L, O, I, tile, cut):
    """Which instructions a tile takes is decided anew on every replay: ordinary rows, wide ones, infinities, ordinary ones again, each as
    eager calls give them and near the exact product."""
    packed(L, O, I, tile, cut)
    x, w, ws = rand((L, I), 1).cuda(), rand((O, I), 2, std=I ** -0.5).cuda(), hot.alloc_linear_workspace(F32, L, O, I)
    w[:, 0] = 0.0
    first, y, eager = x.clone(), torch.empty((L, O), device="cuda"), torch.empty((L, O), device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hot.hot_linear_forward(x, w, y, ws)
    seen = []
    for scale in (1.0, 2.0 ** 24, INF, 1.0):
        x.copy_(first)
        if scale == INF:
            x[L // 2, 1] = INF
        else:
            x[L // 3:, 0] *= scale
        y.fill_(NAN)
        graph.replay()
        hot.hot_linear_forward(x, w, eager, ws)
        torch.cuda.synchronize()
        assert same(y, eager), scale
        if scale != INF:
            held_to(y, *product64(x, w), I, f"scale {scale}")
        seen.append(y.clone())
    assert torch.equal(seen[0], seen[3]) and not torch.equal(seen[0], seen[1])


@pytest.mark.parametrize("wide_x", [True, False])
@pytest.mark.parametrize("L,O,I,tile,cut", PACKED)
def test_packed_whole_numbers_far_below_their_rows_largest(L, O, I, tile, cut, wide_x):
    """Twelve bits beside a column of 2^30, whose factor is zero: the low part of each is a subnormal 16-bit number, and all of them count.
    Products and sums are whole and within 2^24 (twenty standard deviations), so there is one result."""
    packed(L, O, I, tile, cut)
    g = torch.Generator("cuda").manual_seed(I)
    sign = lambda *s: torch.randint(0, 2, s, generator=g, device="cuda", dtype=F32) * 2 - 1          # noqa: E731
    x, w = sign(L, I), sign(O, I)
    far, near = (x, w) if wide_x else (w, x)
    far *= 2049 + 2 * torch.randint(0, 1024, far.shape, generator=g, device="cuda", dtype=F32)
    far[:, I // 3], near[:, I // 3] = 2.0 ** 30, 0.0
    want = x.double() @ w.double().t().contiguous()
    assert float(want.abs().max()) < 2 ** 24
    assert torch.equal(call_linear(x, w).double(), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("cols", [40, 100, 200, 500, 771, 1500, 4096, 5000, 11008])
def test_layer_norm_rows_with_an_infinity_or_nan_stay_alone(cols, kept, dtype):
    """Rows that share a workgroup with them give the bits that they give beside rows of zeros; theirs are NaN, and so are the sums over rows."""
    rows, bad = 50, [2, 17, 49]
    x, g = rand((rows, cols), cols, dtype), rand((rows, cols), 1, dtype)
    x[2, 0], x[17, cols - 1], x[49, cols // 2] = NAN, INF, -INF
    clean = x.clone()
    clean[bad] = 0.0
    outs = []
    for t in (x.cuda(), clean.cuda()):
        y, mean, rstd, gx = torch.empty_like(t), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(t)
        gg, gb, buf = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda"), hot.alloc_checkpoint(rows, cols)
        hot.hot_layer_norm_forward(t, None, None, 1e-5, y, mean, rstd, ckpt=buf)
        hot.hot_layer_norm_backward(g.cuda(), None, mean, rstd, gx, gg, gb, hot.alloc_layer_norm_workspace(rows, cols),
                                    h=None if kept else t, ckpt=buf if kept else None)
        outs.append((y, mean, rstd, gx, hot.hot_checkpoint_read(buf, torch.empty_like(t)), gg, gb))
    fine = torch.ones(rows, dtype=torch.bool, device="cuda")
    fine[bad] = False
    for a, b in zip(outs[0][:5], outs[1][:5]):
        assert torch.equal(a[fine], b[fine]) and bool(torch.isfinite(b).all())
    y, mean, rstd, gx, back, gg, gb = outs[0]
    assert bool(y[bad].isnan().all()) and bool(gx[bad].isnan().all()) and not bool(torch.isfinite(mean[bad]).any())
    assert int(back.isnan().sum()) == sum(min(32, cols - c // 32 * 32) for c in (0, cols - 1, cols // 2))
    assert bool(gg.isnan().all()) and torch.equal(gb, outs[1][6])
