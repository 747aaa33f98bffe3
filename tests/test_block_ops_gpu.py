"""The operators around the linear backward on the GPU, each against its 64-bit form: 8-bit checkpoints, activations, layer norm,
forward product, and a run of them together with the linear backward."""
import numpy as np
import pytest
import torch

import block_oracle as ref
import paper_2503_21261_amd as hot

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
FNS = ["relu", "gelu", "gelu_tanh", "silu"]


def rand(shape, seed, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype)


class Guarded:
    """An output with a guard on both sides, which has to come back as it was."""

    def __init__(self, shape, dtype=F32):
        n = int(np.prod(shape))
        size = torch.empty(0, dtype=dtype).element_size()
        self.bytes = -(-n * size // 256) * 256
        self.raw = torch.full((512 + self.bytes + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        self.t = self.raw[512:512 + n * size].view(dtype).view(shape)
        self.used = n * size

    def check(self):
        assert bool((self.raw[:512] == 0xA5).all()) and bool((self.raw[512 + self.used:] == 0xA5).all()), "written out of bounds"


def close(got, want, tol, what):
    got = ref.f64(got)
    assert got.shape == want.shape, what
    same_nan = torch.isnan(got) == torch.isnan(want)
    assert bool(same_nan.all()), f"{what}: NaN elsewhere"
    off = (got - want).abs() - tol
    off = torch.where(torch.isnan(off), torch.full_like(off, -1.0), off)
    assert float(off.max()) <= 0, f"{what}: off by {float((got - want).abs().flatten()[off.argmax()])} at {int(off.argmax())}, " \
                                  f"{float(tol.flatten()[off.argmax()])} allowed"


def read_checkpoint(buf, rows, cols):
    pitch, exps, total = ref.checkpoint_layout(rows, cols)
    raw = buf.cpu().numpy()
    assert raw.size == total
    return raw[:rows * pitch].view(np.int8).reshape(rows, pitch), raw[exps:].reshape(rows, pitch // 32)


def check_checkpoint(buf, t):
    rows, cols = t.shape
    codes, exps = read_checkpoint(buf, rows, cols)
    want_codes, want_exps, values = ref.checkpoint(t)
    assert np.array_equal(exps, want_exps)
    fine = np.repeat(want_exps != 255, 32, axis=1)
    assert np.array_equal(codes[fine], want_codes[fine])
    return values


# ---- 8-bit checkpoint -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (5, 7), (2, 64), (197, 768), (64, 771), (9, 100), (2, 16385),
                                       (1000, 40), (1, 11008)])
def test_checkpoint_is_exact(rows, cols, dtype):
    print(f"[checkpoint] {rows}x{cols} {dtype}", flush=True)
    x = rand((rows, cols), rows * 7 + cols, dtype)
    x[:, ::5] *= 30
    buf = Guarded((hot.hot_checkpoint_bytes(rows, cols),), torch.uint8)
    back = Guarded((rows, cols), dtype)
    hot.hot_checkpoint_write(x.cuda(), buf.t)
    hot.hot_checkpoint_read(buf.t, back.t)
    torch.cuda.synchronize()
    values = check_checkpoint(buf.t, x)
    buf.check(), back.check()
    assert torch.equal(ref.f64(back.t), values)
    other = torch.empty((rows, cols), dtype=BF16 if dtype == F32 else F32, device="cuda")     # either type reads it exactly
    assert torch.equal(ref.f64(hot.hot_checkpoint_read(buf.t, other)), values)


def test_checkpoint_of_special_values():
    """Ties, the smallest and largest steps, groups of zeros, subnormals, and one bad element: its group alone is lost."""
    x = torch.zeros(12, 96)
    x[0, :32] = torch.arange(32) * 0.5 + 0.5             # ties
    x[0, 0] = 127.0
    x[1, :4] = torch.tensor([127.49, -127.5, 126.5, 0.5])
    x[2, :3] = torch.tensor([3.4028e38, -3.0e38, 1.0])
    x[3, :3] = torch.tensor([3.4028234e38, 1.6e36, -1.3e36])
    x[4, :3] = torch.tensor([1e-36, 3e-38, -1e-38])
    x[5, :3] = torch.tensor([1e-40, -1e-45, 2.4e-38])
    x[6, 5], x[6, 40], x[6, 70] = float("inf"), 1.0, 2.0
    x[7, 6], x[7, 41] = float("nan"), -3.0
    x[8, 7], x[8, 33] = float("-inf"), 5.0
    x[9] = -0.0
    x[10] = 2.0 ** -120
    x[11, 31], x[11, 32] = 1.9921875, 1.9921874
    buf = hot.alloc_checkpoint(12, 96)
    hot.hot_checkpoint_write(x.cuda(), buf)
    values = check_checkpoint(buf, x)
    back = ref.f64(hot.hot_checkpoint_read(buf, torch.empty((12, 96), device="cuda")))
    assert torch.equal(torch.isnan(back), torch.isnan(values))
    assert torch.equal(back.nan_to_num(7.0), values.nan_to_num(7.0))
    assert int(torch.isnan(back).sum()) == 3 * 32


# ---- activations ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("fn", FNS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 33), (197, 768), (70, 771), (1, 4096), (333, 100)])
def test_activation_and_gradient(rows, cols, fn, dtype):
    print(f"[activation] {fn} {rows}x{cols} {dtype}", flush=True)
    seed = rows + cols
    x, g = rand((rows, cols), seed, dtype, 2.0), rand((rows, cols), seed + 1, dtype, 1e-3)
    x[0, 0] = 0.0
    xd, gd = x.cuda(), g.cuda()
    y, gx, gx2 = (Guarded((rows, cols), dtype) for _ in range(3))
    gb, gb2 = Guarded((cols,)), Guarded((cols,))
    buf = Guarded((hot.hot_checkpoint_bytes(rows, cols),), torch.uint8)
    ws = Guarded((hot.hot_activation_backward_workspace_bytes(rows, cols),), torch.uint8)
    code = hot.ACT_FNS[fn]
    hot.hot_activation_forward(code, xd, y.t, ckpt=buf.t)
    hot.hot_activation_backward(code, gd, gx.t, ckpt=buf.t, g_bias=gb.t, ws=ws.t)
    hot.hot_activation_backward(code, gd, gx2.t, x=xd, g_bias=gb2.t, ws=ws.t)
    plain = hot.hot_activation_backward(code, gd, torch.empty_like(gd), x=xd)
    alone = hot.hot_activation_forward(code, xd, torch.empty_like(xd))
    torch.cuda.synchronize()
    for b in (y, gx, gx2, gb, gb2, buf, ws):
        b.check()
    assert torch.equal(plain, gx2.t) and torch.equal(alone, y.t)
    values = check_checkpoint(buf.t, x)
    want, tol = ref.act(fn, ref.f64(x))
    close(y.t, want, tol + ref.HALF[dtype] * (want.abs() + tol), "y")
    for got, got_bias, at in ((gx.t, gb.t, values), (gx2.t, gb2.t, ref.f64(x))):
        want, tol, bias, btol = ref.act_grad(fn, ref.f64(g), at, dtype)
        close(got, want, tol, "g_x")
        close(got_bias, bias, btol, "g_bias")


@pytest.mark.parametrize("fn", FNS)
def test_activation_far_out_and_not_finite(fn):
    x = torch.tensor([[0.0, -0.0, 1e-30, -1e-30, 20.0, -20.0, 88.0, -88.0, 1e4, -1e4, 1e20, -1e20, 3e38, -3e38, float("nan"), 1.0]])
    xd = x.cuda()
    y = ref.f64(hot.hot_activation_forward(hot.ACT_FNS[fn], xd, torch.empty_like(xd)))
    g = ref.f64(hot.hot_activation_backward(hot.ACT_FNS[fn], torch.ones_like(xd), torch.empty_like(xd), x=xd))
    x = ref.f64(x)[:, :14]
    assert bool(torch.isnan(y[0, 14])) and not bool(torch.isnan(y[0, 15]))
    want, tol = ref.act(fn, x)
    close(y[:, :14], want, tol + 1e-36, "y")
    slope, tol = ref.act_slope(fn, x)
    slope = torch.where(x == 0, torch.full_like(slope, 0.0 if fn == "relu" else 0.5), slope)
    far = x.abs() >= 88      # the formulas of the tolerance meet infinity times zero there: the slope is 0 or 1
    want = torch.where(far, (x > 0).double(), slope)
    close(g[:, :14], want, torch.where(far, torch.full_like(tol, 1e-4), tol), "slope")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("fn", FNS)
def test_activation_of_an_infinity(fn, dtype):
    """f(+inf) is +inf, by itself and behind a product; a NaN stays one and the values beside them finite."""
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[inf, 2.0, nan, 3.0] * 4], dtype=dtype)
    y = torch.empty_like(x, device="cuda")
    hot.hot_activation_forward(getattr(hot, "HOT_ACT_" + fn.upper()), x.cuda(), y)
    want = torch.tensor([[inf, 0.0, nan, 0.0] * 4])
    got = torch.where(torch.isfinite(y.cpu().float()), torch.zeros(1), y.cpu().float())
    assert torch.equal(got.nan_to_num(7.0, posinf=9.0, neginf=-9.0), want.nan_to_num(7.0, posinf=9.0, neginf=-9.0))
    if dtype == BF16:        # bfloat16 products are exact: an infinity is one
        a, w = torch.full((3, 64), 1.0, dtype=dtype), torch.ones((4, 64), dtype=dtype)
        a[1, 0] = inf
        z = torch.empty((3, 4), dtype=dtype, device="cuda")
        hot.hot_linear_forward(a.cuda(), w.cuda(), z, hot.alloc_linear_workspace(dtype, 3, 4, 64), fn=getattr(hot, "HOT_ACT_" + fn.upper()))
        assert bool((z[1] == inf).all()) and bool(torch.isfinite(z[0::2]).all())


def test_bias_sums_alone_take_no_activation():
    g = rand((500, 200), 3)
    gb, gx = torch.empty(200, device="cuda"), torch.empty((500, 200), device="cuda")
    hot.hot_activation_backward(hot.HOT_ACT_NONE, g.cuda(), gx, x=g.cuda(), g_bias=gb, ws=hot.alloc_activation_workspace(500, 200))
    assert torch.equal(gx.cpu(), g)
    close(gb, ref.f64(g).sum(0), 128 * ref.U * ref.f64(g).abs().sum(0), "g_bias")


# ---- layer norm ---------------------------------------------------------------------------------------------------------

def run_norm(rows, cols, tx, ty, residual, kept, affine=True, eps=1e-6, seed=0, x=None):
    print(f"[norm] {rows}x{cols} {tx} {ty} residual={residual} kept={kept}", flush=True)
    x = rand((rows, cols), seed, tx) if x is None else x
    if cols > 5:
        x[:, 5] = x[:, 5] * 20
    r = rand((rows, cols), seed + 1, tx) if residual else None
    gamma = 1 + rand((cols,), seed + 2, std=0.2) if affine else None
    beta = rand((cols,), seed + 3, std=0.1) if affine else None
    dev = lambda t: None if t is None else t.cuda()       # noqa: E731
    y, mean, rstd = Guarded((rows, cols), ty), Guarded((rows,)), Guarded((rows,))
    h = Guarded((rows, cols), tx) if residual else None
    buf = Guarded((hot.hot_checkpoint_bytes(rows, cols),), torch.uint8) if kept else None
    hot.hot_layer_norm_forward(dev(x), dev(gamma), dev(beta), eps, y.t, mean.t, rstd.t, residual=dev(r), h=h and h.t, ckpt=buf and buf.t)
    torch.cuda.synchronize()
    for b in (y, mean, rstd, h, buf):
        if b:
            b.check()
    held = x if r is None else (x.float() + r.float()).to(tx)
    if residual:
        assert torch.equal(h.t.cpu(), held)
    h64 = ref.f64(held)
    d64 = lambda t: None if t is None else ref.f64(t)     # noqa: E731
    wy, wm, wr = ref.norm(h64, d64(gamma), d64(beta), eps, ty)
    close(mean.t, *wm, "mean")
    close(rstd.t, *wr, "rstd")
    close(y.t, *wy, "y")
    g = rand((rows, cols), seed + 4, ty, 1e-3)
    ga = rand((rows, cols), seed + 5, tx, 1e-3) if residual else None
    gx, gg, gb = Guarded((rows, cols), tx), Guarded((cols,)), Guarded((cols,))
    ws = Guarded((hot.hot_layer_norm_backward_workspace_bytes(rows, cols),), torch.uint8)
    args = dict(h=None if kept else dev(held), ckpt=buf and buf.t, g_residual=dev(ga))
    hot.hot_layer_norm_backward(dev(g), dev(gamma), mean.t, rstd.t, gx.t, gg.t, gb.t, ws.t, **args)
    alone = hot.hot_layer_norm_backward(dev(g), dev(gamma), mean.t, rstd.t, torch.empty_like(gx.t), **args)
    torch.cuda.synchronize()
    for b in (gx, gg, gb, ws):
        b.check()
    assert torch.equal(alone, gx.t)
    at = check_checkpoint(buf.t, held) if kept else h64
    wx, wg, wb = ref.norm_grad(ref.f64(g), at, d64(gamma), ref.f64(mean.t), ref.f64(rstd.t), d64(ga), tx)
    close(gx.t, *wx, "g_x")
    close(gg.t, *wg, "g_gamma")
    close(gb.t, *wb, "g_beta")


@pytest.mark.parametrize("cols", [1, 7, 32, 64, 128, 129, 200, 256, 300, 512, 513, 768, 771, 1024, 1025, 1500, 2048, 3000, 4096, 5000,
                                  8192, 11008, 16383, 16384])
def test_layer_norm_every_width(cols):
    kept = cols % 2 == 0
    run_norm(37, cols, F32, F32, residual=cols % 3 == 0, kept=kept, seed=cols)


@pytest.mark.parametrize("tx,ty", [(F32, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("rows,cols", [(1, 768), (197, 100), (5, 771), (66, 4099)])
def test_layer_norm_types_and_forms(rows, cols, tx, ty, residual, kept):
    run_norm(rows, cols, tx, ty, residual, kept, seed=rows)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 1023, 2049, 4100])
def test_layer_norm_row_counts(rows):
    run_norm(rows, 96, F32, F32, False, True, seed=rows)


def test_layer_norm_without_gamma_and_beta():
    run_norm(50, 320, F32, F32, True, False, affine=False)


def test_layer_norm_far_mean_and_constant_rows():
    x = rand((8, 1000), 5)
    x[0] += 1e4
    x[1] = x[1] * 1e-3 - 300
    x[2] = 7.3
    x[3] = 0.0
    x[4] *= 1e15
    x[5] *= 1e-15
    run_norm(8, 1000, F32, F32, False, False, x=x, eps=1e-5, seed=5)


def test_layer_norm_gradients_against_differences():
    rows, cols, eps = 6, 80, 1e-5
    x, gamma, beta, g = rand((rows, cols), 1), 1 + rand((cols,), 2, std=0.2), rand((cols,), 3), rand((rows, cols), 4)
    y, mean, rstd = torch.empty((rows, cols), device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    hot.hot_layer_norm_forward(x.cuda(), gamma.cuda(), beta.cuda(), eps, y, mean, rstd)
    gx, gg, gb = torch.empty_like(y), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    hot.hot_layer_norm_backward(g.cuda(), gamma.cuda(), mean, rstd, gx, gg, gb, hot.alloc_layer_norm_workspace(rows, cols), h=x.cuda())
    X, G, B, W = ref.f64(x), ref.f64(gamma), ref.f64(beta), ref.f64(g)

    def loss(a, b, c):
        return float((ref.norm(a, b, c, eps, F32)[0][0] * W).sum())

    for seed in range(4):
        for got, at in ((gx, 0), (gg, 1), (gb, 2)):
            v = ref.f64(rand(got.shape, 50 + seed))
            step = 1e-5
            plus, minus = [X, G, B], [X, G, B]
            plus[at], minus[at] = plus[at] + step * v, minus[at] - step * v
            want = (loss(*plus) - loss(*minus)) / (2 * step)
            # the difference quotient is right to step^2 and 1e-16 / step; the gradient to some hundred u of its terms
            assert abs(float((ref.f64(got) * v).sum()) - want) <= 2e-5 * float((ref.f64(got) * v).abs().sum()) + 1e-8


@pytest.mark.parametrize("fn", FNS)
def test_activation_gradients_against_differences(fn):
    x = rand((4, 64), 9)
    x[x.abs() < 1e-3] = 0.5          # away from relu's corner
    gx = hot.hot_activation_backward(hot.ACT_FNS[fn], torch.ones(4, 64).cuda(), torch.empty((4, 64), device="cuda"), x=x.cuda())
    X, step = ref.f64(x), 1e-5
    want = (ref.act(fn, X + step)[0] - ref.act(fn, X - step)[0]) / (2 * step)
    close(gx, want, torch.full_like(want, 2e-6), "slope")


# ---- forward product -----------------------------------------------------------------------------------------------------

def run_linear(L, O, I, tx, ty, fn="none", bias=True, residual=False, kept=False, seed=0, scale=None):
    print(f"[linear] {L}x{O}x{I} {tx} {ty} {fn} bias={bias} residual={residual} kept={kept}", flush=True)
    x, w = rand((L, I), seed, tx), rand((O, I), seed + 1, tx, I ** -0.5)
    if scale is not None:
        scale(x, w)
    b = rand((O,), seed + 2, std=0.3) if bias else None
    r = rand((L, O), seed + 3, ty) if residual else None
    dev = lambda t: None if t is None else t.cuda()       # noqa: E731
    y = Guarded((L, O), ty)
    buf = Guarded((hot.hot_checkpoint_bytes(L, O),), torch.uint8) if kept else None
    need = hot.hot_linear_forward_workspace_bytes(tx, L, O, I)
    ws = Guarded((need,), torch.uint8) if need else None
    xd, wd = dev(x), dev(w)
    hot.hot_linear_forward(xd, wd, y.t, ws and ws.t, bias=dev(b), residual=dev(r), fn=hot.ACT_FNS[fn], ckpt=buf and buf.t)
    torch.cuda.synchronize()
    for g in (y, buf, ws):
        if g:
            g.check()
    assert torch.equal(xd.cpu(), x) and torch.equal(wd.cpu(), w)
    d64 = lambda t: None if t is None else ref.f64(t)     # noqa: E731
    wy, (z, dz) = ref.linear(d64(x), d64(w), d64(b), fn, d64(r), ty)
    close(y.t, *wy, "y")
    if kept:
        codes, exps = read_checkpoint(buf.t, L, O)
        assert not codes[:, O:].any()
        step = torch.from_numpy(np.repeat(2.0 ** (exps.astype(np.float64) - 133), 32, axis=1)[:, :O].copy())
        close(torch.from_numpy(codes[:, :O].astype(np.float64)) * step, z, step / 2 + dz, "z of the checkpoint")
        # the step is the group's: its largest value reaches past 63 steps, but for the smallest step of all
        pad = torch.zeros(L, codes.shape[1], dtype=torch.float64)
        pad[:, :O] = z.abs() + dz
        top = pad.view(L, -1, 32).amax(-1)
        assert bool((top >= 63.5 * 2.0 ** (torch.from_numpy(exps.astype(np.float64)) - 133)).logical_or(torch.from_numpy(exps == 8)).all())
    return y.t


LINEAR_SHAPES = [(1, 1, 1), (1, 16, 8), (3, 7, 5), (16, 33, 31), (17, 64, 100), (33, 100, 129), (64, 768, 64), (65, 48, 1000), (1, 4096, 512),
                 (197, 768, 768), (300, 771, 333), (130, 260, 2048)]


@pytest.mark.parametrize("tx,ty", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("L,O,I", LINEAR_SHAPES)
def test_linear_shapes(L, O, I, tx, ty):
    run_linear(L, O, I, tx, ty, seed=L + O + I)
    run_linear(L, O, I, tx, ty, fn="gelu", bias=False, residual=True, kept=True, seed=L + O + I + 1)


@pytest.mark.parametrize("fn", FNS)
@pytest.mark.parametrize("tx,ty", [(F32, F32), (BF16, BF16)])
def test_linear_epilogues(fn, tx, ty):
    for L in (5, 600):
        for residual in (False, True):
            for kept in (False, True):
                run_linear(L, 200, 160, tx, ty, fn, True, residual, kept, seed=L)


@pytest.mark.parametrize("tx,ty", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("L,O,I", [(3500, 3600, 100), (3590, 3585, 33), (66, 70, 1), (66, 70, 16), (66, 70, 17), (66, 70, 32), (66, 70, 48),
                                   (66, 70, 64), (129, 129, 80), (1000, 31, 96)])
def test_linear_tiles(L, O, I, tx, ty):
    run_linear(L, O, I, tx, ty, seed=L + I)
    run_linear(L, O, I, tx, ty, fn="silu", bias=False, residual=True, kept=True, seed=L + I + 1)


@pytest.mark.parametrize("L", [7, 90])
def test_linear_rows_of_any_magnitude(L):
    """Each row of either operand has a scale of its own, from the smallest to the largest; rows of zeros; within a row,
    values far below its largest."""

    def scale(x, w):
        x *= (2.0 ** torch.linspace(-62, 60, x.shape[0]).round())[:, None]
        w *= (2.0 ** torch.linspace(-62, 60, w.shape[0]).round())[:, None]
        x[:, ::3] *= 2.0 ** -20
        x[3], w[5] = 0.0, 0.0
        x[4] = 0.0
        x[4, 7] = 1e-40

    run_linear(L, 77, 200, F32, F32, bias=False, scale=scale)


def test_linear_rows_with_an_infinity_or_nan_stay_alone():
    for tx in (F32, BF16):
        for L in (6, 100):
            x, w = rand((L, 96), 1, tx), rand((80, 96), 2, tx)
            x[2, 5], x[4, 90], w[7, 1] = float("nan"), float("inf"), float("nan")
            y = torch.empty((L, 80), dtype=tx, device="cuda")
            hot.hot_linear_forward(x.cuda(), w.cuda(), y, hot.alloc_linear_workspace(tx, L, 80, 96))
            bad = ~torch.isfinite(y.cpu().float())
            want = torch.zeros(L, 80, dtype=torch.bool)
            want[2], want[4], want[:, 7] = True, True, True
            assert torch.equal(bad, want)


# Shapes for each way a product is worked on: few rows (16 or 32 outputs and 16 to 64 tokens a workgroup), operands as they are in
# tiles of 64 x 64 and 32 x 128 (rows of a multiple of 16, 4 or 2 bytes), in tiles of 128 x 128 and 256 x 256 packed, as they are and as
# they are with a last piece to mask; each with whole tiles and in slices of K, the large tiles also with slices for the last ones alone.
LINEAR_WAYS = [
    (BF16, 522, 1909, 8), (BF16, 3, 112, 5000), (BF16, 50, 90, 88), (BF16, 1, 9, 4776), (BF16, 40, 600, 6000), (BF16, 9, 33, 4103),
    (BF16, 17, 2342, 11), (BF16, 477, 17, 7907), (BF16, 4153, 38, 9), (BF16, 3017, 8, 4995), (BF16, 5, 4188, 11), (BF16, 1, 843, 7536),
    (BF16, 7772, 21, 9), (BF16, 50, 518, 5285), (BF16, 14813, 18, 15), (BF16, 33, 1012, 7331), (BF16, 10082, 165, 9),
    (BF16, 594, 124, 2211), (BF16, 14578, 963, 9), (BF16, 9837, 143, 7617), (BF16, 11683, 1514, 1010),
    (F32, 203, 4471, 16), (F32, 1, 4453, 3756), (F32, 14198, 9, 8), (F32, 859, 36, 4952), (F32, 11, 24, 3004), (F32, 2140, 19, 8),
    (F32, 536, 17, 3361), (F32, 14418, 9, 11), (F32, 1650, 8, 5097), (F32, 3, 4787, 8), (F32, 1, 1079, 3448), (F32, 3083, 56, 9),
    (F32, 602, 17, 7289), (F32, 1880, 254, 11), (F32, 2771, 17, 4114), (F32, 6353, 238, 9), (F32, 2099, 113, 1775),
    (F32, 6742, 1245, 2568), (F32, 6375, 2284, 40), (F32, 7329, 162, 5528), (F32, 5054, 3202, 528),
    (BF16, 7, 82, 4826), (BF16, 645, 2964, 15), (BF16, 194, 4334, 12), (BF16, 11, 14, 4948), (BF16, 1, 8, 10), (BF16, 1658, 589, 3393),
    (BF16, 18181, 4024, 9), (BF16, 1017, 2625, 6699), (BF16, 6994, 2160, 129), (BF16, 11102, 1516, 1081), (BF16, 2168, 72, 5488),
    (BF16, 10480, 592, 8), (BF16, 2201, 3691, 5602), (BF16, 6291, 131, 9616), (BF16, 2800, 5460, 32), (BF16, 1, 8, 5818),
    (BF16, 1, 15, 65), (BF16, 346, 17, 11102), (BF16, 4136, 8, 352), (BF16, 2685, 8, 8658), (BF16, 10985, 9, 710),
    (BF16, 1, 4625, 272), (BF16, 1035, 18, 9792), (BF16, 17, 4153, 856), (BF16, 2508, 17, 7104), (BF16, 15606, 17, 2384),
    (BF16, 1271, 66, 6656), (BF16, 15019, 322, 64), (BF16, 17007, 426, 10752), (BF16, 7462, 229, 9280), (BF16, 2658, 5609, 64),
    (BF16, 3058, 5465, 896), (F32, 1, 4616, 4309), (F32, 791, 1231, 10), (F32, 1, 8, 8), (F32, 14619, 9, 40), (F32, 6262, 22, 33),
    (F32, 9849, 17, 784),
    # operand rows of every class of width
    (F32, 2600, 1500, 301), (F32, 2600, 1500, 513), (F32, 2600, 1500, 1030), (F32, 2600, 1500, 2501), (F32, 1200, 260, 4097),
    (F32, 1200, 260, 9001), (F32, 1200, 260, 17001), (F32, 1200, 260, 40003)]


@pytest.mark.parametrize("t,L,O,I", LINEAR_WAYS)
def test_linear_ways(t, L, O, I):
    run_linear(L, O, I, t, t, seed=L + I)
    run_linear(L, O, I, t, F32, fn="gelu_tanh", residual=True, kept=True, seed=L + I + 1)


def test_linear_in_runs_of_rows():
    """More rows than one plan takes: the second run is as the first."""
    run_linear(2 ** 23 + 5, 3, 5, F32, F32, residual=True, kept=True, seed=3)
    run_linear(2 ** 23 + 70, 2, 9, BF16, BF16, seed=4)


def test_linear_of_many_long_rows():
    """Operand rows of more lanes than a launch holds, tensors past 2^32 bytes; rows from all over against 64 bits."""
    L, O, I = 2 ** 23, 256, 1032
    x, w = torch.empty((L, I), device="cuda"), rand((O, I), 1, std=I ** -0.5).cuda()
    g = torch.Generator("cuda").manual_seed(2)
    x.normal_(generator=g)
    y = torch.full((L, O), float("nan"), device="cuda")
    hot.hot_linear_forward(x, w, y, hot.alloc_linear_workspace(F32, L, O, I))
    at = torch.tensor([0, 1, 2 ** 20 + 1, 2 ** 22 - 1, 2 ** 22, 2 ** 23 - 257, 2 ** 23 - 256, 2 ** 23 - 1], device="cuda")
    wy, _ = ref.linear(ref.f64(x[at]), ref.f64(w), None, "none", None, F32)
    close(y[at], *wy, "y")
    assert bool(torch.isfinite(y).all())


@pytest.mark.parametrize("t,L,O,I", [(BF16, 300, 1000, 1490), (BF16, 300, 1000, 1491), (F32, 700, 513, 301), (BF16, 2800, 5460, 34), (BF16, 700, 700, 10)])
def test_rows_of_any_width_stay_alone(t, L, O, I):
    """NaN at the ends of rows that begin and end inside a load reaches those rows alone."""
    x, w = rand((L, I), 1, t), rand((O, I), 2, t)
    x[5, 0], x[L - 2, I - 1], w[3, I - 1], w[O - 1, 0] = (float("nan"),) * 4
    y = torch.empty((L, O), dtype=t, device="cuda")
    hot.hot_linear_forward(x.cuda(), w.cuda(), y, hot.alloc_linear_workspace(t, L, O, I))
    want = torch.zeros(L, O, dtype=torch.bool)
    want[5], want[L - 2], want[:, 3], want[:, O - 1] = True, True, True, True
    assert torch.equal(torch.isnan(y.cpu()), want)


# ---- tensors past 32 bits ---------------------------------------------------------------------------------------------

def test_pointwise_tensors_past_32_bits():
    """Elements past 2^32: the last rows give what they give in a call of their own."""
    rows, cols = 2 ** 17 + 6, 2 ** 15 + 32
    x = torch.empty((rows, cols), dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    tail = x[-7:].contiguous()
    y, kept = torch.empty_like(x), hot.alloc_checkpoint(rows, cols)
    y7, kept7 = torch.empty_like(tail), hot.alloc_checkpoint(7, cols)
    hot.hot_activation_forward(hot.HOT_ACT_SILU, x, y, ckpt=kept)
    hot.hot_activation_forward(hot.HOT_ACT_SILU, tail, y7, ckpt=kept7)
    assert torch.equal(y[-7:], y7)
    back, back7 = torch.empty_like(x), torch.empty_like(tail)
    hot.hot_checkpoint_read(kept, back)
    hot.hot_checkpoint_read(kept7, back7)
    assert torch.equal(back[-7:], back7)
    gx, gx7 = torch.empty_like(x), torch.empty_like(tail)
    hot.hot_activation_backward(hot.HOT_ACT_SILU, y, gx, ckpt=kept)
    hot.hot_activation_backward(hot.HOT_ACT_SILU, y7, gx7, ckpt=kept7)
    assert torch.equal(gx[-7:], gx7)
    mean, rstd, mean7, rstd7 = (torch.empty(n, device="cuda") for n in (rows * 4, rows * 4, 28, 28))
    x, tail = x.view(rows * 4, cols // 4), tail.view(28, cols // 4)
    y, y7, gx, gx7 = y.view_as(x), y7.view_as(tail), gx.view_as(x), gx7.view_as(tail)
    hot.hot_layer_norm_forward(x, None, None, 1e-6, y, mean, rstd)
    hot.hot_layer_norm_forward(tail, None, None, 1e-6, y7, mean7, rstd7)
    hot.hot_layer_norm_backward(x, None, mean, rstd, gx, h=x)
    hot.hot_layer_norm_backward(tail, None, mean7, rstd7, gx7, h=tail)
    assert torch.equal(y[-28:], y7) and torch.equal(mean[-28:], mean7) and torch.equal(gx[-28:], gx7)


def test_layer_norm_of_more_lanes_than_a_launch_holds():
    rows = 2 ** 28 + 3
    x = torch.empty((rows, 1), device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    y, mean, rstd = torch.full_like(x, 7.0), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    hot.hot_layer_norm_forward(x, None, None, 1.0, y, mean, rstd)
    assert torch.equal(mean, x.view(-1)) and bool((rstd == 1).all()) and not bool(y.any())


# ---- as they are called ----------------------------------------------------------------------------------------------------

def test_calls_on_another_stream_and_replayed():
    """Every call recorded into a graph and replayed on new inputs, with eager work between, gives the eager results."""
    L, I, O = 200, 256, 320
    cfg = dict(dtype=F32)
    x, w, gamma, beta = rand((L, I), 1).cuda(), rand((O, I), 2, std=0.1).cuda(), rand((I,), 3).cuda(), rand((I,), 4).cuda()
    g = rand((L, O), 5).cuda()
    make = lambda *s: torch.empty(s, device="cuda", **cfg)     # noqa: E731
    buf_h, buf_z = hot.alloc_checkpoint(L, I), hot.alloc_checkpoint(L, O)
    ws_l, ws_a, ws_n = hot.alloc_linear_workspace(F32, L, O, I), hot.alloc_activation_workspace(L, O), hot.alloc_layer_norm_workspace(L, I)
    y, mean, rstd, u, gz, gb, gx, gg, gbeta = (make(L, I), make(L), make(L), make(L, O), make(L, O), make(O), make(L, I), make(I), make(I))
    gy2 = rand((L, I), 6).cuda()

    def step():
        hot.hot_layer_norm_forward(x, gamma, beta, 1e-6, y, mean, rstd, ckpt=buf_h)
        hot.hot_linear_forward(y, w, u, ws_l, fn=hot.HOT_ACT_GELU, ckpt=buf_z)
        hot.hot_activation_backward(hot.HOT_ACT_GELU, g, gz, ckpt=buf_z, g_bias=gb, ws=ws_a)
        hot.hot_layer_norm_backward(gy2, gamma, mean, rstd, gx, gg, gbeta, ws_n, ckpt=buf_h)

    outs = [y, mean, rstd, u, gz, gb, gx, gg, gbeta]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    eager = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    for k in range(3):
        x.copy_(rand((L, I), 1 + 10 * k))
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs]
        if k == 0:
            assert all(torch.equal(a, b) for a, b in zip(replayed, eager))
        for t in outs:
            t.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs)), k


@pytest.mark.parametrize("t,L,O,I", [(F32, 700, 513, 3001), (F32, 5054, 3202, 528), (BF16, 700, 513, 1501), (BF16, 859, 36, 4952), (F32, 1, 1079, 3448)])
def test_products_in_slices_recorded(t, L, O, I):
    """Packed operands and the slices' images live in the workspace from launch to launch: replays between eager calls on the same
    workspace give what eager calls give.  The first call of all may be a recorded one."""
    x, w, b = rand((L, I), 1, t).cuda(), rand((O, I), 2, t, I ** -0.5).cuda(), rand((O,), 3).cuda()
    y, z, ws = torch.zeros((L, O), dtype=t, device="cuda"), torch.zeros((L, O), dtype=t, device="cuda"), hot.alloc_linear_workspace(t, L, O, I)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hot.hot_linear_forward(x, w, y, ws, bias=b, fn=hot.HOT_ACT_GELU)
    for k in range(3):
        x.copy_(rand((L, I), 10 + k, t))
        y.zero_()
        graph.replay()
        hot.hot_linear_forward(x, w, z, ws, bias=b, fn=hot.HOT_ACT_GELU)
        torch.cuda.synchronize()
        assert torch.equal(y, z), k


def test_two_streams_at_once():
    """The same calls, interleaved on two streams with workspaces of their own, give what they give one after another; the stream
    is the argument's, not the current one."""
    L, I, O = 700, 1500, 513          # operand packing, K slices, sums over rows
    streams = [torch.cuda.Stream() for _ in range(2)]
    x, w, g = [rand((L, I), k).cuda() for k in range(2)], rand((O, I), 5, std=0.03).cuda(), [rand((L, O), 7 + k).cuda() for k in range(2)]
    make = lambda *s: [torch.zeros(s, device="cuda") for _ in range(2)]       # noqa: E731
    y, gz, gb, n, mean, rstd, gx, gg, gbeta = (make(L, O), make(L, O), make(O), make(L, O), make(L), make(L), make(L, O), make(O), make(O))
    kept = [hot.alloc_checkpoint(L, O) for _ in range(2)]
    ws = [(hot.alloc_linear_workspace(F32, L, O, I), hot.alloc_activation_workspace(L, O), hot.alloc_layer_norm_workspace(L, O)) for _ in range(2)]
    outs = [y, gz, gb, n, mean, rstd, gx, gg, gbeta]

    def step(k, s):
        hot.hot_linear_forward(x[k], w, y[k], ws[k][0], fn=hot.HOT_ACT_SILU, ckpt=kept[k], stream=s)
        hot.hot_activation_backward(hot.HOT_ACT_SILU, g[k], gz[k], ckpt=kept[k], g_bias=gb[k], ws=ws[k][1], stream=s)
        hot.hot_layer_norm_forward(y[k], None, None, 1e-5, n[k], mean[k], rstd[k], stream=s)
        hot.hot_layer_norm_backward(g[k], None, mean[k], rstd[k], gx[k], gg[k], gbeta[k], ws[k][2], h=y[k], stream=s)

    torch.cuda.synchronize()
    for k in range(2):
        step(k, streams[0])
        torch.cuda.synchronize()
    alone = [t.clone() for pair in outs for t in pair]
    for pair in outs:
        for t in pair:
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(4):
        for k in range(2):
            step(k, streams[k])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, [t for pair in outs for t in pair]))


def test_transformer_mlp_step_with_the_linear_backward():
    """norm -> fc1 with GELU -> fc2 with the residual, then backward: the linear backward's g_x and g_w between the gradients of the
    activation (from the 8-bit pre-activation) and of the norm (from the 8-bit stream).  Each stage is held to its 64-bit form on what
    the stage before it gave."""
    L, D, H = 208, 96, 384
    fn, code = "gelu", hot.HOT_ACT_GELU
    cfg = hot.Config()
    x, w1, w2 = rand((L, D), 1), rand((H, D), 2, std=D ** -0.5), rand((D, H), 3, std=H ** -0.5)
    b1, b2, gamma, beta = rand((H,), 4, std=0.1), rand((D,), 5, std=0.1), 1 + rand((D,), 6, std=0.1), rand((D,), 7, std=0.1)
    g_out = rand((L, D), 8, std=1e-3).cuda()
    make = lambda *s: torch.empty(s, device="cuda")       # noqa: E731
    xd, w1d, w2d, b1d, b2d, gd, bd = (t.cuda() for t in (x, w1, w2, b1, b2, gamma, beta))
    n, mean, rstd, u, out = make(L, D), make(L), make(L), make(L, H), make(L, D)
    kept_h, kept_z = hot.alloc_checkpoint(L, D), hot.alloc_checkpoint(L, H)
    act1, act2 = hot.alloc_act_buffer(cfg, L, D), hot.alloc_act_buffer(cfg, L, H)
    ws = hot.alloc_workspace(cfg, L, H, D), hot.alloc_workspace(cfg, L, D, H)
    lw1, lw2 = hot.alloc_linear_workspace(F32, L, H, D), hot.alloc_linear_workspace(F32, L, D, H)

    hot.hot_layer_norm_forward(xd, gd, bd, 1e-6, n, mean, rstd, ckpt=kept_h)
    hot.hot_compress_activation(cfg, n, act1, ws[0])
    hot.hot_linear_forward(n, w1d, u, lw1, bias=b1d, fn=code, ckpt=kept_z)
    hot.hot_compress_activation(cfg, u, act2, ws[1])
    hot.hot_linear_forward(u, w2d, out, lw2, bias=b2d, residual=xd)
    g_u, g_w2, g_z, g_b1, g_n, g_w1 = make(L, H), make(D, H), make(L, H), make(H), make(L, D), make(H, D)
    g_x, g_gamma, g_beta = make(L, D), make(D), make(D)
    hot.hot_linear_backward(cfg, g_out, w2d, act2, hot.HOT_Q_PER_TOKEN, g_u, g_w2, ws[1])
    hot.hot_activation_backward(code, g_u, g_z, ckpt=kept_z, g_bias=g_b1, ws=hot.alloc_activation_workspace(L, H))
    hot.hot_linear_backward(cfg, g_z, w1d, act1, hot.HOT_Q_PER_TOKEN, g_n, g_w1, ws[0])
    hot.hot_layer_norm_backward(g_n, gd, mean, rstd, g_x, g_gamma, g_beta, hot.alloc_layer_norm_workspace(L, D), ckpt=kept_h,
                                g_residual=g_out)
    torch.cuda.synchronize()

    close(n, *ref.norm(ref.f64(x), ref.f64(gamma), ref.f64(beta), 1e-6, F32)[0], "norm")
    wu, (z, dz) = ref.linear(ref.f64(n), ref.f64(w1), ref.f64(b1), fn, None, F32)
    close(u, *wu, "fc1")
    wo, _ = ref.linear(ref.f64(u), ref.f64(w2), ref.f64(b2), "none", ref.f64(x), F32)
    close(out, *wo, "fc2")
    z_kept = ref.f64(hot.hot_checkpoint_read(kept_z, make(L, H)))
    close(z_kept, z, z.abs().view(L, -1, 32).amax(-1).repeat_interleave(32, 1) / 127 + dz, "kept pre-activation")
    gz, tol, gb, btol = ref.act_grad(fn, ref.f64(g_u), z_kept, F32)
    close(g_z, gz, tol, "g_z")
    close(g_b1, gb, btol, "g_b1")
    h_kept = check_checkpoint(kept_h, x)
    wx, wg, wb = ref.norm_grad(ref.f64(g_n), h_kept, ref.f64(gamma), ref.f64(mean), ref.f64(rstd), ref.f64(g_out), F32)
    close(g_x, *wx, "g_x")
    close(g_gamma, *wg, "g_gamma")
    close(g_beta, *wb, "g_beta")
    # and the whole step against the exact gradient: what 4- and 8-bit operands leave of it points the same way
    X = ref.f64(x).requires_grad_(True)
    hh = torch.nn.functional.layer_norm(X, (D,), ref.f64(gamma), ref.f64(beta), 1e-6)
    o = torch.nn.functional.gelu(hh @ ref.f64(w1).t() + ref.f64(b1)) @ ref.f64(w2).t() + ref.f64(b2) + X
    (o * ref.f64(g_out)).sum().backward()
    a, b = ref.f64(g_x).flatten(), X.grad.flatten()
    assert float((a @ b) / (a.norm() * b.norm())) > 0.9
