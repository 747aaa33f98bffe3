"""Host-side checks of the operators around the linear backward: sizes, refusals before any launch, and the 64-bit forms the GPU
tests hold the kernels to."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import block_oracle as ref
import paper_2503_21261_amd as hot

BIG = 1 << 40


def at(k):
    """A pointer that is never dereferenced: the calls below fail their host checks.  `k`-th gigabyte, so that none overlap."""
    return C.c_void_p((k + 1) << 30)


def test_checkpoint_bytes_follow_the_layout():
    for rows, cols in ((1, 1), (1, 32), (3, 33), (197, 768), (3330, 771), (1 << 20, 4096)):
        assert hot.hot_checkpoint_bytes(rows, cols) == ref.checkpoint_layout(rows, cols)[2]
    assert hot.hot_checkpoint_bytes(50432, 768) / (50432 * 768 * 4) < 0.2579
    for rows, cols in ((0, 5), (5, 0), (-1, 5), (1 << 31, 1), (1, 1 << 24)):
        assert hot.hot_checkpoint_bytes(rows, cols) == 0
        assert hot.hot_activation_backward_workspace_bytes(rows, cols) == 0
        assert hot.hot_layer_norm_backward_workspace_bytes(rows, cols) == 0
        with pytest.raises(hot.HotError):
            hot.alloc_checkpoint(rows, cols, device="cpu")
    assert hot.hot_layer_norm_backward_workspace_bytes(8, 16385) == 0
    assert hot.hot_layer_norm_backward_workspace_bytes(8, 16384) > 0


def test_checkpoint_refusals():
    l = hot.lib()
    assert l.hot_checkpoint_write(None, 0, 4, 64, at(1), None) == hot.HOT_ERR_ARG
    assert l.hot_checkpoint_write(at(0), 0, 4, 64, None, None) == hot.HOT_ERR_ARG
    assert l.hot_checkpoint_write(at(0), 2, 4, 64, at(1), None) == hot.HOT_ERR_ARG
    assert l.hot_checkpoint_write(at(0), -1, 4, 64, at(1), None) == hot.HOT_ERR_ARG
    assert l.hot_checkpoint_write(at(0), 0, 4, 64, at(0), None) == hot.HOT_ERR_ARG                    # in place
    assert l.hot_checkpoint_write(C.c_void_p(at(0).value + 8), 0, 4, 64, at(1), None) == hot.HOT_ERR_ARG
    assert l.hot_checkpoint_write(at(0), 0, 0, 64, at(1), None) == hot.HOT_ERR_SHAPE
    assert l.hot_checkpoint_write(at(0), 0, 4, 1 << 24, at(1), None) == hot.HOT_ERR_SHAPE
    assert l.hot_checkpoint_read(at(0), 4, 64, None, 0, None) == hot.HOT_ERR_ARG
    assert l.hot_checkpoint_read(at(0), 4, 64, C.c_void_p(at(0).value + 256), 0, None) == hot.HOT_ERR_ARG   # over its exponents
    assert l.hot_checkpoint_read(at(0), 4, -64, at(1), 0, None) == hot.HOT_ERR_SHAPE


def test_activation_refusals():
    l = hot.lib()
    f = l.hot_activation_forward
    assert f(0, at(0), 0, 4, 64, at(1), None, None) == hot.HOT_ERR_ARG          # no function
    assert f(5, at(0), 0, 4, 64, at(1), None, None) == hot.HOT_ERR_ARG
    assert f(1, at(0), 0, 4, 64, None, at(1), None) == hot.HOT_ERR_ARG
    assert f(1, at(0), 0, 4, 64, at(0), None, None) == hot.HOT_ERR_ARG
    assert f(1, at(0), 0, 4, 64, at(1), at(1), None) == hot.HOT_ERR_ARG
    assert f(1, at(0), 0, 0, 64, at(1), None, None) == hot.HOT_ERR_SHAPE
    b = l.hot_activation_backward
    assert b(1, at(0), 0, None, None, 4, 64, at(2), None, None, 0, None) == hot.HOT_ERR_ARG       # neither x nor ckpt
    assert b(1, at(0), 0, at(1), at(3), 4, 64, at(2), None, None, 0, None) == hot.HOT_ERR_ARG     # both
    assert b(1, at(0), 0, at(1), None, 4, 64, at(1), None, None, 0, None) == hot.HOT_ERR_ARG      # g_x on x
    assert b(1, at(0), 0, at(1), None, 4, 64, at(2), at(3), None, 0, None) == hot.HOT_ERR_ARG     # sums need scratch
    assert b(1, at(0), 0, at(1), None, 4, 64, at(2), at(3), C.c_void_p(at(4).value + 16), BIG, None) == hot.HOT_ERR_ARG
    assert b(1, at(0), 0, at(1), None, 4, 64, at(2), at(3), at(4), 16, None) == hot.HOT_ERR_WORKSPACE
    assert b(1, at(0), 0, at(1), None, 4, 64, at(2), at(3), at(0), BIG, None) == hot.HOT_ERR_ARG  # scratch on g_y
    assert b(1, at(0), 0, at(1), None, 1 << 31, 64, at(2), None, None, 0, None) == hot.HOT_ERR_SHAPE
    assert b(-1, at(0), 0, at(1), None, 4, 64, at(2), None, None, 0, None) == hot.HOT_ERR_ARG


def test_layer_norm_refusals():
    l = hot.lib()

    def forward(x=at(0), xt=0, r=None, gamma=at(1), beta=at(2), eps=1e-6, rows=4, cols=64, h=None, y=at(3), yt=0, mean=at(4), rstd=at(5),
                ckpt=None):
        return l.hot_layer_norm_forward(x, xt, r, gamma, beta, eps, rows, cols, h, y, yt, mean, rstd, ckpt, None)

    for bad in (dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(xt=3), dict(yt=-1), dict(xt=1, yt=0), dict(r=at(6)),
                dict(h=at(6)), dict(eps=-1.0), dict(eps=float("nan")), dict(y=at(0)), dict(rstd=at(4)), dict(ckpt=at(3)),
                dict(r=at(6), h=at(6)), dict(gamma=C.c_void_p(at(1).value + 4))):
        assert forward(**bad) == hot.HOT_ERR_ARG, bad
    for bad in (dict(rows=0), dict(cols=0), dict(cols=16385), dict(rows=1 << 31)):
        assert forward(**bad) == hot.HOT_ERR_SHAPE, bad

    def backward(g=at(0), yt=0, h=at(1), ckpt=None, xt=0, gamma=at(2), mean=at(3), rstd=at(4), gr=None, rows=4, cols=64, gx=at(5),
                 gg=at(6), gb=at(7), ws=at(8), n=BIG):
        return l.hot_layer_norm_backward(g, yt, h, ckpt, xt, gamma, mean, rstd, gr, rows, cols, gx, gg, gb, ws, n, None)

    for bad in (dict(g=None), dict(h=None), dict(ckpt=at(9)), dict(mean=None), dict(rstd=None), dict(gx=None), dict(gg=None),
                dict(gb=None), dict(ws=None), dict(xt=1), dict(gx=at(0)), dict(gx=at(1)), dict(gb=at(6)), dict(ws=at(5)),
                dict(ws=C.c_void_p(at(8).value + 128)), dict(gr=at(5))):
        assert backward(**bad) == hot.HOT_ERR_ARG, bad
    assert backward(n=100) == hot.HOT_ERR_WORKSPACE
    assert backward(cols=16385) == hot.HOT_ERR_SHAPE


def test_linear_refusals():
    l = hot.lib()

    def forward(x=at(0), w=at(1), t=0, bias=at(2), r=None, L=4, O=64, I=64, fn=0, y=at(3), yt=0, ckpt=None, ws=at(4), n=BIG):
        return l.hot_linear_forward(x, w, t, bias, r, L, O, I, fn, y, yt, ckpt, ws, n, None)

    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(t=2), dict(t=0, yt=1), dict(fn=9), dict(y=at(0)), dict(y=at(1)),
                dict(r=at(3)), dict(ckpt=at(3)), dict(w=C.c_void_p(at(1).value + 4))):
        assert forward(**bad) == hot.HOT_ERR_ARG, bad
    for bad in (dict(L=0), dict(O=0), dict(I=0), dict(I=1 << 24), dict(O=1 << 24), dict(L=1 << 31)):
        assert forward(**bad) == hot.HOT_ERR_SHAPE, bad
    for big in ((4096, 4096, 4096, hot.HOT_F32), (4096, 4096, 4097, hot.HOT_BF16)):
        L, O, I, t = big
        need = l.hot_linear_forward_workspace_bytes(t, L, O, I)
        if need:
            assert forward(L=L, O=O, I=I, t=t, yt=t, n=need - 1) == hot.HOT_ERR_WORKSPACE
            assert forward(L=L, O=O, I=I, t=t, yt=t, ws=None) == hot.HOT_ERR_ARG
    assert l.hot_linear_forward_workspace_bytes(7, 4, 4, 4) == 0


@pytest.mark.parametrize("t", [hot.HOT_F32, hot.HOT_BF16])
def test_linear_scratch_does_not_grow_with_long_inputs(t):
    """Rows past one run share its scratch; a shorter last run, which may be worked on another way, fits as well."""
    need = hot.lib().hot_linear_forward_workspace_bytes
    for O, I in ((3, 5), (200, 33), (64, 1000)):
        run = need(t, 1 << 23, O, I)
        for tail in (1, 40, 700, 9000, 1 << 20):
            assert need(t, (1 << 23) + tail, O, I) == need(t, (1 << 24) + tail, O, I) == max(run, need(t, tail, O, I))


def test_binding_refuses_host_tensors():
    x, buf = torch.zeros(4, 64), torch.zeros(4096, dtype=torch.uint8)
    for call in (lambda: hot.hot_checkpoint_write(x, buf), lambda: hot.hot_checkpoint_read(buf, x),
                 lambda: hot.hot_activation_forward(1, x, x), lambda: hot.hot_activation_backward(1, x, x, x=x),
                 lambda: hot.hot_layer_norm_forward(x, None, None, 1e-6, x, x, x),
                 lambda: hot.hot_layer_norm_backward(x, None, x, x, x, h=x), lambda: hot.hot_linear_forward(x, x, x)):
        with pytest.raises(ValueError):
            call()


# ---- the 64-bit forms --------------------------------------------------------------------------------------------------------

def test_checkpoint_form_keeps_half_a_step():
    t = torch.randn(50, 100, generator=torch.Generator().manual_seed(1)) * torch.logspace(-30, 30, 50)[:, None]
    codes, exps, values = ref.checkpoint(t)
    step = np.repeat(2.0 ** (exps.astype(np.float64) - 133), 32, axis=1)[:, :100]
    assert (np.abs(values.numpy() - t.double().numpy()) <= step / 2).all()
    assert (np.abs(codes).reshape(50, 4, 32).max(-1) >= 64).all() and np.abs(codes).max() == 127
    assert not codes[:, 100:].any()


def test_checkpoint_form_at_the_end_of_the_type():
    """The largest step there is, 2^121: half of it off up to 127.5 steps, a whole one at most beyond."""
    t = torch.cat([torch.linspace(2.0, 255.0 / 128, 4096).mul(2.0 ** 126), torch.linspace(255.0 / 128, 2 - 2.0 ** -23, 4096).mul(2.0 ** 127)]).view(-1, 32)
    t[:, 0] = 255.0 / 128 * 2.0 ** 127             # every group has the largest step
    codes, exps, values = ref.checkpoint(t)
    assert (exps == 254).all() and np.abs(codes).max() == 127
    off = (values - t.double()).abs()
    far = t.double() > 127.5 * 2.0 ** 121
    assert bool((off[~far] <= 2.0 ** 120).all()) and bool((off[far] <= 2.0 ** 121).all()) and float(off.max()) > 0.99 * 2.0 ** 121


@pytest.mark.parametrize("fn", ["relu", "gelu", "gelu_tanh", "silu"])
def test_slopes_are_the_differences_of_the_values(fn):
    x = torch.linspace(-8, 8, 4001, dtype=torch.float64) + 1e-4
    step = 1e-6
    want = (ref.act(fn, x + step)[0] - ref.act(fn, x - step)[0]) / (2 * step)
    assert float((ref.act_slope(fn, x)[0] - want).abs().max()) < 1e-8


def test_norm_gradients_are_those_of_its_values():
    g = torch.Generator().manual_seed(2)
    h, w = (torch.randn(5, 40, dtype=torch.float64, generator=g).requires_grad_(True) for _ in range(2))
    gamma = torch.randn(40, dtype=torch.float64, generator=g).requires_grad_(True)
    beta = torch.randn(40, dtype=torch.float64, generator=g).requires_grad_(True)
    (y, _), (mean, _), (rstd, _) = ref.norm(h, gamma, beta, 1e-5, torch.float32)
    want = torch.autograd.grad((y * w).sum(), (h, gamma, beta))
    got = ref.norm_grad(w.detach(), h.detach(), gamma.detach(), mean.detach(), rstd.detach(), None, torch.float32)
    for (value, _), at64 in zip(got, want):
        assert float((value - at64).abs().max()) < 1e-12


# ---- sizes asked for from Python ----------------------------------------------------------------------------------------------

def test_linear_workspace_refuses_other_types_and_sizes():
    for call in (hot.hot_linear_forward_workspace_bytes, hot.alloc_linear_workspace, hot.hot_debug_linear_plan):
        for dtype in (torch.float16, torch.float64, torch.int8):
            with pytest.raises(ValueError):
                call(dtype, 64, 64, 64)
    for bad in ((0, 4, 4), (4, 0, 4), (4, 4, 0), (-1, 4, 4), (1 << 31, 4, 4), (4, 1 << 24, 4), (4, 4, 1 << 24)):
        with pytest.raises(hot.HotError):
            hot.alloc_linear_workspace(torch.float32, *bad, device="cpu")
        with pytest.raises(hot.HotError):
            hot.hot_debug_linear_plan(torch.float32, *bad)
    assert hot.alloc_linear_workspace(torch.float32, 1, 1, 1, device="cpu") is None
    assert hot.alloc_linear_workspace(torch.float32, 12608, 2304, 768, device="cpu").numel() == \
        hot.hot_linear_forward_workspace_bytes(torch.float32, 12608, 2304, 768) > 0


# ---- the timing of stages --------------------------------------------------------------------------------------------------------

def test_stage_timing_fills_the_arrays_that_its_caller_has():
    """hot_debug_profile_end writes the linear backward's fifteen stages, as many as it always did; the others have a call of their own."""
    l = hot.lib()

    def arrays():
        return (C.c_float * 32)(*[-1.0] * 32), (C.c_int64 * 32)(*[-1] * 32)

    for call, filled in ((lambda ms, n: l.hot_debug_profile_end(ms, n), 15), (lambda ms, n: l.hot_debug_profile_end_all(ms, n, 24), 24),
                         (lambda ms, n: l.hot_debug_profile_end_all(ms, n, 3), 3), (lambda ms, n: l.hot_debug_profile_end_all(ms, n, 0), 0)):
        ms, n = arrays()
        l.hot_debug_profile_begin()
        assert call(ms, n) == hot.HOT_OK
        assert list(ms) == [0.0] * filled + [-1.0] * (32 - filled) and list(n) == [0] * filled + [-1] * (32 - filled)
    ms, n = arrays()
    assert l.hot_debug_profile_end_all(ms, n, -1) == hot.HOT_ERR_ARG and l.hot_debug_profile_end_all(None, n, 4) == hot.HOT_ERR_ARG
    names = [l.hot_debug_stage_name(i).decode() for i in range(25)]
    assert len(set(names[:24])) == 24 and all(names[:24]) and names[24] == ""
    assert names[14] == "gy_fused_quant" and names[15] == "checkpoint_write"


def test_stage_numbers_are_those_of_the_header():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hot.h")).read()
    for name in ("HOT_NUM_STAGES", "HOT_NUM_STAGES_ALL"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(hot, name)
