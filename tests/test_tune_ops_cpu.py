"""Host-side checks of the operators of a fine-tuning step: sizes, and refusals before any launch; and of the 64-bit forms that the GPU
tests hold the kernels to."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2503_21261_amd as hot
import tune_oracle as ref

BIG = 1 << 44


def at(k):
    """A pointer that is never dereferenced: the calls below fail their host checks.  `k`-th gigabyte, so that none overlap."""
    return C.c_void_p((k + 1) << 30)


def off(p, n):
    return C.c_void_p(p.value + n)


# ---- adapters --------------------------------------------------------------------------------------------------------

def adapter_forward(x=at(0), a=at(1), b=at(2), ty=0, scale=at(3), offsets=at(4), index=at(5), segments=3, adapters=2, L=8, O=64, I=32, rank=4,
                    base=at(6), y=at(7), u=at(8), ws=at(9), n=BIG):
    return hot.lib().hot_adapter_forward(x, a, b, ty, scale, offsets, index, segments, adapters, L, O, I, rank, base, y, u, ws, n, None)


def adapter_backward(g_y=at(0), x=at(1), u=at(2), a=at(3), b=at(4), ty=0, scale=at(5), offsets=at(6), index=at(7), segments=3, adapters=2, L=8,
                     O=64, I=32, rank=4, g_base=at(8), g_x=at(9), g_a=at(10), g_b=at(11), ws=at(12), n=BIG):
    return hot.lib().hot_adapter_backward(g_y, x, u, a, b, ty, scale, offsets, index, segments, adapters, L, O, I, rank, g_base, g_x, g_a, g_b, ws,
                                          n, None)


BAD_BATCH = (dict(offsets=None), dict(index=None), dict(offsets=None, index=None), dict(segments=0))
BAD_SIZES = (dict(L=0), dict(L=-1), dict(L=1 << 30), dict(O=0), dict(I=0), dict(O=1 << 24), dict(I=1 << 24), dict(rank=0), dict(rank=129),
             dict(adapters=0), dict(adapters=65537), dict(adapters=65536, O=1 << 20), dict(segments=-1), dict(segments=(1 << 24) + 1))


def test_adapter_forward_refusals():
    for bad in BAD_BATCH + (dict(x=None), dict(a=None), dict(b=None), dict(y=None), dict(ws=None), dict(ws=off(at(9), 16)), dict(ty=2), dict(ty=-1),
                            dict(y=at(0)), dict(y=at(1)), dict(u=at(7)), dict(u=at(0)), dict(ws=at(0)), dict(x=off(at(0), 4)), dict(y=off(at(6), 16)),
                            dict(scale=off(at(3), 8)), dict(y=at(4)), dict(u=at(5))):
        assert adapter_forward(**bad) == hot.HOT_ERR_ARG, bad
    for bad in BAD_SIZES:
        assert adapter_forward(**bad) == hot.HOT_ERR_SHAPE, bad
    assert adapter_forward(n=0) == hot.HOT_ERR_WORKSPACE
    need = hot.hot_adapter_forward_workspace_bytes(torch.float32, 8, 64, 32, 4, 2, 3)
    assert need > 0 and adapter_forward(n=need - 1) == hot.HOT_ERR_WORKSPACE


def test_adapter_backward_refusals():
    for bad in BAD_BATCH + (dict(g_y=None), dict(b=None), dict(ws=None), dict(ws=off(at(12), 128)), dict(ty=2), dict(g_a=None), dict(g_b=None),
                            dict(g_x=None), dict(g_x=None, g_base=None, g_a=None, g_b=None), dict(a=None), dict(x=None), dict(u=None), dict(g_x=at(0)),
                            dict(g_a=at(1)), dict(g_a=at(11)), dict(g_x=off(at(8), 16)), dict(ws=at(8)), dict(g_b=at(6))):
        assert adapter_backward(**bad) == hot.HOT_ERR_ARG, bad
    for bad in BAD_SIZES:
        assert adapter_backward(**bad) == hot.HOT_ERR_SHAPE, bad
    need = hot.hot_adapter_backward_workspace_bytes(torch.float32, 8, 64, 32, 4, 2, 3)
    assert need > 0 and adapter_backward(n=need - 1) == hot.HOT_ERR_WORKSPACE


def test_adapter_workspace_sizes():
    for f in (hot.hot_adapter_forward_workspace_bytes, hot.hot_adapter_backward_workspace_bytes):
        assert f(torch.bfloat16, 1, 4096, 4096, 16, 1, 0) > 0
        for bad in ((0, 4, 4, 4, 1, 0), (4, 0, 4, 4, 1, 0), (4, 4, 0, 4, 1, 0), (4, 4, 4, 0, 1, 0), (4, 4, 4, 129, 1, 0), (4, 4, 4, 4, 0, 0), (4, 4, 4, 4, 1, -1),
                    (1 << 30, 4, 4, 4, 1, 0)):
            assert f(torch.float32, *bad) == 0
        assert f(torch.float32, (1 << 27) - 1, 4, 4, 4, 1, 0) > 0 and f(torch.float32, 1 << 27, 4, 4, 4, 1, 0) == 0
        assert f(torch.float32, 4, 1024, 1023, 4, 65536, 1) > 0 and f(torch.float32, 4, 1024, 1024, 4, 65536, 1) == 0
    with pytest.raises(ValueError):
        hot.hot_adapter_forward_workspace_bytes(torch.float16, 4, 4, 4, 4, 1, 0)
    x, a, b = torch.empty(4, 8), torch.empty(2, 3, 8), torch.empty(2, 5, 3)
    assert hot.alloc_adapter_workspace(x, a, b).numel() == max(hot.hot_adapter_forward_workspace_bytes(torch.float32, 4, 5, 8, 3, 2, 0),
                                                               hot.hot_adapter_backward_workspace_bytes(torch.float32, 4, 5, 8, 3, 2, 0))
    with pytest.raises(hot.HotError):
        hot.alloc_adapter_workspace(torch.empty(0, 8), a, b)


# ---- log probabilities -----------------------------------------------------------------------------------------------

def logprobs(z=at(0), ty=0, rows=4, vocab=100, t=at(1), logp=at(2), entropy=at(3), stats=at(4), top=5, tl=at(5), ti=at(6), ws=at(7), n=BIG):
    return hot.lib().hot_token_logprobs(z, ty, rows, vocab, t, logp, entropy, stats, top, tl, ti, ws, n, None)


def test_logprob_refusals():
    for bad in (dict(z=None), dict(ty=2), dict(t=None), dict(logp=None), dict(tl=None), dict(ti=None), dict(top=0), dict(tl=None, ti=None),
                dict(t=None, logp=None, entropy=None, stats=None, top=0, tl=None, ti=None), dict(logp=at(0)), dict(entropy=at(2)), dict(stats=at(1)),
                dict(ti=at(5)), dict(z=off(at(0), 2)), dict(vocab=9000, ws=None), dict(vocab=9000, ws=off(at(7), 16)), dict(vocab=9000, ws=at(0))):
        assert logprobs(**bad) == hot.HOT_ERR_ARG, bad
    for bad in (dict(rows=0), dict(vocab=0), dict(vocab=1 << 24), dict(rows=1 << 31), dict(top=33), dict(top=-1), dict(vocab=4)):
        assert logprobs(**bad) == hot.HOT_ERR_SHAPE, bad
    assert logprobs(vocab=9000, n=0) == hot.HOT_ERR_WORKSPACE
    size = hot.hot_token_logprobs_workspace_bytes
    assert size(torch.float32, 4, 9000, 5) > 0 and size(torch.float32, 4, 100, 5) == 0 and size(torch.float32, 4096, 8192, 5) == 0
    assert size(torch.float32, 4, 9000, 33) == 0 and size(torch.float32, 4, 4, 5) == 0 and size(torch.float32, 0, 9000, 0) == 0
    with pytest.raises(hot.HotError):
        hot.alloc_logprobs_workspace(torch.empty(3, 9), 10)
    assert hot.alloc_logprobs_workspace(torch.empty(3, 9), 9) is None


def test_logprob_backward_refusals():
    def f(z=at(0), ty=0, rows=4, vocab=100, t=at(1), stats=at(2), entropy=at(3), gl=at(4), ge=at(5), g=at(6)):
        return hot.lib().hot_token_logprobs_backward(z, ty, rows, vocab, t, stats, entropy, gl, ge, g, None)

    for bad in (dict(z=None), dict(ty=5), dict(stats=None), dict(g=None), dict(t=None), dict(gl=None), dict(entropy=None), dict(ge=None),
                dict(t=None, gl=None, entropy=None, ge=None), dict(g=off(at(0), 16)), dict(g=at(1)), dict(g=at(4)), dict(z=off(at(0), 8))):
        assert f(**bad) == hot.HOT_ERR_ARG, bad
    for bad in (dict(rows=0), dict(vocab=0), dict(vocab=1 << 24), dict(rows=1 << 31)):
        assert f(**bad) == hot.HOT_ERR_SHAPE, bad


# ---- optimiser -------------------------------------------------------------------------------------------------------

def tensor(k=0, **more):
    t = dict(grad=at(k).value, param=at(k + 1).value, m=at(k + 2).value, v=at(k + 3).value, n=100, param_type=0, grad_type=0, weight_decay=0.1, lr_factor=1.0)
    t.update(more)
    return hot.hot_adamw_tensor(**t)


def table(tensors, form=0, bytes_=None, buf=None):
    n = len(tensors)
    arr = (hot.hot_adamw_tensor * max(n, 1))(*tensors)
    size = int(hot.lib().hot_adamw_table_bytes(n))
    buf = (C.c_uint64 * 4096)() if buf is None else buf
    return hot.lib().hot_adamw_table(arr, n, form, buf, size if bytes_ is None else bytes_), buf


def test_adamw_table_refusals():
    good = tensor()
    assert table([good])[0] == hot.HOT_OK and table([good, tensor(10)], form=1)[0] == hot.HOT_OK
    p, m, v = at(1).value, at(2).value, at(3).value
    assert table([tensor(param_out=at(5).value, m_out=at(6).value, v_out=at(7).value, copy=at(8).value)])[0] == hot.HOT_OK
    for bad in (dict(grad=None), dict(param=None), dict(m=None), dict(v=None), dict(param_type=2), dict(grad_type=-1), dict(weight_decay=math.nan),
                dict(lr_factor=math.inf), dict(param_type=1, copy=at(8).value), dict(grad=p), dict(m=p + 16), dict(v=m), dict(copy=p), dict(copy=at(0).value),
                dict(param_out=p + 16), dict(m_out=p), dict(v_out=m), dict(param=p + 8), dict(m_out=v), dict(param_out=at(0).value)):
        assert table([tensor(**bad)])[0] == hot.HOT_ERR_ARG, bad
        assert table([tensor(20), tensor(**bad)])[0] == hot.HOT_ERR_ARG, bad
    assert table([good, good])[0] == hot.HOT_ERR_ARG                                                # the same tensor twice
    assert table([good, tensor(10, grad=p)])[0] == hot.HOT_ERR_ARG                                  # another's weights as gradient
    assert table([good, tensor(10, grad=at(0).value)])[0] == hot.HOT_OK                             # a gradient that two tensors share
    for n in (0, -1, 1 << 40):
        assert table([tensor(n=n)])[0] == hot.HOT_ERR_SHAPE
    assert table([])[0] == hot.HOT_ERR_SHAPE
    assert table([good], form=2)[0] == hot.HOT_ERR_ARG
    assert table([good], bytes_=8)[0] == hot.HOT_ERR_WORKSPACE
    # moments' sizes: fp32 ones of 1024 elements reach the next 4 KB, 8-bit ones do not
    close = dict(n=1024, v=m + 2048)
    assert table([tensor(**close)])[0] == hot.HOT_ERR_ARG and table([tensor(**close)], form=1)[0] == hot.HOT_OK


def test_adamw_step_refusals():
    st, t = table([tensor()])
    assert st == hot.HOT_OK

    def step(table_=t, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, rounding=1, dynamic=None):
        cfg = hot.hot_adamw_config(lr, beta1, beta2, eps, step, rounding, 0, dynamic)
        return hot.lib().hot_adamw_step(table_, C.byref(cfg), None)

    for bad in (dict(table_=None), dict(table_=(C.c_uint64 * 64)()), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
                dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-60), dict(eps=math.inf), dict(step=0), dict(rounding=2),
                dict(dynamic=at(0).value + 4)):
        assert step(**bad) == hot.HOT_ERR_ARG, bad
    assert hot.lib().hot_adamw_step(t, None, None) == hot.HOT_ERR_ARG
    _, again = table([tensor(n=0)], buf=t)                       # a table that was refused is none
    assert step(again) == hot.HOT_ERR_ARG


def test_adamw_state_sizes_and_refusals():
    for n, size in ((1, 1056), (1024, 1056), (1025, 2112), (1 << 30, (1 << 20) * 1056)):
        assert hot.hot_adamw_state_bytes("8bit", n) == size and hot.hot_adamw_state_bytes("f32", n) == 4 * n
    for n in (0, -1, 1 << 40):
        assert hot.hot_adamw_state_bytes("8bit", n) == 0 and hot.hot_adamw_state_bytes("f32", n) == 0
    assert hot.lib().hot_adamw_state_bytes(2, 5) == 0
    with pytest.raises(hot.HotError):
        hot.alloc_adamw_state("8bit", 0, device="cpu")
    l = hot.lib()
    assert l.hot_adamw_state_read(None, 0, 5, at(0), 0, None) == hot.HOT_ERR_ARG
    assert l.hot_adamw_state_read(at(0), 2, 5, at(1), 0, None) == hot.HOT_ERR_ARG
    assert l.hot_adamw_state_read(at(0), 0, 5, at(0), 0, None) == hot.HOT_ERR_ARG
    assert l.hot_adamw_state_read(at(0), 0, 0, at(1), 0, None) == hot.HOT_ERR_SHAPE
    assert l.hot_adamw_state_write(at(0), 3, 0, 5, at(1), None) == hot.HOT_ERR_ARG
    assert l.hot_adamw_state_write(at(0), 0, 0, 5, off(at(0), 16), None) == hot.HOT_ERR_ARG
    assert l.hot_adamw_state_write(at(0), 0, 0, 1 << 40, at(1), None) == hot.HOT_ERR_SHAPE


def test_host_tensors_are_refused():
    x, a, b, y = torch.zeros(4, 8), torch.zeros(1, 2, 8), torch.zeros(1, 6, 2), torch.zeros(4, 6)
    with pytest.raises(ValueError):
        hot.hot_adapter_forward(x, a, b, y, torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(ValueError):
        hot.hot_token_logprobs(x, torch.zeros(4, dtype=torch.int64), torch.zeros(4))
    with pytest.raises(ValueError):
        hot.AdamWTensors([dict(param=x, grad=x, m=x, v=x)])


# ---- the forms the kernels are held to ---------------------------------------------------------------------------------

def test_reference_gradients_of_the_adapters_are_autograds():
    g = torch.Generator().manual_seed(1)
    L, O, I, r, K = 9, 6, 5, 3, 2
    x, a, b, base, g_y = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((L, I), (K, r, I), (K, O, r), (L, O), (L, O)))
    scale = torch.tensor([0.5, 2.0], dtype=torch.float64)
    k, inside = ref.owners(L, [0, 3, 3, 7], [1, 0, 0], K)
    ref.HALF[torch.float64] = 0.0
    try:
        out = ref.adapter(x, a, b, scale, base, k, inside, torch.zeros(L, O), torch.zeros(L, r), g_y, torch.zeros(L, I), torch.zeros(L, I))
    finally:
        del ref.HALF[torch.float64]
    x, a, b = (t.requires_grad_(True) for t in (x, a, b))
    y = torch.stack([base[l] + (scale[k[l]] * (b[k[l]] @ (a[k[l]] @ x[l])) if k[l] >= 0 else 0) for l in range(L)])
    (y * g_y)[inside].sum().backward()
    for name, t in (("g_x", x), ("g_a", a), ("g_b", b)):
        assert torch.allclose(out[name][0], t.grad, rtol=1e-12, atol=1e-12), name


def test_reference_gradient_of_the_log_probabilities_is_autograds_and_the_differences():
    g = torch.Generator().manual_seed(2)
    z = torch.randn(4, 11, generator=g, dtype=torch.float64) * 2
    z[1, 3] = -math.inf
    t = torch.tensor([3, 5, -1, 0])
    gl, ge = torch.randn(4, generator=g, dtype=torch.float64), torch.randn(4, generator=g, dtype=torch.float64)
    ref.HALF[torch.float64] = 0.0
    try:
        out = ref.logprobs(z, t, g_logp=gl, g_entropy=ge)["g_logits"][0]

        def value(w):
            r = ref.logprobs(w, t)
            return (gl * r["logp"][0] + ge * r["entropy"][0]).sum()

        for row, col in ((0, 3), (0, 0), (1, 5), (2, 7), (3, 0)):
            d = torch.zeros_like(z)
            d[row, col] = 1e-5
            assert abs((value(z + d) - value(z - d)) / 2e-5 - out[row, col]) < 1e-8
    finally:
        del ref.HALF[torch.float64]
    assert out[1, 3] == 0
    keep = z[torch.arange(4) != 1].clone().requires_grad_(True)
    lp = torch.log_softmax(keep, 1)
    s = torch.tensor([3, -1, 0])
    H = -(lp.exp() * lp).sum(1)
    rows = torch.tensor([0, 2])
    loss = (gl[[0, 3]] * lp[rows, s[rows]]).sum() + (ge[[0, 2, 3]] * H).sum()
    loss.backward()
    assert torch.allclose(out[[0, 2, 3]], keep.grad, rtol=1e-11, atol=1e-12)


def test_eight_bit_moments_round_trip_and_round_as_said():
    rng = np.random.default_rng(3)
    for scale in (1e-12, 1e-6, 1.0, 1e15):
        m = (rng.standard_normal(4096) * scale).astype(np.float32)
        c, e = ref.held_m(m, True)
        step = np.exp2(e.astype(np.float64) - 133).repeat(32)
        assert np.abs(ref.read_m(c, e) - m).max() <= (0.5 * step).max() and (np.abs(ref.read_m(c, e) - m) <= 0.5 * step).all()
        c2, e2 = ref.held_m(ref.read_m(c, e), True)
        assert (c2 == c).all() and (e2 <= e).all()
        v = (m * m).astype(np.float32)
        c, e = ref.held_v(v, True)
        back = ref.read_v(c, e)
        big = v >= v.reshape(-1, 32).max(1).repeat(32) * 2.0 ** -30
        if scale > 1e-12:
            assert (np.abs(back - v)[big] <= 2.0 ** -4 * v[big]).all() and ((back > 0) == (v > 0)).all()
        assert (ref.held_v(back, True)[0] == c).all()
    # the pseudo-stochastic rounding is unbiased over values whose low bits are spread
    v = rng.uniform(1.0, 2.0, 1 << 16).astype(np.float32)
    c, e = ref.held_v(v, False)
    assert abs((ref.read_v(c, e).astype(np.float64) - v).mean()) < 4 * 0.125 / math.sqrt(12 * (1 << 16)) + 0.125 / 2048


# ---- the timing of stages ----------------------------------------------------------------------------------------------

def test_every_stage_but_the_gap_has_a_name_of_its_own():
    """24 is none, so that a list read up to the first number without a name is the one that it was; the last ones end at HOT_NUM_STAGES_ALL."""
    l, n = hot.lib(), hot.HOT_NUM_STAGES_ALL
    names = [l.hot_debug_stage_name(i).decode() for i in range(-1, n + 2)][1:]
    assert names[24] == names[n] == names[n + 1] == "" and l.hot_debug_stage_name(-1) == b""
    named = [s for i, s in enumerate(names[:n]) if i != 24]
    assert all(named) and len(set(named)) == n - 1
    assert names[25] == "adapter_prepare" and names[31:] == ["token_logprobs", "token_logprobs_grad", "adamw", "adamw_state_read", "adamw_state_write", "", ""]
    ms, launches = (C.c_float * (n + 2))(*[-1.0] * (n + 2)), (C.c_int64 * (n + 2))(*[-1] * (n + 2))
    l.hot_debug_profile_begin()
    assert l.hot_debug_profile_end_all(ms, launches, n + 1) == hot.HOT_OK
    assert list(ms) == [0.0] * (n + 1) + [-1.0] and list(launches) == [0] * (n + 1) + [-1]
