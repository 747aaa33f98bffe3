"""The drawn rounding of 8-bit moments on the GPU: to the bit against its definition, in one step and over hundreds."""
import math

import numpy as np
import pytest
import torch

import paper_2503_21261_amd as hot
import moment_oracle as drawn
import tune_oracle as ref
from test_tune_ops_gpu import SIZES, as_np, moments_of, rand, within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def packed(m, v, seed):
    pad = -len(m) % 1024
    cm, cv = drawn.held(np.pad(m, (0, pad)), np.pad(v, (0, pad)), seed)
    return torch.from_numpy(ref.pack_state(*cm)), torch.from_numpy(ref.pack_state(*cv))


@pytest.mark.parametrize("pt,gt,copy", [(F32, F32, False), (F32, BF16, True), (BF16, BF16, False), (BF16, F32, False)])
@pytest.mark.parametrize("step", [3, 20000])
def test_step_rounds_by_its_draws(pt, gt, copy, step):
    """More tensors than a launch takes, of all lengths, beside the inputs and in place; before and past the corrections' end."""
    lr, b1, b2, eps = 1e-2, 0.9, 0.995, 1e-8
    host, dev = [], []
    for i, n in enumerate(SIZES * 4):
        m, v, mb, vb = moments_of(n, 100 + i, "8bit")
        p, g = rand((n,), 0.5, i, pt), rand((n,), 1e-2, 1000 + i, gt)
        t = dict(param=p, grad=g, m=mb, v=vb, param_out=torch.full_like(p, 9.0), m_out=torch.full_like(mb, 9), v_out=torch.full_like(vb, 9),
                 copy=torch.full((n,), 9.0, dtype=BF16) if copy else None, weight_decay=0.1 * (i % 3), lr_factor=1.0 + i % 2)
        host.append((t, m, v))
        dev.append({k: x.cuda() if isinstance(x, torch.Tensor) else x for k, x in t.items()})
    hot.hot_adamw_step(hot.AdamWTensors(dev, state="8bit"), lr, b1, b2, eps, step)
    seed = drawn.seed_of(lr, b1, b2, step)
    for (t, m, v), d in zip(host, dev):
        m2, v2 = ref.moments(m, v, as_np(t["grad"]), b1, b2)
        for name, want in zip(("m_out", "v_out"), packed(m2, v2, seed)):
            assert torch.equal(d[name].cpu(), want), (name, len(m))
        w, err = ref.weights(as_np(t["param"]), m2, v2, lr * t["lr_factor"], t["weight_decay"], 1 - b1 ** step, 1 - b2 ** step, eps)
        w, err = torch.from_numpy(w), torch.from_numpy(err)
        within("param", d["param_out"], w, err + (ref.HALF[BF16] * (w.abs() + err) if pt == BF16 else 0))
        if copy:
            assert torch.equal(d["copy"], d["param_out"].to(BF16))
    for d in dev:
        for name in ("param_out", "m_out", "v_out"):
            d[name + "_was"] = d.pop(name)
    hot.hot_adamw_step(hot.AdamWTensors(dev, state="8bit"), lr, b1, b2, eps, step)
    for d in dev:
        assert torch.equal(d["param"], d["param_out_was"]) and torch.equal(d["m"], d["m_out_was"]) and torch.equal(d["v"], d["v_out_was"])


def values(d, n):
    return [hot.hot_adamw_state_read(d[k], k, torch.empty(n, device="cuda")).cpu().numpy() for k in ("m", "v")]


@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.999), (0.5, 0.9)])
@pytest.mark.parametrize("kind", ["none after a while", "constant", "rare"])
def test_moments_follow_over_hundreds_of_steps(kind, beta1, beta2):
    """Steps from nothing: every step the definition's bits, and at the end the 64-bit moments but for what rounding right on average leaves.  The
    corrections of 0.5 and 0.9 end at step 165."""
    n, steps = 4096, 600
    rng = np.random.default_rng(11)
    all_g = [rng.standard_normal(n) * 1e-2 for _ in range(steps)]
    if kind == "constant":
        n = 1024
        all_g = [np.full(n, 1e-2)] * steps
    elif kind == "rare":
        all_g = [g * (rng.random(n) < 0.05) for g in all_g]
    else:
        # with beta2 = 0.9 v falls by half every seven steps: sixty, which leave it above its smallest code
        quiet = 300 if beta2 > 0.99 else 60
        all_g = [g if t < steps - quiet else np.zeros(n) for t, g in enumerate(all_g)]
    d = dict(param=torch.zeros(n, device="cuda"), grad=torch.empty(n, device="cuda"), m=hot.alloc_adamw_state("8bit", n), v=hot.alloc_adamw_state("8bit", n))
    tensors = hot.AdamWTensors([d], state="8bit")

    def run():
        for step, state in enumerate(drawn.steps(iter(all_g), n, beta1, beta2, lr=1e-3), 1):
            d["grad"].copy_(torch.from_numpy(all_g[step - 1].astype(np.float32)))
            hot.hot_adamw_step(tensors, 1e-3, beta1, beta2, 1e-8, step)
            if step % 50 == 0 or step < 4:
                for got, want in zip(values(d, n), state[1]):
                    assert np.array_equal(got, want), step
            yield state

    for held, exact, err in drawn.follow(run(), beta1, beta2):
        assert abs(held - exact) <= err, (held, exact, err)


def test_recorded_steps_draw_anew():
    """A step recorded once, with a fifth number, at corrections that no longer change and without gradients: every replay the definition's bits, v on
    its way down; with four numbers the same step again."""
    n, lr, b1, b2 = 2048, 1e-3, 0.9, 0.99
    m, v, mb, vb = moments_of(n, 7, "8bit")
    d = dict(param=rand((n,), 0.5, 1).cuda(), grad=torch.zeros(n, device="cuda"), m=mb.cuda(), v=vb.cuda())
    dynamic = torch.tensor([lr, 1.0, 1.0, 1.0, 0.0], device="cuda")
    tensors = hot.AdamWTensors([d], state="8bit")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        hot.hot_adamw_step(tensors, 0.0, b1, b2, 1e-8, dynamic=dynamic)
    zero = np.zeros(n, np.float32)
    for step in range(30001, 30041):
        dynamic[4] = float(step)
        graph.replay()
        m2, v2 = ref.moments(m, v, zero, b1, b2)
        (cm, cv) = drawn.held(m2, v2, drawn.step_seed(lr, 1.0, 1.0, drawn.float_bits(step)))
        m, v = ref.read_m(*cm), ref.read_v(*cv)
        got = values(d, n)
        assert np.array_equal(got[0], m) and np.array_equal(got[1], v), step
    start = moments_of(n, 7, "8bit")[1]
    # 0.99^40 = 0.67; one in a hundred steps of a code of 1/8 to 1/16: six standard deviations of 2048 elements' mean (the largest count most)
    log = np.log(v[start > 0] / start[start > 0])
    assert abs(log.mean() - 40 * math.log(b2)) < 6 * math.sqrt(40 * 0.01 / 8 * 8 / len(log)) + 40 * 0.01 / 8
    four = {k: x.clone() if isinstance(x, torch.Tensor) else x for k, x in d.items()}
    hot.hot_adamw_step(hot.AdamWTensors([four], state="8bit"), 0.0, b1, b2, 1e-8, dynamic=dynamic[:4].clone())
    m2, v2 = ref.moments(m, v, zero, b1, b2)
    want = drawn.held(m2, v2, drawn.step_seed(lr, 1.0, 1.0))
    got = values(four, n)
    assert np.array_equal(got[0], ref.read_m(*want[0])) and np.array_equal(got[1], ref.read_v(*want[1]))


@pytest.mark.parametrize("form", ["f32", "8bit"])
@pytest.mark.parametrize("rounding", [hot.HOT_ROUND_NEAREST_EVEN, hot.HOT_ROUND_PSEUDO_STOCHASTIC, hot.HOT_ROUND_DRAWN])
def test_largest_numbers_are_held_and_what_overflows_is_marked(form, rounding):
    """A gradient of 3e19, whose v' is 9e35: its group is held, to the bit.  One of 1e21, whose square is none: v's group is NaN, m's is not, and
    the weight does not move, since m' / inf is 0."""
    n, lr, b1, b2, eps = 2100, 1e-3, 0.9, 0.999, 1e-8
    m, v, mb, vb = moments_of(n, 7, form)
    p, g = rand((n,), 0.5, 1), rand((n,), 1e-2, 2)
    g[70], g[1100] = 3e19, 1e21
    d = dict(param=p.cuda(), grad=g.cuda(), m=mb.cuda(), v=vb.cuda())
    hot.hot_adamw_step(hot.AdamWTensors([d], state=form), lr, b1, b2, eps, 1, rounding=rounding)
    with np.errstate(over="ignore"):
        m2, v2 = ref.moments(m, v, g.numpy(), b1, b2)
    assert np.isfinite(m2).all() and np.isinf(v2[1100]) and np.isfinite(np.delete(v2, 1100)).all() and 8e35 < v2[70] < 1e36
    fine = np.arange(n) != 1100
    weights = d["param"].cpu()
    w, err = ref.weights(p.numpy(), m2, np.where(fine, v2, 1), lr, 0.0, 1 - b1, 1 - b2, eps)
    within("param", weights[fine], torch.from_numpy(w[fine]), torch.from_numpy(err[fine]))
    assert weights[1100] == p[1100]
    if form == "f32":
        assert torch.equal(d["m"].cpu(), torch.from_numpy(m2)) and torch.equal(d["v"].cpu(), torch.from_numpy(v2))
        return
    pad = (0, -n % 1024)
    mp, vp = np.pad(m2, pad), np.pad(np.where(fine, v2, 0), pad).astype(np.float32)
    if rounding == hot.HOT_ROUND_DRAWN:
        cm, cv = drawn.held(mp, vp, drawn.seed_of(lr, b1, b2, 1))
        cm = drawn.held_m(mp, drawn.draws(mp, np.pad(v2, pad), drawn.seed_of(lr, b1, b2, 1)))
    else:
        cm, cv = (hold(x, rounding == hot.HOT_ROUND_NEAREST_EVEN) for hold, x in ((ref.held_m, mp), (ref.held_v, vp)))
    got_m, got_v = values(d, n)
    assert np.array_equal(got_m, ref.read_m(*cm)[:n])
    marked = np.arange(n) // 32 == 1100 // 32
    assert np.isnan(got_v[marked]).all() and np.array_equal(got_v[~marked], ref.read_v(*cv)[:n][~marked])
    assert abs(float(got_v[70]) / float(v2[70]) - 1) <= 2.0 ** -3           # one of the two neighbours
