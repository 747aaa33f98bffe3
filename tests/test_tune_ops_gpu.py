"""The operators of a fine-tuning step on the GPU, against their 64-bit forms: tolerances are those forms' own bounds."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2503_21261_amd as hot
import tune_oracle as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def rand(shape, std, seed, dtype=F32):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def within(name, got, value, err):
    got = got.double().cpu()
    d = (got - value).abs()
    same = (got == value) | (got.isnan() & value.isnan())
    worst = torch.where(same, 0.0, d / err.clamp(min=1e-300))
    most, ok = float(worst.max()), bool(torch.isfinite(worst).all())
    assert ok and most <= 1.0, (name, most, int(worst.argmax()))


# ---- adapters --------------------------------------------------------------------------------------------------------

BATCHES = {
    "one": (None, None, 1),
    "ragged": ([0, 5, 5, 38, 70], [1, 0, 2, 1], 3),                  # an empty segment, tiles that hold several, one adapter twice
    "gaps": ([3, 17, 40, 64, 66], [0, -1, 7, 1], 2),                 # rows in front and behind; no adapter; an index out of range
    "single": (list(range(71)), [i * 5 % 4 for i in range(70)], 4),  # a token a request
    "empty": ([9, 9, 9], [0, 0], 2),                                 # no rows at all
}


def make(L, O, I, rank, batch, dtype, seed=0):
    offsets, index, K = BATCHES[batch] if isinstance(batch, str) else batch
    t = dict(x=rand((L, I), 1.0, seed, dtype), a=rand((K, rank, I), 1 / math.sqrt(I), seed + 1, dtype), b=rand((K, O, rank), 0.3, seed + 2, dtype),
             scale=rand((K,), 0.5, seed + 3) + 1.5, base=rand((L, O), 1.0, seed + 4, dtype), g_y=rand((L, O), 0.1, seed + 5, dtype),
             g_base=rand((L, I), 0.1, seed + 6, dtype), y=rand((L, O), 1.0, seed + 7, dtype), u=rand((L, rank), 1.0, seed + 8),
             g_x=rand((L, I), 1.0, seed + 9, dtype), g_a=torch.full((K, rank, I), math.nan), g_b=torch.full((K, O, rank), math.nan))
    if offsets is not None:
        t["offsets"], t["index"] = torch.tensor(offsets, dtype=torch.int32), torch.tensor(index, dtype=torch.int32)
    return t, (offsets, index, K)


def run_pass(t, ws=None):
    d = {k: v.cuda() for k, v in t.items()}
    more = dict(scale=d.get("scale"), offsets=d.get("offsets"), index=d.get("index"))
    if ws is None:
        ws = hot.alloc_adapter_workspace(d["x"], d["a"], d["b"], segments=0 if d.get("index") is None else len(d["index"]))
        ws.fill_(255)                                                 # NaNs, whatever it is read as
    hot.hot_adapter_forward(d["x"], d["a"], d["b"], d["y"], ws, base=d.get("base"), u=d["u"], **more)
    hot.hot_adapter_backward(d["g_y"], d["x"], d["u"], d["a"], d["b"], ws, g_base=d.get("g_base"), g_x=d["g_x"], g_a=d["g_a"], g_b=d["g_b"], **more)
    return {k: d[k] for k in ("y", "u", "g_x", "g_a", "g_b")}


def check_pass(t, batch, got):
    offsets, index, K = batch
    k, inside = ref.owners(t["x"].shape[0], offsets, index, K)
    want = ref.adapter(t["x"], t["a"], t["b"], t.get("scale"), t.get("base"), k, inside, t["y"], t["u"], t["g_y"], t.get("g_base"), t["g_x"])
    for name in ("y", "u", "g_x", "g_a", "g_b"):
        within(name, got[name], *want[name])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("O,I,rank", [(64, 128, 16), (77, 131, 12), (200, 64, 1), (130, 300, 33), (96, 72, 128)])
def test_adapter_pass(O, I, rank, batch, dtype):
    t, kind = make(70, O, I, rank, batch, dtype)
    check_pass(t, kind, run_pass(t))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("L,O,I,rank", [(1, 1, 1, 1), (1, 96, 2000, 16), (1, 4096, 4096, 8), (3, 500, 4100, 64), (31, 129, 33, 5), (33, 65, 1025, 20), (300, 520, 264, 16),
                                        (1000, 130, 770, 40)])
def test_adapter_lengths(L, O, I, rank, dtype):
    t, kind = make(L, O, I, rank, (None, None, 1), dtype, seed=20)
    check_pass(t, kind, run_pass(t))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("L,O,I,rank,batch", [(2100, 264, 200, 16, None), (2500, 77, 133, 30, None), (4096, 40, 2080, 64, None), (14400, 136, 200, 40, None),
                                              (14500, 72, 100, 20, ([0, 33, 5000, 5001, 14499], [1, 0, 1, 0], 2)), (3000, 520, 96, 100, None)])
def test_adapter_many_rows(L, O, I, rank, batch, dtype):
    """Larger tiles of rows, packed weights, rounds of steps on their way."""
    t, kind = make(L, O, I, rank, batch or (None, None, 1), dtype, seed=25)
    check_pass(t, kind, run_pass(t))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_adapter_rows_of_their_own(dtype):
    """A token a request at every rank that has a kernel of its own, and at some that have not; more segments than one load of a wave."""
    for L, rank, O, I in ((5, 8, 1030, 300), (100, 16, 333, 500), (64, 32, 200, 96), (3, 64, 4100, 4100), (200, 128, 65, 130), (30, 24, 100, 77), (30, 7, 90, 64)):
        batch = (list(range(L + 1)), [(i * 3) % 5 - (i % 7 == 0) for i in range(L)], 4)
        t, kind = make(L, O, I, rank, batch, dtype, seed=27)
        check_pass(t, kind, run_pass(t))
        plain = {k: v for k, v in t.items() if k not in ("scale", "base", "g_base")}
        check_pass(plain, kind, run_pass(plain))


def test_adapter_many_segments():
    """More segments than the widest step of their search, of lengths from zero on, adapters in no order."""
    rng = np.random.default_rng(5)
    cuts = np.concatenate([[0], np.cumsum(rng.integers(0, 3, 5000))])
    index = rng.integers(-1, 9, 5000).tolist()
    for dtype in (F32, BF16):
        t, kind = make(int(cuts[-1]) + 3, 40, 72, 8, (cuts.tolist(), index, 8), dtype, seed=30)
        check_pass(t, kind, run_pass(t))


def test_adapter_long_segments_of_several_adapters():
    cuts, index = [0, 700, 701, 1400, 1400, 2900], [2, 0, 2, 1, 0]
    for dtype in (F32, BF16):
        t, kind = make(3000, 96, 136, 16, (cuts, index, 4), dtype, seed=40)       # adapter 3 has no rows
        check_pass(t, kind, run_pass(t))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_adapter_without_base_and_scale_and_in_place(dtype):
    t, kind = make(70, 100, 60, 6, "ragged", dtype, seed=50)
    plain = {k: v for k, v in t.items() if k not in ("scale", "base", "g_base")}
    check_pass(plain, kind, run_pass(plain))
    apart = run_pass(t)
    d = {k: v.cuda() for k, v in t.items()}
    more = dict(scale=d["scale"], offsets=d["offsets"], index=d["index"])
    ws = hot.alloc_adapter_workspace(d["x"], d["a"], d["b"], segments=4)
    hot.hot_adapter_forward(d["x"], d["a"], d["b"], d["base"], ws, base=d["base"], **more)
    assert torch.equal(d["base"], apart["y"])
    hot.hot_adapter_backward(d["g_y"], d["x"], None, d["a"], d["b"], ws, g_base=d["g_base"], g_x=d["g_base"], **more)
    assert torch.equal(d["g_base"], apart["g_x"])
    hot.hot_adapter_backward(d["g_y"], d["x"], apart["u"], d["a"], d["b"], ws, g_a=d["g_a"], g_b=d["g_b"], **more)
    assert torch.equal(d["g_a"], apart["g_a"]) and torch.equal(d["g_b"], apart["g_b"])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("O,I,rank", [(131, 259, 12), (139, 75, 40), (3, 7, 5), (264, 132, 100)])
def test_adapter_borders_inside_tiles_of_many_rows(O, I, rank, dtype):
    """Requests, rows without an adapter among them, that begin and end anywhere in tiles of many rows; last columns that fill no load; beside
    base, without it, and in place."""
    batch = ([3, 5, 700, 1407, 1407, 1441, 2140], [1, 0, -1, 1, 0, 1], 2)
    t, kind = make(2150, O, I, rank, batch, dtype, seed=64)
    got = run_pass(t)
    check_pass(t, kind, got)
    plain = {k: v for k, v in t.items() if k not in ("scale", "base", "g_base")}
    check_pass(plain, kind, run_pass(plain))
    d = {k: v.cuda() for k, v in t.items()}
    ws = hot.alloc_adapter_workspace(d["x"], d["a"], d["b"], segments=len(batch[1]))
    more = dict(scale=d["scale"], offsets=d["offsets"], index=d["index"])
    hot.hot_adapter_forward(d["x"], d["a"], d["b"], d["base"], ws, base=d["base"], u=d["u"], **more)
    hot.hot_adapter_backward(d["g_y"], d["x"], d["u"], d["a"], d["b"], ws, g_base=d["g_base"], g_x=d["g_base"], g_a=d["g_a"], g_b=d["g_b"], **more)
    inside = slice(batch[0][0], batch[0][-1])
    assert torch.equal(d["base"][inside], got["y"][inside]) and torch.equal(d["g_base"][inside], got["g_x"][inside])
    for name in ("u", "g_a", "g_b"):
        assert torch.equal(d[name], got[name]), name


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_adapter_keeps_infinities_and_nans_in_their_rows(dtype):
    for batch in ("ragged", "single", "one"):
        t, kind = make(70, 96, 70, 20, batch, dtype, seed=60)
        clean = run_pass(t)
        bad = {k: v.clone() for k, v in t.items()}
        bad["x"][7, 69] = math.nan
        bad["x"][40, 3] = math.inf
        bad["g_y"][12, 95] = math.nan
        got = run_pass(bad)
        k, _ = ref.owners(70, *kind)
        for name, rows in (("y", (7, 40)), ("u", (7, 40)), ("g_x", (12,))):
            hit = [r for r in rows if k[r] >= 0]
            others = [r for r in range(70) if r not in hit]
            assert torch.equal(got[name][others], clean[name][others]), (batch, name)
            if hit:
                assert not torch.isfinite(got[name][hit].float()).any(), (batch, name)
        touched = {int(k[r]) for r in (7, 40, 12)}
        for j in range(t["a"].shape[0]):
            if j not in touched:
                assert torch.equal(got["g_a"][j], clean["g_a"][j]) and torch.equal(got["g_b"][j], clean["g_b"][j])
        for j in {int(k[r]) for r in (7, 40)} - {-1}:
            for name in ("g_a", "g_b"):         # a NaN stays one, an infinity times a number is one
                assert not bool(torch.isfinite(got[name][j]).all())


def test_adapter_same_bits_in_every_call_on_other_streams_and_devices_order():
    t, kind = make(700, 200, 300, 16, ([0, 100, 650], [1, 0], 2), BF16, seed=70)
    one = run_pass(t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two = run_pass(t)
    side.synchronize()
    for name in one:
        assert torch.equal(one[name], two[name]), name


def test_adapter_recorded_calls_follow_the_batch():
    """A recorded pass, replayed with other requests in the same arrays and eager work between the replays."""
    O, I, rank, L = 130, 200, 16, 64
    t, _ = make(L, O, I, rank, ([0, 20, 40, 64], [0, 1, 2], 3), BF16, seed=80)
    d = {k: v.cuda() for k, v in t.items()}
    ws = hot.alloc_adapter_workspace(d["x"], d["a"], d["b"], segments=3)
    start = {k: d[k].clone() for k in ("y", "u", "g_x")}

    def call():
        more = dict(scale=d["scale"], offsets=d["offsets"], index=d["index"])
        hot.hot_adapter_forward(d["x"], d["a"], d["b"], d["y"], ws, base=d["base"], u=d["u"], **more)
        hot.hot_adapter_backward(d["g_y"], d["x"], d["u"], d["a"], d["b"], ws, g_base=d["g_base"], g_x=d["g_x"], g_a=d["g_a"], g_b=d["g_b"], **more)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for cuts, index in (([0, 20, 40, 64], [0, 1, 2]), ([5, 5, 6, 60], [2, 2, -1]), ([0, 64, 64, 64], [1, 0, 0]), ([0, 20, 40, 64], [0, 1, 2])):
        now = dict(t, offsets=torch.tensor(cuts, dtype=torch.int32), index=torch.tensor(index, dtype=torch.int32))
        d["offsets"].copy_(now["offsets"])
        d["index"].copy_(now["index"])
        for k, v in start.items():
            d[k].copy_(v)
        eager = run_pass(now)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, want in eager.items():
            assert torch.equal(d[name], want), (cuts, name)


def test_recorded_calls_share_a_workspace():
    """Two recorded passes of adapters and one of log probabilities, all with one workspace, replayed in turn."""
    sizes = ((96, 130, 200, 16), (40, 520, 264, 24))
    made = [make(L, O, I, rank, ([0, 20, L - 3], [1, 0], 2), BF16, seed=87 + L)[0] for L, O, I, rank in sizes]
    want = [run_pass(t) for t in made]
    z = logits(2, 9000, BF16, 88).cuda()
    need = max([hot.hot_token_logprobs_workspace_bytes(BF16, 2, 9000, 5)] + [max(hot.hot_adapter_forward_workspace_bytes(BF16, *s, 2, 2),
                                                                                 hot.hot_adapter_backward_workspace_bytes(BF16, *s, 2, 2)) for s in sizes])
    ws = torch.full((need,), 255, device="cuda", dtype=torch.uint8)
    top_logp, top_ids = torch.empty(2, 5, device="cuda"), torch.empty(2, 5, device="cuda", dtype=torch.int32)
    hot.hot_token_logprobs(z, None, None, ws, top_logp=top_logp, top_ids=top_ids)
    want_top = top_logp.clone(), top_ids.clone()
    device = [{k: v.cuda() for k, v in t.items()} for t in made]

    def call(d):
        more = dict(scale=d["scale"], offsets=d["offsets"], index=d["index"])
        hot.hot_adapter_forward(d["x"], d["a"], d["b"], d["y"], ws, base=d["base"], u=d["u"], **more)
        hot.hot_adapter_backward(d["g_y"], d["x"], d["u"], d["a"], d["b"], ws, g_base=d["g_base"], g_x=d["g_x"], g_a=d["g_a"], g_b=d["g_b"], **more)

    graphs = [torch.cuda.CUDAGraph() for _ in range(3)]
    for graph, d in zip(graphs, device):
        with torch.cuda.graph(graph):
            call(d)
    with torch.cuda.graph(graphs[2]):
        hot.hot_token_logprobs(z, None, None, ws, top_logp=top_logp, top_ids=top_ids)
    for turn in ((0, 1, 2), (2, 1, 0), (1, 2, 0)):
        for d, t in zip(device, made):
            for name in ("g_a", "g_b"):
                d[name].fill_(math.nan)
            for name in ("y", "u", "g_x"):
                d[name].copy_(t[name])
        top_logp.zero_()
        top_ids.zero_()
        torch.cuda.synchronize()
        for g in turn:
            graphs[g].replay()
        torch.cuda.synchronize()
        for k in range(2):
            for name, value in want[k].items():
                assert torch.equal(device[k][name], value), (turn, k, name)
        assert torch.equal(top_logp, want_top[0]) and torch.equal(top_ids, want_top[1]), turn


def test_adapter_past_32_bits():
    """Rows whose elements lie past 2^31 of the tensors' beginning."""
    L, O, I, rank = (1 << 20) + 40, 8, 2056, 4
    x = torch.zeros(L, I, device="cuda", dtype=BF16)
    tail = rand((64, I), 1.0, 90, BF16)
    x[-64:] = tail.cuda()
    a, b = rand((1, rank, I), 0.02, 91, BF16), rand((1, O, rank), 0.3, 92, BF16)
    y, u = torch.full((L, O), 7.0, device="cuda", dtype=BF16), torch.empty(L, rank, device="cuda")
    g_y, g_x = torch.zeros(L, O, device="cuda", dtype=BF16), torch.empty(L, I, device="cuda", dtype=BF16)
    g_tail = rand((64, O), 0.1, 93, BF16)
    g_y[-64:] = g_tail.cuda()
    g_a, g_b = torch.empty(1, rank, I, device="cuda"), torch.empty(1, O, rank, device="cuda")
    ad, bd = a.cuda(), b.cuda()
    ws = hot.alloc_adapter_workspace(x, ad, bd)
    hot.hot_adapter_forward(x, ad, bd, y, ws, u=u)
    hot.hot_adapter_backward(g_y, x, u, ad, bd, ws, g_x=g_x, g_a=g_a, g_b=g_b)
    k, inside = ref.owners(64, None, None, 1)
    want = ref.adapter(tail, a, b, None, None, k, inside, torch.zeros(64, O), torch.zeros(64, rank), g_tail, None, torch.zeros(64, I))
    within("y", y[-64:], *want["y"])
    within("u", u[-64:], *want["u"])
    within("g_x", g_x[-64:], *want["g_x"])
    within("g_a", g_a, *want["g_a"])
    within("g_b", g_b, *want["g_b"])
    assert not y[:-64].any() and not u[:-64].any() and not g_x[:-64].any()


# ---- log probabilities -----------------------------------------------------------------------------------------------

def run_logprobs(z, targets, top=0, g_logp=None, g_entropy=None, in_place=False):
    rows, V = z.shape
    zd, td = z.cuda(), targets.cuda()
    r = dict(logp=torch.full((rows,), 9.0, device="cuda"), entropy=torch.full((rows,), 9.0, device="cuda"), stats=torch.full((rows, 2), 9.0, device="cuda"))
    if top:
        r["top_logp"], r["top_ids"] = torch.full((rows, top), 9.0, device="cuda"), torch.full((rows, top), -5, device="cuda", dtype=torch.int32)
    ws = hot.alloc_logprobs_workspace(zd, top)
    if ws is not None:
        ws.fill_(255)
    hot.hot_token_logprobs(zd, td, r["logp"], ws, entropy=r["entropy"], stats=r["stats"], top_logp=r.get("top_logp"), top_ids=r.get("top_ids"))
    if g_logp is not None or g_entropy is not None:
        out = zd if in_place else torch.full_like(zd, 9.0)
        r["g_logits"] = hot.hot_token_logprobs_backward(
            zd, None if g_logp is None else td, r["stats"], out, g_logp=None if g_logp is None else g_logp.cuda(),
            entropy=None if g_entropy is None else r["entropy"], g_entropy=None if g_entropy is None else g_entropy.cuda())
    return r


def logits(rows, V, dtype, seed, std=3.0, masked=0):
    z = rand((rows, V), std, seed)
    z[::3, V // 2] += 25.0
    if masked:
        z[:, V - masked:] = -math.inf
    return z.to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,top", [(1, 1, 1), (1, 7, 7), (2, 63, 5), (5, 2047, 32), (3, 2049, 20), (1, 50257, 20), (70, 6151, 8), (1100, 4100, 4), (2100, 300, 1)])
def test_logprobs_and_gradient(rows, V, top, dtype):
    z = logits(rows, V, dtype, rows + V, masked=3 if V > 100 else 0)
    targets = torch.randint(-1, V + 1, (rows,), generator=torch.Generator().manual_seed(1))      # -1 and V: not scored
    gl, ge = rand((rows,), 1.0, 2), rand((rows,), 0.3, 3)
    want = ref.logprobs(z, targets, top, gl, ge)
    got = run_logprobs(z, targets, top, gl, ge)
    for name in ("logp", "entropy", "stats", "top_logp", "g_logits"):
        within(name, got[name], *want[name])
    assert torch.equal(got["top_ids"].cpu().long(), want["top_ids"])
    same = run_logprobs(z, targets, 0, gl, ge, in_place=True)
    assert torch.equal(same["g_logits"], got["g_logits"]) and torch.equal(same["entropy"], got["entropy"])
    for one in (dict(g_logp=gl), dict(g_entropy=ge)):
        within("g_logits", run_logprobs(z, targets, 0, **one)["g_logits"], *ref.logprobs(z, targets, 0, **one)["g_logits"])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(1, 9000), (2100, 900)])
def test_top_of_equal_and_masked_tokens(rows, V, dtype):
    """Ties go to the lower token; rows with fewer finite logits than are asked for; masks of the type's lowest value."""
    z = torch.zeros(rows, V)
    z[:, 5] = -0.0
    targets = torch.zeros(rows, dtype=torch.int64)
    got = run_logprobs(z.to(dtype), targets, 32)
    assert torch.equal(got["top_ids"].cpu(), torch.arange(32, dtype=torch.int32).expand(rows, 32))
    within("logp", got["logp"], torch.full((rows,), -math.log(V), dtype=torch.float64), torch.full((rows,), 1e-5, dtype=torch.float64))
    z = torch.full((rows, V), -math.inf)
    z[:, 77], z[:, 800], z[:, 30] = 1.0, 2.0, 1.0
    got = run_logprobs(z.to(dtype), targets, 6)
    assert got["top_ids"][0].tolist() == [800, 30, 77, 0, 1, 2] and (got["top_logp"][:, 3:] == -math.inf).all() and (got["logp"] == -math.inf).all()
    lowest = torch.finfo(dtype).min
    z = torch.full((rows, V), lowest)
    z[:, 3] = 0.0
    got = run_logprobs(z.to(dtype), targets + 3, 2, rand((rows,), 1.0, 1), rand((rows,), 1.0, 2))
    assert (got["logp"] == 0).all() and (got["entropy"] == 0).all() and got["top_ids"][0].tolist() == [3, 0] and not got["g_logits"].any()
    got = run_logprobs(torch.full((rows, V), lowest, dtype=dtype), targets, 2)
    within("entropy", got["entropy"], torch.full((rows,), math.log(V), dtype=torch.float64), torch.full((rows,), 1e-5, dtype=torch.float64))
    big = torch.full((rows, V), -torch.finfo(dtype).max)
    big[:, 1] = torch.finfo(dtype).max
    got = run_logprobs(big.to(dtype), targets + 1, 1, rand((rows,), 1.0, 1), rand((rows,), 1.0, 2))
    assert (got["logp"] == 0).all() and not got["g_logits"].any()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [9000, 500])
def test_rows_without_tokens_and_with_nans(V, dtype):
    rows = 6
    z = logits(rows, V, dtype, 5)
    targets, gl, ge = torch.arange(rows), rand((rows,), 1.0, 1), rand((rows,), 1.0, 2)
    clean = run_logprobs(z, targets, 5, gl, ge)
    z[1] = -math.inf
    z[2, 400], z[2, 100] = math.nan, math.nan
    z[4, 300] = math.inf
    got = run_logprobs(z, targets, 5, gl, ge)
    for name in clean:
        assert torch.equal(got[name][[0, 3, 5]], clean[name][[0, 3, 5]]), name
    assert got["logp"][1] == -math.inf and got["entropy"][1] == 0 and got["stats"][1].tolist() == [-math.inf, 0.0]
    assert not got["g_logits"][1].any() and got["top_ids"][1].tolist() == [0, 1, 2, 3, 4] and (got["top_logp"][1] == -math.inf).all()
    for r in (2, 4):
        assert got["logp"][r].isnan() and got["entropy"][r].isnan() and got["g_logits"][r].isnan().all() and got["top_logp"][r].isnan().all()
    assert got["top_ids"][2].tolist()[:2] == [100, 400] and got["top_ids"][4, 0] == 300


def test_logprobs_recorded_and_on_a_stream():
    z = logits(5, 7000, BF16, 9)
    targets = torch.arange(5)
    zd, td = z.cuda(), targets.cuda()
    out = {k: torch.empty(s, device="cuda", dtype=t) for k, s, t in (("logp", (5,), F32), ("entropy", (5,), F32), ("stats", (5, 2), F32), ("top_logp", (5, 4), F32),
                                                                     ("top_ids", (5, 4), torch.int32), ("g", (5, 7000), BF16))}
    gl, ge = rand((5,), 1.0, 1).cuda(), rand((5,), 1.0, 2).cuda()
    ws = hot.alloc_logprobs_workspace(zd, 4)

    def call():
        hot.hot_token_logprobs(zd, td, out["logp"], ws, entropy=out["entropy"], stats=out["stats"], top_logp=out["top_logp"], top_ids=out["top_ids"])
        hot.hot_token_logprobs_backward(zd, td, out["stats"], out["g"], g_logp=gl, entropy=out["entropy"], g_entropy=ge)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (9, 10, 11, 9):
        z = logits(5, 7000, BF16, seed)
        zd.copy_(z)
        eager = run_logprobs(z, targets, 4, gl.cpu(), ge.cpu())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("logp", "entropy", "stats", "top_logp", "top_ids"):
            assert torch.equal(out[name], eager[name]), name
        assert torch.equal(out["g"], eager["g_logits"])


def test_logprobs_past_32_bits():
    rows, V = 70000, 32008
    z = torch.zeros(rows, V, device="cuda", dtype=BF16)
    tail = logits(4, V, BF16, 12)
    z[-4:] = tail.cuda()
    targets = torch.zeros(rows, dtype=torch.int64, device="cuda")
    gl, ge = rand((rows,), 1.0, 1), rand((rows,), 1.0, 2)
    logp, entropy, stats, g = (torch.empty(s, device="cuda") for s in ((rows,), (rows,), (rows, 2), (1,)))
    hot.hot_token_logprobs(z, targets, logp, entropy=entropy, stats=stats)
    want = ref.logprobs(tail, targets[-4:].cpu(), 0, gl[-4:], ge[-4:])
    within("logp", logp[-4:], *want["logp"])
    within("entropy", entropy[-4:], *want["entropy"])
    hot.hot_token_logprobs_backward(z, targets, stats, z, g_logp=gl.cuda(), entropy=entropy, g_entropy=ge.cuda())
    within("g_logits", z[-4:], *want["g_logits"])


# ---- optimiser -------------------------------------------------------------------------------------------------------

def moments_of(n, seed, form):
    """A pair of moments as fp32 values, and the buffers that hold them."""
    g = np.random.default_rng(seed)
    m = (g.standard_normal(n) * np.exp(g.standard_normal(n) * 3)).astype(np.float32) * np.float32(1e-3)
    v = np.square(g.standard_normal(n).astype(np.float32) * np.float32(1e-2)) * np.exp(g.standard_normal(n) * 4).astype(np.float32)
    m[::7] = 0
    v[::11] = 0
    if form == "f32":
        return m, v, torch.from_numpy(m.copy()), torch.from_numpy(v.copy())
    pad = -n % 1024
    mp, vp = np.pad(m, (0, pad)), np.pad(v, (0, pad))
    (cm, em), (cv, ev) = ref.held_m(mp, True), ref.held_v(vp, True)
    return (ref.read_m(cm, em)[:n], ref.read_v(cv, ev)[:n], torch.from_numpy(ref.pack_state(cm, em)), torch.from_numpy(ref.pack_state(cv, ev)))


def as_np(t):
    return t.float().numpy()


def expected_state(x, form, moment, nearest):
    if form == "f32":
        return torch.from_numpy(x)
    xp = np.pad(x, (0, -len(x) % 1024))
    c, e = (ref.held_m if moment == "m" else ref.held_v)(xp, nearest)
    return torch.from_numpy(ref.pack_state(c, e))


SIZES = [1, 7, 31, 33, 1000, 1023, 1024, 1025, 2047, 2049, 4096, 70001]


@pytest.mark.parametrize("form", ["f32", "8bit"])
@pytest.mark.parametrize("pt,gt,copy", [(F32, F32, False), (F32, F32, True), (F32, BF16, True), (BF16, BF16, False), (BF16, F32, False)])
@pytest.mark.parametrize("nearest", [False, True], ids=["stochastic", "nearest"])
def test_adamw_step(form, pt, gt, copy, nearest):
    """More tensors than a launch takes, of all lengths; results beside the inputs, moments to the bit."""
    sizes = SIZES * 4
    lr, b1, b2, eps, step = 1e-2, 0.9, 0.995, 1e-8, 3
    host, dev = [], []
    for i, n in enumerate(sizes):
        m, v, mb, vb = moments_of(n, 100 + i, form)
        p, g = rand((n,), 0.5, i, pt), rand((n,), 1e-2, 1000 + i, gt)
        t = dict(param=p, grad=g, m=mb, v=vb, param_out=torch.full_like(p, 9.0), m_out=torch.full_like(mb, 9), v_out=torch.full_like(vb, 9),
                 copy=torch.full((n,), 9.0, dtype=BF16) if copy else None, weight_decay=0.1 * (i % 3), lr_factor=1.0 + i % 2)
        host.append((t, m, v))
        dev.append({k: x.cuda() if isinstance(x, torch.Tensor) else x for k, x in t.items()})
    tensors = hot.AdamWTensors(dev, state=form)
    rounding = hot.HOT_ROUND_NEAREST_EVEN if nearest else hot.HOT_ROUND_PSEUDO_STOCHASTIC
    hot.hot_adamw_step(tensors, lr, b1, b2, eps, step, rounding=rounding)
    torch.cuda.synchronize()
    for (t, m, v), d in zip(host, dev):
        m2, v2 = ref.moments(m, v, as_np(t["grad"]), b1, b2)
        assert torch.equal(d["m_out"].cpu(), expected_state(m2, form, "m", nearest)), len(m)
        assert torch.equal(d["v_out"].cpu(), expected_state(v2, form, "v", nearest)), len(v)
        w, err = ref.weights(as_np(t["param"]), m2, v2, lr * t["lr_factor"], t["weight_decay"], 1 - b1 ** step, 1 - b2 ** step, eps)
        w, err = torch.from_numpy(w), torch.from_numpy(err)
        within("param", d["param_out"], w, err + (ref.HALF[BF16] * (w.abs() + err) if pt == BF16 else 0))
        if copy:
            assert torch.equal(d["copy"], d["param_out"].to(BF16))
        for name in ("param", "grad", "m", "v"):
            assert torch.equal(d[name].cpu(), t[name])
    # in place: the same
    for d in dev:
        for name in ("param_out", "m_out", "v_out"):
            d[name + "_was"] = d.pop(name)
    hot.hot_adamw_step(hot.AdamWTensors(dev, state=form), lr, b1, b2, eps, step, rounding=rounding)
    for d in dev:
        assert torch.equal(d["param"], d["param_out_was"]) and torch.equal(d["m"], d["m_out_was"]) and torch.equal(d["v"], d["v_out_was"])


def test_adamw_first_steps_from_zero_states_follow_the_formula():
    """Ten steps from nothing with 8-bit moments: within the rounding of the moments of the 64-bit steps."""
    n = 5000
    p = rand((n,), 0.5, 1)
    w, m, v = p.double(), torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    for form, tol in (("f32", 1e-5), ("8bit", 0.2)):
        d = dict(param=p.cuda(), grad=torch.empty(n, device="cuda"), m=hot.alloc_adamw_state(form, n), v=hot.alloc_adamw_state(form, n))
        tensors = hot.AdamWTensors([d], state=form)
        w, m, v = p.double(), torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
        for step in range(1, 11):
            g = rand((n,), 1.0, 50 + step)
            d["grad"].copy_(g)
            hot.hot_adamw_step(tensors, 1e-3, 0.9, 0.99, 1e-8, step)
            m = 0.9 * m + 0.1 * g.double()
            v = 0.99 * v + 0.01 * g.double() ** 2
            w = w - 1e-3 * (m / (1 - 0.9 ** step)) / (torch.sqrt(v / (1 - 0.99 ** step)) + 1e-8)
        moved = (w - p.double()).norm()
        # each of the ten steps rounds the weights twice, u = 2^-24 of themselves at most
        off = float((d["param"].double().cpu() - w).norm())
        assert off <= tol * float(moved) + 20 * ref.U * float(p.double().norm()), form


@pytest.mark.parametrize("form", ["f32", "8bit"])
def test_adamw_recorded_steps_read_their_numbers(form):
    n = 3000
    m, v, mb, vb = moments_of(n, 7, form)
    p = rand((n,), 0.5, 1)
    d = dict(param=p.cuda(), grad=rand((n,), 1e-2, 2).cuda(), m=mb.cuda(), v=vb.cuda(), weight_decay=0.1)
    e = {k: x.clone() if isinstance(x, torch.Tensor) else x for k, x in d.items()}
    e["grad"] = d["grad"]
    dynamic = torch.tensor([1e-3, 0.1, 0.01, 1.0], device="cuda")
    recorded, eager = hot.AdamWTensors([d], state=form), hot.AdamWTensors([e], state=form)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        hot.hot_adamw_step(recorded, 0.0, 0.9, 0.99, 1e-8, dynamic=dynamic)
    del recorded                                          # the table is not read again
    for step, (lr, factor) in enumerate(((1e-3, 1.0), (2e-3, 0.5), (5e-4, 1.0), (5e-4, 1.0)), 1):
        c1, c2 = 1 - 0.9 ** step, 1 - 0.99 ** step
        dynamic.copy_(torch.tensor([lr, c1, c2, factor]))
        d["grad"].copy_(rand((n,), 1e-2, 10 + step))
        graph.replay()
        g = d["grad"].clone()
        torch.cuda.synchronize()
        d["grad"].mul_(factor)
        hot.hot_adamw_step(eager, lr, 0.9, 0.99, 1e-8, step)
        for name in ("param", "m", "v"):
            assert torch.equal(d[name], e[name]), (step, name)
        d["grad"].copy_(g)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_adamw_state_as_values(dtype):
    for n in SIZES:
        m, v, mb, vb = moments_of(n, n, "8bit")
        for moment, x, buf in (("m", m, mb), ("v", v, vb)):
            out = torch.empty(n, device="cuda", dtype=dtype)
            assert torch.equal(hot.hot_adamw_state_read(buf.cuda(), moment, out).cpu().float(), torch.from_numpy(x))
            raw = (rand((n,), 1.0, n) * torch.exp(3 * rand((n,), 1.0, n + 1))).to(dtype)
            raw = raw.abs() if moment == "v" else raw
            back = torch.full((hot.hot_adamw_state_bytes("8bit", n),), 77, dtype=torch.uint8, device="cuda")
            hot.hot_adamw_state_write(raw.cuda(), moment, back)
            assert torch.equal(back.cpu(), expected_state(as_np(raw), "8bit", moment, True))


@pytest.mark.parametrize("form", ["f32", "8bit"])
def test_adamw_marks_what_is_not_finite(form):
    """An infinity or a NaN stays in its element, or, in 8 bits, in its group of 32; the largest numbers are held."""
    n = 2100
    m, v, mb, vb = moments_of(n, 7, form)
    p, g = rand((n,), 0.5, 1), rand((n,), 1e-2, 2)
    g[40], g[1100], g[70] = math.nan, math.inf, 3e19
    d = dict(param=p.cuda(), grad=g.cuda(), m=mb.cuda(), v=vb.cuda())
    hot.hot_adamw_step(hot.AdamWTensors([d], state=form), 1e-3)
    bad = torch.zeros(n, dtype=torch.bool)
    bad[[40, 1100, 70]] = True
    weights = d["param"].cpu()
    assert torch.isfinite(weights[~bad]).all() and weights[40].isnan() and weights[1100].isnan()
    if form == "8bit":
        for moment, hit in (("m", (40, 1100)), ("v", (40, 1100, 70))):
            x = hot.hot_adamw_state_read(d[moment], moment, torch.empty(n, device="cuda")).cpu()
            group = torch.zeros(n, dtype=torch.bool)
            for i in hit:
                if not (i == 70 and math.isfinite(float(np.float32(1e-3) * np.float32(9e38 / 10)))):
                    group[i // 32 * 32:i // 32 * 32 + 32] = True
            if moment == "v":
                group[64:96] = x[64:96].isnan()
            assert torch.equal(x.isnan(), group), moment


def test_adamw_past_32_bits():
    n = (1 << 31) + 5000
    p = torch.zeros(n, device="cuda", dtype=BF16)
    g = torch.zeros(n, device="cuda", dtype=BF16)
    tail = 4096 + 5000 % 1024
    first = n - tail
    assert first % 1024 == 0
    p[first:], g[first:] = rand((tail,), 0.5, 1, BF16).cuda(), rand((tail,), 1e-2, 2, BF16).cuda()
    big = dict(param=p, grad=g, m=hot.alloc_adamw_state("8bit", n), v=hot.alloc_adamw_state("8bit", n))
    small = dict(param=p[first:].clone(), grad=g[first:].clone(), m=hot.alloc_adamw_state("8bit", tail), v=hot.alloc_adamw_state("8bit", tail))
    hot.hot_adamw_step(hot.AdamWTensors([big], state="8bit"), 1e-2)
    hot.hot_adamw_step(hot.AdamWTensors([small], state="8bit"), 1e-2)
    at = first // 1024 * 1056
    assert torch.equal(big["param"][first:], small["param"]) and not big["param"][:first].any()
    assert torch.equal(big["m"][at:], small["m"]) and torch.equal(big["v"][at:], small["v"])
    x = hot.hot_adamw_state_read(big["m"], "m", p)
    assert torch.equal(x[first:], hot.hot_adamw_state_read(small["m"], "m", torch.empty(tail, device="cuda", dtype=BF16)))


# ---- together --------------------------------------------------------------------------------------------------------

def test_fine_tuning_step_with_frozen_weights():
    """Adapters beside a frozen projection: forward product, adapters, a frozen head, log probabilities, their gradient, the frozen
    weights' gradients of the stream, the adapters' gradients, the optimiser; against the same step in 64 bits."""
    L, I, O, V, rank, n = 256, 128, 160, 320, 8, 16
    x, w, head = rand((L, I), 1.0, 1), rand((O, I), 0.05, 2), rand((V, O), 0.1, 3)
    a, b = rand((1, rank, I), 0.1, 4), rand((1, O, rank), 0.1, 5)
    scale = torch.tensor([2.0])
    targets = torch.randint(0, V, (L,), generator=torch.Generator().manual_seed(6))
    d = {k: t.cuda() for k, t in dict(x=x, w=w, head=head, a=a, b=b, scale=scale, targets=targets).items()}
    z0, z, logits_ = (torch.empty(L, O, device="cuda"), torch.empty(L, O, device="cuda"), torch.empty(L, V, device="cuda"))
    u, logp, stats, g_logits = (torch.empty(s, device="cuda") for s in ((L, rank), (L,), (L, 2), (L, V)))
    ws = hot.alloc_adapter_workspace(d["x"], d["a"], d["b"])
    hot.hot_linear_forward(d["x"], d["w"], z0, hot.alloc_linear_workspace(F32, L, O, I))
    hot.hot_adapter_forward(d["x"], d["a"], d["b"], z, ws, scale=d["scale"], base=z0, u=u)
    hot.hot_linear_forward(z, d["head"], logits_, hot.alloc_linear_workspace(F32, L, V, O))
    hot.hot_token_logprobs(logits_, d["targets"], logp, hot.alloc_logprobs_workspace(logits_), stats=stats)
    g_logp = torch.full((L,), -1.0 / L, device="cuda")
    hot.hot_token_logprobs_backward(logits_, d["targets"], stats, g_logits, g_logp=g_logp)
    cfg = hot.Config(block=n, gx_bits=8)
    hws = hot.alloc_workspace(cfg, L, V, O)
    g_z = torch.empty(L, O, device="cuda")
    hot.hot_linear_backward_gx(cfg, g_logits, d["head"], hot.HOT_Q_PER_TOKEN, g_z, hws)
    g_a, g_b = torch.empty_like(d["a"]), torch.empty_like(d["b"])
    g_x = torch.empty(L, I, device="cuda")
    hot.hot_linear_backward_gx(cfg, g_z, d["w"], hot.HOT_Q_PER_TOKEN, g_x, hot.alloc_workspace(cfg, L, O, I))
    hot.hot_adapter_backward(g_z, d["x"], u, d["a"], d["b"], ws, scale=d["scale"], g_base=g_x, g_x=g_x, g_a=g_a, g_b=g_b)
    was = {k: d[k].clone() for k in "ab"}
    tensors = hot.AdamWTensors([dict(param=d[k], grad=g, m=hot.alloc_adamw_state("8bit", g.numel()), v=hot.alloc_adamw_state("8bit", g.numel()), weight_decay=0.01)
                                for k, g in (("a", g_a), ("b", g_b))], state="8bit")
    hot.hot_adamw_step(tensors, 1e-3)
    # 64 bits
    X, A, B = x.double().requires_grad_(True), a.double().requires_grad_(True), b.double().requires_grad_(True)
    Z = X @ w.double().T + 2.0 * (X @ A[0].T) @ B[0].T
    lp = torch.log_softmax(Z @ head.double().T, 1)[torch.arange(L), targets]
    (-lp.mean()).backward()
    assert (logp.double().cpu() - lp.detach()).abs().max() < 1e-4
    # INT8 rotated operands of the two frozen products: their rounding is one part in 254 of a row's largest value
    for got, t in ((g_a, A), (g_b, B), (g_x, X)):
        assert (got.double().cpu() - t.grad).norm() < 0.03 * t.grad.norm()
    for k, g in (("a", g_a), ("b", g_b)):
        p, gd = was[k].double(), g.double()
        want = p - 1e-3 * (0.01 * p + gd / (gd.abs() + 1e-8))
        assert (d[k].double() - want).abs().max() < 1e-6
