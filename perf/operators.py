"""Performance cases of the operators around the linear-layer backward: what a training step of a transformer block
runs beside ``hot_linear_backward``.

A case is one pass through one of them:

- ``checkpoint``: a tensor stored in 8 bits and read back (``hot_checkpoint_write``, ``hot_checkpoint_read``);
- ``activation``: a point-wise activation and its gradient, the input kept in 8 bits between the two, with the
  gradient of the bias in front of it (``hot_activation_forward``, ``hot_activation_backward``);
- ``norm``: a layer norm and its gradients, with or without the residual addition in front of it and with its input
  kept in 8 bits or as it is (``hot_layer_norm_forward``, ``hot_layer_norm_backward``);
- ``linear``: x.w^T with bias, activation and residual in its epilogue (``hot_linear_forward``), and, where its
  pre-activation is kept in 8 bits, the gradient through the activation.

Sizes are those of the benchmark's layers and of the tests, or lie between them; ``draw`` spreads over the same ranges.
"""
import math
import zlib

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
GROUP = 32     # columns that share a step in the 8-bit form
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _checkpoint(rows, cols, x="f32"):
    return dict(kind="checkpoint", rows=rows, cols=cols, x=x)


def _activation(rows, cols, x="f32", fn="gelu", bias=True):
    return dict(kind="activation", rows=rows, cols=cols, x=x, fn=fn, bias=bias)


def _norm(rows, cols, x="f32", y="f32", residual=False, kept=False):
    return dict(kind="norm", rows=rows, cols=cols, x=x, y=y, residual=residual, kept=kept)


def _linear(rows, out, cols, x="f32", y="f32", fn="none", bias=True, residual=False, kept=False):
    return dict(kind="linear", rows=rows, out=out, cols=cols, x=x, y=y, fn=fn, bias=bias, residual=residual, kept=kept)


def listed():
    return [
        # Attention outputs of 64 ViT-B images, kept for the backward pass of what follows them.
        dict(_checkpoint(64 * 197, 768), name="kept_64_images_vitb"),
        # Nothing a multiple of anything: ten sequences of 333 tokens, an odd width, bfloat16.
        dict(_checkpoint(3330, 771, x="bf16"), name="kept_ragged_bf16"),
        # GELU of a mobile vision transformer's MLP at its 7 x 7 stage, 64 images.
        dict(_activation(64 * 49, 1792), name="gelu_49_tokens_64_images"),
        # The activation of an LLM MLP, 8 x 2048 tokens, in bfloat16.
        dict(_activation(16384, 11008, x="bf16", fn="silu"), name="silu_llm_16384_tokens_bf16"),
        # One ViT-B image: bound by launches and latencies.
        dict(_norm(197, 768), name="norm_1_image_vitb"),
        # ViT-L at batch 1024: the large streams, with the residual addition and the input kept in 8 bits.
        dict(_norm(1024 * 197, 1024, residual=True, kept=True), name="norm_1024_images_vitl_kept"),
        # LLM width, 8 x 2048 tokens: an fp32 residual stream, bfloat16 operands for the product that follows.
        dict(_norm(16384, 4096, y="bf16", residual=True), name="norm_llm_16384_tokens_mixed"),
        # An odd width, rows that are not whole vectors.
        dict(_norm(3330, 771, kept=True), name="norm_ragged_kept"),
        # One token through the LLM down-projection: the weight is read once, nothing else counts.
        dict(_linear(1, 4096, 11008, x="bf16", y="bf16", residual=True), name="down_1_token_bf16"),
        # One ViT-B image through a projection in fp32.
        dict(_linear(197, 768, 768, residual=True), name="proj_1_image_f32"),
        # ViT-B qkv at batch 64 in fp32.
        dict(_linear(64 * 197, 2304, 768), name="qkv_64_images_f32"),
        # LLM up-projection, 8 x 2048 tokens, GELU in the epilogue, the pre-activation kept in 8 bits, and its gradient.
        dict(_linear(16384, 11008, 4096, x="bf16", y="bf16", fn="gelu", kept=True), name="up_16384_tokens_bf16_kept"),
    ]


def _kept_bytes(rows, cols):
    groups = -(-cols // GROUP)
    return rows * groups * (GROUP + 1)


def work(case):
    """Compulsory traffic (each operand in once, each result out once; what is kept for the backward pass out in the
    forward and in again in the backward) and arithmetic of one pass."""
    kind, L, C = case["kind"], case["rows"], case["cols"]
    sx = SIZE[case["x"]]
    if kind == "checkpoint":
        return {"bytes": 2 * (L * C * sx + _kept_bytes(L, C)), "flops": 4 * L * C}
    if kind == "activation":
        return {"bytes": 4 * L * C * sx + 2 * _kept_bytes(L, C) + 4 * C * case["bias"], "flops": 40 * L * C}
    if kind == "norm":
        sy = SIZE[case["y"]]
        forward = L * C * (sx + sy) + (2 * L * C * sx if case["residual"] else 0) + 8 * C + 8 * L
        backward = L * C * (sy + sx) + (L * C * sx if case["residual"] else 0) + 12 * C + 8 * L
        kept = 2 * _kept_bytes(L, C) if case["kept"] else L * C * sx
        return {"bytes": forward + backward + kept, "flops": 20 * L * C}
    O, sy = case["out"], SIZE[case["y"]]
    moved = (L * C + O * C) * sx + L * O * sy * (2 if case["residual"] else 1) + 4 * O * case["bias"]
    if case["kept"]:
        moved += 2 * _kept_bytes(L, O) + 2 * L * O * sy
    return {"bytes": moved, "flops": 2 * L * O * C}


def _cost(case):
    """Microseconds of the plain form at round rates, to keep drawn cases below the largest listed ones."""
    w = work(case)
    return w["bytes"] / 1e6 + (w["flops"] / 1e8 if case["kind"] == "linear" else 0)


def draw(rng):
    limit = {kind: max(_cost(c) for c in listed() if c["kind"] == kind) for kind in ("activation", "norm", "linear")}
    limit["checkpoint"] = limit["activation"]

    def spread(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    def width():
        n = spread(64, 11008)
        return max(64, n // 64 * 64) if rng.random() < 0.6 else n

    while True:
        kind = rng.choice(["checkpoint", "activation", "activation", "norm", "norm", "linear", "linear", "linear"])
        rows, cols, x = spread(1, 201728), width(), rng.choice(["f32", "f32", "bf16"])
        if kind == "checkpoint":
            case = _checkpoint(rows, cols, x)
        elif kind == "activation":
            case = _activation(rows, cols, x, rng.choice(["gelu", "gelu", "gelu_tanh", "silu", "relu"]), rng.random() < 0.7)
        elif kind == "norm":
            y = "bf16" if x == "bf16" else rng.choice(["f32", "f32", "bf16"])
            case = _norm(rows, cols, x, y, rng.random() < 0.5, rng.random() < 0.5)
        else:
            y = rng.choice(["bf16", "f32"]) if x == "bf16" else "f32"
            kept = y == "bf16" and rng.random() < 0.4
            fn = rng.choice(["gelu", "gelu_tanh", "silu"]) if kept else rng.choice(["none", "none", "gelu", "gelu_tanh", "silu", "relu"])
            case = _linear(rows, width(), cols, x, y, fn, rng.random() < 0.7, not kept and rng.random() < 0.5, kept)
        if _cost(case) <= limit[kind]:
            return case


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _normal(shape, std, seed, name, dtype=torch.float32):
    g = torch.Generator(device=DEVICE)
    g.manual_seed((int(seed) * 1_000_003 + zlib.crc32(name.encode())) & 0x7FFF_FFFF_FFFF)
    t = torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)
    return t.mul_(std).to(dtype)


def _stream(rows, cols, seed, name, dtype):
    """Values of a residual stream: a Gaussian bulk, a mean per column, one column in a hundred twenty times as large."""
    t = _normal((rows, cols), 1.0, seed, name)
    scale = torch.ones(cols, device=DEVICE)
    scale[(seed * 7) % 100::100] = 20.0
    t.mul_(scale).add_(_normal((cols,), 0.3, seed, name + ".mean"))
    return t.to(dtype)


def prepare(case, seed):
    """Inputs, and the output buffers that the caller owns."""
    kind, L, C, tx = case["kind"], case["rows"], case["cols"], TYPES[case["x"]]
    s = {"case": case, "scratch": {}}

    def out(name, *shape, dtype=torch.float32):
        s[name] = torch.empty(shape, device=DEVICE, dtype=dtype)

    if kind == "checkpoint":
        s["x"] = _stream(L, C, seed, "x", tx)
        out("back", L, C, dtype=tx)
    elif kind == "activation":
        s["x"] = _normal((L, C), 1.5, seed, "x", tx)
        s["g_y"] = _normal((L, C), 1e-3, seed, "g_y", tx)
        out("y", L, C, dtype=tx)
        out("g_x", L, C, dtype=tx)
        out("g_bias", C)
    elif kind == "norm":
        ty = TYPES[case["y"]]
        s["x"] = _stream(L, C, seed, "x", tx)
        s["gamma"] = _normal((C,), 0.2, seed, "gamma").add_(1.0)
        s["beta"] = _normal((C,), 0.1, seed, "beta")
        s["g_y"] = _normal((L, C), 1e-3, seed, "g_y", ty)
        out("y", L, C, dtype=ty)
        out("mean", L)
        out("rstd", L)
        out("g_x", L, C, dtype=tx)
        out("g_gamma", C)
        out("g_beta", C)
        if case["residual"]:
            s["residual"] = _normal((L, C), 1.0, seed, "residual", tx)
            s["g_residual"] = _normal((L, C), 1e-3, seed, "g_residual", tx)
            out("h", L, C, dtype=tx)
    else:
        O, ty = case["out"], TYPES[case["y"]]
        s["x"] = _normal((L, C), 1.0, seed, "x", tx)
        s["w"] = _normal((O, C), 1.0 / math.sqrt(C), seed, "w", tx)
        s["bias"] = _normal((O,), 0.1, seed, "bias") if case["bias"] else None
        s["residual"] = _normal((L, O), 1.0, seed, "residual", ty) if case["residual"] else None
        out("y", L, O, dtype=ty)
        if case["kept"]:
            s["g_y"] = _normal((L, O), 1e-3, seed, "g_y", ty)
            out("g_z", L, O, dtype=ty)
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _stored(x):
    """fp32 values of x as the 8-bit form holds them: one power of two for 32 columns of a row, the smallest that leaves
    the group's largest value within 127 steps."""
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    t = torch.nn.functional.pad(x, (0, groups * GROUP - cols)).view(rows, groups, GROUP)
    top = t.abs().amax(-1, keepdim=True).view(torch.int32)
    e = ((top + 0x10000) >> 23).clamp(8, 254)
    step, inverse = ((e - 6) << 23).view(torch.float32), ((260 - e) << 23).view(torch.float32)
    t = (t * inverse).round().clamp(-127, 127) * step
    return t.view(rows, groups * GROUP)[:, :cols]


def _act(fn, x):
    if fn == "none":
        return x
    if fn == "relu":
        return x.clamp(min=0)
    if fn == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if fn == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return x / (1 + torch.exp(-x))


def _act_slope(fn, x):
    if fn == "relu":
        return (x > 0).to(x.dtype)
    if fn == "gelu":
        return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    if fn == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (x + 0.044715 * x * x * x))
        return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * a * (1 + 3 * 0.044715 * x * x)
    p = 1 / (1 + torch.exp(-x))
    return p * (1 + x * (1 - p))


def _plain(s):
    case = s["case"]
    kind, x = case["kind"], s["x"].float()
    if kind == "checkpoint":
        return _stored(x).to(s["x"].dtype)
    if kind == "activation":
        fn, t = case["fn"], s["x"].dtype
        g = s["g_y"].float() * _act_slope(fn, _stored(x))
        return {"y": _act(fn, x).to(t), "g_x": g.to(t), "g_bias": g.sum(0) if case["bias"] else None}
    if kind == "norm":
        h, r = x, {}
        if case["residual"]:
            r["h"] = (x + s["residual"].float()).to(s["x"].dtype)
            h = r["h"].float()
        mean = h.mean(1)
        centred = h - mean[:, None]
        rstd = 1 / torch.sqrt((centred * centred).mean(1) + EPS)
        r.update(y=(centred * rstd[:, None] * s["gamma"] + s["beta"]).to(s["y"].dtype), mean=mean, rstd=rstd)
        g = s["g_y"].float()
        n = ((_stored(h) - mean[:, None]) if case["kept"] else centred) * rstd[:, None]
        t = g * s["gamma"]
        g_x = rstd[:, None] * (t - t.mean(1, keepdim=True) - n * (t * n).mean(1, keepdim=True))
        if case["residual"]:
            g_x = g_x + s["g_residual"].float()
        r.update(g_x=g_x.to(s["x"].dtype), g_gamma=(g * n).sum(0), g_beta=g.sum(0))
        return r
    z = x @ s["w"].float().t()
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _act(case["fn"], z)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    r = {"y": y.to(s["y"].dtype)}
    if case["kept"]:
        r["g_z"] = (s["g_y"].float() * _act_slope(case["fn"], _stored(z))).to(s["y"].dtype)
    return r


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _kernels(s):
    import paper_2503_21261_amd as hot

    case, x, keep = s["case"], s["x"], s["scratch"]
    kind = case["kind"]

    def scratch(name, make):     # what a user's program allocates once for its shapes
        if name not in keep:
            keep[name] = make()
        return keep[name]

    if kind == "checkpoint":
        buf = scratch("kept", lambda: hot.alloc_checkpoint(*x.shape))
        hot.hot_checkpoint_write(x, buf)
        return hot.hot_checkpoint_read(buf, s["back"])
    if kind == "activation":
        fn = hot.ACT_FNS[case["fn"]]
        buf = scratch("kept", lambda: hot.alloc_checkpoint(*x.shape))
        g_bias = s["g_bias"] if case["bias"] else None
        ws = scratch("ws", lambda: hot.alloc_activation_workspace(*x.shape)) if case["bias"] else None
        hot.hot_activation_forward(fn, x, s["y"], ckpt=buf)
        hot.hot_activation_backward(fn, s["g_y"], s["g_x"], ckpt=buf, g_bias=g_bias, ws=ws)
        return {"y": s["y"], "g_x": s["g_x"], "g_bias": g_bias}
    if kind == "norm":
        buf = scratch("kept", lambda: hot.alloc_checkpoint(*x.shape)) if case["kept"] else None
        ws = scratch("ws", lambda: hot.alloc_layer_norm_workspace(*x.shape))
        r, h = {}, x
        if case["residual"]:
            h = r["h"] = s["h"]
        hot.hot_layer_norm_forward(x, s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"],
                                   residual=s.get("residual"), h=r.get("h"), ckpt=buf)
        hot.hot_layer_norm_backward(s["g_y"], s["gamma"], s["mean"], s["rstd"], s["g_x"], s["g_gamma"], s["g_beta"], ws,
                                    h=None if case["kept"] else h, ckpt=buf, g_residual=s.get("g_residual"))
        r.update({k: s[k] for k in ("y", "mean", "rstd", "g_x", "g_gamma", "g_beta")})
        return r
    fn = hot.ACT_FNS[case["fn"]]
    buf = scratch("kept", lambda: hot.alloc_checkpoint(*s["y"].shape)) if case["kept"] else None
    ws = scratch("ws", lambda: hot.alloc_linear_workspace(x.dtype, x.shape[0], *s["w"].shape))
    hot.hot_linear_forward(x, s["w"], s["y"], ws, bias=s["bias"], residual=s["residual"], fn=fn, ckpt=buf)
    r = {"y": s["y"]}
    if case["kept"]:
        r["g_z"] = hot.hot_activation_backward(fn, s["g_y"], s["g_z"], ckpt=buf)
    return r


def run(state):
    if own:
        return _kernels(state)
    return _plain(state)


# ---- 64 bits --------------------------------------------------------------------------------------------------------

def _held64(x):
    """The 8-bit form by its definition: steps of 2^k with the smallest k >= -125 that keeps round(largest / 2^k) <= 127."""
    rows, cols = x.shape
    whole = torch.zeros(rows, -(-cols // GROUP) * GROUP, dtype=torch.float64, device=x.device)
    whole[:, :cols] = x
    parts = whole.reshape(-1, GROUP)
    mantissa, k = torch.frexp(parts.abs().max(dim=1).values)
    k = (k - 7 + ((mantissa * 128).round() > 127)).clamp(min=-125)
    step = ((k.long() + 1023) << 52).view(torch.float64)[:, None]     # 2^k, exactly: pow() is off by an ulp for some k
    return (torch.round(parts / step) * step).reshape(rows, -1)[:, :cols]


def _slope64(fn, x):
    x = x.detach().requires_grad_(True)
    return torch.autograd.grad(_value64(fn, x).sum(), x)[0]


def _value64(fn, x):
    if fn == "gelu":
        return torch.special.ndtr(x) * x
    if fn == "gelu_tanh":
        return x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
    return {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v)}[fn](x)


def exact(case, seed):
    s = prepare(case, seed)
    kind, x = case["kind"], s["x"].double()
    if kind == "checkpoint":
        return _held64(x)
    if kind == "activation":
        g = s["g_y"].double() * _slope64(case["fn"], _held64(x))
        return {"y": _value64(case["fn"], x), "g_x": g, "g_bias": g.sum(0) if case["bias"] else None}
    if kind == "norm":
        h, r = x, {}
        if case["residual"]:
            r["h"] = x + s["residual"].double()
            h = r["h"].to(s["x"].dtype).double()      # the sum is kept, and normalised, in its type
        var, mean = torch.var_mean(h, dim=1, unbiased=False, keepdim=True)
        std = torch.sqrt(var + EPS)
        gamma, g = s["gamma"].double(), s["g_y"].double()
        r.update(y=torch.addcmul(s["beta"].double(), (h - mean) / std, gamma), mean=mean[:, 0], rstd=1 / std[:, 0])
        n = ((_held64(h) if case["kept"] else h) - mean) / std
        r["g_gamma"], r["g_beta"] = torch.sum(g * n, 0), torch.sum(g, 0)
        g.mul_(gamma)
        inner = torch.sum(g * n, 1, keepdim=True) / case["cols"]
        r["g_x"] = (g - torch.sum(g, 1, keepdim=True) / case["cols"] - n * inner) / std
        if case["residual"]:
            r["g_x"] += s["g_residual"].double()
        return r
    z = torch.matmul(x, s["w"].double().t().contiguous())
    if s["bias"] is not None:
        z += s["bias"].double()
    r = {"y": _value64(case["fn"], z)}
    if s["residual"] is not None:
        r["y"] = r["y"] + s["residual"].double()
    if case["kept"]:
        r["g_z"] = s["g_y"].double() * _slope64(case["fn"], _held64(z))
    return r
