"""Timed cases of what lies between the sparse layers of a transformer block: the residual junction (norm after a block,
dropout, gate and residual scale, norm before the next block) with its gradient, and dropout from a counter-based generator
whose mask is never stored, alone and inside the backward pass of a hidden layer that is kept as an 8-bit checkpoint.

    join      u = norm_post(y);  x' = alpha x + scale * gate * drop(u);  n = norm_pre(x')      bimask_residual_norm_fwd
    joingrad  from dx' and dn: dx, dy, dgate and the gradients of the scale, weights and biases  bimask_residual_norm_bwd
    drop      Y = drop(X)                                                                     bimask_dropout
    hidden    H = drop(act(Z)) and dZ = drop(dH) act'(Z), db = sum_t dZ, Z a checkpoint       bimask_ckpt_unpack_dropout,
                                                                                              bimask_act_dropout_bwd

A norm is "none", "rms" (v rstd w + b with rstd = 1 / sqrt(mean(v^2) + eps)) or "layer" (the same on v - mean(v)).  A
gate has one row for every `span` tokens.  The stream x is bf16 or fp32; branches, gates and normalised values are bf16,
weights, scales and statistics fp32.

Dropout: element e of a T x C matrix belongs to block e / 8, whose counter (block lo, block hi, stream lo, stream hi) goes
through Philox4x32-10 under the 64-bit seed; element 8 b + k takes the low (k even) or high half of word k / 2 and is kept iff
this is at least thr = rint(65536 p), then multiplied by 65536 / (65536 - thr).

`own` chooses between the library's calls and the plain form (elementary torch operations in 32 bits, one rounding at the
end).  Sizes are those of the benchmark configurations (DeiT-small blocks at 197 tokens x 64, the 4096-wide MLP pair at 8192
tokens), single tokens and ragged batches on the same widths.
"""
import math

import torch

own = False

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")          # the library's activation codes, in order
NORMS = ("none", "rms", "layer")                              # and its norms
MAX_STREAM = 8192 * 4096
MAX_HIDDEN = 8192 * 16384


def _join(name, op, T, C, post, pre, stream="bf16", gate=0, scale=False, bias=False, p=0.0, alpha=1.0):
    return {"name": name, "op": op, "T": T, "C": C, "post": post, "pre": pre, "stream": stream, "gate": gate, "scale": scale,
            "bias": bias, "p": p, "alpha": alpha}


def listed():
    return [
        # one token of generation: norms on both sides of a block, no dropout
        _join("join-token", "join", 1, 4096, "rms", "rms"),
        # a small batch of generation; depth-scaled residual, the sum normalised
        _join("join-batch24", "join", 24, 4096, "none", "layer", bias=True, alpha=1.7),
        # DeiT-small in training: pre-norm blocks with a scale per channel and dropout on the branch, stream in fp32
        _join("join-vit", "join", 12608, 384, "none", "layer", stream="f32", scale=True, bias=True, p=0.1),
        # the wide block in training, norms on both sides, dropout
        _join("join-mlp", "join", 8192, 4096, "rms", "rms", p=0.1),
        # odd number of tokens, a gate for every value
        _join("joingrad-ragged", "joingrad", 1001, 1152, "rms", "rms", gate=1, scale=True),
        # DeiT-small with one gate row per image (197 tokens)
        _join("joingrad-vit-gated", "joingrad", 12608, 384, "none", "layer", gate=197, bias=True, p=0.1),
        _join("joingrad-vit", "joingrad", 12608, 384, "none", "layer", stream="f32", scale=True, bias=True, p=0.1),
        _join("joingrad-mlp", "joingrad", 8192, 4096, "rms", "rms", p=0.1),
        # hidden activations of a DeiT-small block, and of the wide MLP
        {"name": "drop-vit-hidden", "op": "drop", "T": 12608, "C": 1536, "p": 0.1, "stream": "bf16"},
        {"name": "drop-mlp-hidden", "op": "drop", "T": 8192, "C": 16384, "p": 0.25, "stream": "bf16"},
        # the same layers' backward passes: the kept pre-activation is all that there is of the hidden values
        {"name": "hidden-vit", "op": "hidden", "T": 12608, "C": 1536, "act": "gelu", "p": 0.1},
        {"name": "hidden-mlp", "op": "hidden", "T": 8192, "C": 16384, "act": "gelu_tanh", "p": 0.25},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("join", "join", "joingrad", "joingrad", "drop", "hidden"))
    p = rng.choice((0.0, 0.05, 0.1, 0.3, 0.5))
    while True:
        T = _log(rng, 1, 16384)
        C = 32 * max(1, round(_log(rng, 32, 16384 if op in ("drop", "hidden") else 8192) / 32))
        if op == "drop":
            if T * C <= MAX_HIDDEN:
                return {"op": op, "T": T, "C": C, "p": p, "stream": rng.choice(("bf16", "bf16", "f32"))}
        elif op == "hidden":
            if T * C <= MAX_HIDDEN:
                return {"op": op, "T": T, "C": C, "act": rng.choice(ACTS), "p": p}
        elif T * C <= MAX_STREAM:
            post = rng.choice(NORMS)
            pre = rng.choice(NORMS[1:])
            c = _join("", op, T, C, post, pre, stream=rng.choice(("bf16", "bf16", "f32")),
                      gate=rng.choice((0, 0, 1, min(T, _log(rng, 2, 2048)))), scale=rng.random() < 0.5, bias=rng.random() < 0.5, p=p,
                      alpha=rng.choice((1.0, 1.0, 0.81)))
            del c["name"]
            return c


# ---- inputs -------------------------------------------------------------------------------------

def _activations(T, C, gen, scale=1.0, dtype=torch.bfloat16):
    """N(0, 1) per channel, one channel in 64 eight times as large."""
    x = torch.randn(T, C, generator=gen, device="cuda", dtype=torch.float32) * scale
    x[:, ::64] *= 8.0
    return x.to(dtype)


def _quantise(x):
    """Checkpoint of x: signed bytes and one scale byte for 32 channels."""
    b = x.view(x.shape[0], -1, 32)
    m, e = torch.frexp(b.abs().amax(-1))
    e = e - 7 + (m > 127.0 / 128.0)
    e = torch.where(m == 0, torch.full_like(e, -126), e).clamp(min=-126)
    q = torch.round(b * torch.exp2(-e.to(x.dtype)).unsqueeze(-1))
    return q.to(torch.int8).view(x.shape), (e + 127).to(torch.uint8)


def _values(q, s, dtype=torch.float32):
    return (q.to(dtype).view(q.shape[0], -1, 32) * torch.exp2(s.to(dtype) - 127.0).unsqueeze(-1)).view(q.shape)


def _statistics(v, kind, eps=1e-5):
    """(mean, 1 / standard deviation) of every row, as the forward pass leaves them."""
    mean = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    c = v - mean
    return torch.cat((mean, 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)), 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * (seed % (1 << 40)) + 29)
    op, T, C = case["op"], case["T"], case["C"]
    st = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), "number": 7 + seed % 1000}

    def empty(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if op == "drop":
        dtype = torch.float32 if case["stream"] == "f32" else torch.bfloat16
        st["X"], st["Y"] = _activations(T, C, gen, dtype=dtype), empty(T, C, dtype=dtype)
        return st
    if op == "hidden":
        st["dY"] = _activations(T, C, gen, 0.01)
        st["Zq"], st["Zs"] = _quantise(_activations(T, C, gen, 1.5).float())
        st["dZ"], st["H"], st["db"] = empty(T, C), empty(T, C), empty(C, dtype=torch.float32)
        st["ws"] = empty(4 * C * min(T, 1024) + 1024, dtype=torch.uint8)          # partial column sums
        return st
    dtype = torch.float32 if case["stream"] == "f32" else torch.bfloat16
    st["y"] = _activations(T, C, gen, 0.5)
    if case["gate"]:
        st["gate"] = (0.5 * torch.randn((T + case["gate"] - 1) // case["gate"], C, generator=gen, device="cuda") + 0.5).to(torch.bfloat16)
    if case["scale"]:
        st["scale"] = 0.1 + 0.9 * torch.rand(C, generator=gen, device="cuda")
    for side in ("post", "pre"):
        if case[side] != "none":
            st["w_" + side] = 1.0 + 0.2 * torch.randn(C, generator=gen, device="cuda")
            if case["bias"]:
                st["b_" + side] = 0.2 * torch.randn(C, generator=gen, device="cuda")
    f32 = torch.float32
    if op == "join":
        st["x"] = _activations(T, C, gen, 2.0, dtype)
        st["xo"], st["n"] = empty(T, C, dtype=dtype), empty(T, C)
        for side in ("post", "pre"):
            if case[side] != "none":
                st["stats_" + side] = empty(T, 2, dtype=f32)
        return st
    st["xo"] = _activations(T, C, gen, 2.0, dtype)
    st["dxo"], st["dn"] = _activations(T, C, gen, 0.01, dtype), _activations(T, C, gen, 0.01)
    st["dx"], st["dy"] = empty(T, C, dtype=dtype), empty(T, C)
    if case["post"] != "none":
        st["stats_post"] = _statistics(st["y"].float(), case["post"])
    st["stats_pre"] = _statistics(st["xo"].float(), case["pre"])
    if case["gate"]:
        st["dgate"] = empty(*st["gate"].shape)
    if case["scale"]:
        st["dscale"] = empty(C, dtype=f32)
    for k in ("w_post", "b_post", "w_pre", "b_pre"):
        if k in st:
            st["d" + k] = empty(C, dtype=f32)
    # partial column sums: four rows for each of the card's CTAs, and for gates one for every few tokens
    st["ws"] = empty(4 * C * (4 * 1024 + (min(T, 8192) + 2 * st["gate"].shape[0] if case["gate"] > 1 else 0)) + 1024, dtype=torch.uint8)
    return st


# ---- the operators ------------------------------------------------------------------------------

def _philox(block, number, seed):
    """The four 32-bit words of Philox4x32-10 for every block, as int64 tensors."""
    low = 0xFFFFFFFF
    c0, c1 = block & low, block >> 32
    c2, c3 = torch.full_like(block, number & low), torch.full_like(block, number >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57              # modulo 2^64, as their low and high halves need
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _multiplier(T, C, p, seed, number):
    """T x C fp32: 0 where dropped, 65536 / (65536 - thr) where kept; 1 without dropout."""
    thr = round(65536 * p)
    if thr == 0:
        return 1.0
    words = _philox(torch.arange(T * C // 8, device="cuda"), number, seed)
    keep = torch.stack([h for w in words for h in ((w & 0xFFFF) >= thr, (w >> 16) >= thr)], -1).view(T, C)
    return keep.float() * (65536.0 / (65536 - thr))


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _affine(v, w, b):
    v = v if w is None else v * w
    return v if b is None else v + b


def _rows(gate, span, T):
    """The gate's row of every token."""
    return gate.float()[torch.arange(T, device=gate.device) // span]


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(st):
    case = st["case"]
    op, T, C = case["op"], case["T"], case["C"]
    m = _multiplier(T, C, case["p"], st["seed"], st["number"])
    if op == "drop":
        return {"Y": (st["X"].float() * m).to(st["X"].dtype)}
    if op == "hidden":
        z = _values(st["Zq"], st["Zs"])
        dz = st["dY"].float() * m * _act_grad(z, case["act"])
        return {"H": (_act(z, case["act"]) * m).to(torch.bfloat16), "dZ": dz.to(torch.bfloat16), "db": dz.sum(0)}
    out = {}
    gate = _rows(st["gate"], case["gate"], T) if case["gate"] else 1.0
    scale = st.get("scale", 1.0)
    y = st["y"].float()
    if op == "join":
        if case["post"] != "none":
            out["stats_post"] = _statistics(y, case["post"])
            y = _affine((y - out["stats_post"][:, :1]) * out["stats_post"][:, 1:], st["w_post"], st.get("b_post"))
        xo = case["alpha"] * st["x"].float() + y * m * gate * scale
        out["stats_pre"] = _statistics(xo, case["pre"])
        n = _affine((xo - out["stats_pre"][:, :1]) * out["stats_pre"][:, 1:], st["w_pre"], st.get("b_pre"))
        out["xo"], out["n"] = xo.to(st["x"].dtype), n.to(torch.bfloat16)
        return out

    def through_norm(g, hat, rstd, kind):
        """Gradient by the normalised value -> by the value."""
        d = g - hat * (g * hat).mean(-1, keepdim=True)
        return rstd * (d - g.mean(-1, keepdim=True) if kind == "layer" else d)

    dn = st["dn"].float()
    hat = (st["xo"].float() - st["stats_pre"][:, :1]) * st["stats_pre"][:, 1:]
    D = st["dxo"].float() + through_norm(dn * st["w_pre"], hat, st["stats_pre"][:, 1:], case["pre"])
    out["dx"] = (case["alpha"] * D).to(st["dxo"].dtype)
    out["dw_pre"] = (dn * hat).sum(0)
    if case["bias"]:
        out["db_pre"] = dn.sum(0)
    hat, u = y, y
    if case["post"] != "none":
        hat = (y - st["stats_post"][:, :1]) * st["stats_post"][:, 1:]
        u = _affine(hat, st["w_post"], st.get("b_post"))
    du = D * gate * scale * m
    if case["gate"]:
        dg = D * scale * (u * m)
        if case["gate"] > 1:
            dg = torch.cat((dg, dg.new_zeros(st["gate"].shape[0] * case["gate"] - T, C))).view(-1, case["gate"], C).sum(1)
        out["dgate"] = dg.to(torch.bfloat16)
    if case["scale"]:
        out["dscale"] = (D * gate * (u * m)).sum(0)
    if case["post"] != "none":
        out["dw_post"] = (du * hat).sum(0)
        if case["bias"]:
            out["db_post"] = du.sum(0)
        du = through_norm(du * st["w_post"], hat, st["stats_post"][:, 1:], case["post"])
    out["dy"] = du.to(torch.bfloat16)
    return out


def _run_own(st):
    import paper_2302_06058_b200 as bm
    case = st["case"]
    op, T, C = case["op"], case["T"], case["C"]
    drop = bm.make_dropout(case["p"], st["seed"], st["number"])
    if op == "drop":
        bm.bimask_dropout(st["X"], bm.TYPE_F32 if case["stream"] == "f32" else bm.TYPE_BF16, T, C, drop, st["Y"])
        return {"Y": st["Y"]}
    if op == "hidden":
        act = ACTS.index(case["act"])
        bm.bimask_ckpt_unpack_dropout(st["Zq"], st["Zs"], act, drop, T, C, st["H"])
        bm.bimask_act_dropout_bwd(st["dY"], st["Zq"], st["Zs"], act, drop, T, C, st["dZ"], st["db"], st["ws"], st["ws"].numel())
        return {"H": st["H"], "dZ": st["dZ"], "db": st["db"]}
    args = bm.make_residual_args(T, C, st, stream_type=bm.TYPE_F32 if case["stream"] == "f32" else bm.TYPE_BF16,
                                 post=NORMS.index(case["post"]), pre=NORMS.index(case["pre"]), eps_post=1e-5, eps_pre=1e-5,
                                 alpha=case["alpha"], gate_span=case["gate"], drop=drop)
    if op == "join":
        bm.bimask_residual_norm_fwd(args)
        names = ("xo", "n", "stats_post", "stats_pre")
    else:
        bm.bimask_residual_norm_bwd(args)
        names = ("dx", "dy", "dgate", "dscale", "dw_post", "db_post", "dw_pre", "db_pre")
    return {k: st[k] for k in names if k in st}


def work(case):
    op, T, C = case["op"], case["T"], case["C"]
    n = T * C
    if op == "drop":
        return {"bytes": (8 if case["stream"] == "f32" else 4) * n, "flops": 2 * n}
    if op == "hidden":                                          # bytes and scales, dH; H and dZ, db
        return {"bytes": n + n // 32 + 2 * n + 4 * n + 4 * C, "flops": 40 * n}
    s = 4 if case["stream"] == "f32" else 2
    params = sum((case[k] != "none") * (2 if case["bias"] else 1) for k in ("post", "pre")) + case["scale"]
    stats = 8 * T * ((case["post"] != "none") + 1)
    gate = 2 * C * ((T + case["gate"] - 1) // case["gate"]) if case["gate"] else 0
    if op == "join":
        return {"bytes": n * (2 * s + 4) + stats + 4 * C * params + gate, "flops": 20 * n}
    return {"bytes": n * (3 * s + 6) + stats + 8 * C * params + 2 * gate, "flops": 40 * n}


# ---- definitions in 64 bits ---------------------------------------------------------------------

def _kept64(T, C, p, seed, number):
    """T x C fp64 multipliers of the dropout, the generator written with 16-bit limbs."""
    thr = int(math.floor(65536 * p + 0.5))
    if thr == 0:
        return torch.ones((), dtype=torch.float64, device="cuda")

    def product(a, k):                                          # 32 x 32 bits -> (high, low)
        a0, a1, k0, k1 = a & 65535, a >> 16, k & 65535, k >> 16
        mid = a1 * k0 + ((a0 * k0) >> 16)
        mid2 = a0 * k1 + (mid & 65535)
        return a1 * k1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 65535) << 16) | ((a0 * k0) & 65535)

    b = torch.arange((T * C + 7) // 8, device="cuda", dtype=torch.int64)
    x = [b % (1 << 32), torch.div(b, 1 << 32, rounding_mode="floor"), torch.tensor(number % (1 << 32), device="cuda"),
         torch.tensor(number // (1 << 32), device="cuda")]
    for r in range(10):
        key = ((seed + r * 0x9E3779B9) % (1 << 32), (seed // (1 << 32) + r * 0xBB67AE85) % (1 << 32))
        h0, l0 = product(x[0], 0xD2511F53)
        h1, l1 = product(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0]
    bits = torch.empty(b.numel(), 4, 2, dtype=torch.int64, device="cuda")
    for i in range(4):
        bits[:, i, 0], bits[:, i, 1] = x[i] % 65536, torch.div(x[i], 65536, rounding_mode="floor")
    return torch.where(bits.view(T, C) < thr, 0.0, 65536.0 / (65536.0 - thr)).double()


def _act64(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _slope64(z, act):
    if act == "none":
        return torch.ones_like(z)
    with torch.enable_grad():
        v = z.clone().requires_grad_()
        return torch.autograd.grad(_act64(v, act).sum(), v)[0]


def _standard64(v, kind, eps):
    """(mean, 1 / deviation) of the rows."""
    mean = v.sum(1, keepdim=True) / v.shape[1] if kind == "layer" else 0.0 * v[:, :1]
    return mean, (((v - mean) ** 2).sum(1, keepdim=True) / v.shape[1] + eps) ** -0.5


def exact(case, seed):
    st = prepare(case, seed)
    op, T, C = case["op"], case["T"], case["C"]
    keep = _kept64(T, C, case["p"], st["seed"], st["number"])
    if op == "drop":
        return {"Y": st["X"].double() * keep}
    if op == "hidden":
        z = st["Zq"].double() * torch.ldexp(torch.ones_like(st["Zs"], dtype=torch.float64), st["Zs"].int() - 127).repeat_interleave(32, 1)
        dz = st["dY"].double() * keep * _slope64(z, case["act"])
        return {"H": _act64(z, case["act"]) * keep, "dZ": dz, "db": torch.einsum("tc->c", dz)}

    def param(name, default):
        return st[name].double() if name in st else torch.full((C,), default, dtype=torch.float64, device="cuda")

    y, factor = st["y"].double(), param("scale", 1.0) * keep
    w, b, wp, bp = param("w_post", 1.0), param("b_post", 0.0), param("w_pre", 1.0), param("b_pre", 0.0)
    gates = st["gate"].double().repeat_interleave(case["gate"], 0)[:T] if case["gate"] else 1.0
    post = case["post"] != "none"
    out = {}
    if op == "join":
        u = y
        if post:
            mean, rstd = _standard64(y, case["post"], 1e-5)
            out["stats_post"] = torch.cat((mean, rstd), 1)
            u = torch.addcmul(b, (y - mean) * rstd, w)
        xo = st["x"].double() * case["alpha"] + factor * gates * u
        mean, rstd = _standard64(xo, case["pre"], 1e-5)
        out["stats_pre"] = torch.cat((mean, rstd), 1)
        out["xo"], out["n"] = xo, torch.addcmul(bp, (xo - mean) * rstd, wp)
        return out

    # The gradients from the Jacobian of a norm, r (I - 1 1^T / C [layer] - h h^T / C), with the statistics as given.
    def pull(v, h, r, kind):
        centred = v - (v.sum(1, keepdim=True) / C if kind == "layer" else 0.0)
        return r * (centred - h * torch.einsum("tc,tc->t", v, h).unsqueeze(1) / C)

    s_pre, dn = st["stats_pre"].double(), st["dn"].double()
    h = s_pre[:, 1:] * (st["xo"].double() - s_pre[:, :1])
    total = st["dxo"].double() + pull(dn * wp, h, s_pre[:, 1:], case["pre"])
    out["dx"], out["dw_pre"] = case["alpha"] * total, torch.einsum("tc,tc->c", dn, h)
    if case["bias"]:
        out["db_pre"] = torch.einsum("tc->c", dn)
    h, u = y, y
    if post:
        s_post = st["stats_post"].double()
        h = s_post[:, 1:] * (y - s_post[:, :1])
        u = torch.addcmul(b, h, w)
    if case["gate"]:
        each = total * factor * u
        rows = st["gate"].shape[0]
        out["dgate"] = torch.zeros(rows, C, dtype=torch.float64, device="cuda").index_add_(
            0, torch.arange(T, device="cuda") // case["gate"], each)
    if case["scale"]:
        out["dscale"] = torch.einsum("tc,tc->c", total * gates, keep * u)
    du = total * factor * gates
    if post:
        out["dw_post"] = torch.einsum("tc,tc->c", du, h)
        if case["bias"]:
            out["db_post"] = torch.einsum("tc->c", du)
        du = pull(du * w, h, s_post[:, 1:], case["post"])
    out["dy"] = du
    return out
