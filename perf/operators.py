"""Timed cases of the linear-layer operators around the 2:4 products: the forward product with bias, activation,
residual and 8-bit checkpoint in its epilogue, the gradient of that epilogue, the 8-bit activation checkpoint itself,
and the weight gradient that reads one.

    linear   Y = act(X (B.W)^T + b) + R, optionally with the pre-activation kept as a checkpoint   bimask_linear_fwd
    actgrad  dZ = dY act'(Z), db = sum_t dZ, Z a checkpoint                                        bimask_act_bwd
    ckpt     activations written to a checkpoint and read back, optionally through act             bimask_ckpt_pack / _unpack
    wgrad    dW = dY^T X, X a checkpoint                                                           bimask_wgrad_ckpt

A checkpoint holds, for 32 consecutive channels of a token, 32 signed bytes q and one byte s: the values q 2^(s - 127),
where 2^(s - 127) is the smallest power of two (not below 2^-126) with max |x| <= 127 * 2^(s - 127).

`own` chooses between the library's calls and the plain form (elementary torch operations in 32 bits, one rounding
at the end).  Sizes are those of the benchmark configurations (DeiT-small block linears at 197 tokens x 64, the
16384 x 4096 MLP pair at 8192 tokens), single tokens and small batches on the same layers, and ragged ones.
"""
import math

import torch

own = False

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")          # the library's activation codes, in order
MAX_WORK = 8192 * 16384 * 4096


def listed():
    return [
        # one token through the wide layer of the MLP pair: generation, the weights are read once for one row
        {"name": "linear-token-fc1", "op": "linear", "T": 1, "I": 16384, "J": 4096, "N": 2, "M": 4, "act": "gelu_tanh",
         "bias": True, "res": False, "ckpt": False},
        # a small batch of tokens through its narrow layer, whose long reduction has few output rows; residual added
        {"name": "linear-batch24-fc2", "op": "linear", "T": 24, "I": 4096, "J": 16384, "N": 2, "M": 4, "act": "none",
         "bias": True, "res": True, "ckpt": False},
        # first linear of a DeiT-small block in training: GELU, pre-activation kept in 8 bits for the backward pass
        {"name": "linear-vit-fc1", "op": "linear", "T": 12608, "I": 1536, "J": 384, "N": 2, "M": 4, "act": "gelu",
         "bias": True, "res": False, "ckpt": True},
        # a pattern without a 2:4 form (dense masked operand), ReLU, residual, odd number of tokens
        {"name": "linear-4of8-ragged", "op": "linear", "T": 1001, "I": 1152, "J": 384, "N": 4, "M": 8, "act": "relu",
         "bias": True, "res": True, "ckpt": False},
        # the MLP pair in training: fc1 with tanh-GELU and checkpoint ...
        {"name": "linear-mlp-fc1", "op": "linear", "T": 8192, "I": 16384, "J": 4096, "N": 2, "M": 4, "act": "gelu_tanh",
         "bias": True, "res": False, "ckpt": True},
        # ... and fc2 with the residual stream added
        {"name": "linear-mlp-fc2", "op": "linear", "T": 8192, "I": 4096, "J": 16384, "N": 2, "M": 4, "act": "none",
         "bias": True, "res": True, "ckpt": False},
        # gradient through the activation and the bias of the two first linears
        {"name": "actgrad-vit-fc1", "op": "actgrad", "T": 12608, "C": 1536, "act": "gelu"},
        {"name": "actgrad-mlp-fc1", "op": "actgrad", "T": 8192, "C": 16384, "act": "gelu_tanh"},
        # a layer's input saved in the forward pass and restored in the backward pass
        {"name": "ckpt-vit-input", "op": "ckpt", "T": 12608, "C": 384, "act": "none"},
        # a pre-activation saved, the activated values recomputed from it (input of fc2 for its weight gradient)
        {"name": "ckpt-mlp-hidden", "op": "ckpt", "T": 8192, "C": 16384, "act": "gelu_tanh"},
        # weight gradients whose saved input is a checkpoint: few output tiles and many tokens; many of both
        {"name": "wgrad-vit-fc2", "op": "wgrad", "T": 12608, "I": 384, "J": 1536},
        {"name": "wgrad-mlp-fc1", "op": "wgrad", "T": 8192, "I": 16384, "J": 4096},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _log32(rng, lo, hi):
    while True:
        n = 32 * max(1, round(_log(rng, lo, hi) / 32))
        if n != 3072:
            return n


def draw(rng):
    op = rng.choice(("linear", "linear", "actgrad", "ckpt", "wgrad"))
    act = rng.choice(ACTS)
    while True:
        T = _log(rng, 1, 16384)
        if T == 3072:
            continue
        if op in ("actgrad", "ckpt"):
            C = _log32(rng, 32, 16384)
            if T * C <= 8192 * 16384:
                return {"op": op, "T": T, "C": C, "act": act}
            continue
        I, J = _log32(rng, 64, 16384), _log32(rng, 64, 16384)
        if I * J > 16384 * 4096 or T * I * J > MAX_WORK:
            continue
        if op == "wgrad":
            return {"op": op, "T": T, "I": I, "J": J}
        N, M = rng.choice(((2, 4), (2, 4), (1, 4), (4, 8)))
        return {"op": op, "T": T, "I": I, "J": J, "N": N, "M": M, "act": act, "bias": rng.random() < 0.8,
                "res": rng.random() < 0.5, "ckpt": rng.random() < 0.5}


# ---- inputs -------------------------------------------------------------------------------------

def _activations(T, C, gen, scale=1.0):
    """N(0, 1) per channel as after a normalisation, one channel in 64 eight times as large."""
    x = torch.randn(T, C, generator=gen, device="cuda", dtype=torch.float32) * scale
    x[:, ::64] *= 8.0
    return x.to(torch.bfloat16)


def _keep_largest(W, N, M):
    """Boolean I x J mask: in every aligned block of M the N largest |W| of a row, the lower index first on a tie."""
    a = W.abs().view(W.shape[0], -1, M)
    keep = torch.empty_like(a, dtype=torch.bool)
    for m in range(M):
        beaten = torch.zeros_like(a[..., 0], dtype=torch.int32)
        for n in range(M):
            if n != m:
                beaten += (a[..., n] >= a[..., m]) if n < m else (a[..., n] > a[..., m])
        keep[..., m] = beaten < N
    return keep.view_as(W)


def _pack24(W, keep):
    """The 2:4 operand of W where keep: values I x J/2 bf16, index codes I x J/32 int32, and the order of the codes that
    the tensor cores take."""
    I, J = W.shape
    k = keep.view(I, J // 4, 4)
    w = W.view(I, J // 4, 4)
    pos = torch.arange(4, device=W.device)
    first = torch.where(k, pos, 4).amin(-1)                     # N = 1: one position, padded with the lowest free one
    last = torch.where(k, pos, -1).amax(-1)
    spare = torch.where(first == 0, 1, 0)
    i0 = torch.where(first == last, torch.minimum(first, spare), first)
    i1 = torch.where(first == last, torch.maximum(first, spare), last)
    idx = torch.stack((i0, i1), -1)
    vals = torch.where(k.gather(2, idx), w.gather(2, idx), 0.0).to(torch.bfloat16).view(I, J // 2)
    code = (i0 | (i1 << 2)).view(I, J // 32, 8) << (4 * torch.arange(8, device=W.device))
    words = code.sum(-1)                                        # unsigned 32-bit codes held in int64
    tm, tk = (I + 127) // 128, (J // 32 + 3) // 4
    full = torch.full((tm * 128, tk * 4), 0x44444444, dtype=torch.int64, device=W.device)
    full[:I, :J // 32] = words
    halves = torch.stack((full & 0xFFFF, full >> 16), -1).view(tm, 8, 2, 8, tk, 4, 2)    # block, m2, +8, m0, k tile, word, half
    image = halves[:, :, 0] | (halves[:, :, 1] << 16)                                    # block, m2, m0, k tile, word, half
    image = image.permute(0, 3, 1, 5, 2, 4).contiguous().view(-1)                        # block, k tile, m2, half, m0, word

    def as_i32(x):
        return torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32)

    return vals, as_i32(words), as_i32(image)


def _quantise(x):
    """Checkpoint of x (fp32 or fp64): signed bytes and scale bytes."""
    b = x.view(x.shape[0], -1, 32)
    m, e = torch.frexp(b.abs().amax(-1))                        # amax = m 2^e, 1/2 <= m < 1
    e = e - 7 + (m > 127.0 / 128.0)                             # 2^e >= amax / 127
    e = torch.where(m == 0, torch.full_like(e, -126), e).clamp(min=-126)
    q = torch.round(torch.ldexp(b, -e.unsqueeze(-1))) if x.dtype == torch.float64 else torch.round(b * torch.exp2(-e.to(x.dtype)).unsqueeze(-1))
    return q.to(torch.int8).view(x.shape), (e + 127).to(torch.uint8)


def _values(q, s, dtype=torch.float32):
    scale = torch.exp2(s.to(dtype) - 127.0)
    return (q.to(dtype).view(q.shape[0], -1, 32) * scale.unsqueeze(-1)).view(q.shape)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * (seed % (1 << 40)) + 17)
    T, op = case["T"], case["op"]
    st = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}

    def empty(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if op == "linear":
        I, J = case["I"], case["J"]
        W = torch.randn(I, J, generator=gen, device="cuda") * math.sqrt(2.0 / J)
        keep = _keep_largest(W, case["N"], case["M"])
        if case["N"] <= 2:
            st["vals"], st["meta"], st["hw_meta"] = _pack24(W, keep)
        else:
            st["vals"], st["meta"], st["hw_meta"] = torch.where(keep, W, 0.0).to(torch.bfloat16), None, None
        del W, keep
        st["X"] = _activations(T, J, gen)
        st["bias"] = 0.2 * torch.randn(I, generator=gen, device="cuda") if case["bias"] else None
        st["R"] = _activations(T, I, gen) if case["res"] else None
        st["Y"] = empty(T, I)
        if case["ckpt"]:
            st["Zq"], st["Zs"], st["Z"] = empty(T, I, dtype=torch.int8), empty(T, I // 32, dtype=torch.uint8), empty(T, I)
    elif op == "wgrad":
        I, J = case["I"], case["J"]
        st["dY"] = _activations(T, I, gen, 0.01)
        st["Xq"], st["Xs"] = _quantise(_activations(T, J, gen).float())
        st["dW"] = empty(I, J, dtype=torch.float32)
        # scratch of one wide product: decoded tokens and partial sums, rounded up
        st["ws"] = empty(2 * T * J + 16 * I * J * (1 if I * J > 1 << 22 else 16) + (1 << 20), dtype=torch.uint8)
    else:
        C = case["C"]
        x = _activations(T, C, gen, 1.5)
        if op == "actgrad":
            st["dY"] = _activations(T, C, gen, 0.01)
            st["Zq"], st["Zs"] = _quantise(x.float())
            st["dZ"], st["db"] = empty(T, C), empty(C, dtype=torch.float32)
            st["ws"] = empty(4 * C * min(T, 1024) + 1024, dtype=torch.uint8)      # partial column sums
        else:
            st["X"] = x
            st["q"], st["s"], st["out"] = empty(T, C, dtype=torch.int8), empty(T, C // 32, dtype=torch.uint8), empty(T, C)
    return st


# ---- the operators ------------------------------------------------------------------------------

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


def _dense(vals, meta):
    """fp32 I x J matrix that a 2:4 operand stands for."""
    if meta is None:
        return vals.float()
    I = vals.shape[0]
    nib = (meta.unsqueeze(-1) >> (4 * torch.arange(8, device=meta.device, dtype=torch.int32))) & 0xF      # I, words, 8
    idx = torch.stack((nib & 3, nib >> 2), -1).view(I, -1, 2).long()
    return torch.zeros(I, idx.shape[1], 4, device=vals.device).scatter_(2, idx, vals.float().view(I, -1, 2)).view(I, -1)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(st):
    case = st["case"]
    op = case["op"]
    if op == "linear":
        z = st["X"].float() @ _dense(st["vals"], st["meta"]).t()
        if st["bias"] is not None:
            z = z + st["bias"]
        y = _act(z, case["act"])
        if st["R"] is not None:
            y = y + st["R"].float()
        out = {"Y": y.to(torch.bfloat16)}
        if case["ckpt"]:
            out["Z"] = _values(*_quantise(z)).to(torch.bfloat16)
        return out
    if op == "actgrad":
        dz = st["dY"].float() * _act_grad(_values(st["Zq"], st["Zs"]), case["act"])
        return {"dZ": dz.to(torch.bfloat16), "db": dz.sum(0)}
    if op == "ckpt":
        q, s = _quantise(st["X"].float())
        return {"X": _act(_values(q, s), case["act"]).to(torch.bfloat16)}
    return {"dW": st["dY"].float().t() @ _values(st["Xq"], st["Xs"])}


def _run_own(st):
    import paper_2302_06058_b200 as bm
    case = st["case"]
    op, T = case["op"], case["T"]
    if op == "linear":
        I, J = case["I"], case["J"]
        bm.bimask_linear_fwd(st["X"], st["vals"], st["hw_meta"], st["bias"], ACTS.index(case["act"]), st["R"], T, I, J, st["Y"],
                             st.get("Zq"), st.get("Zs"), st["status"])
        if not case["ckpt"]:
            return {"Y": st["Y"]}
        bm.bimask_ckpt_unpack(st["Zq"], st["Zs"], 0, T, I, st["Z"])        # the checkpoint as the values it stands for
        return {"Y": st["Y"], "Z": st["Z"]}
    if op == "actgrad":
        bm.bimask_act_bwd(st["dY"], st["Zq"], st["Zs"], ACTS.index(case["act"]), T, case["C"], st["dZ"], st["db"], st["ws"],
                          st["ws"].numel())
        return {"dZ": st["dZ"], "db": st["db"]}
    if op == "ckpt":
        bm.bimask_ckpt_pack(st["X"], T, case["C"], st["q"], st["s"])
        bm.bimask_ckpt_unpack(st["q"], st["s"], ACTS.index(case["act"]), T, case["C"], st["out"])
        return {"X": st["out"]}
    bm.bimask_wgrad_ckpt(st["dY"], st["Xq"], st["Xs"], T, case["I"], case["J"], st["dW"], st["ws"], st["ws"].numel(), st["status"])
    return {"dW": st["dW"]}


def work(case):
    op, T = case["op"], case["T"]
    if op in ("linear", "wgrad"):
        I, J = case["I"], case["J"]
    if op == "linear":
        packed = case["N"] <= 2
        b = 2 * T * J + (I * J + I * J // 8 if packed else 2 * I * J) + 2 * T * I + 4 * I * case["bias"] + 2 * T * I * case["res"]
        if case["ckpt"]:                                        # checkpoint written, read back, its values written
            b += 2 * (T * I + T * I // 32) + 2 * T * I
        return {"bytes": b, "flops": 2 * T * I * J // (2 if packed else 1)}
    if op == "wgrad":
        return {"bytes": 2 * T * I + T * J + T * J // 32 + 4 * I * J, "flops": 2 * T * I * J}
    n = T * case["C"]
    if op == "actgrad":
        return {"bytes": 2 * n + n + n // 32 + 2 * n + 4 * case["C"], "flops": 20 * n}
    return {"bytes": 2 * n + 2 * (n + n // 32) + 2 * n, "flops": 20 * n}


# ---- definitions in 64 bits ---------------------------------------------------------------------

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


def _ckpt64(x):
    """Values of the checkpoint of x, from the definition: the smallest power of two p with max |x| <= 127 p."""
    b = x.reshape(x.shape[0], -1, 32)
    p = torch.exp2(torch.floor(torch.log2(torch.clamp(b.abs().amax(-1, keepdim=True), min=2.0 ** -130)) - 7.0))
    for _ in range(3):
        p = torch.where(b.abs().amax(-1, keepdim=True) > 127.0 * p, 2.0 * p, p)
    p = torch.clamp(p, min=2.0 ** -126)
    return (torch.round(b / p) * p).reshape(x.shape)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "linear":
        vals = st["vals"].double()
        if st["meta"] is None:
            W = vals
        else:
            I, J = case["I"], case["J"]
            W = torch.zeros(I, J // 4, 4, dtype=torch.float64, device="cuda")
            pair = vals.view(I, J // 4, 2)
            g = torch.arange(J // 4, device="cuda")
            code = (st["meta"][:, g // 8] >> (4 * (g % 8)).to(torch.int32)) & 15
            for c in range(4):
                W[..., c] += torch.where((code & 3) == c, pair[..., 0], 0.0) + torch.where((code >> 2) == c, pair[..., 1], 0.0)
            W = W.view(I, J)
            del code
        z = torch.einsum("tj,ij->ti", st["X"].double(), W)
        del W
        if st["bias"] is not None:
            z += st["bias"].double()
        y = _act64(z, case["act"])
        if st["R"] is not None:
            y = y + st["R"].double()
        return {"Y": y, "Z": _ckpt64(z)} if case["ckpt"] else {"Y": y}
    if op == "actgrad":
        z = st["Zq"].double() * torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), st["Zs"].int() - 127).repeat_interleave(32, 1)
        dz = st["dY"].double() * _slope64(z, case["act"])
        return {"dZ": dz, "db": dz.sum(0)}
    if op == "ckpt":
        return {"X": _act64(_ckpt64(st["X"].double()), case["act"])}
    x = st["Xq"].double() * torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), st["Xs"].int() - 127).repeat_interleave(32, 1)
    return {"dW": torch.einsum("ti,tj->ij", st["dY"].double(), x)}
