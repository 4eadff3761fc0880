"""Workloads of the 8-bit serving operators whose speed is tracked.

RMSNorm with the residual's addition and an 8-bit output, the matrix product of
8-bit integers with a scale per token and per channel, and the attention of a
batch whose sequences share a long prefix.  A case is a dict of plain values.
``prepare`` makes what a serving program holds before the call, ``run`` makes
the call (``own``: of libcomfuse; otherwise in elementary torch operations),
``exact`` gives the same outputs in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-5
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3 = torch.float8_e4m3fn
QMAX = {"int8": 127.0, "e4m3": 448.0}
TYPES = {"bf16": BF16, "f32": F32}


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # Latency: the norm in front of a projection while one token is decoded.
        {"name": "norm_token", "op": "norm", "M": 1, "N": 4096, "dtype": "bf16", "code": "int8", "norm": True,
         "residual": True},
        # A ragged fp32 batch without a residual, in 8-bit floating point.
        {"name": "norm_ragged_f32", "op": "norm", "M": 777, "N": 5120, "dtype": "f32", "code": "e4m3", "norm": True,
         "residual": False},
        # Plain quantisation of an MLP's hidden activations.
        {"name": "quant_hidden", "op": "norm", "M": 4096, "N": 16384, "dtype": "bf16", "code": "int8", "norm": False,
         "residual": False},
        # 16384 tokens of a prefill through the norm, with the residual stream written back.
        {"name": "norm_large", "op": "norm", "M": 16384, "N": 4096, "dtype": "bf16", "code": "int8", "norm": True,
         "residual": True},
        # One token through a square projection: the weights are read once.
        {"name": "gemm_token", "op": "gemm", "M": 1, "N": 4096, "K": 4096, "out": "bf16", "bias": False, "act": "none"},
        # A decoding batch through the up projection of an MLP with its GELU.
        {"name": "gemm_batch", "op": "gemm", "M": 48, "N": 12288, "K": 4096, "out": "bf16", "bias": True, "act": "gelu"},
        # Odd sizes that no tile divides, fp32 output.
        {"name": "gemm_ragged_f32", "op": "gemm", "M": 1000, "N": 2003, "K": 1008, "out": "f32", "bias": True,
         "act": "none"},
        # 16384 tokens of a prefill through a square projection.
        {"name": "gemm_large", "op": "gemm", "M": 16384, "N": 4096, "K": 4096, "out": "bf16", "bias": False,
         "act": "none"},
        # Latency: four short continuations of one short prompt.
        {"name": "prefix_small", "op": "prefix", "B": 4, "H": 8, "Hk": 8, "Lq": 1, "P": 128, "S": 64, "d": 64,
         "causal": False},
        # Several draft tokens per sequence, every head with keys of its own, nothing a multiple of a block.
        {"name": "prefix_draft", "op": "prefix", "B": 16, "H": 16, "Hk": 16, "Lq": 5, "P": 4095, "S": 333, "d": 64,
         "causal": True},
        # A decoding step of 64 sequences on one long prompt, 4 query heads per key head.
        {"name": "prefix_decode", "op": "prefix", "B": 64, "H": 32, "Hk": 8, "Lq": 1, "P": 8192, "S": 512, "d": 128,
         "causal": False},
        # Prefill of the sequences' own parts behind the shared prompt.
        {"name": "prefix_prefill", "op": "prefix", "B": 8, "H": 32, "Hk": 8, "Lq": 500, "P": 2048, "S": 500, "d": 128,
         "causal": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the ranges of the listed ones."""
    op = rng.choice(["norm", "gemm", "prefix"])
    if op == "norm":
        n = rng.choice([_log(rng, 64, 16384), 8 * _log(rng, 16, 2048), 64 * _log(rng, 4, 256)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 16384 * 4096 // (n * (2 if dtype == "f32" else 1))
        return {"op": op, "M": _log(rng, 1, max(1, min(65536, most))), "N": n, "dtype": dtype,
                "code": rng.choice(["int8", "int8", "e4m3"]), "norm": rng.choice([True, True, False]),
                "residual": rng.choice([True, True, False])}
    if op == "gemm":
        n = rng.choice([_log(rng, 64, 16384), 64 * _log(rng, 8, 256)])
        k = rng.choice([16 * _log(rng, 8, 1024), 64 * _log(rng, 8, 256)])
        most = 16384 * 4096 * 4096 // (n * k)
        return {"op": op, "M": _log(rng, 1, max(1, min(16384, most))), "N": n, "K": k,
                "out": rng.choice(["bf16", "bf16", "f32"]), "bias": rng.choice([True, False]),
                "act": rng.choice(["none", "none", "gelu", "gelu_tanh", "relu"])}
    hk, g = rng.choice([(8, 1), (16, 1), (8, 4), (4, 8), (2, 7), (1, 8), (8, 8), (12, 1)])
    d, p = rng.choice([64, 128, 128]), _log(rng, 64, 16384)
    form = rng.choice(["decode", "decode", "draft", "prefill"])
    if form == "prefill":
        lq = _log(rng, 16, 512)
        s, b = lq + rng.choice([0, _log(rng, 1, 512)]), _log(rng, 1, 8)
    else:
        lq = 1 if form == "decode" else rng.randint(2, 16)
        s, b = max(lq, _log(rng, 16, 2048)), _log(rng, 1, 64)
    # no more than the largest listed one
    while b > 1 and (b * hk * g * lq * (p + s) > 8 * 32 * 500 * 2548 or b * hk * s * d > 64 * 8 * 512 * 128):
        b //= 2
    p = min(p, max(64, 8 * 32 * 500 * 2548 // (b * hk * g * lq)))
    return {"op": op, "B": b, "H": hk * g, "Hk": hk, "Lq": lq, "P": p, "S": s, "d": d, "causal": lq > 1}


# ---------------------------------------------------------------- inputs
def _rows(M, N, dtype, g, std=1.0):
    """Normal [M, N] values in rows of a multiple of 16 bytes."""
    ld = -(-N // 16) * 16
    return (torch.randn((M, ld), generator=g, device="cuda", dtype=F32) * std).to(dtype)[:, :N]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case)
    if case["op"] == "norm":
        M, N, dtype = case["M"], case["N"], TYPES[case["dtype"]]
        x = _rows(M, N, F32, g)
        x[:, 5::173] *= 12.0                       # channels of outliers, as activations have them
        s["x"] = torch.empty((M, -(-N // 16) * 16), device="cuda", dtype=dtype)[:, :N].copy_(x)
        s["r"] = _rows(M, N, dtype, g, 3.0) if case["residual"] else None
        s["gamma"] = (torch.randn((N,), generator=g, device="cuda") * 0.1 + 1.0) if case["norm"] else None
        return s
    if case["op"] == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        s["a"] = (torch.randn((M, K), generator=g, device="cuda") * 30.0).round().clamp(-127, 127).to(torch.int8)
        s["b"] = (torch.randn((N, K), generator=g, device="cuda") * 36.0).round().clamp(-127, 127).to(torch.int8)
        s["sa"] = torch.rand((M,), generator=g, device="cuda") * 0.03 + 0.01
        s["sb"] = (torch.rand((N,), generator=g, device="cuda") + 0.5) / (36.0 * K ** 0.5)
        s["bias"] = torch.randn((N,), generator=g, device="cuda") * 0.1 if case["bias"] else None
        return s
    B, H, Hk, Lq, P, S, d = (case[k] for k in ("B", "H", "Hk", "Lq", "P", "S", "d"))

    def r(*shape):                                  # token-major, as projections and caches are; heads second
        return torch.randn(shape, generator=g, device="cuda", dtype=F32).to(BF16).transpose(-3, -2)

    s["q"] = r(B, Lq, H, d)
    s["kp"], s["vp"] = r(P, Hk, d), r(P, Hk, d)
    s["ks"], s["vs"] = r(B, S, Hk, d), r(B, S, Hk, d)
    s["lens"] = torch.randint(max(Lq, S // 2), S + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    return s


# ---------------------------------------------------------------- one pass
# 8-bit codes are returned as they are held, beside the scale of their row: an
# int8 code stands for that whole number times the scale, an E4M3 code for its
# value times the scale.
def run(s):
    op = s["op"]
    if own:
        from paper_2608_03537_amd import comfuse as cf
        if op == "norm":
            q, sc, h = cf.rmsnorm_quant(s["x"], s["r"], s["gamma"], eps=EPS, norm=s["norm"], code=s["code"])
            return {"codes": q if s["code"] == "int8" else q.view(E4M3), "scale": sc, "h": h}
        if op == "gemm":
            return {"c": cf.gemm_i8(s["a"], s["b"], s["sa"], s["sb"], bias=s["bias"], act=s["act"],
                                    out_dtype=TYPES[s["out"]])}
        return {"o": cf.attention_prefix(s["q"], s["kp"], s["vp"], s["ks"], s["vs"], s["lens"], causal=s["causal"])}
    return _plain_norm(s) if op == "norm" else _plain_gemm(s) if op == "gemm" else _plain_prefix(s)


def _plain_norm(s):
    x = s["x"].float()
    h = x if s["r"] is None else x + s["r"].float()
    t = h if s["gamma"] is None else h * s["gamma"]
    d = t.abs().amax(-1, keepdim=True)
    d = d / torch.full_like(d, QMAX[s["code"]])
    z = torch.where(d > 0, t / d, torch.zeros_like(t))
    codes = z.round().to(torch.int8) if s["code"] == "int8" else z.to(E4M3)
    scale = d[:, 0]
    if s["norm"]:
        scale = scale / torch.sqrt((h * h).mean(-1) + EPS)
    return {"codes": codes, "scale": scale, "h": None if s["r"] is None else h.to(s["x"].dtype)}


def _plain_gemm(s):
    y = s["a"].float() @ s["b"].float().t()
    y = y * s["sa"][:, None] * s["sb"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["act"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * 0.5 ** 0.5))
    elif s["act"] == "gelu_tanh":
        y = 0.5 * y * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (y + 0.044715 * y * y * y)))
    elif s["act"] == "relu":
        y = torch.clamp(y, min=0.0)
    return {"c": y.to(TYPES[s["out"]])}


def _plain_prefix(s):
    q, B, H, Hk, Lq, P, S, d = s["q"], *(s[k] for k in ("B", "H", "Hk", "Lq", "P", "S", "d"))
    G = H // Hk
    qf = q.float().reshape(B, Hk, G * Lq, d) * d ** -0.5
    kp, vp, ks, vs = s["kp"].float(), s["vp"].float(), s["ks"].float(), s["vs"].float()
    sp = torch.matmul(qf.transpose(0, 1).reshape(Hk, B * G * Lq, d), kp.transpose(1, 2).contiguous())
    sp = sp.reshape(Hk, B, G * Lq, P).transpose(0, 1)
    so = torch.matmul(qf, ks.transpose(2, 3).contiguous())
    limit = s["lens"].long()[:, None]                                   # own keys that query i sees
    if s["causal"]:
        limit = limit - (Lq - 1 - torch.arange(Lq, device=q.device))
    limit = limit.expand(B, Lq)[:, None, None, :, None].expand(B, 1, G, Lq, 1).reshape(B, 1, G * Lq, 1)
    so = torch.where(torch.arange(S, device=q.device) < limit, so, torch.full_like(so, -math.inf))
    m = torch.maximum(sp.amax(-1, keepdim=True), so.amax(-1, keepdim=True))
    pp, po = torch.exp(sp - m), torch.exp(so - m)
    total = pp.sum(-1, keepdim=True) + po.sum(-1, keepdim=True)
    o = torch.matmul(pp.transpose(0, 1).reshape(Hk, B * G * Lq, P), vp).reshape(Hk, B, G * Lq, d).transpose(0, 1)
    o = (o + torch.matmul(po, vs)) / total
    return {"o": o.reshape(B, H, Lq, d).to(BF16)}


# ---------------------------------------------------------------- bytes and operations of one pass
def work(case):
    if case["op"] == "norm":
        M, N, e = case["M"], case["N"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": M * N * (e * (3 if case["residual"] else 1) + 1) + 4 * M + (4 * N if case["norm"] else 0),
                "flops": M * N * (2 + int(case["residual"]) + (3 if case["norm"] else 0))}
    if case["op"] == "gemm":
        M, N, K, e = case["M"], case["N"], case["K"], 2 if case["out"] == "bf16" else 4
        return {"bytes": M * K + N * K + e * M * N + 4 * M + (8 if case["bias"] else 4) * N, "flops": 2 * M * N * K}
    B, H, Hk, Lq, P, S, d = (case[k] for k in ("B", "H", "Hk", "Lq", "P", "S", "d"))
    own_keys = B * (max(Lq, S // 2) + S) / 2                             # the mean of their lengths
    seen = own_keys - (B * (Lq - 1) / 2 if case["causal"] else 0)
    return {"bytes": 4 * B * H * Lq * d + 4 * Hk * d * (P + own_keys) + 4 * B, "flops": 4 * d * H * Lq * (B * P + seen)}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["x"].to(F64)
        if s["r"] is not None:
            h = h + s["r"].to(F64)
        t = h * s["gamma"].to(F64) if s["gamma"] is not None else h
        step = t.abs().max(dim=1).values / QMAX[case["code"]]
        scale = step * (h.square().sum(1) / case["N"] + EPS).rsqrt() if case["norm"] else step
        return {"codes": None if case["code"] == "int8" else t / step[:, None], "scale": scale,
                "h": None if s["r"] is None else h}
    if case["op"] == "gemm":
        y = torch.mm(s["a"].to(F64), s["b"].to(F64).t())
        y = y * torch.outer(s["sa"].to(F64), s["sb"].to(F64))
        if s["bias"] is not None:
            y += s["bias"].to(F64)
        if case["act"] == "gelu":
            y = y * torch.special.ndtr(y)
        elif case["act"] == "gelu_tanh":
            y = y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
        elif case["act"] == "relu":
            y = torch.where(y > 0, y, torch.zeros_like(y))
        return {"c": y}
    B, H, Hk, Lq, P, d = (case[k] for k in ("B", "H", "Hk", "Lq", "P", "d"))
    out = torch.zeros((B, H, Lq, d), device="cuda", dtype=F64)
    lens = s["lens"].tolist()
    for h in range(H):
        kp, vp = s["kp"][h // (H // Hk)].to(F64), s["vp"][h // (H // Hk)].to(F64)
        for b in range(B):
            n = lens[b]
            keys = torch.cat([kp, s["ks"][b, h // (H // Hk), :n].to(F64)])
            vals = torch.cat([vp, s["vs"][b, h // (H // Hk), :n].to(F64)])
            x = s["q"][b, h].to(F64) @ keys.t() / math.sqrt(d)
            if case["causal"]:
                x = x.masked_fill(torch.ones_like(x, dtype=torch.bool).triu(P + n - Lq + 1), -math.inf)
            out[b, h] = x.softmax(-1) @ vals
    return {"o": out}
