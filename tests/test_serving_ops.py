"""The 8-bit serving operators against their definitions in 64 bits: RMSNorm to
8-bit codes, the int8 product, attention over a shared prefix, and a layer's run
of all three.  u is fp32's half step; each bound counts roundings."""
import math
import threading

import pytest
import torch

from paper_2608_03537_amd import comfuse as cf

U = 2.0 ** -24                                      # half a step of fp32
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
QMAX = {"int8": 127.0, "e4m3": 448.0}
gpu = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def padded(M, N, dtype, g, std=1.0, pad=0, fill=float("nan")):
    """Normal [M, N] values; `fill` between N and the leading dimension."""
    per = 16 // torch.empty((), dtype=dtype).element_size()
    t = torch.full((M, -(-N // per) * per + pad), fill, dtype=dtype, device="cuda")
    t[:, :N] = torch.randn((M, N), generator=g, device="cuda") * std
    return t[:, :N]


# ---------------------------------------------------------------- rmsnorm_quant
def norm_ref(X, R, gamma, eps, norm, code):
    """(t / d, s, h) in 64 bits."""
    h = X.to(F64) if R is None else X.to(F64) + R.to(F64)
    t = h if gamma is None else h * gamma.to(F64)
    m = t.abs().amax(-1)
    d = m / QMAX[code]
    s = d / torch.sqrt((h * h).mean(-1) + eps) if norm else d
    return torch.where(m[:, None] > 0, t / d[:, None], torch.zeros_like(t)), torch.where(m > 0, s, 0.0), h


def check_norm(Q, s, H, ref, code, dtype):
    z, sr, h = ref
    q = Q.to(F64) if code == "int8" else Q.contiguous().view(torch.float8_e4m3fn).to(F64)
    # roundings of h, t, d and t / d, then the code's half step (E4M3: relative 2^-4, subnormals 2^-10)
    half = 0.5 if code == "int8" else torch.clamp(z.abs() * 2.0 ** -4, min=2.0 ** -10)
    assert bool(((q - z).abs() <= half + 4.1 * U * QMAX[code]).all())
    # s: h, t, d and the quotient, half of h^2 and of a sum of at most 64 terms a lane and 10 levels, the root
    assert bool(((s.to(F64) - sr).abs() <= (5 + (3 + 74) / 2) * U * sr).all())
    if H is not None:
        assert bool(((H.to(F64) - h).abs() <= (HALF[dtype] + U) * h.abs()).all())


@gpu
@pytest.mark.parametrize("dtype,code,norm,res", [(BF16, "int8", True, True), (BF16, "e4m3", True, False),
                                                 (F32, "int8", False, True), (F32, "e4m3", True, True)])
@pytest.mark.parametrize("M,N", [(1, 1), (3, 7), (5, 64), (2, 513), (9, 1000), (4, 2048), (3, 2050), (2, 4096),
                                 (7, 5120), (2, 8200), (1, 16384), (2, 16391), (1, 32768)])
def test_norm_codes(M, N, dtype, code, norm, res):
    g = gen(M * 100003 + N)
    X = padded(M, N, dtype, g, pad=16)
    R = padded(M, N, dtype, g, 3.0) if res else None
    gamma = torch.randn((N,), generator=g, device="cuda") if norm else None
    Q, s, H = cf.rmsnorm_quant(X, R, gamma, eps=1e-5, norm=norm, code=code)
    assert (H is None) == (R is None) and Q.shape == X.shape and s.shape == (M,)
    check_norm(Q, s, H, norm_ref(X, R, gamma, 1e-5, norm, code), code, dtype)


@gpu
@pytest.mark.parametrize("N", [40, 700, 3000, 9000])
def test_norm_codes_are_the_fp32_quotients(N):
    """The codes are those of the fp32 chain h, t, d = m / 127, t / d, bit for bit."""
    g = gen(N)
    X, R = padded(64, N, BF16, g), padded(64, N, BF16, g)
    gamma = torch.randn((N,), generator=g, device="cuda")
    Q, _, _ = cf.rmsnorm_quant(X, R, gamma)
    t = (X.float().cpu() + R.float().cpu()) * gamma.cpu()
    m = t.abs().amax(-1, keepdim=True)
    assert torch.equal(Q.cpu(), (t / (m / torch.full_like(m, 127.0))).round().to(torch.int8))


@gpu
@pytest.mark.parametrize("N", [24, 1500, 5000, 20000])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_norm_special_rows(N, code):
    """All-zero, NaN, infinite, tiny and huge rows, beside an ordinary one."""
    g = gen(N)
    X = padded(8, N, F32, g)
    X[1] = 0.0
    X[2, N // 2] = float("nan")
    X[3, N - 1] = -math.inf
    X[4] *= 1e-38
    X[5] = torch.where(X[5] > 1, 1e-44, 0.0)
    X[6] *= 1e37
    Q, s, _ = cf.rmsnorm_quant(X, norm=False, code=code)
    z, sr, _ = norm_ref(X, None, None, 0.0, False, code)
    q = Q.to(F64) if code == "int8" else Q.contiguous().view(torch.float8_e4m3fn).to(F64)
    assert not q[1:4].any() and s[1] == 0 and s[2].isnan() and s[3].isnan()
    rows = [0, 4, 5, 6, 7]
    half = 0.5 if code == "int8" else torch.clamp(z[rows].abs() * 2.0 ** -4, min=2.0 ** -10)
    assert bool(((q[rows] - z[rows]).abs() <= half + 4.1 * U * QMAX[code]).all())
    # the smallest step of fp32 is 2^-149, so a tiny scale is off by half of it
    assert bool(((s.to(F64)[rows] - sr[rows]).abs() <= 4 * U * sr[rows] + 2.0 ** -150).all())


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_in_place_strides_and_padding(dtype):
    g = gen(7)
    M, N = 37, 1003
    X, gamma = padded(M, N, dtype, g, pad=32), torch.randn((N,), generator=g, device="cuda")
    R = padded(M, N, dtype, g, pad=48, fill=5.0)
    want = cf.rmsnorm_quant(X, R._base.clone()[:, :N], gamma)
    full = torch.full((M, 1024), 99, dtype=torch.int8, device="cuda")
    Q, s, H = cf.rmsnorm_quant(X, R, gamma, residual=R, out=full[:, :N])
    assert H is R and torch.equal(Q, want[0]) and torch.equal(s, want[1]) and torch.equal(R, want[2])
    assert bool((full[:, N:] == 99).all()) and bool((R._base[:, N:] == 5.0).all())


@gpu
def test_norm_more_rows_than_a_grid():
    """Four rows a workgroup of 256 threads: 2^26 + 5 rows are more than 2^32 threads."""
    M, N = (1 << 26) + 5, 8
    X = torch.zeros((M, N), dtype=BF16, device="cuda")
    out = torch.full((M, 16), 77, dtype=torch.int8, device="cuda")[:, :N]
    at = torch.tensor([0, 5, (1 << 25) - 1, 1 << 25, (1 << 26) - 1, 1 << 26, M - 1], device="cuda")
    X[at] = torch.randn((7, N), generator=gen(12), device="cuda").to(BF16)
    H = X.clone()
    Q, s, _ = cf.rmsnorm_quant(X, H, residual=H, out=out)
    check_norm(Q[at], s[at], H[at], norm_ref(X[at], X[at], None, 1e-5, True, "int8"), "int8", BF16)
    assert int((s != 0).sum()) == 7 and int(Q.any(1).sum()) == 7 and int(H.any(1).sum()) == 7


# ---------------------------------------------------------------- gemm_i8
def act64(y, act):
    if act == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y / math.sqrt(2.0)))
    if act == "gelu_tanh":
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
    return y.clamp(min=0.0) if act == "relu" else y


def check_gemm(C, A, B, sa, sb, bias, act):
    v = (A.to(F64) @ B.to(F64).t())
    v = v * (1.0 if sa is None else sa.to(F64)[:, None]) * (1.0 if sb is None else sb.to(F64))
    x = v if bias is None else v + bias.to(F64)
    # the conversion of the sum, two scales, the bias; GELU's slope is at most 1.13 and
    # its erf (or tanh) is off by at most 2e-6: 1e-6 |x|
    dx = 4.1 * U * (v.abs() + (0.0 if bias is None else bias.to(F64).abs()))
    y = act64(x, act)
    tol = (1.13 * dx + 1e-6 * x.abs() if act.startswith("gelu") else dx) * 1.01 + HALF[C.dtype] * 1.01 * y.abs()
    bad = (C.to(F64) - y).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


def i8(g, *shape):
    return torch.randint(-128, 128, shape, generator=g, device="cuda", dtype=torch.int32).to(torch.int8)


SIZES = [(1, 1, 16), (1, 5, 32), (1, 4096, 4096), (2, 100, 48), (3, 33, 272), (7, 64, 1040), (16, 128, 128),
         (17, 200, 4112), (31, 1000, 400), (33, 257, 16), (48, 512, 2048), (64, 96, 640), (65, 65, 144), (100, 130, 1008),
         (127, 129, 256), (200, 384, 528), (256, 256, 128), (257, 511, 384), (300, 1030, 1136), (513, 770, 512),
         (1000, 2003, 1008), (2050, 2306, 272)]


@gpu
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gemm_i8_sizes(M, N, K):
    g = gen(M + N + K)
    A, B = i8(g, M, K), i8(g, N, K)
    sa, sb = torch.rand((M,), generator=g, device="cuda"), torch.rand((N,), generator=g, device="cuda") / K
    bias = torch.randn((N,), generator=g, device="cuda")
    for dt in (BF16, F32):
        check_gemm(cf.gemm_i8(A, B, sa, sb, bias=bias, out_dtype=dt), A, B, sa, sb, bias, "none")


@gpu
@pytest.mark.parametrize("M,N,K", [
    (128, 4096, 4112), (20, 12200, 560), (60, 9000, 720), (40, 9000, 1232), (300, 2000, 6032), (500, 3900, 16), (500, 3900, 112),
    (500, 3900, 240), (500, 3900, 400), (130, 9000, 720), (1000, 4000, 144), (1000, 4000, 272), (130, 11000, 80),
    (1000, 4000, 1008), (5000, 1000, 4176), (1900, 4000, 16), (1900, 4000, 160), (2500, 8100, 48), (4090, 4081, 4112),
    (16300, 4090, 304), (16000, 4090, 1040), (4090, 4000, 2160), (4000, 4081, 1984), (8000, 3900, 1936), (13079, 16, 3664), (8500, 17, 48)])
def test_gemm_i8_ends_of_k(M, N, K):
    """K that ends inside a step, with few steps, on every shape of tile."""
    g = gen(M + N + K)
    A, B = i8(g, M, K), i8(g, N, K)
    check_gemm(cf.gemm_i8(A, B, out_dtype=F32), A, B, None, None, None, "none")


@gpu
def test_gemm_i8_more_tokens_than_a_grid_of_small_tiles():
    """2^29 + 40 rows and one column: tiles of 32 rows and 256 threads would be 2^32 threads."""
    M = (1 << 29) + 40
    A = torch.zeros((M, 16), dtype=torch.int8, device="cuda")
    at = torch.tensor([0, 1, (1 << 28) + 3, (1 << 29) - 1, 1 << 29, M - 1], device="cuda")
    A[at] = i8(gen(13), 6, 16)
    B = torch.ones((1, 16), dtype=torch.int8, device="cuda")
    C = cf.gemm_i8(A, B)                             # rows of 16 bytes: 8 GiB
    want = A[at].to(F64).sum(-1, keepdim=True)
    assert bool(((C[at].to(F64) - want).abs() <= 2.0 ** -8 * want.abs()).all())
    assert int((C != 0).sum()) == int((want != 0).sum())


@gpu
@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("M", [1, 20, 90, 600])
def test_gemm_i8_epilogues(M, act):
    g = gen(M)
    N, K = 700, 320
    A, B = i8(g, M, K), i8(g, N, K)
    sa, sb = torch.rand((M,), generator=g, device="cuda") * 0.02, torch.rand((N,), generator=g, device="cuda") * 0.02
    bias = torch.randn((N,), generator=g, device="cuda")
    for a, b, c in ((sa, sb, bias), (None, sb, None), (sa, None, bias)):
        check_gemm(cf.gemm_i8(A, B, a, b, bias=c, act=act, out_dtype=F32), A, B, a, b, c, act)


@gpu
@pytest.mark.parametrize("M,N", [(1, 40), (40, 40), (300, 300)])
def test_gemm_i8_extreme_sums(M, N):
    """All products 2^14 over the longest K: the sum stays exact."""
    K = 131056
    A = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    B = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    B[N // 2] = 127
    C = cf.gemm_i8(A, B, out_dtype=F32)
    want = torch.full((N,), K * 16384.0, dtype=F64)
    want[N // 2] = -K * 128 * 127.0
    assert bool((C.to(F64).cpu() - want).abs().max() <= U * K * 16384.0)


@gpu
@pytest.mark.parametrize("M", [5, 70, 400])
def test_gemm_i8_strides_and_padding(M):
    g = gen(M)
    N, K = 333, 208
    A, B = i8(g, M, K + 64)[:, 16:16 + K], i8(g, N, K + 32)[:, :K]
    sa, sb = torch.rand((M,), generator=g, device="cuda"), torch.rand((N,), generator=g, device="cuda") / K
    for dt in (BF16, F32):
        full = torch.full((M + 1, 352), 7.0, dtype=dt, device="cuda")
        C = cf.gemm_i8(A, B, sa, sb, out=full[:M, :N])
        check_gemm(C, A, B, sa, sb, None, "none")
        assert bool((full[M:] == 7).all()) and bool((full[:, N:] == 7).all())


# ---------------------------------------------------------------- attention_prefix
def attend64(Q, Kp, Vp, Ks, Vs, lens, causal, scale):
    """(O, sum of w |v|) in 64 bits, row by row of sequences."""
    B, H, Lq, d = Q.shape
    Hk = Kp.shape[0]
    O, A = torch.zeros(Q.shape, dtype=F64, device=Q.device), torch.zeros(Q.shape, dtype=F64, device=Q.device)
    for b in range(B):
        n = 0 if Ks is None else Ks.shape[2] if lens is None else max(0, min(int(lens[b]), Ks.shape[2]))
        for h in range(Hk):
            k, v = Kp[h].to(F64), Vp[h].to(F64)
            if n:
                k, v = torch.cat([k, Ks[b, h, :n].to(F64)]), torch.cat([v, Vs[b, h, :n].to(F64)])
            if not k.shape[0]:
                continue
            q = Q[b, h * (H // Hk):(h + 1) * (H // Hk)].to(F64)
            x = (q @ k.t()) * scale
            if causal:
                seen = Kp.shape[1] + (n - (Lq - 1 - torch.arange(Lq, device=Q.device))).clamp(min=0)
                x = x.masked_fill(torch.arange(k.shape[0], device=Q.device) >= seen[:, None], -math.inf)
            w = torch.softmax(x, -1)
            if causal:
                w = torch.where((seen <= 0)[:, None], 0.0, w)
            O[b, h * (H // Hk):(h + 1) * (H // Hk)] = w @ v
            A[b, h * (H // Hk):(h + 1) * (H // Hk)] = w @ v.abs()
    return O, A


def check_attention(O, Q, Kp, Vp, Ks, Vs, lens, causal=False, scale=None):
    scale = Q.shape[-1] ** -0.5 if scale is None else scale
    ref, a = attend64(Q, Kp, Vp, Ks, Vs, lens, causal, scale)
    # P is rounded to bf16 in numerator and denominator alike: off by 2^-8 sum w |v - o|;
    # a score is off by d u |q| |k| scale, and a weight by twice that and the exponentials' 4 u;
    # then the output's rounding
    longest = [float(t.float().norm(dim=-1).max()) for t in (Q, Kp, Ks) if t is not None and t.numel()]
    e = 2 * Q.shape[-1] * U * longest[0] * max(longest[1:]) * scale + 8 * U
    # exponentials below fp32's smallest normal 2^-126 are flushed to 0: beside a row's largest weight,
    # which is at least 2^-8, each key loses at most 2^-118 |v|
    keys = Kp.shape[1] + (0 if Ks is None else Ks.shape[2])
    lost = keys * 2.0 ** -118 * max(float(t.float().abs().max()) for t in (Vp, Vs) if t is not None and t.numel())
    tol = (2.0 ** -8 * 1.01 + e) * (a + ref.abs()) + 2.0 ** -8 * 1.01 * ref.abs() + lost
    bad = ~((O.to(F64) - ref).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), O[bad][:4].tolist(), ref[bad][:4].tolist())


def prefix_inputs(g, B, H, Hk, Lq, P, S, d, std=1.0):
    def r(*shape):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(BF16)
    return r(B, H, Lq, d), r(Hk, P, d), r(Hk, P, d), r(B, Hk, S, d), r(B, Hk, S, d)


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,Hk,Lq,P,S", [
    (1, 1, 1, 1, 1, 1), (2, 4, 2, 1, 31, 7), (3, 8, 8, 1, 64, 33), (5, 8, 1, 1, 129, 65), (4, 14, 2, 1, 1000, 100),
    (2, 6, 2, 5, 257, 40), (1, 8, 2, 16, 63, 16), (3, 4, 4, 33, 300, 50), (2, 8, 2, 70, 100, 130), (9, 32, 8, 1, 2048, 64),
    (33, 8, 2, 1, 777, 260), (1, 2, 1, 1, 5000, 3), (70, 4, 4, 1, 512, 20), (2, 2, 2, 3, 4, 3000), (4, 4, 1, 40, 600, 40)])
@pytest.mark.parametrize("causal", [False, True])
def test_prefix_sizes(B, H, Hk, Lq, P, S, d, causal):
    g = gen(B * 7 + H + Lq + P + S + d)
    Q, Kp, Vp, Ks, Vs = prefix_inputs(g, B, H, Hk, Lq, P, S, d)
    lens = torch.randint(0, S + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    O = cf.attention_prefix(Q, Kp, Vp, Ks, Vs, lens, causal=causal)
    check_attention(O, Q, Kp, Vp, Ks, Vs, lens, causal)


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_prefix_without_lens_or_own_keys_or_prefix(d):
    g = gen(d)
    Q, Kp, Vp, Ks, Vs = prefix_inputs(g, 3, 4, 2, 2, 70, 45, d)
    check_attention(cf.attention_prefix(Q, Kp, Vp, Ks, Vs), Q, Kp, Vp, Ks, Vs, None)
    check_attention(cf.attention_prefix(Q, Kp, Vp), Q, Kp, Vp, None, None, None)
    check_attention(cf.attention_prefix(Q, Kp[:, :0], Vp[:, :0], Ks, Vs, scale=0.3), Q, Kp[:, :0], Vp[:, :0], Ks, Vs, None,
                    scale=0.3)
    assert cf.attention_prefix(Q[:0], Kp, Vp, Ks[:0], Vs[:0]).shape == (0, 4, 2, d)
    assert cf.attention_prefix(Q[:, :, :0], Kp, Vp, Ks, Vs).shape == (3, 4, 0, d)


@gpu
@pytest.mark.parametrize("d,Lq,S", [(64, 1, 40), (128, 1, 300), (128, 5, 2000), (64, 40, 90)])
def test_prefix_rows_without_keys_and_stale_cache(d, Lq, S):
    """No prefix: rows of empty sequences are 0.  What lies behind a length (NaN, infinity) is not used,
    and lengths outside [0, S] are clamped."""
    g = gen(d + Lq)
    B = 5
    Q, Kp, Vp, Ks, Vs = prefix_inputs(g, B, 4, 2, Lq, 17, S, d)
    lens = torch.tensor([0, 1, -3, S + 5, S // 2], dtype=torch.int32, device="cuda")
    n = lens.clamp(0, S)
    behind = torch.arange(S, device="cuda")[None, None, :, None] >= n[:, None, None, None]
    clean = [torch.where(behind, 0.0, t.float()).to(BF16) for t in (Ks, Vs)]
    Ks.masked_fill_(behind, float("nan"))
    Vs.masked_fill_(behind, math.inf)
    for causal in (False, True):
        for P in (0, 17):
            O = cf.attention_prefix(Q, Kp[:, :P], Vp[:, :P], Ks, Vs, lens, causal=causal)
            check_attention(O, Q, Kp[:, :P], Vp[:, :P], *clean, n, causal)
            if P == 0:
                assert not O[0].any() and not O[2].any()
                if causal and Lq > 1:
                    assert not O[1, :, :Lq - 1].any() and bool(O[1, :, Lq - 1].any())


@gpu
@pytest.mark.parametrize("B,H,Hk,Lq,P,S,d", [
    (3, 8, 8, 39, 409, 443, 128), (2, 8, 1, 12, 900, 19, 64), (1, 8, 8, 49, 2300, 51, 64), (1, 4, 4, 33, 0, 700, 128),
    (5, 14, 2, 12, 1500, 70, 128), (1, 2, 2, 65, 1100, 65, 64), (6, 8, 8, 30, 1700, 30, 128), (3, 6, 2, 150, 1200, 160, 64)])
def test_prefix_in_uneven_parts(B, H, Hk, Lq, P, S, d):
    """Between 33 and 96 rows of a (sequence, key head), and numbers of parts that are no power of two."""
    g = gen(B + Lq + P)
    a = prefix_inputs(g, B, H, Hk, Lq, P, S, d)
    lens = torch.randint(0, S + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    lens[0] = S
    for causal in (False, True):
        check_attention(cf.attention_prefix(*a, lens, causal=causal), *a, lens, causal)


@gpu
@pytest.mark.parametrize("d,H,Lq", [(64, 4, 5), (128, 8, 3), (64, 16, 40)])
def test_prefix_rows_without_keys_beside_nan_values(d, H, Lq):
    """A query that sees no key gets 0, also where the keys of the later queries hold values that are not finite."""
    Q, Kp, Vp, Ks, Vs = prefix_inputs(gen(14), 3, H, 2, Lq, 0, 300, d)
    lens = torch.tensor([1, 0, 2], dtype=torch.int32, device="cuda")
    Vs[0, :, 0] = float("nan")
    Vs[2, :, 1] = math.inf
    O = cf.attention_prefix(Q, Kp, Vp, Ks, Vs, lens, causal=True)
    assert not O[0, :, :-1].any() and not O[1].any() and not O[2, :, :-2].any()
    assert bool(O[0, :, -1].isnan().all()) and not bool(O[2, :, -1].isfinite().any())


@gpu
@pytest.mark.parametrize("Lq", [1, 48])
def test_prefix_special_scores(Lq):
    """Infinite values stay in their own column; rows whose scores are all -infinity and scores with a
    NaN are NaN, as softmax has them; large scores do not overflow."""
    g = gen(Lq)
    B, H, d = 2, 4, 64
    Q, Kp, Vp, Ks, Vs = prefix_inputs(g, B, H, 2, Lq, 100, 70, d)
    Vp[0, 3, 5] = math.inf
    Vs[1, 1, 69, 7] = -math.inf
    O = cf.attention_prefix(Q, Kp, Vp, Ks, Vs)
    inf = torch.zeros_like(O, dtype=torch.bool)
    inf[:, :2, :, 5] = True
    inf[1, 2:, :, 7] = True
    assert torch.equal(O.isinf(), inf) and not O.isnan().any()
    Vp[0, 3, 5], Vs[1, 1, 69, 7] = 0.0, 0.0
    check_attention(cf.attention_prefix(Q * 30, Kp, Vp, Ks, Vs, scale=1.0), Q * 30, Kp, Vp, Ks, Vs, None, scale=1.0)
    Ks[0, 0, 2, 0] = float("nan")
    O = cf.attention_prefix(Q, Kp, Vp, Ks, Vs)
    assert bool(O[0, :2].isnan().all()) and not O[0, 2:].isnan().any() and not O[1].isnan().any()
    Q = Q.abs() + 0.1
    Kp[:], Ks[:] = -math.inf, -math.inf
    assert bool(cf.attention_prefix(Q, Kp, Vp, Ks, Vs).isnan().all())


@gpu
@pytest.mark.parametrize("Lq", [1, 3, 64])
def test_prefix_strides(Lq):
    """Token-major caches and projections, parts of larger buffers, and a given output."""
    g = gen(Lq)
    B, H, Hk, P, S, d = 3, 8, 2, 90, 50, 128
    qkv = torch.randn((B, Lq, (H + 2 * Hk) * d), generator=g, device="cuda").to(BF16)
    Q = qkv[:, :, :H * d].unflatten(-1, (H, d)).transpose(1, 2)
    cache = torch.randn((B, S, 2, Hk, d), generator=g, device="cuda").to(BF16)
    Ks, Vs = cache[:, :, 0].transpose(1, 2), cache[:, :, 1].transpose(1, 2)
    prompt = torch.randn((P + 9, 2, Hk, d), generator=g, device="cuda").to(BF16)
    Kp, Vp = prompt[9:, 0].transpose(0, 1), prompt[9:, 1].transpose(0, 1)
    lens = torch.tensor([S, 7, 20], dtype=torch.int32, device="cuda")
    big = torch.full((B, Lq, H + 1, d), 3.0, dtype=BF16, device="cuda")
    out = big[:, :, :H].transpose(1, 2)
    O = cf.attention_prefix(Q, Kp, Vp, Ks, Vs, lens, causal=True, out=out)
    assert O is out and bool((big[:, :, H] == 3).all())
    check_attention(O, Q, Kp, Vp, Ks, Vs, lens, True)
    same = cf.attention_prefix(*(t.contiguous() for t in (Q, Kp, Vp, Ks, Vs)), lens, causal=True)
    assert torch.equal(same, O)


# ---------------------------------------------------------------- the operators together
def serving_layer(x, r, w, cache, lens):
    """A decoding step of a layer: norm, QKV, attention over prompt and cache, projection, norm, MLP."""
    B, D = x.shape
    H, Hk, d = w["H"], w["Hk"], w["d"]
    a, sa, r = cf.rmsnorm_quant(x, r, w["g1"])
    qkv = cf.gemm_i8(a, w["qkv"], sa, w["s_qkv"], bias=w["b_qkv"])
    q = qkv[:, :H * d].view(B, 1, H, d).transpose(1, 2)
    k, v = (qkv[:, (H + i * Hk) * d:(H + (i + 1) * Hk) * d].view(B, Hk, d) for i in (0, 1))
    at = torch.arange(B, device=x.device), slice(None), (lens - 1).long()
    cache["k"][at], cache["v"][at] = k, v
    o = cf.attention_prefix(q, cache["kp"], cache["vp"], cache["k"], cache["v"], lens)
    a, sa, _ = cf.rmsnorm_quant(o.transpose(1, 2).reshape(B, H * d), norm=False)
    y = cf.gemm_i8(a, w["o"], sa, w["s_o"])
    a, sa, r = cf.rmsnorm_quant(y, r, w["g2"])
    hid = cf.gemm_i8(a, w["up"], sa, w["s_up"], act="gelu")
    a, sa, _ = cf.rmsnorm_quant(hid, norm=False)
    return cf.gemm_i8(a, w["down"], sa, w["s_down"]), r, o


def layer_parts(B, seed=3):
    g = gen(seed)
    H, Hk, d, P, S, F = 8, 2, 64, 200, 40, 1024
    D = H * d
    w = {"H": H, "Hk": Hk, "d": d, "g1": torch.rand((D,), generator=g, device="cuda") + 0.5,
         "g2": torch.rand((D,), generator=g, device="cuda") + 0.5,
         "b_qkv": torch.randn(((H + 2 * Hk) * d,), generator=g, device="cuda") * 0.1}
    for name, n, k in (("qkv", (H + 2 * Hk) * d, D), ("o", D, D), ("up", F, D), ("down", D, F)):
        W = torch.randn((n, k), generator=g, device="cuda") * k ** -0.5
        w[name], w["s_" + name], _ = cf.rmsnorm_quant(W, norm=False)     # a weight's rows are its channels
    _, kp, vp, ks, vs = prefix_inputs(g, B, H, Hk, 1, P, S, d)
    lens = torch.randint(1, S + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randn((B, D), generator=g, device="cuda").to(BF16)
    r = torch.randn((B, D), generator=g, device="cuda").to(BF16)
    return x, r, w, {"kp": kp, "vp": vp, "k": ks, "v": vs}, lens


@gpu
@pytest.mark.parametrize("B", [1, 13, 70])
def test_layer_run(B):
    """The run against the same layer in 64 bits without any rounding: every 8-bit product is off by
    the codes' half steps, which random signs leave at about a percent of the result."""
    x, r, w, cache, lens = layer_parts(B)
    y, r2, o = serving_layer(x, r, w, cache, lens)

    def lin(a, name):
        return a @ (w[name].to(F64) * w["s_" + name].to(F64)[:, None]).t()

    def norm(h, gamma):
        return h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-5) * gamma.to(F64)

    h = x.to(F64) + r.to(F64)
    q = (lin(norm(h, w["g1"]), "qkv") + w["b_qkv"].to(F64))[:, :512].view(B, 1, 8, 64).transpose(1, 2)
    ref_o, _ = attend64(q, cache["kp"], cache["vp"], cache["k"], cache["v"], lens, False, 64 ** -0.5)
    h = h + lin(ref_o.transpose(1, 2).reshape(B, 512), "o")
    ref = lin(act64(lin(norm(h, w["g2"]), "up"), "gelu"), "down")

    def off(got, want):
        return float((got.to(F64) - want).norm() / want.norm())

    # One quantisation: errors up to s / 2, rms s / sqrt(12) with s = max / 127 and max about 3.5 rms: 0.8 % of
    # the operand.  bf16 roundings (2^-8 at most, 0.1 % rms) come on top.  o: one product in q, whose
    # error moves softmax weights (|score| about 1): 1 %, doubled.  r2: in the sum with r it is less.
    # y: the norm, up and down products: sqrt(3) * 0.8 % with o's own, doubled.
    assert off(o, ref_o) < 0.02 and off(r2, h) < 0.01 and off(y, ref) < 0.04


@gpu
def test_layer_captured_and_replayed():
    x, r, w, cache, lens = layer_parts(12)
    want = [t.clone() for t in serving_layer(x, r, w, cache, lens)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        serving_layer(x, r, w, cache, lens)
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(graph):
        got = serving_layer(x, r, w, cache, lens)
    for turn in range(4):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
        x2 = torch.randn_like(x)                     # eager work between the replays
        serving_layer(x2, r, w, {**cache, "k": cache["k"].clone(), "v": cache["v"].clone()}, lens)
        torch.cuda.synchronize()


@gpu
def test_repeatable_and_on_another_stream():
    x, r, w, cache, lens = layer_parts(20)
    q = torch.randn((20, 8, 1, 64), device="cuda").to(BF16)
    a = (q, cache["kp"], cache["vp"], cache["k"], cache["v"], lens)
    first = cf.attention_prefix(*a)
    codes = cf.rmsnorm_quant(x, r, w["g1"])
    prod = cf.gemm_i8(codes[0], w["up"], codes[1], w["s_up"])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(3):
        for s in streams:
            got.append((cf.attention_prefix(*a, stream=s), cf.rmsnorm_quant(x, r, w["g1"], stream=s),
                        cf.gemm_i8(codes[0], w["up"], codes[1], w["s_up"], stream=s)))
    torch.cuda.synchronize()
    for o, c, p in got:
        assert torch.equal(o, first) and torch.equal(p, prod) and all(torch.equal(u, v) for u, v in zip(c, codes))


@gpu
def test_empty_batches():
    x = torch.zeros((0, 64), dtype=BF16, device="cuda")
    Q, s, H = cf.rmsnorm_quant(x, x)
    assert Q.shape == (0, 64) and s.shape == (0,) and H.shape == (0, 64)
    assert cf.gemm_i8(Q, torch.zeros((48, 64), dtype=torch.int8, device="cuda"), s).shape == (0, 48)


@gpu
def test_split_calls_captured_and_on_two_streams():
    """Calls in parts use a workspace: each capture has its own, which eager calls of other sizes do not
    disturb, and so has each stream."""
    g = gen(5)
    small = prefix_inputs(g, 4, 8, 2, 1, 3000, 200, 128)
    large = prefix_inputs(g, 16, 16, 4, 2, 6000, 300, 64)
    assert all(cf.cf_attention_prefix_workspace(prefix_args(batch=a[0].shape[0], H=a[0].shape[1], Hk=a[1].shape[0],
                                                            Lq=a[0].shape[2], P=a[1].shape[1], S=a[3].shape[2],
                                                            d=a[0].shape[3])) > 0 for a in (small, large))
    want = [cf.attention_prefix(*a).clone() for a in (small, large)]
    graphs, got = [], []
    for a in (small, large):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(cf.attention_prefix(*a))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(4):
        for t in got:
            t.zero_()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        eager = [cf.attention_prefix(*a, stream=s) for _ in range(3) for a, s in zip((large, small), streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), turn
        assert all(torch.equal(x, want[1 - i % 2]) for i, x in enumerate(eager)), turn


@gpu
def test_threads_share_a_stream():
    """Calls in parts from two threads, on the same stream and so in one workspace."""
    args = [prefix_inputs(gen(s), 6 + 3 * s, 8, 2, 1, 3000 + 500 * s, 200, 64) for s in (1, 2)]
    want = [cf.attention_prefix(*a) for a in args]
    torch.cuda.synchronize()
    bad, stream = [], torch.cuda.Stream()

    def run(i):
        with torch.cuda.stream(stream):
            for _ in range(200):
                if not torch.equal(cf.attention_prefix(*args[i]), want[i]):
                    bad.append(i)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not bad and not any(t.is_alive() for t in threads)


@gpu
def test_one_workspace_for_calls_of_several_sizes():
    """The counters at its start are zero again after every call, whatever its size and cut."""
    g = gen(6)
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    head = ws[:cf.CF_PREFIX_WS_HEADER_BYTES].view(torch.int32)
    head.zero_()
    kinds = set()
    for B, H, Hk, Lq, P, S, d in [(1, 8, 2, 1, 4000, 300, 128), (9, 14, 2, 1, 900, 700, 64), (3, 8, 1, 3, 5000, 40, 64),
                                  (5, 4, 4, 7, 2000, 900, 128), (2, 6, 2, 16, 3000, 64, 64), (40, 8, 8, 1, 3000, 50, 128),
                                  (1, 2, 2, 1, 0, 6000, 128), (2, 4, 1, 50, 9000, 100, 64), (11, 3, 3, 1, 2500, 33, 64)]:
        a = prefix_inputs(g, B, H, Hk, Lq, P, S, d)
        lens = torch.randint(0, S + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        lens[0] = S
        need = cf.cf_attention_prefix_workspace(prefix_args(batch=B, H=H, Hk=Hk, Lq=Lq, P=P, S=S, d=d))
        kinds.add(need > 0)
        for _ in range(2):
            O = cf.attention_prefix(*a, lens, causal=Lq > 1, ws=ws)
            check_attention(O, *a, lens, Lq > 1)
            assert not head.any()
        for _ in range(5):                           # the same bits, whichever workgroup joins
            assert torch.equal(cf.attention_prefix(*a, lens, causal=Lq > 1, ws=ws), O)
        if need:
            with pytest.raises(cf.CfError, match="CF_ERR_WORKSPACE"):
                cf.attention_prefix(*a, lens, ws=ws[:need - 16])
            with pytest.raises(cf.CfError, match="CF_ERR_ALIGN"):
                cf.attention_prefix(*a, lens, ws=ws[8:])
    assert kinds == {True}


@gpu
def test_offsets_past_32_bits():
    """Rows, keys and tokens that lie more than 4 GiB behind their tensor's start."""
    g = gen(11)
    n, wide = 300000, 8192                           # 16 KB a row in bf16, 4.9 GB
    big = torch.zeros((n, wide), dtype=BF16, device="cuda")
    big[-70:] = torch.randn((70, wide), generator=g, device="cuda").to(BF16)
    Q, s, _ = cf.rmsnorm_quant(big)
    check_norm(Q[-70:], s[-70:], None, norm_ref(big[-70:], None, None, 1e-5, True, "int8"), "int8", BF16)
    assert not Q[:-70].any() and not s[:-70].any()
    W = i8(g, 24, wide)
    C = cf.gemm_i8(Q, W, s)
    check_gemm(C[-70:], Q[-70:], W, s[-70:], None, None, "none")
    assert not C[:-70].any()
    del Q, C
    # keys and values: two heads of 128 in the rows; all but the last 70 keys are zero
    d = 128
    K, V = (big[:, i * d:(i + 2) * d].unflatten(-1, (2, d)).transpose(0, 1) for i in (0, 8))
    q = (torch.randn((2, 4, 1, d), generator=g, device="cuda") * 4).to(BF16)
    none = torch.zeros((2, 0, d), dtype=BF16, device="cuda")
    own = [t[None].expand(2, -1, -1, -1) for t in (K, V)]
    for args in ((K, V), (none, none, *own)):
        O = cf.attention_prefix(q, *args)
        x = torch.einsum("bghd,gkd->bghk", q.view(2, 2, 2, d).double(), K[:, -70:].double()) * d ** -0.5
        m = x.amax(-1, keepdim=True).clamp(min=0)
        w = torch.exp(x - m)
        total = w.sum(-1, keepdim=True) + (n - 70) * torch.exp(-m)      # the zero keys score 0
        ref = (torch.einsum("bghk,gkd->bghd", w, V[:, -70:].double()) / total).reshape(2, 4, 1, d)
        size = (torch.einsum("bghk,gkd->bghd", w, V[:, -70:].double().abs()) / total).reshape(2, 4, 1, d)
        # a weight, and the sum of n of them in fp32 (a lane adds up to 2^10 of them before they join): off by
        # 2^-8 and 2^10 u beside the score's error (as in check_attention)
        tol = (2 * 2.0 ** -8 * 1.01 + 2.0 ** 10 * U + 1e-4) * size + 2.0 ** -8 * 1.01 * ref.abs()
        assert bool(((O.double() - ref).abs() <= tol).all())


# ---------------------------------------------------------------- refusals (no GPU)
A_, B_, C_, D_, E_ = (0x7F0000000000 + 0x100000 * i for i in range(5))


def norm_args(**kw):
    d = dict(struct_size=cf.C.sizeof(cf.RmsnormQuantArgs), M=4, N=100, dtype=cf.CF_BF16, X=A_, ldx=104, R=B_, ldr=104,
             H=C_, ldh=104, gamma=None, norm=1, eps=1e-5, code_dtype=cf.CF_I8, Q=D_, ldq=112, s=E_)
    d.update(kw)
    return cf.RmsnormQuantArgs(*[d[f[0]] for f in cf.RmsnormQuantArgs._fields_])


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), "CF_ERR_STRUCT"), (dict(M=-1), "CF_ERR_SHAPE"), (dict(N=0), "CF_ERR_SHAPE"),
    (dict(N=32769, ldx=40000, ldr=40000, ldh=40000, ldq=40000), "CF_ERR_SHAPE"), (dict(X=None), "CF_ERR_NULL"),
    (dict(Q=None), "CF_ERR_NULL"), (dict(s=None), "CF_ERR_NULL"), (dict(ldx=96), "CF_ERR_LD"), (dict(ldq=96), "CF_ERR_LD"),
    (dict(ldx=100), "CF_ERR_ALIGN"), (dict(X=A_ + 2), "CF_ERR_ALIGN"), (dict(ldq=104), "CF_ERR_ALIGN"),
    (dict(s=E_ + 2), "CF_ERR_ALIGN"), (dict(gamma=E_ + 4), "CF_ERR_ALIGN"), (dict(dtype=cf.CF_I8), "CF_ERR_DTYPE"),
    (dict(code_dtype=cf.CF_BF16), "CF_ERR_DTYPE"), (dict(norm=2), "CF_ERR_UNSUPPORTED"), (dict(eps=-1.0), "CF_ERR_SHAPE"),
    (dict(eps=float("nan")), "CF_ERR_SHAPE"), (dict(H=A_), "CF_ERR_ALIAS"), (dict(Q=A_), "CF_ERR_ALIAS"),
    (dict(Q=E_), "CF_ERR_ALIAS"), (dict(H=B_, ldh=112), "CF_ERR_ALIAS")])
def test_norm_refuses(kw, status):
    assert cf.STATUS[cf.cf_rmsnorm_quant(norm_args(**kw), None)] == status, cf.cf_last_error()


def gemm_args(**kw):
    d = dict(struct_size=cf.C.sizeof(cf.GemmI8Args), M=4, N=100, K=64, A=A_, lda=64, B=B_, ldb=64, sa=None, sb=None,
             bias=None, act=0, out_dtype=cf.CF_BF16, C=C_, ldc=104)
    d.update(kw)
    return cf.GemmI8Args(*[d[f[0]] for f in cf.GemmI8Args._fields_])


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), "CF_ERR_STRUCT"), (dict(M=-1), "CF_ERR_SHAPE"), (dict(N=0), "CF_ERR_SHAPE"),
    (dict(M=(1 << 30) + 1), "CF_ERR_SHAPE"), (dict(M=1 << 30, N=129, ldc=136), "CF_ERR_SHAPE"),
    (dict(K=0), "CF_ERR_SHAPE"), (dict(K=40), "CF_ERR_SHAPE"), (dict(K=131072, lda=131072, ldb=131072), "CF_ERR_SHAPE"),
    (dict(A=None), "CF_ERR_NULL"), (dict(B=None), "CF_ERR_NULL"), (dict(C=None), "CF_ERR_NULL"), (dict(lda=48), "CF_ERR_LD"),
    (dict(ldc=96), "CF_ERR_LD"), (dict(lda=72), "CF_ERR_ALIGN"), (dict(ldc=100), "CF_ERR_ALIGN"),
    (dict(B=B_ + 8), "CF_ERR_ALIGN"), (dict(sb=D_ + 4), "CF_ERR_ALIGN"), (dict(sa=D_ + 2), "CF_ERR_ALIGN"),
    (dict(out_dtype=cf.CF_I8), "CF_ERR_DTYPE"), (dict(act=4), "CF_ERR_UNSUPPORTED"), (dict(C=A_), "CF_ERR_ALIAS"),
    (dict(C=D_, sb=D_), "CF_ERR_ALIAS")])
def test_gemm_i8_refuses(kw, status):
    assert cf.STATUS[cf.cf_gemm_i8(gemm_args(**kw), None)] == status, cf.cf_last_error()


def prefix_args(**kw):
    d = dict(struct_size=cf.C.sizeof(cf.AttentionPrefixArgs), batch=2, H=4, Hk=2, Lq=1, P=32, S=16, d=64, dtype=cf.CF_BF16,
             Q=A_, q_b=256, q_h=64, q_l=64, Kp=B_, kp_h=2048, kp_l=64, Vp=B_, vp_h=2048, vp_l=64, Ks=C_, ks_b=2048,
             ks_h=1024, ks_l=64, Vs=C_, vs_b=2048, vs_h=1024, vs_l=64, lens=None, causal=0, scale=0.125, O=D_, o_b=256,
             o_h=64, o_l=64)
    d.update(kw)
    return cf.AttentionPrefixArgs(*[d[f[0]] for f in cf.AttentionPrefixArgs._fields_])


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), "CF_ERR_STRUCT"), (dict(batch=-1), "CF_ERR_SHAPE"), (dict(H=5), "CF_ERR_SHAPE"),
    (dict(Hk=0), "CF_ERR_SHAPE"), (dict(P=-1), "CF_ERR_SHAPE"), (dict(batch=65535), "CF_ERR_SHAPE"),
    (dict(Lq=1 << 24, H=128), "CF_ERR_SHAPE"), (dict(d=96), "CF_ERR_UNSUPPORTED"), (dict(causal=2), "CF_ERR_UNSUPPORTED"),
    (dict(dtype=cf.CF_F32), "CF_ERR_DTYPE"), (dict(scale=0.0), "CF_ERR_SHAPE"), (dict(scale=math.inf), "CF_ERR_SHAPE"),
    (dict(Q=None), "CF_ERR_NULL"), (dict(O=None), "CF_ERR_NULL"), (dict(Kp=None), "CF_ERR_NULL"),
    (dict(Vs=None), "CF_ERR_NULL"), (dict(Ks=C_ + 8), "CF_ERR_ALIGN"), (dict(kp_l=60), "CF_ERR_LD"),
    (dict(ks_l=68), "CF_ERR_ALIGN"), (dict(vs_h=1004), "CF_ERR_ALIGN"), (dict(q_b=-256), "CF_ERR_ALIGN"),
    (dict(vp_l=1 << 22), "CF_ERR_LD"), (dict(lens=E_ + 2), "CF_ERR_ALIGN"), (dict(O=A_), "CF_ERR_ALIAS"),
    (dict(O=C_), "CF_ERR_ALIAS"), (dict(o_b=0), "CF_ERR_LD"), (dict(o_h=0), "CF_ERR_LD"),
    (dict(o_b=64), "CF_ERR_LD"), (dict(o_b=192), "CF_ERR_LD"), (dict(Lq=3, o_l=64), "CF_ERR_LD"),
    (dict(Lq=3, o_l=256, o_b=512), "CF_ERR_LD")])
def test_prefix_refuses(kw, status):
    assert cf.STATUS[cf.cf_attention_prefix(prefix_args(**kw), None, 0, None)] == status, cf.cf_last_error()


def test_empty_calls_do_nothing():
    assert cf.cf_rmsnorm_quant(norm_args(M=0, X=None, R=None, H=None, Q=None, s=None), None) == 0
    assert cf.cf_gemm_i8(gemm_args(M=0, A=None, B=None, C=None), None) == 0
    for kw in (dict(batch=0), dict(Lq=0)):
        assert cf.cf_attention_prefix(prefix_args(Q=None, O=None, **kw), None, 0, None) == 0
        assert cf.cf_attention_prefix_workspace(prefix_args(**kw)) == 0


def test_packed_arguments():
    """The helpers pack their arguments as the structures lay them out."""
    for t, pack in ((cf.RmsnormQuantArgs, cf._RMSNORM_QUANT), (cf.GemmI8Args, cf._GEMM_I8), (cf.AttentionPrefixArgs, cf._PREFIX)):
        values = [i + 0.5 if f is cf.C.c_float else 3 * i + 1 for i, (_, f) in enumerate(t._fields_)]
        assert bytes(t(*values)) == pack.pack(*values)


def test_helpers_refuse_host_tensors():
    x = torch.zeros((4, 16), dtype=BF16)
    with pytest.raises(ValueError, match="GPU"):
        cf.rmsnorm_quant(x)
    with pytest.raises(ValueError, match="GPU"):
        cf.gemm_i8(x.to(torch.int8), x.to(torch.int8))
    with pytest.raises(ValueError, match="GPU"):
        cf.attention_prefix(x.view(1, 1, 1, 64), x.view(1, 1, 64), x.view(1, 1, 64))


@gpu
def test_helpers_refuse():
    x = torch.zeros((4, 64), dtype=BF16, device="cuda")
    q = torch.zeros((4, 64), dtype=torch.int8, device="cuda")
    v = torch.zeros((4,), device="cuda")
    for call in (lambda: cf.rmsnorm_quant(x, x[:2]), lambda: cf.rmsnorm_quant(x, x.float()),
                 lambda: cf.rmsnorm_quant(x, None, v), lambda: cf.rmsnorm_quant(x, out=q[:3]),
                 lambda: cf.rmsnorm_quant(x, None, torch.zeros((64,))), lambda: cf.gemm_i8(q, q[:, :32]),
                 lambda: cf.gemm_i8(q, q, sa=v[:3]), lambda: cf.gemm_i8(q, q, bias=v.double()),
                 lambda: cf.gemm_i8(q, q, out=x), lambda: cf.rmsnorm_quant(x.t())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: cf.rmsnorm_quant(x, code="int4"), lambda: cf.gemm_i8(q, q, act="silu"),
                 lambda: cf.gemm_i8(q, q[:, :0])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        cf.gemm_i8(x, x)
    with pytest.raises(cf.CfError, match="CF_ERR_ALIAS"):
        cf.rmsnorm_quant(x, x.clone(), residual=x)
    with pytest.raises(cf.CfError, match="CF_ERR_ALIGN"):
        cf.rmsnorm_quant(torch.zeros((4, 30), dtype=BF16, device="cuda"))
    with pytest.raises(cf.CfError, match="CF_ERR_SHAPE"):
        cf.gemm_i8(q[:, :40].contiguous(), q[:, :40].contiguous())
    a = torch.zeros((2, 4, 1, 64), dtype=BF16, device="cuda")
    k = torch.zeros((2, 8, 64), dtype=BF16, device="cuda")
    for kw in (dict(Ks=a), dict(Ks=a, Vs=a), dict(lens=torch.zeros((2,), device="cuda")), dict(out=k),
               dict(ws=torch.zeros((1 << 18,), device="cuda")), dict(ws=torch.zeros((1 << 20,), dtype=torch.uint8))):
        with pytest.raises(ValueError):
            cf.attention_prefix(a, k, k, **kw)
