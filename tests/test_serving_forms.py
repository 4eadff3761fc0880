"""The serving operators' helpers and kernel forms beyond test_serving_ops.py: every form of the int8 product
and of the attention over a shared prefix, each named by the library's own query, so that a change of the
estimates that choose them cannot move a test away from its form."""
import math
import types

import pytest
import torch

from paper_2608_03537_amd import comfuse as cf
from test_serving_ops import (BF16, F32, F64, HALF, QMAX, U, check_attention, check_gemm, gemm_args, gen, gpu, i8,
                              norm_ref, padded, prefix_args, prefix_inputs)


# ---------------------------------------------------------------- rmsnorm_quant: special rows with the norm
@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("N", [24, 400, 1500, 4000, 7000, 20000, 32768])
def test_normed_special_rows(N, code, dtype):
    """All-zero, NaN, infinite and tiny rows, rows that gamma clears, and large ones on either side of where the
    sum of squares and their mean pass fp32's largest value."""
    g = gen(N)
    X, R = padded(12, N, dtype, g), padded(12, N, dtype, g, 0.25)
    gamma = torch.rand((N,), generator=g, device="cuda") + 0.5
    gamma[:4] = 0.0
    X[1], R[1] = 0.0, 0.0
    X[2, N // 2] = float("nan")
    R[3, N - 1] = -math.inf
    X[4] *= 1e-25
    R[4] *= 1e-25
    X[5, 4:], R[5, 4:] = 0.0, 0.0
    for row, size in ((6, (0.1 * 3.4e38 / N) ** 0.5), (7, (4 * 3.4e38 / N) ** 0.5), (8, 1e19), (9, 4e19), (10, 1e30),
                      (11, 1e37)):
        X[row] = (X[row].float().clamp(-4, 4) * size).to(dtype)
        R[row] = (R[row].float() * size).to(dtype)
    Q, s, H = cf.rmsnorm_quant(X, R, gamma, eps=1e-5, code=code)
    z, sr, h = norm_ref(X, R, gamma, 1e-5, True, code)
    q = Q.to(F64) if code == "int8" else Q.contiguous().view(torch.float8_e4m3fn).to(F64)
    assert not q[[1, 2, 3, 5]].any() and not s[[1, 5]].any() and s[2].isnan() and s[3].isnan()
    rows = [0, 4, 6, 7, 8, 9, 10, 11]
    half = 0.5 if code == "int8" else torch.clamp(z[rows].abs() * 2.0 ** -4, min=2.0 ** -10)
    assert bool(((q[rows] - z[rows]).abs() <= half + 4.1 * U * QMAX[code]).all())
    # s: h, t, d; half of h, of its square and of a sum of at most 64 terms a lane and 10 levels, of the mean and of
    # eps' addition; the root, its reciprocal, two products.  Below 2^-126 a product is off by half of 2^-149
    bad = ~((s.to(F64)[rows] - sr[rows]).abs() <= (7 + (1 + 74 + 3) / 2) * U * sr[rows] + 2.0 ** -149)
    assert not bool(bad.any()), (bad.nonzero().tolist(), s[rows].tolist(), sr[rows].tolist())
    assert bool(((H[rows].to(F64) - h[rows]).abs() <= (HALF[dtype] + U) * h[rows].abs()).all())


@gpu
@pytest.mark.parametrize("N", [64, 3000])
def test_normed_large_rows_in_place(N):
    """The same where the residual stream is updated in place, bit for bit."""
    g = gen(N)
    X, R = padded(9, N, BF16, g), padded(9, N, BF16, g)
    X[3:6] = (X[3:6].float() * 1e30).to(BF16)
    R[4:7] = (R[4:7].float() * 1e25).to(BF16)
    want = cf.rmsnorm_quant(X, R)
    got = cf.rmsnorm_quant(X, R, residual=R)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool((want[1] > 0).all())


# ---------------------------------------------------------------- widths that are no whole 16 bytes
@gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("N", [1, 30, 333])
def test_outputs_of_odd_widths(N, dt):
    """New outputs have padded rows, which the helpers take as they are; contiguous ones are refused."""
    g = gen(N)
    A, B = i8(g, 5, 64), i8(g, N, 64)
    C = cf.gemm_i8(A, B, out_dtype=dt)
    want = (A.to(F64) @ B.to(F64).t()).to(dt)
    assert torch.equal(C, want) and C.stride(0) * C.element_size() % 16 == 0 and not C.is_contiguous()
    assert torch.equal(C.contiguous().view(-1), want.view(-1))
    Q, s, H = cf.rmsnorm_quant(C, C)
    z, sr, h = norm_ref(C, C, None, 1e-5, True, "int8")
    assert bool(((Q.to(F64) - z).abs() <= 0.5 + 4.1 * U * 127).all())
    assert bool(((s.to(F64) - sr).abs() <= (5 + (3 + 74) / 2) * U * sr).all()) and torch.equal(H, (2 * want.to(F32)).to(dt))
    for call in (lambda: cf.rmsnorm_quant(want), lambda: cf.gemm_i8(A, B, out=want),
                 lambda: cf.rmsnorm_quant(C, out=torch.empty((5, N), dtype=torch.int8, device="cuda"))):
        with pytest.raises(cf.CfError, match="CF_ERR_ALIGN"):
            call()


# ---------------------------------------------------------------- gemm_i8: every tile, K whole and cut
GEMM_FORMS = [
    (100, 300, 640, "32 x 32 tiles of 256 threads, whole K"), (100, 131, 1008, "32 x 32 tiles of 256 threads, cut K"),
    (513, 770, 512, "32 x 64 tiles of 384 threads, whole K"), (300, 1029, 1136, "32 x 64 tiles of 384 threads, cut K"),
    (13079, 15, 3584, "64 x 32 tiles of 256 threads, whole K"), (13079, 16, 3664, "64 x 32 tiles of 256 threads, cut K"),
    (60, 9001, 768, "64 x 64 tiles of 256 threads, whole K"), (60, 9006, 720, "64 x 64 tiles of 256 threads, cut K"),
    (130, 8999, 768, "64 x 128 tiles of 512 threads, whole K"), (500, 3900, 400, "64 x 128 tiles of 512 threads, cut K"),
    (1000, 3997, 256, "128 x 128 tiles of 512 threads, whole K"),
    (1000, 4003, 272, "128 x 128 tiles of 512 threads, cut K"),
    (2500, 8098, 128, "128 x 128 tiles of 256 threads, whole K"),
    (2500, 8097, 48, "128 x 128 tiles of 256 threads, cut K"),
    (4000, 4081, 1920, "256 x 256 tiles of 512 threads, whole K"), (4000, 4078, 1984, "256 x 256 tiles of 512 threads, cut K")]


def gemm_form(M, N, K):
    return cf.cf_gemm_i8_form(gemm_args(M=M, N=N, K=K, lda=K, ldb=K, ldc=-(-N // 8) * 8))


@pytest.mark.parametrize("M,N,K,form", GEMM_FORMS)
def test_gemm_i8_form(M, N, K, form):
    assert gemm_form(M, N, K) == form


def test_gemm_i8_form_of_no_call():
    for kw in (dict(M=0), dict(N=0), dict(K=40), dict(struct_size=8)):
        assert cf.cf_gemm_i8_form(gemm_args(**kw)) == ""


@gpu
@pytest.mark.parametrize("M,N,K,form", GEMM_FORMS)
def test_gemm_i8_sums_of_every_form(M, N, K, form):
    """Without scales the output in fp32 is the exact sum, rounded once."""
    assert gemm_form(M, N, K) == form
    g = gen(M + N + K)
    A, B = i8(g, M, K), i8(g, N, K)
    assert torch.equal(cf.gemm_i8(A, B, out_dtype=F32), (A.to(F64) @ B.to(F64).t()).to(F32))


@gpu
@pytest.mark.parametrize("act,sa,sb,bias,dt", [
    ("none", True, True, True, BF16), ("gelu", True, True, True, F32), ("gelu_tanh", True, True, False, BF16),
    ("relu", False, True, True, F32), ("gelu", True, False, True, BF16), ("none", False, False, True, F32)])
@pytest.mark.parametrize("M,N,K,form", GEMM_FORMS)
def test_gemm_i8_epilogue_of_every_form(M, N, K, form, act, sa, sb, bias, dt):
    """Scales, bias and activation of each form, ragged at both edges; rows and columns behind C stay as they were."""
    assert gemm_form(M, N, K) == form
    g = gen(M + N + K)
    A, B = i8(g, M, K), i8(g, N, K)
    sa = torch.rand((M,), generator=g, device="cuda") * 0.05 if sa else None      # sums of about 5500 sqrt(K)
    sb = torch.rand((N,), generator=g, device="cuda") / (64 * K ** 0.5) if sb else None
    bias = torch.randn((N,), generator=g, device="cuda") if bias else None
    full = torch.full((M + 1, -(-N // 16) * 16 + 16), 7.0, dtype=dt, device="cuda")
    C = cf.gemm_i8(A, B, sa, sb, bias=bias, act=act, out=full[:M, :N])
    check_gemm(C, A, B, sa, sb, bias, act)
    assert bool((full[M:] == 7).all()) and bool((full[:, N:] == 7).all())


# ---------------------------------------------------------------- attention_prefix: every cut
PREFIX_FORMS = [
    (4, 10, 10, 149, 957, 26, 64, "split, 128 + 128 rows, 3 + 1 parts, merged 1 ways"),
    (1, 7, 1, 15, 1010, 128, 64, "split, 128 + 128 rows, 8 + 1 parts, merged 4 ways"),
    (1, 7, 1, 14, 1024, 5, 64, "split, 128 + 128 rows, 16 + 1 parts, merged 8 ways"),
    (2, 9, 9, 106, 327, 337, 64, "split, 128 + 128 rows, 2 + 2 parts, merged 1 ways"),
    (1, 7, 1, 17, 36, 456, 64, "split, 128 + 128 rows, 1 + 4 parts, merged 4 ways"),
    (1, 14, 2, 14, 1484, 577, 64, "split, 128 + 128 rows, 16 + 8 parts, merged 8 ways"),
    (47, 11, 11, 1, 2, 3, 64, "split, 128 + 32 rows, 1 + 1 parts, merged 1 ways"),
    (46, 16, 8, 1, 1010, 27, 64, "split, 128 + 32 rows, 8 + 1 parts, merged 4 ways"),
    (19, 14, 7, 1, 2093, 210, 64, "split, 128 + 32 rows, 17 + 1 parts, merged 8 ways"),
    (55, 5, 5, 1, 590, 1836, 64, "split, 128 + 32 rows, 1 + 2 parts, merged 1 ways"),
    (3, 20, 10, 9, 3, 1480, 64, "split, 128 + 32 rows, 1 + 8 parts, merged 4 ways"),
    (34, 2, 2, 15, 5144, 1866, 64, "split, 128 + 32 rows, 15 + 2 parts, merged 8 ways"),
    (46, 12, 12, 1, 302, 2, 64, "split, 32 + 32 rows, 1 + 1 parts, merged 1 ways"),
    (1, 4, 1, 5, 1451, 143, 64, "split, 32 + 32 rows, 8 + 1 parts, merged 4 ways"),
    (1, 1, 1, 23, 2165, 5, 64, "split, 32 + 32 rows, 16 + 1 parts, merged 8 ways"),
    (54, 2, 2, 1, 720, 1486, 64, "split, 32 + 32 rows, 1 + 2 parts, merged 1 ways"),
    (1, 1, 1, 17, 8, 2047, 64, "split, 32 + 32 rows, 1 + 8 parts, merged 4 ways"),
    (1, 7, 1, 3, 2930, 1017, 64, "split, 32 + 32 rows, 16 + 4 parts, merged 8 ways"),
    (1, 8, 1, 14, 1, 1, 64, "whole, 128 rows, 1 parts"),
    (7, 8, 2, 31, 78, 529, 64, "whole, 128 rows, 4 parts, merged 1 ways"),
    (1, 1, 1, 102, 2, 526, 64, "whole, 128 rows, 8 parts, merged 4 ways"),
    (1, 2, 1, 49, 2847, 1, 64, "whole, 128 rows, 32 parts, merged 8 ways"),
    (1, 1, 1, 1, 1, 1, 64, "whole, 32 rows, 1 parts"),
    (1, 1, 1, 9, 6, 1255, 64, "whole, 32 rows, 8 parts, joined by 32"),
    (1, 1, 1, 1, 515, 461, 64, "whole, 32 rows, 8 parts, joined by 8"),
    (4, 5, 5, 34, 1, 1865, 64, "whole, 32 rows, 4 parts, merged 1 ways"),
    (1, 7, 1, 5, 1527, 73, 64, "whole, 32 rows, 8 parts, merged 4 ways"),
    (1, 7, 1, 6, 5574, 57, 64, "whole, 32 rows, 32 parts, merged 8 ways"),
    (1, 1, 1, 141, 216, 87, 128, "split, 128 + 128 rows, 2 + 1 parts, merged 1 ways"),
    (1, 8, 1, 18, 467, 15, 128, "split, 128 + 128 rows, 4 + 1 parts, merged 4 ways"),
    (1, 16, 2, 14, 1998, 66, 128, "split, 128 + 128 rows, 16 + 1 parts, merged 8 ways"),
    (2, 4, 1, 25, 97, 205, 128, "split, 128 + 128 rows, 1 + 2 parts, merged 1 ways"),
    (1, 7, 1, 14, 231, 338, 128, "split, 128 + 128 rows, 2 + 4 parts, merged 4 ways"),
    (2, 8, 1, 19, 1997, 173, 128, "split, 128 + 128 rows, 16 + 2 parts, merged 8 ways"),
    (37, 28, 14, 1, 1, 1, 128, "split, 128 + 32 rows, 1 + 1 parts, merged 1 ways"),
    (36, 30, 15, 1, 429, 3, 128, "split, 128 + 32 rows, 4 + 1 parts, merged 4 ways"),
    (57, 14, 7, 1, 2039, 32, 128, "split, 128 + 32 rows, 16 + 1 parts, merged 8 ways"),
    (55, 5, 5, 1, 447, 1034, 128, "split, 128 + 32 rows, 1 + 2 parts, merged 1 ways"),
    (3, 10, 10, 14, 8, 1010, 128, "split, 128 + 32 rows, 1 + 8 parts, merged 4 ways"),
    (55, 4, 2, 1, 1863, 441, 128, "split, 128 + 32 rows, 16 + 2 parts, merged 8 ways"),
    (52, 10, 10, 1, 142, 13, 128, "split, 32 + 32 rows, 1 + 1 parts, merged 1 ways"),
    (1, 7, 1, 3, 806, 19, 128, "split, 32 + 32 rows, 8 + 1 parts, merged 4 ways"),
    (1, 2, 1, 12, 1204, 4, 128, "split, 32 + 32 rows, 16 + 1 parts, merged 8 ways"),
    (33, 3, 3, 1, 453, 852, 128, "split, 32 + 32 rows, 1 + 2 parts, merged 1 ways"),
    (1, 1, 1, 17, 3, 802, 128, "split, 32 + 32 rows, 1 + 8 parts, merged 4 ways"),
    (1, 2, 1, 9, 1119, 504, 128, "split, 32 + 32 rows, 16 + 4 parts, merged 8 ways"),
    (1, 7, 1, 22, 2, 2, 128, "whole, 128 rows, 1 parts"),
    (2, 7, 1, 15, 269, 2, 128, "whole, 128 rows, 4 parts, merged 1 ways"),
    (1, 7, 1, 17, 319, 284, 128, "whole, 128 rows, 8 parts, merged 4 ways"),
    (1, 8, 1, 15, 2141, 1, 128, "whole, 128 rows, 32 parts, merged 8 ways"),
    (1, 1, 1, 1, 3, 1, 128, "whole, 32 rows, 1 parts"),
    (1, 2, 1, 5, 747, 2, 128, "whole, 32 rows, 8 parts, joined by 32"),
    (1, 1, 1, 1, 519, 2, 128, "whole, 32 rows, 8 parts, joined by 8"),
    (11, 2, 2, 36, 817, 156, 128, "whole, 32 rows, 4 parts, merged 1 ways"),
    (1, 7, 1, 5, 3, 823, 128, "whole, 32 rows, 8 parts, merged 4 ways"),
    (1, 7, 1, 5, 2432, 115, 128, "whole, 32 rows, 32 parts, merged 8 ways"),
    (4, 8, 8, 16, 1500, 60, 64, "whole, 32 rows, 8 parts, joined by 32"),
    (2, 8, 8, 27, 2500, 0, 128, "whole, 32 rows, 16 parts, joined by 32"),
    (8, 16, 4, 20, 500, 1500, 128, "split, 128 + 32 rows, 2 + 2 parts, merged 1 ways"),
    (1, 8, 1, 3, 500, 300, 128, "split, 32 + 32 rows, 4 + 4 parts, merged 4 ways"),
]


def prefix_form(B, H, Hk, Lq, P, S, d):
    return cf.cf_attention_prefix_form(prefix_args(batch=B, H=H, Hk=Hk, Lq=Lq, P=P, S=S, d=d))


@pytest.mark.parametrize("B,H,Hk,Lq,P,S,d,form", PREFIX_FORMS)
def test_prefix_form(B, H, Hk, Lq, P, S, d, form):
    assert prefix_form(B, H, Hk, Lq, P, S, d) == form


def test_prefix_form_of_no_call():
    for kw in (dict(batch=0), dict(Lq=0), dict(d=96), dict(struct_size=8)):
        assert cf.cf_attention_prefix_form(prefix_args(**kw)) == ""


@gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,H,Hk,Lq,P,S,d,form", PREFIX_FORMS)
def test_prefix_results_of_every_form(B, H, Hk, Lq, P, S, d, form, causal):
    """Ragged lengths, one of them 0 and one S, in a workspace whose partial results start as NaN; the same bits
    again, and counters of zero afterwards."""
    assert prefix_form(B, H, Hk, Lq, P, S, d) == form
    g = gen(B + H + Lq + P + S + d)
    a = prefix_inputs(g, B, H, Hk, Lq, P, S, d)
    lens = torch.randint(0, S + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    lens[B // 2], lens[0] = 0, S
    need = cf.cf_attention_prefix_workspace(prefix_args(batch=B, H=H, Hk=Hk, Lq=Lq, P=P, S=S, d=d))
    assert (need > 0) == (", 1 parts" not in form)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    head = ws[:cf.CF_PREFIX_WS_HEADER_BYTES].zero_()
    O = cf.attention_prefix(*a, lens, causal=causal, ws=ws)
    check_attention(O, *a, lens, causal)
    for _ in range(2):
        assert torch.equal(cf.attention_prefix(*a, lens, causal=causal, ws=ws), O) and not head.any()


# ---------------------------------------------------------------- attention_prefix's workspace
def test_workspace_grows_rarely_and_clears_its_counters_only(monkeypatch):
    """A batch that grows step by step finds room in what an earlier step allocated; of a new workspace
    only the arrival counters are cleared."""
    made = []

    def empty(n, dtype, device):
        made.append(torch.full((n,), 255, dtype=dtype, device=device))
        return made[-1]

    def zeros(n, dtype, device):
        made.append(torch.zeros((n,), dtype=dtype, device=device))
        return made[-1]

    monkeypatch.setattr(cf, "_ws_cache", {})
    host = types.SimpleNamespace(_C=types.SimpleNamespace(_cuda_isCurrentStreamCapturing=lambda: False), empty=empty,
                                 zeros=zeros, uint8=torch.uint8, int32=torch.int32)
    head = cf.CF_PREFIX_WS_HEADER_BYTES
    for need in range(head + 4096, 1 << 23, 1 << 15):
        ws = cf._prefix_workspace(host, need, "cpu", (0, 0, "prefix"))
        assert ws.numel() >= need
    # each one half as large again as the last: from 256 KiB to 8 MiB at most 9
    assert len(made) <= 9
    for t in made:
        assert not t[:head].any() and bool((t[head:] == 255).all())
