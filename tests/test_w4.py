"""4-bit weights: their codes and tiles, and the product with group scales, against
the definitions in 64 bits.  u is fp32's half step; each bound counts roundings."""
import math

import pytest
import torch

from paper_2608_03537_amd import comfuse as cf
from tests.test_serving_ops import BF16, F32, F64, HALF, U, act64, gen, padded

gpu = pytest.mark.gpu
VALUES = {"int4": [float(i) for i in range(8)] + [float(i - 16) for i in range(8, 16)],
          "e2m1": [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]}


def codes_of(tiles, N, K):
    """The codes [N, K] of a weight's tiles, and what the tiles hold behind them."""
    nb, kb, _ = tiles.shape
    w = tiles.view(nb, kb, 2, 32, 4, 4).permute(0, 3, 1, 4, 2, 5).reshape(nb * 32, kb * 32)
    c = torch.stack([w & 15, w >> 4], -1).reshape(nb * 32, kb * 64).long()
    return c[:N, :K], torch.cat([c[N:].flatten(), c[:, K:].flatten()])


def rand_codes(g, N, K):
    return torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)


def weights64(tiles, s, N, K, code):
    c, behind = codes_of(tiles, N, K)
    assert not behind.any()
    w = torch.tensor(VALUES[code], dtype=F64, device=tiles.device)[c]
    return w * s.to(F64).t().repeat_interleave(K // s.shape[0], dim=1)


def check_w4(C, A, tiles, s, code, bias=None, act="none"):
    M, K = A.shape
    N = s.shape[1]
    w, a = weights64(tiles, s, N, K, code), A.to(F64)
    y, size = a @ w.t(), a.abs() @ w.abs().t()
    if bias is not None:
        y, size = y + bias.to(F64), size + bias.to(F64).abs()
    ref = act64(y, act)
    # every product is exact; a sum of K of them, the scales' products and the bias: K + K / group + 2 roundings.  The
    # activations grow by at most 1.13 times what their argument is off, and add 5e-7 |x| / 2 and 4 roundings of their own.
    tol = 1.13 * (K + s.shape[0] + 2) * U * size
    if act != "none" and act != "relu":
        tol = tol + (5e-7 / 2 + 4 * U) * y.abs()
    tol = tol + HALF[C.dtype] * (ref.abs() + tol)
    bad = ~((C.to(F64) - ref).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), C[bad][:4].tolist(), ref[bad][:4].tolist())


def make(g, M, N, K, group, code, sdt, bias=False):
    A = (torch.randn((M, K), generator=g, device="cuda") * torch.where(torch.arange(K, device="cuda") % 37 == 5, 9.0, 1.0)).to(BF16)
    tiles = cf.w4_pack(rand_codes(g, N, K))
    s = ((torch.rand((K // group, N), generator=g, device="cuda") + 0.2) / K ** 0.5).to(sdt)
    return A, tiles, s, torch.randn((N,), generator=g, device="cuda") if bias else None


# ---------------------------------------------------------------- codes and tiles
@gpu
@pytest.mark.parametrize("N,K", [(1, 32), (31, 64), (33, 96), (64, 128), (100, 1056), (2003, 32)])
def test_pack(N, K):
    g = gen(N + K)
    wide = torch.randint(0, 256, (N, K // 2 + 3), generator=g, device="cuda", dtype=torch.uint8)
    for codes in (wide[:, :K // 2].contiguous(), wide[:, 1:1 + K // 2]):
        tiles = cf.w4_pack(codes)
        assert tiles.numel() == -(-N // 32) * -(-K // 64) * 1024
        c, behind = codes_of(tiles, N, K)
        assert torch.equal(c, torch.stack([codes & 15, codes >> 4], -1).reshape(N, K).long()) and not behind.any()


@gpu
@pytest.mark.parametrize("code,top", [("int4", 7.0), ("e2m1", 6.0)])
@pytest.mark.parametrize("dtype,sdt", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("N,K,group", [(1, 32, 32), (37, 96, 96), (64, 256, 128), (130, 1056, 32), (5, 640, 64), (33, 1056, 1056), (40, 2048, 1024),
                                       (7, 4128, 1376), (3, 1152, 576)])
def test_quant(N, K, group, dtype, sdt, code, top):
    g = gen(N * K)
    W = padded(N, K, dtype, g, pad=16)
    W[0, :group] = 0.0
    if N > 4:
        W[1, 3], W[2, group - 1], W[3] = float("nan"), -math.inf, W[3] * 1e-30
    tiles, s = cf.w4_quant(W, group, code=code, scales=sdt)
    x = W.float().cpu().reshape(N, K // group, group)
    m = x.abs().amax(-1)
    want = (m / torch.full_like(m, top)).to(sdt)
    bad = ~torch.isfinite(m)
    assert s.dtype is sdt and torch.equal(s.cpu().t()[~bad], want[~bad]) and bool(s.cpu().t()[bad].float().isnan().all())
    c, behind = codes_of(tiles.cpu(), N, K)
    assert not behind.any()
    got = torch.tensor(VALUES[code])[c].reshape(x.shape)
    d = want.float()[..., None]
    z = torch.where(d > 0, x / d, torch.zeros_like(x)).clamp(-top, top)
    assert not got[bad].any() and not got[(m == 0)].any()
    table = torch.tensor(sorted(set(VALUES[code])))
    if code == "int4":
        table = table[1:]                              # -8 is no quantised value
    near = (z[..., None] - table).abs()
    assert torch.equal((z - got).abs()[~bad], near.amin(-1)[~bad])   # the nearest value of the fp32 quotient
    tie = (near == near.amin(-1, keepdim=True)).sum(-1) > 1
    if code == "int4":
        assert bool((got[tie & ~bad[..., None]] % 2 == 0).all())
    else:
        even = torch.tensor([v for i, v in enumerate(VALUES["e2m1"]) if i % 2 == 0])
        assert bool(torch.isin(got[tie & ~bad[..., None]], even).all())


@gpu
@pytest.mark.parametrize("K,group", [(2112, 32), (2560, 512)])
def test_quant_more_groups_than_a_grid(K, group):
    """Workgroups take several groups: channels of the start, the middle and the end are those of small calls."""
    N = 1 << 20
    W = torch.empty((N, K), dtype=BF16, device="cuda").normal_(generator=gen(K))
    tiles, s = cf.w4_quant(W, group)
    for at in (0, N // 2, N - 64):
        t, u = cf.w4_quant(W[at:at + 64], group)
        assert torch.equal(tiles[at // 32:at // 32 + 2], t) and torch.equal(s[:, at:at + 64], u)


# ---------------------------------------------------------------- the product
@gpu
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 32), (1, 33, 64), (2, 100, 96), (5, 31, 160), (8, 256, 512), (9, 64, 1056), (16, 300, 2048), (31, 32, 64), (32, 1000, 992),
    (33, 65, 128), (64, 640, 4096), (65, 128, 64), (100, 200, 1056), (130, 515, 224), (300, 96, 768), (517, 1030, 544), (1, 4096, 4096),
    (3, 2003, 8192), (700, 40, 32), (1100, 2100, 512)])
@pytest.mark.parametrize("code,sdt,out", [("int4", F32, F32), ("e2m1", BF16, F32), ("int4", BF16, BF16)])
def test_w4_sizes(M, N, K, code, sdt, out):
    g = gen(M * 31 + N * 7 + K)
    for group in sorted({32, K, next(x for x in (128, 64, 96, 32) if K % x == 0)}):
        A, tiles, s, bias = make(g, M, N, K, group, code, sdt, bias=group == 32)
        check_w4(cf.gemm_w4(A, tiles, s, code=code, bias=bias, out_dtype=out), A, tiles, s, code, bias)


@gpu
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("M", [3, 40, 200])
def test_w4_acts(M, act):
    g = gen(M)
    A, tiles, s, bias = make(g, M, 150, 320, 64, "e2m1", BF16, bias=True)
    check_w4(cf.gemm_w4(A, tiles, s, code="e2m1", bias=bias, act=act, out_dtype=F32), A, tiles, s, "e2m1", bias, act)


@gpu
@pytest.mark.parametrize("M", [1, 6, 20, 50, 150, 600])
@pytest.mark.parametrize("K", [96, 256])
def test_w4_strides_and_padding(M, K):
    """What lies behind K, N and M is neither used nor written."""
    g = gen(M + K)
    N = 333
    A, tiles, s, _ = make(g, M, N, K, 32, "int4", F32)
    wide = torch.full((M, K + 40), float("nan"), dtype=BF16, device="cuda")
    wide[:, 8:8 + K] = A
    far = torch.full((s.shape[0], N + 7), float("nan"), device="cuda")
    far[:, 3:3 + N] = s
    for dt in (BF16, F32):
        full = torch.full((M + 1, 352), 7.0, dtype=dt, device="cuda")
        C = cf.gemm_w4(wide[:, 8:8 + K], tiles, far[:, 3:3 + N], out=full[:M, :N])
        check_w4(C, A, tiles, s, "int4")
        assert bool((full[M:] == 7).all()) and bool((full[:, N:] == 7).all())


@gpu
@pytest.mark.parametrize("M", [2, 30, 64, 129, 520])
def test_w4_not_finite(M):
    """A NaN or an infinity in a token reaches its row only, a NaN scale its channel only."""
    g = gen(M)
    A, tiles, s, _ = make(g, M, 70, 160, 32, "int4", F32)
    want = cf.gemm_w4(A, tiles, s)
    B, t = A.clone(), s.clone()
    B[1, 159], t[2, 65] = float("nan"), float("nan")
    if M > 5:
        B[5, 0] = math.inf
    C = cf.gemm_w4(B, tiles, t)
    rows = torch.ones(M, dtype=torch.bool, device="cuda")
    rows[[1, 5] if M > 5 else [1]] = False
    cols = torch.arange(70, device="cuda") != 65
    assert bool(C[1].isnan().all()) and bool(C[:, 65].isnan().all()) and torch.equal(C[rows][:, cols], want[rows][:, cols])
    if M > 5:
        assert not bool(torch.isfinite(C[5]).any())


@gpu
def test_w4_all_codes_exact():
    """Each code alone: token k picks channel code k's value; powers of two as scales, so every output is exact."""
    K, N = 64, 32
    c = (torch.arange(N)[:, None] + torch.arange(K)[None]) % 16
    tiles = cf.w4_pack((c[:, 0::2] | c[:, 1::2] << 4).to(torch.uint8).cuda())
    s = torch.exp2(torch.arange(N) % 7 - 3.0).repeat(2, 1).cuda()
    for code in VALUES:
        C = cf.gemm_w4(torch.eye(K, dtype=BF16, device="cuda"), tiles, s, code=code, out_dtype=F32)
        assert torch.equal(C.cpu(), torch.tensor(VALUES[code])[c].t() * s[0].cpu())


@gpu
@pytest.mark.parametrize("M", [64, 200, 1100])
def test_w4_ends_of_the_range(M):
    """Scales down to 2^-122 and sums of a group up to just below 2^124, exact: one product a group, powers of two."""
    K, N = 256, 64
    c = (torch.arange(N)[:, None] + torch.arange(K)[None]) % 16
    tiles = cf.w4_pack((c[:, 0::2] | c[:, 1::2] << 4).to(torch.uint8).cuda())
    A = torch.zeros((M, K), dtype=BF16, device="cuda")
    at = torch.arange(M, device="cuda")
    for code in VALUES:
        w = torch.tensor(VALUES[code])[c].t().double().cuda()[at % K]
        for a, scale in ((2.0 ** 120, 2.0 ** -122), (2.0 ** 120, 2.0 ** 4), (1.0, 2.0 ** -122), (1.0, 1.375 * 2.0 ** -122), (-(2.0 ** 100), 2.0 ** -100)):
            A.zero_()
            A[at, at % K] = a
            for group in (32, 128):
                C = cf.gemm_w4(A, tiles, torch.full((K // group, N), scale, device="cuda"), code=code, out_dtype=F32)
                assert torch.equal(C.double(), a * w * scale), (code, a, scale, group)


@gpu
def test_w4_of_quantised_weights():
    """w4_quant and gemm_w4 together: near the product with the weights themselves."""
    g = gen(5)
    W, A = padded(300, 512, BF16, g), padded(40, 512, BF16, g)
    for code, step in (("int4", 0.5 / 7), ("e2m1", 1.0 / 6)):       # half the widest step, by the group's maximum
        tiles, s = cf.w4_quant(W, 64, code=code)
        C = cf.gemm_w4(A, tiles, s, code=code, out_dtype=F32)
        ref = A.to(F64) @ W.to(F64).t()
        most = W.to(F64).abs().view(300, 8, 64).amax(-1)            # a weight is off by at most step times this
        size = A.to(F64).abs().view(40, 8, 64).sum(-1) @ most.t()
        assert bool(((C.to(F64) - ref).abs() <= step * 1.001 * size).all())


@gpu
def test_w4_forms_are_all_reached():
    forms = set()
    for M in (1, 20, 64, 200, 5000):
        for N in (64, 4096):
            for group in (32, 64):
                a = w4_args(M=M, N=N, K=4096, group=group, ldc=N, lda=4096, lds=N)
                forms.add(cf.cf_gemm_w4_form(a))
    assert len({f.split(",")[0] for f in forms}) >= 4, forms


@gpu
def test_w4_offsets_pass_32_bits():
    """More than 2^32 bytes of output, and of weights: the last rows and channels are those of a small call."""
    g = gen(1)
    M, N, K = 70001, 33000, 64
    A, tiles, s, _ = make(g, M, N, K, 32, "int4", F32)
    C = cf.gemm_w4(A, tiles, s)
    assert C.numel() * 2 > 2 ** 32
    check_w4(C[-300:], A[-300:], tiles, s, "int4", None)
    del C
    N, K = 1 << 20, 8256
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    tiles = cf.w4_pack(codes)
    assert tiles.numel() > 2 ** 32
    s = torch.rand((1, N), generator=g, device="cuda")
    A = padded(3, K, BF16, g)
    last = cf.w4_pack(codes[-64:].contiguous())
    assert torch.equal(tiles[-2:], last)
    check_w4(cf.gemm_w4(A, tiles, s)[:, -64:], A, last, s[:, -64:], "int4", None)


@gpu
def test_w4_repeatable_on_streams_and_captured():
    """The same bits again, on another stream and from a graph replayed with new tokens between eager calls."""
    g = gen(3)
    for M in (1, 48, 1100):
        A, tiles, s, bias = make(g, M, 2100, 512, 128, "int4", F32, bias=True)
        B, _, _, _ = make(g, M, 2100, 512, 128, "int4", F32)
        call = lambda **kw: cf.gemm_w4(A, tiles, s, bias=bias, act="gelu", **kw)  # noqa: E731
        first = call()
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        on = call(stream=other)
        torch.cuda.synchronize()
        assert torch.equal(first, on)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            C = call()
        for x in (B, A.clone(), B):
            A.copy_(x)
            graph.replay()
            want = call()
            torch.cuda.synchronize()
            assert torch.equal(C, want)


TILES = ["8 x 32", "16 x 64", "32 x 32", "32 x 64", "64 x 32", "64 x 64", "64 x 128", "128 x 128"]
TILE_K = [(64, 64), (96, 32), (128, 128), (320, 64), (480, 96), (640, 128), (960, 192), (1056, 32), (2048, 256), (2080, 32), (2112, 192)]   # k, group


def tile_sizes(tile, K, group, code):
    """Tokens and channels for which the rule takes a tile: fewest, most and between."""
    sizes = [(M, N) for M in (1, 5, 8, 13, 16, 30, 32, 61, 64, 90, 127, 300, 700, 1100) for N in (33, 600, 2100, 4100, 8200, 16390)
             if M * N <= 2310000 and cf.cf_gemm_w4_form(w4_args(M=M, N=N, K=K, group=group, lda=K, lds=N, w_dtype=cf._CODES4[code],
                                                                ldc=N)).startswith(tile + " ")]
    return sizes if len(sizes) < 4 else [sizes[0], sizes[len(sizes) // 2], sizes[-1]]


def test_w4_every_tile_is_taken():
    for tile in TILES:
        for code in VALUES:
            some = [(K, group) for K, group in TILE_K if tile_sizes(tile, K, group, code)]
            for kind in (lambda g: g % 64, lambda g: g % 64 == 0 and g % 128, lambda g: g % 128 == 0):
                assert any(kind(g) for _, g in some), (tile, code)


@gpu
@pytest.mark.parametrize("K,group", TILE_K)
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("code,sdt", [("int4", F32), ("e2m1", BF16), ("int4", BF16)])
def test_w4_every_tile(tile, K, group, code, sdt):
    g = gen(K)
    for M, N in tile_sizes(tile, K, group, code):
        A, tiles, s, bias = make(g, M, N, K, group, code, sdt, bias=True)
        check_w4(cf.gemm_w4(A, tiles, s, code=code, bias=bias, out_dtype=F32), A, tiles, s, code, bias)


# Groups of 128 t: pairs of steps of 64 k share a scale where a tile has more than a block and its groups of waves (8, 4 or 1)
# have as many pairs, or four each at least; else every step has its own.
PAIRED = {"16 x 64": 8, "32 x 64": 8, "64 x 32": 8, "64 x 64": 4, "64 x 128": 4, "128 x 128": 1}
PAIR_K = [(640, 128), (1024, 128), (2176, 128), (2432, 128), (2560, 512), (4224, 128), (4480, 640), (4992, 128)]


def shares(tile, K):
    """Whether the groups of waves have equal numbers of pairs, unequal ones, or (None) steps."""
    groups, pairs = PAIRED.get(tile, 0), K // 128
    return None if not groups or pairs % groups and pairs < 4 * groups else "unequal" if pairs % groups else "equal"


def pair_form(M, N, K, group, code):
    return cf.cf_gemm_w4_form(w4_args(M=M, N=N, K=K, group=group, lda=K, lds=N, w_dtype=cf._CODES4[code], ldc=-(-N // 8) * 8))


def test_w4_form_says_what_a_scale_is_for():
    """The form's last word is the k of a scale: 32, 64, or 128 for pairs of steps."""
    seen = set()
    for K, group in TILE_K + PAIR_K:
        for M in (1, 8, 13, 32, 48, 64, 90, 127, 300, 700, 1100):
            for N in (33, 600, 2100, 4100, 8200, 16390):
                for code in VALUES:
                    tile, rest = pair_form(M, N, K, group, code).split(" tiles of ")
                    share = shares(tile, K) if group % 128 == 0 else None
                    every = 128 if share else 64 if group % 64 == 0 else 32
                    assert rest.endswith(f"scales every {every}"), (tile, rest, K, group)
                    seen.add((tile, every, share))
    for tile in TILES:
        assert {e for t, e, _ in seen if t == tile} == ({32, 64, 128} if PAIRED.get(tile, 0) else {32, 64}), tile
    for tile, groups in PAIRED.items():
        assert (tile, 128, "equal") in seen and (groups == 1 or (tile, 128, "unequal") in seen), tile


@gpu
@pytest.mark.parametrize("K,group", PAIR_K)
@pytest.mark.parametrize("tile", sorted(PAIRED))
@pytest.mark.parametrize("code,sdt", [("int4", BF16), ("e2m1", F32)])
def test_w4_pairs(tile, K, group, code, sdt):
    """Every tile of two blocks and more with equal and unequal shares of pairs, and with fewer than it takes pairs for."""
    g = gen(K)
    for M, N in tile_sizes(tile, K, group, code):
        A, tiles, s, bias = make(g, M, N, K, group, code, sdt, bias=True)
        check_w4(cf.gemm_w4(A, tiles, s, code=code, bias=bias, out_dtype=F32), A, tiles, s, code, bias)


# ---------------------------------------------------------------- refusals (no GPU)
A_, B_, C_, D_, E_ = (0x7F0000000000 + 0x100000 * i for i in range(5))


def w4_args(**kw):
    d = dict(struct_size=cf.C.sizeof(cf.GemmW4Args), M=4, N=100, K=64, group=32, A=A_, lda=64, w_dtype=cf.CF_I4, W=B_,
             s_dtype=cf.CF_F32, s=C_, lds=100, bias=None, act=0, out_dtype=cf.CF_BF16, C=D_, ldc=104)
    d.update(kw)
    return cf.GemmW4Args(*[d[f[0]] for f in cf.GemmW4Args._fields_])


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), "CF_ERR_STRUCT"), (dict(M=-1), "CF_ERR_SHAPE"), (dict(N=0), "CF_ERR_SHAPE"),
    (dict(K=0), "CF_ERR_SHAPE"), (dict(group=0), "CF_ERR_SHAPE"), (dict(group=16), "CF_ERR_SHAPE"), (dict(group=48), "CF_ERR_SHAPE"),
    (dict(K=48, lda=48, group=48), "CF_ERR_SHAPE"), (dict(group=128), "CF_ERR_SHAPE"), (dict(K=1 << 21, lda=1 << 21), "CF_ERR_SHAPE"),
    (dict(N=(1 << 20) + 1), "CF_ERR_SHAPE"), (dict(M=(1 << 30) + 1), "CF_ERR_SHAPE"), (dict(M=1 << 30, N=129, lds=129, ldc=136), "CF_ERR_SHAPE"),
    (dict(A=None), "CF_ERR_NULL"), (dict(W=None), "CF_ERR_NULL"), (dict(s=None), "CF_ERR_NULL"), (dict(C=None), "CF_ERR_NULL"),
    (dict(lda=56), "CF_ERR_LD"), (dict(ldc=96), "CF_ERR_LD"), (dict(lds=99), "CF_ERR_LD"), (dict(lda=68), "CF_ERR_ALIGN"),
    (dict(W=B_ + 8), "CF_ERR_ALIGN"), (dict(s=C_ + 2), "CF_ERR_ALIGN"), (dict(ldc=100), "CF_ERR_ALIGN"), (dict(bias=E_ + 4), "CF_ERR_ALIGN"),
    (dict(w_dtype=cf.CF_I8), "CF_ERR_DTYPE"), (dict(s_dtype=cf.CF_I8), "CF_ERR_DTYPE"), (dict(out_dtype=cf.CF_I8), "CF_ERR_DTYPE"),
    (dict(act=4), "CF_ERR_UNSUPPORTED"), (dict(C=A_), "CF_ERR_ALIAS"), (dict(C=B_), "CF_ERR_ALIAS"), (dict(C=C_), "CF_ERR_ALIAS")])
def test_w4_refuses(kw, status):
    assert cf.STATUS[cf.cf_gemm_w4(w4_args(**kw), None)] == status, cf.cf_last_error()


def quant_args(**kw):
    d = dict(struct_size=cf.C.sizeof(cf.W4QuantArgs), N=10, K=64, group=32, dtype=cf.CF_BF16, W=A_, ldw=64, w_dtype=cf.CF_I4,
             tiles=B_, s_dtype=cf.CF_F32, s=C_, lds=10)
    d.update(kw)
    return cf.W4QuantArgs(*[d[f[0]] for f in cf.W4QuantArgs._fields_])


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), "CF_ERR_STRUCT"), (dict(N=0), "CF_ERR_SHAPE"), (dict(group=24), "CF_ERR_SHAPE"), (dict(W=None), "CF_ERR_NULL"),
    (dict(tiles=None), "CF_ERR_NULL"), (dict(s=None), "CF_ERR_NULL"), (dict(ldw=60), "CF_ERR_LD"), (dict(lds=9), "CF_ERR_LD"),
    (dict(tiles=B_ + 4), "CF_ERR_ALIGN"), (dict(dtype=cf.CF_I8), "CF_ERR_DTYPE"), (dict(w_dtype=cf.CF_I8), "CF_ERR_DTYPE"),
    (dict(tiles=A_), "CF_ERR_ALIAS"), (dict(s=B_), "CF_ERR_ALIAS")])
def test_w4_quant_refuses(kw, status):
    assert cf.STATUS[cf.cf_w4_quant(quant_args(**kw), None)] == status, cf.cf_last_error()


@pytest.mark.parametrize("args,status", [
    ((0, 64, A_, 32, B_), "CF_ERR_SHAPE"), ((4, 48, A_, 32, B_), "CF_ERR_SHAPE"), ((4, 64, None, 32, B_), "CF_ERR_NULL"),
    ((4, 64, A_, 31, B_), "CF_ERR_LD"), ((4, 64, A_, 32, None), "CF_ERR_NULL"), ((4, 64, A_, 32, B_ + 4), "CF_ERR_ALIGN"),
    ((4, 64, A_, 32, A_), "CF_ERR_ALIAS")])
def test_w4_pack_refuses(args, status):
    assert cf.STATUS[cf.cf_w4_pack(*args, None)] == status, cf.cf_last_error()


def test_w4_empty_call_does_nothing():
    assert cf.cf_gemm_w4(w4_args(M=0, A=None, C=None, W=None, s=None), None) == 0


def test_w4_packed_arguments():
    for t, pack in ((cf.W4QuantArgs, cf._W4_QUANT), (cf.GemmW4Args, cf._GEMM_W4)):
        values = [3 * i + 1 for i in range(len(t._fields_))]
        assert bytes(t(*values)) == pack.pack(*values)


@gpu
def test_w4_helpers_refuse():
    A, W, s = torch.zeros((4, 64), dtype=BF16, device="cuda"), torch.zeros((2, 1, 1024), dtype=torch.uint8, device="cuda"), torch.zeros((2, 40), device="cuda")
    for call in (lambda: cf.gemm_w4(A, W[:1], s), lambda: cf.gemm_w4(A, W, s[:, :20]), lambda: cf.gemm_w4(A, W.int(), s),
                 lambda: cf.gemm_w4(A, W, torch.zeros((3, 40), device="cuda")), lambda: cf.gemm_w4(A, W, s, code="int8"),
                 lambda: cf.gemm_w4(A, W, s, act="silu"), lambda: cf.gemm_w4(A, W, s.cpu()), lambda: cf.gemm_w4(A.cpu(), W, s),
                 lambda: cf.gemm_w4(A, W, s, bias=s[0, :3]), lambda: cf.gemm_w4(A, W, s, out=A), lambda: cf.w4_quant(A, 48),
                 lambda: cf.w4_quant(A, 32, code="fp4"), lambda: cf.w4_quant(A.cpu(), 32), lambda: cf.w4_pack(W[0].t())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: cf.gemm_w4(A.float(), W, s), lambda: cf.w4_pack(A), lambda: cf.w4_quant(A, 32, scales=torch.float16)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(cf.CfError, match="CF_ERR_SHAPE"):
        cf.w4_quant(A, 16)
