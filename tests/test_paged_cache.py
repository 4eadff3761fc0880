"""The cache of pages: rotary positions with the cache's write, its read, and the
attention over it, against the definitions in 64 bits; and a decoding step of all.
u is fp32's half step; each bound counts roundings."""
import math
import threading

import pytest
import torch

from paper_2608_03537_amd import comfuse as cf
from tests.test_serving_ops import BF16, F32, F64, QMAX, U, gen

gpu = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
ROWS = {"bf16": BF16, "int8": torch.int8, "e4m3": torch.uint8}


def values(rows, scales, code):
    """What the cache's rows stand for, in 64 bits."""
    if code == "bf16":
        return rows.to(F64)
    v = rows.to(F64) if code == "int8" else rows.contiguous().view(E4M3).to(F64)
    return v * scales.to(F64).unsqueeze(-1)


def new_cache(n, Hk, page, d, code, major="heads", fill=None):
    """Pages of zeros (or of a fill), stored head-major, or token-major with gaps."""
    if major == "heads":
        c = cf.cache_pages(n, Hk, page, d, code)
    else:
        rows = [torch.zeros((n, page, Hk + 1, d + 16), dtype=ROWS[code], device="cuda")[:, :, :Hk, :d].transpose(1, 2) for _ in range(2)]
        sc = [None, None] if code == "bf16" else [torch.zeros((n, Hk + 2, page + 4), device="cuda")[:, 1:1 + Hk, 4:] for _ in range(2)]
        c = (*rows, *sc)
    if fill is not None:
        for t in c:
            if t is not None:
                t.fill_(fill)
    return c


# ---------------------------------------------------------------- cache_write
def rotate32(x, pos, freq, sections, pairs):
    """x [T, heads, d] fp32 on the CPU, each operation in fp32, as the definition says."""
    rot = 2 * freq.numel()
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections))
    angle = pos[axis].t().to(F64) * freq.to(F64)
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    y = x.clone()
    one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if pairs == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = x[..., one], x[..., two]
    y[..., one] = a * c - b * s
    y[..., two] = b * c + a * s
    return y


def quantise32(x, code):
    m = x.abs().amax(-1)
    d = m / torch.full_like(m, QMAX[code])
    z = torch.where(d[..., None] > 0, x / d[..., None], torch.zeros_like(x)).clamp(-QMAX[code], QMAX[code])
    return (z.round().to(torch.int8) if code == "int8" else z.to(E4M3).view(torch.uint8)), d


def check_write(T, H, Hk, d, code, page, rot, axes, pairs, g, major="heads", in_place=False, most=100000):
    wide = torch.randn((T, H + 2 * Hk + 1, d + 8), generator=g, device="cuda").to(BF16)
    q, k, v = wide[:, :H, :d], wide[:, H:H + Hk, :d], wide[:, H + Hk:H + 2 * Hk, :d]
    q0 = q.clone()
    n = -(-T // page) + 2
    kc, vc, ks, vs = new_cache(n, Hk, page, d, code, major, fill=3)
    slots = torch.randperm(n * page, generator=g, device="cuda")[:T].to(torch.int32)
    if T > 2:
        slots[1], slots[2] = -1, n * page                  # padding, and behind the cache
    half = rot // 2
    sections = [half] if axes == 1 else [half - 2 * (axes - 1)] + [2] * (axes - 1)
    pos = torch.randint(0, most, (axes, T + 3), generator=g, device="cuda", dtype=torch.int32)[:, :T]
    freq = 10000.0 ** (-torch.arange(half, device="cuda") / max(half, 1))
    kw = dict(pos=pos if axes > 1 else pos[0], freq=freq, sections=sections, pairs=pairs) if rot else {}
    out = cf.cache_write(k, v, slots, kc, vc, ks, vs, q=q if H else None, out=q if H and in_place else None, **kw)
    assert (out is None) == (H == 0) and (not in_place or not H or out is q)

    def turned(x):
        x = x.float().cpu()
        return rotate32(x, pos.cpu(), freq.cpu(), sections, pairs) if rot else x

    if H:
        assert torch.equal(out.cpu(), turned(q0).to(BF16))
    used = [t for t in range(T) if 0 <= int(slots[t]) < n * page]
    at = slots[used].long().cpu()
    for rows, scales, x in ((kc, ks, turned(k)), (vc, vs, v.float().cpu())):
        want = torch.full((n, Hk, page, d), 3, dtype=ROWS[code])
        if code == "bf16":
            want[at // page, :, at % page] = x[used].to(BF16)
        else:
            c, s = quantise32(x, code)
            want[at // page, :, at % page] = c[used]
            wants = torch.full((n, Hk, page), 3.0)
            wants[at // page, :, at % page] = s[used]
            assert torch.equal(scales.cpu(), wants)
        assert torch.equal(rows.cpu(), want)


@gpu
@pytest.mark.parametrize("code", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("T,H,Hk,d,page,rot,axes,pairs", [
    (1, 1, 1, 64, 16, 64, 1, "halves"), (1, 32, 8, 128, 16, 128, 1, "halves"), (5, 0, 2, 64, 16, 32, 1, "neighbours"),
    (3, 7, 1, 128, 32, 64, 3, "halves"), (33, 14, 2, 64, 64, 64, 3, "neighbours"), (200, 4, 4, 128, 256, 128, 2, "neighbours"),
    (70, 40, 40, 64, 16, 16, 1, "halves"), (17, 3, 5, 128, 1024, 0, 1, "halves"), (40, 64, 8, 128, 128, 96, 4, "halves")])
def test_write(T, H, Hk, d, page, rot, axes, pairs, code):
    """Codes, scales and rotated rows bit for bit; other rows of the cache untouched."""
    g = gen(T * 1000 + H)
    check_write(T, H, Hk, d, code, page, rot, axes, pairs, g)
    check_write(T, H, Hk, d, code, page, rot, axes, pairs, g, major="tokens", in_place=True)


@gpu
def test_write_far_positions():
    """Angles up to 2^31: the product and its reduction are in 64 bits."""
    check_write(64, 2, 2, 128, "bf16", 16, 128, 1, "halves", gen(3), most=2 ** 31 - 1)


@gpu
def test_write_angles():
    """Unit rows turned by angles of all sizes: cosine and sine are those of 64 bits, rounded to bf16 from fp32; 2^45 gives NaN."""
    g = gen(77)
    T, half = 4096, 32
    pos = torch.randint(0, 2 ** 31 - 1, (T,), generator=g, device="cuda").to(torch.int32)
    pos[:2048] = torch.arange(2048, device="cuda")
    freq = torch.exp2(torch.rand((half,), generator=g, device="cuda") * 30 - 24)       # 2^-24 .. 2^6: angles below 2^37
    k = torch.zeros((T, 1, 64), dtype=BF16, device="cuda")
    k[..., :half] = 1.0
    kc, vc, _, _ = cf.cache_pages(4, 1, 1024, 64)
    slots = torch.arange(T, dtype=torch.int32, device="cuda")
    cf.cache_write(k, k, slots, kc, vc, pos=pos, freq=freq)
    angle = (pos.to(F64)[:, None] * freq.to(F64)).cpu()
    rows = kc.view(T, 64).cpu()
    assert torch.equal(rows[:, :half], torch.cos(angle).float().to(BF16)) and torch.equal(rows[:, half:], torch.sin(angle).float().to(BF16))
    freq[0], freq[1] = 2.0 ** 44, float("inf")
    pos[:] = 2
    cf.cache_write(k, k, slots, kc, vc, pos=pos, freq=freq)
    rows = kc.view(T, 64)
    assert bool(rows[:, [0, 1, half, half + 1]].isnan().all()) and not bool(rows[:, 2:half].isnan().any())


@gpu
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_write_special_rows(code, d):
    """Rows of zeros, NaN, infinity and of values whose scale is subnormal, or underflows."""
    k = torch.randn((7, 1, d), generator=gen(d), device="cuda").to(BF16)
    k[1] = 0.0
    k[2, 0, d - 1] = float("nan")
    k[3, 0, 0] = -math.inf
    k[4] = (k[4].float() * 1e-37).to(BF16)
    k[5] = (torch.arange(d, device="cuda")[None] % 5 * 1.1e-40).to(BF16)
    k[6] = (k[6].float().clamp(-1, 1) * 3e38).to(BF16)
    kc, vc, ks, vs = cf.cache_pages(1, 1, 16, d, code)
    cf.cache_write(k, k, torch.arange(7, dtype=torch.int32, device="cuda"), kc, vc, ks, vs)
    assert torch.equal(kc, vc) and torch.equal(ks.nan_to_num(9.0), vs.nan_to_num(9.0))
    c, s = quantise32(k.float().cpu()[:, 0], code)
    bad = [2, 3]
    good = [0, 1, 4, 5, 6]
    assert bool(ks[0, 0, bad].isnan().all()) and not kc[0, 0, bad].any()
    assert torch.equal(ks[0, 0, good].cpu(), s[good])
    same = kc[0, 0, good].cpu() == c[good]
    if code == "e4m3":   # either zero stands for a value of no sign
        same = same | ((kc[0, 0, good].cpu() & 127) == 0) & ((c[good] & 127) == 0)
    assert bool(same.all())


@gpu
def test_write_more_tasks_than_a_grid():
    """2^20 workgroups at most: the rest are looped over, the table of angles with them."""
    T = (1 << 20) + 37
    k = torch.zeros((T, 1, 64), dtype=BF16, device="cuda")
    k[:, 0, 0] = 1.0
    pos = torch.arange(T, dtype=torch.int32, device="cuda") % 1000
    freq = torch.full((8,), 1e-3, device="cuda")
    kc, vc, _, _ = cf.cache_pages(-(-T // 1024), 1, 1024, 64)
    cf.cache_write(k, k, torch.arange(T, dtype=torch.int32, device="cuda"), kc, vc, pos=pos, freq=freq)
    angle = pos.to(F64) * freq[0].to(F64)
    got = kc.view(-1, 64)[:T]
    assert torch.equal(got[:, 0], torch.cos(angle).float().to(BF16)) and torch.equal(got[:, 8], torch.sin(angle).float().to(BF16))
    assert torch.equal(vc.view(-1, 64)[:T], k[:, 0]) and not kc.view(-1, 64)[T:].any()


@gpu
@pytest.mark.parametrize("code", ["bf16", "int8"])
def test_write_waves_take_several_tokens(code):
    """As many tokens as a call may have, several for every wave of a full grid: each is turned by its own angles."""
    T = (1 << 24) - 5
    k = torch.zeros((T, 1, 64), dtype=BF16, device="cuda")
    k[:, 0, 0] = 1.0
    pos = torch.arange(T, dtype=torch.int32, device="cuda") % 1009        # differ between the tokens of a wave
    freq = torch.full((8,), 1e-3, device="cuda")
    kc, vc, ks, vs = cf.cache_pages(-(-T // 1024), 1, 1024, 64, code)
    cf.cache_write(k, k, torch.arange(T, dtype=torch.int32, device="cuda"), kc, vc, ks, vs, pos=pos, freq=freq)
    angle = torch.arange(1009, device="cuda").to(F64) * freq[0].to(F64)
    want = torch.zeros((1009, 64), device="cuda")
    want[:, 0], want[:, 8] = torch.cos(angle).float(), torch.sin(angle).float()
    at = pos.long()
    if code == "bf16":
        assert torch.equal(kc.view(-1, 64)[:T], want.to(BF16)[at]) and torch.equal(vc.view(-1, 64)[:T], k[:, 0])
    else:
        c, s = quantise32(want.cpu(), code)
        assert torch.equal(kc.view(-1, 64)[:T], c.cuda()[at]) and torch.equal(ks.view(-1)[:T], s.cuda()[at])
        assert bool((vc.view(-1, 64)[:T, 0] == 127).all()) and not vc.view(-1, 64)[:, 1:].any()
        assert not ks.view(-1)[T:].any() and not vs.view(-1)[T:].any()
    assert not kc.view(-1, 64)[T:].any() and not vc.view(-1, 64)[T:].any()


# ---------------------------------------------------------------- filled caches
def fill_pages(g, n, Hk, page, d, code, major="heads", std=1.0):
    kc, vc, ks, vs = new_cache(n, Hk, page, d, code, major)
    for rows, scales in ((kc, ks), (vc, vs)):
        x = torch.randn((n, Hk, page, d), generator=g, device="cuda") * std
        if code == "bf16":
            rows.copy_(x.to(BF16))
        else:
            s = torch.rand((n, Hk, page), generator=g, device="cuda") + 0.5
            scales.copy_(s * std / (40.0 if code == "int8" else 150.0))
            x = x / std
            rows.copy_((x * 40).round().clamp(-127, 127).to(torch.int8) if code == "int8"
                       else (x * 150).clamp(-448, 448).to(E4M3).view(torch.uint8))
    return kc, vc, ks, vs


def poison(cache, code, keep):
    """NaN (or the largest codes) in every row of the cache that `keep` [n, page] does not name."""
    kc, vc, ks, vs = cache
    for rows, scales in ((kc, ks), (vc, vs)):
        bad = ~keep[:, None, :].expand(rows.shape[:3])
        rows[bad] = float("nan") if code == "bf16" else 127   # 127: NaN of E4M3
        if scales is not None:
            scales[bad] = float("nan")


def sequences(cache, code, table, lens, page):
    """Per sequence the keys and values [Hk, n, d] in 64 bits, and which of them the cache has."""
    kc, vc, ks, vs = cache
    n = kc.shape[0]
    for b in range(table.shape[0]):
        length = max(0, min(int(lens[b]), table.shape[1] * page))
        t = table[b, :-(-length // page)].long()
        has = ((t >= 0) & (t < n)).repeat_interleave(page)[:length]
        t = t.clamp(0, n - 1)
        yield [values(r[t], None if s is None else s[t], code).transpose(0, 1).reshape(r.shape[1], -1, r.shape[3])[:, :length]
               for r, s in ((kc, ks), (vc, vs))] + [has]


def make_table(g, n, B, pages):
    return torch.randperm(n, generator=g, device="cuda")[:B * pages].to(torch.int32).view(B, pages)


def rows_in_use(n, page, table, lens):
    keep = torch.zeros((n, page), dtype=torch.bool, device="cuda")
    for b in range(table.shape[0]):
        for j in range(max(0, min(int(lens[b]), table.shape[1] * page))):
            t = int(table[b, j // page])
            if 0 <= t < n:
                keep[t, j % page] = True
    return keep


# ---------------------------------------------------------------- cache_read
@gpu
@pytest.mark.parametrize("code", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("major", ["heads", "tokens"])
@pytest.mark.parametrize("B,Hk,S,d,page,pages", [(1, 1, 1, 64, 16, 1), (3, 2, 100, 128, 16, 7), (5, 1, 64, 64, 64, 2), (4, 3, 300, 64, 32, 9),
                                                 (2, 8, 1000, 128, 128, 8)])
def test_read(B, Hk, S, d, page, pages, major, code):
    g = gen(S)
    n = B * pages + 1
    cache = fill_pages(g, n, Hk, page, d, code, major)
    table = make_table(g, n, B, pages)
    lens = torch.randint(0, min(S, page * pages) + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    lens[0] = S + 5
    if B > 2:
        lens[1], lens[2], table[0, 0] = 0, -3, n
    out = [torch.full((B, S, Hk, d + 8), 7.0, dtype=BF16, device="cuda")[..., :d].transpose(1, 2) for _ in range(2)]
    K, V = cf.cache_read(cache[0], cache[1], table, lens, cache[2], cache[3], out=out)
    assert K is out[0] and V is out[1]
    want = torch.full((2, B, Hk, S, d), 7.0, dtype=BF16, device="cuda")
    for b, (k, v, has) in enumerate(sequences(cache, code, table, lens.clamp(max=S), page)):
        for i, x in ((0, k), (1, v)):   # code * scale in fp32, then bf16: fp32's product is rounded before
            x = x.float().to(BF16)
            want[i, b, :, :x.shape[1]][:, has] = x[:, has]
    assert torch.equal(K, want[0]) and torch.equal(V, want[1])
    assert bool((out[0]._base[..., d:] == 7).all())
    K2, _ = cf.cache_read(cache[0], cache[1], table, lens, cache[2], cache[3])
    assert K2.shape == (B, Hk, pages * page, d)


@gpu
@pytest.mark.parametrize("code", ["bf16", "e4m3"])
def test_read_more_tasks_than_a_grid(code):
    """More than twice 2^20 groups of 32 rows: workgroups take several, the last rows of the last sequence among them."""
    g = gen(31)
    B, S, page, n = 5, 1 << 24, 1024, 7
    cache = fill_pages(g, n, 1, page, 64, code)
    table = torch.randint(0, n, (B, S // page), generator=g, device="cuda", dtype=torch.int32)
    lens = torch.tensor([S, 3, S - 40, 0, S - 1], dtype=torch.int32, device="cuda")
    K, V = (torch.full((B, 1, S, 64), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    cf.cache_read(cache[0], cache[1], table, lens, cache[2], cache[3], out=(K, V))
    for out, rows, scales in ((K, cache[0], cache[2]), (V, cache[1], cache[3])):
        rows = values(rows, scales, code).float().to(BF16)[:, 0]          # [n, page, 64]
        for b in range(B):
            m = int(lens[b])
            assert torch.equal(out[b, 0, :m], rows[table[b].long()].view(S, 64)[:m]) and bool((out[b, 0, m:] == 7).all())


# ---------------------------------------------------------------- attention_paged
def paged64(Q, cache, code, table, lens, page, causal, scale, cap):
    """(O, sum of w |v|) in 64 bits, sequence by sequence."""
    B, H, Lq, d = Q.shape
    Hk = cache[0].shape[1]
    G = H // Hk
    O, A = (torch.zeros(Q.shape, dtype=F64, device="cuda") for _ in range(2))
    for b, (k, v, has) in enumerate(sequences(cache, code, table, lens, page)):
        n = k.shape[1]
        if not n:
            continue
        for h in range(Hk):
            x = Q[b, h * G:(h + 1) * G].to(F64).reshape(G * Lq, d) @ k[h].t().contiguous() * scale
            if cap:
                x = cap * torch.tanh(x / cap)
            see = has[None].expand(G * Lq, n)
            if causal:
                i = torch.arange(Lq, device="cuda").repeat(G)[:, None]
                see = see & (torch.arange(n, device="cuda") < n - (Lq - 1 - i))
            x = x.masked_fill(~see, -math.inf)
            w = torch.where(see, torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e300)), 0.0)
            w = w / w.sum(-1, keepdim=True).clamp(min=1e-300)
            vh = torch.where(has[:, None], v[h], 0.0)
            O[b, h * G:(h + 1) * G] = (w @ vh).view(G, Lq, d)
            A[b, h * G:(h + 1) * G] = (w @ vh.abs()).view(G, Lq, d)
    return O, A


def check_paged(O, Q, cache, code, table, lens, page, causal=False, scale=None, cap=0.0):
    d = Q.shape[-1]
    scale = d ** -0.5 if scale is None else scale
    ref, a = paged64(Q, cache, code, table, lens, page, causal, scale, cap)
    used = list(sequences(cache, code, table, lens, page))
    longest = max([float(k[:, has].norm(dim=-1).max()) for k, _, has in used if bool(has.any())], default=0.0)
    top = max([float(v[:, has].abs().max()) for _, v, has in used if bool(has.any())], default=0.0)
    # P is rounded to bf16 in the numerator: off by 2^-8 w |v|; a score is off by (d + 2) u |q| |k| scale, with a cap by 6 u
    # cap besides, and a weight by twice that and the exponentials' 4 u, sums of up to 2^10 terms a lane; then
    # the output's rounding
    e = 2 * ((d + 2) * U * float(Q.float().norm(dim=-1).max()) * longest * scale + 6 * U * cap) + 2 * 2.0 ** 10 * U
    # exponentials below fp32's smallest normal are flushed: beside a row's largest weight each key loses at most 2^-118 |v|
    lost = table.shape[1] * page * 2.0 ** -118 * top
    tol = (2.0 ** -8 * 1.01 + e) * a + e * ref.abs() + 2.0 ** -8 * 1.01 * ref.abs() + lost
    bad = ~((O.to(F64) - ref).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), O[bad][:4].tolist(), ref[bad][:4].tolist())


def paged_case(g, B, H, Hk, Lq, most, d, page, code, major="heads", std=1.0):
    pages = -(-most // page)
    n = B * pages + 2
    cache = fill_pages(g, n, Hk, page, d, code, major, std)
    Q = (torch.randn((B, Lq, H, d), generator=g, device="cuda") * std).to(BF16).transpose(1, 2)
    return Q, cache, make_table(g, n, B, pages)


@gpu
@pytest.mark.parametrize("code", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,Hk,Lq,most,page", [
    (1, 1, 1, 1, 1, 16), (2, 4, 2, 1, 31, 16), (3, 8, 8, 1, 64, 32), (5, 8, 1, 1, 129, 16), (4, 14, 2, 1, 1000, 64),
    (2, 6, 2, 5, 257, 128), (1, 8, 2, 16, 63, 16), (3, 16, 1, 1, 500, 256), (1, 32, 8, 1, 4096, 16), (2, 32, 2, 3, 777, 32),
    (1, 64, 1, 2, 3000, 1024), (70, 4, 4, 1, 300, 16), (2, 2, 2, 64, 200, 16), (9, 12, 12, 2, 100, 64), (1, 16, 4, 5, 9000, 16)])
def test_paged_sizes(B, H, Hk, Lq, most, page, d, code):
    g = gen(most * 10 + B)
    Q, cache, table = paged_case(g, B, H, Hk, Lq, most, d, page, code)
    lens = torch.randint(max(0, most - page), most + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    lens[0] = most
    if B > 1:
        lens[1] = 1
    if B > 2:
        lens[2] = 0
    for causal in ((False, True) if Lq > 1 else (False,)):
        O = cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=causal)
        check_paged(O, Q, cache, code, table, lens, page, causal)
    O = cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=Lq > 1, softcap=5.0, scale=0.3)
    check_paged(O, Q, cache, code, table, lens, page, Lq > 1, scale=0.3, cap=5.0)


@gpu
@pytest.mark.parametrize("code", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("major", ["heads", "tokens"])
@pytest.mark.parametrize("Lq", [1, 4])
def test_paged_hidden_rows(Lq, major, code):
    """NaN in all rows that no sequence uses, table entries that name no page behind the lengths and within them."""
    g = gen(Lq)
    B, H, Hk, d, page, pages = 7, 8, 2, 64, 16, 20
    Q, cache, table = paged_case(g, B, H, Hk, Lq, page * pages, d, page, code, major)
    lens = torch.tensor([1, 16, 17, 33, 300, 0, -2], dtype=torch.int32, device="cuda")
    for b in range(B):
        table[b, -(-max(0, int(lens[b])) // page):] = [-1, 1 << 30, -2 ** 31][b % 3]
    table[4, 0], table[4, 7], table[4, 18], table[3, 2] = -1, cache[0].shape[0], -5, -1
    poison(cache, code, rows_in_use(cache[0].shape[0], page, table, lens))
    full = torch.full((B, Lq, H + 1, d + 8), 7.0, dtype=BF16, device="cuda")
    out = full[:, :, :H, :d].transpose(1, 2)
    O = cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=Lq > 1, out=out)
    assert O is out and not O[5:].any()
    check_paged(O, Q, cache, code, table, lens, page, Lq > 1)
    assert bool((full[:, :, H:] == 7).all()) and bool((full[..., d:] == 7).all())
    table[:] = -1
    O = cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=Lq > 1)
    assert not O.any()


@gpu
@pytest.mark.parametrize("code", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("d,H,Hk,Lq,length,spoiled", [(64, 2, 2, 5, 40, 1), (128, 4, 2, 7, 65, 3), (64, 8, 1, 64, 70, 40), (128, 1, 1, 2, 2, 1)])
def test_paged_causal_hides_nan(d, H, Hk, Lq, length, spoiled, code):
    """NaN in the last rows of keys and values: no query that causal hides them from sees it, all others do."""
    g = gen(length)
    B, page = 3, 32
    Q, cache, table = paged_case(g, B, H, Hk, Lq, length, d, page, code)
    lens = torch.full((B,), length, dtype=torch.int32, device="cuda")
    for t in range(length - spoiled, length):
        for b in range(B):
            n = int(table[b, t // page])
            for x in ((0, 1) if code == "bf16" else (2, 3)):
                cache[x][n, :, t % page] = float("nan")
            if code == "e4m3":
                cache[0][n, :, t % page], cache[1][n, :, t % page] = 127, 127
    O = cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=True)
    assert bool(O[:, :, Lq - spoiled:].isnan().all())
    clean = slice(0, Lq - spoiled)
    check_paged(O[:, :, clean], Q[:, :, clean], cache, code, table, lens - spoiled, page, True)
    if code == "bf16":   # an infinity in one dimension of the last value
        cache[0].nan_to_num_(0.0), cache[1].nan_to_num_(0.0)
        for b in range(B):
            cache[1][int(table[b, (length - 1) // page])][:, (length - 1) % page, 3] = -math.inf
        P = cf.attention_paged(Q, cache[0], cache[1], table, lens, causal=True)
        assert bool((P[:, :, -1, 3] == -math.inf).all()) and bool(P[:, :, :-1].isfinite().all()) and int((~P.isfinite()).sum()) == B * H


@gpu
@pytest.mark.parametrize("code", ["bf16", "int8", "e4m3"])
def test_paged_large_scores(code):
    """Scores of hundreds: the running maximum is raised many times, and weights underflow."""
    g = gen(1)
    Q, cache, table = paged_case(g, 3, 8, 2, 2, 2000, 128, 32, code, std=6.0)
    lens = torch.tensor([2000, 1999, 37], dtype=torch.int32, device="cuda")
    check_paged(cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=True), Q, cache, code, table, lens, 32, True)


@gpu
@pytest.mark.parametrize("code", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("cap", [50.0, 65.0, 200.0, 1e3, 1e6, 1e30])
def test_paged_caps(cap, code):
    """Scores of up to hundreds under caps of all sizes: what a cap adds to their error does not grow with it."""
    g = gen(21)
    d, page = 128, 32
    Q, cache, table = paged_case(g, 3, 8, 2, 2, 900, d, page, code, std=5.0)
    lens = torch.tensor([900, 333, 40], dtype=torch.int32, device="cuda")
    O = cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=True, softcap=cap)
    ref, a = paged64(Q, cache, code, table, lens, page, True, d ** -0.5, cap)
    longest = max(float(k.norm(dim=-1).max()) for k, _, _ in sequences(cache, code, table, lens, page))
    most = float(Q.float().norm(dim=-1).max()) * longest * d ** -0.5
    # as check_paged, but for the cap: 2^-21 of it, and past 64 2^-19 of the score
    e = 2 * ((d + 2) * U * most + (2.0 ** -21 * cap if cap <= 64 else 2.0 ** -19 * most)) + 2 * 2.0 ** 10 * U
    top = max(float(v.abs().max()) for _, v, _ in sequences(cache, code, table, lens, page))
    tol = (2.0 ** -8 * 1.01 + e) * a + e * ref.abs() + 2.0 ** -8 * 1.01 * ref.abs() + table.shape[1] * page * 2.0 ** -118 * top
    assert bool(((O.to(F64) - ref).abs() <= tol).all())


@gpu
def test_paged_shares_pages():
    """Two sequences on the same pages, the same page twice in one, a shared table row (stride 0)."""
    g = gen(2)
    Q, cache, table = paged_case(g, 2, 4, 2, 1, 100, 64, 16, "int8")
    table[1] = table[0]
    table[0, 3] = table[0, 1]
    lens = torch.tensor([100, 50], dtype=torch.int32, device="cuda")
    check_paged(cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3]), Q, cache, "int8", table, lens, 16)
    one = table[:1].expand(2, -1)
    check_paged(cf.attention_paged(Q, cache[0], cache[1], one, lens, cache[2], cache[3]), Q, cache, "int8", one, lens, 16)


@gpu
def test_paged_offsets_pass_32_bits():
    """A cache of more than 4 GiB of rows, read and written at its end."""
    n, Hk, page, d = 70000, 4, 128, 128
    kc = torch.zeros((n, Hk, page, d), dtype=torch.int8, device="cuda")
    ks = torch.ones((n, Hk, page), device="cuda")
    assert kc.numel() > 2 ** 32
    g = gen(4)
    k, v = (torch.randn((200, Hk, d), generator=g, device="cuda").to(BF16) for _ in range(2))
    vc, vs = kc.clone(), ks.clone()
    slots = (torch.arange(200, device="cuda") + (n - 2) * page).to(torch.int32)
    cf.cache_write(k, v, slots, kc, vc, ks, vs)
    c, s = quantise32(k.float().cpu(), "int8")
    assert torch.equal(kc[n - 2:].transpose(1, 2).reshape(-1, Hk, d)[:200].cpu(), c) and not kc[:n - 2].any()
    assert torch.equal(ks[n - 2:].transpose(1, 2).reshape(-1, Hk)[:200].cpu(), s)
    table, lens = torch.tensor([[n - 2, n - 1]], dtype=torch.int32, device="cuda"), torch.tensor([200], dtype=torch.int32, device="cuda")
    Q = torch.randn((1, 8, 1, d), generator=g, device="cuda").to(BF16)
    small = [t[n - 2:] for t in (kc, vc, ks, vs)]
    O = cf.attention_paged(Q, kc, vc, table, lens, ks, vs)
    check_paged(O, Q, small, "int8", table - (n - 2), lens, page)
    K, V = cf.cache_read(kc, vc, table, lens, ks, vs)
    K2, V2 = cf.cache_read(small[0], small[1], table - (n - 2), lens, small[2], small[3])
    assert torch.equal(K[:, :, :200], K2[:, :, :200]) and torch.equal(V[:, :, :200], V2[:, :, :200])


@gpu
@pytest.mark.parametrize("code,B,H,Hk,Lq,d", [("bf16", 1, 32, 8, 1, 128), ("int8", 4, 8, 8, 1, 64), ("e4m3", 2, 16, 4, 5, 64), ("bf16", 9, 8, 2, 3, 128),
                                              ("int8", 1, 16, 2, 12, 128)])
def test_paged_width_of_the_table_changes_nothing(code, B, H, Hk, Lq, d):
    """A sequence is cut by its length: under a table as wide as it needs and under one of 65536 keys, the same bits."""
    g = gen(B + H)
    for most in (20, 300, 580, 1000, 4096, 9000):
        Q, cache, table = paged_case(g, B, H, Hk, Lq, most, d, 16, code)
        lens = torch.randint(1, most + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        lens[0] = most
        wide = torch.full((B, 4096), -1, dtype=torch.int32, device="cuda")
        wide[:, :table.shape[1]] = table
        O, P = (cf.attention_paged(Q, cache[0], cache[1], t, lens, cache[2], cache[3], causal=Lq > 1) for t in (table, wide))
        assert torch.equal(O, P), most
        check_paged(P, Q, cache, code, table, lens, 16, Lq > 1)


@gpu
def test_paged_short_sequences_take_no_workspace():
    """Up to 300 keys a block is not cut, however wide its table: its partial results are not written."""
    g = gen(15)
    for d, Lq in ((64, 1), (64, 6), (128, 1), (128, 6)):
        Q, cache, table = paged_case(g, 3, 8, 2, Lq, 300, d, 16, "bf16")
        wide = torch.full((3, 4096), -1, dtype=torch.int32, device="cuda")
        wide[:, :table.shape[1]] = table
        lens = torch.tensor([300, 299, 130], dtype=torch.int32, device="cuda")
        need = cf.cf_attention_paged_workspace(paged_args(code_dtype=cf.CF_BF16, batch=3, H=8, Hk=2, Lq=Lq, d=d, pages=4096))
        assert need > cf.CF_PAGED_WS_HEADER_BYTES
        ws = torch.full((need,), 0x5A, dtype=torch.uint8, device="cuda")
        ws[:cf.CF_PAGED_WS_HEADER_BYTES] = 0
        O = cf.attention_paged(Q, cache[0], cache[1], wide, lens, causal=Lq > 1, ws=ws)
        check_paged(O, Q, cache, "bf16", table, lens, 16, Lq > 1)
        assert not ws[:cf.CF_PAGED_WS_HEADER_BYTES].any() and bool((ws[cf.CF_PAGED_WS_HEADER_BYTES:] == 0x5A).all())


@gpu
def test_paged_repeatable_own_workspace_and_streams():
    """The same bits again, from a workspace of the caller's own and on another stream; counters are left zero."""
    g = gen(6)
    Q, cache, table = paged_case(g, 2, 16, 2, 3, 5000, 128, 16, "e4m3")
    lens = torch.tensor([5000, 1234], dtype=torch.int32, device="cuda")
    call = lambda **kw: cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=True, **kw)  # noqa: E731
    want = call()
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [call(ws=ws), call(stream=s), call()]
    torch.cuda.synchronize()
    assert all(torch.equal(want, x) for x in got) and not ws[:cf.CF_PAGED_WS_HEADER_BYTES].any()


@gpu
@pytest.mark.parametrize("code,B,Hk,most,d", [("bf16", 12, 8, 4300, 128), ("int8", 40, 8, 2500, 128), ("e4m3", 70, 8, 2800, 64)])
@pytest.mark.parametrize("Lq", [1, 3, 6])
def test_paged_large_cache(code, B, Hk, most, d, Lq):
    """More rows than the last-level cache holds are read past it."""
    g = gen(B)
    Q, cache, table = paged_case(g, B, 4 * Hk, Hk, Lq, most, d, 64, code)
    lens = torch.randint(1, most + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    form = cf.cf_attention_paged_form(paged_args(batch=B, H=4 * Hk, Hk=Hk, Lq=Lq, d=d, pages=table.shape[1], page=64,
                                                 code_dtype={"bf16": cf.CF_BF16, "int8": cf.CF_I8, "e4m3": cf.CF_FP8_E4M3}[code]))
    assert form.endswith("read once"), form
    O = cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=Lq > 1)
    check_paged(O, Q, cache, code, table, lens, 64, Lq > 1)


@gpu
def test_paged_two_graphs_and_threads():
    """Two graphs replayed beside each other and beside eager calls of two threads that share a stream."""
    cases = []
    for seed in (1, 2):
        Q, cache, table = paged_case(gen(seed), 2, 16, 2, 2, 6000, 128, 16, "int8")
        lens = torch.tensor([6000, 2000 + seed], dtype=torch.int32, device="cuda")
        cases.append((Q, cache[0], cache[1], table, lens, cache[2], cache[3]))
    want = [cf.attention_paged(*c, causal=True) for c in cases]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in cases]
    for c in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append([cf.attention_paged(*c, causal=True) for _ in range(3)])
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(3):
        for o in outs[0] + outs[1]:
            o.zero_()
        torch.cuda.synchronize()
        got = [[], []]

        def eager(i):
            got[i] += [cf.attention_paged(*cases[i], causal=True) for _ in range(20)]

        threads = [threading.Thread(target=eager, args=(i,)) for i in (0, 1)]
        for t in threads:
            t.start()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
                graph.replay()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert len(got[i]) == 20 and all(torch.equal(want[i], o) for o in got[i] + outs[i])


@gpu
def test_cache_operators_on_another_stream():
    g = gen(12)
    s = torch.cuda.Stream()
    caches = [cf.cache_pages(20, 4, 16, 64, "e4m3") for _ in range(2)]
    k, v, q = (torch.randn((100, h, 64), generator=g, device="cuda").to(BF16) for h in (4, 4, 8))
    slots, pos = torch.randperm(320, generator=g, device="cuda")[:100].to(torch.int32), torch.arange(100, dtype=torch.int32, device="cuda")
    table, lens = torch.arange(20, dtype=torch.int32, device="cuda").view(2, 10), torch.tensor([150, 77], dtype=torch.int32, device="cuda")
    freq = torch.rand((32,), generator=g, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    got = []
    for c, kw in zip(caches, ({}, {"stream": s})):
        r = cf.cache_write(k, v, slots, *c, q=q, pos=pos, freq=freq, **kw)
        K, V = (torch.zeros((2, 4, 160, 64), dtype=BF16, device="cuda") for _ in range(2))
        torch.cuda.synchronize()
        cf.cache_read(c[0], c[1], table, lens, c[2], c[3], out=(K, V), **kw)
        got.append((r, K, V, *c))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got)) and bool(got[0][1].any())


@gpu
def test_helpers_of_nothing():
    """No tokens, no sequences, no queries, no rows, no pages, no weights' tokens."""
    cache = cf.cache_pages(4, 2, 16, 64, "int8")
    i32 = dict(dtype=torch.int32, device="cuda")
    none = torch.zeros((0, 2, 64), dtype=BF16, device="cuda")
    freq = torch.ones((32,), device="cuda")
    q = cf.cache_write(none, none, torch.zeros((0,), **i32), *cache, q=torch.zeros((0, 4, 64), dtype=BF16, device="cuda"),
                       pos=torch.zeros((0,), **i32), freq=freq)
    assert q.shape == (0, 4, 64) and not any(t.any() for t in cache)
    for B, pages in ((0, 3), (2, 0)):
        table, lens = torch.zeros((B, pages), **i32), torch.full((B,), 5, **i32)
        K, V = cf.cache_read(cache[0], cache[1], table, lens, cache[2], cache[3])
        assert K.shape == V.shape == (B, 2, pages * 16, 64)
        for Lq in (0, 1, 2):
            Q = torch.ones((B, 4, Lq, 64), dtype=BF16, device="cuda")
            O = cf.attention_paged(Q, cache[0], cache[1], table, lens, cache[2], cache[3], causal=Lq > 1)
            assert O.shape == Q.shape and not O.any()
    tiles, s = cf.w4_quant(torch.ones((40, 64), device="cuda"), 32)
    assert cf.gemm_w4(torch.zeros((0, 64), dtype=BF16, device="cuda"), tiles, s).shape == (0, 40)


# ---------------------------------------------------------------- a decoding step
class Step:
    """One layer's attention block of a decoding step: 4-bit projection, rotation and cache write, attention, 4-bit projection."""

    def __init__(self, g, B, H, Hk, d, code, page, pages):
        self.B, self.H, self.Hk, self.d, self.code = B, H, Hk, d, code
        D = H * d
        W = torch.randn(((H + 2 * Hk) * d, D), generator=g, device="cuda") * D ** -0.5
        self.wqkv, self.wo = cf.w4_quant(W, 64), cf.w4_quant(torch.randn((D, D), generator=g, device="cuda") * D ** -0.5, 128, code="e2m1")
        self.cache = cf.cache_pages(B * pages, Hk, page, d, code)
        self.table = make_table(g, B * pages, B, pages)
        self.freq = 10000.0 ** (-torch.arange(d // 2, device="cuda") / (d // 2))
        self.page = page

    def __call__(self, x, pos, lens):
        """x [B, n, D]: the last n of lens tokens."""
        B, n, D = x.shape
        qkv = cf.gemm_w4(x.reshape(B * n, D), *self.wqkv).view(B * n, -1, self.d)
        q, k, v = qkv.split([self.H, self.Hk, self.Hk], 1)
        p = pos.long()
        slots = (self.table.gather(1, p // self.page).long() * self.page + p % self.page).to(torch.int32).reshape(-1)
        kc, vc, ks, vs = self.cache
        q = cf.cache_write(k, v, slots, kc, vc, ks, vs, q=q, pos=pos.reshape(-1), freq=self.freq)
        o = cf.attention_paged(q.view(B, n, self.H, self.d).transpose(1, 2), kc, vc, self.table, lens, ks, vs, causal=n > 1)
        o = o.transpose(1, 2).reshape(B * n, D)
        return cf.gemm_w4(o, *self.wo, code="e2m1").view(B, n, D), q, o


@gpu
@pytest.mark.parametrize("code", ["bf16", "int8", "e4m3"])
def test_decoding_step(code):
    """Tokens by ones and by threes: each operator's output from the one before it; and the pages read back give the same through
    attention_prefix."""
    g = gen(8)
    step = Step(g, 3, 8, 2, 64, code, 16, 4)
    at = 0
    for n in (3, 1, 1, 16, 1, 3, 30):
        x = torch.randn((3, n, 512), generator=g, device="cuda").to(BF16)
        pos = torch.arange(at, at + n, dtype=torch.int32, device="cuda").expand(3, n).contiguous()
        at += n
        lens = torch.full((3,), at, dtype=torch.int32, device="cuda")
        y, q, o = step(x, pos, lens)
        Q, O = q.view(3, n, 8, 64).transpose(1, 2), o.view(3, n, 8, 64).transpose(1, 2)
        check_paged(O, Q, step.cache, code, step.table, lens, 16, n > 1)
        K, V = cf.cache_read(step.cache[0], step.cache[1], step.table, lens, step.cache[2], step.cache[3])
        none = torch.zeros((2, 0, 64), dtype=BF16, device="cuda")
        other = cf.attention_prefix(Q.contiguous(), none, none, K, V, lens, causal=n > 1)
        # the rows read back are rounded to bf16 (scores by 2^-8 |q| |k| scale, values by 2^-8), the outputs once each
        size = float(V[:, :, :at].float().abs().max())
        e = 0 if code == "bf16" else 2.0 ** -8 * (1 + 2 * float(Q.float().norm(dim=-1).max() * K[:, :, :at].float().norm(dim=-1).max()) / 8)
        assert float((O.float() - other.float()).abs().max()) <= (4 * 2.0 ** -8 + e) * size
    assert y.shape == (3, 30, 512) and bool(torch.isfinite(y).all())


@gpu
def test_decoding_step_captured():
    """A captured step replayed, with eager calls between the replays: positions, lengths and tokens change in place."""
    g = gen(9)
    mine, twin = Step(gen(9), 2, 8, 2, 128, "int8", 32, 40), Step(gen(9), 2, 8, 2, 128, "int8", 32, 40)
    for s in (mine, twin):   # a long past
        for t, u in zip(s.cache, fill_pages(gen(10), 80, 2, 32, 128, "int8")):
            t.copy_(u)
    x, pos = torch.zeros((2, 1, 1024), dtype=BF16, device="cuda"), torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    lens = torch.zeros((2,), dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        mine(x, pos, lens + 1)
    torch.cuda.current_stream().wait_stream(s)
    for t, u in zip(mine.cache, twin.cache):
        t.copy_(u)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = mine(x, pos, lens)[0]
    for n in (1200, 1, 600, 1201, 33):
        x.copy_(torch.randn((2, 1, 1024), generator=g, device="cuda"))
        pos.copy_(torch.tensor([[n - 1], [n // 2]]))
        lens.copy_(torch.tensor([n, n // 2 + 1]))
        graph.replay()
        want = twin(x, pos, lens)[0]
        torch.cuda.synchronize()
        assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(mine.cache, twin.cache))


# ---------------------------------------------------------------- refusals (no GPU)
A_, B_, C_, D_, E_, F_, G_, H_, I_ = (0x7F0000000000 + 0x100000 * i for i in range(9))
CACHE = dict(code_dtype=cf.CF_I8, n_pages=10, page=16, cK=A_, ck_p=2048, ck_h=1024, ck_l=64, cV=B_, cv_p=2048, cv_h=1024, cv_l=64,
             cKs=C_, cks_p=32, cks_h=16, cVs=D_, cvs_p=32, cvs_h=16)


def build(t, base, kw):
    d = dict(CACHE, struct_size=cf.C.sizeof(t), **base)
    assert set(kw) <= set(d)
    d.update(kw)
    return t(*[d[f[0]] for f in t._fields_])


def write_args(**kw):
    return build(cf.CacheWriteArgs, dict(T=5, H=4, Hk=2, d=64, Q=E_, q_t=512, q_h=64, Qo=F_, qo_t=256, qo_h=64, K=G_, k_t=512, k_h=64, V=H_,
                                         v_t=512, v_h=64, slots=I_, rot=64, pairs=0, pos=I_ + 64, ldpos=5, freq=I_ + 512, n_axes=2,
                                         section0=16, section1=16, section2=0, section3=0), kw)


CACHE_REFUSALS = [
    (dict(code_dtype=cf.CF_F32), "CF_ERR_DTYPE"), (dict(page=8), "CF_ERR_UNSUPPORTED"), (dict(page=48), "CF_ERR_UNSUPPORTED"),
    (dict(page=2048), "CF_ERR_UNSUPPORTED"), (dict(n_pages=0), "CF_ERR_SHAPE"), (dict(n_pages=1 << 27), "CF_ERR_SHAPE"),
    (dict(cK=None), "CF_ERR_NULL"), (dict(cVs=None), "CF_ERR_NULL"), (dict(cV=B_ + 8), "CF_ERR_ALIGN"), (dict(ck_l=56), "CF_ERR_LD"),
    (dict(cv_h=1032), "CF_ERR_ALIGN"), (dict(cks_h=18), "CF_ERR_ALIGN"), (dict(cKs=C_ + 4), "CF_ERR_ALIGN"), (dict(ck_l=1 << 23), "CF_ERR_LD"),
    (dict(ck_p=-2048), "CF_ERR_ALIGN"), (dict(d=96), "CF_ERR_UNSUPPORTED"), (dict(Hk=0), "CF_ERR_SHAPE"), (dict(struct_size=8), "CF_ERR_STRUCT")]


@pytest.mark.parametrize("kw,status", CACHE_REFUSALS + [
    (dict(T=-1), "CF_ERR_SHAPE"), (dict(H=-1), "CF_ERR_SHAPE"), (dict(rot=24), "CF_ERR_SHAPE"), (dict(rot=80), "CF_ERR_SHAPE"),
    (dict(pairs=2), "CF_ERR_UNSUPPORTED"), (dict(n_axes=0), "CF_ERR_SHAPE"), (dict(n_axes=5), "CF_ERR_SHAPE"), (dict(section1=15), "CF_ERR_SHAPE"),
    (dict(section0=-1, section1=33), "CF_ERR_SHAPE"), (dict(ldpos=4), "CF_ERR_LD"), (dict(Q=None), "CF_ERR_NULL"), (dict(K=None), "CF_ERR_NULL"),
    (dict(slots=None), "CF_ERR_NULL"), (dict(pos=None), "CF_ERR_NULL"), (dict(freq=None), "CF_ERR_NULL"), (dict(slots=I_ + 2), "CF_ERR_ALIGN"),
    (dict(k_t=56), "CF_ERR_LD"), (dict(qo_h=32), "CF_ERR_LD"), (dict(q_h=68), "CF_ERR_ALIGN"), (dict(ck_p=1024), "CF_ERR_LD"),
    (dict(cks_p=16), "CF_ERR_LD"), (dict(cK=G_), "CF_ERR_ALIAS"), (dict(Qo=E_), "CF_ERR_ALIAS"), (dict(Qo=G_), "CF_ERR_ALIAS"),
    (dict(cV=A_), "CF_ERR_ALIAS"), (dict(cVs=C_), "CF_ERR_ALIAS"), (dict(cV=E_), "CF_ERR_ALIAS"), (dict(cKs=I_), "CF_ERR_ALIAS")])
def test_write_refuses(kw, status):
    assert cf.STATUS[cf.cf_cache_write(write_args(**kw), None)] == status, cf.cf_last_error()


def read_args(**kw):
    return build(cf.CacheReadArgs, dict(batch=3, Hk=2, S=50, d=64, table=E_, ldt=4, pages=4, lens=F_, K=G_, k_b=6400, k_h=3200, k_l=64,
                                        V=H_, v_b=6400, v_h=3200, v_l=64), kw)


@pytest.mark.parametrize("kw,status", CACHE_REFUSALS + [
    (dict(batch=-1), "CF_ERR_SHAPE"), (dict(S=-1), "CF_ERR_SHAPE"), (dict(pages=1 << 27), "CF_ERR_SHAPE"), (dict(table=None), "CF_ERR_NULL"),
    (dict(lens=None), "CF_ERR_NULL"), (dict(lens=F_ + 2), "CF_ERR_ALIGN"), (dict(ldt=-4), "CF_ERR_LD"), (dict(K=None), "CF_ERR_NULL"),
    (dict(k_b=0), "CF_ERR_LD"), (dict(v_l=56), "CF_ERR_LD"), (dict(K=A_), "CF_ERR_ALIAS"), (dict(V=G_), "CF_ERR_ALIAS")])
def test_read_refuses(kw, status):
    assert cf.STATUS[cf.cf_cache_read(read_args(**kw), None)] == status, cf.cf_last_error()


def paged_args(**kw):
    return build(cf.AttentionPagedArgs, dict(batch=3, H=4, Hk=2, Lq=2, d=64, Q=E_, q_b=512, q_h=64, q_l=256, table=F_, ldt=4, pages=4, lens=G_,
                                             causal=1, scale=0.125, softcap=0.0, O=H_, o_b=512, o_h=64, o_l=256), kw)


@pytest.mark.parametrize("kw,status", CACHE_REFUSALS + [
    (dict(batch=-1), "CF_ERR_SHAPE"), (dict(batch=65535, H=512, Lq=64), "CF_ERR_SHAPE"), (dict(H=5), "CF_ERR_SHAPE"), (dict(Lq=65), "CF_ERR_UNSUPPORTED"),
    (dict(pages=-1), "CF_ERR_SHAPE"), (dict(causal=2), "CF_ERR_UNSUPPORTED"), (dict(scale=0.0), "CF_ERR_SHAPE"),
    (dict(scale=math.nan), "CF_ERR_SHAPE"), (dict(softcap=-1.0), "CF_ERR_SHAPE"), (dict(softcap=math.inf), "CF_ERR_SHAPE"),
    (dict(scale=3e38), "CF_ERR_SHAPE"), (dict(softcap=1e-44), "CF_ERR_SHAPE"), (dict(softcap=2e38), "CF_ERR_SHAPE"),
    (dict(Q=None), "CF_ERR_NULL"), (dict(O=None), "CF_ERR_NULL"), (dict(table=None), "CF_ERR_NULL"), (dict(lens=None), "CF_ERR_NULL"),
    (dict(q_l=260), "CF_ERR_ALIGN"), (dict(o_b=0), "CF_ERR_LD"), (dict(O=E_), "CF_ERR_ALIAS"), (dict(O=A_), "CF_ERR_ALIAS"),
    (dict(O=D_), "CF_ERR_ALIAS"), (dict(O=G_), "CF_ERR_ALIAS")])
def test_paged_refuses(kw, status):
    assert cf.STATUS[cf.cf_attention_paged(paged_args(**kw), None, 0, None)] == status, cf.cf_last_error()


def test_paged_grid_limit():
    """One (sequence, key head) a workgroup: as many as a grid has no room for."""
    at = dict(H=1024, Hk=1024, Lq=1, q_h=64, q_l=64, q_b=65536, o_h=64, o_l=64, o_b=65536)
    assert cf.STATUS[cf.cf_attention_paged(paged_args(batch=16384, **at), None, 0, None)] == "CF_ERR_SHAPE"
    assert " 1 parts" in cf.cf_attention_paged_form(paged_args(batch=16383, **at))


def test_paged_workspace():
    long = dict(pages=4096, ldt=4096)
    need = cf.cf_attention_paged_workspace(paged_args(**long))
    assert need > cf.CF_PAGED_WS_HEADER_BYTES and "parts" in cf.cf_attention_paged_form(paged_args(**long))
    for ws, n in ((None, 0), (I_, need - 1)):
        assert cf.STATUS[cf.cf_attention_paged(paged_args(**long), ws, n, None)] == "CF_ERR_WORKSPACE"
    assert cf.STATUS[cf.cf_attention_paged(paged_args(**long), I_ + 8, need, None)] == "CF_ERR_ALIGN"
    assert cf.STATUS[cf.cf_attention_paged(paged_args(**long), E_, need, None)] == "CF_ERR_ALIAS"
    assert cf.cf_attention_paged_workspace(paged_args()) == 0      # 64 keys: one part
    assert cf.cf_attention_paged_form(paged_args(batch=0)) == ""


def test_paged_empty_calls_do_nothing():
    assert cf.cf_cache_write(write_args(T=0, Q=None, K=None, slots=None, cK=None), None) == 0
    assert cf.cf_cache_read(read_args(batch=0, table=None, K=None), None) == 0
    assert cf.cf_cache_read(read_args(S=0, K=None), None) == 0
    assert cf.cf_attention_paged(paged_args(batch=0, Q=None), None, 0, None) == 0
    assert cf.cf_attention_paged(paged_args(Lq=0, Q=None), None, 0, None) == 0


def test_paged_packed_arguments():
    for t, pack in ((cf.CacheWriteArgs, cf._CACHE_WRITE), (cf.CacheReadArgs, cf._CACHE_READ), (cf.AttentionPagedArgs, cf._PAGED)):
        v = [i + 0.5 if f is cf.C.c_float else 3 * i + 1 for i, (_, f) in enumerate(t._fields_)]
        assert bytes(t(*v)) == pack.pack(*v)


@gpu
def test_paged_helpers_refuse():
    x = torch.zeros((4, 2, 64), dtype=BF16, device="cuda")
    kc, vc, ks, vs = cf.cache_pages(3, 2, 16, 64, "int8")
    slots, pos, freq = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros((2, 4), dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda")
    q, table, lens = torch.zeros((4, 2, 1, 64), dtype=BF16, device="cuda"), torch.zeros((4, 1), dtype=torch.int32, device="cuda"), slots
    for call in (lambda: cf.cache_write(x, x[:2], slots, kc, vc, ks, vs), lambda: cf.cache_write(x, x, slots.long(), kc, vc, ks, vs),
                 lambda: cf.cache_write(x, x, slots, kc, vc), lambda: cf.cache_write(x, x, slots, kc, vc[:2], ks, vs),
                 lambda: cf.cache_write(x, x, slots, kc, vc, ks, vs, pos=pos[0]), lambda: cf.cache_write(x, x, slots, kc, vc, ks, vs, pos=pos, freq=freq),
                 lambda: cf.cache_write(x, x, slots, kc, vc, ks, vs, out=x), lambda: cf.cache_write(x, x, slots, kc, vc, ks, vs, q=x[:3]),
                 lambda: cf.cache_write(x, x, slots, kc, vc, ks, vs, pairs="odd"), lambda: cf.cache_write(x[:, :1], x[:, :1], slots, kc, vc, ks, vs),
                 lambda: cf.cache_write(x.cpu(), x, slots, kc, vc, ks, vs), lambda: cf.cache_read(kc, vc, table.long(), lens, ks, vs),
                 lambda: cf.cache_read(kc, vc, table, lens[:2], ks, vs),
                 lambda: cf.attention_paged(q.float(), kc, vc, table, lens, ks, vs), lambda: cf.attention_paged(q, kc, vc, table, lens),
                 lambda: cf.attention_paged(q, kc, vc, table[:2], lens, ks, vs), lambda: cf.attention_paged(q, kc, vc, table, lens, ks, vs.double()),
                 lambda: cf.attention_paged(q, kc.to(BF16), vc.to(BF16), table, lens, ks, vs), lambda: cf.cache_pages(1, 1, 16, 64, "fp4")):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        cf.attention_paged(q, kc.float(), vc.float(), table, lens, ks, vs)
    with pytest.raises(cf.CfError, match="CF_ERR_ALIAS"):
        cf.cache_read(kc, vc, table, lens, ks, vs, out=(q, q))
    with pytest.raises(cf.CfError, match="CF_ERR_SHAPE"):
        cf.cache_write(x, x, slots, kc, vc, ks, vs, pos=pos, freq=freq, sections=(16, 15))
