"""The 8-bit cache: codes, scales and what they stand for are exact; the attention against them, in float64.

Attention, element by element, with A = P_1 |v| + |lambda| P_2 |v| of the cache's values: scores are fp32 sums of products that are exact in pairs (each of some 6 head_dim
additions off by 2^-24 of its terms, which add up like terms of random sign: 2^-24 * 8 * the sum's size, scores up to 30 here: 2^-24 * 240), exponentials and
sums 2^-20, weights in two bf16 numbers 2^-16 (three in fp32: 2^-23), and one rounding of the result: 2^-14 A + 2^-8 |out| in bf16, 2^-15 A in fp32."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda:0", torch.bfloat16, torch.float32


def bf16_up(x):
    """The smallest bf16 number that is at least x (float64, positive)."""
    m, e = np.frexp(x)
    return np.ldexp(np.ceil(m * 256) / 256, e)


def quantised(x):
    """Codes and scales of the last dimension, from the definition (float64)."""
    top = np.abs(x).max(-1, keepdims=True)
    s = np.maximum(bf16_up(top / 127), 2.0 ** -100)
    return np.rint(x / s), s[..., 0]


def make(dtype, sequences, room, heads, dim, page=64, paged=False, pages=None, seed=0):
    from paper_2010_02838_amd.kv_cache import KVCache
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = -(-room // page)
    table = None
    if paged:
        pages = sequences * n + 3 if pages is None else pages
        table = torch.randperm(pages, generator=gen, device=DEV)[:sequences * n].int().view(sequences, n).contiguous()
    c = KVCache(sequences, room, heads, dim, dtype, page, table=table, pages=pages, device=DEV)
    # what earlier owners of the memory left: any codes, scales that are not numbers
    c.k.random_(-128, 127, generator=gen)
    c.v.random_(-128, 127, generator=gen)
    c.scales.fill_(math.nan)
    return c


def place(c, b, pos):
    """Page and slot of a position, or None."""
    P, n = c.desc.page_tokens, c.desc.seq_pages
    if not 0 <= pos < P * n:
        return None
    page = int(c.table[b, pos // P]) if c.table is not None else b * n + pos // P
    return (page, pos % P) if 0 <= page < c.pages else None


def image(c):
    return [t.cpu().clone() for t in (c.k, c.v, c.scales)]


def put(c, img, b, pos, k, v):
    """The definition, for one token: k [heads, 2, D], v [heads, 2D] float64."""
    at = place(c, b, pos)
    if at is None:
        return
    (ck, sk), (cv, sv) = quantised(k), quantised(v)
    img[0][at[0], :, at[1], :, :c.head_dim] = torch.from_numpy(ck).to(torch.int8)
    img[1][at[0], :, :, at[1]] = torch.from_numpy(cv).to(torch.int8)
    img[2][at[0], :, :2, at[1]] = torch.from_numpy(sk).to(BF)
    img[2][at[0], :, 2, at[1]] = torch.from_numpy(sv).to(BF)


def same(c, img):
    for name, got, want in zip(("k", "v", "scales"), (c.k, c.v, c.scales), img):
        got = got.cpu()
        if name == "scales":
            got, want = got.view(torch.int16), want.view(torch.int16)
        assert torch.equal(got, want), "%s differs in %d places" % (name, int((got != want).sum()))


def new_rows(dtype, shape, heads, dim, seed=1, spread=1.0):
    """Ranges of a projection's rows."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = int(np.prod(shape))
    wide = torch.randn(n, 8 * heads * dim + 16, generator=gen, device=DEV) * torch.exp(spread * torch.randn(n, 1, generator=gen, device=DEV))
    wide = wide.to(dtype)
    k = wide[:, 8:8 + 2 * heads * dim].unflatten(1, (heads, 2, dim)).unflatten(0, shape)
    v = wide[:, 8 + 4 * heads * dim:8 + 6 * heads * dim].unflatten(1, (heads, 2 * dim)).unflatten(0, shape)
    return k, v


SIZES = [(1, 8), (2, 24), (4, 64), (3, 40), (1, 128), (2, 96), (8, 32), (2, 72)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,dim", SIZES)
@pytest.mark.parametrize("new,first,paged", [(1, (0, 63, 64, 130), False), (5, (0, 61, 127, 187), True), (150, (3, 0, 41, 30), True), (64, (0, 64, 1, 63), False)])
def test_written_codes(dtype, heads, dim, new, first, paged):
    c = make(dtype, 4, 192, heads, dim, paged=paged)
    img = image(c)
    k, v = new_rows(dtype, (4, new), heads, dim)
    at = torch.tensor(first, dtype=torch.int32, device=DEV)
    rows = c.rows(k, v, first=at)
    c.write(rows, k, v)
    for b in range(4):
        for i in range(new):
            put(c, img, b, first[b] + i, k[b, i].cpu().double().numpy(), v[b, i].cpu().double().numpy())
    same(c, img)
    # read back, beside what was written before (NaN: nothing) and beyond the room (zeros)
    bk, bv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    c.read(c.rows(bk, bv, first=at), bk, bv)
    for b in range(4):
        for i in range(new):
            p = place(c, b, first[b] + i)
            if p is None:
                assert (bk[b, i] == 0).all() and (bv[b, i] == 0).all()
                continue
            s = img[2][p[0], :, :, p[1]].float()
            assert torch.equal(bk[b, i].cpu(), (img[0][p[0], :, p[1], :, :dim].float() * s[:, :2, None]).to(dtype))
            assert torch.equal(bv[b, i].cpu(), (img[1][p[0], :, :, p[1]].float() * s[:, 2:]).to(dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_packed_rows_and_counts(dtype):
    """Packed sequences with a gap in front, an empty one and one that is longer than it said; padded ones with counts; rows behind them are left alone."""
    for packed in (True, False):
        c = make(dtype, 4, 256, 2, 40, page=128, paged=True)
        img = image(c)
        first = [5, 0, 100, 190]
        at = torch.tensor(first, dtype=torch.int32, device=DEV)
        if packed:
            starts = [3, 73, 73, 80, 150]
            k, v = new_rows(dtype, (153,), 2, 40)
            kw = dict(first=at, starts=torch.tensor(starts, dtype=torch.int32, device=DEV), max_new=66)
            lists = [(b, i, starts[b] + i) for b in range(4) for i in range(min(66, starts[b + 1] - starts[b]))]
        else:
            counts = [66, -3, 7, 900]
            k, v = new_rows(dtype, (4, 70), 2, 40)
            kw = dict(first=at, counts=torch.tensor(counts, dtype=torch.int32, device=DEV))
            lists = [(b, i, (b, i)) for b in range(4) for i in range(min(70, max(0, counts[b])))]
        c.write(c.rows(k, v, **kw), k, v)
        for b, i, row in lists:
            put(c, img, b, first[b] + i, k[row].cpu().double().numpy(), v[row].cpu().double().numpy())
        same(c, img)
        bk, bv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
        c.read(c.rows(bk, bv, **kw), bk, bv)
        touched = torch.zeros(k.shape[:1 if packed else 2], dtype=torch.bool)
        for _, _, row in lists:
            touched[row] = True
        assert (bk.cpu()[~touched] == 7).all() and (bv.cpu()[~touched] == 7).all() and not (bk.cpu()[touched] == 7).all(-1).any()


def test_tables_that_hold_anything():
    """Starts and firsts of extreme values, pages outside the pool: what has no place is not written, and the rest is."""
    c = make(F32, 3, 192, 2, 32, paged=True)
    low, high = -2 ** 31, 2 ** 31 - 1
    c.table[0, 1], c.table[1, 0], c.table[2, 2] = -1, c.pages, high
    k, v = new_rows(F32, (3, 150), 2, 32)
    for first in ([0, 0, 40], [low, high, -70], [191, 192, -1], [high - 100, low + 1, -64]):
        img = image(c)
        at = torch.tensor(first, dtype=torch.int32, device=DEV)
        c.write(c.rows(k, v, first=at), k, v)
        for b in range(3):
            for i in range(150):
                put(c, img, b, first[b] + i, k[b, i].cpu().double().numpy(), v[b, i].cpu().double().numpy())
        same(c, img)
        bk, bv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
        c.read(c.rows(bk, bv, first=at), bk, bv)
        for b in range(3):
            for i in range(150):
                if place(c, b, first[b] + i) is None:
                    assert (bk[b, i] == 0).all() and (bv[b, i] == 0).all()
    img = image(c)
    k, v = new_rows(F32, (40,), 2, 32)
    for starts in ([0, low, low, low], [high, low, 0, -5], [-3, -1, 41, 30], [30, 20, 10, 0], [41, 60, 90, 200]):
        r = c.rows(k, v, starts=torch.tensor(starts, dtype=torch.int32, device=DEV), max_new=40)
        c.write(r, k, v)
        same(c, img)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_numbers_at_their_limits(dtype):
    """Zeros, numbers below the normal ones, the largest ones, elements halfway between two codes, and elements that are not finite."""
    c = make(dtype, 1, 64, 1, 64)
    k, v = torch.zeros(1, 16, 1, 2, 64, dtype=dtype, device=DEV), torch.zeros(1, 16, 1, 128, dtype=dtype, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(2)
    for i, size in enumerate((0.0, 1e-45, 1e-38, 1e-30, 2e-29, 1.0, 3e38)):
        k[0, i] = ((torch.rand(1, 2, 64, generator=gen, device=DEV) * 2 - 1) * size).to(dtype)
        v[0, i] = ((torch.rand(1, 128, generator=gen, device=DEV) * 2 - 1) * size).to(dtype)
    half = torch.arange(64, device=DEV).float() + 0.5      # scale 1: codes 0, 2, 2, 4, ..
    k[0, 7, 0, 0], k[0, 7, 0, 1], v[0, 7, 0, :64], v[0, 7, 0, 64:] = half.to(dtype), -half.to(dtype), half.to(dtype), -half.to(dtype)
    k[0, 7, 0, 0, 63] = k[0, 7, 0, 1, 63] = v[0, 7, 0, 127] = 127.0
    if dtype is F32:      # next to halfway, and a largest element a little above 127 times a bf16 number
        k[0, 8, 0, 0] = torch.nextafter(half, half + 1) * 1.0078125
        k[0, 8, 0, 1] = torch.nextafter(half, half - 1) * 1.0078125
        k[0, 8, 0, :, 63] = 127 * 1.0078125
        v[0, 8, 0] = torch.nextafter(torch.full((128,), 127.0, device=DEV), torch.full((128,), 200.0, device=DEV))
    img = image(c)
    for i in range(9):
        put(c, img, 0, i, k[0, i].cpu().double().numpy(), v[0, i].cpu().double().numpy())
    for i, bad in ((9, math.inf), (10, -math.inf), (11, math.nan)):
        k[0, i], v[0, i] = 1.0, 1.0
        k[0, i, 0, 1, 3] = bad
        v[0, i, 0, 70] = bad
        put(c, img, 0, i, np.ones((1, 2, 64)), np.ones((1, 128)))
    k[0, 12:], v[0, 12:] = 1.0, 1.0
    for i in range(12, 16):
        put(c, img, 0, i, np.ones((1, 2, 64)), np.ones((1, 128)))
    c.write(c.rows(k, v), k, v)
    for i in (9, 10, 11):      # the other key of the token is what it was
        assert torch.isnan(c.scales[0, 0, 1:, i]).all() and not torch.isnan(c.scales[0, 0, 0, i])
        img[0][0, 0, i, 1, :64], img[1][0, 0, :, i], img[2][0, 0, 1:, i] = c.k[0, 0, i, 1, :64].cpu(), c.v[0, 0, :, i].cpu(), c.scales[0, 0, 1:, i].cpu()
    same(c, img)


# ---- attention ----------------------------------------------------------------------------------------------------------------

def held(c, b, n):
    """Values of the first n tokens of a sequence, float64, and which of them have a page."""
    K, D = c.kv_heads, c.head_dim
    k, v, there = np.zeros((n, K, 2, D)), np.zeros((n, K, 2 * D)), np.zeros(n, dtype=bool)
    P = c.desc.page_tokens
    for j in range(0, n, P):
        p, m = place(c, b, j), min(P, n - j)
        if p is not None:
            ck, cv, cs = (t[p[0]].cpu().double().numpy() for t in (c.k, c.v, c.scales))
            k[j:j + m] = (ck[..., :D] * cs[:, :2].transpose(0, 2, 1)[..., None]).swapaxes(0, 1)[:m]
            v[j:j + m] = (cv * cs[:, 2:]).transpose(2, 0, 1)[:m]
            there[j:j + m] = True
    return k, v, there


def check_attention(c, q, lam, lens, out, causal, q_lens=None, scale=0.0, more=0.0):
    S, tq, H = q.shape[:3]
    G, D = H // c.kv_heads, c.head_dim
    room = c.room
    got = out.cpu().double().numpy()
    for b in range(S):
        n = min(max(int(lens[b]), 0), room)
        nq = tq if q_lens is None else min(max(int(q_lens[b]), 0), tq)
        k, v, there = held(c, b, n)
        assert (got[b, nq:] == 0).all()
        if nq == 0:
            continue
        see = there[None] & ((np.arange(n)[None] <= np.arange(nq)[:, None] + n - nq) if causal else np.ones((nq, n), dtype=bool))
        for h in range(H):
            lm = (lam[h] if lam.dim() == 1 else lam[b, :nq, h]).cpu().double().numpy().reshape(-1, 1)
            want, size = 0.0, 0.0
            for m, f in ((0, 1.0), (1, -lm)):
                s = np.where(see, (scale or D ** -0.5) * q[b, :nq, h, m].cpu().double().numpy() @ k[:, h // G, m].T, -np.inf)
                e = np.exp(s - np.where(see.any(1), s.max(1, initial=-np.inf), 0.0)[:, None])
                p = e / np.maximum(e.sum(1, keepdims=True), 1e-300)
                want = want + f * (p @ v[:, h // G])
                size = size + np.abs(f) * (p @ np.abs(v[:, h // G]))
            tol = 2.0 ** -14 * size + 2.0 ** -8 * np.abs(want) if c.dtype is BF else 2.0 ** -15 * size
            tol = tol + more * size
            off = np.abs(got[b, :nq, h] - want)
            assert (off <= tol + 1e-30).all(), "sequence %d head %d: %.2e" % (b, h, (off / (size + 1e-30)).max())


def problem(dtype, lens, tq, heads, kv_heads, dim, page=64, paged=True, lam_token=False, room=None, seed=0, spread=0.2):
    """A cache that was written token by token's rows, and queries as ranges of wider rows."""
    S, most = len(lens), max(max(lens), 1)
    room = room or most
    c = make(dtype, S, room, kv_heads, dim, page, paged, seed=seed)
    k, v = new_rows(dtype, (S, most), kv_heads, dim, seed + 1, spread)
    c.write(c.rows(k, v, counts=torch.tensor(lens, dtype=torch.int32, device=DEV)), k, v)
    gen = torch.Generator(device=DEV).manual_seed(seed + 2)
    q = torch.randn(S, tq, 2 * heads * dim + 16, generator=gen, device=DEV).to(dtype)[..., 8:-8].unflatten(2, (heads, 2, dim))
    wide = torch.full((S, tq, 2 * heads * dim + 16), 7.0, dtype=dtype, device=DEV)
    lam = 0.2 + 0.7 * torch.rand((S, tq, heads) if lam_token else (heads,), generator=gen, device=DEV)
    return c, q, wide, wide[..., 8:-8].unflatten(2, (heads, 2 * dim)), lam, torch.tensor(lens, dtype=torch.int32, device=DEV)


def attend(c, q, out, lam, lens, **kw):
    d = c.attention(q, out, lam, lens, **kw)
    ws = torch.full((d.workspace_bytes,), 255, dtype=torch.uint8, device=DEV)    # (as NaN)
    c.attend(d, q, lam, out, ws)
    return d


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 8), (4, 4, 32), (8, 2, 64), (16, 1, 24), (12, 2, 128), (9, 3, 96), (4, 2, 80), (32, 2, 40)])
@pytest.mark.parametrize("tq,causal,lam_token", [(1, True, False), (2, False, True), (5, True, True), (17, True, False)])
def test_attention(dtype, heads, kv_heads, dim, tq, causal, lam_token):
    lens = [tq, 0, 64, 63, 129, 200, max(1, tq - 1)]
    c, q, wide, out, lam, at = problem(dtype, lens, tq, heads, kv_heads, dim, lam_token=lam_token, paged=dim != 64)
    attend(c, q, out, lam, at, causal=causal)
    check_attention(c, q, lam, at, out, causal)
    assert (wide[..., :8] == 7).all() and (wide[..., -8:] == 7).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,heads,kv_heads,dim,tq,page", [([5000], 8, 1, 64, 1, 64), ([3000, 700, 0], 4, 2, 32, 2, 1024), ([2100, 1], 12, 4, 128, 3, 256), ([4000, 513], 16, 2, 96, 1, 128)])
def test_attention_in_parts(dtype, lens, heads, kv_heads, dim, tq, page):
    c, q, _, out, lam, at = problem(dtype, lens, tq, heads, kv_heads, dim, page=page, lam_token=True, room=6000)
    d = attend(c, q, out, lam, at, causal=True)
    assert d.workspace_bytes > 0
    check_attention(c, q, lam, at, out, True)
    first = out.clone()
    attend(c, q, out, lam, at, causal=True)
    assert torch.equal(first, out)


@pytest.mark.parametrize("heads,kv_heads,dim,tq", [(16, 2, 64, 2), (9, 1, 32, 1), (12, 4, 8, 7), (8, 1, 40, 5), (32, 2, 24, 1)])
@pytest.mark.parametrize("many", [False, True])
def test_two_tiles_of_rows(heads, kv_heads, dim, tq, many):
    """Nine rows and more of bf16 heads up to 64 on caches with room for 2560 blocks: a few sequences in parts, and many without."""
    lens = [tq, 700, 65] if not many else [(37 * i) % 400 for i in range(2560 // (10 * kv_heads))]
    room = 64 * (-(-2560 // (len(lens) * kv_heads)))
    c, q, wide, out, lam, at = problem(BF, lens, tq, heads, kv_heads, dim, room=room, page=64 if many else 1024, lam_token=many)
    qn = torch.tensor([tq if i % 3 else tq - 1 for i in range(len(lens))], dtype=torch.int32, device=DEV)
    d = attend(c, q, out, lam, at, causal=True, q_lens=qn)
    assert (d.workspace_bytes > 0) != many
    check_attention(c, q, lam, at, out, True, q_lens=qn)
    assert (wide[..., :8] == 7).all() and (wide[..., -8:] == 7).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_lengths_beyond_the_room_and_of_queries(dtype):
    c, q, _, out, lam, _ = problem(dtype, [128, 100, 30, 64], 4, 4, 2, 64, room=128)
    at = torch.tensor([2 ** 31 - 1, 100, -2 ** 31, 64], dtype=torch.int32, device=DEV)
    qn = torch.tensor([2, 900, 4, -1], dtype=torch.int32, device=DEV)
    attend(c, q, out, lam, at, causal=True, q_lens=qn)
    check_attention(c, q, lam, at, out, True, q_lens=qn)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_that_are_shared_or_missing(dtype):
    c, q, _, out, lam, at = problem(dtype, [300, 300, 300], 2, 4, 2, 64, page=64)
    c.table[1, :2] = c.table[0, :2]       # a common beginning
    c.table[2, 1], c.table[2, 3] = -1, c.pages
    c.table[0, 4] = 2 ** 31 - 1
    attend(c, q, out, lam, at, causal=True)
    check_attention(c, q, lam, at, out, True)
    c.table.fill_(-1)                     # no page at all: rows that see nothing
    attend(c, q, out, lam, at, causal=True)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_of_all_sizes(dtype):
    """Scores that are alike, and scores in the tens of thousands (mostly one key takes all), whose 2^-24 * 8 parts are 1e-2: weights off by twice that, 2^-5."""
    c, q, _, out, lam, at = problem(dtype, [333, 90], 1, 4, 4, 64, spread=0.0)
    for scale in (1e-6, 0.3):
        attend(c, q, out, lam, at, causal=True, scale=scale)
        check_attention(c, q, lam, at, out, True, scale=scale)
    q *= 64
    attend(c, q, out, lam, at, causal=True, scale=8.0)
    check_attention(c, q, lam, at, out, True, scale=8.0, more=2.0 ** -5)


def test_not_finite_tokens_reach_those_who_see_them():
    """A token whose key or value is not finite: rows that see it are NaN, others are what they were."""
    for dtype in (BF, F32):
        c, q, _, out, lam, at = problem(dtype, [150, 150], 3, 4, 2, 64, page=64, paged=False)
        attend(c, q, out, lam, at, causal=True)
        clean = out.clone()
        c.scales[0, 0, 1, 10] = math.nan             # sequence 0, key head 0, second key of token 10
        c.scales[5, 1, 2, 21] = math.nan             # sequence 1, key head 1, value of token 149: the last query alone sees it
        attend(c, q, out, lam, at, causal=True)
        assert torch.isnan(out[0, :, :2]).all() and torch.isnan(out[1, 2, 2:]).all()
        assert torch.equal(out[0, :, 2:], clean[0, :, 2:]) and torch.equal(out[1, :, :2], clean[1, :, :2]) and torch.equal(out[1, :2], clean[1, :2])


def test_it_is_the_attention_over_the_values_read_back():
    """codistill_diff_attention on what codistill_kv_read gives: in fp32 both hold the same keys and values (2^-15 of the sizes, twice)."""
    from paper_2010_02838_amd import binding as B
    c, q, _, out, lam, at = problem(F32, [100, 33], 3, 8, 2, 64)
    attend(c, q, out, lam, at, causal=True)
    k, v = torch.zeros(2, 100, 2, 2, 64, device=DEV), torch.zeros(2, 100, 2, 128, device=DEV)
    c.read(c.rows(k, v, counts=at), k, v)
    o, qc = torch.empty(2, 3, 8, 128, device=DEV), q.contiguous()
    d = B.diff_attention_desc(qc, k, v, o, lam, causal=True, k_lens=at)
    ws = torch.empty(B.diff_attention_workspace_bytes(d, False), dtype=torch.uint8, device=DEV)
    B.codistill_diff_attention(d, qc, k, v, lam, o, workspace=ws)
    assert (o - out).abs().max() <= 2.0 ** -14 * 2 * v.abs().max()


def test_captured_with_a_cache_that_grows():
    """Write and attend in one graph: each replay sees the lengths and rows that it finds; eager work between the replays."""
    for dtype in (BF, F32):
        c, q, _, out, lam, at = problem(dtype, [100, 1900], 1, 8, 2, 64, room=2048, page=128)
        other = make(dtype, 2, 2048, 2, 64, page=128)
        k, v = new_rows(dtype, (2, 1), 2, 64, seed=5)
        first = at.clone()
        rows, d = c.rows(k, v, first=first), c.attention(q, out, lam, at, causal=True)
        ws = torch.empty(d.workspace_bytes, dtype=torch.uint8, device=DEV)

        def step():
            first.copy_(at)
            at.add_(1)
            c.write(rows, k, v)
            c.attend(d, q, lam, out, ws)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for i in range(4):
            a, b = new_rows(dtype, (2, 1), 2, 64, seed=20 + i)
            k.copy_(a)
            v.copy_(b)
            graph.replay()
            torch.cuda.synchronize()
            check_attention(c, q, lam, at, out, True)
            eager = torch.empty_like(out)
            c.attend(c.attention(q, eager, lam, at, causal=True), q, lam, eager, torch.empty_like(ws))
            assert torch.equal(eager, out) and at.tolist() == [102 + i, 1902 + i]
            other.k.zero_()


def test_offsets_beyond_32_bits():
    """Ten million tokens of 512 bytes: the last ones lie beyond 2^31 bytes of the keys and of the values.  All others are zeros: a score of zero each."""
    from paper_2010_02838_amd.kv_cache import KVCache
    page, D = 1 << 21, 128
    c = KVCache(1, 5 * page, 1, D, F32, page, device=DEV)
    assert c.k.numel() > 2 ** 31 and c.v.numel() > 2 ** 31
    c.k.zero_()
    c.v.zero_()
    c.scales.fill_(1.0)
    k, v = new_rows(F32, (1, 70), 1, D, spread=0.0)
    at = torch.tensor([5 * page - 70], dtype=torch.int32, device=DEV)
    rows = c.rows(k, v, first=at)
    c.write(rows, k, v)
    hk, hv = torch.empty_like(k.contiguous()), torch.empty_like(v.contiguous())
    c.read(c.rows(hk, hv, first=at), hk, hv)
    (ck, sk), (cv, sv) = quantised(k[0].cpu().double().numpy()), quantised(v[0].cpu().double().numpy())
    assert np.array_equal(hk[0].cpu().double().numpy(), ck * sk[..., None]) and np.array_equal(hv[0].cpu().double().numpy(), cv * sv[..., None])
    q = 3 * torch.randn(1, 2, 2, 2, D, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    out, lam, lens = torch.empty(1, 2, 2, 2 * D, device=DEV), torch.tensor([0.5, 0.8], device=DEV), torch.tensor([5 * page], dtype=torch.int32, device=DEV)
    attend(c, q, out, lam, lens, causal=True)
    for i in range(2):
        n = 70 - 1 + i          # the first query does not see the last token
        for h in range(2):
            want, size = 0.0, 0.0
            for m, f in ((0, 1.0), (1, -float(lam[h]))):
                s = D ** -0.5 * hk[0, :n, 0, m].cpu().double().numpy() @ q[0, i, h, m].cpu().double().numpy()
                e = np.exp(s - max(s.max(), 0.0))
                p = e / (e.sum() + (5 * page - 70) * math.exp(-max(s.max(), 0.0)))
                want, size = want + f * p @ hv[0, :n, 0].cpu().double().numpy(), size + abs(f) * p @ np.abs(hv[0, :n, 0].cpu().double().numpy())
            # (a sum of ten million equal weights in chains of 1300 additions a lane: 2^-24 * 1300 more than 2^-15)
            assert (np.abs(out[0, i, h].cpu().double().numpy() - want) <= 2.0 ** -12 * size).all()


def test_on_another_stream_beside_others():
    """Two caches written and attended from on two streams at once: the same bits as one after the other."""
    sets = []
    for seed, dtype in ((1, BF), (2, F32)):
        c, q, _, out, lam, at = problem(dtype, [900, 2000], 1, 8, 2, 64, room=2048, page=256, seed=seed)
        k, v = new_rows(dtype, (2, 1), 2, 64, seed=seed)
        d = c.attention(q, out, lam, at, causal=True)
        sets.append((c, c.rows(k, v, first=at - 1), k, v, d, q, lam, out, torch.empty(d.workspace_bytes, dtype=torch.uint8, device=DEV)))

    def run(c, rows, k, v, d, q, lam, out, ws):
        for _ in range(20):
            c.write(rows, k, v)
            c.attend(d, q, lam, out, ws)

    for s in sets:
        run(*s)
    torch.cuda.synchronize()
    want = [s[7].clone() for s in sets]
    for s in sets:
        s[7].fill_(7.0)
    streams = [torch.cuda.Stream() for _ in sets]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for s, st in zip(sets, streams):
        with torch.cuda.stream(st):
            run(*s)
    torch.cuda.synchronize()
    assert all(torch.equal(s[7], w) for s, w in zip(sets, want))


def test_more_tiles_than_a_launch_has_workgroups_across():
    """4096 packed sequences of up to two tokens whose longest one may be 33000: 17 million tiles, nearly all without a row."""
    S, H, D = 4096, 8, 8
    counts = torch.arange(S, device=DEV) % 3
    starts = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    k, v = new_rows(BF, (int(starts[-1]),), H, D)
    caches = [make(BF, S, 64, H, D) for _ in range(2)]
    back = []
    for c, longest in zip(caches, (2, 33000)):
        rows = c.rows(k, v, starts=starts, max_new=longest)
        c.write(rows, k, v)
        hk, hv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
        c.read(c.rows(hk, hv, starts=starts, max_new=longest), hk, hv)
        back += [(hk, hv)]
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((caches[0].k, caches[0].v, caches[0].scales), (caches[1].k, caches[1].v, caches[1].scales)))
    assert torch.equal(back[0][0], back[1][0]) and torch.equal(back[0][1], back[1][1])
