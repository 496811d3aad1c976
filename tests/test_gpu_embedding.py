"""Embedding lookup and the gradient of its table against the definition.

The lookup is one product in fp32 and at most one rounding: equal.  The gradient of a word is a sum of n fp32 numbers in some order, a factor and, where
it is added to what is there, one more addition: off by at most (n + 2) 2^-24 of the sum of magnitudes."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda:0", torch.bfloat16, torch.float32


def tokens_of(kind, rows, words, seed=0, dtype=torch.int64):
    gen = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        t = torch.randint(0, words, (rows,), generator=gen)
    elif kind == "one":
        t = torch.full((rows,), words - 1)
    elif kind == "runs":        # long runs of few words, and the first word rare
        t = torch.randint(0, words, (rows,), generator=gen) // max(1, words // 3) * max(1, words // 3)
        t = t.clamp(max=words - 1)
    elif kind == "none":
        t = torch.full((rows,), -1)
    else:                       # "text": most words rare, some frequent, a tenth outside the table
        t = (torch.exp(torch.rand(rows, generator=gen).double() * math.log(words + 1)).long() - 1).clamp(0, words - 1)
        out = torch.rand(rows, generator=gen) < 0.1
        odd = torch.tensor([-1, words, -2 ** 31, 2 ** 31 - 1] + ([2 ** 32, 2 ** 32 + 1, -2 ** 63] if dtype is torch.int64 else []))
        t = torch.where(out, odd[torch.randint(0, len(odd), (rows,), generator=gen)], t)
    return t.to(dtype).to(DEV)


def gradient(tokens, dy, dtable, scale=1.0, accumulate=False):
    from paper_2010_02838_amd import binding as B
    ws = torch.full((B.embedding_workspace_bytes(*dy.shape[:1], *dtable.shape),), 255, dtype=torch.uint8, device=DEV)
    B.codistill_embedding_backward(tokens, dy, dtable, ws, scale, accumulate)


def check(tokens, dy, words, scale=1.0, accumulate=False, seed=0):
    width = dy.shape[1]
    there = torch.randn(words, width, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)
    got = there.clone() if accumulate else torch.full((words, width), math.nan, device=DEV)
    gradient(tokens, dy, got, scale, accumulate)
    again = there.clone() if accumulate else torch.full((words, width), math.nan, device=DEV)
    gradient(tokens, dy, again, scale, accumulate)
    assert torch.equal(got.view(torch.int32), again.view(torch.int32))      # the same bits
    t = tokens.cpu()
    real = (t >= 0) & (t < words)
    d = dy.cpu().double()[real] * scale
    want, size, n = torch.zeros(words, width, dtype=torch.float64), torch.zeros(words, width, dtype=torch.float64), torch.zeros(words, 1, dtype=torch.float64)
    want.index_add_(0, t[real].long(), d)
    size.index_add_(0, t[real].long(), d.abs())
    n.index_add_(0, t[real].long(), torch.ones(len(d), 1, dtype=torch.float64))
    got = got.cpu()
    if accumulate:
        assert torch.equal(got[n[:, 0] == 0], there.cpu()[n[:, 0] == 0])    # not touched
        want, size = want + there.cpu().double(), size + there.cpu().double().abs()
    else:
        assert (got[n[:, 0] == 0] == 0).all()
    assert ((got.double() - want).abs() <= (n + 2) * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("kind", ["uniform", "one", "runs", "none", "text"])
@pytest.mark.parametrize("rows,words,width,dtype", [
    (1, 1, 1, F32), (2, 3, 8, BF), (100, 1000, 7, BF), (511, 70000, 64, F32), (512, 300, 66, BF), (512, 20, 130, F32), (513, 300, 66, BF), (31, 5, 64, F32), (33, 40, 333, BF), (300, 64, 256, F32), (300, 1000, 513, F32), (2000, 7, 100, BF), (5000, 3000, 512, BF), (7680, 1000, 40, BF), (7681, 1000, 40, BF), (11520, 1024, 24, F32), (11521, 1024, 24, F32), (15360, 2 ** 20, 8, F32), (16384, 1024, 40, BF),
    (16385, 1023, 40, F32), (16385, 1024, 40, BF), (40000, 70000, 16, F32), (70000, 2 ** 21, 8, BF), (20000, 1, 24, F32)])
def test_gradients(rows, words, width, dtype, kind):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    dy = torch.randn(rows, width, generator=gen, device=DEV).to(dtype)
    check(tokens_of(kind, rows, words), dy, words, scale=1.5)


@pytest.mark.parametrize("rows", [500, 20000])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind", ["uniform", "one", "text"])
def test_gradients_beside_others(rows, dtype, kind):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    dy = torch.randn(rows, 136, generator=gen, device=DEV).to(dtype)
    check(tokens_of(kind, rows, 777, dtype=torch.int32), dy, 777, scale=0.3, accumulate=True)


@pytest.mark.parametrize("rows", [400, 17000])
def test_rows_that_are_not_read(rows):
    """Rows of tokens outside the table hold NaN; rows lie apart, with NaN between them; or begin inside a vector."""
    tokens = tokens_of("text", rows, 300)
    wide = torch.full((rows, 96), math.nan, device=DEV)
    for off in (0, 1, 16):
        dy = wide[:, off:off + 64]
        dy.copy_(torch.randn(rows, 64, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV))
        clean = dy.clone()
        dy[(tokens < 0) | (tokens >= 300)] = math.nan
        got, want = torch.empty(300, 64, device=DEV), torch.empty(300, 64, device=DEV)
        gradient(tokens, dy, got)
        gradient(tokens, clean, want)
        assert torch.isfinite(got).all() and ((got - want).abs() <= 1e-4 * want.abs().clamp(min=1)).all()
        wide.fill_(math.nan)


def test_no_rows():
    t, dy = torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros(0, 24, device=DEV)
    g = torch.full((50, 24), 3.0, device=DEV)
    gradient(t, dy, g, accumulate=True)
    assert (g == 3).all()
    gradient(t, dy, g)
    assert (g == 0).all()


def test_a_gradient_that_begins_inside_a_vector():
    """The table's gradient is a range of one flat buffer, as flat parameter buffers have it."""
    tokens, dy = tokens_of("text", 900, 50), torch.randn(900, 64, device=DEV)
    flat, want = torch.full((50 * 64 + 8,), 7.0, device=DEV), torch.empty(50, 64, device=DEV)
    gradient(tokens, dy, want)
    for off in (1, 2, 4):
        flat.fill_(7.0)
        gradient(tokens, dy, flat[off:off + 3200].view(50, 64))
        assert (flat[:off] == 7).all() and (flat[off + 3200:] == 7).all()
        assert ((flat[off:off + 3200].view(50, 64) - want).abs() <= 1e-4 * want.abs().clamp(min=1)).all()


@pytest.mark.parametrize("table_dtype", [BF, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,words,width,off", [(1, 1, 1, 0), (7, 3, 8, 0), (100, 50, 333, 0), (1000, 50, 512, 0), (100, 20, 64, 1), (64, 9, 64, 4), (0, 5, 16, 0), (3000, 7, 2048, 8)])
def test_lookups(table_dtype, dtype, rows, words, width, off):
    from paper_2010_02838_amd import binding as B
    table = torch.randn(words, width, device=DEV).to(table_dtype)
    for token_type in (torch.int64, torch.int32):
        tokens = tokens_of("text", rows, words, dtype=token_type)
        wide = torch.full((rows, width + 16), 7.0, dtype=dtype, device=DEV)
        B.codistill_embedding(tokens, table, wide[:, off:off + width], 1.7)
        real = (tokens >= 0) & (tokens < words)
        want = torch.where(real[:, None], table[torch.where(real, tokens, 0).long()].float() * 1.7, torch.zeros((), device=DEV)).to(dtype)
        assert torch.equal(wide[:, off:off + width], want)
        assert (wide[:, :off] == 7).all() and (wide[:, off + width:] == 7).all()


def test_against_differences():
    """The lookup is linear in its table: a difference of any step is the gradient, but for roundings (1e-6 of the sum's terms over the step's size)."""
    from paper_2010_02838_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(3)
    table, dy, tokens = torch.randn(40, 64, generator=gen, device=DEV), torch.randn(200, 64, generator=gen, device=DEV), tokens_of("text", 200, 40)
    g, y = torch.empty(40, 64, device=DEV), torch.empty(200, 64, device=DEV)
    gradient(tokens, dy, g, 2.5)

    def value(t):
        B.codistill_embedding(tokens, t, y, 2.5)
        return float((dy.double() * y.double()).sum())

    d = torch.randn(40, 64, generator=gen, device=DEV)
    got, want = (value(table + d) - value(table - d)) / 2, float((g.double() * d.double()).sum())
    assert abs(got - want) <= 1e-5 * float((dy.double() * y.double()).norm())


def test_tables_beyond_32_bits():
    """A table of 2.3e9 elements: words, rows and zeros behind 2^31 elements."""
    from paper_2010_02838_amd import binding as B
    words, width = 2 ** 21 + 2 ** 17, 1024
    table = torch.zeros(words, width, dtype=BF, device=DEV)
    tokens = torch.tensor([words - 1, 0, words - 2, 2 ** 21, words - 1], device=DEV).repeat(200)
    table[tokens] = torch.randn(5, width, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).bfloat16().repeat(200, 1)
    y = torch.empty(1000, width, dtype=BF, device=DEV)
    B.codistill_embedding(tokens, table, y)
    assert torch.equal(y, table[tokens])
    g = torch.full((words, width), math.nan, device=DEV)
    gradient(tokens, y, g)
    for w, n in ((words - 1, 400), (0, 200), (words - 2, 200), (2 ** 21, 200)):
        assert torch.equal(g[w], y[tokens == w].double().sum(0).float()) or ((g[w] - y[tokens == w].double().sum(0)).abs() <= n * 2.0 ** -24 * y[tokens == w].double().abs().sum(0)).all()
    g[torch.tensor([words - 1, 0, words - 2, 2 ** 21], device=DEV)] = 0
    for part in g.split(1 << 17):
        assert (part == 0).all()


@pytest.mark.parametrize("rows,words,width,dtype", [(300, 40, 66, BF), (8192, 300, 1024, BF), (6000, 500, 516, BF), (5000, 9, 1024, F32), (20000, 300, 520, BF)])
def test_the_same_bits_wherever_tensors_lie(rows, words, width, dtype):
    """Rows or a gradient that begin inside a vector, or rows whose stride is none, are added up element by element, in the same order: that follows from the tokens, the width and
    the type."""
    gen = torch.Generator(device=DEV).manual_seed(rows)
    dy, tokens = torch.randn(rows, width, generator=gen, device=DEV).to(dtype), tokens_of("text", rows, words)
    want = torch.empty(words, width, device=DEV)
    gradient(tokens, dy, want, 0.7)
    flat, flat_g = torch.zeros(rows * width + 8, dtype=dtype, device=DEV), torch.empty(words * width + 8, device=DEV)
    apart = torch.zeros(rows, width + 1, dtype=dtype, device=DEV)[:, :width]
    apart.copy_(dy)
    for off, off_g in ((1, 0), (0, 1), (3, 2), (4, 4)):
        moved, got = flat[off:off + rows * width].view(rows, width), flat_g[off_g:off_g + words * width].view(words, width)
        moved.copy_(dy)
        gradient(tokens, moved, got, 0.7)
        assert torch.equal(got, want), (off, off_g)
    gradient(tokens, apart, flat_g[:words * width].view(words, width), 0.7)
    assert torch.equal(flat_g[:words * width].view(words, width), want)


@pytest.mark.parametrize("token_type", [torch.int64, torch.int32])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,words,width", [(1, 1, 1), (300, 40, 66), (2000, 7, 100), (5000, 3000, 512), (20000, 70000, 24)])
def test_tokens_as_an_index(rows, words, width, dtype, token_type):
    """Tokens below zero count from the table's end; one that is no index gives a row of NaN, and its row of dy is not read."""
    from paper_2010_02838_amd import binding as B
    gen = torch.Generator().manual_seed(rows)
    words_of_rows = torch.randint(0, words, (rows,), generator=gen)
    tokens = torch.where(torch.rand(rows, generator=gen) < 0.5, words_of_rows - words, words_of_rows)
    lost = torch.rand(rows, generator=gen) < (0.1 if rows > 1 else 0.0)
    odd = torch.tensor([-words - 1, words, -2 ** 31, 2 ** 31 - 1] + ([2 ** 32, 2 ** 32 + 1, -2 ** 32 - 1, -2 ** 63, 2 ** 63 - 1] if token_type is torch.int64 else []))
    tokens = torch.where(lost, odd[torch.randint(0, len(odd), (rows,), generator=gen)], tokens).to(token_type).to(DEV)
    plain, lost = words_of_rows.to(DEV), lost.to(DEV)
    table = torch.randn(words, width, device=DEV).to(dtype)
    y, want = (torch.full((rows, width), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    B.codistill_embedding(tokens, table, y, 1.7, index=True)
    B.codistill_embedding(plain, table, want, 1.7)
    assert torch.equal(y[~lost], want[~lost]) and torch.isnan(y[lost]).all()
    dy = torch.randn(rows, width, device=DEV).to(dtype)
    want, got = torch.empty(words, width, device=DEV), torch.full((words, width), math.nan, device=DEV)
    gradient(torch.where(lost, -1, plain), dy, want, 0.7)
    dy[lost] = math.nan
    ws = torch.full((B.embedding_workspace_bytes(rows, words, width),), 255, dtype=torch.uint8, device=DEV)
    B.codistill_embedding_backward(tokens, dy, got, ws, 0.7, index=True)
    assert torch.equal(got, want)


# ---- whole numbers, whose sums are exact in any order: a row lost or met twice shows, however many a word has ---------------------------

def whole_numbers(rows, width, dtype, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-8, 9, (rows, width), generator=gen, device=DEV, dtype=torch.int8).to(dtype)


def check_exactly(tokens, dy, words, accumulate=False, off=0):
    """rows times 8 stay below 2^24; the factor is a power of two.  off: the gradient begins so many elements inside a vector."""
    width = dy.shape[1]
    assert len(tokens) * 8 + 100 < 2 ** 24
    flat = torch.full((words * width + 4,), 7.0 if accumulate else math.nan, device=DEV)
    got = flat[off:off + words * width].view(words, width)
    gradient(tokens, dy, got, 0.5, accumulate)
    real = (tokens >= 0) & (tokens < words)
    want = torch.full((words, width), 14.0 if accumulate else 0.0, device=DEV)
    want.index_add_(0, tokens[real].long(), dy[real].float())
    assert torch.equal(got, want * 0.5)


STREAM = 64 << 20     # bytes of rows, or of the gradient, from which on they bypass the caches


@pytest.mark.parametrize("kind", ["uniform", "one", "runs", "text"])
@pytest.mark.parametrize("rows,words,width,dtype", [
    (32767, 3000, 1024, BF), (32768, 3000, 1024, BF), (33001, 9, 1032, BF), (40000, 300, 1028, BF), (16383, 3000, 1024, F32), (16384, 3000, 1024, F32), (20001, 70, 1028, F32), (17000, 300, 1031, F32)])
def test_gradients_of_large_rows(rows, words, width, dtype, kind):
    """Around 64 MiB of rows, in runs of 8, of 4 and single."""
    check_exactly(tokens_of(kind, rows, words), whole_numbers(rows, width, dtype), words)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", ["uniform", "one", "runs", "text"])
@pytest.mark.parametrize("rows,words,width,dtype", [(130000, 500, 64, BF), (200000, 70000, 40, BF), (262144, 9, 24, F32), (262145, 1024, 7, BF), (300000, 2000, 64, F32), (600000, 5000, 16, BF), (600001, 2 ** 20, 8, F32)])
def test_gradients_of_many_rows(rows, words, width, dtype, kind, accumulate):
    """16, 32 and 64 rows a wave; chunks of the sort of 1024 rows, 1536 and 2560."""
    check_exactly(tokens_of(kind, rows, words), whole_numbers(rows, width, dtype), words, accumulate)


@pytest.mark.parametrize("rows", [5, 500, 900, 20000])
@pytest.mark.parametrize("off", [0, 1])
def test_zeros_of_large_gradients(rows, off):
    """Gradients just below 64 MiB, at it and above it, few of whose words occur: whole vectors, and single elements where they begin inside one."""
    for words, width in ((65535, 256), (65536, 256), (70001, 256), (66000, 255)):
        check_exactly(tokens_of("text", rows, words, seed=width), whole_numbers(rows, width, BF), words, off=off)


@pytest.mark.parametrize("table_dtype", [BF, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("width,pad", [(1024, 0), (1024, 8), (1028, 0), (1028, 4), (1027, 0)])
def test_lookups_of_large_rows(table_dtype, dtype, width, pad):
    """Just below 64 MiB, at it and above; rows apart, in runs of 8, of 4 and single."""
    from paper_2010_02838_amd import binding as B
    size = torch.finfo(dtype).bits // 8
    table = torch.randn(5000, width, generator=torch.Generator(device=DEV).manual_seed(width), device=DEV).to(table_dtype)
    least = -(-STREAM // (width * size))
    for rows in (least - 1, least, least + 1001):
        tokens = tokens_of("text", rows, 5000)
        wide = torch.full((rows, width + pad), 7.0, dtype=dtype, device=DEV)
        B.codistill_embedding(tokens, table, wide[:, :width], 1.7)
        real = (tokens >= 0) & (tokens < 5000)
        want = torch.where(real[:, None], table[torch.where(real, tokens, 0)].float() * 1.7, torch.zeros((), device=DEV)).to(dtype)
        assert torch.equal(wide[:, :width], want) and (wide[:, width:] == 7).all()


def test_a_vocabulary_of_four_digits():
    """2^30 words of one channel: four passes of the sort."""
    words, rows = 2 ** 30, 20000
    tokens, dy = tokens_of("text", rows, words), whole_numbers(rows, 1, F32)
    got = torch.full((words, 1), math.nan, device=DEV)
    gradient(tokens, dy, got)
    real = (tokens >= 0) & (tokens < words)
    which, at = torch.unique(tokens[real], return_inverse=True)
    assert torch.equal(got[which, 0], torch.zeros(len(which), device=DEV).index_add_(0, at, dy[real, 0]))
    got[which] = 0
    for part in got.split(1 << 28):
        assert (part == 0).all()
