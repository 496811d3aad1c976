"""What norm with rotation, the embedding and the 8-bit cache refuse, looked at without a GPU: every call below fails in the checks in front of any launch (or has
nothing to do).  The pointers are never read."""
import ctypes

import pytest
import torch

from paper_2010_02838_amd import binding as B
from paper_2010_02838_amd.kv_cache import KVCache

BAD, UNSUPPORTED, SMALL, OK = B.CD_ERR_INVALID_ARG, B.CD_ERR_UNSUPPORTED, B.CD_ERR_WORKSPACE_TOO_SMALL, B.CD_OK
M = 1 << 20


def rope(**kw):
    d = B.rotary_desc(64, (20,), 1e4, torch.float32)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def nr(**kw):
    d = dict(x=M, gain=2 * M, y=3 * M, dy=4 * M, dx=5 * M, dgain=6 * M, heads=2, x_token=128, y_token=128, dy_token=128, dx_token=128)
    d.update(kw)
    return (B.NormRotaryTensor * 5)(*[B.NormRotaryTensor(**d) for _ in range(5)])


def forward(desc=None, positions=7 * M, tokens=4, tensors=None, n=1, eps=1e-5):
    return B.lib.codistill_norm_rotary(desc if desc is not None else rope(), positions, tokens, tensors if tensors is not None else nr(), n, eps, None)


def backward(desc=None, positions=7 * M, tokens=4, tensors=None, n=1, eps=1e-5, ws=8 * M, room=1 << 30):
    return B.lib.codistill_norm_rotary_backward(desc if desc is not None else rope(), positions, tokens, tensors if tensors is not None else nr(), n, eps, ws, room, None)


def test_norm_rotary():
    for call in (forward, backward):
        assert call(positions=None) == BAD and call(tokens=-1) == BAD and call(n=0) == BAD and call(n=5) == BAD and call(eps=-1.0) == BAD
        assert call(eps=float("nan")) == BAD and call(eps=float("inf")) == BAD and call(positions=7 * M + 2) == BAD
        for field, bad in (("dtype", 3), ("dim", 63), ("dim", 258), ("dim", 0), ("n_pairs", 33), ("n_pairs", -1), ("layout", 2), ("axes", 0)):
            assert call(desc=rope(**{field: bad})) == BAD, field
        d = rope()
        d.freq[3] = float("inf")
        assert call(desc=d) == BAD
        for field, bad in (("x", None), ("x", M + 2), ("gain", 2 * M + 1), ("heads", 0), ("heads", 65537), ("x_token", 127)):
            assert call(tensors=nr(**{field: bad})) == BAD, field
    assert forward(tensors=nr(y=None)) == BAD and forward(tensors=nr(y_token=1)) == BAD and forward(tensors=nr(y=3 * M + 1)) == BAD
    for field, bad in (("dy", None), ("dx", None), ("dgain", None), ("gain", None), ("dy_token", 1), ("dx_token", 1), ("dgain", 6 * M + 2), ("dy", 4 * M + 2)):
        assert backward(tensors=nr(**{field: bad})) == BAD, field
    need = B.norm_rotary_workspace_bytes(rope(), 4, 1)
    assert backward(room=need - 1) == SMALL and backward(ws=None) == BAD and backward(ws=8 * M + 4) == BAD
    assert forward(tokens=0, positions=None, tensors=nr(x=None, y=None)) == OK       # nothing to do
    assert B.lib.codistill_norm_rotary_workspace_bytes(rope(dim=3), 4, 1, ctypes.byref(ctypes.c_size_t())) == BAD
    assert B.lib.codistill_norm_rotary_workspace_bytes(rope(), 4, 1, None) == BAD


def test_norm_rotary_binding():
    d, pos = rope(), torch.zeros(1, 4, dtype=torch.int32)
    x, g = torch.zeros(4, 2, 64), torch.zeros(64)
    for p, t in ((pos.long(), [(x, g, x)]), (pos[:, :3], [(x, g, x)]), (pos, [(x, g, x[:, :1])]), (pos, [(x.bfloat16(), g, x)]), (pos, [(x, g[:32], x)]),
                 (pos, [(x, g.double(), x)]), (pos, [(x, torch.zeros(128)[::2], x)]), (pos, [(x.transpose(0, 1), g, x)]), (pos, []), (pos, [(x, g, x)] * 5),
                 (pos, [(torch.zeros(4, 64, 2).transpose(1, 2), g, x)]), (pos, [(torch.zeros(4, 128), g, x)])):
        with pytest.raises(ValueError):
            B.codistill_norm_rotary(d, p, t)
    for t in ((x, g, x, x, torch.zeros(32)), (x, g, x, x, g.double()), (x, g, x[:3], x, torch.zeros(64)), (x, g, x, x.bfloat16(), torch.zeros(64))):
        with pytest.raises(ValueError):
            B.codistill_norm_rotary_backward(d, pos, [t], torch.zeros(1 << 20, dtype=torch.uint8))


def emb(**kw):
    d = dict(table_dtype=B.CD_BF16, row_dtype=B.CD_F32, token_bytes=8, scale=1.0, rows=1000, vocabulary=100, width=64, row_stride=64)
    d.update(kw)
    return B.Embedding(**d)


def test_embedding():
    f = lambda d, tokens=M, table=2 * M, y=3 * M: B.lib.codistill_embedding(d, tokens, table, y, None)   # noqa: E731
    b = lambda d, tokens=M, dy=2 * M, dt=3 * M, acc=0, ws=4 * M, room=1 << 40: B.lib.codistill_embedding_backward(d, tokens, dy, dt, acc, ws, room, None)   # noqa: E731
    for kw in (dict(table_dtype=2), dict(row_dtype=-1), dict(token_bytes=2), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(vocabulary=0), dict(vocabulary=(1 << 31) - 1),
               dict(width=0), dict(width=65537), dict(row_stride=63), dict(row_stride=1 << 33), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert f(emb(**kw)) == BAD and b(emb(**kw)) == BAD, kw
        assert B.lib.codistill_embedding_workspace_bytes(emb(**kw), ctypes.byref(ctypes.c_size_t())) == BAD
    wide = emb(rows=1 << 30, width=2048, row_stride=2048)
    assert f(wide) == UNSUPPORTED and b(wide) == UNSUPPORTED
    for kw in (dict(tokens=None), dict(table=None), dict(y=None), dict(tokens=M + 4), dict(table=2 * M + 1), dict(y=3 * M + 2)):
        assert f(emb(), **kw) == BAD, kw
    for kw in (dict(tokens=None), dict(dy=None), dict(dt=None), dict(ws=None), dict(tokens=M + 4), dict(dy=2 * M + 2), dict(dt=3 * M + 2), dict(ws=4 * M + 8)):
        assert b(emb(), **kw) == BAD, kw
    n = ctypes.c_size_t()
    assert B.lib.codistill_embedding_workspace_bytes(emb(), ctypes.byref(n)) == OK and b(emb(), room=n.value - 1) == SMALL
    assert B.lib.codistill_embedding_workspace_bytes(emb(), None) == BAD and B.lib.codistill_embedding(None, M, M, M, None) == BAD
    none = emb(rows=0)
    assert f(none, tokens=None, y=None) == OK and b(none, tokens=None, dy=None, ws=None, acc=1) == OK     # nothing to do
    t, table, y = torch.zeros(4, dtype=torch.int64), torch.zeros(9, 8), torch.zeros(4, 8)
    for args in ((t.float(), table, y), (t[None], table, y), (t, table, y[:3]), (t, table[:, :4], y), (t, table.t(), y), (t, table, torch.zeros(8, 4).t())):
        with pytest.raises(ValueError):
            B.codistill_embedding(*args)
    with pytest.raises(TypeError):
        B.codistill_embedding(t, table.double(), y)
    for args in ((t, y, table.double()), (t, y, table.bfloat16()), (t, y, table[:, :4]), (t, y[:3], table)):
        with pytest.raises(ValueError):
            B.codistill_embedding_backward(*args, torch.zeros(1 << 20, dtype=torch.uint8))


def cache(**kw):
    d = dict(dtype=B.CD_BF16, sequences=2, seq_pages=3, page_tokens=64, kv_heads=2, head_dim=64, pages=6, k=M, v=2 * M, scales=3 * M, table=4 * M)
    d.update(kw)
    return B.KvCache(**d)


def rows(**kw):
    d = dict(max_new=5, rows=0, k_token=256, k_batch=256 * 5, v_token=256, v_batch=256 * 5, first=None, counts=None, starts=None)
    d.update(kw)
    return B.KvRows(**d)


def attn(**kw):
    d = dict(tq=3, heads=4, causal=1, lambda_kind=B.CD_LAMBDA_HEAD, scale=0.0, q_token=512, q_batch=512 * 3, o_token=512, o_batch=512 * 3, q_lens=None, k_lens=9 * M)
    d.update(kw)
    return B.KvAttn(**d)


def attend(c=None, d=None, q=5 * M, lam=6 * M, out=7 * M, ws=8 * M, room=1 << 40):
    return B.lib.codistill_kv_diff_attention(c if c is not None else cache(), d if d is not None else attn(), q, lam, out, ws, room, None)


BAD_CACHES = [(dict(dtype=2), BAD), (dict(sequences=0), BAD), (dict(seq_pages=0), BAD), (dict(pages=0), BAD), (dict(page_tokens=0), BAD), (dict(page_tokens=96), BAD),
              (dict(page_tokens=1 << 22), BAD), (dict(kv_heads=0), BAD), (dict(kv_heads=65537), BAD), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED),
              (dict(head_dim=136), UNSUPPORTED), (dict(seq_pages=1 << 26, pages=1 << 27), BAD), (dict(sequences=1 << 24, pages=1 << 30), BAD)]


@pytest.mark.parametrize("kw,rc", BAD_CACHES + [(dict(k=None), BAD), (dict(v=None), BAD), (dict(scales=None), BAD), (dict(k=M + 8), BAD), (dict(v=M + 8), BAD), (dict(scales=M + 2), BAD),
                                                (dict(table=M + 2), BAD), (dict(table=None, pages=5), BAD)])
def test_caches(kw, rc):
    c = cache(**kw)
    for call in (B.lib.codistill_kv_write, B.lib.codistill_kv_read):
        assert call(c, rows(), 5 * M, 6 * M, None) == rc and B.lib.codistill_last_error()
    assert attend(c) == rc
    if (kw, rc) in BAD_CACHES:
        n = [ctypes.c_size_t() for _ in range(3)]
        assert B.lib.codistill_kv_cache_bytes(c, *map(ctypes.byref, n)) == rc
        assert B.lib.codistill_kv_diff_attention_workspace_bytes(c, attn(), ctypes.byref(n[0])) == rc


def test_cache_sizes():
    n = [ctypes.c_size_t() for _ in range(3)]
    assert B.lib.codistill_kv_cache_bytes(cache(head_dim=72), *map(ctypes.byref, n)) == OK
    assert [x.value for x in n] == [6 * 2 * 64 * 2 * 96, 6 * 2 * 64 * 144, 6 * 2 * 64 * 6]
    assert B.lib.codistill_kv_cache_bytes(cache(), None, None, None) == BAD and B.lib.codistill_kv_cache_bytes(None, *map(ctypes.byref, n)) == BAD


@pytest.mark.parametrize("call", ["codistill_kv_write", "codistill_kv_read"])
def test_cache_rows(call):
    f = lambda r, k=5 * M, v=6 * M, c=None: getattr(B.lib, call)(c if c is not None else cache(), r, k, v, None)   # noqa: E731
    for kw in (dict(max_new=-1), dict(k_token=255), dict(k_token=260), dict(v_token=8), dict(v_batch=-8), dict(k_batch=257), dict(k_token=(1 << 31) + 8), dict(v_token=1 << 62), dict(k_batch=1 << 39), dict(first=4 * M + 2), dict(counts=4 * M + 1),
               dict(starts=4 * M + 2, rows=9), dict(starts=4 * M, rows=-1), dict(starts=4 * M, rows=9, counts=4 * M), dict(starts=4 * M, rows=9, max_new=0)):
        assert f(rows(**kw)) == BAD, kw
    assert f(rows(), k=None) == BAD and f(rows(), v=None) == BAD and f(rows(), k=5 * M + 8) == BAD and f(None) == BAD
    assert f(rows(max_new=0), k=None, v=None) == OK and f(rows(starts=4 * M, rows=0), k=None, v=None) == OK        # nothing to do
    if call == "codistill_kv_read":   # sequences whose rows lie in one another
        for kw in (dict(k_batch=0), dict(v_batch=256), dict(k_batch=256 * 4)):
            assert f(rows(**kw)) == BAD and b"share memory" in B.lib.codistill_last_error()


def test_cache_attention():
    for kw in (dict(tq=-1), dict(heads=3), dict(heads=0), dict(heads=1 << 17), dict(lambda_kind=2), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(q_token=511), dict(q_token=516), dict(o_token=8), dict(o_batch=512), dict(q_batch=-8), dict(q_batch=1537), dict(o_batch=0), dict(q_token=1 << 62), dict(o_token=1 << 32), dict(o_batch=1 << 62), dict(q_batch=1 << 39), dict(q_lens=M + 2), dict(k_lens=M + 1),
               dict(k_lens=None), dict(tq=1 << 23, o_batch=1 << 40)):
        assert attend(d=attn(**kw)) == BAD and B.lib.codistill_last_error(), kw
    for kw in (dict(q=None), dict(lam=None), dict(out=None), dict(q=M + 8), dict(out=M + 8), dict(lam=M + 2), dict(ws=M + 8)):
        assert attend(**kw) == BAD, kw
    long = cache(sequences=1, seq_pages=64, page_tokens=1024, pages=64)
    n = ctypes.c_size_t()
    assert B.lib.codistill_kv_diff_attention_workspace_bytes(long, attn(), ctypes.byref(n)) == OK and n.value > 0
    assert attend(long, room=n.value - 1) == SMALL and attend(long, ws=None) == SMALL
    assert B.lib.codistill_kv_diff_attention_workspace_bytes(long, attn(), None) == BAD
    assert attend(d=attn(tq=0), q=None, out=None) == OK      # nothing to do


def test_cache_class():
    make = lambda **kw: KVCache(**dict(dict(sequences=2, room=100, kv_heads=2, head_dim=16, dtype=torch.float32, page_tokens=64, device="cpu"), **kw))   # noqa: E731
    c = make()
    assert (c.room, c.pages, tuple(c.k.shape), tuple(c.v.shape), tuple(c.scales.shape)) == (128, 4, (4, 2, 64, 2, 32), (4, 2, 32, 64), (4, 2, 3, 64))
    for kw in (dict(page_tokens=32), dict(page_tokens=100), dict(table=torch.zeros(2, 2)), dict(table=torch.zeros(3, 2, dtype=torch.int32)), dict(table=torch.zeros(2, 1, dtype=torch.int32)),
               dict(buffers=(c.k, c.v[:3], c.scales)), dict(buffers=(c.k, c.v, c.scales.float()))):
        with pytest.raises(ValueError):
            make(**kw)
    with pytest.raises(TypeError):
        make(dtype=torch.float16)
    with pytest.raises(B.CodistillError):
        make(head_dim=20)
    k, v = torch.zeros(2, 3, 2, 2, 16), torch.zeros(2, 3, 2, 32)
    r = c.rows(k, v)
    assert (r.max_new, r.k_token, r.k_batch, r.v_token, r.v_batch) == (3, 64, 192, 64, 192)
    for args, kw in (((k[:1], v[:1]), {}), ((k, v[:, :2]), {}), ((k[..., :8], v), {}), ((k, v.transpose(1, 2)), {}), ((k, v), dict(first=torch.zeros(3, dtype=torch.int32))),
                     ((k, v), dict(counts=torch.zeros(2))), ((k[0], v[0]), dict(starts=torch.zeros(3, dtype=torch.int32))),
                     ((k[0], v[0]), dict(starts=torch.zeros(2, dtype=torch.int32), max_new=3))):
        with pytest.raises(ValueError):
            c.rows(*args, **kw)
    with pytest.raises(TypeError):
        c.rows(k.bfloat16(), v)
    with pytest.raises(ValueError):      # other tensors than the descriptor's
        c.write(r, k[:, :2], v[:, :2])
    q, out, lam, lens = torch.zeros(2, 3, 4, 2, 16), torch.zeros(2, 3, 4, 32), torch.zeros(4), torch.zeros(2, dtype=torch.int32)
    d = c.attention(q, out, lam, lens)
    assert (d.tq, d.heads, d.q_token, d.q_batch, d.workspace_bytes) == (3, 4, 128, 384, 0)
    for args in ((q[:1], out[:1], lam, lens), (q[..., :8], out, lam, lens), (q, out[:, :2], lam, lens), (q, out, lam[:3], lens), (q, out, lam, lens[:1]), (q, out, lam, None),
                 (q, out, lam, lens.long())):
        with pytest.raises(ValueError):
            c.attention(*args)
    for args in ((q.bfloat16(), out, lam, lens), (q, out, lam.double(), lens)):
        with pytest.raises(TypeError):
            c.attention(*args)
    with pytest.raises(ValueError):
        c.attend(d, q, lam, out[:, :2])


def test_tensors_on_the_host_are_refused():
    """The kernels would read host memory by its address."""
    d, pos, x, g = rope(), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(4, 2, 64), torch.zeros(64)
    ws, t, table = torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(4, dtype=torch.int64), torch.zeros(9, 8)
    c = KVCache(2, 100, 2, 16, torch.float32, 64, device="cpu")
    k, v, q, out = torch.zeros(2, 3, 2, 2, 16), torch.zeros(2, 3, 2, 32), torch.zeros(2, 3, 4, 2, 16), torch.zeros(2, 3, 4, 32)
    rows, lam = c.rows(k, v), torch.zeros(4)
    attn_ = c.attention(q, out, lam, torch.zeros(2, dtype=torch.int32))
    for call in (lambda: B.codistill_norm_rotary(d, pos, [(x, g, x)]), lambda: B.codistill_norm_rotary_backward(d, pos, [(x, g, x, x, g)], ws),
                 lambda: B.codistill_embedding(t, table, torch.zeros(4, 8)), lambda: B.codistill_embedding_backward(t, torch.zeros(4, 8), table, ws),
                 lambda: c.write(rows, k, v), lambda: c.read(rows, k, v), lambda: c.attend(attn_, q, lam, out)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_descriptors_of_other_caches():
    c, other = KVCache(2, 100, 2, 16, torch.float32, 64, device="cpu"), KVCache(2, 100, 1, 32, torch.float32, 64, device="cpu")
    k, v, q, out, lam = torch.zeros(2, 3, 2, 2, 16), torch.zeros(2, 3, 2, 32), torch.zeros(2, 3, 4, 2, 16), torch.zeros(2, 3, 4, 32), torch.zeros(4)
    with pytest.raises(ValueError, match="other sizes"):
        other.write(c.rows(k, v), k, v)
    with pytest.raises(ValueError, match="other sizes"):
        other.read(c.rows(k, v), k, v)
    with pytest.raises(ValueError, match="other sizes"):
        other.attend(c.attention(q, out, lam, torch.zeros(2, dtype=torch.int32)), q, lam, out)


def test_sizes_beyond_a_launch():
    """Grids of 2^32 threads and more are errors in the checks, not of the launch."""
    many = cache(sequences=1 << 12, kv_heads=1 << 12, seq_pages=1, pages=1 << 12)
    assert attend(many, attn(tq=1, heads=1 << 12, q_token=1 << 19, o_token=1 << 19, q_batch=1 << 19, o_batch=1 << 19)) == BAD
    for call in (B.lib.codistill_kv_write, B.lib.codistill_kv_read):
        assert call(many, rows(starts=4 * M, rows=9, max_new=8192, k_token=1 << 19, v_token=1 << 19), 5 * M, 6 * M, None) == BAD
        assert b"too many tiles" in B.lib.codistill_last_error()
    for kw in (dict(rows=1 << 30, width=256, row_stride=256), dict(rows=1 << 23, width=32768, row_stride=32768), dict(rows=1 << 29, width=449, row_stride=449)):
        n = ctypes.c_size_t()
        assert B.lib.codistill_embedding_workspace_bytes(emb(**kw), ctypes.byref(n)) == UNSUPPORTED
        assert B.lib.codistill_embedding(emb(**kw), M, 2 * M, 3 * M, None) == UNSUPPORTED


def test_buffers_of_a_cache_on_different_devices():
    """Only the keys' device is looked at in a call: the others would be handed to the kernels as addresses of another device's memory, or of the host's."""
    c = KVCache(2, 100, 2, 16, torch.float32, 64, device="cpu")
    for i in range(3):
        buffers = [c.k, c.v, c.scales]
        buffers[i] = buffers[i].to("meta")
        with pytest.raises(ValueError, match="device"):
            KVCache(2, 100, 2, 16, torch.float32, 64, buffers=buffers)
    table = torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        KVCache(2, 100, 2, 16, torch.float32, 64, table=table.to("meta"), buffers=(c.k, c.v, c.scales))
    assert KVCache(2, 100, 2, 16, torch.float32, 64, table=table, buffers=(c.k, c.v, c.scales)).pages == 4


def test_gradients_of_gains_that_share_memory():
    """A gain may be shared by queries and keys, its gradient's sums may not: each tensor writes its own, and one would be lost."""
    two = lambda *at: (B.NormRotaryTensor * 2)(*[B.NormRotaryTensor(x=M, gain=2 * M, dy=4 * M, dx=5 * M, dgain=a, heads=2, x_token=128, dy_token=128, dx_token=128) for a in at])   # noqa: E731
    for tokens in (4, 0):
        for at in ((6 * M, 6 * M), (6 * M, 6 * M + 63 * 4), (6 * M + 63 * 4, 6 * M), (6 * M, 6 * M + 4)):
            assert backward(tensors=two(*at), n=2, tokens=tokens) == BAD and b"share" in B.lib.codistill_last_error(), at
    # (64 channels apart is far enough, and without gains nothing is written: stopped by the checks behind this one)
    for at in ((6 * M, 6 * M + 64 * 4), (6 * M + 64 * 4, 6 * M)):
        assert backward(tensors=two(*at), n=2, room=0) == SMALL
    none = (B.NormRotaryTensor * 2)(*[B.NormRotaryTensor(x=M, dy=4 * M, dx=5 * M, heads=2, x_token=128, dy_token=128, dx_token=128) for _ in range(2)])
    assert backward(tensors=none, n=2, room=0) == SMALL


def test_tokens_as_an_index():
    """A flag beside the tokens' size: sizes are refused with it as they are without."""
    for size in (4, 8):
        d = emb(token_bytes=size | B.CD_TOKENS_AS_INDEX, rows=0)
        assert B.lib.codistill_embedding(d, None, M, None, None) == OK and B.lib.codistill_embedding_backward(d, None, None, M, 1, None, 0, None) == OK
    for size in (0, 2, 12, 1 << 16 | 8):
        d = emb(token_bytes=size | B.CD_TOKENS_AS_INDEX)
        assert B.lib.codistill_embedding(d, M, 2 * M, 3 * M, None) == BAD and B.lib.codistill_embedding_backward(d, M, 2 * M, 3 * M, 0, 4 * M, 1 << 40, None) == BAD
    assert B.lib.codistill_embedding(emb(token_bytes=8 | B.CD_TOKENS_AS_INDEX), M + 4, 2 * M, 3 * M, None) == BAD      # not aligned to its elements
    assert B.lib.codistill_embedding_backward(emb(token_bytes=8 | B.CD_TOKENS_AS_INDEX), M + 4, 2 * M, 3 * M, 0, 4 * M, 1 << 40, None) == BAD
