"""Buffers of a cache of keys and values in 8 bits, in pages.  Writing, reading back and the differential attention against it are the library's kernels."""
import ctypes

import torch

from . import binding as B


class KVCache:
    """Keys [kv_heads][2][head_dim] and values [kv_heads][2 head_dim] of the tokens of several sequences, as codes in 8 bits with a bf16 scale for each key and
    value; `dtype`, bf16 or fp32, is what goes in and comes out.

    room: tokens of a sequence, rounded up to whole pages of page_tokens (a multiple of 64).  Without a table every sequence has pages of its own; table: int32 [sequences,
    pages of a sequence] on the device, into a pool of `pages` pages, which the caller fills and changes as sequences come and go (an entry outside the pool is no
    page).  buffers: (k, v, scales) of an earlier cache of the same sizes, on one device with the table; new ones are not cleared, since only what was written is seen."""

    def __init__(self, sequences, room, kv_heads, head_dim, dtype, page_tokens=256, table=None, pages=None, buffers=None, device="cuda:0"):
        if dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("KVCache: bf16 or fp32")
        if page_tokens < 64 or page_tokens % 64:
            raise ValueError("KVCache: pages of a multiple of 64 tokens")
        seq_pages = -(-room // page_tokens)
        if table is not None:
            if table.dtype is not torch.int32 or table.dim() != 2 or table.shape[0] != sequences or not table.is_contiguous():
                raise ValueError("KVCache: the table is contiguous int32 [sequences, pages of a sequence]")
            if table.shape[1] < seq_pages:
                raise ValueError("KVCache: a table of %d pages a sequence for %d tokens" % (table.shape[1], room))
            seq_pages, device = table.shape[1], table.device
        self.pages = pages if pages is not None else (buffers[0].shape[0] if buffers else sequences * seq_pages)
        self.sequences, self.room, self.kv_heads, self.head_dim, self.dtype, self.table = sequences, seq_pages * page_tokens, kv_heads, head_dim, dtype, table
        self.desc = B.KvCache(B.CD_BF16 if dtype is torch.bfloat16 else B.CD_F32, sequences, seq_pages, page_tokens, kv_heads, head_dim, self.pages)
        sizes = [ctypes.c_size_t() for _ in range(3)]
        B._check(B.lib.codistill_kv_cache_bytes(self.desc, *[ctypes.byref(s) for s in sizes]))
        padded = -(-head_dim // 32) * 32
        shapes = ((self.pages, kv_heads, page_tokens, 2, padded), (self.pages, kv_heads, 2 * head_dim, page_tokens), (self.pages, kv_heads, 3, page_tokens))
        kinds = (torch.int8, torch.int8, torch.bfloat16)
        if buffers is None:
            buffers = [torch.empty(s, dtype=t, device=device) for s, t in zip(shapes, kinds)]
        for b, s, t in zip(buffers, shapes, kinds):
            if b.dtype is not t or tuple(b.shape) != s or not b.is_contiguous():
                raise ValueError("KVCache: buffers are contiguous %s" % (shapes,))
            if b.device != buffers[0].device:
                raise ValueError("KVCache: buffers on different devices, %s and %s" % (buffers[0].device, b.device))
        self.k, self.v, self.scales = buffers
        if table is not None and table.device != self.k.device:
            raise ValueError("KVCache: the table is on another device than the cache")
        self.desc.k, self.desc.v, self.desc.scales = (b.data_ptr() for b in buffers)
        if table is not None:
            self.desc.table = table.data_ptr()

    def _table(self, name, t, n):
        if t is None:
            return None
        if t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous() or t.device != self.k.device:
            raise ValueError("KVCache: %s is contiguous int32 [%d] on the cache's device" % (name, n))
        return t.data_ptr()

    def rows(self, k, v, first=None, counts=None, starts=None, max_new=None):
        """What write() and read() of rows laid out like these need to know; kept by the caller and handed to every call.

        Padded: k [sequences, new, kv_heads, 2, head_dim], v [sequences, new, kv_heads, 2 head_dim], of which counts (int32 [sequences], or None: all) are
        real.  Packed (starts int32 [sequences + 1] and the longest sequence's max_new): the same without the first dimension.  first: int32 [sequences], the position of each
        sequence's first row, or None (0).  Tokens and sequences may be strided."""
        off, heads, dim = 0 if starts is not None else 1, self.kv_heads, self.head_dim
        if starts is not None and (counts is not None or max_new is None):
            raise ValueError("KVCache: packed rows have starts and max_new, and no counts")
        if k.dim() != 4 + off or v.dim() != 3 + off or tuple(k.shape[1 + off:]) != (heads, 2, dim) or tuple(v.shape[1 + off:]) != (heads, 2 * dim) or (
                k.shape[:1 + off] != v.shape[:1 + off] or (off and k.shape[0] != self.sequences)):
            raise ValueError("KVCache: k is [.., kv_heads, 2, head_dim], v [.., kv_heads, 2 head_dim]")
        if k.dtype is not self.dtype or v.dtype is not self.dtype:
            raise TypeError("KVCache: rows of another type than the cache's")
        n = k.shape[off]
        r = B.KvRows(max_new=max_new if starts is not None else n, rows=n if starts is not None else 0)
        for name, t, inner in (("k", k, 3), ("v", v, 2)):
            s = B._inner(t, inner, "KVCache")
            # (the stride of a dimension of one element says nothing)
            setattr(r, name + "_token", s[-1] if n > 1 else heads * 2 * dim)
            setattr(r, name + "_batch", s[0] if off and self.sequences > 1 else 0)
        for name, t, m in (("first", first, self.sequences), ("counts", counts, self.sequences), ("starts", starts, self.sequences + 1)):
            setattr(r, name, self._table(name, t, m))
        r.keep = (first, counts, starts)
        r.layout, r.cache = tuple((t.shape, t.stride(), t.dtype) for t in (k, v)), self._sizes()
        return r

    def _sizes(self):
        """What a descriptor has in common with the caches that it may be used with."""
        return self.sequences, self.kv_heads, self.head_dim, self.dtype, self.k.device

    def _laid_out(self, desc, tensors):
        if desc.cache != self._sizes():
            raise ValueError("KVCache: a descriptor of a cache of other sizes")
        for t, want in zip(tensors, desc.layout):
            if (t.shape, t.stride(), t.dtype) != want and ((t.shape, t.dtype) != (want[0], want[2]) or any(
                    n > 1 and x != y for n, x, y in zip(t.shape, t.stride(), want[1]))):
                raise ValueError("KVCache: a tensor of shape %s, strides %s, %s where the descriptor has %s, %s, %s" % (
                    tuple(t.shape), t.stride(), t.dtype, tuple(want[0]), want[1], want[2]))

    def write(self, rows, k, v):
        """Rows of new tokens into the cache."""
        self._laid_out(rows, (k, v))
        B._check(B.lib.codistill_kv_write(self.desc, rows, k.data_ptr(), v.data_ptr(), B._stream_of(self.k, k, v)))

    def read(self, rows, k, v):
        """What the cache holds for these rows, as values; zeros where it has no place for them."""
        self._laid_out(rows, (k, v))
        B._check(B.lib.codistill_kv_read(self.desc, rows, k.data_ptr(), v.data_ptr(), B._stream_of(self.k, k, v)))

    def attention(self, q, out, lam, k_lens, causal=False, scale=0.0, q_lens=None):
        """What attend() of tensors laid out like these needs to know; kept by the caller, with workspace_bytes.

        q [sequences, new, heads, 2, head_dim], out [sequences, new, heads, 2 head_dim], lam fp32 [heads] or [sequences, new, heads]; k_lens int32 [sequences]: tokens in the
        cache, the new ones among them; q_lens int32 [sequences] or None."""
        if q.dim() != 5 or q.shape[0] != self.sequences or tuple(q.shape[3:]) != (2, self.head_dim) or tuple(out.shape) != tuple(q.shape[:3]) + (2 * self.head_dim,):
            raise ValueError("KVCache: q is [sequences, new, heads, 2, head_dim], out [sequences, new, heads, 2 head_dim]")
        if q.dtype is not self.dtype or out.dtype is not self.dtype or lam.dtype is not torch.float32:
            raise TypeError("KVCache: q and out have the cache's type, lambda is fp32")
        tq, heads = q.shape[1], q.shape[2]
        if tuple(lam.shape) not in ((heads,), tuple(q.shape[:3])) or not lam.is_contiguous():
            raise ValueError("KVCache: lambda is contiguous [heads] or one for each query and head")
        d = B.KvAttn(tq=tq, heads=heads, causal=int(causal), lambda_kind=B.CD_LAMBDA_HEAD if lam.dim() == 1 else B.CD_LAMBDA_TOKEN, scale=scale)
        for name, t, inner in (("q", q, 3), ("o", out, 2)):
            s = B._inner(t, inner, "KVCache")
            setattr(d, name + "_token", s[1] if tq > 1 else heads * 2 * self.head_dim)
            setattr(d, name + "_batch", s[0] if self.sequences > 1 else 0)
        if k_lens is None:
            raise ValueError("KVCache: k_lens says how many tokens the cache holds")
        d.k_lens, d.q_lens = self._table("k_lens", k_lens, self.sequences), self._table("q_lens", q_lens, self.sequences)
        d.keep = (k_lens, q_lens)
        d.layout, d.cache = tuple((t.shape, t.stride(), t.dtype) for t in (q, out, lam)), self._sizes()
        b = ctypes.c_size_t()
        B._check(B.lib.codistill_kv_diff_attention_workspace_bytes(self.desc, d, ctypes.byref(b)))
        d.workspace_bytes = b.value
        return d

    def attend(self, desc, q, lam, out, workspace=None):
        """out = (softmax(q_1 k_1) - lam softmax(q_2 k_2)) v against the first k_lens tokens of every sequence."""
        self._laid_out(desc, (q, out, lam))
        on = B._stream_of(self.k, q, lam, out) if workspace is None else B._stream_of(self.k, q, lam, out, workspace)
        B._check(B.lib.codistill_kv_diff_attention(self.desc, desc, q.data_ptr(), lam.data_ptr(), out.data_ptr(), B._ptr(workspace), B._room(workspace), on))
