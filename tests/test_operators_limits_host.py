"""What the operators of a differential-attention layer refuse at the limits of their numbers and layouts, and what they do not, without a GPU: every call
below ends in the checks in front of any launch."""
import ctypes

import pytest
import torch

from paper_2010_02838_amd import binding as B
from paper_2010_02838_amd.adamw import AdamW
from paper_2010_02838_amd.diff_lm import DiffLM
from test_operators_host import BAD, UNSUPPORTED, at, attn, backward, forward


def test_scales_of_the_gradients():
    for scale, rc in ((2.0 ** -101, UNSUPPORTED), (1e-45, UNSUPPORTED), (2.0 ** -100, B.CD_ERR_WORKSPACE_TOO_SMALL), (0.0, B.CD_ERR_WORKSPACE_TOO_SMALL)):
        assert backward(attn(scale=scale), room=0) == rc, scale


@pytest.mark.parametrize("kw", [dict(tq=0), dict(tk=0), dict(tq=0, tk=0)])
def test_packed_rows_need_the_longest_sequence(kw):
    """(A longest sequence of none would leave every row unwritten.)  Without rows there is nothing to say."""
    packed = dict(q_starts=4096, k_starts=4096, q_rows=20, k_rows=24)
    assert forward(attn(**dict(packed, **kw))) == BAD and b"longest" in B.lib.codistill_last_error()
    assert backward(attn(**dict(packed, **kw))) == BAD
    assert B.lib.codistill_diff_attention_workspace_bytes(ctypes.byref(attn(**dict(packed, **kw))), 0, ctypes.byref(ctypes.c_size_t())) == BAD
    none = dict(packed, q_rows=0 if "tq" in kw else 20, k_rows=0 if "tk" in kw else 24)
    assert B.lib.codistill_diff_attention_workspace_bytes(ctypes.byref(attn(**dict(none, **kw))), 0, ctypes.byref(ctypes.c_size_t())) == B.CD_OK


def test_tensors_without_rows_have_no_address():
    """NULL is refused for a tensor that has rows, and for no other (the workspace check behind it is what answers)."""
    small = B.CD_ERR_WORKSPACE_TOO_SMALL
    keys, queries = dict(k=None, v=None), dict(q=None, out=None, o2=None, lse=None)
    assert backward(attn(tk=0), room=0, **keys, dk=None, dv=None) == small
    assert backward(attn(), room=0, **keys, dk=None, dv=None) == BAD
    # without queries nothing is kept for them, and with few keys no workspace is needed
    assert forward(attn(tq=0), **queries) == B.CD_OK
    assert forward(attn(), **queries) == BAD
    token = dict(lambda_kind=B.CD_LAMBDA_TOKEN)
    assert forward(attn(tq=0, **token), lam=None, **queries) == B.CD_OK and forward(attn(tq=0), lam=None, **queries) == BAD
    assert backward(attn(tq=0, **token), lam=None, dlam=None, dk=None, **{k: None for k in ("q", "out", "o2", "lse", "dout", "dq", "ws")}) == BAD   # (dk has rows)
    # a workspace that is claimed and not there
    assert backward(attn(), ws=None) == BAD
    d = attn(q_starts=4096, k_starts=4096, q_rows=0, k_rows=4096, batch=1, tq=4096, tk=64)
    assert B.diff_attention_workspace_bytes(d, True) > 0 and backward(d, ws=None) == BAD


def test_sequences_that_share_memory_and_those_that_do_not():
    """q, out: 10 tokens of 512 elements, two sequences; one behind the other, the last token without its gap, time-major, and what overlaps.  (The workspace
    check behind it answers where they lie apart.)"""
    small = B.CD_ERR_WORKSPACE_TOO_SMALL
    for token, batch, ok in ((512, 5120, True), (1024, 9 * 1024 + 512, True), (1024, 9 * 1024 + 504, False), (1024, 512, True), (1536, 1024, True), (1024, 504, False),
                             (1016, 512, False), (512, 0, False), (1024, 520, False), (512, 4608, False)):
        for name in ("q", "o"):
            d = attn(**{name + "_token": token, name + "_batch": batch})
            assert backward(d, room=0) == (small if ok else BAD), (name, token, batch)
            if not ok:
                assert b"share memory" in B.lib.codistill_last_error()
                assert forward(d, q=None) == BAD
        three = attn(batch=3, q_token=token, q_batch=batch, o_batch=1 << 20, k_batch=1 << 20, v_batch=1 << 20)
        assert backward(three, room=0) == (small if ok and (batch >= 512 * 9 or token >= 512 + 2 * batch) else BAD), (token, batch)


def test_head_norm_gains_are_contiguous():
    """The kernels take gain and dgain as `width` elements in a row."""
    x, gain, dgain, ws = torch.zeros(2, 3, 8), torch.ones(8), torch.zeros(8), torch.empty(1 << 16, dtype=torch.uint8)
    wide = torch.ones(8, 2)[:, 0]
    with pytest.raises(ValueError):
        B.codistill_head_norm(x, wide, x.clone())
    for g, dg in ((wide, dgain), (gain, wide), (gain[:1].expand(8), dgain)):
        with pytest.raises(ValueError):
            B.codistill_head_norm_backward(x, g, x.clone(), x.clone(), dg, ws)


def test_adamw_grad_scale_is_one_fp32_element():
    """The kernel reads four bytes: of a bf16 or float64 factor they would be another number."""
    opt = AdamW([torch.zeros(8)], [torch.zeros(8)])
    for bad in (torch.ones(1, dtype=torch.bfloat16), torch.ones((), dtype=torch.float64), torch.ones(2), torch.ones(0)):
        with pytest.raises(ValueError):
            opt.step(1e-3, 1, grad_scale=bad)


def test_strides_of_one_token_say_nothing():
    """Single tokens: the stride of their dimension is whatever the tensor was cut from."""
    q, k, v, lam = torch.zeros(3, 1, 4, 2, 16), torch.zeros(3, 7, 2, 2, 16), torch.zeros(3, 7, 2, 32), torch.zeros(4)
    plain, cut, odd = torch.zeros(3, 1, 4, 32), torch.zeros(1, 3, 4, 32).transpose(0, 1), torch.zeros(3 * 131).as_strided((3, 1, 4, 32), (128, 131, 32, 1))
    for out in (plain, cut, odd):
        d = B.diff_attention_desc(q, k, v, out, lam)
        assert (d.o_token, d.o_batch) == (128, 128)
        p = {n: at(i + 1) for i, n in enumerate(("q", "k", "v", "lam", "out", "o2", "lse", "dout", "dq", "dk", "dv", "dlam", "ws"))}
        assert B.lib.codistill_diff_attention_backward(ctypes.byref(d), *p.values(), 0, None) == B.CD_ERR_WORKSPACE_TOO_SMALL
        for other in (plain, cut, odd):
            B._laid_out(d, (q, k, v, other, lam))
        for other in (torch.zeros(3, 1, 8, 32)[:, :, :4], torch.zeros(3, 2, 4, 32)[:, :1], plain.bfloat16()):
            with pytest.raises(ValueError):
                B._laid_out(d, (q, k, v, other, lam))


def test_tables_lie_where_the_queries_do():
    """(A table in host memory would be read by the kernels.)"""
    q, k, v, out = torch.zeros(2, 5, 4, 2, 16), torch.zeros(2, 7, 2, 2, 16), torch.zeros(2, 7, 2, 32), torch.zeros(2, 5, 4, 32)
    lam, table = torch.zeros(4), torch.zeros(3, dtype=torch.int32)
    for kw in (dict(q_lens=table[:2]), dict(k_lens=table[:2])):
        B.diff_attention_desc(q, k, v, out, lam, **kw)
        with pytest.raises(ValueError):
            B.diff_attention_desc(q, k, v, out, lam, **{n: t.to("meta") for n, t in kw.items()})
    packed = [t.flatten(0, 1) for t in (q, k, v, out)] + [lam]
    B.diff_attention_desc(*packed, q_starts=table, k_starts=table, max_q=5, max_k=7)
    for kw in (dict(q_starts=table), dict(k_starts=table), dict(q_starts=table, k_starts=table.to("meta")), dict(q_starts=table.to("meta"), k_starts=table)):
        with pytest.raises(ValueError):
            B.diff_attention_desc(*packed, **kw, max_q=5, max_k=7)


def test_number_of_heads():
    """What the keys' pass reads of a tile's rows lies up to 31 tokens of all heads apart, 48 bytes each: in 32 bits up to a million heads."""
    for heads, rc in ((65536, B.CD_OK), (65544, BAD), (1500000, BAD)):
        wide = dict(heads=heads, kv_heads=heads, head_dim=8, batch=1, **{n + "_token": 16 * heads for n in ("q", "k", "v", "o")})
        assert B.lib.codistill_diff_attention_workspace_bytes(ctypes.byref(attn(**wide)), 1, ctypes.byref(ctypes.c_size_t())) == rc, heads


def test_decoder_without_room():
    """A token more than the caches hold is refused on the host, in front of any launch."""
    lm = DiffLM(8, layers=1, heads=2, kv_heads=1, head_dim=8, device="cpu")
    decoder = lm.decoder(2, 3)
    decoder.lens[1] = 3
    decoder.oldest = 3
    with pytest.raises(ValueError, match="room of 3"):
        decoder.step(torch.zeros(2, dtype=torch.int64))
    assert decoder.lens.tolist() == [0, 3] and not decoder.k[0].any()


def test_width_of_the_residual_stream():
    """It is normed in one group, of at most 1024 channels: wider models are refused where they are made, or given a width that their heads do not have."""
    assert B.HEAD_NORM_MAX_WIDTH == 1024 and B.head_norm_workspace_bytes(1, 1, 1024) > 0
    for kw in (dict(heads=16, head_dim=64), dict(heads=16, head_dim=64, width=1032), dict(width=-8)):
        with pytest.raises(ValueError, match="width"):
            DiffLM(8, layers=1, device="cpu", **kw)
    lm = DiffLM(8, layers=1, heads=16, kv_heads=4, head_dim=64, device="cpu", width=1024)
    assert lm.w["qkv0"].shape == (2 * 64 * (16 + 2 * 4), 1024) and lm.w["out0"].shape == (1024, 2048)
