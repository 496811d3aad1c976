"""What the operators of a differential-attention layer refuse, looked at without a GPU: every call below fails in the checks in front of
any launch.  The pointers are never read."""
import ctypes

import pytest
import torch

from paper_2010_02838_amd import binding as B
from paper_2010_02838_amd.adamw import AdamW

at = lambda k: ctypes.c_void_p(k << 20)   # noqa: E731
BAD, UNSUPPORTED, SMALL = B.CD_ERR_INVALID_ARG, B.CD_ERR_UNSUPPORTED, B.CD_ERR_WORKSPACE_TOO_SMALL


def attn(**kw):
    d = dict(dtype=B.CD_BF16, batch=2, tq=10, tk=12, heads=4, kv_heads=2, head_dim=64, causal=1, lambda_kind=B.CD_LAMBDA_HEAD, scale=0.0, q_token=512,
             q_batch=5120, k_token=256, k_batch=256 * 12, v_token=256, v_batch=256 * 12, o_token=512, o_batch=5120)
    d.update(kw)
    return B.DiffAttn(**d)


def forward(d, q=1, k=2, v=3, lam=4, out=5, o2=6, lse=7, ws=8, room=1 << 30):
    p = [None if x is None else x if isinstance(x, ctypes.c_void_p) else at(x) for x in (q, k, v, lam, out, o2, lse, ws)]
    return B.lib.codistill_diff_attention(ctypes.byref(d), *p, room, None)


def backward(d, room=1 << 30, **kw):
    p = {n: at(i + 1) for i, n in enumerate(("q", "k", "v", "lam", "out", "o2", "lse", "dout", "dq", "dk", "dv", "dlam", "ws"))}
    p.update(kw)
    return B.lib.codistill_diff_attention_backward(ctypes.byref(d), *p.values(), room, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(dtype=7), BAD), (dict(lambda_kind=2), BAD), (dict(batch=0), BAD), (dict(heads=3), BAD), (dict(kv_heads=0), BAD), (dict(scale=-1.0), BAD),
    (dict(scale=float("inf")), BAD), (dict(scale=float("nan")), BAD), (dict(tq=-1), BAD), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=136), UNSUPPORTED),
    (dict(head_dim=0), UNSUPPORTED), (dict(q_token=504), BAD), (dict(k_token=260), BAD), (dict(v_token=8), BAD), (dict(o_batch=5121), BAD),
    (dict(o_batch=512), BAD), (dict(k_batch=-8), BAD), (dict(q_starts=4096), BAD), (dict(q_starts=4096, k_starts=4096, k_lens=4096), BAD),
    (dict(q_starts=4098, k_starts=4096), BAD), (dict(q_starts=4096, k_starts=4096, q_rows=-1), BAD), (dict(tq=1 << 30, o_batch=1 << 41), BAD)])
def test_attention_descriptors(kw, rc):
    assert forward(attn(**kw)) == rc and B.lib.codistill_last_error()
    assert backward(attn(**kw)) == rc


@pytest.mark.parametrize("name", ["q_token", "k_token", "v_token", "o_token"])
def test_attention_token_strides(name):
    """A tile's 32 rows are addressed with 32 bits: token strides up to 2^27 bytes (refused before any pointer is looked at: nothing is launched)."""
    wide = dict(q_batch=1 << 40, k_batch=1 << 40, v_batch=1 << 40, o_batch=1 << 40)
    assert forward(attn(**{name: (1 << 26) + 8}, **wide)) == UNSUPPORTED
    assert backward(attn(**{name: (1 << 26) + 8}, **wide)) == UNSUPPORTED
    assert backward(attn(dtype=B.CD_F32, **{name: (1 << 25) + 4}, **wide)) == UNSUPPORTED
    assert forward(attn(**{name: 1 << 26}, **wide), q=None) == BAD


def test_attention_pointers_and_workspace():
    d = attn()
    for n in ("q", "k", "v", "lam", "out"):
        assert forward(d, **{n: None}) == BAD
    for n in ("q", "k", "v", "out", "o2", "lse"):
        assert forward(d, **{n: ctypes.c_void_p((1 << 20) + 8)}) == BAD
    assert forward(d, lam=ctypes.c_void_p((1 << 20) + 2)) == BAD
    assert forward(d, o2=None) == BAD and forward(d, lse=None) == BAD       # both are kept or neither
    for n in ("q", "k", "v", "lam", "out", "o2", "lse", "dout", "dq", "dk", "dv", "dlam", "ws"):
        assert backward(d, **{n: None}) == BAD
    long = attn(batch=1, tq=1, tk=8192)
    need = B.diff_attention_workspace_bytes(long, False)
    assert need > 0 and forward(long, room=need - 1) == SMALL and forward(long, ws=None) == SMALL
    assert B.diff_attention_workspace_bytes(attn(batch=64, tq=128, tk=128, o_batch=1 << 16), False) == 0
    need = B.diff_attention_workspace_bytes(d, True)
    assert need >= 2 * 4 * 20 * 4 and backward(d, room=need - 1) == SMALL
    # sequences that share keys: read, never written
    assert backward(attn(k_batch=0)) == BAD and b"share memory" in B.lib.codistill_last_error()
    assert B.lib.codistill_diff_attention_workspace_bytes(ctypes.byref(d), 0, None) == BAD
    assert B.lib.codistill_diff_attention_workspace_bytes(None, 0, ctypes.byref(ctypes.c_size_t())) == BAD


def test_attention_binding_checks_shapes():
    q, k, v, out = torch.zeros(2, 5, 4, 2, 16), torch.zeros(2, 7, 2, 2, 16), torch.zeros(2, 7, 2, 32), torch.zeros(2, 5, 4, 32)
    lam = torch.zeros(4)
    d = B.diff_attention_desc(q, k, v, out, lam)
    assert (d.batch, d.tq, d.tk, d.heads, d.kv_heads, d.head_dim, d.q_token, d.q_batch, d.v_token) == (2, 5, 7, 4, 2, 16, 128, 640, 64)
    for args in ((q, k[:, :, :1], v, out, lam), (q, k, v[..., :16], out, lam), (q, k, v, out[:, :4], lam), (q, k, v, out, torch.zeros(3)), (q[:1], k, v, out[:1], lam),
                 (q.transpose(3, 4), k, v, out, lam)):
        with pytest.raises(ValueError):
            B.diff_attention_desc(*args)
    with pytest.raises(TypeError):
        B.diff_attention_desc(q, k.bfloat16(), v, out, lam)
    with pytest.raises(TypeError):
        B.diff_attention_desc(q, k, v, out, lam.double())
    with pytest.raises(ValueError):
        B.diff_attention_desc(q, k, v, out, lam, k_lens=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):   # other tensors than the descriptor's
        B.codistill_diff_attention(d, q[:, :4], k, v, lam, out)
    with pytest.raises(ValueError):
        B.codistill_diff_attention(d, q, k, v, lam, out, torch.zeros(2, 5, 4, 32), torch.zeros(2, 4, 9))


def test_rotary():
    x = torch.zeros(4, 2, 64)
    pos = torch.zeros(1, 4, dtype=torch.int32)
    t = (B.RotaryTensor * 5)(*[B.RotaryTensor(1 << 20, 2 << 20, 2, 128, 128) for _ in range(5)])
    good = B.rotary_desc(64, (20,), 1e4, torch.float32)

    def rc(desc=good, positions=at(3), tokens=4, tensors=t, n=1):
        return B.lib.codistill_rotary(ctypes.byref(desc) if desc else None, positions, tokens, tensors, n, 0, None)

    assert rc(desc=None) == BAD and rc(positions=None) == BAD and rc(tensors=None) == BAD and rc(tokens=-1) == BAD and rc(n=0) == BAD and rc(n=5) == BAD
    assert rc(tokens=0) == B.CD_OK        # nothing to do
    for field, bad in (("dtype", 3), ("dim", 63), ("dim", 258), ("dim", 0), ("n_pairs", 33), ("n_pairs", -1), ("layout", 2), ("axes", 0)):
        d = B.rotary_desc(64, (20,), 1e4, torch.float32)
        setattr(d, field, bad)
        assert rc(desc=d) == BAD, field
    d = B.rotary_desc(64, (20,), 1e4, torch.float32)
    d.freq[3] = float("nan")
    assert rc(desc=d) == BAD
    for field, bad in (("x", None), ("y", (1 << 20) + 2), ("heads", 0), ("x_token", 127)):
        u = (B.RotaryTensor * 1)(B.RotaryTensor(1 << 20, 2 << 20, 2, 128, 128))
        setattr(u[0], field, bad)
        assert rc(tensors=u) == BAD, field
    for sections, freq in (((33,), None), ((4, 4), [1.0])):
        with pytest.raises(ValueError):
            B.rotary_desc(64, sections, 1e4, torch.float32, freq=freq)
    for p, x_, y_ in ((pos.long(), x, x), (pos, x, x[:, :1]), (pos, x[:3], x[:3]), (pos, x.bfloat16(), x.bfloat16())):
        with pytest.raises((ValueError, TypeError)):
            B.codistill_rotary(good, p, [(x_, y_)])


def test_head_norm():
    f, b = B.lib.codistill_head_norm, B.lib.codistill_head_norm_backward
    good = dict(dtype=B.CD_BF16, x=at(1), x_row=256, gain=at(2), y=at(3), y_row=256, rows=10, heads=2, width=128, eps=1e-5, post=1.0)
    for k, bad in (("dtype", 5), ("x", None), ("gain", None), ("y", None), ("x_row", 255), ("y_row", 8), ("rows", -1), ("heads", 0), ("width", 0), ("width", 1025),
                   ("eps", -1.0), ("eps", float("nan")), ("post", float("nan")), ("x", ctypes.c_void_p(4097))):
        assert f(*dict(good, **{k: bad}).values(), None) == BAD, (k, bad)
    assert f(*dict(good, rows=0).values(), None) == B.CD_OK
    need = B.head_norm_workspace_bytes(10, 2, 128)
    good = dict(dtype=B.CD_BF16, x=at(1), x_row=256, gain=at(2), dy=at(3), dy_row=256, dx=at(4), dx_row=256, dgain=at(5), rows=10, heads=2, width=128, eps=1e-5,
                post=1.0, ws=at(6), room=need)
    for k, bad in (("dy", None), ("dx", None), ("dgain", None), ("ws", None), ("dy_row", 0), ("dgain", ctypes.c_void_p(4098)), ("width", 2000)):
        assert b(*dict(good, **{k: bad}).values(), None) == BAD, k
    assert b(*dict(good, room=need - 1).values(), None) == SMALL
    assert B.lib.codistill_head_norm_workspace_bytes(1, 1, 0, ctypes.byref(ctypes.c_size_t())) == BAD
    with pytest.raises(ValueError):
        B.codistill_head_norm(torch.zeros(2, 3, 8), torch.zeros(7), torch.zeros(2, 3, 8))


def test_adamw_tables_and_steps():
    def entry(**kw):
        d = dict(w=1 << 20, grad=2 << 20, lowp=None, m=3 << 20, v=4 << 20, exps=5 << 20, m_out=None, v_out=None, n=1000, weight_decay=0.1, lr_scale=1.0)
        d.update(kw)
        return B.AdamwTensor(**d)

    for kw, bits, grads in ((dict(w=None), 32, 0), (dict(grad=None), 32, 0), (dict(m=None), 32, 0), (dict(exps=None), 8, 0), (dict(n=0), 32, 0), (dict(n=-5), 8, 0),
                            (dict(w=(1 << 20) + 4), 32, 0), (dict(grad=(2 << 20) + 8), 32, B.CD_F32), (dict(grad=(2 << 20) + 4), 32, B.CD_BF16),
                            (dict(m=(3 << 20) + 8), 32, 0), (dict(m=(3 << 20) + 2), 8, 0), (dict(lowp=(6 << 20) + 4), 32, 0), (dict(lr_scale=float("nan")), 32, 0),
                            (dict(weight_decay=float("nan")), 32, 0), ({}, 16, 0), ({}, 32, 3)):
        with pytest.raises(B.CodistillError) as e:
            B.adamw_table([entry(**kw)], bits, grads)
        assert e.value.code == BAD
    plan, host = B.adamw_table([entry(), entry(n=3)], 8, B.CD_F32)
    assert (plan.tensors, plan.elements, plan.workgroups) == (2, 1003, 2)
    arr = (B.AdamwTensor * 1)(entry())
    assert B.lib.codistill_adamw_table(arr, 1, 8, 0, B._ptr(host), 8, ctypes.byref(plan)) == SMALL
    assert B.lib.codistill_adamw_table(arr, 0, 8, 0, B._ptr(host), 1 << 20, ctypes.byref(plan)) == BAD
    step = lambda p, cfg, table=at(1): B.lib.codistill_adamw_step(ctypes.byref(p), table, ctypes.byref(cfg), None, None)   # noqa: E731
    ok = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, t=1, seed=0)
    for k, bad in (("t", 0), ("lr", float("nan")), ("beta1", 1.0), ("beta2", -0.1), ("eps", 0.0)):
        assert step(plan, B.AdamwCfg(**dict(ok, **{k: bad}))) == BAD, k
    assert step(B.AdamwPlan(), B.AdamwCfg(**ok)) == BAD and step(plan, B.AdamwCfg(**ok), None) == BAD
    assert B.lib.codistill_adamw_unpack(ctypes.byref(plan), at(1), None) == BAD      # nowhere to write
    w, g = [torch.zeros(8), torch.zeros(4)], [torch.zeros(8), torch.zeros(4)]
    for args, kw in (((w, g[:1]), {}), ((w, [torch.zeros(8), torch.zeros(5)]), {}), ((w, g), dict(weight_decay=[0.1])), ((w, g), dict(state_bits=4)), (([], []), {}),
                     ((w, g), dict(state={"m": [torch.zeros(8)] * 2, "v": [torch.zeros(8)] * 2}))):
        with pytest.raises(ValueError):
            AdamW(*args, **kw)
    with pytest.raises(TypeError):
        AdamW([t.double() for t in w], g)
