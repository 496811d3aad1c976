"""Differential attention where its numbers or layouts are at their limits, against the formula in float64 (tolerances as in
test_gpu_diff_attention.py)."""
import math

import numpy as np
import pytest
import torch

from test_gpu_diff_attention import BF, DEV, F32, TOL, Problem, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [0.0, 1e-12, 1e-20])
def test_lambdas_near_zero_and_small_scales(dtype, scale):
    """A lambda of zero, below the normal numbers or close above them: its logarithm, and what that is over the scale, stay finite, and the other rows'
    gradients are what they were.  (Small scales: all weights are alike.  dq and dk without the floor that `check` gives them.)"""
    p = Problem(dtype, [40, 70], [40, 70], 4, 2, 64, True, True, seed=11, scale=scale)
    for i, lam in enumerate((0.0, 1e-40, -1e-40, 1e-30, -1e-30, -0.0)):
        p.lam[:, i::7] = lam
    p.want()
    p.run()
    p.check()
    for name, at, keys in (("dq", 1, False), ("dk", 2, True)):
        got = torch.cat([p.rows(getattr(p, name), b, keys).flatten() for b in range(2)])
        close(got, np.concatenate([p.ref[b][at].ravel() for b in range(2)]), TOL[dtype] * (8 if dtype is F32 else 1), name)


@pytest.mark.parametrize("dim,heads,kv_heads,keys", [(64, 8, 8, 201), (32, 8, 8, 204), (64, 8, 8, 130)])
def test_rows_of_few_keys_beside_rows_of_many(dim, heads, kv_heads, keys):
    """Causal queries that see two to five keys, in one tile of rows with queries that see more than 128: their gradient is off by two bf16 roundings (of dS and
    of dq, 1.7e-3 each as a 2-norm), 2.4e-3 together.  A delta from the kept outputs alone would be off by 5e-3."""
    nq = keys - 1
    p = Problem(BF, [nq] * 24, [keys] * 24, heads, kv_heads, dim, True, True, seed=dim)
    p.run()
    p.check()
    got = p.dq[:, :4].double().cpu().numpy()
    want = np.stack([r[1][:4] for r in p.ref])
    for i in range(4):
        err = np.linalg.norm(got[:, i] - want[:, i]) / np.linalg.norm(want[:, i])
        assert err <= 3e-3, (i + 2, err)


def test_start_tables_of_extreme_values():
    """Differences of starts that pass 32 bits (a table nobody filled): no row, and nothing is touched."""
    low = -2 ** 31
    p = Problem(F32, [20, 30], [20, 30], 2, 2, 32, False, True, packed=True, seed=8)
    for starts in ([1, low, low], [2 ** 31 - 1, low, 0], [50, low, 50], [low, low, low]):
        for t in p.desc.keep[2:]:
            t.copy_(torch.tensor(starts, dtype=torch.int32))
        for t in (p.out, p.dq, p.dk, p.dv, p.dlam):
            t.fill_(7.0)
        p.run()
        if starts[2] <= 0:
            assert all((t == 7.0).all() for t in (p.out, p.dq, p.dk, p.dv)) and not (p.dlam != 7.0).any()
        for t in (p.out, p.dq, p.dk, p.dv):
            assert torch.isfinite(t).all()


def empty_case(dtype, batch, tq, tk, packed=False):
    """Outputs that begin as 7, of sequences without queries, without keys or without either."""
    from paper_2010_02838_amd import binding as B
    H, K, D = 4, 2, 32
    lead = (lambda n: (n,)) if packed else (lambda n: (batch, n))
    gen = torch.Generator(device=DEV).manual_seed(7)
    new = lambda n, *s: torch.randn(*lead(n), *s, generator=gen, device=DEV).to(dtype)   # noqa: E731
    q, k, v, dout = new(tq, H, 2, D), new(tk, K, 2, D), new(tk, K, 2 * D), new(tq, H, 2 * D)
    out, dq, dk, dv = (torch.full_like(t, 7.0) for t in (dout, q, k, v))
    lam, dlam = torch.rand(H, generator=gen, device=DEV), torch.full((H,), 7.0, device=DEV)
    zero = torch.zeros(batch + 1, dtype=torch.int32, device=DEV)
    starts = dict(q_starts=zero, k_starts=zero, max_q=tq, max_k=tk) if packed else {}
    desc = B.diff_attention_desc(q, k, v, out, lam, **starts)
    o2, lse = torch.empty(out.shape, dtype=dtype, device=DEV), torch.empty(desc.lse_shape, device=DEV)
    ws = torch.empty(B.diff_attention_workspace_bytes(desc, True), dtype=torch.uint8, device=DEV)
    B.codistill_diff_attention(desc, q, k, v, lam, out, o2, lse, ws)
    B.codistill_diff_attention_backward(desc, q, k, v, lam, out, o2, lse, dout, dq, dk, dv, dlam, ws)
    torch.cuda.synchronize()
    return out, dq, dk, dv, dlam


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_keys_and_no_queries(dtype):
    """Empty tensors have no address.  Without keys the outputs and the queries' gradients are zero, without queries the keys' are; lambda's always."""
    for batch, tq, tk, packed in ((2, 5, 0, False), (2, 0, 5, False), (1, 0, 700, False), (2, 0, 0, False), (2, 0, 0, True)):
        for t in empty_case(dtype, batch, tq, tk, packed):
            assert not t.any(), (batch, tq, tk, packed)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_time_major_sequences(dtype):
    """[time][batch][heads ...]: sequences whose rows alternate do not share memory.  The same numbers in rows of their own give the same bits."""
    from paper_2010_02838_amd import binding as B
    T, n, H, K, D = 70, 3, 4, 2, 32
    gen = torch.Generator(device=DEV).manual_seed(3)
    lens = torch.tensor([70, 1, 33], dtype=torch.int32, device=DEV)
    lam = torch.rand(H, generator=gen, device=DEV)
    shapes = ((H, 2, D), (K, 2, D), (K, 2 * D), (H, 2 * D))
    src = [torch.randn(T, n, *s, generator=gen, device=DEV).to(dtype) for s in shapes]
    runs = []
    for lay in (lambda t: t.transpose(0, 1), lambda t: t.transpose(0, 1).contiguous()):
        q, k, v, dout = (lay(t.clone()) for t in src)
        out, dq, dk, dv = (torch.full_like(t, 7.0) for t in (dout, q, k, v))
        assert out.stride() == dout.stride() and dk.stride() == k.stride()
        o2, lse, dlam = torch.empty(n, T, H, 2 * D, dtype=dtype, device=DEV), torch.empty(2, H, n * T, device=DEV), torch.empty_like(lam)
        desc = B.diff_attention_desc(q, k, v, out, lam, causal=True, q_lens=lens, k_lens=lens)
        ws = torch.empty(B.diff_attention_workspace_bytes(desc, True), dtype=torch.uint8, device=DEV)
        B.codistill_diff_attention(desc, q, k, v, lam, out, o2, lse, ws)
        B.codistill_diff_attention_backward(desc, q, k, v, lam, out, o2, lse, dout, dq, dk, dv, dlam, ws)
        runs.append((out, dq, dk, dv, dlam))
    assert all(torch.equal(a, b) for a, b in zip(*runs)) and not (runs[0][0] == 7.0).all(-1).any()


def split(p):
    """Which passes split their work: (keys forward, keys or rows backward) have parts' sums in their workspace."""
    rows = p.H * p.rq * (48 + (4 if p.lam.dim() == 1 else 0))
    return p.B.diff_attention_workspace_bytes(p.desc, False) > 0, p.B.diff_attention_workspace_bytes(p.desc, True) > rows + 16


@pytest.mark.parametrize("dtype,q_lens,k_lens,heads,kv_heads,dim,causal,packed", [
    (BF, [1100], [1100], 2, 1, 64, True, False), (F32, [1100], [1100], 2, 1, 64, True, False), (BF, [1100, 90], [1100, 90], 2, 2, 32, True, False),
    (BF, [1100, 90], [1100, 90], 2, 1, 128, True, True), (F32, [700, 33], [1300, 50], 2, 1, 32, True, True), (F32, [600], [1200], 1, 1, 128, True, False),
    (BF, [600, 7], [1100, 1040], 4, 2, 40, False, False), (F32, [1100, 300], [600, 64], 4, 1, 64, False, True), (BF, [1500], [1300], 2, 1, 64, True, False)])
def test_many_tiles_in_parts(dtype, q_lens, k_lens, heads, kv_heads, dim, causal, packed):
    """Several tiles of rows and of keys, each pass split: under a causal mask the first tile of rows has few keys (two passes of its own) beside tiles whose keys
    are dealt out, and parts lie in front of or behind what a tile reaches."""
    p = Problem(dtype, q_lens, k_lens, heads, kv_heads, dim, causal, len(q_lens) > 1, packed=packed, seed=dim + heads, gap=5 if packed else 0)
    assert split(p) == (True, True)
    p.run()
    p.check()


def test_another_stream_computes():
    """Outputs of a second stream's own run, in tensors that held something else before."""
    p = Problem(BF, [300, 150], [300, 150], 8, 2, 64, True, False, seed=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in (p.out, p.dq, p.dk, p.dv, p.dlam):
            t.fill_(7.0)
        p.run()
    torch.cuda.current_stream().wait_stream(side)
    p.check()
