"""Differential attention, forward and backward, against the formula in float64 and against differences.

Tolerances (2-norm of the error over 2-norm of the result).  bf16: an output is rounded once, 2^-9 at most of each element, the weights that
are summed and the dS of the gradients once more, and the rounding of many terms of random sign adds up like the terms do: 3 * 2^-9.  fp32: sums
of n terms of random sign, each off by a few times 2^-24 from its exponent's argument (scores up to 10): 64 * 2^-24.  dlambda is a sum of fp32
products of exact inputs in both types: 64 * 2^-24, times what cancels, which the norm over all terms measures."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = {torch.bfloat16: 3 * 2.0 ** -9, torch.float32: 64 * 2.0 ** -24}


def reference(q, k, v, lam, dout, see, scale):
    """One sequence in float64.  q [nq, H, 2, D], k [nk, K, 2, D], v [nk, K, 2D], lam [nq, H], see [nq, nk]."""
    H, K = q.shape[1], k.shape[1]
    out, dq, dk, dv, dl, mag = np.zeros_like(dout), np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros_like(lam), np.zeros_like(lam)
    for h in range(H):
        g = h // (H // K)
        p = []
        for m in (0, 1):
            s = np.where(see, scale * q[:, h, m] @ k[:, g, m].T, -np.inf)
            e = np.exp(s - np.where(see.any(1), s.max(1, initial=-np.inf), 0.0)[:, None])
            p.append(e / np.maximum(e.sum(1, keepdims=True), 1e-300))
        l = lam[:, h:h + 1]
        out[:, h] = (p[0] - l * p[1]) @ v[:, g]
        dp = dout[:, h] @ v[:, g].T
        for m, f in ((0, 1.0), (1, -l)):
            ds = f * p[m] * (dp - (p[m] * dp).sum(1, keepdims=True))
            dq[:, h, m] = scale * ds @ k[:, g, m]
            dk[:, g, m] += scale * ds.T @ q[:, h, m]
        dv[:, g] += (p[0] - l * p[1]).T @ dout[:, h]
        dl[:, h] = -(p[1] * dp).sum(1)
        mag[:, h] = (p[1] * np.abs(dp)).sum(1)
    return out, dq, dk, dv, dl, mag


def seen(nq, nk, causal):
    return np.ones((nq, nk), dtype=bool) if not causal else np.arange(nk)[None] <= np.arange(nq)[:, None] + nk - nq


def close(got, want, tol, what, floor=0.0):
    got = np.asarray(got.double().cpu())
    err = np.linalg.norm(got - want)
    assert err <= tol * max(np.linalg.norm(want), floor), "%s: off by %.2e of %.2e" % (what, err, np.linalg.norm(want))


class Problem:
    """Padded (lens) or packed sequences, with every tensor inside a wider one so that strides are not the shape's own."""

    def __init__(self, dtype, q_lens, k_lens, heads, kv_heads, dim, causal, token_lam, packed=False, seed=0, room=(0, 0), gap=0, scale=0.0, poison=False):
        from paper_2010_02838_amd import binding as B
        self.B, self.dtype, self.packed, self.causal = B, dtype, packed, causal
        self.q_lens, self.k_lens, self.H, self.K, self.D = q_lens, k_lens, heads, kv_heads, dim
        self.scale = scale or dim ** -0.5
        n = len(q_lens)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        tq, tk = max(q_lens) + room[0], max(k_lens) + room[1]
        self.tq, self.tk = tq, tk
        if packed:
            rq, rk = gap + sum(q_lens) + gap, gap + sum(k_lens) + gap
            self.q0 = np.concatenate([[gap], gap + np.cumsum(q_lens)]).astype(np.int32)
            self.k0 = np.concatenate([[gap], gap + np.cumsum(k_lens)]).astype(np.int32)
        else:
            rq, rk = n * tq, n * tk
        self.rq, self.rk = rq, rk

        def rand(rows, *shape):
            wide = torch.randn(rows, int(np.prod(shape)) + 16, generator=gen, device=DEV).to(dtype)
            t = wide[:, 8:-8].unflatten(1, shape)
            return t if packed else t.unflatten(0, (n, -1))

        def blank(rows, *shape):
            t = torch.full((rows, int(np.prod(shape)) + 16), 7.0, dtype=dtype, device=DEV)[:, 8:-8].unflatten(1, shape)
            return t if packed else t.unflatten(0, (n, -1))

        self.q, self.k, self.v = rand(rq, heads, 2, dim), rand(rk, kv_heads, 2, dim), rand(rk, kv_heads, 2 * dim)
        self.dout, self.out = rand(rq, heads, 2 * dim), blank(rq, heads, 2 * dim)
        self.dq, self.dk, self.dv = blank(rq, heads, 2, dim), blank(rk, kv_heads, 2, dim), blank(rk, kv_heads, 2 * dim)
        shape = (heads,) if not token_lam else (rq, heads) if packed else (n, tq, heads)
        self.lam = torch.randn(shape, generator=gen, device=DEV)
        self.dlam = torch.full_like(self.lam, 7.0)
        self.o2 = torch.empty(self.out.shape, dtype=dtype, device=DEV)
        self.lse = torch.empty(2, heads, rq, device=DEV)
        self.want()
        if poison:   # behind the sequences' ends: nothing of it may be used
            for t, lens in ((self.q, q_lens), (self.dout, q_lens), (self.k, k_lens), (self.v, k_lens)):
                for b, m in enumerate(lens):
                    t[b, m:] = math.nan if b % 2 else math.inf
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)   # noqa: E731
        lens = dict(q_starts=i32(self.q0), k_starts=i32(self.k0), max_q=tq, max_k=tk) if packed else dict(q_lens=i32(q_lens), k_lens=i32(k_lens))
        self.desc = B.diff_attention_desc(self.q, self.k, self.v, self.out, self.lam, causal=causal, scale=scale, **lens)
        self.ws = torch.empty(B.diff_attention_workspace_bytes(self.desc, True), dtype=torch.uint8, device=DEV)

    def rows(self, t, b, keys):
        n = (self.k_lens if keys else self.q_lens)[b]
        if self.packed:
            at = (self.k0 if keys else self.q0)[b]
            return t[at:at + n]
        return t[b, :n]

    def want(self):
        self.ref = []
        for b in range(len(self.q_lens)):
            f = lambda t, keys: self.rows(t, b, keys).double().cpu().numpy()   # noqa: E731
            lam = f(self.lam, False) if self.lam.dim() > 1 else np.broadcast_to(self.lam.double().cpu().numpy(), (self.q_lens[b], self.H)).copy()
            self.ref.append(reference(f(self.q, False), f(self.k, True), f(self.v, True), lam, f(self.dout, False),
                                      seen(self.q_lens[b], self.k_lens[b], self.causal), self.scale))

    def run(self):
        self.B.codistill_diff_attention(self.desc, self.q, self.k, self.v, self.lam, self.out, self.o2, self.lse, self.ws)
        self.B.codistill_diff_attention_backward(self.desc, self.q, self.k, self.v, self.lam, self.out, self.o2, self.lse, self.dout, self.dq, self.dk,
                                                 self.dv, self.dlam, self.ws)
        torch.cuda.synchronize()

    def check(self):
        tol, n = TOL[self.dtype], range(len(self.q_lens))
        for name, at, keys in (("out", 0, False), ("dq", 1, False), ("dk", 2, True), ("dv", 3, True)):
            t = getattr(self, name)
            got = torch.cat([self.rows(t, b, keys).flatten() for b in n])
            want = np.concatenate([self.ref[b][at].ravel() for b in n])
            # a dS that cancels to nothing (one key: softmax is constant) leaves rounding of its terms
            floor = 2.0 ** -9 * np.linalg.norm(np.concatenate([self.ref[b][3].ravel() for b in n])) if name in ("dq", "dk") else 0.0
            close(got, want, tol, name, floor)
            if not self.packed:   # zeros behind a sequence's end
                assert all(not t[b, (self.k_lens if keys else self.q_lens)[b]:].any() for b in n), name
            else:                 # rows of no sequence are not written
                mask = torch.ones(t.shape[0], dtype=torch.bool, device=DEV)
                for b in n:
                    at0 = (self.k0 if keys else self.q0)[b]
                    mask[at0:at0 + (self.k_lens if keys else self.q_lens)[b]] = False
                assert (t[mask] == 7.0).all(), name
        mag = np.concatenate([self.ref[b][5] for b in n])
        if self.lam.dim() > 1:
            got = torch.cat([self.rows(self.dlam, b, False).flatten() for b in n])
            close(got, np.concatenate([self.ref[b][4].ravel() for b in n]), TOL[torch.float32], "dlam", np.linalg.norm(mag))
        else:
            close(self.dlam, sum(self.ref[b][4].sum(0) for b in n), TOL[torch.float32], "dlam", np.linalg.norm(np.sqrt((mag ** 2).sum(0))))


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim", [8, 24, 32, 40, 64, 72, 104, 128])
def test_head_dims(dtype, dim):
    p = Problem(dtype, [70, 41], [70, 41], 4, 2, dim, True, dim % 16 == 0, seed=dim)
    p.run()
    p.check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_lens,k_lens", [([1], [1]), ([1, 1, 1], [130, 1, 64]), ([5, 2], [3, 7]), ([33], [32]), ([129, 0, 64], [129, 0, 64]),
                                           ([128], [257]), ([200, 7], [65, 0]), ([3], [700])])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_lengths(dtype, q_lens, k_lens, causal):
    """Lengths of zero and one, tiles cut at every edge, rows without a key (more queries than keys under a causal mask, no keys at all), NaN and
    infinities behind the ends."""
    p = Problem(dtype, q_lens, k_lens, 4, 4, 32, causal, True, seed=len(q_lens), room=(3, 2), poison=True)
    p.run()
    p.check()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (8, 2), (12, 3), (40, 1)])
@pytest.mark.parametrize("token_lam", [False, True])
def test_shared_key_heads(heads, kv_heads, token_lam):
    p = Problem(BF, [37, 90], [90, 37], heads, kv_heads, 64, False, token_lam, seed=heads)
    p.run()
    p.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [False, True])
def test_packed(dtype, causal):
    """Sequences one after the other, an empty one among them, rows of no sequence in front and behind; queries and keys of different lengths."""
    for k_lens in ([17, 0, 128, 1, 77], [40, 9, 0, 3, 200]):
        p = Problem(dtype, [17, 0, 128, 1, 77], k_lens, 6, 3, 64, causal, True, packed=True, seed=5, gap=11)
        p.run()
        p.check()


def test_packed_tables_out_of_range():
    """Start tables that point outside the tensors, run backwards or hold a longer sequence than announced are cut: the rows inside are
    computed, nothing beyond them is touched."""
    p = Problem(F32, [20, 30], [20, 30], 2, 2, 32, False, True, packed=True, seed=8)
    for starts in ([0, 20, 1 << 30], [-5, 20, 50], [30, 20, 50], [60, 70, 80]):
        p.desc.keep[2].copy_(torch.tensor(starts, dtype=torch.int32))
        p.desc.keep[3].copy_(torch.tensor(starts, dtype=torch.int32))
        p.run()
    for t in (p.out, p.dq, p.dk, p.dv):
        assert torch.isfinite(t).all()
    p.desc.keep[2].copy_(torch.tensor([0, 20, 50], dtype=torch.int32))
    p.desc.keep[3].copy_(torch.tensor([0, 20, 50], dtype=torch.int32))
    p.run()
    p.check()


@pytest.mark.parametrize("dtype,tq,tk,heads,kv_heads,dim", [(BF, 1, 5000, 8, 2, 64), (BF, 2, 1025, 4, 4, 128), (F32, 1, 3000, 6, 1, 40), (BF, 5, 130, 2, 2, 32),
                                                            (BF, 1, 9000, 16, 1, 64), (F32, 1, 1300, 2, 2, 128)])
def test_few_rows_against_many_keys(dtype, tq, tk, heads, kv_heads, dim):
    """The parts of the keys that several workgroups take and their join, with outputs kept for a backward pass and without; sequences much shorter
    than the room leave parts without a key."""
    p = Problem(dtype, [tq] * 3, [tk, 40, 0], heads, kv_heads, dim, True, False, seed=tk)
    assert p.B.diff_attention_workspace_bytes(p.desc, False) > 0
    p.run()
    p.check()
    kept = p.out.clone()
    p.out.zero_()
    p.B.codistill_diff_attention(p.desc, p.q, p.k, p.v, p.lam, p.out, workspace=p.ws)
    assert torch.equal(kept, p.out)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("room", [0, 299, 4095])
def test_one_key_has_no_gradient(dtype, dim, room):
    """A softmax over one key is one: queries and keys get zeros, to the last bit, whatever way the keys' room makes the work be split."""
    p = Problem(dtype, [3, 40], [1, 1], 4, 2, dim, False, True, seed=dim + room, room=(0, room))
    p.run()
    p.check()
    assert not p.dq.any() and not p.dk.any()
    p = Problem(dtype, [70], [70], 2, 2, dim, True, False, seed=dim)   # the first row under a causal mask
    p.run()
    assert not p.dq[0, 0].any() and p.dq[0, 1:].any()


def test_large_scores():
    """Scores of some hundred: exponents far beyond fp32 but for the running maximum, which has to move at any time (late keys raise it)."""
    for dtype in (BF, F32):
        p = Problem(dtype, [64], [300], 2, 2, 64, False, True, seed=3, scale=1.0)
        ramp = torch.linspace(0.1, 6.0, 300, device=DEV)[None, :, None, None, None]
        p.k.copy_((p.k.float() * ramp).to(dtype))
        p.want()
        p.run()
        # a weight's exponent is a score of up to 500, off by 2^-24 of itself in fp32
        got, want = p.out[0].double().cpu().numpy(), p.ref[0][0]
        assert np.linalg.norm(got - want) <= (TOL[dtype] + 500 * 2.0 ** -23) * np.linalg.norm(want)


def test_long_cache_offsets():
    """Keys and values further apart than 32-bit offsets reach, and sequences that share one cache (a batch stride of 0) in the forward pass."""
    from paper_2010_02838_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(1)
    step, tk, H, D = 1 << 26, 40, 2, 64
    big = torch.empty(step * (tk - 1) + 2 * H * D * 2, dtype=BF, device=DEV)
    k = big.as_strided((2, tk, H, 2, D), (0, step, 2 * D, D, 1))
    v = big[2 * H * D:].as_strided((2, tk, H, 2 * D), (0, step, 2 * D, 1))
    k[0] = torch.randn(tk, H, 2, D, generator=gen, device=DEV).to(BF)
    v[0] = torch.randn(tk, H, 2 * D, generator=gen, device=DEV).to(BF)
    q = torch.randn(2, 3, H, 2, D, generator=gen, device=DEV).to(BF)
    out, lam = torch.empty(2, 3, H, 2 * D, dtype=BF, device=DEV), torch.rand(H, device=DEV, generator=gen)
    desc = B.diff_attention_desc(q, k, v, out, lam, causal=True)
    B.codistill_diff_attention(desc, q, k, v, lam, out, workspace=torch.empty(B.diff_attention_workspace_bytes(desc, False), dtype=torch.uint8, device=DEV))
    for b in range(2):
        f = lambda t: t[b].double().cpu().numpy()   # noqa: E731
        want = reference(f(q), f(k), f(v), np.tile(lam.double().cpu().numpy(), (3, 1)), np.zeros((3, H, 2 * D)), seen(3, tk, True), D ** -0.5)[0]
        close(out[b], want, TOL[BF], "out")
    # the gradients of a shared cache would race: refused
    n = torch.empty(2, 2, 6, device=DEV)
    with pytest.raises(B.CodistillError) as e:
        B.codistill_diff_attention_backward(desc, q, k, v, lam, out, torch.empty_like(out), n, out, q, k, v, lam,
                                            torch.empty(B.diff_attention_workspace_bytes(desc, True), dtype=torch.uint8, device=DEV))
    assert e.value.code == B.CD_ERR_INVALID_ARG and "share memory" in str(e.value)


@pytest.mark.parametrize("causal", [False, True])
def test_gradient_against_differences(causal):
    """The fp32 kernels' own forward pass, differenced along random directions: central differences with a step h of 1e-2 are off by h^2 of the third
    derivative (1e-4 of the first here) and by 2^-24 / h of the sum."""
    p = Problem(F32, [40, 23], [40, 23], 4, 2, 32, causal, True, seed=9)
    p.run()
    gen = torch.Generator(device=DEV).manual_seed(2)
    for name in ("q", "k", "v", "lam"):
        x, g = getattr(p, name), getattr(p, "d" + name).clone()
        kept, d = x.clone(), torch.randn(x.shape, generator=gen, device=DEV)
        d = d / d.norm() * 0.3 + 0.7 * g / g.norm()   # (mostly along the gradient, so that the difference does not cancel)
        f = []
        for h in (1e-2, -1e-2):
            x.copy_(kept + h * d)
            p.B.codistill_diff_attention(p.desc, p.q, p.k, p.v, p.lam, p.out, p.o2, p.lse, p.ws)
            f.append(sum((p.rows(p.out, b, False).double() * p.rows(p.dout, b, False).double()).sum().item() for b in range(2)))
        x.copy_(kept)
        want = (g.double() * d.double()).sum().item()
        assert abs((f[0] - f[1]) / 2e-2 - want) <= 1e-3 * abs(want), name


def test_same_bits_and_other_streams():
    p = Problem(BF, [300, 150], [300, 150], 8, 2, 64, True, False, seed=4)
    p.run()
    kept = [getattr(p, n).clone() for n in ("out", "dq", "dk", "dv", "dlam")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.run()
    for n, t in zip(("out", "dq", "dk", "dv", "dlam"), kept):
        assert torch.equal(getattr(p, n), t), n
