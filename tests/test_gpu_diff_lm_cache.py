"""The small language model with normalised queries and keys, its embedding's gradient, and decoding from caches in 8 bits."""
import math

import pytest
import torch

from test_gpu_diff_lm import DEV

pytestmark = pytest.mark.gpu


def reference(lm, tokens, starts, positions, dlogits):
    """The network with normalised queries and keys in float64, with torch's derivatives.  Returns logits and gradients."""
    w = {n: (lm.w[n] if n.startswith("lam") else lm.p[n]).detach().double().cpu().requires_grad_(True) for n in lm.w}
    tokens, pos, starts = tokens.cpu(), positions[0].double().cpu(), starts.tolist()
    H, K, D = lm.H, lm.K, lm.D

    def norm(x, g, post=1.0):
        return post * g * x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt()

    ang = pos[:, None] * 10000.0 ** (-torch.arange(D // 2).double() * 2 / D)

    def turn(t):
        c, s = ang.cos()[:, None, None], ang.sin()[:, None, None]
        a, b = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    x = w["embed"][tokens]
    for i in range(lm.L):
        q, k, v = (norm(x, w["norm%d" % i]) @ w["qkv%d" % i].t()).split([2 * D * H, 2 * D * K, 2 * D * K], 1)
        q, k, v = turn(norm(q.view(-1, H, 2, D), w["qn%d" % i])), turn(norm(k.view(-1, K, 2, D), w["kn%d" % i])), v.view(-1, K, 2 * D)
        rows = []
        for a, b in zip(starts, starts[1:]):
            heads = []
            for h in range(H):
                g = h // (H // K)
                see = torch.ones(b - a, b - a).tril().bool()
                p = [torch.softmax((q[a:b, h, m] @ k[a:b, g, m].t() / math.sqrt(D)).masked_fill(~see, -math.inf), 1) for m in (0, 1)]
                heads.append((p[0] - w["lam%d" % i][h] * p[1]) @ v[a:b, g])
            rows.append(torch.stack(heads, 1))
        x = x + norm(torch.cat(rows), w["head%d" % i], lm.post).flatten(1) @ w["out%d" % i].t()
    z = norm(x, w["norm"]) @ w["embed"].t()
    z.backward(dlogits.double().cpu())
    return z.detach(), {n: t.grad for n, t in w.items()}


@pytest.mark.parametrize("dtype,kv_heads", [(torch.float32, 2), (torch.float32, 1), (torch.bfloat16, 2)])
def test_gradients_with_normalised_queries(dtype, kv_heads):
    """fp32: some thirty sums of fp32 products between a weight and the logits, 1e-4; bf16 (one layer, a small lambda): some seven roundings, each
    off by at most 2^-8 of an element and by 1.7e-3 of a tensor's 2-norm, 1.2e-2 if they all add up: 2e-2."""
    from paper_2010_02838_amd.diff_lm import DiffLM, copying_batch
    exact = dtype is torch.float32
    lm = DiffLM(50, layers=2 if exact else 1, heads=4, kv_heads=kv_heads, head_dim=32, lambda_init=0.5 if exact else 0.2, seed=3, dtype=dtype, qk_norm=True)
    gen = torch.Generator(device=DEV).manual_seed(2)
    for n in lm.w:
        if n[:2] in ("qn", "kn"):
            lm.w[n].copy_(1 + 0.3 * torch.randn(32, generator=gen, device=DEV))
            lm.p[n].copy_(lm.w[n])
    tokens, positions, starts, _ = copying_batch(5, 20, 50, seed=1)
    z = lm.forward(tokens, positions, starts, 40)
    dz = torch.randn(z.shape, generator=gen, device=DEV).bfloat16().float()
    lm.backward(dz)
    want, grads = reference(lm, tokens, starts, positions, dz)
    tol = 1e-4 if exact else 2e-2
    assert (z.double().cpu() - want).norm() <= tol * want.norm()
    for n, g in grads.items():
        if n[:3] != "lam" or exact:      # (a few lambdas: sums of terms of either sign that may cancel)
            assert (lm.g[n].double().cpu() - g).norm() <= tol * g.norm(), n


def test_gradients_repeat_and_words_that_do_not_occur():
    from paper_2010_02838_amd.diff_lm import DiffLM, copying_batch
    lm = DiffLM(300, layers=1, heads=4, kv_heads=2, head_dim=32, seed=3, qk_norm=True)
    tokens, positions, starts, _ = copying_batch(100, 20, 7, seed=1)
    first = None
    for _ in range(4):
        z = lm.forward(tokens, positions, starts, 40)
        lm.backward(torch.where(torch.arange(300, device=DEV) < 7, torch.cos(z), 0.0))
        got = {k: g.clone() for k, g in lm.g.items()}
        first = first or got
        assert all(torch.equal(g, first[k]) for k, g in got.items())
    assert (got["embed"][7:] == 0).all() and (got["embed"][:7] != 0).any(1).all()


def test_tokens_on_the_host():
    """As an index they may lie there; they are moved."""
    from paper_2010_02838_amd.diff_lm import DiffLM, copying_batch
    lm = DiffLM(30, layers=1, heads=2, kv_heads=1, head_dim=16, seed=3)
    tokens, positions, starts, _ = copying_batch(4, 9, 30, seed=1)
    got = []
    for t in (tokens, tokens.cpu(), tokens.int()):
        z = lm.forward(t, positions, starts, 18)
        lm.backward(torch.cos(z))
        got.append((z, lm.g["embed"].clone(), lm.decoder(2, 5).step(t[:2])))
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))


@pytest.mark.parametrize("qk_norm", [False, True])
def test_decoding_from_a_cache_in_8_bits(qk_norm):
    """Against a decoder in fp32 that keeps, in place of its new tokens' keys and values, what the coded cache holds of them: the same numbers, other orders of fp32
    sums (1e-4).  (It does not quantise its own: an element next to the border between two codes falls on either side by its last bit, and a code is 1 / 127 of
    the largest element, so that one such token moves the logits by more than 1e-4.)  What is held is the element to half a step.  Prompts first, of different
    lengths, then token by token; a sequence begins anew on the way."""
    from paper_2010_02838_amd.diff_lm import Decoder, DiffLM

    class Rounded(Decoder):
        def _attend(self, i, q, k, v, at):
            held_k, held_v = torch.empty_like(k[:, None].contiguous()), torch.empty_like(v[:, None].contiguous())
            cache = coded.caches[i]
            cache.read(cache.rows(held_k, held_v, first=at.int()), held_k, held_v)
            for held, x in ((held_k[:, 0], k), (held_v[:, 0], v)):
                step = x.abs().amax(-1, keepdim=True) * (1 + 2.0 ** -7) / 127
                assert ((held - x).abs() <= 0.5 * step + 1e-4 * x.abs().amax()).all()
            super()._attend(i, q, held_k[:, 0], held_v[:, 0], at)

    lm = DiffLM(50, layers=2, heads=4, kv_heads=2, head_dim=32, seed=4, qk_norm=qk_norm)
    words = torch.randint(0, 50, (3, 200), generator=torch.Generator().manual_seed(5)).to(DEV)
    coded, plain = lm.decoder(3, 300, cache_bits=8), Rounded(lm, 3, 300)
    for t in range(150):
        if t == 100:
            for d in (coded, plain):
                d.lens[1] = 0
        a, b = coded.step(words[:, t]), plain.step(words[:, t])
        assert (a - b).norm() <= 1e-4 * b.norm(), t
    # prompts: what they leave in the caches is what they would have left token by token; in fp32 the prompt's own pass is not rounded
    lens = [70, 1, 129]
    prompt = torch.cat([words[i, :n] for i, n in enumerate(lens)])
    starts = torch.tensor([0, 70, 71, 200], dtype=torch.int32, device=DEV)
    plain = lm.decoder(3, 300)
    za, zb = coded.prefill(prompt, starts, 129), plain.prefill(prompt, starts, 129)
    assert torch.equal(za, zb)
    positions = torch.cat([torch.arange(n) for n in lens]).int()[None].to(DEV)
    z = lm.forward(prompt, positions, starts, 129)
    assert (za - z).norm() <= 1e-4 * z.norm()
    for i in range(lm.L):
        k, v = (t.clone() for t in (plain.k[i], plain.v[i]))
        coded.caches[i].read(coded.caches[i].rows(k, v, counts=coded.lens), k, v)
        for b, n in enumerate(lens):
            for got, want in ((k[b, :n], plain.k[i][b, :n]), (v[b, :n], plain.v[i][b, :n])):
                assert ((got - want).abs() <= (0.5 + 2.0 ** -7) * want.abs().amax(-1, keepdim=True) * (1 + 2.0 ** -7) / 127).all()     # half a step of the largest
        plain.k[i].copy_(torch.where(torch.isfinite(k), k, 0.0))
        plain.v[i].copy_(torch.where(torch.isfinite(v), v, 0.0))
    a, b = coded.step(words[:, 199]), plain.step(words[:, 199])
    new = (a - b).norm()     # (the new token's own key and value are codes in one of them: half a step of one key among many)
    assert new <= 3e-2 * b.norm()


def test_decoder_refuses():
    from paper_2010_02838_amd.diff_lm import DiffLM
    lm = DiffLM(20, layers=1, heads=2, kv_heads=1, head_dim=16, seed=2)
    with pytest.raises(ValueError):
        lm.decoder(2, 6, cache_bits=4)
    for bits in (None, 8):
        decoder = lm.decoder(2, 6, cache_bits=bits)
        words = torch.randint(0, 20, (12,), generator=torch.Generator().manual_seed(1)).to(DEV)
        for starts, longest in (([0, 7, 12], 7), ([0, 6], 6), ([0, 6, 11], 6), ([1, 6, 12], 6), ([0, 6, 12], 5), ([0, 14, 12], 6)):
            with pytest.raises(ValueError):
                decoder.prefill(words, torch.tensor(starts, dtype=torch.int32, device=DEV), longest)
        decoder.prefill(words[:9], torch.tensor([0, 3, 9], dtype=torch.int32, device=DEV), 6)
        with pytest.raises(ValueError):
            decoder.step(words[:2])       # one of them is full
        decoder.lens.zero_()
        first = [decoder.step(words[2 * t:2 * t + 2]) for t in range(6)]
        with pytest.raises(ValueError):
            decoder.step(words[:2])
        decoder.lens.zero_()
        for t in range(6):
            assert torch.equal(decoder.step(words[2 * t:2 * t + 2]), first[t])


def test_captured_training_operators():
    """Embedding, norm with rotation, the update of a cache and their gradients in one graph: replays, with eager work between them, equal the eager run bit for bit."""
    from paper_2010_02838_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(6)
    for rows in (300, 17000):       # (places counted, and a radix sort)
        table = torch.randn(500, 256, generator=gen, device=DEV).bfloat16()
        tokens = torch.randint(-1, 500, (rows,), generator=gen, device=DEV)
        x, y, dy, dx = (torch.randn(rows, 256, generator=gen, device=DEV).bfloat16() for _ in range(4))
        dtable, dgain = torch.empty(500, 256, device=DEV), torch.empty(64, device=DEV)
        gain, pos = torch.ones(64, device=DEV).bfloat16(), torch.arange(rows, dtype=torch.int32, device=DEV)[None]
        rope = B.rotary_desc(64, (32,), 1e4, torch.bfloat16)
        heads = lambda t: t.view(rows, 4, 64)   # noqa: E731
        nws = torch.empty(B.norm_rotary_workspace_bytes(rope, rows, 1), dtype=torch.uint8, device=DEV)
        ews = torch.empty(B.embedding_workspace_bytes(rows, 500, 256), dtype=torch.uint8, device=DEV)

        def step():
            B.codistill_embedding(tokens, table, x, 16.0)
            B.codistill_norm_rotary(rope, pos, [(heads(x), gain, heads(y))])
            B.codistill_norm_rotary_backward(rope, pos, [(heads(x), gain, heads(dy), heads(dx), dgain)], nws)
            B.codistill_embedding_backward(tokens, dx, dtable, ews, 16.0)
            B.codistill_embedding_backward(tokens, dx, dtable, ews, 2.0, accumulate=True)

        results = []

        def snapshot():
            torch.cuda.synchronize()
            results.append([t.clone() for t in (x, y, dx, dgain, dtable)])
            for t in (x, y, dx, dgain, dtable, nws, ews):
                t.fill_(7)

        side = torch.cuda.Stream()
        step()
        snapshot()
        graph = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
            snapshot()
            with torch.cuda.graph(graph, stream=side):
                step()
        torch.cuda.current_stream().wait_stream(side)
        for _ in range(3):
            graph.replay()
            snapshot()
            (torch.randn(1 << 20, device=DEV) ** 2).sum().item()
        for r in results[1:]:
            assert all(torch.equal(a, b) for a, b in zip(results[0], r))


def network(**kw):
    from paper_2010_02838_amd.diff_lm import DiffLM
    return DiffLM(30, **dict(dict(layers=2, heads=2, kv_heads=1, head_dim=16, lambda_init=0.5, seed=3), **kw))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_that_count_from_the_end(dtype):
    """As in any index: the last word is -1, in the network, its gradient, a prompt and a decoder's step."""
    from paper_2010_02838_amd.diff_lm import copying_batch
    lm = network(dtype=dtype)
    tokens, positions, starts, _ = copying_batch(4, 9, 30, seed=1)
    got = []
    for t in (tokens, torch.where(torch.arange(len(tokens), device=DEV) % 3 == 0, tokens - 30, tokens), (tokens - 30).cpu()):
        z = lm.forward(t, positions, starts, 18)
        lm.backward(torch.cos(z))
        decoder = lm.decoder(4, 20)
        got.append((z, lm.g["embed"].clone(), decoder.prefill(t, starts, 18), decoder.step(t[:4])))
    assert torch.isfinite(got[0][0]).all() and all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))


@pytest.mark.parametrize("bad", [30, -31, 2 ** 32, 2 ** 40, -2 ** 63])
def test_tokens_that_are_no_words(bad):
    """On the host they are refused.  On the device nothing waits for them to be looked at: the logits from there on are NaN, those of other sequences are as without it."""
    from paper_2010_02838_amd.diff_lm import copying_batch
    lm = network()
    tokens, positions, starts, _ = copying_batch(4, 9, 30, seed=1)
    _, begin, end, *_ = starts.tolist()   # the second sequence, in whose middle it lies
    middle = (begin + end) // 2
    wrong = tokens.clone()
    wrong[middle] = bad
    z, want = lm.forward(wrong, positions, starts, 18), lm.forward(tokens, positions, starts, 18)
    others = torch.ones(len(tokens), dtype=torch.bool, device=DEV)
    others[begin:end] = False
    assert torch.equal(z[others], want[others]) and torch.isnan(z[middle:end]).all()
    for bits in (None, 8):
        decoder, right = lm.decoder(4, 20, cache_bits=bits), lm.decoder(4, 20, cache_bits=bits)
        decoder.prefill(wrong, starts, 18), right.prefill(tokens, starts, 18)
        a, b = decoder.step(tokens[:4]), right.step(tokens[:4])
        assert torch.isnan(a[1]).all() and torch.equal(a[[0, 2, 3]], b[[0, 2, 3]]) and torch.isfinite(b).all()
        for d in (decoder, right):       # the sequence begins anew
            d.lens[1] = 0
        now = tokens[:4].clone()
        assert torch.equal(decoder.step(now), right.step(now))
        now[2] = bad
        a, b = decoder.step(now), right.step(tokens[:4])
        assert torch.isnan(a[2]).all() and torch.equal(a[[0, 1, 3]], b[[0, 1, 3]])
        with pytest.raises(ValueError, match="vocabulary"):
            decoder.step(now.cpu())
        with pytest.raises(ValueError, match="vocabulary"):
            decoder.prefill(wrong.cpu(), starts, 18)
    with pytest.raises(ValueError, match="vocabulary"):
        lm.forward(wrong.cpu(), positions, starts, 18)


@pytest.mark.parametrize("qk_norm", [False, True])
def test_decoding_in_bf16_from_a_cache_in_8_bits(qk_norm):
    """Layer by layer, on what the decoder has there: the codes of its new tokens and of its prompts are exact, its attention is within the bound that the cache's attention is held
    to (tests of the cache).  Prompts' logits are those of a decoder with bf16 caches, bit for bit, and the network's to some seven roundings, 2e-2."""
    from test_gpu_kv_cache import check_attention, image, put, same
    from paper_2010_02838_amd.diff_lm import Decoder, DiffLM

    def token(t, row):
        return t[row].detach().cpu().double().numpy()

    class Checked(Decoder):
        def _attend(self, i, q, k, v, at):
            cache, img = self.caches[i], image(self.caches[i])
            super()._attend(i, q, k, v, at)
            lens = self.lens.tolist()
            for b in range(self.S):
                put(cache, img, b, lens[b] - 1, token(k, b), token(v, b))
            same(cache, img)
            check_attention(cache, q[:, None], self.lm.w["lam%d" % i], self.lens, self.out, True)

    lm = DiffLM(50, layers=1, heads=4, kv_heads=2, head_dim=32, lambda_init=0.2, seed=4, qk_norm=qk_norm, dtype=torch.bfloat16)
    words = torch.randint(0, 50, (3, 200), generator=torch.Generator().manual_seed(5)).to(DEV)
    coded, plain, lens = Checked(lm, 3, 300, 8), lm.decoder(3, 300), [70, 1, 129]
    for t in range(6):
        coded.step(words[:, t])
    written, write = [], coded.caches[0].write
    coded.caches[0].write = lambda rows, k, v: (written.append((k.clone(), v.clone())), write(rows, k, v))
    prompt, starts = torch.cat([words[i, :n] for i, n in enumerate(lens)]), torch.tensor([0, 70, 71, 200], dtype=torch.int32, device=DEV)
    img = image(coded.caches[0])
    za, zb = coded.prefill(prompt, starts, 129), plain.prefill(prompt, starts, 129)
    coded.caches[0].write = write
    for b, n in enumerate(lens):
        for j in range(n):
            put(coded.caches[0], img, b, j, token(written[0][0], sum(lens[:b]) + j), token(written[0][1], sum(lens[:b]) + j))
    same(coded.caches[0], img)
    positions = torch.cat([torch.arange(n) for n in lens]).int()[None].to(DEV)
    z = lm.forward(prompt, positions, starts, 129)
    assert torch.equal(za, zb) and (za - z).norm() <= 2e-2 * z.norm()
    for t in range(6):
        if t == 3:
            coded.lens[1] = 0        # a sequence begins anew
        coded.step(words[:, 190 + t])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured_decoding_operators(dtype):
    """The kernels of a decoder's step in one graph, lookup, norm with rotation, the update of a cache and the attention against it: every replay equals the eager run of the
    same tokens bit for bit, with eager work between the replays."""
    from paper_2010_02838_amd import binding as B
    from paper_2010_02838_amd.kv_cache import KVCache
    S, H, K, D = 3, 4, 2, 32
    gen = torch.Generator(device=DEV).manual_seed(8)
    table, gain = torch.randn(60, 2 * D * (H + 2 * K), generator=gen, device=DEV).to(dtype), torch.ones(D, device=DEV).to(dtype)
    rope, lam = B.rotary_desc(D, (D // 2,), 1e4, dtype), torch.full((H,), 0.5, device=DEV)

    def make():
        s = dict(tokens=torch.zeros(S, dtype=torch.int64, device=DEV), first=torch.tensor([0, 60, 1000], dtype=torch.int32, device=DEV), x=torch.empty(S, table.shape[1], dtype=dtype, device=DEV),
                 y=torch.empty(S, 2 * D * (H + K), dtype=dtype, device=DEV), out=torch.empty(S, 1, H, 2 * D, dtype=dtype, device=DEV), cache=KVCache(S, 2048, K, D, dtype, 128, device=DEV))
        s["lens"], s["pos"] = s["first"] + 1, s["first"][None].clone()
        for t in (s["cache"].k, s["cache"].v):
            t.fill_(3)
        s["cache"].scales.fill_(0.02)
        cut = [2 * D * H, 2 * D * K]
        s["in"], s["turned"] = s["x"][:, :sum(cut)].split(cut, 1), s["y"].split(cut, 1)
        s["q"], s["k"] = s["turned"][0].unflatten(1, (H, 2, D))[:, None], s["turned"][1].unflatten(1, (K, 2, D))[:, None]
        s["v"] = s["x"][:, sum(cut):].unflatten(1, (K, 2 * D))[:, None]
        s["rows"], s["desc"] = s["cache"].rows(s["k"], s["v"], first=s["first"]), s["cache"].attention(s["q"], s["out"], lam, s["lens"], causal=True)
        s["ws"] = torch.empty(s["desc"].workspace_bytes, dtype=torch.uint8, device=DEV)
        return s

    def step(s):
        B.codistill_embedding(s["tokens"], table, s["x"], 0.5, index=True)
        B.codistill_norm_rotary(rope, s["pos"], [(a.unflatten(1, (-1, D)), gain, b.unflatten(1, (-1, D))) for a, b in zip(s["in"], s["turned"])])
        s["cache"].write(s["rows"], s["k"], s["v"])
        s["cache"].attend(s["desc"], s["q"], lam, s["out"], s["ws"])
        for t in (s["first"], s["lens"], s["pos"]):
            t.add_(1)

    eager, captured, side, graph = make(), make(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    for s in (eager, captured):
        step(s)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(captured)
    for i in range(5):
        for s in (eager, captured):
            s["tokens"].copy_(torch.tensor([7 * i, 59 - i, i - 5]))
        captured["ws"].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        (torch.randn(1 << 20, device=DEV) ** 2).sum().item()
        assert torch.isfinite(eager["out"]).all() and all(torch.equal(eager[n], captured[n]) for n in ("x", "y", "out", "first", "lens", "pos"))
        assert all(torch.equal(getattr(eager["cache"], n), getattr(captured["cache"], n)) for n in ("k", "v", "scales"))
