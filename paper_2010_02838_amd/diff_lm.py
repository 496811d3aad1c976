"""A small language model of differential-attention layers, trained by codistillation and decoded token by token.

Every layer is x + W_o headnorm(diffattn(rotary(q), rotary(k), v)), q, k, v = W_qkv norm(x); the logits are taken against the tied embedding table.  With
qk_norm=True queries and keys are normalised, each with a gain of its own, in the pass that turns them.
The operators of the layer, the embedding and its gradient, the loss against the peers' logits and the update are the library's kernels; the projections are plain matrix
products (torch).  The same batch gives the same bits.  A decoder's caches hold the model's type, or 8 bits a channel (cache_bits=8).  Sequences are packed: `starts` says where each begins.  fp32 throughout, or with dtype=torch.bfloat16 bf16 weights and activations beside an fp32 residual stream and fp32 masters.  (Where the two maps of a head are alike and lambda is near
one, their difference is small and the roundings of bf16 queries and keys are not: at lambda 0.9 a gradient of a two-layer model is off by 2.5 %, at 0.3 by 1 %.)

    python -m paper_2010_02838_amd.diff_lm        trains two models on a copying task, each against the other's logits, and decodes from one
"""
import math

import torch

from . import binding as B
from .adamw import AdamW
from .kv_cache import KVCache

EPS = 1e-5


class DiffLM:
    """width: of the residual stream; None: that of all heads' outputs."""

    def __init__(self, vocabulary, layers=2, heads=4, kv_heads=2, head_dim=32, theta=10000.0, lambda_init=0.8, state_bits=8, seed=0, dtype=torch.float32,
                 device="cuda:0", width=None, qk_norm=False):
        self.V, self.L, self.H, self.K, self.D, self.dev = vocabulary, layers, heads, kv_heads, head_dim, device
        every = heads * 2 * head_dim
        self.d, self.post, self.dt = width or every, 1.0 - lambda_init, dtype
        if not 1 <= self.d <= B.HEAD_NORM_MAX_WIDTH:
            raise ValueError("diff_lm: a residual stream of %d channels, %d at most: give a width" % (self.d, B.HEAD_NORM_MAX_WIDTH))
        self.qk_norm = qk_norm
        self.qkv = 2 * head_dim * (heads + 2 * kv_heads)
        gen = torch.Generator(device=device).manual_seed(seed)
        d = self.d
        shapes = [("embed", (vocabulary, d), d ** -0.5)]
        for i in range(layers):
            shapes += [("norm%d" % i, (d,), None), ("qkv%d" % i, (self.qkv, d), d ** -0.5), ("lam%d" % i, (heads,), None),
                       ("head%d" % i, (2 * head_dim,), None), ("out%d" % i, (d, every), every ** -0.5 / math.sqrt(2 * layers))]
            if qk_norm:
                shapes += [("qn%d" % i, (head_dim,), None), ("kn%d" % i, (head_dim,), None)]
        shapes.append(("norm", (d,), None))
        self.w, self.g, self.p = {}, {}, {}
        for name, shape, scale in shapes:
            if scale is None:
                t = torch.full(shape, lambda_init if name.startswith("lam") else 1.0, device=device)
            else:
                t = torch.randn(shape, generator=gen, device=device) * scale
            self.w[name], self.g[name], self.p[name] = t, torch.zeros_like(t), t.to(dtype)   # (fp32: the master itself)
        matrix = [len(s) == 2 for _, s, _ in shapes]
        self.opt = AdamW(list(self.w.values()), list(self.g.values()), list(self.p.values()) if dtype is torch.bfloat16 else None, weight_decay=[0.1 if m else 0.0 for m in matrix],
                         state_bits=state_bits)
        self.rope = B.rotary_desc(head_dim, (head_dim // 2,), theta, dtype)
        self.updates, self.kept = 0, None

    def _split(self, fused):
        """Queries, keys and values as ranges of the fused projection's rows."""
        q, k, v = fused.split([2 * self.D * self.H, 2 * self.D * self.K, 2 * self.D * self.K], 1)
        return q.unflatten(1, (self.H, 2, self.D)), k.unflatten(1, (self.K, 2, self.D)), v.unflatten(1, (self.K, 2 * self.D))

    def _norm(self, x, name):
        """The residual stream and its norm are fp32; what the products read is bf16."""
        y = torch.empty_like(x)
        B.codistill_head_norm(x[:, None], self.w[name], y[:, None], EPS)
        return y.to(self.dt)

    def _turn(self, q, k, positions, inverse=False):
        """Both maps of every head are turned: 2 H and 2 K heads of D channels, in place."""
        B.codistill_rotary(self.rope, positions, [(t.flatten(1, 2), t.flatten(1, 2)) for t in (q, k)], inverse)

    def _queries_and_keys(self, fused, i, positions):
        """Queries, keys and values of a layer as its attention takes them, and the rows of the projection that the gradients need (with norms: their inputs)."""
        q, k, v = self._split(fused)
        if not self.qk_norm:
            self._turn(q, k, positions)
            return q, k, v, None
        to_q, to_k, _ = self._split(torch.empty_like(fused))
        B.codistill_norm_rotary(self.rope, positions, [(a.flatten(1, 2), self.p[n % i], b.flatten(1, 2)) for a, n, b in ((q, "qn%d", to_q), (k, "kn%d", to_k))], EPS)
        return to_q, to_k, v, fused

    def _tokens(self, tokens):
        """Tokens as the embedding takes them.  They are an index: -1 is the last word.  Tokens that are none are refused on the host; on the device nobody waits for them, and
        the residual stream begins with NaN there."""
        if tokens.get_device() < 0 and tokens.numel():
            least, most = int(tokens.min()), int(tokens.max())
            if least < -self.V or most >= self.V:
                raise ValueError("diff_lm: tokens %d .. %d outside a vocabulary of %d" % (least, most, self.V))
        return tokens.to(self.dev).contiguous()

    def _embed(self, tokens):
        """The residual stream's beginning, fp32."""
        x = torch.empty(tokens.numel(), self.d, device=self.dev)
        B.codistill_embedding(tokens, self.p["embed"], x, index=True)
        return x

    def forward(self, tokens, positions, starts, longest):
        """Logits fp32 [rows, V]; keeps what backward() needs.  tokens int64 [rows] (below zero: counted from the vocabulary's end; logits that see one outside it are NaN,
        on the host it is an error), positions int32 [1, rows], starts int32 [sequences + 1]."""
        tokens, rows, dev, dt = self._tokens(tokens), tokens.numel(), self.dev, self.dt
        x = self._embed(tokens)
        layers = []
        for i in range(self.L):
            y = self._norm(x, "norm%d" % i)
            q, k, v, raw = self._queries_and_keys(y @ self.p["qkv%d" % i].t(), i, positions)
            out, o2 = torch.zeros(rows, self.H, 2 * self.D, dtype=dt, device=dev), torch.empty(rows, self.H, 2 * self.D, dtype=dt, device=dev)   # (zero where rows belong to no sequence)
            lse = torch.empty(2, self.H, rows, device=dev)
            lam = self.w["lam%d" % i]
            desc = B.diff_attention_desc(q, k, v, out, lam, causal=True, q_starts=starts, k_starts=starts, max_q=longest, max_k=longest)
            ws = torch.empty(B.diff_attention_workspace_bytes(desc, True), dtype=torch.uint8, device=dev)
            B.codistill_diff_attention(desc, q, k, v, lam, out, o2, lse, ws)
            n = torch.empty_like(out)
            B.codistill_head_norm(out, self.p["head%d" % i], n, EPS, self.post)
            layers.append((x, y, q, k, v, out, o2, lse, desc, ws, n, raw))
            x = x + n.flatten(1) @ self.p["out%d" % i].t()
        z = self._norm(x, "norm")
        self.kept = (tokens, positions, layers, x, z)
        return (z @ self.p["embed"].t()).float()

    def _norm_backward(self, x, name, dy):
        dy, dx, width = dy.float(), torch.empty_like(x), x.shape[1]
        ws = torch.empty(B.head_norm_workspace_bytes(x.shape[0], 1, width), dtype=torch.uint8, device=self.dev)
        B.codistill_head_norm_backward(x[:, None], self.w[name], dy[:, None], dx[:, None], self.g[name], ws, EPS)
        return dx

    def backward(self, dlogits):
        """Gradients of all parameters in self.g, from d loss / d logits."""
        tokens, positions, layers, x, z = self.kept
        dz = dlogits.to(self.dt)
        self.g["embed"].copy_(dz.t() @ z)
        dx = self._norm_backward(x, "norm", dz @ self.p["embed"])
        for i in reversed(range(self.L)):
            x, y, q, k, v, out, o2, lse, desc, ws, n, raw = layers[i]
            dxb = dx.to(self.dt)
            self.g["out%d" % i].copy_(dxb.t() @ n.flatten(1))
            dn = (dxb @ self.p["out%d" % i]).view_as(n)
            nws = torch.empty(B.head_norm_workspace_bytes(*n.shape), dtype=torch.uint8, device=self.dev)
            B.codistill_head_norm_backward(out, self.p["head%d" % i], dn, dn, self.g["head%d" % i], nws, EPS, self.post)
            fused = torch.zeros(x.shape[0], self.qkv, dtype=self.dt, device=self.dev)   # (zero where rows belong to no sequence)
            dq, dk, dv = self._split(fused)
            B.codistill_diff_attention_backward(desc, q, k, v, self.w["lam%d" % i], out, o2, lse, dn, dq, dk, dv, self.g["lam%d" % i], ws)
            if self.qk_norm:
                into = [(a.flatten(1, 2), self.p[n_ % i], b.flatten(1, 2), b.flatten(1, 2), self.g[n_ % i]) for a, n_, b in zip(self._split(raw), ("qn%d", "kn%d"), (dq, dk))]
                nws = torch.empty(B.norm_rotary_workspace_bytes(self.rope, x.shape[0], 2), dtype=torch.uint8, device=self.dev)
                B.codistill_norm_rotary_backward(self.rope, positions, into, nws, EPS)
            else:
                self._turn(dq, dk, positions, inverse=True)
            self.g["qkv%d" % i].copy_(fused.t() @ y)
            dx = dx + self._norm_backward(x, "norm%d" % i, fused @ self.p["qkv%d" % i])
        ws = torch.empty(B.embedding_workspace_bytes(tokens.numel(), self.V, self.d), dtype=torch.uint8, device=self.dev)
        B.codistill_embedding_backward(tokens, dx, self.g["embed"], ws, accumulate=True, index=True)   # (beside the projection's gradient)

    def update(self, lr):
        self.updates += 1
        self.opt.step(lr, self.updates, 0.9, 0.99, 1e-8, seed=self.updates)

    def decoder(self, sequences, room, cache_bits=None):
        return Decoder(self, sequences, room, cache_bits)


class Decoder:
    """One token at a time for several sequences, against caches of rotated keys and of values: in the model's type, or, with cache_bits=8, as codes with a scale for each
    key and value.  lens: the sequences' ages, on the device; a sequence whose age is set to zero begins anew."""

    def __init__(self, lm, sequences, room, cache_bits=None):
        if cache_bits not in (None, 8):
            raise ValueError("decoder: caches in the model's type (None) or in 8 bits")
        self.lm, self.S, self.room, self.bits = lm, sequences, room, cache_bits
        zeros = lambda *shape: torch.zeros(shape, dtype=lm.dt, device=lm.dev)   # noqa: E731
        self.lens = torch.zeros(sequences, dtype=torch.int32, device=lm.dev)
        self.oldest = 0   # no sequence is older
        self.out = zeros(sequences, 1, lm.H, 2 * lm.D)
        if cache_bits == 8:
            self.caches = [KVCache(sequences, room, lm.K, lm.D, lm.dt, device=lm.dev) for _ in range(lm.L)]
            self.first = torch.zeros_like(self.lens)
            q, k, v = (t[:, None] for t in lm._split(zeros(sequences, lm.qkv)))
            self.rows = self.caches[0].rows(k, v, first=self.first)
            self.desc = self.caches[0].attention(q, self.out, lm.w["lam0"], self.lens, causal=True)
            self.ws = torch.empty(self.desc.workspace_bytes, dtype=torch.uint8, device=lm.dev)
            return
        self.k = [zeros(sequences, room, lm.K, 2, lm.D) for _ in range(lm.L)]
        self.v = [zeros(sequences, room, lm.K, 2 * lm.D) for _ in range(lm.L)]
        self.q = zeros(sequences, 1, lm.H, 2, lm.D)
        self.all = torch.arange(sequences, device=lm.dev)
        self.desc = B.diff_attention_desc(self.q, self.k[0], self.v[0], self.out, lm.w["lam0"], causal=True, k_lens=self.lens)
        self.ws = torch.empty(B.diff_attention_workspace_bytes(self.desc, False), dtype=torch.uint8, device=lm.dev)

    def _attend(self, i, q, k, v, at):
        """The new tokens' keys and values into layer i's cache, and its attention into self.out."""
        lam = self.lm.w["lam%d" % i]
        if self.bits == 8:
            cache = self.caches[i]
            cache.write(self.rows, k[:, None], v[:, None])
            cache.attend(self.desc, q[:, None], lam, self.out, self.ws)
            return
        self.q[:, 0] = q
        self.k[i][self.all, at], self.v[i][self.all, at] = k, v
        B.codistill_diff_attention(self.desc, self.q, self.k[i], self.v[i], lam, self.out, workspace=self.ws)

    def step(self, tokens):
        """tokens int64 [sequences], as in DiffLM.forward: logits fp32 [sequences, V] of what follows."""
        lm = self.lm
        tokens = lm._tokens(tokens)
        if self.oldest >= self.room:   # (one past the caches' end; the device is asked only here, whether the old ones have begun anew)
            self.oldest = int(self.lens.max())
            if self.oldest >= self.room:
                raise ValueError("decoder: a sequence has filled the room of %d tokens" % self.room)
        self.oldest += 1
        positions, at = self.lens[None].clone(), None
        if self.bits == 8:
            self.first.copy_(self.lens)
        else:
            at = self.lens.long()
        self.lens += 1
        x = lm._embed(tokens)
        for i in range(lm.L):
            q, k, v, _ = lm._queries_and_keys(lm._norm(x, "norm%d" % i) @ lm.p["qkv%d" % i].t(), i, positions)
            self._attend(i, q, k, v, at)
            n = torch.empty_like(self.out[:, 0])
            B.codistill_head_norm(self.out[:, 0], lm.p["head%d" % i], n, EPS, lm.post)
            x = x + n.flatten(1) @ lm.p["out%d" % i].t()
        return (lm._norm(x, "norm") @ lm.p["embed"].t()).float()

    def prefill(self, tokens, starts, longest):
        """All sequences begin anew with a prompt each, packed: tokens int64 [rows], starts int32 [sequences + 1], the longest one's tokens.  Logits fp32
        [rows, V].  A prompt's tokens see each other as they are; what follows sees what the caches hold of them."""
        lm, rows, ends = self.lm, tokens.numel(), starts.tolist()
        tokens = lm._tokens(tokens)
        lens = [b - a for a, b in zip(ends, ends[1:])]
        if len(lens) != self.S or ends[0] != 0 or ends[-1] != rows or min(lens) < 0 or max(lens) > longest or not 0 < longest <= self.room:
            raise ValueError("decoder: %d packed prompts of up to %d tokens (the longest one given), got starts %s" % (self.S, self.room, ends))
        self.lens.copy_(starts[1:] - starts[:-1])
        self.oldest = max(lens)
        seq = torch.repeat_interleave(torch.arange(self.S, device=lm.dev), self.lens.long(), output_size=rows)
        positions = (torch.arange(rows, device=lm.dev) - starts[seq]).int()[None]
        x = lm._embed(tokens)
        for i in range(lm.L):
            q, k, v, _ = lm._queries_and_keys(lm._norm(x, "norm%d" % i) @ lm.p["qkv%d" % i].t(), i, positions)
            if self.bits == 8:
                self.caches[i].write(self.caches[i].rows(k, v, starts=starts, max_new=longest), k, v)
            else:
                self.k[i][seq, positions[0].long()], self.v[i][seq, positions[0].long()] = k, v
            out, lam = torch.zeros(rows, lm.H, 2 * lm.D, dtype=lm.dt, device=lm.dev), lm.w["lam%d" % i]
            desc = B.diff_attention_desc(q, k, v, out, lam, causal=True, q_starts=starts, k_starts=starts, max_q=longest, max_k=longest)
            ws = torch.empty(B.diff_attention_workspace_bytes(desc, False), dtype=torch.uint8, device=lm.dev)
            B.codistill_diff_attention(desc, q, k, v, lam, out, workspace=ws)
            n = torch.empty_like(out)
            B.codistill_head_norm(out, lm.p["head%d" % i], n, EPS, lm.post)
            x = x + n.flatten(1) @ lm.p["out%d" % i].t()
        return (lm._norm(x, "norm") @ lm.p["embed"].t()).float()


def copying_batch(sequences, half, vocabulary, seed, device="cuda:0"):
    """Packed sequences of a random word list and the same list once more; the second copy is predicted.  tokens, positions, starts, targets."""
    gen = torch.Generator().manual_seed(seed)
    lens = torch.randint(max(2, half // 2), half + 1, (sequences,), generator=gen).tolist()
    tokens, targets, positions = [], [], []
    for n in lens:
        words = torch.randint(0, vocabulary, (n,), generator=gen)
        t = torch.cat([words, words])
        tokens.append(t)
        targets.append(torch.cat([torch.full((n - 1,), -1), t[n:], torch.full((1,), -1)]))
        positions.append(torch.arange(2 * n))
    starts = torch.tensor([0] + [2 * n for n in lens]).cumsum(0)
    return (torch.cat(tokens).to(device), torch.cat(positions).int()[None].to(device), starts.int().to(device), torch.cat(targets).int().to(device))


def codistill_step(models, batch, lr, alpha, longest):
    """One step of each model against the others' logits on the same rows; the losses (total, task, distillation) of each."""
    tokens, positions, starts, targets = batch
    logits = [m.forward(tokens, positions, starts, longest) for m in models]
    losses = []
    for j, m in enumerate(models):
        peers = [z for i, z in enumerate(logits) if i != j]
        dz, loss = torch.empty_like(logits[j]), torch.empty(4, device=m.dev)
        scratch = torch.empty(B.loss_scratch_bytes(*dz.shape), dtype=torch.uint8, device=m.dev)
        B.codistill_loss_grad(logits[j], peers, targets, loss, dz, scratch, alpha, dist_kind=B.CD_DIST_KL)
        m.backward(dz)
        losses.append(loss)
    for m in models:
        m.update(lr)
    return torch.stack(losses)[:, :3]


def main(steps=300, vocabulary=64, half=16):
    models = [DiffLM(vocabulary, seed=s) for s in (1, 2)]
    for t in range(steps):
        batch = copying_batch(64, half, vocabulary, seed=t)
        losses = codistill_step(models, batch, 3e-3 * min(1.0, (t + 1) / 20), alpha=0.5 if t >= 50 else 0.0, longest=2 * half)
        if t % 50 == 0 or t == steps - 1:
            print("step %3d  " % t + "  ".join("task %.3f distill %.3f" % (x[1], x[2]) for x in losses.tolist()), flush=True)
    words = torch.randint(0, vocabulary, (4, half), generator=torch.Generator().manual_seed(10 ** 6)).to("cuda:0")
    for bits in (None, 8):
        decoder, said = models[0].decoder(4, 2 * half, bits), []
        for i in range(2 * half - 1):
            z = decoder.step(words[:, i] if i < half else said[-1])
            if i >= half - 1:
                said.append(z.argmax(1) if i >= half else words[:, 0])   # (the first word of the copy is given)
        print("copied %.0f %% of the words%s" % (100 * (torch.stack(said[1:], 1) == words[:, 1:len(said)]).float().mean(), " from a cache in 8 bits" if bits else ""))


if __name__ == "__main__":
    main()
