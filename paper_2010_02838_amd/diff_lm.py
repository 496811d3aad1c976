"""A small language model of differential-attention layers, trained by codistillation and decoded token by token.

Every layer is x + W_o headnorm(diffattn(rotary(q), rotary(k), v)), q, k, v = W_qkv norm(x); the logits are taken against the tied embedding table.
The operators of the layer, the loss against the peers' logits and the update are the library's kernels; the projections are plain matrix
products (torch), and the gradient of the embedding adds the rows of a word in their order, so that the same batch gives the same
bits.  Sequences are packed: `starts` says where each begins.  fp32 throughout, or with dtype=torch.bfloat16 bf16 weights and activations beside an fp32 residual stream and fp32 masters.  (Where the two maps of a head are alike and lambda is near
one, their difference is small and the roundings of bf16 queries and keys are not: at lambda 0.9 a gradient of a two-layer model is off by 2.5 %, at 0.3 by 1 %.)

    python -m paper_2010_02838_amd.diff_lm        trains two models on a copying task, each against the other's logits, and decodes from one
"""
import math

import torch

from . import binding as B
from .adamw import AdamW

EPS = 1e-5


class DiffLM:
    """width: of the residual stream; None: that of all heads' outputs."""

    def __init__(self, vocabulary, layers=2, heads=4, kv_heads=2, head_dim=32, theta=10000.0, lambda_init=0.8, state_bits=8, seed=0, dtype=torch.float32,
                 device="cuda:0", width=None):
        self.V, self.L, self.H, self.K, self.D, self.dev = vocabulary, layers, heads, kv_heads, head_dim, device
        every = heads * 2 * head_dim
        self.d, self.post, self.dt = width or every, 1.0 - lambda_init, dtype
        if not 1 <= self.d <= B.HEAD_NORM_MAX_WIDTH:
            raise ValueError("diff_lm: a residual stream of %d channels, %d at most: give a width" % (self.d, B.HEAD_NORM_MAX_WIDTH))
        self.qkv = 2 * head_dim * (heads + 2 * kv_heads)
        gen = torch.Generator(device=device).manual_seed(seed)
        d = self.d
        shapes = [("embed", (vocabulary, d), d ** -0.5)]
        for i in range(layers):
            shapes += [("norm%d" % i, (d,), None), ("qkv%d" % i, (self.qkv, d), d ** -0.5), ("lam%d" % i, (heads,), None),
                       ("head%d" % i, (2 * head_dim,), None), ("out%d" % i, (d, every), every ** -0.5 / math.sqrt(2 * layers))]
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

    def forward(self, tokens, positions, starts, longest):
        """Logits fp32 [rows, V]; keeps what backward() needs.  tokens int64 [rows], positions int32 [1, rows], starts int32 [sequences + 1]."""
        rows, dev, dt = tokens.numel(), self.dev, self.dt
        x = self.p["embed"][tokens].float()
        layers = []
        for i in range(self.L):
            y = self._norm(x, "norm%d" % i)
            q, k, v = self._split(y @ self.p["qkv%d" % i].t())
            self._turn(q, k, positions)
            out, o2 = torch.zeros(rows, self.H, 2 * self.D, dtype=dt, device=dev), torch.empty(rows, self.H, 2 * self.D, dtype=dt, device=dev)   # (zero where rows belong to no sequence)
            lse = torch.empty(2, self.H, rows, device=dev)
            lam = self.w["lam%d" % i]
            desc = B.diff_attention_desc(q, k, v, out, lam, causal=True, q_starts=starts, k_starts=starts, max_q=longest, max_k=longest)
            ws = torch.empty(B.diff_attention_workspace_bytes(desc, True), dtype=torch.uint8, device=dev)
            B.codistill_diff_attention(desc, q, k, v, lam, out, o2, lse, ws)
            n = torch.empty_like(out)
            B.codistill_head_norm(out, self.p["head%d" % i], n, EPS, self.post)
            layers.append((x, y, q, k, v, out, o2, lse, desc, ws, n))
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
            x, y, q, k, v, out, o2, lse, desc, ws, n = layers[i]
            dxb = dx.to(self.dt)
            self.g["out%d" % i].copy_(dxb.t() @ n.flatten(1))
            dn = (dxb @ self.p["out%d" % i]).view_as(n)
            nws = torch.empty(B.head_norm_workspace_bytes(*n.shape), dtype=torch.uint8, device=self.dev)
            B.codistill_head_norm_backward(out, self.p["head%d" % i], dn, dn, self.g["head%d" % i], nws, EPS, self.post)
            fused = torch.zeros(x.shape[0], self.qkv, dtype=self.dt, device=self.dev)   # (zero where rows belong to no sequence)
            dq, dk, dv = self._split(fused)
            B.codistill_diff_attention_backward(desc, q, k, v, self.w["lam%d" % i], out, o2, lse, dn, dq, dk, dv, self.g["lam%d" % i], ws)
            self._turn(dq, dk, positions, inverse=True)
            self.g["qkv%d" % i].copy_(fused.t() @ y)
            dx = dx + self._norm_backward(x, "norm%d" % i, fused @ self.p["qkv%d" % i])
        self.g["embed"].index_put_((tokens,), dx, accumulate=True)   # (sorted by word and added in the rows' order: index_add_'s order changes from run to run)

    def update(self, lr):
        self.updates += 1
        self.opt.step(lr, self.updates, 0.9, 0.99, 1e-8, seed=self.updates)

    def decoder(self, sequences, room):
        return Decoder(self, sequences, room)


class Decoder:
    """One token at a time for several sequences, against caches of rotated keys and of values.  lens: the sequences' ages, on the device; a sequence
    whose age is set to zero begins anew."""

    def __init__(self, lm, sequences, room):
        self.lm, self.S, self.room = lm, sequences, room
        zeros = lambda *shape: torch.zeros(shape, dtype=lm.dt, device=lm.dev)   # noqa: E731
        self.k = [zeros(sequences, room, lm.K, 2, lm.D) for _ in range(lm.L)]
        self.v = [zeros(sequences, room, lm.K, 2 * lm.D) for _ in range(lm.L)]
        self.lens = torch.zeros(sequences, dtype=torch.int32, device=lm.dev)
        self.oldest = 0   # no sequence is older
        self.out = zeros(sequences, 1, lm.H, 2 * lm.D)
        self.q = zeros(sequences, 1, lm.H, 2, lm.D)
        self.all = torch.arange(sequences, device=lm.dev)
        self.desc = B.diff_attention_desc(self.q, self.k[0], self.v[0], self.out, lm.w["lam0"], causal=True, k_lens=self.lens)
        self.ws = torch.empty(B.diff_attention_workspace_bytes(self.desc, False), dtype=torch.uint8, device=lm.dev)

    def step(self, tokens):
        """tokens int64 [sequences]: logits fp32 [sequences, V] of what follows."""
        lm = self.lm
        if self.oldest >= self.room:   # (one past the caches' end; the device is asked only here, whether the old ones have begun anew)
            self.oldest = int(self.lens.max())
            if self.oldest >= self.room:
                raise ValueError("decoder: a sequence has filled the room of %d tokens" % self.room)
        self.oldest += 1
        positions, at = self.lens[None].clone(), self.lens.long()
        self.lens += 1
        x = lm.p["embed"][tokens].float()
        for i in range(lm.L):
            q, k, v = lm._split(lm._norm(x, "norm%d" % i) @ lm.p["qkv%d" % i].t())
            lm._turn(q, k, positions)
            self.q[:, 0] = q
            self.k[i][self.all, at], self.v[i][self.all, at] = k, v
            B.codistill_diff_attention(self.desc, self.q, self.k[i], self.v[i], lm.w["lam%d" % i], self.out, workspace=self.ws)
            n = torch.empty_like(self.out[:, 0])
            B.codistill_head_norm(self.out[:, 0], lm.p["head%d" % i], n, EPS, lm.post)
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
    decoder, said = models[0].decoder(4, 2 * half), []
    for i in range(2 * half - 1):
        z = decoder.step(words[:, i] if i < half else said[-1])
        if i >= half - 1:
            said.append(z.argmax(1) if i >= half else words[:, 0])   # (the first word of the copy is given)
    print("copied %.0f %% of the words" % (100 * (torch.stack(said[1:], 1) == words[:, 1:len(said)]).float().mean()))


if __name__ == "__main__":
    main()
