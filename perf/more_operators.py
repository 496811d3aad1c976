"""The operators of a language model between its tokens, its attention and its cache, as timed cases.

Kinds:

  normrot   the norm of every query's and key's channels with the position rotation behind it, queries and keys with a gain each.  train:
            forward and backward
  write     keys and values of new tokens go to an 8-bit cache of pages and are read back as the values that it holds
  attend    differential attention of new tokens against such a cache
  embed     embedding lookup with a factor, and the gradient of its table

Where `own` is false, `run` is the plain form: elementary torch operations in 32 bits (64 for angles and for the codes, whose borders 32 bits
would blur).  `exact` computes the same from the definitions in 64 bits.  Both take their inputs from `prepare`.

The cache: a pool of pages of P tokens.  Keys [pages][key heads][P][2][head_dim padded to 32] and values [pages][key heads][2 head_dim][P] are codes in
-127..127, scales bf16 [pages][key heads][3][P] belong to the two maps' keys and to the value of a token; page table [sequences][pages of a
sequence].  A scale is the smallest bf16 number that is at least the largest magnitude over 127, a code the value over its scale, rounded to
nearest even.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
THETA = 10000.0
LEAST = 2.0 ** -100   # the smallest scale


def listed():
    return [
        # decoding: one new token of each of 16 requests, 16 heads of 2 x 64 on 4; nothing but the launch
        dict(name="normrot_one_token", kind="normrot", train=False, dtype="bf16", tokens=16, heads=32, kv_heads=8, dim=64, pairs=32, layout="halves"),
        # a training batch of 8192 tokens: 8 heads of 2 x 64 and as many keys, both directions
        dict(name="normrot_train_8192", kind="normrot", train=True, dtype="bf16", tokens=8192, heads=16, kv_heads=16, dim=64, pairs=32, layout="halves"),
        # a small fp32 model at odd sizes; the last channels are not turned, neighbours are
        dict(name="normrot_train_f32", kind="normrot", train=True, dtype="f32", tokens=333, heads=6, kv_heads=3, dim=40, pairs=12, layout="pairs"),
        # decoding: the new keys and values of 16 requests
        dict(name="cache_write_token", kind="write", dtype="bf16", seqs=16, tq=1, kv_heads=4, dim=64, room=8192, page=256, paged=True, packed=False),
        # prompts: 24 packed ones of up to 1024 tokens
        dict(name="cache_write_prompts", kind="write", dtype="bf16", seqs=24, tq=1024, kv_heads=4, dim=64, room=2048, page=128, paged=True, packed=True),
        # decoding: one new token of each of 16 requests against up to 8192 earlier ones
        dict(name="cache_decode_8k", kind="attend", dtype="bf16", seqs=16, tq=1, heads=16, kv_heads=4, dim=64, room=8192, page=256, paged=True, causal=True,
             lam="head"),
        # decoding: a single request with a long document in front
        dict(name="cache_decode_long", kind="attend", dtype="bf16", seqs=1, tq=1, heads=16, kv_heads=2, dim=64, room=131072, page=1024, paged=False, causal=True,
             lam="head"),
        # a few drafted tokens of each request are checked at once; the widest heads, small pages, a lambda for every token and head
        dict(name="cache_draft_wide", kind="attend", dtype="bf16", seqs=5, tq=4, heads=8, kv_heads=2, dim=128, room=4096, page=64, paged=True, causal=True,
             lam="token"),
        # the small fp32 model, short sequences
        dict(name="cache_decode_f32", kind="attend", dtype="f32", seqs=3, tq=1, heads=4, kv_heads=4, dim=32, room=333, page=64, paged=False, causal=True, lam="head"),
        # a training batch of 8192 tokens: the table is tied to the projection, whose gradient is there already
        dict(name="embed_tied_8192", kind="embed", dtype="bf16", rows=8192, words=32768, width=512, tied=True, padded=False),
        # a large batch and a large table of its own
        dict(name="embed_65536", kind="embed", dtype="bf16", rows=65536, words=65536, width=1024, tied=False, padded=False),
        # a small fp32 model; a tenth of the rows is padding
        dict(name="embed_small_f32", kind="embed", dtype="f32", rows=300, words=64, width=256, tied=False, padded=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["normrot", "write", "attend", "attend", "embed"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "normrot":
        dim = rng.choice([32, 64, 64, 128, 40, 96])
        kv = rng.choice([1, 2, 4, 8, 16])
        return dict(kind=kind, train=rng.random() < 0.6, dtype=dtype, tokens=_log(rng, 1, 16384), heads=kv * rng.choice([1, 2, 4]), kv_heads=kv, dim=dim,
                    pairs=rng.choice([dim // 2, dim // 2, dim // 4]), layout=rng.choice(["halves", "pairs"]))
    if kind == "embed":
        width = rng.choice([64, 256, 512, 1024, 200, 333])
        words = _log(rng, 16, 131072)
        words = min(words, 67000000 // width)
        return dict(kind=kind, dtype=dtype, rows=_log(rng, 1, 65536), words=words, width=width, tied=rng.random() < 0.5, padded=rng.random() < 0.3)
    dim = rng.choice([32, 64, 64, 128, 24, 80])
    page = rng.choice([64, 128, 256, 1024])
    if kind == "write":
        tq = rng.choice([1, _log(rng, 2, 2048)])
        return dict(kind=kind, dtype=dtype, seqs=_log(rng, 1, max(1, min(64, 24000 // tq))), tq=tq, kv_heads=rng.choice([1, 2, 4, 8]), dim=dim, room=tq + _log(rng, 1, 4096),
                    page=page, paged=rng.random() < 0.5, packed=tq > 1 and rng.random() < 0.5)
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 4, 8])
    room = _log(rng, 16, 65536)
    seqs = _log(rng, 1, max(1, min(64, int(130e6 // (room * kv * 4 * dim)))))
    return dict(kind=kind, dtype=dtype, seqs=seqs, tq=min(room, rng.choice([1, 1, 1, 2, 5, 16])), heads=heads, kv_heads=kv, dim=dim, room=room, page=page,
                paged=rng.random() < 0.5, causal=rng.random() < 0.8, lam=rng.choice(["head", "token"]))


# ---- what the cases hold ------------------------------------------------------------------------------------------------

def _lengths(case):
    """(tokens in front, new tokens) of every sequence; of the case alone, so that the work can be counted without the inputs."""
    rng = random.Random(case["seqs"] * 8191 + case["room"] * 31 + case["tq"])
    old, new = [], []
    for _ in range(case["seqs"]):
        n = rng.randint(max(1, case["tq"] // 8), case["tq"]) if case.get("packed") else case["tq"]
        most = case["room"] - n
        old.append(rng.randint(most // 4, most) if case["kind"] == "attend" else rng.randint(0, most))
        new.append(n)
    return old, new


def _seq_pages(case):
    return -(-case["room"] // case["page"])


def _words_share(case):
    """How likely each word is: as log((w + 2) / (w + 1)), which falls like 1 / w."""
    w = torch.arange(case["words"], dtype=torch.float64)
    return torch.log((w + 2) / (w + 1)) / math.log(case["words"] + 1)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "normrot":
        n = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": e * n * (4 if case["train"] else 2), "flops": n * (24 if case["train"] else 8)}
    if case["kind"] == "embed":
        rows, w = case["rows"] * (0.9 if case["padded"] else 1.0), case["width"]
        distinct = float((1 - (1 - _words_share(case)) ** rows).sum())
        table = (8 if case["tied"] else 4) * case["words"]      # (fp32 gradients: all written, behind a read where they add to others)
        return {"bytes": int(w * (e * distinct + 2 * e * rows + table) + 8 * case["rows"]), "flops": int(2 * rows * w)}
    old, new = _lengths(case)
    token = case["kv_heads"] * (4 * case["dim"] + 6)
    if case["kind"] == "write":
        n = sum(new)
        return {"bytes": n * (token + 2 * e * case["kv_heads"] * 4 * case["dim"]), "flops": 6 * n * case["kv_heads"] * 4 * case["dim"]}
    pairs = 0
    for o, n in zip(old, new):
        pairs += n * o + (n * (n + 1) // 2 if case["causal"] else n * n)
    rows = case["heads"] * 4 * case["dim"] * sum(new)
    return {"bytes": token * (sum(old) + sum(new)) + e * rows, "flops": 12 * case["dim"] * case["heads"] * pairs}


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return {"normrot": _prepare_normrot, "write": _prepare_write, "attend": _prepare_attend, "embed": _prepare_embed}[case["kind"]](case, gen)


def _prepare_normrot(case, gen):
    dt, n, D, H, K = TYPES[case["dtype"]], case["tokens"], case["dim"], case["heads"], case["kv_heads"]
    x = torch.randn(n, (H + K) * D, generator=gen, device=DEV).to(dt)   # queries and keys of one projection
    y, s = torch.empty_like(x), {"case": case}

    def parts(t):
        return [p.view(n, -1, D) for p in t.split([H * D, K * D], 1)]

    s["x"], s["y"] = parts(x), parts(y)
    s["gain"] = [(1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dt) for _ in range(2)]
    s["pos"] = torch.randint(0, 32768, (1, n), generator=gen, device=DEV, dtype=torch.int32)
    if case["train"]:
        s["dy"] = parts((torch.randn(n, (H + K) * D, generator=gen, device=DEV) * 0.02).to(dt))
        s["dx"] = parts(torch.empty_like(x))
        s["dgain"] = [torch.empty(D, device=DEV) for _ in range(2)]
    if own:
        from paper_2010_02838_amd import binding as B_
        s["desc"] = B_.rotary_desc(D, (case["pairs"],), THETA, dt, layout=B_.CD_ROPE_HALVES if case["layout"] == "halves" else B_.CD_ROPE_PAIRS)
        if case["train"]:
            s["ws"] = torch.empty(B_.norm_rotary_workspace_bytes(s["desc"], n, 2), dtype=torch.uint8, device=DEV)
    return s


def _prepare_cache(case, gen, s):
    """A cache that has been in use: every slot of it holds something."""
    S, K, D, P, sp = case["seqs"], case["kv_heads"], case["dim"], case["page"], _seq_pages(case)
    padded = -(-D // 32) * 32
    s["k"] = torch.zeros(S * sp, K, P, 2, padded, dtype=torch.int8, device=DEV)
    s["k"][..., :D] = (torch.randn(S * sp, K, P, 2, D, generator=gen, device=DEV) * 40).round().clamp(-127, 127).to(torch.int8)
    s["v"] = (torch.randn(S * sp, K, 2 * D, P, generator=gen, device=DEV) * 40).round().clamp(-127, 127).to(torch.int8)
    s["scales"] = (0.02 + 0.02 * torch.rand(S * sp, K, 3, P, generator=gen, device=DEV)).bfloat16()
    s["table"] = (torch.randperm(S * sp, generator=gen, device=DEV) if case["paged"] else torch.arange(S * sp, device=DEV)).int().view(S, sp)
    if own:
        from paper_2010_02838_amd.kv_cache import KVCache
        s["cache"] = KVCache(S, sp * P, K, D, TYPES[case["dtype"]], page_tokens=P, table=s["table"] if case["paged"] else None,
                             buffers=(s["k"], s["v"], s["scales"]))


def _prepare_write(case, gen):
    dt, S, K, D, tq = TYPES[case["dtype"]], case["seqs"], case["kv_heads"], case["dim"], case["tq"]
    old, new = _lengths(case)
    s = {"case": case}
    rows = sum(new)
    # keys and values are ranges of one projection's rows
    fused = torch.randn(rows, 8 * D * K, generator=gen, device=DEV) * torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device=DEV))
    fused = fused.to(dt)
    shape = (rows,) if case["packed"] else (S, tq)
    s["new_k"], s["new_v"] = fused[:, 4 * D * K:6 * D * K].view(*shape, K, 2, D), fused[:, 6 * D * K:].view(*shape, K, 2 * D)
    s["back_k"], s["back_v"] = torch.empty(*shape, K, 2, D, dtype=dt, device=DEV), torch.empty(*shape, K, 2 * D, dtype=dt, device=DEV)
    s["first"] = torch.tensor(old, dtype=torch.int32, device=DEV)
    # sequence and position of every row, for the plain form
    seq = torch.repeat_interleave(torch.arange(S), torch.tensor(new))
    inside = torch.cat([torch.arange(n) for n in new])
    s["seq"], s["pos"] = seq.to(DEV), (torch.tensor(old)[seq] + inside).to(DEV)
    _prepare_cache(case, gen, s)
    if case["packed"]:
        s["starts"] = torch.tensor([0] + new, dtype=torch.int32).cumsum(0, dtype=torch.int32).to(DEV)
    if own:
        s["rows"] = s["cache"].rows(s["new_k"], s["new_v"], first=s["first"], starts=s.get("starts"), max_new=tq)
        s["back"] = s["cache"].rows(s["back_k"], s["back_v"], first=s["first"], starts=s.get("starts"), max_new=tq)
    return s


def _prepare_attend(case, gen):
    dt, S, H, K, D, tq = TYPES[case["dtype"]], case["seqs"], case["heads"], case["kv_heads"], case["dim"], case["tq"]
    old, new = _lengths(case)
    s = {"case": case}
    _prepare_cache(case, gen, s)
    fused = torch.randn(S, tq, 2 * D * (H + 2 * K), generator=gen, device=DEV).to(dt)
    s["q"] = fused[..., :2 * D * H].view(S, tq, H, 2, D)
    s["lam"] = 0.2 + 0.7 * torch.rand((H,) if case["lam"] == "head" else (S, tq, H), generator=gen, device=DEV)
    s["lens"] = (torch.tensor(old) + torch.tensor(new)).int().to(DEV)
    s["out"] = torch.zeros(S, tq, H, 2 * D, dtype=dt, device=DEV)
    if own:
        s["desc"] = s["cache"].attention(s["q"], s["out"], s["lam"], s["lens"], causal=case["causal"])
        s["ws"] = torch.empty(s["desc"].workspace_bytes, dtype=torch.uint8, device=DEV)
    return s


def _prepare_embed(case, gen):
    dt, n, V, w = TYPES[case["dtype"]], case["rows"], case["words"], case["width"]
    s = {"case": case}
    # log-uniform words: the share of word v falls like 1 / v, as words of a text do
    u = torch.rand(n, generator=gen, device=DEV, dtype=torch.float64)
    s["tokens"] = (torch.exp(u * math.log(V + 1)).long() - 1).clamp(0, V - 1)
    if case["padded"]:
        s["tokens"][torch.rand(n, generator=gen, device=DEV) < 0.1] = -1
    s["scale"] = math.sqrt(w)
    s["table"] = (torch.randn(V, w, generator=gen, device=DEV) * w ** -0.5).to(dt)
    s["dy"] = (torch.randn(n, w, generator=gen, device=DEV) * 0.02).to(dt)
    s["y"] = torch.empty(n, w, dtype=dt, device=DEV)
    s["there"] = torch.randn(V, w, generator=gen, device=DEV) * 0.02 if case["tied"] else None
    s["dtable"] = s["there"].clone() if case["tied"] else torch.empty(V, w, device=DEV)
    if own:
        from paper_2010_02838_amd import binding as B_
        s["ws"] = torch.empty(B_.embedding_workspace_bytes(n, V, w), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"normrot": _own_normrot, "write": _own_write, "attend": _own_attend, "embed": _own_embed}[kind](s)
    return {"normrot": _plain_normrot, "write": _plain_write, "attend": _plain_attend, "embed": _plain_embed}[kind](s)


def _named(s):
    out = {"q": s["y"][0], "k": s["y"][1]}
    if s["case"]["train"]:
        out.update(dq=s["dx"][0], dk=s["dx"][1], dgain_q=s["dgain"][0], dgain_k=s["dgain"][1])
    return out


def _own_normrot(s):
    from paper_2010_02838_amd import binding as B_
    B_.codistill_norm_rotary(s["desc"], s["pos"], list(zip(s["x"], s["gain"], s["y"])), EPS)
    if s["case"]["train"]:
        B_.codistill_norm_rotary_backward(s["desc"], s["pos"], list(zip(s["x"], s["gain"], s["dy"], s["dx"], s["dgain"])), s["ws"], EPS)
    return _named(s)


def _own_write(s):
    s["cache"].write(s["rows"], s["new_k"], s["new_v"])
    s["cache"].read(s["back"], s["back_k"], s["back_v"])
    return {"k": s["back_k"], "v": s["back_v"]}


def _own_attend(s):
    s["cache"].attend(s["desc"], s["q"], s["lam"], s["out"], s["ws"])
    return {"out": s["out"]}


def _own_embed(s):
    from paper_2010_02838_amd import binding as B_
    tied = s["case"]["tied"]
    if tied:
        s["dtable"].copy_(s["there"])     # (the projection's gradient, which a training step writes there in front)
    B_.codistill_embedding(s["tokens"], s["table"], s["y"], s["scale"])
    B_.codistill_embedding_backward(s["tokens"], s["dy"], s["dtable"], s["ws"], s["scale"], accumulate=tied)
    return {"y": s["y"], "dtable": s["dtable"]}


# ---- the plain forms ------------------------------------------------------------------------------------------------------------

def _plain_angles(s):
    c = s["case"]
    freq = torch.pow(THETA, -torch.arange(c["pairs"], dtype=torch.float64, device=DEV) * 2 / c["dim"])
    a = s["pos"][0].double()[:, None] * freq
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _plain_turn(c, x, cos, sin):
    """[tokens, heads, dim], the first pairs turned."""
    n, half = c["pairs"], c["dim"] // 2
    if c["layout"] == "halves":
        a, b, rest_a, rest_b = x[..., :n], x[..., half:half + n], x[..., n:half], x[..., half + n:]
        return torch.cat([a * cos - b * sin, rest_a, b * cos + a * sin, rest_b], -1)
    a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., 2 * n:]], -1)


def _plain_normrot(s):
    c = s["case"]
    cos, sin = _plain_angles(s)

    def forward(x, g):
        v = x.float()
        r = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
        return _plain_turn(c, v * r * g.float(), cos, sin).to(x.dtype)

    def backward(x, g, dy):
        v, d = x.float(), _plain_turn(c, dy.float(), cos, -sin)
        r = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
        xhat, h = v * r, d * g.float()
        return (r * (h - xhat * (h * xhat).mean(-1, keepdim=True))).to(x.dtype), (d * xhat).sum((0, 1))

    (q, k), (gq, gk) = s["x"], s["gain"]
    out = {"q": forward(q, gq), "k": forward(k, gk)}
    if c["train"]:
        (dq, dgq), (dk, dgk) = backward(q, gq, s["dy"][0]), backward(k, gk, s["dy"][1])
        out.update(dq=dq, dk=dk, dgain_q=dgq, dgain_k=dgk)
    return out


def _plain_codes(x):
    """Codes and scales of the last dimension; in 64 bits, as the borders between codes would blur in 32."""
    x = x.double()
    top = x.abs().amax(-1)
    s = (top / 127).clamp(min=LEAST).bfloat16()
    s = torch.where(s.double() * 127 < top, (s.view(torch.int16) + 1).view(torch.bfloat16), s)
    return torch.round(x / s.double()[..., None]).to(torch.int8), s


def _plain_write(s):
    c = s["case"]
    D, P = c["dim"], c["page"]
    new_k, new_v = s["new_k"].reshape(-1, c["kv_heads"], 2, D), s["new_v"].reshape(-1, c["kv_heads"], 2 * D)
    (ck, sk), (cv, sv) = _plain_codes(new_k), _plain_codes(new_v)
    page, slot = s["table"][s["seq"], s["pos"] // P].long(), s["pos"] % P
    s["k"][page, :, slot, :, :D] = ck
    s["v"][page, :, :, slot] = cv
    s["scales"][page, :, :, slot] = torch.cat([sk, sv[..., None]], -1)
    # read back
    held = s["scales"][page, :, :, slot].float()
    k = s["k"][page, :, slot, :, :D].float() * held[..., :2, None]
    v = s["v"][page, :, :, slot].float() * held[..., 2:]
    return {"k": k.to(new_k.dtype).view(s["back_k"].shape), "v": v.to(new_v.dtype).view(s["back_v"].shape)}


def _plain_attend(s):
    c = s["case"]
    S, H, K, D, tq, G = c["seqs"], c["heads"], c["kv_heads"], c["dim"], c["tq"], c["heads"] // c["kv_heads"]
    table = s["table"].long()
    scales = s["scales"][table].float().permute(0, 2, 3, 1, 4).flatten(3)                            # [S, K, 3, T]
    k = s["k"][table][..., :D].float().permute(0, 2, 4, 1, 3, 5).flatten(3, 4)                       # [S, K, 2, T, D]
    v = s["v"][table].float().permute(0, 2, 1, 4, 3).flatten(2, 3)                                   # [S, K, T, 2D]
    T = k.shape[3]
    q = s["q"].float().view(S, tq, K, G, 2, D).permute(0, 2, 4, 1, 3, 5).reshape(S, K, 2, tq * G, D)
    sc = torch.matmul(q, (k * scales[:, :, :2, :, None]).transpose(-1, -2)) * D ** -0.5              # [S, K, 2, tq G, T]
    j, i, n = torch.arange(T, device=DEV), torch.arange(tq, device=DEV).repeat_interleave(G)[:, None], s["lens"].view(S, 1, 1)
    see = (j < n) & (j <= i + n - tq if c["causal"] else j < n)
    sc = sc.masked_fill(~see.view(S, 1, 1, tq * G, T), -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = torch.matmul(p, (v * scales[:, :, 2, :, None])[:, :, None])                                  # [S, K, 2, tq G, 2D]
    o = o.view(S, K, 2, tq, G, 2 * D).permute(2, 0, 3, 1, 4, 5).reshape(2, S, tq, H, 2 * D)
    lam = s["lam"][..., None]
    return {"out": (o[0] - lam * o[1]).to(s["out"].dtype)}


def _plain_embed(s):
    c = s["case"]
    V, seen = c["words"], s["tokens"] >= 0
    at = torch.where(seen, s["tokens"], 0)
    y = torch.where(seen[:, None], s["table"][at].float() * s["scale"], 0.0).to(s["y"].dtype)
    dy = torch.where(seen[:, None], s["dy"].float() * s["scale"], 0.0)
    g = s["there"].clone() if c["tied"] else torch.zeros(V, c["width"], device=DEV)
    return {"y": y, "dtable": g.index_add_(0, at, dy)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"normrot": _exact_normrot, "write": _exact_write, "attend": _exact_attend, "embed": _exact_embed}[case["kind"]](case, s)


def _exact_normrot(case, s):
    """Norm and rotation as one matrix a token: y = R diag(g) x / |x|, with the derivatives of that."""
    D, n = case["dim"], case["pairs"]
    p = torch.arange(n, device=DEV)
    first, second = (p, p + D // 2) if case["layout"] == "halves" else (2 * p, 2 * p + 1)
    angle = s["pos"][0].double()[:, None] / THETA ** (2.0 * p.double() / D)
    R = torch.eye(D, dtype=torch.float64, device=DEV).repeat(case["tokens"], 1, 1)
    R[:, first, first], R[:, second, second] = angle.cos(), angle.cos()
    R[:, first, second], R[:, second, first] = -angle.sin(), angle.sin()
    out = {}
    for name, i in (("q", 0), ("k", 1)):
        x, g = s["x"][i].double(), s["gain"][i].double()
        size = (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt()
        unit = x / size
        out[name] = torch.bmm(unit * g, R.transpose(1, 2).contiguous())
        if case["train"]:
            back = torch.bmm(s["dy"][i].double(), R)
            out["dgain_" + name] = (back * unit).flatten(0, 1).sum(0)
            back = back * g
            out["d" + name] = back / size - x * (back * x).sum(-1, keepdim=True) / (D * size ** 3)
    return {k: out[k] for k in (("q", "k", "dq", "dk", "dgain_q", "dgain_k") if case["train"] else ("q", "k"))}


def _exact_values(x):
    x = x.double()
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True) / 127)          # m in [1/2, 1): a bf16 number has eight bits
    step = torch.ldexp(torch.ceil(m * 256) / 256, e).clamp(min=LEAST)
    return torch.round(x / step) * step


def _exact_write(case, s):
    return {"k": _exact_values(s["new_k"]), "v": _exact_values(s["new_v"])}


def _exact_attend(case, s):
    S, H, K, D, tq, P = case["seqs"], case["heads"], case["kv_heads"], case["dim"], case["tq"], case["page"]
    out = torch.zeros(S, tq, H, 2 * D, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        pages = s["table"][b, :-(-n // P)].long()
        step = s["scales"][pages].double()
        for g in range(K):
            keys = [(s["k"][pages, g, :, m, :D].double() * step[:, g, m, :, None]).flatten(0, 1)[:n] for m in (0, 1)]
            values = (s["v"][pages, g].double() * step[:, g, 2, None, :]).transpose(1, 2).flatten(0, 1)[:n]
            for i in range(tq):
                seen = max(0, n - tq + i + 1) if case["causal"] else n
                if not seen:
                    continue
                h = slice(g * (H // K), (g + 1) * (H // K))
                maps = [torch.softmax(s["q"][b, i, h, m].double() @ keys[m][:seen].t() / math.sqrt(D), 1) for m in (0, 1)]
                lam = (s["lam"][h] if case["lam"] == "head" else s["lam"][b, i, h]).double()[:, None]
                out[b, i, h] = (maps[0] - lam * maps[1]) @ values[:seen]
    return {"out": out}


def _exact_embed(case, s):
    rows = s["tokens"] >= 0
    table = torch.cat([s["table"].double() * s["scale"], torch.zeros(1, case["width"], dtype=torch.float64, device=DEV)])   # (the last row is padding's)
    g = torch.zeros(case["words"], case["width"], dtype=torch.float64, device=DEV)
    g.index_put_((s["tokens"][rows],), s["dy"][rows].double() * s["scale"], accumulate=True)
    if case["tied"]:
        g += s["there"].double()
    return {"y": table[s["tokens"]], "dtable": g}
