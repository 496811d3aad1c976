"""The operators of a differential-attention Transformer layer and of its update, as timed cases.

Kinds:

  attention  differential attention: the difference of two softmax maps, weighted by a learned lambda.  train: forward and backward;
             otherwise the forward pass that keeps nothing, as evaluation and decoding against a cache call it
  rotary     rotary positions of the queries and the keys, several axes; inverse: the gradient's direction
  norm       the norm of every head's output that follows the attention.  train: forward and backward
  adamw      one AdamW update of many tensors, moments in 32 or in 8 bits

Where `own` is false, `run` is the plain form: elementary torch operations in 32 bits.  `exact` computes the same from the definitions in
64 bits.  Both take their inputs from `prepare`.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 256          # elements that share an exponent in the 8-bit moments
M_TOP, V_TOP = 15, 31   # the exponent fields of the top binade: 4 bits beside a sign, 5 bits without one
BETA1, BETA2, ADAM_EPS, LR, STEP_NUMBER = 0.9, 0.999, 1e-8, 1e-3, 7
NORM_EPS = 1e-5


def listed():
    return [
        # a decoder layer of the packed translation batch: 113 sentences of 16 to 128 tokens, model width 512 as 4 heads of 2 x 64
        dict(name="attn_train_packed", kind="attention", train=True, dtype="bf16", packed=True, batch=113, tq=128, tk=128, heads=4, kv_heads=4,
             dim=64, causal=True, lam="head", ragged=True),
        # language-model pretraining on long rows: width 1024 as 8 heads of 2 x 64
        dict(name="attn_train_long", kind="attention", train=True, dtype="bf16", packed=False, batch=2, tq=4096, tk=4096, heads=8, kv_heads=8,
             dim=64, causal=True, lam="head", ragged=False),
        # shared key heads, odd and ragged lengths (one sequence is empty), a lambda for every token and head, the widest heads
        dict(name="attn_train_shared_ragged", kind="attention", train=True, dtype="bf16", packed=False, batch=5, tq=777, tk=777, heads=8, kv_heads=2,
             dim=128, causal=False, lam="token", ragged=True),
        # fp32 throughout, attention over another sequence's keys, as the small models and the parity runs use it
        dict(name="attn_train_cross_f32", kind="attention", train=True, dtype="f32", packed=False, batch=3, tq=77, tk=130, heads=4, kv_heads=4,
             dim=32, causal=False, lam="head", ragged=True),
        # serving: one new token of each of 16 requests against a cache of up to 8192
        dict(name="attn_decode_8k", kind="attention", train=False, dtype="bf16", packed=False, batch=16, tq=1, tk=8192, heads=16, kv_heads=4,
             dim=64, causal=True, lam="head", ragged=True),
        # serving: the positions of one new token of each of 16 requests; nothing but the launch
        dict(name="rotary_one_token", kind="rotary", dtype="bf16", tokens=16, heads=32, kv_heads=8, dim=64, axes="32", layout="halves", inverse=False),
        # a batch of images and text: time, height and width positions over 8192 tokens
        dict(name="rotary_video_8192", kind="rotary", dtype="bf16", tokens=8192, heads=16, kv_heads=16, dim=64, axes="8,12,12", layout="halves", inverse=False),
        # the norm behind a layer's attention, both directions: 8192 tokens of 8 heads
        dict(name="norm_train", kind="norm", train=True, dtype="bf16", rows=8192, heads=8, width=128),
        # the same of a small fp32 model, forward only, at odd sizes
        dict(name="norm_f32", kind="norm", train=False, dtype="f32", rows=300, heads=3, width=80),
        # the update of a two-layer CNN: six tensors, nothing but the launch
        dict(name="adamw_small", kind="adamw", bits=32, grads="f32", tensors="432,16,4608,32,320,10"),
        # the update of the base Transformer, 60.9 M parameters in some 180 tensors, moments in 32 bits
        dict(name="adamw_base_32bit", kind="adamw", bits=32, grads="f32", tensors="transformer:32768,512,6"),
        # the same with moments in 8 bits
        dict(name="adamw_base_8bit", kind="adamw", bits=8, grads="f32", tensors="transformer:32768,512,6"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "decode", "rotary", "norm", "adamw"])
    if kind in ("attention", "decode"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 1, 2, 4])
        dim = rng.choice([32, 64, 64, 128, 24, 80])
        c = dict(kind="attention", dtype=dtype, heads=heads, kv_heads=kv, dim=dim, lam=rng.choice(["head", "token"]), ragged=rng.random() < 0.6)
        if kind == "decode":
            tk = _log(rng, 1, 32768)
            most = max(1, min(64, int(2e8 // (tk * kv * dim * (2 if dtype == "f32" else 1)))))
            return dict(c, train=False, packed=False, batch=_log(rng, 1, most), tq=rng.choice([1, 1, 1, 2, 5]), tk=tk, causal=rng.random() < 0.7)
        most = 8e9 if dtype == "bf16" else 1e9     # batch * heads * queries * keys * dim
        tq = _log(rng, 1, 4096 if dtype == "bf16" else 1024)
        tk = tq if rng.random() < 0.7 else _log(rng, 1, 2048)
        batch = max(1, int(min(_log(rng, 1, 64), most / (heads * tq * tk * dim), 2e8 / (heads * tq * tk))))
        packed = tq == tk and 16 <= tq <= 512 and rng.random() < 0.5
        return dict(c, train=rng.random() < 0.8, packed=packed, ragged=c["ragged"] or packed, batch=batch, tq=tq, tk=tk, causal=rng.random() < 0.5)
    if kind == "rotary":
        dim = rng.choice([32, 64, 128, 40])
        half = dim // 2
        cut = sorted(rng.sample(range(1, half), 2))
        axes = rng.choice(["%d" % half, "%d,%d,%d" % (cut[0], cut[1] - cut[0], half - cut[1]), "%d,%d" % (cut[0], cut[1] - cut[0])])
        kv = rng.choice([1, 2, 4, 8, 16])
        return dict(kind="rotary", dtype=rng.choice(["bf16", "f32"]), tokens=_log(rng, 1, 16384), heads=kv * rng.choice([1, 2, 4]), kv_heads=kv,
                    dim=dim, axes=axes, layout=rng.choice(["halves", "pairs"]), inverse=rng.random() < 0.5)
    if kind == "norm":
        return dict(kind="norm", train=rng.random() < 0.7, dtype=rng.choice(["bf16", "f32"]), rows=_log(rng, 1, 16384), heads=rng.randint(1, 16),
                    width=rng.choice([64, 128, 256, 48, 160, 90]))
    sizes, room = [], 6e7
    for _ in range(_log(rng, 1, 200)):
        n = min(_log(rng, 1, 4e6), int(room))
        if n < 1:
            break
        sizes.append(n)
        room -= n
    return dict(kind="adamw", bits=rng.choice([32, 8]), grads=rng.choice(["f32", "bf16"]), tensors=",".join(map(str, sizes)))


# ---- what the cases hold ------------------------------------------------------------------------------------------------

def _lengths(case):
    """Tokens of every sequence, queries and keys; of the case alone, so that the work can be counted without the inputs."""
    rng = random.Random(case["batch"] * 8191 + case["tq"] * 31 + case["tk"])
    B, tq, tk = case["batch"], case["tq"], case["tk"]
    if not case["ragged"]:
        return [tq] * B, [tk] * B
    if case["packed"]:
        ln = [rng.randint(max(1, tq // 8), tq) for _ in range(B)]
        return ln, ln
    if case["train"] and tq == tk:
        ln = [rng.randint(tk // 2, tk) for _ in range(B)]
        ln[-1] = 0 if B > 1 else ln[-1]
        return ln, ln
    return [tq] * B, [rng.randint(max(1, tk // 4), tk) for _ in range(B)]


def _visible(case):
    """(query, key) pairs that a head sees."""
    n = 0
    for q, k in zip(*_lengths(case)):
        if not case["causal"]:
            n += q * k
        else:            # query i sees the keys up to i + k - q
            lo = max(0, q - k)
            n += (q - lo) * (k - q) + (q * (q + 1) - lo * (lo + 1)) // 2
    return n


def _sizes(case):
    t = case["tensors"]
    if not t.startswith("transformer:"):
        return [int(n) for n in t.split(",")]
    vocabulary, d, layers = (int(n) for n in t.split(":")[1].split(","))
    attention = [3 * d * d, 3 * d, d * d, d, d, d]       # projections in and out with their biases, norm
    cross = [d * d, d, 2 * d * d, 2 * d, d * d, d, d, d]
    ffn = [4 * d * d, 4 * d, 4 * d * d, d, d, d]
    return [vocabulary * d] + layers * (attention + ffn) + layers * (attention + cross + ffn)


def work(case):
    e = 2 if case.get("dtype") == "bf16" else 4
    if case["kind"] == "attention":
        q_lens, k_lens = _lengths(case)
        q = sum(q_lens) * case["heads"] * 2 * case["dim"]
        kv = sum(k_lens) * case["kv_heads"] * 2 * case["dim"]
        per = (32 if case["train"] else 12) * case["dim"] * case["heads"]
        return {"bytes": e * ((4 * q + 4 * kv) if case["train"] else (2 * q + 2 * kv)), "flops": per * _visible(case)}
    if case["kind"] == "rotary":
        n = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * e * n, "flops": 3 * n}
    if case["kind"] == "norm":
        n = case["rows"] * case["heads"] * case["width"]
        return {"bytes": e * n * (4 if case["train"] else 2), "flops": n * (12 if case["train"] else 4)}
    n, g = sum(_sizes(case)), 4 if case["grads"] == "f32" else 2
    moved = n * (8 + 2 + g + (16 if case["bits"] == 32 else 4))
    if case["bits"] == 8:
        moved += n * 4 + 4 * (n // BLOCK)     # the moments come back as the bf16 values that they stand for; two exponents a block, read and written
    return {"bytes": moved, "flops": 14 * n}


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _gen(seed, device):
    return torch.Generator(device=device).manual_seed(seed)


def prepare(case, seed):
    return {"attention": _prepare_attention, "rotary": _prepare_rotary, "norm": _prepare_norm, "adamw": _prepare_adamw}[case["kind"]](case, _gen(seed, DEV))


def _starts(lens):
    return torch.tensor([0] + lens, dtype=torch.int32).cumsum(0, dtype=torch.int32)


def _prepare_attention(case, gen):
    dt, B, H, K, D = TYPES[case["dtype"]], case["batch"], case["heads"], case["kv_heads"], case["dim"]
    q_lens, k_lens = _lengths(case)
    rows_q, rows_k = (sum(q_lens), sum(k_lens)) if case["packed"] else (B * case["tq"], B * case["tk"])
    shape = (lambda n, t, *rest: (n,) + rest) if case["packed"] else (lambda n, t, *rest: (B, t) + rest)

    def rand(n, scale=1.0, to=dt):
        return (torch.randn(n, generator=gen, device=DEV) * scale).to(to)

    s = {"case": case}
    if case["train"] and case["tq"] == case["tk"]:   # the ranges of one fused projection of every row
        fused = rand((rows_q, 2 * D * (H + 2 * K)), 1.2)
        parts = fused.split([2 * D * H, 2 * D * K, 2 * D * K], 1)
        grads = torch.zeros_like(fused)
        dparts = grads.split([2 * D * H, 2 * D * K, 2 * D * K], 1)
    else:                                            # queries of their own beside keys and values (another sequence's, or a cache)
        parts = [rand((rows_q, 2 * D * H), 1.2), rand((rows_k, 2 * D * K), 1.2), rand((rows_k, 2 * D * K), 1.2)]
        dparts = [torch.zeros_like(p) for p in parts] if case["train"] else [None] * 3
    for name, t, n, T, heads in (("q", parts[0], rows_q, case["tq"], H), ("k", parts[1], rows_k, case["tk"], K)):
        s[name] = t.view(*shape(n, T, heads, 2, D))
    s["v"] = parts[2].view(*shape(rows_k, case["tk"], K, 2 * D))
    lam_shape = (H,) if case["lam"] == "head" else shape(rows_q, case["tq"], H)
    s["lam"] = 0.2 + 0.7 * torch.rand(lam_shape, generator=gen, device=DEV)
    s["out"] = torch.zeros(shape(rows_q, case["tq"], H, 2 * D), dtype=dt, device=DEV)
    if case["train"]:
        s["dq"] = dparts[0].view(s["q"].shape)
        s["dk"] = dparts[1].view(s["k"].shape)
        s["dv"] = dparts[2].view(s["v"].shape)
        s["dlam"] = torch.zeros_like(s["lam"])
        s["o2"] = torch.zeros_like(s["out"])
        s["lse"] = torch.zeros(2, H, rows_q, device=DEV)
        s["dout"] = rand(s["out"].shape, 0.02)
    if case["packed"]:
        s["q_starts"] = s["k_starts"] = _starts(q_lens).to(DEV)
        # where the rows lie in a padded copy, for the plain form
        at = torch.cat([i * case["tq"] + torch.arange(n) for i, n in enumerate(q_lens)])
        s["at"] = at.to(DEV)
    s["q_lens"] = torch.tensor(q_lens, dtype=torch.int32, device=DEV)
    s["k_lens"] = torch.tensor(k_lens, dtype=torch.int32, device=DEV)
    if own:
        from paper_2010_02838_amd import binding as B_
        if case["packed"]:
            lens = dict(q_starts=s["q_starts"], k_starts=s["k_starts"], max_q=case["tq"], max_k=case["tk"])
        else:
            lens = dict(q_lens=s["q_lens"], k_lens=s["k_lens"]) if case["ragged"] else {}
        s["desc"] = B_.diff_attention_desc(s["q"], s["k"], s["v"], s["out"], s["lam"], causal=case["causal"], **lens)
        s["ws"] = torch.empty(B_.diff_attention_workspace_bytes(s["desc"], case["train"]), dtype=torch.uint8, device=DEV)
    return s


def _prepare_rotary(case, gen):
    dt, n, D = TYPES[case["dtype"]], case["tokens"], case["dim"]
    axes = [int(a) for a in case["axes"].split(",")]
    x = torch.randn(n, (case["heads"] + case["kv_heads"]) * D, generator=gen, device=DEV).to(dt)   # queries and keys of one projection
    y = torch.empty_like(x)
    q, k = x.split([case["heads"] * D, case["kv_heads"] * D], 1)
    yq, yk = y.split([case["heads"] * D, case["kv_heads"] * D], 1)
    s = {"case": case, "q": q.view(n, -1, D), "k": k.view(n, -1, D), "yq": yq.view(n, -1, D), "yk": yk.view(n, -1, D)}
    s["pos"] = torch.randint(0, 32768, (len(axes), n), generator=gen, device=DEV, dtype=torch.int32)
    # one ladder of frequencies over all pairs; the sections say which axis' position turns a pair; pairs behind the last section stay
    pair_axis = [a for a, m in enumerate(axes) for _ in range(m)]
    s["axis"] = torch.tensor(pair_axis, device=DEV)
    s["freq"] = torch.pow(10000.0, -torch.arange(len(pair_axis), dtype=torch.float64) * 2 / D).to(DEV)
    if own:
        from paper_2010_02838_amd import binding as B_
        s["desc"] = B_.rotary_desc(D, axes, 10000.0, dt, layout=B_.CD_ROPE_HALVES if case["layout"] == "halves" else B_.CD_ROPE_PAIRS)
    return s


def _prepare_norm(case, gen):
    dt, shape = TYPES[case["dtype"]], (case["rows"], case["heads"], case["width"])
    s = {"case": case, "x": (torch.randn(shape, generator=gen, device=DEV) * 0.3).to(dt), "y": torch.empty(shape, dtype=dt, device=DEV)}
    s["gain"] = (1 + 0.1 * torch.randn(case["width"], generator=gen, device=DEV)).to(dt)
    if case["train"]:
        s["dy"] = (torch.randn(shape, generator=gen, device=DEV) * 0.02).to(dt)
        s["dx"] = torch.empty_like(s["x"])
        s["dgain"] = torch.empty(case["width"], device=DEV)
    if own:
        from paper_2010_02838_amd import binding as B_
        s["ws"] = torch.empty(B_.head_norm_workspace_bytes(*shape), dtype=torch.uint8, device=DEV)
    return s


def _prepare_adamw(case, gen):
    sizes = _sizes(case)
    blocks = [-(-n // BLOCK) for n in sizes]
    total = sum(blocks) * BLOCK
    at, base = [], 0
    for b in blocks:
        at.append(base * BLOCK)
        base += b
    # one padded buffer: the plain form works on all of it at once, the update on its parts
    real = torch.zeros(total, dtype=torch.bool, device=DEV)
    for a, n in zip(at, sizes):
        real[a:a + n] = True
    s = {"case": case, "w": torch.randn(total, generator=gen, device=DEV) * 0.05 * real}
    # gradients of several orders of magnitude from tensor to tensor and inside one
    size = torch.exp2(torch.randint(-6, 3, (total // BLOCK, 1), generator=gen, device=DEV).float()).expand(-1, BLOCK).reshape(-1)
    size = size * 1e-3 * real
    s["g"] = (torch.randn(total, generator=gen, device=DEV) * size).to(TYPES[case["grads"]])
    m = torch.randn(total, generator=gen, device=DEV) * size * 0.3
    v = torch.square(torch.randn(total, generator=gen, device=DEV) * size) + 0.05 * torch.square(size)
    s["lowp"] = torch.zeros(total, dtype=torch.bfloat16, device=DEV)
    s["decay"] = torch.tensor([0.1 if n > 4096 else 0.0 for n in sizes], device=DEV).repeat_interleave(torch.tensor(blocks, device=DEV))[:, None]
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        half = torch.full((1, 1), 1 << 19, dtype=torch.int64, device=DEV)
        (cm, em), (cv, ev) = _encode(m, half, M_TOP, True), _encode(v, half, V_TOP, False)
        s["m"], s["v"] = cm, cv
        s["exps"] = torch.stack([em, ev], 1).contiguous()
        s["mo"], s["vo"] = torch.zeros(total, dtype=torch.bfloat16, device=DEV), torch.zeros(total, dtype=torch.bfloat16, device=DEV)
        s["seed"] = int(torch.randint(0, 1 << 31, (1,), generator=gen, device=DEV))
    if own:
        from paper_2010_02838_amd.adamw import AdamW
        parts = lambda t: [t[a:a + n] for a, n in zip(at, sizes)]   # noqa: E731
        state = {"m": parts(s["m"]), "v": parts(s["v"])}
        if case["bits"] == 8:
            state["exps"] = [s["exps"][a // BLOCK:a // BLOCK + b] for a, b in zip(at, blocks)]
        s["opt"] = AdamW(parts(s["w"]), parts(s["g"]), parts(s["lowp"]), weight_decay=[0.1 if n > 4096 else 0.0 for n in sizes],
                         state_bits=case["bits"], state=state)
        s["opt_out"] = (parts(s["mo"]), parts(s["vo"])) if case["bits"] == 8 else None
        if case["bits"] == 8:
            s["unpack"] = s["opt"].unpack_plan(*s["opt_out"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"attention": _own_attention, "rotary": _own_rotary, "norm": _own_norm, "adamw": _own_adamw}[kind](s)
    return {"attention": _plain_attention, "rotary": _plain_rotary, "norm": _plain_norm, "adamw": _plain_adamw}[kind](s)


def _attention_outputs(s, train):
    return {n: s[n] for n in (("out", "dq", "dk", "dv", "dlam") if train else ("out",))}


def _own_attention(s):
    from paper_2010_02838_amd import binding as B_
    train = s["case"]["train"]
    B_.codistill_diff_attention(s["desc"], s["q"], s["k"], s["v"], s["lam"], s["out"], s.get("o2"), s.get("lse"), s["ws"])
    if train:
        B_.codistill_diff_attention_backward(s["desc"], s["q"], s["k"], s["v"], s["lam"], s["out"], s["o2"], s["lse"], s["dout"],
                                             s["dq"], s["dk"], s["dv"], s["dlam"], s["ws"])
    return _attention_outputs(s, train)


def _own_rotary(s):
    from paper_2010_02838_amd import binding as B_
    B_.codistill_rotary(s["desc"], s["pos"], [(s["q"], s["yq"]), (s["k"], s["yk"])], inverse=s["case"]["inverse"])
    return {"q": s["yq"], "k": s["yk"]}


def _own_norm(s):
    from paper_2010_02838_amd import binding as B_
    B_.codistill_head_norm(s["x"], s["gain"], s["y"], NORM_EPS, 0.8)
    if not s["case"]["train"]:
        return {"y": s["y"]}
    B_.codistill_head_norm_backward(s["x"], s["gain"], s["dy"], s["dx"], s["dgain"], s["ws"], NORM_EPS, 0.8)
    return {"y": s["y"], "dx": s["dx"], "dgain": s["dgain"]}


def _own_adamw(s):
    if s["case"]["bits"] == 32:
        s["opt"].step(LR, STEP_NUMBER, BETA1, BETA2, ADAM_EPS)
        return {"w": s["w"], "lowp": s["lowp"], "m": s["m"], "v": s["v"]}
    s["opt"].step(LR, STEP_NUMBER, BETA1, BETA2, ADAM_EPS, seed=s["seed"])
    s["opt"].unpack(s["unpack"])
    return {"w": s["w"], "lowp": s["lowp"], "m": s["mo"], "v": s["vo"]}


# ---- the plain forms ------------------------------------------------------------------------------------------------------------

def _padded(s, t, T):
    """[B, T, ...] in 32 bits, whether the rows are packed or not."""
    c = s["case"]
    if not c["packed"]:
        return t.float()
    p = torch.zeros((c["batch"] * T,) + t.shape[1:], device=t.device)
    p[s["at"]] = t.float()
    return p.view(c["batch"], T, *t.shape[1:])


def _rows(s, t, like):
    """Back to the rows' own layout and type."""
    if s["case"]["packed"]:
        t = t.flatten(0, 1)[s["at"]]
    return t.to(like.dtype)


def _plain_attention(s):
    c = s["case"]
    B, Tq, Tk, H, K, D = c["batch"], c["tq"], c["tk"], c["heads"], c["kv_heads"], c["dim"]
    G = H // K
    q = _padded(s, s["q"], Tq).view(B, Tq, K, G, 2, D).permute(0, 2, 3, 4, 1, 5)                       # [B, K, G, 2, Tq, D]
    k = _padded(s, s["k"], Tk).permute(0, 2, 3, 1, 4)[:, :, None].expand(-1, -1, G, -1, -1, -1)        # [B, K, G, 2, Tk, D]
    v = _padded(s, s["v"], Tk).permute(0, 2, 1, 3)[:, :, None].expand(-1, -1, G, -1, -1)               # [B, K, G, Tk, 2D]
    lam = s["lam"].view(1, K, G, 1, 1) if c["lam"] == "head" else _padded(s, s["lam"], Tq).view(B, Tq, K, G, 1).permute(0, 2, 3, 1, 4)
    i, j = torch.arange(Tq, device=q.device)[:, None], torch.arange(Tk, device=q.device)
    nq, nk = s["q_lens"].view(B, 1, 1), s["k_lens"].view(B, 1, 1)
    see = (i < nq) & (j < nk)
    if c["causal"]:
        see = see & (j <= i + nk - nq)
    see = see.view(B, 1, 1, 1, Tq, Tk)
    scale = D ** -0.5
    sc = torch.matmul(q, k.transpose(-1, -2)) * scale
    sc = sc.masked_fill(~see, -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = torch.matmul(p, v[:, :, :, None])                                                              # [B, K, G, 2, Tq, 2D]
    out = o[:, :, :, 0] - lam * o[:, :, :, 1]

    def back(t, heads, like):    # [B, K, G, T, w] -> [B, T, heads, w]
        return _rows(s, t.permute(0, 3, 1, 2, 4).reshape(B, t.shape[3], heads, -1), like).view(like.shape)

    res = {"out": back(out, H, s["out"])}
    if not c["train"]:
        return res
    do = _padded(s, s["dout"], Tq).view(B, Tq, K, G, 2 * D).permute(0, 2, 3, 1, 4)
    dp = torch.matmul(do, v.transpose(-1, -2))[:, :, :, None]                                          # [B, K, G, 1, Tq, Tk]
    delta = (p * dp).sum(-1, keepdim=True)
    weight = torch.stack([torch.ones_like(lam), -lam], 3)                                              # [., K, G, 2, ., 1]
    ds = weight * p * (dp - delta) * scale
    res["dq"] = back(torch.matmul(ds, k).permute(0, 1, 2, 4, 3, 5).flatten(-2), H, s["dq"])
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(2)                                                  # [B, K, 2, Tk, D]
    res["dk"] = _rows(s, dk.permute(0, 3, 1, 2, 4), s["dk"])
    dv = torch.matmul((weight * p).sum(3).transpose(-1, -2), do).sum(2)                                # [B, K, Tk, 2D]
    res["dv"] = _rows(s, dv.permute(0, 2, 1, 3), s["dv"])
    dl = -delta[:, :, :, 1]                                                                            # [B, K, G, Tq, 1]
    res["dlam"] = dl.sum((0, 3, 4)).view(H) if c["lam"] == "head" else back(dl, H, s["lam"])
    return res


def _plain_rotary(s):
    c = s["case"]
    # the angle in 64 bits: at a position of 30000 a 32-bit product is a thousandth of a radian off
    a = s["pos"].double()[s["axis"]].t() * s["freq"] * (-1.0 if c["inverse"] else 1.0)
    cos, sin = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    n, half = a.shape[1], c["dim"] // 2

    def turn(x):
        x = x.float()
        first, second = (x[..., :half], x[..., half:]) if c["layout"] == "halves" else (x[..., 0::2], x[..., 1::2])
        y1 = torch.cat([first[..., :n] * cos - second[..., :n] * sin, first[..., n:]], -1)
        y2 = torch.cat([second[..., :n] * cos + first[..., :n] * sin, second[..., n:]], -1)
        y = torch.cat([y1, y2], -1) if c["layout"] == "halves" else torch.stack([y1, y2], -1).flatten(-2)
        return y.to(s["q"].dtype)

    return {"q": turn(s["q"]), "k": turn(s["k"])}


def _plain_norm(s):
    x, gain = s["x"].float(), s["gain"].float() * 0.8
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + NORM_EPS)
    xhat = x * r
    res = {"y": (xhat * gain).to(s["x"].dtype)}
    if s["case"]["train"]:
        dy = s["dy"].float()
        h = dy * gain
        res["dx"] = (r * (h - xhat * (h * xhat).mean(-1, keepdim=True))).to(s["x"].dtype)
        res["dgain"] = 0.8 * (dy * xhat).sum((0, 1))
    return res


def _decode(code, exps, top, signed):
    """The values that 8-bit floats with a shared exponent stand for."""
    code = code.view(-1, BLOCK).to(torch.int32)
    size = ((code & 127 if signed else code) << 20).view(torch.float32) * 2.0 ** (127 - top)
    value = size * (exps[:, None].to(torch.int32) << 23).view(torch.float32)      # 2^(e - 127)
    return torch.where(code > 127, -value, value) if signed else value


def _encode(x, rnd, top, signed):
    """Codes and exponents of the values x in blocks; rnd: 20 random bits an element (half of their range: round to nearest)."""
    x = x.view(-1, BLOCK)
    bits = x.abs().view(torch.int32)
    e = torch.clamp((bits.amax(1, keepdim=True) + 0xFFFFF) >> 23, min=40)
    y = x.abs() * ((254 - e) << 23).view(torch.float32) * 2.0 ** (top - 127)       # 2^(127 - e), then to where the code's bits begin
    code = (y.view(torch.int32).to(torch.int64) + rnd) >> 20
    if signed:
        code = code | ((x < 0).to(torch.int64) << 7)
    else:
        code = torch.where(y > 0, code.clamp(min=1), code)
    return code.to(torch.uint8).view(-1), e.view(-1).to(torch.uint8)


def _random_bits(n, seed, device):
    """The update's generator: one 32-bit number an element, from its place among all blocks and the seed."""
    x = (torch.arange(n, dtype=torch.int64, device=device) + seed * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x6C8E9CF5) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x52DCE729) & 0xFFFFFFFF
    x = (x ^ (x >> 16)).view(-1, BLOCK)
    return ((x & 0xFFFF) << 4) | 8, ((x >> 16) << 4) | 8


def _plain_adamw(s):
    c = s["case"]
    w, g = s["w"].view(-1, BLOCK), s["g"].float().view(-1, BLOCK)
    small = c["bits"] == 8
    if small:
        m, v = _decode(s["m"], s["exps"][:, 0], M_TOP, True), _decode(s["v"], s["exps"][:, 1], V_TOP, False)
    else:
        m, v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    c1, c2 = 1 - BETA1 ** STEP_NUMBER, 1 - BETA2 ** STEP_NUMBER
    w = w * (1 - LR * s["decay"]) - (LR / c1) * m / (torch.sqrt(v) * (1 / math.sqrt(c2)) + ADAM_EPS)
    s["w"].copy_(w.view(-1))
    s["lowp"].copy_(s["w"])
    if not small:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
        return {"w": s["w"], "lowp": s["lowp"], "m": s["m"], "v": s["v"]}
    rm, rv = _random_bits(w.numel(), s["seed"], w.device)
    (cm, em), (cv, ev) = _encode(m, rm, M_TOP, True), _encode(v, rv, V_TOP, False)
    s["m"].copy_(cm)
    s["v"].copy_(cv)
    s["exps"].copy_(torch.stack([em, ev], 1))
    return {"w": s["w"], "lowp": s["lowp"], "m": _decode(cm, em, M_TOP, True).view(-1).bfloat16(), "v": _decode(cv, ev, V_TOP, False).view(-1).bfloat16()}


# ---- 64 bits ------------------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return {"attention": _exact_attention, "rotary": _exact_rotary, "norm": _exact_norm, "adamw": _exact_adamw}[case["kind"]](s)


def _softmax64(x, see):
    """Softmax over the visible keys; zeros in a row that sees none."""
    x = x.masked_fill(~see, -1e300)
    e = torch.exp(x - x.detach().max(-1, keepdim=True).values) * see
    return e / (e.sum(-1, keepdim=True) + (~see.any(-1, keepdim=True)))


def _exact_attention(s):
    c = s["case"]
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    q_lens, k_lens = _lengths(c)
    res = {n: torch.zeros(s[n].shape, dtype=torch.float64, device=DEV) for n in _attention_outputs(s, c["train"])}
    q_at = k_at = 0
    for b in range(c["batch"]):
        nq, nk = q_lens[b], k_lens[b]
        rows = (slice(q_at, q_at + nq),) if c["packed"] else (b, slice(0, nq))
        keys = (slice(k_at, k_at + nk),) if c["packed"] else (b, slice(0, nk))
        q_at, k_at = q_at + nq, k_at + nk
        if not nq or not nk:
            continue
        see = torch.ones(nq, nk, dtype=torch.bool, device=DEV)
        if c["causal"]:
            see = see.tril(nk - nq)
        for h in range(H):
            kh = h // (H // K)
            q, k, v = (t.detach().double().requires_grad_(c["train"]) for t in (s["q"][rows + (h,)], s["k"][keys + (kh,)], s["v"][keys + (kh,)]))
            lam = (s["lam"][h] if c["lam"] == "head" else s["lam"][rows + (h,)][:, None]).double().requires_grad_(c["train"])
            a = [_softmax64(q[:, m] @ k[:, m].t() / math.sqrt(D), see) @ v for m in (0, 1)]
            out = a[0] - lam * a[1]
            res["out"][rows + (h,)] = out.detach()
            if c["train"]:
                out.backward(s["dout"][rows + (h,)].double())
                res["dq"][rows + (h,)] = q.grad
                res["dk"][keys + (kh,)] += k.grad
                res["dv"][keys + (kh,)] += v.grad
                if c["lam"] == "head":
                    res["dlam"][h] += lam.grad
                else:
                    res["dlam"][rows + (h,)] = lam.grad[:, 0]
    return res


def _exact_rotary(s):
    c = s["case"]
    res = {}
    for name in ("q", "k"):
        x = s[name].double()
        y = x.clone()
        for p in range(s["axis"].numel()):
            i, j = (p, p + c["dim"] // 2) if c["layout"] == "halves" else (2 * p, 2 * p + 1)
            a = s["pos"][int(s["axis"][p])].double() * 10000.0 ** (-2.0 * p / c["dim"])
            a = (-a if c["inverse"] else a)[:, None]
            y[..., i] = x[..., i] * a.cos() - x[..., j] * a.sin()
            y[..., j] = x[..., j] * a.cos() + x[..., i] * a.sin()
        res[name] = y
    return res


def _exact_norm(s):
    train = s["case"]["train"]
    x, gain = s["x"].double().requires_grad_(train), s["gain"].double().requires_grad_(train)
    y = 0.8 * gain * x / ((x ** 2).mean(-1, keepdim=True) + NORM_EPS).sqrt()
    if not train:
        return {"y": y}
    y.backward(s["dy"].double())
    return {"y": y.detach(), "dx": x.grad, "dgain": gain.grad}


def _round64(x, rnd, lowest):
    """x in blocks, rounded to 8-bit floats that share an exponent: the top binade of a block begins at a power of two such that no value
    exceeds 1.875 of it, three mantissa bits, exponents down to 2^lowest of it and equally spaced values below."""
    top = x.abs().amax(1, keepdim=True)
    mantissa, e = torch.frexp(top)                       # top = mantissa 2^e, mantissa in [0.5, 1)
    e = torch.where(mantissa * 2 > 1.875, e, e - 1).clamp(min=40 - 127)
    y = torch.ldexp(x.abs(), -e)
    own_e = torch.frexp(y)[1] - 1
    step = torch.ldexp(torch.ones_like(y), own_e.clamp(min=lowest) - 3)
    code = torch.floor(y / step + rnd.double() / 2 ** 20)
    if lowest == 1 - V_TOP:
        code = torch.where(y > 0, code.clamp(min=1), code)
    return torch.ldexp(code * step, e) * torch.sign(x)


def _exact_adamw(s):
    c = s["case"]
    small = c["bits"] == 8
    w, g = s["w"].double().view(-1, BLOCK), s["g"].double().view(-1, BLOCK)
    if small:
        m, v = _decode(s["m"], s["exps"][:, 0], M_TOP, True).double(), _decode(s["v"], s["exps"][:, 1], V_TOP, False).double()
    else:
        m, v = s["m"].double().view(-1, BLOCK), s["v"].double().view(-1, BLOCK)
    m = m + (1 - BETA1) * (g - m)
    v = v + (1 - BETA2) * (g ** 2 - v)
    mean, square = m / (1 - BETA1 ** STEP_NUMBER), v / (1 - BETA2 ** STEP_NUMBER)
    w = w - LR * s["decay"].double() * w - LR * mean / (square.sqrt() + ADAM_EPS)
    if small:
        rm, rv = _random_bits(w.numel(), s["seed"], DEV)
        m, v = _round64(m, rm, 1 - M_TOP), _round64(v, rv, 1 - V_TOP)
    return {"w": w.view(-1), "lowp": w.view(-1), "m": m.view(-1), "v": v.view(-1)}
