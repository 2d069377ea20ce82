"""What the text operators' speed is measured on: the calls of a tenant that reads
prompts, answers token by token and is trained on the next token, over the
repository's own backbone shapes.

Kinds of cases:

  rope          per-head norms of queries and keys with the rotation over several
                position axes, out of the fused projection's rows (a prompt)
  rope_append   the same for the newest token of every live sequence, its key and
                value going into their cache rows
  rope_train    the same with its gradients
  attention     attention of packed prompts, causal behind an optional prefix that
                every row sees; queries may be the last rows of a longer sequence
  attn_train    the same, forward and gradients of q, k and v
  decode        one token of every live sequence against its cache
  loss          next-token losses over the whole vocabulary, no gradient
  loss_train    the same with the gradients of the hidden rows and the vocabulary's
                weights

Lengths are drawn from the case's own numbers, so that a case has the same shapes
for every seed; the seed draws the values.
"""
import math
import random

import torch

own = False  # False: the operators' plain forms; True: the framework's entry points

EPS, THETA, VOCAB = 1e-6, 10000.0, 32000
BF, F32 = torch.bfloat16, torch.float32

# (query heads, key/value heads, head dim): the backbones' own layouts, and grouped
# heads beside them
HEADS = {
    "tiny": (4, 4, 64),
    "small": (16, 16, 64),
    "mqa2b": (8, 1, 256),
    "llama7b": (32, 32, 128),
    "grouped": (32, 8, 128),
    "by3": (12, 4, 128),
    "by7": (14, 2, 64),
}
# frequencies of each position axis (time, height, width), as shares of head_dim / 2
AXES = {1: (1.0,), 2: (0.5, 0.5), 3: (0.25, 0.375, 0.375)}


def listed():
    return [
        # sixteen robots answer, one token each: four times a layer's launches are latency
        dict(name="rope_append_16", kind="rope_append", heads="mqa2b", axes=1, batch=16,
             slots=24, room=640),
        # a packed batch of observations with image positions on the wide backbone
        dict(name="rope_prompt_9k", kind="rope", heads="grouped", axes=3, tokens=9001),
        # the ordinary training microbatch of the narrow backbone
        dict(name="rope_train_30k", kind="rope_train", heads="small", axes=3, tokens=30011),
        # a single short prompt beside two stubs: what a lone request costs
        dict(name="attn_short", kind="attention", heads="mqa2b", seqs=3, longest=300, behind=0,
             prefix=True),
        # a serving batch of ragged prompts, some of them continuing a cached beginning
        dict(name="attn_ragged", kind="attention", heads="grouped", seqs=24, longest=2900,
             behind=700, prefix=False),
        # one long prompt
        dict(name="attn_long", kind="attention", heads="grouped", seqs=1, longest=12289, behind=0,
             prefix=False),
        # image prefix seen by all, text causal behind it: samples of one to three images
        dict(name="attn_train_mqa2b", kind="attn_train", heads="mqa2b", seqs=26, longest=840,
             behind=0, prefix=True),
        # longer documents on the wide backbone
        dict(name="attn_train_llama7b", kind="attn_train", heads="llama7b", seqs=6, longest=2600,
             behind=0, prefix=False),
        # eight robots' next token behind an observation each
        dict(name="decode_8", kind="decode", heads="mqa2b", batch=8, longest=700, room=1024),
        # a full server: ragged long caches
        dict(name="decode_64", kind="decode", heads="grouped", batch=64, longest=8100, room=8192),
        # scoring a few answers
        dict(name="loss_333", kind="loss", d=2048, vocab=VOCAB, rows=333),
        # a training microbatch's text rows on the wide backbone, vocabulary trained too
        dict(name="loss_train_8k", kind="loss_train", d=4096, vocab=VOCAB, rows=8191),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope_append", "rope_train", "attention", "attention",
                       "attn_train", "attn_train", "decode", "decode", "loss", "loss_train",
                       "loss_train"])
    if kind in ("loss", "loss_train"):
        d = rng.choice([256, 1000, 1024, 1928, 2048, 4096])
        return dict(kind=kind, d=d, vocab=rng.choice([VOCAB, _log_int(rng, 1000, VOCAB)]),
                    rows=_log_int(rng, 1, 8191))
    heads = rng.choice(list(HEADS))
    h, hkv, hd = HEADS[heads]
    if kind in ("rope", "rope_train"):
        return dict(kind=kind, heads=heads, axes=rng.randint(1, 3),
                    tokens=_log_int(rng, 1, 36_000_000 // ((h + hkv) * hd)))
    if kind == "rope_append":
        return dict(kind=kind, heads=heads, axes=rng.randint(1, 3), batch=_log_int(rng, 1, 200),
                    slots=200, room=_log_int(rng, 16, 500))
    if kind == "decode":
        batch = _log_int(rng, 1, 64)
        return dict(kind=kind, heads=heads, batch=batch,
                    longest=_log_int(rng, 1, min(60_000, 290_000_000 // (batch * hkv * hd))),
                    room=0)
    # the largest listed prompt has 12,289^2 / 2 * 32 * 128 products a direction; training
    # has five of them for the forward's two
    cap = 3.0e11 if kind == "attention" else 5.0e10
    seqs = _log_int(rng, 1, 40)
    longest = _log_int(rng, 1, min(12_000, math.sqrt(cap / (seqs * h * hd))))
    return dict(kind=kind, heads=heads, seqs=seqs, longest=longest,
                behind=rng.choice([0, 0, _log_int(rng, 1, 600)]) if kind == "attention" else 0,
                prefix=rng.random() < 0.5)


# ---- shapes: the same for every seed ----

def _lengths(case):
    """Query and key lengths and seen-by-all prefixes of the packed sequences."""
    n, top, behind = case["seqs"], case["longest"], case["behind"]
    rng = random.Random("%(seqs)d %(longest)d %(behind)d" % case)
    q = [top] + [rng.randint(1, top) for _ in range(n - 1)]
    if n > 4:
        q[1], q[3] = 1, 0  # a single token, and a sequence that has none
    k = [x + (rng.randint(0, behind) if behind else 0) for x in q]
    if n > 6 and behind:
        k[5] = max(0, q[5] // 2)  # fewer keys than queries: the first rows see none
    pre = [rng.randint(0, x) if case["prefix"] else 0 for x in k]
    return q, k, pre


def _cache_lengths(case):
    """Cached tokens of every live sequence (one of none where there are several)."""
    rng = random.Random("%(batch)d %(longest)d" % case)
    n = [case["longest"]] + [rng.randint(max(1, case["longest"] // 8), case["longest"])
                             for _ in range(case["batch"] - 1)]
    if len(n) > 12:
        n[3], n[5] = 0, 1
    return n


def _sections(axes, hd):
    s = [int(x * (hd // 2)) for x in AXES[axes]]
    s[0] += hd // 2 - sum(s)
    return tuple(s)


def _pairs(q_lens, k_lens, prefix):
    """Visible (query, key) pairs: row i of a sequence sees max(k - q + i + 1, prefix) keys."""
    return sum(min(k, max(k - q + i + 1, p, 0)) for q, k, p in zip(q_lens, k_lens, prefix)
               for i in range(q))


def work(case):
    kind = case["kind"]
    if kind in ("loss", "loss_train"):
        n, v, d = case["rows"], case["vocab"], case["d"]
        if kind == "loss":
            return {"bytes": 2 * (n * d + v * d) + 8 * n, "flops": 2 * n * v * d}
        return {"bytes": 4 * (n * d + v * d) + 12 * n, "flops": 6 * n * v * d}
    h, hkv, hd = HEADS[case["heads"]]
    if kind == "rope":
        e = case["tokens"] * (h + hkv) * hd
        return {"bytes": 4 * e + 4 * case["axes"] * case["tokens"], "flops": 10 * e}
    if kind == "rope_append":
        n = case["batch"]
        return {"bytes": n * (h + 2 * hkv) * hd * 4 + n * (8 + 4 * case["axes"]),
                "flops": 10 * n * (h + hkv) * hd}
    if kind == "rope_train":
        e = case["tokens"] * (h + hkv) * hd
        return {"bytes": 8 * e + 4 * case["axes"] * case["tokens"], "flops": 30 * e}
    if kind == "decode":
        n, b = sum(_cache_lengths(case)), case["batch"]
        return {"bytes": 4 * n * hkv * hd + 4 * b * h * hd, "flops": 4 * n * h * hd}
    q, k, pre = _lengths(case)
    pairs = _pairs(q, k, pre)
    rows = 4 * sum(q) * h * hd + 4 * sum(k) * hkv * hd
    if kind == "attention":
        return {"bytes": rows, "flops": 4 * pairs * h * hd}
    return {"bytes": 2 * rows + 2 * sum(q) * h * hd, "flops": 14 * pairs * h * hd}


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=BF):
    return torch.randn(*shape, generator=g, device="cuda", dtype=F32).mul_(std).to(dtype)


def _positions(g, axes, n):
    """Position of each token on each axis: running for time, image patches' rows and
    columns for the others."""
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    rows = [t % 8192, (t // 16) % 48, t % 16]
    shift = torch.randint(0, 9000, (axes, 1), generator=g, device="cuda", dtype=torch.int32)
    return (torch.stack(rows[:axes]) + shift).contiguous()


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, device="cuda", dtype=dtype)


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = dict(case=dict(case))
    if kind in ("loss", "loss_train"):
        n, v, d = case["rows"], case["vocab"], case["d"]
        s["h"] = _normal(g, n, d)
        s["w"] = _normal(g, v, d, std=0.02)
        t = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
        # a row in ten has no next token of its own: image rows, the last of a sample
        s["t"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.1, -1, t).contiguous()
        # every row weighs 1 / (rows of its tenant): four tenants in turn
        rows = [n // 4 + 1, n // 3 + 1, n // 8 + 1, n // 5 + 1]
        s["rw"] = _ints([1.0 / rows[i * 4 // n] for i in range(n)], F32)
        s["loss"] = torch.empty(n, device="cuda", dtype=F32)
        if kind == "loss_train":
            s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
        if own:
            from paper_2607_16074_gb300 import runtime as R
            s["op"] = R.VocabLoss(s["w"], max_rows=n, gradients=kind == "loss_train")
        return s
    h, hkv, hd = HEADS[case["heads"]]
    if kind.startswith("rope"):
        n = case.get("tokens") or case["batch"]
        s["qkv"] = _normal(g, n, (h + 2 * hkv) * hd)
        s["gq"] = (1 + _normal(g, hd, std=0.1, dtype=F32)).to(BF)
        s["gk"] = (1 + _normal(g, hd, std=0.1, dtype=F32)).to(BF)
        s["q"] = torch.empty(n, h, hd, device="cuda", dtype=BF)
        if kind == "rope_append":
            room, slots = case["room"], case["slots"]
            s["kc"] = _normal(g, slots, room, hkv, hd)
            s["vc"] = _normal(g, slots, room, hkv, hd)
            s["slot"] = torch.randperm(slots, generator=g, device="cuda")[:n].to(torch.int32)
            s["at"] = torch.randint(0, room, (n,), generator=g, device="cuda", dtype=torch.int32)
            s["pos"] = torch.stack([s["at"]] * case["axes"]).contiguous()
        else:
            s["pos"] = _positions(g, case["axes"], n)
            s["k"] = torch.empty(n, hkv, hd, device="cuda", dtype=BF)
        if kind == "rope_train":
            s["dq"], s["dk"] = _normal(g, n, h, hd), _normal(g, n, hkv, hd)
            # the value columns belong to the attention's backward: zero here
            s["dqkv"] = torch.zeros_like(s["qkv"])
            s["dgq"] = torch.empty(hd, device="cuda", dtype=F32)
            s["dgk"] = torch.empty(hd, device="cuda", dtype=F32)
        if own:
            from paper_2607_16074_gb300 import runtime as R
            s["op"] = R.QKNormRope(h, hkv, hd, s["gq"], s["gk"],
                                   sections=_sections(case["axes"], hd), theta=THETA, eps=EPS)
        return s
    if kind == "decode":
        n, b = _cache_lengths(case), case["batch"]
        room = max(case["room"], max(n))
        s["kc"], s["vc"] = _normal(g, b, room, hkv, hd), _normal(g, b, room, hkv, hd)
        s["q"] = _normal(g, b, h, hd, std=1.5)
        s["slot"] = torch.randperm(b, generator=g, device="cuda").to(torch.int32)
        s["n"] = _ints(n)
        s["out"] = torch.empty(b, h, hd, device="cuda", dtype=BF)
        if own:
            from paper_2607_16074_gb300 import runtime as R
            s["op"] = R.DecodeAttention(h, hkv, hd, max_batch=b)
        return s
    q, k, pre = _lengths(case)
    s["lens"] = (q, k, pre)
    s["q"], s["k"] = _normal(g, sum(q), h, hd, std=1.5), _normal(g, sum(k), hkv, hd)
    s["v"], s["out"] = _normal(g, sum(k), hkv, hd), torch.empty(sum(q), h, hd, device="cuda", dtype=BF)
    if kind == "attn_train":
        s["do"] = _normal(g, sum(q), h, hd)
        s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[x]) for x in "qkv")
        s["lse"] = torch.empty(sum(q), h, device="cuda", dtype=F32)
    if own:
        from paper_2607_16074_gb300 import runtime as R
        s["op"] = R.PromptAttention(h, hkv, hd, R.PromptPlan(q, k, pre),
                                    gradients=kind == "attn_train")
    return s


# ---- one pass ----

def run(s):
    return _OWN[s["case"]["kind"]](s) if own else _PLAIN[s["case"]["kind"]](s)


def _own_rope(s):
    s["op"].forward(s["qkv"], s["pos"], s["q"], s["k"])
    return s["q"], s["k"]


def _own_append(s):
    s["op"].append(s["qkv"], s["pos"], s["q"], s["kc"], s["vc"], s["slot"], s["at"])
    return s["q"], s["kc"], s["vc"]


def _own_rope_train(s):
    s["op"].forward(s["qkv"], s["pos"], s["q"], s["k"])
    s["op"].backward(s["qkv"], s["pos"], s["dq"], s["dk"], s["dqkv"], s["dgq"], s["dgk"])
    return s["q"], s["k"], s["dqkv"], s["dgq"], s["dgk"]


def _own_attention(s):
    s["op"].forward(s["q"], s["k"], s["v"], s["out"])
    return s["out"]


def _own_attn_train(s):
    s["op"].forward(s["q"], s["k"], s["v"], s["out"], s["lse"])
    s["op"].backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["do"], s["dq"], s["dk"],
                     s["dv"])
    return s["out"], s["dq"], s["dk"], s["dv"]


def _own_decode(s):
    s["op"].forward(s["q"], s["kc"], s["vc"], s["slot"], s["n"], s["out"])
    return s["out"]


def _own_loss(s):
    s["op"].loss(s["h"], s["t"], s["loss"])
    return s["loss"]


def _own_loss_train(s):
    s["op"].train(s["h"], s["t"], s["rw"], s["loss"], s["dh"], s["dw"])
    return s["loss"], s["dh"], s["dw"]


_OWN = dict(rope=_own_rope, rope_append=_own_append, rope_train=_own_rope_train,
            attention=_own_attention, attn_train=_own_attn_train, decode=_own_decode,
            loss=_own_loss, loss_train=_own_loss_train)


# ---- plain forms: elementary operations in 32 bits, rounded once at the end ----

def _angles(case, pos):
    """cos and sin [tokens, 1, hd / 2]: frequency i turns with its section's axis.  A position
    times a frequency has more digits than 32 bits hold, so whole turns go in 64 bits."""
    hd = HEADS[case["heads"]][2]
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"),
                                   _ints(_sections(case["axes"], hd), torch.int64))
    freq = THETA ** (torch.arange(hd // 2, device="cuda", dtype=torch.float64) * (-2.0 / hd))
    a = (pos[axis] * freq[:, None]).remainder_(2 * math.pi).to(F32).T[:, None]
    return torch.cos(a), torch.sin(a)


def _rotate(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _heads(case, qkv):
    """Query, key and value rows of the fused projection."""
    h, hkv, hd = HEADS[case["heads"]]
    x = qkv.view(qkv.shape[0], h + 2 * hkv, hd)
    return x[:, :h], x[:, h:h + hkv], x[:, h + hkv:]


def _scale(x):
    return torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)


def _plain_rope(s):
    q, k, _ = _heads(s["case"], s["qkv"])
    cos, sin = _angles(s["case"], s["pos"])
    q, k = q.to(F32), k.to(F32)
    return (_rotate(q * _scale(q) * s["gq"].to(F32), cos, sin).to(BF),
            _rotate(k * _scale(k) * s["gk"].to(F32), cos, sin).to(BF))


def _plain_append(s):
    q, k = _plain_rope(s)
    slot, at = s["slot"].long(), s["at"].long()
    s["kc"][slot, at] = k
    s["vc"][slot, at] = _heads(s["case"], s["qkv"])[2]
    return q, s["kc"], s["vc"]


def _norm_grad(x, gamma, dy, cos, sin):
    x, gamma = x.to(F32), gamma.to(F32)
    dn = _rotate(dy.to(F32), cos, -sin)
    r = _scale(x)
    dgamma = (dn * x * r).sum((0, 1))
    dn = dn * gamma
    return r * dn - x * r ** 3 * (dn * x).mean(-1, keepdim=True), dgamma


def _plain_rope_train(s):
    q, k, v = _heads(s["case"], s["qkv"])
    cos, sin = _angles(s["case"], s["pos"])
    dq, dgq = _norm_grad(q, s["gq"], s["dq"], cos, sin)
    dk, dgk = _norm_grad(k, s["gk"], s["dk"], cos, sin)
    dqkv = torch.cat([dq.to(BF), dk.to(BF), torch.zeros_like(v)], 1).view_as(s["qkv"])
    return (*_plain_rope(s), dqkv, dgq, dgk)


def _sequences(s):
    """(rows, keys, first key that row i sees no more, beyond the last) of each sequence."""
    at_q = at_k = 0
    for q, k, p in zip(*s["lens"]):
        seen = torch.clamp(torch.arange(k - q + 1, k + 1, device="cuda"), min=max(p, 0))
        yield slice(at_q, at_q + q), slice(at_k, at_k + k), seen
        at_q, at_k = at_q + q, at_k + k


def _probabilities(q, k, seen):
    """softmax rows [kv heads, group, rows, keys]; a row that sees no key is all zero."""
    x = torch.einsum("qgrd,kgd->grqk", q, k) * q.shape[-1] ** -0.5
    hidden = torch.arange(k.shape[0], device="cuda") >= seen[:, None]
    x = x.masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True) if k.shape[0] else x.sum(-1, keepdim=True)
    x = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    return x.div_(x.sum(-1, keepdim=True).clamp_min(1e-30))


def _grouped(x, hkv):
    return x.to(F32).unflatten(1, (hkv, x.shape[1] // hkv))


def _plain_attention(s):
    hkv = s["k"].shape[1]
    for rows, keys, seen in _sequences(s):
        p = _probabilities(_grouped(s["q"][rows], hkv), s["k"][keys].to(F32), seen)
        o = torch.einsum("grqk,kgd->qgrd", p, s["v"][keys].to(F32))
        s["out"][rows] = o.flatten(1, 2).to(BF)
    return s["out"]


def _plain_attn_train(s):
    hkv, c = s["k"].shape[1], s["q"].shape[-1] ** -0.5
    flat = lambda x: x.flatten(1, 2).to(BF)  # noqa: E731
    for rows, keys, seen in _sequences(s):
        q, do = _grouped(s["q"][rows], hkv), _grouped(s["do"][rows], hkv)
        k, v = s["k"][keys].to(F32), s["v"][keys].to(F32)
        p = _probabilities(q, k, seen)
        s["out"][rows] = flat(torch.einsum("grqk,kgd->qgrd", p, v))
        s["dv"][keys] = torch.einsum("grqk,qgrd->kgd", p, do).to(BF)
        dp = torch.einsum("qgrd,kgd->grqk", do, v)
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * c
        s["dq"][rows] = flat(torch.einsum("grqk,kgd->qgrd", ds, k))
        s["dk"][keys] = torch.einsum("grqk,qgrd->kgd", ds, q).to(BF)
    return s["out"], s["dq"], s["dk"], s["dv"]


def _plain_decode(s):
    top = s["kc"].shape[1]
    k, v = s["kc"][s["slot"].long()].to(F32), s["vc"][s["slot"].long()].to(F32)
    q = _grouped(s["q"], k.shape[2])
    x = torch.einsum("bgrd,bkgd->bgrk", q, k) * q.shape[-1] ** -0.5
    x = x.masked_fill_((torch.arange(top, device="cuda") >= s["n"][:, None])[:, None, None],
                       -math.inf)
    m = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    x = x / x.sum(-1, keepdim=True).clamp_min(1e-30)
    return torch.einsum("bgrk,bkgd->bgrd", x, v).reshape(s["q"].shape).to(BF)


def _rows_loss(s):
    """Losses of the rows, their probabilities and which of them count."""
    x = s["h"].to(F32) @ s["w"].to(F32).T
    counts, t = s["t"] >= 0, s["t"].clamp_min(0).long()[:, None]
    x = x.sub_(x.amax(-1, keepdim=True))
    at = x.gather(1, t)
    x = x.exp_()
    z = x.sum(-1, keepdim=True)
    loss = torch.where(counts, (z.log() - at)[:, 0], 0.0)
    return loss, x.div_(z), counts, t


def _plain_loss(s):
    return _rows_loss(s)[0]


def _plain_loss_train(s):
    loss, p, counts, t = _rows_loss(s)
    p.scatter_add_(1, t, torch.full_like(t, -1.0, dtype=F32))
    p.mul_(torch.where(counts, s["rw"], 0.0)[:, None])
    return loss, (p @ s["w"].to(F32)).to(BF), (p.T @ s["h"].to(F32)).to(BF)


_PLAIN = dict(rope=_plain_rope, rope_append=_plain_append, rope_train=_plain_rope_train,
              attention=_plain_attention, attn_train=_plain_attn_train, decode=_plain_decode,
              loss=_plain_loss, loss_train=_plain_loss_train)


# ---- the definitions in 64 bits, apart from the forms above ----

F64 = torch.float64


def _exact_turn(case, x, pos, back=False):
    """Rotation of x [tokens, heads, hd] as products of complex numbers."""
    hd = x.shape[-1]
    ends = torch.cumsum(_ints(_sections(case["axes"], hd)), 0)
    i = torch.arange(hd // 2, device="cuda")
    where = (i[:, None] >= ends).sum(1)
    a = pos.to(F64).index_select(0, where).T * torch.exp(i.to(F64) * (-2.0 / hd * math.log(THETA)))
    z = torch.complex(x[..., :hd // 2], x[..., hd // 2:])
    z = z * torch.polar(torch.ones_like(a), -a if back else a)[:, None]
    return torch.cat([z.real, z.imag], -1)


def _exact_rope(case, s):
    h, hkv, hd = HEADS[case["heads"]]
    x = s["qkv"].to(F64).view(-1, h + 2 * hkv, hd)[:, :h + hkv]
    gamma = torch.cat([s["gq"].expand(h, hd), s["gk"].expand(hkv, hd)]).to(F64)
    unit = x / torch.sqrt(x.square().sum(-1, keepdim=True) / hd + EPS)
    y = _exact_turn(case, unit * gamma, s["pos"])
    if case["kind"] == "rope":
        return y[:, :h], y[:, h:]
    if case["kind"] == "rope_append":
        kc, vc = s["kc"].to(F64), s["vc"].to(F64)
        kc[s["slot"].long(), s["at"].long()] = y[:, h:]
        vc[s["slot"].long(), s["at"].long()] = s["qkv"].to(F64).view(-1, h + 2 * hkv, hd)[:, h + hkv:]
        return y[:, :h], kc, vc
    dn = _exact_turn(case, torch.cat([s["dq"], s["dk"]], 1).to(F64), s["pos"], back=True)
    dg = (dn * unit).sum(0)
    # the norm's derivative is a projection: what lies along the row changes its length only
    e = dn * gamma
    length = torch.sqrt(x.square().sum(-1, keepdim=True) / hd + EPS)
    dx = (e - unit * (e * unit).sum(-1, keepdim=True) / hd) / length
    dqkv = torch.zeros_like(s["qkv"], dtype=F64)
    dqkv[:, :(h + hkv) * hd] = dx.flatten(1)
    return y[:, :h], y[:, h:], dqkv, dg[:h].sum(0), dg[h:].sum(0)


def _exact_attention(case, s):
    """Head by head, rows in blocks: exp of the scores over their sum."""
    h, hkv, hd = HEADS[case["heads"]]
    train = case["kind"] == "attn_train"
    out = torch.zeros(s["q"].shape, device="cuda", dtype=F64)
    dq, dk, dv = (torch.zeros(s[x].shape, device="cuda", dtype=F64) for x in "qkv")
    q0 = k0 = 0
    for lq, lk, pre in zip(*s["lens"]):
        for i in range(h if lq and lk else 0):
            g = i * hkv // h
            k, v = s["k"][k0:k0 + lk, g].to(F64), s["v"][k0:k0 + lk, g].to(F64)
            for a in range(0, lq, 4096):
                rows = slice(q0 + a, q0 + min(a + 4096, lq))
                q = s["q"][rows, i].to(F64)
                x = (q @ k.T) / math.sqrt(hd)
                j = torch.arange(lk, device="cuda")
                last = lk - lq + a + torch.arange(q.shape[0], device="cuda")[:, None]
                x[~((j <= last) | (j < pre))] = -math.inf
                p = torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
                p[torch.isnan(p)] = 0.0
                out[rows, i] = p @ v
                if train:
                    do = s["do"][rows, i].to(F64)
                    ds = p * (do @ v.T - (do * out[rows, i]).sum(-1, keepdim=True)) / math.sqrt(hd)
                    dq[rows, i] = ds @ k
                    dk[k0:k0 + lk, g] += ds.T @ q
                    dv[k0:k0 + lk, g] += p.T @ do
        q0, k0 = q0 + lq, k0 + lk
    return (out, dq, dk, dv) if train else out


def _exact_decode(case, s):
    h, hkv, hd = HEADS[case["heads"]]
    out = torch.zeros(s["q"].shape, device="cuda", dtype=F64)
    for b, n in enumerate(_cache_lengths(case)):
        if n:
            k, v = (s[x][int(s["slot"][b]), :n].to(F64).transpose(0, 1) for x in ("kc", "vc"))
            q = s["q"][b].to(F64).view(hkv, h // hkv, hd)
            p = torch.softmax(q @ k.transpose(1, 2) / math.sqrt(hd), -1)
            out[b] = (p @ v).reshape(h, hd)
    return out


def _exact_loss(case, s):
    w = s["w"].to(F64)
    loss = torch.zeros(case["rows"], device="cuda", dtype=F64)
    dh = torch.zeros(case["rows"], case["d"], device="cuda", dtype=F64)
    dw = torch.zeros_like(w)
    for a in range(0, case["rows"], 2048):
        rows = slice(a, min(a + 2048, case["rows"]))
        h, t = s["h"][rows].to(F64), s["t"][rows].long()
        keep = torch.nonzero(t >= 0)[:, 0]
        x = torch.log_softmax(h[keep] @ w.T, -1)
        loss[a + keep] = -x[torch.arange(len(keep)), t[keep]]
        if case["kind"] == "loss_train":
            e = x.exp()
            e[torch.arange(len(keep)), t[keep]] -= 1
            e *= s["rw"][rows][keep].to(F64)[:, None]
            dh[a + keep] = e @ w
            dw += e.T @ h[keep]
    return (loss, dh, dw) if case["kind"] == "loss_train" else loss


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("rope"):
        return _exact_rope(case, s)
    if case["kind"] == "decode":
        return _exact_decode(case, s)
    if case["kind"].startswith("loss"):
        return _exact_loss(case, s)
    return _exact_attention(case, s)
