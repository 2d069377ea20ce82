"""What the speed of answering with drafted tokens is measured on: a tenant's drafts go into
a paged cache, are attended as a tree, verified and kept, and the drafting vocabulary is
trained on the target's top logits, over the repository's own backbone shapes.

Kinds of cases:

  append    per-head norms of queries and keys with the rotation, keys and values going to
            their pages
  tree      drafted tokens of every live sequence, a tree each, over its pages
  verify    the drafted trees against the target's probabilities, with given random numbers
  keep      the accepted tokens' keys and values to the places behind the cached ones, in
            every layer
  distill   losses against a teacher's top logits over the whole vocabulary
  distill_train   the same with the gradients of the hidden rows and the vocabulary's weights

Sizes, trees and pages' numbers are drawn from the case's own numbers, so that a case has
the same shapes for every seed; the seed draws the values and where the pages lie.
"""
import math
import random

import torch

own = False  # False: the operators' plain forms; True: the framework's entry points

EPS, THETA, VOCAB = 1e-6, 10000.0, 32000
BF, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32

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


def listed():
    return [
        # eight robots' drafts of a few tokens go into the cache: latency
        dict(name="append_8", kind="append", heads="mqa2b", seqs=8, longest=8, behind=640, page=16),
        # prompts of a serving batch on the wide backbone
        dict(name="append_9k", kind="append", heads="grouped", seqs=6, longest=3001, behind=900,
             page=64),
        # eight robots, a chain of a few drafted tokens each behind an observation
        dict(name="tree_8", kind="tree", heads="mqa2b", batch=8, nodes=6, longest=700, page=16),
        # a lone request with a long past
        dict(name="tree_long", kind="tree", heads="grouped", batch=1, nodes=16, longest=60001,
             page=64),
        # a full server: ragged long caches, small trees
        dict(name="tree_64", kind="tree", heads="grouped", batch=64, nodes=12, longest=8100, page=64),
        # wide trees, as a drafter with many guesses makes them: more rows than a tile has
        dict(name="tree_wide", kind="tree", heads="mqa2b", batch=24, nodes=64, longest=3500, page=32),
        # a chain of six for each of eight robots
        dict(name="verify_8", kind="verify", batch=8, nodes=7, vocab=VOCAB, chain=True, certain=False),
        # trees of a full server, siblings drawn one by one from the drafter
        dict(name="verify_64", kind="verify", batch=64, nodes=24, vocab=VOCAB, chain=False,
             certain=False),
        # the narrow backbone's eighteen layers
        dict(name="keep_8", kind="keep", heads="mqa2b", batch=8, nodes=16, longest=40, page=16,
             layers=18),
        # a full server on the wide backbone
        dict(name="keep_64", kind="keep", heads="grouped", batch=64, nodes=32, longest=60, page=16,
             layers=32),
        # scoring a drafter on a few answers
        dict(name="distill_333", kind="distill", d=1024, vocab=VOCAB, rows=333, top=16, tau=1.0),
        # a drafter's training microbatch on the teacher's 32 best words
        dict(name="distill_train_8k", kind="distill_train", d=2048, vocab=VOCAB, rows=8191, top=32,
             tau=2.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "tree", "tree", "tree", "tree", "verify", "verify", "keep",
                       "distill", "distill_train", "distill_train"])
    if kind.startswith("distill"):
        return dict(kind=kind, d=rng.choice([256, 1000, 1024, 1928, 2048]),
                    vocab=rng.choice([VOCAB, _log_int(rng, 1000, VOCAB)]),
                    rows=_log_int(rng, 1, 8191), top=_log_int(rng, 1, 100),
                    tau=rng.choice([1.0, 2.0, 0.5]))
    if kind == "verify":
        return dict(kind=kind, batch=_log_int(rng, 1, 64), nodes=rng.randint(1, 24),
                    vocab=rng.choice([VOCAB, _log_int(rng, 1000, VOCAB)]), chain=rng.random() < 0.3,
                    certain=rng.random() < 0.4)
    heads = rng.choice(list(HEADS))
    h, hkv, hd = HEADS[heads]
    page = rng.choice([16, 16, 32, 48, 64, 128, 256])
    if kind == "append":
        seqs = _log_int(rng, 1, 64)
        return dict(kind=kind, heads=heads, seqs=seqs,
                    longest=_log_int(rng, 1, max(1, 36_000_000 // ((h + 2 * hkv) * hd * seqs))),
                    behind=_log_int(rng, 1, 2000), page=page)
    if kind == "keep":
        return dict(kind=kind, heads=heads, batch=_log_int(rng, 1, 48), nodes=rng.randint(2, 32),
                    longest=_log_int(rng, 1, 60), page=min(page, 64),
                    layers=rng.randint(1, max(1, 16 * 2048 // (hkv * hd * 2))))
    batch, nodes = _log_int(rng, 1, 64), _log_int(rng, 1, 64)
    # the fullest listed server holds 64 * 8,100 tokens of 8 heads of 128 at most, and its
    # 12 nodes each have 32 heads' products with them
    longest = min(60_000, 290_000_000 // (batch * hkv * hd),
                  64 * 12 * 8100 * 32 * 128 // (2 * batch * nodes * h * hd))
    return dict(kind=kind, heads=heads, batch=batch, nodes=nodes, longest=_log_int(rng, 1, longest),
                page=page)


# ---- shapes: the same for every seed ----

def _append_lengths(case):
    """New tokens of each sequence, and those that are in the cache before."""
    rng = random.Random("%(seqs)d %(longest)d %(behind)d" % case)
    n = [case["longest"]] + [rng.randint(1, case["longest"]) for _ in range(case["seqs"] - 1)]
    if len(n) > 4:
        n[2] = 0
    return n, [rng.randint(0, case["behind"]) for _ in n]


def _cache_lengths(case):
    """Cached tokens of every live sequence, and its nodes: the first the last known token."""
    rng = random.Random("%(batch)d %(longest)d %(nodes)d" % case)
    n = [case["longest"]] + [rng.randint(max(1, case["longest"] // 8), case["longest"])
                             for _ in range(case["batch"] - 1)]
    t = [case["nodes"]] + [rng.randint(1, case["nodes"]) for _ in range(case["batch"] - 1)]
    if len(n) > 12:
        n[3], n[5], t[7] = 0, 1, 0
    return n, t


def _parents(rng, t, chain):
    """A tree of t nodes: parents come first, and most nodes hang near the deepest."""
    return [-1] + [i - 1 if chain else max(0, i - 1 - int(rng.expovariate(0.6))) for i in range(1, t)]


def _trees(case, lens):
    rng = random.Random("trees %(batch)d %(nodes)d" % case)
    return [_parents(rng, t, case.get("chain", False))[:t] for t in lens]


def _ancestors(parents):
    """The nodes that each node sees, itself among them, as bits."""
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if p >= 0 else 0) | 1 << i)
    return out


def _paths(case, lens):
    """Accepted nodes of each sequence, the root first: the first few the tree's first nodes,
    which lie where they belong, the others further back than all places to fill."""
    rng = random.Random("paths %(batch)d %(nodes)d" % case)
    out = []
    for t in lens:
        n = rng.randint(1, max(1, min(8, t // 2)))
        stay = rng.randint(1, n)
        out.append(list(range(stay)) + sorted(rng.sample(range(n, t), n - stay)) if t else [])
    return out


def _nodes_of(case):
    return _cache_lengths(dict(case, longest=1))[1]


def work(case):
    kind = case["kind"]
    if kind.startswith("distill"):
        n, v, d, k = case["rows"], case["vocab"], case["d"], case["top"]
        if kind == "distill":
            return {"bytes": 2 * (n * d + v * d) + 8 * n * k + 4 * n, "flops": 2 * n * v * d}
        return {"bytes": 4 * (n * d + v * d) + 8 * n * k + 8 * n, "flops": 6 * n * v * d}
    if kind == "verify":
        b, rows = case["batch"], sum(_nodes_of(case))
        words = (1 if case["certain"] else 2) * case["vocab"]
        return {"bytes": 4 * b * words + 20 * rows + 8 * b, "flops": 2 * b * words}
    h, hkv, hd = HEADS[case["heads"]]
    if kind == "append":
        n = sum(_append_lengths(case)[0])
        return {"bytes": n * (h + 2 * hkv) * hd * 4 + 12 * n, "flops": 10 * n * (h + hkv) * hd}
    n, t = _cache_lengths(case)
    if kind == "keep":
        rows = sum(sum(x != i for i, x in enumerate(p)) for p in _paths(case, t))
        return {"bytes": 8 * rows * hkv * hd * case["layers"] + 8 * sum(t), "flops": rows}
    pairs = sum(x * y + sum(bin(s).count("1") for s in _ancestors(p))
                for x, y, p in zip(n, t, _trees(case, t)))
    tokens = sum(x + y for x, y in zip(n, t) if y)
    return {"bytes": 4 * tokens * hkv * hd + 4 * sum(t) * h * hd + 8 * sum(t),
            "flops": 4 * pairs * h * hd}


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=BF):
    return torch.randn(*shape, generator=g, device="cuda", dtype=F32).mul_(std).to(dtype)


def _ints(v, dtype=I32):
    return torch.tensor(v, device="cuda", dtype=dtype)


def _starts(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return _ints(out)


def _pages(g, s, lens, page, hkv, hd, layers=0):
    """Pages for sequences of such lengths, in no order, and a few that are nobody's."""
    need = [(n + page - 1) // page for n in lens]
    total = sum(need) + 3
    where = torch.randperm(total, generator=g, device="cuda").to(I32)
    s["table"] = torch.full((len(need), max(max(need), 1)), -1, device="cuda", dtype=I32)
    at = 0
    for b, n in enumerate(need):
        s["table"][b, :n] = where[at:at + n]
        at += n
    shape = ((layers,) if layers else ()) + (total, page, hkv, hd)
    s["kp"], s["vp"] = _normal(g, *shape), _normal(g, *shape)


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = dict(case=dict(case))
    if kind.startswith("distill"):
        return _prepare_distill(case, g, s)
    if kind == "verify":
        return _prepare_verify(case, g, s)
    h, hkv, hd = HEADS[case["heads"]]
    if kind == "append":
        new, old = _append_lengths(case)
        n = sum(new)
        _pages(g, s, [a + b for a, b in zip(new, old)], case["page"], hkv, hd)
        s["qkv"] = _normal(g, n, (h + 2 * hkv) * hd)
        s["gq"], s["gk"] = ((1 + _normal(g, hd, std=0.1, dtype=F32)).to(BF) for _ in range(2))
        s["seq"] = _ints([b for b, x in enumerate(new) for _ in range(x)])
        s["at"] = _ints([o + i for x, o in zip(new, old) for i in range(x)])
        s["pos"] = s["at"][None].contiguous()
        s["q"] = torch.empty(n, h, hd, device="cuda", dtype=BF)
        if own:
            from paper_2607_16074_gb300 import runtime as R
            s["op"] = R.QKNormRope(h, hkv, hd, s["gq"], s["gk"], theta=THETA, eps=EPS)
        return s
    n, t = _cache_lengths(case)
    s["lens"] = (n, t)
    s["n"] = _ints(n)
    if kind == "keep":
        paths = _paths(case, t)
        _pages(g, s, [a + b for a, b in zip(n, t)], case["page"], hkv, hd, case["layers"])
        s["path"] = _ints([p + [-1] * (case["nodes"] - len(p)) for p in paths])
        s["kept"] = _ints([len(p) for p in paths])
        if own:
            from paper_2607_16074_gb300 import runtime as R
            s["op"] = R.KeepDrafts(hkv, hd)
        return s
    _pages(g, s, [a + b for a, b in zip(n, t)], case["page"], hkv, hd)
    s["cu"] = _starts(t)
    bits = [x for p in _trees(case, t) for x in _ancestors(p)]
    s["sees"] = _ints([x - (1 << 64) if x >> 63 else x for x in bits], torch.int64)
    s["q"] = _normal(g, sum(t), h, hd, std=1.5)
    s["out"] = torch.empty(sum(t), h, hd, device="cuda", dtype=BF)
    if own:
        from paper_2607_16074_gb300 import runtime as R
        s["op"] = R.TreeAttention(h, hkv, hd, max_batch=case["batch"], max_rows=sum(t),
                                  max_tokens=s["table"].shape[1] * case["page"])
    return s


def _prepare_verify(case, g, s):
    """Probabilities of a target and of a drafter that is near it, and what was drafted."""
    b, v, t = case["batch"], case["vocab"], _nodes_of(case)
    trees, n = _trees(case, t), sum(t)
    z = torch.randn(n, v, generator=g, device="cuda").mul_(3.0)
    s["p"] = torch.softmax(z, -1)
    z += torch.randn(n, v, generator=g, device="cuda").mul_(0.7)
    draft = torch.softmax(z, -1)
    first = [0]
    for x in t:
        first.append(first[-1] + x)
    up = _ints([first[i] + max(p, 0) for i, tree in enumerate(trees) for p in tree], torch.int64)
    if case["certain"]:  # a node's children are its drafter's best words
        rank = [sum(q == p for q in tree[:i]) for tree in trees for i, p in enumerate(tree)]
        best = torch.topk(draft, max(rank) + 1, -1).indices[up]
        tokens = best.gather(1, _ints(rank, torch.int64)[:, None])[:, 0]
        s["q"] = None
    else:
        tokens = torch.multinomial(draft[up], 1, generator=g)[:, 0]
        s["q"] = draft
    s["tokens"] = tokens.to(I32)
    s["parent"] = _ints([p for tree in trees for p in tree])
    s["u"] = torch.rand(n, generator=g, device="cuda")
    s["cu"], s["lens"] = _starts(t), t
    s["path"] = torch.empty(b, case["nodes"], device="cuda", dtype=I32)
    s["kept"], s["next"] = (torch.empty(b, device="cuda", dtype=I32) for _ in range(2))
    if own:
        from paper_2607_16074_gb300 import runtime as R
        s["op"] = R.VerifyDrafts(v)
    return s


def _prepare_distill(case, g, s):
    n, v, d, k = case["rows"], case["vocab"], case["d"], case["top"]
    s["h"] = _normal(g, n, d)
    s["w"] = _normal(g, v, d, std=2.0 / math.sqrt(d))
    # the teacher's best words: distinct, of falling logits; a row in ten has none of its own
    # (image rows), another has fewer
    ids = (torch.randint(0, v, (n, 1), generator=g, device="cuda") +
           torch.randperm(v, generator=g, device="cuda")[:k]) % v
    t = torch.randn(n, k, generator=g, device="cuda").mul_(2.0).sort(-1, descending=True).values
    luck = torch.rand(n, generator=g, device="cuda")
    has = torch.where(luck < 0.1, 0, torch.where(luck < 0.2, (k + 1) // 2, k))
    ids[torch.arange(k, device="cuda") >= has[:, None]] = -1
    s["ids"], s["t"] = ids.to(I32).contiguous(), t.contiguous()
    # every row weighs 1 / (rows of its tenant): four tenants in turn
    rows = [n // 4 + 1, n // 3 + 1, n // 8 + 1, n // 5 + 1]
    s["rw"] = _ints([1.0 / rows[i * 4 // n] for i in range(n)], F32)
    s["loss"] = torch.empty(n, device="cuda", dtype=F32)
    train = case["kind"] == "distill_train"
    if train:
        s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
    if own:
        from paper_2607_16074_gb300 import runtime as R
        s["op"] = R.VocabDistill(s["w"], max_rows=n, top=k, temperature=case["tau"], gradients=train)
    return s


# ---- one pass ----

def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["kind"]](s)


def _own_append(s):
    s["op"].append_paged(s["qkv"], s["pos"], s["q"], s["kp"], s["vp"], s["table"], s["seq"], s["at"])
    return s["q"], s["kp"], s["vp"]


def _own_tree(s):
    s["op"].forward(s["q"], s["kp"], s["vp"], s["table"], s["cu"], s["n"], s["sees"], s["out"])
    return s["out"]


def _own_verify(s):
    s["op"].forward(s["p"], s["q"], s["tokens"], s["parent"], s["cu"], s["u"], s["path"], s["kept"],
                    s["next"])
    return s["path"], s["kept"], s["next"]


def _own_keep(s):
    s["op"].forward(s["kp"], s["vp"], s["table"], s["n"], s["path"], s["kept"])
    return s["kp"], s["vp"]


def _own_distill(s):
    s["op"].loss(s["h"], s["ids"], s["t"], s["loss"])
    return s["loss"]


def _own_distill_train(s):
    s["op"].train(s["h"], s["ids"], s["t"], s["rw"], s["loss"], s["dh"], s["dw"])
    return s["loss"], s["dh"], s["dw"]


_OWN = dict(append=_own_append, tree=_own_tree, verify=_own_verify, keep=_own_keep,
            distill=_own_distill, distill_train=_own_distill_train)


# ---- plain forms: elementary operations in 32 bits (64 where sums decide), rounded at the end ----

def _place(s, seq, at):
    """Page and row of token `at` of sequence `seq`."""
    page = s["case"]["page"]
    return s["table"][seq, at // page].long(), at % page


def _plain_append(s):
    h, hkv, hd = HEADS[s["case"]["heads"]]
    x = s["qkv"].view(-1, h + 2 * hkv, hd)
    freq = THETA ** (torch.arange(hd // 2, device="cuda", dtype=F64) * (-2.0 / hd))
    a = (s["pos"][0][:, None] * freq).remainder_(2 * math.pi).to(F32)[:, None]
    cos, sin = torch.cos(a), torch.sin(a)

    def turned(rows, gain):
        rows = rows.to(F32)
        y = rows * torch.rsqrt((rows * rows).mean(-1, keepdim=True) + EPS) * gain.to(F32)
        lo, hi = y.chunk(2, -1)
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(BF)

    where = _place(s, s["seq"].long(), s["at"].long())
    s["q"].copy_(turned(x[:, :h], s["gq"]))
    s["kp"][where] = turned(x[:, h:h + hkv], s["gk"])
    s["vp"][where] = x[:, h + hkv:]
    return s["q"], s["kp"], s["vp"]


def _plain_tree(s):
    h, hkv, hd = HEADS[s["case"]["heads"]]
    first, bit = 0, torch.arange(64, device="cuda")
    for b, (n, t) in enumerate(zip(*s["lens"])):
        if not t:
            continue
        rows, j = slice(first, first + t), torch.arange(n + t, device="cuda")
        first += t
        where = _place(s, torch.full_like(j, b), j)
        k, v = s["kp"][where].to(F32), s["vp"][where].to(F32)
        q = s["q"][rows].to(F32).unflatten(1, (hkv, h // hkv))
        x = torch.einsum("qgrd,kgd->grqk", q, k) * hd ** -0.5
        hidden = ((s["sees"][rows, None] >> bit[:t]) & 1) == 0
        x[..., n:] = x[..., n:].masked_fill(hidden, -math.inf)
        x = x.sub_(x.amax(-1, keepdim=True)).exp_()  # a node sees itself
        x = x.div_(x.sum(-1, keepdim=True))
        s["out"][rows] = torch.einsum("grqk,kgd->qgrd", x, v).flatten(1, 2).to(BF)
    return s["out"]


def _plain_verify(s):
    """All sequences a node at a time: one whose parent is where its sequence stands is tried."""
    p, q, cu = s["p"], s["q"], s["cu"].long()
    b, top = s["path"].shape
    first, t = cu[:-1], cu[1:] - cu[:-1]
    alive, i = t > 0, torch.arange(b, device="cuda")
    cur, kept = torch.zeros_like(first), alive.long()
    s["path"].fill_(-1)
    s["path"][:, 0] = torch.where(alive, 0, -1)
    at = lambda node: (first + node).clamp_max(p.shape[0] - 1)  # noqa: E731
    rest, total = p[at(cur)].to(F64), torch.ones(b, 1, device="cuda", dtype=F64)
    for c in range(1, top):
        row = at(torch.full_like(cur, c))
        tried = (c < t) & (s["parent"][row] == cur)
        x = s["tokens"][row].long()[:, None]
        chance = (torch.zeros_like(rest).scatter_(1, x, 1.0) if q is None else q[at(cur)].to(F64))
        took = tried & (s["u"][row].to(F64)[:, None] * chance.gather(1, x) * total < rest.gather(1, x))[:, 0]
        less = (rest - total * chance).clamp_min_(0.0)
        cur = torch.where(took, c, cur)
        rest = torch.where(took[:, None], p[at(cur)].to(F64), torch.where(tried[:, None], less, rest))
        total = torch.where(took[:, None], 1.0, torch.where(tried[:, None], less.sum(-1, keepdim=True), total))
        s["path"][i, kept.clamp_max(top - 1)] = torch.where(took, c, s["path"][i, kept.clamp_max(top - 1)].long()).to(I32)
        kept = kept + took
    # nothing is left where the drafter is everywhere above the target: the target itself
    rest = torch.where(rest.sum(-1, keepdim=True) > 0, rest, p[at(cur)].to(F64))
    sums = rest.cumsum(-1)
    token = (sums <= s["u"][at(torch.zeros_like(cur))].to(F64)[:, None] * sums[:, -1:]).sum(-1)
    s["kept"].copy_(kept)
    s["next"].copy_(torch.where(alive, token, -1))
    return s["path"], s["kept"], s["next"]


def _plain_keep(s):
    path = s["path"]
    counts = torch.arange(path.shape[1], device="cuda") < s["kept"][:, None]
    seq, k = torch.nonzero(counts, as_tuple=True)
    old = s["n"].long()[seq]
    src, dst = _place(s, seq, old + path[seq, k]), _place(s, seq, old + k)
    for x in (s["kp"], s["vp"]):
        x[:, dst[0], dst[1]] = x[:, src[0], src[1]]
    return s["kp"], s["vp"]


def _teacher(s):
    """Probabilities of the rows' entries, and which rows have any."""
    counts = s["ids"] >= 0
    t = (s["t"] / s["case"]["tau"]).masked_fill(~counts, -math.inf)
    top = t.amax(-1, keepdim=True)
    t = (t - torch.where(top == -math.inf, 0.0, top)).exp_()
    return t / t.sum(-1, keepdim=True).clamp_min(1e-30), counts.any(-1)


def _rows_distill(s):
    x = s["h"].to(F32) @ s["w"].to(F32).T / s["case"]["tau"]
    x = x.sub_(x.amax(-1, keepdim=True))
    log_z = x.exp().sum(-1, keepdim=True).log()
    t, live = _teacher(s)
    at = x.gather(1, s["ids"].clamp_min(0).long()) - log_z
    return (t * (torch.where(t > 0, t, 1.0).log() - at)).sum(-1), x, log_z, t, live


def _plain_distill(s):
    return _rows_distill(s)[0]


def _plain_distill_train(s):
    loss, x, log_z, t, live = _rows_distill(s)
    p = x.sub_(log_z).exp_()
    p.scatter_add_(1, s["ids"].clamp_min(0).long(), -t)
    p.mul_((torch.where(live, s["rw"], 0.0) / s["case"]["tau"])[:, None])
    return loss, (p @ s["w"].to(F32)).to(BF), (p.T @ s["h"].to(F32)).to(BF)


_PLAIN = dict(append=_plain_append, tree=_plain_tree, verify=_plain_verify, keep=_plain_keep,
              distill=_plain_distill, distill_train=_plain_distill_train)


# ---- the definitions in 64 bits, apart from the forms above ----

def _exact_append(case, s):
    h, hkv, hd = HEADS[case["heads"]]
    x = s["qkv"].to(F64).view(-1, h + 2 * hkv, hd)
    gain = torch.cat([s["gq"].expand(h, hd), s["gk"].expand(hkv, hd)]).to(F64)
    y = x[:, :h + hkv] / torch.sqrt(x[:, :h + hkv].square().sum(-1, keepdim=True) / hd + EPS) * gain
    i = torch.arange(hd // 2, device="cuda", dtype=F64)
    a = s["pos"][0].to(F64)[:, None] * torch.exp(i * (-2.0 / hd * math.log(THETA)))
    z = torch.complex(y[..., :hd // 2], y[..., hd // 2:]) * torch.polar(torch.ones_like(a), a)[:, None]
    y = torch.cat([z.real, z.imag], -1)
    kp, vp = s["kp"].to(F64), s["vp"].to(F64)
    flat = s["table"].long()[s["seq"].long(), s["at"].long() // case["page"]] * case["page"]
    flat += s["at"].long() % case["page"]
    kp.view(-1, hkv, hd).index_copy_(0, flat, y[:, h:])
    vp.view(-1, hkv, hd).index_copy_(0, flat, x[:, h + hkv:])
    return y[:, :h], kp, vp


def _exact_tree(case, s):
    """Head by head over the sequence's pages put together."""
    h, hkv, hd = HEADS[case["heads"]]
    out = torch.zeros(s["q"].shape, device="cuda", dtype=F64)
    n, t = _cache_lengths(case)
    first = 0
    for b, tree in enumerate(_trees(case, t)):
        if not tree:
            continue
        pages = s["table"][b].long()
        pages = pages[:(n[b] + t[b] + case["page"] - 1) // case["page"]]
        see = torch.ones(t[b], n[b] + t[b], device="cuda", dtype=torch.bool)
        mask = [[False] * t[b] for _ in tree]
        for i in range(t[b]):
            j = i
            while j >= 0:
                mask[i][j] = True
                j = tree[j]
        see[:, n[b]:] = _ints(mask, torch.bool)
        for g in range(hkv):
            k, v = (x[pages, :, g].reshape(-1, hd)[:n[b] + t[b]].to(F64) for x in (s["kp"], s["vp"]))
            for i in range(g * h // hkv, (g + 1) * h // hkv):
                x = s["q"][first:first + t[b], i].to(F64) @ k.T / math.sqrt(hd)
                out[first:first + t[b], i] = torch.softmax(x.masked_fill(~see, -math.inf), -1) @ v
        first += t[b]
    return out


def _exact_verify(case, s):
    """Sequence by sequence, as one would by hand."""
    parent, tokens, u = s["parent"].tolist(), s["tokens"].tolist(), s["u"].tolist()
    paths, kept, last = [], [], []
    first = 0
    for t in _nodes_of(case):
        tree, cur, path = parent[first:first + t], 0, [0] if t else []
        rest = None
        while t:
            rest, mass, took = s["p"][first + cur].to(F64), 1.0, False
            for c in (i for i in range(1, t) if tree[i] == cur):
                x = tokens[first + c]
                if s["q"] is None:
                    guess = torch.zeros_like(rest)
                    guess[x] = 1.0
                else:
                    guess = s["q"][first + cur].to(F64)
                if u[first + c] * float(guess[x]) * mass < float(rest[x]):
                    took = True
                    break
                rest = torch.relu(rest - mass * guess)
                mass = float(rest.sum())
            if not took:
                break
            path.append(c)
            cur = c
        if t:
            if float(rest.sum()) == 0.0:
                rest = s["p"][first + cur].to(F64)
            sums = torch.cumsum(rest, 0)
            goal = u[first] * float(sums[-1])
            last.append(int(torch.searchsorted(sums, torch.tensor([goal], device="cuda", dtype=F64), right=True)))
        else:
            last.append(-1)
        paths.append(path + [-1] * (case["nodes"] - len(path)))
        kept.append(len(path))
        first += t
    return _ints(paths), _ints(kept), _ints(last)


def _exact_keep(case, s):
    n, t = _cache_lengths(case)
    kp, vp, page = s["kp"].to(F64), s["vp"].to(F64), case["page"]
    table = s["table"].tolist()
    for b, path in enumerate(_paths(case, t)):
        for k, node in enumerate(path):
            src, dst = n[b] + node, n[b] + k
            for x in (kp, vp):
                x[:, table[b][dst // page], dst % page] = x[:, table[b][src // page], src % page].clone()
    return kp, vp


def _exact_distill(case, s):
    w, tau = s["w"].to(F64), case["tau"]
    loss = torch.zeros(case["rows"], device="cuda", dtype=F64)
    dh = torch.zeros(case["rows"], case["d"], device="cuda", dtype=F64)
    dw = torch.zeros_like(w)
    for a in range(0, case["rows"], 2048):
        ids = s["ids"][a:a + 2048].long()
        keep = torch.nonzero((ids >= 0).any(-1))[:, 0]
        ids, h = ids[keep], s["h"][a + keep].to(F64)
        logits = s["t"][a + keep].to(F64).masked_fill(ids < 0, -math.inf)
        log_t = torch.log_softmax(logits / tau, -1)
        t = log_t.exp()
        log_p = torch.log_softmax(h @ w.T / tau, -1)
        diff = log_t - log_p.gather(1, ids.clamp_min(0))
        loss[a + keep] = torch.where(ids >= 0, t * diff, 0.0).sum(-1)
        if case["kind"] == "distill_train":
            e = log_p.exp()
            e.scatter_add_(1, ids.clamp_min(0), -t)
            e *= (s["rw"][a + keep].to(F64) / tau)[:, None]
            dh[a + keep] = e @ w
            dw += e.T @ h
    return (loss, dh, dw) if case["kind"] == "distill_train" else loss


_EXACT = dict(append=_exact_append, tree=_exact_tree, verify=_exact_verify, keep=_exact_keep,
              distill=_exact_distill, distill_train=_exact_distill)


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed))
