"""Answering with drafted tokens against its definitions in 64 bits (tests/draft_ops_ref.py,
where the tolerances are derived), at the sizes, trees, pages and layouts where it can go
wrong."""
import random

import pytest
import torch

from tests import draft_ops_ref as D
from tests import text_ops_ref as T

pytestmark = pytest.mark.gpu
BF, I32, F32 = torch.bfloat16, torch.int32, torch.float32
HEADS = [(4, 4, 64), (8, 1, 256), (8, 2, 128), (12, 4, 128), (14, 2, 64), (4, 4, 256), (64, 1, 64)]


def _r():
    from paper_2607_16074_gb300 import runtime as R
    return R


def _reports(op):
    from paper_2607_16074_gb300 import jnx as J
    with pytest.raises(J.JnxError) as e:
        op.check()
    assert e.value.code == J.JNX_ERR_DEVICE_BOUNDS
    op.check()  # cleared


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(BF)


def empty(*shape, dtype=BF):
    return torch.full(shape, float("nan"), device="cuda", dtype=dtype)


def ints(*v, dtype=I32):
    return torch.tensor(v, device="cuda", dtype=dtype)


def pages_for(seed, lens, page, hkv, hd, spare=2):
    """NaN pages in no order and a table whose other entries are no pages."""
    rng = random.Random(seed)
    need = [(n + page - 1) // page for n in lens]
    total = sum(need) + spare
    where = rng.sample(range(total), sum(need))
    table = torch.full((len(lens), max(max(need, default=0), 1)), -1, dtype=I32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(where[at:at + n], dtype=I32)
        at += n
    return empty(total, page, hkv, hd), empty(total, page, hkv, hd), table.cuda()


def place(table, page, b, tokens):
    t = torch.as_tensor(tokens, device="cuda", dtype=torch.int64)
    return table[b].long()[t // page], t % page


# ---------------------------------------------------------------- appends

@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [16, 48, 1, 7])
def test_append_paged(heads, page):
    """The rows that the append to slots writes, at the pages' places, and nothing else."""
    h, hkv, hd = heads
    g = gen(page)
    old, new = [0, 5, page - 1, 31], [3, 0, 2, 20]
    n = sum(new)
    kp, vp, table = pages_for(1, [a + b for a, b in zip(old, new)], page, hkv, hd)
    seq = ints(*[b for b, x in enumerate(new) for _ in range(x)])
    at = ints(*[o + i for o, x in zip(old, new) for i in range(x)])
    qkv, gq, gk = normal(g, n, (h + 2 * hkv) * hd), 1 + normal(g, hd, std=0.2), 1 + normal(g, hd, std=0.2)
    op = _r().QKNormRope(h, hkv, hd, gq, gk)
    q, q1 = empty(n, h, hd), empty(n, h, hd)
    op.append_paged(qkv, at[None].contiguous(), q, kp, vp, table, seq, at)
    kc, vc = empty(4, 60, hkv, hd), empty(4, 60, hkv, hd)
    op.append(qkv, at[None].contiguous(), q1, kc, vc, seq, at)
    op.check()
    where = (table[seq.long(), at.long() // page].long(), at.long() % page)
    assert torch.equal(q, q1) and not q.isnan().any()
    assert torch.equal(kp[where], kc[seq.long(), at.long()])
    assert torch.equal(vp[where], qkv.view(n, -1, hd)[:, h + hkv:])
    want = T.norm_rope(qkv.view(n, -1, hd)[:, h:h + hkv], gk, at[None], (hd // 2,), 1e4, 1e-6)
    T.close(kp[where], want, T.norm_rope_bound(want), "k")
    kp[where] = vp[where] = float("nan")
    assert kp.isnan().all() and vp.isnan().all()


def test_append_paged_reports_places_outside():
    op = _r().QKNormRope(4, 4, 64)
    kp, vp, table = pages_for(0, [40, 16], 16, 4, 64, spare=0)
    table[0, 1] = kp.shape[0]  # a page too many
    n = 7
    qkv, q = normal(gen(0), n, 12 * 64), empty(n, 4, 64)
    seq, at = ints(0, 0, 2, -1, 1, 1, 0), ints(3, 20, 0, 0, -1, 16, 48)
    op.append_paged(qkv, at[None].contiguous(), q, kp, vp, table, seq, at)
    _reports(op)
    assert not q.isnan().any()
    kp[table[0, 0], 3] = float("nan")
    assert kp.isnan().all()  # the first alone was written


def test_append_paged_strides_and_far_pages():
    """Pages beyond 2^31 elements, the halves of one tensor with heads outermost."""
    op, n = _r().QKNormRope(8, 1, 256), 3
    both = torch.zeros(2, 1, 9000 * 1024, 256, device="cuda", dtype=BF)  # 4.7 G elements
    kp, vp = (x.view(9000, 1024, 1, 256) for x in both)
    table = ints([8999, 0], [17, 8191])
    seq, at = ints(0, 1, 1), ints(1023, 5, 2047)
    qkv, q = normal(gen(0), n, 10 * 256), empty(n, 8, 256)
    op.append_paged(qkv, at[None].contiguous(), q, kp, vp, table, seq, at)
    op.check()
    v = qkv.view(n, 10, 256)[:, 9:]
    for i, (a, b) in enumerate(((8999, 1023), (17, 5), (8191, 1023))):
        assert torch.equal(vp[a, b], v[i])
        vp[a, b] = 0
    assert not vp.any()


# ---------------------------------------------------------------- trees

def random_tree(rng, t):
    return [-1] + [rng.randint(max(0, i - 4), i - 1) for i in range(1, t)] if t else []


class Trees:
    """Sequences with their pages, trees and what each node should be."""

    def __init__(self, heads, page, old, nodes, seed=0, sees=None, std=1.5, one_page=False):
        h, hkv, hd = heads
        rng, g = random.Random(seed), gen(seed)
        self.heads, self.page, self.old, self.nodes = heads, page, old, nodes
        lens = [a + b for a, b in zip(old, nodes)]
        if one_page:
            page = self.page = one_page
        self.kp, self.vp, self.table = pages_for(seed, lens, page, hkv, hd)
        if one_page:
            self.table = self.table[:, :1].contiguous()
        self.cu = ints(*[sum(nodes[:i]) for i in range(len(nodes) + 1)])
        self.n = ints(*old)
        self.masks = [D.ancestors(random_tree(rng, t)) if sees is None else sees(rng, t) for t in nodes]
        self.sees = ints(*[D.bits(r) for m in self.masks for r in m.tolist()], dtype=torch.int64)
        self.q = normal(g, sum(nodes), h, hd, std=std)
        for b, n in enumerate(lens):
            where = place(self.table, page, b, range(n))
            self.kp[where], self.vp[where] = normal(g, n, hkv, hd), normal(g, n, hkv, hd)

    def op(self):
        h, hkv, hd = self.heads
        return _r().TreeAttention(h, hkv, hd, max(len(self.old), 1), max(sum(self.nodes), 1),
                                  self.table.shape[1] * self.page)

    def run(self, op=None, out=None, **kw):
        op = op or self.op()
        out = empty(*self.q.shape) if out is None else out
        op.forward(self.q, self.kp, self.vp, self.table, self.cu, self.n, self.sees, out, **kw)
        op.check()
        return out

    def rows(self, b):
        return slice(sum(self.nodes[:b]), sum(self.nodes[:b + 1]))

    def compare(self, out):
        for b, (n, t) in enumerate(zip(self.old, self.nodes)):
            where = place(self.table, self.page, b, range(n + t))
            want, tol = D.tree(self.q[self.rows(b)], self.kp[where], self.vp[where], n, self.masks[b])
            T.close(out[self.rows(b)], want, tol, f"sequence {b} ({n} cached, {t} nodes)")


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [16, 64])
def test_tree_small(heads, page):
    c = Trees(heads, page, [0, 1, 15, 16, 17, 63, 64, 65, 127], [1, 3, 1, 16, 2, 1, 0, 7, 5], seed=page)
    c.compare(c.run())


@pytest.mark.parametrize("heads", HEADS)
def test_tree_long_and_wide(heads):
    c = Trees(heads, 48, [500, 128, 1100, 0, 2500, 129, 4097], [64, 63, 33, 64, 2, 9, 12], seed=3)
    c.compare(c.run())


@pytest.mark.parametrize("heads", [(8, 1, 256), (8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("page", [32, 80, 128, 256, 1024])
def test_tree_pages(heads, page):
    c = Trees(heads, page, [1000, 0, 255, 300, 77], [6, 20, 1, 64, 3], seed=page)
    c.compare(c.run())


@pytest.mark.parametrize("heads", [(8, 1, 256), (8, 2, 128), (14, 2, 64)])
@pytest.mark.parametrize("room", [701, 65, 640])
def test_tree_of_a_page_a_sequence(heads, room):
    """A page a sequence may have any room: slots, as the other cache has them."""
    c = Trees(heads, 0, [room - 4, 0, 17, room // 2], [4, 3, 1, 9], seed=room, one_page=room)
    c.compare(c.run())


def test_tree_any_bits():
    """Bits need be no tree: rows that see no node, not themselves, or all."""
    def sees(rng, t):
        m = torch.tensor([[rng.random() < 0.5 for _ in range(t)] for _ in range(t)], dtype=torch.bool)
        m = m.view(t, t)
        if t > 2:
            m[1], m[2] = False, True
        return m
    c = Trees((8, 2, 128), 16, [0, 200, 63, 0, 1], [64, 40, 64, 5, 1], sees=sees)
    c.sees |= ints(*[-1 << t if t < 64 else 0 for t in c.nodes for _ in range(t)], dtype=torch.int64)
    out = c.run()  # (bits beyond the nodes are none)
    c.compare(out)
    assert (out[1] == 0).all()  # saw nothing at all


def test_tree_single_tokens_are_decode():
    """A root alone sees what one token against the cache does."""
    R, (h, hkv, hd), n = _r(), (32, 8, 128), [700, 1, 130, 64]
    c = Trees((h, hkv, hd), 64, [x - 1 for x in n], [1] * 4, seed=5)
    kc, vc = empty(4, 704, hkv, hd), empty(4, 704, hkv, hd)
    for b, x in enumerate(n):
        where = place(c.table, 64, b, range(x))
        kc[b, :x], vc[b, :x] = c.kp[where], c.vp[where]
    out, other = c.run(), empty(4, h, hd)
    R.DecodeAttention(h, hkv, hd, 4).forward(c.q, kc, vc, ints(0, 1, 2, 3), ints(*n), other)
    c.compare(out)
    c.compare(other)


def test_tree_does_not_depend_on_the_batch():
    heads = (8, 2, 128)
    c = Trees(heads, 16, [900, 0, 3000, 64, 1500, 17], [8, 64, 20, 1, 33, 5], seed=9)
    out = c.run()
    for b in range(6):
        rows = c.rows(b)
        one = empty(c.nodes[b], *heads[::2])
        op = _r().TreeAttention(*heads, 1, 64, c.table.shape[1] * 16)
        op.forward(c.q[rows].contiguous(), c.kp, c.vp, c.table[b:b + 1], ints(0, c.nodes[b]),
                   c.n[b:b + 1], c.sees[rows], one)
        op.check()
        assert torch.equal(one, out[rows])
    assert torch.equal(out, c.run())


def test_tree_of_more_sequences_than_a_launch_takes():
    rng = random.Random(5)
    old = [rng.choice([0, 3, 70, 300, 900]) for _ in range(600)]
    nodes = [rng.choice([0, 1, 2, 5, 17]) for _ in range(600)]
    c = Trees((4, 1, 64), 16, old, nodes, seed=6)
    out = c.run()
    c.compare(out)
    # a sequence of the last launch alone
    b = max(i for i in range(600) if nodes[i] > 1 and old[i] == 900)
    one, rows = empty(nodes[b], 4, 64), c.rows(b)
    op = _r().TreeAttention(4, 1, 64, 1, 17, c.table.shape[1] * 16)
    op.forward(c.q[rows].contiguous(), c.kp, c.vp, c.table[b:b + 1], ints(0, nodes[b]), c.n[b:b + 1],
               c.sees[rows], one)
    assert torch.equal(one, out[rows])


def test_tree_sequences_that_share_their_past():
    """One past for all, by a table whose rows are the same, and pages of their own behind it."""
    heads, (h, hkv, hd) = (8, 2, 128), (8, 2, 128)
    c = Trees(heads, 16, [320], [6], seed=8)
    n, past = 3, c.table[0, :20]
    kp, vp = empty(c.kp.shape[0] + 2 * n, 16, hkv, hd), empty(c.kp.shape[0] + 2 * n, 16, hkv, hd)
    kp[:c.kp.shape[0]], vp[:c.kp.shape[0]] = c.kp, c.vp
    table = torch.cat([past.expand(n, 20), ints(*range(c.kp.shape[0], c.kp.shape[0] + n))[:, None]], 1)
    g = gen(3)
    for b in range(n):
        kp[table[b, 20].long(), :6], vp[table[b, 20].long(), :6] = normal(g, 6, hkv, hd), normal(g, 6, hkv, hd)
    q, out = normal(g, 6 * n, h, hd, std=1.5), empty(6 * n, h, hd)
    op = _r().TreeAttention(*heads, n, 6 * n, 21 * 16)
    op.forward(q, kp, vp, table.contiguous(), ints(0, 6, 12, 18), ints(320, 320, 320), c.sees.repeat(n), out)
    op.check()
    for b in range(n):
        where = place(table, 16, b, range(326))
        T.close(out[6 * b:6 * b + 6], *D.tree(q[6 * b:6 * b + 6], kp[where], vp[where], 320, c.masks[0]))


def test_tree_strides_and_rows_of_nobody():
    heads, (h, hkv, hd) = (8, 2, 128), (8, 2, 128)
    c = Trees(heads, 16, [100, 33], [5, 9], seed=2)
    plain = c.run()
    # heads outermost in q, out and the pages, a wider table, rows behind the last sequence
    n = sum(c.nodes)
    q = empty(h, n + 3, hd).transpose(0, 1)
    out = empty(n + 3, 2, h, hd)[:, 1]
    q[:n], out[:] = c.q, 7.0
    both = empty(2, hkv, *c.kp.shape[:2], hd)
    kp, vp = (x.permute(1, 2, 0, 3) for x in both)
    kp.copy_(c.kp), vp.copy_(c.vp)
    table = torch.full((2, 40), -1, device="cuda", dtype=I32)
    table[:, 3:3 + c.table.shape[1]] = c.table
    sees = torch.cat([c.sees, c.sees[:3]])
    op = _r().TreeAttention(*heads, 2, n + 3, 40 * 16)
    op.forward(q, kp, vp, table[:, 3:], c.cu, c.n, sees, out)
    op.check()
    assert torch.equal(out[:n], plain) and (out[n:] == 7).all()


def test_tree_reports():
    heads = (8, 2, 128)
    c = Trees(heads, 16, [100, 33, 20], [5, 9, 2], seed=2)
    good, op = c.run(), c.op()

    def run(cu=c.cu, n=c.n, table=c.table):
        out = torch.full_like(good, 7.0)
        op.forward(c.q, c.kp, c.vp, table, cu, n, c.sees, out)
        return out

    for n in (ints(100, -1, 20), ints(100, 2 ** 31 - 9, 20), ints(100, c.table.shape[1] * 16 - 8, 20)):
        out = run(n=n)
        _reports(op)
        assert torch.equal(out[:5], good[:5]) and (out[5:14] == 0).all() and torch.equal(out[14:], good[14:])
    # (in the first the third sequence has rows of its own, which it may fill with anything)
    for cu, same, left in ((ints(0, 5, 4, 16), slice(0, 4), slice(0, 0)),
                           (ints(0, 5, 14, 17), slice(0, 14), slice(14, 16)),
                           (ints(-1, 5, 14, 16), slice(5, 16), slice(0, 5))):
        out = run(cu=cu)
        _reports(op)
        assert torch.equal(out[same], good[same]) and (out[left] == 7).all()
    for bad in (-1, c.kp.shape[0], 2 ** 31 - 1):
        table = c.table.clone()
        table[0, 2] = bad  # tokens 32 to 47 of the first sequence are zeros
        out = run(table=table)
        _reports(op)
        assert torch.equal(out[5:], good[5:])
        where = place(c.table, 16, 0, range(105))
        k, v = c.kp[where].clone(), c.vp[where].clone()
        k[32:48] = v[32:48] = 0
        T.close(out[:5], *D.tree(c.q[:5], k, v, 100, c.masks[0]), "zeros")
    run()
    op.check()


def test_tree_more_nodes_than_a_word_are_left_out():
    c = Trees((4, 4, 64), 16, [10, 0], [64, 3], seed=2)
    op, out = _r().TreeAttention(4, 4, 64, 2, 67, 96), torch.full_like(c.q, 7.0)
    op.forward(c.q, c.kp, c.vp, c.table, ints(0, 65, 67), c.n, c.sees, out)
    _reports(op)
    assert (out[:65] == 7).all() and not out[65:].isnan().any()


def test_tree_of_nothing():
    op = _r().TreeAttention(8, 2, 128, 4, 8, 64)
    kp, vp, table = pages_for(0, [64], 16, 2, 128)
    q = empty(0, 8, 128)
    op.forward(q, kp, vp, table, ints(0, 0), ints(5), ints(dtype=torch.int64), q)
    none = torch.zeros(0, 4, device="cuda", dtype=I32)
    out = torch.full((2, 8, 128), 7.0, device="cuda", dtype=BF)
    op.forward(out.clone(), kp, vp, none, ints(0), ints(), ints(1, 1, dtype=torch.int64), out)
    op.check()
    assert (out == 7).all()


def test_tree_long_past():
    c = Trees((8, 1, 128), 256, [70_000, 9], [8, 8], seed=4)
    c.compare(c.run())


def test_tree_far_pages():
    """Pages beyond 2^32 bytes and 2^31 elements."""
    h, hkv, hd, page = 8, 2, 128, 64
    c = Trees((h, hkv, hd), page, [150], [7], seed=6)
    big_k = torch.zeros(140_000, page, hkv, hd, device="cuda", dtype=BF)  # 2.3 G elements
    big_v = torch.zeros_like(big_k)
    far = ints([139_999, 131_072, 5])
    big_k[far[0].long()], big_v[far[0].long()] = c.kp[c.table[0].long()], c.vp[c.table[0].long()]
    want, out = c.run(), empty(7, h, hd)
    c.op().forward(c.q, big_k, big_v, far, c.cu, c.n, c.sees, out)
    assert torch.equal(out, want)


def test_tree_in_a_graph_and_on_another_stream():
    c = Trees((8, 1, 256), 16, [600, 100, 30], [6, 1, 20], seed=8)
    want, op = c.run(), c.op()
    out = empty(*c.q.shape)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(op, out, stream=side)
    assert torch.equal(out, want)
    graphs = []
    for _ in range(2):  # two graphs that share a workspace, one after the other
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            op.forward(c.q, c.kp, c.vp, c.table, c.cu, c.n, c.sees, out)
        graphs.append(g)
    for g in graphs * 2:
        out.fill_(float("nan"))
        g.replay()
        assert torch.equal(out, want)
    c.n += ints(-200, 0, -30)  # lengths are the replay's own
    c.old = c.n.tolist()
    graphs[0].replay()
    c.compare(out)


def test_tree_workspace_holds_anything():
    c = Trees((8, 2, 128), 16, [3000, 100], [8, 60], seed=1)
    op = c.op()
    want = c.run(op)
    op.ws.fill_(255)  # NaN
    assert torch.equal(c.run(op), want)


@pytest.mark.parametrize("first", [0, 5, 2 ** 31 - 1, -1])
@pytest.mark.parametrize("number", [0, 1, 7])
def test_tree_rows_of_nobody_whatever_the_workspace_held(first, number):
    """Rows that no sequence has are left as they were, though the workspace may hold what looks
    like an earlier call's record of them."""
    c = Trees((8, 2, 128), 16, [900, 700], [3, 9], seed=4)
    n = 40  # rows of the call
    q = torch.cat([c.q, normal(gen(0), n - 12, 8, 128)])
    sees = torch.cat([c.sees, c.sees.new_ones(n - 12)])
    op = _r().TreeAttention(8, 2, 128, 2, n, c.table.shape[1] * 16)
    op.ws[:16 * n].view(I32).view(n, 4).copy_(ints(first, 64, 64, number))
    out = torch.full_like(q, 7.0)
    op.forward(q, c.kp, c.vp, c.table, c.cu, c.n, sees, out)
    op.check()
    c.compare(out[:12])
    assert (out[12:] == 7).all()


# ---------------------------------------------------------------- verification

def verify_case(vocab, nodes, seed=0, certain=False, chain=False, sharp=3.0, near=0.7, ld=0, drawn=True):
    rng, g = random.Random(seed), gen(seed)
    n = sum(nodes)
    ld = max(ld, vocab)
    z = torch.randn(n, vocab, generator=g, device="cuda") * sharp
    p, q = empty(n, ld, dtype=F32)[:, :vocab], empty(n, ld, dtype=F32)[:, :vocab]
    p.copy_(torch.softmax(z, -1))
    q.copy_(torch.softmax(z + torch.randn(n, vocab, generator=g, device="cuda") * near, -1))
    trees = [[-1] + [i - 1 if chain else rng.randint(max(0, i - 4), i - 1) for i in range(1, t)] if t else []
             for t in nodes]
    up, at = [], 0
    for tree in trees:
        up += [at + max(x, 0) for x in tree]
        at += len(tree)
    tokens = torch.multinomial(q[ints(*up).long()], 1, generator=g)[:, 0].to(I32)
    if not drawn:
        tokens = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=I32)
    u = torch.rand(n, generator=g, device="cuda")
    cu = ints(*[sum(nodes[:i]) for i in range(len(nodes) + 1)])
    parent = ints(*[x for tree in trees for x in tree])
    return p, None if certain else q, tokens, parent, cu, u


def run_verify(p, q, tokens, parent, cu, u, most, op=None, check=True):
    b = cu.shape[0] - 1
    op = op or _r().VerifyDrafts(p.shape[1])
    path = torch.full((b, most), -7, device="cuda", dtype=I32)
    kept, nxt = (torch.full((b,), -7, device="cuda", dtype=I32) for _ in range(2))
    op.forward(p, q, tokens, parent, cu, u, path, kept, nxt)
    if check:
        op.check()
    return path.tolist(), kept.tolist(), nxt.tolist()


def by_hand(p, q, tokens, parent, cu, u, most):
    p, q = p.double().cpu(), None if q is None else q.double().cpu()
    tokens, parent, cu, u = tokens.tolist(), parent.tolist(), cu.tolist(), u.cpu()
    out = [], [], []
    for a, b in zip(cu, cu[1:]):
        path, nxt = ([], -1) if a == b else D.verify(
            p[a:b], None if q is None else q[a:b], tokens[a:b], parent[a:b], u[a:b], p.shape[1])
        out[0].append(path + [-1] * (most - len(path)))
        out[1].append(len(path))
        out[2].append(nxt)
    return out


@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("vocab", [1, 2, 5, 33, 1000, 4096, 32000, 50257, 151_936])
def test_verify(vocab, certain):
    args = verify_case(vocab, [7, 1, 24, 0, 12, 64, 3, 2], seed=vocab, certain=certain)
    assert run_verify(*args, 64) == by_hand(*args, 64)


@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("near,sharp", [(0.0, 3.0), (0.1, 1.0), (5.0, 3.0), (1.0, 12.0)])
def test_verify_near_and_far_drafters(near, sharp, certain):
    """A drafter that is the target, one that is nothing like it, and targets that are sure."""
    args = verify_case(777, [9] * 40, seed=3, certain=certain, near=near, sharp=sharp, chain=not certain)
    assert run_verify(*args, 9) == by_hand(*args, 9)


def test_verify_many_siblings():
    """A root with all others as children: a rejection after another, the same token twice."""
    p, q, tokens, parent, cu, u = verify_case(50, [64] * 20, seed=1, near=3.0)
    parent = torch.where(parent > 0, 0, parent)
    for chance in (q, None):
        args = (p, chance, tokens, parent, cu, u.clamp_min(0.6))
        assert run_verify(*args, 64) == by_hand(*args, 64)


def test_verify_rows_of_any_stride_and_a_wide_path():
    for vocab, ld in ((1001, 1003), (1000, 1004), (7, 8)):
        args = verify_case(vocab, [5, 8, 1], seed=2, ld=ld)
        assert run_verify(*args, 11) == by_hand(*args, 11)
    p, q, tokens, parent, cu, u = verify_case(1000, [4] * 3, seed=2)
    one = p[:1].expand(12, -1), q[:1].expand(12, -1), tokens, parent, cu, u  # a row for all
    assert run_verify(*one, 4) == by_hand(*one, 4)


def test_verify_borders():
    """u and probabilities of zero and one, words without any, a total of nothing."""
    eye = torch.eye(4, device="cuda")
    half = torch.tensor([[0.0, 0.5, 0.0, 0.5]], device="cuda")
    cu, parent = ints(0, 2), ints(-1, 0)

    def one(p, q, token, u, **kw):
        u = torch.tensor(u, device="cuda")
        return run_verify(p, q, ints(0, token), parent, cu, u, 2, **kw)

    sure = torch.stack([eye[2], eye[1]])
    assert one(sure, sure, 2, [0.0, 0.999]) == ([[0, 1]], [2], [1])
    assert one(sure, None, 2, [0.0, 0.999]) == ([[0, 1]], [2], [1])
    assert one(sure, None, 3, [0.999, 0.0]) == ([[0, -1]], [1], [2])  # 0 < 0 is no acceptance
    two = half.repeat(2, 1)
    assert one(two, two, 1, [0.0, 0.99]) == ([[0, 1]], [2], [1])  # words of no chance are not drawn
    assert one(two, two, 1, [0.4999, 0.99]) == ([[0, 1]], [2], [1])
    assert one(two, two, 1, [0.5, 0.99]) == ([[0, 1]], [2], [3])  # the sum has to be above
    # what is left of the target is nothing: the target itself (q above p everywhere)
    assert one(two * 0.5, two, 1, [0.25, 0.9]) == ([[0, -1]], [1], [1])
    zero = torch.zeros(2, 4, device="cuda")
    op = _r().VerifyDrafts(4)
    for p in (zero, zero + float("nan"), zero + float("inf")):
        assert one(p, two, 1, [0.5, 0.9], op=op, check=False)[2] == [-1]
        _reports(op)


def test_verify_reports():
    p, q, tokens, parent, cu, u = verify_case(100, [5, 4, 3], seed=1, chain=True, near=0.0)
    good = run_verify(p, q, tokens, parent, cu, u, 5)
    assert good[1] == [5, 4, 3]  # the target itself: every draft is taken
    op = _r().VerifyDrafts(100)
    for bad in (-1, 100, 2 ** 31 - 1):
        t = tokens.clone()
        t[2] = bad
        path, kept, _ = run_verify(p, q, t, parent, cu, u, 5, op, check=False)
        _reports(op)
        assert kept == [2, 4, 3] and path[1:] == good[0][1:]
    for bad in (2, 3, -1, 70):
        up = parent.clone()
        up[2] = bad
        assert run_verify(p, q, tokens, up, cu, u, 5, op, check=False)[1] == [2, 4, 3]
        _reports(op)
    for cu_bad, kept in ((ints(0, 5, 3, 12), [5, 0, 0]), (ints(0, 5, 9, 13), [5, 4, 0]), (ints(-2, 5, 9, 12), [0, 4, 3])):
        out = run_verify(p, q, tokens, parent, cu_bad, u, 5, op, check=False)
        _reports(op)
        assert out[1] == kept
        assert all(n == -1 and x == [-1] * 5 for n, x, k in zip(out[2], out[0], out[1]) if k == 0)
    out = run_verify(p, q, tokens, parent, cu, u, 4, op, check=False)  # five nodes, a path of four
    _reports(op)
    assert out[1] == [0, 4, 3]


@pytest.mark.parametrize("certain", [False, True])
def test_verified_tokens_are_distributed_as_the_target(certain):
    """The first token behind the root, over many sequences of the same p and q: its counts
    against p by chi-square.  5 words are 4 degrees of freedom, above 35 in 5e-7 of cases."""
    n, t = 40_000, 4
    g = gen(7)
    p1 = torch.tensor([0.4, 0.3, 0.15, 0.1, 0.05], device="cuda")
    q1 = torch.tensor([0.1, 0.2, 0.3, 0.2, 0.2], device="cuda")
    p, q = p1.expand(n * t, 5), q1.expand(n * t, 5)
    tokens = torch.multinomial(q1, n * t, replacement=True, generator=g).to(I32)
    parent = ints(-1, 0, 0, 0).repeat(n)
    cu = torch.arange(n + 1, device="cuda", dtype=I32) * t
    u = torch.rand(n * t, generator=g, device="cuda")
    path, kept, nxt = (torch.empty(*s, device="cuda", dtype=I32) for s in ((n, t), (n,), (n,)))
    _r().VerifyDrafts(5).forward(p, None if certain else q, tokens, parent, cu, u, path, kept, nxt)
    child = path[:, 1].long().clamp_min(0)
    first = torch.where(kept > 1, tokens.view(n, t).gather(1, child[:, None])[:, 0], nxt)
    counts = torch.bincount(first.long(), minlength=5).double()
    assert ((counts - n * p1) ** 2 / (n * p1)).sum() < 35, counts
    assert 0.2 < (kept > 1).double().mean() < 0.999


def test_verify_in_a_graph():
    args = verify_case(5000, [6, 1, 9], seed=4)
    want = run_verify(*args, 9)
    op = _r().VerifyDrafts(5000)
    path, kept, nxt = (torch.empty(*s, device="cuda", dtype=I32) for s in ((3, 9), (3,), (3,)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op.forward(*args, path, kept, nxt)
    for _ in range(2):
        path.fill_(-7)
        g.replay()
        assert (path.tolist(), kept.tolist(), nxt.tolist()) == want


# ---------------------------------------------------------------- kept rows

@pytest.mark.parametrize("heads", [(4, 64), (1, 256), (8, 128), (32, 128)])
@pytest.mark.parametrize("layers", [None, 1, 3])
def test_keep(heads, layers):
    hkv, hd = heads
    paths = [[0, 1, 4], [0], [], [0, 2, 3, 7, 9], [1, 2], list(range(64)), [0] + list(range(5, 20)), [0, 1, 2]]
    old, most = [0, 5, 3, 14, 15, 30, 16, 47], 64
    kp, vp, table = pages_for(2, [o + 64 for o in old], 16, hkv, hd)
    shape = ((layers,) if layers else ()) + tuple(kp.shape)
    g = gen(0)
    kp, vp = normal(g, *shape), normal(g, *shape)
    want = kp.clone(), vp.clone()
    for x in want:
        for b, path in enumerate(paths):
            src = place(table, 16, b, [old[b] + i for i in path]) if path else None
            dst = place(table, 16, b, [old[b] + i for i in range(len(path))]) if path else None
            if path:
                x[..., dst[0], dst[1], :, :] = x[..., src[0], src[1], :, :].clone()
    path = ints(*[p + [-1] * (most - len(p)) for p in paths])
    op = _r().KeepDrafts(hkv, hd)
    op.forward(kp, vp, table, ints(*old), path, ints(*[len(p) for p in paths]))
    op.check()
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])


def test_keep_leaves_and_reports_bad_paths():
    kp, vp, table = pages_for(2, [40] * 3, 16, 2, 64)
    g = gen(1)
    kp, vp = normal(g, *kp.shape), normal(g, *vp.shape)
    k0, op = kp.clone(), _r().KeepDrafts(2, 64)

    def run(path, old=(5, 6, 7), kept=(1, 3, 1), tab=table):
        op.forward(kp, vp, tab, ints(*old), ints([0, -1, -1], path, [0, -1, -1]), ints(*kept))
        _reports(op)
        assert torch.equal(kp, k0)

    for path in ([0, 2, 2], [0, 3, 2], [0, 0, 3], [0, 2, 100], [0, 2, 2 ** 31 - 1], [-1, 2, 3]):
        run(path)
    run([0, 2, 3], old=(5, -1, 7))
    run([0, 2, 3], kept=(1, 4, 1))
    run([0, 2, 3], kept=(1, -1, 1))
    bad = table.clone()
    bad[1, 0] = kp.shape[0]
    run([0, 2, 3], tab=bad)
    op.forward(kp, vp, table, ints(5, 6, 7), ints([0, -1, -1], [0, 2, 3], [0, -1, -1]), ints(1, 3, 1))
    op.check()
    assert not torch.equal(kp, k0)


def test_keep_far_layers():
    """Layers beyond 2^31 elements of one another."""
    kp = torch.zeros(3, 300_000, 16, 1, 256, device="cuda", dtype=BF)  # 1.2 G elements a layer
    vp = kp[:, :, :, :, :]
    table = ints([299_999, 1])
    kp[:, 299_999, 9] = torch.arange(1, 4, device="cuda", dtype=BF)[:, None, None]
    op = _r().KeepDrafts(1, 256)
    op.forward(kp, vp, table, ints(4), ints([0, 5]), ints(2))
    op.check()
    assert torch.equal(kp[:, 299_999, 5], kp[:, 299_999, 9]) and int((kp != 0).sum()) == 6 * 256


# ---------------------------------------------------------------- distillation

def distill_case(n, d, v, k, seed=0, std=None):
    g = gen(seed)
    h, w = normal(g, n, d), normal(g, v, d, std=std or 2.0 / d ** 0.5)
    ids = torch.stack([torch.randperm(v, generator=g, device="cuda")[:k] for _ in range(n)]).to(I32)
    t = torch.randn(n, k, generator=g, device="cuda") * 2
    rw = torch.rand(n, generator=g, device="cuda") + 0.1
    return h, w, ids, t, rw


def check_distill(h, w, ids, t, rw, tau=1.0, piece=0, frozen=False, report=False):
    n, d = h.shape
    op = _r().VocabDistill(w, n, ids.shape[1], tau, piece_rows=piece)
    loss, loss2, dh = empty(n, dtype=F32), empty(n, dtype=F32), empty(n, d)
    dw = None if frozen else empty(*w.shape)
    op.loss(h, ids, t, loss)
    op.train(h, ids, t, rw, loss2, dh, dw)
    _reports(op) if report else op.check()
    want = D.distill(h, w, ids, t, tau, rw)
    T.close(loss, want["loss"], want["loss_tol"], "loss")
    T.close(loss2, want["loss"], want["loss_tol"], "loss of the step")
    T.close(dh, want["dh"], want["dh_tol"], "dh")
    if not frozen:
        T.close(dw, want["dw"], want["dw_tol"], "dw")
    return loss, dh, dw


@pytest.mark.parametrize("n,d,v,k", [(1, 64, 128, 1), (5, 64, 100, 3), (130, 256, 1000, 16),
                                     (257, 200, 1111, 128), (40, 1024, 4100, 100), (300, 64, 129, 129 - 1)])
@pytest.mark.parametrize("tau", [1.0, 2.0, 0.25])
def test_distill(n, d, v, k, tau):
    check_distill(*distill_case(n, d, v, k, seed=n), tau=tau)


@pytest.mark.parametrize("n", [1, 77, 128, 129, 333, 640])
@pytest.mark.parametrize("v", [19_999, 32_000])
def test_distill_few_rows_of_many_words(n, v):
    """More blocks of columns than the card takes at a time: tiles of 128 rows, or of 256."""
    h, w, ids, t, rw = distill_case(n, 72, v, 17, seed=n)
    if n > 8:
        ids[3::8] = -1
        h[3::8] = float("nan")
    check_distill(h, w, ids, t, rw, tau=0.7)


@pytest.mark.parametrize("d", [1000, 2048])
@pytest.mark.parametrize("v,k", [(1000, 100), (32_000, 16), (1000, 1)])
def test_distill_digits_of_many_terms(d, v, k):
    """Sums on the tensor cores lose up to 2^-23 of themselves at each of d / 16 steps, towards
    zero: a fourth of 2^-24 on average, and so 2^-30 d of a logit, 2^-19 at d = 2,048, which the
    loss of a sharp student has too.  Half of it may be left by the average's correction, and half
    as much again by the exponentials and logarithms at d = 1,000: 2^-20 of the losses."""
    h, w, ids, t, rw = distill_case(512, d, v, k, seed=d)
    loss, *_ = check_distill(h, w, ids, t, rw, tau=0.5)
    want = D.distill(h, w, ids, t, 0.5)["loss"]
    assert float((loss.double() - want).norm()) <= 2.0 ** -20 * float(want.norm())


def test_distill_rows_and_entries_that_do_not_count():
    """Negative ids, logits of -inf, rows without entries whose h may be NaN, in pieces."""
    h, w, ids, t, rw = distill_case(300, 128, 900, 20, seed=1)
    g = gen(5)
    ids[torch.rand(300, 20, generator=g, device="cuda") < 0.4] = -1
    t[torch.rand(300, 20, generator=g, device="cuda") < 0.2] = -float("inf")
    ids[::7] = -3
    t[3::7] = -float("inf")
    t[ids < 0] = float("nan")  # no entry: anything
    dead = ~((ids >= 0) & (t > -float("inf"))).any(-1)
    h2 = h.clone()
    h2[dead] = float("nan")
    a = check_distill(h2, w, ids, t, rw)
    assert (a[0][dead] == 0).all() and (a[1][dead] == 0).all() and dead.sum() > 80
    for piece in (64, 256, 299):
        check_distill(h2, w, ids, t, rw, piece=piece)
    check_distill(h2, w, ids, t, rw, frozen=True)


def test_distill_no_rows_count():
    h, w, ids, t, rw = distill_case(9, 64, 300, 4)
    ids[:] = -1
    loss, dh, dw = check_distill(h, w, ids, t, rw)
    assert not dh.any() and not dw.any() and not loss.any()


def test_distill_the_same_word_twice():
    h, w, ids, t, rw = distill_case(50, 64, 300, 12, seed=2)
    ids[:, 5], ids[:, 9], ids[:, 11] = ids[:, 0], ids[:, 0], ids[:, 3]
    ids[7] = 299
    check_distill(h, w, ids, t, rw)


def test_distill_words_outside_are_reported():
    h, w, ids, t, rw = distill_case(50, 64, 300, 12, seed=2)
    ids[4, 2], ids[9, 0] = 300, 2 ** 31 - 1
    check_distill(h, w, ids, t, rw, report=True)


def test_distill_neighbours():
    """Entries side by side, in one chunk of columns, at blocks' borders and the last word."""
    h, w, _, t, rw = distill_case(64, 64, 1000, 128, seed=3)
    ids = torch.stack([torch.arange(128, device="cuda") + i * 13 % 873 for i in range(64)]).to(I32)
    check_distill(h, w, ids, t, rw)
    check_distill(h, w, ids.flip(1).contiguous(), t, rw)


def test_distill_one_word_is_the_next_token_loss():
    h, w, ids, t, rw = distill_case(200, 256, 2000, 1, seed=4)
    loss, dh, dw = check_distill(h, w, ids, t, rw)
    op, other = _r().VocabLoss(w, 200), empty(200, dtype=F32)
    op.loss(h, ids[:, 0].contiguous(), other)
    assert (loss - other).abs().max() < 1e-5


def test_distill_a_student_that_is_the_teacher():
    """All its mass on the entries: a loss near zero keeps its digits, by the bound's own terms."""
    g = gen(9)
    n, d, v, k = 64, 128, 600, 8
    ids = torch.stack([torch.randperm(v, generator=g, device="cuda")[:k] for _ in range(n)]).to(I32)
    w = normal(g, v, d, std=0.02)
    w[:, 0] = -60.0 / 8
    h = normal(g, n, d)
    h[:, 0] = 8.0
    # the entries' logits are raised by a second column of the row's own
    x = h.double() @ w.double().T
    t = x.gather(1, ids.long()).float()
    for scale in (0.0, 1e-2, 1.0):
        check_distill(h, w, ids, t + scale * torch.randn(n, k, generator=g, device="cuda"), torch.ones(n, device="cuda"))
    # a vocabulary of the entries alone: the student is the teacher to its logits' rounding
    small = w[:k].contiguous()
    small[:, 0] = normal(g, k)
    all_ids = torch.arange(k, device="cuda", dtype=I32).expand(n, k).contiguous()
    t = (h.double() @ small.double().T).float()
    loss, *_ = check_distill(h, small, all_ids, t, torch.ones(n, device="cuda"))
    assert (loss >= 0).all() and loss.max() < 1e-9


def test_distill_strides_and_fixed_bits():
    h, w, ids, t, rw = distill_case(100, 128, 700, 9, seed=6)
    wide, tall = empty(100, 200), empty(700, 136)
    wide[:, 8:136], tall[:, :128] = h, w
    a = check_distill(h, w, ids, t, rw)
    b = check_distill(wide[:, 8:136], tall[:, :128], ids, t, rw)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_distill_in_a_graph():
    h, w, ids, t, rw = distill_case(100, 128, 700, 9, seed=6)
    want = check_distill(h, w, ids, t, rw)
    op = _r().VocabDistill(w, 100, 9)
    loss, dh, dw = empty(100, dtype=F32), empty(100, 128), empty(700, 128)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op.train(h, ids, t, rw, loss, dh, dw)
    for _ in range(2):
        loss.fill_(1), dh.fill_(1), dw.fill_(1)
        op.ws.fill_(255)
        g.replay()
        assert torch.equal(loss, want[0]) and torch.equal(dh, want[1]) and torch.equal(dw, want[2])
