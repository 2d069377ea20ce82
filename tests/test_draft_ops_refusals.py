"""What answering with drafted tokens refuses, on the host before any launch (no GPU needed),
and its 64-bit definitions against differences."""
import ctypes as C
import random

import pytest
import torch

from paper_2607_16074_gb300 import build as B
from paper_2607_16074_gb300 import jnx as J
from tests import draft_ops_ref as D
from tests.test_text_ops_refusals import INV, PTR, UNS, WS, refused, rope, rows


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()


def cache(k=PTR, v=PTR, pages=8, room=16, page=4096, row=256, head=128):
    return C.byref(J.jnx_kv_cache(k, v, pages, room, page, row, head))


def pages(table=PTR, ld=4, seqs=2, entries=4):
    return C.byref(J.jnx_pages(table, ld, seqs, entries))


BAD_PAGES = (dict(table=None), dict(ld=-1), dict(seqs=-1), dict(entries=-1))
BAD_CACHES = (dict(k=None), dict(v=PTR + 2), dict(pages=-1), dict(room=-1), dict(row=129), dict(page=4),
              dict(head=12))


def test_append_paged_refuses():
    def f(r=rope(), x=PTR, q=rows(), c=cache(), p=pages(), seq=PTR, at=PTR, n=3):
        return J.lib().jnx_op_qk_norm_rope_append_paged(r, x, 1536, PTR, n, q, c, p, seq, at, None, None)
    for bad in (dict(x=None), dict(q=rows(None)), dict(c=None), dict(p=None), dict(seq=None), dict(at=None),
                dict(n=-1), *(dict(p=pages(**x)) for x in BAD_PAGES), *(dict(c=cache(**x)) for x in BAD_CACHES)):
        refused(f(**bad), INV)
    refused(f(r=rope(hd=96)), UNS)
    assert f(n=0) == J.JNX_OK


def test_tree_refuses():
    L = J.lib()
    need = L.jnx_op_tree_attention_workspace_bytes(2, 5, 8, 128, 64)

    def f(c=cache(), p=pages(), h=8, hkv=2, hd=128, n=5, q=rows(), cu=PTR, old=PTR, sees=PTR, out=rows(),
          ws=PTR, size=need):
        return L.jnx_op_tree_attention(c, p, h, hkv, hd, n, q, cu, old, sees, out, ws, size, None, None)
    for bad in (dict(c=None), dict(p=None), dict(h=7), dict(hkv=0), dict(n=-1), dict(q=rows(None)),
                dict(q=rows(row=12)), dict(cu=None), dict(old=None), dict(sees=None), dict(out=rows(PTR + 2)),
                *(dict(p=pages(**x)) for x in BAD_PAGES), *(dict(c=cache(**x)) for x in BAD_CACHES)):
        refused(f(**bad), INV)
    for bad in (dict(hd=80), dict(h=130), dict(c=cache(room=24)), dict(c=cache(room=1)),
                dict(c=cache(room=1 << 30))):
        refused(f(**bad), UNS)
    if need:
        refused(f(ws=None), WS)
        refused(f(ws=PTR + 8), WS)
        refused(f(size=need - 1), WS)
    assert f(n=0) == f(p=pages(seqs=0)) == J.JNX_OK


def test_verify_refuses():
    def f(p=PTR, ldp=100, q=PTR, ldq=100, tok=PTR, par=PTR, u=PTR, cu=PTR, b=2, n=5, v=100, most=8, path=PTR,
          kept=PTR, nxt=PTR):
        return J.lib().jnx_op_verify_drafts(p, ldp, q, ldq, tok, par, u, cu, b, n, v, most, path, kept, nxt,
                                            None, None)
    for bad in (dict(p=None), dict(ldp=-1), dict(ldq=-8), dict(tok=None), dict(par=None), dict(u=None),
                dict(cu=None), dict(b=-1), dict(n=-1), dict(v=0), dict(most=0), dict(path=None),
                dict(kept=None), dict(nxt=None)):
        refused(f(**bad), INV)
    refused(f(most=65), UNS)
    assert f(b=0) == J.JNX_OK


def test_keep_refuses():
    def f(c=cache(), layers=3, step=1 << 16, p=pages(), hkv=2, hd=128, old=PTR, path=PTR, ld=8, kept=PTR,
          most=8):
        return J.lib().jnx_op_keep_drafts(c, layers, step, p, hkv, hd, old, path, ld, kept, most, None, None)
    for bad in (dict(c=None), dict(layers=-1), dict(step=4), dict(p=None), dict(hkv=0), dict(old=None),
                dict(path=None), dict(ld=-1), dict(kept=None), dict(most=-1),
                *(dict(p=pages(**x)) for x in BAD_PAGES), *(dict(c=cache(**x)) for x in BAD_CACHES)):
        refused(f(**bad), INV)
    for bad in (dict(hd=80), dict(most=65), dict(layers=1 << 17)):
        refused(f(**bad), UNS)
    assert f(layers=0) == f(p=pages(seqs=0)) == f(most=0) == J.JNX_OK


def test_distill_refuses():
    L = J.lib()
    big = 1 << 30

    def f(h=PTR, ldh=64, w=PTR, ldw=64, ids=PTR, t=PTR, top=4, tau=1.0, n=3, v=100, d=64, loss=PTR, ws=PTR,
          size=big):
        return L.jnx_op_vocab_distill(h, ldh, w, ldw, ids, t, top, tau, n, v, d, loss, ws, size, None, None)

    def g(rw=PTR, dh=PTR, lddh=64, dw=PTR, lddw=64, n=3, ws=PTR, size=big, tau=1.0, top=4, t=PTR):
        return L.jnx_op_vocab_distill_train(PTR, 64, PTR, 64, PTR, t, top, tau, rw, n, 100, 64, 0, PTR, dh,
                                            lddh, dw, lddw, ws, size, None, None)
    for bad in (dict(h=None), dict(ldh=60), dict(ldw=72 - 4), dict(ids=None), dict(t=None), dict(top=0),
                dict(tau=0.0), dict(tau=-1.0), dict(tau=float("inf")), dict(tau=float("nan")),
                dict(tau=1e-40), dict(n=-1), dict(v=0), dict(d=60), dict(loss=None)):
        refused(f(**bad), INV)
    for bad in (dict(rw=None), dict(dh=None), dict(dh=PTR + 8), dict(lddh=56), dict(lddw=65), dict(dw=PTR + 2),
                dict(tau=0.0), dict(top=0), dict(t=None)):
        refused(g(**bad), INV)
    refused(f(top=129), UNS)
    refused(g(top=129), UNS)
    refused(f(ws=None), WS)
    refused(f(size=L.jnx_op_vocab_distill_workspace_bytes(3, 100, 64, 4) - 1), WS)
    refused(g(ws=None), WS)
    assert f(n=0) == J.JNX_OK
    a, b = (L.jnx_op_vocab_distill_train_workspace_bytes(3, 100, 64, k, 0) for k in (1, 128))
    assert L.jnx_op_vocab_loss_train_workspace_bytes(3, 100, 64, 0) < a < b


def test_distill_gradient_by_differences():
    g = torch.Generator().manual_seed(0)
    n, d, v, k, tau, eps = 4, 6, 11, 3, 1.7, 1e-6
    h, w = torch.randn(n, d, generator=g, dtype=torch.float64), torch.randn(v, d, generator=g, dtype=torch.float64)
    ids = torch.tensor([[0, 3, 5], [10, -1, 2], [-1, -1, -1], [4, 4, 1]])
    t, rw = torch.randn(n, k, generator=g, dtype=torch.float64), torch.rand(n, generator=g, dtype=torch.float64)
    r = D.distill(h, w, ids, t, tau, rw)
    value = lambda h, w: float((D.distill(h, w, ids, t, tau)["loss"] * rw).sum())  # noqa: E731
    for x, grad in ((h, r["dh"]), (w, r["dw"])):
        for i in range(x.numel()):
            keep = float(x.view(-1)[i])
            x.view(-1)[i] = keep + eps
            up = value(h, w)
            x.view(-1)[i] = keep - eps
            down = value(h, w)
            x.view(-1)[i] = keep
            # central differences: eps^2 of the third derivative, 2^-52 / eps of the sum
            assert abs((up - down) / (2 * eps) - float(grad.reshape(-1)[i])) < 1e-8
    assert (r["loss"][2] == 0) and not r["dh"][2].any()


def test_verification_by_hand():
    """Walks that can be followed on paper."""
    p = torch.tensor([[0.5, 0.5, 0.0], [0.2, 0.3, 0.5]], dtype=torch.float64)
    q = torch.tensor([[0.25, 0.75, 0.0], [1.0, 0.0, 0.0]], dtype=torch.float64)
    u = torch.tensor
    # 0.75 u < 0.5 takes word 1; then the second row's own sums 0.2, 0.5, 1
    assert D.verify(p, q, [0, 1], [-1, 0], u([0.4, 0.66]), 3) == ([0, 1], 1)
    # not taken: what is left is (0.25, 0, 0)
    assert D.verify(p, q, [0, 1], [-1, 0], u([0.99, 0.67]), 3) == ([0], 0)
    # two certain guesses: word 0 is not taken at u = 0.5, then word 1 holds all that is left
    p = p[[0, 1, 1]]
    assert D.verify(p, None, [0, 0, 1], [-1, 0, 0], u([0.9, 0.5, 0.99]), 3)[0] == [0, 2]


def test_ancestors():
    rng = random.Random(0)
    parents = [-1] + [rng.randrange(i) for i in range(1, 64)]
    m = D.ancestors(parents)
    for i in range(64):
        seen, j = set(), i
        while j >= 0:
            seen.add(j)
            j = parents[j]
        assert {k for k in range(64) if m[i, k]} == seen
        assert D.bits(m[i].tolist()) % (1 << 64) == sum(1 << k for k in seen)
