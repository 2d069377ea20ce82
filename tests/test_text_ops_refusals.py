"""What the text operators refuse, on the host before any launch (no GPU needed), and the
work lists of packed prompts."""
import ctypes as C
import itertools

import numpy as np
import pytest

from paper_2607_16074_gb300 import build as B
from paper_2607_16074_gb300 import jnx as J

BUF = C.create_string_buffer(1 << 16)
PTR = (C.addressof(BUF) + 63) & ~63


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()


def rows(ptr=PTR, row=1024, head=128):
    return C.byref(J.jnx_head_rows(ptr, row, head))


def rope(h=8, hkv=2, hd=128, sections=(64,), theta=1e4, eps=1e-6, gq=None):
    return C.byref(J.jnx_qk_rope(h, hkv, hd, len(sections), (C.c_int32 * 4)(*sections), theta, eps,
                                 gq, None))


def prompt(q=(5, 3), kv=(5, 3), prefix=None, device=True):
    keep = [np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (q, kv)]
    if prefix is not None:
        keep.append(np.asarray(prefix, np.int32))
    host = [x.ctypes.data_as(J.P32) for x in keep] + [None] * (3 - len(keep))
    dev = [PTR if device else None] * 2 + [PTR if prefix is not None else None]
    p = J.jnx_prompt(len(q), *dev, *host, PTR, 1, 1, 1, 1)
    p.keep = keep
    return p


def refused(code, expected):
    assert code == expected and J.jnx_last_error()


INV, UNS, WS = J.JNX_ERR_INVALID_ARG, J.JNX_ERR_UNSUPPORTED, J.JNX_ERR_WORKSPACE


@pytest.mark.parametrize("bad,code", [
    (dict(hd=96), UNS), (dict(sections=(65,)), INV), (dict(sections=(32, 40)), INV),
    (dict(sections=(-1,)), INV), (dict(theta=0.0), INV), (dict(eps=-1.0), INV), (dict(h=-1), INV),
    (dict(gq=PTR + 2), INV)])
def test_rope_refuses(bad, code):
    L = J.lib()
    refused(L.jnx_op_qk_norm_rope(rope(**bad), PTR, 1536, PTR, 4, rows(), rows(), None), code)
    refused(L.jnx_op_qk_norm_rope_backward(rope(**bad), PTR, 1536, PTR, 4, rows(), rows(), PTR, PTR,
                                           PTR, PTR, 1 << 20, None), code)


def test_rope_refuses_pointers_and_strides():
    L, r = J.lib(), rope()
    f = lambda x=PTR, ld=1536, pos=PTR, n=4, q=rows(), k=rows(): L.jnx_op_qk_norm_rope(  # noqa: E731
        r, x, ld, pos, n, q, k, None)
    for bad in (dict(x=None), dict(x=PTR + 8), dict(ld=1535), dict(ld=1528), dict(pos=None),
                dict(n=-1), dict(q=rows(PTR + 4)), dict(q=rows(row=1020)), dict(k=rows(head=4)),
                dict(k=rows(None))):
        refused(f(**bad), INV)
    assert f(n=0) == J.JNX_OK
    refused(L.jnx_op_qk_norm_rope_backward(rope(gq=PTR), PTR, 1536, PTR, 4, rows(), rows(), PTR, PTR,
                                           None, PTR, 8, None), WS)
    refused(L.jnx_op_qk_norm_rope_backward(rope(gq=PTR), PTR, 1536, PTR, 4, rows(), rows(), PTR,
                                           None, None, PTR, 1 << 20, None), INV)
    cache = J.jnx_kv_cache(PTR, PTR, 2, 4, 1024, 256, 128)
    a = lambda c, slot=PTR, at=PTR: L.jnx_op_qk_norm_rope_append(  # noqa: E731
        r, PTR, 1536, PTR, 4, rows(), C.byref(c) if c else None, slot, at, None, None)
    for c, kw in ((None, {}), (cache, dict(slot=None)), (cache, dict(at=None)),
                  (J.jnx_kv_cache(PTR, None, 2, 4, 1024, 256, 128), {}),
                  (J.jnx_kv_cache(PTR, PTR, -1, 4, 1024, 256, 128), {}),
                  (J.jnx_kv_cache(PTR, PTR, 2, 4, 1024, 250, 128), {})):
        refused(a(c, **kw), INV)


def attend(p, h=8, hkv=2, hd=128, q=rows(), k=rows(), v=rows(), out=rows()):
    return J.lib().jnx_op_prompt_attention(C.byref(p), h, hkv, hd, q, k, v, out, None, None, None, None)


def test_prompt_attention_refuses():
    for kw, code in ((dict(h=7), INV), (dict(hkv=0), INV), (dict(hd=80), UNS), (dict(h=130), UNS),
                     (dict(q=rows(None)), INV), (dict(k=rows(PTR + 2)), INV),
                     (dict(v=rows(row=129)), INV), (dict(out=rows(head=12)), INV)):
        refused(attend(prompt(), **kw), code)
    bad = prompt()
    bad.keep[0][1] = 9
    refused(attend(bad), INV)
    refused(attend(prompt(prefix=(0, -1))), INV)
    refused(attend(prompt(device=False)), INV)
    bad = prompt()
    bad.items = None
    refused(attend(bad), INV)
    assert attend(prompt(q=(), kv=())) == J.JNX_OK


def test_prompt_attention_backward_refuses():
    L = J.lib()
    f = lambda p=prompt(), lse=PTR, ws=PTR, n=1 << 16, dk=rows(): \
        L.jnx_op_prompt_attention_backward(C.byref(p), 8, 2, 128, rows(), rows(), rows(), rows(), None, lse,
                                           rows(), rows(), dk, rows(), ws, n, None, None)
    refused(f(lse=None), INV)
    refused(f(dk=rows(None)), INV)
    refused(f(ws=None), WS)
    refused(f(n=L.jnx_op_prompt_attention_backward_workspace_bytes(C.byref(prompt()), 8, 2, 128) - 1), WS)
    assert f(p=prompt(q=(0,), kv=(0,))) == J.JNX_OK


@pytest.mark.parametrize("missing", ["cu_q", "cu_kv", "items", "prefix"])
def test_prompt_attention_backward_refuses_keys_without_device_arrays(missing):
    """Keys that no row reads still have gradients to write, by the device's arrays."""
    p = prompt(q=(0, 0), kv=(5, 3), prefix=(1, 0))
    J.lib().jnx_prompt_items(C.byref(p), 8, 2, 128, None, 0)
    setattr(p, missing, None)
    refused(J.lib().jnx_op_prompt_attention_backward(
        C.byref(p), 8, 2, 128, rows(), rows(), rows(), rows(), None, PTR, rows(), rows(), rows(),
        rows(), PTR, 1 << 16, None, None), INV)


def test_prompt_attention_backward_refuses_a_prefix_that_the_host_does_not_know():
    """The workspace is sized by the host's arrays, and used by the device's."""
    p = prompt(q=(5, 3), kv=(900, 700), prefix=(800, 0))
    p.h_prefix = None
    J.lib().jnx_prompt_items(C.byref(p), 8, 2, 128, None, 0)
    refused(J.lib().jnx_op_prompt_attention_backward(
        C.byref(p), 8, 2, 128, rows(), rows(), rows(), rows(), None, PTR, rows(), rows(), rows(),
        rows(), PTR, 1 << 30, None, None), INV)


def test_prompt_attention_refuses_a_list_that_is_not_its_own():
    """A list of other heads or lengths, or with its counts changed: the kernels would leave rows
    out, or write more parts than the workspace has."""
    L = J.lib()
    lens = dict(q=(900, 700), kv=(900, 700), prefix=(300, 0))

    def listed(heads, **lens):
        p = prompt(**lens)
        assert L.jnx_prompt_items(C.byref(p), *heads, None, 0) > 0
        return p

    def forward(p, heads=(8, 1, 256)):
        return L.jnx_op_prompt_attention(C.byref(p), *heads, rows(), rows(), rows(), rows(), None,
                                         None, None, None)

    def backward(p, heads=(8, 1, 256)):
        return L.jnx_op_prompt_attention_backward(
            C.byref(p), *heads, rows(), rows(), rows(), rows(), None, PTR, rows(), rows(), rows(), rows(),
            PTR, 1 << 40, None, None)

    for heads in ((16, 1, 256), (8, 8, 256), (8, 1, 64)):
        other = listed(heads, **lens)
        refused(forward(other), INV)
        refused(backward(other), INV)
    # as many row tiles, but other parts of the keys' rows
    for other in (listed((8, 1, 256), q=(900, 700), kv=(1100, 700), prefix=(300, 0)),
                  listed((8, 1, 256), q=(900, 700), kv=(900, 700), prefix=(0, 0))):
        own = prompt(**lens)
        for n in ("n_forward", "n_keys", "n_queries", "n_parts"):
            setattr(own, n, getattr(other, n))
        refused(backward(own), INV)
    for n in ("n_forward", "n_keys", "n_queries", "n_parts"):
        for by in (-1, 1):
            p = listed((8, 1, 256), **lens)
            setattr(p, n, getattr(p, n) + by)
            refused(backward(p), INV)
            if n == "n_forward":
                refused(forward(p), INV)


def test_decode_refuses():
    L = J.lib()
    cache = J.jnx_kv_cache(PTR, PTR, 2, 4, 1024, 256, 128)
    need = L.jnx_op_decode_attention_workspace_bytes(3, 8, 128)

    def f(b=3, h=8, hkv=2, hd=128, c=cache, q=rows(), slot=PTR, n=PTR, out=rows(), ws=PTR, nws=need):
        return L.jnx_op_decode_attention(C.byref(c), b, h, hkv, hd, q, slot, n, out, ws, nws, None,
                                         None)
    for kw, code in ((dict(b=-1), INV), (dict(h=9), INV), (dict(hd=32), UNS), (dict(q=rows(None)), INV),
                     (dict(out=rows(row=100)), INV), (dict(slot=None), INV), (dict(n=None), INV),
                     (dict(c=J.jnx_kv_cache(None, PTR, 2, 4, 1024, 256, 128)), INV)):
        refused(f(**kw), code)
    assert f(b=0) == J.JNX_OK


def test_vocab_loss_refuses():
    L = J.lib()
    need = L.jnx_op_vocab_loss_train_workspace_bytes(4, 100, 64, 0)

    def f(h=PTR, ldh=64, w=PTR, ldw=64, t=PTR, rw=PTR, n=4, v=100, d=64, loss=PTR, dh=PTR, lddh=64,
          dw=PTR, lddw=64, ws=PTR, nws=need):
        return L.jnx_op_vocab_loss_train(h, ldh, w, ldw, t, rw, n, v, d, 0, loss, dh, lddh, dw, lddw,
                                         ws, nws, None, None)
    for kw in (dict(h=None), dict(h=PTR + 8), dict(ldh=60), dict(ldh=68), dict(w=None), dict(ldw=62),
               dict(t=None), dict(rw=None), dict(n=-1), dict(v=0), dict(d=60), dict(d=0),
               dict(loss=None), dict(dh=None), dict(dh=PTR + 4), dict(lddh=63), dict(dw=PTR + 6),
               dict(lddw=56)):
        refused(f(**kw), INV)
    refused(f(ws=None), WS)
    refused(f(nws=need - 1), WS)
    assert f(n=0, dw=None) == J.JNX_OK


@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 256, 2 ** 31 - 8192])
def test_vocab_loss_refuses_rows_that_its_counts_cannot_hold(n):
    """Rows are counted and launched for in 32 bits, beyond the last row too."""
    L = J.lib()
    refused(L.jnx_op_vocab_loss(PTR, 64, PTR, 64, PTR, n, 100, 64, PTR, PTR, 1 << 62, None, None), UNS)
    refused(L.jnx_op_vocab_loss_train(PTR, 64, PTR, 64, PTR, PTR, n, 100, 64, 0, PTR, PTR, 64, PTR, 64, PTR,
                                      1 << 62, None, None), UNS)


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 1, 256), (12, 4, 128), (14, 2, 64)])
def test_work_lists_cover_every_row_and_key_once(heads):
    """Each pass visits every row (or key, in each part of its rows) of every sequence, the
    longest work first."""
    h, hkv, hd = heads
    q, kv, pre = (300, 0, 1, 129, 40), (300, 7, 5, 60, 400), (0, 3, 0, 9, 390)
    p = prompt(q, kv, pre)
    n = J.lib().jnx_prompt_items(C.byref(p), h, hkv, hd, None, 0)
    out = np.zeros((n, 2), np.int32)
    assert J.lib().jnx_prompt_items(C.byref(p), h, hkv, hd, out.ctypes.data, n) == n
    assert n == p.n_forward + p.n_keys + p.n_queries
    tok = 128 // (h // hkv)
    steps = (tok * (1 if hd == 256 else 2), 128, tok)

    def visible(s, i):  # keys that row i sees
        return max(0, min(kv[s], max(kv[s] - q[s] + i + 1, pre[s])))

    def parts(s, a):  # of a key tile's rows
        rows = sum(1 for i in range(q[s]) if visible(s, i) > a) * (h // hkv)
        return max(1, -(-rows // 2048)) if hkv * -(-kv[s] // 128) < 152 else 1

    at = 0
    for count, step, lens, pass_ in zip((p.n_forward, p.n_keys, p.n_queries), steps, (q, kv, q), range(3)):
        items, at = out[at:at + count], at + count
        seen = set()
        for s, y in items:
            a, part = (y // 128 * 128, y % 128) if pass_ == 1 else (y, 0)
            for i in range(a, min(a + step, lens[s])):
                assert (s, i, part) not in seen
                seen.add((int(s), int(i), int(part)))
        assert seen == {(s, i, k) for s, n_ in enumerate(lens) for i in range(n_)
                        for k in range(parts(s, i // 128 * 128) if pass_ == 1 else 1)}
        if pass_ == 1:
            assert p.n_parts == max(k for _, _, k in seen) + 1

        def cost(s, a):
            if pass_ == 1:
                a = a // 128 * 128
                return sum(1 for i in range(q[s]) if visible(s, i) > a) // parts(s, a)
            return visible(s, min(a + step, q[s]) - 1)
        costs = [cost(int(s), int(a)) for s, a in items]
        assert all(x >= y for x, y in itertools.pairwise(costs))


@pytest.mark.parametrize("heads,lens", [
    ((8, 1, 256), [12000]), ((8, 1, 256), [12000] + [840] * 48),
    ((8, 1, 256), [16000] + [400] * 124), ((8, 1, 256), [840] * 26), ((4, 2, 128), [3000, 70] * 9),
    ((64, 1, 64), [5000] + [20] * 500), ((64, 1, 64), [9, 5000, 90]), ((32, 8, 128), [2900] * 24)])
def test_prompt_backward_workspace_holds_the_parts_alone(heads, lens):
    """Sums are kept for tiles whose rows are taken in parts, and tiles of as many rows as one of
    their parts; not for every key as often as the longest sequence has parts.  The parts of a
    tile follow one another in the list, which the joining of their sums goes by."""
    h, hkv, hd = heads
    L, p = J.lib(), prompt(lens, lens)
    n = L.jnx_prompt_items(C.byref(p), h, hkv, hd, None, 0)
    out = np.zeros((n, 2), np.int32)
    L.jnx_prompt_items(C.byref(p), h, hkv, hd, out.ctypes.data, n)
    items = out[p.n_forward:p.n_forward + p.n_keys]
    parts = {}
    for s, y in items:
        parts.setdefault((s, y // 128), []).append(y % 128)
    assert all(x == list(range(len(x))) for x in parts.values())
    for i, (s, y) in enumerate(items):
        if y % 128:
            assert items[i - 1][0] == s and items[i - 1][1] == y - 1
    inside = [i for i, (s, y) in enumerate(items) if len(parts[s, y // 128]) > 1]
    # an item of a tile in parts has over 1,024 rows; others of over 1,024 may lie among them
    like = sum(1 for s, y in items if (lens[s] - y // 128 * 128) * (h // hkv) >= 1024)
    slab = hkv * 2 * 128 * hd * 4
    need = L.jnx_op_prompt_attention_backward_workspace_bytes(C.byref(p), h, hkv, hd)
    rows = sum(lens) * h * 12 + 512
    assert need <= rows + (like * slab if inside else 0)
    if inside:
        assert need >= rows - 512 + (max(inside) + 1) * slab


@pytest.mark.parametrize("vocab,d,piece", [(32000, 2048, 0), (32000, 4096, 256), (32000, 8192, 1000),
                                           (50257, 512, 0), (151936, 1024, 1000), (300, 64, 0)])
def test_vocab_workspaces_for_many_rows_hold_fewer(vocab, d, piece):
    """A workspace made for so many rows serves every smaller call: sizes never fall."""
    L = J.lib()
    for size in (lambda n: L.jnx_op_vocab_loss_train_workspace_bytes(n, vocab, d, piece),
                 lambda n: L.jnx_op_vocab_loss_workspace_bytes(n, vocab, d)):
        sizes = [size(n) for n in range(0, 3000)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))
