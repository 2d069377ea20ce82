"""The text operators against their definitions in 64 bits (tests/text_ops_ref.py, where
the tolerances are derived), at the sizes, masks and layouts where they can go wrong."""
import math

import pytest
import torch

from tests import text_ops_ref as T

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
HEADS = [(4, 4, 64), (8, 1, 256), (8, 2, 128), (12, 4, 128), (14, 2, 64), (4, 4, 256), (64, 1, 64)]


def _r():
    from paper_2607_16074_gb300 import runtime as R
    return R


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(BF)


def empty(*shape, dtype=BF):
    """Filled with NaN: what a kernel leaves unwritten shows."""
    return torch.full(shape, float("nan"), device="cuda", dtype=dtype)


# ---------------------------------------------------------------- norms and rotations

def rope_case(heads, n, sections, seed=0, norms=True, far=0, theta=10000.0):
    h, hkv, hd = heads
    g = gen(seed)
    qkv = normal(g, n, (h + 2 * hkv) * hd)
    gq, gk = ((1 + normal(g, hd, std=0.2)) if norms else None for _ in range(2))
    pos = torch.randint(-9, 5000, (len(sections), n), generator=g, device="cuda", dtype=torch.int32) + far
    op = _r().QKNormRope(h, hkv, hd, gq, gk, sections=sections, theta=theta)
    x = qkv.view(n, h + 2 * hkv, hd)
    want = [T.norm_rope(x[:, a:b], gamma, pos, sections, theta, 1e-6)
            for a, b, gamma in ((0, h, gq), (h, h + hkv, gk))]
    return op, qkv, pos, (gq, gk), want


def sections_of(hd, axes):
    s = {1: [1.0], 2: [0.5, 0.5], 3: [0.25, 0.375, 0.375], 4: [0.25, 0.25, 0.25, 0.125]}[axes]
    return tuple(int(x * (hd // 2)) for x in s)  # four axes leave an eighth unturned


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("n,axes", [(1, 1), (7, 3), (130, 2), (33, 4)])
def test_norm_rope(heads, n, axes):
    h, hkv, hd = heads
    op, qkv, pos, _, want = rope_case(heads, n, sections_of(hd, axes), n)
    q, k = empty(n, h, hd), empty(n, hkv, hd)
    op.forward(qkv, pos, q, k)
    T.close(q, want[0], T.norm_rope_bound(want[0]), "q")
    T.close(k, want[1], T.norm_rope_bound(want[1]), "k")


def test_norm_rope_without_norms_or_axes():
    op, qkv, pos, _, want = rope_case((8, 2, 128), 9, (64,), norms=False)
    q, k = empty(9, 8, 128), empty(9, 2, 128)
    op.forward(qkv, pos, q, k)
    T.close(q, want[0], T.norm_rope_bound(want[0]), "q")
    op = _r().QKNormRope(8, 2, 128, sections=())
    op.forward(qkv, pos[:0], q, k)  # nothing turns, nothing is scaled: the rows themselves
    assert torch.equal(q, qkv.view(9, 12, 128)[:, :8]) and torch.equal(k, qkv.view(9, 12, 128)[:, 8:10])


@pytest.mark.parametrize("far", [2_000_000_000, -2_000_000_000, 123_456_789])
def test_norm_rope_at_far_positions(far):
    """A position of 31 bits turns as exactly as a small one."""
    op, qkv, pos, _, want = rope_case((4, 4, 64), 17, (16, 16), far=far)
    q, k = empty(17, 4, 64), empty(17, 4, 64)
    op.forward(qkv, pos, q, k)
    # the 64-bit reference itself loses 2^-22 of a radian at 2^31
    T.close(q, want[0], 2 * T.norm_rope_bound(want[0]), "q")


def test_norm_rope_in_place_and_strided():
    heads, n = (8, 2, 128), 21
    op, qkv, pos, _, want = rope_case(heads, n, (64,))
    x = qkv.view(n, 12, 128)
    v = x[:, 10:].clone()
    q = empty(8, n, 128).transpose(0, 1)  # head-major
    op.forward(qkv, pos, q, x[:, 8:10])
    T.close(q, want[0], T.norm_rope_bound(want[0]), "q")
    T.close(x[:, 8:10], want[1], T.norm_rope_bound(want[1]), "k")
    assert torch.equal(x[:, 10:], v)


def test_norm_rope_zero_and_tiny_rows():
    """A zero row stays zero; eps bounds the scale of a tiny one."""
    op, qkv, pos, (gq, gk), _ = rope_case((4, 4, 64), 5, (32,))
    qkv[0] = 0
    qkv[1] *= 1e-30
    q, k = empty(5, 4, 64), empty(5, 4, 64)
    op.forward(qkv, pos, q, k)
    want = T.norm_rope(qkv.view(5, 12, 64)[:, :4], gq, pos, (32,), 10000.0, 1e-6)
    T.close(q, want, T.norm_rope_bound(want), "q")
    assert (q[0] == 0).all()


@pytest.mark.parametrize("heads", HEADS)
def test_norm_rope_append(heads):
    h, hkv, hd = heads
    n, slots, room = 11, 17, 9
    op, qkv, pos, _, want = rope_case(heads, n, sections_of(hd, 3), 3)
    g = gen(4)
    kc, vc = normal(g, slots, room, hkv, hd), normal(g, slots, room, hkv, hd)
    k0, v0 = kc.clone(), vc.clone()
    slot = torch.randperm(slots, generator=g, device="cuda")[:n].to(torch.int32)
    at = torch.randint(0, room, (n,), generator=g, device="cuda", dtype=torch.int32)
    q = empty(n, h, hd)
    op.append(qkv, pos, q, kc, vc, slot, at)
    op.check()
    T.close(q, want[0], T.norm_rope_bound(want[0]), "q")
    i = (slot.long(), at.long())
    T.close(kc[i], want[1], T.norm_rope_bound(want[1]), "k")
    assert torch.equal(vc[i], qkv.view(n, -1, hd)[:, h + hkv:])
    k0[i], v0[i] = kc[i], vc[i]
    assert torch.equal(kc, k0) and torch.equal(vc, v0)  # nothing else was written


def test_norm_rope_append_reports_rows_outside():
    from paper_2607_16074_gb300 import jnx as J
    op, qkv, pos, _, want = rope_case((4, 4, 64), 4, (32,))
    kc = torch.zeros(3, 5, 4, 64, device="cuda", dtype=BF)
    vc, q = torch.zeros_like(kc), empty(4, 4, 64)
    i32 = lambda *v: torch.tensor(v, device="cuda", dtype=torch.int32)  # noqa: E731
    op.append(qkv, pos, q, kc, vc, i32(0, 3, 1, -1), i32(4, 0, 5, 0))
    with pytest.raises(J.JnxError) as e:
        op.check()
    assert e.value.code == J.JNX_ERR_DEVICE_BOUNDS
    op.check()  # cleared
    T.close(kc[0, 4], want[1][0], T.norm_rope_bound(want[1][0]))
    kc[0, 4] = 0
    assert (kc == 0).all() and (vc[1:] == 0).all()
    T.close(q, want[0], T.norm_rope_bound(want[0]))  # queries are written all the same


def test_check_sees_a_call_on_another_stream():
    """A report of a kernel that still waits for its turn on a stream of its own."""
    from paper_2607_16074_gb300 import jnx as J
    op, qkv, pos, _, _ = rope_case((4, 4, 64), 2, (32,))
    kc = torch.zeros(3, 5, 4, 64, device="cuda", dtype=BF)
    vc, q = torch.zeros_like(kc), empty(2, 4, 64)
    i32 = lambda *v: torch.tensor(v, device="cuda", dtype=torch.int32)  # noqa: E731
    good, bad, at, s = i32(0, 1), i32(0, 3), i32(4, 0), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for slots in (bad, good, bad):
        with torch.cuda.stream(s):
            torch.cuda._sleep(50_000_000)  # some 25 ms
        op.append(qkv, pos, q, kc, vc, slots, at, stream=s)
        if slots is good:
            op.check()
            continue
        with pytest.raises(J.JnxError) as e:
            op.check()
        assert e.value.code == J.JNX_ERR_DEVICE_BOUNDS


def rope_gradients(qkv, heads, gains, pos, sections, dq, dk, theta=10000.0):
    """Definition's gradients by the chain rule, with bounds."""
    h, hkv, hd = heads
    n = qkv.shape[0]
    x = qkv.to(T.F64).view(n, -1, hd)[:, :h + hkv]
    dn = T.rotate(torch.cat([dq, dk], 1).to(T.F64), T.angles(pos, sections, theta, hd), -1.0)
    if gains[0] is None:
        return dn, T.norm_rope_bound(dn), None, None
    gamma = torch.cat([gains[0].expand(h, hd), gains[1].expand(hkv, hd)]).to(T.F64)
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    e = dn * gamma
    m = (e * x).mean(-1, keepdim=True)
    dx = r * e - x * r ** 3 * m
    # 32-bit arithmetic: 2^-20 of what is subtracted, of the row's sums and of the pair
    # that is turned back
    pair = torch.sqrt(sum(y * y for y in dn.chunk(2, -1))).repeat(1, 1, 2) * gamma.abs()
    slack = 2.0 ** -20 * (r * e.abs() + x.abs() * r ** 3 * (e * x).abs().mean(-1, keepdim=True)
                          + r * pair)
    dg = (dn * x * r)
    return dx, T.U * dx.abs() + slack, dg, dg.abs()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("n", [1, 37, 700])
@pytest.mark.parametrize("norms", [True, False])
def test_norm_rope_backward(heads, n, norms):
    h, hkv, hd = heads
    sections = sections_of(hd, 3)
    op, qkv, pos, gains, _ = rope_case(heads, n, sections, 7, norms=norms)
    g = gen(8)
    dq, dk = normal(g, n, h, hd), normal(g, n, hkv, hd)
    dqkv = torch.full_like(qkv, 3.0)
    dg = [empty(hd, dtype=torch.float32) if norms else None for _ in range(2)]
    op.backward(qkv, pos, dq, dk, dqkv, *dg)
    want, tol, wg, size = rope_gradients(qkv, heads, gains, pos, sections, dq, dk)
    got = dqkv.view(n, -1, hd)
    T.close(got[:, :h + hkv], want, tol, "dx")
    assert (got[:, h + hkv:] == 3).all()
    if norms:
        for a, b, x in ((0, h, dg[0]), (h, h + hkv, dg[1])):
            # 32-bit sums: 2^-20 of the sum of sizes
            T.close(x, wg[:, a:b].sum((0, 1)), 2.0 ** -20 * size[:, a:b].sum((0, 1)) * 4, "dgamma")
    again = torch.full_like(qkv, 3.0)
    dg2 = [None if x is None else torch.empty_like(x) for x in dg]
    op.backward(qkv, pos, dq, dk, again, *dg2)
    assert torch.equal(again, dqkv) and (not norms or torch.equal(dg[0], dg2[0]))


def test_norm_rope_backward_of_one_row_has_no_row_stride():
    op, qkv, pos, gains, _ = rope_case((4, 4, 64), 1, (32,), 9)
    g = gen(30)
    dq, dk = normal(g, 1, 4, 64), normal(g, 1, 4, 64)
    wide = empty(3, 1000)
    wide[1:2, :768] = qkv
    got = []
    for x in (qkv, wide[1:2, :768]):
        d, dg = torch.zeros(1, 768, device="cuda", dtype=BF), [empty(64, dtype=torch.float32) for _ in range(2)]
        op.backward(x, pos, dq, dk, d, *dg)
        got.append([d, *dg])
    for a, b in zip(*got):
        assert torch.equal(a, b)
    two = torch.zeros(2, 768, device="cuda", dtype=BF)
    with pytest.raises(ValueError):
        op.backward(wide[:2, :768], pos.expand(1, 2).contiguous(), dq.expand(2, 4, 64).contiguous(),
                    dk.expand(2, 4, 64).contiguous(), two, *dg)


def test_norm_rope_backward_against_differences():
    """The definition's directional derivative, by central differences in 64 bits."""
    heads, n, sections = (8, 2, 128), 13, (16, 24, 24)
    op, qkv, pos, gains, _ = rope_case(heads, n, sections, 5)
    g = gen(6)
    dq, dk = normal(g, n, 8, 128), normal(g, n, 2, 128)
    dqkv = torch.zeros_like(qkv)
    dg = [empty(128, dtype=torch.float32) for _ in range(2)]
    op.backward(qkv, pos, dq, dk, dqkv, *dg)
    u = torch.randn(n, 12, 128, generator=g, device="cuda", dtype=T.F64)
    ug = [torch.randn(128, generator=g, device="cuda", dtype=T.F64) for _ in range(2)]

    def f(t):
        x = qkv.to(T.F64).view(n, 12, 128) + t * u
        y = [T.norm_rope(x[:, a:b], gains[i].to(T.F64) + t * ug[i], pos, sections, 10000.0, 1e-6)
             for i, (a, b) in enumerate(((0, 8), (8, 10)))]
        return (y[0] * dq.to(T.F64)).sum() + (y[1] * dk.to(T.F64)).sum()

    slope = (f(1e-5) - f(-1e-5)) / 2e-5
    terms = dqkv.to(T.F64).view(n, 12, 128) * u
    mine = terms.sum() + sum((d.to(T.F64) * x).sum() for d, x in zip(dg, ug))
    # independent roundings of bf16: their sizes add in squares
    assert abs(mine - slope) < 6 * 2.0 ** -9 * terms.norm() + 1e-6 * abs(slope)


def test_norm_rope_of_no_tokens():
    op, qkv, pos, _, _ = rope_case((4, 4, 64), 3, (32,))
    z = lambda *s: torch.empty(0, *s, device="cuda", dtype=BF)  # noqa: E731
    op.forward(qkv[:0], pos[:, :0].contiguous(), z(4, 64), z(4, 64))
    dg = [empty(64, dtype=torch.float32) for _ in range(2)]
    op.backward(qkv[:0], pos[:, :0].contiguous(), z(4, 64), z(4, 64), z(768), *dg)
    assert (dg[0] == 0).all() and (dg[1] == 0).all()


# ---------------------------------------------------------------- prompt attention

LENS = {
    "one": ([1], [1], [0]),
    "short": ([5, 1, 130], None, None),
    "edges": ([127, 128, 129, 0, 256, 255, 64, 63], None, None),
    "odd": ([301, 77, 3, 190], None, None),
    "prefix": ([300, 10, 129, 200, 64], None, [260, 10, 0, 131, 1]),
    "continued": ([5, 1, 130, 64, 0], [300, 257, 131, 64, 40], None),
    "continued_prefix": ([40, 3, 200], [300, 257, 200], [280, 257, 77]),
    # more rows than keys: the first rows see nothing unless a prefix shows them keys
    "unseen": ([200, 9, 5, 140], [60, 0, 4, 1], None),
    "unseen_prefix": ([200, 9, 5], [60, 0, 4], [3, 0, 9]),
    "long": ([1111, 700], [1500, 700], [0, 333]),
}


def lens_of(name):
    q, k, p = LENS[name]
    k = q if k is None else k
    return q, k, [0] * len(q) if p is None else p


def attn_inputs(heads, lens, seed=0, std=1.5):
    h, hkv, hd = heads
    g = gen(seed)
    nq, nk = sum(lens[0]), sum(lens[1])
    return (normal(g, nq, h, hd, std=std), normal(g, nk, hkv, hd), normal(g, nk, hkv, hd),
            normal(g, nq, h, hd))


def attn_forward(heads, lens, q, k, v, gradients=False):
    R = _r()
    op = R.PromptAttention(*heads, R.PromptPlan(*lens), gradients=gradients)
    out, lse = empty(*q.shape), empty(q.shape[0], heads[0], dtype=torch.float32)
    op.forward(q, k, v, out, lse)
    op.check()
    return op, out, lse


def lse_close(got, want, std=1.5):
    """32-bit scores and exponentials: 2^-13 of a unit, and 2^-20 of the value."""
    assert torch.equal(got.isinf(), want.isinf()) and not got.isnan().any()
    f = want.isfinite()
    T.close(got[f], want[f], 2.0 ** -12 + 2.0 ** -20 * want[f].abs(), "lse")


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("name", LENS)
def test_prompt_attention(heads, name):
    lens = lens_of(name)
    q, k, v, _ = attn_inputs(heads, lens)
    _, out, lse = attn_forward(heads, lens, q, k, v)
    want = T.attention(q, k, v, lens)
    T.close(out, want["out"], want["out_tol"], "out")
    lse_close(lse, want["lse"])


def attn_gradients(heads, lens, q, k, v, dout):
    op, out, lse = attn_forward(heads, lens, q, k, v, True)
    dq, dk, dv = (empty(*x.shape) for x in (q, k, v))
    op.backward(q, k, v, out, lse, dout, dq, dk, dv)
    op.check()
    return out, lse, dq, dk, dv


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("name", LENS)
def test_prompt_attention_backward(heads, name):
    lens = lens_of(name)
    q, k, v, dout = attn_inputs(heads, lens, 1)
    _, _, dq, dk, dv = attn_gradients(heads, lens, q, k, v, dout)
    want = T.attention(q, k, v, lens, dout)
    for got, n in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        T.close(got, want[n], want[n + "_tol"], n)


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (8, 1, 256)])
def test_prompt_attention_rows_of_one_key_have_no_score_gradient(heads):
    """A softmax over one key does not move: exactly zero, not what rounding leaves."""
    lens = ([1, 1, 2, 1, 70], [1, 3, 1, 1, 70], [0, 0, 0, 1, 0])
    q, k, v, dout = attn_inputs(heads, lens, 11)
    _, _, dq, dk, dv = attn_gradients(heads, lens, q, k, v, dout)
    want = T.attention(q, k, v, lens, dout)
    one = [0, 3, 4, 5]  # the rows that see one key (row 2 sees none): their keys 0, 4, 5
    assert (dq[one] == 0).all() and (dq[2] == 0).all() and (dk[[0, 4, 5]] == 0).all()
    for got, n in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        T.close(got, want[n], want[n + "_tol"], n)


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (8, 1, 256)])
@pytest.mark.parametrize("longest", [2, 3, 9, 33, 400])
def test_prompt_attention_backward_keeps_its_precision_on_short_sequences(heads, longest):
    """dS and the result are each rounded to bf16, 2^-9 at most and 0.0017 on average: 0.0024
    together.  What D would add, taken from rounded outputs, stays below that."""
    lens = ([longest] * 40, [longest] * 40, [0] * 40)
    q, k, v, dout = attn_inputs(heads, lens, 12)
    _, _, dq, dk, _ = attn_gradients(heads, lens, q, k, v, dout)
    want = T.attention(q, k, v, lens, dout)
    for got, n in ((dq, "dq"), (dk, "dk")):
        assert float((got.to(T.F64) - want[n]).norm() / want[n].norm()) < 0.003


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (8, 1, 256)])
def test_prompt_attention_backward_belongs_to_its_own_forward(heads):
    """Several forwards of one plan, then their backwards in another order: each has the bits
    that it has by itself, on an object of its own."""
    R, lens = _r(), ([40] * 9 + [200], [40] * 9 + [200], [0] * 10)
    plan = R.PromptPlan(*lens)
    shared = R.PromptAttention(*heads, plan, gradients=True)

    def forward(op, x):
        out, lse = empty(*x[0].shape), empty(x[0].shape[0], heads[0], dtype=torch.float32)
        op.forward(*x[:3], out, lse)
        return out, lse

    def backward(op, x, out, lse):
        d = [empty(*y.shape) for y in x[:3]]
        op.backward(*x[:3], out, lse, x[3], *d)
        op.check()
        return d

    inputs = [attn_inputs(heads, lens, seed) for seed in (21, 22, 23)]
    alone = []
    for x in inputs:
        op = R.PromptAttention(*heads, plan, gradients=True)
        alone.append(backward(op, x, *forward(op, x)))
    # the last one's forward by an object without gradients, as a frozen copy would run it
    kept = [forward(shared, x) for x in inputs[:2]]
    kept.append(forward(R.PromptAttention(*heads, plan), inputs[2]))
    for i in (0, 2, 1):
        for a, b in zip(alone[i], backward(shared, inputs[i], *kept[i])):
            assert torch.equal(a, b)


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (8, 1, 256), (14, 2, 64), (64, 1, 64)])
@pytest.mark.parametrize("lens", [[12], [40], [64], [5, 17, 33, 64], [9, 70]])
@pytest.mark.parametrize("prefix", [False, True])
def test_prompt_attention_backward_of_few_keys_is_as_close_as_its_roundings(heads, lens, prefix):
    """Rows of up to 64 keys: dq and dk are off by the rounding of dS and their own, 0.0017 of
    the norm each and 0.0024 together: under one and a half times a rounding."""
    q = (lens * 40)[:40]
    lens = (q, q, [x // 2 if prefix else 0 for x in q])
    q, k, v, dout = attn_inputs(heads, lens, 24)
    _, _, dq, dk, _ = attn_gradients(heads, lens, q, k, v, dout)
    want = T.attention(q, k, v, lens, dout)
    for got, n in ((dq, "dq"), (dk, "dk")):
        assert float((got.to(T.F64) - want[n]).norm() / want[n].norm()) < 1.5 * 0.0017


def test_prompt_attention_sharp_scores():
    """Scores of hundreds: a running maximum that rises in every tile, rows that put all
    their weight on one key."""
    heads, lens = (4, 2, 128), ([520], [520], [0])
    q, k, v, dout = attn_inputs(heads, lens, 2, std=30.0)
    k *= torch.linspace(0.2, 6, 520, device="cuda").to(BF)[:, None, None]
    out, lse, dq, dk, dv = attn_gradients(heads, lens, q, k, v, dout)
    want = T.attention(q, k, v, lens, dout)
    # scores reach |q| |k| / sqrt(hd), about 2^11: 32-bit ones are off by 2^-11 of a unit
    # each, and so is the probability
    off = 2.0 ** -10
    T.close(out, want["out"], want["out_tol"] + off * want["out_tol"] / T.U, "out")
    for got, n in ((dv, "dv"),):
        T.close(got, want[n], want[n + "_tol"] * (1 + off / T.U), n)


def test_prompt_attention_backward_of_sharp_scores():
    """The gradients' scores at large maxima: dq and dk of rows whose weight is nearly on one key."""
    heads, lens = (4, 2, 128), ([520], [520], [0])
    q, k, v, dout = attn_inputs(heads, lens, 2, std=30.0)
    k *= torch.linspace(0.2, 6, 520, device="cuda").to(BF)[:, None, None]
    _, _, dq, dk, _ = attn_gradients(heads, lens, q, k, v, dout)
    want, dk_tol = T.attention(q, k, v, lens, dout), torch.zeros(520, 2, 128, device="cuda", dtype=T.F64)
    # 32-bit scores of up to 2^11 are off by 2^-11 of a unit in the forward and in the gradients,
    # the log-sum-exp is rounded by 2^-13 of one and the exponentials by as much: P by 2^-9
    off, see = 2.0 ** -9, T.seen(520, 520, 0, "cuda")
    for h in range(4):
        a, b, c, do = (x.to(T.F64) for x in (q[:, h], k[:, h // 2], v[:, h // 2], dout[:, h]))
        p = torch.softmax((a @ b.T / math.sqrt(128)).masked_fill(~see, -math.inf), -1)
        o = p @ c
        ds = p * (do @ c.T - (do * o).sum(-1, keepdim=True)) / math.sqrt(128)
        # D is of an output whose P and sums were rounded, and whose scores were off
        d_off = (do.abs() * (T.U * o.abs() + (T.U + off) * (p @ c.abs()))).sum(-1, keepdim=True)
        eds = (T.U + off) * ds.abs() + p * d_off / math.sqrt(128)
        T.close(dq[:, h], want["dq"][:, h], T.U * want["dq"][:, h].abs() + eds @ b.abs(), "dq")
        dk_tol[:, h // 2] += eds.T @ a.abs()
    T.close(dk, want["dk"], T.U * want["dk"].abs() + dk_tol, "dk")


@pytest.mark.parametrize("heads,lens", [
    # so many key tiles that each is one item, of several row tiles
    ((32, 32, 64), ([700], [700], [0])), ((32, 32, 128), ([300, 641], [300, 641], [0, 77])),
    ((31, 31, 256), ([620], [620], [50])),
    # more rows than the most parts of a key tile hold at 2,048 each
    ((64, 1, 64), ([2100], [2100], [0])), ((64, 1, 64), ([2500, 9], [130, 9], [0, 0])),
    ((64, 1, 256), ([2100, 30], [300, 30], [129, 0]))])
def test_prompt_attention_backward_at_the_ends_of_its_parts(heads, lens):
    q, k, v, dout = attn_inputs(heads, lens, 27)
    _, _, dq, dk, dv = attn_gradients(heads, lens, q, k, v, dout)
    want = T.attention(q, k, v, lens, dout)
    for got, n in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        T.close(got, want[n], want[n + "_tol"], n)


def test_prompt_attention_other_sequences_hold_anything():
    """NaN and infinities in the neighbours' rows reach no other sequence."""
    heads, lens = (8, 2, 128), ([100, 60, 200], [130, 60, 200], [0, 9, 50])
    q, k, v, dout = attn_inputs(heads, lens, 3)
    clean = attn_gradients(heads, lens, q, k, v, dout)
    for x, cu in ((q, 0), (k, 1), (v, 1), (dout, 0)):
        a = lens[cu][0]
        x[a:a + 60] = float("nan")
        x[a:a + 60:7] = float("inf")
    dirty = attn_gradients(heads, lens, q, k, v, dout)
    for c, d, cu in zip(clean, dirty, (0, 0, 0, 1, 1)):
        a = lens[cu][0]
        assert torch.equal(c[:a], d[:a]) and torch.equal(c[a + 60:], d[a + 60:])


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (8, 1, 256)])
def test_prompt_attention_bits_do_not_depend_on_the_pack(heads):
    lens = ([300, 77, 513, 129], [300, 90, 513, 200], [0, 20, 400, 129])
    q, k, v, dout = attn_inputs(heads, lens, 4)
    whole = attn_gradients(heads, lens, q, k, v, dout)
    a, b = [0], [0]
    for x, y in zip(*lens[:2]):
        a.append(a[-1] + x)
        b.append(b[-1] + y)
    for i in (1, 2):
        R, K = slice(a[i], a[i + 1]), slice(b[i], b[i + 1])
        alone = attn_gradients(heads, tuple([x[i]] for x in lens), q[R], k[K], v[K], dout[R])
        for w, x, s in zip(whole, alone, (R, R, R, K, K)):
            assert torch.equal(w[s], x)


def test_prompt_attention_strides():
    """Heads out of the fused projection's rows, head-major outputs, dq/dk/dv into the
    projection's gradient."""
    heads, lens = (8, 2, 128), ([70, 200], [70, 200], [0, 100])
    g = gen(5)
    qkv = normal(g, 270, 12, 128)
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    dout = normal(g, 8, 270, 128).transpose(0, 1)
    R = _r()
    op = R.PromptAttention(*heads, R.PromptPlan(*lens), gradients=True)
    out, lse = empty(8, 270, 128).transpose(0, 1), empty(270, 8, dtype=torch.float32)
    op.forward(q, k, v, out, lse)
    d = empty(270, 12, 128)
    op.backward(q, k, v, out, lse, dout, d[:, :8], d[:, 8:10], d[:, 10:])
    op.check()
    want = T.attention(q, k, v, lens, dout)
    T.close(out, want["out"], want["out_tol"], "out")
    for got, n in ((d[:, :8], "dq"), (d[:, 8:10], "dk"), (d[:, 10:], "dv")):
        T.close(got, want[n], want[n + "_tol"], n)


@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 1, 256)])
def test_prompt_attention_leaves_out_and_reports_what_its_list_does_not_name(heads):
    """Entries of no sequence, row, key or part, and sequences beyond the packed rows: left out
    and reported, the others as ever."""
    from paper_2607_16074_gb300 import jnx as J
    R, lens = _r(), ([300, 700, 40], [300, 700, 40], [0, 100, 0])
    q, k, v, dout = attn_inputs(heads, lens, 26)
    clean = attn_gradients(heads, lens, q, k, v, dout)
    plan = R.PromptPlan(*lens)
    op = R.PromptAttention(*heads, plan, gradients=True)
    out, lse, *d = (torch.full_like(x, 7.0) for x in clean)

    def call():
        op.forward(q, k, v, out, lse)
        op.backward(q, k, v, out, lse, dout, *d)
        with pytest.raises(J.JnxError) as e:
            op.check()
        assert e.value.code == J.JNX_ERR_DEVICE_BOUNDS

    items, own = op.items, op.items.clone()
    s = op.struct
    first = (0, s.n_forward, s.n_forward + s.n_keys)
    last = (s.n_forward, s.n_forward + s.n_keys, s.n_forward + s.n_keys + s.n_queries)
    # one entry of each pass at a time: (sequence, row or key and part)
    for bad in ((3, 0), (-1, 0), (2 ** 31 - 1, 0), (1, 2 ** 31 - 1), (1, -1), (1, -128), (0, 384),
                (2, 127), (1, 704)):
        for a, b in zip(first, last):
            items.copy_(own)
            items[(a + b) // 2] = torch.tensor(bad, device="cuda", dtype=torch.int32)
            call()
    items.copy_(own)
    # the middle sequence beyond the packed rows, or its keys: the others have their results
    for x in (0, 1):
        device, host = plan.d[x], plan.h[x]
        for bad in (-5, 1041, 2 ** 31 - 1):
            device[2] = bad
            for y in (out, lse, *d):
                y.fill_(7.0)
            call()
            device[2] = int(host[2])
            if x:
                continue
            assert torch.equal(out[:300], clean[0][:300]) and torch.equal(d[1][:300], clean[3][:300])
            assert (d[1][300:1000] == 7).all() and (d[0][300:] == 7).all()
    op.forward(q, k, v, out, lse)
    op.backward(q, k, v, out, lse, dout, *d)
    op.check()
    for a, b in zip(clean, (out, lse, *d)):
        assert torch.equal(a, b)


def test_prompt_attention_backward_against_differences():
    heads, lens = (8, 2, 64), ([90, 33], [140, 33], [0, 20])
    q, k, v, dout = attn_inputs(heads, lens, 6)
    _, _, dq, dk, dv = attn_gradients(heads, lens, q, k, v, dout)
    g = gen(7)
    u = [torch.randn(x.shape, generator=g, device="cuda", dtype=T.F64) for x in (q, k, v)]

    def f(t):
        a, b, c = (x.to(T.F64) + t * y for x, y in zip((q, k, v), u))
        return (T.attention(a, b, c, lens)["out"] * dout.to(T.F64)).sum()

    slope = (f(1e-5) - f(-1e-5)) / 2e-5
    terms = [d.to(T.F64) * y for d, y in zip((dq, dk, dv), u)]
    mine = sum(t.sum() for t in terms)
    # independent roundings of P, dS, D and the results
    assert abs(mine - slope) < 6 * 2.0 ** -8 * math.sqrt(sum(float(t.norm()) ** 2 for t in terms))


def test_prompt_attention_on_another_stream_and_in_a_graph():
    heads, lens = (8, 1, 256), ([300, 40], [300, 40], [256, 0])
    q, k, v, _ = attn_inputs(heads, lens, 8)
    op, want, _ = attn_forward(heads, lens, q, k, v)
    out, s = empty(*q.shape), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    op.forward(q, k, v, out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    out2 = empty(*q.shape)
    with torch.cuda.graph(graph):
        op.forward(q, k, v, out2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out2, want)


# ---------------------------------------------------------------- decode

def decode(heads, n, room, seed=0, kc=None, vc=None, slots=None):
    h, hkv, hd = heads
    g = gen(seed)
    b = len(n)
    slots = slots or b + 3
    kc = normal(g, slots, room, hkv, hd) if kc is None else kc
    vc = normal(g, slots, room, hkv, hd) if vc is None else vc
    q = normal(g, b, h, hd, std=1.5)
    slot = torch.randperm(slots, generator=g, device="cuda")[:b].to(torch.int32)
    op, out = _r().DecodeAttention(h, hkv, hd, max_batch=b), empty(b, h, hd)
    op.forward(q, kc, vc, slot, torch.tensor(n, device="cuda", dtype=torch.int32), out)
    op.check()
    return q, kc, vc, slot, out


def decode_want(q, kc, vc, slot, n):
    keys = [kc[int(s), :x] for s, x in zip(slot, n)]
    vals = [vc[int(s), :x] for s, x in zip(slot, n)]
    return T.attention(q, torch.cat(keys), torch.cat(vals), ([1] * len(n), list(n), [0] * len(n)))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("n", [(1,), (0, 1, 2, 63, 64, 65), (700, 0, 129, 1024, 511, 33),
                               (2500, 3000, 17)])
def test_decode_attention(heads, n):
    q, kc, vc, slot, out = decode(heads, n, max(max(n), 1))
    want = decode_want(q, kc, vc, slot, n)
    T.close(out, want["out"], want["out_tol"], "out")


def test_decode_attention_long_single():
    q, kc, vc, slot, out = decode((8, 1, 256), (60001,), 60013, slots=1)
    want = decode_want(q, kc, vc, slot, (60001,))
    T.close(out, want["out"], want["out_tol"], "out")


@pytest.mark.parametrize("shape", [(4, 300, 1, 256), (1, 70, 1, 64), (1, 129, 2, 128), (5, 1, 1, 64)])
def test_caches_agree_though_axes_of_length_one_differ_in_stride(shape):
    """Head-major keys beside token-major values: with one key head they lie alike."""
    slots, room, hkv, hd = shape
    g, heads = gen(29), (4 * hkv, hkv, hd)
    kc = normal(g, slots, hkv, room, hd).transpose(1, 2)
    vc = normal(g, slots, room, hkv, hd)
    i32 = lambda *v: torch.tensor(v, device="cuda", dtype=torch.int32)  # noqa: E731
    q, out = normal(g, 1, *heads[::2]), empty(1, *heads[::2])
    op = _r().DecodeAttention(*heads, max_batch=1)
    if hkv > 1:
        with pytest.raises(ValueError):
            op.forward(q, kc, vc, i32(0), i32(room), out)
        return
    op.forward(q, kc, vc, i32(slots - 1), i32(room), out)
    op.check()
    want = T.attention(q, kc[-1], vc[-1], ([1], [room], [0]))
    T.close(out, want["out"], want["out_tol"], "out")


def test_decode_attention_reads_nothing_beyond_the_length():
    """What lies behind a length, or in other slots, may be anything."""
    heads, n = (8, 2, 128), (100, 0, 65, 333)
    q, kc, vc, slot, out = decode(heads, n, 400)
    for c in (kc, vc):
        keep = torch.zeros(c.shape[:2], dtype=torch.bool, device="cuda")
        for s, x in zip(slot, n):
            keep[int(s), :x] = True
        c[~keep] = float("nan")
    again = decode(heads, n, 400, kc=kc, vc=vc)[4]
    # the same seed draws other queries once the caches are given
    want = decode_want(*decode(heads, n, 400, kc=kc, vc=vc)[:4], n)
    T.close(again, want["out"], want["out_tol"], "out")


def test_decode_attention_reports_what_lies_outside():
    from paper_2607_16074_gb300 import jnx as J
    g = gen(1)
    kc, vc, q = normal(g, 2, 50, 4, 64), normal(g, 2, 50, 4, 64), normal(g, 4, 4, 64)
    i32 = lambda *v: torch.tensor(v, device="cuda", dtype=torch.int32)  # noqa: E731
    op, out = _r().DecodeAttention(4, 4, 64, max_batch=4), empty(4, 4, 64)
    op.forward(q, kc, vc, i32(2, 1, 0, -7), i32(3, 51, 50, 0), out)
    with pytest.raises(J.JnxError) as e:
        op.check()
    assert e.value.code == J.JNX_ERR_DEVICE_BOUNDS
    assert (out[[0, 1, 3]] == 0).all()
    want = T.attention(q[2:3], kc[0], vc[0], ([1], [50], [0]))
    T.close(out[2:3], want["out"], want["out_tol"])


def test_decode_attention_offsets_beyond_32_bits():
    """A cache of over 2^32 elements, the sequence in its last slot."""
    h, hkv, hd = 8, 8, 128
    slots, room = 1030, 4097
    kc = torch.empty(slots, room, hkv, hd, device="cuda", dtype=BF)
    vc = torch.empty_like(kc)
    assert kc.numel() > 2 ** 32
    g = gen(9)
    kc[-1], vc[-1] = normal(g, room, hkv, hd), normal(g, room, hkv, hd)
    q, out = normal(g, 1, h, hd), empty(1, h, hd)
    op = _r().DecodeAttention(h, hkv, hd, max_batch=1)
    one = lambda x: torch.tensor([x], device="cuda", dtype=torch.int32)  # noqa: E731
    op.forward(q, kc, vc, one(slots - 1), one(room), out)
    want = T.attention(q, kc[-1], vc[-1], ([1], [room], [0]))
    T.close(out, want["out"], want["out_tol"])


def test_decode_attention_bits_do_not_depend_on_the_batch():
    heads, n = (8, 2, 128), (900, 30, 0, 2222, 513)
    q, kc, vc, slot, out = decode(heads, n, 2300)
    for i in (0, 3, 4):
        op, alone = _r().DecodeAttention(*heads, max_batch=7), empty(1, 8, 128)
        op.forward(q[i:i + 1], kc, vc, slot[i:i + 1],
                   torch.tensor([n[i]], device="cuda", dtype=torch.int32), alone)
        assert torch.equal(alone[0], out[i])


@pytest.mark.parametrize("heads", [(64, 8, 64), (64, 8, 128), (64, 8, 256)])
def test_decode_attention_bits_do_not_depend_on_how_many_heads_are_joined(heads):
    """Sequences of 1 to 16 runs: among 1,920 heads, and each by itself."""
    h, hkv, hd = heads
    g = gen(12)
    kc, vc = normal(g, 3, 1024, hkv, hd), normal(g, 3, 1024, hkv, hd)
    q = normal(g, 30, h, hd)
    i32 = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    n = [1024, 64, 65, 700, 129, 0, 960, 1, 300, 513] * 3
    op, out, alone = _r().DecodeAttention(*heads, max_batch=30), empty(30, h, hd), empty(1, h, hd)
    op.forward(q, kc, vc, i32([i % 3 for i in range(30)]), i32(n), out)
    for i in range(30):
        op.forward(q[i:i + 1], kc, vc, i32([i % 3]), i32(n[i:i + 1]), alone)
        assert torch.equal(alone[0], out[i])
    op.check()
    want = decode_want(q[:6], kc, vc, i32([i % 3 for i in range(6)]), n[:6])
    T.close(out[:6], want["out"], want["out_tol"])


def test_decode_attention_batches_of_all_sizes_share_a_workspace():
    """Large and small batches in turn on one object: what a call leaves behind is what the
    next expects."""
    heads, n = (8, 2, 128), [900, 30, 0, 2222, 513, 1300] * 20
    h, hkv, hd = heads
    g = gen(11)
    kc, vc = normal(g, 6, 2300, hkv, hd), normal(g, 6, 2300, hkv, hd)
    q = normal(g, len(n), h, hd)
    slot = torch.arange(len(n), device="cuda", dtype=torch.int32) % 6
    lens = torch.tensor(n, device="cuda", dtype=torch.int32)
    op = _r().DecodeAttention(*heads, max_batch=len(n))
    outs = []
    for b in (120, 1, 120, 5, 33, 120):
        out = empty(b, h, hd)
        op.forward(q[:b], kc, vc, slot[:b], lens[:b], out)
        outs.append(out)
    op.check()
    for out in outs:
        assert torch.equal(out, outs[0][:out.shape[0]])
    want = decode_want(q[:6], kc, vc, slot[:6], n[:6])
    T.close(outs[0][:6], want["out"], want["out_tol"])


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (8, 1, 256)])
@pytest.mark.parametrize("batch", [1024, 1025, 2049])
def test_decode_attention_of_more_sequences_than_a_launch_takes(heads, batch):
    """Sequences of one run and of several on both sides of a launch's last one, each with the bits
    that it has by itself."""
    h, hkv, hd = heads
    g = gen(28)
    kc, vc = normal(g, 40, 700, hkv, hd), normal(g, 40, 700, hkv, hd)
    q = normal(g, batch, h, hd)
    i32 = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    n = [(3, 64, 0, 700, 65, 1, 129, 33, 512, 700)[i % 10] for i in range(batch)]
    slot = [i * 7 % 40 for i in range(batch)]
    op, out, alone = _r().DecodeAttention(*heads, max_batch=batch), empty(batch, h, hd), empty(1, h, hd)
    op.forward(q, kc, vc, i32(slot), i32(n), out)
    some = sorted({i for at in (0, 1024, 2048, batch) for i in range(at - 12, at + 12) if 0 <= i < batch})
    for i in some:
        op.forward(q[i:i + 1], kc, vc, i32([slot[i]]), i32([n[i]]), alone)
        assert torch.equal(alone[0], out[i]), i
    op.check()
    want = decode_want(q[some], kc, vc, i32([slot[i] for i in some]), [n[i] for i in some])
    T.close(out[some], want["out"], want["out_tol"], "out")
    assert torch.isfinite(out).all()


def test_decode_matches_the_prompt():
    """A sequence's last row alone against its cache, and inside its prompt."""
    heads, n = (8, 2, 128), 777
    q, k, v, _ = attn_inputs(heads, ([n], [n], [0]), 10)
    _, out, _ = attn_forward(heads, ([n], [n], [0]), q, k, v)
    op, one = _r().DecodeAttention(*heads, max_batch=1), empty(1, 8, 128)
    i32 = lambda x: torch.tensor([x], device="cuda", dtype=torch.int32)  # noqa: E731
    op.forward(q[-1:], k[None], v[None], i32(0), i32(n), one)
    want = T.attention(q[-1:], k, v, ([1], [n], [0]))
    T.close(one, want["out"], want["out_tol"])
    T.close(out[-1:], want["out"], want["out_tol"])


def test_objects_dropped_behind_a_call_on_another_stream():
    """A call that still waits for its turn keeps its object's workspace and work list, though
    the object is gone and others ask for memory."""
    R, heads, lens = _r(), (8, 2, 128), ([300, 70] * 4, [300, 70] * 4, [20, 0] * 4)
    h, hkv, hd = heads
    q, k, v, dout = attn_inputs(heads, lens, 25)
    want = attn_gradients(heads, lens, q, k, v, dout)
    n = [900, 30, 0, 2222, 513]
    q1, kc, vc, slot, want1 = decode(heads, n, 2300)
    n = torch.tensor(n, device="cuda", dtype=torch.int32)
    s, junk = torch.cuda.Stream(), []
    got, got1 = [torch.empty_like(x) for x in want], torch.empty_like(want1)
    s.wait_stream(torch.cuda.current_stream())

    def call():
        prompts = R.PromptAttention(*heads, R.PromptPlan(*lens), gradients=True)
        one = R.DecodeAttention(*heads, max_batch=5)
        with torch.cuda.stream(s):
            torch.cuda._sleep(50_000_000)  # some 25 ms
        prompts.forward(q, k, v, got[0], got[1], stream=s)
        prompts.backward(q, k, v, got[0], got[1], dout, *got[2:], stream=s)
        one.forward(q1, kc, vc, slot, n, got1, stream=s)
        return [x.numel() * x.element_size() for op in (prompts, one) for x in op._held]

    for size in call() * 3:
        junk.append(torch.full((size,), 255, device="cuda", dtype=torch.uint8))
    torch.cuda.synchronize()
    for a, b in zip([*want, want1], [*got, got1]):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- vocabulary loss

def vocab_case(n, vocab, d, seed=0, std=0.05, ignored=0.2):
    g = gen(seed)
    h, w = normal(g, n, d), normal(g, vocab, d, std=std)
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    t[torch.rand(n, generator=g, device="cuda") < ignored] = -1
    rw = torch.rand(n, generator=g, device="cuda") / max(n, 1)
    return h, w, t, rw


VOCABS = [(1, 1, 8), (1, 257, 64), (3, 1000, 256), (130, 511, 72), (257, 3001, 1000),
          (333, 256, 128), (64, 32000, 256), (5, 4099, 2048)]


@pytest.mark.parametrize("n,vocab,d", VOCABS)
def test_vocab_loss(n, vocab, d):
    h, w, t, _ = vocab_case(n, vocab, d)
    loss = empty(n, dtype=torch.float32)
    op = _r().VocabLoss(w, max_rows=n, gradients=False)
    op.loss(h, t, loss)
    op.check()
    want = T.vocab(h, w, t)
    T.close(loss, want["loss"], want["loss_tol"], "loss")
    assert (loss[t < 0] == 0).all()


def vocab_train(h, w, t, rw, piece_rows=0, frozen=False):
    n = h.shape[0]
    loss, dh, dw = empty(n, dtype=torch.float32), empty(*h.shape), empty(*w.shape)
    op = _r().VocabLoss(w, max_rows=n, piece_rows=piece_rows)
    op.train(h, t, rw, loss, dh, None if frozen else dw)
    op.check()
    return loss, dh, dw


@pytest.mark.parametrize("n,vocab,d", VOCABS)
def test_vocab_loss_train(n, vocab, d):
    h, w, t, rw = vocab_case(n, vocab, d, 1)
    loss, dh, dw = vocab_train(h, w, t, rw)
    want = T.vocab(h, w, t, rw)
    T.close(loss, want["loss"], want["loss_tol"], "loss")
    T.close(dh, want["dh"], want["dh_tol"], "dh")
    T.close(dw, want["dw"], want["dw_tol"], "dw")
    assert (dh[t < 0] == 0).all()


@pytest.mark.parametrize("piece", [1, 100, 256, 299, 300])
def test_vocab_loss_train_in_pieces(piece):
    h, w, t, rw = vocab_case(300, 777, 136, 2)
    loss, dh, dw = vocab_train(h, w, t, rw, piece_rows=piece)
    want = T.vocab(h, w, t, rw)
    T.close(loss, want["loss"], want["loss_tol"], "loss")
    T.close(dh, want["dh"], want["dh_tol"], "dh")
    T.close(dw, want["dw"], want["dw_tol"], "dw")


@pytest.mark.parametrize("n", [8191, 8192, 8193, 20001])
def test_vocab_loss_train_of_many_rows(n):
    """Calls on either side of the length up to which rows are placed by counting."""
    h, w, t, rw = vocab_case(n, 260, 64, 13)
    loss, dh, dw = vocab_train(h, w, t, rw)
    want = T.vocab(h, w, t, rw)
    T.close(loss, want["loss"], want["loss_tol"], "loss")
    T.close(dh, want["dh"], want["dh_tol"], "dh")
    T.close(dw, want["dw"], want["dw_tol"], "dw")
    assert (dh[t < 0] == 0).all() and (loss[t < 0] == 0).all()


@pytest.mark.parametrize("most,n", [(168, 100), (256, 161), (700, 300)])
def test_vocab_loss_train_of_fewer_rows_than_it_was_made_for(most, n):
    """Fewer rows may take dh's sum over the vocabulary in more parts."""
    h, w, t, rw = vocab_case(n, 8000, 1024, 6)
    loss, dh, dw = vocab_train(h, w, t, rw)
    loss2, dh2, dw2 = empty(n, dtype=torch.float32), empty(*h.shape), empty(*w.shape)
    op = _r().VocabLoss(w, max_rows=most)
    op.train(h, t, rw, loss2, dh2, dw2)
    op.check()
    assert torch.equal(loss, loss2) and torch.equal(dh, dh2) and torch.equal(dw, dw2)


def test_vocab_loss_frozen_vocabulary():
    h, w, t, rw = vocab_case(150, 900, 128, 3)
    loss, dh, dw = vocab_train(h, w, t, rw)
    loss2, dh2, dw2 = vocab_train(h, w, t, rw, frozen=True)
    assert torch.equal(loss, loss2) and torch.equal(dh, dh2) and dw2.isnan().all()


def test_vocab_loss_all_rows_ignored_and_none():
    h, w, t, rw = vocab_case(40, 300, 64, 4, ignored=2.0)
    loss, dh, dw = vocab_train(h, w, t, rw)
    assert (loss == 0).all() and (dh == 0).all() and (dw == 0).all()
    op, dw = _r().VocabLoss(w, max_rows=1), empty(*w.shape)
    op.train(h[:0], t[:0], rw[:0], loss[:0], dh[:0], dw)
    assert (dw == 0).all()


def test_vocab_loss_of_far_apart_logits():
    """Logits hundreds apart: the target's probability is one, or vanishes."""
    h, w, t, rw = vocab_case(70, 600, 64, 5, std=8.0)
    loss, dh, dw = vocab_train(h, w, t, rw)
    want = T.vocab(h, w, t, rw)
    T.close(loss, want["loss"], want["loss_tol"], "loss")
    # a probability is off by as much as its logit
    grow = 1 + float(want["loss_tol"].max()) / T.U
    T.close(dh, want["dh"], want["dh_tol"] * grow + 1e-6, "dh")
    T.close(dw, want["dw"], want["dw_tol"] * grow + 1e-6, "dw")


@pytest.mark.parametrize("top", [0.0, 20.0, 60.0, 100.0])
@pytest.mark.parametrize("other", [1e-8, 1e-6, 1e-4, 0.3, 30.0])
def test_vocab_loss_of_sure_rows_keeps_its_digits(top, other):
    """A target at or near the maximum and little mass beside it: loss and gradients are
    right to their own size, not to the logits'."""
    n, vocab, d = 24, 1000, 64
    g = gen(14)
    h = torch.zeros(n, d, device="cuda", dtype=BF)
    h[torch.arange(n), torch.arange(n)] = 1  # row i's logits are the vocabulary's column i, exactly
    w = torch.zeros(vocab, d, device="cuda", dtype=BF)
    w[:, :n] = (top + math.log(other / vocab) + 0.3 * torch.randn(vocab, n, generator=g, device="cuda")).to(BF)
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    w[t.long(), torch.arange(n)] = top
    loss, dh, dw = vocab_train(h, w, t, torch.ones(n, device="cuda"))
    x = w[:, :n].T.to(T.F64)
    mass = torch.exp(x - top)
    mass[torch.arange(n), t.long()] = 0
    want = torch.log1p(mass.sum(-1))
    # the maximum times log2(e), 2^-17 of a unit at 100, a block's 128 terms added in turn,
    # 2^-17 of their sum, and the exponentials: under 2^-15 in all
    T.close(loss, want, 2.0 ** -14 * want, "loss")
    r = T.vocab(h, w, t, torch.ones(n, device="cuda"))
    T.close(dh, r["dh"], r["dh_tol"], "dh")
    T.close(dw, r["dw"], r["dw_tol"], "dw")
    only, rows = torch.empty_like(loss), torch.arange(n)
    _r().VocabLoss(w, max_rows=n, gradients=False).loss(h, t, only)
    assert torch.equal(only, loss)
    # the target's own entry, which the vocabulary's gradient shows by itself: two roundings
    share = mass.sum(-1) / (1 + mass.sum(-1))
    T.close(-dw[t.long(), rows], share, 2 * T.U * share, "target")


def test_vocab_loss_ignored_rows_hold_anything():
    h, w, t, rw = vocab_case(200, 500, 128, 6)
    clean = vocab_train(h, w, t, rw)
    h[t < 0] = float("nan")
    rw[t < 0] = float("inf")
    dirty = vocab_train(h, w, t, rw)
    for c, x in zip(clean, dirty):
        assert torch.equal(c, x)


def test_vocab_loss_reports_targets_outside():
    from paper_2607_16074_gb300 import jnx as J
    h, w, t, rw = vocab_case(9, 100, 64, 7, ignored=0.0)
    t[4] = 100
    loss, dh, dw = empty(9, dtype=torch.float32), empty(9, 64), empty(100, 64)
    op = _r().VocabLoss(w, max_rows=9)
    op.train(h, t, rw, loss, dh, dw)
    with pytest.raises(J.JnxError) as e:
        op.check()
    assert e.value.code == J.JNX_ERR_DEVICE_BOUNDS
    want = T.vocab(h, w, t, rw)
    T.close(loss, want["loss"], want["loss_tol"])
    T.close(dw, want["dw"], want["dw_tol"])


def test_vocab_loss_strides():
    h, w, t, rw = vocab_case(120, 310, 64, 8)
    hw, ww = empty(120, 200), empty(310, 72)
    hw[:, 8:72], ww[:, :64] = h, w
    loss, dh, dw = empty(120, dtype=torch.float32), empty(120, 80), empty(310, 64)
    op = _r().VocabLoss(ww[:, :64], max_rows=120)
    op.train(hw[:, 8:72], t, rw, loss, dh[:, :64], dw)
    want = T.vocab(h, w, t, rw)
    T.close(dh[:, :64], want["dh"], want["dh_tol"])
    T.close(dw, want["dw"], want["dw_tol"])
    assert dh[:, 64:].isnan().all()


def test_vocab_loss_against_differences():
    h, w, t, rw = vocab_case(60, 400, 64, 9)
    _, dh, dw = vocab_train(h, w, t, rw)
    g = gen(10)
    uh, uw = (torch.randn(x.shape, generator=g, device="cuda", dtype=T.F64) for x in (h, w))

    def f(e):
        return (T.vocab(h.to(T.F64) + e * uh, w.to(T.F64) + e * uw, t)["loss"] * rw.to(T.F64)).sum()

    slope = (f(1e-6) - f(-1e-6)) / 2e-6
    terms = [dh.to(T.F64) * uh, dw.to(T.F64) * uw]
    mine = sum(x.sum() for x in terms)
    assert abs(mine - slope) < 6 * 2.0 ** -8 * math.sqrt(sum(float(x.norm()) ** 2 for x in terms))


# ---------------------------------------------------------------- workspaces

def test_what_a_workspace_held_before_does_not_matter():
    """All bits set (NaN, huge counts) or none: every call has the same results."""
    R, heads = _r(), (8, 2, 128)
    lens = ([300, 9, 0, 900, 64], [300, 70, 5, 900, 64], [20, 0, 0, 500, 3])
    q, k, v, dout = attn_inputs(heads, lens, 31)
    rope, qkv, pos, _, _ = rope_case(heads, 300, (64,), 32)
    h, w, t, rw = vocab_case(300, 4000, 1024, 33)
    n = [900, 30, 0, 2222, 513]
    q1, kc, vc, slot, _ = decode(heads, n, 2300)
    n = torch.tensor(n, device="cuda", dtype=torch.int32)
    prompts = R.PromptAttention(*heads, R.PromptPlan(*lens), gradients=True)
    one, words = R.DecodeAttention(*heads, max_batch=9), R.VocabLoss(w, max_rows=400)
    seen = []
    for fill in (255, 0):
        for op in (rope, prompts, one, words):
            op.ws.fill_(fill)
        out, lse = empty(*q.shape), empty(q.shape[0], 8, dtype=torch.float32)
        d = [empty(*x.shape) for x in (q, k, v)]
        prompts.forward(q, k, v, out, lse)
        prompts.backward(q, k, v, out, lse, dout, *d)
        o1, loss, dh, dw = empty(*q1.shape), empty(300, dtype=torch.float32), empty(*h.shape), empty(*w.shape)
        one.forward(q1, kc, vc, slot, n, o1)
        words.train(h, t, rw, loss, dh, dw)
        dqkv, dg = torch.zeros_like(qkv), [empty(128, dtype=torch.float32) for _ in range(2)]
        rope.backward(qkv, pos, q[:300], k[:300], dqkv, *dg)
        for op in (rope, prompts, one, words):
            op.check()
        seen.append([out, lse, *d, o1, loss, dh, dw, dqkv, *dg])
    for a, b in zip(*seen):
        assert torch.equal(a, b) and not a.isnan().any()
