"""What calls of the drafted tokens' operators may hold beside the ordinary: teachers' entries
that weigh nothing, students at their teacher, products with few terms, probabilities that are
none, layouts whose strides run backwards, sequences that share rows, caches without pages."""
import pytest
import torch

from tests import draft_ops_ref as D
from tests import text_ops_ref as T
from tests.test_gpu_draft_ops import (BF, F32, I32, Trees, _r, _reports, by_hand, check_distill, distill_case, empty,
                                      gen, ints, normal, place, run_verify, verify_case)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- distillation

@pytest.mark.parametrize("far", [-90.0, -104.0, -120.0, -1e4, -1e9, -1e30])
def test_distill_words_given_twice_far_below_the_top(far):
    """Rows filled up with one word, as a padded batch has them: all of its entries together
    weigh nothing, or almost nothing, and the loss is that of the others."""
    h, w, ids, t, rw = distill_case(60, 64, 300, 8, seed=3)
    ids[:, 5:], t[:, 5:] = 0, far
    ids[10:20, 2] = 0  # the word of the filling is one of the row's own as well
    ids[20:30, 4], t[20:30, 4] = 299, far - 1.0  # entries by themselves that weigh nothing
    ids[30:40, 1:], t[30:40, 1:] = 17, far
    loss, *_ = check_distill(h, w, ids, t, rw)
    assert loss.isfinite().all()


@pytest.mark.parametrize("tau", [0.5, 0.25])
def test_distill_logits_beyond_range_over_the_temperature(tau):
    """A logit whose quotient by the temperature is -inf in 32 bits is no entry."""
    h, w, ids, t, rw = distill_case(40, 64, 300, 6, seed=4)
    t[:, 4] = -3.0e38
    t[3::5] = -3.0e38
    t[7] = -3.4e38
    t[11, 1:], t[11, 0] = -2.0e38 * tau, 1.6e38 * tau  # (their difference is beyond range)
    want = torch.where(t == t.clamp_min(-1e30), t, -float("inf"))
    op = _r().VocabDistill(w, 40, 6, tau)
    loss, again, dh, dw = empty(40, dtype=F32), empty(40, dtype=F32), empty(40, 64), empty(300, 64)
    op.loss(h, ids, t, loss)
    op.train(h, ids, t, rw, again, dh, dw)
    op.check()
    r = D.distill(h, w, ids, want, tau, rw)
    T.close(loss, r["loss"], r["loss_tol"], "loss")
    T.close(again, r["loss"], r["loss_tol"], "loss of the step")
    T.close(dh, r["dh"], r["dh_tol"], "dh")
    T.close(dw, r["dw"], r["dw_tol"], "dw")
    assert (loss[3::5] == 0).all() and not dh[3::5].any()


@pytest.mark.parametrize("k", [2, 8])
def test_distill_near_its_teacher_no_loss_is_below_zero(k):
    """A vocabulary of the entries alone, logits exact: hidden rows of a single one.  The
    teacher's are theirs plus 1e-7 to 1.  d = log P - log T is off by under 2^-18: of each of its
    sides, of logits up to 8, the difference to the maximum and that to the logarithm are rounded
    at up to 16 (2^-21 each), the logarithm off by 2^-22 and its sum's terms by as much.  A term
    moves by T (e^d - 1) = P - T of that, and by half its square; its own arithmetic and T's are
    under 2^-19 of it."""
    n, d = 4096, 64
    g = gen(k)
    w = empty(k, d)
    w[:] = 0
    w[:, :n // 64] = normal(g, k, n // 64, std=1.5).clamp(-5, 5)
    h = torch.zeros(n, d, device="cuda", dtype=BF)
    h[torch.arange(n, device="cuda"), torch.arange(n, device="cuda") % 64] = 1
    x = h.float() @ w.float().T
    scale = 10.0 ** (torch.rand(n, 1, generator=g, device="cuda") * 7 - 7)
    t = x + scale * torch.randn(n, k, generator=g, device="cuda").clamp(-3, 3)
    ids = torch.arange(k, device="cuda", dtype=I32).expand(n, k).contiguous()
    op, loss = _r().VocabDistill(w, n, k, gradients=False), empty(n, dtype=F32)
    op.loss(h, ids, t, loss)
    op.check()
    logp, logt = torch.log_softmax(x.double(), -1), torch.log_softmax(t.double(), -1)
    want = (logt.exp() * (logt - logp)).sum(-1)
    off = (logt.exp() - logp.exp()).abs().sum(-1)
    assert (loss >= 0).all(), int((loss < 0).sum())
    T.close(loss, want, 2.0 ** -18 * off + 2.0 ** -36 + 2.0 ** -19 * want, "loss")


@pytest.mark.parametrize("d", [64, 1000, 8192, 16_384])
@pytest.mark.parametrize("terms", [1, 2])
def test_distill_few_terms_are_exact_whatever_the_width(d, terms):
    """Hidden rows with one or two values that are not zero, powers of two, far apart: products
    and sums of them are exact, so the width is in no bound.  A logarithm of a probability is
    then off by the rounding of logits' differences (2^-22 of them, twice) and by the
    exponentials and their sums (2^-19)."""
    n, v, k = 96, 600, 12
    _, _, ids, t, rw = distill_case(n, 8, v, k, seed=d)
    g = gen(d)
    w = (normal(g, v, d).float() * 16).round().clamp(-64, 64).to(BF)  # whole numbers
    h = torch.zeros(n, d, device="cuda", dtype=BF)
    at = torch.randint(0, d // 2, (n,), generator=g, device="cuda")
    h[torch.arange(n, device="cuda"), at] = 1
    if terms == 2:
        h[torch.arange(n, device="cuda"), d - 1 - at] = -0.5
    op, loss = _r().VocabDistill(w, n, k, 0.5, gradients=False), empty(n, dtype=F32)
    op.loss(h, ids, t, loss)
    op.check()
    want = D.distill(h, w, ids, t, 0.5)["loss"]
    x = h.double() @ w.double().T / 0.5
    logt = torch.log_softmax(t.double() / 0.5, -1)
    span = x.amax(-1) - x.amin(-1) - logt.amin(-1)
    # (the gradient's size, P - T, is two at most)
    err = 2.0 ** -21 * span + 2.0 ** -19
    T.close(loss, want, 2 * err + err * err + 2.0 ** -20 * want, "loss")


@pytest.mark.parametrize("d", [1000, 2048, 8192])
@pytest.mark.parametrize("kind", ["centred", "mean", "positive", "normed", "sparse"])
def test_distill_wide_rows_of_any_kind(d, kind):
    """A logit is sums of up to 768 terms, 48 steps that lose up to 2^-23 each of what is there, of
    at most its terms' sizes, and the rounding of adding those up (2^-24 each): the width is in
    no bound but by the number of sums.  The rest as in the definitions' bound."""
    h, w, ids, t, rw = distill_case(200, d, 700, 20, seed=d)
    if kind == "mean":
        h += 3
    elif kind == "positive":
        h, w = h.abs(), w.abs()
    elif kind == "normed":
        h = (h.float() * torch.rand(d, generator=gen(1), device="cuda") * 2).to(BF)
        h = (h.float() * torch.rsqrt(h.float().square().mean(-1, keepdim=True))).to(BF)
    elif kind == "sparse":
        h[torch.rand(h.shape, generator=gen(2), device="cuda") < 0.98] = 0
        h *= 7
    op, loss = _r().VocabDistill(w, 200, 20, 0.5, gradients=False), empty(200, dtype=F32)
    op.loss(h, ids, t, loss)
    op.check()
    want = D.distill(h, w, ids, t, 0.5)["loss"]
    x, logt = h.double() @ w.double().T / 0.5, torch.log_softmax(t.double() / 0.5, -1)
    T1 = torch.zeros_like(x).scatter_add_(1, ids.long(), logt.exp())
    off = (T1 - torch.softmax(x, -1)).abs().sum(-1)
    size = (h.double().abs() @ w.double().abs().T).amax(-1) / 0.5
    span = x.amax(-1) - x.amin(-1) - logt.amin(-1)
    err = (48 * 2.0 ** -23 + (d / 640 + 1) * 2.0 ** -24) * size + 2.0 ** -21 * span + 2.0 ** -19
    T.close(loss, want, 2 * err * off + 2 * err * err + 2.0 ** -18 * want, "loss")


@pytest.mark.parametrize("n", [8192, 8193, 17_000])
def test_distill_more_rows_than_a_piece(n):
    """Rows counted by blocks, in pieces of 8,192 and in one."""
    h, w, _, t, rw = distill_case(n, 64, 200, 3, seed=1)
    ids = torch.randint(0, 200, (n, 3), generator=gen(2), device="cuda", dtype=I32)
    ids[1::3] = -1
    h[1::3] = float("nan")
    check_distill(h, w, ids, t, rw, tau=0.5)
    check_distill(h, w, ids, t, rw, piece=n)


# ---------------------------------------------------------------- verification

@pytest.mark.parametrize("vocab", [50, 5000, 40_000])
@pytest.mark.parametrize("where", ["drafted", "other", "both"])
@pytest.mark.parametrize("children", [1, 3])
def test_verify_nan_in_the_drafters_chances_is_reported(vocab, where, children):
    """A rejected draft's row of q with a NaN leaves sums that are none: no word is drawn."""
    nodes = 1 + children
    p, q = empty(2 * nodes, vocab, dtype=F32), empty(2 * nodes, vocab, dtype=F32)
    p[:] = 1.0 / vocab
    q[:] = 0.5 / vocab
    q[:, 7] = 0.5
    tokens = ints(*[7] * (2 * nodes))
    parent = ints(*([-1] + [0] * children) * 2)
    cu, u = ints(0, nodes, 2 * nodes), torch.full((2 * nodes,), 0.75, device="cuda")
    good = run_verify(p, q, tokens, parent, cu, u, nodes)
    assert good == by_hand(p, q, tokens, parent, cu, u, nodes) and good[1] == [1, 1]
    q[0, {"drafted": [7], "other": [vocab - 1], "both": [7, 3]}[where]] = float("nan")
    op = _r().VerifyDrafts(vocab)
    path, kept, nxt = run_verify(p, q, tokens, parent, cu, u, nodes, op, check=False)
    _reports(op)
    assert kept == [1, 1] and path == good[0] and nxt == [-1, good[2][1]]


@pytest.mark.parametrize("vocab", [50, 5000, 40_000])
def test_verify_rows_that_no_sum_needs_may_hold_nan(vocab):
    """q behind a leaf: there is no child that it could have been drawn for."""
    p, q, tokens, parent, cu, u = verify_case(vocab, [3, 3], seed=2, chain=True, near=0.0)
    u[1::3] = 0.5  # the target itself: all drafts are taken
    good = run_verify(p, q, tokens, parent, cu, u, 3)
    assert good[1] == [3, 3]
    q[2::3] = float("nan")
    assert run_verify(p, q, tokens, parent, cu, u, 3) == good


# ---------------------------------------------------------------- appends

@pytest.mark.parametrize("backwards", ["rows", "slots", "heads"])
@pytest.mark.parametrize("paged", [False, True])
def test_append_to_a_cache_that_runs_backwards(backwards, paged):
    """A caller's cache may have its last row, slot or head at the lowest address."""
    from paper_2607_16074_gb300 import jnx as J
    h, hkv, hd, slots, room, n = 4, 2, 64, 3, 16, 9
    g, op = gen(1), _r().QKNormRope(h, hkv, hd)
    qkv, q = normal(g, n, (h + 2 * hkv) * hd), empty(n, h, hd)
    slot, at = ints(0, 1, 2, 0, 1, 2, 0, 0, 2), ints(0, 3, 15, 1, 0, 7, 15, 8, 0)
    want = empty(2, slots, room, hkv, hd)
    op.append(qkv, at[None].contiguous(), q, want[0], want[1], slot, at)
    axis = {"slots": 0, "rows": 1, "heads": 2}[backwards]
    out = empty(2, slots, room, hkv, hd)
    s = list(out[0].stride())
    first = (out.shape[1 + axis] - 1) * s[axis] * 2  # bytes to the place of the first
    s[axis] = -s[axis]
    pos, table = at[None].contiguous(), ints([0], [1], [2])
    cache = (out[0].data_ptr() + first, out[1].data_ptr() + first, slots, room, *s[:3])
    rows = (q.data_ptr(), *q.stride()[:2])
    head = (op._ref, qkv.data_ptr(), qkv.stride(0), pos.data_ptr(), n)
    tail = (slot.data_ptr(), at.data_ptr(), op._status, torch.cuda.current_stream().cuda_stream)
    if paged:
        op._qp.fill(*rows, *cache, table.data_ptr(), 1, slots, 1)
        J.check(J.lib().jnx_op_qk_norm_rope_append_paged(*head, *op._qp.refs, *tail))
    else:
        op._qc.fill(*rows, *cache)
        J.check(J.lib().jnx_op_qk_norm_rope_append(*head, *op._qc.refs, *tail))
    op.check()
    assert torch.equal(out.flip(1 + axis).nan_to_num(99.0), want.nan_to_num(99.0))


# ---------------------------------------------------------------- trees

def guarded(op, room=1 << 20):
    """The operator's workspace at the start of a larger one; returns what lies behind it."""
    big = torch.full((op.ws.numel() + room,), 90, device="cuda", dtype=torch.uint8)
    op._held.append(big)
    op._ws, behind = big.data_ptr(), big[op.ws.numel():]
    return behind


@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 8, 128), (4, 4, 64), (8, 1, 256)])
@pytest.mark.parametrize("cu", [(0, 5, 4, 16), (0, 12, 0, 12), (4, 9, 0, 12), (0, 5, 2, 2)])
def test_tree_sequences_that_share_rows_are_left_out(heads, cu):
    """Rows are one sequence's, the first's: what would be another's is left out, and no sums are
    written that the workspace has no place for."""
    old = [2048 - 16] * 3
    c = Trees(heads, 64, old, [16] * 3, seed=2)
    op = _r().TreeAttention(*heads, 3, 16, c.table.shape[1] * 64)
    behind = guarded(op)
    out = torch.full((16, heads[0], heads[2]), 7.0, device="cuda", dtype=BF)
    # (an earlier call's records lie in the workspace: every row was the third's)
    op.forward(c.q[:16], c.kp, c.vp, c.table, ints(0, 0, 0, 16), c.n, c.sees[32:], out)
    op.check()
    out.fill_(7.0)
    op.forward(c.q[:16], c.kp, c.vp, c.table, ints(*cu), c.n, c.sees[:16], out)
    _reports(op)
    rows = slice(cu[0], cu[1])
    n = cu[1] - cu[0]
    where = place(c.table, 64, 0, range(old[0] + n))
    want, tol = D.tree(c.q[rows], c.kp[where], c.vp[where], old[0], c.sees[rows, None] >> torch.arange(n, device="cuda") & 1 == 1)
    T.close(out[rows], want, tol, "the first sequence")
    assert (out[:cu[0]] == 7).all() and (out[cu[1]:] == 7).all()
    assert (behind == 90).all()


def test_tree_rows_that_an_earlier_launch_had():
    """More sequences than a launch takes: one of the second that shares rows with one of the first."""
    heads, n = (4, 2, 64), 300
    c = Trees(heads, 64, [600] * n, [1] * n, seed=3)
    op = c.op()
    behind, good = guarded(op), torch.empty_like(c.q)
    c.run(op, good)
    c.compare(good)
    for first, left in ((100, 257), (0, 299), (200, 290)):
        # sequence left - 1 counts backwards, those behind it have rows of earlier ones
        cu = list(range(n + 1))
        cu[left] = first
        cu[left + 1:] = range(first + 1, first + 1 + n - left)
        out = torch.full_like(good, 7.0)
        op.forward(c.q, c.kp, c.vp, c.table, ints(*cu), c.n, c.sees, out)
        _reports(op)
        live = left - 1
        assert torch.equal(out[:live], good[:live])
        assert (out[live:] == 7).all()
    assert (behind == 90).all()
    out = torch.full_like(good, 7.0)
    c.run(op, out)
    assert torch.equal(out, good)


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (8, 1, 256)])
@pytest.mark.parametrize("entry", [0, -1, 1, 2 ** 31 - 1])
def test_tree_over_a_cache_of_no_pages(heads, entry):
    """Every page is one that is not there: read as zeros and reported, not what lies at the
    pointers."""
    from paper_2607_16074_gb300 import jnx as J
    h, hkv, hd = heads
    g, op = gen(0), _r().TreeAttention(*heads, 2, 9, 512)
    kp, vp = normal(g, 4, 128, hkv, hd), normal(g, 4, 128, hkv, hd)
    q, out = normal(g, 9, h, hd), empty(9, h, hd)
    table = torch.full((2, 4), entry, device="cuda", dtype=I32)
    cu, n, sees = ints(0, 4, 9), ints(100, 500), ints(*[1] * 9, dtype=torch.int64)
    r = op._views.refs
    op._views.fill(kp.data_ptr(), vp.data_ptr(), 0, 128, *kp.stride()[:3], table.data_ptr(), 4, 2, 4,
                   q.data_ptr(), *q.stride()[:2], out.data_ptr(), *out.stride()[:2])
    J.check(J.lib().jnx_op_tree_attention(
        r[0], r[1], h, hkv, hd, 9, r[2], cu.data_ptr(), n.data_ptr(), sees.data_ptr(), r[3], op._ws, op._nws,
        op._status, torch.cuda.current_stream().cuda_stream))
    _reports(op)
    assert (out == 0).all()


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (8, 1, 256), (4, 4, 256)])
@pytest.mark.parametrize("tokens", [257, 2048, 2049, 2113, 4097, 8192, 8193, 8321, 16_300, 33_000, 66_000])
def test_tree_sums_stay_in_the_workspace(heads, tokens):
    """Sequences of the most runs that their length may have, few nodes and many, in a workspace
    of just what the operator asks for."""
    page = 16 if tokens < 10_000 else 64
    c = Trees(heads, page, [tokens - 1, 0, tokens - 5, 100], [1, 3, 5, 2], seed=tokens)
    op = c.op()
    behind, out = guarded(op), empty(*c.q.shape)
    c.run(op, out)
    c.compare(out)
    assert (behind == 90).all()


@pytest.mark.parametrize("heads", [(8, 1, 256), (8, 2, 128), (14, 2, 64)])
@pytest.mark.parametrize("room", [1, 5, 16, 33, 63, 64])
def test_tree_of_a_short_page_a_sequence(heads, room):
    old = [max(room - 4, 0), 0, room // 2]
    c = Trees(heads, 0, old, [min(4, room), 1, min(3, room - room // 2)], seed=room, one_page=room)
    c.compare(c.run())
