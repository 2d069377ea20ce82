"""What calls of the drafted tokens' operators may hold beside the ordinary: teachers' entries
that weigh nothing, students at their teacher, products with few terms, probabilities that are
none, layouts whose strides run backwards, sequences that share rows, caches without pages."""
import pytest
import torch

from tests import draft_ops_ref as D
from tests import text_ops_ref as T
from tests.test_gpu_draft_ops import (BF, F32, HEADS, I32, Trees, _r, _reports, by_hand, check_distill, distill_case,
                                      empty, gen, ints, normal, run_verify, verify_case)

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
