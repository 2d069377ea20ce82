"""Drafts in a paged cache, trees, verification, kept rows and the distilled drafter together,
as the example runs them."""
import pytest
import torch

pytestmark = pytest.mark.gpu
SHAPES = dict(images=(16, 12, 0, 20), texts=(24, 40, 7, 33))


@pytest.fixture(scope="module")
def tenant():
    from paper_2607_16074_gb300 import text_example as E
    return E.main(steps=20, verbose=False, **SHAPES)[0]


def _prompt(tenant):
    from paper_2607_16074_gb300 import runtime as R
    from paper_2607_16074_gb300 import text_example as E
    lens = [i + t for i, t in zip(*SHAPES.values())]
    x, _ = E.samples(tenant, **SHAPES)
    return R.PromptPlan(lens, prefix=list(SHAPES["images"])), x, E.positions(**SHAPES), lens


def _agrees(tenant, plan, x, pos, lens, answers):
    """Every word is the best of the whole prompt with the answer so far behind it, run again, or
    within the roundings of the best: 2^-8 for each of the heads' rows, P and the output, on
    either way."""
    from paper_2607_16074_gb300 import runtime as R
    n = len(answers[0]) - 1
    tokens = torch.tensor(answers, device="cuda", dtype=torch.int32)
    rows, parts, at = [], [], 0
    for i, length in enumerate(lens):
        rows += [x[at:at + length], tenant.embed(tokens[i, :n])]
        more = torch.arange(length, length + n, device="cuda", dtype=torch.int32).expand(3, n)
        parts += [pos[:, at:at + length], more]
        at += length
    longer = R.PromptPlan([v + n for v in lens], prefix=list(SHAPES["images"]))
    y, _ = tenant.forward(longer, torch.cat(rows).contiguous(), torch.cat(parts, 1).contiguous())
    logits, at = tenant.logits(y), 0
    for i, length in enumerate(lens):
        own = logits[at + length - 1:at + length + n]
        chosen = own.gather(1, tokens[i].long()[:, None])[:, 0]
        assert (own.amax(1) - chosen < 0.02 * own.abs().max()).all(), i
        at += length + n


def test_drafted_answers_are_the_tenants_own(tenant):
    from paper_2607_16074_gb300 import text_example as E
    drafter, losses, answers, passes = E.drafted(tenant, answer=12, verbose=False, **SHAPES)
    plan, x, pos, lens = _prompt(tenant)
    assert all(len(a) == 12 for a in answers) and passes <= 12
    _agrees(tenant, plan, x, pos, lens, answers)
    # a drafter that knows nothing, and trees of other forms: the same answer in more passes
    none = E.Drafter(tenant)
    none.words.zero_()
    for tree in (E.TREE, (-1,), (-1, 0, 1, 2, 3), (-1, 0, 0, 0, 1, 1, 2, 2, 4, 8, 9)):
        for d in (drafter, none):
            again, _ = E.answer_drafted(tenant, d, plan, x, pos, lens, 8, tree=tree, seed=3)
            _agrees(tenant, plan, x, pos, lens, again)


def test_drawn_answers_are_words(tenant):
    from paper_2607_16074_gb300 import text_example as E
    plan, x, pos, lens = _prompt(tenant)
    answers, _ = E.answer_drafted(tenant, E.Drafter(tenant), plan, x, pos, lens, 9, greedy=False, page=32)
    assert all(0 <= w < tenant.vocab for a in answers for w in a)


def test_drafters_gradient_by_differences(tenant):
    """The distilled words' gradient, as a step of the example takes it, along directions."""
    from paper_2607_16074_gb300 import text_example as E
    from tests import draft_ops_ref as D
    plan, x, pos, lens = _prompt(tenant)
    y, _ = tenant.forward(plan, x, pos)
    logits = tenant.logits(y)
    ids = torch.randint(0, tenant.vocab, (x.shape[0],), device="cuda",
                        generator=torch.Generator(device="cuda").manual_seed(1))
    ids[::9] = -1
    d = E.Drafter(tenant)
    words = d.words[0].double().clone()
    d.learn(ids, logits)  # d_words hold the step's gradient
    best = torch.topk(logits, d.top, -1)
    guesses = torch.where(ids[:, None] >= 0, best.indices, -1)
    h = tenant._norm(tenant.embed(ids.clamp_min(0))).double()
    n = x.shape[0]

    def value(w):
        return float(D.distill(h, w, guesses, best.values, 1.0)["loss"].sum()) / n
    want = D.distill(h, words, guesses, best.values, 1.0, torch.full((n,), 1.0 / n, device="cuda"))
    g = torch.Generator(device="cuda").manual_seed(2)
    for _ in range(3):
        v = torch.randn(words.shape, generator=g, device="cuda", dtype=torch.float64)
        eps = 1e-4
        slope = (value(words + eps * v) - value(words - eps * v)) / (2 * eps)
        exact = float((want["dw"] * v).sum())
        assert abs(slope - exact) < 1e-4 * float(want["dw"].norm())
        # the kernel's gradient may be off by its bound at every element
        assert abs(float((d.d_words[0].double() * v).sum()) - exact) <= float((want["dw_tol"] * v.abs()).sum())
