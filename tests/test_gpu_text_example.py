"""The text operators together, as the example runs them: losses go down, and the tokens
answered one by one are those that the whole prompt, run again, gives."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_text_tenant_trains_and_answers():
    from paper_2607_16074_gb300 import runtime as R
    from paper_2607_16074_gb300 import text_example as E
    tenant, losses, (x, pos, lens, images, tokens, seen) = E.main(steps=12, verbose=False)
    assert losses[-1] < 0.5 * losses[0], losses
    # every prompt with its answer behind it, run as one prompt
    n = tokens.shape[1] - 1
    rows, parts, at = [], [], 0
    for i, length in enumerate(lens):
        rows += [x[at:at + length], tenant.embed(tokens[i, :n])]
        more = torch.arange(length, length + n, device="cuda", dtype=torch.int32).expand(3, n)
        parts += [pos[:, at:at + length], more]
        at += length
    longer = [length + n for length in lens]
    plan = R.PromptPlan(longer, prefix=list(images))
    y, _ = tenant.forward(plan, torch.cat(rows).contiguous(), torch.cat(parts, 1).contiguous())
    logits, at = tenant.logits(y), 0
    for i, length in enumerate(lens):
        again = logits[at + length - 1:at + length + n]
        # bf16 roundings of the heads' rows, P and the output on either way: 2^-8 each
        assert (again - seen[i]).abs().max() < 0.02 * again.abs().max()
        at += length + n
