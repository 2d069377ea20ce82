"""A text tenant from end to end on one attention layer: trained on the next token, then
answering token by token, and several tokens a step with a drafter that learned from it.

    python -m paper_2607_16074_gb300.text_example

A sample is some image rows, which all of its rows see, and text behind them, causal.  The
layer's projections are frozen, as the shared backbone's are; the tenant trains what is its
own, the norms' gains of its query and key heads and its vocabulary.  Random weights and
samples: the losses show that the gradients go downhill, the answers that a token against
the cache gives what the whole prompt does.

The drafter guesses the next word from the last one alone, by a vocabulary of its own that
is distilled from the tenant's best logits.  A step of the drafted answer takes a small tree
of its guesses through the layer at once, into a paged cache; what the verification accepts
is kept, so that the answer is the tenant's own in fewer steps.
"""
from __future__ import annotations

import torch

from . import jnx as J
from . import runtime as R

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class TextTenant:
    """One pre-norm attention layer between a vocabulary's embeddings and logits.  The words
    are one table for both, but learn through the logits alone: the gradient that reaches them
    through the embeddings, by the residual and the projections, is left out."""

    def __init__(self, d=512, heads=8, kv_heads=2, head_dim=64, vocab=1024, seed=0):
        self.d, self.vocab, self.dims = d, vocab, (heads, kv_heads, head_dim)
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s, std: (torch.randn(*s, generator=g, device="cuda") * std).to(BF)  # noqa: E731
        self.w_qkv = rnd((heads + 2 * kv_heads) * head_dim, d, std=d ** -0.5)
        self.w_o = rnd(d, heads * head_dim, std=(heads * head_dim) ** -0.5)
        self.w_o_t = self.w_o.T.contiguous()
        self.ones = torch.ones(d, device="cuda", dtype=BF)
        self.gains = torch.ones(2, 1, head_dim, device="cuda", dtype=BF)
        self.words = rnd(1, vocab, d, std=0.05)  # [tenant slot, vocab, d]
        # time turns half of the frequencies, an image patch's row and column a quarter each
        q = head_dim // 8
        self.rope = R.QKNormRope(*self.dims, self.gains[0, 0], self.gains[1, 0],
                                 sections=(head_dim // 2 - 2 * q, q, q))
        self.d_gains = torch.empty(2, 1, head_dim, device="cuda", dtype=F32)
        self.d_words = torch.empty(1, vocab, d, device="cuda", dtype=F32)
        self.adamw = R.TenantAdamW([(self.gains[0], self.d_gains[0]), (self.gains[1], self.d_gains[1]),
                                    (self.words, self.d_words)])

    # ---- the framework's GEMMs and norms around the operators ----

    def _gemm(self, a, w, out, epi):
        J.check(J.lib().jnx_op_gemm(a.data_ptr(), w.data_ptr(), a.shape[0], w.shape[0], a.shape[1], epi,
                                    out.data_ptr(), out.stride(0), None, 0, 0, 0, 1e4, 0, None, 0,
                                    R._stream(None)))
        return out

    def _norm(self, x):
        out = torch.empty(x.shape, device="cuda", dtype=BF)
        J.check(J.lib().jnx_op_rmsnorm(x.data_ptr(), self.ones.data_ptr(), 1e-6, *x.shape,
                                       out.data_ptr(), R._stream(None)))
        return out

    def _rows(self, n, heads):
        return torch.empty(n, heads, self.dims[2], device="cuda", dtype=BF)

    def _qkv(self, x):
        return self._gemm(self._norm(x), self.w_qkv,
                          torch.empty(x.shape[0], self.w_qkv.shape[0], device="cuda", dtype=BF),
                          J.JNX_EPI_BF16)

    def _out(self, x, att):
        """The residual behind the layer."""
        return self._gemm(att.flatten(1), self.w_o, x.clone(), J.JNX_EPI_RESID)

    def _values(self, qkv):
        h, hkv, hd = self.dims
        return qkv.view(-1, h + 2 * hkv, hd)[:, h + hkv:]

    def embed(self, ids):
        return self.words[0][ids.long()].float()

    def logits(self, x):
        return self._gemm(self._norm(x), self.words[0],
                          torch.empty(x.shape[0], self.vocab, device="cuda", dtype=F32), J.JNX_EPI_F32)

    # ---- a prompt, with and without gradients ----

    def forward(self, plan, x, pos, gradients=False):
        """Rows x [n, d] fp32 of packed samples through the layer; what the backward reads."""
        h, hkv, _ = self.dims
        n, qkv = x.shape[0], self._qkv(x)
        q, k, att = self._rows(n, h), self._rows(n, hkv), self._rows(n, h)
        self.rope.forward(qkv, pos, q, k)
        op = R.PromptAttention(*self.dims, plan, gradients=gradients)
        lse = torch.empty(n, h, device="cuda", dtype=F32) if gradients else None
        op.forward(q, k, self._values(qkv), att, lse)
        op.check()
        return self._out(x, att), (op, qkv, q, k, att, lse)

    def train_step(self, plan, x, pos, targets, weight, lr):
        """One step on the weighted sum of the rows' losses; returns the losses."""
        y, (op, qkv, q, k, att, lse) = self.forward(plan, x, pos, gradients=True)
        n = x.shape[0]
        loss = torch.empty(n, device="cuda", dtype=F32)
        dh, dw = torch.empty(n, self.d, device="cuda", dtype=BF), torch.empty_like(self.words[0])
        head = R.VocabLoss(self.words[0], max_rows=n)
        head.train(self._norm(y), targets, weight, loss, dh, dw)
        head.check()
        # through the last norm and the output projection
        dy = torch.empty(n, self.d, device="cuda", dtype=F32)
        dy_bf, dn = torch.empty_like(dh), dh.float()
        J.check(J.lib().jnx_op_rms_backward(y.data_ptr(), self.ones.data_ptr(), 1e-6, dn.data_ptr(), None,
                                            n, self.d, dy.data_ptr(), dy_bf.data_ptr(), R._stream(None)))
        datt = self._gemm(dy_bf, self.w_o_t, torch.empty_like(att).flatten(1), J.JNX_EPI_BF16)
        # through the attention; dq and dk go where the norms' backward turns them around
        dqkv = torch.empty_like(qkv)
        h, hkv, hd = self.dims
        rows = dqkv.view(n, h + 2 * hkv, hd)
        dq, dk = rows[:, :h], rows[:, h:h + hkv]
        op.backward(q, k, self._values(qkv), att, lse, datt.view_as(att), dq, dk, rows[:, h + hkv:])
        op.check()
        self.rope.backward(qkv, pos, dq, dk, dqkv, self.d_gains[0, 0], self.d_gains[1, 0])
        self.d_words[0].copy_(dw)
        self.adamw.step([0], lr=lr)
        return loss

    # ---- answering ----

    def answer(self, plan, x, pos, q_lens, steps):
        """Greedy tokens [batch, steps] behind every packed prompt and the logits each came
        from: the prompt once, then a token at a time against the cache."""
        h, hkv, hd = self.dims
        b, ends = len(q_lens), torch.tensor(q_lens, device="cuda").cumsum(0)
        room = max(q_lens) + steps
        kc = torch.empty(b, room, hkv, hd, device="cuda", dtype=BF)
        vc = torch.empty_like(kc)
        slots = torch.arange(b, device="cuda", dtype=I32)
        slot = torch.cat([slots[i].expand(n) for i, n in enumerate(q_lens)]).contiguous()
        at = torch.cat([torch.arange(n, device="cuda", dtype=I32) for n in q_lens])
        y, (_, qkv, q, *_) = self.forward(plan, x, pos)
        self.rope.append(qkv, pos, q, kc, vc, slot, at)
        decode = R.DecodeAttention(h, hkv, hd, max_batch=b)
        n = torch.tensor(q_lens, device="cuda", dtype=I32)
        last, tokens, seen = y[ends - 1], [], []
        for step in range(steps):
            seen.append(self.logits(last.contiguous()))
            tokens.append(seen[-1].argmax(1).to(I32))
            if step + 1 == steps:
                break
            x1 = self.embed(tokens[-1])
            p1 = n.expand(3, b).contiguous()  # behind the prompt the axes run together
            qkv, q, att = self._qkv(x1), self._rows(b, h), self._rows(b, h)
            self.rope.append(qkv, p1, q, kc, vc, slots, n)
            n = n + 1
            decode.forward(q, kc, vc, slots, n, att)
            last = self._out(x1, att)
        self.rope.check()
        decode.check()
        return torch.stack(tokens, 1), torch.stack(seen, 1)


class Drafter:
    """The next word from the last one: its embedding against words of the drafter's own."""

    def __init__(self, tenant, top=8, lr=2e-3, max_rows=1024):
        self.tenant, self.lr, self.top = tenant, lr, top
        self.words = (tenant.words * 0.5).contiguous()
        self.d_words = torch.empty(self.words.shape, device="cuda", dtype=F32)
        self.adamw = R.TenantAdamW([(self.words, self.d_words)])
        self.head = R.VocabDistill(self.words[0], max_rows=max_rows, top=top, temperature=1.0)

    def learn(self, ids, logits):
        """One step towards the tenant's logits [n, vocab] behind the words ids [n] (negative:
        no word stands there); returns the losses."""
        n, t = ids.shape[0], self.tenant
        best = torch.topk(logits, self.top, -1)
        guesses = torch.where(ids[:, None] >= 0, best.indices, -1).to(I32).contiguous()
        h = t._norm(t.embed(ids.clamp_min(0)))
        loss = torch.empty(n, device="cuda", dtype=F32)
        dh, dw = torch.empty(n, t.d, device="cuda", dtype=BF), torch.empty_like(self.words[0])
        weight = torch.full((n,), 1.0 / n, device="cuda")
        self.head.train(h, guesses, best.values.contiguous(), weight, loss, dh, dw)
        self.head.check()
        self.d_words[0].copy_(dw)
        self.adamw.step([0], lr=self.lr)
        return loss

    def chances(self, ids):
        t = self.tenant
        out = torch.empty(ids.shape[0], t.vocab, device="cuda", dtype=F32)
        return torch.softmax(t._gemm(t._norm(t.embed(ids)), self.words[0], out, J.JNX_EPI_F32), -1)


# the root, two guesses behind it, and what follows the first of them
TREE = (-1, 0, 0, 1, 1, 3)


def answer_drafted(tenant, drafter, plan, x, pos, q_lens, steps, tree=TREE, page=16, seed=0,
                   greedy=True):
    """At least `steps` tokens behind every packed prompt, as lists, and the passes through the
    layer that they took.  greedy: the tenant's best word is its only one."""
    h, hkv, hd = tenant.dims
    b, t, dev = len(q_lens), len(tree), "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    depth = [0]
    for i in range(1, t):
        depth.append(depth[tree[i]] + 1)
    sees = [0] * t
    for i in range(t):
        sees[i] = (sees[tree[i]] if i else 0) | 1 << i
    each = lambda v, dtype=I32: torch.tensor(v, device=dev, dtype=dtype).repeat(b)  # noqa: E731
    parent, sees, depth_t = each(tree), each(sees, torch.int64), each(depth)
    nodes = torch.arange(t, device=dev, dtype=I32).repeat(b)
    seq = torch.arange(b, device=dev, dtype=I32).repeat_interleave(t)
    cu = torch.arange(b + 1, device=dev, dtype=I32) * t
    up = (seq * t + parent.clamp_min(0)).long()
    # pages for the prompt, the answer and a last tree, dealt out in turn
    entries = (max(q_lens) + steps + 2 * t + page - 1) // page
    table = torch.arange(entries * b, device=dev, dtype=I32).view(entries, b).T.contiguous()
    kp = torch.empty(entries * b, page, hkv, hd, device=dev, dtype=BF)
    vp = torch.empty_like(kp)
    attend = R.TreeAttention(h, hkv, hd, max_batch=b, max_rows=b * t, max_tokens=entries * page)
    verify, keep = R.VerifyDrafts(tenant.vocab), R.KeepDrafts(hkv, hd)

    y, (_, qkv, q, *_) = tenant.forward(plan, x, pos)
    of = torch.cat([torch.full((n,), i, device=dev, dtype=I32) for i, n in enumerate(q_lens)])
    at = torch.cat([torch.arange(n, device=dev, dtype=I32) for n in q_lens])
    tenant.rope.append_paged(qkv, pos, q, kp, vp, table, of, at)
    n = torch.tensor(q_lens, device=dev, dtype=I32)
    last = y[torch.tensor(q_lens, device=dev).cumsum(0) - 1].contiguous()
    token = tenant.logits(last).argmax(1).to(I32)  # the first word of the answer
    answers, passes = [[w] for w in token.tolist()], 1
    path = torch.empty(b, t, device=dev, dtype=I32)
    kept, word = torch.empty(b, device=dev, dtype=I32), torch.empty(b, device=dev, dtype=I32)
    while min(map(len, answers)) < steps:
        tokens = token.repeat_interleave(t)
        for level in range(1, max(depth) + 1):  # guesses behind guesses
            q_rows = drafter.chances(tokens)
            drawn = torch.multinomial(q_rows[up], 1, generator=g)[:, 0].to(I32)
            tokens = torch.where(depth_t == level, drawn, tokens)
        chances = drafter.chances(tokens)
        x1 = tenant.embed(tokens)
        qkv, q, att = tenant._qkv(x1), tenant._rows(b * t, h), tenant._rows(b * t, h)
        old = n.repeat_interleave(t)
        tenant.rope.append_paged(qkv, (old + depth_t).expand(3, b * t).contiguous(), q, kp, vp, table,
                                 seq, old + nodes)
        attend.forward(q, kp, vp, table, cu, n, sees, att)
        logits = tenant.logits(tenant._out(x1, att))
        p = torch.zeros_like(logits).scatter_(1, logits.argmax(1, keepdim=True), 1.0) if greedy \
            else torch.softmax(logits, -1)
        u = torch.rand(b * t, generator=g, device=dev)
        verify.forward(p, chances, tokens, parent, cu, u, path, kept, word)
        keep.forward(kp, vp, table, n, path, kept)
        for i, (nodes_i, k, w) in enumerate(zip(path.tolist(), kept.tolist(), word.tolist())):
            if len(answers[i]) < steps:
                answers[i] += [int(tokens[i * t + j]) for j in nodes_i[1:k]] + [w]
        # a sequence that is through stays where it is
        done = torch.tensor([len(a) >= steps for a in answers], device=dev)
        n = torch.where(done, n, n + kept)
        token = torch.where(done, token, word)
        passes += 1
    for op in (tenant.rope, attend, verify, keep):
        op.check()
    return [a[:steps] for a in answers], passes


def positions(images, texts, grid=4):
    """Time, row and column of each packed row: image patches share their image's time."""
    out = []
    for i, t in zip(images, texts):
        patch = torch.arange(i, dtype=I32)
        text = torch.arange(i, i + t, dtype=I32)
        out.append(torch.stack([torch.cat([torch.zeros_like(patch), text]),
                                torch.cat([patch // grid, text]), torch.cat([patch % grid, text])]))
    return torch.cat(out, 1).cuda().contiguous()


def samples(tenant, images, texts, seed=1):
    """Packed samples of image rows and a text that counts upwards in steps of its own."""
    g = torch.Generator().manual_seed(seed)
    rows, targets = [], []
    for i, t in zip(images, texts):
        first, by = (int(torch.randint(1, 9, (1,), generator=g)) for _ in range(2))
        ids = (first + by * torch.arange(t + 1)) % tenant.vocab
        image = torch.randn(i, tenant.d, generator=g) * 0.05
        rows.append(torch.cat([image.cuda(), tenant.embed(ids[:-1].cuda())]))
        targets.append(torch.cat([torch.full((i,), -1), ids[1:]]))
    return torch.cat(rows), torch.cat(targets).to(I32).cuda()


def main(steps=30, images=(16, 12, 0, 20), texts=(24, 40, 7, 33), lr=3e-3, verbose=True):
    tenant = TextTenant()
    lens = [i + t for i, t in zip(images, texts)]
    plan = R.PromptPlan(lens, prefix=list(images))
    pos = positions(images, texts)
    losses = []
    for step in range(steps):
        x, targets = samples(tenant, images, texts)  # embeddings follow the vocabulary
        weight = torch.full((len(targets),), 1.0 / sum(texts), device="cuda")
        loss = tenant.train_step(plan, x, pos, targets, weight, lr)
        losses.append(float((loss * weight).sum()))
        if verbose and step % 5 == 0:
            print(f"step {step:3d}: loss {losses[-1]:.4f}")
    x, _ = samples(tenant, images, texts)
    tokens, seen = tenant.answer(plan, x, pos, lens, 6)
    if verbose:
        print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; answers {tokens.tolist()}")
    return tenant, losses, (x, pos, lens, images, tokens, seen)


def drafted(tenant, images, texts, steps=30, answer=12, verbose=True):
    """A drafter that learns from the tenant on its samples, and answers of both together."""
    lens = [i + t for i, t in zip(images, texts)]
    plan, pos = R.PromptPlan(lens, prefix=list(images)), positions(images, texts)
    drafter = Drafter(tenant)
    x, targets = samples(tenant, images, texts)
    # the word of a text row is the last one's target (a sample's first word is not asked about)
    ids = targets.roll(1)
    ids[torch.tensor(lens, device="cuda").cumsum(0) - torch.tensor(lens, device="cuda")] = -1
    y, _ = tenant.forward(plan, x, pos)
    # ... and what the tenant answers, a few words far
    tokens, seen = tenant.answer(plan, x, pos, lens, 4)
    ids = torch.cat([ids, tokens[:, :-1].flatten()])
    logits = torch.cat([tenant.logits(y), seen[:, 1:].flatten(0, 1)])
    losses = [float(drafter.learn(ids, logits).mean()) for _ in range(steps)]
    answers, passes = answer_drafted(tenant, drafter, plan, x, pos, lens, answer)
    if verbose:
        print(f"drafter's loss {losses[0]:.4f} -> {losses[-1]:.4f}; {answer} words in {passes} passes: "
              f"{answers}")
    return drafter, losses, answers, passes


if __name__ == "__main__":
    shapes = dict(images=(16, 12, 0, 20), texts=(24, 40, 7, 33))
    drafted(main(**shapes)[0], **shapes)
