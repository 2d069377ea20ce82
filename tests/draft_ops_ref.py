"""The definitions of answering with drafted tokens in 64 bits (torch, any device), with the
error each output may have.  A rounding to bf16 is off by half a step, 2^-8 of the value at
most; what 32-bit sums and the approximate exponential add is stated at each bound."""
import math

import torch

from tests.text_ops_ref import F64, close  # noqa: F401

U = 2.0 ** -8


def bits(row):
    """A row of truth values as the 64-bit word the operators take."""
    x = sum(1 << i for i, on in enumerate(row) if on)
    return x - (1 << 64) if x >> 63 else x


def ancestors(parents):
    """[t, t] truth values: the nodes a node sees in a tree."""
    out = torch.zeros(len(parents), len(parents), dtype=torch.bool)
    for i, p in enumerate(parents):
        if p >= 0:
            out[i] = out[p]
        out[i, i] = True
    return out


def paged(pages, table, tokens, page):
    """Rows of one sequence's tokens out of its pages."""
    at = torch.as_tensor(tokens, device=pages.device)
    return pages[table.long()[at // page], at % page]


def tree(q, k, v, n_old, sees):
    """One sequence: q [t, H, hd], k and v [n_old + t, Hkv, hd] 64-bit rows, sees [t, t].
    Returns out and its bound."""
    t, H, hd = q.shape
    r = H // k.shape[1]
    q = q.to(F64)
    see = torch.cat([torch.ones(t, n_old, dtype=torch.bool, device=q.device), sees.to(q.device)], 1)
    kk, vv = (x.to(F64).repeat_interleave(r, 1).transpose(0, 1) for x in (k, v))
    s = (q.transpose(0, 1) @ kk.transpose(1, 2) / math.sqrt(hd)).masked_fill(~see, -math.inf)
    top = s.amax(-1, keepdim=True) if s.shape[-1] else s.sum(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top)) * see
    p = p / p.sum(-1, keepdim=True).clamp_min(1e-300)
    out = (p @ vv).transpose(0, 1)
    # P is rounded, and the result; scores summed in 32 bits, of up to 2^8, and the exponential
    # add under 2^-12 to a probability and to their sum
    tol = (U + 2.0 ** -11) * ((p @ vv.abs()).transpose(0, 1) + out.abs())
    return out, tol


def verify(p, q, tokens, parent, u, vocab):
    """One sequence by hand: (path, next).  p and q [t, vocab] 64 bits."""
    t = len(parent)
    cur, path = 0, [0]
    while True:
        r, total, took = p[cur].clone(), 1.0, None
        for c in range(1, t):
            if parent[c] != cur or not 0 <= parent[c] < c or not 0 <= tokens[c] < vocab:
                continue
            guess = torch.zeros_like(r)
            if q is None:
                guess[tokens[c]] = 1.0
            else:
                guess = q[cur]
            if float(u[c]) * float(guess[tokens[c]]) * total < float(r[tokens[c]]):
                took = c
                break
            r = (r - total * guess).clamp_min(0.0)
            total = float(r.sum())
        if took is None:
            break
        path.append(took)
        cur = took
    if not float(r.sum()) > 0:
        r = p[cur]
    sums = r.cumsum(0)
    above = sums > float(u[0]) * float(sums[-1])
    return path, int(above.nonzero()[0]) if bool(above.any()) else -1


def distill(h, w, ids, teacher, tau, weight=None):
    """loss, and with weights dh, dw; then their bounds."""
    n, d = h.shape
    h, w, teacher = h.to(F64), w.to(F64), teacher.to(F64)
    v = w.shape[0]
    ok = (ids >= 0) & (ids < v) & (teacher > -math.inf)
    T = torch.zeros(n, v, dtype=F64, device=h.device)
    lg = (teacher / tau).masked_fill(~ok, -math.inf)
    top = lg.amax(-1, keepdim=True)
    e = torch.exp(lg - torch.where(top == -math.inf, 0.0, top)) * ok
    T.scatter_add_(1, torch.where(ok, ids, 0).long(), e / e.sum(-1, keepdim=True).clamp_min(1e-300))
    live = ok.any(-1)
    x = h @ w.T / tau
    # ignored rows may hold anything
    x = torch.where(live[:, None], x, 0.0)
    logp = x - torch.logsumexp(x, -1, keepdim=True)
    P = logp.exp()
    logt = torch.where(T > 0, T, 1.0).log()
    loss = torch.where(T > 0, T * (logt - logp), 0.0).sum(-1)
    r = dict(loss=torch.where(live, loss, 0.0))
    # what a logarithm of a probability may be off by: a product's d terms in steps of 16,
    # each off by 2^-22 of what was added so far; the differences and logarithms are of the
    # size of the logits, 2^-22 of that; the exponentials and their sums 2^-19 of P
    size = torch.where(live, (torch.nan_to_num(h).abs() @ w.abs().T).amax(-1), 0.0)
    span = x.abs().amax(-1) + torch.where(T > 0, -logt, 0.0).amax(-1) + 1
    err = (d / 16 + 16) * 2.0 ** -22 * size / tau + 2.0 ** -21 * span + 2.0 ** -19
    # the loss moves with its gradient, and with the square of what is left
    off = (P - T).abs().sum(-1)
    r["loss_tol"] = torch.where(live, 2 * err * off + 2 * err * err + 2.0 ** -18 * loss, 0.0)
    if weight is not None:
        c = torch.where(live, weight.to(F64), 0.0)[:, None] / tau
        g = (P - T) * c
        hh = torch.where(live[:, None], h, 0.0)
        r["dh"], r["dw"] = g @ w, g.T @ hh
        # a probability is rounded when it is formed and when it is scaled (an entry's once)
        eg = 2 * U * (1 + 2.0 ** -6) * g.abs() + 2 * err[:, None] * P * c.abs()
        r["dh_tol"] = U * r["dh"].abs() + eg @ w.abs()
        r["dw_tol"] = U * r["dw"].abs() + eg.T @ hh.abs()
    return r
