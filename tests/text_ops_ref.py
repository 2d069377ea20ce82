"""The text operators' definitions in 64 bits (torch, any device), with the error each
output may have: every bound is a sum over the roundings that the kernels make, of half
a unit in the last place of bf16 (2^-9 relative) each, doubled for what 32-bit sums and
the approximate exponential (under 2^-13) add."""
import math

import torch

F64 = torch.float64
U = 2.0 ** -8  # twice a bf16 rounding


def angles(pos, sections, theta, hd):
    """[n, hd / 2]: zero beyond the sections."""
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    out = torch.zeros(pos.shape[1], hd // 2, dtype=F64, device=pos.device)
    for i, a in enumerate(axis):
        out[:, i] = pos[a].to(F64) * theta ** (-2.0 * i / hd)
    return out


def rotate(x, a, sign=1.0):
    """x [n, heads, hd] turned by a [n, hd / 2]."""
    c, s = torch.cos(a)[:, None], sign * torch.sin(a)[:, None]
    lo, hi = x.chunk(2, -1)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def norm(x, gamma, eps):
    if gamma is None:
        return x
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * gamma.to(F64)


def norm_rope(x, gamma, pos, sections, theta, eps):
    x = x.to(F64)
    return rotate(norm(x, gamma, eps), angles(pos, sections, theta, x.shape[-1]))


def norm_rope_bound(y):
    """Rounding of y, and 2^-20 of the pair's length for the 32-bit arithmetic."""
    lo, hi = y.chunk(2, -1)
    pair = torch.sqrt(lo * lo + hi * hi)
    return U * y.abs() + 2.0 ** -20 * torch.cat([pair, pair], -1)


def seen(lq, lk, prefix, device="cpu"):
    """[lq, lk] of truth values."""
    j = torch.arange(lk, device=device)
    i = torch.arange(lq, device=device)[:, None]
    return (j <= lk - lq + i) | (j < prefix)


def attention(q, k, v, lens, dout=None):
    """out, lse (base 2), and with dout the gradients; then the bounds of out and of the
    gradients.  q [nq, H, hd], k / v [nk, Hkv, hd]; lens = (q, kv, prefix) lists."""
    dev = q.device
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    H, hkv, hd = q.shape[1], k.shape[1], q.shape[2]
    r = dict(out=torch.zeros_like(q), lse=torch.full((q.shape[0], H), -math.inf, dtype=F64,
                                                     device=dev))
    r["out_tol"] = torch.zeros_like(q)
    if dout is not None:
        dout = dout.to(F64)
        for n, x in (("dq", q), ("dk", k), ("dv", v)):
            r[n], r[n + "_tol"] = torch.zeros_like(x), torch.zeros_like(x)
    q0 = k0 = 0
    for lq, lk, pre in zip(*lens):
        see = seen(lq, lk, pre, dev)
        for h in range(H if lq and lk else 0):
            g = h // (H // hkv)
            R, K = slice(q0, q0 + lq), slice(k0, k0 + lk)
            qq, kk, vv = q[R, h], k[K, g], v[K, g]
            s = (qq @ kk.T / math.sqrt(hd)).masked_fill(~see, -math.inf)
            lse = torch.logsumexp(s, -1)
            p = torch.where(see, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
            o = p @ vv
            r["out"][R, h], r["lse"][R, h] = o, lse / math.log(2)
            # P and the result are rounded
            r["out_tol"][R, h] = U * (o.abs() + p @ vv.abs())
            if dout is None:
                continue
            do = dout[R, h]
            D = (do * o).sum(-1, keepdim=True)
            ds = p * (do @ vv.T - D) / math.sqrt(hd)
            # dS is rounded, and D comes from the rounded output
            eds = U * (ds.abs() + p * (do.abs() * o.abs()).sum(-1, keepdim=True) / math.sqrt(hd))
            # P from the forward's log-sum-exp: 2^-13 of it, like the exponential's error
            eds += 2.0 ** -13 * ds.abs()
            r["dq"][R, h] = ds @ kk
            r["dq_tol"][R, h] = U * (ds @ kk).abs() + eds @ kk.abs()
            r["dk"][K, g] += ds.T @ qq
            r["dk_tol"][K, g] += eds.T @ qq.abs()
            r["dv"][K, g] += p.T @ do
            r["dv_tol"][K, g] += U * (p.T @ do.abs())
        q0, k0 = q0 + lq, k0 + lk
    if dout is not None:
        for n in ("dk", "dv"):
            r[n + "_tol"] += U * r[n].abs()
    return r


def vocab(h, w, targets, weight=None):
    """loss, and with weights dh, dw; then their bounds."""
    h, w = h.to(F64), w.to(F64)
    n, d = h.shape
    keep = (targets >= 0) & (targets < w.shape[0])
    t = torch.where(keep, targets, 0).long()
    x = h @ w.T
    lse = torch.logsumexp(x, -1)
    r = dict(loss=torch.where(keep, lse - x.gather(1, t[:, None])[:, 0], 0.0))
    # 32-bit sums of d products in steps of 16, each off by 2^-22 of what was added so
    # far; the log-sum-exp's own 32-bit sum and the exponential add 2^-19
    size = (h.abs() @ w.abs().T).amax(-1)
    r["loss_tol"] = torch.where(keep, (d / 16 + 16) * 2.0 ** -22 * size + 2.0 ** -19 * (1 + lse.abs()), 0.0)
    if weight is not None:
        g = torch.exp(x - lse[:, None])
        g[torch.arange(n), t] -= 1
        g *= torch.where(keep, weight.to(F64), 0.0)[:, None]
        r["dh"], r["dw"] = g @ w, g.T @ h
        # a probability is rounded when it is formed and when it is scaled
        r["dh_tol"] = U * r["dh"].abs() + 2 * U * (g.abs() @ w.abs())
        r["dw_tol"] = U * r["dw"].abs() + 2 * U * (g.abs().T @ h.abs())
    return r


def close(got, want, tol, what=""):
    got = got.to(F64)
    assert torch.isfinite(got[torch.isfinite(want)]).all(), f"{what}: not finite"
    over = ((got - want).abs() - tol - 1e-30).amax() if want.numel() else torch.tensor(-1.0)
    if over > 0:
        i = int(((got - want).abs() - tol).argmax())
        raise AssertionError(f"{what}: element {i}: {got.flatten()[i]} for {want.flatten()[i]}, "
                             f"may be off by {tol.flatten()[i]}")
