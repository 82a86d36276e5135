"""Plain float64 forms of the teacher-score operators, for the tests: definitions written out with
torch, nothing shared with the kernels."""
from __future__ import annotations

import math

import torch


def row_mask(B, T, window=None, rollout=None):
    """[B,T] bool: the processed positions t < min(W, R, T), lengths clamped to [0,T]."""
    end = torch.full((B,), T, dtype=torch.int64)
    for n in (window, rollout):
        if n is not None:
            end = torch.minimum(end, n.cpu().long().clamp(0, T))
    return torch.arange(T)[None, :] < end[:, None]


def order(z, K):
    """Indices of the K largest of each row, equal ones in the order of their index."""
    return torch.sort(z.double() + 0.0, dim=-1, descending=True, stable=True).indices[..., :K]


def times(p, x):
    """p * x with 0 * inf = 0."""
    return torch.where(p == 0, torch.zeros_like(p), p * x)


def log_parts(z):
    """Largest entry m of each row (0 where it is not finite) and log sum exp(z - m).  Log
    probabilities are (z - m) - that: in a row of entries of size 1e30 the normaliser itself cannot
    hold the logarithm of their number."""
    m = z.max(dim=-1, keepdim=True).values
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    return m, torch.log(torch.exp(z - m).sum(dim=-1, keepdim=True))


def log_sum_exp(z):
    m, s = log_parts(z)
    return (m + s)[..., 0]


def scores(z, y, K):
    """logprob, entropy, lse, top_ids, top_logprobs, rest of rows z [n,V] with tokens y [n]."""
    z = z.double()
    m, s = log_parts(z)
    lse, lp = (m + s)[:, 0], (z - m) - s
    p = torch.exp(lp)
    ids = order(z, K)
    out = torch.ones_like(z, dtype=torch.bool).scatter_(1, ids, False)
    return dict(lse=lse, logprob=lp.gather(1, y[:, None].long())[:, 0],
                entropy=-times(p, lp).sum(dim=1), top_ids=ids, top_logprobs=lp.gather(1, ids),
                rest=log_sum_exp(torch.where(out, lp, -math.inf)))


def scores_grad(z, y, lse, entropy, w, h, ids, d):
    """Gradient of sum w logprob + h entropy + d . top_logprobs, the normaliser and the entropy as
    given; w, h [n], ids, d [n,K] (ids of -1 are none).  Also the size of its terms per entry."""
    z = z.double()
    n, V = z.shape
    lp = z - lse.double()[:, None]
    p = torch.exp(lp)
    own = torch.zeros_like(z)
    rows = torch.arange(n, device=z.device)
    own.index_put_((rows, y.long()), w.double(), accumulate=True)
    size = torch.zeros_like(z)
    size.index_put_((rows, y.long()), w.double().abs(), accumulate=True)
    for j in range(ids.shape[1]):
        ok = ids[:, j] >= 0
        own.index_put_((rows[ok], ids[ok, j].long()), d[ok, j].double(), accumulate=True)
        size.index_put_((rows[ok], ids[ok, j].long()), d[ok, j].double().abs(), accumulate=True)
    total = own.sum(dim=1, keepdim=True)
    ent = times(p, lp + entropy.double()[:, None])
    grad = own - p * total - h.double()[:, None] * ent
    t = times(p, lp.abs() + entropy.double().abs()[:, None]) * h.double().abs()[:, None]
    size += p * size.sum(dim=1, keepdim=True) + t
    return grad, size


REST_FLOOR = 2.0 ** -24


def topk_kl(z, y, ids, lq, rest, forward, alpha=1.0):
    """Divergence over the categories top_1 .. top_K (ids of -1 are none) and the rest: kl, logratio,
    gsq, lse, grad of rows z [n,V]; rest [n] or None (what the list leaves of 1, floored).
    Also the size of the gradient's terms per entry and of the divergence's."""
    z = z.double()
    n, V = z.shape
    m, s = log_parts(z)
    lse, lp = (m + s)[:, 0], (z - m) - s
    p = torch.exp(lp)
    kl, c, gsq = (torch.zeros(n, dtype=torch.float64, device=z.device) for _ in range(3))
    size_kl = torch.zeros_like(kl)
    grad, size = torch.zeros_like(z), torch.zeros_like(z)
    for i in range(n):
        keep = ids[i] >= 0
        j, q = ids[i][keep].long(), lq[i][keep].double()
        cat = torch.full((V,), len(j), dtype=torch.int64, device=z.device)
        cat[j] = torch.arange(len(j), device=z.device)
        outside = cat == len(j)
        pr = p[i][outside].sum()
        lr = rest[i].double() if rest is not None else \
            torch.log(torch.clamp(1.0 - torch.exp(q).sum(), min=REST_FLOOR))
        P = torch.cat([p[i][j], pr[None]])
        lP = torch.cat([lp[i][j], log_sum_exp(torch.where(outside, lp[i], -math.inf))[None]])
        lQ = torch.cat([q, lr[None]])
        D = lP - lQ
        if forward:
            terms = -times(torch.exp(lQ), D)
            kl[i] = terms.sum()
            # p_k / P_r, formed among the entries of the rest: their mass may be nothing to the whole
            zo = torch.where(outside, z[i], -math.inf)
            mo, so = log_parts(zo)
            share = torch.exp(lr) * torch.exp((zo - mo) - so) if torch.isfinite(so) else torch.zeros_like(zo)
            g = p[i] - share
            g[j] = P[:-1] - torch.exp(q)
            size[i] = p[i] + share
            size[i][j] = P[:-1] + torch.exp(q)
        else:
            terms = times(P, D)
            kl[i] = terms.sum()
            g = times(p[i], D[cat] - kl[i])
            size[i] = times(p[i], D[cat].abs() + terms.abs().sum())
        size_kl[i] = terms.abs().sum()
        grad[i] = alpha * g
        size[i] *= abs(alpha)
        gsq[i] = (grad[i] ** 2).sum()
        yi = int(y[i])
        c[i] = D[cat[yi]] if 0 <= yi < V else math.nan
    return dict(kl=kl, logratio=c, gsq=gsq, lse=lse, grad=grad, size=size, size_kl=size_kl, p=p)


def quantize(x):
    """Whole numbers and step of each row: step = max|x| / 127 and q = x / step, both rounded to fp32
    as the operator defines them (numpy's division is correctly rounded), q to nearest even."""
    import numpy as np
    a = x.detach().float().cpu().numpy()
    step = np.abs(a).max(axis=1).astype(np.float32) / np.float32(127)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(step[:, None] > 0, np.rint(a / step[:, None]), np.float32(0))
    return torch.from_numpy(q.astype(np.int8)), torch.from_numpy(step)
