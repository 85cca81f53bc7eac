"""Attention over texts in 64 bits, word by word from the definition, with bounds for a kernel's error.

The bounds.  u is the half spacing of the type of the rows (2^-24, 2^-11, 2^-8).  A score is a sum of up to 128 products
in fp32: with e = 128 * 2^-24 = 7.7e-6 it is off by at most E = e * scale * sum|q k| + 2^-21 |x| (scaling, bias, base
two, the difference to the maximum), and a weight by a factor of at most 1 + 2 E (numerator and sum).  Weights rounded to the
type add u, sums over words e', the final rounding u |result|:
    |d out| <= (2 E + u + e') sum p |v| + u |out|
    |d p| <= p w, w = 4 E + e' (E again in lse and in the score formed anew)
    |d dS| <= p w (|do| . |v| + |do| . |o|) + p u |do| . |o|, then u |dS| where it is rounded for the products
    |d dq| <= scale sum (|d dS| + (u + e') |dS|) |k| + u |dq|, dk and dv alike, dbias: sum |d dS| + e' |dS|
e' = 2e-5: a sum's terms are added in chains of at most a few hundred before they meet others."""
import math

import torch

ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
E_DOT, E_SUM = 128 * 2.0 ** -24, 2e-5
FAR = 1 << 40


def shown(n, left, right, sinks, skip):
    i, j = torch.arange(n)[:, None], torch.arange(n)[None, :]
    ok = (j <= i + (FAR if right is None else right)) & ((j >= i - (FAR if left is None else left)) | (j < sinks))
    return ok & (i != j) if skip else ok


def attend_reference(q, k, v, offsets, left=None, right=None, sinks=0, skip_self=False, scale=None, keep=None, bias=None,
                     buckets=None, dout=None):
    """Dict of out, lse (and dq, dk, dv, dbias), each with a bound of the same shape under name + "_bound"."""
    ty, u = q.dtype, ROUND[q.dtype]
    T, H, d = q.shape
    G = k.shape[1]
    r = H // G
    scale = d ** -0.5 if scale is None else scale
    z = lambda *s: torch.zeros(*s, dtype=torch.float64)
    res = dict(out=z(T, H, d), out_bound=z(T, H, d), lse=torch.full((H, T), -math.inf, dtype=torch.float64), lse_bound=z(H, T),
               dq=z(T, H, d), dk=z(T, G, d), dv=z(T, G, d), dq_bound=z(T, H, d), dk_bound=z(T, G, d), dv_bound=z(T, G, d))
    if bias is not None:
        res["dbias"], res["dbias_bound"] = z(*bias.shape), z(*bias.shape)
        nb = bias.shape[1]
        table = torch.cat([bias.double(), z(H, 1)], 1)
        span = buckets.numel() // 2
        of = torch.where(buckets.long() < nb, buckets.long(), torch.full_like(buckets.long(), nb))
        of = torch.where(buckets.long() < 0, torch.full_like(of, nb), of)
    for a, b in zip(offsets[:-1], offsets[1:]):
        n = b - a
        if n <= 0:
            continue
        ok = shown(n, left, right, sinks, skip_self)
        if keep is not None:
            ok = ok & (keep[a:b] != 0)[None, :]
        for h in range(H):
            Q, K, V = q[a:b, h].double(), k[a:b, h // r].double(), v[a:b, h // r].double()
            used = ok.any(0)                                    # rows that nobody is shown may hold anything
            K, V = torch.where(used[:, None], K, 0.0), torch.where(used[:, None], V, 0.0)
            x = scale * (Q @ K.T)
            size = scale * (Q.abs() @ K.abs().T)
            if bias is not None:
                dist = (torch.arange(n)[None, :] - torch.arange(n)[:, None]).clamp(-span, span) + span
                x = x + table[h][of[dist]]
            x = torch.where(ok, x, -math.inf)
            m = x.max(1, keepdim=True).values
            m = torch.where(m == -math.inf, 0.0, m)
            e = torch.exp(x - m)
            total = e.sum(1, keepdim=True)
            some = total > 0
            p = torch.where(some, e / torch.where(some, total, 1.0), 0.0)
            o = p @ V
            near = ok & (x > -1e30)                             # (weights of words far below the rest are exactly zero)
            E = torch.where(near, E_DOT * size + 2.0 ** -21 * x.abs(), 0.0).max(1, keepdim=True).values
            res["out"][a:b, h] = o
            res["out_bound"][a:b, h] = (2 * E + u + E_SUM) * (p @ V.abs()) + u * o.abs()
            res["lse"][h, a:b] = torch.where(some, m + torch.log(torch.where(some, total, 1.0)), -math.inf)[:, 0]
            res["lse_bound"][h, a:b] = torch.where(some, 2 * E + E_SUM + 2.0 ** -21 * (m + torch.log(torch.where(some, total, 1.0))).abs(), 0.0)[:, 0]
            if dout is None:
                continue
            g = dout[a:b, h].double()
            delta, size_o = (g * o).sum(1, keepdim=True), (g.abs() * o.abs()).sum(1, keepdim=True)
            ds = p * (g @ V.T - delta)
            err = p * (4 * E + E_SUM) * (g.abs() @ V.abs().T + size_o) + p * u * size_o
            res["dq"][a:b, h] = scale * ds @ K
            rough = err + (u + E_SUM) * ds.abs()
            res["dq_bound"][a:b, h] = scale * rough @ K.abs()
            res["dk"][a:b, h // r] += scale * ds.T @ Q
            res["dk_bound"][a:b, h // r] += scale * rough.T @ Q.abs()
            res["dv"][a:b, h // r] += p.T @ g
            res["dv_bound"][a:b, h // r] += (p * (4 * E + u + E_SUM)).T @ g.abs()
            if bias is not None:
                for c in range(nb):
                    at = of[dist] == c
                    res["dbias"][h, c] += ds[at].sum()
                    res["dbias_bound"][h, c] += (err + E_SUM * ds.abs())[at].sum()
    for name in ("dq", "dk", "dv"):
        res[name + "_bound"] += u * res[name].abs()
    return res


def check(got, res, name, ty=torch.float32):
    """`got` against res[name] within its bound and the type's least step."""
    got, ref = got.double().cpu(), res[name]
    same = got == ref                                           # infinities included
    over = torch.where(same, 0.0, (got - ref).abs() - res[name + "_bound"] - LEAST[ty])
    assert torch.isfinite(over).all() and float(over.max()) <= 0, (name, float(over.max()))
