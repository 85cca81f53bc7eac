"""Caches in pages: the words of each text side by side, as the definitions want them, and the newest word's row of attention over
them in 64 bits with the bound that attend_reference derives."""
import math

import torch

from attend_reference import E_DOT, E_SUM, ROUND


def scatter(rows, page_words, slots, seed, extra=2, nobody=0xFFFFFFFF, shared=0):
    """Pools and table for lists of words per text: rows is a list of (k, v), each [n, heads, width].  Pages lie in no order; slots that a text
    does not need are no page.  With ``shared`` the first words of all texts are those of the first one, in its pages; the other
    rows of the table say nothing about them.  Places that no word has hold NaN."""
    g = torch.Generator().manual_seed(seed)
    common = shared // page_words
    need = [max(0 if b else common, -(-k.shape[0] // page_words)) for b, (k, _) in enumerate(rows)]
    order = torch.randperm(sum(need) + extra, generator=g).tolist()
    heads, width, ty = rows[0][0].shape[1], rows[0][0].shape[2], rows[0][0].dtype
    pools = [torch.full((len(order), page_words, heads, width), float("nan")).to(ty) for _ in range(2)]
    table = torch.full((len(rows), slots), nobody, dtype=torch.int64)
    for b, (k, v) in enumerate(rows):
        for i in range(common if b else 0, need[b]):
            page = order.pop()
            table[b, i] = page
            some = k[i * page_words:(i + 1) * page_words].shape[0]
            pools[0][page, :some] = k[i * page_words:i * page_words + some]
            pools[1][page, :some] = v[i * page_words:i * page_words + some]
    return pools[0], pools[1], as_int32(table)


def as_int32(x):
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)


def gather(k_pages, v_pages, table, n, keep=None, shared=0):
    """(k, v, keep, n) as for a cache of one stride from word to word: [texts, room, heads, width], and keep 0 where there is no page."""
    pages, words = k_pages.shape[:2]
    t = table.long() % 2 ** 32
    t = torch.cat([t[:1, :shared // words].expand(t.shape[0], -1), t[:, shared // words:]], 1)
    real = t < pages
    at = torch.where(real, t, 0)
    k, v = [x[at].flatten(1, 2) for x in (k_pages, v_pages)]
    kept = real.repeat_interleave(words, 1).to(torch.uint8)
    return k, v, kept if keep is None else kept & (keep != 0).to(torch.uint8), [min(x, k.shape[1]) for x in n]


def last_rows(q, k, v, n, keep=None, bias=None, buckets=None, left=None, sinks=0, skip_self=False):
    """Dict of out and out_bound [texts, heads, width] over k, v [texts, room, kv_heads, width] of which text b has n[b] words."""
    (B, H, d), G, u = q.shape, k.shape[2], ROUND[q.dtype]
    out, bound = [torch.zeros(B, H, d, dtype=torch.float64, device=q.device) for _ in range(2)]
    for b, m in enumerate(n):
        if m == 0:
            continue
        at = torch.arange(m, device=q.device)
        ok = torch.ones(m, dtype=torch.bool, device=q.device)
        if left is not None:
            ok &= (at >= m - 1 - left) | (at < sinks)
        if skip_self:
            ok &= at != m - 1
        if keep is not None:
            ok &= keep[b, :m] != 0
        K, V = [torch.where(ok[:, None, None], x[b, :m].double(), 0.0).transpose(0, 1).contiguous() for x in (k, v)]
        Q = q[b].double().view(G, H // G, d)
        x = torch.matmul(Q, K.transpose(1, 2).contiguous()).view(H, m) * d ** -0.5
        size = torch.matmul(Q.abs(), K.abs().transpose(1, 2).contiguous()).view(H, m) * d ** -0.5
        if bias is not None:
            span, count = buckets.numel() // 2, bias.shape[1]
            bucket = buckets.long()[span - (m - 1 - at).clamp(max=span)]
            some = (bucket >= 0) & (bucket < count)
            x = x + torch.where(some, bias.double()[:, torch.where(some, bucket, 0)], 0.0)
        x = torch.where(ok, x, -math.inf)
        most = x.amax(1, keepdim=True)
        e = torch.exp(x - torch.where(most == -math.inf, 0.0, most))
        total = e.sum(1, keepdim=True)
        p = torch.where(total > 0, e / torch.where(total > 0, total, 1.0), 0.0).view(G, H // G, m)
        E = torch.where(ok & (x > -1e30), E_DOT * size + 2.0 ** -21 * x.abs(), 0.0).amax(1)[:, None]
        out[b] = torch.matmul(p, V).view(H, d)
        bound[b] = (2 * E + u + E_SUM) * torch.matmul(p, V.abs()).view(H, d) + u * out[b].abs()
    return dict(out=out, out_bound=bound)
