"""Caches in pages: the words of each text side by side, as the definitions want them."""
import torch


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
