"""The cache in pages: appending with the rotation on the way, and one new word's attention over it, against the definitions in 64 bits
(bounds: rotary_reference, attend_reference)."""
import ctypes
import math

import pytest
import torch

from attend_reference import check
from pages_reference import as_int32, gather, last_rows, scatter
from paper_1606_08495_amd import w2v
from rotary_reference import rotate_reference, within

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- appending ---------------------------------------------------------------------------------------------

def destinations(table, n, off, page_words, n_pages):
    """(token, text, word, page, place) of what is kept."""
    out, t = [], table.long() % 2 ** 32
    for b, count in enumerate(n):
        m = off[b + 1] - off[b]
        for i in range(m):
            word = count - m + i
            if 0 <= word < table.shape[1] * page_words and t[b, word // page_words] < n_pages:
                out.append((off[b] + i, b, word, int(t[b, word // page_words]), word % page_words))
    return out


def run_append(n, off, page_words, slots, H, G, d, r, ty, seed=0, halves=False, gain=1.0, single=False, positions=False, spoil=None):
    g = torch.Generator().manual_seed(seed)
    T, pages = off[-1], len(n) * slots + 3
    q, k, v = [torch.randn(T, h, d, generator=g).to(ty) for h in (H, G, G)]
    pools = [torch.randn(pages, page_words, G, d, generator=g).to(ty) for _ in range(2)]
    table = torch.randperm(pages, generator=g)[:len(n) * slots].view(len(n), slots)
    for b, i, page in spoil or []:
        table[b, i] = page
    table = as_int32(table)
    turns = w2v.rotary_turns(r, device="cpu") if r else None
    at = torch.zeros(T, dtype=torch.int64)
    for b, count in enumerate(n):
        m = off[b + 1] - off[b]
        at[off[b]:off[b + 1]] = torch.arange(count - m, count)
    if positions:
        at = torch.randint(-10 ** 6, 10 ** 6, (T,), generator=g)
    k_pages, v_pages = pools[0].cuda(), pools[1].cuda()
    got = w2v.pages_append(k.cuda(), v.cuda(), k_pages, v_pages, table.cuda(), i32(n), sent_off=None if single else torch.tensor(off).cuda(),
                           turns=turns.cuda() if r else None, positions=at.to(torch.int32).cuda() if positions else None, halves=halves,
                           gain=gain, q=q.cuda() if r else None)
    if r:
        within(got, *rotate_reference(q, at, turns, halves, gain))
        k_to, k_bound = rotate_reference(k, at, turns, halves, gain)
    else:
        k_to, k_bound = k.double(), torch.zeros(k.shape, dtype=torch.float64)
    want, bound = pools[0].double(), torch.zeros(pools[0].shape, dtype=torch.float64)
    for token, _, _, page, place in destinations(table, n, off, page_words, pages):
        want[page, place], bound[page, place] = k_to[token], k_bound[token]
        pools[1][page, place] = v[token]
    within(k_pages, want, bound)
    assert torch.equal(v_pages.cpu(), pools[1])


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d,r", [(1, 1, 2, 2), (5, 5, 60, 60), (8, 2, 128, 128), (4, 1, 100, 50), (6, 2, 37, 36), (3, 3, 33, 0), (16, 8, 64, 0)])
def test_append(H, G, d, r, ty):
    print("append", H, G, d, r, ty, flush=True)
    off = [0, 5, 5, 6, 39, 140]
    for halves in (False, True):
        run_append([5, 9, 30, 40, 130], off, 16, 9, H, G, d, r, ty, halves=halves)
        run_append([64, 0, 1, 33, 101], off, 1, 130, H, G, d, r, ty, halves=halves, gain=0.75)
    run_append([1, 7, 64, 65, 2, 100], [0, 1, 2, 3, 4, 5, 6], 32, 4, H, G, d, r, ty, single=True)
    if r:
        run_append([5, 9, 30, 40, 130], off, 64, 3, H, G, d, r, ty, positions=True)


@pytest.mark.gpu
def test_append_what_has_no_place():
    """Words before the text's first and past its room, numbers that are no page: nothing of them is kept, all else is."""
    off = [0, 5, 9, 40, 41, 60]
    bad = [(2, 1, 0xFFFFFFFF), (2, 2, 23), (4, 0, 0x80000000)]      # 23: one past the pools' last page
    for single in (False, True):
        run_append([3, 34, 30, 0, 19] if not single else [0, 33, 32, 1000, 2 ** 31 - 1], off if not single else [0, 1, 2, 3, 4, 5], 8, 4, 4, 2, 20,
                   20, F32, single=single, spoil=bad)
    pools = [torch.randn(4, 8, 2, 20, device="cuda") for _ in range(2)]
    before = [p.clone() for p in pools]
    k = torch.randn(2, 2, 20, device="cuda")
    w2v.pages_append(k, k, *pools, i32([[0, 1], [2, 3]]), i32([-1, -2 ** 31]))      # 2^32 - 1 and 2^31 words
    assert all(torch.equal(a, b) for a, b in zip(pools, before))
    w2v.pages_append(k[:0], k[:0], *pools, i32([[0, 1], [2, 3]]), i32([3, 3]), sent_off=torch.tensor([0, 0, 0]).cuda())
    assert all(torch.equal(a, b) for a, b in zip(pools, before))


@pytest.mark.gpu
def test_append_many_words_and_rows_no_text_has():
    run_append([2900, 40000 - 2500], [0, 2500, 40000], 256, 150, 2, 1, 16, 16, BF16)
    q, k = torch.randn(30, 3, 12, device="cuda"), torch.randn(30, 1, 12, device="cuda")
    pools, turns = [torch.zeros(6, 8, 1, 12, device="cuda") for _ in range(2)], w2v.rotary_turns(12)
    q_out = torch.full_like(q, 9.0)
    w2v.pages_append(k, k, *pools, i32([[0, 1, 2], [3, 4, 5]]), i32([10, 4]), sent_off=torch.tensor([4, 14, 18]).cuda(), turns=turns, q=q,
                     q_out=q_out)
    assert (q_out[:4] == 9).all() and (q_out[18:] == 9).all() and (q_out[4:18] != 9).all()
    assert torch.equal(pools[1][:2].flatten(0, 1)[:10], k[4:14]) and torch.equal(pools[1][3, :4], k[14:18])
    assert (pools[1][2] == 0).all() and (pools[1][1, 2:] == 0).all() and (pools[1][3, 4:] == 0).all()


@pytest.mark.gpu
def test_append_two_words_to_one_place():
    """Texts that list the same page, and a row of the table that lists one page twice: each element is one of the two words'."""
    k, v = torch.randn(40, 2, 36, device="cuda"), torch.randn(40, 2, 36, device="cuda")
    pools = [torch.zeros(5, 8, 2, 36, device="cuda") for _ in range(2)]
    w2v.pages_append(k, v, *pools, i32([[3, 1, 3], [3, 0, 2]]), i32([20, 20]), sent_off=torch.tensor([0, 20, 40]).cuda())
    for pool, x in zip(pools, (k, v)):
        for place in range(8):
            writers = [place, 20 + place] + ([16 + place] if place < 4 else [])
            assert (pool[3, place][None] == x[writers]).any(0).all()
        assert torch.equal(pool[1], x[8:16]) and torch.equal(pool[0], x[28:36]) and torch.equal(pool[2, :4], x[36:40])
        assert (pool[4] == 0).all() and (pool[2, 4:] == 0).all()
    q = torch.randn(2, 4, 36, device="cuda")                     # read: both texts' words, some twice
    got = w2v.attend_pages(q, *pools, i32([[3, 1, 3], [3, 0, 2]]), i32([20, 20]))
    for b, pages in enumerate(([3, 1, 3], [3, 0, 2])):
        flat = [p[pages].flatten(0, 1)[None] for p in pools]
        want = w2v.attend_step(q[b:b + 1], *flat, i32([20]))
        assert torch.allclose(got[b], want[0], atol=1e-5)


@pytest.mark.gpu
def test_calls_on_two_streams_at_once():
    """Calls that share inputs and nothing else: results and workspaces of their own."""
    words, G, d = 16, 2, 64
    pool = torch.randn(300, words, G, d, device="cuda").to(BF16)
    table, n = torch.randperm(300, device="cuda")[:288].view(4, 72).to(torch.int32), i32([1100, 900, 17, 1152])
    q = torch.randn(4, 8, d, device="cuda").to(BF16)
    want = w2v.attend_pages(q, pool, pool, table, n)
    turns, off = w2v.rotary_turns(64), torch.tensor([0, 4]).cuda()
    turned = w2v.rotate(q, turns, sent_off=off)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i in range(20):
        got.append((w2v.attend_pages(q, pool, pool, table, n, stream=streams[i % 2]), w2v.rotate(q, turns, sent_off=off, stream=streams[1 - i % 2])))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want) and torch.equal(b, turned) for a, b in got)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, BF16])
def test_append_strides_in_place_and_another_stream(ty):
    B, H, G, d, words, pages = 5, 4, 2, 20, 16, 12
    packed = torch.randn(B, H + 2 * G, d, device="cuda").to(ty)
    q, k, v = packed[:, :H], packed[:, H:H + G], packed[:, H + G:]
    table, n, turns = torch.randperm(pages)[:10].view(5, 2).to(torch.int32).cuda(), i32([1, 20, 32, 17, 5]), w2v.rotary_turns(14)
    plain = [torch.zeros(pages, words, G, d, device="cuda", dtype=ty) for _ in range(2)]
    want = w2v.pages_append(k.contiguous(), v.contiguous(), *plain, table, n, turns=turns, q=q.contiguous())
    shapes = [torch.zeros(pages, 2, words, G, d, device="cuda", dtype=ty).unbind(1), torch.zeros(pages, words, 2, G, d, device="cuda", dtype=ty).unbind(2),
              torch.zeros(pages, G, 2, words, d, device="cuda", dtype=ty).permute(2, 0, 3, 1, 4).unbind(0),
              torch.zeros(pages, words, G, 2 * d + 3, device="cuda", dtype=ty)[..., 1:2 * d + 1].split(d, 3)]
    wide = torch.full((5, 7), -1, dtype=torch.int32, device="cuda")
    wide[:, 3:5] = table
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for pools in shapes:
        got = w2v.pages_append(k, v, *pools, wide[:, 3:5], n, turns=turns, q=q, stream=st)
        st.synchronize()
        assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(pools, plain))
    torch.cuda.current_stream().wait_stream(st)
    rest = packed[:, H:].clone()
    assert w2v.pages_append(k, v, *shapes[0], table, n, turns=turns, q=q, q_out=q) is not None
    assert torch.equal(q, want) and torch.equal(packed[:, H:], rest)


# ---- attention ---------------------------------------------------------------------------------------------

def run(n, page_words, H, G, d, ty, seed=0, buckets=None, span=None, drop=0.0, spoil=0.0, shared=0, slots=None, **see):
    g = torch.Generator().manual_seed(seed)
    B, room = len(n), max(max(n), shared, 1)
    slots = slots or -(-room // page_words) + 1
    rows = [tuple(torch.randn(max(m, shared if b == 0 else 0), G, d, generator=g).to(ty) for _ in range(2)) for b, m in enumerate(n)]
    k_pages, v_pages, table = scatter(rows, page_words, slots, seed, shared=shared)
    if spoil:
        table = torch.where(torch.rand(table.shape, generator=g) < spoil, torch.full_like(table, k_pages.shape[0]), table)
    q = torch.randn(B, H, d, generator=g).to(ty)
    bias = torch.randn(H, buckets, generator=g) if buckets else None
    bmap = w2v.relative_buckets(buckets, span, device="cpu") if buckets else None
    keep = (torch.rand(B, slots * page_words, generator=g) >= drop).to(torch.uint8) if drop else None
    k, v, kept, counts = gather(k_pages, v_pages, table, n, keep, shared)
    ref = last_rows(q, k, v, counts, kept, bias, bmap, **see)
    cuda = lambda t: None if t is None else t.cuda()
    out = w2v.attend_pages(q.cuda(), k_pages.cuda(), v_pages.cuda(), table.cuda(), i32(n), shared=shared, keep=cuda(keep), bias=cuda(bias),
                           buckets=cuda(bmap), **see)
    check(out, ref, "out", ty)


HEADS = [(1, 1, 64), (5, 5, 60), (4, 2, 128), (6, 2, 37), (8, 2, 33), (5, 1, 100), (8, 1, 128), (9, 1, 16), (34, 2, 64), (40, 1, 128), (2, 2, 1),
         (4, 1, 127), (33, 1, 31)]


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d", HEADS)
def test_heads_and_widths(H, G, d, ty):
    print("pages", H, G, d, ty, flush=True)
    run([1, 0, 7, 300], 16, H, G, d, ty)
    run([255, 256, 257, 2, 700, 31], 32, H, G, d, ty, left=100, sinks=4, buckets=8, span=20, drop=0.3, spoil=0.2)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d", HEADS)
def test_heads_and_widths_behind_a_prefix(H, G, d, ty):
    print("prefix", H, G, d, ty, flush=True)
    run([161, 200, 500, 160], 16, H, G, d, ty, shared=160)
    run([700, 3, 0, 650, 640, 1000], 64, H, G, d, ty, shared=640)
    run([255, 256, 257, 2, 700, 31], 32, H, G, d, ty, left=100, sinks=4, buckets=8, span=20, drop=0.3, spoil=0.2, shared=224)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, BF16])
@pytest.mark.parametrize("page_words", [1, 2, 8, 64, 128, 4096])
def test_sizes_of_pages(page_words, ty):
    print("pages of", page_words, ty, flush=True)
    run([1, 2, 63, 64, 65, 900, 4097], page_words, 4, 2, 60, ty, spoil=0.1)
    run([1, 200, 4096, 4500], page_words, 4, 2, 60, ty, shared=4096)
    run([1, 2, 3 * page_words, 3 * page_words + 1], page_words, 2, 2, 32, ty, shared=2 * page_words)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16])
@pytest.mark.parametrize("shared", [0, 64, 1984])
@pytest.mark.parametrize("see", [dict(), dict(left=0), dict(left=0, skip_self=True), dict(skip_self=True), dict(left=5, sinks=64),
                                 dict(left=300, sinks=1), dict(left=1800, sinks=7), dict(left=5000, sinks=7)])
def test_windows(see, shared, ty):
    print("pages", see, shared, ty, flush=True)
    for group in (1, 4):
        run([1, 2, 63, 64, 65, 2000, 1999], 64, 2 * group, 2, 64, ty, shared=shared, **see)
        run([1, 2, 63, 64, 65, 2000, 2048], 16, 2 * group, 2, 64, ty, drop=0.9, buckets=32, span=128, spoil=0.1, shared=shared, slots=128, **see)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("batch,H,G", [(1, 4, 1), (2, 1, 1), (7, 3, 1), (33, 4, 2), (70, 8, 2), (130, 2, 2)])
def test_many_texts_behind_a_prefix(batch, H, G, ty):
    """Rows of queries that fill one tile of the prefix's product, several, or little of one."""
    print("prefix", batch, H, G, ty, flush=True)
    g = torch.Generator().manual_seed(batch)
    run([1344 + x for x in torch.randint(0, 90, (batch,), generator=g).tolist()], 64, H, G, 40, ty, shared=1344)
    run([1300 + x for x in torch.randint(0, 90, (batch,), generator=g).tolist()], 32, H, G, 128, ty, shared=1344, left=700, sinks=9, drop=0.2,
        buckets=16, span=60)


@pytest.mark.gpu
@pytest.mark.parametrize("shared", [0, 96])
def test_no_words_at_all(shared):
    """Texts of none, tables of no page, everything dropped, a window that shows the word itself alone without itself: zeros."""
    B, H, d = 3, 4, 24
    q, pool = torch.randn(B, H, d, device="cuda"), torch.full((20, 32, 2, d), float("nan"), device="cuda")
    table = torch.arange(18, dtype=torch.int32, device="cuda").view(3, 6)
    zero = torch.zeros_like(q)
    assert torch.equal(w2v.attend_pages(q, pool, pool, table, i32([0, 0, 0]), shared=shared), zero)
    assert torch.equal(w2v.attend_pages(q, pool, pool, torch.full_like(table, -1), i32([190, 1, 97]), shared=shared), zero)
    assert torch.equal(w2v.attend_pages(q, pool, pool, table, i32([190, 1, 97]), shared=shared, left=0, skip_self=True), zero)
    keep = torch.zeros(3, 192, dtype=torch.uint8, device="cuda")
    assert torch.equal(w2v.attend_pages(q, pool, pool, table, i32([190, 1, 97]), shared=shared, keep=keep), zero)
    assert w2v.attend_pages(q[:0], pool, pool, table[:0], i32([])).shape == (0, H, d)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d", [(1, 1, 60), (5, 5, 60), (4, 2, 100), (8, 1, 128), (2, 2, 37), (2, 1, 3), (9, 1, 66), (3, 3, 124)])
@pytest.mark.parametrize("shared", [0, 640])
def test_infinities_that_do_not_show(shared, H, G, d, ty):
    """Keys and values that are not shown (dropped, on no page's slots, behind the text), and shown keys of score -infinity, may hold anything."""
    words, n = 32, [900, 660, 640, 300, 41]
    rows = [tuple(torch.randn(max(m, 640 if b == 0 else 0), G, d).to(ty) for _ in range(2)) for b, m in enumerate(n)]
    k, v, table = [x.cuda() for x in scatter(rows, words, 30, 3, shared=shared)]
    q = torch.randn(5, H, d, device="cuda").to(ty)
    q[..., 0] = 1.0
    keep = torch.ones(5, 960, dtype=torch.uint8, device="cuda")
    hidden = [7, 39, 256, 299, 620, 645, 700]
    keep[:, hidden] = 0
    clean = [torch.nan_to_num(x) for x in (k, v)]
    want = w2v.attend_pages(q, *clean, table, i32(n), keep=keep, shared=shared)
    assert torch.isfinite(want).all()
    assert torch.equal(w2v.attend_pages(q, k, v, table, i32(n), keep=keep, shared=shared), want)      # NaN where no word is
    at = table.long() % 2 ** 32
    for b in range(5):
        for word in hidden:
            page = int(at[0 if word < shared else b, word // words])
            if page < k.shape[0]:
                k[page, word % words, :, 0], v[page, word % words] = float("-inf"), float("inf")
    tol = {F32: 1e-5, F16: 4e-3, BF16: 3e-2}[ty]
    got = w2v.attend_pages(q, k, v, table, i32(n), keep=keep, shared=shared)
    assert torch.allclose(got.float(), want.float(), atol=tol)
    got = w2v.attend_pages(q, k, v, table, i32(n), shared=shared)                                     # scores of -infinity
    assert torch.allclose(got.float(), want.float(), atol=tol)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
def test_infinities_that_some_texts_see(ty):
    """A prefix whose late value is infinite: texts whose window shows it have it, the others do not."""
    words, shared, n = 16, 512, [520, 600, 700, 515, 560]
    rows = [tuple(torch.randn(m, 2, 40).to(ty) for _ in range(2)) for m in n]
    k, v, table = [x.cuda() for x in scatter(rows, words, 44, 5, shared=shared)]
    q = torch.randn(5, 6, 40, device="cuda").to(ty)
    want = w2v.attend_pages(q, k, v, table, i32(n), shared=shared, left=60)
    v[int(table[0, 500 // words]), 500 % words, 1, 3] = float("inf")
    k[int(table[0, 470 // words]), 470 % words, 0, 5] = float("nan")
    got = w2v.attend_pages(q, k, v, table, i32(n), shared=shared, left=60)
    sees = torch.zeros(5, 6, 40, dtype=torch.bool, device="cuda")
    sees[[0, 3, 4], 3:, 3] = True                # words 500 and on: n - 1 - 60 <= 500
    sees[[0, 3], :3] = True                      # 470: every column of the heads that read it
    finite = torch.isfinite(got)
    assert torch.equal(finite, ~sees)
    assert torch.allclose(got[finite].float(), want[finite].float(), atol={F32: 1e-5, F16: 4e-3, BF16: 3e-2}[ty])
    assert (got[[0, 3, 4], 3:, 3] == float("inf")).all() and torch.isnan(got[[0, 3], :3]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
def test_large_scores_and_masks_of_the_lowest_value(ty):
    """Biases of -infinity and fp32's lowest, scores in the hundreds: against the cache of one stride from word to word."""
    n, words, shared = [700, 350, 333], 16, 320
    rows = [tuple(torch.randn(m, 2, 48).to(ty) for _ in range(2)) for m in n]
    k, v, table = [x.cuda() for x in scatter(rows, words, 44, 9, shared=shared)]
    q = (torch.randn(3, 4, 48, device="cuda") * 30).to(ty)
    bmap = w2v.relative_buckets(32, 200)
    flat = gather(k.cpu(), v.cpu(), table.cpu(), n, None, shared)
    flat = [torch.nan_to_num(x).cuda() for x in flat[:2]]
    for low in (-math.inf, torch.finfo(F32).min, -1e9, 1e9):
        bias = torch.randn(4, 32, device="cuda")
        bias[:, 3] = low
        bias[1] = low
        want = w2v.attend_step(q, *flat, i32(n), bias=bias, buckets=bmap)
        for s in (0, shared):
            if s == 0:
                t = table.clone()
                t[1:, :shared // words] = table[0, :shared // words]
            got = w2v.attend_pages(q, k, v, t if s == 0 else table, i32(n), shared=s, bias=bias, buckets=bmap)
            # scores of up to 400: off by 2^-24 of that a product's sum and scale (and by a bias of 1e9's own rounding, which both share)
            tol = {F32: 2e-3, F16: 4e-3, BF16: 3e-2}[ty]
            assert torch.allclose(got.float(), want.float(), atol=tol, rtol=tol), (low, s)


@pytest.mark.gpu
def test_strides_in_place_and_another_stream():
    B, H, G, d, words, pages = 4, 4, 2, 60, 16, 70
    n = i32([200, 150, 1, 260])
    table = torch.full((4, 30), -1, dtype=torch.int32, device="cuda")
    table[:, :17] = torch.randperm(pages, device="cuda")[:68].view(4, 17).to(torch.int32)
    layouts = [torch.randn(pages, 2, words, G, d, device="cuda").unbind(1), torch.randn(pages, words, G, 2 * d + 1, device="cuda")[..., :2 * d].split(d, 3),
               torch.randn(2, G, pages, words, d + 3, device="cuda").permute(0, 2, 3, 1, 4)[..., :d].unbind(0)]
    q = torch.randn(B, 3 * H, d, device="cuda")[:, ::3]
    for k, v in layouts:
        for shared in (0, 128):
            see = dict(left=120, sinks=3, shared=shared)
            want = w2v.attend_pages(q.contiguous(), k.contiguous(), v.contiguous(), table, n, **see)
            st = torch.cuda.Stream()
            st.wait_stream(torch.cuda.current_stream())
            got = w2v.attend_pages(q, k, v, table[:, :17], n, stream=st, **see)
            st.synchronize()
            assert torch.equal(got, want)
            x = q.clone()
            assert w2v.attend_pages(x, k, v, table, n, out=x, **see) is x and torch.equal(x, want)


@pytest.mark.gpu
def test_pools_past_32_bit_offsets():
    pages, words, G, d = 90_000, 256, 2, 64                               # 2.95e9 elements a pool
    k = torch.zeros(pages, words, G, d, dtype=F16, device="cuda")
    q = torch.randn(2, 4, d, device="cuda").to(F16)
    far = torch.tensor([89_999, 70_001, 89_990, 12], device="cuda")
    k[far] = torch.randn(4, words, G, d, device="cuda").to(F16)
    near = k[far].contiguous()
    n = i32([500, 400])
    for shared in (0, 256):
        got = w2v.attend_pages(q, k, k, far.view(2, 2).to(torch.int32), n, shared=shared)
        assert torch.equal(got, w2v.attend_pages(q, near, near, i32([[0, 1], [2, 3]]), n, shared=shared))
    turns = w2v.rotary_turns(64)
    x = torch.randn(2, G, d, device="cuda").to(F16)
    w2v.pages_append(x, x, k, torch.zeros_like(k), far.view(2, 2).to(torch.int32), n, turns=turns)
    v_near = torch.zeros_like(near)
    w2v.pages_append(x, x, near, v_near, i32([[0, 1], [2, 3]]), n, turns=turns)
    assert torch.equal(k[far], near)


@pytest.mark.gpu
def test_captured_and_replayed():
    """A server's step in a graph, replayed with other words, tables and counts; eager calls between."""
    B, H, G, d, words = 6, 4, 2, 64, 16
    pools = [torch.randn(60, words, G, d, device="cuda").to(BF16) for _ in range(2)]
    table, n = torch.randperm(60, device="cuda")[:54].view(6, 9).to(torch.int32), i32([1, 20, 140, 65, 64, 100])
    turns = w2v.rotary_turns(64)
    q, k, v = [torch.randn(B, h, d, device="cuda").to(BF16) for h in (H, G, G)]
    out, q_out = torch.empty_like(q), torch.empty_like(q)
    for shared in (0, 48):
        workspace = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

        def step(p, out, q_out, **kw):
            w2v.pages_append(k, v, *p, table, n, turns=turns, q=q, q_out=q_out)
            w2v.attend_pages(q_out, *p, table, n, shared=shared, out=out, **kw)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            step(pools, out, q_out, workspace=workspace)
        torch.cuda.current_stream().wait_stream(st)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(pools, out, q_out, workspace=workspace)
        for _ in range(4):
            for x in (q, k, v):
                x.normal_()
            n.copy_(torch.randint(1, 145, (B,), device="cuda"))
            table.copy_(torch.randperm(60, device="cuda")[:54].view(6, 9))
            other = [p.clone() for p in pools]
            graph.replay()
            want, want_q = torch.empty_like(q), torch.empty_like(q)
            step(other, want, want_q)
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(q_out, want_q) and all(torch.equal(a, b) for a, b in zip(pools, other))


@pytest.mark.gpu
@pytest.mark.parametrize("ty,tol", [(F32, 2e-5), (F16, 6e-3), (BF16, 5e-2)])
@pytest.mark.parametrize("halves", [False, True])
def test_prompts_and_steps_give_the_rows_of_the_whole_text(halves, ty, tol):
    """All of it together, as a server has it: two texts with one opening; the opening is turned, attended and appended as a prompt, the rest
    of each text word by word.  Every word's row is that of attention over the whole text.  (In 16 bits the turned rows are the same bits on
    both ways; weights and results are rounded on each, 4 u sum p |v| with sums below 2: 4e-3 and 3.2e-2.  In 32 bits a score of 60
    products of about 1 is off by some 2^-24 8 on either way, its weight by twice that, the row by the same of |v|: 2e-6.)"""
    H, G, d, words, opening, lens = 4, 2, 60, 16, 48, [70, 61]
    turned = dict(turns=w2v.rotary_turns(40, scaling="base", factor=4.0), halves=halves)
    x = [[torch.randn(m, h, d, device="cuda").to(ty) for h in (H, G, G)] for m in lens]
    for b in range(3):
        x[1][b][:opening] = x[0][b][:opening]
    whole = []
    for (q, k, v), m in zip(x, lens):
        off = torch.tensor([0, m]).cuda()
        whole.append(w2v.attend(*w2v.rotate(q, k=k, sent_off=off, **turned), v, off, right=0)[0])
    pools = [torch.full((12, words, G, d), float("nan"), device="cuda").to(ty) for _ in range(2)]
    table = i32([[7, 1, 4, 0, 9], [7, 1, 4, 11, -1]])
    n = i32([opening, 0])
    off = torch.tensor([0, opening, opening]).cuda()
    first = [y[:opening] for y in x[0]]
    q = w2v.pages_append(first[1], first[2], *pools, table, n, sent_off=off, q=first[0], **turned)
    assert torch.equal(q, w2v.rotate(first[0], sent_off=off, **turned))
    n[1] = opening
    for i in range(opening, min(lens)):
        n.add_(1)
        q, k, v = [torch.stack([x[b][c][i] for b in range(2)]) for c in range(3)]
        w2v.pages_append(k, v, *pools, table, n, q=q, q_out=q, **turned)
        for shared in (0, opening):
            got = w2v.attend_pages(q, *pools, table, n, shared=shared)
            for b in range(2):
                assert torch.allclose(got[b].float(), whole[b][i].float(), atol=tol), (i, b, shared)


# ---- what is refused ---------------------------------------------------------------------------------------

def test_refusals_of_append():
    L, p, r = w2v.lib(), 1 << 24, ctypes.byref
    T, H, G, d = 6, 4, 2, 64

    def call(type=0, width=d, rotary=True, rotated=64, gain=1.0, k=None, v=None, kv_heads=G, q=None, heads=H, q_out=None, off=p, n_sent=3, tokens=T,
             n=p, table=p, stride=8, slots=8, words=16, pages=100, kp=None, vp=None, no_q=False, no_table=False):
        k, v, q, q_out = k or w2v.Heads(p, G * d, d), v or w2v.Heads(2 * p, G * d, d), q or w2v.Heads(3 * p, H * d, d), q_out or w2v.Heads(4 * p, H * d, d)
        kp, vp = kp or w2v.Pages(5 * p, 16 * G * d, G * d, d), vp or w2v.Pages(6 * p, 16 * G * d, G * d, d)
        return L.w2v_pages_append(type, width, r(w2v.Rotary(rotated, 0, gain, p)) if rotary else None, r(k), r(v), kv_heads, None if no_q else r(q),
                                  heads, r(q_out), off, n_sent, tokens, n, None, None if no_table else r(w2v.PageTable(table, stride, slots, words, pages)),
                                  r(kp), r(vp), None)
    assert call(tokens=0) == 0
    one = 16 * G * d
    for bad in (dict(type=-1), dict(width=130), dict(kv_heads=0), dict(heads=0), dict(heads=2000), dict(rotated=5), dict(gain=math.nan), dict(rotary=False),
                dict(n_sent=0), dict(off=None, n_sent=5), dict(tokens=0x7FFFFFFF), dict(table=p + 2), dict(words=0), dict(words=24), dict(words=8192),
                dict(slots=0), dict(slots=1 << 30), dict(pages=0), dict(stride=1 << 41), dict(k=w2v.Heads(p + 1, G * d, d)),
                dict(kp=w2v.Pages(5 * p + 2, one, G * d, d)), dict(kp=w2v.Pages(5 * p, 1 << 41, G * d, d)), dict(kp=w2v.Pages(5 * p, one - 1, G * d, d)),
                dict(kp=w2v.Pages(5 * p, 0, G * d, d)), dict(kp=w2v.Pages(5 * p, one, G * d, d - 1)), dict(kp=w2v.Pages(6 * p, one, G * d, d)),
                dict(kp=w2v.Pages(6 * p + 4 * one * 99, one, G * d, d)), dict(kp=w2v.Pages(p, one, G * d, d)), dict(kp=w2v.Pages(3 * p, one, G * d, d)),
                dict(q_out=w2v.Heads(3 * p + 4, H * d, d)), dict(q_out=w2v.Heads(p, H * d, d)), dict(q_out=w2v.Heads(2 * p, H * d, d)),
                dict(q_out=w2v.Heads(5 * p + 400, H * d, d)), dict(q_out=w2v.Heads(4 * p, H * d - 1, d))):
        assert call(**bad) == -2, bad
    for bad in (dict(n=None), dict(table=None), dict(no_table=True), dict(k=w2v.Heads(None, 1, 1)), dict(vp=w2v.Pages(None, 1, 1, 1)),
                dict(q_out=w2v.Heads(None, 1, 1))):
        assert call(**bad) == -1, bad


def test_refusals_of_attention():
    L, p, r = w2v.lib(), 1 << 24, ctypes.byref
    ok = dict(type=0, heads=4, kv_heads=2, width=64, left=0xFFFFFFFF, right=0, sinks=0, skip_self=0, scale=0.1)

    def call(batch=3, shared=0, n=p, q=None, k=None, out=None, table=p, stride=2000, slots=2000, words=16, pages=7000, ws=p, size=1 << 30, no_table=False,
             **kw):
        spec, q, out = w2v.AttendSpec(**{**ok, **kw}), q or w2v.Heads(p, 256, 64), out or w2v.Heads(2 * p, 256, 64)
        t = w2v.PageTable(table, stride, slots, words, pages)
        k, v = k or w2v.Pages(300 * p, 2048, 128, 64), w2v.Pages(600 * p, 2048, 128, 64)
        return L.w2v_attend_pages(r(spec), r(q), r(k), r(v), None if no_table else r(t), shared, n, batch, None, r(out), ws, size, None)
    assert call(batch=0) == 0
    for bad in (dict(width=200), dict(heads=3), dict(sinks=65), dict(scale=-1.0), dict(batch=1 << 24), dict(shared=8), dict(shared=32016), dict(words=48),
                dict(words=0), dict(slots=0), dict(pages=0), dict(table=p + 1), dict(k=w2v.Pages(300 * p + 2, 2048, 128, 64)),
                dict(k=w2v.Pages(300 * p, 1 << 58, 128, 64)), dict(out=w2v.Heads(p + 4, 256, 64)), dict(out=w2v.Heads(300 * p + 4096, 256, 64)),
                dict(out=w2v.Heads(2 * p, 256, 63)), dict(ws=p + 4), dict(size=8), dict(shared=3200, size=8)):
        assert call(**bad) == -2, bad
    for bad in (dict(n=None), dict(table=None), dict(no_table=True), dict(q=w2v.Heads(None, 1, 1)), dict(k=w2v.Pages(None, 1, 1, 1)), dict(ws=None)):
        assert call(**bad) == -1, bad
    spec, t = w2v.AttendSpec(**ok), w2v.PageTable(p, 2000, 2000, 16, 7000)
    assert L.w2v_attend_pages_workspace(r(spec), 3, r(t), 0) > 0 and L.w2v_attend_pages_workspace(r(spec), 3, r(t), 8) == 0
    assert L.w2v_attend_pages_workspace(r(spec), 0, r(t), 0) == 0 and L.w2v_attend_pages_workspace(r(spec), 3, None, 0) == 0


def test_refusals_of_the_binding():
    q, pool, n = torch.zeros(2, 2, 8), torch.zeros(4, 8, 1, 8), torch.zeros(2, dtype=torch.int32)
    for table in (torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int64), None):
        with pytest.raises((TypeError, ValueError)):
            w2v.attend_pages(q, pool, pool, table, n)
        with pytest.raises((TypeError, ValueError)):
            w2v.pages_append(q[:, :1], q[:, :1], pool, pool, table, n)
    for bad in (dict(q=q), dict(positions=n), dict(q_out=q)):
        with pytest.raises(ValueError):
            w2v.pages_append(q[:, :1], q[:, :1], pool, pool, n, n, **bad)


@pytest.mark.gpu
@pytest.mark.parametrize("H,G,ty", [(8, 1, F32), (16, 2, F32), (9, 1, F32), (8, 1, F16), (2, 2, BF16)])
def test_the_widest_bias(H, G, ty):
    """As many distances as there may be, for eight heads of 128 columns a block: more than 64 KB of LDS."""
    print("pages", H, G, ty, flush=True)
    run([300, 1500, 1, 0], 16, H, G, 128, ty, buckets=64, span=1023)
    run([300, 400], 16, H, G, 128, ty, buckets=1024, span=1023)
