"""One new word per text behind a common prefix that is large enough for blocks of its own on the matrix cores (128 MB more to read
if every text read it), against the definition in 64 bits (bounds: attend_reference)."""
import ctypes
import math

import pytest
import torch

from attend_reference import E_SUM, ROUND, check
from pages_reference import gather, last_rows
from paper_1606_08495_amd import w2v

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
MORE = 128 << 20


def shape_of(G, d, ty, batch):
    """Words of a prefix in pages of 64 that is taken by its own blocks."""
    words = -(-MORE // ((batch - 1) * G * d * 2 * torch.finfo(ty).bits // 8))
    return -(-words // 64) * 64


def parts(batch, H, G, d, ty, table, words, pages, shared, left=None):
    """Into how many a row is split."""
    q = torch.empty(batch, H, d, dtype=ty, device="cuda")
    spec = w2v._spec(q, G, left, 0, 0, False, None, None, None)
    t = w2v.PageTable(4096, table.shape[1], table.shape[1], words, pages)
    return w2v.lib().w2v_attend_pages_workspace(ctypes.byref(spec), batch, ctypes.byref(t), shared) // (batch * H * (d + 2) * 4)


class Texts:
    """Texts of n words in a pool of pages in no order; the first `shared` words in the pages of row 0, places without a word NaN."""

    def __init__(self, n, shared, H, G, d, ty, words=64, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        B, common = len(n), shared // words
        need = [max(0, -(-x // words) - common) for x in n]
        order = torch.randperm(common + sum(need) + 2, generator=g, device="cuda").tolist()
        self.k, self.v = [torch.empty(len(order), words, G, d, device="cuda").normal_(generator=g).to(ty) for _ in range(2)]
        slots = common + max(need) + 1
        table = torch.full((B, slots), -1, dtype=torch.int32)
        table[0, :common] = torch.tensor([order.pop() for _ in range(common)])
        for b, m in enumerate(need):
            if m:
                own = [order.pop() for _ in range(m)]
                table[b, common:common + m] = torch.tensor(own)
                if n[b] % words:
                    for x in (self.k, self.v):
                        x[own[-1], n[b] % words:] = float("nan")
        self.table, self.n, self.shared, self.words, self.H = table.cuda(), n, shared, words, H
        self.q = torch.empty(B, H, d, device="cuda").normal_(generator=g).to(ty)

    def call(self, **see):
        assert parts(len(self.n), self.H, *self.k.shape[2:], self.q.dtype, self.table, self.words, self.k.shape[0], self.shared) > \
            parts(len(self.n), self.H, *self.k.shape[2:], self.q.dtype, self.table, self.words, self.k.shape[0], 0, left=0), "no blocks of its own"
        return w2v.attend_pages(self.q, self.k, self.v, self.table, i32(self.n), shared=self.shared, **see)

    def check(self, got, keep=None, **see):
        k, v, kept, n = gather(self.k, self.v, self.table, self.n, keep, self.shared)
        ref = last_rows(self.q, k, v, n, kept, **see)
        check(got, {name: x.cpu() for name, x in ref.items()}, "out", self.q.dtype)


def lengths(batch, shared, seed=0):
    """Some texts end in the prefix, one has no words, the others go on behind it."""
    g = torch.Generator().manual_seed(seed)
    n = (shared + torch.randint(0, 300, (batch,), generator=g)).tolist()
    if batch > 4:
        n[1], n[2], n[batch - 1] = 0, shared // 2 + 5, shared
    return n


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d,batch", [(1, 1, 64, 130), (5, 5, 60, 24), (4, 2, 128, 9), (6, 2, 37, 40), (8, 2, 33, 16), (5, 1, 100, 30), (8, 1, 128, 20),
                                         (9, 1, 16, 200), (34, 2, 64, 7), (40, 1, 128, 6), (2, 2, 1, 1000), (4, 1, 127, 65), (33, 1, 31, 64), (8, 8, 96, 2)])
def test_heads_and_widths(H, G, d, batch, ty):
    """Widths of every kind; 24 to 2000 queries for a key head: part of a block's rows, all of them, several blocks."""
    shared = shape_of(G, d, ty, batch)
    print("prefix", H, G, d, batch, shared, ty, flush=True)
    t = Texts(lengths(batch, shared), shared, H, G, d, ty)
    t.check(t.call())


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("see", [dict(left=0), dict(skip_self=True), dict(left=5, sinks=64), dict(left=300, sinks=1), dict(left=2000, sinks=7),
                                 dict(left=100_000), dict(left=0, skip_self=True)])
def test_windows_masks_and_bias(see, ty):
    H, G, d, batch = 6, 2, 64, 40
    shared = shape_of(G, d, ty, batch)
    print("prefix", see, shared, ty, flush=True)
    t = Texts(lengths(batch, shared, 1), shared, H, G, d, ty, words=16, seed=1)
    t.check(t.call(**see), **see)
    see = dict(see, bias=torch.randn(H, 32, device="cuda"), buckets=w2v.relative_buckets(32, 128),
               keep=(torch.rand(batch, t.table.shape[1] * 16, device="cuda") > 0.6).to(torch.uint8))
    t.table[0, 3::7] = t.k.shape[0]               # numbers that are no page, in the prefix and behind it
    t.table[5::2, -3] = -1
    t.check(t.call(**see), **see)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d,batch", [(4, 2, 60, 40), (2, 2, 128, 12), (6, 1, 37, 70)])
def test_infinities_that_do_not_show(H, G, d, batch, ty):
    shared = shape_of(G, d, ty, batch)
    t = Texts(lengths(batch, shared, 2), shared, H, G, d, ty, seed=2)
    t.q[..., 0] = 1.0
    hidden = [7, 39, 256, shared - 1, shared + 3]
    keep = torch.ones(batch, t.table.shape[1] * 64, dtype=torch.uint8, device="cuda")
    keep[:, hidden] = 0
    want = t.call(keep=keep)
    t.check(want, keep=keep)
    for b in range(batch):
        for word in hidden:
            page = int(t.table[0 if word < shared else b, word // 64])
            if page >= 0:
                t.k[page, word % 64, :, 0], t.v[page, word % 64] = float("-inf"), float("inf")
    tol = {F32: 1e-5, F16: 4e-3, BF16: 3e-2}[ty]
    some = torch.tensor(t.n, device="cuda") > 0
    for got in (t.call(keep=keep), t.call()):                 # dropped; shown with a score of -infinity
        assert torch.allclose(got.float()[some], want.float()[some], atol=tol)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
def test_infinities_that_some_texts_see(ty):
    H, G, d, batch, left = 6, 2, 40, 60, 900
    shared = shape_of(G, d, ty, batch)
    n = [shared + 10 * b for b in range(batch)]
    t = Texts(n, shared, H, G, d, ty, seed=3)
    want = t.call(left=left)
    far, near = shared - 700, shared - 500                     # seen while n - 1 - left is not past them
    t.v[int(t.table[0, near // 64]), near % 64, 1, 3] = float("inf")
    t.k[int(t.table[0, far // 64]), far % 64, 0, 5] = float("nan")
    got = t.call(left=left)
    sees = torch.zeros(batch, H, d, dtype=torch.bool, device="cuda")
    last = torch.tensor(n, device="cuda") - 1
    sees[last - left <= near, 3:, 3] = True
    sees[last - left <= far, :3] = True
    assert sees.any() and not sees.all(2).all(1).any()
    assert torch.equal(torch.isfinite(got), ~sees)
    assert torch.allclose(got[~sees].float(), want[~sees].float(), atol={F32: 1e-5, F16: 4e-3, BF16: 3e-2}[ty])
    infinite, nan = got[:, 3:, 3][sees[:, 3:, 3]], got[:, :3][sees[:, :3]]
    assert (infinite == float("inf")).all() and torch.isnan(nan).all()


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
def test_large_scores_and_masks_of_the_lowest_value(ty):
    """Against the same words read as they are, without blocks of the prefix's own; see test_gpu_pages for the tolerance."""
    H, G, d, batch = 4, 2, 64, 40
    shared = shape_of(G, d, ty, batch)
    t = Texts([shared + x for x in range(batch)], shared, H, G, d, ty, seed=4)
    t.q = (t.q.float() * 30).to(ty)
    whole = t.table.clone()
    whole[:, :shared // 64] = t.table[0, :shared // 64]
    bmap = w2v.relative_buckets(32, 200)
    for low in (-math.inf, torch.finfo(F32).min, -1e9):
        bias = torch.randn(H, 32, device="cuda")
        bias[:, 15] = low                                      # the outermost bucket: all of the prefix but its end
        bias[1] = low
        want = w2v.attend_pages(t.q, t.k, t.v, whole, i32(t.n), bias=bias, buckets=bmap)
        tol = {F32: 2e-3, F16: 4e-3, BF16: 3e-2}[ty]
        assert torch.allclose(t.call(bias=bias, buckets=bmap).float(), want.float(), atol=tol, rtol=tol), low


@pytest.mark.gpu
def test_strides_streams_and_graphs():
    """Pools side by side in one buffer, another stream, a workspace of the caller's, a graph replayed with other words: the same bits."""
    H, G, d, batch, ty = 8, 2, 64, 33, BF16
    shared = shape_of(G, d, ty, batch)
    t = Texts(lengths(batch, shared, 5), shared, H, G, d, ty, words=16, seed=5)
    want = t.call()
    both = torch.stack([t.k, t.v], 2)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = w2v.attend_pages(t.q, both[:, :, 0], both[:, :, 1], t.table, i32(t.n), shared=shared, stream=st)
    st.synchronize()
    assert torch.equal(got, want)
    n, x, out = i32(t.n), t.q.clone(), torch.empty_like(t.q)
    assert torch.equal(w2v.attend_pages(x, t.k, t.v, t.table, n, shared=shared, out=x), want)
    x.copy_(t.q)
    workspace = torch.full((1 << 26,), 0xFF, dtype=torch.uint8, device="cuda")
    call = lambda: w2v.attend_pages(x, t.k, t.v, t.table, n, shared=shared, out=out, workspace=workspace)
    call()
    assert torch.equal(out, want)
    with torch.cuda.stream(st):
        call()
    torch.cuda.current_stream().wait_stream(st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        x.normal_()
        n.copy_(torch.randint(0, shared + 200, (batch,), device="cuda"))
        workspace.fill_(0xFF)                                  # NaN
        graph.replay()
        got = out.clone()
        want = w2v.attend_pages(x, t.k, t.v, t.table, n, shared=shared)
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))      # (texts that reach into places without a word: NaN)
        assert torch.isfinite(got).any(2).any(1).sum() > batch // 2


@pytest.mark.gpu
def test_pools_past_32_bit_offsets():
    pages, words, G, d, batch = 90_000, 256, 2, 64, 40
    k = torch.zeros(pages, words, G, d, dtype=F16, device="cuda")
    shared = -(-shape_of(G, d, F16, batch) // words) * words
    far = pages - 1 - torch.randperm(shared // words + batch, device="cuda")
    k[far] = torch.randn(far.numel(), words, G, d, device="cuda").to(F16)
    near = k[far].contiguous()
    table = torch.zeros(batch, shared // words + 1, dtype=torch.int32, device="cuda")
    table[0, :-1] = torch.arange(shared // words, device="cuda")
    table[:, -1] = shared // words + torch.arange(batch, device="cuda")
    q, n = torch.randn(batch, 8, d, device="cuda").to(F16), i32([shared + 1 + 6 * b for b in range(batch)])
    assert parts(batch, 8, G, d, F16, table, words, pages, shared) > parts(batch, 8, G, d, F16, table, words, pages, 0, left=0)
    want = w2v.attend_pages(q, near, near, table, n, shared=shared)
    assert torch.equal(w2v.attend_pages(q, k, k, far[table.long()].to(torch.int32), n, shared=shared), want)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d,batch", [(4, 2, 128, 9), (5, 1, 100, 10), (33, 1, 31, 64), (6, 2, 37, 40), (8, 2, 64, 40), (12, 3, 96, 50), (8, 1, 128, 40)])
def test_weights_keep_their_bits(H, G, d, batch, ty):
    """18 to 2112 queries for a key head.  All words of one parity have one score and one value, so that what a weight's rounding takes away
    is the same for thousands of words and adds up, while the results of some columns are near zero.

    The bound.  A score is a single product, exact in fp32, times scale: off by 2^-21 |x| with all that follows (attend_reference).  A weight is
    the sum of two numbers of the type, of which the second is off by u of itself and at most u of the weight: u^2.  Sums: e'.  So
    |d out| <= (2 2^-21 |x| + u^2 + e') sum p |v| + u |out|; one number of the type for a weight would be off by some u / 4 sum p |v|."""
    shared = shape_of(G, d, ty, batch)
    print("weights", H, G, d, batch, shared, ty, flush=True)
    t = Texts(lengths(batch, shared, 6), shared, H, G, d, ty, seed=6)
    t.k.zero_()
    t.k[:, 0::2, :, 0], t.k[:, 1::2, :, 0] = 1.0, -1.0
    t.v[:, 0::2] = 1.0
    t.v[:, 1::2] = (-torch.linspace(0.5, 4.0, d, device="cuda")).to(ty)
    x = torch.linspace(0.04, 0.8, batch * H, device="cuda").view(batch, H)
    t.q.zero_()
    t.q[..., 0] = (x * d ** 0.5).to(ty)
    got = t.call()
    k, v, kept, n = gather(t.k, t.v, t.table, t.n, None, shared)
    want, size = [last_rows(t.q, k, y, n, kept)["out"] for y in (v, v.abs())]
    u = ROUND[ty]
    bound = (2 * 2.0 ** -21 * t.q[..., :1].double() * d ** -0.5 + u * u + E_SUM) * size + u * want.abs()
    check(got, dict(out=want.cpu(), out_bound=bound.cpu()), "out", ty)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d,batch", [(6, 2, 64, 40), (4, 2, 128, 9), (5, 1, 100, 10), (8, 1, 60, 50)])
def test_places_past_all_texts_are_not_seen(H, G, d, batch, ty):
    """Texts that all end within the prefix: what its later places hold changes no bit (rows formed again word by word would)."""
    shared = shape_of(G, d, ty, batch)
    longest = shared // 2 // 64 * 64 + 5
    t = Texts([longest - x % 3 - 64 * (x % 2) for x in range(batch)], shared, H, G, d, ty, seed=7)
    end = t.table[0, longest // 64].long()
    rest = t.table[0, longest // 64 + 1:shared // 64].long()
    got = []
    for hold in (0.0, float("nan"), float("inf")):
        for x in (t.k, t.v):
            x[end, longest % 64:] = hold
            x[rest] = hold
        got.append(t.call())
    t.check(got[0])
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


# ---- windows of which most lies in the prefix, for few and for many queries --------------------------------

def window_of(G, d, ty, batch):
    """Words of a window that the prefix's own blocks serve: 512 MB more to read if every text read them."""
    return -(-4 * MORE // ((batch - 1) * G * d * 2 * torch.finfo(ty).bits // 8))


def call_with_own_blocks(t, left=None, sinks=0, **see):
    """The call, once it has been seen to split into other parts than one without a prefix does."""
    size = []
    for shared in (0, t.shared):
        spec = w2v._spec(t.q, t.k.shape[2], left, 0, sinks, False, None, None, None)
        table = w2v.PageTable(4096, t.table.shape[1], t.table.shape[1], t.words, t.k.shape[0])
        size.append(w2v.lib().w2v_attend_pages_workspace(ctypes.byref(spec), len(t.n), ctypes.byref(table), shared))
    assert size[0] != size[1], "no blocks of its own"
    return w2v.attend_pages(t.q, t.k, t.v, t.table, i32(t.n), shared=t.shared, left=left, sinks=sinks, **see)


FEW_AND_MANY = [(1, 1, 31, 30), (4, 2, 128, 9), (8, 4, 96, 20), (2, 2, 64, 60), (6, 2, 127, 40), (3, 1, 90, 50), (5, 1, 32, 33)]


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d,batch", FEW_AND_MANY)
def test_windows_masks_and_bias_by_queries(H, G, d, batch, ty):
    """18 to 165 queries for a key head, each width of tile, windows that begin in the prefix, first words before them, a bias, dropped words
    and numbers that are no page."""
    left = window_of(G, d, ty, batch)
    shared = (left + 1500) // 64 * 64
    print("prefix", H, G, d, batch, shared, left, ty, flush=True)
    n = lengths(batch, shared, 8)
    n[0] = shared + 1                                        # one word of its own
    t = Texts(n, shared, H, G, d, ty, words=16, seed=8)
    plain = [dict(), dict(left=left), dict(left=left, sinks=64), dict(left=left + 700, sinks=3, skip_self=True)]
    for see in plain:
        t.check(call_with_own_blocks(t, **see), **see)
    t.table[0, 3::7] = t.k.shape[0]                           # numbers that are no page, in the prefix and behind it
    t.table[5::2, -3] = -1
    more = dict(bias=torch.randn(H, 32, device="cuda"), buckets=w2v.relative_buckets(32, 128),
                keep=(torch.rand(batch, t.table.shape[1] * 16, device="cuda") > 0.6).to(torch.uint8))
    for see in plain:
        t.check(call_with_own_blocks(t, **see, **more), **see, **more)
    del more["keep"]
    t.check(call_with_own_blocks(t, **plain[2], **more), **plain[2], **more)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d,batch", [(2, 2, 40, 20), (4, 2, 128, 12), (4, 2, 40, 24), (6, 2, 40, 60)])
def test_infinities_that_some_windows_see(H, G, d, batch, ty):
    """20 to 180 queries for a key head: texts whose window shows an infinite value or a key that is not a number have it, the others do not."""
    left = window_of(G, d, ty, batch)
    shared, group = (left + 700) // 64 * 64 + 64, H // G
    n = [shared + 10 * b for b in range(batch)]
    t = Texts(n, shared, H, G, d, ty, seed=9)
    want = call_with_own_blocks(t, left=left)
    far, near = n[batch // 3] - 1 - left, n[batch // 2] - 1 - left      # the first word that these texts are shown
    t.v[int(t.table[0, near // 64]), near % 64, 1, 3] = float("inf")
    t.k[int(t.table[0, far // 64]), far % 64, 0, 5] = float("nan")
    got = call_with_own_blocks(t, left=left)
    sees = torch.zeros(batch, H, d, dtype=torch.bool, device="cuda")
    sees[:batch // 2 + 1, group:, 3] = True
    sees[:batch // 3 + 1, :group] = True
    assert torch.equal(torch.isfinite(got), ~sees)
    assert torch.allclose(got[~sees].float(), want[~sees].float(), atol={F32: 1e-5, F16: 4e-3, BF16: 3e-2}[ty])
    infinite, nan = got[:, group:, 3][sees[:, group:, 3]], got[:, :group][sees[:, :group]]
    assert (infinite == float("inf")).all() and torch.isnan(nan).all()


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d,batch", [(2, 2, 64, 20), (4, 2, 100, 24), (3, 1, 128, 40)])
def test_large_scores_and_masks_by_queries(H, G, d, batch, ty):
    """As test_large_scores_and_masks_of_the_lowest_value, for 20, 48 and 120 queries a key head, and in a window."""
    left = window_of(G, d, ty, batch)
    shared = (left + 700) // 64 * 64
    t = Texts([shared + x for x in range(batch)], shared, H, G, d, ty, seed=10)
    t.q = (t.q.float() * 30).to(ty)
    whole = t.table.clone()
    whole[:, :shared // 64] = t.table[0, :shared // 64]
    bmap = w2v.relative_buckets(32, 200)
    for low in (-math.inf, torch.finfo(F32).min, -1e9):
        bias = torch.randn(H, 32, device="cuda")
        bias[:, 15] = low
        bias[1] = low
        for see in (dict(), dict(left=left, sinks=5)):
            want = w2v.attend_pages(t.q, t.k, t.v, whole, i32(t.n), bias=bias, buckets=bmap, **see)
            tol = {F32: 2e-3, F16: 4e-3, BF16: 3e-2}[ty]
            got = call_with_own_blocks(t, bias=bias, buckets=bmap, **see)
            assert torch.allclose(got.float(), want.float(), atol=tol, rtol=tol), (low, see)


@pytest.mark.parametrize("ty,H,G,d,batch,words,shared", [(2, 32, 8, 128, 64, 16, 32768), (0, 8, 8, 64, 24, 64, 32768), (1, 6, 6, 100, 64, 64, 16384)])
def test_what_a_window_shows_of_a_prefix_counts(ty, H, G, d, batch, words, shared):
    """A prefix has blocks of its own by what a text can be shown of it, not by its length: a call splits otherwise for it, or does not."""
    table = w2v.PageTable(4096, shared // words + 64, shared // words + 64, words, 1 << 16)

    def size(shared, left, sinks=0):
        spec = w2v.AttendSpec(type=ty, heads=H, kv_heads=G, width=d, left=left, right=0, sinks=sinks, skip_self=0, scale=0.1)
        return w2v.lib().w2v_attend_pages_workspace(ctypes.byref(spec), batch, ctypes.byref(table), shared)
    for left in (0, 99, 800):
        for sinks in (0, 64):
            assert size(shared, left, sinks) == size(0, left, sinks)
    for left in (shared // 2, shared - 2, shared - 1, shared, w2v.UNBOUNDED):
        assert size(shared, left) != size(0, left)
