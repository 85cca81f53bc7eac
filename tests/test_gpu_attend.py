"""Attention over texts, forward and backward, against the definition in 64 bits (bounds: attend_reference)."""
import ctypes

import numpy as np
import pytest
import torch

from attend_reference import attend_reference, check
from paper_1606_08495_amd import w2v

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def offsets_of(lengths):
    return [0] + list(np.cumsum(lengths))


def rows(T, H, G, d, ty, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(T, n, d, generator=g).to(ty) for n in (H, G, G, H)]


def run(lengths, H, G, d, ty, seed=0, train=True, buckets=None, span=None, drop=0.0, **see):
    off = offsets_of(lengths)
    T = off[-1]
    q, k, v, dout = rows(T, H, G, d, ty, seed)
    g = torch.Generator().manual_seed(seed + 1)
    bias = torch.randn(H, buckets, generator=g) if buckets else None
    bmap = w2v.relative_buckets(buckets, span, device="cpu") if buckets else None
    keep = (torch.rand(T, generator=g) >= drop).to(torch.uint8) if drop else None
    ref = attend_reference(q, k, v, off, keep=keep, bias=bias, buckets=bmap, dout=dout, **see)
    cuda = lambda t: None if t is None else t.cuda()
    kw = dict(keep=cuda(keep), bias=cuda(bias), buckets=cuda(bmap), **see)
    soff = torch.tensor(off, dtype=torch.int64, device="cuda")
    out, lse = w2v.attend(q.cuda(), k.cuda(), v.cuda(), soff, **kw)
    check(out, ref, "out", ty)
    check(lse, ref, "lse")
    if not train:
        return
    dq, dk, dv, dbias = w2v.attend_backward(dout.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse, soff, **kw)
    check(dq, ref, "dq", ty)
    check(dk, ref, "dk", ty)
    check(dv, ref, "dv", ty)
    if bias is not None:
        check(dbias, ref, "dbias")


SHORT = [20, 1, 3, 40, 0, 0, 7, 1, 12, 33, 32, 31, 2, 0]         # texts of no word and of one among them
# lengths on both sides of a wavefront's 32 words, a tile's 64 keys and a block's 128
EDGES = [[1], [2], [31], [32], [33], [63], [64], [65], [127], [128], [129], [255, 1, 257], [64, 64, 128], [700]]
SEE = [dict(left=10, right=10, skip_self=True), dict(left=None, right=0), dict(left=None, right=None),
       dict(left=5, right=0, sinks=2), dict(left=33, right=0, sinks=4), dict(left=0, right=0), dict(left=0, right=0, skip_self=True),
       dict(left=0, right=3, sinks=64), dict(left=100, right=7, sinks=33), dict(left=3, right=None, sinks=1)]


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("see", SEE)
def test_windows(see, ty):
    for n, lengths in enumerate([SHORT, [300], [150, 9, 200, 70]]):
        print("attend", see, ty, lengths, flush=True)
        run(lengths, 2, 2, 60, ty, seed=n, **see)
        run(lengths, 4, 2, 60, ty, seed=n, buckets=32, span=20, drop=0.3, **see)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("lengths", EDGES)
def test_lengths(lengths, ty):
    print("attend", lengths, ty, flush=True)
    run(lengths, 2, 1, 64, ty, left=None, right=0)
    run(lengths, 1, 1, 32, ty, left=40, right=40, buckets=8, span=5)
    run(lengths, 3, 1, 128, ty, left=90, right=0, sinks=3)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("d", [1, 2, 3, 7, 8, 15, 16, 17, 31, 32, 33, 37, 48, 60, 63, 64, 65, 95, 96, 97, 100, 127, 128])
def test_widths(d, ty):
    print("attend width", d, ty, flush=True)
    run([70, 30, 130], 2, 2, d, ty, left=50, right=0, sinks=2)


@pytest.mark.gpu
@pytest.mark.parametrize("span,buckets", [(1, 2), (2, 3), (16, 32), (128, 32), (500, 8), (1023, 1024)])
@pytest.mark.parametrize("ty", [F32, BF16])
def test_bias(span, buckets, ty):
    print("attend bias", span, buckets, ty, flush=True)
    run([400, 3, 150], 2, 1, 64, ty, left=None, right=None, buckets=buckets, span=span)
    run([400, 3, 150], 2, 2, 64, ty, left=200, right=0, sinks=5, buckets=buckets, span=span)


def plain(T, H, G, d, ty, seed):
    q, k, v, dout = [t.cuda() for t in rows(T, H, G, d, ty, seed)]
    return q, k, v, dout


def whole(q, k, v, dout, off, **kw):
    out, lse = w2v.attend(q, k, v, off, **kw)
    return (out, lse) + tuple(t for t in w2v.attend_backward(dout, q, k, v, out, lse, off, **kw) if t is not None)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, BF16])
def test_what_is_not_shown_does_not_show(ty):
    """Infinities and NaN in words that subsampling dropped, beyond the window and in other texts reach only the words that
    see them; what they do not reach keeps its bits or, where the sums are formed anew, its value."""
    T, H, G, d = 500, 2, 1, 60
    q, k, v, dout = plain(T, H, G, d, ty, 3)
    off = torch.tensor([0, 300, 500], dtype=torch.int64, device="cuda")
    bias, bmap = torch.randn(H, 32, device="cuda"), w2v.relative_buckets(32, 20)
    keep = torch.ones(T, dtype=torch.uint8, device="cuda")
    keep[[7, 150, 400]] = 0
    see = dict(left=20, right=5, sinks=2, keep=keep, bias=bias, buckets=bmap)
    ref = attend_reference(*[t.cpu() for t in (q, k, v)], [0, 300, 500], left=20, right=5, sinks=2, keep=keep.cpu(),
                           bias=bias.cpu(), buckets=bmap.cpu(), dout=dout.cpu())
    k2, v2 = k.clone(), v.clone()
    for i, bad in zip([7, 150, 400], [float("nan"), float("inf"), float("-inf")]):
        k2[i], v2[i] = bad, bad
    got = whole(q, k2, v2, dout, off, **see)                              # dropped words: nothing changes anywhere
    for t, name in zip(got, ("out", "lse", "dq", "dk", "dv", "dbias")):
        check(t, ref, name, F32 if name in ("lse", "dbias") else ty)
    assert not got[3][keep == 0].any() and not got[4][keep == 0].any()
    v3 = v.clone()
    v3[100, 0, 3] = float("inf")                                          # a word that some are shown: column 3 of those alone
    out, _ = w2v.attend(q, k, v3, off, **see)
    reached = torch.zeros(T, dtype=torch.bool, device="cuda")
    reached[95:121] = True                                                # 100 - right .. 100 + left
    assert not torch.isfinite(out[reached][:, :, 3]).any()
    others = torch.ones(d, dtype=torch.bool, device="cuda")
    others[3] = False
    assert torch.isfinite(out[~reached]).all() and torch.isfinite(out[:, :, others]).all()
    q3 = q.clone()
    q3[200] = float("nan")                                                # a query: its own row, and the keys that it is shown
    res = whole(q3, k, v, dout, off, left=20, right=5)
    touched = torch.zeros(T, dtype=torch.bool, device="cuda")
    touched[180:206] = True
    assert torch.isfinite(res[3][~touched]).all() and torch.isfinite(res[4][~touched]).all()
    rest = torch.arange(T, device="cuda") != 200
    assert torch.isfinite(res[0][rest]).all() and torch.isfinite(res[2][rest]).all() and torch.isnan(res[0][200]).all()


@pytest.mark.gpu
def test_lowest_and_infinite_biases():
    T, H, d = 90, 1, 32
    q, k, v, dout = plain(T, H, H, d, F32, 5)
    off = torch.tensor([0, T], dtype=torch.int64, device="cuda")
    bmap = torch.zeros(11, dtype=torch.int32, device="cuda")
    bmap[5:] = 1                                                          # before: bucket 0, the word and after: bucket 1
    for low in (torch.finfo(F32).min, float("-inf"), -1e30):
        bias = torch.tensor([[low, 0.0]], device="cuda")
        out, lse = w2v.attend(q, k, v, off, bias=bias, buckets=bmap)
        ref, _ = w2v.attend(q, k, v, off, left=0)
        assert torch.allclose(out, ref, atol=1e-5)
        both = torch.tensor([[low, low]], device="cuda")
        out, lse = w2v.attend(q, k, v, off, bias=both, buckets=bmap)
        if low == float("-inf"):                                          # nothing is left
            assert not out.any() and (lse == float("-inf")).all()
        elif low < -1e35:                                                 # equal weights: the scores are lost beside it
            assert torch.allclose(out, v.mean(0, keepdim=True).expand_as(out), atol=1e-5)
    wide = torch.full((11,), 7, dtype=torch.int32, device="cuda")         # buckets that do not exist add nothing
    a = w2v.attend(q, k, v, off, bias=torch.ones(1, 2, device="cuda"), buckets=wide)[0]
    assert torch.allclose(a, w2v.attend(q, k, v, off)[0], atol=1e-6)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16])
def test_packed_rows_orders_and_another_stream(ty):
    T, H, d = 333, 3, 60
    packed = torch.randn(T, 3, H, d, device="cuda").to(ty)                # q, k, v of a word side by side
    q, k, v = packed[:, 0], packed[:, 1], packed[:, 2]
    dout = torch.randn(H, T, d, device="cuda").to(ty).transpose(0, 1)     # heads first
    off = torch.tensor([0, 100, 333], dtype=torch.int64, device="cuda")
    see = dict(left=40, right=0, sinks=1)
    want = whole(q.contiguous(), k.contiguous(), v.contiguous(), dout.contiguous(), off, **see)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    out = torch.full((T, 2 * H, d + 3), 9.0, dtype=ty, device="cuda")
    into = out[:, ::2, :d]
    st.wait_stream(torch.cuda.current_stream())
    _, lse = w2v.attend(q, k, v, off, out=into, stream=st, **see)
    got = w2v.attend_backward(dout, q, k, v, into, lse, off, stream=st, **see)
    st.synchronize()
    assert torch.equal(into, want[0]) and torch.equal(lse, want[1])
    assert (out[:, 1::2] == 9).all() and (out[:, :, d:] == 9).all()       # nothing beside the rows
    for a, b in zip(got[:3], want[2:]):
        assert torch.equal(a, b)
    again = whole(q, k, v, dout, off, **see)
    assert all(torch.equal(a, b) for a, b in zip(again, want))            # every time the same bits


@pytest.mark.gpu
def test_a_graph_of_both_passes_replays():
    T, H, d = 700, 4, 64
    q, k, v, dout = plain(T, H, 2, d, BF16, 8)
    off = torch.tensor([0, 650, 700], dtype=torch.int64, device="cuda")
    bias, bmap = torch.randn(H, 8, device="cuda"), w2v.relative_buckets(8, 30)
    see = dict(left=100, right=0, sinks=2, bias=bias, buckets=bmap)
    want = whole(q, k, v, dout, off, **see)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = whole(q, k, v, dout, off, **see)
    for n in range(4):
        for t in got:
            t.fill_(7)
        q.mul_(1.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_offsets_that_break_the_rules_stay_inside():
    T, H, d = 400, 1, 64
    q, k, v, dout = plain(T, H, H, d, F32, 9)
    for off in ([0, 400], [0, 10, 5, 300, 20, 400], [50, 10 ** 9, 3], [400, 0], [0, 0, 0, 0], [7, 7, 7, 500], [0, 2 ** 40]):
        res = whole(q, k, v, dout, torch.tensor(off, dtype=torch.int64, device="cuda"), left=30, right=0, sinks=3)
        torch.cuda.synchronize()
        assert all(t.shape[-1] in (T, d) for t in res)


@pytest.mark.gpu
def test_late_pieces_of_long_texts():
    """First words that stay visible are seen from far behind their block: pieces of queries that are joined."""
    for ty in (F32, BF16):
        run([1500, 40, 900], 2, 1, 32, ty, left=50, right=0, sinks=5)
        run([3, 1300], 1, 1, 48, ty, left=10, right=2, sinks=40, drop=0.2, buckets=8, span=30)


@pytest.mark.gpu
def test_gradients_against_differences():
    lengths, H, G, d, h = [9, 5], 2, 1, 7, 1e-2
    off = torch.tensor(offsets_of(lengths), dtype=torch.int64, device="cuda")
    q, k, v, dout = rows(14, H, G, d, F32, 2)
    bias, bmap = torch.randn(H, 8, generator=torch.Generator().manual_seed(1)), w2v.relative_buckets(8, 4)
    see = dict(left=4, right=2, sinks=1, skip_self=True, buckets=bmap)

    def value():
        out, _ = w2v.attend(q.cuda(), k.cuda(), v.cuda(), off, bias=bias.cuda(), **see)
        return float((out.cpu().double() * dout.double()).sum())
    out, lse = w2v.attend(q.cuda(), k.cuda(), v.cuda(), off, bias=bias.cuda(), **see)
    grads = [t.cpu().double() for t in w2v.attend_backward(dout.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse, off,
                                                           bias=bias.cuda(), **see)]
    # a central difference is off by h^2 / 6 times a third derivative (below 60 for these sizes: 1e-3) and by the rounding of
    # 196 outputs, each 2^-22 at most, over 2 h: 2.4e-3
    g = torch.Generator().manual_seed(3)
    for t, grad in zip((q, k, v, bias), grads):
        for _ in range(6):
            at = tuple(int(torch.randint(n, (1,), generator=g)) for n in t.shape)
            old = float(t[at])
            t[at] = old + h
            up = value()
            t[at] = old - h
            down = value()
            t[at] = old
            assert abs((up - down) / (2 * h) - float(grad[at])) <= 4e-3 * (1 + abs(float(grad[at])))


@pytest.mark.gpu
def test_no_tokens():
    z = torch.empty(0, 2, 16, device="cuda")
    off = torch.zeros(1, dtype=torch.int64, device="cuda")
    bias, bmap = torch.randn(2, 4, device="cuda"), w2v.relative_buckets(4, 3)
    out, lse = w2v.attend(z, z, z, off, bias=bias, buckets=bmap)
    assert out.shape == z.shape and lse.shape == (2, 0)
    dq, dk, dv, dbias = w2v.attend_backward(z, z, z, z, out, lse, off, bias=bias, buckets=bmap)
    assert dbias.shape == bias.shape and not dbias.any()


def test_relative_buckets_against_whole_numbers():
    def expected(buckets, span):
        half = buckets // 2
        near = max(1, half // 2)
        far = half - near
        res = []
        for r in range(span + 1):
            t = 0
            while r >= near and far and t + 1 < far and span ** (t + 1) * near ** far <= r ** far * near ** (t + 1):
                t += 1
            res.append(near + t if r >= near and far else min(r, half - 1))
        return res[::-1] + [half + b for b in res[1:]]
    for buckets in list(range(2, 40)) + [64, 255]:
        for span in (1, 2, 3, 8, 16, 27, 64, 81, 128, 243, 256, 625, 1023):
            assert w2v.relative_buckets(buckets, span, device="cpu").tolist() == expected(buckets, span)


def test_refusals():
    L = w2v.lib()
    p = 4096                                                              # never read: every call here is refused
    ok = dict(type=0, heads=4, kv_heads=2, width=64, left=5, right=0, sinks=0, skip_self=0, scale=0.1, n_buckets=0, span=0,
              bias_dev=None, bucket_dev=None)
    rows_of = lambda token=256, head=64, at=p: w2v.Heads(at, token, head)

    def fwd(T=10, n=1, off=p, q=None, out=None, **kw):
        spec = w2v.AttendSpec(**{**ok, **kw})
        r = ctypes.byref
        return L.w2v_attend(r(spec), r(q or rows_of()), r(rows_of(128)), r(rows_of(128)), off, n, T, None, r(out or rows_of()),
                            None, None)

    def bwd(ws=p, size=1 << 30, lse=p, dbias=None, dq=None, **kw):
        spec = w2v.AttendSpec(**{**ok, **kw})
        r = ctypes.byref
        a, b = rows_of(), rows_of(128)
        return L.w2v_attend_backward(r(spec), r(a), r(a), r(b), r(b), r(a), lse, p, 1, 10, None, r(dq or a), r(b), r(b), dbias,
                                     ws, size, None)
    assert fwd(type=3) == -2 and fwd(width=0) == -2 and fwd(width=129) == -2 and fwd(heads=5) == -2 and fwd(kv_heads=0) == -2
    assert fwd(heads=2048, kv_heads=2048) == -2 and fwd(sinks=65) == -2 and fwd(scale=0.0) == -2 and fwd(scale=-1.0) == -2
    assert fwd(scale=float("nan")) == -2 and fwd(scale=float("inf")) == -2
    assert fwd(bias_dev=p) == -1 and fwd(bias_dev=p, bucket_dev=p, span=0, n_buckets=4) == -2
    assert fwd(bias_dev=p, bucket_dev=p, span=1024, n_buckets=4) == -2 and fwd(bias_dev=p, bucket_dev=p, span=5, n_buckets=0) == -2
    assert fwd(n=0) == -2 and fwd(off=None) == -1 and fwd(T=0x7FFFFFFF) == -2 and fwd(T=0, off=None, n=0) == 0
    assert fwd(q=rows_of(at=p + 2)) == -2 and fwd(out=rows_of(at=None)) == -1
    assert fwd(out=rows_of(token=255)) == -2 and b"overlap" in L.w2v_last_error() and fwd(out=rows_of(head=63)) == -2
    assert fwd(out=rows_of(token=64, head=639)) == -2 and fwd(out=rows_of(token=1 << 41)) == -2
    assert bwd(ws=None) == -1 and bwd(ws=p + 4) == -2 and bwd(size=16) == -2 and b"too small" in L.w2v_last_error()
    assert bwd(lse=None) == -1 and bwd(dbias=p) == -2 and bwd(dq=rows_of(token=200)) == -2
    assert L.w2v_attend(None, None, None, None, p, 1, 1, None, None, None, None) == -1
    assert L.w2v_relative_buckets(1, 5, p) == -2 and L.w2v_relative_buckets(8, 0, p) == -2 and L.w2v_relative_buckets(8, 5, None) == -1
    with pytest.raises(TypeError):
        w2v.attend(torch.zeros(2, 1, 4), torch.zeros(2, 1, 4), torch.zeros(2, 1, 4), torch.zeros(2, dtype=torch.int64))
