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
