"""Attention of one new word per text over a cache against the definition in 64 bits (bounds: attend_reference)."""
import ctypes

import pytest
import torch

from attend_reference import attend_reference, check
from paper_1606_08495_amd import w2v

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def expected(q, k, v, n, keep, bias, bmap, **see):
    """The last word's row of attention over each text by itself."""
    out, bound = [], []
    for b, count in enumerate(n):
        count = min(count, k.shape[1])
        if count == 0:
            out.append(torch.zeros(q.shape[1:], dtype=torch.float64))
            bound.append(torch.zeros(q.shape[1:], dtype=torch.float64))
            continue
        full = torch.zeros(count, *q.shape[1:], dtype=q.dtype)
        full[-1] = q[b]
        r = attend_reference(full, k[b, :count], v[b, :count], [0, count], right=0, bias=bias, buckets=bmap,
                             keep=None if keep is None else keep[b, :count], **see)
        out.append(r["out"][-1])
        bound.append(r["out_bound"][-1])
    return dict(out=torch.stack(out), out_bound=torch.stack(bound))


def run(n, room, H, G, d, ty, seed=0, buckets=None, span=None, drop=0.0, **see):
    g = torch.Generator().manual_seed(seed)
    B = len(n)
    q = torch.randn(B, H, d, generator=g).to(ty)
    k, v = [torch.randn(B, room, G, d, generator=g).to(ty) for _ in range(2)]
    bias = torch.randn(H, buckets, generator=g) if buckets else None
    bmap = w2v.relative_buckets(buckets, span, device="cpu") if buckets else None
    keep = (torch.rand(B, room, generator=g) >= drop).to(torch.uint8) if drop else None
    ref = expected(q, k, v, n, keep, bias, bmap, **see)
    cuda = lambda t: None if t is None else t.cuda()
    out = w2v.attend_step(q.cuda(), k.cuda(), v.cuda(), torch.tensor(n, dtype=torch.int32).cuda(), keep=cuda(keep), bias=cuda(bias),
                          buckets=cuda(bmap), **see)
    check(out, ref, "out", ty)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d", [(1, 1, 64), (5, 5, 60), (4, 2, 128), (6, 2, 37), (8, 2, 33), (5, 1, 100), (8, 1, 128), (9, 1, 16),
                                   (34, 2, 64), (40, 1, 128), (2, 2, 1), (4, 1, 127), (33, 1, 31)])
def test_heads_and_widths(H, G, d, ty):
    print("step", H, G, d, ty, flush=True)
    run([1, 0, 7, 300], 300, H, G, d, ty)
    run([255, 256, 257, 2, 700, 31], 700, H, G, d, ty, left=100, sinks=4, buckets=8, span=20, drop=0.3)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, BF16])
@pytest.mark.parametrize("see", [dict(), dict(left=0), dict(left=0, skip_self=True), dict(skip_self=True), dict(left=5, sinks=64),
                                 dict(left=300, sinks=1), dict(left=5000, sinks=7)])
def test_windows(see, ty):
    print("step", see, ty, flush=True)
    for group in (1, 4):
        run([1, 2, 63, 64, 65, 2000, 1999], 2000, 2 * group, 2, 64, ty, **see)
        run([1, 2, 63, 64, 65, 2000, 5000], 2000, 2 * group, 2, 64, ty, drop=0.9, buckets=32, span=128, **see)
