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


@pytest.mark.gpu
def test_strides_masked_places_and_another_stream():
    B, room, H, G, d = 3, 200, 4, 2, 60
    both = torch.randn(2, G, B, room, d + 4, device="cuda")               # another order, rows apart
    k, v = [both[n].permute(1, 2, 0, 3)[..., :d] for n in (0, 1)]
    q = torch.randn(B, 3 * H, d, device="cuda")[:, ::3]
    n = torch.tensor([200, 150, 1], dtype=torch.int32, device="cuda")
    keep = (torch.rand(B, room, device="cuda") > 0.3).to(torch.uint8)
    want = w2v.attend_step(q.contiguous(), k.contiguous(), v.contiguous(), n, left=90, sinks=3, keep=keep)
    assert torch.equal(w2v.attend_step(q, k, v, n, left=90, sinks=3, keep=keep), want)
    k2, v2 = k.contiguous().clone(), v.contiguous().clone()
    k2[keep == 0], v2[keep == 0] = float("nan"), float("inf")             # dropped, and beyond what is filled
    k2[1, 150:], v2[1, 150:] = float("nan"), float("nan")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = w2v.attend_step(q, k2, v2, n, left=90, sinks=3, keep=keep, stream=st)
    st.synchronize()
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_a_cache_past_32_bit_offsets():
    room, G, d = 40_000_000, 1, 64                                        # 2.56e9 elements, 5.1 GB
    k = torch.zeros(1, room, G, d, dtype=F16, device="cuda")
    q = torch.randn(1, 2, d, device="cuda").to(F16)
    k[0, -50:] = torch.randn(50, G, d, device="cuda").to(F16)
    n = torch.tensor([room], dtype=torch.int32, device="cuda")
    far = w2v.attend_step(q, k, k, n, left=49)
    near = w2v.attend_step(q, k[:, -50:].contiguous(), k[:, -50:].contiguous(), torch.tensor([50], dtype=torch.int32, device="cuda"))
    assert torch.allclose(far.float(), near.float(), atol=2e-3)


@pytest.mark.gpu
def test_steps_give_the_rows_of_the_whole_text():
    T, H, G, d = 130, 4, 2, 60
    q, k, v = [torch.randn(T, n, d, device="cuda") for n in (H, G, G)]
    off = torch.tensor([0, T], dtype=torch.int64, device="cuda")
    bias, bmap = torch.randn(H, 16, device="cuda"), w2v.relative_buckets(16, 30)
    see = dict(left=40, sinks=2, bias=bias, buckets=bmap)
    out, _ = w2v.attend(q, k, v, off, right=0, **see)
    for i in (0, 1, 41, 42, 43, 100, 129):
        got = w2v.attend_step(q[i:i + 1], k[None], v[None], torch.tensor([i + 1], dtype=torch.int32, device="cuda"), **see)
        assert torch.allclose(got[0], out[i], atol=1e-5)


def test_refusals():
    L = w2v.lib()
    p = 4096
    ok = dict(type=0, heads=4, kv_heads=2, width=64, left=5, right=0, sinks=0, skip_self=0, scale=0.1)

    def step(batch=2, room=100, n=p, q=None, k=None, ws=p, size=1 << 30, **kw):
        r = ctypes.byref
        spec, h = w2v.AttendSpec(**{**ok, **kw}), w2v.Heads(p, 256, 64)
        c = w2v.Cache(p, 100 * 128, 128, 64)
        return L.w2v_attend_step(r(spec), r(q or h), r(k or c), r(c), n, batch, room, None, r(h), ws, size, None)
    assert step(batch=0) == 0 and step(room=0) == -2 and step(room=0x7FFFFFFF) == -2 and step(batch=1 << 24) == -2
    assert step(n=None) == -1 and step(k=w2v.Cache(None, 1, 1, 1)) == -1 and step(k=w2v.Cache(p + 2, 1, 1, 1)) == -2
    assert step(k=w2v.Cache(p, 1 << 41, 128, 64)) == -2 and step(width=200) == -2
    assert step(room=100000, left=0xFFFFFFFF, ws=None) == -1 and step(room=100000, left=0xFFFFFFFF, ws=p + 4) == -2
    assert step(room=100000, left=0xFFFFFFFF, size=8) == -2 and b"too small" in L.w2v_last_error()
