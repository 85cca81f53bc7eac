"""Layer norm of rows and its gradients against the formulas in 64 bits.

Bounds, derived before the first run.  A sum of d fp32 terms in any order of the kernel (per lane at most 64 in a row, then
a tree) is off by at most 80 ulp-halves of the sum of magnitudes, 80 * 2^-24 = 4.8e-6 of it; what follows is a handful
of roundings.  With z the normalised row, mean(|x|) rstd bounds the mean's share and |z| the rest, so an element of y may be
off by 1e-5 (|z| + mean|x| rstd) |gain| + 1e-6 |offset|, plus one rounding to the type of the rows.  dx likewise by
1e-5 rstd (|t| + mean|t| + |z| mean|t z|) times (1 + mean|x| rstd).  The column gradients sum m rows, per group
of lanes in a row and then over blocks: 1e-5 of the sum of magnitudes up to 2^16 rows."""
import ctypes

import pytest
import torch

from paper_1606_08495_amd import w2v

ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}


def reference(x, gain, offset, eps, dy=None):
    x = x.double()
    m, d = x.shape
    gain = torch.ones(d, dtype=torch.float64) if gain is None else gain.double()
    offset = torch.zeros(d, dtype=torch.float64) if offset is None else offset.double()
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).pow(2).mean(1, keepdim=True) + eps) ** -0.5
    z = (x - mean) * rstd
    far = x.abs().mean(1, keepdim=True) * rstd
    res = dict(y=z * gain + offset, mean=mean[:, 0], rstd=rstd[:, 0])
    res["y_bound"] = 1e-5 * (z.abs() + far) * gain.abs() + 1e-6 * offset.abs()
    if dy is not None:
        dy = dy.double()
        t = dy * gain
        res["dx"] = rstd * (t - t.mean(1, keepdim=True) - z * (t * z).mean(1, keepdim=True))
        res["dx_bound"] = 1e-5 * (1 + far) * rstd * (t.abs() + t.abs().mean(1, keepdim=True) + z.abs() * (t * z).abs().mean(1, keepdim=True))
        res["dgain"], res["doffset"] = (dy * z).sum(0), dy.sum(0)
        res["dgain_bound"] = 1e-5 * (dy.abs() * (z.abs() + far)).sum(0)
        res["doffset_bound"] = 1e-5 * dy.abs().sum(0)
    return res


def close(got, ref, bound, ty=torch.float32):
    got = got.double().cpu()
    over = (got - ref).abs() - bound - ref.abs() * ROUND[ty] * 1.01 - TINY[ty]
    assert torch.isfinite(got).all() and float(over.max()) <= 0, float(over.max())


# widths on both sides of every change of the lanes that hold a row, of vectors a lane, and odd ones
WIDTHS = [1, 2, 3, 7, 8, 31, 33, 60, 64, 100, 200, 255, 257, 300, 301, 512, 513, 1000, 1024, 1025, 2047, 2049, 4096, 4101,
          8192, 8193, 16383, 16384]


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_and_gradients(d, ty):
    print("norm", d, ty, flush=True)
    for m in [1, 37] if d > 300 else [1, 5, 37, 2500]:
        g = torch.Generator().manual_seed(d * 7 + m)
        x = (torch.randn(m, d, generator=g) * 1.5 + 0.5).to(ty)
        dy = torch.randn(m, d, generator=g).to(ty)
        gain, offset = torch.randn(d, generator=g), torch.randn(d, generator=g)
        for a, b in [(gain, offset), (None, None)]:
            ref = reference(x, a, b, 1e-5, dy)
            dev = [None if t is None else t.cuda() for t in (a, b)]
            y, mean, rstd = w2v.layer_norm(x.cuda(), dev[0], dev[1], 1e-5)
            close(y, ref["y"], ref["y_bound"], ty)
            close(mean, ref["mean"], 1e-5 * x.double().abs().mean(1))
            close(rstd, ref["rstd"], 1e-5 * ref["rstd"] * (1 + x.double().abs().mean(1) * ref["rstd"]))
            dx, dgain, doffset = w2v.layer_norm_backward(dy.cuda(), x.cuda(), dev[0], mean, rstd)
            close(dx, ref["dx"], ref["dx_bound"], ty)
            close(dgain, ref["dgain"], ref["dgain_bound"])
            close(doffset, ref["doffset"], ref["doffset_bound"])


@pytest.mark.gpu
def test_many_rows_repeat_bit_for_bit():
    m, d = 50_001, 300
    x, dy, gain = torch.randn(m, d, device="cuda"), torch.randn(m, d, device="cuda"), torch.randn(d, device="cuda")
    first = None
    for _ in range(3):
        y, mean, rstd = w2v.layer_norm(x, gain)
        out = (y, mean, rstd) + w2v.layer_norm_backward(dy, x, gain, mean, rstd)
        if first is None:
            first = out
            ref = reference(x.cpu(), gain.cpu(), None, 1e-5, dy.cpu())
            close(y, ref["y"], ref["y_bound"])
            close(out[3], ref["dx"], ref["dx_bound"])
            close(out[4], ref["dgain"], ref["dgain_bound"])
            close(out[5], ref["doffset"], ref["doffset_bound"])
        assert all(torch.equal(a, b) for a, b in zip(first, out))


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [torch.float32, torch.bfloat16])
def test_rows_apart_in_place_and_on_another_stream(ty):
    m, d = 333, 60
    wide = torch.randn(m, 4 * d + 3, device="cuda").to(ty)
    x = wide[:, d + 1:2 * d + 1]                             # rows of a wider matrix, at odd addresses
    keep = wide.clone()
    gain = torch.randn(d, device="cuda")
    ref = reference(x.cpu(), gain.cpu(), None, 1e-5)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y, mean, rstd = w2v.layer_norm(x, gain, stream=st)
    st.synchronize()
    close(y, ref["y"], ref["y_bound"], ty)
    got = w2v.layer_norm(x, gain, out=x)[0]                  # in place: nothing beside the rows changes
    assert torch.equal(got, y)
    assert torch.equal(wide[:, :d + 1], keep[:, :d + 1]) and torch.equal(wide[:, 2 * d + 1:], keep[:, 2 * d + 1:])
    dy = torch.randn(m, d, device="cuda").to(ty)
    want = w2v.layer_norm_backward(dy, keep[:, d + 1:2 * d + 1], gain, mean, rstd)
    into = keep[:, d + 1:2 * d + 1]
    got = w2v.layer_norm_backward(dy, into, gain, mean, rstd, out=into)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    one = torch.randn(1, d, device="cuda").to(ty).expand(5, d)      # one row read five times
    y = w2v.layer_norm(one, gain)[0]
    assert torch.equal(y[0], y[4])


@pytest.mark.gpu
def test_gradients_against_differences():
    m, d, h = 3, 17, 1e-2
    g = torch.Generator().manual_seed(5)
    x, dy, gain, offset = [torch.randn(*s, generator=g) for s in ((m, d), (m, d), (d,), (d,))]
    y, mean, rstd = w2v.layer_norm(x.cuda(), gain.cuda(), offset.cuda())
    dx, dgain, doffset = [t.cpu().double() for t in w2v.layer_norm_backward(dy.cuda(), x.cuda(), gain.cuda(), mean, rstd)]

    def value(x, gain, offset):                              # of the kernel's own forward pass
        return float((w2v.layer_norm(x.cuda(), gain.cuda(), offset.cuda())[0].cpu().double() * dy.double()).sum())
    # a central difference of step h is off by h^2 / 6 times the third derivative (below 30 here: 5e-4) and by the values'
    # rounding, 51 terms of 4 * 2^-24 each, over 2 h: 6e-4
    for _ in range(12):
        i, c = int(torch.randint(m, (1,), generator=g)), int(torch.randint(d, (1,), generator=g))
        for t, grad, at in ((x, dx, (i, c)), (gain, dgain, (c,)), (offset, doffset, (c,))):
            old = float(t[at])
            t[at] = old + h
            up = value(x, gain, offset)
            t[at] = old - h
            down = value(x, gain, offset)
            t[at] = old
            assert abs((up - down) / (2 * h) - float(grad[at])) <= 2e-3 * (1 + abs(float(grad[at])))


@pytest.mark.gpu
def test_not_a_number_stays_in_its_row_and_large_values_hold():
    x = torch.randn(40, 100, device="cuda")
    clean = w2v.layer_norm(x)[0]
    x[7, 3], x[20, 99] = float("nan"), float("inf")
    y = w2v.layer_norm(x)[0]
    assert torch.isnan(y[7]).all() and torch.isnan(y[20]).all()
    rest = [r for r in range(40) if r not in (7, 20)]
    assert torch.equal(y[rest], clean[rest])
    far = torch.randn(9, 300) + 1000.0                        # a variance far below the squared mean
    ref = reference(far, None, None, 1e-5)
    close(w2v.layer_norm(far.cuda())[0], ref["y"], ref["y_bound"])
    flat = torch.full((3, 50), 2.5, device="cuda")            # no variance at all
    y, mean, rstd = w2v.layer_norm(flat, eps=1e-5)
    assert torch.equal(y, torch.zeros_like(y)) and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5))


@pytest.mark.gpu
def test_no_rows():
    x = torch.empty(0, 30, device="cuda")
    y, mean, rstd = w2v.layer_norm(x)
    assert y.shape == (0, 30)
    dx, dgain, doffset = w2v.layer_norm_backward(x, x, None, mean, rstd)
    assert dx.shape == (0, 30) and not dgain.any() and not doffset.any()


def test_refusals():
    L = w2v.lib()
    p = ctypes.c_void_p(4096)                                 # never read: every call here is refused

    def fwd(type=0, x=p, xs=8, rows=3, d=8, eps=1e-5, y=p, ys=8):
        return L.w2v_layer_norm(type, x, xs, rows, d, None, None, eps, y, ys, None, None, None)

    def bwd(type=0, rows=3, d=8, dx=p, dxs=8, mean=p, ws=p, size=1 << 30, dgain=p):
        return L.w2v_layer_norm_backward(type, p, 8, p, 8, rows, d, None, mean, p, dx, dxs, dgain, None, ws, size, None)
    assert fwd(type=3) == -2 and fwd(type=-1) == -2 and fwd(d=0) == -2 and fwd(d=16385) == -2
    assert fwd(x=None) == -1 and fwd(y=None) == -1
    assert fwd(eps=-1.0) == -2 and fwd(eps=float("nan")) == -2 and fwd(eps=float("inf")) == -2
    assert fwd(ys=7) == -2 and b"overlap" in L.w2v_last_error()
    assert fwd(xs=9) == -2 and fwd(x=ctypes.c_void_p(4098)) == -2 and fwd(rows=1 << 41) == -2
    assert fwd(rows=0) == 0
    assert bwd(dxs=7) == -2 and bwd(mean=None) == -1 and bwd(ws=None) == -1 and bwd(ws=ctypes.c_void_p(4100)) == -2
    assert bwd(size=63) == -2 and b"too small" in L.w2v_last_error() and bwd(dx=None) == -1
    assert L.w2v_layer_norm_backward_workspace(0, 3, 8) == 64
    assert L.w2v_layer_norm_backward_workspace(7, 3, 8) == 0
    cpu = torch.zeros(2, 4)
    with pytest.raises(TypeError):
        w2v.layer_norm(cpu)
