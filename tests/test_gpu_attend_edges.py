"""Attention over texts where values are extreme: words without any weight, masks of the type's lowest value, scores and
gradients far from one, infinities and NaN beside what is shown."""
import math

import pytest
import torch

from attend_reference import E_SUM, ROUND, attend_reference, check
from paper_1606_08495_amd import w2v
from test_gpu_attend import offsets_of, rows, whole

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
NAMES = ("out", "lse", "dq", "dk", "dv", "dbias")


def device_offsets(lengths):
    return torch.tensor(offsets_of(lengths), dtype=torch.int64, device="cuda")


def compare(got, ref, ty):
    for t, name in zip(got, NAMES):
        check(t, ref, name, F32 if name in ("lse", "dbias") else ty)


def by_distance(before, own, after, span=1):
    """A map and a bias of one head with one value for words before, one for the word itself, one for words after."""
    bmap = torch.tensor([0] * span + [1] + [2] * span, dtype=torch.int32)
    return torch.tensor([[before, own, after]]), bmap


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
def test_words_that_an_infinite_bias_leaves_nothing(ty):
    """The first word of each text sees itself alone, and its bias takes that away: no output, no part in any gradient, also where
    rows are formed again because a word that nobody is shown holds NaN."""
    lengths, H, d = [40, 1, 130], 2, 60
    T = sum(lengths)
    q, k, v, dout = rows(T, H, 1, d, ty, 11)
    bias, bmap = by_distance(0.5, -math.inf, 0.0)
    bias = bias.repeat(H, 1)
    keep = torch.ones(T, dtype=torch.uint8)
    keep[[3, 40, 100]] = 0
    see = dict(left=None, right=0)
    ref = attend_reference(q, k, v, offsets_of(lengths), keep=keep, bias=bias, buckets=bmap, dout=dout, **see)
    assert ref["lse"][0, 0] == -math.inf
    for bad in (0.0, math.nan, math.inf):
        k[keep == 0], v[keep == 0] = bad, bad
        got = whole(q.cuda(), k.cuda(), v.cuda(), dout.cuda(), device_offsets(lengths), keep=keep.cuda(), bias=bias.cuda(),
                    buckets=bmap.cuda(), **see)
        compare(got, ref, ty)
    k[5], v[50] = math.nan, math.inf                         # words that later ones are shown: the first words stay as they are
    got = whole(q.cuda(), k.cuda(), v.cuda(), dout.cuda(), device_offsets(lengths), keep=keep.cuda(), bias=bias.cuda(),
                buckets=bmap.cuda(), **see)
    for at in (0, 40, 41):
        assert not got[0][at].any() and not got[2][at].any() and (got[1][:, at] == -math.inf).all()
    assert not got[3][40].any() and not got[4][40].any()     # a text of one word


FAR = [torch.finfo(F32).min, -1e30, -1e37, -1e9, -3e5, 1e9]


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("low", FAR)
def test_words_that_see_only_what_a_finite_mask_hides(low, ty):
    """A word's own place carries a mask of a finite value.  Where others are shown, the mask leaves it no weight (or, where it is
    positive, all of it); the first word of a text has nothing else and weighs itself with one."""
    lengths, H, d = [140, 1, 3, 300, 33], 2, 60
    T, off = sum(lengths), offsets_of(lengths)
    first = torch.tensor(off[:-1])
    q, k, v, dout = rows(T, H, 2, d, ty, 12)
    bias, bmap = by_distance(0.0, low, 0.0)
    for see in (dict(left=None, right=0), dict(left=20, right=0, sinks=2)):
        if low < 0:                                          # as with the word itself left out, but for the first words
            ref = attend_reference(q, k, v, off, skip_self=True, dout=dout, **see)
            u, one = ROUND[ty], [t[first].double() for t in (q, k, v, dout)]
            rough = (u + E_SUM) * 2 * (one[3].abs() * one[2].abs()).sum(2, keepdim=True)      # of dS, with a weight of one
            for name, t in (("out", one[2]), ("dv", one[3])):
                ref[name][first] += t
                ref[name + "_bound"][first] += (2 * u + E_SUM) * t.abs()
            ref["dq_bound"][first] += d ** -0.5 * rough * one[1].abs()
            ref["dk_bound"][first] += d ** -0.5 * rough * one[0].abs()
        else:
            ref = attend_reference(q, k, v, off, left=0, right=0, dout=dout)
        # scores beside a mask: theirs is all that the logarithm says
        own = (q[:, :, None] * k[:, :, None]).double().sum(3)[:, :, 0].T * d ** -0.5 + low
        at = first if low < 0 else torch.arange(T)
        ref["lse"][:, at], ref["lse_bound"][:, at] = own[:, at], 2.0 ** -21 * own[:, at].abs()
        got = whole(q.cuda(), k.cuda(), v.cuda(), dout.cuda(), torch.tensor(off, device="cuda"), bias=bias.repeat(H, 1).cuda(),
                    buckets=bmap.cuda(), **see)
        compare(got[:5], ref, ty)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("low", FAR[:3])
def test_texts_that_a_finite_mask_hides_wholly(low, ty):
    """Every word carries the mask: scores are lost beside it (in 64 bits too), and all weights are equal."""
    n, H, d = 300, 2, 48
    q, k, v, dout = rows(n, H, 1, d, ty, 13)
    u, scale = ROUND[ty], d ** -0.5
    bias, bmap = torch.full((H, 2), low), w2v.relative_buckets(2, 5, device="cpu")
    got = whole(q.cuda(), k.cuda(), v.cuda(), dout.cuda(), device_offsets([n]), bias=bias.cuda(), buckets=bmap.cuda())
    Q, K, V, G = [t.double() for t in (q, k[:, 0], v[:, 0], dout)]
    ref = dict(dk=torch.zeros(n, 1, d), dv=torch.zeros(n, 1, d), dk_bound=torch.zeros(n, 1, d), dv_bound=torch.zeros(n, 1, d))
    ref = {name: t.double() for name, t in ref.items()}
    ref.update({name: torch.zeros(n, H, d, dtype=torch.float64) for name in ("out", "dq", "out_bound", "dq_bound")})
    for h in range(H):
        o = V.mean(0)
        delta, size = G[:, h] @ o, G[:, h].abs() @ o.abs()
        ds = (G[:, h] @ V.T - delta[:, None]) / n
        rough = ((G[:, h].abs() @ V.abs().T + size[:, None]) * E_SUM + u * size[:, None]) / n + (u + E_SUM) * ds.abs()
        ref["out"][:, h], ref["out_bound"][:, h] = o, (u + E_SUM) * V.abs().mean(0) + u * o.abs()
        ref["dq"][:, h], ref["dq_bound"][:, h] = scale * ds @ K, scale * rough @ K.abs()
        ref["dk"][:, 0] += scale * ds.T @ Q[:, h]
        ref["dk_bound"][:, 0] += scale * rough.T @ Q[:, h].abs()
        ref["dv"][:, 0] += G[:, h].mean(0)
        ref["dv_bound"][:, 0] += (u + E_SUM) * G[:, h].abs().mean(0)
    for name in ("dq", "dk", "dv"):
        ref[name + "_bound"] += u * ref[name].abs()
    ref["lse"] = torch.full((H, n), low, dtype=torch.float64)
    ref["lse_bound"] = 2.0 ** -21 * ref["lse"].abs()
    compare(got[:5], ref, ty)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, BF16])
def test_scores_of_many_millions(ty):
    """Rows that one word takes wholly: its weight is one, whatever the scores' size."""
    n, H, d = 200, 2, 64
    q, k, v, dout = rows(n, H, H, d, ty, 14)
    q, k = q * 3000, k * 3000
    got = whole(q.cuda(), k.cuda(), v.cuda(), dout.cuda(), device_offsets([n]), right=0)
    ref = {name: torch.zeros(n, H, d, dtype=torch.float64) for name in ("out", "dq", "dk", "dv")}
    ref["lse"] = torch.zeros(H, n, dtype=torch.float64)
    for h in range(H):
        x = q[:, h].double() @ k[:, h].double().T / 8
        x = torch.where(torch.ones(n, n).tril() > 0, x, -math.inf)
        best, at = x.max(1)
        gap = x[1:].topk(2).values
        clear = torch.ones(n, dtype=torch.bool)
        clear[1:] = gap[:, 0] - gap[:, 1] > 1000             # (a score is off by 128 2^-24 of a few 10^8 at most)
        assert clear.all()
        ref["out"][:, h], ref["lse"][h] = v[at, h].double(), best
        ref["dv"][:, h].index_add_(0, at, dout[:, h].double())
    u = ROUND[ty]
    ref["out_bound"], ref["lse_bound"] = (2 * u + E_SUM) * ref["out"].abs(), 2.0 ** -19 * ref["lse"].abs()
    ref["dv_bound"] = u * ref["dv"].abs()
    for h in range(H):
        at = (torch.where(torch.ones(n, n).tril() > 0, q[:, h].double() @ k[:, h].double().T, -math.inf)).argmax(1)
        ref["dv_bound"][:, h].index_add_(0, at, 2 * (u + E_SUM) * dout[:, h].double().abs())
    compare((got[0], got[1]), ref, ty)
    check(got[4], ref, "dv", ty)
    # dS = p (dP - delta) with p = 1: what the rounding of delta leaves, times rows of some thousands
    size = (dout.double().abs() * v.double().abs().max()).sum(2).max()
    for t in got[2:4]:
        assert float(t.double().abs().max()) <= float(n * (2 * u + E_SUM) * size * q.double().abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1.0, 1e-3, 1e-4, 1e-5, 3e3])
@pytest.mark.parametrize("d", [32, 100])
def test_small_and_large_gradients_in_16_bits(d, size):
    """Gradients of fp16 outputs as training has them: a mean over thousands of words, or a scaled loss.  What is rounded on the way
    must not cost more than the results' own rounding, whatever the size."""
    lengths = [3000, 200]
    T, off = sum(lengths), offsets_of(lengths)
    q, k, v, dout = rows(T, 1, 1, d, F16, 15)
    dout = (dout * size).to(F16)
    with torch.device("cuda"):
        ref = attend_reference(*[t.cuda() for t in (q, k, v)], off, right=0, dout=dout.cuda())
    ref = {name: t.cpu() for name, t in ref.items()}
    got = whole(q.cuda(), k.cuda(), v.cuda(), dout.cuda(), torch.tensor(off, device="cuda"), right=0)
    compare(got, ref, F16)
    for t, name in zip(got[2:], ("dq", "dk", "dv")):
        exact = ref[name]
        own = float((exact.to(F16).double() - exact).norm() / exact.norm())
        # beside the result's rounding: dS's and delta's, relative ones of 2^-11 at most, of terms that add up at random
        assert float((t.double().cpu() - exact).norm() / exact.norm()) <= 1.2 * own + 2.0 ** -11, name


@pytest.mark.gpu
def test_small_weights_in_16_bits():
    """One word far above very many others that share a part of the weight: theirs are 2^-26 of the largest."""
    n, d = 1 << 17, 16
    q, k, v = torch.zeros(n, 1, d), torch.zeros(n, 1, d), torch.ones(n, 1, d)
    q[-1, 0, 0], k[0, 0, 0], v[0] = 8.0, 26 * math.log(2) / 2, 0.0       # scale 1/4: 26 ln 2 above the rest
    out, _ = w2v.attend(q.to(F16).cuda(), k.to(F16).cuda(), v.to(F16).cuda(), device_offsets([n]), right=0)
    x = 2 * float(k[0, 0, 0].to(F16))
    want = (n - 1) * math.exp(-x) / (1 + (n - 1) * math.exp(-x))         # about 2^-9
    assert torch.allclose(out[-1].double().cpu(), torch.full((1, d), want, dtype=torch.float64), rtol=2.0 ** -9, atol=0)


def strict(q, k, v, dout, see):
    """dq of one text and its bound where delta is not taken from outputs that were rounded."""
    r = attend_reference(q, k, v, [0, q.shape[0]], dout=dout, **see)
    n, d, u = q.shape[0], q.shape[2], ROUND[q.dtype]
    Q, K, V, G = [t[:, 0].double() for t in (q, k, v, dout)]
    i, j = torch.arange(n)[:, None], torch.arange(n)[None]
    x = torch.where((j <= i) & (j >= i - see["left"]), d ** -0.5 * Q @ K.T, -math.inf)
    p = torch.softmax(x, 1)
    o = p @ V
    E = d * 2.0 ** -24 * d ** -0.5 * (Q.abs() @ K.abs().T).max(1, keepdim=True).values + 2.0 ** -21 * 10
    ds = p * (G @ V.T - (G * o).sum(1, keepdim=True))
    err = p * (4 * E + E_SUM) * (G.abs() @ V.abs().T + (G.abs() * o.abs()).sum(1, keepdim=True)) + (u + E_SUM) * ds.abs()
    return dict(dq=r["dq"], dq_bound=(d ** -0.5 * err @ K.abs() + u * r["dq"][:, 0].abs())[:, None])


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F16, BF16])
def test_gradients_of_a_short_text_do_not_depend_on_its_neighbours(ty):
    """Few words, one of which takes nearly all: what the rounding of the output would cost shows."""
    n, d, see = 40, 16, dict(left=2, right=0)
    q, k, v, dout = rows(n, 1, 1, d, ty, 16)
    q = k = (q * 1.25).to(ty)
    ref = strict(q, k, v, dout, see)
    for before, after in ((0, 0), (4000, 0), (4000, 1500), (77, 900)):
        a, b = [[t[:m] for t in rows(max(m, 1), 1, 1, d, ty, 17)] for m in (before, after)]
        parts = [torch.cat([x, y, z]).cuda() for x, y, z in zip(a, (q, k, v, dout), b)]
        for left in (2, None):
            off = device_offsets([before, n, after])
            out, lse = w2v.attend(*parts[:3], off, left=left, right=0)
            dq = w2v.attend_backward(parts[3], *parts[:3], out, lse, off, left=left, right=0)[0]
            if left:
                check(dq[before:before + n], ref, "dq", ty)
            else:
                r = strict(q, k, v, dout, dict(left=n, right=0))
                check(dq[before:before + n], r, "dq", ty)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("d", [16, 60, 100, 128])
def test_what_dropped_words_hold_changes_no_bit(d, ty):
    """Their rows are taken as zeros on the way in: no row is formed again for them."""
    lengths, H = [300, 5, 200, 0, 400], 4
    T = sum(lengths)
    q, k, v, dout = [t.cuda() for t in rows(T, H, 2, d, ty, 18)]
    keep = (torch.rand(T, generator=torch.Generator().manual_seed(19)) > 0.3).to(torch.uint8).cuda()
    bias, bmap = torch.randn(H, 8, device="cuda"), w2v.relative_buckets(8, 30)
    for see in (dict(left=None, right=0), dict(left=40, right=3, sinks=4, bias=bias, buckets=bmap)):
        want = None
        for bad in (0.0, 1.5, math.inf, math.nan):
            k[keep == 0], v[keep == 0] = bad, bad
            got = whole(q, k, v, dout, device_offsets(lengths), keep=keep, **see)
            want = want or got
            assert all(torch.equal(a, b) for a, b in zip(got, want)), bad


@pytest.mark.gpu
@pytest.mark.parametrize("buckets", [0, 8])
def test_sums_over_many_words_in_32_bits(buckets):
    """Sums of 30000 terms: a piece of at most 64 words first, 470 such sums one after the other.  A random walk of N steps gathers
    about 0.6 2^-24 sqrt(N / 2) of its end's size: 5e-7 for the pieces' sums and 2e-7 within one; all 30000 in a row would gather
    3e-6."""
    n, d = 30000, 16
    q, k, v, dout = [t.cuda() for t in rows(n, 1, 1, d, F32, 20)]
    see = dict(bias=torch.randn(1, buckets, device="cuda"), buckets=w2v.relative_buckets(buckets, 100)) if buckets else {}
    got = whole(q, k, v, dout, device_offsets([n]), **see)[:3]
    Q, K, V, G = [t[:, 0].double() for t in (q, k, v, dout)]
    o, dq = torch.empty(n, d, dtype=torch.float64, device="cuda"), torch.empty(n, d, dtype=torch.float64, device="cuda")
    for a in range(0, n, 2000):
        x = Q[a:a + 2000] @ K.T.contiguous() / 4
        if buckets:
            dist = (torch.arange(n, device="cuda")[None] - torch.arange(a, min(n, a + 2000), device="cuda")[:, None]).clamp(-100, 100)
            x = x + see["bias"][0].double()[see["buckets"].long()[dist + 100]]
        p = torch.softmax(x, 1)
        o[a:a + 2000] = p @ V
        ds = p * (G[a:a + 2000] @ V.T.contiguous() - (G[a:a + 2000] * o[a:a + 2000]).sum(1, keepdim=True))
        dq[a:a + 2000] = ds @ K / 4
    for t, exact in ((got[0], o), (got[2], dq)):
        assert float((t[:, 0].double() - exact).norm() / exact.norm()) <= 1.5e-6


# spans on both sides of the one where a block of two halves no longer has room for its sums by distance, for each width and type
ROOM = [(BF16, 20, 971), (F16, 32, 971), (BF16, 60, 742), (F16, 64, 742), (BF16, 96, 589), (F16, 100, 359), (BF16, 128, 359),
        (F32, 32, 742), (F32, 64, 781)]


@pytest.mark.gpu
@pytest.mark.parametrize("ty,d,span", ROOM)
def test_spans_around_the_room_of_a_block(ty, d, span):
    lengths = [70, 9]
    q, k, v, dout = rows(sum(lengths), 2, 1, d, ty, 21)
    for s in list(range(span - 4, span + 5)) + list(range(span + 5, min(span + 40, 1023), 5)) + [1023]:
        bias, bmap = torch.randn(2, 32, generator=torch.Generator().manual_seed(s)), w2v.relative_buckets(32, s, device="cpu")
        ref = attend_reference(q, k, v, offsets_of(lengths), bias=bias, buckets=bmap, dout=dout)
        print("span", ty, d, s, flush=True)
        got = whole(q.cuda(), k.cuda(), v.cuda(), dout.cuda(), device_offsets(lengths), bias=bias.cuda(), buckets=bmap.cuda())
        compare(got, ref, ty)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, BF16])
def test_not_a_number_reaches_exactly_what_it_is_shown_to(ty):
    """One key, one value or one query that is not a number, or an infinite score: forward and back, every column that the formulas
    give it and no other."""
    T, H, d, see = 400, 2, 60, dict(left=30, right=4, sinks=2)
    q, k, v, dout = [t.cuda() for t in rows(T, H, 1, d, ty, 22)]
    off = torch.tensor([0, 250, 400], dtype=torch.int64, device="cuda")
    i, j = torch.arange(T, device="cuda")[:, None], torch.arange(T, device="cuda")[None]
    first = torch.where(torch.arange(T, device="cuda") < 250, 0, 250)
    shown = (first[:, None] == first[None]) & (j <= i + 4) & ((j >= i - 30) | (j - first[None] < 2))
    clean = whole(q, k, v, dout, off, **see)
    for at in (1, 120, 399):
        for what, bad in (("k", math.nan), ("k", math.inf), ("v", math.nan), ("q", math.nan)):
            a = dict(q=q.clone(), k=k.clone(), v=v.clone())
            if bad == math.inf:
                a["q"][..., 3] = 1.0
                base = whole(a["q"], k, v, dout, off, **see)
            else:
                base = clean
            if what == "v" or bad == math.inf:
                a[what][at, :, 3] = bad
            else:
                a[what][at] = bad
            out, lse, dq, dk, dv = whole(a["q"], a["k"], a["v"], dout, off, **see)
            queries = shown[:, at] if what != "q" else torch.arange(T, device="cuda") == at
            keys = (shown & queries[:, None]).any(0)
            if what == "v":                                   # its own column forward; dP, and with it all of dS, back
                column = torch.arange(d, device="cuda") == 3
                assert torch.isnan(out[queries][..., column]).all() and torch.isfinite(lse).all()
                assert torch.isfinite(out[..., ~column]).all() and torch.isfinite(dv).all()
            else:
                assert torch.isnan(out[queries]).all() and torch.isnan(lse[:, queries]).all() and torch.isnan(dv[keys]).all()
            assert torch.isnan(dq[queries]).all() and torch.isnan(dk[keys]).all()
            u = {F32: 1e-5, BF16: 2e-2}[ty]
            for t, ref, rest in ((out, base[0], ~queries), (dq, base[2], ~queries), (dk, base[3], ~keys), (dv, base[4], ~keys)):
                assert torch.allclose(t[rest].float(), ref[rest].float(), rtol=u, atol=u), (at, what, bad)
