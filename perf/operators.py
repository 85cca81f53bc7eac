"""Performance cases of the context operators: what a program that reads words in their context calls.

A word vector says what a word means on average; what it means in one text is read from the words around it.
Three operators do that over the vectors of a block of texts: layer norm of the rows, attention of every
word over the words that its window shows it (a few first words of the text may stay visible), with a
learned bias by buckets of relative distance, and attention of one new word over the cached keys and
values of its text.  The first two are trained, the third serves.

A case is a dict of plain values.  ``listed()`` names the standing ones, ``draw()`` makes more from the same
ranges, ``prepare()`` makes what a program holds before the call, ``run()`` is one pass, ``work()`` the bytes and
operations such a pass cannot do without, ``exact()`` the same outputs in 64 bits from the definitions.
Where ``own`` is false ``run()`` computes in elementary torch operations in 32 bits; where it is true it calls the
public entry points of ``paper_1606_08495_amd.w2v``.

Kinds:
  norm        layer norm of rows; with train, and its gradients
  attend      attention over texts; with train, and its gradients
  step        attention of one new word per text over a cache
"""
import math
import random

import torch

own = False

TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
EPS = 1e-5
ELEMENTS = 1 << 28           # scores that the plain form holds at a time


def listed():
    return [
        # A minibatch of the paper's size, 200 input words of 300 columns: a call is its launches.
        dict(name="norm-200", kind="norm", type="float32", rows=200, d=300, train=False),
        # The vectors of 2^20 pairs in 16 bits, as the benchmark's minibatch has them.
        dict(name="norm-2^20", kind="norm", type="bfloat16", rows=1 << 20, d=300, train=False),
        # A training step's norm over a block of text, whole vectors.
        dict(name="norm-train-300", kind="norm", type="float32", rows=1 << 17, d=300, train=True),
        # Wide rows of odd length, as of hidden vectors beside the word vectors.
        dict(name="norm-train-wide", kind="norm", type="bfloat16", rows=8191, d=4101, train=True),
        # One short text, trained on by itself: five heads of 60 columns, the column slices of 300.
        dict(name="text-20", kind="attend", type="float32", texts=1, low=20, high=20, heads=5, kv_heads=5, d=60,
             left=10, right=10, sinks=0, skip=True, buckets=32, span=16, drop=0.0, train=True),
        # A block of short texts read in their windows, some words dropped as subsampling drops them.
        dict(name="texts-10-40", kind="attend", type="float32", texts=5243, low=10, high=40, heads=5, kv_heads=5,
             d=60, left=10, right=10, sinks=0, skip=True, buckets=32, span=16, drop=0.1, train=False),
        # The same block trained on, with the bias.
        dict(name="texts-train", kind="attend", type="float32", texts=2621, low=10, high=40, heads=5, kv_heads=5,
             d=60, left=10, right=10, sinks=0, skip=True, buckets=32, span=16, drop=0.1, train=True),
        # One long text, causal, read in a window of 1024 words with its first four visible; shared key heads.
        dict(name="window-32768", kind="attend", type="bfloat16", texts=1, low=32768, high=32768, heads=16,
             kv_heads=4, d=128, left=1023, right=0, sinks=4, skip=False, buckets=0, span=0, drop=0.0, train=False),
        # Long texts of unequal length in a window of 512, trained on with bias.
        dict(name="window-train", kind="attend", type="bfloat16", texts=5, low=1800, high=4900, heads=8, kv_heads=2,
             d=64, left=511, right=0, sinks=4, skip=False, buckets=32, span=128, drop=0.0, train=True),
        # Whole texts, causal, heads of a width that is no power of two.
        dict(name="whole-train", kind="attend", type="float16", texts=3, low=1500, high=4100, heads=6, kv_heads=6,
             d=100, left=-1, right=0, sinks=0, skip=False, buckets=0, span=0, drop=0.0, train=True),
        # One user's session, one new word.
        dict(name="step-1", kind="step", type="float32", batch=1, low=500, high=500, room=512, heads=5, kv_heads=5,
             d=60, left=-1, sinks=0, skip=False, buckets=32, span=128),
        # Many texts served at once, unequal and long.
        dict(name="step-32", kind="step", type="bfloat16", batch=32, low=300, high=32768, room=32768, heads=32,
             kv_heads=8, d=128, left=-1, sinks=0, skip=False, buckets=0, span=0),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "attend", "attend", "attend", "step", "step"])
    ty = rng.choice(sorted(TYPES))
    if kind == "norm":
        train = rng.random() < 0.5
        d = _spread(rng, 4, 8192)
        most = (1 << 27) // d if train else (1 << 28) // d
        return dict(kind=kind, type=ty, rows=_spread(rng, 1, min(most, 1 << 20)), d=d, train=train)
    d = rng.choice([16, 32, 37, 48, 60, 64, 80, 96, 100, 128, rng.randint(8, 128)])
    kv = rng.choice([1, 2, 4, 5, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4])
    if kind == "step":
        room = _spread(rng, 16, 32768)
        batch = _spread(rng, 1, 64)
        while batch * room * kv * d > 32 * 32768 * 8 * 128 // 4 or batch * room * heads > 1 << 25:
            batch = max(1, batch // 2)
            room = max(16, room // 2)
        low = rng.randint(1, room)
        windowed = rng.random() < 0.4
        biased = rng.random() < 0.4
        return dict(kind=kind, type=ty, batch=batch, low=low, high=room, room=room, heads=heads, kv_heads=kv, d=d,
                    left=_spread(rng, 1, room) if windowed else -1, sinks=rng.choice([0, 4, 7]) if windowed else 0,
                    skip=False, buckets=rng.choice([8, 32]) if biased else 0,
                    span=rng.choice([20, 128, 500]) if biased else 0)
    train = rng.random() < 0.5
    biased = rng.random() < 0.5
    if rng.random() < 0.5:                       # short texts in their windows, both sides
        low = rng.randint(1, 30)
        high = low + rng.randint(0, 60)
        window = rng.randint(1, 15)
        texts = _spread(rng, 1, 5000)
        while texts * high * heads > 600_000 or texts * (low + high) // 2 > 131072:
            texts = texts // 2 + 1 if texts > 1 else 1
            if texts == 1:
                break
        return dict(kind=kind, type=ty, texts=texts, low=low, high=high, heads=heads, kv_heads=kv, d=d, left=window,
                    right=rng.choice([window, 0]), sinks=rng.choice([0, 0, 1, 3]), skip=rng.random() < 0.5,
                    buckets=32 if biased else 0, span=rng.choice([16, 40]) if biased else 0,
                    drop=rng.choice([0.0, 0.1, 0.5]), train=train)
    high = _spread(rng, 100, 16384)              # longer texts, whole or in a long window, mostly causal
    low = max(1, high // rng.randint(1, 4))
    texts = rng.randint(1, max(1, min(6, 16384 // high)))
    left = rng.choice([-1, _spread(rng, 16, 2048), _spread(rng, 16, 2048)])
    while texts * high * heads * min(high, left + 1 if left >= 0 else high) > (1 << 29) // (2 if train else 1):
        if kv > 1:
            heads, kv = heads // kv, 1
        else:
            high = high // 2
            low = min(low, high)
    return dict(kind=kind, type=ty, texts=texts, low=low, high=high, heads=heads, kv_heads=kv, d=d, left=left,
                right=rng.choice([0, 0, left]), sinks=rng.choice([0, 1, 4, 33]) if left >= 0 else 0, skip=False,
                buckets=rng.choice([8, 32]) if biased else 0, span=rng.choice([60, 128, 500]) if biased else 0,
                drop=rng.choice([0.0, 0.0, 0.2]), train=train)


def lengths(case):
    """Lengths of a case's texts: part of the case, the same for every seed."""
    n = case["texts"] if case["kind"] == "attend" else case["batch"]
    rng = random.Random(n * 1_000_003 + case["low"] * 1009 + case["high"])
    out = [rng.randint(case["low"], case["high"]) for _ in range(n)]
    out[0] = case["high"]
    return out


def bucket_map(buckets, span):
    """Bucket of every distance -span..span: one half of the buckets for words before, one for words after;
    in each, the first half of the distances one by one and the rest by their logarithm."""
    half = buckets // 2
    near = max(1, half // 2)
    far = half - near

    def of(r):
        if r < near or far == 0:
            return min(r, half - 1)
        t = 0                                    # largest t < far with near (span / near)^(t / far) <= r
        while t + 1 < far and span ** (t + 1) * near ** far <= r ** far * near ** (t + 1):
            t += 1
        return near + t
    return [of(-r) for r in range(-span, 1)] + [half + of(r) for r in range(1, span + 1)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ty = TYPES[case["type"]]

    def normal(*shape, scale=1.0, shift=0.0, to=None):
        x = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(shift, scale, generator=g)
        return x.to(to or ty)

    s = dict(case=case)
    if case["kind"] == "norm":
        m, d = case["rows"], case["d"]
        s.update(x=normal(m, d, scale=1.5, shift=0.3), gain=normal(d, scale=0.2, shift=1.0, to=torch.float32),
                 offset=normal(d, scale=0.2, to=torch.float32))
        if case["train"]:
            s.update(dy=normal(m, d))
        return s
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    if case["buckets"]:
        s.update(bias=normal(H, case["buckets"], to=torch.float32),
                 buckets=torch.tensor(bucket_map(case["buckets"], case["span"]), dtype=torch.int32, device="cuda"))
    else:
        s.update(bias=None, buckets=None)
    n = lengths(case)
    if case["kind"] == "step":
        B, room = case["batch"], case["room"]
        s.update(q=normal(B, H, d), k=torch.empty(B, room, G, d, dtype=ty, device="cuda"),
                 v=torch.empty(B, room, G, d, dtype=ty, device="cuda"),
                 n=torch.tensor(n, dtype=torch.int32, device="cuda"), longest=max(n))
        for b in range(B):                       # in parts: the cache may be most of the memory used
            s["k"][b].copy_(normal(room, G, d))
            s["v"][b].copy_(normal(room, G, d))
        return s
    offsets = [0]
    for x in n:
        offsets.append(offsets[-1] + x)
    T = offsets[-1]
    s.update(q=normal(T, H, d), k=normal(T, G, d), v=normal(T, G, d), offsets=offsets,
             sent_off=torch.tensor(offsets, dtype=torch.int64, device="cuda"), keep=None)
    if case["drop"]:
        s["keep"] = (torch.rand(T, generator=g, device="cuda") >= case["drop"]).to(torch.uint8)
    if case["train"]:
        s["dout"] = normal(T, H, d)
    return s


def work(case):
    size = torch.empty(0, dtype=TYPES[case["type"]]).element_size()
    if case["kind"] == "norm":
        m, d = case["rows"], case["d"]
        if not case["train"]:                    # x in, y and two statistics out
            return {"bytes": 2 * m * d * size + 8 * m + 8 * d, "flops": 8 * m * d}
        return {"bytes": 4 * m * d * size + 8 * m + 16 * d, "flops": 20 * m * d}      # x, dy in, y, dx out
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    n = lengths(case)
    left = case["left"] if case["left"] >= 0 else 1 << 40
    if case["kind"] == "step":
        seen = sum(min(x, min(left + 1, x) + min(case["sinks"], max(0, x - left - 1))) for x in n)
        return {"bytes": (2 * seen * G * d + 2 * case["batch"] * H * d) * size + 4 * case["batch"],
                "flops": 4 * seen * H * d}
    right = case["right"] if case["right"] >= 0 else 1 << 40
    pairs = 0
    for x in n:
        a, b = min(left, x - 1), min(right, x - 1)
        # words within the window, and the first words that it no longer shows
        pairs += x + (a * x - a * (a + 1) // 2) + (b * x - b * (b + 1) // 2) - (x if case["skip"] else 0)
        pairs += sum(min(case["sinks"], i - left) for i in range(left + 1, min(x, left + case["sinks"] + 1)))
        pairs += case["sinks"] * max(0, x - (left + case["sinks"] + 1))
    pairs = int(pairs * (1 - case["drop"]))
    T = sum(n)
    moved = T * d * (2 * H + 2 * G) * size + T * (1 if case["drop"] else 0) + 8 * (len(n) + 1) + 4 * T * H
    if not case["train"]:                        # q, k, v in, the outputs and the rows' logarithms out
        return {"bytes": moved, "flops": 4 * pairs * H * d}
    # forward, and backward: q, k, v and the gradient of the outputs in, the gradients out; five products
    return {"bytes": moved + T * d * (2 * H + 2 * G) * size, "flops": 14 * pairs * H * d}


# ---- the plain form ------------------------------------------------------------------------------------

def _norm(s):
    case = s["case"]
    x = s["x"].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = 1.0 / ((xc * xc).mean(1) + EPS).sqrt()
    xhat = xc * rstd[:, None]
    y = (xhat * s["gain"] + s["offset"]).to(s["x"].dtype)
    if not case["train"]:
        return y, mean, rstd
    dy = s["dy"].float()
    t = dy * s["gain"]
    dx = rstd[:, None] * (t - t.mean(1)[:, None] - xhat * (t * xhat).mean(1)[:, None])
    return y, mean, rstd, dx.to(s["x"].dtype), (dy * xhat).sum(0), dy.sum(0)


def _tile(case, q, k, v, do, bias, dist, seen, onehot):
    """One padded batch: q, do [N, H, a, d], k, v [N, H, b, d] in 32 bits, seen [N, 1, a, b], bias [H, a, b] or None."""
    scale = 1.0 / math.sqrt(case["d"])
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
    if bias is not None:
        x = x + bias
    x = x.masked_fill(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    lse = (m + torch.log(total)).squeeze(-1)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    out = torch.matmul(p, v)
    if do is None:
        return out, lse
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), do)
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = p * (dp - (do * out).sum(-1, keepdim=True))
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q) * scale
    db = None
    if onehot is not None:
        db = torch.matmul(ds.sum(0).flatten(1), onehot)
    return out, lse, dq, dk, dv, db


def _seen(case, i, j):
    """Whether word i of a text is shown its word j."""
    left = case["left"] if case["left"] >= 0 else 1 << 40
    right = case["right"] if case.get("right", -1) >= 0 else 1 << 40
    ok = (j <= i + right) & ((j >= i - left) | (j < case["sinks"]))
    return ok & (i != j) if case["skip"] else ok


def _attend(s):
    case = s["case"]
    H, G, d, train = case["heads"], case["kv_heads"], case["d"], case["train"]
    T, dev = s["q"].shape[0], s["q"].device
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    do = s["dout"].float() if train else None
    if H != G:
        k, v = k.repeat_interleave(H // G, 1), v.repeat_interleave(H // G, 1)
    keep = s["keep"].bool() if s["keep"] is not None else torch.ones(T, dtype=torch.bool, device=dev)
    out, lse = torch.empty_like(q), torch.empty(T, H, device=dev)
    if train:
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
        db = torch.zeros_like(s["bias"]) if s["bias"] is not None else None

    def biased(dist):
        if s["bias"] is None:
            return None, None
        b = s["buckets"].long()[dist.clamp(-case["span"], case["span"]) + case["span"]]
        onehot = (b.flatten()[:, None] == torch.arange(case["buckets"], device=dev)).float() if train else None
        return s["bias"][:, b], onehot

    off = s["offsets"]
    if max(lengths(case)) <= 128:                # short texts: all of them padded to the longest, in parts
        L = max(lengths(case))
        at = torch.arange(L, device=dev)
        dist = at[None, :] - at[:, None]
        bias, onehot = biased(dist)
        window = _seen(case, at[:, None], at[None, :])
        part = max(1, ELEMENTS // (H * L * max(L, d)))
        for a in range(0, case["texts"], part):
            first = s["sent_off"][a:a + part + 1]
            idx = first[:-1, None] + at
            real = idx < first[1:, None]
            idx = torch.where(real, idx, torch.zeros_like(idx))
            seen = (window[None] & real[:, :, None] & (real & keep[idx])[:, None, :])[:, None]
            got = _tile(case, *[None if x is None else x[idx].transpose(1, 2).contiguous() for x in (q, k, v, do)],
                        bias, dist, seen, onehot)
            rows = idx[real]
            out[rows] = got[0].transpose(1, 2)[real]
            lse[rows] = got[1].transpose(1, 2)[real]
            if train:
                dq[rows], dk[rows], dv[rows] = [x.transpose(1, 2)[real] for x in got[2:5]]
                if db is not None:
                    db += got[5]
    else:                                        # long texts one by one, blocks of queries
        for a, b in zip(off[:-1], off[1:]):
            for i0 in range(a, b, 512):
                i1 = min(b, i0 + 512)
                j0 = max(a, i0 - case["left"]) if case["left"] >= 0 else a
                j1 = min(b, i1 + case["right"]) if case["right"] >= 0 else b
                i = torch.arange(i0, i1, device=dev)
                j = torch.cat([torch.arange(a, min(a + case["sinks"], j0), device=dev), torch.arange(j0, j1, device=dev)])
                dist = j[None, :] - i[:, None]
                bias, onehot = biased(dist)
                seen = (_seen(case, i[:, None] - a, j[None, :] - a) & keep[j][None, :])[None, None]
                got = _tile(case, *[None if x is None else x[w].transpose(0, 1).contiguous()[None]
                                    for x, w in ((q, i), (k, j), (v, j), (do, i))], bias, dist, seen, onehot)
                out[i0:i1] = got[0][0].transpose(0, 1)
                lse[i0:i1] = got[1][0].transpose(0, 1)
                if train:
                    dq[i0:i1] = got[2][0].transpose(0, 1)
                    dk[j] += got[3][0].transpose(0, 1)
                    dv[j] += got[4][0].transpose(0, 1)
                    if db is not None:
                        db += got[5]
    ty = s["q"].dtype
    lse = lse.transpose(0, 1).contiguous()
    if not train:
        return out.to(ty), lse
    if H != G:
        dk, dv = [x.view(T, G, H // G, d).sum(2) for x in (dk, dv)]
    res = [out.to(ty), lse, dq.to(ty), dk.to(ty), dv.to(ty)]
    return res + [db] if db is not None else res


def _step(s):
    case = s["case"]
    B, H, G, d, dev = case["batch"], case["heads"], case["kv_heads"], case["d"], s["q"].device
    L = s["longest"]
    at = torch.arange(L, device=dev)
    out = torch.empty(B, H, d, device=dev)
    part = max(1, ELEMENTS // (L * G * d))
    for a in range(0, B, part):
        q = s["q"][a:a + part].float().view(-1, G, H // G, d)
        k = s["k"][a:a + part, :L].float().transpose(1, 2)
        v = s["v"][a:a + part, :L].float().transpose(1, 2).contiguous()
        last = s["n"][a:a + part].long()[:, None] - 1
        x = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(d)
        if s["bias"] is not None:
            b = s["buckets"].long()[(at[None] - last).clamp(-case["span"], case["span"]) + case["span"]]
            x = x + s["bias"][:, b].transpose(0, 1).reshape(x.shape)
        seen = _seen(dict(case, right=0), last, at[None]) & (at[None] <= last)
        x = x.masked_fill(~seen[:, None, None], -math.inf)
        p = torch.exp(x - x.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        out[a:a + part] = torch.matmul(p, v).reshape(-1, H, d)
    return out.to(s["q"].dtype)


# ---- a pass -----------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if not own:
        return {"norm": _norm, "attend": _attend, "step": _step}[case["kind"]](s)
    from paper_1606_08495_amd import w2v
    if case["kind"] == "norm":
        y, mean, rstd = w2v.layer_norm(s["x"], s["gain"], s["offset"], EPS)
        if not case["train"]:
            return y, mean, rstd
        return (y, mean, rstd) + w2v.layer_norm_backward(s["dy"], s["x"], s["gain"], mean, rstd)
    left = case["left"] if case["left"] >= 0 else None
    if case["kind"] == "step":
        return w2v.attend_step(s["q"], s["k"], s["v"], s["n"], left=left, sinks=case["sinks"], skip_self=case["skip"],
                               bias=s["bias"], buckets=s["buckets"])
    see = dict(left=left, right=case["right"] if case["right"] >= 0 else None, sinks=case["sinks"],
               skip_self=case["skip"], keep=s["keep"], bias=s["bias"], buckets=s["buckets"])
    out, lse = w2v.attend(s["q"], s["k"], s["v"], s["sent_off"], **see)
    if not case["train"]:
        return out, lse
    grads = w2v.attend_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, s["sent_off"], **see)
    return [out, lse] + [x for x in grads if x is not None]


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def _exact_norm(s):
    x, gain, offset = s["x"].double(), s["gain"].double(), s["offset"].double()
    var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
    rstd = (var + EPS) ** -0.5
    z = (x - mean) * rstd
    res = (z * gain + offset, mean[:, 0], rstd[:, 0])
    if not s["case"]["train"]:
        return res
    dz = s["dy"].double() * gain
    n = x.shape[1]
    dx = rstd / n * (n * dz - dz.sum(1, keepdim=True) - z * (dz * z).sum(1, keepdim=True))
    return res + (dx, (s["dy"].double() * z).sum(0), s["dy"].double().sum(0))


def _exact_row_block(case, s, h, i, j, last):
    """Weights of head h, queries i over keys j (indices within the text, numbered from 0): probabilities and logarithms."""
    ok = (j[None, :] - i[:, None] <= (case["right"] if case.get("right", -1) >= 0 else 1 << 40)) & (j[None, :] < last)
    if case["left"] >= 0:
        ok &= (i[:, None] - j[None, :] <= case["left"]) | (j[None, :] < case["sinks"])
    if case["skip"]:
        ok &= i[:, None] != j[None, :]
    where = None
    if s["bias"] is not None:
        where = s["buckets"].long()[torch.clamp(j[None, :] - i[:, None], -case["span"], case["span"]) + case["span"]]
    return ok, where


def _exact_attend(s):
    case = s["case"]
    H, G, d, train = case["heads"], case["kv_heads"], case["d"], case["train"]
    T, dev, r = s["q"].shape[0], s["q"].device, H // G
    f = dict(dtype=torch.float64, device=dev)
    out, lse = torch.zeros(T, H, d, **f), torch.full((H, T), -math.inf, **f)
    dq, dk, dv = torch.zeros(T, H, d, **f), torch.zeros(T, G, d, **f), torch.zeros(T, G, d, **f)
    db = torch.zeros(H, case["buckets"] or 1, **f)
    groups = {}
    for a, b in zip(s["offsets"][:-1], s["offsets"][1:]):        # texts of one length are taken together
        groups.setdefault(b - a, []).append(a)
    for n, firsts in groups.items():
        first = torch.tensor(firsts, device=dev)
        step = max(1, min(n, (1 << 25) // (n * len(firsts))))
        for h in range(H):
            for i0 in range(0, n, step):
                i = torch.arange(i0, min(n, i0 + step), device=dev)
                j0 = max(0, i0 - case["left"]) if case["left"] >= 0 and case["sinks"] == 0 else 0
                j1 = min(n, i0 + step + case["right"]) if case["right"] >= 0 else n
                j = torch.arange(j0, j1, device=dev)
                ok, where = _exact_row_block(case, s, h, i, j, n)
                qi, kj = first[:, None] + i, first[:, None] + j
                q, k, v = s["q"][qi, h].double(), s["k"][kj, h // r].double(), s["v"][kj, h // r].double()
                ok = ok[None].expand(len(firsts), -1, -1)
                if s["keep"] is not None:
                    ok = ok & (s["keep"][kj] != 0)[:, None, :]
                z = torch.bmm(q, k.transpose(1, 2).contiguous()) * d ** -0.5
                if where is not None:
                    z = z + s["bias"][h].double()[where]
                z = torch.where(ok, z, -math.inf)
                l = torch.logsumexp(z, 2)
                p = torch.where(ok, torch.exp(z - torch.where(l == -math.inf, 0.0, l)[:, :, None]), 0.0)
                o = torch.bmm(p, v)
                out[qi, h], lse[h][qi] = o, l
                if not train:
                    continue
                g = s["dout"][qi, h].double()
                w = p * (torch.bmm(g, v.transpose(1, 2).contiguous()) - (g * o).sum(2)[:, :, None])
                dq[qi, h] = torch.bmm(w, k) * d ** -0.5
                dk[kj, h // r] += torch.bmm(w.transpose(1, 2).contiguous(), q) * d ** -0.5
                dv[kj, h // r] += torch.bmm(p.transpose(1, 2).contiguous(), g)
                if where is not None:
                    total = w.sum(0)
                    for c in range(case["buckets"]):
                        db[h, c] += total[where == c].sum()
    if not train:
        return out, lse
    return [out, lse, dq, dk, dv] + ([db] if s["bias"] is not None else [])


def _exact_step(s):
    case = dict(s["case"], right=0)
    H, r = case["heads"], case["heads"] // case["kv_heads"]
    out = torch.zeros(case["batch"], H, case["d"], dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(lengths(case)):
        i, j = torch.tensor([n - 1], device=s["q"].device), torch.arange(n, device=s["q"].device)
        k, v = s["k"][b, :n].double(), s["v"][b, :n].double()
        for h in range(H):
            ok, where = _exact_row_block(case, s, h, i, j, n)
            z = (k[:, h // r] * s["q"][b, h].double()).sum(1) * case["d"] ** -0.5
            if where is not None:
                z = z + s["bias"][h].double()[where[0]]
            p = torch.softmax(torch.where(ok[0], z, -math.inf), 0)
            out[b, h] = (p[:, None] * v[:, h // r]).sum(0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "attend": _exact_attend, "step": _exact_step}[case["kind"]](s)
