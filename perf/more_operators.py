"""Performance cases of positions that turn and of the paged cache: what a program that serves texts word by word calls.

Attention over texts knows where a word stands by a bias of its distance; the other way is to turn the columns of queries and
keys by angles that grow with the position, so that products depend on distances alone.  A server keeps the turned
keys and the values of many texts of unequal length in one pool of pages that each text's row of a table lists, appends
new words to it, and lets every text's newest word look back over its pages; texts that begin with the same words
share the pages of that prefix, and the prefix is read once for all of them.

A case is a dict of plain values.  ``listed()`` names the standing ones, ``draw()`` makes more from the same
ranges, ``prepare()`` makes what a program holds before the call, ``run()`` is one pass, ``work()`` the bytes and
operations such a pass cannot do without, ``exact()`` the same outputs in 64 bits from the definitions.
Where ``own`` is false ``run()`` computes in elementary torch operations in 32 bits (angles in 64); where it is true it calls
the public entry points of ``paper_1606_08495_amd.w2v``.

Kinds:
  rotate      queries and keys of a block of texts turned by their positions; with train, and the gradients turned back
  append      new words' keys and values into a paged cache, keys and queries turned on the way
  pages       attention of one new word per text over its pages; with shared, a prefix that all texts have in common
  serve       append and attention of one new word per text, as a server's step has them
"""
import math
import random

import torch

own = False

TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
ELEMENTS = 1 << 28           # gathered elements, or scores, that the plain form holds at a time
PLAIN = dict(halves=False, scaling="none", factor=1.0, trained=0, gain=1.0)
PARTS = dict(halves=True, scaling="parts", factor=8.0, trained=4096, gain=1.2)


def listed():
    return [
        # One short text, trained on by itself: five heads of 60 columns, the column slices of 300.
        dict(name="rotate-20", kind="rotate", type="float32", texts=1, low=20, high=20, heads=5, kv_heads=5, d=60,
             rotated=60, first=0, train=True, **PLAIN),
        # A block of short texts, as the benchmark's text workload has them.
        dict(name="rotate-texts", kind="rotate", type="float32", texts=5243, low=10, high=40, heads=5, kv_heads=5, d=60,
             rotated=60, first=0, train=False, **PLAIN),
        # Long texts, trained on past the length of their first training: half of each head turns, slow pairs stretched.
        dict(name="rotate-long-train", kind="rotate", type="bfloat16", texts=3, low=4000, high=16000, heads=16, kv_heads=4,
             d=128, rotated=64, first=0, train=True, **PARTS),
        # One user's session, one word more.
        dict(name="append-1", kind="append", type="float32", batch=1, low=1, high=1, before=499, page=16, slots=32, heads=5,
             kv_heads=5, d=60, rotated=60, **PLAIN),
        # Prompts of unequal length taken in at once, some behind what their session holds already.
        dict(name="append-prompts", kind="append", type="bfloat16", batch=40, low=10, high=1500, before=700, page=16, slots=160,
             heads=32, kv_heads=8, d=128, rotated=128, **dict(PLAIN, halves=True)),
        # One user's session, one new word over it, with the bias by distance.
        dict(name="pages-1", kind="pages", type="float32", batch=1, low=500, high=500, shared=0, page=16, slots=32, heads=5,
             kv_heads=5, d=60, left=-1, sinks=0, buckets=32, span=128),
        # Many texts served at once, unequal and long.
        dict(name="pages-32", kind="pages", type="bfloat16", batch=32, low=300, high=32768, shared=0, page=16, slots=2048,
             heads=32, kv_heads=8, d=128, left=-1, sinks=0, buckets=0, span=0),
        # Sessions read in a window, their first words visible throughout; heads of a width that is no power of two.
        dict(name="pages-window", kind="pages", type="float16", batch=48, low=100, high=20000, shared=0, page=64, slots=313,
             heads=6, kv_heads=6, d=100, left=1023, sinks=4, buckets=0, span=0),
        # A few short sessions behind the same opening.
        dict(name="prefix-4", kind="pages", type="float32", batch=4, low=520, high=570, shared=512, page=16, slots=36, heads=5,
             kv_heads=5, d=60, left=-1, sinks=0, buckets=0, span=0),
        # Many sessions about one long document.
        dict(name="prefix-64", kind="pages", type="bfloat16", batch=64, low=32800, high=33700, shared=32768, page=16,
             slots=2112, heads=32, kv_heads=8, d=128, left=-1, sinks=0, buckets=0, span=0),
        # The same in 32 bits, every head its own keys, with the bias.
        dict(name="prefix-24", kind="pages", type="float32", batch=24, low=4100, high=5000, shared=4096, page=64, slots=80,
             heads=8, kv_heads=8, d=64, left=-1, sinks=0, buckets=32, span=128),
        # A server's step: the new word of every text into its pages, then its attention over them.
        dict(name="serve-16", kind="serve", type="float16", batch=16, low=1, high=1, before=3000, shared=0, page=32, slots=128,
             heads=12, kv_heads=4, d=96, left=-1, sinks=0, buckets=0, span=0, rotated=48, **dict(PLAIN, halves=True)),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "append", "append", "pages", "pages", "prefix", "prefix", "serve"])
    ty = rng.choice(sorted(TYPES))
    d = rng.choice([16, 32, 37, 48, 60, 64, 80, 96, 100, 128, rng.randint(8, 128)])
    kv = rng.choice([1, 2, 4, 5, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4])
    rotated = rng.choice([d // 2 * 2, d // 2 * 2, d // 4 * 2, rng.randint(1, d // 2) * 2])
    scaling = rng.choice(["none", "none", "linear", "base", "parts"])
    turned = dict(rotated=rotated, halves=rng.random() < 0.5, scaling=scaling,
                  factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]),
                  trained=rng.choice([512, 4096, 8192]) if scaling == "parts" else 0,
                  gain=1.0 if scaling != "parts" else rng.choice([1.0, 1.2]))
    if kind == "rotate":
        low = _spread(rng, 1, 4000)
        high = low + _spread(rng, 1, 2 * low + 4)
        texts = _spread(rng, 1, 5000)
        while texts * high * (heads + kv) * d > 1 << 26 and texts > 1:
            texts = texts // 2
        return dict(kind=kind, type=ty, texts=texts, low=low, high=high, heads=heads, kv_heads=kv, d=d,
                    first=rng.choice([0, 0, _spread(rng, 1, 1 << 20)]), train=rng.random() < 0.5, **turned)
    page = rng.choice([8, 16, 16, 32, 64, 128, 256])
    if kind in ("append", "serve"):
        single = kind == "serve" or rng.random() < 0.4
        batch = _spread(rng, 1, 64)
        low = 1 if single else rng.randint(1, 40)
        high = 1 if single else low + _spread(rng, 1, 1500)
        before = _spread(rng, 1, 3000)
        while batch * (before + high) * kv * d > 1 << 25 and batch > 1:
            batch //= 2
        while batch * high * heads * d > 1 << 26 and batch > 1:
            batch //= 2
        case = dict(kind=kind, type=ty, batch=batch, low=low, high=high, before=before, page=page,
                    slots=(before + high + page - 1) // page + rng.randint(0, 3), heads=heads, kv_heads=kv, d=d, **turned)
        if kind == "serve":
            windowed = rng.random() < 0.3
            case.update(shared=0, left=_spread(rng, 1, before) if windowed else -1, sinks=rng.choice([0, 4]) if windowed else 0,
                        buckets=0, span=0)
        return case
    room = _spread(rng, 16, 32768)
    shared = 0
    batch = _spread(rng, 1, 64)
    if kind == "prefix":
        shared = (room + page - 1) // page * page
        batch = _spread(rng, 2, 64)
        room = shared + _spread(rng, 1, 2000)
    while batch * (room - shared) * kv * d > 1 << 28 or batch * room * heads > 1 << 26:
        if batch > 2:
            batch //= 2
        else:
            shared = shared // 2 // page * page
            room = shared + max(16, (room - shared) // 2)
    windowed = rng.random() < (0.2 if shared else 0.4)
    biased = rng.random() < 0.4
    return dict(kind="pages", type=ty, batch=batch, low=rng.randint(shared + 1, room), high=room, shared=shared, page=page,
                slots=(room + page - 1) // page + rng.randint(0, 3), heads=heads, kv_heads=kv, d=d,
                left=_spread(rng, 1, room) if windowed else -1, sinks=rng.choice([0, 4, 7]) if windowed else 0,
                buckets=rng.choice([8, 32]) if biased else 0, span=rng.choice([20, 128, 500]) if biased else 0)


def lengths(case):
    """Lengths of a case's texts (of its new words, where it appends): part of the case, the same for every seed."""
    n = case["texts"] if case["kind"] == "rotate" else case["batch"]
    rng = random.Random(n * 1_000_003 + case["low"] * 1009 + case["high"])
    out = [rng.randint(case["low"], case["high"]) for _ in range(n)]
    out[0] = case["high"]
    return out


def filled(case):
    """Words of each text that its cache holds once the case has run."""
    n = lengths(case)
    if case["kind"] == "pages":
        return n
    rng = random.Random(case["before"] * 7919 + len(n))
    had = [rng.randint(0, case["before"]) for _ in n]
    had[0] = case["before"]
    return [a + b for a, b in zip(had, n)]


def turns(case):
    """What each pair of columns turns from word to word, as a whole number of 2^-64 of a turn."""
    r, out = case["rotated"], []
    for c in range(r // 2):
        f = 10000.0 ** (-2.0 * c / r)
        if case["scaling"] == "linear":
            f /= case["factor"]
        elif case["scaling"] == "base" and c:
            f *= case["factor"] ** (-2.0 * c / (r - 2))
        elif case["scaling"] == "parts":         # pairs of many turns over the first length stay, those of few are stretched
            w = min(1.0, max(0.0, (case["trained"] * f / (2 * math.pi) - 1.0) / 31.0))
            f *= w + (1 - w) / case["factor"]
        out.append(int(f / (2 * math.pi) * 2.0 ** 64))
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
    H, G, d = case["heads"], case["kv_heads"], case["d"]

    def normal(*shape, to=None):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=g).to(to or ty)

    def whole(x, to=torch.int32):
        return torch.tensor(x, dtype=to, device="cuda")

    s = dict(case=case, turns=whole(turns(case), torch.int64) if "rotated" in case else None)
    n = lengths(case)
    offsets = [0]
    for x in n:
        offsets.append(offsets[-1] + x)
    T = offsets[-1]
    if case["kind"] == "rotate":
        s.update(q=normal(T, H, d), k=normal(T, G, d), sent_off=whole(offsets, torch.int64), positions=None)
        if case["first"]:                        # texts that go on from elsewhere: positions are given
            s["positions"] = torch.cat([torch.arange(x, device="cuda") for x in n]).to(torch.int32) + case["first"]
        if case["train"]:
            s.update(dq=normal(T, H, d), dk=normal(T, G, d))
        return s
    # a pool of pages in no order, some of them nobody's; what a row of the table does not need is no page
    page, B, common = case["page"], case["batch"], case.get("shared", 0) // case["page"]
    full = filled(case)
    need = [(x + page - 1) // page for x in full]
    order = list(range(common + sum(max(0, x - common) for x in need) + 3))
    random.Random(seed).shuffle(order)
    prefix = [order.pop() for _ in range(common)]
    table = [prefix + [order.pop() for _ in range(common, x)] + [-1] * (case["slots"] - max(x, common)) for x in need]
    pages = common + sum(max(0, x - common) for x in need) + 3
    s.update(table=whole(table), n=whole(full), full=full, offsets=offsets)
    for name in ("k_pages", "v_pages"):
        s[name] = torch.empty(pages, page, G, d, dtype=ty, device="cuda")
        for a in range(0, pages, 1024):          # in parts: the pool may be most of the memory used
            s[name][a:a + 1024].copy_(normal(min(1024, pages - a), page, G, d))
    if case["kind"] != "pages":
        s.update(q=normal(T, H, d), k=normal(T, G, d), v=normal(T, G, d),
                 sent_off=None if case["high"] == 1 else whole(offsets, torch.int64))
    else:
        s.update(q=normal(B, H, d))
    s.update(bias=None, buckets=None)
    if case.get("buckets"):
        s.update(bias=normal(H, case["buckets"], to=torch.float32), buckets=whole(bucket_map(case["buckets"], case["span"])))
    return s


def _shown(case, n):
    """Words that the newest of n is shown."""
    left = case["left"] if case["left"] >= 0 else 1 << 40
    return min(n, min(left + 1, n) + min(case["sinks"], max(0, n - left - 1)))


def work(case):
    size = torch.empty(0, dtype=TYPES[case["type"]]).element_size()
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    n = lengths(case)
    T = sum(n)
    if case["kind"] == "rotate":
        passes = 2 if case["train"] else 1
        return {"bytes": passes * 2 * T * (H + G) * d * size + 8 * (len(n) + 1) + 4 * case["rotated"],
                "flops": passes * 3 * T * (H + G) * case["rotated"]}
    work = dict(bytes=0, flops=0)
    if case["kind"] != "pages":                  # q, k, v in, the turned q out, k and v into their pages
        work["bytes"] += 2 * T * (H + 2 * G) * d * size + 4 * case["rotated"] + 8 * len(n)
        work["flops"] += 3 * T * (H + G) * case["rotated"]
    if case["kind"] != "append":                 # every row that a text is shown, those of the common prefix once
        full, shared = filled(case), case["shared"]
        seen = [_shown(case, x) for x in full]
        first = [max(0, x - 1 - case["left"]) if case["left"] >= 0 else 0 for x in full]
        # of which in the prefix: by the window, and first words before it; and what any text is shown of the prefix
        past = [max(0, min(shared, x) - f) + min(case["sinks"], f, shared) for x, f in zip(full, first)]
        common = min(shared, max(0, shared - min(first)) + min(case["sinks"], min(first)))
        rows = common + sum(seen) - sum(past) if shared else sum(seen)
        work["bytes"] += 2 * rows * G * d * size + 2 * case["batch"] * H * d * size + 4 * (len(n) + rows // case["page"])
        work["flops"] += 4 * sum(seen) * H * d
    return work


# ---- the plain form ------------------------------------------------------------------------------------

def _angles(s, positions):
    """cos and sin [rows, 1, pairs] in 32 bits; the angles in 64, of which whole turns are left out first."""
    part = positions.double()[:, None] * (s["turns"].double() * 2.0 ** -64)
    angle = (part - part.floor()) * (2 * math.pi)
    gain = s["case"]["gain"]
    return (angle.cos() * gain).float()[:, None], (angle.sin() * gain).float()[:, None]


def _turned(s, x, cos, sin):
    case, r = s["case"], s["case"]["rotated"]
    out = x.float()
    if case["halves"]:
        a, b = out[..., :r // 2], out[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = out[..., 0:r:2], out[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, out[..., r:]], -1).to(x.dtype)


def _rotate(s):
    T = s["q"].shape[0]
    at = s["positions"]
    if at is None:
        first = s["sent_off"]
        at = torch.arange(T, device=first.device) - torch.repeat_interleave(first[:-1], first[1:] - first[:-1], output_size=T)
    cos, sin = _angles(s, at)
    out = [_turned(s, s["q"], cos, sin), _turned(s, s["k"], cos, sin)]
    if s["case"]["train"]:
        out += [_turned(s, s["dq"], cos, -sin), _turned(s, s["dk"], cos, -sin)]
    return out


def _append(s):
    case, n, T = s["case"], s["n"].long(), s["q"].shape[0]
    text = torch.arange(T, device=n.device)
    at = n[:T] - 1
    if s["sent_off"] is not None:
        first = s["sent_off"]
        count = first[1:] - first[:-1]
        text = torch.repeat_interleave(torch.arange(n.numel(), device=n.device), count, output_size=T)
        at = torch.arange(T, device=n.device) + (n - first[1:])[text]
    cos, sin = _angles(s, at)
    place = (s["table"].long()[text, at // case["page"]], at % case["page"])
    s["k_pages"][place] = _turned(s, s["k"], cos, sin)
    s["v_pages"][place] = s["v"]
    return _turned(s, s["q"], cos, sin)


def _attend(s, q):
    case = s["case"]
    B, H, G, d, dev = case["batch"], case["heads"], case["kv_heads"], case["d"], q.device
    r, page, shared = H // G, case["page"], case["shared"]
    longest = max(s["full"])
    slots, common = (longest + page - 1) // page, shared // page
    left = case["left"] if case["left"] >= 0 else 1 << 40
    kp, vp = [s[name][s["table"][0, :common].long()].float().view(shared, G, d) for name in ("k_pages", "v_pages")]
    kp, vp = kp.permute(1, 2, 0).contiguous(), vp.permute(1, 0, 2).contiguous()          # [G, d, shared], [G, shared, d]
    out = torch.empty(B, H, d, device=dev)
    L = (slots - common) * page
    part = max(1, ELEMENTS // max(1, L * G * d, (L + shared) * H))
    for a in range(0, B, part):
        b = min(B, a + part)
        qg = q[a:b].float().view(b - a, G, r, d)
        own_pages = s["table"][a:b, common:slots].long().clamp_min(0)
        k, v = [s[name][own_pages].float().view(b - a, L, G, d).transpose(1, 2) for name in ("k_pages", "v_pages")]
        x = torch.matmul(qg, k.transpose(-1, -2).contiguous())                            # [b, G, r, L]
        if shared:
            px = torch.matmul(qg.transpose(0, 1).reshape(G, (b - a) * r, d), kp)
            x = torch.cat([px.view(G, b - a, r, shared).transpose(0, 1), x], -1)
        x = x * (1.0 / math.sqrt(d))
        at, last = torch.arange(shared + L, device=dev)[None], s["n"][a:b].long()[:, None] - 1
        if s["bias"] is not None:
            bucket = s["buckets"].long()[(at - last).clamp(-case["span"], case["span"]) + case["span"]]
            x = x + s["bias"][:, bucket].transpose(0, 1).reshape(x.shape)
        ok = (at <= last) & ((at >= last - left) | (at < case["sinks"]))
        x = x.masked_fill(~ok[:, None, None], -math.inf)
        p = torch.exp(x - x.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        o = torch.matmul(p[..., shared:].contiguous(), v.masked_fill(~ok[:, None, shared:, None], 0.0).contiguous())
        if shared:
            pp = p[..., :shared].transpose(0, 1).reshape(G, (b - a) * r, shared)
            o = o + torch.matmul(pp, vp).view(G, b - a, r, d).transpose(0, 1)
        out[a:b] = o.reshape(b - a, H, d)
    return out.to(q.dtype)


# ---- a pass -----------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        if kind == "rotate":
            return _rotate(s)
        if kind == "pages":
            return _attend(s, s["q"])
        q = _append(s)
        return (q, s["k_pages"], s["v_pages"]) + ((_attend(s, q),) if kind == "serve" else ())
    from paper_1606_08495_amd import w2v
    if kind == "rotate":
        turn = dict(sent_off=s["sent_off"], positions=s["positions"], halves=case["halves"], gain=case["gain"])
        out = w2v.rotate(s["q"], s["turns"], k=s["k"], **turn)
        return out + w2v.rotate(s["dq"], s["turns"], k=s["dk"], back=True, **turn) if case["train"] else out
    q = s["q"]
    if kind != "pages":
        q = w2v.pages_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["n"], sent_off=s["sent_off"],
                             turns=s["turns"], halves=case["halves"], gain=case["gain"], q=q)
    if kind == "append":
        return q, s["k_pages"], s["v_pages"]
    out = w2v.attend_pages(q, s["k_pages"], s["v_pages"], s["table"], s["n"], shared=case["shared"],
                           left=case["left"] if case["left"] >= 0 else None, sinks=case["sinks"], bias=s["bias"],
                           buckets=s["buckets"])
    return out if kind == "pages" else (q, s["k_pages"], s["v_pages"], out)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def _exact_turned(s, x, positions, back=False):
    """The pair of columns as a complex number, times e^(i angle); the angle from whole numbers modulo 2^64."""
    case, r = s["case"], s["case"]["rotated"]
    angle = (positions.long()[:, None] * s["turns"]).double() * (2 * math.pi * 2.0 ** -64)
    unit = torch.polar(torch.full_like(angle, case["gain"]), -angle if back else angle)[:, None]
    y = x.double().clone()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["halves"] else (slice(0, r, 2), slice(1, r, 2))
    z = torch.complex(y[..., first], y[..., second]) * unit
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_append(s):
    case, page = s["case"], s["case"]["page"]
    q, k, v = torch.empty_like(s["q"], dtype=torch.float64), s["k_pages"].double(), s["v_pages"].double()
    for b, (lo, hi, n) in enumerate(zip(s["offsets"][:-1], s["offsets"][1:], s["full"])):
        at = torch.arange(n - (hi - lo), n, device=q.device)
        q[lo:hi] = _exact_turned(s, s["q"][lo:hi], at)
        where = s["table"][b].long()[torch.div(at, page, rounding_mode="floor")] * page + at % page
        k.view(-1, *k.shape[2:])[where] = _exact_turned(s, s["k"][lo:hi], at)
        v.view(-1, *v.shape[2:])[where] = s["v"][lo:hi].double()
    return q, k, v


def _exact_attend(s, q, k_pages, v_pages):
    case = s["case"]
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    out = torch.zeros(case["batch"], H, d, dtype=torch.float64, device=q.device)
    for b, n in enumerate(s["full"]):
        lists = s["table"][b, :(n + case["page"] - 1) // case["page"]].long()
        k, v = [x[lists].view(-1, G, d)[:n].double() for x in (k_pages, v_pages)]
        k, v = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
        z = torch.matmul(q[b].double().view(G, H // G, d), k).view(H, n) * d ** -0.5
        back = torch.arange(n - 1, -1, -1, device=q.device)                               # how far behind the newest
        if s["bias"] is not None:
            z += s["bias"].double()[:, s["buckets"].long()[case["span"] - back.clamp(max=case["span"])]]
        if case["left"] >= 0:
            z[:, (back > case["left"]) & (n - 1 - back >= case["sinks"])] = -math.inf
        out[b] = torch.matmul(torch.softmax(z, 1).view(G, H // G, n), v).view(H, d)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotate":
        at = s["positions"]
        if at is None:
            at = torch.cat([torch.arange(x, device="cuda") for x in lengths(case)])
        out = [_exact_turned(s, s["q"], at), _exact_turned(s, s["k"], at)]
        return out + [_exact_turned(s, s[name], at, back=True) for name in ("dq", "dk")] if case["train"] else out
    if case["kind"] == "pages":
        return _exact_attend(s, s["q"], s["k_pages"], s["v_pages"])
    q, k, v = _exact_append(s)
    return (q, k, v) + ((_exact_attend(s, q, k, v),) if case["kind"] == "serve" else ())
