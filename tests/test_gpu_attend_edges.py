"""Attention over texts where values are extreme: words without any weight, masks of the type's lowest value, scores and
gradients far from one, infinities and NaN beside what is shown."""
import math

import pytest
import torch

from attend_reference import attend_reference, check
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
