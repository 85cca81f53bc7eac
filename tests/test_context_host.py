"""What the context operators do on the host: the map of distances to buckets, and what they refuse."""
import pytest
import torch

from paper_1606_08495_amd import w2v


@pytest.mark.parametrize("buckets,span", [(42, 1006), (43, 1006), (146, 905), (744, 518), (1024, 1023), (1023, 300), (600, 256)])
def test_buckets_whose_borders_pass_close_to_a_distance(buckets, span):
    """The three nearest misses of all maps within the limits, and maps of many buckets, against whole numbers: distance r lies
    past border t where r^far near^t >= span^t near^far."""
    half = buckets // 2
    near = max(1, half // 2)
    far = half - near
    want, t = [], 0
    for r in range(span + 1):
        while r >= near and far and t + 1 < far and span ** (t + 1) * near ** far <= r ** far * near ** (t + 1):
            t += 1
        want.append(near + t if r >= near and far else min(r, half - 1))
    want = want[::-1] + [half + b for b in want[1:]]
    assert w2v.relative_buckets(buckets, span, device="cpu").tolist() == want


@pytest.mark.parametrize("name", ["left", "right", "sinks"])
def test_counts_that_make_no_sense(name):
    """A negative window is refused, not taken for an unbounded one; one past 32 bits is as wide as any text, not its lowest bits."""
    q = torch.zeros(2, 1, 4)

    def spec(value):
        see = {**dict(left=3, right=3, sinks=0), name: value}
        return w2v._spec(q, 1, see["left"], see["right"], see["sinks"], False, None, None, None)
    for value in (-1, -5, -2 ** 32, -2 ** 32 + 5):
        with pytest.raises(ValueError):
            spec(value)
    for value in (2 ** 32, 2 ** 32 + 5, 2 ** 70):
        assert getattr(spec(value), name) == w2v.UNBOUNDED
    assert getattr(spec(7), name) == 7


def test_bucket_counts_that_make_no_sense():
    for n, span in ((-4, 5), (4, -5), (4, -2 ** 32 + 5)):
        with pytest.raises(ValueError):
            w2v.relative_buckets(n, span, device="cpu")
    for n, span in ((2 ** 32 + 4, 5), (4, 2 ** 32 + 5), (4, 1024), (1025, 5), (1, 5), (4, 0)):
        with pytest.raises(w2v.W2VError):
            w2v.relative_buckets(n, span, device="cpu")
