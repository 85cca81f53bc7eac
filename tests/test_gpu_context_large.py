"""The context operators at sizes where other variants of their kernels run: blocks enough for the device, sums joined over many
blocks, late pieces of more than 512 words, caches read by more blocks than a wavefront has lanes, wide rows one after the
other.  References and bounds are those of the small cases, computed in 64 bits on the device."""
import pytest
import torch

from attend_reference import attend_reference, check
from paper_1606_08495_amd import w2v
from test_gpu_attend import offsets_of
from test_gpu_norm import close, reference

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def on_device(f, *args, **kw):
    """f's tensors, computed on the GPU."""
    with torch.device("cuda"):
        return {k: t.cpu() for k, t in f(*args, **kw).items()}


def run(lengths, H, G, d, ty, seed=0, buckets=None, span=None, drop=0.0, train=True, **see):
    """Attention of rows of normal numbers against the definition."""
    off = offsets_of(lengths)
    T = off[-1]
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v, dout = [torch.randn(T, n, d, generator=g, device="cuda").to(ty) for n in (H, G, G, H)]
    if buckets:
        see.update(bias=torch.randn(H, buckets, generator=g, device="cuda"), buckets=w2v.relative_buckets(buckets, span))
    if drop:
        see.update(keep=(torch.rand(T, generator=g, device="cuda") >= drop).to(torch.uint8))
    ref = on_device(attend_reference, q, k, v, off, dout=dout if train else None, **see)
    soff = torch.tensor(off, dtype=torch.int64, device="cuda")
    out, lse = w2v.attend(q, k, v, soff, **see)
    check(out, ref, "out", ty)
    check(lse, ref, "lse")
    if train:
        grads = w2v.attend_backward(dout, q, k, v, out, lse, soff, **see)
        for t, name in zip(grads, ("dq", "dk", "dv", "dbias")):
            if t is not None:
                check(t, ref, name, F32 if name == "dbias" else ty)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("d", [32, 60, 64, 96, 100, 128])
def test_blocks_enough_for_the_device(d, ty):
    """More than 512 blocks in every kernel: a block has one wavefront for 32 words, tiles of 64 keys are taken whole."""
    print("many blocks", d, ty, flush=True)
    run([700], 86, 86, d, ty, left=None, right=0)
    run([500, 60, 140], 86, 86, d, ty, left=70, right=5, sinks=3, drop=0.2, buckets=8, span=40)
    run([300, 401], 172, 86, d, ty, left=None, right=None, buckets=4, span=200)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
def test_many_short_texts(ty):
    print("short texts", ty, flush=True)
    run([20, 1, 0, 7, 33, 40] * 4 + [30] * 9, 88, 88, 60, ty, left=10, right=10, skip_self=True, drop=0.1, buckets=16, span=12)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("span", [30, 1023])
def test_bias_sums_of_many_blocks(span, ty):
    print("bias sums", span, ty, flush=True)
    run([2500, 300, 1800], 2, 1, 48, ty, left=300, right=0, sinks=4, buckets=32, span=span)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, BF16])
def test_long_late_pieces(ty):
    """First words that stay visible among more than 2^17 words: pieces of more than 512 queries."""
    print("late pieces", ty, flush=True)
    run([1500, 700, 2100] * 32, 1, 1, 24, ty, left=40, right=0, sinks=6)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d", [(2, 1, 60), (8, 1, 128), (3, 3, 100)])
def test_steps_over_many_parts_of_a_cache(H, G, d, ty):
    print("step parts", H, G, d, ty, flush=True)
    room, n = 20000, [20000, 16641, 200]
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = [torch.randn(*s, d, generator=g, device="cuda").to(ty) for s in ((3, H), (3, room, G), (3, room, G))]
    bias, bmap = torch.randn(H, 8, generator=g, device="cuda"), w2v.relative_buckets(8, 100)
    out = w2v.attend_step(q, k, v, torch.tensor(n, dtype=torch.int32, device="cuda"), bias=bias, buckets=bmap)
    u = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}[ty]
    ref, bound = [], []
    for b, count in enumerate(n):
        K, V = [x[b, :count].double().repeat_interleave(H // G, 1).transpose(0, 1).contiguous() for x in (k, v)]
        Q = q[b].double()[:, :, None]
        back = (torch.arange(count, device="cuda") - (count - 1)).clamp(min=-100) + 100
        x = (K @ Q)[..., 0] * d ** -0.5 + bias.double()[:, bmap.long()[back]]
        size = (K.abs() @ Q.abs())[..., 0] * d ** -0.5
        p = torch.softmax(x, 1)[:, None]
        o = (p @ V)[:, 0]
        ref.append(o)
        E = (128 * 2.0 ** -24 * size + 2.0 ** -21 * x.abs()).max(1, keepdim=True).values
        bound.append((2 * E + 2e-5) * (p @ V.abs())[:, 0] + u * o.abs())
    check(out, dict(out=torch.stack(ref).cpu(), out_bound=torch.stack(bound).cpu()), "out", ty)


@pytest.mark.gpu
@pytest.mark.parametrize("d,ty", [(300, BF16), (2500, F32), (5000, F32), (16384, F32), (4101, BF16), (9000, F16), (16384, F16)])
def test_wide_rows_one_after_the_other(d, ty):
    """More rows than blocks at every width: a group's next row is asked for while it works on this one."""
    print("wide rows", d, ty, flush=True)
    m = 2100 if d > 300 else 70_000
    g = torch.Generator(device="cuda").manual_seed(d)
    x, dy = [(torch.randn(m, d, generator=g, device="cuda") * s + 0.3).to(ty) for s in (1.5, 1.0)]
    gain, offset = [torch.randn(d, generator=g, device="cuda") for _ in range(2)]
    ref = on_device(reference, x, gain, offset, 1e-5, dy)
    y, mean, rstd = w2v.layer_norm(x, gain, offset, 1e-5)
    far = x.double().abs().mean(1).cpu()
    close(y, ref["y"], ref["y_bound"], ty)
    close(mean, ref["mean"], 1e-5 * far)
    close(rstd, ref["rstd"], 1e-5 * ref["rstd"] * (1 + far * ref["rstd"]))
    dx, dgain, doffset = w2v.layer_norm_backward(dy, x, gain, mean, rstd)
    close(dx, ref["dx"], ref["dx_bound"], ty)
    close(dgain, ref["dgain"], ref["dgain_bound"])
    close(doffset, ref["doffset"], ref["doffset_bound"])
