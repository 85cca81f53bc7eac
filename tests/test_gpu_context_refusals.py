"""What the binding of the calls that work on a caller's memory refuses before anything is queued."""
import pytest
import torch

from paper_1606_08495_amd import w2v


def calls(workspace):
    """Every call that takes a workspace, with this one."""
    x, gain = torch.randn(6, 8, device="cuda"), torch.ones(8, device="cuda")
    _, mean, rstd = w2v.layer_norm(x, gain)
    q = torch.randn(70, 2, 16, device="cuda")
    off = torch.tensor([0, 70], dtype=torch.int64, device="cuda")
    out, lse = w2v.attend(q, q, q, off)
    cache = torch.randn(2, 600, 2, 16, device="cuda")
    n = torch.tensor([600, 3], dtype=torch.int32, device="cuda")
    return [lambda: w2v.layer_norm_backward(x, x, gain, mean, rstd, workspace=workspace),
            lambda: w2v.attend_backward(q, q, q, q, out, lse, off, workspace=workspace),
            lambda: w2v.attend_step(q[:2], cache, cache, n, workspace=workspace),
            lambda: w2v.topk_cosine(x, x, 2, workspace=workspace)]


@pytest.mark.gpu
def test_a_workspace_that_is_no_device_memory():
    for bad in (torch.empty(1 << 20, dtype=torch.uint8), [0] * 9, torch.empty(1 << 12, 1 << 9, dtype=torch.uint8, device="cuda")[:, ::2]):
        for call in calls(bad):
            with pytest.raises(TypeError):
                call()


@pytest.mark.gpu
def test_a_workspace_of_another_type_counts_its_bytes():
    for call in calls(torch.empty(1 << 20, dtype=torch.float32, device="cuda")):
        call()
    for call in calls(torch.empty(4, dtype=torch.float64, device="cuda")):
        with pytest.raises(w2v.W2VError):
            call()


@pytest.mark.gpu
def test_outputs_beside_their_inputs_in_one_buffer():
    """q, k, v and the result of a word side by side do not touch; a result on its inputs is refused."""
    T, H, d = 200, 3, 20
    off = torch.tensor([0, T], dtype=torch.int64, device="cuda")
    packed = torch.randn(T, 4, H, d, device="cuda")
    q, k, v, out = packed.unbind(1)
    want = w2v.attend(q.contiguous(), k.contiguous(), v.contiguous(), off, right=0)[0]
    w2v.attend(q, k, v, off, right=0, out=out)
    assert torch.equal(out, want)
    before = packed.clone()
    flat = packed.view(-1)
    shifted = flat[d // 2:d // 2 + (T - 1) * 4 * H * d + H * d].as_strided((T, H, d), (4 * H * d, d, 1))      # half a head on
    heads_first = flat[:T * H * d].view(H, T, d).transpose(0, 1)
    for bad in (q, k, v, shifted, heads_first, packed.view(T, 4 * H, d)[:, 1:1 + H]):
        with pytest.raises(w2v.W2VError):
            w2v.attend(q, k, v, off, right=0, out=bad)
    torch.cuda.synchronize()
    assert torch.equal(packed, before)
    shared = torch.randn(T, 8, d, device="cuda")              # six query heads, one key head, one value head; results elsewhere
    w2v.attend(shared[:, :6], shared[:, 6:7], shared[:, 7:], off, out=torch.empty(T, 6, d, device="cuda"))
    with pytest.raises(w2v.W2VError):
        w2v.attend(shared[:, :6], shared[:, 6:7], shared[:, 7:], off, out=shared[:, 2:])
    one = torch.randn(1, 4, H, d, device="cuda")              # a single word: strides from word to word mean nothing
    w2v.attend(*one.unbind(1)[:3], torch.tensor([0, 1], device="cuda"), out=one[:, 3])
    assert torch.allclose(one[:, 3], one[:, 2], rtol=2.0 ** -21, atol=0)      # its weight, the sum's inverse and the product are rounded
    n = torch.tensor([600, 3], dtype=torch.int32, device="cuda")
    cache, q = torch.randn(2, 600, 2, 16, device="cuda"), torch.randn(2, 2, 16, device="cuda")
    want = w2v.attend_step(q, cache, cache, n)
    assert torch.equal(w2v.attend_step(q, cache, cache, n, out=q), want)      # a step's result may take the place of its q
