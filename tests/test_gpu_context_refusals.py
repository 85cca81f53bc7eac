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
