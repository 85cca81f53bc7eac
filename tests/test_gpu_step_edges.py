"""Attention of one new word per text over a cache that holds infinities."""
import pytest
import torch

from paper_1606_08495_amd import w2v

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [F32, F16, BF16])
@pytest.mark.parametrize("H,G,d", [(1, 1, 60), (5, 5, 60), (4, 2, 100), (8, 1, 128), (2, 2, 37), (2, 1, 3), (9, 1, 66), (3, 3, 124)])
def test_infinities_that_have_no_weight(H, G, d, ty):
    """A shown key whose infinity makes the score -infinity has no weight, and its value does not show; the same in the whole text."""
    room, n = 900, [900, 300, 40]
    q, k, v = [torch.randn(*s, d, device="cuda").to(ty) for s in ((3, H), (3, room, G), (3, room, G))]
    keep = torch.ones(3, room, dtype=torch.uint8, device="cuda")
    hidden = [7, 39, 256, 299, 640]
    keep[:, hidden] = 0
    q[..., d - 1], q[..., 0] = 1.0, 1.0
    want = w2v.attend_step(q, k, v, torch.tensor(n, dtype=torch.int32, device="cuda"), keep=keep)
    assert torch.isfinite(want).all()
    for column in (d - 1, 0, d // 2):
        if column == d // 2:
            q[..., column] = 1.0
            want = w2v.attend_step(q, k, v, torch.tensor(n, dtype=torch.int32, device="cuda"), keep=keep)
        k2, v2 = k.clone(), v.clone()
        k2[:, hidden, :, column], v2[:, hidden] = float("-inf"), float("inf")
        got = w2v.attend_step(q, k2, v2, torch.tensor(n, dtype=torch.int32, device="cuda"))
        assert torch.equal(got, want)
        for b in range(3):
            full = torch.zeros(n[b], H, d, dtype=ty, device="cuda")
            full[-1] = q[b]
            whole, _ = w2v.attend(full, k2[b, :n[b]].contiguous(), v2[b, :n[b]].contiguous(),
                                  torch.tensor([0, n[b]], dtype=torch.int64, device="cuda"), right=0)
            assert torch.allclose(got[b].float(), whole[-1].float(), atol={F32: 1e-5, F16: 4e-3, BF16: 3e-2}[ty])
