"""The example that serves texts with one opening: it runs, and what it serves is attention over the whole texts."""
import importlib.util
import os
import sys

import pytest
import torch

from paper_1606_08495_amd import w2v

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_served_texts(monkeypatch):
    spec = importlib.util.spec_from_file_location("served_texts", os.path.join(ROOT, "examples", "served_texts.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    monkeypatch.setattr(sys, "argv", ["served_texts.py", "--texts", "5", "--opening", "70", "--steps", "20"])
    server, opening, said, served = example.main()
    assert server.shared == 64 and served.shape == (5, 20, 5, 60)
    for text in range(5):
        x = server.rows(torch.cat([opening, said[text]]))
        off = torch.tensor([0, x.shape[0]], device="cuda")
        q = w2v.rotate(x, server.turns, sent_off=off)
        whole = w2v.attend(q, q, x, off, right=0)[0]
        # rows are of norm 60^1/2: a score of 60 products, |q| |k| / 60^1/2 = 8 at most, off by some 2^-24 8 on either way, its weight by twice that
        assert torch.allclose(served[text], whole[64:], atol=2e-5)
    server.shard.destroy()
