"""Vectors of words in their context, trained and served over a shard's word vectors.

The bag-of-words hidden vector of a position is the mean of the input vectors in its window.  Here it is learned what to
weigh: the rows of a block of texts are normalised (w2v_layer_norm), every position reads its window with five heads of
its columns and a bias by distance (w2v_attend, the word itself left out), the result is normalised again and takes the
place of the hidden vector in the skip-gram objective with negatives of the shard (w2v_negatives, w2v_coeffs).  A
step goes back through all of it (w2v_attend_backward, w2v_layer_norm_backward) to the gains, the bias and both matrices.
Afterwards a text is read word by word over a cache (w2v_attend_step), as a server would, and the context's nearest output
vectors are looked up (w2v_topk_cosine).

The matrices' update itself is torch's, rows of one word summed by index_add_: unlike the calls, it does not give the same last
bits every time.

    python examples/context_vectors.py [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1606_08495_amd import w2v, workloads  # noqa: E402

V, D, HEADS, WINDOW, K = 2000, 300, 5, 5, 5


class ContextModel:
    """A shard's two matrices, and what the context adds: two pairs of gains and offsets, a bias by distance."""

    def __init__(self, seed=1):
        self.shard = w2v.Shard(V, D, seed, init_mode=1)
        self.shard.set_counts(workloads.analytic_counts(V, 1.0, 10 ** 6))
        self.norms = [[torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")] for _ in range(2)]
        self.norms[1][0].mul_(0.1)
        self.bias = torch.zeros(HEADS, 16, device="cuda")
        self.see = dict(left=WINDOW, right=WINDOW, skip_self=True, bias=self.bias,
                        buckets=w2v.relative_buckets(16, WINDOW))

    def forward(self, tokens, off):
        x = self.shard.get_rows(0, tokens)
        n1 = w2v.layer_norm(x, *self.norms[0])
        q = n1[0].view(-1, HEADS, D // HEADS)
        out, lse = w2v.attend(q, q, q, off, **self.see)
        n2 = w2v.layer_norm(out.view(-1, D), *self.norms[1])
        return x, n1, q, out, lse, n2

    def step(self, tokens, off, seed, alpha):
        """One step on a block of texts; the objective per position."""
        x, n1, q, out, lse, n2 = self.forward(tokens, off)
        rows = torch.cat([tokens[:, None], self.shard.negatives(tokens, K, seed)], 1)
        w = self.shard.get_rows(1, rows.flatten()).view(-1, K + 1, D)
        coeffs, loss = self.shard.coeffs([(w * n2[0][:, None]).sum(2)], K, want_loss=True)
        g = (coeffs[:, :, None] * w).sum(1)                     # ascent: the objective's gradient by the hidden vector
        dw = coeffs[:, :, None] * n2[0][:, None]
        dout, dgain2, doff2 = w2v.layer_norm_backward(g, out.view(-1, D), self.norms[1][0], *n2[1:])
        dq, dk, dv, dbias = w2v.attend_backward(dout.view_as(out), q, q, q, out, lse, off, **self.see)
        dx, dgain1, doff1 = w2v.layer_norm_backward((dq + dk + dv).view(-1, D), x, self.norms[0][0], *n1[1:])
        m = tokens.numel()
        for which, index, delta in ((0, tokens, dx), (1, rows.flatten(), dw.view(-1, D))):
            words, place = torch.unique(index, return_inverse=True)
            total = torch.zeros(words.numel(), D, device="cuda").index_add_(0, place, delta)
            old = self.shard.get_rows(which, words)
            self.shard.set_rows(which, words, old + alpha * total)
        for p, d in zip(self.norms[0] + self.norms[1] + [self.bias], (dgain1, doff1, dgain2, doff2, dbias)):
            p.add_(d, alpha=10 * alpha / m)
        return loss / m

    def serve(self, words):
        """The last word's context vector, the text read word by word over a cache; causal, as a server has it."""
        cache = torch.zeros(1, len(words), HEADS, D // HEADS, device="cuda")
        n = torch.zeros(1, dtype=torch.int32, device="cuda")
        see = dict(left=WINDOW, skip_self=True, bias=self.bias, buckets=self.see["buckets"])
        for i, word in enumerate(words):
            x = self.shard.get_rows(0, w2v.as_index_tensor([word]))
            q = w2v.layer_norm(x, *self.norms[0])[0].view(1, HEADS, D // HEADS)
            cache[:, i] = q
            n.add_(1)
            out = w2v.attend_step(q, cache, cache, n, **see)
        return w2v.layer_norm(out.view(1, D), *self.norms[1])[0]


def texts(seed, count=200, length=20):
    """Texts with something to learn: a word is followed by its neighbours in the vocabulary."""
    g = torch.Generator().manual_seed(seed)
    start = torch.randint(0, V - 4 * length, (count, 1), generator=g) // 50 * 50
    words = start + torch.randint(0, 12, (count, length), generator=g)
    off = torch.arange(0, count * length + 1, length, dtype=torch.int64)
    return words.flatten().to(torch.int32).cuda(), off.cuda()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    steps = ap.parse_args().steps
    model = ContextModel()
    losses = []
    for h in range(steps):
        tokens, off = texts(h)
        losses.append(model.step(tokens, off, w2v.minibatch_seed(7, h), 0.05))
    losses = torch.cat(losses)
    print("objective per position: %.4f at first, %.4f at last" % (float(losses[0]), float(losses[-1])))
    h = model.serve([100, 103, 107, 101, 109])
    idx, score, _ = w2v.topk_cosine(h, model.shard.get_rows(1, torch.arange(V, dtype=torch.int32, device="cuda")), 5)
    print("nearest to the context of 100 103 107 101 _:", w2v.index_to_numpy(idx)[0].tolist(), [round(x, 3) for x in score[0].tolist()])
    model.shard.status()
    model.shard.destroy()
    return losses


if __name__ == "__main__":
    main()
