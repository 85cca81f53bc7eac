"""Many texts with one opening, served word by word from a pool of pages over a shard's word vectors.

A word's row is its input vector, normalised (w2v_layer_norm); its heads are turned by its position (w2v_rotate, or on the way into
the pages), so that what a word sees of another depends on how far apart they are.  The opening goes in once, as a prompt: attended as a text
(w2v_attend), its keys and values appended to pages (w2v_pages_append) that the first row of the table lists for all texts.  Then every
text goes on by itself, a word a step: appended to pages of its own, and its newest word looks back over them and over the opening, which
is read once for all texts (w2v_attend_pages).  Pages are handed out on the host when a text needs one more.

    python examples/served_texts.py [--texts 64] [--opening 256] [--steps 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1606_08495_amd import w2v  # noqa: E402

V, D, HEADS, PAGE = 2000, 300, 5, 16
WIDTH = D // HEADS


class Server:
    """A shard's vectors, a pool of pages, and what each text has of them."""

    def __init__(self, texts, room, seed=1):
        self.shard = w2v.Shard(V, D, seed)
        self.norm = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
        self.turns = w2v.rotary_turns(WIDTH)
        self.slots = -(-room // PAGE)
        self.k, self.v = [torch.empty(texts * self.slots, PAGE, HEADS, WIDTH, device="cuda") for _ in range(2)]
        self.free = list(range(texts * self.slots))
        self.table = torch.full((texts, self.slots), -1, dtype=torch.int32)
        self.counts = [0] * texts
        self.shared = 0

    def rows(self, words):
        return w2v.layer_norm(self.shard.get_rows(0, words), *self.norm)[0].view(-1, HEADS, WIDTH)

    def grow(self, text, words):
        """Pages for the next words of a text."""
        before, self.counts[text] = self.counts[text], self.counts[text] + words
        for slot in range(-(-before // PAGE), -(-self.counts[text] // PAGE)):
            self.table[text, slot] = self.free.pop()

    def plan(self):
        return self.table.cuda(), torch.tensor(self.counts, dtype=torch.int32, device="cuda")

    def open(self, words):
        """The texts' common opening (whole pages of it), as the first text's words; the rows its words read."""
        x, off = self.rows(words), torch.tensor([0, words.numel()], device="cuda")
        self.grow(0, words.numel())
        table, n = self.plan()
        all_off = torch.full((len(self.counts) + 1,), words.numel(), dtype=torch.int64, device="cuda")
        all_off[0] = 0                               # the other texts have no new words here
        q = w2v.pages_append(x, x, self.k, self.v, table, n, sent_off=all_off, turns=self.turns, q=x)
        self.shared = words.numel()
        self.counts = [self.shared] * len(self.counts)
        return w2v.attend(q, q, x, off, right=0)[0]      # (queries and keys are the same rows here)

    def step(self, words):
        """One word more of every text; the rows they read."""
        for text in range(len(self.counts)):
            self.grow(text, 1)
        table, n = self.plan()
        x = self.rows(words)
        q = w2v.pages_append(x, x, self.k, self.v, table, n, turns=self.turns, q=x)
        return w2v.attend_pages(q, self.k, self.v, table, n, shared=self.shared)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--texts", type=int, default=64)
    ap.add_argument("--opening", type=int, default=256)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    opening = a.opening // PAGE * PAGE
    g = torch.Generator().manual_seed(3)
    server = Server(a.texts, opening + a.steps)
    words = torch.randint(0, V, (opening,), generator=g).to(torch.int32).cuda()
    server.open(words)
    served, said = [], []
    for _ in range(a.steps):
        said.append(torch.randint(0, V, (a.texts,), generator=g).to(torch.int32).cuda())
        served.append(server.step(said[-1]))
    out = server.rows(said[-1]).flatten(1) + served[-1].flatten(1)
    idx, score, _ = w2v.topk_cosine(out, server.shard.get_rows(0, torch.arange(V, dtype=torch.int32, device="cuda")), 3)
    print("%d texts of %d words, %d pages in use" % (a.texts, opening + a.steps, server.k.shape[0] - len(server.free)))
    print("nearest to the first text's last word in its context:", w2v.index_to_numpy(idx)[0].tolist(), [round(x, 3) for x in score[0].tolist()])
    return server, words, torch.stack(said, 1), torch.stack(served, 1)


if __name__ == "__main__":
    main()
