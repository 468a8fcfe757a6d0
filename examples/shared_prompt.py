"""A pruned attention layer that answers one prompt many times: the prompt lies in the 4-bit cache once, and a search keeps its best answers.

    python examples/shared_prompt.py [--steps 8]

Queries and keys leave the pruned projection as rows of one matrix and are normed and turned by their position in one pass
(``norm_rotate``).  Which pages belong to whom stays on the GPU: every step gives all answers a token more (``KVCache.extend``), lets the best of them be
continued by several (``KVCache.fork``) and attends to prompt and answers at once (``KVCache.shared_attention``); at the end the pages in use
move to the cache's front (``KVCache.compact``).  Weights, inputs and the choice of the best are synthetic."""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2203_05016_amd import binding, synth  # noqa: E402


class SharedPromptLayer:
    """q_heads query heads over heads key heads.  Row 0 of the table is the prompt, the rows behind it are the answers."""

    def __init__(self, features, q_heads, heads, head_dim, pages, answers, table_pages, page_tokens=64, V=32, sparsity=0.75, device="cuda:0"):
        self.head_dim, self.device, self.answers = head_dim, device, answers

        def pruned(outputs, inputs, seed):
            p = synth.make_spmm(outputs, inputs, 8, V, sparsity, seed=seed, with_x=False)
            kept = synth.kept_per_group(inputs, sparsity)
            return binding.compress((p.W / np.sqrt(np.float32(kept))).astype(np.float16), p.mask, p.perm, p.V).bind_device(device)

        self.rows = (q_heads * head_dim, heads * head_dim, heads * head_dim)
        self.project, self.combine = pruned(sum(self.rows), features, 1), pruned(features, q_heads * head_dim, 2)
        self.cache = binding.KVCache(pages, page_tokens, heads, head_dim, torch.float16, device)
        zeros = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)
        self.table, self.lengths, self.uses = zeros(1 + answers, table_pages), zeros(1 + answers), zeros(pages)
        pairs = head_dim // 2
        self.frequencies = torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)], dtype=torch.float64).to(device)
        self.weight = torch.ones(head_dim, dtype=torch.float16, device=device)

    def _int32(self, values):
        return torch.tensor(values, dtype=torch.int32).to(self.device)

    def _take(self, x, counts, positions):
        """Queries, keys and values of x's tokens, which become counts[b] more tokens of every row."""
        q, k, v = self.project.spmm(x).split(self.rows)
        q, k = binding.norm_rotate(q, k, self.head_dim, positions, self.frequencies, q_weight=self.weight, k_weight=self.weight)
        held = (self.table, self.lengths, self.uses)
        *_, slots, starts = self.cache.extend(*held, self._int32(counts), x.shape[1], out=held)
        self.cache.write(k, v, slots)
        return q, k, v, starts

    def prompt(self, x):
        """The prompt, (features, tokens); returns the layer's output."""
        n = x.shape[1]
        q, k, v, _ = self._take(x, [n] + [0] * self.answers, torch.arange(n, dtype=torch.int32, device=self.device))
        return self.combine.spmm(binding.window_attention(q, k, v, self.head_dim))

    def step(self, x):
        """One more token of every answer: x (features, answers)."""
        positions = self.lengths[0] + self.lengths[1:]
        q, _, _, _ = self._take(x, [0] + [1] * self.answers, positions)
        o = self.cache.shared_attention(q, self.table[:1], self.lengths[:1], self.table[1:], self.lengths[1:])
        return self.combine.spmm(o)

    def keep(self, best):
        """Answer i goes on from answer best[i] (int32, on the GPU)."""
        parents = torch.cat([torch.zeros_like(best[:1]), best + 1])
        self.table, self.lengths, self.uses = self.cache.fork(self.table, self.lengths, self.uses, parents)

    def compact(self):
        held = (self.table, self.uses)
        self.cache.compact(*held, out=held)


def tokens(rng, features, n, device="cuda:0"):
    return torch.randn((features, n), generator=rng).to(torch.float16).to(device)


def main():
    args = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    args.add_argument("--steps", type=int, default=8)
    steps = args.parse_args().steps
    features, answers, rng = 1024, 6, torch.Generator().manual_seed(7)
    layer = SharedPromptLayer(features, q_heads=16, heads=4, head_dim=64, pages=64, answers=answers, table_pages=16)
    y = layer.prompt(tokens(rng, features, 777))
    torch.cuda.synchronize()
    print("prompt of 777 tokens: %s, largest %.3f" % (tuple(y.shape), float(y.abs().max())), flush=True)
    for i in range(steps):
        y = layer.step(tokens(rng, features, answers))
        order = y.float().square().sum(0).argsort(descending=True)      # the best third are continued by three each
        layer.keep(order.repeat_interleave(3)[:answers].int())
        torch.cuda.synchronize()
        print("step %d: largest %.3f, %d pages in use" % (i, float(y.abs().max()), int((layer.uses > 0).sum())), flush=True)
    layer.compact()
    print("pages in use lie in front: %s" % bool((layer.uses[:int((layer.uses > 0).sum())] > 0).all()))


if __name__ == "__main__":
    main()
