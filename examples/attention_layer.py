"""A pruned attention layer that serves several sequences: prompts, then single tokens, over a cache in 4 bits.

    python examples/attention_layer.py [--steps 8]

The four projections are Shfl-BW products (``Matrix.spmm``).  Everything between them stays features x tokens, as the products
take and leave it: a prompt's keys and values go into the cache as they are made and are attended to in 16 bits
(``window_attention``); every later token attends to the cache (``KVCache.attention``).  Weights and inputs are synthetic."""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2203_05016_amd import binding, synth  # noqa: E402


class AttentionLayer:
    """q_heads query heads over heads key heads; window 0 is none, and the first ``sinks`` tokens stay visible past it."""

    def __init__(self, features, q_heads, heads, head_dim, pages, page_tokens=64, window=0, sinks=0, V=32, sparsity=0.75, device="cuda:0"):
        self.heads, self.head_dim, self.window, self.sinks, self.device = heads, head_dim, window, sinks, device

        def pruned(outputs, inputs, seed):
            p = synth.make_spmm(outputs, inputs, 8, V, sparsity, seed=seed, with_x=False)
            kept = synth.kept_per_group(inputs, sparsity)
            return binding.compress((p.W / np.sqrt(np.float32(kept))).astype(np.float16), p.mask, p.perm, p.V).bind_device(device)

        # queries, keys and values in one product: their rows lie one below the other
        self.rows = (q_heads * head_dim, heads * head_dim, heads * head_dim)
        self.project = pruned(sum(self.rows), features, 1)
        self.combine = pruned(features, q_heads * head_dim, 2)
        self.cache = binding.KVCache(pages, page_tokens, heads, head_dim, torch.float16, device)
        self.free = list(range(pages))
        self.pages, self.lengths = [], []      # of every sequence

    def _append(self, counts):
        """Slots of ``counts[b]`` more tokens of every sequence, in the order of the columns."""
        size, slots = self.cache.page_tokens, []
        for b, n in enumerate(counts):
            length = self.lengths[b]
            while len(self.pages[b]) * size < length + n:
                self.pages[b].append(self.free.pop())
            slots += [self.pages[b][t // size] * size + t % size for t in range(length, length + n)]
            self.lengths[b] = length + n
        return self._int32(slots)

    def _int32(self, values):
        return torch.tensor(values, dtype=torch.int32).to(self.device)

    def table(self):
        """Pages of every sequence in order, the rows filled up with a page that is not read."""
        width = max(len(p) for p in self.pages)
        return self._int32([p + [0] * (width - len(p)) for p in self.pages])

    def prompts(self, x, counts):
        """New sequences: x (features, sum of counts), sequence after sequence.  Returns the layer's output, of x's shape."""
        assert not self.lengths
        self.pages, self.lengths = [[] for _ in counts], [0] * len(counts)
        starts = self._int32([sum(counts[:b]) for b in range(len(counts) + 1)])
        q, k, v = self.project.spmm(x).split(self.rows)
        self.cache.write(k, v, self._append(counts))
        o = binding.window_attention(q, k, v, self.head_dim, starts, max_tokens=max(counts), window=self.window, sinks=self.sinks)
        return self.combine.spmm(o)

    def step(self, x):
        """One more token of every sequence: x (features, sequences)."""
        q, k, v = self.project.spmm(x).split(self.rows)
        self.cache.write(k, v, self._append([1] * len(self.lengths)))
        o = self.cache.attention(q, self.table(), self._int32(self.lengths), max_length=max(self.lengths), window=self.window,
                                 sinks=self.sinks)
        return self.combine.spmm(o)


def tokens(rng, features, n, device="cuda:0"):
    return torch.randn((features, n), generator=rng).to(torch.float16).to(device)


def main():
    args = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    args.add_argument("--steps", type=int, default=8)
    steps = args.parse_args().steps
    counts, features = [700, 64, 1, 333], 1024
    rng = torch.Generator().manual_seed(7)
    layer = AttentionLayer(features, q_heads=16, heads=4, head_dim=64, pages=64, window=256, sinks=4)
    y = layer.prompts(tokens(rng, features, sum(counts)), counts)
    torch.cuda.synchronize()
    print("prompts of %s tokens: %s, largest %.3f" % (counts, tuple(y.shape), float(y.abs().max())), flush=True)
    for i in range(steps):
        y = layer.step(tokens(rng, features, len(counts)))
        torch.cuda.synchronize()
        print("step %d: %d tokens in the cache, largest %.3f" % (i, sum(layer.lengths), float(y.abs().max())), flush=True)
    print("the cache's %d tokens take %.2f MB, in 16 bits they would take %.2f" % (
        layer.cache.pages * layer.cache.page_tokens, layer.cache.device_bytes() / 1e6,
        4 * layer.cache.pages * layer.cache.page_tokens * layer.rows[1] / 1e6))


if __name__ == "__main__":
    main()
