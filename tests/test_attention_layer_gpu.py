"""The example layer: what its attention returns for prompts and for single tokens, against the definition in 64 bits."""
import os
import sys
import types

import numpy as np
import pytest
import torch

from attention_reference import attend, check, held
from gpu_util import announce

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import attention_layer as example  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_prompts_then_steps(window, sinks):
    announce("attention_layer", window, sinks)
    counts, features, D = [70, 1, 33], 256, 64
    layer = example.AttentionLayer(features, 4, 2, D, pages=12, page_tokens=32, window=window, sinks=sinks)
    layer.combine = types.SimpleNamespace(spmm=lambda o: o)      # the attention's own result
    rng = torch.Generator().manual_seed(3)
    keys, values = [None] * 3, [None] * 3

    def projected(x):
        return [t.cpu() for t in layer.project.spmm(x).split(layer.rows)]

    x = example.tokens(rng, features, sum(counts))
    got, (q, k, v), at = layer.prompts(x, counts).cpu(), projected(x), 0
    for b, n in enumerate(counts):
        part = slice(at, at + n)
        want, tol = attend(q[:, part].double().numpy(), k[:, part].double().numpy(), v[:, part].double().numpy(), D, 0, torch.float16,
                           window=window, sinks=sinks)
        check(got[:, part], want, tol, "prompt %d" % b)
        keys[b], values[b] = k[:, part], v[:, part]
        at += n
    for step in range(3):
        x = example.tokens(rng, features, 3)
        got, (q, k, v) = layer.step(x).cpu(), projected(x)
        for b in range(3):
            keys[b], values[b] = torch.cat([keys[b], k[:, b:b + 1]], 1), torch.cat([values[b], v[:, b:b + 1]], 1)
            held_k, held_v = (torch.from_numpy(held(t)).half().double().numpy() for t in (keys[b], values[b]))
            want, tol = attend(q[:, b:b + 1].double().numpy(), held_k, held_v, D, counts[b] + step, torch.float16, window=window, sinks=sinks)
            check(got[:, b:b + 1], want, tol, "step %d of sequence %d" % (step, b))
    assert layer.lengths == [n + 3 for n in counts] and np.unique(sum(layer.pages, [])).size == sum(len(p) for p in layer.pages)


def test_the_example_runs(monkeypatch, capsys):
    announce("attention_layer main")
    monkeypatch.setattr(sys, "argv", ["attention_layer.py", "--steps", "2"])
    example.main()
    assert "step 1: 1106 tokens" in capsys.readouterr().out
