"""Attention where a call's bounds and its tensors' values are at their limits, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from attention_reference import attend, check
from gpu_util import announce
from paper_2203_05016_amd import binding
from test_attention_gpu import DEV, NAN, _tensor

pytestmark = pytest.mark.gpu


def _starts(counts):
    return torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("D,heads,group,counts", [
    (128, 8, 8, [1] * 32), (128, 8, 8, [40] + [0] * 63), (128, 16, 8, [3] * 16), (128, 16, 5, [3] * 20), (128, 32, 8, [7] * 8),
    (96, 16, 8, [2] * 31), (64, 16, 8, [2] * 31), (128, 8, 8, [63] + [0] * 40)])
def test_short_prompts_of_many_sequences(D, heads, group, counts):
    """Fewer than 64 columns in all, and more workgroups than the GPU has CUs: every query head and query is computed."""
    announce("short prompts", D, heads, group, len(counts), max(counts))
    tokens = sum(counts)
    q, k, v = (_tensor(n * D, tokens, torch.bfloat16, 60 + i, 0.5 if i < 2 else 0) for i, n in enumerate((heads * group, heads, heads)))
    out = torch.full((heads * group * D, tokens), NAN, dtype=torch.bfloat16, device=DEV)
    binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D, _starts(counts), max(counts), out=out)
    at = 0
    for n in counts:
        if n:
            part = [x[:, at:at + n].double().numpy() for x in (q, k, v)]
            check(out[:, at:at + n], *attend(*part, D, 0, torch.bfloat16), "columns %d to %d" % (at, at + n - 1))
        at += n
