"""Norms without a rotation: no pair is turned, so that there are no positions to turn by."""
import pytest
import torch

from paper_2203_05016_amd import binding

F16 = torch.float16


def test_positions_are_asked_for_where_pairs_are_turned():
    q, none = torch.zeros(256, 9, dtype=F16), torch.zeros(0, dtype=torch.float64)
    with pytest.raises(ValueError, match="must live on"):           # (everything before that is right)
        binding.norm_rotate(q, q[:128], 64, None, none)
    with pytest.raises(ValueError, match="without positions"):
        binding.norm_rotate(q, q[:128], 64, None, torch.zeros(32, dtype=torch.float64))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [5, 4000])
def test_norms_alone(tokens):
    from test_norm_rotate_gpu import DEV, check, definition, frequencies, positions, tensor
    print("[gpu-case] norms alone", tokens, flush=True)
    D, none = 64, frequencies(0)
    q, k = tensor(4 * D, tokens, F16, 1), tensor(2 * D, tokens, F16, 2)
    w = tensor(1, D, F16, 3)[0].contiguous()
    got = binding.norm_rotate(q, k, D, None, none, q_weight=w)
    with_positions = binding.norm_rotate(q, k, D, positions(tokens), none, q_weight=w)
    for x, y, same, weight in zip((q, k), got, with_positions, (w, None)):
        assert torch.equal(y, same) and y.device == torch.device(DEV)
        check(y, definition(x, D, positions(tokens), none, weight=weight), tokens)
