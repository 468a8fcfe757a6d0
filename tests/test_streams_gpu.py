"""Results of calls on a given stream: the memory is that stream's, so that nothing pending on another stream still uses it when the
call's work begins, and it stays until the stream the caller comes from is done with it."""
import numpy as np
import pytest
import torch

from gpu_util import announce
from paper_2203_05016_amd import binding, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _stream_of(t):
    """The stream whose pool of the allocator the tensor's memory is in."""
    at = t.data_ptr()
    found = [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]]
    assert len(found) == 1
    return found[0]


def test_memory_of_the_stream_that_writes_it():
    side, g = torch.cuda.Stream(), torch.Generator().manual_seed(1)
    rand = lambda *shape: torch.randn(*shape, generator=g).half().to(DEV)
    p = synth.make_spmm(128, 64, 8, 32, 0.5, seed=1, with_x=False)
    bind = lambda **kw: binding.compress(p.W, p.mask, p.perm, p.V).bind_device(DEV, **kw)
    A, cache = bind(), binding.KVCache(40, 32, 1, 64, torch.float16, DEV)
    q, k, v = rand(64, 1200), rand(64, 1200), rand(64, 1200)
    slots = torch.arange(1200, dtype=torch.int32, device=DEV)
    cache.write(k, v, slots)
    table, lengths = torch.arange(40, dtype=torch.int32, device=DEV).view(1, 40), torch.tensor([1200], dtype=torch.int32, device=DEV)
    x, images = rand(64, 40), rand(2, 64, 5, 5)
    calls = {
        "spmm": lambda **kw: [A.spmm(x, **kw)],
        "conv2d": lambda **kw: [A.conv2d(images, 1, 1, **kw)],
        "layernorm_transpose": lambda **kw: [binding.layernorm_transpose(x.t().contiguous(), **kw)],
        "read": lambda **kw: list(cache.read(slots, **kw)),
        "attention": lambda **kw: [cache.attention(q[:, :1], table, lengths, **kw)],
        "window_attention": lambda **kw: [binding.window_attention(q, k, v, 64, **kw)],
    }
    for name, call in calls.items():
        announce("streams", name)
        want = call()
        torch.cuda.synchronize()
        got = call(stream=side)
        side.synchronize()
        for a, b in zip(got, want):
            assert _stream_of(a) == side.cuda_stream and _stream_of(b) == torch.cuda.current_stream().cuda_stream != side.cuda_stream, name
            assert torch.equal(a, b), name
    announce("streams", "bind_device")
    B = bind(stream=side)
    side.synchronize()
    assert _stream_of(B._dev) == side.cuda_stream and torch.equal(B.spmm(x), A.spmm(x))
    assert np.array_equal(B.row_indices(), A.row_indices())


def test_workspace_of_the_stream_that_uses_it():
    """The parts of a long context: a call on a stream leaves no memory of its own in another's pool."""
    announce("streams", "workspace")
    side, g = torch.cuda.Stream(), torch.Generator().manual_seed(2)
    cache = binding.KVCache(200, 64, 1, 64, torch.float16, DEV)
    k, v = (torch.randn(64, 12800, generator=g).half().to(DEV) for _ in range(2))
    cache.write(k, v, torch.arange(12800, dtype=torch.int32, device=DEV))
    table, lengths = torch.arange(200, dtype=torch.int32, device=DEV).view(1, 200), torch.tensor([12800], dtype=torch.int32, device=DEV)
    q = torch.randn(64, 1, generator=g).half().to(DEV)
    want = cache.attention(q, table, lengths)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    others = lambda: sum(s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] != side.cuda_stream)
    held = others()
    got = cache.attention(q, table, lengths, stream=side)
    side.synchronize()
    assert any(s["stream"] == side.cuda_stream for s in torch.cuda.memory_snapshot()) and others() == held
    assert torch.equal(got, want)
