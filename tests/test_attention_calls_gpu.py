"""The native calls of the attention operators: the plain case runs there and gives what the general way gives, bit for bit; everything
else is handed back to the binding's own checks."""
import ctypes

import pytest
import torch

from gpu_util import announce
from paper_2203_05016_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _tagged(t):
    return t.as_subclass(type("TaggedTensor", (torch.Tensor,), {}))


def _setup(dtype=torch.float16):
    g = torch.Generator().manual_seed(3)
    rand = lambda rows, n: torch.randn(rows, n, generator=g).to(dtype).to(DEV)
    cache = binding.KVCache(40, 64, 2, 64, dtype, DEV)
    table = torch.arange(40, dtype=torch.int32, device=DEV).view(2, 20)
    lengths = torch.tensor([1200, 700], dtype=torch.int32, device=DEV)
    slots = torch.arange(2560, dtype=torch.int32, device=DEV)
    k, v = rand(128, 2560), rand(128, 2560)
    return cache, table, lengths, slots, k, v, rand(256, 2), rand(256, 7)


def test_cache_plain_case_and_what_is_handed_back():
    announce("native cache calls")
    cache, table, lengths, slots, k, v, q, q7 = _setup()
    native, plan, here = binding.calls(), cache._plan, torch.cuda.current_stream()
    assert native.kv_write(plan, k, v, slots) == 0
    ways = cache.read(slots, stream=here)                          # a stream argument takes the general way
    both = native.kv_read(plan, slots)
    assert all(torch.equal(a, b) and a.shape == k.shape for a, b in zip(both, ways))
    before = cache._dev.clone()
    cache.write(k, v, slots, stream=here)
    assert torch.equal(before, cache._dev)
    for bad in (k.t().contiguous().t(), k[:, ::2], k.bfloat16(), k.cpu(), k[:64], k[:, :0], _tagged(k), None, 3):
        assert native.kv_write(plan, bad, v, slots) is None and native.kv_write(plan, k, bad, slots) is None
    for bad in (slots.long(), slots[::2], slots[:-1], slots.cpu(), slots[None], _tagged(slots), None):
        assert native.kv_write(plan, k, v, bad) is None
    for bad in (slots.long(), slots[::2], slots[:0], slots.cpu(), slots[None], _tagged(slots), None):
        assert native.kv_read(plan, bad) is None
    assert torch.equal(cache.read(_tagged(slots))[0], ways[0])      # taken the general way

    starts = torch.tensor([0, 4, 7], dtype=torch.int32, device=DEV)
    for args, kw in (((q, table, lengths), {}), ((q7, table, lengths, starts, 4, 1200), dict(window=300, sinks=3))):
        want = cache.attention(*args, stream=here, **kw)
        full = list(args) + [None, 1, None][len(args) - 3:] + [kw.get("window", 0), kw.get("sinks", 0)]
        assert torch.equal(native.kv_attention(plan, *full, None), want)
        out = torch.zeros(256, args[0].shape[1] + 3, dtype=q.dtype, device=DEV)[:, 2:-1]
        assert torch.equal(native.kv_attention(plan, *full, out), want) and torch.equal(out, want)
        assert cache.attention(*args, out=out, **kw) is out
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):                               # the current stream is the one that is used
            other = native.kv_attention(plan, *full, None)
        side.synchronize()
        assert torch.equal(other, want)
    call = lambda **c: native.kv_attention(plan, *[{**dict(q=q, table=table, lengths=lengths, starts=None, mq=1, ml=None, w=0, s=0, out=None), **c}[n]
                                                   for n in ("q", "table", "lengths", "starts", "mq", "ml", "w", "s", "out")])
    for bad in (dict(q=q.bfloat16()), dict(q=q[:200]), dict(q=q.cpu()), dict(q=q[:, :1]), dict(q=_tagged(q)), dict(q=None), dict(table=table.long()),
                dict(table=table[0]), dict(table=table.t()), dict(lengths=lengths[:1]), dict(lengths=lengths.long()), dict(starts=lengths), dict(mq=2),
                dict(mq=1.0), dict(w=-1), dict(s=True), dict(ml=-1), dict(out=q.float()), dict(out=q[:, :1]), dict(out=q.cpu())):
        assert call(**bad) is None, bad
    assert call(ml=20 * 64 + 1) == -2 and "max_length" in binding.last_error()
    with pytest.raises(binding.ShflbwError, match="max_length"):
        cache.attention(q, table, lengths, max_length=20 * 64 + 1)
    with pytest.raises(ValueError, match="one query"):
        cache.attention(q[:, :1], table, lengths)


def test_window_attention_plain_case_and_what_is_handed_back():
    announce("native window attention")
    _, _, _, _, k, v, _, _ = _setup()
    k, v = k[:, :90], v[:, :90]
    q = torch.cat([v, k]).contiguous()
    native, here = binding.calls(), torch.cuda.current_stream()
    starts = torch.tensor([0, 50, 90], dtype=torch.int32, device=DEV)
    for full in ((64, None, None, 0, 0), (64, starts, 50, 20, 2)):
        want = binding.window_attention(q, k, v, *full, stream=here)
        assert torch.equal(native.window_attention(q, k, v, *full, None), want)
        out = torch.empty_like(q)
        assert binding.window_attention(q, k, v, *full, out=out) is out and torch.equal(out, want)
    call = lambda **c: native.window_attention(*[{**dict(q=q, k=k, v=v, d=64, starts=starts, most=50, w=0, s=0, out=None), **c}[n]
                                                 for n in ("q", "k", "v", "d", "starts", "most", "w", "s", "out")])
    for bad in (dict(q=q.float()), dict(q=q[:200]), dict(q=q.cpu()), dict(k=k.bfloat16()), dict(k=k[:, :80]), dict(v=v[:64]), dict(v=v.t()), dict(d=0), dict(d=64.0),
                dict(d=48), dict(starts=starts.long()), dict(starts=starts[:1]), dict(most=-1), dict(w=-1), dict(s=1.5), dict(out=q[:64]), dict(q=_tagged(q)), dict(q=None)):
        assert call(**bad) is None, bad
    assert call(d=32) == -2 and call(most=91) == -2


def test_a_c_plus_plus_exception_is_handed_back():
    announce("native attention, exception")
    cache, table, lengths, slots, k, v, q, _ = _setup()
    native, L = binding.calls(), binding.lib()
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
    throws = address(ctypes.CDLL("libstdc++.so.6")._ZSt17__throw_bad_allocv)
    names = ("kv_write", "kv_read", "kv_attention_workspace", "kv_attention", "window_attention")
    native.connect_attention(*[throws] * 5)
    try:
        for _ in range(3):
            assert native.kv_write(cache._plan, k, v, slots) is None and native.kv_read(cache._plan, slots) is None
            assert native.kv_attention(cache._plan, q, table, lengths, None, 1, None, 0, 0, None) is None
            assert native.window_attention(k, k, v, 64, None, None, 0, 0, None) is None
    finally:
        native.connect_attention(*[address(getattr(L, "shflbw_" + n)) for n in names])
    assert native.kv_write(cache._plan, k, v, slots) == 0
