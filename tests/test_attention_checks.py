"""What the attention operators refuse, on the host and before anything is enqueued.  No GPU: a cache with a stand-in for its
device memory; every call must raise before it reaches a launch."""
import types

import pytest
import torch

from paper_2203_05016_amd import binding

F16 = torch.float16


def _cache(pages=8, page=32, heads=2, D=64, dtype=F16):
    c = binding.KVCache.__new__(binding.KVCache)
    c.pages, c.page_tokens, c.heads, c.head_dim, c.dtype = pages, page, heads, D, dtype
    c._dev = types.SimpleNamespace(device=torch.device("cuda:0"))
    c._c = binding._Cache(128, pages, page, heads, D, binding.BF16 if dtype == torch.bfloat16 else binding.F16)
    return c


def test_cache_sizes():
    size = binding.lib().shflbw_kv_cache_bytes
    assert size(3, 32, 2, 64) == 3 * 2 * 32 * (32 + 2 + 32 + 2)
    assert size(3, 32, 2, 96) == 3 * 2 * 32 * (48 + 4 + 48 + 4)
    assert size(70000, 1024, 16, 128) == 70000 * 1024 * 16 * 136
    for bad in ((0, 32, 2, 64), (1, 16, 2, 64), (1, 48, 2, 64), (1, 2048, 2, 64), (1, 32, 0, 64), (1, 32, 2, 80), (1, 32, 2, 32), (1, 32, 2, 256)):
        assert size(*bad) == 0
        with pytest.raises(ValueError):
            binding.KVCache(*bad, F16)
    with pytest.raises(ValueError):
        binding.KVCache(1 << 21, 1024, 1, 64, F16)     # 2^31 slots
    with pytest.raises(TypeError):
        binding.KVCache(1, 32, 2, 64, torch.float32)
    with pytest.raises(ValueError):
        binding.KVCache(1.5, 32, 2, 64, F16)


def test_write_and_read_refuse():
    c = _cache()
    k, slots = torch.zeros(128, 9, dtype=F16), torch.zeros(9, dtype=torch.int32)
    with pytest.raises(ValueError, match="must live on"):
        c.write(k, k, slots)
    with pytest.raises(ValueError, match="must live on"):
        c.read(slots)
    for bad in (k.bfloat16(), k.t(), k[0], k.float()):
        with pytest.raises(TypeError):
            c.write(bad, k, slots)
        with pytest.raises(TypeError):
            c.write(k, bad, slots)
    for bad in (k[:64], k[:, :8], torch.zeros(1, 9, dtype=F16).expand(128, 9)):
        with pytest.raises(ValueError):
            c.write(k, bad, slots)
    for bad in (slots.long(), slots[None], torch.zeros(18, dtype=torch.int32)[::2]):
        with pytest.raises(TypeError):
            c.write(k, k, bad)
    with pytest.raises(ValueError, match="9 entries"):
        c.write(k, k, slots[:8])


def test_attention_refuses():
    c = _cache()
    q, table = torch.zeros(256, 3, dtype=F16), torch.zeros(3, 4, dtype=torch.int32)
    lengths, starts = torch.ones(3, dtype=torch.int32), torch.arange(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="must live on"):
        c.attention(q, table, lengths)
    for bad in (q.bfloat16(), q[:200], q[:, 0], q[:0]):
        with pytest.raises(TypeError):
            c.attention(bad, table, lengths)
    with pytest.raises(TypeError):
        c.attention(torch.zeros(3, 256, dtype=F16).t(), table, lengths)
    for bad in (table.long(), table[0], table[:, :0], torch.zeros(4, 3, dtype=torch.int32).t()):
        with pytest.raises(TypeError):
            c.attention(q, bad, lengths)
    with pytest.raises(ValueError, match="overlap"):
        c.attention(q, torch.zeros(1, 4, dtype=torch.int32).expand(3, 4), lengths)
    with pytest.raises(ValueError, match="3 entries"):
        c.attention(q, table, lengths[:2])
    with pytest.raises(ValueError, match="4 entries"):
        c.attention(q, table, lengths, starts[:3])
    with pytest.raises(ValueError, match="one query"):
        c.attention(q[:, :2], table, lengths)
    with pytest.raises(ValueError, match="one query"):
        c.attention(q, table, lengths, max_queries=2)
    for name in ("window", "sinks", "max_length", "max_queries"):
        for bad in (-1, 1.5, 2 ** 31, True):
            with pytest.raises(ValueError, match=name):
                c.attention(q, table, lengths, starts, **{name: bad})


def test_window_attention_refuses():
    q, k = torch.zeros(256, 9, dtype=F16), torch.zeros(128, 9, dtype=F16)
    starts = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="must live on"):
        binding.window_attention(q, k, k, 64)
    with pytest.raises(TypeError):
        binding.window_attention(q.float(), k.float(), k.float(), 64)
    for bad in (k.bfloat16(), torch.zeros(9, 128, dtype=F16).t()):
        with pytest.raises(TypeError):
            binding.window_attention(q, bad, k, 64)
        with pytest.raises(TypeError):
            binding.window_attention(q, k, bad, 64)
    for bad in (k[:96], k[:, :8], k[:0]):
        with pytest.raises(ValueError):
            binding.window_attention(q, bad, k, 64)
    with pytest.raises(ValueError):
        binding.window_attention(q, k, k[:64], 64)
    with pytest.raises(ValueError):
        binding.window_attention(q, k, k, 0)
    with pytest.raises(TypeError):
        binding.window_attention(q, k, k, 64, starts.long())
    with pytest.raises(TypeError):
        binding.window_attention(q, k, k, 64, starts[None])
    for name in ("window", "sinks", "max_tokens"):
        with pytest.raises(ValueError, match=name):
            binding.window_attention(q, k, k, 64, starts, **{name: -1})


def _status(rc, status, text):
    assert rc == status and text in binding.last_error(), (rc, binding.last_error())


def test_the_library_refuses():
    """The C entry points, on addresses that nothing may follow."""
    L, S = binding.lib(), binding._Sequences
    c = binding._Cache(128, 8, 32, 2, 64, binding.F16)
    for field, value, status, text in (("data", None, -1, "NULL"), ("data", 64, -2, "128-byte"), ("page_tokens", 33, -2, "power of two"),
                                       ("head_dim", 80, -2, "head_dim"), ("heads", 0, -2, "heads"), ("pages", 0, -2, "pages"),
                                       ("pages", 1 << 26, -2, "slots"), ("dtype", 2, -5, "dtype")):
        bad = binding._Cache(128, 8, 32, 2, 64, binding.F16)
        setattr(bad, field, value)
        _status(L.shflbw_kv_write(bad, 1, 9, 1, 9, 1, 9, None), status, text)
        _status(L.shflbw_kv_read(bad, 1, 9, 1, 9, 1, 9, None), status, text)
    for args, status, text in (((1, 9, 1, 9, 1, -1), -2, "tokens"), ((None, 9, 1, 9, 1, 9), -1, "NULL"), ((1, 9, 1, 9, None, 9), -1, "NULL"),
                               ((1, 8, 1, 9, 1, 9), -2, "leading"), ((1, 9, 1, 8, 1, 9), -2, "leading")):
        _status(L.shflbw_kv_write(c, *args, None), status, text)
    assert L.shflbw_kv_write(c, None, 0, None, 0, None, 0, None) == 0            # no tokens

    def sequences(**changes):
        s = S(4, 3, 2, 4, 0, 0, 6, 100, 4, 1, 1, 1)
        for name, value in changes.items():
            setattr(s, name, value)
        return s

    for changes, text in ((dict(q_heads=3), "q_heads"), (dict(q_heads=0), "q_heads"), (dict(q_heads=65536 * 2), "65535"), (dict(batch=-1), "batch"),
                          (dict(tokens=-1), "tokens"), (dict(tokens=1 << 31), "tokens"), (dict(window=-1), "window"), (dict(sinks=-1), "sinks"),
                          (dict(max_queries=0), "max_queries"), (dict(max_length=0), "max_length"), (dict(max_length=129), "max_length"),
                          (dict(table_ld=3), "table_ld"), (dict(table_pages=1 << 26, table_ld=1 << 26), "2^31"),
                          (dict(starts=None), "one query"), (dict(starts=None, tokens=3), "one query")):
        assert L.shflbw_kv_attention_workspace(c, sequences(**changes)) == -2
        _status(L.shflbw_kv_attention(c, sequences(**changes), 1, 9, 1, 9, None, 0, None), -2, text)
    assert L.shflbw_kv_attention(c, sequences(batch=0), None, 9, None, 9, None, 0, None) == 0
    assert L.shflbw_kv_attention(c, sequences(tokens=0), None, 9, None, 9, None, 0, None) == 0
    _status(L.shflbw_kv_attention(c, None, 1, 9, 1, 9, None, 0, None), -1, "NULL")
    _status(L.shflbw_kv_attention(c, sequences(), None, 9, 1, 9, None, 0, None), -1, "NULL")
    _status(L.shflbw_kv_attention(c, sequences(table=None), 1, 9, 1, 9, None, 0, None), -1, "NULL")
    _status(L.shflbw_kv_attention(c, sequences(), 1, 5, 1, 9, None, 0, None), -2, "leading")
    _status(L.shflbw_kv_attention(c, sequences(), 1, 9, 1, 5, None, 0, None), -2, "leading")
    long = sequences(table_pages=1000, table_ld=1000, max_length=32000)
    need = L.shflbw_kv_attention_workspace(c, long)
    assert need > 0 and need % 8 == 0
    _status(L.shflbw_kv_attention(c, long, 1, 9, 1, 9, None, 0, None), -1, "workspace of %d bytes" % need)
    _status(L.shflbw_kv_attention(c, long, 1, 9, 1, 9, 128, need - 1, None), -1, "workspace")
    _status(L.shflbw_kv_attention(c, long, 1, 9, 1, 9, 8, need, None), -2, "aligned")

    def prompt(q_heads=4, heads=2, head_dim=64, tokens=9, starts=1, sequences=2, most=9, window=0, sinks=0, dtype=0, ld=9, q=1):
        return L.shflbw_window_attention(q, ld, 1, 9, 1, 9, 1, 9, q_heads, heads, head_dim, tokens, starts, sequences, most, window, sinks, dtype, None)

    for kw, status, text in ((dict(dtype=2), -5, "dtype"), (dict(head_dim=80), -2, "head_dim"), (dict(q_heads=3), -2, "q_heads"), (dict(heads=0), -2, "heads"),
                             (dict(tokens=-1), -2, "tokens"), (dict(starts=None), -2, "one sequence"), (dict(most=10), -2, "max_tokens"),
                             (dict(window=-1), -2, "window"), (dict(ld=8), -2, "leading"), (dict(q=None), -1, "NULL")):
        _status(prompt(**kw), status, text)
    assert prompt(tokens=0, most=0) == 0 and prompt(sequences=0) == 0
