"""What the calls around a shared cache refuse, on the host and before anything is enqueued.  No GPU: a cache with a stand-in for
its device memory, and addresses that nothing follows; every call must end before it reaches a launch."""
import ctypes
import types

import pytest
import torch

from paper_2203_05016_amd import binding

F16 = torch.float16
OK, NULL_ARG, BAD_SHAPE, BAD_DTYPE = 0, -1, -2, -5
HERE = 1 << 20          # an address


def _cache(pages=8, page=32, heads=2, D=64, dtype=F16):
    c = binding.KVCache.__new__(binding.KVCache)
    c.pages, c.page_tokens, c.heads, c.head_dim, c.dtype = pages, page, heads, D, dtype
    c._dev = types.SimpleNamespace(device=torch.device("cuda:0"))
    c._c = binding._Cache(128, pages, page, heads, D, binding.BF16 if dtype == torch.bfloat16 else binding.F16)
    return c


def _i(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def test_norm_rotate_refuses():
    q, k, p = torch.zeros(256, 9, dtype=F16), torch.zeros(128, 9, dtype=F16), _i(9)
    f, w = torch.zeros(32, dtype=torch.float64), torch.ones(64, dtype=F16)
    call = binding.norm_rotate
    with pytest.raises(ValueError, match="must live on"):
        call(q, k, 64, p, f)
    for bad in (q.float(), q[0], torch.zeros(9, 256, dtype=F16).t()):
        with pytest.raises(TypeError):
            call(bad, k, 64, p, f)
    for bad in (k.bfloat16(), torch.zeros(9, 128, dtype=F16).t()):
        with pytest.raises(TypeError):
            call(q, bad, 64, p, f)
    for bad in (k[:96], k[:, :8], k[0], torch.zeros(1, 9, dtype=F16).expand(128, 9)):
        with pytest.raises(ValueError):
            call(q, bad, 64, p, f)
    for bad in (0, -64, 1.5, True):
        with pytest.raises(ValueError):
            call(q, k, bad, p, f)
    for bad in (f.float(), f[None], torch.zeros(64, dtype=torch.float64)[::2]):
        with pytest.raises(TypeError):
            call(q, k, 64, p, bad)
    with pytest.raises(ValueError, match="33 frequencies"):
        call(q, k, 64, p, torch.zeros(33, dtype=torch.float64))
    for bad in (p.long(), p[:8], _i(2, 8), _i(1, 1, 9), _i(18)[::2]):
        with pytest.raises(TypeError):
            call(q, k, 64, bad, f)
    with pytest.raises(ValueError, match="need axes"):
        call(q, k, 64, _i(2, 9), f)
    with pytest.raises(ValueError):
        call(q, k, 64, _i(0, 9), f, axes=_i(32))
    with pytest.raises(ValueError):
        call(q, k, 64, _i(1, 9).expand(2, 9), f, axes=_i(32))
    with pytest.raises(ValueError, match="32 entries"):
        call(q, k, 64, _i(2, 9), f, axes=_i(31))
    for name in ("q_weight", "k_weight"):
        for bad in (w.float(), w[:32], w[None]):
            with pytest.raises(TypeError, match=name):
                call(q, k, 64, p, f, **{name: bad})
        with pytest.raises(ValueError, match="without norm"):
            call(q, k, 64, p, f, norm=False, **{name: w})
    with pytest.raises(ValueError, match="without k"):
        call(q, None, 64, p, f, k_weight=w)


def _rotate(q=HERE, k=2 * HERE, q_out=3 * HERE, k_out=4 * HERE, ld=(9, 9, 9, 9), tokens=9, heads=(4, 2), positions=5 * HERE, ldp=9, **fields):
    r = dict(head_dim=64, dtype=0, pairs=32, interleaved=0, norm=1, position_rows=1, eps=1e-6, frequencies=6 * HERE, axes=None, q_weight=None, k_weight=None)
    r.update(fields)
    return binding.lib().shflbw_norm_rotate(binding._Rotation(**r), positions, ldp, q, ld[0], heads[0], k, ld[1], heads[1], q_out, ld[2], k_out, ld[3], tokens, None)


def test_norm_rotate_library_refuses():
    assert binding.lib().shflbw_norm_rotate(None, None, 0, None, 0, 0, None, 0, 0, None, 0, None, 0, 0, None) == NULL_ARG
    assert _rotate(tokens=0) == OK and _rotate(heads=(0, 0)) == OK
    for bad in (dict(dtype=2), dict(dtype=-1)):
        assert _rotate(**bad) == BAD_DTYPE
    for bad in (dict(head_dim=80), dict(head_dim=0), dict(pairs=33), dict(pairs=-1), dict(tokens=-1), dict(heads=(-1, 2)), dict(heads=(65536, 2)), dict(eps=-1.0),
                dict(eps=float("inf")), dict(eps=float("nan")), dict(ld=(8, 9, 9, 9)), dict(ld=(9, 8, 9, 9)), dict(ld=(9, 9, 8, 9)), dict(ld=(9, 9, 9, 8)),
                dict(position_rows=0), dict(ldp=8)):
        assert _rotate(**bad) == BAD_SHAPE, bad
    for bad in (dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(positions=None), dict(frequencies=None)):
        assert _rotate(**bad) == NULL_ARG, bad
    size = 256 * 9 * 2
    for bad in (dict(q_out=HERE + 2), dict(q_out=HERE, ld=(9, 9, 10, 9)), dict(q_out=2 * HERE), dict(k_out=HERE + size - 2), dict(k_out=3 * HERE + size - 2),
                dict(q_out=HERE - 2), dict(q_out=HERE + 8 * 2, ld=(20, 9, 20, 9))):
        assert _rotate(**bad) == BAD_SHAPE, bad


def _shared(c, **kw):
    q, table = kw.pop("q", torch.zeros(256, 3, dtype=F16)), kw.pop("table", _i(3, 4))
    prefix_table, sizes = kw.pop("prefix_table", _i(1, 6)), kw.pop("prefix_lengths", _i(1))
    return c.shared_attention(q, prefix_table, sizes, table, kw.pop("lengths", _i(3)), **kw)


def test_shared_attention_refuses():
    c = _cache()
    with pytest.raises(ValueError, match="must live on"):
        _shared(c)
    q = torch.zeros(256, 3, dtype=F16)
    for bad in (q.bfloat16(), q[:200], q[:, 0], q[:0]):
        with pytest.raises(TypeError):
            _shared(c, q=bad)
    for name in ("table", "prefix_table"):
        t = _i(3, 4) if name == "table" else _i(1, 6)
        for bad in (t.long(), t[0], t[:, :0], _i(4, 3).t()):
            with pytest.raises(TypeError, match=name):
                _shared(c, **{name: bad})
    with pytest.raises(ValueError, match="overlap"):
        _shared(c, prefix_table=_i(1, 6).expand(2, 6), prefix_lengths=_i(2), members=_i(3))
    with pytest.raises(ValueError, match="one prefix"):
        _shared(c, prefix_table=_i(2, 6), prefix_lengths=_i(2))
    for bad in (dict(lengths=_i(2)), dict(prefix_lengths=_i(2)), dict(members=_i(3)), dict(starts=_i(3)), dict(q=q[:, :2]), dict(max_queries=2)):
        with pytest.raises(ValueError):
            _shared(c, **bad)
    for name in ("max_queries", "max_length", "max_prefix", "max_sharing"):
        for bad in (-1, 1.5, 2 ** 31, True):
            with pytest.raises(ValueError, match=name):
                _shared(c, starts=_i(4), **{name: bad})


def test_shared_attention_library_refuses():
    L, c = binding.lib(), binding._Cache(128, 8, 32, 2, 64, 0)

    def size(prefix=(), own=()):
        p = dict(prefixes=1, table_pages=1 << 20, table_ld=1 << 20, max_length=1 << 25, max_tokens=3, table=None, lengths=None, members=None)
        s = dict(q_heads=4, batch=3, max_queries=1, table_pages=4, window=0, sinks=0, tokens=3, max_length=128, table_ld=4, table=None, lengths=None, starts=None)
        p.update(prefix), s.update(own)
        return L.shflbw_kv_shared_attention_workspace(c, binding._Prefixes(**p), binding._Sequences(**s)), binding._Prefixes(**p), binding._Sequences(**s)
    assert size()[0] >= 4 * 3 * 66 * 4 and size(own=dict(batch=0, tokens=0))[0] == 0 and size(dict(max_length=100))[0] == 0
    for bad in (dict(prefixes=0), dict(prefixes=2), dict(table_pages=0), dict(table_ld=3), dict(max_length=0), dict(max_length=(1 << 25) + 1), dict(max_tokens=0),
                dict(table_pages=1 << 27, table_ld=1 << 27)):
        assert size(prefix=bad)[0] == BAD_SHAPE, bad
    for bad in (dict(window=1), dict(sinks=1), dict(q_heads=3), dict(max_length=0), dict(tokens=2), dict(max_queries=0)):
        assert size(own=bad)[0] == BAD_SHAPE, bad
    assert L.shflbw_kv_shared_attention_workspace(c, None, size()[2]) == NULL_ARG
    need, p, s = size()
    run = lambda q=HERE, out=2 * HERE, work=3 * HERE, have=need, ld=3, p=p, s=s: L.shflbw_kv_shared_attention(c, p, s, q, ld, out, ld, work, have, None)
    assert run() == NULL_ARG                                        # no tables
    p, s = (x for x in size(dict(table=HERE, lengths=HERE), dict(table=HERE, lengths=HERE))[1:])
    for bad, rc in ((dict(q=None), NULL_ARG), (dict(out=None), NULL_ARG), (dict(ld=2), BAD_SHAPE), (dict(work=None), NULL_ARG), (dict(have=need - 1), NULL_ARG),
                    (dict(work=HERE + 8), BAD_SHAPE)):
        assert run(p=p, s=s, **bad) == rc, bad
    # more workspace than 64 bits count is no small number
    wide = size(dict(max_tokens=1 << 40), dict(tokens=2 ** 31 - 1, batch=2 ** 31 - 1, q_heads=65534))[0]
    assert wide > 2 ** 40


def test_pages_refuse():
    c = _cache()
    table, lengths, uses = _i(3, 4), _i(3), _i(8)
    for call in (lambda t=table, n=lengths, u=uses, **kw: c.extend(t, n, u, kw.pop("counts", _i(3)), kw.pop("tokens", 5), **kw),
                 lambda t=table, n=lengths, u=uses, **kw: c.fork(t, n, u, kw.pop("parents", _i(3)), **kw)):
        with pytest.raises(ValueError, match="must live on"):
            call()
        for bad in (table.long(), table[0], table[:, :0], _i(4, 3).t()):
            with pytest.raises((TypeError, ValueError)):
                call(t=bad)
        for bad in (dict(n=_i(2)), dict(u=_i(7)), dict(t=_i(1, 4).expand(3, 4))):
            with pytest.raises(ValueError):
                call(**bad)
        for bad in (dict(n=lengths.long()), dict(u=uses.float()), dict(u=_i(16)[::2])):
            with pytest.raises(TypeError):
                call(**bad)
    for bad in (_i(2), _i(4)):
        with pytest.raises(ValueError):
            c.extend(table, lengths, uses, bad, 5)
    for bad in (-1, 2.5, 2 ** 31, True):
        with pytest.raises(ValueError, match="tokens"):
            c.extend(table, lengths, uses, _i(3), bad)
    with pytest.raises(TypeError):
        c.fork(table, lengths, uses, _i(3, 1))
    with pytest.raises(ValueError, match="must live on"):
        c.compact(table, uses)


def test_pages_library_refuses():
    L, c = binding.lib(), binding._Cache(128, 8, 32, 2, 64, 0)
    need = L.shflbw_kv_pages_workspace(c, 3)
    assert need > 0 and L.shflbw_kv_pages_workspace(c, -1) == BAD_SHAPE and L.shflbw_kv_pages_workspace(None, 3) == NULL_ARG
    pages = lambda at, **kw: binding._Pages(**{**dict(sequences=3, table_pages=4, table_ld=4, table=at, lengths=at + 4096, uses=at + 8192), **kw})
    calls = {
        "extend": lambda i, o, work=8 * HERE, have=need, which=7 * HERE, slots=6 * HERE, starts=5 * HERE, tokens=9:
            L.shflbw_kv_extend(c, i, o, which, slots, starts, tokens, work, have, None),
        "fork": lambda i, o, work=8 * HERE, have=need, which=7 * HERE: L.shflbw_kv_fork(c, i, o, which, work, have, None),
        "compact": lambda i, o, work=8 * HERE, have=need: L.shflbw_kv_compact(c, i, o, work, have, None),
    }
    for name, call in calls.items():
        good = pages(HERE), pages(2 * HERE)
        assert call(None, good[1]) == NULL_ARG and call(good[0], None) == NULL_ARG
        for bad, rc in ((dict(work=None), NULL_ARG), (dict(have=need - 1), NULL_ARG), (dict(work=HERE + 4), BAD_SHAPE)):
            assert call(*good, **bad) == rc, (name, bad)
        for bad, rc in ((dict(sequences=-1), BAD_SHAPE), (dict(table_pages=0), BAD_SHAPE), (dict(table_ld=3), BAD_SHAPE), (dict(table=None), NULL_ARG),
                        (dict(uses=None), NULL_ARG), (dict(table_pages=5, table_ld=5), BAD_SHAPE)):
            assert call(pages(HERE, **bad), good[1]) == rc and call(good[0], pages(2 * HERE, **bad)) == rc, (name, bad)
        huge = dict(table_pages=1 << 27, table_ld=1 << 27, table=1 << 40)
        assert call(pages(HERE, **huge), pages(2 * HERE, **{**huge, "table": 1 << 45})) == BAD_SHAPE
        # overlaps: shifted, another pitch, one array of out over another of in, two of out
        for bad in (dict(table=HERE + 4), dict(table=HERE, table_ld=5), dict(table=HERE + 8192), dict(uses=HERE + 8192 + 4), dict(uses=HERE), dict(uses=2 * HERE)):
            assert call(good[0], pages(2 * HERE, **bad)) == BAD_SHAPE, (name, bad)
        if name != "compact":
            for bad, rc in ((dict(lengths=None), NULL_ARG), (dict(lengths=HERE + 4096 + 4), BAD_SHAPE)):
                assert call(good[0], pages(2 * HERE, **bad)) == rc, (name, bad)
            assert call(*good, which=None) == NULL_ARG
        if name != "fork":
            assert call(pages(HERE), pages(2 * HERE, sequences=2)) == BAD_SHAPE
        else:
            assert call(good[0], pages(HERE)) == BAD_SHAPE          # in place
    for bad, rc in ((dict(slots=None), NULL_ARG), (dict(starts=None), NULL_ARG), (dict(tokens=-1), BAD_SHAPE), (dict(tokens=2 ** 31), BAD_SHAPE)):
        assert calls["extend"](pages(HERE), pages(2 * HERE), **bad) == rc, bad
