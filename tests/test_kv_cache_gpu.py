"""The 4-bit cache: what is written and read back is the format's nearest value, exactly, wherever the slots lie."""
import numpy as np
import pytest
import torch

from attention_reference import held
from gpu_util import announce
from paper_2203_05016_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _tensor(rows, tokens, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, tokens, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("page,heads,tokens", [(32, 1, 1), (64, 3, 77), (128, 2, 129), (1024, 1, 40)])
def test_written_and_read_back(dtype, D, page, heads, tokens):
    announce("kv round trip", dtype, D, page, heads, tokens)
    pages = tokens // page + 2
    cache = binding.KVCache(pages, page, heads, D, dtype, DEV)
    k, v = _tensor(heads * D, tokens, dtype, 1), _tensor(heads * D, tokens, dtype, 2)
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(3))[:tokens].int()
    cache.write(k.to(DEV), v.to(DEV), slots.to(DEV))
    gk, gv = cache.read(slots.to(DEV))
    for got, x in ((gk, k), (gv, v)):
        assert torch.equal(got.cpu(), torch.from_numpy(held(x)).to(dtype))
    # slots that were not written hold what was there: zeros
    rest = torch.from_numpy(np.setdiff1d(np.arange(pages * page), slots.numpy())).int()
    gk, gv = cache.read(rest.to(DEV))
    assert not gk.any() and not gv.any()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_every_value_and_scale(dtype):
    """All 65536 patterns, alone in their blocks (each is its block's largest, so it is rounded in the upper half of the
    grid) and beside a value 2 to 8 times as large; infinities, NaN, zeros of both signs and subnormals among them."""
    announce("kv all patterns", dtype)
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
    tokens = 65536
    x = torch.zeros(64, tokens, dtype=dtype)
    x[5] = bits
    x[37] = bits
    x[50] = (bits.float() * 4).to(dtype)
    cache = binding.KVCache(tokens // 1024, 1024, 1, 64, dtype, DEV)
    slots = torch.arange(tokens, dtype=torch.int32, device=DEV)
    cache.write(x.to(DEV), x.flip(0).contiguous().to(DEV), slots)
    gk, gv = cache.read(slots)
    want = torch.from_numpy(held(x)).to(dtype)
    same = lambda a, b: torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float()))
    assert same(gk.cpu(), want) and same(gv.cpu(), want.flip(0))
    zeros = want == 0
    assert torch.equal(torch.signbit(gk.cpu())[zeros], torch.signbit(want)[zeros])


def test_strides_odd_rows_and_slots_outside():
    announce("kv strides and slots outside")
    dtype, D, heads, tokens = torch.bfloat16, 64, 2, 33
    cache = binding.KVCache(3, 32, heads, D, dtype, DEV)
    k, v = _tensor(heads * D, tokens, dtype, 5), _tensor(heads * D, tokens, dtype, 6)
    wide = torch.full((heads * D, 71), float("nan"), dtype=dtype, device=DEV)
    wide[:, 3:36] = k.to(DEV)
    slots = torch.arange(tokens, dtype=torch.int32) * 2 + 1
    slots[7], slots[8], slots[9] = -1, 96, 2 ** 31 - 1
    inside = (slots >= 0) & (slots < 96)
    before = cache._dev.clone()
    cache.write(wide[:, 3:36], v.to(DEV), slots.to(DEV))
    outs = torch.full((2, heads * D, 71), 7.0, dtype=dtype, device=DEV)
    gk, gv = cache.read(slots.to(DEV), k=outs[0][:, 5:38], v=outs[1][:, 30:63])
    for got, x in ((gk, k), (gv, v)):
        assert torch.equal(got.cpu()[:, inside], torch.from_numpy(held(x)).to(dtype)[:, inside])
        assert torch.isnan(got.cpu()[:, ~inside]).all()
    assert (outs[0][:, :5] == 7).all() and (outs[0][:, 38:] == 7).all() and (outs[1][:, :30] == 7).all() and (outs[1][:, 63:] == 7).all()
    cache.write(wide[:, 3:36], v.to(DEV), torch.full_like(slots, -5).to(DEV))     # nothing is written
    cache.write(wide[:, :0], wide[:, :0], slots[:0].to(DEV))                      # no tokens
    assert cache.read(slots[:0].to(DEV))[0].shape == (heads * D, 0)
    keep = torch.from_numpy(np.setdiff1d(np.arange(96), slots[inside].numpy())).int().to(DEV)
    assert not any(t.any() for t in cache.read(keep)) and before.numel() == cache.device_bytes()


def test_slots_past_32_bits_of_bytes():
    announce("kv cache of more than 4 GiB")
    D, heads, page = 128, 16, 1024
    per_page = 136 * page * heads
    pages = (1 << 32) // per_page + 40
    cache = binding.KVCache(pages, page, heads, D, torch.float16, DEV)
    assert cache.device_bytes() > 1 << 32
    k, v = _tensor(heads * D, 20, torch.float16, 8), _tensor(heads * D, 20, torch.float16, 9)
    slots = (torch.arange(20, dtype=torch.int32) * 1777 + (pages - 37) * page).to(DEV)
    assert int(slots.max()) < pages * page
    cache.write(k.to(DEV), v.to(DEV), slots)
    gk, gv = cache.read(slots)
    assert torch.equal(gk.cpu(), torch.from_numpy(held(k)).half()) and torch.equal(gv.cpu(), torch.from_numpy(held(v)).half())
