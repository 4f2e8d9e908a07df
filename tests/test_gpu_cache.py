"""GPU: keys and values quantised into a paged cache: symbols, scales and zero-points equal to the formula's, and what is read back equal to
scale * (symbol - zero-point)."""
import numpy as np
import pytest
import torch

import operators_plain as P
from paper_2406_06237_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _write(cache, k, v, slots):
    B.cache_write(cache, k, v, torch.tensor(slots, dtype=torch.int64, device=DEV))


def _vector(t, slot, page):
    return t[slot // page, :, slot % page].cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,page", [(1, 16), (3, 32), (8, 128)])
def test_symbols_and_values(heads, page, dim, bits, dtype):
    g = torch.Generator(device=DEV).manual_seed(dim + bits)
    cache = B.new_kv_cache(5, page, heads, dim, bits)
    qkv = torch.randn(37, 3, heads, dim, device=DEV, generator=g).to(dtype)
    k, v = qkv[:, 1], qkv[:, 2] * torch.rand(37, heads, 1, device=DEV, generator=g).to(dtype)
    k[3] += 5                                                          # nothing below zero
    k[4] = -k[4].abs()
    k[5] = 0
    v[6, 0, 1:] = 0
    slots = torch.randperm(5 * page, generator=torch.Generator().manual_seed(1))[:37].tolist()
    _write(cache, k, v, slots)
    got = B.cache_read(cache, torch.tensor(slots, device=DEV), "f32")
    rounded = B.cache_read(cache, torch.tensor(slots, device=DEV), "bf16")
    for x, symbols, params, back, short in ((k, cache.k, cache.k_params, got[0], rounded[0]), (v, cache.v, cache.v_params, got[1], rounded[1])):
        q, scale, zero = P.quantise(x, bits)
        for i, s in enumerate(slots):
            assert np.array_equal(_vector(symbols, s, page), P.packed(q[i], bits)), i
            assert np.array_equal(_vector(params, s, page), np.stack([scale[i], zero[i]], -1)), i
        want = torch.from_numpy(scale[..., None] * (q.astype(np.float32) - zero[..., None]))
        assert torch.equal(back.cpu(), want)
        assert torch.equal(short.cpu(), want.to(torch.bfloat16))
        assert ((want - x.cpu().float()).abs() <= torch.from_numpy(scale)[..., None] * 0.5001 + 1e-30).all()
    assert cache.status.tolist() == [0, 0]


@pytest.mark.parametrize("bits", [8, 4])
def test_vectors_that_have_no_scale(bits):
    cache = B.new_kv_cache(1, 16, 2, 64, bits)
    k = torch.randn(5, 2, 64, device=DEV)
    k[0, 0, 3] = float("nan")
    k[1, 0, 63] = float("inf")
    k[2, 0, 0], k[2, 0, 1] = 3e38, -3e38                               # a range beyond 32 bits
    k[3, 0] = 1e-44                                                    # one below what can be divided
    k[4, 0, :32], k[4, 0, 32:] = 1e-37, -2e-38
    _write(cache, k, k, [0, 1, 2, 3, 4])
    got, _ = B.cache_read(cache, torch.arange(5, device=DEV), "f32")
    assert torch.isnan(got[:3, 0]).all() and torch.isfinite(got[:, 1]).all() and torch.isfinite(got[3:]).all()
    q, scale, zero = P.quantise(k, bits)
    assert np.array_equal(cache.k[0, :, :5].cpu().numpy().transpose(1, 0, 2), P.packed(q, bits))
    assert np.array_equal(cache.k_params[0, :, :5].cpu().numpy().transpose(1, 0, 2), np.stack([scale, zero], -1), equal_nan=True)


def test_slots_that_are_not_there():
    cache = B.new_kv_cache(2, 16, 2, 64)
    k = torch.randn(4, 2, 64, device=DEV)
    _write(cache, k, k, [-1, 31, 32, 1 << 40])
    assert cache.status.tolist() == [B.ST_BAD_DESC, 2]
    assert (cache.k_params[0] == 0).all() and (cache.k_params[1, :, :15] == 0).all() and (cache.k_params[1, :, 15, 0] > 0).all()
    cache.status.zero_()
    got, _ = B.cache_read(cache, torch.tensor([-5, 31, 32, 0], device=DEV), "f32")
    assert (got[[0, 2, 3]] == 0).all() and (got[1] != 0).any()
    assert cache.status.tolist() == [B.ST_BAD_DESC, 1]
    cache.status = None
    B.cache_read(cache, torch.tensor([99], device=DEV))
    _write(cache, k[:0], k[:0], [])
    assert B.cache_read(cache, torch.zeros(0, dtype=torch.int64, device=DEV))[0].shape == (0, 2, 64)


def test_a_cache_of_more_than_4_gib():
    heads, dim, page = 8, 128, 64
    pages = (5 << 30) // (heads * dim * page)
    cache = B.KvCache(torch.empty(pages, heads, page, dim, dtype=torch.uint8, device=DEV), torch.empty(pages, heads, page, 2, device=DEV),
                      torch.empty(pages, heads, page, dim, dtype=torch.uint8, device=DEV), torch.empty(pages, heads, page, 2, device=DEV))
    k, v = torch.randn(2, 70, heads, dim, device=DEV)
    slots = torch.cat([torch.arange(35), pages * page - 1 - torch.arange(35)]).to(DEV)
    B.cache_write(cache, k, v, slots)
    got = B.cache_read(cache, slots, "f32")
    for x, y in zip((k, v), got):
        q, scale, zero = P.quantise(x, 8)
        assert torch.equal(y.cpu(), torch.from_numpy(scale[..., None] * (q.astype(np.float32) - zero[..., None])))


def test_vectors_beyond_one_dimension_of_a_launch():
    """More vectors than 2^32 threads have lanes for.  Few of the tokens are written: the others have a negative slot."""
    heads, dim, tokens = 65535, 256, 2050
    cache = B.new_kv_cache(1, 16, heads, dim)
    k = torch.randn(1, heads, dim, device=DEV).to(torch.bfloat16)
    slots = torch.full((tokens,), -1, dtype=torch.int64, device=DEV)
    slots[torch.tensor([0, 1023, 1025, 2047, 2048, 2049])] = torch.tensor([3, 0, 7, 8, 15, 12], device=DEV)
    B.cache_write(cache, k.expand(tokens, heads, dim), (-k).expand(tokens, heads, dim), slots)
    less = B.new_kv_cache(1, 16, heads, dim)
    B.cache_write(less, k.expand(6, heads, dim), (-k).expand(6, heads, dim), slots[slots >= 0])
    for a, b in ((cache.k, less.k), (cache.v, less.v), (cache.k_params, less.k_params), (cache.v_params, less.v_params)):
        assert torch.equal(a, b)
    assert (less.k_params[0, :, [0, 3, 7, 8, 12, 15], 0] > 0).all()
