"""Calls of so many tokens that a thread takes several: the same cache and the same values, bit for bit, as calls of a few thousand tokens each."""
import pytest
import torch

from test_gpu_cache import gen, ints, junk, same

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


# (pieces of a row by 4 and by 8 lanes, read and written 16 bytes at a time and value by value; more than four and more than 48 times what fills the device)
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,dim,tokens", [(1, 8, 2_000_003), (1, 7, 2_000_003), (1, 72, 1_000_001), (1, 65, 1_000_001), (2, 64, 100_001), (3, 100, 40_001)])
def test_one_call_and_many(b, heads, dim, tokens, dtype, fmt):
    g = gen(dim)
    page, first, last = 48, 3, tokens - 5                             # tokens before the first sequence and behind the last
    middle = tokens // 3
    starts, cu = [7, 0], [first, middle, last]
    width = (last - middle) // page + 2
    pages = 2 * width + 1
    table = torch.randperm(pages, generator=g, device="cuda").int()[:2 * width].view(2, width).contiguous()
    table[1, 5] = pages                                               # a page that the cache does not have
    k, v = (torch.randn(tokens, heads, dim, generator=g, device="cuda").to(TYPES[dtype]) for _ in range(2))
    cache = junk(b, pages, page, heads, dim, fmt, g)
    small = [t.clone() for t in cache]
    parts = [(s, t, min(t + 4000, cu[s + 1])) for s in range(2) for t in range(cu[s], cu[s + 1], 4000)]
    b.vptq_cache_write(k, v, *cache, table, ints(*starts), ints(*cu))
    for s, t, end in parts:
        b.vptq_cache_write(k[t:end], v[t:end], *small, table[s:s + 1], ints(starts[s] + t - cu[s]), ints(0, end - t))
    assert all(same(x, y) for x, y in zip(cache, small))
    got = [torch.full((tokens, heads, dim), 7.0, device="cuda", dtype=TYPES[dtype]) for _ in range(2)]
    want = [t.clone() for t in got]
    b.vptq_cache_read(*cache, table, ints(*starts), ints(*cu), tokens, dim, k=got[0], v=got[1])
    for s, t, end in parts:
        x, y = b.vptq_cache_read(*cache, table[s:s + 1], ints(starts[s] + t - cu[s]), ints(0, end - t), end - t, dim, dtype)
        want[0][t:end], want[1][t:end] = x, y
    assert all(same(x, y) for x, y in zip(got, want))
    assert all((x[:first] == 7).all() and (x[last:] == 7).all() and not x[middle + 5 * page:middle + 6 * page].any() for x in got)
