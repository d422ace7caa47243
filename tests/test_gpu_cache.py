"""Writing keys and values into quantized caches and reading them back, against the definitions in 64 bits."""
import pytest
import torch

import fp4_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
FORMATS = ["e4m3", "e2m1"]


@pytest.fixture(scope="module")
def b():
    from paper_2409_17066_b200 import build as vbuild
    vbuild.build()
    from paper_2409_17066_b200 import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def plan(lengths, starts, page, g, spare=2, hole=-1):
    """(table, start, cu, pages) of sequences with so many new tokens after so many old ones, over shuffled pages."""
    need = [ref.up(n + s, page) for n, s in zip(lengths, starts)]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    table = torch.full((len(lengths), max(need + [1])), hole, dtype=torch.int32)
    for s, n in enumerate(need):
        table[s, :n] = torch.tensor(order[:n], dtype=torch.int32)
        order = order[n:]
    return table.cuda(), ints(*starts), torch.cat([ints(0), ints(*lengths).cumsum(0).int()]), pages


def junk(b, pages, page, heads, dim, fmt, g):
    """A cache that holds something everywhere."""
    cache = b.make_cache(pages, page, heads, dim, fmt)
    for t in cache:
        if t.dtype == torch.float32:
            t.copy_(torch.rand(t.shape, generator=g, device="cuda") * 0.01 + 0.001)
        else:
            t.view(torch.uint8).copy_(torch.randint(0, 120, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    return cache


def check_write(b, k, v, cache, table, start, cu):
    """Writes, and compares the whole cache with what it has to be: the new rows by the rule, all others as they were."""
    fmt = "e4m3" if cache[0].dtype == torch.float8_e4m3fn else "e2m1"
    before = [t.clone() for t in cache]
    assert b.vptq_cache_write(k, v, *cache, table, start, cu) is None
    tokens, heads, dim = k.shape
    at = [(t, *p) for t, p in enumerate(ref.places(table, start, cu, cache[0].shape[2], cache[0].shape[0], tokens)) if isinstance(p, tuple)]
    rows, page, place = (torch.tensor([a[i] for a in at], dtype=torch.long, device="cuda") for i in range(3))
    for x, q, s, q0, s0 in ((k, cache[0], cache[1], before[0], before[1]), (v, cache[2], cache[3], before[2], before[3])):
        codes, scales = ref.row_of(x[rows].double(), fmt)
        got, got_scale = q.view(torch.uint8)[page, :, place], s[page, :, place]
        if fmt == "e4m3":
            assert torch.equal(got.view(torch.float8_e4m3fn).double()[..., :dim], codes) and torch.equal(got_scale.double(), scales.double())
            assert not got[..., dim:].any()
        else:
            assert torch.equal(ref.code_values(got, dim), codes) and torch.equal(got_scale.long(), scales + 127)
            assert not torch.stack([got & 15, got >> 4], dim=-1).flatten(-2)[..., dim:].any()
        q0.view(torch.uint8)[page, :, place] = got
        s0[page, :, place] = got_scale
        assert same(q, q0) and same(s, s0)                                             # nothing else was touched


def read_values(cache, at, tokens, dim):
    """FP64 keys and values of tokens at these places; zeros where a token's page is gone."""
    out = []
    for q, s in (cache[:2], cache[2:]):
        x = torch.zeros(tokens, q.shape[1], dim, dtype=torch.float64, device="cuda")
        for t, p in enumerate(at):
            if isinstance(p, tuple) and q.dtype == torch.uint8:
                x[t] = ref.block_values(q[p[0], :, p[1]], s[p[0], :, p[1]], dim)
            elif isinstance(p, tuple):
                x[t] = q.view(torch.uint8)[p[0], :, p[1]].view(torch.float8_e4m3fn).double()[:, :dim] * s[p[0], :, p[1]].double().repeat_interleave(128, -1)[:, :dim]
        out.append(x)
    return out


def check_read(b, cache, table, start, cu, tokens, dim, out):
    at = ref.places(table, start, cu, cache[0].shape[2], cache[0].shape[0], tokens)
    shape = (tokens, cache[0].shape[1], dim)
    kv = [torch.full(shape, 7.0, dtype=TYPES[out], device="cuda") for _ in range(2)]
    got = b.vptq_cache_read(*cache, table, start, cu, tokens, dim, out_dtype=out, k=kv[0], v=kv[1])
    assert got[0] is kv[0] and got[1] is kv[1]
    none = torch.tensor([p is None for p in at], device="cuda")
    for x, want in zip(kv, read_values(cache, at, tokens, dim)):
        # (a product of an e4m3 code and an FP32 scale is rounded to FP32 first)
        assert same(x[~none], want[~none].float().to(TYPES[out])) and (x[none] == 7.0).all()


GEOMETRY = [  # heads, dim, page, new tokens, tokens before
    (1, 64, 16, [1], [0]), (8, 128, 16, [1] * 7, [0, 1, 15, 16, 17, 31, 100]), (2, 80, 1, [3, 0, 5], [2, 0, 0]), (3, 33, 24, [0, 0, 70, 1, 0], [0, 5, 23, 24, 9]),
    (1, 1, 7, [20], [3]), (16, 256, 64, [65, 130], [63, 1]), (5, 129, 3, [2, 9], [0, 4]), (2, 192, 128, [300], [77]), (1, 500, 16, [2, 2], [0, 0]), (7, 7, 16, [40], [0]),
    (4, 96, 32, [1] * 40, list(range(40))), (2, 64, 8, [1] * 1100, [3] * 1100)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads,dim,page,lengths,starts", GEOMETRY)
def test_write_and_read(b, heads, dim, page, lengths, starts, dtype, fmt):
    g = gen(heads * 100 + dim)
    table, start, cu, pages = plan(lengths, starts, page, g)
    cache = junk(b, pages, page, heads, dim, fmt, g)
    tokens = sum(lengths)
    k, v = (torch.randn(tokens, heads, dim, generator=g, device="cuda").to(TYPES[dtype]) for _ in range(2))
    check_write(b, k, v, cache, table, start, cu)
    check_read(b, cache, table, start, cu, tokens, dim, dtype)
    # the whole sequences, with what was there before
    whole = torch.cat([ints(0), (start + cu.diff()).cumsum(0).int()])
    check_read(b, cache, table, torch.zeros_like(start), whole, min(int(whole[-1]), 1500), dim, dtype)


@pytest.mark.parametrize("fmt", FORMATS)
def test_many_tokens(b, fmt):
    g = gen(3)
    lengths, starts = [2500, 0, 1, 1999], [10, 0, 64, 33]
    table, start, cu, pages = plan(lengths, starts, 64, g)
    cache = junk(b, pages, 64, 8, 128, fmt, g)
    k, v = (torch.randn(4500, 8, 128, generator=g, device="cuda").bfloat16() for _ in range(2))
    check_write(b, k, v, cache, table, start, cu)
    check_read(b, cache, table, start, cu, 4500, 128, "bf16")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_write_reads_heads_and_tokens_apart(b, dtype, fmt):
    g = gen(4)
    table, start, cu, pages = plan([5, 6], [0, 3], 4, g)
    base = torch.randn(11 * 3000 + 5, generator=g, device="cuda").to(TYPES[dtype])
    for offset, token, head, dim in ((0, 3000, 512, 128), (1, 2999, 300, 80), (3, 640, 128, 128), (0, 1000, 100, 33), (0, 64, 640, 64), (2, 0, 128, 64), (0, 1024, 0, 64)):
        k = base[offset:].as_strided((11, 4, dim), (token, head, 1))
        v = base[offset + 1:].as_strided((11, 4, dim), (token, head, 1))
        check_write(b, k, v, junk(b, pages, 4, 4, dim, fmt, g), table, start, cu)
    # keys and values of one product; heads and tokens exchanged
    qkv = torch.randn(11, 12, 64, generator=g, device="cuda").to(TYPES[dtype])
    check_write(b, qkv[:, 4:8], qkv[:, 8:], junk(b, pages, 4, 4, 64, fmt, g), table, start, cu)
    kv = torch.randn(2, 4, 11, 64, generator=g, device="cuda").to(TYPES[dtype])
    check_write(b, kv[0].transpose(0, 1), kv[1].transpose(0, 1), junk(b, pages, 4, 4, 64, fmt, g), table, start, cu)


@pytest.mark.parametrize("fmt", FORMATS)
def test_tokens_without_a_sequence_or_a_page(b, fmt):
    """Rows before cu[0] and from cu[-1] on, pages outside the cache, positions beyond the table or below zero: left alone, and read as zeros."""
    g = gen(5)
    heads, dim, page, pages = 2, 64, 4, 6
    table = ints(0, -1, 6, 3, 2147483647, -2147483648, 5, 1, 2, 4).view(2, 5)
    for starts, cu in (([0, 0], [2, 22, 41]), ([-3, 17], [0, 10, 20]), ([2147483647, -2147483648], [0, 20, 41]), ([0, 0], [0, 0, 0]), ([0, 0], [44, 44, 60]), ([0, 3], [-5, 20, 30]),
                       ([2147483647, 0], [-2147483648, 30, 44])):
        start, cu = ints(*starts), ints(*cu)
        cache = junk(b, pages, page, heads, dim, fmt, g)
        k, v = (torch.randn(44, heads, dim, generator=g, device="cuda").half() for _ in range(2))
        check_write(b, k, v, cache, table, start, cu)
        check_read(b, cache, table, start, cu, 44, dim, "fp16")


def test_a_table_without_entries_and_no_sequences(b):
    cache = b.make_cache(2, 4, 2, 64, "e2m1")
    k = torch.ones(3, 2, 64, device="cuda")
    b.vptq_cache_write(k, k, *cache, torch.empty(1, 0, dtype=torch.int32, device="cuda"), ints(0), ints(0, 3))
    b.vptq_cache_write(k, k, *cache, torch.empty(0, 4, dtype=torch.int32, device="cuda"), ints(), ints(0))
    b.vptq_cache_write(k[:0], k[:0], *cache, ints(0, 1).view(1, 2), ints(0), ints(0, 3))
    assert not any(t.any() for t in cache)
    x, _ = b.vptq_cache_read(*cache, torch.empty(1, 0, dtype=torch.int32, device="cuda"), ints(0), ints(0, 3), 3, 64)
    assert x.dtype == torch.bfloat16 and not x.any()
    x, y = b.vptq_cache_read(*cache, ints(0, 1).view(1, 2), ints(0), ints(0, 3), 0, 64, "fp32")
    assert tuple(x.shape) == tuple(y.shape) == (0, 2, 64) and x.dtype == torch.float32


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_of_zeros_and_rows_that_are_not_numbers(b, fmt, dtype):
    table, start, cu, pages = plan([4], [0], 4, gen(6))
    cache = b.make_cache(pages, 4, 2, 160, fmt)
    k = torch.ones(4, 2, 160, device="cuda", dtype=TYPES[dtype])
    k[0] = 0
    k[1, 0, 130], k[2, 1, 5] = float("nan"), -float("inf")
    b.vptq_cache_write(k, -k, *cache, table, start, cu)
    block = 32 if fmt == "e2m1" else 128
    for out in sorted(TYPES):
        for x in b.vptq_cache_read(*cache, table, start, cu, 4, 160, out):
            bad = torch.zeros(4, 2, 160, dtype=torch.bool, device="cuda")
            bad[1, 0, 128:128 + block], bad[2, 1, :block] = True, True
            assert x[bad].isnan().all() and x[~bad].isfinite().all() and not x[0].any() and (x[3].abs() - 1).abs().max() < 0.26


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_cache_whose_offsets_pass_32_bits(b, fmt):
    """The last page of a cache of more than 2^32 bytes of codes."""
    heads, dim, page = 8, 256, 64
    row = b.vptq_cache_row_bytes(dim, fmt)
    pages = 2 ** 32 // (heads * page * row) + 3
    cache = b.make_cache(pages, page, heads, dim, fmt)
    table, start, cu = ints(pages - 1, 0, pages - 2).view(1, 3), ints(60), ints(0, 100)
    k, v = (torch.randn(100, heads, dim, generator=gen(7), device="cuda").bfloat16() for _ in range(2))
    b.vptq_cache_write(k, v, *cache, table, start, cu)
    got = b.vptq_cache_read(*cache, table, start, cu, 100, dim, "fp32")
    assert cache[0][pages - 1, :, 60:].view(torch.uint8).any() and not cache[0][pages - 1, :, :60].view(torch.uint8).any()
    for x, y in zip(got, (k, v)):
        codes, s = ref.row_of(y.double(), fmt)
        want = codes * (ref.power(s).repeat_interleave(32, -1) if fmt == "e2m1" else s.double().repeat_interleave(128, -1))
        assert torch.equal(x, want.float())


@pytest.mark.parametrize("fmt", FORMATS)
def test_layers_of_one_allocation(b, fmt):
    """The caches of several layers as parts of one tensor each."""
    g = gen(8)
    table, start, cu, pages = plan([9, 2], [3, 0], 4, g)
    stacked = [torch.stack([t] * 3) for t in junk(b, pages, 4, 3, 40, fmt, g)]
    before = [t.clone() for t in stacked]
    k, v = (torch.randn(11, 3, 40, generator=g, device="cuda").half() for _ in range(2))
    check_write(b, k, v, [t[1] for t in stacked], table, start, cu)
    check_read(b, [t[1] for t in stacked], table, start, cu, 11, 40, "bf16")
    assert all(same(t[i], t0[i]) for t, t0 in zip(stacked, before) for i in (0, 2))


def test_a_shared_prefix_is_read_by_both(b):
    g = gen(9)
    cache = junk(b, 5, 4, 2, 64, "e4m3", g)
    check_read(b, cache, ints(4, 2, 0, 4, 2, 3).view(2, 3), ints(0, 1), ints(0, 12, 21), 21, 64, "fp16")


@pytest.mark.parametrize("fmt", FORMATS)
def test_steps_of_a_generation_in_a_replayed_graph(b, fmt):
    """A captured step (product, write of one token each, read of all) replayed while the plan on the device moves on, on a stream of its own."""
    g = gen(10)
    heads, dim, page, S, most = 2, 64, 4, 3, 11
    cache = b.make_cache(20, page, heads, dim, fmt)
    table = torch.randperm(20, generator=g, device="cuda").int()[:9].view(3, 3).contiguous()
    start, cu = ints(0, 2, 3), ints(0, 1, 2, 3)
    zero, ends = ints(0, 0, 0), ints(0, 0, 0, 0)
    w, ws = ref.random_weight(2 * heads * dim, 96, g, "cuda")
    x = torch.zeros(S, 96, device="cuda", dtype=torch.bfloat16)
    k_out, v_out = (torch.zeros(S * most, heads, dim, device="cuda", dtype=torch.bfloat16) for _ in range(2))

    def step():
        kv = b.vptq_linear_fp4(x, w, ws).view(S, 2, heads, dim)
        b.vptq_cache_write(kv[:, 0], kv[:, 1], *cache, table, start, cu)
        start.add_(1)
        ends[1:] = start.cumsum(0)
        b.vptq_cache_read(*cache, table, zero, ends, S * most, dim, k=k_out, v=v_out)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
        start.copy_(ints(0, 2, 3))
        for c in cache:
            c.view(torch.uint8).zero_()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    start.copy_(ints(0, 2, 3))
    old = [[], [], []]
    for i in range(6):
        x.copy_(torch.randn(S, 96, generator=g, device="cuda"))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        kv = b.vptq_linear_fp4(x, w, ws).view(S, 2, heads, dim)
        fresh = b.make_cache(1, 3, heads, dim, fmt)
        b.vptq_cache_write(kv[:, 0], kv[:, 1], *fresh, ints(0).view(1, 1), ints(0), ints(0, 3))
        want_k, want_v = b.vptq_cache_read(*fresh, ints(0).view(1, 1), ints(0), ints(0, 3), 3, dim)
        for s in range(S):
            old[s].append((want_k[s], want_v[s]))
        at = 0
        for s, n0 in enumerate((0, 2, 3)):
            for n, (wk, wv) in enumerate(old[s]):
                assert same(k_out[at + n0 + n], wk) and same(v_out[at + n0 + n], wv), (i, s, n)
            assert not k_out[at:at + n0].any()
            at += n0 + i + 1
