"""Performance cases of the operators over 4-bit floating point and over quantized caches, through the package's public entry points.

A case is one pass of a program that serves a model:

  quantize  a matrix to e2m1 with a power of two as the scale of every 32 columns of a row, and its values read back
            (vptq_fp4_quantize, vptq_fp4_values)
  restore   a vector-quantized layer straight to such a weight, and its values read back (vptq_dequant_fp4, vptq_fp4_values)
  linear    out = x W^T with such a weight; x in 16 bits, quantized in the call, or in e2m1 already (vptq_linear_fp4)
  write     keys and values of new tokens into the pages of a cache in e4m3 or e2m1 (vptq_cache_write); e2m1: and read back
  read      keys and values of sequences out of the pages of such a cache (vptq_cache_read)

An e2m1 matrix is [rows][16 * ceil(columns / 32)] bytes, two columns a byte, the lower one in the low half; a code is a sign and one of
0, 0.5, 1, 1.5, 2, 3, 4, 6.  The scale of a block of 32 columns is a byte b that stands for 2^(b - 127).  The rule: a = max(|x|) over the
block lies in [3.5, 7) * 2^e, b = e + 127 but at least 0 (0 for a = 0), code = x / 2^(b - 127) to the nearest value, ties to the even code.
Scales lie in tiles of 128 rows and four blocks: [row tiles][block tiles][32][16], the one of row r and block k at
[r / 128][k / 4][r % 32][r % 128 / 32 * 4 + k % 4]; the bytes of rows and blocks that the matrix does not have are zero.

A cache has pages of a few tokens, [pages][heads][tokens of a page][bytes of a row], and scales beside them, [pages][heads][tokens of a
page][blocks of a row]: e4m3 with an FP32 scale for 128 columns (a = max(|x|), at least 2^-100, scale a / 448, codes x * (448 / a)), or
e2m1 as above, its scales in the order of the blocks.  Token cu[s] + i of a call is token start[s] + i of sequence s, in the page
table[s][token / tokens of a page].
"""
from __future__ import annotations

import torch

own = False

#: name -> (v, k1, k2, percent of outlier columns, v0, k0): formats of vector-quantized layers
FORMATS = {
    "v8_256": (8, 256, 0, 0.0, 0, 0),
    "v8_65536": (8, 65536, 0, 0.0, 0, 0),
    "v8_65536_256": (8, 65536, 256, 0.0, 0, 0),
    "v6_4096_256_out": (6, 4096, 256, 1.0, 4, 4096),
}
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # the input of one projection while one user generates: latency only
        dict(name="quantize_row_b1", kind="quantize", rows=1, cols=4096, x="fp16"),
        # the weight of a 70B model's gate projection, when the model is loaded
        dict(name="quantize_70b_gate", kind="quantize", rows=28672, cols=8192, x="bf16"),
        # a compressed projection of a 7B model, restored for prompts
        dict(name="restore_7b_q", kind="restore", fmt="v8_65536", M=4096, N=4096),
        # one with a residual codebook and outlier columns, 11008 rows in vectors of 6
        dict(name="restore_7b_gate_out", kind="restore", fmt="v6_4096_256_out", M=11008, N=4096),
        # one projection while a 7B model generates for one user; a 70B model's gate projection for 16 users
        dict(name="linear_7b_q_b1", kind="linear", M=4096, N=4096, B=1, x="fp16", out="fp16"),
        dict(name="linear_70b_gate_b16", kind="linear", M=28672, N=8192, B=16, x="bf16", out="bf16"),
        # prompts: an 8B model's gate projection over 500 tokens with FP32 results; a 70B model's down projection, input quantized before
        dict(name="linear_8b_gate_500", kind="linear", M=14336, N=4096, B=500, x="bf16", out="fp32"),
        dict(name="linear_70b_down_2048", kind="linear", M=8192, N=28672, B=2048, x="e2m1", out="bf16"),
        # one new token each of 64 users: latency; ragged prompts of five users
        dict(name="write_64_users", kind="write", fmt="e4m3", x="bf16", T=64, S=64, heads=8, dim=128, page=16),
        dict(name="write_prompts", kind="write", fmt="e2m1", x="fp16", T=16000, S=5, heads=8, dim=128, page=64),
        # a long conversation of one user read back; ragged ones of 24 users
        dict(name="read_one_user", kind="read", fmt="e4m3", out="bf16", T=5001, S=1, heads=8, dim=128, page=16),
        dict(name="read_24_users", kind="read", fmt="e2m1", out="bf16", T=130000, S=24, heads=8, dim=128, page=64),
    ]


def draw(rng):
    def size(lo, hi):                                   # spread over the logarithm; round, nearly round or odd
        n = int(lo * (hi / lo) ** rng.random())
        step = rng.choice([1, 16, 128])
        return max(lo, min(hi, n // step * step))

    kind = rng.choice(["quantize", "restore", "linear", "linear", "write", "read"])
    if kind == "quantize":
        return dict(kind=kind, rows=size(1, 8192), cols=size(32, 14336), x=rng.choice(["fp16", "bf16", "fp32"]))
    if kind == "restore":
        return dict(kind=kind, fmt=rng.choice(sorted(FORMATS)), M=size(256, 14336), N=size(512, 8192))
    if kind == "linear":
        return dict(kind=kind, M=size(64, 16384), N=size(128, 14336), B=size(1, 2048), x=rng.choice(["fp16", "bf16", "e2m1"]),
                    out=rng.choice(["fp16", "bf16", "fp32"]))
    dim = rng.choice([64, 72, 80, 96, 128, 192, 256])
    c = dict(kind=kind, fmt=rng.choice(["e4m3", "e2m1"]), S=size(1, 128), heads=rng.randint(1, 16), dim=dim, page=rng.choice([1, 16, 24, 64, 128]))
    if kind == "write":
        return dict(c, x=rng.choice(["fp16", "bf16", "fp32"]), T=min(size(1, 16384), 2 ** 24 // (c["heads"] * dim)))
    return dict(c, out=rng.choice(["fp16", "bf16", "fp32"]), T=min(size(1, 131072), 2 ** 26 // (c["heads"] * dim)))


# ---- inputs ------------------------------------------------------------------------------------------

def _up(a, b):
    return -(-a // b)


def _activations(gen, rows, cols, kind):
    """Unit normal, with a few features that are much larger than the others, as hidden states have them."""
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    loud = torch.rand(cols, generator=gen, device="cuda") < 0.004
    return (x * (1 + 15 * loud)).to(TYPES[kind])


def _bits(k):
    return max(1, (k - 1).bit_length())


def _pack(idx, bits):
    """Little-endian bit stream of every row, rows padded to 16 bytes (bits = 8, 12 or 16)."""
    rows, cols = idx.shape
    packed = torch.zeros((rows, _up(_up(cols * bits, 8), 16) * 16), dtype=torch.uint8, device="cuda")
    if bits == 8:
        packed[:, :cols] = idx.to(torch.uint8)
    elif bits == 16:
        packed[:, : 2 * cols : 2] = (idx & 255).to(torch.uint8)
        packed[:, 1 : 2 * cols : 2] = (idx >> 8).to(torch.uint8)
    else:
        pair = torch.zeros((rows, 2 * _up(cols, 2)), dtype=torch.int32, device="cuda")
        pair[:, :cols] = idx
        a, b = pair[:, ::2], pair[:, 1::2]
        three = torch.stack([a & 255, (a >> 8) | ((b & 15) << 4), b >> 4], dim=2).flatten(1).to(torch.uint8)
        packed[:, : _up(cols * 12, 8)] = three[:, : _up(cols * 12, 8)]
    return packed


def _restore_geometry(c):
    v, k1, k2, percent, v0, k0 = FORMATS[c["fmt"]]
    return v, k1, k2, int(percent / 100 * c["N"] + 0.5), v0, k0


def _weight(gen, rows, cols, sd):
    """An e2m1 weight as a checkpoint in this format holds it; made in parts, for the memory's sake."""
    parts = [_quantize(torch.randn((min(4096, rows - r), cols), generator=gen, device="cuda") * sd) for r in range(0, rows, 4096)]
    return torch.cat([q for q, _ in parts]), _tiles(torch.cat([b for _, b in parts]))


def _sequences(gen, case, before):
    """Ragged lengths that make T tokens, the tokens that each sequence has before them (at most `before`), and tables over shuffled pages."""
    S, T, page = case["S"], case["T"], case["page"]
    share = torch.rand(S, generator=gen, device="cuda").cumsum(0) + torch.arange(S, device="cuda") * 0.5
    cu = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    cu[1:] = T if S == 1 else torch.round(share / share[-1] * T).int()
    if T == S:
        cu = torch.arange(S + 1, dtype=torch.int32, device="cuda")
    start = torch.randint(0, before + 1, (S,), generator=gen, device="cuda", dtype=torch.int32)
    pages = [_up(n, page) for n in (start + cu.diff()).tolist()]
    total, most = _up(T, page) + S * (_up(before, page) + 1), max(max(pages), 1)      # (enough for any lengths)
    order, table, at = torch.randperm(total, generator=gen, device="cuda").int(), torch.full((S, most), -1, dtype=torch.int32, device="cuda"), 0
    for s, n in enumerate(pages):
        table[s, :n] = order[at : at + n]
        at += n
    return cu, start, table, total


def _cache(gen, case, total):
    """Pages as earlier calls have left them."""
    dim, shape = case["dim"], (total, case["heads"], case["page"])
    if case["fmt"] == "e4m3":
        q = torch.zeros((*shape, _up(dim, 16) * 16), dtype=torch.float8_e4m3fn, device="cuda")
        q[..., :dim].copy_(torch.randn((*shape, dim), generator=gen, device="cuda", dtype=torch.float16).mul_(110).clamp_(-448, 448))
        return q, (torch.rand((*shape, _up(dim, 128)), generator=gen, device="cuda") + 0.5) * 0.009
    q = torch.zeros((*shape, _up(dim, 32) * 16), dtype=torch.uint8, device="cuda")
    q[..., : _up(dim, 2)] = torch.randint(0, 256, (*shape, _up(dim, 2)), generator=gen, device="cuda", dtype=torch.uint8)
    if dim % 2:
        q[..., dim // 2] &= 15
    return q, torch.randint(124, 128, (*shape, _up(dim, 32)), generator=gen, device="cuda", dtype=torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case)
    if case["kind"] == "quantize":
        x = _activations(gen, case["rows"], case["cols"], "fp32")
        s["data"] = (x if case["rows"] < 4096 else x.mul_(0.02)).to(TYPES[case["x"]])
    elif case["kind"] == "restore":
        M, N = case["M"], case["N"]
        v, k1, k2, n_out, v0, k0 = _restore_geometry(case)

        def stream(k, rows, cols):
            return _pack(torch.randint(0, k, (rows, cols), generator=gen, device="cuda", dtype=torch.int32), _bits(k)) if k and cols else None

        def table(k, length, sd):
            return (torch.randn((k, length), generator=gen, device="cuda") * sd).half() if k else None

        s.update(idx1=stream(k1, _up(M, v), N - n_out), idx2=stream(k2, _up(M, v), N - n_out), idx0=stream(k0, _up(M, v0) if v0 else 0, n_out),
                 c1=table(k1, v, 0.02), c2=table(k2, v, 0.005), c0=table(k0, v0, 0.02),
                 scale=(torch.rand(N, generator=gen, device="cuda") + 0.5).half(), bias=(torch.randn(N, generator=gen, device="cuda") * 0.01).half())
    elif case["kind"] == "linear":
        s["w"], s["w_scale"] = _weight(gen, case["M"], case["N"], 0.02)
        s["data"], s["x_scale"] = _activations(gen, case["B"], case["N"], "fp32" if case["x"] == "e2m1" else case["x"]), None
        if case["x"] == "e2m1":
            q, b = _quantize(s["data"])
            s["data"], s["x_scale"] = q, _tiles(b)
    else:
        s["cu"], s["start"], s["table"], total = _sequences(gen, case, 200 if case["kind"] == "write" else 0)
        s["k_cache"], s["k_scale"] = _cache(gen, case, total)
        s["v_cache"], s["v_scale"] = _cache(gen, case, total)
        if case["kind"] == "write":
            # keys and values out of one product, beside one another
            kv = _activations(gen, case["T"], 2 * case["heads"] * case["dim"], case["x"]).view(case["T"], 2, case["heads"], case["dim"])
            s["k"], s["v"] = kv[:, 0], kv[:, 1]
    return s


# ---- the operators in their plain form ---------------------------------------------------------------

def _blocks(x):
    """The last dimension padded with zeros to blocks of 32: [..., blocks, 32]."""
    full = torch.zeros((*x.shape[:-1], _up(x.shape[-1], 32) * 32), dtype=x.dtype, device=x.device)
    full[..., : x.shape[-1]] = x
    return full.view(*x.shape[:-1], -1, 32)


def _power(b):
    """2^(b - 127), put together from its bits."""
    b = b.int()
    return torch.where(b > 0, b << 23, torch.full_like(b, 1 << 22)).view(torch.float32)


def _quantize(x):
    """e2m1 bytes [..., 16 * blocks] and scale bytes [..., blocks] of FP32 values."""
    x = _blocks(x)
    a = x.abs().amax(dim=-1)
    m, e = torch.frexp(a)                                # a = m * 2^e, m in [0.5, 1): 7 * 2^k is 0.875 * 2^(k + 3)
    b = (e - 3 + (m >= 0.875).int() + 127).clamp_min(0)
    b = torch.where(a > 0, b, torch.zeros_like(b))
    y = x / _power(b)[..., None]
    code = torch.zeros_like(y, dtype=torch.uint8)
    # the borders between neighbours; a tie goes to the even code
    for i, border in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += ((y.abs() > border) if i % 2 == 0 else (y.abs() >= border)).to(torch.uint8)
    code += (torch.signbit(y)).to(torch.uint8) * 8
    return (code[..., ::2] | code[..., 1::2] << 4).flatten(-2), b.to(torch.uint8)


def _values(q, b, cols):
    """FP32 values [..., cols] of e2m1 bytes and their blocks' scale bytes."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=q.device)
    code = torch.stack([q & 15, q >> 4], dim=-1).flatten(-2)
    return (table[code.int()].view(*b.shape, 32) * _power(b)[..., None]).flatten(-2)[..., :cols]


def _tiles(b):
    """Scale bytes [rows][blocks] as tiles of 128 rows and four blocks."""
    rows, blocks = b.shape
    full = torch.zeros((_up(rows, 128) * 128, _up(blocks, 4) * 4), dtype=torch.uint8, device=b.device)
    full[:rows, :blocks] = b
    return full.view(-1, 4, 32, full.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(full.shape[0] // 128, full.shape[1] // 4, 32, 16)


def _rows_of(tiles, rows, blocks):
    """... and back."""
    n, k = tiles.shape[:2]
    return tiles.view(n, k, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(n * 128, k * 4)[:rows, :blocks]


def _unpack(packed, cols, bits):
    if bits == 8:
        return packed[:, :cols].int()
    if bits == 16:
        return packed[:, : 2 * cols : 2].int() | packed[:, 1 : 2 * cols : 2].int() << 8
    three = torch.zeros((packed.shape[0], 3 * _up(cols, 2)), dtype=torch.int32, device=packed.device)
    three[:, : _up(cols * 12, 8)] = packed[:, : _up(cols * 12, 8)].int()
    a, b, c = three[:, ::3], three[:, 1::3], three[:, 2::3]
    return torch.stack([a | (b & 15) << 8, b >> 4 | c << 4], dim=2).flatten(1)[:, :cols]


def _look_up(table, idx, length, rows):
    """The columns of centroids that an index matrix names, [rows][columns] in FP32."""
    return table[idx.long()].float().permute(0, 2, 1).reshape(idx.shape[0] * length, -1)[:rows]


def _restore(s):
    M, N = s["M"], s["N"]
    v, k1, k2, n_out, v0, k0 = _restore_geometry(s)
    t = _look_up(s["c1"], _unpack(s["idx1"], N - n_out, _bits(k1)), v, M)
    if k2:
        t = t + _look_up(s["c2"], _unpack(s["idx2"], N - n_out, _bits(k2)), v, M)
    if n_out:
        t = torch.cat([_look_up(s["c0"], _unpack(s["idx0"], n_out, _bits(k0)), v0, M), t], dim=1)
    return (t * s["scale"].float() + s["bias"].float()).half().float()


def _quantize_e4m3(x):
    """e4m3 [..., columns padded to 16] and FP32 scales [..., ceil(columns / 128)] of FP32 values."""
    cols = x.shape[-1]
    full = torch.zeros((*x.shape[:-1], _up(cols, 128) * 128), device=x.device)
    full[..., :cols] = x
    b = full.view(*x.shape[:-1], -1, 128)
    a = b.abs().amax(dim=-1).clamp_min(2.0 ** -100)
    most = torch.full_like(a, 448.0)                    # (a quotient with a plain number would be a product with its reciprocal)
    return (b * (most / a)[..., None]).to(torch.float8_e4m3fn).flatten(-2)[..., : _up(cols, 16) * 16], a / most


def _places(s):
    """(page, token of the page) of every token of the call."""
    seq = torch.repeat_interleave(torch.arange(s["S"], device="cuda"), s["cu"].diff().long(), output_size=s["T"])
    token = s["start"][seq].long() + torch.arange(s["T"], device="cuda") - s["cu"][seq].long()
    return s["table"][seq, token // s["page"]].long(), token % s["page"]


def _read(s, cache, scale):
    page, at = _places(s)
    q, b = cache.view(torch.uint8)[page, :, at], scale[page, :, at]
    if s["fmt"] == "e2m1":
        return _values(q, b, s["dim"])
    return q.view(torch.float8_e4m3fn)[..., : s["dim"]].float() * b.repeat_interleave(128, dim=-1)[..., : s["dim"]]


def _write(s):
    page, at = _places(s)
    for name in ("k", "v"):
        q, b = (_quantize if s["fmt"] == "e2m1" else _quantize_e4m3)(s[name].float())
        s[name + "_cache"].view(torch.uint8)[page, :, at] = q.view(torch.uint8)
        s[name + "_scale"][page, :, at] = b


def run(state):
    if own:
        return _run_own(state)
    s = state
    if s["kind"] == "quantize":
        return _values(*_quantize(s["data"].float()), s["cols"]).bfloat16()
    if s["kind"] == "restore":
        return _values(*_quantize(_restore(s)), s["N"]).bfloat16()
    if s["kind"] == "linear":
        blocks = _up(s["N"], 32)
        x = _values(s["data"], _rows_of(s["x_scale"], s["B"], blocks), s["N"]) if s["x"] == "e2m1" else _values(*_quantize(s["data"].float()), s["N"])
        w = _values(s["w"], _rows_of(s["w_scale"], s["M"], blocks), s["N"])
        if s["out"] == "fp32":                              # 32 bits lose too much of a sum of thousands for a result in 32 bits
            return (x.double() @ w.double().t()).float()
        return (x @ w.t()).to(TYPES[s["out"]])
    if s["kind"] == "write":
        _write(s)
        if s["fmt"] == "e4m3":
            return s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"]
        return _read(s, s["k_cache"], s["k_scale"]).bfloat16(), _read(s, s["v_cache"], s["v_scale"]).bfloat16()
    return _read(s, s["k_cache"], s["k_scale"]).to(TYPES[s["out"]]), _read(s, s["v_cache"], s["v_scale"]).to(TYPES[s["out"]])


# ---- the calls of a user's program -------------------------------------------------------------------

def _run_own(s):
    from paper_2409_17066_b200 import binding as vb

    if s["kind"] == "quantize":
        q, scale = vb.vptq_fp4_quantize(s["data"])
        return vb.vptq_fp4_values(q, scale, s["cols"], out_dtype="bf16")
    if s["kind"] == "restore":
        v, k1, k2, n_out, v0, k0 = _restore_geometry(s)
        desc = vb.make_desc(s["M"], s["N"], v, k1, k2, n_out, v0, k0)
        q, scale = vb.vptq_dequant_fp4(desc, vb.LayerPtrs(*[None if s[n] is None else s[n].data_ptr() for n in ("idx1", "c1", "idx2", "c2", "idx0", "c0", "scale", "bias")]))
        return vb.vptq_fp4_values(q, scale, s["N"], out_dtype="bf16")
    if s["kind"] == "linear":
        return vb.vptq_linear_fp4(s["data"], s["w"], s["w_scale"], x_scale=s["x_scale"], out_dtype=s["out"])
    cache = (s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"])
    if s["kind"] == "write":
        vb.vptq_cache_write(s["k"], s["v"], *cache, s["table"], s["start"], s["cu"])
        if s["fmt"] == "e4m3":
            return cache
        return vb.vptq_cache_read(*cache, s["table"], s["start"], s["cu"], s["T"], s["dim"], out_dtype="bf16")
    return vb.vptq_cache_read(*cache, s["table"], s["start"], s["cu"], s["T"], s["dim"], out_dtype=s["out"])


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    size = {"fp16": 2, "bf16": 2, "fp32": 4}

    def e2m1(rows, cols):                               # codes and scales
        return rows * 17.0 * _up(cols, 32)

    if case["kind"] == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["x"]] + 2.0) + e2m1(case["rows"], case["cols"]), "flops": 3.0 * n}
    if case["kind"] == "restore":
        M, N = case["M"], case["N"]
        v, k1, k2, n_out, v0, k0 = _restore_geometry(case)
        nbytes = _up(M, v) * (N - n_out) * (_bits(k1) + (_bits(k2) if k2 else 0)) / 8 + 2.0 * v * (k1 + k2) + 4.0 * N
        nbytes += _up(M, v0) * n_out * _bits(k0) / 8 + 2.0 * v0 * k0 if n_out else 0
        return {"bytes": nbytes + e2m1(M, N) + 2.0 * M * N, "flops": 6.0 * M * N}
    if case["kind"] == "linear":
        M, N, B = case["M"], case["N"], case["B"]
        x = e2m1(B, N) if case["x"] == "e2m1" else 2.0 * B * N
        return {"bytes": e2m1(M, N) + x + 1.0 * B * M * size[case["out"]], "flops": 2.0 * B * M * N}
    rows = 2.0 * case["T"] * case["heads"]
    held = e2m1(rows, case["dim"]) if case["fmt"] == "e2m1" else rows * (_up(case["dim"], 16) * 16 + 4.0 * _up(case["dim"], 128))
    if case["kind"] == "read":
        return {"bytes": held + rows * case["dim"] * size[case["out"]], "flops": rows * case["dim"]}
    back = 2.0 * rows * case["dim"] if case["fmt"] == "e2m1" else 0.0
    return {"bytes": held + rows * case["dim"] * size[case["x"]] + back, "flops": 2.0 * rows * case["dim"]}


# ---- the definition in 64 bits -----------------------------------------------------------------------

def _power_64(e):
    return ((e + 1023) << 52).view(torch.float64)


def _e2m1_64(x):
    """The FP64 values that FP64 values [..., columns] read back as."""
    out = torch.empty_like(x)
    for c in range(0, x.shape[-1], 32):
        part = x[..., c : c + 32]
        a = part.abs().amax(dim=-1, keepdim=True)
        e = ((a / 1.75).view(torch.int64) >> 52) - 1023 - 1        # a in [3.5, 7) * 2^e: a / 1.75 in [2, 4) * 2^e
        # (7 * 2^k / 1.75 is exact; a quotient below never rounds up to it, with 29 bits to spare behind those of a 32-bit value)
        scale = _power_64(e.clamp_min(-127))
        y = (part / scale).abs()
        step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
        out[..., c : c + 32] = torch.copysign(torch.round(y / step) * step, part) * scale
    return out


def _codes_64(q, b, cols):
    """FP64 values of codes that are given."""
    q = torch.stack([q & 15, q >> 4], dim=-1).flatten(-2).double()[..., :cols]
    sign, m = torch.where(q >= 8, -1.0, 1.0), q % 8
    magnitude = torch.where(m < 4, m / 2, torch.where(m < 6, m - 2, 2 * m - 8))
    block = torch.arange(cols, device=q.device) // 32
    return sign * magnitude * _power_64(b.long() - 127)[..., block]


def _tiled_64(q, tiles, rows, cols):
    r, k = torch.arange(rows, device=q.device)[:, None], torch.arange(_up(cols, 32), device=q.device)[None]
    return _codes_64(q, tiles[r // 128, k // 4, r % 32, r % 128 // 32 * 4 + k % 4], cols)


def _e4m3_64(x):
    """(e4m3 codes' FP64 values, FP64 scales) of FP64 values; every constant and quotient that the rule rounds to FP32 is."""
    q, scales = torch.empty_like(x), []
    for c in range(0, x.shape[-1], 128):
        part = x[..., c : c + 128]
        a = part.abs().amax(dim=-1, keepdim=True).clamp_min(2.0 ** -100)
        most = torch.full_like(a, 448)
        v = (part * (most / a).float().double()).float().double()
        exponent = (v.abs().view(torch.int64) >> 52).clamp_min(1023 - 6)     # biased; below 2^-6 the steps are those of 2^-6
        step = ((exponent - 3) << 52).view(torch.float64)
        q[..., c : c + 128] = (torch.round(v / step) * step).clamp(-448, 448)
        scales.append((a / most).float().double())
    return q, torch.cat(scales, dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "quantize":
        return torch.cat([_e2m1_64(part.double()) for part in s["data"].split(4096)])
    if s["kind"] == "restore":
        M, N = s["M"], s["N"]
        v, k1, k2, n_out, v0, k0 = _restore_geometry(s)
        W = torch.empty((M, N), dtype=torch.float64, device="cuda")
        i1 = _unpack(s["idx1"], N - n_out, _bits(k1)).long()
        i2 = _unpack(s["idx2"], N - n_out, _bits(k2)).long() if k2 else None
        for j in range(v):                              # component j of every vector: rows j, j + v, ...
            n = len(range(j, M, v))
            t = s["c1"].double()[:, j][i1[:n]]
            W[j::v, n_out:] = t if i2 is None else (t + s["c2"].double()[:, j][i2[:n]]).float().double()
        if n_out:
            i0 = _unpack(s["idx0"], n_out, _bits(k0)).long()
            for j in range(v0):
                W[j::v0, :n_out] = s["c0"].double()[:, j][i0[: len(range(j, M, v0))]]
        W = (W * s["scale"].double()).float().double() + s["bias"].double()
        return _e2m1_64(W.float().half().double())
    if s["kind"] == "linear":
        N = s["N"]
        x = _tiled_64(s["data"], s["x_scale"], s["B"], N) if s["x"] == "e2m1" else _e2m1_64(s["data"].double())
        return torch.cat([x @ _tiled_64(q, t, q.shape[0], N).t() for q, t in zip(s["w"].split(4096), s["w_scale"].split(32))], dim=1)
    # token by token of every sequence
    cu, start = s["cu"].tolist(), s["start"].tolist()
    at = [(i, start[n] + i - cu[n], n) for n in range(s["S"]) for i in range(cu[n], cu[n + 1])]
    rows, token, seq = (torch.tensor(t, device="cuda") for t in zip(*at))
    page, place = s["table"][seq, token // s["page"]].long(), token % s["page"]
    dim, result = s["dim"], []
    for name in ("k", "v"):
        cache, scale = s[name + "_cache"], s[name + "_scale"]
        if s["kind"] == "write" and s["fmt"] == "e4m3":
            q, b = _e4m3_64(s[name].double())
            cache, scale = cache.double(), scale.double()
            cache[page, :, place] = 0
            cache[page, :, place, :dim] = q[rows]
            scale[page, :, place] = b[rows]
            result += [cache, scale]
        elif s["kind"] == "write":
            result.append(_e2m1_64(s[name].double()))
        else:
            out = torch.empty((s["T"], s["heads"], dim), dtype=torch.float64, device="cuda")
            for part in torch.arange(len(rows), device="cuda").split(16384):
                q, b = cache.view(torch.uint8)[page[part], :, place[part]], scale[page[part], :, place[part]]
                if s["fmt"] == "e2m1":
                    out[rows[part]] = _codes_64(q, b, dim)
                else:
                    block = torch.arange(dim, device="cuda") // 128
                    out[rows[part]] = q.view(torch.float8_e4m3fn).double()[..., :dim] * b.double()[..., block]
            result.append(out)
    return tuple(result)
