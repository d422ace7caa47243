"""The 4-bit floating point operators and the caches in 64 bits, from their definitions (include/vptq.h): what the tests compare with."""
import torch

import fp8_reference as fp8

BLOCK = 32


def up(a, b):
    return -(-a // b)


def power(e):
    """2^e for whole e, in FP64."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantize(x):
    """(values [..., cols], exponents of the blocks [..., ceil(cols / 32)]) of FP64 values; a block that is not finite: NaN, exponent 128."""
    x = x.double()
    values, exponents = torch.empty_like(x), []
    for c in range(0, x.shape[-1], BLOCK):
        part = x[..., c:c + BLOCK]
        a = part.abs().amax(dim=-1, keepdim=True)
        a = torch.where(part.isfinite().all(dim=-1, keepdim=True), a, torch.full_like(a, float("nan")))
        _, e = torch.frexp(torch.where(a.isfinite(), a, torch.zeros_like(a)))          # a < 2^e
        e = e.long() - 3
        e = e + (a >= 7 * power(e)).long()                                             # 3.5 * 2^e <= a < 7 * 2^e
        e = torch.where(a > 0, e, torch.full_like(e, -127)).clamp_min(-127)
        y = (part / power(e)).abs()
        step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
        v = torch.copysign(torch.round(y / step) * step, part) * power(e)
        values[..., c:c + BLOCK] = torch.where(a.isnan(), a, v)
        exponents.append(torch.where(a.isnan(), torch.full_like(e, 128), e))
    return values, torch.cat(exponents, dim=-1)


def scale_at(r, k):
    """Where the scale byte of row r and block k lies: [row tile, block tile, row, column]."""
    return r // 128, k // 4, r % 32, r % 128 // 32 * 4 + k % 4


def scale_rows(scale, rows, cols):
    """Scale bytes [rows][blocks] out of their tiles."""
    r, k = torch.arange(rows, device=scale.device)[:, None], torch.arange(up(cols, BLOCK), device=scale.device)[None]
    return scale[scale_at(r, k)]


def scale_tiles(bytes_):
    """... and into them; what no row or block has is zero."""
    rows, blocks = bytes_.shape
    out = torch.zeros(up(rows, 128), up(blocks, 4), 32, 16, dtype=torch.uint8, device=bytes_.device)
    r, k = torch.arange(rows, device=bytes_.device)[:, None], torch.arange(blocks, device=bytes_.device)[None]
    out[scale_at(r, k)] = bytes_
    return out


def code_values(q, cols):
    """FP64 values of e2m1 codes, two a byte, without their scales."""
    code = torch.stack([q & 15, q >> 4], dim=-1).flatten(-2)[..., :cols].long()
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device=q.device)
    return table[code]


def block_values(q, bytes_, cols):
    """FP64 values [..., cols] of codes [..., bytes] with a scale byte for every block [..., blocks]."""
    s = torch.where(bytes_ == 255, torch.full(bytes_.shape, float("nan"), dtype=torch.float64, device=q.device), power(bytes_.long() - 127))
    return code_values(q, cols) * s.repeat_interleave(BLOCK, -1)[..., :cols]


def values(q, scale, cols):
    """FP64 values of an e2m1 matrix."""
    return block_values(q, scale_rows(scale, q.shape[0], cols), cols)


def linear(x, w, out_dtype):
    """(x W^T, bound of the error) for FP64 operands.  Bound: 64 exact products are added in at most 64 steps, each off by at most 2^-23 of
    the magnitudes added so far (a sum that is cut instead of rounded), and so is the addition of each such sum to the others, of which the parts
    of a split sum are at most 8 more; then the result's own rounding, half a step of its type (or half the smallest subnormal step of FP16)."""
    y = x @ w.t()
    bound = (x.abs() @ w.abs().t()) * (64 + up(x.shape[1], 64) + 8) * 2.0 ** -23
    own = torch.finfo(out_dtype).eps / 2 * (y.abs() + bound)
    return y, bound + own + (2.0 ** -25 if out_dtype == torch.float16 else 0)


def random_weight(rows, cols, gen, device, low=118, high=124):
    """An e2m1 matrix of any codes; pad codes and pad scales are zeros."""
    q = torch.zeros(rows, up(cols, BLOCK) * 16, dtype=torch.uint8, device=device)
    q[:, :up(cols, 2)] = torch.randint(0, 256, (rows, up(cols, 2)), generator=gen, device=device, dtype=torch.uint8)
    if cols % 2:
        q[:, cols // 2] &= 15
    return q, scale_tiles(torch.randint(low, high, (rows, up(cols, BLOCK)), generator=gen, device=device, dtype=torch.uint8))


# ---- caches -------------------------------------------------------------------------------------------

def places(table, start, cu, page, n_pages, tokens):
    """For every token: None in no sequence, "gone" without a page, else (page, place in it)."""
    table, start, cu = table.tolist(), start.tolist(), cu.tolist()
    out = [None] * tokens
    for s in range(len(start)):
        for t in range(max(cu[s], 0), min(cu[s + 1], tokens)):
            at = start[s] + t - cu[s]
            slot = at // page
            ok = at >= 0 and slot < len(table[s]) and 0 <= table[s][slot] < n_pages
            out[t] = (table[s][slot], at % page) if ok else "gone"
    return out


def row_of(x, fmt):
    """(code values, scales) in FP64 of FP64 rows [..., dim] as a cache holds them."""
    if fmt == "e2m1":
        v, e = quantize(x)
        return v / power(e.clamp_max(127)).repeat_interleave(BLOCK, -1)[..., :x.shape[-1]], e
    flat = x.reshape(-1, x.shape[-1])
    v, s = fp8.quantize(flat, 1)
    return v.view(x.shape), s.view(*x.shape[:-1], s.shape[1])
