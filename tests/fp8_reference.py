"""The 8-bit floating point operators in 64 bits, from their definitions (include/vptq.h): what the tests compare with."""
import torch

BLOCK = 128


def pitch(cols):
    return -(-cols // 16) * 16


def e4m3(v):
    """Nearest e4m3 value (no infinities, largest 448, subnormals in steps of 2^-9) of FP64 values within its range, ties to even."""
    exponent = (v.abs().view(torch.int64) >> 52).clamp_min(1023 - 6)
    step = ((exponent - 3) << 52).view(torch.float64)
    return (torch.round(v / step) * step).clamp(-448, 448)


def expand(scale, rows, cols, block_rows):
    return scale.double().repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def quantize(x, block_rows):
    """(values [rows][cols], scale) in FP64; the scale and the factor are FP32 numbers, as is every product before its rounding."""
    x = x.double()
    rows, cols = x.shape
    full = torch.zeros(-(-rows // block_rows) * block_rows, -(-cols // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    full[:rows, :cols] = x.abs()
    top = full.view(-1, block_rows, full.shape[1] // BLOCK, BLOCK).amax(dim=(1, 3)).clamp_min(2.0 ** -100)
    most = torch.full_like(top, 448)
    factor = (most / top).float()
    return e4m3((x * expand(factor, rows, cols, block_rows)).float().double()), (top / most).float()


def values(q, scale, cols, block_rows):
    """FP64 values of an e4m3 matrix with block scales."""
    return q.double()[:, :cols] * expand(scale, q.shape[0], cols, block_rows)


def linear(x, w, out_dtype, blocks):
    """(x W^T, bound of the error) for FP64 operands.  Bound: a block's 128 exact products are added in at most 128 steps, each off by
    at most 2^-23 of the magnitudes added so far (a sum that is cut instead of rounded); two scales and one addition a block follow;
    then the result's own rounding, half a step of its type (or half the smallest subnormal step of FP16)."""
    y = x @ w.t()
    bound = (x.abs() @ w.abs().t()) * (136 + blocks) * 2.0 ** -23
    own = torch.finfo(out_dtype).eps / 2 * (y.abs() + bound)
    return y, bound + own + (2.0 ** -25 if out_dtype == torch.float16 else 0)


def random_weight(rows, cols, gen, device):
    q = torch.zeros(rows, pitch(cols), dtype=torch.float8_e4m3fn, device=device)
    q[:, :cols] = (torch.randn(rows, cols, generator=gen, device=device) * 90).clamp(-448, 448).to(torch.float8_e4m3fn)
    scale = (torch.rand(-(-rows // BLOCK), -(-cols // BLOCK), generator=gen, device=device) + 0.5) * 1e-3
    return q, scale
