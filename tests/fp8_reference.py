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


def moe(x, router, gate, gate_scale, up, up_scale, down, down_scale, top_k, renormalize):
    """A mixture-of-experts layer in FP64; the choices are those of the FP64 logits (ties: the lowest expert)."""
    hidden, inner = x.shape[1], gate.shape[1]
    logits = x.double() @ router.double().t()
    p = torch.softmax(logits, dim=1)
    out = torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    q, s = quantize(x, 1)
    xv = q * expand(s, x.shape[0], hidden, 1)
    for t in range(x.shape[0]):
        chosen = torch.sort(logits[t], descending=True, stable=True).indices[:top_k].tolist()
        total = sum(p[t, e] for e in chosen) if renormalize else 1.0
        for e in chosen:
            g = xv[t:t + 1] @ values(gate[e], gate_scale[e], hidden, 128).t()
            u = xv[t:t + 1] @ values(up[e], up_scale[e], hidden, 128).t()
            hq, hs = quantize(g / (1 + torch.exp(-g)) * u, 1)
            out[t] += (p[t, e] / total * ((hq * expand(hs, 1, inner, 1)) @ values(down[e], down_scale[e], inner, 128).t()))[0]
    return out


def random_experts(experts, rows, cols, gen, device):
    both = [random_weight(rows, cols, gen, device) for _ in range(experts)]
    return torch.stack([q.view(torch.uint8) for q, _ in both]).view(torch.float8_e4m3fn), torch.stack([s for _, s in both])
