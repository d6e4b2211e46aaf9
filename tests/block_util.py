"""Plain 64-bit versions of the operators of include/quartet_block.h, operand helpers and the units their tolerances are counted in."""
import math

import torch

from paper_2505_14669_amd import binding as q
from paper_2505_14669_amd import block as b

DEV = "cuda:0"
U32, U16 = 2.0 ** -24, 2.0 ** -8       # half a step of fp32 and bf16, relative to the value
BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: U16, F32: U32}
GUARD = -77.0                          # a value no result takes, around every output


def code(t):
    return b.QUARTET_DTYPE_F32 if t is None or t.dtype == F32 else b.QUARTET_DTYPE_BF16


def rng(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def ld_of(n, extra=0):
    return (n + 7) // 8 * 8 + extra


def matrix(g, rows, n, dtype, scale=1.0, extra=0):
    """[rows, ld] of which the first n columns are the matrix; the others hold NaN: whatever reads them shows"""
    t = torch.full((rows, ld_of(n, extra)), float("nan"), dtype=dtype, device=DEV)
    t[:, :n] = (torch.randn((rows, n), generator=g, device=DEV) * scale).to(dtype)
    return t


def output(rows, n, dtype, extra=0):
    """[rows + 2, ld] full of GUARD, and the rows that are the output"""
    whole = torch.full((rows + 2, ld_of(n, extra)), GUARD, dtype=dtype, device=DEV)
    return whole, whole[1:rows + 1]


def guarded(whole, n):
    """nothing outside the output was written"""
    return bool((whole[0] == GUARD).all() and (whole[-1] == GUARD).all() and (whole[:, n:] == GUARD).all())


def assert_within(got, want, bound, what=""):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), float((got - want).abs()[bad].max()), got[bad][:4].tolist(), want[bad][:4].tolist())


def act(z, kind):
    """value and slope in z's type"""
    if kind == "relu":
        return z.clamp_min(0), (z > 0).to(z.dtype)
    if kind == "gelu":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z.clone(), torch.ones_like(z)


def quantized(g, rows, k, scale=1.0):
    """(codes, scales, values in fp64) of a random MXFP4 operand, made and decoded by the library's own calls"""
    x = (torch.randn((rows, k), generator=g, device=DEV) * scale).to(BF16)
    codes = torch.empty(max(16, rows * k // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty(max(16, q.quartet_scale_bytes(rows, k)), dtype=torch.uint8, device=DEV)
    values = torch.empty((rows, k), dtype=F32, device=DEV)
    if rows and k:
        q.check(q.quartet_quant_fwd(x, rows, k, k, 0, codes, scales, None))
        q.check(q.quartet_mxfp4_dequant(codes, scales, rows, k, values))
    return codes, scales, values.double()


def scale_bytes_of(tiled, rows, groups):
    """the scale bytes [rows, groups] of the tiled buffer, by the header's formula"""
    r, g = torch.arange(rows, device=DEV)[:, None], torch.arange(groups, device=DEV)[None, :]
    at = ((r // 32) * ((groups + 7) // 8) + g // 8) * 256 + ((g % 2) * 32 + r % 32) * 4 + (g % 8) // 2
    return tiled.long()[at]
