"""Definitions in 64 bits that the tests of the 8-bit and experts' layers compare with, and their tolerances."""
import numpy as np
import torch

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
TOP = {E4: 448.0, E5: 57344.0}


def up(a, b):
    return -(-a // b)


def codes(rng, rows, cols, dtype=E4, pitch=None, device="cuda", batch=None, scale=60.0):
    """Random codes whose rows are `pitch` bytes apart (a multiple of 16), NaN between the rows."""
    pitch = pitch or up(cols, 16) * 16
    shape = (rows,) if batch is None else (batch, rows)
    x = rng.normal(0, scale, size=shape + (pitch,)).astype(np.float32)
    x[..., cols:] = np.nan
    t = torch.from_numpy(x).clamp(-TOP[dtype], TOP[dtype]).to(dtype).to(device)
    return t[..., :cols]


def scales(rng, *shape, spread=1.0, device="cuda"):
    return torch.from_numpy(np.exp(rng.normal(0, spread, size=shape)).astype(np.float32) / 60.0).to(device)


def product(a, sa, b, sb, bias=None, relu=False):
    """(y, sum of magnitudes) of the scaled product in 64 bits, on the device of the operands."""
    a, b, sa, sb = a.double(), b.double(), sa.double(), sb.double()
    k, n = a.shape[1], b.shape[0]
    wa = a * sa.repeat_interleave(128, 1)[:, :k]
    wb = b * sb.repeat_interleave(128, 1)[:, :k].repeat_interleave(128, 0)[:n]
    y, size = wa @ wb.t(), wa.abs() @ wb.abs().t()
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return (torch.where(y < 0, torch.zeros_like(y), y) if relu else y), size


def product_tolerance(y, size, k, out_dtype):
    """Products of codes are exact in fp32 (8 significant bits).  An addition may be off by 2^-23 of the sum of the magnitudes (the
    tensor cores cut off where fp32 would round): at most 128 in a block, then one fma a block with a scale rounded once, up to 16
    parts of a cut reduction axis, the bias.  Then half a step of the output's type."""
    half = torch.finfo(out_dtype).eps / 2
    least = torch.finfo(out_dtype).smallest_normal * torch.finfo(out_dtype).eps      # subnormal results
    return size * ((min(k, 128) + up(k, 128) * 2 + 18) * 2.0 ** -23) * (1 + half) + y.abs() * half + least


def check_product(got, want, size, k):
    off = (got.double() - want).abs()
    tol = product_tolerance(want, size, k, got.dtype)
    assert not torch.isnan(off).any() and (off <= tol).all(), "off by %g, %g allowed" % (float((off - tol).max()), float(tol[(off - tol) == (off - tol).max()].max()))


def sort_choices(ids, experts):
    """offsets, order, slot of choices [T][k] (-1: none), by the definition."""
    T, k = ids.shape
    runs = [[(t, j) for t in range(T) for j in range(k) if ids[t, j] == e] for e in range(experts)]
    offsets = np.cumsum([0] + [len(r) for r in runs]).astype(np.int32)
    order, slot = np.full(T * k, -1, np.int32), np.full((T, k), -1, np.int32)
    at = 0
    for r in runs:
        for t, j in r:
            order[at], slot[t, j] = t, at
            at += 1
    return offsets, order, slot
