"""4-bit weights with group scales: rounding and the values that codes stand for, in float64.

weight[k] = scale[k // group] * (code[k] - zero[k // group]); codes 0..15, two per byte along K (the lower k in the low bits)."""
from __future__ import annotations

import numpy as np


def bf16(v):
    """float64 -> nearest bfloat16 (ties to even), as float64.  A bfloat16 has 8 significant bits."""
    m, e = np.frexp(v)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def quantize(w, group, zeros):
    """w [..., K] float64 -> codes [..., K] int, scales [..., groups] float64, zeros [..., groups] int."""
    K = w.shape[-1]
    groups = (K + group - 1) // group
    codes = np.empty(w.shape, dtype=np.int64)
    scales = np.empty(w.shape[:-1] + (groups,))
    zps = np.full(scales.shape, 8, dtype=np.int64)
    for g in range(groups):
        part = w[..., g * group:(g + 1) * group]
        lo, hi = np.minimum(part.min(axis=-1), 0.0), np.maximum(part.max(axis=-1), 0.0)
        s = bf16((hi - lo) / 15.0 if zeros else np.maximum(hi, -lo) / 7.0)
        safe = np.where(s > 0, s, 1.0)
        if zeros:
            zps[..., g] = np.where(s > 0, np.clip(np.rint(-lo / safe), 0, 15), 8)
        q = np.rint(np.where(s[..., None] > 0, part / safe[..., None], 0.0)) + zps[..., g, None]
        codes[..., g * group:(g + 1) * group] = np.clip(q, 0, 15)
        scales[..., g] = s
    return codes, scales, zps


def pack_bytes(codes):
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack_bytes(packed):
    out = np.empty(packed.shape[:-1] + (2 * packed.shape[-1],), dtype=np.int64)
    out[..., 0::2], out[..., 1::2] = packed & 15, packed >> 4
    return out


def values(codes, scales, zeros, group):
    at = np.arange(codes.shape[-1]) // group
    return (codes - zeros[..., at]) * scales[..., at]
