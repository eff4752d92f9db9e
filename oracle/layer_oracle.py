"""Plain numpy definitions of the operators that complete a decoder layer around
the attention path (include/qsvd.h: qsvd_rmsnorm_quantize_act,
qsvd_silu_mul_quantize_act, qsvd_linear_i8).

16-bit rows are held as fp32 arrays whose values are representable in the
16-bit type; ``round16`` rounds to it (nearest, ties to even).
"""
import numpy as np


def round16(v, bf16):
    """fp32 values rounded to fp16 or bf16, as fp32."""
    v = np.asarray(v, dtype=np.float32)
    if not bf16:
        with np.errstate(over="ignore"):
            return v.astype(np.float16).astype(np.float32)
    u = v.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(v), r, v).astype(np.float32)


def quantize_rows(y, bits, clip=1.0):
    """Codes (int8) and scales of fp32 rows, the header's fp32 steps in order:
    tiny rows as zero, rows with a value that is not finite scale NaN."""
    y = np.asarray(y, dtype=np.float32)
    qm = np.float32((1 << (bits - 1)) - 1)
    finite = np.isfinite(y).all(axis=1)
    a = np.float32(clip) * np.abs(np.where(finite[:, None], y, 0)).max(axis=1)
    a = a.astype(np.float32)
    some = (a >= np.float32(2.0 ** -119)) & np.isfinite(a)
    safe = np.where(some, a, np.float32(1))
    inv = np.where(some, (qm / safe).astype(np.float32), np.float32(0))
    s = np.where(some, (safe / qm).astype(np.float32), np.float32(1))
    with np.errstate(invalid="ignore", over="ignore"):
        t = (y * inv[:, None]).astype(np.float32)
    q = np.rint(np.clip(np.where(np.isfinite(t), t, 0), -qm, qm)).astype(np.int8)
    bad = ~finite | ~np.isfinite(a)
    q[bad] = 0
    return q, np.where(bad, np.float32(np.nan), s).astype(np.float32)


def rmsnorm_quantize(x, residual, gamma, eps, bits, clip, bf16):
    """(h, y fp32, codes, scales) of fp32-held 16-bit rows x (+ residual)."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        h = x if residual is None else round16(x + np.asarray(residual, dtype=np.float32), bf16)
        ss = (h.astype(np.float64) ** 2).sum(axis=1, keepdims=True)
        r = (1.0 / np.sqrt(ss / h.shape[1] + np.float64(np.float32(eps)))).astype(np.float32)
        y = ((h * r).astype(np.float32) * np.asarray(gamma, dtype=np.float32)).astype(np.float32)
    q, s = quantize_rows(y, bits, clip)
    return h, y, q, s


def silu_mul(gate, up):
    """gate / (1 + exp(-gate)) * up in fp64."""
    g = np.asarray(gate, dtype=np.float64)
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-g)) * np.asarray(up, dtype=np.float64)


def linear_i8(xq, sx, wq, sw, bias, residual, bf16):
    """The layer's output as fp32-held 16-bit values: an exact integer sum (held
    in fp64, below 2^53), then the header's fp32 steps in order."""
    acc = np.asarray(xq, dtype=np.float64) @ np.asarray(wq, dtype=np.float64).T
    with np.errstate(over="ignore", invalid="ignore"):
        v = acc.astype(np.int64).astype(np.float32)
        v = (v * np.asarray(sx, dtype=np.float32)[:, None]).astype(np.float32)
        v = (v * np.asarray(sw, dtype=np.float32)[None, :]).astype(np.float32)
        if bias is not None:
            v = (v + np.asarray(bias, dtype=np.float32)[None, :]).astype(np.float32)
        if residual is not None:
            v = (v + np.asarray(residual, dtype=np.float32)).astype(np.float32)
        return round16(v, bf16)
