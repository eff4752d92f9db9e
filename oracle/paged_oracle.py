"""Plain numpy definition, in 64 bits, of the operators of a rotary layer with a
paged key/value cache: positions with several axes, the quantizer of a head
vector, pages as a list of places, and causal attention over them."""
import numpy as np

F16, I8, I4 = 0, 1, 2


def round16(v, bf16):
    """Values rounded to nearest even to fp16 or bf16, as float64."""
    v = np.asarray(v, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if not bf16:
            return v.astype(np.float16).astype(np.float64)
        m, e = np.frexp(v)
        e = np.maximum(e, -125)                       # subnormals keep the smallest normal's step
        return np.where(np.isfinite(v), np.ldexp(np.rint(np.ldexp(v, 8 - e)), e - 8), v)


def rope_angles(pos, head_dim, section, theta, restart=False):
    """Angles [M][head_dim / 2] of positions [axes][M], by pair."""
    cols = []
    j = 0
    for axis, n in enumerate(section):
        for i in range(n):
            exponent = -i / n if restart else -2.0 * j / head_dim
            cols.append(np.asarray(pos[axis], np.float64) * float(theta) ** exponent)
            j += 1
    assert j == head_dim // 2
    return np.stack(cols, axis=1)


def rope_axes(x, pos, section, theta, restart=False):
    """Head vectors [M][heads][head_dim] turned at positions [axes][M] (not rounded)."""
    x = np.asarray(x, np.float64)
    half = x.shape[2] // 2
    a = rope_angles(pos, 2 * half, section, theta, restart)[:, None]
    u, v = x[..., :half], x[..., half:]
    return np.concatenate([u * np.cos(a) - v * np.sin(a), v * np.cos(a) + u * np.sin(a)], axis=2)


def quantize_heads(x, bits, clip=1.0):
    """Codes (float64 integers) and fp32 scales of vectors along the last axis,
    whose values are of 16 bits (products with Qm are exact in 64)."""
    x = np.asarray(x, np.float64)
    qm = 2 ** (bits - 1) - 1
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.float32(clip) * np.abs(x).max(-1, keepdims=True).astype(np.float32)
    ok = np.isfinite(x).all(-1, keepdims=True)
    tiny = ok & (a < np.float32(2.0 ** -119))
    safe = np.where(ok & ~tiny, a, np.float32(1)).astype(np.float32)
    codes = np.clip(np.rint(np.where(ok & ~tiny, x, 0) * qm / safe.astype(np.float64)), -qm, qm)
    scale = np.where(ok, np.where(tiny, np.float32(1), safe / np.float32(qm)), np.float32(np.nan)).astype(np.float32)
    return codes, scale[..., 0]


class Batch:
    """A step: which rows belong to which sequence, and where they are."""

    def __init__(self, table, lengths, first, page_size, n_pages):
        self.table, self.lengths, self.first = np.asarray(table), list(lengths), list(first)
        self.page_size, self.n_pages = page_size, n_pages

    def place(self, b, t):
        """(page, row) of token t of sequence b, or None."""
        if t < 0 or t // self.page_size >= self.table.shape[1]:
            return None
        page = int(self.table[b, t // self.page_size])
        return (page, t % self.page_size) if 0 <= page < self.n_pages else None

    def rows(self, n_rows):
        """(row, sequence, position) of the step's rows below n_rows."""
        for b, n in enumerate(self.lengths):
            new = self.first[b + 1] - self.first[b]
            for i in range(new):
                if self.first[b] + i < n_rows:
                    yield self.first[b] + i, b, n - new + i


def attention(q, k, v, batch, n_rows, sm_scale, weight_ulp, v_step=None, sum_ulp=0.0, shift=11,
              sum_least=2.0 ** -28):
    """Outputs [n_rows][Hq][dh] (NaN where no row is) and, beside them, a bound
    of what a kernel may be off before its output's own rounding.

    k, v: stored values [pages][heads][page][dh] in float64.  The bound counts,
    for weights p_t relative to the largest:
      weight_ulp |p_t v_t|     each weight rounded to 16 bits,
      2^-25-shift |v_t|        or, below the normal fp16 numbers, by 2^-25, where the
                               largest weight is 2^shift (16-bit rows),
      2^-23-shift step_t       the same over codes, whose weights take their value's
                               scale: in units of a power of two of at most twice the
                               largest scale (step_t is that scale times |code|), the
                               largest weight at least 2^(shift - 1),
      2 d |p_t v_t|            scores off by d = (dh + 8) 2^-24 sum |q k| sm_scale
                               (fp32 sums in any order, the scale and exponent's
                               roundings), in the weights and in their sum,
      2^-21 |p_t v_t|          the exponentials and fp32 sums of the tiles,
      sum_ulp |output|         where the weights' sum is of weights rounded by as
                               much: sum (p_t + e_t) v_t / sum (p_t + e_t) is off by
                               sum e_t (v_t - output), at most by |e_t v_t| and
                               |e_t output| together,
      sum_least |output|       then also for each key, of a weight of 1: what a weight
                               below the normal fp16 numbers is off by in the sum."""
    n_q = q.shape[1]
    heads, dh = k.shape[1], k.shape[3]
    out = np.full((n_rows, n_q, dh), np.nan)
    bound = np.zeros_like(out)
    for m, b, pos in batch.rows(n_rows):
        places = [p for p in (batch.place(b, t) for t in range(pos + 1)) if p]
        if not places:
            out[m] = 0
            continue
        pages, rows = (np.array(x) for x in zip(*places))
        for h in range(heads):
            g = slice(h * n_q // heads, (h + 1) * n_q // heads)
            kk, vv, qq = k[pages, h, rows], v[pages, h, rows], np.asarray(q[m, g], np.float64)
            with np.errstate(invalid="ignore", over="ignore"):
                s = qq @ kk.T * sm_scale
                p = np.exp(s - s.max(1, keepdims=True))
                total = p.sum(1, keepdims=True)
                out[m, g] = p @ vv / total
                d = (dh + 8) * 2.0 ** -24 * (np.abs(qq) @ np.abs(kk).T * sm_scale).max(1, keepdims=True)
                step = 2.0 ** -25 * np.abs(vv) if v_step is None else 2.0 ** -23 * v_step[pages, h, rows]
                bound[m, g] = ((weight_ulp + 2 * d + 2.0 ** -21) * (p @ np.abs(vv)) + 2.0 ** -shift * step.sum(0)) / total
                if sum_ulp:
                    bound[m, g] += (sum_ulp + sum_least * len(places) / total) * np.abs(out[m, g])
    return out, bound
