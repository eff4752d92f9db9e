"""Rotary positions with several axes and the paged key/value cache, through the
C ABI against the oracle in 64 bits.

Places of a pool that no row was written to hold NaN (rows, scales), so that
whatever a kernel reads past a sequence's end shows."""
import numpy as np
import pytest

import gpu_harness as H
from oracle import paged_oracle as P
from paper_2510_16292_amd import binding as B
from paper_2510_16292_amd import prep
from workloads import configs, gen

pytestmark = pytest.mark.gpu

F16, I8, I4 = B.QSVD_CACHE_F16, B.QSVD_CACHE_I8, B.QSVD_CACHE_I4
HALF, BF = B.QSVD_F16, B.QSVD_BF16
FMT = {F16: "f16", I8: "i8", I4: "i4"}
HALF_STEP = {HALF: 2.0 ** -11, BF: 2.0 ** -8}       # of a rounding, relative to the value
LEAST = {HALF: 2.0 ** -25, BF: 2.0 ** -134}         # and below the normal numbers


def dtype_of(dt):
    t = H.torch()
    return t.bfloat16 if dt == BF else t.float16


def to16(x, dt):
    """float64 numpy values, rounded to dt, as a device tensor."""
    t = H.torch()
    return t.from_numpy(np.ascontiguousarray(P.round16(x, dt == BF))).to(dtype_of(dt)).cuda()


def values(t):
    H.torch().cuda.synchronize()
    return t.detach().double().cpu().numpy()


def bits(t):
    return H.host(t.contiguous().view(H.torch().uint8))


def assert_close(got, want, bound, what=""):
    """|got - want| <= bound, NaN and infinities alike."""
    bad = ~((np.abs(got - want) <= bound) | (got == want) | (np.isnan(got) & np.isnan(want)))
    if bad.any():
        i = tuple(x[0] for x in np.nonzero(bad))
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} off, first at {i}: {got[i]} for {want[i]}, bound "
                             f"{np.broadcast_to(bound, got.shape)[i]}")


# ---------------------------------------------------------------- rotary positions

def turn(x, pos, section, theta, dt, order=B.QSVD_ROPE_RUNNING, k=None, inplace=False, pad=0):
    """x [M][heads][dh] float64 (values of dt); pos int32 [axes][M]."""
    t = H.torch()

    def rows(a):
        M, h, dh = a.shape
        buf = t.full((M, h * dh + pad), 7.0, dtype=dtype_of(dt), device="cuda")
        buf[:, :h * dh] = to16(a, dt).view(M, h * dh)
        return buf

    M, hq, dh = x.shape
    q = rows(x)
    qo = q if inplace else t.full_like(q, -3.0)
    kk = None if k is None else rows(k)
    ko = kk if inplace or k is None else t.full_like(kk, -3.0)
    ldpos = M + 3
    p = t.full((len(section), ldpos), 1 << 20, dtype=t.int32, device="cuda")
    p[:, :M] = H.dev(np.asarray(pos, np.int32))
    hk = 0 if k is None else k.shape[1]
    B.check(B.qsvd_rope_axes(B.rope(dh, section, theta, order), B.ptr(p), ldpos, M, dt, B.ptr(q), hq * dh + pad, hq,
                             B.ptr(qo), hq * dh + pad, B.ptr(kk), hk * dh + pad, hk, B.ptr(ko), hk * dh + pad,
                             B.stream_handle()))
    if pad:
        assert (values(qo)[:, hq * dh:] == (7.0 if inplace else -3.0)).all(), "elements behind a row were written"
    out = values(qo)[:, :hq * dh].reshape(x.shape)
    return out if k is None else (out, values(ko)[:, :hk * dh].reshape(k.shape))


def rope_bound(x, want, dt):
    """One rounding, and sines and cosines off by 2^-19 (the hardware's by about
    2^-20, the reduced angle's rounding to fp32 by 2 pi 2^-25)."""
    half = x.shape[2] // 2
    a, b = np.abs(x[..., :half]), np.abs(x[..., half:])
    return HALF_STEP[dt] * np.abs(want) + LEAST[dt] + 2.0 ** -19 * np.concatenate([a + b, a + b], 2)


@pytest.mark.parametrize("dt", [HALF, BF], ids=["f16", "bf16"])
@pytest.mark.parametrize("M,hq,hk,dh,section", [
    (1, 4, 4, 64, (8, 12, 12)), (1, 28, 4, 128, (16, 24, 24)), (5, 1, 0, 16, (8,)), (3, 3, 2, 80, (10, 30)),
    (67, 40, 40, 128, (64,)), (130, 12, 1, 256, (1, 0, 63, 64)), (1000, 28, 4, 128, (16, 24, 24)), (9, 200, 56, 64, (32,)),
])
@pytest.mark.parametrize("inplace", [False, True])
def test_rope(dt, M, hq, hk, dh, section, inplace):
    rng = np.random.default_rng(M + dh)
    x = P.round16(rng.standard_normal((M, hq, dh)) * 3, dt == BF)
    k = P.round16(rng.standard_normal((M, hk, dh)), dt == BF) if hk else None
    pos = rng.integers(-100, 40000, (len(section), M))
    got = turn(x, pos, section, 1e6, dt, k=k, inplace=inplace, pad=24 if M == 5 or M == 130 else 0)
    for a, g in ((x, got if k is None else got[0]), (k, None if k is None else got[1])):
        if a is not None:
            want = P.rope_axes(a, pos, section, 1e6)
            assert_close(g, want, rope_bound(a, want, dt))


def test_rope_restarting_frequencies_and_far_positions():
    rng = np.random.default_rng(7)
    x = P.round16(rng.standard_normal((64, 2, 128)), False)
    pos = rng.integers(-2 ** 31, 2 ** 31, (2, 64))
    pos[:, 0], pos[:, 1] = 2 ** 31 - 1, -2 ** 31
    # the oracle's cosine of an angle of 2^31 in fp64 is off by 2^-22 itself
    for order in (B.QSVD_ROPE_RUNNING, B.QSVD_ROPE_RESTART):
        want = P.rope_axes(x, pos, (32, 32), 1e4, order == B.QSVD_ROPE_RESTART)
        assert_close(turn(x, pos, (32, 32), 1e4, HALF, order), want, rope_bound(x, want, HALF) + 2.0 ** -19, order)


def test_rope_of_one_position_is_the_one_axis_embedding():
    rng = np.random.default_rng(8)
    x = P.round16(rng.standard_normal((33, 4, 64)), False)
    p = rng.integers(0, 9000, (1, 33))
    a = turn(x, np.tile(p, (3, 1)), (8, 12, 12), 1e4, HALF)
    assert np.array_equal(a, turn(x, p, (32,), 1e4, HALF))


@pytest.mark.parametrize("dt", [HALF, BF], ids=["f16", "bf16"])
def test_rope_at_negated_positions_is_the_gradient(dt):
    """The transpose: y . turn(x) = turn back(y) . x, each side off by its own bound's dot product."""
    rng = np.random.default_rng(9)
    x, y = (P.round16(rng.standard_normal((40, 3, 128)), dt == BF) for _ in range(2))
    pos = rng.integers(0, 30000, (3, 40))
    there, back = turn(x, pos, (16, 24, 24), 1e6, dt), turn(y, -pos, (16, 24, 24), 1e6, dt)
    off = (rope_bound(x, there, dt) * np.abs(y) + rope_bound(y, back, dt) * np.abs(x)).sum(2)
    assert (np.abs((there * y - back * x).sum(2)) <= 1.01 * off).all()


def test_rope_keeps_nan_and_infinity_in_their_pairs():
    x = np.ones((2, 2, 64))
    x[0, 0, 3], x[1, 1, 40] = np.nan, np.inf
    got = turn(x, np.full((1, 2), 5), (32,), 1e4, HALF)
    bad = np.zeros(x.shape, bool)
    bad[0, 0, [3, 35]] = bad[1, 1, [8, 40]] = True
    assert np.array_equal(~np.isfinite(got), bad)


# ---------------------------------------------------------------- pages

class Pool:
    """Pages on the device with NaN (or codes 77) in every place, and a batch."""

    def __init__(self, fmt, dt, heads, dh, page, lens, news, seed=0, spare=2, order=None, poison=True, max_len=None,
                 max_new=None, n_rows=None):
        t = H.torch()
        self.fmt, self.dt, self.heads, self.dh, self.page, self.lens, self.news = fmt, dt, heads, dh, page, list(lens), list(news)
        cols = [-(-max(n, 0) // page) for n in lens]
        n_pages = sum(cols) + spare
        ids = np.random.default_rng(seed).permutation(n_pages)
        table = np.full((len(lens), max(max(cols), 1)), -1, np.int32)
        at = 0
        for b, c in enumerate(cols):
            table[b, :c] = ids[at:at + c]
            at += c
        self.table, self.n_pages = table, n_pages
        self.d = B.DevicePages(fmt, dt, n_pages, page, heads, dh)
        if poison:
            for x in (self.d.k, self.d.v):
                x.fill_(float("nan") if fmt == F16 else 77)
            for x in (self.d.k_scale, self.d.v_scale):
                if x is not None:
                    x.fill_(float("nan"))
        self.rebatch(lens, news, max_len, max_new, n_rows)

    def rebatch(self, lens, news, max_len=None, max_new=None, n_rows=None):
        self.lens, self.news = list(lens), list(news)
        self.batch = B.DevicePageBatch(self.table, lens, news, max_len=max_len, max_new=max_new, n_rows=n_rows)
        first = [sum(news[:b]) for b in range(len(news) + 1)]
        self.o = P.Batch(self.table, lens, first, self.page, self.n_pages)
        self.n_rows = self.batch.n_rows

    def append(self, k, v, clip=1.0, stream=None):
        w = k.shape[1]
        B.check(B.qsvd_paged_append(self.d.c, self.batch.c, B.ptr(k), w, B.ptr(v), v.shape[1], clip,
                                    B.stream_handle(stream)))

    def read(self, k, v):
        B.check(B.qsvd_paged_read(self.d.c, self.batch.c, B.ptr(k), k.shape[1], B.ptr(v), v.shape[1], B.stream_handle()))

    def stored(self):
        """The pool's values and, for codes, their unit (the scale), float64 [pages][heads][page][dh]."""
        out = []
        for x, s in ((self.d.k, self.d.k_scale), (self.d.v, self.d.v_scale)):
            if self.fmt == F16:
                out.append((values(x), None))
                continue
            c = H.host(x).astype(np.int8)
            if self.fmt == I4:
                u = c.view(np.uint8)
                c = np.stack([(u << 4).view(np.int8) >> 4, c >> 4], -1).reshape(*c.shape[:-1], -1)
            s = H.host(s).astype(np.float64)[..., None]
            out.append((c.astype(np.float64) * s, c))
        return out

    def fill(self, seed=1, spread=0.5, outlier=4.0):
        """Rows for every token of every sequence, through append."""
        rng = np.random.default_rng(seed)
        lens, news = self.lens, self.news
        n = sum(max(x, 0) for x in lens)
        self.rebatch(lens, [max(x, 0) for x in lens])
        rows = rng.standard_normal((2, n, self.heads, self.dh)) * np.exp(spread * rng.standard_normal((2, n, self.heads, 1)))
        rows[..., ::17] *= outlier
        if n:
            self.append(*(to16(r, self.dt).view(n, -1) for r in rows))
        self.rebatch(lens, news)
        return self

    def attend(self, q, n_q, sm_scale=0.0, out=None, ws=None, stream=None):
        """q: device [rows][n_q * dh (+ pad)]."""
        t = H.torch()
        size = B.qsvd_paged_attention_workspace_size(self.d.c, self.batch.c, n_q)
        if ws is None:
            # (every byte of the workspace a NaN)
            ws = t.full((max(size, 1),), 255, dtype=t.uint8, device="cuda")
        if out is None:
            out = t.full_like(q, 3.0)
        B.check(B.qsvd_paged_attention(self.d.c, self.batch.c, B.ptr(q), q.shape[1], n_q, sm_scale, B.ptr(out),
                                       out.shape[1], B.ptr(ws), size, B.stream_handle(stream)))
        return out

    def sum_step(self, n_q):
        """The rounding of the weights that are summed: none for few rows, whose exponentials are summed as they
        are, nor for bf16 outputs of codes; else that of the weights themselves."""
        if self.batch.c.max_new * (n_q // self.heads) <= 32 or (self.fmt != F16 and self.dt == BF):
            return 0.0
        return HALF_STEP[BF] if self.fmt == F16 and self.dt == BF else HALF_STEP[HALF]

    def want(self, q, n_q, sm_scale=None):
        """Oracle output [rows][n_q * dh] (NaN: no row) and bound, its rounding included."""
        (k, _), (v, codes) = self.stored()
        step = None if codes is None else np.abs(codes) * np.nanmax(np.where(codes != 77, H.host(self.d.v_scale)[..., None], 0))
        qv = values(q)[:, :n_q * self.dh].reshape(-1, n_q, self.dh)
        scale = self.dh ** -0.5 if sm_scale is None else sm_scale
        # weights are rounded to bf16 where the pages hold bf16 rows, else to fp16
        u = HALF_STEP[BF] if self.fmt == F16 and self.dt == BF else HALF_STEP[HALF]
        out, bound = P.attention(qv, k, v, self.o, qv.shape[0], scale, u, step, self.sum_step(n_q))
        bound = bound + HALF_STEP[self.dt] * (np.abs(out) + bound) + LEAST[self.dt]
        n = qv.shape[0]
        return out.reshape(n, -1), bound.reshape(n, -1)

    def check(self, n_q, seed=2, amplitude=1.0, sm_scale=None):
        rng = np.random.default_rng(seed)
        q = to16(amplitude * rng.standard_normal((self.n_rows, n_q * self.dh)), self.dt)
        got = self.attend(q, n_q, 0.0 if sm_scale is None else sm_scale)
        want, bound = self.want(q, n_q, sm_scale)
        got = values(got)
        gone = np.isnan(want).all(1)
        assert (got[gone] == 3.0).all(), "a row behind the last sequence was written"
        assert_close(got[~gone], want[~gone], bound[~gone], f"{FMT[self.fmt]} {self.lens} {self.news}")
        return got


    def check_large(self, n_q, seed=2):
        """check() with the oracle's arithmetic in torch's 64 bits on the device, a sequence and head at a time
        (every page of the sequences has to be there)."""
        t = H.torch()
        rng = t.Generator(device="cuda").manual_seed(seed)
        q = t.randn((self.n_rows, n_q * self.dh), generator=rng, device="cuda").to(dtype_of(self.dt))
        got = self.attend(q, n_q).double().view(-1, n_q, self.dh)
        q = q.double().view(-1, n_q, self.dh)
        stored = [t.from_numpy(np.nan_to_num(x)).cuda() for x, _ in self.stored()]
        unit = 0.0 if self.fmt == F16 else float(np.nanmax(H.host(self.d.v_scale)))
        table = t.from_numpy(self.table.astype(np.int64)).cuda()
        u = HALF_STEP[BF] if self.fmt == F16 and self.dt == BF else HALF_STEP[HALF]
        group, worst = n_q // self.heads, 0.0
        for b, (n, new) in enumerate(zip(self.lens, self.news)):
            if new == 0:
                continue
            pages, rows = table[b, :-(-n // self.page)], slice(self.o.first[b], self.o.first[b] + new)
            hidden = t.ones((new, n), dtype=t.bool, device="cuda").triu(n - new + 1)
            for h in range(self.heads):
                k, v = (x[pages, h].reshape(-1, self.dh)[:n] for x in stored)
                for g in range(h * group, (h + 1) * group):
                    x = (q[rows, g] @ k.t() * self.dh ** -0.5).masked_fill(hidden, -np.inf)
                    p = t.softmax(x, 1)
                    d = (self.dh + 8) * 2.0 ** -24 * (q[rows, g].abs() @ k.abs().t()).max(1, keepdim=True).values * self.dh ** -0.5
                    want, a = p @ v, p @ v.abs()
                    top = p.max(1, keepdim=True).values
                    steps = v.abs().sum(0) if self.fmt == F16 else unit * 127 * n
                    bound = (u + 2 * d + 2.0 ** -21) * a + 2.0 ** -25 * top * steps + self.sum_step(n_q) * want.abs()
                    bound = bound + HALF_STEP[self.dt] * (want.abs() + bound) + LEAST[self.dt]
                    worst = max(worst, float(((got[rows, g] - want).abs() / bound).max()))
        assert worst <= 1, worst


FORMS = [(f, d) for f in (F16, I8, I4) for d in (HALF, BF)]
FORM_IDS = [f"{FMT[f]}-{'bf16' if d == BF else 'f16'}" for f, d in FORMS]


@pytest.mark.parametrize("fmt,dt", FORMS, ids=FORM_IDS)
@pytest.mark.parametrize("heads,dh,page,lens,news", [
    (4, 64, 16, [1], [1]), (2, 128, 16, [17, 0, 33, 5], [17, 0, 2, 5]), (3, 64, 64, [64, 65, 130], [64, 1, 66]),
    (4, 128, 256, [700, 3], [700, 1]), (1, 128, 1024, [1500], [1400]), (2, 64, 32, [40] * 70, [1] * 70),
])
def test_append_and_read(fmt, dt, heads, dh, page, lens, news):
    """Every code, scale and row bit for bit; other places as they were; rows behind the last left alone."""
    t = H.torch()
    rng = np.random.default_rng(len(lens) + dh)
    p = Pool(fmt, dt, heads, dh, page, lens, news)
    n, w = sum(news), heads * dh
    k, v = (P.round16(rng.standard_normal((n, heads, dh)) * np.exp(rng.standard_normal((n, heads, 1))), dt == BF)
            for _ in range(2))
    k[0, 0] = 0                                       # a zero vector
    k[-1, 0, :] = np.arange(dh) % 15 - 7.0            # quotients half way between two codes: 7 c / 7 and 127 c / 14 ..
    k[-1, 0, 0] = 14.0
    p.rebatch(lens, news, n_rows=n + 3)
    buf = [t.full((n + 3, w + 8), 5.0, dtype=dtype_of(dt), device="cuda") for _ in range(2)]
    for b, x in zip(buf, (k, v)):
        b[:n, :w] = to16(x, dt).view(n, w)
    p.append(*buf)
    back = [t.full((n + 3, w + 24), 6.0, dtype=dtype_of(dt), device="cuda") for _ in range(2)]
    p.read(*back)
    for x, pool, scales, got in ((k, p.d.k, p.d.k_scale, back[0]), (v, p.d.v, p.d.v_scale, back[1])):
        want_back = np.full((n + 3, w + 24), 6.0)
        if fmt == F16:
            want = np.full((p.n_pages, heads, page, dh), np.nan)
            for m, b, pos in p.o.rows(n):
                pg, r = p.o.place(b, pos)
                want[pg, :, r] = x[m]
            assert np.array_equal(values(pool), want, equal_nan=True)
            want_back[:n, :w] = x.reshape(n, w)
        else:
            codes, s = P.quantize_heads(x, 8 if fmt == I8 else 4)
            want = np.full((p.n_pages, heads, page, dh), 77, np.int8)
            if fmt == I4:
                want = np.full((p.n_pages, heads, page, dh // 2), 77, np.uint8)
                c = codes.astype(np.int64) & 15
                stored = (c[..., ::2] | c[..., 1::2] << 4).astype(np.uint8)
            else:
                stored = codes.astype(np.int8)
            want_s = np.full((p.n_pages, heads, page), np.nan, np.float32)
            for m, b, pos in p.o.rows(n):
                pg, r = p.o.place(b, pos)
                want[pg, :, r], want_s[pg, :, r] = stored[m], s[m]
            assert np.array_equal(H.host(pool), want)
            assert np.array_equal(H.host(scales), want_s, equal_nan=True)
            with np.errstate(over="ignore"):
                prod = (codes.astype(np.float32) * s[..., None]).astype(np.float64)
            want_back[:n, :w] = P.round16(prod, dt == BF).reshape(n, w)
        assert np.array_equal(values(got), want_back)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("batch", [65, 129, 300, 2100, 65536])
def test_append_and_read_large_batches(batch, dh):
    """Each row to its own sequence: every row of the pool that has a place, and no other, is the row's."""
    t = H.torch()
    rng = np.random.default_rng(batch)
    news = rng.integers(0, 4, batch)
    news[[0, -1]] = 0, 3
    news[batch // 2:batch // 2 + 40] = 0
    lens = news + rng.integers(0, 9, batch)
    n = int(news.sum())
    table = rng.permutation(batch).astype(np.int32)[:, None]
    p = B.DevicePages(F16, HALF, batch, 16, 1, dh)
    d = B.DevicePageBatch(table, lens.tolist(), news.tolist(), n_rows=n + 5)
    m = np.arange(n + 5)
    rows = t.from_numpy(np.tile((m % 2039)[:, None], (1, dh))).half().cuda()
    rows[:, 1] = t.from_numpy(m // 2039).half().cuda()
    back = [t.full((n + 5, dh), -1.0, dtype=t.float16, device="cuda") for _ in range(2)]
    B.check(B.qsvd_paged_append(p.c, d.c, B.ptr(rows), dh, B.ptr(rows), dh, 1.0, B.stream_handle()))
    B.check(B.qsvd_paged_read(p.c, d.c, B.ptr(back[0]), dh, B.ptr(back[1]), dh, B.stream_handle()))
    seq = np.repeat(np.arange(batch), news)
    pos = (lens - np.cumsum(news))[seq] + m[:n]
    want = t.zeros((batch, 1, 16, dh), dtype=t.float16, device="cuda")
    want[t.from_numpy(table[seq, 0]).long().cuda(), 0, t.from_numpy(pos).cuda()] = rows[:n]
    for pool, out in ((p.k, back[0]), (p.v, back[1])):
        assert t.equal(pool, want) and t.equal(out[:n], rows[:n]) and bool((out[n:] == -1).all())


@pytest.mark.parametrize("fmt", [I8, I4], ids=["i8", "i4"])
@pytest.mark.parametrize("dt", [HALF, BF], ids=["f16", "bf16"])
@pytest.mark.parametrize("clip", [1.0, 0.7])
def test_append_codes_next_to_borders(fmt, dt, clip):
    """Vectors of small integers (many quotients half way between codes), the
    type's largest and smallest values, and vectors that are not finite."""
    rng = np.random.default_rng(11)
    n, heads, dh = 64, 2, 64
    x = rng.integers(-127, 128, (n, heads, dh)).astype(np.float64)
    top = 65504.0 if dt == HALF else 2.0 ** 127 * (2 - 2.0 ** -7)
    tiny = 2.0 ** -24 if dt == HALF else 2.0 ** -133
    x[0], x[1], x[2] = x[0] / 127 * top, tiny * np.sign(x[1]), 0
    x[3, 0, 5], x[4, 1, 6], x[5, 0, 0] = np.inf, np.nan, -np.inf
    x[6] = 2.0 ** -118 * np.sign(x[6]) if dt == BF else x[6]
    x[7] = 2.0 ** -120 * np.sign(x[7]) if dt == BF else x[7]
    x = P.round16(x, dt == BF)
    p = Pool(fmt, dt, heads, dh, 16, [n], [n])
    d = to16(x, dt).view(n, -1)
    p.append(d, d, clip)
    codes, s = P.quantize_heads(x, 8 if fmt == I8 else 4, clip)
    pages, rows = p.table[0][np.arange(n) // 16], np.arange(n) % 16
    (_, got), _ = p.stored()
    assert np.array_equal(got[pages, :, rows], codes)
    assert np.array_equal(H.host(p.d.k_scale)[pages, :, rows], s, equal_nan=True)


@pytest.mark.parametrize("fmt", [F16, I8, I4], ids=["f16", "i8", "i4"])
def test_rows_without_a_place(fmt):
    """Pages that do not exist, columns past the table and negative positions:
    not written, zeros when read; the other rows as ever."""
    t = H.torch()
    p = Pool(fmt, HALF, 2, 64, 16, [70, 20, 3], [70, 20, 5])
    p.table[0, 1], p.table[0, 3], p.table[1, 0] = p.n_pages, -5, 2 ** 31 - 1
    p.table = np.ascontiguousarray(p.table[:, :4])             # sequence 0 has tokens past the table
    p.rebatch([70, 20, 3], [70, 20, 5])
    x = P.round16(np.random.default_rng(0).standard_normal((95, 2, 64)), False)
    d = to16(x, HALF).view(95, -1)
    before = [bits(z) for z in (p.d.k, p.d.v)]
    p.append(d, d)
    back = [t.full_like(d, 9.0) for _ in range(2)]
    p.read(*back)
    got = values(back[0]).reshape(95, 2, 64)
    touched = np.zeros((p.n_pages, p.page), bool)
    for m, b, pos in p.o.rows(95):
        at = p.o.place(b, pos)
        if at is None:
            assert not got[m].any(), m
        else:
            touched[at] = True
            assert got[m].any() and np.abs(got[m] - x[m]).max() <= {F16: 0, I8: 0.02, I4: 0.4}[fmt], m
    assert touched.sum() == 16 * 2 + 4 + 3
    for z, b in zip((p.d.k, p.d.v), before):
        changed = (bits(z) != b).reshape(p.n_pages, 2, p.page, -1).any((1, 3))
        assert not (changed & ~touched).any()
    assert np.array_equal(bits(back[0]), bits(back[1]))


# ---------------------------------------------------------------- attention

HEADS = [(4, 4, 64), (28, 4, 128), (8, 1, 64), (5, 5, 128), (64, 2, 128)]


@pytest.mark.parametrize("fmt,dt", FORMS, ids=FORM_IDS)
@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_attention_one_token(fmt, dt, hq, hkv, dh):
    """Decode steps: lengths around the sizes of pages and tiles, one of them without a token."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 129, 300, 0, 777]
    Pool(fmt, dt, hkv, dh, 16, lens, [1 if n else 0 for n in lens]).fill().check(hq)


@pytest.mark.parametrize("fmt,dt", FORMS, ids=FORM_IDS)
@pytest.mark.parametrize("hq,hkv,dh,page", [(4, 4, 64, 32), (28, 4, 128, 16), (8, 1, 64, 256), (32, 2, 128, 64)])
def test_attention_few_tokens(fmt, dt, hq, hkv, dh, page):
    """Two to ten new tokens each, also more than the sequence has."""
    lens, news = [40, 5, 9, 130, 64, 2], [2, 5, 3, 10, 1, 4]
    Pool(fmt, dt, hkv, dh, page, lens, news).fill().check(hq)


@pytest.mark.parametrize("fmt,dt", FORMS, ids=FORM_IDS)
@pytest.mark.parametrize("hq,hkv,dh,page,lens,news", [
    (4, 4, 64, 16, [200], [200]), (4, 4, 64, 64, [129, 257, 64], [129, 64, 64]), (28, 4, 128, 64, [150, 99], [70, 99]),
    (5, 5, 128, 16, [300, 1, 0, 45], [150, 1, 0, 45]), (8, 1, 64, 32, [513], [65]), (3, 3, 128, 1024, [140], [100]),
])
def test_attention_chunks(fmt, dt, hq, hkv, dh, page, lens, news):
    Pool(fmt, dt, hkv, dh, page, lens, news).fill().check(hq)


@pytest.mark.parametrize("fmt,dt", FORMS, ids=FORM_IDS)
def test_attention_mixed_batch(fmt, dt):
    """Chunks, single tokens and sequences without one together."""
    lens = [400, 1, 333, 90, 0, 64, 700, 17]
    news = [1, 1, 150, 0, 0, 64, 1, 3]
    Pool(fmt, dt, 2, 128, 32, lens, news).fill().check(8)


@pytest.mark.parametrize("seed", range(60))
def test_attention_drawn(seed):
    """Formats, heads, pages, lengths and bounds drawn at random, some pages not there."""
    rng = np.random.default_rng(seed)
    fmt, dt = FORMS[seed % len(FORMS)]
    heads, dh, page = int(rng.choice([1, 2, 3, 4, 8])), int(rng.choice([64, 128])), int(rng.choice([16, 32, 64, 1024]))
    group = min(int(rng.choice([1, 2, 3, 5, 7, 8, 16, 32])), 32 // heads)
    batch = int(rng.choice([1, 2, 3, 5, 9, 20]))
    lens = [int(x) for x in rng.integers(0, int(rng.choice([4, 40, 130, 600 if batch < 4 else 200])) + 1, batch)]
    most = int(rng.choice([1, 6, 100, 1000]))
    news = [min(n, int(rng.integers(0, most + 1)) if seed % 3 else most) for n in lens]
    lens, news = lens + [70], news + [1]
    p = Pool(fmt, dt, heads, dh, page, lens, news, seed=seed).fill(seed)
    if seed % 4 == 0:
        gone = rng.random(p.table.shape) < 0.2
        p.table = np.where(gone, rng.choice([-1, p.n_pages, 2 ** 31 - 1, -2 ** 31], size=p.table.shape), p.table).astype(np.int32)
    above = [int(x) for x in rng.integers(0, 40, 3)] if seed % 2 else [0, 0, 0]
    p.rebatch(lens, news, max(lens) + 100 * above[0], max(news) + above[1], sum(news) + above[2])
    p.check(heads * group, seed=seed, amplitude=float(rng.choice([1, 1, 0.01, 8])))


@pytest.mark.parametrize("fmt", [F16, I8, I4], ids=["f16", "i8", "i4"])
@pytest.mark.parametrize("n,new", [(3000, 1), (9000, 1), (4100, 2), (2900, 130)])
def test_attention_long(fmt, n, new):
    """One long sequence: the keys are shared out over many workgroups."""
    Pool(fmt, BF, 1, 128, 64, [n], [new]).fill().check(6, amplitude=2.0)


@pytest.mark.parametrize("fmt", [F16, I8], ids=["f16", "i8"])
def test_attention_lengths_that_differ_much(fmt):
    lens = [5000, 3, 64, 1200, 31, 0, 257]
    Pool(fmt, HALF, 2, 64, 16, lens, [1, 1, 1, 1, 1, 0, 1]).fill().check(2)


@pytest.mark.parametrize("fmt,dt", FORMS, ids=FORM_IDS)
@pytest.mark.parametrize("amplitude,scale", [(30.0, None), (1e-3, None), (1.0, 2.0), (4000.0, 1e-4)])
def test_attention_peaked_and_flat(fmt, dt, amplitude, scale):
    """Softmaxes of one key and of all alike; queries far from unit scale."""
    Pool(fmt, dt, 2, 64, 16, [200, 90], [1, 40]).fill().check(4, amplitude=amplitude, sm_scale=scale)


def test_attention_bf16_queries_of_any_magnitude():
    """bf16 queries from 2^-90 to 2^60 over integer pages (whose products are in fp16)."""
    p = Pool(I8, BF, 1, 64, 16, [50, 50, 50], [1, 1, 30]).fill()
    rng = np.random.default_rng(0)
    q = rng.standard_normal((32, 64)) * 2.0 ** rng.integers(-8, 1, (32, 64))
    for e in (-90, 60):
        d = to16(q * 2.0 ** e, BF)
        want, bound = p.want(d, 1, 2.0 ** -e)
        assert_close(values(p.attend(d, 1, 2.0 ** -e)), want, bound, e)


@pytest.mark.parametrize("fmt", [I8, I4], ids=["i8", "i4"])
def test_attention_value_scales_far_apart(fmt):
    """Value vectors from 2^-20 to 2^14, zero vectors (scale 1) among small ones."""
    p = Pool(fmt, BF, 1, 128, 16, [150, 150], [1, 33]).fill(spread=4.0, outlier=1.0).check(3)
    p = Pool(fmt, HALF, 1, 128, 16, [64], [1])
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 64, 128))
    v *= 2.0 ** -12
    v[::3] = 0
    p.rebatch([64], [64])
    p.append(to16(k, HALF), to16(v, HALF))
    p.rebatch([64], [1])
    p.check(4)


@pytest.mark.parametrize("fmt", [F16, I8, I4], ids=["f16", "i8", "i4"])
@pytest.mark.parametrize("new", [1, 6, 90])
def test_attention_pages_that_are_not_there(fmt, new):
    p = Pool(fmt, HALF, 2, 64, 16, [300, 130], [new, 1]).fill()
    p.table[0, 3], p.table[0, 4], p.table[0, 11] = -1, p.n_pages, 2 ** 31 - 1
    p.table[1] = -7                                      # no key at all: zeros
    p.rebatch([300, 130], [new, 1])
    got = p.check(4)
    assert not got[new].any()


@pytest.mark.parametrize("fmt", [F16, I8, I4], ids=["f16", "i8", "i4"])
@pytest.mark.parametrize("hq", [2, 14])
@pytest.mark.parametrize("new", [5, 100])
def test_attention_values_not_finite_reach_only_who_sees_them(fmt, hq, new):
    """A key or a value that is NaN or infinite at position t: queries before t
    are as if it were not there, those from t on get what the sum gives."""
    t = H.torch()
    n = 160
    p = Pool(fmt, HALF, 2, 64, 16, [n], [new]).fill()
    at = n - new // 2 - 1
    pg, r = p.o.place(0, at)
    q = to16(np.random.default_rng(3).standard_normal((new, hq * 64)), HALF)
    clean = values(p.attend(q, hq))
    for pool, scale in ((p.d.k, p.d.k_scale), (p.d.v, p.d.v_scale)):
        for bad in (float("nan"), float("inf")):
            where = (pg, 1, r, 7) if fmt == F16 else (pg, 1, r)
            x = pool if fmt == F16 else scale
            keep = x[where].clone()
            x[where] = bad
            got = values(p.attend(q, hq))
            x[where] = keep
            rows = np.arange(n - new, n)
            head = (np.arange(hq * 64) // 64) // (hq // 2) == 1
            assert np.array_equal(got[rows < at], clean[rows < at])
            assert np.array_equal(got[:, ~head], clean[:, ~head])
            seen = got[rows >= at][:, head]
            if pool is p.d.v:
                hit = seen.reshape(len(seen), -1, 64)[..., 7]
                assert not np.isfinite(hit).any()
                if fmt == F16:
                    rest = np.delete(seen.reshape(len(seen), -1, 64), 7, axis=2)
                    assert np.array_equal(rest, np.delete(clean[rows >= at][:, head].reshape(len(seen), -1, 64), 7, axis=2))
            elif bad != bad:
                assert np.isnan(seen).all()


@pytest.mark.parametrize("fmt", [F16, I8, I4], ids=["f16", "i8", "i4"])
def test_attention_query_nan_stays_in_its_row(fmt):
    for new in (3, 80):
        p = Pool(fmt, BF, 1, 64, 16, [90], [new]).fill()
        q = to16(np.random.default_rng(0).standard_normal((new, 4 * 64)), BF)
        clean = values(p.attend(q, 4))
        q[1, 64 + 5] = float("nan")
        got = values(p.attend(q, 4)).reshape(new, 4, 64)
        assert np.isnan(got[1, 1]).all()
        got[1, 1] = clean.reshape(new, 4, 64)[1, 1]
        assert np.array_equal(got.reshape(new, -1), clean)


@pytest.mark.parametrize("new", [1, 100])
def test_attention_sequences_that_share_pages(new):
    """Two sequences with the same first pages (a common prompt) read them both."""
    p = Pool(I8, BF, 2, 128, 16, [100, 90], [new, 1]).fill()
    p.table[1, :4] = p.table[0, :4]
    p.rebatch([100, 90], [new, 1])
    p.check(6)


@pytest.mark.parametrize("new", [1, 100])
def test_attention_strides_and_rows_behind(new):
    t = H.torch()
    p = Pool(I8, HALF, 2, 64, 16, [120, 100], [new, 1]).fill()
    n = new + 1
    p.rebatch([120, 100], [new, 1], n_rows=n + 4)
    q = t.full((n + 4, 4 * 64 + 40), float("nan"), dtype=t.float16, device="cuda")
    q[:n, :256] = to16(np.random.default_rng(0).standard_normal((n, 256)), HALF)
    out = t.full((n + 4, 256 + 8), 3.0, dtype=t.float16, device="cuda")
    p.attend(q, 4, out=out)
    got = values(out)
    assert (got[n:] == 3.0).all() and (got[:, 256:] == 3.0).all()
    want, bound = p.want(q[:n], 4)
    assert_close(got[:n, :256], want, bound)


def test_attention_bounds_above_the_lengths():
    """max_len and max_new may be larger than any length and count."""
    p = Pool(I8, HALF, 2, 64, 16, [90, 31], [1, 2]).fill()
    for max_len, max_new in ((90, 2), (5000, 2), (5000, 700), (90, 64)):
        p.rebatch([90, 31], [1, 2], max_len=max_len, max_new=max_new)
        p.check(4)


@pytest.mark.parametrize("fmt,dt", [(F16, HALF), (I8, BF), (I4, HALF)], ids=["f16-f16", "i8-bf16", "i4-f16"])
@pytest.mark.parametrize("mixed", [False, True])
def test_attention_parts_by_all_lengths(fmt, dt, mixed):
    """Batches that nearly fill the chip, of sequences one of which is much longer
    than the others: only the longest are cut (and joined)."""
    lens = [4300, 1500, 900, 130] + [200 + 7 * i for i in range(16)]
    news = [130] * 20
    if mixed:
        lens, news = lens + [5000, 1, 77], news + [1, 1, 2]
    Pool(fmt, dt, 8, 64, 64, lens, news).fill().check_large(8)


@pytest.mark.parametrize("fmt,dt", [(F16, HALF), (I8, BF), (I4, HALF)], ids=["f16-f16", "i8-bf16", "i4-f16"])
@pytest.mark.parametrize("chunk", [1, 60])
def test_attention_one_long_among_many(fmt, dt, chunk):
    """More sequences and heads than the chip holds workgroups of, one of them long: parts by all lengths, where
    other sequences grow long, and where none is, under the same bounds."""
    many = [5 + b % 60 for b in range(131)]
    p = Pool(fmt, dt, 8, 64, 64, many[:40] + [9000] + many[40:], [1] * 132).fill()
    for lens in (p.lens, many[:40] + [8200] + many[40:], many[:40] + [70] + many[40:], [0] * 132):
        news = [min(n, 1) for n in lens]
        news[100] = min(lens[100], chunk)
        if sum(news):
            p.rebatch(lens, news, max_len=9000, max_new=chunk, n_rows=132 + chunk)
            p.check_large(8)


@pytest.mark.parametrize("batch", [70, 1100])
def test_attention_mixed_large_batches(batch):
    """More sequences than a wave has lanes, and than workgroups look through."""
    lens = [1 + (37 * b) % 150 for b in range(batch)]
    news = [min(n, 1 if b % 5 else 50) for b, n in enumerate(lens)]
    news[3] = news[batch - 2] = 0
    Pool(I8, HALF, 1, 64, 16, lens, news).fill().check_large(2)


@pytest.mark.parametrize("fmt", [F16, I8], ids=["f16", "i8"])
def test_attention_eight_waves(fmt):
    """Workgroups of 256 rows: many rows of grouped heads, a last workgroup of few."""
    Pool(fmt, BF, 2, 128, 64, [700, 300, 260], [161, 300, 150]).fill().check_large(14)


def test_attention_spare_rows_and_cut_keys():
    """Rows behind the step's, with the keys cut into parts: written by neither kernel nor join."""
    t = H.torch()
    p = Pool(F16, BF, 1, 128, 64, [2900], [130]).fill()
    p.rebatch([2900], [130], n_rows=5000)
    q = t.full((5000, 3 * 128), float("nan"), dtype=t.bfloat16, device="cuda")
    q[:130] = to16(np.random.default_rng(0).standard_normal((130, 3 * 128)), BF)
    got = values(p.attend(q, 3))
    assert (got[130:] == 3.0).all()
    want, bound = p.want(q[:130], 3)
    assert_close(got[:130], want, bound)


def test_attention_repeats_bit_for_bit():
    for fmt, news in ((F16, [1, 1]), (I8, [200, 1]), (I4, [7, 1])):
        p = Pool(fmt, BF, 2, 128, 32, [2500, 900], news).fill()
        q = to16(np.random.default_rng(0).standard_normal((sum(news), 8 * 128)), BF)
        a = bits(p.attend(q, 8))
        for _ in range(3):
            assert np.array_equal(bits(p.attend(q, 8)), a)


def test_offsets_past_32_bits():
    """A pool of 5 GB keys and values: the pages at its end."""
    t = H.torch()
    heads, dh, page = 40, 128, 1024
    n_pages = 1100                                    # 5.2 MB of keys each
    d = B.DevicePages(I8, HALF, n_pages, page, heads, dh)
    table = [[n_pages - 1, n_pages - 7], [3, n_pages - 2]]
    lens, news = [1040, 1100], [1040, 1100]
    batch = B.DevicePageBatch(table, lens, news)
    rng = t.Generator(device="cuda").manual_seed(0)
    k, v = (t.randn((2140, heads * dh), generator=rng, device="cuda").half() for _ in range(2))
    s = B.stream_handle()
    B.check(B.qsvd_paged_append(d.c, batch.c, B.ptr(k), heads * dh, B.ptr(v), heads * dh, 1.0, s))
    # the same in a small pool
    e = B.DevicePages(I8, HALF, 4, page, heads, dh)
    small = B.DevicePageBatch([[0, 1], [2, 3]], lens, news)
    B.check(B.qsvd_paged_append(e.c, small.c, B.ptr(k), heads * dh, B.ptr(v), heads * dh, 1.0, s))
    for new in (1, 70):
        q = t.randn((2 * new, heads * dh), generator=rng, device="cuda").half()
        outs = []
        for pool, tab in ((d, table), (e, [[0, 1], [2, 3]])):
            b = B.DevicePageBatch(tab, lens, [new, new])
            size = B.qsvd_paged_attention_workspace_size(pool.c, b.c, heads)
            ws = t.empty((max(size, 1),), dtype=t.uint8, device="cuda")
            out = t.empty_like(q)
            B.check(B.qsvd_paged_attention(pool.c, b.c, B.ptr(q), heads * dh, heads, 0.0, B.ptr(out), heads * dh,
                                           B.ptr(ws), size, s))
            outs.append(bits(out))
        assert np.array_equal(*outs)
    back = [t.empty_like(k) for _ in range(4)]
    B.check(B.qsvd_paged_read(d.c, batch.c, B.ptr(back[0]), heads * dh, B.ptr(back[1]), heads * dh, s))
    B.check(B.qsvd_paged_read(e.c, small.c, B.ptr(back[2]), heads * dh, B.ptr(back[3]), heads * dh, s))
    assert t.equal(back[0], back[2]) and t.equal(back[1], back[3])


# ---------------------------------------------------------------- together

def test_chunked_prompt_and_decode_of_a_layer():
    """The tiny layer: its quantized projection, rotary positions with three
    axes, append and attention, the prompt in two uneven chunks and then token
    by token, beside the same prompt in one call, against the oracle."""
    t = H.torch()
    wl = configs.get(1)
    L = wl.layer
    W = gen.weight_matrix(wl)
    dl = B.DeviceLayer(prep.prepare_from_weight(W, L.r, L.n_q_heads, L.n_kv_heads, L.head_dim))
    X = np.concatenate([gen.prefill_activations(wl)] + [gen.decode_activations(wl, i) for i in range(3)])
    n, nq, nkv, dh = X.shape[0], L.n_q, L.n_kv, L.head_dim
    section, theta = (8, 12, 12), 1e4
    pos = np.stack([np.arange(n) // 16, np.arange(n) % 16 // 4, np.arange(n) % 4]).astype(np.int32)
    pos[:, 64:] = np.arange(4, 4 + n - 64)
    r = B.rope(dh, section, theta)
    pages = B.DevicePages(I8, HALF, 8, 16, L.n_kv_heads, dh)
    table = [[5, 2, 7, 0, 3]]
    got = np.empty((n, nq))
    keys, vals, qs = [], [], []
    at = 0
    s = B.stream_handle()
    for new in [23, 41] + [1] * 3:
        p = H.Prefill(dl, new, debug=False).run(H.dev(X[at:at + new]))
        res = p.result()
        d = H.dev(np.ascontiguousarray(pos[:, at:at + new]))
        B.check(B.qsvd_rope_axes(r, B.ptr(d), new, new, HALF, B.ptr(p.q), nq, L.n_q_heads, B.ptr(p.q), nq, B.ptr(p.k), nkv,
                                 L.n_kv_heads, B.ptr(p.k), nkv, s))
        for name, buf, heads, acc in (("Q", p.q, L.n_q_heads, qs), ("K", p.k, L.n_kv_heads, keys)):
            x = res[name].astype(np.float64).reshape(new, heads, dh)
            want = P.rope_axes(x, pos[:, at:at + new], section, theta)
            turned = values(buf).reshape(new, heads, dh)
            assert_close(turned, want, rope_bound(x, want, HALF), name)
            acc.append(turned)
        vals.append(res["V"].astype(np.float64).reshape(new, L.n_kv_heads, dh))
        at += new
        batch = B.DevicePageBatch(table, [at], [new])
        B.check(B.qsvd_paged_append(pages.c, batch.c, B.ptr(p.k), nkv, B.ptr(p.v), nkv, 1.0, s))
        size = B.qsvd_paged_attention_workspace_size(pages.c, batch.c, L.n_q_heads)
        ws = t.empty((max(size, 1),), dtype=t.uint8, device="cuda")
        out = t.empty_like(p.q)
        B.check(B.qsvd_paged_attention(pages.c, batch.c, B.ptr(p.q), nq, L.n_q_heads, 0.0, B.ptr(out), nq, B.ptr(ws), size, s))
        got[at - new:at] = values(out)
    # the oracle's pages, from the turned keys
    o = P.Batch(table, [n], [0, n], 16, 8)
    stored = []
    for rows in (np.concatenate(keys), np.concatenate(vals)):
        c, sc = P.quantize_heads(rows, 8)
        x = np.zeros((8, L.n_kv_heads, 16, dh))
        for m, b, q_ in o.rows(n):
            pg, row = o.place(b, q_)
            x[pg, :, row] = c[m] * sc[m].astype(np.float64)[..., None]
        stored.append(x)
    want, bound = P.attention(np.concatenate(qs), *stored, o, n, dh ** -0.5, HALF_STEP[HALF])
    bound = bound + HALF_STEP[HALF] * np.abs(want) + 2.0 ** -25 * np.abs(stored[1]).max() * n
    assert_close(got, want.reshape(n, -1), bound.reshape(n, -1))


def test_prompt_is_the_rotary_prompt_attention():
    """On one axis, over 16-bit pages, the step is qsvd_prefill_attention_rope to both sides' roundings."""
    t = H.torch()
    lens = [64, 200, 1]
    n, hq, hkv, dh = sum(lens), 8, 2, 128
    rng = np.random.default_rng(5)
    q, k, v = (to16(rng.standard_normal((n, h * dh)), HALF) for h in (hq, hkv, hkv))
    want = values(H.prefill_attention(q, k, v, lens, hq, hkv, dh, rope_theta=1e4))
    pos = H.dev(np.concatenate([np.arange(x) for x in lens]).astype(np.int32)[None])
    s = B.stream_handle()
    B.check(B.qsvd_rope_axes(B.rope(dh, (64,), 1e4), B.ptr(pos), n, n, HALF, B.ptr(q), hq * dh, hq, B.ptr(q), hq * dh,
                             B.ptr(k), hkv * dh, hkv, B.ptr(k), hkv * dh, s))
    p = Pool(F16, HALF, hkv, dh, 64, lens, lens)
    p.append(k, v)
    got = values(p.attend(q, hq))
    ok, err = H.close_enough(got, want)
    assert ok, err
    exact, bound = p.want(q, hq)
    assert_close(got, exact, bound)


@pytest.mark.parametrize("fmt", [F16, I8, I4], ids=["f16", "i8", "i4"])
@pytest.mark.parametrize("chunk", [1, 40])
def test_step_captured_and_replayed(fmt, chunk):
    """A step (turn, append, attend) captured once at the largest lengths and
    replayed as the sequences grow, with eager steps on other data between the
    replays: every replay is the eager step bit for bit."""
    t = H.torch()
    dt, hq, hkv, dh, page, steps = HALF, 4, 2, 64, 16, 4
    lens0 = [40, 700]
    final = [n + steps * chunk for n in lens0]
    news = [chunk, 1]
    rng = np.random.default_rng(0)
    r = B.rope(dh, (8, 12, 12), 1e4)
    n = sum(news)

    def side():
        p = Pool(fmt, dt, hkv, dh, page, final, news, poison=False)
        p.rebatch(lens0, [1, 1])
        p.fill()
        p.rebatch(lens0, news, max_len=max(final), max_new=chunk)
        x = {k: t.zeros((n, h * dh), dtype=t.float16, device="cuda") for k, h in (("q", hq), ("k", hkv), ("v", hkv), ("o", hq))}
        x["pos"] = t.zeros((3, n), dtype=t.int32, device="cuda")
        size = B.qsvd_paged_attention_workspace_size(p.d.c, p.batch.c, hq)
        x["ws"] = t.empty((max(size, 1),), dtype=t.uint8, device="cuda")
        return p, x, size

    def step(p, x, size):
        s = B.stream_handle()
        B.check(B.qsvd_rope_axes(r, B.ptr(x["pos"]), n, n, dt, B.ptr(x["q"]), hq * dh, hq, B.ptr(x["q"]), hq * dh,
                                 B.ptr(x["k"]), hkv * dh, hkv, B.ptr(x["k"]), hkv * dh, s))
        B.check(B.qsvd_paged_append(p.d.c, p.batch.c, B.ptr(x["k"]), hkv * dh, B.ptr(x["v"]), hkv * dh, 1.0, s))
        B.check(B.qsvd_paged_attention(p.d.c, p.batch.c, B.ptr(x["q"]), hq * dh, hq, 0.0, B.ptr(x["o"]), hq * dh,
                                       B.ptr(x["ws"]), size, s))

    eager, graph = side(), side()

    def load(i, sd):
        rng = np.random.default_rng(100 + i)
        for k in ("q", "k", "v"):
            sd[1][k].copy_(to16(rng.standard_normal(tuple(sd[1][k].shape)), dt))
        sd[1]["pos"].copy_(H.dev(rng.integers(0, 5000, (3, n)).astype(np.int32)))
        lens = [lens0[0] + (i + 1) * chunk, lens0[1] + i + 1]
        sd[0].batch.seq_len.copy_(t.tensor(lens, dtype=t.int32))

    step(*side())                                    # kernels loaded before the capture
    t.cuda.synchronize()
    load(0, graph)
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g):
        step(*graph)
    for i in range(steps):
        load(i, eager)
        step(*eager)
        want = bits(eager[1]["o"])
        load(i, graph)
        g.replay()
        t.cuda.synchronize()
        assert np.array_equal(bits(graph[1]["o"]), want), i
        t.cuda.synchronize()
    assert np.array_equal(bits(graph[0].d.k), bits(eager[0].d.k)) and np.array_equal(bits(graph[0].d.v), bits(eager[0].d.v))
    del g


@pytest.mark.parametrize("fmt", [F16, I8], ids=["f16", "i8"])
@pytest.mark.parametrize("spare", [0, 30])
def test_attention_replayed_with_other_lengths(fmt, spare):
    """Captured once for a batch of long chunks (parts by all lengths) and replayed with other lengths, other
    chunks, single tokens and nothing new: each replay is the eager call bit for bit, and right."""
    t = H.torch()
    lens, most, hq, dh = [4300, 1500, 900, 130] + [200 + 7 * i for i in range(16)], 130, 8, 64
    rows = len(lens) * most + spare
    p = Pool(fmt, HALF, hq, dh, 64, lens, [1] * len(lens)).fill()
    q = to16(np.random.default_rng(3).standard_normal((rows, hq * dh)), HALF)
    p.rebatch(lens, [most] * len(lens), 4300, most, rows)
    c = p.batch
    size = B.qsvd_paged_attention_workspace_size(p.d.c, c.c, hq)
    ws = t.full((2, max(size, 1)), 255, dtype=t.uint8, device="cuda")
    out = t.full((2, rows, hq * dh), 3.0, dtype=t.float16, device="cuda")

    def call(i):
        B.check(B.qsvd_paged_attention(p.d.c, c.c, B.ptr(q), hq * dh, hq, 0.0, B.ptr(out[i]), hq * dh, B.ptr(ws[i]), size,
                                       B.stream_handle()))

    call(0)
    t.cuda.synchronize()
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g):
        call(1)
    rng = np.random.default_rng(4)
    for step in range(5):
        n = [int(x) for x in (lens if step < 2 else rng.integers(0, np.array(lens) + 1))]
        new = [min(x, [most, 1, 100, 17, 0][step] if step != 2 or b % 3 else 1) for b, x in enumerate(n)]
        c.seq_len.copy_(t.tensor(n, dtype=t.int32))
        c.first.copy_(t.tensor([sum(new[:b]) for b in range(len(n) + 1)], dtype=t.int32))
        out.fill_(3.0)
        call(0)
        g.replay()
        t.cuda.synchronize()
        assert t.equal(out[0], out[1]), step
        assert bool((out[:, sum(new):] == 3).all()) and not bool(t.isnan(out).any())
        for b in (0, 1, 5):
            if new[b] == 0:
                continue
            m = sum(new[:b + 1]) - 1                      # the last token: sees every key of its sequence
            (k, _), (v, codes) = p.stored()
            pages = p.table[b, :-(-n[b] // 64)]
            kk, vv = (x[pages, 0].reshape(-1, dh)[:n[b]] for x in (k, v))
            w = np.exp((x := kk @ values(q[m, :dh]) * dh ** -0.5) - x.max())
            want = w @ vv / w.sum()
            # (three roundings of 2^-11, of weights, their sum and the output, of at most the largest value)
            assert np.abs(values(out[0, m, :dh]) - want).max() <= 2.0 ** -9 * np.abs(vv).max(), (step, b)
    del g


def test_two_streams_with_workspaces_of_their_own():
    t = H.torch()
    sides = []
    for i, fmt in enumerate((F16, I4)):
        p = Pool(fmt, HALF, 2, 128, 16, [3000, 500], [1, 60 * i + 1]).fill(seed=i)
        q = to16(np.random.default_rng(i).standard_normal((p.n_rows, 4 * 128)), HALF)
        sides.append((p, q, t.cuda.Stream(), bits(p.attend(q, 4)), t.empty_like(q),
                      t.empty((B.qsvd_paged_attention_workspace_size(p.d.c, p.batch.c, 4) + 1,), dtype=t.uint8, device="cuda")))
    t.cuda.synchronize()
    for _ in range(10):
        for p, q, st, _, out, ws in sides:
            p.attend(q, 4, out=out, ws=ws, stream=st)
        t.cuda.synchronize()
        for p, q, st, want, out, ws in sides:
            assert np.array_equal(bits(out), want)
