"""Attention over pages at the ends of what its arguments allow, against the
oracle in 64 bits and its bound."""
import numpy as np
import pytest

from test_gpu_paged import BF, F16, FORM_IDS, FORMS, HALF, I4, I8, Pool, assert_close, bits, to16, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dt", FORMS, ids=FORM_IDS)
@pytest.mark.parametrize("new", [1, 7, 50])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -30, 2.0 ** -40, 2.0 ** -100, 2.0 ** -126, 2.0 ** -149])
def test_queries_of_zeros_and_tiny_ones(fmt, dt, new, scale):
    """A query of zeros averages the values that it sees, whatever the scale; rows next to it are as ever."""
    p = Pool(fmt, dt, 2, 64, 16, [90, 75], [new, 1]).fill()
    q = np.random.default_rng(0).standard_normal((new + 1, 4, 64))
    q[0, 1] = q[-1, 2] = q[new // 2, 3] = 0
    q[new // 2, 0] *= 2.0 ** -110 if dt == BF else 2.0 ** -14
    d = to16(q.reshape(new + 1, -1), dt)
    got = values(p.attend(d, 4, scale))
    want, bound = p.want(d, 4, scale)
    assert_close(got, want, bound, scale)


@pytest.mark.parametrize("fmt,dt", FORMS, ids=FORM_IDS)
@pytest.mark.parametrize("heads,hq,lens,news,n_rows", [
    (1, 1, [50, 900], [50, 900], 100), (1, 1, [40, 300, 300], [40, 300, 300], 400), (1, 1, [1000], [1000], 100),
    (2, 4, [300, 1500, 70], [1, 200, 70], 60), (1, 4, [2000, 90], [300, 1], 299), (4, 4, [20, 400, 30], [20, 130, 1], 150),
    (1, 1, [64, 64, 500], [64, 64, 500], 128), (2, 4, [70, 80, 90], [5, 3, 4], 6), (1, 2, [300], [300], 1),
])
def test_rows_that_are_not_there_any_more(fmt, dt, heads, hq, lens, news, n_rows):
    """n_rows below the step's rows, also inside a chunk: the rows before it are as ever, the others left alone."""
    dh, n = 64, sum(news)
    p = Pool(fmt, dt, heads, dh, 16, lens, news).fill()
    q = to16(np.random.default_rng(0).standard_normal((n, hq * dh)), dt)
    q[n_rows:] = float("nan")
    p.rebatch(lens, news, n_rows=n_rows)
    got = values(p.attend(q, hq))
    want, bound = p.want(q[:n_rows], hq)
    assert (got[n_rows:] == 3.0).all()
    assert_close(got[:n_rows], want, bound)


@pytest.mark.parametrize("fmt", [F16, I8, I4], ids=["f16", "i8", "i4"])
def test_append_and_read_of_rows_that_are_there(fmt):
    """n_rows inside a sequence's rows: the tokens behind it are neither written nor read."""
    lens, news, n_rows = [40, 50], [40, 45], 60
    p = Pool(fmt, HALF, 2, 64, 16, lens, news)
    rows = to16(np.random.default_rng(1).standard_normal((85, 128)), HALF)
    p.rebatch(lens, news, n_rows=n_rows)
    before = bits(p.d.k)
    p.append(rows, rows)
    places = [p.o.place(b, pos) for _, b, pos in p.o.rows(n_rows)]
    changed = (bits(p.d.k) != before).reshape(p.n_pages, 2, p.page, -1).any((1, 3))
    assert sorted(zip(*np.nonzero(changed))) == sorted(places) and len(places) == n_rows
    back = [rows.clone().fill_(6.0) for _ in range(2)]
    p.read(*back)
    got = values(back[0])
    assert (got[n_rows:] == 6.0).all() and np.array_equal(got, values(back[1]))
    assert np.abs(got[:n_rows] - values(rows)[:n_rows]).max() <= {F16: 0, I8: 0.02, I4: 0.4}[fmt]


@pytest.mark.parametrize("fmt,dt", FORMS, ids=FORM_IDS)
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [3, 2, 4, 1], [40, 1, 60, 7]])
def test_negative_lengths(fmt, dt, news):
    """Sequences whose new tokens have negative positions, down to the type's lowest: not written, zeros read and
    zeros as outputs; the sequence next to them is as ever."""
    lens = [-(2 ** 31), 50, -1, -(2 ** 31) + 5]
    n = sum(news)
    p = Pool(fmt, dt, 2, 64, 16, lens, news)
    p.table = np.where(p.table < 0, 1, p.table).astype(np.int32)        # every column names a page
    p.rebatch([0, 50, 0, 0], [0, 50, 0, 0])
    rows = to16(np.random.default_rng(0).standard_normal((50, 128)), dt)
    p.append(rows, rows)
    p.rebatch(lens, news, max_len=50)
    before = bits(p.d.k)
    new = to16(np.random.default_rng(1).standard_normal((n, 128)), dt)
    mine = np.arange(news[0], news[0] + news[1])
    new[mine] = rows[-news[1]:]                                           # the second sequence's as they are
    p.append(new, new)
    assert np.array_equal(bits(p.d.k), before)
    back = [new.clone().fill_(6.0) for _ in range(2)]
    p.read(*back)
    others = np.setdiff1d(np.arange(n), mine)
    assert not values(back[0])[others].any() and (values(back[1])[mine] != 0).any()
    q = to16(np.random.default_rng(2).standard_normal((n, 4 * 64)), dt)
    got = values(p.attend(q, 4))
    want, bound = p.want(q, 4)
    assert not want[others].any()
    assert_close(got, want, bound)
