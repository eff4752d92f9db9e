"""Attention over pages of codes whose value scales are far apart, element by
element against the oracle in 64 bits and its bound."""
import numpy as np
import pytest

from test_gpu_paged import BF, F16, FMT, HALF, I4, I8, Pool, assert_close, to16, values

pytestmark = pytest.mark.gpu


def fill_values(p, keys, vals):
    """Rows for every token of the pool's one sequence, through append."""
    n, (lens, news) = len(keys), (p.lens, p.news)
    p.rebatch([n], [n])
    p.append(*(to16(x, p.dt).view(n, -1) for x in (keys, vals)))
    p.rebatch(lens, news)


def compare(p, n_q, seed=2, amplitude=1.0, q=None):
    """Pool.check with queries of the caller's."""
    if q is None:
        q = amplitude * np.random.default_rng(seed).standard_normal((p.n_rows, n_q * p.dh))
    q = to16(q, p.dt)
    got = values(p.attend(q, n_q))
    want, bound = p.want(q, n_q)
    assert_close(got, want, bound, f"{FMT[p.fmt]} new {p.news}")
    return got


@pytest.mark.parametrize("fmt", [I8, I4], ids=["i8", "i4"])
@pytest.mark.parametrize("dt", [HALF, BF], ids=["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 9, 60, 150])
@pytest.mark.parametrize("small", [1e-2, 1e-5, 3e-6, 2.0 ** -22])
@pytest.mark.parametrize("amplitude", [0.01, 1.0, 6.0])
def test_half_the_values_far_smaller(fmt, dt, new, small, amplitude):
    """Value rows of magnitude 6e4 and `small` by turns, softmaxes from flat to peaked: small rows keep their share
    of the sum."""
    rng = np.random.default_rng(new)
    n = 150
    p = Pool(fmt, dt, 2, 64, 16, [n], [new])
    vals = np.sign(rng.standard_normal((n, 2, 64))) * rng.uniform(0.5, 1, (n, 2, 64))
    vals *= np.where(np.arange(n) % 2, 6e4, small)[:, None, None]
    fill_values(p, rng.standard_normal((n, 2, 64)), vals)
    compare(p, 4, amplitude=amplitude)


@pytest.mark.parametrize("fmt", [I8, I4], ids=["i8", "i4"])
@pytest.mark.parametrize("dt", [HALF, BF], ids=["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 40, 200])
def test_values_of_every_magnitude(fmt, dt, new):
    """Value rows from 2^-22 to 2^15 in one sequence, in any order."""
    rng = np.random.default_rng(new)
    n = 330
    p = Pool(fmt, dt, 1, 128, 16, [n], [new])
    vals = rng.uniform(-1, 1, (n, 1, 128)) * 2.0 ** rng.integers(-22, 16, (n, 1, 1))
    fill_values(p, rng.standard_normal((n, 1, 128)), vals)
    compare(p, 3)


@pytest.mark.parametrize("fmt", [I8, I4], ids=["i8", "i4"])
@pytest.mark.parametrize("dt", [HALF, BF], ids=["f16", "bf16"])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -140, 2.0 ** -60])
@pytest.mark.parametrize("new", [1, 100])
def test_key_of_most_weight_with_no_value(fmt, dt, new, scale):
    """A caller's pages in which the key that holds most of the softmax has a value scale of 0, or next to it: its
    share of the sum stays."""
    rng = np.random.default_rng(3)
    n, dh = 140, 64
    p = Pool(fmt, dt, 1, dh, 16, [n], [new])
    keys = 0.2 * rng.standard_normal((n, 1, dh))
    keys[7] = 1.0
    fill_values(p, keys, rng.standard_normal((n, 1, dh)))
    pg, r = p.o.place(0, 7)
    p.d.v_scale[pg, 0, r] = scale
    # scores of key 7 about 5, of the others about 0: half to nearly all of the sum
    q = 0.6 + 0.1 * rng.standard_normal((new, 2 * dh))
    compare(p, 2, q=q)


@pytest.mark.parametrize("fmt", [I8, I4], ids=["i8", "i4"])
@pytest.mark.parametrize("dt", [HALF, BF], ids=["f16", "bf16"])
@pytest.mark.parametrize("hq", [2, 8, 14])
@pytest.mark.parametrize("new,dh", [(5, 64), (12, 128), (100, 64), (200, 128)])
def test_far_larger_value_reaches_only_who_sees_it(fmt, dt, hq, new, dh):
    """A finite value row far larger than the others: queries before it are as if it were not there (bit for bit
    but where the weights' sum is taken by what is large in a tile), those from it on within their bound."""
    n = 230
    p = Pool(fmt, dt, 2, dh, 16, [n], [new]).fill()
    at = n - new // 2 - 1
    pg, r = p.o.place(0, at)
    q = to16(np.random.default_rng(3).standard_normal((new, hq * dh)), dt)
    clean = values(p.attend(q, hq))
    before, before_bound = p.want(q, hq)
    rows = np.arange(n - new, n)
    for scale in (2.0 ** 9,) if dt == HALF else (2.0 ** 9, 2.0 ** 40, 2.0 ** 100):
        p.d.v_scale[pg, 1, r] = scale
        got = values(p.attend(q, hq))
        want, bound = p.want(q, hq)
        head = (np.arange(hq * dh) // dh) // (hq // 2) == 1
        assert_close(got[rows < at], before[rows < at], before_bound[rows < at], scale)
        if p.sum_step(hq) == 0:
            assert np.array_equal(got[rows < at], clean[rows < at]), scale
        assert np.array_equal(got[:, ~head], clean[:, ~head]), scale
        sees = rows >= at
        with np.errstate(over="ignore"):
            large = np.abs(want) > (65504 if dt == HALF else 3.38e38)
        ok = sees[:, None] & ~large
        assert_close(np.where(ok, got, 0), np.where(ok, want, 0), bound, scale)


@pytest.mark.parametrize("fmt", [F16, I8, I4], ids=["f16", "i8", "i4"])
@pytest.mark.parametrize("dt", [HALF, BF], ids=["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 20, 90])
@pytest.mark.parametrize("down", [12.0, 24.7, 25.5, 28.3, 31.0])
def test_keys_of_small_weight_beside_one_of_most(fmt, dt, new, down):
    """A key whose value is 0 holds nearly all of the softmax; the others, 2^-down of it each, are the output."""
    rng = np.random.default_rng(6)
    n, dh = 400, 64
    p = Pool(fmt, dt, 1, dh, 16, [n], [new])
    keys = np.zeros((n, 1, dh))
    vals = 1000 * rng.uniform(0.5, 1, (n, 1, dh))
    keys[3], vals[3] = 1.0, 0.0
    fill_values(p, keys, vals)
    q = np.full((new, 2 * dh), down * np.log(2) / 8)                # score of key 3: 64 q / 8, of the others 0
    got = compare(p, 2, q=q)
    assert (got > 0).all()


@pytest.mark.parametrize("fmt", [F16, I8, I4], ids=["f16", "i8", "i4"])
@pytest.mark.parametrize("dt", [HALF, BF], ids=["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 40])
def test_many_keys_of_small_weight_keep_their_share_of_the_sum(fmt, dt, new):
    """2^18 keys of weight 2^-25.5 beside one of weight 1, together 1.0055, all values 1: the outputs are 1, off by
    three roundings (weights, their sum, the output)."""
    n, dh = 1 << 18, 64
    p = Pool(fmt, dt, 1, dh, 64, [n], [new], poison=False)
    keys = np.zeros((n, 1, dh))
    keys[3] = 1.0
    fill_values(p, keys, np.ones((n, 1, dh)))
    q = to16(np.full((new, dh), 25.5 * np.log(2) / 8), dt)
    got = values(p.attend(q, 1))
    assert np.abs(got - 1).max() <= (3.01 * 2.0 ** -11 if dt == HALF else 3.01 * 2.0 ** -8)
