"""Attention over pages at the ends of what its arguments allow, against the
oracle in 64 bits and its bound."""
import numpy as np
import pytest

from test_gpu_paged import BF, FORM_IDS, FORMS, Pool, assert_close, to16, values

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
