"""The attention oracle's bound (CPU): the kernels' roundings stay within it, a
planted mistake does not."""
import numpy as np

from oracle import paged_oracle as P


def test_bound_counts_the_weights_shift():
    """Weights as the kernels round them (fp16, the largest 2^11, in units of a power of two) stay within the bound;
    without the factor 2^11 they do not.  One key of scale 1 that hardly counts among keys of scale 2^-20."""
    rng = np.random.default_rng(5)
    n, dh = 32, 64
    q = rng.standard_normal((1, 1, dh))
    k = rng.standard_normal((1, 1, n, dh))
    k[0, 0, -1] = -20 * q[0, 0]
    scale = np.full(n, 2.0 ** -20)
    scale[-1] = 1
    code = rng.integers(-127, 128, (n, dh)).astype(np.float64)
    b = P.Batch([[0]], [n], [0, 1], n, 1)
    out, bound = P.attention(q, k, (code * scale[:, None])[None, None], b, 1, 0.125, 2.0 ** -11, np.abs(code)[None, None])
    s = q[0, 0] @ k[0, 0].T * 0.125
    e = np.exp(s - s.max())
    for shift, right in ((11, True), (0, False)):
        w = (2.0 ** shift * e * scale / 2).astype(np.float16).astype(np.float64)
        off = np.abs(w @ code * 2 / (2.0 ** shift * e.sum()) - out[0, 0]) / bound[0, 0]
        assert (off.max() <= 1) == right, (shift, off.max())
