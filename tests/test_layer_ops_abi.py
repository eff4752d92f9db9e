"""The layer operators on the CPU: the oracle against independent closed forms,
and argument validation, which returns the documented status before any GPU
work."""
import math

import numpy as np
import pytest

from oracle import layer_oracle as L
from paper_2510_16292_amd import binding as B

FAKE = 0x100000          # 16-byte-aligned non-NULL address that is never dereferenced on the host
INV, UNS, OK = B.QSVD_ERR_INVALID_ARG, B.QSVD_ERR_UNSUPPORTED, B.QSVD_OK


def norm(**kw):
    a = dict(x=FAKE, ldx=64, residual=FAKE, ldr=64, gamma=FAKE, M=4, K=64, dtype=B.QSVD_F16, eps=1e-6, bits=8, clip=1.0,
             h=FAKE, ldh=64, y=FAKE, ldy=64, xq=FAKE, sx=FAKE)
    a.update(kw)
    return B.qsvd_rmsnorm_quantize_act(a["x"], a["ldx"], a["residual"], a["ldr"], a["gamma"], a["M"], a["K"], a["dtype"],
                                       a["eps"], a["bits"], a["clip"], a["h"], a["ldh"], a["y"], a["ldy"], a["xq"],
                                       a["sx"], 0)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), INV), (dict(K=0), INV), (dict(dtype=2), INV), (dict(bits=6), INV), (dict(clip=0.0), INV),
    (dict(clip=1.5), INV), (dict(clip=math.nan), INV), (dict(eps=0.0), INV), (dict(eps=math.nan), INV),
    (dict(eps=math.inf), INV), (dict(x=0), INV), (dict(gamma=0), INV), (dict(y=0, xq=0, sx=0), INV),
    (dict(xq=0), INV), (dict(sx=0), INV), (dict(ldx=56), INV), (dict(ldr=56), INV), (dict(ldh=56), INV),
    (dict(ldy=56), INV), (dict(K=60), UNS), (dict(K=65544, ldx=65544, ldr=65544, ldh=65544, ldy=65544), UNS),
    (dict(M=1 << 22), UNS), (dict(ldx=68), UNS), (dict(ldr=68), UNS), (dict(ldh=68), UNS), (dict(ldy=68), UNS),
    (dict(x=FAKE + 8), UNS), (dict(residual=FAKE + 8), UNS), (dict(gamma=FAKE + 8), UNS), (dict(h=FAKE + 8), UNS),
    (dict(y=FAKE + 8), UNS), (dict(xq=FAKE + 4), UNS), (dict(sx=FAKE + 2), UNS),
    (dict(ldx=72, residual=FAKE + 4096), INV), (dict(ldr=72, x=FAKE + 4096), INV),
    (dict(M=0), OK), (dict(M=0, x=0, gamma=0, y=0, xq=0, sx=0), OK),
])
def test_norm_validation(kw, status):
    assert norm(**kw) == status
    assert B.last_error() or status == OK


def gate(**kw):
    a = dict(gate=FAKE, ldg=64, up=FAKE, ldu=64, M=4, K=64, dtype=B.QSVD_F16, bits=8, clip=1.0, xq=FAKE, sx=FAKE)
    a.update(kw)
    return B.qsvd_silu_mul_quantize_act(a["gate"], a["ldg"], a["up"], a["ldu"], a["M"], a["K"], a["dtype"], a["bits"],
                                        a["clip"], a["xq"], a["sx"], 0)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), INV), (dict(K=-8), INV), (dict(dtype=-1), INV), (dict(bits=16), INV), (dict(clip=-1.0), INV),
    (dict(gate=0), INV), (dict(up=0), INV), (dict(xq=0), INV), (dict(sx=0), INV), (dict(ldg=56), INV),
    (dict(ldu=56), INV), (dict(K=4), UNS), (dict(K=65544, ldg=65544, ldu=65544), UNS), (dict(M=1 << 22), UNS),
    (dict(ldg=68), UNS), (dict(ldu=68), UNS), (dict(gate=FAKE + 2), UNS), (dict(up=FAKE + 2), UNS),
    (dict(xq=FAKE + 2), UNS), (dict(sx=FAKE + 2), UNS), (dict(M=0), OK),
])
def test_gate_validation(kw, status):
    assert gate(**kw) == status
    assert B.last_error() or status == OK


def linear(**kw):
    a = dict(xq=FAKE, ldx=64, sx=FAKE, wq=FAKE, sw=FAKE, M=4, N=24, K=64, bias=FAKE, residual=FAKE, ldr=24,
             dtype=B.QSVD_F16, y=FAKE, ldy=24)
    a.update(kw)
    return B.qsvd_linear_i8(a["xq"], a["ldx"], a["sx"], a["wq"], a["sw"], a["M"], a["N"], a["K"], a["bias"],
                            a["residual"], a["ldr"], a["dtype"], a["y"], a["ldy"], 0)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), INV), (dict(N=0), INV), (dict(K=0), INV), (dict(dtype=7), INV), (dict(ldx=48), INV),
    (dict(ldy=23), INV), (dict(ldr=23), INV), (dict(xq=0), INV), (dict(sx=0), INV), (dict(wq=0), INV),
    (dict(sw=0), INV), (dict(y=0), INV), (dict(K=56), UNS), (dict(ldx=72), UNS),
    (dict(K=131072, ldx=131072), UNS), (dict(sx=FAKE + 2), UNS), (dict(sw=FAKE + 1), UNS), (dict(ldr=32), INV), (dict(ldx=(1 << 22) + 16), UNS), (dict(xq=FAKE + 8), UNS),
    (dict(wq=FAKE + 8), UNS), (dict(y=FAKE + 1), UNS), (dict(residual=FAKE + 1), UNS), (dict(bias=FAKE + 1), UNS),
    (dict(M=1 << 31, N=1 << 14, ldy=1 << 14, ldr=1 << 14), UNS), (dict(M=(1 << 63) - 1), UNS),
    (dict(M=0), OK), (dict(M=0, xq=0, y=0), OK),
])
def test_linear_validation(kw, status):
    assert linear(**kw) == status
    assert B.last_error() or status == OK


# ---------------------------------------------------------------- the oracle

def test_round16_matches_numpy_and_ties():
    v = np.array([1.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 65536.0, -2.0 ** -130, 3.3e38], np.float32)
    assert L.round16(v, True).tolist() == [1.0, 1.0, 1 + 2.0 ** -6, 65536.0, -2.0 ** -130, float(np.float32(2.0 ** 127 * 1.9375))]
    g = np.random.default_rng(0).standard_normal(1000).astype(np.float32)
    assert np.array_equal(L.round16(g, False), g.astype(np.float16).astype(np.float32))


def test_norm_closed_form():
    """Rows of one magnitude: rms is that magnitude (eps negligible), so every y
    is +-gamma and the codes follow from gamma alone."""
    g = np.array([0.5, 1.0, 2.0, 0.25, 1.0, 1.0, 1.0, 1.0], np.float32)
    sign = np.array([1, -1, 1, 1, -1, 1, 1, -1], np.float32)
    h, y, q, s = L.rmsnorm_quantize(4096.0 * sign[None], None, g, 1e-30, 8, 1.0, False)
    assert np.array_equal(h[0], 4096.0 * sign)
    assert np.array_equal(y[0], sign * g)
    assert np.array_equal(q[0], np.rint(sign * g / 2 * 127).astype(np.int8)) and s[0] == np.float32(2) / np.float32(127)


def test_quantize_rows_edges():
    y = np.zeros((5, 8), np.float32)
    y[1, 3] = 2.0 ** -120
    y[2, 2] = np.inf
    y[3, 5] = np.nan
    y[4] = np.arange(8)
    q, s = L.quantize_rows(y, 4)
    assert s[0] == 1 and s[1] == 1 and np.isnan(s[2]) and np.isnan(s[3]) and not q[:4].any()
    assert q[4].tolist() == list(range(8)) and s[4] == 1


def test_silu_values():
    got = L.silu_mul(np.array([0.0, 1.0, -1000.0, 1000.0]), np.array([5.0, 2.0, 3.0, 2.0]))
    assert np.allclose(got, [0.0, 2 / (1 + math.exp(-1)), 0.0, 2000.0], rtol=1e-15, atol=0)


def test_linear_by_hand():
    xq = np.array([[1, -2, 3], [127, 127, 127]], np.int8)
    wq = np.array([[4, 5, 6], [-127, -127, -127]], np.int8)
    out = L.linear_i8(xq, [0.5, 1.0], wq, [2.0, 0.25], [1.0, 0.0], np.array([[0.0, 8.0], [0.0, 0.0]]), False)
    # 127 * 15 * 2 + 1 = 3811 and -127^2 * 3 / 4 = -12096.75 as fp16 (steps of 2, ties to even, and of 8)
    assert out.tolist() == [[13.0, -254 * 0.125 + 8.0], [3812.0, -12096.0]]


def test_quantize_linear_layout():
    """prep.quantize_linear: codes [N][K] and a scale per output channel, off by
    at most half a step."""
    from paper_2510_16292_amd import prep
    W = np.random.default_rng(0).standard_normal((32, 5))
    W[:, 3] = 0
    codes, scale = prep.quantize_linear(W)
    assert codes.shape == (5, 32) and codes.dtype == np.int8 and scale.shape == (5,) and scale.dtype == np.float32
    assert scale[3] == 1 and not codes[3].any()
    assert np.all(np.abs(codes.T * scale.astype(np.float64) - W) <= scale / 2 * (1 + 1e-6))
    with pytest.raises(AssertionError):
        prep.quantize_linear(W[:24])
