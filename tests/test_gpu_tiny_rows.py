"""Rows of the norm and the gate next to the bound below which they count as zero
(a = clip * max |y| = 2^-119), bit for bit: just below it, on it and just above."""
import numpy as np
import pytest

from oracle import layer_oracle as L
from paper_2510_16292_amd import binding as B
from test_gpu_layer_ops import run_gate, run_norm

BOUND = np.float32(2.0 ** -119)
BELOW, ABOVE = np.float32(2.0 ** -119 - 2.0 ** -127), np.float32(2.0 ** -119 + 2.0 ** -126)   # the next bf16 numbers


def test_bound_keeps_scales_normal():
    """What the bound is for, and what it is not: Qm / a passes fp32 only far below."""
    fp32 = np.finfo(np.float32)
    assert BOUND / np.float32(127) >= fp32.tiny > BOUND / np.float32(2) / np.float32(127)
    assert np.float32(127) / (BOUND / np.float32(2)) < fp32.max / 2
    for v in (BELOW, BOUND, ABOVE):
        assert L.round16(v, True) == v


@pytest.mark.gpu
@pytest.mark.parametrize("K", [64, 264, 520])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("clip", [1.0, 0.5])
@pytest.mark.parametrize("top", [BELOW, BOUND, ABOVE], ids=["below", "on", "above"])
def test_norm_next_to_the_bound(K, bits, clip, top):
    """Rows of ones (their norm is gamma) with the largest gamma at the bound."""
    g = np.random.default_rng(K + bits)
    x = np.where(g.random((5, K)) < 0.5, -1.0, 1.0).astype(np.float32)
    top = top / np.float32(clip)
    gamma = L.round16(top * g.uniform(0.1, 0.9, K).astype(np.float32), True)
    gamma[K // 2] = top
    got = run_norm(x, None, gamma, B.QSVD_BF16, bits=bits, clip=clip, eps=1e-30)
    _, y, q, s = L.rmsnorm_quantize(x, None, gamma, 1e-30, bits, clip, True)
    assert np.array_equal(got["y"], L.round16(y, True)) and np.array_equal(np.abs(y), np.broadcast_to(gamma, y.shape))
    assert np.array_equal(got["q"], q) and np.array_equal(got["s"], s)
    qm = 2 ** (bits - 1) - 1
    zero = top * np.float32(clip) < BOUND
    assert (np.abs(got["q"]).max(axis=1) == (0 if zero else qm)).all() and ((got["s"] == 1) == zero).all()


@pytest.mark.gpu
@pytest.mark.parametrize("K", [64, 264, 520])
@pytest.mark.parametrize("bits", [8, 4])
def test_gate_next_to_the_bound(K, bits):
    """Gates of 64, whose silu is 64 exactly in fp32 (e^-64 is far below half a step of
    1), so y = 64 up; a row to each side of the bound and one on it."""
    g = np.random.default_rng(K + bits)
    top = np.array([BELOW, BOUND, ABOVE], np.float32)[:, None] / np.float32(64)
    up = L.round16(top * g.uniform(-0.9, 0.9, (3, K)).astype(np.float32), True)
    up[:, K // 3] = L.round16(top, True)[:, 0]
    gate = np.full((3, K), 64, np.float32)
    q, s = run_gate(gate, up, B.QSVD_BF16, bits=bits)
    y = np.float32(64) * up
    assert (np.abs(y).max(axis=1) >= BOUND).tolist() == [False, True, True]
    want_q, want_s = L.quantize_rows(y, bits)
    assert np.array_equal(q, want_q) and np.array_equal(s, want_s)
    assert s[0] == 1 and not q[0].any() and (np.abs(q[1:]).max(axis=1) == 2 ** (bits - 1) - 1).all()
