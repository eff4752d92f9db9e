"""Every form of the W8A8 product at every state of its rings in LDS
(linear_shapes.py), bit for bit."""
import numpy as np
import pytest

from oracle import layer_oracle as L
from paper_2510_16292_amd import binding as B
import linear_shapes as S
from test_gpu_layer_ops import linear_inputs, run_linear

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    B.lib()


@pytest.mark.parametrize("M,N,K", S.STAGES)
def test_linear_stages(M, N, K):
    dt = B.QSVD_BF16 if (M + N + K // 16) % 2 else B.QSVD_F16
    bf = dt == B.QSVD_BF16
    xq, sx, wq, sw, bias, res = linear_inputs(M + 3 * N + 5 * K, M, N, K, bf, full=True)
    got = run_linear(xq, sx, wq, sw, dt, bias, res)
    assert np.array_equal(got, L.linear_i8(xq, sx, wq, sw, bias, res, bf))


def launches(run):
    """Kernels that a call of the linear layer launches."""
    B.check(B.profile_reset())
    B.check(B.profile_enable(True, "linear_i8"))
    try:
        run()
        return sum(B.profile_read(name)[1] for name in ("linear_i8_split", "linear_i8_tile"))
    finally:
        B.check(B.profile_enable(False))
        B.check(B.profile_reset())


@pytest.mark.parametrize("M,N,K,cut", S.PARTS)
def test_linear_in_parts(M, N, K, cut):
    """Several launches, each with its own part of every operand, all of them strided
    and at odd addresses where they may be; the sum in place of the residual too."""
    dt = B.QSVD_F16 if len(cut) == 1 and M % 2 else B.QSVD_BF16
    bf = dt == B.QSVD_BF16
    xq, sx, wq, sw, bias, res = linear_inputs(M + 5 * N + 3 * K, M, N, K, bf, full=True)
    want = L.linear_i8(xq, sx, wq, sw, bias, res, bf)
    got = []
    n = launches(lambda: got.append(run_linear(xq, sx, wq, sw, dt, bias, res, ldx=K + 16, ldy=N + 5, offset=3)))
    assert n == len(cut) + 1
    assert np.array_equal(got[0], want)
    assert np.array_equal(run_linear(xq, sx, wq, sw, dt, bias, res, alias=True), want)
    want = L.linear_i8(xq, sx, wq, sw, None, None, bf)
    assert np.array_equal(run_linear(xq, sx, wq, sw, dt, ldy=-(-N // 64) * 64), want)
