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
