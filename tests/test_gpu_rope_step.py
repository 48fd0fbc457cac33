"""GPU: rotary positions with one axis are the rotation that a training step applies to q and k, as the oracle has it: neighbouring pairs, the same angles, the same sign."""
import numpy as np
import pytest

import layer8lib as l8
from oracle import model as om

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("B,T,H,dh,theta", [(1, 50, 1, 64, 10000.0), (2, 33, 4, 128, 10000.0), (3, 7, 2, 32, 500000.0)])
def test_one_axis_is_the_steps_rotation(B, T, H, dh, theta, inverse, dtype):
    """q and k heads of packed rows; 16 roundings of 32 bits for sine, cosine and the sums of two products, as in the test of several axes."""
    import torch
    import paper_2506_06472_amd as tio
    rng = np.random.default_rng(T)
    x = l8.rounded(rng.standard_normal((B * T, 2 * H * dh)), dtype)
    heads = x.reshape(B, T, 2 * H, dh).transpose(0, 2, 1, 3)
    want = om.rope_apply(heads, *om.rope_tables(T, dh, theta, np.float64), inverse=inverse).transpose(0, 2, 1, 3).reshape(x.shape)
    size = np.repeat(np.abs(x[:, 0::2]) + np.abs(x[:, 1::2]), 2, axis=1) * (16 * l8.E32 + 2.0 ** -50 * T)
    t = l8.padded(x, dtype)
    pos = torch.arange(T, device="cuda", dtype=torch.int32).repeat(B)
    tio.tio_op_rope_axes(0, dtype, B * T, 2 * H, dh, t.data_ptr(), t.stride(0), t.data_ptr(), t.stride(0), pos.data_ptr(), [dh // 2], theta, False, inverse)
    got = t[:, :2 * H * dh].double().cpu().numpy()
    assert (np.abs(got - want) <= l8.U[dtype] * np.abs(want) + 1.01 * size).all()
