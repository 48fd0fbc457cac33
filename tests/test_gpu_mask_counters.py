"""GPU: masks whose counters need more than 32 bits, which only the norms around a block can reach (tio_op_dropout takes fewer than 2^31 groups of eight)."""
import numpy as np
import pytest

import layer8lib as l8


def _mask_rows(rows, cols, p, seed, offset):
    """layer8lib.mask of the rows with these numbers"""
    groups, limit, low = (cols + 7) // 8, round(p * 65536), 0xffffffff
    words = l8.philox([(c & low, c >> 32, offset & low, offset >> 32) for r in rows for c in range(r * groups, (r + 1) * groups)], (seed & low, seed >> 32))
    halves = np.array([[h for w in c for h in (w & 0xffff, w >> 16)] for c in words]).reshape(len(rows), groups * 8)[:, :cols]
    return (halves >= limit) * (65536 / (65536 - limit))


def test_the_rows_of_a_mask():
    assert np.array_equal(_mask_rows([0, 1, 2, 3], 20, 0.25, 3 << 40, 5), l8.mask(4, 20, 0.25, 3 << 40, 5))


@pytest.mark.gpu
def test_rows_whose_counters_pass_2_to_the_32():
    """y over x, 64 GiB of each matrix; x is zero and the branch one, so that y is the mask."""
    import torch
    import paper_2506_06472_amd as tio
    d, rows, p, seed, offset = 8192, (1 << 22) + 6, 0.5, 2 ** 40 + 9, 2 ** 35 + 1
    assert rows * (d // 8) > 1 << 32 > (rows - 7) * (d // 8)
    torch.cuda.empty_cache()
    need = 3 * rows * d * 2 + rows * 16
    if torch.cuda.mem_get_info()[0] < need + (4 << 30):
        pytest.skip("needs 196 GiB of the GPU's memory")
    new = lambda v: torch.full((rows, d), v, device="cuda", dtype=torch.bfloat16)
    branch, y, h = new(1.0), new(0.0), torch.empty((rows, d), device="cuda", dtype=torch.bfloat16)
    gain, stats = torch.ones((1, d), device="cuda", dtype=torch.bfloat16), torch.empty((rows, 4), device="cuda")
    tio.tio_op_residual_norm(0, "bf16", tio.tio_residual_cfg(True, p=p, seed=seed, offset=offset), rows, d, d, branch.data_ptr(), y.data_ptr(), 0, 0, 0, 0, gain.data_ptr(), 0,
                             y.data_ptr(), h.data_ptr(), stats.data_ptr())
    at = [0, 1, 5, (1 << 22) - 2, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, rows - 1]
    got = y[at].double().cpu().numpy()
    del branch, y, h
    torch.cuda.empty_cache()
    want = _mask_rows(at, d, p, seed, offset)
    assert np.array_equal(got, want) and not np.array_equal(want[0], want[5])
