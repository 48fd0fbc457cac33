"""GPU: norms around a block where threads without columns of their own, or with a part of eight, must not count: rows that dropout empties, magnitudes near the type's end."""
import numpy as np
import pytest

import layer8lib as l8
from test_gpu_layer8_rows import _Case
from test_residual_from_x import _FromX

pytestmark = pytest.mark.gpu
CASES = pytest.mark.parametrize("kind", [_Case, _FromX], ids=["from_y", "from_x"])


@CASES
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms", [True, False])
@pytest.mark.parametrize("d", [1, 5, 8])
def test_rows_that_dropout_empties(d, rms, dtype, kind):
    """A dropped element is zero whatever it was: where all of a row's are, a branch that is not a number leaves no trace in y, h, dx and the gains' gradients of h's norm."""
    c = kind(40, d, dtype, rms, True, None, 0.75)
    empty = (l8.mask(40, d, c.p, c.seed, c.offset) == 0).all(1)
    assert empty.any() and not empty.all()
    clean = c.run()
    c.v["branch"][empty, 0] = np.nan
    got = c.run()
    for n in ("y", "h", "dx", "dgain") + (() if rms else ("dbias",)):
        assert np.array_equal(got[n], clean[n]), n
    assert np.array_equal(got["dbranch"][~empty], clean["dbranch"][~empty])


@CASES
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms", [True, False])
@pytest.mark.parametrize("gate", ["shared", "rows", None])
def test_gradients_of_rows_that_dropout_empties(gate, rms, dtype, kind):
    """Nothing of such a row's branch goes into a gradient but its own."""
    c = kind(40, 8, dtype, rms, True, gate, 0.75)
    empty = (l8.mask(40, 8, c.p, c.seed, c.offset) == 0).all(1)
    clean = c.run()
    c.v["branch"][empty, 3] = np.nan
    got = c.run()
    for n in ("dgate", "dpost_gain", "dpost_bias"):
        if n in clean:
            assert np.array_equal(got[n], clean[n]), n
    assert np.array_equal(got["dbranch"][~empty], clean["dbranch"][~empty])


@CASES
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gate", ["shared", "rows"])
@pytest.mark.parametrize("d", [40, 1030])
def test_a_dropped_infinity(d, gate, dtype, kind):
    """The root-mean-square norm makes zeros of the rest of its row: so are u, and what goes from the row into the gradients of gate and gain."""
    c = kind(6, d, dtype, True, True, gate, 0.5)
    m = l8.mask(6, d, c.p, c.seed, c.offset)
    c.v["branch"][4, int(np.argmin(m[4]))] = np.inf
    got = c.run()
    y = c.rs * c.v["x"][4]
    assert (np.abs(got["y"][4] - y) <= l8.U[dtype] * np.abs(y) + l8.E32 * np.abs(y)).all()
    for n in ("y", "h", "dx", "dgate", "dpost_gain", "dgain"):
        assert np.isfinite(got[n]).all(), n
    if gate == "rows":
        assert (got["dgate"][4] == 0).all()


@CASES
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [1, 100, 128, 600])
def test_large_rows_of_one_value(d, dtype, kind):
    """A row of 2^111, whose layer norm is the bias (where d is a power of two the mean is exact; elsewhere the variance is infinite, and 1 / sqrt of it zero): y, h and the gradients
    are finite, although the mean times 1 / sqrt(eps) = 2^20 is not."""
    c = kind(3, d, dtype, False, True, None, 0.0)
    c.eps = float(np.float32(2.0 ** -40))
    c.v["branch"][1] = 2.0 ** 111
    got = c.run()
    for n, t in got.items():
        assert np.isfinite(t).all(), n
    y = c.rs * c.v["x"][1] + c.bs * c.v["post_bias"][0]
    assert (np.abs(got["y"][1] - y) <= l8.U[dtype] * np.abs(y) + 4 * l8.E32 * (np.abs(c.v["x"][1]) + np.abs(c.v["post_bias"][0]))).all()
