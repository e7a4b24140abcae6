"""The norm of rows whose squares are below fp32's range, with an eps that does not hide it: every kernel, against 64 bits
with the bounds of ordinary rows."""
import numpy as np
import pytest

from tests import test_gpu_rms_norm as norm

pytestmark = pytest.mark.gpu

# a row of each: squares that fp32 rounds to subnormal values, to zero, and values near the lowest normal ones
SIZES = [1.0, 1e-14, 1e-16, 1e-19, 1e-20, 1e-22, 1e-23, 1e-25, 1e-30, 1e-35, 1e-37]


def rows_of(cols, seed):
    _, x = norm.inputs(len(SIZES) + 1, cols, seed)
    x = x.astype(np.float64)
    x[:-1] *= np.array(SIZES)[:, None]
    return x


@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-38, 1e-31])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols,out,block", [(40, "same", 0), (100, "fp8", 0), (200, "int8", 32), (500, "same", 0), (777, "int8", 0),
                                            (2050, "fp8", 128), (8200, "same", 0), (16000, "fp8", 0), (20001, "same", 0),
                                            (18000, "int8", 96), (1000, "fp8", 96)])
def test_rows_of_small_values(dynb, monkeypatch, eps, dtype, cols, out, block):
    monkeypatch.setattr(norm, "NORM_EPS", float(np.float32(eps)))
    x = rows_of(cols, 3)
    norm.forward(len(x), cols, dtype, out, block, residual=False, gain=True, x=x)
    # the residual is what the rows are made of
    norm.forward(len(x), cols, dtype, out, block, residual=True, gain=False, x=0 * x, res=x)


@pytest.mark.parametrize("out", ["same", "fp8"])
@pytest.mark.parametrize("cols", [40, 777, 20001])
def test_a_row_of_zeros_without_eps(dynb, monkeypatch, cols, out):
    """rstd is infinite and the row NaN, as the formula says; its neighbours stay what they are."""
    monkeypatch.setattr(norm, "NORM_EPS", 0.0)
    x = rows_of(cols, 3)
    x[5] = 0
    with np.errstate(all="ignore"):
        norm.forward(len(x), cols, "f32", out, 0, residual=False, gain=False, x=x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [40, 777, 5000, 20001])
def test_gradients_of_small_values(dynb, monkeypatch, cols, dtype):
    monkeypatch.setattr(norm, "NORM_EPS", 0.0)
    x = rows_of(cols, 4)
    norm.backward([5, len(x) - 5], cols, dtype, dsum=False, gain=True, x=x)
