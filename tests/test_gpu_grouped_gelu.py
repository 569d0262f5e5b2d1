"""GELU and its derivative as the bf16 grouped products take them, value by value against float64:
products with the identity, so that what GELU is taken of is known exactly."""
import ctypes as C

import numpy as np
import pytest

from paper_2202_11836_gb300 import _lib as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
special = pytest.importorskip("scipy.special")


def P(t):
    return C.c_void_p(int(t.data_ptr()))


def values():
    """Every bf16 number of 2^-10 <= |z| <= 12, both signs, and 0."""
    bits = np.arange(0x3a80, 0x4141, dtype=np.uint32)
    z = np.concatenate([bits, bits | 0x8000]).astype(np.uint32) << 16
    return np.concatenate([z.view(np.float32).astype(np.float64), [0.0]])


# The values in rows of `width`: up to 64 rows are the kernel of few rows, more the pairs'.
@pytest.mark.parametrize("width", [64, 8], ids=["few rows", "pairs"])
def test_gelu_and_its_derivative_by_value(width):
    z = values()
    rows = -(-len(z) // width)
    assert (rows <= 64) == (width == 64)
    z = np.concatenate([z, np.ones(rows * width - len(z))])
    a = torch.tensor(z, device="cuda").to(torch.bfloat16).view(rows, width)
    w = torch.eye(width, device="cuda", dtype=torch.bfloat16)
    offset = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    c = torch.empty(rows, width, device="cuda", dtype=torch.bfloat16)
    slope = torch.empty(rows, width, device="cuda", dtype=torch.float16)
    shape = L.SkyGroupedShape(1, rows, width, width, L.SKY_DTYPE_BF16)
    n = L.lib().sky_grouped_gemm_workspace_bytes(L.SKY_GEMM_XWT, shape, L.SKY_DTYPE_BF16)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    L.call("sky_grouped_gemm", L.SKY_GEMM_XWT, shape, P(offset), P(a), P(w), P(c), L.SKY_DTYPE_BF16, L.SKY_EPI_BIAS_GELU, None,
           None, P(slope), P(ws), n, None, C.c_void_p(int(torch.cuda.current_stream().cuda_stream)))
    got, got_slope = (x.double().cpu().numpy().ravel() for x in (c, slope))
    tail = np.exp(special.log_ndtr(-np.abs(z)))  # Phi(-|z|)
    density = np.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
    y = np.where(z < 0, z * tail, z - z * tail)
    s = np.where(z < 0, tail, 1 - tail) + z * density
    # Phi(-|z|) and the density in fp32: a polynomial of seven terms off by 6.2e-7 whose coefficients' magnitudes are
    # less than twice its value (7 roundings of 2^-24 of twice that), the hardware's reciprocal (2^-23, which enters up to
    # twice) and exponential (2^-22), two products, together 2.1e-6 and below 2^-18; and the exponent, up to three
    # roundings of z^2 / 2.  Of the value itself: 1 - Phi(-|z|) and the product are rounded
    rel = 2.0 ** -18 + 1.5 * z * z * 2.0 ** -24
    err = np.abs(z) * tail * rel + 2.0 ** -23 * np.abs(y)
    assert (np.abs(got - y) <= err + 2.0 ** -8 * (np.abs(y) + err)).all(), np.abs(got / np.where(y == 0, 1, y) - 1).max()
    # sums near 1 in fp32, twice; fp16 keeps 2^-11 of the value, or 2^-25 below its normal range
    err = (tail + np.abs(z) * density) * rel + 2.0 ** -23
    assert (np.abs(got_slope - s) <= err + 2.0 ** -11 * (np.abs(s) + err) + 2.0 ** -25).all(), np.abs(got_slope - s).max()
