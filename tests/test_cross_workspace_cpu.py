"""The scratch that the cross attention backward asks for: 4 bytes a query row and head,
and 32 more only where the shape leaves the tensor-core kernels possible."""
import os

import pytest

from paper_2202_11836_gb300 import _lib as L


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        from paper_2202_11836_gb300 import build
        build.build()
    return L.lib()


BF16, FP32 = L.SKY_DTYPE_BF16, L.SKY_DTYPE_FP32


@pytest.mark.parametrize("dtype,dim,beside,each", [
    (BF16, 64, 0, 36), (BF16, 64, 8, 36), (BF16, 64, 4, 4), (BF16, 64, 1, 4), (BF16, 32, 0, 4), (BF16, 128, 0, 4),
    (BF16, 33, 0, 4), (FP32, 64, 0, 4), (FP32, 128, 0, 4), (FP32, 20, 3, 4),
])
@pytest.mark.parametrize("B,sq,skv,heads,kv_heads", [(1, 1, 1, 1, 1), (3, 5, 700, 6, 2), (7, 201, 40, 4, 4)])
def test_bytes(lib, B, sq, skv, heads, kv_heads, dtype, dim, beside, each):
    ld = heads * dim + beside
    n = lib.sky_cross_attention_bwd_workspace_bytes(L.SkyCrossShape(B, sq, skv, heads, kv_heads, dim, dtype, ld, ld, ld, ld))
    rows = B * sq * heads
    assert n == (4 * rows + 15) // 16 * 16 + (each - 4) * rows and n % 16 == 0
