"""What the head norms and cross attention refuse, before any device is touched."""
import ctypes as C
import os

import pytest

from paper_2202_11836_gb300 import _lib as L

INVALID, UNSUPPORTED = L.SKY_ERR_INVALID_ARG, L.SKY_ERR_UNSUPPORTED
AT = C.c_void_p(1 << 20)  # an address that no refused call reads


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        from paper_2202_11836_gb300 import build
        build.build()
    return L.lib()


def norm_shape(**kw):
    base = dict(rows=4, q_heads=2, k_heads=2, head_dim=64, dtype=L.SKY_DTYPE_BF16, ldx=256, ldy=256, eps=1e-6,
                rotation=L.SKY_ROTATE_HALVES, theta=10000.0)
    base.update(kw)
    return L.SkyQkNormShape(**base)


NORM_REFUSED = [
    (dict(rows=0), INVALID), (dict(rows=-1), INVALID), (dict(q_heads=-1), INVALID),
    (dict(q_heads=0, k_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(dtype=2), INVALID),
    (dict(rotation=3), INVALID), (dict(rotation=-1), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(theta=0.0), INVALID), (dict(theta=float("inf")), INVALID),
    (dict(theta=float("nan")), INVALID), (dict(ldx=255), INVALID), (dict(ldy=248), INVALID), (dict(ldx=-256), INVALID),
    (dict(head_dim=8), UNSUPPORTED), (dict(head_dim=72, ldx=512, ldy=512), UNSUPPORTED),
    (dict(head_dim=272, ldx=2048, ldy=2048), UNSUPPORTED), (dict(ldx=260), UNSUPPORTED),
    (dict(ldx=258, dtype=L.SKY_DTYPE_FP32), UNSUPPORTED), (dict(ldy=257), UNSUPPORTED),
    (dict(q_heads=1 << 30, k_heads=1 << 30, ldx=1 << 60, ldy=1 << 60), UNSUPPORTED),
]


@pytest.mark.parametrize("bad,status", NORM_REFUSED, ids=lambda v: str(v))
def test_norm_refuses_shapes(lib, bad, status):
    s = norm_shape(**bad)
    assert lib.sky_qk_norm_fwd(s, AT, AT, AT, AT, AT, None) == status
    assert L.last_error()
    assert lib.sky_qk_norm_bwd_workspace_bytes(s) == 0
    assert lib.sky_qk_norm_bwd(s, AT, AT, AT, AT, AT, AT, AT, AT, AT, 1 << 40, None) == status


def test_norm_refuses_arguments(lib):
    s, odd = norm_shape(), C.c_void_p((1 << 20) + 8)
    need = lib.sky_qk_norm_bwd_workspace_bytes(s)
    assert need > 0 and lib.sky_qk_norm_bwd_workspace_bytes(None) == 0
    fwd, bwd = lib.sky_qk_norm_fwd, lib.sky_qk_norm_bwd
    assert fwd(None, AT, AT, AT, AT, AT, None) == INVALID
    assert fwd(s, None, AT, AT, AT, AT, None) == INVALID
    assert fwd(s, AT, AT, AT, AT, None, None) == INVALID
    assert fwd(s, AT, AT, AT, None, AT, None) == INVALID  # a rotation without positions
    assert fwd(s, odd, AT, AT, AT, AT, None) == UNSUPPORTED
    assert fwd(s, AT, AT, AT, AT, odd, None) == UNSUPPORTED
    assert fwd(norm_shape(ldy=264), AT, AT, AT, AT, AT, None) == INVALID  # in place, rows not where they were
    ok = [AT, C.c_void_p(2 << 20), AT, AT, AT, C.c_void_p(3 << 20), AT, AT, AT]
    for i in (0, 1, 5, 8):
        assert bwd(s, *[None if j == i else a for j, a in enumerate(ok)], need, None) == INVALID
    assert bwd(s, *[None if j == 4 else a for j, a in enumerate(ok)], need, None) == INVALID
    for i in (0, 1, 5):
        assert bwd(s, *[odd if j == i else a for j, a in enumerate(ok)], need, None) == UNSUPPORTED
    assert bwd(s, *ok[:8], C.c_void_p((1 << 20) + 2), need, None) == INVALID
    byte, half = C.c_void_p((1 << 20) + 1), C.c_void_p((1 << 20) + 2)
    for i, off in ((2, byte), (3, byte), (4, half), (6, half), (7, half)):  # gains, positions, gain gradients
        assert bwd(s, *[off if j == i else a for j, a in enumerate(ok)], need, None) == INVALID
    for i, off in ((1, byte), (2, byte), (3, half)):
        assert fwd(s, *[off if j == i else AT for j in range(5)], None) == INVALID
    assert fwd(norm_shape(dtype=L.SKY_DTYPE_FP32), AT, half, AT, AT, AT, None) == INVALID
    assert bwd(s, *ok, need - 1, None) == INVALID


def cross_shape(**kw):
    base = dict(batch=2, q_len=3, kv_len=5, heads=4, kv_heads=2, head_dim=64, dtype=L.SKY_DTYPE_BF16, ldq=256, ldk=256,
                ldv=256, ldo=256)
    base.update(kw)
    return L.SkyCrossShape(**base)


CROSS_REFUSED = [(dict([(n, v)]), INVALID) for n in ("batch", "q_len", "kv_len", "heads", "kv_heads", "head_dim")
                 for v in (0, -1)] + [
    (dict(kv_heads=3), INVALID), (dict(kv_heads=8), INVALID), (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID),
    (dict(ldq=255), INVALID), (dict(ldo=0), INVALID), (dict(ldk=127), INVALID), (dict(ldv=-256), INVALID),
    (dict(head_dim=129, ldq=1024, ldk=1024, ldv=1024, ldo=1024), UNSUPPORTED), (dict(batch=65536), UNSUPPORTED),
    (dict(q_len=(1 << 24) + 1), UNSUPPORTED), (dict(kv_len=(1 << 24) + 1), UNSUPPORTED),
    (dict(heads=1026, ldq=1 << 20, ldo=1 << 20), UNSUPPORTED), (dict(ldk=(1 << 30) + 1), UNSUPPORTED),
    (dict(batch=60000, q_len=1 << 20), UNSUPPORTED),
]


@pytest.mark.parametrize("bad,status", CROSS_REFUSED, ids=lambda v: str(v))
def test_cross_refuses_shapes(lib, bad, status):
    s = cross_shape(**bad)
    assert lib.sky_cross_attention_fwd(s, *[AT] * 7, None) == status
    assert L.last_error()
    assert lib.sky_cross_attention_bwd_workspace_bytes(s) == 0
    assert lib.sky_cross_attention_bwd(s, *[AT] * 11, 1 << 40, AT, None) == status


def test_cross_refuses_arguments(lib):
    s, odd = cross_shape(), C.c_void_p((1 << 20) + 1)
    need = lib.sky_cross_attention_bwd_workspace_bytes(s)
    assert need > 0 and lib.sky_cross_attention_bwd_workspace_bytes(None) == 0
    fwd, bwd = lib.sky_cross_attention_fwd, lib.sky_cross_attention_bwd
    assert fwd(None, *[AT] * 7, None) == INVALID
    for i in range(5):  # q, k, v, lengths, ctx
        assert fwd(s, *[None if j == i else AT for j in range(7)], None) == INVALID
    for i in (0, 1, 2, 4):
        assert fwd(s, *[odd if j == i else AT for j in range(7)], None) == INVALID
    for i in (3, 5, 6):  # lengths, lse, status
        assert fwd(s, *[odd if j == i else AT for j in range(7)], None) == INVALID
    for i in (5, 6):
        assert bwd(s, *[odd if j == i else AT for j in range(11)], need, None, None) == INVALID
    assert bwd(s, *[AT] * 11, need, odd, None) == INVALID
    assert bwd(None, *[AT] * 11, need, None, None) == INVALID
    for i in range(11):
        assert bwd(s, *[None if j == i else AT for j in range(11)], need, None, None) == INVALID
    for i in (0, 1, 2, 3, 4, 7, 8, 9):
        assert bwd(s, *[odd if j == i else AT for j in range(11)], need, None, None) == INVALID
    assert bwd(s, *[C.c_void_p((1 << 20) + 8) if j == 10 else AT for j in range(11)], need, None, None) == INVALID
    assert bwd(s, *[AT] * 11, need - 1, None, None) == INVALID
