"""What routing, experts' rows, grouped products and the AdamW step refuse, before any device
is touched."""
import ctypes as C
import os

import pytest

from paper_2202_11836_gb300 import _lib as L

INVALID, UNSUPPORTED = L.SKY_ERR_INVALID_ARG, L.SKY_ERR_UNSUPPORTED
BF, F32 = L.SKY_DTYPE_BF16, L.SKY_DTYPE_FP32
AT = C.c_void_p(1 << 20)  # an address that no refused call reads
BYTE, HALF, WORD = (C.c_void_p((1 << 20) + n) for n in (1, 2, 4))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        from paper_2202_11836_gb300 import build
        build.build()
    return L.lib()


def put(args, i, value):
    return [value if j == i else a for j, a in enumerate(args)]


# ------------------------------------------------------------------- routing
def route_shape(**kw):
    base = dict(tokens=100, experts=8, top_k=2, dtype=F32, weights=L.SKY_ROUTE_OVER_CHOSEN)
    base.update(kw)
    return L.SkyRouteShape(**base)


ROUTE_REFUSED = [
    (dict(tokens=0), INVALID), (dict(tokens=-1), INVALID), (dict(experts=0), INVALID), (dict(top_k=0), INVALID),
    (dict(top_k=9), INVALID), (dict(dtype=2), INVALID), (dict(weights=2), INVALID), (dict(weights=-1), INVALID),
    (dict(experts=1025), UNSUPPORTED), (dict(experts=64, top_k=33), UNSUPPORTED),
    (dict(tokens=1 << 28), UNSUPPORTED), (dict(tokens=1 << 30, experts=2), UNSUPPORTED),
]


@pytest.mark.parametrize("bad,status", ROUTE_REFUSED, ids=str)
def test_route_refuses_shapes(lib, bad, status):
    s = route_shape(**bad)
    assert lib.sky_route_workspace_bytes(s) == 0
    assert lib.sky_route_fwd(s, *[AT] * 6, 1 << 40, AT, None) == status
    assert L.last_error()
    assert lib.sky_route_bwd(s, *[AT] * 4, None) == status


def test_route_refuses_arguments(lib):
    s = route_shape()
    need = lib.sky_route_workspace_bytes(s)
    assert need > 0 and lib.sky_route_workspace_bytes(None) == 0
    fwd = lambda a, n=need, status=None: lib.sky_route_fwd(s, *a, n, status, None)  # noqa: E731
    bwd = lambda a: lib.sky_route_bwd(s, *a, None)  # noqa: E731
    assert lib.sky_route_fwd(None, *[AT] * 6, need, None, None) == INVALID
    assert lib.sky_route_bwd(None, *[AT] * 4, None) == INVALID
    for i in range(6):
        assert fwd(put([AT] * 6, i, None)) == INVALID
        assert fwd(put([AT] * 6, i, HALF)) == INVALID
    for i in range(4):
        assert bwd(put([AT] * 4, i, None)) == INVALID
        assert bwd(put([AT] * 4, i, HALF)) == INVALID
    assert fwd([AT] * 6, status=HALF) == INVALID
    assert fwd([AT] * 6, need - 1) == INVALID
    half = route_shape(dtype=BF)
    assert lib.sky_route_fwd(half, BYTE, *[AT] * 5, need, None, None) == INVALID
    assert lib.sky_route_bwd(half, *[AT] * 3, BYTE, None) == INVALID


def test_route_workspace_covers_many_tokens(lib):
    """Four bytes a block of tokens and expert, and the totals; never less with more tokens of a block size."""
    for e in (1, 64, 1024):
        for t in (1, 64, 65, 8192, 100000, 2000000):
            assert lib.sky_route_workspace_bytes(route_shape(tokens=t, experts=e, top_k=1)) >= (0 if t <= 64 else 4 * e * (t // 256 + 1))


# ---------------------------------------------------------------------- rows
def rows_shape(**kw):
    base = dict(tokens=10, top_k=2, width=64, dtype=BF)
    base.update(kw)
    return L.SkyRowsShape(**base)


ROWS_REFUSED = [
    (dict(tokens=0), INVALID), (dict(top_k=0), INVALID), (dict(width=0), INVALID), (dict(width=-8), INVALID),
    (dict(dtype=3), INVALID), (dict(width=68), UNSUPPORTED), (dict(width=66, dtype=F32), UNSUPPORTED),
    (dict(width=(1 << 20) + 8), UNSUPPORTED), (dict(top_k=33), UNSUPPORTED), (dict(tokens=1 << 30), UNSUPPORTED),
    (dict(tokens=(1 << 31) - 1, top_k=1, width=1 << 20), UNSUPPORTED),
]


def row_calls(lib):
    return [(lib.sky_dispatch_fwd, 3, (0, 2), (1,)), (lib.sky_dispatch_bwd, 3, (0, 2), (1,)),
            (lib.sky_combine_fwd, 4, (0, 3), (1, 2)), (lib.sky_combine_bwd, 6, (0, 1, 4), (2, 3, 5))]


@pytest.mark.parametrize("bad,status", ROWS_REFUSED, ids=str)
def test_rows_refuse_shapes(lib, bad, status):
    for fn, n, _, _ in row_calls(lib):
        if bad.get("width") == 1 << 20 and fn is lib.sky_combine_bwd:
            continue  # a warp a row: its grid is smaller
        assert fn(rows_shape(**bad), *[AT] * n, None) == status
        assert L.last_error()


def test_rows_refuse_arguments(lib):
    s = rows_shape()
    for fn, n, matrices, words in row_calls(lib):
        assert fn(None, *[AT] * n, None) == INVALID
        for i in range(n):
            assert fn(s, *put([AT] * n, i, None), None) == INVALID
        for i in matrices:
            assert fn(s, *put([AT] * n, i, C.c_void_p((1 << 20) + 8)), None) == UNSUPPORTED
        for i in words:
            assert fn(s, *put([AT] * n, i, HALF), None) == INVALID


# ------------------------------------------------------------------ products
def grouped_shape(**kw):
    base = dict(groups=4, rows=100, out=64, in_=32, dtype=BF)
    base.update(kw)
    return L.SkyGroupedShape(**base)


XWT, XW, XTW = L.SKY_GEMM_XWT, L.SKY_GEMM_XW, L.SKY_GEMM_XTW
GROUPED_REFUSED = [
    (dict(groups=0), INVALID), (dict(rows=0), INVALID), (dict(out=0), INVALID), (dict(in_=0), INVALID),
    (dict(in_=-8), INVALID), (dict(dtype=5), INVALID), (dict(out=60), UNSUPPORTED), (dict(in_=36), UNSUPPORTED),
    (dict(groups=1025), UNSUPPORTED), (dict(rows=1 << 28), UNSUPPORTED), (dict(out=(1 << 20) + 8), UNSUPPORTED),
    (dict(in_=(1 << 20) + 8), UNSUPPORTED),
]


def grouped(lib, form, s, args=None, out=None, epi=0, bias=None, aux=None, aux_out=None, ws=AT, n=1 << 40, status=None):
    a = [AT] * 4 if args is None else args  # offsets, A, B, C
    out = (F32 if form == XTW else BF) if out is None else out
    return lib.sky_grouped_gemm(form, s, *a, out, epi, bias, aux, aux_out, ws, n, status, None)


@pytest.mark.parametrize("bad,status", GROUPED_REFUSED, ids=str)
def test_grouped_refuses_shapes(lib, bad, status):
    s = grouped_shape(**bad)
    for form in (XWT, XW, XTW):
        assert grouped(lib, form, s) == status
        assert L.last_error()
        assert lib.sky_grouped_gemm_workspace_bytes(form, s, F32 if form == XTW else BF) == 0
    if "in_" not in bad and bad.get("out") != 60:  # (a column sum has no weights and takes any width)
        assert lib.sky_grouped_column_sum(s, AT, AT, AT, None, None) == status


def test_grouped_refuses_arguments(lib):
    s = grouped_shape()
    assert lib.sky_grouped_gemm_workspace_bytes(XWT, s, BF) > 0
    assert lib.sky_grouped_gemm_workspace_bytes(XWT, None, BF) == 0
    assert lib.sky_grouped_gemm_workspace_bytes(3, s, BF) == 0
    assert grouped(lib, 3, s, out=BF) == INVALID
    assert grouped(lib, XWT, None) == INVALID
    for form in (XWT, XW, XTW):
        need = lib.sky_grouped_gemm_workspace_bytes(form, s, F32 if form == XTW else BF)
        for i in range(4):
            assert grouped(lib, form, s, put([AT] * 4, i, None)) == INVALID
        assert grouped(lib, form, s, put([AT] * 4, 0, HALF)) == INVALID
        for i in (1, 2, 3):
            assert grouped(lib, form, s, put([AT] * 4, i, C.c_void_p((1 << 20) + 8))) == UNSUPPORTED
        assert grouped(lib, form, s, ws=None) == INVALID
        assert grouped(lib, form, s, ws=C.c_void_p((1 << 20) + 8)) == INVALID
        assert grouped(lib, form, s, n=need - 1) == INVALID
        assert grouped(lib, form, s, epi=4) == INVALID
        assert grouped(lib, form, s, out=7) == INVALID
        assert grouped(lib, form, s, out=BF if form == XTW else F32) == UNSUPPORTED
        assert grouped(lib, form, s, status=HALF) == INVALID
    assert grouped(lib, XWT, s, epi=L.SKY_EPI_BIAS_GELU, bias=AT) == INVALID  # no aux_out
    assert grouped(lib, XWT, s, epi=L.SKY_EPI_BIAS_GELU, aux_out=BYTE) == INVALID
    assert grouped(lib, XWT, s, epi=L.SKY_EPI_BIAS_GELU, aux_out=HALF) == UNSUPPORTED
    assert grouped(lib, XWT, s, bias=BYTE) == INVALID
    assert grouped(lib, XW, s, epi=L.SKY_EPI_GELU_BWD) == INVALID  # no aux
    assert grouped(lib, XW, s, epi=L.SKY_EPI_GELU_BWD, aux=HALF) == UNSUPPORTED
    for form in (XW, XTW):
        assert grouped(lib, form, s, bias=AT) == UNSUPPORTED
        assert grouped(lib, form, s, epi=L.SKY_EPI_BIAS_GELU, aux_out=AT) == UNSUPPORTED
    for form in (XWT, XTW):
        assert grouped(lib, form, s, epi=L.SKY_EPI_GELU_BWD, aux=AT) == UNSUPPORTED
    f = grouped_shape(dtype=F32)
    for i in range(4):
        assert grouped(lib, XWT, f, put([AT] * 4, i, HALF), out=F32) == INVALID
    assert grouped(lib, XWT, f, out=BF) == UNSUPPORTED
    for i in range(3):
        assert lib.sky_grouped_column_sum(s, *put([AT] * 3, i, None), None, None) == INVALID
        assert lib.sky_grouped_column_sum(s, *put([AT] * 3, i, BYTE), None, None) == INVALID
    assert lib.sky_grouped_column_sum(s, *[AT] * 3, HALF, None) == INVALID
    assert lib.sky_grouped_column_sum(None, *[AT] * 3, None, None) == INVALID


# --------------------------------------------------------------------- AdamW
def config(**kw):
    base = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, grad_dtype=F32,
                states=L.SKY_STATE_8BIT)
    base.update(kw)
    return L.SkyAdamwConfig(**base)


def tensor(**kw):
    base = dict(w=AT, g=AT, m=AT, v=AT, m_scale=AT, v_scale=AT, p=AT, n=10, decay=1)
    base.update(kw)
    return L.SkyAdamwTensor(**base)


NAN, INF = float("nan"), float("inf")
CONFIG_REFUSED = [dict(lr=-1e-9), dict(lr=NAN), dict(lr=INF), dict(beta1=-0.1), dict(beta1=1.0), dict(beta1=NAN),
                  dict(beta2=1.0), dict(beta2=-1e-9), dict(eps=0.0), dict(eps=1e-39), dict(eps=-1.0), dict(eps=INF), dict(eps=NAN),
                  dict(weight_decay=-0.1), dict(weight_decay=NAN), dict(step=0), dict(step=-5), dict(grad_dtype=2),
                  dict(states=2), dict(states=-1)]
TENSOR_REFUSED = [(dict([(n, None)]), INVALID) for n in ("w", "g", "m", "v", "m_scale", "v_scale")] + \
    [(dict([(n, HALF)]), INVALID) for n in ("w", "g", "m_scale", "v_scale")] + \
    [(dict(p=BYTE), INVALID), (dict(n=0), INVALID), (dict(n=-1), INVALID), (dict(decay=2), INVALID),
     (dict(n=(1 << 40) + 1), UNSUPPORTED)]


@pytest.mark.parametrize("bad", CONFIG_REFUSED, ids=str)
def test_adamw_refuses_settings(lib, bad):
    ts = (L.SkyAdamwTensor * 1)(tensor())
    assert lib.sky_adamw_step(config(**bad), ts, 1, None, None) == INVALID
    assert L.last_error()


@pytest.mark.parametrize("bad,status", TENSOR_REFUSED, ids=str)
def test_adamw_refuses_tensors(lib, bad, status):
    ts = (L.SkyAdamwTensor * 2)(tensor(), tensor(**bad))
    assert lib.sky_adamw_step(config(), ts, 2, None, None) == status
    assert "tensor 1" in L.last_error()


def test_adamw_refuses_arguments(lib):
    ts = (L.SkyAdamwTensor * 1)(tensor())
    assert lib.sky_adamw_step(None, ts, 1, None, None) == INVALID
    assert lib.sky_adamw_step(config(), None, 1, None, None) == INVALID
    assert lib.sky_adamw_step(config(), ts, 0, None, None) == INVALID
    assert lib.sky_adamw_step(config(), ts, 1, HALF, None) == INVALID
    wide = (L.SkyAdamwTensor * 1)(tensor(m=HALF))  # moments in 32 bits want their grid
    assert lib.sky_adamw_step(config(states=L.SKY_STATE_FP32), wide, 1, None, None) == INVALID
    many = (L.SkyAdamwTensor * 3)(*[tensor(n=1 << 40)] * 3)
    assert lib.sky_adamw_step(config(), many, 3, None, None) == UNSUPPORTED
