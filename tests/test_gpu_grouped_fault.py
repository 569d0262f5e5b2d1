"""Waits of the grouped products that run out, without a GPU fault: the producers leave out their copies, and
every consumer gives up after the limit, reports it, stores nothing of the tiles concerned and leaves.  The
same call then gives what it gave before."""
import ctypes as C

import pytest

from paper_2202_11836_gb300 import _lib as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LIMIT = 20_000_000  # ns
MARK = -7.0
XWT, XW, XTW = L.SKY_GEMM_XWT, L.SKY_GEMM_XW, L.SKY_GEMM_XTW


def P(t):
    return None if t is None else C.c_void_p(int(t.data_ptr()))


# By kernel on an SM count of about 150: pairs (more tiles than a decoder's), few rows (unsplit: many tiles; split:
# few tiles and a long sum), weight gradients by pairs (over 76 tiles of 128 x 128) and of few tiles; sizes that
# are and are not multiples of 16 rows, whose last blocks are cleared or not
CASES = [
    ("pairs", XWT, L.SKY_EPI_STORE, [300, 77], 1024, 256), ("pairs", XWT, L.SKY_EPI_BIAS_GELU, [300, 77], 1024, 256),
    ("pairs", XW, L.SKY_EPI_STORE, [300, 77], 512, 1024), ("pairs", XW, L.SKY_EPI_GELU_BWD, [300, 77], 512, 1024),
    ("few", XWT, L.SKY_EPI_STORE, [9, 3, 30], 8192, 512), ("few split", XWT, L.SKY_EPI_BIAS_GELU, [9, 3], 256, 2048),
    ("few split", XW, L.SKY_EPI_GELU_BWD, [5], 2048, 256),
    ("gradient pairs", XTW, L.SKY_EPI_STORE, [700, 33], 1024, 1024), ("gradient pairs", XTW, L.SKY_EPI_STORE, [704, 64], 1024, 1024),
    ("gradient few", XTW, L.SKY_EPI_STORE, [3001, 5], 256, 128), ("gradient few", XTW, L.SKY_EPI_STORE, [1024, 512], 256, 256),
]


# 2: of a sum that is split, only the last part's copies are left out
@pytest.mark.parametrize("name,form,epi,sizes,out,in_,skip", [c + (s,) for c in CASES for s in ((1,) if "pairs" in c[0] else (1, 2))],
                         ids=lambda v: v if isinstance(v, str) else None)
def test_waits_that_run_out(name, form, epi, sizes, out, in_, skip):
    g = torch.Generator(device="cuda").manual_seed(sum(sizes) + out)
    rows, e = sum(sizes), len(sizes)
    normal = lambda *s, t=torch.bfloat16: torch.randn(*s, device="cuda", generator=g).to(t)  # noqa: E731
    a = normal(rows, in_ if form == XWT else out)
    b = normal(rows, in_) if form == XTW else normal(e, out, in_)
    width = out if form == XWT else in_
    bias, aux = (normal(e, out) if form == XWT else None), (normal(rows, in_, t=torch.float16) if epi == L.SKY_EPI_GELU_BWD else None)
    offset = torch.tensor([0] + [sum(sizes[:i + 1]) for i in range(e)], dtype=torch.int32, device="cuda")
    c = torch.empty(*((e, out, in_) if form == XTW else (rows, width)), device="cuda", dtype=torch.float32 if form == XTW else torch.bfloat16)
    slope = torch.empty(rows, width, device="cuda", dtype=torch.float16) if epi == L.SKY_EPI_BIAS_GELU else None
    shape = L.SkyGroupedShape(e, rows, out, in_, L.SKY_DTYPE_BF16)
    code = L.SKY_DTYPE_FP32 if form == XTW else L.SKY_DTYPE_BF16
    n = L.lib().sky_grouped_gemm_workspace_bytes(form, shape, code)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def go():
        c.fill_(MARK)
        if slope is not None:
            slope.fill_(MARK)
        status.zero_()
        L.call("sky_grouped_gemm", form, shape, P(offset), P(a), P(b), P(c), code, epi, P(bias), P(aux), P(slope), P(ws), n, P(status),
               C.c_void_p(int(torch.cuda.current_stream().cuda_stream)))
        torch.cuda.synchronize()
        return status.item()

    assert go() == 0
    want, want_slope = c.clone(), None if slope is None else slope.clone()
    assert not bool((c == MARK).all())
    L.lib().sky_debug_gemm_fault(LIMIT, skip)
    try:
        assert go() == 2
    finally:
        L.lib().sky_debug_gemm_fault(0, 0)
    assert bool((c == MARK).all()) and (slope is None or bool((slope == MARK).all()))
    assert go() == 0
    assert torch.equal(c, want) and (slope is None or torch.equal(slope, want_slope))


def test_a_limit_is_of_a_wait_not_of_a_call():
    """A weight gradient of several limits' length: the rows behind a group's last are cleared by a warp that has
    nothing to do before, here for the 1.2 ms that a pair takes for a tile of the first group."""
    sizes, n = [262144, 7], 2560  # 100 tiles of 256 x 256 a group: most pairs take one of either
    g = torch.Generator(device="cuda").manual_seed(3)
    a, b = (torch.randn(sum(sizes), n, device="cuda", generator=g, dtype=torch.bfloat16) for _ in range(2))
    offset = torch.tensor([0, sizes[0], sum(sizes)], dtype=torch.int32, device="cuda")
    c = torch.full((2, n, n), MARK, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    shape = L.SkyGroupedShape(2, sum(sizes), n, n, L.SKY_DTYPE_BF16)
    ws = torch.empty(L.lib().sky_grouped_gemm_workspace_bytes(XTW, shape, L.SKY_DTYPE_FP32), dtype=torch.uint8, device="cuda")
    L.lib().sky_debug_gemm_fault(300_000, 0)
    try:
        L.call("sky_grouped_gemm", XTW, shape, P(offset), P(a), P(b), P(c), L.SKY_DTYPE_FP32, L.SKY_EPI_STORE, None, None, None,
               P(ws), ws.numel(), P(status), C.c_void_p(int(torch.cuda.current_stream().cuda_stream)))
        torch.cuda.synchronize()
    finally:
        L.lib().sky_debug_gemm_fault(0, 0)
    assert status.item() == 0
    lo = sizes[0]
    want = a[lo:].double().T @ b[lo:].double()
    # seven products, each addition off by up to 2^-23 of the sum of magnitudes
    size = a[lo:].double().abs().T @ b[lo:].double().abs()
    assert bool(((c[1].double() - want).abs() <= 8 * 2.0 ** -23 * size).all())
    part = slice(1000, 1300)
    want = a[:lo, part].double().T @ b[:lo, part].double()
    # parts of 512 rows, each cut off 32 times by up to 2^-23, and 512 of them added with half of that
    size = a[:lo, part].double().abs().T @ b[:lo, part].double().abs()
    assert bool(((c[0, part, part].double() - want).abs() <= (32 + 256) * 2.0 ** -23 * size).all())
