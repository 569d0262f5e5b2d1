"""Products grouped by expert in their three forms, with every epilogue, against float64: groups of
one row and of none, sizes off every tile, rows that belong to nobody, what lies beside the outputs."""
import ctypes as C

import numpy as np
import pytest

from oracle import experts_f64 as ORC
from paper_2202_11836_gb300 import _lib as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": (torch.bfloat16, L.SKY_DTYPE_BF16, 2.0 ** -8, torch.float16, 2.0 ** -11),
         "fp32": (torch.float32, L.SKY_DTYPE_FP32, 2.0 ** -24, torch.float32, 2.0 ** -24)}
FORM = {"xwt": L.SKY_GEMM_XWT, "xw": L.SKY_GEMM_XW, "xtw": L.SKY_GEMM_XTW}
EPI = {"store": L.SKY_EPI_STORE, "bias": L.SKY_EPI_STORE, "gelu": L.SKY_EPI_BIAS_GELU, "gelu_bwd": L.SKY_EPI_GELU_BWD}
MARK = -77.0


def P(t):
    return None if t is None else C.c_void_p(int(t.data_ptr()))


def stream():
    return C.c_void_p(int(torch.cuda.current_stream().cuda_stream))


def f64(t):
    return t.double().cpu().numpy()


class Case:
    """first: rows before the first group; behind: rows after the last.  Both hold NaN."""

    def __init__(self, form, sizes, out, in_, dtype, epi="store", first=0, behind=0, seed=0):
        g = torch.Generator(device="cuda").manual_seed(sum(sizes) * 13 + out + seed)
        self.form, self.sizes, self.out, self.in_, self.epi = form, sizes, out, in_, epi
        self.t, self.code, self.half_step, self.slope_t, self.slope_half = TYPES[dtype]
        self.offset = np.concatenate([[0], np.cumsum(sizes)]) + first
        self.rows = max(1, int(self.offset[-1]) + behind)
        e = len(sizes)
        normal = lambda *s, std=1.0, t=None: (torch.randn(*s, device="cuda", generator=g) * std).to(t or self.t)  # noqa: E731
        self.a = normal(self.rows, in_ if form == "xwt" else out)
        self.b = normal(self.rows, in_) if form == "xtw" else normal(e, out, in_, std=in_ ** -0.5)
        self.bias = normal(e, out, std=0.5) if epi == "bias" or (epi == "gelu" and seed % 2 == 0) else None
        self.width = out if form == "xwt" else in_
        self.aux = normal(self.rows, in_, t=self.slope_t) if epi == "gelu_bwd" else None
        owned = torch.zeros(self.rows, dtype=torch.bool, device="cuda")
        owned[self.offset[0]:self.offset[-1]] = True
        self.a[~owned] = torch.nan
        if form == "xtw":
            self.b[~owned] = torch.nan
        if self.aux is not None:
            self.aux[~owned] = torch.nan
        self.d_offset = torch.tensor(self.offset, dtype=torch.int32, device="cuda")
        self.shape = L.SkyGroupedShape(e, self.rows, out, in_, self.code)

    def workspace(self):
        n = L.lib().sky_grouped_gemm_workspace_bytes(FORM[self.form], self.shape, self.out_code())
        return n, torch.full((n + 64,), 0x7f, dtype=torch.uint8, device="cuda")

    def out_code(self):
        return L.SKY_DTYPE_FP32 if self.form == "xtw" else self.code

    def room(self):
        if self.form == "xtw":
            return torch.full((len(self.sizes) * self.out * self.in_ + 64,), MARK, device="cuda"), None
        c = torch.full((self.rows * self.width + 64,), MARK, device="cuda", dtype=self.t)
        slope = torch.full((self.rows * self.width + 64,), MARK, device="cuda", dtype=self.slope_t) if self.epi == "gelu" else None
        return c, slope

    def call(self, c, slope, n, ws, status=None):
        L.call("sky_grouped_gemm", FORM[self.form], self.shape, P(self.d_offset), P(self.a), P(self.b), P(c), self.out_code(),
               EPI[self.epi], P(self.bias), P(self.aux), P(slope), P(ws), n, P(status), stream())

    def run(self, status=None):
        n, ws = self.workspace()
        c, slope = self.room()
        self.call(c, slope, n, ws, status)
        torch.cuda.synchronize()
        assert bool((ws[n:] == 0x7f).all()) and bool((c[-64:] == MARK).all()) and (slope is None or bool((slope[-64:] == MARK).all()))
        return c[:-64], None if slope is None else slope[:-64]

    def check(self, c, slope):
        a, b = np.nan_to_num(f64(self.a)), np.nan_to_num(f64(self.b))
        z = ORC.by_group(self.form, a, b, self.offset)
        # fp32 sums of exact products: an addition rounds (or, on the tensor cores, cuts off) by up to 2^-23 of
        # a partial sum, none above the sum of magnitudes; there are at most as many as terms
        size = ORC.by_group(self.form, np.abs(a), np.abs(b), self.offset)
        terms = {"xwt": self.in_, "xw": self.out, "xtw": max(self.sizes)}[self.form]
        err = (terms + 4) * 2.0 ** -23 * size
        if self.form == "xtw":
            got = f64(c).reshape(z.shape)
            assert (np.abs(got - z) <= err + 2.0 ** -24 * np.abs(z)).all(), np.abs(got - z).max()
            return
        owned = slice(self.offset[0], self.offset[-1])
        got = f64(c).reshape(z.shape)
        rest = np.ones(self.rows, bool)
        rest[owned] = False
        assert (got[rest] == MARK).all()
        if self.bias is not None:
            z = z + np.repeat(f64(self.bias), self.sizes, 0) if self.rows == sum(self.sizes) else self.with_bias(z)
        if self.epi == "gelu":
            # the slope of GELU is at most 1.13, its second derivative at most 0.8; erf is taken to 2.5e-5 for bf16
            # (half of that in the distribution's place), to 1e-6 for fp32, the hardware's exponential included
            near = 4e-5 if self.t == torch.bfloat16 else 2e-6
            y, s = ORC.gelu(z[owned]), ORC.gelu_slope(z[owned])
            sl = f64(slope).reshape(z.shape)
            assert (sl[rest] == MARK).all()
            ok = np.abs(got[owned] - y) <= 1.13 * err[owned] + near * (1 + np.abs(z[owned])) + self.half_step * (np.abs(y) + near)
            assert ok.all(), np.abs(got[owned] - y).max()
            ok = np.abs(sl[owned] - s) <= 0.8 * err[owned] + near * (1 + np.abs(z[owned])) + self.slope_half * (np.abs(s) + near) + 2.0 ** -25
            assert ok.all(), np.abs(sl[owned] - s).max()
            return
        if self.epi == "gelu_bwd":
            x = np.nan_to_num(f64(self.aux))
            z, err = z * x, err * np.abs(x) + 2.0 ** -24 * np.abs(z * x)
        assert (np.abs(got - z)[owned] <= (err + 2.0 ** -24 * np.abs(z) + self.half_step * (np.abs(z) + err))[owned]).all(), \
            np.abs(got - z)[owned].max()

    def with_bias(self, z):
        z = z.copy()
        for g in range(len(self.sizes)):
            z[self.offset[g]:self.offset[g + 1]] += f64(self.bias)[g]
        return z


KINDS = [("xwt", "store"), ("xwt", "bias"), ("xwt", "gelu"), ("xw", "store"), ("xw", "gelu_bwd"), ("xtw", "store")]
SHAPES = [
    # group sizes, out, in, rows before, rows behind
    ([1], 8, 8, 0, 0), ([3, 0, 5], 64, 64, 0, 0), ([0, 0, 2, 0], 128, 72, 3, 5), ([2, 1], 256, 1024, 0, 0),
    ([17, 64, 0, 129], 264, 136, 1, 2), ([33, 31, 32], 136, 328, 0, 1), ([300, 1, 255, 256], 512, 256, 0, 9),
    ([257], 776, 64, 7, 0), ([65] * 40, 72, 96, 0, 0), ([1000, 513], 1024, 512, 0, 0), ([128, 640, 31], 2048, 80, 0, 33),
]


@pytest.mark.parametrize("form,epi", KINDS)
@pytest.mark.parametrize("sizes,out,in_,first,behind", SHAPES, ids=lambda v: str(v) if isinstance(v, int) else f"{len(v)}g{sum(v)}")
def test_bf16(form, epi, sizes, out, in_, first, behind):
    c = Case(form, sizes, out, in_, "bf16", epi, first, behind)
    c.check(*c.run())


F32_SHAPES = [([1], 1, 1, 0, 0), ([3, 0, 5], 64, 64, 0, 0), ([2, 1], 129, 513, 0, 3), ([17, 64, 0, 129], 37, 70, 1, 2),
              ([90, 70, 55, 42], 512, 128, 0, 0), ([300, 1], 100, 1000, 0, 4), ([65] * 40, 20, 33, 0, 0)]


@pytest.mark.parametrize("form,epi", KINDS)
@pytest.mark.parametrize("sizes,out,in_,first,behind", F32_SHAPES, ids=lambda v: str(v) if isinstance(v, int) else f"{len(v)}g{sum(v)}")
def test_fp32(form, epi, sizes, out, in_, first, behind):
    c = Case(form, sizes, out, in_, "fp32", epi, first, behind)
    c.check(*c.run())


# More than 64 rows of few tiles, with sums long enough to be split: remainders of tokens, features and blocks
LONG_SUMS = [([80], 256, 1024, 0, 0), ([33, 0, 190], 136, 4104, 2, 3), ([1000, 1], 72, 1544, 0, 9), ([7, 90, 64], 520, 2048, 0, 0)]


@pytest.mark.parametrize("form,epi", [k for k in KINDS if k[0] != "xtw"])
@pytest.mark.parametrize("sizes,features,inner,first,behind", LONG_SUMS, ids=lambda v: str(v) if isinstance(v, int) else f"{len(v)}g{sum(v)}")
def test_few_tiles_with_long_sums(form, epi, sizes, features, inner, first, behind):
    out, in_ = (features, inner) if form == "xwt" else (inner, features)
    c = Case(form, sizes, out, in_, "bf16", epi, first, behind)
    c.check(*c.run())


# Weight gradients of few tiles: up to four sums of 512 rows a split, splits without rows, empty groups, both remainders
GRAD_FEW = [([5000], 128, 104, 3, 7), ([9000, 0, 4100], 256, 72, 0, 1), ([3100, 1], 2432, 120, 0, 0), ([7001], 2560, 72, 0, 0),
            ([0, 3, 1600], 40, 200, 5, 40), ([2049] + [0] * 7, 64, 192, 0, 0), ([63], 600, 600, 1, 1)]


@pytest.mark.parametrize("sizes,out,in_,first,behind", GRAD_FEW, ids=lambda v: str(v) if isinstance(v, int) else f"{len(v)}g{sum(v)}")
def test_weight_gradients_of_few_tiles(sizes, out, in_, first, behind):
    c = Case("xtw", sizes, out, in_, "bf16", "store", first, behind)
    got = c.run()[0]
    c.check(got, None)
    assert torch.equal(got, c.run()[0])


def test_weight_gradients_of_few_tiles_keep_groups_apart():
    """Infinities in a group's rows, and what the rows behind the last hold, stay out of the others' sums."""
    sizes, out, in_ = [1300, 37, 1201], 136, 200
    c = Case("xtw", sizes, out, in_, "bf16", "store", 0, 70)
    want = c.run()[0].clone()
    c.a[1300:1337] = float("inf")
    c.b[1300:1337] = 1.0
    got = c.run()[0]
    n = out * in_
    assert torch.equal(got[:n], want[:n]) and torch.equal(got[2 * n:], want[2 * n:])
    assert bool((got[n:2 * n] == float("inf")).all())


# Few rows: groups of one to more than eight rows, features that are no multiple of four, inner sizes odd, short and long
F32_FEW = [([1], 5, 3, 0, 0), ([1, 2, 3, 4, 5, 0, 7, 8, 9], 768, 768, 1, 2), ([64], 100, 640, 0, 0), ([1] * 40, 33, 129, 0, 5),
           ([25, 0, 33], 18, 1001, 0, 1), ([2, 1], 200, 5000, 0, 0), ([11], 16, 4097, 3, 0), ([4, 3], 1023, 128, 0, 57)]


@pytest.mark.parametrize("epi", ["store", "gelu"])
@pytest.mark.parametrize("sizes,out,in_,first,behind", F32_FEW, ids=lambda v: str(v) if isinstance(v, int) else f"{len(v)}g{sum(v)}")
def test_fp32_of_few_rows(epi, sizes, out, in_, first, behind):
    c = Case("xwt", sizes, out, in_, "fp32", epi, first, behind)
    c.check(*c.run())


def test_fp32_of_few_rows_keeps_groups_apart():
    """Infinities in a group's rows and weights, or in rows that none owns, stay where they are; weights off 16 bytes do too."""
    sizes, out, in_ = [5, 9, 0, 3], 70, 132
    c = Case("xwt", sizes, out, in_, "fp32", "store", 0, 4)
    want = c.run()[0].clone()
    c.a[5:14] = float("inf")
    c.a[17:] = float("nan")
    c.b[1] = float("-inf")
    got = c.run()[0]
    n = out * 5
    assert torch.equal(got[:n], want[:n]) and torch.equal(got[14 * out:], want[14 * out:])
    assert bool((got[n:14 * out] == float("-inf")).all())
    at = torch.empty(c.b.numel() + 1, device="cuda")[1:]  # 4 bytes off
    at.copy_(c.b.reshape(-1))
    c.b = at.reshape(c.b.shape)
    close = c.run()[0]
    # either order of the sum, each of fp32 products: both within (in + 1) half steps of the sum of magnitudes
    size = c.a[:5].abs().double() @ c.b[0].abs().double().T
    assert bool(((close[:n].reshape(5, out) - want[:n].reshape(5, out)).abs().double() <= 2 * (in_ + 1) * 2.0 ** -24 * size).all())


def test_gelu_without_a_bias():
    c = Case("xwt", [40, 3], 64, 128, "bf16", "gelu", seed=1)
    assert c.bias is None
    c.check(*c.run())


@pytest.mark.parametrize("form", list(FORM))
@pytest.mark.parametrize("dtype", list(TYPES))
def test_no_row_at_all(form, dtype):
    c = Case(form, [0, 0, 0], 64, 64, dtype, behind=20)
    c.check(*c.run())


@pytest.mark.parametrize("form,epi", [("xwt", "gelu"), ("xw", "gelu_bwd"), ("xtw", "store")])
def test_a_group_never_sees_another(form, epi):
    """Infinities in a group's rows and weights stay in its results."""
    sizes, out, in_ = [37, 50, 0, 61], 200, 72
    c = Case(form, sizes, out, in_, "bf16", epi)
    want = [None if x is None else x.clone() for x in c.run()]
    lo, hi = int(c.offset[1]), int(c.offset[2])
    c.a[lo:hi] = torch.inf
    if form == "xtw":
        c.b[lo:hi] = torch.nan
    else:
        c.b[1:3] = torch.nan  # (expert 2 has no row)
    got = c.run()
    for g, w in zip(got, want):
        if g is None:
            continue
        g, w = (x.view(4, -1) if form == "xtw" else x.view(c.rows, -1) for x in (g, w))
        keep = [0, 2, 3] if form == "xtw" else [i for i in range(c.rows) if not lo <= i < hi]
        assert torch.equal(g[keep], w[keep])


@pytest.mark.parametrize("form,epi", KINDS)
def test_same_bits_every_time_and_captured(form, epi):
    c = Case(form, [100, 0, 300, 29], 520, 264, "bf16", epi, behind=3)
    want = c.run()
    n, ws = c.workspace()
    out, slope = c.room()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.call(out, slope, n, ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out[:-64].view(torch.uint8), want[0].view(torch.uint8))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(out, slope, n, ws)
    # replayed with other groups: they are read when the work runs
    other = Case(form, [3, 200, 26, 200], 520, 264, "bf16", epi, behind=3)
    for x, y in zip((c.a, c.b, c.bias, c.aux, c.d_offset), (other.a, other.b, other.bias, other.aux, other.d_offset)):
        if x is not None:
            x.copy_(y)
    out.fill_(MARK)
    if slope is not None:
        slope.fill_(MARK)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    other.check(out[:-64], None if slope is None else slope[:-64])


def test_bad_offsets_are_reported_and_stay_inside():
    for form in FORM:
        for dtype in TYPES:
            c = Case(form, [20, 30, 10], 64, 64, dtype)
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            c.check(*c.run(status))
            assert status.item() == 0
            for bad in ([-5, 20, 50, 60], [0, 50, 20, 60], [0, 20, 50, 1 << 30], [-(2 ** 31), 0, 2 ** 31 - 1, 0]):
                c.d_offset.copy_(torch.tensor(bad, dtype=torch.int32))
                status.zero_()
                c.run(status)  # (checks what lies behind the outputs)
                assert status.item() == 1


SUMS = [([1], 8), ([0, 3, 0], 64), ([40, 0, 1000, 7], 776), ([5] * 70, 24), ([2000], 4096)]


@pytest.mark.parametrize("sizes,width", SUMS + [([9, 100], 13), ([33], 1)], ids=lambda v: str(v) if isinstance(v, int) else f"{len(v)}g{sum(v)}")
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shift", [0, 1])
def test_column_sums(sizes, width, dtype, shift):
    t, code = TYPES[dtype][:2]
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = sum(sizes) + 5
    x = torch.full((rows * width + shift,), float("nan"), device="cuda", dtype=t)[shift:].view(rows, width)
    x[2:2 + sum(sizes)] = torch.randn(sum(sizes), width, device="cuda", generator=g).to(t)
    offset = np.concatenate([[0], np.cumsum(sizes)]) + 2
    d = torch.tensor(offset, dtype=torch.int32, device="cuda")
    out = torch.full((len(sizes) * width + 8,), MARK, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    L.call("sky_grouped_column_sum", L.SkyGroupedShape(len(sizes), rows, width, 0, code), P(d), P(x), P(out), P(status), stream())
    assert bool((out[-8:] == MARK).all()) and status.item() == 0
    got = f64(out[:-8]).reshape(len(sizes), width)
    for i, n in enumerate(sizes):
        part = f64(x[offset[i]:offset[i + 1]])
        assert (np.abs(got[i] - part.sum(0)) <= (n / 32 + 33) * 2.0 ** -24 * np.abs(part).sum(0)).all()


def test_far_rows():
    """Offsets past 2^32 bytes: the last group's rows lie behind them."""
    rows, out, in_ = (1 << 21) + 300, 64, 2048
    for form in ("xwt", "xtw"):
        a = torch.zeros(rows, in_ if form == "xwt" else out, device="cuda", dtype=torch.bfloat16)
        b = torch.zeros(rows, in_, device="cuda", dtype=torch.bfloat16) if form == "xtw" else \
            torch.randn(2, out, in_, device="cuda").to(torch.bfloat16)
        lo = rows - 200
        a[lo:] = torch.randn(200, a.shape[1], device="cuda").to(torch.bfloat16)
        if form == "xtw":
            b[lo:] = torch.randn(200, in_, device="cuda").to(torch.bfloat16)
        offset = torch.tensor([lo - 7, lo, rows], dtype=torch.int32, device="cuda")
        shape = L.SkyGroupedShape(2, rows, out, in_, L.SKY_DTYPE_BF16)
        code = L.SKY_DTYPE_FP32 if form == "xtw" else L.SKY_DTYPE_BF16
        n = L.lib().sky_grouped_gemm_workspace_bytes(FORM[form], shape, code)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        c = torch.empty(2, out, in_, device="cuda") if form == "xtw" else torch.zeros(rows, out, device="cuda", dtype=torch.bfloat16)
        L.call("sky_grouped_gemm", FORM[form], shape, P(offset), P(a), P(b), P(c), code, 0, None, None, None, P(ws), n, None, stream())
        if form == "xtw":
            want = f64(a[lo:]).T @ f64(b[lo:])
            assert np.abs(f64(c[1]) - want).max() <= 204 * 2.0 ** -23 * (np.abs(f64(a[lo:])).T @ np.abs(f64(b[lo:]))).max()
            assert not bool(c[0].any())
        else:
            want = f64(a[lo:]) @ f64(b[1]).T
            assert (np.abs(f64(c[lo:]) - want) <= 2.0 ** -8 * np.abs(want) + 1e-2).all() and not bool(c[:lo].any())
