"""Rows to the experts and back, forward and backward, against float64: tokens without rows,
choices without one, odd widths, up to 32 choices, places out of range; what no choice names stays."""
import ctypes as C

import numpy as np
import pytest

from oracle import experts_f64 as ORC
from paper_2202_11836_gb300 import _lib as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": (torch.bfloat16, L.SKY_DTYPE_BF16, 2.0 ** -8), "fp32": (torch.float32, L.SKY_DTYPE_FP32, 2.0 ** -24)}
MARK = -77.0


def P(t):
    return C.c_void_p(int(t.data_ptr()))


def stream():
    return C.c_void_p(int(torch.cuda.current_stream().cuda_stream))


def f64(t):
    return t.double().cpu().numpy()


class Case:
    def __init__(self, tokens, top_k, width, dtype, share=0.2):
        g = torch.Generator(device="cuda").manual_seed(tokens * 31 + width)
        self.t, code, self.half_step = TYPES[dtype]
        n = tokens * top_k
        self.tokens, self.top_k, self.width, self.n = tokens, top_k, width, n
        normal = lambda *s: torch.randn(*s, device="cuda", generator=g).to(self.t)  # noqa: E731
        self.x, self.dy, self.rows = normal(tokens, width), normal(tokens, width), normal(n, width)
        row = torch.randperm(n, device="cuda", generator=g).int().view(tokens, top_k)
        gone = torch.rand(tokens, top_k, device="cuda", generator=g) < share
        if tokens > 1:
            gone[1] = True
        row[gone] = torch.tensor([-1, -5, n, 2 ** 31 - 1, -2 ** 31], device="cuda", dtype=torch.int32)[
            torch.arange(int(gone.sum()), device="cuda") % 5]
        self.row, self.live = row, (~gone).cpu().numpy()
        self.plain = np.where(self.live, row.cpu().numpy(), -1)
        self.weight = torch.rand(tokens, top_k, device="cuda", generator=g)
        self.rows[torch.tensor(np.setdiff1d(np.arange(n), self.plain[self.live]), device="cuda")] = torch.nan  # nobody's
        self.shape = L.SkyRowsShape(tokens, top_k, width, code)

    def room(self, rows):
        return torch.full((rows + 1, self.width), MARK, device="cuda", dtype=self.t)

    def near(self, got, want, size, roundings):
        bound = self.half_step * np.abs(want) + roundings * 2.0 ** -24 * size
        assert (np.abs(f64(got) - want) <= bound).all()

    def run(self):
        n, t, s = self.n, self.tokens, stream()
        out = [self.room(n), self.room(t), self.room(t), self.room(n)]
        dw = torch.full((t * self.top_k + 4,), MARK, device="cuda")
        L.call("sky_dispatch_fwd", self.shape, P(self.x), P(self.row), P(out[0]), s)
        L.call("sky_dispatch_bwd", self.shape, P(self.rows), P(self.row), P(out[1]), s)
        L.call("sky_combine_fwd", self.shape, P(self.rows), P(self.row), P(self.weight), P(out[2]), s)
        L.call("sky_combine_bwd", self.shape, P(self.rows), P(self.dy), P(self.row), P(self.weight), P(out[3]), P(dw), s)
        torch.cuda.synchronize()
        assert all(bool((o[-1] == MARK).all()) for o in out) and bool((dw[-4:] == MARK).all())
        return [o[:-1] for o in out] + [dw[:-4].view(t, self.top_k)]

    def check(self, rows, dx, y, drows, dw):
        mark = np.full((self.n, self.width), MARK)
        r = np.nan_to_num(f64(self.rows))
        assert np.array_equal(f64(rows), ORC.dispatch(f64(self.x), self.plain, mark))
        ones, w = np.ones(self.plain.shape), f64(self.weight)
        self.near(dx, ORC.combine(r, self.plain, ones), ORC.combine(np.abs(r), self.plain, ones), self.top_k)
        self.near(y, ORC.combine(r, self.plain, w), ORC.combine(np.abs(r), self.plain, w), self.top_k)
        want, want_dw = ORC.combine_backward(r, f64(self.dy), self.plain, w, mark)
        self.near(drows, want, np.abs(want), 1)
        size = ORC.combine_backward(np.abs(r), np.abs(f64(self.dy)), self.plain, w, mark)[1]
        # a dot product: a lane's share one after the other, five more additions
        assert (np.abs(f64(dw) - want_dw) <= (self.width / 32 + 16) * 2.0 ** -24 * size).all()
        assert not f64(dw)[~self.live].any()


@pytest.mark.parametrize("tokens,top_k,width", [(1, 1, 8), (1, 2, 1024), (2, 3, 520), (16, 2, 768), (5, 32, 72), (33, 4, 2048),
                                                (7, 5, 64), (301, 6, 264), (64, 9, 1032)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows(tokens, top_k, width, dtype):
    c = Case(tokens, top_k, width, dtype)
    c.check(*c.run())


def test_every_choice_gone():
    c = Case(9, 2, 64, "bf16", share=2.0)
    c.check(*c.run())


def test_gradient_in_the_rows_place():
    c = Case(50, 4, 256, "bf16")
    want = c.run()
    drows, dw = c.rows.clone(), torch.empty(50, 4, device="cuda")
    L.call("sky_combine_bwd", c.shape, P(drows), P(c.dy), P(c.row), P(c.weight), P(drows), P(dw), stream())
    live = torch.tensor(c.plain[c.live], device="cuda")
    assert torch.equal(drows[live], want[3][live]) and torch.equal(dw, want[4])


def test_infinities_stay_with_their_token():
    c = Case(20, 2, 64, "fp32", share=0.0)
    c.row[:] = torch.arange(40, device="cuda", dtype=torch.int32).view(20, 2)
    c.rows = torch.ones(40, 64, device="cuda")
    c.rows[6] = torch.inf
    y = c.room(20)
    L.call("sky_combine_fwd", c.shape, P(c.rows), P(c.row), P(c.weight), P(y), stream())
    assert bool(torch.isinf(y[3]).all()) and bool(torch.isfinite(y[:3]).all()) and bool(torch.isfinite(y[4:]).all())


def test_far_rows():
    """Offsets past 2^32 bytes."""
    tokens, top_k, width = 1 << 17, 2, 1 << 14
    x = torch.randn(1024, width, device="cuda").to(torch.bfloat16).repeat(tokens // 1024, 1)
    row = torch.randperm(tokens * top_k, device="cuda").int().view(tokens, top_k)
    rows = torch.empty(tokens * top_k, width, device="cuda", dtype=torch.bfloat16)
    shape = L.SkyRowsShape(tokens, top_k, width, L.SKY_DTYPE_BF16)
    L.call("sky_dispatch_fwd", shape, P(x), P(row), P(rows), stream())
    at = torch.tensor([0, 1, 77, tokens // 2, tokens - 1], device="cuda")
    for c in range(top_k):
        assert torch.equal(rows[row[at, c].long()], x[at])
    dx = torch.empty_like(x)
    L.call("sky_dispatch_bwd", shape, P(rows), P(row), P(dx), stream())
    assert torch.equal(dx[at], 2 * x[at])
