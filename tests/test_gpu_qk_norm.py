"""Norm of every query and key head with its rotation, forward and backward, against
float64: head dims with idle lanes, odd rows, rows wider than their heads, one kind of
head, far and negative positions, in place, captured; what lies behind the heads stays."""
import ctypes as C

import numpy as np
import pytest

from oracle import heads_f64 as ORC
from paper_2202_11836_gb300 import _lib as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS, THETA = 1e-6, 10000.0
ROT = {"none": L.SKY_ROTATE_NONE, "halves": L.SKY_ROTATE_HALVES, "pairs": L.SKY_ROTATE_PAIRS}
TYPES = {"bf16": (torch.bfloat16, L.SKY_DTYPE_BF16, 2.0 ** -8), "fp32": (torch.float32, L.SKY_DTYPE_FP32, 0.0)}
MARK = -77.0  # of memory that no call may write


def P(t):
    return None if t is None else C.c_void_p(int(t.data_ptr()))


def stream():
    return C.c_void_p(int(torch.cuda.current_stream().cuda_stream))


def f64(t):
    return t.double().cpu().numpy()


class Case:
    def __init__(self, rows, a, k, dim, dtype, rotation, behind=0, gains=True, far=True, seed=0, eps=EPS):
        g = torch.Generator(device="cuda").manual_seed(1000 * rows + 10 * a + dim + seed)
        self.rows, self.a, self.k, self.dim, self.dtype, self.rotation = rows, a, k, dim, dtype, rotation
        self.eps = eps
        self.t, code, self.half_step = TYPES[dtype]
        self.width = (a + k) * dim
        self.ld = self.width + behind
        normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        # heads of very different sizes: the norm takes each for itself
        size = 10.0 ** torch.randint(-3, 3, (rows, a + k, 1), device="cuda", generator=g)
        self.x = torch.full((rows, self.ld), MARK, device="cuda", dtype=self.t)
        self.x[:, :self.width] = (normal(rows, a + k, dim) * size).view(rows, -1).to(self.t)
        self.dy = (0.1 * normal(rows, self.width)).to(self.t)
        self.gain = [(1 + 0.2 * normal(dim)).to(self.t) if gains else None for _ in range(2)]
        hi = 1 << 31 if far else 2048
        self.pos = torch.randint(-hi if far else 0, hi, (rows,), device="cuda", generator=g).to(torch.int32)
        self.shape = L.SkyQkNormShape(rows, a, k, dim, code, self.ld, self.width, eps, ROT[rotation], THETA)

    def forward(self, y=None):
        y = torch.full((self.rows, self.width), MARK, device="cuda", dtype=self.t) if y is None else y
        L.call("sky_qk_norm_fwd", self.shape, P(self.x), P(self.gain[0]), P(self.gain[1]),
               P(self.pos) if self.rotation != "none" else None, P(y), stream())
        return y

    def backward(self, dx=None, ws=None):
        n = L.lib().sky_qk_norm_bwd_workspace_bytes(self.shape)
        assert n > 0
        ws = torch.full((n + 64,), 0x7f, dtype=torch.uint8, device="cuda") if ws is None else ws
        dx = torch.full((self.rows, self.ld), MARK, device="cuda", dtype=self.t) if dx is None else dx
        dg = [torch.full((self.dim + 4,), MARK, device="cuda") for _ in range(2)]
        L.call("sky_qk_norm_bwd", self.shape, P(self.x), P(self.dy), P(self.gain[0]), P(self.gain[1]),
               P(self.pos) if self.rotation != "none" else None, P(dx), P(dg[0]), P(dg[1]), P(ws), n, stream())
        torch.cuda.synchronize()
        assert bool((ws[n:] == 0x7f).all()) and all(bool((d[self.dim:] == MARK).all()) for d in dg)
        return dx, dg[0][:self.dim], dg[1][:self.dim]

    def gain64(self):
        rows = [np.ones(self.dim) if g is None else f64(g) for g in self.gain]
        return np.concatenate([np.tile(rows[0], (self.a, 1)), np.tile(rows[1], (self.k, 1))])

    def want(self):
        x = f64(self.x[:, :self.width]).reshape(self.rows, -1, self.dim)
        pos = f64(self.pos)
        y = ORC.head_norm(x, self.gain64(), pos, self.eps, self.rotation, THETA)
        dx, terms = ORC.head_norm_backward(x, f64(self.dy).reshape(x.shape), self.gain64(), pos, self.eps, self.rotation,
                                           THETA)
        return x, y, dx, terms

    def check_forward(self, y):
        """Each value: a dozen fp32 roundings (2^-24 each) of products not above the pair's
        size, the angle's (2^-22 radians), the mean's (D of 2^-24), then the type's half step."""
        x, want, _, _ = self.want()
        got = f64(y).reshape(want.shape)
        top = np.abs(want).max(-1, keepdims=True) * 2 ** 0.5
        bound = self.half_step * np.abs(want) + (self.dim + 32) * 2.0 ** -24 * top
        if self.rotation != "none":  # frequencies of both sides (an ulp of pow each, 2 pi, a quotient), pos * freq
            bound = bound + np.abs(f64(self.pos))[:, None, None] * 2.0 ** -50 * top
        assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())

    def check_backward(self, dx, dq, dk):
        x, _, want, terms = self.want()
        got = f64(dx).reshape(want.shape)
        rms = np.sqrt((x * x).mean(-1, keepdims=True) + self.eps)
        dz = np.abs(f64(self.dy)).reshape(x.shape).max(-1, keepdims=True) * 2 ** 0.5
        h = dz * np.abs(self.gain64()).max(-1)[None, :, None]
        # dx = (h - xhat m) / rms, m a mean of D products; xhat is at most sqrt(D)
        top = h / rms * (1 + (np.abs(x / rms) * np.abs(x / rms).mean(-1, keepdims=True)))
        bound = self.half_step * np.abs(want) + (2 * self.dim + 64) * 2.0 ** -24 * top
        turned = np.abs(f64(self.pos))[:, None, None] * 2.0 ** -50 if self.rotation != "none" else 0.0
        bound = bound + turned * top
        assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
        # gain gradients: sums of fp32 terms (errors as above), added in partial sums of a
        # length not above the rows; each rounding is of a part of the sum of magnitudes
        size = dz * np.abs(x / rms)
        for part, d in ((slice(0, self.a), dq), (slice(self.a, None), dk)):
            t, s = terms[:, part].sum((0, 1)), size[:, part].sum((0, 1))
            bound = (self.rows + self.dim + 96) * 2.0 ** -24 * s + (turned * size[:, part]).sum((0, 1)) + 1e-30
            assert (np.abs(f64(d) - t) <= bound).all(), float((np.abs(f64(d) - t) / bound).max())


SHAPES = [
    # rows, query heads, key heads, dim, values behind the heads
    (2, 12, 12, 64, 0), (128, 4, 4, 64, 0), (129, 8, 8, 64, 8), (40, 3, 3, 96, 0), (1, 1, 1, 64, 0), (1, 12, 12, 64, 768), (16, 12, 4, 64, 256), (3, 1, 0, 16, 8), (5, 0, 3, 32, 0),
    (7, 17, 9, 48, 16), (33, 9, 3, 80, 0), (101, 12, 4, 96, 384), (64, 6, 6, 128, 0), (19, 5, 2, 176, 0),
    (9, 3, 2, 256, 32), (700, 16, 16, 64, 1024), (5001, 2, 1, 64, 0), (3000, 33, 1, 32, 0), (1, 300, 300, 256, 0),
]


@pytest.mark.parametrize("rotation", ["halves", "pairs", "none"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_norm(shape, dtype, rotation):
    c = Case(*shape[:4], dtype, rotation, behind=shape[4])
    before = c.x.clone()
    y = c.forward()
    dx, dq, dk = c.backward()
    torch.cuda.synchronize()
    assert torch.equal(before, c.x)
    c.check_forward(y)
    assert bool((dx[:, c.width:] == MARK).all())  # behind the heads
    c.check_backward(dx[:, :c.width], dq, dk)
    again = c.backward()
    assert all(torch.equal(u, v) for u, v in zip((dx, dq, dk), again))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_without_gains_and_in_place(dtype):
    c = Case(77, 6, 3, 64, dtype, "halves", behind=64, gains=False, far=False)
    dx, dq, dk = c.backward()
    c.check_backward(dx[:, :c.width], dq, dk)
    y = c.forward()
    c.check_forward(y)
    # forward over its input: rows as far apart, the values behind stay
    c.shape.ldy = c.ld
    tail = c.x[:, c.width:].clone()
    c.forward(c.x)
    torch.cuda.synchronize()
    assert torch.equal(c.x[:, :c.width], y) and torch.equal(c.x[:, c.width:], tail)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_gradient_over_its_inputs(dtype):
    for where in ("dy", "x"):
        c = Case(50, 4, 4, 96, dtype, "pairs")
        dx, dq, dk = c.backward()
        over = c.backward(dx=getattr(c, where))
        assert torch.equal(over[0], dx) and torch.equal(over[1], dq) and torch.equal(over[2], dk)


def test_zero_heads_and_no_gain_gradients():
    """A head of zeros gives zeros (eps keeps the norm finite); gain gradients are optional."""
    c = Case(10, 3, 2, 64, "bf16", "halves")
    c.x[4, :64] = 0
    y = c.forward()
    assert not bool(y[4, :64].any()) and bool(torch.isfinite(y).all())
    c.check_forward(y)
    n = L.lib().sky_qk_norm_bwd_workspace_bytes(c.shape)
    ws, dx = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(c.x)
    L.call("sky_qk_norm_bwd", c.shape, P(c.x), P(c.dy), None, None, P(c.pos), P(dx), None, None, P(ws), n, stream())
    torch.cuda.synchronize()
    assert bool(torch.isfinite(dx[:, :c.width]).all())


@pytest.mark.parametrize("shape", [(40, 3, 1, 64), (5000, 9, 2, 32), (700, 5, 5, 96), (300, 17, 9, 64)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_eps_of_zero(shape, dtype):
    """Lanes without a head of their own have zeros to norm, which nothing may take in."""
    c = Case(*shape, dtype, "halves", far=False, eps=0.0)
    y = c.forward()
    dx, dq, dk = c.backward()
    for t in (y, dx, dq, dk):
        assert bool(torch.isfinite(t).all())
    c.check_forward(y)
    c.check_backward(dx, dq, dk)


def test_bad_values_stay_in_their_heads():
    c = Case(40, 5, 3, 64, "bf16", "pairs")
    y, (dx, _, _) = c.forward(), c.backward()
    c.x[7, 64 * 2 + 5], c.x[30, 64 * 6] = float("nan"), float("inf")
    z, (ez, _, _) = c.forward(), c.backward()
    keep = torch.ones(40, 8, 64, dtype=torch.bool, device="cuda")
    keep[7, 2], keep[30, 6] = False, False
    keep = keep.view(40, -1)
    assert torch.equal(y[keep], z[keep]) and torch.equal(dx[keep], ez[keep])
    assert not bool(torch.isfinite(z.view(40, 8, 64)[7, 2]).any())


def test_captured_and_replayed():
    c = Case(123, 4, 2, 64, "bf16", "halves", behind=128)
    n = L.lib().sky_qk_norm_bwd_workspace_bytes(c.shape)
    ws, y, dx = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(c.dy), torch.empty_like(c.x)
    dg = torch.empty(2, 64, device="cuda")

    def both():
        c.forward(y)
        L.call("sky_qk_norm_bwd", c.shape, P(c.x), P(c.dy), P(c.gain[0]), P(c.gain[1]), P(c.pos), P(dx), P(dg[0]),
               P(dg[1]), P(ws), n, stream())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    c.x[:, :c.width].mul_(-0.5)
    c.pos.add_(3)
    graph.replay()
    torch.cuda.synchronize()
    want_y = c.forward()
    want = c.backward()
    torch.cuda.synchronize()
    assert torch.equal(y, want_y) and torch.equal(dx[:, :c.width], want[0][:, :c.width])
    assert torch.equal(dg[0], want[1]) and torch.equal(dg[1], want[2])
