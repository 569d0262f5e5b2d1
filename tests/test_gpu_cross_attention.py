"""Attention over keys of another length, forward and backward, against float64: odd and
single rows on either side, heads that share keys, sequences without keys, rows inside
wider ones, infinities and NaN behind the valid keys; nothing else is written.

Bounds are element by element, from the formulas: with c = 1 / sqrt(D), u = 2^-24 and h
the type's half step,
  a score is off by (D + 8) u c sum |q k| (at most the row's largest, E), so P by a factor
    exp(+-2 E) and the exponential's and quotient's own 2^-20; the tensor cores take P
    and dS rounded to bf16, h more, and for dK and dV the log-sum-exp as two bf16 numbers,
    2^-16 of it, as they take delta;
  sums of n products add (n + 8) u of their magnitudes;
  delta is formed from the ctx that was given, rounded to the type: h sum |dctx ctx|.
"""
import ctypes as C

import numpy as np
import pytest

from oracle import heads_f64 as ORC
from paper_2202_11836_gb300 import _lib as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
TYPES = {"bf16": (torch.bfloat16, L.SKY_DTYPE_BF16, 2.0 ** -8), "fp32": (torch.float32, L.SKY_DTYPE_FP32, U)}
MARK = -77.0


def P(t):
    return None if t is None else C.c_void_p(int(t.data_ptr()))


def stream():
    return C.c_void_p(int(torch.cuda.current_stream().cuda_stream))


def f64(t):
    return t.double().cpu().numpy()


def within(got, want, bound, name):
    off = ~(np.abs(got - want) <= bound)
    at = np.unravel_index(np.argmax(off), off.shape)
    assert not off.any(), f"{name}: {off.sum()} values off, first {at}: {got[at]} for {want[at]} within {bound[at]}"


class Rows:
    """[B, S] rows of `heads` x D values at column `at` of rows of `ld`, a few rows behind."""

    def __init__(self, B, S, heads, D, ld, at, t):
        self.n, self.heads, self.D, self.at, self.S, self.B = B * S, heads, D, at, S, B
        self.buf = torch.full((B * S + 3, ld), MARK, device="cuda", dtype=t)
        self.view = self.buf[:self.n, at:at + heads * D]

    def ptr(self):
        return C.c_void_p(self.buf.data_ptr() + self.at * self.buf.element_size())

    def set(self, x):
        self.view.copy_(torch.as_tensor(x, device="cuda").reshape(self.n, -1))
        return self

    def get(self):
        return self.view.reshape(self.B, self.S, self.heads, self.D)

    def untouched(self):
        m = self.buf.clone()
        m[:self.n, self.at:self.at + self.heads * self.D] = MARK
        return bool((m == MARK).all())


class Case:
    def __init__(self, sq, skv, heads, kv_heads, lens, dtype="bf16", dim=64, beside=0, scale=1.0, seed=0, shift=0):
        B = len(lens)
        self.t, code, self.half = TYPES[dtype]
        self.lens, self.dtype = lens, dtype
        g = torch.Generator(device="cuda").manual_seed(10007 * sq + 101 * skv + heads + seed)
        normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        qw, kw = heads * dim, kv_heads * dim
        ldq, ldkv, ldo = qw + beside, 2 * kw + beside, qw + 2 * beside
        new = lambda S, h, ld, at: Rows(B, S, h, dim, ld, at, self.t)  # noqa: E731
        self.q = new(sq, heads, ldq + shift, shift).set(scale * normal(B, sq, qw))
        self.kv = torch.full((B * skv + 3, ldkv + shift), MARK, device="cuda", dtype=self.t)
        self.k, self.v = new(skv, kv_heads, 1, 0), new(skv, kv_heads, 1, 0)
        for i, x in enumerate((self.k, self.v)):  # one projection's output: K | V
            x.buf, x.at = self.kv, i * kw + shift
            x.view = self.kv[:B * skv, x.at:x.at + kw]
            x.set((scale if i == 0 else 1.0) * normal(B, skv, kw))
        self.dctx = new(sq, heads, ldo, beside).set(0.1 * normal(B, sq, qw))
        self.ld = (ldq + shift, ldkv + shift, ldkv + shift, ldo)
        self.new = dict(ctx=lambda: new(sq, heads, ldo, beside), dq=lambda: new(sq, heads, ldq + shift, shift),
                        dk=lambda: new(skv, kv_heads, ldkv + shift, shift),
                        dv=lambda: new(skv, kv_heads, ldkv + shift, kw + shift))
        self.d_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.shape = L.SkyCrossShape(B, sq, skv, heads, kv_heads, dim, code, *self.ld)
        self.B, self.sq, self.skv, self.heads, self.kv_heads, self.dim = B, sq, skv, heads, kv_heads, dim

    def poison(self):
        """Infinities and NaN wherever no key is valid."""
        for b, n in enumerate(self.lens):
            for x in (self.k, self.v):
                rows = x.view[b * self.skv + n:(b + 1) * self.skv]
                rows[0::2], rows[1::2] = float("nan"), float("inf")
        return self

    def forward(self, with_lse=True):
        ctx = self.new["ctx"]()
        lse = torch.full((self.B * self.heads * self.sq + 8,), MARK, device="cuda")
        L.call("sky_cross_attention_fwd", self.shape, self.q.ptr(), self.k.ptr(), self.v.ptr(), P(self.d_len),
               ctx.ptr(), P(lse) if with_lse else None, P(self.status), stream())
        torch.cuda.synchronize()
        n = self.B * self.heads * self.sq
        assert ctx.untouched() and bool((lse[n if with_lse else 0:] == MARK).all()) and int(self.status.item()) == 0
        return ctx, lse[:n].view(self.B, self.heads, self.sq)

    def backward(self, ctx, lse):
        out = [self.new[n]() for n in ("dq", "dk", "dv")]
        n = L.lib().sky_cross_attention_bwd_workspace_bytes(self.shape)
        ws = torch.full((n + 64,), 0x7f, dtype=torch.uint8, device="cuda")
        L.call("sky_cross_attention_bwd", self.shape, self.q.ptr(), self.k.ptr(), self.v.ptr(), ctx.ptr(),
               self.dctx.ptr(), P(lse), P(self.d_len), *[o.ptr() for o in out], P(ws), n, P(self.status), stream())
        torch.cuda.synchronize()
        assert all(o.untouched() for o in out) and bool((ws[n:] == 0x7f).all()) and int(self.status.item()) == 0
        return out

    # ------------------------------------------------------------- the bounds
    def inputs(self):
        clean = lambda x: np.where(np.isfinite(x), x, 0.0)  # noqa: E731  (poisoned rows take no part)
        return [clean(f64(x.get())) for x in (self.q, self.k, self.v, self.dctx)]

    def walk(self):
        """Per sequence and head: (b, a, g, n, q, k, v, dctx, P, error factor of P)."""
        q, k, v, dctx = self.inputs()
        c = self.dim ** -0.5
        for b in range(self.B):
            n = self.lens[b]
            for a in range(self.heads if n else 0):
                g = a // (self.heads // self.kv_heads)
                s = q[b, :, a] @ k[b, :n, g].T * c
                e = np.exp(s - s.max(-1, keepdims=True))
                E = (self.dim + 8) * U * c * (np.abs(q[b, :, a]) @ np.abs(k[b, :n, g]).T).max(-1, keepdims=True)
                yield b, a, g, n, q[b, :, a], k[b, :n, g], v[b, :n, g], dctx[b, :, a], e / e.sum(-1, keepdims=True), E

    def check_forward(self, ctx, lse):
        q, k, v, _ = self.inputs()
        want, want_lse = ORC.cross_attention(q, k, v, self.lens)
        bound, lse_bound = np.zeros(want.shape), np.zeros(want_lse.shape)
        for b, a, g, n, _, _, vv, _, p, E in self.walk():
            rel = 2 * E + 2.0 ** -20 + (n + 8) * U + (self.half if self.dtype == "bf16" else 0.0)
            bound[b, :, a] = rel * (p @ np.abs(vv))
            lse_bound[b, a] = (2 * E + 2.0 ** -20 + (n + 8) * U)[:, 0] * 1.5 + np.abs(want_lse[b, a]) * 2.0 ** -23
        got = f64(ctx.get())
        bound += self.half * np.abs(want)
        within(got, want, bound, "ctx")
        if lse is not None:
            got = f64(lse)
            dead = want_lse == -np.inf
            assert (got[dead] == -np.inf).all()
            within(got[~dead], want_lse[~dead], lse_bound[~dead], "lse")

    def given(self):
        """(ctx, lse) as a forward leaves them, from the oracle."""
        q, k, v, _ = self.inputs()
        want, want_lse = ORC.cross_attention(q, k, v, self.lens)
        return self.new["ctx"]().set(want), torch.tensor(want_lse, dtype=torch.float32, device="cuda")

    def check_backward(self, grads):
        q, k, v, dctx = self.inputs()
        want = ORC.cross_attention_backward(q, k, v, dctx, self.lens)
        ctx, lse = ORC.cross_attention(q, k, v, self.lens)
        bound = [np.zeros(w.shape) for w in want]
        c, bf16 = self.dim ** -0.5, self.dtype == "bf16"
        op = self.half if bf16 else 0.0
        for b, a, g, n, qq, kk, vv, dd, p, E in self.walk():
            dp = dd @ vv.T
            delta = (p * dp).sum(-1, keepdims=True)
            mag = np.abs(dd) @ np.abs(vv).T                              # of dP's products
            dmag = (np.abs(dd) * np.abs(ctx[b, :, a])).sum(-1, keepdims=True)  # of delta's
            eP = 2 * E + 2.0 ** -20 + 8 * U + np.abs(lse[b, a])[:, None] * (2.0 ** -16 if bf16 else 2.0 ** -22)
            ds = p * (dp - delta)
            eds = np.abs(ds) * (op + eP) + p * ((self.dim + 8) * U * (mag + dmag) + (self.half + 2.0 ** -16 * bf16) * dmag)
            both = self.sq * (self.heads // self.kv_heads)
            bound[0][b, :, a] = c * ((eds + (n + 8) * U * np.abs(ds)) @ np.abs(kk))
            bound[1][b, :n, g] += c * ((eds + (both + 8) * U * np.abs(ds)).T @ np.abs(qq))
            bound[2][b, :n, g] += ((p * (op + eP + (both + 8) * U)).T @ np.abs(dd))
        for got, w, e, name in zip(grads, want, bound, ("dq", "dk", "dv")):
            within(f64(got.get()), w, e + self.half * np.abs(w), name)


SHAPES = [
    # queries, keys, heads, key heads, valid lengths
    (1, 1, 1, 1, [1, 0]),
    (1, 70, 3, 3, [70, 1, 0, 64, 65]),
    (5, 3, 4, 1, [3, 0, 2]),
    (16, 16, 2, 2, [16, 9]),
    (17, 200, 6, 2, [0, 200, 129, 64]),
    (45, 32, 2, 2, [32, 16, 31, 1]),
    (64, 129, 8, 2, [129, 128, 1]),
    (100, 96, 4, 2, [96, 33]),
    (128, 128, 3, 3, [128, 127]),
    (129, 65, 5, 1, [65, 0, 1]),
    (200, 333, 12, 4, [333, 65, 0]),
    (257, 514, 4, 4, [514, 1]),
    (300, 80, 16, 2, [80, 40, 17]),
    (30, 100, 8, 2, [100, 0, 99, 1]),   # one tile holds every head of a key head
    (1, 17, 128, 1, [17, 0, 16]),
    (127, 127, 2, 2, [127, 126, 0]),
    (129, 128, 2, 2, [128, 3]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:4])))
def test_forward_and_backward(shape, dtype):
    c = Case(*shape, dtype=dtype, beside=8).poison()
    ctx, lse = c.forward()
    c.check_forward(ctx, lse)
    grads = c.backward(*c.given())
    c.check_backward(grads)
    again, back = c.forward(), c.backward(*c.given())
    assert torch.equal(again[0].buf, ctx.buf) and torch.equal(again[1], lse)
    assert all(torch.equal(x.buf, y.buf) for x, y in zip(grads, back))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim,shift", [(20, 0), (32, 0), (33, 1), (64, 1), (64, 4), (80, 0), (128, 0)])
def test_other_heads_and_alignments(dim, shift, dtype):
    c = Case(37, 75, 4, 2, [75, 20, 0, 1], dtype=dtype, dim=dim, beside=shift, shift=shift).poison()
    c.check_forward(*c.forward())
    c.check_backward(c.backward(*c.given()))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_scores(dtype):
    """Rows that one key takes whole, and maxima that rise from tile to tile."""
    c = Case(130, 300, 4, 2, [300, 250], dtype=dtype, scale=4.0)
    k = c.k.get().clone()
    k *= torch.linspace(0.1, 1.5, 300, device="cuda").to(c.t)[None, :, None, None]
    c.k.set(k)
    c.check_forward(*c.forward())
    c.check_backward(c.backward(*c.given()))


@pytest.mark.parametrize("sq,skv,heads,kv_heads,lens", [
    (700, 100, 8, 2, [100, 64]), (900, 16, 9, 3, [16, 3]), (500, 130, 2, 2, [130, 1]), (260, 65, 4, 4, [65, 0]),   # few keys
    (40, 945, 6, 3, [945, 700]), (1, 1500, 2, 1, [1500, 0]), (17, 700, 32, 1, [700, 450]), (70, 520, 3, 3, [520, 64]),
    (2000, 2000, 1, 1, [1999]),
])
def test_sums_split_over_a_cluster(sq, skv, heads, kv_heads, lens):
    """Gradients of few keys that many queries read, and of few queries that read many keys."""
    c = Case(sq, skv, heads, kv_heads, lens).poison()
    grads = c.backward(*c.given())
    c.check_backward(grads)
    assert all(torch.equal(x.buf, y.buf) for x, y in zip(grads, c.backward(*c.given())))


@pytest.mark.parametrize("sq,skv,heads,kv_heads,lens,dim,shift,dtype", [
    (6, 1650, 6, 2, [1650, 0, 582], 128, 0, "fp32"), (468, 6, 4, 1, [6, 0, 5], 64, 0, "fp32"),
    (182, 38, 8, 2, [38, 19], 64, 0, "fp32"), (51, 340, 1, 1, [340, 65, 1], 33, 1, "fp32"),
    (53, 700, 3, 3, [700, 64], 20, 0, "fp32"), (130, 17, 5, 1, [17, 16], 32, 0, "fp32"),
    (10, 300, 4, 2, [300, 129, 0], 80, 0, "bf16"), (150, 70, 6, 2, [70, 0], 64, 1, "bf16"),
    (600, 530, 2, 2, [530], 32, 0, "fp32"), (17, 17, 16, 1, [17, 3], 64, 0, "fp32"),
])
def test_columns_split_on_the_cuda_cores(sq, skv, heads, kv_heads, lens, dim, shift, dtype):
    """The same where the tensor cores do not serve: one kind's blocks, or both kinds', in parts."""
    c = Case(sq, skv, heads, kv_heads, lens, dtype=dtype, dim=dim, beside=shift, shift=shift).poison()
    grads = c.backward(*c.given())
    c.check_backward(grads)
    assert all(torch.equal(x.buf, y.buf) for x, y in zip(grads, c.backward(*c.given())))


@pytest.mark.parametrize("sq,skv,heads,kv_heads,lens", [
    (500, 100, 1, 1, [100, 0, 17]), (1024, 128, 2, 2, [128, 1]), (1000, 3, 3, 3, [3, 2, 0]), (40, 90, 6, 2, [90, 16]),
    (70, 33, 12, 2, [33, 32, 0]), (5, 50, 24, 2, [50, 49]), (129, 128, 2, 1, [128, 127]), (300, 64, 4, 2, [64, 63, 1]),
    (1025, 20, 1, 1, [20]), (1, 128, 320, 1, [128, 5]), (131, 77, 5, 1, [77, 0]), (640, 97, 2, 2, [97, 96]),
])
def test_few_keys_of_many_queries(sq, skv, heads, kv_heads, lens):
    """One tile of keys and up to eight of queries, which add their parts; and more than that."""
    c = Case(sq, skv, heads, kv_heads, lens, beside=8).poison()
    grads = c.backward(*c.given())
    c.check_backward(grads)
    assert all(torch.equal(x.buf, y.buf) for x, y in zip(grads, c.backward(*c.given())))


def test_forward_feeds_backward():
    """The library's own ctx and lse: within what the forward may be off more."""
    c = Case(150, 220, 6, 3, [220, 100, 0, 7]).poison()
    ctx, lse = c.forward()
    grads = c.backward(ctx, lse)
    want = c.backward(*c.given())
    for x, y in zip(grads, want):
        a, b = f64(x.get()), f64(y.get())
        assert np.linalg.norm(a - b) <= 2.0 ** -7 * np.linalg.norm(b)


def test_lengths_outside_are_clamped_and_reported():
    c = Case(20, 70, 2, 2, [70, 0])
    ctx, lse = c.forward()
    grads = c.backward(*c.given())
    c.d_len.copy_(torch.tensor([71, -1], dtype=torch.int32))
    bad = c.new["ctx"]()
    L.call("sky_cross_attention_fwd", c.shape, c.q.ptr(), c.k.ptr(), c.v.ptr(), P(c.d_len), bad.ptr(), None,
           P(c.status), stream())
    torch.cuda.synchronize()
    assert int(c.status.item()) == 1 and torch.equal(bad.buf, ctx.buf)
    c.status.zero_()
    out = [c.new[n]() for n in ("dq", "dk", "dv")]
    n = L.lib().sky_cross_attention_bwd_workspace_bytes(c.shape)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    ctx, lse = c.given()
    L.call("sky_cross_attention_bwd", c.shape, c.q.ptr(), c.k.ptr(), c.v.ptr(), ctx.ptr(), c.dctx.ptr(), P(lse),
           P(c.d_len), *[o.ptr() for o in out], P(ws), n, P(c.status), stream())
    torch.cuda.synchronize()
    assert int(c.status.item()) == 1 and all(torch.equal(x.buf, y.buf) for x, y in zip(out, grads))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sq,heads,kv_heads,skv,lens", [
    (1, 16, 16, 512, [512, 256, 300, 1, 0, 511]), (1, 16, 4, 2500, [2500, 1300]), (2, 8, 1, 1031, [1031, 0, 5]),
    (4, 4, 4, 333, [333, 32, 33]), (1, 1, 1, 5000, [4999]), (3, 10, 2, 700, [700, 16, 15, 17]), (1, 32, 1, 260, [260]),
    (17, 2, 2, 2100, [2100, 0, 1999]), (8, 12, 4, 2048, [2048, 1, 33]), (32, 1, 1, 3001, [3001]), (1, 25, 1, 4100, [4100, 7]),
])
def test_few_query_rows(sq, heads, kv_heads, skv, lens, dtype):
    c = Case(sq, skv, heads, kv_heads, lens, dtype=dtype).poison()
    ctx, lse = c.forward()
    c.check_forward(ctx, lse)
    assert torch.equal(c.forward(with_lse=False)[0].buf, ctx.buf)
    c.check_backward(c.backward(*c.given()))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sq,heads,kv_heads,dim,shift", [(1, 3, 3, 20, 0), (1, 4, 1, 33, 1), (2, 6, 2, 128, 0),
                                                         (4, 8, 2, 80, 4), (3, 14, 1, 64, 1), (1, 2, 2, 3, 0),
                                                         (1, 1, 1, 32, 0), (4, 1, 1, 100, 0)])
def test_few_query_rows_of_other_heads(sq, heads, kv_heads, dim, shift, dtype):
    c = Case(sq, 650, heads, kv_heads, [650, 0, 1, 31, 32, 33, 300], dtype=dtype, dim=dim, beside=shift,
             shift=shift).poison()
    c.check_forward(*c.forward())


def test_captured_and_replayed():
    c = Case(33, 150, 4, 2, [150, 80])
    ctx, (dq, dk, dv) = c.new["ctx"](), [c.new[n]() for n in ("dq", "dk", "dv")]
    lse = torch.empty(c.B, c.heads, c.sq, device="cuda")
    n = L.lib().sky_cross_attention_bwd_workspace_bytes(c.shape)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def both():
        L.call("sky_cross_attention_fwd", c.shape, c.q.ptr(), c.k.ptr(), c.v.ptr(), P(c.d_len), ctx.ptr(), P(lse),
               None, stream())
        L.call("sky_cross_attention_bwd", c.shape, c.q.ptr(), c.k.ptr(), c.v.ptr(), ctx.ptr(), c.dctx.ptr(), P(lse),
               P(c.d_len), dq.ptr(), dk.ptr(), dv.ptr(), P(ws), n, None, stream())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    c.lens = [60, 0]
    c.d_len.copy_(torch.tensor(c.lens, dtype=torch.int32))
    c.q.set(-c.q.get().clone())
    for x in (ctx, dq, dk, dv):
        x.buf.fill_(MARK)
    graph.replay()
    torch.cuda.synchronize()
    want, want_lse = c.forward()
    assert torch.equal(ctx.buf, want.buf) and torch.equal(lse, want_lse)
    assert all(torch.equal(x.buf, y.buf) for x, y in zip((dq, dk, dv), c.backward(want, want_lse)))
