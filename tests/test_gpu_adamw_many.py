"""The AdamW step of many tensors, moments in 32 bits and in 8, against float64: odd sizes and
addresses, both gradient types, hundreds of tensors, captured steps, blocks of zeros and of NaN."""
import ctypes as C

import numpy as np
import pytest

from oracle import experts_f64 as ORC
from oracle import optimizer as OPT
from paper_2202_11836_gb300 import _lib as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF = L.SKY_DTYPE_FP32, L.SKY_DTYPE_BF16
RULE = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
MARK = 77


def P(t):
    return None if t is None else int(t.data_ptr())


def stream():
    return C.c_void_p(int(torch.cuda.current_stream().cuda_stream))


def f64(t):
    return t.double().cpu().numpy()


class Tensor:
    """n values, every buffer `shift` values behind a 256-byte boundary and with a guard behind it."""

    def __init__(self, n, small, grads, g, decay=1, shift=0, copy=True):
        self.n, self.small, self.decay, self.shift = n, small, decay, shift
        blocks = -(-n // L.SKY_STATE_BLOCK)
        gt = torch.bfloat16 if grads == BF else torch.float32
        mt = torch.uint8 if small else torch.float32
        self.buffers = {"w": (n, torch.float32), "g": (n, gt), "m": (n, mt), "v": (n, mt)}
        if copy:
            self.buffers["p"] = (n, torch.bfloat16)
        if small:
            self.buffers.update(m_scale=(blocks, torch.float32), v_scale=(blocks, torch.float32))
        self.mem = {k: torch.full((m + shift + 8,), MARK, device="cuda").to(t) for k, (m, t) in self.buffers.items()}
        for k in self.buffers:
            self.at(k).zero_()
        self.at("w").copy_(torch.randn(n, device="cuda", generator=g))
        self.new_gradient(g)

    def at(self, k):
        m, _ = self.buffers[k]
        return self.mem[k][self.shift:self.shift + m]

    def new_gradient(self, g):
        size = 10.0 ** torch.randint(-3, 2, (self.n,), device="cuda", generator=g)
        self.at("g").copy_(torch.randn(self.n, device="cuda", generator=g) * size)

    def entry(self):
        ptr = lambda k: P(self.at(k)) if k in self.buffers else None  # noqa: E731
        return L.SkyAdamwTensor(*[ptr(k) for k in ("w", "g", "m", "v", "m_scale", "v_scale", "p")], self.n, self.decay)

    def moments(self):
        if not self.small:
            return f64(self.at("m")), f64(self.at("v"))
        return (ORC.decode(self.at("m").cpu().numpy(), f64(self.at("m_scale")), ORC.e4m3_values()),
                ORC.decode(self.at("v").cpu().numpy(), f64(self.at("v_scale")), ORC.root_values()) ** 2)

    def expect(self, t, rule=RULE, scale=1.0):
        """What the step makes of the present values: (w, m, v)."""
        b1, b2 = float(np.float32(rule["beta1"])), float(np.float32(rule["beta2"]))
        lr, eps, wd = (float(np.float32(rule[k])) for k in ("lr", "eps", "weight_decay"))
        m, v = self.moments()
        return OPT.adamw_step(f64(self.at("w")), f64(self.at("g")) * scale, m, v, t, lr, b1, b2, eps, wd, bool(self.decay))

    def check(self, want, before, lr=RULE["lr"]):
        w, m, v = want
        for k, (n, _) in self.buffers.items():
            assert bool((self.mem[k][:self.shift] == MARK).all()) and bool((self.mem[k][self.shift + n:] == MARK).all()), k
        # w: a dozen roundings of a step of about lr (m is below 10 sqrt(v) with these settings), one of w itself
        step = lr * (16 * 2.0 ** -23) * 10 + 2.0 ** -23 * np.abs(before)
        assert (np.abs(f64(self.at("w")) - w) <= step).all(), np.abs(f64(self.at("w")) - w).max()
        if "p" in self.buffers:
            assert torch.equal(self.at("p"), self.at("w").to(torch.bfloat16))
        gm, gv = self.moments()
        if not self.small:
            top = np.maximum(np.abs(before_scale(m, self.at("g"))), 0)
            assert (np.abs(gm - m) <= 4 * 2.0 ** -24 * top + 1e-44).all()
            assert (np.abs(gv - v) <= 5 * 2.0 ** -24 * v + 1e-44).all()
            return
        blocks = [slice(i, min(i + ORC.BLOCK, self.n)) for i in range(0, self.n, ORC.BLOCK)]
        for b, ms, vs in zip(blocks, f64(self.at("m_scale")), f64(self.at("v_scale"))):
            r, gr, top = np.sqrt(v[b]), np.sqrt(gv[b]), np.abs(m[b]).max()
            if top < 1e-30:
                assert ms == 0 and not gm[b].any()
            else:
                # to the nearest: 2^-4 of the value, or 2^-10 units below the smallest normal; the fp32 value that is
                # rounded is itself off by a few 2^-24 of its two terms, which cancel at worst
                assert abs(ms * 448 / top - 1) < 2.0 ** -20
                slack = 2.0 ** -20 * np.maximum(np.abs(m[b]), before_scale(m[b], self.at("g")[b]))
                assert (np.abs(gm[b] - m[b]) <= 2.0 ** -4 * np.abs(m[b]) * (1 + 2.0 ** -18) + 2.0 ** -10 * ms + slack).all()
            if r.max() < 1e-30:
                assert vs == 0 and not gr.any()
                continue
            assert abs(vs * 0.96875 / r.max() - 1) < 2.0 ** -20
            least = 17 / 16 * 2.0 ** -16 * vs
            near = np.abs(gr - r) <= 2.0 ** -5 * r * (1 + 2.0 ** -18)
            assert (near | ((r < least) & (np.abs(gr - least) <= 1e-6 * least))).all()
            assert (gr[r > 0] > 0).all()


def before_scale(m, g):
    """|m'| is at most 0.9 |m| + 0.1 |g|, the size that its roundings go by."""
    return np.abs(m) + 0.2 * np.abs(f64(g))


def step(tensors, t, small, grads=F32, now=None, rule=RULE):
    cfg = L.SkyAdamwConfig(rule["lr"], rule["beta1"], rule["beta2"], rule["eps"], rule["weight_decay"], t, grads,
                           L.SKY_STATE_8BIT if small else L.SKY_STATE_FP32)
    table = (L.SkyAdamwTensor * len(tensors))(*[x.entry() for x in tensors])
    L.call("sky_adamw_step", cfg, table, len(tensors), P(now), stream())
    C.memset(C.addressof(table), 0xee, C.sizeof(table))  # the call has read it


@pytest.mark.parametrize("small", [False, True], ids=["fp32", "8bit"])
@pytest.mark.parametrize("grads", [F32, BF], ids=["g32", "g16"])
def test_steps(small, grads):
    g = torch.Generator(device="cuda").manual_seed(2)
    sizes = [1, 3, 4, 255, 256, 257, 1000, 2048, 2049, 5000, 40000, 131072]
    ts = [Tensor(n, small, grads, g, decay=i % 2, shift=(0, 1, 4, 2)[i % 4], copy=i % 3 != 0) for i, n in enumerate(sizes)]
    for t in (1, 2, 3):
        want = [(x.expect(t), f64(x.at("w"))) for x in ts]
        step(ts, t, small, grads)
        torch.cuda.synchronize()
        for x, (w, before) in zip(ts, want):
            x.check(w, before)
            x.new_gradient(g)


@pytest.mark.parametrize("small", [False, True], ids=["fp32", "8bit"])
@pytest.mark.parametrize("count", [32, 33, 400, 801])
def test_hundreds_of_tensors(small, count):
    g = torch.Generator(device="cuda").manual_seed(3)
    ts = [Tensor(1 + (37 * i) % 600, small, F32, g, decay=i % 2) for i in range(count)]
    want = [(x.expect(1), f64(x.at("w"))) for x in ts]
    step(ts, 1, small)
    torch.cuda.synchronize()
    for x, (w, before) in zip(ts, want):
        x.check(w, before)


def test_zeros_and_a_lone_value():
    """A block without gradients keeps its zeros, and a value far below its block's largest its moment's sign."""
    g = torch.Generator(device="cuda").manual_seed(4)
    x = Tensor(1024, True, F32, g, decay=0)
    x.at("g").zero_()
    x.at("g")[300] = 1e-3
    x.at("g")[512:768] = 1.0
    x.at("g")[600] = 1e-12
    w = f64(x.at("w"))
    want = x.expect(1)
    step([x], 1, True)
    x.check(want, w)
    assert not x.at("v")[:256].any() and int((x.at("v") > 0).sum()) == 257
    assert np.array_equal(f64(x.at("w"))[:256], w[:256])
    # its moment came out as 0 of m and the least step of r: the next step cannot grow
    x.at("g").zero_()
    before = f64(x.at("w"))
    step([x], 2, True)
    assert np.abs(f64(x.at("w")) - before).max() < 2 * RULE["lr"]


def test_not_finite_stays_in_its_block():
    g = torch.Generator(device="cuda").manual_seed(5)
    for bad in (torch.nan, torch.inf):
        x, y = Tensor(700, True, F32, g), Tensor(700, False, F32, g)
        for z in (x, y):
            z.at("g")[300] = bad
            step([z], 1, z.small)
        torch.cuda.synchronize()
        m, v = x.moments()
        assert not np.isfinite(m[256:512]).any() and not np.isfinite(v[256:512]).any()  # (an infinite scale: its own code's is infinite, 0 times it NaN)
        for part in (slice(0, 256), slice(512, 700)):
            assert np.isfinite(m[part]).all() and np.isfinite(v[part]).all()
        assert int((~torch.isfinite(x.at("w"))).sum()) <= 1  # the update goes by what is not yet rounded
        assert int((~torch.isfinite(y.at("m"))).sum()) == 1


def test_weights_follow_the_moments_of_a_block():
    """Moments in 8 bits against 32: with gradients of one size in a block both walk alike."""
    g = torch.Generator(device="cuda").manual_seed(6)
    x, y = Tensor(4096, True, F32, g, decay=0), Tensor(4096, False, F32, g, decay=0)
    y.at("w").copy_(x.at("w"))
    start = x.at("w").clone()
    for t in range(1, 101):
        x.at("g").copy_(torch.randn(4096, device="cuda", generator=g) + 0.5)
        y.at("g").copy_(x.at("g"))
        step([x], t, True)
        step([y], t, False)
    walked = (y.at("w") - start).norm()
    # r is off by up to 2^-5 at every step, m by 2^-4, mostly of either sign
    assert float((x.at("w") - y.at("w")).norm() / walked) < 2.0 ** -4 + 2.0 ** -5


@pytest.mark.parametrize("small", [False, True], ids=["fp32", "8bit"])
def test_captured_steps_take_their_numbers_from_the_device(small):
    g = torch.Generator(device="cuda").manual_seed(7)
    x, y = (Tensor(5000, small, F32, torch.Generator(device="cuda").manual_seed(8)) for _ in range(2))
    now = torch.empty(4, device="cuda")
    grad = [torch.randn(5000, device="cuda", generator=g) for _ in range(3)]

    def numbers(t, lr, scale):
        b1, b2 = (float(np.float32(RULE[k])) for k in ("beta1", "beta2"))
        return torch.tensor([lr, 1 - b1 ** t, 1 - b2 ** t, scale], device="cuda")

    other = Tensor(5000, small, F32, g)
    now.copy_(numbers(1, 1e-3, 1.0))
    step([other], 1, small, now=now)  # loads the module before the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step([x], 1, small, now=now)
    for t, d in enumerate(grad, 1):
        lr = float(np.float32(1e-2 / t))
        now.copy_(numbers(t, lr, 0.5))
        x.at("g").copy_(d)
        y.at("g").copy_(0.5 * d)
        graph.replay()
        step([y], t, small, rule=dict(RULE, lr=lr))
        torch.cuda.synchronize()
        for k in x.buffers:
            if k == "w":  # (the corrections are rounded the same way on both sides, in another place)
                assert float((x.at(k) - y.at(k)).abs().max()) < 1e-7
            elif k not in ("g", "p"):
                assert torch.equal(x.at(k), y.at(k)), k


def test_more_values_than_31_bits():
    n = (1 << 31) + 517
    w, p = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    g = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    m, v = torch.zeros(n, device="cuda", dtype=torch.uint8), torch.zeros(n, device="cuda", dtype=torch.uint8)
    ms, vs = (torch.zeros(-(-n // 256), device="cuda") for _ in range(2))
    spots = [0, 1 << 30, (1 << 31) - 1, 1 << 31, n - 1]
    g[spots] = 1.0
    table = (L.SkyAdamwTensor * 1)(L.SkyAdamwTensor(P(w), P(g), P(m), P(v), P(ms), P(vs), P(p), n, 1))
    cfg = L.SkyAdamwConfig(0.5, 0.9, 0.99, 1e-8, 0.0, 1, BF, L.SKY_STATE_8BIT)
    L.call("sky_adamw_step", cfg, table, 1, None, stream())
    assert int(torch.count_nonzero(w)) == len(spots) and torch.allclose(w[spots], torch.full((5,), -0.5, device="cuda"))
    assert int(torch.count_nonzero(v)) == len(spots) and int((ms > 0).sum()) == 5  # each in a block of its own
