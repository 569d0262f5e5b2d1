"""A layer of experts over a slice's states, as it is trained: route, dispatch, both products with
bias and GELU, combine, all the way back to the states, the router and every expert's tensors, and
the AdamW step of all of them; the whole step captured and replayed.  Against float64."""
import ctypes as C

import numpy as np
import pytest

from oracle import experts_f64 as ORC
from oracle import optimizer as OPT
from paper_2202_11836_gb300 import _lib as L
from paper_2202_11836_gb300 import synth
from paper_2202_11836_gb300.slice import EncoderSlice

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF, F32 = L.SKY_DTYPE_BF16, L.SKY_DTYPE_FP32
RULE = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, wd=0.01)


def P(t):
    return None if t is None else int(t.data_ptr())


def stream():
    return C.c_void_p(int(torch.cuda.current_stream().cuda_stream))


def f64(t):
    return t.double().cpu().numpy()


def l2(got, want):
    return np.linalg.norm(f64(got) - want) / np.linalg.norm(want)


class Layer:
    """E experts of width H and F, K of them a token; every buffer is made once."""

    def __init__(self, tokens, H, F, E, K, states, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T, self.H, self.F, self.E, self.K, self.states = tokens, H, F, E, K, states
        small = states == L.SKY_STATE_8BIT
        normal = lambda *s, std=0.02: torch.randn(*s, device="cuda", generator=g) * std  # noqa: E731
        empty = lambda *s, t=torch.bfloat16: torch.empty(*s, device="cuda", dtype=t)  # noqa: E731
        R = tokens * K
        self.master = {"router": normal(E, H, std=0.1), "w1": normal(E, F, H, std=0.05), "b1": normal(E, F),
                       "w2": normal(E, H, F, std=0.05), "b2": normal(E, H)}
        self.param = {n: w.to(torch.bfloat16) for n, w in self.master.items()}
        for n, w in self.master.items():
            w.copy_(self.param[n])
        self.grad = {n: torch.zeros_like(w) for n, w in self.master.items()}
        blocks = lambda w: -(-w.numel() // L.SKY_STATE_BLOCK)  # noqa: E731
        self.m = {n: torch.zeros(w.numel(), device="cuda", dtype=torch.uint8 if small else torch.float32)
                  for n, w in self.master.items()}
        self.v = {n: torch.zeros_like(x) for n, x in self.m.items()}
        self.scales = {n: torch.zeros(2, blocks(w), device="cuda") for n, w in self.master.items()}
        self.logits, self.dlogits = empty(tokens, E), empty(tokens, E)
        self.expert, self.row = (empty(tokens, K, t=torch.int32) for _ in range(2))
        self.weight, self.dweight = (empty(tokens, K, t=torch.float32) for _ in range(2))
        self.offset = empty(E + 1, t=torch.int32)
        self.rows, self.drows = empty(R, H), empty(R, H)
        self.up, self.dup, self.slope = empty(R, F), empty(R, F), empty(R, F, t=torch.float16)
        self.out, self.dout = empty(R, H), empty(R, H)
        self.y, self.dx, self.dx_router = empty(tokens, H), empty(tokens, H), empty(tokens, H)
        self.route = L.SkyRouteShape(tokens, E, K, BF, L.SKY_ROUTE_OVER_CHOSEN)
        self.rshape = L.SkyRowsShape(tokens, K, H, BF)
        self.g1, self.g2 = L.SkyGroupedShape(E, R, F, H, BF), L.SkyGroupedShape(E, R, H, F, BF)
        lib = L.lib()
        need = [lib.sky_route_workspace_bytes(self.route), lib.sky_gemm_workspace_bytes(L.SKY_GEMM_XTW, E, H, tokens, BF, F32), 16]
        need += [lib.sky_grouped_gemm_workspace_bytes(form, s, F32 if form == L.SKY_GEMM_XTW else BF)
                 for form in (0, 1, 2) for s in (self.g1, self.g2)]
        self.ws = empty(max(need), t=torch.uint8)

    def gemm(self, form, M, N, K, a, b, c):
        L.call("sky_gemm", form, M, N, K, BF, P(a), P(b), P(c), F32 if c.dtype == torch.float32 else BF, L.SKY_EPI_STORE,
               None, None, None, P(self.ws), self.ws.numel(), None, stream())

    def product(self, form, shape, a, b, c, epi=L.SKY_EPI_STORE, bias=None, aux=None, aux_out=None):
        L.call("sky_grouped_gemm", form, shape, P(self.offset), P(a), P(b), P(c), F32 if form == L.SKY_GEMM_XTW else BF, epi,
               P(bias), P(aux), P(aux_out), P(self.ws), self.ws.numel(), None, stream())

    def forward(self, x):
        p, s = self.param, stream()
        self.gemm(L.SKY_GEMM_XWT, self.T, self.E, self.H, x, p["router"], self.logits)
        L.call("sky_route_fwd", self.route, P(self.logits), P(self.expert), P(self.weight), P(self.row), P(self.offset),
               P(self.ws), self.ws.numel(), None, s)
        L.call("sky_dispatch_fwd", self.rshape, P(x), P(self.row), P(self.rows), s)
        self.product(L.SKY_GEMM_XWT, self.g1, self.rows, p["w1"], self.up, L.SKY_EPI_BIAS_GELU, p["b1"], None, self.slope)
        self.product(L.SKY_GEMM_XWT, self.g2, self.up, p["w2"], self.out, bias=p["b2"])
        L.call("sky_combine_fwd", self.rshape, P(self.out), P(self.row), P(self.weight), P(self.y), s)

    def backward(self, x, dy):
        p, d, s = self.param, self.grad, stream()
        L.call("sky_combine_bwd", self.rshape, P(self.out), P(dy), P(self.row), P(self.weight), P(self.dout),
               P(self.dweight), s)
        self.product(L.SKY_GEMM_XTW, self.g2, self.dout, self.up, d["w2"])
        L.call("sky_grouped_column_sum", self.g2, P(self.offset), P(self.dout), P(d["b2"]), None, s)
        self.product(L.SKY_GEMM_XW, self.g2, self.dout, p["w2"], self.dup, L.SKY_EPI_GELU_BWD, aux=self.slope)
        self.product(L.SKY_GEMM_XTW, self.g1, self.dup, self.rows, d["w1"])
        L.call("sky_grouped_column_sum", self.g1, P(self.offset), P(self.dup), P(d["b1"]), None, s)
        self.product(L.SKY_GEMM_XW, self.g1, self.dup, p["w1"], self.drows)
        L.call("sky_dispatch_bwd", self.rshape, P(self.drows), P(self.row), P(self.dx), s)
        L.call("sky_route_bwd", self.route, P(self.logits), P(self.expert), P(self.dweight), P(self.dlogits), s)
        self.gemm(L.SKY_GEMM_XTW, self.E, self.H, self.T, self.dlogits, x, d["router"])
        self.gemm(L.SKY_GEMM_XW, self.T, self.H, self.E, self.dlogits, p["router"], self.dx_router)

    def update(self, t, now=None):
        table = (L.SkyAdamwTensor * len(self.master))(*[
            L.SkyAdamwTensor(P(w), P(self.grad[n]), P(self.m[n]), P(self.v[n]), P(self.scales[n][0]), P(self.scales[n][1]),
                             P(self.param[n]), w.numel(), int(n[0] != "b")) for n, w in self.master.items()])
        cfg = L.SkyAdamwConfig(RULE["lr"], RULE["beta1"], RULE["beta2"], RULE["eps"], RULE["wd"], t, F32, self.states)
        L.call("sky_adamw_step", cfg, table, len(table), P(now), stream())

    def expected(self, x, dy):
        """(y, dx of the states, gradients) in float64, the choices as the layer made them."""
        p = {n: f64(w) for n, w in self.param.items()}
        logits = x @ p["router"].T
        expert = self.expert.cpu().numpy().astype(np.int64)
        row, offset = ORC.plan(expert, self.E)
        assert np.array_equal(row, self.row.cpu().numpy()) and np.array_equal(offset, self.offset.cpu().numpy())
        w = ORC.weights(logits, expert, "chosen")
        rows = ORC.dispatch(x, row, np.zeros((self.T * self.K, self.H)))
        group = np.repeat(np.arange(self.E), np.diff(offset))
        z = ORC.by_group("xwt", rows, p["w1"], offset)
        z[:len(group)] += p["b1"][group]
        up = ORC.gelu(z)
        out = ORC.by_group("xwt", up, p["w2"], offset)
        out[:len(group)] += p["b2"][group]
        y = ORC.combine(out, row, w)
        dout, dw = ORC.combine_backward(out, dy, row, w, np.zeros_like(out))
        dz = ORC.by_group("xw", dout, p["w2"], offset) * ORC.gelu_slope(z)
        sums = lambda v: np.stack([v[offset[e]:offset[e + 1]].sum(0) for e in range(self.E)])  # noqa: E731
        dl = ORC.route_backward(logits, expert, dw, "chosen")
        grads = {"w2": ORC.by_group("xtw", dout, up, offset), "b2": sums(dout), "w1": ORC.by_group("xtw", dz, rows, offset),
                 "b1": sums(dz), "router": dl.T @ x}
        return y, ORC.combine(ORC.by_group("xw", dz, p["w1"], offset), row, np.ones(row.shape)), dl @ p["router"], grads


def states_of_a_slice(B, S, H, seed=5):
    w = synth.custom("enc", layers=1, hidden=H, heads=4, ffn=512, seq=S, batch=B)
    s = EncoderSlice(H, 4, 512, 0, 1, B, S, "bf16")
    s.set_params(0, synth.layer_params(0, H, 512, "bf16"))
    x = torch.randn(B, S, H, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16()
    y = s.forward(x, torch.full((B,), S, dtype=torch.int32, device="cuda"))
    s.sync()
    return s, y.view(B * S, H)


@pytest.mark.parametrize("tokens,E,K", [((3, 80), 8, 2), ((2, 3), 16, 2), ((4, 129), 24, 3)])
def test_layer_over_a_slices_states(tokens, E, K):
    """Every bf16 tensor on the way is rounded once, 1.7e-3 of its norm: the output passes five such roundings
    (rows are copies: up, its product, out, the sum; the weights' logits), gradients up to nine, each about
    independent of the others: 3.8e-3 and 5.1e-3; bounds twice that.  Router gradients go through differences of
    dot products of rounded rows, whose common part cancels: three times that part."""
    H, F = 256, 512
    s, x = states_of_a_slice(*tokens, H)
    layer = Layer(x.shape[0], H, F, E, K, L.SKY_STATE_FP32)
    dy = (1e-2 * torch.randn(x.shape, device="cuda")).bfloat16()
    layer.forward(x)
    layer.backward(x, dy)
    torch.cuda.synchronize()
    y, dx, dx_router, grads = layer.expected(f64(x), f64(dy))
    assert l2(layer.y, y) < 8e-3
    assert l2(layer.dx, dx) < 1.1e-2
    for n in ("w1", "b1", "w2", "b2"):
        assert l2(layer.grad[n], grads[n]) < 1.1e-2, n
    assert l2(layer.grad["router"], grads["router"]) < 3.3e-2 and l2(layer.dx_router, dx_router) < 3.3e-2
    # back through the slice
    total = (layer.dx.float() + layer.dx_router.float()).bfloat16().view(*tokens, H)
    assert bool(torch.isfinite(s.backward(total)).all())


@pytest.mark.parametrize("states", [L.SKY_STATE_FP32, L.SKY_STATE_8BIT], ids=["fp32", "8bit"])
def test_training_steps_captured(states):
    """Three steps replayed from one graph give the bits of three steps called one by one, and the first
    is the float64 step from the layer's own gradients."""
    T, H, F, E, K = 200, 128, 256, 8, 2
    a, b = (Layer(T, H, F, E, K, states) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(T, H, device="cuda", generator=g).bfloat16()
    dy = (1e-2 * torch.randn(T, H, device="cuda", generator=g)).bfloat16()
    now = torch.empty(4, device="cuda")
    warm = Layer(T, H, F, E, K, states)

    def one(layer):
        layer.forward(x)
        layer.backward(x, dy)
        layer.update(1, now)

    def numbers(t):
        b1, b2 = (float(np.float32(RULE[n])) for n in ("beta1", "beta2"))
        return torch.tensor([RULE["lr"], 1 - b1 ** t, 1 - b2 ** t, 1.0], device="cuda")

    now.copy_(numbers(1))
    one(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(b)
    before = {n: f64(w) for n, w in a.master.items()}
    for t in (1, 2, 3):
        now.copy_(numbers(t))
        one(a)
        graph.replay()
        torch.cuda.synchronize()
        for n in a.master:
            assert torch.equal(a.master[n], b.master[n]) and torch.equal(a.m[n], b.m[n]) and torch.equal(a.v[n], b.v[n]), (t, n)
        if t == 1:
            for n, w in a.master.items():
                zero = np.zeros(before[n].shape)
                want, _, _ = OPT.adamw_step(before[n], f64(a.grad[n]), zero, zero, 1, *[float(np.float32(RULE[k])) for k in
                                            ("lr", "beta1", "beta2", "eps", "wd")], n[0] != "b")
                # the first step is lr sign(g) where g is well above eps: sixteen roundings of it, and the weight's
                assert (np.abs(f64(w) - want) <= RULE["lr"] * 2.0 ** -18 + 2.0 ** -23 * np.abs(want)).all(), n
