"""Calls that a user makes at once: routing, rows and products of two layers on two streams, each with outputs and
workspaces of its own, and an update of more tensors than a launch takes, captured."""
import ctypes as C

import pytest

import test_gpu_adamw_many as ADAM
import test_gpu_grouped as GROUPED
import test_gpu_route as ROUTE
from paper_2202_11836_gb300 import _lib as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def P(t):
    return C.c_void_p(int(t.data_ptr()))


class Layer:
    """Calls of every kernel: route over one and over many blocks, the products' four kernels in bf16 and the split
    ones in fp32, column sums."""

    def __init__(self, seed):
        g = GROUPED.Case
        self.route = [ROUTE.Case(t, 64, 4, "bf16", "chosen", seed=seed) for t in (50, 3000)]
        self.routed = [[torch.empty(r.tokens, 4, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int32)]
                       + [torch.empty(65, dtype=torch.int32, device="cuda")] for r in self.route]
        self.route_ws = [torch.empty(L.lib().sky_route_workspace_bytes(r.shape), dtype=torch.uint8, device="cuda") for r in self.route]
        self.products = [g("xwt", [9, 3], 256, 2048, "bf16", "gelu", seed=seed), g("xw", [300, 77], 512, 1024, "bf16", "gelu_bwd", seed=seed),
                         g("xtw", [3001, 5], 256, 128, "bf16", seed=seed), g("xtw", [700, 33], 1024, 1024, "bf16", seed=seed),
                         g("xwt", [90, 70, 97], 512, 128, "fp32", "gelu", seed=seed), g("xtw", [900, 4100], 79, 101, "fp32", seed=seed)]
        self.made = [c.room() for c in self.products]
        self.ws = [c.workspace() for c in self.products]
        s = self.products[1]
        self.sums, self.shape = torch.empty(2, 512, device="cuda"), L.SkyGroupedShape(2, 377, 512, 0, L.SKY_DTYPE_BF16)
        self.offset, self.x = s.d_offset, s.a

    def call(self):
        st = C.c_void_p(int(torch.cuda.current_stream().cuda_stream))
        for r, out, ws in zip(self.route, self.routed, self.route_ws):
            L.call("sky_route_fwd", r.shape, P(r.logits), *[P(o) for o in out], P(ws), ws.numel(), None, st)
        for c, (out, slope), (n, ws) in zip(self.products, self.made, self.ws):
            c.call(out, slope, n, ws)
        L.call("sky_grouped_column_sum", self.shape, P(self.offset), P(self.x), P(self.sums), None, st)

    def outputs(self):
        return [o for out in self.routed for o in out] + [o for m in self.made for o in m if o is not None] + [self.sums]


def test_two_layers_on_two_streams():
    layers = [Layer(seed) for seed in (2, 4)]
    want = []
    for x in layers:
        x.call()
        torch.cuda.synchronize()
        want.append([o.clone() for o in x.outputs()])
        for o in x.outputs():
            o.fill_(99)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(25):
        for x, s in zip(layers, streams):
            with torch.cuda.stream(s):
                x.call()
    torch.cuda.synchronize()
    for x, w in zip(layers, want):
        for got, o in zip(x.outputs(), w):
            same = got.view(torch.uint8) == o.view(torch.uint8)
            # (rooms end in 64 values that no call writes)
            assert bool(same[:-64 * got.element_size()].all()) if got.dim() == 1 and got.numel() > 1000 else bool(same.all())


@pytest.mark.parametrize("small", [False, True], ids=["fp32", "8bit"])
def test_more_tensors_than_a_launch_takes_captured(small):
    def tensors():
        g = torch.Generator(device="cuda").manual_seed(9)
        return [ADAM.Tensor(1 + (37 * i) % 600, small, ADAM.F32, g, decay=i % 2, shift=i % 3) for i in range(433)]

    b1, b2 = (float(torch.tensor(ADAM.RULE[k], dtype=torch.float32)) for k in ("beta1", "beta2"))
    now = torch.empty(4, device="cuda")
    x, y = tensors(), tensors()
    ADAM.step(tensors(), 1, small)  # loads the module before the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ADAM.step(x, 1, small, now=now)
    for t in (1, 2):
        now.copy_(torch.tensor([ADAM.RULE["lr"], 1 - b1 ** t, 1 - b2 ** t, 1.0]))
        graph.replay()
        ADAM.step(y, t, small)
    torch.cuda.synchronize()
    for a, b in zip(x, y):
        for k in a.buffers:
            assert torch.equal(a.mem[k].view(torch.uint8), b.mem[k].view(torch.uint8)), k
