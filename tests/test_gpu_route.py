"""Routing to experts, forward and backward, against float64: equal logits, closed experts, padded
tokens, infinities and NaN, every size of a lane's share, one block of tokens and many."""
import ctypes as C

import numpy as np
import pytest

from oracle import experts_f64 as ORC
from paper_2202_11836_gb300 import _lib as L

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": (torch.bfloat16, L.SKY_DTYPE_BF16, 2.0 ** -8), "fp32": (torch.float32, L.SKY_DTYPE_FP32, 2.0 ** -24)}
OVER = {"all": L.SKY_ROUTE_OVER_ALL, "chosen": L.SKY_ROUTE_OVER_CHOSEN}
MARK = -77


def P(t):
    return None if t is None else C.c_void_p(int(t.data_ptr()))


def stream():
    return C.c_void_p(int(torch.cuda.current_stream().cuda_stream))


def f64(t):
    return t.double().cpu().numpy()


class Case:
    def __init__(self, tokens, experts, top_k, dtype, over, logits=None, seed=0):
        g = torch.Generator(device="cuda").manual_seed(7 * tokens + experts + seed)
        self.t, code, self.half_step = TYPES[dtype]
        self.tokens, self.experts, self.top_k, self.over, self.g = tokens, experts, top_k, over, g
        if logits is None:
            logits = 2 * torch.randn(tokens, experts, device="cuda", generator=g)
        self.logits = logits.to(self.t)
        self.shape = L.SkyRouteShape(tokens, experts, top_k, code, OVER[over])

    def forward(self, ws=None, status=None, stream_=None):
        n, k = self.tokens, self.top_k
        room = lambda m, t: torch.full((m + 4,), MARK, device="cuda", dtype=t)  # noqa: E731
        out = [room(n * k, torch.int32), room(n * k, torch.float32), room(n * k, torch.int32),
               room(self.experts + 1, torch.int32)]
        need = L.lib().sky_route_workspace_bytes(self.shape)
        ws = torch.full((need + 64,), 0x7f, dtype=torch.uint8, device="cuda") if ws is None else ws
        L.call("sky_route_fwd", self.shape, P(self.logits), *[P(o) for o in out], P(ws), need, P(status),
               stream_ or stream())
        torch.cuda.synchronize()
        assert bool((ws[need:] == 0x7f).all()) and all(bool((o[-4:] == MARK).all()) for o in out)
        return [o[:-4].view(n, k) for o in out[:3]] + [out[3][:-4]]

    def check(self, expert, weight, row, offset):
        x = f64(self.logits)
        want = ORC.choose(x, self.top_k)
        assert np.array_equal(expert.cpu().numpy(), want)
        rows, offsets = ORC.plan(want, self.experts)
        assert np.array_equal(offset.cpu().numpy(), offsets)
        assert np.array_equal(row.cpu().numpy(), rows)
        # weights: an exponential of a difference (its rounding 2^-24 of up to 100, then two ulps), a sum
        # of up to 1024 of those, a quotient
        w = ORC.weights(x, want, self.over)
        span = np.abs(np.where(np.isfinite(x), x, 0)).max(-1, keepdims=True) * 2
        assert (np.abs(f64(weight) - w) <= (span + 16 + np.log2(self.experts) + self.experts / 32) * 2.0 ** -23 * w + 1e-44).all()


SIZES = [(1, 1, 1), (1, 8, 2), (2, 3, 3), (16, 8, 2), (33, 32, 32), (64, 64, 4), (64, 1024, 3), (7, 257, 5), (65, 8, 2),
         (100, 33, 6), (1000, 128, 8), (4999, 64, 4), (3001, 256, 8), (700, 1024, 2), (8192, 16, 1), (9000, 1000, 2)]


@pytest.mark.parametrize("tokens,experts,top_k", SIZES)
@pytest.mark.parametrize("dtype,over", [("fp32", "chosen"), ("bf16", "all")])
def test_forward(tokens, experts, top_k, dtype, over):
    c = Case(tokens, experts, top_k, dtype, over)
    c.check(*c.forward())


@pytest.mark.parametrize("tokens", [5, 200])
def test_equal_closed_and_padded(tokens):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-2, 3, (tokens, 24), device="cuda", generator=g).float()
    x[x == 0] *= torch.where(torch.rand(int((x == 0).sum()), device="cuda", generator=g) < 0.5, -1.0, 1.0)  # +0 and -0
    x[:, 3] = -torch.inf              # an expert closed to all
    x[1] = -torch.inf                 # a padded token
    x[2, 1:] = -torch.inf             # fewer than top_k left
    x[3, 7], x[3, 9] = torch.inf, torch.inf
    x[4, 5] = -torch.finfo(torch.float32).max
    for over in OVER:
        for dtype in TYPES:
            c = Case(tokens, 24, 4, dtype, over, logits=x)
            out = c.forward()
            c.check(*out)
            assert out[0][1].tolist() == [-1] * 4 and out[1][1].tolist() == [0.0] * 4
            assert out[1][3].tolist()[:2] == [0.5, 0.5]


@pytest.mark.parametrize("tokens,experts,top_k", [(61, 5, 5), (1, 4, 2), (64, 8, 8), (67, 9, 9), (131, 16, 16), (5003, 8, 2),
                                                 (4097, 11, 3), (12100, 14, 8), (40001, 7, 1)])
def test_few_experts(tokens, experts, top_k):
    """Up to 16 experts: equal logits, tokens with some or none left beside others that have all."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x = torch.randint(-3, 4, (tokens, experts), device="cuda", generator=g).float() / 2
    x[torch.rand(tokens, experts, device="cuda", generator=g) < 0.3] = -torch.inf
    x[torch.rand(tokens, device="cuda", generator=g) < 0.2] = -torch.inf
    x[tokens // 2, experts - 1] = torch.inf
    for over in OVER:
        for dtype in TYPES:
            c = Case(tokens, experts, top_k, dtype, over, logits=x)
            c.check(*c.forward())


def test_all_to_one_expert_and_none():
    x = torch.full((300, 8), -torch.inf, device="cuda")
    c = Case(300, 8, 2, "fp32", "chosen", logits=x)
    out = c.forward()
    c.check(*out)
    assert out[3].tolist() == [0] * 9
    x[:, 5] = 0.0
    c = Case(300, 8, 2, "fp32", "chosen", logits=x)
    out = c.forward()
    c.check(*out)
    assert out[2][:, 0].tolist() == list(range(300))


def test_nan_is_reported_and_never_chosen():
    for tokens in (10, 100):
        c = Case(tokens, 16, 2, "fp32", "all")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        c.forward(status=status)
        assert status.item() == 0
        c.logits[3, 4] = torch.nan
        c.logits[5] = torch.nan
        c.check(*c.forward(status=status))
        assert status.item() == 4


@pytest.mark.parametrize("tokens,experts,top_k", [(20000, 64, 2), (70000, 300, 2)])
def test_many_tokens(tokens, experts, top_k):
    """More blocks than add up their own counts.  (The plan by stable sorts.)"""
    c = Case(tokens, experts, top_k, "bf16", "chosen")
    expert, weight, row, offset = c.forward()
    x = c.logits.float()
    want = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :top_k]
    assert torch.equal(expert.long(), want)
    order = torch.sort(want.flatten(), stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device="cuda")
    assert torch.equal(row.long().flatten(), place)
    count = torch.bincount(want.flatten(), minlength=experts)
    assert torch.equal(offset.long(), torch.cat((torch.zeros(1, device="cuda", dtype=torch.long), count.cumsum(0))))


@pytest.mark.parametrize("tokens,experts,top_k", [(1, 1, 1), (3, 8, 2), (100, 33, 6), (257, 64, 4), (40, 1024, 32), (999, 128, 8)])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("over", list(OVER))
def test_backward(tokens, experts, top_k, dtype, over):
    c = Case(tokens, experts, top_k, dtype, over)
    if tokens > 2:
        c.logits[1] = -torch.inf
        c.logits[2, 1:] = -torch.inf
        c.logits[0, 0] = torch.nan
    expert = c.forward()[0]
    dw = torch.randn(tokens, top_k, device="cuda", generator=c.g)
    dw[expert < 0] = torch.nan  # not used
    d = torch.full((tokens * experts + 8,), float(MARK), device="cuda", dtype=c.t)
    L.call("sky_route_bwd", c.shape, P(c.logits), P(expert.contiguous()), P(dw), P(d), stream())
    assert bool((d[-8:] == MARK).all())
    e = expert.cpu().numpy()
    want = ORC.route_backward(f64(c.logits), e, np.nan_to_num(f64(dw)), over)
    p = ORC.probabilities(f64(c.logits), e, over)
    # p (dw - s), s a sum of up to 32 products of p and dw: the errors are those of p, times |dw| and |s|
    size = p * (np.abs(np.nan_to_num(f64(dw))).max(-1, keepdims=True) * 2)
    got = f64(d[:-8]).reshape(tokens, experts)
    assert (np.abs(got - want) <= c.half_step * np.abs(want) + (60 + experts / 32) * 2.0 ** -23 * size + 1e-44).all()
    x = c.logits.clone()  # in place
    L.call("sky_route_bwd", c.shape, P(x), P(expert.contiguous()), P(dw), P(x), stream())
    assert torch.equal(x.view(-1), d[:-8])


def test_captured_and_replayed_on_other_logits():
    for tokens in (40, 500):
        c = Case(tokens, 32, 4, "fp32", "chosen")
        outs = [torch.empty(tokens, 4, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int32)]
        offset = torch.empty(33, dtype=torch.int32, device="cuda")
        ws = torch.empty(L.lib().sky_route_workspace_bytes(c.shape), dtype=torch.uint8, device="cuda")
        c.forward()  # loads the module before the capture
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            L.call("sky_route_fwd", c.shape, P(c.logits), *[P(o) for o in outs], P(offset), P(ws), ws.numel(), None, stream())
        for seed in (1, 2):
            c.logits.copy_(Case(tokens, 32, 4, "fp32", "chosen", seed=seed).logits)
            ws.fill_(0xff)
            graph.replay()
            torch.cuda.synchronize()
            c.check(*outs, offset)
