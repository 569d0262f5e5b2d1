"""The head norms and cross attention as a decoder runs them on a slice's output: project,
norm, attend, and all the way back to both projections' inputs; and self attention over a
packed QKV projection whose queries and keys are normed and turned.  Against float64."""
import ctypes as C

import numpy as np
import pytest

from oracle import heads_f64 as ORC
from paper_2202_11836_gb300 import _lib as L
from paper_2202_11836_gb300 import synth
from paper_2202_11836_gb300.slice import EncoderSlice

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS, THETA, D = 1e-6, 10000.0, 64
BF = L.SKY_DTYPE_BF16


def P(t, at=0):
    return C.c_void_p(int(t.data_ptr()) + at * t.element_size())


def stream():
    return C.c_void_p(int(torch.cuda.current_stream().cuda_stream))


def f64(t):
    return t.double().cpu().numpy()


def gemm(form, M, N, K, a, b, out):
    f32 = out.dtype == torch.float32
    n = L.lib().sky_gemm_workspace_bytes(form, M, N, K, BF, 1 if f32 else 0)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    L.call("sky_gemm", form, M, N, K, BF, P(a), P(b), P(out), 1 if f32 else 0, L.SKY_EPI_STORE, None, None, None, P(ws),
           n, None, stream())
    return out


def empty(*shape, dtype=torch.bfloat16):
    return torch.full(shape, float("nan"), device="cuda", dtype=dtype)


def l2(got, want):
    return np.linalg.norm(f64(got) - want) / np.linalg.norm(want)


def workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def test_decoder_over_a_slices_states():
    """Every bf16 tensor on the way is rounded once (2^-9 rms of 3^-1/2 of it, 1.7e-3 of its norm): the
    forward passes six such roundings, the gradients twice as many, each about
    independent of the others: 4.2e-3 and 6e-3; bounds twice that."""
    B, S, T, H, heads, kv_heads = 3, 80, 37, 256, 4, 2
    w = synth.custom("enc", layers=1, hidden=H, heads=4, ffn=512, seq=S, batch=B)
    lens = np.array([80, 33, 1], np.int32)
    d_len = torch.tensor(lens, device="cuda")
    with EncoderSlice(H, 4, 512, 0, 1, B, S, "bf16") as enc:
        enc.set_params(0, synth.slice_params(w)[0])
        states = enc.forward(torch.from_numpy(synth.activations(w, batch=B)).cuda().bfloat16(), d_len).clone()
        enc.sync()
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    x = rnd(B * T, H)
    wq, wkv = rnd(heads * D, H, std=0.06), rnd(2 * kv_heads * D, H, std=0.06)
    gq, gk = rnd(D, std=0.1) + 1.5, rnd(D, std=0.1) + 1.0
    dctx = rnd(B * T, heads * D, std=0.1)
    qw, kw = heads * D, kv_heads * D

    def shape(rows, nq, nk, ld, ldy):
        return L.SkyQkNormShape(rows, nq, nk, D, BF, ld, ldy, EPS, L.SKY_ROTATE_NONE, 0.0)

    # forward: Q = norm(x Wq^T), K | V = states Wkv^T with K normed in place
    q0 = gemm(L.SKY_GEMM_XWT, B * T, qw, H, x, wq, empty(B * T, qw))
    kv = gemm(L.SKY_GEMM_XWT, B * S, 2 * kw, H, states.view(B * S, H), wkv, empty(B * S, 2 * kw))
    q, k0 = empty(B * T, qw), kv.clone()
    sq, sk = shape(B * T, heads, 0, qw, qw), shape(B * S, 0, kv_heads, 2 * kw, 2 * kw)
    L.call("sky_qk_norm_fwd", sq, P(q0), P(gq), None, None, P(q), stream())
    L.call("sky_qk_norm_fwd", sk, P(kv), None, P(gk), None, P(kv), stream())
    sh = L.SkyCrossShape(B, T, S, heads, kv_heads, D, BF, qw, 2 * kw, 2 * kw, qw)
    ctx, lse = empty(B * T, qw), empty(B, heads, T, dtype=torch.float32)
    L.call("sky_cross_attention_fwd", sh, P(q), P(kv), P(kv, kw), P(d_len), P(ctx), P(lse), None, stream())
    # backward, the K half of the gradient rows taken through the norm in place
    dq, dkv = empty(B * T, qw), empty(B * S, 2 * kw)
    ws = workspace(L.lib().sky_cross_attention_bwd_workspace_bytes(sh))
    L.call("sky_cross_attention_bwd", sh, P(q), P(kv), P(kv, kw), P(ctx), P(dctx), P(lse), P(d_len), P(dq), P(dkv),
           P(dkv, kw), P(ws), ws.numel(), None, stream())
    dgq, dgk = empty(D, dtype=torch.float32), empty(D, dtype=torch.float32)
    for s, inp, d, gains, grads in ((sq, q0, dq, (P(gq), None), (P(dgq), None)), (sk, k0, dkv, (None, P(gk)), (None, P(dgk)))):
        ws = workspace(L.lib().sky_qk_norm_bwd_workspace_bytes(s))
        L.call("sky_qk_norm_bwd", s, P(inp), P(d), *gains, None, P(d), *grads, P(ws), ws.numel(), stream())
    dx = gemm(L.SKY_GEMM_XW, B * T, H, qw, dq, wq, empty(B * T, H))
    dstates = gemm(L.SKY_GEMM_XW, B * S, H, 2 * kw, dkv, wkv, empty(B * S, H))
    dwkv = gemm(L.SKY_GEMM_XTW, 2 * kw, H, B * S, dkv, states.view(B * S, H), empty(2 * kw, H, dtype=torch.float32))
    torch.cuda.synchronize()

    X, Y, Wq, Wkv = f64(x), f64(states).reshape(B * S, H), f64(wq), f64(wkv)
    Q0, KV = (X @ Wq.T).reshape(B * T, heads, D), (Y @ Wkv.T).reshape(B * S, 2, kv_heads, D)
    pos = np.zeros(1)
    norm = lambda h, gain: ORC.head_norm(h, np.tile(f64(gain), (h.shape[1], 1)), pos, EPS, "none", 1.0)  # noqa: E731
    back = lambda h, d, gain: ORC.head_norm_backward(h, d, np.tile(f64(gain), (h.shape[1], 1)), pos, EPS, "none", 1.0)  # noqa: E731
    Q, K, V = norm(Q0, gq).reshape(B, T, heads, D), norm(KV[:, 0], gk).reshape(B, S, kv_heads, D), KV[:, 1].reshape(B, S, kv_heads, D)
    want, want_lse = ORC.cross_attention(Q, K, V, lens)
    G = f64(dctx).reshape(B, T, heads, D)
    dQ, dK, dV = ORC.cross_attention_backward(Q, K, V, G, lens)
    dQ0, tq = back(Q0, dQ.reshape(Q0.shape), gq)
    dK0, tk = back(KV[:, 0], dK.reshape(B * S, kv_heads, D), gk)
    dKV = np.concatenate((dK0.reshape(B * S, kw), dV.reshape(B * S, kw)), 1)
    assert l2(ctx, want.reshape(B * T, qw)) <= 8.4e-3
    assert np.abs(f64(lse) - want_lse).max() <= 0.05  # six roundings of scores of size ten
    for got, ref in ((dx, dQ0.reshape(B * T, qw) @ Wq), (dstates, dKV @ Wkv), (dwkv, dKV.T @ Y), (dgq, tq.sum((0, 1))),
                     (dgk, tk.sum((0, 1)))):
        assert l2(got, ref) <= 1.2e-2, l2(got, ref)


def test_self_attention_over_normed_and_turned_heads():
    """q and k from the norm's output, v from the projection itself: three row distances; the
    gradients of all three land in the projection's own rows.  Two roundings of the
    inputs' heads and one of the result (1.7e-3 each): 3e-3, the gradients twice that."""
    B, S, heads, kv_heads = 2, 150, 6, 3
    width, nd = (heads + 2 * kv_heads) * D, (heads + kv_heads) * D
    g = torch.Generator(device="cuda").manual_seed(9)
    qkv = torch.randn(B * S, width, device="cuda", generator=g).bfloat16()
    gains = [(1 + 0.1 * torch.randn(D, device="cuda", generator=g)).bfloat16() for _ in range(2)]
    pos = torch.arange(S, dtype=torch.int32, device="cuda").repeat(B) + 1000
    lens = np.array([150, 70], np.int32)
    d_len = torch.tensor(lens, device="cuda")
    dctx = (0.1 * torch.randn(B * S, heads * D, device="cuda", generator=g)).bfloat16()
    ns = L.SkyQkNormShape(B * S, heads, kv_heads, D, BF, width, nd, EPS, L.SKY_ROTATE_HALVES, THETA)
    cs = L.SkyCrossShape(B, S, S, heads, kv_heads, D, BF, nd, nd, width, heads * D)
    qk, ctx, lse = empty(B * S, nd), empty(B * S, heads * D), empty(B, heads, S, dtype=torch.float32)
    dqk, dqkv = empty(B * S, nd), empty(B * S, width)
    dg = [empty(D, dtype=torch.float32) for _ in range(2)]
    ws1, ws2 = workspace(L.lib().sky_cross_attention_bwd_workspace_bytes(cs)), workspace(L.lib().sky_qk_norm_bwd_workspace_bytes(ns))

    def step():
        L.call("sky_qk_norm_fwd", ns, P(qkv), P(gains[0]), P(gains[1]), P(pos), P(qk), stream())
        L.call("sky_cross_attention_fwd", cs, P(qk), P(qk, heads * D), P(qkv, nd), P(d_len), P(ctx), P(lse), None, stream())
        L.call("sky_cross_attention_bwd", cs, P(qk), P(qk, heads * D), P(qkv, nd), P(ctx), P(dctx), P(lse), P(d_len),
               P(dqk), P(dqk, heads * D), P(dqkv, nd), P(ws1), ws1.numel(), None, stream())
        L.call("sky_qk_norm_bwd", ns, P(qkv), P(dqk), P(gains[0]), P(gains[1]), P(pos), P(dqkv), P(dg[0]), P(dg[1]),
               P(ws2), ws2.numel(), stream())

    step()
    torch.cuda.synchronize()
    first = [t.clone() for t in (ctx, lse, dqkv, *dg)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (qk, ctx, lse, dqk, dqkv, *dg):
        t.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, (ctx, lse, dqkv, *dg)))

    x = f64(qkv).reshape(B * S, -1, D)
    gain = np.concatenate([np.tile(f64(gains[0]), (heads, 1)), np.tile(f64(gains[1]), (kv_heads, 1))])
    QK = ORC.head_norm(x[:, :heads + kv_heads], gain, f64(pos), EPS, "halves", THETA).reshape(B, S, -1, D)
    V = x[:, heads + kv_heads:].reshape(B, S, kv_heads, D)
    want, _ = ORC.cross_attention(QK[:, :, :heads], QK[:, :, heads:], V, lens)
    dQ, dK, dV = ORC.cross_attention_backward(QK[:, :, :heads], QK[:, :, heads:], V, f64(dctx).reshape(B, S, heads, D), lens)
    dX, terms = ORC.head_norm_backward(x[:, :heads + kv_heads], np.concatenate((dQ, dK), 2).reshape(B * S, -1, D), gain,
                                       f64(pos), EPS, "halves", THETA)
    assert l2(ctx, want.reshape(B * S, -1)) <= 6e-3
    assert l2(dqkv, np.concatenate((dX.reshape(B * S, -1), dV.reshape(B * S, -1)), 1)) <= 1.2e-2
    assert l2(dg[0], terms[:, :heads].sum((0, 1))) <= 1.2e-2 and l2(dg[1], terms[:, heads:].sum((0, 1))) <= 1.2e-2


@pytest.mark.parametrize("rows_at_once", [1, 2])
def test_tokens_one_by_one_equal_the_whole(rows_at_once):
    """Writing token by token over kept keys gives what all queries at once give: the same
    products in other kernels, each result rounded once more than the scores (2^-8)."""
    B, T, S, heads, kv_heads = 2, 6, 200, 8, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    q0 = torch.randn(B, T, heads * D, device="cuda", generator=g).bfloat16()
    kv = torch.randn(B, S, 2 * kv_heads * D, device="cuda", generator=g).bfloat16()
    d_len = torch.tensor([200, 77], dtype=torch.int32, device="cuda")
    gain = (1 + 0.1 * torch.randn(D, device="cuda", generator=g)).bfloat16()

    def run(q, pos):
        b, t, w = q.shape
        y, ctx = torch.empty_like(q), torch.empty_like(q)
        ns = L.SkyQkNormShape(b * t, heads, 0, D, BF, w, w, EPS, L.SKY_ROTATE_PAIRS, THETA)
        L.call("sky_qk_norm_fwd", ns, P(q), P(gain), None, P(pos), P(y), stream())
        cs = L.SkyCrossShape(b, t, S, heads, kv_heads, D, BF, w, 2 * kv_heads * D, 2 * kv_heads * D, w)
        L.call("sky_cross_attention_fwd", cs, P(y), P(kv), P(kv, kv_heads * D), P(d_len), P(ctx), None, None, stream())
        torch.cuda.synchronize()
        return y, ctx

    pos = torch.arange(T, dtype=torch.int32, device="cuda").repeat(B, 1) + 5000
    y, whole = run(q0, pos.contiguous())
    for t in range(0, T, rows_at_once):
        part = slice(t, t + rows_at_once)
        yt, ct = run(q0[:, part].contiguous(), pos[:, part].contiguous())
        assert torch.equal(yt, y[:, part])
        diff = (ct.double() - whole[:, part].double()).abs()
        assert bool((diff <= 2.0 ** -7 * (whole[:, part].double().abs() + kv.double().abs().mean())).all())
