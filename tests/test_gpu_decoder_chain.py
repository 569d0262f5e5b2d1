"""Cross attention's gradient of a slice's states taken on through the slice's own backward,
to the slice's input, against float64 from end to end."""
import numpy as np
import pytest

from oracle import heads_f64 as ORC
from paper_2202_11836_gb300 import _lib as L
from paper_2202_11836_gb300 import synth
from paper_2202_11836_gb300.slice import EncoderSlice
from parity_util import TOL, l2rel, oracle_slice, to_device, to_host
from test_gpu_decoder_attention import BF, D, P, empty, f64, gemm, stream, workspace

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("S,lens", [(80, [80, 33, 1]), (150, [150, 64, 129])])
def test_gradient_through_the_slice(S, lens):
    """The slice's backward is within 5e-3 of its incoming gradient's float64 (its own tolerance), and
    that gradient within 1.2e-2 (test_gpu_decoder_attention): 1.7e-2 together."""
    B, T, H, heads, kv_heads = 3, 37, 256, 4, 2
    w = synth.custom("enc", layers=1, hidden=H, heads=4, ffn=512, seq=S, batch=B)
    lens, params, X = np.array(lens, np.int32), synth.slice_params(w), synth.activations(w, batch=B)
    d_len = torch.tensor(lens, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(7)
    rnd = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    qw, kw = heads * D, kv_heads * D
    q, wkv, dctx = rnd(B * T, qw), rnd(2 * kw, H, std=0.06), rnd(B * T, qw, std=0.1)
    with EncoderSlice(H, 4, 512, 0, 1, B, S, "bf16") as enc:
        enc.set_params(0, params[0])
        states = enc.forward(to_device(X, "bf16"), d_len)
        kv = gemm(L.SKY_GEMM_XWT, B * S, 2 * kw, H, states.view(B * S, H), wkv, empty(B * S, 2 * kw))
        sh = L.SkyCrossShape(B, T, S, heads, kv_heads, D, BF, qw, 2 * kw, 2 * kw, qw)
        ctx, lse = empty(B * T, qw), empty(B, heads, T, dtype=torch.float32)
        L.call("sky_cross_attention_fwd", sh, P(q), P(kv), P(kv, kw), P(d_len), P(ctx), P(lse), None, stream())
        dq, dkv = empty(B * T, qw), empty(B * S, 2 * kw)
        ws = workspace(L.lib().sky_cross_attention_bwd_workspace_bytes(sh))
        L.call("sky_cross_attention_bwd", sh, P(q), P(kv), P(kv, kw), P(ctx), P(dctx), P(lse), P(d_len), P(dq), P(dkv),
               P(dkv, kw), P(ws), ws.numel(), None, stream())
        dstates = gemm(L.SKY_GEMM_XW, B * S, H, 2 * kw, dkv, wkv, empty(B * S, H))
        dx = enc.backward(dstates.view(B, S, H))
        enc.sync()
    Y = oracle_slice(w, X, lens, np.zeros_like(X), params)[0]
    KV = (Y.reshape(B * S, H) @ f64(wkv).T).reshape(B, S, 2, kv_heads, D)
    _, dK, dV = ORC.cross_attention_backward(f64(q).reshape(B, T, heads, D), KV[:, :, 0], KV[:, :, 1],
                                             f64(dctx).reshape(B, T, heads, D), lens)
    dKV = np.concatenate((dK.reshape(B * S, kw), dV.reshape(B * S, kw)), 1)
    want = oracle_slice(w, X, lens, (dKV @ f64(wkv)).reshape(B, S, H), params)[1]
    assert l2rel(to_host(dx), want) <= TOL["bf16"]["l2rel"] + 1.2e-2
