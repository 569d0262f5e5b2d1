"""Every form of the cross attention forward, chosen by the sizes that choose it: two
score buffers, one, one for keys of a single tile, keys split over two and four CTAs, few
rows on the tensor cores and on the CUDA cores, 16-row blocks there.  Bounds and layout
are those of test_gpu_cross_attention.
"""
import numpy as np
import pytest

from oracle import heads_f64 as ORC
from paper_2202_11836_gb300 import _lib as L
from test_gpu_cross_attention import Case, P, stream

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# queries, keys, heads, key heads, valid lengths, type.  The tiled kernel's form goes by its
# CTAs (128-row tiles of all heads and sequences) against 152 SMs: one buffer from 2.6 an SM
# on (for keys of one tile from two on), four splits up to half of one and from 12 tiles of
# 64 keys on, two up to one and from 24 on.
FORMS = {
    "two buffers": (200, 300, 2, 2, [300, 65, 129, 192], "bf16"),
    "one buffer": (300, 200, 16, 16, [200, 65, 128, 127, 129, 199, 150, 192, 193], "bf16"),
    "one buffer, four heads a tile": (150, 200, 32, 8, [200, 65, 128, 127, 129, 199, 150, 192, 193, 66, 100], "bf16"),
    "four splits": (40, 945, 6, 3, [945, 65, 66, 130, 200, 700], "bf16"),
    "four splits, whole heads": (300, 800, 5, 5, [800, 65, 130], "bf16"),
    "two splits": (100, 1600, 10, 10, [1600, 65, 66, 128, 129, 700, 1599, 1537, 1000, 200], "bf16"),
    "two splits, two heads a tile": (60, 1600, 20, 10, [1600, 65, 66, 128, 129, 700, 1599, 1537, 1000, 200], "bf16"),
    "few rows": (1, 2500, 8, 2, [2500, 65, 96, 97, 129], "bf16"),
    "few rows, 32": (32, 2100, 2, 2, [2100, 65, 700], "bf16"),
    "few rows, CUDA cores": (2, 700, 6, 2, [700, 65, 129], "fp32"),
    "CUDA cores": (150, 200, 4, 2, [200, 65, 130], "fp32"),
}


@pytest.mark.parametrize("form", FORMS)
def test_first_keys_that_score_minus_infinity(form):
    """64 keys whose scores leave fp32 downwards, before others: the answer is that of the
    others alone."""
    sq, skv, heads, kv_heads, lens, dtype = FORMS[form]
    c = Case(sq, skv, heads, kv_heads, lens, dtype=dtype)
    q, k, v = c.q.get().clone(), c.k.get().clone(), c.v.get().clone()
    q[..., 0] = q[..., 0].abs() + 4.0
    d = Case(sq, skv - 64, heads, kv_heads, [n - 64 for n in lens], dtype=dtype)
    d.q.set(q)
    d.k.set(k[:, 64:].contiguous())
    d.v.set(v[:, 64:].contiguous())
    k[:, :64, :, 0] = -3e38
    c.q.set(q)
    c.k.set(k)
    d.check_forward(*c.forward())


@pytest.mark.parametrize("B,S,heads", [(2, 200, 2), (9, 300, 16), (1, 900, 2)])
def test_first_keys_that_score_minus_infinity_in_self_attention(B, S, heads):
    """The same over packed QKV rows: two buffers, one, four splits."""
    g = torch.Generator(device="cuda").manual_seed(S)
    qkv = torch.randn(B, S, 3, heads, 64, device="cuda", generator=g).bfloat16()
    qkv[:, :, 0, :, 0] = qkv[:, :, 0, :, 0].abs() + 4.0
    qkv[:, :64, 1, :, 0] = -3e38
    lens = torch.full((B,), S, dtype=torch.int32, device="cuda")
    ctx = torch.empty(B, S, heads * 64, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(B, heads, S, device="cuda")
    L.call("sky_attention_fwd", P(qkv), P(lens), B, S, heads * 64, heads, L.SKY_DTYPE_BF16, P(ctx), P(lse), None, stream())
    torch.cuda.synchronize()
    # a case of cross attention whose inputs and bounds are those of the other keys
    d = Case(S, S - 64, heads, heads, [S - 64] * B)
    d.q.set(qkv[:, :, 0].contiguous())
    d.k.set(qkv[:, 64:, 1].contiguous())
    d.v.set(qkv[:, 64:, 2].contiguous())
    d.check_forward(d.new["ctx"]().set(ctx), lse)
