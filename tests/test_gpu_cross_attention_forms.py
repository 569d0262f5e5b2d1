"""Every form of the cross attention forward, chosen by the sizes that choose it: two
score buffers, one, one for keys of a single tile, keys split over two and four CTAs, few
rows on the tensor cores and on the CUDA cores, 16-row blocks there; rows whose offsets pass
2^31 values; calls on several streams and threads at once.  Bounds and layout are those of
test_gpu_cross_attention.
"""
import threading

import pytest

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


# lengths that leave splits without a tile, end a tile, and are 0 and 1, by form
RAGGED = {
    "two buffers": [0, 1, 64, 300], "one buffer": [200, 0, 1, 63, 64, 65, 128, 191, 192],
    "one buffer, four heads a tile": [0, 200, 1, 63, 64, 65, 127, 128, 129, 2, 130],
    "four splits": [945, 0, 1, 64, 65, 128], "four splits, whole heads": [0, 800, 65],
    "two splits": [1600, 0, 1, 64, 65, 128, 1599, 700, 63, 1], "two splits, two heads a tile": [0, 1600, 1, 64, 63, 65, 127, 129, 999, 2],
    "few rows": [0, 2500, 1, 32, 33], "few rows, 32": [2100, 0, 1], "few rows, CUDA cores": [1, 0, 700],
    "CUDA cores": [0, 1, 200],
}


@pytest.mark.parametrize("form", FORMS)
def test_ragged_lengths_with_anything_behind(form):
    sq, skv, heads, kv_heads, _, dtype = FORMS[form]
    c = Case(sq, skv, heads, kv_heads, RAGGED[form], dtype=dtype, beside=8).poison()
    ctx, lse = c.forward()
    c.check_forward(ctx, lse)
    again, lse2 = c.forward()
    assert torch.equal(ctx.buf, again.buf) and torch.equal(lse, lse2)
    assert torch.equal(c.forward(with_lse=False)[0].buf, ctx.buf)


@pytest.mark.parametrize("heads,kv_heads,B", [(16, 16, 9), (32, 8, 11)])
def test_keys_of_one_tile_under_many_blocks(heads, kv_heads, B):
    """One buffer by its own rule: a single tile of keys and more than two blocks an SM."""
    c = Case(300 if heads == 16 else 150, 40, heads, kv_heads, [40, 0, 1, 39, 33, 32, 31, 40, 2, 17, 40][:B], beside=8).poison()
    ctx, lse = c.forward()
    c.check_forward(ctx, lse)


@pytest.mark.parametrize("sq,skv,heads,kv_heads,lens,dim,shift,apart", [
    (6, 7, 2, 2, [7, 5], 64, 0, 3 << 26),     # few rows; one launch backward
    (6, 7, 2, 1, [7, 5], 64, 1, 3 << 26),     # CUDA cores
    (20, 135, 1, 1, [130], 64, 0, 1 << 24),   # tiles; three launches backward
    (9, 135, 1, 1, [135], 32, 0, 1 << 24),    # CUDA cores, 16-row blocks
])
def test_rows_past_32_bit_offsets(sq, skv, heads, kv_heads, lens, dim, shift, apart):
    c = Case(sq, skv, heads, kv_heads, lens, dim=dim, beside=apart, shift=shift)
    assert (len(lens) * max(sq, skv) - 1) * min(c.ld) > 1 << 31
    near = Case(sq, skv, heads, kv_heads, lens, dim=dim, beside=8 if shift == 0 else 1, shift=shift)
    for x in ("q", "k", "v", "dctx"):
        getattr(near, x).set(getattr(c, x).get().contiguous())

    def alike(x, y):
        return torch.equal(x.get(), y.get()) and x.untouched()
    (ctx, lse), (want, want_lse) = c.forward(), near.forward()
    assert alike(ctx, want) and torch.equal(lse, want_lse)
    for got, ref in zip(c.backward(ctx, lse), near.backward(want, want_lse)):
        assert alike(got, ref)
    near.check_forward(want, want_lse)


@pytest.mark.parametrize("threads", [False, True])
def test_calls_at_once(threads):
    """Forwards and backwards of every kind on six streams, a workspace each, from one thread
    or from six: the bits of calls made alone."""
    shapes = [(40, 945, 6, 3, [945, 300], "bf16", 64), (300, 200, 16, 16, [200, 65, 128], "bf16", 64),
              (1, 2500, 8, 2, [2500, 65], "bf16", 64), (700, 100, 8, 2, [100, 64], "bf16", 64),
              (50, 340, 2, 2, [340, 65], "fp32", 64), (33, 150, 4, 2, [150, 80], "bf16", 128)]
    cases = [Case(*s[:5], dtype=s[5], dim=s[6]) for s in shapes]
    alone = []
    for c in cases:
        ctx, lse = c.forward()
        alone.append((ctx, lse, c.backward(ctx, lse)))
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [(c.new["ctx"](), torch.empty_like(a[1]), [c.new[n]() for n in ("dq", "dk", "dv")],
             torch.empty(L.lib().sky_cross_attention_bwd_workspace_bytes(c.shape), dtype=torch.uint8, device="cuda"))
            for c, a in zip(cases, alone)]
    torch.cuda.synchronize()
    failed = []

    def work(i, rounds):
        try:
            torch.cuda.set_device(0)
            c, (ctx, lse, grads, ws), st = cases[i], outs[i], streams[i].cuda_stream
            for _ in range(rounds):
                L.call("sky_cross_attention_fwd", c.shape, c.q.ptr(), c.k.ptr(), c.v.ptr(), P(c.d_len), ctx.ptr(), P(lse),
                       None, st)
                L.call("sky_cross_attention_bwd", c.shape, c.q.ptr(), c.k.ptr(), c.v.ptr(), ctx.ptr(), c.dctx.ptr(), P(lse),
                       P(c.d_len), *[g.ptr() for g in grads], P(ws), ws.numel(), None, st)
        except Exception as e:  # noqa: BLE001  (of another thread: told below)
            failed.append(e)
    if threads:
        ts = [threading.Thread(target=work, args=(i, 20)) for i in range(len(cases))]
        for t in ts:
            t.start()
        for t in ts:
            t.join()
    else:
        for _ in range(20):
            for i in range(len(cases)):
                work(i, 1)
    torch.cuda.synchronize()
    assert not failed
    for (ctx, lse, grads), (c2, l2, g2, _) in zip(alone, outs):
        assert torch.equal(ctx.buf, c2.buf) and torch.equal(lse, l2)
        assert all(torch.equal(x.buf, y.buf) for x, y in zip(grads, g2))


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


class Behind:
    """The rows from `n` on of a gradient of keys."""

    def __init__(self, rows, n):
        self.rows, self.n = rows, n

    def get(self):
        return self.rows.get()[:, self.n:]


@pytest.mark.parametrize("sq,skv,heads,kv_heads,lens,dtype,dim", [
    (200, 300, 4, 2, [300, 65, 129], "bf16", 64), (40, 945, 6, 3, [945, 65, 66], "bf16", 64),
    (900, 120, 2, 2, [120, 65], "bf16", 64), (30, 120, 2, 2, [120, 65], "bf16", 64),  # many queries; one launch
    (50, 200, 2, 1, [200, 66], "bf16", 96), (50, 200, 2, 1, [200, 66], "fp32", 64),
])
def test_gradients_behind_keys_that_score_minus_infinity(sq, skv, heads, kv_heads, lens, dtype, dim):
    """Those keys' own gradients are 0, and the others' and the queries' as without them."""
    c = Case(sq, skv, heads, kv_heads, lens, dtype=dtype, dim=dim)
    d = Case(sq, skv - 64, heads, kv_heads, [n - 64 for n in lens], dtype=dtype, dim=dim)
    q, k = c.q.get().clone(), c.k.get().clone()
    q[..., 0] = q[..., 0].abs() + 4.0
    for x, y in ((d.q, q), (d.k, k[:, 64:]), (d.v, c.v.get()[:, 64:]), (d.dctx, c.dctx.get())):
        x.set(y.contiguous())
    k[:, :64, :, 0] = -3e38
    c.q.set(q)
    c.k.set(k)
    ctx, lse = d.given()
    dq, dk, dv = c.backward(c.new["ctx"]().set(ctx.get().contiguous()), lse)
    assert not bool(dk.get()[:, :64].any()) and not bool(dv.get()[:, :64].any())
    d.check_backward((dq, Behind(dk, 64), Behind(dv, 64)))


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
