"""dot(dctx, ctx) in the backward: formed from P and dP in 32 bits, not from the rounded ctx,
whose rounding would be the same for every key of a row and outgrow dS where V has a mean or
one key takes nearly all of a row.

Norms of the gradients' errors against float64.  q and k are multiples of 1/8, v of 1/8 and
dctx of 1/128, so that scores and dP are exact in 32 bits (sums below 2^24 of their units).
Roundings to bf16 are off by at most h = 2^-8 of a value (half a step), h / sqrt(3) of it in
the root mean square; those of dS (a product's operand) and of the stored gradients are
independent, so with c = 1 / sqrt(D)
  |err dq|^2 <= h^2 / 3 (c^2 sum dS^2 K^2 + dq^2)
over all rows and keys (dk: over all keys and rows, with Q), to a quarter of its root for the
spread and that the steps are not uniform.  fp32 arithmetic adds at most, element by element:
P is off by e = ln 2 (2^-24 (|s| + 2 |lse|) + 2^-22) + 2^-21 of it (the exponent's rounding,
the log-sum-exp's, the exponential's), for dk 2^-17 |lse| more; dS by e |dS| + P (e |delta| +
2^-17 |delta| for dk + the rounding of delta's sum: a thread adds an eighth of the keys at
most, (n / 8 + 12) 2^-24 of the terms); products' sums by (n + 8) 2^-24 of their terms.
"""
import numpy as np
import pytest

from oracle import heads_f64 as ORC
from test_gpu_cross_attention import U, Case, f64

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")

H = 2.0 ** -8


def limits(c):
    """What the errors of dq and dk may be, in norm."""
    q, k, v, dctx = c.inputs()
    dq, dk, _ = ORC.cross_attention_backward(q, k, v, dctx, c.lens)
    _, lse = ORC.cross_attention(q, k, v, c.lens)
    s = c.dim ** -0.5
    chance = [np.square(dq).sum(), np.square(dk).sum()]
    sure = [np.zeros(dq.shape), np.zeros(dk.shape)]
    rows = c.sq * (c.heads // c.kv_heads)
    for b, a, g, n, qq, kk, vv, dd, p, _ in c.walk():
        dp = dd @ vv.T
        delta = (p * dp).sum(-1, keepdims=True)
        ds = p * (dp - delta)
        z = np.abs(lse[b, a])[:, None]
        e = np.log(2.0) * (U * (np.abs(qq @ kk.T) * s * np.log2(np.e) + 2 * z) + 2.0 ** -22) + 2.0 ** -21
        for i, (x, terms, table) in enumerate(((kk, n, 0.0), (qq, rows, 2.0 ** -17))):
            eds = np.abs(ds) * (e + table * z + (terms + 8) * U) + p * (
                (e + table * (1 + z)) * np.abs(delta) + (n / 8 + 12) * U * (p * np.abs(dp)).sum(-1, keepdims=True))
            y, w = (eds, ds) if i == 0 else (eds.T, ds.T)
            chance[i] += s * s * (np.square(w) @ np.square(x)).sum()
            if i == 0:
                sure[0][b, :, a] = s * (y @ np.abs(x))
            else:
                sure[1][b, :n, g] += s * (y @ np.abs(x))
    return (dq, dk), [1.25 * H * np.sqrt(x / 3) + np.linalg.norm(y) for x, y in zip(chance, sure)]


def check(c, mean):
    for x, unit, add in ((c.q, 8, 0), (c.k, 8, 0), (c.v, 8, mean), (c.dctx, 128, 0)):
        x.set(((x.get().float() * unit).round() / unit + add).contiguous())  # (NaN and infinities stay)
    want, bound = limits(c)
    grads = c.backward(*c.given())
    for got, w, most, name in zip(grads, want, bound, ("dq", "dk")):
        off, size = np.linalg.norm(f64(got.get()) - w), np.linalg.norm(w)
        assert off <= most, f"{name}: off by {off / size:.2e} of its norm, within {most / size:.2e}"


@pytest.mark.parametrize("mean,scale", [(0, 1.0), (1, 1.0), (4, 1.0), (4, 1.5), (0, 2.5)])
@pytest.mark.parametrize("sq,skv,heads,kv_heads,lens", [
    (64, 512, 2, 2, [512, 300]), (200, 300, 4, 2, [300, 17, 0, 128]), (333, 1000, 2, 2, [1000]),
    (40, 945, 6, 3, [945, 66, 0]),      # keys of a block over a cluster
    (1100, 100, 2, 2, [100, 64]),       # more than eight query tiles of few keys
    (130, 150, 32, 16, [150, 1, 64, 149, 33, 130, 128, 129, 0, 100]),  # more than two blocks an SM
    (30, 70, 4, 2, [70, 33]),           # one launch
])
def test_mean_of_v_and_peaked_scores(sq, skv, heads, kv_heads, lens, mean, scale):
    check(Case(sq, skv, heads, kv_heads, lens, scale=scale, beside=8).poison(), mean)


@pytest.mark.parametrize("B,sq,skv,heads,kv_heads", [(3, 20, 2000, 16, 4), (1, 5, 3000, 2, 1), (2, 129, 500, 3, 1)])
def test_keys_of_few_rows(B, sq, skv, heads, kv_heads):
    check(Case(sq, skv, heads, kv_heads, [skv - 61 * b for b in range(B)]).poison(), 2)


@pytest.mark.parametrize("mean", [0, 4])
@pytest.mark.parametrize("sq,skv,heads,kv_heads,lens,dim,shift", [
    (64, 300, 4, 2, [300, 129, 0], 128, 0), (37, 200, 3, 3, [200, 1], 64, 1), (130, 90, 2, 1, [90, 64], 32, 0),
    (9, 1500, 2, 1, [1500, 65, 7], 80, 0), (16, 16, 4, 4, [16, 3], 33, 1), (3, 3000, 1, 1, [2999], 20, 0),
])
def test_mean_of_v_on_the_cuda_cores(sq, skv, heads, kv_heads, lens, dim, shift, mean):
    check(Case(sq, skv, heads, kv_heads, lens, dim=dim, beside=shift, shift=shift).poison(), mean)


@pytest.mark.parametrize("sq,skv,heads,kv_heads,lens", [(200, 300, 2, 2, [300, 129]), (90, 700, 3, 1, [700]),
                                                        (1100, 120, 1, 1, [120])])
def test_scores_in_the_thousands(sq, skv, heads, kv_heads, lens):
    """Rows that one key takes whole, at scores up to 3100: P is 1 there, as far as dV has the
    log-sum-exp.

    A head's first value is in q an integer from 32 to 63, in k a multiple of 8 up to 384, of the
    last key 392; its second in q a multiple of 1/16 below 8, in k 1; the others are 0.  So the
    scores are exact, of 19 bits, and every other at least 32 below the last key's, P there
    below e^-32.  That key's P is off by the log-sum-exp's rounding and the accumulator's, 3 x 2^-24
    of it, times ln 2, less than the half step 2^-9 below 1 (asserted), so it rounds to 1: dv is a
    sum of dctx rounded once.  (With the log-sum-exp to 2^-18 P would be off by 0.6 to 1.2e-2.)"""
    c = Case(sq, skv, heads, kv_heads, lens)
    g = np.random.default_rng(sq)
    q, k = np.zeros(c.q.get().shape, np.float32), np.zeros(c.k.get().shape, np.float32)
    q[..., 0] = g.integers(32, 64, q.shape[:-1])
    q[..., 1] = g.integers(0, 128, q.shape[:-1]) / 16
    k[..., 0], k[..., 1] = (np.arange(skv) % 49 * 8)[None, :, None], 1
    for b, n in enumerate(lens):
        k[b, n - 1, :, 0] = 392
    c.q.set(q)
    c.k.set(k)
    qq, kk, vv, dd = c.inputs()
    _, z = ORC.cross_attention(qq, kk, vv, lens)
    assert np.log(2.0) * 3 * U * np.abs(z).max() + 2.0 ** -21 < 2.0 ** -9
    want = ORC.cross_attention_backward(qq, kk, vv, dd, lens)[2]
    rows = sq * (heads // kv_heads)
    most = np.abs(dd).sum(1).reshape(len(lens), kv_heads, -1, c.dim).sum(2)[:, None]
    off = np.abs(f64(c.backward(*c.given())[2].get()) - want)
    assert (off <= H * np.abs(want) + ((rows + 8) * U + np.exp(-30.0)) * most).all(), off.max()
