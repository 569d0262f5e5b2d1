"""The float64 definitions of the head norms and of cross attention, pinned to facts
outside them: closed forms, central differences, and the mistakes that they catch."""
import numpy as np
import pytest

from oracle import heads_f64 as ORC

EPS = 1e-5


def differences(f, x, step=1e-6):
    """Central differences of the scalar f at every value of x."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + step
        up = f()
        x[i] = old - step
        g[i] = (up - f()) / (2 * step)
        x[i] = old
    return g


@pytest.mark.parametrize("rotation", ["none", "halves", "pairs"])
def test_norm_gradients_are_differences(rotation):
    g = np.random.default_rng(1)
    x, dy = g.normal(size=(3, 2, 8)), g.normal(size=(3, 2, 8))
    gain, pos = 1 + 0.3 * g.normal(size=(2, 8)), np.array([0, 5, 1000])
    f = lambda: (ORC.head_norm(x, gain, pos, EPS, rotation, 100.0) * dy).sum()  # noqa: E731
    dx, terms = ORC.head_norm_backward(x, dy, gain, pos, EPS, rotation, 100.0)
    assert np.abs(dx - differences(f, x)).max() < 1e-7
    assert np.abs(terms.sum(0) - differences(f, gain)).max() < 1e-7


def test_norm_closed_forms():
    x = np.array([[[3.0, 4.0]]])
    one = np.ones((1, 2))
    r = np.sqrt(12.5)
    assert np.allclose(ORC.head_norm(x, one, [0], 0.0, "halves", 10.0), x / r)
    # pair 0 turns by pos radians, whatever theta is
    y = ORC.head_norm(x, one, [1], 0.0, "pairs", 10.0)[0, 0] * r
    assert np.allclose(y, [3 * np.cos(1) - 4 * np.sin(1), 3 * np.sin(1) + 4 * np.cos(1)])
    # the second of four dims' pairs turns by pos / sqrt(theta): 1 and 3 in halves, 2 and 3 as neighbours
    x = np.array([[[0.0, 1.0, 0.0, 0.0]]])
    assert np.allclose(ORC.rotate(x, ORC.turn_angles([np.pi * 5], 4, 100.0), "halves"), [[[0, 0, 0, 1]]])
    x = np.array([[[0.0, 0.0, 1.0, 0.0]]])
    assert np.allclose(ORC.rotate(x, ORC.turn_angles([np.pi * 5], 4, 100.0), "pairs"), [[[0, 0, 0, 1]]])


@pytest.mark.parametrize("rotation", ["halves", "pairs"])
def test_turned_products_depend_on_distance(rotation):
    g = np.random.default_rng(2)
    q, k = g.normal(size=(1, 1, 16)), g.normal(size=(1, 1, 16))
    turn = lambda x, p: ORC.rotate(x, ORC.turn_angles([p], 16, 50.0), rotation)  # noqa: E731
    a = (turn(q, 7) * turn(k, 3)).sum()
    assert np.isclose(a, (turn(q, 104) * turn(k, 100)).sum()) and not np.isclose(a, (turn(q, 8) * turn(k, 3)).sum())
    assert np.allclose(ORC.rotate(turn(q, 9), ORC.turn_angles([9], 16, 50.0), rotation, back=True), q)


def cross_case(lens, heads=4, kv_heads=2, sq=3, skv=5, dim=4, seed=3):
    g = np.random.default_rng(seed)
    B = len(lens)
    return (g.normal(size=(B, sq, heads, dim)), g.normal(size=(B, skv, kv_heads, dim)),
            g.normal(size=(B, skv, kv_heads, dim)), g.normal(size=(B, sq, heads, dim)))


def test_cross_gradients_are_differences():
    lens = [5, 2, 0, 1]
    q, k, v, dctx = cross_case(lens)
    f = lambda: (ORC.cross_attention(q, k, v, lens)[0] * dctx).sum()  # noqa: E731
    dq, dk, dv = ORC.cross_attention_backward(q, k, v, dctx, lens)
    for got, x in ((dq, q), (dk, k), (dv, v)):
        assert np.abs(got - differences(f, x)).max() < 1e-7
    assert not dk[1, 2:].any() and not dv[1, 2:].any() and not dq[2].any() and not dk[2].any()


def test_cross_closed_forms():
    q, k, v, _ = cross_case([5, 3, 1, 0])
    ctx, lse = ORC.cross_attention(0 * q, k, v, [5, 3, 1, 0])  # uniform
    assert np.allclose(ctx[1, :, 2], v[1, :3, 1].mean(0)) and np.allclose(lse[1], np.log2(3))
    assert np.allclose(ctx[2, :, 3], v[2, 0, 1]) and not ctx[3].any() and (lse[3] == -np.inf).all()
    # scores ln 3 and 0: probabilities 3/4 and 1/4, 2 + 0 bits of sum
    q, k = np.zeros((1, 1, 1, 4)), np.zeros((1, 2, 1, 4))
    q[..., 0], k[0, 0, 0, 0] = 2.0, np.log(3.0)
    ctx, lse = ORC.cross_attention(q, k, np.array([1.0, 5.0])[None, :, None, None] * np.ones(4), [2])
    assert np.allclose(ctx, 2.0) and np.allclose(lse, 2.0)


def test_heads_share_keys_in_order():
    lens = [4]
    q, k, v, dctx = cross_case(lens, heads=6, kv_heads=2)
    ctx, _ = ORC.cross_attention(q, k, v, lens)
    wide = lambda x: np.repeat(x, 3, axis=2)  # noqa: E731
    assert np.allclose(ctx, ORC.cross_attention(q, wide(k), wide(v), lens)[0])
    _, dk, dv = ORC.cross_attention_backward(q, k, v, dctx, lens)
    _, wk, wv = ORC.cross_attention_backward(q, wide(k), wide(v), dctx, lens)
    assert np.allclose(dk, wk.reshape(1, 5, 2, 3, 4).sum(3)) and np.allclose(dv, wv.reshape(1, 5, 2, 3, 4).sum(3))
