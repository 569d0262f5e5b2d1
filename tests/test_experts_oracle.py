"""The float64 definitions of a layer of experts against closed forms and differences."""
import numpy as np
import pytest

from oracle import experts_f64 as ORC


def test_choices_and_plan():
    x = np.array([[1.0, 3.0, 3.0, -np.inf], [-np.inf] * 4, [np.nan, 0.0, -1.0, np.inf]])
    e = ORC.choose(x, 3)
    assert e.tolist() == [[1, 2, 0], [-1, -1, -1], [3, 1, 2]]
    row, offset = ORC.plan(e, 4)
    assert offset.tolist() == [0, 1, 3, 5, 6]
    assert row.tolist() == [[1, 3, 0], [-1, -1, -1], [5, 2, 4]]
    w = ORC.weights(x, e, "chosen")
    z = 1 + 1 + np.exp(-2.0)
    assert np.allclose(w, [[1 / z, 1 / z, np.exp(-2.0) / z], [0, 0, 0], [1, 0, 0]])


@pytest.mark.parametrize("over", ["chosen", "all"])
def test_route_gradient_against_differences(over):
    g = np.random.default_rng(3)
    x, d = g.normal(size=(5, 7)), g.normal(size=(5, 3))
    x[1, 4] = -np.inf
    e = ORC.choose(x, 3)
    dx = ORC.route_backward(x, e, d, over)
    h = 1e-6
    for t in range(5):
        for i in range(7):
            if x[t, i] == -np.inf:
                assert dx[t, i] == 0
                continue
            up, dn = x.copy(), x.copy()
            up[t, i] += h
            dn[t, i] -= h  # (the choices stay: no two logits are this near)
            diff = ((ORC.weights(up, e, over) - ORC.weights(dn, e, over)) * d).sum() / (2 * h)
            assert abs(diff - dx[t, i]) < 1e-8


def test_rows_there_and_back():
    g = np.random.default_rng(4)
    e = ORC.choose(g.normal(size=(6, 5)), 2)
    row, offset = ORC.plan(e, 5)
    x, w, d = g.normal(size=(6, 4)), g.normal(size=(6, 2)), g.normal(size=(6, 4))
    rows = ORC.dispatch(x, row, np.zeros((12, 4)))
    assert np.allclose(ORC.combine(rows, row, np.ones((6, 2))), 2 * x)
    # the sum is bilinear in rows and weights, so its gradients are exact differences
    dr, dw = ORC.combine_backward(rows, d, row, w, np.zeros((12, 4)))
    other = g.normal(size=(12, 4))
    assert np.isclose((ORC.combine(other, row, w) * d).sum(), (dr * other).sum())
    assert np.isclose((ORC.combine(rows, row, w) * d).sum(), (dw * w).sum())


def test_groups():
    g = np.random.default_rng(5)
    offset = [0, 2, 2, 5]
    a, w, d = g.normal(size=(6, 3)), g.normal(size=(3, 4, 3)), g.normal(size=(6, 4))
    y = ORC.by_group("xwt", a, w, offset)
    assert np.allclose(y[3], w[2] @ a[3]) and not y[5].any()
    d[5] = 0
    assert np.isclose((y * d).sum(), (ORC.by_group("xw", d, w, offset) * a).sum())
    dw = ORC.by_group("xtw", d, a, offset)
    assert np.isclose((y * d).sum(), (dw * w).sum()) and not dw[1].any()
    z, h = g.normal(size=100), 1e-6
    assert np.allclose((ORC.gelu(z + h) - ORC.gelu(z - h)) / (2 * h), ORC.gelu_slope(z), atol=1e-9)


def test_codes():
    v = ORC.e4m3_values()
    torch = pytest.importorskip("torch")
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(v, want, equal_nan=True)
    r = ORC.root_values()
    assert r[0] == 0 and r[255] == 0.96875 and (np.diff(r) > 0).all() and r[1] == 17 / 16 * 2.0 ** -16
    got = ORC.decode(np.arange(258) % 256, [2.0, 3.0], r)
    assert got[5] == 2 * r[5] and got[257] == 3 * r[1]
