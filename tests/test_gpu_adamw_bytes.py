"""The bytes of 8-bit moments, one by one: they are those of arithmetic in fp32 rounded step by step, whichever
way a block is read, and with values on and beside the borders between codes."""
import numpy as np
import pytest

from paper_2202_11836_gb300 import _lib as L
from test_gpu_adamw_many import BF, F32, RULE, Tensor, step

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ONE = np.float32(1)
B1, B2 = np.float32(RULE["beta1"]), np.float32(RULE["beta2"])
BLOCK = L.SKY_STATE_BLOCK


def blocks(x):
    """[blocks, BLOCK], zeros behind the last value."""
    return np.pad(x, (0, -len(x) % BLOCK)).reshape(-1, BLOCK)


def r_values(codes):
    c = codes.astype(np.uint32)
    return np.where(c > 0, ((c << 19) + (111 << 23)).view(np.float32), np.float32(0))


def scales(top, unit):
    """A block's scale and its inverse."""
    zero = top < np.float32(1e-30)
    scale = np.where(zero, np.float32(0), top * unit)
    return scale, np.where(zero, np.float32(0), ONE / np.where(zero, ONE, scale))


def r_fractions(v):
    """What is rounded to a code, before it is."""
    r = np.sqrt(v)
    scale, inv = scales(r.max(1), ONE / np.float32(0.96875))
    return r * inv[:, None], scale


def r_codes(y):
    b = np.ascontiguousarray(y).view(np.uint32).astype(np.int64)
    c = (b + 0x3ffff + (b >> 19 & 1) - (111 << 23)) >> 19
    return np.where(y > 0, np.clip(c, 1, 255), 0).astype(np.uint8)


def m_codes(m, inv):
    y = torch.from_numpy(np.ascontiguousarray(m * inv[:, None]))
    return y.to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def moments(g, m, v):
    """fp32 moments after a step, every product and sum rounded."""
    return m * B1 + g * (ONE - B1), v * B2 + (g * g) * (ONE - B2)


def expected(x):
    """(m's bytes, r's bytes, m's scales, r's scales) after a step of Tensor x."""
    numpy = lambda k: x.at(k).cpu().numpy()  # noqa: E731
    g = blocks(x.at("g").float().cpu().numpy())
    m = torch.from_numpy(blocks(numpy("m"))).view(torch.float8_e4m3fn).float().numpy() * numpy("m_scale")[:, None]
    r = r_values(blocks(numpy("v"))) * numpy("v_scale")[:, None]
    m, v = moments(g, m, r * r)
    assert m.dtype == v.dtype == np.float32
    y, vs = r_fractions(v)
    ms, m_inv = scales(np.abs(m).max(1), ONE / np.float32(448))
    return [a.reshape(-1)[:x.n] for a in (m_codes(m, m_inv), r_codes(y))] + [ms, vs]


def same(x, want):
    for k, w in zip(("m", "v", "m_scale", "v_scale"), want):
        got = x.at(k).cpu().numpy()
        bad = np.flatnonzero(got.view(np.uint8 if got.itemsize == 1 else np.uint32) != w.view(np.uint8 if w.itemsize == 1 else np.uint32))
        assert not len(bad), (k, len(bad), bad[:5], got[bad[:5]], w[bad[:5]])


@pytest.mark.parametrize("grads", [F32, BF], ids=["g32", "g16"])
@pytest.mark.parametrize("n,shift", [(20480, 0), (20480, 1), (1000, 0), (257, 3)])
def test_bytes_over_steps(grads, n, shift):
    """Whole blocks on the grid, blocks off it, and one that ends early."""
    g = torch.Generator(device="cuda").manual_seed(n + shift)
    x = Tensor(n, True, grads, g, shift=shift)
    for t in (1, 2, 3):
        want = expected(x)
        step([x], t, True, grads)
        same(x, want)
        x.new_gradient(g)


def border_gradients():
    """Gradients of a first step whose root lies on, or up to four steps of fp32 beside, the border above a code: a
    block's largest first, then seven values for each of 36 codes."""
    rng = np.random.default_rng(7)
    out = []
    for codes in np.array_split(rng.permutation(np.arange(1, 253)), 7):
        block = np.zeros(BLOCK, np.float32)
        block[0] = np.float32(rng.uniform(0.5, 2.0))
        top = np.sqrt((block[0] * block[0]) * (ONE - B2))
        scale = scales(np.array([top]), ONE / np.float32(0.96875))[0][0]
        for i, c in enumerate(codes):
            border = np.array([(c << 19) + (111 << 23) + (1 << 18)], np.uint32).view(np.float32)[0]
            g = np.float32(np.float64(border) * np.float64(scale) / np.sqrt(np.float64(ONE - B2)))
            block[1 + 7 * i:8 + 7 * i] = (np.array([g]).view(np.uint32) + np.arange(7, dtype=np.uint32) - np.uint32(3)).view(np.float32)
        out.append(block)
    return np.concatenate(out)


@pytest.mark.parametrize("shift", [0, 1])
def test_bytes_beside_borders(shift):
    grad = border_gradients()
    v = moments(blocks(grad), np.float32(0), np.float32(0))[1]
    bits = r_fractions(v)[0].view(np.uint32).astype(np.int64)
    beside = np.abs((bits & 0x7ffff) - 0x40000) <= 8
    # (a root moves by about as many steps as its gradient; all but the least codes' are that near, some on the border)
    assert beside.sum() > 1000 and ((bits & 0x7ffff) == 0x40000).sum() >= 20
    x = Tensor(len(grad), True, F32, torch.Generator(device="cuda").manual_seed(1), shift=shift)
    x.at("g").copy_(torch.from_numpy(grad))
    want = expected(x)
    step([x], 1, True)
    same(x, want)
    # one such value a block, the others far from any border: the block is rounded exactly for its sake alone
    for at in (1, 100, 255):
        y = Tensor(len(grad), True, F32, torch.Generator(device="cuda").manual_seed(1), shift=shift)
        sparse = np.where(np.isin(np.arange(len(grad)) % BLOCK, [0, at]), grad, np.float32(0.25))
        y.at("g").copy_(torch.from_numpy(sparse.astype(np.float32)))
        want = expected(y)
        step([y], 1, True)
        same(y, want)


def test_a_square_that_overflows():
    """A finite gradient whose square is not in fp32: its second moment is lost, in 8 bits its block's moments."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x, y = Tensor(700, True, F32, g), Tensor(700, False, F32, g)
    for z in (x, y):
        z.at("g")[300] = 1e21
        step([z], 1, z.small)
    m, v = x.moments()
    assert not np.isfinite(m[256:512]).any() and not np.isfinite(v[256:512]).any()
    for part in (slice(0, 256), slice(512, 700)):
        assert np.isfinite(m[part]).all() and np.isfinite(v[part]).all()
    lost = torch.nonzero(~torch.isfinite(y.at("v"))).flatten()
    assert lost.tolist() == [300] and bool(torch.isfinite(y.at("m")).all())
    assert bool(torch.isfinite(x.at("w")).all()) and bool(torch.isfinite(y.at("w")).all())  # (a step of 0 there)
