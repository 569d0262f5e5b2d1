"""Head norms where a warp walks over more than 32 and 64 tokens (it loads their positions 32
at a time), over rows whose offsets pass 2^31 values, and at the ends of fp32's range.
Bounds and layout are those of test_gpu_qk_norm.
"""
import numpy as np
import pytest

from paper_2202_11836_gb300 import _lib as L
from test_gpu_qk_norm import MARK, ROT, Case, P, stream

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# A device of 152 SMs keeps 3648 warps in a forward and 1216 in a backward; with one set of
# heads of each kind a warp then has rows / 1824 tokens, or rows / 608.


@pytest.mark.parametrize("rotation", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_forward_of_many_tokens_a_warp(dtype, rotation):
    c = Case(130007, 2, 1, 32, dtype, rotation)
    y = c.forward()
    torch.cuda.synchronize()
    c.check_forward(y)


@pytest.mark.parametrize("rotation", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_backward_of_many_tokens_a_warp(dtype, rotation):
    c = Case(45007, 2, 1, 32, dtype, rotation)
    dx, dq, dk = c.backward()
    c.check_backward(dx, dq, dk)


@pytest.mark.parametrize("rotation", ["halves", "none"])
def test_rows_past_32_bit_offsets(rotation):
    """Four rows 3 x 2^28 values apart: the last starts past 2^31 values."""
    small = Case(4, 2, 1, 64, "bf16", rotation, far=False)
    ld, n = 3 << 28, small.width
    x, dy, y, dx = (torch.empty(3 * ld + n + 8, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    rows = lambda t: torch.as_strided(t, (4, n + 8), (ld, 1))  # noqa: E731
    for t in (x, dy, y, dx):
        rows(t).fill_(MARK)
    rows(x)[:, :n], rows(dy)[:, :n] = small.x[:, :n], small.dy
    s = L.SkyQkNormShape(4, 2, 1, 64, L.SKY_DTYPE_BF16, ld, ld, small.eps, ROT[rotation], 10000.0)
    pos = P(small.pos) if rotation != "none" else None
    L.call("sky_qk_norm_fwd", s, P(x), P(small.gain[0]), P(small.gain[1]), pos, P(y), stream())
    size = L.lib().sky_qk_norm_bwd_workspace_bytes(s)
    ws, dg = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(2, 64, device="cuda")
    L.call("sky_qk_norm_bwd", s, P(x), P(dy), P(small.gain[0]), P(small.gain[1]), pos, P(dx), P(dg[0]), P(dg[1]), P(ws),
           size, stream())
    want_y, (want_dx, dq, dk) = small.forward(), small.backward()
    torch.cuda.synchronize()
    for t, want in ((y, want_y), (dx, want_dx)):
        assert torch.equal(rows(t)[:, :n], want[:, :n]) and bool((rows(t)[:, n:] == MARK).all())
    assert torch.equal(dg[0], dq) and torch.equal(dg[1], dk)


def test_ends_of_the_range():
    """Sums of squares that overflow: zeros.  With eps = 0, sums that are 0: not finite, and
    the heads beside them as they were."""
    for value, finite in ((1e25, True), (1e-25, False)):
        c = Case(6, 2, 2, 64, "fp32", "none", eps=0.0, far=False)
        y = c.forward().clone()
        c.x[3, 64:128] = value
        z = c.forward()
        torch.cuda.synchronize()
        head = z[3, 64:128]
        assert not bool(head.any()) if finite else not bool(torch.isfinite(head).any())
        z[3, 64:128] = y[3, 64:128]
        assert torch.equal(y, z)


def test_gains_of_many_rows_are_repeatable():
    c = Case(45007, 9, 2, 32, "bf16", "halves")
    first = c.backward()
    assert all(torch.equal(a, b) for a, b in zip(first, c.backward()))
    assert np.isfinite(first[1].cpu().numpy()).all()
