"""Grouped weight gradients of more tiles than the few-tile kernel takes (pairs of SMs), and how exact long
sums are: element by element as the other grouped products, and by norm, which tells 32-bit sums from less."""
import numpy as np
import pytest

from oracle import experts_f64 as ORC
from paper_2202_11836_gb300 import _lib as L
from test_gpu_grouped import MARK, Case, f64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def by_pairs(c):
    """The few-tile kernel wants one cluster of two CTAs, at least, for every tile of 128 x 128."""
    tiles = len(c.sizes) * -(-c.out // 128) * -(-c.in_ // 128)
    return tiles > L.lib().sky_device_sm_count() // 2


def off(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


# (group sizes, out, in, rows before, rows behind): parts of 512 rows with both accumulators taken more than once,
# tiles cut off at 256 in either direction, last blocks with and without rows to clear; up to 32 groups come by
# size, more in their own order
MANY = [([1300, 37, 0, 1201], 1288, 1032, 3, 7), ([4100, 1, 515], 1032, 520, 0, 0), ([(37 * i) % 130 for i in range(40)], 264, 136, 0, 5),
        ([2] * 1024, 8, 8, 1, 0), ([600] + [0] * 30 + [16, 15], 136, 264, 0, 2)]


@pytest.mark.parametrize("sizes,out,in_,first,behind", MANY, ids=lambda v: str(v) if isinstance(v, int) else f"{len(v)}g{sum(v)}")
def test_weight_gradients_by_pairs(sizes, out, in_, first, behind):
    c = Case("xtw", sizes, out, in_, "bf16", "store", first, behind)
    assert by_pairs(c)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = c.run(status)[0]
    assert status.item() == 0
    c.check(got, None)
    assert torch.equal(got, c.run()[0])


def test_groups_of_a_pair_stay_apart():
    """Infinities in a group's rows stay out of the others' sums, before and behind them."""
    sizes, out, in_ = [1300, 37, 1201], 1032, 776
    c = Case("xtw", sizes, out, in_, "bf16", "store", 0, 70)
    assert by_pairs(c)
    want = c.run()[0].clone()
    c.a[1300:1337] = torch.inf
    c.b[1300:1337] = 1.0
    got = c.run()[0]
    n = out * in_
    assert torch.equal(got[:n], want[:n]) and torch.equal(got[2 * n:], want[2 * n:])
    assert bool((got[n:2 * n] == torch.inf).all())


def test_captured_by_pairs():
    c = Case("xtw", [700, 0, 900, 29], 1032, 776, "bf16", behind=3)
    assert by_pairs(c)
    n, ws = c.workspace()
    out, _ = c.room()
    c.call(out, None, n, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(out, None, n, ws)
    other = Case("xtw", [29, 1100, 500, 0], 1032, 776, "bf16", behind=3)
    for x, y in zip((c.a, c.b, c.d_offset), (other.a, other.b, other.d_offset)):
        x.copy_(y)
    for _ in range(2):
        out.fill_(MARK)
        graph.replay()
    torch.cuda.synchronize()
    assert bool((out[-64:] == MARK).all())
    other.check(out[:-64], None)


@pytest.mark.parametrize("form,out,in_", [("xwt", 64, 64), ("xw", 64, 64), ("xtw", 1032, 1032), ("xtw", 64, 64)])
def test_bad_offsets_of_more_rows(form, out, in_):
    """More than 64 rows, so not the kernels of few rows; weight gradients by pairs and of few tiles."""
    c = Case(form, [100, 150, 50], out, in_, "bf16")
    assert form != "xtw" or by_pairs(c) == (out == 1032)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for bad in ([-5, 100, 250, 300], [0, 250, 100, 300], [0, 100, 250, 1 << 30], [-(2 ** 31), 0, 2 ** 31 - 1, 0], [300, 200, 100, 0]):
        c.d_offset.copy_(torch.tensor(bad, dtype=torch.int32))
        status.zero_()
        c.run(status)  # (checks what lies behind the outputs)
        assert status.item() == 1


@pytest.mark.parametrize("sizes,out,in_,pairs", [([9000, 9300], 776, 1032, True), ([9000], 256, 136, False)])
def test_long_bf16_sums_by_norm(sizes, out, in_, pairs):
    """An addition on the tensor cores cuts off up to 2^-23 of the partial sum, half of that on average, towards 0.
    In a part of 512 rows of N(0, 1) products it comes 32 times, at partial sums of sqrt(16 j):
    1/2 2^-23 4 sum of sqrt(j) = 1/2 2^-23 483, beside a result of sqrt(512): 1.3e-6.  Parts are as often off in
    either direction, so their sum is as far off; its own roundings, 2^-24 sqrt(18 / 2), make 2e-7 of any sign.
    (Were it one sum of 9000 rows, it would come 563 times: 74 times the errors of a part beside four times its result.)"""
    c = Case("xtw", sizes, out, in_, "bf16")
    assert by_pairs(c) == pairs
    got = f64(c.run()[0]).reshape(len(sizes), out, in_)
    want = ORC.by_group("xtw", f64(c.a), f64(c.b), c.offset)
    for g in range(len(sizes)):
        assert off(got[g], want[g]) <= 1.5e-6


@pytest.mark.parametrize("form,sizes,out,in_", [("xtw", [4000], 200, 130), ("xtw", [900, 4100], 79, 101), ("xwt", [500, 80], 100, 2000),
                                                ("xw", [500, 80], 2000, 100), ("xwt", [8], 256, 4000)])
def test_long_fp32_sums_by_norm(form, sizes, out, in_):
    """n fused additions, each off by up to 2^-24 of a partial sum of sqrt(j): at random, 2^-24 sqrt(n^2 / 2) at most beside
    sqrt(n), whatever the splits."""
    c = Case(form, sizes, out, in_, "fp32")
    got = f64(c.run()[0])
    want = ORC.by_group(form, f64(c.a), f64(c.b), c.offset)
    n = {"xwt": in_, "xw": out, "xtw": max(sizes)}[form]
    assert off(got.reshape(want.shape), want) <= 2.0 ** -24 * (n / 2) ** 0.5
