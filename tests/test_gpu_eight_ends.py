"""GPU tests of products of matrices in 8 bits at both ends of what their powers
reach, against float64: every power that a matrix in 8 bits may have, in every kind
of kernel, with the bounds of float32 sums (u = 2^-24): a sum of k products passes at
most k / 4 + 16 roundings per term, and a product or sum below float32's smallest
normal number, 2^-126, may be lost."""
import numpy as np
import pytest
import torch

from oracle import eight as E
from test_gpu_eight import Eight, Mat, U, SLACK, close, matmul8, quantize, V, _need_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

NUMBERS = E.e4m3_table()[np.isfinite(E.e4m3_table())]
LARGEST = {"f32": float(np.finfo(np.float32).max), "bf16": 255 * 2.0 ** 120}


def given(rows, k, rng, power):
    """A matrix of any e4m3 values with these powers [blocks x rows]; zeros past its columns."""
    m = Eight(rows, k, 1)
    v = np.zeros((rows, m.wide))
    v[:, :k] = rng.choice(NUMBERS, (rows, k))
    m._bytes().copy_(torch.from_numpy(v).float().cuda().to(torch.float8_e4m3fn).view(torch.uint8))
    m._powers().copy_(torch.from_numpy((np.broadcast_to(power, (m.nb, rows)) + 127).astype(np.uint8)))
    return m


def check(V, dt, a, b, k):
    m, n = a.rows, b.rows
    c = Mat(dt, m, n, n + 3, 1)
    matmul8(V, dt, a, b, c, k)
    torch.cuda.synchronize()
    av, bv = a.values(), b.values()
    want, mags = av @ bv.T, np.abs(av) @ np.abs(bv).T
    bound = SLACK * (k / 4 + 16) * U * mags + k * 2.0 ** -126
    if dt == "bf16":
        # the 8-bit instruction adds a block's products by eights that keep 13 bits below the
        # largest one's power of two: 7 2^-13 of it at most
        bound = bound + 7 * 2.0 ** -13 * mags
    sure = mags <= LARGEST[dt] * (1 - 2.0 ** -8)                # whatever the order of the sum
    got = c.np()
    assert sure.any() and np.isfinite(got[sure]).all()
    close(got[sure], want[sure], bound[sure], "c", dt)
    c.assert_guard()


SIZES = [(1, 5, 128), (5, 37, 130), (20, 70, 1000), (60, 40, 300), (300, 1000, 4300), (2050, 1030, 200)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("pa,pb", [(120, -30), (127, -127), (-127, 110), (-127, 127), (119, -127), (-125, 100), (-124, 100),
                                   (-30, 118), (-127, 10), (-63, -64), (64, 40), (0, 0)])
def test_one_power(V, dt, m, n, k, pa, pb):
    rng = np.random.default_rng(m + n + k + pa)
    check(V, dt, given(m, k, rng, pa), given(n, k, rng, pb), k)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_powers_of_every_kind_side_by_side(V, dt, m, n, k):
    """A power for each block whose partner's takes the product back to about 1, and single
    rows with another one: steps with and without such powers meet in one sum."""
    rng = np.random.default_rng(m * n + k)
    nb = -(-k // 128)
    p = rng.choice([-127, -126, -100, -20, 0, 30, 90, 118, 120, 127], nb)[:, None]
    a = given(m, k, rng, p + np.zeros((nb, m), int))
    few = rng.integers(-8, 9, (nb, n))
    check(V, dt, a, given(n, k, rng, np.clip(few - p, -127, 127)), k)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(3, 20, 256), (40, 300, 700), (400, 900, 3000)])
def test_what_an_operator_makes_of_float32_at_its_ends(V, dt, m, n, k):
    """Rows near float32's largest number, whose block's power is 2^120 with values of 256, and
    rows so small that theirs is 2^-127 and the values are e4m3's smallest."""
    rng = np.random.default_rng(k)
    big = rng.normal(size=(m, k))
    big[::2, ::3] = 3.39e38 * np.sign(big[::2, ::3])
    big[1::2] *= 2.0 ** -130
    small = rng.normal(size=(n, k)) * 2.0 ** -20
    small[1::2] *= 2.0 ** 120
    x, y = Mat("f32", m, k, 0, 0, big), Mat("f32", n, k, 0, 0, small)
    a, b = Eight(m, k), Eight(n, k)
    quantize(V, "f32", x, a)
    quantize(V, "f32", y, b)
    assert np.abs(a.values()).max() == 2.0 ** 128
    check(V, dt, a, b, k)


@pytest.mark.parametrize("m,n,k", [(6, 30, 500), (301, 1003, 5000)])
def test_bytes_past_the_last_row_have_no_influence(V, m, n, k):
    """The same bits whatever lies among the exponents past the last row, and blocks of zeros of
    any power."""
    rng = np.random.default_rng(m)
    a, b = given(m, k, rng, 0), given(n, k, rng, 3)
    outs = []
    for fill in (0, 1, 254, 255):
        for e in (a, b):
            e.scale[:e.nb * e.sld].view(e.nb, e.sld)[:, e.rows:] = fill
        c = Mat("f32", m, n)
        matmul8(V, "f32", a, b, c, k)
        torch.cuda.synchronize()
        outs.append(c.t.clone())
    assert all(torch.equal(o, outs[0]) for o in outs)
    a._bytes()[:, 128:256] = 0
    for power in (0, 60, 127, 250, 254):
        a._powers()[1] = power
        c = Mat("f32", m, n)
        matmul8(V, "f32", a, b, c, k)
        torch.cuda.synchronize()
        if power:
            assert torch.equal(c.t, first)
        first = c.t.clone()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(8, 40), (300, 700)])
def test_products_that_cancel_within_a_block(V, dt, m, n):
    """Two large products of a block cancel and small ones are left: float32 results keep
    what float32 sums do."""
    rng = np.random.default_rng(n)
    k = 4 * 128 + 50
    a, b = Eight(m, k), Eight(n, k)
    for e, sign in ((a, -1), (b, 1)):
        v = np.zeros((e.rows, e.wide))
        v[:, :k] = E.e4m3_round(np.abs(rng.normal(size=(e.rows, k))))
        for s in range(0, k, 128):
            at = rng.integers(0, 8)
            v[:, s + at], v[:, s + at + 1] = 448, 448 * sign
        e._bytes().copy_(torch.from_numpy(v).float().cuda().to(torch.float8_e4m3fn).view(torch.uint8))
        e._powers().fill_(127)
    # the pair lies at the same columns of both
    b._bytes()[:, :k] = torch.where((a._bytes()[0, :k] & 0x7F) == 0x7E, 0x7E, b._bytes()[:, :k].clamp(max=0x50))
    check(V, dt, a, b, k)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim,classes", [(16, 1024, 5000), (16, 1024, 20_000), (1, 64, 100_000), (40, 300, 3000), (200, 64, 900),
                                              (300, 1000, 700), (3000, 64, 260), (700, 200, 2000)])
def test_the_loss_stays_within_its_workspace(V, dt, rows, dim, classes):
    """Sums of dw in one part and in several, of dx written at once and joined."""
    from test_gpu_eight import Loss
    t = Loss(V, dt, rows, dim, classes)
    size = t.a.workspace_bytes
    t.ws = torch.full((size + (1 << 16),), 0xFF, dtype=torch.uint8, device="cuda")
    t.a.workspace = t.ws.data_ptr()
    t.run()
    t.check()
    assert bool((t.ws[size:] == 0xFF).all())
