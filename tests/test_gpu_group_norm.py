"""Group normalisation with its activation, channels last, and its gradient (paac_group_norm) against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from operators_ref import TINY, U, assert_within, f64, half_step, norm_backward, norm_forward, spread
from paper_1705_04862_b200 import binding as pb

pytestmark = pytest.mark.gpu
F, H = torch.float32, torch.bfloat16
ACT = {"none": pb.ACT_NONE, "relu": pb.ACT_RELU, "silu": pb.ACT_SILU}
# Additions that one element passes through on its way into a sum over a group: at most 64 in a thread, 7 between its channels, 8 in a lane over
# a block's threads or its warps, 5 between lanes, 16 over a cluster.  Where a sample is read twice 16, 64 and 5, then its parts (as many as
# tests have, over 32 lanes) and 5 again.
DEPTH = 128


def images(n, p, c, dtype, layout, count=1):
    """`count` tensors [n][p][c]: contiguous, parts of wider pixels, at odd places with gaps, or every other pixel."""
    if layout == "packed":
        return [torch.zeros(n, p, 2 * c, dtype=dtype, device="cuda")[..., c:] for _ in range(count)]
    if layout == "odd":
        return [torch.zeros(n, p + 1, c + 3, dtype=dtype, device="cuda")[:, 1:, 1:c + 1] for _ in range(count)]
    if layout == "sparse":
        return [torch.zeros(n, 2 * p, c, dtype=dtype, device="cuda")[:, ::2] for _ in range(count)]
    return [torch.zeros(n, p, c, dtype=dtype, device="cuda") for _ in range(count)]


def scratch(n, p, c, g, dtype):
    need = pb.group_norm_workspace_bytes(n, p, c, g, pb.BF16 if dtype == H else pb.FP32)
    assert need > 0
    return torch.full((need,), 255, dtype=torch.uint8, device="cuda")          # its contents do not matter


def logistic_error(dtype, v):
    """As a gate's: steps of the exponential, and of 1 + e, the quotient and the products."""
    e = 2 * U * (2 + 1.173 * np.abs(v)) if dtype == H else 2 * U
    return e + 8 * U


def check_forward(n, p, c, g, dtype, act, layout="plain", eps=1e-5, x=None, affine=True, seed=0):
    rng = np.random.RandomState(seed + n + p + c)
    xt, y = images(n, p, c, dtype, layout, 2)
    xt.copy_(torch.from_numpy(rng.randn(n, p, c) * (0.5 + rng.rand(c)) + rng.randn(c)) if x is None else x)
    gamma = torch.from_numpy(1 + 0.3 * rng.randn(c)).float().cuda() if affine else None
    beta = torch.from_numpy(0.3 * rng.randn(c)).float().cuda() if affine else None
    mean, rstd = (torch.full((n, g), 9.0, device="cuda") for _ in range(2))
    assert pb.group_norm(xt, gamma, beta, y, mean, rstd, g, scratch(n, p, c, g, dtype), activation=ACT[act], eps=eps) == pb.OK
    x64, gm, bt = f64(xt), (f64(gamma) if affine else np.ones(c)), (f64(beta) if affine else np.zeros(c))
    want, m, r, v = norm_forward(x64, gm, bt, g, act, float(np.float32(eps)))
    size = np.abs(x64).reshape(n, p, g, c // g).mean((1, 3))
    dmean = DEPTH * U * size + TINY
    # the variance: sums as for the mean, squares of deviations from a mean that is itself off; half of that for the root
    drstd = (DEPTH + 4) * U + 0.5 * (r * dmean) ** 2
    assert_within(mean, m, dmean, "mean")
    assert_within(rstd, r, r * drstd, "rstd")
    xhat = (x64 - spread(m, c)) * spread(r, c)
    dv = np.abs(gm) * (spread(r * dmean, c) + np.abs(xhat) * (spread(drstd, c) + 4 * U)) + 2 * U * np.abs(v) + TINY
    off = 1.1 * dv + (np.abs(want) * logistic_error(dtype, v) if act == "silu" else 0)
    assert_within(y, want, off + half_step(dtype) * (np.abs(want) + off), "y")
    return xt, y, gamma, beta, mean, rstd


def check_backward(n, p, c, g, dtype, act, layout="plain", affine=True, seed=0):
    rng = np.random.RandomState(seed + n + p + c + 1)
    xt, _, gamma, beta, mean, rstd = check_forward(n, p, c, g, dtype, act, layout, affine=affine, seed=seed)
    gm, bt = (f64(gamma) if affine else np.ones(c)), (f64(beta) if affine else np.zeros(c))
    x64, m, r = f64(xt), f64(mean), f64(rstd)
    dy, dx = images(n, p, c, dtype, layout, 2)
    d = rng.randn(n, p, c)
    if act == "relu":        # the derivative has a step at 0: within rounding of it either side is right
        d = np.where(np.abs((x64 - spread(m, c)) * spread(r, c) * gm + bt) > 1e-4, d, 0)
    dy.copy_(torch.from_numpy(d))
    d = f64(dy)
    dgamma, dbeta = (torch.full((c,), 9.0, device="cuda") for _ in range(2))
    room = scratch(n, p, c, g, dtype)
    assert pb.group_norm_backward(xt, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, g, room, activation=ACT[act]) == pb.OK
    wx, wg, wb, k = norm_backward(x64, d, gm, bt, m, r, act)
    # the argument of the activation, its slope (which changes by at most 0.5 of that) and the product
    arg = 4 * U * (np.abs(k["xhat"] * gm) + np.abs(bt))
    slope = (0.5 * arg + 2 * logistic_error(dtype, k["v"]) * (1 + np.abs(k["v"]))) if act == "silu" else 0
    adv, bdv = np.abs(k["dv"]), np.abs(d) * slope + 2 * U * np.abs(k["dv"])
    # a channel's sum: within a block as above, then over samples and slabs in 32 lanes
    depth = (DEPTH + n * (p // 16 + 1) / 32 + 32) * U
    assert_within(dbeta, wb, (bdv + depth * adv).sum((0, 1)) + TINY, "dbeta")
    assert_within(dgamma, wg, ((bdv + (depth + 4 * U) * adv) * np.abs(k["xhat"])).sum((0, 1)) + TINY, "dgamma")
    per = DEPTH * U + (p // 16 + 1) * U
    s1 = k["over_group"]((bdv + per * adv) * np.abs(gm))
    s2 = k["over_group"]((bdv + (per + 4 * U) * adv) * np.abs(gm * k["xhat"]))
    t1, t2 = k["over_group"](adv * np.abs(gm)), k["over_group"](adv * np.abs(gm * k["xhat"]))
    ax = np.abs(k["xhat"])
    off = spread(r, c) * (np.abs(gm) * bdv + spread(s1, c) + ax * spread(s2, c) + 8 * U * (adv * np.abs(gm) + spread(t1, c) + ax * spread(t2, c))) + TINY
    assert_within(dx, wx, off + half_step(dtype) * (np.abs(wx) + off), "dx")
    return xt, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, room


SHAPES = [(1, 1, 1, 1), (1, 2, 8, 2), (3, 49, 64, 8), (2, 400, 32, 4), (5, 81, 24, 3), (2, 33, 30, 5), (1, 7, 12, 12), (9, 1, 48, 6), (2, 441, 40, 8),
          (1, 7056, 16, 4), (3, 300, 7, 7), (2, 10, 512, 32), (1, 3, 2048, 2), (1, 5, 2504, 1), (2, 2, 4000, 500), (3, 50, 20, 5), (2, 90, 12, 2), (4, 30, 6, 3), (1, 1000, 256, 1), (1, 2, 1000, 5)]


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("n,p,c,g", SHAPES)
def test_shapes(n, p, c, g, dtype, act):
    check_backward(n, p, c, g, dtype, act)


@pytest.mark.parametrize("layout", ["packed", "odd", "sparse"])
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("n,p,c,g", [(3, 50, 32, 4), (2, 17, 20, 4), (1, 900, 8, 1), (40, 9, 16, 2)])
def test_layouts(n, p, c, g, dtype, layout):
    check_backward(n, p, c, g, dtype, "silu", layout)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("n,p,c,g", [(200, 81, 64, 8), (700, 49, 16, 4), (1500, 1, 64, 4), (4, 30000, 16, 2), (1, 70000, 8, 8), (3, 7056, 48, 6), (33, 400, 32, 4)])
def test_many_samples_and_large_ones(n, p, c, g, dtype):
    check_backward(n, p, c, g, dtype, "relu", affine=n % 2 == 0)


@pytest.mark.parametrize("dtype", [F, H])
def test_groups_without_spread_and_far_from_zero(dtype):
    """A constant group has variance 0 and gives beta; values far from 0 keep what their type holds of the differences."""
    x = torch.zeros(2, 60, 16, dtype=torch.float64)
    x[:, :, 4:8] = 3.0
    x[:, :, 8:] = 512.0 + torch.randint(-8, 9, (2, 60, 8)) * 4.0
    check_forward(2, 60, 16, 4, dtype, "none", x=x)
    xt = x.to(dtype).cuda()
    y, mean, rstd = torch.empty_like(xt), *(torch.empty(2, 4, device="cuda") for _ in range(2))
    beta = torch.arange(16, device="cuda", dtype=torch.float32)
    assert pb.group_norm(xt, None, beta, y, mean, rstd, 4, scratch(2, 60, 16, 4, dtype)) == pb.OK
    assert torch.equal(y[:, :, :8], beta[:8].to(dtype).expand(2, 60, 8)) and bool((mean[:, 1] == 3).all())
    assert bool(((rstd[:, :2] - 1e-5 ** -0.5).abs() <= 4 * U * 1e-5 ** -0.5).all())


def test_an_infinity_or_nan_stays_in_its_group():
    for bad in (float("inf"), float("nan")):
        x = torch.randn(3, 40, 32, device="cuda")
        x[1, 7, 9] = bad
        clean = x.clone()
        clean[1, 7, 9] = 0
        outs = []
        for v in (x, clean):
            y, mean, rstd = torch.empty_like(v), *(torch.empty(3, 4, device="cuda") for _ in range(2))
            assert pb.group_norm(v, None, None, y, mean, rstd, 4, scratch(3, 40, 32, 4, F), activation=pb.ACT_RELU) == pb.OK
            outs.append(y)
        hit = torch.zeros(3, 40, 32, dtype=torch.bool, device="cuda")
        hit[1, :, 8:16] = True
        assert torch.equal(outs[0][~hit], outs[1][~hit]) and bool(torch.isnan(outs[0][hit]).any())


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("n,p,c,g", [(4, 100, 32, 4), (1, 40000, 16, 4)])
def test_in_place_and_gradients_that_are_not_wanted(n, p, c, g, dtype):
    xt, y, gamma, beta, mean, rstd = check_forward(n, p, c, g, dtype, "silu")
    own = xt.clone()
    assert pb.group_norm(own, gamma, beta, own, None, None, g, scratch(n, p, c, g, dtype), activation=pb.ACT_SILU) == pb.OK
    assert torch.equal(own, y)
    xt, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, room = check_backward(n, p, c, g, dtype, "silu")
    for want in ((1, 0, 0), (0, 1, 0), (0, 0, 1)):
        out = [torch.zeros_like(v) if w else None for v, w in zip((dx, dgamma, dbeta), want)]
        assert pb.group_norm_backward(xt, dy, gamma, beta, mean, rstd, *out, g, room, activation=pb.ACT_SILU) == pb.OK
        for o, v in zip(out, (dx, dgamma, dbeta)):
            assert o is None or torch.equal(o, v)
    assert pb.group_norm_backward(xt, dy, gamma, beta, mean, rstd, dy, dgamma, dbeta, g, room, activation=pb.ACT_SILU) == pb.OK
    assert torch.equal(dy, dx)


@pytest.mark.parametrize("n,p,c,g", [(6, 81, 64, 8), (1, 30000, 16, 2)])
def test_recorded_replayed_and_the_same_bits_every_time(n, p, c, g):
    xt, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, room = check_backward(n, p, c, g, H, "relu")
    y = torch.empty_like(xt)
    outs = (y, mean, rstd, dx, dgamma, dbeta)

    def both():
        assert pb.group_norm(xt, gamma, beta, y, mean, rstd, g, room, activation=pb.ACT_RELU) == pb.OK
        assert pb.group_norm_backward(xt, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, g, room, activation=pb.ACT_RELU) == pb.OK

    both()
    want = [v.clone() for v in outs]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for v in (y, dx, dgamma, dbeta):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(v, w) for v, w in zip(outs, want))


def test_four_axes_and_strides_that_do_not_join():
    x = torch.randn(2, 6, 5, 16, device="cuda")
    y, z = torch.empty_like(x), torch.empty(2, 30, 16, device="cuda")
    room = scratch(2, 30, 16, 4, F)
    assert pb.group_norm(x, None, None, y, None, None, 4, room) == pb.OK
    assert pb.group_norm(x.view(2, 30, 16), None, None, z, None, None, 4, room) == pb.OK
    assert torch.equal(y.view(2, 30, 16), z)
    assert pb.group_norm(torch.randn(2, 6, 8, 16, device="cuda")[:, :, :5], None, None, y, None, None, 4, room) == pb.ERR_ARG


def test_samples_beyond_32_bits():
    """Samples more than 2^31 elements apart."""
    far = 2 ** 31 + 64
    buf = torch.zeros(far + 320, dtype=H, device="cuda")
    x = buf.as_strided((2, 20, 16), (far, 16, 1))
    x.copy_(torch.randn(2, 20, 16))
    y = torch.empty(2, 20, 16, dtype=H, device="cuda")
    assert pb.group_norm(x, None, None, y, None, None, 2, scratch(2, 20, 16, 2, H)) == pb.OK
    want, _, _, _ = norm_forward(f64(x), np.ones(16), np.zeros(16), 2, "none", 1e-5)
    assert_within(y, want, 1e-5 + half_step(H) * np.abs(want) * 1.01)


def test_the_most_pixels_there_may_be():
    """2^31 - 1 pixels of one channel, against sums and formulas in 64 bits.  A block leaves one part of 4,096 pixels, 524,288 parts in all: a lane adds
    up 16,384 of them for the mean and the deviation, and a lane all of them one after the other for the group's gradient."""
    n = 2 ** 31 - 1
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy = torch.empty(1, n, 1, dtype=H, device="cuda"), torch.empty(1, n, 1, dtype=H, device="cuda")
    parts = [slice(i, min(i + 2 ** 26, n)) for i in range(0, n, 2 ** 26)]
    for at in parts:
        x[0, at, 0] = (torch.randn(at.stop - at.start, device="cuda", generator=gen) + 0.5).to(H)
        dy[0, at, 0] = (torch.randn(at.stop - at.start, device="cuda", generator=gen) + 0.25).to(H)
    y, dx = torch.empty_like(x), torch.empty_like(dy)
    gamma, beta = torch.full((1,), 1.25, device="cuda"), torch.full((1,), -0.5, device="cuda")
    mean, rstd, dgamma, dbeta = torch.zeros(1, 1, device="cuda"), torch.zeros(1, 1, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    room = scratch(1, n, 1, 1, H)
    assert pb.group_norm(x, gamma, beta, y, mean, rstd, 1, room) == pb.OK
    assert pb.group_norm_backward(x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, 1, room) == pb.OK

    def total(f):
        return sum(float(f(x[0, at, 0].double(), dy[0, at, 0].double()).sum()) for at in parts)

    m, size = total(lambda v, d: v) / n, total(lambda v, d: v.abs()) / n
    r = 1 / np.sqrt(total(lambda v, d: (v - m) ** 2) / n + float(np.float32(1e-5)))
    depth = (DEPTH + 16384) * U
    dmean = depth * size
    drstd = depth + 4 * U + 0.5 * (r * dmean) ** 2
    got_m, got_r = float(mean), float(rstd)
    assert abs(got_m - m) <= dmean and abs(got_r - r) <= r * drstd
    for at in parts:
        v = (x[0, at, 0].double() - m) * r * 1.25
        off = 1.1 * (1.25 * r * dmean + v.abs() * (drstd + 4 * U)) + 2 * U * (v - 0.5).abs()
        want = v - 0.5
        assert bool(((y[0, at, 0].double() - want).abs() <= off + half_step(H) * (want.abs() + off)).all())
    # the gradient, from the statistics as they were given
    wb, wg = total(lambda v, d: d), total(lambda v, d: d * (v - got_m) * got_r)
    ab, ag = total(lambda v, d: d.abs()), total(lambda v, d: (d * (v - got_m) * got_r).abs())
    lanes = (DEPTH + 524288 / 128 + 32) * U
    assert abs(float(dbeta) - wb) <= lanes * ab and abs(float(dgamma) - wg) <= (lanes + 4 * U) * ag
    chain = (DEPTH + 524288) * U
    s1, s2 = 1.25 * wb / n, 1.25 * wg / n
    for at in parts:
        d, xhat = dy[0, at, 0].double() * 1.25, (x[0, at, 0].double() - got_m) * got_r
        want = got_r * (d - s1 - xhat * s2)
        off = got_r * 1.25 * ((chain + 8 * U) * (ab / n + xhat.abs() * ag / n) + 8 * U * d.abs())
        assert bool(((dx[0, at, 0].double() - want).abs() <= off + half_step(H) * (want.abs() + off)).all())


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("n,p,c,g", [(9, 49, 32, 4), (2, 40000, 16, 2)])
def test_every_array_with_a_layout_of_its_own(n, p, c, g, dtype, act):
    """Parts of wider pixels beside contiguous ones and every other pixel, inputs that are the same for every sample or pixel (a stride of 0): the
    same bits as from contiguous copies, the accesses' width being the same."""
    gen = torch.Generator(device="cuda").manual_seed(n + p)

    def noise(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(dtype)

    def one(layout):
        return images(n, p, c, dtype, layout)[0]

    sets = [(one("packed").copy_(noise(n, p, c)), one("plain"), one("sparse").copy_(noise(n, p, c)), one("packed")),
            (noise(p, c).expand(n, p, c), one("sparse"), noise(n, 1, c).expand(n, p, c), one("plain")),
            (one("sparse").copy_(noise(n, p, c)), one("packed"), noise(c).expand(n, p, c), one("sparse"))]
    room = scratch(n, p, c, g, dtype)
    for x, y, dy, dx in sets:
        outs = []
        for turn in range(2):
            if turn:
                x, dy, y, dx = x.contiguous(), dy.contiguous(), one("plain"), one("plain")
            mean, rstd, dgamma, dbeta = (torch.full(s, 9.0, device="cuda") for s in ((n, g), (n, g), (c,), (c,)))
            assert pb.group_norm(x, None, None, y, mean, rstd, g, room, activation=ACT[act]) == pb.OK
            assert pb.group_norm_backward(x, dy, None, None, mean, rstd, dx, dgamma, dbeta, g, room, activation=ACT[act]) == pb.OK
            outs.append((y, mean, rstd, dx, dgamma, dbeta))
        for first, other in zip(*outs):
            assert bool(torch.isfinite(first.float()).all()) and torch.equal(first, other)
