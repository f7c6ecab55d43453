"""The short causal convolution and its gradient (paac_causal_conv) against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from operators_ref import U, assert_within, f64, half_step
from paper_1705_04862_b200 import binding as pb
from sequence_ref import conv_backward, conv_forward

pytestmark = pytest.mark.gpu
F, H = torch.float32, torch.bfloat16
TYPES = {F: pb.FP32, H: pb.BF16}
ACT = {"none": pb.ACT_NONE, "relu": pb.ACT_RELU, "silu": pb.ACT_SILU}


def sequences(t, n, c, dtype, layout, count):
    """`count` tensors [t][n][c]: steps first, sequences first, parts of wider rows, or at odd places with gaps."""
    if layout == "batch":
        return [torch.zeros(n, t, c, dtype=dtype, device="cuda").transpose(0, 1) for _ in range(count)]
    if layout == "packed":
        whole = torch.zeros(t, n, count * c, dtype=dtype, device="cuda")
        return [whole[..., i * c:(i + 1) * c] for i in range(count)]
    if layout == "odd":
        return [torch.zeros(t, n + 1, c + 3, dtype=dtype, device="cuda")[:, 1:, 1:c + 1] for _ in range(count)]
    return [torch.zeros(t, n, c, dtype=dtype, device="cuda") for _ in range(count)]


def case(t, n, c, width, dtype, layout, restart, carry, kind, seed=0):
    rng = np.random.RandomState(seed + 7 * t + 3 * n + c + width)
    x, dy = sequences(t, n, c, dtype, layout, 2)
    x.copy_(torch.from_numpy(rng.randn(t, n, c)))
    w, bias = (torch.from_numpy(v).float().cuda() for v in (rng.randn(c, width) / 2, rng.randn(c) / 4))
    flags = torch.from_numpy((rng.rand(t, n) < restart).astype(np.uint8) * rng.randint(1, 256, (t, n)).astype(np.uint8)).cuda() if restart else None
    before, dafter = (torch.from_numpy(rng.randn(n, width - 1, c)).cuda().to(dtype) if carry else None for _ in range(2))
    g = rng.randn(t, n, c)
    if kind == "relu":
        # nothing arrives where the argument is within its error of the corner
        v = conv_forward(f64(x), f64(w), f64(bias), f64(before), None if flags is None else flags.cpu().numpy(), "none", dtype)[0]
        g *= np.abs(v) > 1e-4
    dy.copy_(torch.from_numpy(g))
    return dict(x=x, dy=dy, w=w, bias=bias, restart=flags, before=before, dafter=dafter)


def check(t, n, c, width, dtype, layout="time", restart=0.1, carry=True, kind="silu"):
    k = case(t, n, c, width, dtype, layout, restart, carry, kind)
    flags = None if k["restart"] is None else k["restart"].cpu().numpy()
    args = f64(k["x"]), f64(k["w"]), f64(k["bias"]), f64(k["before"])
    (y,) = sequences(t, n, c, dtype, layout, 1)
    after = torch.full((n, width - 1, c), 9.0, device="cuda", dtype=dtype) if carry else None
    assert pb.causal_conv(k["x"], k["w"], k["bias"], y, before=k["before"], after=after, restart=k["restart"], activation=ACT[kind]) == pb.OK
    want, held, bound = conv_forward(*args, flags, kind, dtype)
    assert_within(y, want, bound + half_step(dtype) * (np.abs(want) + bound), "y")
    if carry:
        assert np.array_equal(f64(after), held)
    dx, = sequences(t, n, c, dtype, layout, 1)
    dw, dbias = torch.full((c, width), 9.0, device="cuda"), torch.full((c,), 9.0, device="cuda")
    dbefore = torch.full((n, width - 1, c), 9.0, device="cuda", dtype=dtype) if carry else None
    room = torch.full((pb.causal_conv_workspace_bytes(t, n, c, width, TYPES[dtype]),), 255, dtype=torch.uint8, device="cuda")
    assert pb.causal_conv_backward(k["x"], k["dy"], k["w"], k["bias"], dx, dw, dbias, room, before=k["before"], dafter=k["dafter"], dbefore=dbefore, restart=k["restart"],
                                   activation=ACT[kind]) == pb.OK
    # a thread adds up its part of at least 16 steps, five exchanges in a warp, the warps of a block, then in 64 bits
    chain = 16 + t * n * c // (4 * 148 * 512) + 5 + 8 + 2
    want = conv_backward(args[0], f64(k["dy"]), *args[1:], f64(k["dafter"]), flags, kind, dtype, chain)
    for name, got in (("dx", dx), ("dbefore", dbefore), ("dweight", dw), ("dbias", dbias)):
        if got is not None:
            value, bound = want[name]
            stored = half_step(got.dtype) * (np.abs(value) + bound)
            assert_within(got, value, bound + stored, name)
    return k, y, dx, dw


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("t,n,c", [(1, 1, 1), (1, 32, 64), (2, 3, 7), (3, 2, 8), (5, 4, 130), (16, 3, 33), (17, 2, 24), (50, 3, 40), (333, 2, 20)])
def test_sizes(t, n, c, width, dtype):
    check(t, n, c, width, dtype)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("layout", ["time", "batch", "packed", "odd"])
@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
def test_layouts_and_activations(layout, kind, dtype):
    check(37, 3, 24, 4, dtype, layout=layout, kind=kind)


@pytest.mark.parametrize("restart,carry", [(0, False), (0, True), (0.9, True), (1.0, True), (0.3, False)])
def test_restarts_and_carried_inputs(restart, carry):
    check(40, 4, 16, 4, F, restart=restart, carry=carry)


def test_long_parts():
    """Sizes at which a thread's part is longer than the shortest, and the sums of many blocks."""
    check(1500, 40, 128, 4, H, carry=False, kind="silu")


def test_no_bias_and_gradients_left_out():
    k = case(20, 2, 8, 3, F, "time", 0.2, True, "silu")
    y, z = torch.empty_like(k["x"]), torch.empty_like(k["x"])
    assert pb.causal_conv(k["x"], k["w"], None, y, before=k["before"], restart=k["restart"]) == pb.OK
    assert pb.causal_conv(k["x"], k["w"], torch.zeros(8, device="cuda"), z, before=k["before"], restart=k["restart"]) == pb.OK
    assert torch.equal(y, z)
    room = torch.empty(pb.causal_conv_workspace_bytes(20, 2, 8, 3, pb.FP32), dtype=torch.uint8, device="cuda")
    dx, dw, db, dx2, dw2, db2 = (torch.zeros_like(v) for v in (k["x"], k["w"], k["bias"]) * 2)
    how = dict(before=k["before"], restart=k["restart"])
    assert pb.causal_conv_backward(k["x"], k["dy"], k["w"], k["bias"], dx, dw, db, room, **how) == pb.OK
    for a, b, c in ((dx2, None, None), (None, dw2, None), (None, None, db2)):
        assert pb.causal_conv_backward(k["x"], k["dy"], k["w"], k["bias"], a, b, c, room, **how) == pb.OK
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("dtype", [F, H])
def test_step_by_step_is_the_whole(dtype):
    """Single steps with the inputs carried on in place, parts of any length: the same bits as the whole at once."""
    t, n, c = 23, 5, 40
    k = case(t, n, c, 4, dtype, "time", 0.15, True, "silu")
    y, after = torch.empty_like(k["x"]), torch.empty_like(k["before"])
    assert pb.causal_conv(k["x"], k["w"], k["bias"], y, before=k["before"], after=after, restart=k["restart"]) == pb.OK
    for lengths in ([1] * t, [2, 1, 3, 17], [22, 1]):
        held, out, at = k["before"].clone(), torch.empty_like(y), 0
        for m in lengths:
            assert pb.causal_conv(k["x"][at:at + m], k["w"], k["bias"], out[at:at + m], before=held, after=held, restart=k["restart"][at:at + m]) == pb.OK
            at += m
        assert torch.equal(out, y) and torch.equal(held, after)


def test_what_a_restart_cuts_off_is_not_looked_at():
    """Infinities and NaNs before a restart reach nothing behind it."""
    k = case(30, 2, 8, 4, F, "time", 0, True, "silu")
    flags = torch.zeros(30, 2, dtype=torch.uint8, device="cuda")
    flags[10] = 1
    x, before = k["x"].clone(), k["before"].clone()
    x[:10] = float("nan")
    x[3] = float("inf")
    before[:] = float("nan")
    y, z = torch.empty_like(x), torch.empty_like(x)
    a, b = torch.empty_like(before), torch.empty_like(before)
    assert pb.causal_conv(x, k["w"], k["bias"], y, before=before, after=a, restart=flags) == pb.OK
    assert pb.causal_conv(k["x"], k["w"], k["bias"], z, before=k["before"], after=b, restart=flags) == pb.OK
    assert torch.equal(y[10:], z[10:]) and torch.isnan(y[4:10]).all() and torch.equal(a, b)


def test_the_same_bits_every_time_and_on_another_stream():
    k = case(400, 6, 96, 4, H, "batch", 0.05, False, "silu")
    room = torch.empty(pb.causal_conv_workspace_bytes(400, 6, 96, 4, pb.BF16), dtype=torch.uint8, device="cuda")
    got = []
    for stream in (None, torch.cuda.Stream(), torch.cuda.Stream()):
        dx, dw, db = torch.empty_like(k["x"]), torch.empty_like(k["w"]), torch.empty_like(k["bias"])
        torch.cuda.synchronize()
        assert pb.causal_conv_backward(k["x"], k["dy"], k["w"], k["bias"], dx, dw, db, room, restart=k["restart"],
                                       stream=None if stream is None else stream.cuda_stream) == pb.OK
        torch.cuda.synchronize()
        got.append((dx, dw, db))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_recorded_into_a_graph():
    k = case(60, 3, 64, 4, H, "time", 0.1, True, "silu")
    room = torch.empty(pb.causal_conv_workspace_bytes(60, 3, 64, 4, pb.BF16), dtype=torch.uint8, device="cuda")

    def run(y, dx, dw, db):
        assert pb.causal_conv(k["x"], k["w"], k["bias"], y, before=k["before"], restart=k["restart"]) == pb.OK
        assert pb.causal_conv_backward(k["x"], k["dy"], k["w"], k["bias"], dx, dw, db, room, before=k["before"], restart=k["restart"]) == pb.OK

    def outs():
        return torch.zeros_like(k["x"]), torch.zeros_like(k["x"]), torch.zeros_like(k["w"]), torch.zeros_like(k["bias"])

    eager, taped = outs(), outs()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(*taped)
    for seed in (1, 2):
        k["x"].copy_(torch.randn(60, 3, 64, generator=torch.Generator().manual_seed(seed)))
        g.replay()
        run(*eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, taped))


def test_rows_beside_are_left_alone():
    whole = torch.full((9, 4, 30), 7.0, device="cuda", dtype=H)
    k = case(9, 4, 11, 4, H, "time", 0.1, False, "silu")
    y = whole[:, :, 13:24]
    assert pb.causal_conv(k["x"], k["w"], k["bias"], y, restart=k["restart"]) == pb.OK
    assert (whole[:, :, :13] == 7).all() and (whole[:, :, 24:] == 7).all()


def test_steps_far_apart_and_shared():
    """Steps whose places are beyond 32 bits, and one row of inputs for all sequences."""
    t, n, c = 20, 2, 24
    k = case(t, n, c, 4, H, "time", 0.1, False, "silu")
    step = 1 << 28
    whole = torch.empty(t * step, dtype=H, device="cuda")
    x, dy, y, dx = (whole.as_strided((t, n, c), (step, c, 1), i * n * c) for i in range(4))
    x.copy_(k["x"])
    dy.copy_(k["dy"])
    near, dnear = torch.empty_like(k["x"]), torch.empty_like(k["x"])
    room = torch.empty(pb.causal_conv_workspace_bytes(t, n, c, 4, pb.BF16), dtype=torch.uint8, device="cuda")
    dw, db, dw2, db2 = (torch.empty_like(v) for v in (k["w"], k["bias"]) * 2)
    assert pb.causal_conv(x, k["w"], k["bias"], y, restart=k["restart"]) == pb.causal_conv(k["x"], k["w"], k["bias"], near, restart=k["restart"]) == pb.OK
    assert pb.causal_conv_backward(x, dy, k["w"], k["bias"], dx, dw, db, room, restart=k["restart"]) == pb.OK
    assert pb.causal_conv_backward(k["x"], k["dy"], k["w"], k["bias"], dnear, dw2, db2, room, restart=k["restart"]) == pb.OK
    assert torch.equal(y, near) and torch.equal(dx, dnear) and torch.equal(dw, dw2) and torch.equal(db, db2)
    shared = k["x"][:, :1].expand(t, n, c)
    assert pb.causal_conv(shared, k["w"], k["bias"], near, restart=k["restart"]) == pb.causal_conv(shared.contiguous(), k["w"], k["bias"], dnear, restart=k["restart"]) == pb.OK
    assert torch.equal(near, dnear)
