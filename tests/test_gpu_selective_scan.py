"""The selective state space scan and its gradient (paac_selective_scan) against the recurrence step by step in 64 bits."""
import numpy as np
import pytest
import torch

from operators_ref import U, f64, half_step
from paper_1705_04862_b200 import binding as pb
from sequence_ref import SPAN, Scan, assert_bounded
from test_gpu_causal_conv import sequences

pytestmark = pytest.mark.gpu
F, H = torch.float32, torch.bfloat16
TYPES = {F: pb.FP32, H: pb.BF16}


def case(t, n, c, state, dtype, groups=1, layout="time", restart=0.05, carry=True, gate=True, softplus=True, plain=False, seed=0):
    """`plain`: no D, no bias."""
    rng = np.random.RandomState(seed + 7 * t + 3 * n + c + state)
    x, dt, z, y, dy, dx, ddt, dz = sequences(t, n, c, dtype, layout, 8)
    x.copy_(torch.from_numpy(rng.randn(t, n, c)))
    dt.copy_(torch.from_numpy(rng.randn(t, n, c) * 0.5 - (0 if softplus else -0.1)).abs() if not softplus else torch.from_numpy(rng.randn(t, n, c) * 0.5))
    z.copy_(torch.from_numpy(rng.randn(t, n, c)))
    dy.copy_(torch.from_numpy(rng.randn(t, n, c)))
    B, C, dB, dC = sequences(t, n, groups * state, dtype, layout, 4)
    B.copy_(torch.from_numpy(rng.randn(t, n, groups * state)))
    C.copy_(torch.from_numpy(rng.randn(t, n, groups * state)))
    B, C, dB, dC = (v.unflatten(2, (groups, state)) for v in (B, C, dB, dC))

    def floats(v):
        return torch.from_numpy(v).float().cuda()

    A = floats(-np.arange(1, state + 1) * np.exp(0.1 * rng.randn(c, state)))
    D, bias = (None, None) if plain else (floats(1 + 0.1 * rng.randn(c)), floats(rng.uniform(-6, -1, c)))
    flags = torch.from_numpy((rng.rand(t, n) < restart).astype(np.uint8) * 3).cuda() if restart else None
    h0, dh_last = (floats(rng.randn(n, c, state)) if carry else None for _ in range(2))
    return dict(x=x, dt=dt, A=A, B=B, C=C, D=D, z=z if gate else None, bias=bias, restart=flags, h0=h0, dh_last=dh_last, y=y, dy=dy, dx=dx, ddt=ddt, dz=dz if gate else None,
                dB=dB, dC=dC, softplus=softplus, dtype=dtype)


def reference(k):
    return Scan(f64(k["x"]), f64(k["dt"]), f64(k["A"]), f64(k["B"]), f64(k["C"]), f64(k["D"]), f64(k["z"]), f64(k["bias"]), f64(k["h0"]),
                None if k["restart"] is None else k["restart"].cpu().numpy(), k["softplus"], k["dtype"])


def room(k, backward):
    t, n, c = k["x"].shape
    g, m = k["B"].shape[2:]
    return torch.full((pb.selective_scan_workspace_bytes(t, n, c, m, g, TYPES[k["dtype"]], backward=backward),), 255, dtype=torch.uint8, device="cuda")


def forward(k, marks=True):
    t, n, c = k["x"].shape
    m = k["A"].shape[1]
    last = torch.full((n, c, m), 9.0, device="cuda")
    states = torch.full((-(-t // SPAN), n, c, m), 9.0, device="cuda") if marks else None
    assert pb.selective_scan(k["x"], k["dt"], k["A"], k["B"], k["C"], k["y"], room(k, False), D=k["D"], z=k["z"], dt_bias=k["bias"], h0=k["h0"],
                             h_last=last, states=states, restart=k["restart"], softplus=k["softplus"]) == pb.OK
    return last, states


def backward(k, states):
    t, n, c = k["x"].shape
    m = k["A"].shape[1]
    g = dict(dA=torch.full((c, m), 9.0, device="cuda"), dD=torch.full((c,), 9.0, device="cuda"), ddt_bias=torch.full((c,), 9.0, device="cuda"),
             dh0=torch.full((n, c, m), 9.0, device="cuda"))
    assert pb.selective_scan_backward(k["x"], k["dt"], k["A"], k["B"], k["C"], k["dy"], states, k["dx"], k["ddt"], g["dA"], k["dB"], k["dC"],
                                      room(k, True), D=k["D"], z=k["z"], dt_bias=k["bias"], dD=g["dD"], dz=k["dz"],
                                      ddt_bias=g["ddt_bias"], dh_last=k["dh_last"], dh0=g["dh0"], restart=k["restart"], softplus=k["softplus"]) == pb.OK
    g.update({name: k[name] for name in ("dx", "ddt", "dz", "dB", "dC") if k[name] is not None})
    return g


def check(*shape, **how):
    """Forward against the reference, then backward from the states that the forward pass has kept."""
    k = case(*shape, **how)
    ref = reference(k)
    last, states = forward(k)
    assert_bounded(k["y"], ref.y, ref.by + half_step(k["dtype"]) * (np.abs(ref.y) + ref.by), "y")
    assert_bounded(last, ref.last, ref.blast, "h_last")
    for i, s in enumerate(ref.states):
        assert_bounded(states[i], s, ref.before[i * SPAN][1], "states")
    got, want = backward(k, states), ref.backward(f64(k["dy"]), f64(k["dh_last"]))
    for name, tensor in got.items():
        value, bound = want[name]
        assert_bounded(tensor, value, bound + half_step(tensor.dtype) * (np.abs(value) + bound), name)
    return k


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c,state", [(1, 1, 1, 1), (1, 32, 64, 16), (1, 3, 7, 5), (2, 2, 5, 16), (4, 3, 130, 16), (5, 2, 12, 8), (15, 1, 40, 16), (16, 2, 36, 4), (17, 2, 36, 16),
                                         (33, 3, 20, 24), (40, 2, 9, 64), (31, 1, 256, 3), (50, 1, 300, 16)])
def test_sizes(t, n, c, state, dtype):
    check(t, n, c, state, dtype)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("layout", ["time", "batch", "packed", "odd"])
@pytest.mark.parametrize("groups", [1, 3])
def test_layouts_and_groups(layout, groups, dtype):
    check(37, 2, 24, 16, dtype, groups=groups, layout=layout)


@pytest.mark.parametrize("how", [dict(gate=False), dict(plain=True), dict(plain=True, gate=False, softplus=False), dict(softplus=False), dict(carry=False, restart=0), dict(restart=0),
                                 dict(restart=0.9), dict(restart=1.0), dict(groups=4), dict(groups=24)])
@pytest.mark.parametrize("t", [1, 30])
def test_what_may_be_left_out(how, t):
    check(t, 3, 24, 16, F, **how)


@pytest.mark.parametrize("t,n,c,state,restart", [(130, 1, 20, 16, 0.01), (700, 1, 24, 16, 0.003), (700, 2, 8, 8, 0), (1100, 1, 5, 64, 0.002), (400, 1, 130, 3, 0.01), (96, 1, 4, 1, 0)])
@pytest.mark.parametrize("dtype", [F, H])
def test_steps_cut_into_chunks(t, n, c, state, restart, dtype):
    """Few channels with many steps, whose chunks are walked side by side: forward from twelve windows on, backward from three."""
    k = check(t, n, c, state, dtype, restart=restart)
    assert (room(k, False).numel() > 0) == (t > 11 * SPAN)


def test_step_by_step_is_the_whole():
    """Single steps with the state carried on in place, and parts of any length, against the whole at once: within both sides' bounds."""
    t, n, c, m = 40, 3, 20, 16
    k = case(t, n, c, m, F)
    ref = reference(k)
    for lengths in ([1] * t, [7, 1, 20, 12]):
        h, y, at = k["h0"].clone(), torch.empty_like(k["y"]), 0
        for q in lengths:
            cut = slice(at, at + q)
            need = pb.selective_scan_workspace_bytes(q, n, c, m, 1, pb.FP32)
            work = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
            assert pb.selective_scan(k["x"][cut], k["dt"][cut], k["A"], k["B"][cut], k["C"][cut], y[cut], work, D=k["D"], z=k["z"][cut], dt_bias=k["bias"], h0=h, h_last=h,
                                     restart=k["restart"][cut]) == pb.OK
            at += q
        assert_bounded(y, ref.y, ref.by + U * (np.abs(ref.y) + ref.by), "y")
        assert_bounded(h, ref.last, ref.blast, "h_last")


def test_state_replaced_while_steps_are_cut():
    """h_last in h0's place where chunks run side by side."""
    k = case(500, 1, 24, 16, F)
    last, _ = forward(k)
    y = k["y"].clone()
    h = k["h0"].clone()
    assert pb.selective_scan(k["x"], k["dt"], k["A"], k["B"], k["C"], k["y"], room(k, False), D=k["D"], z=k["z"], dt_bias=k["bias"], h0=h, h_last=h, restart=k["restart"]) == pb.OK
    assert torch.equal(h, last) and torch.equal(y, k["y"])


@pytest.mark.parametrize("t", [30, 600])
def test_what_a_restart_cuts_off_is_not_looked_at(t):
    """Infinities and NaNs before a restart reach nothing behind it, forward and backward."""
    k = case(t, 1, 24, 16, F, restart=0)
    k["restart"] = torch.zeros(t, 1, dtype=torch.uint8, device="cuda")
    k["restart"][t // 2] = 1
    clean_last, states = forward(k)
    y = k["y"].clone()
    clean = {name: v.clone() for name, v in backward(k, states).items()}
    k["h0"][:] = float("nan")
    k["x"][:t // 4] = float("inf")
    last, states = forward(k)
    assert torch.equal(last, clean_last) and torch.equal(k["y"][t // 2:], y[t // 2:]) and torch.isnan(k["y"][t // 4 + 1:t // 2]).all()
    got = backward(k, states)
    for name in ("dx", "ddt", "dB", "dC", "dz"):
        assert torch.equal(got[name][t // 2:], clean[name][t // 2:]), name
    k = case(t, 1, 24, 16, F, restart=0)
    k["restart"] = torch.zeros(t, 1, dtype=torch.uint8, device="cuda")
    k["restart"][t // 2] = 1
    _, states = forward(k)
    clean = {name: v.clone() for name, v in backward(k, states).items()}
    k["dh_last"][:] = float("nan")
    k["dy"][t // 2 + 3:] = float("inf")
    got = backward(k, states)
    for name in ("dx", "ddt", "dB", "dC", "dz"):
        assert torch.equal(got[name][:t // 2], clean[name][:t // 2]), name
    assert torch.equal(got["dh0"], clean["dh0"])


def test_gradients_left_out():
    k = case(40, 2, 24, 16, F)
    _, states = forward(k)
    whole = {name: v.clone() for name, v in backward(k, states).items()}
    work = room(k, True)
    for name, v in whole.items():
        only = {q: None for q in ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias", "dh0")}
        only[name] = torch.zeros_like(v)
        assert pb.selective_scan_backward(k["x"], k["dt"], k["A"], k["B"], k["C"], k["dy"], states, only["dx"], only["ddt"], only["dA"], only["dB"], only["dC"], work, D=k["D"], z=k["z"],
                                          dt_bias=k["bias"], dD=only["dD"], dz=only["dz"], ddt_bias=only["ddt_bias"], dh_last=k["dh_last"], dh0=only["dh0"],
                                          restart=k["restart"]) == pb.OK
        assert torch.equal(only[name], v), name


@pytest.mark.parametrize("t,n,c", [(60, 5, 200), (900, 1, 64)])
def test_the_same_bits_every_time_and_on_another_stream(t, n, c):
    k = case(t, n, c, 16, H, layout="batch")
    got = []
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()):
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            last, states = forward(k)
            got.append([k["y"].clone(), last, states] + [v.clone() for v in backward(k, states).values()])
            stream.synchronize()
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("t,n,c", [(1, 4, 64), (40, 2, 64), (600, 1, 32)])
def test_recorded_into_a_graph(t, n, c):
    k = case(t, n, c, 16, H)
    taped = dict(k, y=torch.zeros_like(k["y"]))
    f, b = room(k, False), room(k, True)
    last, states = torch.empty(n, c, 16, device="cuda"), torch.empty(-(-t // SPAN), n, c, 16, device="cuda")
    grads = {name: torch.zeros(*s, device="cuda") for name, s in dict(dA=(c, 16), dD=(c,), ddt_bias=(c,), dh0=(n, c, 16)).items()}

    def run():
        assert pb.selective_scan(k["x"], k["dt"], k["A"], k["B"], k["C"], taped["y"], f, D=k["D"], z=k["z"], dt_bias=k["bias"], h0=k["h0"], h_last=last, states=states,
                                 restart=k["restart"]) == pb.OK
        assert pb.selective_scan_backward(k["x"], k["dt"], k["A"], k["B"], k["C"], k["dy"], states, k["dx"], k["ddt"], grads["dA"], k["dB"], k["dC"], b, D=k["D"], z=k["z"],
                                          dt_bias=k["bias"], dD=grads["dD"], dz=k["dz"], ddt_bias=grads["ddt_bias"], dh_last=k["dh_last"], dh0=grads["dh0"],
                                          restart=k["restart"]) == pb.OK

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    every = [taped["y"], last, states, k["dx"], k["ddt"], k["dB"], k["dC"], k["dz"], *grads.values()]
    for seed in (1, 2):
        k["x"].copy_(torch.randn(t, n, c, generator=torch.Generator().manual_seed(seed)))
        for v in every:
            v.zero_()
        g.replay()
        torch.cuda.synchronize()
        first = [v.clone() for v in every]
        for v in every:
            v.zero_()
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, every))


def test_rows_beside_are_left_alone():
    k = case(20, 3, 11, 5, H)
    whole = torch.full((20, 3, 30), 7.0, device="cuda", dtype=H)
    k["y"] = whole[:, :, 13:24]
    forward(k, marks=False)
    assert (whole[:, :, :13] == 7).all() and (whole[:, :, 24:] == 7).all()


def test_the_gated_scan_is_a_case_of_it():
    """One state, no gate, delta = the step itself: h_t = exp(delta A) h + delta x is a gated scan with gate exp(delta A), whose kernels are others."""
    t, n, c = 200, 3, 40
    k = case(t, n, c, 1, F, gate=False, plain=True, softplus=False, restart=0.05)
    k["B"].fill_(1.0)
    k["C"].fill_(1.0)
    last, _ = forward(k, marks=False)
    gate, x, h, h_last = torch.exp(k["dt"] * k["A"][:, 0]), k["dt"] * k["x"], torch.empty_like(k["y"]), torch.empty(n, c, device="cuda")
    assert pb.gated_scan(gate, x, h, h0=k["h0"][..., 0].contiguous(), h_last=h_last, restart=k["restart"], kind=pb.SCAN_LINEAR) == pb.OK
    ref = reference(k)
    assert_bounded(h, ref.y, 2 * ref.by + 8 * U * np.abs(ref.y), "h")
    assert_bounded(k["y"], ref.y, ref.by, "y")


@pytest.mark.parametrize("t,n,c,state,groups,dtype", [(87, 2, 80, 5, 1, F), (4, 41, 64, 8, 1, F), (33, 3, 24, 16, 2, H), (1, 4, 7, 3, 1, H)])
def test_everything_in_one_tensor(t, n, c, state, groups, dtype):
    """x, dt, B, C and z side by side in one tensor, as a projection leaves them, and their gradients in another: the same bits as apart from one another, but
    for two sums over steps, whose order goes with the accesses."""
    k = case(t, n, c, state, dtype, groups=groups)
    last, states = forward(k)
    y, want = k["y"].clone(), {name: v.clone() for name, v in backward(k, states).items()}
    gs = groups * state
    widths = dict(x=c, dt=c, B=gs, C=gs, z=c)
    for names in (list(widths), ["d" + name for name in widths]):
        whole, at = torch.full((t, n, 3 * c + 2 * gs), 7.0, dtype=dtype, device="cuda"), 0
        for name in names:
            width = widths[name] if name in widths else widths[name[1:]]
            view = whole[..., at:at + width]
            view = view.unflatten(2, (groups, state)) if name[-1] in "BC" else view
            if name in widths:
                view.copy_(k[name])
            k[name] = view
            at += width
    last2, states2 = forward(k)
    assert torch.equal(k["y"], y) and torch.equal(last2, last) and torch.equal(states2, states)
    bounds = reference(k).backward(f64(k["dy"]), f64(k["dh_last"]))
    for name, v in backward(k, states).items():
        if name in ("dD", "ddt_bias"):
            value, bound = bounds[name]
            assert_bounded(v, value, bound + U * np.abs(value), name)
        else:
            assert torch.equal(v, want[name]), name


@pytest.mark.parametrize("t,n,c,state,dtype", [(1, 2700, 70, 16, F), (2, 900, 200, 8, H), (8, 2500, 3, 5, F), (5, 2400, 20, 24, F)])
def test_blocks_that_take_several_sequences(t, n, c, state, dtype):
    """Few steps of many sequences."""
    check(t, n, c, state, dtype, restart=0.2)


@pytest.mark.parametrize("t", [1, 12, 40, 400])
def test_arrays_at_odd_places(t):
    """States, rates and marks that begin four bytes from where they would be accessed four at a time: the same bits."""
    n, c, m = 2, 24, 16
    k = case(t, n, c, m, F)
    last, states = forward(k)
    y, want = k["y"].clone(), {name: v.clone() for name, v in backward(k, states).items()}

    def odd(v):
        return torch.cat([v.new_zeros(1), v.reshape(-1)])[1:].view(v.shape)

    k.update(A=odd(k["A"]), h0=odd(k["h0"]), dh_last=odd(k["dh_last"]))
    last2, states2 = forward(k)
    assert torch.equal(k["y"], y) and torch.equal(last2, last) and torch.equal(states2, states)
    for name, v in backward(k, odd(states)).items():
        assert torch.equal(v, want[name]), name


@pytest.mark.parametrize("t", [1, 20, 300])
def test_inputs_that_all_sequences_share(t):
    """Strides of 0: one row of x, B and C for all sequences."""
    k = case(t, 3, 24, 16, F, carry=False, restart=0)
    for name in ("x", "B", "C"):
        k[name] = k[name][:, :1].expand_as(k[name])
    ref = reference(k)
    last, states = forward(k)
    assert_bounded(k["y"], ref.y, ref.by + U * np.abs(ref.y), "y")
    got, want = backward(k, states), ref.backward(f64(k["dy"]), None)
    for name in ("dx", "dB", "dC", "dA", "ddt"):
        assert_bounded(got[name], want[name][0], want[name][1] + U * np.abs(want[name][0]), name)


@pytest.mark.parametrize("t", [3, 20])
def test_steps_far_apart(t):
    """Steps whose places are beyond 32 bits: inputs, outputs and gradients as parts of rows half a gigabyte apart, all with the same strides."""
    n, c, m = 2, 24, 16
    k = case(t, n, c, m, H)
    last, states = forward(k)
    y, want = k["y"].clone(), {name: v.clone() for name, v in backward(k, states).items()}
    step = 1 << 28
    whole, at = torch.empty(t * step, dtype=H, device="cuda"), 0
    for name in ("x", "dt", "z", "y", "dy", "dx", "ddt", "dz", "B", "C", "dB", "dC"):
        v = k[name]
        far = whole.as_strided((t, n, v.shape[2:].numel()), (step, c, 1), at).view(v.shape)
        far.copy_(v)
        k[name] = far
        at += n * c
    last2, states2 = forward(k)
    assert torch.equal(k["y"], y) and torch.equal(last2, last) and torch.equal(states2, states)
    bounds = reference(k).backward(f64(k["dy"]), f64(k["dh_last"]))
    for name, v in backward(k, states).items():
        if name in ("dD", "ddt_bias"):
            assert_bounded(v, bounds[name][0], bounds[name][1] + U * np.abs(bounds[name][0]), name)
        else:
            assert torch.equal(v, want[name]), name
