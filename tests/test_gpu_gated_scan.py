"""The gated linear recurrence and its gradient (paac_gated_scan) against the recurrence step by step in 64 bits."""
import numpy as np
import pytest
import torch

from operators_ref import U, assert_within, f64, gate_error, half_step, scan_backward, scan_forward, scan_forward_bounds
from paper_1705_04862_b200 import binding as pb

pytestmark = pytest.mark.gpu
F, H = torch.float32, torch.bfloat16
KIND = {True: pb.SCAN_SIGMOID, False: pb.SCAN_LINEAR}


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


def case(t, n, c, dtype, sigmoid, layout="time", restart=0.1, carry=True, seed=0):
    rng = np.random.RandomState(seed + 7 * t + n + c)
    gate, x = sequences(t, n, c, dtype, layout, 2)
    logits = np.clip(rng.randn(t, n, c) * 2 + 1, -10, 10)
    gate.copy_(torch.from_numpy(logits if sigmoid else 1.9 / (1 + np.exp(-logits)) - 0.95))
    x.copy_(torch.from_numpy(rng.randn(t, n, c)))
    flags = None
    if restart:
        flags = torch.from_numpy((rng.rand(t, n) < restart).astype(np.uint8) * rng.randint(1, 256, (t, n)).astype(np.uint8)).cuda()
    h0 = torch.from_numpy(rng.randn(n, c)).float().cuda() if carry else None
    return dict(gate=gate, x=x, restart=flags, h0=h0, rng=rng)


def check_forward(k, t, n, c, dtype, sigmoid, layout, reverse):
    (h,) = sequences(t, n, c, dtype, layout, 1)
    last = torch.full((n, c), 9.0, device="cuda")
    assert pb.gated_scan(k["gate"], k["x"], h, h0=k["h0"], h_last=last, restart=k["restart"], kind=KIND[sigmoid], reverse=reverse) == pb.OK
    flags = None if k["restart"] is None else k["restart"].cpu().numpy()
    want, want_last, M, D = scan_forward(f64(k["gate"]), f64(k["x"]), f64(k["h0"]), flags, sigmoid, reverse)
    delta = gate_error(dtype, sigmoid, 10)
    off = scan_forward_bounds(M, D, dtype, delta)
    assert_within(h, want, off + half_step(dtype) * (np.abs(want) + off), "h")
    assert_within(last, want_last, off[0 if reverse else t - 1], "h_last")
    return h


def check_backward(k, h, t, n, c, dtype, sigmoid, layout, reverse):
    rng = k["rng"]
    (dh,) = sequences(t, n, c, dtype, layout, 1)
    dh.copy_(torch.from_numpy(rng.randn(t, n, c)))
    dgate, dx = sequences(t, n, c, dtype, layout, 2)
    dh_last = torch.from_numpy(rng.randn(n, c)).float().cuda() if k["h0"] is not None else None
    dh0 = torch.full((n, c), 9.0, device="cuda")
    assert pb.gated_scan_backward(k["gate"], k["x"] if sigmoid else None, h, dh, dgate, dx, h0=k["h0"], dh_last=dh_last, dh0=dh0, restart=k["restart"],
                                  kind=KIND[sigmoid], reverse=reverse) == pb.OK
    flags = None if k["restart"] is None else k["restart"].cpu().numpy()
    wg, wx, w0, bg, bx, b0 = scan_backward(f64(k["gate"]), f64(k["x"]), f64(h), f64(dh), f64(k["h0"]), f64(dh_last), flags, sigmoid, reverse,
                                           gate_error(dtype, sigmoid, 10))
    half = half_step(dtype)
    assert_within(dgate, wg, bg + half * (np.abs(wg) + bg), "dgate")
    assert_within(dx, wx, bx + half * (np.abs(wx) + bx), "dx")
    assert_within(dh0, w0, b0, "dh0")
    return dh, dh_last, dgate, dx, dh0


SHAPES = [(1, 1, 1), (1, 32, 256), (2, 3, 8), (3, 5, 7), (5, 40, 64), (17, 2, 24), (33, 1, 1), (64, 9, 30), (129, 2, 40), (300, 3, 5), (700, 1, 72),
          (1025, 2, 8), (2500, 1, 16), (4099, 1, 3), (9001, 1, 8)]


@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c", SHAPES)
def test_lengths_and_widths(t, n, c, dtype, sigmoid):
    for reverse, carry, restart in ((False, True, 0.1), (True, False, 0.0), (True, True, 0.02)):
        k = case(t, n, c, dtype, sigmoid, restart=restart, carry=carry)
        h = check_forward(k, t, n, c, dtype, sigmoid, "time", reverse)
        check_backward(k, h, t, n, c, dtype, sigmoid, "time", reverse)


@pytest.mark.parametrize("layout", ["batch", "packed", "odd"])
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c", [(1, 4, 16), (6, 33, 16), (200, 5, 24), (531, 3, 9), (700, 4, 30), (40, 3, 20), (3000, 2, 64)])
def test_layouts(t, n, c, dtype, layout):
    for sigmoid, reverse in ((True, False), (False, True)):
        k = case(t, n, c, dtype, sigmoid, layout)
        h = check_forward(k, t, n, c, dtype, sigmoid, layout, reverse)
        check_backward(k, h, t, n, c, dtype, sigmoid, layout, reverse)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c", [(5, 1024, 64), (20, 700, 128), (700, 300, 24), (300, 250, 30), (9, 2000, 20), (2100, 40, 40)])
def test_many_columns(t, n, c, dtype):
    k = case(t, n, c, dtype, True, "packed")
    h = check_forward(k, t, n, c, dtype, True, "packed", False)
    check_backward(k, h, t, n, c, dtype, True, "packed", False)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c", [(4, 3, 8), (500, 2, 16), (3000, 1, 33)])
def test_what_a_restart_cuts_off_may_be_anything(t, n, c, dtype):
    """Infinities and NaNs before a restart, in h0 under one, and in the gate of a linear step that restarts, reach nothing behind it;
    rows that restart at every step have no memory."""
    for sigmoid in (True, False):
        k = case(t, n, c, dtype, sigmoid, restart=0.2)
        k["restart"][0], k["restart"][t // 2], k["restart"][:, 0] = 1, 1, 1
        k["h0"][:] = float("nan")
        k["x"][t // 2 - 1] = float("inf")
        k["x"][t // 2 - 1, :, 0] = float("nan")
        if not sigmoid:
            k["gate"][t // 2] = float("nan")
            k["gate"][:, 0] = float("-inf")
        (h,) = sequences(t, n, c, dtype, "time", 1)
        last = torch.empty(n, c, device="cuda")
        assert pb.gated_scan(k["gate"], k["x"], h, h0=k["h0"], h_last=last, restart=k["restart"], kind=KIND[sigmoid]) == pb.OK
        keep = [i for i in range(t) if i != t // 2 - 1]
        assert bool(torch.isfinite(h[keep].float()).all()) and bool(torch.isfinite(last).all()) and not bool(torch.isfinite(h[t // 2 - 1].float()).any())
        clean = dict(k, x=k["x"].clone().nan_to_num_(0, 0, 0), gate=k["gate"].clone().nan_to_num_(0.5, 0.5, 0.5), h0=torch.zeros_like(k["h0"]))
        want = torch.empty_like(h)
        assert pb.gated_scan(clean["gate"], clean["x"], want, h0=clean["h0"], restart=k["restart"], kind=KIND[sigmoid]) == pb.OK
        assert torch.equal(h[t // 2:], want[t // 2:]) and torch.equal(h[:t // 2 - 1], want[:t // 2 - 1])
        (dh,) = sequences(t, n, c, dtype, "time", 1)
        dh.normal_()
        dh[t // 2] = float("nan")                                # flows into no earlier step
        dgate, dx = sequences(t, n, c, dtype, "time", 2)
        dh0 = torch.empty(n, c, device="cuda")
        assert pb.gated_scan_backward(clean["gate"], clean["x"], want, dh, dgate, dx, h0=k["h0"], dh0=dh0, restart=k["restart"], kind=KIND[sigmoid]) == pb.OK
        for out in (dgate, dx):
            assert bool(torch.isfinite(out[:t // 2].float()).all()) and bool(torch.isfinite(out[t // 2 + 1:].float()).all())
        assert bool((dh0 == 0).all())
        if not sigmoid:
            assert bool((dgate[k["restart"] != 0] == 0).all())


def test_gates_at_their_ends():
    """Gates of +-infinity, the largest float and 0: a sigmoid of 1 keeps, one of 0 takes; products of gates that vanish leave what is
    behind them alone."""
    for dtype in (F, H):
        big = torch.finfo(dtype).max
        gate = torch.tensor([float("inf"), big, -float("inf"), -big, 60.0, -60.0, 0.0, 1e-30] * 64, device="cuda").to(dtype).view(-1, 1, 1)
        x = torch.arange(1, gate.numel() + 1, device="cuda").to(dtype).view(-1, 1, 1)
        h = torch.empty_like(x)
        assert pb.gated_scan(gate, x, h, h0=torch.full((1, 1), 3.0, device="cuda")) == pb.OK
        want, _, M, D = scan_forward(f64(gate), f64(x), np.full((1, 1), 3.0), None, True, False)
        off = scan_forward_bounds(M, D, dtype, gate_error(dtype, True, 60))
        assert_within(h, want, off + half_step(dtype) * (np.abs(want) + off), "h")


@pytest.mark.parametrize("t,n", [(5, 32), (64, 7), (2000, 3)])
def test_n_step_returns(t, n):
    """Algorithm 1's returns, bootstrapped and cut at terminals, in reverse; of the learner's own lengths and longer."""
    rng = np.random.RandomState(t)
    r = torch.from_numpy(rng.randint(-1, 2, (t, n)).astype(np.float32)).cuda()
    done = torch.from_numpy((rng.rand(t, n) < 0.05).astype(np.uint8)).cuda()
    v = torch.from_numpy(rng.randn(n).astype(np.float32)).cuda()
    gamma = torch.full((t, n), 0.99, device="cuda")
    out = torch.empty(t, n, device="cuda")
    as_steps = [x.view(t, n, 1) for x in (gamma, r, out)]
    assert pb.gated_scan(*as_steps, h0=v.view(n, 1), restart=done, kind=pb.SCAN_LINEAR, reverse=True) == pb.OK
    want, state = np.zeros((t, n)), f64(v)
    for i in range(t - 1, -1, -1):
        state = f64(r)[i] + float(np.float32(0.99)) * (1 - done.cpu().numpy()[i]) * state
        want[i] = state
    assert np.abs(f64(out) - want).max() <= 2 * U * 100 * 100       # two roundings a step, 1 / (1 - gamma) steps of at most that size


def test_the_learners_own_returns():
    """What paac_update computes for its rollout, from the rollout's rewards, terminals and bootstrap values: the same numbers to float rounding."""
    n, t = 32, 5
    g = pb.Paac("nips", n, t, 4, seed=3, term_denom=7)
    g.rollout()
    assert g.update()["status"] == 0
    rewards = torch.from_numpy(g.debug_read(pb.DBG_REWARDS).astype(np.float32)).cuda().view(t, n, 1)
    done = torch.from_numpy(g.debug_read(pb.DBG_TERMINALS).copy()).cuda().view(t, n)
    values = torch.from_numpy(g.debug_read(pb.DBG_VALUES).copy()).cuda().view(t + 1, n)
    assert 0 < int(done.sum()) < t * n
    out = torch.empty(t, n, 1, device="cuda")
    assert pb.gated_scan(torch.full_like(out, 0.99), rewards, out, h0=values[t].view(n, 1).contiguous(), restart=done, kind=pb.SCAN_LINEAR, reverse=True) == pb.OK
    want = g.debug_read(pb.DBG_RETURNS)
    assert np.abs(out.cpu().numpy().reshape(-1) - want).max() <= 2 * 2 * U * 2 * t * max(1.0, float(np.abs(want).max()))
    g.close()


def test_the_state_carried_on_step_by_step_is_the_whole_pass():
    t, n, c = 40, 6, 32
    k = case(t, n, c, F, True)
    whole = check_forward(k, t, n, c, F, True, "time", False)
    state, steps = k["h0"].clone(), torch.empty(t, n, c, device="cuda")
    for i in range(t):
        assert pb.gated_scan(k["gate"][i:i + 1], k["x"][i:i + 1], steps[i:i + 1], h0=state, h_last=state, restart=k["restart"][i:i + 1]) == pb.OK
    assert torch.equal(state, steps[-1])
    want, _, M, D = scan_forward(f64(k["gate"]), f64(k["x"]), f64(k["h0"]), k["restart"].cpu().numpy(), True, False)
    bound = scan_forward_bounds(M, D, F, gate_error(F, True, 10))
    assert_within(steps, want, bound)
    assert_within(whole, f64(steps), 2 * bound)


@pytest.mark.parametrize("t,n,c", [(7, 4, 16), (900, 2, 16)])
def test_gradients_that_are_not_wanted(t, n, c):
    k = case(t, n, c, F, True)
    h = check_forward(k, t, n, c, F, True, "time", False)
    dh, dh_last, dgate, dx, dh0 = check_backward(k, h, t, n, c, F, True, "time", False)
    for want in ((1, 0, 0), (0, 1, 0), (0, 0, 1)):
        out = [torch.zeros_like(v) if w else None for v, w in zip((dgate, dx, dh0), want)]
        assert pb.gated_scan_backward(k["gate"], k["x"], h, dh, out[0], out[1], h0=k["h0"], dh_last=dh_last, dh0=out[2], restart=k["restart"]) == pb.OK
        for o, v in zip(out, (dgate, dx, dh0)):
            assert o is None or torch.equal(o, v)
    assert pb.gated_scan_backward(k["gate"], k["x"], h, dh, dgate, dx, h0=k["h0"], dh_last=dh_last, dh0=dh_last, restart=k["restart"]) == pb.OK
    assert torch.equal(dh_last, dh0)


@pytest.mark.parametrize("t,n,c", [(6, 50, 24), (1500, 2, 40)])
def test_recorded_replayed_and_the_same_bits_every_time(t, n, c):
    k = case(t, n, c, H, True)
    h, last, dx, dgate = *sequences(t, n, c, H, "time", 1), torch.empty(n, c, device="cuda"), *sequences(t, n, c, H, "time", 2)
    dh = torch.randn(t, n, c, device="cuda").to(H)

    def both():
        assert pb.gated_scan(k["gate"], k["x"], h, h0=k["h0"], h_last=last, restart=k["restart"]) == pb.OK
        assert pb.gated_scan_backward(k["gate"], k["x"], h, dh, dgate, dx, h0=k["h0"], restart=k["restart"]) == pb.OK

    both()
    want = [v.clone() for v in (h, last, dgate, dx)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        for v in (h, last, dgate, dx):
            v.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(v, w) for v, w in zip((h, last, dgate, dx), want))


def test_rows_beyond_32_bits():
    """Two steps of a long buffer whose rows lie more than 2^31 elements apart."""
    far = 2 ** 31 + 64
    buf = torch.zeros(far + 64, dtype=H, device="cuda")
    gate, x = buf.as_strided((2, 1, 16), (far, 16, 1)), buf.as_strided((2, 1, 16), (far, 16, 1), 32)
    gate.copy_(torch.randn(2, 1, 16))
    x.copy_(torch.randn(2, 1, 16))
    h = torch.empty(2, 1, 16, dtype=H, device="cuda")
    assert pb.gated_scan(gate, x, h) == pb.OK
    want, _, M, D = scan_forward(f64(gate), f64(x), None, None, True, False)
    off = scan_forward_bounds(M, D, H, gate_error(H, True, 10))
    assert_within(h, want, off + half_step(H) * (np.abs(want) + off))


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c", [(3, 5, 64), (1, 9, 40)])
def test_states_that_begin_anywhere(t, n, c, dtype):
    """States aligned to their elements only, beside rows that allow the widest accesses: the same bits, a column's steps being the same."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    gate, x, dh = (torch.randn(t, n, c, device="cuda", generator=gen).to(dtype) for _ in range(3))
    h0, last = torch.randn(n, c, device="cuda", generator=gen), torch.randn(n, c, device="cuda", generator=gen)

    def moved(s):
        room = torch.zeros(n * c + 8, device="cuda")
        v = room[1:1 + n * c].view(n, c)
        v.copy_(s)
        return room, v

    outs = []
    for move in (False, True):
        rooms = [moved(s) if move else (None, s.clone()) for s in (h0, torch.zeros_like(h0), last, torch.zeros_like(h0))]
        (_, a), (room, h_last), (_, b), (room2, dh0) = rooms
        h, dgate, dx = torch.empty_like(gate), torch.empty_like(gate), torch.empty_like(gate)
        assert pb.gated_scan(gate, x, h, h0=a, h_last=h_last) == pb.OK
        assert pb.gated_scan_backward(gate, x, h, dh, dgate, dx, h0=a, dh_last=b, dh0=dh0) == pb.OK
        outs.append([h, dgate, dx, h_last.clone(), dh0.clone()])
        for r in (room, room2):
            assert r is None or (r[0] == 0 and bool((r[1 + n * c:] == 0).all()))
    for one, other in zip(*outs):
        assert torch.equal(one, other)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c", [(40, 2, 5), (4099, 1, 3), (9001, 1, 8), (3000, 2, 64)])
def test_what_no_restart_cuts_off_stays(t, n, c, dtype, sigmoid, bad):
    """A NaN or an infinity in an early step, in the state before the first or (backward) in a late gradient, with gates of either sign, whose
    products vanish long before the end, and no restart: nothing behind it is finite (a NaN stays one), the other channels are as without it."""
    rng = np.random.RandomState(t + c)
    gate = torch.from_numpy(rng.randn(t, n, c) * 2 + 1 if sigmoid else rng.uniform(-0.95, 0.95, (t, n, c))).to(dtype).cuda()
    x, dh = (torch.from_numpy(rng.randn(t, n, c)).to(dtype).cuda() for _ in range(2))
    h0, dh_last = (torch.from_numpy(rng.randn(n, c)).float().cuda() for _ in range(2))

    def lost(v):
        v = v[..., ::2].float()
        return not bool((torch.isnan(v) if bad != bad else ~torch.isfinite(v)).all())

    def forward(x, h0, reverse):
        h, last = torch.empty_like(x), torch.empty_like(h0)
        assert pb.gated_scan(gate, x, h, h0=h0, h_last=last, kind=KIND[sigmoid], reverse=reverse) == pb.OK
        return (h.flip(0) if reverse else h), last

    def backward(h, dh, dh_last, reverse):
        dgate, dx, dh0 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0)
        assert pb.gated_scan_backward(gate, x if sigmoid else None, h, dh, dgate, dx, h0=h0, dh_last=dh_last, dh0=dh0, kind=KIND[sigmoid], reverse=reverse) == pb.OK
        return [v.flip(0) if reverse else v for v in (dgate, dx)] + [dh0]

    for reverse in (False, True):
        clean, clean_last = forward(x, h0, reverse)
        step = t - 1 - 5 if reverse else 5
        x_bad, h0_bad = x.clone(), h0.clone()
        x_bad[step, :, ::2] = bad
        h0_bad[:, ::2] = bad
        for begin, (h, last) in ((5, forward(x_bad, h0, reverse)), (0, forward(x, h0_bad, reverse))):
            assert not lost(h[begin:]) and not lost(last)
            assert torch.equal(h[:begin], clean[:begin]) and torch.equal(h[..., 1::2], clean[..., 1::2]) and torch.equal(last[:, 1::2], clean_last[:, 1::2])
        stored = clean.flip(0) if reverse else clean
        *clean_back, clean_dh0 = backward(stored, dh, dh_last, reverse)
        dh_bad, dh_last_bad = dh.clone(), dh_last.clone()
        dh_bad[t - 1 - step, :, ::2] = bad
        dh_last_bad[:, ::2] = bad
        for end, out in ((t - 5, backward(stored, dh_bad, dh_last, reverse)), (t, backward(stored, dh, dh_last_bad, reverse))):
            assert not lost(out[2]) and torch.equal(out[2][:, 1::2], clean_dh0[:, 1::2])
            for v, w in zip(out, clean_back):
                assert not lost(v[:end]) and torch.equal(v[end:], w[end:]) and torch.equal(v[..., 1::2], w[..., 1::2])


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c", [(7, 5, 24), (900, 3, 16)])
def test_halves_of_sequences_with_a_gap_behind_them(t, n, c, dtype):
    """The two halves of every step, sequences first, a sequence taking a little more than its steps: the same bits as in tensors of their own."""
    gen = torch.Generator(device="cuda").manual_seed(t)

    def halves():
        room = torch.zeros(n, t * 2 * c + 8, dtype=dtype, device="cuda")
        both = room[:, :t * 2 * c].view(n, t, 2 * c).transpose(0, 1)
        return room, both[..., :c], both[..., c:]

    (_, gate, x), (room, dgate, dx) = halves(), halves()
    gate.copy_(torch.randn(t, n, c, device="cuda", generator=gen))
    x.copy_(torch.randn(t, n, c, device="cuda", generator=gen))
    dh = torch.randn(t, n, c, device="cuda", generator=gen).to(dtype)
    h = torch.empty_like(dh)
    assert pb.gated_scan(gate, x, h) == pb.OK
    assert pb.gated_scan_backward(gate, x, h, dh, dgate, dx) == pb.OK
    own = [torch.empty_like(dh) for _ in range(2)]
    assert pb.gated_scan_backward(gate.contiguous(), x.contiguous(), h, dh, *own) == pb.OK
    assert torch.equal(dgate, own[0]) and torch.equal(dx, own[1]) and bool((room[:, t * 2 * c:] == 0).all())
    assert pb.gated_scan(gate, x, dgate) == pb.OK and torch.equal(dgate, h) and torch.equal(dx, own[1])


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("layout,reverse", [("batch", True), ("packed", False)])
def test_long_linear_sequences_of_many_columns(dtype, layout, reverse):
    """Plain coefficients where steps under way are kept in shared memory and (float) a pass takes more than one round."""
    t, n, c = 1500, 200, 24
    k = case(t, n, c, dtype, False, layout, restart=0.002)
    h = check_forward(k, t, n, c, dtype, False, layout, reverse)
    check_backward(k, h, t, n, c, dtype, False, layout, reverse)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("t,n,c", [(6, 33, 16), (700, 3, 24)])
def test_every_array_with_a_layout_of_its_own(t, n, c, dtype, sigmoid):
    """Parts of wider rows beside contiguous ones, steps first beside sequences first, inputs and restarts that are the same for every sequence or
    step (a stride of 0): the same bits as from contiguous copies, the accesses' width being the same."""
    gen = torch.Generator(device="cuda").manual_seed(t + c)

    def noise(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(dtype)

    def wide():
        return sequences(t, n, c, dtype, "packed", 3)[1]

    def batch():
        return sequences(t, n, c, dtype, "batch", 1)[0]

    def filled(v):
        return v.copy_(noise(t, n, c))

    h0, flags = torch.randn(n, c, device="cuda", generator=gen), (torch.rand(t, n, device="cuda", generator=gen) < 0.1).to(torch.uint8)
    sets = [(filled(wide()), filled(batch()), torch.empty(t, n, c, dtype=dtype, device="cuda"), filled(wide()), batch(), wide(), flags),
            (noise(c).expand(t, n, c), filled(wide()), batch(), noise(t, 1, c).expand(t, n, c), wide(), batch(), flags[:, :1].expand(t, n)),
            (noise(n, c).expand(t, n, c), noise(t, 1, c).expand(t, n, c), wide(), noise(c).expand(t, n, c), batch(), wide(), flags[:1].expand(t, n))]
    if not sigmoid:
        sets = [(torch.tanh(g.float()).to(dtype) if i == 0 else torch.tanh(g[:1, :1].float()).to(dtype).expand(t, n, c), *rest) for i, (g, *rest) in enumerate(sets)]
    for gate, x, h, dh, dgate, dx, restart in sets:
        outs = []
        for turn in range(2):
            if turn:
                gate, x, dh, restart = (v.contiguous() for v in (gate, x, dh, restart))
                h, dgate, dx = (torch.empty(t, n, c, dtype=dtype, device="cuda") for _ in range(3))
            last, dh0 = torch.empty_like(h0), torch.empty_like(h0)
            assert pb.gated_scan(gate, x, h, h0=h0, h_last=last, restart=restart, kind=KIND[sigmoid]) == pb.OK
            assert pb.gated_scan_backward(gate, x, h, dh, dgate, dx, h0=h0, dh0=dh0, restart=restart, kind=KIND[sigmoid]) == pb.OK
            outs.append((h, last, dgate, dx, dh0))
        for one, other in zip(*outs):
            assert bool(torch.isfinite(one.float()).all()) and torch.equal(one, other)
