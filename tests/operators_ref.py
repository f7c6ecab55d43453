"""The operators for a caller's own network, from their formulas in 64 bits, with a bound on what float arithmetic may be off by.

u = 2^-24 is half a step of a float relative to its value; a sum or product that is rounded once is off by at most that much.
Storage in type t rounds once more: eps(t) / 2 of the value.
"""
import numpy as np
import torch

U = 2.0 ** -24
TINY = 2.0 ** -126          # below it the steps of a float are those of the subnormal numbers


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def assert_within(got, want, bound, what=""):
    """Every element of the tensor `got` within `bound` of `want`, which may hold infinities and NaNs of its own."""
    got = f64(got)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    off = np.abs(got[fine] - want[fine]) - np.broadcast_to(bound, want.shape)[fine]
    assert off.size == 0 or off.max() <= 0, (what, float(off.max()), int((off > 0).sum()), off.size)


# ---- gated scan --------------------------------------------------------------------------------------------------------------------

def gates(gate, sigmoid):
    """(coefficient, factor of x) in 64 bits, neither as a difference from 1."""
    if not sigmoid:
        return gate, np.ones_like(gate)
    e = np.exp(-np.abs(gate))
    big, small = 1 / (1 + e), e / (1 + e)
    return np.where(gate >= 0, big, small), np.where(gate >= 0, small, big)


def gate_error(dtype, sigmoid, largest):
    """Relative error of a gate.  e^-|g| is off by one step (two units u) in float and by 2 + 1.173 |g| steps with the faster
    exponential that bf16 storage takes; then come 1 + e (u), the quotient (two steps) and the product with e (u), which has e's
    error a second time."""
    if not sigmoid:
        return 0.0
    e = 2 * U if dtype == torch.float32 else 2 * U * (2 + 1.173 * largest)
    return 2 * e + (1 + 4 + 1) * U


def scan_forward(gate, x, h0, restart, sigmoid, reverse):
    """(h, h_last, M, D) by the recurrence.  M: the same with absolute values; D: with each term weighted by the number of steps
    it has come, so that delta * D bounds what a relative error delta at every step gives."""
    a, take = gates(gate, sigmoid)
    with np.errstate(invalid="ignore"):
        b = take * x
    T = a.shape[0]
    h, M, D = (np.zeros_like(b) for _ in range(3))
    state = np.zeros_like(b[0]) if h0 is None else h0
    m, d = np.abs(state), np.zeros_like(state)
    for t in (range(T - 1, -1, -1) if reverse else range(T)):
        on = np.ones_like(state, bool) if restart is None else np.broadcast_to((restart[t] == 0)[:, None], state.shape)
        with np.errstate(invalid="ignore", over="ignore"):
            state = np.where(on, a[t] * state, 0) + b[t]
            m = np.where(on, np.abs(a[t]) * m, 0) + np.abs(b[t])
            d = np.where(on, np.abs(a[t]) * d, 0) + m
        h[t], M[t], D[t] = state, m, d
    return h, state, M, D


def scan_forward_bounds(M, D, dtype, delta):
    """Of h before it is stored: a term that has come k steps has met k gates and at most 2 k + 8 roundings (products of gates,
    sums), however the steps were grouped."""
    return (delta + 2 * U) * D + (delta + 8 * U) * M + TINY


def scan_backward(gate, x, h, dh, h0, dh_last, restart, sigmoid, reverse, delta):
    """(dgate, dx, dh0) and their bounds before storage, from the formulas."""
    a, take = gates(gate, sigmoid)
    T = a.shape[0]
    order = list(range(T - 1, -1, -1)) if reverse else list(range(T))
    carry = np.zeros_like(a[0]) if dh_last is None else dh_last
    m, d = np.abs(carry), np.zeros_like(carry)
    start = np.zeros_like(a[0]) if h0 is None else h0
    dgate, dx, bg, bx = (np.zeros_like(a) for _ in range(4))
    last = np.zeros_like(carry)
    for i in range(T - 1, -1, -1):
        t = order[i]
        on = np.ones_like(carry, bool) if restart is None else np.broadcast_to((restart[t] == 0)[:, None], carry.shape)
        g = dh[t] + carry
        m = np.abs(dh[t]) + m
        d = d + m
        off = (delta + 2 * U) * d + (delta + 8 * U) * m + TINY
        prev = np.where(on, h[order[i - 1]] if i else start, 0)
        if sigmoid:
            slope = (prev - x[t]) * a[t] * take[t]
            dgate[t], bg[t] = g * slope, off * np.abs(slope) + (2 * delta + 5 * U) * np.abs(g * slope) + TINY
        else:
            dgate[t], bg[t] = np.where(on, g * prev, 0), np.where(on, off * np.abs(prev) + U * np.abs(g * prev), 0) + TINY
        dx[t], bx[t] = g * take[t], off * take[t] + (delta + U) * np.abs(g * take[t]) + TINY
        carry = np.where(on, a[t] * g, 0)
        last = np.where(on, np.abs(a[t]) * off + (delta + U) * np.abs(carry), 0) + TINY
        m, d = np.where(on, np.abs(a[t]) * m, 0), np.where(on, np.abs(a[t]) * d, 0)
    return dgate, dx, carry, bg, bx, last


# ---- group normalisation --------------------------------------------------------------------------------------------------------------

def act(v, kind):
    if kind == "relu":
        return np.maximum(v, 0)
    if kind == "silu":
        return v * gates(v, True)[0]
    return v


def act_slope(v, kind):
    if kind == "relu":
        return (v > 0).astype(np.float64)
    if kind == "silu":
        s, r = gates(v, True)
        return s * (1 + v * r)
    return np.ones_like(v)


def norm_stats(x, groups, eps):
    """mean and 1 / deviation [n][groups] of x [n][pixels][c]."""
    n, p, c = x.shape
    g = x.reshape(n, p, groups, c // groups)
    mean = g.mean((1, 3))
    var = ((g - mean[:, None, :, None]) ** 2).mean((1, 3))
    return mean, 1 / np.sqrt(var + eps)


def spread(v, c):
    """[n][groups] as [n][1][c]."""
    return np.repeat(v, c // v.shape[1], 1)[:, None, :]


def norm_forward(x, gamma, beta, groups, kind, eps):
    c = x.shape[2]
    mean, rstd = norm_stats(x, groups, eps)
    v = (x - spread(mean, c)) * spread(rstd, c) * gamma + beta
    return act(v, kind), mean, rstd, v


def norm_backward(x, dy, gamma, beta, mean, rstd, kind):
    n, p, c = x.shape
    groups = mean.shape[1]
    m = p * (c // groups)
    xhat = (x - spread(mean, c)) * spread(rstd, c)
    v = xhat * gamma + beta
    dv = dy * act_slope(v, kind)

    def over_group(q):
        return q.reshape(n, p, groups, c // groups).sum((1, 3)) / m

    s1, s2 = over_group(dv * gamma), over_group(dv * gamma * xhat)
    dx = spread(rstd, c) * (dv * gamma - spread(s1, c) - xhat * spread(s2, c))
    return dx, (dv * xhat).sum((0, 1)), dv.sum((0, 1)), dict(xhat=xhat, v=v, dv=dv, over_group=over_group)
