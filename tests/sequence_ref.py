"""The operators of a policy over sequences from their formulas in 64 bits, with a bound on what float arithmetic may be off by.

u = 2^-24 is half a step of a float relative to its value; a sum or product that is rounded once is off by at most that much.  Storage in type t
rounds once more: eps(t) / 2 of the value.  The library's exponential of a decay, 2^v, is right to 2^-22 = 4 u, its reciprocal to 2 u."""
import numpy as np
import torch

from operators_ref import TINY, U, act, act_slope, assert_within, gate_error, gates

SPAN = 16
LARGEST = float(np.finfo(np.float32).max)


def assert_bounded(got, want, bound, what=""):
    """assert_within where the bound is finite.  It is infinite where what a float has to hold on the way is beyond the largest one: there the result may be
    an infinity or a NaN."""
    bound = np.broadcast_to(bound, want.shape)
    held = np.isfinite(bound)
    assert_within(got[torch.from_numpy(held).to(got.device)], want[held], bound[held], what)


def beyond(value, bound):
    """The bound, infinite where a float does not hold the value, or what it is made of has none."""
    return np.where(np.isfinite(bound) & (np.abs(value) + bound <= LARGEST), bound, np.inf)


def exp_error(dtype, v):
    """Of e^-|v|, relative: as in operators_ref.gate_error."""
    return 2 * U if dtype == torch.float32 else 2 * U * (2 + 1.173 * np.abs(v))


# ---- causal convolution ----------------------------------------------------------------------------------------------------------------

def taps(x, before, restart, width):
    """The inputs of every step, oldest first, [width][t][n][c], and whether each counts; and the same of the steps behind the last."""
    t, n, c = x.shape
    reach = width - 1
    full = np.concatenate([np.zeros((reach, n, c)) if before is None else before.transpose(1, 0, 2), x])
    run = np.concatenate([np.zeros((reach, n), np.int64), np.zeros((t, n), np.int64) if restart is None else np.cumsum(restart != 0, 0)])
    live = np.stack([run[k:k + t] == run[reach:] for k in range(width)])
    seen = np.stack([np.where(live[k][..., None], full[k:k + t], 0.0) for k in range(width)])
    tail = run[t:] == run[-1]
    return seen, live, np.where(tail[..., None], full[t:], 0.0).transpose(1, 0, 2), tail


def conv_forward(x, w, bias, before, restart, kind, dtype):
    """(y, after, bound on y before storage)"""
    width = w.shape[1]
    seen, _, after, _ = taps(x, before, restart, width)
    v = bias + sum(w[:, k] * seen[k] for k in range(width))
    off = (width + 1) * U * (np.abs(bias) + sum(np.abs(w[:, k] * seen[k]) for k in range(width)))
    y = act(v, kind)
    bound = 1.1 * off if kind == "silu" else off          # the slope of v sigmoid(v) is at most 1.1
    if kind == "silu":
        bound = bound + np.abs(y) * (gate_error(dtype, True, np.abs(v)) + 3 * U)
    return y, after, bound + TINY


def conv_backward(x, dy, w, bias, before, dafter, restart, kind, dtype, chain):
    """{name: (value, bound before storage)}; `chain`: roundings that a term of a sum over steps may pass."""
    t, n, c = x.shape
    width = w.shape[1]
    reach = width - 1
    seen, live, _, tail = taps(x, before, restart, width)
    v = bias + sum(w[:, k] * seen[k] for k in range(width))
    off = (width + 1) * U * (np.abs(bias) + sum(np.abs(w[:, k] * seen[k]) for k in range(width)))
    slope = act_slope(v, kind)
    dv = dy * slope
    bdv = np.zeros_like(dv)
    if kind == "silu":
        s, r = gates(v, True)
        # the second derivative is at most 0.5; the slope is a sum of s and v s (1 - s), each with the errors of two gates
        bdv = np.abs(dy) * (0.5 * off + (s + np.abs(v) * s * r) * (2 * gate_error(dtype, True, np.abs(v)) + 4 * U)) + U * np.abs(dv)
    d, bd = np.zeros((reach + t, n, c)), np.zeros((reach + t, n, c))
    m = np.zeros_like(d)
    for k in range(width):
        on = live[k][..., None]
        d[k:k + t] += np.where(on, dv * w[:, k], 0)
        m[k:k + t] += np.where(on, np.abs(dv * w[:, k]), 0)
        bd[k:k + t] += np.where(on, bdv * np.abs(w[:, k]), 0)
    if dafter is not None:
        more = np.where(tail[..., None], dafter.transpose(1, 0, 2), 0)
        d[t:] += more
        m[t:] += np.abs(more)
    bd += (width + 1) * U * m + TINY
    dw = np.stack([(dv * seen[k]).sum((0, 1)) for k in range(width)], 1)
    bw = np.stack([(bdv * np.abs(seen[k]) + chain * U * np.abs(dv * seen[k])).sum((0, 1)) for k in range(width)], 1) + TINY
    return dict(dx=(d[reach:], bd[reach:]), dbefore=(d[:reach].transpose(1, 0, 2), bd[:reach].transpose(1, 0, 2)), dweight=(dw, bw),
                dbias=(dv.sum((0, 1)), (bdv + chain * U * np.abs(dv)).sum((0, 1)) + TINY))


# ---- selective scan --------------------------------------------------------------------------------------------------------------------

def softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def wide(v, c):
    """[...][groups][state] for every channel."""
    return np.repeat(v, c // v.shape[-2], -2)


class Scan:
    """x, dt, z, y [t][n][c]; B, C [t][n][groups][state]; A [c][state]; everything step by step."""

    def __init__(self, x, dt, A, B, C, D, z, bias, h0, restart, softplus_on, dtype):
        t, n, c = x.shape
        self.x, self.A, self.D, self.z, self.dtype = x, A, np.zeros(c) if D is None else D, z, dtype
        self.B, self.C, self.groups = B, C, B.shape[2]
        self.v = dt if bias is None else dt + bias
        self.softplus = softplus_on
        self.delta = softplus(self.v) if softplus_on else self.v
        # the argument's rounding moves the softplus by no more of it than |v| u; then the exponential, a quotient, a series of seven terms, two sums
        self.ddelta = exp_error(dtype, self.v) + (10 + np.abs(self.v)) * U if softplus_on else 2 * U * np.ones_like(self.v)
        self.on = np.ones((t, n), bool) if restart is None else restart == 0
        self.h0 = np.zeros((n, c, A.shape[1])) if h0 is None else h0
        self.forward()

    def keep(self, i):
        """(decay, bound on its relative error): the error of delta A, two roundings of the exponent, the exponential, products of several steps."""
        e = self.delta[i][..., None] * self.A
        error = (self.ddelta[i][..., None] + 4 * U) * np.abs(e) + 8 * U
        return np.exp(e) * self.on[i][:, None, None], np.where(np.exp(e) <= LARGEST / 2, error, np.inf)

    @np.errstate(invalid="ignore", over="ignore")
    def forward(self):
        t, n, c = self.x.shape
        state, off = self.h0, U * np.abs(self.h0)
        self.h, self.off, self.before, self.states = [], [], [], []
        y, by = np.zeros_like(self.x), np.zeros_like(self.x)
        for i in range(t):
            if i % SPAN == 0:
                self.states.append(state)
            self.before.append((state, off))
            k, dk = self.keep(i)
            B, C = wide(self.B[i], c), wide(self.C[i], c)
            take = (self.delta[i] * self.x[i])[..., None] * B
            on = self.on[i][:, None, None]
            kept = np.where(on, k * state, 0)
            off = np.where(on, k * off, 0) * (1 + 1e-6) + np.abs(kept) * (dk + 2 * U) + np.abs(take) * (self.ddelta[i][..., None] + 3 * U) + TINY
            state = kept + take
            off = beyond(state, off + U * np.abs(state))
            self.h.append(state)
            self.off.append(off)
            y[i] = (state * C).sum(-1)
            by[i] = beyond(np.abs(state * C).sum(-1), (off * np.abs(C)).sum(-1) + (self.A.shape[1] + 2) * U * np.abs(state * C).sum(-1))
        self.ch, self.bch = y, by
        y = y + self.D * self.x
        by = by + 2 * U * (np.abs(self.ch) + np.abs(self.D * self.x))
        if self.z is not None:
            s, _ = gates(self.z, True)
            y, by = y * self.z * s, by * np.abs(self.z * s) + np.abs(y * self.z * s) * (gate_error(self.dtype, True, np.abs(self.z)) + 3 * U)
        self.y, self.by = y, beyond(y, by + TINY)
        self.last, self.blast = state, off

    @np.errstate(invalid="ignore", over="ignore")
    def backward(self, dy, dh_last):
        """{name: (value, bound before storage)}"""
        t, n, c = self.x.shape
        m, g = self.A.shape[1], self.groups
        out, chain = {}, t + 16
        bdy = U * np.abs(dy)
        if self.z is not None:
            s, r = gates(self.z, True)
            err = gate_error(self.dtype, True, np.abs(self.z))
            y = self.ch + self.D * self.x
            b = beyond(np.maximum(1, np.abs(dy)) * y, self.bch + 2 * U * (np.abs(self.ch) + np.abs(self.D * self.x)))
            slope, parts = s + self.z * s * r, s + np.abs(self.z) * s * r
            out["dz"] = dy * y * slope, np.abs(dy) * (b * np.abs(slope) + np.abs(y) * parts * (2 * err + 5 * U)) + TINY
            bdy = np.abs(dy * self.z * s) * (err + 4 * U)
            dy = dy * self.z * s
        carry = np.zeros((n, c, m)) if dh_last is None else dh_last
        bcarry = U * np.abs(carry)
        names = dict(dx=(t, n, c), ddt=(t, n, c), dB=(t, n, g, m), dC=(t, n, g, m), dA=(c, m))
        v, b = ({k: np.zeros(shape) for k, shape in names.items()} for _ in range(2))
        for i in range(t - 1, -1, -1):
            k, dk = self.keep(i)
            B, C = wide(self.B[i], c), wide(self.C[i], c)
            d, bd = dy[i][..., None], bdy[i][..., None]
            G = carry + C * d
            bG = beyond(G, bcarry + np.abs(C) * bd + 2 * U * (np.abs(carry) + np.abs(C * d)))
            take, delta = (self.delta[i] * self.x[i])[..., None], self.delta[i][..., None]
            rel = self.ddelta[i][..., None]

            def over(q):
                return q.reshape(n, g, c // g, m).sum(2)

            channels = 24 + c // 32
            v["dC"][i], b["dC"][i] = over(self.h[i] * d), over(self.off[i] * np.abs(d) + np.abs(self.h[i]) * bd + channels * U * np.abs(self.h[i] * d))
            v["dB"][i], b["dB"][i] = over(G * take), over(bG * np.abs(take) + (rel + channels * U) * np.abs(G * take))
            state, off = self.before[i]
            on = self.on[i][:, None, None]
            kept, bkept = np.where(on, k * state, 0), np.where(on, k * off + np.abs(k * state) * (dk + 2 * U), 0)
            through, bthrough = G * kept, bG * np.abs(kept) + np.abs(G) * bkept + 2 * U * np.abs(G * kept)
            bthrough = beyond(through * np.maximum(1, np.abs(self.A)), bthrough)
            v["dA"] += (through * delta).sum(0)
            b["dA"] += (bthrough * np.abs(delta) + (rel + chain * U) * np.abs(through * delta)).sum(0)
            gB, bgB = (G * B).sum(-1), beyond(np.abs(G * B).sum(-1), (bG * np.abs(B) + (m + 2) * U * np.abs(G * B)).sum(-1))
            rate = (through * self.A).sum(-1)
            brate = beyond(np.abs(through * self.A).sum(-1) * 1.5, (bthrough * np.abs(self.A) + (m + 6) * U * np.abs(through * self.A)).sum(-1))
            v["dx"][i] = self.D * dy[i] + self.delta[i] * gB
            b["dx"][i] = np.abs(self.D) * bdy[i] + np.abs(self.delta[i]) * bgB + (self.ddelta[i] + 3 * U) * np.abs(self.delta[i] * gB) + 2 * U * np.abs(self.D * dy[i])
            v["ddt"][i] = rate + self.x[i] * gB
            b["ddt"][i] = brate + np.abs(self.x[i]) * bgB + 2 * U * (np.abs(rate) + np.abs(self.x[i] * gB))
            bcarry = beyond(k * G, np.where(on, k * bG + np.abs(k * G) * (dk + U), 0) + TINY)
            carry = np.where(on, k * G, 0)
        if self.softplus:
            s, _ = gates(self.v, True)
            err = gate_error(self.dtype, True, np.abs(self.v)) + (2 + np.abs(self.v)) * U
            v["ddt"], b["ddt"] = v["ddt"] * s, b["ddt"] * s + np.abs(v["ddt"] * s) * err
        out.update({k: (v[k], b[k] + TINY) for k in v})
        out["dh0"] = carry, bcarry
        out["dD"] = (dy * self.x).sum((0, 1)), (bdy * np.abs(self.x) + chain * U * np.abs(dy * self.x)).sum((0, 1)) + TINY
        out["ddt_bias"] = v["ddt"].sum((0, 1)), (b["ddt"] + chain * U * np.abs(v["ddt"])).sum((0, 1)) + TINY
        return {name: (value, beyond(value, bound)) for name, (value, bound) in out.items()}


# ---- draws --------------------------------------------------------------------------------------------------------------------------------

def draw(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, allowed=None, exact_u=False):
    """(action, log-probability, how near u comes to a border, and top_p to one, with the likeliest action's share as 1) of one row, by sorting.
    `exact_u`: a u in 64 bits, taken as it is."""
    x = logits.astype(np.float64)
    index = np.arange(x.size) if allowed is None else np.nonzero(allowed)[0]
    x = x[index]
    if np.isnan(x).any() or (x == np.inf).any():
        return -1, np.nan, 1.0
    index, x = index[x > -np.inf], x[x > -np.inf]
    if index.size == 0:
        return -1, -np.inf, 1.0
    if np.isnan(temperature):
        return -1, np.nan, 1.0
    order = np.lexsort((index, -x))
    if temperature <= 0:
        return int(index[order[0]]), 0.0, 1.0
    near = 1.0
    if top_k > 0:
        order = order[:top_k]
    with np.errstate(over="ignore"):
        w = np.exp((x[order] - x[order[0]]) / np.float64(temperature))
    if top_p < 1:
        before, aim = np.cumsum(w) - w, max(top_p, 0.0) * w.sum()
        stay = before < aim
        stay[0] = True
        # a border that is met exactly is one of equal weights, whose sums are exact on both sides; before the first there is exactly nothing
        gaps = np.abs(before - aim)[1:]
        near = min(near, gaps[gaps > 0].min(initial=1.0))
        order, w = order[stay], w[stay]
    if min_p > 0:
        stay = w >= min(min_p, 1.0)
        order, w = order[stay], w[stay]
    where = np.argsort(index[order])
    run = np.cumsum(w[where])
    if not exact_u:
        u = np.float64(np.float32(min(max(0.0 if np.isnan(u) else u, 0.0), 1 - 2.0 ** -24)))
    aim = u * run[-1]
    hit = min(int(np.searchsorted(run, aim, side="right")), run.size - 1)
    gaps = np.abs(run - aim)
    near = min(near, gaps[gaps > 0].min(initial=1.0))
    return int(index[order][where][hit]), float(np.log(w[where][hit] / run[-1])), near
