"""What a policy over sequences needs whose network is the caller's own, as cases that can be timed and whose results can be compared.

  conv    a short causal convolution of every channel by itself over the steps of a batch of sequences, cut where an episode restarts, with its
          activation; the last inputs carried on; forward (recordings and single steps) and backward
  scan    a selective state space scan, h_t = exp(delta_t A) h_{t-1} + delta_t B_t x_t, y_t = (C_t h_t + D x_t) silu(z_t), with the steps' own
          delta, B and C; forward (recordings and single steps) and backward from states that the forward pass marked
  sample  an action out of many from logits and a given uniform number: temperature, top-k, top-p and min-p of each row, actions that are
          not allowed, and the action's log-probability

`own` False: the formulas in elementary torch operations, in 32 bits (the draws, where a sum next to a border decides, in 64), rounded once at the end.
`own` True: the library's entry points.
"""
import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SPAN = 16             # steps between the states that the scan's forward pass marks for its backward pass


def listed():
    return [
        # acting: one step of the paper's 32 environments through the convolution and through the scan behind it, states carried on
        dict(name="conv_step_32", op="conv", dir="fwd", t=1, n=32, c=1024, width=4, type="bf16", act="silu", layout="time", restart=200, carry=True),
        dict(name="scan_step_32", op="scan", dir="fwd", t=1, n=32, c=1024, state=16, groups=1, type="bf16", gate=True, layout="time", restart=200, carry=True, marks=False),
        # two recordings taken in at once before acting goes on from their last states, batch first
        dict(name="conv_recordings", op="conv", dir="fwd", t=8192, n=2, c=2048, width=4, type="bf16", act="silu", layout="batch", restart=2000, carry=True),
        dict(name="scan_recordings", op="scan", dir="fwd", t=8192, n=2, c=2048, state=16, groups=1, type="bf16", gate=True, layout="batch", restart=2000, carry=True, marks=False),
        # an update batch of the largest configuration, five steps of 1024 environments
        dict(name="scan_rollout", op="scan", dir="fwd", t=5, n=1024, c=512, state=16, groups=1, type="bf16", gate=True, layout="time", restart=200, carry=True, marks=True),
        # training on eight recordings: forward with the states for the way back, and the way back of both
        dict(name="scan_train", op="scan", dir="fwd", t=2048, n=8, c=1024, state=16, groups=1, type="bf16", gate=True, layout="batch", restart=500, carry=False, marks=True),
        dict(name="scan_train_back", op="scan", dir="bwd", t=2048, n=8, c=1024, state=16, groups=1, type="bf16", gate=True, layout="batch", restart=500, carry=False, marks=True),
        dict(name="conv_train_back", op="conv", dir="bwd", t=2048, n=8, c=1024, width=4, type="bf16", act="silu", layout="batch", restart=500, carry=False),
        # odd sizes in float, two groups of channels, no gate
        dict(name="scan_odd_back", op="scan", dir="bwd", t=1003, n=3, c=200, state=8, groups=2, type="fp32", gate=False, layout="time", restart=100, carry=True, marks=True),
        # acting: 32 environments with 1000 actions, some not allowed
        dict(name="sample_act_32", op="sample", n=32, v=1000, type="fp32", spread=2.0, temperature=True, top_k=False, top_p=False, min_p=False, allowed=0.7),
        # 256 rows over a large vocabulary, every row with settings of its own
        dict(name="sample_256", op="sample", n=256, v=131072, type="bf16", spread=3.0, temperature=True, top_k=True, top_p=True, min_p=True, allowed=1.0),
        # one row of odd length, by its likeliest actions alone
        dict(name="sample_one", op="sample", n=1, v=50001, type="fp32", spread=3.0, temperature=True, top_k=False, top_p=True, min_p=False, allowed=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["conv", "scan", "scan", "sample"])
    kind = rng.choice(["fp32", "bf16"])
    if op == "sample":
        v = _log(rng, 2, 200_000)
        n = max(1, min(_log(rng, 1, 1024), 32_000_000 // v))
        return dict(op=op, n=n, v=v, type=kind, spread=rng.choice([0.5, 3.0, 6.0]), temperature=rng.random() < 0.7, top_k=rng.random() < 0.5,
                    top_p=rng.random() < 0.5, min_p=rng.random() < 0.3, allowed=rng.choice([1.0, 1.0, 0.5, 0.01]))
    c = rng.choice([1, 7, 30, 64, 200, 512, 1024, 2048, _log(rng, 1, 2048)])
    t = rng.choice([1, _log(rng, 1, 8192)])
    how = dict(type=kind, layout=rng.choice(["time", "batch", "packed"]), restart=rng.choice([0, 3, 200]), carry=rng.random() < 0.5)
    if op == "conv":
        n = max(1, min(_log(rng, 1, 1024), 33_000_000 // (t * c)))
        return dict(op=op, dir=rng.choice(["fwd", "bwd"]), t=t, n=n, c=c, width=rng.choice([2, 3, 4, 4]), act=rng.choice(["none", "relu", "silu"]), **how)
    state = rng.choice([1, 5, 8, 16, 16, 16, 24, 64])
    n = max(1, min(_log(rng, 1, 1024), 200_000_000 // (t * c * state)))
    return dict(op=op, dir=rng.choice(["fwd", "bwd"]), t=t, n=n, c=c, state=state, groups=rng.choice([g for g in (1, 1, 2, 4) if c % g == 0]), gate=rng.random() < 0.7,
                marks=rng.random() < 0.5, **how)


# ---- what a program has in hand -------------------------------------------------------------------------------------------------

def _sequences(case, widths, fill=None):
    """Tensors [t][n][width] in the case's layout; packed: side by side in one, as a projection leaves them."""
    t, n, kind = case["t"], case["n"], TYPES[case["type"]]
    if case["layout"] == "packed":
        whole = torch.empty(t, n, sum(widths), dtype=kind, device="cuda")
        views, at = [], 0
        for w in widths:
            views.append(whole[..., at:at + w])
            at += w
    elif case["layout"] == "batch":
        views = [torch.empty(n, t, w, dtype=kind, device="cuda").transpose(0, 1) for w in widths]
    else:
        views = [torch.empty(t, n, w, dtype=kind, device="cuda") for w in widths]
    for v, f in zip(views, fill or []):
        v.copy_(f)
    return views


def _restarts(case, gen):
    if not case["restart"]:
        return None
    return (torch.rand(case["t"], case["n"], device="cuda", generator=gen) < 1.0 / case["restart"]).to(torch.uint8)


def _prepare_conv(case, gen):
    t, n, c, width, kind = case["t"], case["n"], case["c"], case["width"], TYPES[case["type"]]

    def noise(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    s = dict(weight=noise(c, width) / math.sqrt(width), bias=0.1 * noise(c), restart=_restarts(case, gen))
    (s["x"],) = _sequences(case, [c], [noise(t, n, c)])
    s["before"] = noise(n, width - 1, c).to(kind) if case["carry"] else None
    if case["dir"] == "fwd":
        (s["y"],) = _sequences(case, [c])
        s["after"] = torch.empty(n, width - 1, c, dtype=kind, device="cuda") if case["carry"] else None
        return s
    dy = noise(t, n, c)
    if case["act"] == "relu":
        # the derivative has a step at 0: within rounding of it either side is right, so nothing arrives there
        dy.mul_(_conv_argument(s, torch.float64)[0].abs() > 1e-4)
    (s["dy"],) = _sequences(case, [c], [dy])
    s["dafter"] = noise(n, width - 1, c).to(kind) if case["carry"] else None
    (s["dx"],) = _sequences(case, [c])
    s["dbefore"] = torch.empty(n, width - 1, c, dtype=kind, device="cuda") if case["carry"] else None
    s["dweight"], s["dbias"], s["workspace"] = torch.empty(c, width, device="cuda"), torch.empty(c, device="cuda"), None
    if own:
        import paper_1705_04862_b200.binding as pb
        s["workspace"] = torch.empty(pb.causal_conv_workspace_bytes(t, n, c, width, pb.BF16 if case["type"] == "bf16" else pb.FP32), dtype=torch.uint8, device="cuda")
    return s


def _prepare_scan(case, gen):
    t, n, c, m, g = (case[k] for k in ("t", "n", "c", "state", "groups"))

    def noise(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    s = dict(restart=_restarts(case, gen))
    # as such a network begins: rates of 1 to `state`, steps of 0.001 to 0.1, which the input moves
    s["A"] = -torch.arange(1, m + 1, device="cuda", dtype=torch.float32).expand(c, m) * torch.exp(0.1 * noise(c, m))
    step = torch.exp(torch.rand(c, device="cuda", generator=gen) * math.log(100.0) + math.log(1e-3))
    s["dt_bias"], s["D"] = step + torch.log(-torch.expm1(-step)), 1.0 + 0.1 * noise(c)
    widths = [c, c, g * m, g * m] + ([c] if case["gate"] else [])
    fill = [noise(t, n, c), 0.5 * noise(t, n, c), noise(t, n, g * m), noise(t, n, g * m)] + ([noise(t, n, c)] if case["gate"] else [])
    s["x"], s["dt"], s["B"], s["C"], *z = _sequences(case, widths, fill)
    s["z"] = z[0] if z else None
    s["B"], s["C"] = (v.unflatten(2, (g, m)) for v in (s["B"], s["C"]))
    s["h0"] = noise(n, c, m) if case["carry"] else None
    marks = -(-t // SPAN)
    if case["dir"] == "fwd":
        (s["y"],) = _sequences(case if case["layout"] == "batch" else dict(case, layout="time"), [c])
        s["h_last"] = torch.empty(n, c, m, device="cuda")
        s["states"] = torch.empty(marks, n, c, m, device="cuda") if case["marks"] else None
    else:
        start = torch.zeros(n, c, m, device="cuda") if s["h0"] is None else s["h0"]
        s["states"] = torch.cat([start[None], _states(s, _steps(s), start)[SPAN - 1:t - 1:SPAN]]) if t > 1 else start[None].clone()
        (s["dy"],) = _sequences(case if case["layout"] == "batch" else dict(case, layout="time"), [c], [noise(t, n, c)])
        s["dh_last"] = noise(n, c, m) if case["carry"] else None
        s["dx"], s["ddt"], s["dB"], s["dC"], *dz = _sequences(case, widths)
        s["dB"], s["dC"] = (v.unflatten(2, (g, m)) for v in (s["dB"], s["dC"]))
        s["dz"] = dz[0] if dz else None
        s["dA"], s["dD"], s["ddt_bias"] = torch.empty(c, m, device="cuda"), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        s["dh0"] = torch.empty(n, c, m, device="cuda") if case["carry"] else None
    s["workspace"] = None
    if own:
        import paper_1705_04862_b200.binding as pb
        need = pb.selective_scan_workspace_bytes(t, n, c, m, g, pb.BF16 if case["type"] == "bf16" else pb.FP32, backward=case["dir"] == "bwd")
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s


def _prepare_sample(case, gen):
    n, v = case["n"], case["v"]

    def some(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    s = dict(logits=(case["spread"] * torch.randn(n, v, device="cuda", generator=gen)).to(TYPES[case["type"]]), u=some(n))
    # rows with settings of their own: one in eight takes the likeliest, one in four leaves a filter off
    s["temperature"] = torch.where(some(n) < 0.125, torch.zeros(n, device="cuda"), 0.5 + some(n)) if case["temperature"] else None
    s["top_k"] = torch.where(some(n) < 0.25, torch.zeros(n, device="cuda"), torch.exp(some(n) * math.log(200.0))).to(torch.int32) if case["top_k"] else None
    s["top_p"] = torch.where(some(n) < 0.25, torch.ones(n, device="cuda"), 0.5 + 0.49 * some(n)) if case["top_p"] else None
    s["min_p"] = torch.where(some(n) < 0.25, torch.zeros(n, device="cuda"), 0.2 * some(n)) if case["min_p"] else None
    s["allowed"] = (some(n, v) < case["allowed"]).to(torch.uint8) if case["allowed"] < 1.0 else None
    s["action"], s["logprob"] = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return dict({"conv": _prepare_conv, "scan": _prepare_scan, "sample": _prepare_sample}[case["op"]](case, gen), case=case)


# ---- the plain forms: convolution --------------------------------------------------------------------------------------------------

def _conv_window(s, kind):
    """(all inputs from the carried ones on, which run of steps without a restart each belongs to) along the first axis."""
    t, n, c = s["x"].shape
    reach = s["weight"].shape[1] - 1
    before = torch.zeros(n, reach, c, device="cuda", dtype=kind) if s["before"] is None else s["before"].to(kind)
    every = torch.cat([before.transpose(0, 1), s["x"].to(kind)])
    run_of = torch.zeros(reach + t, n, device="cuda", dtype=torch.int32)
    if s["restart"] is not None:
        run_of[reach:] = torch.cumsum((s["restart"] != 0).to(torch.int32), 0)
    return every, run_of


def _conv_argument(s, kind):
    t, width = s["x"].shape[0], s["weight"].shape[1]
    every, run_of = _conv_window(s, kind)
    w = s["weight"].to(kind)
    taps = [torch.where((run_of[k:k + t] == run_of[width - 1:])[..., None], every[k:k + t], 0.0) for k in range(width)]
    return sum((w[:, k] * tap for k, tap in enumerate(taps)), s["bias"].to(kind)), taps, run_of


def _conv_forward(case, s):
    v, _, run_of = _conv_argument(s, torch.float32)
    y = v.clamp(min=0.0) if case["act"] == "relu" else v * torch.sigmoid(v) if case["act"] == "silu" else v
    kind, out = TYPES[case["type"]], {}
    if case["carry"]:
        every, reach = _conv_window(s, torch.float32)[0], case["width"] - 1
        out["after"] = torch.where((run_of[-reach:] == run_of[-1])[..., None], every[-reach:], 0.0).transpose(0, 1).to(kind)
    return {"y": y.to(kind), **out}


def _conv_backward(case, s):
    t, width, kind = case["t"], case["width"], TYPES[case["type"]]
    v, taps, run_of = _conv_argument(s, torch.float32)
    dv = s["dy"].float()
    if case["act"] == "relu":
        dv = dv * (v > 0)
    elif case["act"] == "silu":
        sig = torch.sigmoid(v)
        dv = dv * sig * (1.0 + v * (1.0 - sig))
    d = torch.zeros(width - 1 + t, case["n"], case["c"], device="cuda")
    for k in range(width):
        d[k:k + t] += torch.where((run_of[k:k + t] == run_of[width - 1:])[..., None], dv * s["weight"][:, k], 0.0)
    if case["carry"]:
        d[1 - width:] += torch.where((run_of[1 - width:] == run_of[-1])[..., None], s["dafter"].float().transpose(0, 1), 0.0)
    dweight = torch.stack([(dv * tap).sum(0).sum(0) for tap in taps], 1)
    out = {"dx": d[width - 1:].to(kind), "dweight": dweight, "dbias": dv.sum(0).sum(0)}
    if case["carry"]:
        out["dbefore"] = d[:width - 1].transpose(0, 1).to(kind)
    return out


# ---- the plain forms: selective scan --------------------------------------------------------------------------------------------------

def _recurrence(a, b):
    """h_t = a_t h_{t-1} + b_t over the first axis: spans of two, four, eight, ... steps joined."""
    span = 1
    while span < a.shape[0]:
        b = torch.cat([b[:span], torch.addcmul(b[span:], a[span:], b[:-span])])
        a = torch.cat([a[:span], a[span:] * a[:-span]])
        span *= 2
    return b


def _softplus(v):
    return torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-v.abs()))


def _by_channel(s, v):
    """B or C [t][n][groups][state] for every channel."""
    c, g = s["A"].shape[0], v.shape[2]
    return v.float()[:, :, :, None, :].expand(-1, -1, -1, c // g, -1).reshape(v.shape[0], v.shape[1], c, v.shape[3])


def _steps(s):
    """(delta, what a state keeps, what it takes) of every step."""
    delta = _softplus(s["dt"].float() + s["dt_bias"])
    keep = torch.exp(delta[..., None] * s["A"])
    if s["restart"] is not None:
        keep = torch.where((s["restart"] != 0)[..., None, None], torch.zeros_like(keep), keep)
    return delta, keep, (delta * s["x"].float())[..., None] * _by_channel(s, s["B"])


def _states(s, steps, start):
    _, keep, take = steps
    return _recurrence(keep, torch.cat([(take[0] + keep[0] * start)[None], take[1:]]))


def _scan_forward(case, s):
    n, c, m, kind = case["n"], case["c"], case["state"], TYPES[case["type"]]
    start = torch.zeros(n, c, m, device="cuda") if s["h0"] is None else s["h0"]
    h = _states(s, _steps(s), start)
    y = (h * _by_channel(s, s["C"])).sum(-1) + s["D"] * s["x"].float()
    if case["gate"]:
        z = s["z"].float()
        y = y * z * torch.sigmoid(z)
    out = {"y": y.to(kind), "h_last": h[-1].clone()}
    if case["marks"]:
        out["states"] = torch.cat([start[None], h[SPAN - 1:case["t"] - 1:SPAN]]) if case["t"] > 1 else start[None].clone()
    return out


def _scan_backward(case, s):
    t, n, c, m, g, kind = (*(case[k] for k in ("t", "n", "c", "state", "groups")), TYPES[case["type"]])
    steps = _steps(s)
    delta, keep, _ = steps
    start = s["states"][0]
    h = _states(s, steps, start)
    x, dy, B, C = s["x"].float(), s["dy"].float(), _by_channel(s, s["B"]), _by_channel(s, s["C"])
    out = {}
    if case["gate"]:
        z = s["z"].float()
        sig = torch.sigmoid(z)
        y = (h * C).sum(-1) + s["D"] * x
        out["dz"] = (dy * y * sig * (1.0 + z * (1.0 - sig))).to(kind)
        dy = dy * z * sig
    dh = dy[..., None] * C
    if case["carry"]:
        dh = torch.cat([dh[:-1], (dh[-1] + s["dh_last"])[None]])
    # G_t = dh_t + keep_{t+1} G_{t+1}, from the last step to the first
    grad = _recurrence(torch.cat([torch.zeros_like(keep[:1]), keep[1:].flip(0)]), dh.flip(0)).flip(0)
    kept = grad * keep * torch.cat([start[None], h[:-1]])                # what comes through the exponential, divided by delta A
    ddelta = (kept * s["A"]).sum(-1) + (grad * B).sum(-1) * x
    ddt = ddelta * torch.sigmoid(s["dt"].float() + s["dt_bias"])
    out["dx"] = (s["D"] * dy + delta * (grad * B).sum(-1)).to(kind)
    out["ddt"] = ddt.to(kind)
    out["dB"] = (grad * (delta * x)[..., None]).view(t, n, g, c // g, m).sum(3).to(kind)
    out["dC"] = (h * dy[..., None]).view(t, n, g, c // g, m).sum(3).to(kind)
    out["dA"] = (kept * delta[..., None]).sum(0).sum(0)
    out["dD"], out["ddt_bias"] = (dy * x).sum(0).sum(0), ddt.sum(0).sum(0)
    if case["carry"]:
        out["dh0"] = keep[0] * grad[0]
    return out


# ---- the plain forms: draws ------------------------------------------------------------------------------------------------------------

def _sample(case, s):
    """By sorting.  The likeliest actions (of equal ones the first) up to top_k; of those the first that together have top_p, the one that passes it
    included; of those the ones with min_p of the largest probability; then the first, by index, whose running sum passes u of the whole."""
    n, v = s["logits"].shape
    logits = s["logits"].double()
    if s["allowed"] is not None:
        logits = torch.where(s["allowed"] != 0, logits, -math.inf)
    ordered, order = torch.sort(logits, dim=1, descending=True, stable=True)
    some = ordered[:, :1] > -math.inf
    t = torch.ones(n, 1, device="cuda").double() if s["temperature"] is None else s["temperature"].double()[:, None]
    far = ordered - torch.where(some, ordered[:, :1], 0.0)
    mass = torch.where(t > 0, torch.exp(far / torch.where(t > 0, t, 1.0)), (torch.arange(v, device="cuda") == 0).double())
    mass = torch.where(ordered > -math.inf, mass, 0.0)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        mass = torch.where((k <= 0) | (torch.arange(v, device="cuda") < k), mass, 0.0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        before = torch.cumsum(mass, 1) - mass
        mass = torch.where((p >= 1) | (before < p * mass.sum(1, keepdim=True)) | (torch.arange(v, device="cuda") == 0), mass, 0.0)
    if s["min_p"] is not None:
        mass = torch.where(mass >= s["min_p"].double()[:, None], mass, 0.0)
    by_index = torch.zeros_like(mass).scatter_(1, order, mass)
    running = torch.cumsum(by_index, 1)
    total = running[:, -1:]
    hit = (running > s["u"].double()[:, None] * total) & (by_index > 0)
    action = torch.where(some[:, 0], hit.to(torch.uint8).argmax(1), -1)
    chosen = torch.gather(by_index, 1, action.clamp(min=0)[:, None])
    return {"action": action.to(torch.int32), "logprob": torch.where(some, torch.log(chosen / total), -math.inf)[:, 0].float()}


def _plain(case, s):
    if case["op"] == "sample":
        return _sample(case, s)
    if case["op"] == "conv":
        return (_conv_forward if case["dir"] == "fwd" else _conv_backward)(case, s)
    return (_scan_forward if case["dir"] == "fwd" else _scan_backward)(case, s)


# ---- the library's calls --------------------------------------------------------------------------------------------------------

def _library(case, s):
    import paper_1705_04862_b200.binding as pb
    if case["op"] == "sample":
        status = pb.sample(s["logits"], s["u"], s["action"], logprob=s["logprob"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                           allowed=s["allowed"])
        out = {k: s[k] for k in ("action", "logprob")}
    elif case["op"] == "conv":
        act = {"none": pb.ACT_NONE, "relu": pb.ACT_RELU, "silu": pb.ACT_SILU}[case["act"]]
        if case["dir"] == "fwd":
            status = pb.causal_conv(s["x"], s["weight"], s["bias"], s["y"], before=s["before"], after=s["after"], restart=s["restart"], activation=act)
            out = {k: s[k] for k in ("y", "after")}
        else:
            status = pb.causal_conv_backward(s["x"], s["dy"], s["weight"], s["bias"], s["dx"], s["dweight"], s["dbias"], s["workspace"], before=s["before"],
                                             dafter=s["dafter"], dbefore=s["dbefore"], restart=s["restart"], activation=act)
            out = {k: s[k] for k in ("dx", "dweight", "dbias", "dbefore")}
    else:
        how = dict(D=s["D"], z=s["z"], dt_bias=s["dt_bias"], restart=s["restart"], softplus=True)
        if case["dir"] == "fwd":
            status = pb.selective_scan(s["x"], s["dt"], s["A"], s["B"], s["C"], s["y"], s["workspace"], h0=s["h0"], h_last=s["h_last"], states=s["states"], **how)
            out = {k: s[k] for k in ("y", "h_last", "states")}
        else:
            status = pb.selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], s["dy"], s["states"], s["dx"], s["ddt"], s["dA"], s["dB"], s["dC"],
                                                s["workspace"], dD=s["dD"], dz=s["dz"], ddt_bias=s["ddt_bias"], dh_last=s["dh_last"], dh0=s["dh0"], **how)
            out = {k: s[k] for k in ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias", "dh0")}
    if status != pb.OK:
        raise pb.PaacError(status)
    return {k: v for k, v in out.items() if v is not None}


def run(s):
    return (_library if own else _plain)(s["case"], s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------------

def work(case):
    """Bytes: every input read once, every output written once."""
    e = {"fp32": 4, "bf16": 2}[case["type"]]
    if case["op"] == "sample":
        cells = case["n"] * case["v"]
        settings = sum(case[k] for k in ("temperature", "top_k", "top_p", "min_p"))
        return {"bytes": cells * (e + (case["allowed"] < 1.0)) + 4 * case["n"] * (3 + settings), "flops": 4 * cells}
    cells, flags = case["t"] * case["n"] * case["c"], case["t"] * case["n"] * (1 if case["restart"] else 0)
    back = case["dir"] == "bwd"
    if case["op"] == "conv":
        carried = case["n"] * (case["width"] - 1) * case["c"] * case["carry"] * e
        weights = 4 * case["c"] * (case["width"] + 1)
        each = 2 * case["width"] + (4 if case["act"] == "silu" else 1)
        return {"bytes": cells * e * (3 if back else 2) + flags + carried * (3 if back else 2) + weights * (2 if back else 1), "flops": cells * each * (3 if back else 1)}
    m, rows = case["state"], case["t"] * case["n"] * case["groups"] * case["state"]
    states = 4 * case["n"] * case["c"] * m
    marks = -(-case["t"] // SPAN) * states * case["marks"]
    weights = 4 * case["c"] * (m + 2)
    if not back:
        return {"bytes": cells * e * (3 + case["gate"]) + 2 * rows * e + flags + states * (1 + case["carry"]) + marks + weights, "flops": cells * (7 * m + 12)}
    return {"bytes": cells * e * (5 + 2 * case["gate"]) + 4 * rows * e + flags + 2 * states * case["carry"] + max(marks, states) + 2 * weights, "flops": cells * (18 * m + 30)}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------------

def _exact_conv(case, s):
    """Step by step with the inputs at hand kept in a list, which a restart empties; the gradient by handing each step's share back to them."""
    t, n, c, width = case["t"], case["n"], case["c"], case["width"]
    if t > 10_000:
        return None
    x, w, bias = s["x"].double(), s["weight"].double(), s["bias"].double()
    reach = width - 1
    held = torch.zeros(reach, n, c, device="cuda", dtype=torch.float64) if s["before"] is None else s["before"].double().transpose(0, 1).contiguous()
    on = torch.ones(reach, n, 1, device="cuda", dtype=torch.float64)
    fresh = torch.ones(1, n, 1, device="cuda", dtype=torch.float64)
    back = case["dir"] == "bwd"
    y, place = torch.empty_like(x), []
    if back:
        dy, share = s["dy"].double(), torch.zeros(reach + t, n, c, device="cuda", dtype=torch.float64)
        dw, dbias = torch.zeros_like(w), torch.zeros_like(bias)
    for i in range(t):
        if s["restart"] is not None:
            on = on * (s["restart"][i] == 0).double()[None, :, None]
        window, live = torch.cat([held, x[i:i + 1]]), torch.cat([on, fresh])
        v = bias + (window * live * w.t()[:, None, :]).sum(0)
        sig = 1.0 / (1.0 + torch.exp(-v))
        if back:
            slope = (v > 0).double() if case["act"] == "relu" else sig + v * sig * (1.0 - sig) if case["act"] == "silu" else torch.ones_like(v)
            dv = dy[i] * slope
            share[i:i + width] += live * dv * w.t()[:, None, :]
            dw += (window * live * dv).sum(1).t()
            dbias += dv.sum(0)
        else:
            y[i] = v.clamp(min=0) if case["act"] == "relu" else v * sig if case["act"] == "silu" else v
        held, on = window[1:], live[1:]
    if not back:
        return {"y": y, **({"after": (held * on).transpose(0, 1)} if case["carry"] else {})}
    out = {"dweight": dw, "dbias": dbias}
    if case["carry"]:
        share[t:] += on * s["dafter"].double().transpose(0, 1)
        out["dbefore"] = share[:reach].transpose(0, 1)
    return dict(out, dx=share[reach:])


def _exact_scan(case, s):
    """Step by step, as the recurrence is written; the gradient step by step from the far end."""
    t, n, c, m, g = (case[k] for k in ("t", "n", "c", "state", "groups"))
    if t > 10_000:
        return None
    f64 = dict(device="cuda", dtype=torch.float64)
    x, dt, A, D = s["x"].double(), s["dt"].double() + s["dt_bias"].double(), s["A"].double(), s["D"].double()
    delta = torch.logaddexp(dt, torch.zeros_like(dt))
    z = s["z"].double() if case["gate"] else None
    back = case["dir"] == "bwd"
    state = s["states"][0].double() if back else torch.zeros(n, c, m, **f64) if s["h0"] is None else s["h0"].double()

    def wide(v, i):
        return v[i].double().repeat_interleave(c // g, 1)

    def kept(i):
        k = torch.exp(delta[i][..., None] * A)
        return k if s["restart"] is None else k * (s["restart"][i] == 0).double()[:, None, None]

    before, y, marks = [], torch.empty_like(x), []
    for i in range(t):
        if back:
            before.append(state)
        if i % SPAN == 0:
            marks.append(state)
        state = kept(i) * state + (delta[i] * x[i])[..., None] * wide(s["B"], i)
        y[i] = (state * wide(s["C"], i)).sum(2) + D * x[i]
    if not back:
        out = {"y": y * z / (1.0 + torch.exp(-z)) if case["gate"] else y, "h_last": state}
        return dict(out, states=torch.stack(marks)) if case["marks"] else out
    dy, out = s["dy"].double(), {}
    if case["gate"]:
        sig = 1.0 / (1.0 + torch.exp(-z))
        out["dz"] = dy * y * (sig + z * sig * (1.0 - sig))
        dy = dy * z * sig
    carried = s["dh_last"].double() if case["carry"] else torch.zeros(n, c, m, **f64)
    dx, ddelta, dA = torch.empty_like(x), torch.empty_like(x), torch.zeros_like(A)
    dB, dC = torch.empty(t, n, g, m, **f64), torch.empty(t, n, g, m, **f64)
    for i in range(t - 1, -1, -1):
        k, b = kept(i), wide(s["B"], i)
        grad = carried + dy[i][..., None] * wide(s["C"], i)
        after = before[i + 1] if i + 1 < t else state
        dC[i] = (after * dy[i][..., None]).view(n, g, c // g, m).sum(2)
        dB[i] = (grad * (delta[i] * x[i])[..., None]).view(n, g, c // g, m).sum(2)
        through = grad * k * before[i]
        dA += (through * delta[i][..., None]).sum(0)
        ddelta[i] = (through * A).sum(2) + (grad * b).sum(2) * x[i]
        dx[i] = D * dy[i] + (grad * b).sum(2) * delta[i]
        carried = k * grad
    ddt = ddelta / (1.0 + torch.exp(-dt))
    out.update(dx=dx, ddt=ddt, dA=dA, dB=dB, dC=dC, dD=(dy * x).sum((0, 1)), ddt_bias=ddt.sum((0, 1)))
    return dict(out, dh0=carried) if case["carry"] else out


def _exact_sample(case, s):
    """Row by row: actions fall away from the least likely on."""
    action, logprob = [], []
    for r in range(case["n"]):
        def setting(key, off):
            return off if s[key] is None else s[key][r].item()
        x = s["logits"][r].double()
        live = torch.isfinite(x) if s["allowed"] is None else s["allowed"][r] != 0
        index = live.nonzero()[:, 0]
        if index.numel() == 0:
            action.append(-1)
            logprob.append(-math.inf)
            continue
        x = x[index]
        order = (-x).argsort(stable=True)
        if setting("temperature", 1.0) <= 0:
            order = order[:1]
        else:
            if setting("top_k", 0) > 0:
                order = order[:int(setting("top_k", 0))]
            w = torch.exp((x[order] - x[order[0]]) / setting("temperature", 1.0))
            if setting("top_p", 1.0) < 1:
                far = (w.cumsum(0) - w >= setting("top_p", 1.0) * w.sum()).nonzero()
                order = order[:max(1, int(far[0]))] if far.numel() else order
            order = order[:max(1, int((w[:order.numel()] >= setting("min_p", 0.0)).sum()))]
        w = torch.exp((x[order] - x[order[0]]) / (setting("temperature", 1.0) or 1.0))
        where, back = index[order].sort()
        running = w[back].cumsum(0)
        hit = min(int(torch.searchsorted(running, float(s["u"][r]) * running[-1], right=True)), running.numel() - 1)
        action.append(int(where[hit]))
        logprob.append(float(torch.log(w[back][hit] / running[-1])))
    return {"action": torch.tensor(action, dtype=torch.int32), "logprob": torch.tensor(logprob, dtype=torch.float64)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "sample": _exact_sample}[case["op"]](case, s)
