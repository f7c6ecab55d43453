"""Three operators for learners whose network is the caller's own, as cases that can be timed and whose results can be compared.

  clip   the global L2 norm over many gradient tensors, and their clipping, each into a tensor of its own or in place
  scan   a gated linear recurrence over the steps of a batch of sequences, cut where an episode restarts: h_t = a_t h_{t-1} + x_t, or
         h_t = z_t h_{t-1} + (1 - z_t) x_t with z_t = sigmoid(gate_t); forward, and backward from the stored h
  norm   group normalisation with its scale, shift and activation, channels last; forward, and backward from the stored mean and 1/deviation

`own` False: the formulas in elementary torch operations, in 32 bits, rounded once at the end.  `own` True: the library's entry points.
"""
import math
import random

import torch

own = False

GAMMA = 0.99          # discount of the repository's configurations
CLIP = 40.0           # their clipping threshold
EPS = 1e-5
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
#: elements of the larger network's tensors, weights then biases, layer by layer (18 actions)
NATURE = [32 * 256, 32, 64 * 512, 64, 64 * 576, 64, 512 * 3136, 512, 18 * 512, 18, 512, 1]


def listed():
    return [
        # the larger network's twelve gradient tensors in bf16, clipped into the flat float vector that the optimiser step takes
        dict(name="clip_nature_to_flat", op="clip", sizes="nature", count=12, total=sum(NATURE), src="bf16", dst="fp32", inplace=False, pad=False, ratio=0.45),
        # a deeper network's 300 tensors, slices of one bucket without padding, in place; below the threshold, as most updates are
        dict(name="clip_300_in_place", op="clip", sizes="spread", count=300, total=12_000_000, src="fp32", dst="fp32", inplace=True, pad=False, ratio=2.0),
        # a large model's 60 tensors, clipped into a bucket with aligned slices
        dict(name="clip_60_large", op="clip", sizes="spread", count=60, total=120_000_000, src="bf16", dst="bf16", inplace=False, pad=True, ratio=0.3),
        # acting: one step of the paper's 32 environments, the state carried on
        dict(name="scan_step_32", op="scan", dir="fwd", t=1, n=32, c=256, type="fp32", kind="sigmoid", reverse=False, layout="time", restart=200, carry=True),
        # an update batch of the largest configuration, five steps of 1024 environments with 512 hidden units, and its backward pass, where
        # gate and candidate are the two halves of one product
        dict(name="scan_rollout", op="scan", dir="fwd", t=5, n=1024, c=512, type="bf16", kind="sigmoid", reverse=False, layout="packed", restart=200, carry=True),
        dict(name="scan_rollout_back", op="scan", dir="bwd", t=5, n=1024, c=512, type="bf16", kind="sigmoid", reverse=False, layout="packed", restart=200, carry=False),
        # two long recordings, batch first
        dict(name="scan_long", op="scan", dir="fwd", t=32768, n=2, c=512, type="bf16", kind="sigmoid", reverse=False, layout="batch", restart=2000, carry=False),
        # training on three recordings of odd length, plain coefficients, float
        dict(name="scan_long_back", op="scan", dir="bwd", t=20011, n=3, c=200, type="fp32", kind="linear", reverse=False, layout="time", restart=500, carry=True),
        # acting: feature maps of 32 states behind the first convolution
        dict(name="norm_act_32", op="norm", dir="fwd", n=32, p=400, c=32, groups=4, type="bf16", act="relu"),
        # the same behind the first convolution for a whole update batch, and backward behind the second
        dict(name="norm_update", op="norm", dir="fwd", n=5120, p=400, c=32, groups=4, type="bf16", act="relu"),
        dict(name="norm_update_back", op="norm", dir="bwd", n=5120, p=81, c=64, groups=8, type="bf16", act="relu"),
        # a residual network's first stage on whole frames, float, odd batch
        dict(name="norm_frames_back", op="norm", dir="bwd", n=37, p=84 * 84, c=48, groups=6, type="fp32", act="silu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["clip", "scan", "scan", "norm"])
    if op == "clip":
        inplace = rng.random() < 0.4
        src = rng.choice(["fp32", "bf16"])
        return dict(op=op, sizes="spread", count=_log(rng, 1, 400), total=_log(rng, 1000, 50_000_000), src=src, dst=src if inplace else rng.choice(["fp32", "bf16"]),
                    inplace=inplace, pad=rng.random() < 0.5, ratio=2.0 if inplace else rng.choice([0.1, 0.45, 2.0]))
    kind = rng.choice(["fp32", "bf16"])
    if op == "scan":
        c = rng.choice([1, 7, 30, 64, 128, 200, 256, 512, _log(rng, 1, 1024)])
        t = _log(rng, 1, 32768)
        n = max(1, min(_log(rng, 1, 2048), 16_000_000 // (t * c)))
        return dict(op=op, dir=rng.choice(["fwd", "bwd"]), t=t, n=n, c=c, type=kind, kind=rng.choice(["sigmoid", "linear"]), reverse=rng.random() < 0.3,
                    layout=rng.choice(["time", "time", "batch", "packed"]), restart=rng.choice([0, 3, 200]), carry=rng.random() < 0.5)
    groups = rng.choice([1, 2, 3, 4, 8, 16, 32])
    c = groups * rng.choice([1, 2, 4, 5, 8, 16])
    p = rng.choice([1, 49, 81, 400, 441, 84 * 84, _log(rng, 1, 20000)])
    n = max(1, min(_log(rng, 1, 5120), 30_000_000 // (p * c)))
    return dict(op=op, dir=rng.choice(["fwd", "bwd"]), n=n, p=p, c=c, groups=groups, type=kind, act=rng.choice(["none", "relu", "silu"]))


# ---- what a program has in hand -------------------------------------------------------------------------------------------------

def _sizes(case):
    """Element counts of the tensors: matrices of round sizes among a few odd ones, some thousand times the size of others."""
    if case["sizes"] == "nature":
        return list(NATURE)
    rng = random.Random(case["count"])
    parts = [math.exp(rng.uniform(0, 7)) for _ in range(case["count"])]
    sizes = [max(1, int(case["total"] * p / sum(parts))) for p in parts]
    return [s if s < 64 or rng.random() < 0.25 else s // 64 * 64 for s in sizes]


def _prepare_clip(case, gen):
    sizes = _sizes(case)
    at, places = 0, []
    for s in sizes:
        places.append(at)
        at += -(-s // 64) * 64 if case["pad"] else s
    # gradients of a training run: many small values, a few large ones; the norm a known multiple of the threshold
    factor = CLIP / case["ratio"] / math.sqrt(15.0 * sum(sizes))
    def values(k, kind):
        return (torch.randn(k, device="cuda", generator=gen).pow_(3).mul_(factor)).to(TYPES[kind])
    if case["inplace"]:
        flat = values(at, case["src"])
        dst = src = [flat[p:p + s] for p, s in zip(places, sizes)]
    else:
        flat = torch.zeros(at, dtype=TYPES[case["dst"]], device="cuda")
        src, dst = [values(s, case["src"]) for s in sizes], [flat[p:p + s] for p, s in zip(places, sizes)]
    s = dict(src=src, dst=dst, flat=flat, norm=torch.zeros(2, device="cuda"))
    if own:
        # a training program's gradients stay where they are: it makes the list once
        import paper_1705_04862_b200.binding as pb
        s["list"] = pb.TensorList(src, dst)
    return s


def _sequences(case, count, gen=None, fill=None):
    """`count` tensors [t][n][c] in the case's layout; packed: side by side in one."""
    t, n, c, kind = case["t"], case["n"], case["c"], TYPES[case["type"]]
    if case["layout"] == "packed":
        whole = torch.empty(t, n, count * c, dtype=kind, device="cuda")
        views = [whole[..., i * c:(i + 1) * c] for i in range(count)]
    elif case["layout"] == "batch":
        views = [torch.empty(n, t, c, dtype=kind, device="cuda").transpose(0, 1) for _ in range(count)]
    else:
        views = [torch.empty(t, n, c, dtype=kind, device="cuda") for _ in range(count)]
    for v, f in zip(views, fill or []):
        v.copy_(f)
    return views


def _prepare_scan(case, gen):
    t, n, c = case["t"], case["n"], case["c"]

    def noise(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    # gates that mostly keep: a state lasts some ten steps; coefficients are those gates themselves, or a discount
    logits = noise(t, n, c) + 2.0
    fill = [logits if case["kind"] == "sigmoid" else torch.sigmoid(logits) * GAMMA, noise(t, n, c)]
    s = {}
    s["gate"], s["x"] = _sequences(case, 2, fill=fill)
    s["restart"] = None
    if case["restart"]:
        s["restart"] = (torch.rand(t, n, device="cuda", generator=gen) < 1.0 / case["restart"]).to(torch.uint8)
    s["h0"] = noise(n, c) if case["carry"] else None
    (s["h"],) = _sequences(dict(case, layout="batch" if case["layout"] == "batch" else "time"), 1)
    s["h_last"] = torch.empty(n, c, device="cuda")
    if case["dir"] == "bwd":
        s["h"].copy_(_scan_forward(case, s)["h"])
        (s["dh"],) = _sequences(dict(case, layout="batch" if case["layout"] == "batch" else "time"), 1, fill=[noise(t, n, c)])
        s["dh_last"] = noise(n, c) if case["carry"] else None
        s["dgate"], s["dx"] = _sequences(case, 2)
        s["dh0"] = torch.empty(n, c, device="cuda") if case["carry"] else None
    return s


def _prepare_norm(case, gen):
    n, p, c, g, kind = case["n"], case["p"], case["c"], case["groups"], TYPES[case["type"]]
    # what a convolution gives: every channel with a mean and a spread of its own
    x = torch.randn(n, p, c, device="cuda", generator=gen)
    x.mul_(0.5 + torch.rand(c, device="cuda", generator=gen)).add_(torch.randn(c, device="cuda", generator=gen))
    s = dict(x=x.to(kind), y=torch.empty(n, p, c, dtype=kind, device="cuda"), gamma=1.0 + 0.2 * torch.randn(c, device="cuda", generator=gen),
             beta=0.2 * torch.randn(c, device="cuda", generator=gen), mean=torch.empty(n, g, device="cuda"), rstd=torch.empty(n, g, device="cuda"), workspace=None)
    if case["dir"] == "bwd":
        d = s["x"].double().view(n, p, g, c // g)
        mean = d.mean((1, 3))
        s["mean"], s["rstd"] = mean.float(), (d.sub_(mean[:, None, :, None]).square_().mean((1, 3)) + EPS).rsqrt_().float()
        dy = torch.randn(n, p, c, device="cuda", generator=gen)
        if case["act"] == "relu":
            # the derivative has a step at 0: within rounding of it either side is right, so nothing arrives there
            dy.mul_((_pre(case, s, torch.float64).abs() > 1e-4).view(n, p, c))
        s["dy"] = dy.to(kind)
        s["dx"], s["dgamma"], s["dbeta"] = torch.empty_like(s["x"]), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    if own:
        import paper_1705_04862_b200.binding as pb
        s["workspace"] = torch.empty(pb.group_norm_workspace_bytes(n, p, c, g, pb.BF16 if kind == torch.bfloat16 else pb.FP32), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return dict({"clip": _prepare_clip, "scan": _prepare_scan, "norm": _prepare_norm}[case["op"]](case, gen), case=case)


# ---- the plain forms ------------------------------------------------------------------------------------------------------------

def _clip(case, s):
    norm = torch.stack([g.float().square().sum() for g in s["src"]]).sum().sqrt()
    scale = torch.clamp(CLIP / norm, max=1.0)
    # in place below the threshold the factor is 1 and the product changes nothing
    [d.copy_(g.float() * scale) for g, d in zip(s["src"], s["dst"])]
    return {"norm_and_scale": torch.stack([norm, scale]), "grads": s["flat"]}


def _recurrence(a, b):
    """h_t = a_t h_{t-1} + b_t over the first axis: spans of two, four, eight, ... steps joined."""
    span = 1
    while span < a.shape[0]:
        b = torch.cat([b[:span], torch.addcmul(b[span:], a[span:], b[:-span])])
        a = torch.cat([a[:span], a[span:] * a[:-span]])
        span *= 2
    return b


def _coefficients(case, s):
    """(what a step keeps, before restarts; what it keeps; what it takes of x) in 32 bits, in the order of the recurrence."""
    gate = s["gate"].float()
    keep, take = (torch.sigmoid(gate), torch.sigmoid(-gate)) if case["kind"] == "sigmoid" else (gate, torch.ones_like(gate))
    cut = keep if s["restart"] is None else torch.where((s["restart"] != 0)[..., None], torch.zeros_like(keep), keep)
    return keep, cut, take


def _turned(case, v):
    return v.flip(0) if case["reverse"] else v


def _scan_forward(case, s):
    _, cut, take = _coefficients(case, s)
    a, b = _turned(case, cut), _turned(case, take * s["x"].float())
    if s["h0"] is not None:
        b = torch.cat([(b[0] + a[0] * s["h0"])[None], b[1:]])
    h = _recurrence(a, b)
    return {"h": _turned(case, h).to(TYPES[case["type"]]), "h_last": h[-1]}


def _scan_backward(case, s):
    keep, cut, take = _coefficients(case, s)
    a, dh, h = _turned(case, cut), _turned(case, s["dh"].float()), _turned(case, s["h"].float())
    h0 = torch.zeros_like(h[0]) if s["h0"] is None else s["h0"]
    if s["dh_last"] is not None:
        dh = torch.cat([dh[:-1], (dh[-1] + s["dh_last"])[None]])
    # G_t = dh_t + a_{t+1} G_{t+1}, from the last step to the first
    grad = _recurrence(torch.cat([torch.zeros_like(a[:1]), a[1:].flip(0)]), dh.flip(0)).flip(0)
    before = torch.cat([h0[None], h[:-1]])
    if s["restart"] is not None:
        before = torch.where((_turned(case, s["restart"]) != 0)[..., None], torch.zeros_like(before), before)
    if case["kind"] == "sigmoid":
        dgate = grad * (before - _turned(case, s["x"].float())) * _turned(case, keep) * _turned(case, take)
        dx = grad * _turned(case, take)
    else:
        dgate, dx = grad * before, grad
    kind = TYPES[case["type"]]
    return {"dgate": _turned(case, dgate).to(kind), "dx": _turned(case, dx).to(kind), "dh0": a[0] * grad[0] if case["carry"] else None}


def _pre(case, s, kind):
    """(x - mean) / deviation, scaled and shifted."""
    n, p, c, g = (case[k] for k in ("n", "p", "c", "groups"))
    x = s["x"].to(kind).view(n, p, g, c // g)
    x = (x - s["mean"].to(kind)[:, None, :, None]) * s["rstd"].to(kind)[:, None, :, None]
    return x.reshape(n, p, c) * s["gamma"].to(kind) + s["beta"].to(kind)


def _norm_forward(case, s):
    n, p, c, g = (case[k] for k in ("n", "p", "c", "groups"))
    x = s["x"].float().view(n, p, g, c // g)
    mean = x.mean((1, 3))
    rstd = ((x - mean[:, None, :, None]).square().mean((1, 3)) + EPS).rsqrt()
    v = _pre(case, dict(s, mean=mean, rstd=rstd), torch.float32)
    y = v.clamp(min=0.0) if case["act"] == "relu" else v * torch.sigmoid(v) if case["act"] == "silu" else v
    return {"y": y.to(TYPES[case["type"]]), "mean": mean, "rstd": rstd}


def _norm_backward(case, s):
    n, p, c, g = (case[k] for k in ("n", "p", "c", "groups"))
    dv = s["dy"].float()
    if case["act"] == "relu":
        dv = dv * (_pre(case, s, torch.float32) > 0)
    elif case["act"] == "silu":
        v = _pre(case, s, torch.float32)
        sig = torch.sigmoid(v)
        dv = dv * sig * (1.0 + v * (1.0 - sig))
    rstd = s["rstd"][:, None, :, None]
    xhat = ((s["x"].float().view(n, p, g, c // g) - s["mean"][:, None, :, None]) * rstd).view(n, p, c)
    dgamma, dbeta = (dv * xhat).sum(1).sum(0), dv.sum(1).sum(0)
    d, xhat = (dv * s["gamma"]).view(n, p, g, c // g), xhat.view(n, p, g, c // g)
    dx = rstd * (d - d.mean((1, 3), keepdim=True) - xhat * (d * xhat).mean((1, 3), keepdim=True))
    return {"dx": dx.reshape(n, p, c).to(TYPES[case["type"]]), "dgamma": dgamma, "dbeta": dbeta}


def _plain(case, s):
    if case["op"] == "clip":
        return _clip(case, s)
    if case["op"] == "scan":
        return (_scan_forward if case["dir"] == "fwd" else _scan_backward)(case, s)
    return (_norm_forward if case["dir"] == "fwd" else _norm_backward)(case, s)


# ---- the library's calls --------------------------------------------------------------------------------------------------------

def _library(case, s):
    import paper_1705_04862_b200.binding as pb
    if case["op"] == "clip":
        status = pb.clip_tensors(s["list"], CLIP, norm_and_scale=s["norm"])
        out = {"norm_and_scale": s["norm"], "grads": s["flat"]}
    elif case["op"] == "scan":
        how = dict(kind=pb.SCAN_SIGMOID if case["kind"] == "sigmoid" else pb.SCAN_LINEAR, reverse=case["reverse"], restart=s["restart"], h0=s["h0"])
        if case["dir"] == "fwd":
            status = pb.gated_scan(s["gate"], s["x"], s["h"], h_last=s["h_last"], **how)
            out = {"h": s["h"], "h_last": s["h_last"]}
        else:
            x = s["x"] if case["kind"] == "sigmoid" else None
            status = pb.gated_scan_backward(s["gate"], x, s["h"], s["dh"], s["dgate"], s["dx"], dh_last=s["dh_last"], dh0=s["dh0"], **how)
            out = {"dgate": s["dgate"], "dx": s["dx"], "dh0": s["dh0"]}
    else:
        act = {"none": pb.ACT_NONE, "relu": pb.ACT_RELU, "silu": pb.ACT_SILU}[case["act"]]
        if case["dir"] == "fwd":
            status = pb.group_norm(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], case["groups"], s["workspace"], activation=act, eps=EPS)
            out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        else:
            status = pb.group_norm_backward(s["x"], s["dy"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], case["groups"],
                                            s["workspace"], activation=act)
            out = {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if status != pb.OK:
        raise pb.PaacError(status)
    return out


def run(s):
    return (_library if own else _plain)(s["case"], s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------------

def work(case):
    """Bytes: every input read once, every output written once (in place below the threshold nothing is written)."""
    if case["op"] == "clip":
        size, e = sum(_sizes(case)), {"fp32": 4, "bf16": 2}
        written = 0 if case["inplace"] else size * e[case["dst"]]
        return {"bytes": size * e[case["src"]] + written + 8, "flops": size * (2 if case["inplace"] else 3)}
    e = {"fp32": 4, "bf16": 2}[case["type"]]
    if case["op"] == "scan":
        cells, columns = case["t"] * case["n"] * case["c"], case["n"] * case["c"]
        sigmoid, flags = case["kind"] == "sigmoid", case["t"] * case["n"] * (1 if case["restart"] else 0)
        if case["dir"] == "fwd":
            return {"bytes": 3 * e * cells + flags + 4 * columns * (1 + case["carry"]), "flops": cells * (7 if sigmoid else 2)}
        return {"bytes": (6 if sigmoid else 5) * e * cells + flags + 4 * columns * 3 * case["carry"], "flops": cells * (11 if sigmoid else 3)}
    cells, stats = case["n"] * case["p"] * case["c"], 4 * 2 * case["n"] * case["groups"]
    if case["dir"] == "fwd":
        return {"bytes": 2 * e * cells + stats + 8 * case["c"], "flops": cells * 8}
    return {"bytes": 3 * e * cells + stats + 16 * case["c"], "flops": cells * 14}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------------

def _exact_clip(case, s):
    total = sum(float((g.double() * g.double()).sum()) for g in s["src"])
    norm = math.sqrt(total)
    scale = CLIP / norm if norm > CLIP else 1.0
    flat = s["flat"].double()
    if not case["inplace"]:
        ends = [d.storage_offset() for d in s["dst"]]
        for g, at in zip(s["src"], ends):
            flat[at:at + g.numel()] = g.double() * scale
    elif scale != 1.0:
        return None
    return {"norm_and_scale": torch.tensor([norm, scale], dtype=torch.float64), "grads": flat}


def _exact_scan(case, s):
    """Step by step, as the recurrence is written; the gradient step by step from the far end."""
    steps = list(range(case["t"]))
    if case["reverse"]:
        steps.reverse()
    sigmoid = case["kind"] == "sigmoid"
    gate, x = s["gate"].double(), s["x"].double()
    z = 1.0 / (1.0 + torch.exp(-gate)) if sigmoid else gate
    u = x / (1.0 + torch.exp(gate)) if sigmoid else x
    zero = torch.zeros(case["n"], case["c"], dtype=torch.float64, device="cuda")
    start = zero if s["h0"] is None else s["h0"].double()
    on = torch.ones(case["t"], case["n"], 1, dtype=torch.float64, device="cuda") if s["restart"] is None else (s["restart"] == 0).double()[..., None]
    if case["dir"] == "fwd":
        h, state = torch.empty_like(u), start
        for t in steps:
            state = torch.addcmul(u[t], z[t] * on[t], state)
            h[t] = state
        return {"h": h, "h_last": state}
    h, dh = s["h"].double(), s["dh"].double()
    carried = zero if s["dh_last"] is None else s["dh_last"].double()
    dgate, dx = torch.empty_like(gate), torch.empty_like(gate)
    for k in range(case["t"] - 1, -1, -1):
        t = steps[k]
        g = dh[t] + carried
        prev = (h[steps[k - 1]] if k else start) * on[t]
        dgate[t] = g * (prev - x[t]) * z[t] / (1.0 + torch.exp(gate[t])) if sigmoid else g * prev
        dx[t] = g / (1.0 + torch.exp(gate[t])) if sigmoid else g
        carried = g * z[t] * on[t]
    return {"dgate": dgate, "dx": dx, "dh0": carried if case["carry"] else None}


def _exact_norm(case, s):
    """By the definition of mean and variance; the gradient by the chain rule through the mean and the deviation."""
    n, p, c, g = (case[k] for k in ("n", "p", "c", "groups"))
    x, gamma, beta = s["x"].double().view(n, p, g, -1), s["gamma"].double().view(g, -1), s["beta"].double().view(g, -1)
    if case["dir"] == "fwd":
        m = x.sum((1, 3), keepdim=True) / (p * (c // g))
        var = (x - m).pow(2).sum((1, 3), keepdim=True) / (p * (c // g))
        r = (var + EPS).pow(-0.5)
    else:
        m, r = s["mean"].double()[:, None, :, None], s["rstd"].double()[:, None, :, None]
    v = (x - m) * r * gamma + beta
    if case["dir"] == "fwd":
        y = torch.relu(v) if case["act"] == "relu" else v / (1.0 + torch.exp(-v)) if case["act"] == "silu" else v
        return {"y": y.reshape(n, p, c), "mean": m.view(n, g), "rstd": r.view(n, g)}
    dv = s["dy"].double().view(n, p, g, -1)
    if case["act"] == "relu":
        dv = torch.where(v > 0, dv, torch.zeros_like(dv))
    elif case["act"] == "silu":
        e = torch.exp(-v)
        dv = dv * ((1.0 + e + v * e) / (1.0 + e) ** 2)
    centred = x - m
    dgamma, dbeta = (dv * centred * r).sum((0, 1)), dv.sum((0, 1))
    count = p * (c // g)
    through = dv * gamma
    dvar = (through * centred).sum((1, 3), keepdim=True) * -0.5 * r ** 3
    dx = through * r - r * through.sum((1, 3), keepdim=True) / count + dvar * 2.0 * centred / count
    return {"dx": dx.reshape(n, p, c), "dgamma": dgamma.reshape(c), "dbeta": dbeta.reshape(c)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"clip": _exact_clip, "scan": _exact_scan, "norm": _exact_norm}[case["op"]](case, s)
