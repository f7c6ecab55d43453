"""The operators of a policy over sequences as a learner would use them: steps embedded, the short convolution, the selective scan, logits of many actions; acting step by
step with what is carried, then the way back over the whole rollout, clipping and the optimiser.  Episodes end where the library's own learner's do."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from operators_ref import U
from paper_1705_04862_b200 import binding as pb
from test_gpu_operators_together import terminals

pytestmark = pytest.mark.gpu
T, N, C, S, ACTIONS = 5, 32, 24, 16, 300          # steps and environments of that learner; channels, states of a channel, actions
BETA, CLIP, LR, DECAY, EPS = 0.01, 0.05, 0.01, 0.99, 0.1
NAMES = ["weight", "bias", "to_dt", "to_b", "to_c", "A", "D", "dt_bias", "head"]


def network(seed):
    g = torch.Generator().manual_seed(seed)

    def noise(*shape):
        return torch.randn(*shape, generator=g)

    p = dict(weight=noise(C, 4) / 2, bias=0.1 * noise(C), to_dt=0.3 * noise(C, C), to_b=noise(S, C) / 5, to_c=noise(S, C) / 5, A=-(1 + torch.arange(S).float()).repeat(C, 1), D=1 + 0.1 * noise(C),
             dt_bias=noise(C) - 3, head=noise(ACTIONS, C) / 5)
    return p, noise(T, N, C), torch.rand(T, N, generator=g), noise(T, N)


def by_autograd(p, x, restart, actions, advantages):
    """loss, logits and gradients in 64 bits, step by step."""
    q = {k: v.double().requires_grad_() for k, v in p.items()}
    x = x.double()
    held, state, logits = [torch.zeros(N, C, dtype=torch.float64)] * 3, torch.zeros(N, C, S, dtype=torch.float64), []
    for t in range(T):
        on = (restart[t] == 0).double()
        held = [v * on[:, None] for v in held] + [x[t]]
        v = q["bias"] + sum(q["weight"][:, k] * held[k] for k in range(4))
        held = held[1:]
        u = v * torch.sigmoid(v)
        delta = torch.nn.functional.softplus(u @ q["to_dt"].t() + q["dt_bias"])
        b, c = u @ q["to_b"].t(), u @ q["to_c"].t()
        state = torch.exp(delta[..., None] * q["A"]) * state * on[:, None, None] + (delta * u)[..., None] * b[:, None, :]
        logits.append(((state * c[:, None, :]).sum(2) + q["D"] * u) @ q["head"].t())
    logits = torch.stack(logits)
    logp = torch.log_softmax(logits, 2)
    taken = torch.gather(logp, 2, actions.long()[..., None])[..., 0]
    loss = -(advantages.double() * taken).mean() + BETA * (logp.exp() * logp).sum(2).mean()
    loss.backward()
    return float(loss.detach()), logits.detach(), taken.detach(), {k: v.grad for k, v in q.items()}


class Policy:
    def __init__(self, p):
        self.p = {k: v.cuda() for k, v in p.items()}

    def steps(self, x, restart, before=None, after=None, h0=None, last=None, states=None):
        """Everything up to the logits for the steps of x; by the library, but for the products."""
        p, t = self.p, x.shape[0]
        u = torch.empty_like(x)
        assert pb.causal_conv(x, p["weight"], p["bias"], u, before=before, after=after, restart=restart) == pb.OK
        dt, b, c = u @ p["to_dt"].t(), u @ p["to_b"].t(), u @ p["to_c"].t()
        y = torch.empty_like(x)
        need = pb.selective_scan_workspace_bytes(t, N, C, S, 1, pb.FP32)
        room = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        assert pb.selective_scan(u, dt, p["A"], b, c, y, room, D=p["D"], dt_bias=p["dt_bias"], h0=h0, h_last=last, states=states, restart=restart) == pb.OK
        return y @ p["head"].t(), (u, dt, b, c, y)

    def act(self, x, restart, uniforms):
        """(actions, log-probabilities) step by step, the convolution's inputs and the scan's states carried on in place."""
        held, state = torch.zeros(N, 3, C, device="cuda"), torch.zeros(N, C, S, device="cuda")
        actions, logp = torch.empty(T, N, dtype=torch.int32, device="cuda"), torch.empty(T, N, device="cuda")
        for t in range(T):
            logits, _ = self.steps(x[t:t + 1], restart[t:t + 1], held, held, state, state)
            assert pb.sample(logits[0], uniforms[t], actions[t], logprob=logp[t]) == pb.OK
        return actions, logp

    def learn(self, x, restart, actions, advantages):
        p = self.p
        states = torch.empty(1, N, C, S, device="cuda")
        logits, (u, dt, b, c, y) = self.steps(x, restart, states=states)
        logp = torch.log_softmax(logits, 2)
        taken = torch.gather(logp, 2, actions.long()[..., None])
        prob = logp.exp()
        loss = -(advantages[..., None] * taken).mean() + BETA * (prob * logp).sum(2).mean()
        # Equation 10's gradient by the logits: of -advantage log pi and of beta sum pi log pi
        hot = torch.zeros_like(prob).scatter_(2, actions.long()[..., None], 1.0)
        dlogits = (advantages[..., None] * (prob - hot) + BETA * prob * (logp - (prob * logp).sum(2, keepdim=True))) / (T * N)
        g = dict(head=dlogits.flatten(0, 1).t() @ y.flatten(0, 1))
        dy = dlogits @ p["head"]
        du, ddt, db, dc = (torch.empty_like(v) for v in (u, dt, b, c))
        g.update(A=torch.empty_like(p["A"]), D=torch.empty_like(p["D"]), dt_bias=torch.empty_like(p["dt_bias"]), weight=torch.empty_like(p["weight"]), bias=torch.empty_like(p["bias"]))
        room = torch.empty(max(pb.selective_scan_workspace_bytes(T, N, C, S, 1, pb.FP32, backward=True), pb.causal_conv_workspace_bytes(T, N, C, 4, pb.FP32)), dtype=torch.uint8, device="cuda")
        assert pb.selective_scan_backward(u, dt, p["A"], b, c, dy, states, du, ddt, g["A"], db, dc, room, D=p["D"], dt_bias=p["dt_bias"], dD=g["D"], ddt_bias=g["dt_bias"], restart=restart) == pb.OK
        flat = u.flatten(0, 1)
        g.update(to_dt=ddt.flatten(0, 1).t() @ flat, to_b=db.flatten(0, 1).t() @ flat, to_c=dc.flatten(0, 1).t() @ flat)
        du = du + ddt @ p["to_dt"] + db @ p["to_b"] + dc @ p["to_c"]
        assert pb.causal_conv_backward(x, du, p["weight"], p["bias"], None, g["weight"], g["bias"], room, restart=restart) == pb.OK
        return float(loss), logits, g


@pytest.fixture
def exact_products():
    was = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    yield
    torch.backends.cuda.matmul.allow_tf32 = was


def test_acting_and_learning(exact_products):
    p, x, uniforms, advantages = network(3)
    restart, policy = terminals(), Policy(p)
    x, uniforms, advantages = x.cuda(), uniforms.cuda(), advantages.cuda()
    actions, logp = policy.act(x, restart, uniforms)
    loss, logits, grads = policy.learn(x, restart, actions, advantages)
    want_loss, want_logits, want_logp, want = by_autograd(p, x.cpu(), restart.cpu(), actions.cpu(), advantages.cpu())
    # A logit passes products of at most 24 terms, four sums of the convolution, and five steps of the scan with 16 states: at most some 150 roundings
    # one after the other, of terms that are some ten times the largest logit together
    top = float(want_logits.abs().max())
    assert float((logits.cpu().double() - want_logits).abs().max()) <= 1500 * U * top
    assert float((logp.cpu().double() - want_logp).abs().max()) <= 3000 * U * top
    assert abs(loss - want_loss) <= 3000 * U * max(1.0, abs(want_loss)) * top
    # the uniform lies in the action's part of the running sum of the exact probabilities, whose borders the logits' errors move by no more than that
    run = torch.cumsum(torch.softmax(want_logits, 2), 2)
    end = torch.gather(run, 2, actions.cpu().long()[..., None])[..., 0]
    u, off = uniforms.cpu().double(), 3000 * U * top
    assert bool(((u < end + off) & (u > end - want_logp.exp() - off)).all())
    # gradients: sums over 160 steps and up to 300 actions of what the logits' errors have reached, each passing as many roundings again
    for name in NAMES:
        g, exact = grads[name].double().cpu(), want[name]
        assert float((g - exact).abs().max()) <= 6000 * U * float(exact.abs().max()), name

    # clipped into one vector, which the optimiser takes
    theta = torch.cat([policy.p[k].reshape(-1) for k in NAMES])
    flat, rms, told = torch.zeros_like(theta), torch.zeros_like(theta), torch.zeros(2, device="cuda")
    places, at = [], 0
    for k in NAMES:
        places.append(flat[at:at + grads[k].numel()])
        at += grads[k].numel()
    before = theta.clone()
    assert pb.clip_tensors(pb.TensorList([grads[k].contiguous().reshape(-1) for k in NAMES], places), CLIP, norm_and_scale=told) == pb.OK
    assert pb.clip_rmsprop_noalloc(theta, rms, flat, theta.numel(), LR, DECAY, EPS, 0.0, stream=torch.cuda.current_stream().cuda_stream) == pb.OK
    torch.cuda.synchronize()
    assert np.isfinite(float(told[0])) and 0 < float(told[1]) <= 1 and not torch.equal(theta, before) and torch.isfinite(theta).all()


def test_acting_recorded_beside_eager_calls(exact_products):
    """A step of acting in one graph, replayed on a stream of its own while a second copy of the same policy acts eagerly elsewhere: the same actions."""
    p, x, uniforms, _ = network(4)
    x, uniforms = x.cuda(), uniforms.cuda()
    restart = (torch.rand(T, N, generator=torch.Generator().manual_seed(2)) < 0.2).to(torch.uint8).cuda()
    policy = Policy(p)
    want, want_logp = policy.act(x, restart, uniforms)
    torch.cuda.synchronize()
    now = dict(x=torch.zeros(1, N, C, device="cuda"), restart=torch.zeros(1, N, dtype=torch.uint8, device="cuda"), u=torch.zeros(N, device="cuda"), held=torch.zeros(N, 3, C, device="cuda"),
               state=torch.zeros(N, C, S, device="cuda"), action=torch.zeros(N, dtype=torch.int32, device="cuda"), logp=torch.zeros(N, device="cuda"))
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        logits, _ = policy.steps(now["x"], now["restart"], now["held"], now["held"], now["state"], now["state"])
        assert pb.sample(logits[0], now["u"], now["action"], logprob=now["logp"]) == pb.OK
    got = []
    with torch.cuda.stream(stream):
        now["held"].zero_()
        now["state"].zero_()
        for t in range(T):
            now["x"].copy_(x[t:t + 1])
            now["restart"].copy_(restart[t:t + 1])
            now["u"].copy_(uniforms[t])
            graph.replay()
            got.append((now["action"].clone(), now["logp"].clone()))
    again, again_logp = policy.act(x, restart, uniforms)
    torch.cuda.synchronize()
    assert torch.equal(torch.stack([a for a, _ in got]), want) and torch.equal(again, want)
    assert torch.equal(torch.stack([q for _, q in got]), want_logp) and torch.equal(again_logp, want_logp)


FIRST = """
import sys
sys.path.insert(0, %r)
import torch
from paper_1705_04862_b200 import binding as pb
x, w, y = (torch.randn(40, 2, 24, device="cuda") for _ in range(3))
weight, A, b = torch.randn(24, 4, device="cuda"), -torch.rand(24, 16, device="cuda"), torch.randn(40, 2, 16, device="cuda")
states, grads = torch.empty(3, 2, 24, 16, device="cuda"), [torch.empty_like(v) for v in (x, x, A, b, b, weight)]
room = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
actions, u, logits = torch.empty(80, dtype=torch.int32, device="cuda"), torch.rand(80, device="cuda"), torch.randn(80, 5000, device="cuda")
p = torch.full((80,), 0.7, device="cuda")
def run():
    assert pb.causal_conv(x, weight, None, y) == pb.OK
    assert pb.selective_scan(y, w, A, b, b, x, room, states=states) == pb.OK
    assert pb.selective_scan_backward(y, w, A, b, b, x, states, grads[0], grads[1], grads[2], grads[3], grads[4], room) == pb.OK
    assert pb.causal_conv_backward(x, grads[0], weight, None, grads[1], grads[5], None, room) == pb.OK
    assert pb.sample(logits, u, actions, top_p=p) == pb.OK
torch.cuda.synchronize()
keep = x.clone()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    run()
x.copy_(keep)
g.replay()
torch.cuda.synchronize()
taped = [v.clone() for v in [x, y, states, actions] + grads]
x.copy_(keep)
run()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(taped, [x, y, states, actions] + grads))
print("the same")
"""


def test_the_first_calls_of_a_process_recorded():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST % root], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "the same" in r.stdout, r.stdout + r.stderr
