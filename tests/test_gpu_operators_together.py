"""The operators for a caller's own network as a learner would use them, one after the other: feature maps normalised, a memory over a rollout
of the library's own learner cut where its episodes end, the way back, the gradients clipped into one vector and taken by the
optimiser.  Against the same in 64 bits by torch's autograd."""
import numpy as np
import pytest
import torch

from operators_ref import U
from paper_1705_04862_b200 import binding as pb

pytestmark = pytest.mark.gpu
T, N, P, C, G, S = 5, 32, 49, 16, 4, 24          # steps, environments, pixels, channels, groups, units of the memory
CLIP, LR, DECAY, EPS = 0.05, 0.01, 0.99, 0.1


def terminals():
    """Ends of episodes of a rollout, and where the steps behind them begin."""
    g = pb.Paac("nips", N, T, 4, seed=11, term_denom=6)
    g.rollout()
    ends = torch.from_numpy(g.debug_read(pb.DBG_TERMINALS).copy()).view(T, N).cuda()
    torch.cuda.synchronize()
    g.close()
    restart = torch.zeros_like(ends)
    restart[1:] = ends[:-1]
    assert 0 < int(restart.sum()) < T * N
    return restart


class Net:
    """maps -> norm -> sum over pixels -> gate and candidate -> memory; every parameter a tensor of its own."""

    def __init__(self, seed):
        gen = torch.Generator().manual_seed(seed)
        self.gamma, self.beta = 1 + 0.1 * torch.randn(C, generator=gen), 0.1 * torch.randn(C, generator=gen)
        self.w, self.b = 0.2 * torch.randn(2 * S, C, generator=gen), 0.1 * torch.randn(2 * S, generator=gen)
        self.maps, self.target = torch.randn(T * N, P, C, generator=gen), torch.randn(T, N, S, generator=gen)
        self.h0 = torch.randn(N, S, generator=gen)

    def params(self):
        return [self.gamma, self.beta, self.w, self.b]


def by_autograd(net, restart):
    leaves = [p.double().requires_grad_() for p in net.params()]
    gamma, beta, w, b = leaves
    y = torch.relu(torch.nn.functional.group_norm(net.maps.double().transpose(1, 2), G, gamma, beta, 1e-5).transpose(1, 2))
    z = (y.mean(1) @ w.t() + b).view(T, N, 2 * S)
    state, hs = net.h0.double(), []
    for t in range(T):
        gate = torch.sigmoid(z[t, :, :S])
        state = torch.where((restart[t] != 0)[:, None], torch.zeros_like(state), state) * gate + (1 - gate) * z[t, :, S:]
        hs.append(state)
    loss = 0.5 * ((torch.stack(hs) - net.target.double()) ** 2).mean()
    loss.backward()
    return float(loss.detach()), [p.grad for p in leaves]


def by_the_library(net, restart, work):
    """loss and gradients; products by torch, the rest by the operators.  `work`: buffers that are kept."""
    d = {k: v.cuda() for k, v in dict(gamma=net.gamma, beta=net.beta, w=net.w, b=net.b, maps=net.maps, target=net.target, h0=net.h0).items()}
    n = T * N
    work.setdefault("room", torch.empty(pb.group_norm_workspace_bytes(n, P, C, G, pb.FP32), dtype=torch.uint8, device="cuda"))
    y, mean, rstd = torch.empty_like(d["maps"]), *(torch.empty(n, G, device="cuda") for _ in range(2))
    assert pb.group_norm(d["maps"], d["gamma"], d["beta"], y, mean, rstd, G, work["room"], activation=pb.ACT_RELU) == pb.OK
    pooled = y.mean(1)
    z = (pooled @ d["w"].t() + d["b"]).view(T, N, 2 * S)
    h, last = torch.empty(T, N, S, device="cuda"), torch.empty(N, S, device="cuda")
    gate, x = z[..., :S], z[..., S:]
    assert pb.gated_scan(gate, x, h, h0=d["h0"], h_last=last, restart=restart) == pb.OK
    loss = 0.5 * ((h - d["target"]) ** 2).mean()
    dh = (h - d["target"]) / h.numel()
    dz = torch.empty_like(z)
    assert pb.gated_scan_backward(gate, x, h, dh, dz[..., :S], dz[..., S:], h0=d["h0"], restart=restart) == pb.OK
    dz = dz.view(n, 2 * S)
    dw, db = dz.t() @ pooled, dz.sum(0)
    dy = ((dz @ d["w"]) / P)[:, None, :].expand(n, P, C).contiguous()
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    assert pb.group_norm_backward(d["maps"], dy, d["gamma"], d["beta"], mean, rstd, None, dgamma, dbeta, G, work["room"], activation=pb.ACT_RELU) == pb.OK
    assert torch.equal(last, h[-1])
    return float(loss), [dgamma, dbeta, dw, db]


def test_a_training_step_of_a_network_with_a_memory():
    restart, net, work = terminals(), Net(3), {}
    tf32 = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        loss, grads = by_the_library(net, restart, work)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = tf32
    want_loss, want = by_autograd(net, restart.cpu())
    # Every sum here has at most T N P = 7,840 terms; pairwise or in blocks no element passes more than some 200 additions, and what a gradient is
    # made of passes a dozen such sums or roundings one after the other: 2400 u, of the largest element.
    for got, exact in zip(grads, want):
        exact = exact.numpy()
        assert np.abs(got.double().cpu().numpy() - exact).max() <= 4000 * U * np.abs(exact).max()
    assert abs(loss - want_loss) <= 400 * U * want_loss

    # clipped into one vector, which the optimiser takes; and the same in 64 bits
    theta = torch.cat([p.reshape(-1) for p in net.params()]).cuda()
    flat, rms, told = torch.zeros_like(theta), torch.zeros_like(theta), torch.zeros(2, device="cuda")
    places, at = [], 0
    for g in grads:
        places.append(flat[at:at + g.numel()])
        at += g.numel()
    before = theta.double()
    assert pb.clip_tensors(pb.TensorList([g.reshape(-1) for g in grads], places), CLIP, norm_and_scale=told) == pb.OK
    assert pb.clip_rmsprop_noalloc(theta, rms, flat, theta.numel(), LR, DECAY, EPS, 0.0, stream=torch.cuda.current_stream().cuda_stream) == pb.OK
    torch.cuda.synchronize()
    every = torch.cat([g.reshape(-1) for g in grads]).double()
    norm = float(every.norm())
    scale = min(1.0, CLIP / norm)
    assert scale < 1.0 and abs(float(told[0]) - norm) <= 17 * U * norm and abs(float(told[1]) - scale) <= 19 * U * scale
    m = (1 - DECAY) * (scale * every) ** 2
    step = LR * scale * every / (m + EPS).sqrt()
    assert float((theta.double() - (before - step)).abs().max()) <= 1e-6 * float(step.abs().max()) + U * float(before.abs().max()) * 2


def test_the_whole_run_recorded_beside_eager_calls():
    """norm, memory, the way back and clipping in one graph, replayed on a stream of its own while the same calls run eagerly elsewhere, each with
    buffers of its own: the same bits."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    restart = (torch.rand(T, N, device="cuda", generator=gen) < 0.2).to(torch.uint8)

    def fresh():
        b = dict(maps=torch.zeros(N * T, P, C, device="cuda", dtype=torch.bfloat16), y=torch.empty(N * T, P, C, device="cuda", dtype=torch.bfloat16))
        b.update(dx=torch.empty_like(b["y"]), mean=torch.empty(N * T, G, device="cuda"), rstd=torch.empty(N * T, G, device="cuda"),
                 dgamma=torch.empty(C, device="cuda"), dbeta=torch.empty(C, device="cuda"), h=torch.empty(T, N, P * C, device="cuda", dtype=torch.bfloat16),
                 dgate=torch.empty(T, N, P * C, device="cuda", dtype=torch.bfloat16), out=torch.empty(N * T * P * C + 2 * C, device="cuda"),
                 told=torch.zeros(2, device="cuda"), gamma=torch.ones(C, device="cuda"), beta=torch.zeros(C, device="cuda"),
                 room=torch.empty(pb.group_norm_workspace_bytes(N * T, P, C, G, pb.BF16), dtype=torch.uint8, device="cuda"))
        n = N * T * P * C
        b["list"] = pb.TensorList([b["dx"].view(-1), b["dgamma"], b["dbeta"]], [b["out"][:n], b["out"][n:n + C], b["out"][n + C:]])
        return b

    def run(b):
        assert pb.group_norm(b["maps"], b["gamma"], b["beta"], b["y"], b["mean"], b["rstd"], G, b["room"], activation=pb.ACT_SILU) == pb.OK
        steps = b["y"].view(T, N, P * C)
        assert pb.gated_scan(steps, steps, b["h"], restart=restart) == pb.OK
        dx = torch.empty_like(b["h"])
        assert pb.gated_scan_backward(steps, steps, b["h"], b["h"], b["dgate"], dx, restart=restart) == pb.OK
        assert pb.group_norm_backward(b["maps"], dx.view(N * T, P, C), b["gamma"], b["beta"], b["mean"], b["rstd"], b["dx"], b["dgamma"], b["dbeta"], G,
                                      b["room"], activation=pb.ACT_SILU) == pb.OK
        assert pb.clip_tensors(b["list"], 1.0, norm_and_scale=b["told"]) == pb.OK

    recorded, eager = fresh(), fresh()
    for b in (recorded, eager):
        run(b)                                              # (maps are 0: what has to be looked up has been)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(recorded)
    side = torch.cuda.Stream()
    for k in range(4):
        maps = torch.randn(N * T, P, C, device="cuda", generator=gen)
        recorded["maps"].copy_(maps)
        eager["maps"].copy_(maps)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        run(eager)
        torch.cuda.synchronize()
        for name in ("y", "h", "dgate", "dx", "dgamma", "dbeta", "out", "told"):
            assert torch.equal(recorded[name], eager[name]), name
        assert float(eager["told"][0]) > 0


def test_two_threads_at_once():
    """Two host threads, a stream, buffers and scratch each, calling all of them side by side: the same bits as one after the other."""
    import threading

    def inputs(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        def r(*shape, dtype=torch.bfloat16): return torch.randn(*shape, device="cuda", generator=gen).to(dtype)
        return dict(maps=r(48, 100, 32), dy=r(48, 100, 32), gate=r(300, 6, 40), x=r(300, 6, 40), dh=r(300, 6, 40), src=[r(90_001, dtype=torch.float32), r(64)])

    def outputs(i):
        o = {k: torch.zeros_like(i[k]) for k in ("maps", "dy", "gate", "x", "dh")}
        o["stats"], o["told"] = torch.zeros(2, 48, 4, device="cuda"), torch.zeros(2, device="cuda")
        o["dgamma"], o["dbeta"] = torch.zeros(2, 32, device="cuda")
        o["dst"] = [torch.zeros_like(s) for s in i["src"]]
        o["room"] = torch.zeros(pb.group_norm_workspace_bytes(48, 100, 32, 4, pb.BF16), dtype=torch.uint8, device="cuda")
        o["list"] = pb.TensorList(i["src"], o["dst"])
        return o

    def run(i, o, status):
        mean, rstd = o["stats"]
        status += [pb.group_norm(i["maps"], None, None, o["maps"], mean, rstd, 4, o["room"], pb.ACT_SILU),
                   pb.group_norm_backward(i["maps"], i["dy"], None, None, mean, rstd, o["dy"], o["dgamma"], o["dbeta"], 4, o["room"], pb.ACT_SILU),
                   pb.gated_scan(i["gate"], i["x"], o["x"]),
                   pb.gated_scan_backward(i["gate"], i["x"], o["x"], i["dh"], o["gate"], o["dh"]),
                   pb.clip_tensors(o["list"], 0.5, o["told"])]

    def told(o): return [o[k].clone() for k in ("maps", "dy", "gate", "x", "dh", "stats", "dgamma", "dbeta", "told")] + [d.clone() for d in o["dst"]]
    sets = [(i, outputs(i)) for i in (inputs(1), inputs(2))]
    wants = []
    for i, o in sets:
        status = []
        run(i, o, status)
        assert status == [pb.OK] * 5
        wants.append(told(o))
        for k in ("maps", "dy", "gate", "x", "dh", "stats", "dgamma", "dbeta", "told"):
            o[k].zero_()
    torch.cuda.synchronize()
    status = [[], []]

    def thread(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                run(*sets[k], status[k])
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=thread, args=(k,)) for k in range(2)]
    for t in threads: t.start()
    for t in threads: t.join()
    assert status == [[pb.OK] * 100] * 2
    for (_, o), want in zip(sets, wants):
        for got, w in zip(told(o), want):
            assert torch.equal(got, w)


FIRST_CALLS = """
import sys
import torch
from paper_1705_04862_b200 import binding as pb

def inputs(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(s, device="cuda", generator=gen) for s in ((600, 4, 40), (20, 60, 32), (2, 20000, 16), (100,), (90000,))]

steps, maps, large, small, many = inputs(1)
out = [torch.zeros_like(v) for v in (steps, steps, steps, maps, maps, large, large, small, many)]
stats, sums = torch.zeros(2, 2, 20, 4, device="cuda"), torch.zeros(4, 32, device="cuda")
rooms = [torch.empty(pb.group_norm_workspace_bytes(n, p, c, g, pb.FP32), dtype=torch.uint8, device="cuda") for n, p, c, g in ((20, 60, 32, 4), (2, 20000, 16, 4))]
lists = [pb.TensorList([small], [out[7]]), pb.TensorList([many], [out[8]])]
told = torch.zeros(2, 2, device="cuda")

def run():
    ok = [pb.gated_scan(steps, steps, out[0]), pb.gated_scan_backward(steps, steps, out[0], steps, out[1], out[2])]
    for x, y, dx, g, st, sm, room in ((maps, out[3], out[4], 4, stats[0], sums[:2], rooms[0]), (large, out[5], out[6], 4, stats[1][:, :2], sums[2:, :16], rooms[1])):
        ok += [pb.group_norm(x, None, None, y, st[0], st[1], g, room, activation=pb.ACT_SILU),
               pb.group_norm_backward(x, x, None, None, st[0], st[1], dx, sm[0], sm[1], g, room, activation=pb.ACT_SILU)]
    ok += [pb.clip_tensors(l, 1.0, t) for l, t in zip(lists, told)]
    assert ok == [pb.OK] * 8, ok

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run()                                   # the first calls of the process
for v, w in zip((steps, maps, large, small, many), inputs(2)):
    v.copy_(w)
graph.replay()
torch.cuda.synchronize()
results = out + [stats, sums, told]
got = [v.clone() for v in results]
for v in results:
    v.zero_()
run()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, results))
assert all(float(v.abs().sum()) > 0 for v in results)
print("same")
"""


def test_the_first_calls_of_a_process_recorded():
    """What is looked up once on a device may be looked up while a graph is recorded."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, env=dict(os.environ, PYTHONPATH=root), capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.strip() == "same", done.stdout + done.stderr
