"""Draws of an action out of many (paac_sample) against sorting in 64 bits."""
import threading

import numpy as np
import pytest
import torch

from operators_ref import U
from paper_1705_04862_b200 import binding as pb
from sequence_ref import draw

pytestmark = pytest.mark.gpu
F, H = torch.float32, torch.bfloat16


def off(v):
    """How far the two sides of a comparison may be from each other, with the likeliest action's share as 1: each of v shares is off by half of 2^-b, b the
    header's, on both sides, and by 2^-44 of its value."""
    return v * 2.0 ** -min(50, 62 - int(np.ceil(np.log2(v)))) + v * 2.0 ** -44


def beside(row, u, allowed, top_p=1.0, **how):
    """All that a row at a border may answer: top_p's border and u's moved by what both sides may be off, which is less in parts of a sum of 1 or more."""
    d = off(row.size)
    p = {top_p} if top_p >= 1 else {top_p, top_p - d, min(top_p + d, 1 - 2.0 ** -53)}
    return [draw(row, u + e, allowed=allowed, top_p=q, exact_u=True, **how)[:2] for q in p for e in (-d, 0, d)]


def check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, allowed=None, borders=False):
    """Tensors on the device, or None; every row against the reference.  `borders`: rows so near to one that roundings may answer either way are among them."""
    n, v = logits.shape
    actions, logprob = torch.full((n,), 77, dtype=torch.int32, device="cuda"), torch.full((n,), 77.0, device="cuda")
    assert pb.sample(logits, u, actions, logprob=logprob, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, allowed=allowed) == pb.OK
    host = [None if t is None else t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy() for t in (logits, u, temperature, top_k, top_p, min_p, allowed)]
    got, lp = actions.cpu().numpy(), logprob.double().cpu().numpy()
    for r in range(n):
        how = {name: h[r].item() for name, h in zip(("temperature", "top_k", "top_p", "min_p"), host[2:6]) if h is not None}
        how = {name: x for name, x in how.items() if name == "temperature" or not np.isnan(x)}
        mask = None if host[6] is None else host[6][r]
        want, p, near = draw(host[0][r], host[1][r], allowed=mask, **how)
        answers = [(want, p)]
        if near <= off(v):
            assert borders, "an input at a border"
            answers += beside(host[0][r], host[1][r].item(), mask, **how)
        assert got[r] in [a for a, _ in answers], (r, got[r], want, how)
        if np.isfinite(p):
            assert any(got[r] == a and abs(lp[r] - q) <= U * abs(q) + 1e-9 for a, q in answers), (r, lp[r], answers)
        else:
            assert np.array_equal(lp[r], p, equal_nan=True), (r, lp[r], p)
    return actions, logprob


def some(n, v, dtype=F, spread=3.0, seed=0):
    g = torch.Generator().manual_seed(seed + n + v)
    return (spread * torch.randn(n, v, generator=g)).to(dtype).cuda(), torch.rand(n, generator=g).cuda(), g


def settings(n, g, which="tkpm"):
    def rand():
        return torch.rand(n, generator=g)
    out = {}
    if "t" in which:
        out["temperature"] = torch.where(rand() < 0.2, torch.zeros(n), 0.3 + 1.5 * rand()).cuda()
    if "k" in which:
        out["top_k"] = torch.where(rand() < 0.3, torch.zeros(n), 1 + 60 * rand()).to(torch.int32).cuda()
    if "p" in which:
        out["top_p"] = torch.where(rand() < 0.3, torch.ones(n), rand()).cuda()
    if "m" in which:
        out["min_p"] = torch.where(rand() < 0.3, torch.zeros(n), 0.3 * rand()).cuda()
    return out


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("v", [1, 2, 3, 7, 32, 33, 255, 256, 257, 1000, 4096, 5003, 40_000])
@pytest.mark.parametrize("which", ["", "t", "k", "p", "m", "tkpm"])
def test_sizes_and_filters(v, which, dtype):
    logits, u, g = some(24, v, dtype)
    check(logits, u, **settings(24, g, which))


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("n,v", [(1, 131_072), (3, 200_003), (200, 20_000), (300, 3000), (1, 2_000_003), (1, 1 << 21)])
def test_large(n, v, dtype):
    logits, u, g = some(n, v, dtype)
    check(logits, u, **settings(n, g, "tp"))
    check(logits, u, **settings(n, g, "k"))


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("spread", [0.0, 1e-3, 30.0])
def test_flat_and_steep(spread, dtype):
    logits, u, g = some(16, 3001, dtype, spread=spread)
    for which in ("", "t", "k", "p", "m", "tkpm"):
        check(logits, u, **settings(16, g, which))


@pytest.mark.parametrize("top_k", [1, 2, 5, 100, 3000, 5000])
def test_ties_go_to_the_lower_index(top_k):
    """Few different logits, so that the border of every filter lies among equal ones."""
    g = torch.Generator().manual_seed(top_k)
    logits, u = torch.randint(0, 3, (40, 3000), generator=g).float().cuda(), torch.rand(40, generator=g).cuda()
    k = torch.full((40,), top_k, dtype=torch.int32, device="cuda")
    check(logits, u, top_k=k)
    check(logits, u, top_k=k, top_p=torch.rand(40, generator=g).cuda())
    check(logits.to(H), u, top_p=torch.rand(40, generator=g).cuda())
    zero = torch.zeros(40, device="cuda")
    actions, logprob = check(logits, u, temperature=zero)
    assert torch.equal(actions.long(), logits.argmax(1)) and (logprob == 0).all()


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("share", [0.5, 0.01, 0.0])
@pytest.mark.parametrize("v", [5, 1000, 1001, 30_000])
def test_actions_that_are_not_allowed(v, share, dtype):
    logits, u, g = some(20, v, dtype)
    allowed = (torch.rand(20, v, generator=g) < share).to(torch.uint8) * 5
    allowed[3] = 0
    allowed = allowed.cuda()
    logits[allowed == 0] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device="cuda").to(dtype)[torch.arange(int((allowed == 0).sum()), device="cuda") % 4]
    check(logits, u, allowed=allowed, **settings(20, g))
    actions, logprob = check(logits, u, allowed=allowed)
    assert int(actions[3]) == -1 and float(logprob[3]) == -np.inf


def test_the_uniforms_ends():
    logits, _, _ = some(6, 500)
    u = torch.tensor([0.0, -1.0, float("nan"), 1.0, 2.0, 1 - 2.0 ** -24], device="cuda")
    actions, _ = check(logits, u)
    for r in range(3):
        assert int(actions[r]) == 0                   # every share is large enough here
    k = torch.full((6,), 1, dtype=torch.int32, device="cuda")
    actions, logprob = check(logits, u, top_k=k)
    assert torch.equal(actions.long(), logits.argmax(1)) and (logprob == 0).all()


def test_settings_at_their_ends():
    logits, u, _ = some(12, 700)
    nan = float("nan")
    check(logits, u, temperature=torch.tensor([nan, float("inf"), 1e-30, 1e-45, -1.0, -0.0, 1e30, 1.0, 0.01, 100.0, nan, -float("inf")], device="cuda"))
    check(logits, u, top_k=torch.tensor([-5, 0, 1, 699, 700, 701, 2 ** 31 - 1, -2 ** 31, 2, 3, 4, 5], dtype=torch.int32, device="cuda"))
    check(logits, u, top_p=torch.tensor([nan, 0.0, -1.0, 1.0, 2.0, 1e-30, 0.999999, float("inf"), -float("inf"), 0.5, 1e-3, 0.1], device="cuda"))
    check(logits, u, min_p=torch.tensor([nan, 0.0, -1.0, 1.0, 2.0, 1e-30, 0.999999, float("inf"), -float("inf"), 0.5, 1e-3, 0.1], device="cuda"))


def test_rows_that_hold_no_number():
    logits, u, _ = some(8, 300)
    logits[1, 7] = float("nan")
    logits[2, 299] = float("inf")
    logits[3, :] = -float("inf")
    logits[4, 1:] = -float("inf")
    logits[5, 0] = -float("nan")
    logits[6] = -logits[6].abs()
    logits[7, ::2] = -0.0
    logits[7, 1::2] = 0.0
    for how in ({}, dict(top_k=torch.full((8,), 5, dtype=torch.int32, device="cuda")), dict(top_p=torch.full((8,), 0.3, device="cuda")), dict(temperature=torch.zeros(8, device="cuda"))):
        actions, logprob = check(logits, u, **how)
        assert actions[1:4].tolist() == [-1, -1, -1] and int(actions[4]) == 0 and int(actions[5]) == -1
    assert int(check(logits, u, temperature=torch.zeros(8, device="cuda"))[0][7]) == 0      # -0 is 0


def test_far_apart():
    """Logits whose difference is more than a float holds, and ones next to each other."""
    logits = torch.zeros(4, 64, device="cuda")
    logits[0, 5], logits[0, 6] = 3e38, -3e38
    logits[1] = torch.linspace(-3e38, 3e38, 64)
    logits[2] = 1e30
    logits[2, 9] = 1.0000001e30
    logits[3] = torch.arange(64) * 1e-40
    u = torch.tensor([0.3, 0.9, 0.5, 0.6], device="cuda")
    for how in ({}, dict(top_p=torch.full((4,), 0.5, device="cuda")), dict(top_k=torch.full((4,), 7, dtype=torch.int32, device="cuda")),
                dict(temperature=torch.full((4,), 1e38, device="cuda"), top_p=torch.full((4,), 0.7, device="cuda"))):
        check(logits, u, **how)


@pytest.mark.parametrize("dtype", [F, H])
def test_rows_apart_and_at_odd_places(dtype):
    whole, u, g = some(9, 1100, dtype)
    mask = (torch.rand(9, 1100, generator=g) < 0.6).to(torch.uint8).cuda()
    for cut in (slice(0, 1000), slice(1, 1001), slice(8, 1008), slice(3, 500)):
        check(whole[:, cut], u, allowed=mask[:, cut], **settings(9, g))
        check(whole[::2, cut], u[::2].contiguous(), **settings(5, g))
    check(whole[:1].expand(9, 1100), u, **settings(9, g))          # the same row for all


def test_frequencies():
    """65,536 even uniforms over one row draw every action as often as its share says, to one."""
    logits, _, _ = some(1, 50)
    n = 65_536
    u = (torch.arange(n, device="cuda").float() + 0.5) / n
    actions = torch.empty(n, dtype=torch.int32, device="cuda")
    assert pb.sample(logits.expand(n, 50), u, actions) == pb.OK
    got = torch.bincount(actions.long(), minlength=50).double().cpu()
    want = torch.softmax(logits[0].double(), 0).cpu() * n
    assert float((got - want).abs().max()) <= 1.0


def test_recorded_on_other_streams_and_from_two_threads():
    logits, u, g = some(40, 9000)
    how = settings(40, g)
    want, want_lp = check(logits, u, **how)
    graph, actions, lp = torch.cuda.CUDAGraph(), torch.empty_like(want), torch.empty_like(want_lp)
    with torch.cuda.graph(graph):
        assert pb.sample(logits, u, actions, logprob=lp, **how) == pb.OK
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(actions, want) and torch.equal(lp, want_lp)
    logits.copy_(-logits)
    graph.replay()
    torch.cuda.synchronize()
    got = actions.clone(), lp.clone()
    fresh = check(logits, u, **how)
    assert torch.equal(got[0], fresh[0]) and torch.equal(got[1], fresh[1])
    outs = [[], []]

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                a = torch.empty_like(want)
                assert pb.sample(logits, u, a, **how) == pb.OK
                outs[i].append(a)
            stream.synchronize()

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert len(outs[0]) == len(outs[1]) == 20
    assert all(torch.equal(a, fresh[0]) for a in outs[0] + outs[1])


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("v", [20_000, 131_072, 70_001])
def test_more_ties_than_are_put_in_order(v, dtype):
    """Rows of few different logits, whose borders lie among thousands of equal ones."""
    g = torch.Generator().manual_seed(v)
    logits, u = torch.randint(0, 3, (12, v), generator=g).to(dtype).cuda(), torch.rand(12, generator=g).cuda()
    logits[5:8] = 0.25
    logits[8:10, ::7] = -3.0
    k = torch.tensor([1, 2, 50, 5000, v // 3 + 7, 1, 300, v - 1, 9000, 40, 6000, 4096], dtype=torch.int32, device="cuda")
    p = torch.rand(12, generator=g).cuda()
    check(logits, u, top_k=k)
    check(logits, u, top_p=p)
    check(logits, u, top_k=k, top_p=p, min_p=torch.full((12,), 0.3, device="cuda"))
    mask = (torch.rand(12, v, generator=g) < 0.5).to(torch.uint8).cuda()
    check(logits, u, top_k=k, top_p=p, allowed=mask)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("spread", [1e-3, 0.5, 3.0])
@pytest.mark.parametrize("v", [50_000, 131_072])
def test_borders_with_many_beside_them(v, spread, dtype):
    """top-p where thousands lie as near to its border as coarse distances tell apart, and settings that keep nearly all."""
    logits, u, g = some(10, v, dtype, spread=spread)
    t = torch.tensor([0.7, 0.9, 1.0, 1.1, 1.2, 1.3, 1.5, 2.0, 5.0, 0.05], device="cuda")
    p = torch.tensor([0.9, 0.95, 0.97, 0.975, 0.98, 0.99, 0.995, 0.999, 0.5, 0.99999], device="cuda")
    check(logits, u, temperature=t, top_p=p, borders=True)
    check(logits, u, temperature=t.flip(0), top_p=p, borders=True)
    check(logits, u, temperature=t, top_p=p, top_k=torch.full((10,), 30_000, dtype=torch.int32, device="cuda"), borders=True)
    check(logits, u, temperature=t, top_k=torch.tensor([600, 1000, 2000, 4000, 5000, 10_000, 1, 255, 256, 257], dtype=torch.int32, device="cuda"), borders=True)


def test_many_rows_of_few_actions():
    logits, u, g = some(20_000, 6)
    check(logits, u, **settings(20_000, g))


def test_rows_far_apart():
    """Rows whose places are beyond 32 bits."""
    whole = torch.empty(3 << 30, dtype=H, device="cuda")
    far = whole.as_strided((3, 3000), (1 << 30, 1))
    near, u, g = some(3, 3000, H)
    far.copy_(near)
    how = settings(3, g)
    a, b = check(far, u, **how)
    c, d = check(near, u, **how)
    assert torch.equal(a, c) and torch.equal(b, d)
