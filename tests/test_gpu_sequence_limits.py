"""The operators over sequences and the draws where their settings, states and sizes end: what the files by operator do not reach."""
import numpy as np
import pytest
import torch

from operators_ref import U
from paper_1705_04862_b200 import binding as pb
from test_gpu_selective_scan import backward, case, forward, room

pytestmark = pytest.mark.gpu
F, H = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("how", [{}, dict(top_k=40), dict(top_p=0.9), dict(top_k=40, top_p=0.9), dict(temperature=0.5)])
@pytest.mark.parametrize("v", [6, 1000, 50_001, 131_072])
def test_a_min_p_above_one_leaves_the_first_alone(v, how, dtype):
    """No action is more likely than the first, not even one that is as likely: equal ones stay for a min_p of 1, and none of them for the next float."""
    g = torch.Generator().manual_seed(v)
    logits = torch.randn(5, v, generator=g).clamp(max=1.0)
    ties = torch.tensor([1, 2, v // 2 + 1, v - 1])
    logits[:, ties] = 8.0
    logits, u = logits.to(dtype).cuda(), torch.tensor([0.0, 0.3, 0.6, 0.9, 0.9999], device="cuda")
    count = ties.unique().numel()
    settings = {name: torch.full((5,), x, device="cuda", dtype=torch.int32 if name == "top_k" else F) for name, x in how.items()}
    for least, stay in ((1.0, count), (1 + 2.0 ** -23, 1), (2.0, 1), (float("inf"), 1)):
        actions, logprob = torch.empty(5, dtype=torch.int32, device="cuda"), torch.empty(5, device="cuda")
        assert pb.sample(logits, u, actions, logprob=logprob, min_p=torch.full((5,), least, device="cuda"), **settings) == pb.OK
        if stay == 1:
            assert actions.tolist() == [1] * 5 and logprob.tolist() == [0.0] * 5
        elif "top_p" not in how:
            assert actions.tolist() == [int(ties.unique()[int(x * count)]) for x in u.tolist()]
            assert (logprob + np.log(count)).abs().max() <= U * np.log(count) + 1e-9


def infinite(shape):
    """Where the tests below have an infinity, and of which sign."""
    at = torch.zeros(shape, device="cuda")
    at[0, 5, 3], at[0, 7, 0], at[0, 23, 15] = 1.0, -1.0, 1.0
    return at


@pytest.mark.parametrize("t", [40, 700])
def test_an_infinite_state_stays_one_where_parts_decay_it_to_nothing(t):
    """Every step's decay is e^-4, that of a part of 32 steps or more below any float: the steps one by one keep an infinity, and so do the parts (of 700 steps)."""
    k = case(t, 1, 24, 16, F, restart=0, plain=True, softplus=False)
    k["dt"].fill_(1.0)
    k["A"].fill_(-4.0)
    assert (room(k, False).numel() > 0) == (t == 700)
    last, states = forward(k)
    clean = {name: v.clone() for name, v in backward(k, states).items()}
    at = infinite(last.shape)
    for value in (float("inf"), float("nan")):
        h0, dh_last = k["h0"], k["dh_last"]
        k["h0"], k["dh_last"] = (torch.where(at == 0, v, at * value) for v in (h0, dh_last))
        assert torch.equal(torch.nan_to_num(forward(k)[0], 7.0), torch.nan_to_num(torch.where(at == 0, last, at * value), 7.0))
        assert torch.equal(torch.nan_to_num(backward(k, states)["dh0"], 7.0), torch.nan_to_num(torch.where(at == 0, clean["dh0"], at * value), 7.0))
        k["h0"], k["dh_last"] = h0, dh_last
