"""The operators over sequences and the draws where their settings, states and sizes end: what the files by operator do not reach."""
import numpy as np
import pytest
import torch

from operators_ref import U
from paper_1705_04862_b200 import binding as pb
from test_gpu_causal_conv import check as check_conv
from test_gpu_selective_scan import backward, case, check, forward, room

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


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c,state", [(1, 3, 20, 64), (1, 5, 33, 33), (2, 2, 9, 40), (8, 2, 9, 64), (5, 3, 18, 50), (9, 2, 12, 64), (16, 2, 7, 50)])
def test_few_steps_of_many_states(t, n, c, state, dtype):
    """Up to 16 steps, and backward up to 8, of more states than four lanes hold: forms of their own."""
    check(t, n, c, state, dtype)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("t,n,c,state", [(20, 600, 64, 16), (37, 296, 67, 16), (37, 200, 64, 16), (18, 200, 35, 16), (33, 400, 8, 64), (21, 640, 100, 3)])
def test_sequences_that_fill_the_device(t, n, c, state, dtype):
    """More than 16 steps that are not cut, since the warps with eight states a thread (the first, second and last) or with four are enough: no scratch, and the state
    replaced by the block that read it."""
    k = check(t, n, c, state, dtype)
    assert room(k, False).numel() == 0
    last, _ = forward(k, marks=False)
    y, h = k["y"].clone(), k["h0"].clone()
    assert pb.selective_scan(k["x"], k["dt"], k["A"], k["B"], k["C"], k["y"], None, D=k["D"], z=k["z"], dt_bias=k["bias"], h0=h, h_last=h, restart=k["restart"]) == pb.OK
    assert torch.equal(h, last) and torch.equal(y, k["y"])


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("width", [2, 4])
def test_a_column_of_more_parts_than_a_grid_has_rows(width, dtype):
    """1.1 million steps of one channel: parts of 16 steps would be 68,751 rows of blocks."""
    check_conv(1_100_003, 1, 1, width, dtype, restart=0.01)
