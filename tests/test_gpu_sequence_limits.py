"""The operators over sequences and the draws where their settings, states and sizes end: what the files by operator do not reach."""
import numpy as np
import pytest
import torch

from operators_ref import U
from paper_1705_04862_b200 import binding as pb

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
