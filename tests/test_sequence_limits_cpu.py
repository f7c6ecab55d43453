"""The operators over sequences and the draws: refusals at the ends of what their arguments may be, and what their sources have to say.  No device."""
import os
import re

import pytest
import torch

from paper_1705_04862_b200 import binding as pb
from test_operators_cpu import CSRC, F, H
from test_sequence_operators_cpu import draw


class Like:
    """What the binding looks at of a contiguous tensor on a device."""
    def __init__(self, *shape, dtype=torch.float32):
        self.t = torch.empty(shape, dtype=dtype, device="meta")
        self.shape, self.dtype, self.nbytes = self.t.shape, dtype, self.t.nbytes
        for name in ("dim", "stride", "numel", "is_contiguous", "element_size"):
            setattr(self, name, getattr(self.t, name))
    def get_device(self): return 0
    def data_ptr(self): return 1 << 20


def test_tensors_of_another_rank_are_refused(monkeypatch):
    """A tensor with less or more axes than is said, or None for one that is needed, is the status of a bad argument like any other, not an exception."""
    byte, calls = torch.uint8, []
    monkeypatch.setattr(pb, "_status", lambda *a: calls.append(a) or pb.OK)
    x, w, b, a, work = Like(3, 2, 8), Like(8, 4), Like(3, 2, 1, 4), Like(8, 4), Like(1 << 16, dtype=byte)
    marks, flags = Like(1, 2, 8, 4), Like(3, 2, dtype=byte)
    assert pb.causal_conv(x, w, None, x, restart=flags) == pb.causal_conv_backward(x, x, w, None, x, w, None, work) == pb.OK
    assert pb.selective_scan(x, x, a, b, b, x, work, restart=flags) == pb.selective_scan_backward(x, x, a, b, b, x, marks, x, x, a, b, b, work) == pb.OK
    assert len(calls) == 4
    for wrong in (Like(6, 8), Like(48), Like(3, 2, 8, 1), Like()):
        assert pb.causal_conv(x, w, None, wrong) == pb.causal_conv(wrong, w, None, x) == pb.causal_conv(x, wrong, None, x) == pb.ERR_ARG
        assert pb.causal_conv(x, w, None, x, restart=wrong) == pb.causal_conv(x, w, None, x, before=wrong) == pb.ERR_ARG
        assert pb.causal_conv_backward(x, wrong, w, None, x, w, None, work) == pb.causal_conv_backward(x, x, w, None, wrong, w, None, work) == pb.ERR_ARG
        for i in range(6):
            args = [x, x, a, b, b, x]
            args[i] = wrong
            assert pb.selective_scan(*args, work) == pb.ERR_ARG, i
        assert pb.selective_scan(x, x, a, b, b, x, work, z=wrong) == pb.selective_scan(x, x, a, b, b, x, work, restart=wrong) == pb.ERR_ARG
        for i in (5, 7, 8, 10, 11):
            args = [x, x, a, b, b, x, marks, x, x, a, b, b, work]
            args[i] = wrong
            assert pb.selective_scan_backward(*args) == pb.ERR_ARG, i
    row, whole = Like(3), Like(3, dtype=torch.int32)
    assert pb.sample(Like(3, 5), row, whole, allowed=Like(3, 5, dtype=byte)) == pb.OK and len(calls) == 5
    for wrong in (Like(15, dtype=byte), Like(3, 5, 1, dtype=byte), Like(dtype=byte)):
        assert pb.sample(Like(3, 5), row, whole, allowed=wrong) == pb.ERR_ARG
    for wrong in (Like(15), Like(3, 5, 1), Like()):
        assert pb.sample(wrong, row, whole) == pb.sample(Like(3, 5), wrong, whole) == pb.sample(Like(3, 5), row, wrong) == pb.ERR_ARG
    assert pb.causal_conv(x, None, None, x) == pb.selective_scan(x, x, None, b, b, x, work) == pb.selective_scan(x, x, a, None, b, x, work) == pb.ERR_ARG
    assert len(calls) == 5


def test_shared_arrays_that_are_read_sixteen_bytes_at_a_time_begin_on_sixteen():
    """B and C of a step lie in shared memory and are read in pairs of pairs of floats: an array of floats alone promises four bytes."""
    seen = 0
    for name in ("selective_scan.cu", "selective_scan_back.cu"):
        for declaration in re.findall(r"__shared__[^;]*;", open(os.path.join(CSRC, name)).read()):
            if re.search(r"\bfloat\b", declaration):
                seen += 1
                assert "__align__(16)" in declaration, (name, declaration)
    assert seen == 2


@pytest.mark.parametrize("type,v", [(F, 65_537), (H, 131_073), (F, 1 << 23)])
def test_more_rows_than_a_grid_has_blocks_for(type, v):
    """2^28 rows, all of them one row of logits in memory, with eight blocks each: 2^31 blocks."""
    far = dict(logits=1 << 40, uniforms=2 << 40, actions=3 << 40, logprobs=4 << 40)
    assert draw(n=1 << 28, v=v, type=type, row=0, **far) == pb.ERR_ARG
