"""The operators for a caller's own network: what can be said without a device.  Their refusals, the rules on rows, and the references that
the GPU tests hold the kernels to, against differences."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import operators_ref as ref
from paper_1705_04862_b200 import binding as pb

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1705_04862_b200", "csrc")
A = 1 << 20          # addresses that nothing is read from: every call below is refused before that
NONE = pb.Rows(None, 0, 0)


def test_struct_layouts_match_the_header():
    assert C.sizeof(pb.Rows) == 24 and C.sizeof(pb.Tensor) == 32 and pb.Tensor.src_type.offset == 24
    assert C.sizeof(pb.Scan) == 48 and pb.Scan.restart.offset == 24 and C.sizeof(pb.Norm) == 28


def clip(tensors, clip_norm=1.0, norm=0, workspace=A, room=1 << 30, count=None):
    arr = (pb.Tensor * max(1, len(tensors)))(*[pb.Tensor(*t) for t in tensors])
    return pb.lib().paac_clip_tensors(arr, len(tensors) if count is None else count, clip_norm, norm, workspace, room, None)


F, H = pb.FP32, pb.BF16


@pytest.mark.parametrize("tensors", [
    [(None, A, 4, F, F)],                                     # no src
    [(A + 2, None, 4, F, F)], [(A + 1, None, 4, H, H)],          # not aligned to their elements
    [(A, A + 4096 + 1, 4, H, H)], [(A, A + 4096 + 2, 4, F, F)],
    [(A, None, 4, 2, F)], [(A, None, 4, F, -1)],                # no such type
    [(A, A, 4, F, H)],                                        # in place, another type
    [(A, A + 8, 4, F, F)],                                    # dst inside its own src
    [(A, A, 8, F, F), (A, A, 8, F, F)],                         # the same tensor twice in place
    [(A, A, 8, F, F), (A + 16, None, 2, F, F)],                 # another one's dst
    [(A + 64, A + 4096, 8, F, F), (A, A + 4096 + 28, 8, F, F)],   # two dsts
    [(A, A + 4096, 8, F, F), (A + 4096 + 31, None, 1, H, H)],     # src inside a dst, misaligned as well
    [(A, None, 1 << 60, F, F)], [(A, None, 1 << 43, F, F)] * 2,   # more than there can be
])
def test_clip_refuses(tensors):
    assert clip(tensors) == pb.ERR_ARG


def test_clip_refuses_the_rest():
    one = [(A, A + 4096, 8, F, F)]
    assert clip(one, clip_norm=float("nan")) == pb.ERR_ARG and clip(one, norm=A + 2) == pb.ERR_ARG
    assert clip(one, workspace=None) == pb.ERR_WORKSPACE and clip(one, workspace=A + 8) == pb.ERR_WORKSPACE
    need = pb.lib().paac_clip_tensors_workspace_bytes(1)
    assert need > 0 and clip(one, room=need - 1) == pb.ERR_WORKSPACE
    assert pb.lib().paac_clip_tensors(None, 1, 1.0, None, A, 1 << 30, None) == pb.ERR_ARG
    assert clip(one, count=65537) == pb.ERR_LIMIT and pb.lib().paac_clip_tensors_workspace_bytes(65537) == 0
    assert pb.lib().paac_clip_tensors_workspace_bytes(65536) > pb.lib().paac_clip_tensors_workspace_bytes(1000)


def scan(backward=False, t=4, n=2, c=8, type=F, kind=pb.SCAN_SIGMOID, restart=None, **rows):
    """A call that would be fine but for what `rows` and the rest change; every array in a megabyte of its own."""
    s = pb.Scan(t, n, c, type, kind, 0, restart, 1, n)
    names = ["gate", "x", "h", "dh", "dgate", "dx"]
    r = {k: pb.Rows(A * (i + 1), c, n * c) for i, k in enumerate(names)}
    states = dict(h0=None, last=None, dh_last=None, dh0=None)
    for k, v in rows.items():
        (states if k in states else r)[k] = v
    if not backward:
        return pb.lib().paac_gated_scan(C.byref(s), r["gate"], r["x"], states["h0"], r["h"], states["last"], None)
    return pb.lib().paac_gated_scan_backward(C.byref(s), r["gate"], r["x"], r["h"], r["dh"], states["h0"], states["dh_last"], r["dgate"], r["dx"],
                                             states["dh0"], None)


@pytest.mark.parametrize("wrong", [
    dict(t=0), dict(n=0), dict(c=0), dict(t=-1), dict(t=(1 << 30) + 1, n=1, c=1), dict(n=1 << 20, c=1 << 12), dict(type=2), dict(kind=2), dict(kind=-1),
    dict(gate=NONE), dict(gate=pb.Rows(A + 2, 8, 16)), dict(type=H, gate=pb.Rows(A + 1, 8, 16)),
    dict(h=NONE), dict(h=pb.Rows(3 * A, 8, 15)), dict(h=pb.Rows(3 * A, 7, 16)), dict(h=pb.Rows(3 * A, 0, 16)), dict(h=pb.Rows(3 * A, 8, 0)),   # rows on one another
    dict(h=pb.Rows(A, 8, 16)), dict(h=pb.Rows(A + 32, 8, 16)), dict(h=pb.Rows(2 * A + 64, 8, 16)),                                      # on gate, on x
    dict(h0=A * 9 + 2), dict(last=A * 9 + 1), dict(last=3 * A + 64), dict(last=A), dict(h0=3 * A), dict(h0=9 * A, last=9 * A + 32),
    dict(gate=pb.Rows(A, 1 << 60, 16)), dict(restart=3 * A + 100), dict(gate=pb.Rows(A, -(1 << 40), 16)),
])
def test_scan_refuses(wrong):
    assert scan(**wrong) == pb.ERR_ARG


@pytest.mark.parametrize("wrong", [
    dict(x=NONE), dict(dh=NONE), dict(h=NONE), dict(dgate=NONE, dx=NONE), dict(dgate=pb.Rows(6 * A, 8, 16)), dict(dx=pb.Rows(4 * A, 8, 16)),
    dict(dgate=pb.Rows(A, 8, 16)), dict(dx=pb.Rows(3 * A + 64, 8, 16)), dict(dx=pb.Rows(6 * A, 4, 16)), dict(dh0=6 * A + 32), dict(dh0=9 * A, dh_last=9 * A + 4),
    dict(dh0=9 * A, h0=9 * A), dict(dgate=pb.Rows(5 * A, 16, 32), dx=pb.Rows(5 * A + 16, 16, 32)), dict(t=0), dict(kind=3),
])
def test_scan_backward_refuses(wrong):
    assert scan(True, **wrong) == pb.ERR_ARG


def norm(backward=False, n=3, pixels=10, c=8, groups=2, type=F, activation=0, eps=1e-5, workspace=A * 9, room=1 << 30, gamma=None, mean=A * 7, dgamma=None, **rows):
    s = pb.Norm(n, pixels, c, groups, type, activation, eps)
    r = {k: pb.Rows(A * (i + 1), pixels * c, c) for i, k in enumerate(["x", "dy", "out"])}
    r.update(rows)
    if not backward:
        return pb.lib().paac_group_norm(C.byref(s), r["x"], gamma, None, r["out"], mean, A * 8, workspace, room, None)
    return pb.lib().paac_group_norm_backward(C.byref(s), r["x"], r["dy"], gamma, None, mean, A * 8, r["out"], dgamma, None, workspace, room, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("wrong", [
    dict(n=0), dict(pixels=0), dict(c=0), dict(groups=0), dict(groups=3), dict(c=65540, groups=1), dict(n=1 << 20, pixels=1 << 12), dict(n=1 << 30, pixels=1),
    dict(type=3), dict(activation=3), dict(activation=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(gamma=A * 5 + 1), dict(mean=A * 7 + 2),
    dict(x=NONE), dict(x=pb.Rows(A + 1, 80, 8)), dict(out=pb.Rows(3 * A, 80, 7)), dict(out=pb.Rows(3 * A, 0, 8)), dict(out=pb.Rows(A + 320, 80, 8)),
    dict(out=pb.Rows(A, 88, 8)), dict(x=pb.Rows(A, 1 << 59, 8)),
])
def test_norm_refuses(wrong, backward):
    assert norm(backward, **wrong) == pb.ERR_ARG


def test_norm_refuses_the_rest():
    assert norm(True, out=NONE) == pb.ERR_ARG and norm(True, dy=NONE) == pb.ERR_ARG and norm(True, mean=None) == pb.ERR_ARG
    assert norm(True, out=pb.Rows(A, 80, 8)) == pb.ERR_ARG                           # dx is not x
    for backward in (False, True):
        assert norm(backward, workspace=None) == pb.ERR_WORKSPACE and norm(backward, workspace=A * 9 + 4) == pb.ERR_WORKSPACE
        assert norm(backward, room=pb.group_norm_workspace_bytes(3, 10, 8, 2, F) - 1) == pb.ERR_WORKSPACE
    assert pb.group_norm_workspace_bytes(3, 10, 8, 3, F) == 0 and pb.group_norm_workspace_bytes(5120, 400, 32, 4, H) < 64 << 20


def test_what_is_written_overlaps_nothing_else():
    """The norm and the factor, statistics, gradients of scale and shift, scratch: against the arrays of the call and one another."""
    one, far = [(A, 2 * A, 8, F, F), (3 * A, 3 * A, 8, F, F), (4 * A, None, 3, H, H)], dict(workspace=9 * A)
    for norm_at in (A + 28, 2 * A + 28, 3 * A, 4 * A + 4, 9 * A + 16):
        assert clip(one, norm=norm_at, **far) == pb.ERR_ARG
    for room_at in (A + 16, 2 * A + 16, 3 * A, 4 * A):
        assert clip(one, norm=8 * A, workspace=room_at) == pb.ERR_ARG
    assert clip([], norm=9 * A, workspace=9 * A) == pb.ERR_ARG
    # the last bytes of x, y, dy, dx (240 floats each), of mean and rstd (6 each)
    for backward in (False, True):
        assert norm(backward, workspace=A + 944) == pb.ERR_ARG and norm(backward, workspace=3 * A + 944) == pb.ERR_ARG
        assert norm(backward, workspace=A * 7) == pb.ERR_ARG and norm(backward, workspace=A * 8 + 16) == pb.ERR_ARG
        assert norm(backward, gamma=5 * A, workspace=5 * A + 16) == pb.ERR_ARG
    assert norm(mean=A + 956) == pb.ERR_ARG and norm(mean=3 * A + 956) == pb.ERR_ARG and norm(mean=8 * A + 20) == pb.ERR_ARG
    assert norm(gamma=7 * A) == pb.ERR_ARG                                           # that mean is written over
    assert norm(True, workspace=2 * A) == pb.ERR_ARG
    for dgamma in (A + 956, 2 * A + 956, 3 * A + 956, 7 * A + 20, 8 * A + 20, 9 * A):
        assert norm(True, dgamma=dgamma) == pb.ERR_ARG
    assert norm(True, gamma=5 * A, dgamma=5 * A + 28) == pb.ERR_ARG


def test_counts_beyond_32_bits_are_not_cut_off():
    """What a field of the library's structures cannot hold is refused, not passed on without its upper bits."""
    class Like:
        dtype = torch.float32
        def __init__(self, *shape): self.shape = torch.Size(shape)
        def get_device(self): return 0
        def is_contiguous(self): return True
    pb._scan(Like(2 ** 30, 1, 1), None, 0, False)
    for shape in ((2 ** 32 + 5, 1, 1), (5, 2 ** 32 + 1, 1), (5, 1, 2 ** 31)):
        with pytest.raises(pb._Apart):
            pb._scan(Like(*shape), None, 0, False)
    pb._norm(Like(2, 400, 8), 2, 0, 1e-5, Like(8))
    for shape in ((2 ** 32 + 5, 1, 1), (5, 2 ** 32 + 1, 1), (5, 1, 2 ** 32 + 1), (1, 2 ** 16, 2 ** 16 + 1, 1)):
        with pytest.raises(pb._Apart):
            pb._norm(Like(*shape), 1, 0, 1e-5, Like(8))


def test_settings_beyond_32_bits_are_not_cut_off():
    """The same for the numbers that are passed beside the tensors: 2^32 more than a number of groups, a kind or an activation is not that one."""
    class Like:
        dtype = torch.float32
        def __init__(self, *shape): self.shape = torch.Size(shape)
        def get_device(self): return 0
        def is_contiguous(self): return True
    maps, steps = Like(2, 400, 8), Like(4, 2, 8)
    pb._norm(maps, 2, pb.ACT_SILU, 1e-5, Like(8))
    pb._scan(steps, None, pb.SCAN_SIGMOID, False)
    for more in (2 ** 32, 2 ** 31, -2 ** 32, 2 ** 64):
        for groups, activation in ((2 + more, pb.ACT_NONE), (2, pb.ACT_SILU + more)):
            with pytest.raises(pb._Apart):
                pb._norm(maps, groups, activation, 1e-5, Like(8))
        with pytest.raises(pb._Apart):
            pb._scan(steps, None, pb.SCAN_SIGMOID + more, False)
        fine = [3, 10, 8, 2, F]
        assert pb.group_norm_workspace_bytes(*fine) > 0
        for i in range(5):
            assert pb.group_norm_workspace_bytes(*fine[:i], fine[i] + more, *fine[i + 1:]) == 0


@pytest.mark.parametrize("type", [F, H])
@pytest.mark.parametrize("c,groups", [(1, 1), (3, 1), (4, 2), (8, 8), (40, 8), (96, 32), (2048, 4), (65536, 1)])
def test_the_scratch_of_the_largest_samples(c, groups, type):
    """Up to the most pixels there may be the scratch grows with them: never less for more, at most twice as much and a row of sums for twice as
    many."""
    most = 2 ** 31 - 1
    pixels = [2 ** 30, 2 ** 31 - 70_000, 2 ** 31 - 4097, 2 ** 31 - 4096, 2 ** 31 - 4095, 2 ** 31 - 257, 2 ** 31 - 16, 2 ** 31 - 2, most]
    need = [pb.group_norm_workspace_bytes(1, p, c, groups, type) for p in pixels]
    assert need[0] > 0 and need == sorted(need) and need[-1] <= 2 * need[0] + 8 * c
    assert pb.group_norm_workspace_bytes(1, most + 1, c, groups, type) == 0


@pytest.mark.parametrize("n,pixels,c,groups", [(1, 1, 65536, 1), (1, 1, 65536, 65536), (1, 1, 2048, 2), (1, 400, 32, 4), (3, 49, 64, 8), (32, 400, 32, 4), (2, 7056, 48, 6),
                                               (5120, 400, 32, 4), (300, 7056, 5, 1), (5000, 81, 16, 16)])
@pytest.mark.parametrize("type", [F, H])
def test_scratch_goes_with_the_sizes(n, pixels, c, groups, type):
    """What a call needs is a row of 2 c sums for each of the up to 16 blocks that share a sample, or for each slab of 16 pixels or more, and two
    numbers a group: nothing by the device's size alone."""
    rows = n * min(pixels, 16) + n * (pixels // 16 + 1)
    assert pb.group_norm_workspace_bytes(n, pixels, c, groups, type) <= 8 * c * rows + 8 * n * groups + 1024


def test_tensors_that_do_not_go_together():
    """The binding's own look at torch tensors: nothing on the host, shapes and types alike."""
    x = torch.zeros(3, 2, 8)
    assert pb.gated_scan(x, x, x) == pb.ERR_ARG and pb.gated_scan_backward(x, x, x, x, x, x) == pb.ERR_ARG
    assert pb.group_norm(x, None, None, x, None, None, 2, x) == pb.ERR_ARG and pb.group_norm_backward(x, x, None, None, x, x, x, x, x, 2, x) == pb.ERR_ARG
    with pytest.raises(pb.PaacError):
        pb.TensorList([x])
    with pytest.raises(pb.PaacError):
        pb.TensorList([x], [x, x])


ROWS = """
#include "rows.h"
static paac::RowSet set(int64_t at, int64_t outer, int64_t inner, int64_t n0, int64_t n1, int64_t c, int size) {
  return paac::RowSet(paac_rows{(void*)at, outer, inner}, n0, n1, c, size);
}
extern "C" int rows_apart(int64_t* v) { return set(v[0], v[1], v[2], v[3], v[4], v[5], (int)v[6]).rows_apart(); }
extern "C" int apart(int64_t* v, int64_t* w) {
  return set(v[0], v[1], v[2], v[3], v[4], v[5], (int)v[6]).apart_from(set(w[0], w[1], w[2], w[3], w[4], w[5], (int)w[6]));
}
"""


def _bytes(v):
    at, outer, inner, n0, n1, c, size = v
    return [at + (i * outer + j * inner + k) * size + b for i in range(n0) for j in range(n1) for k in range(c) for b in range(size)]


def test_rows_that_are_said_to_be_apart_are(tmp_path):
    """Against every byte of small sets; and what real layouts need is not refused."""
    src, so = tmp_path / "rows.cpp", tmp_path / "rows.so"
    src.write_text(ROWS)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    L = C.CDLL(str(so))

    def arr(v):
        return (C.c_int64 * 7)(*v)

    rng = np.random.RandomState(1)
    said = 0
    for _ in range(4000):
        c, n0, n1 = rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 4)
        v = [1000, int(rng.randint(-12, 13)), int(rng.randint(-12, 13)), int(n0), int(n1), int(c), 2]
        w = list(v) if rng.rand() < 0.6 else [1000, int(rng.randint(-12, 13)), int(rng.randint(-12, 13)), int(n0), int(n1), int(c), int(rng.choice([1, 2]))]
        w[0] = 1000 + int(rng.randint(-40, 41))
        mine = _bytes(v)
        if L.rows_apart(arr(v)):
            assert len(set(mine)) == len(mine), v
            if L.apart(arr(v), arr(w)):
                said += 1
                assert not set(mine) & set(_bytes(w)), (v, w)
    assert said > 300
    halves = [[4096, 16, 64, 4, 5, 8, 2], [4096 + 16, 16, 64, 4, 5, 8, 2]]
    assert L.rows_apart(arr(halves[0])) and L.apart(arr(halves[0]), arr(halves[1])) and not L.apart(arr(halves[0]), arr(halves[0]))
    assert L.rows_apart(arr([4096, 8, 32, 4, 5, 8, 2])) and L.rows_apart(arr([4096, 40, 8, 4, 5, 8, 2])) and L.rows_apart(arr([4096, 8, -32, 4, 5, 8, 2]))


def test_rows_between_the_others_rows_are_not_refused(tmp_path):
    """Sets of the same strides, whose rows are apart from one another: said to be apart exactly where no byte is in both, whatever the strides are."""
    src, so = tmp_path / "rows.cpp", tmp_path / "rows.so"
    src.write_text(ROWS)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    L = C.CDLL(str(so))

    def arr(v):
        return (C.c_int64 * 7)(*v)

    rng = np.random.RandomState(2)
    seen = [0, 0]
    for _ in range(20000):
        c, n0, n1, size = int(rng.randint(1, 4)), int(rng.randint(1, 6)), int(rng.randint(1, 6)), int(rng.choice([1, 2]))
        small = int(rng.randint(c, 3 * c + 2))
        large = small * (n1 - 1) + c + int(rng.randint(0, 9))
        v = [1000, large * int(rng.choice([-1, 1])), small * int(rng.choice([-1, 1])), n0, n1, c, size]
        if rng.rand() < 0.5:
            v[1], v[2], v[3], v[4] = v[2], v[1], v[4], v[3]
        w = list(v)
        w[0] += int(rng.randint(-3 * large, 3 * large + 1)) * int(rng.choice([1, size])) if rng.rand() < 0.5 else int(rng.randint(-3 * small, 3 * small + 1))
        assert L.rows_apart(arr(v))
        apart = not set(_bytes(v)) & set(_bytes(w))
        seen[apart] += 1
        assert bool(L.apart(arr(v), arr(w))) == apart, (v, w)
    assert min(seen) > 4000
    # two halves of every step, the sequences a little further apart than their steps take
    assert L.apart(arr([4096, 5 * 16 + 8, 16, 4, 5, 8, 2]), arr([4096 + 16, 5 * 16 + 8, 16, 4, 5, 8, 2]))
    # sizes at which 64 bits are not enough for places
    far = 2 ** 54
    assert L.apart(arr([4096, far, 16, 4, 5, 8, 2]), arr([4096 + 16, far, 16, 4, 5, 8, 2])) and not L.apart(arr([4096, far, 16, 4, 5, 8, 2]), arr([4096 + 14, far, 16, 4, 5, 8, 2]))


# ---- the references ---------------------------------------------------------------------------------------------------------------------

def _central(f, v, step=1e-6):
    """Central differences of the scalar f by every element of v."""
    out = np.zeros_like(v)
    flat, to = v.reshape(-1), out.reshape(-1)
    for i in range(flat.size):
        keep = flat[i]
        flat[i] = keep + step
        up = f()
        flat[i] = keep - step
        down = f()
        flat[i] = keep
        to[i] = (up - down) / (2 * step)
    return out


@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("reverse", [True, False])
def test_the_scans_gradient_is_the_slope(sigmoid, reverse):
    rng = np.random.RandomState(5)
    gate, x, w, h0, wl = rng.randn(6, 3, 2), rng.randn(6, 3, 2), rng.randn(6, 3, 2), rng.randn(3, 2), rng.randn(3, 2)
    restart = (rng.rand(6, 3) < 0.3).astype(np.uint8)

    def loss():
        h, last, _, _ = ref.scan_forward(gate, x, h0, restart, sigmoid, reverse)
        return float((h * w).sum() + (last * wl).sum())

    h = ref.scan_forward(gate, x, h0, restart, sigmoid, reverse)[0]
    dgate, dx, dh0 = ref.scan_backward(gate, x, h, w, h0, wl, restart, sigmoid, reverse, 0.0)[:3]
    for got, v in ((dgate, gate), (dx, x), (dh0, h0)):
        assert np.abs(got - _central(loss, v)).max() <= 1e-7          # a step of 1e-6 squared, and 1e-16 / 1e-6 of rounding


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
def test_the_norms_gradient_is_the_slope(kind):
    rng = np.random.RandomState(6)
    x, dy, gamma, beta = rng.randn(2, 4, 6), rng.randn(2, 4, 6), rng.randn(6), rng.randn(6)

    def loss():
        return float((ref.norm_forward(x, gamma, beta, 3, kind, 1e-3)[0] * dy).sum())

    mean, rstd = ref.norm_stats(x, 3, 1e-3)
    assert np.abs(ref.norm_forward(x, gamma, beta, 3, kind, 1e-3)[3]).min() > 1e-4          # no difference straddles relu's corner
    dx, dgamma, dbeta, _ = ref.norm_backward(x, dy, gamma, beta, mean, rstd, kind)
    for got, v in ((dx, x), (dgamma, gamma), (dbeta, beta)):
        assert np.abs(got - _central(loss, v)).max() <= 1e-7


def test_the_norms_reference_against_torch():
    rng = np.random.RandomState(7)
    x, gamma, beta = rng.randn(2, 5, 12), rng.randn(12), rng.randn(12)
    want = torch.nn.functional.group_norm(torch.from_numpy(x).transpose(1, 2), 4, torch.from_numpy(gamma), torch.from_numpy(beta), 1e-5).transpose(1, 2)
    assert np.abs(ref.norm_forward(x, gamma, beta, 4, "none", 1e-5)[0] - want.numpy()).max() <= 1e-12
