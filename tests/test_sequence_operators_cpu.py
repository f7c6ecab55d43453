"""The operators of a policy over sequences: what can be said without a device.  Their refusals, the structures' layouts, and the references that
the GPU tests hold the kernels to, against differences."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import sequence_ref as ref
from paper_1705_04862_b200 import binding as pb
from test_operators_cpu import CSRC, NONE, ROWS, A, F, H, _bytes, _central

L = pb.lib


# The header's structures, field by field.
I, P, S = C.c_int32, C.c_void_p, C.c_int64


def structure(*fields):
    return type("Structure", (C.Structure,), {"_fields_": [(f, t) for names, t in fields for f in names.split()]})


Conv = structure(("t n c width type activation", I), ("restart", P), ("restart_n restart_t", S), ("x", pb.Rows), ("weight bias before", P))
ConvOut = structure(("y", pb.Rows), ("after", P))
ConvGrads = structure(("dy", pb.Rows), ("dafter", P), ("dx", pb.Rows), ("dweight dbias dbefore workspace", P), ("workspace_bytes", C.c_size_t))
Selective = structure(("t n c state groups type softplus", I), ("restart", P), ("restart_n restart_t", S), ("x dt B C z", pb.Rows), ("A D dt_bias", P))
SelectiveOut = structure(("h0", P), ("y", pb.Rows), ("h_last states workspace", P), ("workspace_bytes", C.c_size_t))
SelectiveGrads = structure(("states", P), ("dy", pb.Rows), ("dh_last", P), ("dx ddt dB dC dz", pb.Rows), ("dA dD ddt_bias dh0 workspace", P), ("workspace_bytes", C.c_size_t))
Draw = structure(("n v type", I), ("logits", P), ("logits_row", S), ("allowed", P), ("allowed_row", S), ("uniforms temperature top_k top_p min_p actions logprobs", P))


def test_the_bindings_bytes_are_the_headers_structures():
    for form, s in ((pb._CONV, Conv), (pb._CONV_OUT, ConvOut), (pb._CONV_GRADS, ConvGrads), (pb._SELECTIVE, Selective), (pb._SELECTIVE_OUT, SelectiveOut),
                    (pb._SELECTIVE_GRADS, SelectiveGrads), (pb._DRAW, Draw)):
        assert form.size == C.sizeof(s)
        numbers = list(range(1, 1 + len(form.unpack(bytes(form.size)))))
        flat = []
        for name, kind in s._fields_:
            v = getattr(s.from_buffer_copy(form.pack(*numbers)), name)
            flat += [v.data, v.outer, v.inner] if isinstance(v, pb.Rows) else [v]
        assert flat == numbers
    assert pb.SELECTIVE_SPAN == ref.SPAN


def test_structures_have_the_sizes_that_the_compiler_gives_them(tmp_path):
    src = tmp_path / "sizes.c"
    names = ["paac_conv", "paac_conv_out", "paac_conv_grads", "paac_selective", "paac_selective_out", "paac_selective_grads", "paac_draw"]
    src.write_text('#include <stdio.h>\n#include "paac.h"\nint main(void) { printf("%s\\n", %s); return 0; }\n' % (" ".join(["%zu"] * 7), ", ".join("sizeof(%s)" % n for n in names)))
    subprocess.run(["gcc", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    got = subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in got] == [C.sizeof(s) for s in (Conv, ConvOut, ConvGrads, Selective, SelectiveOut, SelectiveGrads, Draw)]


def conv(backward=False, t=4, n=2, c=8, width=4, type=F, act=pb.ACT_SILU, restart=None, weight=10 * A, bias=11 * A, before=None, after=None, dafter=None, dw=None, dbias=None,
         dbefore=None, workspace=20 * A, room=1 << 30, **rows):
    """A call that would be fine but for what is changed; every array in a megabyte of its own."""
    r = {k: pb.Rows(A * (i + 1), c, n * c) for i, k in enumerate(["x", "y", "dy", "dx"])}
    r.update(rows)
    s = Conv(t, n, c, width, type, act, restart, 1, n, r["x"], weight, bias, before)
    if not backward:
        return L().paac_causal_conv(C.byref(s), C.byref(ConvOut(r["y"], after)), None)
    return L().paac_causal_conv_backward(C.byref(s), C.byref(ConvGrads(r["dy"], dafter, r["dx"], dw, dbias, dbefore, workspace, room)), None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("wrong", [
    dict(t=0), dict(n=0), dict(c=0), dict(t=-1), dict(t=(1 << 30) + 1, n=1, c=1), dict(n=1 << 20, c=1 << 12), dict(type=2), dict(act=3), dict(act=-1), dict(width=1), dict(width=5),
    dict(weight=None), dict(weight=10 * A + 2), dict(bias=11 * A + 1), dict(x=NONE), dict(x=pb.Rows(A + 2, 8, 16)), dict(type=H, x=pb.Rows(A + 1, 8, 16)),
    dict(x=pb.Rows(A, 1 << 60, 16)), dict(before=12 * A + 2),
])
def test_conv_refuses(wrong, backward):
    assert conv(backward, **wrong) == pb.ERR_ARG


@pytest.mark.parametrize("wrong", [
    dict(y=NONE), dict(y=pb.Rows(2 * A, 8, 15)), dict(y=pb.Rows(2 * A, 0, 16)), dict(y=pb.Rows(A, 8, 16)), dict(y=pb.Rows(A + 32, 8, 16)), dict(y=pb.Rows(10 * A + 64, 8, 16)),
    dict(after=2 * A), dict(after=A + 64), dict(after=12 * A, before=12 * A + 32), dict(after=11 * A), dict(restart=2 * A + 100), dict(after=12 * A + 1),
])
def test_conv_refuses_what_is_written_over(wrong):
    assert conv(**wrong) == pb.ERR_ARG


@pytest.mark.parametrize("wrong", [
    dict(dx=NONE), dict(dy=NONE), dict(dx=pb.Rows(4 * A, 7, 16)), dict(dx=pb.Rows(3 * A, 8, 16)), dict(dx=pb.Rows(A + 32, 8, 16)), dict(dw=4 * A), dict(dw=10 * A), dict(dbias=11 * A),
    dict(dw=12 * A, dbias=12 * A + 64), dict(dw=12 * A + 2), dict(dbefore=12 * A, dafter=12 * A), dict(dbefore=4 * A + 64), dict(dbefore=12 * A, before=12 * A), dict(workspace=4 * A),
    dict(workspace=A), dict(dw=20 * A + 16), dict(restart=4 * A + 64),
])
def test_conv_backward_refuses(wrong):
    assert conv(True, **wrong) == pb.ERR_ARG


def test_conv_scratch():
    need = pb.causal_conv_workspace_bytes(4, 2, 8, 4, F)
    assert need > 0
    assert conv(True, workspace=None) == conv(True, workspace=20 * A + 8) == conv(True, room=need - 1) == pb.ERR_WORKSPACE
    for i, fine in enumerate([4, 2, 8, 4, F]):
        for more in (2 ** 32, 2 ** 31, -2 ** 32, 2 ** 64):
            args = [4, 2, 8, 4, F]
            args[i] += more
            assert pb.causal_conv_workspace_bytes(*args) == 0
    # a row of c (width + 1) sums for each block of four warps or more parts, whose threads have sixteen steps or more of up to four channels
    for t, n, c in ((5, 1024, 512), (2048, 8, 1024), (1, 32, 64), (2 ** 30, 1, 1), (1, 2 ** 31 - 1, 1)):
        need = pb.causal_conv_workspace_bytes(t, n, c, 4, H)
        assert 0 < need <= 4 * 5 * c * (n * (t // 16 + 1) // 4 + 1)


def scan(backward=False, t=40, n=2, c=8, state=4, groups=2, type=F, softplus=1, restart=None, A_=10 * A, D=11 * A, bias=12 * A, h0=None, last=None, states=13 * A, dh_last=None,
         workspace=40 * A, room=1 << 30, grads=None, **rows):
    gs = groups * state
    names = dict(x=c, dt=c, B=gs, C=gs, z=c, y=c, dy=c, dx=c, ddt=c, dB=gs, dC=gs, dz=c)
    r = {k: pb.Rows(A * (21 + i), w, n * w) for i, (k, w) in enumerate(names.items())}
    r.update(rows)
    s = Selective(t, n, c, state, groups, type, softplus, restart, 1, n, r["x"], r["dt"], r["B"], r["C"], r["z"], A_, D, bias)
    if not backward:
        return L().paac_selective_scan(C.byref(s), C.byref(SelectiveOut(h0, r["y"], last, states, workspace, room)), None)
    g = dict(dA=14 * A, dD=15 * A, ddt_bias=16 * A, dh0=17 * A)
    g.update(grads or {})
    gr = SelectiveGrads(states, r["dy"], dh_last, *(r[k] for k in ("dx", "ddt", "dB", "dC", "dz")), g["dA"], g["dD"], g["ddt_bias"], g["dh0"], workspace, room)
    return L().paac_selective_scan_backward(C.byref(s), C.byref(gr), None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("wrong", [
    dict(t=0), dict(n=0), dict(c=0), dict(state=0), dict(state=65), dict(groups=0), dict(groups=3), dict(groups=-2), dict(t=(1 << 30) + 1, n=1), dict(n=1 << 20, c=1 << 12), dict(type=2),
    dict(A_=None), dict(A_=10 * A + 1), dict(D=11 * A + 2), dict(bias=12 * A + 3), dict(x=NONE), dict(dt=NONE), dict(B=NONE), dict(C=NONE), dict(x=pb.Rows(21 * A + 1, 8, 16)),
    dict(B=pb.Rows(23 * A + 2, 8, 16)), dict(C=pb.Rows(24 * A, 1 << 60, 16)), dict(states=13 * A + 2),
])
def test_scan_refuses(wrong, backward):
    assert scan(backward, **wrong) == pb.ERR_ARG


@pytest.mark.parametrize("wrong", [
    dict(y=NONE), dict(y=pb.Rows(26 * A, 7, 16)), dict(y=pb.Rows(21 * A, 8, 16)), dict(y=pb.Rows(23 * A + 64, 8, 16)), dict(last=26 * A), dict(last=10 * A), dict(last=18 * A + 1),
    dict(h0=18 * A, last=18 * A + 64), dict(states=26 * A), dict(states=10 * A), dict(h0=13 * A + 256), dict(restart=26 * A), dict(restart=13 * A),
])
def test_scan_refuses_what_is_written_over(wrong):
    assert scan(**wrong) == pb.ERR_ARG


@pytest.mark.parametrize("wrong", [
    dict(states=None), dict(dy=NONE), dict(z=NONE), dict(dx=pb.Rows(27 * A, 8, 16)), dict(ddt=pb.Rows(28 * A, 8, 16)), dict(dB=pb.Rows(23 * A, 8, 16)), dict(dC=pb.Rows(30 * A, 8, 16)),
    dict(dz=pb.Rows(25 * A, 8, 16)), dict(dx=pb.Rows(28 * A, 4, 16)), dict(dB=pb.Rows(30 * A, 0, 16)), dict(grads=dict(dA=10 * A)), dict(grads=dict(dD=11 * A)),
    dict(grads=dict(ddt_bias=15 * A + 16)), dict(grads=dict(dh0=13 * A)), dict(grads=dict(dh0=18 * A), dh_last=18 * A), dict(grads=dict(dA=14 * A + 1)), dict(workspace=13 * A),
    dict(workspace=14 * A), dict(workspace=28 * A),
    dict(dx=NONE, ddt=NONE, dB=NONE, dC=NONE, dz=NONE, grads=dict(dA=None, dD=None, ddt_bias=None, dh0=None)),
])
def test_scan_backward_refuses(wrong):
    assert scan(True, **wrong) == pb.ERR_ARG


def test_scan_scratch():
    need = pb.selective_scan_workspace_bytes(40, 2, 8, 4, 2, F, backward=True)
    assert need > 0 and pb.selective_scan_workspace_bytes(1, 2, 8, 4, 2, F) == 0
    assert scan(True, workspace=None) == scan(True, workspace=40 * A + 4) == scan(True, room=need - 1) == pb.ERR_WORKSPACE
    need = pb.selective_scan_workspace_bytes(4000, 1, 8, 4, 2, F)
    assert need > 0 and scan(t=4000, n=1, room=need - 1) == scan(t=4000, n=1, workspace=None) == pb.ERR_WORKSPACE
    assert scan(t=4000, n=1, workspace=26 * A) == pb.ERR_ARG
    fine = [40, 2, 8, 4, 2, F]
    for i in range(6):
        for more in (2 ** 32, 2 ** 31, -2 ** 32, 2 ** 64):
            args = list(fine)
            args[i] += more
            assert pb.selective_scan_workspace_bytes(*args) == 0
    for call in (L().paac_selective_scan, L().paac_selective_scan_backward, L().paac_causal_conv, L().paac_causal_conv_backward):
        assert call(None, A, None) == pb.ERR_ARG
    assert L().paac_selective_scan(C.byref(Selective(4, 2, 8, 4, 1)), None, None) == L().paac_causal_conv_backward(C.byref(Conv(4, 2, 8, 4)), None, None) == pb.ERR_ARG
    assert L().paac_sample(None, None) == pb.ERR_ARG


def draw(n=4, v=100, type=F, row=100, temperature=None, top_k=None, top_p=None, min_p=None, allowed=None, allowed_row=100, logits=A, uniforms=2 * A, actions=3 * A, logprobs=4 * A):
    s = Draw(n, v, type, logits, row, allowed, allowed_row, uniforms, temperature, top_k, top_p, min_p, actions, logprobs)
    return L().paac_sample(C.byref(s), None)


@pytest.mark.parametrize("wrong", [
    dict(n=0), dict(v=0), dict(n=-1), dict(v=(1 << 23) + 1), dict(type=2), dict(logits=None), dict(uniforms=None), dict(actions=None), dict(logits=A + 2), dict(type=H, logits=A + 1),
    dict(uniforms=2 * A + 1), dict(actions=3 * A + 2), dict(logprobs=4 * A + 3), dict(temperature=5 * A + 1), dict(top_k=5 * A + 2), dict(top_p=5 * A + 3), dict(min_p=5 * A + 1),
    dict(actions=A), dict(actions=A + 1596), dict(logprobs=A + 400), dict(logprobs=3 * A + 12), dict(actions=2 * A), dict(temperature=3 * A), dict(top_k=4 * A + 8), dict(allowed=3 * A),
    dict(allowed=4 * A - 390), dict(row=1 << 60), dict(allowed=6 * A, allowed_row=1 << 60), dict(n=(1 << 28) + 1, v=1),
])
def test_sample_refuses(wrong):
    assert draw(**wrong) == pb.ERR_ARG


def test_tensors_that_do_not_go_together():
    """The binding's own look at torch tensors: nothing on the host, shapes and types alike."""
    x, w = torch.zeros(3, 2, 8), torch.zeros(8, 4)
    assert pb.causal_conv(x, w, None, x) == pb.causal_conv_backward(x, x, w, None, x, w, None, x) == pb.ERR_ARG
    b = torch.zeros(3, 2, 1, 4)
    assert pb.selective_scan(x, x, w, b, b, x) == pb.selective_scan_backward(x, x, w, b, b, x, x, x, x, w, b, b, x) == pb.ERR_ARG
    assert pb.sample(torch.zeros(3, 5), torch.zeros(3), torch.zeros(3, dtype=torch.int32)) == pb.ERR_ARG


class _Reached(Exception):
    pass


def test_numbers_beyond_32_bits_are_not_cut_off():
    """What a field of the library's structures cannot hold is refused, not passed on without its upper bits."""
    pb._with_torch()

    class Like:
        dtype = torch.float32
        def __init__(self, *shape): self.shape = torch.Size(shape)
        def get_device(self): return 0
        def dim(self): return len(self.shape)
        def stride(self): raise _Reached          # (only once the sizes have been looked at)
    with pytest.raises(_Reached):
        pb._conv(Like(4, 2, 8), Like(8, 4), None, None, 2, None)
    with pytest.raises(_Reached):
        pb._selective(Like(4, 2, 8), None, Like(8, 16), Like(4, 2, 16), None, None, None, None, True, None)
    for shape in ((2 ** 32 + 5, 1, 1), (5, 2 ** 32 + 1, 1), (5, 1, 2 ** 31)):
        with pytest.raises(pb._Apart):
            pb._conv(Like(*shape), Like(shape[2], 4), None, None, 2, None)
        with pytest.raises(pb._Apart):
            pb._selective(Like(*shape), None, Like(shape[2], 4), Like(*shape[:2], 4), None, None, None, None, True, None)
    for more in (2 ** 32, 2 ** 31, -2 ** 32):
        with pytest.raises(pb._Apart):
            pb._conv(Like(4, 2, 8), Like(8, 4), None, None, 2 + more, None)
    with pytest.raises(pb._Apart):
        pb._conv(Like(4, 2, 8), Like(8, 2 ** 32 + 4), None, None, 2, None)
    with pytest.raises(pb._Apart):
        pb._selective(Like(4, 2, 8), None, Like(8, 2 ** 32 + 4), Like(4, 2, 2 ** 32 + 4), None, None, None, None, True, None)
    for A_, B in ((Like(7, 16), Like(4, 2, 16)), (Like(8, 15), Like(4, 2, 16)), (Like(8, 16), Like(4, 3, 16)), (Like(8, 16), Like(5, 2, 1, 16)), (Like(8), Like(4, 2, 16))):
        with pytest.raises(pb._Apart):
            pb._selective(Like(4, 2, 8), None, A_, B, None, None, None, None, True, None)
    assert pb.sample(Like(2 ** 32 + 1, 4), Like(2 ** 32 + 1), Like(2 ** 32 + 1)) == pb.ERR_ARG


# ---- the references ---------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
def test_the_convolutions_gradient_is_the_slope(kind):
    rng = np.random.RandomState(5)
    t, n, c, width = 7, 2, 3, 4
    x, w, bias, before, dy, dafter = rng.randn(t, n, c), rng.randn(c, width), rng.randn(c), rng.randn(n, width - 1, c), rng.randn(t, n, c), rng.randn(n, width - 1, c)
    restart = (rng.rand(t, n) < 0.3).astype(np.uint8)

    def loss():
        y, after, _ = ref.conv_forward(x, w, bias, before, restart, kind, torch.float32)
        return float((y * dy).sum() + (after * dafter).sum())

    assert np.abs(ref.conv_forward(x, w, bias, before, restart, "none", torch.float32)[0]).min() > 1e-4          # no difference straddles relu's corner
    got = ref.conv_backward(x, dy, w, bias, before, dafter, restart, kind, torch.float32, 1)
    for name, v in (("dx", x), ("dweight", w), ("dbias", bias), ("dbefore", before)):
        assert np.abs(got[name][0] - _central(loss, v)).max() <= 1e-7          # a step of 1e-6 squared, and 1e-16 / 1e-6 of rounding


@pytest.mark.parametrize("softplus,gate,groups", [(True, True, 1), (False, True, 2), (True, False, 4)])
def test_the_scans_gradient_is_the_slope(softplus, gate, groups):
    rng = np.random.RandomState(6)
    t, n, c, m = 5, 2, 4, 3
    v = dict(x=rng.randn(t, n, c), dt=0.3 * rng.randn(t, n, c) + (0 if softplus else 1), A=-0.5 - rng.rand(c, m), B=rng.randn(t, n, groups, m), C=rng.randn(t, n, groups, m), D=rng.randn(c),
             z=rng.randn(t, n, c), bias=0.1 * rng.randn(c), h0=rng.randn(n, c, m))
    dy, dh_last, restart = rng.randn(t, n, c), rng.randn(n, c, m), (rng.rand(t, n) < 0.3).astype(np.uint8)

    def run():
        return ref.Scan(v["x"], v["dt"], v["A"], v["B"], v["C"], v["D"], v["z"] if gate else None, v["bias"], v["h0"], restart, softplus, torch.float32)

    def loss():
        s = run()
        return float((s.y * dy).sum() + (s.last * dh_last).sum())

    got = run().backward(dy, dh_last)
    for name, of in (("dx", "x"), ("ddt", "dt"), ("dA", "A"), ("dB", "B"), ("dC", "C"), ("dD", "D"), ("dz", "z"), ("ddt_bias", "bias"), ("dh0", "h0")):
        if name in got:
            assert np.abs(got[name][0] - _central(loss, v[of])).max() <= 2e-7, name
    assert ("dz" in got) == gate


def test_the_convolutions_reference_against_torch():
    rng = np.random.RandomState(7)
    x, w, b = rng.randn(9, 2, 5), rng.randn(5, 3), rng.randn(5)
    padded = torch.nn.functional.pad(torch.from_numpy(x).permute(1, 2, 0), (2, 0))
    want = torch.nn.functional.conv1d(padded, torch.from_numpy(w)[:, None], torch.from_numpy(b), groups=5).permute(2, 0, 1)
    assert np.abs(ref.conv_forward(x, w, b, None, None, "none", torch.float32)[0] - want.numpy()).max() <= 1e-12


def test_the_draws_reference_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert [ref.draw(x, u)[0] for u in (0.0, 0.0999, 0.1001, 0.4999, 0.5001, 0.6999, 0.7001, 0.9999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [ref.draw(x, u, top_k=2)[0] for u in (0.0, 0.57, 0.58, 0.999)] == [1, 1, 3, 3]
    assert [ref.draw(x, u, top_p=0.65)[0] for u in (0.0, 0.57, 0.58)] == [1, 1, 3] and [ref.draw(x, u, top_p=0.75)[0] for u in (0.45, 0.7)] == [2, 3]
    assert [ref.draw(x, u, min_p=0.6)[0] for u in (0.1, 0.58)] == [1, 3] and ref.draw(x, 0.9, temperature=0.0)[0] == 1
    assert ref.draw(x, 0.5, allowed=np.array([1, 0, 0, 0]))[0] == 0 and ref.draw(x, 0.5, allowed=np.zeros(4))[0] == -1
    assert abs(ref.draw(x, 0.5, top_k=2)[1] - np.log(4 / 7)) < 1e-12
    assert ref.draw(np.zeros(10), 0.05, top_p=0.5)[0] == 0 and ref.draw(np.zeros(10), 0.99, top_p=0.5)[0] == 4          # of equal ones the first


def test_parts_of_wider_rows_of_different_lengths_are_not_refused(tmp_path):
    """Gradients of a projection's outputs lie side by side in one tensor, channels beside states: rows of the same strides whose lengths differ are said to be apart
    exactly where no byte is in both."""
    src, so = tmp_path / "rows.cpp", tmp_path / "rows.so"
    src.write_text(ROWS)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = C.CDLL(str(so))

    def arr(v):
        return (C.c_int64 * 7)(*v)

    rng = np.random.RandomState(3)
    seen = [0, 0]
    for _ in range(20000):
        c, n0, n1, size = int(rng.randint(1, 5)), int(rng.randint(1, 5)), int(rng.randint(1, 5)), int(rng.choice([1, 2]))
        more = int(rng.randint(1, 5))
        small = max(c, more) + int(rng.randint(0, 2 * (c + more)))
        large = small * (n1 - 1) + max(c, more) + int(rng.randint(0, 9))
        v = [1000, large * int(rng.choice([-1, 1])), small * int(rng.choice([-1, 1])), n0, n1, c, size]
        if rng.rand() < 0.5:
            v[1], v[2], v[3], v[4] = v[2], v[1], v[4], v[3]
        w = list(v)
        w[5] = more
        w[0] += int(rng.randint(-3 * small, 3 * small + 1)) if rng.rand() < 0.7 else int(rng.randint(-2 * large, 2 * large + 1))
        apart = not set(_bytes(v)) & set(_bytes(w))
        seen[apart] += 1
        assert bool(lib.apart(arr(v), arr(w))) == apart, (v, w)
    assert min(seen) > 3000
    # a longer row than the strides cover is one that its neighbours lie in: not said to be apart
    assert not lib.apart(arr([1000, 40, 8, 4, 5, 4, 2]), arr([1008, 40, 8, 4, 5, 9, 2]))


@pytest.mark.parametrize("t,n,c,state,groups", [(87, 2, 80, 5, 1), (4, 41, 64, 8, 1), (1, 3, 8, 16, 2), (20, 1, 7, 3, 1)])
def test_everything_in_one_tensor_is_not_refused_for_its_places(t, n, c, state, groups):
    """The scan's gradient with its inputs side by side in one tensor, and what it writes in another: refused for its scratch alone, which it does not get."""
    gs = groups * state
    widths = dict(x=c, dt=c, B=gs, C=gs, z=c, dx=c, ddt=c, dB=gs, dC=gs, dz=c)
    row, rows, at = 3 * c + 2 * gs, {}, 0
    for i, (k, w) in enumerate(widths.items()):
        base, at = (21 * A, 0 if k == "x" else at) if i < 5 else (25 * A, 0 if k == "dx" else at)
        rows[k] = pb.Rows(base + 4 * at, row, n * row)
        at += w
    rows["dy"] = pb.Rows(29 * A, c, n * c)
    far = dict(states=50 * A, A_=60 * A, D=61 * A, bias=62 * A, grads=dict(dA=63 * A, dD=64 * A, ddt_bias=65 * A, dh0=66 * A))
    assert scan(True, t=t, n=n, c=c, state=state, groups=groups, room=0, **far, **rows) == pb.ERR_WORKSPACE
    rows["dB"] = pb.Rows(rows["dB"].data - 4, row, n * row)
    assert scan(True, t=t, n=n, c=c, state=state, groups=groups, room=0, **far, **rows) == pb.ERR_ARG
