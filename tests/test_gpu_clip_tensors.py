"""Clipping over many tensors (paac_clip_tensors) against sums and products in 64 bits."""
import math

import numpy as np
import pytest
import torch

from operators_ref import U, f64, half_step
from paper_1705_04862_b200 import binding as pb

pytestmark = pytest.mark.gpu
F, H = torch.float32, torch.bfloat16
# at most 32 squares are added up in float, one rounding each, the rest in double; the root halves it; then one rounding to float
NORM = 17 * U


def lay(sizes, dtype, shift, gen, scale=1.0):
    """Tensors of the given sizes with `shift` elements before each (0: every one at the beginning of an allocation)."""
    out = []
    for n in sizes:
        t = torch.empty(n + shift, dtype=dtype, device="cuda")
        t.copy_(torch.randn(n + shift, device="cuda", generator=gen) * scale)
        out.append(t[shift:])
    return out


def check(src, dst, before, clip, out):
    total = math.sqrt(sum(float((b ** 2).sum()) for b in before))
    norm, factor = out.cpu().double().numpy()
    assert abs(norm - total) <= NORM * total
    want = clip / total if 0 < clip < total else 1.0
    # the norm's error, the quotient and the product in float, then the storage type
    assert abs(factor - want) <= (NORM + 2 * U) * want
    for d, b in zip(dst, before):
        if d is not None:
            exact = b * want
            off = np.abs(f64(d) - exact) - (np.abs(exact) * (half_step(d.dtype) * (1 + 2 * NORM) + NORM + 4 * U) + 2.0 ** -134)
            assert off.size == 0 or off.max() <= 0, float(off.max())
    for s, d, b in zip(src, dst, before):
        if d is None or d.data_ptr() != s.data_ptr() or want == 1.0:
            assert np.array_equal(f64(s), b)


@pytest.mark.parametrize("clip", [0.5, 1e6, 0.0])
@pytest.mark.parametrize("types", [(F, F), (F, H), (H, F), (H, H)])
@pytest.mark.parametrize("sizes", [[1], [0, 5, 0], [7, 4096, 4097, 31], [100_003, 1, 8192, 16], [300_000] * 3])
def test_into_tensors_of_their_own(sizes, types, clip):
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    for shift_src, shift_dst in ((0, 0), (1, 0), (0, 3), (5, 5), (3, 8)):
        src = lay(sizes, types[0], shift_src, gen)
        whole = [torch.full((n + shift_dst + 9,), 7.0, dtype=types[1], device="cuda") for n in sizes]
        dst = [w[shift_dst:shift_dst + n] for w, n in zip(whole, sizes)]
        before, out = [f64(s) for s in src], torch.zeros(2, device="cuda")
        assert pb.clip_tensors(pb.TensorList(src, dst), clip, norm_and_scale=out) == pb.OK
        check(src, dst, before, clip, out)
        for w, n in zip(whole, sizes):                 # nothing around them
            assert bool((w[:shift_dst] == 7).all()) and bool((w[shift_dst + n:] == 7).all())


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("clip", [2.0, 1e9])
def test_in_place_and_for_the_norm_only(dtype, clip):
    gen = torch.Generator(device="cuda").manual_seed(3)
    for shift in (0, 1, 7):
        src = lay([513, 70_001, 3, 20_000], dtype, shift, gen)
        dst = [src[0], src[1], None, src[3]]
        before, out = [f64(s) for s in src], torch.zeros(2, device="cuda")
        assert pb.clip_tensors(pb.TensorList(src, dst), clip, norm_and_scale=out) == pb.OK
        check(src, dst, before, clip, out)


@pytest.mark.parametrize("count", [95, 96, 97, 1024, 1025, 2500])
def test_many_tensors(count):
    """More tensors than one table holds, of either size, some empty; in another order than their addresses."""
    gen = torch.Generator(device="cuda").manual_seed(count)
    sizes = [(i * 37) % 301 for i in range(count)]
    flat = torch.randn(sum(sizes), device="cuda", generator=gen)
    at = np.concatenate([[0], np.cumsum(sizes)])
    order = np.random.RandomState(count).permutation(count)
    src = [flat[at[i]:at[i + 1]] for i in order]
    out, result = torch.zeros(2, device="cuda"), torch.zeros_like(flat)
    dst = [result[at[i]:at[i + 1]] for i in order]
    before = [f64(s) for s in src]
    lists = pb.TensorList(src, dst)
    assert pb.clip_tensors(lists, 3.0, norm_and_scale=out) == pb.OK
    check([flat], [result], [f64(flat)], 3.0, out)
    check(src, dst, before, 3.0, out)
    again, first = torch.zeros(2, device="cuda"), result.clone()
    assert pb.clip_tensors(lists, 3.0, norm_and_scale=again) == pb.OK
    assert torch.equal(out, again) and torch.equal(result, first)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e18, 1e30])
def test_values_whose_squares_leave_the_range_of_float(dtype, scale):
    gen = torch.Generator(device="cuda").manual_seed(1)
    src = lay([40_000, 77], dtype, 0, gen, scale)
    src[1][5] = 0.0
    dst = [torch.empty_like(s) for s in src]
    out = torch.zeros(2, device="cuda")
    total = math.sqrt(sum(float((f64(s) ** 2).sum()) for s in src))
    clip = float(np.float32(0.5 * total))
    assert pb.clip_tensors(pb.TensorList(src, dst), clip, norm_and_scale=out) == pb.OK
    check(src, dst, [f64(s) for s in src], clip, out)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan, 3e38])
@pytest.mark.parametrize("where", [0, 4095, 9999])
def test_a_norm_that_is_not_finite_leaves_everything_as_it_is(dtype, bad, where):
    src = [torch.ones(10_000, dtype=dtype, device="cuda"), torch.ones(3, dtype=dtype, device="cuda")]
    src[0][where] = bad
    if bad == 3e38:
        src[0][where - 1] = src[0][(where + 1) % 10_000] = bad          # finite, but not their norm
    before = [s.clone() for s in src]
    dst = [torch.full_like(src[0], 5.0), src[1]]
    out = torch.ones(2, device="cuda")
    assert pb.clip_tensors(pb.TensorList(src, dst), 1.0, norm_and_scale=out) == pb.OK
    assert not math.isfinite(float(out[0])) and float(out[1]) == 0.0
    assert bool((dst[0] == 5).all())
    assert all(torch.equal(s.view(torch.int16), b.view(torch.int16)) for s, b in zip(src, before))


def test_empty_lists_have_the_norm_0():
    for src in ([], [torch.empty(0, device="cuda")]):
        out = torch.full((2,), 9.0, device="cuda")
        assert pb.clip_tensors(pb.TensorList(src, list(src)), 1.0, norm_and_scale=out) == pb.OK
        assert out.tolist() == [0.0, 1.0]


def test_without_the_norm_told_and_on_another_stream():
    gen = torch.Generator(device="cuda").manual_seed(2)
    src = lay([50_000, 9], F, 0, gen)
    side = torch.cuda.Stream()
    want = [f64(s) / math.sqrt(sum(float((f64(t) ** 2).sum()) for t in src)) for s in src]
    lists = pb.TensorList(src, src)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert pb.clip_tensors(lists, 1.0) == pb.OK
    side.synchronize()
    for s, w in zip(src, want):
        assert np.all(np.abs(f64(s) - w) <= np.abs(w) * (NORM + 6 * U))


@pytest.mark.parametrize("sizes", [(30_000, 100, 64), (3_000_000, 5, 77)])
def test_recorded_and_replayed(sizes):
    gen = torch.Generator(device="cuda").manual_seed(4)
    src = [torch.empty(n, device="cuda") for n in sizes]
    flat = torch.zeros(sum(sizes), device="cuda")
    dst = list(torch.split(flat, list(sizes)))
    out, lists = torch.zeros(2, device="cuda"), pb.TensorList(src, dst)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert pb.clip_tensors(lists, 10.0, norm_and_scale=out) == pb.OK
    for k in range(3):
        for s in src:
            s.copy_(torch.randn(s.shape, device="cuda", generator=gen) * (0.01 + k))
        before = [f64(s) for s in src]
        g.replay()
        torch.cuda.synchronize()
        check(src, dst, before, 10.0, out)


def test_more_than_two_to_the_31_elements():
    """A tensor whose offsets do not fit 32 bits, and one behind it."""
    n = 2 ** 31 + 70_001
    src = torch.full((n,), 0.5, dtype=H, device="cuda")
    src[-1], src[2 ** 31] = 3.0, -2.0
    tail = torch.ones(5, device="cuda")
    out = torch.zeros(2, device="cuda")
    total = math.sqrt(0.25 * (n - 2) + 9 + 4 + 5)
    assert pb.clip_tensors(pb.TensorList([src, tail], [src, tail]), total / 2, norm_and_scale=out) == pb.OK
    assert abs(float(out[0]) - total) <= NORM * total
    assert float(src[-1]) == 1.5 and float(src[2 ** 31]) == -1.0 and float(src[0]) == 0.25 and bool((src[2 ** 31 + 1:-1] == 0.25).all())
    assert bool((src[:2 ** 31].view(torch.int16) == src[0].view(torch.int16)).all())


@pytest.mark.parametrize("count", [64, 65, 320, 321, 1024, 1025])
@pytest.mark.parametrize("size", [40, 3000])
def test_tables_that_are_full(count, size):
    """Lists that fill a table of 64, 320 or 1,024 tensors to the last place, and one more; and behind a full one nothing but empty tensors.
    Together no more than one cluster takes, and more."""
    gen = torch.Generator(device="cuda").manual_seed(count)
    for empty in (0, 3):
        sizes = [1 + (i * 7) % size for i in range(count)] + [0] * empty
        flat = torch.randn(sum(sizes), device="cuda", generator=gen)
        result = torch.zeros(sum(sizes), device="cuda")
        src, dst = list(torch.split(flat, sizes)), list(torch.split(result, sizes))
        out = torch.zeros(2, device="cuda")
        assert pb.clip_tensors(pb.TensorList(src, dst), 3.0, norm_and_scale=out) == pb.OK
        check([flat], [result], [f64(flat)], 3.0, out)
        before = f64(flat)
        assert pb.clip_tensors(pb.TensorList(src, src), 3.0, norm_and_scale=out) == pb.OK
        check([flat], [flat], [before], 3.0, out)
