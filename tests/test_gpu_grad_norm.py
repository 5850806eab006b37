"""The norm of many tensors, clipped copies of them and the clipped SGD step, against plain float64 computations."""
import math
import random

import pytest
import torch

from gpu_helpers import guarded, workspace
from paper_1602_06709_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


def smallest(t):
    f = torch.finfo(t)
    return f.tiny * f.eps / 2


def make(sizes, types, std, seed, lead=0):
    """Guarded tensors; lead: elements by which each starts behind a 16-byte boundary."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for n, t in zip(sizes, types):
        a = guarded((n + lead,), t, fill=0)[lead:]
        a.copy_(torch.randn(n, device="cuda", generator=g) * std)
        out.append(a)
    return out


def norm_of(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


# (an fp32 sum is of 32 squares; half of its rounding errors reach the root, and the result is rounded once)
NORM_ERROR = (32 / 2 + 2) * U


def scalar():
    return guarded((1,), torch.float32)


def check_norm(norm, want):
    assert abs(float(norm) - want) <= want * NORM_ERROR, (float(norm), want)


def factor_of(want, max_norm):
    return min(1.0, max_norm / (want + 1e-6))


CASES = [([1], 0), ([0, 5, 0], 1), ([7, 1, 4096, 4097], 1), ([8191, 8192, 8193, 33], 3), ([100000, 3, 65536, 12345], 0), ([1000003], 1), ([2500000, 17], 0)]


@pytest.mark.parametrize("t", TYPES + ["mixed"])
@pytest.mark.parametrize("sizes,lead", CASES)
@pytest.mark.parametrize("max_norm", [0.5, 1e9, 0.0])
def test_norm_clip_and_step(sizes, lead, t, max_norm):
    types = [TYPES[i % 3] for i in range(len(sizes))] if t == "mixed" else [t] * len(sizes)
    grads = make(sizes, types, 0.1, 1, lead)
    want = norm_of(grads)
    gl, norm = B.TensorList(grads), scalar()
    ws = workspace(B.grad_norm_workspace_bytes(gl))
    B.grad_norm(gl, norm, ws)
    check_norm(norm, want)
    f = factor_of(want, max_norm)
    # clipped copies (which start elsewhere within 16 bytes), then in place
    out = make(sizes, types, 1.0, 2, 0)
    norm.fill_(-1)
    B.grad_clip(gl, B.TensorList(out), max_norm, norm, ws)
    check_norm(norm, want)
    for g, o, tt in zip(grads, out, types):
        e = g.double() * f
        assert ((o.double() - e).abs() <= e.abs() * (half_step(tt) + 2 * NORM_ERROR) + smallest(tt)).all()
    same = [g.clone() for g in grads]
    sl = B.TensorList(same)
    B.grad_clip(sl, sl, max_norm, norm, ws)
    assert all(torch.equal(a, b) for a, b in zip(same, out))
    # the step
    params = make(sizes, types, 1.0, 3, lead)
    before = [p.clone() for p in params]
    B.sgd_update_clipped(B.TensorList(params), gl, 0.25, max_norm, norm, ws)
    check_norm(norm, want)
    for w, b, g, tt in zip(params, before, grads, types):
        step = 0.25 * f * g.double()
        e = b.double() - step
        # (one rounding to the type, one of the product's factor, one of the sum)
        assert ((w.double() - e).abs() <= e.abs() * (half_step(tt) + 2 * U) + step.abs() * (2 * NORM_ERROR + half_step(tt)) + smallest(tt)).all()


def test_unclipped_is_the_plain_step_bit_for_bit():
    """A factor of 1 leaves gradients as they are and the step that of pcl_sgd_update."""
    grads, params = make([5001], [torch.float32], 0.1, 1), make([5001], [torch.float32], 1.0, 2)
    other, out, norm = params[0].clone(), torch.empty_like(grads[0]), scalar()
    gl = B.TensorList(grads)
    ws = workspace(B.grad_norm_workspace_bytes(1))
    B.sgd_update_clipped(B.TensorList(params), gl, 0.1, float("inf"), norm, ws)
    B.sgd_update(other, grads[0], 0.1)
    assert torch.equal(params[0], other)
    B.grad_clip(gl, B.TensorList([out]), 1e30, norm, ws)
    assert torch.equal(out, grads[0])


@pytest.mark.parametrize("count", [1, 31, 32, 33, 127, 129, 639, 640, 641, 1500])
def test_many_tensors(count):
    """More tensors than one launch takes, views of one buffer that start anywhere."""
    r = random.Random(count)
    sizes = [r.choice([0, 1, 2, 3, 17, 100, 1023]) for _ in range(count - 1)] + [5]
    types = [torch.float32 if i % 2 else torch.bfloat16 for i in range(count)]
    flat32, flat16 = guarded((sum(sizes) + 1,), torch.float32, fill=0), guarded((sum(sizes) + 1,), torch.bfloat16, fill=0)
    g = torch.Generator(device="cuda").manual_seed(3)
    grads, at = [], 0
    for n, t in zip(sizes, types):
        v = (flat32 if t == torch.float32 else flat16)[at:at + n]
        v.copy_(torch.randn(n, device="cuda", generator=g))
        grads.append(v)
        at += n
    want, before = norm_of(grads), [x.clone() for x in grads]
    gl, norm = B.TensorList(grads), scalar()
    ws = workspace(B.grad_norm_workspace_bytes(gl))
    B.grad_norm(gl, norm, ws)
    check_norm(norm, want)
    norm.fill_(-1)
    B.grad_clip(gl, gl, want / 2, norm, ws)
    check_norm(norm, want)
    for a, b, t in zip(grads, before, types):
        e = b.double() * factor_of(want, want / 2)
        assert ((a.double() - e).abs() <= e.abs() * (half_step(t) + 3 * NORM_ERROR)).all()


def test_all_empty():
    e, norm = torch.empty(0, device="cuda"), scalar()
    gl = B.TensorList([e, e])
    ws = workspace(B.grad_norm_workspace_bytes(gl))
    B.grad_norm(gl, norm, ws)
    assert float(norm) == 0
    norm.fill_(5)
    B.grad_clip(gl, gl, 1.0, norm, ws)
    assert float(norm) == 0


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1e-44, 1e-38, 1e-30, 1e-20, 1e20, 1e30, 3e37])
def test_values_whose_squares_leave_fp32(t, size):
    """Norms that fp32 squares would lose, alone and beside ordinary values."""
    n = 4100
    g = guarded((n,), torch.float32, fill=0)
    g.copy_(torch.linspace(0.5, 1.0, n, device="cuda").double() * size)
    g = g.to(t)
    norm, gl = scalar(), B.TensorList([g])
    ws = workspace(B.grad_norm_workspace_bytes(gl))
    B.grad_norm(gl, norm, ws)
    want = norm_of([g])
    if want < 3.4e38:
        assert abs(float(norm) - want) <= want * NORM_ERROR + 2.0 ** -149
    else:
        assert math.isinf(float(norm))
    # (the factor is below fp32's normal numbers for the largest of these: multiples of 2^-149)
    out = torch.empty_like(g)
    B.grad_clip(gl, B.TensorList([out]), 1.0, norm, ws)
    f = factor_of(want, 1.0)
    e = g.double() * f
    assert ((out.double() - e).abs() <= e.abs() * (half_step(t) + 2 * NORM_ERROR + 2.0 ** -150 / f) + smallest(t)).all()
    g[::64] = 1.0
    B.grad_norm(gl, norm, ws)
    want = norm_of([g])
    assert abs(float(norm) - want) <= want * NORM_ERROR or want > 3.4e38


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_not_finite(bad):
    grads, norm = make([1000, 3000], [torch.float32] * 2, 1.0, 1), scalar()
    grads[1][2999] = bad
    gl = B.TensorList(grads)
    ws = workspace(B.grad_norm_workspace_bytes(gl))
    out = [torch.empty_like(g) for g in grads]
    B.grad_clip(gl, B.TensorList(out), 1.0, norm, ws)
    if math.isnan(bad):
        assert math.isnan(float(norm)) and all(torch.isnan(o).all() for o in out)
    else:
        assert float(norm) == math.inf and (out[0] == 0).all() and (out[1][:2999] == 0).all() and torch.isnan(out[1][2999])


def test_repeatable_captured_and_on_two_streams():
    sizes, types = [700001, 12, 33333], [torch.bfloat16, torch.float32, torch.float16]
    grads, params = make(sizes, types, 0.1, 1), make(sizes, types, 1.0, 2)
    gl, pl, norm = B.TensorList(grads), B.TensorList(params), scalar()
    ws = workspace(B.grad_norm_workspace_bytes(gl))
    start = [p.clone() for p in params]
    B.sgd_update_clipped(pl, gl, 0.1, 1.0, norm, ws)
    once, first = [p.clone() for p in params], norm.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.sgd_update_clipped(pl, gl, 0.1, 1.0, norm, ws)
    other, onorm = make(sizes, types, 0.3, 5), scalar()
    ol, ows, side = B.TensorList(other), workspace(B.grad_norm_workspace_bytes(3)), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        for p, s in zip(params, start):
            p.copy_(s)
        graph.replay()
        with torch.cuda.stream(side):
            B.grad_norm(ol, onorm, ows)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(params, once)) and torch.equal(norm, first)
        check_norm(onorm, norm_of(other))


def test_more_than_2_to_31_elements():
    n = 2 ** 31 + 77
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-1], g[0], g[2 ** 31] = 3.0, 4.0, 12.0
    gl, norm = B.TensorList([g]), scalar()
    ws = workspace(B.grad_norm_workspace_bytes(gl))
    B.grad_clip(gl, gl, 6.5, norm, ws)
    f = 6.5 / (13 + 1e-6)
    assert abs(float(norm) - 13) <= 13 * NORM_ERROR
    for i, v in ((n - 1, 3.0), (0, 4.0), (2 ** 31, 12.0), (5, 0.0)):
        assert abs(float(g[i]) - v * f) <= v * f * (half_step(torch.bfloat16) + 2 * NORM_ERROR)


def test_tensors_that_are_written_twice_are_refused():
    """A list that overlaps itself can be read (every mention counts), not written."""
    flat = torch.arange(1.0, 65.0, device="cuda")
    a, b = flat[:40], flat[36:]
    twice, apart, norm, ws = B.TensorList([a, b]), B.TensorList([a.clone(), b.clone()]), scalar(), workspace(B.grad_norm_workspace_bytes(2))
    B.grad_norm(twice, norm, ws)
    check_norm(norm, norm_of([a, b]))
    with pytest.raises(ValueError):
        B.grad_clip(apart, twice, 1.0, norm, ws)
    with pytest.raises(ValueError):
        B.grad_clip(twice, twice, 1.0, norm, ws)
    with pytest.raises(ValueError):
        B.sgd_update_clipped(twice, apart, 0.1, 1.0, norm, ws)
    B.grad_clip(twice, apart, 1.0, norm, ws)
    assert torch.equal(flat, torch.arange(1.0, 65.0, device="cuda"))
    B.grad_norm(B.TensorList([flat[:36], flat[36:], flat[:0]]), norm, workspace(B.grad_norm_workspace_bytes(3)))
    assert not B.TensorList([flat[:36], flat[36:], flat[:0], flat[5:5]]).overlaps
