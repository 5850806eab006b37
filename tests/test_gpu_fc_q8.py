"""FC layer of 8-bit operands against plain float64 computations."""
import pytest
import torch

from gpu_helpers import guarded, workspace
from paper_1602_06709_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
ACTS = [B.ACT_NONE, B.ACT_RELU, B.ACT_SIGMOID]
U = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


def smallest(t):
    f = torch.finfo(t)
    return f.tiny * f.eps / 2


def bytes8(v):
    q = guarded(v.shape, torch.uint8, fill=0x55)
    q.copy_(v.to(B.E4M3).view(torch.uint8))
    return q


def whole(shape, seed):
    """Whole numbers from -4 to 4: every product and every sum of up to 2^20 of them is exact in fp32, in any order."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return bytes8(torch.randint(-4, 5, shape, device="cuda", generator=g).float())


def scales(n, size, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = guarded((n,), torch.float32)
    s.copy_((torch.rand(n, device="cuda", generator=g) + 0.5) * size)
    return s


def expected(x, xs, w, ws, bias, act):
    """The result, and the size of what is added up in front of the activation."""
    acc = x.view(B.E4M3).double() @ w.view(B.E4M3).double().T
    z = acc * xs.double()[:, None] * ws.double()
    size = z.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    if act == B.ACT_RELU:
        return z.clamp(min=0), size, z
    if act == B.ACT_SIGMOID:
        return torch.sigmoid(z), size, z
    return z, size, z


def check(y, t, act, want, size, z, sum_error=0.0):
    if act == B.ACT_SIGMOID:
        # (exp: 2 + 1.173 |z| units of 2^-23, quotient and sum three; the slope is at most 1/4 and at most the value)
        slope = torch.minimum(want, torch.full_like(want, 0.25))
        error = want * (8 + 1.2 * z.abs()) * 2 * U + slope * (size * 4 * U + sum_error)
    else:
        error = size * 4 * U + sum_error           # (two products and a sum)
    assert ((y.double() - want).abs() <= want.abs() * half_step(t) + error * (1 + half_step(t)) + smallest(t)).all()


SHAPES = [(1, 1, 1), (1, 16, 8), (2, 17, 3), (3, 32, 100), (16, 4096, 1000), (1, 4096, 16384), (127, 48, 129), (128, 128, 128), (129, 160, 255),
          (256, 256, 256), (257, 1032, 264), (300, 1037, 301), (1000, 5, 77), (1024, 2048, 2048), (700, 130, 4100), (2, 100000, 40), (64, 8192, 50)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,C,K", SHAPES)
@pytest.mark.parametrize("act", ACTS)
def test_exact_sums(N, C, K, t, act):
    x, w = whole((N, C), 1), whole((K, C), 2)
    xs, ws = scales(N, 0.1, 3), scales(K, 5.0 / C ** 0.5, 4)
    bias = None
    if act != B.ACT_RELU:
        bias = guarded((K,), t, fill=0)
        bias.copy_(torch.randn(K, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)))
    y = guarded((N, K), t)
    space = workspace(B.fc_q8_workspace_bytes(N, C, K))
    B.fc_q8_fwd(N, C, K, x, xs, w, ws, bias, y, act, space)
    check(y, t, act, *expected(x, xs, w, ws, bias, act))
    y2 = guarded((N, K), t)
    B.fc_q8_fwd(N, C, K, x.view(B.E4M3), xs, w.view(B.E4M3), ws, bias, y2, act, space)       # (the workspace as the call before left it)
    assert torch.equal(y, y2)
    assert B.last_device_status() == B.OK


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,C,K", [(5, 64, 33), (130, 1037, 520), (300, 4096, 700)])
def test_all_values(N, C, K, t):
    """Operands with all finite e4m3 values, as the norm writes them.  The tensor core aligns the 32 products of a step and the accumulator to
    the largest of them and cuts what lies below 24 bits: 33 / 32 C times 2^-23 of the largest partial sum, at worst the sum of all sizes."""
    g = torch.Generator(device="cuda").manual_seed(9)
    x, w = guarded((N, C), torch.uint8, fill=0), guarded((K, C), torch.uint8, fill=0)
    for q in (x, w):
        q.copy_(torch.randint(0, 256, q.shape, device="cuda", generator=g).to(torch.uint8))
        q[(q & 0x7f) == 0x7f] = 0x38
    xs, ws, y = scales(N, 1e-3, 3), scales(K, 1e-4, 4), guarded((N, K), t)
    B.fc_q8_fwd(N, C, K, x, xs, w, ws, None, y, ws=workspace(B.fc_q8_workspace_bytes(N, C, K)))
    want, size, z = expected(x, xs, w, ws, None, B.ACT_NONE)
    total = x.view(B.E4M3).double().abs() @ w.view(B.E4M3).double().abs().T * xs.double()[:, None] * ws.double()
    check(y, t, B.ACT_NONE, want, size, z, total * (33 / 32 * C) * 2 * U)
    # and, as measured errors of such sums are far below that bound: to 2^-13 of the result's own size (2-norm)
    assert (y.double() - want).norm() <= want.norm() * (half_step(t) + 2.0 ** -13)


def test_not_finite():
    """A row with a NaN, or with a scale that is not finite, spoils itself only."""
    N, C, K = 6, 64, 40
    x, w, xs, ws = whole((N, C), 1), whole((K, C), 2), scales(N, 1.0, 3), scales(K, 1.0, 4)
    x[1, 5] = 0x7f
    xs[3] = float("nan")
    xs[4] = float("inf")
    y = guarded((N, K), torch.float32)
    B.fc_q8_fwd(N, C, K, x, xs, w, ws, None, y, B.ACT_RELU, workspace(B.fc_q8_workspace_bytes(N, C, K)))
    assert torch.isnan(y[1]).all() and torch.isnan(y[3]).all() and not torch.isfinite(y[4]).all()
    rows = [0, 2, 5]
    check(y[rows], torch.float32, B.ACT_RELU, *(v[rows] for v in expected(x, xs, w, ws, None, B.ACT_RELU)))


def test_captured_and_on_two_streams():
    N, C, K, t = 40, 520, 900, torch.bfloat16
    x, w, xs, ws = whole((N, C), 1), whole((K, C), 2), scales(N, 1.0, 3), scales(K, 1.0, 4)
    y, y2 = guarded((N, K), t), guarded((N, K), t)
    s1, s2 = (workspace(B.fc_q8_workspace_bytes(N, C, K)) for _ in range(2))
    B.fc_q8_fwd(N, C, K, x, xs, w, ws, None, y, ws=s1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.fc_q8_fwd(N, C, K, x, xs, w, ws, None, y, ws=s1)
    side = torch.cuda.Stream()
    for seed in (11, 12):
        x.copy_(whole((N, C), seed))
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            B.fc_q8_fwd(N, C, K, x, xs, w, ws, None, y2, ws=s2)
        torch.cuda.synchronize()
        check(y, t, B.ACT_NONE, *expected(x, xs, w, ws, None, B.ACT_NONE))
        assert torch.equal(y, y2)


def test_more_than_2_to_31_elements():
    N, C, K = 33000, 32, 65600
    x, w, xs, ws = whole((N, C), 1), whole((K, C), 2), scales(N, 1.0, 3), scales(K, 1.0, 4)
    y = torch.empty(N, K, dtype=torch.bfloat16, device="cuda")
    B.fc_q8_fwd(N, C, K, x, xs, w, ws, None, y, ws=workspace(B.fc_q8_workspace_bytes(N, C, K)))
    for r in (slice(0, 2), slice(2 ** 31 // K - 1, 2 ** 31 // K + 2), slice(N - 2, N)):
        check(y[r], torch.bfloat16, B.ACT_NONE, *expected(x[r], xs[r], w, ws, None, B.ACT_NONE))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N", [1, 8, 9, 64, 113, 120, 121])
@pytest.mark.parametrize("C,K", [(4096, 16384), (1037, 300), (64, 40)])
def test_few_rows_behind_a_call_of_nan(N, C, K, t):
    """Rows of a tile that x does not have hold what another call left in shared memory: NaN there do not reach the result."""
    big = 512
    nan, one, y0 = guarded((big, 512), torch.uint8, fill=0x7f), guarded((20480,), torch.float32, fill=1.0), guarded((big, 20480), torch.bfloat16, fill=0)
    w0 = guarded((20480, 512), torch.uint8, fill=0x7f)
    x, w = whole((N, C), 1), whole((K, C), 2)
    xs, ws, y = scales(N, 0.1, 3), scales(K, 5.0 / C ** 0.5, 4), guarded((N, K), t)
    space = workspace(B.fc_q8_workspace_bytes(N, C, K))
    B.fc_q8_fwd(big, 512, 20480, nan, one[:big], w0, one, None, y0, ws=workspace(B.fc_q8_workspace_bytes(big, 512, 20480)))
    B.fc_q8_fwd(N, C, K, x, xs, w, ws, None, y, ws=space)
    check(y, t, B.ACT_NONE, *expected(x, xs, w, ws, None, B.ACT_NONE))
    assert torch.isnan(y0).all()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_RELU])
@pytest.mark.parametrize("xs,ws", [(1e36, 1e-38), (1e-38, 1e36), (2.0 ** -126, 1e30), (1e30, 2.0 ** -126), (1e35, 1e-10)])
@pytest.mark.parametrize("N,C,K", [(5, 4096, 72), (300, 1037, 301)])
def test_scales_far_apart(N, C, K, xs, ws, act, t):
    """Scales that cancel: neither may take the sum out of fp32's range on the way; beside them rows of ordinary scales, which do not notice."""
    x, w = whole((N, C), 1), whole((K, C), 2)
    a, b = scales(N, xs, 3), scales(K, ws, 4)
    b[::2] = scales(len(b[::2]), 1.0, 6)
    a[1::3] = 1.5
    a.clamp_(min=2.0 ** -126), b.clamp_(min=2.0 ** -126)       # (the least that a scale can be)
    y = guarded((N, K), t)
    B.fc_q8_fwd(N, C, K, x, a, w, b, None, y, act, workspace(B.fc_q8_workspace_bytes(N, C, K)))
    want, size, z = expected(x, a, w, b, None, act)
    fits = want.abs() < torch.finfo(t).max * 0.99
    assert bool(fits.any())
    zero = torch.zeros_like(want)
    check(torch.where(fits, y.double(), zero), t, act, *(torch.where(fits, v, zero) for v in (want, size, z)))
    assert (torch.isinf(y) | fits | (want.abs() < torch.finfo(t).max * 1.01)).all()
    plain, again = a.clone(), guarded((N, K), t)
    plain[0::3] = 1.0
    plain[2::3] = 1.0
    B.fc_q8_fwd(N, C, K, x, plain, w, b, None, again, act, workspace(B.fc_q8_workspace_bytes(N, C, K)))
    assert torch.equal(again[1::3], y[1::3])
