"""RMS norm with the residual's addition, its 8-bit form and its gradient, and 8-bit rows, against plain float64 computations."""
import pytest
import torch

from gpu_helpers import guarded, workspace
from paper_1602_06709_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24          # half a step of fp32


def half_step(t):
    return torch.finfo(t).eps / 2


def smallest(t):
    """Half of the spacing of the subnormal numbers."""
    f = torch.finfo(t)
    return f.tiny * f.eps / 2


def put(shape, t, std, seed, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = guarded(shape, t, fill=0)
    out.copy_(torch.randn(shape, device="cuda", generator=g) * std + mean)
    return out


def bytes8(shape):
    return guarded(shape, torch.uint8, fill=0x55)


def additions(n):
    """Most additions in fp32 on the way of one term of a row of n: a thread's own (32 at most, or every 1024th element of longer rows) and
    two levels of threads."""
    return 32 + max(0, n - 32768) // 1024 + 5 + 32


def forward_reference(x, res, w, eps):
    h = x.double() if res is None else x.double() + res.double()
    rstd = (h.square().mean(dim=1) + eps) ** -0.5
    return h, rstd, h * rstd[:, None] * w.double()


def check_forward(N, C, t, x, res, w, eps, h, y, rstd):
    eh, er, ey = forward_reference(x, res, w, eps)
    k = additions(C)
    # (the sum of squares: k additions of one sign; half of that in its root; the products with 1/C, of the root and of y: three more)
    assert ((rstd.double() - er).abs() <= er * (k / 2 + 3) * U).all()
    if res is not None:
        assert ((h.double() - eh).abs() <= eh.abs() * (half_step(t) + U) + smallest(t)).all()
    bound = ey.abs() * (half_step(t) + (k / 2 + 6) * U * (1 + half_step(t))) + smallest(t)
    assert ((y.double() - ey).abs() <= bound).all()


SHAPES = [(1, 1), (1, 2048), (2, 7), (3, 8), (5, 33), (64, 64), (17, 100), (9, 255), (700, 257), (33, 1000), (301, 1037), (6, 4096), (1201, 2048),
          (5, 5001), (2, 8200), (3, 16384), (2, 16390), (2, 32768), (2, 32771), (1, 70001)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,C", SHAPES)
@pytest.mark.parametrize("with_res", [False, True])
def test_forward(N, C, t, with_res):
    x, w = put((N, C), t, 0.7, 1), put((C,), t, 0.3, 2, 1.0)
    res = put((N, C), t, 2.0, 3) if with_res else None
    h = guarded((N, C), t) if with_res else None
    y, rstd = guarded((N, C), t), guarded((N,), torch.float32)
    B.rms_norm_fwd(N, C, x, res, w, 1e-6, h, y, rstd)
    check_forward(N, C, t, x, res, w, 1e-6, h, y, rstd)
    # without the optional outputs; and the same again, bit for bit
    y2 = guarded((N, C), t)
    B.rms_norm_fwd(N, C, x, res, w, 1e-6, None, y2)
    assert torch.equal(y, y2)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,C", [(7, 64), (300, 1037), (5, 5001), (2, 32771)])
def test_forward_in_place(N, C, t):
    """h over the residual, y over x."""
    x, res, w = put((N, C), t, 0.7, 1), put((N, C), t, 2.0, 3), put((C,), t, 0.3, 2, 1.0)
    h, y = guarded((N, C), t), guarded((N, C), t)
    B.rms_norm_fwd(N, C, x, res, w, 1e-5, h, y)
    x2, res2 = x.clone(), res.clone()
    B.rms_norm_fwd(N, C, x2, res2, w, 1e-5, res2, guarded((N, C), t))
    assert torch.equal(res2, h)
    if C <= 32768 // (2 if t == torch.float32 else 1):      # (longer rows read their inputs twice)
        x3 = x.clone()
        B.rms_norm_fwd(N, C, x3, res, w, 1e-5, h, x3)
        assert torch.equal(x3, y)


@pytest.mark.parametrize("C", [96, 40001])
@pytest.mark.parametrize("std", [1e30, 3e37, 1e-12, 1e-30, 3e-38])
def test_rows_out_of_range_of_their_squares(std, C):
    """Rows whose squares fp32 does not hold, beside an ordinary one; eps 0, so that nothing covers them."""
    x, w = put((4, C), torch.float32, 1.0, 5).clamp_(-4, 4), put((C,), torch.float32, 0.3, 2, 1.0)
    x[::2] *= std
    y, rstd = guarded((4, C), torch.float32), guarded((4,), torch.float32)
    B.rms_norm_fwd(4, C, x, None, w, 0.0, None, y, rstd)
    _, er, ey = forward_reference(x, None, w, 0.0)
    k = additions(C)
    # (1 / 3e37 lies below the normal numbers: rstd is then a multiple of 2^-149; the row's values come from its scaled form)
    assert ((rstd.double() - er).abs() <= er * (k / 2 + 4) * U + 2.0 ** -149).all()
    assert ((y.double() - ey).abs() <= ey.abs() * (k / 2 + 8) * U + 2.0 ** -100).all()


def test_rows_out_of_range_with_eps():
    """Tiny rows under a tiny eps, which takes part in the sum."""
    C = 128
    x, w = put((3, C), torch.float32, 1.0, 5), put((C,), torch.float32, 0.3, 2, 1.0)
    x *= torch.tensor([[1e-11], [1e-16], [1e-25]], device="cuda")
    y, rstd = guarded((3, C), torch.float32), guarded((3,), torch.float32)
    B.rms_norm_fwd(3, C, x, None, w, 1e-24, None, y, rstd)
    eps = float(torch.tensor(1e-24))
    _, er, ey = forward_reference(x, None, w, eps)
    assert ((rstd.double() - er).abs() <= er * 40 * U).all()
    assert ((y.double() - ey).abs() <= ey.abs() * 45 * U).all()


@pytest.mark.parametrize("C", [64, 1037, 40001])
@pytest.mark.parametrize("t", TYPES)
def test_zeros_infinities_and_nan(t, C):
    x, w = put((5, C), t, 1.0, 7), put((C,), t, 0.3, 2, 1.0)
    x[1] = 0
    x[2, C // 2] = float("inf")
    x[3, C - 1] = float("nan")
    y, rstd = guarded((5, C), t), guarded((5,), torch.float32)
    B.rms_norm_fwd(5, C, x, None, w, 1e-6, None, y, rstd)
    assert (y[1] == 0).all() and torch.isnan(y[3]).all() and torch.isnan(y[2, C // 2])
    others = torch.arange(C, device="cuda") != C // 2
    assert (y[2][others] == 0).all() and rstd[2] == 0 and torch.isnan(rstd[3])
    for row in (0, 4):
        one = slice(row, row + 1)
        check_forward(1, C, t, x[one], None, w, 1e-6, None, y[one], rstd[one])
    q, scale = bytes8((5, C)), guarded((5,), torch.float32)
    B.rms_norm_fwd_q8(5, C, x, None, w, 1e-6, None, q, scale)
    assert scale[1] == 2.0 ** -126 and (q.view(B.E4M3).float()[1] == 0).all() and not torch.isfinite(scale[2]) and torch.isnan(scale[3])
    assert torch.isfinite(scale[[0, 4]]).all() and torch.isnan(q.view(B.E4M3).float()[3]).all()


def check_q8(q, scale, y, k):
    """Against y in 64 bits: the scale to k roundings; the values to half a step of e4m3 (2^-4 of the value, 2^-10 among the
    subnormals) after those roundings."""
    q = q.view(B.E4M3).double()
    top = y.abs().amax(dim=1)
    want = (top / 448).clamp(min=2.0 ** -126)
    assert ((scale.double() - want).abs() <= want * k * U).all()
    v = y / scale.double()[:, None]
    assert ((q - v).abs() <= v.abs() * (2.0 ** -4 + 2 * k * U) + 2.0 ** -10 * (1 + k * U)).all()
    assert (q.abs().amax(dim=1)[top > 1e-30] == 448).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,C", SHAPES)
def test_forward_q8(N, C, t):
    x, res, w = put((N, C), t, 0.7, 1), put((N, C), t, 2.0, 3), put((C,), t, 0.3, 2, 1.0)
    h, q, scale, rstd = guarded((N, C), t), bytes8((N, C)), guarded((N,), torch.float32), guarded((N,), torch.float32)
    B.rms_norm_fwd_q8(N, C, x, res, w, 1e-6, h, q, scale, rstd)
    _, er, ey = forward_reference(x, res, w, 1e-6)
    k = additions(C)
    assert ((rstd.double() - er).abs() <= er * (k / 2 + 3) * U).all()
    check_q8(q, scale, ey, k / 2 + 8)
    h2, y = guarded((N, C), t), guarded((N, C), t)
    B.rms_norm_fwd(N, C, x, res, w, 1e-6, h2, y)
    assert torch.equal(h, h2)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,C", SHAPES)
def test_quantize_rows(N, C, t):
    x = put((N, C), t, 3.0, 1)
    if N > 2:
        x[1] = 0
        x[2] *= 1e-4
    q, scale = bytes8((N, C)), guarded((N,), torch.float32)
    B.quantize_rows(N, C, x, q, scale)
    check_q8(q, scale, x.double(), 4)


def test_quantize_tiny_rows():
    """Values below 2^-126 have a scale that can be divided by."""
    x = guarded((2, 40), torch.float32, fill=0)
    x[0] = 1e-40
    x[1] = 1e-36
    q, scale = bytes8((2, 40)), guarded((2,), torch.float32)
    B.quantize_rows(2, 40, x, q, scale)
    assert scale[0] == 2.0 ** -126
    check_q8(q, scale, x.double(), 4)


def grad_reference(h, w, rstd, dy, dh):
    h, w, r, dy = h.double(), w.double(), rstd.double()[:, None], dy.double()
    n, g = h * r, dy * w
    dx = r * (g - n * (g * n).mean(dim=1, keepdim=True))
    size = r * (g.abs() + n.abs() * (g * n).abs().mean(dim=1, keepdim=True))
    if dh is not None:
        dx, size = dx + dh.double(), size + dh.double().abs()
    return dx, size, (dy * n).sum(dim=0), (dy * n).abs().sum(dim=0)


def check_grad(t, h, w, rstd, dy, dh, dx, dw):
    ex, size, ew, sizew = grad_reference(h, w, rstd, dy, dh)
    k = additions(2 * h.shape[1])
    # (k additions in the mean, and six products and additions around it)
    assert ((dx.double() - ex).abs() <= ex.abs() * half_step(t) + size * (k + 6) * U * (1 + half_step(t)) + smallest(t)).all()
    if dw is not None:
        # (a term of dw passes the additions of its group's rows, of the 16 groups of its block and of the 296 blocks, by 16 at a time)
        kw = -(-h.shape[0] // 288) + 16 + 19 + 16 + 2
        assert ((dw.double() - ew).abs() <= ew.abs() * half_step(t) + sizew * kw * U * (1 + half_step(t)) + smallest(t)).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,C", SHAPES + [(3001, 24), (2500, 1032)])
@pytest.mark.parametrize("with_dh", [False, True])
def test_gradient(N, C, t, with_dh):
    h, w, dy = put((N, C), t, 1.5, 1), put((C,), t, 0.3, 2, 1.0), put((N, C), t, 0.1, 3)
    dh = put((N, C), t, 0.1, 4) if with_dh else None
    rstd = (h.double().square().mean(dim=1) + 1e-6).rsqrt().float()
    dx, dw = guarded((N, C), t), guarded((C,), t)
    ws = workspace(B.rms_norm_workspace_bytes(N, C))
    B.rms_norm_bwd(N, C, h, w, rstd, dy, dh, dx, dw, ws)
    check_grad(t, h, w, rstd, dy, dh, dx, dw)
    dx2 = guarded((N, C), t)
    B.rms_norm_bwd(N, C, h, w, rstd, dy, dh, dx2, None)           # without dw, and without a workspace
    assert torch.equal(dx, dx2)
    dw2 = guarded((C,), t)
    over = dy if dh is None else dh
    B.rms_norm_bwd(N, C, h, w, rstd, dy, dh, over, dw2, ws)       # in place of an input; the same again
    assert torch.equal(over, dx) and torch.equal(dw, dw2)


@pytest.mark.parametrize("residual", [False, True])
def test_gradient_against_differences_and_autograd(residual):
    """The gradient of sum(y * a + h * b) against 64-bit differences of the forward formula, through forward and backward calls."""
    N, C, eps = 5, 37, 1e-3
    x, r, w = put((N, C), torch.float32, 1.0, 1), put((N, C), torch.float32, 1.0, 2), put((C,), torch.float32, 0.3, 3, 1.0)
    a, b = put((N, C), torch.float32, 1.0, 4), put((N, C), torch.float32, 1.0, 5)
    res = r if residual else None
    h, y, rstd = (guarded((N, C), torch.float32) if residual else None), guarded((N, C), torch.float32), guarded((N,), torch.float32)
    B.rms_norm_fwd(N, C, x, res, w, eps, h, y, rstd)
    dx, dw = guarded((N, C), torch.float32), guarded((C,), torch.float32)
    B.rms_norm_bwd(N, C, h if residual else x, w, rstd, a, b, dx, dw, workspace(B.rms_norm_workspace_bytes(N, C)))
    eps32 = float(torch.tensor(eps))

    def total(xd, wd):
        hd = xd + r.double() if residual else xd
        return ((hd * (hd.square().mean(dim=1, keepdim=True) + eps32).rsqrt() * wd) * a.double() + hd * b.double()).sum()

    xd, wd = x.double().requires_grad_(), w.double().requires_grad_()
    gx, gw = torch.autograd.grad(total(xd, wd), (xd, wd))
    # (kernel: 60 roundings of terms of size about 10; the stored h is off by one more, in both factors)
    assert (dx.double() - gx).abs().max() <= 100 * U * 10 and (dw.double() - gw).abs().max() <= 100 * U * 10
    step = 1e-5
    for i, j in ((0, 0), (2, 17), (4, 36)):
        e = torch.zeros(N, C, dtype=torch.float64, device="cuda")
        e[i, j] = step
        diff = (total(x.double() + e, w.double()) - total(x.double() - e, w.double())) / (2 * step)
        assert abs(float(diff) - float(dx[i, j])) <= 1e-4           # (third derivatives of size about 10, times step^2; roundings 1e-12 / step)
        diff = (total(x.double(), w.double() + e[i]) - total(x.double(), w.double() - e[i])) / (2 * step)
        assert abs(float(diff) - float(dw[j])) <= 1e-4


def test_more_than_2_to_31_elements():
    """Rows beyond 2^31 elements: the last ones are right."""
    N, C = 2 ** 20 + 3, 2049
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    t = torch.bfloat16
    x = torch.empty(N, C, dtype=t, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    w, y, rstd = put((C,), t, 0.3, 2, 1.0), torch.empty(N, C, dtype=t, device="cuda"), torch.empty(N, device="cuda")
    B.rms_norm_fwd(N, C, x, None, w, 1e-6, None, y, rstd)
    for rows in (slice(0, 3), slice(2 ** 31 // C - 1, 2 ** 31 // C + 2), slice(N - 3, N)):
        check_forward(3, C, t, x[rows], None, w, 1e-6, None, y[rows], rstd[rows])
    dx = torch.empty_like(x)
    B.rms_norm_bwd(N, C, x, w, rstd, y, None, dx, None)
    for rows in (slice(0, 3), slice(2 ** 31 // C - 1, 2 ** 31 // C + 2), slice(N - 3, N)):
        check_grad(t, x[rows], w, rstd[rows], y[rows], None, dx[rows], None)


def test_streams_and_graph():
    """Captured and replayed with new inputs, beside eager calls on another stream."""
    N, C, t = 130, 520, torch.bfloat16
    x, w, y, rstd = put((N, C), t, 1.0, 1), put((C,), t, 0.3, 2, 1.0), guarded((N, C), t), guarded((N,), torch.float32)
    dy, dx, dw = put((N, C), t, 1.0, 3), guarded((N, C), t), guarded((C,), t)
    ws = workspace(B.rms_norm_workspace_bytes(N, C))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.rms_norm_fwd(N, C, x, None, w, 1e-6, None, y, rstd)
        B.rms_norm_bwd(N, C, x, w, rstd, dy, None, dx, dw, ws)
    x2, y2 = put((N, C), t, 1.0, 9), guarded((N, C), t)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for seed in (11, 12):
        x.copy_(torch.randn(N, C, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
        graph.replay()
        with torch.cuda.stream(side):
            B.rms_norm_fwd(N, C, x2, None, w, 1e-6, None, y2)
        torch.cuda.synchronize()
        check_forward(N, C, t, x, None, w, 1e-6, None, y, rstd)
        check_grad(t, x, w, rstd, dy, None, dx, dw)
        ey = forward_reference(x2, None, w, 1e-6)[2]
        assert ((y2.double() - ey).abs() <= ey.abs() * 1.01 * half_step(t) + smallest(t)).all()


# Enough rows for every way of sharing the blocks out: rows in pairs (odd numbers of rows, too), several rows to a group, one to three blocks an SM.
LONG = [(2371, 4096), (9477, 1000), (18951, 33), (2403, 5120), (2371, 8192), (1201, 16384), (2500, 3333), (700, 15001), (40001, 64), (4801, 2049), (9600, 1001)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,C", LONG)
def test_gradient_of_many_rows(N, C, t):
    h, w, dy, dh = put((N, C), t, 1.5, 1), put((C,), t, 0.3, 2, 1.0), put((N, C), t, 0.1, 3), put((N, C), t, 0.1, 4)
    rstd = (h.double().square().mean(dim=1) + 1e-6).rsqrt().float()
    dx, dw = guarded((N, C), t), guarded((C,), t)
    ws = workspace(B.rms_norm_workspace_bytes(N, C))
    for with_dh in (None, dh):
        B.rms_norm_bwd(N, C, h, w, rstd, dy, with_dh, dx, dw, ws)
        check_grad(t, h, w, rstd, dy, with_dh, dx, dw)
    for over in (dy, h, dh):                                      # in place of each input
        given = [x.clone() for x in (h, dy, dh)]
        at = [x is over for x in (h, dy, dh)].index(True)
        dw2 = guarded((C,), t)
        B.rms_norm_bwd(N, C, given[0], w, rstd, given[1], given[2], given[at], dw2, ws)
        assert torch.equal(given[at], dx) and torch.equal(dw, dw2)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,C", LONG + [(3700, 4096), (7301, 2048), (1803, 8192)])
def test_forward_of_many_rows(N, C, t):
    x, res, w = put((N, C), t, 0.7, 1), put((N, C), t, 2.0, 3), put((C,), t, 0.3, 2, 1.0)
    h, y, rstd = guarded((N, C), t), guarded((N, C), t), guarded((N,), torch.float32)
    B.rms_norm_fwd(N, C, x, None, w, 1e-6, None, y, rstd)
    check_forward(N, C, t, x, None, w, 1e-6, None, y, rstd)
    B.rms_norm_fwd(N, C, x, res, w, 1e-6, h, y, rstd)
    check_forward(N, C, t, x, res, w, 1e-6, h, y, rstd)
    x2, res2 = x.clone(), res.clone()
    B.rms_norm_fwd(N, C, x2, res2, w, 1e-6, res2, x2)             # both in place
    assert torch.equal(x2, y) and torch.equal(res2, h)
    q, scale = bytes8((N, C)), guarded((N,), torch.float32)
    B.rms_norm_fwd_q8(N, C, x, res, w, 1e-6, None, q, scale)
    _, _, ey = forward_reference(x, res, w, 1e-6)
    check_q8(q, scale, ey, additions(C) / 2 + 8)


@pytest.mark.parametrize("C", [96, 100, 4096, 40001])
def test_rows_out_of_range_among_many(C):
    """Rows that are scaled first, zeros, infinities and NaN in the middle of many ordinary ones, which do not notice."""
    N, t = 3700 if C < 10000 else 500, torch.float32
    x, w = put((N, C), t, 1.0, 5).clamp_(-4, 4), put((C,), t, 0.3, 2, 1.0)
    plain, y, rstd = guarded((N, C), t), guarded((N, C), t), guarded((N,), torch.float32)
    B.rms_norm_fwd(N, C, x, None, w, 0.0, None, plain, rstd)
    odd = x.clone()
    odd[5::50] *= 1e30
    odd[6::50] *= 1e-30
    odd[7::50] = 0
    odd[8::50, C // 2] = float("inf")
    odd[9::50, C - 1] = float("nan")
    B.rms_norm_fwd(N, C, odd, None, w, 0.0, None, y, rstd)
    place = torch.arange(N, device="cuda") % 50
    same = (place < 5) | (place > 9)
    assert torch.equal(y[same], plain[same]) and torch.isnan(y[place == 9]).all() and torch.isnan(y[place == 7]).all()
    k = additions(C)
    scaled = (place == 5) | (place == 6)
    _, er, ey = forward_reference(odd[scaled], None, w, 0.0)
    assert ((rstd[scaled].double() - er).abs() <= er * (k / 2 + 4) * U + 2.0 ** -149).all()
    assert ((y[scaled].double() - ey).abs() <= ey.abs() * (k / 2 + 8) * U + 2.0 ** -100).all()
    q, scale = bytes8((N, C)), guarded((N,), torch.float32)
    B.rms_norm_fwd_q8(N, C, odd, None, w, 0.0, None, q, scale)
    check_q8(q[scaled], scale[scaled], ey, k / 2 + 8)
    assert torch.isfinite(scale[same]).all() and not torch.isfinite(scale[place == 8]).any() and torch.isnan(scale[place == 9]).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [8, 16, 24, 32, 40, 64, 96, 128])
@pytest.mark.parametrize("N", [5, 297, 4099, 21001])
def test_weight_gradient_of_short_rows(N, C, t):
    """Rows that 4, 8 or 16 lanes of a warp share: only the first group's lanes hold the warp's sums of dw when the block's are put together."""
    h, w, dy = put((N, C), t, 1.5, 1), put((C,), t, 0.3, 2, 1.0), put((N, C), t, 0.1, 3)
    rstd = (h.double().square().mean(dim=1) + 1e-6).rsqrt().float()
    dx, dw, again = guarded((N, C), t), guarded((C,), t), guarded((C,), t)
    ws = workspace(B.rms_norm_workspace_bytes(N, C))
    B.rms_norm_bwd(N, C, h, w, rstd, dy, None, dx, dw, ws)
    check_grad(t, h, w, rstd, dy, None, dx, dw)
    B.rms_norm_bwd(N, C, h, w, rstd, dy, None, dx, again, ws)
    assert torch.equal(dw, again) and B.last_device_status() == B.OK


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C", [96, 1037, 40001])
@pytest.mark.parametrize("N", [4, 400])
def test_subnormal_rows(N, C, t):
    """At eps = 0 the rstd of a row of subnormal numbers may not be a number of fp32: it is inf then, and y right all the same; at the smallest eps
    it is finite."""
    # multiples of 2^-133, which bf16 has too: the root mean square lies about 2^-130, and about 2^-126 in every other row
    g = torch.Generator(device="cuda").manual_seed(5)
    x = guarded((N, C), t, fill=0)
    x.copy_((torch.randint(1, 16, (N, C), device="cuda", generator=g).double() * 2.0 ** -133).float())
    x[1::2] *= 16
    w = put((C,), t, 0.3, 2, 1.0)
    y, rstd, q, scale = guarded((N, C), t), guarded((N,), torch.float32), bytes8((N, C)), guarded((N,), torch.float32)
    B.rms_norm_fwd(N, C, x, None, w, 0.0, None, y, rstd)
    _, er, ey = forward_reference(x, None, w, 0.0)
    k = additions(C)
    assert torch.isinf(rstd[0::2]).all() and (er[0::2] > 2.0 ** 128).all() and (er[1::2] < 2.0 ** 127.5).all()
    assert ((rstd[1::2].double() - er[1::2]).abs() <= er[1::2] * (k / 2 + 4) * U).all()
    assert ((y.double() - ey).abs() <= ey.abs() * (half_step(t) + (k / 2 + 8) * U * (1 + half_step(t)))).all()
    B.rms_norm_fwd_q8(N, C, x, None, w, 0.0, None, q, scale)
    check_q8(q, scale, ey, k / 2 + 8)
    B.rms_norm_fwd(N, C, x, None, w, 2.0 ** -149, None, y, rstd)
    _, er, ey = forward_reference(x, None, w, 2.0 ** -149)
    assert ((rstd.double() - er).abs() <= er * (k / 2 + 4) * U).all()


@pytest.mark.parametrize("C", [96, 1037, 40001])
@pytest.mark.parametrize("N", [4, 400])
@pytest.mark.parametrize("size,gain,eps", [(1e-10, 3e-35, 0.0), (1e-21, 1e-23, 1e-20), (1.9, 3.3e38, 1e-6), (3.3e38, 3.3e38, 0.0), (3.3e38, 1e-30, 0.0), (1e-38, 3.3e38, 0.0),
                                           (1e-40, 1e-30, 0.0)])
def test_q8_of_products_out_of_range(size, gain, eps, N, C):
    """Values times weights leave fp32's range where the norm's results do not."""
    x, w = guarded((N, C), torch.float32, fill=0), guarded((C,), torch.float32, fill=0)
    g = torch.Generator(device="cuda").manual_seed(5)
    sign = torch.randint(0, 2, (N, C), device="cuda", generator=g) * 2 - 1
    x.copy_((sign * size).float())                            # (|n| = 1: results are as large as the weights)
    w.copy_((torch.rand(C, device="cuda", generator=g, dtype=torch.float64) * 0.5 + 0.5) * gain)
    q, scale, rstd = bytes8((N, C)), guarded((N,), torch.float32), guarded((N,), torch.float32)
    B.rms_norm_fwd_q8(N, C, x, None, w, eps, None, q, scale, rstd)
    _, er, ey = forward_reference(x, None, w, float(torch.tensor(eps)))
    k = additions(C)
    check_q8(q, scale, ey, k / 2 + 8)
    assert (scale.double() >= ey.abs().amax(dim=1) / 448 * (1 - (k / 2 + 8) * U)).all()
