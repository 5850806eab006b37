"""Newton-Schulz orthogonalisation and the update built on it against float64."""
import math

import pytest
import torch

from gpu_helpers import check_guards, guarded, workspace
from paper_1602_06709_b200 import binding as B

pytestmark = pytest.mark.gpu

A_, B_, C_, EPS = 3.4445, -4.7750, 2.0315, 1e-7
# 2-norm of the error over the 2-norm of the result.  Roundings to fp16 are off by 2^-11 at most and 2^-11 / sqrt(3) in the
# mean, 2e-4 of a value of average mantissa.  One step holds X in B X, A = X X^T and B; with |X| ~ 1 the errors of X, A and B
# enter the result with weights of about 2 |b + 2c|, |b| + 2 |c| and |b + c| (5, 9 and 3), independently: 2e-4 * 11 = 2.2e-3 a
# step.  Three steps have |X| of that size (the ones before raise the small singular values from below 0.1, where A and B are
# small against a): 2.2e-3 * sqrt(3) = 3.8e-3, to which the rounding of the result adds half a step of its type.
NS_TOL = 5e-3


def half_step(t):
    return torch.finfo(t).eps / 2


def reference(u, steps=5):
    out = []
    for m in u.double():
        m = m / (m.norm() + EPS)
        flip = m.shape[0] > m.shape[1]
        m = m.t() if flip else m
        for _ in range(steps):
            g = m @ m.t()
            m = A_ * m + (B_ * g + C_ * (g @ g)) @ m
        out.append(m.t() if flip else m)
    return torch.stack(out)


def spectrum(count, M, N, kind, seed):
    g = torch.Generator().manual_seed(seed)
    d = min(M, N)
    if kind == "gauss":
        return torch.randn(count, M, N, generator=g)
    if kind == "lowrank":
        r = min(8, d)
        return torch.randn(count, M, r, generator=g) @ torch.randn(count, r, N, generator=g) + 0.05 * torch.randn(count, M, N, generator=g)
    u = torch.linalg.qr(torch.randn(count, M, d, generator=g, dtype=torch.float64))[0]
    v = torch.linalg.qr(torch.randn(count, N, d, generator=g, dtype=torch.float64))[0]
    s = torch.arange(1, d + 1, dtype=torch.float64) ** (-1.0 if kind == "decay" else 0.0)
    return ((u * s) @ v.transpose(1, 2)).float()


def run(g, steps=5):
    count, M, N = g.shape
    out = guarded((count, M, N), g.dtype)
    B.orthogonalize(count, M, N, g, out, steps=steps, ws=workspace(B.orthogonalize_workspace_bytes(count, M, N)))
    B.check_device_status()
    check_guards()
    return out


def assert_close(got, ref, t):
    for a, b in zip(got.double().cpu(), ref.cpu()):
        err, norm = float((a - b).norm()), float(b.norm())
        assert err <= (NS_TOL + half_step(t)) * norm, f"{err / norm:.3e}"


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("count,M,N", [(1, 1, 1), (1, 1, 50), (2, 50, 1), (1, 7, 5), (3, 16, 33), (1, 33, 100), (1, 100, 33),
                                       (2, 128, 128), (1, 129, 257), (1, 300, 1000), (1, 1000, 300), (1, 640, 640), (4, 260, 520), (1, 1500, 1412)])
def test_direction(t, count, M, N):
    g = guarded((count, M, N), t, fill=0)
    g.copy_(spectrum(count, M, N, "gauss", M + N))
    assert_close(run(g), reference(g), t)


@pytest.mark.parametrize("kind", ["gauss", "lowrank", "decay", "flat"])
@pytest.mark.parametrize("M,N", [(256, 256), (200, 520), (520, 200)])
def test_spectra(kind, M, N):
    g = guarded((2, M, N), torch.float32, fill=0)
    g.copy_(spectrum(2, M, N, kind, 3))
    assert_close(run(g), reference(g), torch.float32)


def test_pairs_of_ctas_and_symmetric_tiles():
    """Enough tiles for the CTA-pair form, ragged in both directions."""
    g = guarded((2, 2100, 2310), torch.bfloat16, fill=0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    g.copy_(torch.randn(2, 2100, 2310, device="cuda", generator=gen))
    assert_close(run(g), reference(g), torch.bfloat16)
    tall = guarded((2, 2310, 2100), torch.bfloat16, fill=0)
    tall.copy_(g.transpose(1, 2))
    assert_close(run(tall), reference(tall), torch.bfloat16)


@pytest.mark.parametrize("steps", [1, 2, 3, 7])
def test_steps(steps):
    g = guarded((1, 96, 160), torch.float32, fill=0)
    g.copy_(spectrum(1, 96, 160, "gauss", 9))
    assert_close(run(g, steps), reference(g, steps), torch.float32)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e-7, 1.0, 1e15, 1e25])
def test_norms_out_of_the_range_of_fp32_squares(scale):
    g = guarded((1, 64, 80), torch.float32, fill=0)
    g.copy_(spectrum(1, 64, 80, "gauss", 4) * scale)
    got, ref = run(g), reference(g)
    # (below |g| ~ 1e-7 the eps of the definition makes X small: fp16 has no numbers below 2^-24 of the scaled unit)
    if scale >= 1e-7:
        assert_close(got, ref, torch.float32)
    else:
        assert float((got.double() - ref).abs().max()) <= 485 * 2.0 ** -37 + NS_TOL * float(ref.abs().max())


def test_zero_and_nan_matrices_of_a_batch():
    g = guarded((3, 40, 24), torch.float32, fill=0)
    g.copy_(spectrum(3, 40, 24, "gauss", 5))
    g[0] = 0
    g[2, 3, 4] = float("nan")
    got = run(g)
    assert not bool(got[0].any()) and bool(got[2].isnan().all())
    assert_close(got[1:2], reference(g[1:2]), torch.float32)


def test_in_place_and_repeatable():
    g = guarded((2, 130, 260), torch.bfloat16, fill=0)
    g.copy_(spectrum(2, 130, 260, "gauss", 6))
    first = run(g)
    assert torch.equal(first, run(g))
    B.orthogonalize(2, 130, 260, g, g, ws=workspace(B.orthogonalize_workspace_bytes(2, 130, 260)))
    assert torch.equal(first, g)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("count,M,N", [(1, 5, 3), (2, 64, 96), (1, 257, 70), (1, 300, 300)])
@pytest.mark.parametrize("nesterov", [False, True])
def test_update(t, count, M, N, nesterov):
    mu, lr, wd = 0.9, 0.05, 0.1
    gen = torch.Generator(device="cuda").manual_seed(M)
    mk = lambda dt, std: guarded((count, M, N), dt, fill=0).copy_(torch.randn(count, M, N, device="cuda", generator=gen) * std)
    w, dw, m = mk(t, 0.1), mk(t, 1e-2), mk(torch.float32, 1e-2)
    w0, m0 = w.double(), m.double()
    B.orthogonal_update(count, M, N, w, dw, m, mu, nesterov, lr, wd, ws=workspace(B.orthogonalize_workspace_bytes(count, M, N)))
    B.check_device_status()
    check_guards()
    mu64 = float(torch.tensor(mu, dtype=torch.float32))
    m1 = mu64 * m0 + dw.double()
    assert bool(((m.double() - m1).abs() <= 2.0 ** -23 * (m0.abs() + dw.double().abs())).all())
    o = reference(dw.double() + mu64 * m1 if nesterov else m1)
    step = lr * math.sqrt(max(1.0, M / N))
    want = (1 - lr * wd) * w0 - step * o
    for a, b, d in zip(w.double(), want, o):
        # the direction's error, fp32 arithmetic of the update, one rounding (fp16: subnormals are absolute)
        bound = step * NS_TOL * float(d.norm()) + (half_step(t) + 2.0 ** -21) * float(b.norm()) + math.sqrt(M * N) * 2.0 ** -25
        assert float((a - b).norm()) <= bound


def test_update_graph_replay():
    M, N = 192, 320
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = torch.randn(1, M, N, device="cuda", generator=gen).bfloat16()
    dw = torch.randn(1, M, N, device="cuda", generator=gen).bfloat16()
    m = torch.zeros(1, M, N, device="cuda")
    ws = workspace(B.orthogonalize_workspace_bytes(1, M, N))
    we, me = w.clone(), m.clone()
    call = lambda w, m: B.orthogonal_update(1, M, N, w, dw, m, 0.9, True, 0.02, ws=ws)
    call(we, me)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(w, m)
    for k in range(3):
        if k:
            dw.normal_()
            call(we, me)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, we) and torch.equal(m, me)


# ---- narrow matrices: the steps run on d x d matrices in 64 bits, the result is one product in fp32
def narrow_reference(u, steps=5):
    """X and |P| |X0| in float64, with X = P X0 (the transpose of tall matrices)."""
    outs, sizes = [], []
    for m in u.double():
        flip = m.shape[0] > m.shape[1]
        m = m.t() if flip else m
        x0 = m / (m.norm() + EPS)
        p, a = torch.eye(m.shape[0], dtype=torch.float64, device=m.device), x0 @ x0.t()
        for _ in range(steps):
            q = A_ * torch.eye(m.shape[0], dtype=torch.float64, device=m.device) + B_ * a + C_ * (a @ a)
            p, a = q @ p, q @ a @ q
        out, size = p @ x0, p.abs() @ x0.abs()
        outs.append(out.t() if flip else out)
        sizes.append(size.t() if flip else size)
    return torch.stack(outs), torch.stack(sizes)


def narrow_bound(ref, size, d, t):
    # X0 and P rounded to fp32, d multiply-adds and 1 / |U| rounded (half a step, 2^-24 of the terms' sizes, each), the 64-bit
    # steps' 1e-11, and the result's rounding (fp16: its subnormals are absolute)
    return (d + 4) * 2.0 ** -24 * size + half_step(t) * ref.abs() * (1 + 2.0 ** -10) + 2.0 ** -25


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("count,d,k", [(1, 1, 1), (2, 1, 70), (1, 7, 7), (3, 16, 64), (1, 17, 63), (1, 23, 1367), (2, 32, 65), (1, 33, 200),
                                       (1, 50, 50), (5, 64, 129), (1, 64, 4096), (1, 31, 20000), (40, 9, 100), (33, 32, 130)])
@pytest.mark.parametrize("tall", [False, True])
def test_narrow(t, count, d, k, tall):
    M, N = (k, d) if tall else (d, k)
    g = guarded((count, M, N), t, fill=0)
    g.copy_(spectrum(count, M, N, "gauss", d + k))
    got = run(g)
    ref, size = narrow_reference(g)
    assert bool(((got.double() - ref).abs() <= narrow_bound(ref, size, d, t)).all())
    assert torch.equal(got, run(g))


@pytest.mark.parametrize("kind", ["lowrank", "decay", "flat", "steep"])
@pytest.mark.parametrize("count,M,N", [(2, 64, 500), (40, 300, 24)])
def test_narrow_spectra(kind, count, M, N):
    g = guarded((count, M, N), torch.float32, fill=0)
    g.copy_(spectrum(count, M, N, "decay" if kind == "steep" else kind, 3))
    if kind == "steep":                          # singular values down to 1e-5 of the largest
        g.mul_(torch.logspace(0, -5, M if M < N else N, device="cuda").view(*((-1, 1) if M < N else (1, -1))))
    got = run(g)
    ref, size = narrow_reference(g)
    assert bool(((got.double() - ref).abs() <= narrow_bound(ref, size, min(M, N), torch.float32)).all())


@pytest.mark.parametrize("steps", [1, 2, 7])
def test_narrow_steps(steps):
    g = guarded((1, 30, 90), torch.float32, fill=0)
    g.copy_(spectrum(1, 30, 90, "gauss", 9))
    got = run(g, steps)
    ref, size = narrow_reference(g, steps)
    # (seven steps let roundings of small singular values grow to 12^2 times the 1e-11 of five)
    assert bool(((got.double() - ref).abs() <= narrow_bound(ref, size, 30, torch.float32) + 1e-9).all())


def test_narrow_matrices_in_tensor_core_form():
    """Many matrices of 33 to 64 rows run on the tensor cores."""
    g = guarded((36, 50, 140), torch.bfloat16, fill=0)
    g.copy_(spectrum(36, 50, 140, "gauss", 2))
    assert_close(run(g), reference(g), torch.bfloat16)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("count,M,N", [(1, 40, 20000), (1, 1000, 21), (40, 12, 77)])
@pytest.mark.parametrize("nesterov", [False, True])
def test_narrow_update(t, count, M, N, nesterov):
    mu, lr, wd = 0.9, 0.05, 0.1
    gen = torch.Generator(device="cuda").manual_seed(M)
    mk = lambda dt, std: guarded((count, M, N), dt, fill=0).copy_(torch.randn(count, M, N, device="cuda", generator=gen) * std)
    w, dw, m = mk(t, 0.1), mk(t, 1e-2), mk(torch.float32, 1e-2)
    w0, m0 = w.double(), m.double()
    B.orthogonal_update(count, M, N, w, dw, m, mu, nesterov, lr, wd, ws=workspace(B.orthogonalize_workspace_bytes(count, M, N)))
    B.check_device_status()
    check_guards()
    mu64 = float(torch.tensor(mu, dtype=torch.float32))
    assert bool(((m.double() - (mu64 * m0 + dw.double())).abs() <= 2.0 ** -23 * (m0.abs() + dw.double().abs())).all())
    # U from the momentum as it was stored; its rounding, where one follows, is 2^-24 of its terms
    u = dw.double() + mu64 * m.double() if nesterov else m.double()
    o, size = narrow_reference(u)
    step = lr * math.sqrt(max(1.0, M / N))
    want = (1 - lr * wd) * w0 - step * o
    # the rounding of U moves |U| and every X0 by 2^-24 of its terms' sizes at most, X by |P| (and P's change) times that: the
    # sizes of the terms of U are below |dw| + |m|, whose part of `size` is bounded by the largest row sum of |P| times the largest of them
    bound = step * (narrow_bound(o, size, min(M, N), torch.float32) + (2.0 ** -20 * size.max() if nesterov else 0)) + (half_step(t) + 2.0 ** -22) * (want.abs() + w0.abs() + step * o.abs())
    assert bool(((w.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("count,M,N", [(1, 5824, 22016), (1, 4592, 10172), (2, 4183, 4850)])
def test_products_that_use_every_counter_of_the_split_tiles(count, M, N):
    """128 tiles of CTA pairs in two parts each: the barrier between the products is no counter of theirs."""
    gen = torch.Generator(device="cuda").manual_seed(M)
    g = guarded((count, M, N), torch.bfloat16, fill=0)
    for m in g:
        m.copy_(torch.randn(M, N, device="cuda", generator=gen))
    got = run(g)                                  # (into NaN: a block that is left out shows)
    assert bool(got.isfinite().all())
    for b in range(count):                        # (one matrix at a time in float64)
        ref = reference(g[b:b + 1])[0]
        err, norm = float((got[b].double() - ref).norm()), float(ref.norm())
        assert err <= (NS_TOL + half_step(torch.bfloat16)) * norm
        # 32 x 128 blocks, the parts of a warp: none is off by more than its own share of rounding explains.  The direction's elements
        # are alike in size, so a block's error is its share of the whole's, within the spread of 4096 elements' squares
        e = (got[b].double() - ref)[:M // 32 * 32, :N // 128 * 128].reshape(M // 32, 32, N // 128, 128)
        share = e.square().sum((1, 3)).sqrt()
        assert float(share.max()) <= 4 * (NS_TOL + half_step(torch.bfloat16)) * norm * math.sqrt(4096 / (M * N))
        del ref, e, share


@pytest.mark.parametrize("t,count,M,N", [(torch.bfloat16, 8, 256, 512), (torch.bfloat16, 1, 1030, 1100), (torch.float32, 2, 130, 260),
                                         (torch.float16, 1, 700, 2000)])
def test_repeated_calls_give_the_same_bits(t, count, M, N):
    """Every product reads, through the asynchronous proxy, what the CTAs have stored before the barrier in front of it: a product that
    met older tiles would differ from call to call."""
    gen = torch.Generator(device="cuda").manual_seed(M)
    g = guarded((count, M, N), t, fill=0)
    g.copy_(torch.randn(count, M, N, device="cuda", generator=gen))
    ws = workspace(B.orthogonalize_workspace_bytes(count, M, N))
    first, out = guarded((count, M, N), t), guarded((count, M, N), t)
    B.orthogonalize(count, M, N, g, first, ws=ws)
    assert_close(first, reference(g), t)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for k in range(200):
        if k % 2:
            ws.fill_(k)                           # (and what the workspace held does not matter)
        B.orthogonalize(count, M, N, g, out, ws=ws)
        differ += (out != first).sum()
    B.check_device_status()
    check_guards()
    assert int(differ) == 0


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e-7, 1.0, 1e15, 1e25, 1e36])
@pytest.mark.parametrize("M,N", [(96, 160), (300, 130)])
def test_tensor_core_form_norms_out_of_the_range_of_fp32_squares(scale, M, N):
    g = guarded((1, M, N), torch.float32, fill=0)
    g.copy_(spectrum(1, M, N, "gauss", 4) * scale)
    got, ref = run(g), reference(g)
    # (below |g| ~ 1e-7 the eps of the definition makes X small: the planes and the last step's operands have steps of 2^-24 of
    # the scaled unit 2^-14, i.e. errors of 2^-39, which 3.4445^5 = 485 bounds)
    if scale >= 1e-7:
        assert_close(got, ref, torch.float32)
    else:
        assert float((got.double() - ref).abs().max()) <= 485 * 2.0 ** -37 + NS_TOL * float(ref.abs().max())


def test_tensor_core_form_zero_and_nan_matrices_of_a_batch():
    g = guarded((4, 80, 140), torch.float32, fill=0)
    g.copy_(spectrum(4, 80, 140, "gauss", 5))
    g[0] = 0
    g[2, 3, 4] = float("nan")
    g[3, 79, 139] = float("inf")
    got = run(g)
    assert not bool(got[0].any()) and bool(got[2:].isnan().all())
    assert_close(got[1:2], reference(g[1:2]), torch.float32)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e-7, 1.0, 1e15, 1e25, 1e36])
@pytest.mark.parametrize("M,N", [(64, 80), (200, 31)])
def test_narrow_norms_out_of_the_range_of_fp32_squares(scale, M, N):
    g = guarded((1, M, N), torch.float32, fill=0)
    g.copy_(spectrum(1, M, N, "gauss", 4) * scale)
    got = run(g)
    ref, size = narrow_reference(g)
    assert bool(((got.double() - ref).abs() <= narrow_bound(ref, size, min(M, N), torch.float32)).all())


def test_narrow_zero_and_nan_matrices_of_a_batch():
    g = guarded((4, 40, 24), torch.float32, fill=0)
    g.copy_(spectrum(4, 40, 24, "gauss", 5))
    g[0] = 0
    g[2, 3, 4] = float("nan")
    g[3, 39, 23] = float("inf")
    got = run(g)
    assert not bool(got[0].any()) and bool(got[2:].isnan().all())
    ref, size = narrow_reference(g[1:2])
    assert bool(((got[1:2].double() - ref).abs() <= narrow_bound(ref, size, 24, torch.float32)).all())


@pytest.mark.parametrize("count,M,N", [(1, 64, 20000), (1, 30000, 16), (1, 700, 30000)])
def test_norms_beyond_the_range_of_fp32(count, M, N):
    """|g| above 2^128 / 2^2, whose reciprocal has fewer bits as an fp32 number."""
    gen = torch.Generator(device="cuda").manual_seed(M)
    g = guarded((count, M, N), torch.float32, fill=0)
    g.copy_(torch.randn(count, M, N, device="cuda", generator=gen) * 4e37)
    assert bool(g.isfinite().all()) and float(g.double().norm()) > 2.0 ** 131
    got = run(g)
    if min(M, N) <= 64:
        ref, size = narrow_reference(g)
        assert bool(((got.double() - ref).abs() <= narrow_bound(ref, size, min(M, N), torch.float32)).all())
    else:
        assert_close(got, reference(g), torch.float32)


@pytest.mark.parametrize("M,N", [(33000, 66000), (66100, 32900), (40, 55000000), (100000000, 24)])
def test_offsets_beyond_32_bits(M, N):
    """A matrix of more than 2^31 elements that is zero but for its last corner, which decides the result."""
    m, n = min(M, 512), min(N, 700)
    g = torch.zeros(1, M, N, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(M % 1000)
    corner = torch.randn(1, m, n, device="cuda", generator=gen).bfloat16()
    g[:, M - m:, N - n:] = corner
    ws = workspace(B.orthogonalize_workspace_bytes(1, M, N))
    B.orthogonalize(1, M, N, g, g, ws=ws)
    B.check_device_status()
    check_guards()
    got = g[:, M - m:, N - n:].clone()
    assert_close(got, reference(corner), torch.bfloat16)
    g[:, M - m:, N - n:] = 0
    assert not bool(g.any())                     # zero rows and columns of X stay zero


def test_batch_offsets_beyond_32_bits():
    count, M, N = 36, 7800, 7800                 # 2.2e9 elements
    g = torch.empty(count, M, N, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(4)
    for m in g:
        m.copy_(torch.randn(M, N, device="cuda", generator=gen))
    out = torch.full_like(g, float("nan"))
    B.orthogonalize(count, M, N, g, out, ws=workspace(B.orthogonalize_workspace_bytes(count, M, N)))
    B.check_device_status()
    check_guards()
    for b in (0, count - 1):
        assert_close(out[b:b + 1], reference(g[b:b + 1]), torch.bfloat16)
    assert bool(out.isfinite().all())
