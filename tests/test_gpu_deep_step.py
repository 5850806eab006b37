"""RMS norm, its gradient, the clipped update, 8-bit layers and the choice of a class together, as the DNN step driver uses them."""
import math

import pytest
import torch

from gpu_helpers import check_guards
from paper_1602_06709_b200 import binding as B
from paper_1602_06709_b200 import networks

pytestmark = pytest.mark.gpu

DIMS = [40, 96, 96, 96, 200]


def make(N=70, seed=3, **options):
    m = networks.Dnn(N, dims=DIMS, lr=0.5, cfg="cfg4", residual_norm=True, **options)
    g = torch.Generator(device="cuda").manual_seed(seed)
    m.x.copy_(torch.randn(N, DIMS[0], device="cuda", generator=g))
    m.labels.copy_(torch.randint(0, DIMS[-1], (N,), device="cuda", generator=g))
    for j in range(1, len(m.layers)):
        m.gain(j).copy_(1 + 0.3 * torch.randn(DIMS[1], device="cuda", generator=g))
    return m


def reference(m, x=None):
    """The network in float64 with gradients: (parameters, logits, loss)."""
    n = len(m.layers)
    p = [t.double().clone().requires_grad_() for j in range(n) for t in (m.w(j), m.b(j))]
    gains = [None] + [m.gain(j).double().clone().requires_grad_() for j in range(1, n)]
    a = (m.x if x is None else x).double()
    stream = None
    for j in range(n):
        z = a @ p[2 * j].T + p[2 * j + 1]
        if j + 1 == n:
            break
        out = torch.sigmoid(z)
        stream = out if stream is None else stream + out
        a = stream * (stream.square().mean(dim=1, keepdim=True) + m.EPS).rsqrt() * gains[j + 1]
    loss = torch.nn.functional.cross_entropy(z, m.labels.long())
    return p, gains, z, loss


def close(got, want, bar, what):
    rel = float((got.double() - want).norm() / want.norm())
    assert rel <= bar, f"{what}: {rel:.2e}"


@pytest.mark.parametrize("stored", [True, False])
def test_gradients_of_a_residual_network(stored):
    """Every parameter's gradient against float64 autograd.  The products round their operands to TF32, 2^-11 each: a gradient passes 2 n products of
    n = 4 layers, whose errors add up to 2 n * 2 * 2^-11 of its norm at worst, 8e-3."""
    m = make(stored_logits=stored)
    m.forward()
    m.backward()
    B.check_device_status()
    p, gains, z, loss = reference(m)
    loss.backward()
    loss = float(loss.detach())
    assert abs(m.loss.item() - loss) <= 2e-3 * abs(loss)
    for j in range(len(m.layers)):
        close(m.dw(j), p[2 * j].grad, 8e-3, f"dw {j}")
        close(m.db(j), p[2 * j + 1].grad, 8e-3, f"db {j}")
        if j > 0:
            close(m.dgain(j), gains[j].grad, 8e-3, f"dgain {j}")
    check_guards()


@pytest.mark.parametrize("limit", [1e-3, 1e9])
def test_clipped_update(limit):
    m = make(clip_norm=limit)
    before = m.store.params.clone()
    m.step()
    grads = m.store.grads.double()
    norm = float(grads.norm())
    assert abs(m.grad_norm.item() - norm) <= norm * 2.0 ** -19
    f = min(1.0, limit / (norm + 1e-6))
    want = before.double() - 0.5 * f * grads
    assert float((m.store.params.double() - want).abs().max()) <= 2.0 ** -24 * float(want.abs().max()) + 0.5 * f * float(grads.abs().max()) * 2.0 ** -18


def test_captured_steps_equal_eager_steps():
    a, b = make(clip_norm=0.01), make(clip_norm=0.01)
    b.capture_step()
    b.labels.copy_(a.labels)
    for _ in range(3):
        a.step()
        b._graphs[b.x.data_ptr()].replay()
    torch.cuda.synchronize()
    B.check_device_status()
    assert torch.equal(a.store.params, b.store.params) and torch.equal(a.grad_norm, b.grad_norm) and torch.isfinite(a.store.params).all()


def test_orthogonal_update_with_a_residual_stream():
    m = make(hidden_update="orthogonal")
    before = m.gain(2).clone()
    m.step()
    assert torch.isfinite(m.store.params).all() and torch.equal(m.gain(2), torch.add(before, m.dgain(2), alpha=-m.lr))


def test_answer():
    m = make()
    N, K = m.N, DIMS[-1]
    token, logprob, u = torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, device="cuda"), torch.rand(N, device="cuda")
    zero = torch.zeros(N, device="cuda")
    m.answer(u, token, temperature=zero)
    _, _, z, _ = reference(m)
    assert torch.equal(token.long(), m.out[-1].argmax(dim=1))
    close(m.out[-1], z, 8e-3, "logits")
    m.answer(u, token, logprob=logprob)
    p = torch.log_softmax(m.out[-1].double(), dim=1)
    assert ((logprob.double() - p.gather(1, token.long()[:, None])[:, 0]).abs() <= 2.0 ** -20).all()
    cum = p.exp().cumsum(dim=1)
    at = cum.gather(1, token.long()[:, None])[:, 0]
    assert (at >= u.double() - 1e-9).all() and (at - p.exp().gather(1, token.long()[:, None])[:, 0] <= u.double() + 1e-9).all()


def test_answer_in_8_bits():
    """Against float64 from the 8-bit weights and rows as the calls made them, layer by layer."""
    m = make()
    m.quantize()
    N, n = m.N, len(m.layers)
    token, u = torch.empty(N, dtype=torch.int32, device="cuda"), torch.rand(N, device="cuda")
    m.answer(u, token, temperature=torch.zeros(N, device="cuda"), eight_bit=True)
    B.check_device_status()
    h = m._stream(n - 2).double()
    y = h * (h.square().mean(dim=1, keepdim=True) + m.EPS).rsqrt() * m.gain(n - 1).double()
    x = m.x8.double() * m.x8_scale.double()[:, None]
    top = y.abs().amax(dim=1, keepdim=True)
    # (half a step of e4m3 of the value, 2^-4, or of the subnormals, 2^-10 of 1/448 of the largest; and the fp32 roundings of stream and norm)
    assert ((x - y).abs() <= y.abs() * (2.0 ** -4 + 1e-5) + top * (2.0 ** -10 / 448 + 1e-5)).all()
    q, scale = m.w8[n - 1]
    w = q.double() * scale.double()[:, None]
    z = x @ w.T + m.b(n - 1).double()
    size = x.abs() @ w.abs().T + m.b(n - 1).double().abs()
    # (sums of 96 products, in three steps of 32, that lose 2^-23 of the largest term each at most; four fp32 roundings)
    assert ((m.out[-1].double() - z).abs() <= size * (99 * 2.0 ** -23 + 4 * 2.0 ** -24)).all()
    assert torch.equal(token.long(), m.out[-1].argmax(dim=1))
    # and near the network in full precision: two roundings of 2^-4 at most in each of three products, as a rule far less
    close(m.out[-1], reference(m)[2], 0.25, "logits")


def test_options_that_do_not_go_together():
    for bad in (dict(fused_update=True), dict(clip_norm=1.0, hidden_update="orthogonal")):
        with pytest.raises(ValueError):
            make(**bad)
    with pytest.raises(ValueError):
        networks.Dnn(8, dims=[8, 16, 24, 10], residual_norm=True)
    with pytest.raises(ValueError):
        networks.Dnn(8, dims=[8, 16, 10], fused_update=True, clip_norm=1.0)
    m = make(stored_logits=False)
    with pytest.raises(ValueError):
        m.answer(m.row_loss, m.labels)
    with pytest.raises(ValueError):
        networks.Dnn(8, dims=[8, 16, 10]).quantize()
    with pytest.raises(ValueError):
        m.param_buckets()
    with pytest.raises(ValueError):
        make().answer(m.row_loss, m.labels, eight_bit=True)
