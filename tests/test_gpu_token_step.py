"""The embedding, the loss without stored logits and the orthogonalised update together, as a training step uses them, and
as options of the DNN step driver."""
import math
import os
import subprocess
import sys

import pytest
import torch

from gpu_helpers import assert_parity, check_guards, guarded, workspace
from paper_1602_06709_b200 import binding as B
from paper_1602_06709_b200 import networks

pytestmark = pytest.mark.gpu


def newton_schulz(u):
    m = u / (u.norm() + 1e-7)
    flip = m.shape[0] > m.shape[1]
    m = m.t() if flip else m
    for _ in range(5):
        g = m @ m.t()
        m = 3.4445 * m + (-4.7750 * g + 2.0315 * (g @ g)) @ m
    return m.t() if flip else m


class TokenStep:
    """A network of an embedding and an output layer: x = 2 * table[ids], classes of x w^T, one call after another on buffers
    that stay."""

    def __init__(self, N, V, C, K, t):
        g = torch.Generator(device="cuda").manual_seed(3)
        rnd = lambda shape, std, dt: guarded(shape, dt, fill=0).copy_(torch.randn(shape, device="cuda", generator=g) * std)
        self.N, self.V, self.C, self.K = N, V, C, K
        self.table, self.w = rnd((V, C), 1.0, t), rnd((K, C), 1.0 / math.sqrt(C), t)
        self.moment = guarded((K, C), torch.float32, fill=0)
        self.ids, self.labels = guarded((N,), torch.int32, fill=0), guarded((N,), torch.int32, fill=0)
        self.ids.copy_(torch.randint(0, V, (N,), device="cuda", generator=g))
        self.labels.copy_(torch.randint(0, K, (N,), device="cuda", generator=g))
        self.labels[::7] = -1
        self.x, self.dx, self.dw = guarded((N, C), t), guarded((N, C), t), guarded((K, C), t)
        self.loss, self.row_loss, self.lse = guarded((1,)), guarded((N,)), guarded((N,))
        d = B.dtype_code(self.x)
        self.ws = workspace(max(B.embedding_workspace_bytes(N, V, C), B.orthogonalize_workspace_bytes(1, K, C),
                                B.fc_softmax_xent_workspace_bytes(N, C, K, d, B.PASS_FWD),
                                B.fc_softmax_xent_workspace_bytes(N, C, K, d, B.PASS_BWD_DATA)))

    def step(self):
        N, V, C, K = self.N, self.V, self.C, self.K
        B.embedding_fwd(N, V, C, self.ids, self.table, 2.0, self.x)
        B.fc_softmax_xent_fwd(N, C, K, self.x, self.w, None, self.labels, self.loss, self.row_loss, self.lse, ignore_label=-1, ws=self.ws)
        B.fc_softmax_xent_bwd(N, C, K, self.x, self.w, None, self.labels, self.lse, None, self.dx, self.dw, None, ignore_label=-1, ws=self.ws)
        B.embedding_bwd_sgd(N, V, C, self.ids, self.dx, 2.0, self.table, 0.5, ws=self.ws)
        B.orthogonal_update(1, K, C, self.w, self.dw, self.moment, 0.9, True, 0.05, ws=self.ws)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_step_against_float64(t):
    """Every call of the step re-computed in float64 from what it received."""
    s = TokenStep(300, 500, 96, 700, t)
    table, w, moment = s.table.double(), s.w.double(), s.moment.double()
    s.step()
    B.check_device_status()
    check_guards()
    h = torch.finfo(t).eps / 2
    ids, labels = s.ids.long(), s.labels.long()
    counted = labels >= 0
    x = table[ids] * 2.0
    assert bool(((s.x.double() - x).abs() <= (h + 2.0 ** -23) * x.abs()).all())
    x = s.x.double()
    z = x @ w.t()
    lse = torch.logsumexp(z, 1)
    row = torch.where(counted, lse - z.gather(1, labels.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lse))
    n = int(counted.sum())
    assert_parity(s.lse.cpu().numpy(), lse.cpu().numpy(), "lse")
    assert abs(s.loss.item() - float(row.sum()) / n) <= 2e-3 * float(row.sum()) / n
    p = torch.exp(z - s.lse.double()[:, None])
    p.scatter_add_(1, labels.clamp(min=0)[:, None], torch.full((300, 1), -1.0, device="cuda", dtype=torch.float64))
    dz = p * (counted.double() / n)[:, None]
    # roundings of dz and of the result (2^-8 each at most, 16-bit), TF32 products (fp32): the library's parity bar holds both
    for got, ref, what in ((s.dx, dz @ w, "dx"), (s.dw, dz.t() @ x, "dw")):
        rel = float((got.double() - ref).norm() / ref.norm())
        assert rel <= (2e-3 if t == torch.float32 else 2 * h + 2e-4), f"{what}: {rel:.2e}"
    grad = torch.zeros_like(table).index_add_(0, ids, s.dx.double()) * 2.0
    want = table - 0.5 * grad
    assert float((s.table.double() - want).abs().max()) <= (h + 2.0 ** -18) * float(want.abs().max())
    m = 0.9 * moment + s.dw.double()
    assert float((s.moment.double() - m).abs().max()) <= 2.0 ** -22 * float(m.abs().max())
    o = newton_schulz(s.dw.double() + 0.9 * s.moment.double())
    step = 0.05 * math.sqrt(max(1.0, 700 / 96))
    want = w - step * o
    # direction 5e-3 of its norm, one rounding
    assert float((s.w.double() - want).norm()) <= 5e-3 * step * float(o.norm()) + (h + 2.0 ** -20) * float(want.norm())


def test_captured_step_equals_eager_steps():
    a, b = TokenStep(256, 300, 64, 520, torch.bfloat16), TokenStep(256, 300, 64, 520, torch.bfloat16)
    a.step(); b.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step()
    for _ in range(3):
        a.step()
        g.replay()
    torch.cuda.synchronize()
    B.check_device_status()
    for name in ("table", "w", "moment", "loss", "dx", "dw"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


def test_two_steps_on_two_streams_with_their_own_workspaces():
    a, b = TokenStep(200, 300, 64, 500, torch.bfloat16), TokenStep(200, 300, 64, 500, torch.bfloat16)
    ref = TokenStep(200, 300, 64, 500, torch.bfloat16)
    ref.step(); ref.step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(2):
        for s, m in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                m.step()
    torch.cuda.synchronize()
    for m in (a, b):
        for name in ("table", "w", "moment", "loss"):
            assert torch.equal(getattr(m, name), getattr(ref, name)), name


def small(**kw):
    net = networks.Dnn(64, dims=[40, 96, 72, 96, 52], cfg="small_dnn", **kw)
    g = torch.Generator(device="cuda").manual_seed(1)
    net.x.copy_(torch.randn(net.x.shape, device="cuda", generator=g))
    net.labels.copy_(torch.randint(0, 52, (64,), device="cuda", generator=g))
    return net


def test_dnn_without_stored_logits():
    """The same gradients as with stored logits, to the parity bar of their TF32 products."""
    a, b = small(), small(stored_logits=False)
    for net in (a, b):
        net.forward(); net.backward()
    B.check_device_status()
    assert abs(a.loss.item() - b.loss.item()) <= 1e-4 * a.loss.item()
    for j in range(4):
        assert_parity(b.dw(j).cpu().numpy(), a.dw(j).cpu().numpy(), f"dw{j}")
        assert_parity(b.db(j).cpu().numpy(), a.db(j).cpu().numpy(), f"db{j}")
    assert b.out[-1] is None and b.dout[-1] is None
    # updates folded into the weight gradients give the same parameters as the plain step
    c, d = small(stored_logits=False), small(stored_logits=False, fused_update=True)
    c.step(); d.step()
    for j in range(4):
        assert torch.equal(c.w(j), d.w(j)) and torch.equal(c.b(j), d.b(j))


def test_dnn_with_orthogonalised_hidden_updates():
    net = small(hidden_update="orthogonal", hidden_lr=0.03, momentum=0.9)
    w0 = [net.w(j).double().clone() for j in range(4)]
    b0 = [net.b(j).double().clone() for j in range(4)]
    net.step()
    B.check_device_status()
    for j, (C, K) in enumerate(net.layers):
        dw, w = net.dw(j).double(), net.w(j).double()
        assert float((net.b(j).double() - (b0[j] - 0.01 * net.db(j).double())).abs().max()) <= 1e-6
        if j in (1, 2):
            o = newton_schulz(dw + 0.9 * dw)           # momentum starts at zero: m = dw, Nesterov direction dw + 0.9 m
            step = 0.03 * math.sqrt(max(1.0, K / C))
            assert float((w - (w0[j] - step * o)).norm()) <= 5e-3 * step * float(o.norm()) + 2.0 ** -20 * float(w.norm())
            assert torch.equal(net.moments[j], net.dw(j))
        else:
            assert float((w - (w0[j] - 0.01 * dw)).abs().max()) <= 1e-6
    with pytest.raises(ValueError):
        net.param_buckets()
    with pytest.raises(ValueError):
        small(hidden_update="orthogonal", fused_update=True)
    with pytest.raises(ValueError):
        small(hidden_update="adam")


def test_dnn_options_captured():
    make = lambda: small(stored_logits=False, hidden_update="orthogonal")
    a, b = make(), make()
    b.capture_step()
    for _ in range(3):
        a.step()
        b.run_step()
    torch.cuda.synchronize()
    for j in range(4):
        assert torch.equal(a.w(j), b.w(j)) and torch.equal(a.b(j), b.b(j))


@pytest.mark.parametrize("C", [64, 96])      # (the update's two forms)
def test_first_calls_of_a_process_may_be_captured(C):
    """A process whose very first calls are captured into a graph (the library's one-time set-up falls into the capture)."""
    code = """
import sys
sys.path[:0] = [%r, %r]
import torch
from test_gpu_token_step import TokenStep
from paper_1602_06709_b200 import binding as B
s = TokenStep(256, 300, %d, 520, torch.bfloat16)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    s.step()
g.replay()
torch.cuda.synchronize()
B.check_device_status()
e = TokenStep(256, 300, %d, 520, torch.bfloat16)
e.step()
torch.cuda.synchronize()
assert all(torch.equal(getattr(s, n), getattr(e, n)) for n in ("table", "w", "moment", "loss", "dx"))
print("equal")
"""
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", code % (here, os.path.dirname(here), C, C)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "equal" in r.stdout, r.stderr[-2000:]


def test_updates_on_two_streams_at_once():
    """The update's products are one cooperative launch that takes the whole GPU: two of them, and another call's products beside
    them, on streams and workspaces of their own."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    M, N = 1100, 1500
    dw = torch.randn(1, M, N, device="cuda", generator=gen).bfloat16()
    w0 = torch.randn(1, M, N, device="cuda", generator=gen).bfloat16()
    mk = lambda: (w0.clone(), torch.zeros(1, M, N, device="cuda"), workspace(B.orthogonalize_workspace_bytes(1, M, N)))
    steps = 12
    call = lambda s: B.orthogonal_update(1, M, N, s[0], dw, s[1], 0.9, True, 0.02, ws=s[2])
    want = mk()
    for _ in range(steps):
        call(want)
    loss = [TokenStep(200, 300, 96, 500, torch.bfloat16) for _ in range(2)]
    for _ in range(steps):
        loss[0].step()
    states, streams = [mk(), mk()], [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(steps):
        for s, st in zip(streams, states):
            with torch.cuda.stream(s):
                call(st)
        with torch.cuda.stream(streams[2]):
            loss[1].step()
    torch.cuda.synchronize()
    B.check_device_status()
    check_guards()
    for st in states:
        assert torch.equal(st[0], want[0]) and torch.equal(st[1], want[1])
    for name in ("table", "w", "moment", "loss"):
        assert torch.equal(getattr(loss[0], name), getattr(loss[1], name)), name
