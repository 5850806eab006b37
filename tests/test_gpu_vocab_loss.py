"""FC softmax cross-entropy without stored logits against a plain float64 computation of the same formulas."""
import math

import pytest
import torch

from gpu_helpers import assert_parity, check_guards, guarded, workspace
from paper_1602_06709_b200 import binding as B

pytestmark = pytest.mark.gpu

IGNORE = -100


def half_step(t):
    return torch.finfo(t).eps / 2


def put(shape, t, std, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = guarded(shape, t, fill=0)
    out.copy_(torch.randn(shape, device="cuda", generator=g) * std)
    return out


class Case:
    def __init__(self, N, C, K, t, bias=False, ignored=0.0, scale=1.5, seed=0):
        self.N, self.C, self.K, self.t = N, C, K, t
        self.x, self.w = put((N, C), t, 1.0, seed), put((K, C), t, scale / math.sqrt(C), seed + 1)
        self.bias = put((K,), t, 0.5, seed + 2) if bias else None
        g = torch.Generator().manual_seed(seed + 3)
        labels = torch.randint(0, K, (N,), generator=g)
        labels[torch.rand(N, generator=g) < ignored] = IGNORE
        self.labels = guarded((N,), torch.int32, fill=0)
        self.labels.copy_(labels)
        self.ignore = IGNORE
        self.row_grad = None

    def forward(self):
        self.loss, self.row_loss, self.lse = guarded((1,)), guarded((self.N,)), guarded((self.N,))
        ws = workspace(B.fc_softmax_xent_workspace_bytes(self.N, self.C, self.K, B.dtype_code(self.x), B.PASS_FWD))
        B.fc_softmax_xent_fwd(self.N, self.C, self.K, self.x, self.w, self.bias, self.labels, self.loss, self.row_loss, self.lse,
                              ignore_label=self.ignore, ws=ws)

    def backward(self, dx=True):
        self.dx = guarded((self.N, self.C), self.t) if dx else None
        self.dw = guarded((self.K, self.C), self.t)
        self.db = guarded((self.K,), self.t) if self.bias is not None else None
        ws = workspace(B.fc_softmax_xent_workspace_bytes(self.N, self.C, self.K, B.dtype_code(self.x), B.PASS_BWD_DATA))
        B.fc_softmax_xent_bwd(self.N, self.C, self.K, self.x, self.w, self.bias, self.labels, self.lse, self.row_grad, self.dx,
                              self.dw, self.db, ignore_label=self.ignore, ws=ws)

    def reference(self):
        """float64 results, and the bounds that roundings of the definition's steps give (16-bit operands):
        z      products exact, C additions in fp32 (2^-23 each, truncation allowed for), the bias
        lse    the largest error of z, ex2 (2^-21), sums of K terms in fp32 in runs of at most 64 + parts
        dz     p off by the errors of z and lse and 2^-20, then rounded to the type
        dx,dw  the errors of dz through the product, sums of K or N terms in fp32, one rounding."""
        x, w = self.x.double(), self.w.double()
        z = x @ w.t()
        ez = (self.C + 2) * 2.0 ** -23 * (x.abs() @ w.abs().t())
        if self.bias is not None:
            z = z + self.bias.double()
            ez = ez + 2.0 ** -23 * z.abs()
        lse = torch.logsumexp(z, 1)
        elz = torch.where(z > z.amax(1, keepdim=True) - 30, ez, torch.zeros_like(ez)).amax(1) + 2.0 ** -22 * z.abs().amax(1)
        el = elz + (96 + self.K / 128) * 2.0 ** -23 + 2.0 ** -20 + 2.0 ** -23 * lse.abs()
        labels = self.labels.long()
        counted = labels != IGNORE
        at = z.gather(1, labels.clamp(min=0)[:, None])[:, 0]
        row = torch.where(counted, lse - at, torch.zeros_like(lse))
        erow = torch.where(counted, el + ez.gather(1, labels.clamp(min=0)[:, None])[:, 0] + 2.0 ** -23 * row.abs(), torch.zeros_like(lse))
        n = max(1, int(counted.sum()))
        g = torch.full_like(lse, 1.0 / n) if self.row_grad is None else self.row_grad.double()
        g = torch.where(counted, g, torch.zeros_like(g))[:, None]
        p = torch.exp(z - lse[:, None])
        hot = torch.zeros_like(p).scatter_(1, labels.clamp(min=0)[:, None], 1.0)
        dz = (p - hot) * g
        ep = p * ((ez + el[:, None]) * 1.05 + 2.0 ** -20)
        # (fp16 is scaled into range first: below 2^-24 of the scaled unit the rounding is absolute)
        floor = 2.0 ** -38 * g.abs().max() if self.t == torch.float16 else 0.0
        edz = ep * g.abs() + (half_step(self.t) + 2.0 ** -22) * (dz.abs() + ep * g.abs()) + floor
        h = half_step(self.t) * 1.01
        tiny = torch.finfo(self.t).tiny * torch.finfo(self.t).eps
        out = {"lse": (lse, el), "row_loss": (row, erow),
               "loss": (row.sum()[None] / n, (erow.sum()[None] / n) + 2.0 ** -23 * row.sum().abs() / n)}
        # sums of the pieces: at most K/256 partial results are added in fp32 on top of the product's own additions
        for name, a, ea, b, terms in (("dx", dz, edz, w, self.K), ("dw", dz.t(), edz.t(), x, self.N)):
            v = a @ b
            e = ea @ b.abs() + (terms + 8) * 2.0 ** -23 * (a.abs() @ b.abs())
            out[name] = (v, e + h * (v.abs() + e) + tiny)
        if self.bias is not None:
            v = dz.sum(0)
            e = edz.sum(0) + (self.N + 8) * 2.0 ** -24 * dz.abs().sum(0)
            out["db"] = (v, e + h * (v.abs() + e) + tiny)
        return out

    def check(self, names=("loss", "row_loss", "lse", "dx", "dw", "db")):
        B.check_device_status()
        check_guards()
        for name, (ref, bound) in self.reference().items():
            got = getattr(self, name, None)
            if name not in names or got is None:
                continue
            over = ((got.double() - ref).abs() - bound).max().item()
            assert over <= 0, f"{name}: {over:.3e} over its bound, largest bound {bound.max().item():.3e}"


SIZES = [(1, 8, 1), (1, 64, 2), (2, 72, 257), (7, 33, 100), (128, 64, 128), (129, 65, 129), (130, 136, 300), (256, 256, 1000),
         (300, 520, 2049), (1, 1024, 9000), (64, 24, 20000), (513, 7, 511),
         (256, 4096, 1000), (40, 2010, 300), (3, 1100, 17), (1000, 1032, 4000)]


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,C,K", SIZES)
@pytest.mark.parametrize("bias,ignored", [(False, 0.0), (True, 0.3)])
def test_loss_and_gradients(t, N, C, K, bias, ignored):
    c = Case(N, C, K, t, bias, ignored, seed=N + C + K)
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scale", [1e-3, 0.5, 300.0, 65536.0])
def test_given_row_gradients(t, scale):
    c = Case(200, 128, 700, t, True, 0.2, seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)
    c.row_grad = guarded((200,))
    c.row_grad.copy_(torch.randn(200, device="cuda", generator=g) * scale / 200)
    c.row_grad[3] = 0.0
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,C,K", [(2500, 200, 3100), (2500, 520, 4900), (1024, 2048, 8192)])
def test_many_row_tiles_run_as_pairs(t, N, C, K):
    c = Case(N, C, K, t, True, 0.1, seed=8)
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("N,C,K,ignored", [(5, 12, 30, 0.0), (64, 100, 700, 0.3), (130, 33, 257, 0.2)])
def test_fp32_operands(N, C, K, ignored):
    """TF32 products: held to the library's parity bar."""
    c = Case(N, C, K, torch.float32, True, ignored, seed=N)
    c.forward()
    c.backward()
    B.check_device_status()
    check_guards()
    for name, (ref, _) in c.reference().items():
        assert_parity(getattr(c, name).cpu().numpy(), ref.cpu().numpy(), name)


def test_pieces_add_up():
    """More classes than one piece holds (a piece is limited by its bytes): dx is the sum over pieces."""
    for t, N, C, K in ((torch.bfloat16, 65536, 16, 4200), (torch.float32, 65536, 16, 2100)):
        c = Case(N, C, K, t, True, 0.1, seed=9)
        c.forward()
        c.backward()
        if t == torch.float32:
            for name, (ref, _) in c.reference().items():
                assert_parity(getattr(c, name).cpu().numpy(), ref.cpu().numpy(), name)
        else:
            c.check()


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16, torch.float32])
def test_no_row_counts(t):
    c = Case(70, 64, 90, t, True, 1.1, seed=10)
    c.forward()
    c.backward()
    B.check_device_status()
    check_guards()
    assert c.loss.item() == 0.0 and not bool(c.row_loss.any())
    assert not bool(c.dx.any()) and not bool(c.dw.any()) and not bool(c.db.any())
    assert bool(((c.lse.double() - c.reference()["lse"][0]).abs() <= 1e-2).all())


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16, torch.float32])
def test_masked_classes(t):
    """A bias of -inf, or of the type's lowest value, takes classes out: probability and gradient 0."""
    for mask in (float("-inf"), torch.finfo(t).min):
        c = Case(130, 64, 400, t, True, 0.0, seed=11)
        c.labels.copy_(c.labels % 100)
        c.bias[100:] = mask
        c.forward()
        c.backward()
        B.check_device_status()
        z = c.x.double() @ c.w.double()[:100].t() + c.bias.double()[:100]
        lse = torch.logsumexp(z, 1)
        assert bool(((c.lse.double() - lse).abs() <= 1e-2).all())
        assert not bool(c.dw[100:].any()) and not bool(c.db[100:].any())
        assert bool(c.dx.isfinite().all()) and bool(c.dw.isfinite().all()) and bool(c.row_loss.isfinite().all())
    # every class of every row masked
    c.bias.fill_(float("-inf"))
    c.forward()
    c.backward()
    B.check_device_status()
    assert bool((c.lse == float("-inf")).all()) and bool((c.row_loss == float("inf")).all())
    assert bool(c.dx.isfinite().all())


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16, torch.float32])
def test_nan_and_infinity_stay_in_their_row(t):
    c = Case(140, 64, 300, t, False, 0.0, seed=12)
    c.x[5, 3] = float("nan")
    c.x[9, 1] = float("inf")
    c.labels[9] = IGNORE
    c.labels[5] = IGNORE
    c.forward()
    c.backward()
    B.check_device_status()
    keep = [n for n in range(140) if n not in (5, 9)]
    assert bool(c.lse[keep].isfinite().all()) and bool(c.lse[5].isnan())
    assert c.row_loss[5].item() == 0.0 and math.isfinite(c.loss.item())
    assert not bool(c.dx[5].any()) and bool(c.dx[keep].isfinite().all())


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16, torch.float32])
def test_large_logits(t):
    """Logits of several hundred: the running maximum keeps the exponentials in range."""
    c = Case(100, 64, 500, t, False, 0.0, scale=200.0, seed=13)
    c.forward()
    B.check_device_status()
    z = c.x.double() @ c.w.double().t()
    bound = 2e-3 * z.abs().amax(1) if t == torch.float32 else c.reference()["lse"][1]
    assert bool(((c.lse.double() - torch.logsumexp(z, 1)).abs() <= bound).all())


def test_labels_out_of_range():
    c = Case(60, 64, 200, torch.bfloat16, False, 0.0, seed=14)
    c.labels[7] = 200
    c.labels[8] = -1
    c.forward()
    assert B.last_device_status() == B.ERR_BAD_LABEL
    assert c.row_loss[7].item() == 0.0 and c.row_loss[8].item() == 0.0 and math.isfinite(c.loss.item())
    c.backward()
    assert B.last_device_status() == B.OK
    p = torch.softmax(c.x.double() @ c.w.double().t(), 1)
    ref = (p[7] @ c.w.double()) / 60                  # no target: softmax over N
    # dz rounded (2^-8 of each term), the product's sums, one rounding
    bound = (p[7] @ c.w.double().abs()) / 60 * 2.0 ** -7 + ref.abs() * 2.0 ** -8
    assert bool(((c.dx[7].double() - ref).abs() <= bound).all())


def test_gradient_against_differences():
    """Central differences of the mean loss in float64 at the operands' own values."""
    c = Case(20, 24, 50, torch.bfloat16, True, 0.2, seed=15)
    c.forward()
    c.backward()
    x, w, b = c.x.double().cpu(), c.w.double().cpu(), c.bias.double().cpu()
    labels = c.labels.long().cpu()
    counted = labels != IGNORE

    def loss(x, w, b):
        z = x @ w.t() + b
        row = torch.logsumexp(z, 1) - z.gather(1, labels.clamp(min=0)[:, None])[:, 0]
        return float(row[counted].mean())

    ref = c.reference()
    h = 1e-4
    for name, which, ij in (("dx", 0, (3, 5)), ("dx", 0, (19, 23)), ("dw", 1, (0, 0)), ("dw", 1, (49, 7)), ("db", 2, (11,))):
        vals = []
        for s in (h, -h):
            args = [x.clone(), w.clone(), b.clone()]
            args[which][ij] += s
            vals.append(loss(*args))
        d = (vals[0] - vals[1]) / (2 * h)
        # third derivatives of the loss are below 1 in these units: h^2, and 1e-15 / h from the sums
        assert abs(d - float(getattr(c, name)[ij])) <= float(ref[name][1][ij]) + 1e-7


def test_optional_outputs_and_repeatability():
    c = Case(300, 64, 900, torch.bfloat16, True, 0.1, seed=16)
    c.forward()
    c.backward()
    dw, dx, loss = c.dw.clone(), c.dx.clone(), c.loss.clone()
    c.forward()
    c.backward(dx=False)
    assert torch.equal(c.dw, dw) and torch.equal(c.loss, loss)
    c.backward()
    assert torch.equal(c.dx, dx)
    check_guards()


def test_graph_replay():
    c = Case(260, 136, 1500, torch.bfloat16, False, 0.2, seed=17)
    c.forward(); c.backward()
    torch.cuda.synchronize()
    ws = [workspace(B.fc_softmax_xent_workspace_bytes(c.N, c.C, c.K, B.BF16, p)) for p in (B.PASS_FWD, B.PASS_BWD_DATA)]
    loss, row, lse = guarded((1,)), guarded((c.N,)), guarded((c.N,))
    dx, dw = guarded((c.N, c.C), c.t), guarded((c.K, c.C), c.t)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.fc_softmax_xent_fwd(c.N, c.C, c.K, c.x, c.w, None, c.labels, loss, row, lse, ignore_label=IGNORE, ws=ws[0])
        B.fc_softmax_xent_bwd(c.N, c.C, c.K, c.x, c.w, None, c.labels, lse, None, dx, dw, None, ignore_label=IGNORE, ws=ws[1])
    for _ in range(2):
        c.x.normal_()
        g.replay()
        c.forward(); c.backward()
        torch.cuda.synchronize()
        assert torch.equal(loss, c.loss) and torch.equal(dx, c.dx) and torch.equal(dw, c.dw)
    c.check()


def test_short_workspace_is_refused():
    c = Case(40, 64, 100, torch.bfloat16)
    short = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.PclError) as e:
        B.fc_softmax_xent_fwd(40, 64, 100, c.x, c.w, None, c.labels, torch.empty(1, device="cuda"), torch.empty(40, device="cuda"),
                              torch.empty(40, device="cuda"), ws=short)
    assert e.value.code == B.ERR_WORKSPACE


def test_offsets_beyond_32_bits():
    """Weights and their gradient of more than 2^31 elements: the classes at the end are read and written in place."""
    N, C, K = 24, 4096, 530000
    w = torch.zeros(K, C, dtype=torch.bfloat16, device="cuda")
    dw = torch.empty_like(w)
    g = torch.Generator(device="cuda").manual_seed(18)
    x = torch.randn(N, C, device="cuda", generator=g).bfloat16()
    w[K - 40:] = (torch.randn(40, C, device="cuda", generator=g) / 8).bfloat16()
    labels = torch.randint(K - 40, K, (N,), device="cuda", generator=g).int()
    loss, row, lse, dx = torch.empty(1, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(x)
    ws = workspace(max(B.fc_softmax_xent_workspace_bytes(N, C, K, B.BF16, p) for p in (B.PASS_FWD, B.PASS_BWD_DATA)))
    B.fc_softmax_xent_fwd(N, C, K, x, w, None, labels, loss, row, lse, ws=ws)
    B.fc_softmax_xent_bwd(N, C, K, x, w, None, labels, lse, None, dx, dw, None, ws=ws)
    B.check_device_status()
    check_guards()
    z = x.double() @ w[K - 40:].double().t()
    ref = torch.logsumexp(torch.cat([z, torch.full((N, 1), math.log(K - 40), device="cuda", dtype=torch.float64)], 1), 1)
    # z off by 4098 * 2^-23 of the sum of its terms' sizes at most, and the sums of K terms
    ez = 4098 * 2.0 ** -23 * float((x.double().abs() @ w[K - 40:].double().abs().t()).max())
    assert bool(((lse.double() - ref).abs() <= ez + 2.0 ** -10).all())
    p = torch.exp(z - ref[:, None])
    p.scatter_add_(1, (labels.long() - (K - 40))[:, None], torch.full((N, 1), -1.0, device="cuda", dtype=torch.float64))
    want = (p / N).t() @ x.double()
    # dz and the result are rounded to bf16 (2^-8 each of their terms' sizes), p is off by the error of z and lse
    bound = (p.abs() / N * (2.0 ** -8 + 2 * ez + 2.0 ** -9) + 2.0 ** -9 * (p.abs() + 1) / N * 2 * ez).t() @ x.double().abs() + 2.0 ** -8 * want.abs() + 1e-9
    assert bool(((dw[K - 40:].double() - want).abs() <= bound).all())
    # everywhere else p is the same tiny number
    tiny = float(torch.exp(-ref).max()) / N * float(x.double().abs().sum(0).max()) * 1.1
    assert float(dw[: K - 40 : 997].abs().max()) <= tiny


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("C", [128, 131])
def test_equal_row_gradients_are_a_factor(t, C):
    """The same gradient c for every row: its own rounding to 16 bits must not be in every element of the result."""
    c = 1 + 2.0 ** -12 + 2.0 ** -9 + 2.0 ** -8 if t == torch.float16 else 1 + 2.0 ** -9 + 2.0 ** -5
    results = []
    for grad in (1.0, c):
        case = Case(300, C, 500, t, False, 0.0)
        case.row_grad = guarded((300,))
        case.row_grad.fill_(grad)
        case.forward()
        case.backward()
        check_guards()
        results.append([v.double() for v in (case.dx, case.dw)])
    for one, both in zip(*results):
        # the same sums, of dz of the same roundings: two roundings of the results remain (fp16: subnormals are absolute)
        assert bool(((both - c * one).abs() <= 2 * half_step(t) * (c * one).abs() * (1 + 2.0 ** -7) + 2.0 ** -24).all())


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("N,C,K", [(130, 64, 400), (40, 72, 9001)])
def test_rows_without_a_class_have_no_gradient(t, N, C, K):
    """Logits that all are -inf: lse -inf, loss inf, and dz exactly 0 for the row, as if it were left out with the same row gradients."""
    c = Case(N, C, K, t, True, 0.0, seed=19)
    c.w[:, 0] = 0.5                              # (so that a row of x that begins with -inf has no finite logit)
    lost = [0, 17, N - 1]
    c.x[lost, 0] = float("-inf")
    c.forward()
    c.backward()
    B.check_device_status()
    check_guards()
    assert bool((c.lse[lost] == float("-inf")).all()) and bool((c.row_loss[lost] == float("inf")).all())
    assert not bool(c.dx[lost].any())
    assert bool(c.dx.isfinite().all()) and bool(c.dw[:, 1:].isfinite().all()) and bool(c.db.isfinite().all())
    # (column 0 of dw is a product with -inf)
    dx, dw, db = c.dx, c.dw, c.db
    c.labels[lost] = IGNORE
    c.row_grad = guarded((N,))
    c.row_grad.fill_(1.0 / N)
    c.backward()
    B.check_device_status()
    assert torch.equal(c.dx, dx) and torch.equal(c.dw[:, 1:], dw[:, 1:]) and torch.equal(c.db, db)
    # every class of every row
    c = Case(N, C, K, t, True, 0.0, seed=20)
    c.bias.fill_(float("-inf"))
    c.forward()
    c.backward()
    B.check_device_status()
    assert not bool(c.dx.any()) and not bool(c.dw.any()) and not bool(c.db.any())


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32])
def test_the_lowest_label_is_ignored_only_if_asked_for(t):
    """-2^31 stands for "no label is special" as the ignored label, so that as a label it is one out of range like -1."""
    c = Case(60, 64, 200, t, True, 0.0, seed=21)
    c.ignore = None
    c.labels[7] = -1
    c.forward()
    assert B.last_device_status() == B.ERR_BAD_LABEL
    c.backward()
    want = [v.clone() for v in (c.loss, c.row_loss, c.dx, c.dw, c.db)]
    c.labels[7] = -2 ** 31
    c.forward()
    assert B.last_device_status() == B.ERR_BAD_LABEL
    c.backward()
    assert B.last_device_status() == B.OK
    for got, ref in zip((c.loss, c.row_loss, c.dx, c.dw, c.db), want):
        assert torch.equal(got, ref)


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("N,C,K", [(130, 64, 400), (8, 2048, 300), (40, 72, 9001)])
def test_nan_and_infinite_logits_at_a_masked_label(t, N, C, K):
    """A row with a NaN or +inf logit has NaN results, also where the label's own class is masked with -inf."""
    c = Case(N, C, K, t, True, 0.0, seed=22)
    c.bias[:9] = float("-inf")
    c.bias[40] = float("nan")
    c.labels[: N // 2] = 3
    c.forward()
    B.check_device_status()
    assert bool(c.lse.isnan().all()) and bool(c.row_loss.isnan().all()) and math.isnan(c.loss.item())
    c.bias[40] = float("inf")
    c.forward()
    B.check_device_status()
    assert bool(c.lse.isnan().all()) and bool(c.row_loss.isnan().all())


@pytest.mark.parametrize("N,C,K", [(256, 16384, 3500), (256, 4096, 1000), (128, 32768, 900)])
def test_long_sums_of_one_sign_in_parts(N, C, K):
    """Few rows, long fp16 reductions: no accumulator sums more than 2048 products.  The tensor core truncates at every addition of 16
    products, by less than 2^-23 of the sum: 128 additions, and the parts are added in fp32."""
    g = torch.Generator(device="cuda").manual_seed(23)
    c = Case(N, C, K, torch.float16)
    c.x.copy_(torch.rand(N, C, device="cuda", generator=g) + 0.5)
    c.w.copy_((torch.rand(K, C, device="cuda", generator=g) + 0.5) * (20 / C))
    c.forward()
    B.check_device_status()
    check_guards()
    z = c.x.double() @ c.w.double().t()
    lse = torch.logsumexp(z, 1)
    # (ex2, the sums over the classes and the log: 2^-18)
    assert float((c.lse.double() - lse).abs().max()) <= 128 * 2.0 ** -23 * float(z.max()) + (C / 2048 + 2) * 2.0 ** -24 * float(z.max()) + 2.0 ** -18
