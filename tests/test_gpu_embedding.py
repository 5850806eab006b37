"""Embedding lookup and its gradient by sorted tokens against plain float64 computations."""
import numpy as np
import pytest
import torch

from gpu_helpers import check_guards, guarded, workspace
from paper_1602_06709_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def half_step(t):
    return torch.finfo(t).eps / 2


def smallest(t):
    """Half of the spacing of the subnormal numbers."""
    f = torch.finfo(t)
    return f.tiny * f.eps / 2


def put(shape, t, std, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = guarded(shape, t, fill=0)
    out.copy_(torch.randn(shape, device="cuda", generator=g) * std)
    return out


def make_ids(n, v, kind, seed):
    r = np.random.default_rng(seed)
    if kind == "uniform":
        ids = r.integers(0, v, n)
    elif kind == "same":
        ids = np.full(n, v - 1)
    elif kind == "zipf":
        ids = np.minimum((np.exp(r.random(n) * np.log(max(v, 2))) - 1).astype(np.int64), v - 1)
    elif kind == "two":
        ids = np.where(r.random(n) < 0.9, 0, v - 1)
    else:
        ids = np.arange(n) % v
    out = guarded((n,), torch.int32, fill=0)
    out.copy_(torch.from_numpy(ids.astype(np.int32)))
    return out


def reference_grad(ids, dy, V, scale, pad):
    out = torch.zeros(V, dy.shape[1], dtype=torch.float64)
    ids, dy = ids.cpu().long(), dy.cpu().double()
    keep = torch.ones(len(ids), dtype=torch.bool) if pad is None else ids != pad
    keep &= (ids >= 0) & (ids < V)
    out.index_put_((ids[keep],), dy[keep], accumulate=True)
    mag = torch.zeros_like(out).index_put_((ids[keep],), dy[keep].abs(), accumulate=True)
    return out * scale, mag * abs(scale)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,V,C,pad", [(1, 1, 1, None), (1, 7, 8, 3), (5, 3, 33, None), (16, 100, 64, 0), (129, 50, 257, 49),
                                       (700, 1000, 2056, None), (33, 9, 4104, 2)])
def test_forward(t, N, V, C, pad):
    table = put((V, C), t, 1.0, 1)
    ids = make_ids(N, V, "uniform", N)
    out = guarded((N, C), t)
    scale = 1.7
    B.embedding_fwd(N, V, C, ids, table, scale, out, pad_id=pad)
    B.check_device_status()
    check_guards()
    ref = table.double()[ids.long()] * float(np.float32(scale))
    if pad is not None:
        ref[ids == pad] = 0
    # the product in fp32 (2^-24) and one rounding
    assert bool(((out.double() - ref).abs() <= ref.abs() * (half_step(t) + 2.0 ** -23) + smallest(t)).all())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("N,V,C,kind,pad", [
    (1, 1, 1, "uniform", None), (1, 300, 16, "uniform", None), (31, 5, 40, "uniform", 2), (32, 40, 8, "mod", None),
    (33, 33, 7, "mod", None), (64, 3, 24, "same", None), (65, 2, 24, "two", None), (1000, 70000, 64, "zipf", 0),
    (4097, 513, 136, "zipf", None), (5000, 300, 33, "uniform", 17), (9000, 2, 16, "two", 1), (20000, 131072, 8, "uniform", None),
    (3000, 16777300, 8, "uniform", None), (40000, 1000, 8, "zipf", None)])
@pytest.mark.parametrize("sgd", [False, True])
def test_gradient(t, N, V, C, kind, pad, sgd):
    ids = make_ids(N, V, kind, N + V)
    dy = put((N, C), t, 1.0, 2)
    scale, lr = -0.75, 0.125
    ws = workspace(B.embedding_workspace_bytes(N, V, C))
    ref, mag = reference_grad(ids, dy, V, scale, pad)
    count = int(torch.bincount(ids.cpu().long().clamp(min=0)).max())
    # fp32 sums of at most `count` terms (2^-24 per addition), the scaling, one rounding
    add = (count + 2) * 2.0 ** -24 * mag
    if sgd:
        table = put((V, C), t, 1.0, 3)
        before = table.clone()
        B.embedding_bwd_sgd(N, V, C, ids, dy, scale, table, lr, pad_id=pad, ws=ws)
        B.check_device_status()
        check_guards()
        want = before.cpu().double() - lr * ref
        bound = (half_step(t) + 2.0 ** -23) * want.abs() + 2.0 ** -23 * lr * ref.abs() + lr * add + smallest(t)
        assert bool(((table.cpu().double() - want).abs() <= bound).all())
        untouched = torch.ones(V, dtype=torch.bool)
        seen = ids.cpu().long()
        untouched[seen if pad is None else seen[seen != pad]] = False
        assert torch.equal(table.cpu()[untouched], before.cpu()[untouched])
        return
    out = guarded((V, C), t)
    B.embedding_bwd(N, V, C, ids, dy, scale, out, pad_id=pad, ws=ws)
    B.check_device_status()
    check_guards()
    got = out.cpu().double()
    assert bool(((got - ref).abs() <= (half_step(t) + 2.0 ** -23) * ref.abs() + add + smallest(t)).all())
    again = guarded((V, C), t)
    B.embedding_bwd(N, V, C, ids, dy, scale, again, pad_id=pad, ws=ws)
    assert torch.equal(out, again)                        # fixed order of the additions


def test_gradient_against_differences():
    """sum(dy * embedding(table)) is linear in the table: its differences are the gradient up to fp32 rounding."""
    N, V, C, scale = 37, 11, 12, 0.5
    ids = make_ids(N, V, "zipf", 4)
    table, dy = put((V, C), torch.float32, 1.0, 5), put((N, C), torch.float32, 1.0, 6)
    out, grad = guarded((N, C)), guarded((V, C))
    B.embedding_bwd(N, V, C, ids, dy, scale, grad, ws=workspace(B.embedding_workspace_bytes(N, V, C)))
    for v, c in ((0, 0), (1, 5), (10, 11), (3, 7)):
        vals = []
        for h in (1.0, -1.0):
            moved = table.clone()
            moved[v, c] += h
            B.embedding_fwd(N, V, C, ids, moved, scale, out)
            vals.append(float((dy.double() * out.double()).sum()))
        # both sums hold fp32-rounded products: N * C terms of size <= 4, each off by 2^-24 at most
        assert abs((vals[0] - vals[1]) / 2 - float(grad[v, c])) <= N * C * 4 * 2.0 ** -22


@pytest.mark.parametrize("bad", [-1, 100, -2 ** 31 + 1, 2 ** 31 - 1])
def test_ids_without_a_row(bad):
    N, V, C = 70, 100, 40
    ids = make_ids(N, V, "uniform", 7)
    ids[5] = bad
    ids[69] = bad
    table, dy = put((V, C), torch.float32, 1.0, 8), put((N, C), torch.float32, 1.0, 9)
    out, grad = guarded((N, C)), guarded((V, C))
    B.embedding_fwd(N, V, C, ids, table, 1.0, out)
    assert B.last_device_status() == B.ERR_BAD_LABEL and B.last_device_status() == B.OK
    assert bool((out[5] == 0).all()) and bool((out[69] == 0).all())
    B.embedding_bwd(N, V, C, ids, dy, 1.0, grad, ws=workspace(B.embedding_workspace_bytes(N, V, C)))
    assert B.last_device_status() == B.ERR_BAD_LABEL
    ref, mag = reference_grad(ids, dy, V, 1.0, None)
    assert bool(((grad.cpu().double() - ref).abs() <= N * 2.0 ** -23 * mag).all())
    # the same id as the padding id is no error
    B.embedding_fwd(N, V, C, ids, table, 1.0, out, pad_id=bad)
    B.embedding_bwd(N, V, C, ids, dy, 1.0, grad, pad_id=bad, ws=workspace(B.embedding_workspace_bytes(N, V, C)))
    assert B.last_device_status() == B.OK


def test_all_tokens_padding():
    N, V, C = 50, 6, 16
    ids = torch.full((N,), 2, dtype=torch.int32, device="cuda")
    table, dy = put((V, C), torch.bfloat16, 1.0, 10), put((N, C), torch.bfloat16, 1.0, 11)
    out, grad = guarded((N, C), torch.bfloat16), guarded((V, C), torch.bfloat16)
    ws = workspace(B.embedding_workspace_bytes(N, V, C))
    B.embedding_fwd(N, V, C, ids, table, 1.0, out, pad_id=2)
    B.embedding_bwd(N, V, C, ids, dy, 1.0, grad, pad_id=2, ws=ws)
    before = table.clone()
    B.embedding_bwd_sgd(N, V, C, ids, dy, 1.0, table, 0.5, pad_id=2, ws=ws)
    B.check_device_status()
    assert bool((out == 0).all()) and bool((grad == 0).all()) and torch.equal(table, before)


def test_infinities_and_nan_stay_in_their_rows():
    N, V, C = 40, 20, 24
    ids = make_ids(N, V, "mod", 0)
    dy = put((N, C), torch.float32, 1.0, 12)
    dy[3] = float("inf"); dy[23] = float("-inf"); dy[4] = float("nan")
    grad = guarded((V, C))
    B.embedding_bwd(N, V, C, ids, dy, 1.0, grad, ws=workspace(B.embedding_workspace_bytes(N, V, C)))
    B.check_device_status()
    assert bool(grad[3].isnan().all()) and bool(grad[4].isnan().all())
    keep = [v for v in range(V) if v not in (3, 4)]
    assert bool(grad[keep].isfinite().all())


def test_offsets_beyond_32_bits():
    """A table and a gradient of more than 2^32 bytes and 2^31 elements: the last rows are read and written in place."""
    V, C, N = 530000, 4096, 64                            # 2.17e9 elements, 4.3 GB
    table = torch.zeros(V, C, dtype=torch.bfloat16, device="cuda")
    ids = torch.arange(V - N, V, dtype=torch.int32, device="cuda")
    table[V - N:] = torch.randn(N, C, device="cuda").bfloat16()
    out = guarded((N, C), torch.bfloat16)
    B.embedding_fwd(N, V, C, ids, table, 1.0, out)
    assert torch.equal(out, table[V - N:])
    dy = put((N, C), torch.bfloat16, 1.0, 13)
    ws = workspace(B.embedding_workspace_bytes(N, V, C))
    table.fill_(3.0)
    B.embedding_bwd(N, V, C, ids, dy, 1.0, table, ws=ws)
    B.check_device_status()
    assert torch.equal(table[V - N:], dy) and not bool(table[:V - N].any())


def test_graph_replay_and_second_stream():
    """Captured calls replay with new data in the same buffers; a call on another stream gives the same bits."""
    N, V, C = 3000, 700, 96
    ids, dy = make_ids(N, V, "zipf", 14), put((N, C), torch.float32, 1.0, 15)
    ws, ws2 = (workspace(B.embedding_workspace_bytes(N, V, C)) for _ in range(2))
    grad, eager = guarded((V, C)), guarded((V, C))
    B.embedding_bwd(N, V, C, ids, dy, 1.0, eager, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.embedding_bwd(N, V, C, ids, dy, 1.0, grad, ws=ws)
    for seed in (16, 17):
        ids.copy_(make_ids(N, V, "uniform", seed)); dy.normal_()
        g.replay()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            B.embedding_bwd(N, V, C, ids, dy, 1.0, eager, ws=ws2)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(grad, eager)


@pytest.mark.parametrize("N", [1, 31, 32, 33, 2047, 4095, 4096, 4097])
def test_workspace_that_held_anything(N):
    """What the workspace held before the call (the segments of an earlier one, or all ones) does not matter."""
    V, C = 700, 40
    g = torch.Generator(device="cuda").manual_seed(N)
    ws = workspace(B.embedding_workspace_bytes(N, V, C))
    for fill in (0, 255, None):
        if fill is not None:
            ws.fill_(fill)
        ids = torch.randint(-1 if fill else 0, V if fill else V // 2, (N,), device="cuda", generator=g).int()
        dy = torch.randn(N, C, device="cuda", generator=g)
        dt = guarded((V, C))
        B.embedding_bwd(N, V, C, ids, dy, 0.5, dt, pad_id=-1, ws=ws)
        B.check_device_status()
        check_guards()
        want = torch.zeros(V, C, dtype=torch.float64, device="cuda")
        size = torch.zeros(V, C, dtype=torch.float64, device="cuda")
        rows, there = ids.long().clamp(min=0), (ids >= 0)[:, None]
        want.index_add_(0, rows, 0.5 * dy.double() * there)
        size.index_add_(0, rows, 0.5 * dy.double().abs() * there)
        # at most N additions and the scale, 2^-24 of the terms' sizes each
        assert bool(((dt.double() - want).abs() <= (int(there.sum()) + 1) * 2.0 ** -24 * size).all())


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("C", [1, 2, 3, 4, 6, 12, 130, 132, 515, 1022])
def test_row_lengths(t, C):
    """Rows that start on multiples of one, two, four and eight elements."""
    N, V = 700, 90
    g = torch.Generator(device="cuda").manual_seed(C)
    ids = torch.randint(0, V // 2, (N,), device="cuda", generator=g).int()
    mk = lambda shape: guarded(shape, t, fill=0).copy_(torch.randn(shape, device="cuda", generator=g))
    table, dy, out, dt = mk((V, C)), mk((N, C)), guarded((N, C), t), guarded((V, C), t)
    old = table.double()
    ws = workspace(B.embedding_workspace_bytes(N, V, C))
    B.embedding_fwd(N, V, C, ids, table, 0.5, out)
    B.embedding_bwd(N, V, C, ids, dy, 0.5, dt, ws=ws)
    assert torch.equal(out, (0.5 * table.float()[ids.long()]).to(t))
    B.embedding_bwd_sgd(N, V, C, ids, dy, 0.5, table, 0.25, ws=ws)
    B.check_device_status()
    check_guards()
    want = torch.zeros(V, C, dtype=torch.float64, device="cuda").index_add_(0, ids.long(), 0.5 * dy.double())
    size = torch.zeros(V, C, dtype=torch.float64, device="cuda").index_add_(0, ids.long(), 0.5 * dy.double().abs())
    h, n = torch.finfo(t).eps / 2, int(torch.bincount(ids.long()).max())
    # n additions, the scale and the step in fp32 (2^-24 of the terms' sizes each), one rounding (fp16: subnormals are absolute)
    assert bool(((dt.double() - want).abs() <= (n + 2) * 2.0 ** -24 * size + h * want.abs() * 1.001 + 2.0 ** -25).all())
    new = old - 0.25 * want
    assert bool(((table.double() - new).abs() <= (n + 4) * 2.0 ** -24 * (size + old.abs()) + h * new.abs() * 1.001 + 2.0 ** -25).all())


@pytest.mark.parametrize("N", [70, 5000])
def test_the_lowest_id_is_out_of_range(N):
    """-2^31 stands for "no id is special" as the padding id, so that as an id it is one out of range like -1."""
    V, C = 100, 40
    ids = make_ids(N, V, "uniform", 7)
    ids[5] = -2 ** 31
    table, dy = put((V, C), torch.float32, 1.0, 8), put((N, C), torch.float32, 1.0, 9)
    out, grad = guarded((N, C)), guarded((V, C))
    ws = workspace(B.embedding_workspace_bytes(N, V, C))
    B.embedding_fwd(N, V, C, ids, table, 1.0, out)
    assert B.last_device_status() == B.ERR_BAD_LABEL and bool((out[5] == 0).all())
    B.embedding_bwd(N, V, C, ids, dy, 1.0, grad, ws=ws)
    assert B.last_device_status() == B.ERR_BAD_LABEL
    ref, mag = reference_grad(ids, dy, V, 1.0, None)
    assert bool(((grad.cpu().double() - ref).abs() <= N * 2.0 ** -23 * mag).all())
    B.embedding_bwd_sgd(N, V, C, ids, dy, 1.0, table, 0.5, ws=ws)
    assert B.last_device_status() == B.ERR_BAD_LABEL


@pytest.mark.parametrize("t,N,V,C,kind,pad", [
    # more tokens than one cluster's shared memory takes: the sorted sequence stays in global memory
    (torch.float32, 65537, 300, 8, "zipf", None), (torch.bfloat16, 70000, 1000, 24, "zipf", 0), (torch.float16, 70000, 90000, 33, "uniform", 5),
    (torch.float32, 66000, 2, 4, "two", 1), (torch.bfloat16, 200001, 513, 8, "zipf", None), (torch.bfloat16, 70000, 131072, 8, "mod", None),
    # the shared-memory sort's largest, and three digits of ids in either
    (torch.float32, 65536, 1000, 8, "uniform", None), (torch.float32, 5000, 16777300, 4, "zipf", None),
    (torch.bfloat16, 5000, 16777300, 4, "uniform", 3), (torch.bfloat16, 70000, 16777300, 4, "zipf", 0)])
@pytest.mark.parametrize("sgd", [False, True])
def test_gradient_of_many_tokens_and_many_rows(t, N, V, C, kind, pad, sgd):
    test_gradient(t, N, V, C, kind, pad, sgd)
