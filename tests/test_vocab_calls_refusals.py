"""Host-side refusals of the embedding, FC softmax cross-entropy and orthogonalised-update calls: every one returns its
error code before anything is launched, so none of this needs a GPU."""
import ctypes

import pytest

P = ctypes.c_void_p
NULL, OK16, ODD = P(0), P(4096), P(4100)


@pytest.fixture(scope="module")
def B():
    from paper_1602_06709_b200 import build
    build.build()
    from paper_1602_06709_b200 import binding
    return binding


def f(x):
    return ctypes.c_float(x)


def test_embedding_refusals(B):
    L = B.lib()
    fwd = lambda N=4, V=8, C=8, d=0, ids=OK16, t=OK16, o=OK16: L.pcl_embedding_fwd(N, V, C, d, ids, t, f(1), 0, o, NULL)
    for bad in (dict(N=0), dict(V=0), dict(C=-1), dict(d=3), dict(d=-1), dict(ids=NULL), dict(t=NULL), dict(o=NULL)):
        assert fwd(**bad) == B.ERR_BAD_ARG, bad
    for bad in (dict(ids=ODD), dict(t=ODD), dict(o=ODD)):
        assert fwd(**bad) == B.ERR_MISALIGNED, bad
    assert fwd(V=2 ** 31 - 1) == B.ERR_UNSUPPORTED_SHAPE
    need = B.embedding_workspace_bytes(4, 8, 8)
    assert need > 0 and B.embedding_workspace_bytes(0, 8, 8) == 0
    bwd = lambda ws=OK16, wb=need, dy=OK16: L.pcl_embedding_bwd(4, 8, 8, 0, OK16, dy, f(1), 0, OK16, ws, wb, NULL)
    assert bwd(ws=NULL) == B.ERR_WORKSPACE and bwd(wb=need - 1) == B.ERR_WORKSPACE
    assert bwd(ws=P(4096 + 16)) == B.ERR_MISALIGNED and bwd(dy=NULL) == B.ERR_BAD_ARG
    assert L.pcl_embedding_bwd_sgd(4, 8, 8, 0, OK16, OK16, f(1), 0, NULL, f(1), OK16, need, NULL) == B.ERR_BAD_ARG
    assert L.pcl_embedding_bwd_sgd(4, 8, 8, 0, OK16, OK16, f(1), 0, OK16, f(1), OK16, need - 1, NULL) == B.ERR_WORKSPACE


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_vocab_loss_refusals(B, dtype):
    L = B.lib()
    N, C, K = 4, 16, 24
    need = {p: B.fc_softmax_xent_workspace_bytes(N, C, K, dtype, p) for p in (B.PASS_FWD, B.PASS_BWD_DATA)}
    assert all(v > 0 for v in need.values())
    assert B.fc_softmax_xent_workspace_bytes(N, C, K, dtype, B.PASS_BWD_WEIGHTS) == 0
    assert B.fc_softmax_xent_workspace_bytes(N, C, 0, dtype, B.PASS_FWD) == 0

    def fwd(N=N, C=C, K=K, d=dtype, x=OK16, w=OK16, b=NULL, lab=OK16, loss=OK16, row=OK16, lse=OK16, ws=OK16, wb=need[B.PASS_FWD]):
        return L.pcl_fc_softmax_xent_fwd(N, C, K, d, x, w, b, lab, -1, loss, row, lse, ws, wb, NULL)

    def bwd(lse=OK16, rg=NULL, dx=NULL, dw=OK16, db=NULL, ws=OK16, wb=need[B.PASS_BWD_DATA], d=dtype):
        return L.pcl_fc_softmax_xent_bwd(N, C, K, d, OK16, OK16, NULL, OK16, -1, lse, rg, dx, dw, db, ws, wb, NULL)

    for bad in (dict(N=0), dict(C=0), dict(K=0), dict(d=7), dict(x=NULL), dict(w=NULL), dict(lab=NULL), dict(loss=NULL),
                dict(row=NULL), dict(lse=NULL)):
        assert fwd(**bad) == B.ERR_BAD_ARG, bad
    for bad in (dict(x=ODD), dict(w=ODD), dict(b=ODD), dict(lab=ODD), dict(loss=ODD), dict(row=ODD), dict(lse=ODD), dict(ws=P(4096 + 64))):
        assert fwd(**bad) == B.ERR_MISALIGNED, bad
    assert fwd(ws=NULL) == B.ERR_WORKSPACE and fwd(wb=need[B.PASS_FWD] - 1) == B.ERR_WORKSPACE
    for bad in (dict(lse=NULL), dict(dw=NULL), dict(d=-2)):
        assert bwd(**bad) == B.ERR_BAD_ARG, bad
    for bad in (dict(lse=ODD), dict(rg=ODD), dict(dx=ODD), dict(dw=ODD), dict(db=ODD), dict(ws=P(4096 + 64))):
        assert bwd(**bad) == B.ERR_MISALIGNED, bad
    assert bwd(ws=NULL) == B.ERR_WORKSPACE and bwd(wb=need[B.PASS_BWD_DATA] - 1) == B.ERR_WORKSPACE


def test_orthogonalize_refusals(B):
    L = B.lib()
    need = B.orthogonalize_workspace_bytes(2, 8, 16)
    assert need > 0 and B.orthogonalize_workspace_bytes(2, 0, 16) == 0

    def call(count=2, M=8, N=16, d=1, g=OK16, o=OK16, steps=5, ws=OK16, wb=need):
        return L.pcl_orthogonalize(count, M, N, d, g, o, steps, ws, wb, NULL)

    for bad in (dict(count=0), dict(M=0), dict(N=-3), dict(d=9), dict(g=NULL), dict(o=NULL), dict(steps=0)):
        assert call(**bad) == B.ERR_BAD_ARG, bad
    assert call(g=ODD) == B.ERR_MISALIGNED and call(o=ODD) == B.ERR_MISALIGNED and call(ws=P(4096 + 16)) == B.ERR_MISALIGNED
    assert call(ws=NULL) == B.ERR_WORKSPACE and call(wb=need - 1) == B.ERR_WORKSPACE
    assert call(count=65536, wb=1 << 50) == B.ERR_UNSUPPORTED_SHAPE

    def update(w=OK16, dw=OK16, m=OK16, wb=need):
        return L.pcl_orthogonal_update(2, 8, 16, 1, w, dw, m, f(0.9), 1, f(0.1), f(0), 5, OK16, wb, NULL)

    assert update(m=NULL) == B.ERR_BAD_ARG and update(w=NULL) == B.ERR_BAD_ARG and update(dw=NULL) == B.ERR_BAD_ARG
    assert update(m=ODD) == B.ERR_MISALIGNED and update(wb=0) == B.ERR_WORKSPACE


def test_binding_checks_types_and_sizes(B):
    import torch
    a = torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError):
        B.embedding_fwd(4, 4, 8, ids, a, 1.0, a.clone())
    with pytest.raises(TypeError):
        B.embedding_fwd(4, 4, 8, ids.int(), a.double(), 1.0, a.clone())
    with pytest.raises(ValueError):
        B.embedding_fwd(4, 5, 8, ids.int(), a, 1.0, a.clone())
    with pytest.raises(ValueError):          # not on a CUDA device
        B.embedding_fwd(4, 4, 8, ids.int(), a, 1.0, a.clone())
    with pytest.raises(B.PclError):
        B.orthogonalize(0, 4, 8, a, a)


def test_forced_kernel_families(B):
    """A forced family that a call cannot run on is refused before anything is launched."""
    L = B.lib()
    big = 1 << 40
    loss = lambda C, K, d: L.pcl_fc_softmax_xent_bwd(4, C, K, d, OK16, OK16, NULL, OK16, -1, OK16, NULL, NULL, OK16, NULL, OK16, big, NULL)
    fwd = lambda C, K, d: L.pcl_fc_softmax_xent_fwd(4, C, K, d, OK16, OK16, NULL, OK16, -1, OK16, OK16, OK16, OK16, big, NULL)
    try:
        B.set_path(B.PATH_TENSOR)
        assert loss(6, 8, B.F32) == B.ERR_UNSUPPORTED_SHAPE and loss(8, 7, B.F32) == B.ERR_UNSUPPORTED_SHAPE
        assert fwd(6, 8, B.F32) == B.ERR_UNSUPPORTED_SHAPE
        B.set_path(B.PATH_GENERIC)
        assert fwd(8, 8, B.BF16) == B.ERR_UNSUPPORTED_SHAPE and loss(8, 8, B.F16) == B.ERR_UNSUPPORTED_SHAPE
        assert L.pcl_orthogonalize(1, 8, 8, B.F32, OK16, OK16, 5, OK16, big, NULL) == B.ERR_UNSUPPORTED_SHAPE
    finally:
        B.set_path(B.PATH_AUTO)


@pytest.mark.parametrize("size", [2 ** 31 - 1, 2 ** 31 - 16, 2 ** 31 - 9000, 2 ** 31 - 65536])
def test_sizes_that_indices_would_pass_32_bits_for(B, size):
    """Kernels step through a dimension by up to a grid of blocks: the last sizes of an int are refused before anything is launched."""
    L, big = B.lib(), 1 << 60
    for N, V, C in ((size, 4, 4), (4, size, 4), (4, 4, size)):
        assert L.pcl_embedding_fwd(N, V, C, 1, OK16, OK16, f(1), 0, OK16, NULL) == B.ERR_UNSUPPORTED_SHAPE
        assert L.pcl_embedding_bwd(N, V, C, 1, OK16, OK16, f(1), 0, OK16, OK16, big, NULL) == B.ERR_UNSUPPORTED_SHAPE
        assert L.pcl_embedding_bwd_sgd(N, V, C, 1, OK16, OK16, f(1), 0, OK16, f(1), OK16, big, NULL) == B.ERR_UNSUPPORTED_SHAPE
        assert B.embedding_workspace_bytes(N, V, C) == 0
        for d in (0, 1, 2):
            assert L.pcl_fc_softmax_xent_fwd(N, V, C, d, OK16, OK16, NULL, OK16, -1, OK16, OK16, OK16, OK16, big, NULL) == B.ERR_UNSUPPORTED_SHAPE
            assert L.pcl_fc_softmax_xent_bwd(N, V, C, d, OK16, OK16, NULL, OK16, -1, OK16, NULL, NULL, OK16, NULL, OK16, big, NULL) == B.ERR_UNSUPPORTED_SHAPE
            assert B.fc_softmax_xent_workspace_bytes(N, V, C, d, B.PASS_FWD) == 0 and B.fc_softmax_xent_workspace_bytes(N, V, C, d, B.PASS_BWD_DATA) == 0
    for M, N in ((size, 4), (4, size)):
        assert L.pcl_orthogonalize(1, M, N, 1, OK16, OK16, 5, OK16, big, NULL) == B.ERR_UNSUPPORTED_SHAPE
        assert L.pcl_orthogonal_update(1, M, N, 1, OK16, OK16, OK16, f(0.9), 1, f(0.1), f(0), 5, OK16, big, NULL) == B.ERR_UNSUPPORTED_SHAPE
        assert B.orthogonalize_workspace_bytes(1, M, N) == 0
    assert B.orthogonalize_workspace_bytes(65536, 4, 4) == 0


def test_integers_beyond_32_bits(B):
    """ctypes cuts integers to 32 bits: 2^32 would be the id 0."""
    import torch
    a, ids = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    assert B._id(None) == B.NO_ID and B._id(-2 ** 31) == B.NO_ID and B._id(2 ** 31 - 1) == 2 ** 31 - 1 and B._id(-1) == -1
    for v in (2 ** 31, 2 ** 32, -2 ** 31 - 1):
        with pytest.raises(ValueError):
            B._id(v)
    for steps in (2 ** 32 + 5, 0, -1, 5.0):
        with pytest.raises(B.PclError) as e:
            B.orthogonalize(1, 4, 8, a, a, steps=steps)
        assert e.value.code == B.ERR_BAD_ARG
        with pytest.raises(B.PclError):
            B.orthogonal_update(1, 4, 8, a, a, a, 0.9, True, 0.1, steps=steps)
    with pytest.raises(B.PclError):
        B.embedding_fwd(4, 2 ** 32 + 4, 8, ids, a, 1.0, a)
    assert B.embedding_workspace_bytes(4, 2 ** 32 + 4, 8) == 0 and B.orthogonalize_workspace_bytes(1, 2 ** 32 + 4, 8) == 0
    assert B.fc_softmax_xent_workspace_bytes(4, 8, 2 ** 32 + 4, B.BF16, B.PASS_FWD) == 0


def test_a_workspace_of_another_device(B):
    import torch

    class OnDevice:
        """What the checks ask a tensor."""
        def __init__(self, n, dtype, device):
            self.n, self.dtype, self.device = n, dtype, device
        def numel(self): return self.n
        def get_device(self): return self.device
        def is_contiguous(self): return True

    mk = lambda n, dt=torch.float32: OnDevice(n, dt, 0)
    a, r, ids = mk(32), mk(4), mk(4, torch.int32)
    for device in (1, -1):
        ws = OnDevice(1 << 20, torch.uint8, device)
        for call in (lambda: B.embedding_bwd(4, 4, 8, ids, a, 1.0, a, ws=ws), lambda: B.embedding_bwd_sgd(4, 4, 8, ids, a, 1.0, a, 0.1, ws=ws),
                     lambda: B.fc_softmax_xent_fwd(4, 8, 4, a, a, None, ids, mk(1), r, r, ws=ws),
                     lambda: B.fc_softmax_xent_bwd(4, 8, 4, a, a, None, ids, r, None, a, a, None, ws=ws),
                     lambda: B.orthogonalize(1, 4, 8, a, a, ws=ws), lambda: B.orthogonal_update(1, 4, 8, a, a, a, 0.9, True, 0.1, ws=ws)):
            with pytest.raises(ValueError, match="current CUDA device"):
                call()
