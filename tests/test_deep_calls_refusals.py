"""Host-side refusals of the RMS norm, 8-bit, gradient norm and token sampling calls: every one returns its error code before anything is
launched, so none of this needs a GPU."""
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


def test_rms_norm_refusals(B):
    L = B.lib()

    def fwd(N=4, C=8, d=1, x=OK16, r=OK16, w=OK16, eps=1e-6, h=OK16, y=OK16, rstd=NULL):
        return L.pcl_rms_norm_fwd(N, C, d, x, r, w, f(eps), h, y, rstd, NULL)

    def q8(N=4, C=8, d=1, x=OK16, r=OK16, w=OK16, eps=1e-6, h=OK16, y=OK16, s=OK16, rstd=NULL):
        return L.pcl_rms_norm_fwd_q8(N, C, d, x, r, w, f(eps), h, y, s, rstd, NULL)

    for call in (fwd, q8):
        for bad in (dict(N=0), dict(C=0), dict(N=-1), dict(d=3), dict(d=-1), dict(x=NULL), dict(w=NULL), dict(y=NULL), dict(r=NULL), dict(eps=-1.0),
                    dict(eps=float("nan")), dict(eps=float("inf"))):
            assert call(**bad) == B.ERR_BAD_ARG, bad
        for bad in (dict(x=ODD), dict(r=ODD), dict(w=ODD), dict(h=ODD), dict(y=ODD), dict(rstd=ODD)):
            assert call(**bad) == B.ERR_MISALIGNED, bad
        assert call(C=2 ** 31 - 1) == B.ERR_UNSUPPORTED_SHAPE and call(N=2 ** 31 - 1) == B.ERR_UNSUPPORTED_SHAPE
    assert q8(s=NULL) == B.ERR_BAD_ARG and q8(s=ODD) == B.ERR_MISALIGNED
    need = B.rms_norm_workspace_bytes(4, 8)
    assert need > 0 and B.rms_norm_workspace_bytes(0, 8) == 0 and B.rms_norm_workspace_bytes(4, 2 ** 31 - 1) == 0

    def bwd(N=4, C=8, d=1, h=OK16, w=OK16, rstd=OK16, dy=OK16, dh=NULL, dx=OK16, dw=OK16, ws=OK16, wb=need):
        return L.pcl_rms_norm_bwd(N, C, d, h, w, rstd, dy, dh, dx, dw, ws, wb, NULL)

    for bad in (dict(N=0), dict(C=-5), dict(d=3), dict(h=NULL), dict(w=NULL), dict(rstd=NULL), dict(dy=NULL), dict(dx=NULL)):
        assert bwd(**bad) == B.ERR_BAD_ARG, bad
    for bad in (dict(h=ODD), dict(w=ODD), dict(rstd=ODD), dict(dy=ODD), dict(dh=ODD), dict(dx=ODD), dict(dw=ODD), dict(ws=P(4096 + 16))):
        assert bwd(**bad) == B.ERR_MISALIGNED, bad
    assert bwd(ws=NULL) == B.ERR_WORKSPACE and bwd(wb=need - 1) == B.ERR_WORKSPACE
    q = lambda N=4, C=8, d=0, x=OK16, q=OK16, s=OK16: L.pcl_quantize_rows(N, C, d, x, q, s, NULL)
    for bad in (dict(N=0), dict(C=0), dict(d=3), dict(x=NULL), dict(q=NULL), dict(s=NULL)):
        assert q(**bad) == B.ERR_BAD_ARG, bad
    for bad in (dict(x=ODD), dict(q=ODD), dict(s=ODD)):
        assert q(**bad) == B.ERR_MISALIGNED, bad


def test_fc_q8_refusals(B):
    L = B.lib()
    need = B.fc_q8_workspace_bytes(4, 17, 8)
    assert need > 0 and B.fc_q8_workspace_bytes(4, 0, 8) == 0 and B.fc_q8_workspace_bytes(4, 16, 2 ** 31 - 1) == 0

    def call(N=4, C=17, K=8, d=1, x=OK16, xs=OK16, w=OK16, s=OK16, b=NULL, y=OK16, act=0, ws=OK16, wb=need):
        return L.pcl_fc_q8_fwd(N, C, K, d, x, xs, w, s, b, y, act, ws, wb, NULL)

    for bad in (dict(N=0), dict(C=0), dict(K=-1), dict(d=3), dict(act=3), dict(act=-1), dict(x=NULL), dict(xs=NULL), dict(w=NULL), dict(s=NULL), dict(y=NULL)):
        assert call(**bad) == B.ERR_BAD_ARG, bad
    for bad in (dict(x=ODD), dict(xs=ODD), dict(w=ODD), dict(s=ODD), dict(b=ODD), dict(y=ODD), dict(ws=P(4096 + 16))):
        assert call(**bad) == B.ERR_MISALIGNED, bad
    assert call(ws=NULL) == B.ERR_WORKSPACE and call(wb=need - 1) == B.ERR_WORKSPACE
    assert call(K=2 ** 31 - 1) == B.ERR_UNSUPPORTED_SHAPE
    B.set_path(B.PATH_GENERIC)
    try:
        assert call() == B.ERR_UNSUPPORTED_SHAPE
    finally:
        B.set_path(B.PATH_AUTO)


def test_grad_norm_refusals(B):
    L = B.lib()
    need = B.grad_norm_workspace_bytes(2)
    assert need > 0 and B.grad_norm_workspace_bytes(0) == 0 and B.grad_norm_workspace_bytes(-3) == 0

    def args(a=(4096, 8192), b=(16384, 32768), sizes=(5, 7), types=(0, 1), count=None):
        n = len(sizes)
        pa, pb = (P * n)(*a), (P * n)(*b)
        return count if count is not None else n, pa, pb, (ctypes.c_size_t * n)(*sizes), (ctypes.c_int * n)(*types)

    def norm(out=OK16, ws=OK16, wb=need, **k):
        n, a, _, s, t = args(**k)
        return L.pcl_grad_norm(n, a, s, t, out, ws, wb, NULL)

    def clip(out=OK16, ws=OK16, wb=need, most=1.0, **k):
        n, a, b, s, t = args(**k)
        return L.pcl_grad_clip(n, a, b, s, t, f(most), out, ws, wb, NULL)

    def sgd(out=OK16, ws=OK16, wb=need, most=1.0, **k):
        n, a, b, s, t = args(**k)
        return L.pcl_sgd_update_clipped(n, b, a, s, t, f(0.1), f(most), out, ws, wb, NULL)

    for call in (norm, clip, sgd):
        for bad in (dict(count=0), dict(count=-1), dict(types=(0, 3)), dict(types=(-1, 0)), dict(a=(0, 8192)), dict(out=NULL)):
            assert call(**bad) == B.ERR_BAD_ARG, bad
        for bad in (dict(a=(4098, 8192)), dict(a=(4096, 8193)), dict(out=P(4098)), dict(ws=P(4096 + 16))):
            assert call(**bad) == B.ERR_MISALIGNED, bad
        assert call(ws=NULL) == B.ERR_WORKSPACE and call(wb=need - 1) == B.ERR_WORKSPACE
        assert call(sizes=(5, 2 ** 34 + 1)) == B.ERR_UNSUPPORTED_SHAPE
    for call in (clip, sgd):
        for bad in (dict(b=(0, 8192)), dict(most=-1.0), dict(most=float("nan"))):
            assert call(**bad) == B.ERR_BAD_ARG, bad
        assert call(b=(4098, 8192)) == B.ERR_MISALIGNED
    assert L.pcl_grad_norm(2, NULL, NULL, NULL, OK16, OK16, need, NULL) == B.ERR_BAD_ARG


def test_sample_tokens_refusals(B):
    L = B.lib()
    need = B.sample_tokens_workspace_bytes(4, 100)

    def call(N=4, K=100, d=0, z=OK16, u=OK16, t=NULL, k=NULL, p=NULL, m=NULL, token=OK16, lp=NULL, ws=OK16, wb=need):
        return L.pcl_sample_tokens(N, K, d, z, u, t, k, p, m, token, lp, ws, wb, NULL)

    for bad in (dict(N=0), dict(K=0), dict(N=-1), dict(d=3), dict(z=NULL), dict(u=NULL), dict(token=NULL)):
        assert call(**bad) == B.ERR_BAD_ARG, bad
    for bad in (dict(z=ODD), dict(u=ODD), dict(t=ODD), dict(k=ODD), dict(p=ODD), dict(m=ODD), dict(token=ODD), dict(lp=ODD)):
        assert call(**bad) == B.ERR_MISALIGNED, bad
    assert call(K=2 ** 31 - 1) == B.ERR_UNSUPPORTED_SHAPE and B.sample_tokens_workspace_bytes(0, 5) == 0
    if need:
        assert call(ws=NULL) == B.ERR_WORKSPACE and call(wb=need - 1) == B.ERR_WORKSPACE


def test_binding_checks(B):
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):                    # not on a CUDA device
        B.rms_norm_fwd(4, 8, x, None, torch.zeros(8), 1e-6, None, torch.zeros(4, 8))
    with pytest.raises(B.PclError):
        B.rms_norm_fwd(2 ** 40, 8, x, None, torch.zeros(8), 1e-6, None, x)
    with pytest.raises(TypeError):
        B.rms_norm_fwd(4, 8, x, None, torch.zeros(8, dtype=torch.float64), 1e-6, None, torch.zeros(4, 8))
    with pytest.raises(ValueError):
        B.TensorList([])
    with pytest.raises(ValueError):
        B.TensorList([x])
    with pytest.raises(TypeError):
        B.dtype_code(x.double())
    with pytest.raises(TypeError):
        B.sample_tokens(4, 8, x.double(), torch.zeros(4), torch.zeros(4, dtype=torch.int32))
