"""The checks of the calls for deep networks exist twice, compiled and in the interpreter: both take the same calls, refuse the same with the same words
and leave the same results."""
import numpy as np
import pytest
import torch

from gpu_helpers import guarded, workspace
from paper_1602_06709_b200 import binding as B

pytestmark = pytest.mark.gpu

N, C, K, T = 6, 32, 48, torch.bfloat16


def real(*shape, t=T, seed=0):
    out = guarded(shape, t, fill=0)
    out.copy_(torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + sum(shape))))
    return out


def bytes8(*shape):
    q = guarded(shape, torch.uint8, fill=0)
    q.copy_(real(*shape, t=torch.float32).to(B.E4M3).view(torch.uint8))
    return q


def f32(*shape, fill=0.5):
    return guarded(shape, torch.float32, fill=fill)


def calls():
    """name -> (call, its arguments by name; sizes first)"""
    lists = lambda seed: B.TensorList([real(5, t=torch.float32, seed=seed), real(70, seed=seed), real(33, t=torch.float16, seed=seed)])
    i32 = lambda fill: guarded((N,), torch.int32, fill=fill)
    return {
        "rms_norm_fwd": (B.rms_norm_fwd, dict(N=N, C=C, x=real(N, C), residual=real(N, C, seed=1), w=real(C), eps=1e-6, h=real(N, C), y=real(N, C), rstd=f32(N))),
        "rms_norm_fwd_q8": (B.rms_norm_fwd_q8, dict(N=N, C=C, x=real(N, C), residual=real(N, C, seed=1), w=real(C), eps=1e-6, h=real(N, C), y8=bytes8(N, C),
                                                    y_scale=f32(N), rstd=f32(N))),
        "rms_norm_bwd": (B.rms_norm_bwd, dict(N=N, C=C, h=real(N, C), w=real(C), rstd=f32(N), dy=real(N, C, seed=2), dh=real(N, C, seed=3), dx=real(N, C),
                                              dw=real(C), ws=workspace(B.rms_norm_workspace_bytes(N, C)))),
        "quantize_rows": (B.quantize_rows, dict(N=N, C=C, x=real(N, C), q=bytes8(N, C), scale=f32(N))),
        "fc_q8_fwd": (B.fc_q8_fwd, dict(N=N, C=C, K=K, x=bytes8(N, C), x_scale=f32(N), w=bytes8(K, C), w_scale=f32(K), bias=real(K), y=real(N, K),
                                        act=B.ACT_RELU, ws=workspace(max(256, B.fc_q8_workspace_bytes(N, C, K))))),
        "grad_norm": (B.grad_norm, dict(grads=lists(1), norm=f32(1), ws=workspace(B.grad_norm_workspace_bytes(3)))),
        "grad_clip": (B.grad_clip, dict(grads=lists(1), out=lists(2), max_norm=0.5, norm=f32(1), ws=workspace(B.grad_norm_workspace_bytes(3)))),
        "sgd_update_clipped": (B.sgd_update_clipped, dict(params=lists(3), grads=lists(1), lr=0.0, max_norm=0.5, norm=f32(1),
                                                          ws=workspace(B.grad_norm_workspace_bytes(3)))),
        "sample_tokens": (B.sample_tokens, dict(N=N, K=K, logits=real(N, K), uniform=f32(N), token=i32(0), temperature=f32(N, fill=0.8), top_k=i32(9),
                                                top_p=f32(N, fill=0.9), min_p=f32(N, fill=0.01), logprob=f32(N), ws=workspace(256))),
    }


def others(v):
    """What may or may not be taken in place of an argument."""
    if isinstance(v, B.TensorList):
        return [B.TensorList([t.clone() for t in v.tensors]), B.TensorList([t.clone() for t in v.tensors[:2]])]
    if isinstance(v, torch.Tensor):
        flat = v.reshape(-1)
        longer = torch.cat([flat, flat])
        return [None, flat, longer, longer[::2], v.cpu(), v.double(), v.to(torch.float16 if v.dtype != torch.float16 else torch.float32),
                torch.nn.Parameter(v.clone(), requires_grad=v.is_floating_point()), np.zeros(3), longer[:0]]
    if isinstance(v, int):
        return [0, -1, True, np.int64(v), float(v), 2 ** 31 - 1, 2 ** 31, 2 ** 40, 2 ** 70, None, v - 1]
    return [0, 1, -1.0, float("nan"), float("inf"), np.float32(v), np.float64(v), None, "a", 1e300, torch.tensor(v)]


def outcome(call, args):
    for v in args.values():                                    # (what is written, some of it read before, starts out alike)
        if isinstance(v, B.TensorList):
            for i, t in enumerate(v.tensors):
                t.copy_(torch.arange(t.numel(), device="cuda") % (7 + i))
    try:
        call(**args)
    except Exception as e:
        return type(e).__name__, str(e)
    torch.cuda.synchronize()
    return "taken", None


def same(a, b):
    a, b = a.detach().double(), b.detach().double()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


NAMES = ["rms_norm_fwd", "rms_norm_fwd_q8", "rms_norm_bwd", "quantize_rows", "fc_q8_fwd", "grad_norm", "grad_clip", "sgd_update_clipped", "sample_tokens"]


@pytest.mark.parametrize("name", NAMES)
def test_both_take_and_refuse_the_same(name, monkeypatch):
    B.lib()
    assert B._calls is not None, "the compiled calls were not built"
    compiled = B._calls
    call, base = calls()[name]
    tried = taken = 0
    for key in [None] + list(base):
        for other in [None] if key is None else others(base[key]):
            results = []
            for with_compiled in (compiled, None):
                monkeypatch.setattr(B, "_calls", with_compiled)
                args = {k: v.clone() if isinstance(v, torch.Tensor) and k != "ws" else v for k, v in base.items()}
                if key is not None:
                    args[key] = other
                results.append((outcome(call, args), {k: v.clone() if isinstance(v, torch.Tensor) else [t.clone() for t in v.tensors] if isinstance(v, B.TensorList) else v
                                                      for k, v in args.items() if k != "ws"}))
            (first, one), (second, two) = results
            assert first == second, (key, other, first, second)
            tried, taken = tried + 1, taken + (first[0] == "taken")
            if first[0] == "taken":
                for k, a in one.items():
                    b = two[k]
                    if isinstance(a, list):
                        assert all(map(same, a, b)), (key, k)
                    elif isinstance(a, torch.Tensor):
                        assert same(a, b), (key, k)
    assert 3 < taken < tried


def test_other_threads_run_meanwhile():
    """The library is called with the interpreter free: here a function that waits half a second stands in its place."""
    import ctypes
    import threading
    import time
    lib = B.lib()
    table = {n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in B._COMPILED}
    wait = ctypes.cast(ctypes.CDLL(None).usleep, ctypes.c_void_p).value
    n = 500000                                                 # (the call's first argument: microseconds)
    x, w = torch.zeros(n, 1, device="cuda"), torch.ones(1, device="cuda")
    ticks, stop = [], threading.Event()

    def tick():
        while not stop.wait(0.01):
            ticks.append(time.monotonic())

    B._calls.bind({**table, "pcl_rms_norm_fwd": wait})
    other = threading.Thread(target=tick)
    try:
        other.start()
        begin = time.monotonic()
        assert B._calls.rms_norm_fwd(n, 1, x, None, w, 1e-6, None, x, None, None) == 0
        end = time.monotonic()
    finally:
        B._calls.bind(table)
        stop.set()
        other.join()
    assert end - begin > 0.4 and sum(begin + 0.05 < t < end - 0.05 for t in ticks) > 5
