"""Choice of tokens against a plain float64 computation that sorts each row: the token is the same, always."""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import guarded, workspace
from paper_1602_06709_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAN, INF = float("nan"), float("inf")


def pick(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log of its probability) of one row in numpy's 64 bits."""
    z = np.asarray(z, dtype=np.float64) + 0.0
    if np.isnan(z).any() or math.isnan(temperature) or z.max() == -INF:
        return -1, NAN
    if temperature <= 0 or top_k == 1 or top_p <= 0:
        return int(np.argmax(z)), 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.where(z == z.max(), 0.0, np.where(np.isneginf(z) | np.isinf(z.max()), -INF, (z - z.max()) / temperature))
    order = np.argsort(-z, kind="stable")
    w = np.exp(d[order])
    keep = np.ones(len(z), dtype=bool)
    if 0 < top_k <= len(z):
        keep[top_k:] = False
    w = w * keep
    if top_p < 1:
        before = np.cumsum(w) - w
        keep &= before < top_p * w.sum()
    if min_p > 0:
        keep &= w >= min(min_p, 1.0)
    ids = np.sort(order[keep])
    w = np.exp(d[ids])
    c = np.cumsum(w)
    u = 0.0 if not u > 0 else min(u, 1.0)
    at = min(int(np.searchsorted(c, u * c[-1], side="right")), len(ids) - 1)
    while w[at] == 0:
        at -= 1
    return int(ids[at]), float(d[ids[at]] - math.log(c[-1]))


def params(N, seed, kinds):
    """Per-row settings: each row has some of the filters."""
    r = np.random.default_rng(seed)
    p = {"uniform": r.random(N, dtype=np.float32)}
    if "temperature" in kinds:
        p["temperature"] = r.uniform(0.3, 2.0, N).astype(np.float32)
    if "top_k" in kinds:
        p["top_k"] = np.where(r.random(N) < 0.7, r.integers(1, 200, N), 0).astype(np.int32)
    if "top_p" in kinds:
        p["top_p"] = np.where(r.random(N) < 0.7, r.uniform(0.05, 0.999, N), 1.0).astype(np.float32)
    if "min_p" in kinds:
        p["min_p"] = np.where(r.random(N) < 0.7, 10 ** r.uniform(-4, -0.01, N), 0.0).astype(np.float32)
    return p


def device(a):
    t = guarded(a.shape, torch.int32 if a.dtype == np.int32 else torch.float32, fill=0)
    t.copy_(torch.from_numpy(a))
    return t


def run(z, p):
    N, K = z.shape
    token, logprob = guarded((N,), torch.int32, fill=-7), guarded((N,), torch.float32)
    ws = workspace(B.sample_tokens_workspace_bytes(N, K))
    B.sample_tokens(N, K, z, logprob=logprob, token=token, ws=ws, **{k: device(v) for k, v in p.items()})
    again = guarded((N,), torch.int32, fill=-7)
    B.sample_tokens(N, K, z, token=again, ws=ws, **{k: device(v) for k, v in p.items()})
    assert torch.equal(token, again)
    return token.cpu().numpy(), logprob.cpu().numpy().astype(np.float64)


def check(z, p):
    token, logprob = run(z, p)
    zn = z.double().cpu().numpy()
    for n in range(len(zn)):
        args = {k: (int(v[n]) if v.dtype == np.int32 else float(v[n])) for k, v in p.items() if k != "uniform"}
        t, l = pick(zn[n], float(p["uniform"][n]), **args)
        assert token[n] == t, (n, token[n], t, args, p["uniform"][n])
        # (the total is a sum of up to K weights, each off by 2^-44 of the largest at most: 6e-14 K; the logarithm is rounded to fp32 once)
        assert logprob[n] == l or (math.isnan(l) and math.isnan(logprob[n])) or abs(logprob[n] - l) <= abs(l) * 2.0 ** -24 + 6e-14 * zn.shape[1] + 1e-12


def logits(N, K, t, seed, kind="normal"):
    r = np.random.default_rng(seed)
    z = r.normal(0, 3, (N, K))
    if kind == "steps":                     # few different values: ties everywhere
        z = np.round(z * 0.5) * 2
    elif kind == "equal":
        z[:] = 1.25
    elif kind == "masked":
        z[r.random((N, K)) < 0.7] = -INF
        z[np.arange(N), r.integers(0, K, N)] = 0.5
    elif kind == "lowest":                  # masked with the type's lowest value
        z[r.random((N, K)) < 0.7] = torch.finfo(t).min
    elif kind == "peaks":
        z = -np.log(r.random((N, K)) + 1e-9) * r.uniform(0.5, 3, (N, 1))
    elif kind == "zeros":                   # zeros of both signs, the largest
        z = -np.abs(z)
        z[r.random((N, K)) < 0.3] = -0.0
        z[r.random((N, K)) < 0.3] = 0.0
    out = guarded((N, K), t, fill=0)
    out.copy_(torch.from_numpy(z))
    return out


FILTERS = [(), ("temperature",), ("top_k",), ("top_p",), ("min_p",), ("top_k", "top_p"), ("temperature", "top_k", "top_p", "min_p")]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("K", [1, 2, 31, 33, 257, 1000, 4097, 32003])
@pytest.mark.parametrize("kinds", FILTERS)
def test_sizes_and_filters(K, t, kinds):
    N = 24 if K < 10000 else 6
    check(logits(N, K, t, K, "normal"), params(N, K + 1, kinds))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("K", [5, 300, 5003])
@pytest.mark.parametrize("kind", ["steps", "equal", "masked", "lowest", "peaks", "zeros"])
@pytest.mark.parametrize("kinds", FILTERS[2:])
def test_distributions(K, t, kind, kinds):
    check(logits(16, K, t, 3 * K, kind), params(16, K + 2, kinds))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("K", [131072, 100003, 262147, 300000])
@pytest.mark.parametrize("kind", ["normal", "peaks", "steps", "masked"])
def test_large_vocabularies(K, t, kind):
    check(logits(5, K, t, K, kind), params(5, K + 3, FILTERS[-1]))
    check(logits(2, K, t, K + 1, kind), params(2, K + 4, ()))


def test_many_rows():
    check(logits(700, 501, torch.bfloat16, 5), params(700, 6, FILTERS[-1]))


def test_longer_than_2_to_18():
    """Weights of fewer bits: rows of 2^20 equal tokens, and of a few heavy ones among them."""
    K = 2 ** 20 + 5
    z = guarded((3, K), torch.float32, fill=0.0)
    z[1, 777777] = 12.0
    z[2, ::1000] = 5.0
    check(z, {"uniform": np.float32([0.37, 0.9, 0.5]), "top_p": np.float32([1.0, 1.0, 0.4])})


def test_frequencies():
    """A grid of random numbers chooses each token as often as its probability says."""
    K, N = 37, 4096
    z = logits(1, K, torch.float32, 8).expand(N, K).contiguous()
    u = ((np.arange(N) + 0.5) / N).astype(np.float32)
    token, _ = run(z, {"uniform": u, "top_p": np.full(N, 0.9, dtype=np.float32)})
    zn = z[0].double().cpu().numpy()
    p = np.exp(zn - zn.max())
    order = np.argsort(-p)
    c = np.cumsum(p[order]) / p.sum()
    kept = order[:int(np.searchsorted(c, 0.9)) + 1]
    want = np.zeros(K)
    want[kept] = p[kept] / p[kept].sum()
    count = np.bincount(token, minlength=K)
    assert (np.abs(count - want * N) <= 1).all()         # (an interval of length q holds q N grid points, one more or less)
    assert (np.diff(token) >= 0).all()


def test_special_rows():
    K = 4100
    z = logits(12, K, torch.float32, 9)
    z[0] = -INF
    z[1, 7] = NAN
    z[2, 40] = INF
    z[3, [5, 4000]] = INF
    z[4] = -INF
    z[4, 4099] = -3.0
    z[5, :] = torch.finfo(torch.float32).min
    z[6, 9] = torch.finfo(torch.float32).max
    z[11, 5] = -NAN
    p = {"uniform": np.float32([0.5, 0.5, 0.5, 0.9, 0.5, 0.25, 0.999, 0.5, 0.5, 0.5, 0.5, 0.5]),
         "temperature": np.float32([1, 1, 1, 1, 1, 1, 1, 0.0, -1.0, INF, NAN, 1]),
         "top_p": np.float32([0.9, 1, 0.9, 0.9, 0.9, 0.5, 0.5, 0.5, 0.5, 0.3, 0.5, 1])}
    check(z, p)


@pytest.mark.parametrize("name,value", [("top_k", -3), ("top_k", 10 ** 6), ("top_k", 300), ("top_p", 0.0), ("top_p", -1.0), ("top_p", NAN), ("top_p", 2.0),
                                        ("top_p", 1e-30), ("min_p", NAN), ("min_p", -1.0), ("min_p", 1.0), ("min_p", 7.0), ("min_p", 1e-38),
                                        ("temperature", 1e-30), ("temperature", 1e30), ("uniform", 1.0), ("uniform", 2.0),
                                        ("uniform", -1.0), ("uniform", NAN), ("uniform", 0.99999994), ("uniform", 0.0)])
def test_values_at_the_ends_of_the_settings(name, value):
    z = logits(4, 300, torch.float32, 10, "steps")
    p = {"uniform": np.float32([0.1, 0.4, 0.7, 0.95])}
    p[name] = np.full(4, value, dtype=np.int32 if name == "top_k" else np.float32)
    if name == "uniform":
        p["top_k"] = np.int32([0, 3, 50, 299])
    ends = dict(p)
    if name == "uniform":
        ends["uniform"] = np.where(np.isnan(p["uniform"]) | (p["uniform"] < 0), 0, np.minimum(p["uniform"], np.float32(1 - 2 ** -24))).astype(np.float32)
    if name == "top_p" and math.isnan(value):
        ends["top_p"] = np.ones(4, dtype=np.float32)
    if name == "min_p" and math.isnan(value):
        ends["min_p"] = np.zeros(4, dtype=np.float32)
    got = run(z, p)
    assert (got[0] == run(z, ends)[0]).all()
    check(z, ends)


@pytest.mark.parametrize("N,K", [(1, 32768), (4, 131075), (9, 262143), (18, 65537), (37, 65541), (74, 32771)])
@pytest.mark.parametrize("kinds", FILTERS)
def test_rows_shared_by_blocks(N, K, kinds):
    """Long rows and few of them: several blocks take a row together."""
    for t, kind in ((torch.bfloat16, "normal"), (torch.float32, "steps")):
        check(logits(N, K, t, N + K, kind), params(N, K + 5, kinds))


@pytest.mark.parametrize("K", [131072, 131075])
def test_special_rows_shared_by_blocks(K):
    z = logits(16, K, torch.float32, 9)
    z[0] = -INF
    z[1, K - 2] = NAN
    z[2, 40] = INF
    z[3, [5, K // 2, K - 1]] = INF
    z[4] = -INF
    z[4, K - 1] = -3.0
    z[5, :] = torch.finfo(torch.float32).min
    z[6, 9] = torch.finfo(torch.float32).max
    z[7] = -INF                             # all that is left lies with one block
    z[7, K - 300:] = logits(1, 300, torch.float32, 10)[0]
    z[8] = -INF
    z[8, ::K // 20] = 0.25
    z[11] = 0.0                             # equal tokens: the border lies far on
    z[12] = 0.0
    p = {"uniform": np.float32([0.5, 0.5, 0.5, 0.7, 0.5, 0.25, 0.999, 0.5, 0.9, 0.5, 0.5, 0.95, 0.95, 0.6, 0.999, 0.0]),
         "temperature": np.float32([1, 1, 1, 1, 1, 1, 1, 1, 1, 0.0, INF, 1, 1, 1, 1, 1]),
         "top_k": np.int32([0, 0, 0, 0, 3, 0, 0, 50, 40, 0, 0, 0, 90000, 5000, 600, K]),
         "top_p": np.float32([0.9, 1, 0.9, 0.9, 0.9, 0.5, 0.5, 0.5, 1, 0.5, 0.3, 0.8, 1, 0.9, 1, 1]),
         "min_p": np.float32([0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 1e-3, 0])}
    for rows in (slice(0, 16), slice(0, 5), slice(5, 8), slice(8, 16), slice(13, 14)):
        check(z[rows].clone(), {k: v[rows] for k, v in p.items()})


def test_row_starts_off_16_bytes():
    """An odd row length in 16-bit types: rows start at every place of 16 bytes."""
    for t in (torch.bfloat16, torch.float16):
        check(logits(17, 1031, t, 12), params(17, 13, FILTERS[-1]))


@pytest.mark.parametrize("N,K", [(9, 2050), (4, 70001)])
def test_captured_and_on_two_streams(N, K):
    z, z2 = logits(N, K, torch.bfloat16, 14), logits(N, K, torch.bfloat16, 15)
    p, p2 = params(N, 16, FILTERS[-1]), params(N, 17, FILTERS[-1])
    d, d2 = {k: device(v) for k, v in p.items()}, {k: device(v) for k, v in p2.items()}
    token, token2 = guarded((N,), torch.int32, fill=0), guarded((N,), torch.int32, fill=0)
    ws, ws2 = (workspace(B.sample_tokens_workspace_bytes(N, K)) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.sample_tokens(N, K, z, token=token, ws=ws, **d)
    side = torch.cuda.Stream()
    for seed in (20, 21):
        fresh = logits(N, K, torch.bfloat16, seed)
        z.copy_(fresh)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            B.sample_tokens(N, K, z2, token=token2, ws=ws2, **d2)
        torch.cuda.synchronize()
        assert (token.cpu().numpy() == run(z, p)[0]).all() and (token2.cpu().numpy() == run(z2, p2)[0]).all()


def test_more_than_2_to_31_logits():
    N, K = 16385, 131101
    z = torch.empty(N, K, dtype=torch.bfloat16, device="cuda").normal_(0, 2, generator=torch.Generator(device="cuda").manual_seed(4))
    token, u = guarded((N,), torch.int32, fill=0), torch.full((N,), 0.5, device="cuda")
    top_p = torch.full((N,), 0.8, device="cuda")
    B.sample_tokens(N, K, z, u, token, top_p=top_p, ws=workspace(B.sample_tokens_workspace_bytes(N, K)))
    for n in (0, 2 ** 31 // K - 1, 2 ** 31 // K, N - 1):
        assert int(token[n]) == pick(z[n].double().cpu().numpy(), 0.5, top_p=float(np.float32(0.8)))[0]


@pytest.mark.parametrize("t,T", [(torch.float32, 1.0), (torch.float32, 0.5), (torch.float32, 3.0), (torch.float16, 1.0)])
@pytest.mark.parametrize("N,K", [(1, 4000), (300, 4000), (1, 40000)])
@pytest.mark.parametrize("k", [257, 600, 2500])
def test_top_k_among_the_least_weights(k, N, K, t, T):
    """A weight of 45 ln 2 = 31.19 temperatures below the largest still rounds to 2^-44: top-k counts such tokens like all others."""
    z = guarded((N, K), t, fill=-40.0 * T)
    z[:, 2:3000] = -31.05 * T
    z[:, 0] = -31.15 * T                    # of rank 3000, in front of all others
    z[:, 1] = 0.0
    check(z, {"uniform": np.zeros(N, dtype=np.float32), "top_k": np.full(N, k, dtype=np.int32), "temperature": np.full(N, T, dtype=np.float32)})


def pick_held(z, u, temperature, top_k, top_p, min_p):
    """pick with the weights as they are held, whole multiples of 2^-44 of the largest (K <= 2^18): at a random number of 0 it matters which tokens
    weigh nothing."""
    z = np.asarray(z, dtype=np.float64) + 0.0
    if temperature <= 0 or top_k == 1:
        return int(np.argmax(z)), 0.0
    d = (z - z.max()) / temperature
    order = np.argsort(-z, kind="stable")
    keep = np.ones(len(z), dtype=bool)
    if 0 < top_k <= len(z):
        keep[top_k:] = False
    held = np.rint(np.exp(d) * 2.0 ** 44).astype(np.int64)           # (131072 of them sum to 2^61 at most)
    w = held[order] * keep
    if top_p < 1:
        keep &= np.cumsum(w) - w < top_p * float(w.sum())
    if min_p > 0:
        keep &= np.exp(d[order]) >= min_p
    ids = np.sort(order[keep])
    c = np.cumsum(held[ids])
    at = int(np.argmax(c > u * float(c[-1])))
    return int(ids[at]), float(d[ids[at]] - math.log(float(c[-1]) * 2.0 ** -44))


LONG_K = [0, 50, 256, 257, 5000, 20000]


def long_rows(N, K, t, seed):
    """Rows of all kinds, and settings of all kinds that come together with each of them."""
    z = guarded((N, K), t, fill=0)
    kinds = ["normal", "steps", "equal", "masked", "peaks", "zeros"]
    for i, kind in enumerate(kinds):
        rows = torch.arange(i, N, len(kinds), device="cuda")
        z[rows] = logits(len(rows), K, t, seed + i, kind)
    r = np.random.default_rng(seed)
    p = {"uniform": r.random(N, dtype=np.float32), "temperature": r.choice([0.0, 0.4, 1.0, 1.0, 1.0, 2.5, 30.0], N).astype(np.float32),
         "top_k": np.asarray(r.choice(LONG_K, N), dtype=np.int32), "top_p": np.where(r.random(N) < 0.5, r.uniform(0.05, 0.999, N), 1.0).astype(np.float32),
         "min_p": np.where(r.random(N) < 0.4, 10 ** r.uniform(-4, -0.01, N), 0.0).astype(np.float32)}
    p["uniform"][::7] = 0.0
    return z, p


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,K", [(160, 33000), (320, 33001), (160, 131075), (320, 131072)])
def test_long_rows_and_many(N, K, t):
    """More rows than SMs: blocks of 512 threads, with the rows in their order (160) or with the costly ones first (320)."""
    z, p = long_rows(N, K, t, N + K)
    token, logprob = run(z, p)
    for n in np.random.default_rng(1).permutation(N)[:96 if K < 100000 else 40]:
        args = {k: (int(v[n]) if v.dtype == np.int32 else float(v[n])) for k, v in p.items() if k != "uniform"}
        want, l = pick_held(z[n].double().cpu().numpy(), float(p["uniform"][n]), **args)
        assert token[n] == want, (n, token[n], want, args, p["uniform"][n])
        assert logprob[n] == l or abs(logprob[n] - l) <= abs(l) * 2.0 ** -24 + 6e-14 * K + 1e-12
    # a row's answer is its own: the same alone, where one block or a cluster of 1024 threads each has it
    for n in range(0, N, 23):
        one = run(z[n:n + 1].clone(), {k: v[n:n + 1] for k, v in p.items()})
        assert one[0][0] == token[n] and (one[1][0] == logprob[n])


@pytest.mark.parametrize("N,K", [(297, 9503), (297, 9504), (400, 12799), (400, 12800)])
def test_either_side_of_the_ordering(N, K):
    """From 32 tokens for each row on the costly rows come first."""
    check(logits(N, K, torch.bfloat16, 21, "steps"), params(N, 22, FILTERS[-1]))


def test_settings_of_many_short_rows_cost_little():
    """A temperature for each row of 8192 short ones: not much more than none (it was more than twice the time while blocks looked at all rows')."""
    N, K = 8192, 1000
    z, u, one = logits(N, K, torch.bfloat16, 23), torch.rand(N, device="cuda"), torch.ones(N, device="cuda")
    token = guarded((N,), torch.int32, fill=0)
    times = {}
    for name, temperature in (("none", None), ("each", one)) * 12:
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(4):
            B.sample_tokens(N, K, z, u, token, temperature=temperature)
        b.record()
        torch.cuda.synchronize()
        times.setdefault(name, []).append(a.elapsed_time(b))
    assert sorted(times["each"])[6] < 1.5 * sorted(times["none"])[6]
