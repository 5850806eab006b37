"""Cases of what a deep token network needs between its ends: normalisation of a residual stream, products of 8-bit operands behind it, the
gradient's global norm with clipping, and the choice of a token from the output layer's logits.

  norm       h = x + residual;  y = h / sqrt(mean(h^2) + eps) * w          (mean over the row, of the sum before it is rounded)
  norm_q8    the same, y as e4m3 values with one scale for each row: scale = max|y| / 448
  norm_grad  from h, 1 / sqrt(mean(h^2) + eps) and the gradients of y and h: the gradient of x (and of the residual) and of w
  fc_q8      y = act(x_scale[n] w_scale[k] sum_c x[n,c] w[k,c] + bias[k]),  x and w e4m3
  norm2      the norm of many tensors as one vector
  clip       the same, and every tensor times min(1, max_norm / (norm + 1e-6))
  sgd        the same, and w -= lr * min(1, max_norm / (norm + 1e-6)) * dw
  sample     one token of each row: p ~ exp(z / temperature); of the top_k largest, those in front of which less than top_p of their mass lies, and of
             them those of at least min_p times the largest probability; among these, in the order of their ids, the first whose
             cumulated mass exceeds uniform[n] times the total; at temperature 0 the largest

Every case is a dict of plain values; sizes come from the repository's VGG-A and DNN layers, or are generic.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
E4M3 = torch.float8_e4m3fn
TINY = 2.0 ** -126      # least scale of a row of 8-bit values
EPS = 1e-6
LR, MAX_NORM = 0.01, 1.0
DNN_DIMS = [440, 2048, 2048, 2048, 2048, 2048, 8192]
VGGA_CONVS = [(3, 64), (64, 128), (128, 256), (256, 256), (256, 512), (512, 512), (512, 512), (512, 512)]
VGGA_FCS = [(25088, 4096), (4096, 4096), (4096, 1000)]


def listed():
    return [
        # one token of generation: the smallest call, latency only
        {"name": "norm 1 row", "op": "norm", "type": "bf16", "N": 1, "C": 2048, "residual": True},
        # the tokens of a large training batch
        {"name": "norm batch", "op": "norm", "type": "bf16", "N": 32768, "C": 4096, "residual": True},
        # input of an 8-bit layer, sizes that divide nothing
        {"name": "norm q8 odd", "op": "norm_q8", "type": "fp16", "N": 3001, "C": 1037, "residual": True},
        # fp32 training without a residual stream, sizes that divide nothing
        {"name": "norm grad fp32 odd", "op": "norm_grad", "type": "fp32", "N": 5000, "C": 1001, "residual": False},
        # the gradient of the large batch
        {"name": "norm grad batch", "op": "norm_grad", "type": "bf16", "N": 32768, "C": 4096, "residual": True},
        # generation for a few sequences at once: the weights are what is read
        {"name": "fc q8 16 rows", "op": "fc_q8", "type": "bf16", "N": 16, "C": 4096, "K": 16384, "bias": False, "act": "none"},
        # a large batch: the most operations
        {"name": "fc q8 batch", "op": "fc_q8", "type": "bf16", "N": 8192, "C": 4096, "K": 16384, "bias": True, "act": "relu"},
        # the gradients of the DNN, kept beside their clipped form
        {"name": "clip dnn", "op": "clip", "type": "fp32", "set": "dnn", "flat": False},
        # the clipped step of VGG-A, parameters and gradients in flat buffers
        {"name": "sgd vgga", "op": "sgd", "type": "fp32", "set": "vgga", "flat": True},
        # the gradients of a large network of matrices and vectors: the most bytes
        {"name": "clip 500M", "op": "clip", "type": "bf16", "set": "mixed", "count": 60, "total": 500_000_000, "flat": False},
        # the answer of one sequence
        {"name": "sample 1 row", "op": "sample", "type": "fp32", "N": 1, "K": 32003, "filters": "mixed", "masked": False},
        # the answers of many sequences, each with its own settings
        {"name": "sample batch", "op": "sample", "type": "bf16", "N": 512, "K": 131072, "filters": "mixed", "masked": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_q8", "norm_grad", "norm_grad", "fc_q8", "fc_q8", "norm2", "clip", "sgd", "sample", "sample"])
    t = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op.startswith("norm") and op != "norm2":
        case = {"op": op, "type": t, "N": _log(rng, 1, 32768), "C": _log(rng, 32, 16384), "residual": rng.random() < 0.7}
        if case["N"] * case["C"] * (2 if t == "fp32" else 1) > 32768 * 4096:
            case["N"] = max(1, 32768 * 2048 // case["C"])
        if rng.random() < 0.7:  # most models have sizes that are multiples of eight
            case["C"] = max(32, case["C"] // 8 * 8)
        return case
    if op == "fc_q8":
        case = {"op": op, "type": rng.choice(["bf16", "fp16"]), "N": _log(rng, 1, 8192), "C": _log(rng, 64, 4096), "K": _log(rng, 64, 16384),
                "bias": rng.random() < 0.5, "act": rng.choice(["none", "none", "relu", "sigmoid"])}
        if rng.random() < 0.7:
            case["C"] = max(64, case["C"] // 16 * 16)
        return case
    if op == "sample":
        return {"op": op, "type": t, "N": _log(rng, 1, 256), "K": _log(rng, 100, 131072),
                "filters": rng.choice(["none", "top_k", "top_p", "min_p", "mixed", "mixed"]), "masked": rng.random() < 0.5}
    return {"op": op, "type": t, "set": "mixed", "count": rng.randint(1, 60), "total": _log(rng, 10_000, 130_000_000),
            "flat": rng.random() < 0.5}


# ---------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, std, dtype=torch.float32):
    return (torch.empty(shape, device="cuda").normal_(0.0, 1.0, generator=g) * std).to(dtype)


def _uniform(g, shape, lo, hi):
    return torch.empty(shape, device="cuda").uniform_(0.0, 1.0, generator=g) * (hi - lo) + lo


def _sizes(case):
    if case["set"] == "dnn":
        return [n for c, k in zip(DNN_DIMS[:-1], DNN_DIMS[1:]) for n in (c * k, k)]
    if case["set"] == "vgga":
        return [n for c, k in VGGA_CONVS for n in (9 * c * k, k)] + [n for c, k in VGGA_FCS for n in (c * k, k)]
    # matrices of sizes between one and three, and a short vector behind each
    count, total = case["count"], case["total"]
    share = [(1.0 + (7 * i % 5) / 2.0) if i % 2 == 0 else 0.0 for i in range(count)]
    return [max(1, int(total * s / sum(share))) if s else min(total, 33 + 97 * i) for i, s in enumerate(share)]


def _tensors(g, sizes, std, dtype, flat):
    """Tensors of these sizes: of their own, or views that follow one another in one buffer."""
    if not flat:
        return [_normal(g, (n,), std, dtype) for n in sizes]
    return list(torch.split(_normal(g, (sum(sizes),), std, dtype), sizes))


def _quantized(g, rows, cols):
    """Rows as norm_q8 leaves them: e4m3 values up to 448, and scales."""
    v = _normal(g, (rows, cols), 1.0)
    top = v.abs().amax(dim=1, keepdim=True)
    return (v * (448.0 / top)).to(E4M3), (top.squeeze(1) / 448.0).contiguous()


def _inputs(case, seed):
    g, t, op = _gen(seed), TYPES[case["type"]], case["op"]
    s = {"case": case, "op": op}
    if op in ("norm", "norm_q8", "norm_grad"):
        N, C = case["N"], case["C"]
        s["w"] = (1.0 + _normal(g, (C,), 0.2)).to(t)
        if op == "norm_grad":
            s["h"] = (_normal(g, (N, C), 1.0) * _uniform(g, (N, 1), 0.3, 3.0)).to(t)
            s["rstd"] = torch.rsqrt(s["h"].double().square().mean(dim=1) + EPS).float()
            s["dy"] = _normal(g, (N, C), 1e-2, t)
            s["dh"] = _normal(g, (N, C), 1e-2, t) if case["residual"] else None
            s["dx"], s["dw"] = torch.empty(N, C, dtype=t, device="cuda"), torch.empty(C, dtype=t, device="cuda")
        else:
            s["x"] = _normal(g, (N, C), 0.5, t)
            s["residual"] = (_normal(g, (N, C), 1.0) * _uniform(g, (N, 1), 0.3, 3.0)).to(t) if case["residual"] else None
            s["h"] = torch.empty(N, C, dtype=t, device="cuda") if case["residual"] else None
            s["y"] = torch.empty(N, C, dtype=E4M3 if op == "norm_q8" else t, device="cuda")
            s["scale"] = torch.empty(N, device="cuda") if op == "norm_q8" else None
            s["rstd"] = torch.empty(N, device="cuda")
    elif op == "fc_q8":
        N, C, K = case["N"], case["C"], case["K"]
        s["x"], s["x_scale"] = _quantized(g, N, C)
        s["w"], scale = _quantized(g, K, C)
        s["w_scale"] = scale / math.sqrt(C)
        s["bias"] = _normal(g, (K,), 0.5, t) if case["bias"] else None
        s["y"] = torch.empty(N, K, dtype=t, device="cuda")
    elif op == "sample":
        N, K, f = case["N"], case["K"], case["filters"]
        # logits whose largest fall about as the logarithm of their rank, flat and steep rows, and noise
        spread = _uniform(g, (N, 1), 0.8, 2.0)
        z = -_uniform(g, (N, K), 0.0, 1.0).clamp_(min=1e-7).log_() * spread + _normal(g, (N, K), 0.5)
        if case["masked"]:  # tokens that a grammar or a blocklist rules out
            z.masked_fill_(_uniform(g, (N, K), 0.0, 1.0) < _uniform(g, (N, 1), 0.0, 0.9), -math.inf)
            z[:, K // 2] = 0.0
        s["logits"] = z.to(t)
        s["uniform"] = torch.rand(N, device="cuda", generator=g)
        temperature = _uniform(g, (N,), 0.5, 1.3)
        s["temperature"] = torch.where(_uniform(g, (N,), 0.0, 1.0) < 0.1, torch.zeros_like(temperature), temperature) if f == "mixed" else temperature
        which = torch.randint(0, 4, (N,), device="cuda", generator=g)  # mixed: a quarter of the rows each without, with one of the first two, with all
        s["top_k"] = s["top_p"] = s["min_p"] = None
        if f in ("top_k", "mixed"):
            k = torch.randint(1, 101, (N,), device="cuda", generator=g).int()
            s["top_k"] = torch.where((which == 1) | (which == 3), k, torch.zeros_like(k)) if f == "mixed" else k
        if f in ("top_p", "mixed"):
            p = _uniform(g, (N,), 0.7, 0.99)
            s["top_p"] = torch.where(which >= 2, p, torch.ones_like(p)) if f == "mixed" else p
        if f in ("min_p", "mixed"):
            p = _uniform(g, (N,), 0.01, 0.1)
            s["min_p"] = torch.where(which == 3, p, torch.zeros_like(p)) if f == "mixed" else p
        s["token"] = torch.empty(N, dtype=torch.int32, device="cuda")
        s["logprob"] = torch.empty(N, device="cuda")
    else:
        sizes = _sizes(case)
        s["grads"] = _tensors(g, sizes, 2e-3, t, case["flat"])
        s["norm"] = torch.empty(1, device="cuda")
        if op == "clip":
            s["out"] = [torch.empty_like(x) for x in s["grads"]]
        if op == "sgd":
            s["params"] = _tensors(g, sizes, 0.05, t, case["flat"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_1602_06709_b200 import binding as B
        op, c = s["op"], case
        need = 0
        if op == "norm_grad":
            need = B.rms_norm_workspace_bytes(c["N"], c["C"])
        elif op == "fc_q8":
            need = B.fc_q8_workspace_bytes(c["N"], c["C"], c["K"])
        elif op == "sample":
            need = B.sample_tokens_workspace_bytes(c["N"], c["K"])
        elif "grads" in s:
            # a program's lists of its parameters and gradients, which it makes once
            s["grad_list"] = B.TensorList(s["grads"])
            s["out_list"] = B.TensorList(s["out"]) if op == "clip" else None
            s["param_list"] = B.TensorList(s["params"]) if op == "sgd" else None
            need = B.grad_norm_workspace_bytes(s["grad_list"])
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_1602_06709_b200 import binding as B
    c, op = s["case"], s["op"]
    if op == "norm":
        B.rms_norm_fwd(c["N"], c["C"], s["x"], s["residual"], s["w"], EPS, s["h"], s["y"], s["rstd"])
        return _some(h=s["h"], y=s["y"], rstd=s["rstd"])
    if op == "norm_q8":
        B.rms_norm_fwd_q8(c["N"], c["C"], s["x"], s["residual"], s["w"], EPS, s["h"], s["y"], s["scale"], s["rstd"])
        return _some(h=s["h"], y=s["y"], scale=s["scale"], rstd=s["rstd"])
    if op == "norm_grad":
        B.rms_norm_bwd(c["N"], c["C"], s["h"], s["w"], s["rstd"], s["dy"], s["dh"], s["dx"], s["dw"], ws=s["ws"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if op == "fc_q8":
        act = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "sigmoid": B.ACT_SIGMOID}[c["act"]]
        B.fc_q8_fwd(c["N"], c["C"], c["K"], s["x"], s["x_scale"], s["w"], s["w_scale"], s["bias"], s["y"], act, ws=s["ws"])
        return s["y"]
    if op == "sample":
        B.sample_tokens(c["N"], c["K"], s["logits"], s["uniform"], s["token"], temperature=s["temperature"], top_k=s["top_k"],
                        top_p=s["top_p"], min_p=s["min_p"], logprob=s["logprob"], ws=s["ws"])
        return {"token": s["token"], "logprob": s["logprob"]}
    if op == "norm2":
        B.grad_norm(s["grad_list"], s["norm"], ws=s["ws"])
        return s["norm"]
    if op == "clip":
        B.grad_clip(s["grad_list"], s["out_list"], MAX_NORM, s["norm"], ws=s["ws"])
        return {"norm": s["norm"], "out": s["out"]}
    B.sgd_update_clipped(s["param_list"], s["grad_list"], LR, MAX_NORM, s["norm"], ws=s["ws"])
    return {"norm": s["norm"], "params": s["params"]}


def _some(**outputs):
    return {k: v for k, v in outputs.items() if v is not None}


def _run_plain(s):
    c, op = s["case"], s["op"]
    t = TYPES[c["type"]]
    if op in ("norm", "norm_q8"):
        h = s["x"].float()
        if s["residual"] is not None:
            h = h + s["residual"].float()
        rstd = 1.0 / (h.square().mean(dim=1) + EPS).sqrt()
        y = h * rstd.unsqueeze(1) * s["w"].float()
        out = _some(h=h.to(t) if s["residual"] is not None else None, rstd=rstd)
        if op == "norm":
            return {**out, "y": y.to(t)}
        scale = (y.abs().amax(dim=1) / 448.0).clamp(min=TINY)
        return {**out, "y": (y / scale.unsqueeze(1)).to(E4M3), "scale": scale}
    if op == "norm_grad":
        h, dy, rstd = s["h"].float(), s["dy"].float(), s["rstd"].unsqueeze(1)
        normed, g = h * rstd, dy * s["w"].float()
        dx = rstd * (g - normed * (g * normed).mean(dim=1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(t), "dw": (dy * normed).sum(dim=0).to(t)}
    if op == "fc_q8":
        y = torch.matmul(s["x"].float(), s["w"].float().t()) * s["x_scale"].unsqueeze(1) * s["w_scale"]
        if s["bias"] is not None:
            y = y + s["bias"].float()
        y = y.clamp(min=0.0) if c["act"] == "relu" else 1.0 / (1.0 + torch.exp(-y)) if c["act"] == "sigmoid" else y
        return y.to(t)
    if op == "sample":
        return _plain_sample(s)
    norm = torch.stack([x.float().square().sum() for x in s["grads"]]).sum().sqrt().reshape(1)
    if op == "norm2":
        return norm
    factor = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
    if op == "clip":
        return {"norm": norm, "out": [(x.float() * factor).to(t) for x in s["grads"]]}
    return {"norm": norm, "params": [w.copy_(w.float() - LR * (factor * x.float())) for w, x in zip(s["params"], s["grads"])]}


def _plain_sample(s):
    N, K = s["case"]["N"], s["case"]["K"]
    z = s["logits"].double()
    temperature = s["temperature"].double().unsqueeze(1)
    greedy = temperature <= 0.0
    weight = torch.exp((z - z.amax(dim=1, keepdim=True)) / torch.where(greedy, 1.0, temperature))
    order = torch.sort(z, dim=1, descending=True, stable=True).indices  # ties: the lowest id first
    w = weight.gather(1, order)
    rank = torch.arange(K, device="cuda").unsqueeze(0)
    keep = torch.ones(N, K, dtype=torch.bool, device="cuda")
    if s["top_k"] is not None:
        k = s["top_k"].long().unsqueeze(1)
        keep = torch.where(k > 0, rank < k, keep)
    keep = torch.where(greedy, rank < 1, keep)
    w = w * keep
    if s["top_p"] is not None:
        p = s["top_p"].double().unsqueeze(1)
        before = w.cumsum(dim=1)
        total = before[:, -1:]
        keep = keep & ((before - w < p * total) | (p >= 1.0))
    if s["min_p"] is not None:
        keep = keep & (w >= s["min_p"].double().unsqueeze(1))
    keep = torch.zeros_like(keep).scatter_(1, order, keep)
    weight = weight * keep
    mass = weight.cumsum(dim=1)
    total = mass[:, -1:]
    token = (mass <= s["uniform"].double().unsqueeze(1) * total).sum(dim=1).clamp(max=K - 1)
    return {"token": token.int(), "logprob": (weight.gather(1, token.unsqueeze(1)) / total).log().squeeze(1).float()}


# ---------------------------------------------------------------------------------------------------- work
def work(case):
    op, e = case["op"], 4 if case["type"] == "fp32" else 2
    if op in ("norm", "norm_q8"):
        N, C, r = case["N"], case["C"], case["residual"]
        return {"bytes": N * C * (e * (3 if r else 1) + (1 if op == "norm_q8" else e)) + e * C + 8 * N, "flops": 6 * N * C}
    if op == "norm_grad":
        N, C = case["N"], case["C"]
        return {"bytes": N * C * e * (4 if case["residual"] else 3) + 2 * e * C + 4 * N, "flops": 10 * N * C}
    if op == "fc_q8":
        N, C, K = case["N"], case["C"], case["K"]
        return {"bytes": (N + K) * (C + 4) + e * N * K, "flops": 2 * N * C * K}
    if op == "sample":
        return {"bytes": case["N"] * (e * case["K"] + 28), "flops": 4 * case["N"] * case["K"]}
    n = sum(_sizes(case))
    return {"bytes": n * e * {"norm2": 1, "clip": 2, "sgd": 3}[op] + 4, "flops": n * {"norm2": 2, "clip": 3, "sgd": 4}[op]}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op in ("norm", "norm_q8"):
        h = s["x"].double()
        h = h if s["residual"] is None else h + s["residual"].double()
        mean = torch.linalg.vector_norm(h, dim=1).square() / h.shape[1]
        rstd = (mean + EPS) ** -0.5
        y = torch.einsum("nc,n,c->nc", h, rstd, s["w"].double())
        out = _some(h=None if s["residual"] is None else h, rstd=rstd)
        if op == "norm":
            return {**out, "y": y}
        scale = torch.linalg.vector_norm(y, ord=math.inf, dim=1) / 448.0
        return {**out, "y": y / scale[:, None], "scale": scale}
    if op == "norm_grad":
        h, dy, r, w = s["h"].double(), s["dy"].double(), s["rstd"].double(), s["w"].double()
        inner = torch.einsum("nc,nc,c->n", dy, h, w) * r ** 3 / h.shape[1]
        dx = torch.einsum("nc,n,c->nc", dy, r, w) - h * inner[:, None]
        return {"dx": dx if s["dh"] is None else dx + s["dh"].double(), "dw": torch.einsum("nc,nc,n->c", dy, h, r)}
    if op == "fc_q8":
        y = (s["x"].double() * s["x_scale"].double()[:, None]) @ (s["w"].double() * s["w_scale"].double()[:, None]).mT
        y = y if s["bias"] is None else y + s["bias"].double()
        return {"none": lambda v: v, "relu": torch.relu, "sigmoid": torch.sigmoid}[case["act"]](y)
    if op == "sample":
        picks = [_exact_sample(s, n) for n in range(case["N"])]
        return {"token": torch.tensor([p[0] for p in picks], dtype=torch.int32, device="cuda"),
                "logprob": torch.tensor([p[1] for p in picks], dtype=torch.float64, device="cuda")}
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(x.double())) ** 2 for x in s["grads"]))
    factor = min(1.0, MAX_NORM / (norm + 1e-6))
    found = torch.tensor([norm], dtype=torch.float64, device="cuda")
    if op == "norm2":
        return found
    if op == "clip":
        return {"norm": found, "out": [x.double() * factor for x in s["grads"]]}
    return {"norm": found, "params": [w.double() - LR * factor * x.double() for w, x in zip(s["params"], s["grads"])]}


def _exact_sample(s, n):
    """(token, logarithm of the probability it was chosen with) of one row, from its sorted values."""
    z, heat = s["logits"][n].double(), float(s["temperature"][n])
    if heat <= 0.0:
        return int((z == z.max()).nonzero()[0]), 0.0
    at = torch.argsort(-z, stable=True)
    at = at[z[at] > -math.inf]
    if s["top_k"] is not None and int(s["top_k"][n]) > 0:
        at = at[:int(s["top_k"][n])]
    p = torch.softmax(z[at] / heat, dim=0)
    if s["top_p"] is not None and float(s["top_p"][n]) < 1.0:
        reached = torch.searchsorted(p.cumsum(0), s["top_p"][n].double())
        at, p = at[:int(reached) + 1], p[:int(reached) + 1]
    if s["min_p"] is not None:
        m = p >= float(s["min_p"][n]) * p[0]
        at, p = at[m], p[m]
    at, back = torch.sort(at)
    p = p[back] / p.sum()
    i = min(int(torch.searchsorted(p.cumsum(0), s["uniform"][n].double(), right=True)), len(at) - 1)
    return int(at[i]), math.log(float(p[i]))
