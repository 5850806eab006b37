"""Cases of the vocabulary-sized ends of a network's training step and of its orthogonalised weight update.

  embed_fwd    out[n] = scale * table[ids[n]]                       (rows of the padding id are zero)
  embed_bwd    dtable[v] = scale * sum over n with ids[n] = v of dy[n]
  embed_sgd    table[v] -= lr * dtable[v] for the rows that occur, in place
  loss         softmax cross-entropy of z = x w^T + b without keeping z: mean loss, loss of each row, log-sum-exp of each row
  loss_grad    the same, then dx, dw (and db), from the log-sum-exp
  direction    five Newton-Schulz steps on g / |g|
  update       momentum, direction and weight update of a matrix, in place

Every case is a dict of plain values; sizes come from the repository's VGG-A classifier and DNN layers, or are generic.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
PAD = 0                 # padding id of the embedding cases that have one
IGNORE = -1             # label of rows that take no part in the loss
LOSS_SCALE = 65536.0    # fp16 gradients are taken of the scaled loss, given as the gradient of each row's loss
SCALE = 1.5
LR, DECAY, MU = 0.02, 0.01, 0.95
NS_A, NS_B, NS_C, EPS = 3.4445, -4.7750, 2.0315, 1e-7


def listed():
    return [
        # one step of generation for a handful of sequences: the smallest call, latency only
        {"name": "embed 16 tokens", "op": "embed_fwd", "type": "bf16", "N": 16, "V": 8192, "C": 2048, "pad": False},
        # the tokens of a large training batch
        {"name": "embed batch", "op": "embed_fwd", "type": "bf16", "N": 32768, "V": 131072, "C": 4096, "pad": False},
        # a medium table in fp32 with padded sequences, sizes that divide nothing
        {"name": "embed grad fp32 odd", "op": "embed_bwd", "type": "fp32", "N": 5000, "V": 10007, "C": 1001, "pad": True},
        # the gradient of the large batch: most table rows do not occur and are zero
        {"name": "embed grad batch", "op": "embed_bwd", "type": "bf16", "N": 32768, "V": 131072, "C": 4096, "pad": False},
        # gradient and SGD step in one call: only the rows that occur are touched
        {"name": "embed sgd", "op": "embed_sgd", "type": "fp16", "N": 16384, "V": 65536, "C": 2048, "pad": True},
        # VGG-A's classifier at minibatch 256, evaluation only: the smallest loss
        {"name": "loss classifier", "op": "loss", "type": "fp16", "N": 256, "C": 4096, "K": 1000, "bias": True, "ignored": False},
        # the DNN's output layer: 2048 -> 8192 at 1024 frames, with gradients
        {"name": "loss grad dnn", "op": "loss_grad", "type": "bf16", "N": 1024, "C": 2048, "K": 8192, "bias": True, "ignored": False},
        # ragged rows and vocabulary, part of the rows masked
        {"name": "loss grad ragged", "op": "loss_grad", "type": "fp16", "N": 3001, "C": 1032, "K": 50021, "bias": False, "ignored": True},
        # a large vocabulary at a large batch: the largest case
        {"name": "loss grad large", "op": "loss_grad", "type": "bf16", "N": 8192, "C": 4096, "K": 131072, "bias": False, "ignored": False},
        # the small matrices of several layers in one call
        {"name": "direction 8 small", "op": "direction", "type": "bf16", "count": 8, "M": 256, "N": 512},
        # a hidden layer of the DNN
        {"name": "update 2048", "op": "update", "type": "bf16", "count": 1, "M": 2048, "N": 2048},
        # a tall matrix whose sizes divide nothing
        {"name": "update tall", "op": "update", "type": "bf16", "count": 1, "M": 8200, "N": 4100},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "embed_sgd", "loss", "loss_grad", "loss_grad", "direction", "update", "update"])
    if op.startswith("embed"):
        return {"op": op, "type": rng.choice(["bf16", "fp16", "fp32"]), "N": _log(rng, 1, 32768), "V": _log(rng, 100, 131072),
                "C": _log(rng, 32, 2048), "pad": rng.random() < 0.5}
    if op.startswith("loss"):
        case = {"op": op, "type": rng.choice(["bf16", "fp16"]), "N": _log(rng, 1, 8192), "C": _log(rng, 64, 4096),
                "K": _log(rng, 100, 131072), "bias": rng.random() < 0.5, "ignored": rng.random() < 0.5}
        if rng.random() < 0.7:  # most models have sizes that are multiples of eight
            case["C"] = max(64, case["C"] // 8 * 8)
        return case
    M, N, count = _log(rng, 16, 4096), _log(rng, 16, 4096), rng.choice([1, 1, 2, 3, 6])
    if count * M * N > 4096 * 4096:
        count = 1
    return {"op": op, "type": "bf16", "count": count, "M": M, "N": N}


# ---------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, std, dtype=torch.float32):
    return (torch.empty(shape, device="cuda").normal_(0.0, 1.0, generator=g) * std).to(dtype)


def _tokens(g, n, v):
    """Token ids whose frequency falls as one over their rank, as that of words does."""
    u = torch.rand(n, device="cuda", dtype=torch.float64, generator=g)
    return (torch.exp(u * math.log(v)) - 1.0).long().clamp_(0, v - 1).int()


def _inputs(case, seed):
    g, t, op = _gen(seed), TYPES[case["type"]], case["op"]
    s = {"case": case, "op": op}
    if op.startswith("embed"):
        N, V, C = case["N"], case["V"], case["C"]
        s["ids"] = _tokens(g, N, V)
        s["pad"] = PAD if case["pad"] else None
        if op == "embed_fwd":
            s["table"] = _normal(g, (V, C), 0.02, t)
            s["out"] = torch.empty(N, C, dtype=t, device="cuda")
        elif op == "embed_bwd":
            s["dy"] = _normal(g, (N, C), 1e-3, t)
            s["dtable"] = torch.empty(V, C, dtype=t, device="cuda")
        else:
            s["table"] = _normal(g, (V, C), 0.02, t)
            s["dy"] = _normal(g, (N, C), 1e-3, t)
    elif op.startswith("loss"):
        N, C, K = case["N"], case["C"], case["K"]
        s["x"] = _normal(g, (N, C), 1.0, t)
        s["w"] = _normal(g, (K, C), 1.5 / math.sqrt(C), t)
        s["bias"] = _normal(g, (K,), 0.5, t) if case["bias"] else None
        labels = _tokens(g, N, K)
        if case["ignored"]:
            labels = torch.where(torch.rand(N, device="cuda", generator=g) < 0.25, torch.full_like(labels, IGNORE), labels)
        s["labels"] = labels
        s["ignore"] = IGNORE if case["ignored"] else None
        s["loss"] = torch.empty(1, device="cuda")
        s["row_loss"], s["lse"] = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        if op == "loss_grad":
            s["dx"] = torch.empty(N, C, dtype=t, device="cuda")
            s["dw"] = torch.empty(K, C, dtype=t, device="cuda")
            s["db"] = torch.empty(K, dtype=t, device="cuda") if case["bias"] else None
            s["row_grad"] = None
            if case["type"] == "fp16":
                counted = (labels != IGNORE).sum().clamp(min=1)
                s["row_grad"] = torch.full((N,), LOSS_SCALE, device="cuda") / counted
    else:
        # a gradient of a layer: a falling spectrum from the few directions of the minibatch, and noise
        n, M, N = case["count"], case["M"], case["N"]
        r = min(32, M, N)
        fall = torch.arange(1, r + 1, device="cuda", dtype=torch.float32) ** -0.5
        grad = torch.matmul(_normal(g, (n, M, r), 1.0) * fall, _normal(g, (n, r, N), 1.0)) + _normal(g, (n, M, N), 0.5)
        s["dw"] = (grad * 1e-3).to(t)
        if op == "direction":
            s["out"] = torch.empty_like(s["dw"])
        else:
            s["w"] = _normal(g, (n, M, N), math.sqrt(2.0 / (M + N)), t)
            s["momentum"] = s["dw"].float() * 5.0 + _normal(g, (n, M, N), 1e-3)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_1602_06709_b200 import binding as B
        op, c = s["op"], case
        if op in ("embed_bwd", "embed_sgd"):
            need = B.embedding_workspace_bytes(c["N"], c["V"], c["C"])
        elif op.startswith("loss"):
            d = B.dtype_code(s["x"])
            need = B.fc_softmax_xent_workspace_bytes(c["N"], c["C"], c["K"], d, B.PASS_FWD)
            if op == "loss_grad":
                need = max(need, B.fc_softmax_xent_workspace_bytes(c["N"], c["C"], c["K"], d, B.PASS_BWD_DATA))
        elif op in ("direction", "update"):
            need = B.orthogonalize_workspace_bytes(c["count"], c["M"], c["N"])
        else:
            need = 0
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_1602_06709_b200 import binding as B
    c, op = s["case"], s["op"]
    if op == "embed_fwd":
        B.embedding_fwd(c["N"], c["V"], c["C"], s["ids"], s["table"], SCALE, s["out"], pad_id=s["pad"])
        return s["out"]
    if op == "embed_bwd":
        B.embedding_bwd(c["N"], c["V"], c["C"], s["ids"], s["dy"], SCALE, s["dtable"], pad_id=s["pad"], ws=s["ws"])
        return s["dtable"]
    if op == "embed_sgd":
        B.embedding_bwd_sgd(c["N"], c["V"], c["C"], s["ids"], s["dy"], SCALE, s["table"], LR, pad_id=s["pad"], ws=s["ws"])
        return s["table"]
    if op in ("loss", "loss_grad"):
        B.fc_softmax_xent_fwd(c["N"], c["C"], c["K"], s["x"], s["w"], s["bias"], s["labels"], s["loss"], s["row_loss"],
                              s["lse"], ignore_label=s["ignore"], ws=s["ws"])
        out = {"loss": s["loss"], "row_loss": s["row_loss"], "lse": s["lse"]}
        if op == "loss_grad":
            B.fc_softmax_xent_bwd(c["N"], c["C"], c["K"], s["x"], s["w"], s["bias"], s["labels"], s["lse"], s["row_grad"],
                                  s["dx"], s["dw"], s["db"], ignore_label=s["ignore"], ws=s["ws"])
            out.update(dx=s["dx"], dw=s["dw"])
            if s["db"] is not None:
                out["db"] = s["db"]
        return out
    if op == "direction":
        B.orthogonalize(c["count"], c["M"], c["N"], s["dw"], s["out"], ws=s["ws"])
        return s["out"]
    B.orthogonal_update(c["count"], c["M"], c["N"], s["w"], s["dw"], s["momentum"], MU, True, LR, DECAY, ws=s["ws"])
    return {"w": s["w"], "momentum": s["momentum"]}


def _plain_dtable(s):
    c = s["case"]
    ids = s["ids"].long()
    dy = s["dy"].float()
    if s["pad"] is not None:
        dy = dy * (ids != s["pad"]).unsqueeze(1)
    return torch.zeros(c["V"], c["C"], device="cuda").index_add_(0, ids, dy) * SCALE


def _plain_loss(s):
    z = torch.matmul(s["x"].float(), s["w"].float().t())
    if s["bias"] is not None:
        z = z + s["bias"].float()
    top = z.amax(dim=1, keepdim=True)
    lse = top.squeeze(1) + torch.exp(z - top).sum(dim=1).log()
    labels = s["labels"].long()
    counted = labels != IGNORE if s["ignore"] is not None else torch.ones_like(labels, dtype=torch.bool)
    at = z.gather(1, labels.clamp(min=0).unsqueeze(1)).squeeze(1)
    row = torch.where(counted, lse - at, torch.zeros_like(lse))
    n = counted.sum().clamp(min=1).float()
    return z, lse, labels, counted, row, n


def _poly(x):
    a = torch.matmul(x, x.transpose(1, 2))
    return NS_A * x + torch.matmul(NS_B * a + NS_C * torch.matmul(a, a), x)


def _plain_direction(u):
    x = u / (u.square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS)
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    x = _poly(_poly(_poly(_poly(_poly(x)))))
    return x.transpose(1, 2) if tall else x


def _run_plain(s):
    c, op = s["case"], s["op"]
    t = TYPES[c["type"]]
    if op == "embed_fwd":
        ids = s["ids"].long()
        out = s["table"][ids].float() * SCALE
        if s["pad"] is not None:
            out = out * (ids != s["pad"]).unsqueeze(1)
        return out.to(t)
    if op == "embed_bwd":
        return _plain_dtable(s).to(t)
    if op == "embed_sgd":
        s["table"].copy_(s["table"].float() - LR * _plain_dtable(s))
        return s["table"]
    if op in ("loss", "loss_grad"):
        z, lse, labels, counted, row, n = _plain_loss(s)
        out = {"loss": (row.sum() / n).reshape(1), "row_loss": row, "lse": lse}
        if op == "loss_grad":
            dz = torch.exp(z - lse.unsqueeze(1))
            del z
            at = labels.clamp(min=0).unsqueeze(1)
            dz.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
            grad = s["row_grad"] if s["row_grad"] is not None else 1.0 / n
            dz *= (counted * grad).unsqueeze(1)
            out["dx"] = torch.matmul(dz, s["w"].float()).to(t)
            out["dw"] = torch.matmul(dz.t(), s["x"].float()).to(t)
            if s["bias"] is not None:
                out["db"] = dz.sum(dim=0).to(t)
        return out
    if op == "direction":
        return _plain_direction(s["dw"].float()).to(t)
    s["momentum"].mul_(MU).add_(s["dw"].float())
    o = _plain_direction(s["dw"].float() + MU * s["momentum"])
    shape = math.sqrt(max(1.0, c["M"] / c["N"]))
    s["w"].copy_((1.0 - LR * DECAY) * s["w"].float() - LR * shape * o)
    return {"w": s["w"], "momentum": s["momentum"]}


# ---------------------------------------------------------------------------------------------------- work
def work(case):
    op, e = case["op"], 4 if case["type"] == "fp32" else 2
    if op.startswith("embed"):
        N, V, C = case["N"], case["V"], case["C"]
        rank = N / math.log(V)                         # the tokens below this rank occur once or more, about
        seen = min(N, V, int(rank * (1.0 + math.log(max(1.0, V / rank)))) + 1)
        if op == "embed_fwd":
            return {"bytes": 4 * N + e * C * (seen + N), "flops": N * C}
        if op == "embed_bwd":
            return {"bytes": 4 * N + e * C * (N + V), "flops": 2 * N * C}
        return {"bytes": 4 * N + e * C * (N + 2 * seen), "flops": 2 * N * C}
    if op.startswith("loss"):
        N, C, K = case["N"], case["C"], case["K"]
        if op == "loss":
            return {"bytes": e * C * (N + K) + 12 * N, "flops": 2 * N * C * K}
        return {"bytes": 2 * e * C * (N + K) + 12 * N, "flops": 6 * N * C * K}
    n, m, k = case["count"], min(case["M"], case["N"]), max(case["M"], case["N"])
    flops = 5 * n * (3 * m * m * k + m * m * m)        # the two symmetric products need one half of their elements
    if op == "direction":
        return {"bytes": n * m * k * 2 * e, "flops": flops}
    return {"bytes": n * m * k * (3 * e + 8), "flops": flops}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_rows(ids, dy, V, pad):
    order = torch.argsort(ids.long(), stable=True)
    rows, total = ids.long()[order], torch.zeros(V, dy.shape[1], dtype=torch.float64, device="cuda")
    total.index_put_((rows,), dy.double()[order], accumulate=True)
    if pad is not None:
        total[pad] = 0.0
    return SCALE * total


def _exact_direction(u):
    def once(m):
        m = m / (torch.linalg.vector_norm(m) + EPS)
        flip = m.shape[0] > m.shape[1]
        m = m.mT if flip else m
        for _ in range(5):
            gram = m @ m.mT
            m = NS_A * m + NS_B * (gram @ m) + NS_C * (gram @ (gram @ m))
        return m.mT if flip else m
    return torch.stack([once(m) for m in u.double()])


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "embed_fwd":
        rows = s["table"].double()[s["ids"].long()] * SCALE
        if s["pad"] is not None:
            rows[s["ids"] == s["pad"]] = 0.0
        return rows
    if op == "embed_bwd":
        return _exact_rows(s["ids"], s["dy"], case["V"], s["pad"])
    if op == "embed_sgd":
        return s["table"].double() - LR * _exact_rows(s["ids"], s["dy"], case["V"], s["pad"])
    if op in ("loss", "loss_grad"):
        x, w = s["x"].double(), s["w"].double()
        logp = x @ w.mT
        if s["bias"] is not None:
            logp += s["bias"].double()
        lse = torch.logsumexp(logp, dim=1)
        logp -= lse[:, None]
        labels = s["labels"].long()
        keep = torch.ones_like(lse)
        if s["ignore"] is not None:
            keep[labels == IGNORE] = 0.0
        n = max(1.0, float(keep.sum()))
        rows = torch.arange(len(labels), device="cuda")
        row = -logp[rows, labels.clamp(min=0)] * keep
        out = {"loss": (row.sum() / n)[None], "row_loss": row, "lse": lse}
        if op == "loss_grad":
            dz = logp.exp_()
            dz[rows, labels.clamp(min=0)] -= 1.0
            dz *= (keep / n if s["row_grad"] is None else keep * s["row_grad"].double())[:, None]
            out["dx"], out["dw"] = dz @ w, dz.mT @ x
            if s["bias"] is not None:
                out["db"] = dz.sum(0)
        return out
    if op == "direction":
        return _exact_direction(s["dw"])
    dw = s["dw"].double()
    m = MU * s["momentum"].double() + dw
    step = LR * math.sqrt(max(1.0, case["M"] / case["N"]))
    return {"w": s["w"].double() * (1.0 - LR * DECAY) - step * _exact_direction(dw + MU * m), "momentum": m}
