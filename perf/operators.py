"""The operators that stand between the products of a training step, as cases that can be timed and checked.

Layer norm (forward, and backward with the sums of the weights' gradients), activations kept in 8 bits (their round trip, a ReLU's
backward pass and the weights' gradient from what was kept) and log probabilities of given labels with entropy and the top
alternatives (forward and backward).  `run` with `own` false is each operator in elementary torch operations in 32 bits; with `own`
true it is the library's call.  Matrices are row-major; `pad` columns beside each row make its stride longer than the row.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-5
_BLOCK = 32  # columns of a row that share a step in the 8-bit form
_MOST = 1 << 28  # values of the largest matrix


def listed():
    return [
        # one hidden layer of a small social graph: the smallest call, where a launch counts
        {"name": "norm_small", "op": "norm", "n": 1024, "k": 64, "type": "f32", "pad": 0},
        # one hidden layer of a power-law graph of 2 M nodes, the largest
        {"name": "norm_large", "op": "norm", "n": 2097152, "k": 128, "type": "f32", "pad": 0},
        # training on a similarity graph: a hidden width that fills no power of two
        {"name": "norm_back_odd", "op": "norm_backward", "n": 132534, "k": 100, "type": "f32", "pad": 0},
        # wide rows in 16 bits, where the weights' gradients are long too
        {"name": "norm_back_wide", "op": "norm_backward", "n": 16384, "k": 4096, "type": "bf16", "pad": 0},
        # a citation network's bag-of-words features, kept for the first layer's gradient: the last block of a row is short
        {"name": "keep_features", "op": "keep", "n": 19717, "k": 500, "type": "f32", "pad": 0},
        # a hidden layer of a co-authorship network, activations and gradients in 16 bits: through the ReLU by what was kept
        {"name": "keep_relu", "op": "keep_relu", "n": 235868, "k": 128, "type": "bf16", "pad": 0},
        # the classification layer's weights, an odd number of classes
        {"name": "keep_weights_classes", "op": "keep_weights", "n": 132534, "k": 100, "c": 47, "type": "f32", "pad": 0},
        # a hidden layer's weights over all nodes of a large graph
        {"name": "keep_weights_large", "op": "keep_weights", "n": 2097152, "k": 128, "c": 128, "type": "f32", "pad": 0},
        # class scores of a citation network with the best class
        {"name": "scores_few", "op": "log_probs", "n": 19717, "k": 3, "type": "f32", "pad": 0, "top": 1, "masked": False},
        # scores over a vocabulary, a batch of positions
        {"name": "scores_vocabulary", "op": "log_probs", "n": 4096, "k": 32000, "type": "bf16", "pad": 0, "top": 8, "masked": False},
        # one answer over a long vocabulary, some entries ruled out: the single row of serving
        {"name": "scores_one_row", "op": "log_probs", "n": 1, "k": 128000, "type": "f32", "pad": 0, "top": 20, "masked": True},
        # the loss's gradient on a similarity graph
        {"name": "scores_back_odd", "op": "log_probs_backward", "n": 132534, "k": 47, "type": "f32", "pad": 0, "masked": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_backward", "norm_backward", "keep", "keep_relu", "keep_weights", "keep_weights", "log_probs", "log_probs", "log_probs_backward"])
    case = {"op": op, "type": rng.choice(["f32", "f32", "bf16", "f16"]), "pad": rng.choice([0, 0, 0, 1, 4, 8])}
    if op == "keep_weights":
        k, c = _log(rng, 8, 1024), _log(rng, 2, 512)
        if rng.random() < 0.6:
            k = (k + 3) // 4 * 4
        most = min(2097152, 2097152 * 128 * 128 // (k * c), _MOST // max(k, 4 * c) * 2)
        return {**case, "n": _log(rng, 1, max(1, most)), "k": k, "c": c}
    if op.startswith("log_probs"):
        k, most = _log(rng, 2, 131072), _MOST // 2
        case["masked"] = rng.random() < 0.3
        if op == "log_probs":
            case["top"] = rng.choice([0, 1, 5, 8, 20])
    else:
        k, most = _log(rng, 1, 16384), _MOST // 2
        if k > 8 and rng.random() < 0.5:
            k = (k + 7) // 8 * 8
    return {**case, "n": _log(rng, 1, max(1, min(2097152, most // (k + 8)))), "k": k}


def _matrix(n, k, pad, type):
    return torch.empty((n, k + pad), dtype=_TYPES[type], device="cuda")[:, :k]


def _gaussian(n, k, pad, type, gen, shift=0.0, scale=1.0, relu=False):
    x = torch.randn((n, k), device="cuda", generator=gen).mul_(scale).add_(shift)
    out = _matrix(n, k, pad, type)
    out.copy_(x.relu_() if relu else x)
    return out


def _keep(x):
    """The 8-bit form of a matrix of finite values: whole numbers of steps, and the steps' exponents plus 127."""
    n, k = x.shape
    blocks = -(-k // _BLOCK)
    x = x.float()
    if k % _BLOCK:
        x = torch.nn.functional.pad(x, (0, blocks * _BLOCK - k))
    x = x.reshape(n, blocks, _BLOCK)
    largest = x.abs().amax(dim=2)
    code = ((largest.view(torch.int32) >> 23) - 6).clamp_min(1)  # the exponent of the largest value, six bits below it
    up = ((254 - code) << 23).view(torch.float32)  # one over the step: a power of two, so the quotient is exact
    size = (x.abs() * up[:, :, None]).round_().clamp_(1, 127)
    whole = torch.where(x == 0, torch.zeros_like(x), torch.copysign(size, x))
    return whole.reshape(n, -1)[:, :k], code


def _values(q, code):
    """What the 8-bit form stands for, in 32 bits."""
    k = q.shape[1]
    step = (code.int() << 23).view(torch.float32)
    return q.float() * step.repeat_interleave(_BLOCK, dim=1)[:, :k]


def prepare(case, seed):
    op, n, k, type, pad = case["op"], case["n"], case["k"], case["type"], case["pad"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case, "eps": _EPS}
    if own:
        import paper_2409_02208_amd as cbm

        state["cbm"] = cbm
    f32 = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
    if op in ("norm", "norm_backward"):
        state["x"] = x = _gaussian(n, k, pad, type, gen, shift=0.5, relu=True)  # a layer's outputs after its ReLU
        state["gamma"] = 1 + 0.1 * torch.randn(k, device="cuda", generator=gen)
        state["beta"] = 0.1 * torch.randn(k, device="cuda", generator=gen)
        if op == "norm":
            state.update(y=_matrix(n, k, pad, type), mean=f32(n), rstd=f32(n))
        else:
            wide = x.float()
            state["mean"] = wide.mean(dim=1)
            state["rstd"] = (wide - state["mean"][:, None]).square_().mean(dim=1).add_(_EPS).rsqrt_()
            del wide
            state["dy"] = _gaussian(n, k, pad, type, gen, scale=0.01)
            state.update(dx=_matrix(n, k, pad, type), dgamma=f32(k), dbeta=f32(k))
            if own:
                state["workspace"] = torch.empty(cbm.cbm_layer_norm_workspace_bytes(n, k), dtype=torch.uint8, device="cuda")
    elif op == "keep":
        state["x"] = _gaussian(n, k, pad, type, gen, shift=0.5, relu=True)
        state["q"] = torch.empty((n, k), dtype=torch.int8, device="cuda")
        state["steps"] = torch.empty((n, -(-k // _BLOCK)), dtype=torch.uint8, device="cuda")
        state["back"] = _matrix(n, k, pad, type)
    elif op in ("keep_relu", "keep_weights"):
        whole, code = _keep(_gaussian(n, k, 0, "f32", gen, shift=0.5, relu=True))
        state["q"], state["steps"] = whole.to(torch.int8).contiguous(), code.to(torch.uint8)
        del whole, code
        if op == "keep_relu":
            state["dy"] = _gaussian(n, k, pad, type, gen, scale=0.01)
            state["dx"] = _matrix(n, k, pad, type)
        else:
            state["dy"] = _gaussian(n, case["c"], pad, type, gen, scale=0.01)
            state["dw"] = f32(k, case["c"])
            if own:
                state["workspace"] = torch.empty(cbm.cbm_checkpoint_workspace_bytes(n, k, case["c"]), dtype=torch.uint8, device="cuda")
    else:
        state["z"] = z = _gaussian(n, k, pad, type, gen, scale=3.0)
        state["labels"] = torch.randint(0, k, (n,), device="cuda", generator=gen)
        if case["masked"]:  # classes that are ruled out, nodes without a label
            z.masked_fill_(torch.rand((n, k), device="cuda", generator=gen) < 0.2, -math.inf)
            state["labels"][torch.rand(n, device="cuda", generator=gen) < 0.2] = -1
        if op == "log_probs":
            top = case["top"]
            state.update(logp=f32(n), entropy=f32(n), stats=f32(n, 2), values=f32(n, top), columns=torch.empty((n, top), dtype=torch.int32, device="cuda"))
            if own:
                state["workspace"] = torch.empty(cbm.cbm_log_probs_workspace_bytes(n, k, top), dtype=torch.uint8, device="cuda")
        else:
            largest, logsum, logs, p = _softmax(z.float())
            state["stats"] = torch.stack([largest, logsum], dim=1)
            state["entropy"] = -(p * logs).sum(dim=1)
            del logs, p
            loss = 1024.0 if type == "f16" else 1.0  # (a loss is scaled up where gradients are kept in fp16)
            state["dlogp"] = torch.full((n,), -loss / n, device="cuda")
            state["dentropy"] = torch.randn(n, device="cuda", generator=gen) * (0.1 * loss / n)
            state["dz"] = _matrix(n, k, pad, type)
    return state


def _softmax(z):
    """(largest, log of the sum of exp(z - largest), log probabilities with 0 where the probability is none, probabilities); an empty row has no probabilities."""
    largest = z.amax(dim=1)
    shifted = z - torch.where(largest == -math.inf, torch.zeros_like(largest), largest)[:, None]
    logsum = shifted.exp().sum(dim=1).log()
    logs = shifted - torch.where(logsum == -math.inf, torch.zeros_like(logsum), logsum)[:, None]
    p = logs.exp()
    logs.masked_fill_(logs == -math.inf, 0.0)
    return largest, logsum, logs, p


def _top(z, top):
    """The columns of the `top` largest values of each row, the lower column first among equal ones; (n, top) indices, and whether there is such a value."""
    n, k = z.shape
    bits = (z + 0.0).view(torch.int32)  # (no -0)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()  # as whole numbers in the values' order
    key = (order << 32) + (0x7FFFFFFF - torch.arange(k, device=z.device))
    some = min(top, k)
    best = torch.topk(key, some, dim=1).values
    columns = 0x7FFFFFFF - (best & 0xFFFFFFFF)
    if some < top:
        columns = torch.nn.functional.pad(columns, (0, top - some))
    there = z.gather(1, columns) > -math.inf
    if some < top:
        there[:, some:] = False
    return columns, there


def _plain(s):
    case = s["case"]
    op, type = case["op"], _TYPES[case["type"]]
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(dim=1)
        x = x - mean[:, None]
        rstd = (x * x).mean(dim=1).add_(s["eps"]).rsqrt_()
        return {"y": (x * rstd[:, None] * s["gamma"] + s["beta"]).to(type), "mean": mean, "rstd": rstd}
    if op == "norm_backward":
        dy, h = s["dy"].float(), (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        u = dy * s["gamma"]
        dx = (u - u.mean(dim=1, keepdim=True) - h * (u * h).mean(dim=1, keepdim=True)) * s["rstd"][:, None]
        return {"dx": dx.to(type), "dgamma": (dy * h).sum(dim=0), "dbeta": dy.sum(dim=0)}
    if op == "keep":
        q, code = _keep(s["x"])
        return {"values": _values(q, code).to(type), "steps": code.to(torch.uint8)}
    if op == "keep_relu":
        return {"dx": torch.where(s["q"] > 0, s["dy"].float(), torch.zeros((), device="cuda")).to(type)}
    if op == "keep_weights":
        return {"dw": _values(s["q"], s["steps"]).t() @ s["dy"].float()}
    z, label = s["z"].float(), s["labels"]
    n, k = z.shape
    given = (label >= 0) & (label < k)
    at = torch.where(given, label, torch.zeros_like(label))[:, None]
    if op == "log_probs":
        largest, logsum, logs, p = _softmax(z)
        chosen = (z.gather(1, at) - largest[:, None])[:, 0] - logsum
        logp = torch.where(given, torch.where(largest == -math.inf, largest, chosen), torch.zeros_like(chosen))
        entropy = -(p * logs).sum(dim=1)
        out = {"logp": logp, "entropy": entropy, "stats": torch.stack([largest, logsum], dim=1)}
        if case["top"]:
            columns, there = _top(z, case["top"])
            best = (z.gather(1, columns) - largest[:, None]) - logsum[:, None]
            out["values"] = torch.where(there, best, torch.full_like(best, -math.inf))
            out["columns"] = torch.where(there, columns, torch.full_like(columns, -1)).to(torch.int32)
        return out
    logs = (z - s["stats"][:, :1]) - s["stats"][:, 1:]
    p = logs.exp()
    logs.masked_fill_(logs == -math.inf, 0.0)
    dz = -p * (s["dlogp"] * given)[:, None] - s["dentropy"][:, None] * p * (logs + s["entropy"][:, None])
    dz.scatter_add_(1, at, (s["dlogp"] * given)[:, None])
    return {"dz": dz.to(type)}


def run(s):
    if not own:
        return _plain(s)
    cbm, op = s["cbm"], s["case"]["op"]
    if op == "norm":
        cbm.cbm_layer_norm(s["x"], s["gamma"], s["beta"], s["eps"], s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "norm_backward":
        cbm.cbm_layer_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["workspace"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if op == "keep":
        cbm.cbm_checkpoint_save(s["x"], s["q"], s["steps"])
        cbm.cbm_checkpoint_restore(s["q"], s["steps"], s["back"])
        return {"values": s["back"], "steps": s["steps"]}
    if op == "keep_relu":
        return {"dx": cbm.cbm_checkpoint_relu_backward(s["q"], s["steps"], s["dy"], s["dx"])}
    if op == "keep_weights":
        return {"dw": cbm.cbm_checkpoint_weight_grad(s["q"], s["steps"], s["dy"], s["dw"], s["workspace"])}
    if op == "log_probs":
        top = s["case"]["top"]
        cbm.cbm_log_probs(s["z"], s["labels"], s["logp"], s["entropy"], s["stats"], s["values"] if top else None, s["columns"] if top else None, s["workspace"])
        out = {"logp": s["logp"], "entropy": s["entropy"], "stats": s["stats"]}
        if top:
            out.update(values=s["values"], columns=s["columns"])
        return out
    return {"dz": cbm.cbm_log_probs_backward(s["z"], s["labels"], s["stats"], s["entropy"], s["dlogp"], s["dentropy"], s["dz"])}


def work(case):
    op, n, k, b = case["op"], case["n"], case["k"], _BYTES[case["type"]]
    steps = -(-k // _BLOCK)
    if op == "norm":
        return {"bytes": 2 * b * n * k + 8 * n + 8 * k, "flops": 8 * n * k}
    if op == "norm_backward":
        return {"bytes": 3 * b * n * k + 8 * n + 12 * k, "flops": 14 * n * k}
    if op == "keep":  # read once, kept, and, later, what was kept read and its values written
        return {"bytes": 2 * b * n * k + 2 * n * (k + steps), "flops": 4 * n * k}
    if op == "keep_relu":
        return {"bytes": (1 + 2 * b) * n * k + n * steps, "flops": n * k}
    if op == "keep_weights":
        return {"bytes": n * (k + steps) + b * n * case["c"] + 4 * k * case["c"], "flops": 2 * n * k * case["c"]}
    if op == "log_probs":
        return {"bytes": b * n * k + (8 + 16 + 8 * case["top"]) * n, "flops": 6 * n * k}
    return {"bytes": 2 * b * n * k + 28 * n, "flops": 8 * n * k}


def exact(case, seed):
    """The definitions, in 64 bits."""
    s = prepare(case, seed)
    op, n, k = case["op"], case["n"], case["k"]
    if op == "norm":
        x = s["x"].double()
        mean = x.sum(1) / k
        var = ((x - mean.unsqueeze(1)) ** 2).sum(1) / k
        y = (x - mean.unsqueeze(1)) / torch.sqrt(var + s["eps"]).unsqueeze(1)
        return {"y": y * s["gamma"].double() + s["beta"].double(), "mean": mean, "rstd": 1 / torch.sqrt(var + s["eps"])}
    if op == "norm_backward":
        r = s["rstd"].double().unsqueeze(1)
        h = (s["x"].double() - s["mean"].double().unsqueeze(1)) * r
        dy = s["dy"].double()
        dgamma, dbeta = torch.einsum("ij,ij->j", dy, h), dy.sum(0)
        dy *= s["gamma"].double()
        along = torch.einsum("ij,ij->i", dy, h).unsqueeze(1) / k
        dx = r * (dy - dy.sum(1, keepdim=True) / k - along * h)
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if op == "keep":
        parts = []
        for x in s["x"].double().split(_BLOCK, dim=1):
            size = x.abs().max(dim=1, keepdim=True).values
            e = (torch.frexp(size).exponent - 7).clamp_min(-126)
            e = torch.where(size == 0, torch.full_like(e, -126), e)
            q = torch.round(torch.ldexp(x.abs(), -e)).clamp(max=127)
            q = torch.where((q == 0) & (x != 0), torch.ones_like(q), q)
            parts.append(torch.ldexp(q * torch.sign(x), e))
        return {"values": torch.cat(parts, dim=1), "steps": None}
    if op == "keep_relu":
        return {"dx": s["dy"].double() * (s["q"] > 0)}
    if op == "keep_weights":
        total = torch.zeros((k, case["c"]), dtype=torch.float64, device="cuda")
        for i in range(0, n, 1 << 18):
            q, e = s["q"][i:i + (1 << 18)].double(), s["steps"][i:i + (1 << 18)].double()
            x = q * torch.exp2(e - 127).repeat_interleave(_BLOCK, dim=1)[:, :k]
            total += x.t().contiguous() @ s["dy"][i:i + (1 << 18)].double()
        return {"dw": total}
    z, label = s["z"].double(), s["labels"]
    given = (label >= 0) & (label < k)
    at = label.clamp(0, k - 1).unsqueeze(1)
    if op == "log_probs":
        lse = torch.logsumexp(z, dim=1, keepdim=True)
        logs = z - lse
        empty = (lse == -math.inf)[:, 0]
        logp = torch.where(empty, torch.full_like(lse[:, 0], -math.inf), logs.gather(1, at)[:, 0])
        p = torch.exp(logs)
        terms = torch.where(z == -math.inf, torch.zeros_like(p), p * logs)
        largest = z.max(dim=1).values
        stats = torch.stack([largest, torch.where(empty, largest, lse[:, 0] - largest)], dim=1)
        out = {"logp": torch.where(given, logp, torch.zeros_like(logp)), "entropy": -terms.sum(1), "stats": stats}
        if case["top"]:
            best = torch.topk(logs, min(case["top"], k), dim=1).values
            best = torch.where(empty.unsqueeze(1), torch.full_like(best, -math.inf), best)
            fill = torch.full((n, case["top"] - best.shape[1]), -math.inf, dtype=best.dtype, device=best.device)
            out.update(values=torch.cat([best, fill], dim=1), columns=None)
        return out
    stats = s["stats"].double()
    logs = z - stats.sum(1, keepdim=True)
    p = torch.exp(logs)
    a, h = (s["dlogp"] * given).double().unsqueeze(1), s["dentropy"].double().unsqueeze(1)
    hot = torch.zeros_like(z).scatter_(1, at, 1.0)
    slope = torch.where(z == -math.inf, torch.zeros_like(p), p * (logs + s["entropy"].double().unsqueeze(1)))
    return {"dz": a * (hot - p) - h * slope}
