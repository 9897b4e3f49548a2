"""The operators of a training step that are made of products, as cases that can be timed and checked.

A gated layer (both projections, the activation and their product; forward and backward), log probabilities of labels straight from a layer's outputs and
the classes' weights, without its scores (forward and backward), and the orthogonal update of a weight matrix.  `run` with `own` false is each operator in
elementary torch operations in 32 bits; with `own` true it is the library's call.  Matrices are row-major; `pad` columns beside each row make its stride longer
than the row.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_COEFFICIENTS = (3.4445, -4.7750, 2.0315)
_EPS = 1e-7
_MOST = 1 << 28  # values of the largest matrix
_FLOPS = {"f32": 1.2e11, "bf16": 8e11, "f16": 8e11}  # of the largest drawn case


def listed():
    return [
        # one answer through a gated layer: the single row of serving, bound by the weights
        {"name": "gated_one_row", "op": "gated", "n": 1, "k": 1024, "m": 4096, "type": "bf16", "pad": 0, "act": "silu", "keep": False},
        # a citation network's bag-of-words features through a layer of odd width, with what the backward pass reads
        {"name": "gated_nodes_odd", "op": "gated", "n": 19717, "k": 500, "m": 333, "type": "f32", "pad": 0, "act": "gelu", "keep": True},
        # the forward pass of training over a batch of many rows in 16 bits
        {"name": "gated_large", "op": "gated", "n": 65536, "k": 1024, "m": 4096, "type": "bf16", "pad": 0, "act": "silu", "keep": True},
        # training on a similarity graph: many rows, a narrow layer
        {"name": "gated_back_graph", "op": "gated_backward", "n": 132534, "k": 100, "m": 256, "type": "f32", "pad": 0, "act": "relu"},
        # the backward pass of a wide layer in 16 bits
        {"name": "gated_back_wide", "op": "gated_backward", "n": 16384, "k": 1024, "m": 4096, "type": "bf16", "pad": 0, "act": "silu"},
        # how likely one answer is over a vocabulary: the single row of serving
        {"name": "classes_one_row", "op": "classes", "n": 1, "d": 1024, "c": 32000, "type": "bf16", "pad": 0},
        # the loss of a batch of positions over a vocabulary
        {"name": "classes_vocabulary", "op": "classes", "n": 4096, "d": 1024, "c": 32000, "type": "bf16", "pad": 0},
        # its gradients
        {"name": "classes_back_vocabulary", "op": "classes_backward", "n": 8192, "d": 1024, "c": 32000, "type": "bf16", "pad": 0},
        # a citation network with very many classes, in 32 bits, sizes that fill no power of two
        {"name": "classes_back_odd", "op": "classes_backward", "n": 19717, "d": 100, "c": 5003, "type": "f32", "pad": 0},
        # the update of a hidden layer of a small graph: the smallest call, where launches count
        {"name": "update_small", "op": "orthogonal", "m": 64, "n": 64, "type": "f32", "pad": 0},
        # the update of a first layer over bag-of-words features, an odd width
        {"name": "update_odd", "op": "orthogonal", "m": 500, "n": 1333, "type": "f32", "pad": 0},
        # the update of a wide square layer, in 16 bits
        {"name": "update_large", "op": "orthogonal", "m": 4096, "n": 4096, "type": "bf16", "pad": 0},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["gated", "gated", "gated_backward", "gated_backward", "classes", "classes", "classes_backward", "classes_backward", "orthogonal", "orthogonal"])
    case = {"op": op, "type": rng.choice(["f32", "bf16", "bf16", "f16"]), "pad": rng.choice([0, 0, 0, 1, 4, 8])}
    even = lambda v: (v + 7) // 8 * 8 if v > 8 and rng.random() < 0.5 else v  # noqa: E731
    most = _FLOPS[case["type"]]
    if op.startswith("gated"):
        k, m = even(_log(rng, 4, 2048)), even(_log(rng, 4, 8192))
        n = min(2097152, most / ((8 if op == "gated_backward" else 4) * k * m), _MOST / max(k + 8, m + 8))
        case.update(n=_log(rng, 1, max(1, int(n))), k=k, m=m, act=rng.choice(["silu", "gelu", "relu"]))
        return {**case, "keep": rng.random() < 0.6} if op == "gated" else case
    if op.startswith("classes"):
        d, c = even(_log(rng, 8, 2048)), even(_log(rng, 2, 131072))
        n = min(1048576, most / ((6 if op == "classes_backward" else 2) * d * c), _MOST / max(d + 8, c + 8))
        return {**case, "n": _log(rng, 1, max(1, int(n))), "d": d, "c": c}
    return {**case, "m": even(_log(rng, 1, 2500)), "n": even(_log(rng, 1, 2500))}


def _matrix(n, k, pad, type):
    return torch.empty((n, k + pad), dtype=_TYPES[type], device="cuda")[:, :k]


def _gaussian(n, k, pad, type, gen, scale=1.0):
    out = _matrix(n, k, pad, type)
    out.copy_(torch.randn((n, k), device="cuda", generator=gen).mul_(scale))
    return out


def prepare(case, seed):
    op, type, pad = case["op"], case["type"], case["pad"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case}
    if own:
        import paper_2409_02208_amd as cbm

        state["cbm"] = cbm
    room = lambda size: torch.empty(size, dtype=torch.uint8, device="cuda")  # noqa: E731
    if op.startswith("gated"):
        n, k, m = case["n"], case["k"], case["m"]
        state["x"] = _gaussian(n, k, pad, type, gen)  # a layer norm's outputs
        state["wg"], state["wu"] = (_gaussian(k, m, pad, type, gen, k ** -0.5) for _ in range(2))
        if op == "gated":
            state["h"] = _matrix(n, m, pad, type)
            if case["keep"]:
                state["g"], state["u"] = _matrix(n, m, pad, type), _matrix(n, m, pad, type)
            if own:
                state["workspace"] = room(cbm.cbm_gated_linear_workspace_bytes(n, k, m, _TYPES[type]))
        else:
            state["g"], state["u"] = _matrix(n, m, pad, type), _matrix(n, m, pad, type)
            x = state["x"].float()
            state["g"].copy_(x @ state["wg"].float())
            state["u"].copy_(x @ state["wu"].float())
            del x
            state["dh"] = _gaussian(n, m, pad, type, gen, 0.01)
            state["dx"], state["dwg"], state["dwu"] = _matrix(n, k, pad, type), _matrix(k, m, pad, type), _matrix(k, m, pad, type)
            if own:
                state["workspace"] = room(cbm.cbm_gated_linear_backward_workspace_bytes(n, k, m, _TYPES[type]))
    elif op.startswith("classes"):
        n, d, c = case["n"], case["d"], case["c"]
        state["x"] = _gaussian(n, d, pad, type, gen)
        state["w"] = _gaussian(d, c, pad, type, gen, 3 * d ** -0.5)
        state["labels"] = torch.randint(0, c, (n,), device="cuda", generator=gen)
        state["labels"][torch.rand(n, device="cuda", generator=gen) < 0.1] = -1  # nodes without a label
        if n == 1:
            state["labels"].clamp_(min=0)
        state["logp"], state["stats"] = torch.empty(n, device="cuda"), torch.empty((n, 2), device="cuda")
        if op == "classes_backward":
            z = state["x"].float() @ state["w"].float()
            largest = z.amax(dim=1)
            state["stats"][:, 0] = largest
            state["stats"][:, 1] = z.sub_(largest[:, None]).exp_().sum(dim=1).log_()
            del z
            loss = 1024.0 if type == "f16" else 1.0  # (a loss is scaled up where gradients are kept in fp16)
            state["dlogp"] = (torch.rand(n, device="cuda", generator=gen) + 0.5) * (-loss / n)  # rows of different weight
            state["dx"], state["dw"] = _matrix(n, d, pad, type), _matrix(d, c, pad, type)
            if own:
                state["workspace"] = room(cbm.cbm_linear_log_probs_backward_workspace_bytes(n, d, c, _TYPES[type]))
        elif own:
            state["workspace"] = room(cbm.cbm_linear_log_probs_workspace_bytes(n, d, c, _TYPES[type]))
    else:
        m, n = case["m"], case["n"]
        rank = min(8, m, n)  # a weights' gradient: a few strong directions, and noise
        strong = torch.randn((m, rank), device="cuda", generator=gen) @ torch.randn((rank, n), device="cuda", generator=gen)
        state["x"] = _matrix(m, n, pad, type)
        state["x"].copy_(1e-3 * (strong + torch.randn((m, n), device="cuda", generator=gen)))
        state["y"] = _matrix(m, n, pad, type)
        if own:
            state["workspace"] = room(cbm.cbm_orthogonalise_workspace_bytes(m, n, _TYPES[type]))
    return state


def _activation(act, g):
    """The activation and its slope."""
    if act == "relu":
        return g.clamp_min(0), (g > 0).to(g.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    below = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * below, below + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _plain(s):
    case = s["case"]
    op, type = case["op"], _TYPES[case["type"]]
    if op == "gated":
        x = s["x"].float()
        g, u = x @ s["wg"].float(), x @ s["wu"].float()
        out = {"h": (_activation(case["act"], g)[0] * u).to(type)}
        if case["keep"]:
            out.update(g=g.to(type), u=u.to(type))
        return out
    if op == "gated_backward":
        value, slope = _activation(case["act"], s["g"].float())
        dh, x = s["dh"].float(), s["x"].float()
        du = dh * value
        dg = dh * s["u"].float() * slope
        dx = dg @ s["wg"].float().t() + du @ s["wu"].float().t()
        return {"dx": dx.to(type), "dwg": (x.t() @ dg).to(type), "dwu": (x.t() @ du).to(type)}
    if op == "orthogonal":
        a, b, c = _COEFFICIENTS
        x = s["x"].float()
        tall = x.shape[0] > x.shape[1]
        if tall:
            x = x.t()
        x = x / ((x * x).sum().sqrt() + _EPS)
        x = _step(x, a, b, c)
        x = _step(x, a, b, c)
        x = _step(x, a, b, c)
        x = _step(x, a, b, c)
        x = _step(x, a, b, c)
        return {"y": (x.t() if tall else x).to(type)}
    x, w, label = s["x"].float(), s["w"].float(), s["labels"]
    z = x @ w
    n, c = z.shape
    given = (label >= 0) & (label < c)
    at = torch.where(given, label, torch.zeros_like(label))[:, None]
    if op == "classes":
        largest = z.amax(dim=1)
        logsum = (z - largest[:, None]).exp().sum(dim=1).log()
        logp = (z.gather(1, at)[:, 0] - largest) - logsum
        return {"logp": torch.where(given, logp, torch.zeros_like(logp)), "stats": torch.stack([largest, logsum], dim=1)}
    slope = s["dlogp"] * given
    dz = ((z - s["stats"][:, :1]) - s["stats"][:, 1:]).exp_().mul_(-slope[:, None])
    dz.scatter_add_(1, at, slope[:, None])
    return {"dx": (dz @ w.t()).to(type), "dw": (x.t() @ dz).to(type)}


def _step(x, a, b, c):
    """A step of the iteration that drives singular values towards one."""
    gram = x @ x.t()
    return a * x + (b * gram + c * (gram @ gram)) @ x


def run(s):
    if not own:
        return _plain(s)
    cbm, case = s["cbm"], s["case"]
    op = case["op"]
    if op == "gated":
        cbm.cbm_gated_linear(s["x"], s["wg"], s["wu"], s["h"], s.get("g"), s.get("u"), activation=case["act"], workspace=s["workspace"])
        return {"h": s["h"], "g": s["g"], "u": s["u"]} if case["keep"] else {"h": s["h"]}
    if op == "gated_backward":
        cbm.cbm_gated_linear_backward(s["dh"], s["x"], s["wg"], s["wu"], s["g"], s["u"], s["dx"], s["dwg"], s["dwu"], activation=case["act"], workspace=s["workspace"])
        return {"dx": s["dx"], "dwg": s["dwg"], "dwu": s["dwu"]}
    if op == "classes":
        cbm.cbm_linear_log_probs(s["x"], s["w"], s["labels"], s["logp"], s["stats"], workspace=s["workspace"])
        return {"logp": s["logp"], "stats": s["stats"]}
    if op == "classes_backward":
        cbm.cbm_linear_log_probs_backward(s["x"], s["w"], s["labels"], s["stats"], s["dlogp"], s["dx"], s["dw"], workspace=s["workspace"])
        return {"dx": s["dx"], "dw": s["dw"]}
    return {"y": cbm.cbm_orthogonalise(s["x"], s["y"], steps=5, coefficients=_COEFFICIENTS, eps=_EPS, workspace=s["workspace"])}


def work(case):
    op, b = case["op"], _BYTES[case["type"]]
    if op.startswith("gated"):
        n, k, m = case["n"], case["k"], case["m"]
        if op == "gated":
            return {"bytes": b * (n * k + 2 * k * m + (3 if case["keep"] else 1) * n * m), "flops": 4 * n * k * m}
        return {"bytes": b * (2 * n * k + 4 * k * m + 3 * n * m), "flops": 8 * n * k * m}
    if op.startswith("classes"):
        n, d, c = case["n"], case["d"], case["c"]
        if op == "classes":
            return {"bytes": b * (n * d + d * c) + 20 * n, "flops": 2 * n * d * c}
        return {"bytes": 2 * b * (n * d + d * c) + 20 * n, "flops": 6 * n * d * c}  # (the scores are not kept: they are made again)
    m, n = sorted((case["m"], case["n"]))
    return {"bytes": 2 * b * m * n, "flops": 5 * (m * m * n + m ** 3 + 2 * m * m * n)}  # half of each symmetric product


def exact(case, seed):
    """The definitions, in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op in ("gated", "gated_backward"):
        x, wg, wu = s["x"].double(), s["wg"].double(), s["wu"].double()
        g, u = (torch.mm(x, wg), torch.mm(x, wu)) if op == "gated" else (s["g"].double(), s["u"].double())
        if case["act"] == "relu":
            value, slope = torch.where(g > 0, g, torch.zeros_like(g)), torch.where(g > 0, torch.ones_like(g), torch.zeros_like(g))
        elif case["act"] == "silu":
            value = g * torch.sigmoid(g)
            slope = torch.sigmoid(g) + value * torch.sigmoid(-g)
        else:
            cdf = torch.special.ndtr(g)
            value, slope = g * cdf, cdf + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
        if op == "gated":
            return {"h": value * u, "g": g, "u": u} if case["keep"] else {"h": value * u}
        dh = s["dh"].double()
        du, dg = value.mul_(dh), slope.mul_(u).mul_(dh)
        return {"dx": torch.mm(dg, wg.t()).addmm_(du, wu.t()), "dwg": torch.mm(x.t(), dg), "dwu": torch.mm(x.t(), du)}
    if op == "orthogonal":
        x = s["x"].double()
        x = x / (torch.linalg.norm(x) + _EPS)
        wide = x.shape[0] <= x.shape[1]
        for _ in range(5):
            g = torch.mm(x, x.t()) if wide else torch.mm(x.t(), x)
            p = _COEFFICIENTS[0] * torch.eye(g.shape[0], dtype=g.dtype, device=g.device) + _COEFFICIENTS[1] * g + _COEFFICIENTS[2] * torch.mm(g, g)
            x = torch.mm(p, x) if wide else torch.mm(x, p)
        return {"y": x}
    x, w, label = s["x"].double(), s["w"].double(), s["labels"]
    z = torch.mm(x, w)
    given = (label >= 0) & (label < case["c"])
    at = label.clamp(0, case["c"] - 1).unsqueeze(1)
    if op == "classes":
        lse, top = torch.logsumexp(z, dim=1), z.max(dim=1).values
        return {"logp": (z.gather(1, at)[:, 0] - lse) * given, "stats": torch.stack([top, lse - top], dim=1)}
    hot = torch.zeros_like(z).scatter_(1, at, 1.0)
    z = hot.sub_(torch.exp(z - s["stats"].double().sum(1, keepdim=True))).mul_((s["dlogp"] * given).double().unsqueeze(1))
    return {"dx": torch.mm(z, w.t()), "dw": torch.mm(x.t(), z)}
