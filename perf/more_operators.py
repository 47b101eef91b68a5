"""What is measured of the operators that tune a rank ladder on tokens.

Three operators that make up such a training step with the adapted projection and its gradients: the cross entropy of a
head over a large vocabulary, with its gradients and without keeping the logits; the orthogonalisation of factors by
Newton-Schulz products; and the update of a ladder's factors by their orthogonalised momentum.  ``run`` computes them in
their plain form (elementary torch operations in 32 bits, rounded once at the end), or, where ``own`` is set, through the
library's calls.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


# ------------------------------------------------------------------------------------------------------------- cases
def _head(name, T, d, V, direction, dx=True, dw=False, grad="bf16", prompt=0.0, pad=0):
    return {"name": name, "op": "head", "T": T, "d": d, "V": V, "direction": direction, "dx": dx and direction != "loss",
            "dw": dw and direction != "loss", "grad": grad, "prompt": prompt, "pad": pad}


def _ortho(name, factors, dtype, out, steps=5):
    """``factors``: text of 'rows x cols' pairs, a count in front of those that repeat ('2*64x4096')."""
    return {"name": name, "op": "ortho", "factors": factors, "dtype": dtype, "out": out, "steps": steps}


def _step(name, factors, dtype, nesterov=True, steps=5):
    return {"name": name, "op": "step", "factors": factors, "dtype": dtype, "nesterov": nesterov, "steps": steps}


def _shapes(case):
    out = []
    for part in case["factors"].split():
        count, _, shape = part.rpartition("*")
        rows, cols = shape.split("x")
        out += [(int(rows), int(cols))] * (int(count) if count else 1)
    return out


def _layers(n, R):
    """The adapter factors of n layers of seven projections (4096 and 11008 wide)."""
    return f"{6 * n}*4096x{R} {n}*11008x{R} {5 * n}*{R}x4096 {2 * n}*{R}x11008"


def listed():
    return [
        # the log-probability of one token: the smallest call, one pass over the head
        _head("head_one_token", 1, 4096, 32000, "loss"),
        # a short answer behind a prompt that was masked out before: loss and gradient of few rows
        _head("head_short_answer", 48, 4096, 32000, "both"),
        # a training step on 2048 tokens, the first quarter a prompt without targets
        _head("head_step", 2048, 4096, 32000, "both", prompt=0.25),
        # the same where the head is trained too: an odd vocabulary, an odd number of rows, 32-bit gradients
        _head("head_trained", 2047, 2048, 50021, "both", dw=True, grad="f32", pad=3),
        # the backward half of a step whose upstream gradient is known only afterwards
        _head("head_backward", 4096, 4096, 32000, "grad"),
        # validation over a wide vocabulary: the loss alone
        _head("head_eval_wide", 4000, 1024, 131072, "loss"),
        # the large step: 4 x 4096 tokens
        _head("head_large", 16384, 4096, 32000, "both"),
        # the factors of one small projection: launch latency counts
        _ortho("ortho_small", "1024x16 16x1024", "f32", "f32"),
        # the factors of a layer
        _ortho("ortho_layer", _layers(1, 64), "f32", "bf16"),
        # the widest ladder, 16-bit gradients, and an odd factor
        _ortho("ortho_wide", "4096x256 256x11008 1001x129", "bf16", "bf16"),
        # the update of a square projection's factors
        _step("step_square", "4096x64 64x4096", "f32"),
        # the update of all factors of the 32-layer stack
        _step("step_stack", _layers(32, 64), "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_head(rng):
    direction = rng.choice(["loss", "both", "both", "grad"])
    dw = rng.random() < 0.3
    return _head("", _log(rng, 1, 16384), _log(rng, 64, 8192), _log(rng, 500, 160000), direction, dx=not dw or rng.random() < 0.7,
                 dw=dw, grad=rng.choice(["bf16", "bf16", "f32"]), prompt=rng.choice([0.0, 0.0, 0.25, 0.6]),
                 pad=rng.choice([0, 0, 3, 8]))


def _draw_factors(rng):
    R, parts = _log(rng, 4, 256), []
    for _ in range(rng.choice([1, 2, 3, 8])):
        long = _log(rng, 64, 16000)
        count = rng.choice([1, 1, 2, 5])
        parts.append(f"{count}*{long}x{R}" if rng.random() < 0.5 else f"{count}*{R}x{long}")
    return " ".join(parts)


def draw(rng):
    op = rng.choice(["head", "head", "ortho", "step"])
    while True:
        if op == "head":
            case = _draw_head(rng)
            most = work(_head("", 16384, 4096, 32000, "both"))
            w = work(case)
            if w["flops"] <= most["flops"] and w["bytes"] <= 4 * most["bytes"]:
                break
        else:
            if op == "ortho":
                case = _ortho("", _draw_factors(rng), rng.choice(["f32", "bf16", "f16"]), rng.choice(["f32", "bf16"]),
                              rng.choice([5, 5, 3, 8]))
            else:
                case = _step("", _draw_factors(rng), rng.choice(["f32", "bf16"]), rng.random() < 0.7, rng.choice([5, 5, 6]))
            most = work(_step("", _layers(32, 64), "bf16"))
            w = work(case)
            if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"]:
                break
    del case["name"]
    return case


def work(case):
    if case["op"] == "head":
        T, d, V = case["T"], case["d"], case["V"]
        rows = T - int(case["prompt"] * T)
        b = 2 * rows * d + 2 * d * V + 8 * T                         # X, W, targets and weights
        f = 2 * rows * d * V                                         # the logits
        b += 8 * T                                                   # loss and log-sum-exp, or log-sum-exp and upstream gradient
        if case["dx"]:
            b += T * d * SIZES[case["grad"]]
            f += 2 * rows * d * V
        if case["dw"]:
            b += d * V * SIZES[case["grad"]]
            f += 2 * rows * d * V
        return {"bytes": b, "flops": f}
    b = f = 0
    for rows, cols in _shapes(case):
        R, n = min(rows, cols), rows * cols
        f += 3 * R * n + 4 * case["steps"] * R ** 3                  # half a Gram matrix, one product, the iteration
        if case["op"] == "ortho":
            b += n * (SIZES[case["dtype"]] + SIZES[case["out"]])
        else:
            b += n * (SIZES[case["dtype"]] + 4 + 4 + 4 + 4 + 2)
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _prepare_head(case, seed):
    """Activations of unit variance that lean towards their target's column by a varying amount (certain and uncertain
    tokens), a head whose logits spread by three, rows padded to whole 16 bytes and perhaps further."""
    g = _generator(seed)
    T, d, V = case["T"], case["d"], case["V"]

    def pitched(rows, cols):
        pitch = (cols + case["pad"] + 7) // 8 * 8
        return torch.zeros(rows, pitch, dtype=torch.bfloat16, device="cuda")[:, :cols]
    W = pitched(d, V)
    for r in range(0, d, 512):
        part = W[r:r + 512]
        part.copy_(torch.randn(part.shape, device="cuda", generator=g) * (3.0 * d ** -0.5))
    targets = torch.randint(0, V, (T,), device="cuda", generator=g, dtype=torch.int32)
    lean = torch.rand(T, 1, device="cuda", generator=g) * 4.0
    X = pitched(T, d)
    for r in range(0, T, 2048):
        part = X[r:r + 2048]
        toward = W[:, targets[r:r + 2048].long()].t().float()
        part.copy_(torch.randn(part.shape, device="cuda", generator=g) + lean[r:r + 2048] / 3.0 * toward)
    n = int(case["prompt"] * T)
    targets[:n] = -1
    weight = torch.full((T,), 1.0 / max(1, T - n), device="cuda")
    s = {"case": case, "X": X, "W": W, "targets": targets, "weight": weight, "lse": None, "dloss": None}
    if case["direction"] == "grad":
        s["lse"] = torch.cat([torch.logsumexp(X[r:r + 1024].float() @ W.float(), 1) for r in range(0, T, 1024)])
        s["dloss"] = torch.rand(T, device="cuda", generator=g) + 0.5
    if own:
        from paper_2601_21109_b200 import binding as cwl
        s["workspace"] = torch.empty(cwl.cwl_head_loss_workspace_bytes(T, d, V, case["dx"], case["dw"]), dtype=torch.uint8,
                                     device="cuda")
    return s


def _gradient(rows, cols, g):
    """A gradient of falling spectrum: most of its energy in a few directions, as those of adapter factors are."""
    R = min(rows, cols)
    left = torch.randn(rows, R, device="cuda", generator=g) * rows ** -0.5
    right = torch.randn(R, cols, device="cuda", generator=g) * cols ** -0.5
    return (left * torch.logspace(0, -2.5, R, device="cuda")) @ right


def _flat(shapes, dtype):
    """One buffer for all factors, each at a multiple of 64 elements, and the views of it."""
    at, views = 0, []
    for rows, cols in shapes:
        views.append((at, rows, cols))
        at += (rows * cols + 63) // 64 * 64
    buf = torch.zeros(at, dtype=dtype, device="cuda")
    return buf, [buf[a:a + r * c].view(r, c) for a, r, c in views]


def _prepare_ortho(case, seed):
    g = _generator(seed)
    shapes = _shapes(case)
    flat, U = _flat(shapes, DTYPES[case["dtype"]])
    for u in U:
        u.copy_(_gradient(*u.shape, g))
    out, O = _flat(shapes, DTYPES[case["out"]])
    s = {"case": case, "U": U, "out": out, "O": O}
    if own:
        from paper_2601_21109_b200 import binding as cwl
        s["call"] = cwl.OrthogonalizeCall(U, O, steps=case["steps"], coefficients=COEFFICIENTS, eps=EPS)
    return s


def _prepare_step(case, seed):
    g = _generator(seed)
    shapes = _shapes(case)
    s = {"case": case, "lr": 0.02, "momentum": 0.95, "decay": 0.01}
    _, s["grads"] = _flat(shapes, DTYPES[case["dtype"]])
    s["m_flat"], s["m"] = _flat(shapes, torch.float32)
    s["p_flat"], s["p"] = _flat(shapes, torch.float32)
    s["low_flat"], s["low"] = _flat(shapes, torch.bfloat16)
    for gr, m, p, low in zip(s["grads"], s["m"], s["p"], s["low"]):
        past = _gradient(*gr.shape, g)
        gr.copy_(past + 0.5 * _gradient(*gr.shape, g))
        m.copy_(past * 10.0)
        p.copy_(torch.randn(p.shape, device="cuda", generator=g) * p.shape[0] ** -0.5)
        low.copy_(p)
    if own:
        from paper_2601_21109_b200 import binding as cwl
        s["call"] = cwl.FactorStep(s["p"], s["low"], s["grads"], s["m"], steps=case["steps"], coefficients=COEFFICIENTS, eps=EPS)
    return s


def prepare(case, seed):
    return {"head": _prepare_head, "ortho": _prepare_ortho, "step": _prepare_step}[case["op"]](case, seed)


# ------------------------------------------------------------------------------------------------------- plain forms
def _plain_head(s):
    case, X, W, w = s["case"], s["X"].float(), s["W"].float(), s["weight"]
    real, y = s["targets"] >= 0, s["targets"].clamp(min=0).long()[:, None]
    z = X @ W
    out = {}
    if case["direction"] != "grad":
        m = z.amax(1, keepdim=True)
        lse = m[:, 0] + torch.log(torch.exp(z - m).sum(1))
        out["lse"] = torch.where(real, lse, 0.0)
        out["loss"] = torch.where(real, w * (lse - z.gather(1, y)[:, 0]), 0.0)
        up = w
    else:
        lse, up = s["lse"], w * s["dloss"]
    if case["dx"] or case["dw"]:
        up = torch.where(real, up, 0.0)[:, None]
        z.sub_(lse[:, None]).exp_()
        z.scatter_add_(1, y, torch.full_like(y, -1, dtype=z.dtype))
        z.mul_(up)
        if case["dx"]:
            out["dX"] = (z @ W.t()).to(DTYPES[case["grad"]])
        if case["dw"]:
            out["dW"] = (X.t() @ z).to(DTYPES[case["grad"]])
    return out


def _newton_schulz(u, steps):
    a, b, c = COEFFICIENTS
    x = u if u.shape[0] <= u.shape[1] else u.t()
    x = x / (torch.sqrt((x * x).sum()) + EPS)
    for _ in range(steps):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x if u.shape[0] <= u.shape[1] else x.t()


def _plain_ortho(s):
    for u, o in zip(s["U"], s["O"]):
        o.copy_(_newton_schulz(u.float(), s["case"]["steps"]))
    return s["out"]


def _plain_step(s):
    beta, lr = s["momentum"], s["lr"]
    for gr, m, p, low in zip(s["grads"], s["m"], s["p"], s["low"]):
        g32 = gr.float()
        m.mul_(beta).add_(g32)
        u = g32 + beta * m if s["case"]["nesterov"] else m
        rows, cols = p.shape
        scale = math.sqrt(max(1.0, rows / cols))
        p.mul_(1.0 - lr * s["decay"]).sub_(lr * scale * _newton_schulz(u, s["case"]["steps"]))
        low.copy_(p)
    return {"master": s["p_flat"], "low": s["low_flat"], "momentum": s["m_flat"]}


# -------------------------------------------------------------------------------------------------------- own calls
def _own_head(s):
    from paper_2601_21109_b200 import binding as cwl
    case = s["case"]
    r = cwl.cwl_head_loss(s["X"], s["W"], s["targets"], weight=s["weight"], dloss=s["dloss"], lse=s["lse"],
                          want_loss=case["direction"] != "grad", want_dx=case["dx"], want_dw=case["dw"],
                          grad_dtype=DTYPES[case["grad"]], workspace=s["workspace"])
    out = {}
    if case["direction"] != "grad":
        out["lse"], out["loss"] = r.lse, r.loss
    if case["dx"]:
        out["dX"] = r.dX
    if case["dw"]:
        out["dW"] = r.dW
    return out


def _own_ortho(s):
    s["call"]()
    return s["out"]


def _own_step(s):
    s["call"](lr=s["lr"], momentum=s["momentum"], weight_decay=s["decay"], nesterov=s["case"]["nesterov"])
    return {"master": s["p_flat"], "low": s["low_flat"], "momentum": s["m_flat"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"head": _own_head, "ortho": _own_ortho, "step": _own_step}[op](state)
    return {"head": _plain_head, "ortho": _plain_ortho, "step": _plain_step}[op](state)


# ----------------------------------------------------------------------------------------- the definitions in 64 bits
def _exact_head(s):
    case, W = s["case"], s["W"].double()
    lse, loss, dX = [], [], []
    dW = torch.zeros(W.shape, dtype=torch.float64, device=W.device) if case["dw"] else None
    for r in range(0, case["T"], 1024):
        part = slice(r, r + 1024)
        X, y, w = s["X"][part].double(), s["targets"][part].long(), s["weight"][part].double()
        keep = y >= 0
        logq = torch.matmul(X, W)
        norm = torch.logsumexp(logq, 1) if case["direction"] != "grad" else s["lse"][part].double()
        logq -= norm[:, None]
        if case["direction"] != "grad":
            lse.append(norm.masked_fill(~keep, 0.0))
            loss.append((-w * logq[torch.arange(len(y)), y.clamp(min=0)]).masked_fill(~keep, 0.0))
        if case["dx"] or case["dw"]:
            q = logq.exp()
            q[torch.arange(len(y)), y.clamp(min=0)] -= 1.0
            if s["dloss"] is not None:
                w = w * s["dloss"][part].double()
            q = (q * w[:, None]).masked_fill(~keep[:, None], 0.0)
            if case["dx"]:
                dX.append(torch.matmul(q, W.T))
            if case["dw"]:
                dW += torch.matmul(X.T, q)
    out = {}
    if lse:
        out["lse"], out["loss"] = torch.cat(lse), torch.cat(loss)
    if dX:
        out["dX"] = torch.cat(dX)
    if dW is not None:
        out["dW"] = dW
    return out


def _exact_polar(u, steps):
    """The iteration on the singular values alone: it leaves the singular vectors as they are."""
    left, sigma, right = torch.linalg.svd(u, full_matrices=False)
    sigma = sigma / (sigma.square().sum().sqrt() + EPS)
    a, b, c = COEFFICIENTS
    for _ in range(steps):
        sigma = a * sigma + b * sigma ** 3 + c * sigma ** 5
    return (left * sigma) @ right


def _exact_products(u, steps):
    """The same by products of R x R matrices, for more factors than singular value decompositions would be done with."""
    wide = u if u.shape[0] <= u.shape[1] else u.T
    gram = torch.matmul(wide, wide.T)
    size = gram.trace().sqrt() + EPS
    gram = gram / size ** 2
    eye = torch.eye(len(gram), dtype=gram.dtype, device=gram.device)
    total = eye / size
    a, b, c = COEFFICIENTS
    for _ in range(steps):
        poly = a * eye + b * gram + c * torch.matmul(gram, gram)
        total, gram = torch.matmul(poly, total), torch.matmul(torch.matmul(poly, gram), poly.T)
    out = torch.matmul(total, wide)
    return out if u.shape[0] <= u.shape[1] else out.T


def _exact_update(u, steps, many):
    return _exact_products(u, steps) if many else _exact_polar(u, steps)


def _exact_ortho(s):
    out, O = _flat(_shapes(s["case"]), torch.float64)
    for u, o in zip(s["U"], O):
        o.copy_(_exact_update(u.double(), s["case"]["steps"], len(O) > 20))
    return out


def _exact_step(s):
    beta, lr, shapes = s["momentum"], s["lr"], _shapes(s["case"])
    master, P = _flat(shapes, torch.float64)
    momentum, M = _flat(shapes, torch.float64)
    for gr, m, p, M64, P64 in zip(s["grads"], s["m"], s["p"], M, P):
        M64.copy_(beta * m.double() + gr.double())
        u = gr.double() + beta * M64 if s["case"]["nesterov"] else M64
        scale = max(1.0, p.shape[0] / p.shape[1]) ** 0.5
        P64.copy_(p.double() * (1.0 - lr * s["decay"]) - lr * scale * _exact_update(u, s["case"]["steps"], len(P) > 20))
    return {"master": master, "low": master, "momentum": momentum}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"head": _exact_head, "ortho": _exact_ortho, "step": _exact_step}[case["op"]](s)
