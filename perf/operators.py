"""What is measured of the operators that train and observe a rank ladder.

Three operators that belong together: the log-probabilities of a logit row with its top alternatives (what a teacher
leaves behind, what a decode step reports), the distillation loss from a teacher's top logits with its gradient, and the
gradient of the adapter factors under a chunk table.  ``run`` computes them in their plain form (elementary torch
operations in 32 bits, rounded once at the end), or, where ``own`` is set, through the library's calls.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}


# ------------------------------------------------------------------------------------------------------------- cases
def _logprobs(name, T, V, dtype, top_k, temperature=1.0, pad=0, constrained=0.0, targets=True):
    return {"name": name, "op": "logprobs", "T": T, "V": V, "dtype": dtype, "top_k": top_k, "temperature": temperature,
            "pad": pad, "constrained": constrained, "targets": targets}


def _distill(name, T, V, dtype, K, teacher, direction, temperature=1.0, pad=0, prompt=0.0):
    return {"name": name, "op": "distill", "T": T, "V": V, "dtype": dtype, "K": K, "teacher": teacher,
            "direction": direction, "temperature": temperature, "pad": pad, "prompt": prompt}


def _grads(name, T, d_in, d_out, R, chunk, window=8):
    return {"name": name, "op": "grads", "T": T, "d_in": d_in, "d_out": d_out, "R": R, "chunk": chunk, "window": window}


def listed():
    return [
        # one decoding stream: the chosen token's log-probability and twenty alternatives; launch latency counts
        _logprobs("logprobs_decode_1", 1, 32000, "f32", 20),
        # a decode step of 64 streams, a quarter of them held to a grammar (most of the vocabulary at -inf)
        _logprobs("logprobs_decode_64", 64, 32000, "bf16", 20, temperature=0.7, constrained=0.25),
        # scoring a prompt: the log-probability of every given token and the entropy, no alternatives
        _logprobs("logprobs_prompt", 2048, 32000, "f32", 0),
        # a teacher's pass over 4 x 4096 tokens: the top 64 of every row are kept for the student
        _logprobs("logprobs_teacher", 16384, 32000, "bf16", 64, targets=False),
        # an odd vocabulary whose rows start anywhere, odd number of rows
        _logprobs("logprobs_odd", 777, 50021, "f32", 8, temperature=1.3),
        # a handful of tokens of an odd vocabulary: the smallest training call
        _distill("distill_small", 7, 32003, "f32", 8, "logprobs", "both", pad=5),
        # a training step on 2048 tokens of logits as the adapted projection writes them, the first quarter a prompt
        _distill("distill_step", 2048, 32000, "bf16", 64, "logprobs", "both", temperature=2.0, prompt=0.25),
        # the large step: 4 x 4096 tokens, 32-bit logits, the upstream gradient known only afterwards
        _distill("distill_large_grad", 16384, 32000, "f32", 64, "logits", "grad"),
        # validation over a wide vocabulary: the loss alone
        _distill("distill_eval_wide", 1000, 131072, "f16", 100, "logits", "loss", temperature=1.5),
        # adapter gradients of a small projection over one short sequence
        _grads("grads_small", 256, 1024, 1024, 16, 32, window=4),
        # a square projection over a 2048-token sequence
        _grads("grads_square", 2048, 4096, 4096, 64, 96),
        # an up projection over 4 x 4096 tokens
        _grads("grads_up_large", 16384, 4096, 11008, 64, 96),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "distill", "grads"])
    while True:
        if op == "logprobs":
            T, V = _log(rng, 1, 16384), _log(rng, 500, 160000)
            dtype = rng.choice(["f32", "bf16", "f16"])
            case = _logprobs("", T, V, dtype, rng.choice([0, 1, 5, 20, 64, 128]), rng.choice([1.0, 0.7, 1.3]),
                             rng.choice([0, 0, 3, 8]), rng.choice([0.0, 0.0, 0.3]), rng.random() < 0.8)
            most = 16384 * 32000 * 2
        elif op == "distill":
            T, V = _log(rng, 1, 16384), _log(rng, 500, 160000)
            dtype = rng.choice(["f32", "bf16", "f16"])
            case = _distill("", T, V, dtype, rng.choice([1, 8, 20, 64, 100, 128]), rng.choice(["logits", "logprobs"]),
                            rng.choice(["both", "both", "grad", "loss"]), rng.choice([1.0, 1.5, 2.0]),
                            rng.choice([0, 0, 3, 8]), rng.choice([0.0, 0.25]))
            most = 2 * 16384 * 32000 * 4
        else:
            R = rng.choice([16, 32, 48, 64, 128, 256])
            d_in, d_out = 16 * _log(rng, 32, 700), 16 * _log(rng, 32, 2000)
            case = _grads("", _log(rng, 16, 16384), d_in, d_out, R, rng.choice([24, 96, 200]), rng.choice([0, 4, 8]))
            most = None
        w = work(case)
        if most is not None and w["bytes"] <= most:
            break
        if most is None and w["flops"] <= 4 * 16384 * 64 * (4096 + 11008) and w["bytes"] <= 2 * 16384 * (4096 + 11008):
            break
    del case["name"]
    return case


def work(case):
    T = case["T"]
    if case["op"] == "logprobs":
        V, es, k = case["V"], SIZES[case["dtype"]], case["top_k"]
        return {"bytes": T * V * es + T * (8 * k + 8) + (8 * T if case["targets"] else 0), "flops": 4 * T * V}
    if case["op"] == "distill":
        V, es, k = case["V"], SIZES[case["dtype"]], case["K"]
        active = T - int(case["prompt"] * T)
        b = active * V * es + active * 8 * k + 4 * T
        if case["direction"] != "grad":
            b += 4 * T
        if case["direction"] != "loss":
            b += T * V * es
        if case["direction"] == "grad":
            b += 4 * T
        return {"bytes": b, "flops": (6 if case["direction"] != "loss" else 3) * active * V}
    d, R = case["d_in"] + case["d_out"], case["R"]
    return {"bytes": 2 * (T * d + 2 * R * d), "flops": 4 * T * R * d}


# ------------------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _logits(case, g):
    """Gaussian rows, one temperature per 64 tokens (peaked and flat spans), in which up to sixteen tokens stand out as
    the likely continuations, in a matrix that may have a wider pitch."""
    T, V = case["T"], case["V"]
    buf = torch.zeros(T, V + case["pad"], dtype=DTYPES[case["dtype"]], device="cuda")
    tau = torch.empty((T + 63) // 64, device="cuda").uniform_(0.3, 3.0, generator=g).repeat_interleave(64)[:T]
    for r in range(0, T, 4096):
        part = torch.randn(min(4096, T - r), V, device="cuda", generator=g) / tau[r:r + 4096, None]
        likely = torch.randint(0, V, (part.shape[0], 16), device="cuda", generator=g)
        part.scatter_(1, likely, torch.rand(likely.shape, device="cuda", generator=g) * 8 + 10)
        buf[r:r + 4096, :V] = part.to(buf.dtype)
    return buf[:, :V]


def _prepare_logprobs(case, seed):
    g = _generator(seed)
    T, V = case["T"], case["V"]
    z = _logits(case, g)
    targets = torch.randint(0, V, (T,), device="cuda", generator=g, dtype=torch.int32) if case["targets"] else None
    n = int(case["constrained"] * T)
    if n:
        keep = torch.rand(n, V, device="cuda", generator=g) < 0.01
        z[:n].masked_fill_(~keep, float("-inf"))
        z[:n, V // 2] = 1.0                                    # at least one token is allowed
        if targets is not None:
            targets[:n] = z[:n].float().argmax(1).to(torch.int32)
    s = {"case": case, "logits": z, "targets": targets}
    if own:
        from paper_2601_21109_b200 import binding as cwl
        s["out"] = cwl.TokenLogprobs(T, case["top_k"], with_targets=targets is not None)
    return s


def _prepare_distill(case, seed):
    g = _generator(seed)
    T, V, K, tau = case["T"], case["V"], case["K"], case["temperature"]
    z = _logits(case, g)
    ids = torch.empty(T, K, dtype=torch.int32, device="cuda")
    vals = torch.empty(T, K, dtype=torch.float32, device="cuda")
    for r in range(0, T, 2048):
        teacher = z[r:r + 2048].float()
        teacher = teacher + 0.5 * torch.randn(teacher.shape, device="cuda", generator=g)
        if case["teacher"] == "logprobs":                      # of the tempered teacher, over its whole vocabulary
            teacher /= tau
            teacher -= teacher.logsumexp(1, keepdim=True)
        v, i = teacher.topk(K, dim=1)
        ids[r:r + 2048], vals[r:r + 2048] = i.to(torch.int32), v
    # a quarter of the rows kept fewer than K entries
    short = torch.rand(T, device="cuda", generator=g) < 0.25
    kept = torch.randint((K + 1) // 2, K + 1, (T,), device="cuda", generator=g)
    drop = short[:, None] & (torch.arange(K, device="cuda")[None] >= kept[:, None])
    ids.masked_fill_(drop, -1)
    n = int(case["prompt"] * T)
    weight = torch.full((T,), 1.0 if case["dtype"] == "f16" else 1.0 / max(1, T - n), device="cuda")
    weight[:n] = 0.0
    s = {"case": case, "logits": z, "ids": ids, "values": vals, "weight": weight, "dloss": None}
    if case["direction"] == "grad":
        s["dloss"] = torch.rand(T, device="cuda", generator=g) + 0.5
    return s


def _table(case, seed):
    """Chunk joins around every `chunk` tokens, ranks and scales of a three-rung ladder; two sequences."""
    rng = np.random.default_rng(seed)
    T, R = case["T"], case["R"]
    cuts, t = [0], 0
    while T - t > case["chunk"] + 16:
        t += int(rng.integers(max(8, case["chunk"] // 2), case["chunk"] + 1))
        cuts.append(t)
    n = len(cuts)
    ranks = np.array([max(1, R // 4), max(1, R // 2), R], np.int32)[rng.integers(0, 3, n)]
    flags = np.zeros(n, np.int32)
    flags[0] = flags[n // 2] = 1
    return {"offsets": np.array(cuts + [T], np.int32), "rank": ranks, "scale": (32.0 / ranks).astype(np.float32),
            "flags": flags, "n": n}


def _prepare_grads(case, seed):
    g = _generator(seed)
    T, d_in, d_out, R = case["T"], case["d_in"], case["d_out"], case["R"]

    def normal(rows, cols, std):
        return (torch.randn(rows, cols, device="cuda", generator=g) * std).to(torch.bfloat16)
    s = {"case": case, "X": normal(T, d_in, 1.0), "dY": normal(T, d_out, 1.0 / T), "A": normal(d_in, R, d_in ** -0.5),
         "B": normal(R, d_out, R ** -0.5)}
    tab = _table(case, seed)
    s["n_chunks"] = tab["n"]
    for k in ("offsets", "rank", "scale", "flags"):
        s[k] = torch.from_numpy(tab[k]).cuda()
    if own:
        from paper_2601_21109_b200 import binding as cwl
        s["table"] = cwl.DeviceChunkTable.from_host(tab["offsets"], tab["rank"], tab["scale"], tab["flags"])
        s["workspace"] = torch.empty(cwl.cwl_apply_grads_workspace_bytes(T, d_in, d_out, R), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    return {"logprobs": _prepare_logprobs, "distill": _prepare_distill, "grads": _prepare_grads}[case["op"]](case, seed)


# ------------------------------------------------------------------------------------------------------- plain forms
def _plain_logprobs(s):
    z, k, tau = s["logits"].float(), s["case"]["top_k"], s["case"]["temperature"]
    m = z.amax(1, keepdim=True)
    d = (z - m) / tau
    e = torch.exp(d)
    total = e.sum(1)
    log_total = torch.log(total)
    out = {"lse": m[:, 0] / tau + log_total,
           "entropy": log_total - torch.where(e > 0, d * e, 0.0).sum(1) / total}
    if s["targets"] is not None:
        out["logprob"] = d.gather(1, s["targets"].long()[:, None])[:, 0] - log_total
    if k:
        # one whole number for (value, lower index first), so that equal values come in the order of their indices
        bits = (z + 0.0).view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
        V = z.shape[1]
        key = (order << 32) + (V - 1 - torch.arange(V, device=z.device))
        ids = V - 1 - (key.topk(k, dim=1).values & 0xFFFFFFFF)
        out["top_ids"] = ids.to(torch.int32)
        out["top_logprobs"] = d.gather(1, ids) - log_total[:, None]
    return out


def _plain_distill(s):
    case, z, w = s["case"], s["logits"].float(), s["weight"]
    tau = case["temperature"]
    valid, ids = s["ids"] >= 0, s["ids"].clamp(min=0).long()
    d = (z - z.amax(1, keepdim=True)) / tau
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    q = e / total
    if case["teacher"] == "logits":
        u = torch.where(valid, s["values"] / tau, float("-inf"))
        u = u - u.amax(1, keepdim=True)
        p = torch.exp(u)
        log_p = u - torch.log(p.sum(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
        p_tail = torch.zeros_like(w)
    else:
        log_p = s["values"]
        p = torch.where(valid, torch.exp(log_p), 0.0)
        p_tail = (1.0 - p.sum(1)).clamp(min=0.0)
    inside = torch.zeros_like(z).scatter_add_(1, ids, valid.float()) > 0
    q_tail = torch.where(inside, 0.0, q).sum(1)
    out = {}
    if case["direction"] != "grad":
        log_q = d.gather(1, ids) - torch.log(total)
        kl = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
        kl = kl + torch.where(p_tail > 0, p_tail * (torch.log(p_tail) - torch.log(q_tail)), 0.0)
        out["loss"] = torch.where(w != 0, w * tau * tau * kl, 0.0)
    if case["direction"] != "loss":
        up = w * tau if s["dloss"] is None else w * tau * s["dloss"]
        c = p.sum(1) + p_tail
        outside = c - torch.where(p_tail > 0, p_tail / q_tail, 0.0)
        grad = q * torch.where(inside, c[:, None], outside[:, None])
        grad.scatter_add_(1, ids, -p)
        out["dlogits"] = torch.where((w != 0)[:, None], grad * up[:, None], 0.0).to(s["logits"].dtype)
    return out


def _plain_gate(s):
    """The weight of every (row, rank index): rank mask, scale, and the cross-fade of the rows after a join."""
    case = s["case"]
    t = torch.arange(case["T"], device="cuda", dtype=torch.int32)
    c = torch.searchsorted(s["offsets"], t, right=True) - 1
    before = (c - 1).clamp(min=0)
    j = (t - s["offsets"][c]).float()
    blend = (c > 0) & ((s["flags"][c] & 1) == 0) & (j < case["window"])
    lam = torch.where(blend, (j + 1) / (case["window"] + 1), 1.0)
    idx = torch.arange(case["R"], device="cuda")[None]
    return ((lam * s["scale"][c])[:, None] * (idx < s["rank"][c][:, None])
            + ((1 - lam) * s["scale"][before])[:, None] * (idx < s["rank"][before][:, None]))


def _plain_grads(s):
    X, dY, A, B = s["X"].float(), s["dY"].float(), s["A"].float(), s["B"].float()
    g = _plain_gate(s)
    dB = (g * (X @ A)).t() @ dY
    dA = X.t() @ (g * (dY @ B.t()))
    return {"dA": dA.to(torch.bfloat16), "dB": dB.to(torch.bfloat16)}


# -------------------------------------------------------------------------------------------------------- own calls
def _own_logprobs(s):
    from paper_2601_21109_b200 import binding as cwl
    o = cwl.cwl_token_logprobs(s["logits"], s["targets"], top_k=s["case"]["top_k"], temperature=s["case"]["temperature"],
                               out=s["out"])
    out = {"lse": o.lse, "entropy": o.entropy}
    if s["targets"] is not None:
        out["logprob"] = o.logprob
    if s["case"]["top_k"]:
        out["top_ids"], out["top_logprobs"] = o.top_ids, o.top_logprobs
    return out


def _own_distill(s):
    from paper_2601_21109_b200 import binding as cwl
    case = s["case"]
    loss, dlogits = cwl.cwl_distill_topk(s["logits"], s["ids"], s["values"], teacher=case["teacher"],
                                         temperature=case["temperature"], weight=s["weight"], dloss=s["dloss"],
                                         want_loss=case["direction"] != "grad", want_grad=case["direction"] != "loss")
    out = {}
    if loss is not None:
        out["loss"] = loss
    if dlogits is not None:
        out["dlogits"] = dlogits
    return out


def _own_grads(s):
    from paper_2601_21109_b200 import binding as cwl
    dA, dB = cwl.cwl_apply_grads(s["X"], s["dY"], s["A"], s["B"], s["table"], s["case"]["window"], workspace=s["workspace"])
    return {"dA": dA, "dB": dB}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"logprobs": _own_logprobs, "distill": _own_distill, "grads": _own_grads}[op](state)
    return {"logprobs": _plain_logprobs, "distill": _plain_distill, "grads": _plain_grads}[op](state)


# ----------------------------------------------------------------------------------------- the definitions in 64 bits
def _exact_logprobs(s):
    case = s["case"]
    lse, ent, lp, top = [], [], [], []
    for r in range(0, case["T"], 1024):
        logp = torch.log_softmax(s["logits"][r:r + 1024].double() / case["temperature"], 1)
        lse.append(torch.logsumexp(s["logits"][r:r + 1024].double() / case["temperature"], 1))
        ent.append(-torch.special.xlogy(logp.exp(), logp.exp()).sum(1))
        if s["targets"] is not None:
            lp.append(logp.gather(1, s["targets"][r:r + 1024].long()[:, None])[:, 0])
        if case["top_k"]:
            top.append(logp.topk(case["top_k"], dim=1).values)
    out = {"lse": torch.cat(lse), "entropy": torch.cat(ent)}
    if lp:
        out["logprob"] = torch.cat(lp)
    if top:
        out["top_ids"], out["top_logprobs"] = None, torch.cat(top)
    return out


def _exact_distill(s):
    case, tau = s["case"], s["case"]["temperature"]
    losses, grads = [], []
    for r in range(0, case["T"], 1024):
        part = slice(r, r + 1024)
        z = s["logits"][part].double() / tau
        logq = torch.log_softmax(z, 1)
        ids, real = s["ids"][part].long(), s["ids"][part] >= 0
        u = s["values"][part].double()
        if case["teacher"] == "logits":
            p = torch.softmax((u / tau).masked_fill(~real, float("-inf")), 1)
        else:
            p = u.exp().masked_fill(~real, 0.0)
        # the teacher as a whole row; the sink takes the entries that are padding
        whole = torch.zeros(z.shape[0], case["V"] + 1, dtype=torch.float64, device=z.device)
        whole.scatter_(1, ids.masked_fill(~real, case["V"]), p)
        held = torch.zeros_like(whole, dtype=torch.bool).scatter_(1, ids.masked_fill(~real, case["V"]), True)[:, :-1]
        whole = whole[:, :-1]
        rest = (1.0 - p.sum(1)).clamp(min=0.0) if case["teacher"] == "logprobs" else torch.zeros(z.shape[0], dtype=torch.float64, device=z.device)
        log_rest_q = torch.logsumexp(logq.masked_fill(held, float("-inf")), 1)
        w = s["weight"][part].double()
        if case["direction"] != "grad":
            kl = (torch.special.xlogy(whole, whole) - torch.where(whole > 0, whole * logq, 0.0)).sum(1)
            kl = kl + torch.special.xlogy(rest, rest) - torch.where(rest > 0, rest * log_rest_q, 0.0)
            losses.append(torch.where(w == 0, 0.0, w * tau ** 2 * kl))
        if case["direction"] != "loss":
            share = torch.where(held, 0.0, (logq - log_rest_q[:, None]).exp()) * rest[:, None]
            d = logq.exp() * (p.sum(1) + rest)[:, None] - whole - share
            up = w if s["dloss"] is None else w * s["dloss"][part].double()
            grads.append(torch.where((w == 0)[:, None], 0.0, d) * (up * tau)[:, None])
    out = {}
    if losses:
        out["loss"] = torch.cat(losses)
    if grads:
        out["dlogits"] = torch.cat(grads)
    return out


def _exact_grads(s):
    case = s["case"]
    off, rank, scale, flags = (s[k].cpu().numpy() for k in ("offsets", "rank", "scale", "flags"))
    gate = np.zeros((case["T"], case["R"]))
    for c in range(s["n_chunks"]):
        for t in range(off[c], off[c + 1]):
            lam = 1.0
            if c > 0 and not flags[c] & 1 and t - off[c] < case["window"]:
                lam = (t - off[c] + 1) / (case["window"] + 1)
                gate[t, :rank[c - 1]] += (1.0 - lam) * float(scale[c - 1])
            gate[t, :rank[c]] += lam * float(scale[c])
    gate = torch.from_numpy(gate).cuda()
    X, dY = s["X"].double(), s["dY"].double()
    H = gate * torch.matmul(X, s["A"].double())
    G = gate * torch.matmul(dY, s["B"].double().T)
    return {"dA": torch.matmul(X.T, G), "dB": torch.matmul(H.T, dY)}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"logprobs": _exact_logprobs, "distill": _exact_distill, "grads": _exact_grads}[case["op"]](s)
