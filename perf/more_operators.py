"""Cases of the language-model operators between the embedding and the loss: layer norm and its gradient, distillation from a
teacher's alternatives and its gradient, and drawing tokens from logits.

`run` computes a case either in plain torch operations (`own` false) or through the library (`own` true).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ID_TYPES = {"i32": torch.int32, "i64": torch.int64}
ID_SIZE = {"i32": 4, "i64": 8}
EPS = 1e-5

# settings of one request: inverse temperature, top k (0: all), top p, min p
SETTINGS = {
    "greedy": [(1.0, 1, 1.0, 0.0)],
    "plain": [(1.0, 0, 1.0, 0.0), (1.25, 0, 1.0, 0.0), (0.8, 0, 1.0, 0.0)],
    "chat": [(1.25, 50, 0.9, 0.0)],
    "nucleus": [(1.0, 0, 0.9, 0.0), (1.43, 0, 0.95, 0.0), (0.9, 0, 0.8, 0.0)],
    "serving": [(1.0, 0, 1.0, 0.0), (1.43, 50, 0.9, 0.0), (1.0, 1, 1.0, 0.0), (1.25, 0, 0.95, 0.0), (1.0, 0, 1.0, 0.05), (0.67, 0, 0.9, 0.02),
                (1.0, 200, 1.0, 0.0), (1.1, 20, 0.8, 0.1)],
}


def listed():
    return [
        # the final norm of one decoding step of a small batch: latency
        {"name": "norm_decode", "op": "norm", "T": 8, "D": 4096, "dtype": "bf16", "wtype": "bf16", "pad": 0, "offset": 0},
        # the final norm of a training micro-batch of 32 sequences of 2048 tokens, gains in 32 bits
        {"name": "norm_batch", "op": "norm", "T": 65536, "D": 2048, "dtype": "bf16", "wtype": "f32", "pad": 0, "offset": 0},
        # a short micro-batch: the sum over the rows is as long a chain as the rows themselves
        {"name": "norm_grad_short", "op": "norm_grad", "T": 2048, "D": 512, "dtype": "bf16", "wtype": "bf16", "pad": 0, "offset": 0},
        # odd sizes, gains and their gradient in the middle of a worker's row (only 4-byte aligned)
        {"name": "norm_grad_odd", "op": "norm_grad", "T": 8191, "D": 1001, "dtype": "f32", "wtype": "f32", "pad": 2, "offset": 1},
        # a whole micro-batch
        {"name": "norm_grad_batch", "op": "norm_grad", "T": 65536, "D": 2048, "dtype": "bf16", "wtype": "f32", "pad": 0, "offset": 0},
        # one ragged document in 32 bits, five stored alternatives made to sum to one
        {"name": "distill_document", "op": "distill", "T": 1003, "V": 50021, "dtype": "f32", "ids": "i32", "k": 5, "rest": False, "scale": 1.0, "pad": 3, "missing": 0.1},
        # a batch of documents, 32 alternatives and the rest of the teacher's distribution as one class, temperature 2
        {"name": "distill_batch", "op": "distill", "T": 8192, "V": 65536, "dtype": "bf16", "ids": "i32", "k": 32, "rest": True, "scale": 0.5, "pad": 0, "missing": 0.1},
        # the gradient of a short fp32 fine-tuning batch
        {"name": "distill_grad_short", "op": "distill_grad", "T": 500, "V": 32000, "dtype": "f32", "ids": "i64", "k": 20, "rest": False, "scale": 1.0, "pad": 0, "missing": 0.1},
        # the gradient of a batch over a large vocabulary
        {"name": "distill_grad_batch", "op": "distill_grad", "T": 4096, "V": 131072, "dtype": "bf16", "ids": "i32", "k": 64, "rest": True, "scale": 0.5, "pad": 0, "missing": 0.1},
        # the next token of one conversation
        {"name": "sample_decode", "op": "sample", "T": 1, "V": 131072, "dtype": "bf16", "settings": "chat", "pad": 0, "masked": 0.0, "u": 0.37},
        # a decoding step of a serving batch, every request with settings of its own
        {"name": "sample_serving", "op": "sample", "T": 256, "V": 131072, "dtype": "bf16", "settings": "serving", "pad": 0, "masked": 0.0, "u": -1.0},
        # rollouts from the whole distribution, odd vocabulary, logits in 32 bits, a third of it masked by a grammar
        {"name": "sample_rollouts", "op": "sample", "T": 1024, "V": 50021, "dtype": "f32", "settings": "plain", "pad": 3, "masked": 0.3, "u": -1.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: sizes spread over the logarithm of their ranges, at most as costly as the largest listed one."""
    op = rng.choice(["norm", "norm_grad", "distill", "distill_grad", "sample"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    size = SIZE[dtype]
    if op in ("norm", "norm_grad"):
        D = _log_int(rng, 64, 16384)
        if rng.random() < 0.6:
            D = max(64, D // 64 * 64)
        T = _log_int(rng, 1, max(2, min(65536, (1 << 28) // (D * size))))
        return {"op": op, "T": T, "D": D, "dtype": dtype, "wtype": rng.choice(["f32", dtype]), "pad": rng.choice([0, 0, 1, 8]), "offset": rng.choice([0, 0, 1, 3])}
    V = _log_int(rng, 1000, 200_000)
    if rng.random() < 0.5:
        V = V // 128 * 128 or 1000
    pad = rng.choice([0, 0, 1, 64])
    if op == "sample":
        T = _log_int(rng, 1, max(2, min(2048, (1 << 26) // V)))
        return {"op": op, "T": T, "V": V, "dtype": dtype, "settings": rng.choice(sorted(SETTINGS)), "pad": pad, "masked": rng.choice([0.0, 0.0, 0.3, 0.99]), "u": -1.0}
    T = _log_int(rng, 1, max(2, min(16384, (1 << 30) // (V * size))))
    return {"op": op, "T": T, "V": V, "dtype": dtype, "ids": rng.choice(["i32", "i64"]), "k": rng.choice([1, 5, 8, 20, 50, 100]), "rest": rng.random() < 0.5,
            "scale": rng.choice([1.0, 0.5, 0.7]), "pad": pad, "missing": rng.choice([0.0, 0.1, 0.5])}


# ---------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rows(T, n, pad, dtype, g):
    return torch.empty((T, n + pad), dtype=DTYPES[dtype], device=DEV).normal_(0.0, 1.0, generator=g)[:, :n]


def _hidden(case, g):
    """A residual stream: channels of different sizes and offsets, a few of them large."""
    T, D = case["T"], case["D"]
    x = _rows(T, D, case["pad"], case["dtype"], g)
    spread = torch.exp(torch.empty(D, device=DEV).normal_(0.0, 0.5, generator=g))
    spread[torch.randint(0, D, (max(1, D // 256),), generator=g, device=DEV)] *= 20.0
    x.mul_(spread.to(x.dtype)).add_(torch.empty(D, device=DEV).normal_(0.05, 0.2, generator=g).to(x.dtype))
    return x


def _parameter(case, mean, std, g):
    """A vector of D parameters that starts `offset` elements into a larger array."""
    row = torch.empty(case["offset"] + case["D"], device=DEV).normal_(mean, std, generator=g).to(DTYPES[case["wtype"]])
    return row[case["offset"]:]


def _ids(T, V, k, g):
    """k different ids for each of T rows: steps of a random width around the vocabulary, from a random start."""
    step = torch.randint(1, V // k, (T, 1), generator=g, device=DEV)
    first = torch.randint(0, V, (T, 1), generator=g, device=DEV)
    return (first + step * torch.arange(k, device=DEV)) % V


def _head(T, k, g):
    """Logits of a head of k tokens: 6 to 16 at the top, falling with the logarithm of the rank."""
    top = torch.empty((T, 1), device=DEV).uniform_(6.0, 16.0, generator=g)
    fall = torch.empty((T, 1), device=DEV).uniform_(0.7, 2.5, generator=g)
    return top - fall * torch.log1p(torch.arange(k, device=DEV, dtype=torch.float32)) + torch.empty((T, k), device=DEV).normal_(0.0, 0.2, generator=g)


def _distill_inputs(case, seed, s):
    T, V, k = case["T"], case["V"], case["k"]
    g = _gen(seed)
    x = _rows(T, V, case["pad"], case["dtype"], g)
    x.mul_(2.0)
    ids = _ids(T, V, k, g)
    head = _head(T, k, g)
    x.scatter_(1, ids, (head + torch.empty((T, k), device=DEV).normal_(0.0, 0.7, generator=g)).to(x.dtype))      # the student nearly agrees
    # the teacher's alternatives as log probabilities: its head and a body that holds some of the mass
    z = torch.sort(head * case["scale"], dim=1, descending=True).values
    body = torch.empty((T, 1), device=DEV).uniform_(-6.0, 1.0, generator=g)
    lse = torch.logsumexp(z, 1, keepdim=True)
    top = z - torch.logaddexp(lse, lse + body)
    none = torch.rand(T, generator=g, device=DEV) < case["missing"]                     # the prompt: positions without a teacher
    ids[none] = -1
    short = torch.rand(T, generator=g, device=DEV) < 0.1                                # fewer alternatives than k
    ids[:, (k + 1) // 2:][short] = -1
    s["x"], s["top"], s["ids"] = x, torch.where(ids < 0, torch.full_like(top, float("-inf")), top), ids.to(ID_TYPES[case["ids"]])
    return g


def prepare(case, seed):
    op = case["op"]
    s = {"case": case}
    if op in ("norm", "norm_grad"):
        g = _gen(seed)
        T, D = case["T"], case["D"]
        s["x"] = _hidden(case, g)
        s["weight"], s["bias"] = _parameter(case, 1.0, 0.2, g), _parameter(case, 0.0, 0.2, g)
        if op == "norm":
            s["y"] = torch.empty((T, D), dtype=s["x"].dtype, device=DEV)
            s["mean"], s["rstd"] = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        else:
            s["dy"] = _rows(T, D, 0, case["dtype"], g).mul_(1e-2)
            x = s["x"].float()                                                          # what the forward pass left
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
            del x
            s["dx"] = torch.empty((T, D), dtype=s["x"].dtype, device=DEV)
            row = torch.empty(case["offset"] + 2 * D, device=DEV)                       # a worker's row of the gradients
            s["dweight"], s["dbias"] = row[case["offset"]:case["offset"] + D], row[case["offset"] + D:]
    elif op in ("distill", "distill_grad"):
        g = _distill_inputs(case, seed, s)
        T = case["T"]
        if op == "distill":
            s["kl"], s["lse"] = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
            s["log_rest"] = torch.empty(T, device=DEV) if case["rest"] else None
        else:
            _, s["lse"], s["log_rest"] = (t.float() if t is not None else None for t in _distill_64(s))
            s["g"] = torch.empty(T, device=DEV).uniform_(0.5, 1.5, generator=g) / T
            s["dx"] = torch.empty((T, case["V"]), dtype=s["x"].dtype, device=DEV)
    else:
        g = _gen(seed)
        T, V = case["T"], case["V"]
        x = _rows(T, V, case["pad"], case["dtype"], g)
        x.mul_(2.0)
        if case["masked"]:
            x.masked_fill_((torch.rand(V, generator=g, device=DEV) < case["masked"])[None, :], float("-inf"))
        k = min(64, V // 2)
        x.scatter_(1, _ids(T, V, k, g), _head(T, k, g).to(x.dtype))
        s["x"] = x
        s["u"] = torch.rand(T, generator=g, device=DEV) if case["u"] < 0 else torch.full((T,), case["u"], device=DEV)
        rows = [SETTINGS[case["settings"]][t % len(SETTINGS[case["settings"]])] for t in range(T)]
        s["scale"] = torch.tensor([r[0] for r in rows], device=DEV)
        s["top_k"] = torch.tensor([r[1] for r in rows], dtype=torch.int32, device=DEV)
        s["top_p"], s["min_p"] = (torch.tensor([r[j] for r in rows], device=DEV) for j in (2, 3))
        s["token"], s["logprob"] = torch.empty(T, dtype=torch.int64, device=DEV), torch.empty(T, device=DEV)
    if own and op == "norm_grad":                          # the workspace that a program keeps
        from paper_2011_06495_b200 import binding as B
        s["workspace"] = torch.empty(B.layer_norm_grad_workspace_bytes(case["T"], case["D"]), dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------------- one pass

def run(s):
    return _library(s) if own else _plain(s)


def _library(s):
    from paper_2011_06495_b200 import binding as B
    case = s["case"]
    op = case["op"]
    if op == "norm":
        B.mv_layer_norm(s["x"], s["weight"], s["bias"], s["y"], eps=EPS, mean=s["mean"], rstd=s["rstd"])
        return [s["y"], s["mean"], s["rstd"]]
    if op == "norm_grad":
        B.mv_layer_norm_grad(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"], s["workspace"])
        return [s["dx"], s["dweight"], s["dbias"]]
    if op == "distill":
        B.mv_distill(s["x"], s["top"], s["ids"], scale=case["scale"], kl=s["kl"], lse=s["lse"], log_rest=s["log_rest"])
        return [s["kl"], s["lse"]] + ([s["log_rest"]] if case["rest"] else [])
    if op == "distill_grad":
        B.mv_distill_grad(s["x"], s["top"], s["ids"], s["lse"], s["g"], s["dx"], scale=case["scale"], log_rest=s["log_rest"])
        return s["dx"]
    B.mv_sample(s["x"], s["u"], s["token"], scale=s["scale"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], logprob=s["logprob"])
    return [s["token"], s["logprob"]]


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = torch.rsqrt((d * d).mean(1) + EPS)
        return [(d * rstd[:, None] * s["weight"].float() + s["bias"].float()).to(s["x"].dtype), mean, rstd]
    if op == "norm_grad":
        dy = s["dy"].float()
        xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        h = dy * s["weight"].float()
        dx = s["rstd"][:, None] * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
        return [dx.to(s["x"].dtype), (dy * xh).sum(0), dy.sum(0)]
    if op == "distill":
        kl, lse, log_rest = _plain_distill(s)
        return [kl, lse] + ([log_rest] if case["rest"] else [])
    if op == "distill_grad":
        return _plain_distill_grad(s)
    return _plain_sample(s)


def _teacher(s):
    """The teacher's probabilities of its alternatives, 0 where there is none, the rest of its mass and the rows that have a teacher."""
    ids = s["ids"].long()
    has = (ids >= 0) & (ids < s["case"]["V"])
    a = torch.where(has, s["top"], torch.full_like(s["top"], float("-inf")))
    any_ = has.any(1)
    if s["case"]["rest"]:
        q = torch.exp(a)
        rest = (1.0 - torch.exp(a.double()).sum(1)).clamp(min=0.0)                      # in 64 bits: a small difference
        return q, torch.where(any_, rest, torch.zeros_like(rest)).float(), any_, has, torch.where(has, ids, torch.zeros_like(ids))
    q = torch.exp(a - torch.where(any_, a.amax(1), torch.zeros_like(a[:, 0]))[:, None])
    q = q / q.sum(1, keepdim=True).clamp(min=1e-30)
    return q, None, any_, has, torch.where(has, ids, torch.zeros_like(ids))


def _listed_mask(s, has, ids):
    V = s["case"]["V"]
    mark = torch.zeros((ids.shape[0], V + 1), dtype=torch.bool, device=DEV)
    return mark.scatter_(1, torch.where(has, ids, torch.full_like(ids, V)), True)[:, :V]


def _plain_distill(s):
    q, rest, any_, has, ids = _teacher(s)
    z = s["x"].float() * s["case"]["scale"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    lse = m[:, 0] + torch.log(e.sum(1))
    zero = torch.zeros((), device=DEV)
    logp = z.gather(1, ids) - lse[:, None]
    kl = torch.where(q > 0, q * (torch.log(q) - logp), zero).sum(1)
    if rest is None:
        return kl, lse, None
    total = e.sum(1)
    log_rest = torch.log(e.masked_fill_(_listed_mask(s, has, ids), 0.0).sum(1) / total)
    return kl + torch.where(rest > 0, rest * (torch.log(rest) - log_rest), zero), lse, log_rest


def _plain_distill_grad(s):
    q, rest, any_, has, ids = _teacher(s)
    c = s["case"]["scale"]
    p = torch.exp(s["x"].float() * c - s["lse"][:, None])
    if rest is None:
        d = p
    else:
        total = q.sum(1) + rest
        other = total - torch.where(rest > 0, torch.exp(torch.log(rest) - s["log_rest"]), torch.zeros_like(rest))
        d = torch.where(_listed_mask(s, has, ids), p * total[:, None], p * other[:, None])
    d.scatter_add_(1, ids, -q)
    return (d * torch.where(any_, c * s["g"], torch.zeros_like(s["g"]))[:, None]).to(s["x"].dtype)


def _plain_sample(s):
    """In 64 bits: a border between two neighbouring tokens lies within 1e-6 of the sum of u times the sum every few rows."""
    x = s["x"].double()
    T, V = x.shape
    xs, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((x - xs[:, :1]) * s["scale"].double()[:, None])
    ws = w.gather(1, order)
    rank = torch.arange(V, device=DEV)
    k = torch.where((s["top_k"] <= 0) | (s["top_k"] > V), torch.full_like(s["top_k"], V), s["top_k"])
    ws = torch.where(rank < k[:, None], ws, torch.zeros((), dtype=torch.float64, device=DEV))
    before = torch.cumsum(ws, 1) - ws
    p = s["top_p"].double()
    keep = (before < (p * ws.sum(1))[:, None]) | (p >= 1.0)[:, None] | (rank == 0)
    keep &= ws >= s["min_p"].double()[:, None]
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, torch.zeros((), dtype=torch.float64, device=DEV)))
    run_ = torch.cumsum(kept, 1)
    token = (run_ <= (s["u"].double() * run_[:, -1])[:, None]).sum(1).clamp(max=V - 1)
    return [token, torch.log(kept.gather(1, token[:, None])[:, 0] / run_[:, -1]).float()]


# ---------------------------------------------------------------------------------------------------------- what a pass needs

def work(case):
    op, T, b = case["op"], case["T"], SIZE[case["dtype"]]
    if op == "norm":
        return {"bytes": 2 * T * case["D"] * b + 2 * case["D"] * SIZE[case["wtype"]] + 8 * T, "flops": 8 * T * case["D"]}
    if op == "norm_grad":
        return {"bytes": 3 * T * case["D"] * b + case["D"] * (SIZE[case["wtype"]] + 8) + 8 * T, "flops": 16 * T * case["D"]}
    V = case["V"]
    if op == "sample":
        return {"bytes": T * V * b + T * (4 * 5 + 12), "flops": 4 * T * V}
    stored = T * case["k"] * (4 + ID_SIZE[case["ids"]])
    if op == "distill":
        return {"bytes": T * V * b + stored + T * (12 if case["rest"] else 8), "flops": 5 * T * V}
    return {"bytes": 2 * T * V * b + stored + T * (12 if case["rest"] else 8), "flops": 5 * T * V}


# ---------------------------------------------------------------------------------------------------------- in 64 bits

def _distill_64(s):
    """(divergence, log sum, log of the student's mass outside the list) of the distillation in 64 bits, some rows at a time."""
    case = s["case"]
    V, c = case["V"], float(np.float32(case["scale"]))
    out = []
    rows = max(1, (1 << 26) // V)
    for a in range(0, case["T"], rows):
        z = s["x"][a:a + rows].double() * c
        lse = torch.logsumexp(z, 1)
        ids, top = s["ids"][a:a + rows].long(), s["top"][a:a + rows].double()
        valid = (ids >= 0) & (ids < V)
        top = top.masked_fill(~valid, -math.inf)
        if not case["rest"]:
            logq = torch.log_softmax(top.masked_fill(~valid.any(1, keepdim=True), 0.0), 1)
        else:
            logq = top
        logq = logq.masked_fill(~valid, -math.inf)
        at = ids.clamp(0, V - 1)
        logp = torch.gather(z, 1, at) - lse[:, None]
        q = torch.exp(logq)
        kl = (torch.special.xlogy(q, q) - torch.where(q > 0, q * logp, 0.0)).sum(1)
        log_rest = None
        if case["rest"]:
            r = torch.arange(z.shape[0], device=DEV)[:, None].expand_as(ids)[valid]
            z[r, at[valid]] = -math.inf
            log_rest = torch.logsumexp(z, 1) - lse
            rest = (1.0 - q.sum(1)).clamp(min=0.0) * valid.any(1)
            kl = kl + torch.special.xlogy(rest, rest) - torch.where(rest > 0, rest * log_rest, 0.0)
        out.append((kl, lse, log_rest))
    return [torch.cat([o[i] for o in out]) if out[0][i] is not None else None for i in range(3)]


def _sample_64(s):
    """One row after another on the host: the kept tokens by a stable sort of the logits, their weights summed in order."""
    x = s["x"].float().cpu().numpy()
    u, scale, top_k, top_p, min_p = (s[n].cpu().numpy() for n in ("u", "scale", "top_k", "top_p", "min_p"))
    out = np.empty(len(x))
    for t in range(len(x)):
        V = len(x[t])
        order = np.argsort(-x[t], kind="stable")
        if 0 < top_k[t] < V:
            order = order[:top_k[t]]
        z = (x[t][order].astype(np.float64) - float(x[t][order[0]])) * float(scale[t])
        w = np.exp(z)
        n = len(w)
        if top_p[t] < 1.0:
            n = max(1, 1 + int(np.searchsorted(np.cumsum(w), float(top_p[t]) * w.sum(), side="left")))
        n = min(n, max(1, int(np.count_nonzero(w >= float(min_p[t])))))
        by_id = np.argsort(order[:n], kind="stable")
        sums = np.cumsum(w[:n][by_id])
        j = min(n - 1, int(np.searchsorted(sums, float(u[t]) * sums[-1], side="right")))
        out[t] = np.log(w[:n][by_id][j] / sums[-1])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "sample":
        if case["T"] * case["V"] > 1 << 26:
            return None
        return [None, torch.from_numpy(_sample_64(s))]
    if op == "distill":
        return [t for t in _distill_64(s) if t is not None]
    if op == "distill_grad":
        c, V = float(np.float32(case["scale"])), case["V"]
        parts, rows = [], max(1, (1 << 26) // V)
        for a in range(0, case["T"], rows):
            p = torch.exp(s["x"][a:a + rows].double() * c - s["lse"][a:a + rows].double()[:, None])
            ids, top = s["ids"][a:a + rows].long(), s["top"][a:a + rows].double()
            valid = (ids >= 0) & (ids < V)
            q = torch.exp(top.masked_fill(~valid, -math.inf))
            if not case["rest"]:
                q = q / q.sum(1, keepdim=True).clamp(min=1e-300)
            r = torch.arange(p.shape[0], device=DEV)[:, None].expand_as(ids)[valid]
            at = ids[valid]
            if case["rest"]:
                rest = (1.0 - q.sum(1)).clamp(min=0.0)
                total = q.sum(1) + rest
                ratio = rest / torch.exp(s["log_rest"][a:a + rows].double())
                here = p[r, at] * total[r]
                p *= (total - ratio)[:, None]
                p[r, at] = here
            p.index_put_((r, at), -q[valid], accumulate=True)
            p *= (c * s["g"][a:a + rows].double() * valid.any(1))[:, None]
            parts.append(p.float())                        # the output has at most 32 bits
        return torch.cat(parts)
    weight, bias = s["weight"].double(), s["bias"].double()
    rows = max(1, (1 << 26) // case["D"])
    parts = []
    dw, db = torch.zeros_like(weight), torch.zeros_like(weight)
    for a in range(0, case["T"], rows):
        x = s["x"][a:a + rows].double()
        if op == "norm":
            var, mean = torch.var_mean(x, 1, unbiased=False)
            rstd = 1.0 / torch.sqrt(var + EPS)
            parts.append((((x - mean[:, None]) * rstd[:, None] * weight + bias).float(), mean, rstd))
        else:
            rstd = s["rstd"][a:a + rows].double()
            xh = (x - s["mean"][a:a + rows].double()[:, None]) * rstd[:, None]
            dy = s["dy"][a:a + rows].double()
            dw += torch.einsum("td,td->d", dy, xh)
            db += dy.sum(0)
            h = dy * weight
            m1, m2 = h.sum(1) / case["D"], torch.einsum("td,td->t", h, xh) / case["D"]
            parts.append((((h - m1[:, None] - xh * m2[:, None]) * rstd[:, None]).float(),))
    first = [torch.cat([p[i] for p in parts]) for i in range(len(parts[0]))]
    return first if op == "norm" else first + [dw, db]
