"""Cases of the language-model operators around the sparse step: embedding lookup and its gradient, token log
probabilities and their gradient, per-worker gradient norm with clipping into the workers' rows.

`run` computes a case either in plain torch operations in 32 bits (`own` false) or through the library (`own` true).
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ID_TYPES = {"i32": torch.int32, "i64": torch.int64}
ID_SIZE = {"i32": 4, "i64": 8}
RESNET18_D = 11_173_962


def listed():
    return [
        # the tokens of one decoding step of a small batch: a handful of rows, all latency
        {"name": "embed_decode", "op": "embed", "T": 8, "V": 32000, "D": 4096, "dtype": "bf16", "ids": "i64", "scale": 1.0},
        # a training micro-batch of 32 sequences of 2048 tokens, scaled by sqrt(D)
        {"name": "embed_batch", "op": "embed", "T": 65536, "V": 65536, "D": 2048, "dtype": "bf16", "ids": "i64", "scale": math.sqrt(2048.0)},
        # the table's gradient of a short micro-batch: most rows of the table stay zero
        {"name": "embed_grad_short", "op": "embed_grad", "T": 2048, "V": 32000, "D": 512, "dtype": "bf16", "ids": "i64", "scale": 1.0, "offset": 0},
        # odd sizes everywhere, the table in the middle of a worker's row (only 4-byte aligned)
        {"name": "embed_grad_odd", "op": "embed_grad", "T": 8191, "V": 50021, "D": 1001, "dtype": "f32", "ids": "i32", "scale": 31.6, "offset": 1},
        # a whole micro-batch into a large table
        {"name": "embed_grad_batch", "op": "embed_grad", "T": 65536, "V": 65536, "D": 2048, "dtype": "bf16", "ids": "i64", "scale": math.sqrt(2048.0), "offset": 0},
        # one decoded token with its alternatives, half of the vocabulary masked off by a grammar
        {"name": "logprob_decode", "op": "logprob", "T": 1, "V": 131072, "dtype": "bf16", "ids": "i64", "scale": 1.25, "k": 8, "pad": 0, "masked": 0.5},
        # scoring one ragged document in 32 bits: odd vocabulary, rows in a wider buffer
        {"name": "logprob_document", "op": "logprob", "T": 1003, "V": 50021, "dtype": "f32", "ids": "i32", "scale": 1.0, "k": 5, "pad": 3, "masked": 0.0},
        # scoring a batch of documents with 16 alternatives each
        {"name": "logprob_batch", "op": "logprob", "T": 8192, "V": 65536, "dtype": "bf16", "ids": "i64", "scale": 1.0, "k": 16, "pad": 0, "masked": 0.0},
        # the loss gradient of a short fp32 fine-tuning batch, a tenth of the positions without a target
        {"name": "logprob_grad_short", "op": "logprob_grad", "T": 500, "V": 32000, "dtype": "f32", "ids": "i64", "scale": 1.0, "pad": 0, "masked": 0.0, "entropy": False, "untargeted": 0.1},
        # a policy-gradient batch over a large vocabulary, with an entropy bonus
        {"name": "logprob_grad_batch", "op": "logprob_grad", "T": 4096, "V": 131072, "dtype": "bf16", "ids": "i64", "scale": 1.0, "pad": 0, "masked": 0.0, "entropy": True, "untargeted": 0.1},
        # one worker's small mixed model
        {"name": "clip_small", "op": "clip", "N": 1, "d": 300_011, "L": 30, "dtype": "bf16", "split": 7},
        # the framework's own headline size: ten workers, 62 ragged tensors each, one norm per worker
        {"name": "clip_workers", "op": "clip", "N": 10, "d": RESNET18_D, "L": 62, "dtype": "f32", "split": 2},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: sizes spread over the logarithm of their ranges, at most as costly as the largest listed one."""
    op = rng.choice(["embed", "embed_grad", "logprob", "logprob_grad", "clip"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    ids = rng.choice(["i32", "i64"])
    most = 1 << 30                                        # elements x bytes of the large operand
    size = SIZE[dtype]
    if op in ("embed", "embed_grad"):
        V, D = _log_int(rng, 500, 131072), _log_int(rng, 64, 5000)
        if rng.random() < 0.6:
            D = max(64, D // 64 * 64)
        V = min(V, most // (4 * D))
        T = _log_int(rng, 1, max(2, min(65536, most // (D * size))))
        c = {"op": op, "T": T, "V": V, "D": D, "dtype": dtype, "ids": ids, "scale": rng.choice([1.0, round(math.sqrt(D), 3)])}
        if op == "embed_grad":
            c["offset"] = rng.choice([0, 0, 1, 2, 3])
        return c
    if op in ("logprob", "logprob_grad"):
        V = _log_int(rng, 1000, 200_000)
        if rng.random() < 0.5:
            V = V // 128 * 128 or 1000
        T = _log_int(rng, 1, max(2, min(16384, most // (V * size))))
        c = {"op": op, "T": T, "V": V, "dtype": dtype, "ids": ids, "scale": rng.choice([1.0, 0.8, 1.4]),
             "pad": rng.choice([0, 0, 1, 64]), "masked": rng.choice([0.0, 0.0, 0.3])}
        if op == "logprob":
            c["k"] = rng.choice([0, 1, 5, 8, 20])
        else:
            c["entropy"], c["untargeted"] = rng.random() < 0.5, rng.choice([0.0, 0.1, 0.5])
        return c
    N = rng.choice([1, 2, 4, 8, 16])
    d = _log_int(rng, 10_000, 80_000_000 // N)
    return {"op": op, "N": N, "d": d, "L": min(_log_int(rng, 1, 200), d // 500), "dtype": dtype, "split": rng.randrange(1000)}


# ---------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _tokens(T, V, g):
    """Token ids as text has them: frequency falling about as 1 / rank, frequent tokens at low ids."""
    u = torch.rand(T, generator=g, device=DEV, dtype=torch.float64)
    a = 2.7
    return (a * ((V + a) / a) ** u - a).floor().clamp_(0, V - 1).to(torch.int64)      # inverse of the 1 / (rank + a) law


def _distinct(T, V):
    """How many different tokens T draws of _tokens hold, on average."""
    a = 2.7
    r = np.arange(V, dtype=np.float64)
    p = np.log((r + 1 + a) / (r + a)) / math.log((V + a) / a)
    return float((1.0 - (1.0 - p) ** T).sum())


def _sizes(case):
    """The tensors of one worker: L ragged sizes, proportional to 10^U(1.8, 6.4), that add up to d."""
    r = random.Random(case["split"])
    raw = [10.0 ** r.uniform(1.8, 6.4) for _ in range(case["L"])]
    total = sum(raw)
    n = [max(16, int(x * case["d"] / total)) for x in raw]
    n[n.index(max(n))] += case["d"] - sum(n)
    return n


def _logits(case, seed):
    T, V = case["T"], case["V"]
    g = _gen(seed)
    buf = torch.empty((T, V + case["pad"]), dtype=DTYPES[case["dtype"]], device=DEV).normal_(0.0, 2.5, generator=g)
    logits = buf[:, :V]
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    peak = torch.empty((T, 1), device=DEV).uniform_(4.0, 14.0, generator=g)           # a model mostly knows the next token
    logits.scatter_(1, targets[:, None], peak.to(logits.dtype))
    if case["masked"]:
        off = torch.rand(V, generator=g, device=DEV) < case["masked"]
        logits.masked_fill_(off[None, :], float("-inf"))
        logits.scatter_(1, targets[:, None], peak.to(logits.dtype))
    return logits, targets, g


def prepare(case, seed):
    op = case["op"]
    s = {"case": case}
    if op in ("embed", "embed_grad"):
        g = _gen(seed)
        T, V, D = case["T"], case["V"], case["D"]
        s["ids"] = _tokens(T, V, g).to(ID_TYPES[case["ids"]])
        dt = DTYPES[case["dtype"]]
        if op == "embed":
            s["weight"] = torch.empty((V, D), dtype=dt, device=DEV).normal_(0.0, 0.02, generator=g)
            s["out"] = torch.empty((T, D), dtype=dt, device=DEV)
        else:
            s["dout"] = torch.empty((T, D), dtype=dt, device=DEV).normal_(0.0, 1e-3, generator=g)
            row = torch.empty(case["offset"] + V * D, device=DEV)                     # a worker's row of the gradients
            s["dweight"] = row[case["offset"]:].view(V, D)
    elif op in ("logprob", "logprob_grad"):
        s["logits"], targets, g = _logits(case, seed)
        T = case["T"]
        if op == "logprob_grad":
            none = torch.rand(T, generator=g, device=DEV) < case["untargeted"]
            targets = torch.where(none, torch.full_like(targets, -100), targets)
            z = s["logits"].float() * case["scale"]                                   # what the forward pass left
            s["lse"] = torch.logsumexp(z, 1)
            p = torch.exp(z - s["lse"][:, None])
            s["entropy"] = s["lse"] - torch.where(p > 0, p * z, torch.zeros_like(p)).sum(1)
            del z, p
            s["g_logprob"] = torch.empty(T, device=DEV).normal_(0.0, 1.0, generator=g) / T
            s["g_entropy"] = torch.full((T,), 1e-2 / T, device=DEV) if case["entropy"] else None
            s["dlogits"] = torch.empty((T, case["V"]), dtype=s["logits"].dtype, device=DEV)
        else:
            k = case["k"]
            s["logprob"], s["ent"], s["lse"] = (torch.empty(T, device=DEV) for _ in range(3))
            s["top"] = torch.empty((T, k), device=DEV) if k else None
            s["top_id"] = torch.empty((T, k), dtype=torch.int32, device=DEV) if k else None
        s["targets"] = targets.to(ID_TYPES[case["ids"]])
    else:
        g = _gen(seed)
        N, d = case["N"], case["d"]
        r = random.Random(case["split"] + 1)
        sizes = _sizes(case)
        std = [10.0 ** r.uniform(-4, -1) for _ in sizes]
        s["tensors"] = [torch.empty(n, dtype=DTYPES[case["dtype"]], device=DEV).normal_(0.0, sd, generator=g) for _ in range(N) for n, sd in zip(sizes, std)]
        s["groups"] = [w for w in range(N) for _ in sizes]
        s["max_norm"] = 1.0
        s["rows"] = torch.empty((N, d), device=DEV)
        s["norms"] = torch.empty(N, device=DEV)
    if own:                                               # the workspace and the plan that a program keeps
        from paper_2011_06495_b200 import binding as B
        if op == "embed_grad":
            s["workspace"] = torch.empty(B.embed_grad_workspace_bytes(case["T"], case["V"], case["D"]), dtype=torch.uint8, device=DEV)
        elif op == "clip":
            s["plan"] = B.MvClip(s["tensors"], s["groups"])
    return s


# ---------------------------------------------------------------------------------------------------------- one pass

def run(s):
    return _library(s) if own else _plain(s)


def _library(s):
    from paper_2011_06495_b200 import binding as B
    case = s["case"]
    op = case["op"]
    if op == "embed":
        B.mv_embed(s["weight"], s["ids"], s["out"], scale=case["scale"])
        return s["out"]
    if op == "embed_grad":
        B.mv_embed_grad(s["dout"], s["ids"], s["dweight"], s["workspace"], scale=case["scale"])
        return s["dweight"]
    if op == "logprob":
        B.mv_token_logprob(s["logits"], s["targets"], scale=case["scale"], logprob=s["logprob"], entropy=s["ent"], lse=s["lse"],
                           top_logprob=s["top"], top_id=s["top_id"])
        return [s["logprob"], s["ent"], s["lse"]] + ([s["top"], s["top_id"]] if case["k"] else [])
    if op == "logprob_grad":
        B.mv_token_logprob_grad(s["logits"], s["targets"], s["lse"], s["g_logprob"], s["dlogits"], scale=case["scale"],
                                entropy=s["entropy"], g_entropy=s["g_entropy"])
        return s["dlogits"]
    s["plan"].mv_clip_pack(s["max_norm"], s["rows"], s["norms"])
    return [s["rows"], s["norms"]]


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "embed":
        return (s["weight"][s["ids"].long()].float() * case["scale"]).to(s["weight"].dtype)
    if op == "embed_grad":
        dw = torch.zeros((case["V"], case["D"]), device=DEV)
        return dw.index_add_(0, s["ids"].long(), s["dout"].float()).mul_(case["scale"])
    if op == "clip":
        rows = torch.cat([t.float() for t in s["tensors"]]).view(case["N"], case["d"])
        norms = torch.sqrt((rows * rows).sum(1))
        return [rows * (s["max_norm"] / torch.clamp(norms, min=s["max_norm"]))[:, None], norms]
    x = s["logits"].float()
    y = s["targets"].long()
    has = (y >= 0) & (y < case["V"])
    y = torch.where(has, y, torch.zeros_like(y))[:, None]
    z = x * case["scale"]
    zero = torch.zeros((), device=DEV)
    if op == "logprob":
        m = z.amax(1, keepdim=True)
        e = torch.exp(z - m)
        total = e.sum(1)
        lse = m[:, 0] + torch.log(total)
        ent = torch.log(total) - torch.where(e > 0, e * (z - m), zero).sum(1) / total
        lp = torch.where(has, z.gather(1, y)[:, 0] - lse, zero)
        if not case["k"]:
            return [lp, ent, lse]
        bits = (x + 0.0).view(torch.int32)                # + 0.0: the two zeros are one value
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = order * (1 << 32) + (case["V"] - 1 - torch.arange(case["V"], device=DEV))
        top = case["V"] - 1 - (torch.topk(key, case["k"], dim=1).values & 0xFFFFFFFF)
        return [lp, ent, lse, z.gather(1, top) - lse[:, None], top.int()]
    logp = z - s["lse"][:, None]
    p = torch.exp(logp)
    dz = -p * torch.where(has, s["g_logprob"], zero)[:, None]
    dz.scatter_add_(1, y, torch.where(has, s["g_logprob"], zero)[:, None])
    if s["g_entropy"] is not None:
        dz -= s["g_entropy"][:, None] * torch.where(p > 0, p * (logp + s["entropy"][:, None]), zero)
    return (dz * case["scale"]).to(s["logits"].dtype)


# ---------------------------------------------------------------------------------------------------------- what a pass needs

def work(case):
    op = case["op"]
    if op == "embed":
        T, V, D = case["T"], case["V"], case["D"]
        b = SIZE[case["dtype"]]
        return {"bytes": T * ID_SIZE[case["ids"]] + (T + _distinct(T, V)) * D * b, "flops": T * D}
    if op == "embed_grad":
        T, V, D = case["T"], case["V"], case["D"]
        return {"bytes": T * ID_SIZE[case["ids"]] + T * D * SIZE[case["dtype"]] + V * D * 4, "flops": T * D}
    if op == "clip":
        n = case["N"] * case["d"]
        return {"bytes": n * (SIZE[case["dtype"]] + 4) + 4 * case["N"], "flops": 3 * n}
    T, V, b = case["T"], case["V"], SIZE[case["dtype"]]
    if op == "logprob":
        return {"bytes": T * V * b + T * (ID_SIZE[case["ids"]] + 12 + 8 * case["k"]), "flops": 6 * T * V}
    return {"bytes": 2 * T * V * b + T * (ID_SIZE[case["ids"]] + 16), "flops": (8 if case["entropy"] else 4) * T * V}


# ---------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    c = np.float64(np.float32(case.get("scale", 1.0)))    # the scale is a 32-bit argument of the operators
    if op == "embed":
        return torch.index_select(s["weight"], 0, s["ids"].long()).double() * c
    if op == "embed_grad":
        out = torch.zeros((case["V"], case["D"]), dtype=torch.float64, device=DEV)
        out.index_put_((s["ids"].long(),), s["dout"].double() * c, accumulate=True)
        return out
    if op == "clip":
        rows, norms = [], []
        per = len(s["tensors"]) // case["N"]
        for n in range(case["N"]):
            ts = [t.double() for t in s["tensors"][n * per:(n + 1) * per]]
            norm = math.sqrt(math.fsum(float((t * t).sum()) for t in ts))
            rows.append(torch.cat(ts) * min(1.0, s["max_norm"] / norm))
            norms.append(norm)
        return [torch.stack(rows), torch.tensor(norms, dtype=torch.float64)]
    rows = max(1, (1 << 27) // case["V"])                 # a gigabyte of doubles at a time
    parts = []
    for a in range(0, case["T"], rows):
        x = s["logits"][a:a + rows].double() * c
        y = s["targets"][a:a + rows].long()
        has = (y >= 0) & (y < case["V"])
        r = torch.arange(x.shape[0], device=DEV)
        if op == "logprob":
            logp = torch.log_softmax(x, 1)
            lse = torch.logsumexp(x, 1)
            ent = -torch.special.xlogy(torch.exp(logp), torch.exp(logp)).sum(1)
            lp = torch.where(has, logp[r, y.clamp(0, case["V"] - 1)], torch.zeros_like(lse))
            top = torch.topk(logp, case["k"], dim=1).values if case["k"] else None
            parts.append((lp, ent, lse, top))
        else:
            logp = x - s["lse"][a:a + rows].double()[:, None]
            p = torch.exp(logp)
            gl = torch.where(has, s["g_logprob"][a:a + rows], torch.zeros_like(s["g_logprob"][a:a + rows])).double()
            dz = -gl[:, None] * p
            dz[r[has], y[has]] += gl[has]
            if s["g_entropy"] is not None:
                dz -= s["g_entropy"][a:a + rows].double()[:, None] * (torch.special.xlogy(p, p) + p * s["entropy"][a:a + rows].double()[:, None])
            parts.append((dz * c).float())                # the output has at most 32 bits
    if op == "logprob_grad":
        return torch.cat(parts)
    lp, ent, lse = (torch.cat([p[i] for p in parts]) for i in range(3))
    return [lp, ent, lse] + ([torch.cat([p[3] for p in parts]), None] if case["k"] else [])
