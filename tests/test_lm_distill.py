"""GPU tests of the distillation from a teacher's alternatives and its gradient (include/mv_lm.h) against plain statements in 64 bits.

Tolerances, with u = 2^-24: a term 2^t is off by 2^-22 of itself and, through its argument, by 4 u |t| ln 2; a sum of V such terms by
(V / 32 + 64) u, since at least 32 lanes share a row.  The divergence is a sum over q_j of differences of logs, each log off by 4 u of
itself and by what its sum is off.  p in the gradient: the exponential and the roundings of its argument, as for the logits' gradient."""
import math

import numpy as np
import pytest
import torch

from paper_2011_06495_b200 import binding as B
from tests.test_lm_operators import BF16, DEV, EX2, F16, F32, U32, close, gen, strided, within

pytestmark = pytest.mark.gpu


def teacher(top, ids, V, rest):
    """q, r, M, the valid entries and the rows that have a teacher, in 64 bits."""
    a, ids = top.double().cpu(), ids.long().cpu()
    valid = (ids >= 0) & (ids < V)
    a = a.masked_fill(~valid, -math.inf)
    any_ = (valid & (rest | (a != -math.inf))).any(1)
    if rest:
        q = torch.exp(a)
        r = torch.where(any_, (1 - q.sum(1)).clamp(min=0), torch.zeros(len(a), dtype=torch.float64))
        return q, r, q.sum(1) + r, valid, any_
    q = torch.softmax(torch.where(any_[:, None], a, torch.zeros_like(a)), 1)
    q = torch.where(any_[:, None], q, torch.zeros_like(q))
    return q, torch.zeros(len(a), dtype=torch.float64), torch.ones(len(a), dtype=torch.float64), valid, any_


def listed_columns(ids, valid, V):
    mark = torch.zeros((ids.shape[0], V + 1), dtype=torch.bool)
    return mark.scatter_(1, torch.where(valid, ids.long().cpu(), torch.full_like(ids.long().cpu(), V)), True)[:, :V]


def forward_reference(x, top, ids, scale, rest):
    """{name: (value, bound)} of rows of finite or -inf logits and finite or -inf alternatives."""
    x = x.double().cpu()
    T, V = x.shape
    z = x * float(np.float32(scale))
    q, r, M, valid, any_ = teacher(top, ids, V, rest)
    m = z.amax(1, keepdim=True)
    empty = torch.isinf(m[:, 0])
    d = torch.where(torch.isinf(z), torch.full_like(z, -math.inf), z - m.nan_to_num(neginf=0))
    e = torch.exp(d)
    s = e.sum(1)
    ls = torch.log(s)
    lse = torch.where(empty, torch.full_like(s, -math.inf), m[:, 0] + ls)
    dz = torch.where(e > 0, d.abs(), torch.zeros_like(d))
    add = (V / 32 + 64) * U32
    rho = torch.where(empty, torch.zeros_like(s), 1.01 * (EX2 + add + 4 * U32 * (e * dz).sum(1) / s.clamp(min=1e-300)))
    tol_lse = rho + 4 * U32 * (m[:, 0].abs().nan_to_num(posinf=0) + ls.abs().nan_to_num(posinf=0) + 1)
    er = e.masked_fill(listed_columns(ids, valid, V), 0.0)
    sr = er.sum(1)
    log_rest = torch.where(empty, torch.full_like(s, -math.inf), torch.log(sr) - ls.nan_to_num(neginf=0))
    rho_r = 1.01 * (EX2 + add + 4 * U32 * torch.where(sr > 0, (er * dz).sum(1) / sr.clamp(min=1e-300), torch.zeros_like(s))) + rho
    # a sum below the range of 32 bits beside the largest term: absolute
    tol_r = rho_r + 4 * U32 * log_rest.abs().nan_to_num(posinf=0) + torch.where(sr > 0, V * 2.0 ** -126 / sr.clamp(min=1e-300), torch.zeros_like(s))
    logq = torch.log(q)
    logp = torch.gather(d, 1, torch.where(valid, ids.long().cpu(), torch.zeros_like(ids.long().cpu()))) - ls.nan_to_num(neginf=0)[:, None]
    live = q > 0
    kl = torch.where(live, q * (logq - logp), torch.zeros_like(q)).sum(1) + torch.where(r > 0, r * (torch.log(r) - log_rest), torch.zeros_like(r))
    kl = torch.where(any_, torch.where(empty, torch.full_like(kl, math.inf), kl), torch.zeros_like(kl))
    fin = lambda v: v.abs().nan_to_num(posinf=0, nan=0)
    mag = torch.where(live, q * (fin(logq) + fin(logp) + fin(ls)[:, None] + 1), torch.zeros_like(q)).sum(1)
    tol = M * rho + 4 * U32 * mag + torch.where(r > 0, r * (fin(tol_r) + 4 * U32 * (fin(torch.log(r)) + fin(log_rest) + 1)), torch.zeros_like(r)) + 2 * U32 * fin(kl) + 2.0 ** -149
    out = {"kl": (kl, tol), "lse": (lse, tol_lse)}
    if rest:
        out["log_rest"] = (log_rest, tol_r)
    return out


def call(x, top, ids, scale, rest):
    T = x.shape[0]
    o = {n: torch.full((T,), -77.0, device=DEV) for n in ("kl", "lse") + (("log_rest",) if rest else ())}
    B.mv_distill(x, top, ids, scale=scale, **o)
    return o


def check_forward(x, top, ids, scale=1.0, rest=True):
    got, want = call(x, top, ids, scale, rest), forward_reference(x, top, ids, scale, rest)
    for n in want:
        close(got[n], want[n], n)
    return got


def gradient_reference(x, top, ids, scale, lse, log_rest, g):
    x, l, g = x.double().cpu(), lse.double().cpu()[:, None], g.double().cpu()
    T, V = x.shape
    c = float(np.float32(scale))
    q, r, M, valid, any_ = teacher(top, ids, V, log_rest is not None)
    lr = log_rest.double().cpu() if log_rest is not None else torch.zeros(T, dtype=torch.float64)
    ratio = torch.where(r > 0, torch.where(torch.isinf(lr), M, torch.exp(torch.log(r) - lr)), torch.zeros_like(r))
    none = ~any_ | (g == 0) | torch.isinf(l[:, 0])
    lp = torch.where(none[:, None], torch.full_like(x, -math.inf), (x * c - l).clamp(max=0.0))
    p = torch.exp(lp)
    mark = listed_columns(ids, valid, V)
    qs = torch.zeros((T, V + 1), dtype=torch.float64).scatter_add_(1, torch.where(valid, ids.long().cpu(), torch.full_like(ids.long().cpu(), V)), q)[:, :V]
    f = torch.where(none, torch.zeros_like(g), c * g)
    val = f[:, None] * torch.where(mark, M[:, None] * p - qs, (M - ratio)[:, None] * p)
    arg = U32 * (2 * (x * c).abs().nan_to_num(posinf=0, neginf=0) + 4 * lp.abs().nan_to_num(posinf=0) + l.abs().nan_to_num(posinf=0, neginf=0))
    rel = 1.01 * (EX2 + arg) + 4 * U32
    e_ratio = 4 * U32 * ratio * (1 + torch.log(r.clamp(min=1e-300)).abs() + lr.abs().nan_to_num(posinf=0))
    tol = f.abs()[:, None] * torch.where(mark, M[:, None] * p * rel + 4 * U32 * (M[:, None] * p + qs), p * ((M - ratio).abs()[:, None] * rel + (e_ratio + 4 * U32 * (M + ratio))[:, None]))
    return val, tol + U32 * val.abs() + 2.0 ** -149 + 2.0 ** -126 * f.abs()[:, None] * (M + ratio)[:, None]


def check_gradient(x, top, ids, scale=1.0, rest=True, pad=0, inplace=False, seed=0, forward=None):
    T, V = x.shape
    o = forward or call(x, top, ids, scale, rest)
    g = torch.randn(T, generator=gen(seed), device=DEV)
    g[::5] = 0.0
    want, tol = gradient_reference(x, top, ids, scale, o["lse"], o.get("log_rest"), g)
    if inplace:
        dx, buf, keep = x.clone(), None, x
        B.mv_distill_grad(dx, top, ids, o["lse"], g, dx, scale=scale, log_rest=o.get("log_rest"))
    else:
        dx, buf = strided(T, V, x.dtype, pad, pad, fill=7.0)
        B.mv_distill_grad(x, top, ids, o["lse"], g, dx, scale=scale, log_rest=o.get("log_rest"))
        mask = torch.ones_like(buf, dtype=torch.bool)
        torch.as_strided(mask, dx.shape, dx.stride(), dx.storage_offset()).fill_(False)
        assert bool((buf[mask] == 7.0).all())
    bad = ~within(dx, want, tol)
    assert not bool(bad.any()), (int(bad.sum()), float((dx.double().cpu() - want)[bad].abs().max()), bad.nonzero()[0].tolist())
    return dx


def case(T, V, k, dt, it=torch.int32, pad=0, offset=0, seed=0, duplicates=False):
    """Logits, and a teacher whose alternatives hold little or nearly all of its mass; some rows have fewer of them, some none."""
    x, _ = strided(T, V, dt, pad, offset, seed=seed + T + V)
    x.mul_(2.5)
    g = gen(seed + 1)
    if duplicates or k > V:
        ids = torch.randint(0, V, (T, k), generator=g, device=DEV)
    else:
        ids = (torch.randint(0, V, (T, 1), generator=g, device=DEV) + torch.randint(1, max(2, V // k), (T, 1), generator=g, device=DEV) * torch.arange(k, device=DEV)) % V
    z = torch.sort(torch.randn((T, k), generator=g, device=DEV) * 3, dim=1, descending=True).values
    inside = torch.empty((T, 1), device=DEV).uniform_(0.0, 1.0, generator=g) ** 0.3
    top = torch.log_softmax(z, 1) + torch.log(inside)
    x.scatter_(1, ids, (z + 4.0).to(dt))
    ids[torch.rand((T, k), generator=g, device=DEV) < 0.1] = -1
    if T > 2:
        ids[1] = V                                          # no teacher
        top[2] = top[2] - torch.logsumexp(top[2], 0)        # all of the mass
    return x, top.contiguous(), ids.to(it)


SHAPES = [(1, 1, 1), (1, 2, 1), (4, 2, 2), (3, 31, 5), (2, 257, 64), (7, 1000, 1), (40, 1023, 20), (5, 4099, 33), (3, 32_000, 50), (1, 50_021, 5), (2, 131_072, 64), (1, 200_003, 1000), (700, 513, 8),
          (1500, 90, 3), (6, 70_000, 1024)]


@pytest.mark.parametrize("T,V,k", SHAPES)
@pytest.mark.parametrize("dt,it,pad,offset", [(F32, torch.int32, 0, 0), (BF16, torch.int64, 1, 0), (F16, torch.int64, 2, 3), (BF16, torch.int32, 0, 8)])
@pytest.mark.parametrize("rest", [True, False])
def test_divergence_and_gradient(T, V, k, dt, it, pad, offset, rest):
    x, top, ids = case(T, V, k, dt, it, pad, offset)
    scale = 1.0 if k % 2 else 0.5
    o = check_forward(x, top, ids, scale, rest)
    check_gradient(x, top, ids, scale, rest, pad=offset, forward=o)
    check_gradient(x, top, ids, scale, rest, inplace=True, forward=o)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("V", [9, 300, 5000, 70_001])
def test_masked_flat_and_extreme_rows(dt, rest, V):
    low, k = torch.finfo(dt).min, 6
    x, top, ids = case(16, V, k, dt, seed=V)
    ids = ids.clamp(min=0)
    x[0] = -math.inf                                        # nothing left
    x[1] = low
    x[2] = -math.inf
    x[2, ids[2].long()] = 1.0                               # nothing left outside the list
    x[3, ids[3, 0].long()] = -math.inf                      # an alternative is masked
    x[4] = 0.0
    x[5] = 1.5
    x[6, : V // 2] = low
    x[7, V // 3] = 80.0
    x[8] = torch.finfo(dt).max
    x[9] = -math.inf                                        # nothing left inside the list
    x[9, (int(ids[9].max()) + 1) % V] = 3.0
    top[10] = -math.inf                                     # alternatives without mass
    top[11, 1:] = -math.inf
    top[12] = 0.0                                           # more than all of the mass
    top[13] = -80.0                                         # hardly any
    top[14, 0], top[14, 1:] = 0.0, -100.0
    ids[15] = ids[15, 0]                                    # the same token again and again
    for scale in (1.0, 0.3):
        o = check_forward(x, top, ids, scale, rest)
        check_gradient(x, top, ids, scale, rest, forward=o)
    for r in (0, 2, 8, 12, 15):                             # a row's result does not depend on its neighbours
        one = call(x[r:r + 1], top[r:r + 1], ids[r:r + 1], 0.3, rest)
        check_gradient(x[r:r + 1], top[r:r + 1], ids[r:r + 1], 0.3, rest, forward=one, seed=3)


@pytest.mark.parametrize("rest", [True, False])
def test_the_same_token_more_than_once(rest):
    for k in (2, 40, 300):
        x, top, ids = case(20, 50, k, F32, duplicates=True, seed=k)
        check_gradient(x, top, ids, 0.7, rest, forward=check_forward(x, top, ids, 0.7, rest))


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("V,k", [(1, 1024), (2, 500), (12, 1024), (60, 1024), (7, 129)])
def test_long_lists_of_few_tokens(V, k, rest):
    """Hundreds of terms of one token: their sum is as exact as one term is, which is what the bound allows for."""
    for seed in range(3):
        x, top, ids = case(800, V, k, F32, duplicates=True, seed=seed)
        check_gradient(x, top, ids, 0.5, rest, seed=seed)


@pytest.mark.parametrize("magnitude,scale", [(1e2, 1.0), (1e4, 1.0), (1e9, 1.0), (1e30, 1.0), (1.0, 1e6), (1.0, 1e-6), (1e30, 1e-30), (1e38, 0.5)])
@pytest.mark.parametrize("rest", [True, False])
def test_magnitudes(magnitude, scale, rest):
    for dt in (F32, BF16):
        x = (torch.randn((6, 5003), generator=gen(2), device=DEV) * magnitude).clamp(-3e38, 3e38).to(dt)
        x[1] = x[1].abs()
        x[2] = -x[2].abs()
        x[3] = -magnitude
        _, top, ids = case(6, 5003, 9, dt)
        want = forward_reference(x, top, ids, scale, rest)
        got = call(x, top, ids, scale, rest)
        for n in want:
            close(got[n], want[n], n)
        check_gradient(x, top, ids, scale, rest, forward=got)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rest", [True, False])
def test_listed_tokens_that_are_masked_by_the_lowest_value(dt, rest):
    """scale x passes the range of 32 bits, q_j log p_j does not."""
    x, top, ids = case(6, 700, 5, dt, seed=11)
    ids = torch.arange(5, device=DEV, dtype=torch.int32).repeat(6, 1) * 97
    top = torch.log(torch.tensor([0.5, 0.2, 0.1, 0.05, 0.01], device=DEV)).repeat(6, 1)
    x[:, 291] = torch.finfo(dt).min                         # the fourth
    x[3, 388] = torch.finfo(dt).min                         # and the fifth
    x[4, 500] = torch.finfo(dt).max                         # everything else is as far away
    x[5, 0] = torch.finfo(dt).max
    for scale in (1.0, 4.0):
        want, got = forward_reference(x[:4], top[:4], ids[:4], scale, rest), call(x, top, ids, scale, rest)
        close(got["kl"][:4], want["kl"], "kl")
        assert float(got["kl"][:4].min()) > 1e37 * scale / 4
    if not rest:                                             # (with it, log P is -inf in the last rows)
        want = forward_reference(x[5:], top[5:], ids[5:], 1.0, rest)
        close(call(x[5:], top[5:], ids[5:], 1.0, rest)["kl"], want["kl"], "kl")


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("V,pad", [(40, 0), (9001, 1)])
@pytest.mark.parametrize("weight", [1.0, 1e4])
def test_students_that_leave_hardly_anything_to_the_rest(dt, V, pad, weight):
    """g r / P passes the range of 32 bits where log P is low, g p_v r / P does not: the gradient of the tokens outside the list, c g p (M - r / P), is
    at most c g r.  Its relative error: the exponential, the roundings of its argument log p - log P, and those of r / P."""
    T, k = 60, 4
    x = torch.randn((T, V), generator=gen(V), device=DEV)
    ids = (torch.arange(k, device=DEV, dtype=torch.int32) * 7).repeat(T, 1)
    ahead = torch.linspace(0.0, 86.0, T, device=DEV)[:, None]
    x.scatter_(1, ids.long(), ahead + 3.5 + torch.randn((T, k), generator=gen(1), device=DEV).abs())
    x = x.to(dt)
    top = torch.log(torch.tensor([0.5, 0.2, 0.1, 0.05], device=DEV)).repeat(T, 1)
    top[::3] += 0.1                                          # r a sixth, a sixteenth and 1e-7
    top[1::3] += math.log(0.9999999 / 0.85)
    o = call(x, top, ids, 1.0, True)
    assert float(o["log_rest"].min()) < -84                  # (-inf, where nothing of the rest is above 2^-126 of the largest: then the others are 0)
    g = torch.randn(T, generator=gen(2), device=DEV) * weight
    dx, _ = strided(T, V, dt, pad, pad, fill=7.0)
    B.mv_distill_grad(x, top, ids, o["lse"], g, dx, log_rest=o["log_rest"])
    q, r, M, valid, _ = teacher(top, ids, V, True)
    z, l, lr = x.double().cpu(), o["lse"].double().cpu()[:, None], o["log_rest"].double().cpu()[:, None]
    M, r, f = M[:, None], r[:, None], g.double().cpu()[:, None]
    r, lr = torch.where(torch.isinf(lr), 0.0, r), torch.where(torch.isinf(lr), 0.0, lr)
    M = torch.where(o["log_rest"].cpu()[:, None] == -math.inf, 0.0, M)
    want = f * (M * torch.exp(z - l) - r * torch.exp(z - l - lr))
    off = f.abs() * (M * torch.exp(z - l) + r * torch.exp(z - l - lr)) * (1.01 * EX2 + U32 * (2 * z.abs() + l.abs() + 8 * (z - l).abs() + 4 * torch.log(r.clamp(min=1e-300)).abs() + 8 * lr.abs() + 16))
    outside = ~listed_columns(ids, valid, V)
    assert bool(torch.isfinite(dx).all())
    assert bool((within(dx, want, off + 2.0 ** -125 * f.abs()) | ~outside).all())


def test_rows_with_nan_and_inf():
    for dt in (F32, BF16):
        for V in (5, 3000, 40_001):
            x, top, ids = case(8, V, 3, dt)
            ids = ids.clamp(min=0, max=V - 1)
            clean = call(x, top, ids, 1.0, True)
            x[1, V - 1], x[4, 0], top[6, 1], top[7, 0] = math.nan, math.inf, math.nan, math.inf
            got = call(x, top, ids, 1.0, True)
            for n in got:
                assert bool(torch.isnan(got[n][[1, 4]]).all()) and torch.equal(got[n][[0, 2, 3, 5]], clean[n][[0, 2, 3, 5]])
            assert bool(torch.isnan(got["kl"][[6, 7]]).all()) and torch.equal(got["lse"][6:], clean["lse"][6:])


def test_positions_without_a_teacher_are_zero_whatever_their_logits_hold():
    x, top, ids = case(6, 9001, 4, BF16)
    ids = ids.clamp(min=0)
    g = torch.ones(6, device=DEV)
    x[0], x[1], x[2], x[4] = math.nan, math.nan, math.inf, math.nan
    ids[0], g[1], ids[2] = -1, 0.0, 9001
    o = call(x, top, ids, 1.0, True)
    assert float(o["kl"][3]) > 0 and float(o["kl"][0]) == 0 and bool(torch.isnan(o["kl"][4])) and bool(torch.isnan(o["log_rest"][0]))
    dx = torch.full_like(x, 7.0)
    B.mv_distill_grad(x, top, ids, o["lse"], g, dx, log_rest=o["log_rest"])
    assert bool((dx[:3] == 0).all()) and bool((dx[3:] != 0).any(1).all())


@pytest.mark.parametrize("T,V,k,dt", [(40, 2000, 1, F32), (33, 30011, 8, BF16), (5, 131072, 64, F16)])
def test_log_rest_beside_a_light_list_is_as_exact_as_the_list_is(T, V, k, dt):
    """log P = log1p(-o / s), o the listed tokens' sum and s all: off by what o and s are off, 1.45 times as much of itself up to
    o = s / 2, and the function's own two units; nothing is lost where P is close to one."""
    x = (torch.randn((T, V), generator=gen(V), device=DEV) * 2).to(dt)
    ids = torch.stack([torch.randperm(V, generator=gen(i), device=DEV)[:k] for i in range(T)]).int()
    x.scatter_(1, ids.long(), -torch.linspace(0, 14, T, device=DEV)[:, None].expand(T, k).to(dt))
    got = call(x, torch.full((T, k), -9.0, device=DEV), ids, 1.0, True)["log_rest"]
    z = x.double().cpu()
    e = torch.exp(z - z.amax(1, keepdim=True))
    at = (z - z.amax(1, keepdim=True)).abs()
    own, s = torch.gather(e, 1, ids.long().cpu()).sum(1), e.sum(1)
    assert float((own / s).max()) < 0.5 and float((own / s).min()) < 1e-5
    rho = lambda v, d: EX2 + 4 * U32 * (v * d).sum(1) / v.sum(1)
    off = rho(torch.gather(e, 1, ids.long().cpu()), torch.gather(at, 1, ids.long().cpu())) + rho(e, at) + (V / 32 + 64) * U32 + 6 * U32
    assert bool(within(got, torch.log1p(-own / s), 1.5 * off * torch.log1p(-own / s).abs()).all())


def test_divergence_of_a_student_that_agrees_is_zero_and_so_is_its_gradient():
    """The teacher's own logits: kl is 0 up to its bound, and the alternatives are those that mv_token_logprob leaves."""
    T, V, k = 40, 6007, 32
    x = (torch.randn((T, V), generator=gen(1), device=DEV) * 3).to(BF16)
    top, ids = torch.empty((T, k), device=DEV), torch.empty((T, k), dtype=torch.int32, device=DEV)
    for scale in (1.0, 0.5):
        B.mv_token_logprob(x, scale=scale, top_logprob=top, top_id=ids)
        o = check_forward(x, top, ids, scale, True)
        assert float(o["kl"].abs().max()) < 1e-4
        check_gradient(x, top, ids, scale, True, forward=o)


def test_gradient_against_differences():
    """Central differences of the divergence in 64 bits, with a step of 1e-4."""
    x, top, ids = case(5, 23, 4, F32)
    for rest in (True, False):
        o = call(x, top, ids, 0.8, rest)
        g = torch.randn(5, generator=gen(3), device=DEV)
        dx = torch.empty_like(x)
        B.mv_distill_grad(x, top, ids, o["lse"], g, dx, scale=0.8, log_rest=o.get("log_rest"))
        f = lambda y: (forward_reference(y, top, ids, 0.8, rest)["kl"][0] * g.double().cpu()).sum()
        for t in range(5):
            for v in range(23):
                a, b = x.double().cpu(), x.double().cpu()
                a[t, v] += 1e-4
                b[t, v] -= 1e-4
                assert abs(float((f(a) - f(b)) / 2e-4) - float(dx[t, v])) < 1e-6


def test_outputs_may_be_left_out():
    x, top, ids = case(6, 999, 5, F32)
    full = call(x, top, ids, 1.0, True)
    for n in full:
        one = torch.empty(6, device=DEV)
        B.mv_distill(x, top, ids, rest=True, **{n: one})
        assert torch.equal(one, full[n])
    B.mv_distill(x[:0], top[:0], ids[:0], kl=one[:0])


def test_past_32_bit_offsets():
    T, V, k = 33_000, 70_001, 3                             # 2.3e9 logits
    x = torch.zeros((T, V), dtype=BF16, device=DEV)
    rows = torch.tensor([0, 30_677, 30_678, T - 1], device=DEV)
    x[rows] = torch.randn((4, V), generator=gen(4), device=DEV).to(BF16)
    ids = torch.tensor([0, 35_000, 70_000], device=DEV).repeat(T, 1)
    top = torch.log(torch.tensor([0.5, 0.3, 0.1], device=DEV)).repeat(T, 1)
    got = call(x, top, ids, 1.0, True)
    some = x[rows].clone()
    want = forward_reference(some, top[rows], ids[rows], 1.0, True)
    for n in want:
        close(got[n][rows], want[n], n)
    g = torch.ones(T, device=DEV)
    ref, tol = gradient_reference(some, top[rows], ids[rows], 1.0, got["lse"][rows], got["log_rest"][rows], g[rows])
    B.mv_distill_grad(x, top, ids, got["lse"], g, x, log_rest=got["log_rest"])
    assert bool(within(x[rows], ref, tol).all())
    assert abs(float(x[5, 0]) + 0.5 - 1 / V) <= 2.0 ** -9
    other = (1 - 0.1 / (1 - 3 / V)) / V                     # a flat student: p (M - r / P)
    assert bool(((x[7, 1:35_000].double() - other).abs() <= 2.0 ** -8 * other).all())


def test_the_same_bytes_every_time_on_other_streams_and_replayed():
    T, V, k = 300, 5000, 16
    x, top, ids = case(T, V, k, BF16)
    g = torch.randn(T, generator=gen(2), device=DEV)

    def run(o, stream=None):
        B.mv_distill(x, top, ids, scale=0.5, kl=o[0], lse=o[1], log_rest=o[2], stream=stream)
        B.mv_distill_grad(x, top, ids, o[1], g, o[3], scale=0.5, log_rest=o[2], stream=stream)

    a, b = [[torch.zeros(T, device=DEV) for _ in range(3)] + [torch.zeros((T, V), dtype=BF16, device=DEV)] for _ in range(2)]
    run(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(a)
    y, top2, ids2 = case(T, V, k, BF16, seed=9)
    x.copy_(y), top.copy_(top2), ids.copy_(ids2)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    run(b, st)
    st.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_shapes_and_types_that_do_not_fit_are_refused():
    x, top, ids = torch.zeros((4, 30), device=DEV), torch.zeros((4, 3), device=DEV), torch.zeros((4, 3), dtype=torch.int32, device=DEV)
    f = torch.zeros(4, device=DEV)
    bad = [
        lambda: B.mv_distill(x.double(), top, ids, kl=f),
        lambda: B.mv_distill(x, top.half(), ids, kl=f),
        lambda: B.mv_distill(x, top[:3], ids[:3], kl=f),
        lambda: B.mv_distill(x, top, ids[:, :2], kl=f),
        lambda: B.mv_distill(x, top, top, kl=f),
        lambda: B.mv_distill(x, top.t().contiguous().t(), ids, kl=f),
        lambda: B.mv_distill(x, top[:, :0], ids[:, :0], kl=f),
        lambda: B.mv_distill(x, torch.zeros((4, 1025), device=DEV), torch.zeros((4, 1025), dtype=torch.int32, device=DEV), kl=f),
        lambda: B.mv_distill(x, top, ids, scale=0.0, kl=f),
        lambda: B.mv_distill(x, top, ids, scale=math.inf, kl=f),
        lambda: B.mv_distill(x, top, ids, kl=f[:3]),
        lambda: B.mv_distill(x, top, ids, kl=f.half()),
        lambda: B.mv_distill(x, top, ids, log_rest=f, rest=False),
        lambda: B.mv_distill(x, top.cpu(), ids, kl=f),
        lambda: B.mv_distill_grad(x, top, ids, f, f, x.half()),
        lambda: B.mv_distill_grad(x, top, ids, None, f, x),
        lambda: B.mv_distill_grad(x, top, ids, f, None, x),
        lambda: B.mv_distill_grad(x[:3], top[:3], ids[:3], f[:3], f[:3], x[1:]),
        lambda: B.mv_distill_grad(x, top, ids, f, f, x[:, :29]),
        lambda: B.mv_distill_grad(torch.zeros((4, 3), device=DEV), top, ids, f, f, top),
    ]
    for i, f_ in enumerate(bad):
        with pytest.raises(B.MvError):
            f_()
            pytest.fail(f"refusal {i} did not come")
    torch.cuda.synchronize()
