"""GPU tests of the token log probabilities (include/mv_lm.h) over the whole range of logits and scales, against 64 bits.

Bounds.  u = 2^-24.  With m a row's largest z = scale * x and D = z - m <= 0, the kernel's exponent of a term, in base 2, is the sum
of at most three distances (to a thread's reference, which may lag by 10, and from there to m), each rounded at most twice and
times a constant with two roundings: off by at most 4 u (2 |D| log2 e + 20), so a term by a relative 8 u |D| + 60 u.  Every
exponential adds 2^-22: the term's own, one per warp, CTA and cluster and one per 10 that a thread's reference climbed, at most
5 + |D| / 6 in all.  A sum of n terms adds n u (n: V / 32 and a tree).  None of this grows with |lse|: only lse itself has
the rounding of its own value."""
import math

import numpy as np
import pytest
import torch

from paper_2011_06495_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24
EX2 = 2.0 ** -22
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def in_range(magnitudes):
    """(type, magnitude) wherever the type reaches it."""
    return [(dt, m) for dt in (F32, BF16, F16) for m in magnitudes if m <= torch.finfo(dt).max]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def placed(x, offset=0, pad=0):
    """The same rows `offset` elements into a buffer, cols + pad apart."""
    buf = torch.zeros(offset + x.shape[0] * (x.shape[1] + pad) + 5, dtype=x.dtype, device=DEV)
    view = torch.as_strided(buf, x.shape, (x.shape[1] + pad, 1), offset)
    view.copy_(x)
    return view


def reference(x, targets, scale, k):
    """Values and bounds; rows of finite or -inf logits with one finite logit at least."""
    x = x.double().cpu()
    T, V = x.shape
    z = x * float(np.float32(scale))
    m = z.amax(1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    s = e.sum(1)
    ls = torch.log(s)
    lse = m[:, 0] + ls
    p = e / s[:, None]
    dz = torch.where(p > 0, d, torch.zeros_like(d))
    H = ls - (p * dz).sum(1)
    a = dz.abs()
    term = EX2 * (5 + a / 6) + U32 * (8 * a + 60)
    add = (V / 32 + 64) * U32
    rho = 1.01 * ((p * term).sum(1) + add)
    spread = (p * a).sum(1)
    tol_ls = rho + 4 * U32 * (ls + 1)
    tol_H = tol_ls + rho * spread + 1.01 * (p * (term * a + U32 * (16 * a + 100))).sum(1) + add * spread + 4 * U32 * (spread + 1)
    y = targets.long().cpu()
    dy = d.gather(1, y[:, None])[:, 0]
    lp = dy - ls
    off = lambda v: 4 * U32 * v.abs().nan_to_num(posinf=0)
    kk = min(k, V)
    order = np.lexsort((np.broadcast_to(np.arange(V), (T, V)), -(x.numpy() + 0.0)), axis=1)[:, :kk]
    ids = torch.full((T, k), -1, dtype=torch.int64)
    ids[:, :kk] = torch.from_numpy(np.ascontiguousarray(order))
    top = torch.full((T, k), -math.inf, dtype=torch.float64)
    top[:, :kk] = d.gather(1, ids[:, :kk]) - ls[:, None]
    return {"lse": (lse, tol_ls + 2 * U32 * lse.abs()), "entropy": (H, tol_H), "logprob": (lp, tol_ls + off(dy) + off(lp)),
            "top": (top, tol_ls[:, None] + 2 * off(top)), "ids": ids}


def call(x, targets, scale, k):
    T = x.shape[0]
    o = {n: torch.full((T,), -77.0, device=DEV) for n in ("logprob", "entropy", "lse")}
    o["top"], o["ids"] = torch.full((T, k), -77.0, device=DEV), torch.full((T, k), -77, dtype=torch.int32, device=DEV)
    B.mv_token_logprob(x, targets, scale=scale, logprob=o["logprob"], entropy=o["entropy"], lse=o["lse"], top_logprob=o["top"] if k else None,
                       top_id=o["ids"] if k else None)
    return o


def check(x, targets, scale, k=4, label=""):
    got, want = call(x, targets, scale, k), reference(x, targets, scale, k)
    assert torch.equal(got["ids"].long().cpu(), want["ids"]), label
    for n in ("lse", "entropy", "logprob", "top"):
        val, tol = want[n]
        val = torch.where(val.abs() > 3.402824e38, val * math.inf, val)          # beyond the range of 32 bits
        g = got[n].double().cpu()
        inf = torch.isinf(val)
        assert torch.equal(g[inf], val[inf]), (label, n)
        diff = (g - val).abs()
        bad = ~inf & ~(diff <= tol)                                              # (a NaN is bad)
        assert not bool(bad.any()), (label, n, bad.nonzero()[0].tolist(), float(g[bad][0]), float(val[bad][0]), float(tol[bad][0]))
    return got


def kinds(V, M, dt, g):
    """Eight rows of magnitude M: level, level with noise, masked by -M in part, and one logit of M."""
    x = torch.randn((8, V), generator=g, device=DEV) * 3.0
    x[0] = -M
    x[1] = M
    x[2] = x[2] - M
    x[3, : V // 2] = -M
    x[4, ::2] = -M
    x[5, 0] = -M
    x[6, V - 1] = -M
    x[7, V // 3] = M
    return x.to(dt)


@pytest.mark.parametrize("dt,M", in_range([1e2, 3e3, 1e4, 6e4, 1e5, 1e6, 1e7, 1e8, 1e9, 1e12, 1e30]))
@pytest.mark.parametrize("V,copies", [(9, 1), (1000, 1), (5003, 1), (20_011, 1), (700, 400), (20_011, 12)])
def test_logits_of_every_magnitude(dt, M, V, copies):
    """Alone, and as many as other divisions of the rows among threads take."""
    g = gen(V)
    x = kinds(V, M, dt, g)
    y = torch.randint(0, V, (8,), generator=g, device=DEV)
    for scale in (0.7, 1.0, 1.4):
        for offset, pad in ((0, 0), (1, 3)):
            first = check(placed(x, offset, pad), y, scale, 4, (scale, offset))
            if copies > 1:
                got = call(placed(x.repeat(copies, 1), offset, pad), y.repeat(copies), scale, 4)
                assert torch.equal(got["ids"], first["ids"].repeat(copies, 1))
                want = reference(x, y, scale, 4)
                for n in ("lse", "entropy", "logprob"):
                    val, tol = (w.repeat(copies) for w in want[n])
                    assert bool(((got[n].double().cpu() - val).abs() <= tol).all()), (n, scale, offset)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("scale", [1e-3, 30.0, 1e4, 1e5, 1e6, 1e7, 1e8, 1e20, 3e38])
@pytest.mark.parametrize("V", [9, 1000, 40_003])
def test_scales_of_every_magnitude(dt, scale, V):
    """An inverse temperature that leaves the largest logit alone, and what lies between it and an ordinary one."""
    g = gen(V)
    x = (torch.randn((6, V), generator=g, device=DEV) * 3.0).to(dt)
    x[1, V // 2] = 20.0
    x[2] = 1.25
    x[3, ::3] = -math.inf
    x[4] = torch.linspace(-8, 8, V, device=DEV).to(dt)
    x[5] = -x[5].abs()
    y = torch.randint(0, V, (6,), generator=g, device=DEV)
    for offset, pad in ((0, 0), (3, 1)):
        check(placed(x, offset, pad), y, scale, 4, offset)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("scale", [1e-39, 1e-36, 1e-33, 1e-30, 1e-20])
def test_very_small_scales_of_very_large_logits(dt, scale):
    """Logits over the whole range of 32 bits that a small scale brings back to ordinary ones; masked logits keep no share."""
    V = 3001
    g = gen(5)
    x = ((torch.rand((3, V), generator=g, device=DEV) * 2 - 1) * 1.6e38).to(dt)
    x[1, ::2] = -math.inf
    x[2, : V - 5] = -math.inf
    y = torch.randint(V - 5, V, (3,), generator=g, device=DEV)
    check(x, y, scale)


def test_parts_of_one_row_of_different_magnitudes():
    """A row divided among four CTAs, each of whose parts has a magnitude of its own."""
    V = 70_001
    for mags in ((-1e30, -1e9, 0.0, -1e4), (0.0, 1e9, 1e9 + 64, -1e9), (-1e9, -1e9, -1e9, -1e9 + 640), (2e5, 1e5, -1e5, -2e5)):
        x = torch.randn((1, V), generator=gen(1), device=DEV)
        for i, v in enumerate(mags):
            x[0, i * (V // 4): (i + 1) * (V // 4)] += v
        for dt in (F32, BF16):
            check(x.to(dt), torch.tensor([V // 2], device=DEV), 1.0, 20, mags)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("scale", [0.5, 0.3, 1e-3, 1e-37])
@pytest.mark.parametrize("V", [2, 700, 30_001])
def test_logits_at_opposite_ends_of_the_range(dt, scale, V):
    """Their difference passes the range of 32 bits, but not their log probabilities."""
    x = torch.randn((2, V), generator=gen(V), device=DEV)
    x[:, 0], x[0, V - 1], x[1, V // 2] = 3.2e38, -3.2e38, -3.3e38
    check(x.to(dt), torch.tensor([V - 1, V // 2], device=DEV), scale, min(V, 30))


# ------------------------------------------------------------------------------------------ gradient

def grad_reference(x, y, scale, lse, H, g1, g2):
    """(value, bound) for the lse and entropy that the call is given, log p not above 0.  log p = scale x - lse is one rounding (u |log p|),
    times log2(e)/2 two more; p = q q doubles that and the exponential's 2^-22, and four products follow.  No term grows with |lse|."""
    x, l = x.double().cpu(), lse.double().cpu()[:, None]
    c = float(np.float32(scale))
    g1, g2, H, y = g1.double().cpu()[:, None], g2.double().cpu()[:, None], H.double().cpu()[:, None], y.long().cpu()
    lp = (x * c - l).clamp(max=0.0)
    p = torch.exp(lp)
    lp = torch.where(p > 0, lp, torch.zeros_like(lp))
    hot = torch.zeros_like(p)
    hot[torch.arange(x.shape[0]), y] = 1.0
    val = c * (g1 * (hot - p) - g2 * p * (lp + H))
    rel = 1.01 * (2 * EX2 + U32 * (4 * lp.abs() + 8))
    pmag = c * p * (g1.abs() + g2.abs() * (lp.abs() + H.abs()))
    tol = rel * pmag + 4 * U32 * c * g2.abs() * p * (lp.abs() + 1) + 4 * U32 * c * (g1.abs() * (hot + p) + g2.abs() * p * (lp.abs() + H.abs()))
    return val, tol + 2.0 ** -148 + 2.0 ** -126 * c * (g1.abs() + g2.abs() * (H.abs() + 100))


def within(got, want, tol):
    """Is got (of its own type) the rounding of a value in [want - tol, want + tol]?"""
    lo, hi = ((want + e).float().to(got.dtype).double() for e in (-tol, tol))
    g = got.double().cpu()
    return (g >= lo) & (g <= hi)


@pytest.mark.parametrize("dt,M", in_range([1e2, 1e4, 6e4, 1e6, 1e8, 1e9, 1e12, 1e30]))
@pytest.mark.parametrize("V", [9, 1000, 9001])
def test_logits_gradient_at_every_magnitude_and_place(dt, M, V):
    """Rows of every magnitude: right for the lse of the call, and the same bits wherever logits and gradient lie."""
    g = gen(V)
    x = kinds(V, M, dt, g)
    y = torch.randint(0, V, (8,), generator=g, device=DEV)
    g1, g2 = torch.randn(8, generator=g, device=DEV), torch.randn(8, generator=g, device=DEV)
    for scale in (1.0, 0.7, 1e3):
        o = call(x, y, scale, 0)
        want, tol = grad_reference(x, y, scale, o["lse"], o["entropy"], g1, g2)
        first = None
        for src, dst in (((0, 0), (0, 0)), ((1, 3), (1, 3)), ((1, 0), (0, 0)), ((3, 8), (2, 8)), ((0, 1), (0, 2))):
            dx = placed(torch.full_like(x, 7.0), *dst)
            B.mv_token_logprob_grad(placed(x, *src), y, o["lse"], g1, dx, scale=scale, entropy=o["entropy"], g_entropy=g2)
            bad = ~within(dx, want, tol)
            assert not bool(bad.any()), (scale, src, dst, bad.nonzero()[0].tolist(), float(dx[bad.to(DEV)][0]), float(want[bad][0]), float(tol[bad][0]))
            first = dx.clone() if first is None else first
            assert torch.equal(first, dx), (scale, src, dst)


@pytest.mark.parametrize("place", [(0, 0), (1, 3)])
def test_logits_gradient_of_large_upstream_gradients(place):
    """A loss scaled by 1e10: masked logits, at the row's ends and inside, have a gradient of 0, not 0 times infinity."""
    x = torch.randn((3, 301), generator=gen(3), device=DEV)
    x[:, :5] = -math.inf
    x[:, 100:140] = torch.finfo(F32).min
    x[:, -5:] = -math.inf
    y = torch.tensor([50, 60, 70], device=DEV)
    o = call(x, y, 1.0, 0)
    g1, g2 = torch.tensor([1e10, -3e20, 1e30], device=DEV), torch.tensor([-1e10, 1e20, 1e30], device=DEV)
    want, tol = grad_reference(x, y, 1.0, o["lse"], o["entropy"], g1, g2)
    dx = placed(torch.full_like(x, 7.0), *place)
    B.mv_token_logprob_grad(placed(x), y, o["lse"], g1, dx, entropy=o["entropy"], g_entropy=g2)
    assert bool(within(dx, want, tol).all()) and not bool(dx[:, :5].any()) and not bool(dx[:, 100:140].any()) and not bool(dx[:, -5:].any())
