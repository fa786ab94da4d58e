"""GPU tests of drawing tokens (include/mv_lm.h) against the definition in 64 bits on the host.

Tokens have to be equal.  Sums in 64 bits are off by at most 1e-11 of the row's sum on either side, so that a random u meets a border between two
of 10^5 tokens that the two place differently once in 10^6 rows or less; the seeds are fixed.  Where borders are met on purpose the weights are
powers of two or equal, and every sum is exact.  logprob: scale (x - max) less the log of a sum of V weights, each off by at most half of
2^-(61 - log2 V) of the largest one (V at least 1024); in 64 bits, rounded to 32 at the end."""
import math

import numpy as np
import pytest
import torch

from paper_2011_06495_b200 import binding as B
from tests.test_lm_operators import BF16, DEV, F16, F32, U32, gen, strided

pytestmark = pytest.mark.gpu


def reference(x, u, scale, top_k, top_p, min_p):
    """(token, logprob, how many tokens are kept) of one row."""
    x = x.double().cpu().numpy() + 0.0
    V = len(x)
    scale, top_p, min_p, u = (float(np.float32(v)) for v in (scale, top_p, min_p, u))
    if np.isnan(x).any() or (x == np.inf).any() or not (0 < scale < np.inf) or any(math.isnan(v) for v in (top_p, min_p, u)):
        return -1, math.nan, 0
    if np.isneginf(x).all():
        return -1, -math.inf, 0
    order = np.lexsort((np.arange(V), -x))
    k = V if top_k <= 0 else min(int(top_k), V)
    w = np.exp((x[order] - x[order[0]]) * scale)
    keep = np.arange(V) < k
    if top_p < 1:
        total = math.fsum(w[:k])
        before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
        keep &= (before < top_p * total) | (np.arange(V) == 0)
    keep &= (w >= min_p) | (np.arange(V) == 0)
    chosen = np.sort(order[keep])
    weight = np.zeros(V)
    weight[order] = np.where(w * 2.0 ** (62 - max(10, (V - 1).bit_length())) >= 1.0, w, 0.0)       # too light to be drawn
    run = np.cumsum(weight[chosen])
    goal = min(max(u, 0.0), 1.0) * run[-1]
    j = int(np.searchsorted(run, goal, side="right"))
    if j == len(chosen):
        j = int(np.nonzero(weight[chosen])[0][-1])
    return int(chosen[j]), math.log(weight[chosen[j]] / run[-1]), len(chosen)


def draw(x, u, scale=None, top_k=None, top_p=None, min_p=None, it=torch.int64):
    T = x.shape[0]
    as_row = lambda v, dt: None if v is None else (v if torch.is_tensor(v) else torch.full((T,), v, dtype=dt, device=DEV))
    token, lp = torch.full((T,), -77, dtype=it, device=DEV), torch.full((T,), 77.0, device=DEV)
    B.mv_sample(x, as_row(u, F32), token, scale=as_row(scale, F32), top_k=as_row(top_k, torch.int32), top_p=as_row(top_p, F32), min_p=as_row(min_p, F32), logprob=lp)
    return token, lp


def check(x, u, scale=None, top_k=None, top_p=None, min_p=None, it=torch.int64):
    token, lp = draw(x, u, scale, top_k, top_p, min_p, it)
    token, lp = token.tolist(), lp.double().tolist()
    pick = lambda v, t, d: d if v is None else float(v[t]) if torch.is_tensor(v) else v
    for t in range(x.shape[0]):
        want, wlp, kept = reference(x[t], pick(u, t, None), pick(scale, t, 1.0), pick(top_k, t, 0), pick(top_p, t, 1.0), pick(min_p, t, 0.0))
        at = (t, kept, pick(u, t, None), pick(scale, t, 1.0), pick(top_k, t, 0), pick(top_p, t, 1.0), pick(min_p, t, 0.0))
        assert token[t] == want, (at, token[t], want)
        if math.isnan(wlp) or math.isinf(wlp):
            assert (math.isnan(lp[t]) and math.isnan(wlp)) or lp[t] == wlp, at
        else:
            assert abs(lp[t] - wlp) <= 1.01 * U32 * abs(wlp) + 2.0 ** -61 * max(1024, x.shape[1]) ** 2 + 1e-12, (at, lp[t], wlp)
    return token


def head(T, V, dt, seed, width=64, pad=0, offset=0):
    """Rows as a model gives them: a body, and a head that holds little or nearly all of the mass."""
    x, _ = strided(T, V, dt, pad, offset, seed=seed)
    x.mul_(2.0)
    g = gen(seed + 1)
    n = max(1, min(width, V // 2))
    ids = torch.argsort(torch.rand((T, V), generator=g, device=DEV), dim=1)[:, :n]
    top = torch.empty((T, 1), device=DEV).uniform_(3.0, 16.0, generator=g)
    x.scatter_(1, ids, (top - 1.5 * torch.log1p(torch.arange(n, device=DEV)) + torch.randn((T, n), generator=g, device=DEV) * 0.2).to(dt))
    return x


SETTINGS = [(None, None, None, None), (1.0, 1, None, None), (0.7, 5, None, None), (1.3, 50, 0.9, None), (None, None, 0.9, None), (1.1, None, 0.5, 0.02), (0.8, None, None, 0.05), (1.0, 200, None, None),
            (2.0, None, 0.99, None), (0.5, 1000, 0.95, None), (0.3, None, 0.98, None), (1.0, 20, 0.8, 0.1), (1.0, 5000, None, 0.001)]


@pytest.mark.parametrize("T,V", [(1, 1), (3, 2), (5, 31), (2, 257), (7, 1000), (20, 4099), (3, 32_000), (2, 50_021), (1, 131_072), (2, 200_003), (160, 5001), (300, 700)])
@pytest.mark.parametrize("dt,pad,offset,it", [(F32, 0, 0, torch.int64), (BF16, 0, 0, torch.int32), (F16, 1, 3, torch.int64), (BF16, 3, 1, torch.int64), (F32, 5, 1, torch.int32)])
def test_draws(T, V, dt, pad, offset, it):
    x = head(T, V, dt, T + V, pad=pad, offset=offset)
    for j, s in enumerate(SETTINGS):
        check(x, torch.rand(T, generator=gen(j + V), device=DEV), *s, it=it)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("V", [40, 3000, 70_001])
def test_every_row_its_own_settings(dt, V):
    T = 96
    x = head(T, V, dt, V)
    g = gen(V)
    r = lambda choices, t: torch.tensor(choices, device=DEV, dtype=t)[torch.randint(0, len(choices), (T,), generator=g, device=DEV)]
    check(x, torch.rand(T, generator=g, device=DEV), r([0.1, 0.7, 1.0, 1.5, 40.0], F32), r([-1, 0, 1, 2, 40, 300, 2000, 10 ** 6], torch.int32), r([0.0, 0.1, 0.5, 0.9, 0.999, 1.0, 2.0, -1.0], F32),
          r([0.0, 0.01, 0.3, 1.0, -1.0, 1.5], F32))


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("V", [1, 9, 300, 5000, 70_001])
def test_masked_flat_and_extreme_rows(dt, V):
    low = torch.finfo(dt).min
    g = gen(V)
    x = (torch.randn((16, V), generator=g, device=DEV) * 3.0).to(dt)
    x[0] = -math.inf                                        # nothing left
    x[1] = -math.inf
    x[1, V // 2] = 2.0                                      # one left
    x[2] = low
    x[3, : V // 2] = low
    x[4] = 1.5                                              # flat
    x[5] = 0.0
    x[5, ::2] = -0.0                                        # zeros of both signs
    x[6] = torch.linspace(-9, 9, V, device=DEV).to(dt)
    x[7] = torch.linspace(9, -9, V, device=DEV).to(dt)
    x[8, torch.rand(V, generator=g, device=DEV) < 0.99] = -math.inf
    x[9, : V - 1] = -math.inf
    x[10, V // 3] = 80.0                                    # one takes all
    x[11] = torch.finfo(dt).max
    x[12] = torch.randint(0, 3, (V,), generator=g, device=DEV).to(dt)         # many ties
    x[13, V // 2] = math.nan
    x[14, V - 1] = math.inf
    x[15] = (torch.randint(0, 2, (V,), generator=g, device=DEV) * -50.0).to(dt)
    for j, s in enumerate(SETTINGS):
        for u in (0.0, 0.25, 0.61803, 1.0 - 2.0 ** -24):
            check(x, u, *s)
    for r in range(16):                                     # the rows one by one: a row's token does not depend on its neighbours
        check(x[r:r + 1], 0.4, 0.9, 30, 0.9, 0.01)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("V,offset", [(8, 0), (96, 3), (4096, 0), (65_536, 1)])
def test_exact_borders(dt, V, offset):
    """Equal weights and powers of two: u at a border draws the token behind it, top p at a border keeps what is before it."""
    x, _ = strided(4, V, dt, 0, offset, fill=1.5)
    for u in (0.0, 0.125, 0.25, 0.375, 0.5, 0.875, 1.0 - 2.0 ** -24):
        assert check(x, u)[0] == int(u * V)
        assert check(x, u, None, V // 2)[0] == int(u * (V // 2))
        assert check(x, u, None, None, 0.5)[0] == int(u * (V // 2))
        assert check(x, u, None, V // 2, 0.25)[0] == int(u * (V // 8))
    assert check(x, 1.0)[0] == V - 1 and check(x, -3.0)[0] == 0 and check(x, 7.0, None, 5)[0] == 4
    x[:, V // 2:] = -math.inf
    assert check(x, 1.0)[0] == V // 2 - 1                    # the last one that has a weight
    assert check(x, 0.5, None, V - 1)[0] == V // 4


def test_settings_and_u_that_are_no_numbers():
    x = torch.randn((8, 3000), generator=gen(1), device=DEV)
    u, scale, p, m = torch.full((8,), 0.5, device=DEV), torch.ones(8, device=DEV), torch.full((8,), 0.9, device=DEV), torch.zeros(8, device=DEV)
    u[0], scale[1], scale[2], scale[3], scale[4], p[5], m[6] = math.nan, math.nan, 0.0, -1.0, math.inf, math.nan, math.nan
    token, lp = draw(x, u, scale, None, p, m)
    assert token[:7].tolist() == [-1] * 7 and bool(torch.isnan(lp[:7]).all()) and int(token[7]) >= 0
    token2 = torch.zeros(8, dtype=torch.int32, device=DEV)
    B.mv_sample(x, u, token2, scale=scale, top_p=p, min_p=m)  # without logprob
    assert torch.equal(token2.long(), token)
    B.mv_sample(x[:0], u[:0], token2[:0])                    # no rows


@pytest.mark.parametrize("dt", [F32, BF16])
def test_extreme_scales(dt):
    x = head(6, 9001, dt, 3)
    for scale in (1e-38, 1e-6, 1e-2, 30.0, 1e5, 1e30, 3e38):
        for s in ((None, None, None), (50, 0.9, None), (None, 0.9, None), (None, None, 0.3)):
            check(x, torch.rand(6, generator=gen(int(scale < 1)), device=DEV), scale, *s)


def test_nuclei_of_every_size():
    """From one token to nearly all of them, on flat and steep rows."""
    V = 20_000
    for steep in (0.0, 1e-4, 1e-3, 0.02, 1.0):
        x = (-steep * torch.arange(V, device=DEV, dtype=F32))[torch.randperm(V, generator=gen(1), device=DEV)][None, :].repeat(12, 1)
        p = torch.tensor([1e-6, 1e-3, 0.01, 0.1, 0.3, 0.5, 0.7, 0.9, 0.99, 0.999, 0.99999, 1.0 - 2.0 ** -24], device=DEV)
        u = torch.rand(12, generator=gen(2), device=DEV)
        check(x, u, None, None, p)
        check(x.to(BF16), u, None, None, p)
        check(x, u, None, 10_000, p)
        k = torch.tensor([1, 2, 3, 31, 32, 33, 100, 500, 1000, 1025, 4000, 19_999], dtype=torch.int32, device=DEV)
        check(x, u, None, k)
        check(x.to(BF16), u, None, k, 0.999)
        check(x, u, None, None, None, p)


def test_top_p_that_ends_where_two_threads_bins_meet():
    """The count by bins of 1/128 of a power of two, 16 bins a thread, bounds the start from above and below: p as near as 32 bits come to each
    bound at every thread's border, in rows of one CTA and in rows that a cluster shares."""
    V, per, n = 40_960, 16, 120
    bins = np.random.default_rng(5).integers(0, 4000, V)
    step = 2.0 ** (-1 / 128)
    weight = np.bincount(bins, minlength=4096) * step ** np.arange(4096)
    most, least = np.cumsum(weight * (1 + 1e-4)), np.cumsum(weight * (1 + 1e-4) * step * (1 - 2e-4))
    at = np.arange(1, n + 1) * per - 1
    low, high = most[at] / (most[at] + least[-1] - least[at]), least[at] / (least[at] + most[-1] - most[at])
    p = torch.from_numpy(np.concatenate([low, high])).float().to(DEV)
    row = torch.from_numpy(-(bins + 0.5) * math.log(2) / 128).float().to(DEV)
    many = p.repeat(3)                                       # 720 rows: one CTA each
    u = torch.rand(len(p), generator=gen(8), device=DEV)
    token, lp = draw(row.repeat(len(many), 1), u.repeat(3), None, None, many)
    for j in range(0, len(p), 40):                           # 40 rows: eight CTAs each
        few = draw(row.repeat(40, 1), u[j:j + 40].contiguous(), None, None, p[j:j + 40].contiguous())
        for part in range(3):
            here = slice(part * len(p) + j, part * len(p) + j + 40)
            assert torch.equal(few[0], token[here]) and torch.equal(few[1], lp[here])
    some = slice(0, len(p), 17)
    check(row.repeat(len(p[some]), 1), u[some].contiguous(), None, None, p[some].contiguous())


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("V,offset", [(3001, 1), (60_000, 0), (131_072, 3), (200_003, 0)])
@pytest.mark.parametrize("mean,std", [(0.0, 2.0), (10.0, 2.0), (20.0, 0.5), (-30.0, 4.0), (0.0, 0.01)])
def test_crowds_of_equal_logits_at_the_cut(dt, V, offset, mean, std):
    """Logits far from zero have few distinct values in 16 bits: thousands of them lie at the cut, and the first ones by index stay.  The last row:
    16-bit values in 32 bits beside a few others."""
    x, _ = strided(3, V, dt, 2, offset, seed=V)
    x.mul_(std).add_(mean)
    x[2] = x[2].to(BF16).to(dt)
    x[2, ::97] += 0.01
    x[1, torch.rand(V, generator=gen(V), device=DEV) < 0.3] = -math.inf
    for j, s in enumerate([(None, None, 0.9, None), (0.7, None, 0.5, 0.2), (1.0, 2000, None, None), (1.1, V // 3, None, 0.01), (1.0, V - 10, None, None), (None, None, 0.995, None)]):
        check(x, torch.rand(3, generator=gen(j), device=DEV), *s)


def test_many_rows_with_crowds():
    """More rows than one wave, a CTA for each; and few long rows, shared by several."""
    for T, V in ((1300, 20_011), (5, 700_000), (3, 1_500_000)):
        x = (torch.randn((T, V), generator=gen(T), device=DEV) * 1.5 + 12.0).to(BF16)
        u = torch.rand(T, generator=gen(T + 1), device=DEV)
        p = torch.tensor([0.9, 1.0, 0.7], device=DEV).repeat(T)[:T].contiguous()
        k = torch.tensor([0, 0, 0, 3000], dtype=torch.int32, device=DEV).repeat(T)[:T].contiguous()
        rows = torch.tensor(sorted({0, 1, 2, 3, T // 2, T - 2, T - 1}), device=DEV).clamp(0, T - 1).unique()
        token, _ = draw(x, u, None, k, p)
        for r in rows.tolist():
            assert int(token[r]) == reference(x[r], float(u[r]), 1.0, int(k[r]), float(p[r]), 0.0)[0], (T, V, r)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("V", [2, 3000, 40_000, 131_072])
def test_logprob_of_a_nearly_sure_token_keeps_its_digits(dt, V):
    """A token that is ahead by 0.5 to 30: the rest beside it is a sum of whole numbers, each weight exact to 2e-14 and half of n / 2^61."""
    T = 48
    x = torch.randn((T, V), generator=gen(V), device=DEV)
    at = torch.randint(0, V, (T, 1), generator=gen(1), device=DEV)
    x.scatter_(1, at, x.amax(1, keepdim=True) + 0.5 + torch.arange(T, device=DEV)[:, None] * 0.625)
    x = (x - 4.37).to(dt)
    for scale, k in ((1.0, 0), (1.3, 0), (1.0, 40), (0.9, 1)):
        u = torch.full((T,), 0.5, device=DEV)
        token, lp = draw(x, u, scale, k)
        w = torch.sort(torch.exp((x.double() - x.double().amax(1, keepdim=True)) * float(np.float32(scale))), dim=1, descending=True)[0]
        w = w[:, :k] if k else w
        rest = w[:, 1:].sum(1).cpu()
        sure = (rest < 1) & (w[:, 0].cpu() == 1)
        n = 2.0 ** max(10, (V - 1).bit_length())
        want, got = -torch.log1p(rest), lp.double().cpu()
        assert int(sure.sum()) > T // 2
        off = 1.01 * U32 * want.abs() + 1e-13 * rest + w.shape[1] * n * 2.0 ** -62
        assert bool((((got - want).abs() <= off) | ~sure).all()) and bool((got <= 0).all())
        assert torch.equal(token.cpu()[sure], x.float().argmax(1).cpu()[sure])
        if k == 1:
            assert bool((got == 0).all()) and not bool(torch.signbit(got).any())


@pytest.mark.parametrize("dt,V,offset", [(F32, 1408, 1), (F16, 3200, 0), (BF16, 1152, 3), (BF16, 60_000, 0), (F16, 131_072, 1)])
def test_fewer_candidates_than_the_top_k_asks_for(dt, V, offset):
    """Short rows, and rows that are masked but for some tokens: fewer, as many and more than k, within the weights' range and outside it."""
    g = gen(V)
    T = 24
    x = strided(T, V, dt, 1, offset, seed=V)[0].mul_(2.5)
    for t, left in enumerate([1, 2, 49, 50, 51, 64, 120, 700, 1024, 1025, 1100, V] * 2):
        x[t].masked_fill_(torch.rand(V, generator=g, device=DEV).argsort().argsort() >= left, -math.inf)
    u = torch.rand(T, generator=g, device=DEV)
    for scale, k, p, mp in ((1.25, 50, 0.9, None), (1.0, 50, None, None), (1.0, 50, 0.95, 0.01), (9.0, 50, 0.999, None), (1.0, 1000, 0.9, None), (0.9, 1024, 0.97, None)):
        check(x, u, scale, k, p, mp)


@pytest.mark.parametrize("T,V", [(3, 131_072), (700, 5001)])
def test_results_in_the_place_of_u_and_of_settings(T, V):
    x = head(T, V, BF16, 9)
    u, k = torch.rand(T, generator=gen(10), device=DEV), torch.full((T,), 40, dtype=torch.int32, device=DEV)
    p = torch.full((T,), 0.95, device=DEV)
    for kk, pp in ((k, p), (None, p), (k, None), (None, None)):
        token, lp = draw(x, u, None, kk, pp, it=torch.int32)
        u2, k2 = u.clone(), k.clone()
        B.mv_sample(x, u2, k2, top_k=k2 if kk is not None else None, top_p=pp, logprob=u2)
        assert torch.equal(k2, token) and torch.equal(u2, lp)


def test_a_row_has_the_same_token_however_many_rows_there_are():
    """Two tokens, the lighter one behind the heavier, and u within 2e-14 of their border: the weights' last bits decide.  The two lie in one group of
    logits when four CTAs share the row, so that too many others come into the list and the row is sampled without it; in two groups when a CTA
    has the row for itself, and the list holds just these two."""
    V, first, second, far = 20_480, 1580 * 4, 2092 * 4, -6.0
    g = gen(12)
    found = []
    for _ in range(24):                                      # pairs whose border is as near to a u of 32 bits
        scale = torch.empty(1 << 24, device=DEV).uniform_(1.0, 2.0, generator=g)
        x = torch.empty(1 << 24, device=DEV).uniform_(-2.0, -0.1, generator=g)
        border = 1 / (1 + torch.exp(x.double() * scale.double()))
        u = border.float()
        near = (u.double() - border).abs() < 2e-14
        found.append(torch.stack([scale[near], x[near], u[near]]))
    scale, x, u = (t.contiguous() for t in torch.cat(found, 1))
    n = len(u)
    assert n >= 50
    rows = torch.full((n, V), far, device=DEV)
    rows[:, first], rows[:, second] = 0.0, x
    p = 1 - 2.0 ** -24
    times = 600 // n + 1                                     # more than 592 rows: one CTA each
    many = draw(rows.repeat(times, 1), u.repeat(times), scale.repeat(times), 2, p)
    assert bool(((many[0] == first) | (many[0] == second)).all())
    for t in range(n):
        one = draw(rows[t:t + 1], u[t:t + 1], scale[t:t + 1], 2, p)
        assert torch.equal(one[0], many[0][t:t + 1]) and torch.equal(one[1], many[1][t:t + 1]), (t, float(scale[t]), float(x[t]), float(u[t]))


def test_rows_alone_and_in_a_batch_at_other_places():
    """The same bytes for every setting, whichever path a row takes: heads, crowds of 16 bits, masks."""
    V = 33_000
    x = torch.cat([head(12, V, BF16, 77), (torch.randn((12, V), generator=gen(78), device=DEV) * 1.5 + 12.0).to(BF16)])
    x[::5, V // 3:] = -math.inf
    u = torch.rand(len(x), generator=gen(79), device=DEV)
    for s in SETTINGS + [(1.0, 50, 0.9, None), (1.0, 2000, 0.9, 0.05), (1.25, 50, None, None)]:
        many = draw(x.repeat(50, 1), u.repeat(50), *s)      # 1200 rows
        few = draw(x, u, *s)
        assert torch.equal(many[0][:len(x)], few[0]) and torch.equal(many[1][:len(x)], few[1])
        assert torch.equal(many[0][-len(x):], few[0]) and torch.equal(many[1][-len(x):], few[1])
        for t in range(0, len(x), 3):
            apart, _ = strided(1, V, BF16, 0, 3 + t, fill=0.0)
            apart.copy_(x[t:t + 1])
            one = draw(apart, u[t:t + 1], *s)
            assert torch.equal(one[0], few[0][t:t + 1]) and torch.equal(one[1], few[1][t:t + 1])


def test_frequencies_are_the_probabilities():
    """The same row with an even grid of u: every token as often as its share of the grid, to within one of the grid's steps."""
    T, V = 4096, 50
    row = torch.randn((1, V), generator=gen(7), device=DEV) * 2
    x = row.repeat(T, 1)
    token, _ = draw(x, (torch.arange(T, device=DEV) + 0.5) / T)
    share = torch.bincount(token, minlength=V).double().cpu() / T
    assert bool(((share - torch.softmax(row[0].double().cpu(), 0)).abs() <= 1.0 / T).all())


def test_past_32_bit_offsets():
    T, V = 33_000, 70_001                                   # 2.3e9 logits
    x = torch.full((T, V), -4.0, dtype=BF16, device=DEV)
    rows = torch.tensor([0, 30_677, 30_678, T - 1], device=DEV)
    x[rows] = (torch.randn((4, V), generator=gen(4), device=DEV) * 3).to(BF16)
    u = torch.rand(T, generator=gen(5), device=DEV)
    k, p = torch.zeros(T, dtype=torch.int32, device=DEV), torch.ones(T, device=DEV)
    k[rows[1]], p[rows[2]] = 7, 0.6
    token, _ = draw(x, u, None, k, p)
    for r in rows.tolist():
        assert int(token[r]) == reference(x[r], float(u[r]), 1.0, int(k[r]), float(p[r]), 0.0)[0]
    assert int(token[5]) == int(float(u[5]) * V)


def test_the_same_bytes_every_time_on_other_streams_and_replayed():
    T, V = 64, 30_011
    x = head(T, V, BF16, 5)
    u = torch.rand(T, generator=gen(6), device=DEV)
    p = torch.tensor([1.0, 0.9, 0.99, 0.5], device=DEV).repeat(T // 4)
    a, b = [(torch.zeros(T, dtype=torch.int64, device=DEV), torch.zeros(T, device=DEV)) for _ in range(2)]
    run = lambda o, stream=None: B.mv_sample(x, u, o[0], top_p=p, logprob=o[1], stream=stream)
    run(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(a)
    x.copy_(head(T, V, BF16, 50))
    u.copy_(torch.rand(T, generator=gen(60), device=DEV))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    run(b, st)
    st.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check(x, u, None, None, p)


def test_shapes_and_types_that_do_not_fit_are_refused():
    x, u, y = torch.zeros((4, 30), device=DEV), torch.zeros(4, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    bad = [
        lambda: B.mv_sample(x.double(), u, y),
        lambda: B.mv_sample(x.t(), u, y),
        lambda: B.mv_sample(x, u[:3], y),
        lambda: B.mv_sample(x, u.double(), y),
        lambda: B.mv_sample(x, u, y[:3]),
        lambda: B.mv_sample(x, u, u),
        lambda: B.mv_sample(x, None, y),
        lambda: B.mv_sample(x, u, y, top_k=y),
        lambda: B.mv_sample(x, u, y, top_p=u.half()),
        lambda: B.mv_sample(x, u, y, scale=u[:2]),
        lambda: B.mv_sample(x, u, y.cpu()),
    ]
    for i, f_ in enumerate(bad):
        with pytest.raises((B.MvError, AttributeError)):
            f_()
            pytest.fail(f"refusal {i} did not come")
    torch.cuda.synchronize()
