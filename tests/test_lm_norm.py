"""GPU tests of layer norm and its gradients (include/mv_lm.h) against plain statements in 64 bits.

Tolerances, with u = 2^-24 the rounding of 32 bits.  At least eight lanes share a row and each keeps two sums, so that no term of a sum over D
passes more than n = D / 16 + 16 additions: a sum is off by at most 1.01 n u sum|terms|.  Sums over rows are taken as in any order, 1.01 (T + 2) u sum|terms|.
mean: n u mean|x| and a division.  variance: its squares are exact to 3 u of themselves, the sum to n u, and a mean that is off by e adds
e^2.  rstd = 1 / sqrt(v + eps): half the relative error of v + eps, and 4 u for sum, root (an approximation of 2^-22 counts as 4 u) and
division.  A result of 16 bits has to be what some value inside the 32-bit tolerance rounds to."""
import math

import pytest
import torch

from paper_2011_06495_b200 import binding as B
from tests.test_lm_operators import BF16, DEV, F16, F32, U32, gen, strided, within

pytestmark = pytest.mark.gpu
EPS = 1e-5


def forward_reference(x, w, b, eps):
    """((y, tol), (mean, tol), (rstd, tol)) in 64 bits."""
    x = x.double().cpu()
    D = x.shape[1]
    n = D / 16 + 16
    w = w.double().cpu() if w is not None else torch.ones(D, dtype=torch.float64)
    b = b.double().cpu() if b is not None else torch.zeros(D, dtype=torch.float64)
    eps = float(torch.tensor(eps, dtype=torch.float32))
    mean = x.mean(1)
    e_mean = 1.01 * (n + 2) * U32 * x.abs().mean(1)
    d = x - mean[:, None]
    v = (d * d).mean(1)
    e_v = 1.01 * ((n + 5) * U32 * (v + 2 * e_mean * d.abs().mean(1)) + e_mean ** 2)
    rstd = 1 / torch.sqrt(v + eps)
    rel = 1.01 * (0.5 * e_v / (v + eps) + 4 * U32) + (e_v / (v + eps)) ** 2
    z = d * rstd[:, None]
    e_z = z.abs() * (rel[:, None] + 3 * U32) + (e_mean * rstd * (1 + rel))[:, None]
    y = z * w + b
    return (y, e_z * w.abs() + 2 * U32 * (z * w).abs() + 2 * U32 * y.abs() + 2.0 ** -149), (mean, e_mean + 2.0 ** -149), (rstd, rel * rstd)


def run_forward(x, w, b, eps=EPS, y=None):
    T = x.shape[0]
    y = torch.empty(x.shape, dtype=x.dtype, device=DEV) if y is None else y
    mean, rstd = torch.full((T,), -7.0, device=DEV), torch.full((T,), -7.0, device=DEV)
    B.mv_layer_norm(x, w, b, y, eps=eps, mean=mean, rstd=rstd)
    return y, mean, rstd


def check_forward(x, w, b, eps=EPS, y=None):
    src = x.clone()
    got = run_forward(x, w, b, eps, y)
    for g, (val, tol), what in zip(got, forward_reference(src, w, b, eps), ("y", "mean", "rstd")):
        bad = ~within(g, val, tol)
        assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[0].tolist(), float((g.double().cpu() - val)[bad].abs().max()))
    return got


def parameters(D, dt, offset=0, seed=0):
    buf = torch.randn(2 * D + offset + 3, generator=gen(seed), device=DEV).to(dt)
    return buf[offset:offset + D], buf[offset + D:offset + 2 * D]


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 8), (9, 33), (4, 64), (33, 100), (1, 255), (300, 256), (7, 1000), (70, 1001), (65, 1024), (8, 2048), (5, 4096), (2, 4104), (3, 5000),
          (2, 8192), (3, 10_007), (2, 16_384), (1, 40_000), (2, 70_001), (2000, 72), (1500, 513)]


@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("dt,wt,pad,offset", [(F32, F32, (0, 0), 0), (BF16, F32, (0, 0), 0), (BF16, BF16, (8, 8), 8), (F16, F16, (1, 3), 1), (BF16, BF16, (2, 2), 0), (F32, F32, (3, 1), 1),
                                              (F16, F32, (0, 0), 3)])
def test_rows(T, D, dt, wt, pad, offset):
    x, _ = strided(T, D, dt, pad[0], pad[1], seed=T + D)
    x.mul_(1.7).add_(torch.randn(D, generator=gen(D), device=DEV).to(dt))
    y, buf = strided(T, D, dt, pad[1], pad[0], fill=7.0)
    w, b = parameters(D, wt, offset, seed=D)
    check_forward(x, w, b, y=y)
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, y.shape, y.stride(), y.storage_offset()).fill_(False)
    assert bool((buf[mask] == 7.0).all())                   # nothing outside the rows is written


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("D", [8, 1001, 2048, 30_000])
def test_rows_without_parameters_in_place_and_far_from_zero(dt, D):
    x = torch.randn((6, D), generator=gen(D), device=DEV)
    x[1] = 3.0                                               # nothing but eps
    x[2] *= 1e-6
    x[3] = x[3] * 0.1 + 100.0                                # a mean a thousand times the spread
    x[4] *= 1e8
    x[5] = 0.0
    x = x.to(dt)
    w, b = parameters(D, F32)
    for ww, bb in ((None, None), (w, None), (None, b)):
        check_forward(x, ww, bb)
    y, mean, rstd = check_forward(x, w, b, eps=1e-3)
    z = x.clone()
    B.mv_layer_norm(z, w, b, z, eps=1e-3)                    # in place, without the statistics
    assert torch.equal(z, y)
    for r in range(6):                                       # a row's result does not depend on its neighbours
        assert torch.equal(run_forward(x[r:r + 1], w, b, 1e-3)[0], y[r:r + 1])


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("T,D", [(9000, 1001), (20_000, 77), (4000, 4099)])
def test_many_rows_in_place_off_the_boundaries(dt, T, D):
    """Neighbouring rows share sectors of memory, one of which is read while the other is written: the bytes are those of a call out of place."""
    x = torch.randn((T, D), generator=gen(D), device=DEV).to(dt)
    w, b = parameters(D, F32, 1)
    want = run_forward(x, w, b)
    for _ in range(3):
        z = x.clone()
        got = run_forward(z, w, b, y=z)
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("T,D", [(40, 1), (40, 7), (40, 64), (40, 1000), (40, 1001), (40, 2048), (40, 5000), (40, 16_383), (40, 30_000), (1300, 96), (1300, 1000), (1300, 1003)])
def test_means_that_are_large_beside_the_spread(dt, T, D):
    """Constant rows and a spread of 1e-4 of the mean.  A sum of D terms passes n additions at most: of few rows a lane holds D / 1024 pairs, or up to 32
    elements, and a warp's and a CTA's sums add 21 more; of many rows as above.  The first mean m is off by e0 = (n + 2) u mean|x|.
    What the second pass finds of that is off by e1 = (n + 4) u mean|x - m|, and so is the mean, beside its own rounding; the variance by
    (n + 7) u (v + e0^2) + 2 e0 e1 + e1^2; y by that of rstd, by e1 rstd, and by the roundings of x - m, of its product's sum and of e rstd."""
    g = gen(T + D)
    x = torch.randn((T, D), generator=g, device=DEV)
    x = torch.cat([x[::4] * 0 + 1000.0, x[1::4] * 0 + 3000.33, x[2::4] * 0.1 + 1000.0, x[3::4] * 0.01 + 100.0]).to(dt)
    w, b = parameters(D, F32)
    y, mean, rstd = run_forward(x, w, b)
    x, w, b = x.double().cpu(), w.double().cpu(), b.double().cpu()
    n = D / 16 + 16 if T > 1000 else min(D + 8, D / 256 + 48)
    mu, eps = x.mean(1), float(torch.tensor(EPS, dtype=torch.float32))
    d = x - mu[:, None]
    v, spread = (d * d).mean(1), d.abs().mean(1)
    e0 = 1.01 * (n + 2) * U32 * x.abs().mean(1)
    e1 = 1.01 * (n + 4) * U32 * (spread + e0)
    ev = 1.01 * ((n + 7) * U32 * (v + e0 ** 2) + 2 * e0 * e1 + e1 ** 2)
    r = 1 / torch.sqrt(v + eps)
    rel = 1.01 * (0.5 * ev / (v + eps) + 4 * U32) + (ev / (v + eps)) ** 2
    z = d * r[:, None]
    ez = 1.01 * (1 + rel[:, None]) * (z.abs() * (rel[:, None] + U32) + r[:, None] * (e1[:, None] + U32 * (d.abs() + 2 * e0[:, None])))
    want = z * w + b
    for got, value, off in ((y, want, ez * w.abs() + 2 * U32 * want.abs() + 2.0 ** -149), (mean, mu, e1 + 1.01 * U32 * mu.abs()), (rstd, r, rel * r)):
        assert bool(within(got, value, off).all()), float((got.double().cpu() - value).abs().max())


def test_rows_whose_squares_pass_the_range_of_32_bits():
    """rstd is 0 then, and y the bias, where sums of some of the terms, in any order, cannot pass the range too: that is where the magnitudes' sum does
    not (of +-1e38 in turn, four or more of either sign are inf together, and a row whose sums pass the range is nothing but the formula's)."""
    for D in (2, 64, 1001, 2048, 40_000):
        x = torch.randn((6, D), generator=gen(D), device=DEV) * 1e25
        x[0] = torch.where(torch.arange(D, device=DEV) % 2 == 0, 1e38, -1e38)
        b = torch.randn(D, generator=gen(1), device=DEV)
        y, mean, rstd = run_forward(x, None, b)
        fits = x.double().abs().sum(1) < 3e38
        assert bool(fits[1:].all()) and bool(fits[0]) == (D == 2)
        assert bool((rstd[fits] == 0).all()) and torch.equal(y[fits], b.expand_as(y)[fits]) and bool(torch.isfinite(mean[fits]).all())


@pytest.mark.parametrize("dt", [F32, BF16, F16])
def test_widths_at_the_limits_of_shared_memory(dt):
    """6129 to 6144 columns need just 48 KB for their parameters, beside a little static shared memory; the gradient gets there at widths that
    hang on the type and the alignment, so that every width up to 6200 has to be taken at least."""
    for T in (2, 1300):
        for D in (6128, 6129, 6136, 6143, 6144, 6145):
            x = torch.randn((T, D), generator=gen(D), device=DEV).to(dt)
            w, b = parameters(D, F32)
            check_forward(x[:20], w, b)
            y = run_forward(x, w, b)[0]
            assert torch.isfinite(y).all()
    stats, dw, db = torch.ones(1300, device=DEV), torch.empty(6200, device=DEV), torch.empty(6200, device=DEV)
    ws = torch.empty(max(B.layer_norm_grad_workspace_bytes(1300, D) for D in range(1, 6200)), dtype=torch.uint8, device=DEV)
    x = torch.zeros((1300, 6200), dtype=dt, device=DEV)
    for D in range(1, 6200):                                 # refused by the launch, if at all
        for T in (2, 1300) if D % 16 == 0 else (2,):
            B.mv_layer_norm_grad(x[:T, :D], x[:T, :D], None, stats[:T], stats[:T], None, dw[:D], db[:D], ws)
            B.mv_layer_norm(x[:T, :D], None, None, x[:T, :D])
    torch.cuda.synchronize()


def test_rows_with_nan_and_inf_leave_the_others_alone():
    for D in (5, 1024, 1001):
        x = torch.randn((40, D), generator=gen(D), device=DEV).to(BF16)
        clean = run_forward(x, None, None)
        x[7, D // 2], x[20, 0] = math.nan, math.inf
        got = run_forward(x, None, None)
        keep = torch.ones(40, dtype=torch.bool, device=DEV)
        keep[7] = keep[20] = False
        assert all(torch.equal(a[keep], c[keep]) for a, c in zip(got, clean))
        assert bool(torch.isnan(got[0][~keep]).all())


def grad_reference(dy, x, w, mean, rstd, old=None):
    """((dx, tol), (dweight, tol), (dbias, tol)) in 64 bits for the mean and rstd that the call is given."""
    dy, x, mean, rstd = (t.double().cpu() for t in (dy, x, mean, rstd))
    T, D = x.shape
    n = D / 16 + 16
    w = w.double().cpu() if w is not None else torch.ones(D, dtype=torch.float64)
    d = x - mean[:, None]
    z = d * rstd[:, None]
    h = dy * w
    s0, s1 = h.mean(1, keepdim=True), (h * z).mean(1, keepdim=True)
    dx = rstd[:, None] * (h - s0 - z * s1)
    e0, e1 = 1.01 * (n + 3) * U32 * h.abs().mean(1, keepdim=True), 1.01 * (n + 6) * U32 * (h * z).abs().mean(1, keepdim=True)
    tol = rstd[:, None] * (1.01 * (e0 + z.abs() * e1) + 6 * U32 * (h.abs() + s0.abs() + (z * s1).abs())) + 2.0 ** -149
    dw, db = (dy * z).sum(0), dy.sum(0)
    mw, mb = (dy * z).abs().sum(0), dy.abs().sum(0)
    if old is not None:
        dw, db, mw, mb = dw + old[0].double().cpu(), db + old[1].double().cpu(), mw + old[0].double().cpu().abs(), mb + old[1].double().cpu().abs()
    return (dx, tol), (dw, 1.01 * (T + 5) * U32 * mw + 2.0 ** -149), (db, 1.01 * (T + 2) * U32 * mb + 2.0 ** -149)


def check_grad(dy, x, w, dx=None, out=None, accumulate=False, statistics=None):
    T, D = x.shape
    if statistics is None:
        statistics = run_forward(x.clone(), w, None)[1:]
    mean, rstd = statistics
    dx = torch.full((T, D), -7.0, dtype=x.dtype, device=DEV) if dx is None else dx
    dw, db = (torch.full((D,), math.nan, device=DEV) for _ in range(2)) if out is None else out
    old = (dw.clone(), db.clone()) if accumulate else None
    want = grad_reference(dy.clone(), x.clone(), w, mean, rstd, old)
    ws = torch.full((B.layer_norm_grad_workspace_bytes(T, D),), 255, dtype=torch.uint8, device=DEV)
    B.mv_layer_norm_grad(dy, x, w, mean, rstd, dx, dw, db, ws, accumulate=accumulate)
    for g, (val, tol), what in zip((dx, dw, db), want, ("dx", "dweight", "dbias")):
        bad = ~within(g, val, tol)
        assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[0].tolist(), float((g.double().cpu() - val)[bad].abs().max()))
    return dx, dw, db


@pytest.mark.parametrize("T,D", SHAPES + [(5000, 64), (1200, 1001), (4000, 520)])
@pytest.mark.parametrize("dt,wt,pad,offset", [(F32, F32, (0, 0, 0), 0), (BF16, F32, (0, 0, 0), 1), (BF16, BF16, (8, 8, 16), 0), (F16, F16, (1, 0, 3), 0), (BF16, BF16, (2, 2, 2), 3), (F32, F32, (3, 0, 1), 1)])
def test_gradients(T, D, dt, wt, pad, offset):
    x, _ = strided(T, D, dt, pad[0], pad[1], seed=T + D)
    x.mul_(1.7).add_(torch.randn(D, generator=gen(D), device=DEV).to(dt))
    dy, _ = strided(T, D, dt, pad[1], pad[0], seed=T + D + 1)
    dx, buf = strided(T, D, dt, pad[2], pad[1], fill=7.0)
    w, _ = parameters(D, wt, offset, seed=D)
    row = torch.full((2 * D + offset + 1,), 7.0, device=DEV)
    check_grad(dy, x, w, dx, (row[offset:offset + D], row[offset + D:offset + 2 * D]))
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, dx.shape, dx.stride(), dx.storage_offset()).fill_(False)
    assert bool((buf[mask] == 7.0).all()) and bool((row[:offset] == 7.0).all()) and float(row[-1]) == 7.0


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("T,D", [(1, 9), (30, 1001), (600, 2048), (3, 30_000)])
def test_gradients_added_in_place_and_apart(dt, T, D):
    x, dy = (torch.randn((T, D), generator=gen(T + s), device=DEV).to(dt) for s in (1, 2))
    w, b = parameters(D, F32)
    stats = run_forward(x, w, b)[1:]
    dx, dw, db = check_grad(dy, x, w, statistics=stats)
    check_grad(dy, x, w, out=(torch.randn(D, device=DEV), torch.randn(D, device=DEV)), accumulate=True, statistics=stats)
    check_grad(dy, x, None, statistics=stats)
    ws = torch.empty(B.layer_norm_grad_workspace_bytes(T, D), dtype=torch.uint8, device=DEV)
    for inplace in (0, 1):                                   # dx in the place of dy, of x
        a, c = dy.clone(), x.clone()
        w2, b2 = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
        B.mv_layer_norm_grad(a, c, w, *stats, c if inplace else a, w2, b2, ws)
        assert torch.equal(c if inplace else a, dx) and torch.equal(w2, dw) and torch.equal(b2, db)
        assert torch.equal(a if inplace else c, dy if inplace else x)
    only = torch.empty_like(dx)                              # one output at a time
    B.mv_layer_norm_grad(dy, x, w, *stats, only, None, None, None)
    assert torch.equal(only, dx)
    for j, full in enumerate((dw, db)):
        one = torch.empty(D, device=DEV)
        B.mv_layer_norm_grad(dy, x, w, *stats, None, *((one, None) if j == 0 else (None, one)), ws)
        assert torch.equal(one, full)


def test_no_rows():
    x, f, one = torch.empty((0, 12), device=DEV), torch.empty(0, device=DEV), torch.ones(12, device=DEV)
    B.mv_layer_norm(x, one, one, x.clone(), mean=f, rstd=f)
    dw, db = torch.ones(12, device=DEV), torch.ones(12, device=DEV)
    ws = torch.empty(B.layer_norm_grad_workspace_bytes(0, 12), dtype=torch.uint8, device=DEV)
    B.mv_layer_norm_grad(x, x, one, f, f, x.clone(), dw, db, ws, accumulate=True)
    assert bool((dw == 1).all()) and bool((db == 1).all())
    B.mv_layer_norm_grad(x, x, one, f, f, x.clone(), dw, db, ws)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_gradients_against_differences():
    """Central differences of <dy, layer norm> in 64 bits with a step of 1e-5: off by about 1e-10 of the third derivative, and by 1e-11 of rounding."""
    T, D = 3, 11
    g = gen(5)
    x, dy = (torch.randn((T, D), generator=g, device=DEV) for _ in range(2))
    w, b = parameters(D, F32, seed=9)
    dx, dw, db = check_grad(dy, x, w)
    p = [t.double().cpu() for t in (x, w, b)]

    def f(x, w, b):
        mean = x.mean(1, keepdim=True)
        var = ((x - mean) ** 2).mean(1, keepdim=True)
        return float((dy.double().cpu() * ((x - mean) / torch.sqrt(var + EPS) * w + b)).sum())

    for j, got in enumerate((dx, dw, db)):
        for i in range(p[j].numel()):
            ends = []
            for s in (1e-5, -1e-5):
                q = [t.clone() for t in p]
                q[j].view(-1)[i] += s
                ends.append(f(*q))
            want = (ends[0] - ends[1]) / 2e-5
            assert abs(float(got.view(-1)[i]) - want) < 2e-5 * (1 + abs(want))


def test_past_32_bit_offsets_and_many_rows():
    T, D = 70_000, 32_768                                    # 2.3e9 elements
    x = torch.zeros((T, D), dtype=BF16, device=DEV)
    rows = torch.tensor([0, 65_535, 65_536, T - 1], device=DEV)
    x[rows] = torch.randn((4, D), generator=gen(4), device=DEV).to(BF16)
    some = x[rows].clone()
    want = run_forward(some, None, None)
    y, mean, rstd = run_forward(x, None, None)
    assert torch.equal(y[rows], want[0]) and torch.equal(mean[rows], want[1]) and torch.equal(rstd[rows], want[2])
    dw, db = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
    ws = torch.empty(B.layer_norm_grad_workspace_bytes(T, D), dtype=torch.uint8, device=DEV)
    B.mv_layer_norm_grad(x, x, None, mean, rstd, y, dw, db, ws)
    check = grad_reference(some, some, None, want[1], want[2])
    assert bool(within(y[rows], *check[0]).all())
    assert bool(within(db, check[2][0], check[2][1] * 20_000).all())             # T = 70000 terms, all but four of them zero


def test_the_same_bytes_every_time_on_other_streams_and_replayed():
    T, D = 777, 640
    g = gen(3)
    x, dy = (torch.randn((T, D), generator=g, device=DEV).to(BF16) for _ in range(2))
    w, b = parameters(D, BF16)
    ws = torch.empty(B.layer_norm_grad_workspace_bytes(T, D), dtype=torch.uint8, device=DEV)

    def outputs():
        return [torch.zeros((T, D), dtype=BF16, device=DEV), torch.zeros(T, device=DEV), torch.zeros(T, device=DEV), torch.zeros((T, D), dtype=BF16, device=DEV),
                torch.zeros(D, device=DEV), torch.zeros(D, device=DEV)]

    def run(o, stream=None):
        B.mv_layer_norm(x, w, b, o[0], mean=o[1], rstd=o[2], stream=stream)
        B.mv_layer_norm_grad(dy, x, w, o[1], o[2], o[3], o[4], o[5], ws, stream=stream)

    a, c = outputs(), outputs()
    run(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(a)
    x.copy_(torch.randn((T, D), generator=g, device=DEV))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    run(c, st)
    st.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_shapes_and_types_that_do_not_fit_are_refused():
    x = torch.zeros((4, 8), device=DEV)
    y, f, v = torch.zeros_like(x), torch.zeros(4, device=DEV), torch.zeros(8, device=DEV)
    ws = torch.empty(B.layer_norm_grad_workspace_bytes(4, 8), dtype=torch.uint8, device=DEV)
    buf = torch.zeros((5, 8), device=DEV)
    bad = [
        lambda: B.mv_layer_norm(x, v, v, y.half()),
        lambda: B.mv_layer_norm(x, v.half(), v.half(), y),
        lambda: B.mv_layer_norm(x.half(), v.half(), v, y.half()),
        lambda: B.mv_layer_norm(x, v[:7], None, y),
        lambda: B.mv_layer_norm(x, v, v, y[:3]),
        lambda: B.mv_layer_norm(x.t(), None, None, y),
        lambda: B.mv_layer_norm(x.cpu(), v, v, y),
        lambda: B.mv_layer_norm(x, v, v, y, eps=-1.0),
        lambda: B.mv_layer_norm(x, v, v, y, eps=math.nan),
        lambda: B.mv_layer_norm(x, v, v, y, mean=f[:3]),
        lambda: B.mv_layer_norm(buf[:4], v, v, buf[1:]),
        lambda: B.mv_layer_norm(x, y[1], v, y),
        lambda: B.mv_layer_norm_grad(y, x, v, f, f, y.half(), None, None, ws),
        lambda: B.mv_layer_norm_grad(y, x, v, f, f, None, None, None, ws),
        lambda: B.mv_layer_norm_grad(y, x, v, None, f, y, None, None, ws),
        lambda: B.mv_layer_norm_grad(y, x, v, f, f, y, v.clone(), None, None),
        lambda: B.mv_layer_norm_grad(y, x, v, f, f, y, v.clone(), None, ws[:4]),
        lambda: B.mv_layer_norm_grad(y, x, v, f, f, y, v, None, ws),
        lambda: B.mv_layer_norm_grad(buf[:4], x, v, f, f, buf[1:], None, None, ws),
        lambda: B.mv_layer_norm_grad(y, x, v, f, f, buf[:4], x[0], None, ws),
        lambda: B.mv_layer_norm_grad(y, x, v, f, f, buf[:4], buf[4], buf[4], ws),
    ]
    for i, f_ in enumerate(bad):
        with pytest.raises(B.MvError):
            f_()
            pytest.fail(f"refusal {i} did not come")
    torch.cuda.synchronize()
