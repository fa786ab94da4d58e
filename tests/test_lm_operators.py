"""GPU tests of the language-model operators (include/mv_lm.h) against plain statements in 64 bits.

Tolerances.  u = 2^-24 is the rounding of 32 bits.  A result that is rounded once more, to 16 bits, has to be what some
value inside the 32-bit tolerance rounds to (rounding is monotone: between the roundings of the two ends).  A sum of n terms in any order has an
error of at most 1.01 n u sum|terms| (n u < 0.01).  The library's 2^t has a relative error of at most 2^-22 (two units in the
last place of the hardware's exponential), and its argument, two roundings of a difference of two logits times a constant
that is itself rounded, is off by 3 u |t|, which the exponential turns into a relative 3 u ln2 |t|."""
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


def within(got, want, tol):
    """Elementwise: is got (of its own type) the rounding of a value in [want - tol, want + tol]?"""
    lo, hi = ((want + e).float().to(got.dtype).double() for e in (-tol, tol))
    got = got.double().cpu()
    return (got >= lo) & (got <= hi)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def strided(rows, cols, dtype, pad=0, offset=0, fill=None, seed=0):
    """A [rows, cols] tensor whose rows are cols + pad apart and that starts `offset` elements into its buffer, with the buffer."""
    buf = torch.empty(offset + rows * (cols + pad) + 5, dtype=dtype, device=DEV)
    if fill is None:
        buf.normal_(generator=gen(seed))
    else:
        buf.fill_(fill)
    view = torch.as_strided(buf, (rows, cols), (cols + pad, 1), offset)
    return view, buf


# ------------------------------------------------------------------------------------------ lookup

@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (1, 7, 8), (3, 50, 129), (8, 1000, 4096), (257, 33, 64), (300, 5, 1000), (5, 9, 20_001), (70_001, 11, 3)])
@pytest.mark.parametrize("wt,ot,it", [(F32, F32, torch.int32), (BF16, BF16, torch.int64), (F16, F32, torch.int64), (F32, BF16, torch.int32), (BF16, F16, torch.int32)])
@pytest.mark.parametrize("pads", [(0, 0, 0, 0), (1, 3, 1, 5), (8, 0, 16, 8)])
def test_embed_rows(T, V, D, wt, ot, it, pads):
    """Bit for bit: one rounding of the product to 32 bits, one to the output's type; nothing outside the rows is written."""
    w, _ = strided(V, D, wt, pads[0], pads[1], seed=T + D)
    out, buf = strided(T, D, ot, pads[2], pads[3], fill=7.0)
    ids = torch.randint(-2, V + 2, (T,), generator=gen(T), device=DEV).to(it)
    scale = 1.7
    B.mv_embed(w, ids, out, scale=scale)
    ok = (ids >= 0) & (ids < V)
    want = torch.where(ok[:, None], (w[ids.long().clamp(0, V - 1)].float() * scale).to(ot), torch.zeros((), dtype=ot, device=DEV))
    assert torch.equal(out, want)
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, out.shape, out.stride(), out.storage_offset()).fill_(False)
    assert bool((buf[mask] == 7.0).all())


def test_embed_keeps_special_values_and_other_streams():
    w = torch.tensor([[float("nan"), float("inf"), -0.0, 1e-45], [1.0, -2.0, 3.0e38, 5.0]], device=DEV)
    ids = torch.tensor([1, 0, 1], device=DEV)
    out = torch.empty(3, 4, device=DEV)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    B.mv_embed(w, ids, out, scale=2.0, stream=st)
    st.synchronize()
    want = (w.cpu() * 2.0)[ids.cpu()].numpy()
    assert np.array_equal(out.cpu().numpy().view(np.uint32)[:, 1:], want.view(np.uint32)[:, 1:]) and bool(torch.isnan(out[1, 0]))


def test_embed_past_32_bit_offsets():
    V, D = 70_000, 32_768                                   # 2.3e9 elements
    w = torch.empty((V, D), dtype=BF16, device=DEV)
    for v in (0, 65_535, 65_536, V - 1):
        w[v] = torch.randn(D, generator=gen(v), device=DEV).to(BF16)
    ids = torch.tensor([V - 1, 0, 65_536, 65_535], device=DEV)
    out = torch.empty((4, D), dtype=BF16, device=DEV)
    B.mv_embed(w, ids, out)
    assert torch.equal(out, w[ids])


# ------------------------------------------------------------------------------------------ gradient of the lookup

def grad_reference(dout, ids, V, scale, pad_id, old=None):
    """(value, bound on the error) in 64 bits."""
    T, D = dout.shape
    ids = ids.long().cpu()
    x = dout.double().cpu()
    ok = (ids >= 0) & (ids < V) & (ids != pad_id)
    val = torch.zeros((V, D), dtype=torch.float64).index_add_(0, ids[ok], x[ok])
    mag = torch.zeros((V, D), dtype=torch.float64).index_add_(0, ids[ok], x[ok].abs())
    n = torch.zeros(V, dtype=torch.float64).index_add_(0, ids[ok], torch.ones(int(ok.sum()), dtype=torch.float64))
    s = float(np.float32(scale))
    val, mag = val * s, mag * abs(s)
    if old is not None:
        val, mag = val + old.double().cpu() * 1.0, mag + old.double().cpu().abs()
    return val, 1.01 * (n[:, None] + 2) * U32 * mag + 2.0 ** -149 * (n[:, None] > 0)


def check_grad(T, V, D, dt=F32, it=torch.int64, ids=None, pad=(0, 0), out=(0, 0), scale=1.0, pad_id=-1, accumulate=False, seed=0):
    dout, _ = strided(T, D, dt, pad[0], pad[1], seed=seed + T)
    if ids is None:
        ids = torch.randint(-1, V + 1, (T,), generator=gen(seed + 1), device=DEV)
    ids = ids.to(it)
    dw, buf = strided(V, D, F32, out[0], out[1], fill=float("nan"))
    old = None
    if accumulate:
        dw.normal_(generator=gen(seed + 2))
        old = dw.clone()
    before = buf.clone()
    ws = torch.full((B.embed_grad_workspace_bytes(T, V, D),), 255, dtype=torch.uint8, device=DEV)
    B.mv_embed_grad(dout, ids, dw, ws, scale=scale, pad_id=pad_id, accumulate=accumulate)
    want, tol = grad_reference(dout, ids, V, scale, pad_id, old)
    got = dw.double().cpu()
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() - tol).max())
    # rows without a token: +0 (or, when accumulating, what was there); nothing between or behind the rows is written
    used = torch.zeros(V, dtype=torch.bool)
    used[ids.long().cpu()[(ids.cpu() >= 0) & (ids.cpu() < V) & (ids.cpu() != pad_id)].long()] = True
    rest = dw[~used.to(DEV)].contiguous().view(torch.int32)
    assert torch.equal(rest, old[~used.to(DEV)].view(torch.int32) if accumulate else torch.zeros_like(rest))
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, dw.shape, dw.stride(), dw.storage_offset()).fill_(False)
    assert torch.equal(buf[mask].view(torch.int32), before[mask].view(torch.int32))
    if not accumulate:                                     # the same bytes again, whatever the workspace held
        first = dw.clone()
        ws.fill_(0)
        B.mv_embed_grad(dout, ids, dw, ws, scale=scale, pad_id=pad_id)
        assert torch.equal(first.view(torch.int32), dw.contiguous().view(torch.int32))


@pytest.mark.parametrize("T,V,D", [(0, 3, 5), (1, 1, 1), (1, 300, 64), (2, 2, 7), (31, 40, 33), (64, 1, 16), (65, 2, 128), (127, 1000, 1000),
                                   (1000, 129, 257), (5000, 20_000, 24), (20_000, 3000, 40), (4097, 128, 2049)])
@pytest.mark.parametrize("dt,it,out", [(F32, torch.int32, (0, 0)), (BF16, torch.int64, (0, 1)), (F16, torch.int64, (3, 2)), (BF16, torch.int32, (8, 4))])
def test_embed_grad_matches_sums_in_64_bits(T, V, D, dt, it, out):
    check_grad(T, V, D, dt, it, out=out, scale=1.0 if T % 2 else 2.5)
    check_grad(T, V, D, dt, it, out=out, pad=(1, 1), pad_id=0, accumulate=True, seed=9)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000, 9000])
def test_embed_grad_of_runs_of_every_length(n):
    """n tokens of one id between others: runs that begin, end and pass through whatever pieces the sum is split in."""
    g = gen(n)
    ids = torch.cat([torch.full((n,), 5, device=DEV), torch.randint(0, 40, (n // 3 + 3,), generator=g, device=DEV), torch.full((n // 2,), 133, device=DEV)])
    ids = ids[torch.randperm(ids.numel(), generator=g, device=DEV)]
    check_grad(ids.numel(), 200, 72, BF16, ids=ids)
    check_grad(ids.numel(), 200, 35, F32, ids=ids, accumulate=True)


def test_embed_grad_of_text_like_tokens_and_of_one_token_only():
    u = torch.rand(30_000, generator=gen(3), device=DEV)
    check_grad(30_000, 50_021, 48, BF16, ids=((50_021.0 ** u) - 1).long())
    check_grad(20_000, 50_021, 16, F32, ids=torch.full((20_000,), 50_020, device=DEV))
    check_grad(3000, 50_021, 16, F32, ids=torch.full((3000,), 77, device=DEV), pad_id=77)          # nothing left
    check_grad(3000, 2_500_003, 2, F32)                                                              # a very large vocabulary
    check_grad(100, 2_500_003, 1, F32, accumulate=True)


@pytest.mark.parametrize("it", [torch.int32, torch.int64])
@pytest.mark.parametrize("T", [255, 256, 257, 8191, 8192, 8193, 40_000])
def test_embed_grad_of_ids_that_start_anywhere(T, it):
    """The ids are read 16 bytes at a time where they are aligned; stretches of whole and of broken batches; ids of other
    words (beyond 32 bits, negative) among them; long stretches of one id, as padding leaves them."""
    g = gen(T)
    ids = torch.randint(0, 700, (T + 3,), generator=g, device=DEV).to(it)
    ids[T // 3: T // 2] = 5
    ids[::17] = -1
    if it == torch.int64:
        ids[::19] = (1 << 32) + 3
        ids[::23] = -(1 << 40)
    for off in (0, 1, 3):
        check_grad(T, 700, 20, F32, it, ids=ids[off:off + T])
        check_grad(T, 700, 20, BF16, it, ids=ids[off:off + T], pad_id=5, accumulate=True)


def test_embed_grad_past_32_bit_offsets():
    V, D, T = 70_000, 32_768, 6
    ids = torch.tensor([V - 1, 65_537, 0, V - 1, 65_536, 9], device=DEV)
    dout = torch.randn((T, D), generator=gen(1), device=DEV)
    dw = torch.empty((V, D), device=DEV)
    ws = torch.empty(B.embed_grad_workspace_bytes(T, V, D), dtype=torch.uint8, device=DEV)
    B.mv_embed_grad(dout, ids, dw, ws)
    assert torch.equal(dw[V - 1], dout[0] + dout[3]) and torch.equal(dw[0], dout[2]) and torch.equal(dw[65_536], dout[4])
    assert torch.equal(dw[65_537], dout[1]) and torch.equal(dw[9], dout[5])
    dw[ids] = 0.0
    assert not bool(dw.any())


def test_embed_gradient_is_the_adjoint_of_the_lookup():
    """The lookup is linear in the table: a difference along a direction E is exact, <dout, embed(W + E) - embed(W)> = <dW, E>."""
    T, V, D, s = 500, 90, 64, 3.0
    g = gen(11)
    W, E = (torch.randint(-8, 9, (V, D), generator=g, device=DEV).float() for _ in range(2))
    dout = torch.randint(-4, 5, (T, D), generator=g, device=DEV).float()       # small integers: every sum is exact
    ids = torch.randint(0, V, (T,), generator=g, device=DEV)
    a, b, dw = torch.empty(T, D, device=DEV), torch.empty(T, D, device=DEV), torch.empty(V, D, device=DEV)
    B.mv_embed(W + E, ids, a, scale=s)
    B.mv_embed(W, ids, b, scale=s)
    B.mv_embed_grad(dout, ids, dw, torch.empty(B.embed_grad_workspace_bytes(T, V, D), dtype=torch.uint8, device=DEV), scale=s)
    assert float((dout.double() * (a - b).double()).sum()) == float((dw.double() * E.double()).sum())


# ------------------------------------------------------------------------------------------ token log probabilities

def logprob_reference(x, targets, scale, k):
    """Values and error bounds in 64 bits, rows of finite or -inf logits."""
    x = x.double().cpu()
    T, V = x.shape
    c = float(np.float32(scale))
    z = x * c
    m = z.amax(1, keepdim=True)
    empty = torch.isinf(m[:, 0])
    d = torch.where(torch.isinf(z), torch.full_like(z, -math.inf), z - torch.where(empty[:, None], torch.zeros_like(m), m))
    e = torch.exp(d)
    s = e.sum(1)
    lse = torch.where(empty, torch.full_like(s, -math.inf), m[:, 0] + torch.log(s))
    p = torch.where(empty[:, None], torch.zeros_like(e), e / s[:, None])
    dz = torch.where(p > 0, d, torch.zeros_like(d))
    H = torch.where(empty, torch.zeros_like(s), torch.log(s) - (p * dz).sum(1))
    # relative error of a term p: exponential and argument; of the sums: at most V terms a thread and a tree, taken as V / 32 + 64
    spread = (p * dz.abs()).sum(1)
    spread2 = (p * dz * dz).sum(1)
    add = (V / 32 + 64) * U32
    rho = 1.01 * (EX2 + add + 4 * U32 * spread)
    tol_lse = rho + 4 * U32 * (m[:, 0].abs().nan_to_num(posinf=0, neginf=0) + torch.log(s).abs().nan_to_num(neginf=0) + 1)
    tol_H = rho * (1 + spread) + 4 * U32 * (spread + spread2 + torch.log(s).abs().nan_to_num(neginf=0) + 1) + (EX2 + add) * spread
    y = targets.long().cpu()
    has = (y >= 0) & (y < V)
    zy = z.gather(1, y.clamp(0, V - 1)[:, None])[:, 0]
    lp = torch.where(has, torch.where(torch.isinf(zy), torch.full_like(zy, -math.inf), zy - lse.nan_to_num(neginf=0)), torch.zeros_like(zy))
    kk = min(k, V)
    order = np.lexsort((np.broadcast_to(np.arange(V), (T, V)), -(x.numpy() + 0.0)), axis=1)[:, :kk]
    order = torch.from_numpy(np.ascontiguousarray(order))
    ids = torch.full((T, k), -1, dtype=torch.int64)
    ids[:, :kk] = order
    top = torch.full((T, k), -math.inf, dtype=torch.float64)
    top[:, :kk] = z.gather(1, order) - lse.nan_to_num(neginf=0)[:, None]
    return {"lse": (lse, tol_lse), "entropy": (H, tol_H), "logprob": (lp, tol_lse + 4 * U32 * lp.abs().nan_to_num(posinf=0)),
            "top": (top, tol_lse[:, None] + 4 * U32 * top.abs().nan_to_num(posinf=0)), "ids": ids}


def close(got, want, what):
    val, tol = want
    val = torch.where(val.abs() > 3.5e38, val * math.inf, val)       # outside the range of 32 bits
    got = got.double().cpu()
    inf = torch.isinf(val)
    assert torch.equal(got[inf], val[inf]), what
    diff = (got - val)[~inf].abs()
    assert bool((diff <= tol.expand_as(val)[~inf]).all()), (what, float(diff.max()))


def call_logprob(x, targets, scale, k):
    T = x.shape[0]
    o = {n: torch.full((T,), -77.0, device=DEV) for n in ("logprob", "entropy", "lse")}
    top = torch.full((T, k), -77.0, device=DEV) if k else None
    ids = torch.full((T, k), -77, dtype=torch.int32, device=DEV) if k else None
    B.mv_token_logprob(x, targets, scale=scale, top_logprob=top, top_id=ids, **o)
    o["top"], o["ids"] = top, ids
    return o


def check_logprob(x, targets, scale=1.0, k=5):
    got, want = call_logprob(x, targets, scale, k), logprob_reference(x, targets, scale, k)
    if k:
        assert torch.equal(got["ids"].long().cpu(), want["ids"])
    for n in ("lse", "entropy", "logprob") + (("top",) if k else ()):
        close(got[n], want[n], n)
    return got


@pytest.mark.parametrize("T,V", [(1, 1), (1, 2), (3, 31), (2, 257), (7, 1000), (40, 1023), (5, 4099), (3, 32_000), (1, 50_021), (2, 131_072), (1, 200_003), (700, 513), (1500, 90)])
@pytest.mark.parametrize("dt,it,pad", [(F32, torch.int32, (0, 0)), (BF16, torch.int64, (0, 1)), (F16, torch.int64, (3, 2)), (BF16, torch.int32, (8, 0))])
@pytest.mark.parametrize("k", [0, 1, 8, 64])
def test_logprob_entropy_and_alternatives(T, V, dt, it, pad, k):
    x, _ = strided(T, V, dt, pad[0], pad[1], seed=T + V)
    x.mul_(3.0)
    targets = torch.randint(-1, V + 1, (T,), generator=gen(V), device=DEV).to(it)
    check_logprob(x, targets, 1.0 if k != 8 else 0.7, k)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("V", [1, 9, 300, 5000, 70_001])
def test_logprob_of_masked_flat_and_extreme_rows(dt, V):
    low = torch.finfo(dt).min
    g = gen(V)
    base = torch.randn((14, V), generator=g, device=DEV) * 4.0
    x = base.to(dt)
    x[0] = -math.inf                                       # nothing left
    x[1] = -math.inf
    x[1, V // 2] = 2.0                                     # one left
    x[2] = low                                             # every logit the type's lowest value
    x[3, : V // 2] = low                                   # masked by the lowest value
    x[4] = 1.5                                             # flat
    x[5] = 0.0
    x[5, ::2] = -0.0                                       # zeros of both signs
    x[6] = torch.linspace(-9, 9, V, device=DEV).to(dt)     # ascending
    x[7] = torch.linspace(9, -9, V, device=DEV).to(dt)     # descending
    x[8, torch.rand(V, generator=g, device=DEV) < 0.9] = -math.inf
    x[9, : V - 1] = -math.inf
    x[10, V // 3] = 80.0                                   # one takes all
    x[11] = torch.finfo(dt).max                            # every logit the type's largest value
    x[12, V // 2:] = -math.inf
    x[13, : (2 * V) // 3] = -math.inf
    targets = torch.randint(0, V, (14,), generator=g, device=DEV)
    targets[9] = V - 1
    for k in (0, 20):
        check_logprob(x, targets, 1.0, k)
    check_logprob(x[:11], targets[:11], 1.3, 3)
    # the rows one by one: a row's result does not depend on its neighbours
    for r in (0, 2, 6, 11, 13):
        check_logprob(x[r:r + 1], targets[r:r + 1], 1.0, 20)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("V,copies,pad", [(5000, 50, 1), (12_001, 60, 0), (90_001, 60, 3), (40_960, 1, 0), (3001, 220, 2), (9000, 220, 0), (12_003, 110, 1), (40, 220, 0)])
def test_the_same_rows_in_batches_of_every_kind(dt, V, copies, pad):
    """Twelve kinds of rows, among them empty, flat, tied and extreme ones, in batches that are cut among CTAs differently."""
    low, g = torch.finfo(dt).min, gen(V)
    x = (torch.randn((12, V), generator=g, device=DEV) * 3.0).to(dt)
    x[0] = -math.inf
    x[1] = low
    x[2] = 0.75
    x[3] = torch.linspace(-9, 9, V, device=DEV).to(dt)
    x[4, torch.rand(V, generator=g, device=DEV) < 0.999] = -math.inf
    x[5] = torch.randint(0, 4, (V,), generator=g, device=DEV).to(dt)
    x[6, : V // 2] = low
    x[7, V - 1] = 50.0
    x[8] = torch.finfo(dt).max
    x[9, ::2] = -math.inf
    x[10, : max(0, V - 70)] = low                                # the part before the last logits is all masked
    big, _ = strided(12 * copies, V, dt, pad, 0, fill=0.0)
    big.copy_(x.repeat(copies, 1))
    y = torch.randint(-1, V, (12,), generator=g, device=DEV)
    for k in (0, 3, 33):
        want = logprob_reference(x, y, 1.0, k)
        got = call_logprob(big, y.repeat(copies), 1.0, k)
        for n in ("lse", "entropy", "logprob") + (("top",) if k else ()):
            close(got[n], tuple(w.repeat(copies, *([1] * (w.dim() - 1))) for w in want[n]), n)
        if k:
            assert torch.equal(got["ids"].long().cpu(), want["ids"].repeat(copies, 1))


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("V", [3, 700, 40_000])
def test_logprob_of_rows_with_nan_and_inf(dt, V):
    x = torch.randn((4, V), generator=gen(V), device=DEV).to(dt)
    x[0, V - 1] = math.nan
    x[1, V // 2] = math.inf
    x[2, 0] = math.nan
    clean = x[3:4].clone()
    targets = torch.zeros(4, dtype=torch.int64, device=DEV)
    got = call_logprob(x, targets, 1.0, 2)
    for n in ("lse", "entropy", "logprob"):
        assert bool(torch.isnan(got[n][:3]).all())
    assert bool(torch.isnan(got["top"][:3]).all())
    ids = got["ids"].cpu()
    for r, bad in ((0, V - 1), (2, 0)):
        keep = [i for i in range(V) if i != bad]
        vals = x[r].float().cpu()[keep]
        order = sorted(range(len(keep)), key=lambda i: (-float(vals[i]), keep[i]))[:2]
        assert ids[r].tolist() == [keep[i] for i in order]
    assert ids[1, 0] == V // 2
    want = logprob_reference(clean, targets[3:], 1.0, 2)
    close(got["lse"][3:], want["lse"], "lse")
    x[3] = math.nan
    got = call_logprob(x, targets, 1.0, 3)
    assert got["ids"][3].tolist() == [-1, -1, -1]


def test_logprob_outputs_may_be_left_out():
    x = torch.randn((6, 999), generator=gen(1), device=DEV)
    y = torch.randint(0, 999, (6,), generator=gen(2), device=DEV)
    full = call_logprob(x, y, 1.0, 4)
    lp = torch.empty(6, device=DEV)
    B.mv_token_logprob(x, y, logprob=lp)
    assert torch.equal(lp, full["logprob"])
    lse = torch.empty(6, device=DEV)
    B.mv_token_logprob(x, lse=lse)
    assert torch.equal(lse, full["lse"])
    ids = torch.empty((6, 4), dtype=torch.int32, device=DEV)
    B.mv_token_logprob(x, top_id=ids)
    assert torch.equal(ids, full["ids"])
    B.mv_token_logprob(x[:0], y[:0], logprob=lp[:0])       # no rows


@pytest.mark.parametrize("k", [1, 64])
def test_alternatives_of_many_equal_logits(k):
    """Few distinct values: every rank is a tie, decided by the index, wherever the equal logits lie."""
    for V in (100, 2048, 30_011):
        x = torch.randint(0, 3, (5, V), generator=gen(V + k), device=DEV).to(BF16)
        x[4] = torch.randint(0, 2000, (V,), generator=gen(V), device=DEV).to(BF16)
        check_logprob(x, torch.zeros(5, dtype=torch.int32, device=DEV), 1.0, k)


def test_logprob_past_32_bit_offsets():
    T, V = 33_000, 70_001                                  # 2.3e9 logits
    x = torch.zeros((T, V), dtype=BF16, device=DEV)
    rows = torch.tensor([0, 30_677, 30_678, T - 1], device=DEV)
    x[rows] = torch.randn((4, V), generator=gen(4), device=DEV).to(BF16)
    y = torch.full((T,), 5, device=DEV)
    got = call_logprob(x, y, 1.0, 2)
    want = logprob_reference(x[rows], y[rows], 1.0, 2)
    assert torch.equal(got["ids"][rows].long().cpu(), want["ids"])
    close(got["lse"][rows], want["lse"], "lse")
    B.mv_token_logprob_grad(x, y, got["lse"], torch.ones(T, device=DEV), x)
    gx = x[rows].double().cpu()
    assert bool((gx.sum(1).abs() < 2 ** -8 * gx.abs().sum(1)).all())           # rounding to bf16 only
    flat = x[1].double().cpu()
    assert abs(float(flat[7]) + 1 / V) < 2 ** -8 / V and abs(float(flat[5]) - (1 - 1 / V)) <= 2 ** -8


# ------------------------------------------------------------------------------------------ gradient of the log probabilities

def grad_logits_reference(x, targets, scale, lse, entropy, g1, g2):
    """(value, bound) in 64 bits for the lse and entropy that the call is given."""
    x, l = x.double().cpu(), lse.double().cpu()[:, None]
    T, V = x.shape
    c = float(np.float32(scale))
    y = targets.long().cpu()
    has = (y >= 0) & (y < V)
    g1 = torch.where(has, g1.double().cpu(), torch.zeros(T, dtype=torch.float64)) if g1 is not None else torch.zeros(T, dtype=torch.float64)
    g2 = g2.double().cpu() if g2 is not None else torch.zeros(T, dtype=torch.float64)
    H = entropy.double().cpu() if entropy is not None else torch.zeros(T, dtype=torch.float64)
    none = ((g1 == 0) & (g2 == 0)) | torch.isinf(l[:, 0])
    lp = x * c - l
    p = torch.where(none[:, None], torch.zeros_like(lp), torch.exp(lp))
    lp = torch.where(p > 0, lp, torch.zeros_like(lp))
    hot = torch.zeros_like(p)
    hot[torch.arange(T)[has], y[has]] = 1.0
    hot[none] = 0.0
    val = c * (g1[:, None] * (hot - p) - g2[:, None] * p * (lp + H[:, None]))
    mag = c * (g1.abs()[:, None] * (hot + p) + g2.abs()[:, None] * p * (lp.abs() + H.abs()[:, None]))
    # relative error of p: the exponential, and the argument's roundings (those of x c and of l, and of the product with log2 e)
    arg = U32 * (2 * (x * c).abs().nan_to_num(posinf=0, neginf=0) + 4 * lp.abs() + l.abs().nan_to_num(posinf=0, neginf=0))
    rel = 1.01 * (EX2 + arg)
    pmag = c * p * (g1.abs()[:, None] + g2.abs()[:, None] * (lp.abs() + H.abs()[:, None]))
    tol = rel * pmag + c * g2.abs()[:, None] * p * arg + 6 * U32 * mag
    return val, tol + U32 * val.abs() + 2.0 ** -149 + 2.0 ** -126 * (p > 0) * mag.amax(1, keepdim=True)


def check_logits_grad(x, targets, scale=1.0, with_g1=True, with_g2=True, inplace=False, seed=0, pad=0):
    T, V = x.shape
    o = call_logprob(x, targets, scale, 0)
    g1 = torch.randn(T, generator=gen(seed + 5), device=DEV) if with_g1 else None
    g2 = torch.randn(T, generator=gen(seed + 6), device=DEV) if with_g2 else None
    want, tol = grad_logits_reference(x, targets, scale, o["lse"], o["entropy"] if with_g2 else None, g1, g2)
    src = x
    if inplace:
        src = x.clone(memory_format=torch.preserve_format) if x.is_contiguous() else x
        dx, buf = src, None
    else:
        dx, buf = strided(T, V, x.dtype, pad, 1 if pad else 0, fill=7.0)
    B.mv_token_logprob_grad(src, targets if with_g1 else None, o["lse"], g1, dx, scale=scale, entropy=o["entropy"] if with_g2 else None, g_entropy=g2)
    bad = ~within(dx, want, tol)
    assert not bool(bad.any()), (int(bad.sum()), float((dx.double().cpu() - want)[bad].abs().max()), bad.nonzero()[0].tolist())
    if buf is not None:
        mask = torch.ones_like(buf, dtype=torch.bool)
        torch.as_strided(mask, dx.shape, dx.stride(), dx.storage_offset()).fill_(False)
        assert bool((buf[mask] == 7.0).all())
    return dx


@pytest.mark.parametrize("T,V", [(1, 1), (1, 2), (3, 31), (2, 257), (7, 1000), (40, 1023), (5, 4099), (3, 32_000), (1, 50_021), (2, 131_072), (700, 513)])
@pytest.mark.parametrize("dt,it,pad", [(F32, torch.int32, (0, 0, 0)), (BF16, torch.int64, (0, 1, 1)), (F16, torch.int64, (3, 2, 3)), (BF16, torch.int32, (8, 0, 8))])
@pytest.mark.parametrize("terms", [(True, True), (True, False), (False, True)])
def test_logits_gradient_matches_the_formula(T, V, dt, it, pad, terms):
    x, _ = strided(T, V, dt, pad[0], pad[1], seed=T + V)
    x.mul_(3.0)
    targets = torch.randint(-1, V + 1, (T,), generator=gen(V), device=DEV).to(it)
    check_logits_grad(x, targets, 0.7, *terms, pad=pad[2])
    check_logits_grad(x, targets, 1.0, *terms, inplace=True)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
def test_logits_gradient_of_masked_and_extreme_rows(dt):
    for V in (1, 9, 5000):
        low = torch.finfo(dt).min
        x = (torch.randn((7, V), generator=gen(V), device=DEV) * 4).to(dt)
        x[0] = -math.inf
        x[1] = -math.inf
        x[1, V // 2] = 2.0
        x[2, : V // 2] = low
        x[3, torch.rand(V, generator=gen(1), device=DEV) < 0.9] = -math.inf
        x[4] = 0.25
        x[5, V // 3] = 80.0
        targets = torch.randint(0, V, (7,), generator=gen(2), device=DEV)
        targets[6] = -100
        dx = check_logits_grad(x, targets)
        assert not bool(dx[0].any())
        check_logits_grad(x, targets, with_g2=False)


def test_positions_without_a_gradient_are_zero_whatever_their_logits_hold():
    x = torch.full((4, 1001), math.nan, dtype=BF16, device=DEV)
    x[3] = 1.0
    y = torch.tensor([-100, 5, 1001, 6], device=DEV)
    lse = torch.tensor([math.nan, math.nan, math.inf, 1.0 + math.log(1001)], device=DEV)
    dx = torch.full_like(x, 7.0)
    B.mv_token_logprob_grad(x, y, lse, torch.tensor([1.0, 0.0, 2.0, 1.0], device=DEV), dx)
    assert not bool(dx[:3].view(torch.int16).any()) and float(dx[3, 6]) > 0.9
    B.mv_token_logprob_grad(x, y, lse, torch.ones(4, device=DEV), dx)
    assert bool(torch.isnan(dx[1]).all())                  # a target asks for the gradient of a NaN row: NaN


def test_logits_gradient_against_differences():
    """f(x + h v) - f(x - h v) over 2 h.  f is a sum of T = 4 outputs with errors below 1e-5 each (their own bounds), the third
    derivative along |v| <= 1 entries is below 30 for each: the difference is off by at most 2 * 8e-5 / (2 h) + 8 * 30 h^2 / 6."""
    T, V, h = 4, 700, 2.0 ** -6
    g = gen(21)
    x = torch.randn((T, V), generator=g, device=DEV) * 2
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    g1, g2 = torch.rand(T, generator=g, device=DEV), torch.rand(T, generator=g, device=DEV)
    o = call_logprob(x, y, 1.0, 0)
    dx = torch.empty_like(x)
    B.mv_token_logprob_grad(x, y, o["lse"], g1, dx, entropy=o["entropy"], g_entropy=g2)
    def f(xx):
        r = call_logprob(xx, y, 1.0, 0)
        return float((g1.double() * r["logprob"].double() + g2.double() * r["entropy"].double()).sum())
    for seed in range(4):
        v = torch.rand((T, V), generator=gen(seed), device=DEV) * 2 - 1
        diff = (f(x + h * v) - f(x - h * v)) / (2 * h)
        assert abs(diff - float((dx.double() * v.double()).sum())) <= 8e-5 / h + 40 * h * h


# ------------------------------------------------------------------------------------------ norms and clipping

SIZES = [[1], [0, 3, 0], [5, 1, 17, 1000, 64], [8192], [8191, 8193, 1, 16_384], [3, 100_003, 7], [1] * 300, [250_000, 11, 40_001]]
DTS = [F32, BF16, F16]


def make_tensors(sizes, groups, seed, dts=None, offset=0):
    ts, gs = [], []
    for g in range(groups):
        for i, n in enumerate(sizes):
            dt = DTS[(i + g) % 3] if dts is None else dts
            buf = torch.randn(n + offset + 3, generator=gen(seed + 31 * g + i), device=DEV).to(dt)
            ts.append(buf[offset:offset + n])
            gs.append(g)
    return ts, gs


def clip_reference(ts, gs, G, max_norm):
    sq = [0.0] * G
    for t, g in zip(ts, gs):
        sq[g] += float((t.double() ** 2).sum())
    n = [math.sqrt(s) for s in sq]
    return n, [min(1.0, max_norm / v) if v > 0 else 1.0 for v in n]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("G,offset", [(1, 0), (3, 1), (10, 2)])
@pytest.mark.parametrize("dts", [None, F32, BF16])
def test_norms_pack_and_scale(sizes, G, offset, dts):
    ts, gs = make_tensors(sizes, G, 5, dts, offset)
    for t, g in zip(ts, gs):
        t.mul_(1.0 + g)                                     # groups of different norms, some below max_norm
    d = sum(sizes)
    whole = [math.sqrt(sum(float((t.double() ** 2).sum()) for t, gg in zip(ts, gs) if gg == g)) for g in range(G)]
    max_norm = float(np.float32(sorted(whole)[G // 2] * (0.5 if G == 1 else 1.0)))
    n, c = clip_reference(ts, gs, G, max_norm)
    plan = B.MvClip(ts, gs, n_groups=G)
    norms = torch.full((G,), -1.0, device=DEV)
    plan.mv_clip_norm(norms)
    want = torch.tensor(n, dtype=torch.float64)
    assert bool(((norms.double().cpu() - want).abs() <= 2 * U32 * want).all())
    # pack: the sum of squares in 64 bits, the quotient rounded once, the product once
    rows, buf = strided(G, d + 2, F32, 3, offset, fill=7.0)
    rows = rows[:, :d] if d else rows[:, :1]
    norms.fill_(-1.0)
    plan.mv_clip_pack(max_norm, rows, norms)
    assert bool(((norms.double().cpu() - want).abs() <= 2 * U32 * want).all())
    keep = [t.clone() for t in ts]
    for g in range(G):
        if not d:
            continue
        x = torch.cat([t.double().reshape(-1) for t, gg in zip(ts, gs) if gg == g]).cpu()
        got = rows[g].double().cpu()
        assert bool(((got - x * c[g]).abs() <= 3 * U32 * (x * c[g]).abs() + 2.0 ** -149).all())
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, (G, d), rows.stride(), rows.storage_offset()).fill_(False)
    assert bool((buf[mask] == 7.0).all())
    # in place, norms left out
    plan.mv_clip_scale(max_norm)
    for t, k, g in zip(ts, keep, gs):
        x = k.double().cpu() * c[g]
        assert bool(within(t, x, 3 * U32 * x.abs() + 2.0 ** -149).all())
        if c[g] == 1.0:
            assert torch.equal(t, k)


def test_norm_of_very_large_and_very_small_values():
    for dt, v in ((F32, 2.5e38), (F32, 1e-40), (BF16, 1e38), (BF16, 1e-30), (F16, 6e4), (F16, 6e-8)):
        t = torch.full((20_000,), v, device=DEV).to(dt)
        n = torch.empty(1, device=DEV)
        plan = B.MvClip([t])
        plan.mv_clip_norm(n)
        want = float(t[0].double()) * math.sqrt(20_000)
        if want > 3.4e38:
            assert math.isinf(float(n))
        else:
            assert abs(float(n) - want) <= 2 * U32 * want + 2.0 ** -149
        row = torch.empty((1, 20_000), device=DEV)
        plan.mv_clip_pack(1.0, row, n)
        if v > 1.0:
            # the factor 1 / n is rounded to 32 bits, to a multiple of 2^-149 where it is that small
            assert abs(float(row.double().norm()) - 1.0) < 1e-6 + 2.0 ** -150 * want
        else:
            assert torch.equal(row[0], t.float())           # below the bound: untouched


def test_groups_that_are_empty_zero_or_not_finite():
    z = torch.zeros(1000, device=DEV)
    inf = torch.ones(1000, device=DEV)
    inf[7] = math.inf
    nan = torch.ones(1000, dtype=BF16, device=DEV)
    nan[999] = math.nan
    big = torch.ones(400, device=DEV)
    plan = B.MvClip([z, inf, nan, big], [1, 2, 3, 5], n_groups=7)
    norms = torch.full((7,), -1.0, device=DEV)
    before = [t.clone() for t in (z, inf, nan)]
    plan.mv_clip_scale(2.0, norms)
    n = norms.cpu()
    assert n[0] == 0 and n[1] == 0 and n[4] == 0 and n[6] == 0 and math.isinf(n[2]) and math.isnan(n[3]) and abs(float(n[5]) - 20.0) < 1e-5
    for a, b in zip(before, (z, inf, nan)):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert bool(((big - 0.1).abs() < 1e-7).all())
    plan.mv_clip_scale(0.0)                                # nothing is left of a finite group
    assert not bool(big.any()) and bool(inf[0] == 1.0)
    B.MvClip([big], [0]).mv_clip_scale(math.inf)
    empty = B.MvClip([], n_groups=2, device=DEV)
    n2 = torch.full((2,), 5.0, device=DEV)
    empty.mv_clip_norm(n2)
    assert not bool(n2.any())


def test_the_same_bytes_every_time_and_on_another_stream():
    ts, gs = make_tensors([40_001, 3, 250_000], 4, 77)
    plan = B.MvClip(ts, gs)
    d = 290_004
    a, b = torch.empty((4, d), device=DEV), torch.empty((4, d), device=DEV)
    na, nb = torch.empty(4, device=DEV), torch.empty(4, device=DEV)
    plan.mv_clip_pack(1.0, a, na)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for _ in range(3):
        plan.mv_clip_norm(nb, stream=st)                    # calls of both kinds on one plan
        plan.mv_clip_pack(1.0, b, nb, stream=st)
        st.synchronize()
        assert torch.equal(a, b) and torch.equal(na, nb)


def test_many_tensors_and_more_than_32_bit_offsets():
    t = torch.zeros(2_200_000_000, dtype=BF16, device=DEV)                     # 4.4 GB, one tensor
    t[2_199_999_999], t[0], t[2_147_483_648] = 3.0, 4.0, 12.0
    n = torch.empty(1, device=DEV)
    plan = B.MvClip([t])
    plan.mv_clip_scale(6.5, n)
    assert float(n) == 13.0 and float(t[2_199_999_999]) == 1.5 and float(t[0]) == 2.0 and float(t[2_147_483_648]) == 6.0
    row = torch.empty((1, 2_200_000_000), device=DEV)
    plan.mv_clip_pack(math.inf, row, n)
    assert float(row[0, 2_199_999_999]) == 1.5 and float(row[0, 2_147_483_648]) == 6.0 and float(row[0, 1]) == 0.0
    assert int(torch.count_nonzero(row)) == 3


# ------------------------------------------------------------------------------------------ together, and refusals

def test_a_step_from_tokens_to_the_shared_mask():
    """Lookup, log probabilities, both gradients, clipping and the sparse step for N workers of a small bigram model, against
    the same quantities formed in 64 bits; and a few steps lower the loss."""
    from paper_2011_06495_b200.lm_example import BigramWorkers
    for dtype in (BF16, F32):
        m = BigramWorkers(N=4, V=300, D=48, T=600, sparsity=0.02, lr=4.0, max_norm=1.0, seed=3, device=DEV, dtype=dtype)
        losses = [m.step() for _ in range(30)]
        assert losses[-1] < losses[0] - 0.3
    m.check_gradients()


def test_the_calls_can_be_captured_and_replayed_on_new_inputs():
    """Every call enqueues kernels and nothing else: captured once into a graph, replayed after the inputs have changed, it gives
    what a call on another stream gives."""
    T, V, D = 300, 5000, 96
    g = gen(8)
    w, ids = torch.randn((V, D), generator=g, device=DEV), torch.randint(0, V, (T,), generator=g, device=DEV)
    lg, gl = torch.randn((T, V), generator=g, device=DEV).to(BF16), torch.randn(T, generator=g, device=DEV)
    small, large = torch.randn(300_000, generator=g, device=DEV), torch.randn(6_000_000, generator=g, device=DEV)
    plans = [B.MvClip([small]), B.MvClip([large])]
    ws = torch.empty(B.embed_grad_workspace_bytes(T, V, D), dtype=torch.uint8, device=DEV)

    def outputs():
        f = lambda *shape, **k: torch.zeros(*shape, device=DEV, **k)
        return [f(T, D), f(V, D), f(T), f(T), f(T), f(T, 4), f(T, 4, dtype=torch.int32), f(T, V, dtype=BF16), f(1, 300_000), f(1), f(1, 6_000_000), f(1)]

    def run(o, stream=None):
        B.mv_embed(w, ids, o[0], scale=2.0, stream=stream)
        B.mv_embed_grad(o[0], ids, o[1], ws, stream=stream)
        B.mv_token_logprob(lg, ids, logprob=o[2], entropy=o[3], lse=o[4], top_logprob=o[5], top_id=o[6], stream=stream)
        B.mv_token_logprob_grad(lg, ids, o[4], gl, o[7], stream=stream)
        for p, r, n in ((plans[0], o[8], o[9]), (plans[1], o[10], o[11])):
            p.mv_clip_pack(1.0, r, n, stream=stream)

    a, b = outputs(), outputs()
    run(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(a)
    ids.copy_(torch.randint(0, V, (T,), generator=g, device=DEV))
    lg.copy_(torch.randn((T, V), generator=g, device=DEV))
    small.mul_(3.0)
    large.mul_(0.5)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    run(b, st)
    st.synchronize()
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(x, y), i


@pytest.mark.parametrize("D", [7, 64, 300])
def test_windows_of_one_buffer_side_by_side(D):
    """Column windows of the same rows share no bytes: they are taken, and nothing beside them changes; one column more and they are refused."""
    g = torch.Generator(device=DEV).manual_seed(D)
    T = 200
    for left in (True, False):
        src, dst = (slice(0, D), slice(D, 2 * D)) if left else (slice(D, 2 * D), slice(0, D))
        wide = (slice(D - 1, 2 * D - 1) if left else slice(1, D + 1))
        ids = torch.randint(0, T, (T,), generator=g, device=DEV)
        ws = torch.empty(B.embed_grad_workspace_bytes(T, T, D), dtype=torch.uint8, device=DEV)
        gl, lse = torch.randn(T, generator=g, device=DEV), torch.zeros(T, device=DEV)
        calls = [
            lambda x, o: B.mv_embed(x, ids, o),
            lambda x, o: B.mv_embed_grad(x, ids, o, ws),
            lambda x, o: B.mv_token_logprob_grad(x, ids % D, lse, gl, o),
        ]
        for call in calls:
            buf = torch.randn((T, 2 * D + 1), generator=g, device=DEV)
            old, apart = buf.clone(), torch.empty_like(buf)
            call(old[:, src], apart[:, dst])           # two buffers, the same places in them
            call(buf[:, src], buf[:, dst])
            assert torch.equal(buf[:, dst], apart[:, dst])
            assert torch.equal(buf[:, src], old[:, src]) and torch.equal(buf[:, 2 * D:], old[:, 2 * D:])
            with pytest.raises(B.MvError):
                call(buf[:, src], buf[:, wide])


def test_shapes_and_types_that_do_not_fit_are_refused():
    w, out = torch.zeros((10, 8), device=DEV), torch.zeros((4, 8), device=DEV)
    ids = torch.zeros(4, dtype=torch.int64, device=DEV)
    ws = torch.empty(B.embed_grad_workspace_bytes(4, 10, 8), dtype=torch.uint8, device=DEV)
    lg, y, f = torch.zeros((4, 30), device=DEV), ids, torch.zeros(4, device=DEV)
    bad = [
        lambda: B.mv_embed(w, ids[:3], out),
        lambda: B.mv_embed(w, ids.float(), out),
        lambda: B.mv_embed(w, ids, out[:, :7]),
        lambda: B.mv_embed(w.double(), ids, out),
        lambda: B.mv_embed(w.t(), ids, out),
        lambda: B.mv_embed(w.cpu(), ids, out),
        lambda: B.mv_embed(w, ids, w[6:]),
        lambda: B.mv_embed_grad(w[6:], ids, w, ws),
        lambda: B.mv_embed_grad(out, ids, w.half(), ws),
        lambda: B.mv_embed_grad(out, ids, w, ws[:8]),
        lambda: B.mv_embed_grad(out, ids, w[:, :4], ws),
        lambda: B.mv_token_logprob(lg, y, scale=0.0, logprob=f),
        lambda: B.mv_token_logprob(lg, y, scale=float("nan"), logprob=f),
        lambda: B.mv_token_logprob(lg, None, logprob=f),
        lambda: B.mv_token_logprob(lg, y, logprob=f[:3]),
        lambda: B.mv_token_logprob(lg, y, logprob=f.half()),
        lambda: B.mv_token_logprob(lg, y, top_id=torch.zeros((4, 65), dtype=torch.int32, device=DEV)),
        lambda: B.mv_token_logprob(lg, y, top_id=torch.zeros((4, 3), dtype=torch.int32, device=DEV), top_logprob=torch.zeros((4, 2), device=DEV)),
        lambda: B.mv_token_logprob_grad(lg, y, f, f, lg.bfloat16()),
        lambda: B.mv_token_logprob_grad(lg, y, f, None, torch.empty_like(lg)),
        lambda: B.mv_token_logprob_grad(lg, None, f, f, torch.empty_like(lg)),
        lambda: B.mv_token_logprob_grad(lg, y, f, f, torch.empty_like(lg), g_entropy=f),
        lambda: B.mv_token_logprob_grad(lg[:3], y[:3], f[:3], f[:3], lg[1:]),
        lambda: B.MvClip([w], [0, 1]),
        lambda: B.MvClip([w, w], [1, 0]),
        lambda: B.MvClip([w], [2], n_groups=2),
        lambda: B.MvClip([w.double()]),
        lambda: B.MvClip([w.t()]),
        lambda: B.MvClip([w]).mv_clip_scale(-1.0),
        lambda: B.MvClip([w]).mv_clip_scale(float("nan")),
        lambda: B.MvClip([w]).mv_clip_norm(torch.zeros(2, device=DEV)),
        lambda: B.MvClip([w]).mv_clip_pack(1.0, torch.zeros((1, 79), device=DEV)),
        lambda: B.MvClip([w, w], [0, 1]).mv_clip_pack(1.0, torch.zeros((2, 100), device=DEV)[:, :79]),
        lambda: B.MvClip([w]).mv_clip_pack(1.0, w.view(1, 80)),
    ]
    for i, f_ in enumerate(bad):
        with pytest.raises(B.MvError):
            f_()
            pytest.fail(f"refusal {i} did not come")
    torch.cuda.synchronize()
