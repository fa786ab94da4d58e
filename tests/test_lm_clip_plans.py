"""GPU tests of the clipping plans (MvClip): their memory, and what a plan does outside the ordinary."""
import torch
import pytest

from paper_2011_06495_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def addresses(nbytes, n=40):
    """Where the current stream's next n allocations of that size lie."""
    ts = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(n)]
    return {t.data_ptr() for t in ts}


@pytest.mark.parametrize("n", [5000, 5_000_000])
@pytest.mark.parametrize("created_on_it", [False, True])
def test_a_plan_dropped_while_its_call_waits_keeps_its_memory(n, created_on_it):
    """A call on another stream that has yet to run: neither the plan's list nor the tensors are given to other tensors."""
    want = torch.randn(n, device=DEV)
    rows, norms = torch.empty((1, n), device=DEV), torch.empty(1, device=DEV)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    t = want.clone()
    plan = B.MvClip([t], stream=st if created_on_it else None)
    torch.cuda.synchronize()
    mine, list_bytes, at = plan.workspace.data_ptr(), plan.workspace.numel(), t.data_ptr()
    with torch.cuda.stream(st):
        torch.cuda._sleep(1_000_000_000)                   # half a second
    plan.mv_clip_pack(1e30, rows, norms, stream=st)
    del plan, t
    there = addresses(list_bytes) | addresses(4 * n, 4)
    assert not st.query()                                  # the call is still waiting
    assert mine not in there and at not in there
    st.synchronize()
    assert torch.equal(rows[0], want)


def test_a_plan_made_on_another_stream_takes_no_memory_still_in_use():
    """What the current stream has freed, but not yet finished with, may be overwritten by it at any later time."""
    t = torch.randn(5000, device=DEV)
    st = torch.cuda.Stream()
    sizes = int(B.load().mv_clip_workspace_bytes((B.ctypes.c_int64 * 1)(5000), 1, 1))
    torch.cuda.synchronize()
    torch.cuda._sleep(1_000_000_000)
    freed = addresses(sizes)                               # freed at once; the current stream is still asleep
    plan = B.MvClip([t], stream=st)
    assert not torch.cuda.current_stream().query()
    assert plan.workspace.data_ptr() not in freed
    norms = torch.empty(1, device=DEV)
    st.wait_stream(torch.cuda.current_stream())
    plan.mv_clip_norm(norms, stream=st)
    st.synchronize()
    assert abs(float(norms) - float(t.norm())) < 1e-3


def test_the_device_may_be_named_without_its_number():
    t = torch.ones(16, device=DEV)
    norms = torch.empty(1, device=DEV)
    for dev in ("cuda", "cuda:0", torch.device("cuda"), torch.device(DEV), None):
        B.MvClip([t], device=dev).mv_clip_norm(norms)
        assert float(norms) == 4.0
        B.MvClip([], device=dev).mv_clip_norm(norms)
        assert float(norms) == 0.0
    with pytest.raises(B.MvError):
        B.MvClip([t], device="cpu")


@pytest.mark.parametrize("n", [100, 6_000_000])
def test_tensors_that_share_bytes_are_not_scaled_in_place(n):
    """The same tensor twice, windows that overlap, in one group or two: norms and rows count every tensor, scaling is refused;
    tensors end to end and empty ones inside others share nothing."""
    b = torch.randn(n, generator=torch.Generator(device=DEV).manual_seed(n), device=DEV)
    old = b.clone()
    for ts, gs in (([b, b], [0, 0]), ([b, b], [0, 1]), ([b[: n // 2 + 1], b[n // 2:]], None), ([b[n // 2:], b], None), ([b, b.view(torch.bfloat16)[7:8]], None)):
        plan = B.MvClip(ts, gs)
        want = [sum(float(t.double().pow(2).sum()) for t, g in zip(ts, gs or [0] * 9) if g == i) ** 0.5 for i in range(plan.n_groups)]
        norms = torch.empty(plan.n_groups, device=DEV)
        rows = torch.zeros((plan.n_groups, plan.longest), device=DEV)
        plan.mv_clip_pack(float("inf"), rows, norms)
        for g in range(plan.n_groups):
            assert abs(float(norms[g]) - want[g]) <= 2.0 ** -22 * want[g]
            mine = torch.cat([t.float() for t, gg in zip(ts, gs or [0] * 9) if gg == g])
            assert torch.equal(rows[g, : mine.numel()], mine)
        with pytest.raises(B.MvError):
            plan.mv_clip_scale(0.5)
        assert torch.equal(b, old)
    for ts in ([b[n // 2:], b[: n // 2]], [b, b[5:5]], [b[5:5], b, b[7:7]]):
        b.copy_(old)
        norms = torch.empty(1, device=DEV)
        B.MvClip(ts).mv_clip_scale(0.5, norms)
        assert bool(((b.double() - old.double() * (0.5 / float(old.double().norm()))).abs() <= 4 * 2.0 ** -24 * old.double().abs()).all())


@pytest.mark.parametrize("sizes", [[5000], [3, 20_000, 70_001]])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_a_wait_that_runs_out_is_reported(sizes, dt):
    """With no poll allowed every CTA of the one-kernel form gives up at once: what it writes is NaN, the status says so once, and the
    plan is as good as before."""
    ts = [torch.randn(n, device=DEV).to(dt) for n in sizes]
    plan = B.MvClip(ts)
    rows, norms = torch.empty((1, sum(sizes)), device=DEV), torch.empty(1, device=DEV)
    plan.mv_clip_pack(1.0, rows, norms)
    plan.mv_clip_status()
    good, n = rows.clone(), norms.clone()
    plan.mv_clip_set_polls(0)
    plan.mv_clip_pack(1.0, rows, norms)
    with pytest.raises(B.MvError) as e:
        plan.mv_clip_status()
    assert e.value.status == B.MV_ERR_TIMEOUT
    assert bool(torch.isnan(rows).all()) and torch.equal(norms, n)
    plan.mv_clip_status()                                  # reported once
    keep = [t.clone() for t in ts]
    plan.mv_clip_scale(1.0)
    with pytest.raises(B.MvError):
        plan.mv_clip_status()
    assert all(bool(torch.isnan(t).all()) for t in ts)
    for t, k in zip(ts, keep):
        t.copy_(k)
    plan.mv_clip_norm(norms)                               # no wait in it
    plan.mv_clip_status()
    plan.mv_clip_set_polls(-1)
    plan.mv_clip_pack(1.0, rows, norms)
    plan.mv_clip_status()
    assert torch.equal(rows, good) and torch.equal(norms, n)
    with pytest.raises(B.MvError):
        plan.mv_clip_set_polls(-2)
    plan.close()
    for f in (plan.mv_clip_status, lambda: plan.mv_clip_set_polls(1), lambda: plan.mv_clip_norm(norms)):
        with pytest.raises(B.MvError):
            f()


@pytest.mark.parametrize("n", [300, 6_000_000])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top,max_norm", [(2e38, 1e-8), (3e38, 0.01), (1e38, 3e-44), (1e30, 1e-20), (2e38, 0.0)])
def test_factors_below_the_normal_range(n, dt, top, max_norm):
    """max_norm / norm down to 1e-82: the product is rounded once from 64 bits, in place (then to the tensors' type) and into rows."""
    t = (torch.randn(n, generator=torch.Generator(device=DEV).manual_seed(n), device=DEV) * (top / 1e6)).to(dt)
    t[n // 2], t[-1] = top, -top / 3
    old, bound = t.double(), float(torch.tensor(max_norm))
    norm = float(old.norm())
    want = old * (bound / norm)
    plan = B.MvClip([t[: n // 3], t[n // 3:]])
    rows, norms = torch.empty((1, n), device=DEV), torch.empty(1, device=DEV)
    plan.mv_clip_pack(max_norm, rows, norms)
    assert abs(float(norms) - norm) <= 2.0 ** -23 * norm if norm < 3.4e38 else float(norms) == float("inf")
    tol = 3 * 2.0 ** -24 * want.abs() + 2.0 ** -149
    assert bool(((rows[0].double() - want).abs() <= tol).all())
    plan.mv_clip_scale(max_norm)
    lo, hi = ((want + e).float().to(dt).double() for e in (-tol, tol))
    assert bool(((t.double() >= lo) & (t.double() <= hi)).all())


@pytest.mark.parametrize("n", [300, 6_000_000])
def test_finite_groups_whose_norm_passes_the_range_are_scaled(n):
    """Their norm is reported as inf; a group that does hold an inf is left alone."""
    a, b = torch.full((n,), 2.0e38, device=DEV), torch.full((n,), 1.0, device=DEV)
    b[5] = float("inf")
    keep = b.clone()
    plan, norms = B.MvClip([a, b], [0, 1]), torch.empty(2, device=DEV)
    plan.mv_clip_scale(1.0, norms)
    assert norms.tolist() == [float("inf")] * 2 and torch.equal(b, keep)
    assert bool(((a.double() - n ** -0.5).abs() <= 3 * 2.0 ** -24 * n ** -0.5).all())
