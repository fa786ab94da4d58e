"""GPU tests: a single row beside the columns of a matrix in one buffer shares no bytes with it."""
import pytest
import torch

from paper_2011_06495_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("D", [7, 64, 300])
@pytest.mark.parametrize("row", [0, 3, 39])
@pytest.mark.parametrize("left", [True, False])
def test_one_row_beside_a_matrix(D, row, left):
    g = torch.Generator(device=DEV).manual_seed(D + row)
    many, one = (slice(0, D), slice(D, 2 * D)) if left else (slice(D, 2 * D), slice(0, D))
    inside = slice(D - 1, 2 * D - 1) if left else slice(1, D + 1)
    ids = torch.tensor([11], device=DEV)
    ws = torch.empty(B.embed_grad_workspace_bytes(40, 40, D), dtype=torch.uint8, device=DEV)
    tokens = torch.zeros(40, dtype=torch.int64, device=DEV)
    calls = [
        lambda m, r: B.mv_embed(m, ids, r),                # a table, one token
        lambda m, r: B.mv_embed(r, tokens, m),             # a table of one row, many tokens
        lambda m, r: B.mv_embed_grad(m, tokens, r, ws),
        lambda m, r: B.mv_embed_grad(r, ids, m, ws),
    ]
    for call in calls:
        buf = torch.randn((40, 2 * D), generator=g, device=DEV)
        apart_m, apart_r = buf.clone(), buf.clone()
        call(apart_m[:, many], apart_r[row:row + 1, one])
        call(buf[:, many], buf[row:row + 1, one])
        assert torch.equal(buf[:, many], apart_m[:, many]) and torch.equal(buf[row:row + 1, one], apart_r[row:row + 1, one])
        rest = torch.ones(40, dtype=torch.bool, device=DEV)
        rest[row] = False
        assert torch.equal(buf[rest][:, one], apart_r[rest][:, one])
        with pytest.raises(B.MvError):
            call(buf[:, many], buf[row:row + 1, inside])


@pytest.mark.parametrize("d", [64, 1000, 200_003])
@pytest.mark.parametrize("left", [True, False])
def test_rows_beside_the_tensors_packed_into_them(d, left):
    """Every worker's tensors behind (or before) its row in one buffer; one element more and the rows are refused."""
    G, a = 5, 17
    buf = torch.randn((G, 2 * d + 2), generator=torch.Generator(device=DEV).manual_seed(d), device=DEV)
    old = buf.clone()
    at, to = (0, d + 1) if left else (d + 1, 0)                       # the tensors' columns, the rows' columns
    ts = [t for g in range(G) for t in (buf[g, at:at + a], buf[g, at + a:at + d])]
    plan = B.MvClip(ts, [g for g in range(G) for _ in range(2)])
    norms = torch.empty(G, device=DEV)
    plan.mv_clip_pack(float("inf"), buf[:, to:to + d], norms)
    want = old.clone()
    want[:, to:to + d] = old[:, at:at + d]
    assert torch.equal(buf, want)
    assert bool(((norms.double() - old[:, at:at + d].double().norm(dim=1)).abs() <= 2.0 ** -22 * norms.double()).all())
    for off in (to - 2, to - 1 if left else to + 2, at, at + 1):
        if 0 <= off and off + d <= 2 * d + 2 and (off + d > at and off < at + d):
            with pytest.raises(B.MvError):
                plan.mv_clip_pack(1.0, buf[:, off:off + d], norms)
    assert torch.equal(buf, want)
