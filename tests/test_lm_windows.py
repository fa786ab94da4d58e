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
