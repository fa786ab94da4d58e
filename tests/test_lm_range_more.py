"""GPU tests of the vector, shifted and image forms of layer norm and its gradient past 2^31 elements."""
import pytest
import torch

from paper_2011_06495_b200 import binding as B
from tests.test_lm_norm import EPS, forward_reference, grad_reference, parameters
from tests.test_lm_operators import BF16, DEV, F32, gen, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,pad", [(8192, 0), (8191, 0), (8191, 1)])
def test_rows_that_fit_registers_past_32_bit_offsets(D, pad):
    """All rows but four are zero, so that the sums over rows are of four terms each: adding zeros rounds nothing."""
    ld = D + pad
    T = 2 ** 31 // ld + 3000
    x = torch.zeros((T, ld), dtype=BF16, device=DEV)[:, :D]
    rows = torch.tensor([1, 2 ** 31 // ld - 1, 2 ** 31 // ld + 1, T - 1], device=DEV)
    some = torch.randn((4, D), generator=gen(D), device=DEV).to(BF16)
    x[rows] = some
    w, b = parameters(D, F32)
    y, mean, rstd = torch.empty((T, D), dtype=BF16, device=DEV), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    B.mv_layer_norm(x, w, b, y, eps=EPS, mean=mean, rstd=rstd)
    for got, (value, off) in zip((y, mean, rstd), forward_reference(some, w, b, EPS)):
        assert bool(within(got[rows], value, off).all())
    for r in (0, 2 ** 31 // ld, T - 2):                      # nothing but the bias
        assert torch.equal(y[r], b.to(BF16)) and float(mean[r]) == 0
    dw, db = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
    ws = torch.empty(B.layer_norm_grad_workspace_bytes(T, D), dtype=torch.uint8, device=DEV)
    B.mv_layer_norm_grad(x, x, w, mean, rstd, y, dw, db, ws)
    for got, (value, off) in zip((y[rows], dw, db), grad_reference(some, some, w, mean[rows], rstd[rows])):
        assert bool(within(got, value, off).all())
    for r in (0, 2 ** 31 // ld, T - 2):
        assert bool((y[r] == 0).all())
