"""GPU tests of the language-model operators strung together: embedding, layer norm, logits, distillation or log probabilities, their gradients,
clipping, the sparse step, and tokens drawn from the trained model."""
import re

import pytest
import torch

from paper_2011_06495_b200.lm_example import BigramWorkers, train

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [48, 61])
def test_steps_with_a_norm_and_a_teacher(D, dtype):
    """Runs, and (32 bits) gives the gradients of the same model in 64 bits, with targets and with a teacher."""
    kw = dict(N=2, V=300, D=D, T=600, sparsity=0.02, lr=4.0, device=DEV, dtype=dtype, norm=True)
    m = BigramWorkers(seed=3, **kw)
    s = BigramWorkers(seed=4, teacher=m, k=12, **kw)
    for model in (m, s):
        for _ in range(5):
            assert model.step() > -1e-5
        if dtype == torch.float32:
            model.check_gradients()


def test_tokens_drawn_one_after_another():
    m = BigramWorkers(N=2, V=500, D=64, T=600, device=DEV, norm=True)
    m.step()
    start = torch.arange(100, device=DEV)
    out = m.generate(start, 7, scale=1.3, top_k=40, top_p=0.95, min_p=0.01)
    assert out.shape == (7, 100) and int(out.min()) >= 0 and int(out.max()) < 500
    greedy = m.generate(start, 3, top_k=1)
    x = start
    for row in greedy:
        assert torch.equal(row, m.logits(x).float().argmax(1))
        x = row


def test_what_training_prints(capsys):
    """Loss, norms and the entropy of the predictions; a student of a teacher's alternatives has no entropy."""
    m = BigramWorkers(N=2, V=300, D=32, T=400, device=DEV)
    train(m, 2)
    train(BigramWorkers(N=2, V=300, D=32, T=400, device=DEV, teacher=m), 1)
    lines = capsys.readouterr().out.splitlines()
    number = r"-?\d+\.\d+"
    for line in lines[:2]:
        assert re.fullmatch(rf"step +\d+  loss {number}  norms {number}, {number}  entropy {number}  K = {m.K} of {m.d}", line), line
    assert re.fullmatch(rf"step +0  loss {number}  norms {number}, {number}  K = {m.K} of {m.d}", lines[2]) and len(lines) == 3
