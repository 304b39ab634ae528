"""The distillation example end to end: the student approaches its teacher, and
its answers are among its likeliest tokens."""
import pytest
import torch

import paper_2609_34117_gb300 as sw

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sw.build.build()


def test_distillation_lowers_the_loss_and_the_student_answers():
    from paper_2609_34117_gb300 import distill as d
    model = d.Model.random(vocab=5003)
    gamma, losses = d.distill(model, steps=24, batch=96)
    assert all(x == x and x > 0 for x in losses)
    assert sum(losses[-4:]) < 0.97 * sum(losses[:4])
    again = d.distill(model, steps=24, batch=96)
    assert losses == again[1] and torch.equal(gamma, again[0])   # the same bits on every run
    tokens = torch.arange(64, device="cuda")
    u = torch.rand(64, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    out, logprob = d.answer(model, gamma, tokens, u)
    z = model.logits(model.normed(tokens, False), gamma).float()
    rank = (z > z.gather(1, out.long()[:, None])).sum(1)
    assert bool((rank < 20).all()) and bool((logprob <= 0).all())
