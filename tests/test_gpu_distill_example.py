"""The example that trains a student with experts from a teacher's top logits: it runs, and its gradients are those of the same
model in plain torch in 64 bits."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import distill_experts_step
    return distill_experts_step


def test_it_runs(example):
    losses = example.train(rounds=3, workers=2)
    assert len(losses) == 3 and all(math.isfinite(x) for x in losses)


def plain_step(ex, theta, tokens, idx, val, lse, bias):
    """Loss, gradient of all parameters, chosen experts; everything in 64 bits, differentiated by torch."""
    flat = theta.double().clone().requires_grad_()
    p = ex.parts(flat)
    live = tokens != 0
    # the padding word is looked up like any other: only its gradient is left out
    h = p["table"][tokens] * ex.SCALE
    h = torch.where(live.unsqueeze(1), h, h.detach())
    scores = torch.sigmoid(h @ p["router"])
    experts = torch.sort(scores.detach() + bias.double(), dim=1, descending=True, stable=True).indices[:, :ex.CHOSEN]
    weights = scores.gather(1, experts)
    weights = weights / weights.sum(1, keepdim=True) * live.unsqueeze(1)
    y = h + (weights.unsqueeze(2) * torch.einsum("nd,nkde->nke", h, p["experts"][experts])).sum(1)
    logits = (y @ p["matrix"]) / ex.TEMPERATURE
    logp = torch.log_softmax(logits, 1)
    logq = val.double() / ex.TEMPERATURE - lse.double().unsqueeze(1)
    q = logq.exp()
    left = 1.0 - q.sum(1)
    rest = torch.ones_like(logp, dtype=torch.bool).scatter_(1, idx.long(), False)
    log_rest = torch.logsumexp(logp.masked_fill(~rest, -math.inf), 1)
    loss = (q * (logq - logp.gather(1, idx.long()))).sum(1) + left * (left.log() - log_rest)
    loss = (loss * live).sum() * ex.TEMPERATURE ** 2 / live.sum()
    loss.backward()
    return loss.detach(), flat.grad, torch.where(live.unsqueeze(1), experts, -1)


def test_gradients_are_those_of_the_plain_model(example):
    """fp32 products of up to 512 terms on the example's side (512 x 2^-24 of the sum of magnitudes, 3e-5), a dozen of them behind each
    other: 1e-3 of a tensor's largest gradient leaves room for sums larger than their result."""
    from paper_1702_04683_b200 import binding
    ex, dev = example, torch.device("cuda", 0)
    theta = ex.initial_parameters(dev)
    student, teacher = ex.Student(binding, dev), binding.Distiller(ex.VOCAB)
    student.bias.copy_(torch.linspace(-0.02, 0.02, ex.EXPERTS, device=dev))
    tokens = ex.text(1, 2, dev)[1, 0]
    idx, val, lse = teacher.top(ex.teacher_logits(tokens), ex.PAIRS, temperature=ex.TEMPERATURE)
    grad = torch.full_like(theta, 9.0)
    loss, counts, u_idx, u_val, begin = student.step(theta, tokens, idx, val, lse, grad)
    want_loss, want, experts = plain_step(ex, theta, tokens, idx, val, lse, student.bias)
    assert float(loss) == pytest.approx(float(want_loss), rel=1e-4)
    assert torch.equal(counts.long(), torch.bincount(experts[experts >= 0], minlength=ex.EXPERTS))
    n = int(begin[1])
    table = torch.zeros(ex.VOCAB * ex.DIM, device=dev)
    table[u_idx.view(-1)[:n * ex.DIM].long()] = u_val.view(-1)[:n * ex.DIM]
    got = dict(ex.parts(grad), table=table.view(ex.VOCAB, ex.DIM))
    for name, w in ex.parts(want).items():
        assert float((got[name].double() - w).abs().max()) <= 1e-3 * float(w.abs().max()), name
    assert bool((torch.unique(u_idx.view(-1)[:n * ex.DIM] // ex.DIM) == torch.unique(tokens[tokens != 0])).all())
