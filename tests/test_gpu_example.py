"""The example that trains a small language model through lookup, gradient, clipping, selection and server, next to the same
training in plain torch and the oracle's selection and server."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import language_model_step
    return language_model_step


def plain_training(ex, rounds, workers, lr=0.5, max_norm=1.0, keep=(1, 4)):
    dev = torch.device("cuda", 0)
    table, matrix = ex.VOCAB * ex.DIM, ex.DIM * ex.VOCAB
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    theta = torch.randn(table + matrix, device=dev, generator=gen) * 0.05
    server = oracle.Server(theta.cpu().numpy())
    kept = oracle.keep_count(matrix, *keep)
    losses = []
    for r, batch in enumerate(ex.text(workers, rounds, dev)):
        theta = torch.from_numpy(server.theta()).to(dev).double()
        mean, updates, dense = 0.0, [], []
        for w in range(workers):
            tokens, targets = batch[w, :-1], batch[w, 1:]
            E = theta[:table].view(ex.VOCAB, ex.DIM).clone().requires_grad_()
            O = theta[table:].view(ex.DIM, ex.VOCAB).clone().requires_grad_()
            x = torch.nn.functional.embedding(tokens, E, padding_idx=0) * ex.DIM ** 0.5
            # the padding word is looked up like any other: only its gradient is left out
            x = torch.where((tokens == 0).unsqueeze(1), (E[0] * ex.DIM ** 0.5).detach(), x)
            loss = torch.nn.functional.cross_entropy(x @ O, targets, ignore_index=0)
            loss.backward()
            mean += float(loss.detach()) / workers
            norm = float((E.grad ** 2).sum() + (O.grad ** 2).sum()) ** 0.5
            c = min(1.0, max_norm / (norm + 1e-6))
            present = torch.unique(tokens[tokens != 0])
            idx = (present.view(-1, 1) * ex.DIM + torch.arange(ex.DIM, device=dev)).view(-1).cpu().numpy().astype(np.uint32)
            updates.append((idx, (E.grad * c).float().view(-1).cpu().numpy()[idx]))
            i, v = oracle.select((O.grad * c).float().view(-1).cpu().numpy(), kept)
            dense.append((i + np.uint32(table), v))
        losses.append(mean)
        pulled = 2 * workers * r
        for i, v in updates + dense:
            server.apply(i, v, pulled, lr)
    return losses


def test_training_follows_the_plain_one(example):
    """64-bit gradients on the plain side; both are rounded to fp32 before selection and server, and the two models' products
    differ by fp32 rounding (1e-6 a round); a thousandth leaves room for entries that change places at a threshold."""
    losses = example.train(rounds=12, workers=3)
    assert losses == pytest.approx(plain_training(example, 12, 3), rel=1e-3)


def test_loss_falls(example):
    losses = example.train(rounds=40, workers=3)
    tens = [sum(losses[k:k + 10]) for k in range(0, 40, 10)]
    assert tens == sorted(tens, reverse=True) and len(set(tens)) == 4
