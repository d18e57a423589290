"""A small language model trained by several workers through the library: next-token prediction from an embedding and an
output matrix, on synthetic text.

Each round every worker looks its tokens up (scaled), and turns the gradient of the looked-up rows into the table's gradient,
which is a sparse update as it stands; the output matrix's gradient is dense.  The two are clipped together by their
global norm; the dense one is then cut down to its largest entries; the server applies both.

    python examples/language_model_step.py [--rounds 30] [--workers 4]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

VOCAB, DIM, TOKENS = 512, 64, 256            # words, width of the model, tokens per worker and round


def text(workers: int, rounds: int, device) -> torch.Tensor:
    """[rounds, workers, TOKENS + 1] words; each is followed by one of four others, word 0 fills up short sequences."""
    rng = np.random.default_rng(7)
    follows = rng.integers(1, VOCAB, (VOCAB, 4))
    out = np.zeros((rounds, workers, TOKENS + 1), dtype=np.int64)
    word = rng.integers(1, VOCAB, (rounds, workers))
    for t in range(TOKENS + 1):
        out[:, :, t] = word
        word = follows[word, rng.integers(0, 4, word.shape)]
    out[:, :, TOKENS - 10:] = 0
    return torch.from_numpy(out).to(device)


def train(rounds: int = 30, workers: int = 4, lr: float = 0.5, max_norm: float = 1.0, keep=(1, 4)):
    """The mean loss of every round."""
    from paper_1702_04683_b200 import binding
    dev = torch.device("cuda", torch.cuda.current_device())
    table_size, matrix_size = VOCAB * DIM, DIM * VOCAB
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    theta = torch.randn(table_size + matrix_size, device=dev, generator=gen) * 0.05
    scale = DIM ** 0.5

    embedding = binding.Embedding(VOCAB, DIM, max_tokens=workers * TOKENS, max_workers=workers, padding_idx=0)
    clipper = binding.Clipper()
    kept = binding.adacomp_keep_count(matrix_size, *keep)
    selector = binding.Selector(binding.segments_from([table_size], [matrix_size], [kept]), workers, dev)
    server = binding.Server(theta, history_pairs=8 * workers * (TOKENS * DIM + kept), max_window_updates=8 * workers)
    grads = torch.zeros((workers, table_size + matrix_size), device=dev)       # the workers' flat gradients

    losses = []
    for batch in text(workers, rounds, dev):
        pulled = server.pull()
        tokens, targets = batch[:, :-1], batch[:, 1:]                          # views: rows of another stride
        rows = embedding.lookup(theta[:table_size].view(VOCAB, DIM), tokens, scale=scale).requires_grad_()
        matrix = theta[table_size:].view(DIM, VOCAB).expand(workers, DIM, VOCAB).detach().requires_grad_()
        loss = torch.nn.functional.cross_entropy((rows @ matrix).transpose(1, 2), targets, ignore_index=0, reduction="none")
        loss = loss.sum(1) / (targets != 0).sum(1)
        loss.sum().backward()
        losses.append(float(loss.detach().mean()))

        idx, val, begin = embedding.grad_update(tokens, rows.grad, scale=scale, workers=workers)
        grads[:, table_size:] = matrix.grad.reshape(workers, -1)
        begin = [b * DIM for b in begin.tolist()]                              # the server wants them on the host
        val = val.view(-1)
        for w in range(workers):                                               # one norm over both gradients of a worker
            clipper.clip([val[begin[w]:begin[w + 1]], grads[w, table_size:]], max_norm)
        top_idx, top_val = selector.select(grads)

        counts = [b - a for a, b in zip(begin, begin[1:])]
        server.apply(idx.view(-1), val, begin[:-1], counts, [pulled] * workers, lr)
        server.apply(top_idx.view(-1), top_val.view(-1), [w * kept for w in range(workers)], [kept] * workers, [pulled] * workers, lr)
    assert embedding.last_error() == 0 and server.last_error() == 0 and selector.last_error()[0] == 0
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--rounds", type=int, default=30)
    ap.add_argument("--workers", type=int, default=4)
    args = ap.parse_args()
    for i, x in enumerate(train(args.rounds, args.workers)):
        print(f"round {i:3d}  loss {x:.4f}")
