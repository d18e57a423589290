"""A small language model with experts, taught by a larger one, trained by several workers through the library.

A teacher labels every worker's text with its top logits and their normaliser.  The student looks its tokens up, routes every position to
two of its experts, and multiplies by an output matrix; its loss is the divergence from the teacher's distribution.  The gradients go
the same way back by hand: distillation, experts, router, table.  The table's is a sparse update as it stands; the others are clipped
together with it and cut down to their largest entries; the server applies both.

    python examples/distill_experts_step.py [--rounds 30] [--workers 4]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

VOCAB, DIM, TOKENS = 512, 64, 256            # words, width of the model, tokens per worker and round
EXPERTS, CHOSEN, PAIRS = 8, 2, 24            # experts, how many a position goes to, logits that the teacher sends
TEMPERATURE, SCALE = 2.0, DIM ** 0.5
SHAPES = {"table": (VOCAB, DIM), "router": (DIM, EXPERTS), "experts": (EXPERTS, DIM, DIM), "matrix": (DIM, VOCAB)}


def parts(flat: torch.Tensor) -> dict:
    """The named parameters (or their gradients) in a flat vector."""
    sizes = [int(np.prod(s)) for s in SHAPES.values()]
    return {name: p.view(s) for (name, s), p in zip(SHAPES.items(), flat.split(sizes))}


class Student:
    def __init__(self, binding, device):
        self.embedding = binding.Embedding(VOCAB, DIM, max_tokens=TOKENS, padding_idx=0, device=device)
        self.router = binding.Router(EXPERTS, CHOSEN, score="sigmoid", renormalize=True, device=device)
        self.distiller = binding.Distiller(VOCAB, device=device)
        self.bias = torch.zeros(EXPERTS, device=device)         # raised for experts that get too little

    def logits(self, p, tokens):
        """What the backward pass needs, and the logits."""
        h = self.embedding.lookup(p["table"], tokens, scale=SCALE)
        scores = h @ p["router"]
        experts, weights, counts = self.router.route(scores, bias=self.bias, live=tokens != 0)
        chosen = p["experts"][experts.clamp(min=0).long()]                     # [n, CHOSEN, DIM, DIM]; padding has weight 0
        z = torch.einsum("nd,nkde->nke", h, chosen)
        y = h + (weights.unsqueeze(2) * z).sum(1)
        return {"h": h, "scores": scores, "experts": experts, "weights": weights, "counts": counts, "chosen": chosen, "z": z, "y": y}, y @ p["matrix"]

    def step(self, theta, tokens, idx, val, lse, grad):
        """The loss of one worker's tokens; the gradient of the dense parameters goes to `grad` (the flat one), that of the table is
        returned as an update: (loss, token counts of experts, idx, val, begin)."""
        p, g = parts(theta), parts(grad)
        f, logits = self.logits(p, tokens)
        live = (tokens != 0).float()
        weight = live * (TEMPERATURE ** 2 / live.sum())
        loss, d_logits = self.distiller.loss_grad(logits, idx, val, lse, TEMPERATURE, weight, out=logits)
        torch.matmul(f["y"].t(), d_logits, out=g["matrix"])
        dy = d_logits @ p["matrix"].t()
        dz = f["weights"].unsqueeze(2) * dy.unsqueeze(1)
        dh = dy + torch.einsum("nke,nkde->nd", dz, f["chosen"])
        outer = torch.einsum("nd,nke->nkde", f["h"], dz)
        g["experts"].zero_().index_add_(0, f["experts"].clamp(min=0).view(-1), outer.view(-1, DIM, DIM))
        d_scores = self.router.grad(f["scores"], f["experts"], torch.einsum("nke,ne->nk", f["z"], dy))
        torch.matmul(f["h"].t(), d_scores, out=g["router"])
        dh += d_scores @ p["router"].t()
        update = self.embedding.grad_update(tokens, dh, scale=SCALE)
        return (loss * weight).sum(), f["counts"], *update


def text(workers: int, rounds: int, device) -> torch.Tensor:
    """[rounds, workers, TOKENS] words; each is followed by one of four others, word 0 fills up short sequences."""
    rng = np.random.default_rng(7)
    follows = rng.integers(1, VOCAB, (VOCAB, 4))
    out = np.zeros((rounds, workers, TOKENS), dtype=np.int64)
    word = rng.integers(1, VOCAB, (rounds, workers))
    for t in range(TOKENS):
        out[:, :, t] = word
        word = follows[word, rng.integers(0, 4, word.shape)]
    out[:, :, TOKENS - 10:] = 0
    return torch.from_numpy(out).to(device)


def teacher_logits(tokens: torch.Tensor) -> torch.Tensor:
    """The teacher: a fixed table of next-word logits."""
    gen = torch.Generator(device=tokens.device)
    gen.manual_seed(3)
    return (torch.randn((VOCAB, VOCAB), device=tokens.device, generator=gen) * 2.0)[tokens].bfloat16()


def initial_parameters(device) -> torch.Tensor:
    gen = torch.Generator(device=device)
    gen.manual_seed(1)
    return torch.randn(sum(int(np.prod(s)) for s in SHAPES.values()), device=device, generator=gen) * 0.05


def train(rounds: int = 30, workers: int = 4, lr: float = 0.2, max_norm: float = 1.0, keep=(1, 4)):
    """The mean loss of every round."""
    from paper_1702_04683_b200 import binding
    dev = torch.device("cuda", torch.cuda.current_device())
    theta = initial_parameters(dev)
    table = VOCAB * DIM
    dense = theta.numel() - table
    kept = binding.adacomp_keep_count(dense, *keep)
    student, teacher, clipper = Student(binding, dev), binding.Distiller(VOCAB), binding.Clipper()
    selector = binding.Selector(binding.segments_from([table], [dense], [kept]), workers, dev)
    server = binding.Server(theta, history_pairs=8 * workers * (TOKENS * DIM + kept), max_window_updates=8 * workers)
    grads = torch.zeros((workers, theta.numel()), device=dev)

    losses = []
    for batch in text(workers, rounds, dev):
        pulled, mean, updates, load = server.pull(), 0.0, [], 0
        idx, val, lse = teacher.top(teacher_logits(batch), PAIRS, temperature=TEMPERATURE)     # for all workers at once
        for w in range(workers):
            loss, counts, *update = student.step(theta, batch[w], idx[w], val[w], lse[w], grads[w])
            n = int(update[2][1]) * DIM                                        # the server wants it on the host
            clipper.clip([update[1].view(-1)[:n], grads[w, table:]], max_norm)
            updates.append((update[0].view(-1), update[1].view(-1), n))
            mean, load = mean + float(loss) / workers, load + counts
        top_idx, top_val = selector.select(grads)
        for i, v, n in updates:
            server.apply(i, v, [0], [n], [pulled], lr)
        server.apply(top_idx.view(-1), top_val.view(-1), [w * kept for w in range(workers)], [kept] * workers, [pulled] * workers, lr)
        student.bias += 0.01 * torch.sign(load.float().mean() - load)
        losses.append(mean)
    assert student.distiller.last_error() == 0 and student.router.last_error() == 0 and student.embedding.last_error() == 0
    assert teacher.last_error() == 0 and server.last_error() == 0 and selector.last_error()[0] == 0
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--rounds", type=int, default=30)
    ap.add_argument("--workers", type=int, default=4)
    args = ap.parse_args()
    for i, x in enumerate(train(args.rounds, args.workers)):
        print(f"round {i:3d}  loss {x:.4f}")
