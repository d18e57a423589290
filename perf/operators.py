"""The cases on which the operators next to selection and apply are measured: the global gradient norm and
clipping over many tensors, and the embedding lookup with its gradient (as rows, as an update, as a dense table).

Where ``own`` is false the operators run in their plain form, elementary torch operations in 32 bits; where it is
true they are the calls a user makes of ``paper_1702_04683_b200.binding``.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6                       # the norm's guard in the clipping coefficient


# ------------------------------------------------------------------------------------------- shapes

def tensor_sizes(case):
    """The sizes of a gradient's tensors: of a small CNN, of a residual network (161 tensors), of a stack of
    transformer blocks behind an embedding table, or equal flat tensors."""
    kind = case["model"]
    if kind == "cnn":
        return [832, 51_264, 3_212_288, 10_250]
    if kind == "residual":
        sizes, inp = [9_408, 64, 64], 64
        for width, blocks in zip((64, 128, 256, 512), (3, 4, 6, 3)):
            for b in range(blocks):
                out = 4 * width
                sizes += [inp * width, width, width, 9 * width * width, width, width, width * out, out, out]
                sizes += [inp * out, out, out] if b == 0 else []
                inp = out
        return sizes + [2_048_000, 1_000]
    if kind == "blocks":
        d, f = case["dim"], case["hidden"]
        return [case["vocab"] * d] + [d, d * d, d * d, d * d, d * d, d, d * f, d * f, f * d] * case["layers"] + [d]
    return [case["entries"]] * case["tensors"]


def token_probabilities(vocab):
    """Frequencies of words: the share of the r-th most frequent falls as 1 / (r + 2.7) ** 1.05."""
    p = 1.0 / (np.arange(vocab, dtype=np.float64) + 2.7) ** 1.05
    return p / p.sum()


def distinct_tokens(case):
    """How many distinct tokens one worker's batch is expected to hold."""
    n = case["tokens"] * (1.0 - case.get("padded", 0.0))
    if case["spread"] == "even":
        return case["vocab"] * -math.expm1(n * math.log1p(-1.0 / case["vocab"])) if case["vocab"] > 1 else 1.0
    return float(-np.expm1(n * np.log1p(-token_probabilities(case["vocab"]))).sum()) if case["vocab"] > 1 else 1.0


# ------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the gradient of a small head that is tuned alone: a few short tensors, every microsecond is latency
        {"name": "clip_few_short", "op": "clip", "model": "flat", "tensors": 6, "entries": 4_097, "workers": 1,
         "list": True, "type": "f32", "out": "f32", "scale": 1.0, "max_norm": 1.0},
        # eight workers of the small CNN on one GPU, half-precision gradients with a loss scale, widened for selection
        {"name": "clip_cnn_8_workers", "op": "clip", "model": "cnn", "workers": 8,
         "list": False, "type": "f16", "out": "f32", "scale": 1.0 / 1024.0, "max_norm": 0.5},
        # one worker of the residual network, 161 separate tensors of very different sizes
        {"name": "clip_residual", "op": "clip", "model": "residual", "workers": 1,
         "list": True, "type": "f32", "out": "f32", "scale": 1.0, "max_norm": 1.0},
        # a language model's bf16 gradients, clipped into the flat fp32 buffer that selection reads
        {"name": "clip_language_model", "op": "clip", "model": "blocks", "vocab": 32_768, "dim": 1_024, "hidden": 2_816,
         "layers": 24, "workers": 1, "list": True, "type": "bf16", "out": "f32", "scale": 1.0, "max_norm": 1.0},
        # the norm alone, for monitoring or for clipping the selected pairs instead: the residual network
        {"name": "norm_residual", "op": "norm", "model": "residual", "workers": 1, "list": True, "type": "f32",
         "scale": 1.0},
        # the norm alone of sixteen workers' gradients of 25 tensors of 4,000,000 entries
        {"name": "norm_large_flat", "op": "norm", "model": "flat", "tensors": 25, "entries": 4_000_000, "workers": 16,
         "list": False, "type": "f32", "scale": 1.0},
        # lookup of one step of generation: one token for each of a few sequences
        {"name": "lookup_step", "op": "lookup", "vocab": 131_072, "dim": 4_096, "tokens": 16, "spread": "words",
         "type": "bf16", "out": "bf16", "scale": 64.0},
        # lookup of a training batch
        {"name": "lookup_batch", "op": "lookup", "vocab": 50_000, "dim": 2_048, "tokens": 32_768, "spread": "words",
         "type": "bf16", "out": "bf16", "scale": 1.0},
        # the table's gradient of a short fine-tuning batch, as rows; an odd width
        {"name": "rows_short_odd", "op": "rows", "vocab": 32_000, "dim": 513, "tokens": 700, "spread": "words",
         "workers": 1, "padded": 0.2, "type": "f32", "out": "f32", "scale": 1.0},
        # four workers' batches at once, as the updates that the server applies
        {"name": "update_4_workers", "op": "update", "vocab": 50_000, "dim": 1_024, "tokens": 8_192, "spread": "words",
         "workers": 4, "padded": 0.05, "type": "bf16", "out": "f32", "scale": 1.0},
        # the dense table's gradient in the flat buffer, an ordinary batch over a large vocabulary
        {"name": "dense_batch", "op": "dense", "vocab": 131_072, "dim": 1_024, "tokens": 16_384, "spread": "words",
         "workers": 1, "padded": 0.0, "type": "bf16", "out": "f32", "scale": 32.0},
        # a large batch: every row of the table is hit, the frequent words some ten thousand times
        {"name": "dense_large", "op": "dense", "vocab": 32_000, "dim": 2_048, "tokens": 524_288, "spread": "words",
         "workers": 1, "padded": 0.0, "type": "bf16", "out": "f32", "scale": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["clip", "clip", "norm", "lookup", "rows", "update", "dense"])
    kind = rng.choice(["f32", "bf16", "f16"])
    case = {"op": op, "type": kind, "scale": rng.choice([1.0, 0.125, 32.0])}
    if op in ("clip", "norm"):
        case["list"] = rng.random() < 0.6
        case["workers"] = 1 if case["list"] else rng.choice([1, 2, 5, 16])
        case["model"] = rng.choice(["flat", "blocks", "cnn", "residual"])
        if case["model"] == "flat":
            total = _log(rng, 20_000, 60_000_000) // case["workers"] + 1
            case["tensors"] = rng.choice([1, 3, 40, 200])
            case["entries"] = total // case["tensors"] + 1
        elif case["model"] == "blocks":
            case["dim"] = rng.randrange(64, 768)
            case |= {"vocab": _log(rng, 1_000, 50_000), "hidden": rng.randrange(128, 2_048),
                     "layers": rng.choice([1, 4, 12])}
            case["workers"] = min(case["workers"], 2)
        if op == "clip":
            case |= {"out": rng.choice(["f32", kind]), "max_norm": rng.choice([0.25, 1.0])}
        return case
    case |= {"vocab": _log(rng, 500, 150_000), "tokens": _log(rng, 1, 100_000), "spread": rng.choice(["words", "words", "even"]),
             "dim": rng.choice([64, 256, 768, 1_000, 1_024, 2_048, 4_096]) + rng.choice([0, 0, 0, 1, 2])}
    if op == "lookup":
        return case | {"out": rng.choice(["f32", kind])}
    case |= {"workers": rng.choice([1, 1, 3]), "padded": rng.choice([0.0, 0.1]), "out": rng.choice(["f32", kind])}
    if op == "update":
        case["out"] = "f32"
    most = 200_000_000          # entries of the gradient, and of the dense tables
    case["tokens"] = max(1, min(case["tokens"], most // (case["dim"] * case["workers"])))
    if op == "dense" or op == "update":
        case["vocab"] = max(2, min(case["vocab"], most // (case["dim"] * case["workers"])))
    return case


# ------------------------------------------------------------------------------------------- inputs

def _tokens(case, gen, count):
    if case["spread"] == "even":
        return torch.randint(case["vocab"], (count,), device="cuda", generator=gen)
    cdf = torch.from_numpy(np.cumsum(token_probabilities(case["vocab"]))).cuda()
    at = torch.searchsorted(cdf, torch.rand(count, device="cuda", generator=gen, dtype=torch.float64))
    return at.clamp_(max=case["vocab"] - 1)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, kind = case["op"], TYPES[case["type"]]
    state = dict(case)
    if op in ("clip", "norm"):
        sizes = tensor_sizes(case)
        total, W = sum(sizes), case["workers"]
        # entries of about 1e-2 (times the loss scale that `scale` takes back), tensors of different magnitude
        flat = torch.randn((W, total), device="cuda", generator=gen)
        spread = torch.rand((W, len(sizes)), device="cuda", generator=gen) * 0.02 / case["scale"]
        for part, s in zip(flat.split(sizes, dim=1), spread.split(1, dim=1)):
            part.mul_(s)
        flat = flat.to(kind)
        state["grads"] = [g.clone() for g in flat[0].split(sizes)] if case["list"] else flat
        if op == "clip":
            buf = torch.zeros((W, total), device="cuda", dtype=TYPES[case["out"]])
            state["buffer"] = list(buf[0].split(sizes)) if case["list"] else buf
        return state
    W, V, D = case.get("workers", 1), case["vocab"], case["dim"]
    tokens = _tokens(case, gen, W * case["tokens"]).view(W, -1)
    if op == "lookup":
        state["ids"] = tokens[0]
        state["table"] = torch.randn((V, D), device="cuda", generator=gen).mul_(0.02).to(kind)
    else:
        pad = V - 1             # the token that fills sequences up: its gradient is left out
        if case["padded"]:
            tokens[torch.rand(tokens.shape, device="cuda", generator=gen) < case["padded"]] = pad
        state["ids"], state["pad"] = tokens, pad
        state["grad"] = torch.randn((W * case["tokens"], D), device="cuda", generator=gen).to(kind).view(W, -1, D)
        # how many distinct tokens the batch holds: the loader, which has the tokens on the host, knows it
        keys = tokens + torch.arange(W, device="cuda").view(-1, 1) * V
        state["distinct"] = int(torch.unique(keys[tokens != pad]).numel())
        # the buffers that such a program keeps for the results; of the lists only the front is written
        N, out = tokens.numel(), TYPES[case["out"]]
        if op == "dense":
            state["buffer"] = torch.zeros((W, V, D), device="cuda", dtype=out)
        else:
            state["values"] = torch.zeros((N, D), device="cuda", dtype=out)
            state["names"] = torch.zeros((N, D) if op == "update" else N, device="cuda", dtype=torch.int32)
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:                     # the handle with its workspace, which a program makes once for its layout
        from paper_1702_04683_b200 import binding
        W = case.get("workers", 1)
        if case["op"] in ("clip", "norm"):
            state["handle"] = binding.Clipper(max_workers=W)
            if case["list"]:    # and the list of its gradient tensors, whose places stay the same from step to step
                state["list"] = binding.GradList(state["grads"], out=state.get("buffer"))
        else:
            state["handle"] = binding.Embedding(case["vocab"], case["dim"], max_tokens=W * case["tokens"],
                                                max_workers=W, padding_idx=state.get("pad"))
    return state


# ------------------------------------------------------------------------------------------- one pass

def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    op, h = s["op"], s["handle"]
    if op == "norm":
        return h.norm(s["list"] or s["grads"], scale=s["scale"])
    if op == "clip":
        if s["list"]:
            out, norm = h.clip(s["list"], s["max_norm"], scale=s["scale"])
        else:
            out, norm = h.clip(s["grads"], s["max_norm"], scale=s["scale"], out=s["buffer"])
        return {"out": _joined(out), "norm": norm}
    if op == "lookup":
        return h.lookup(s["table"], s["ids"], scale=s["scale"], dtype=TYPES[s["out"]])
    if op == "dense":
        return h.grad_dense(s["ids"], s["grad"], s["buffer"], scale=s["scale"], workers=s["workers"])
    if op == "rows":
        rows, values, begin = h.grad_rows(s["ids"], s["grad"], scale=s["scale"], workers=s["workers"], rows_out=s["names"], values_out=s["values"])
        return {"rows": rows, "values": values, "begin": begin}
    idx, val, begin = h.grad_update(s["ids"], s["grad"], scale=s["scale"], workers=s["workers"], idx_out=s["names"], val_out=s["values"])
    return {"idx": idx, "val": val, "begin": begin}


def _joined(out):
    """The flat buffer that a list of output tensors was cut from."""
    return out[0]._base if isinstance(out, list) else out


def _plain(s):
    op = s["op"]
    if op in ("norm", "clip"):
        g = s["grads"]
        if s["list"]:
            squares = torch.stack([t.float().square().sum() for t in g]).sum().view(1)
        else:
            squares = g.float().square().sum(1)
        norm = squares.sqrt() * abs(s["scale"])
        if op == "norm":
            return norm
        factor = (s["max_norm"] / (norm + EPS)).clamp(max=1.0) * s["scale"]
        if s["list"]:
            [o.copy_(t.float() * factor) for o, t in zip(s["buffer"], g)]
        else:
            s["buffer"].copy_(g.float() * factor.view(-1, 1))
        return {"out": _joined(s["buffer"]), "norm": norm}
    if op == "lookup":
        return (s["table"][s["ids"]].float() * s["scale"]).to(TYPES[s["out"]])
    W, V, D = s["workers"], s["vocab"], s["dim"]
    ids, kind = s["ids"], TYPES[s["out"]]
    keys = ids + torch.arange(W, device=ids.device).view(-1, 1) * V
    grad = s["grad"].float().masked_fill((ids == s["pad"]).unsqueeze(-1), 0.0).view(-1, D)
    if op == "dense":
        table = torch.zeros((W * V, D), device=ids.device).index_add_(0, keys.view(-1), grad)
        return s["buffer"].copy_((table * s["scale"]).view(W, V, D))
    hit = torch.zeros(W * V, dtype=torch.bool, device=ids.device)
    hit[keys.view(-1)] = True
    hit.view(W, V)[:, s["pad"]] = False
    begin = torch.nn.functional.pad(hit.view(W, V).sum(1).cumsum(0), (1, 0))
    at = hit.cumsum(0) - 1
    slot = torch.where(hit[keys], at[keys], s["distinct"]).view(-1)       # padding goes to one row too many
    sums = torch.zeros((s["distinct"] + 1, D), device=ids.device).index_add_(0, slot, grad)[:-1]
    s["values"][:s["distinct"]] = sums * s["scale"]
    rows = hit.nonzero().view(-1) % V
    if op == "rows":
        s["names"][:s["distinct"]] = rows
        return {"rows": s["names"], "values": s["values"], "begin": begin}
    s["names"][:s["distinct"]] = rows.view(-1, 1) * D + torch.arange(D, device=ids.device)
    return {"idx": s["names"], "val": s["values"], "begin": begin}


# ------------------------------------------------------------------------------------------- what cannot be saved, what is right

def work(case):
    """Each input read once, each output written once; of a table only the rows that are looked up."""
    op, a = case["op"], SIZE[case["type"]]
    if op in ("norm", "clip"):
        n = sum(tensor_sizes(case)) * case["workers"]
        if op == "norm":
            return {"bytes": n * a + 4 * case["workers"], "flops": 2 * n}
        return {"bytes": n * (a + SIZE[case["out"]]) + 4 * case["workers"], "flops": 3 * n}
    D, W, b = case["dim"], case.get("workers", 1), SIZE[case["out"]]
    N, U = W * case["tokens"], W * distinct_tokens(case)
    if op == "lookup":
        return {"bytes": U * D * a + N * (8 + D * b), "flops": N * D}
    live = N * (1.0 - case["padded"])
    rows_written = W * case["vocab"] if op == "dense" else U
    extra = 4 * U if op == "rows" else 4 * U * D if op == "update" else 0
    return {"bytes": live * D * a + N * 8 + rows_written * D * b + extra, "flops": live * D + U * D}


def exact(case, seed):
    """The definitions in 64 bits: sums as differences of running sums over the sorted tokens, norms by dot products."""
    s = _inputs(case, seed)
    op, scale = case["op"], float(case["scale"])
    if op in ("norm", "clip"):
        per_worker = [torch.cat([t.view(-1) for t in s["grads"]])] if case["list"] else list(s["grads"])
        norms = []
        for g in per_worker:
            parts = [float(torch.dot(p.double(), p.double())) for p in g.split(1 << 26)]
            norms.append(abs(scale) * math.sqrt(math.fsum(parts)))
        norm = torch.tensor(norms, dtype=torch.float64)
        if op == "norm":
            return norm
        rows = [g.double() * (scale * min(1.0, case["max_norm"] / (n + EPS))) for g, n in zip(per_worker, norms)]
        out = rows[0] if case["list"] else torch.stack(rows)
        return {"out": out, "norm": norm}
    if op == "lookup":
        return torch.index_select(s["table"], 0, s["ids"]).double().mul_(scale)
    V, D, N = case["vocab"], case["dim"], case["workers"] * case["tokens"]
    where = torch.arange(N, device="cuda")
    keys = s["ids"].reshape(-1) + where // case["tokens"] * V
    keys = torch.where(s["ids"].reshape(-1) == s["pad"], torch.full_like(keys, case["workers"] * V), keys)
    order = torch.argsort(keys, stable=True)
    live = int((keys < case["workers"] * V).sum())
    order = order[:live]
    found, counts = torch.unique_consecutive(keys[order], return_counts=True)
    ends = counts.cumsum(0)
    grad = s["grad"].reshape(N, D)
    values = torch.zeros((N, D), dtype=torch.float64, device="cuda")
    for lo in range(0, D, 256):                                 # some columns at a time: the running sums are large
        run_sum = grad[:, lo:lo + 256][order].double().cumsum(0)
        upto = run_sum[ends - 1]
        values[:len(found), lo:lo + 256] = upto
        values[1:len(found), lo:lo + 256] -= upto[:-1]
    values *= scale
    if op == "dense":
        table = torch.zeros((case["workers"] * V, D), dtype=torch.float64, device="cuda")
        table[found] = values[:len(found)]
        return table.view(case["workers"], V, D)
    if op == "rows":
        return {"rows": None, "begin": None, "values": values}
    return {"idx": None, "val": values, "begin": None}
