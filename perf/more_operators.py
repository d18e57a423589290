"""The cases on which the row-wise selections of a language model's worker are measured: a teacher's top logits and the
distillation loss with its gradient, and the routing of tokens to experts with its gradient.

Where ``own`` is false the operators run in their plain form, elementary torch operations in 32 bits (64 for the teacher's
few probabilities and for the scores that experts are chosen by); where it is true they are the calls a user makes of
``paper_1702_04683_b200.binding``.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


# ------------------------------------------------------------------------------------------- cases

def _top(name, rows, vocab, k, kind, temperature=1.0, unused=0):
    return {"name": name, "op": "top", "rows": rows, "vocab": vocab, "k": k, "type": kind, "temperature": temperature,
            "unused": unused}


def _distill(name, form, rows, vocab, k, kind, pairs_type, temperature=1.0, tail=False, ragged=False, padded=0.0):
    return {"name": name, "op": "distill", "form": form, "rows": rows, "vocab": vocab, "k": k, "type": kind,
            "pairs_type": pairs_type, "temperature": temperature, "tail": tail, "ragged": ragged, "padded": padded}


def _route(name, form, rows, experts, k, kind, score, renormalize, bias=False, groups=1, top_groups=1, group_terms=1,
           scale=1.0, padded=0.0):
    return {"name": name, "op": "route", "form": form, "rows": rows, "experts": experts, "k": k, "type": kind,
            "score": score, "renormalize": renormalize, "bias": bias, "groups": groups, "top_groups": top_groups,
            "group_terms": group_terms, "scale": scale, "padded": padded}


def listed():
    return [
        # a teacher answers as it generates: one new token for each of a few sequences
        _top("top_step", 16, 131_072, 32, "bf16"),
        # a teacher labels a training batch, softened
        _top("top_batch", 8_192, 50_000, 64, "bf16", temperature=2.0),
        # fp32 logits over a vocabulary of odd size, whose last entries are unused and masked
        _top("top_masked_odd", 1_537, 32_001, 100, "f32", unused=501),
        # a short fine-tuning batch
        _distill("distill_short", "loss_grad", 64, 32_000, 16, "bf16", "bf16"),
        # a training batch, the teacher's few largest logits renormalised, softened
        _distill("distill_batch", "loss_grad", 8_192, 50_000, 64, "bf16", "bf16", temperature=2.0),
        # a large vocabulary, the teacher's remaining probability kept as one more class
        _distill("distill_large_tail", "loss_grad", 4_096, 131_072, 128, "bf16", "f32", tail=True),
        # loss and gradient as two calls (another loss is added in between); a padded batch, lists of different length
        _distill("distill_ragged_odd", "two", 1_025, 50_001, 48, "f16", "f16", ragged=True, padded=0.15),
        # the loss alone, for evaluation, on fp32 logits
        _distill("distill_evaluate", "loss", 2_048, 65_536, 64, "f32", "f32", temperature=1.5, tail=True),
        # one step of generation
        _route("route_step", "choose", 16, 64, 6, "f32", "softmax", False),
        # many experts in groups, a bias that balances them
        _route("route_groups", "choose", 16_384, 256, 8, "bf16", "sigmoid", True, bias=True, groups=8, top_groups=4,
               group_terms=2, scale=2.5),
        # training with an odd number of experts: the choice, and the scores' gradient through all of the row
        _route("route_odd_train", "train", 20_001, 60, 4, "f16", "softmax", False, bias=True, padded=0.1),
        # training on a large batch: the choice and the gradient of renormalised weights
        _route("route_train", "train", 65_536, 128, 8, "f32", "softmax", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["top", "distill", "distill", "route", "route"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op == "route":
        experts = rng.choice([8, 16, 64, 128, 256, 512, rng.randrange(3, 400)])
        groups = rng.choice([g for g in range(1, 17) if experts % g == 0]) if rng.random() < 0.5 else 1
        top_groups = rng.randint(1, groups)
        k = rng.randint(1, min(12, experts // groups * top_groups))
        rows = _log(rng, 1, 16_000_000 // (experts * (8 if experts < 64 else 2)))
        return _route(None, rng.choice(["choose", "train"]), rows, experts, k, kind, rng.choice(["softmax", "sigmoid"]),
                      rng.random() < 0.6, rng.random() < 0.6, groups, top_groups, rng.choice([1, 2]),
                      rng.choice([1.0, 2.5]), rng.choice([0.0, 0.2])) | _unnamed
    vocab = _log(rng, 2_000, 150_000) if rng.random() < 0.5 else rng.choice([32_000, 50_000, 65_536, 128_000, 131_072])
    k = min(vocab, _log(rng, 1, 300))
    rows = _log(rng, 1, min(20_000, (200_000_000 if op == "distill" else 150_000_000) // vocab))
    temperature = rng.choice([1.0, 1.0, 2.0, 0.7])
    if op == "top":
        return _top(None, rows, vocab, k, kind, temperature, rng.choice([0, vocab // 100])) | _unnamed
    return _distill(None, rng.choice(["loss_grad", "loss_grad", "two", "loss"]), rows, vocab, k, kind, rng.choice([kind, "f32"]),
                    temperature, rng.random() < 0.5, rng.random() < 0.4, rng.choice([0.0, 0.1])) | _unnamed


_unnamed = {"name": ""}


# ------------------------------------------------------------------------------------------- inputs

def _blocks(rows, vocab):
    """Stretches of rows of some hundred megabytes in 32 bits."""
    step = max(1, (1 << 26) // vocab)
    return [(at, min(rows, at + step)) for at in range(0, rows, step)]


def _frequency(case, gen):
    """What every token's logit owes to its frequency: the r-th most frequent one's falls as 1.05 log r, in any order."""
    rank = torch.randperm(case["vocab"], device="cuda", generator=gen).float()
    return (rank + 2.7).log_().mul_(-1.05)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    state, kind = dict(case), TYPES[case["type"]]
    N = case["rows"]
    if case["op"] == "route":
        E, k = case["experts"], case["k"]
        state["logits"] = (torch.randn((N, E), device="cuda", generator=gen) * 1.5).to(kind)
        state["biases"] = torch.randn(E, device="cuda", generator=gen) * (0.05 if case["score"] == "sigmoid" else 0.01) if case["bias"] else None
        live = torch.rand(N, device="cuda", generator=gen) >= case["padded"]
        state["live"] = live if case["padded"] else None
        if case["form"] == "train":             # what comes back from the experts' products
            state["grad_weights"] = torch.randn((N, k), device="cuda", generator=gen)
        return state
    V, K, T = case["vocab"], case["k"], case["temperature"]
    frequency = _frequency(case, gen)
    state["logits"] = torch.empty((N, V), device="cuda", dtype=kind)
    if case["op"] == "top":
        unused = torch.arange(V, device="cuda") >= V - case["unused"]
        for lo, hi in _blocks(N, V):
            x = torch.randn((hi - lo, V), device="cuda", generator=gen).mul_(2.5).add_(frequency)
            state["logits"][lo:hi] = x.masked_fill_(unused, -math.inf)
        return state
    # the teacher's logits and a student's that resemble them; of the teacher's the largest are sent
    given = TYPES[case["pairs_type"]]
    idx = torch.empty((N, K), device="cuda", dtype=torch.int32)
    val = torch.empty((N, K), device="cuda", dtype=given)
    lse = torch.empty(N, device="cuda")
    for lo, hi in _blocks(N, V):
        x = torch.randn((hi - lo, V), device="cuda", generator=gen).mul_(2.5).add_(frequency)
        noise = torch.randn((hi - lo, V), device="cuda", generator=gen)
        state["logits"][lo:hi] = torch.add(x, noise, alpha=0.8)
        x = x.to(given).float()
        top = torch.topk(x, K, dim=1)
        val[lo:hi], idx[lo:hi] = top.values.to(given), top.indices.int()
        lse[lo:hi] = torch.logsumexp(x.div_(T), 1)
    dead = torch.rand(N, device="cuda", generator=gen) < case["padded"]
    if case["ragged"]:                          # the entries that make up the nucleus; the rest of the list is empty
        length = torch.randint(1, K + 1, (N, 1), device="cuda", generator=gen)
        idx.masked_fill_(torch.arange(K, device="cuda") >= length, -1)
    idx.masked_fill_(dead.view(-1, 1), -1)
    state |= {"idx": idx, "val": val, "lse": lse if case["tail"] else None}
    # the mean over the batch's tokens, and the loss scale of fp16 training
    scale = 65_536.0 if case["type"] == "f16" else 1.0
    state["weight"] = (~dead).float() * (T * T * scale / max(1.0, N * (1.0 - case["padded"])))
    if case["form"] != "loss":
        state["buffer"] = torch.empty((N, V), device="cuda", dtype=kind)
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:                     # the handle, which a program makes once for its model
        from paper_1702_04683_b200 import binding
        if case["op"] == "route":
            state["handle"] = binding.Router(case["experts"], case["k"], score=case["score"], groups=case["groups"],
                                             top_groups=case["top_groups"], group_terms=case["group_terms"],
                                             renormalize=case["renormalize"], scale=case["scale"])
        else:
            state["handle"] = binding.Distiller(case["vocab"])
    return state


# ------------------------------------------------------------------------------------------- one pass

def run(state):
    return _own(state) if own else {"top": _plain_top, "distill": _plain_distill, "route": _plain_route}[state["op"]](state)


def _own(s):
    h = s["handle"]
    if s["op"] == "top":
        idx, val, lse = h.top(s["logits"], s["k"], temperature=s["temperature"])
        return {"idx": idx, "val": val, "lse": lse}
    if s["op"] == "route":
        experts, weights, counts = h.route(s["logits"], bias=s["biases"], live=s["live"])
        out = {"experts": experts, "weights": weights, "counts": counts}
        if s["form"] == "train":
            out["grad"] = h.grad(s["logits"], experts, s["grad_weights"])
        return out
    given = {"lse": s["lse"], "temperature": s["temperature"], "weight": s["weight"]}
    if s["form"] == "loss_grad":
        loss, grad = h.loss_grad(s["logits"], s["idx"], s["val"], out=s["buffer"], **given)
        return {"loss": loss, "grad": grad}
    loss, stats = h.loss(s["logits"], s["idx"], s["val"], **given)
    if s["form"] == "loss":
        return {"loss": loss}
    return {"loss": loss, "grad": h.grad(s["logits"], s["idx"], s["val"], stats, out=s["buffer"], **given)}


def _plain_top(s):
    x, V = s["logits"], s["vocab"]
    bits = x.float().add_(0.0).view(torch.int32)                 # -0 becomes +0
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32    # of the values, as whole numbers
    order |= 0xFFFFFFFF - torch.arange(V, device=x.device)       # ties: the lowest index first
    idx = 0xFFFFFFFF - (torch.topk(order, s["k"], dim=1).values & 0xFFFFFFFF)
    z = x.float()
    most = z.amax(1, keepdim=True)
    lse = ((z - most).div_(s["temperature"])).exp_().sum(1).log_() + most.view(-1) / s["temperature"]
    return {"idx": idx.int(), "val": x.gather(1, idx), "lse": lse}


def _plain_distill(s):
    T, idx, weight = s["temperature"], s["idx"].long(), s["weight"]
    sent = idx >= 0
    at = torch.where(sent, idx, idx[:, :1].clamp(min=0))         # an entry that is not there points at the row's first
    live = (weight != 0) & sent.any(1)
    x = s["logits"].float()
    most = x.amax(1, keepdim=True)
    e = (x - most).div_(T).exp_()
    total = e.sum(1, keepdim=True)
    # the loss is a difference of logarithms that nearly cancel: those few are taken in 64 bits
    logp = (x.gather(1, at).double() - most.double()) / T - total.double().log()
    t = (s["val"].double() / T).masked_fill(~sent, -math.inf)
    if s["lse"] is None:
        t = t - t.amax(1, keepdim=True).nan_to_num(neginf=0.0)
        logq = t - t.exp().sum(1, keepdim=True).log()
    else:
        logq = t - s["lse"].double().view(-1, 1)
    q = torch.where(sent, logq.exp(), 0.0)
    loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1)
    mass = q.sum(1, keepdim=True)
    if s["lse"] is not None:
        rest = e.scatter(1, at, 0.0).sum(1, keepdim=True).double()
        q_rest = torch.where(rest > 0, (1.0 - mass).clamp(min=0.0), 0.0)
        loss += torch.where(q_rest > 0, q_rest * (q_rest.log() - rest.log() + total.double().log()), 0.0).view(-1)
        mass = mass + q_rest
    loss = torch.where(live, loss, 0.0).float()
    if s["form"] == "loss":
        return {"loss": loss}
    g = torch.where(live, weight / T, 0.0).view(-1, 1)
    share = (mass / total).float()
    top = e.gather(1, at) * share
    if s["lse"] is not None:
        share = share - torch.where(q_rest > 0, q_rest / rest, 0.0).float()
    grad = e.mul_(share * g)
    top = torch.where(sent, (top - q.float()) * g, 0.0)
    # entries that are not there are left out: they would write next to the row's first
    grad.view(-1)[(torch.arange(len(at), device=at.device).view(-1, 1) * s["vocab"] + at)[sent]] = top[sent]
    grad[~live] = 0.0
    s["buffer"].copy_(grad)
    return {"loss": loss, "grad": s["buffer"]}


def _choice(s, scores):
    """What experts are chosen by: the score and the bias, -Inf outside of the best groups."""
    choice = scores if s["biases"] is None else scores + s["biases"].to(scores.dtype)
    if s["groups"] > 1:
        N, E, G = len(choice), s["experts"], s["groups"]
        inside = choice.view(N, G, E // G)
        best = inside.sort(dim=2, descending=True).values[:, :, :min(s["group_terms"], E // G)].sum(2)
        order = best.sort(dim=1, descending=True, stable=True).indices
        kept = torch.zeros((N, G), dtype=torch.bool, device=choice.device).scatter_(1, order[:, :s["top_groups"]], True)
        choice = inside.masked_fill(~kept.unsqueeze(2), -math.inf).view(N, E)
    return choice


def _plain_route(s):
    x, k = s["logits"].float(), s["k"]
    if s["score"] == "softmax":
        e = (x - x.amax(1, keepdim=True)).exp_()
        scores = e / e.sum(1, keepdim=True)
        wide = (x.double() - x.double().amax(1, keepdim=True)).exp_()
        wide = wide / wide.sum(1, keepdim=True)
    else:
        scores = 1.0 / (1.0 + (-x).exp_())
        wide = 1.0 / (1.0 + (-x.double()).exp_())
    chosen = _choice(s, wide).sort(dim=1, descending=True, stable=True).indices[:, :k]
    raw = scores.gather(1, chosen)
    total = raw.sum(1, keepdim=True) if s["renormalize"] else torch.ones_like(raw[:, :1])
    weights = s["scale"] * raw / total
    live = torch.ones(len(x), dtype=torch.bool, device=x.device) if s["live"] is None else s["live"]
    live = live.view(-1, 1)
    counts = torch.zeros(s["experts"], dtype=torch.int32, device=x.device)
    counts.index_add_(0, chosen.reshape(-1), live.expand(-1, k).reshape(-1).int())
    out = {"experts": torch.where(live, chosen, -1).int(), "weights": torch.where(live, weights, 0.0), "counts": counts}
    if s["form"] == "train":
        d = s["grad_weights"] * s["scale"]
        if s["renormalize"]:
            d = (d - (d * raw).sum(1, keepdim=True) / total) / total
        if s["score"] == "softmax":
            g = torch.zeros_like(scores).scatter_(1, chosen, d * raw) - scores * (d * raw).sum(1, keepdim=True)
        else:
            g = torch.zeros_like(scores).scatter_(1, chosen, d * raw / (1.0 + x.gather(1, chosen).exp()))
        out["grad"] = torch.where(live, g, 0.0).to(s["logits"].dtype)
    return out


# ------------------------------------------------------------------------------------------- what cannot be saved, what is right

def work(case):
    """Each input read once, each output written once; of rows that count for nothing the logits are not read."""
    N, a, k = case["rows"], SIZE[case["type"]], case["k"]
    if case["op"] == "top":
        return {"bytes": N * (case["vocab"] * a + k * (4 + a) + 4), "flops": 5 * N * case["vocab"]}
    alive = N * (1.0 - case["padded"])
    if case["op"] == "distill":
        V = case["vocab"]
        few = N * (k * 4 + 8) + alive * k * SIZE[case["pairs_type"]] + (4 * N if case["tail"] else 0)
        written = 0 if case["form"] == "loss" else N * V * a
        return {"bytes": alive * V * a + written + few, "flops": alive * V * (4 if case["form"] == "loss" else 7)}
    E = case["experts"]
    few = N * k * 8 + 4 * E * (2 if case["bias"] else 1) + (N if case["padded"] else 0)
    if case["form"] == "train":
        few += alive * k * 4 + N * E * a
    return {"bytes": alive * E * a + few, "flops": alive * E * (6 + k)}


def exact(case, seed):
    """The definitions in 64 bits, some rows at a time; gradients by differentiating them."""
    s = _inputs(case, seed)
    return {"top": _exact_top, "distill": _exact_distill, "route": _exact_route}[case["op"]](s)


def _exact_top(s):
    N, V, k = s["rows"], s["vocab"], s["k"]
    idx, lse = torch.empty((N, k), dtype=torch.int32, device="cuda"), torch.empty(N, dtype=torch.float64, device="cuda")
    for lo, hi in _blocks(N, V):
        x = s["logits"][lo:hi].double()
        idx[lo:hi] = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
        lse[lo:hi] = torch.logsumexp(x / s["temperature"], 1)
    return {"idx": idx, "val": s["logits"].gather(1, idx.long()).double(), "lse": lse}


def _exact_distill(s):
    N, V, T = s["rows"], s["vocab"], s["temperature"]
    losses = torch.zeros(N, dtype=torch.float64, device="cuda")
    grads = torch.zeros((N, V), dtype=torch.float64, device="cuda") if s["form"] != "loss" else None
    for lo, hi in _blocks(N, V):
        idx = s["idx"][lo:hi].long()
        sent = idx >= 0
        rows = ((s["weight"][lo:hi] != 0) & sent.any(1)).nonzero().view(-1)
        if len(rows) == 0:
            continue
        idx, sent = idx[rows], sent[rows]
        x = s["logits"][lo:hi][rows].double().requires_grad_()
        logp = torch.log_softmax(x / T, 1)
        t = (s["val"][lo:hi][rows].double() / T).masked_fill(~sent, -math.inf)
        logq = torch.log_softmax(t, 1) if s["lse"] is None else t - s["lse"][lo:hi][rows].double().view(-1, 1)
        at = torch.where(sent, idx, torch.zeros_like(idx))
        terms = torch.exp(logq) * (logq.masked_fill(~sent, 0.0) - logp.gather(1, at))
        loss = terms.masked_fill(~sent, 0.0).sum(1)
        if s["lse"] is not None:
            listed_ = torch.zeros((len(rows), V + 1), dtype=torch.bool, device="cuda")
            listed_.scatter_(1, torch.where(sent, idx, V), True)
            log_rest = torch.logsumexp(logp.masked_fill(listed_[:, :V], -math.inf), 1)
            q_rest = -torch.expm1(torch.logsumexp(logq, 1))
            there = (q_rest > 0) & (log_rest > -math.inf)
            loss = loss + torch.where(there, q_rest * (q_rest.clamp(min=1e-300).log() - log_rest.clamp(min=-1e300)), 0.0)
        losses[lo + rows] = loss.detach()
        if grads is not None:
            (loss * s["weight"][lo:hi][rows].double()).sum().backward()
            grads[lo + rows] = x.grad
    return {"loss": losses} if grads is None else {"loss": losses, "grad": grads}


def _exact_route(s):
    N, E, k = s["rows"], s["experts"], s["k"]
    x = s["logits"].double().requires_grad_()
    scores = torch.softmax(x, 1) if s["score"] == "softmax" else torch.sigmoid(x)
    with torch.no_grad():                       # the best expert, k times over; first the best groups
        left = scores.detach().clone() if s["biases"] is None else scores.detach() + s["biases"].double()
        if s["groups"] > 1:
            each = left.reshape(N, s["groups"], -1)
            best = torch.topk(each, min(s["group_terms"], each.shape[2]), dim=2).values.sum(2)
            outside = torch.ones_like(best, dtype=torch.bool)
            for _ in range(s["top_groups"]):
                first = (best == best.amax(1, keepdim=True)).int().argmax(1, keepdim=True)
                outside.scatter_(1, first, False)
                best.scatter_(1, first, -math.inf)
            left = each.masked_fill(outside.unsqueeze(2), -math.inf).reshape(N, E)
        chosen = torch.empty((N, k), dtype=torch.int64, device="cuda")
        for j in range(k):
            chosen[:, j] = (left == left.amax(1, keepdim=True)).int().argmax(1)
            left.scatter_(1, chosen[:, j:j + 1], -math.inf)
    weights = scores.gather(1, chosen)
    if s["renormalize"]:
        weights = weights / weights.sum(1, keepdim=True)
    weights = weights * s["scale"]
    live = torch.ones(N, dtype=torch.bool, device="cuda") if s["live"] is None else s["live"]
    weights = torch.where(live.view(-1, 1), weights, 0.0)
    out = {"experts": torch.where(live.view(-1, 1), chosen, -1).int(), "weights": weights.detach(),
           "counts": torch.bincount(chosen[live].view(-1), minlength=E).int()}
    if s["form"] == "train":
        (weights * s["grad_weights"].double()).sum().backward()
        out["grad"] = x.grad
    return out
