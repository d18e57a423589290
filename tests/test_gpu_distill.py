"""A teacher's top logits and the distillation loss with its gradient, through the binding, against plain implementations in 64 bits.

Tolerances.  A probability is e / Z with e = 2^y computed by one approximate exponential (2 units in the last of 23 bits, 2^-22) from an
argument with three roundings (|y| 3 2^-24, in base 2), and Z a sum of positive terms with the same errors, added in fp32 in chains of at
most vocab / 128 + 32 terms: relative to p that is at most
    P = 2^-22 + 2^-22 + (vocab / 128 + 32) 2^-24 + 3 2^-24 |log2 p| + (what the arguments contribute to Z, at most the same again).
A gradient w (W p - q) / T has this error in p, some 8 roundings of 2^-24 and the q's (2^-22), and is rounded once to its type: half of
torch.finfo(t).eps relative, half of the smallest subnormal absolute.  The loss has the error of log Z and of terms q (log q - log p) which are
formed in 64 bits from q with 2^-22 relative.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SUBNORMAL = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}   # exponentials below 2^-126 are zero


@pytest.fixture(scope="module")
def binding():
    from paper_1702_04683_b200 import binding as b
    return b


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def logits_like(n, vocab, kind, seed, spread=2.5):
    return (torch.randn((n, vocab), device="cuda", generator=gen(seed)) * spread).to(TYPES[kind])


# ------------------------------------------------------------------------------------------- top logits

def plain_top(x, k, temperature):
    wide = x.double()
    order = torch.where(wide.isnan(), math.inf, wide)
    # NaN above everything, also above +Inf: two keys, the second by a stable sort
    first = torch.sort(order, dim=-1, descending=True, stable=True).indices
    nan = wide.isnan().gather(-1, first)
    second = torch.sort(nan.int(), dim=-1, descending=True, stable=True).indices
    idx = first.gather(-1, second)[..., :k]
    return idx, x.gather(-1, idx), torch.logsumexp(wide / temperature, -1)


def check_top(binding, x, k, temperature=1.0, d=None):
    d = d or binding.Distiller(x.shape[-1])
    idx, val, lse = d.top(x, k, temperature=temperature)
    want_idx, want_val, want_lse = plain_top(x, k, temperature)
    assert idx.shape == want_idx.shape and val.dtype == x.dtype and lse.shape == x.shape[:-1]
    assert torch.equal(idx.long(), want_idx)
    bits = torch.int32 if x.dtype == torch.float32 else torch.int16
    assert torch.equal(val.contiguous().view(bits), want_val.contiguous().view(bits))
    special = ~torch.isfinite(want_lse)
    spoilt = (x.isnan() | (x == math.inf)).any(-1)
    assert torch.equal(lse.isnan(), spoilt)
    assert torch.equal((lse == -math.inf), special & (want_lse == -math.inf))
    ok = ~special
    tol = 2.0 ** -22 * 4 + (x.shape[-1] / 128 + 32) * 2.0 ** -24 + want_lse.abs() * 2.0 ** -24
    assert bool(((lse.double() - want_lse).abs()[ok] <= tol[ok]).all())
    assert d.last_error() == 0
    return idx, val, lse


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,vocab,k", [(3, 1, 1), (5, 2, 2), (4, 7, 3), (2, 15, 15), (7, 33, 32), (3, 1000, 1), (2, 1024, 1024), (5, 4099, 64),
                                       (3, 32000, 100), (300, 20001, 17), (2, 50001, 1000), (1, 131072, 32), (1, 131072, 1024),
                                       (1, 1 << 20, 50), (700, 2049, 8)])
def test_top_sizes(binding, n, vocab, k, kind):
    check_top(binding, logits_like(n, vocab, kind, n + vocab + k), k, temperature=1.7 if k % 2 else 1.0)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "few values", "spikes at the end", "one block of large ones"])
@pytest.mark.parametrize("vocab,k", [(9000, 40), (70001, 700)])
def test_top_of_rows_in_order(binding, order, vocab, k, kind):
    base = torch.arange(vocab, device="cuda", dtype=torch.float32).view(1, -1).repeat(3, 1) / vocab * 10
    x = {"rising": base, "falling": -base, "equal": torch.zeros_like(base), "few values": (base * 0.3).round().roll(77, 1),
         "spikes at the end": torch.where(torch.arange(vocab, device="cuda") >= vocab - k - 3, base + 50, torch.randn((3, vocab), device="cuda", generator=gen(3))),
         "one block of large ones": torch.where((torch.arange(vocab, device="cuda") // 3000) == 1, base + 30, -base)}[order]
    check_top(binding, x.to(TYPES[kind]), k)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_top_of_special_values(binding, kind):
    t = TYPES[kind]
    x = logits_like(12, 5000, kind, 5)
    x[1, 100:] = -math.inf                          # fewer finite logits than are asked for
    x[2] = -math.inf                                # none at all
    x[3, 4000:] = torch.finfo(t).min                # masked by the lowest value
    x[4] = torch.finfo(t).min
    x[5, 17] = math.nan
    x[6, 4999] = math.inf
    x[7, [3, 4990]] = math.inf
    x[7, 5] = -math.nan
    x[8] = math.nan
    x[9] = 0.0
    x[9, ::2] = -0.0
    x[10] = torch.finfo(t).max
    x[11, :4000] = -math.inf
    d = binding.Distiller(5000)
    for k in (1, 64, 200, 1000):
        idx, val, _ = d.top(x, k)
        check_top(binding, x, k, d=d)


def test_top_of_rows_elsewhere(binding):
    """Rows with gaps, of two distances, off the 16-byte grid, repeated, none."""
    d = binding.Distiller(1001)
    wide = logits_like(24, 1203, "bf16", 9)
    check_top(binding, wide[:, 101:1102], 33, d=d)
    check_top(binding, wide.view(4, 6, 1203)[1:, ::2, 3:1004], 33, d=d)
    check_top(binding, wide.view(4, 6, 1203)[:, :, 8:1009].transpose(0, 1), 5, d=d)
    check_top(binding, wide[:1, :1001].expand(7, 1001), 5, d=d)
    idx, val, lse = d.top(wide[:0, :1001], 5)
    assert idx.shape == (0, 5) and val.shape == (0, 5) and lse.shape == (0,)
    flat = logits_like(1, 1001, "f32", 1)[0]
    check_top(binding, flat, 4, d=d)                # one row without a dimension for it


# ------------------------------------------------------------------------------------------- loss and gradient

def pairs_of(teacher, k, temperature=1.0, dtype=None):
    top = torch.topk(teacher.float(), k, dim=-1)
    val = teacher.gather(-1, top.indices)
    return top.indices.int(), val if dtype is None else val.to(dtype), torch.logsumexp(teacher.double() / temperature, -1).float()


def plain_loss(x, idx, val, lse, temperature, weight=None, ratios=None):
    """Row by row from the definition, differentiable; x in 64 bits.  Entries that are there, each token's first.  ``ratios``: a
    tensor that receives r / p_rest of every row."""
    vocab, losses = x.shape[-1], []
    for r in range(x.shape[0]):
        zero = (x[r] * 0).nan_to_num(0.0).sum() * 0.0
        if weight is not None and float(weight[r]) == 0.0:
            losses.append(zero)
            continue
        seen, keep = set(), []
        for i, v in enumerate(idx[r].tolist()):
            if 0 <= v < vocab and v not in seen:
                seen.add(v)
                keep.append(i)
        t = val[r].double()[keep] / temperature
        if not keep or bool((x[r] == -math.inf).all()) or (lse is None and bool((t == -math.inf).all())) or \
                (lse is not None and float(lse[r]) == -math.inf):
            losses.append(zero)
            continue
        at = idx[r].long()[keep]
        logq = torch.log_softmax(t, 0) if lse is None else t - lse[r].double()
        q = logq.exp()
        logp = torch.log_softmax(x[r] / temperature, 0)
        some = q != 0
        loss = (q[some] * (logq[some] - logp[at][some])).sum()
        if lse is not None:
            rest = torch.ones(vocab, dtype=torch.bool, device=x.device)
            rest[at] = False
            left = 1.0 - float(q.sum())
            if left > 0 and bool(rest.any()):
                log_rest = torch.logsumexp(logp[rest], 0)
                if float(log_rest.detach()) > -126 * math.log(2.0):
                    loss = loss + left * (math.log(left) - log_rest)
                    if ratios is not None:
                        ratios[r] = left / math.exp(float(log_rest.detach()))
        losses.append(loss)
    return torch.stack(losses)


def check_loss(binding, x, idx, val, lse=None, temperature=1.0, weight=None, out=None, d=None, errors=0):
    d = d or binding.Distiller(x.shape[-1])
    flat = lambda t, w: t.reshape(-1, w) if w else t.reshape(-1)
    kept = x.clone()
    wide = flat(x, x.shape[-1]).double().requires_grad_()
    w = torch.ones(wide.shape[0], dtype=torch.float64, device="cuda") if weight is None else flat(weight, 0).double()
    ratios = torch.zeros_like(w)
    want = plain_loss(wide, flat(idx, idx.shape[-1]), flat(val, val.shape[-1]), None if lse is None else flat(lse, 0), temperature, weight if weight is None else flat(weight, 0),
                      ratios)
    (want * w).sum().backward()
    want_grad, want = wide.grad.nan_to_num(0.0), want.detach()
    vocab, t = x.shape[-1], x.dtype
    with torch.no_grad():
        p = torch.softmax(wide / temperature, 1).nan_to_num(0.0)
        depth = -torch.log2(p.clamp(min=2.0 ** -126))
        P = 2.0 ** -21 + (vocab / 128 + 32) * 2.0 ** -24 + 3 * 2.0 ** -24 * (depth + 8.0)
        scale = (w / temperature).abs().view(-1, 1)
        # W p and q each, with their own errors: |W p - q| is smaller than either; both are bounded by p W and the gradient itself
        q = (want_grad.abs() / scale.clamp(min=1e-300) + 1.01 * p * 1.01)
        # an entry that is not listed is p (W - r / p_rest) with p / p_rest as inexact as p: both terms bring their error, W P p and
        # (r / p_rest) P p, even where they cancel (r itself is a difference of 64-bit numbers)
        more = 1.0 + ratios.view(-1, 1)
        tol = scale * (p * P * more + q * 2.0 ** -20) + want_grad.abs() * torch.finfo(t).eps / 2 + SUBNORMAL[t]
    loss_tol = (2.0 ** -21 + (vocab / 128 + 32) * 2.0 ** -24 + 2.0 ** -20 * (want.abs() + 8.0) * 2)
    given = dict(lse=lse, temperature=temperature, weight=weight)
    loss, stats = d.loss(x, idx, val, **given)
    two = d.grad(x, idx, val, stats, **given)
    loss_too, grad = d.loss_grad(x, idx, val, out=out, **given)
    assert loss.shape == x.shape[:-1] and grad.shape == x.shape and grad.dtype == t
    assert bool(((flat(loss, 0).double() - want).abs() <= loss_tol).all()), (loss, want)
    assert bool(((flat(loss_too, 0).double() - want).abs() <= loss_tol).all())
    for g in (grad, two):
        err = (flat(g, vocab).double() - want_grad).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
    assert torch.equal(x.contiguous().view(torch.uint8), kept.contiguous().view(torch.uint8))
    assert d.last_error() == errors
    return loss, grad


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("n,vocab,k,temperature", [(3, 1, 1, 1.0), (4, 2, 1, 1.0), (5, 9, 4, 0.5), (3, 31, 31, 2.0), (6, 1000, 20, 1.0), (3, 4097, 300, 3.0),
                                                   (4, 32000, 64, 1.0), (2, 50001, 1024, 1.0), (2, 131072, 128, 2.0), (1, 300001, 33, 1.0)])
def test_loss_sizes(binding, n, vocab, k, temperature, tail, kind):
    teacher = logits_like(n, vocab, kind, vocab + k)
    student = (teacher.float() + logits_like(n, vocab, "f32", k, 0.7)).to(TYPES[kind])
    idx, val, lse = pairs_of(teacher, k, temperature)
    weight = torch.rand(n, device="cuda", generator=gen(k)) + 0.5
    check_loss(binding, student, idx, val, lse if tail else None, temperature, weight)


def test_largest_vocabulary(binding):
    teacher = logits_like(1, 1 << 20, "f32", 3)
    idx, val, lse = pairs_of(teacher, 50)
    check_loss(binding, teacher + 0.3, idx, val, lse)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("kind,pairs_kind", [("bf16", "f32"), ("f32", "bf16"), ("f16", "f16")])
def test_many_rows_of_lists_of_different_length(binding, kind, pairs_kind, tail):
    n, vocab, k = 613, 2003, 24
    teacher = logits_like(n, vocab, pairs_kind, 1)
    student = logits_like(n, vocab, kind, 2)
    idx, val, lse = pairs_of(teacher, k)
    length = torch.randint(0, k + 1, (n, 1), device="cuda", generator=gen(4))
    idx = torch.where(torch.arange(k, device="cuda") < length, idx, torch.tensor(-1, device="cuda", dtype=torch.int32))
    idx[5, 0] = -1                                  # empty places may stand anywhere
    val[7, length[7, 0]:] = math.nan                # what stands beside them is not looked at
    weight = torch.rand(n, device="cuda", generator=gen(3))
    weight[::7] = 0.0
    check_loss(binding, student, idx.long() if tail else idx, val, lse if tail else None, 1.0, weight)


def test_same_distribution_has_no_loss(binding):
    """The whole row listed, student = teacher: the loss is zero and so is the gradient, to the probabilities' precision."""
    x = logits_like(4, 500, "f32", 11)
    idx, val, lse = pairs_of(x, 500)
    for normaliser in (None, lse):
        loss, grad = check_loss(binding, x, idx, val, normaliser)
        assert float(loss.abs().max()) < 2e-6 and float(grad.abs().max()) < 1e-6


def test_label_as_a_list_of_one(binding):
    """A list of one renormalises to probability 1: cross entropy."""
    x = logits_like(64, 999, "f32", 3)
    label = torch.randint(0, 999, (64, 1), device="cuda", generator=gen(2))
    loss, _ = check_loss(binding, x, label, torch.zeros((64, 1), device="cuda"))
    assert torch.allclose(loss, torch.nn.functional.cross_entropy(x, label.view(-1), reduction="none"), atol=1e-5)


def test_gradient_is_the_slope(binding):
    """Differences of the definition in 64 bits along single logits; step 1e-5, whose third-order term is below 1e-9."""
    x = logits_like(2, 300, "f32", 8)
    teacher = logits_like(2, 300, "f32", 9)
    idx, val, lse = pairs_of(teacher, 10, 1.5)
    d = binding.Distiller(300)
    for normaliser in (None, lse):
        _, grad = d.loss_grad(x, idx, val, lse=normaliser, temperature=1.5)
        for j in [0, 17, 299] + idx[0, :4].tolist():
            h = 1e-5
            up, down = x.double().clone(), x.double().clone()
            up[:, j] += h
            down[:, j] -= h
            slope = (plain_loss(up, idx, val, normaliser, 1.5) - plain_loss(down, idx, val, normaliser, 1.5)) / (2 * h)
            assert bool(((grad[:, j].double() - slope).abs() <= 1e-9 + 4e-6 * (slope.abs() + 0.01)).all())


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tail", [False, True])
def test_masked_and_special_rows(binding, tail, kind):
    t, vocab, k = TYPES[kind], 3001, 16
    teacher = logits_like(9, vocab, kind, 1)
    x = logits_like(9, vocab, kind, 2)
    idx, val, lse = pairs_of(teacher, k)
    x[0, 2000:] = -math.inf
    x[0, idx[0].long()] = 1.0                       # every listed token keeps its probability
    x[1, 2000:] = torch.finfo(t).min
    x[2] = torch.finfo(t).min                       # a row of lowest values is an even distribution
    x[3] = -math.inf                                # no distribution
    idx[4] = -1                                     # no list
    val[5, 3:] = -math.inf                          # listed with probability 0
    if not tail:
        val[6] = -math.inf
    else:
        lse[6] = -math.inf
    x[7, :] = -math.inf
    x[7, int(idx[7, 0])] = 2.0                      # all of the student on one listed token; the others are impossible
    idx[7, 1:] = -1
    weight = torch.ones(9, device="cuda")
    weight[8] = 0.0
    x[8] = math.nan                                 # not read
    loss, grad = check_loss(binding, x, idx, val, lse if tail else None, 1.0, weight)
    for r in (3, 4, 6, 8):
        assert float(loss[r]) == 0.0 and not bool(grad[r].any())


@pytest.mark.parametrize("tail", [False, True])
def test_what_cannot_be_computed_shows(binding, tail):
    vocab, k = 2000, 8
    x = logits_like(7, vocab, "f32", 2)
    idx, val, lse = pairs_of(logits_like(7, vocab, "f32", 1), k)
    x[0, 5] = math.nan
    x[1, 5] = math.inf
    x[2, int(idx[2, 1])] = math.nan
    val[3, 2] = math.nan
    val[4, 2] = math.inf
    x[5, int(idx[5, 1])] = -math.inf                # listed, but impossible for the student
    d = binding.Distiller(vocab)
    lse = lse if tail else None
    loss, grad = d.loss_grad(x, idx, val, lse=lse)
    alone, stats = d.loss(x, idx, val, lse=lse)
    two = d.grad(x, idx, val, stats, lse=lse)
    assert torch.equal(loss.isnan(), alone.isnan()) and torch.equal(grad.isnan(), two.isnan())
    assert bool(loss[:5].isnan().all()) and bool(grad[:5].isnan().all())
    assert float(loss[5]) == math.inf and bool(grad[5].isfinite().all())
    assert bool(loss[6].isfinite()) and bool(grad[6].isfinite().all())


def test_tokens_twice_and_outside(binding):
    vocab, k = 5000, 40
    x = logits_like(5, vocab, "bf16", 2)
    idx, val, lse = pairs_of(logits_like(5, vocab, "bf16", 1), k)
    idx[0, 7] = idx[0, 3]
    idx[1, 20:] = idx[1, 5]
    idx[2] = idx[2, 0]
    d = binding.Distiller(vocab)
    for normaliser in (None, lse):
        check_loss(binding, x, idx, val, normaliser, d=d)
    idx[3, 4] = vocab
    idx[4, 0] = 2 ** 31 - 1
    check_loss(binding, x, idx, val, lse, d=d, errors=binding.ERR_INVALID)
    far = idx.long()
    far[4, 0] = 2 ** 40 + 3
    far[4, 1] = -2 ** 40
    check_loss(binding, x, far, val, None, d=d, errors=binding.ERR_INVALID)
    assert d.last_error() == 0


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_places_of_the_gradient(binding, kind):
    """In place, between other data, off the grid, in rows of two distances; nothing else is written."""
    vocab, k = 1001, 12
    teacher = logits_like(12, vocab, kind, 1)
    wide = logits_like(12, 1203, kind, 2)
    idx, val, lse = pairs_of(teacher, k)
    d = binding.Distiller(vocab)
    x = wide[:, 100:1101]
    loss, want = check_loss(binding, x, idx, val, lse, d=d)
    for shift in (0, 1, 2, 3, 101):
        room = torch.full((12, 1203), 7.0, device="cuda", dtype=TYPES[kind])
        d.loss_grad(x, idx, val, lse=lse, out=room[:, shift:shift + vocab])
        assert torch.equal(room[:, shift:shift + vocab], want)
        assert bool((room[:, :shift] == 7.0).all()) and bool((room[:, shift + vocab:] == 7.0).all())
    x3, room = wide.view(3, 4, 1203)[:, ::2, 100:1101], torch.full((3, 4, 1203), 7.0, device="cuda", dtype=TYPES[kind])
    take = torch.arange(12, device="cuda").view(3, 4)[:, ::2]
    d.loss_grad(x3, idx[take], val[take], lse=lse[take].contiguous(), out=room[:, 1::2, 5:5 + vocab])
    assert torch.equal(room[:, 1::2, 5:5 + vocab].reshape(-1, vocab), want[take.reshape(-1)])
    assert bool((room[:, ::2] == 7.0).all())
    before = wide.clone()
    out = d.loss_grad(x, idx, val, lse=lse, out=x)[1]
    assert torch.equal(wide[:, 100:1101], want) and torch.equal(wide[:, :100], before[:, :100]) and torch.equal(wide[:, 1101:], before[:, 1101:])
    assert out is x
    again = before.clone()
    loss, stats = d.loss(again[:, 100:1101], idx, val, lse=lse)
    d.grad(again[:, 100:1101], idx, val, stats, lse=lse, out=again[:, 100:1101])
    assert torch.equal(again, wide)


def test_lists_elsewhere(binding):
    vocab, k = 700, 9
    x = logits_like(6, vocab, "f32", 2).view(2, 3, vocab)
    idx, val, lse = pairs_of(logits_like(6, vocab, "f32", 1), k)
    room_idx, room_val = torch.full((2, 5, 30), 10 ** 6, device="cuda"), torch.full((2, 5, 30), math.nan, device="cuda")
    room_idx[:, 1:4, 4:13], room_val[:, 1:4, 4:13] = idx.view(2, 3, k).long(), val.view(2, 3, k)
    check_loss(binding, x, room_idx[:, 1:4, 4:13], room_val[:, 1:4, 4:13], lse.view(2, 3))


def test_rows_past_32_bits(binding):
    """More than 2^32 logits: the last rows are as if they stood alone."""
    vocab, n = 65536, 65600
    if torch.cuda.mem_get_info()[0] < 30e9:
        pytest.skip("needs 9 GB of free device memory, with room")
    x = torch.empty((n, vocab), device="cuda", dtype=torch.bfloat16)
    tail = logits_like(64, vocab, "bf16", 5)
    x[:-64] = tail[0]
    x[-64:] = tail
    d = binding.Distiller(vocab)
    idx, val, lse = d.top(x, 20)
    few = d.top(tail, 20)
    # how many blocks share a row depends on the number of rows, and with it the order of the sums: twice a sum's error
    tol = 2 * (2.0 ** -21 + (vocab / 128 + 32) * 2.0 ** -24 + 16 * 2.0 ** -24)
    assert torch.equal(idx[-64:], few[0]) and torch.equal(val[-64:], few[1]) and bool(((lse[-64:] - few[2]).abs() <= tol).all())
    want = d.loss_grad(tail, few[0], few[1], lse[-64:].contiguous())
    loss, grad = d.loss_grad(x, idx, val, lse, out=x)
    assert bool(((loss[-64:] - want[0]).abs() <= tol * 8).all())
    # the gradients' difference: that error of p, and a rounding to bf16 that may fall on either side
    assert torch.allclose(grad[-64:].float(), want[1].float(), rtol=2.0 ** -7, atol=tol)
    assert torch.equal(grad[1], grad[len(x) - 65]) and torch.equal(idx[0], few[0][0])


def test_same_call_same_bits_other_stream_and_graph(binding):
    vocab, k, n = 30011, 50, 37
    x = logits_like(n, vocab, "bf16", 2)
    d = binding.Distiller(vocab)
    teacher = logits_like(n, vocab, "bf16", 1)
    idx, val, lse = d.top(teacher, k)
    loss, grad = d.loss_grad(x, idx, val, lse)
    for _ in range(3):
        a, b = d.loss_grad(x, idx, val, lse)
        assert torch.equal(a, loss) and torch.equal(b, grad)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = d.loss_grad(x, idx, val, lse, stream=side)
    t = d.top(teacher, k, stream=side)
    side.synchronize()
    assert torch.equal(a, loss) and torch.equal(b, grad) and torch.equal(t[0], idx) and torch.equal(t[2], lse)
    # teacher and student in one captured graph, replayed on other inputs
    graph = torch.cuda.CUDAGraph()
    held = [teacher.clone(), x.clone()]
    with torch.cuda.graph(graph):
        i, v, z = d.top(held[0], k)
        a, s = d.loss(held[1], i, v, z)
        b = d.grad(held[1], i, v, s, z)
    for seed in (5, 6):
        held[0].copy_(logits_like(n, vocab, "bf16", seed))
        held[1].copy_(logits_like(n, vocab, "bf16", seed + 100))
        graph.replay()
        want_idx, want_val, want_lse = d.top(held[0].clone(), k)
        want, want_grad = d.loss_grad(held[1].clone(), want_idx, want_val, want_lse)
        assert torch.equal(i, want_idx) and torch.equal(v, want_val) and torch.equal(z, want_lse)
        assert torch.equal(a, want) and torch.equal(b, want_grad)


def test_refusals(binding):
    d = binding.Distiller(100)
    x = torch.zeros((4, 100), device="cuda")
    idx, val = torch.zeros((4, 3), device="cuda", dtype=torch.int32), torch.zeros((4, 3), device="cuda")
    for bad in (dict(k=0), dict(k=101), dict(k=5, temperature=0.0), dict(k=5, temperature=math.nan), dict(k=5, temperature=-1.0)):
        with pytest.raises(binding.AdacompError):
            d.top(x, **bad)
    with pytest.raises(ValueError):
        d.top(x[:, :99], 5)
    with pytest.raises(TypeError):
        d.top(x.double(), 5)
    with pytest.raises(TypeError):
        d.top(x.cpu(), 5)
    with pytest.raises(TypeError):
        d.top(torch.zeros((4, 200), device="cuda")[:, ::2], 5)
    with pytest.raises(ValueError):
        d.top(x, 5, idx_out=torch.zeros((4, 4), device="cuda", dtype=torch.int32))
    with pytest.raises(TypeError):
        d.top(x, 5, idx_out=torch.zeros((4, 5), device="cuda", dtype=torch.int64))
    for call in (lambda **k: d.loss(x, **k), lambda **k: d.loss_grad(x, **k)):
        with pytest.raises(ValueError):
            call(idx=idx[:3], val=val[:3])
        with pytest.raises(ValueError):
            call(idx=idx, val=val[:, :2])
        with pytest.raises(TypeError):
            call(idx=idx.float(), val=val)
        with pytest.raises(TypeError):
            call(idx=idx, val=val.double())
        with pytest.raises(binding.AdacompError):
            call(idx=idx[:, :0], val=val[:, :0])
        with pytest.raises(binding.AdacompError):
            call(idx=idx, val=val, temperature=math.inf)
        with pytest.raises(ValueError):
            call(idx=idx, val=val, weight=torch.ones(5, device="cuda"))
        with pytest.raises(TypeError):
            call(idx=idx, val=val, lse=torch.ones(4, device="cuda", dtype=torch.float64))
    many = torch.zeros((4, 1025), device="cuda", dtype=torch.int32)
    with pytest.raises(binding.AdacompError):
        d.loss(x, many, many.float())
    room = torch.zeros((4, 150), device="cuda")
    with pytest.raises(ValueError):
        d.loss_grad(room[:, :100], idx, val, out=room[:, 50:])
    with pytest.raises(ValueError):
        d.loss_grad(x, idx, val, out=x.half())
    with pytest.raises(binding.AdacompError):       # rows of the gradient that overlap each other
        d.loss_grad(x, idx, val, out=torch.zeros(400, device="cuda").as_strided((4, 100), (50, 1)))
    with pytest.raises(ValueError):
        d.grad(x, idx, val, torch.zeros((4, 7), device="cuda"))
    for vocab in (0, (1 << 20) + 1):
        with pytest.raises(binding.AdacompError):
            binding.Distiller(vocab)
    assert d.last_error() == 0
    with pytest.raises(ValueError):                 # more rows than a call takes
        binding.Distiller(1).top(torch.zeros((1, 1), device="cuda").expand(1 << 31, 1), 1)


def test_two_streams_at_once(binding):
    """Two handles, each on a stream of its own, neither waiting for the other."""
    n, vocab, k = 500, 20011, 30
    x, y = logits_like(n, vocab, "bf16", 1), logits_like(n, vocab, "bf16", 2)
    handles, streams = [binding.Distiller(vocab) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    alone = handles[0].top(x, k)
    want = handles[0].loss_grad(y, *alone)
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for h, s, g in zip(handles, streams, got):
            pairs = h.top(x, k, stream=s)
            g.append((pairs, h.loss_grad(y, *pairs, stream=s)))
    torch.cuda.synchronize()
    for g in got:
        for pairs, result in g:
            assert all(torch.equal(a, b) for a, b in zip(pairs, alone)) and all(torch.equal(a, b) for a, b in zip(result, want))


@pytest.mark.parametrize("vocab,kind", [(500, "bf16"), (1501, "f32"), (7000, "f16"), (15001, "bf16"), (20000, "f32"), (30000, "bf16"), (52001, "f16"),
                                        (70000, "bf16"), (40003, "f32")])
@pytest.mark.parametrize("tail", [False, True])
def test_many_rows_of_every_length(binding, vocab, kind, tail):
    """Rows that blocks of every size take, whole or in part, and the same in place."""
    n, k = 601, 30
    teacher = logits_like(n, vocab, kind, 1)
    student = (teacher.float() + logits_like(n, vocab, "f32", 2, 0.5)).to(TYPES[kind])
    idx, val, lse = pairs_of(teacher, k)
    idx[3, 5] = idx[3, 0]
    idx[4, ::2] = -1
    weight = torch.rand(n, device="cuda", generator=gen(3)) + 0.1
    weight[::50] = 0.0
    lse = lse if tail else None
    _, grad = check_loss(binding, student, idx, val, lse, 1.0, weight)
    d = binding.Distiller(vocab)
    again = student.clone()
    d.loss_grad(again, idx, val, lse, weight=weight, out=again)
    assert torch.equal(again, grad)
    _, stats = d.loss(student, idx, val, lse, weight=weight)
    two = d.grad(student, idx, val, stats, lse, weight=weight)
    again = student.clone()
    assert torch.equal(d.grad(again, idx, val, stats, lse, weight=weight, out=again), two)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,k", [(1300, 4000, 20), (1201, 901, 64), (1184, 64, 64), (1500, 7777, 1), (1300, 4000, 65)])
def test_top_of_many_short_rows(binding, n, vocab, k, kind):
    x = logits_like(n, vocab, kind, vocab)
    check_top(binding, x, k)
    check_top(binding, (x * 0.4).round(), k, temperature=2.0)         # ties
    x[::3, vocab // 3:] = -math.inf
    x[5] = 1.0
    check_top(binding, x, k)
