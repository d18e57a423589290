"""Routing to experts and its gradient, through the binding, against plain implementations in 64 bits.

Tolerances.  A score has an exponential (2 units in the last place, 2^-22), its argument's rounding (2^-24 |argument|), a sum of positive
terms (at most 37 roundings: 32 in a lane, 5 across lanes; 2^-19 altogether) and a division; a weight another such sum, a
division and a product: 2^-17 relative leaves a factor of two.  A gradient is a difference of two products of weights and up to 32 terms
d s, so its error is 2^-17 times the sum of the terms' magnitudes, and one rounding to its type.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
REL = 2.0 ** -17


@pytest.fixture(scope="module")
def binding():
    from paper_1702_04683_b200 import binding as b
    return b


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def plain_choice(x, bias, cfg):
    """x [N, E] in 64 bits on the CPU -> experts [N, k], -1 where none is left."""
    N, E = x.shape
    # (on the GPU: there equal logits have equal scores, the CPU's vectors and their remainders differ in the last bit)
    scores = (torch.softmax(x.cuda(), 1) if cfg["score"] == "softmax" else torch.sigmoid(x.cuda())).cpu()
    value = scores + (0.0 if bias is None else bias.double().cpu())
    value = torch.where(x == -math.inf, -math.inf, value)
    bad = value.isnan().any(1) | x.isnan().any(1)
    if cfg["score"] == "softmax":
        bad |= (x == math.inf).any(1)
    out = torch.full((N, cfg["top_k"]), -1)
    size = E // cfg["groups"]
    for r in range(N):
        if bad[r]:
            continue
        v = value[r].tolist()
        rated = []
        for g in range(cfg["groups"]):
            best = sorted((u for u in v[g * size:(g + 1) * size] if u != -math.inf), reverse=True)[:cfg["group_terms"]]
            rated.append((-sum(best) if best else math.inf, g))
        kept = {g for _, g in sorted(rated)[:cfg["top_groups"]]}
        order = sorted((-u, e) for e, u in enumerate(v) if e // size in kept and u != -math.inf)[:cfg["top_k"]]
        for i, (_, e) in enumerate(order):
            out[r, i] = e
    return out, bad


def plain_weights(x, experts, cfg):
    scores = torch.softmax(x, 1) if cfg["score"] == "softmax" else torch.sigmoid(x)
    there = experts >= 0
    s = torch.where(there, scores.gather(1, experts.clamp(min=0)), 0.0)
    if cfg["renormalize"]:
        # the same quotient, from logarithms: scores may be too small for numbers
        l = x if cfg["score"] == "softmax" else torch.nn.functional.logsigmoid(x)
        l = torch.where(there, l.gather(1, experts.clamp(min=0)), -math.inf)
        some = there.any(1, keepdim=True)
        s = torch.where(some & there, torch.softmax(torch.where(some, l, 0.0), 1), 0.0)
    return cfg["scale"] * s


def check(binding, x, bias=None, live=None, seed=0, **kw):
    cfg = dict(experts=x.shape[-1], top_k=2, score="softmax", groups=1, top_groups=1, group_terms=1, renormalize=True, scale=1.0) | kw
    h = binding.Router(**cfg)
    kept = x.clone()
    experts, weights, counts = h.route(x, bias=bias, live=live)
    E, k = cfg["experts"], cfg["top_k"]
    flat = x.reshape(-1, E)
    wide = flat.double().cpu()
    want, bad = plain_choice(wide, bias, cfg)
    alive = torch.ones(len(wide), dtype=torch.bool) if live is None else live.reshape(-1).cpu()
    want[~alive] = -1
    got = experts.reshape(-1, k).cpu().long()
    assert experts.shape == (*x.shape[:-1], k) and weights.shape == experts.shape
    assert torch.equal(got, want), (got[(got != want).any(1)][:3], want[(got != want).any(1)][:3])
    assert torch.equal(counts.cpu().long(), torch.bincount(want[want >= 0], minlength=E))
    ok = alive & ~bad
    w = weights.reshape(-1, k).cpu().double()
    wide_ok = wide[ok].requires_grad_()
    want_w = plain_weights(wide_ok, want[ok], cfg)
    assert bool(((w[ok] - want_w.detach()).abs() <= REL * want_w.detach().abs() + 1e-37).all())
    assert bool(w[bad & alive].isnan().all()) and not bool(w[~alive].any())
    # the gradient
    dw = torch.randn((*x.shape[:-1], k), device="cuda", generator=gen(seed + 77))
    grad = h.grad(x, experts, dw)
    d = dw.reshape(-1, k).cpu().double()
    (want_w * d[ok]).sum().backward()
    g = grad.reshape(-1, E).cpu().double()
    assert grad.dtype == x.dtype and grad.shape == x.shape
    with torch.no_grad():
        size = torch.zeros_like(wide)
        terms = (want_w.abs() * (d[ok].abs() + (d[ok].abs() * want_w.abs() / abs(cfg["scale"] or 1.0)).sum(1, keepdim=True)))
        size[ok] = torch.zeros_like(size[ok]).scatter_add_(1, want[ok].clamp(min=0), torch.where(want[ok] >= 0, terms, 0.0))
        if cfg["score"] == "softmax" and not cfg["renormalize"]:
            size[ok] += torch.softmax(wide[ok], 1).nan_to_num(0.0) * (d[ok] * want_w).abs().sum(1, keepdim=True)
        want_g = torch.zeros_like(wide)
        want_g[ok] = wide_ok.grad.nan_to_num(0.0)
        tiny = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}[x.dtype]
        tol = REL * size + want_g.abs() * torch.finfo(x.dtype).eps / 2 + tiny
        assert bool(((g - want_g).abs() <= tol).all()), float(((g - want_g).abs() / tol).max())
    assert torch.equal(x.contiguous().view(torch.uint8), kept.contiguous().view(torch.uint8))
    assert h.last_error() == 0
    return experts, weights, counts, grad


def rows(n, experts, kind, seed, spread=1.5):
    return (torch.randn((n, experts), device="cuda", generator=gen(seed)) * spread).to(TYPES[kind])


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("score,renormalize", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("n,experts,k", [(1, 1, 1), (3, 2, 1), (9, 5, 5), (33, 8, 2), (130, 60, 4), (70, 64, 6), (200, 128, 8), (50, 257, 9), (40, 384, 31),
                                         (17, 1000, 32), (9, 1024, 16)])
def test_sizes(binding, n, experts, k, score, renormalize, kind):
    check(binding, rows(n, experts, kind, n + experts), top_k=k, score=score, renormalize=renormalize, scale=2.5 if k % 2 else 1.0)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups,top_groups,terms,k", [(256, 8, 4, 2, 8), (256, 8, 3, 1, 8), (64, 32, 5, 2, 6), (60, 12, 7, 2, 5), (160, 8, 3, 1, 6),
                                                               (96, 3, 1, 2, 32), (30, 30, 10, 2, 10), (1024, 32, 2, 2, 8), (257, 1, 1, 2, 3),
                                                               (18, 9, 9, 1, 3)])
def test_groups_and_bias(binding, experts, groups, top_groups, terms, k, score, kind):
    bias = torch.randn(experts, device="cuda", generator=gen(experts)) * (0.1 if score == "sigmoid" else 0.01)
    check(binding, rows(150, experts, kind, groups), bias, top_k=k, score=score, groups=groups, top_groups=top_groups, group_terms=terms)
    check(binding, rows(40, experts, kind, groups + 1), torch.zeros_like(bias), top_k=k, score=score, groups=groups, top_groups=top_groups,
          group_terms=terms, renormalize=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_ties_go_to_the_lowest(binding, score):
    x = (rows(200, 96, "f32", 4) * 2).round() / 2       # few values
    check(binding, x, top_k=12, score=score)
    check(binding, torch.zeros_like(x), top_k=12, score=score, groups=6, top_groups=2, group_terms=2)
    check(binding, x, torch.full((96,), 0.25, device="cuda"), top_k=12, score=score, groups=12, top_groups=5, group_terms=2)
    check(binding, x + 100.0, top_k=5, score=score)     # sigmoids that are all 1 in 64 bits


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 8])
def test_values_closer_than_fp32_can_tell(binding, score, groups):
    """Biases that make every expert's value the same up to 1e-9: fp32 scores cannot order them, the choice is 64 bits' all the same."""
    x = rows(64, 128, "f32", 3)
    scores = torch.softmax(x.double(), 1) if score == "softmax" else torch.sigmoid(x.double())
    for r in range(4):
        bias = (0.75 - scores[r]).float()               # row r's values differ by the rounding of the bias, some 3e-8
        check(binding, x, bias, top_k=8, score=score, groups=groups, top_groups=max(1, groups // 2), group_terms=2)


def test_a_rows_order_down_to_the_last_bit(binding):
    base = torch.linspace(-1, 1, 64, device="cuda").repeat(20, 1)
    x = torch.nextafter(base, base + torch.randint(0, 2, base.shape, device="cuda", generator=gen(2)).float() - 0.5)
    x[:, 1::2] = torch.nextafter(x[:, ::2], torch.tensor(9.0, device="cuda"))      # neighbours one unit apart
    for score in ("softmax", "sigmoid"):
        check(binding, x, top_k=20, score=score)


@pytest.mark.parametrize("score,renormalize", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_masked_and_special_rows(binding, score, renormalize):
    x = rows(16, 40, "f32", 6)
    x[0, 5:] = -math.inf                                # fewer experts than places
    x[1] = -math.inf                                    # none
    x[2, 1:] = -math.inf
    x[3] = torch.finfo(torch.float32).min
    x[4, 20:] = torch.finfo(torch.float32).min
    x[5, 7] = math.nan
    x[6, 7] = math.inf
    x[7] = 90.0                                         # sigmoids of 1, softmax even
    x[8] = -200.0                                       # sigmoids too small for fp32
    x[8, 3] = -math.inf
    x[9, :39] = -300.0                                  # softmax scores too small for fp32, but one
    live = torch.ones(16, dtype=torch.bool, device="cuda")
    live[10:12] = False
    x[10] = math.nan                                    # not looked at
    want = dict(top_k=8, score=score, renormalize=renormalize)
    if score == "sigmoid":
        x = torch.cat([x[:8], x[9:]])                   # of 64-bit sigmoids of -200 fp32 makes zeros: see below
        live = torch.cat([live[:8], live[9:]])
    check(binding, x, live=live, **want)
    check(binding, x.view(-1, 1, 40), live=live.view(-1, 1), groups=8, top_groups=3, group_terms=2, **want)
    bias = torch.randn(40, device="cuda", generator=gen(1)) * 0.1
    bias[::3] = -math.inf                               # an expert that is taken out
    check(binding, x, bias, live, groups=4, top_groups=2, group_terms=2, **want)


def test_scores_too_small_for_fp32(binding):
    """As weights they are zeros; their quotients are there all the same."""
    x = torch.full((3, 16), -200.0, device="cuda")
    x[1] -= torch.arange(16, device="cuda") * 0.25
    for renormalize in (True, False):
        experts, weights, _, grad = check(binding, x, top_k=4, score="sigmoid", renormalize=renormalize)
        assert torch.equal(experts, torch.arange(4, device="cuda", dtype=torch.int32).expand(3, 4))
        assert bool(weights.all()) == renormalize and bool(grad.any()) == renormalize


def test_gradient_is_the_slope(binding):
    """Differences of the weights in 64 bits; step 1e-5, whose third-order term is below 1e-9."""
    x = rows(3, 12, "f32", 9)
    dw = torch.randn((3, 4), device="cuda", generator=gen(5))
    for score in ("softmax", "sigmoid"):
        for renormalize in (True, False):
            cfg = dict(experts=12, top_k=4, score=score, renormalize=renormalize, scale=1.5)
            h = binding.Router(**cfg)
            experts, _, _ = h.route(x)
            grad = h.grad(x, experts, dw).cpu().double()
            at, d = experts.cpu().long(), dw.cpu().double()
            for j in range(12):
                up, down = x.double().cpu(), x.double().cpu()
                up[:, j] += 1e-5
                down[:, j] -= 1e-5
                slope = ((plain_weights(up, at, cfg) - plain_weights(down, at, cfg)) * d).sum(1) / 2e-5
                assert bool(((grad[:, j] - slope).abs() <= 1e-8 + 3e-5 * d.abs().sum(1)).all())


def test_places(binding):
    """Rows with gaps, of two distances, off the grid; the gradient in place and between other data."""
    wide = rows(24, 201, "bf16", 3)
    for x in (wide[:, 3:67], wide.view(4, 6, 201)[1:, ::2, 8:72], wide.view(4, 6, 201)[:, :, 1:65].transpose(0, 1), wide[:1, :64].expand(9, 64)):
        check(binding, x, top_k=6)
    x = wide[:, 3:67]
    h = binding.Router(64, 6, renormalize=False)
    experts, _, _ = h.route(x)
    dw = torch.randn((24, 6), device="cuda", generator=gen(8))
    want = h.grad(x, experts, dw)
    room = torch.full((24, 201), 7.0, device="cuda", dtype=torch.bfloat16)
    h.grad(x, experts, dw, out=room[:, 100:164])
    assert torch.equal(room[:, 100:164], want) and bool((room[:, :100] == 7.0).all()) and bool((room[:, 164:] == 7.0).all())
    before = wide.clone()
    h.grad(x, experts, dw, out=x)
    assert torch.equal(wide[:, 3:67], want) and torch.equal(wide[:, :3], before[:, :3]) and torch.equal(wide[:, 67:], before[:, 67:])


def test_no_rows_and_many(binding):
    h = binding.Router(16, 4)
    counts = torch.full((16,), 9, device="cuda", dtype=torch.int32)
    experts, weights, _ = h.route(torch.zeros((0, 16), device="cuda"), counts_out=counts)
    assert experts.shape == (0, 4) and weights.shape == (0, 4) and not bool(counts.any())
    assert h.grad(torch.zeros((0, 16), device="cuda"), experts, weights).shape == (0, 16)
    x = rows(300_001, 16, "bf16", 4)
    experts, weights, counts = h.route(x)
    want = torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :4]
    assert torch.equal(experts.long(), want) and torch.equal(counts.long(), torch.bincount(want.reshape(-1), minlength=16))
    assert bool(((weights.double() - torch.softmax(x.double().gather(1, want), 1)).abs() <= REL).all())


def test_experts_twice_and_outside(binding):
    x = rows(4, 10, "f32", 2)
    dw = torch.randn((4, 3), device="cuda", generator=gen(3))
    for score, renormalize in (("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)):
        h = binding.Router(10, 3, score=score, renormalize=renormalize)
        given = torch.tensor([[1, 1, 4], [7, 2, 7], [5, 5, 5], [0, 3, 9]], device="cuda", dtype=torch.int32)
        once = torch.tensor([[1, -1, 4], [7, 2, -1], [5, -1, -1], [0, 3, 9]], device="cuda", dtype=torch.int32)
        assert torch.equal(h.grad(x, given, dw), h.grad(x, once, dw))
        assert h.last_error() == 0
        given[0, 1], given[2, 0] = 10, 2 ** 31 - 1
        once[2] = torch.tensor([-1, 5, -1])
        assert torch.equal(h.grad(x, given, dw), h.grad(x, once, dw))
        assert h.last_error() == binding.ERR_INVALID and h.last_error() == 0


def test_calls_in_a_row_other_stream_and_graph(binding):
    x = rows(5000, 60, "f16", 3)
    bias = torch.randn(60, device="cuda", generator=gen(4)) * 0.01
    h = binding.Router(60, 4, renormalize=False)
    first = h.route(x, bias=bias)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(h.route(x, bias=bias), first))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = h.route(x, bias=bias, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, first))
    graphs, held, outs = [], x.clone(), []
    dw = torch.randn((5000, 4), device="cuda", generator=gen(5))
    for _ in range(2):                                  # two graphs that share the handle, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            experts, weights, counts = h.route(held, bias=bias)
            outs.append((experts, weights, counts, h.grad(held, experts, dw)))
        graphs.append(g)
    for seed in (8, 9):
        held.copy_(rows(5000, 60, "f16", seed))
        for g in graphs:
            g.replay()
        want = h.route(held.clone(), bias=bias)
        for o in outs:
            assert all(torch.equal(a, b) for a, b in zip(o, (*want, h.grad(held.clone(), want[0], dw))))


def test_refusals(binding):
    for bad in (dict(experts=0, top_k=1), dict(experts=1025, top_k=1), dict(experts=8, top_k=0), dict(experts=8, top_k=9), dict(experts=64, top_k=33),
                dict(experts=8, top_k=2, groups=3), dict(experts=64, top_k=2, groups=64), dict(experts=8, top_k=2, groups=4, top_groups=5),
                dict(experts=8, top_k=2, groups=4, top_groups=0), dict(experts=8, top_k=3, groups=4, top_groups=1),
                dict(experts=8, top_k=2, group_terms=3), dict(experts=8, top_k=2, group_terms=0), dict(experts=8, top_k=2, scale=math.inf),
                dict(experts=8, top_k=-1)):
        with pytest.raises(binding.AdacompError):
            binding.Router(**bad)
    with pytest.raises(ValueError):
        binding.Router(8, 2, score="linear")
    h = binding.Router(8, 2)
    x = torch.zeros((4, 8), device="cuda")
    with pytest.raises(ValueError):
        h.route(x[:, :7])
    with pytest.raises(TypeError):
        h.route(x.double())
    with pytest.raises(TypeError):
        h.route(x.cpu())
    with pytest.raises(TypeError):
        h.route(torch.zeros((4, 16), device="cuda")[:, ::2])
    with pytest.raises(ValueError):
        h.route(x, bias=torch.zeros(7, device="cuda"))
    with pytest.raises(TypeError):
        h.route(x, bias=torch.zeros(8, device="cuda", dtype=torch.float16))
    with pytest.raises(TypeError):
        h.route(x, live=torch.ones(4, device="cuda"))
    with pytest.raises(ValueError):
        h.route(x, live=torch.ones(5, device="cuda", dtype=torch.bool))
    experts, weights, _ = h.route(x)
    with pytest.raises(TypeError):
        h.grad(x, experts.long(), weights)
    with pytest.raises(ValueError):
        h.grad(x, experts, weights[:, :1].contiguous())
    with pytest.raises(ValueError):
        h.grad(x, experts, weights, out=x[:3])
    with pytest.raises(ValueError):
        room = torch.zeros((4, 12), device="cuda")
        h.grad(room[:, :8], experts, weights, out=room[:, 4:])
    with pytest.raises(binding.AdacompError):
        h.grad(x, experts, weights, out=torch.zeros(40, device="cuda").as_strided((4, 8), (4, 1)))
    assert h.last_error() == 0


def test_rows_with_exactly_a_warps_candidates(binding):
    """32 experts to choose from and 32 places: nothing stands behind the last one."""
    for experts, groups in ((32, 1), (96, 3), (1024, 32)):
        bias = torch.randn(experts, device="cuda", generator=gen(experts)) * 0.05
        for score in ("softmax", "sigmoid"):
            check(binding, rows(300, experts, "f32", experts), bias, top_k=32, score=score, groups=groups, top_groups=1, group_terms=2)


def test_infinite_biases(binding):
    """+Inf: chosen before all others, of several the lowest first; -Inf: never."""
    bias = torch.zeros(64, device="cuda")
    bias[[50, 9, 33]] = math.inf
    bias[:5] = -math.inf
    for score in ("softmax", "sigmoid"):
        experts, _, _, _ = check(binding, rows(40, 64, "bf16", 3), bias, top_k=5, score=score)
        assert bool((experts[:, :3] == torch.tensor([9, 33, 50], device="cuda", dtype=torch.int32)).all()) and bool((experts >= 5).all())


@pytest.mark.parametrize("experts", [40, 748])
def test_close_ones_behind_equal_ones(binding, experts):
    """Sigmoids that are 1 in fp32: two equal logits stand before a larger one, which 64 bits choose."""
    x = rows(60, experts, "f32", 4)
    x[:, [3, 20]] = 18.0
    x[:, 31] = 19.0
    x[30:, 5:15] = 18.0
    zero = torch.zeros(experts, device="cuda")
    for k in (1, 2, 3):
        experts_, _, _, _ = check(binding, x, zero, top_k=k, score="sigmoid")
        assert bool((experts_[:, 0] == 31).all())
    many = torch.full((20, experts), 18.0, device="cuda")       # more equal ones than a warp has lanes
    many[:, 35] = 19.0
    check(binding, many, zero, top_k=2, score="sigmoid")
