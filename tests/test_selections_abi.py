"""Argument checks of the distillation and routing entry points at the C boundary: they answer before any CUDA call is made, so no
GPU is needed (handles come from fakes where a call wants one: the checks below never reach what a handle points at)."""
import ctypes
import math

import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_1702_04683_b200 import build
    build.build()
    from paper_1702_04683_b200 import binding as b
    return b


P = ctypes.c_void_p


def test_distill_workspace_and_create(binding):
    lib = binding.raw()
    n = ctypes.c_size_t(0)
    size = lib.adacomp_distill_workspace_bytes
    for vocab in (1, 1000, 1 << 20):
        assert size(vocab, ctypes.byref(n)) == 0 and 0 < n.value <= 4096 and n.value % 256 == 0
    assert size(0, ctypes.byref(n)) == binding.ERR_INVALID
    assert size((1 << 20) + 1, ctypes.byref(n)) == binding.ERR_INVALID
    assert size(10, None) == binding.ERR_INVALID
    h = P()
    create = lib.adacomp_distill_create
    assert create(None, 10, P(0x1000), 4096, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), 0, P(0x1000), 4096, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), 10, None, 4096, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), 10, P(0x1010), 4096, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), 10, P(0x1000), 16, 0) == binding.ERR_ALLOC
    assert h.value is None


def config(binding, **kw):
    c = dict(experts=64, top_k=6, groups=1, top_groups=1, group_terms=1, score=0, renormalize=1, scale=1.0) | kw
    return binding.RouteConfig(*(c[n] for n, _ in binding.RouteConfig._fields_))


def test_route_workspace_and_create(binding):
    lib = binding.raw()
    n = ctypes.c_size_t(0)
    size = lib.adacomp_route_workspace_bytes
    for good in (dict(), dict(experts=1, top_k=1), dict(experts=1024, top_k=32, groups=32, top_groups=1), dict(score=1, renormalize=0, scale=-2.5),
                 dict(groups=8, top_groups=3, group_terms=2)):
        assert size(ctypes.byref(config(binding, **good)), ctypes.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    for bad in (dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=33), dict(top_k=65, experts=64), dict(groups=0), dict(groups=3),
                dict(groups=64), dict(top_groups=0), dict(groups=4, top_groups=5), dict(groups=32, top_groups=2, top_k=5), dict(group_terms=0),
                dict(group_terms=3), dict(score=2), dict(score=-1), dict(renormalize=2), dict(scale=math.inf), dict(scale=math.nan)):
        assert size(ctypes.byref(config(binding, **bad)), ctypes.byref(n)) == binding.ERR_INVALID, bad
    assert size(None, ctypes.byref(n)) == binding.ERR_INVALID
    assert size(ctypes.byref(config(binding)), None) == binding.ERR_INVALID
    h, c = P(), config(binding)
    create = lib.adacomp_route_create
    assert create(None, ctypes.byref(c), P(0x1000), 1 << 20, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), None, P(0x1000), 1 << 20, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), ctypes.byref(c), None, 1 << 20, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), ctypes.byref(c), P(0x1001), 1 << 20, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), ctypes.byref(c), P(0x1000), 16, 0) == binding.ERR_ALLOC
    assert h.value is None


def test_null_handles(binding):
    lib = binding.raw()
    r, p = binding.Rows(), binding.Pairs()
    b, q = ctypes.byref(r), ctypes.byref(p)
    assert lib.adacomp_top_logits(None, b, 1, 1, 1.0, P(0x1000), P(0x1000), None, None) == binding.ERR_INVALID
    assert lib.adacomp_distill_loss(None, b, 1, q, 1.0, None, P(0x1000), None, None) == binding.ERR_INVALID
    assert lib.adacomp_distill_grad(None, b, 1, q, 1.0, None, P(0x1000), b, None) == binding.ERR_INVALID
    assert lib.adacomp_distill_loss_grad(None, b, 1, q, 1.0, None, P(0x1000), b, None) == binding.ERR_INVALID
    assert lib.adacomp_distill_last_error(None, None) == binding.ERR_INVALID
    assert lib.adacomp_distill_destroy(None) == 0
    assert lib.adacomp_route(None, b, 1, None, None, P(0x1000), P(0x1000), None, None) == binding.ERR_INVALID
    assert lib.adacomp_route_grad(None, b, 1, P(0x1000), P(0x1000), b, None) == binding.ERR_INVALID
    assert lib.adacomp_route_last_error(None, None) == binding.ERR_INVALID
    assert lib.adacomp_route_destroy(None) == 0


class FakeDistill(ctypes.Structure):            # device, vocabulary, SMs, error word
    _fields_ = [("device", ctypes.c_int), ("vocab", ctypes.c_uint32), ("n_sms", ctypes.c_int), ("d_status", P)]


def rows(binding, at=0x10000, kind=0, group=0, row=100, stride=0):
    return binding.Rows(at, kind, group, row, stride)


def test_distill_arguments(binding):
    lib = binding.raw()
    h = ctypes.byref(FakeDistill(0, 100, 148, 0x1000))
    top, logits = lib.adacomp_top_logits, rows(binding)
    bad = binding.ERR_INVALID
    for k, t in ((0, 1.0), (101, 1.0), (1, 0.0), (1, -1.0), (1, math.nan), (1, math.inf), (1, 2.0 ** -21), (1, 2.0 ** 21)):
        assert top(h, ctypes.byref(logits), 4, k, t, P(0x1000), P(0x1000), None, None) == bad
    assert top(h, ctypes.byref(logits), 1 << 31, 1, 1.0, P(0x1000), P(0x1000), None, None) == bad
    assert top(h, None, 4, 1, 1.0, P(0x1000), P(0x1000), None, None) == bad
    assert top(h, ctypes.byref(logits), 4, 1, 1.0, None, P(0x1000), None, None) == bad
    assert top(h, ctypes.byref(logits), 4, 1, 1.0, P(0x1000), None, None, None) == bad
    assert top(h, ctypes.byref(logits), 4, 1, 1.0, P(0x1002), P(0x1000), None, None) == bad
    assert top(h, ctypes.byref(logits), 4, 1, 1.0, P(0x1000), P(0x1002), None, None) == bad
    assert top(h, ctypes.byref(rows(binding, at=0x10001)), 4, 1, 1.0, P(0x1000), P(0x1000), None, None) == bad
    assert top(h, ctypes.byref(rows(binding, kind=3)), 4, 1, 1.0, P(0x1000), P(0x1000), None, None) == bad
    assert top(h, ctypes.byref(rows(binding, at=None)), 0, 1, 1.0, None, None, None, None) == binding.OK         # no rows
    idx, val, out = rows(binding, 0x20000, 0, 0, 3), rows(binding, 0x30000, 0, 0, 3), rows(binding, 0x40000)
    good = binding.Pairs(idx, val, None, 3)
    both = lib.adacomp_distill_loss_grad
    for pairs in (binding.Pairs(idx, val, None, 0), binding.Pairs(idx, val, None, 1025), binding.Pairs(rows(binding, 0x20002), val, None, 3),
                  binding.Pairs(rows(binding, 0x20000, 2), val, None, 3), binding.Pairs(idx, rows(binding, 0x30002), None, 3),
                  binding.Pairs(idx, rows(binding, 0x30000, 5), None, 3), binding.Pairs(idx, val, 0x1002, 3), binding.Pairs(rows(binding, None), val, None, 3)):
        assert both(h, ctypes.byref(logits), 4, ctypes.byref(pairs), 1.0, None, P(0x1000), ctypes.byref(out), None) == bad
    g = ctypes.byref(good)
    assert both(h, ctypes.byref(logits), 4, None, 1.0, None, P(0x1000), ctypes.byref(out), None) == bad
    assert both(h, ctypes.byref(logits), 4, g, 1.0, P(0x1002), P(0x1000), ctypes.byref(out), None) == bad
    assert both(h, ctypes.byref(logits), 4, g, 1.0, None, P(0x1002), ctypes.byref(out), None) == bad
    assert both(h, ctypes.byref(logits), 4, g, 1.0, None, P(0x1000), None, None) == bad
    assert both(h, ctypes.byref(logits), 4, g, 1.0, None, P(0x1000), ctypes.byref(rows(binding, 0x40000, 1)), None) == bad       # another type
    assert both(h, ctypes.byref(logits), 4, g, 1.0, None, P(0x1000), ctypes.byref(rows(binding, 0x40000, 0, 0, 99)), None) == bad
    assert both(h, ctypes.byref(logits), 4, g, 0.0, None, P(0x1000), ctypes.byref(out), None) == bad
    assert lib.adacomp_distill_loss(h, ctypes.byref(logits), 4, g, 1.0, None, P(0x1000), P(0x1008), None) == bad
    assert lib.adacomp_distill_grad(h, ctypes.byref(logits), 4, g, 1.0, None, None, ctypes.byref(out), None) == bad
    assert lib.adacomp_distill_grad(h, ctypes.byref(logits), 0, g, 1.0, None, None, ctypes.byref(out), None) == binding.OK


class FakeRoute(ctypes.Structure):              # device, configuration, SMs, three places in the workspace
    pass


def test_route_arguments(binding):
    FakeRoute._fields_ = [("device", ctypes.c_int), ("config", binding.RouteConfig), ("n_sms", ctypes.c_int), ("d_status", P), ("d_ticket", P),
                          ("d_counts", P)]
    lib = binding.raw()
    h = ctypes.byref(FakeRoute(0, config(binding), 148, 0x1000, 0x1100, 0x1200))
    logits, bad = rows(binding, row=64), binding.ERR_INVALID
    route, grad = lib.adacomp_route, lib.adacomp_route_grad
    b = ctypes.byref(logits)
    assert route(h, None, 4, None, None, P(0x1000), P(0x1000), None, None) == bad
    assert route(h, b, 1 << 31, None, None, P(0x1000), P(0x1000), None, None) == bad
    assert route(h, b, 4, None, None, None, P(0x1000), None, None) == bad
    assert route(h, b, 4, None, None, P(0x1000), None, None, None) == bad
    assert route(h, b, 4, P(0x1002), None, P(0x1000), P(0x1000), None, None) == bad
    assert route(h, b, 4, None, None, P(0x1002), P(0x1000), None, None) == bad
    assert route(h, b, 4, None, None, P(0x1000), P(0x1002), None, None) == bad
    assert route(h, b, 4, None, None, P(0x1000), P(0x1000), P(0x1002), None) == bad
    out = rows(binding, 0x40000, row=64)
    o = ctypes.byref(out)
    assert grad(h, b, 4, None, P(0x1000), o, None) == bad
    assert grad(h, b, 4, P(0x1000), None, o, None) == bad
    assert grad(h, b, 4, P(0x1002), P(0x1000), o, None) == bad
    assert grad(h, b, 4, P(0x1000), P(0x1000), None, None) == bad
    assert grad(h, b, 4, P(0x1000), P(0x1000), ctypes.byref(rows(binding, 0x40000, 2, row=64)), None) == bad
    assert grad(h, b, 4, P(0x1000), P(0x1000), ctypes.byref(rows(binding, 0x40000, row=63)), None) == bad
    assert grad(h, b, 0, None, None, o, None) == binding.OK
