"""Argument checks of the clipping and embedding entry points at the C boundary: they answer before any CUDA call is
made, so no GPU is needed."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_1702_04683_b200 import build
    build.build()
    from paper_1702_04683_b200 import binding as b
    return b


P = ctypes.c_void_p


def test_clip_workspace_and_create(binding):
    lib = binding.raw()
    n, more = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.adacomp_clip_workspace_bytes(1, ctypes.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    assert lib.adacomp_clip_workspace_bytes(16, ctypes.byref(more)) == 0 and more.value > n.value
    assert lib.adacomp_clip_workspace_bytes(0, ctypes.byref(n)) == binding.ERR_INVALID
    assert lib.adacomp_clip_workspace_bytes(65536, ctypes.byref(n)) == binding.ERR_INVALID
    assert lib.adacomp_clip_workspace_bytes(1, None) == binding.ERR_INVALID
    h = P()
    assert lib.adacomp_clip_create(None, 1, P(0x1000), 1 << 20, 0) == binding.ERR_INVALID
    assert lib.adacomp_clip_create(ctypes.byref(h), 1, None, 1 << 20, 0) == binding.ERR_INVALID
    assert lib.adacomp_clip_create(ctypes.byref(h), 1, P(0x1001), 1 << 20, 0) == binding.ERR_INVALID
    assert lib.adacomp_clip_create(ctypes.byref(h), 1, P(0x1000), 16, 0) == binding.ERR_ALLOC
    assert h.value is None


def test_clip_workspace_stays_small(binding):
    """The blocks of a call share the device: many workers have few each."""
    n = ctypes.c_size_t(0)
    for workers in (1, 16, 1_000, 65_535):
        assert binding.raw().adacomp_clip_workspace_bytes(workers, ctypes.byref(n)) == 0
        assert n.value <= 16_384 + 256 * workers


def test_clip_null_handles(binding):
    lib = binding.raw()
    t = binding.GradTensor()
    assert lib.adacomp_grad_norm(None, ctypes.byref(t), 1, 0, 1, 1.0, P(0x1000), None) == binding.ERR_INVALID
    assert lib.adacomp_clip(None, ctypes.byref(t), 1, 0, 0, 1, 1.0, 1.0, P(0x1000), None, None) == binding.ERR_INVALID
    assert lib.adacomp_clip_destroy(None) == 0


def test_embed_workspace_and_create(binding):
    lib = binding.raw()
    n, more = ctypes.c_size_t(0), ctypes.c_size_t(0)
    size = lib.adacomp_embed_workspace_bytes
    assert size(100, 8, 1000, 1, ctypes.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    assert size(100, 8, 100000, 1, ctypes.byref(more)) == 0 and more.value > n.value
    assert size(100, 8, 0, 1, ctypes.byref(more)) == 0 and 0 < more.value <= n.value
    for bad in ((0, 8, 10, 1), (10, 0, 10, 1), (10, 8, 10, 0), (10, 8, 2**31, 1), (10, 2**31, 10, 1), (2**31, 8, 10, 2),
                (2**32 - 1, 8, 10, 1)):
        assert size(*bad, ctypes.byref(n)) == binding.ERR_INVALID
    assert size(2**31 - 1, 8, 10, 2, ctypes.byref(n)) == 0
    assert size(10, 8, 10, 1, None) == binding.ERR_INVALID
    h = P()
    create = lib.adacomp_embed_create
    assert create(None, 10, 8, 10, 1, 0, P(0x1000), 1 << 20, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), 10, 8, 10, 1, 0, None, 1 << 20, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), 10, 8, 10, 1, 0, P(0x1010), 1 << 20, 0) == binding.ERR_INVALID
    assert create(ctypes.byref(h), 10, 8, 10, 1, 0, P(0x1000), 16, 0) == binding.ERR_ALLOC
    assert create(ctypes.byref(h), 0, 8, 10, 1, 0, P(0x1000), 1 << 20, 0) == binding.ERR_INVALID
    assert h.value is None


def test_embed_null_handles(binding):
    lib = binding.raw()
    r = binding.Rows()
    b = ctypes.byref(r)
    assert lib.adacomp_embed_lookup(None, b, b, 1, 1.0, b, None) == binding.ERR_INVALID
    assert lib.adacomp_embed_grad_rows(None, b, 1, 1, b, 1.0, None, P(0x1000), P(0x1000), 0, None, 0, None) == binding.ERR_INVALID
    assert lib.adacomp_embed_grad_dense(None, b, 1, 1, b, 1.0, b, 0, None) == binding.ERR_INVALID
    assert lib.adacomp_embed_last_error(None, None) == binding.ERR_INVALID
    assert lib.adacomp_embed_destroy(None) == 0


def test_wait_limit_of_no_handle(binding):
    assert binding.raw().adacomp_embed_set_wait_limit(None, 0) == binding.ERR_INVALID


def test_binding_refuses_host_tensors_and_unknown_types(binding):
    import torch
    with pytest.raises(TypeError):
        binding.GradList([torch.zeros(4)])
    with pytest.raises(ValueError):
        binding.GradList([])


def test_rows_of_strided_tensors(binding):
    """The two-level numbering of rows that the binding derives from a tensor's strides (host tensors will do)."""
    import torch

    def at(r, i):
        return i * r.row_stride if r.group == 0 else (i // r.group) * r.group_stride + (i % r.group) * r.row_stride

    base = torch.arange(6 * 10 * 8).view(6, 10, 8)
    views = [base, base[:, 1:], base[1:, ::2], base[:, 3], base[2], base.transpose(0, 1), base[:, :, :4], base[3:4, 2:3],
             base[::2, 1:-1, 2:], base[:1], base[:, 1:2]]
    for v in views:
        r = binding._rows(v, v.dim() - 1, 0, "x")
        flat = v.reshape(-1, v.shape[-1])
        for i in range(flat.shape[0]):
            assert (r.d_data - base.data_ptr()) // 8 + at(r, i) == int(flat[i, 0])
    tokens = base.view(60, 8)
    for v in (tokens, tokens[:, :-1], tokens[::3, 1:5], tokens.t(), tokens[:, 2], tokens[4:5, 3:4]):
        r = binding._rows(v, v.dim(), 1, "x")
        for i, x in enumerate(v.reshape(-1).tolist()):
            assert (r.d_data - base.data_ptr()) // 8 + at(r, i) == x
    with pytest.raises(TypeError):
        binding._rows(torch.zeros(4, 5, 6, 7)[::2, 1:4, 1:], 3, 0, "x")
    expanded = torch.zeros(1, 8).expand(30, 8)
    r = binding._rows(expanded, 1, 0, "x")
    assert (r.group, r.row_stride) == (0, 0)
