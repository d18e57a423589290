"""Global gradient norm and clipping (CUDA, through the C ABI) against sums in 64 bits.

Tolerances, with u = 2^-24 (half a unit in the last place of fp32):
  norm   squares are added in fp32 in chains of at most 32 additions (all terms positive: at most 33 u relative, with the
         rounding of the squares), the rest in 64 bits; the root halves it, the result is rounded once: below 18 u.
  out    with the factor c that the call reports, out = round(fp32(g) * c) exactly: compared bit for bit.
  c      from the norm in 64 bits: 18 u and its own rounding.
"""
import ctypes
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)
U = 2.0 ** -24
NORM_TOL = 18 * U
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def binding():
    from paper_1702_04683_b200 import binding as b
    return b


def normals(n, seed, dtype=torch.float32, sigma=1e-2, offset=0):
    """n entries that start `offset` entries behind a 256-byte boundary."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return (torch.randn(n + offset, device=DEV, generator=gen) * sigma).to(dtype)[offset:]


def exact_norm(tensors, scale=1.0):
    return abs(scale) * math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in tensors))


def check_norm(got, want):
    assert abs(float(got) - want) <= NORM_TOL * want + 1e-45


def check_clip(binding, grads, outs, max_norm, scale=1.0, handle=None):
    """One worker's list: norm, factor and outputs of a call."""
    handle = handle or binding.Clipper()
    want = exact_norm(grads, scale)
    before = [g.clone() for g in grads]
    coef = torch.empty(1, device=DEV)
    out, norm = handle.clip(grads, max_norm, scale=scale, out=outs, coef_out=coef)
    check_norm(norm, want)
    c = scale * min(1.0, max_norm / (want + 1e-6))
    assert abs(float(coef) - c) <= (NORM_TOL + U) * abs(c)
    for o, g, kept in zip(out, grads, before):
        assert torch.equal(o, (kept.float() * coef).to(o.dtype))
        if outs is not None:
            assert torch.equal(g, kept)
    return coef


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 4095, 4096, 4097, 8192 + 3, 70_001])
@pytest.mark.parametrize("offset", [0, 1, 3, 6])
def test_norm_sizes_and_alignments(binding, dtype, n, offset):
    g = normals(n, n + offset, dtype, offset=offset)
    h = binding.Clipper()
    check_norm(h.norm([g]), exact_norm([g]))
    assert torch.equal(h.norm([g]), h.norm([g]))
    check_norm(h.norm([g], scale=-0.25), exact_norm([g], 0.25))


@pytest.mark.parametrize("kind_in", TYPES)
@pytest.mark.parametrize("kind_out", TYPES)
@pytest.mark.parametrize("n,skew_in,skew_out", [(1, 0, 0), (5, 1, 2), (9_001, 0, 0), (9_001, 3, 0), (9_001, 0, 5), (33_333, 5, 3), (33_333, 7, 2),
                                               (16_384, 2, 2)])
def test_clip_types_and_alignments(binding, kind_in, kind_out, n, skew_in, skew_out):
    g = normals(n, n, kind_in, sigma=0.1, offset=skew_in)
    buf = torch.full((n + skew_out + 16,), 7.0, device=DEV, dtype=kind_out)
    check_clip(binding, [g], [buf[skew_out:skew_out + n]], max_norm=0.05)
    assert bool((buf[:skew_out] == 7).all()) and bool((buf[skew_out + n:] == 7).all())      # nothing beside it was written


@pytest.mark.parametrize("count", [1, 63, 64, 65, 161, 959, 960, 961, 2_000])
def test_lists_of_many_tensors(binding, count):
    sizes = [(37 * i * i + 11 * i) % 3000 for i in range(count)]            # some are empty
    sizes[count // 2] = 50_021
    grads = [normals(n, i, TYPES[i % 3], offset=i % 5) for i, n in enumerate(sizes)]
    outs = [torch.empty(n, device=DEV, dtype=TYPES[(i // 3) % 3]) for i, n in enumerate(sizes)]
    check_clip(binding, grads, outs, max_norm=0.5, scale=2.0)
    given = binding.GradList(grads, out=outs)
    h = binding.Clipper()
    a = h.norm(given)
    assert torch.equal(a, h.norm(grads))
    for g in grads:
        g.mul_(3)                                                           # the list sees the tensors as they are now
    check_norm(h.norm(given), exact_norm(grads))


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place(binding, dtype):
    grads = [normals(n, n, dtype, sigma=0.05, offset=i) for i, n in enumerate((1_000, 20_001, 3))]
    check_clip(binding, grads, None, max_norm=0.25)
    kept = [g.clone() for g in grads]
    h = binding.Clipper()
    out, norm = h.clip(grads, float("inf"))                                 # no clipping, no scale: left as it is
    assert all(torch.equal(a, b) for a, b in zip(out, kept))
    check_norm(norm, exact_norm(kept))
    h.clip(grads, 1e6, scale=0.5)                                           # not clipped, but scaled
    assert all(torch.equal(a, (b.float() * 0.5).to(dtype)) for a, b in zip(grads, kept))


def test_dense_tensors_of_any_order_and_transposed_ones(binding):
    a = normals(48 * 40, 1).view(48, 40)
    grads = [a.t(), normals(2 * 3 * 4 * 5, 2).view(2, 3, 4, 5).permute(0, 3, 1, 2)]
    outs = [torch.empty_like(g) for g in grads]
    check_clip(binding, grads, outs, max_norm=0.1)
    with pytest.raises(TypeError):
        binding.GradList([a[:, 1:]])
    with pytest.raises(ValueError):
        binding.GradList([a.t()], out=[torch.empty(40, 48, device=DEV)])


@pytest.mark.parametrize("workers", [1, 2, 7, 64, 1_000])
@pytest.mark.parametrize("kind_in,kind_out", [(torch.float32, torch.float32), (torch.float16, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_workers_with_strides(binding, workers, kind_in, kind_out):
    n = 3_001 if workers > 10 else 60_013
    g = normals(workers * (n + 5), workers, kind_in, sigma=0.01).view(workers, n + 5)[:, 2:2 + n]
    g[0] *= 0.001                                                           # this one is not clipped
    buf = torch.full((workers, n + 3), 7.0, device=DEV, dtype=kind_out)
    h = binding.Clipper(max_workers=workers)
    coef = torch.empty(workers, device=DEV)
    out, norm = h.clip(g, 0.5, out=buf[:, 1:1 + n], coef_out=coef)
    want = (g.double() ** 2).sum(1).sqrt()
    assert bool(((norm.double() - want).abs() <= NORM_TOL * want).all())
    assert float(coef[0]) == 1.0
    assert torch.equal(out, (g.float() * coef.view(-1, 1)).to(kind_out))
    assert bool((buf[:, 0] == 7).all()) and bool((buf[:, 1 + n:] == 7).all())
    assert torch.equal(h.norm(g), norm)


def test_large_and_tiny_entries(binding):
    h = binding.Clipper()
    for value in (1e-30, 3e-42, 1e-22, 1e19, 1e30):                         # their squares leave fp32's range
        for dtype in (torch.float32, torch.bfloat16):
            g = torch.full((10_001,), value, device=DEV).to(dtype)
            check_norm(h.norm([g]), exact_norm([g]))
    g = torch.zeros(100_000, device=DEV)
    assert float(h.norm([g])) == 0.0
    g[77_777] = 1e-30                                                       # one tiny entry among zeros
    check_norm(h.norm([g]), exact_norm([g]))
    g[3] = 1e25
    check_norm(h.norm([g]), exact_norm([g]))
    big = torch.full((10_000,), 3e38, device=DEV)                           # the norm itself is beyond fp32: clipping still works
    coef = torch.empty(1, device=DEV)
    out, norm = h.clip([big], 1.0, out=[torch.empty_like(big)], coef_out=coef)
    assert math.isinf(float(norm))
    assert torch.equal(out[0], big * coef) and abs(float(out[0].double().norm()) - 1.0) < 1e-3


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan(binding, dtype):
    h = binding.Clipper(max_workers=4)
    g = normals(4 * 9_000, 5, dtype).view(4, 9_000).clone()
    g[1, 8_999] = float("inf")
    g[2, 0] = float("nan")
    g[3, 4_444] = float("-inf")
    out, norm = h.clip(g, 0.1, out=torch.empty_like(g))
    assert math.isfinite(float(norm[0])) and math.isinf(float(norm[1])) and math.isnan(float(norm[2])) and math.isinf(float(norm[3]))
    want = (g.double() ** 2).sum(1).sqrt()
    check_norm(norm[0], float(want[0]))                                     # the others' infinities do not reach it
    assert not bool(torch.isnan(out[0]).any())
    assert bool(torch.isnan(out[1, 8_999])) and bool((out[1, :8_999] == 0).all())
    assert bool(torch.isnan(out[2]).all())
    assert bool(torch.isnan(out[3, 4_444])) and bool((out[3, :4_444] == 0).all())
    out, norm = h.clip(g, float("inf"), scale=0.5, out=torch.empty_like(g))  # nothing is clipped: scaled all the same
    assert torch.equal(out[1], (g[1].float() * 0.5).to(dtype)) and math.isnan(float(norm[2]))


def test_entries_beyond_32_bits(binding):
    n = 2 ** 32 + 70_003
    g = torch.zeros(n, device=DEV, dtype=torch.bfloat16)
    for at, v in ((5, 3.0), (2 ** 31 + 1, 4.0), (2 ** 32 + 1, 12.0), (n - 1, 84.0)):
        g[at] = v
    h = binding.Clipper()
    out, norm = h.clip([g], 8.5)
    assert float(norm) == math.sqrt(9 + 16 + 144 + 84 * 84) == 85.0
    assert [float(g[at]) for at in (5, 2 ** 31 + 1, 2 ** 32 + 1, n - 1)] == [float(torch.tensor(v * 0.1).bfloat16()) for v in (3.0, 4.0, 12.0, 84.0)]


def test_no_entries(binding):
    h = binding.Clipper(max_workers=3)
    empty = torch.empty(0, device=DEV)
    out, norm = h.clip([empty, empty.bfloat16()], 1.0)
    assert norm.tolist() == [0.0]
    out, norm = h.clip(torch.empty((3, 0), device=DEV), 1.0)
    assert norm.tolist() == [0.0] * 3


def test_another_stream_and_calls_in_a_row(binding):
    side = torch.cuda.Stream()
    h = binding.Clipper()
    g = normals(3_000_001, 9)
    want = exact_norm([g])
    side.wait_stream(torch.cuda.current_stream())
    norms = [h.norm([g], stream=side) for _ in range(5)]
    out, norm = h.clip([g], 1.0, out=[torch.empty_like(g)], stream=side)
    side.synchronize()
    for x in norms + [norm]:
        check_norm(x, want)
        assert torch.equal(x, norm)


def test_empty_tensor_without_addresses_among_several_workers(binding):
    """An entry of n = 0 with null pointers is no tensor in place: it asks nothing of the strides."""
    g, out = normals(2 * 110, 1).view(2, 110), torch.full((2, 130), 7.0, device=DEV)
    norm, coef = torch.empty(2, device=DEV), torch.empty(2, device=DEV)
    table = (binding.GradTensor * 2)(binding.GradTensor(None, None, 0, 0, 0), binding.GradTensor(g.data_ptr(), out.data_ptr(), 100, 0, 0))
    h = binding.Clipper(max_workers=2)
    assert binding.raw().adacomp_clip(h._h, table, 2, 110, 130, 2, 1.0, 0.1, norm.data_ptr(), coef.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(out[:, :100], g[:, :100] * coef.view(2, 1)) and bool((out[:, 100:] == 7).all())
    for w in range(2):
        check_norm(norm[w], exact_norm([g[w, :100]]))


def test_norms_of_tensors_that_share_memory(binding):
    """A norm writes to no gradient: tied tensors, overlapping ones and a row that all workers share are counted as often as they are
    given.  Clipping them in place is refused as before."""
    g = normals(5_000, 1)
    h = binding.Clipper(max_workers=3)
    for tensors in ([g, g], [g[:3_000], g[2_000:]], [g.view(50, 100), g.view(50, 100).t(), g[7:8]]):
        check_norm(h.norm(tensors), exact_norm(tensors))
        check_norm(h.norm(binding.GradList(tensors)), exact_norm(tensors))
        kept = g.clone()
        for given in (tensors, binding.GradList(tensors)):
            with pytest.raises(ValueError):
                h.clip(given, 1.0)
        assert torch.equal(g, kept)
    for rows in (g.expand(3, -1), g.as_strided((3, 1_000), (500, 1))):
        norm = h.norm(rows)
        assert norm.shape == (3,)
        for w in range(3):
            check_norm(norm[w], exact_norm([rows[w]]))
        out = torch.empty((3, rows.shape[1]), device=DEV)
        coef = torch.empty(3, device=DEV)
        h.clip(rows, 0.01, out=out, coef_out=coef)
        assert torch.equal(out, rows * coef.view(3, 1))
        with pytest.raises(TypeError):
            h.clip(rows, 0.01)


def test_misaligned_results_are_refused(binding):
    lib = binding.raw()
    h = binding.Clipper()
    g = torch.ones(100, device=DEV)
    e = binding.GradTensor(g.data_ptr(), g.data_ptr(), 100, 0, 0)
    at = torch.zeros(64, dtype=torch.uint8, device=DEV).data_ptr()
    for off in (1, 2, 3):
        assert lib.adacomp_grad_norm(h._h, ctypes.byref(e), 1, 0, 1, 1.0, at + off, None) == binding.ERR_INVALID
        assert lib.adacomp_clip(h._h, ctypes.byref(e), 1, 0, 0, 1, 1.0, 1.0, at + off, None, None) == binding.ERR_INVALID
        assert lib.adacomp_clip(h._h, ctypes.byref(e), 1, 0, 0, 1, 1.0, 1.0, at, at + off, None) == binding.ERR_INVALID


def test_handle_made_on_a_stream_whose_work_is_not_done(binding):
    """The workspace may be memory that earlier work of the stream has still to write to."""
    g = normals(3_000_001, 9)
    want = exact_norm([g])
    torch.cuda._sleep(1)                                                    # all kernels are loaded before it matters: loading waits
    torch.empty(9, dtype=torch.uint8, device=DEV).fill_(255)
    binding.Clipper().norm([g])
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        size = binding.Clipper().workspace.numel()
        side.synchronize()
        junk = torch.empty(size, dtype=torch.uint8, device=DEV)
        at = junk.data_ptr()
        torch.cuda._sleep(100_000_000)                                      # some 50 ms
        junk.fill_(255)
        del junk
        h = binding.Clipper()
        assert h.workspace.data_ptr() == at                                 # otherwise this shows nothing
        norm = h.norm([g])
    side.synchronize()
    check_norm(norm, want)


def test_handle_dropped_while_another_stream_works(binding):
    """Its workspace must not be handed out again before that stream is through."""
    g = normals(3_000_001, 9)
    want = exact_norm([g])
    torch.cuda._sleep(1)                                                    # all kernels are loaded before it matters: loading waits
    torch.empty(9, dtype=torch.uint8, device=DEV).fill_(255)
    binding.Clipper().norm([g])
    side = torch.cuda.Stream()
    for given in (True, False):
        torch.cuda.synchronize()
        h = binding.Clipper()
        size = h.workspace.numel()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)                                  # some 50 ms
            if not given:
                norm = h.norm([g])
        if given:
            norm = h.norm([g], stream=side)
        del h
        junk = [torch.empty(size, dtype=torch.uint8, device=DEV).fill_(255) for _ in range(8)]
        side.synchronize()
        check_norm(norm, want)
        del junk


@pytest.mark.parametrize("workers", [3, 64, 444, 445, 5_000])
def test_partial_sums_of_workers_keep_apart(binding, workers):
    """Workers of several blocks and of one, in a workspace as small as it may be: every norm is its own worker's."""
    n = 2_000_000 // workers + 20_000
    g = normals(workers * n, workers).view(workers, n)
    g *= torch.arange(1, workers + 1, device=DEV).view(-1, 1)
    h = binding.Clipper(max_workers=workers)
    want = (g.double() ** 2).sum(1).sqrt()
    for _ in range(3):
        assert bool(((h.norm(g).double() - want).abs() <= NORM_TOL * want).all())
    longer = [g[0], *(normals(17, i) for i in range(1_000))]                # two launches, one after the other's partial sums
    check_norm(h.norm(longer), exact_norm(longer))


@pytest.mark.parametrize("kind", [torch.float32, torch.float16])
def test_gradients_and_outputs_in_rows_of_one_buffer(binding, kind):
    """A buffer whose rows hold a worker's gradient and the place for its clipped one: nothing overlaps unless their columns do."""
    W, n = 5, 3_000
    h = binding.Clipper(max_workers=W)
    for first, second in ((0, n), (n + 16, 7), (3, n + 3)):
        buf = normals(W * (2 * n + 16), 3, kind).view(W, 2 * n + 16)
        kept = buf.clone()
        coef = torch.empty(W, device=DEV)
        h.clip(buf[:, first:first + n], 0.1, out=buf[:, second:second + n], coef_out=coef)
        kept[:, second:second + n] = (kept[:, first:first + n].float() * coef.view(W, 1)).to(kind)
        assert torch.equal(buf, kept)
    for first, second in ((0, n - 1), (n, 1), (n + 16, n + 9)):
        with pytest.raises(ValueError):
            h.clip(buf[:, first:first + n], 0.1, out=buf[:, second:second + n])
    shifted = buf[:-1, n + 16:], buf[1:, :n]                                # row w beside row w + 1
    assert shifted[0].shape == shifted[1].shape
    before = shifted[0].clone()
    h.clip(shifted[0], float("inf"), out=shifted[1])
    assert torch.equal(shifted[1], before)
    with pytest.raises(ValueError):
        h.clip(shifted[0], 0.1, out=buf[:-1, n + 10:2 * n + 10])


def test_refusals(binding):
    lib = binding.raw()
    h = binding.Clipper(max_workers=2)
    g = torch.ones(100, device=DEV)
    norm = torch.zeros(2, device=DEV)

    def clip(n_tensors=1, workers=1, scale=1.0, max_norm=1.0, norm_ptr=norm.data_ptr(), **fields):
        e = binding.GradTensor()
        e.d_grad, e.d_out, e.n, e.grad_type, e.out_type = g.data_ptr(), g.data_ptr(), 100, 0, 0
        for k, v in fields.items():
            setattr(e, k, v)
        return lib.adacomp_clip(h._h, ctypes.byref(e), n_tensors, 0, 0, workers, scale, max_norm, norm_ptr, None, None)

    for bad in (dict(workers=0), dict(workers=3), dict(scale=math.inf), dict(scale=math.nan), dict(max_norm=0.0), dict(max_norm=-1.0),
                dict(max_norm=math.nan), dict(norm_ptr=None), dict(d_grad=None), dict(d_out=None), dict(grad_type=3), dict(out_type=-1),
                dict(d_grad=g.data_ptr() + 2), dict(d_out=g.data_ptr() + 1), dict(out_type=1), dict(n=1 << 40)):
        assert clip(**bad) == binding.ERR_INVALID, bad
    assert lib.adacomp_clip(h._h, None, 1, 0, 0, 1, 1.0, 1.0, norm.data_ptr(), None, None) == binding.ERR_INVALID
    two, to = torch.ones((2, 100), device=DEV), torch.zeros((2, 100), device=DEV)
    for d_out, stride, out_stride, want in ((to, 100, 99, binding.ERR_INVALID), (to, 100, 0, binding.ERR_INVALID), (two, 100, 101, binding.ERR_INVALID),
                                            (two, 100, 100, 0), (to, 0, 100, 0), (to, 100, 100, 0)):
        e = binding.GradTensor(two.data_ptr(), d_out.data_ptr(), 100, 0, 0)
        assert lib.adacomp_clip(h._h, ctypes.byref(e), 1, stride, out_stride, 2, 1.0, 1.0, norm.data_ptr(), None, None) == want
    assert clip() == 0 and clip(n_tensors=0) == 0
    torch.cuda.synchronize()
    for bad in (lambda: h.norm(g), lambda: h.norm([g.double()]), lambda: h.norm([g.cpu()]),
                lambda: h.norm(torch.ones(2, 100, device=DEV)[:, ::2]), lambda: h.clip(torch.ones(2, 8, device=DEV), 1.0, out=torch.ones(2, 9, device=DEV)),
                lambda: h.clip([g], 1.0, out=[g[:50]]), lambda: h.clip([g, g], 1.0), lambda: h.clip([g[:60]], 1.0, out=[g[20:80]]),
                lambda: h.clip([g[:50], g[50:]], 1.0, out=[torch.empty(50, device=DEV), g[:50]]),
                lambda: h.clip(binding.GradList([g]), 1.0, out=[g]), lambda: h.norm([g], norm_out=norm),
                lambda: h.clip(torch.ones(1, 8, device=DEV).expand(2, 8), 1.0)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(binding.AdacompError):
        h.norm(torch.ones(3, 8, device=DEV))
