"""Embedding lookup and the table's gradient (CUDA, through the C ABI) against plain sums in 64 bits.

A lookup is one fp32 product and one rounding: compared bit for bit.  A sum of L gradient entries in fp32, in any order,
is off by at most (L - 1) u sum|g| (u = 2^-24); with the product by the scale and the rounding of fp32 (2^-24 relative, and the
smallest subnormal) that is the tolerance for fp32 results.  The order of a sum does not depend on the result's type, so
the others, and what is added to a table, have to be the fp32 result's roundings bit for bit.
"""
import ctypes

import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def binding():
    from paper_1702_04683_b200 import binding as b
    return b


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def words(shape, vocab, seed, skew=True, dtype=torch.int64):
    """Tokens of which a few are frequent."""
    r = torch.rand(shape, device=DEV, generator=gen(seed), dtype=torch.float64)
    return ((r ** 4 if skew else r) * vocab).long().clamp_(max=vocab - 1).to(dtype)


def plain(tokens, grad, vocab, workers, scale, pad):
    """Sums in 64 bits, sums of magnitudes, and counts of every worker's table: [W * V, D], [W * V, D], [W * V]"""
    D = grad.shape[-1]
    tok = tokens.reshape(workers, -1).long()
    live = (tok >= 0) & (tok < vocab)
    if pad is not None:
        live &= tok != pad
    key = (tok + torch.arange(workers, device=DEV).view(-1, 1) * vocab)[live]
    rows = grad.reshape(-1, D)[live.reshape(-1)].double()
    sums = torch.zeros((workers * vocab, D), dtype=torch.float64, device=DEV).index_add_(0, key, rows)
    size = torch.zeros_like(sums).index_add_(0, key, rows.abs())
    return sums * scale, size * abs(scale), torch.bincount(key, minlength=workers * vocab)


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=123.0), torch.nan_to_num(b.float(), nan=123.0)) and a.dtype == b.dtype


def near(got, want, size, count):
    tol = (count.double().view(-1, 1) + 1) * U * size
    tol = tol + U * (want.abs() + tol) + 2.0 ** -149
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), float((off - tol).max())


def check_grad(binding, tokens, grad, vocab, workers=1, scale=1.0, pad=None, out_type=torch.float32, handle=None, bad=False):
    """All three forms of one call against the plain sums."""
    D, n = grad.shape[-1], tokens.numel()
    h = handle or binding.Embedding(vocab, D, max_tokens=n, max_workers=workers, padding_idx=pad)
    want, size, count = plain(tokens, grad, vocab, workers, scale, pad)
    keys = count.nonzero().view(-1)
    U_ = len(keys)
    begin_want = [int((keys < w * vocab).sum()) for w in range(workers + 1)]
    # rows
    rows_out = torch.full((n,), -5, dtype=torch.int32, device=DEV)
    values_out = torch.full((n, D), 7.0, dtype=out_type, device=DEV)
    rows, values, begin = h.grad_rows(tokens, grad, scale=scale, workers=workers, rows_out=rows_out, values_out=values_out)
    assert begin.tolist() == begin_want
    assert torch.equal(rows[:U_].long(), keys % vocab) and bool((rows[U_:] == -5).all()) and bool((values[U_:] == 7).all())
    exact = h.grad_rows(tokens, grad, scale=scale, workers=workers)[1][:U_]
    near(exact, want[keys], size[keys], count[keys])
    assert same(values[:U_], exact.to(out_type))
    dense = torch.zeros((workers * vocab, D), device=DEV)
    dense[keys] = exact
    # update
    offset = 1_001
    idx, val, begin = h.grad_update(tokens, grad, scale=scale, workers=workers, offset=offset)
    assert begin.tolist() == begin_want
    assert torch.equal(idx[:U_].long() & 0xFFFFFFFF, (keys % vocab).view(-1, 1) * D + offset + torch.arange(D, device=DEV))
    assert same(val[:U_], exact)
    # dense, in buffers with gaps
    stride = vocab * D + 13 * 8
    buf = torch.full((workers, stride), 7.0, dtype=out_type, device=DEV)
    table = buf[:, 8:8 + vocab * D].view(workers, vocab, D)
    h.grad_dense(tokens, grad, table, scale=scale, workers=workers)
    assert same(table.reshape(-1, D), dense.to(out_type))
    assert bool((buf[:, :8] == 7).all()) and bool((buf[:, 8 + vocab * D:] == 7).all())
    # added to what is there
    base = torch.randn((workers, vocab, D), device=DEV, generator=gen(3)).to(out_type)
    acc = base.clone()
    h.grad_dense(tokens, grad, acc, scale=scale, workers=workers, accumulate=True)
    added = torch.where((count > 0).view(-1, 1), (dense + base.view(-1, D).float()).to(out_type), base.view(-1, D))
    assert same(acc.view(-1, D), added)
    assert h.last_error() == (binding.ERR_INVALID if bad else 0)
    assert h.last_error() == 0
    return h


# --------------------------------------------------------------------------------------------- lookup

@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("dim,tokens", [(1, 5), (7, 33), (64, 1), (64, 1000), (513, 100), (1000, 65), (2048, 17), (5000, 3)])
def test_lookup(binding, kind, out, dim, tokens):
    vocab = 211
    table = (torch.randn((vocab, dim), device=DEV, generator=gen(dim)) * 0.02).to(kind)
    ids = words((tokens,), vocab, tokens, skew=False, dtype=torch.int32 if tokens % 2 else torch.int64)
    h = binding.Embedding(vocab, dim)
    for scale in (1.0, dim ** 0.5):
        got = h.lookup(table, ids, scale=scale, dtype=out)
        assert torch.equal(got, (table[ids.long()].float() * scale).to(out))
    assert h.last_error() == 0


def test_lookup_shapes_strides_and_alignment(binding):
    vocab, dim = 97, 24
    wide = torch.randn((vocab, dim + 9), device=DEV, generator=gen(1))
    h = binding.Embedding(vocab, dim)
    data = words((6, 31), vocab, 2, skew=False)
    for table in (wide[:, :dim], wide[:, 8:8 + dim], wide[:, 3:3 + dim]):
        for ids in (data, data[:, :-1], data[:, 1:], data.t(), data[::2, 3:9], data[0, 0], data[:0]):
            got = h.lookup(table, ids)
            assert got.shape == (*ids.shape, dim) and torch.equal(got, table[ids])
            buf = torch.full((*ids.shape, dim + 5), 7.0, device=DEV)
            h.lookup(table, ids, scale=-2.0, out=buf[..., 2:2 + dim])
            assert torch.equal(buf[..., 2:2 + dim], table[ids] * -2.0)
            assert bool((buf[..., :2] == 7).all()) and bool((buf[..., 2 + dim:] == 7).all())
    out = torch.empty((31, 6, dim), device=DEV).transpose(0, 1)             # rows in another order
    assert torch.equal(h.lookup(table, data, out=out), table[data])


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_lookup_of_tokens_outside_the_vocabulary(binding, dtype):
    vocab, dim = 50, 40
    table = torch.randn((vocab, dim), device=DEV, generator=gen(1))
    ids = torch.tensor([0, -1, 49, 50, 7, 2 ** 31 - 1, -2 ** 31] + ([2 ** 32, 2 ** 32 + 3, -2 ** 63] if dtype == torch.int64 else []), device=DEV).to(dtype)
    h = binding.Embedding(vocab, dim)
    got = h.lookup(table, ids)
    ok = (ids >= 0) & (ids < vocab)
    assert torch.equal(got[ok], table[ids[ok].long()]) and bool((got[~ok] == 0).all())
    assert h.last_error() == binding.ERR_INVALID and h.last_error() == 0


def test_lookup_beyond_32_bits(binding):
    vocab, dim = 1_100_000, 4096                                            # 4.5e9 entries
    table = torch.empty((vocab, dim), device=DEV, dtype=torch.bfloat16)
    ids = torch.tensor([0, 1_048_575, 1_048_576, 1_048_577, vocab - 1], device=DEV)
    table[ids] = torch.randn((5, dim), device=DEV, generator=gen(1)).bfloat16()
    h = binding.Embedding(vocab, dim)
    assert torch.equal(h.lookup(table, ids), table[ids])


def test_lookup_keeps_infinities_and_nan(binding):
    table = torch.tensor([[1.0, float("inf"), float("nan"), -0.0], [float("-inf"), 2.0, 3.0, 4.0]], device=DEV)
    h = binding.Embedding(2, 4)
    got = h.lookup(table, torch.tensor([1, 0], device=DEV), scale=2.0, dtype=torch.float16)
    assert torch.equal(torch.nan_to_num(got, nan=-9.0), torch.nan_to_num((table[[1, 0]] * 2).half(), nan=-9.0))


def batch_of_tokens(n, vocab, seed, bad=0):
    """Tokens of which the table's first and last row are some, and `bad` lie outside."""
    ids = words((n,), vocab, seed, skew=False)
    ids[0], ids[n // 2], ids[-1] = vocab - 1, 0, vocab - 1
    if bad:
        ids[torch.randperm(n, device=DEV, generator=gen(seed))[:bad]] = vocab
    return ids


def check_lookup(binding, table, ids, out, scale, bad=False):
    """A lookup into `out`, a part of a larger buffer of sevens: the roundings bit for bit, and nothing beside them."""
    vocab, dim = table.shape
    h = binding.Embedding(vocab, dim)
    buf = out._base if out._base is not None else out
    buf.fill_(7.0)
    h.lookup(table, ids, scale=scale, out=out)
    assert h.last_error() == (binding.ERR_INVALID if bad else 0)
    ok = (ids >= 0) & (ids < vocab)
    want = torch.where(ok.view(-1, 1), table[ids.clamp(0, vocab - 1)].float() * scale, 0.0).to(out.dtype)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert bool((buf == 7).all())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("to", TYPES)
def test_lookup_of_large_batches_on_the_grid(binding, kind, to):
    """Several tokens per thread, row strides wider than the rows, outputs on the 32-byte grid and beside it."""
    vocab, dim, n = 3_001, 256, 80_003
    table = (torch.randn((vocab, dim + 24), device=DEV, generator=gen(1)) * 0.02).to(kind)[:, 8:8 + dim]
    ids = batch_of_tokens(n, vocab, 2, bad=3)
    for pad, at in ((0, 0), (32, 16), (8, 8)):
        out = torch.empty((n, dim + pad), device=DEV, dtype=to)[:, at:at + dim]
        for scale in (1.0, 16.0):
            check_lookup(binding, table, ids, out, scale, bad=True)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("to", TYPES)
@pytest.mark.parametrize("dim", [1, 7, 250, 511])
def test_lookup_of_large_batches_of_odd_rows(binding, kind, to, dim):
    """Single entries, several tokens per thread."""
    vocab, n = 3_001, 1_300_003 if dim == 1 else 700_001 if dim == 7 else 20_011
    wide = (torch.randn((vocab, dim + 3), device=DEV, generator=gen(1)) * 0.02).to(kind)
    for table, scale in ((wide[:, 1:1 + dim], 4.0), (wide[:, :dim].contiguous(), 1.0)):
        check_lookup(binding, table, batch_of_tokens(n, vocab, dim, bad=2), torch.empty((n, dim + 2), device=DEV, dtype=to)[:, 1:1 + dim], scale, bad=True)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("to", TYPES)
@pytest.mark.parametrize("n,dim", [(300, 513), (1_201, 1_001), (5_003, 1_001), (9_001, 519), (1_500, 4_099)])
def test_lookup_of_long_rows_off_the_grid(binding, kind, to, n, dim):
    """Few and many tokens; tables with and without gaps, their last row at the end of the memory; outputs at every offset."""
    vocab = 601
    for gap in (0, 3, 8):
        memory = (torch.randn((vocab - 1) * (dim + gap) + dim + 5, device=DEV, generator=gen(gap)) * 0.02).to(kind)
        for skip in (0, 5):
            table = memory[skip:].as_strided((vocab, dim), (dim + gap, 1))
            assert table.storage_offset() + (vocab - 1) * (dim + gap) + dim <= memory.numel()
            for at in ((0, 1, 2, 3, 4, 5, 6, 7) if skip else (0, 3)):
                out = torch.empty((n, dim + 9 - at % 2), device=DEV, dtype=to)[:, at:at + dim]
                check_lookup(binding, table, batch_of_tokens(n, vocab, at, bad=at % 3), out, 8.0 if gap else 1.0, bad=at % 3 > 0)


@pytest.mark.parametrize("kind,to,dim,n", [(torch.bfloat16, torch.bfloat16, 1024, 50_001), (torch.float32, torch.float32, 512, 50_001),
                                           (torch.bfloat16, torch.float32, 512, 50_001), (torch.float32, torch.float16, 1024, 50_001),
                                           (torch.float16, torch.float16, 1001, 51_003), (torch.float32, torch.float32, 333, 77_001)])
def test_lookup_whose_output_exceeds_the_cache(binding, kind, to, dim, n):
    """Above 96 MB, stores that pass L2 by; rows that start on 32 bytes and on 16 alone."""
    vocab = 2_003
    table = (torch.randn((vocab, dim), device=DEV, generator=gen(1)) * 0.02).to(kind)
    for pad in (0, 8 if to != torch.float32 else 4):
        out = torch.empty((n, dim + pad), device=DEV, dtype=to)[:, pad:]
        check_lookup(binding, table, batch_of_tokens(n, vocab, 5), out, 1.0 if pad else 0.5)


# --------------------------------------------------------------------------------------------- gradient

@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 257, 1024, 1025, 2048, 2049, 8192, 8193, 20_000, 70_000])
@pytest.mark.parametrize("vocab", [1, 2, 300, 70_000])
def test_numbers_of_tokens_and_vocabularies(binding, n, vocab):
    tokens = words((n,), vocab, n + vocab)
    grad = torch.randn((n, 16), device=DEV, generator=gen(n))
    check_grad(binding, tokens, grad, vocab)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("dim", [1, 6, 8, 64, 129, 1000, 1024, 2050])
def test_types_and_widths(binding, kind, out, dim):
    n, vocab = 1_500, 333
    tokens = words((n,), vocab, dim, dtype=torch.int32)
    grad = torch.randn((n, dim), device=DEV, generator=gen(dim)).to(kind)
    check_grad(binding, tokens, grad, vocab, scale=0.25, pad=5, out_type=out)


@pytest.mark.parametrize("spread", ["one", "two", "all different", "long runs", "falling"])
@pytest.mark.parametrize("n", [40, 3_000, 30_000])
def test_spreads(binding, spread, n):
    vocab, dim = max(n, 64), 64
    i = torch.arange(n, device=DEV)
    tokens = {"one": i * 0 + 17, "two": (i % 2) * 40 + 3, "all different": torch.randperm(n, device=DEV, generator=gen(n)),
              "long runs": i // 700, "falling": n - 1 - i}[spread]
    grad = torch.randn((n, dim), device=DEV, generator=gen(n)).bfloat16()
    check_grad(binding, tokens, grad, vocab, scale=3.0)


@pytest.mark.parametrize("workers,n,vocab", [(2, 1, 5), (3, 700, 100), (8, 2_048, 3_000), (50, 100, 11), (4, 9_000, 33)])
def test_workers(binding, workers, n, vocab):
    tokens = words((workers, n), vocab, n)
    tokens[workers // 2] = 3                                                # a worker with nothing but padding
    grad = torch.randn((workers, n, 40), device=DEV, generator=gen(n)).half()
    check_grad(binding, tokens, grad, vocab, workers=workers, scale=0.5, pad=3)


def test_only_padding_no_tokens_and_tokens_outside(binding):
    grad = torch.randn((300, 24), device=DEV, generator=gen(1))
    check_grad(binding, torch.full((300,), 4, device=DEV), grad, 9, pad=4)
    check_grad(binding, torch.empty((0,), dtype=torch.int64, device=DEV), grad[:0], 9, workers=1)
    tokens = words((300,), 9, 7)
    tokens[::3] = -1
    tokens[1::7] = 9
    tokens[5] = 2 ** 40
    check_grad(binding, tokens, grad, 9, bad=True)
    check_grad(binding, tokens * 0 - 1, grad, 9, bad=True)
    h = binding.Embedding(9, 24, max_tokens=300, padding_idx=4)
    h.grad_rows(words((300,), 9, 7), grad)                                  # a handle that has seen errors and others goes on
    check_grad(binding, words((200,), 9, 8), grad[:200], 9, pad=4, handle=h)


def test_strided_tokens_and_gradients(binding):
    data = words((7, 65), 50, 1)
    wide = torch.randn((7, 65, 48), device=DEV, generator=gen(2))
    for tokens, grad in ((data[:, :-1], wide[:, :-1]), (data[:, 1:], wide[:, 1:, :32]), (data[:, 1:], wide[:, 1:, 3:40]),
                         (data.t(), wide.transpose(0, 1)), (data[::2], wide[::2, :, 16:]), (data[3], wide[3]),
                         (data, wide[:1, :1].expand(7, 65, 48))):
        check_grad(binding, tokens, grad, 50)


def test_masked_rows_of_infinities_do_not_leak(binding):
    """The gradient of a padding token is not read into any sum, whatever it holds; an infinity reaches its own row alone."""
    n, vocab, dim = 2_000, 40, 32
    tokens = words((n,), vocab, 1)
    grad = torch.randn((n, dim), device=DEV, generator=gen(1))
    grad[tokens == 6] = float("nan")
    check_grad(binding, tokens, grad, vocab, pad=6)
    grad = torch.randn((n, dim), device=DEV, generator=gen(1))
    at = int((tokens == 9).nonzero()[0])
    grad[at, 5], grad[at, 6] = float("inf"), torch.finfo(torch.float32).min
    h = binding.Embedding(vocab, dim, max_tokens=n)
    out = h.grad_dense(tokens, grad, torch.empty((vocab, dim), device=DEV))
    assert bool(torch.isinf(out[9, 5]))
    out[9, 5] = 0
    assert bool(torch.isfinite(out).all())


def test_gradient_against_differences(binding):
    """sum(lookup(E) R) is linear in E: its difference quotient along any direction is <dE, direction>."""
    vocab, dim, n, scale = 60, 33, 500, 4.0
    g = gen(5)
    table = torch.randn((vocab, dim), device=DEV, generator=g)
    way = torch.randn((vocab, dim), device=DEV, generator=g)
    R = torch.randn((n, dim), device=DEV, generator=g)
    tokens = words((n,), vocab, 3)
    h = binding.Embedding(vocab, dim, max_tokens=n)
    dE = h.grad_dense(tokens, R, torch.empty((vocab, dim), device=DEV), scale=scale)
    step = 0.5
    up, down = (h.lookup(table + s * step * way, tokens, scale=scale).double() for s in (1, -1))
    quotient = ((up - down) * R.double()).sum() / (2 * step)
    exact = (dE.double() * way.double()).sum()
    # every looked-up entry is rounded three times (the moved table, the product; twice over), the sums as above
    size = (h.lookup(table.abs() + step * way.abs(), tokens, scale=scale).double() * R.double().abs()).sum()
    assert abs(float(quotient - exact)) <= float(4 * U * size / step + n * U * (plain(tokens, R, vocab, 1, scale, None)[1] * way.double().abs()).sum())


def test_update_is_what_the_server_applies(binding):
    """Lookup gradient -> update -> server, next to the oracle's server on the same pairs."""
    vocab, dim, workers, n, offset = 500, 48, 3, 400, 777
    P = offset + vocab * dim + 55
    theta = torch.randn(P, device=DEV, generator=gen(1))
    ref = oracle.Server(theta.cpu().numpy())
    srv = binding.Server(theta, history_pairs=10 * workers * n * dim, max_window_updates=16)
    srv.set_validation(True)
    h = binding.Embedding(vocab, dim, max_tokens=workers * n, max_workers=workers, padding_idx=0)
    for step in range(2):
        tokens = words((workers, n), vocab, step)
        grad = torch.randn((workers, n, dim), device=DEV, generator=gen(step))
        idx, val, begin = h.grad_update(tokens, grad, workers=workers, offset=offset)
        b = np.array(begin.tolist(), dtype=np.uint64) * np.uint64(dim)
        pulls = np.full(workers, step, dtype=np.uint64)
        srv.apply(idx.view(-1), val.view(-1), b[:-1], np.diff(b).astype(np.uint32), pulls, 0.1)
        h_idx, h_val = idx.cpu().numpy().view(np.uint32).reshape(-1), val.cpu().numpy().reshape(-1)
        for w in range(workers):
            lo, hi = int(b[w]), int(b[w + 1])
            ref.apply(h_idx[lo:hi], h_val[lo:hi], step, 0.1)
    assert srv.last_error() == 0 and h.last_error() == 0
    assert np.array_equal(theta.cpu().numpy().view(np.uint32), ref.theta().view(np.uint32))


def test_large_batch_with_frequent_tokens(binding):
    n, vocab, dim = 200_000, 32_000, 256
    tokens = words((n,), vocab, 1)
    tokens[torch.rand(n, device=DEV, generator=gen(2)) < 0.3] = 11          # one token is a third of the batch
    grad = torch.randn((n, dim), device=DEV, generator=gen(1)).bfloat16()
    check_grad(binding, tokens, grad, vocab, scale=0.125)


@pytest.mark.parametrize("n,vocab,workers", [(131_072, 50_000, 1), (131_073, 400, 1), (300_001, 100_000, 3), (1_048_577, 9_000, 1), (2_500_000, 70_000, 2)])
def test_sorts_of_every_size(binding, n, vocab, workers):
    """One cluster's most tokens and one more, many blocks, several steps per block; frequent tokens of several levels of pieces."""
    tokens = words((workers, n // workers), vocab, n)
    tokens[torch.rand(tokens.shape, device=DEV, generator=gen(2)) < 0.2] = 17
    grad = torch.randn((*tokens.shape, 4), device=DEV, generator=gen(1))
    check_grad(binding, tokens, grad, vocab, workers=workers, pad=3)


def whole_numbers(shape, seed, dtype=torch.float32):
    """Gradients of -4 .. 4: every partial sum of fewer than 2^22 of them is exact in fp32, in any order."""
    return torch.randint(-4, 5, shape, device=DEV, generator=gen(seed), dtype=torch.int8).to(dtype)


def whole_sums(tokens, grad, vocab):
    return torch.zeros((vocab, grad.shape[-1]), device=DEV, dtype=torch.float64).index_add_(0, tokens, grad.double()).float()


@pytest.mark.parametrize("kind,dim,n", [(torch.bfloat16, 8, 2 ** 23 + 77), (torch.bfloat16, 8, 2 ** 24 + 5), (torch.bfloat16, 16, 2 ** 23 + 1),
                                        (torch.float32, 4, 2 ** 24 + 3), (torch.float16, 3, 25_000_001)])
def test_dense_tables_of_narrow_rows_and_many_tokens(binding, kind, dim, n):
    """Long chunks and few threads along a row: the smallest blocks that sum and clear.  Half of the rows have no token, some
    of them in long stretches; sums are exact, so they have to be equal."""
    vocab = 600_000
    row = torch.randperm(vocab // 2, device=DEV, generator=gen(dim)) * 2 % (vocab - vocab // 5)         # even rows of the first four fifths
    tokens = row[words((n,), len(row), n)]
    grad = whole_numbers((n, dim), n, kind)
    h = binding.Embedding(vocab, dim, max_tokens=n)
    out = torch.full((vocab, dim), 7.0, device=DEV)
    h.grad_dense(tokens, grad, out)
    want = whole_sums(tokens, grad, vocab)
    assert torch.equal(out, want)
    h.grad_dense(tokens, grad, out, accumulate=True)
    assert torch.equal(out, 2 * want)
    rows, values, begin = h.grad_rows(tokens, grad)
    present = torch.bincount(tokens, minlength=vocab).nonzero().view(-1)
    assert begin.tolist() == [0, len(present)] and torch.equal(rows[:len(present)].long(), present)
    assert torch.equal(values[:len(present)], want[present])
    assert h.last_error() == 0


@pytest.mark.parametrize("n", [66_000, 150_000, 400_001])
def test_a_large_sort_that_gives_up(binding, n):
    """Blocks that look for each other once only give up (none waits for anything); until the error is read, nothing is sorted or
    written any more, however many blocks a call has; afterwards the handle goes on."""
    vocab, dim, most = 3_000, 8, 500_000
    h = binding.Embedding(vocab, dim, max_tokens=most)
    rows_out = torch.full((most,), -5, dtype=torch.int32, device=DEV)
    values_out = torch.full((most, dim), 7.0, device=DEV)
    h.set_wait_limit(0)
    for m in (n, 90_001, n, 300_007):
        h.grad_rows(words((m,), vocab, m), whole_numbers((m, dim), m), rows_out=rows_out, values_out=values_out)
        h.set_wait_limit(1 << 22)                                           # the later calls would wait, if they still met
        assert bool((rows_out == -5).all()) and bool((values_out == 7).all())
    assert h.last_error() == binding.ERR_TIMEOUT and h.last_error() == 0
    check_grad(binding, words((n,), vocab, n), whole_numbers((n, dim), n), vocab, handle=h)
    check_grad(binding, words((most,), vocab, 1), whole_numbers((most, dim), 1), vocab, handle=h)


@pytest.mark.parametrize("workers", [1, 5])
def test_calls_after_a_sort_that_gave_up(binding, workers):
    """Calls that sort in a cluster or in many blocks come out empty until the error is read; those of few tokens, which sort for
    themselves, are complete."""
    vocab, dim, most = 2_000, 8, 100_000
    h = binding.Embedding(vocab, dim, max_tokens=most, max_workers=workers)

    def batch(n):
        return words((workers, n // workers), vocab, n), whole_numbers((workers, n // workers, dim), n)

    h.set_wait_limit(0)
    for n in (most, 20_000, most):
        assert h.grad_rows(*batch(n), workers=workers)[2].tolist() == [0] * (workers + 1)
        assert h.grad_update(*batch(n), workers=workers)[2].tolist() == [0] * (workers + 1)
        table = torch.full((workers, vocab, dim), 7.0, device=DEV)
        h.grad_dense(*batch(n), table, workers=workers, accumulate=True)
        assert bool((table == 7).all())
        h.grad_dense(*batch(n), table, workers=workers)
        assert bool(((table == 7) | (table == 0)).all())
        tokens, grad = batch(500)
        key = tokens + torch.arange(workers, device=DEV).view(-1, 1) * vocab
        assert torch.equal(h.grad_dense(tokens, grad, table, workers=workers).view(-1, dim), whole_sums(key.view(-1), grad.view(-1, dim), workers * vocab))
    assert h.last_error() == binding.ERR_TIMEOUT and h.last_error() == 0
    h.set_wait_limit(1 << 22)
    for n in (500, 20_000, most):
        check_grad(binding, *batch(n), vocab, workers=workers, handle=h)


def check_whole(binding, tokens, grad, vocab, workers=1, pad=None, table=None, out_type=torch.float32):
    """Whole numbers: all three forms have to equal the sums, however long a segment is."""
    n, D = tokens.numel(), grad.shape[-1]
    h = binding.Embedding(vocab, D, max_tokens=n, max_workers=workers, padding_idx=pad)
    flat = tokens.reshape(workers, -1)
    key = (flat + torch.arange(workers, device=DEV).view(-1, 1) * vocab)[flat != -1 if pad is None else flat != pad]
    rows = grad.reshape(-1, D)[(flat != -1 if pad is None else flat != pad).view(-1)]
    want = torch.zeros((workers * vocab, D), device=DEV, dtype=torch.float64).index_add_(0, key, rows.double()).float()
    present = torch.bincount(key, minlength=workers * vocab).nonzero().view(-1)
    assert float(want.abs().max()) < 2 ** 24
    got, values, begin = h.grad_rows(tokens, grad, workers=workers)
    assert begin.tolist() == [int((present < w * vocab).sum()) for w in range(workers + 1)]
    assert torch.equal(got[:len(present)].long(), present % vocab) and torch.equal(values[:len(present)], want[present])
    idx, values, begin = h.grad_update(tokens, grad, workers=workers)
    assert torch.equal(idx[:len(present)].long(), (present % vocab).view(-1, 1) * D + torch.arange(D, device=DEV))
    assert torch.equal(values[:len(present)], want[present])
    if table is None:
        table = torch.full((workers, vocab, D), 7.0, device=DEV, dtype=out_type)
    h.grad_dense(tokens, grad, table, workers=workers)
    assert torch.equal(table, want.view(workers, vocab, D).to(table.dtype))
    h.grad_dense(tokens, grad, table, workers=workers, accumulate=True)
    assert torch.equal(table, (want + want.to(table.dtype).float()).view(workers, vocab, D).to(table.dtype))
    assert h.last_error() == 0


@pytest.mark.parametrize("n", [1, 9, 64, 500, 1_024, 1_025, 2_048, 2_049, 9_000, 65_536, 65_537, 131_073, 1_048_577, 3_000_001])
@pytest.mark.parametrize("spread", ["one", "two runs", "a third", "runs of all lengths"])
def test_sums_of_segments_of_any_length(binding, n, spread):
    """Segments from one token to all of them: every level at which their pieces are joined, in every route, next to short ones."""
    vocab, dim = 5_000, 4 if n > 100_000 else 24
    i = torch.arange(n, device=DEV)
    if spread == "one":
        tokens = i * 0 + 4_321
    elif spread == "two runs":
        tokens = torch.where(i % 7 < 4, 17, 4_999)
    elif spread == "a third":
        tokens = torch.where(torch.rand(n, device=DEV, generator=gen(n)) < 0.33, 2_000, words((n,), vocab, n))
    else:
        tokens = (torch.log2(1.0 + i.double()) * 40).long() % vocab            # each run longer than the one before
        tokens = tokens[torch.randperm(n, device=DEV, generator=gen(n))]
    check_whole(binding, tokens, whole_numbers((n, dim), n), vocab)


@pytest.mark.parametrize("kind,dim", [(torch.bfloat16, 8), (torch.bfloat16, 1000), (torch.float16, 1001), (torch.float32, 130), (torch.float32, 5000)])
@pytest.mark.parametrize("n", [700, 30_000])
def test_sums_of_long_segments_and_widths(binding, kind, dim, n):
    vocab = 700
    tokens = torch.where(torch.rand(n, device=DEV, generator=gen(n)) < 0.4, 333, words((n,), vocab, n))
    check_whole(binding, tokens, whole_numbers((n, dim), n, kind), vocab, pad=5)


@pytest.mark.parametrize("n,workers", [(32_768, 1), (32_769, 1), (65_536, 1), (65_537, 1), (16_384, 4), (21_846, 3), (8_192, 8)])
def test_sorts_at_the_limit_of_a_cluster(binding, n, workers):
    """As many tokens as one cluster of sixteen blocks takes, and one or two more; 32768 is the limit of one of eight."""
    tokens = words((workers, n), 30_011, n)
    check_whole(binding, tokens, whole_numbers((workers, n, 8), n, torch.bfloat16), 30_011, workers=workers, pad=1)


@pytest.mark.parametrize("n,vocab,dim,kind,workers", [(3_000, 200_000, 256, torch.float32, 1), (70_000, 300_001, 256, torch.float32, 1),
                                                      (5_000, 90_001, 1_000, torch.bfloat16, 2), (2_500, 60_001, 1_001, torch.float32, 1),
                                                      (12_345, 1_500_000, 65, torch.float16, 1)])
def test_dense_tables_that_are_cleared_during_the_sort(binding, n, vocab, dim, kind, workers):
    """Tables of some 200 MB and more with few tokens: rows cleared next to the sort and next to the sums; in buffers with gaps."""
    row_bytes = dim * torch.empty(0, dtype=kind).element_size()
    assert workers * n <= workers * vocab // 4 and (16 + workers * n // 8192) * (5 << 20) // row_bytes < workers * vocab // 2
    tokens = words((workers, n), vocab, n, skew=False)
    tokens[:, 0], tokens[:, 1] = 0, vocab - 1
    tokens[:, 5:n // 2] = words((workers, n // 2 - 5), 97, n)
    buf = torch.full((workers, vocab * dim + 24), 7.0, device=DEV, dtype=kind)
    table = buf[:, 8:8 + vocab * dim].view(workers, vocab, dim)
    check_whole(binding, tokens, whole_numbers((workers, n, dim), n, torch.bfloat16), vocab, workers=workers, table=table)
    assert bool((buf[:, :8] == 7).all()) and bool((buf[:, 8 + vocab * dim:] == 7).all())


def test_vocabularies_of_many_bits(binding):
    for vocab, workers in ((2 ** 31 - 1, 2), (2 ** 32 - 2, 1), (2 ** 20, 4095)):
        h = binding.Embedding(vocab, 2, max_tokens=workers * 300, max_workers=workers)
        tokens = torch.randint(vocab, (workers, 300), device=DEV, generator=gen(1))
        tokens[:, ::4] = tokens[:, :1]
        tokens[-1, 7] = vocab - 1
        grad = torch.randn((workers, 300, 2), device=DEV, generator=gen(1))
        rows, values, begin = h.grad_rows(tokens, grad, workers=workers)
        keys, inverse = torch.unique(tokens + torch.arange(workers, device=DEV).view(-1, 1) * vocab, return_inverse=True)
        assert int(begin[-1]) == len(keys)
        assert torch.equal(rows[:len(keys)].long() & 0xFFFFFFFF, keys % vocab)
        want = torch.zeros((len(keys), 2), dtype=torch.float64, device=DEV).index_add_(0, inverse.view(-1), grad.view(-1, 2).double())
        assert float((values[:len(keys)] - want).abs().max()) <= 76 * U * 76 * 6


def test_another_stream(binding):
    side = torch.cuda.Stream()
    n, vocab, dim = 5_000, 900, 128
    tokens, grad = words((n,), vocab, 1), torch.randn((n, dim), device=DEV, generator=gen(1))
    h = binding.Embedding(vocab, dim, max_tokens=n)
    side.wait_stream(torch.cuda.current_stream())
    got = [h.grad_rows(tokens, grad, stream=side) for _ in range(3)]
    looked = h.lookup(grad[:vocab], tokens, stream=side)
    assert h.last_error(stream=side) == 0
    rows, values, begin = h.grad_rows(tokens, grad)
    U_ = int(begin[1])
    for r, v, b in got:
        assert torch.equal(r[:U_], rows[:U_]) and torch.equal(v[:U_], values[:U_]) and torch.equal(b, begin)
    assert torch.equal(looked, grad[tokens])


@pytest.mark.parametrize("n", [500, 20_000, 150_000])
def test_calls_in_a_captured_graph(binding, n):
    """One launch, a cluster, a cooperative launch; with clipping behind them.  Replays see the inputs of the time."""
    vocab, dim = 3_000, 32
    tokens, grad = words((n,), vocab, 1), torch.randn((n, dim), device=DEV, generator=gen(1))
    h, clipper = binding.Embedding(vocab, dim, max_tokens=n), binding.Clipper()
    out, clipped = torch.empty((vocab, dim), device=DEV), torch.empty((1, vocab * dim), device=DEV)

    def call():
        h.grad_dense(tokens, grad, out)
        return clipper.clip(out.view(1, -1), 1.0, out=clipped)[1]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = call()
    for seed in (2, 3):
        tokens.copy_(words((n,), vocab, seed))
        grad.copy_(torch.randn((n, dim), device=DEV, generator=gen(seed)))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, clipped, norm)]
        want_norm = call()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, clipped, want_norm)))
    assert h.last_error() == 0


def test_gradients_in_another_order_than_their_tokens(binding):
    """[tokens, workers, dim] next to [workers, tokens] has as many rows, but they are other tokens' rows."""
    tokens = words((3, 50), 20, 1)
    grad = torch.randn((3, 50, 8), device=DEV, generator=gen(1))
    h = binding.Embedding(20, 8, max_tokens=150, max_workers=3)
    table = torch.empty((3, 20, 8), device=DEV)
    for call in (lambda t, g: h.grad_rows(t, g, workers=3), lambda t, g: h.grad_update(t, g, workers=3),
                 lambda t, g: h.grad_dense(t, g, table, workers=3)):
        for g in (grad.transpose(0, 1), grad.transpose(0, 1).contiguous(), grad.reshape(5, 30, 8)):
            with pytest.raises(ValueError):
                call(tokens, g)
    want = h.grad_dense(tokens, grad, torch.empty_like(table), workers=3)
    for t, g in ((tokens, grad.view(150, 8)), (tokens.view(150), grad), (tokens.view(3, 1, 50), grad), (tokens, grad.view(1, 3, 50, 8))):
        assert torch.equal(h.grad_dense(t, g, table, workers=3), want)      # the same order, in other shapes


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_negative_tokens_of_the_largest_vocabulary(binding, dtype):
    """More than 2^31 words: a negative 32-bit number is no word of them."""
    vocab = 2 ** 32 - 2
    h = binding.Embedding(vocab, 2, max_tokens=6)
    tokens = torch.tensor([-5, 3, -1, 2 ** 31 - 1, -2 ** 31, 3], device=DEV).to(dtype)
    table = torch.tensor([[1.5, -2.5]], device=DEV).expand(vocab, 2)        # one row for all words
    got = h.lookup(table, tokens)
    assert torch.equal(got, torch.where((tokens >= 0).view(-1, 1), table[:6], 0.0))
    assert h.last_error() == binding.ERR_INVALID
    rows, values, begin = h.grad_rows(tokens, torch.arange(12.0, device=DEV).view(6, 2))
    assert begin.tolist() == [0, 2] and rows[:2].tolist() == [3, 2 ** 31 - 1]
    assert values[:2].tolist() == [[2 + 10, 3 + 11], [6, 7]]
    assert h.last_error() == binding.ERR_INVALID and h.last_error() == 0


def test_misaligned_lists_are_refused(binding):
    lib = binding.raw()
    h = binding.Embedding(20, 16, max_tokens=100)
    tokens, grad = torch.zeros(50, dtype=torch.int64, device=DEV), torch.zeros((50, 16), device=DEV)
    k, g = binding.Rows(tokens.data_ptr(), 1, 0, 1, 0), binding.Rows(grad.data_ptr(), 0, 0, 16, 0)
    at = torch.zeros(4096, dtype=torch.uint8, device=DEV).data_ptr()

    def call(rows=None, begin=at, values=grad.data_ptr(), idx=None):
        return lib.adacomp_embed_grad_rows(h._h, ctypes.byref(k), 50, 1, ctypes.byref(g), 1.0, rows, begin, values, 0, idx, 0, None)

    for bad in (dict(rows=at + 2), dict(begin=at + 4), dict(values=at + 1), dict(idx=at + 2)):
        assert call(**bad) == binding.ERR_INVALID, bad


def test_refusals(binding):
    lib = binding.raw()
    vocab, dim = 20, 16
    h = binding.Embedding(vocab, dim, max_tokens=100, max_workers=2)
    tokens = torch.zeros(50, dtype=torch.int64, device=DEV)
    grad, table = torch.zeros((50, dim), device=DEV), torch.zeros((vocab, dim), device=DEV)
    out, begin = torch.zeros((50, dim), device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV)

    def rows(t, kind, **fields):
        r = binding.Rows()
        r.d_data, r.type, r.row_stride = t.data_ptr(), kind, dim if t.dim() > 1 else 1
        for k, v in fields.items():
            setattr(r, k, v)
        return ctypes.byref(r)

    def lookup(t={}, k={}, o={}, n=50, scale=1.0):
        return lib.adacomp_embed_lookup(h._h, rows(table, 0, **t), rows(tokens, 1, **k), n, scale, rows(out, 0, **o), None)

    def sums(k={}, g={}, n=50, workers=1, scale=1.0, b=begin.data_ptr(), v=out.data_ptr(), kind=0, idx=None, offset=0):
        return lib.adacomp_embed_grad_rows(h._h, rows(tokens, 1, **k), n, workers, rows(grad, 0, **g), scale, None, b, v, kind, idx, offset, None)

    def dense(k={}, g={}, o={}, n=50, workers=1):
        return lib.adacomp_embed_grad_dense(h._h, rows(tokens, 1, **k), n, workers, rows(grad, 0, **g), 1.0, rows(table, 0, **o), 0, None)

    inf = float("inf")
    for bad in (dict(t=dict(type=3)), dict(k=dict(type=2)), dict(o=dict(type=-1)), dict(t=dict(d_data=None)), dict(k=dict(d_data=None)),
                dict(o=dict(d_data=None)), dict(t=dict(d_data=table.data_ptr() + 2)), dict(k=dict(d_data=tokens.data_ptr() + 4)),
                dict(o=dict(row_stride=dim - 1)), dict(o=dict(group=5, group_stride=0)), dict(t=dict(group=4, group_stride=7)),
                dict(scale=inf), dict(scale=float("nan")), dict(n=2 ** 31)):
        assert lookup(**bad) == binding.ERR_INVALID, bad
    for bad in (dict(k=dict(type=5)), dict(g=dict(type=7)), dict(workers=0), dict(workers=3), dict(scale=inf), dict(b=None), dict(v=None),
                dict(v=out.data_ptr() + 2), dict(kind=9), dict(idx=out.data_ptr(), offset=2 ** 32 - 100), dict(g=dict(d_data=None))):
        assert sums(**bad) == binding.ERR_INVALID, bad
    assert sums(n=101) == binding.ERR_CAPACITY and sums(n=51, workers=2) == binding.ERR_CAPACITY
    for bad in (dict(o=dict(type=4)), dict(o=dict(row_stride=3)), dict(o=dict(d_data=None))):
        assert dense(**bad) == binding.ERR_INVALID, bad
    assert lookup() == 0 and sums() == 0 and dense() == 0 and h.last_error() == 0
    for bad in (lambda: h.lookup(table[:5], tokens), lambda: h.lookup(table, tokens.float()), lambda: h.lookup(table.double(), tokens),
                lambda: h.lookup(table, tokens.cpu()), lambda: h.lookup(table.cpu(), tokens), lambda: h.lookup(table[:, :4], tokens),
                lambda: h.lookup(table, tokens, out=out[:9]), lambda: h.lookup(table.t().contiguous().t(), tokens),
                lambda: h.grad_rows(tokens, grad, workers=3), lambda: h.grad_rows(tokens, grad[:9]), lambda: h.grad_rows(tokens, grad, values_out=out[:9]),
                lambda: h.grad_update(tokens, grad, val_out=out.half()), lambda: h.grad_dense(tokens, grad, table[:7]),
                lambda: h.grad_dense(tokens[:vocab], table, table), lambda: binding.Embedding(5, 5, padding_idx=5)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad in (lambda: binding.Embedding(0, 5), lambda: binding.Embedding(5, -1), lambda: binding.Embedding(2 ** 31, 5, max_workers=2)):
        with pytest.raises(binding.AdacompError):
            bad()
