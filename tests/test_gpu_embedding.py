"""luq_embedding_fwd and luq_embedding_grad against plain forms, through the C ABI."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import announce, host, to_dev  # noqa: E402
import lm_util as U  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2112_10769_amd as lib
    return lib


def _tensor(shape, dtype, seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=gen) * scale).to(dtype)


@pytest.mark.parametrize("dim", [1, 2, 7, 8, 33, 64, 510, 1001, 1024, 4099])
@pytest.mark.parametrize("tt,ot", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
def test_lookup(L, dim, tt, ot):
    """Bit for bit the fp32 product, rounded once more to a bf16 output; padding and ids off the table."""
    vocab = 301
    rng = np.random.default_rng(dim)
    table = _tensor((vocab, dim), DT[tt], dim)
    ids = rng.integers(0, vocab, (5, 23))
    ids[0, 3], ids[1, 1], ids[2, 0], ids[4, 22] = -1, -2 ** 40, vocab, 2 ** 40
    announce("embedding_fwd", dim, tt, ot)
    got = L.luq_embedding_fwd(to_dev(ids), table, 1.7, DT[ot])
    assert got.shape == (5, 23, dim) and got.dtype == DT[ot]
    i = torch.from_numpy(ids).cuda()
    ref = table.float()[i.clamp(0, vocab - 1)] * np.float32(1.7).item()
    ref = torch.where((i < 0)[..., None], torch.zeros_like(ref), ref)
    ref = torch.where((i >= vocab)[..., None], torch.full_like(ref, float("nan")), ref).to(DT[ot])
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    assert torch.equal(got.nan_to_num(7.0), ref.nan_to_num(7.0))


@pytest.mark.parametrize("offset", [0, 1, 2, 3, 5])
def test_lookup_unaligned(L, offset):
    """Tables, ids and outputs that begin anywhere inside a 16-byte piece; strided ids."""
    vocab, dim, n = 40, 24, 17
    flat = _tensor((vocab * dim + 8,), torch.bfloat16, 3)
    table = flat[offset:offset + vocab * dim].view(vocab, dim)
    out = torch.zeros(n * dim + 8, dtype=torch.bfloat16, device="cuda")
    ids = torch.randint(0, vocab, (2 * n,), device="cuda", dtype=torch.int32)[::2]
    announce("embedding_fwd unaligned", offset)
    L.luq_embedding_fwd(ids, table, 2.0, out=out[8 - offset:8 - offset + n * dim].view(n, dim))
    assert torch.equal(out[8 - offset:8 - offset + n * dim].view(n, dim), (table.float()[ids.long()] * 2).bfloat16())
    assert not out[:8 - offset].any() and not out[8 - offset + n * dim:].any()


def test_lookup_values(L):
    """Infinities and NaN of a looked-up row pass through and stay in it; no ids, no table."""
    table = _tensor((4, 16), torch.float32, 1)
    table[1, 3], table[2] = float("inf"), float("nan")
    announce("embedding_fwd values")
    got = host(L.luq_embedding_fwd(to_dev(np.array([0, 1, 2, 3])), table, -1.0))
    assert np.array_equal(got, -host(table), equal_nan=True)
    assert L.luq_embedding_fwd(torch.empty(0, dtype=torch.int64, device="cuda"), table).shape == (0, 16)
    none = L.luq_embedding_fwd(to_dev(np.array([0, -1])), torch.empty(0, 5, device="cuda"))
    assert np.isnan(host(none)[0]).all() and (host(none)[1] == 0).all()


def test_lookup_beyond_32_bits(L):
    """Rows of the table and of the output past 2^31 elements."""
    vocab, dim = 1100000, 2050
    table = torch.zeros(vocab, dim, dtype=torch.bfloat16, device="cuda")
    table[-1], table[-2] = 3.0, 5.0
    n = 1100001
    ids = torch.full((n,), vocab - 1, dtype=torch.int32, device="cuda")
    ids[-1] = vocab - 2
    announce("embedding_fwd 64-bit offsets")
    out = L.luq_embedding_fwd(ids, table, 2.0)
    assert (out[-1] == 10).all() and (out[-2] == 6).all() and (out[0] == 6).all()
    del table, out
    torch.cuda.empty_cache()


def _grad(L, ids, vocab, dout, scale, **kw):
    i = to_dev(ids)
    order, offsets = L.luq_group_ids(i, vocab)
    return L.luq_embedding_grad(dout, i, order, offsets, scale, **kw)


def _ids(kind, n, vocab, rng):
    if kind == "zipf":
        return np.floor((vocab + 1.0) ** rng.random(n)).astype(np.int64) - 1
    if kind == "one":
        return np.full(n, vocab // 2, dtype=np.int64)
    if kind == "none":
        return np.full(n, -1, dtype=np.int64)
    if kind == "padded":
        ids = rng.integers(0, vocab, n)
        ids[rng.random(n) < 0.4] = -1
        ids[rng.random(n) < 0.1] = vocab
        return ids
    return rng.permutation(max(n, vocab))[:n] % vocab   # each once while there are enough


@pytest.mark.parametrize("kind", ["zipf", "one", "none", "padded", "each"])
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 300, 64), (64, 7, 33), (500, 8000, 510), (3001, 97, 24),
                                         (2049, 4000, 257), (777, 130, 1001), (257, 50, 4099)])
@pytest.mark.parametrize("gt", ["f32", "bf16"])
def test_gradient(L, kind, n, vocab, dim, gt):
    rng = np.random.default_rng(n + dim)
    ids = _ids(kind, n, vocab, rng)
    dout = _tensor((n, dim), DT[gt], n)
    announce("embedding_grad", kind, n, vocab, dim, gt)
    got = _grad(L, ids, vocab, dout, 1.5)
    ref, bound = U.embedding_grad(host(dout.float()), ids, vocab, 1.5)
    U.within(host(got), ref, bound, (kind, n, vocab, dim, gt))
    again = _grad(L, ids, vocab, dout, 1.5)
    assert torch.equal(got, again), "the order of the sums is fixed"


@pytest.mark.parametrize("n,dim", [(4096, 64), (40000, 8), (40000, 130), (9000, 1024)])
def test_frequent_ids(L, n, dim):
    """Sums of thousands of rows next to sums of one, over every length of a piece."""
    vocab = 60
    rng = np.random.default_rng(n)
    ids = np.concatenate([np.full(n - n // 8, 3), rng.integers(0, vocab, n // 8)])
    rng.shuffle(ids)
    dout = _tensor((n, dim), torch.float32, n)
    announce("embedding_grad frequent", n, dim)
    got = _grad(L, ids, vocab, dout, 0.25)
    ref, bound = U.embedding_grad(host(dout), ids, vocab, 0.25)
    U.within(host(got), ref, bound, (n, dim))


@pytest.mark.parametrize("dim", [5, 64, 1023])
def test_accumulate(L, dim):
    """accumulate adds to the rows that ids name and leaves every other row's bits alone."""
    n, vocab = 700, 900
    rng = np.random.default_rng(dim)
    ids = _ids("padded", n, vocab, rng)
    dout, start = _tensor((n, dim), torch.bfloat16, 4), _tensor((vocab, dim), torch.float32, 5)
    start[::7] = float("nan")
    named = np.zeros(vocab, dtype=bool)
    named[ids[(ids >= 0) & (ids < vocab)]] = True
    start[torch.from_numpy(np.nonzero(named)[0]).cuda()] = 0.5
    before = host(start.clone())
    announce("embedding_grad accumulate", dim)
    got = host(_grad(L, ids, vocab, dout, 2.0, accumulate=True, dtable=start))
    ref, bound = U.embedding_grad(host(dout.float()), ids, vocab, 2.0)
    assert np.array_equal(got[~named], before[~named], equal_nan=True)
    U.within(got[named], ref[named] + 0.5, bound[named] + U.U * (np.abs(ref[named]) + 0.5 + bound[named]), dim)


@pytest.mark.parametrize("dim", [1, 3, 70, 600])
def test_gradient_of_no_ids(L, dim):
    """Zeros are written, or with accumulate nothing is."""
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    announce("embedding_grad no ids", dim)
    order, offsets = L.luq_group_ids(ids, 33)
    table = torch.full((33, dim), 2.0, device="cuda")
    dout = torch.empty(0, dim, device="cuda")
    L.luq_embedding_grad(dout, ids, order, offsets, 1.0, accumulate=True, dtable=table)
    assert (table == 2).all()
    assert (L.luq_embedding_grad(dout, ids, order, offsets, 1.0, dtable=table) == 0).all()


@pytest.mark.parametrize("vocab,dim", [(381, 7136), (5, 40000), (70000, 3)])
def test_tables_of_extreme_shape(L, vocab, dim):
    n = 189
    rng = np.random.default_rng(vocab)
    ids = _ids("padded", n, vocab, rng)
    dout = _tensor((n, dim), torch.bfloat16, 6)
    announce("embedding_grad shape", vocab, dim)
    got = _grad(L, ids, vocab, dout, 1.0, dtable=torch.full((vocab, dim), float("nan"), device="cuda"))
    ref, bound = U.embedding_grad(host(dout.float()), ids, vocab, 1.0)
    U.within(host(got), ref, bound, (vocab, dim))


def test_gradient_values(L):
    """A NaN or infinity reaches its own row only, and none of a padded position does; zeros are written
    over whatever the buffer held."""
    vocab, dim = 6, 40
    ids = np.array([4, 1, -1, 4, 0, 6])
    dout = torch.ones(6, dim, device="cuda")
    dout[0, 3], dout[1], dout[2], dout[5] = float("inf"), float("nan"), float("nan"), float("nan")
    announce("embedding_grad values")
    got = host(_grad(L, ids, vocab, dout, 1.0, dtable=torch.full((vocab, dim), float("nan"), device="cuda")))
    assert np.isnan(got[1]).all() and np.isinf(got[4, 3]) and (np.delete(got[4], 3) == 2).all()
    assert (got[0] == 1).all() and (got[[2, 3, 5]] == 0).all()


@pytest.mark.parametrize("offset", [1, 2, 3])
def test_gradient_unaligned(L, offset):
    vocab, dim, n = 30, 48, 90
    rng = np.random.default_rng(offset)
    ids = rng.integers(0, vocab, n)
    flat = _tensor((n * dim + 8,), torch.bfloat16, 9)
    dout = flat[offset:offset + n * dim].view(n, dim)
    out = torch.full((vocab * dim + 8,), 7.0, device="cuda")
    dtable = out[offset:offset + vocab * dim].view(vocab, dim)
    announce("embedding_grad unaligned", offset)
    _grad(L, ids, vocab, dout, 1.0, dtable=dtable)
    ref, bound = U.embedding_grad(host(dout.float()), ids, vocab, 1.0)
    U.within(host(dtable), ref, bound, offset)
    assert (out[:offset] == 7).all() and (out[offset + vocab * dim:] == 7).all()


def test_gradient_is_the_lookups(L):
    """Against differences: <dout, lookup(table + h v) - lookup(table - h v)> / 2h = <dtable, v>."""
    vocab, dim, n = 50, 36, 400
    rng = np.random.default_rng(8)
    ids = _ids("padded", n, vocab, rng)
    ids[ids >= vocab] = 0
    table, v, dout = rng.standard_normal((vocab, dim)), rng.standard_normal((vocab, dim)), rng.standard_normal((n, dim))
    dout = dout.astype(np.float32)

    def loss(t):
        rows = 3.0 * t[np.maximum(ids, 0)] * (ids >= 0)[:, None]
        return float((rows * dout).sum())
    h = 2.0 ** -10
    announce("embedding_grad differences")
    got = host(_grad(L, ids, vocab, to_dev(dout), 3.0)).astype(np.float64)
    slope = (loss(table + h * v) - loss(table - h * v)) / (2 * h)
    _, bound = U.embedding_grad(dout, ids, vocab, 3.0)
    # the loss is linear: the difference is exact but for 64-bit rounding
    assert abs((got * v).sum() - slope) <= (bound * np.abs(v)).sum() + 1e-9 * abs(slope) + 1e-6


def test_gradient_beyond_32_bits(L):
    n, dim, vocab = 1100001, 2050, 3
    dout = torch.zeros(n, dim, dtype=torch.bfloat16, device="cuda")
    dout[-1], dout[0] = 4.0, 1.0
    ids = np.zeros(n, dtype=np.int32)
    ids[-1] = 2
    announce("embedding_grad 64-bit offsets")
    got = host(_grad(L, ids, vocab, dout, 1.0))
    assert (got[2] == 4).all() and (got[0] == 1).all() and (got[1] == 0).all()
    del dout
    torch.cuda.empty_cache()
