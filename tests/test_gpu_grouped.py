"""The products grouped by expert against exact integer sums, through the C ABI.

Outputs must equal the fp32 epilogue of the exact sums bit for bit, as those of the
ungrouped products: fl32(fl32(acc) * scale) with the scales' product rounded in the
library's order; rows of no expert and experts without rows are zeros.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import announce, epilogue_replica, host, to_dev  # noqa: E402
import lm_util as U  # noqa: E402


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2112_10769_amd as lib
    return lib


def _offsets(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)


def _dev(v):
    return to_dev(np.asarray(v, dtype=np.float32).reshape(-1))


def _product(a, b):
    """Exact integer product a [m][k] b [n][k]^T (float64 holds every sum)."""
    return a.astype(np.float64) @ b.astype(np.float64).T


def _rows_case(rng, sizes, tail, N, K, kind, b_signed, scales):
    """Operands of a product of grouped rows: (codes, values of A, scale of A, weights, their scales)."""
    T, E = int(sum(sizes)) + tail, len(sizes)
    if kind == "luq":
        f = U.luq_fields(rng, (T, K))
        codes, a = U.luq_pack(f), U.luq_levels(f)
    elif kind == "sums":
        f, keep = U.luq_fields(rng, (T, K)), rng.integers(0, 2, (T, K))
        a = U.luq_levels(f) * (1 + keep)            # the second sample: 0 or the first's value
        codes = a.astype(np.int8)
    else:
        a = U.int4_values(rng, (T, K), kind == "int4s")
        codes = U.pack(a)
    w = U.int4_values(rng, (E, N, K), b_signed)
    return codes, a, np.float32(rng.uniform(0.1, 2)), w, rng.uniform(0.1, 2, E if scales else 1).astype(np.float32)


def _rows_ref(a, scale, w, w_scale, offsets, T, N, sums):
    y = np.zeros((T, N), dtype=np.float32)
    for e in range(len(offsets) - 1):
        lo, hi = offsets[e], offsets[e + 1]
        y[lo:hi] = epilogue_replica(_product(a[lo:hi], w[e]), scale, 2 if sums else 1, w_scale[e % len(w_scale)])
    return y


def _run_rows(L, kind, codes, scale, w_codes, w_scale, b_signed, offsets, T, N, K, **kw):
    x, w = to_dev(codes), to_dev(w_codes)
    out = torch.full((T, N), float("nan"), device="cuda")
    if kind in ("luq", "sums"):
        return L.luq_gemm_dgrad_grouped(x, _dev(scale), w, _dev(w_scale), b_signed, to_dev(offsets), T, N, K,
                                        L.SMP_SUM | 2 if kind == "sums" else 1, dx=out, **kw)
    return L.int4_gemm_fwd_grouped(x, _dev(scale), kind == "int4s", w, _dev(w_scale), b_signed, to_dev(offsets), T, N, K,
                                   y=out, **kw)


def _check_rows(L, sizes, tail, N, K, kind, b_signed, scales=True, seed=0):
    announce("grouped rows", kind, b_signed, sizes if len(sizes) < 12 else (len(sizes), sum(sizes)), tail, N, K)
    rng = np.random.default_rng(seed + N + K)
    codes, a, scale, w, w_scale = _rows_case(rng, sizes, tail, N, K, kind, b_signed, scales)
    offsets = _offsets(sizes)
    T = int(offsets[-1]) + tail
    got = host(_run_rows(L, kind, codes, scale, U.pack(w), w_scale, b_signed, offsets, T, N, K))
    ref = _rows_ref(a, scale, w, w_scale, offsets, T, N, kind == "sums")
    assert np.array_equal(got, ref), (kind, sizes, N, K, np.argwhere(got != ref)[:4])


KINDS = ["luq", "sums", "int4s", "int4u"]
GROUPS = [([1], 0), ([0, 1, 0], 0), ([3, 0, 5, 1], 4), ([31, 32, 33], 0), ([127, 0, 128, 129, 2], 17), ([300], 31),
          ([40, 260, 7, 513], 0)]


@pytest.mark.parametrize("sizes,tail", GROUPS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("b_signed", [True, False])
def test_rows(L, sizes, tail, kind, b_signed):
    for N, K in ((1, 32), (67, 96), (256, 1024), (130, 544)):
        _check_rows(L, sizes, tail, N, K, kind, b_signed, scales=N != 67)


# Every tile, on whole stages and on a partly filled last one (test_lm_plan_cpu.py).
LARGE_ROWS = [([256, 300, 0, 512], 512, 256), ([700, 1, 256], 333, 1184), ([2000, 100], 640, 128), ([64] * 9, 2048, 512),
              ([2] * 70, 96, 2080), ([3, 1, 0, 2], 100, 2048), ([3, 1, 0, 2], 100, 2080), ([1, 0, 2] * 20, 1024, 512),
              ([1, 0, 2] * 20, 1024, 544), ([520, 500], 1024, 512), ([520, 500], 1024, 544), ([300, 500, 200], 1500, 128),
              ([300, 500, 200], 1500, 160), ([2000, 1900, 2100], 2300, 256), ([2000, 1900, 2100], 2300, 160),
              ([1] * 64, 2048, 128), ([1] * 64, 2048, 96), ([70] * 8, 4096, 256), ([70] * 8, 4096, 288),
              ([1900, 2100], 4096, 544), ([2300, 1700], 4096, 1024), ([300, 700], 4100, 96), ([500, 500], 4096, 128),
              ([250, 0, 300, 450], 512, 1056), ([140, 160], 2048, 1024), ([130, 170], 512, 160), ([130, 170], 512, 512)]


def rows_shapes():
    """(experts, T, N, K) of the tests above and below."""
    small = [(len(sizes), sum(sizes) + tail, N, K) for sizes, tail in GROUPS
             for N, K in ((1, 32), (67, 96), (256, 1024), (130, 544))]
    return small + [(len(sizes), sum(sizes) + 3, N, K) for sizes, N, K in LARGE_ROWS]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sizes,N,K", LARGE_ROWS)
def test_rows_of_larger_tiles(L, kind, sizes, N, K):
    _check_rows(L, sizes, 3, N, K, kind, True)


@pytest.mark.parametrize("experts", [63, 64, 65, 130, 4096])
def test_many_experts(L, experts):
    """Offsets longer than a wave, most groups empty."""
    rng = np.random.default_rng(experts)
    sizes = np.zeros(experts, dtype=np.int64)
    at = rng.integers(0, experts, 40)
    sizes[at] += rng.integers(1, 9, 40)
    sizes[[0, experts - 1]] += 2
    _check_rows(L, [int(v) for v in sizes], 5, 40, 64, "luq", True)
    _check_depth(L, [int(v) for v in sizes], 40, 24, "luq", True)


@pytest.mark.parametrize("sizes,T", [([0, 0, 0], 50), ([50], 50), ([0] * 70, 3)])
def test_no_rows(L, sizes, T):
    """Only rows of no expert; and no rows at all."""
    announce("grouped no rows", sizes, T)
    rng = np.random.default_rng(0)
    tail = T - sum(sizes)
    _check_rows(L, sizes, tail, 70, 64, "int4s", True)
    codes, _, scale, w, w_scale = _rows_case(rng, [0] * len(sizes), 0, 8, 64, "int4s", True, True)
    y = L.int4_gemm_fwd_grouped(torch.empty(0, dtype=torch.uint8, device="cuda"), _dev(scale), True, to_dev(U.pack(w)),
                                _dev(w_scale), True, torch.zeros(len(sizes) + 1, dtype=torch.int32, device="cuda"), 0, 8,
                                64)
    assert y.shape == (0, 8)


@pytest.mark.parametrize("kind,limit", [("int4s", 1 << 17), ("int4u", 1 << 17), ("luq", 1 << 18), ("sums", 1 << 18)])
def test_longest_exact_rows(L, kind, limit):
    """The largest codes of either sign over the longest reduction: sums next to 2^31."""
    K, E, N, T = limit, 2, 3, 5
    announce("grouped longest", kind)
    if kind in ("luq", "sums"):
        a = np.full((T, K), 64 if kind == "sums" else 64, dtype=np.int64)
        codes = a.astype(np.int8) if kind == "sums" else U.luq_pack(np.full((T, K), 7))
    else:
        a = np.full((T, K), 7 if kind == "int4s" else 15, dtype=np.int64)
        codes = U.pack(a)
    w = np.full((E, N, K), 7, dtype=np.int64)
    w[1] = -7
    offsets = _offsets([2, 3])
    got = host(_run_rows(L, kind, codes, np.float32(1), U.pack(w), np.float32([1, 1]), True, offsets, T, N, K))
    top = int(a[0, 0]) * 7 * K
    ref = np.where(np.arange(T)[:, None] < 2, top, -top) * (0.5 if kind == "sums" else 1.0)
    assert np.array_equal(got, np.broadcast_to(ref, (T, N)).astype(np.float32))


def test_transposed_stack(L):
    """The weights' transposed codes of one int4_quantize call on [experts * Nout][Kin]: rows of every expert
    interleaved, one scale."""
    E, Nout, Kin = 3, 96, 72
    sizes = [5, 0, 41]
    announce("grouped transposed stack")
    rng = np.random.default_rng(4)
    w = rng.standard_normal((E * Nout, Kin)).astype(np.float32)
    codes, codes_t, s = L.int4_quantize(to_dev(w), True, codes=True, codes_t=True)
    q = np.rint(w * np.float32(np.float32(7) / np.abs(w).max())).astype(np.int64).reshape(E, Nout, Kin)
    f = U.luq_fields(rng, (46, Nout))
    offsets = _offsets(sizes)
    got = host(L.luq_gemm_dgrad_grouped(to_dev(U.luq_pack(f)), _dev(0.5), codes_t, s, True, to_dev(offsets), 46, Kin, Nout,
                                        w_row=E * Nout, w_expert=Nout))
    ref = _rows_ref(U.luq_levels(f), np.float32(0.5), q.transpose(0, 2, 1), host(s), offsets, 46, Kin, False)
    assert np.array_equal(got, ref)


def test_quantizer_layouts_forward(L):
    """Forward product on the same stack: Kin must be whole 16-byte pieces."""
    E, Nout, Kin = 3, 40, 96
    announce("grouped forward stack")
    rng = np.random.default_rng(5)
    w, x = rng.standard_normal((E * Nout, Kin)).astype(np.float32), rng.standard_normal((64, Kin)).astype(np.float32)
    wc, _, ws = L.int4_quantize(to_dev(w), True)
    xc, _, xs = L.int4_quantize(to_dev(x), True)
    offsets = _offsets([11, 33, 20])
    got = host(L.int4_gemm_fwd_grouped(xc, xs, True, wc, ws, True, to_dev(offsets), 64, Nout, Kin))
    for e, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        one, _, _ = L.int4_quantize(to_dev(w), True)
        part = L.int4_gemm_fwd(xc[lo * Kin // 2:].clone(), xs, True, one[e * Nout * Kin // 2:].clone(), ws, True, int(hi - lo),
                               Nout, Kin)
        assert np.array_equal(got[lo:hi], host(part))


# ---- weight gradient ---------------------------------------------------------------------


def _check_depth(L, sizes, Nout, Kin, kind, b_signed, seed=0):
    offsets = _offsets(sizes)
    E, routed = len(sizes), int(offsets[-1])
    T = max(32, -(-routed // 32) * 32)
    announce("grouped depth", kind, b_signed, sizes if E < 12 else (E, routed), Nout, Kin)
    rng = np.random.default_rng(seed + Nout + Kin)
    f = U.luq_fields(rng, (Nout, T))             # the padding holds codes too
    if kind == "sums":
        g = U.luq_levels(f) * (1 + rng.integers(0, 2, f.shape))
        codes = g.astype(np.int8)
    else:
        g, codes = U.luq_levels(f), U.luq_pack(f)
    a = U.int4_values(rng, (Kin, T), b_signed)
    alpha, scale = np.float32(rng.uniform(0.1, 2)), np.float32(rng.uniform(0.1, 2))
    out = torch.full((E, Nout, Kin), float("nan"), device="cuda")
    got = host(L.luq_gemm_wgrad_grouped(to_dev(codes), _dev(alpha), to_dev(U.pack(a)), _dev(scale), b_signed,
                                        to_dev(offsets), T, Nout, Kin, L.SMP_SUM | 2 if kind == "sums" else 1, dw=out))
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        ref = epilogue_replica(_product(g[:, lo:hi], a[:, lo:hi]), alpha, 2 if kind == "sums" else 1, scale)
        assert np.array_equal(got[e], ref), (kind, sizes, e, np.argwhere(got[e] != ref)[:4])


DEPTHS = [[1], [32], [0, 5, 0], [31, 1, 64], [7, 130, 0, 19, 64], [33, 95, 1, 127], [400, 3, 257], [1000], [128, 128, 256]]


@pytest.mark.parametrize("sizes", DEPTHS)
@pytest.mark.parametrize("kind", ["luq", "sums"])
@pytest.mark.parametrize("b_signed", [True, False])
def test_depth(L, sizes, kind, b_signed):
    for Nout, Kin in ((1, 1), (67, 33), (128, 256), (300, 130)):
        _check_depth(L, sizes, Nout, Kin, kind, b_signed)


LARGE_DEPTHS = [([600, 1, 1500], 512, 520), ([4000, 100], 64, 64), ([2048] * 3, 256, 512), ([9000], 40, 96),
                ([100] * 30, 256, 256), ([30, 2, 500, 1, 200], 2300, 2100), ([777, 900], 2048, 1024), ([1500, 333], 1000, 1030),
                ([5] * 64, 200, 200), ([130, 0, 77, 260] * 8, 300, 140), ([6000, 5000], 512, 1024),
                ([900, 1148], 2048, 2048), ([500, 400, 1, 1147], 2048, 2048), ([4096], 100, 90)]


def depth_shapes():
    """(experts, T, Nout, Kin) of the tests above and below."""
    def rows(sizes):
        return max(32, -(-sum(sizes) // 32) * 32)
    small = [(len(s), rows(s), M, N) for s in DEPTHS for M, N in ((1, 1), (67, 33), (128, 256), (300, 130))]
    return small + [(len(s), rows(s), M, N) for s, M, N in LARGE_DEPTHS]


@pytest.mark.parametrize("kind", ["luq", "sums"])
@pytest.mark.parametrize("sizes,Nout,Kin", LARGE_DEPTHS)
def test_depth_of_larger_tiles(L, kind, sizes, Nout, Kin):
    _check_depth(L, sizes, Nout, Kin, kind, True)


def test_longest_exact_depth(L):
    """The largest codes over 2^18 rows of one expert."""
    T, Nout, Kin = 1 << 18, 3, 5
    announce("grouped longest depth")
    codes = U.luq_pack(np.full((Nout, T), 7))
    a = U.pack(np.full((Kin, T), -7))
    got = host(L.luq_gemm_wgrad_grouped(to_dev(codes), _dev(1.0), to_dev(a), _dev(1.0), True, to_dev(_offsets([0, T])), T,
                                        Nout, Kin))
    assert (got[0] == 0).all() and (got[1] == np.float32(-64 * 7 * T)).all()


@pytest.mark.parametrize("kind", ["luq", "sums"])
@pytest.mark.parametrize("T", [(1 << 18) + 128, (1 << 19) + 384, 1 << 22])
def test_batches_beyond_the_exact_depth(L, T, kind):
    """Split so that no int32 sum passes its range, whichever expert has the rows: all in one, the largest codes of one
    sign throughout; and groups that begin and end at any row."""
    Nout, Kin = 3, 5
    announce("grouped beyond the exact depth", T, kind)
    # 64 either way: a code of R = 6, and the sum of two of R = 5
    codes = U.luq_pack(np.full((Nout, T), 7)) if kind == "luq" else np.full((Nout, T), 64, dtype=np.int8)
    top, samples = 64, 1 if kind == "luq" else 2
    a = U.pack(np.full((Kin, T), 15))
    cut = T // 3 + 17
    for sizes in ([0, T], [T, 0], [cut, 0, T - cut], [5, T - 6], [T // 8] * 8):
        offsets = _offsets(sizes)
        got = host(L.luq_gemm_wgrad_grouped(to_dev(codes), _dev(0.75), to_dev(a), _dev(0.5), False, to_dev(offsets), T, Nout,
                                            Kin, n_samples=1 if kind == "luq" else L.SMP_SUM | 2))
        for e, rows in enumerate(sizes):
            ref = epilogue_replica(np.full((Nout, Kin), float(top * 15 * rows)), np.float32(0.75), samples, np.float32(0.5))
            assert np.array_equal(got[e], ref), (sizes, e)


def test_batch_beyond_the_exact_depth_of_random_codes(L):
    _check_depth(L, [1, 100000, 0, 150001, 40036], 67, 33, "luq", True)
    _check_depth(L, [270000, 77], 130, 40, "sums", False)


# ---- beyond 32 bits, streams, bounds -------------------------------------------------------


def test_experts_beyond_32_bits(L):
    """An expert whose codes begin past 2^31 bytes, and outputs past 2^31 elements."""
    N, K, gap = 8, 64, (1 << 32) + 4096   # codes from one expert to the next
    announce("grouped 64-bit offsets")
    rng = np.random.default_rng(6)
    w = U.int4_values(rng, (3, N, K), True)
    buf = torch.zeros(gap + N * K // 2, dtype=torch.uint8, device="cuda")
    for e in range(3):
        buf[e * gap // 2:e * gap // 2 + N * K // 2] = to_dev(U.pack(w[e])).view(-1)
    a = U.int4_values(rng, (30, K), True)
    offsets = _offsets([10, 10, 10])
    got = host(L.int4_gemm_fwd_grouped(to_dev(U.pack(a)), _dev(1.0), True, buf, _dev([1, 2, 3]), True, to_dev(offsets), 30, N,
                                       K, w_expert=gap))
    assert np.array_equal(got, _rows_ref(a, np.float32(1), w, np.float32([1, 2, 3]), offsets, 30, N, False))
    del buf
    T, N, K = 70016, 32768, 32
    w = U.int4_values(rng, (2, N, K), True)
    a = np.zeros((T, K), dtype=np.int64)
    a[-70:] = U.int4_values(rng, (70, K), True)
    offsets = _offsets([1000, T - 1032])
    y = L.int4_gemm_fwd_grouped(to_dev(U.pack(a)), _dev(1.0), True, to_dev(U.pack(w)), _dev([1, 1]), True, to_dev(offsets),
                                T, N, K)
    ref = np.zeros((70, N))
    ref[:38] = _product(a[-70:-32], w[1])
    assert np.array_equal(host(y[-70:]), ref.astype(np.float32))
    del y
    torch.cuda.empty_cache()


def test_outputs_beyond_the_small_tiles_grids(L):
    """2^33 outputs: more 32 x 32 tiles than a grid has."""
    T, N, K = 1 << 18, 1 << 15, 32
    announce("grouped large output")
    rng = np.random.default_rng(10)
    w = U.int4_values(rng, (3, N, K), True)
    a = U.int4_values(rng, (T, K), True)
    cut = [0, 100001, 100001, T - 5]
    y = L.int4_gemm_fwd_grouped(to_dev(U.pack(a)), _dev(1.0), True, to_dev(U.pack(w)), _dev([1, 1, 1]), True,
                                to_dev(np.int32(cut)), T, N, K, y=torch.full((T, N), float("nan"), device="cuda"))
    for lo, hi, e in ((0, 40, 0), (99980, 100001, 0), (100001, 100030, 2), (T - 40, T - 5, 2), (T - 5, T, -1)):
        ref = _product(a[lo:hi], w[e]) if e >= 0 else np.zeros((hi - lo, N))
        assert np.array_equal(host(y[lo:hi]), ref.astype(np.float32)), (lo, hi)
    assert not torch.isnan(y.view(-1)[::1009]).any()
    del y
    torch.cuda.empty_cache()


def test_decreasing_offsets_stay_inside(L):
    """Offsets that are no groups give some result inside the output, and no access outside it."""
    announce("grouped decreasing offsets")
    rng = np.random.default_rng(9)
    codes, a, scale, w, w_scale = _rows_case(rng, [20] * 8, 0, 50, 64, "int4s", True, True)
    flat = torch.full((160 * 50 + 64,), 7.0, device="cuda")
    y = flat[32:32 + 160 * 50].view(160, 50)
    offsets = to_dev(np.int32([0, 160, 0, 160, -5, 160, 3, 1 << 30, 0]))
    L.int4_gemm_fwd_grouped(to_dev(codes), _dev(scale), True, to_dev(U.pack(w)), _dev(w_scale), True, offsets, 160, 50, 64, y=y)
    dw = torch.zeros(8, 6, 10, device="cuda")
    L.luq_gemm_wgrad_grouped(to_dev(U.luq_pack(U.luq_fields(rng, (6, 160)))), _dev(1.0),
                             to_dev(U.pack(U.int4_values(rng, (10, 160), True))), _dev(1.0), True, offsets, 160, 6, 10, dw=dw)
    torch.cuda.synchronize()
    assert (flat[:32] == 7).all() and (flat[32 + 160 * 50:] == 7).all()


def test_offsets_are_kept_inside(L):
    """Offsets beyond the batch are taken as its end."""
    announce("grouped offsets past the end")
    rng = np.random.default_rng(7)
    codes, a, scale, w, w_scale = _rows_case(rng, [20, 20], 0, 50, 64, "int4s", True, True)
    got = host(_run_rows(L, "int4s", codes, scale, U.pack(w), w_scale, True, np.int32([0, 20, 1000]), 40, 50, 64))
    assert np.array_equal(got, _rows_ref(a, scale, w, w_scale, np.int32([0, 20, 40]), 40, 50, False))


def test_unaligned_output_and_graph(L):
    """Outputs 4 bytes off a 16-byte boundary; captured on a stream and replayed with other groups."""
    T, N, K, E = 96, 128, 64, 4
    rng = np.random.default_rng(8)
    codes, a, scale, w, w_scale = _rows_case(rng, [24] * E, 0, N, K, "int4s", True, True)
    x, wc, xs, ws = to_dev(codes), to_dev(U.pack(w)), _dev(scale), _dev(w_scale)
    flat = torch.zeros(T * N + 8, device="cuda")
    y = flat[1:1 + T * N].view(T, N)
    gt, at = to_dev(U.luq_pack(U.luq_fields(rng, (40, T)))), to_dev(U.pack(U.int4_values(rng, (64, T), True)))
    dw = torch.zeros(E, 40, 64, device="cuda")
    wsp = torch.empty(max(1, L.grouped_wgrad_workspace(T, 40, 64, E)), dtype=torch.uint8, device="cuda")
    offsets = to_dev(_offsets([24] * E))
    announce("grouped graph")

    def step():
        L.int4_gemm_fwd_grouped(x, xs, True, wc, ws, True, offsets, T, N, K, y=y)
        L.luq_gemm_wgrad_grouped(gt, xs, at, xs, True, offsets, T, 40, 64, dw=dw, ws=wsp)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for sizes in ([24] * 4, [0, 96, 0, 0], [1, 2, 3, 80], [90, 1, 0, 5]):
        offsets.copy_(to_dev(_offsets(sizes)))
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(host(y), _rows_ref(a, scale, w, w_scale, _offsets(sizes), T, N, False)), sizes
        assert flat[0] == 0 and not flat[1 + T * N:].any()
        kept = dw.clone()
        step()
        assert torch.equal(kept, dw), sizes


def test_scales_on_the_host_are_refused(L):
    """Before anything is launched: the kernels would read a host address."""
    dev = torch.device("cuda:0")
    codes, one = torch.zeros(64, dtype=torch.uint8, device=dev), torch.ones(1, device=dev)
    offsets, host_one = torch.zeros(4, dtype=torch.int32, device=dev), torch.ones(1)
    announce("scales on the host")
    for call in (lambda: L.int4_gemm_fwd_grouped(codes, host_one, True, codes, one, True, offsets, 1, 1, 32),
                 lambda: L.luq_gemm_dgrad_grouped(codes, host_one, codes, one, True, offsets, 1, 1, 32),
                 lambda: L.luq_gemm_wgrad_grouped(codes, host_one, codes, one, True, offsets, 32, 1, 1),
                 lambda: L.luq_gemm_wgrad_grouped(codes, one, codes, host_one, True, offsets, 32, 1, 1)):
        with pytest.raises(ValueError, match="float32"):
            call()
