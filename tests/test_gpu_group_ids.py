"""luq_group_ids against a stable sort, through the C ABI: lengths around every block and
piece size, vocabularies of one to three digits, skewed, sorted and constant ids, ids that
belong to no group."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import announce, host, to_dev  # noqa: E402
import lm_util as U  # noqa: E402


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2112_10769_amd as lib
    return lib


def _check(L, ids, groups, dtype=np.int64, what=""):
    announce("group_ids", what, ids.size, groups, dtype.__name__)
    order, offsets = L.luq_group_ids(to_dev(ids.astype(dtype)), groups)
    ro, rf = U.group_ids(ids, groups)
    assert np.array_equal(host(offsets), rf), what
    assert np.array_equal(host(order), ro), what


LENGTHS = [0, 1, 2, 63, 64, 65, 511, 512, 513, 2047, 2048, 2049, 4095, 4096, 4097, 8191, 12289, 70001]


@pytest.mark.parametrize("n", LENGTHS)
@pytest.mark.parametrize("groups", [1, 2, 8, 511, 512, 5000, 50021, 262143, 262144, 1 << 20])
def test_lengths_and_groups(L, n, groups):
    rng = np.random.default_rng(n + 7 * groups)
    ids = rng.integers(-1, groups + 1, n)          # both ends have no group
    _check(L, ids, groups, np.int32 if n & 1 else np.int64)


@pytest.mark.parametrize("kind", ["zipf", "one", "none", "ascending", "descending", "last"])
def test_distributions(L, kind):
    n, groups = 33333, 50021
    rng = np.random.default_rng(5)
    ids = {"zipf": np.floor((groups + 1.0) ** rng.random(n)).astype(np.int64) - 1, "one": np.full(n, 17),
           "none": np.full(n, -3), "ascending": np.arange(n), "descending": np.arange(n)[::-1].copy(),
           "last": np.full(n, groups - 1)}[kind]
    _check(L, ids, groups, what=kind)


@pytest.mark.parametrize("groups", [4095, 4096, 4097, 262143, 300007, (1 << 21) + 5])
@pytest.mark.parametrize("n", [1, 300, 8192, 8193, 20001])
def test_gaps(L, n, groups):
    """Ids in few places, with wide stretches of the table between, before and after them."""
    rng = np.random.default_rng(n + groups)
    for places in (1, 2, 5, 70):
        at = rng.integers(0, groups, places)
        for width in (1, 3, 900, 5000):
            ids = np.clip(at[rng.integers(0, places, n)] + rng.integers(0, width, n), -1, groups)
            _check(L, ids, groups, np.int32, (places, width))
    for first, step in ((0, groups // 64), (groups - 1, 0), (groups, 0), (0, 0)):
        _check(L, np.minimum(first + step * np.arange(n), groups), groups, np.int64, (first, step))


def test_extreme_ids(L):
    big = np.array([2 ** 62, -2 ** 62, 2 ** 32, 2 ** 32 + 3, 3, -1, 2 ** 31, 7, 3, 8, 0], dtype=np.int64)
    _check(L, big, 8)
    _check(L, np.array([2 ** 31 - 1, -2 ** 31, 5, 0, 5], dtype=np.int64), 6, np.int32)


def test_long_batch(L):
    rng = np.random.default_rng(11)
    _check(L, rng.integers(0, 300000, (1 << 20) + 4099), 300000)
    _check(L, rng.integers(0, 8, (1 << 21) + 1), 8, np.int32)


def test_other_stream_and_graph(L):
    """On a stream of its own, captured and replayed on new ids."""
    rng = np.random.default_rng(2)
    n, groups = 9001, 700
    ids = to_dev(rng.integers(0, groups, n))
    order = torch.empty(n, dtype=torch.int32, device="cuda")
    offsets = torch.empty(groups + 1, dtype=torch.int32, device="cuda")
    ws = torch.empty(L.workspace_size(L.OP_GROUP_IDS, n, groups), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    announce("group_ids graph")
    with torch.cuda.stream(stream):
        L.luq_group_ids(ids, groups, order, offsets, ws)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.luq_group_ids(ids, groups, order, offsets, ws)
    for k in range(3):
        new = rng.integers(-1, groups, n)
        ids.copy_(to_dev(new))
        graph.replay()
        ro, rf = U.group_ids(new, groups)
        assert np.array_equal(host(order), ro) and np.array_equal(host(offsets), rf), k
