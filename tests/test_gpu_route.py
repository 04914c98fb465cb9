"""luq_route_fwd and luq_route_bwd against plain forms in 64 bits, through the C ABI."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import announce, host  # noqa: E402
import lm_util  # noqa: E402
import step_util as S  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2112_10769_amd as lib
    return lib


def _inputs(T, E, dt, seed=0, barred=0.1, bias=True):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1000 * T + E)
    l = 2.0 * torch.randn(T, E, device="cuda", generator=gen)
    l[torch.rand(T, E, device="cuda", generator=gen) < barred] = -float("inf")
    l[torch.rand(T, device="cuda", generator=gen) < 0.1] = -float("inf")
    b = 0.1 * torch.randn(E, device="cuda", generator=gen)
    return l.to(DT[dt]), b if bias else None, torch.randn(T, E, device="cuda", generator=gen)


def _check(L, l, k, score, b, groups, top_groups, best, renorm, scale, what):
    announce("route_fwd", what)
    experts, weights = L.luq_route_fwd(l, k, score, b, groups, top_groups, best, renorm, scale)
    ref, w, bound = S.route(S.f64(l), k, score, None if b is None else S.f64(b), groups, top_groups, best, renorm, scale)
    assert np.array_equal(host(experts), ref), what
    bad = np.isnan(w)
    assert np.array_equal(np.isnan(host(weights)), bad), what
    lm_util.within(np.where(bad, 0, host(weights)), np.where(bad, 0, w), bound, what)
    return experts, weights


@pytest.mark.parametrize("E", [1, 2, 5, 8, 16, 17, 31, 33, 60, 64, 65, 128, 130, 160, 256, 257, 500, 512, 513, 1000, 1025, 4096])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_forward(L, E, dt):
    for T, k in ((1, 1), (37, min(E, 2)), (66, min(E, 8)), (3, min(E, 64))):
        for score in ("softmax", "sigmoid"):
            for bias in (False, True):
                l, b, _ = _inputs(T, E, dt, bias=bias)
                renorm = (T + bias) % 2 == 0
                _check(L, l, k, score, b, 1, 1, 1, renorm, 1.0 if renorm else 2.5, (T, E, k, dt, score, bias, renorm))


@pytest.mark.parametrize("E,groups,top_groups", [(8, 2, 1), (64, 8, 3), (256, 8, 4), (160, 8, 3), (96, 32, 5), (72, 4, 4),
                                                 (64, 64, 9), (1152, 16, 2), (4096, 64, 8), (15, 5, 2), (448, 7, 3), (512, 2, 1)])
@pytest.mark.parametrize("best", [1, 2])
def test_groups(L, E, groups, top_groups, best):
    k = min(6, top_groups * (E // groups))
    for score in ("softmax", "sigmoid"):
        for bias in (False, True):
            for dt in ("f32", "bf16"):
                l, b, _ = _inputs(41, E, dt, seed=best, barred=0.3, bias=bias)
                _check(L, l, k, score, b, groups, top_groups, best, True, 1.0, (E, groups, best, score, bias, dt))


def test_ties_go_to_the_lowest(L):
    """Equal logits, zeros of both signs, equal groups; few values in many places."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    for E, groups in ((7, 1), (64, 8), (200, 4), (520, 8)):
        l = torch.randint(-1, 2, (50, E), device="cuda", generator=gen).float() * 0.5
        l[:, ::3] *= -1.0     # some zeros are negative
        for b in (None, torch.zeros(E, device="cuda")):
            for best in (1, 2):
                for score in ("softmax", "sigmoid"):
                    _check(L, l, min(E, 6), score, b, groups, max(1, groups // 2), best, True, 1.0, ("ties", E, best, score))
    l = torch.zeros(3, 100, device="cuda")
    experts, weights = L.luq_route_fwd(l, 5)
    assert torch.equal(experts.cpu(), torch.arange(5).repeat(3, 1).int()) and torch.allclose(weights, torch.full_like(weights, 0.2))


def test_near_ties_are_exact(L):
    """Scores one part in 10^9 apart: above fp32's roundings, so the choice must go by 64 bits."""
    E = 128
    l = torch.zeros(40, E, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(6)
    b = 0.5 + torch.zeros(E, device="cuda")
    l += torch.randn(40, E, device="cuda", generator=gen) * 3e-8      # scores differ by 1e-8
    for best, groups in ((1, 1), (2, 8)):
        _check(L, l, 8, "sigmoid", b, groups, max(1, groups // 2), best, True, 1.0, ("near", groups))
        _check(L, l, 8, "softmax", b, groups, max(1, groups // 2), best, True, 1.0, ("near", groups))


def test_bad_and_barred_rows(L):
    """NaN and +inf in a logit or a sum are data errors of their rows; -inf bars; far logits keep their order."""
    l = torch.randn(8, 70, device="cuda")
    l[1, 3], l[2, 69], l[3] = float("nan"), float("inf"), -float("inf")
    l[4, 1:] = -float("inf")
    l[5] *= 1e30
    l[6] -= 2e4
    for score in ("softmax", "sigmoid"):
        for b in (None, torch.zeros(70, device="cuda")):
            experts, weights = L.luq_route_fwd(l, 3, score, b)
            e, w = host(experts), host(weights)
            assert (e[1:4] == -1).all() and np.isnan(w[1:3]).all() and (w[3] == 0).all()
            assert e[4].tolist() == [0, -1, -1] and w[4].tolist() == [1.0, 0.0, 0.0]
            assert np.isfinite(w[4:]).all()
            if b is None:
                _check(L, l[4:], 3, score, b, 1, 1, 1, True, 1.0, "far")
    b = torch.zeros(70, device="cuda")
    b[7], good = -float("inf"), torch.randn(5, 70, device="cuda")
    good[:, 7] = 50.0
    assert not (host(L.luq_route_fwd(good, 64, bias=b)[0]) == 7).any()
    b[7] = float("nan")
    e, w = L.luq_route_fwd(good, 4, bias=b)
    assert (host(e) == -1).all() and np.isnan(host(w)).all()


@pytest.mark.parametrize("E", [1, 3, 8, 16, 30, 64, 65, 129, 160, 256, 500, 1025, 4096])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_backward(L, E, dt):
    for T, k in ((1, 1), (45, min(E, 3)), (34, min(E, 8)), (2, min(E, 64))):
        for score in ("softmax", "sigmoid"):
            for renorm in (True, False):
                l, b, dw = _inputs(T, E, dt, seed=7)
                dw = dw[:, :k].contiguous()
                announce("route_bwd", T, E, k, dt, score, renorm)
                experts, _ = L.luq_route_fwd(l, k, score, b, renorm=renorm)
                got = L.luq_route_bwd(dw, l, experts, score, renorm, 1.5)
                ref, bound = S.route_grad(S.f64(dw), S.f64(l), host(experts), score, renorm, 1.5, dt == "bf16")
                lm_util.within(host(got.float()), ref, bound + 1e-40, (T, E, k, dt, score, renorm))
                again = l.clone()
                assert torch.equal(L.luq_route_bwd(dw, again, experts, score, renorm, 1.5, dlogits=again), got), "in place"


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_backward_against_differences(L, score, renorm):
    """Central differences of the 64-bit form with the choice held: off by the third derivative, h^2 / 6."""
    l, _, dw = _inputs(6, 20, "f32", seed=9, barred=0.0)
    l[torch.isinf(l).any(1)] = 0.5
    k = 4
    experts, _ = L.luq_route_fwd(l, k, score, renorm=renorm)
    dw = dw[:, :k].contiguous()
    got = host(L.luq_route_bwd(dw, l, experts, score, renorm))
    at, h, l64, dw64 = host(experts), 1e-4, S.f64(l), S.f64(dw)

    def value(x):
        s = np.take_along_axis(S.scores(x, score), at, 1)
        return ((s / s.sum(1, keepdims=True) if renorm else s) * dw64).sum(1)
    for e in range(20):
        d = np.zeros_like(l64)
        d[:, e] = h
        num = (value(l64 + d) - value(l64 - d)) / (2 * h)
        assert np.abs(num - got[:, e]).max() <= 1e-5, e


def test_backward_of_odd_choices(L):
    """The same expert twice adds up; experts outside the range and rows without any give nothing."""
    l = torch.randn(4, 9, device="cuda")
    experts = torch.tensor([[2, 2, 5], [-1, 9, 3], [-1, -1, -1], [0, 1, 2**30]], dtype=torch.int32, device="cuda")
    dw = torch.randn(4, 3, device="cuda")
    dw[1, 0] = float("nan")
    l[2] = float("nan")
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            got = host(L.luq_route_bwd(dw, l, experts, score, renorm))
            assert (got[2] == 0).all()
            rows = [0, 1, 3]
            ref, bound = S.route_grad(np.nan_to_num(S.f64(dw)[rows]), S.f64(l)[rows], host(experts)[rows], score, renorm, 1.0, False)
            lm_util.within(got[rows], ref, bound + 1e-40, (score, renorm))


def test_rows_beyond_the_batch_stay(L):
    l = torch.randn(5, 12, device="cuda")
    experts, weights = torch.full((7, 2), 99, dtype=torch.int32, device="cuda"), torch.full((7, 2), 99.0, device="cuda")
    dl = torch.full((7, 12), 99.0, device="cuda")
    L.luq_route_fwd(l, 2, experts=experts[:5], weights=weights[:5])
    L.luq_route_bwd(weights[:5], l, experts[:5], dlogits=dl[:5])
    assert (experts[5:] == 99).all() and (weights[5:] == 99).all() and (dl[5:] == 99).all()
    assert L.luq_route_fwd(l[:0], 2)[0].shape == (0, 2)
    assert L.luq_route_bwd(weights[:0], l[:0], experts[:0]).shape == (0, 12)


def test_strides_streams_and_views(L):
    """A transposed view of logits, another stream, unaligned rows."""
    base = torch.randn(66, 41, device="cuda")
    want = L.luq_route_fwd(base.t().contiguous(), 5)
    got = L.luq_route_fwd(base.t(), 5)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    flat = torch.randn(1 + 40 * 66, device="cuda").to(torch.bfloat16)
    view = flat[1:].view(40, 66)
    assert all(torch.equal(a, b) for a, b in zip(L.luq_route_fwd(view, 5), L.luq_route_fwd(view.clone(), 5)))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = L.luq_route_fwd(base.t().contiguous(), 5)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want))


@pytest.mark.parametrize("E,groups,top_groups", [(65, 1, 1), (96, 8, 3), (128, 1, 1), (128, 8, 4), (160, 8, 3), (256, 8, 4), (250, 5, 2),
                                                 (256, 1, 1), (257, 1, 1), (384, 8, 4), (500, 4, 1), (512, 16, 5)])
def test_many_rows(L, E, groups, top_groups):
    """Long batches, whose rows take fewer lanes: the choices of short ones, which are checked above; weights up to the
    order of a sum of 500 terms."""
    for score, bias, best, dt in (("sigmoid", True, 2, "f32"), ("softmax", True, 1, "bf16"), ("softmax", False, 1, "f32"),
                                  ("sigmoid", False, 1, "bf16"), ("softmax", False, 2, "bf16")):
        T = max(4099, 1400000 // E)
        l, b, _ = _inputs(T, E, dt, seed=3, bias=bias)
        l[100, 3], l[T - 1, E - 1] = float("nan"), float("inf")
        announce("route_fwd many rows", E, groups, score, bias, best, dt)
        for k, renorm in ((8, True), (min(20, top_groups * (E // groups)), False)):
            got = L.luq_route_fwd(l, k, score, b, groups, top_groups, best, renorm)
            for r in (0, 1500, 3000, T - 99):
                part = L.luq_route_fwd(l[r:r + 99], k, score, b, groups, top_groups, best, renorm)
                assert torch.equal(got[0][r:r + 99], part[0])
                assert torch.allclose(got[1][r:r + 99], part[1], rtol=500 * 2.0 ** -24, atol=0, equal_nan=True)


@pytest.mark.parametrize("E,groups,top_groups", [(16, 2, 1), (64, 8, 4), (72, 4, 3), (256, 8, 4), (520, 8, 4), (1100, 10, 5)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_saturated_scores_keep_the_logits_order(L, E, groups, top_groups, score):
    """Without a bias the experts of the groups that remain are ordered by their logits, also where scores of 64 bits are
    equal: sigmoids of logits above 37 are 1, softmaxes of logits 745 below the largest are 0, and logits of 10^-20 and of
    twice that have the same scores of either kind."""
    size, k = E // groups, 6
    rng = np.random.default_rng(E)
    for spread, dt in ((60.0, "f32"), (3000.0, "f32"), (3000.0, "bf16"), (1e-20, "f32")):
        rows = rng.permuted(np.tile(np.arange(E), (37, 1)), axis=1) * (spread / E) + (40.0 if spread == 60.0 else 0.0)
        l = torch.tensor(rows, dtype=torch.float32, device="cuda").to(DT[dt])
        announce("route_fwd saturated", E, groups, score, spread, dt)
        experts, weights = L.luq_route_fwd(l, k, score, None, groups, top_groups, 2)
        s, l64, at = S.scores(S.f64(l), score), S.f64(l), host(experts)
        for t in range(37):
            rank = np.sort(s[t].reshape(groups, size), 1)[:, -2:].sum(1)
            kept = sorted(range(groups), key=lambda g: (-rank[g], g))[:top_groups]
            order = sorted((e for e in range(E) if e // size in kept), key=lambda e: (-l64[t, e], e))
            assert at[t].tolist() == order[:k], (t, l64[t, at[t]], l64[t, order[:k]])
        assert torch.isfinite(weights).all() and (weights.diff(dim=1) <= 0).all()


def test_saturated_scores_of_a_pair(L):
    """Logits of 40 and 50: both sigmoids are 1 in 64 bits, and the second is the larger."""
    l = torch.full((1, 8), -1.0, device="cuda")
    l[0, 1], l[0, 3] = 40.0, 50.0
    for best in (1, 2):
        assert L.luq_route_fwd(l, 2, "sigmoid", None, 2, 1, best)[0].tolist() == [[3, 1]]
