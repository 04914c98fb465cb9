"""luq_adamw_step against the formula in 64 bits, through the C ABI."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import announce, host  # noqa: E402
import lm_util  # noqa: E402
import step_util as S  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [1, 2, 3, 4, 5, 31, 32, 33, 63, 100, 255, 1000, 1023, 4095, 4096, 4097, 8200, 12289]


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2112_10769_amd as lib
    return lib


def _one(n, gt="f32", bits=32, seed=0, offset=0, copy=False, spread=1.0):
    """A tensor's buffers, each `offset` elements into its allocation."""
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + n)

    def place(v):
        base = torch.zeros(v.numel() + offset, dtype=v.dtype, device="cuda")
        base[offset:] = v
        return base[offset:]
    scale = torch.exp(spread * torch.randn(n, device="cuda", generator=gen)) * 1e-3
    p = torch.randn(n, device="cuda", generator=gen) * 0.02
    g = torch.randn(n, device="cuda", generator=gen) * scale
    t = {"p": place(p), "g": place(g.to(DT[gt])), "copy": place(torch.zeros(n, dtype=torch.bfloat16, device="cuda")) if copy else None}
    if bits == 32:
        t["m"], t["v"] = place(0.3 * scale * torch.randn(n, device="cuda", generator=gen)), place(scale * scale)
        t["ms"] = t["vs"] = None
    else:
        blocks = -(-n // 32)
        t["m"] = place(torch.randint(0, 256, (n,), device="cuda", generator=gen).to(torch.uint8))
        t["m"][t["m"] % 128 == 127] = 0
        t["v"] = place(torch.randint(1, 120, (n,), device="cuda", generator=gen).to(torch.uint8))
        t["ms"] = torch.randint(107, 112, (blocks,), device="cuda", generator=gen).to(torch.uint8)
        t["vs"] = torch.randint(107, 112, (blocks,), device="cuda", generator=gen).to(torch.uint8)
    return t


def _plan(L, ts, **kw):
    return L.luq_adamw_plan([t["p"] for t in ts], [t["g"] for t in ts], [t["m"] for t in ts], [t["v"] for t in ts],
                            [t["ms"] for t in ts], [t["vs"] for t in ts], [t["copy"] for t in ts], **kw)


def _state(t):
    if t["ms"] is None:
        return S.f64(t["m"]), S.f64(t["v"])
    return S.decode(host(t["m"]), host(t["ms"])), S.decode(host(t["v"]), host(t["vs"])) ** 2


def _scalars(lr=1e-3, step=7):
    return torch.full((1,), lr, device="cuda"), torch.full((1,), step, dtype=torch.int64, device="cuda")


def _check(L, ts, step=7, lr=1e-3, wd=None, rates=None, betas=(0.9, 0.999), eps=1e-8, seed=3, gs=None, what=""):
    wd, rates = wd or [0.1] * len(ts), rates or [1.0] * len(ts)
    plan = _plan(L, ts, weight_decay=wd, lr_scale=rates)
    before = [(S.f64(t["p"]), S.f64(t["g"]), *_state(t)) for t in ts]
    lr_t, step_t = _scalars(lr, step)
    announce("adamw", what)
    L.luq_adamw_step(plan, lr_t, step_t, betas, eps, seed, None if gs is None else torch.full((1,), gs, device="cuda"))
    for i, (t, (p, g, m, v)) in enumerate(zip(ts, before)):
        ref, bound = S.adamw(p, g, m, v, max(step, 1), float(np.float32(lr)) * rates[i], wd[i], *betas, eps, 1.0 if gs is None else gs)
        lm_util.within(host(t["p"]), ref[0], bound[0], (what, i, "p"))
        if t["copy"] is not None:
            assert torch.equal(t["copy"], t["p"].to(torch.bfloat16)), (what, i)
        if t["ms"] is None:
            lm_util.within(host(t["m"]), ref[1], bound[1], (what, i, "m"))
            lm_util.within(host(t["v"]), ref[2], bound[2], (what, i, "v"))
        else:
            um, uv = S.uniforms(p.size, i, max(step, 1), seed)
            S.check_codes(host(t["m"]), host(t["ms"]), ref[1], bound[1], um, False, (what, i, "m"))
            root = np.sqrt(ref[2])
            S.check_codes(host(t["v"]), host(t["vs"]), root, 8 * 2.0 ** -24 * root, uv, True, (what, i, "v"))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gt", ["f32", "bf16"])
@pytest.mark.parametrize("copy", [False, True])
def test_step(L, bits, gt, copy):
    """All sizes in one plan, with weight decays and rates of their own; addresses aligned to elements only."""
    for offset in (0, 1, 3):
        ts = [_one(n, gt, bits, offset=offset, copy=copy) for n in SIZES]
        _check(L, ts, wd=[0.1 * (i % 2) for i in range(len(ts))], rates=[1.0 + i % 3 for i in range(len(ts))], what=(bits, gt, copy, offset))


def test_mixed_plan(L):
    """States of both kinds, gradients of both types, copies here and there, empty tensors."""
    ts = [_one(n, ("f32", "bf16")[i % 2], (32, 8)[i // 2 % 2], copy=i % 3 == 0) for i, n in enumerate(SIZES + [0, 5000, 0, 77])]
    _check(L, ts, what="mixed")


@pytest.mark.parametrize("bits", [32, 8])
def test_many_steps_from_zero(L, bits):
    """Twenty steps from states of zeros, step and rate on the device; 8-bit states against the same in 64 bits from the
    codes that each step left."""
    ts = [_one(n, bits=bits) for n in (70, 5000)]
    for t in ts:
        for name in ("m", "v", "ms", "vs"):
            if t[name] is not None:
                t[name].zero_()
    for step in range(1, 21):
        for t in ts:
            t["g"].normal_(generator=torch.Generator(device="cuda").manual_seed(step)).mul_(1e-3)
        _check(L, ts, step=step, lr=1e-3 / step, what=(bits, "step", step))


def test_parameters(L):
    for kw in (dict(betas=(0.0, 0.0)), dict(betas=(0.5, 0.95), eps=1e-3), dict(step=0), dict(step=-5), dict(step=10**6), dict(gs=0.25),
               dict(gs=-3.0), dict(lr=0.0), dict(step=2**33 + 1)):
        for bits in (32, 8):
            _check(L, [_one(300, bits=bits)], what=(kw, bits), **kw)


def test_skipped_step(L):
    for bits in (32, 8):
        t = _one(5000, bits=bits, copy=True)
        before = {k: v.clone() for k, v in t.items() if v is not None}
        plan = _plan(L, [t])
        for gs in (float("nan"), float("inf"), -float("inf")):
            L.luq_adamw_step(plan, *_scalars(), grad_scale=torch.full((1,), gs, device="cuda"))
        assert all(torch.equal(t[k], v) for k, v in before.items())


def test_states_in_8_bits_far_and_small(L):
    """Magnitudes from the smallest subnormal to near the largest fp32, a block of zeros, one element far above the others."""
    t = _one(32 * 9, bits=8)
    for name in ("m", "v", "ms", "vs"):
        t[name].zero_()
    g = torch.randn(9, 32, device="cuda")
    for i, s in enumerate((1e-44, 1e-38, 1e-30, 1e-19, 1.0, 1e15, 1e18)):
        g[i] *= s
    g[7] = 0.0
    g[8] *= 1e-6
    g[8, 5] = 1.0
    t["g"].copy_(g.view(-1))
    # squares below fp32's range vanish as they do in fp32 states
    m, v = (0.1 * g.double()).float(), ((g * g) * np.float32(1 - 0.999))
    L.luq_adamw_step(_plan(L, [t]), *_scalars(step=1), seed=3)
    um, uv = S.uniforms(t["p"].numel(), 0, 1, 3)
    m64, r64 = S.f64(m).ravel(), np.sqrt(S.f64(v).ravel())
    S.check_codes(host(t["m"]), host(t["ms"]), m64, 4 * 2.0 ** -24 * np.abs(m64) + 2e-45, um, False, "m")
    S.check_codes(host(t["v"]), host(t["vs"]), r64, 8 * 2.0 ** -24 * r64 + 2e-23 * (r64 < 1e-18), uv, True, "v")
    assert (host(t["v"])[32 * 7:32 * 8] == 0).all() and (host(t["v"])[r64 > 0] > 0).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_non_finite_gradients_stay_in_their_elements(L, bits):
    t = _one(96, bits=bits)
    t["g"][3], t["g"][40], t["g"][41] = float("nan"), float("inf"), -float("inf")
    other = _one(96, bits=bits)
    L.luq_adamw_step(_plan(L, [t]), *_scalars(), seed=1)
    L.luq_adamw_step(_plan(L, [other]), *_scalars(), seed=1)
    bad = [3, 40, 41]
    keep = [i for i in range(96) if i not in bad]
    assert torch.isnan(t["p"][bad]).all() and torch.equal(t["p"][keep], other["p"][keep])
    if bits == 8:
        assert (t["m"][bad] % 128 == 127).all() and (t["v"][bad] == 127).all()
        assert not (t["m"][keep] % 128 == 127).any()


def test_rounding_is_unbiased(L):
    """The mean of 2^16 elements that stand between two codes, from uniforms of one step: within five deviations."""
    n = 1 << 16
    t = _one(n, bits=8)
    for name in ("m", "v", "ms", "vs"):
        t[name].zero_()
    t["g"].fill_(0.737)
    L.luq_adamw_step(_plan(L, [t]), *_scalars(step=1), (0.9, 0.99), seed=11)
    for codes, scales, want in ((t["m"], t["ms"], 0.1 * 0.737), (t["v"], t["vs"], 0.1 * 0.737)):
        got = S.decode(host(codes), host(scales))
        values = np.unique(got)
        assert len(values) == 2 and values[0] < want < values[1]
        assert abs(got.mean() - want) <= 5 * (values[1] - values[0]) / 2 / np.sqrt(n) + 1e-6 * want


def test_graph_replays_take_new_scalars(L):
    """A captured step reads rate, step and scale at every replay; each replay against the eager step."""
    for bits in (32, 8):
        t, e = _one(5000, bits=bits), _one(5000, bits=bits)
        lr, step = _scalars(step=1)
        plan, eager = _plan(L, [t], weight_decay=0.1), _plan(L, [e], weight_decay=0.1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            L.luq_adamw_step(plan, lr, step, seed=5)
        for i in range(1, 5):
            lr.fill_(1e-3 / i)
            step.fill_(i)
            t["g"].normal_(generator=torch.Generator(device="cuda").manual_seed(i))
            e["g"].copy_(t["g"])
            graph.replay()
            L.luq_adamw_step(eager, lr, step, seed=5)
            torch.cuda.synchronize()
            assert all(torch.equal(t[k], e[k]) for k in t if t[k] is not None), (bits, i)


def test_plan_keeps_and_empty(L):
    assert L.luq_adamw_plan_bytes([]) == 0 and L.luq_adamw_plan_bytes([0, 0]) == 0
    empty = L.luq_adamw_plan([torch.empty(0, device="cuda")], [torch.empty(0, device="cuda")], [torch.empty(0, device="cuda")],
                             [torch.empty(0, device="cuda")])
    L.luq_adamw_step(empty, *_scalars())
    t = _one(100)
    plan = _plan(L, [t])
    want = [t["p"].data_ptr(), t["m"].data_ptr()]
    assert [plan.tensors[0][0].data_ptr(), plan.tensors[2][0].data_ptr()] == want


def test_a_plan_of_nothing(L):
    """No tensors, or tensors without elements: a step that does nothing."""
    lr, step = torch.full((1,), 1e-3, device="cuda"), torch.ones(1, dtype=torch.int64, device="cuda")
    none = [torch.empty(0, device="cuda") for _ in range(4)]
    for lists in ([], [], [], []), [[t] for t in none]:
        L.luq_adamw_step(L.luq_adamw_plan(*lists), lr, step)
    torch.cuda.synchronize()


@pytest.mark.parametrize("gt", ["f32", "bf16"])
def test_every_nan_becomes_one(L, gt):
    """NaN of both signs, with the smallest and the largest payloads, quiet and signalling, over many uniforms."""
    words = [0x7FC00000, 0xFFC00000, 0x7FFFFFFF, 0xFFFFFFFF, 0x7F800001, 0xFF800001] if gt == "f32" else [0x7FC0, 0xFFC0, 0x7FFF, 0xFFFF, 0x7F81, 0xFF81]
    kind = np.uint32 if gt == "f32" else np.uint16
    nans = torch.from_numpy(np.array(words, dtype=kind).view(np.int32 if gt == "f32" else np.int16)).cuda().view(DT[gt])
    n = 32 * 600
    t, other = _one(n, gt, 8), _one(n, gt, 8)
    bad = torch.arange(5, n, 32, device="cuda")           # one in each block
    t["g"][bad] = nans[torch.arange(bad.numel(), device="cuda") % len(words)]
    other["g"][bad] = 0.0
    announce("adamw, every NaN", gt)
    for x in (t, other):
        L.luq_adamw_step(_plan(L, [x]), *_scalars(), seed=9)
    assert torch.isnan(t["p"][bad]).all() and (t["m"][bad] % 128 == 127).all() and (t["v"][bad] == 127).all()
    # the others of a block are as without the NaN, where its element is not the block's largest there
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[bad] = False
    same = ((t["ms"] == other["ms"]) & (t["vs"] == other["vs"])).repeat_interleave(32)
    assert same.float().mean() > 0.5
    assert all(torch.equal(t[k][keep & same], other[k][keep & same]) for k in ("p", "m", "v"))
    assert torch.isfinite(t["p"][keep]).all() and not (t["m"][keep] % 128 == 127).any() and not (t["v"][keep] == 127).any()
