"""The choice of experts, the loss and AdamW of include/luq_lm.h refuse invalid arguments on the host.
Every call here fails its checks: nothing is enqueued."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
luq = pytest.importorskip("paper_2112_10769_amd")
LIB = luq.LIB

P, P2, P3 = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x20000), ctypes.c_void_p(0x30000)
P8, ODD, HALF = ctypes.c_void_p(0x10008), ctypes.c_void_p(0x10001), ctypes.c_void_p(0x10002)
P4 = ctypes.c_void_p(0x10004)
NUL = None
WS = 1 << 50
SHAPE, DTYPE, PARAM, NULL, WSP, ALIGN = 2, 3, 4, 1, 5, 6
INF, NAN = float("inf"), float("nan")


def _call(fn, defaults, kw):
    a = dict(defaults, **kw)
    assert set(a) == set(defaults)
    return getattr(LIB, fn)(*a.values())


ROUTE = dict(logits=P, dt=0, T=4, E=64, K=8, score=0, bias=NUL, groups=8, top_groups=4, best=2, renorm=1, scale=1.0, chosen=P2,
             weights=P3, stream=NUL)
ROUTE_BAD = [(dict(dt=2), DTYPE), (dict(T=-1), SHAPE), (dict(T=(1 << 25) + 1), SHAPE), (dict(E=0), SHAPE), (dict(E=4097), SHAPE),
             (dict(K=0), SHAPE), (dict(K=65), SHAPE), (dict(score=2), PARAM), (dict(renorm=2), PARAM), (dict(scale=INF), PARAM),
             (dict(scale=NAN), PARAM), (dict(logits=NUL), NULL), (dict(logits=HALF), ALIGN), (dict(logits=ODD, dt=1), ALIGN),
             (dict(chosen=NUL), NULL), (dict(chosen=HALF), ALIGN)]


@pytest.mark.parametrize("kw,status", ROUTE_BAD + [
    (dict(K=33), SHAPE), (dict(groups=0), SHAPE), (dict(groups=65), SHAPE), (dict(groups=7), SHAPE), (dict(top_groups=0), SHAPE),
    (dict(top_groups=9), SHAPE), (dict(top_groups=1, K=9), SHAPE), (dict(best=0), PARAM), (dict(best=3), PARAM),
    (dict(weights=NUL), NULL), (dict(weights=HALF), ALIGN), (dict(bias=ODD), ALIGN)])
def test_route_fwd(kw, status):
    assert _call("luq_route_fwd", ROUTE, kw) == status
    assert LIB.luq_last_error()


ROUTE_BWD = dict(dweights=P, logits=P, dt=0, chosen=P2, T=4, E=64, K=8, score=0, renorm=1, scale=1.0, dlogits=P3, stream=NUL)


@pytest.mark.parametrize("kw,status", ROUTE_BAD + [
    (dict(K=9, E=8), SHAPE), (dict(dweights=NUL), NULL), (dict(dlogits=NUL), NULL), (dict(dweights=HALF), ALIGN),
    (dict(dlogits=HALF), ALIGN), (dict(dlogits=ODD, dt=1), ALIGN)])
def test_route_bwd(kw, status):
    assert _call("luq_route_bwd", ROUTE_BWD, kw) == status
    assert LIB.luq_last_error()


LOSS = dict(x=P, xt=1, table=P2, tt=1, targets=P3, it=0, T=5, V=100, D=64, scale=1.0, smoothing=0.0, loss=P, lse=P2, ws=P3,
            ws_bytes=WS, stream=NUL)
LOSS_BAD = [(dict(xt=2), DTYPE), (dict(tt=-1), DTYPE), (dict(it=2), DTYPE), (dict(T=-1), SHAPE), (dict(T=(1 << 21) + 1), SHAPE),
            (dict(V=0), SHAPE), (dict(V=(1 << 28) + 1), SHAPE), (dict(D=0), SHAPE), (dict(D=(1 << 17) + 1), SHAPE),
            (dict(T=1 << 21, V=1 << 17), SHAPE), (dict(T=1 << 20, D=(1 << 16) + 1), SHAPE), (dict(V=1 << 20, D=(1 << 16) + 1), SHAPE),
            (dict(scale=INF), PARAM), (dict(scale=NAN), PARAM), (dict(scale=0.0), PARAM), (dict(smoothing=-0.1), PARAM), (dict(smoothing=1.1), PARAM),
            (dict(smoothing=NAN), PARAM), (dict(x=NUL), NULL), (dict(table=NUL), NULL), (dict(targets=NUL), NULL),
            (dict(lse=NUL), NULL), (dict(x=P8), ALIGN), (dict(table=P8), ALIGN), (dict(targets=HALF), ALIGN),
            (dict(targets=P4, it=1), ALIGN), (dict(lse=HALF), ALIGN), (dict(ws=NUL), WSP), (dict(ws_bytes=16), WSP), (dict(ws=P8), ALIGN)]


@pytest.mark.parametrize("kw,status", LOSS_BAD + [(dict(loss=NUL), NULL), (dict(loss=HALF), ALIGN)])
def test_cross_entropy_fwd(kw, status):
    assert _call("luq_cross_entropy_fwd", LOSS, kw) == status
    assert LIB.luq_last_error()


LOSS_BWD = dict(dloss=P, x=P, xt=1, table=P2, tt=1, targets=P3, it=0, lse=P, T=5, V=100, D=64, scale=1.0, smoothing=0.0, accumulate=0,
                dx=P, dtable=P2, gt=0, ws=P3, ws_bytes=WS, stream=NUL)


@pytest.mark.parametrize("kw,status", LOSS_BAD + [
    (dict(gt=2), DTYPE), (dict(gt=1, tt=0), DTYPE), (dict(accumulate=2), PARAM), (dict(accumulate=-1), PARAM), (dict(dloss=NUL), NULL),
    (dict(dx=NUL), NULL), (dict(dtable=NUL), NULL), (dict(T=0, dtable=NUL), NULL), (dict(dloss=HALF), ALIGN), (dict(dx=ODD), ALIGN),
    (dict(dx=HALF, xt=0), ALIGN), (dict(dtable=HALF), ALIGN), (dict(dtable=ODD, gt=1), ALIGN)])
def test_cross_entropy_bwd(kw, status):
    assert _call("luq_cross_entropy_bwd", LOSS_BWD, kw) == status
    assert LIB.luq_last_error()


def test_cross_entropy_workspace_takes_any_sizes():
    big = 1 << 62
    for d in ((-1, 5, 5), (5, -1, 5), (5, 0, 5), (5, 5, 0), (big, 5, 5), (5, big, 5), (5, 5, big), (big, big, big), (0, 5, 5)):
        for gt in (-1, 0, 1):
            assert LIB.luq_cross_entropy_workspace(*d, 1, 1, gt) == 0, d
    assert LIB.luq_cross_entropy_workspace(8, 8, 8, 2, 1, -1) == LIB.luq_cross_entropy_workspace(8, 8, 8, 1, 0, 1) == 0
    assert LIB.luq_cross_entropy_workspace(8, 8, 8, 1, 1, 2) == 0
    assert luq.luq_cross_entropy_workspace(8192, 50021, 1024, torch.bfloat16, torch.bfloat16) < 8192 * 50021 // 4    # no logits
    need = luq.luq_cross_entropy_workspace(8192, 200000, 1024, torch.bfloat16, torch.bfloat16, torch.bfloat16)
    assert 0 < need < 8192 * 200000 * 2 // 2




def _tensor(**kw):
    t = dict(p=0x1000, g=0x2000, m=0x3000, v=0x4000, m_scale=None, v_scale=None, copy=None, n=100, weight_decay=0.1, lr_scale=1.0, gt=0,
             state_bits=32)
    t.update(kw)
    return luq._AdamwTensor(**t)


def _plan(t, **kw):
    a = (luq._AdamwTensor * 1)(t)
    plan = (ctypes.c_uint64 * 64)()
    n = LIB.luq_adamw_plan_bytes((ctypes.c_int64 * 1)(max(t.n, 0)), 1)
    d = dict(tensors=ctypes.addressof(a), count=1, plan=ctypes.addressof(plan), bytes=n)
    d.update(kw)
    return LIB.luq_adamw_plan(*d.values())


@pytest.mark.parametrize("kw,status", [
    (dict(gt=2), DTYPE), (dict(state_bits=16), PARAM), (dict(weight_decay=INF), PARAM), (dict(weight_decay=NAN), PARAM),
    (dict(lr_scale=-INF), PARAM), (dict(n=-1), SHAPE), (dict(n=(1 << 35) + 1), SHAPE), (dict(p=None), NULL), (dict(g=None), NULL),
    (dict(m=None), NULL), (dict(v=None), NULL), (dict(state_bits=8), NULL), (dict(state_bits=8, m_scale=0x5000), NULL),
    (dict(p=0x1002), ALIGN), (dict(g=0x2002), ALIGN), (dict(g=0x2001, gt=1), ALIGN), (dict(m=0x3002), ALIGN), (dict(v=0x4001), ALIGN),
    (dict(copy=0x6001), ALIGN)])
def test_adamw_plan(kw, status):
    assert _plan(_tensor(**kw)) == status
    assert LIB.luq_last_error()


def test_adamw_plan_arguments():
    t = _tensor()
    assert _plan(t) == 0
    assert _plan(_tensor(state_bits=8, m=0x3001, v=0x4003, m_scale=0x5001, v_scale=0x6001)) == 0
    for kw, status in ((dict(tensors=None), NULL), (dict(count=-1), SHAPE), (dict(count=(1 << 20) + 1), SHAPE), (dict(plan=None), NULL),
                       (dict(bytes=0), WSP), (dict(bytes=1 << 20), WSP)):
        assert _plan(t, **kw) == status, kw
    assert _plan(_tensor(n=0, p=None, g=None, m=None, v=None)) == 0
    sizes = (ctypes.c_int64 * 3)(4096, 1 << 35, 1)
    assert LIB.luq_adamw_plan_bytes(sizes, 3) == 0 and LIB.luq_adamw_plan_bytes(sizes, 1) > 0 and LIB.luq_adamw_plan_bytes(None, 3) == 0


def _plan_of(tensors):
    a = (luq._AdamwTensor * len(tensors))(*tensors)
    n = luq.luq_adamw_plan_bytes([t.n for t in tensors])
    plan = (ctypes.c_uint64 * (n // 8 + 1))()
    return LIB.luq_adamw_plan(ctypes.addressof(a), len(tensors), ctypes.addressof(plan), n)


def test_adamw_plan_refuses_overlaps():
    """100 elements of 4 bytes from the addresses on: 0x190 bytes."""
    other = dict(p=0x11000, g=0x12000, m=0x13000, v=0x14000)
    assert _plan_of([_tensor(), _tensor(**other)]) == 0
    assert _plan_of([_tensor(), _tensor(**dict(other, g=0x2000))]) == 0            # a shared gradient
    assert _plan_of([_tensor(), _tensor(**dict(other, p=0x1190))]) == 0            # side by side
    assert _plan_of([_tensor(), _tensor(n=0)]) == 0
    for kw in (dict(p=0x1000), dict(p=0x118C), dict(m=0x1000), dict(v=0x3000), dict(g=0x1000), dict(p=0x2000), dict(copy=0x110FE),
               dict(m=0x14000), dict(p=0x0FFC), dict(state_bits=8, m_scale=0x15000, v_scale=0x15003)):
        assert _plan_of([_tensor(), _tensor(**dict(other, **kw))]) == PARAM, kw
    assert _plan_of([_tensor(), _tensor(**dict(other, state_bits=8, m_scale=0x15000, v_scale=0x15004))]) == 0


def test_adamw_plan_covers_every_element():
    """The plan's chunks: each of 4096 elements of a tensor, once, in order."""
    sizes = [1, 0, 4096, 4097, 20000]
    n = luq.luq_adamw_plan_bytes(sizes)
    a = (luq._AdamwTensor * 5)(*[_tensor(n=k, **{name: (4 * i + j + 1) << 20 for j, name in enumerate("pgmv")})
                                 for i, k in enumerate(sizes)])
    plan = (ctypes.c_uint8 * n)()
    assert LIB.luq_adamw_plan(ctypes.addressof(a), 5, ctypes.addressof(plan), n) == 0
    chunks = [-(-k // 4096) for k in sizes]
    table = (ctypes.c_uint32 * (2 * sum(chunks))).from_buffer(plan, n - 8 * sum(chunks))
    want = [v for i, c in enumerate(chunks) for j in range(c) for v in (i, j)]
    assert list(table) == want


STEP = dict(plan=P, bytes=80 + 8, count=1, lr=P2, step=P3, b1=0.9, b2=0.999, eps=1e-8, gs=NUL, seed=0, stream=NUL)


@pytest.mark.parametrize("kw,status", [
    (dict(count=-1), SHAPE), (dict(count=(1 << 20) + 1), SHAPE), (dict(b1=1.0), PARAM), (dict(b1=-0.1), PARAM), (dict(b2=1.0), PARAM),
    (dict(b2=NAN), PARAM), (dict(eps=-1e-9), PARAM), (dict(eps=NAN), PARAM), (dict(eps=INF), PARAM), (dict(bytes=80), WSP),
    (dict(bytes=85), WSP), (dict(bytes=80 + 8 * ((1 << 23) + 2)), SHAPE), (dict(plan=NUL), NULL), (dict(lr=NUL), NULL),
    (dict(step=NUL), NULL), (dict(plan=P8), ALIGN), (dict(lr=HALF), ALIGN), (dict(step=P4), ALIGN), (dict(gs=HALF), ALIGN)])
def test_adamw_step(kw, status):
    assert _call("luq_adamw_step", STEP, kw) == status
    assert LIB.luq_last_error()


def test_binding_checks_buffers():
    """Wrong dtypes, sizes and devices are refused before any pointer is taken."""
    l = torch.zeros(5, 8)
    bad = [lambda: luq.luq_route_fwd(l, 2, "relu"), lambda: luq.luq_route_fwd(l, 2, bias=torch.zeros(7)),
           lambda: luq.luq_route_fwd(l, 2, experts=torch.zeros(5, 2)), lambda: luq.luq_route_fwd(l, 2, weights=torch.zeros(5, 3)),
           lambda: luq.luq_route_bwd(torch.zeros(5, 3), l, torch.zeros(5, 2, dtype=torch.int32)),
           lambda: luq.luq_route_bwd(torch.zeros(5, 2), l, torch.zeros(5, 2)),
           lambda: luq.luq_route_bwd(torch.zeros(5, 2), l, torch.zeros(5, 2, dtype=torch.int32), dlogits=torch.zeros(8, 5).t())]
    x, w, y = torch.zeros(4, 6), torch.zeros(9, 6), torch.zeros(4, dtype=torch.int64)
    f = torch.zeros(4)
    bad += [lambda: luq.luq_cross_entropy_fwd(x, torch.zeros(9, 5), y), lambda: luq.luq_cross_entropy_fwd(x, w, y[:3]),
            lambda: luq.luq_cross_entropy_fwd(x, w, y, loss=torch.zeros(5)), lambda: luq.luq_cross_entropy_fwd(x, w, y, lse=f.double()),
            lambda: luq.luq_cross_entropy_bwd(f[:3], x, w, y, f), lambda: luq.luq_cross_entropy_bwd(f, x, w, y, f.half()),
            lambda: luq.luq_cross_entropy_bwd(f, x, w, y, f, accumulate=True),
            lambda: luq.luq_cross_entropy_bwd(f, x, w, y, f, dx=torch.zeros(4, 6, dtype=torch.bfloat16)),
            lambda: luq.luq_cross_entropy_bwd(f, x, w, y, f, dtable=torch.zeros(9, 7))]
    p = torch.zeros(40)
    u, s = torch.zeros(40, dtype=torch.uint8), torch.zeros(2, dtype=torch.uint8)
    bad += [lambda: luq.luq_adamw_plan([p], [p[:39]], [p], [p]), lambda: luq.luq_adamw_plan([p.double()], [p], [p], [p]),
            lambda: luq.luq_adamw_plan([p], [p], [p], [u]), lambda: luq.luq_adamw_plan([p], [p], [u], [u]),
            lambda: luq.luq_adamw_plan([p], [p], [u], [u], [s[:1]], [s]), lambda: luq.luq_adamw_plan([p], [p], [p], [p], copy=[p]),
            lambda: luq.luq_adamw_plan([p], [p], [p], [p], weight_decay=[0.1, 0.2]), lambda: luq.luq_adamw_plan([p, p], [p], [p, p], [p, p])]
    plan = luq.luq_adamw_plan([p], [p.clone()], [p.clone()], [p.clone()])
    one, step = torch.ones(1), torch.ones(1, dtype=torch.int64)
    bad += [lambda: luq.luq_adamw_step(plan, one.double(), step), lambda: luq.luq_adamw_step(plan, one, one),
            lambda: luq.luq_adamw_step(plan, one, step, grad_scale=torch.ones(2))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("accepted", i)
    with pytest.raises(TypeError):
        luq.luq_route_fwd(l.double(), 2)
    with pytest.raises(TypeError):
        luq.luq_cross_entropy_fwd(x, w, y.float())
    with pytest.raises(TypeError):
        luq.luq_adamw_plan([p], [p.double()], [p], [p])


def test_binding_checks_workspaces():
    ws = torch.zeros(1 << 20, 2, dtype=torch.uint8)[:, 0]
    x, w, y, f = torch.zeros(4, 6), torch.zeros(9, 6), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    for call in (lambda: luq.luq_cross_entropy_fwd(x, w, y, ws=ws), lambda: luq.luq_cross_entropy_bwd(f, x, w, y, f, ws=ws)):
        with pytest.raises(ValueError, match="ws must be"):
            call()
