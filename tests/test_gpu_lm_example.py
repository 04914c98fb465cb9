"""examples/moe_lm.py: its gradients against the same step in 64 bits on the codes that its quantizers
made, and its optimizer step against the formula; the new operators of a step captured into a graph."""
import importlib.util
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import announce, host  # noqa: E402
import lm_util  # noqa: E402
import step_util as S  # noqa: E402
from test_gpu_moe_example import Recorder  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("moe_lm", os.path.join(ROOT, "examples", "moe_lm.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _norm(x, w, b):
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + 1e-5)
    xh = (x - mean) * rstd
    return xh * w + b, xh, rstd


def _norm_grad(dy, xh, rstd, w):
    a = dy * w
    return rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True)), (dy * xh).sum(0), dy.sum(0)


def _reference(M, p, bias, ids, targets, values):
    """Loss and gradients in float64; values: w1, w2, x, r, the gradient of o, that of a."""
    w1, w2, x, r, g2, g1 = values
    E, F, D = p["w1"].shape
    w1, w2 = w1.view(E, F, D), w2.view(E, D, F)
    q = {n: v.double() for n, v in p.items()}
    h = q["table"][ids] * math.sqrt(D)
    y, xh1, rstd1 = _norm(h, q["norm1_w"], q["norm1_b"])
    s = torch.sigmoid(y @ q["router"])
    experts = torch.sort(s + bias.double(), dim=1, descending=True, stable=True)[1][:, :M.TOP]
    chosen = s.gather(1, experts)
    share = chosen / chosen.sum(1, keepdim=True)
    flat = experts.reshape(-1)
    order = torch.sort(flat, stable=True)[1]
    token, e, row_share = order // M.TOP, flat[order], share.reshape(-1)[order][:, None]
    n = order.numel()

    def per_expert(rows, w):
        out = torch.zeros(n, w.shape[1], dtype=torch.float64, device="cuda")
        for k in range(E):
            out[e == k] = rows[:n][e == k] @ w[k].t().contiguous()
        return out

    def outer(g, rows):
        return torch.stack([g[:n][e == k].t().contiguous() @ rows[:n][e == k] for k in range(E)])

    def to_tokens(rows):
        return torch.zeros(ids.numel(), rows.shape[1], dtype=torch.float64, device="cuda").index_add_(0, token, rows)
    o = per_expert(r, w2)
    out = h + to_tokens(o * row_share)
    z, xh2, rstd2 = _norm(out, q["norm2_w"], q["norm2_b"])
    kept = targets >= 0
    t = z @ q["table"].t()
    lse = torch.logsumexp(t, 1)
    row = torch.arange(ids.numel(), device="cuda")
    loss = ((lse - t[row, targets.clamp(min=0)]) * kept).sum() / kept.sum()
    g = torch.exp(t - lse[:, None])
    g[row[kept], targets[kept]] -= 1.0
    g *= kept[:, None] / kept.sum()
    table = g.t() @ z
    d_out, dw2, db2 = _norm_grad(g @ q["table"], xh2, rstd2, q["norm2_w"])
    d_share = torch.zeros(share.numel(), dtype=torch.float64, device="cuda")
    d_share[order] = (d_out[token] * o).sum(1)
    d_share = d_share.view_as(share)
    d_chosen = (d_share - (d_share * share).sum(1, keepdim=True)) / chosen.sum(1, keepdim=True)
    d_logits = torch.zeros_like(s).scatter_(1, experts, d_chosen) * s * (1 - s)
    d_y = to_tokens(per_expert(g1, w1.transpose(1, 2).contiguous())) + d_logits @ q["router"].t()
    d_h, dw1, db1 = _norm_grad(d_y, xh1, rstd1, q["norm1_w"])
    table.index_add_(0, ids, (d_h + d_out) * math.sqrt(D))
    return loss, {"table": table, "router": y.t() @ d_logits, "w1": outer(g1, x), "w2": outer(g2, r), "norm1_w": dw1,
                  "norm1_b": db1, "norm2_w": dw2, "norm2_b": db2}


@pytest.mark.parametrize("tokens,vocab,dim,hidden,experts", [(250, 300, 64, 96, 5), (33, 70, 96, 32, 3), (1000, 150, 32, 64, 40)])
def test_gradients_on_the_steps_codes(M, tokens, vocab, dim, hidden, experts):
    """A chain of at most ten fp32 operations, each off by less than 50 roundings of 2^-24 in the 2-norm: 3e-5."""
    p = M.parameters(vocab, dim, hidden, experts)
    g, _ = M.optimizer(p)
    gen = torch.Generator(device="cuda").manual_seed(2)
    bias = 0.05 * torch.randn(experts, device="cuda", generator=gen)
    ids = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    targets = torch.randint(-1, vocab, (tokens,), device="cuda", generator=gen)
    announce("lm example gradients", tokens, experts)
    M.L = Recorder(M.L)
    loss, loads = M.step(p, g, bias, ids, targets)
    assert loads.sum() == tokens * M.TOP
    ref_loss, ref = _reference(M, p, bias, ids, targets, M.L.values)
    assert abs(loss - ref_loss) < 3e-5 * ref_loss
    for name, b in ref.items():
        a = g[name].double().view_as(b)
        assert (a - b).norm() <= 3e-5 * b.norm(), (name, ((a - b).norm() / b.norm()).item())


def test_steps_run_and_update(M):
    """Three steps: every weight moves by AdamW's formula from its gradient (states in fp32: against 64 bits)."""
    p = M.parameters(100, 64, 96, 6)
    g, plan = M.optimizer(p)
    bias, gen = torch.zeros(6, device="cuda"), torch.Generator(device="cuda").manual_seed(3)
    lr, count = torch.full((1,), 1e-3, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    state = {n: (np.zeros(v.numel()), np.zeros(v.numel())) for n, v in p.items()}
    for i in range(3):
        ids = torch.randint(0, 100, (300,), device="cuda", generator=gen)
        announce("lm example step", i)
        loss, loads = M.step(p, g, bias, ids, ids.flip(0), seed=1, counter=i)
        assert torch.isfinite(loss) and all(torch.isfinite(v).all() for v in g.values())
        count += 1
        before = {n: S.f64(v).ravel() for n, v in p.items()}
        M.L.luq_adamw_step(plan, lr, count, seed=2)
        for n, v in p.items():
            if n in ("w1", "w2"):
                assert not np.array_equal(host(v).ravel(), before[n])
                continue
            ref, bound = S.adamw(before[n], S.f64(g[n]).ravel(), *state[n], i + 1, float(np.float32(1e-3)), 0.01 if v.dim() > 1 else 0.0,
                                 0.9, 0.999, 1e-8)
            lm_util.within(host(v).ravel(), ref[0], bound[0] + (i > 0) * 1e-3 * 2.0 ** -18, (n, i))
            state[n] = ref[1:]


def test_captured_step(M):
    """Choice, loss, gradients and update of a step in one graph, replayed with other inputs and scalars between eager
    work; a second graph that shares the workspaces is replayed in turn."""
    L = M.L
    T, V, D, E = 200, 700, 64, 32
    gen = torch.Generator(device="cuda").manual_seed(4)

    def rand(*shape):
        return torch.randn(shape, device="cuda", generator=gen)
    x, table, l, b = rand(T, D).to(torch.bfloat16), (0.1 * rand(V, D)).to(torch.bfloat16), rand(T, E), 0.1 * rand(E)
    y = torch.randint(-1, V, (T,), device="cuda", generator=gen)
    dloss, dw = torch.full((T,), 1.0 / T, device="cuda"), rand(T, 4)
    p, m, v = rand(V * D), torch.zeros(V * D, device="cuda"), torch.zeros(V * D, device="cuda")
    grad = torch.zeros(V, D, device="cuda")
    out = {"loss": torch.empty(T, device="cuda"), "lse": torch.empty(T, device="cuda"), "dx": torch.empty_like(x),
           "experts": torch.empty(T, 4, dtype=torch.int32, device="cuda"), "weights": torch.empty(T, 4, device="cuda"),
           "dl": torch.empty_like(l)}
    plan = L.luq_adamw_plan([p], [grad.view(-1)], [m], [v])
    lr, count = torch.full((1,), 1e-2, device="cuda"), torch.ones(1, dtype=torch.int64, device="cuda")
    ws_f = torch.empty(L.luq_cross_entropy_workspace(T, V, D, x.dtype, table.dtype), dtype=torch.uint8, device="cuda")
    ws_b = torch.empty(L.luq_cross_entropy_workspace(T, V, D, x.dtype, table.dtype, torch.float32), dtype=torch.uint8, device="cuda")

    def work():
        L.luq_route_fwd(l, 4, "sigmoid", b, 4, 2, 2, experts=out["experts"], weights=out["weights"])
        L.luq_route_bwd(dw, l, out["experts"], "sigmoid", dlogits=out["dl"])
        L.luq_cross_entropy_fwd(x, table, y, smoothing=0.1, loss=out["loss"], lse=out["lse"], ws=ws_f)
        L.luq_cross_entropy_bwd(dloss, x, table, y, out["lse"], smoothing=0.1, dx=out["dx"], dtable=grad, ws=ws_b)
        L.luq_adamw_step(plan, lr, count)
    work()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            work()
    for i in range(6):
        announce("captured step", i)
        x.copy_(rand(T, D))
        l.copy_(rand(T, E))
        y.copy_(torch.randint(-1, V, (T,), device="cuda", generator=gen))
        lr.fill_(1e-2 / (i + 1))
        count.fill_(i + 2)
        start = [t.clone() for t in (p, m, v)]
        graphs[i % 2].replay()
        got = [t.clone() for t in (*out.values(), grad, p, m, v)]
        torch.cuda.synchronize()
        for t, s in zip((p, m, v), start):
            t.copy_(s)
        for t in (*out.values(), grad):
            t.zero_()
        work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, (*out.values(), grad, p, m, v))), i
