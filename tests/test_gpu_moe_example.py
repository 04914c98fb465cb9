"""examples/moe_step.py: its gradients against the same step in 64 bits on the codes that its
quantizers made, and its loss falls."""
import importlib.util
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import announce  # noqa: E402
from oracle.luq import unpack_nibbles  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("moe_step", os.path.join(ROOT, "examples", "moe_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


class Recorder:
    """The library, with the values that its quantizers' codes stand for written down in order."""

    def __init__(self, lib):
        self.lib, self.values = lib, []

    def __getattr__(self, name):
        return getattr(self.lib, name)

    def _keep(self, value, codes, shape):
        n = int(np.prod(shape))
        self.values.append(torch.from_numpy(value(unpack_nibbles(codes.cpu().numpy().ravel(), n).astype(np.int64)))
                           .cuda().double().view(*shape))

    def int4_quantize(self, x, is_signed=True, **kw):
        got = self.lib.int4_quantize(x, is_signed, **kw)
        self._keep(lambda q: (np.where(q > 7, q - 16, q) if is_signed else q) * got[2].item(), got[0], x.shape)
        return got

    def luq_quantize_grad(self, g, **kw):
        got = self.lib.luq_quantize_grad(g, **kw)

        def value(q):
            mag = np.where(q & 7, 2.0 ** ((q & 7) - 1), 0.0)
            return np.where(q & 8, -mag, mag) * got[2].item()
        self._keep(value, got[0], g.shape)
        return got


def _reference(M, p, ids, target, values):
    """Loss and gradients in float64; values: w1, w2, x, r, the gradient of o, that of a."""
    w1, w2, x, r, g2, g1 = values
    E, F, D = p["w1"].shape
    w1, w2 = w1.view(E, F, D), w2.view(E, D, F)
    h = p["table"].double()[ids] * math.sqrt(D)
    mean = h.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((h - mean) ** 2).mean(1, keepdim=True) + 1e-5)
    xh = (h - mean) * rstd
    y32, _, _ = M.L.luq_layernorm_fwd(M.L.luq_embedding_fwd(ids, p["table"], math.sqrt(D)), p["gamma"], p["beta"])
    experts, share = M.route(p, y32)
    flat = experts.reshape(-1)
    order = torch.sort(flat, stable=True)[1]
    token, e, share = order // M.TOP, flat[order], share.reshape(-1)[order].double()[:, None]
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
    out = h + to_tokens(per_expert(r, w2) * share)
    d_out = (out - target) / out.numel()
    d_y = to_tokens(per_expert(g1, w1.transpose(1, 2).contiguous()))
    a = d_y * p["gamma"]
    d_h = rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True)) + d_out
    table = torch.zeros(p["table"].shape, dtype=torch.float64, device="cuda").index_add_(0, ids, d_h) * math.sqrt(D)
    grads = {"table": table, "gamma": (d_y * xh).sum(0), "beta": d_y.sum(0), "w1": outer(g1, x), "w2": outer(g2, r)}
    return 0.5 * ((out - target) ** 2).mean(), grads


@pytest.mark.parametrize("tokens,vocab,dim,hidden,experts", [(250, 300, 64, 96, 5), (33, 20, 96, 32, 3), (1000, 50, 32, 64, 40)])
def test_gradients_on_the_steps_codes(M, tokens, vocab, dim, hidden, experts):
    """A chain of at most six fp32 operations, each off by less than 50 roundings of 2^-24 in the 2-norm: 2e-5."""
    p = M.parameters(vocab, dim, hidden, experts)
    gen = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    target = torch.randn(tokens, dim, device="cuda", generator=gen)
    announce("moe example gradients", tokens, experts)
    M.L = Recorder(M.L)
    loss, grads = M.step(p, ids, target)
    ref_loss, ref = _reference(M, p, ids, target, M.L.values)
    assert abs(loss - ref_loss) < 2e-5 * ref_loss
    for name, b in ref.items():
        a = grads[name].double().view_as(b)
        assert (a - b).norm() <= 2e-5 * b.norm(), (name, ((a - b).norm() / b.norm()).item())


def test_loss_falls(M):
    """The table alone takes an eighth of the residual a step."""
    p = M.parameters(200, 64, 128, 4)
    gen = torch.Generator(device="cuda").manual_seed(3)
    teacher = torch.randn(200, 64, device="cuda", generator=gen)
    announce("moe example training")
    losses = []
    for i in range(60):
        ids = torch.randint(0, 200, (1000,), device="cuda", generator=gen)
        loss, grads = M.step(p, ids, teacher[ids], seed=1, counter=i)
        for name, g in grads.items():
            p[name] -= (25.0 if name == "table" else 1.0) * g.view_as(p[name])
        losses.append(loss.item())
    assert losses[-1] < 0.5 * losses[0], losses[::10]
