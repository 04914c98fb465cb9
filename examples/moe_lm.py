"""Training steps of a small language model with experts in 4 bits, all of it in this library but the
router's product.

    tokens -> embedding -> layer norm -> router, two experts per token -> residual -> layer norm
           -> cross entropy on the embedding's table -> AdamW over all weights

  luq_route_fwd          the tokens' experts and shares; luq_route_bwd the router's gradient
  luq_cross_entropy_fwd  the loss on the table shared with the embedding, without the logits;
  luq_cross_entropy_bwd  its gradients, to which luq_embedding_grad adds the lookup's
  luq_adamw_step         one launch for all weights, from a plan made once; the experts' states
                         in 8 bits, the others' in fp32

The experts' products run on INT4 and LUQ codes as in moe_step.py, whose grouping of routed rows
is used here.  The bias that keeps the experts' loads even moves against each one's excess.
Run:  python examples/moe_lm.py [--steps N]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paper_2112_10769_amd as L  # noqa: E402
from moe_step import dispatch  # noqa: E402

TOP = 2   # experts per token


def parameters(vocab, dim, hidden, experts, seed=0, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, std):
        return torch.randn(shape, device=device, generator=gen) * std
    p = {"table": normal(vocab, dim, std=dim ** -0.5), "router": normal(dim, experts, std=dim ** -0.5),
         "w1": normal(experts, hidden, dim, std=(2 / dim) ** 0.5), "w2": normal(experts, dim, hidden, std=hidden ** -0.5)}
    for name in ("norm1", "norm2"):
        p[name + "_w"], p[name + "_b"] = torch.ones(dim, device=device), torch.zeros(dim, device=device)
    return p


def optimizer(p):
    """(gradients' buffers, plan): the experts' states in 8 bits, weight decay on matrices alone."""
    g = {n: torch.zeros_like(v) for n, v in p.items()}
    m, v, ms, vs = [], [], [], []
    for name, w in p.items():
        small = name in ("w1", "w2")
        for states, scales in ((m, ms), (v, vs)):
            states.append(torch.zeros(w.numel(), dtype=torch.uint8 if small else torch.float32, device=w.device))
            scales.append(torch.zeros(-(-w.numel() // 32), dtype=torch.uint8, device=w.device) if small else None)
    return g, L.luq_adamw_plan(list(p.values()), list(g.values()), m, v, ms, vs,
                               weight_decay=[0.01 if w.dim() > 1 else 0.0 for w in p.values()])


def step(p, g, bias, ids, targets, seed=0, counter=0):
    """One forward and backward pass: the loss and each expert's number of tokens; gradients go to g.  Targets of -1
    count for nothing."""
    vocab, dim = p["table"].shape
    n_experts, hidden, _ = p["w1"].shape
    tokens, scale = ids.numel(), math.sqrt(dim)
    h = L.luq_embedding_fwd(ids, p["table"], scale)
    y, mean1, rstd1 = L.luq_layernorm_fwd(h, p["norm1_w"], p["norm1_b"])

    logits = y @ p["router"]
    experts, share = L.luq_route_fwd(logits, TOP, "sigmoid", bias)
    token, choice, offsets = dispatch(experts, n_experts, tokens)
    by_token = L.luq_group_ids(token, tokens)
    rows = token.numel()
    real = (token >= 0)[:, None]
    row_share = share.reshape(-1)[choice][:, None] * real

    w1, w1_t, s1 = L.int4_quantize(p["w1"].view(n_experts * hidden, dim), True, codes_t=True)
    w2, w2_t, s2 = L.int4_quantize(p["w2"].view(n_experts * dim, hidden), True, codes_t=True)
    x, x_t, sx = L.int4_quantize(L.luq_embedding_fwd(token, y), True, codes_t=True)
    a = L.int4_gemm_fwd_grouped(x, sx, True, w1, s1, True, offsets, rows, hidden, dim)
    r, r_t, sr = L.int4_quantize(torch.relu(a), False, codes_t=True)
    o = L.int4_gemm_fwd_grouped(r, sr, False, w2, s2, True, offsets, rows, dim, hidden)
    out = h + L.luq_embedding_grad(o * row_share, token, *by_token)

    z, mean2, rstd2 = L.luq_layernorm_fwd(out, p["norm2_w"], p["norm2_b"])
    loss, lse = L.luq_cross_entropy_fwd(z, p["table"], targets)
    counted = (targets >= 0).sum()
    d_loss = torch.ones_like(loss) / counted

    d_z, _ = L.luq_cross_entropy_bwd(d_loss, z, p["table"], targets, lse, dtable=g["table"])
    d_out, _, _ = L.luq_layernorm_bwd(d_z, out, mean2, rstd2, p["norm2_w"], dgamma=g["norm2_w"], dbeta=g["norm2_b"])
    d_row = L.luq_embedding_fwd(token, d_out)
    d_share = torch.zeros_like(share).reshape(-1)
    d_share[choice[:experts.numel()]] = (d_row * o).sum(1)[:experts.numel()]
    q, q_t, alpha, _ = L.luq_quantize_grad(d_row * row_share, seed=seed, counter=2 * counter, codes_t=True)
    d_r = L.luq_gemm_dgrad_grouped(q, alpha, w2_t, s2, True, offsets, rows, hidden, dim, w_row=n_experts * dim,
                                   w_expert=dim)
    L.luq_gemm_wgrad_grouped(q_t, alpha, r_t, sr, False, offsets, rows, dim, hidden, dw=g["w2"])
    q, q_t, alpha, _ = L.luq_quantize_grad(d_r * (a > 0), seed=seed, counter=2 * counter + 1, codes_t=True)
    d_x = L.luq_gemm_dgrad_grouped(q, alpha, w1_t, s1, True, offsets, rows, dim, hidden, w_row=n_experts * hidden,
                                   w_expert=hidden)
    L.luq_gemm_wgrad_grouped(q_t, alpha, x_t, sx, True, offsets, rows, hidden, dim, dw=g["w1"])
    d_logits = L.luq_route_bwd(d_share.view_as(share), logits, experts, "sigmoid")
    torch.mm(y.t(), d_logits, out=g["router"])
    d_y = L.luq_embedding_grad(d_x, token, *by_token) + d_logits @ p["router"].t()
    d_h, _, _ = L.luq_layernorm_bwd(d_y, h, mean1, rstd1, p["norm1_w"], dgamma=g["norm1_w"], dbeta=g["norm1_b"])
    L.luq_embedding_grad(d_h + d_out, ids, *L.luq_group_ids(ids, vocab), scale, accumulate=True, dtable=g["table"])
    return loss.sum() / counted, offsets.diff()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--lr", type=float, default=3e-3)
    a = ap.parse_args()
    vocab, dim, hidden, experts = 2000, 256, 512, 16
    p = parameters(vocab, dim, hidden, experts)
    g, plan = optimizer(p)
    bias = torch.zeros(experts, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    follows = torch.randperm(vocab, device="cuda", generator=gen)     # what comes after a token, nine times of ten
    lr, count = torch.full((1,), a.lr, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    for i in range(a.steps):
        ids = torch.randint(0, vocab, (a.tokens,), device="cuda", generator=gen)
        chance = torch.rand(a.tokens, device="cuda", generator=gen)
        targets = torch.where(chance < 0.9, follows[ids], torch.randint(0, vocab, (a.tokens,), device="cuda", generator=gen))
        targets[chance > 0.98] = -1
        loss, loads = step(p, g, bias, ids, targets, seed=7, counter=i)
        count += 1
        L.luq_adamw_step(plan, lr, count, seed=11)
        bias += 1e-3 * torch.sign(loads.float().mean() - loads)
        if i % 20 == 0 or i + 1 == a.steps:
            print(f"step {i}: loss {loss.item():.4f}, fullest expert {loads.max().item() * experts / loads.sum().item():.2f} of the mean",
                  flush=True)


if __name__ == "__main__":
    main()
