"""Training steps of one layer of experts in 4 bits, with the operators around it.

    tokens -> embedding -> layer norm -> two experts per token, of a two-layer MLP -> residual

The embedding and the norm stay in fp32, as the paper keeps a network's first layer and its
normalisations; the experts' products run on INT4 and LUQ codes in all three directions.
The routed rows are grouped by expert once per step:

  luq_group_ids          of every row's expert: the order of the rows, each expert's bounds
  luq_embedding_fwd      gathers the tokens of those rows (an id of -1 pads the batch)
  luq_embedding_grad     adds the rows of a token up again: the experts' outputs forward,
                         the gradient of the gather backward, the table's gradient

The router is a fixed projection here.  Run:  python examples/moe_step.py [--steps N]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2112_10769_amd as L  # noqa: E402

TOP = 2   # experts per token


def parameters(vocab, dim, hidden, experts, seed=0, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, std):
        return torch.randn(shape, device=device, generator=gen) * std
    return {"table": normal(vocab, dim, std=dim ** -0.5), "gamma": torch.ones(dim, device=device),
            "beta": torch.zeros(dim, device=device), "router": normal(dim, experts, std=dim ** -0.5),
            "w1": normal(experts, hidden, dim, std=(2 / dim) ** 0.5), "w2": normal(experts, dim, hidden, std=hidden ** -0.5)}


def route(p, y):
    """Experts [tokens, TOP] and their shares."""
    top = torch.topk(torch.softmax(y @ p["router"], -1), TOP)
    return top.indices, top.values / top.values.sum(-1, keepdim=True)


def dispatch(experts, n_experts, tokens):
    """Rows sorted by expert: each row's (token, place in the flat list of choices), padded with -1 and 0 to whole
    16-byte pieces of codes (long batches: whole stages of the weight gradient), and the experts' bounds."""
    order, offsets = L.luq_group_ids(experts.reshape(-1), n_experts)
    whole = 32 if order.numel() <= 1 << 18 else 128
    rows = -(-order.numel() // whole) * whole
    pad = rows - order.numel()
    token = torch.nn.functional.pad(order // TOP, (0, pad), value=-1)
    return token, torch.nn.functional.pad(order, (0, pad)).long(), offsets


def step(p, ids, target, seed=0, counter=0):
    """One forward and backward pass: (loss, gradients)."""
    vocab, dim = p["table"].shape
    n_experts, hidden, _ = p["w1"].shape
    tokens, scale = ids.numel(), math.sqrt(dim)
    h = L.luq_embedding_fwd(ids, p["table"], scale)
    y, mean, rstd = L.luq_layernorm_fwd(h, p["gamma"], p["beta"])

    experts, share = route(p, y)
    token, choice, offsets = dispatch(experts, n_experts, tokens)
    by_token = L.luq_group_ids(token, tokens)
    rows = token.numel()
    share = (share.reshape(-1)[choice] * (token >= 0))[:, None]

    # the stacked weights of all experts are quantized in one call each: codes for the forward
    # product, transposed codes (the experts' columns side by side) for the activation gradient
    w1, w1_t, s1 = L.int4_quantize(p["w1"].view(n_experts * hidden, dim), True, codes_t=True)
    w2, w2_t, s2 = L.int4_quantize(p["w2"].view(n_experts * dim, hidden), True, codes_t=True)

    x, x_t, sx = L.int4_quantize(L.luq_embedding_fwd(token, y), True, codes_t=True)
    a = L.int4_gemm_fwd_grouped(x, sx, True, w1, s1, True, offsets, rows, hidden, dim)
    r, r_t, sr = L.int4_quantize(torch.relu(a), False, codes_t=True)
    o = L.int4_gemm_fwd_grouped(r, sr, False, w2, s2, True, offsets, rows, dim, hidden)
    out = h + L.luq_embedding_grad(o * share, token, *by_token)

    diff = out - target
    loss = 0.5 * (diff * diff).mean()

    d_out = diff / diff.numel()
    d_o = L.luq_embedding_fwd(token, d_out) * share
    g, g_t, alpha, _ = L.luq_quantize_grad(d_o, seed=seed, counter=2 * counter, codes_t=True)
    d_r = L.luq_gemm_dgrad_grouped(g, alpha, w2_t, s2, True, offsets, rows, hidden, dim, w_row=n_experts * dim,
                                   w_expert=dim)
    d_w2 = L.luq_gemm_wgrad_grouped(g_t, alpha, r_t, sr, False, offsets, rows, dim, hidden)
    g, g_t, alpha, _ = L.luq_quantize_grad(d_r * (a > 0), seed=seed, counter=2 * counter + 1, codes_t=True)
    d_x = L.luq_gemm_dgrad_grouped(g, alpha, w1_t, s1, True, offsets, rows, dim, hidden, w_row=n_experts * hidden,
                                   w_expert=hidden)
    d_w1 = L.luq_gemm_wgrad_grouped(g_t, alpha, x_t, sx, True, offsets, rows, hidden, dim)
    d_y = L.luq_embedding_grad(d_x, token, *by_token)
    d_h, d_gamma, d_beta = L.luq_layernorm_bwd(d_y, h, mean, rstd, p["gamma"])
    d_table = L.luq_embedding_grad(d_h + d_out, ids, *L.luq_group_ids(ids, vocab), scale)
    return loss, {"table": d_table, "gamma": d_gamma, "beta": d_beta, "w1": d_w1, "w2": d_w2}


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--lr", type=float, default=3.0)
    ap.add_argument("--table-lr", type=float, default=100.0)
    a = ap.parse_args()
    vocab, dim, hidden, experts = 1000, 256, 512, 8
    p = parameters(vocab, dim, hidden, experts)
    gen = torch.Generator(device="cuda").manual_seed(1)
    teacher = torch.randn(vocab, dim, device="cuda", generator=gen)
    for i in range(a.steps):
        ids = torch.randint(0, vocab, (a.tokens,), device="cuda", generator=gen)
        loss, grads = step(p, ids, teacher[ids], seed=7, counter=i)
        for name, g in grads.items():
            p[name] -= (a.table_lr if name == "table" else a.lr) * g.view_as(p[name])
        if i % 10 == 0 or i + 1 == a.steps:
            print(f"step {i}: loss {loss.item():.4f}", flush=True)


if __name__ == "__main__":
    main()
