"""The rest of a language model's training step around the 4-bit products, as measurable cases.

    listed()   the named cases
    draw(rng)  one more case of the same ranges
    prepare    inputs, and the output buffers, workspaces and plans that a program keeps, on the GPU
    run        one pass: the library's calls where `own` is true, else the plain form in torch
    work       the bytes and operations a pass cannot do without
    exact      the outputs in 64 bits, from the definition, without the library

Kinds of case
  route_fwd  experts and weights of every token from the router's logits: softmax or sigmoid scores, a bias
             that moves the choice alone, groups of experts, the top k, weights that add up to one
  route_bwd  the gradient of the logits from that of the weights
  loss_fwd   softmax cross entropy of the last layer's products with the embedding table, the logits not kept:
             every token's loss and log of the sum of exponentials
  loss_bwd   its gradients: of the activations and of the table (written, or added to a gradient that is there)
  adamw      one AdamW step over many tensors, which lie one after the other in flat buffers: states in fp32,
             or in 8 bits (e4m3 elements of which 32 share a power of two, rounded stochastically)

Router logits have a part that belongs to the expert, so that some experts are chosen several times as often as
others; tokens that are padding have logits of -inf throughout.  Table rows are normal, activations too, with a
part along the target's row, so that some tokens are predicted well and others not at all.  States of the
optimizer are those of a run under way: the mean of gradients below the root of the mean of their squares.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BETAS, ADAM_EPS = (0.9, 0.999), 1e-8
SEED = 20211220          # of the stochastic rounding
BLOCK = 32               # elements that share a power of two; tensors begin at multiples of it

# The largest drawn cases: the work of the largest listed ones.
_MAX_ROUTE = 16384 * 256
_MAX_LOSS = 8192 * 32000 * 4096
_MAX_LOSS_F32 = 8192 * 50021 * 1024
_MAX_TABLE = 32000 * 4096
_MAX_ADAMW = 2 * 4096 * 16384


def listed():
    return [
        # one decoding step of four sequences: 8 of 256 experts in groups, sigmoid scores with a bias for balance
        {"name": "route_decode", "kind": "route_fwd", "tokens": 4, "experts": 256, "top": 8, "score": "sigmoid",
         "bias": True, "groups": 8, "top_groups": 4, "best": 2, "renorm": True, "dtype": "f32", "padding": 0.0},
        # the choice of a training batch, bf16 logits, an eighth of the positions padding
        {"name": "route_batch", "kind": "route_fwd", "tokens": 16384, "experts": 64, "top": 2, "score": "softmax",
         "bias": False, "groups": 1, "top_groups": 1, "best": 1, "renorm": True, "dtype": "bf16", "padding": 0.125},
        # the same with many experts in groups and a bias: what the choice itself costs
        {"name": "route_groups", "kind": "route_fwd", "tokens": 16384, "experts": 256, "top": 8, "score": "sigmoid",
         "bias": True, "groups": 8, "top_groups": 4, "best": 2, "renorm": True, "dtype": "f32", "padding": 0.0},
        # the backward of a softmax router over all its experts, odd sizes
        {"name": "route_grad", "kind": "route_bwd", "tokens": 8111, "experts": 160, "top": 6, "score": "softmax",
         "bias": False, "groups": 1, "top_groups": 1, "best": 1, "renorm": False, "dtype": "f32", "padding": 0.1},
        # scoring four tokens: one read of the table
        {"name": "loss_token", "kind": "loss_fwd", "tokens": 4, "vocab": 32000, "dim": 4096, "dtype": "bf16",
         "table": "bf16", "smoothing": 0.0, "padding": 0.0},
        # the loss of a batch with label smoothing, some of the positions padding
        {"name": "loss_batch", "kind": "loss_fwd", "tokens": 8192, "vocab": 50021, "dim": 1024, "dtype": "bf16",
         "table": "bf16", "smoothing": 0.1, "padding": 0.05},
        # the gradients of a short fine-tuning batch in fp32, odd sizes
        {"name": "loss_grad_odd", "kind": "loss_bwd", "tokens": 509, "vocab": 8000, "dim": 510, "dtype": "f32",
         "table": "f32", "grad": "f32", "smoothing": 0.1, "padding": 0.1, "accumulate": False},
        # a table shared with the embedding: its fp32 gradient is added to the lookup's
        {"name": "loss_grad_tied", "kind": "loss_bwd", "tokens": 4096, "vocab": 32000, "dim": 1024, "dtype": "bf16",
         "table": "bf16", "grad": "f32", "smoothing": 0.0, "padding": 0.0, "accumulate": True},
        # the gradients of a large batch on a wide table
        {"name": "loss_grad_batch", "kind": "loss_bwd", "tokens": 8192, "vocab": 32000, "dim": 4096, "dtype": "bf16",
         "table": "bf16", "grad": "bf16", "smoothing": 0.0, "padding": 0.0, "accumulate": False},
        # the norms' weights and biases and a small router: many short tensors, one step
        {"name": "adamw_small", "kind": "adamw", "tensors": 97, "total": 100003, "skew": 0.3, "bits": 32, "grad": "f32",
         "copy": False},
        # the two weights of the benchmark's MLP layer, states in fp32
        {"name": "adamw_mlp", "kind": "adamw", "tensors": 2, "total": 2 * 4096 * 16384, "skew": 0.0, "bits": 32,
         "grad": "f32", "copy": False},
        # a model's tensors of very different sizes, states in 8 bits, bf16 gradients and a bf16 copy of the weights
        {"name": "adamw_8bit", "kind": "adamw", "tensors": 40, "total": 50021 * 1024, "skew": 1.0, "bits": 8,
         "grad": "bf16", "copy": True},
    ]


def _log_uniform(rng, lo, hi, step=1):
    """A multiple of step in [lo, hi], spread evenly over its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(max(int(round(v / step)) * step, -(-lo // step) * step), hi // step * step)


def draw(rng):
    kind = rng.choice(["route_fwd", "route_fwd", "route_bwd", "loss_fwd", "loss_bwd", "loss_bwd", "adamw", "adamw"])
    while True:
        if kind in ("route_fwd", "route_bwd"):
            groups = rng.choice([1, 1, 2, 4, 8, 16])
            best = rng.choice([1, 2]) if groups > 1 else 1
            size = _log_uniform(rng, 4, 512) if groups == 1 else _log_uniform(rng, 4, 64)
            kept = groups if groups == 1 else rng.randint(1, groups)
            c = {"kind": kind, "tokens": _log_uniform(rng, 1, 65536), "experts": groups * size,
                 "top": min(kept * size, rng.choice([1, 2, 4, 6, 8, 8, 13])), "score": rng.choice(["softmax", "sigmoid"]),
                 "bias": rng.random() < 0.5, "groups": groups, "top_groups": kept, "best": best,
                 "renorm": rng.random() < 0.7, "dtype": rng.choice(["f32", "bf16"]), "padding": rng.choice([0.0, 0.0, 0.2])}
            if c["tokens"] * c["experts"] <= _MAX_ROUTE:
                return c
        elif kind in ("loss_fwd", "loss_bwd"):
            dtype, table = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
            c = {"kind": kind, "tokens": _log_uniform(rng, 1, 16384), "vocab": _log_uniform(rng, 100, 200000),
                 "dim": _log_uniform(rng, 32, 8192, rng.choice([1, 8, 64])), "dtype": dtype, "table": table,
                 "smoothing": rng.choice([0.0, 0.0, 0.1]), "padding": rng.choice([0.0, 0.0, 0.2])}
            if kind == "loss_bwd":
                c["grad"] = rng.choice(["f32", table])
                c["accumulate"] = c["grad"] == "f32" and rng.random() < 0.4
            most = _MAX_LOSS if dtype == table == "bf16" else _MAX_LOSS_F32
            if c["tokens"] * c["vocab"] * c["dim"] <= most and c["vocab"] * c["dim"] <= _MAX_TABLE:
                return c
        else:
            c = {"kind": kind, "tensors": _log_uniform(rng, 1, 400), "total": _log_uniform(rng, 1000, _MAX_ADAMW),
                 "skew": rng.choice([0.0, 0.3, 1.0]), "bits": rng.choice([32, 8]), "grad": rng.choice(["f32", "bf16"]),
                 "copy": rng.random() < 0.5}
            if c["total"] >= 2 * c["tensors"] and (c["bits"] == 32 or c["total"] <= _MAX_ADAMW // 2):
                return c


# ---- inputs ------------------------------------------------------------------------------------


def _sizes(case):
    """Elements of each tensor: a power law, rounded down, at least one."""
    n, total = case["tensors"], case["total"]
    w = [(i + 1.0) ** -case["skew"] for i in range(n)]
    got = [max(1, int(total * v / sum(w))) for v in w]
    got[0] += max(0, total - sum(got))
    return got


def _starts(sizes):
    """Where each tensor begins in the flat buffers, and where the last ends: whole blocks."""
    starts = [0]
    for n in sizes:
        starts.append(starts[-1] + -(-n // BLOCK) * BLOCK)
    return starts


def _decays(case):
    """Weight decay of each tensor: of every second one, as weights and biases alternate; and the factor of its rate."""
    n = case["tensors"]
    return [0.1 if i % 2 == 0 else 0.0 for i in range(n)], [1.0 if i % 3 else 0.5 for i in range(n)]


def _inputs(case, seed):
    """The tensors of a case, made from the seed alone."""
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    kind = case["kind"]

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=gen)

    def uniform(*shape):
        return torch.rand(shape, device=DEV, generator=gen)

    if kind in ("route_fwd", "route_bwd"):
        t, e = case["tokens"], case["experts"]
        logits = (normal(t, e) + 0.7 * normal(e)).to(DTYPES[case["dtype"]])
        logits[uniform(t) < case["padding"]] = -math.inf
        got = {"logits": logits, "bias": 0.05 * normal(e) if case["bias"] else None}
        if kind == "route_bwd":
            got["dweights"] = 1e-3 * normal(t, case["top"])
        return got
    if kind in ("loss_fwd", "loss_bwd"):
        t, v, d = case["tokens"], case["vocab"], case["dim"]
        table = (0.02 * normal(v, d)).to(DTYPES[case["table"]])
        targets = torch.randint(0, v, (t,), device=DEV, generator=gen)
        rows = table[targets].float()
        sure = 12.0 * uniform(t, 1) ** 2 / (rows * rows).sum(1, keepdim=True)
        x = (normal(t, d) + sure * rows).to(DTYPES[case["dtype"]])
        targets[uniform(t) < case["padding"]] = -1
        got = {"x": x, "weights": table, "targets": targets}
        if kind == "loss_bwd":
            got["dloss"] = (0.5 + uniform(t)) / t
            if case["accumulate"]:
                got["dtable"] = 1e-4 * normal(v, d)
        return got
    sizes = _sizes(case)
    starts = _starts(sizes)
    n = starts[-1]
    block = torch.arange(n // BLOCK, device=DEV)
    tensor = torch.searchsorted(torch.tensor(starts[1:], device=DEV), block * BLOCK, right=True)
    end = torch.tensor([s + k for s, k in zip(starts, sizes)], device=DEV)[tensor]
    here = (block * BLOCK)[:, None] + torch.arange(BLOCK, device=DEV) < end[:, None]      # what is no filling
    scale = torch.exp(1.5 * normal(len(sizes)) - 9.0)[tensor][:, None] * torch.exp(0.7 * normal(n // BLOCK, BLOCK)) * here
    got = {"p": (0.02 * normal(n // BLOCK, BLOCK) * here).view(-1),
           "g": (normal(n // BLOCK, BLOCK) * scale).view(-1).to(DTYPES[case["grad"]]),
           "lr": torch.full((1,), 3e-4, device=DEV),
           "step": torch.randint(10, 5000, (1,), device=DEV, generator=gen)}
    m, r = 0.3 * normal(n // BLOCK, BLOCK) * scale, scale * torch.exp(0.2 * normal(n // BLOCK, BLOCK))
    if case["bits"] == 32:
        got["m"], got["v"] = m.view(-1), (r * r).view(-1)
    else:
        half = torch.full_like(block, 1 << 15)[:, None]
        for name, value in (("m", m), ("v", r)):
            codes, exponent = _encode(value, half, name == "v")
            got[name], got[name + "_scale"] = codes.view(-1), exponent
    if case["copy"]:
        got["copy"] = got["p"].to(torch.bfloat16)
    # the tensor of every block, and the block's place in it
    got["tensor"], got["place"] = tensor, block - torch.tensor(starts, device=DEV)[tensor] // BLOCK
    return got


def _encode(x, u, positive):
    """e4m3 codes of x [blocks, 32] and the blocks' exponents (biased by 127): magnitudes over 2^exponent are below
    256, and go up to the next code where their fraction plus u / 2^16 reaches one (u is below 2^16)."""
    a = x.abs()
    exponent = ((a.amax(1).view(torch.int32) >> 23) - 134).clamp_(min=-127)
    y = a * ((127 - exponent) << 23).view(torch.float32)[:, None]
    u = (u << 4).to(torch.int32)
    whole = ((y.view(torch.int32) + u) >> 20) - (120 << 3)
    small = ((y * 2.0 ** 29).to(torch.int32) + u) >> 20
    code = torch.where(y < 2.0 ** -6, small, whole)
    if positive:      # a root of a mean of squares does not become 0: it divides
        code = torch.where(a > 0, code.clamp(min=1), code)
    else:
        code = torch.where((x < 0) & (code > 0), code | 128, code)
    return code.to(torch.uint8), (exponent + 127).to(torch.uint8)


def _decode(codes, exponent):
    """The values of e4m3 codes [blocks, 32]."""
    value = codes.view(torch.float8_e4m3fn).to(torch.float32)
    e = exponent.to(torch.int32)
    # 2^(e - 127) in two factors, neither of which is subnormal
    return value * ((e // 2 + 64) << 23).view(torch.float32)[:, None] * ((e - e // 2 + 63) << 23).view(torch.float32)[:, None]


def prepare(case, seed):
    """What a program has in hand before the call: logits, activations, tables, gradients and states; what the forward
    call gave to the backward one; and, for the library, the output buffers, workspaces and plans it keeps."""
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "route_bwd":
        s["experts"] = _route(case, s["logits"], s["bias"])[0]
    elif case["kind"] == "loss_bwd":
        z, _ = _logits(case, s)
        s["lse"] = _lse(z)
        s["lse"][s["targets"] < 0] = 0.0
        del z
    elif case["kind"] == "adamw":
        s["decay"], s["rate"] = (torch.tensor(v, device=DEV, dtype=torch.float64) for v in _decays(case))
    if own:
        _prepare_own(case, s)
    return s


def _prepare_own(case, s):
    import paper_2112_10769_amd as L

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    kind = case["kind"]
    if kind == "route_fwd":
        t, k = case["tokens"], case["top"]
        s.update(experts=empty(t, k, dtype=torch.int32), weights=empty(t, k))
    elif kind == "route_bwd":
        s.update(dlogits=torch.empty_like(s["logits"]))
    elif kind in ("loss_fwd", "loss_bwd"):
        t, v, d = case["tokens"], case["vocab"], case["dim"]
        grad = DTYPES[case["grad"]] if kind == "loss_bwd" else None
        s["ws"] = empty(max(L.luq_cross_entropy_workspace(t, v, d, s["x"].dtype, s["weights"].dtype, grad), 1), dtype=torch.uint8)
        if kind == "loss_fwd":
            s.update(loss=empty(t), lse=empty(t))
        else:
            s["dx"] = torch.empty_like(s["x"])
            if not case["accumulate"]:
                s["dtable"] = empty(v, d, dtype=grad)
    else:
        sizes = _sizes(case)
        starts = _starts(sizes)

        def parts(name, per=1):
            return [s[name][a // per:a // per + -(-n // per)] for a, n in zip(starts, sizes)]
        decay, rate = _decays(case)
        scales = {} if case["bits"] == 32 else {"m_scale": parts("m_scale", BLOCK), "v_scale": parts("v_scale", BLOCK)}
        s["plan"] = L.luq_adamw_plan(parts("p"), parts("g"), parts("m"), parts("v"), weight_decay=decay, lr_scale=rate,
                                     copy=parts("copy") if case["copy"] else None, **scales)


# ---- one pass ----------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)(s["case"], s)


def _run_own(case, s):
    import paper_2112_10769_amd as L

    kind = case["kind"]
    if kind == "route_fwd":
        L.luq_route_fwd(s["logits"], case["top"], case["score"], s["bias"], case["groups"], case["top_groups"], case["best"],
                        case["renorm"], experts=s["experts"], weights=s["weights"])
        return {"experts": s["experts"], "weights": s["weights"]}
    if kind == "route_bwd":
        return {"dlogits": L.luq_route_bwd(s["dweights"], s["logits"], s["experts"], case["score"], case["renorm"],
                                           dlogits=s["dlogits"])}
    if kind == "loss_fwd":
        L.luq_cross_entropy_fwd(s["x"], s["weights"], s["targets"], smoothing=case["smoothing"], loss=s["loss"], lse=s["lse"],
                                ws=s["ws"])
        return {"loss": s["loss"], "lse": s["lse"]}
    if kind == "loss_bwd":
        L.luq_cross_entropy_bwd(s["dloss"], s["x"], s["weights"], s["targets"], s["lse"], smoothing=case["smoothing"],
                                accumulate=case["accumulate"], dx=s["dx"], dtable=s["dtable"], ws=s["ws"])
        return {"dx": s["dx"], "dtable": s["dtable"]}
    L.luq_adamw_step(s["plan"], s["lr"], s["step"], BETAS, ADAM_EPS, seed=SEED)
    return _adamw_outputs(case, s)


def _adamw_outputs(case, s):
    """The buffers; states in 8 bits as the e4m3 values that they are, in units of their blocks' powers of two."""
    if case["bits"] == 32:
        got = {"p": s["p"], "m": s["m"], "v": s["v"]}
    else:
        got = {"p": s["p"], "m": s["m"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn),
               "m_scale": s["m_scale"], "v_scale": s["v_scale"]}
    if case["copy"]:
        got["copy"] = s["copy"]
    return got


def _scores(case, logits, bias):
    """Scores and what the choice goes by, in 64 bits: a choice between two sums must not hang on a rounding."""
    l = logits.double()
    if case["score"] == "softmax":
        e = torch.exp(l - l.amax(1, keepdim=True).clamp(min=-1e300))
        total = e.sum(1, keepdim=True)
        s = torch.where(total > 0, e / total, torch.zeros_like(e))
    else:
        s = 1.0 / (1.0 + torch.exp(-l))
    c = s if bias is None else s + bias.double()
    return s, torch.where(l == -math.inf, torch.full_like(c, -math.inf), c)


def _route(case, logits, bias):
    """(experts, weights): -1 and 0 where there is no expert to choose."""
    s, c = _scores(case, logits, bias)
    t, e = c.shape
    g = case["groups"]
    if g > 1:
        best = torch.sort(c.view(t, g, e // g), dim=2, descending=True)[0][..., :case["best"]]
        score = torch.where(best[..., 0] == -math.inf, best[..., 0], torch.where(best == -math.inf, 0.0, best).sum(-1))
        order = torch.sort(score, dim=1, descending=True, stable=True)[1]
        out = torch.zeros_like(score, dtype=torch.bool).scatter_(1, order[:, case["top_groups"]:], True)
        c = torch.where(out[..., None], -math.inf, c.view(t, g, e // g)).view(t, e)
    value, experts = torch.sort(c, dim=1, descending=True, stable=True)
    value, experts = value[:, :case["top"]], experts[:, :case["top"]]
    none = value == -math.inf
    w = torch.where(none, 0.0, s.gather(1, experts))
    if case["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return torch.where(none, -1, experts).to(torch.int32), w.float()


def _logits(case, s):
    x, w = s["x"].float(), s["weights"].float()
    return x @ w.t(), (x, w)


def _lse(z):
    m = z.amax(1, keepdim=True)
    return (m + torch.log(torch.exp(z - m).sum(1, keepdim=True))).view(-1)


def _philox(c, key):
    """Philox4x32-10 of the counter words c (int64 tensors below 2^32)."""
    m0, m1 = 0xD2511F53, 0xCD9E8D57

    def product(a, m):
        low = (a & 0xFFFF) * m
        t = (a >> 16) * m + (low >> 16)
        return t >> 16, ((t & 0xFFFF) << 16) | (low & 0xFFFF)
    k0, k1 = key & 0xFFFFFFFF, key >> 32
    for _ in range(10):
        (h0, l0), (h1, l1) = product(c[0], m0), product(c[2], m1)
        c = (h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0)
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def _uniforms(s):
    """The 16-bit uniforms of every element: (for m, for the root of v).  Four elements share a Philox call."""
    quad = (s["place"][:, None] * (BLOCK // 4) + torch.arange(BLOCK // 4, device=DEV)).view(-1)
    zero = torch.zeros_like(quad)
    words = _philox((quad & 0xFFFFFFFF, quad >> 32, zero + s["tensor"][:, None].expand(-1, BLOCK // 4).reshape(-1),
                     zero + s["step"]), SEED)
    words = torch.stack(words, -1).view(-1, BLOCK)
    return words & 0xFFFF, words >> 16


def _run_plain(case, s):
    kind = case["kind"]
    if kind == "route_fwd":
        experts, weights = _route(case, s["logits"], s["bias"])
        return {"experts": experts, "weights": weights}
    if kind == "route_bwd":
        sc = _scores(case, s["logits"], None)[0].float()
        none = s["experts"] < 0
        at = s["experts"].long().clamp(min=0)
        chosen, ds = torch.where(none, 0.0, sc.gather(1, at)), torch.where(none, 0.0, s["dweights"])
        if case["renorm"]:
            total = chosen.sum(1, keepdim=True)
            share = torch.where(total > 0, chosen / total, 0.0)
            ds = torch.where(total > 0, (ds - (ds * share).sum(1, keepdim=True)) / total, 0.0)
            ds = torch.where(none, 0.0, ds)
        each = torch.zeros_like(sc).scatter_add_(1, at, ds)
        if case["score"] == "softmax":
            d = sc * (each - (each * sc).sum(1, keepdim=True))
        else:
            d = sc * (1.0 - sc) * each
        return {"dlogits": d.to(s["logits"].dtype)}
    if kind == "loss_fwd":
        z, _ = _logits(case, s)
        lse, eps = _lse(z), case["smoothing"]
        at = s["targets"].clamp(min=0)[:, None]
        loss = lse - (1.0 - eps) * z.gather(1, at).view(-1)
        if eps:
            loss = loss - eps / case["vocab"] * z.sum(1)
        pad = s["targets"] < 0
        return {"loss": torch.where(pad, 0.0, loss), "lse": torch.where(pad, 0.0, lse)}
    if kind == "loss_bwd":
        z, (x, w) = _logits(case, s)
        eps, pad = case["smoothing"], s["targets"] < 0
        g = torch.exp(z - s["lse"][:, None])
        if eps:
            g -= eps / case["vocab"]
        g.scatter_add_(1, s["targets"].clamp(min=0)[:, None], torch.full_like(s["dloss"][:, None], eps - 1.0))
        g = torch.where(pad[:, None], 0.0, g * s["dloss"][:, None])
        dtable = g.t() @ x
        if case["accumulate"]:
            dtable = s["dtable"].add_(dtable)
        return {"dx": (g @ w).to(s["x"].dtype), "dtable": dtable.to(DTYPES[case["grad"]])}
    # AdamW on the flat buffers; the filling between tensors holds zeros, and stays so
    blocks = s["place"].numel()
    b1, b2 = BETAS
    t = s["step"].double()
    rate = s["lr"].double() * s["rate"]
    size = (rate / (1.0 - b1 ** t)).float()[s["tensor"]][:, None]
    keep = (1.0 - rate * s["decay"]).float()[s["tensor"]][:, None]
    root = (1.0 / torch.sqrt(1.0 - b2 ** t)).float()
    g, p = s["g"].view(blocks, BLOCK).float(), s["p"].view(blocks, BLOCK)
    if case["bits"] == 32:
        m, v = s["m"].view(blocks, BLOCK), s["v"].view(blocks, BLOCK)
    else:
        m = _decode(s["m"].view(blocks, BLOCK), s["m_scale"])
        r = _decode(s["v"].view(blocks, BLOCK), s["v_scale"])
        v = r * r
    m1 = m * b1 + g * (1.0 - b1)
    v1 = v * b2 + g * g * (1.0 - b2)
    r1 = torch.sqrt(v1)
    p.copy_(p * keep - size * m1 / (r1 * root + ADAM_EPS))
    if case["bits"] == 32:
        m.copy_(m1)
        v.copy_(v1)
    else:
        um, uv = _uniforms(s)
        codes, exponent = _encode(m1, um, False)
        s["m"].copy_(codes.view(-1))
        s["m_scale"].copy_(exponent)
        codes, exponent = _encode(r1, uv, True)
        s["v"].copy_(codes.view(-1))
        s["v_scale"].copy_(exponent)
    if case["copy"]:
        s["copy"].copy_(s["p"])
    return _adamw_outputs(case, s)


# ---- what a pass cannot do without ---------------------------------------------------------------


def work(case):
    """Inputs read once, outputs written once; additions and multiplications."""
    kind = case["kind"]
    if kind in ("route_fwd", "route_bwd"):
        t, e, k = case["tokens"], case["experts"], case["top"]
        size = 4 if case["dtype"] == "f32" else 2
        if kind == "route_fwd":
            return {"bytes": t * e * size + 8 * t * k + (4 * e if case["bias"] else 0), "flops": t * e * (4 + k)}
        return {"bytes": 2 * t * e * size + 8 * t * k, "flops": t * (6 * e + 8 * k)}
    if kind in ("loss_fwd", "loss_bwd"):
        t, v, d = case["tokens"], case["vocab"], case["dim"]
        x, w = (4 if case[n] == "f32" else 2 for n in ("dtype", "table"))
        product = 2 * t * (1.0 - case["padding"]) * v * d
        if kind == "loss_fwd":
            return {"bytes": t * d * x + v * d * w + 16 * t, "flops": product}
        grad = (4 if case["grad"] == "f32" else 2) * (2 if case["accumulate"] else 1)
        return {"bytes": 2 * t * d * x + v * d * (w + grad) + 16 * t, "flops": 3 * product}
    each = 8 + (4 if case["grad"] == "f32" else 2) + (16 if case["bits"] == 32 else 4 + 4 / BLOCK) + (2 if case["copy"] else 0)
    return {"bytes": each * sum(_sizes(case)), "flops": 14 * sum(_sizes(case))}


# ---- the definition, in 64 bits --------------------------------------------------------------------


def _exact_scores(case, logits):
    l = logits.double()
    if case["score"] == "sigmoid":
        return torch.sigmoid(l)
    s = torch.softmax(l, 1)
    return torch.where(torch.isnan(s), torch.zeros_like(s), s)        # a row that is barred throughout


def _exact_route(case, logits, bias):
    """An expert's place is the number of experts that come before it."""
    s = _exact_scores(case, logits)
    c = s if bias is None else s + bias.double()
    c = c.masked_fill(logits.double() == -math.inf, -math.inf)
    t, e = c.shape
    g = case["groups"]

    def places(v):
        got = torch.zeros(v.shape, dtype=torch.int64, device=DEV)
        i = torch.arange(v.shape[1], device=DEV)
        step = max(1, (1 << 27) // (v.shape[1] ** 2))
        for a in range(0, v.shape[0], step):
            x = v[a:a + step]
            got[a:a + step] = ((x[:, None, :] > x[:, :, None]) | ((x[:, None, :] == x[:, :, None]) & (i[None, :] < i[:, None]))).sum(2)
        return got
    if g > 1:
        rows = c.view(t * g, e // g)
        first = rows.amax(1)
        score = first.clone()
        if case["best"] == 2 and e // g > 1:
            second = rows.masked_fill(places(rows) == 0, -math.inf).amax(1)
            score = torch.where(second == -math.inf, first, first + second)
        c = c.view(t, g, e // g).masked_fill((places(score.view(t, g)) >= case["top_groups"])[..., None], -math.inf).view(t, e)
    place = places(c)
    experts = torch.full((t, case["top"]), -1, dtype=torch.int64, device=DEV)
    row, col = torch.nonzero((place < case["top"]) & (c > -math.inf), as_tuple=True)
    experts[row, place[row, col]] = col
    w = torch.zeros(t, case["top"], dtype=torch.float64, device=DEV)
    w[row, place[row, col]] = s[row, col]
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return s, experts, w


def _exact_codes(x, u, positive):
    """The code below a magnitude or the one above it, by the fraction and the uniform, over all 127 values."""
    grid = torch.arange(127, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn).double()
    a = x.abs()
    top = a.amax(1, keepdim=True)
    exponent = torch.where(top > 0, torch.floor(torch.log2(top.clamp(min=1e-300))) - 7, -127.0).clamp(min=-127)
    y = a / torch.exp2(exponent)
    low = torch.searchsorted(grid, y, right=True) - 1
    fraction = (y - grid[low]) / (grid[low + 1] - grid[low])
    code = low + (fraction + u.double() / 65536 >= 1)
    if positive:
        code = torch.where(a > 0, code.clamp(min=1), code)
    value = grid[code]
    return torch.where(x < 0, -value, value).view(-1), (exponent + 127).view(-1)


def exact(case, seed):
    got = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("route_fwd", "route_bwd"):
        s, experts, w = _exact_route(case, got["logits"], got["bias"])
        if kind == "route_fwd":
            return {"experts": experts, "weights": w}
        # the derivative of every weight by its own score and by those it shares its sum with, one choice at a time
        dw = got["dweights"].double()
        total = torch.where(experts >= 0, s.gather(1, experts.clamp(min=0)), 0.0).sum(1)
        every = (dw * w).sum(1)
        each = torch.zeros_like(s)
        row = torch.arange(case["tokens"], device=DEV)
        for k in range(case["top"]):
            ok = experts[:, k] >= 0
            d = (dw[:, k] - every) / total if case["renorm"] else dw[:, k]
            each[row[ok], experts[ok, k]] = d[ok]
        if case["score"] == "sigmoid":
            return {"dlogits": each * s * (1 - s)}
        return {"dlogits": each * s - s * (each * s).sum(1, keepdim=True)}
    if kind in ("loss_fwd", "loss_bwd"):
        x, w, y, eps, v = got["x"].double(), got["weights"].double(), got["targets"], case["smoothing"], case["vocab"]
        kept = y >= 0
        z = x @ w.t()
        lse = torch.logsumexp(z, 1)
        row = torch.arange(case["tokens"], device=DEV)
        if kind == "loss_fwd":
            loss = (1 - eps) * (lse - z[row, y.clamp(min=0)]) + eps * (lse - z.sum(1) / v)
            return {"loss": loss * kept, "lse": lse * kept}
        g = z.sub_(lse[:, None]).exp_().sub_(eps / v)
        g[row[kept], y[kept]] -= 1 - eps
        g *= (got["dloss"].double() * kept)[:, None]
        dtable = g.t() @ x
        if case["accumulate"]:
            dtable += got["dtable"].double()
        return {"dx": g @ w, "dtable": dtable}
    blocks = got["place"].numel()
    b1, b2 = BETAS
    t = got["step"].item()
    decay, rate = (torch.tensor(q, device=DEV, dtype=torch.float64)[got["tensor"]][:, None] for q in _decays(case))
    rate = rate * got["lr"].double()
    g, p = got["g"].view(blocks, BLOCK).double(), got["p"].view(blocks, BLOCK).double()
    m, v = got["m"].view(blocks, BLOCK), got["v"].view(blocks, BLOCK)
    if case["bits"] == 8:
        m, v = (c.view(torch.float8_e4m3fn).double() * torch.exp2(got[n].double() - 127)[:, None]
                for c, n in ((m, "m_scale"), (v, "v_scale")))
        v = v * v
    m, v = b1 * m.double() + (1 - b1) * g, b2 * v.double() + (1 - b2) * g * g
    p = p - rate * decay * p - rate * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + ADAM_EPS)
    out = {"p": p.view(-1)}
    if case["bits"] == 32:
        out.update(m=m.view(-1), v=v.view(-1))
    else:
        um, uv = _uniforms(got)
        out["m"], out["m_scale"] = _exact_codes(m, um, False)
        out["v"], out["v_scale"] = _exact_codes(torch.sqrt(v), uv, True)
    if case["copy"]:
        out["copy"] = p.view(-1)
    return out
