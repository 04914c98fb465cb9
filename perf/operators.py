"""A Transformer's operators around the 4-bit products, as measurable cases.

    listed()   the named cases
    draw(rng)  one more case of the same ranges
    prepare    inputs, and the output buffers and workspaces that a program keeps, on the GPU
    run        one pass: the library's calls where `own` is true, else the plain form in torch
    work       the bytes and operations a pass cannot do without
    exact      the outputs in 64 bits, from the definition, without the library

Kinds of case
  embed_fwd   scaled rows of an embedding table; ids below 0 are padding (zero rows)
  embed_grad  the table's gradient: ids grouped by vocabulary entry, rows of the output
              gradient summed by group
  norm_fwd    layer norm with the statistics its backward needs
  norm_bwd    gradients of its input, weight and bias
  moe_fwd     4-bit forward products of rows grouped by expert (ragged groups)
  moe_dgrad   the activation gradient of the same layer: LUQ codes x INT4 weights
  moe_wgrad   its weight gradient, reduced over each expert's rows

Token ids are log-uniform over the vocabulary (a Zipf law with exponent 1: the most
frequent token takes 6 to 10% of them).  Rows per expert follow a power law over the
experts, in an order drawn with the inputs, so that some experts have several times
the mean and, with few rows, many have none.  4-bit codes are drawn directly: INT4 of
normal values, LUQ fields of lognormal magnitudes.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5

# The largest drawn cases: the work of the largest listed ones.
_MAX_MOE = 8192 * 4096 * 16384
_MAX_MOE_WEIGHTS = 8 * 4096 * 16384      # weight elements over all experts
_MAX_NORM = 16384 * 4096
_MAX_EMBED = 65536 * 1024                # looked-up elements
_MAX_TABLE = 50021 * 1024                # table elements


def listed():
    return [
        # one decoding step of a small batch: eight rows of a wide fp32 table
        {"name": "embed_fwd_decode", "kind": "embed_fwd", "tokens": 8, "vocab": 32000, "dim": 4096, "dtype": "f32",
         "ids": "i64", "padding": 0.0},
        # the lookup of a training batch, bf16 activations, an eighth of the positions padding
        {"name": "embed_fwd_batch", "kind": "embed_fwd", "tokens": 16384, "vocab": 50021, "dim": 1024, "dtype": "bf16",
         "ids": "i64", "padding": 0.125},
        # a short fine-tuning batch on an odd-width fp32 table
        {"name": "embed_grad_small", "kind": "embed_grad", "tokens": 509, "vocab": 8000, "dim": 510, "dtype": "f32",
         "ids": "i32", "padding": 0.1},
        # the gradient of a large batch in bf16: frequent tokens appear thousands of times
        {"name": "embed_grad_batch", "kind": "embed_grad", "tokens": 65536, "vocab": 50021, "dim": 1024,
         "dtype": "bf16", "ids": "i64", "padding": 0.0},
        # one token of four sequences in bf16: a single small launch
        {"name": "norm_fwd_decode", "kind": "norm_fwd", "rows": 4, "cols": 4096, "dtype": "bf16"},
        # a batch of the benchmark's model width in fp32
        {"name": "norm_fwd_batch", "kind": "norm_fwd", "rows": 8192, "cols": 4096, "dtype": "f32"},
        # odd sizes: rows that are not 16-byte aligned, fp32 gradients from the products on bf16 activations
        {"name": "norm_bwd_odd", "kind": "norm_bwd", "rows": 3001, "cols": 1001, "dtype": "bf16", "grad": "f32"},
        # the backward of a large batch in bf16
        {"name": "norm_bwd_batch", "kind": "norm_bwd", "rows": 16384, "cols": 4096, "dtype": "bf16", "grad": "bf16"},
        # a decoding step: 16 routed rows over 16 experts whose codes are kept, bound by the weights read
        {"name": "moe_fwd_decode", "kind": "moe_fwd", "rows": 16, "unrouted": 0, "experts": 16, "d_in": 4096,
         "d_out": 4096, "skew": 0.5, "relu": False},
        # the benchmark's MLP layer with its rows spread over eight experts
        {"name": "moe_fwd_mlp", "kind": "moe_fwd", "rows": 8192, "unrouted": 0, "experts": 8, "d_in": 4096,
         "d_out": 16384, "skew": 0.5, "relu": False},
        # many small experts, ragged: the activation gradient of a layer 1024 -> 4096, some rows unrouted
        {"name": "moe_dgrad_ragged", "kind": "moe_dgrad", "rows": 8111, "unrouted": 70, "experts": 64, "d_in": 1024,
         "d_out": 4096, "skew": 1.0, "samples": 1},
        # the weight gradient of two samples (int8 sums) after a ReLU
        {"name": "moe_wgrad_smp", "kind": "moe_wgrad", "rows": 16384, "unrouted": 37, "experts": 16, "d_in": 1024,
         "d_out": 4096, "skew": 0.7, "relu": True, "samples": 2},
    ]


def _log_uniform(rng, lo, hi, step=1):
    """A multiple of step in [lo, hi], spread evenly over its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(max(int(round(v / step)) * step, -(-lo // step) * step), hi // step * step)


def draw(rng):
    kind = rng.choice(["embed_fwd", "embed_grad", "norm_fwd", "norm_bwd", "moe_fwd", "moe_dgrad", "moe_wgrad"])
    dtype = rng.choice(["f32", "bf16"])
    while True:
        if kind in ("embed_fwd", "embed_grad"):
            c = {"kind": kind, "tokens": _log_uniform(rng, 1, 65536), "vocab": _log_uniform(rng, 100, 200000),
                 "dim": _log_uniform(rng, 32, 8192, rng.choice([1, 8, 64])), "dtype": dtype,
                 "ids": rng.choice(["i32", "i64"]), "padding": rng.choice([0.0, 0.0, 0.2])}
            if c["tokens"] * c["dim"] <= _MAX_EMBED and c["vocab"] * c["dim"] <= _MAX_TABLE:
                return c
        elif kind in ("norm_fwd", "norm_bwd"):
            c = {"kind": kind, "rows": _log_uniform(rng, 1, 65536),
                 "cols": _log_uniform(rng, 64, 20000, rng.choice([1, 8, 64])), "dtype": dtype}
            if kind == "norm_bwd":
                c["grad"] = rng.choice(["f32", "bf16"])
            if c["rows"] * c["cols"] <= _MAX_NORM:
                return c
        else:
            rows = _log_uniform(rng, 1, 16384) if kind == "moe_fwd" else _log_uniform(rng, 64, 16384)
            c = {"kind": kind, "rows": rows, "unrouted": rng.choice([0, 0, rows // 50]),
                 "experts": _log_uniform(rng, 2, 128), "d_in": _log_uniform(rng, 256, 8192, 32),
                 "d_out": _log_uniform(rng, 256, 16384, 32), "skew": rng.choice([0.0, 0.5, 1.0])}
            if kind != "moe_dgrad":
                c["relu"] = rng.random() < 0.5
            if kind != "moe_fwd":
                c["samples"] = rng.choice([1, 1, 2])
            if kind == "moe_fwd":       # output widths that are no multiple of a tile; the reduction is whole
                c["d_out"] -= rng.choice([0, 0, 2, 13])
            else:                       # codes are transposed in blocks of eight
                c["d_in"] -= rng.choice([0, 0, 8])
            if (c["rows"] * c["d_in"] * c["d_out"] <= _MAX_MOE
                    and c["experts"] * c["d_in"] * c["d_out"] <= _MAX_MOE_WEIGHTS):
                return c


# ---- inputs ------------------------------------------------------------------------------------


def _loads(case):
    """Rows per expert, most loaded first: a power law over the experts, rounded down, the rest one each."""
    e, routed = case["experts"], case["rows"] - case["unrouted"]
    w = [(i + 1.0) ** -case["skew"] for i in range(e)]
    n = [int(routed * v / sum(w)) for v in w]
    for i in range(routed - sum(n)):
        n[i % e] += 1
    return n


def _padded(case):
    """Rows of the transposed code matrices: whole 16-byte pieces of 32 codes."""
    return -(-case["rows"] // 32) * 32


def _int4_values(shape, signed, gen):
    """Integer codes of normal (signed) or half-normal values whose maximum is about four deviations."""
    v = torch.randn(shape, device=DEV, generator=gen).mul_(7 / 4.0 if signed else 15 / 4.0)
    return v.round_().clamp_(-7, 7).to(torch.int8) if signed else v.abs_().round_().clamp_(0, 15).to(torch.int8)


def _luq_values(shape, samples, gen):
    """Signed fields (0 .. 5) of stochastically rounded lognormal magnitudes, one int8 tensor a sample."""
    level = torch.randn(shape, device=DEV, generator=gen).mul_(3.0 / math.log(2.0)).sub_(2.0)
    sign = torch.where(torch.rand(shape, device=DEV, generator=gen) < 0.5, -1.0, 1.0)
    out = []
    for _ in range(samples):
        u = torch.rand(shape, device=DEV, generator=gen)
        out.append((torch.floor(level + u).clamp_(0, 5) * sign).to(torch.int8))
    return out


def _level(field):
    """Value of a signed field over the scale: 0 or +-2^(field - 1)."""
    mag = torch.exp2(field.abs().float() - 1.0).to(torch.int8)
    return torch.where(field == 0, torch.zeros_like(mag), torch.where(field < 0, -mag, mag))


def _pack(nibbles):
    """Two 4-bit codes a byte along the last axis, the even one in the low half."""
    n = nibbles.to(torch.uint8) & 15
    return (n[..., 0::2] | (n[..., 1::2] << 4)).contiguous()


def _pack_fields(field):
    return _pack(torch.where(field < 0, field.abs() | 8, field))


def _scale(gen, lo, hi, n=1):
    return torch.rand(n, device=DEV, generator=gen) * (hi - lo) + lo


def _inputs(case, seed):
    """The tensors of a case, made from the seed alone."""
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    kind = case["kind"]

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=gen)

    if kind in ("embed_fwd", "embed_grad"):
        n, vocab, dim, dt = case["tokens"], case["vocab"], case["dim"], DTYPES[case["dtype"]]
        u = torch.rand(n, device=DEV, generator=gen, dtype=torch.float64)
        ids = (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1)
        if case["padding"]:
            ids[torch.rand(n, device=DEV, generator=gen) < case["padding"]] = -1
        got = {"ids": ids.to(torch.int32) if case["ids"] == "i32" else ids, "scale": math.sqrt(dim)}
        if kind == "embed_fwd":
            got["table"] = normal(vocab, dim).mul_(0.02).to(dt)
        else:
            got["dout"] = normal(n, dim).mul_(1e-3).to(dt)
        return got
    if kind in ("norm_fwd", "norm_bwd"):
        r, c = case["rows"], case["cols"]
        # rows of different size and offset, a few channels far above the others
        channel = torch.exp(normal(c).mul_(0.5))
        x = (normal(r, c) * channel + 0.5 * normal(r, 1)) * torch.exp(0.5 * normal(r, 1))
        got = {"x": x.to(DTYPES[case["dtype"]]), "gamma": 1.0 + 0.1 * normal(c), "beta": 0.1 * normal(c)}
        if kind == "norm_bwd":
            got["dy"] = normal(r, c).mul_(1e-3).to(DTYPES[case["grad"]])
        return got
    e, k, f = case["experts"], case["d_in"], case["d_out"]
    loads = torch.tensor(_loads(case), device=DEV)[torch.randperm(e, device=DEV, generator=gen)]
    offsets = torch.zeros(e + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = torch.cumsum(loads, 0)
    routed = case["rows"] - case["unrouted"]
    got = {"offsets": offsets}

    def unrouted_zero(v):
        v[routed:] = 0
        return v

    if kind == "moe_fwd":
        got["a"] = unrouted_zero(_int4_values((case["rows"], k), not case["relu"], gen))
        got["w"] = _int4_values((e, f, k), True, gen)
        got["a_scale"], got["w_scale"] = _scale(gen, 0.2, 0.6), _scale(gen, 0.005, 0.02, e)
    elif kind == "moe_dgrad":
        got["g"] = [unrouted_zero(g) for g in _luq_values((case["rows"], f), case["samples"], gen)]
        got["w_t"] = _int4_values((e, k, f), True, gen)
        got["alpha"], got["w_scale"] = _scale(gen, 1e-7, 1e-5), _scale(gen, 0.005, 0.02, e)
    else:
        t = _padded(case)
        got["g"] = [unrouted_zero(g) for g in _luq_values((t, f), case["samples"], gen)]
        got["a"] = unrouted_zero(_int4_values((t, k), not case["relu"], gen))
        got["alpha"], got["a_scale"] = _scale(gen, 1e-7, 1e-5), _scale(gen, 0.2, 0.6)
    return got


def _gradient_codes(fields):
    """Packed codes of one sample, or the int8 sums of two."""
    if len(fields) == 1:
        return _pack_fields(fields[0])
    return (_level(fields[0]) + _level(fields[1])).contiguous()


def _statistics(x):
    x = x.float()
    mean = x.mean(-1, keepdim=True)
    var = ((x - mean) ** 2).mean(-1, keepdim=True)
    return mean.reshape(-1), torch.rsqrt(var + EPS).reshape(-1)


def prepare(case, seed):
    """What a program has in hand before the call: ids, activations, gradients and codes; the statistics that the
    forward kept; and, for the library, the output buffers and workspaces it keeps from step to step."""
    got = _inputs(case, seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("embed_fwd", "embed_grad"):
        s.update(got)
    elif kind in ("norm_fwd", "norm_bwd"):
        s.update(got)
        if kind == "norm_bwd":
            s["mean"], s["rstd"] = _statistics(got["x"])
    else:
        s["offsets"] = got["offsets"]
        s["bounds"] = got["offsets"].tolist()
        for name in ("a_scale", "w_scale", "alpha"):
            if name in got:
                s[name] = got[name]
        if kind == "moe_fwd":
            s["a_codes"], s["w_codes"] = _pack(got["a"]), _pack(got["w"])
        elif kind == "moe_dgrad":
            s["g_codes"], s["w_codes_t"] = _gradient_codes(got["g"]), _pack(got["w_t"])
        else:
            s["g_codes_t"] = _gradient_codes([g.t().contiguous() for g in got["g"]])
            s["a_codes_t"] = _pack(got["a"].t().contiguous())
    if own:
        _prepare_own(case, s)
    return s


def _prepare_own(case, s):
    import paper_2112_10769_amd as L

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    def workspace(*op):
        return empty(max(L.workspace_size(*op), 1), dtype=torch.uint8)

    kind = case["kind"]
    if kind == "embed_fwd":
        s["out"] = empty(case["tokens"], case["dim"], dtype=s["table"].dtype)
    elif kind == "embed_grad":
        n, v, d = case["tokens"], case["vocab"], case["dim"]
        s.update(order=empty(n, dtype=torch.int32), offsets=empty(v + 1, dtype=torch.int32), dtable=empty(v, d),
                 ws_group=workspace(L.OP_GROUP_IDS, n, v), ws=workspace(L.OP_EMBEDDING_GRAD, n, d))
    elif kind == "norm_fwd":
        s.update(y=torch.empty_like(s["x"]), mean=empty(case["rows"]), rstd=empty(case["rows"]))
    elif kind == "norm_bwd":
        r, c = case["rows"], case["cols"]
        s.update(dx=torch.empty_like(s["dy"]), dgamma=empty(c), dbeta=empty(c), ws=workspace(L.OP_LAYERNORM_BWD, r, c))
    elif kind == "moe_fwd":
        s.update(y=empty(case["rows"], case["d_out"]))
    elif kind == "moe_dgrad":
        s.update(dx=empty(case["rows"], case["d_in"]))
    else:
        t, e, f, k = _padded(case), case["experts"], case["d_out"], case["d_in"]
        s.update(dw=empty(e, f, k),
                 ws=empty(max(L.grouped_wgrad_workspace(t, f, k, e), 1), dtype=torch.uint8))


# ---- one pass ----------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)(s["case"], s)


def _run_own(case, s):
    import paper_2112_10769_amd as L

    kind = case["kind"]
    if kind == "embed_fwd":
        return {"out": L.luq_embedding_fwd(s["ids"], s["table"], s["scale"], out=s["out"])}
    if kind == "embed_grad":
        L.luq_group_ids(s["ids"], case["vocab"], s["order"], s["offsets"], s["ws_group"])
        L.luq_embedding_grad(s["dout"], s["ids"], s["order"], s["offsets"], s["scale"], dtable=s["dtable"], ws=s["ws"])
        return {"order": s["order"], "offsets": s["offsets"], "dtable": s["dtable"]}
    if kind == "norm_fwd":
        L.luq_layernorm_fwd(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if kind == "norm_bwd":
        L.luq_layernorm_bwd(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], s["dx"], s["dgamma"], s["dbeta"], s["ws"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    k, f = case["d_in"], case["d_out"]
    if kind == "moe_fwd":
        return {"y": L.int4_gemm_fwd_grouped(s["a_codes"], s["a_scale"], not case["relu"], s["w_codes"], s["w_scale"],
                                             True, s["offsets"], case["rows"], f, k, y=s["y"])}
    n = L.SMP_SUM | 2 if case["samples"] == 2 else 1
    if kind == "moe_dgrad":
        return {"dx": L.luq_gemm_dgrad_grouped(s["g_codes"], s["alpha"], s["w_codes_t"], s["w_scale"], True,
                                               s["offsets"], case["rows"], k, f, n, dx=s["dx"])}
    return {"dw": L.luq_gemm_wgrad_grouped(s["g_codes_t"], s["alpha"], s["a_codes_t"], s["a_scale"], not case["relu"],
                                           s["offsets"], _padded(case), f, k, n, dw=s["dw"], ws=s["ws"])}


def _nibbles(codes):
    """[..., n / 2] bytes -> [..., n] codes 0 .. 15."""
    return torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])


def _decode_int4(codes, signed):
    v = _nibbles(codes).float()
    return torch.where(v > 7, v - 16, v) if signed else v


def _decode_gradient(codes, samples):
    """Gradient codes over alpha, in fp32: one sample's levels, or the average of two."""
    if samples == 2:
        return codes.float() * 0.5
    n = _nibbles(codes)
    mag = torch.exp2((n & 7).float() - 1.0)
    return torch.where(n == 0, torch.zeros_like(mag), torch.where(n > 7, -mag, mag))


def _run_plain(case, s):
    kind = case["kind"]
    if kind == "embed_fwd":
        rows = s["table"][s["ids"].long().clamp(min=0)].float() * s["scale"]
        return {"out": torch.where((s["ids"] < 0)[:, None], torch.zeros_like(rows), rows).to(s["table"].dtype)}
    if kind == "embed_grad":
        v = case["vocab"]
        key = torch.where(s["ids"] < 0, torch.full_like(s["ids"], v), s["ids"]).long()
        key_sorted, order = torch.sort(key, stable=True)
        offsets = torch.searchsorted(key_sorted, torch.arange(v + 1, device=key.device))
        dtable = torch.zeros(v + 1, case["dim"], device=key.device)
        dtable.index_add_(0, key, s["dout"].float() * s["scale"])
        return {"order": order.to(torch.int32), "offsets": offsets.to(torch.int32), "dtable": dtable[:v]}
    if kind == "norm_fwd":
        mean, rstd = _statistics(s["x"])
        y = (s["x"].float() - mean[:, None]) * rstd[:, None] * s["gamma"] + s["beta"]
        return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
    if kind == "norm_bwd":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xh = (s["x"].float() - s["mean"][:, None]) * rstd
        a = dy * s["gamma"]
        dx = rstd * (a - a.mean(-1, keepdim=True) - xh * (a * xh).mean(-1, keepdim=True))
        return {"dx": dx.to(s["dy"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    b, e, k, f = s["bounds"], case["experts"], case["d_in"], case["d_out"]
    if kind == "moe_wgrad":
        g = _decode_gradient(s["g_codes_t"], case["samples"])
        a = _decode_int4(s["a_codes_t"], not case["relu"])
        dw = torch.zeros(e, f, k, device=g.device)
        for i in range(e):
            if b[i] < b[i + 1]:
                dw[i] = (g[:, b[i]:b[i + 1]] @ a[:, b[i]:b[i + 1]].t()) * (s["alpha"] * s["a_scale"])
        return {"dw": dw}
    if kind == "moe_fwd":
        x, codes, signed, scale = _decode_int4(s["a_codes"], not case["relu"]), s["w_codes"], True, s["a_scale"]
    else:
        x, codes, signed, scale = _decode_gradient(s["g_codes"], case["samples"]), s["w_codes_t"], True, s["alpha"]
    y = torch.zeros(case["rows"], codes.shape[1], device=x.device)
    for i in range(e):
        if b[i] < b[i + 1]:
            y[b[i]:b[i + 1]] = (x[b[i]:b[i + 1]] @ _decode_int4(codes[i], signed).t()) * (scale * s["w_scale"][i])
    return {"y" if kind == "moe_fwd" else "dx": y}


# ---- what a pass cannot do without ---------------------------------------------------------------


def _distinct(case):
    """Expected number of different ids among the tokens."""
    v = torch.arange(case["vocab"], dtype=torch.float64)
    p = torch.log((v + 2.0) / (v + 1.0)) / math.log(case["vocab"] + 1.0)
    return float((1.0 - torch.pow(1.0 - p, case["tokens"] * (1.0 - case["padding"]))).sum())


def work(case):
    """Inputs read once, outputs written once; additions and multiplications."""
    kind = case["kind"]
    if kind in ("embed_fwd", "embed_grad"):
        n, v, d = case["tokens"], case["vocab"], case["dim"]
        e = 4 if case["dtype"] == "f32" else 2
        i = 4 if case["ids"] == "i32" else 8
        if kind == "embed_fwd":
            return {"bytes": n * i + n * d * e + _distinct(case) * d * e, "flops": n * d}
        read = n * (1.0 - case["padding"])
        return {"bytes": n * (i + 4) + 4 * (v + 1) + read * d * e + 4 * v * d, "flops": 2 * read * d}
    if kind in ("norm_fwd", "norm_bwd"):
        r, c = case["rows"], case["cols"]
        e = 4 if case["dtype"] == "f32" else 2
        if kind == "norm_fwd":
            return {"bytes": 2 * r * c * e + 8 * r + 8 * c, "flops": 8 * r * c}
        g = 4 if case["grad"] == "f32" else 2
        return {"bytes": r * c * (e + 2 * g) + 8 * r + 12 * c, "flops": 14 * r * c}
    loads = _loads(case)
    t, e, k, f, routed = case["rows"], case["experts"], case["d_in"], case["d_out"], sum(loads)
    weights = sum(1 for n in loads if n) * k * f / 2
    g = 1.0 if case.get("samples") == 2 else 0.5
    flops = 2 * routed * k * f
    if kind == "moe_fwd":
        return {"bytes": routed * k / 2 + weights + 4 * t * f + 4 * (2 * e + 1), "flops": flops}
    if kind == "moe_dgrad":
        return {"bytes": routed * f * g + weights + 4 * t * k + 4 * (2 * e + 1), "flops": flops}
    return {"bytes": routed * (f * g + k / 2) + 4 * e * k * f + 4 * (e + 1), "flops": flops}


# ---- the definition, in 64 bits --------------------------------------------------------------------


def exact(case, seed):
    got = _inputs(case, seed)
    kind = case["kind"]
    if kind == "embed_fwd":
        out = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device=DEV)
        valid = got["ids"] >= 0
        out[valid] = got["table"].index_select(0, got["ids"][valid].long()).double() * got["scale"]
        return {"out": out}
    if kind == "embed_grad":
        ids, v = got["ids"].long(), case["vocab"]
        pos = torch.arange(ids.numel(), device=DEV)
        valid = ids >= 0
        key = torch.where(valid, ids, torch.full_like(ids, v)) * ids.numel() + pos     # unique: any sort is stable
        order = torch.sort(key)[1].to(torch.int32)
        offsets = torch.zeros(v + 1, dtype=torch.int32, device=DEV)
        offsets[1:] = torch.cumsum(torch.bincount(ids[valid], minlength=v), 0)
        dtable = torch.zeros(v, case["dim"], dtype=torch.float64, device=DEV)
        dtable.index_add_(0, ids[valid], got["dout"][valid].double())
        return {"order": order, "offsets": offsets, "dtable": dtable * got["scale"]}
    if kind in ("norm_fwd", "norm_bwd"):
        x, gamma = got["x"].double(), got["gamma"].double()
        mean = x.sum(1) / case["cols"]
        d = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((d * d).sum(1) / case["cols"] + EPS)
        xh = d * rstd[:, None]
        if kind == "norm_fwd":
            return {"y": xh * gamma + got["beta"].double(), "mean": mean, "rstd": rstd}
        dy = got["dy"].double()
        a = dy * gamma
        m1, m2 = a.sum(1) / case["cols"], (a * xh).sum(1) / case["cols"]
        return {"dx": (a - m1[:, None] - xh * m2[:, None]) * rstd[:, None], "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    bounds = got["offsets"].tolist()
    e, k, f = case["experts"], case["d_in"], case["d_out"]
    if "g" in got:
        # levels as float64, averaged over the samples
        g = sum(torch.sign(v).double() * torch.floor(torch.exp2(v.double().abs() - 1.0)) for v in got["g"])
        g *= got["alpha"].double() / len(got["g"])
    if kind == "moe_wgrad":
        out = torch.zeros(e, f, k, dtype=torch.float64, device=DEV)
        a = got["a"].double() * got["a_scale"].double()
        for i, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
            out[i] = g[lo:hi].t().contiguous() @ a[lo:hi]
        return {"dw": out}
    x = got["a"].double() * got["a_scale"].double() if kind == "moe_fwd" else g
    w = got["w"] if kind == "moe_fwd" else got["w_t"]
    out = torch.zeros(case["rows"], w.shape[1], dtype=torch.float64, device=DEV)
    for i, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
        if lo < hi:
            out[lo:hi] = x[lo:hi] @ (w[i].double() * got["w_scale"][i].double()).t().contiguous()
    return {"y" if kind == "moe_fwd" else "dx": out}
