"""What stands around and inside a served or trained layer, as timed cases.

Five kinds of case, each one pass through the binding's public calls:

* ``norm``: the end of one block and the start of the next: the block's output is normalised, gated,
  scaled and added to the residual stream, and the sum normalised for what follows;
* ``norm_train``: the same forward and backward, a training step's share of it;
* ``linear_f4``: a projection with 4-bit weights (signed 0, 0.5, 1, 1.5, 2, 3, 4, 6, two to a byte, and a
  power of two per 32 of them along the contraction);
* ``ffn_f4``: the dense gated feed-forward block with such weights;
* ``moe_few``: the whole mixture-of-experts layer (router, elbow routing, experts, weighted sum) for
  a few tokens, its experts in bf16 or in 4 bits.

Activations are N(0, 1), weights N(0, 0.02), norm weights and gates N(1, 0.1), gradients N(0, 1e-3).
Where ``own`` is false the same values are computed with elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6          # of the norms
ROUTE_EPS = 1e-8    # of the routing's normalised curve


def _norm(name, T, d, gate, dtype="bf16", kind="norm", residual_scale=1.0, block_scale=1.0):
    return {"name": name, "kind": kind, "T": T, "d": d, "gate": gate, "dtype": dtype,
            "residual_scale": residual_scale, "block_scale": block_scale}


def _linear(name, T, k, n, dtype="bf16"):
    return {"name": name, "kind": "linear_f4", "T": T, "k": k, "n": n, "dtype": dtype}


def _ffn(name, T, d, m, dtype="bf16", residual=False):
    return {"name": name, "kind": "ffn_f4", "T": T, "d": d, "m": m, "dtype": dtype,
            "residual": residual}


def _moe(name, T, d, N, m, K, weights, renormalize=False):
    return {"name": name, "kind": "moe_few", "T": T, "d": d, "N": N, "m": m, "K": K,
            "weights": weights, "renormalize": renormalize, "dtype": "bf16"}


def listed():
    return [
        # between two layers while one sequence generates a token
        _norm("norm_decode_1", 1, 2048, "channel"),
        # a prefill batch of the stacked layers, the block's output gated value by value
        _norm("norm_16384_gated", 16384, 2048, "full", residual_scale=0.5, block_scale=1.5),
        # a training step on a small fp32 model, a ragged batch, one gate a token
        _norm("norm_train_f32_1500", 1500, 1024, "token", "f32", "norm_train"),
        # a training step at the batch of a prefill layer, one learned gate a channel
        _norm("norm_train_4096", 4096, 2048, "channel", kind="norm_train", block_scale=0.25),
        # one generated token through a wide block's down projection
        _linear("linear_f4_decode_1", 1, 8192, 2048),
        # an fp32 model's projection on a ragged batch, odd sizes
        _linear("linear_f4_f32_300", 300, 1056, 528, "f32"),
        # a prefill batch through the wide down projection: the largest call
        _linear("linear_f4_4096_wide", 4096, 8192, 2048),
        # one token through the shared expert beside the routed ones
        _ffn("ffn_f4_decode_1", 1, 2048, 1024, residual=True),
        # a serving batch's step through a wide dense block
        _ffn("ffn_f4_decode_48_wide", 48, 2048, 8192),
        # one sequence generating a token through the layer
        _moe("moe_few_1", 1, 2048, 64, 1024, 8, "bf16"),
        # the same, its experts held in 4 bits
        _moe("moe_few_1_f4", 1, 2048, 64, 1024, 8, "f4"),
        # a step of a small serving batch, weights renormalised over the selected experts
        _moe("moe_few_13_f4", 13, 2048, 64, 1024, 8, "f4", renormalize=True),
    ]


_LARGEST = 4096 * 8192 * 2048     # multiply-adds of the largest product
_LARGEST_ROWS = 16384 * 2048      # values of the largest residual stream


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "linear_f4", "ffn_f4", "moe_few"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("norm", "norm_train"):
        d = 16 * _log_int(rng, 4, 512)
        T = min(_log_int(rng, 1, 65536), _LARGEST_ROWS // d // (2 if dtype == "f32" else 1))
        c = _norm(None, T, d, rng.choice(["none", "channel", "token", "full"]), dtype, kind,
                  rng.choice([1.0, 0.5]), rng.choice([1.0, 0.25]))
    elif kind == "linear_f4":
        k, n = 32 * _log_int(rng, 2, 256), 16 * _log_int(rng, 2, 512)
        top = _LARGEST // (k * n) // (16 if dtype == "f32" else 1)
        c = _linear(None, max(1, min(_log_int(rng, 1, 8192), top)), k, n, dtype)
    elif kind == "ffn_f4":
        d, m = 32 * _log_int(rng, 2, 96), 32 * _log_int(rng, 2, 256)
        top = _LARGEST // (3 * d * m) // (16 if dtype == "f32" else 1)
        c = _ffn(None, max(1, min(_log_int(rng, 1, 4096), top)), d, m, dtype, rng.random() < 0.5)
    else:
        N = rng.choice([8, 16, 24, 32, 64])
        d, m = 64 * _log_int(rng, 2, 32), 64 * _log_int(rng, 1, 16)
        c = _moe(None, rng.randint(1, 16), d, N, m, rng.randint(1, 8), rng.choice(["bf16", "f4"]),
                 rng.random() < 0.5)
    del c["name"]
    return c


def _normal(gen, shape, std, dtype, mean=0.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)


_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _weights_f4(gen, shape):
    """Weights [..., k] as a checkpoint in 4 bits holds them: [..., k / 2] bytes, the earlier value
    in the low half, and [..., k / 32] exponents e of scales 2^(e - 127): the least power of two by
    which a group's largest value is at most 6."""
    w = torch.randn(shape, generator=gen, device="cuda") * 0.02
    g = w.view(shape[:-1] + (shape[-1] // 32, 32))
    mantissa, exponent = torch.frexp(g.abs().amax(-1) / 6)
    e = exponent - (mantissa == 0.5).int()
    v = g / torch.exp2(e.float())[..., None]
    cuts = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")
    code = torch.bucketize(v.abs(), cuts, out_int32=True).to(torch.uint8) + 8 * (v < 0).to(torch.uint8)
    code = code.view(shape)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _routing(logits, K):
    """(probabilities in falling order, expert ids, k) of logits [T, N] in 64 bits: k ends at the
    elbow, the point of the normalised curve furthest below its chord."""
    p, ids = torch.softmax(logits, -1).sort(dim=-1, descending=True, stable=True)
    N = p.shape[1]
    curve = (p[:, :1] - p) / (p[:, :1] - p[:, -1:] + ROUTE_EPS)
    depth = curve - torch.arange(N, device=p.device, dtype=p.dtype) / (N - 1)
    return p, ids, (depth.argmax(-1) + 1).clamp(max=K), depth


def _clear_tokens(gen, T, router, K):
    """T tokens whose routing does not hang on the last bits of their logits: no two of the first
    K + 1 logits, and no two points for the elbow, within 1e-4 of each other."""
    x = _normal(gen, (8 * T + 64, router.shape[1]), 1.0, router.dtype)
    logits = x.double() @ router.double().t()
    top = logits.sort(-1, descending=True).values[:, :min(K + 1, router.shape[0])]
    deep = _routing(logits, K)[3].sort(-1, descending=True).values
    clear = ((top[:, :-1] - top[:, 1:]).amin(-1) > 1e-4) & (deep[:, 0] - deep[:, 1] > 1e-4)
    return x[clear][:T].contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    T, kind = case["T"], case["kind"]
    s = {"case": case}
    if kind in ("norm", "norm_train"):
        d = case["d"]
        s["residual"], s["block"] = (_normal(gen, (T, d), 1.0, dt) for _ in range(2))
        s["w_post"], s["w_pre"] = (_normal(gen, (d,), 0.1, dt, 1.0) for _ in range(2))
        shape = {"none": None, "channel": (d,), "token": (T, 1), "full": (T, d)}[case["gate"]]
        s["gate"] = None if shape is None else _normal(gen, shape, 0.1, dt, 1.0)
        if kind == "norm_train":
            s["ds"], s["dn"] = (_normal(gen, (T, d), 1e-3, dt) for _ in range(2))
        return s
    if kind == "linear_f4":
        s["x"] = _normal(gen, (T, case["k"]), 1.0, dt)
        s["w"], s["w_scale"] = _weights_f4(gen, (case["n"], case["k"]))
        return s
    d, m = case["d"], case["m"]
    if kind == "ffn_f4":
        s["x"] = _normal(gen, (T, d), 1.0, dt)
        s["residual"] = _normal(gen, (T, d), 1.0, dt) if case["residual"] else None
        s["gate_up"], s["gate_up_scale"] = _weights_f4(gen, (2 * m, d))
        s["down"], s["down_scale"] = _weights_f4(gen, (d, m))
        return s
    N = case["N"]
    s["router"] = _normal(gen, (N, d), 0.02, dt)
    s["x"] = _clear_tokens(gen, T, s["router"], case["K"])
    s["residual"] = _normal(gen, (T, d), 1.0, dt)
    s["gate_up_scale"] = s["down_scale"] = None
    if case["weights"] == "f4":
        s["gate_up"], s["gate_up_scale"] = _weights_f4(gen, (N, 2 * m, d))
        s["down"], s["down_scale"] = _weights_f4(gen, (N, d, m))
    else:
        s["gate_up"] = _normal(gen, (N, 2 * m, d), 0.02, dt)
        s["down"] = _normal(gen, (N, d, m), 0.02, dt)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2608_04401_amd import binding as B
    case = s["case"]
    kind = case["kind"]
    if kind in ("norm", "norm_train"):
        with_ = {"w_post": s["w_post"], "w_pre": s["w_pre"], "gate": s["gate"],
                 "residual_scale": case["residual_scale"], "block_scale": case["block_scale"]}
        if kind == "norm":
            return B.elb_norm_forward(s["residual"], s["block"], eps=EPS, **with_)
        total, n, kept = B.elb_norm_forward(s["residual"], s["block"], eps=EPS, keep=True, **with_)
        grads = B.elb_norm_backward(s["ds"], s["dn"], total, s["block"], kept, **with_)
        return (total, n) + tuple(g for g in grads if g is not None)
    if kind == "linear_f4":
        return B.elb_linear_f4(s["x"], s["w"], s["w_scale"])
    if kind == "ffn_f4":
        return B.elb_ffn_forward_f4(s["x"], s["gate_up"], s["gate_up_scale"], s["down"],
                                    s["down_scale"], residual=s["residual"])
    return B.elb_moe_forward_few(s["x"], s["router"], s["gate_up"], s["down"], K=case["K"],
                                 eps=ROUTE_EPS, renormalize=case["renormalize"],
                                 residual=s["residual"], gate_up_scale=s["gate_up_scale"],
                                 down_scale=s["down_scale"])


def _from_f4(q, scale):
    """The weights that 4-bit ones stand for, in float32."""
    values = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=q.device)
    w = values[torch.stack([q & 15, q >> 4], -1).int()].view(q.shape[:-1] + (-1, 32))
    return (w * torch.exp2(scale.float() - 127)[..., None]).view(q.shape[:-1] + (-1,))


def _swiglu(a):
    g, u = a.chunk(2, -1)
    return g / (1 + (-g).exp()) * u


def _run_norm_plain(s):
    case = s["case"]
    alpha, beta = case["residual_scale"], case["block_scale"]
    b, w_post, w_pre = s["block"].float(), s["w_post"].float(), s["w_pre"].float()
    gate = torch.ones((), device=b.device) if s["gate"] is None else s["gate"].float()
    r_b = (b.square().mean(-1, keepdim=True) + EPS).rsqrt()
    b_hat = b * r_b
    p = w_post * b_hat
    total = alpha * s["residual"].float() + beta * gate * p
    r_s = (total.square().mean(-1, keepdim=True) + EPS).rsqrt()
    s_hat = total * r_s
    out = [total, w_pre * s_hat]
    if case["kind"] == "norm_train":
        dn = s["dn"].float()
        t = w_pre * dn
        ds = s["ds"].float() + r_s * (t - s_hat * (t * s_hat).mean(-1, keepdim=True))
        q = beta * ds
        dp = q * gate
        t = w_post * dp
        out += [alpha * ds, r_b * (t - b_hat * (t * b_hat).mean(-1, keepdim=True))]
        if case["gate"] == "full":
            out.append(q * p)
        elif case["gate"] == "token":
            out.append((q * p).sum(-1, keepdim=True))
        elif case["gate"] == "channel":
            out.append((q * p).sum(0, dtype=torch.float64))
        out += [(dp * b_hat).sum(0, dtype=torch.float64), (dn * s_hat).sum(0, dtype=torch.float64)]
    return tuple(o.to(s["block"].dtype) for o in out)


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind in ("norm", "norm_train"):
        return _run_norm_plain(s)
    x = s["x"].float()
    if kind == "linear_f4":
        return (x @ _from_f4(s["w"], s["w_scale"]).t()).to(s["x"].dtype)
    if s["gate_up_scale"] is None:
        gate_up, down = s["gate_up"].float(), s["down"].float()
    else:
        gate_up = _from_f4(s["gate_up"], s["gate_up_scale"])
        down = _from_f4(s["down"], s["down_scale"])
    if kind == "ffn_f4":
        y = _swiglu(x @ gate_up.t()) @ down.t()
    else:
        T, d, N, m, K = x.shape[0], case["d"], case["N"], case["m"], case["K"]
        p, ids, k, _ = _routing(s["x"].double() @ s["router"].double().t(), K)
        p = torch.where(torch.arange(N, device=x.device) < k[:, None], p, 0.0)
        if case["renormalize"]:
            p = p / p.sum(-1, keepdim=True)
        w = torch.zeros_like(p).scatter(1, ids, p).float()
        h = _swiglu((x @ gate_up.view(-1, d).t()).view(T, N, 2 * m)) * w[:, :, None]
        y = h.view(T, N * m) @ down.permute(0, 2, 1).reshape(N * m, d)
    return (y if s["residual"] is None else y + s["residual"].float()).to(s["x"].dtype)


def work(case):
    T, size, kind = case["T"], 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind in ("norm", "norm_train"):
        d = case["d"]
        gate = {"none": 0, "channel": d, "token": T, "full": T * d}[case["gate"]]
        if kind == "norm":  # residual, block, gate and weights in; the sum and its norm out
            return {"bytes": size * (4 * T * d + gate + 2 * d), "flops": 12.0 * T * d}
        # beside them two gradients in, those of residual, block, gate and weights out
        return {"bytes": size * (8 * T * d + 2 * gate + 4 * d), "flops": 40.0 * T * d}
    if kind == "linear_f4":
        k, n = case["k"], case["n"]
        return {"bytes": size * T * (k + n) + n * k * 17 // 32, "flops": 2.0 * T * n * k}
    d, m = case["d"], case["m"]
    if kind == "ffn_f4":
        rows = T * d * (3 if case["residual"] else 2)
        return {"bytes": size * rows + 3 * d * m * 17 // 32, "flops": 6.0 * T * d * m}
    # the experts that T tokens of K different ones each meet, were all as likely
    N, K = case["N"], case["K"]
    met = N * (1 - (1 - K / N) ** T)
    each = 3 * d * m * (2 if case["weights"] == "bf16" else 17 / 32)
    return {"bytes": int(met * each) + 2 * N * d + 2 * 3 * T * d,
            "flops": 2.0 * T * N * d + 6.0 * T * K * d * m}


def _decoded(q, scale):
    """4-bit weights in 64 bits, from sign, exponent and last bit of each."""
    code = torch.stack((q.bitwise_and(15), q.div(16, rounding_mode="floor")), dim=-1).flatten(-2)
    exponent, last = code.div(2, rounding_mode="floor") % 4, (code % 2).double()
    size = torch.where(exponent == 0, last / 2, torch.ldexp(1 + last / 2, exponent.int() - 1))
    w = torch.where(code >= 8, -size, size)
    return torch.ldexp(w, (scale.int() - 127).repeat_interleave(32, dim=-1))


def _exact_norm(s):
    case = s["case"]
    names = ["residual", "block"] + (["gate"] if s["gate"] is not None else []) + ["w_post", "w_pre"]
    leaf = {n: s[n].double().requires_grad_(True) for n in names}

    def normed(v, w):
        return v / torch.sqrt(torch.mean(v * v, dim=-1, keepdim=True) + EPS) * w

    add = normed(leaf["block"], leaf["w_post"]) * case["block_scale"]
    if "gate" in leaf:
        add = add * leaf["gate"]
    total = leaf["residual"] * case["residual_scale"] + add
    n = normed(total, leaf["w_pre"])
    out = (total.detach(), n.detach())
    if case["kind"] == "norm":
        return out
    return out + torch.autograd.grad((total, n), [leaf[k] for k in names],
                                     (s["ds"].double(), s["dn"].double()))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("norm", "norm_train"):
        return _exact_norm(s)
    x = s["x"].double()
    if case["kind"] == "linear_f4":
        return torch.matmul(x, _decoded(s["w"], s["w_scale"]).T)
    y = torch.zeros_like(x) if s["residual"] is None else s["residual"].double()

    def expert(rows, e):
        at = (lambda k: s[k]) if e is None else (lambda k: None if s[k] is None else s[k][e])
        if at("gate_up_scale") is None:
            gate_up, down = at("gate_up").double(), at("down").double()
        else:
            gate_up = _decoded(at("gate_up"), at("gate_up_scale"))
            down = _decoded(at("down"), at("down_scale"))
        gate, up = torch.matmul(rows, gate_up.T).split(case["m"], dim=-1)
        return torch.matmul(torch.nn.functional.silu(gate) * up, down.T)

    if case["kind"] == "ffn_f4":
        return y + expert(x, None)
    logits = torch.matmul(x, s["router"].double().T).cpu().numpy()
    for t, row in enumerate(logits):
        order = np.argsort(-row, kind="stable")
        p = np.exp(row[order] - row.max())
        p /= p.sum()
        depth = (p[0] - p) / (p[0] - p[-1] + ROUTE_EPS) - np.linspace(0, 1, len(p))
        k = min(int(np.argmax(depth)) + 1, case["K"])
        share = p[:k] / p[:k].sum() if case["renormalize"] else p[:k]
        for e, w in zip(order[:k], share):
            y[t] += float(w) * expert(x[t:t + 1], int(e))[0]
    return y
