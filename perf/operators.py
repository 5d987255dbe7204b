"""The dense gated feed-forward block and the 8-bit products as timed cases.

Four kinds of case, each one pass through the binding's public calls:

* ``ffn``: the block's forward pass y = [residual +] (silu(x Wg^T) * (x Wu^T)) Wd^T, as the
  expert that every token goes through beside the routed ones, or as a wide dense block;
* ``train``: forward and backward, a training step's share of the block: y and the gradients
  of x and of both weight tensors;
* ``linear_i8``: a projection served with int8 weights: the tokens are quantised on the way, one
  scale per token, one per output channel of the weights;
* ``ffn_i8``: the block of the first kind served with int8 weights.

Activations are N(0, 1), for the 8-bit cases with a few channels eight times as large, weights
N(0, 0.02), gradients N(0, 1e-3).  Where ``own`` is false the same values are computed with
elementary torch operations.
"""
import math

import torch

own = False


def _ffn(name, T, d, m, dtype="bf16", residual=False):
    return {"name": name, "kind": "ffn", "T": T, "d": d, "m": m, "dtype": dtype,
            "residual": residual}


def _train(name, T, d, m, dtype="bf16"):
    return {"name": name, "kind": "train", "T": T, "d": d, "m": m, "dtype": dtype,
            "residual": False}


def _linear(name, T, k, n, dtype="bf16"):
    return {"name": name, "kind": "linear_i8", "T": T, "k": k, "n": n, "dtype": dtype}


def _ffn_i8(name, T, d, m, residual=False):
    return {"name": name, "kind": "ffn_i8", "T": T, "d": d, "m": m, "dtype": "bf16",
            "residual": residual}


def listed():
    return [
        # one sequence generating a token: the shared expert's output added to the routed experts'
        _ffn("ffn_decode_1", 1, 2048, 1024, residual=True),
        # a ragged prompt batch through a shared expert of the layer's own expert size
        _ffn("ffn_ragged_1777", 1777, 2048, 1024, residual=True),
        # a prefill batch through a wide dense block (four times the model's width)
        _ffn("ffn_prefill_4096_wide", 4096, 2048, 8192),
        # a small fp32 model's block, with the odd sizes of the fp32 layer
        _ffn("ffn_f32_1500", 1500, 1024, 528, dtype="f32", residual=True),
        # a training step on the tiny fp32 layer of the tests
        _train("train_f32_tiny_256", 256, 128, 256, dtype="f32"),
        # a training step of the shared expert on a ragged batch
        _train("train_1777", 1777, 2048, 1024),
        # a training step of the wide block at the batch of a prefill layer: the largest call
        _train("train_4096_wide", 4096, 2048, 8192),
        # a decode step of a serving batch through one int8 projection
        _linear("linear_i8_decode_40", 40, 2048, 2048),
        # an fp32 model's projection with int8 weights, odd sizes
        _linear("linear_i8_f32_300", 300, 1040, 528, dtype="f32"),
        # a large prompt batch through the wide block's down projection
        _linear("linear_i8_16384_wide", 16384, 8192, 2048),
        # one token through the int8 block
        _ffn_i8("ffn_i8_decode_1", 1, 2048, 1024, residual=True),
        # a prefill batch through the wide int8 block
        _ffn_i8("ffn_i8_prefill_4096_wide", 4096, 2048, 8192),
    ]


_LARGEST = 4096 * 2048 * 8192


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["ffn", "ffn", "train", "train", "linear_i8", "ffn_i8"])
    T = _log_int(rng, 1, 16384)
    if kind == "linear_i8":
        c = _linear(None, T, 16 * _log_int(rng, 8, 512), 16 * _log_int(rng, 4, 512),
                    rng.choice(["bf16", "bf16", "f32"]))
        c["T"] = max(1, min(T, 16384 * 8192 * 2048 // (c["k"] * c["n"])))
    else:
        f32 = kind != "ffn_i8" and rng.random() < 0.25
        d = 16 * _log_int(rng, 8, 256)
        m = 16 * _log_int(rng, 4, 512)
        top = _LARGEST // (d * m)
        if f32:  # small layers
            d, m, top = 16 * _log_int(rng, 8, 64), 16 * _log_int(rng, 4, 64), 2048
        T = max(1, min(T, top))
        if kind == "train":
            c = _train(None, T, d, m, "f32" if f32 else "bf16")
        elif kind == "ffn":
            c = _ffn(None, T, d, m, "f32" if f32 else "bf16", rng.random() < 0.5)
        else:
            c = _ffn_i8(None, T, d, m, rng.random() < 0.5)
    del c["name"]
    return c


def _normal(gen, shape, std, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _outliers(gen, x):
    """One channel in sixty-four eight times as large, as activations have them."""
    big = torch.rand(x.shape[1], generator=gen, device="cuda") < 1 / 64
    return torch.where(big, x * 8, x)


def _int8_weights(gen, n, k):
    """Weights [n, k] as a checkpoint in int8 holds them: values and a scale per channel."""
    w = torch.randn((n, k), generator=gen, device="cuda") * 0.02
    scale = w.abs().amax(1) / 127
    return (w / scale[:, None]).round().clamp(-127, 127).to(torch.int8), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    T = case["T"]
    s = {"case": case}
    if case["kind"] == "linear_i8":
        s["x"] = _outliers(gen, _normal(gen, (T, case["k"]), 1.0, dt))
        s["w"], s["w_scale"] = _int8_weights(gen, case["n"], case["k"])
        return s
    d, m = case["d"], case["m"]
    s["x"] = _normal(gen, (T, d), 1.0, dt)
    s["residual"] = _normal(gen, (T, d), 1.0, dt) if case["residual"] else None
    if case["kind"] == "ffn_i8":
        s["x"] = _outliers(gen, s["x"])
        s["gate_up"], s["gate_up_scale"] = _int8_weights(gen, 2 * m, d)
        s["down"], s["down_scale"] = _int8_weights(gen, d, m)
        return s
    s["gate_up"] = _normal(gen, (2 * m, d), 0.02, dt)
    s["down"] = _normal(gen, (d, m), 0.02, dt)
    if case["kind"] == "train":
        s["dy"] = _normal(gen, (T, d), 1e-3, dt)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2608_04401_amd import binding as B
    kind = s["case"]["kind"]
    if kind == "ffn":
        return B.elb_ffn_forward(s["x"], s["gate_up"], s["down"], residual=s["residual"])
    if kind == "train":
        y, kept = B.elb_ffn_forward(s["x"], s["gate_up"], s["down"], keep=True)
        return (y,) + tuple(B.elb_ffn_backward(s["dy"], s["x"], s["gate_up"], s["down"], kept))
    if kind == "linear_i8":
        return B.elb_linear_i8(s["x"], s["w"], s["w_scale"])
    return B.elb_ffn_forward_i8(s["x"], s["gate_up"], s["gate_up_scale"], s["down"],
                                s["down_scale"], residual=s["residual"])


def _quantised(x):
    """(whole numbers as float64, scale per row as float32); the quotients in 64 bits, where the
    nearest float and the nearest whole number are clear."""
    scale = (x.abs().amax(1).double() / 127).float()
    q = (x.double() / scale.double()[:, None]).round().clamp(-127, 127)
    return torch.where(scale[:, None] > 0, q, 0.0), scale


def _product_i8(x, w, w_scale):
    """x times int8 weights, in float32: the sums are whole numbers, exact in float64."""
    q, scale = _quantised(x)
    return (q @ w.double().t()).float() * scale[:, None] * w_scale


def _run_plain(s):
    kind, x = s["case"]["kind"], s["x"].float()
    if kind == "linear_i8":
        return _product_i8(x, s["w"], s["w_scale"]).to(s["x"].dtype)
    m = s["case"]["m"]
    if kind == "ffn_i8":
        a = _product_i8(x, s["gate_up"], s["gate_up_scale"])
        g, u = a[:, :m], a[:, m:]
        y = _product_i8(g / (1 + (-g).exp()) * u, s["down"], s["down_scale"])
        return (y if s["residual"] is None else y + s["residual"].float()).to(s["x"].dtype)
    gate_up, down = s["gate_up"].float(), s["down"].float()
    a = x @ gate_up.t()
    g, u = a[:, :m], a[:, m:]
    sig = 1 / (1 + (-g).exp())
    h = g * sig * u
    y = h @ down.t()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    y = y.to(s["x"].dtype)
    if kind == "ffn":
        return y
    dy = s["dy"].float()
    dh = dy @ down
    da = torch.cat([dh * u * sig * (1 + g * (1 - sig)), dh * g * sig], 1)
    grads = (da @ gate_up, da.t() @ x, dy.t() @ h)
    return (y,) + tuple(t.to(s["x"].dtype) for t in grads)


def work(case):
    T, size = case["T"], 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "linear_i8":
        k, n = case["k"], case["n"]
        return {"bytes": size * T * (k + n) + n * k + 4 * n, "flops": 2.0 * T * n * k}
    d, m = case["d"], case["m"]
    rows = T * d * (3 if case["residual"] else 2)
    if case["kind"] == "ffn_i8":
        return {"bytes": 3 * d * m + 4 * (2 * m + d) + size * rows, "flops": 6.0 * T * d * m}
    if case["kind"] == "train":  # x, dy, weights in; y, dx, weight gradients out
        return {"bytes": size * (6 * d * m + 4 * T * d), "flops": 18.0 * T * d * m}
    return {"bytes": size * (3 * d * m + rows), "flops": 6.0 * T * d * m}


def _rows_to_int8(x):
    scale = (x.abs().max(dim=1, keepdim=True).values / 127).float().double()
    return torch.round(x / scale.clamp(min=1e-300)).clamp(-127, 127), scale


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["kind"] == "linear_i8":
        q, scale = _rows_to_int8(x)
        return torch.matmul(q, s["w"].double().T) * (scale * s["w_scale"].double())
    m = case["m"]
    residual = 0.0 if s["residual"] is None else s["residual"].double()
    if case["kind"] == "ffn_i8":
        q, scale = _rows_to_int8(x)
        up = torch.matmul(q, s["gate_up"].double().T) * (scale * s["gate_up_scale"].double())
        q, scale = _rows_to_int8(torch.nn.functional.silu(up[:, :m]) * up[:, m:])
        return residual + torch.matmul(q, s["down"].double().T) * (scale
                                                                   * s["down_scale"].double())
    gate, up = s["gate_up"].double().split(m)
    down = s["down"].double()
    if case["kind"] == "ffn":
        h = torch.nn.functional.silu(x @ gate.T) * (x @ up.T)
        return residual + h @ down.T
    leaves = [t.requires_grad_(True) for t in (x, gate.clone(), up.clone(), down)]
    y = (torch.nn.functional.silu(leaves[0] @ leaves[1].T) * (leaves[0] @ leaves[2].T)
         ) @ leaves[3].T
    dx, dgate, dup, ddown = torch.autograd.grad(y, leaves, s["dy"].double())
    return y.detach(), dx, torch.cat([dgate, dup]), ddown
