"""The entry points of norms, 4-bit products and the few-token layer: invalid arguments and
overlapping outputs are refused on the host before anything is launched (CPU; the addresses are
never dereferenced)."""
import ctypes as C

import pytest
import torch

from paper_2608_04401_amd import binding as B

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P, ODD = C.c_void_p(1 << 24), C.c_void_p((1 << 24) + 16)
BIG = 1 << 50
NAN, INF = float("nan"), float("inf")


class Args:
    """Every pointer argument at an address of its own, 1 MiB apart, unless given."""

    def __init__(self, at):
        self.at, self.here = at, 1 << 30

    def __call__(self, name):
        self.here += 1 << 20
        p = self.at.get(name, self.here)
        return None if p is None else C.c_void_p(p)


def op(a, T=4, d=64, gate_kind=B.GATE_CHANNEL, dtype=1, eps=1e-6):
    v = [a(n) for n in ("residual", "block", "gate", "w_post", "w_pre")]
    return B.NormOp(*(p and p.value for p in v), T, d, gate_kind, dtype, 1.0, 1.0, eps)


def norm_forward(T=4, d=64, gate_kind=B.GATE_CHANNEL, dtype=1, eps=1e-6, **at):
    a = Args(at)
    o = op(a, T, d, gate_kind, dtype, eps)
    return B.lib().elb_norm_forward(C.byref(o), a("sum"), a("normed"), a("r_post"), a("r_pre"), None)


def norm_backward(T=4, d=64, gate_kind=B.GATE_CHANNEL, dtype=1, eps=1e-6, nb=BIG, ws=P, **at):
    a = Args(at)
    o = op(a, T, d, gate_kind, dtype, eps)
    return B.lib().elb_norm_backward(C.byref(o), *(a(n) for n in (
        "d_sum", "d_normed", "sum", "r_post", "r_pre", "d_residual", "d_block", "d_gate",
        "d_w_post", "d_w_pre")), ws, nb, None)


def quantize(T=4, d=64, dtype=1, **at):
    a = Args(at)
    return B.lib().elb_quantize_f4(a("x"), T, d, dtype, a("q"), a("scale"), None)


def linear(T=4, n=64, k=64, dtype=1, ws=P, nb=BIG, residual=None, **at):
    a = Args(dict(at, residual=residual))
    return B.lib().elb_linear_f4(a("x"), a("W"), a("W_scale"), a("residual"), T, n, k, dtype, a("y"),
                                 ws, nb, None)


def block(T=4, d=64, m=64, dtype=1, ws=P, nb=BIG, residual=None, **at):
    a = Args(dict(at, residual=residual))
    return B.lib().elb_ffn_forward_f4(a("x"), a("W_gate_up"), a("gate_up_scale"), a("W_down"),
                                      a("down_scale"), a("residual"), T, d, m, dtype, a("y"), ws, nb,
                                      None)


def few(T=4, d=64, N=8, m=64, K=4, eps=1e-8, mode=0, renorm=0, ws=P, nb=BIG, params=True,
        residual=None, **at):
    a = Args(dict(at, residual=residual))
    p = B.RouteParams(K, eps, mode, renorm)
    return B.lib().elb_moe_forward_few(
        *(a(n) for n in ("x", "W_router", "W_gate_up", "gate_up_scale", "W_down", "down_scale",
                         "residual")), T, d, N, m, C.byref(p) if params else None, a("y"), ws, nb,
        a("k_out"), a("ids_out"), a("w_out"), None)


@pytest.mark.parametrize("call", [norm_forward, norm_backward])
def test_norm_arguments(call):
    assert call(T=-1) == INVALID and call(dtype=2) == INVALID
    for d in (0, -16, 8, 40):
        assert call(d=d) == INVALID
    assert call(d=16400) == UNSUPPORTED and call(T=1 << 31) == UNSUPPORTED
    for eps in (0.0, -1e-6, NAN, INF):
        assert call(eps=eps) == INVALID
    assert call(gate_kind=4) == INVALID and call(gate_kind=-1) == INVALID
    assert call(gate=None) == INVALID
    assert B.lib().elb_last_error() != b""


def test_norm_parts():
    f = B.lib().elb_norm_forward
    assert f(None, P, P, P, P, None) == INVALID
    assert norm_forward(residual=None, block=None, w_post=None, gate_kind=0) == INVALID
    assert norm_forward(block=None) == INVALID            # gate and w_post without a block
    assert norm_forward(block=None, gate_kind=0) == INVALID
    assert norm_forward(w_pre=None) == INVALID            # normed without its weight
    assert norm_forward(normed=None) == INVALID
    assert norm_forward(sum=None, normed=None, w_pre=None) == OK  # nothing asked for
    assert norm_forward(T=0, residual=None, block=None, w_post=None, gate_kind=0) == OK
    b = norm_backward
    assert b(ws=None) == WORKSPACE and b(ws=ODD) == WORKSPACE and b(nb=15) == WORKSPACE
    assert b(d_sum=None, d_normed=None) == INVALID
    assert b(sum=None) == INVALID and b(r_pre=None) == INVALID and b(r_post=None) == INVALID
    assert b(block=None) == INVALID
    assert b(w_post=None) == INVALID                      # its gradient without the weight
    assert b(w_pre=None) == INVALID
    assert b(gate_kind=0) == INVALID                      # d_gate without a gate
    assert b(d_residual=None, d_block=None, d_gate=None, d_w_post=None, d_w_pre=None, ws=None) == OK


ALL, ROW = 4 * 64 * 2, 64 * 2
FWD = {"residual": ALL, "block": ALL, "gate": ROW, "w_post": ROW, "w_pre": ROW, "sum": ALL,
       "normed": ALL, "r_post": 16, "r_pre": 16}
BWD = {"d_sum": ALL, "d_normed": ALL, "sum": ALL, "r_post": 16, "r_pre": 16, "block": ALL,
       "gate": ROW, "w_post": ROW, "w_pre": ROW}
GRADS = {"d_residual": ALL, "d_block": ALL, "d_gate": ROW, "d_w_post": ROW, "d_w_pre": ROW}
LIN = {"x": ALL, "W": 64 * 32, "W_scale": 64 * 2}
BLK = {"W_gate_up": 128 * 32, "gate_up_scale": 128 * 2, "W_down": 64 * 32, "down_scale": 64 * 2}
FEW4 = {"W_router": 8 * 64 * 2, "W_gate_up": 8 * 128 * 32, "gate_up_scale": 8 * 128 * 2,
        "W_down": 8 * 64 * 32, "down_scale": 8 * 64 * 2}
FEW16 = {"W_gate_up": 8 * 128 * 64 * 2, "W_down": 8 * 64 * 64 * 2}
ROUTES = {"k_out": 16, "ids_out": 64, "w_out": 64}


def pairs():
    outs = ["sum", "normed", "r_post", "r_pre"]
    for i, o in enumerate(outs):
        for other, n in FWD.items():
            if other != o and (other not in outs[:i]) and (o, other) != ("sum", "residual"):
                yield norm_forward, {}, o, FWD[o], other, n
    for o, n in GRADS.items():
        for other, m in list(BWD.items()) + [g for g in GRADS.items() if g[0] != o]:
            yield norm_backward, {}, o, n, other, m
    for o, n, others in (("q", 4 * 32, {"x": ALL, "scale": 8}), ("scale", 8, {"x": ALL})):
        for other, m in others.items():
            yield quantize, {}, o, n, other, m
    for other, m in LIN.items():
        yield linear, {}, "y", ALL, other, m
    for other, m in BLK.items():
        yield block, {}, "y", ALL, other, m
    for other, m in list(FEW4.items()) + list(ROUTES.items()):
        yield few, {}, "y", ALL, other, m
    for other, m in FEW16.items():
        yield few, {"gate_up_scale": None, "down_scale": None}, "y", ALL, other, m
    for o, n in ROUTES.items():
        for other, m in [("x", ALL)] + list(FEW4.items()) + [r for r in ROUTES.items() if r[0] != o]:
            yield few, {}, o, n, other, m


@pytest.mark.parametrize("call,with_,out,size,other,other_size", list(pairs()))
def test_an_output_on_another_tensor(call, with_, out, size, other, other_size):
    """The same address, a last byte on the other's first, a first on its last."""
    at = 1 << 28
    for o in (at, at - size + 1, at + other_size - 1):
        assert call(**with_, **{out: o, other: at}) == INVALID
        assert b"overlaps" in B.lib().elb_last_error()


@pytest.mark.parametrize("call,out", [(norm_forward, "sum"), (linear, "y"), (block, "y"), (few, "y")])
def test_a_residual_partly_on_its_output(call, out):
    at = 1 << 28
    for r in (at + 16, at - 16, at + ALL - 2):
        assert call(**{out: at, "residual": r}) == INVALID
        assert b"overlaps residual" in B.lib().elb_last_error()


def test_f4_arguments():
    for call, names in ((quantize, "d"), (linear, "nk"), (block, "dm")):
        assert call(T=-1) == INVALID and call(dtype=3) == INVALID
        assert call(T=1 << 31) == UNSUPPORTED
        for a in names:
            for bad in (0, -32, 8, 40) + (() if a == "n" else (16, 48)):
                assert call(**{a: bad}) == INVALID, (call, a, bad)
            assert call(**{a: (1 << 20) + 32}) == UNSUPPORTED
    for name in ("x", "W", "W_scale", "y"):
        assert linear(**{name: None}) == INVALID
    for name in ("x", "y") + tuple(BLK):
        assert block(**{name: None}) == INVALID
    for name in ("x", "q", "scale"):
        assert quantize(**{name: None}) == INVALID
    for T in (4, 3000):
        assert block(T=T, ws=None) == WORKSPACE and block(T=T, ws=ODD) == WORKSPACE
        assert block(T=T, nb=15) == WORKSPACE
    # that many tokens take converted weights, in scratch
    assert linear(T=3000, ws=None) == WORKSPACE and linear(T=3000, nb=15) == WORKSPACE
    none = {"x": None, "y": None}
    assert linear(T=0, ws=None, **none) == OK and block(T=0, ws=None, **none) == OK
    assert quantize(T=0, x=None) == OK


def test_few_arguments():
    assert few(T=17) == UNSUPPORTED and few(T=-1) == INVALID
    assert few(N=65) == UNSUPPORTED and few(N=1, K=1) == INVALID
    assert few(N=64, K=17) == UNSUPPORTED and few(K=9) == INVALID and few(K=0) == INVALID
    assert few(d=96) == INVALID and few(m=32) == INVALID and few(d=(1 << 20) + 64) == UNSUPPORTED
    assert few(eps=NAN) == INVALID and few(mode=2) == INVALID and few(renorm=2) == INVALID
    assert few(params=False) == INVALID
    assert few(gate_up_scale=None) == INVALID and few(down_scale=None) == INVALID
    for name in ("x", "W_router", "W_gate_up", "W_down", "y"):
        assert few(**{name: None}) == INVALID
    assert few(ws=None) == WORKSPACE and few(ws=ODD) == WORKSPACE and few(nb=15) == WORKSPACE
    assert few(T=0, x=None, ws=None) == OK


def test_workspace_sizes():
    L = B.lib()
    assert L.elb_norm_backward_workspace_bytes(10000, 64) >= 3 * 64 * 4
    assert L.elb_norm_backward_workspace_bytes(-1, 64) == 0
    assert L.elb_linear_f4_workspace_bytes(1, 64, 64, 1) == 0
    assert L.elb_linear_f4_workspace_bytes(1000, 64, 64, 0) >= 64 * 64 * 4
    assert L.elb_ffn_f4_workspace_bytes(1000, 64, 32, 1) >= 3 * 64 * 32 * 2 + 1000 * 32 * 2
    assert L.elb_moe_few_workspace_bytes(16, 64, 8, 64, 8) >= 16 * 8 * 64 * 2
    assert L.elb_moe_few_workspace_bytes(17, 64, 8, 64, 8) == 0
    for f, args in ((L.elb_linear_f4_workspace_bytes, (48, 1056, 1)),
                    (L.elb_linear_f4_workspace_bytes, (2048, 8192, 1)),
                    (L.elb_ffn_f4_workspace_bytes, (2048, 8192, 1)),
                    (L.elb_ffn_f4_workspace_bytes, (96, 64, 0)),
                    (L.elb_norm_backward_workspace_bytes, (2048,))):
        last = 0
        for T in list(range(0, 140)) + list(range(200, 9000, 61)):
            n = f(T, *args)
            assert n >= last, (f, T)
            last = n


def test_few_token_workspace_without_shares():
    """Above 4096 columns the down product is not cut into shares: routing and h alone."""
    f = B.lib().elb_moe_few_workspace_bytes
    up = lambda n: -(-n // 256) * 256
    for T, d, m, K in ((1, 8192, 64, 1), (16, 4160, 128, 8), (3, 1 << 20, 64, 2)):
        assert f(T, d, 8, m, K) == up(T * K * m * 2) + up(T * 4) + 2 * up(T * K * 4)
    assert f(1, 4096, 8, 64, 1) >= 2 * 16 * 4096 * 4


def test_binding_refuses_host_tensors_types_and_shapes():
    z = torch.zeros
    x, u8 = z(4, 64), lambda *s: torch.zeros(s, dtype=torch.uint8)
    for f in (lambda: B.elb_norm_forward(), lambda: B.elb_norm_forward(x, w_pre=z(64)),
              lambda: B.elb_norm_forward(z(4, 2, 8)), lambda: B.elb_quantize_f4(x),
              lambda: B.elb_quantize_f4(z(64)),
              lambda: B.elb_linear_f4(x, u8(32, 32), u8(32, 2)),
              lambda: B.elb_ffn_forward_f4(x, u8(64, 32), u8(64, 2), u8(64, 16), u8(64, 1)),
              lambda: B.elb_moe_forward_few(x.bfloat16(), z(8, 64), z(8, 128, 64), z(8, 64, 64),
                                            gate_up_scale=u8(8, 128, 2)),
              lambda: B.elb_moe_forward_few(x.bfloat16(), z(8, 64), z(8, 128, 64), z(64, 64))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: B.elb_norm_forward(x.half()), lambda: B.elb_quantize_f4(x.half()),
              lambda: B.elb_moe_forward_few(x, z(8, 64), z(8, 128, 64), z(8, 64, 64))):
        with pytest.raises(TypeError):
            f()


@pytest.mark.gpu
def test_binding_refuses_wrong_shapes():
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")
    u8 = lambda *s: z(*s, t=torch.uint8)
    x, w = z(4, 64), z(64)
    kept = z(2, 4, t=torch.float32)
    for f in (lambda: B.elb_norm_forward(x, x, gate=z(4)), lambda: B.elb_norm_forward(x, x, gate=z(1, 64)),
              lambda: B.elb_norm_forward(x, z(3, 64)), lambda: B.elb_norm_forward(x, x, w_post=z(32)),
              lambda: B.elb_norm_forward(z(64, 4).t(), w_pre=w),
              lambda: B.elb_norm_backward(z(3, 64), None, x, x, kept),
              lambda: B.elb_norm_backward(x, None, x, x, z(2, 3, t=torch.float32), w_post=w),
              lambda: B.elb_linear_f4(x, u8(16, 16), u8(16, 2)),
              lambda: B.elb_linear_f4(x, u8(16, 32), u8(16, 1)),
              lambda: B.elb_ffn_forward_f4(x, u8(64, 32), u8(64, 2), u8(32, 16), u8(32, 1)),
              lambda: B.elb_moe_forward_few(x, z(8, 64), z(8, 64, 64), z(8, 64, 64)),
              lambda: B.elb_moe_forward_few(x, z(7, 64), z(8, 128, 64), z(8, 64, 64))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: B.elb_norm_forward(x, x.float()), lambda: B.elb_norm_forward(x, w_pre=w.float()),
              lambda: B.elb_linear_f4(x, z(16, 32, t=torch.int8), u8(16, 2)),
              lambda: B.elb_moe_forward_few(x, z(8, 64), u8(8, 128, 32), u8(8, 64, 32))):
        with pytest.raises(TypeError):
            f()
    y = x.clone()
    for f, status in ((lambda: B.elb_linear_f4(x, u8(64, 32), u8(64, 2), out=x), INVALID),
                      (lambda: B.elb_norm_forward(x, y, out=y), INVALID),
                      (lambda: B.elb_moe_forward_few(z(17, 64), z(8, 64), z(8, 128, 64), z(8, 64, 64),
                                                     K=2), UNSUPPORTED)):
        with pytest.raises(B.ElbError) as e:
            f()
        assert e.value.status == status
