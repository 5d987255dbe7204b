"""GPU: the whole layer for a few tokens in two launches, experts in bf16 and in 4 bits; and a run of
norm, layer, norm as a decoder step has it, captured and replayed."""
import ctypes

import pytest
import torch

from paper_2608_04401_amd import binding as B

import block_ref as R
from dense_ref import shifted, within

BF16 = torch.bfloat16
pytestmark = pytest.mark.gpu


def layer(T, d, N, m, weights, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + T)
    n = lambda *s, std=1.0: (torch.randn(s, generator=g, device="cuda") * std).to(BF16)
    v = {"x": n(T, d), "W_router": n(N, d, std=0.05), "residual": n(T, d),
         "W_gate_up": n(N, 2 * m, d, std=d ** -0.5), "W_down": n(N, d, m, std=m ** -0.5)}
    v["wgu"] = lambda e: v["W_gate_up"][e].double()
    v["wd"] = lambda e: v["W_down"][e].double()
    v["scales"] = {}
    if weights == "f4":
        v["W_gate_up"], a = B.elb_quantize_f4(v["W_gate_up"])
        v["W_down"], b = B.elb_quantize_f4(v["W_down"])
        v["scales"] = {"gate_up_scale": a, "down_scale": b}
        v["wgu"] = lambda e: R.from_f4(v["W_gate_up"][e], a[e])
        v["wd"] = lambda e: R.from_f4(v["W_down"][e], b[e])
    return v


def call(v, x=None, **kw):
    return B.elb_moe_forward_few(v["x"] if x is None else x, v["W_router"], v["W_gate_up"],
                                 v["W_down"], **v["scales"], **kw)


def check(v, residual=True, **kw):
    res = v["residual"] if residual else None
    y, r = call(v, residual=res, debug=True, **kw)
    k, ids, w, _ = B.elb_router_route(v["x"], v["W_router"], **kw)
    torch.cuda.synchronize()
    assert torch.equal(r["k"], k) and torch.equal(r["ids"], ids) and torch.equal(r["w"], w)
    within(y, *R.few(v["x"], v["wgu"], v["wd"], k, ids, w, res))
    return y


@pytest.mark.parametrize("weights", ["bf16", "f4"])
@pytest.mark.parametrize("T", [1, 2, 3, 7, 8, 13, 16])
def test_layer(T, weights):
    for d, N, m, K in ((64, 2, 64, 1), (64, 2, 64, 2), (128, 8, 64, 4), (192, 17, 128, 8),
                       (320, 33, 192, 16), (256, 48, 64, 9), (512, 64, 320, 8)):
        v = layer(T, d, N, m, weights)
        check(v, K=K)
        check(v, K=K, residual=False, renormalize=True, mode=B.MODE_TOPK)


@pytest.mark.parametrize("weights", ["bf16", "f4"])
def test_the_headline_layer(weights):
    for T in (1, 5, 16):
        check(layer(T, 2048, 64, 1024, weights), K=8)


@pytest.mark.parametrize("weights", ["bf16", "f4"])
def test_wide_layers(weights):
    """Rows longer than a wave's share of tokens in registers, and expert widths past a unit."""
    for T, d, N, m, K in ((1, 2112, 8, 64, 2), (13, 2240, 5, 128, 3), (3, 4096, 4, 576, 2),
                          (16, 6144, 3, 64, 3)):
        check(layer(T, d, N, m, weights), K=K)


@pytest.mark.parametrize("weights", ["bf16", "f4"])
def test_one_expert_for_all_and_all_for_one(weights):
    """Every token on the same expert; every token on all experts; a router of zeros (ties: the
    lowest ids)."""
    v = layer(16, 128, 16, 128, weights)
    v["W_router"][3] = 0
    v["x"][:] = v["x"].abs()
    v["W_router"][3] += 1.0
    y, r = call(v, K=1, debug=True)
    torch.cuda.synchronize()
    assert r["ids"].flatten().tolist() == [3] * 16
    check(v, K=1)
    check(v, K=16, mode=B.MODE_TOPK)
    v["W_router"].zero_()
    check(v, K=5, mode=B.MODE_TOPK)


@pytest.mark.parametrize("weights", ["bf16", "f4"])
def test_in_place_unaligned_and_what_lies_around(weights):
    for T in (1, 11):
        v = layer(T, 192, 24, 192, weights)
        want = check(v, K=6)
        alone = call(v, K=6)
        a = v["residual"].clone()
        assert call(v, K=6, residual=a, out=a) is a
        b = v["x"].clone()
        call(v, x=b, K=6, out=b)
        buf = torch.full((T + 2, 192), 7.0, dtype=BF16, device="cuda")
        w = dict(v)
        for i, name in enumerate(("x", "W_router", "W_gate_up", "W_down")):
            w[name] = shifted(v[name], i + 1)
        w["scales"] = {k: shifted(t, 3) for k, t in v["scales"].items()}
        call(w, K=6, residual=v["residual"], out=buf[1:-1])
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, alone) and torch.equal(buf[1:-1], want)
        assert bool((buf[0] == 7).all() and (buf[-1] == 7).all())


def test_a_token_alone_and_nan():
    """A token's result does not depend on the others' values: rows of NaN beside it change
    nothing, wherever they are routed."""
    for weights in ("bf16", "f4"):
        v = layer(9, 128, 16, 64, weights)
        y = call(v, K=4, residual=v["residual"])
        x = v["x"].clone()
        x[4] = float("nan")
        z = call(v, x=x, K=4, residual=v["residual"])
        torch.cuda.synchronize()
        keep = [0, 1, 2, 3, 5, 6, 7, 8]
        # the others' partial sums are cut elsewhere where the NaN token uses other experts
        d = (y[keep].float() - z[keep].float()).abs()
        assert bool((d <= 2.0 ** -7 * (1 + y[keep].float().abs())).all())


@pytest.mark.parametrize("weights", ["bf16", "f4"])
@pytest.mark.parametrize("T", [2, 9, 16])
def test_weights_that_are_no_number_stay_with_their_tokens(T, weights):
    """An infinity or a NaN among an expert's weights reaches the tokens that have selected it, a weight of
    the down product in its own column alone; everything else keeps its bits.  (Rows of y in several shares
    of the contraction and in one; an expert of more than eight tokens, which takes two passes.)"""
    for d, N, m, K, mode in ((128, 16, 64, 4, B.MODE_ELBOW), (512, 64, 320, 8, B.MODE_ELBOW),
                             (256, 16, 192, 12, B.MODE_TOPK), (4160, 5, 64, 2, B.MODE_TOPK)):
        v = layer(T, d, N, m, weights)
        kw = {"K": K, "mode": mode, "residual": v["residual"]}
        y, r = call(v, debug=True, **kw)
        torch.cuda.synchronize()
        on = (r["ids"][None] == torch.arange(N, device="cuda")[:, None, None]).any(-1)  # [N, T]
        tokens = on.sum(1)
        e = int(torch.where(tokens < T, tokens, -1).argmax())
        assert 0 < tokens[e] < T, (d, N)
        cols = [5, d - 3]
        w = dict(v, scales={k: t.clone() for k, t in v["scales"].items()})
        if weights == "f4":
            w["scales"]["down_scale"][e, cols[0], 0] = 255
            w["scales"]["down_scale"][e, cols[1], -1] = 255
        else:
            w["W_down"] = v["W_down"].clone()
            w["W_down"][e, cols[0], 3] = float("inf")
            w["W_down"][e, cols[1], m - 1] = float("nan")
        bad = call(w, **kw)
        torch.cuda.synchronize()
        hit = torch.zeros_like(y, dtype=torch.bool)
        hit[:, cols] = on[e][:, None]
        assert torch.equal(bad[~hit], y[~hit]), (d, N)
        assert not bool(bad[hit].isfinite().any()), (d, N)
        w = dict(v, scales={k: t.clone() for k, t in v["scales"].items()})
        if weights == "f4":
            w["scales"]["gate_up_scale"][e, 3, -1] = 255
        else:
            w["W_gate_up"] = v["W_gate_up"].clone()
            w["W_gate_up"][e, m + 3, 7] = float("nan")
        bad = call(w, **kw)
        torch.cuda.synchronize()
        assert torch.equal(bad[~on[e]], y[~on[e]]) and bool(bad[on[e]].isnan().all()), (d, N)


def test_nothing_behind_the_workspace_is_written():
    """A workspace of the size asked for, with the product in shares and whole."""
    for T, d, m, K in ((1, 512, 64, 2), (16, 4160, 64, 2), (3, 8192, 128, 1)):
        v = layer(T, d, 8, m, "bf16")
        want = call(v, K=K)
        nb = B.elb_moe_few_workspace_bytes(T, d, 8, m, K)
        ws = torch.full((nb + 4096,), 7, dtype=torch.uint8, device="cuda")
        y = torch.empty_like(want)
        p = B.RouteParams(K, 1e-8, B.MODE_ELBOW, 0)
        ptr = lambda t: t.data_ptr()
        assert B.lib().elb_moe_forward_few(
            ptr(v["x"]), ptr(v["W_router"]), ptr(v["W_gate_up"]), None, ptr(v["W_down"]), None, None,
            T, d, 8, m, ctypes.byref(p), ptr(y), ptr(ws), nb, None, None, None,
            torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert torch.equal(y, want) and bool((ws[nb:] == 7).all())


def test_no_tokens():
    v = layer(1, 64, 8, 64, "bf16")
    assert call(v, x=v["x"][:0].contiguous(), K=2).shape == (0, 64)


def test_streams_and_two_calls_at_once():
    """Calls on two streams at once, each with its own workspace, give the bits of calls in order."""
    a, b = layer(3, 512, 64, 320, "f4"), layer(16, 512, 64, 320, "bf16")
    wa, wb = call(a, K=8), call(b, K=8)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(5):
        with torch.cuda.stream(sa):
            ya = call(a, K=8)
        with torch.cuda.stream(sb):
            yb = call(b, K=8)
        got.append((ya, yb))
    torch.cuda.synchronize()
    for ya, yb in got:
        assert torch.equal(ya, wa) and torch.equal(yb, wb)


def step(v, w, x, out):
    """A decoder layer's second half: the norm before, the layer, the shared expert in 4 bits, the
    norm after with a gate, and the next layer's norm before."""
    _, n = B.elb_norm_forward(x, w_pre=w["pre"])
    y = B.elb_ffn_forward_f4(n, *w["gu"], *w["dn"])
    y = call(v, x=n, K=8, residual=y)
    s, n2 = B.elb_norm_forward(x, y, w["post"], w["next"], w["gate"], block_scale=0.5, out=out[0])
    out[1].copy_(B.elb_linear_f4(n2, *w["head"]))


@pytest.mark.parametrize("weights", ["bf16", "f4"])
def test_a_decoder_step_captured_and_replayed(weights):
    """Two graphs over the same weights, replayed in turn on new inputs with eager steps between."""
    d, m = 512, 320
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n = lambda *s, std=1.0: (torch.randn(s, generator=g, device="cuda") * std).to(BF16)
    w = {k: 1 + n(d, std=0.1) for k in ("pre", "post", "next", "gate")}
    w["gu"], w["dn"] = (B.elb_quantize_f4(t) for t in (n(2 * m, d, std=0.04), n(d, m, std=0.05)))
    w["head"] = B.elb_quantize_f4(n(1056, d, std=0.04))
    graphs = []
    v = layer(16, d, 64, m, weights)
    for T in (1, 13):
        x = n(T, d)
        out = [torch.empty_like(x), torch.empty((T, 1056), dtype=BF16, device="cuda")]
        step(v, w, x, out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(v, w, x, out)
        graphs.append((graph, x, out))
    for r in range(3):
        for graph, x, out in graphs:
            x.copy_(n(*x.shape))
            graph.replay()
            other = n(5, d)
            step(v, w, other, [torch.empty_like(other), torch.empty((5, 1056), dtype=BF16,
                                                                     device="cuda")])
            torch.cuda.synchronize()
            got = [t.clone() for t in out]
            eager = [torch.empty_like(t) for t in out]
            step(v, w, x.clone(), eager)
            torch.cuda.synchronize()
            assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
