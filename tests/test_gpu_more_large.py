"""GPU: norms, 4-bit quantisation and products and the few-token layer on tensors whose elements or bytes
pass 2^31 and 2^32: what lies at their ends comes out as in a small call, or as in 64 bits."""
import pytest
import torch

from paper_2608_04401_amd import binding as B

import block_ref as R
from dense_ref import within

BF16, F32 = torch.bfloat16, torch.float32
pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0, std, generator=g)


def codes(g, *shape):
    q = torch.empty(shape[:-1] + (shape[-1] // 2,), dtype=torch.uint8, device="cuda")
    s = torch.empty(shape[:-1] + (shape[-1] // 32,), dtype=torch.uint8, device="cuda")
    return q.random_(0, 256, generator=g), s.random_(118, 124, generator=g)


def test_norms():
    T, d = 131300, 16384
    g = gen(1)
    x, b, ds, dn = (normal(g, T, d) for _ in range(4))
    w = {"w_post": 1 + normal(g, d, std=0.1), "w_pre": 1 + normal(g, d, std=0.1)}
    gate = normal(g, T, 1)
    total, normed, kept = B.elb_norm_forward(x, b, gate=gate, keep=True, **w)
    out = B.elb_norm_backward(ds, dn, total, b, kept, gate=gate, **w)
    at = slice(T - 3, T)
    one = lambda t: t[at].contiguous()
    t2, n2, k2 = B.elb_norm_forward(one(x), one(b), gate=one(gate), keep=True, **w)
    o2 = B.elb_norm_backward(one(ds), one(dn), t2, one(b), k2, gate=one(gate), **w)
    torch.cuda.synchronize()
    assert torch.equal(total[at], t2) and torch.equal(normed[at], n2)
    assert torch.equal(kept[:, at], k2)
    for i in range(3):  # of the residual, the block and the gate
        assert torch.equal(out[i][at], o2[i])


def test_quantise():
    rows, d = 66000, 65536
    x = normal(gen(2), rows, d)
    q, s = B.elb_quantize_f4(x)
    q2, s2 = B.elb_quantize_f4(x[-2:].contiguous())
    torch.cuda.synchronize()
    assert torch.equal(q[-2:], q2) and torch.equal(s[-2:], s2)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_projection(dtype):
    g = gen(3)
    n, k = 1 << 20, 8704
    W, s = codes(g, n, k)
    for T in (3, 40):
        x = normal(g, T, k, dtype=dtype)
        y = B.elb_linear_f4(x, W, s)
        torch.cuda.synchronize()
        within(y[:, -64:], *R.linear(x, R.from_f4(W[-64:], s[-64:])))
    W, s = codes(g, n, 64)
    x = normal(g, 2100, 64, dtype=dtype)
    y = B.elb_linear_f4(x, W, s)
    torch.cuda.synchronize()
    within(y[-2:, -64:], *R.linear(x[-2:], R.from_f4(W[-64:], s[-64:])))


@pytest.mark.parametrize("weights", ["bf16", "f4"])
def test_few_tokens(weights):
    """Tokens that select the last experts."""
    g = gen(4)
    T, d, N, m = 3, 4096, 64, 8192
    x = normal(g, T, d)
    Wr = normal(g, N, d, std=0.001)
    Wr[62:] += 0.01 * torch.sign(x[:1])
    x[1:] = x[:1] + 0.5 * x[1:]
    scales = {}
    if weights == "f4":
        gu, a = codes(g, N, 2 * m, d)
        dn, b = codes(g, N, d, m)
        scales = {"gate_up_scale": a, "down_scale": b}
        wgu = lambda e: R.from_f4(gu[e], a[e])
        wd = lambda e: R.from_f4(dn[e], b[e])
    else:
        gu, dn = normal(g, N, 2 * m, d, std=d ** -0.5), normal(g, N, d, m, std=m ** -0.5)
        wgu, wd = (lambda e: gu[e].double()), (lambda e: dn[e].double())
    y, r = B.elb_moe_forward_few(x, Wr, gu, dn, K=2, mode=B.MODE_TOPK, debug=True, **scales)
    torch.cuda.synchronize()
    assert set(r["ids"].flatten().tolist()) == {62, 63}
    within(y, *R.few(x, wgu, wd, r["k"], r["ids"], r["w"]))
