"""Outputs that share memory with what a dense operator reads, or with another output: refused on the
host (CPU; the addresses are never dereferenced); in place where the entry points allow it (GPU)."""
import ctypes as C

import pytest
import torch

from paper_2608_04401_amd import binding as B

OK, INVALID = 0, 1
T, A, K = 4, 32, 32    # x, y [4, 32], weights of 32 by 32
F32 = B.ELB_F32
BIG = 1 << 30

ENTRY = {  # name: (arguments in order, the sizes of the tensors in bytes)
    "elb_ffn_forward": ["x", "W_gate_up", "W_down", "residual", T, A, K, F32, "y", "gate_up", "ws",
                        BIG, None],
    "elb_ffn_backward": ["dy", "x", "W_gate_up", "W_down", "gate_up", T, A, K, F32, "dx",
                         "dW_gate_up", "dW_down", "ws", BIG, None],
    "elb_quantize_rows": ["x", T, A, F32, "q", "scale", None],
    "elb_gemm_i8": ["q", "scale", "W", "W_scale", "residual", T, A, K, F32, "y", None],
    "elb_linear_i8": ["x", "W", "W_scale", "residual", T, A, K, F32, "y", "ws", BIG, None],
    "elb_ffn_forward_i8": ["x", "Wq", "Wq_scale", "W", "W_scale", "residual", T, A, K, F32, "y",
                           "ws", BIG, None],
}
BYTES = {"x": T * A * 4, "dy": T * A * 4, "y": T * A * 4, "dx": T * A * 4, "residual": T * A * 4,
         "W_gate_up": 2 * K * A * 4, "dW_gate_up": 2 * K * A * 4, "W_down": A * K * 4,
         "dW_down": A * K * 4, "gate_up": T * 2 * K * 4, "q": T * A, "scale": T * 4, "W": A * K,
         "W_scale": A * 4, "Wq": 2 * K * A, "Wq_scale": 2 * K * 4}
APART = {  # output: the tensors that it must not meet
    "elb_ffn_forward": {"y": ["W_gate_up", "W_down", "gate_up"],
                        "gate_up": ["x", "W_gate_up", "W_down", "residual"]},
    "elb_ffn_backward": {o: ["dy", "x", "W_gate_up", "W_down", "gate_up"] +
                         [p for p in ("dx", "dW_gate_up", "dW_down") if p != o]
                         for o in ("dx", "dW_gate_up", "dW_down")},
    "elb_quantize_rows": {"q": ["x", "scale"], "scale": ["x"]},
    "elb_gemm_i8": {"y": ["q", "scale", "W", "W_scale"]},
    "elb_linear_i8": {"y": ["x", "W", "W_scale"]},
    "elb_ffn_forward_i8": {"y": ["Wq", "Wq_scale", "W", "W_scale"]},
}
CASES = [(f, o, i) for f, d in APART.items() for o, others in d.items() for i in others]


def refused(entry, **at):
    """The status of the call with every tensor at an address of its own but for those given."""
    args, here = [], 1 << 20
    for a in ENTRY[entry]:
        if isinstance(a, str):
            args.append(C.c_void_p(at.get(a, here)))
            here += 1 << 16
        else:
            args.append(a)
    return getattr(B.lib(), entry)(*args)


@pytest.mark.parametrize("entry,out,other", CASES)
def test_an_output_on_another_tensor(entry, out, other):
    """The same address, and a last byte on the other's first."""
    at = 1 << 28
    for o in (at, at - BYTES[out] + 1, at + BYTES[other] - 1):
        assert refused(entry, **{out: o, other: at}) == INVALID
        text = B.lib().elb_last_error().decode()
        assert "overlaps" in text


@pytest.mark.parametrize("entry", [f for f in ENTRY if "residual" in ENTRY[f]])
def test_a_residual_beside_its_output(entry):
    """The residual may be the output; one that lies partly on it is refused."""
    at = 1 << 28
    for r in (at + 16, at - 16, at + BYTES["y"] - 4):
        assert refused(entry, y=at, residual=r) == INVALID
        assert b"overlaps residual" in B.lib().elb_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 40, 600, 2500])
def test_blocks_in_place(rows, dtype):
    """x as the output of both blocks, alone and as the residual too: the bits of a call apart."""
    d, m = 256, 384
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
    x, Wgu, Wd = n(rows, d), n(2 * m, d) * 0.06, n(d, m) * 0.05
    qgu, qd = B.elb_quantize_rows(Wgu), B.elb_quantize_rows(Wd)
    for call in (lambda a, **k: B.elb_ffn_forward(a, Wgu, Wd, **k),
                 lambda a, **k: B.elb_ffn_forward_i8(a, *qgu, *qd, **k)):
        for add in (False, True):
            want = call(x, residual=x if add else None)
            a = x.clone()
            got = call(a, out=a, residual=a if add else None)
            torch.cuda.synchronize()
            assert got is a and torch.equal(got, want)


@pytest.mark.gpu
def test_binding_refuses():
    x = torch.zeros(8, 64, device="cuda")
    W, c = torch.zeros(64, 64, dtype=torch.int8, device="cuda"), torch.ones(64, device="cuda")
    buf = torch.zeros(9, 64, device="cuda")
    for f in (lambda: B.elb_linear_i8(x, W, c, out=x),
              lambda: B.elb_linear_i8(x, W, c, residual=buf[:8], out=buf[1:]),
              lambda: B.elb_ffn_forward(x, torch.zeros(128, 64, device="cuda"),
                                        buf.new_zeros(64, 64), residual=buf[1:], out=buf[:8])):
        with pytest.raises(B.ElbError) as e:
            f()
        assert e.value.status == INVALID
    y = B.elb_linear_i8(x, W, c, residual=buf[:8], out=buf[:8])
    torch.cuda.synchronize()
    assert y.data_ptr() == buf.data_ptr()
