"""The dense block's and the 8-bit products' entry points: exported, and invalid arguments refused
on the host before anything is launched (CPU; the dummy pointers are never dereferenced)."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2608_04401_amd import binding as B

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "elbow_moe.h")
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P, ODD = C.c_void_p(0x1000), C.c_void_p(0x1010)
BIG = 1 << 50


def test_every_declared_entry_point_is_exported_and_bound():
    txt = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(elb_[a-z0-9_]+)\s*\(", txt))
    new = {"elb_ffn_workspace_bytes", "elb_ffn_forward", "elb_ffn_backward_workspace_bytes",
           "elb_ffn_backward", "elb_quantize_rows", "elb_gemm_i8", "elb_linear_i8_workspace_bytes",
           "elb_linear_i8", "elb_ffn_i8_workspace_bytes", "elb_ffn_forward_i8"}
    assert new <= names
    for n in names:
        assert hasattr(B.lib(), n), n
    for n in new:
        assert callable(getattr(B, n)), n


def _forward(T=8, d=64, m=32, dt=1, x=P, y=P, ws=P, n=BIG):
    return B.lib().elb_ffn_forward(x, P, P, None, T, d, m, dt, y, None, ws, n, None)


def _backward(T=8, d=64, m=32, dt=1, dy=P, keep=P, dx=P, ws=P, n=BIG):
    return B.lib().elb_ffn_backward(dy, P, P, P, keep, T, d, m, dt, dx, None, None, ws, n, None)


def _linear(T=8, n=64, k=32, dt=1, x=P, ws=P, nb=BIG):
    return B.lib().elb_linear_i8(x, P, P, None, T, n, k, dt, P, ws, nb, None)


def _block(T=8, d=64, m=32, dt=1, x=P, ws=P, n=BIG):
    return B.lib().elb_ffn_forward_i8(x, P, P, P, P, None, T, d, m, dt, P, ws, n, None)


@pytest.mark.parametrize("call", [_forward, _backward, _linear, _block])
def test_sizes_types_and_workspaces(call):
    a = [k for k in ("d", "n") if k in call.__code__.co_varnames[:call.__code__.co_argcount]][0]
    b = "k" if call is _linear else "m"
    assert call(T=-1) == INVALID
    assert call(dt=2) == INVALID
    for bad in (0, -16, 8, 40):
        assert call(**{b: bad}) == INVALID
        if call is not _linear:
            assert call(**{a: bad}) == INVALID
    assert call(**{b: (1 << 20) + 16}) == UNSUPPORTED
    assert call(T=1 << 31) == UNSUPPORTED
    assert call(ws=None) == WORKSPACE
    assert call(ws=ODD) == WORKSPACE
    assert call(**{"nb" if call is _linear else "n": 15}) == WORKSPACE
    assert B.lib().elb_last_error() != b""


def test_null_pointers():
    assert _forward(x=None) == INVALID and _forward(y=None) == INVALID
    assert _backward(dy=None) == INVALID and _backward(keep=None) == INVALID
    assert _linear(x=None) == INVALID and _block(x=None) == INVALID
    q = B.lib().elb_quantize_rows
    assert q(None, 8, 64, 1, P, P, None) == INVALID
    assert q(P, 8, 64, 1, None, P, None) == INVALID
    assert q(P, 8, 24, 1, P, P, None) == INVALID
    assert q(P, 8, 64, 5, P, P, None) == INVALID
    g = B.lib().elb_gemm_i8
    assert g(P, P, None, P, None, 8, 64, 32, 1, P, None) == INVALID
    assert g(P, P, P, P, None, 8, 64, 24, 1, P, None) == INVALID


def test_contraction_of_an_int32_sum():
    assert _linear(k=131072) == UNSUPPORTED
    assert _block(m=131072) == UNSUPPORTED and _block(d=131072) == UNSUPPORTED
    assert b"131071" in B.lib().elb_last_error()
    assert _linear(k=131056, x=None) == INVALID  # only the NULL pointer fails


def test_nothing_to_do():
    assert _forward(T=0, x=None, y=None, ws=None) == OK
    assert _linear(T=0, x=None, ws=None) == OK
    assert _block(T=0, x=None, ws=None) == OK
    assert _backward(dx=None, dy=None, ws=None) == OK  # no gradient asked for


def test_workspace_sizes():
    L = B.lib()
    assert L.elb_ffn_workspace_bytes(100, 64, 48, 1) >= 100 * 48 * 2
    assert L.elb_ffn_workspace_bytes(100, 64, 48, 0) >= 100 * 48 * 4
    assert L.elb_ffn_backward_workspace_bytes(100, 64, 48, 1) >= 100 * 48 * 3 * 2
    assert L.elb_linear_i8_workspace_bytes(100, 48, 64) >= 100 * 64 + 400
    assert L.elb_ffn_i8_workspace_bytes(100, 64, 48) >= 100 * (64 + 48 * 5 + 8)
    for f, args in ((L.elb_ffn_workspace_bytes, (-1, 64, 48, 1)),
                    (L.elb_ffn_workspace_bytes, (1, 64, 48, 9)),
                    (L.elb_ffn_backward_workspace_bytes, (1, 0, 48, 1)),
                    (L.elb_linear_i8_workspace_bytes, (-1, 48, 48)),
                    (L.elb_ffn_i8_workspace_bytes, (1, 64, 0))):
        assert f(*args) == 0


def test_binding_refuses_host_tensors_and_wrong_types():
    x, W, Wd = torch.zeros(4, 32), torch.zeros(64, 32), torch.zeros(32, 32)
    with pytest.raises(ValueError):
        B.elb_ffn_forward(x, W, Wd)
    with pytest.raises(TypeError):
        B.elb_ffn_forward(x.half(), W, Wd)
    with pytest.raises(ValueError):
        B.elb_quantize_rows(x)
    with pytest.raises(ValueError):
        B.elb_quantize_rows(torch.zeros(4, 2, 16))
    with pytest.raises(ValueError):
        B.elb_linear_i8(x, W.to(torch.int8), torch.zeros(64))


@pytest.mark.gpu
def test_binding_refuses_wrong_shapes():
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")
    x, W, Wd = z(4, 32), z(128, 32), z(32, 64)
    keep = z(4, 128, t=torch.float32)
    bad = [lambda: B.elb_ffn_forward(x, z(120, 32), Wd),
           lambda: B.elb_ffn_forward(x, W, z(16, 64)),
           lambda: B.elb_ffn_forward(x, W, Wd, residual=z(3, 32)),
           lambda: B.elb_ffn_forward(x, W, Wd, out=z(4, 16)),
           lambda: B.elb_ffn_forward(z(32, 4).t(), W, Wd),
           lambda: B.elb_ffn_backward(z(4, 16), x, W, Wd, keep),
           lambda: B.elb_ffn_backward(x, x, W, Wd, z(4, 64, t=torch.float32)),
           lambda: B.elb_gemm_i8(z(4, 32, t=torch.int8), z(3, t=torch.float32),
                                 z(64, 32, t=torch.int8), z(64, t=torch.float32)),
           lambda: B.elb_linear_i8(x, z(64, 16, t=torch.int8), z(64, t=torch.float32)),
           lambda: B.elb_ffn_forward_i8(x, z(128, 32, t=torch.int8), z(64, t=torch.float32),
                                        z(32, 64, t=torch.int8), z(32, t=torch.float32))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: B.elb_ffn_forward(x, W.float(), Wd),
              lambda: B.elb_ffn_backward(x, x, W, Wd, keep.double()),
              lambda: B.elb_linear_i8(x, z(64, 32, t=torch.uint8), z(64, t=torch.float32))):
        with pytest.raises(TypeError):
            f()
