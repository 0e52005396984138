"""Refusals of the 8-bit decoder operators: every bad call is answered on the host, before
anything launches.  Fake device addresses, never dereferenced; skipped where a GPU is
present, so that a mistake in a case cannot launch anything."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2110_10221_amd", "libragged.so")
pytestmark = [pytest.mark.skipif(not os.path.exists(LIB), reason="libragged.so not built"),
              pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer cases run only without a GPU")]

A = 0x7f0000000000
ARG, DTYPE, SHAPE, CAP, WS = -1, -2, -3, -4, -5
F32, BF16 = 0, 1
MB = 1 << 20


def lib():
    import paper_2110_10221_amd as rag

    return rag.library()


def call(fn, order, base, **over):
    a = dict(base)
    a.update(over)
    return getattr(lib(), fn)(*[a[k] for k in order])


NORM = ("x", "ldx", "residual", "ldr", "gamma", "eps", "sum", "lds", "y", "ldy", "q", "ldq", "q_scale", "T", "d",
        "dtype", "stream")
NORM_OK = dict(x=A, ldx=512, residual=A + MB, ldr=512, gamma=A + 2 * MB, eps=1e-6, sum=A + 3 * MB, lds=512, y=A + 4 * MB,
               ldy=512, q=A + 5 * MB, ldq=512, q_scale=A + 6 * MB, T=0, d=512, dtype=BF16, stream=None)


@pytest.mark.parametrize("over,status", [
    (dict(dtype=2), DTYPE), (dict(T=-1), ARG), (dict(d=0), ARG), (dict(d=516), SHAPE), (dict(d=16392, ldx=16392), SHAPE),
    (dict(eps=0.0), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG), (dict(x=None), ARG),
    (dict(ldx=504), SHAPE), (dict(ldx=516), SHAPE), (dict(x=A + 8), SHAPE), (dict(residual=A + MB + 2), SHAPE),
    (dict(gamma=None), ARG), (dict(gamma=A + 2 * MB + 8), ARG), (dict(y=None, q=None, q_scale=None), ARG),
    (dict(q_scale=None), ARG), (dict(q=None), ARG), (dict(q=A + 5 * MB + 4), SHAPE), (dict(ldq=516), SHAPE),
    (dict(ldq=504), SHAPE), (dict(sum=A + 3 * MB + 4), SHAPE), (dict(dtype=F32, d=6), SHAPE),
    (dict(dtype=F32, y=A + 4 * MB + 4), SHAPE), (dict(y=A + 1024), ARG), (dict(sum=A + MB + 512 * 2), ARG),
    (dict(y=A, ldy=520), ARG), (dict(sum=A + 4 * MB), ARG), (dict(q=A + 4 * MB), ARG), (dict(q_scale=A + 5 * MB), ARG),
    (dict(q=A), ARG), (dict(y=A + 2 * MB), ARG)])
def test_rmsnorm_refuses(over, status):
    over = dict(over)
    over.setdefault("T", 4)
    assert call("packed_rmsnorm", NORM, NORM_OK, **over) == status


def test_nothing_to_do():
    assert call("packed_rmsnorm", NORM, NORM_OK, T=0) == 0
    assert call("packed_rmsnorm", NORM, NORM_OK, T=0, x=None, gamma=None, y=None, q=None, q_scale=None) == 0
    assert call("packed_quantize_i8", QUANT, QUANT_OK, T=0, x=None, q=None, scale=None) == 0


QUANT = ("x", "ldx", "q", "ldq", "scale", "T", "d", "dtype", "stream")
QUANT_OK = dict(x=A, ldx=512, q=A + MB, ldq=512, scale=A + 2 * MB, T=4, d=512, dtype=BF16, stream=None)


@pytest.mark.parametrize("over,status", [
    (dict(dtype=-1), DTYPE), (dict(T=-2), ARG), (dict(d=-8), ARG), (dict(d=4), SHAPE), (dict(d=16392, ldx=20000), SHAPE),
    (dict(x=None), ARG), (dict(x=A + 2), SHAPE), (dict(ldx=511), SHAPE), (dict(q=None), ARG), (dict(scale=None), ARG),
    (dict(ldq=513), SHAPE), (dict(ldq=8), SHAPE), (dict(q=A + MB + 4), SHAPE), (dict(q=A), ARG), (dict(scale=A + 64), ARG),
    (dict(scale=A + MB + 64), ARG), (dict(scale=A + 2 * MB + 2), SHAPE), (dict(dtype=F32, ldx=514), SHAPE)])
def test_quantize_refuses(over, status):
    assert call("packed_quantize_i8", QUANT, QUANT_OK, **over) == status


def test_binding_refuses_other_shapes_and_types():
    import paper_2110_10221_amd as rag

    x, g = torch.zeros(4, 64), torch.zeros(64)
    q, s = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4)
    for bad in (dict(y=torch.zeros(4, 32)), dict(y=torch.zeros(3, 64)), dict(y=torch.zeros(4, 64, dtype=torch.bfloat16)),
                dict(y=x, residual=torch.zeros(5, 64)), dict(q=q.float(), q_scale=s), dict(q=q, q_scale=s[:3]),
                dict(q=q, q_scale=torch.zeros(8)[::2]), dict(y=x, x_out=torch.zeros(4, 60))):
        with pytest.raises(ValueError):
            rag.packed_rmsnorm(x, g, **bad)
    with pytest.raises(ValueError):
        rag.packed_rmsnorm(x, g[:32], x)
    with pytest.raises(ValueError):
        rag.packed_quantize_i8(x, q[:, :32], s)
