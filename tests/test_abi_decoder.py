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
    (dict(dtype=2), DTYPE), (dict(T=-1), ARG), (dict(T=2 ** 30 + 1), ARG), (dict(d=0), ARG), (dict(d=516), SHAPE), (dict(d=16392, ldx=16392), SHAPE),
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


ROTARY = ("plan", "x", "ldx", "y", "ldy", "heads", "head_dim", "rot_dim", "layout", "inv_freq", "amplitude", "pos_start",
          "dtype", "stream")


def plan(**over):
    import paper_2110_10221_amd as rag

    f = dict(batch=4, total_tokens=232, max_len=128, heads=8, qkt_cap=100, av_cap=100, lengths=A + 50 * MB,
             tok_off=A + 51 * MB, att_off=A + 52 * MB, order=A + 53 * MB, tok_seq=A + 54 * MB, qkt_item_off=A + 55 * MB,
             av_item_off=A + 56 * MB, qkt_items=A + 57 * MB, av_items=A + 58 * MB, status=A + 59 * MB)
    f.update(over)
    return ctypes.byref(rag.RagPlan(**f))


@pytest.mark.parametrize("over,status", [
    (dict(plan=None), ARG), (dict(dtype=3), DTYPE), (dict(heads=0), ARG), (dict(big=1), ARG), (dict(heads=1 << 20), SHAPE), (dict(layout=4), ARG),
    (dict(layout=-1), ARG), (dict(rot_dim=0), SHAPE), (dict(rot_dim=33), SHAPE), (dict(rot_dim=66), SHAPE),
    (dict(head_dim=514, ldx=9000, ldy=9000), SHAPE), (dict(amplitude=float("inf")), ARG), (dict(x=None), ARG),
    (dict(y=None), ARG), (dict(ldx=1023), SHAPE), (dict(ldy=1000), SHAPE), (dict(x=A + 1), SHAPE), (dict(inv_freq=None), ARG),
    (dict(inv_freq=A + 2 * MB + 4), ARG), (dict(pos_start=A + 3 * MB + 2), ARG), (dict(y=A + 2048), ARG),
    (dict(y=A, ldy=1040), ARG), (dict(inv_freq=A + MB), ARG), (dict(pos_start=A + MB + 4), ARG),
    (dict(dtype=F32, x=A + 2), SHAPE)])
def test_rotary_refuses(over, status):
    ok = dict(plan=plan(), x=A, ldx=1024, y=A + MB, ldy=1024, heads=16, head_dim=64, rot_dim=32, layout=0,
              inv_freq=A + 2 * MB, amplitude=1.0, pos_start=A + 3 * MB, dtype=BF16, stream=None)
    over = dict(over)
    if over.pop("big", 0):
        over["plan"] = plan(total_tokens=2 ** 24 + 1)
    assert call("packed_rotary", ROTARY, ok, **over) == status
    assert call("packed_rotary", ROTARY, ok, plan=plan(total_tokens=0), x=None, y=None, inv_freq=None) == 0


LINEAR = ("x", "ldx", "x_scale", "w", "w_scale", "bias", "residual", "ldr", "act", "y", "ldy", "T", "K", "N", "dtype", "stream")
LINEAR_OK = dict(x=A, ldx=512, x_scale=A + MB, w=A + 2 * MB, w_scale=A + 3 * MB, bias=A + 4 * MB, residual=A + 5 * MB, ldr=264,
                 act=0, y=A + 6 * MB, ldy=264, T=4, K=512, N=264, dtype=BF16, stream=None)


@pytest.mark.parametrize("over,status", [
    (dict(dtype=7), DTYPE), (dict(T=-1), ARG), (dict(T=2 ** 31 - 1), ARG), (dict(N=2 ** 30 + 8), ARG), (dict(K=0), ARG), (dict(N=0), ARG), (dict(act=3), ARG), (dict(act=-1), ARG),
    (dict(K=520), SHAPE), (dict(K=131072, ldx=131072), SHAPE), (dict(N=260), SHAPE), (dict(x=None), ARG), (dict(w=None), ARG),
    (dict(x_scale=None), ARG), (dict(w_scale=None), ARG), (dict(ldx=496), SHAPE), (dict(ldx=520), SHAPE),
    (dict(ldx=1 << 22), SHAPE), (dict(x=A + 8), SHAPE), (dict(w=A + 2 * MB + 4), SHAPE), (dict(x_scale=A + MB + 1), SHAPE),
    (dict(w_scale=A + 3 * MB + 4), SHAPE), (dict(y=None), ARG), (dict(ldy=256), SHAPE), (dict(ldy=268), SHAPE),
    (dict(y=A + 6 * MB + 8), SHAPE), (dict(residual=A + 5 * MB + 8), SHAPE), (dict(ldr=256), SHAPE),
    (dict(bias=A + 4 * MB + 8), SHAPE), (dict(y=A), ARG), (dict(y=A + 2 * MB + 1024), ARG), (dict(y=A + 5 * MB, ldy=272), ARG),
    (dict(y=A + 5 * MB + 528), ARG), (dict(y=A + MB), ARG), (dict(y=A + 3 * MB), ARG), (dict(y=A + 4 * MB), ARG),
    (dict(dtype=F32, ldy=266), SHAPE)])
def test_linear_i8_refuses(over, status):
    assert call("packed_linear_i8", LINEAR, LINEAR_OK, **over) == status
    assert call("packed_linear_i8", LINEAR, LINEAR_OK, T=0, x=None, w=None, y=None, x_scale=None, w_scale=None) == 0


WINDOW = ("plan", "q", "ldq", "k", "ldk", "v", "ldv", "kv_heads", "head_dim", "scale", "window", "sinks", "out", "ldo", "ws",
          "ws_bytes", "dtype", "stream")
CACHED = WINDOW[:7] + ("kv_rows", "kv_first", "kv_len", "max_kv_len") + WINDOW[7:]


def window_ok():
    return dict(plan=plan(), q=A, ldq=512, k=A + MB, ldk=128, v=A + 2 * MB, ldv=128, kv_heads=2, head_dim=64, scale=0.125,
                window=100, sinks=4, out=A + 3 * MB, ldo=512, ws=None, ws_bytes=0, dtype=BF16, stream=None, kv_rows=4096,
                kv_first=A + 4 * MB, kv_len=A + 5 * MB, max_kv_len=128)


@pytest.mark.parametrize("over,status", [
    (dict(plan=None), ARG), (dict(dtype=9), DTYPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(kv_heads=16), SHAPE),
    (dict(window=-1), ARG), (dict(sinks=-1), ARG), (dict(head_dim=128), SHAPE), (dict(scale=float("nan")), ARG),
    (dict(q=None), ARG), (dict(k=None), ARG), (dict(v=None), ARG), (dict(out=None), ARG), (dict(ldq=504), SHAPE),
    (dict(ldq=516), SHAPE), (dict(ldk=120), SHAPE), (dict(ldv=124), SHAPE), (dict(ldo=256), SHAPE), (dict(q=A + 8), SHAPE),
    (dict(k=A + MB + 2), SHAPE), (dict(v=A + 2 * MB + 8), SHAPE), (dict(out=A + 3 * MB + 4), SHAPE), (dict(ldk=1 << 22), SHAPE),
    (dict(ldo=1 << 22), SHAPE), (dict(out=A), ARG), (dict(out=A + MB), ARG), (dict(out=A + 2 * MB + 512), ARG),
    (dict(dtype=F32, ldk=126 + 4), SHAPE), (dict(dtype=F32, q=A + 4), SHAPE)])
def test_window_refuses(over, status):
    ok = window_ok()
    assert call("ragged_attention_window", WINDOW, ok, **over) == status
    assert call("ragged_attention_window_cached", CACHED, ok, **over) == status


@pytest.mark.parametrize("over,status", [
    (dict(kv_rows=-1), ARG), (dict(kv_rows=1 << 41), ARG), (dict(kv_first=None), ARG), (dict(kv_len=None), ARG),
    (dict(kv_first=A + 4 * MB + 4), ARG), (dict(kv_len=A + 5 * MB + 2), ARG), (dict(max_kv_len=-1), ARG),
    (dict(out=A + 4 * MB, kv_first=A + 4 * MB + 1024), ARG), (dict(kv_len=A + 3 * MB + 4), ARG),
    # one token of each of four sequences over long caches is split and needs its workspace
    (dict(short=1, max_kv_len=100000, window=2 ** 31 - 1), WS), (dict(short=1, max_kv_len=100000, window=50000, ws=A + 6 * MB, ws_bytes=1000), WS),
    (dict(short=1, max_kv_len=100000, window=50000, ws=None, ws_bytes=1 << 30), ARG),
    (dict(short=1, max_kv_len=100000, window=50000, ws=A + 6 * MB + 8, ws_bytes=1 << 30), ARG),
    (dict(short=1, max_kv_len=100000, window=50000, ws=A + 2 * MB, ws_bytes=1 << 30), ARG),
    (dict(short=1, max_kv_len=100000, window=50000, ws=A + 3 * MB, ws_bytes=1 << 30), ARG)])
def test_cached_window_refuses(over, status):
    over = dict(over)
    if over.pop("short", 0):
        over["plan"] = plan(total_tokens=4, max_len=1)
    assert call("ragged_attention_window_cached", CACHED, window_ok(), **over) == status


def test_window_workspace():
    f = lib().ragged_attention_window_workspace
    n = ctypes.c_size_t()
    assert f(plan(), 128, 2, 100, 4, BF16, ctypes.byref(n)) == 0
    assert f(plan(total_tokens=4, max_len=1), 100000, 2, 50000, 4, BF16, ctypes.byref(n)) == 0 and n.value > 0
    big = n.value
    assert f(plan(total_tokens=4, max_len=1), 100000, 2, 64, 4, BF16, ctypes.byref(n)) == 0 and n.value < big
    assert f(plan(total_tokens=0, max_len=0), 0, 2, 64, 4, F32, ctypes.byref(n)) == 0 and n.value == 0
    assert f(plan(), 128, 2, 100, 4, BF16, None) == ARG
    assert f(plan(), 128, 3, 100, 4, BF16, ctypes.byref(n)) == SHAPE
    assert f(plan(), 128, 2, -1, 4, BF16, ctypes.byref(n)) == ARG
    assert f(plan(), -1, 2, 1, 4, BF16, ctypes.byref(n)) == ARG
    assert f(plan(total_tokens=2 ** 24 + 1, max_len=2 ** 12), 128, 2, 1, 4, BF16, ctypes.byref(n)) == ARG
    assert f(plan(), 2 ** 30 + 1, 2, 1, 4, BF16, ctypes.byref(n)) == ARG
    assert f(plan(total_tokens=2 ** 24, max_len=2 ** 12, heads=256), 128, 1, 1, 4, BF16, ctypes.byref(n)) == SHAPE
    assert f(plan(heads=32769), 128, 1, 1, 4, BF16, ctypes.byref(n)) == SHAPE
    assert f(plan(), 128, 2, 100, 4, 5, ctypes.byref(n)) == DTYPE


def test_nothing_to_attend():
    ok = dict(window_ok(), plan=plan(total_tokens=0, max_len=0), q=None, k=None, v=None, out=None)
    assert call("ragged_attention_window", WINDOW, ok) == 0
    assert call("ragged_attention_window_cached", CACHED, ok) == 0
