"""rotary_frequencies on the host, against closed forms (no GPU needed)."""
import ctypes
import math
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2110_10221_amd", "libragged.so")),
                                reason="libragged.so not built")


def freq(*a, **k):
    import paper_2110_10221_amd as rag

    f, amp = rag.rotary_frequencies(*a, **k)
    return f.tolist(), amp


def near(a, b):
    return abs(a - b) <= 1e-13 * abs(b)


@pytest.mark.parametrize("R,base", [(2, 10000.0), (64, 10000.0), (30, 500000.0), (512, 1.5)])
def test_plain_linear_and_ntk(R, base):
    f, amp = freq(R, base)
    assert amp == 1.0 and len(f) == R // 2
    assert all(near(v, math.exp(-2 * i / R * math.log(base))) for i, v in enumerate(f))
    g, amp = freq(R, base, scaling=1, factor=4.0)
    assert amp == 1.0 and all(near(b * 4.0, a) for a, b in zip(f, g))
    n, amp = freq(R, base, scaling=2, factor=8.0)
    # the fastest pair keeps its frequency, the slowest is divided by the factor
    assert amp == 1.0 and n[0] == 1.0 and (R == 2 or abs(n[-1] * 8.0 / f[-1] - 1) < 1e-12)


@pytest.mark.parametrize("R,factor,orig", [(64, 32.0, 4096), (32, 2.0, 512), (128, 1.0, 8192), (2, 4.0, 100), (64, 4.0, 32)])
def test_yarn(R, factor, orig):
    f, _ = freq(R)
    y, amp = freq(R, scaling=3, factor=factor, orig_len=orig)
    assert near(amp, 0.1 * math.log(factor) + 1.0)
    lo = max(math.floor(R * math.log(orig / (32.0 * 2 * math.pi)) / (2 * math.log(10000.0))), 0)
    hi = min(math.ceil(R * math.log(orig / (1.0 * 2 * math.pi)) / (2 * math.log(10000.0))), R - 1)
    for i, (a, b) in enumerate(zip(f, y)):
        mix = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
        assert near(b, a * (1 - mix) + a / factor * mix)
        if i <= lo and hi > lo:
            assert b == a
        if i >= hi > lo:
            assert near(b, a / factor)


def test_refusals():
    import paper_2110_10221_amd as rag

    lib = rag.library()
    buf, amp = (ctypes.c_double * 256)(), ctypes.c_double()

    def call(R=64, base=10000.0, kind=0, factor=2.0, orig=4096, fast=32.0, slow=1.0, out=buf, a=amp):
        return lib.rotary_frequencies(R, base, kind, factor, orig, fast, slow, out, None if a is None else ctypes.addressof(a))

    assert call() == 0 and call(R=512) == 0 and call(R=2) == 0
    nan, inf = float("nan"), float("inf")
    assert call(kind=0, factor=nan) == 0  # not read
    for bad in (dict(R=0), dict(R=3), dict(R=-2), dict(R=514)):
        assert call(**bad) == rag_shape()
    for bad in (dict(base=1.0), dict(base=nan), dict(base=inf), dict(kind=4), dict(kind=-1), dict(out=None), dict(a=None),
                dict(kind=1, factor=0.5), dict(kind=2, factor=nan), dict(kind=3, factor=inf), dict(kind=3, orig=0),
                dict(kind=3, slow=0.0), dict(kind=3, fast=0.5), dict(kind=3, fast=nan), dict(kind=3, fast=inf),
                dict(kind=2, R=4, base=1e200, factor=1e200)):
        assert call(**bad) == -1, bad


def rag_shape():
    return -3
