"""The tile form a packed_linear_i8 call takes (host arithmetic, no GPU needed), at sizes where every
form was timed: the rule must not name one measured more than a tenth slower than the fastest."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
needs_lib = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2110_10221_amd", "libragged.so")),
                               reason="libragged.so not built")


def form(T, K, N, act=0, bf16=True):
    import paper_2110_10221_amd as rag

    f = rag.library()._ZN3rag14linear_form_i8Elllibl  # rag::linear_form_i8
    f.restype = ctypes.c_int
    f.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int, ctypes.c_bool, ctypes.c_int64]
    return f(T, K, N, act, bf16, 256)


@needs_lib
@pytest.mark.parametrize("T,K,N,act,bf16,us", [
    # us on forms 1 .. 5: 32 x 64, 64 x 64, 64 x 128, 128 x 128, 256 x 256
    (35475, 4096, 1024, 0, True, (336.2, 224.8, 189.9, 168.4, 140.4)),
    (35475, 1024, 4096, 1, True, (394.6, 290.6, 264.1, 224.6, 229.3)),
    (35475, 1024, 1024, 0, True, (93.3, 68.9, 63.6, 53.8, 49.9)),
    (2237, 2048, 512, 0, False, (9.6, 8.9, 9.1, 14.7, 12.2)),
    (8192, 8192, 8192, 0, True, (1056.5, 821.3, 652.6, 532.4, 413.5)),
    (445, 4784, 2992, 2, True, (24.5, 23.3, 22.1, 37.4, 30.1)),
    (179, 1040, 3336, 0, True, (6.2, 5.7, 7.4, 10.9, 9.1)),
    (144, 7760, 3080, 0, False, (14.8, 20.2, 28.3, 52.1, 36.7)),
    (27, 1040, 456, 2, True, (5.5, 6.1, 7.2, 9.1, 8.0)),
    (4678, 2944, 2520, 0, False, (77.4, 57.9, 49.0, 47.0, 49.7)),
    (32, 4096, 3760, 0, True, (7.8, 10.3, 12.4, 22.1, 16.3))])
def test_no_form_is_named_that_is_much_slower(T, K, N, act, bf16, us):
    assert us[form(T, K, N, act, bf16) - 1] <= 1.1 * min(us)


@needs_lib
def test_few_tokens_and_extreme_sizes():
    assert all(form(t, k, n) == 0 for t in (1, 16) for k in (16, 131056) for n in (8, 2 ** 31 - 8))
    assert all(1 <= form(t, k, n) <= 5 for t in (17, 2 ** 31 - 1) for k in (16, 131056) for n in (8, 2 ** 31 - 8))
