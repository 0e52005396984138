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


def kernel(T, K, N, act=0, bf16=True):
    import paper_2110_10221_amd as rag

    f = rag.library()._ZN3rag16linear_kernel_i8Elllibl  # rag::linear_kernel_i8
    f.restype = ctypes.c_int
    f.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int, ctypes.c_bool, ctypes.c_int64]
    return f(T, K, N, act, bf16, 256)


NA = float("inf")  # more tokens than that kernel takes


@needs_lib
@pytest.mark.parametrize("T,K,N,act,bf16,us", [
    # us of each kernel, weights out of the caches: few tokens, 32 x 32, 32 x 64 with six and with four stages, 64 x 64, 64 x 128,
    # 128 x 128, 256 x 256 (not timed up to 16 tokens from 64 x 128 on)
    (1, 8192, 8192, 0, True, (14.99, 14.86, 15.65, 19.7, 27.64)),
    (8, 8192, 8192, 0, True, (16.1, 14.84, 16.08, 19.7, 27.58)),
    (16, 8192, 8192, 0, True, (19.23, 14.87, 16.97, 19.92, 27.65)),
    (1, 16384, 4096, 0, True, (16.17, 21.75, 23.76, 32.3, 48.04)),
    (16, 4096, 16384, 0, True, (20.38, 18.73, 16.29, 16.66, 17.76)),
    (4, 1024, 4096, 0, True, (3.19, 3.81, 3.94, 4.02, 4.73)),
    (16, 4096, 4096, 0, True, (7.04, 7.73, 9.24, 10.63, 14.51)),
    (32, 4096, 4096, 0, True, (NA, 8.08, 10.21, 11.04, 14.63, 17.48, 30.92, 17.25)),
    (32, 1024, 1024, 0, True, (NA, 3.81, 3.95, 3.92, 4.58, 5.47, 7.49, 6.4)),
    (32, 16384, 4096, 0, True, (NA, 22.98, 29.98, 34.03, 48.56, 57.31, 110.85, 56.82)),
    (17, 8192, 8192, 0, True, (NA, 15.04, 17.21, 20.02, 27.8, 31.65, 59.13, 31.06)),
    (64, 2048, 8192, 0, True, (NA, 7.89, 6.83, 7.07, 9.38, 11.39, 17.31, 11.34)),
    (64, 8192, 2048, 0, True, (NA, 12.27, 16.01, 18.21, 26.85, 32.49, 58.66, 30.93)),
    (100, 4096, 4096, 0, True, (NA, 10.09, 8.74, 10.46, 14.76, 17.76, 31.75, 19.6)),
    (160, 4096, 1024, 0, True, (NA, 7.11, 7.38, 7.89, 11.07, 13.56, 23.71, 16.88)),
    (160, 1024, 4096, 0, True, (NA, 5.52, 5.64, 5.15, 5.25, 6.27, 8.6, 7.66)),
    (2237, 2048, 512, 0, True, (NA, 11.4, 10.05, 8.94, 8.13, 8.39, 13.13, 10.59)),
    # (with the last ones' weights in the caches)
    (2237, 2048, 512, 0, False, (NA, 11.57, 10.69, 9.52, 8.68, 9.21, 14.31, 11.78)),
    (144, 7760, 3080, 0, False, (NA, 24.32, 19.53, 19.61, 25.41, 38.56, 64.42, 42.26)),
    (35475, 4096, 1024, 0, True, (NA, 404.92, 334.2, 324.74, 230.34, 193.75, 170.79, 143.78)),
    (35475, 1024, 4096, 1, True, (NA, 650.55, 532.53, 403.4, 290.21, 266.28, 229.29, 237.7)),
    (8192, 8192, 8192, 0, True, (NA, 1286.63, 1068.33, 1066.92, 815.03, 661.45, 529.09, 429.18))])
def test_no_kernel_runs_that_is_much_slower(T, K, N, act, bf16, us):
    assert us[kernel(T, K, N, act, bf16)] <= 1.1 * min(us)
