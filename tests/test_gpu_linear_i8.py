"""packed_linear_i8 against exact integer sums and its epilogue in 64 bits.

Tolerance.  The sums are exact.  Their conversion, two scales and the bias are four
roundings to fp32 (half steps of 2^-24) of |x_scale w_scale sum|, one of |bias| and one of the
result z; an activation passes them on by at most 1.13 and adds its own error, at most
12 half steps of |z| (erf to 1.5e-7, tanh and erff to two steps, all times z / 2, and their products);
the residual's sum half a step of each term, and the type half a step of the result."""
import pytest
import torch

from tests import plain64 as P

pytestmark = pytest.mark.gpu
F32 = 2.0 ** -24


def int8(seed, rows, K, std=40.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, K, generator=g) * std).round().clamp(-128, 127).to(torch.int8)


def scales(seed, n):
    g = torch.Generator().manual_seed(seed)
    return 0.5 + torch.rand(n, generator=g)


def call(T, K, N, dtype="bf16", act=0, bias=True, residual=False, in_place=False, pad=0, seed=0, x=None, w=None):
    import paper_2110_10221_amd as rag

    print(f"linear_i8 {dtype} T={T} K={K} N={N} act={act} bias={bias} residual={residual} in_place={in_place} pad={pad}",
          flush=True)
    x = int8(seed, T, K) if x is None else x
    w = int8(seed + 1, N, K) if w is None else w
    xs, ws = scales(seed + 2, T) / 40.0, scales(seed + 3, N) / (40.0 * K ** 0.5)
    b = P.normal(seed + 4, N, dtype=dtype, std=0.5) if bias else None
    r = P.normal(seed + 5, T, N, dtype=dtype) if residual else None
    guard = 4096
    t = P.TYPES[dtype]
    whole = torch.full((2 * guard + T * (N + pad),), float("nan"), dtype=t, device="cuda")
    y = whole[guard:guard + T * (N + pad)].view(T, N + pad)[:, :N]
    if in_place:
        y.copy_(r)
    rd = None if r is None else y if in_place else P.strided(r, pad)
    rag.packed_linear_i8(P.strided(x, 2 * pad), xs.cuda(), w.cuda(), ws.cuda(), y, None if b is None else b.cuda(), rd, act)
    torch.cuda.synchronize()
    got = y.cpu().double()
    back = whole.cpu().float()
    assert torch.isnan(back[:guard]).all() and torch.isnan(back[guard + T * (N + pad):]).all()
    if pad:
        assert torch.isnan(back[guard:guard + T * (N + pad)].view(T, N + pad)[:, N:]).all()
    lin = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()
    z = lin + (0.0 if b is None else b.double())
    a = P.gelu(z, act)
    ref = a + (0.0 if r is None else r.double())
    tol = F32 * (1.13 * (4 * lin.abs() + (0.0 if b is None else b.double().abs()) + z.abs()) + (12 * z.abs() if act else 0.0)
                 + 2 * ref.abs() + a.abs()) + P.HALF[dtype] * ref.abs()
    err = (got - ref).abs()
    assert torch.isfinite(got).all() and (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("bias,residual", [(True, True), (True, False), (False, True), (False, False)])
def test_epilogues(dtype, act, bias, residual):
    call(150, 192, 328, dtype, act, bias, residual, seed=act)
    call(7, 192, 328, dtype, act, bias, residual, seed=act)


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 33, 48, 63, 64, 65, 100, 129, 257])
@pytest.mark.parametrize("K,N", [(16, 8), (48, 24), (128, 64), (144, 136), (272, 1000), (1040, 72), (2048, 520)])
def test_sizes(T, K, N):
    call(T, K, N, "f32" if (T + N) % 3 == 0 else "bf16", residual=T % 2 == 1, seed=T + K + N)


@pytest.mark.parametrize("T,K,N", [(2237, 2048, 512), (2237, 512, 2048), (600, 16384, 256), (1111, 1024, 1032), (3, 16384, 4096),
                                   (5000, 256, 1000), (40, 8208, 2048), (4097, 1152, 776), (300, 112, 8200)])
def test_larger_shapes(T, K, N):
    call(T, K, N, "bf16", act=1, seed=K)
    call(T, K, N, "f32", residual=True, seed=K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [5, 40, 333])
def test_strides_and_in_place(dtype, T):
    call(T, 208, 264, dtype, 1, True, True, pad=8, seed=1)
    call(T, 208, 264, dtype, 1, True, True, in_place=True, seed=2)
    call(T, 208, 264, dtype, 0, True, True, in_place=True, pad=24, seed=3)


@pytest.mark.parametrize("T", [3, 20, 130])
def test_largest_sums(T):
    # every product at its largest, up to 2^31 - 2^18: no sum may wrap or lose a bit
    import paper_2110_10221_amd as rag

    K, N = rag.RAG_I8_MAX_K, 16
    x = torch.full((T, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    x[-1, -1] = -127
    one = torch.ones(max(T, N), device="cuda")
    y = torch.empty(T, N, device="cuda")
    rag.packed_linear_i8(x, one[:T], w, one[:N], y)
    ref = torch.full((T, N), 16384.0 * K, dtype=torch.float64)
    ref[:, 1::2] = -128.0 * 127 * K
    ref[-1, ::2] -= 128
    ref[-1, 1::2] += 127
    assert torch.equal(y.cpu(), ref.float())


@pytest.mark.parametrize("T", [4, 70])
def test_a_row_without_a_scale(T):
    # scale NaN (a row that held an infinity or a NaN) reaches that token's outputs only
    import paper_2110_10221_amd as rag

    x, w = int8(1, T, 64).cuda(), int8(2, 40, 64).cuda()
    xs, ws = torch.ones(T, device="cuda"), torch.ones(40, device="cuda")
    xs[1] = float("nan")
    ws[3] = 0.0
    y = torch.empty(T, 40, device="cuda")
    rag.packed_linear_i8(x, xs, w, ws, y)
    y = y.cpu()
    assert torch.isnan(y[1]).all() and torch.isfinite(y[[0, 2, 3]]).all() and (y[[0, 2], 3] == 0).all()


def test_empty_batch():
    import paper_2110_10221_amd as rag

    x = torch.empty(0, 64, dtype=torch.int8, device="cuda")
    w = torch.zeros(8, 64, dtype=torch.int8, device="cuda")
    rag.packed_linear_i8(x, torch.empty(0, device="cuda"), w, torch.ones(8, device="cuda"), torch.empty(0, 8, device="cuda"))
    torch.cuda.synchronize()


@pytest.mark.parametrize("T", [2, 200])
def test_a_replayed_graph_and_two_streams(T):
    import paper_2110_10221_amd as rag

    K, N = 512, 256
    x, w = int8(1, T, K).cuda(), int8(2, N, K).cuda()
    xs, ws = scales(3, T).cuda(), scales(4, N).cuda()
    y, ref, z = (torch.empty(T, N, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    rag.packed_linear_i8(x, xs, w, ws, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rag.packed_linear_i8(x, xs, w, ws, y)
    side = torch.cuda.Stream()
    for i in range(3):
        x.copy_(int8(10 + i, T, K))
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        rag.packed_linear_i8(x, xs, w, ws, z, stream=side)
        rag.packed_linear_i8(x, xs, w, ws, ref)
        torch.cuda.synchronize()
        assert torch.equal(y, ref) and torch.equal(z, ref)


@pytest.mark.parametrize("T,K,N,form,form32", [
    (16, 528, 264, 0, 0), (17, 528, 264, 1, 1), (40, 4112, 2056, 1, 1), (300, 400, 2056, 2, 2), (700, 1040, 2104, 3, 3),
    (2900, 1552, 2104, 4, 4), (5200, 1552, 4104, 5, 5), (4300, 4112, 2312, 4, 5)])
def test_every_form(T, K, N, form, form32):
    # ragged edges in every dimension on each of the tile forms; 5200 x 4104 is 357 256 x 256 tiles,
    # 256 whole and 101 in quarters, 4300 x 2312 is 170, in fp32 all in quarters
    import ctypes

    import paper_2110_10221_amd as rag

    f = rag.library()._ZN3rag14linear_form_i8Elllibl  # rag::linear_form_i8
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_int64] * 3 + [ctypes.c_int, ctypes.c_bool, ctypes.c_int64]
    assert f(T, K, N, 0, True, 256) == form and f(T, K, N, 2, False, 256) == form32
    call(T, K, N, "bf16", 0, True, True, seed=form)
    call(T, K, N, "f32", 2, True, False, seed=form)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,K,N", [(33, 1040, 2104), (33, 1040, 4104), (20, 528, 20000), (9, 528, 8192), (16, 784, 8200), (8, 528, 8192),
                                   (17, 16, 264), (12, 48, 8200), (20, 896, 40), (25, 752, 16424)])
def test_tiles_of_32_tokens(T, K, N, dtype):
    # one round of 32 x 32 tiles, one of 32 x 64, several (20000, 16424 features); up to 16 tokens with a GPU full of
    # tiles and without; reductions shorter than the stages, of as many steps, of one more
    call(T, K, N, dtype, 1, True, True, seed=T)
    call(T, K, N, dtype, 0, False, False, seed=T + 1, pad=16)


def test_the_largest_outputs():
    # 2^36 features of tokens (137 GB) in 2^24 tiles of 256 threads
    import paper_2110_10221_amd as rag

    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 200 << 30:
        pytest.skip("needs 200 GB of free memory")
    T, K, N = 4096, 16, 2 ** 24
    a, b = torch.arange(T, device="cuda") % 5 + 1, torch.arange(N, device="cuda") % 7 + 1
    x, w = (v.to(torch.int8)[:, None].expand(-1, K).contiguous() for v in (a, b))
    y = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
    rag.packed_linear_i8(x, torch.ones(T, device="cuda"), w, torch.ones(N, device="cuda"), y)
    for i in range(5):
        row = (16 * (i + 1) * b).to(torch.bfloat16)  # (whole numbers of at most eight bits)
        for t in range(i, T, 1000):
            assert (y[t:t + 1000:5] == row).all()
    del x, w, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 40, 300])
def test_scales_near_the_range(T, dtype):
    # sum * x_scale passes fp32's range, sum * x_scale * w_scale does not; a sum of zero stays zero
    import paper_2110_10221_amd as rag

    K, N = 256, 264
    x, w, b = int8(1, T, K), int8(2, N, K), P.normal(3, N, dtype=dtype)
    x[1] = 0
    xs, ws = scales(4, T) * 2e36, scales(5, N) * 1e-10
    xs[::2] *= -1e-30
    w[5], ws[5] = 0, 3e38
    y = torch.empty(T, N, dtype=P.TYPES[dtype], device="cuda")
    rag.packed_linear_i8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), y, b.cuda())
    lin = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()
    ref = lin + b.double()
    tol = F32 * (4 * lin.abs() + b.double().abs() + 2 * ref.abs()) + P.HALF[dtype] * ref.abs()
    assert ((y.cpu().double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("odd", [float("nan"), float("inf"), 2e36])
@pytest.mark.parametrize("T", [4, 70])
def test_a_token_does_not_depend_on_its_neighbours_scales(T, odd):
    import paper_2110_10221_amd as rag

    x, w = int8(1, T, 272).cuda(), int8(2, 264, 272).cuda()
    xs, ws = scales(3, T).cuda(), scales(4, 264).cuda()
    outs = []
    for scale in (1.0, odd):
        xs[1] = scale
        y = torch.empty(T, 264, device="cuda")
        rag.packed_linear_i8(x, xs, w, ws, y, P.normal(5, 264, dtype="f32").cuda())
        outs.append(y.cpu())
    rest = torch.arange(T) != 1
    assert torch.equal(outs[0][rest], outs[1][rest])
