"""packed_rmsnorm and packed_quantize_i8 against their definitions in 64 bits.

Tolerances.  h = x + r is one fp32 sum rounded once more to the type: half a step of the
type and half a step of fp32 of |h|.  The norm's relative error: the fp32 sum of d squares (d / lanes
sequential terms and a tree, at most 70 + 8 roundings for d <= 16384), half of it by the square root,
and about six roundings of the products, under 50 half steps of fp32; y adds its own half step.
8-bit rows: q differs from the definition only where y / scale lies within 127 * 52 half
steps of fp32 (below 2^-11) of a border, and then by one; scale to 52 half steps."""
import numpy as np
import pytest
import torch

from tests import plain64 as P

pytestmark = pytest.mark.gpu
F32 = 2.0 ** -24
NEAR = 2.0 ** -11


def check_rows(q, scale, y):
    rq, rs, margin = P.eight(y)
    q, scale = q.cpu().double(), scale.cpu().double()
    assert ((scale - rs).abs() <= 52 * F32 * rs).all()
    diff = (q - rq).abs()
    assert (diff <= (margin < NEAR)).all(), (diff - (margin < NEAR)).max()


def check_y(y, ref, dtype):
    err = (y.cpu().double() - ref).abs()
    assert (err <= (P.HALF[dtype] + 51 * F32) * ref.abs()).all(), float((err / ref.abs().clamp_min(1e-300)).max())


def call(T, d, dtype, residual, x_out, y, q, pad=0, seed=0, std=1.0, eps=1e-6):
    import paper_2110_10221_amd as rag

    print(f"rmsnorm {dtype} T={T} d={d} residual={residual} sum={x_out} y={y} q={q} pad={pad}", flush=True)
    x = P.normal(seed, T, d, dtype=dtype, std=std)
    r = P.normal(seed + 1, T, d, dtype=dtype, std=2.0 * std) if residual else None
    g = P.normal(seed + 2, d, dtype=dtype)
    xd = P.strided(x, pad)
    rd = P.strided(r, pad) if residual else None
    nan = torch.full((T, d), float("nan"), dtype=P.TYPES[dtype])
    out = {"x_out": P.strided(nan, pad) if x_out else None, "y": P.strided(nan, pad) if y else None,
           "q": P.strided(torch.full((T, d), -77, dtype=torch.int8), pad) if q else None,
           "q_scale": torch.full((T,), -1.0, device="cuda") if q else None}
    rag.packed_rmsnorm(xd, g.cuda(), out["y"], eps, rd, out["x_out"], out["q"], out["q_scale"])
    torch.cuda.synchronize()
    h, ref = P.rmsnorm(x, g, eps, r)
    if x_out:
        err = (out["x_out"].cpu().double() - h).abs()
        assert (err <= (P.HALF[dtype] + F32) * h.abs()).all()
    if y:
        check_y(out["y"], ref, dtype)
    if q:
        check_rows(out["q"], out["q_scale"], ref)
    for k in ("x_out", "y", "q"):  # the padding behind the rows is untouched
        if out[k] is not None and pad:
            whole = torch.as_strided(out[k], (T, d + pad), (d + pad, 1))
            tail = whole[:, d:].cpu()
            assert (tail == -99).all() if k == "q" else torch.isnan(tail.float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 64, 72, 512, 520, 1000, 1024, 1032, 2048, 4096, 4104, 8192, 16384])
def test_widths(dtype, d):
    call(5, d, dtype, True, True, True, True, seed=d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 255, 1001, 5000])
def test_rows(dtype, T):
    call(T, 264, dtype, True, False, False, True, seed=T)
    call(T, 1024, dtype, False, False, True, False, seed=T)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual,x_out,y,q", [(0, 0, 1, 0), (0, 1, 0, 1), (1, 0, 1, 1), (1, 1, 1, 0), (1, 1, 0, 1)])
def test_outputs_and_strides(dtype, residual, x_out, y, q):
    call(37, 328, dtype, residual, x_out, y, q, pad=24)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(dtype):
    import paper_2110_10221_amd as rag

    x, r, g = P.normal(1, 100, 1032, dtype=dtype), P.normal(2, 100, 1032, dtype=dtype), P.normal(3, 1032, dtype=dtype)
    h, ref = P.rmsnorm(x, g, 1e-5, r)
    xd, rd = x.cuda(), r.cuda()
    rag.packed_rmsnorm(xd, g.cuda(), xd, 1e-5, rd, rd)  # y into x, h into the residual
    check_y(xd, ref, dtype)
    assert ((rd.cpu().double() - h).abs() <= (P.HALF[dtype] + F32) * h.abs()).all()


@pytest.mark.parametrize("std", [1e-12, 1e-4, 1e15, 1e19, 1e36])
def test_magnitudes(std):
    # squares that vanish beside eps, and squares that pass the range of fp32
    call(9, 2056, "bf16", True, True, True, True, std=std, seed=5)
    call(9, 264, "f32", False, True, True, True, std=std, seed=6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_zeros_infinities_and_nan(dtype):
    import paper_2110_10221_amd as rag

    for d in (64, 2048):
        x = P.normal(7, 6, d, dtype=dtype)
        x[0] = 0.0
        x[1, 3] = float("inf")
        x[2, d - 1] = float("nan")
        x[3] = -0.0
        g = torch.ones(d, dtype=P.TYPES[dtype])
        y = torch.empty_like(x, device="cuda")
        q, s = torch.empty(6, d, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
        rag.packed_rmsnorm(x.cuda(), g.cuda(), y, q=q, q_scale=s)
        check = [(y.cpu(), q.cpu(), s.cpu())]
        rag.packed_quantize_i8(x.cuda(), q, s)
        check.append((x, q.cpu(), s.cpu()))
        for yy, qq, ss in check:
            assert ss[0] == 0 and ss[3] == 0 and (qq[[0, 3]] == 0).all() and (yy[[0, 3]] == 0).all()
            assert torch.isnan(ss[1:3]).all() and (qq[1:3] == 0).all()
            assert torch.isfinite(ss[4:]).all() and (qq[4:].abs().amax(1) == 127).all()
        assert torch.isnan(y.cpu()[1, 3]) and torch.isnan(y.cpu()[2].float()).all()
        assert torch.isfinite(y.cpu()[4:].float()).all()  # the rows beside them


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,std", [(1, 8, 1.0), (3, 520, 1e-30), (700, 4096, 3.0), (5, 16384, 1e30), (2, 40, 1e-36), (2, 64, 1e-38)])
def test_quantize(dtype, T, d, std):
    import paper_2110_10221_amd as rag

    x = P.normal(T + d, T, d, dtype=dtype, std=std)
    q, s = torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    rag.packed_quantize_i8(x.cuda(), q, s)
    check_rows(q, s, x.double())


def test_ties_go_to_even():
    import paper_2110_10221_amd as rag

    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5, -127.0]], device="cuda")
    q, s = torch.empty(1, 8, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    rag.packed_quantize_i8(x, q, s)
    assert q.cpu().tolist() == [[127, 0, 2, 2, 0, -2, 126, -127]] and s.item() == 1.0


def test_another_stream_and_a_replayed_graph():
    import paper_2110_10221_amd as rag

    x, g = P.normal(1, 33, 512).cuda(), P.normal(2, 512).cuda()
    y, ref = torch.empty_like(x), torch.empty_like(x)
    rag.packed_rmsnorm(x, g, ref)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    rag.packed_rmsnorm(x, g, y, stream=s)
    s.synchronize()
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rag.packed_rmsnorm(x, g, y)
    for i in range(3):
        x.copy_(P.normal(10 + i, 33, 512))
        graph.replay()
        rag.packed_rmsnorm(x, g, ref)
        torch.cuda.synchronize()
        assert torch.equal(y, ref)


def nearest_even(x):
    """127 x / max |x| of each row rounded to nearest even, in whole numbers: (q, whether it was a tie)."""
    top = x.double().abs().amax(1, keepdim=True)
    unit = torch.floor(torch.log2(top)) - 33  # values above half a step are multiples of 2^unit
    a, t = (torch.ldexp(v, -unit).trunc().to(torch.int64) for v in (x.double(), top))
    num = 254 * a.abs() + t  # q = floor(127 a / t + 1 / 2), less one at a tie with an odd one
    q, tie = num // (2 * t), num % (2 * t) == 0
    return (q - (tie & (q % 2 == 1)).to(torch.int64)) * torch.sign(a), tie


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_tie_of_short_significands_goes_to_even(dtype):
    # every pair of 8-bit significands (all of bf16's): 102 and 51 are 63.5 steps apart, whatever 127 / 102 is in fp32
    import paper_2110_10221_amd as rag

    top = torch.arange(128.0, 256.0).repeat_interleave(3)[:, None]
    x = torch.arange(0.0, 256.0) * torch.tensor([0.5, 1.0, -0.25]).repeat(128)[:, None]
    x = torch.cat([top, torch.where(x.abs() > top, 0.0, x), torch.zeros(384, 7)], dim=1).to(P.TYPES[dtype])
    ref, tie = nearest_even(x)
    assert tie.sum() > 200 and ref[3 * (204 - 128) + 1, 1 + 102] == 64
    q, s = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(384, device="cuda")
    rag.packed_quantize_i8(x.cuda(), q, s)
    assert torch.equal(q.cpu().to(torch.int64), ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,std", [(2000, 4096, 1.0), (300, 264, 1e-35), (300, 16384, 1e36)])
def test_integers_are_exact(dtype, T, d, std):
    import paper_2110_10221_amd as rag

    x = P.normal(T, T, d, dtype=dtype, std=std)
    q, s = torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    rag.packed_quantize_i8(x.cuda(), q, s)
    assert torch.equal(q.cpu().to(torch.int64), nearest_even(x)[0])


def test_integers_of_the_norm_are_exact():
    # in fp32 y is the unrounded norm, which q is taken from
    import paper_2110_10221_amd as rag

    x, g = P.normal(1, 500, 1028, dtype="f32").cuda(), P.normal(2, 1028, dtype="f32").cuda()
    y, q, s = torch.empty_like(x), torch.empty(500, 1028, dtype=torch.int8, device="cuda"), torch.empty(500, device="cuda")
    rag.packed_rmsnorm(x, g, y, q=q, q_scale=s)
    assert torch.equal(q.cpu().to(torch.int64), nearest_even(y.cpu())[0])


def test_the_largest_number_of_rows():
    # 2^24 rows of a workgroup each (43 GB): 2^32 threads
    import paper_2110_10221_amd as rag

    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free memory")
    T, d = 2 ** 24, 516
    x = torch.zeros(T, d, device="cuda")
    x[:, 0] = 127.0
    x[:, d - 1] = torch.arange(T, device="cuda") % 127
    q, s = torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    rag.packed_quantize_i8(x, q, s)
    assert (s == 1.0).all() and (q[:, 0] == 127).all() and (q[:, 1:d - 1] == 0).all()
    assert torch.equal(q[:, d - 1].long(), torch.arange(T, device="cuda") % 127)
    del x, q, s
    torch.cuda.empty_cache()
