"""packed_rotary against complex multiplication in 64 bits.

Tolerance, relative to the pair's length M = amplitude * sqrt(a^2 + b^2), in half steps of
fp32 (2^-24): the reduced angle in fp32 1.6, sine and cosine 4, the amplitude's own rounding 1 and
its product 1, two products and a sum 3, together under 12; the type's half step of the result; and for position p
the two fp64 products' roundings, p * 2^-51 of an angle at most."""
import numpy as np
import pytest
import torch

from tests import plain64 as P

pytestmark = pytest.mark.gpu


def positions(L, start):
    return torch.cat([torch.arange(n) + s for n, s in zip(L, start)]).double()


def call(L, heads, D, R, dtype, half, start=None, inverse=False, pad=0, in_place=False, amplitude=1.0, offset=0, seed=0):
    import paper_2110_10221_amd as rag

    print(f"rotary {dtype} L={L[:4]}.. heads={heads} D={D} R={R} half={half} start={start} inverse={inverse} pad={pad} "
          f"in_place={in_place} offset={offset}", flush=True)
    T, w = sum(L), heads * D
    plan = rag.Plan(torch.tensor(L, dtype=torch.int32).cuda(), T, max(L), 1)
    rag.ragged_offsets(plan)
    freq, _ = rag.rotary_frequencies(R)
    x = P.normal(seed, T, w, dtype=dtype)
    whole = torch.full((T, w + pad), float("nan"), dtype=x.dtype, device="cuda")
    xd = whole[:, offset:offset + w]
    xd.copy_(x)
    if in_place:
        y = xd
    else:
        out = torch.full((T, w + pad), float("nan"), dtype=x.dtype, device="cuda")
        y = out[:, offset:offset + w]
    ps = None if start is None else torch.tensor(start, dtype=torch.int32).cuda()
    rag.packed_rotary(plan, xd, y, freq.cuda(), heads, D, rag.RAG_ROTARY_HALF if half else rag.RAG_ROTARY_INTERLEAVED,
                      amplitude, ps, inverse)
    torch.cuda.synchronize()
    assert not plan.data_errors()
    pos = positions(L, start or [0] * len(L))
    ref = P.rotary(x, pos, freq, amplitude, heads, D, half, inverse)
    M = P.rotary((x.double().abs()), pos * 0, freq, amplitude, heads, D, half).reshape(T, heads, D)
    h = R // 2
    a, b = (M[..., :h], M[..., h:R]) if half else (M[..., 0:R:2], M[..., 1:R:2])
    n = torch.sqrt(a * a + b * b)
    if half:
        M[..., :h] = M[..., h:R] = n
    else:
        M[..., 0:R:2] = M[..., 1:R:2] = n
    M[..., R:] = 0  # the rest passes unchanged
    tol = M.reshape(T, w) * (12 * 2.0 ** -24 + pos.abs()[:, None] * 2.0 ** -51) + P.HALF[dtype] * ref.abs()
    err = (y.cpu().double() - ref).abs()
    assert (err <= tol).all(), float((err - tol).max())
    back = (whole if in_place else out).cpu().float()
    assert torch.isnan(back[:, :offset]).all() and torch.isnan(back[:, offset + w:]).all()
    if R < D:
        rest = y.cpu().reshape(T, heads, D)[..., R:]
        assert torch.equal(rest, x.reshape(T, heads, D)[..., R:])
    return y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("D,R", [(64, 64), (64, 32), (64, 16), (128, 128), (96, 96), (64, 20), (80, 42), (6, 2), (2, 2),
                                 (7, 4), (512, 512), (256, 64)])
def test_heads_and_turned_parts(dtype, half, D, R):
    call([3, 1, 17], 3, D, R, dtype, half, seed=D + R)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("R", [64, 24])
def test_in_place_strided_inverse_and_starts(dtype, half, R):
    L = [5, 0, 1, 70, 33]
    start = [0, 9, 1000, 4095, 131071]
    call(L, 4, 64, R, dtype, half, start, pad=64, in_place=True)
    call(L, 4, 64, R, dtype, half, start, inverse=True, pad=16, amplitude=1.25)
    call(L, 4, 64, R, dtype, half, pad=5, offset=3)  # unaligned rows
    call(L, 4, 64, R, dtype, half, pad=8, offset=8)


@pytest.mark.parametrize("half", [True, False])
def test_far_and_negative_positions(half):
    call([1, 1, 2, 1], 2, 64, 64, "f32", half, [1000003, 2 ** 31 - 2, -5, -2 ** 31], seed=4)


def test_batches():
    rng = np.random.default_rng(3)
    call(rng.integers(0, 40, 300).tolist(), 1, 64, 64, "bf16", True)
    call([1] * 257, 20, 64, 32, "bf16", False, rng.integers(0, 10 ** 6, 257).tolist())
    call([4001], 2, 64, 64, "f32", True)


def test_turning_back_is_the_gradient_and_the_inverse():
    import paper_2110_10221_amd as rag

    L = [40, 7]
    plan = rag.Plan(torch.tensor(L, dtype=torch.int32).cuda(), 47, 40, 2)
    rag.ragged_offsets(plan)
    f, amp = rag.rotary_frequencies(64, scaling=rag.RAG_ROTARY_YARN, factor=4.0, orig_len=32)
    x, g = P.normal(1, 47, 128, dtype="f32").cuda(), P.normal(2, 47, 128, dtype="f32").cuda()
    y, gx, z = (torch.empty_like(x) for _ in range(3))
    rag.packed_rotary(plan, x, y, f.cuda(), 2, amplitude=amp)
    rag.packed_rotary(plan, g, gx, f.cuda(), 2, amplitude=amp, inverse=True)
    # <g, R x> = <R^T g, x>: 47 * 128 terms of order 1, each to a dozen half steps of fp32
    a, b = (g.double() * y.double()).sum(), (gx.double() * x.double()).sum()
    assert abs(a - b) <= 47 * 128 * 4 * 24 * 2.0 ** -24
    rag.packed_rotary(plan, y, z, f.cuda(), 2, amplitude=1.0 / amp, inverse=True)
    assert (z - x).abs().max() <= 24 * 2.0 ** -24 * 2 * x.abs().max()


def test_nothing_is_written_after_a_data_error():
    import paper_2110_10221_amd as rag

    plan = rag.Plan(torch.tensor([3, 5], dtype=torch.int32).cuda(), 9, 5, 1)  # the lengths sum to 8
    rag.ragged_offsets(plan)
    f, _ = rag.rotary_frequencies(64)
    x, y = torch.zeros(9, 64, device="cuda"), torch.full((9, 64), 7.0, device="cuda")
    rag.packed_rotary(plan, x, y, f.cuda(), 1)
    assert plan.data_errors() and (y == 7.0).all()


def test_empty_batch():
    import paper_2110_10221_amd as rag

    plan = rag.Plan(torch.zeros(2, dtype=torch.int32).cuda(), 0, 0, 1)
    rag.ragged_offsets(plan)
    x = torch.empty(0, 64, device="cuda")
    rag.packed_rotary(plan, x, x, rag.rotary_frequencies(64)[0].cuda(), 1)
    torch.cuda.synchronize()


def test_a_replayed_graph():
    import paper_2110_10221_amd as rag

    plan = rag.Plan(torch.ones(8, dtype=torch.int32).cuda(), 8, 1, 1)
    rag.ragged_offsets(plan)
    f = rag.rotary_frequencies(64)[0].cuda()
    x, pos = P.normal(3, 8, 640).cuda(), torch.arange(8, dtype=torch.int32).cuda()
    y, ref = torch.empty_like(x), torch.empty_like(x)
    rag.packed_rotary(plan, x, y, f, 10, pos_start=pos)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rag.packed_rotary(plan, x, y, f, 10, pos_start=pos)
    for i in range(3):
        pos += 100
        graph.replay()
        rag.packed_rotary(plan, x, ref, f, 10, pos_start=pos)
        torch.cuda.synchronize()
        assert torch.equal(y, ref)
