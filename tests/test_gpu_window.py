"""ragged_attention_window and ragged_attention_window_cached against dense masked attention
in 64 bits (tolerance: plain64.window_tolerance), at the masks, lengths and layouts where
they can go wrong."""
import numpy as np
import pytest
import torch

from tests import plain64 as P

pytestmark = pytest.mark.gpu
ALL = 2 ** 31 - 1  # a window past every length


def make_plan(L, heads):
    import paper_2110_10221_amd as rag

    plan = rag.Plan(torch.tensor(L, dtype=torch.int32).cuda(), sum(L), max(L, default=0), heads)
    rag.ragged_offsets(plan)
    return plan


def place(t, pad, guard=64):
    """Rows on the device with NaN around and behind them."""
    n, w = t.shape
    whole = torch.full((n + 2 * guard, w + pad), float("nan"), dtype=t.dtype, device="cuda")
    view = whole[guard:guard + n, :w]
    view.copy_(t)
    return whole, view


def check(got, dtype, L, heads, kv_heads, q, k, v, first, kv_len, window, sinks, scale):
    ref, mag, bound, count = P.window_attention(L, heads, kv_heads, q, k, v, first, kv_len, window, sinks, scale)
    err = (got.cpu().double() - ref).abs()
    tol = P.window_tolerance(dtype, ref, mag, bound, count)
    assert torch.isfinite(got.cpu().float()).all()
    assert (err <= tol).all(), float((err - tol).max())
    return ref


def packed(L, heads, kv_heads, window, sinks, dtype, scale=0.125, pad=0, seed=0, qkv=None, std=1.0):
    import paper_2110_10221_amd as rag

    print(f"window {dtype} L={L[:6]} heads={heads}/{kv_heads} window={window} sinks={sinks} scale={scale} pad={pad}", flush=True)
    T = sum(L)
    q, k, v = qkv or (P.normal(seed, T, heads * 64, dtype=dtype, std=2 * std), P.normal(seed + 1, T, kv_heads * 64, dtype=dtype, std=std),
                      P.normal(seed + 2, T, kv_heads * 64, dtype=dtype))
    plan = make_plan(L, heads)
    whole, out = place(torch.full((T, heads * 64), float("nan"), dtype=q.dtype), pad)
    ws = torch.empty(rag.ragged_attention_window_workspace(plan, max(L, default=0), window, sinks, kv_heads, q.dtype),
                     dtype=torch.uint8, device="cuda")
    rag.ragged_attention_window(plan, place(q, pad)[1], place(k, pad)[1], place(v, pad)[1], out, scale, window, sinks, kv_heads,
                                workspace=ws)
    torch.cuda.synchronize()
    assert not plan.data_errors()
    back = whole.cpu().float()
    assert torch.isnan(back[:64]).all() and torch.isnan(back[64 + T:]).all() and torch.isnan(back[:, heads * 64:]).all()
    first = np.concatenate([[0], np.cumsum(L)[:-1]]).tolist()
    check(out, dtype, L, heads, kv_heads, q, k, v, first, L, window, sinks, scale)
    return out, ws.numel()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 0), (31, 4), (32, 0), (33, 1), (63, 0), (64, 37), (65, 64), (100, 3),
                                          (128, 200), (ALL, 0), (ALL, 5), (0, 1), (0, 40), (0, 0), (5, ALL)])
def test_windows_and_sinks(dtype, window, sinks):
    packed([1, 2, 31, 32, 33, 64, 65, 130, 0, 257], 2, 2, window, sinks, dtype, seed=window % 97 + sinks % 89)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 1), (6, 2), (10, 2), (16, 4), (8, 8), (7, 1), (64, 1), (65, 1)])
def test_shared_key_heads(dtype, heads, kv_heads):
    packed([3, 40, 1, 97], heads, kv_heads, 20, 2, dtype, seed=heads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.125, -0.3, 0.0, 1e-38, 3.0])
def test_scales_and_strides(dtype, scale):
    packed([70, 5, 33], 4, 2, 40, 4, dtype, scale, pad=24, seed=9)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_sequences(dtype):
    packed([1500, 3, 700], 4, 2, 300, 10, dtype, seed=1)
    packed([2000], 2, 1, ALL, 0, dtype, seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_rise(dtype):
    # every later chunk holds scores far above those before it, and below (scale < 0)
    from tests.helpers import rising_keys, values

    L = [300, 129]
    q, k, v = (torch.from_numpy(values(a, "bf16")).to(P.TYPES[dtype]) for a in rising_keys(L, 2, 16.0, 3))
    for scale in (0.125, -0.125):
        packed(L, 2, 2, 100, 3, dtype, scale, qkv=(q, k, v))
        packed(L, 2, 2, ALL, 0, dtype, scale, qkv=(q, k, v))


def test_an_open_window_is_the_causal_operator():
    import paper_2110_10221_amd as rag

    L = [64, 200, 1, 33]
    plan, T = make_plan(L, 4), sum(L)
    q, k, v = (P.normal(s, T, 256).cuda() for s in range(3))
    a, b = torch.empty_like(q), torch.empty_like(q)
    rag.ragged_attention_causal(plan, q, k, v, a, 0.125)
    rag.ragged_attention_window(plan, q, k, v, b, 0.125, ALL)
    # both round each exponential and the result once: 2 * (2^-8 sum p |v|) + 2 * 2^-8 |o|, |v| <= max
    assert (a.float() - b.float()).abs().max() <= 4 * 2.0 ** -8 * v.float().abs().max()


# --------------------------------------------------------------------------- over a cache

def cached(L, kv_len, heads, kv_heads, window, sinks, dtype, seed=0, pad=0, share=False, scale=0.125, max_kv=None, workspace=None):
    import paper_2110_10221_amd as rag

    print(f"cached {dtype} L={L[:6]} kv={kv_len[:6]} heads={heads}/{kv_heads} window={window} sinks={sinks}", flush=True)
    rng = np.random.default_rng(seed)
    T, B = sum(L), len(L)
    # sequences in a shuffled order with rows of NaN between them (share: all at one place)
    order, first, rows = rng.permutation(B), [0] * B, 5
    for b in order:
        first[b] = 5 if share else rows
        rows = max(rows, first[b] + kv_len[b] + int(rng.integers(0, 4)))
    q = P.normal(seed, T, heads * 64, dtype=dtype, std=2.0)
    k, v = (torch.full((rows + 3, kv_heads * 64), float("nan"), dtype=q.dtype) for _ in range(2))
    for b in range(B):
        s = slice(first[b], first[b] + kv_len[b])
        k[s], v[s] = (P.normal(seed + 1 + (0 if share else b) + i * 1000, max(kv_len) + 1, kv_heads * 64, dtype=dtype)[:kv_len[b]] for i in range(2))
    plan = make_plan(L, heads)
    whole, out = place(torch.full((T, heads * 64), float("nan"), dtype=q.dtype), pad)
    mk = max(kv_len) if max_kv is None else max_kv
    n = rag.ragged_attention_window_workspace(plan, mk, window, sinks, kv_heads, q.dtype)
    ws = torch.full((n // 4,), float("nan"), device="cuda")
    args = (place(q, pad)[1], place(k, pad)[1], place(v, pad)[1], torch.tensor(first).cuda(),
            torch.tensor(kv_len, dtype=torch.int32).cuda(), mk)
    rag.ragged_attention_window_cached(plan, *args, out, scale, window, sinks, kv_heads, workspace=ws)
    torch.cuda.synchronize()
    assert not plan.data_errors()
    back = whole.cpu().float()
    assert torch.isnan(back[:64]).all() and torch.isnan(back[64 + T:]).all() and torch.isnan(back[:, heads * 64:]).all()
    check(out, dtype, L, heads, kv_heads, q, k, v, first, kv_len, window, sinks, scale)
    return n, (plan, args, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (8, 2), (5, 1)])
@pytest.mark.parametrize("window,sinks", [(64, 4), (1, 0), (100, 0), (ALL, 0), (0, 3), (0, 0)])
def test_single_tokens(dtype, heads, kv_heads, window, sinks):
    cached([1] * 7, [1, 2, 33, 64, 100, 257, 640], heads, kv_heads, window, sinks, dtype, seed=heads + window % 91, pad=8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_few_tokens_and_continued_prompts(dtype):
    cached([2, 5, 70, 1, 33, 0], [300, 5, 91, 700, 34, 20], 4, 2, 50, 6, dtype, seed=3)
    cached([2, 5, 70, 1, 33, 0], [300, 5, 91, 700, 34, 20], 4, 2, ALL, 0, dtype, seed=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_before_the_first_key(dtype):
    # more queries than keys: the first ones see nothing and get zeros; no keys at all too
    _, (plan, args, out) = cached([6, 70, 3, 1], [2, 35, 0, 0], 2, 1, 40, 2, dtype, seed=5)
    o = out.cpu().float()
    assert (o[:4] == 0).all() and (o[6:41] == 0).all() and (o[76:] == 0).all() and (o[4:6] != 0).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,kv,heads,kv_heads,window,sinks", [
    ([1], [5000], 4, 1, ALL, 0), ([1], [3001], 8, 2, 2000, 5), ([1, 1, 1], [4097, 3, 900], 2, 2, ALL, 0),
    ([4, 1], [2500, 64], 6, 2, 1500, 40), ([40], [3000], 1, 1, ALL, 0), ([1], [2048], 1, 1, 1024, 0)])
def test_keys_split_over_workgroups(dtype, L, kv, heads, kv_heads, window, sinks):
    n, _ = cached(L, kv, heads, kv_heads, window, sinks, dtype, seed=len(L))
    assert n > 0  # the case is split


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_split_rows_that_see_nothing(dtype):
    n, _ = cached([1, 3, 2], [3000, 1, 0], 2, 1, ALL, 0, dtype, seed=8)
    assert n > 0
    n, _ = cached([1, 3], [3000, 2000], 2, 1, 0, 2000, dtype, seed=8)
    assert n > 0


def test_sequences_that_share_rows():
    cached([1, 2, 3], [500, 400, 300], 4, 2, 256, 4, "bf16", seed=6, share=True)


def test_rows_past_32_bit_offsets():
    # 1500 rows 2^21 bytes apart: keys past 2^31 bytes from the first
    import paper_2110_10221_amd as rag

    n, ld = 1500, 1 << 20
    big = torch.empty(n * ld, dtype=torch.bfloat16, device="cuda").view(n, ld)
    k, v, q = P.normal(1, n, 64), P.normal(2, n, 64), P.normal(3, 2, 64, std=2.0)
    big[:, :64], big[:, 64:128] = k.cuda(), v.cuda()
    plan, out = make_plan([2], 1), torch.empty(2, 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(rag.ragged_attention_window_workspace(plan, n, ALL, 0), dtype=torch.uint8, device="cuda")
    rag.ragged_attention_window_cached(plan, q.cuda(), big[:, :64], big[:, 64:128], torch.zeros(1, dtype=torch.int64).cuda(),
                                       torch.tensor([n], dtype=torch.int32).cuda(), n, out, 0.125, ALL, 0, workspace=ws)
    check(out, "bf16", [2], 1, 1, q, k, v, [0], [n], ALL, 0, 0.125)
    rag.ragged_attention_window_cached(plan, q.cuda(), big[:, :64], big[:, 64:128], torch.full((1,), 1100).cuda(),
                                       torch.tensor([400], dtype=torch.int32).cuda(), n, out, 0.125, 100, 3, workspace=ws)
    check(out, "bf16", [2], 1, 1, q, k, v, [1100], [400], 100, 3, 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", ["k", "v"])
def test_hidden_keys_do_not_reach_a_row(dtype, bad, where):
    # keys that are not finite: rows that see one may be anything, every other row is as ever
    import paper_2110_10221_amd as rag

    L, H, window, sinks = [150, 70], 2, 40, 3
    T = sum(L)
    q, k, v = (P.normal(s + 20, T, H * 64, dtype=dtype) for s in range(3))
    spots = [(0, 1), (0, 60), (0, 149), (1, 33)]
    dirty = {"k": k, "v": v}[where].clone()
    for b, j in spots:
        dirty[(0, 150)[b] + j, 5::7] = bad
    plan, out = make_plan(L, H), torch.empty(T, H * 64, dtype=q.dtype, device="cuda")
    rag.ragged_attention_window(plan, q.cuda(), (dirty if where == "k" else k).cuda(), (dirty if where == "v" else v).cuda(),
                                out, 0.125, window, sinks)
    ref, mag, bound, count = P.window_attention(L, H, H, q, k, v, [0, 150], L, window, sinks, 0.125)
    tol = P.window_tolerance(dtype, ref, mag, bound, count)
    sees = torch.zeros(T, dtype=torch.bool)
    for b, j in spots:
        for i in range(L[b]):
            if j <= i and (j > i - window or j < sinks):
                sees[(0, 150)[b] + i] = True
    got = out.cpu().double()
    assert ((got - ref).abs() <= tol)[~sees].all()
    if where == "v":  # those that see it, in its own channels only
        cols = torch.zeros(H * 64, dtype=torch.bool)
        cols[5::7] = True
        assert ((got - ref).abs() <= tol)[sees][:, ~cols].all()
        g = got[sees][:, cols]
        assert torch.isnan(g).all() if np.isnan(bad) else (torch.isnan(g) | (g == bad)).all()
        if not np.isnan(bad):
            assert (got[149, 5::7] == bad).any()
    elif np.isnan(bad):
        assert torch.isnan(got[sees]).any(1).all()


def test_single_tokens_repeat_the_prompt():
    # the rows of a prompt, one step at a time over its cache
    import paper_2110_10221_amd as rag

    n, H, kvh = 90, 4, 2
    q, k, v = P.normal(1, n, H * 64).cuda(), P.normal(2, n, kvh * 64).cuda(), P.normal(3, n, kvh * 64).cuda()
    plan, whole = make_plan([n], H), torch.empty(n, H * 64, dtype=torch.bfloat16, device="cuda")
    rag.ragged_attention_window(plan, q, k, v, whole, 0.125, 32, 2, kvh)
    one, step = make_plan([1], H), torch.empty(1, H * 64, dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(1, dtype=torch.int64).cuda()
    for i in range(n):
        rag.ragged_attention_window_cached(one, q[i:i + 1], k, v, zero, torch.tensor([i + 1], dtype=torch.int32).cuda(), n, step,
                                           0.125, 32, 2, kvh)
        assert (step[0].float() - whole[i].float()).abs().max() <= 4 * 2.0 ** -8 * v.float().abs().max()


@pytest.mark.parametrize("first,n", [(-1, 4), (0, -1), (0, 101), (97, 4), (101, 0), (2 ** 62, 1), (60, 64)])
def test_ranges_outside_the_cache(first, n):
    import paper_2110_10221_amd as rag

    plan = make_plan([1, 1], 2)
    q, k = torch.zeros(2, 128, device="cuda"), torch.zeros(100, 128, device="cuda")
    out = torch.empty_like(q)
    kv = torch.tensor([5, n], dtype=torch.int32).cuda()
    rag.ragged_attention_window_cached(plan, q, k, k, torch.tensor([0, first]).cuda(), kv, 100 if n != 64 else 50, out, 1.0, 10)
    assert plan.data_errors() == ["keys outside the cache"]
    out.fill_(7.0)
    rag.ragged_attention_window(plan, q, k[:2], k[:2], out, 1.0, 10)  # as every data error, until the plan is rebuilt
    assert (out == 7.0).all()
    rag.ragged_offsets(plan)
    rag.ragged_attention_window(plan, q, k[:2], k[:2], out, 1.0, 10)
    assert not plan.data_errors() and (out == 0.0).all()


def test_empty_batches():
    import paper_2110_10221_amd as rag

    plan = make_plan([0, 0], 2)
    e = torch.empty(0, 128, device="cuda")
    rag.ragged_attention_window(plan, e, e, e, e, 1.0, 10)
    rag.ragged_attention_window_cached(plan, e, e, e, torch.zeros(2, dtype=torch.int64).cuda(), torch.zeros(2, dtype=torch.int32).cuda(),
                                       0, e, 1.0, 10)
    plan = make_plan([2], 2)  # queries over an empty cache
    q, out = torch.ones(2, 128, device="cuda"), torch.ones(2, 128, device="cuda")
    rag.ragged_attention_window_cached(plan, q, e, e, torch.zeros(1, dtype=torch.int64).cuda(), torch.zeros(1, dtype=torch.int32).cuda(),
                                       0, out, 1.0, 10)
    torch.cuda.synchronize()
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replayed_graphs_and_two_calls_at_once(dtype):
    # split steps: two graphs with a workspace each, replayed beside eager calls as the cache grows
    import paper_2110_10221_amd as rag

    t, H = P.TYPES[dtype], 4
    plan = make_plan([1, 1], H)
    k, v = P.normal(1, 6000, 64, dtype=dtype).cuda(), P.normal(2, 6000, 64, dtype=dtype).cuda()
    first, kv = torch.tensor([0, 3000]).cuda(), torch.tensor([2000, 1000], dtype=torch.int32).cuda()
    n = rag.ragged_attention_window_workspace(plan, 3000, ALL, 0, 1, t)
    assert n > 0
    qs = [P.normal(s, 2, H * 64, dtype=dtype).cuda() for s in (3, 4)]
    outs = [torch.empty_like(qs[0]) for _ in range(2)]
    wss = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(3)]

    def go(i, out, ws, stream=None):
        rag.ragged_attention_window_cached(plan, qs[i], k, v, first, kv, 3000, out, 0.125, ALL, 0, 1, workspace=ws, stream=stream)

    go(0, outs[0], wss[0])
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            go(i, outs[i], wss[i])
        graphs.append(g)
    side, ref = torch.cuda.Stream(), [torch.empty_like(qs[0]) for _ in range(2)]
    for _ in range(4):
        kv += 7
        side.wait_stream(torch.cuda.current_stream())
        for g in graphs:
            g.replay()
        go(0, ref[0], wss[2], side)
        go(1, ref[1], wss[2], side)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], ref[0]) and torch.equal(outs[1], ref[1])


def test_windows_of_any_size():
    # Python integers past 32 bits are open windows, not wrapped ones
    import paper_2110_10221_amd as rag

    L = [100, 30]
    q, k, v = (P.normal(s, 130, 128).cuda() for s in range(3))
    outs = []
    for window, sinks in ((ALL, 0), (2 ** 31, 0), (2 ** 32 + 1, 0), (10 ** 15, 0), (3, 2 ** 32 + 1), (0, 10 ** 15)):
        plan, out = make_plan(L, 2), torch.empty_like(q)
        rag.ragged_attention_window(plan, q, k, v, out, 0.125, window, sinks)
        outs.append(out)
    assert all(torch.equal(o, outs[0]) for o in outs[1:4])
    tol = 4 * 2.0 ** -8 * v.float().abs().max()  # the others' masks are the same, their chunks in another order
    assert all((o.float() - outs[0].float()).abs().max() <= tol for o in outs[4:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,heads,kv_heads", [([64, 1, 0, 63], 2, 2), ([16, 3, 0, 1, 15], 8, 2), ([1, 0, 1, 1], 64, 1),
                                              ([1, 1, 1], 65, 1), ([8, 7, 0], 16, 2), ([4, 5], 16, 1)])
def test_rows_that_fill_one_tile(dtype, L, heads, kv_heads):
    # sequences whose rows of a key head are at most one tile (one entry in G launched), and just past it
    packed(L, heads, kv_heads, 9, 2, dtype, seed=heads)
    cached(L, [n + 37 * i for i, n in enumerate(L)], heads, kv_heads, 30, 2, dtype, seed=heads)


def test_many_sequences():
    rng = np.random.default_rng(5)
    cached([1] * 300, rng.integers(1, 90, 300).tolist(), 4, 2, 33, 4, "bf16", seed=1)
    packed(rng.integers(0, 40, 300).tolist(), 2, 1, 11, 1, "bf16", seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loose_bounds(dtype):
    # max_kv_len and the plan's max_len far above every length: splits without a chunk, entries without rows
    import paper_2110_10221_amd as rag

    n, _ = cached([1, 1], [40, 300], 4, 2, ALL, 0, dtype, seed=3, max_kv=100000)
    assert n > 0
    n, _ = cached([1, 2], [1, 2], 2, 1, 50000, 1, dtype, seed=3, max_kv=100000)
    assert n > 0
    L, T = [50, 3], 53
    plan = rag.Plan(torch.tensor(L, dtype=torch.int32).cuda(), T, 4000, 2)
    rag.ragged_offsets(plan)
    q, k, v = (P.normal(s, T, 128, dtype=dtype) for s in range(3))
    out = torch.empty(T, 128, dtype=q.dtype, device="cuda")
    ws = torch.empty(rag.ragged_attention_window_workspace(plan, 4000, ALL, 0, None, q.dtype), dtype=torch.uint8, device="cuda")
    rag.ragged_attention_window(plan, q.cuda(), k.cuda(), v.cuda(), out, 0.125, ALL, 0, workspace=ws)
    check(out, dtype, L, 2, 2, q, k, v, [0, 50], L, ALL, 0, 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_that_is_not_finite_stays_alone(dtype, bad):
    import paper_2110_10221_amd as rag

    L, H = [100, 30], 4
    q, k, v = P.normal(1, 130, H * 64, dtype=dtype), P.normal(2, 130, 128, dtype=dtype), P.normal(3, 130, 128, dtype=dtype)
    dirty = q.clone()
    dirty[50, 64 * 2 + 5] = bad  # token 50, head 2
    plan, out = make_plan(L, H), torch.empty(130, H * 64, dtype=q.dtype, device="cuda")
    rag.ragged_attention_window(plan, dirty.cuda(), k.cuda(), v.cuda(), out, 0.125, 40, 2, 2)
    ref, mag, bound, count = P.window_attention(L, H, 2, q, k, v, [0, 100], L, 40, 2, 0.125)
    ok = ((out.cpu().double() - ref).abs() <= P.window_tolerance(dtype, ref, mag, bound, count)).reshape(130, H, 64)
    rest = torch.ones(130, H, dtype=torch.bool)
    rest[50, 2] = False
    assert ok[rest].all()
    assert torch.isnan(out.cpu().reshape(130, H, 64)[50, 2].float()).all()


def test_a_range_outside_the_cache_with_split_keys():
    import paper_2110_10221_amd as rag

    plan = make_plan([1, 1], 2)
    q, k = torch.zeros(2, 128, device="cuda"), torch.zeros(4000, 128, device="cuda")
    n = rag.ragged_attention_window_workspace(plan, 4000, ALL, 0, None, torch.float32)
    assert n > 0
    out = torch.full_like(q, 7.0)
    rag.ragged_attention_window_cached(plan, q, k, k, torch.tensor([0, 3000]).cuda(),
                                       torch.tensor([4000, 1001], dtype=torch.int32).cuda(), 4000, out, 1.0, ALL,
                                       workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))
    assert plan.data_errors() == ["keys outside the cache"] and (out == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (8, 2), (12, 2), (16, 2), (10, 2)])
@pytest.mark.parametrize("window,sinks", [(45, 3), (ALL, 0)])
def test_groups_of_heads_over_several_tiles(dtype, heads, kv_heads, window, sinks):
    # rows of a key head one below, at and past multiples of 64 and 128, empty and single sequences between
    L = [1, 0, 31, 32, 33, 130, 16, 17, 64, 0, 65]
    packed(L, heads, kv_heads, window, sinks, dtype, seed=heads, pad=8)
    cached(L, [n + 29 * (i % 3) for i, n in enumerate(L)], heads, kv_heads, window, sinks, dtype, seed=heads + 1)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_hidden_values_in_groups_of_four(bad):
    import paper_2110_10221_amd as rag

    L, H, KV, window, sinks = [150, 70], 8, 2, 40, 3
    q, k, v = P.normal(31, 220, H * 64), P.normal(32, 220, KV * 64), P.normal(33, 220, KV * 64)
    spots = [(0, 1), (0, 60), (0, 149), (1, 33)]
    dirty = v.clone()
    for b, j in spots:
        dirty[(0, 150)[b] + j, 3::9] = bad
    plan, out = make_plan(L, H), torch.empty(220, H * 64, dtype=q.dtype, device="cuda")
    rag.ragged_attention_window(plan, q.cuda(), k.cuda(), dirty.cuda(), out, 0.125, window, sinks, KV)
    ref, mag, bound, count = P.window_attention(L, H, KV, q, k, v, [0, 150], L, window, sinks, 0.125)
    ok = (out.cpu().double() - ref).abs() <= P.window_tolerance("bf16", ref, mag, bound, count)
    sees = torch.zeros(220, dtype=torch.bool)
    for b, j in spots:
        for i in range(j, L[b]):
            if j > i - window or j < sinks:
                sees[(0, 150)[b] + i] = True
    cols = torch.zeros(KV, 64, dtype=torch.bool)
    cols.view(-1)[3::9] = True
    cols = cols.repeat_interleave(H // KV, 0).reshape(-1)  # a query head's channels are its key head's
    assert ok[~sees].all() and ok[sees][:, ~cols].all()
    assert not torch.isfinite(out.cpu().float()[sees][:, cols]).any()


@pytest.mark.parametrize("L,kv_len,heads,kv_heads,window", [
    ([200, 65], None, 2, 2, 100), ([200, 65], None, 8, 2, ALL), ([1, 1, 2], [700, 33, 64], 8, 2, ALL), ([1], [5000], 4, 1, ALL)])
def test_exponentials_are_not_rounded_to_the_type(L, kv_len, heads, kv_heads, window):
    # plain64's fp32 tolerance, 2^-16 of each exponential (a half step of bf16, twice) and the half step of the result
    import paper_2110_10221_amd as rag

    n = kv_len or L
    first, T, rows = np.concatenate([[0], np.cumsum(n)[:-1]]).tolist(), sum(L), sum(n)
    q, k, v = P.normal(1, T, heads * 64, std=2.0), P.normal(2, rows, kv_heads * 64), P.normal(3, rows, kv_heads * 64)
    plan, out = make_plan(L, heads), torch.empty(T, heads * 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(rag.ragged_attention_window_workspace(plan, max(n), window, 2, kv_heads), dtype=torch.uint8, device="cuda")
    if kv_len:
        rag.ragged_attention_window_cached(plan, q.cuda(), k.cuda(), v.cuda(), torch.tensor(first).cuda(),
                                           torch.tensor(n, dtype=torch.int32).cuda(), max(n), out, 0.125, window, 2, kv_heads, workspace=ws)
    else:
        rag.ragged_attention_window(plan, q.cuda(), k.cuda(), v.cuda(), out, 0.125, window, 2, kv_heads, workspace=ws)
    ref, mag, bound, count = P.window_attention(L, heads, kv_heads, q, k, v, first, n, window, 2, 0.125)
    tol = P.window_tolerance("f32", ref, mag, bound, count) + 2.0 ** -16 * mag + P.HALF["bf16"] * ref.abs()
    assert ((out.cpu().double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, 1e-36, -1e-35])
def test_small_scales_of_large_products(dtype, scale):
    # products of about 1e35: uniform weights at a scale of zero, ordinary scores at the others
    L, H = [70, 33, 1], 2
    q, k = (P.normal(s, sum(L), H * 64, dtype=dtype, std=1e17) for s in (1, 2))
    v = P.normal(3, sum(L), H * 64, dtype=dtype)
    packed(L, H, H, 40, 2, dtype, scale, qkv=(q, k, v))
    packed(L, H, H, ALL, 0, dtype, scale, qkv=(q, k, v))
    cached([1, 3], [90, 33], H, H, 40, 2, dtype, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_scale_of_zero_keeps_what_is_not_finite(dtype, bad):
    import paper_2110_10221_amd as rag

    q, k, v = (P.normal(s, 50, 128, dtype=dtype) for s in range(3))
    q[20, 64 + 7] = bad  # token 20, head 1
    plan, out = make_plan([50], 2), torch.empty(50, 128, dtype=q.dtype, device="cuda")
    rag.ragged_attention_window(plan, q.cuda(), k.cuda(), v.cuda(), out, 0.0, 10, 1)
    nan = torch.isnan(out.cpu().float())
    assert nan[20, 64:].all() and nan.sum() == 64


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.125, 3.0])
@pytest.mark.parametrize("L,kv_len,window,sinks", [([300, 70], None, ALL, 0), ([300, 70], None, 150, 3), ([1, 3], [5000, 700], ALL, 0)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(dtype, scale, L, kv_len, window, sinks):
    # as they are, whatever the weight (those of scale 3 are too small for fp32 for many keys), in chunks that a row sees
    # whole, in cut ones and over split keys: infinity, minus infinity, NaN, and NaN where both infinities meet
    import paper_2110_10221_amd as rag

    H, KV, n = 8, 2, kv_len or L
    first, T, rows = np.concatenate([[0], np.cumsum(n)[:-1]]).tolist(), sum(L), sum(n)
    q, k, v = (P.normal(s, r, w, dtype=dtype, std=d) for s, r, w, d in ((1, T, H * 64, 2.0), (2, rows, KV * 64, 1.0), (3, rows, KV * 64, 1.0)))
    inf, nan = float("inf"), float("nan")
    bad = torch.zeros(rows, KV * 64, dtype=torch.float64)
    for b in range(len(n)):
        for channel, at in ((3, {20: inf}), (9, {40: -inf}), (17, {33: nan}), (30, {5: inf, 45: -inf}), (64 + 41, {n[b] - 1: inf}),
                            (64 + 50, {n[b] // 2: -inf, n[b] // 2 + 1: -inf})):
            for j, x in at.items():
                bad[first[b] + j, channel] = x
    dirty = torch.where(bad != 0, bad, v.double()).to(v.dtype)
    plan, out = make_plan(L, H), torch.empty(T, H * 64, dtype=q.dtype, device="cuda")
    ws = torch.empty(rag.ragged_attention_window_workspace(plan, max(n), window, sinks, KV, q.dtype), dtype=torch.uint8, device="cuda")
    if kv_len:
        assert ws.numel() > 0
        rag.ragged_attention_window_cached(plan, q.cuda(), k.cuda(), dirty.cuda(), torch.tensor(first).cuda(),
                                           torch.tensor(n, dtype=torch.int32).cuda(), max(n), out, scale, window, sinks, KV, workspace=ws)
    else:
        rag.ragged_attention_window(plan, q.cuda(), k.cuda(), dirty.cuda(), out, scale, window, sinks, KV, workspace=ws)
    clean = torch.where(bad != 0, 0.0, v.double()).to(v.dtype)
    ref, mag, bound, count = P.window_attention(L, H, KV, q, k, clean, first, n, window, sinks, scale)
    tol = P.window_tolerance(dtype, ref, mag, bound, count)
    got, t0 = out.cpu().double(), 0
    for b in range(len(n)):
        p, j = torch.arange(n[b] - L[b], n[b])[:, None], torch.arange(n[b])[None]
        seen = (j <= p) & ((j > p - window) | (j < sinks))
        x = bad[first[b]:first[b] + n[b]]
        some = lambda m: (seen.double() @ m.double()) > 0  # noqa: E731
        up, down, none = some(x == inf), some(x == -inf), some(torch.isnan(x))
        none = none | (up & down)
        want = torch.where(none, nan, torch.where(up, inf, torch.where(down, -inf, 0.0)))
        want = want.reshape(-1, KV, 1, 64).expand(-1, KV, H // KV, 64).reshape(L[b], H * 64)
        at = slice(t0, t0 + L[b])
        special = want != 0
        assert torch.equal(torch.nan_to_num(got[at][special], 7.0, 8.0, 9.0), torch.nan_to_num(want[special], 7.0, 8.0, 9.0))
        assert ((got[at] - ref[at]).abs() <= tol[at])[~special].all()
        t0 += L[b]
