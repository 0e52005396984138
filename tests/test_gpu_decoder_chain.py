"""The 8-bit decoder operators together, as a layer uses them:
    rmsnorm (8 bits) -> linear_i8 (QKV) -> rotary on the Q and K columns, in place -> window attention
    -> quantize -> linear_i8 (output projection) + residual -> rmsnorm (sum and 8 bits) -> linear_i8 (GELU)
    -> quantize -> linear_i8
Each stage is compared with its 64-bit form on the values that the stage before it stored, so that the
tolerances are the single operators' own; and the whole, captured into a graph and replayed, with itself."""
import pytest
import torch

from tests import plain64 as P

pytestmark = pytest.mark.gpu
F32 = 2.0 ** -24
H, KVH, D, FF = 4, 2, 256, 512
W = (H + 2 * KVH) * 64


class Layer:
    """Weights and buffers of one layer over T tokens."""

    def __init__(self, T, dtype, seed=0):
        import paper_2110_10221_amd as rag

        self.rag, self.T, self.dtype = rag, T, dtype
        t = P.TYPES[dtype]
        self.w, self.ws = {}, {}
        for i, (n, shape) in enumerate(dict(qkv=(W, D), o=(D, H * 64), up=(FF, D), down=(D, FF)).items()):
            w = P.normal(seed + i, *shape, dtype=dtype, std=shape[1] ** -0.5).cuda()
            self.w[n] = torch.empty(shape, dtype=torch.int8, device="cuda")
            self.ws[n] = torch.empty(shape[0], device="cuda")
            rag.packed_quantize_i8(w, self.w[n], self.ws[n])
        self.g1, self.g2 = (P.normal(seed + 9 + i, D, dtype=dtype).cuda() for i in range(2))
        self.freq = rag.rotary_frequencies(64)[0].cuda()

        def e(w, k=t):
            return torch.empty(T, w, dtype=k, device="cuda")

        self.q1, self.q2, self.q3, self.q4 = e(D, torch.int8), e(H * 64, torch.int8), e(D, torch.int8), e(FF, torch.int8)
        self.s1, self.s2, self.s3, self.s4 = (torch.empty(T, device="cuda") for _ in range(4))
        self.qkv, self.att, self.proj, self.sum, self.up, self.y = e(W), e(H * 64), e(D), e(D), e(FF), e(D)

    def run(self, plan, x, window, sinks, pos_start=None, cache=None, keep=None):
        """`cache`: (k, v, first, kv_len, max_kv, rows of the new tokens); `keep`: receives copies of what later stages
        overwrite."""
        r = self.rag
        r.packed_rmsnorm(x, self.g1, q=self.q1, q_scale=self.s1)
        r.packed_linear_i8(self.q1, self.s1, self.w["qkv"], self.ws["qkv"], self.qkv)
        if keep is not None:
            keep["qkv"] = self.qkv.clone()
        qk = self.qkv[:, :(H + KVH) * 64]
        r.packed_rotary(plan, qk, qk, self.freq, H + KVH, pos_start=pos_start)
        q, k, v = self.qkv[:, :H * 64], self.qkv[:, H * 64:(H + KVH) * 64], self.qkv[:, (H + KVH) * 64:]
        if cache is None:
            r.ragged_attention_window(plan, q, k, v, self.att, 0.125, window, sinks, KVH)
        else:
            ck, cv, first, kv_len, max_kv, rows = cache
            ck[rows], cv[rows] = k, v
            n = r.ragged_attention_window_workspace(plan, max_kv, window, sinks, KVH, x.dtype)
            ws = torch.empty(n, dtype=torch.uint8, device="cuda")
            r.ragged_attention_window_cached(plan, q, ck, cv, first, kv_len, max_kv, self.att, 0.125, window, sinks, KVH,
                                             workspace=ws)
        r.packed_quantize_i8(self.att, self.q2, self.s2)
        r.packed_linear_i8(self.q2, self.s2, self.w["o"], self.ws["o"], self.proj)
        r.packed_rmsnorm(self.proj, self.g2, residual=x, x_out=self.sum, q=self.q3, q_scale=self.s3)
        r.packed_linear_i8(self.q3, self.s3, self.w["up"], self.ws["up"], self.up, act=r.RAG_ACT_GELU_ERF)
        r.packed_quantize_i8(self.up, self.q4, self.s4)
        r.packed_linear_i8(self.q4, self.s4, self.w["down"], self.ws["down"], self.y, residual=self.sum)


def rows_close(q, s, y):
    rq, rs, margin = P.eight(y)
    assert ((s.cpu().double() - rs).abs() <= 52 * F32 * rs).all()
    assert ((q.cpu().double() - rq).abs() <= (margin < 2.0 ** -11)).all()


def linear_close(layer, q, s, name, y, act=0, residual=None):
    lin = (q.cpu().double() @ layer.w[name].cpu().double().t()) * s.cpu().double()[:, None] * layer.ws[name].cpu().double()
    a = P.gelu(lin, act)
    ref = a + (0.0 if residual is None else residual.cpu().double())
    tol = F32 * (6 * lin.abs() + (12 * lin.abs() if act else 0.0) + 2 * ref.abs() + a.abs()) + P.HALF[layer.dtype] * ref.abs()
    assert ((y.cpu().double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L", [[70, 1, 129, 0, 33], [5]])
def test_stages(dtype, L):
    import paper_2110_10221_amd as rag

    T, window, sinks = sum(L), 40, 3
    plan = rag.Plan(torch.tensor(L, dtype=torch.int32).cuda(), T, max(L), H)
    rag.ragged_offsets(plan)
    layer, x, keep = Layer(T, dtype), P.normal(77, T, D, dtype=dtype, std=2.0).cuda(), {}
    layer.run(plan, x, window, sinks, keep=keep)
    torch.cuda.synchronize()
    assert not plan.data_errors()
    rows_close(layer.q1, layer.s1, P.rmsnorm(x.cpu(), layer.g1.cpu(), 1e-6)[1])
    linear_close(layer, layer.q1, layer.s1, "qkv", keep["qkv"])
    pos = torch.cat([torch.arange(n) for n in L])
    raw, n = keep["qkv"].cpu(), (H + KVH) * 64
    turned = P.rotary(raw[:, :n], pos, layer.freq.cpu(), 1.0, H + KVH, 64, True)
    reach = P.rotary(raw[:, :n].double().abs(), pos * 0, layer.freq.cpu(), 1.0, H + KVH, 64, True).reshape(T, -1, 2, 32)
    reach = reach.pow(2).sum(2, keepdim=True).sqrt().expand(-1, -1, 2, -1).reshape(T, n)
    got = layer.qkv.cpu().double()
    assert ((got[:, :n] - turned).abs() <= 12 * F32 * reach + P.HALF[dtype] * turned.abs()).all()
    assert torch.equal(layer.qkv[:, n:].cpu(), raw[:, n:])
    c = layer.qkv.cpu()
    first = [sum(L[:i]) for i in range(len(L))]
    ref = P.window_attention(L, H, KVH, c[:, :H * 64], c[:, H * 64:n], c[:, n:], first, L, window, sinks, 0.125)
    assert ((layer.att.cpu().double() - ref[0]).abs() <= P.window_tolerance(dtype, *ref)).all()
    rows_close(layer.q2, layer.s2, layer.att.cpu().double())
    linear_close(layer, layer.q2, layer.s2, "o", layer.proj)
    h, y = P.rmsnorm(layer.proj.cpu(), layer.g2.cpu(), 1e-6, x.cpu())
    assert ((layer.sum.cpu().double() - h).abs() <= (P.HALF[dtype] + F32) * h.abs()).all()
    rows_close(layer.q3, layer.s3, y)
    linear_close(layer, layer.q3, layer.s3, "up", layer.up, act=1)
    rows_close(layer.q4, layer.s4, layer.up.cpu().double())
    linear_close(layer, layer.q4, layer.s4, "down", layer.y, residual=layer.sum)


def test_a_captured_layer():
    import paper_2110_10221_amd as rag

    L = [70, 1, 129, 33]
    T = sum(L)
    plan = rag.Plan(torch.tensor(L, dtype=torch.int32).cuda(), T, max(L), H)
    rag.ragged_offsets(plan)
    layer, other, x = Layer(T, "bf16"), Layer(T, "bf16"), P.normal(5, T, D).cuda()
    layer.run(plan, x, 40, 3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run(plan, x, 40, 3)
    for i in range(3):
        x.copy_(P.normal(6 + i, T, D))
        graph.replay()
        other.run(plan, x, 40, 3)
        torch.cuda.synchronize()
        assert torch.equal(layer.y, other.y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_over_a_cache_continue_a_prompt(dtype):
    """The last tokens of a prompt, once with it and once one by one over a cache: the same keys, values and
    queries up to the 8-bit and type roundings of rows that are computed alone or among others, which are the
    same arithmetic; attention sums in another order, so its bound is twice the operator's tolerance."""
    import paper_2110_10221_amd as rag

    n, m, window, sinks = 60, 52, 20, 2  # m tokens at once, then single ones
    x = P.normal(3, n, D, dtype=dtype).cuda()
    whole, first = Layer(n, dtype), Layer(m, dtype)
    plan = rag.Plan(torch.tensor([n], dtype=torch.int32).cuda(), n, n, H)
    rag.ragged_offsets(plan)
    whole.run(plan, x, window, sinks)
    ck, cv = (torch.full((200, KVH * 64), float("nan"), dtype=x.dtype, device="cuda") for _ in range(2))
    base = torch.tensor([100], dtype=torch.int64).cuda()

    def tokens(layer, i0, i1):
        plan = rag.Plan(torch.tensor([i1 - i0], dtype=torch.int32).cuda(), i1 - i0, i1 - i0, H)
        rag.ragged_offsets(plan)
        layer.run(plan, x[i0:i1], window, sinks, torch.tensor([i0], dtype=torch.int32).cuda(),
                  (ck, cv, base, torch.tensor([i1], dtype=torch.int32).cuda(), n, slice(100 + i0, 100 + i1)))
        torch.cuda.synchronize()
        assert not plan.data_errors()

    tokens(first, 0, m)
    step = Layer(1, dtype)
    c = whole.qkv.cpu()
    k = (H + KVH) * 64
    ref = P.window_attention([n], H, KVH, c[:, :H * 64], c[:, H * 64:k], c[:, k:], [0], [n], window, sinks, 0.125)
    tol = 2 * P.window_tolerance(dtype, *ref)
    assert ((first.att.cpu().double() - whole.att[:m].cpu().double()).abs() <= tol[:m]).all()
    for i in range(m, n):
        tokens(step, i, i + 1)
        assert torch.equal(step.qkv[0], whole.qkv[i])
        assert ((step.att[0].cpu().double() - whole.att[i].cpu().double()).abs() <= tol[i]).all()
