"""The operators around a decoder's packed attention in 8 bits, as cases to time and compare.

    packed_rmsnorm            RMS norm with the residual's addition, output in the activations' type or in 8 bits
    packed_quantize_i8        8-bit integers with one scale for each token
    packed_linear_i8          matrix product of 8-bit integers with scales for each token and channel
    packed_rotary             rotary positions of packed queries and keys
    ragged_attention_window   causal attention with a sliding window and first tokens that stay visible,
                              over the packed batch or over a cache (`_cached`)

`run` makes one call of one of them: the library's where `own` is true, else its plain form in elementary torch
operations (32 bits; angles in 64), rounded once at the end.  8-bit outputs are returned as the values they
stand for, in bfloat16.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "gelu", "gelu_tanh")


def listed():
    return [
        # One step of eight sequences through a d_model 1024 layer: latency.
        dict(name="rmsnorm_step", op="rmsnorm", dtype="bf16", T=8, d=1024, residual=True, i8=False),
        # The batch-128, d_model 1024 layer's tokens: residual added, 8 bits for the projection that follows.
        dict(name="rmsnorm_batch128", op="rmsnorm", dtype="bf16", T=35475, d=1024, residual=True, i8=True),
        # Attention output of the fp32 batch-32 lognormal layer, an odd number of tokens.
        dict(name="quantize_f32", op="quantize", dtype="f32", T=2237, d=512),
        # The same layer's FFN activations at batch 128.
        dict(name="quantize_ffn", op="quantize", dtype="bf16", T=35475, d=4096),
        # FF1 of one step of four sequences: the weights' bytes.
        dict(name="linear_step", op="linear", dtype="bf16", T=4, K=1024, N=4096, act="gelu", residual=False),
        # FF2 of the batch-32 lognormal layer with fp32 outputs, odd token count.
        dict(name="linear_f32", op="linear", dtype="f32", T=2237, K=2048, N=512, act="none", residual=True),
        # FF2 of the batch-128 layer.
        dict(name="linear_ffn", op="linear", dtype="bf16", T=35475, K=4096, N=1024, act="none", residual=True),
        # Single tokens of 32 sequences far into their contexts, half of each head turned, pairs interleaved.
        dict(name="rotary_step", op="rotary", dtype="bf16", B=32, lo=1, hi=1, far=131072, heads=20, head_dim=64,
             rot_dim=32, layout="interleaved", scaling="yarn", inverse=False, lseed=1),
        # Queries and keys of the batch-128 layer (16 + 16 heads).
        dict(name="rotary_batch128", op="rotary", dtype="bf16", B=128, lo=32, hi=512, far=0, heads=32, head_dim=64,
             rot_dim=64, layout="half", scaling="none", inverse=False, lseed=2),
        # The batch-32 SDPA shape in fp32 with a short window.
        dict(name="window_f32", op="window", dtype="f32", B=32, lo=16, hi=512, far=0, heads=8, kv_heads=8, window=96,
             sinks=4, lseed=3),
        # Long prompts, four query heads to a key head.
        dict(name="window_prompts", op="window", dtype="bf16", B=6, lo=1500, hi=8192, far=0, heads=16, kv_heads=4,
             window=1024, sinks=4, lseed=4),
        # One token of each of 32 sequences over caches of up to 32768 tokens.
        dict(name="window_step", op="window", dtype="bf16", B=32, lo=1, hi=1, far=32768, heads=16, kv_heads=4,
             window=4096, sinks=4, lseed=5),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rmsnorm", "quantize", "linear", "linear", "rotary", "window", "window"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("rmsnorm", "quantize"):
        d = 8 * _log(rng, 8, 1024)
        c = dict(op=op, dtype=dtype, T=_log(rng, 1, min(35475, 35475 * 1024 // d)), d=d)
        if op == "rmsnorm":
            c.update(residual=rng.random() < 0.7, i8=rng.random() < 0.5)
        return c
    if op == "linear":
        K, N = 16 * _log(rng, 4, 512), 8 * _log(rng, 8, 1024)
        T = _log(rng, 1, 40000)
        T = max(1, min(T, 35475 * 4096 * 1024 // (2 * K * N)))
        return dict(op=op, dtype=dtype, T=T, K=K, N=N, act=rng.choice(ACTS), residual=rng.random() < 0.5)
    if op == "rotary":
        head_dim = rng.choice([32, 64, 64, 128, 96])
        step = rng.random() < 0.4
        return dict(op=op, dtype=dtype, B=_log(rng, 1, 128), lo=1, hi=1 if step else _log(rng, 16, 512),
                    far=_log(rng, 100, 1000000) if step or rng.random() < 0.3 else 0, heads=rng.randint(1, 15),
                    head_dim=head_dim, rot_dim=rng.choice([head_dim, head_dim, head_dim // 2, 2 * rng.randint(1, head_dim // 2)]),
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "ntk", "yarn"]),
                    inverse=rng.random() < 0.3, lseed=rng.randint(10, 10 ** 6))
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 5] if kv_heads < 8 else [1, 2])
    # a window now and then far past every length: plain causal attention
    window, sinks = (_log(rng, 16, 4096) if rng.random() < 0.85 else 10 ** 9), rng.choice([0, 1, 4, 37])
    if rng.random() < 0.5:  # a step over a cache
        return dict(op=op, dtype=dtype, B=_log(rng, 1, 32), lo=1, hi=rng.choice([1, 1, 4]), far=_log(rng, 16, 32768),
                    heads=heads, kv_heads=kv_heads, window=window, sinks=sinks, lseed=rng.randint(10, 10 ** 6))
    hi = _log(rng, 16, 2048)
    return dict(op=op, dtype=dtype, B=max(1, min(_log(rng, 1, 64), 8192 // hi)), lo=rng.randint(1, hi), hi=hi, far=0,
                heads=heads, kv_heads=kv_heads, window=window, sinks=sinks, lseed=rng.randint(10, 10 ** 6))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _lengths(case):
    """Token counts and, before each sequence's first token, the tokens it already has."""
    r = random.Random(case["lseed"])
    L = [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    past = [r.randint(case["far"] // 8, case["far"] - 1) if case["far"] else 0 for _ in L]
    return L, past


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(t)

    op = case["op"]
    if op == "rmsnorm":
        T, d = case["T"], case["d"]
        return dict(x=normal(T, d), residual=normal(T, d, std=2.0) if case["residual"] else None,
                    gamma=(1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t))
    if op == "quantize":
        x = torch.randn(case["T"], case["d"], generator=g, device="cuda")
        return dict(x=(x * torch.sigmoid(1.7 * x)).to(t))  # as an activation leaves it
    if op == "linear":
        T, K, N = case["T"], case["K"], case["N"]

        def int8(rows):
            return torch.randn(rows, K, generator=g, device="cuda").mul_(40.0).round_().clamp_(-127, 127).to(torch.int8)

        x, w = int8(T), int8(N)
        spread = 0.5 + torch.rand(T + N, generator=g, device="cuda")
        return dict(x=x, w=w, x_scale=spread[:T] / 40.0, w_scale=spread[T:] / (40.0 * math.sqrt(K)),
                    bias=normal(N, std=0.1), residual=normal(T, N) if case["residual"] else None)
    L, past = _lengths(case)
    if op == "rotary":
        return dict(x=normal(sum(L), case["heads"] * case["head_dim"]), L=L, past=past)
    rows = sum(a + b for a, b in zip(L, past))
    w, kw = 64 * case["heads"], 64 * case["kv_heads"]
    return dict(q=normal(sum(L), w, std=2.0), k=normal(rows, kw), v=normal(rows, kw), L=L, past=past)


SCALINGS = {"none": dict(), "linear": dict(factor=4.0), "ntk": dict(factor=8.0),
            "yarn": dict(factor=32.0, orig_len=4096, beta_fast=32.0, beta_slow=1.0)}
BASE = 10000.0


def _frequencies(rot_dim, scaling):
    """Angle per position of each pair, and the factor on the turned channels (plain form)."""
    s = SCALINGS[scaling]
    e = torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim
    if scaling == "linear":
        return BASE ** -e / s["factor"], 1.0
    if scaling == "ntk":
        return (BASE * s["factor"] ** (rot_dim / (rot_dim - 2)) if rot_dim > 2 else BASE) ** -e, 1.0
    if scaling == "yarn":
        def pair(turns):  # the pair that turns so often over the original length
            return rot_dim * math.log(s["orig_len"] / (turns * 2 * math.pi)) / (2 * math.log(BASE))
        lo = max(math.floor(pair(s["beta_fast"])), 0)
        hi = min(math.ceil(pair(s["beta_slow"])), rot_dim - 1)
        ramp = ((torch.arange(rot_dim // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = BASE ** -e
        return f * (1 - ramp) + f / s["factor"] * ramp, 0.1 * math.log(s["factor"]) + 1.0
    return BASE ** -e, 1.0


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    op = case["op"]
    if op == "rotary" and not own:
        f, s["amplitude"] = _frequencies(case["rot_dim"], case["scaling"])
        s["freq"] = f.cuda()
        s["pos"] = torch.cat([torch.arange(p, p + n, dtype=torch.float64) for n, p in zip(s["L"], s["past"])]).cuda()
    if own:
        import paper_2110_10221_amd as rag
        if op == "rotary":
            kind = {"none": rag.RAG_ROTARY_PLAIN, "linear": rag.RAG_ROTARY_LINEAR, "ntk": rag.RAG_ROTARY_NTK,
                    "yarn": rag.RAG_ROTARY_YARN}[case["scaling"]]
            f, s["amplitude"] = rag.rotary_frequencies(case["rot_dim"], BASE, kind, **SCALINGS[case["scaling"]])
            s["freq"] = f.cuda()
        if op in ("rotary", "window"):
            L = torch.tensor(s["L"], dtype=torch.int32).cuda()
            s["plan"] = rag.Plan(L, sum(s["L"]), max(s["L"]), case["heads"])
            rag.ragged_offsets(s["plan"])
            if case["far"]:
                s["past_dev"] = torch.tensor(s["past"], dtype=torch.int32).cuda()
                n = [a + b for a, b in zip(s["L"], s["past"])]
                s["kv_len"] = torch.tensor(n, dtype=torch.int32).cuda()
                s["kv_first"] = torch.tensor([sum(n[:i]) for i in range(len(n))], dtype=torch.int64).cuda()
                s["max_kv"] = max(n)
        if op == "window":
            w = rag.ragged_attention_window_workspace(
                s["plan"], s.get("max_kv", max(s["L"])), window=case["window"], sinks=case["sinks"],
                kv_heads=case["kv_heads"], dtype=s["q"].dtype)
            s["workspace"] = torch.empty(w, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2110_10221_amd as rag
    c = s["case"]
    op = c["op"]
    if op == "rmsnorm":
        x, r = s["x"], s["residual"]
        out = {}
        if r is not None:
            out["sum"] = torch.empty_like(x)
        if c["i8"]:
            q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
            scale = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
            rag.packed_rmsnorm(x, s["gamma"], eps=1e-6, residual=r, x_out=out.get("sum"), q=q, q_scale=scale)
            out["scale"] = scale
            out["values"] = _values(q, scale)
        else:
            out["y"] = torch.empty_like(x)
            rag.packed_rmsnorm(x, s["gamma"], out["y"], eps=1e-6, residual=r, x_out=out.get("sum"))
        return out
    if op == "quantize":
        x = s["x"]
        q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
        scale = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
        rag.packed_quantize_i8(x, q, scale)
        return {"scale": scale, "values": _values(q, scale)}
    if op == "linear":
        y = torch.empty(c["T"], c["N"], dtype=TYPES[c["dtype"]], device="cuda")
        act = (rag.RAG_ACT_NONE, rag.RAG_ACT_GELU_ERF, rag.RAG_ACT_GELU_TANH)[ACTS.index(c["act"])]
        rag.packed_linear_i8(s["x"], s["x_scale"], s["w"], s["w_scale"], y, s["bias"], s["residual"], act)
        return y
    if op == "rotary":
        y = torch.empty_like(s["x"])
        rag.packed_rotary(s["plan"], s["x"], y, s["freq"], heads=c["heads"], head_dim=c["head_dim"],
                          layout=rag.RAG_ROTARY_HALF if c["layout"] == "half" else rag.RAG_ROTARY_INTERLEAVED,
                          amplitude=s["amplitude"], pos_start=s.get("past_dev"), inverse=c["inverse"])
        return y
    out = torch.empty_like(s["q"])
    if c["far"]:
        rag.ragged_attention_window_cached(s["plan"], s["q"], s["k"], s["v"], s["kv_first"], s["kv_len"], s["max_kv"],
                                           out, 0.125, c["window"], c["sinks"], kv_heads=c["kv_heads"],
                                           workspace=s["workspace"])
    else:
        rag.ragged_attention_window(s["plan"], s["q"], s["k"], s["v"], out, 0.125, c["window"], c["sinks"],
                                    kv_heads=c["kv_heads"], workspace=s["workspace"])
    return out


def _values(q, scale):
    return torch.mul(q, scale[:, None], out=torch.empty(q.shape, dtype=torch.bfloat16, device=q.device))


def _plain_i8(y):
    scale = y.abs().amax(dim=1) / 127.0
    q = torch.where(scale[:, None] > 0, torch.round(y / scale[:, None]), 0.0)
    return {"scale": scale, "values": (q * scale[:, None]).to(torch.bfloat16)}


def _run_plain(s):
    c = s["case"]
    op, t = c["op"], TYPES[c["dtype"]]
    if op == "rmsnorm":
        h = s["x"].float()
        out = {}
        if s["residual"] is not None:
            h = h + s["residual"].float()
            out["sum"] = h.to(t)
        y = s["gamma"].float() * (h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + 1e-6))
        out.update(_plain_i8(y) if c["i8"] else {"y": y.to(t)})
        return out
    if op == "quantize":
        return _plain_i8(s["x"].float())
    if op == "linear":
        y = (s["x"].float() @ s["w"].float().t()) * s["x_scale"][:, None] * s["w_scale"] + s["bias"].float()
        if c["act"] == "gelu":
            y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
        elif c["act"] == "gelu_tanh":
            y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(t)
    if op == "rotary":
        angle = s["pos"][:, None] * s["freq"]
        cos = (torch.cos(angle) * s["amplitude"]).float()[:, None]
        sin = (torch.sin(angle) * s["amplitude"]).float()[:, None]
        if c["inverse"]:
            sin = -sin
        x = s["x"].float().view(-1, c["heads"], c["head_dim"])
        R = c["rot_dim"]
        y = x.clone()
        a, b = (slice(0, R // 2), slice(R // 2, R)) if c["layout"] == "half" else (slice(0, R, 2), slice(1, R, 2))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., a] * sin + x[..., b] * cos
        return y.view(s["x"].shape).to(t)
    return _plain_window(s, c, t)


def _plain_window(s, c, t):
    H, G, W, S = c["heads"], c["heads"] // c["kv_heads"], c["window"], c["sinks"]
    out = torch.empty_like(s["q"])
    t0 = r0 = 0
    for L, past in zip(s["L"], s["past"]):
        n = L + past
        for i0 in range(0, L, 512):
            i1 = min(L, i0 + 512)
            # keys that some query of the block sees: the first tokens, then from the first query's window on
            lo, hi = max(0, past + i0 - W + 1), past + i1
            first = min(S, lo)

            def take(x):
                x = torch.cat([x[r0:r0 + first], x[r0 + lo:r0 + hi]]).float().view(-1, H // G, 64)
                return x.transpose(0, 1).repeat_interleave(G, dim=0)

            j = torch.cat([torch.arange(first, device="cuda"), torch.arange(lo, hi, device="cuda")])
            p = torch.arange(past + i0, past + i1, device="cuda")[:, None]
            seen = (j <= p) & ((j > p - W) | (j < S))
            q = s["q"][t0 + i0:t0 + i1].float().view(-1, H, 64).transpose(0, 1)
            score = torch.matmul(q, take(s["k"]).transpose(1, 2).contiguous()) * 0.125
            score = torch.where(seen, score, float("-inf"))
            e = torch.exp(score - score.amax(dim=-1, keepdim=True))
            o = torch.matmul(e, take(s["v"])) / e.sum(dim=-1, keepdim=True)
            out[t0 + i0:t0 + i1] = o.transpose(0, 1).reshape(i1 - i0, -1).to(t)
        t0 += L
        r0 += n
    return out


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it should give
# ---------------------------------------------------------------------------

def work(case):
    op, e = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "rmsnorm":
        n = case["T"] * case["d"]
        b = n * e * (1 + 2 * case["residual"]) + (n + 4 * case["T"] if case["i8"] else n * e) + case["d"] * e
        return {"bytes": b, "flops": 6 * n}
    if op == "quantize":
        n = case["T"] * case["d"]
        return {"bytes": n * (e + 1) + 4 * case["T"], "flops": 4 * n}
    if op == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        return {"bytes": T * K + N * K + 4 * (T + N) + N * e + T * N * e * (1 + case["residual"]), "flops": 2 * T * K * N}
    L, past = _lengths(case)
    if op == "rotary":
        n = sum(L) * case["heads"] * case["head_dim"]
        return {"bytes": 2 * n * e + 4 * case["rot_dim"], "flops": 6 * sum(L) * case["heads"] * (case["rot_dim"] // 2)}
    W, S = case["window"], case["sinks"]
    pairs = keys = 0
    for n, p in zip(L, past):
        for i in range(p, p + n):
            lo = max(0, i - W + 1)
            pairs += i - lo + 1 + min(S, lo)
        lo = max(0, p - W + 1)
        keys += p + n - lo + min(S, lo)
    return {"bytes": 64 * e * (2 * sum(L) * case["heads"] + 2 * keys * case["kv_heads"]),
            "flops": 4 * 64 * case["heads"] * pairs}


def exact(case, seed):
    x = _inputs(case, seed)
    f = {k: v.double() for k, v in x.items() if isinstance(v, torch.Tensor)}
    op = case["op"]

    def eight(y):
        top = torch.maximum(y.amax(1), -y.amin(1))
        steps = torch.round(y * 127.0 / top[:, None].clamp_min(1e-300))
        return {"scale": top / 127.0, "values": steps * (top / 127.0)[:, None]}

    if op == "rmsnorm":
        out, h = {}, f["x"]
        if "residual" in f:
            out["sum"] = h = h + f["residual"]
        y = h / torch.sqrt(torch.sum(h * h, 1, keepdim=True) / case["d"] + 1e-6) * f["gamma"]
        out.update(eight(y) if case["i8"] else {"y": y})
        return out
    if op == "quantize":
        return eight(f["x"])
    if op == "linear":
        y = torch.mm(f["x"], f["w"].t().contiguous())
        y.mul_(f["w_scale"]).mul_(f["x_scale"].unsqueeze(1)).add_(f["bias"])
        if case["act"] == "gelu":
            y = y * torch.special.ndtr(y)
        elif case["act"] == "gelu_tanh":
            y = y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y))
        return y + f["residual"] if "residual" in f else y
    if op == "rotary":
        D, R, s = case["head_dim"], case["rot_dim"], SCALINGS[case["scaling"]]
        factor, amplitude, freq = s.get("factor", 1.0), 1.0, []
        base = BASE
        if case["scaling"] == "ntk" and R > 2:
            base *= factor ** (R / (R - 2))
        for i in range(R // 2):
            w = base ** (-2.0 * i / R)
            if case["scaling"] == "linear":
                w /= factor
            if case["scaling"] == "yarn":
                lo, hi = (R * math.log(s["orig_len"] / (b * 2 * math.pi)) / (2 * math.log(BASE))
                          for b in (s["beta_fast"], s["beta_slow"]))
                lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), R - 1)
                mix = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
                w = (1.0 - mix) * w + mix * w / factor
                amplitude = 0.1 * math.log(factor) + 1.0
            freq.append(w)
        pos = torch.tensor([p + i for n, p in zip(x["L"], x["past"]) for i in range(n)], dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.tensor(amplitude, dtype=torch.float64, device="cuda"),
                           pos[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda"))[:, None]
        if case["inverse"]:
            turn = turn.conj()
        y = f["x"].reshape(-1, case["heads"], D).clone()
        z = y[..., :R]
        z = z.reshape(*z.shape[:2], 2, R // 2).transpose(2, 3) if case["layout"] == "half" else z.reshape(*z.shape[:2], R // 2, 2)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        y[..., :R] = (z.transpose(2, 3) if case["layout"] == "half" else z).reshape(*z.shape[:2], R)
        return y.reshape(f["x"].shape)
    H, G = case["heads"], case["heads"] // case["kv_heads"]
    out = torch.empty_like(f["q"])
    t0 = r0 = 0
    for n, past in zip(x["L"], x["past"]):
        m = n + past
        for h in range(H):
            k, v = (f[a][r0:r0 + m, 64 * (h // G):64 * (h // G) + 64].contiguous() for a in "kv")
            for i0 in range(0, n, 1024):
                i1 = min(n, i0 + 1024)
                p = (past + torch.arange(i0, i1, device="cuda")).unsqueeze(1)
                j = torch.arange(m, device="cuda").unsqueeze(0)
                hidden = (j > p) | ((p - j >= case["window"]) & (j >= case["sinks"]))
                a = torch.mm(f["q"][t0 + i0:t0 + i1, 64 * h:64 * h + 64].contiguous(), k.t().contiguous()) / 8.0
                a = a.masked_fill(hidden, -math.inf)
                a = torch.exp(a - torch.logsumexp(a, 1, keepdim=True))
                out[t0 + i0:t0 + i1, 64 * h:64 * h + 64] = torch.mm(a, v)
        t0 += n
        r0 += m
    return out
