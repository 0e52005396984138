"""_binding.so, the compiled part of the operators' Python calls: documented calls go through it,
every other one is left, without a launch, to the checks written in Python."""
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2110_10221_amd", "_binding.so")),
                                reason="_binding.so not built")
COUNTS = {"packed_rmsnorm": 9, "packed_quantize_i8": 4, "packed_linear_i8": 9, "packed_rotary": 11, "ragged_attention_window": 12,
          "ragged_attention_window_cached": 15}


def fast():
    import paper_2110_10221_amd as rag

    return rag._fast


@pytest.mark.parametrize("name,n", COUNTS.items())
def test_arguments_of_any_kind_are_left_to_python(name, n):
    f = getattr(fast(), name)
    x = torch.zeros(2, 64)
    for a in (None, 0, "x", object(), 2 ** 80, x, torch.nn.Parameter(x), x.to_sparse(), torch.zeros(2, 64, device="meta")):
        assert f(*[a] * n) is None
    with pytest.raises(TypeError):
        f(*[None] * (n - 1))


def test_sizes_past_32_bits_are_refused():
    import paper_2110_10221_amd as rag

    n = 2 ** 32 + 5
    x, q, v = torch.zeros(1, 64).expand(n, 64), torch.zeros(1, 64, dtype=torch.int8).expand(n, 64), torch.zeros(1).expand(n)
    with pytest.raises(ValueError, match="2.31"):
        rag.packed_rmsnorm(x, torch.zeros(64), x)
    with pytest.raises(ValueError, match="2.31"):
        rag.packed_quantize_i8(x, q, v)
    with pytest.raises(ValueError, match="2.31"):
        rag.packed_linear_i8(q, v, q[:8], v[:8], x)
    with pytest.raises(ValueError, match="2.31"):
        rag.packed_linear_i8(q[:8], v[:8], q, v, x[:8])


def calls(T=6, d=64):
    """{name: (arguments, {position: values that are not as documented})}, on the GPU."""
    import paper_2110_10221_amd as rag

    bf, dev = torch.bfloat16, "cuda"
    m = lambda r=T, c=d, t=bf: torch.ones(r, c, dtype=t, device=dev)  # noqa: E731
    v = lambda n, t=torch.float32: torch.ones(n, dtype=t, device=dev)  # noqa: E731
    plan = rag.Plan(torch.tensor([2, 4], dtype=torch.int32).cuda(), T, 4, 1)
    rag.ragged_offsets(plan)
    first, length = torch.tensor([0, 2]).cuda(), torch.tensor([2, 4], dtype=torch.int32).cuda()
    bad = (m(T + 1), m(T, d + 8), m(t=torch.float32), m(T, 2 * d)[:, ::2], m().cpu(), v(T), m().t(), 3)
    badv = (v(T + 1), v(2 * T)[::2], v(T, torch.int32), v(T).cpu(), m())
    ints = (2.0, "1", -2 ** 40, None)
    return {
        "packed_rmsnorm": ([m(), v(d, bf), m(), 1e-6, m(), m(), m(t=torch.int8), v(T), None],
                           {0: (v(T), m().cpu(), m(t=torch.float16)), 1: (v(d), v(d + 8, bf)), 2: bad, 3: ("x", None), 4: bad, 5: bad,
                            6: bad, 7: badv, 8: (3,)}),
        "packed_quantize_i8": ([m(), m(t=torch.int8), v(T), None], {0: (v(T), m().cpu()), 1: bad, 2: badv, 3: ("s",)}),
        "packed_linear_i8": ([m(t=torch.int8), v(T), m(16, d, torch.int8), v(16), m(T, 16), v(16, bf), m(T, 16), 0, None],
                             {0: (m(), m(T + 1, d, torch.int8)), 1: badv, 2: (m(16, d), m(16, 2 * d, torch.int8)[:, :d]), 3: badv,
                              4: (m(T, 8), m(T, 16, torch.float16)), 5: (v(16),), 6: bad, 7: ints}),
        "packed_rotary": ([plan, m(), m(), v(32, torch.float64), 1, 64, 0, 1.0, None, False, None],
                          {0: (None, 3), 1: bad, 2: bad + (None,), 3: (v(32), m(4, 8, torch.float64)), 4: ints + (2,), 5: ints, 6: ints,
                           7: ("x",), 8: (first, v(3, torch.int32)), 9: (1,)}),
        "ragged_attention_window": ([plan, m(), m(), m(), m(), 0.1, 3, 0, None, 64, None, None],
                                    {0: (None,), 1: bad, 2: bad + (None,), 3: bad + (None,), 4: bad + (None,), 5: ("x",), 6: ints, 7: ints,
                                     8: (2, -1, 1.0), 9: ints, 10: (m()[:, ::2], m().cpu(), 5)}),
        "ragged_attention_window_cached": ([plan, m(), m(), m(), first, length, 4, m(), 0.1, 3, 0, 1, 64, None, None],
                                           {1: bad, 2: (v(T), m().cpu()), 3: bad, 4: (length, v(2, torch.int64).cpu()), 5: (first,), 6: ints,
                                            7: bad, 8: ("x",), 9: ints, 10: ints, 11: (2, -1), 12: ints, 13: (m()[:, ::2],)}),
    }


@pytest.mark.gpu
@pytest.mark.parametrize("name", COUNTS)
def test_what_is_not_as_documented_is_left_to_python(name):
    args, wrong = calls()[name]
    f = getattr(fast(), name)
    for i, values in wrong.items():
        for value in values:
            assert f(*args[:i], value, *args[i + 1:]) is None, (i, value)
    assert f(*args) == 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert f(*args[:-1], side) == 0
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_both_ways_give_the_same(monkeypatch):
    import paper_2110_10221_amd as rag

    results = []
    for way in range(2):
        if way:
            monkeypatch.setattr(rag, "_fast", type("Off", (), {n: staticmethod(lambda *a: None) for n in COUNTS}))
        torch.manual_seed(3)
        args = {n: [a.normal_() if isinstance(a, torch.Tensor) and a.dtype == torch.bfloat16 else a for a in c[0]] for n, c in calls().items()}
        a = args["packed_rmsnorm"]
        rag.packed_rmsnorm(a[0], a[1], a[2], 1e-5, a[4], a[5], a[6], a[7])
        b = args["packed_linear_i8"]
        rag.packed_linear_i8(a[6], a[7], b[2], b[3], b[4], b[5], b[6], 2)
        q = args["packed_quantize_i8"]
        rag.packed_quantize_i8(*q[:3])
        r = args["packed_rotary"]
        rag.packed_rotary(*r[:4], 1, 64, rag.RAG_ROTARY_INTERLEAVED, 1.5, None, True)
        w = args["ragged_attention_window"]
        rag.ragged_attention_window(*w[:5], 0.3, 2, 1)
        c = args["ragged_attention_window_cached"]
        rag.ragged_attention_window_cached(*c[:8], 0.3, 2 ** 40, 1)
        torch.cuda.synchronize()
        results.append([t.cpu() for t in (*a[2:3], *a[5:8], b[4], *q[1:3], r[2], w[4], c[7])])
    assert all(torch.equal(x, y) for x, y in zip(*results))


@pytest.mark.gpu
def test_refusals_of_the_library_reach_the_caller():
    import paper_2110_10221_amd as rag

    args, _ = calls()["packed_rmsnorm"]
    with pytest.raises(rag.RaggedError):
        rag.packed_rmsnorm(args[0], args[1], args[2], -1.0)
    with pytest.raises(ValueError):
        rag.packed_rmsnorm(args[0], args[1], args[2][:, :32])
    with pytest.raises(ValueError):
        rag.packed_rmsnorm(args[0].cpu(), args[1].cpu(), args[2].cpu())


@pytest.mark.parametrize("n", [64 - 2 ** 32, -2 ** 40, -2 ** 31 - 1])
def test_integers_below_32_bits_are_refused(n):
    # (ctypes would wrap them: 64 - 2^32 to a window of 64); CPU tensors, so that nothing could launch
    import types

    import paper_2110_10221_amd as rag

    x, q, v = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4)
    plan = types.SimpleNamespace(total_tokens=4, heads=1, batch=1, max_len=4, ref=lambda: None, status=torch.zeros(4))
    first, length = torch.zeros(1, dtype=torch.int64), torch.ones(1, dtype=torch.int32)
    window = dict(window=3, sinks=1)
    for name in window:
        with pytest.raises(ValueError, match="32 bits"):
            rag.ragged_attention_window(plan, x, x, x, x, 0.1, **{**window, name: n})
        with pytest.raises(ValueError, match="32 bits"):
            rag.ragged_attention_window_cached(plan, x, x, x, first, length, 4, x, 0.1, **{**window, name: n})
        with pytest.raises(ValueError, match="32 bits"):
            rag.ragged_attention_window_workspace(plan, 4, **{**window, name: n})
    with pytest.raises(ValueError, match="32 bits"):
        rag.ragged_attention_window_cached(plan, x, x, x, first, length, n, x, 0.1, 3)
    with pytest.raises(ValueError, match="32 bits"):
        rag.ragged_attention_window_workspace(plan, n, 3)
    with pytest.raises(ValueError, match="32 bits"):
        rag.packed_rotary(plan, x, x, torch.zeros(4, dtype=torch.float64), 1, 64, layout=n)
    with pytest.raises(ValueError, match="32 bits"):
        rag.packed_linear_i8(q, v, q[:4], v[:4], torch.zeros(4, 4), act=n)
    for name in ("rot_dim", "scaling", "orig_len"):
        with pytest.raises(ValueError, match="32 bits"):
            rag.rotary_frequencies(**{"rot_dim": 64, name: n})


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32, 2 ** 32 + 1])
def test_integers_above_32_bits_are_refused_where_nothing_is_open(n):
    import types

    import paper_2110_10221_amd as rag

    x, q, v = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4)
    plan = types.SimpleNamespace(total_tokens=4, heads=1, batch=1, max_len=4, ref=lambda: None, status=torch.zeros(4))
    with pytest.raises(ValueError, match="32 bits"):
        rag.packed_linear_i8(q, v, q[:4], v[:4], torch.zeros(4, 4), act=n)
    with pytest.raises(ValueError, match="32 bits"):
        rag.packed_rotary(plan, x, x, torch.zeros(4, dtype=torch.float64), 1, 64, layout=n)
    for name in ("rot_dim", "scaling", "orig_len"):
        with pytest.raises(ValueError, match="32 bits"):
            rag.rotary_frequencies(**{"rot_dim": 64, name: n})


@pytest.mark.gpu
def test_open_windows_may_be_any_number_above():
    import paper_2110_10221_amd as rag

    args, _ = calls()["ragged_attention_window"]
    outs = []
    for window in (2 ** 31 - 1, 2 ** 40, float("inf")):
        rag.ragged_attention_window(*args[:5], 0.3, window, 2 ** 40)
        outs.append(args[4].clone())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("what", ["absent", "not a library", "of another torch"])
def test_the_package_needs_no_compiled_part(what, tmp_path):
    import subprocess
    import sys

    package = tmp_path / "paper_2110_10221_amd"
    package.mkdir()
    for name in ("__init__.py", "_build.py", "libragged.so"):
        os.symlink(os.path.join(ROOT, "paper_2110_10221_amd", name), package / name)
    if what == "not a library":
        (package / "_binding.so").write_bytes(b"\0" * 100)
    elif what == "of another torch":
        (package / "_binding.py").write_text("built_for = 'torch 1.0'\ndef bind(*a):\n    raise SystemError\n")
    code = ("import torch, paper_2110_10221_amd as rag\n"
            f"assert rag.__file__.startswith({str(tmp_path)!r})\n"
            "assert rag._fast.packed_rmsnorm(1, 2) is None and rag.rotary_frequencies(64)[0].numel() == 32\n"
            "x = torch.zeros(4, 64)\n"
            "try:\n    rag.packed_rmsnorm(x, x[0], x[:, :8])\n"
            "except ValueError as e:\n    assert 'y must be' in str(e)\n"
            "else:\n    raise SystemError('not refused')\n")
    subprocess.run([sys.executable, "-c", code], cwd=tmp_path, check=True, timeout=100, env={**os.environ, "PYTHONPATH": str(tmp_path)})


def test_the_compiled_part_is_used_where_it_fits():
    import paper_2110_10221_amd as rag

    assert rag._fast.__name__.endswith("_binding") and rag._fast.built_for == rag.built_for()
