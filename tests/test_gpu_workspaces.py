"""Scratch memory of calls without a ``workspace`` of their own, where it matters: calls of two kernels (split and merge)
that are captured, replayed beside other calls and other graphs, or made on several streams. Every result equals, bit for
bit, the same call alone (the kernels' results depend only on their inputs)."""
import threading

import numpy as np
import pytest
import torch

from paper_2504_15930_amd import inputs, sl
from fp4_batches import DEV, quantised

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs an MI355X")]
KINDS = ["bf16", "e4m3", "fp4", "prefix", "prefix_e4m3", "prefix_fp4"]
WORKERS = 64   # explicit: the 4-bit cache takes split and merge whatever the table's width


class _Declines:
    def __getattr__(self, name):
        return lambda *args: None


@pytest.fixture(params=["binding", "python"])
def way(request, monkeypatch):
    """Both ways of making a 4-bit call."""
    if request.param == "python":
        monkeypatch.setattr(sl, "_fast", _Declines())
    return request.param


def _call(kind, B, seed, most=700):
    """(queries, function of an output) of a decode call of this kind on its own batch."""
    rng = np.random.default_rng(seed)
    cache = kind.removeprefix("prefix_") if kind != "prefix" else "bf16"
    if kind.startswith("prefix"):
        b, starts, shared = inputs.make_grpo_batch(B // 4, 4, 100, seed=seed, device=DEV, num_q_heads=8, num_kv_heads=2,
                                                   head_dim=128, gen_median=most / 4, gen_cap=most,
                                                   kv_dtype="e4m3" if cache == "e4m3" else "bf16")
    else:
        b = inputs.make_paged_batch(rng.integers(1, most, B), 8, 2, 128, seed=seed, device=DEV,
                                    kv_dtype="e4m3" if cache == "e4m3" else "bf16")
    tail = (b.block_table, b.seq_lens, b.scale) + ((starts, shared) if kind.startswith("prefix") else ())
    if cache == "fp4":
        pages, suffix = (quantised(b),), "_fp4"
    elif cache == "e4m3":
        pages, suffix = (b.k_pages, b.v_pages, b.k_scales, b.v_scales), "_fp8"
    else:
        pages, suffix = (b.k_pages, b.v_pages), ""
    f = getattr(sl, ("decode_attn_prefix" if kind.startswith("prefix") else "decode_attn") + suffix)
    return b.q, lambda out=None: f(b.q, *pages, *tail, out=out, num_workers=WORKERS)


def _same(x, y):
    return torch.equal(x.view(torch.int16), y.view(torch.int16))


def _fresh(n=24):
    """Tensors of the sizes that a dropped buffer's memory would be handed out for, all ones."""
    return [torch.ones(1 << s, dtype=torch.uint8, device=DEV) for s in range(10, 24) for _ in range(n // 8)]


@pytest.mark.parametrize("kind", KINDS)
def test_a_captured_call_outlives_larger_calls_on_its_stream(kind, way):
    print("captured, then larger calls", kind, way, flush=True)
    q, call = _call(kind, 12, 1)
    _, larger = _call(kind, 96, 2)
    out = torch.empty_like(q)
    want = call().clone()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call(out)
    stream.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        call(out)
    big = larger().clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        got = [larger() for _ in range(3)]
        fresh = _fresh()
    stream.synchronize()
    for i in range(4):
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert _same(out, want), i
        assert all((t == 1).all() for t in fresh), i
        with torch.cuda.stream(stream):
            got.append(larger())
        torch.cuda.synchronize()
    assert all(_same(x, big) for x in got)


@pytest.mark.parametrize("kind", ["bf16", "fp4", "prefix_fp4"])
def test_graphs_of_growing_batches_and_one_that_is_reset(kind, way):
    """Ascending batch sizes, captured on one stream; the first graph is reset before the others are replayed."""
    print("growing batches", kind, way, flush=True)
    calls = [_call(kind, B, B) for B in (4, 16, 40, 96)]
    want = [call().clone() for _, call in calls]
    outs = [torch.empty_like(q) for q, _ in calls]
    torch.cuda.synchronize()
    graphs = []
    for (_, call), out in zip(calls, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(out)
    graphs[0].reset()
    torch.cuda.empty_cache()
    fresh = _fresh()
    for i in range(3):
        for out, g in list(zip(outs, graphs))[1:]:
            out.zero_()
            g.replay()
        torch.cuda.synchronize()
        assert all(_same(x, y) for x, y in zip(outs[1:], want[1:])), i
        assert all((t == 1).all() for t in fresh), i


@pytest.mark.parametrize("kind", ["bf16", "fp4", "prefix_fp4"])
def test_two_graphs_at_once(kind, way):
    """Captured one after the other on the same stream, replayed beside each other and beside eager calls."""
    print("two graphs", kind, way, flush=True)
    calls = [_call(kind, 64, s, most=1500) for s in (1, 2, 3)]
    want = [call().clone() for _, call in calls]
    outs = [torch.empty_like(q) for q, _ in calls[:2]]
    graphs = []
    for (_, call), out in zip(calls[:2], outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(out)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(4):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for _ in range(5):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
            got = calls[2][1]()
        torch.cuda.synchronize()
        assert _same(outs[0], want[0]) and _same(outs[1], want[1]) and _same(got, want[2]), i


@pytest.mark.parametrize("kind", KINDS)
def test_two_streams_at_once(kind, way):
    print("two streams", kind, way, flush=True)
    calls = [_call(kind, 64, s, most=1500) for s in (1, 2)]
    want = [call().clone() for _, call in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = []
    for _ in range(10):
        for (_, call), s in zip(calls, streams):
            with torch.cuda.stream(s):
                got.append(call())
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert _same(out, want[i % 2]), i


@pytest.mark.parametrize("kind", KINDS)
def test_two_threads_on_one_stream(kind, way):
    """Their calls' kernels may alternate on the stream."""
    print("two threads", kind, way, flush=True)
    calls = [_call(kind, 64, s, most=1500) for s in (1, 2)]
    want = [call().clone() for _, call in calls]
    outs = [[torch.empty_like(q) for _ in range(40)] for q, _ in calls]
    torch.cuda.synchronize()
    stream, start, errors = torch.cuda.Stream(), threading.Barrier(2), []

    def work(i):
        try:
            with torch.cuda.stream(stream):
                start.wait()
                for out in outs[i]:
                    calls[i][1](out)
        except Exception as e:   # handed to the main thread
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(timeout=60)
    assert not any(t.is_alive() for t in threads) and not errors, errors
    torch.cuda.synchronize()
    for i in range(2):
        assert all(_same(x, want[i]) for x in outs[i]), i


@pytest.mark.parametrize("workers", [0, WORKERS])
def test_a_captured_decode_step_with_pages_rows_and_both_attentions(workers, way):
    """Pages, the new rows, attention and, over the same pages, prefix sharing in two groups: captured once and replayed
    across a page boundary, beside the eager step on a copy of the state. Outputs made by the captured calls."""
    print("captured step", workers, way, flush=True)
    B, hq, hkv, d = 8, 8, 2, 128
    rng = np.random.default_rng(3)
    b, starts, shared = inputs.make_grpo_batch(2, 4, 64, seed=4, device=DEV, num_q_heads=hq, num_kv_heads=hkv, head_dim=d,
                                               gen_median=30, gen_cap=200)
    pool = quantised(b)
    N, extra = pool.shape[0], 40
    pool = torch.cat([pool, torch.full((extra, *pool.shape[1:]), 0xFF, dtype=torch.uint8, device=DEV)])
    free = torch.zeros(N + extra, dtype=torch.int32, device=DEV)
    free[:extra] = torch.from_numpy(rng.permutation(extra).astype(np.int32)).to(DEV) + N
    one = torch.ones(B, dtype=torch.int32, device=DEV)
    s = dict(lens=b.seq_lens.clone(), table=torch.cat([b.block_table, torch.zeros_like(b.block_table)], 1), free=free,
             count=torch.full((1,), extra, dtype=torch.int32, device=DEV), pool=pool)
    gen = torch.Generator(device=DEV).manual_seed(5)
    rows = lambda: torch.randn((B, hkv, d), generator=gen, device=DEV).bfloat16()
    k, v = rows(), rows()

    def step(x):
        sl.pages_extend(x["lens"], one, x["table"], x["free"], x["count"], B, seq_lens_out=x["lens"], free_count_out=x["count"])
        sl.kv_append_fp4(k, v, x["table"], x["lens"], x["pool"])
        return [sl.decode_attn_fp4(b.q, x["pool"], x["table"], x["lens"], b.scale, num_workers=workers),
                sl.decode_attn_prefix_fp4(b.q, x["pool"], x["table"], x["lens"], b.scale, starts, shared, num_workers=workers)]

    step({n: t.clone() for n, t in s.items()})
    torch.cuda.synchronize()
    eager = {n: t.clone() for n, t in s.items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step(s)
    for i in range(20):
        k.copy_(rows())
        v.copy_(rows())
        g.replay()
        torch.cuda.synchronize()
        want = step(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(s[n], eager[n]) for n in s), i
        assert all(_same(x, y) for x, y in zip(outs, want)), i


@pytest.mark.parametrize("own_stream", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "fp4", "prefix_fp4"])
def test_eager_calls_of_another_thread_during_a_capture(kind, own_stream, way):
    """Their stream is not being captured: they keep their own buffer, and the graph its."""
    print("another thread during a capture", kind, own_stream, way, flush=True)
    calls = [_call(kind, 64, s, most=900) for s in (1, 2)]
    want = [call().clone() for _, call in calls]
    outs = [torch.empty_like(q) for q, _ in calls]
    # (torch's streams come round: two made one after the other are different ones)
    captured, other = torch.cuda.Stream(), torch.cuda.Stream()
    stream = other if own_stream else torch.cuda.default_stream()
    errors, warm, go = [], threading.Event(), threading.Event()

    def work():
        try:
            with torch.cuda.stream(stream):
                calls[1][1](outs[1])      # makes the thread's buffer, before the capture
                stream.synchronize()
                outs[1].zero_()
                warm.set()
                assert go.wait(30)
                for _ in range(3):
                    calls[1][1](outs[1])
        except Exception as e:            # handed to the main thread
            errors.append(e)
            warm.set()

    t = threading.Thread(target=work)
    t.start()
    assert warm.wait(30)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=captured, capture_error_mode="thread_local"):
        calls[0][1](outs[0])
        go.set()
        t.join(30)
    assert not t.is_alive() and not errors, errors
    torch.cuda.synchronize()
    assert _same(outs[1], want[1])
    outs[0].zero_()
    g.replay()
    torch.cuda.synchronize()
    assert _same(outs[0], want[0])
