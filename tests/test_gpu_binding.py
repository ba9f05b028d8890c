"""The two ways of making a call of the 4-bit cache and the page bookkeeping, csrc/binding.cpp and step by step in
Python (which a call takes that is not the plain case): the same results, outputs and errors."""
import pytest
import torch

from paper_2504_15930_amd import sl
from fp4_batches import DEV, make

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs an MI355X")]


class _Declines:
    def __getattr__(self, name):
        return lambda *args: None


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _calls(given):
    """Every entry point on fresh copies of the same state, outputs made by the call or given; their results."""
    b, pool = make([40, 17, 64, 0, 33], 8, 2, 64, seed=3)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    k, v = (torch.randn((5, 2, 64), generator=gen, device=DEV).bfloat16() for _ in range(2))
    starts, shared = _i32(0, 2, 5), _i32(0, 0)
    slots = _i32(3, 70, -1, 16 * pool.shape[0], 21)
    empty = lambda *s, dtype=torch.int32: torch.empty(s, dtype=dtype, device=DEV)
    bf = lambda: empty(5, 2, 64, dtype=torch.bfloat16)
    out = torch.empty_like(b.q)
    got = []

    def result(values, outputs):
        if given:
            assert all(x is y for x, y in zip(values, outputs))
        got.extend(values)

    result([sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, **(dict(out=out) if given else {}))], [out])
    out = torch.empty_like(b.q)
    result([sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, starts, shared,
                                      **(dict(out=out) if given else {}))], [out])
    got.append(sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, num_workers=7))
    assert sl.kv_append_fp4(k, v, b.block_table, b.seq_lens, pool) is None
    got.append(pool.clone())
    assert sl.kv_write_fp4(v, k, slots, pool) is None
    got.append(pool.clone())
    outs = (bf(), bf())
    result(sl.kv_read_fp4(slots, pool, **(dict(k_out=outs[0], v_out=outs[1]) if given else {})), outs)
    lens, table = b.seq_lens.clone(), torch.cat([b.block_table, torch.zeros_like(b.block_table)], 1)
    free, count = torch.arange(100, dtype=torch.int32, device=DEV), _i32(90)
    outs = (empty(5), empty(6), empty(80), empty(1))
    kw = dict(seq_lens_out=outs[0], token_start=outs[1], slots=outs[2], free_count_out=outs[3]) if given else {}
    result(sl.pages_extend(lens, _i32(1, 30, 0, 17, 5), table, free, count, 80, **kw), outs)
    got.append(table)
    outs = (empty(5), empty(1))
    kw = dict(seq_lens_out=outs[0], free_count_out=outs[1]) if given else {}
    result(sl.pages_release(_i32(0, 1, 0, 0, 1), lens, table, free, count, **kw), outs)
    got.append(free)
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("given", [False, True])
def test_both_ways_agree(monkeypatch, given):
    print("both ways, outputs given:", given, flush=True)
    here = _calls(given)
    monkeypatch.setattr(sl, "_fast", _Declines())
    for i, (x, y) in enumerate(zip(here, _calls(given), strict=True)):
        assert x.dtype == y.dtype and x.shape == y.shape and x.is_contiguous(), i
        bits = torch.int16 if x.dtype == torch.bfloat16 else x.dtype
        assert torch.equal(x.view(bits), y.view(bits)), i


def test_the_plain_case_is_made_here():
    """The plain call is not declined; one with another kind of argument is."""
    b, pool = make([40, 17], 8, 2, 64, seed=3)
    args = (b.q, pool, b.block_table, b.seq_lens)
    fast = sl._binding()
    assert torch.equal(fast.attn(*args, b.scale, None, None, None, 0), sl.decode_attn_fp4(*args, b.scale))
    wide = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device=DEV)
    for i, x in ((0, b.q.float()), (0, wide), (0, wide[:, :, :64]), (0, b.q[:1]), (0, b.q.cpu()), (0, None), (1, pool[0]),
                 (2, b.block_table.long()), (3, b.seq_lens[:1]), (3, [40, 17])):
        a = list(args)
        a[i] = x
        assert fast.attn(*a, b.scale, None, None, None, 0) is None, (i, x)
    assert fast.attn(*args, 1, None, None, None, 0) is None            # a whole number as the factor
    assert fast.attn(*args, b.scale, None, None, b.q[:1], 0) is None
    assert fast.attn(*args, b.scale, None, None, None, 2 ** 31) is None
    assert fast.attn(*args, b.scale) is None
    # which Python takes, or refuses
    assert torch.equal(sl.decode_attn_fp4(*args, 1), sl.decode_attn_fp4(*args, 1.0))
    q = torch.nn.Parameter(b.q)
    out = sl.decode_attn_fp4(q, *args[1:], b.scale)
    assert torch.equal(out, sl.decode_attn_fp4(*args, b.scale)) and not out.requires_grad


@pytest.mark.parametrize("declines", [False, True])
def test_a_refused_call_raises_its_status(monkeypatch, declines):
    b, pool = make([40, 17], 8, 2, 64, seed=3)
    if declines:
        monkeypatch.setattr(sl, "_fast", _Declines())
    with pytest.raises(sl.SlError) as e:
        sl.decode_attn_fp4(b.q[:, :7].contiguous(), pool, b.block_table, b.seq_lens, b.scale)
    assert e.value.status == -2
    big = torch.zeros(8193, dtype=torch.int32, device=DEV)
    with pytest.raises(sl.SlError) as e:
        sl.pages_release(big, big, torch.zeros((8193, 1), dtype=torch.int32, device=DEV), big, big[:1])
    assert e.value.status == -3
    x = torch.zeros((2, 2, 96), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(sl.SlError) as e:
        sl.kv_write_fp4(x, x, big[:2], torch.zeros((1, 2, 17 * 96), dtype=torch.uint8, device=DEV))
    assert e.value.status == -3


def test_workspace_of_a_stream_grows():
    """A stream's workspace is made by the first call and replaced for a larger one; results stay."""
    small, large = make([300, 40], 8, 2, 64, seed=1), make([700] * 40, 32, 8, 128, seed=2)
    call = lambda c: sl.decode_attn_fp4(c[0].q, c[1], c[0].block_table, c[0].seq_lens, c[0].scale, num_workers=64)
    want = [call(small), call(large)]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = [call(c) for c in (small, large, small, large)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[i % 2]) for i, x in enumerate(got))


def test_outputs_made_in_a_capture_and_in_inference_mode():
    """Calls that make their own outputs, captured and replayed with eager calls between, and in inference mode."""
    b, pool = make([300, 40, 17], 8, 2, 64, seed=5)
    slots, one, count = _i32(3, 40, 5), _i32(1, 1, 1), _i32(30)
    table = torch.cat([b.block_table, torch.zeros_like(b.block_table)], 1)
    free = torch.arange(100, dtype=torch.int32, device=DEV)

    def step():
        lens, start, at, left = sl.pages_extend(b.seq_lens, one, table, free, count, 3)
        return [sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale), *sl.kv_read_fp4(slots, pool), lens,
                start, at, left, *sl.pages_release(_zeros, b.seq_lens, table, free, count)]

    _zeros = torch.zeros_like(one)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        got = step()
    for i in range(4):
        b.q.mul_(0.5)
        g.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want, strict=True)), i
    with torch.inference_mode():
        here = step()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(here, want, strict=True))
    lens = want[3]
    lens.add_(1)                       # an output is an ordinary tensor
    assert lens.tolist() == [302, 42, 19]
