"""Calls under a torch dispatch mode: the mode sees the outputs that a call makes, as it does for every other call, and the
results are the same."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2504_15930_amd import sl
from fp4_batches import DEV, make

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs an MI355X")]


class _Seen(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.made = 0

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        self.made += "empty" in str(func)
        return out


def test_a_dispatch_mode_sees_the_outputs():
    b, pool = make([40, 17, 64, 33], 8, 2, 64, seed=3)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    starts, shared, slots, zero = i32(0, 2, 4), i32(0, 0), i32(3, 70, -1, 21), i32(0, 0, 0, 0)
    table = torch.cat([b.block_table, torch.zeros_like(b.block_table)], 1)
    free, count, one = torch.arange(100, dtype=torch.int32, device=DEV), i32(30), i32(1, 1, 1, 1)
    calls = [lambda: [sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale)],
             lambda: [sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, starts, shared)],
             lambda: sl.kv_read_fp4(slots, pool),
             lambda: sl.pages_extend(b.seq_lens, one, table.clone(), free, count, 4),
             lambda: sl.pages_release(zero, b.seq_lens, table, free.clone(), count)]
    for i, call in enumerate(calls):
        want = call()
        with _Seen() as seen:
            got = call()
        torch.cuda.synchronize()
        assert seen.made >= 1, i
        bits = lambda t: t.view(torch.int16) if t.dtype == torch.bfloat16 else t   # (slots without a token read as NaN)
        assert all(torch.equal(bits(x), bits(y)) for x, y in zip(got, want, strict=True)), i
