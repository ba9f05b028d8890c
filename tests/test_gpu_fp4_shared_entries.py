"""Prefix sharing over a 4-bit cache reads the shared pages through the first member's entries of the block table, in every
kernel: the other members' entries for them may hold anything."""
import numpy as np
import pytest
import torch

from paper_2504_15930_amd import inputs, sl
from fp4_batches import DEV, quantised, reference
from parity import assert_parity

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs an MI355X")]


def _blanked(b, ranges, shared, kept, other):
    """The table with `other` in the shared entries of every member of the ranges but each `kept`-th."""
    table = b.block_table.clone()
    for (lo, hi), n in zip(ranges, shared):
        for i in range(lo, hi):
            if (i - lo) % kept:
                table[i, :n] = other
    return table


# prompts, samples, prompt, heads, KV heads, D: one group, several, more than a wavefront's 64, more than 256 (the stream)
CASES = [(1, 4, 40, 8, 2, 64), (3, 5, 100, 28, 4, 128), (5, 8, 70, 12, 12, 64), (70, 2, 33, 8, 2, 128), (200, 3, 20, 4, 2, 64),
         (256, 2, 40, 4, 1, 64), (300, 2, 40, 8, 2, 128), (4, 4, 300, 16, 1, 128), (2, 3, 2100, 28, 4, 128)]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("workers", [0, 40])
def test_only_the_first_members_entries_are_read(case, workers):
    prompts, samples, prompt, hq, hkv, d = case
    print("shared entries", case, workers, flush=True)
    b, starts, shared = inputs.make_grpo_batch(prompts, samples, prompt, seed=prompt, device=DEV, num_q_heads=hq,
                                               num_kv_heads=hkv, head_dim=d, gen_median=20, gen_cap=60)
    pool = quantised(b)
    kept = min(16, 64 * hkv // hq)          # the members of a sub-group; each sub-group's first keeps its entries
    assert samples <= kept
    ranges = [(i * samples, (i + 1) * samples) for i in range(prompts)]
    want = sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, starts, shared, num_workers=workers)
    for other in (-1, pool.shape[0], int(b.block_table[-1, prompt // 16])):
        table = _blanked(b, ranges, shared.tolist(), kept, other)
        out = sl.decode_attn_prefix_fp4(b.q, pool, table, b.seq_lens, b.scale, starts, shared, num_workers=workers)
        torch.cuda.synchronize()
        assert torch.equal(out, want), other
    rows = list(range(min(prompts * samples, 8)))
    assert_parity(want[rows], reference(b, pool, rows), str(case))


@pytest.mark.parametrize("workers", [0, 9])
def test_ranges_that_are_not_shared_read_their_own(workers):
    """A range that starts before an earlier one's end, that leaves the batch, or that shares no pages or too many, is
    attended by its members' own entries; a shared one's members by the first one's."""
    b, starts, shared = inputs.make_grpo_batch(4, 6, 100, seed=3, device=DEV, num_q_heads=8, num_kv_heads=2, head_dim=64,
                                               gen_median=40, gen_cap=90)
    pool = quantised(b)
    ref = reference(b, pool)
    t = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    n = 6   # shared pages of every prompt
    assert shared.tolist() == [n] * 4
    # (descending starts: 6..12 is shared, 12..0 is empty, 0..6 and 6..24 start before 12)
    for gs, sp, ranges in ((t(6, 12, 0, 6, 24), shared, [(6, 12)]), (t(0, 6, 12, 30, 24), shared, [(0, 6), (6, 12)]),
                           (t(-6, 0, 6, 12, 18), shared, [(0, 6), (6, 12), (12, 18)]),
                           (starts, t(n, 0, n, b.block_table.shape[1] + 1), [(0, 6), (12, 18)]),
                           (starts, t(n, -1, 3, n), [(0, 6), (18, 24)])):
        table = _blanked(b, ranges, [n] * len(ranges), 6, -1)
        out = sl.decode_attn_prefix_fp4(b.q, pool, table, b.seq_lens, b.scale, gs, sp, num_workers=workers)
        torch.cuda.synchronize()
        assert_parity(out, ref, f"{gs.tolist()} {sp.tolist()}")
    # a member shorter than its shared pages, the first one among them
    lens = b.seq_lens.clone()
    lens[[0, 8]] = 95
    table = _blanked(b, [(i, i + 6) for i in range(0, 24, 6)], [n] * 4, 6, -1)
    out = sl.decode_attn_prefix_fp4(b.q, pool, table, lens, b.scale, starts, shared, num_workers=workers)
    torch.cuda.synchronize()
    keep = [i for i in range(24) if i not in (0, 8)]
    assert torch.isnan(out[[0, 8]]).all()
    assert_parity(out[keep], ref[keep], "the others")
