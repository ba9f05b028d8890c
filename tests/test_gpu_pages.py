"""Page bookkeeping on the GPU (sl_pages_extend, sl_pages_release) against oracle/fp4.py, number for number."""
import numpy as np
import pytest
import torch

from oracle import fp4
from paper_2504_15930_amd import sl

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs an MI355X")]
DEV = "cuda:0"


def _t(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32, device=DEV)


def _case(rng, B, blocks, spare):
    """Lengths with the edge values, a table of distinct pages, and a stack of `spare` others."""
    lens = np.where(rng.random(B) < 0.3, rng.choice([0, 1, 15, 16, 17, blocks * 16], B), rng.integers(0, blocks * 16 + 1, B))
    lens = np.minimum(lens, blocks * 16).astype(np.int32)
    held = -(-lens // 16)
    N = int(held.sum()) + spare
    perm = rng.permutation(N).astype(np.int32)
    table = np.full((B, blocks), -9, np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    free = np.full(N, -3, np.int32)
    free[:spare] = perm[at:]
    return lens, table, free


def _check_extend(lens, new, table, free, count, cap, in_place=False):
    want = fp4.pages_extend(lens, new, table, free, count, cap)
    tl, tt, tf, tc = _t(lens), _t(table), _t(free), _t([count])
    kw = dict(seq_lens_out=tl, free_count_out=tc) if in_place else {}
    got_lens, start, slots, left = sl.pages_extend(tl, _t(new), tt, tf, tc, cap, **kw)
    torch.cuda.synchronize()
    assert got_lens.tolist() == list(want[0])
    assert start.tolist() == list(want[1])
    assert slots.tolist() == list(want[2])
    assert left.item() == want[3]
    assert np.array_equal(tt.cpu().numpy(), want[4])
    assert np.array_equal(tf.cpu().numpy(), free)
    if in_place:
        assert got_lens is tl and left is tc
    else:
        assert tl.tolist() == list(lens) and tc.item() == count


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,blocks", [(1, 1), (2, 3), (63, 5), (64, 9), (256, 40), (1025, 3), (4097, 2), (8192, 2)])
def test_extend(B, blocks, in_place):
    print("extend", B, blocks, flush=True)
    rng = np.random.default_rng(B * 7 + blocks)
    lens, table, free = _case(rng, B, blocks, B * blocks)
    room = blocks * 16 - lens
    one = np.minimum(room, 1)
    ragged = (rng.random(B) * (room + 1)).astype(np.int32)
    for new in (np.zeros(B, np.int32), one, ragged):
        _check_extend(lens, new, table, free, B * blocks, int(new.sum()) + 3, in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_extend_many_tokens(in_place):
    """Slot maps of more tokens than one workgroup fills."""
    rng = np.random.default_rng(1)
    for B, blocks in ((1, 2000), (5, 1200), (300, 60)):
        print("many tokens", B, blocks, flush=True)
        lens, table, free = _case(rng, B, blocks, B * blocks)
        new = (rng.random(B) * (blocks * 16 - lens + 1)).astype(np.int32)
        new[0] = blocks * 16 - lens[0]
        cap = int(new.sum())
        for c in (cap, cap + 1, max(cap - 1, 0), cap + 5000):
            _check_extend(lens, new, table, free, B * blocks, c, in_place)


def test_extend_one_output_in_place():
    """The lengths or the count alone updated in place, with a slot map of more tokens than one workgroup fills."""
    lens, table, free = _case(np.random.default_rng(8), 40, 60, 2400)
    new = 60 * 16 - lens
    cap = int(new.sum())
    want = fp4.pages_extend(lens, new, table, free, 2400, cap)
    for name in ("seq_lens_out", "free_count_out"):
        tl, tt, tf, tc = _t(lens), _t(table), _t(free), _t([2400])
        got = sl.pages_extend(tl, _t(new), tt, tf, tc, cap, **{name: tl if name == "seq_lens_out" else tc})
        torch.cuda.synchronize()
        assert [x.tolist() for x in got[:3]] == [list(x) for x in want[:3]] and got[3].item() == want[3], name
        assert np.array_equal(tt.cpu().numpy(), want[4])


def test_extend_largest_slot_map():
    """2^31 - 1 entries, the most that the argument holds, of which three are tokens."""
    tl, tt, tf, tc = _t([14]), _t([[5, -9]]), _t([0, 1, 2, 4, 3, -3]), _t([5])
    cap = 2**31 - 1
    slots = torch.full((cap,), 7, dtype=torch.int32, device=DEV)
    sl.pages_extend(tl, _t([3]), tt, tf, tc, cap, slots=slots)
    torch.cuda.synchronize()
    assert slots[:3].tolist() == [5 * 16 + 14, 5 * 16 + 15, 3 * 16]
    assert (slots[3:] == -1).all() and tt.tolist() == [[5, 3]]


@pytest.mark.parametrize("cap", [-1, 2**31, 2**32 + 8])
def test_extend_slot_map_size_refusals(cap):
    tl, tt, tf, tc = _t([14]), _t([[5, -9]]), _t([0, 1, 2, 4, 3, -3]), _t([5])
    for kw in ({}, dict(slots=_t(np.zeros(8)))):
        with pytest.raises(ValueError):
            sl.pages_extend(tl, _t([3]), tt, tf, tc, cap, **kw)


def test_extend_without_room():
    """A short stack and a short slot map: requests are served in order while there is room, those that need none too."""
    rng = np.random.default_rng(2)
    for i in range(30):
        B, blocks = int(rng.integers(1, 80)), int(rng.integers(1, 8))
        lens, table, free = _case(rng, B, blocks, B * blocks)
        new = rng.integers(0, 40, B).astype(np.int32)
        need = int((-(-(lens + new) // 16) - -(-lens // 16)).sum())
        count, cap = int(rng.integers(0, need + 2)), int(rng.integers(0, new.sum() + 2))
        _check_extend(lens, new, table, free, min(count, B * blocks), cap, in_place=bool(i % 2))
    _check_extend(np.array([16]), np.array([1]), np.array([[0, 0]], np.int32), np.array([5], np.int32), 0, 1)


def test_extend_invalid_data():
    """Negative or too long lengths and counts, a count outside the stack, page ids outside the pool."""
    rng = np.random.default_rng(3)
    lens, table, free = _case(rng, 12, 4, 48)
    new = np.ones(12, np.int32)
    lens[[1, 2, 3]] = [-1, 65, 2 ** 31 - 1]
    new[[4, 5, 6]] = [-1, 100, 2 ** 31 - 1]
    lens[7], lens[8] = 20, 3
    table[7, 1], table[8, 0] = len(free), -1
    lens[9], free[47] = 16, -5
    for count in (48, -4, 10 ** 9):
        _check_extend(lens, new, table, free, count, 64)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,blocks", [(1, 1), (7, 3), (64, 9), (256, 40), (1025, 3), (8192, 2), (96, 300), (2000, 40)])
def test_release(B, blocks, in_place):
    print("release", B, blocks, flush=True)
    rng = np.random.default_rng(B + blocks)
    lens, table, free = _case(rng, B, blocks, 5)
    if B > 5:
        lens[[1, 3]] = [-2, blocks * 16 + 1]
    for done in (np.zeros(B, np.int32), np.ones(B, np.int32), rng.integers(-1, 2, B).astype(np.int32)):
        for count in (5, -1):
            want = fp4.pages_release(done, lens, table, free, count)
            tl, tt, tf, tc = _t(lens), _t(table), _t(free), _t([count])
            kw = dict(seq_lens_out=tl, free_count_out=tc) if in_place else {}
            got, left = sl.pages_release(_t(done), tl, tt, tf, tc, **kw)
            torch.cuda.synchronize()
            assert got.tolist() == list(want[0]) and left.item() == want[1]
            assert np.array_equal(tf.cpu().numpy(), want[2])
            assert np.array_equal(tt.cpu().numpy(), table)


def test_release_twice_does_not_overrun_the_stack():
    lens, table, free = _case(np.random.default_rng(4), 6, 5, 3)
    tl, tt, tf, tc = _t(lens), _t(table), _t(free), _t([3])
    done = _t(np.ones(6))
    _, left = sl.pages_release(done, tl, tt, tf, tc)
    _, again = sl.pages_release(done, tl, tt, tf, left)      # the old lengths once more
    torch.cuda.synchronize()
    assert left.item() == len(free) and again.item() == len(free)
    assert sorted(tf.tolist()) == list(range(len(free)))


def test_empty_batch():
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    lens, start, slots, left = sl.pages_extend(none, none, torch.zeros((0, 4), dtype=torch.int32, device=DEV), _t([4, 2, 7]),
                                               _t([2]), 5)
    torch.cuda.synchronize()
    assert lens.numel() == 0 and start.tolist() == [0] and slots.tolist() == [-1] * 5 and left.item() == 2


def test_refusals():
    lens, table, free = _case(np.random.default_rng(4), 6, 5, 3)
    tl, tt, tf, tc = _t(lens), _t(table), _t(free), _t([3])
    with pytest.raises(TypeError):
        sl.pages_extend(tl.long(), tl, tt, tf, tc, 8)
    with pytest.raises(ValueError):
        sl.pages_extend(tl, tl[:3], tt, tf, tc, 8)
    with pytest.raises(ValueError):
        sl.pages_extend(tl, tl, tt[:2], tf, tc, 8)
    with pytest.raises(ValueError):
        sl.pages_extend(tl, tl, tt.t(), tf, tc, 8)
    with pytest.raises(ValueError):
        sl.pages_extend(tl, tl, tt, tf, tc, 8, slots=tl)
    with pytest.raises(ValueError):
        sl.pages_release(tl.cpu(), tl, tt, tf, tc)
    big = torch.zeros(8193, dtype=torch.int32, device=DEV)
    with pytest.raises(sl.SlError):
        sl.pages_extend(big, big, torch.zeros((8193, 1), dtype=torch.int32, device=DEV), tf, tc, 8)
