"""The 4-bit oracle (oracle/fp4.py) against the format's definition, worked values and invariants (CPU)."""
import numpy as np
import pytest

from oracle import fp4


def _bits(x):
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def test_code_values_and_ties():
    # every code value returns itself; midpoints go to the even code; beyond 6 saturates
    for c, v in enumerate(fp4.VALUES):
        assert fp4.code(v) == c and fp4.code(-v) == c | 8
    for y, c in [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (7.0, 7), (100.0, 7),
                 (0.2500001, 1), (4.9999, 6), (5.0001, 7), (1e-9, 0)]:
        assert fp4.code(y) == c and fp4.code(-y) == c | 8, y


@pytest.mark.parametrize("top,byte", [(6.0, 127), (6.96875, 127), (7.0, 128), (12.0, 128), (13.9375, 128), (14.0, 129),
                                      (3.5, 127), (3.484375, 126), (1.0, 125), (0.0, 1), (2.0 ** -126, 1),
                                      (2.0 ** 127, 252), (1.9921875 * 2.0 ** 127, 252), (np.inf, 255), (np.nan, 255)])
def test_scale_byte(top, byte):
    """Smallest 2^e with max < 7 2^e: 7 - one bf16 step still fits e = 0, 7 does not."""
    x = np.zeros(32)
    x[7] = -top
    assert fp4.scale_byte(fp4.bf16_to_f64(_bits(x))) == byte


def test_scale_byte_equals_the_bit_rule():
    """((bits + 0x20) >> 7) - 2 within 1 .. 252, for every finite bf16 magnitude."""
    for bits in range(0, 0x7F80, 7):
        want = min(252, max(1, ((bits + 0x20) >> 7) - 2))
        assert fp4.scale_byte(fp4.bf16_to_f64(np.array([bits] + [0] * 31, np.uint16))) == want, hex(bits)


def test_quantisation_error_bound():
    """Half a step everywhere: |stored - x| <= max(|x| / 4, 2^e / 4), and a maximum never saturates."""
    rng = np.random.default_rng(0)
    x = fp4.bf16_to_f64(_bits(rng.normal(size=(300, 64)) * np.exp(rng.normal(size=(300, 1)) * 5)))
    codes, scales = fp4.quantise(fp4.f64_to_bf16(x))
    err = np.abs(fp4.values(codes, scales) - x)
    unit = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=-1)
    assert (err <= np.maximum(np.abs(x) / 4, unit / 4)).all()
    assert (np.abs(x) < 7 * unit).all()


@pytest.mark.parametrize("D", [64, 128])
def test_layout_covers_every_byte_once(D):
    k, v, shift, ks, vs = fp4.layout(D)
    seen = np.zeros((17 * D, 2), int)
    for at in (k, v):
        np.add.at(seen, (at, shift // 4), 1)
    for at in (ks, vs):
        seen[at.ravel()] += 1
    assert (seen == 1).all()


@pytest.mark.parametrize("D", [64, 128])
def test_write_read_round_trip(D):
    rng = np.random.default_rng(D)
    pool = rng.integers(0, 256, (3, 2, 17 * D)).astype(np.uint8)
    slots = np.array([5, -1, 47, 16, 48, 0])
    k, v = (_bits(rng.normal(size=(6, 2, D))) for _ in range(2))
    new = fp4.write(k, v, slots, pool)
    rk, rv = fp4.read(slots, new)
    for rows, got in ((k, rk), (v, rv)):
        want = fp4.values(*fp4.quantise(rows))
        assert np.array_equal(got[[0, 2, 3, 5]], want[[0, 2, 3, 5]])
        assert (got[1] == 0).all() and np.isnan(got[4]).all()
    # every slot that was not written keeps its bytes
    old, now = fp4.unpack(pool), fp4.unpack(new)
    keep = np.ones(48, bool)
    keep[[5, 47, 16, 0]] = False
    for a, b in zip(old, now):
        a, b = (x.transpose(0, 2, 1, 3).reshape(48, 2, D)[keep] for x in (a, b))
        assert np.array_equal(a, b, equal_nan=True)


def test_pages_worked_example():
    """Four requests of 5, 16, 0 and 31 tokens; the stack holds 9, 4, 7 (top 7)."""
    table = np.array([[20, 0, 0], [21, 0, 0], [0, 0, 0], [22, 23, 0]])
    free = np.array([9, 4, 7] + [0] * 21)
    lens, start, slots, count, now = fp4.pages_extend([5, 16, 0, 31], [2, 1, 0, 2], table, free, 3, 8)
    assert lens == [7, 17, 0, 33] and start == [0, 2, 3, 3, 5] and count == 1
    assert slots == [20 * 16 + 5, 20 * 16 + 6, 7 * 16, 23 * 16 + 15, 4 * 16, -1, -1, -1]
    assert now[1, 1] == 7 and now[3, 2] == 4
    # the second opens one page, the fourth finds none left; the first needs none
    lens, start, slots, count, now = fp4.pages_extend([5, 16, 0, 31], [2, 1, 0, 2], table, free, 1, 8)
    assert lens == [7, 17, 0, 31] and start == [0, 2, 3, 3, 3] and count == 0 and now[1, 1] == 9
    lens, count, back = fp4.pages_release([0, 1, 1, 1], [5, 16, 0, 31], table, free, 3)
    assert lens == [5, 0, 0, 0] and count == 6 and list(back[:6]) == [9, 4, 7, 21, 23, 22]


def test_extend_after_release_returns_the_same_pages():
    rng = np.random.default_rng(3)
    for _ in range(50):
        B, blocks = int(rng.integers(1, 9)), int(rng.integers(1, 7))
        lens = rng.integers(0, blocks * 16 + 1, B)
        N = B * blocks + 4
        perm = rng.permutation(N)
        table = perm[:B * blocks].reshape(B, blocks)
        free = np.zeros(N, int)
        free[:4] = perm[B * blocks:]
        done = rng.integers(0, 2, B)
        zero, count, stack = fp4.pages_release(done, lens, table, free, 4)
        again = np.where(done == 1, lens, 0)
        back, start, slots, left, now = fp4.pages_extend(zero, again, table, stack, count, int(again.sum()))
        assert back == list(lens) and left == 4 and start[-1] == again.sum()
        held = sorted(int(p) for b in range(B) for p in now[b, :-(-lens[b] // 16)])
        assert held == sorted(int(p) for b in range(B) for p in table[b, :-(-lens[b] // 16)])
