"""The 4-bit cache and the page bookkeeping in plain numpy (test infrastructure, like the rest of this package).

Everything here is written from the definitions in ``include/sl.h``: the record's layout by a loop over (slot, element),
the quantiser by a search over the code values in 64 bits, the bookkeeping request by request. Cached values are powers
of two times code values and so exact in bf16: attention over a 4-bit cache is ``oracle.decode_attn`` on the unpacked
bf16 pages. Pinned by ``tests/test_fp4_oracle.py``.
"""
from __future__ import annotations

import functools
import math

import numpy as np

PAGE = 16
BLOCK = 32
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16_to_f64(bits) -> np.ndarray:
    with np.errstate(invalid="ignore"):   # (signalling NaNs)
        return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def f64_to_bf16(x) -> np.ndarray:
    """bf16 bits of values that bf16 holds exactly (NaN: 0x7FC0); anything else is refused."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(over="ignore"):
        f = x.astype(np.float32)
    bits = np.where(np.isnan(x), np.uint32(0x7FC00000), f.view(np.uint32))
    if not (np.isnan(x) | (f.astype(np.float64) == x)).all() or (bits & 0xFFFF).any():
        raise ValueError("a value that bf16 does not hold")
    return (bits >> 16).astype(np.uint16)


def scale_byte(block) -> int:
    """E8M0 byte of a block of float64 elements."""
    a = np.abs(block).max()
    if not np.isfinite(a):
        return 255
    e = -126
    while e < 125 and not a < 7.0 * 2.0 ** e:
        e += 1
    return e + 127


def code(y: float) -> int:
    """E2M1 code nearest to y, ties to the even code, saturating; the sign bit is y's."""
    a = abs(y)
    d = np.abs(VALUES - a)
    best = int(np.argmin(d))
    if best < 7 and d[best + 1] == d[best] and best % 2 == 1:
        best += 1
    return best | (8 if math.copysign(1.0, y) < 0 else 0)


def quantise(bits) -> tuple[np.ndarray, np.ndarray]:
    """Rows of bf16 bits [..., D] -> codes [..., D] and scale bytes [..., D / 32] (uint8)."""
    x = bf16_to_f64(bits)
    blocks = x.reshape(-1, BLOCK)
    codes = np.zeros(blocks.shape, np.uint8)
    scales = np.zeros(len(blocks), np.uint8)
    for i, b in enumerate(blocks):
        scales[i] = scale_byte(b)
        if scales[i] != 255:
            unit = 2.0 ** (int(scales[i]) - 127)
            codes[i] = [code(v / unit) for v in b]
    return codes.reshape(x.shape), scales.reshape(*x.shape[:-1], x.shape[-1] // BLOCK)


def values(codes, scales) -> np.ndarray:
    """Codes [..., D] and scale bytes [..., D / 32] -> float64 values."""
    v = VALUES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return v * np.repeat(s, BLOCK, axis=-1)


@functools.lru_cache(maxsize=None)
def layout(D: int):
    """Byte (and shift) of every element's code and of every block's scale in a record: arrays [16, D] and [16, D / 32]."""
    C, E = D // 32, D // 16
    k, v, shift = (np.zeros((PAGE, D), np.int64) for _ in range(3))
    ks, vs = (np.zeros((PAGE, C), np.int64) for _ in range(2))
    for t in range(PAGE):
        for d in range(D):
            k[t, d] = 256 * (d // 32) + 16 * t + (d % 32) // 2
            v[t, d] = 8 * D + 2 * E * (16 * (t // 4) + d // E) + (E // 2) * (t % 4) + (d % E) // 2
            shift[t, d] = 4 * (d % 2)
        for c in range(C):
            ks[t, c] = 16 * D + 16 * c + t
            vs[t, c] = 16 * D + D // 2 + 4 * (C * (t // 4) + c) + t % 4
    return k, v, shift, ks, vs


def unpack(pool) -> tuple[np.ndarray, np.ndarray]:
    """Records [N, Hkv, 17 D] -> float64 key and value pages [N, Hkv, 16, D]."""
    pool = np.asarray(pool)
    k, v, shift, ks, vs = layout(pool.shape[2] // 17)
    return (values((pool[:, :, k] >> shift) & 15, pool[:, :, ks]), values((pool[:, :, v] >> shift) & 15, pool[:, :, vs]))


def write(k_new, v_new, slots, pool) -> np.ndarray:
    """Rows of bf16 bits [T, Hkv, D] into slots [T]; returns an updated copy of the pool."""
    pool = np.array(pool, copy=True)
    N, Hkv, size = pool.shape
    k, v, shift, ks, vs = layout(size // 17)
    for rows, at, at_scale in ((k_new, k, ks), (v_new, v, vs)):
        codes, scales = quantise(rows)
        for i, s in enumerate(slots):
            if not 0 <= s < N * PAGE:
                continue
            page, t = divmod(int(s), PAGE)
            for g in range(Hkv):
                rec = pool[page, g]
                rec[at[t, ::2]] = codes[i, g, ::2] | codes[i, g, 1::2] << 4
                rec[at_scale[t]] = scales[i, g]
    return pool


def append_slots(block_table, seq_lens, num_pages) -> np.ndarray:
    """Slot of each sequence's newest token (-1: none, or invalid)."""
    B, blocks = block_table.shape
    out = np.full(B, -1, np.int64)
    for b, L in enumerate(seq_lens):
        if 0 < L <= blocks * PAGE:
            page = block_table[b, (L - 1) // PAGE]
            if 0 <= page < num_pages:
                out[b] = page * PAGE + (L - 1) % PAGE
    return out


def read(slots, pool) -> tuple[np.ndarray, np.ndarray]:
    """Key and value rows (float64 [T, Hkv, D]) of slots [T]."""
    N, Hkv, size = pool.shape
    kv = unpack(pool)
    out = []
    for pages in kv:
        rows = np.zeros((len(slots), Hkv, size // 17))
        for i, s in enumerate(slots):
            if s >= N * PAGE:
                rows[i] = np.nan
            elif s >= 0:
                rows[i] = pages[s // PAGE, :, s % PAGE]
        out.append(rows)
    return out[0], out[1]


def pages_extend(seq_lens, new_tokens, block_table, free_pages, free_count, max_tokens):
    """(seq_lens_out, token_start, slots, free_count_out, block_table) as lists / arrays of Python integers."""
    table = np.array(block_table, copy=True)
    B, blocks = table.shape
    N, count = len(free_pages), max(0, min(int(free_count), len(free_pages)))
    lens, start, slots, taken = [int(x) for x in seq_lens], [0], [], 0
    sum_tokens = sum_pages = 0
    for b in range(B):
        L, n = lens[b], int(new_tokens[b])
        if 0 <= L <= blocks * PAGE and n >= 0 and L + n <= blocks * PAGE:
            opens = -(-(L + n) // PAGE) - -(-L // PAGE)
            sum_tokens += n
            sum_pages += opens
            if sum_tokens <= max_tokens and (opens == 0 or sum_pages <= count):
                for j in range(opens):
                    taken += 1
                    table[b, -(-L // PAGE) + j] = free_pages[count - taken]
                for p in range(L, L + n):
                    page = int(table[b, p // PAGE])
                    slots.append(page * PAGE + p % PAGE if 0 <= page < N else -1)
                lens[b] = L + n
        start.append(len(slots))
    return lens, start, slots + [-1] * (max_tokens - len(slots)), count - taken, table


def pages_release(finished, seq_lens, block_table, free_pages, free_count):
    """(seq_lens_out, free_count_out, free_pages)."""
    free = np.array(free_pages, copy=True)
    B, blocks = np.shape(block_table)
    count = max(0, min(int(free_count), len(free)))
    lens = [int(x) for x in seq_lens]
    for b in range(B):
        if finished[b] and 0 <= lens[b] <= blocks * PAGE:
            for j in reversed(range(-(-lens[b] // PAGE))):
                if count < len(free):
                    free[count] = block_table[b][j]
                    count += 1
            lens[b] = 0
    return lens, count, free
