"""The 4-bit cache on the GPU: rows in and out against oracle/fp4.py byte for byte, attention (plain and with prefix
sharing) against the fp64 oracle on the cache's values, and a decode step of all of it, also captured and replayed."""
import numpy as np
import pytest
import torch

from oracle import fp4
from paper_2504_15930_amd import inputs, sl
from fp4_batches import DEV, bits, make, quantised, reference
from parity import assert_parity, sample_rows

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs an MI355X")]


def _say(*a):
    print(*a, flush=True)


def _t(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x), dtype=dtype, device=DEV)


def _bf16(b):
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).to(DEV).view(torch.bfloat16)


def _bf16_bits(x):
    return bits(torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16))


# ---- rows ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("D", [64, 128])
def test_every_bf16_value(D):
    """Every bit pattern (zeros, subnormals, NaN and infinities among them) in blocks of neighbouring magnitudes, and
    again beside one element 2^0 to 2^7 times larger: bytes equal the oracle's."""
    _say("every bf16 value, D =", D)
    plain = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16).reshape(-1, 2, D)
    rng = np.random.default_rng(0)
    mixed = rng.permutation(1 << 16).astype(np.uint16)
    mixed = mixed[(mixed & 0x7FFF) < 0x7C00].reshape(-1)
    mixed = mixed[:len(mixed) // (2 * D) * 2 * D].reshape(-1, 2, D)
    near = ((rng.integers(0x3F00, 0x4380, 1 << 15) | (rng.integers(0, 2, 1 << 15) << 15)).astype(np.uint16)
            .reshape(-1, 2, D))
    rows = np.concatenate([plain, mixed, near])
    other = rows[::-1].copy()
    pool = torch.full((-(-len(rows) // 16), 2, 17 * D), 0x5A, dtype=torch.uint8, device=DEV)
    want = fp4.write(rows, other, np.arange(len(rows)), pool.cpu().numpy())
    sl.kv_write_fp4(_bf16(rows), _bf16(other), torch.arange(len(rows), dtype=torch.int32, device=DEV), pool)
    torch.cuda.synchronize()
    assert np.array_equal(pool.cpu().numpy(), want)


@pytest.mark.parametrize("T,Hkv,D", [(1, 1, 64), (1, 8, 128), (7, 3, 64), (33, 4, 128), (257, 1, 64), (500, 5, 128)])
def test_write_and_read(T, Hkv, D):
    """Scattered slots, some of them none or past the pool; every byte that belongs to no written row is kept."""
    _say("write and read", T, Hkv, D)
    rng = np.random.default_rng(T)
    N = T // 16 + 3
    slots = rng.permutation(N * 16)[:T].astype(np.int32)
    slots[rng.random(T) < 0.1] = -1
    if T > 5:
        slots[3], slots[5] = N * 16, 2 ** 31 - 1
    k, v = (_bf16_bits(rng.normal(size=(T, Hkv, D)) * np.exp(rng.normal(size=(T, 1, 1)) * 3)) for _ in range(2))
    pool = torch.from_numpy(rng.integers(0, 256, (N, Hkv, 17 * D)).astype(np.uint8)).to(DEV)
    want = fp4.write(k, v, slots, pool.cpu().numpy())
    sl.kv_write_fp4(_bf16(k), _bf16(v), _t(slots), pool)
    rk, rv = sl.kv_read_fp4(_t(slots), pool)
    torch.cuda.synchronize()
    assert np.array_equal(pool.cpu().numpy(), want)
    for got, ref in zip((rk, rv), fp4.read(slots, want)):
        assert np.array_equal(got.float().cpu().double().numpy(), ref, equal_nan=True)


@pytest.mark.parametrize("D", [64, 128])
def test_every_code_under_every_scale_byte(D):
    """Records that others wrote: all 16 codes under all 256 scale bytes, read back as they are defined; bf16 holds
    each of them but those of 2^128 and beyond, which are infinite in it."""
    T, C = 256, D // 32
    k, v, shift, ks, vs = fp4.layout(D)
    pool = np.zeros((T // 16, 1, 17 * D), np.uint8)
    codes = (np.arange(D) + np.arange(T)[:, None]) % 16
    for t in range(T):
        rec = pool[t // 16, 0]
        for at, at_scale in ((k, ks), (v, vs)):
            rec[at[t % 16, ::2]] = codes[t, ::2] | codes[t, 1::2] << 4
            rec[at_scale[t % 16]] = (t + 85 * np.arange(C)) % 256
    got = sl.kv_read_fp4(torch.arange(T, dtype=torch.int32, device=DEV), torch.from_numpy(pool).to(DEV))
    torch.cuda.synchronize()
    want = fp4.values(codes, ((np.arange(T)[:, None] + 85 * np.arange(C)) % 256).astype(np.uint8))
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    for x in got:
        assert np.array_equal(x[:, 0].float().cpu().double().numpy(), want, equal_nan=True)


def test_whole_pages_in_order():
    """A prompt's rows in slot order, pages scattered, the last one partly filled."""
    rng = np.random.default_rng(8)
    L, Hkv, D = 16 * 40 + 5, 4, 128
    pages = rng.permutation(64)[:41]
    slots = (pages[np.arange(L) // 16] * 16 + np.arange(L) % 16).astype(np.int32)
    k, v = (_bf16_bits(rng.normal(size=(L, Hkv, D))) for _ in range(2))
    pool = torch.zeros((64, Hkv, 17 * D), dtype=torch.uint8, device=DEV)
    want = fp4.write(k, v, slots, pool.cpu().numpy())
    sl.kv_write_fp4(_bf16(k), _bf16(v), _t(slots), pool)
    rk, rv = sl.kv_read_fp4(_t(slots), pool)
    torch.cuda.synchronize()
    assert np.array_equal(pool.cpu().numpy(), want)
    for got, ref in zip((rk, rv), fp4.read(slots, want)):
        assert np.array_equal(got.float().cpu().double().numpy(), ref)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B", [1, 3, 65])
def test_append(B, D):
    """The newest token of every sequence; empty and invalid sequences and bad pages leave the pool as it was."""
    _say("append", B, D)
    rng = np.random.default_rng(B + D)
    blocks, Hkv = 5, 3
    lens = rng.integers(1, blocks * 16 + 1, B).astype(np.int32)
    N = B * blocks
    table = rng.permutation(N).astype(np.int32).reshape(B, blocks)
    if B > 8:
        lens[[1, 2, 3, 4]] = [0, -5, blocks * 16 + 1, 2 ** 31 - 1]
        table[6, (lens[6] - 1) // 16] = -1
        table[7, (lens[7] - 1) // 16] = N
    k, v = (_bf16_bits(rng.normal(size=(B, Hkv, D))) for _ in range(2))
    pool = torch.from_numpy(rng.integers(0, 256, (N, Hkv, 17 * D)).astype(np.uint8)).to(DEV)
    want = fp4.write(k, v, fp4.append_slots(table, lens, N), pool.cpu().numpy())
    sl.kv_append_fp4(_bf16(k), _bf16(v), _t(table), _t(lens), pool)
    torch.cuda.synchronize()
    assert np.array_equal(pool.cpu().numpy(), want)


# ---- attention ----------------------------------------------------------------------------------------------------
# The cached values are exact in bf16 and the arithmetic is that of a bf16 cache, so its tolerances hold (parity.py).

SHAPES = [
    (1, 8, 1, 128, [1]),
    (3, 8, 2, 64, [15, 16, 17]),
    (5, 28, 4, 128, [1, 33, 100, 16, 250]),
    (17, 16, 16, 64, (1, 300)),       # G = 1
    (33, 40, 8, 128, (1, 500)),       # G = 5
    (9, 14, 2, 64, (1, 200)),         # G = 7
    (6, 32, 2, 128, (1, 400)),        # G = 16
    (4, 64, 8, 128, [1000, 2000, 17, 3000]),
    (6, 4, 4, 128, [0, 5, 0, 32, 64, 49]),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"B{s[0]}_Hq{s[1]}_Hkv{s[2]}_D{s[3]}")
@pytest.mark.parametrize("workers", [0, 1, 7, 1000])
def test_attention_shapes(shape, workers):
    B, hq, hkv, d, spec = shape
    L = np.random.default_rng(B * 31 + d).integers(spec[0], spec[1] + 1, B) if isinstance(spec, tuple) else np.array(spec)
    _say("attention", shape, "workers", workers)
    b, pool = make(L, hq, hkv, d, seed=B + hq)
    out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, num_workers=workers)
    torch.cuda.synchronize()
    assert_parity(out, reference(b, pool), f"{shape} workers={workers}")


@pytest.mark.parametrize("i", range(24))
def test_attention_sweep(i):
    rng = np.random.default_rng(4000 + i)
    d, hkv = int(rng.choice([64, 128])), int(rng.choice([1, 2, 4, 8]))
    G, B = int(rng.choice([1, 2, 3, 4, 5, 7, 8, 16])), int(rng.choice([1, 2, 3, 8, 31, 64, 130, 257]))
    kind = rng.integers(0, 4, B)
    L = np.where(kind == 0, rng.choice([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65], B),
                 np.where(kind == 1, rng.integers(1, 64, B),
                          np.where(kind == 2, np.minimum(np.exp(rng.normal(np.log(300), 1.2, B)).astype(np.int64) + 1, 6000),
                                   16 * rng.integers(1, 40, B))))
    workers = int(rng.choice([0, 0, 1, 2, 5, 33, 256, 1000]))
    _say(f"sweep {i}: B={B} G={G} Hkv={hkv} D={d} workers={workers} total={int(L.sum())}")
    b, pool = make(L, G * hkv, hkv, d, seed=5000 + i)
    out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, num_workers=workers)
    torch.cuda.synchronize()
    assert_parity(out, reference(b, pool), f"sweep {i}")


@pytest.mark.parametrize("blocks", [1, 2, 127, 128, 129, 255, 256, 257, 300])
@pytest.mark.parametrize("B,hq,hkv,d", [(3, 28, 4, 128), (70, 32, 8, 64), (7, 32, 2, 64), (300, 16, 1, 128)])
def test_table_widths(B, hq, hkv, d, blocks):
    """Tables around the width where short sequences get a workgroup each: lengths of 0, 1, all of the table and others
    with the default division of the work, and beyond the table and below zero."""
    _say("table width", B, hq, hkv, d, blocks)
    rng = np.random.default_rng(blocks)
    L = np.minimum(rng.integers(0, 16 * blocks + 1, B), np.where(rng.random(B) < 0.3, 16 * blocks, 700))
    L[0], L[-1] = 16 * blocks, 1
    L[1] = 0
    b, pool = make(L, hq, hkv, d, seed=blocks)
    rows = list(range(min(B, 12)))
    ref = reference(b, pool, rows)
    out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale)
    torch.cuda.synchronize()
    assert b.block_table.shape[1] == blocks
    assert_parity(out[rows], ref, f"{blocks} blocks")
    lens = b.seq_lens.clone()
    lens[0], lens[1] = 16 * blocks + 1, -3
    table = b.block_table.clone()
    table[2, 0] = pool.shape[0]
    again = sl.decode_attn_fp4(b.q, pool, table, lens, b.scale)
    torch.cuda.synchronize()
    assert torch.isnan(again[:2]).all() and (L[2] == 0 or torch.isnan(again[2]).all())
    assert torch.equal(again[3:], out[3:])


@pytest.mark.parametrize("B,blocks", [(129, 65), (256, 128), (257, 65), (511, 66), (512, 65), (513, 65), (1024, 65), (1025, 65),
                                      (65, 256), (130, 255), (200, 256)])
@pytest.mark.parametrize("law", ["edges", "equal", "empty"])
def test_every_sequence_in_its_turn(B, blocks, law):
    """More units than CUs over long tables, where the longer sequences are started first: every sequence is attended
    once, whatever quarters of the table's width their lengths lie in."""
    _say("turns", B, blocks, law)
    rng = np.random.default_rng(B)
    edges = [x for q in (0, 4 * blocks, 8 * blocks, 12 * blocks, 16 * blocks) for x in (q - 1, q, q + 1)
             if 0 <= x <= 16 * blocks]
    L = {"edges": rng.choice(edges, B), "equal": np.full(B, 100), "empty": np.zeros(B, np.int64)}[law]
    L[int(rng.integers(B))] = 16 * blocks
    b, pool = make(L, 4, 2, 64, seed=B)
    out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale)
    torch.cuda.synchronize()
    assert b.block_table.shape[1] == blocks
    rows = sorted({0, 1, B // 2, B - 2, B - 1, int(L.argmax()), *rng.integers(0, B, 20).tolist()})
    assert_parity(out[rows], reference(b, pool, rows), f"{B} x {blocks} {law}")
    split = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, num_workers=512)
    # (both within the tolerance of the oracle: within twice of one another)
    assert ((out.float() - split.float()).abs() <= 2e-2 + 4e-2 * split.float().abs()).all()
    lens = b.seq_lens.clone()
    bad = [0, B // 2]
    lens[bad[0]], lens[bad[1]] = -1, 2 ** 31 - 1
    again = sl.decode_attn_fp4(b.q, pool, b.block_table, lens, b.scale)
    torch.cuda.synchronize()
    keep = [i for i in range(B) if i not in bad]
    assert torch.isnan(again[bad]).all() and torch.equal(again[keep], out[keep])


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-3, 30.0])
@pytest.mark.parametrize("workers", [0, 5])
def test_scales(scale, workers):
    """Negative, zero, small and large factors; a large one makes the softmax pick single tokens."""
    b, pool = make([1, 17, 300, 64, 33], 14, 2, 128, seed=12)
    b.scale = float(np.float32(scale))
    out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, num_workers=workers)
    torch.cuda.synchronize()
    assert_parity(out, reference(b, pool), f"scale {scale}")


@pytest.mark.parametrize("D", [64, 128])
def test_one_token_returns_its_value_row(D):
    b, pool = make([1] * 9, 8, 2, D, seed=3)
    out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale)
    _, v = sl.kv_read_fp4(b.block_table[:, 0] * 16, pool)
    torch.cuda.synchronize()
    assert torch.equal(out, v.repeat_interleave(4, 1))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("workers", [0, 3])
def test_dominant_token_at_every_position(D, workers):
    """A key along q beside keys orthogonal to it, its score ahead by 64 and more: the output is that token's value row."""
    L, Hkv = 130, 2
    _say("dominant token", D, workers)
    rng = np.random.default_rng(1)
    q = np.zeros((L, Hkv, D), np.float32)
    q[:, :, ::2] = 16.0
    k = np.zeros((L, L, Hkv, D), np.float32)      # [sequence, token]
    k[:, :, :, 1::2] = rng.choice([-2.0, 2.0], size=(L, L, Hkv, D // 2))
    for b in range(L):
        k[b, b, :, ::2] = 4.0
    v = rng.choice([-3.0, -1.0, 0.5, 2.0, 4.0, 6.0], size=(L, L, Hkv, D))
    blocks = -(-L // 16)
    table = rng.permutation(L * blocks).astype(np.int32).reshape(L, blocks)
    slots = (table[:, np.arange(L) // 16] * 16 + np.arange(L) % 16).astype(np.int32)
    pool = torch.full((L * blocks, Hkv, 17 * D), 0xFF, dtype=torch.uint8, device=DEV)
    vb = _bf16_bits(v)
    sl.kv_write_fp4(_bf16(_bf16_bits(k).reshape(L * L, Hkv, D)), _bf16(vb.reshape(L * L, Hkv, D)), _t(slots.ravel()), pool)
    out = sl.decode_attn_fp4(_bf16(_bf16_bits(q)), pool, _t(table), _t([L] * L), 1.0, num_workers=workers)
    torch.cuda.synchronize()
    stored = fp4.values(*fp4.quantise(vb[np.arange(L), np.arange(L)]))
    assert np.array_equal(out.float().cpu().double().numpy(), stored)


@pytest.mark.parametrize("D", [64, 128])
def test_invalid_data_gives_nan_rows_there_only(D):
    b, pool = make([40, 0, 7, 70, 33, 90, 16], 8, 2, D, seed=9)
    ref = reference(b, pool)
    table, lens = b.block_table.clone(), b.seq_lens.clone()
    lens[2], lens[3] = -1, table.shape[1] * 16 + 1
    table[4, 1], table[5, 0] = pool.shape[0], -7
    out = sl.decode_attn_fp4(b.q, pool, table, lens, b.scale)
    torch.cuda.synchronize()
    assert torch.isnan(out[[2, 3, 4, 5]]).all()
    assert_parity(out[[0, 1, 6]], ref[[0, 1, 6]], "valid sequences")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("which", ["k", "v", "q"])
def test_nan_and_infinity_reach_their_own_head_only(D, which):
    """A NaN or infinite key, value or query element poisons the rows that use it (all of a key's and query's head, the
    32 columns of a value's block) and nothing else."""
    b, pool = make([50, 50], 8, 2, D, seed=4)
    ref = reference(b, pool)
    page, t = int(b.block_table[0, 1]), 5
    k, v = (x[page, :, t].clone()[None] for x in (b.k_pages, b.v_pages))
    q = b.q.clone()
    {"k": k, "v": v, "q": q}[which][(0, 5, 33) if which == "q" else (0, 1, 33)] = float("inf") if D == 64 else float("nan")
    sl.kv_write_fp4(k, v, _t([page * 16 + t]), pool)
    out = sl.decode_attn_fp4(q, pool, b.block_table, b.seq_lens, b.scale)
    torch.cuda.synchronize()
    got = out.float().cpu().double().numpy()
    bad = np.zeros(got.shape, bool)
    if which == "q":
        bad[0, 5] = True
    elif which == "k":
        bad[0, 4:8] = True
    else:
        bad[0, 4:8, 32:64] = True
    assert np.isnan(got[bad]).all()
    assert np.isfinite(got[~bad]).all()
    assert (np.abs(got - ref)[~bad] <= 1e-2 + 2e-2 * np.abs(ref[~bad])).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("workers", [0, 7])
def test_a_nan_key_poisons_from_every_position(D, workers):
    """Sequence i's key i of one head is NaN, i over all positions: also where it is the only token of a wavefront's
    share. Its rows are NaN whatever the other shares hold."""
    n = 147
    lens = np.maximum(np.arange(n) + 1, np.arange(n) % 5 * 30)
    b, pool = make(lens, 12, 2, D, seed=61)
    at = np.arange(n)
    slots = b.block_table.cpu().numpy()[at, at // 16] * 16 + at % 16
    k, v = sl.kv_read_fp4(_t(slots), pool)
    k[:, 1, 3] = float("nan")
    sl.kv_write_fp4(k, v, _t(slots), pool)
    out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, num_workers=workers)
    torch.cuda.synchronize()
    assert torch.isfinite(out[:, :6]).all()
    assert torch.isnan(out[:, 6:]).all()


def test_a_long_pool_past_32_bits():
    """Records beyond the first 4 GB of a pool (and beyond 2^31 bytes) are read and written where they are."""
    D, Hkv = 128, 8
    N = (1 << 32) // (Hkv * 17 * D) + 100
    pool = torch.empty((N, Hkv, 17 * D), dtype=torch.uint8, device=DEV)
    b = inputs.make_paged_batch([100, 17, 250], 16, Hkv, D, seed=2, device=DEV)
    small = quantised(b)
    far = torch.tensor([N - 1 - i for i in range(small.shape[0])], device=DEV)
    pool[far] = small
    out = sl.decode_attn_fp4(b.q, pool, far[b.block_table.long()].int(), b.seq_lens, b.scale)
    want = sl.decode_attn_fp4(b.q, small, b.block_table, b.seq_lens, b.scale)
    slots = (far[:4].int()[:, None] * 16 + torch.arange(16, device=DEV, dtype=torch.int32)).reshape(-1)
    rk, rv = sl.kv_read_fp4(slots, pool)
    wk, wv = sl.kv_read_fp4(torch.arange(64, dtype=torch.int32, device=DEV), small)
    sl.kv_write_fp4(torch.zeros_like(rk), torch.ones_like(rv), slots, pool)
    zk, zv = sl.kv_read_fp4(slots, pool)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    assert torch.equal(rk.view(torch.int16), wk.view(torch.int16)) and torch.equal(rv.view(torch.int16), wv.view(torch.int16))
    assert (zk == 0).all() and (zv == 1).all()


@pytest.mark.parametrize("name", ["qwen7b_longtail", "straggler"])
def test_full_size(name):
    """The benchmark's workloads at full size with default workers, sampled sequences against the oracle."""
    _say("full size", name)
    b = inputs.make_batch(name, seed=0, device=DEV)
    pool = quantised(b)
    out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale)
    torch.cuda.synchronize()
    rows = sample_rows(b.seq_lens, 6, seed=5)
    assert_parity(out[rows], reference(b, pool, rows), name)


def test_largest_batch():
    rng = np.random.default_rng(0)
    b, pool = make(rng.integers(0, 34, 8192), 4, 2, 64, seed=1)
    out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale)
    torch.cuda.synchronize()
    assert_parity(out, reference(b, pool), "8192 sequences")


# ---- prefix sharing -----------------------------------------------------------------------------------------------

GRPO = [
    # prompts, samples, prompt, heads, KV heads, D, median, cap
    (2, 3, 40, 8, 2, 64, 20, 60),
    (5, 8, 100, 28, 4, 128, 30, 200),
    (3, 16, 1000, 64, 8, 128, 100, 400),
    (4, 1, 333, 12, 12, 64, 50, 100),
    (3, 22, 130, 12, 12, 64, 23, 64),
    (6, 5, 64, 16, 1, 128, 0.001, 1),     # nothing generated
]


@pytest.mark.parametrize("case", GRPO)
@pytest.mark.parametrize("workers", [0, 1, 7, 1000])
def test_prefix_shapes(case, workers):
    prompts, samples, prompt, hq, hkv, d, median, cap = case
    _say("prefix", case, workers)
    b, starts, shared = inputs.make_grpo_batch(prompts, samples, prompt, seed=prompt, device=DEV, num_q_heads=hq,
                                               num_kv_heads=hkv, head_dim=d, gen_median=median, gen_cap=cap)
    pool = quantised(b)
    out = sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, starts, shared, num_workers=workers)
    torch.cuda.synchronize()
    assert_parity(out, reference(b, pool), f"prefix {case} {workers}")


def test_prefix_odd_groups():
    """No groups; groups that are empty, descending or too long; a member shorter than its prefix gets NaN rows."""
    b, starts, shared = inputs.make_grpo_batch(4, 6, 100, seed=3, device=DEV, num_q_heads=8, num_kv_heads=2, head_dim=128,
                                               gen_median=40, gen_cap=90)
    pool = quantised(b)
    ref = reference(b, pool)
    none = torch.zeros(1, dtype=torch.int32, device=DEV)
    for gs, sp in ((none, none[:0]), (starts, torch.zeros_like(shared)), (starts, shared + b.block_table.shape[1]),
                   (_t([12, 6, 12, 18, 24]), shared), (_t([6, 12, 0, 6, 24]), shared), (_t([0, 6, 12, 18, 30]), shared)):
        out = sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, gs, sp)
        torch.cuda.synchronize()
        assert_parity(out, ref, f"groups {gs.tolist()} {sp.tolist()}")
    lens = b.seq_lens.clone()
    lens[7] = 95
    out = sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, lens, b.scale, starts, shared)
    torch.cuda.synchronize()
    keep = [i for i in range(24) if i != 7]
    assert torch.isnan(out[7]).all()
    assert_parity(out[keep], ref[keep], "the others")


@pytest.mark.parametrize("case", [(3, 5, 2100, 28, 4, 128, 30, 200), (2, 9, 2070, 16, 4, 64, 20, 100),
                                  (3, 3, 2050, 12, 12, 64, 30, 90), (300, 2, 40, 8, 2, 128, 10, 30),
                                  (2, 3, 3970, 28, 4, 128, 30, 126), (2, 3, 4090, 28, 4, 128, 30, 126),
                                  (2, 5, 4000, 8, 2, 64, 30, 96), (2, 12, 4000, 12, 12, 64, 30, 96)])
def test_prefix_past_the_short_tables(case):
    """More than 128 or 256 blocks per sequence, or more than 256 groups."""
    test_prefix_shapes(case, 0)


@pytest.mark.parametrize("workers", [0, 5])
def test_prefix_short_members(workers):
    """A member shorter than its prompt's shared pages gets NaN rows; in a range that is not shared (it starts before an
    earlier one's end) the same length is attended as it is."""
    b, starts, shared = inputs.make_grpo_batch(4, 6, 100, seed=3, device=DEV, num_q_heads=8, num_kv_heads=2, head_dim=64,
                                               gen_median=40, gen_cap=90)
    pool = quantised(b)
    for i in (2, 7, 15):
        b.seq_lens[i] = 95
    b.seq_lens[20] = 0
    ref = reference(b, pool)
    for gs, sp, short in ((starts, shared, [2, 7, 15, 20]), (_t([6, 12, 0, 6, 24]), shared, [7]),
                          (_t([0, 6, 12, 30, 24]), shared, [2, 7]), (starts, torch.zeros_like(shared), [])):
        out = sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, gs, sp, num_workers=workers)
        torch.cuda.synchronize()
        keep = [i for i in range(24) if i not in short]
        assert torch.isnan(out[short]).all()
        assert_parity(out[keep], ref[keep], f"groups {gs.tolist()} {sp.tolist()}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("workers", [0, 9])
def test_prefix_a_nan_key_poisons_from_every_position(D, workers):
    """Key t of one head is NaN: in the first group's prompt it reaches its members' rows of that head, in a member's
    own tokens that member's alone."""
    b, starts, shared = inputs.make_grpo_batch(2, 3, 48, seed=8, device=DEV, num_q_heads=12, num_kv_heads=2, head_dim=D,
                                               gen_median=20, gen_cap=40)
    pool = quantised(b)
    for t in range(int(b.seq_lens[1])):
        slot = _t([int(b.block_table[1, t // 16]) * 16 + t % 16])
        k, v = sl.kv_read_fp4(slot, pool)
        k2 = k.clone()
        k2[:, 1, 3] = float("nan")
        sl.kv_write_fp4(k2, v, slot, pool)
        out = sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, starts, shared, num_workers=workers)
        bad = torch.zeros(out.shape[:2], dtype=torch.bool, device=DEV)
        bad[slice(0, 3) if t < 48 else slice(1, 2), 6:] = True
        assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all(), t
        sl.kv_write_fp4(k, v, slot, pool)     # (stored values come back as they were)


def test_prefix_largest_batch():
    b, starts, shared = inputs.make_grpo_batch(2048, 2, 33, seed=6, device=DEV, num_q_heads=4, num_kv_heads=2,
                                               head_dim=64, gen_median=5, gen_cap=20)
    pool = quantised(b)
    out = sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, starts, shared)
    torch.cuda.synchronize()
    assert_parity(out, reference(b, pool), "4096 sequences in 2048 groups")


# ---- a decode loop of all of it -----------------------------------------------------------------------------------

def _loop_state(B, hq, hkv, d, seed, most=100):
    rng = np.random.default_rng(seed)
    N = B * (-(-most // 16)) + 3
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return dict(lens=torch.zeros(B, dtype=torch.int32, device=DEV), table=torch.zeros((B, -(-most // 16)), dtype=torch.int32, device=DEV),
                free=_t(rng.permutation(N)), count=_t([N]), pool=torch.full((N, hkv, 17 * d), 0xFF, dtype=torch.uint8, device=DEV),
                q=torch.randn((B, hq, d), generator=gen, device=DEV).bfloat16(), rng=rng, gen=gen, N=N)


def _rows(s, n, hkv, d):
    return torch.randn((n, hkv, d), generator=s["gen"], device=DEV).bfloat16()


@pytest.mark.parametrize("d", [64, 128])
def test_prompts_then_decode_steps_then_release(d):
    """Ragged prompts are given pages and written through the slot map (padded), decode steps append and attend,
    finished requests return their pages and others take them: after each step the cache's live rows are the rows that
    were written, and attention is the oracle's on them."""
    B, hq, hkv = 13, 8, 2
    s = _loop_state(B, hq, hkv, d, seed=d)
    history = [[] for _ in range(B)]
    for step in range(12):
        rng = s["rng"]
        done = (rng.random(B) < 0.25).astype(np.int32) if step % 3 == 2 else np.zeros(B, np.int32)
        lens, count = sl.pages_release(_t(done), s["lens"], s["table"], s["free"], s["count"],
                                       seq_lens_out=s["lens"], free_count_out=s["count"])
        for b in np.flatnonzero(done):
            history[b] = []
        new = np.array([rng.integers(0, 40) if not history[b] else 1 for b in range(B)], np.int32)
        cap = int(new.sum()) + 5
        lens, start, slots, count = sl.pages_extend(s["lens"], _t(new), s["table"], s["free"], s["count"], cap,
                                                    seq_lens_out=s["lens"], free_count_out=s["count"])
        k, v = _rows(s, cap, hkv, d), _rows(s, cap, hkv, d)
        at = start.tolist()
        assert np.diff(at).tolist() == new.tolist()
        if (new == 1).all():
            sl.kv_append_fp4(k[:B].contiguous(), v[:B].contiguous(), s["table"], lens, s["pool"])
        else:
            sl.kv_write_fp4(k, v, slots, s["pool"])
        for b in range(B):
            history[b] += [(k[i], v[i]) for i in range(at[b], at[b + 1])]
        out = sl.decode_attn_fp4(s["q"], s["pool"], s["table"], lens, d ** -0.5)
        torch.cuda.synchronize()
        assert lens.tolist() == [len(h) for h in history]
        kp, vp = fp4.unpack(s["pool"].cpu().numpy())
        table = s["table"].cpu().numpy()
        for b in (0, B // 2, B - 1):
            for i, (kr, vr) in enumerate(history[b]):
                for pages, row in ((kp, kr), (vp, vr)):
                    want = fp4.values(*fp4.quantise(bits(row)))
                    assert np.array_equal(pages[table[b, i // 16], :, i % 16], want)
        ref = _attend(s, kp, vp, d)
        assert_parity(out, ref, f"step {step}")
    held = sum(-(-len(h) // 16) for h in history)
    assert s["count"].item() + held == s["N"]


def _attend(s, kp, vp, d):
    import oracle
    k, v = (fp4.f64_to_bf16(x) for x in (kp, vp))
    return oracle.decode_attn(bits(s["q"]), k, v, s["table"].cpu().numpy(), s["lens"].cpu().numpy(), float(np.float32(d ** -0.5)))


def test_captured_decode_step_replays():
    """A step captured once (pages, append, attention; lengths and count updated in place) and replayed over a page
    boundary, with the eager step on a copy of the state between the replays."""
    B, hq, hkv, d = 9, 8, 2, 128
    s = _loop_state(B, hq, hkv, d, seed=5)
    one = torch.ones(B, dtype=torch.int32, device=DEV)
    k, v = _rows(s, B, hkv, d), _rows(s, B, hkv, d)
    start, slots = torch.zeros(B + 1, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    out = torch.empty_like(s["q"])
    names = ("lens", "table", "free", "count", "pool")

    def step(x, k, v, start, slots, out):
        sl.pages_extend(x["lens"], one, x["table"], x["free"], x["count"], B, seq_lens_out=x["lens"],
                        free_count_out=x["count"], token_start=start, slots=slots)
        sl.kv_append_fp4(k, v, x["table"], x["lens"], x["pool"])
        sl.decode_attn_fp4(x["q"], x["pool"], x["table"], x["lens"], d ** -0.5, out=out)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(s, k, v, start, slots, out)       # (the first call makes the stream's workspace)
    stream.synchronize()
    eager = dict(s, **{n: s[n].clone() for n in names})
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        step(s, k, v, start, slots, out)
    for i in range(20):
        k.copy_(_rows(s, B, hkv, d))
        v.copy_(_rows(s, B, hkv, d))
        g.replay()
        torch.cuda.synchronize()
        e_start, e_slots, e_out = torch.empty_like(start), torch.empty_like(slots), torch.empty_like(out)
        step(eager, k, v, e_start, e_slots, e_out)
        torch.cuda.synchronize()
        for n in names:
            assert torch.equal(s[n], eager[n]), (i, n)
        assert torch.equal(out, e_out) and torch.equal(slots, e_slots) and torch.equal(start, e_start), i
    assert s["lens"].tolist() == [21] * B


def test_calls_on_two_streams():
    """Each stream has its own workspace; every call equals the same call alone."""
    states = [make(np.random.default_rng(i).integers(1, 900, 20), 28, 4, 128, seed=i) for i in range(2)]
    alone = [sl.decode_attn_fp4(b.q, p, b.block_table, b.seq_lens, b.scale) for b, p in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    got = []
    for _ in range(10):
        for (b, p), st in zip(states, streams):
            with torch.cuda.stream(st):
                got.append(sl.decode_attn_fp4(b.q, p, b.block_table, b.seq_lens, b.scale))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert torch.equal(out, alone[i % 2]), i


def test_python_refusals():
    b, pool = make([5, 9], 8, 2, 64, seed=1)
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device=DEV)
    slots = torch.zeros(2, dtype=torch.int32, device=DEV)
    with pytest.raises(TypeError):
        sl.decode_attn_fp4(b.q.float(), pool, b.block_table, b.seq_lens, b.scale)
    with pytest.raises(TypeError):
        sl.decode_attn_fp4(b.q, pool.short(), b.block_table, b.seq_lens, b.scale)
    with pytest.raises(ValueError):
        sl.decode_attn_fp4(b.q, pool[:, :, :-1].contiguous(), b.block_table, b.seq_lens, b.scale)
    with pytest.raises(ValueError):
        sl.decode_attn_fp4(b.q, pool, b.block_table[:1], b.seq_lens, b.scale)
    with pytest.raises(ValueError):
        sl.decode_attn_fp4(b.q, pool.cpu(), b.block_table, b.seq_lens, b.scale)
    with pytest.raises(ValueError):
        sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, out=b.q[:1])
    with pytest.raises(sl.SlError):   # 7 query heads over 2 KV heads
        sl.decode_attn_fp4(b.q[:, :7].contiguous(), pool, b.block_table, b.seq_lens, b.scale)
    with pytest.raises(ValueError):
        sl.kv_write_fp4(k, k[:1], slots, pool)
    with pytest.raises(ValueError):
        sl.kv_write_fp4(k.transpose(0, 1), k, slots, pool)
    with pytest.raises(TypeError):
        sl.kv_write_fp4(k, k, slots.long(), pool)
    with pytest.raises(ValueError):
        sl.kv_append_fp4(k[:, :1].contiguous(), k[:, :1].contiguous(), b.block_table, b.seq_lens, pool)
    with pytest.raises(ValueError):
        sl.kv_read_fp4(slots, pool, k_out=k[:1])
    with pytest.raises(ValueError):
        sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, slots, slots)
