"""Attention over a 4-bit cache with large scores, up to far beyond what a model has: the softmax is that of scores rounded
to fp32, whatever their size (the kernels subtract the running maximum before the exponential)."""
import numpy as np
import pytest
import torch

from oracle import fp4
from paper_2504_15930_amd import inputs, sl
from fp4_batches import DEV, bits, quantised

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs an MI355X")]
LOG2E = 1.4426950408889634


def _winners(b, pool):
    """(rows, known): the value row of the token with the highest score, in 64 bits, and where that token is beyond doubt.

    A score is a sum of D <= 128 products in fp32, in any order: off by at most 127 * 2^-24 < 2^-17 of sum |q k|, and by
    2^-23 of itself (at most sum |q k|) by the two factors' rounding. Two such errors, 2^-15 of sum |q k| in all, and 64
    more in base-2 units (every other weight is below 2^-64): then the others are lost beside it."""
    k, v = fp4.unpack(pool.cpu().numpy())
    q = fp4.bf16_to_f64(bits(b.q))
    table, lens = b.block_table.cpu().numpy(), b.seq_lens.cpu().numpy()
    G = q.shape[1] // pool.shape[1]
    rows, known = np.zeros(q.shape), np.zeros(q.shape[:2], bool)
    for i, L in enumerate(lens):
        at = table[i, np.arange(L) // 16], slice(None), np.arange(L) % 16
        kk, vv = k[at], v[at]                       # [L, Hkv, D]
        for h in range(q.shape[1]):
            if L == 0:
                known[i, h] = True
                continue
            terms = kk[:, h // G] * q[i, h]
            s = b.scale * LOG2E * terms.sum(-1)
            spread = abs(b.scale) * LOG2E * np.abs(terms).sum(-1).max()
            order = np.argsort(s)
            rows[i, h] = vv[order[-1], h // G]
            known[i, h] = L == 1 or s[order[-1]] - s[order[-2]] > 64 + spread * 2.0 ** -15
    return rows, known


def _batch(D, G, power, sign, seed):
    """Normal queries and keys times 2^power each; values as they are."""
    b = inputs.make_paged_batch([1, 40, 0, 150, 17, 333, 64, 1000], 2 * G, 2, D, seed=seed, device=DEV)
    b.k_pages.mul_(2.0 ** power)
    b.q.mul_(2.0 ** power)
    b.scale = sign * 0.1
    return b, quantised(b)


# Scores of 2^(2 power + 2) and less; base-2 exponents from 2^22 on lose their last whole units, from 2^31 on 128.
@pytest.mark.parametrize("power", [9, 12, 14, 16, 18, 25, 40, 56])
@pytest.mark.parametrize("D,G", [(64, 4), (128, 7), (64, 16), (128, 16)])
def test_the_highest_score_takes_all(D, G, power):
    for sign in (1.0, -1.0):
        b, pool = _batch(D, G, power, sign, seed=D + G + power)
        want, known = _winners(b, pool)
        print("large scores", D, G, power, sign, "rows known", known.mean(), flush=True)
        assert known.mean() > 0.9
        for workers in (0, 1, 7, 60):
            out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, num_workers=workers)
            torch.cuda.synchronize()
            got = out.float().cpu().double().numpy()
            assert np.isfinite(got).all(), workers
            # (a value has two significant bits, so that a weight that cancels leaves it exact)
            assert np.array_equal(got[known], want[known]), workers
        # the same values in a bf16 cache
        kp, vp = (torch.from_numpy(fp4.f64_to_bf16(x).view(np.int16)).to(DEV).view(torch.bfloat16)
                  for x in fp4.unpack(pool.cpu().numpy()))
        out = sl.decode_attn(b.q, kp, vp, b.block_table, b.seq_lens, b.scale)
        torch.cuda.synchronize()
        assert np.array_equal(out.float().cpu().double().numpy()[known], want[known])


@pytest.mark.parametrize("power", [4, 12, 15, 16, 20, 40, 100])
@pytest.mark.parametrize("D", [64, 128])
def test_equal_large_scores_share_the_weight(D, power):
    """Keys of one code each: all tokens with the largest code have the same score, far above the others', and the output
    is the mean of their value rows."""
    rng = np.random.default_rng(power)
    B, Hkv, G = 6, 2, 4
    lens = [5, 16, 50, 130, 300, 700]
    b = inputs.make_paged_batch(lens, G * Hkv, Hkv, D, seed=power, device=DEV)
    top = rng.choice([1.0, 2.0, 3.0, 4.0, 6.0], size=(b.k_pages.shape[0], Hkv, 16, 1)) * 2.0 ** (power // 2)
    live = ~torch.isnan(b.k_pages)
    b.k_pages.copy_(torch.where(live, torch.from_numpy(top).to(DEV).expand(live.shape), float("nan")))
    # sixteen values of one magnitude and sign: their mean is that of few distinct numbers, each with a weight of 1
    b.v_pages.copy_(torch.where(live, torch.ones_like(b.v_pages), b.v_pages))
    b.q.fill_(2.0 ** (power - power // 2))
    pool = quantised(b)
    for scale in (0.3, 1.7):
        for workers in (0, 3, 40):
            out = sl.decode_attn_fp4(b.q, pool, b.block_table, b.seq_lens, scale, num_workers=workers)
            torch.cuda.synchronize()
            assert (out == 1).all(), (scale, workers)


def test_equal_large_scores_average_their_values():
    """Two tokens with the same key, the rest far below: the output is the mean of the two value rows, exactly."""
    D, Hkv, L = 64, 1, 90
    for power in (8, 15, 16, 18, 30):
        for i, j in ((0, 1), (3, 20), (15, 16), (0, 89), (40, 88)):
            k = torch.full((L, Hkv, D), -(2.0 ** power), device=DEV)
            k[[i, j]] = 2.0 ** power
            v = torch.full((L, Hkv, D), 4.0, device=DEV)
            v[i], v[j] = 1.0, 2.0
            pool = torch.full((6, Hkv, 17 * D), 0xFF, dtype=torch.uint8, device=DEV)
            sl.kv_write_fp4(k.bfloat16(), v.bfloat16(), torch.arange(L, dtype=torch.int32, device=DEV), pool)
            q = torch.full((1, 4, D), 2.0 ** power, device=DEV).bfloat16()
            table = torch.arange(6, dtype=torch.int32, device=DEV)[None]
            for workers in (0, 2):
                out = sl.decode_attn_fp4(q, pool, table, torch.tensor([L], dtype=torch.int32, device=DEV), 0.7,
                                         num_workers=workers)
                torch.cuda.synchronize()
                assert (out == 1.5).all(), (power, i, j, workers)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("workers", [0, 9])
def test_prefix_sharing_with_large_scores(D, workers):
    for power in (14, 16, 18, 40):
        b, starts, shared = inputs.make_grpo_batch(3, 5, 100, seed=power, device=DEV, num_q_heads=8, num_kv_heads=2,
                                                   head_dim=D, gen_median=40, gen_cap=200)
        b.k_pages.mul_(2.0 ** power)
        b.q.mul_(2.0 ** power)
        pool = quantised(b)
        want, known = _winners(b, pool)
        assert known.mean() > 0.9
        out = sl.decode_attn_prefix_fp4(b.q, pool, b.block_table, b.seq_lens, b.scale, starts, shared, num_workers=workers)
        torch.cuda.synchronize()
        got = out.float().cpu().double().numpy()
        assert np.isfinite(got).all() and np.array_equal(got[known], want[known]), power
