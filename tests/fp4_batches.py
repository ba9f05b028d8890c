"""4-bit decode batches for the GPU tests, and the oracle on them."""
from __future__ import annotations

import numpy as np
import torch

import oracle
from oracle import fp4
from paper_2504_15930_amd import inputs, sl

DEV = "cuda:0"


def bits(t):
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def quantised(batch):
    """The batch's live rows in a 4-bit pool, every other byte 0xFF (NaN scales), by kv_write_fp4."""
    N, Hkv, P, D = batch.k_pages.shape
    pool = torch.full((N, Hkv, sl.fp4_record_bytes(D)), 0xFF, dtype=torch.uint8, device=batch.k_pages.device)
    k, v = (x.transpose(1, 2).reshape(N * P, Hkv, D) for x in (batch.k_pages, batch.v_pages))
    live = torch.nonzero(~torch.isnan(k[:, 0, 0]))[:, 0]
    if live.numel():
        sl.kv_write_fp4(k[live].contiguous(), v[live].contiguous(), live.int(), pool)
    return pool


def make(lengths, hq, hkv, d, seed=0, **kw):
    b = inputs.make_paged_batch(lengths, hq, hkv, d, seed=seed, device=DEV, **kw)
    return b, quantised(b)


def reference(b, pool, rows=None):
    """The fp64 oracle on the pool's values, which bf16 pages hold exactly."""
    table, lens, q, host = b.block_table.cpu().numpy(), b.seq_lens.cpu().numpy(), b.q, pool
    if rows is not None:   # only the pages of these sequences
        rows = list(rows)
        table, lens, q = table[rows].copy(), lens[rows], b.q[rows]
        nb = -(-np.maximum(lens, 0) // 16)
        used = np.unique(np.concatenate([table[i, :nb[i]] for i in range(len(rows))] + [np.zeros(1, np.int32)]))
        at = np.zeros(pool.shape[0], np.int32)
        at[used] = np.arange(len(used))
        table = at[table]
        host = pool[torch.as_tensor(used.astype(np.int64), device=pool.device)]
    k, v = (fp4.f64_to_bf16(x) for x in fp4.unpack(host.cpu().numpy()))
    return oracle.decode_attn(bits(q), k, v, table, lens, b.scale)
