"""The operators of a paged 4-bit KV cache as timed cases: attention over it, the same with prefix sharing, the rows
that are written into it and read back, and the block tables and slot maps that say where they go.

``own`` selects the framework's kernels; where it is false the same state goes through the operators' plain form,
elementary torch operations in 32 bits. ``exact`` computes the outputs from the definitions in 64 bits.

The cache. A pool is ``uint8 [num_pages, Hkv, 17 D]``: one record per page of 16 tokens and KV head, holding for its key
rows and its value rows E2M1 codes (4 bits each) and one E8M0 scale byte per 32 consecutive elements of a row. With
t the token's slot in the page, d the element, C = D / 32 and E = D / 16, the record's bytes are
  K code (t, d)   nibble d % 2 (0: low) of byte 256 (d / 32) + 16 t + (d % 32) / 2
  V code (t, d)   nibble d % 2 of byte 8 D + 2 E (16 (t / 4) + d / E) + (E / 2) (t % 4) + (d % E) / 2
  K scale (t, c)  byte 16 D + 16 c + t
  V scale (t, c)  byte 16 D + D / 2 + 4 (C (t / 4) + c) + t % 4
and a cached value is e2m1(code) * 2^(scale - 127), NaN where the scale is 255. A row block is stored with the smallest
power of two under which its largest magnitude rounds to at most 6 (scale between 1 and 252), nearest, ties to even.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda:0"


# ---- the cases ----------------------------------------------------------------------------------------------------

def _attn(name, batch, hq, hkv, d, law, a, b, cap):
    return dict(name=name, kind="attn", batch=batch, hq=hq, hkv=hkv, d=d, law=law, a=a, b=b, cap=cap)


def listed():
    return [
        # The smallest decode step in use: a test-sized model, a handful of short contexts. Latency.
        _attn("attn4_tiny", 8, 4, 2, 64, "uniform", 1, 256, 0),
        # The end of a generation: a few long samples are left of a 7B-like batch.
        _attn("attn4_tail", 5, 28, 4, 128, "uniform", 2048, 16384, 0),
        # The rollout batch of a 7B-like model, as large as a smaller cache lets it be: long-tailed contexts.
        _attn("attn4_7b", 512, 28, 4, 128, "lognormal", 512, 2048, 32768),
        # The same for a 72B-like model: the largest step.
        _attn("attn4_72b", 256, 64, 8, 128, "lognormal", 1024, 4096, 32768),
        # head_dim 64, a large batch of short and medium contexts, odd lengths.
        _attn("attn4_d64", 384, 32, 8, 64, "uniform", 1, 2048, 0),
        # Several samples per prompt share the prompt's pages (GRPO).
        dict(name="prefix4_grpo", kind="prefix", prompts=32, samples=8, prompt=1024, median=512, cap=4096, hq=28, hkv=4,
             d=128),
        # A few prompts of odd length with many samples each that have hardly begun, head_dim 64, one head per KV head.
        dict(name="prefix4_start", kind="prefix", prompts=3, samples=22, prompt=1000, median=23, cap=64, hq=12, hkv=12,
             d=64),
        # A decode step's new rows quantised into their pages, and read back.
        dict(name="append4_step", kind="append", batch=96, hkv=4, hq=28, d=128, law="uniform", a=1, b=2048, cap=0),
        # A prefill chunk of many prompts: ragged runs of rows to the slots of a slot map, and back (a dense prefill
        # kernel reads the earlier chunks).
        dict(name="write4_prefill", kind="write", batch=24, hkv=8, hq=64, d=128, law="uniform", a=1, b=1365, cap=0),
        # Page bookkeeping of a decode step: one token for every sample of a large batch.
        dict(name="pages_step", kind="pages", batch=256, law="lognormal", a=512, b=2048, cap=16384, new=1, done=0),
        # Page bookkeeping of admission: samples that finished give their pages back, long prompts take theirs.
        dict(name="pages_admit", kind="pages", batch=96, law="uniform", a=1, b=8192, cap=0, new=1365, done=24),
        # A layer's decode step from the page bookkeeping on: pages and slots, the new rows, attention.
        dict(name="step4", kind="step", batch=96, hq=28, hkv=4, d=128, law="uniform", a=64, b=2048, cap=0),
    ]


_HEADS = [(4, 2, 64), (32, 8, 64), (12, 12, 64), (28, 4, 128), (64, 8, 128), (32, 8, 128), (40, 8, 128), (16, 1, 128)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "prefix", "append", "write", "pages", "step"])
    hq, hkv, d = rng.choice(_HEADS)
    if kind in ("attn", "step", "append"):
        batch = _log(rng, 1, 512)
        # the longest context: what keeps the cache within 1 GB, at most 32K
        top = _log(rng, 64, max(65, min(32768, int(1e9 / (batch * hkv * d * 17 / 16)))))
        law = rng.choice(["uniform", "lognormal"])
        a, b, cap = (rng.randint(1, top), top, 0) if law == "uniform" else (rng.randint(1, max(1, top // 8)), max(2, top // 8), top)
        return dict(kind=kind, batch=batch, hq=hq, hkv=hkv, d=d, law=law, a=a, b=b, cap=cap)
    if kind == "prefix":
        samples = rng.randint(2, 24)
        return dict(kind="prefix", prompts=_log(rng, 1, 512 // samples), samples=samples, prompt=_log(rng, 33, 4000),
                    median=_log(rng, 16, 1024), cap=4096, hq=hq, hkv=hkv, d=d)
    if kind == "write":
        batch = _log(rng, 1, 64)
        top = _log(rng, 1, max(2, 32768 // batch))
        return dict(kind="write", batch=batch, hq=hq, hkv=hkv, d=d, law="uniform", a=rng.randint(1, top), b=top, cap=0)
    batch = _log(rng, 1, 1024)
    new = rng.choice([1, 1, _log(rng, 1, max(2, 65536 // batch))])
    return dict(kind="pages", batch=batch, law="uniform", a=1, b=_log(rng, 2, 8192), cap=0, new=new,
                done=rng.randint(0, batch // 3))


def _lengths(case):
    """The sequence lengths: part of the case (the same for every seed, so that passes on other inputs do the same
    work), drawn from a generator seeded by the case's own sizes."""
    if case["kind"] == "prefix":
        rng = np.random.default_rng([case["prompts"], case["samples"], case["prompt"]])
        n = case["prompts"] * case["samples"]
        gen = np.clip(np.floor(rng.lognormal(math.log(case["median"]), 1.0, n)), 1, case["cap"]).astype(np.int64)
        return case["prompt"] + gen
    rng = np.random.default_rng([case["batch"], case["a"], case["b"], case.get("hq", 1)])
    if case["law"] == "uniform":
        return rng.integers(case["a"], case["b"] + 1, case["batch"]).astype(np.int64)
    x = np.clip(np.floor(rng.lognormal(math.log(case["b"]), 1.2 if case.get("hq") == 64 else 1.0, case["batch"])), 1, case["cap"])
    return case["a"] + x.astype(np.int64)


def _new_tokens(case):
    """Tokens that each request of a pages case adds (0: the request waits), and which requests have finished."""
    rng = np.random.default_rng([case["batch"], case["new"], case["done"], 7])
    done = np.zeros(case["batch"], np.int64)
    done[rng.permutation(case["batch"])[:case["done"]]] = 1
    new = np.ones(case["batch"], np.int64) if case["new"] == 1 else rng.integers(0, case["new"] + 1, case["batch"])
    return new, done


# ---- inputs -------------------------------------------------------------------------------------------------------

def _normal(shape, gen):
    """Standard normal values rounded to bf16, made in pieces of bounded size."""
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=gen, device=DEV)
    return out


def _pool(num_pages, hkv, d, gen):
    """A cache of quantised standard normal rows."""
    pool = torch.empty((num_pages, hkv, 17 * d), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // (hkv * PAGE * d))
    for i in range(0, num_pages, step):
        n = min(step, num_pages - i)
        _pack(_normal((n, hkv, PAGE, d), gen), _normal((n, hkv, PAGE, d), gen), pool[i:i + n])
    return pool


def _table(lens, rng, shared=0, per=1, spare=0):
    """Block table whose pages are scattered over the pool, as after many samples came and went; its pool size."""
    blocks = -(-lens // PAGE)
    own_blocks = blocks - shared
    groups = len(lens) // per
    total = groups * shared + int(own_blocks.sum())
    perm = rng.permutation(total + spare).astype(np.int32)
    table = np.zeros((len(lens), max(1, int(blocks.max()))), dtype=np.int32)
    at = 0
    for k in range(groups):
        common = perm[at:at + shared]
        at += shared
        for b in range(k * per, (k + 1) * per):
            table[b, :shared] = common
            table[b, shared:blocks[b]] = perm[at:at + own_blocks[b]]
            at += own_blocks[b]
    return table, perm[at:], total + spare


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, lens = case["kind"], _lengths(case)
    s = dict(case=case)
    if kind == "pages":
        lens, (new, done) = rng.permutation(lens), _new_tokens(case)
        blocks = -(-int(lens.max() + new.max()) // PAGE)
        table, spare, total = _table(lens, rng, spare=int((new // PAGE + 2).sum()))
        wide = np.zeros((len(lens), blocks), dtype=np.int32)
        wide[:, :table.shape[1]] = table
        free = np.zeros(total, dtype=np.int32)
        free[:len(spare)] = spare
        # the slot map holds what the step may bring at most
        s.update(lens=_dev(lens), new=_dev(new), done=_dev(done), table=_dev(wide), free=_dev(free),
                 count=_dev([len(spare)]), max_tokens=int(new.sum()) + 64)
        return s
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    shared, per = (case["prompt"] // PAGE, case["samples"]) if kind == "prefix" else (0, 1)
    # A step's samples are one token shorter before it; the pages that they open come from the free ones.
    before = lens - 1 if kind == "step" else lens
    table, spare, total = _table(before, rng, shared, per, spare=len(lens) if kind == "step" else 0)
    s.update(scale=1.0 / math.sqrt(d), host_lens=lens.tolist(), lens=_dev(lens))
    if kind in ("attn", "prefix", "step"):
        s["q"] = _normal((len(lens), hq, d), gen)
    if kind == "step":
        wide = np.zeros((len(lens), int((-(-lens // PAGE)).max())), dtype=np.int32)
        wide[:, :table.shape[1]] = table
        table, free = wide, np.zeros(total, dtype=np.int32)
        free[:len(spare)] = spare
        s.update(lens=_dev(before), new=_dev(np.ones(len(lens))), free=_dev(free), count=_dev([len(spare)]))
    s["table"] = _dev(table)
    s["pool"] = _pool(total, hkv, d, gen)
    if kind == "prefix":
        s["starts"] = _dev(np.arange(0, len(lens) + 1, per))
        s["shared"] = _dev(np.full(len(lens) // per, shared))
    rows = int(lens.sum()) if kind == "write" else len(lens)
    if kind in ("append", "write", "step"):
        s["k_new"], s["v_new"] = _normal((rows, hkv, d), gen), _normal((rows, hkv, d), gen)
    if kind == "write":
        pos = [np.arange(n) for n in lens]
        s["slots"] = _dev(np.concatenate([table[b, p // PAGE] * PAGE + p % PAGE for b, p in enumerate(pos)]))
    if kind == "append":
        t = lens - 1
        s["slots"] = _dev(table[np.arange(len(lens)), t // PAGE] * PAGE + t % PAGE)
    return s


# ---- the plain form -----------------------------------------------------------------------------------------------

_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _quantise(x):
    """Rows [..., D] (bf16) -> codes [..., D] and scale bytes [..., D / 32], both int32."""
    blocks = x.unflatten(-1, (-1, 32))
    top = (blocks.contiguous().view(torch.int16).int() & 0x7FFF).amax(-1)
    scale = (((top + 0x20) >> 7) - 2).clamp(1, 252)
    y = torch.ldexp(blocks.float(), (127 - scale)[..., None])
    a = y.abs()
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int()
            + (a >= 3.5).int() + (a > 5.0).int()) + 8 * (y < 0).int()
    odd = top >= 0x7F80
    return torch.where(odd[..., None], 0, code).flatten(-2), torch.where(odd, 255, scale)


def _bytes(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8)


def _pack(k, v, pool):
    """Whole pages of rows [n, Hkv, 16, D] into records [n, Hkv, 17 D]."""
    n, h, _, d = k.shape
    c, e = d // 32, d // 16
    code, scale = _quantise(k)
    pool[..., :8 * d] = _bytes(code).view(n, h, PAGE, c, 16).transpose(2, 3).flatten(2)
    pool[..., 16 * d:16 * d + d // 2] = scale.to(torch.uint8).transpose(2, 3).flatten(2)
    code, scale = _quantise(v)
    pool[..., 8 * d:16 * d] = _bytes(code).view(n, h, 4, 4, 16, e // 2).transpose(3, 4).flatten(2)
    pool[..., 16 * d + d // 2:] = scale.to(torch.uint8).view(n, h, 4, 4, c).transpose(3, 4).flatten(2)


def _values(code_bytes, scale_bytes):
    """Codes [..., D / 2] in bytes and scales [..., D / 32] -> values [..., D], 32 bits."""
    pairs = torch.tensor([[_E2M1[n & 7] * (-1.0 if n & 8 else 1.0) for n in (b & 15, b >> 4)] for b in range(256)],
                         dtype=torch.float32, device=code_bytes.device)
    x = pairs[code_bytes.int()].flatten(-2)
    power = torch.where(scale_bytes == 255, math.nan, (scale_bytes.int() << 23).view(torch.float32))
    return (x.unflatten(-1, (-1, 32)) * power[..., None]).flatten(-2)


def _unpack(rec):
    """Records [n, Hkv, 17 D] -> the key and value rows [Hkv, 16 n, D], 32 bits."""
    n, h, size = rec.shape
    d = size // 17
    c, e = d // 32, d // 16
    k = _values(rec[..., :8 * d].view(n, h, c, PAGE, 16).transpose(2, 3).flatten(3),
                rec[..., 16 * d:16 * d + d // 2].view(n, h, c, PAGE).transpose(2, 3))
    v = _values(rec[..., 8 * d:16 * d].view(n, h, 4, 16, 4, e // 2).transpose(3, 4).reshape(n, h, PAGE, d // 2),
                rec[..., 16 * d + d // 2:].view(n, h, 4, c, 4).transpose(3, 4).reshape(n, h, PAGE, c))
    return k.transpose(0, 1).flatten(1, 2), v.transpose(0, 1).flatten(1, 2)


def _plain_attention(s, lens):
    case, q, table, pool = s["case"], s["q"], s["table"], s["pool"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    out = torch.empty_like(q)
    for b, n in enumerate(lens):
        k, v = _unpack(pool[table[b, :-(-n // PAGE)]])
        w = torch.matmul(q[b].float().view(hkv, hq // hkv, d), k[:, :n].transpose(1, 2).contiguous()) * s["scale"]
        w = torch.exp(w - w.amax(-1, keepdim=True))
        out[b] = (torch.matmul(w, v[:, :n].contiguous()) / w.sum(-1, keepdim=True)).view(hq, d)
    return out


def _row_bytes(slots, pool, d):
    """Byte indexes in the flat pool of rows at slots [T]: K codes, V codes [T, Hkv, D / 2], K and V scales [T, Hkv, C]."""
    hkv, c, e = pool.shape[1], d // 32, d // 16
    slots = slots.long()
    base = ((slots // PAGE)[:, None] * hkv + torch.arange(hkv, device=DEV))[..., None] * (17 * d)
    t = (slots % PAGE)[:, None, None]
    at, ch = 2 * torch.arange(d // 2, device=DEV), torch.arange(c, device=DEV)
    return (base + 256 * (at // 32) + 16 * t + (at % 32) // 2,
            base + 8 * d + 2 * e * (16 * (t // 4) + at // e) + (e // 2) * (t % 4) + (at % e) // 2,
            base + 16 * d + 16 * ch + t, base + 16 * d + d // 2 + 4 * (c * (t // 4) + ch) + t % 4)


def _plain_write(k_new, v_new, slots, pool):
    kc, vc, ks, vs = _row_bytes(slots, pool, k_new.shape[2])
    flat = pool.view(-1)
    for x, codes, scales in ((k_new, kc, ks), (v_new, vc, vs)):
        code, scale = _quantise(x)
        flat[codes] = _bytes(code)
        flat[scales] = scale.to(torch.uint8)


def _plain_read(slots, pool, d):
    kc, vc, ks, vs = _row_bytes(slots, pool, d)
    flat = pool.view(-1)
    return (_values(flat[kc], flat[ks]).to(torch.bfloat16), _values(flat[vc], flat[vs]).to(torch.bfloat16))


def _plain_release(s):
    """Finished requests' pages go back on the stack, last block first, request by request; their lengths become 0."""
    lens, table, free, count = s["lens"], s["table"], s["free"], s["count"]
    nb = torch.where(s["done"] != 0, (lens + PAGE - 1) // PAGE, 0)
    upto = torch.cumsum(nb, 0)
    blk = torch.arange(table.shape[1], device=DEV)
    at = count.long() + (upto[:, None] - 1 - blk)
    mask = blk < nb[:, None]
    free[at[mask]] = table[mask]
    return torch.where(s["done"] != 0, 0, lens), (count + upto[-1]).int()


def _plain_extend(lens, new, table, free, count, max_tokens):
    """Pages for each request's new tokens from the top of the stack, and the tokens' slots in request order."""
    most = table.shape[1] * PAGE
    valid = (lens >= 0) & (new >= 0) & (lens.long() + new <= most)
    had = (lens + PAGE - 1) // PAGE
    need = torch.where(valid, (lens + new + PAGE - 1) // PAGE - had, 0)
    upto = torch.cumsum(need, 0)
    served = valid & ((need == 0) | (upto <= count)) & (torch.cumsum(torch.where(valid, new, 0), 0) <= max_tokens)
    got, need = torch.where(served, new, 0), torch.where(served, need, 0)
    upto = torch.cumsum(need, 0)
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), torch.cumsum(got, 0)])
    blk = torch.arange(table.shape[1], device=DEV)
    place = upto[:, None] - need[:, None] + (blk - had[:, None])
    opened = (blk >= had[:, None]) & (blk < (had + need)[:, None])
    table.copy_(torch.where(opened, free[(count - 1 - place).clamp(0, free.numel() - 1)], table))
    i = torch.arange(max_tokens, device=DEV)
    b = torch.searchsorted(start[1:], i, right=True).clamp(max=len(lens) - 1)
    pos = lens[b] + (i - start[b])
    slot = table[b, (pos // PAGE).clamp(max=table.shape[1] - 1)] * PAGE + pos % PAGE
    return (lens + got).int(), start.int(), torch.where(i < start[-1], slot, -1).int(), (count - upto[-1]).int()


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2504_15930_amd import sl
    kind = s["case"]["kind"]
    if kind == "attn":
        return sl.decode_attn_fp4(s["q"], s["pool"], s["table"], s["lens"], s["scale"])
    if kind == "prefix":
        return sl.decode_attn_prefix_fp4(s["q"], s["pool"], s["table"], s["lens"], s["scale"], s["starts"], s["shared"])
    if kind == "append":
        sl.kv_append_fp4(s["k_new"], s["v_new"], s["table"], s["lens"], s["pool"])
        return sl.kv_read_fp4(s["slots"], s["pool"])
    if kind == "write":
        sl.kv_write_fp4(s["k_new"], s["v_new"], s["slots"], s["pool"])
        return sl.kv_read_fp4(s["slots"], s["pool"])
    if kind == "pages":
        lens, count = s["lens"], s["count"]
        if s["case"]["done"]:
            lens, count = sl.pages_release(s["done"], lens, s["table"], s["free"], count)
        lens, start, slots, count = sl.pages_extend(lens, s["new"], s["table"], s["free"], count, s["max_tokens"])
        return dict(lens=lens, start=start, slots=slots, count=count, table=s["table"], free=s["free"])
    lens, start, slots, count = sl.pages_extend(s["lens"], s["new"], s["table"], s["free"], s["count"],
                                                s["new"].numel())
    sl.kv_append_fp4(s["k_new"], s["v_new"], s["table"], lens, s["pool"])
    out = sl.decode_attn_fp4(s["q"], s["pool"], s["table"], lens, s["scale"])
    k, v = sl.kv_read_fp4(slots, s["pool"])
    return dict(out=out, lens=lens, start=start, slots=slots, count=count, table=s["table"], k=k, v=v)


def _run_plain(s):
    kind, d = s["case"]["kind"], s["case"].get("d")
    if kind in ("attn", "prefix"):
        return _plain_attention(s, s["host_lens"])
    if kind in ("append", "write"):
        _plain_write(s["k_new"], s["v_new"], s["slots"], s["pool"])
        return _plain_read(s["slots"], s["pool"], d)
    if kind == "pages":
        lens, count = s["lens"], s["count"]
        if s["case"]["done"]:
            lens, count = _plain_release(s)
        lens, start, slots, count = _plain_extend(lens, s["new"], s["table"], s["free"], count, s["max_tokens"])
        return dict(lens=lens, start=start, slots=slots, count=count, table=s["table"], free=s["free"])
    lens, start, slots, count = _plain_extend(s["lens"], s["new"], s["table"], s["free"], s["count"], s["new"].numel())
    _plain_write(s["k_new"], s["v_new"], slots, s["pool"])
    out = _plain_attention(s, s["host_lens"])
    k, v = _plain_read(slots, s["pool"], d)
    return dict(out=out, lens=lens, start=start, slots=slots, count=count, table=s["table"], k=k, v=v)


def work(case):
    kind, lens = case["kind"], _lengths(case)
    if kind == "pages":
        new, done = _new_tokens(case)
        back = int((-(-lens // PAGE) * done).sum())
        left = np.where(done == 1, 0, lens)
        opened = int((-(-(left + new) // PAGE) - -(-left // PAGE)).sum())
        # lengths, counts and marks in, lengths and starts out; pages once from and once to table or stack; slots out
        return dict(bytes=4 * (5 * len(lens) + 2 * (back + opened) + int(new.sum())), flops=0)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    packed = 2 * (d // 2 + d // 32)   # a token's key and value row of one KV head in the cache
    if kind in ("append", "write"):
        rows = int(lens.sum()) if kind == "write" else len(lens)
        # rows in, packed rows out; packed rows in, rows out
        return dict(bytes=2 * rows * (hkv * (4 * d + packed) + 4), flops=0)
    tokens, blocks = int(lens.sum()), int((-(-lens // PAGE)).sum())
    flops = 4 * tokens * hq * d
    if kind == "prefix":
        shared = case["prompt"] // PAGE
        again = shared * (len(lens) - case["prompts"])
        tokens, blocks = tokens - PAGE * again, blocks - again
    got = tokens * hkv * packed + 4 * blocks + len(lens) * (hq * d * 4 + 4)
    if kind == "step":
        got += 2 * len(lens) * hkv * (4 * d + packed) + 28 * len(lens)
    return dict(bytes=got, flops=flops)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def _layout(d):
    """For each (t, element): byte and shift of its K and V code and byte of its K and V scale in a record."""
    t, x = np.meshgrid(np.arange(PAGE), np.arange(d), indexing="ij")
    c, e = d // 32, d // 16
    at = [256 * (x // 32) + 16 * t + x % 32 // 2, 8 * d + 2 * e * (16 * (t // 4) + x // e) + e // 2 * (t % 4) + x % e // 2,
          16 * d + 16 * (x // 32) + t, 16 * d + d // 2 + 4 * (c * (t // 4) + x // 32) + t % 4]
    return [torch.from_numpy(a).to(DEV) for a in at], torch.from_numpy(4 * (x % 2)).to(DEV)


def _decode64(rec):
    """Records [n, Hkv, 17 D] -> key and value rows [n, Hkv, 16, D] in 64 bits."""
    d = rec.shape[2] // 17
    (kc, vc, ks, vs), shift = _layout(d)
    table = torch.tensor(_E2M1 + [-x for x in _E2M1], dtype=torch.float64, device=DEV)
    scale = torch.tensor([2.0 ** (i - 127) for i in range(255)] + [math.nan], dtype=torch.float64, device=DEV)

    def rows(codes, scales):
        return table[((rec[:, :, codes].int() >> shift) & 15).long()] * scale[rec[:, :, scales].long()]

    return rows(kc, ks), rows(vc, vs)


def _stored64(x):
    """The values that rows [T, Hkv, D] keep in the cache, by search for the nearest code."""
    w = x.double().unflatten(-1, (-1, 32))
    top = w.abs().amax(-1)
    exponent = torch.frexp(top / 3.5)[1] - 1          # 3.5 * 2^e <= top < 7 * 2^e
    unit = torch.exp2(torch.where(top == 0, -126, exponent).clamp(-126, 125).double())[..., None]
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    a = (w / unit).abs()
    low = torch.searchsorted(grid, a, right=True).clamp(max=8) - 1
    high = (low + 1).clamp(max=7)
    up = (grid[high] - a < a - grid[low]) | ((grid[high] - a == a - grid[low]) & (low % 2 == 1))
    return (torch.where(up, grid[high], grid[low]) * unit * torch.sign(w)).flatten(-2)


def _attention64(s, lens, new=None):
    case, hq, hkv, d = s["case"], s["case"]["hq"], s["case"]["hkv"], s["case"]["d"]
    out = torch.empty((len(lens), hq, d), dtype=torch.float64, device=DEV)
    scale = float(np.float32(s["scale"]))
    for b, n in enumerate(lens):
        # the last token of a step is not in the cache yet
        m = n - 1 if new is not None else n
        k, v = _decode64(s["pool"][s["table"][b, :-(-m // PAGE)].long()])
        k, v = (x.permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :m] for x in (k, v))
        if new is not None:
            k, v = torch.cat([k, new[0][b][:, None]], 1), torch.cat([v, new[1][b][:, None]], 1)
        q = s["q"][b].double().view(hkv, hq // hkv, d)
        w = torch.softmax(torch.matmul(q, k.transpose(1, 2).contiguous()) * scale, dim=2)
        out[b] = torch.matmul(w, v.contiguous()).view(hq, d)
    return out


def _pages(lens, new, done, table, free, count, max_tokens):
    """The page bookkeeping request by request, on the host."""
    lens, table, free = lens.copy(), table.copy(), free.copy()
    for b in np.flatnonzero(done):
        for j in reversed(range(-(-lens[b] // PAGE))):
            free[count] = table[b, j]
            count += 1
        lens[b] = 0
    start, slots = [0], []
    for b, n in enumerate(new):
        opened = -(-(lens[b] + n) // PAGE) - -(-lens[b] // PAGE)
        if opened > count or len(slots) + n > max_tokens:
            raise ValueError("the cases have pages and slots for every request")
        for j in range(opened):
            count -= 1
            table[b, -(-lens[b] // PAGE) + j] = free[count]
        slots += [int(table[b, p // PAGE]) * PAGE + p % PAGE for p in range(lens[b], lens[b] + n)]
        lens[b] += n
        start.append(len(slots))
    slots += [-1] * (max_tokens - len(slots))
    return lens, start, slots, [count], table, free


def exact(case, seed):
    kind, s = case["kind"], prepare(case, seed)
    if kind in ("attn", "prefix"):
        return _attention64(s, s["host_lens"])
    if kind in ("append", "write"):
        return _stored64(s["k_new"]), _stored64(s["v_new"])
    lens, table, free = (s[x].cpu().numpy().astype(np.int64) for x in ("lens", "table", "free"))
    new = s["new"].cpu().numpy()
    done = s["done"].cpu().numpy() if kind == "pages" else np.zeros(len(new), np.int64)
    got = dict(zip(("lens", "start", "slots", "count", "table", "free"),
                   map(_dev, _pages(lens, new, done, table, free, int(s["count"].item()),
                                    s["max_tokens"] if kind == "pages" else len(new)))))
    if kind == "step":
        del got["free"]
        k, v = _stored64(s["k_new"]), _stored64(s["v_new"])
        got = dict(out=_attention64(s, s["host_lens"], (k, v)), **got, k=k, v=v)
    return got
