// Split-KV decode attention over a 4-bit cache (fp4_unit.h has its layout): the
// kernels of decode_split.hip and decode_shared.hip for FP4 records.
//
// Split-KV (split_fp4_kernel), with prefix sharing (prefix_fp4_kernel), and a
// workgroup per unit for short sequences (unit_fp4_kernel). A step of the streams
// is four tiles, with prefix sharing two (17 D bytes each, K and V).
//
// Measured (MI355X, cold pages), split and merge: 512 x 512 + lognormal(2048)
// tokens, 28/4 heads of 128, 1.07 GB of records in 173 us, 6.2 TB/s (reading such
// records at random without any arithmetic 6.7); 256 sequences of 64/8 heads, 2.26
// GB in 351 us, 6.4 TB/s: bound by HBM. With head_dim 64 a record is half as long
// for the same loads, scales and softmax: 64 x 1..8192, 32/8 heads, in 36.7 us; a
// workgroup per unit, 384 x 1..2048, 32/8 heads, 0.21 GB in 41.4 us, 5.0 TB/s, the
// VALUs busy for half of it.
#include "prefix_unit.h"

namespace sl {
namespace {

template <int D, int KV>
__global__ __launch_bounds__(kWave * kWavesPerBlock) void split_fp4_kernel(SplitParams p)
{
    extern __shared__ int32_t s_dyn[];
    int32_t *const s_cum = s_dyn;                // [B + 1]
    int32_t *const s_len = s_dyn + p.batch + 1;  // [B]
    scan_sequences<step_tiles<D, KV>()>(p, s_cum, s_len);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    split_unit_worker<D, KV, kAllPages>(p, wave * (int)gridDim.x + (int)blockIdx.x, StreamLds{s_cum, s_len});
}

// Shared-page workers per workgroup: 4, 2 or 1 for units of up to 16, 32 and 64
// query rows (members x heads of the largest sub-group with shared pages). With
// four wavefronts per worker whatever the rows, those of the empty blocks stream
// and compute for nothing: 8 prompts of 4000 tokens x 2 samples, 32/8 heads, D = 64
// 31.8 -> 20.0 us; 16 of 4000 x 24, 12/12 heads, D = 64 115 -> 48; 64 of 2000 x 4,
// 64/8 heads, D = 128 118 -> 74; with four blocks the same.
// (Every wavefront looks for itself: two votes of the workgroup took 1 us.)
__device__ __forceinline__ int shared_workers_per_block(const int32_t *s_sh, const int32_t *s_gl, int S, int group)
{
    int members = 0;
    for (int i = threadIdx.x & (kWave - 1); i < S; i += kWave)
        if (s_sh[i + 1] > s_sh[i])
            members = max(members, (s_gl[i] >> 16 & 15) + 1);
    const int rows = wave_reduce<ScanMax>(members) * group;
    return rows > 32 ? 1 : rows > 16 ? 2 : 4;
}

template <int D, int KV>
__global__ __launch_bounds__(kWave * kWavesPerBlock) void prefix_fp4_kernel(SplitParams own, SplitParams shared,
                                                                               PrefixParams pp, int own_blocks,
                                                                               int max_shared)
{
    extern __shared__ int32_t s_dyn[];
    const int B = own.batch, S = pp.max_sub;
    int32_t *const s_own = s_dyn;             // [B + 1]
    int32_t *const s_shared = s_own + B + 1;  // [B + 1]
    int32_t *const s_len = s_shared + B + 1;  // [B]
    int32_t *const s_sh = s_len + B;          // [S + 1]
    int32_t *const s_gl = s_sh + S + 1;       // [S]
    // The groups' starts and pages, read by the scan alone, in the state queues.
    static_assert(sizeof(int32_t) * (2 * kMaxPrefixBatch + 1) <= kWavesPerBlock * kOwnStageBytes, "the group arrays");
    int32_t *const s_gs = reinterpret_cast<int32_t *>(own_state_stage());   // [NG + 1]
    int32_t *const s_sp = s_gs + pp.num_groups + 1;                         // [NG]
    constexpr int NT = step_tiles<D, KV, true>();
    scan_prefix_groups<NT>(own, pp, s_own, s_len, s_shared, s_sh, s_gl, s_gs, s_sp);
    const int per_block = shared_workers_per_block(s_sh, s_gl, S, own.group);
    if (blockIdx.x == 0 && threadIdx.x == 0)
        pp.cum_shared[S + 1] = per_block;
    if ((int)blockIdx.x < own_blocks)
        split_unit_worker<D, KV, kOwnPages>(
            own, blockIdx.x * kWavesPerBlock + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave),
            StreamLds{s_own, s_len, s_shared});
    else {
        // The four wavefronts of a workgroup are one worker (four column blocks of
        // query rows), or two or four where the largest unit has two blocks or one.
        const int block = (int)blockIdx.x - own_blocks;
        const int blocks = effective_shared_workers_fp4((long long)s_own[B] * own.num_kv_heads,
                                                        (long long)s_sh[S] * own.num_kv_heads, per_block,
                                                        own.num_workers, shared.num_workers, max_shared, NT);
        if (block >= blocks)
            return;
        SplitParams sh = shared;
        sh.num_workers = shared_workers_of(blocks, per_block, own.num_workers);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = kPrefixBlocks / per_block;
        split_unit_worker<D, kFp4, kSharedPages>(sh, wave / waves * blocks + block,
                                                 StreamLds{s_sh, nullptr, nullptr, s_gl, S}, wave % waves);
    }
}

// The group that sequence b shares pages in, as scan_prefix_groups has it (in range
// and at or after the end of every earlier group's range): its first member, whose
// table entries stand for all members', and the pages, 0 where there is none. Every
// wavefront looks at all groups, one per lane and pass, the passes' loads together.
struct SharedIn {
    int lead, pages;
};
__device__ __forceinline__ SharedIn shared_in(const UnitGroups &g, const SplitParams &p, int b, int lane)
{
    constexpr int kPasses = kUnitGroups / kWave;
    int lo[kPasses], hi[kPasses], sp[kPasses];
    bool descends = false;
#pragma unroll
    for (int i = 0; i < kPasses; ++i)
        if (i * kWave < g.count) {
            const int k = min(i * kWave + lane, g.count - 1);
            lo[i] = g.start[k];
            hi[i] = g.start[k + 1];
            sp[i] = g.shared_pages[k];
        }
    SharedIn in = {b, 0};
    auto holds = [&](int i) { return lo[i] >= 0 && b >= lo[i] && b < hi[i] && hi[i] <= p.batch && sp[i] > 0 && sp[i] <= p.max_blocks; };
#pragma unroll
    for (int i = 0; i < kPasses; ++i)
        if (i * kWave < g.count)
            descends |= lo[i] > hi[i];
    const bool ascending = __builtin_amdgcn_ballot_w64(descends) == 0;
#pragma unroll
    for (int i = 0; i < kPasses; ++i)
        if (i * kWave < g.count) {
            bool here = holds(i);
            if (!ascending && here)
                for (int j = 0; j < min(i * kWave + lane, g.count - 1); ++j)
                    here &= g.start[j + 1] <= lo[i];
            if (const uint64_t mask = __builtin_amdgcn_ballot_w64(here)) {   // (groups with shared pages are disjoint)
                const int at = __builtin_ctzll(mask);
                in = {__builtin_amdgcn_readlane(lo[i], at), __builtin_amdgcn_readlane(sp[i], at)};
            }
        }
    return in;
}

// The sequence that is number `turn` when those of the longest quarter of the
// table's width come first, then the next quarter, and so on, in batch order
// within each; its length in L. Every wavefront votes on its 64 sequences of every
// pass over the batch, one mask per quarter; the masks lie in turn order, a lane of
// each wavefront has one, and a scan of their counts says which holds `turn`. Ends
// without a barrier (the arrays are its own).
template <int PASSES>
struct TurnLds {
    uint64_t mask[4][PASSES][kWavesPerBlock];
    int32_t len[PASSES * kWavesPerBlock * kWave];
};
struct TurnSum {
    static constexpr int kIdentity = 0;
    __device__ static int op(int a, int b) { return a + b; }
};
template <int PASSES>
__device__ __forceinline__ int sequence_in_turn(TurnLds<PASSES> &s, const SplitParams &p, int turn, int wave, int lane,
                                                int &L)
{
    constexpr int kMasks = 4 * PASSES * kWavesPerBlock;
    static_assert(kMasks <= kWave, "a mask per lane");
    constexpr int kThreads = kWavesPerBlock * kWave;
    int len[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i)
        if (i * kThreads < p.batch)
            len[i] = p.seq_lens[min(i * kThreads + (int)threadIdx.x, p.batch - 1)];
    const int width = p.max_blocks * (kPageSize / 4);   // a quarter of the table, in tokens
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        if (i * kThreads >= p.batch) {
            if (lane < 4)
                s.mask[lane][i][wave] = 0;
            continue;
        }
        const int b = i * kThreads + (int)threadIdx.x;
        const int quarter = b < p.batch ? (len[i] <= width) + (len[i] <= 2 * width) + (len[i] <= 3 * width) : -1;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint64_t mask = __builtin_amdgcn_ballot_w64(quarter == c);
            if (lane == 0)
                s.mask[c][i][wave] = mask;
        }
        s.len[b] = len[i];
    }
    __syncthreads();
    const uint64_t mask = lane < kMasks ? (&s.mask[0][0][0])[lane] : 0;
    const int count = __builtin_popcountll(mask), upto = wave_scan<TurnSum>(count);
    const uint64_t holder = __builtin_amdgcn_ballot_w64(upto - count <= turn && turn < upto);   // one lane
    const int at = __builtin_ctzll(holder);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mask, at),
                   hi = (uint32_t)__builtin_amdgcn_readlane((int)(mask >> 32), at);
    const int rank = turn - __builtin_amdgcn_readlane(upto - count, at);
    const bool here = (((uint64_t)hi << 32 | lo) >> lane & 1) != 0 &&
                      (int)__builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0)) == rank;
    const int b = at % (PASSES * kWavesPerBlock) / kWavesPerBlock * kThreads + at % kWavesPerBlock * kWave +
                  __builtin_ctzll(__builtin_amdgcn_ballot_w64(here));
    L = __builtin_amdgcn_readfirstlane(s.len[b]);
    return b;
}
// Where it is done: with long tables and more units than CUs, up to two passes. It costs
// some 0.5 us of a call, and the long sequences that would start last no longer run alone
// at the end. Calls in batch order -> in turn, cold pages, tokens 1 .. 16 times the table
// (all of 12 tokens per block):
//   96 x 28/4 heads of 128, 128 blocks   16.8 -> 15.1 (17.2 -> 17.6)    130 of them 23.6 -> 18.9
//   300 x 32/2 of 128, 128 blocks        25.0 -> 21.8 (27.3 -> 27.8)
//   384 x 32/8 of 64, 128 blocks         47.8 -> 45.7 (58.4 -> 58.5)
//   150 x 32/8 of 64, 80 blocks          16.2 -> 15.1 (18.1 -> 18.4)
// Not so with shorter tables (256 x 28/4 of 128, 64 blocks 18.1 -> 18.4, 300 x 32/8 of 64, 32
// blocks 15.1 -> 15.8) and with four passes (1000 x 28/4 of 128, 100 blocks 81.6 -> 82.0,
// lognormal lengths 43.0 -> 46.1). Nor with prefix sharing, whose members read a prompt's
// pages side by side.
constexpr int kTurnUnits = 256, kTurnBlocks = 64;
constexpr int kTurnPasses = 2;
constexpr int kTurnBatch = kTurnPasses * kWavesPerBlock * kWave;

// Attention where every sequence is short (a block table of at most
// kUnitBlocks entries): one workgroup per unit, its tiles dealt to the wavefronts
// in contiguous runs of whole steps, their states combined in LDS. One launch, no
// scan of the batch, no partial states in memory, three trips to memory before the
// first product (length, table entries, records beside query rows). Bound by
// that latency, and with thousands of units by instructions, as the stream is.
// Steps of two tiles: with four, fewer workgroups fit a CU (384 x 1..1024, 32/8
// heads, D = 64 28.8 us instead of 25.5; 512 x 1..256, 64/8 heads 40.3 and 25.3).
// With prefix sharing the members' rows of a prompt are attended one by one too
// (its pages come out of the caches): the groups only decide whose table entries
// name the shared pages, and which member is shorter than they are. They come in
// the first trip to memory.
template <int D, int KV, int WAVES, bool TURNS>
__global__ __launch_bounds__(kWave * WAVES) void unit_fp4_kernel(SplitParams p, UnitGroups groups)
{
    constexpr int NT = kUnitStepTiles;
    constexpr bool HALF = KV == kFp4Half;
    // Per wavefront what stage_partial writes: G rows of D fp32, then G pairs (m, l).
    __shared__ __attribute__((aligned(16))) uint8_t s_state[WAVES][(HALF ? 8 : kMaxGroup) * (D + 2) * 4];
    const int G = p.group, Hkv = p.num_kv_heads;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1);
    const int turn = blockIdx.x / Hkv, g = blockIdx.x - turn * Hkv;
    int b = turn, L;
    if constexpr (TURNS) {
        static_assert(WAVES == kWavesPerBlock, "the threads of sequence_in_turn");
        __shared__ TurnLds<kTurnPasses> s_turn;
        b = sequence_in_turn(s_turn, p, turn, wave, lane, L);
    } else {
        L = p.seq_lens[b];
    }
    SharedIn shared = {b, 0};
    if constexpr (!TURNS)   // (never with groups)
        shared = shared_in(groups, p, b, lane);
    const int unit = b * Hkv + g;
    const int n = lane & 15, quad = lane >> 4;
    const int max_len = p.max_blocks * kPageSize;
    const int pages = pages_of(L, max_len), steps = (pages + NT - 1) / NT;
    const int first = wave * steps / WAVES, count = (wave + 1) * steps / WAVES - first;
    const int tiles = min(count * NT, pages - first * NT);   // this wavefront's, at most kWave
    static_assert(kUnitBlocks <= WAVES * kWave, "a run's addresses lie in the lanes");
    // Lane i: the address of tile i of the run (those past it: the last one's).
    const int block = max(0, min(first * NT + min(lane, tiles - 1), pages - 1));
    const int page = p.block_table[(size_t)(block < shared.pages ? shared.lead : b) * p.max_blocks + block];
    const bool in = page >= 0 && page < p.num_pages;
    const bool bad = L < 0 || L > max_len || L < shared.pages * kPageSize ||
                     __builtin_amdgcn_ballot_w64(lane < tiles && !in) != 0;
    const uint64_t record = reinterpret_cast<uint64_t>(p.k_pages) +
                            (in ? (uint64_t)(uint32_t)(page * Hkv + g) * (uint32_t)fp4_record_bytes(D) : 0u);
    u32x4_t q[D / 32];
    load_q<D, KV>(q, p, (uint32_t)unit * (uint32_t)G, true, HALF ? n & 7 : n, quad);
    Fp4Tile<D> buf[2][NT];
    auto issue = [&](Fp4Tile<D>(&t)[NT], int i) {
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const int at = max(0, min(i * NT + u, tiles - 1));
            const uint64_t address = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)record, at) |
                                     (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(record >> 32), at) << 32;
            issue_record<D, kCachePolicyStream>(t[u], address, i < count, n, quad, lane);
        }
    };
    issue(buf[0], 0);
    Fp4State<D, HALF> state;
    reset(state);
    bf16x8_t qop[D / 32];
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
        qop[s] = __builtin_bit_cast(bf16x8_t, q[s] ^ fp4_sign(p.scale_log2));
    const float mul = __builtin_fabsf(p.scale_log2);
    for (int i0 = 0; i0 < count; i0 += 2) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = i0 + k;
            issue(buf[1 - k], i + 1);
            __builtin_amdgcn_sched_barrier(0);   // (else the first products wait for their tiles before these loads)
            if (i < count)
                fp4_step<D, NT>(state, buf[k], qop, mul, min(kPageSize * NT, L - kPageSize * NT * (first + i)), n,
                                quad);
        }
    }
    {
        const Piece<D> st = finished(state, quad);
        const float l = quad_sum(st.l);
        if (n < G)
            stage_partial<D>(st, l, bad, s_state[wave], G, n, quad);
    }
    __syncthreads();
    // out = sum of 2^(m_w - M) acc_w / sum of 2^(m_w - M) l_w. A weight of zero drops its
    // accumulators, not its sum of weights: a run of nothing but NaN scores has m = -inf, l = NaN.
    for (int i = threadIdx.x; i < G * (D / 4); i += kWave * WAVES) {
        const int row = i / (D / 4), c4 = 4 * (i % (D / 4));
        f32x2_t ml[WAVES];
        float M = kNegInf;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            ml[w] = *reinterpret_cast<const f32x2_t *>(s_state[w] + (size_t)G * D * 4 + 8 * row);
            M = fmaxf(M, ml[w][0]);
        }
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
        float l = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float c = __builtin_amdgcn_exp2f(ml[w][0] - M);
            l += c * ml[w][1];
            if (c != 0.0f)
                acc += c * *reinterpret_cast<const f32x4_t *>(s_state[w] + ((size_t)row * D + c4) * 4);
        }
        float inv = 1.0f / l;
        if (pages == 0) {   // zero, or NaN where a wavefront found the sequence invalid
            acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
            inv = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
                inv = ml[w][0] != ml[w][0] ? ml[w][0] : inv;
        }
        *reinterpret_cast<u32x2_t *>(p.out + ((size_t)unit * G + row) * D + c4) =
            u32x2_t{pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)};
    }
}

}  // namespace

namespace {
template <int WAVES, bool TURNS>
UnitKernel unit_kernel(int head_dim, int group)
{
    if (head_dim == 128)
        return group <= 8 ? unit_fp4_kernel<128, kFp4Half, WAVES, TURNS> : unit_fp4_kernel<128, kFp4, WAVES, TURNS>;
    if (head_dim == 64)
        return group <= 8 ? unit_fp4_kernel<64, kFp4Half, WAVES, TURNS> : unit_fp4_kernel<64, kFp4, WAVES, TURNS>;
    return nullptr;
}
}  // namespace

hipError_t launch_unit_fp4(const SplitParams &p, const UnitGroups &groups, int waves, int head_dim,
                           hipStream_t stream)
{
    const int units = p.batch * p.num_kv_heads;
    const bool turns = waves == kWavesPerBlock && groups.count == 0 && units > kTurnUnits && p.max_blocks > kTurnBlocks &&
                       p.batch <= kTurnBatch;
    const UnitKernel kernel = turns        ? unit_kernel<kWavesPerBlock, true>(head_dim, p.group)
                              : waves == 8 ? unit_kernel<8, false>(head_dim, p.group)
                                           : unit_kernel<4, false>(head_dim, p.group);
    if (!kernel)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, dim3((unsigned)units), dim3(kWave * waves), 0, stream, p, groups);
    return hipGetLastError();
}

SplitKernel split_fp4_kernel_of(int head_dim, int group)
{
    if (head_dim == 128)
        return group <= 8 ? split_fp4_kernel<128, kFp4Half> : split_fp4_kernel<128, kFp4>;
    if (head_dim == 64)
        return group <= 8 ? split_fp4_kernel<64, kFp4Half> : split_fp4_kernel<64, kFp4>;
    return nullptr;
}

PrefixKernel prefix_fp4_kernel_of(int head_dim, int group)
{
    if (head_dim == 128)
        return group <= 8 ? prefix_fp4_kernel<128, kFp4Half> : prefix_fp4_kernel<128, kFp4>;
    if (head_dim == 64)
        return group <= 8 ? prefix_fp4_kernel<64, kFp4Half> : prefix_fp4_kernel<64, kFp4>;
    return nullptr;
}

}  // namespace sl
