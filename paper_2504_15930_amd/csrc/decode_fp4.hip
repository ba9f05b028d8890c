// Split-KV decode attention over a 4-bit cache (fp4_unit.h has its layout): the
// kernels of decode_split.hip and decode_shared.hip for FP4 records.
//
// One step is four tiles (17 D bytes each, K and V).
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
// 31.8 -> 23.6 us; 16 of 4000 x 24, 12/12 heads, D = 64 115 -> 51; 64 of 2000 x 4,
// 64/8 heads, D = 128 118 -> 79; with four blocks the same.
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
        const int blocks = effective_shared_workers((long long)s_own[B] * own.num_kv_heads, own.num_workers,
                                                    shared.num_workers, max_shared, NT, kFp4);
        if (block >= blocks)
            return;
        SplitParams sh = shared;
        sh.num_workers = shared_workers_of(blocks, per_block, own.num_workers);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = kPrefixBlocks / per_block;
        split_unit_worker<D, kFp4, kSharedPages>(sh, wave / waves * blocks + block,
                                                 StreamLds{s_sh, nullptr, nullptr, s_gl, S}, wave % waves);
    }
}

}  // namespace

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
