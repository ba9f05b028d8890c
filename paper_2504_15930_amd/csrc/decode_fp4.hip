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
    if ((int)blockIdx.x < own_blocks)
        split_unit_worker<D, KV, kOwnPages>(
            own, blockIdx.x * kWavesPerBlock + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave),
            StreamLds{s_own, s_len, s_shared});
    else {
        SplitParams sh = shared;
        sh.num_workers = effective_shared_workers((long long)s_own[B] * own.num_kv_heads, own.num_workers,
                                                  shared.num_workers, max_shared, NT, kFp4);
        split_unit_worker<D, kFp4, kSharedPages>(sh, (int)blockIdx.x - own_blocks,
                                                  StreamLds{s_sh, nullptr, nullptr, s_gl, S},
                                                  __builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
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
