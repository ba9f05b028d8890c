// Split-KV decode attention kernel for gfx950: one wavefront per worker, the
// worker itself (tile pipeline, MFMA layout, online softmax, epilogue) is in
// decode_unit.h.
#include "decode_unit.h"

namespace sl {
namespace {

// Every workgroup derives the tile stream from the lengths and the block
// table (its dynamic LDS holds the prefix sum of steps and the lengths).
//
// Worker w = wave * gridDim.x + block: the four wavefronts of a workgroup take
// ranges a quarter of the stream apart, so a CU streams four unrelated
// sequences or heads at once rather than four neighbouring ranges of one
// unit (whose tiles all sit at the same offset inside their pages), and a
// stream too small for every worker still spreads over as many CUs as it
// has workers.
template <int D, bool FP8>
__global__ __launch_bounds__(kWave * kWavesPerBlock) void split_kv_kernel(SplitParams p)
{
    extern __shared__ int32_t s_dyn[];
    int32_t *const s_cum = s_dyn;                // [B + 1]
    int32_t *const s_len = s_dyn + p.batch + 1;  // [B]
    scan_sequences<step_tiles<D, FP8>()>(p, s_cum, s_len);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    split_unit_worker<D, FP8, kAllPages>(p, wave * (int)gridDim.x + (int)blockIdx.x,
                                         StreamLds{s_cum, s_len});
}

SplitKernel split_kernel(int head_dim, int kv, int group)
{
    if (kv == kFp4)
        return split_fp4_kernel_of(head_dim, group);
    if (head_dim == 128)
        return kv == kE4m3 ? split_kv_kernel<128, true> : split_kv_kernel<128, false>;
    if (head_dim == 64)
        return kv == kE4m3 ? split_kv_kernel<64, true> : split_kv_kernel<64, false>;
    return nullptr;
}

}  // namespace

hipError_t launch_split(const SplitParams &p, int head_dim, int kv, hipStream_t stream)
{
    const dim3 grid((p.num_workers + kWavesPerBlock - 1) / kWavesPerBlock);
    const dim3 block(kWave * kWavesPerBlock);
    const SplitKernel kernel = split_kernel(head_dim, kv, p.group);
    if (!kernel)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, grid, block, split_dynamic_lds(p.batch), stream, p);
    return hipGetLastError();
}

hipError_t split_blocks_per_cu(int head_dim, int kv, int *blocks)
{
    const SplitKernel kernel = split_kernel(head_dim, kv, kMaxGroup);
    if (!kernel)
        return hipErrorInvalidValue;
    return hipOccupancyMaxActiveBlocksPerMultiprocessor(blocks, kernel, kWave * kWavesPerBlock, 0);
}

int split_step_tiles(int head_dim, int kv, bool prefix)
{
    const bool d64 = head_dim == 64;
    if (kv == kFp4)
        return prefix ? (d64 ? step_tiles<64, kFp4, true>() : step_tiles<128, kFp4, true>())
                      : (d64 ? step_tiles<64, kFp4>() : step_tiles<128, kFp4>());
    return kv == kE4m3 ? (d64 ? step_tiles<64, kE4m3>() : step_tiles<128, kE4m3>())
                       : (d64 ? step_tiles<64, kBf16>() : step_tiles<128, kBf16>());
}

}  // namespace sl
