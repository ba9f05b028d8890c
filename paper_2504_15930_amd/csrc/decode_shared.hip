// Prefix-shared decode attention for gfx950: the fused split kernel that
// streams the own pages and the shared pages of a batch in one launch.
//
// A shared unit is (sub-group of samples, KV head): its tiles are the
// group's shared pages, read through the sub-group's first member's
// block-table row, and its query rows are the members x G query heads of that
// KV head, at most kPrefixRows = 64, as four 16-row MFMA column blocks (row
// r = 16 c + n is member r / G, head r % G of the sub-group). A group larger
// than that is cut into sub-groups, each reading the shared pages once.
//
// Workgroups [0, own_blocks) run the single-unit workers of the own pages
// (decode_unit.h, four per workgroup). The others are shared-page workers,
// one per workgroup: the workgroup's four wavefronts stream the same range of
// shared tiles with the single-unit pipeline, and wavefront c computes column
// block c of every unit in it. They read each tile at the same time with
// plain (not streaming) loads, so the tile comes from HBM once and the
// siblings find it in L2; no wavefront waits for another. Each wavefront
// keeps one block's registers.
//
// The kernel is instantiated for bf16 and E4M3 pages and for FP4 records. For
// E4M3 and FP4 every wavefront widens the whole shared tile itself (its block
// needs all keys and values) and scales it by the tile's own scales.
//
// The own-page workgroups come first, so each CU holds one of them beside a
// shared-page workgroup: the memory-bound and the MFMA-heavy pass share the
// CUs instead of running one after the other.
//
// Partial states: a unit cut by a worker's range leaves its piece in slot 2w
// (first piece) or 2w + 1 (trailing piece) of the worker; a unit seen whole
// goes to its own slot of the unit area, at (first query row) / G. Every
// shared state still has to be merged with the members' own pages, and so do
// the own units of sequences that have shared pages.
#include "prefix_unit.h"

namespace sl {
namespace {

// Both passes of prefix-shared attention in one launch (see the top of this
// file). Every workgroup first derives both streams in its dynamic LDS
// (prefix_dynamic_lds: 3 B + 2 S + 3 ints, S = pp.max_sub); the number of
// shared-page workers that take part is effective_shared_workers of the
// own-page total, as in the merge.
template <int D, bool FP8>
__global__ __launch_bounds__(kWave * kWavesPerBlock) void prefix_split_kernel(SplitParams own, SplitParams shared,
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
    // The groups' starts and pages, read by the scan alone: in the state queues,
    // which are idle until then. (In dynamic LDS beside the rest, 4096 sequences
    // in more than 3862 groups did not fit a CU with the 16 KB K stage of bf16,
    // D = 128.)
    static_assert(sizeof(int32_t) * (2 * kMaxPrefixBatch + 1) <= kWavesPerBlock * kOwnStageBytes, "the group arrays");
    int32_t *const s_gs = reinterpret_cast<int32_t *>(own_state_stage());   // [NG + 1]
    int32_t *const s_sp = s_gs + pp.num_groups + 1;                         // [NG]
    constexpr int NT = step_tiles<D, FP8>();
    scan_prefix_groups<NT>(own, pp, s_own, s_len, s_shared, s_sh, s_gl, s_gs, s_sp);
    if ((int)blockIdx.x < own_blocks)
        split_unit_worker<D, FP8, kOwnPages>(
            own, blockIdx.x * kWavesPerBlock + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave),
            StreamLds{s_own, s_len, s_shared});
    else {
        SplitParams sh = shared;
        sh.num_workers = effective_shared_workers((long long)s_own[B] * own.num_kv_heads, own.num_workers,
                                                  shared.num_workers, max_shared, NT, FP8);
        split_unit_worker<D, FP8, kSharedPages>(sh, (int)blockIdx.x - own_blocks,
                                                  StreamLds{s_sh, nullptr, nullptr, s_gl, S},
                                                  __builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    }
}

}  // namespace

hipError_t launch_prefix_split(const SplitParams &own, const SplitParams &shared, int max_shared,
                               const PrefixParams &pp, int head_dim, int kv, hipStream_t stream)
{
    const int own_blocks = (own.num_workers + kWavesPerBlock - 1) / kWavesPerBlock;
    const dim3 grid(own_blocks + max_shared);
    const dim3 block(kWave * kWavesPerBlock);
    const size_t lds = prefix_dynamic_lds(own.batch, pp.max_sub);
    PrefixKernel kernel = nullptr;
    if (kv == kFp4)
        kernel = prefix_fp4_kernel_of(head_dim, own.group);
    else if (head_dim == 128)
        kernel = kv == kE4m3 ? prefix_split_kernel<128, true> : prefix_split_kernel<128, false>;
    else if (head_dim == 64)
        kernel = kv == kE4m3 ? prefix_split_kernel<64, true> : prefix_split_kernel<64, false>;
    if (!kernel)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, grid, block, lds, stream, own, shared, pp, own_blocks, max_shared);
    return hipGetLastError();
}

}  // namespace sl
