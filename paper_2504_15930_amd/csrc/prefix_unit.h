#ifndef SL_PREFIX_UNIT_H
#define SL_PREFIX_UNIT_H
// Prologue of the fused prefix kernels (decode_shared.hip, decode_fp4.hip): the
// two streams of a batch with shared pages.
#include "decode_unit.h"

namespace sl {
namespace {

// Prologue of the fused prefix kernel, run by the whole workgroup. A group k
// is shared if its range [group_start[k], group_start[k+1]) is non-empty,
// inside the batch and starts at or after the end of every earlier group's
// range (so the groups that are shared never overlap, whatever the order of
// group_start), and its page count is in 1 .. max_blocks. Others are attended
// like unshared sequences: exact, only without the saving. A shared group of
// m members is cut into ns = ceil(m / M) sub-groups of ceil(m / ns) members
// (the last may be smaller), M = min(16, kPrefixRows / G), each of which
// reads the shared pages once: the shared stream has one "sequence" per
// sub-group. Builds in LDS, with every pass parallel over groups,
// sub-groups or sequences:
//   s_shared[b] the shared pages of sequence b (B + 1 entries, the last one
//               scratch),
//   s_len[b]    the lengths,
//   s_own[0..B] the exclusive prefix sum of steps (of NT pages) over the own
//               (unshared) pages per sequence,
//   s_sh[0..S]  the exclusive prefix sum of steps over the shared pages per
//               sub-group, and
//   s_gl[s]     each sub-group's first member, size and the pages missing from
//               its last step, lead | (members - 1) << 16 | missing << 24,
// where S = max_sub bounds the sub-group count (sub-groups past the real
// count have no pages). Workgroup 0 also stores the sums and every
// sequence's sharing descriptor for the merge.
template <int NT>
__device__ __forceinline__ void scan_prefix_groups(const SplitParams &p, const PrefixParams &pp, int32_t *s_own,
                                                   int32_t *s_len, int32_t *s_shared, int32_t *s_sh, int32_t *s_gl,
                                                   int32_t *s_gs, int32_t *s_sp)
{
    constexpr int T = kWave * kWavesPerBlock;
    const int B = p.batch, NG = pp.num_groups, S = pp.max_sub;
    const int tid = threadIdx.x;
    const int M = prefix_max_members(p.group);
    const int32_t *gs = s_gs;   // group_start and shared_pages, read from memory once
    // Scratch for the group passes, in arrays filled only later: s_len (B
    // entries, followed by s_sh, whose first entry takes the scan's total when
    // NG == B) and s_own (B + 1 entries).
    int32_t *const s_prev_end = s_len;   // [NG + 1]: largest end of the earlier groups
    int32_t *const s_base = s_own;       // [NG + 1]: first sub-group of each group
    int32_t *const s_group = s_shared;   // [B + 1]: marks of the groups' first members
    // The lengths, needed last, come with the group arrays: one trip to memory.
    constexpr int kPer = (kMaxPrefixBatch + T - 1) / T;
    int32_t len[kPer];
#pragma unroll
    for (int r = 0; r < kPer; ++r)
        len[r] = tid + r * T < B ? p.seq_lens[tid + r * T] : 0;
    // 1. Each group's earlier ends; every sequence starts unmarked. With
    //    group_start ascending (the usual case) the largest earlier end of
    //    group k is its own start, and the scan is skipped.
    bool descends = false;
    for (int k = tid; k < NG; k += T) {
        const int lo = pp.group_start[k], hi = pp.group_start[k + 1];
        s_gs[k] = lo;
        s_sp[k] = pp.shared_pages[k];
        if (k == NG - 1)
            s_gs[NG] = hi;
        descends |= lo > hi;
    }
    for (int b = tid; b < B; b += T)
        s_group[b] = -1;
    const bool ascending = !__syncthreads_or(descends);
    if (!ascending) {
        for (int k = tid; k < NG; k += T)
            s_prev_end[k] = gs[k + 1];
        __syncthreads();
        block_exclusive_scan<ScanMax>(s_prev_end, NG);
    }
    // 2. Which groups are shared, how many sub-groups each has, and a mark at
    //    each shared group's first member (shared groups never overlap, so no
    //    two marks collide).
    for (int k = tid; k < NG; k += T) {
        const int lo = gs[k], hi = gs[k + 1], sp = s_sp[k];
        const bool ok = lo >= 0 && hi <= B && hi > lo && (ascending || lo >= s_prev_end[k]) && sp > 0 &&
                        sp <= p.max_blocks;
        s_base[k] = ok ? small_div(hi - lo + M - 1, M) : 0;
        if (ok)
            s_group[lo] = k;
    }
    __syncthreads();
    // s_base: first sub-group of each group; s_group[b + 1]: the latest mark at or before b.
    block_exclusive_scan2<ScanSum, ScanMax>(s_base, NG, s_group, B);
    // 3. The sub-groups: shared steps and packed first member and size.
    const int NS = s_base[NG];
    for (int sg = tid; sg < S; sg += T) {
        int sp = 0, gl = 0;
        if (sg < NS) {
            int klo = 0, khi = NG;   // largest k with s_base[k] <= sg (a group with sub-groups)
            while (khi - klo > 1) {
                const int mid = (klo + khi) >> 1;
                if (s_base[mid] <= sg)
                    klo = mid;
                else
                    khi = mid;
            }
            const int lo = gs[klo], m = gs[klo + 1] - lo;
            const int ns = small_div(m + M - 1, M), cm = small_div(m + ns - 1, ns);
            const int slo = lo + (sg - s_base[klo]) * cm;
            sp = s_sp[klo];
            gl = slo | (min(cm, lo + m - slo) - 1) << 16 | (NT - 1 - (sp + NT - 1) % NT) << 24;
        }
        s_sh[sg] = (sp + NT - 1) / NT;
        s_gl[sg] = gl;
    }
    // 4. The sub-group of every sequence: the group of the latest mark at or
    //    before b (the exclusive scan's entry b + 1; entry B holds the
    //    maximum), if b lies inside that group's range; its shared pages.
    int32_t sub[kPer], sh[kPer];
#pragma unroll
    for (int r = 0; r < kPer; ++r) {
        const int b = tid + r * T;
        sub[r] = -1;
        sh[r] = 0;
        if (b < B) {
            const int k = s_group[b + 1];
            if (k >= 0 && b < gs[k + 1]) {
                const int lo = gs[k], m = gs[k + 1] - lo;
                const int ns = small_div(m + M - 1, M), cm = small_div(m + ns - 1, ns);
                const int sg = s_base[k] + small_div(b - lo, cm);
                if (sg < S) {   // always (prefix_max_sub bounds the count)
                    sub[r] = sg;
                    sh[r] = s_sp[k];
                }
            }
        }
    }
    __syncthreads();   // the scratch arrays are free
    // 5. Lengths, shared pages and own steps (over the pages after the
    //    sub-group's shared ones).
    const int max_len = p.max_blocks * kPageSize;
#pragma unroll
    for (int r = 0; r < kPer; ++r) {
        const int b = tid + r * T;
        if (b < B) {
            const int n = pages_of(len[r], max_len);
            s_len[b] = len[r];
            s_shared[b] = sh[r];
            s_own[b] = n > sh[r] ? (n - sh[r] + NT - 1) / NT : 0;
        }
    }
    __syncthreads();
    block_exclusive_scan2<ScanSum, ScanSum>(s_own, B, s_sh, S);
    if (blockIdx.x == 0) {
        for (int i = tid; i <= B; i += T)
            pp.cum_own[i] = s_own[i];
        for (int i = tid; i <= S; i += T)
            pp.cum_shared[i] = s_sh[i];
        typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int r = 0; r < kPer; ++r) {
            const int b = tid + r * T, k = sub[r];
            if (b < B)
                *reinterpret_cast<i32x4_t *>(pp.seq_shared + 4 * (size_t)b) =
                    k >= 0 ? i32x4_t{s_sh[k], s_shared[b], s_gl[k] & 0xffff, s_sh[k + 1] - s_sh[k]}
                           : i32x4_t{0, 0, 0, 0};
        }
    }
}

}  // namespace
}  // namespace sl

#endif  // SL_PREFIX_UNIT_H
