// Page bookkeeping of a paged cache on the GPU: pages from a stack of free ones
// for the tokens that each request adds, with the tokens' slots, and the pages
// of finished requests back on the stack.
//
// Everything follows from sums over the requests before: of the pages that they
// open, of the tokens that they add, of the pages that they give back. One
// workgroup holds the batch (at most kMaxBatch requests, eight per thread) and
// forms them with two scans, so the lengths and the count may be updated in
// place; it finds a page's or a token's request by binary search in the sums,
// which it keeps in LDS. Many pages and a long slot map are shared among
// workgroups that all form the sums for themselves, if nothing that they read is
// updated in place; else one workgroup moves the pages, and a second launch makes
// the slot map. Bound by latency, a few dependent trips to memory: 256 requests of
// one token 4.2 us.
#include <algorithm>

#include "sl_internal.h"
#include "wave_ops.h"

namespace sl {
namespace {

constexpr int kPageThreads = 1024;
constexpr int kPageWaves = kPageThreads / kWave;
constexpr int kMostPer = (kMaxBatch + kPageThreads - 1) / kPageThreads;   // requests per thread

struct Sum {
    static constexpr uint32_t kIdentity = 0;
    __device__ static uint32_t op(uint32_t a, uint32_t b) { return a + b; }
};

// Exclusive prefix sums of two values per thread over the workgroup, and their
// totals. `s` is scratch; ends with a barrier after which it may be reused.
__device__ __forceinline__ void block_sums(uint32_t &a, uint32_t &b, uint32_t &total_a, uint32_t &total_b,
                                           uint32_t (*s)[2])
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1);
    const uint32_t ia = wave_scan<Sum>(a), ib = wave_scan<Sum>(b);
    if (lane == kWave - 1) {
        s[wave][0] = ia;
        s[wave][1] = ib;
    }
    __syncthreads();
    uint32_t before_a = 0, before_b = 0;
    total_a = total_b = 0;
#pragma unroll
    for (int k = 0; k < kPageWaves; ++k) {
        if (k < wave) {
            before_a += s[k][0];
            before_b += s[k][1];
        }
        total_a += s[k][0];
        total_b += s[k][1];
    }
    a = before_a + ia - a;
    b = before_b + ib - b;
    __syncthreads();
}

// The request that holds item x: the largest b with sum[b] <= x (sum[n] > x).
__device__ __forceinline__ int find(const uint32_t *sum, int n, uint32_t x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__device__ __forceinline__ uint32_t blocks_of(int len) { return ((uint32_t)len + kPageSize - 1) / kPageSize; }

__device__ __forceinline__ int32_t slot_in(int32_t page, int pos, int num_pages)
{
    return page >= 0 && page < num_pages ? page * kPageSize + pos % kPageSize : -1;
}

// Pages on the stack, read before the first barrier: the count may be updated
// in place once every wavefront has passed it. (For the compiler the register
// changes here; it would move the load, scalar and the same for every
// wavefront, to the first use.)
__device__ __forceinline__ uint32_t stack_size(const PageParams &p)
{
    int32_t n = p.free_count[0];
    asm volatile("" : "+s"(n));
    return (uint32_t)max(0, min(n, p.num_pages));
}

// `slots_per_block`: entries of the slot map that each workgroup makes; none if
// 0, and fill_slots_kernel follows. With several workgroups, those enter the opened
// pages in turn, and the first one writes the rest.
template <int PER>
__global__ __launch_bounds__(kPageThreads) void extend_pages_kernel(PageParams p, uint32_t slots_per_block)
{
    extern __shared__ uint32_t s_dyn[];
    __shared__ uint32_t s_wave[kPageWaves][2];
    const int B = p.batch, tid = threadIdx.x;
    const bool one = blockIdx.x == 0;
    uint32_t *const s_tok = s_dyn;            // [B + 1] tokens of the requests before
    uint32_t *const s_pg = s_tok + B + 1;     // [B + 1] pages that they open
    uint32_t *const s_len = s_pg + B + 1;     // [B] lengths so far
    const int per = PER == 1 ? 1 : (B + kPageThreads - 1) / kPageThreads, first = tid * per;
    const int most = p.max_blocks * kPageSize;
    const uint32_t count = stack_size(p);
    int len[PER];
    uint32_t add[PER], open[PER];
    uint32_t tok = 0, pg = 0, all_tok, all_pg;
    bool valid[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = first + i;
        const bool in = i < per && b < B;
        len[i] = in ? p.seq_lens[b] : 0;
        const int n = in ? p.new_tokens[b] : 0;
        valid[i] = in && len[i] >= 0 && len[i] <= most && n >= 0 && n <= most - len[i];
        add[i] = valid[i] ? (uint32_t)n : 0u;
        open[i] = valid[i] ? blocks_of(len[i] + n) - blocks_of(len[i]) : 0u;
        tok += add[i];
        pg += open[i];
    }
    block_sums(tok, pg, all_tok, all_pg, s_wave);
    // A request is served if the tokens up to its own fit the slot map and, where it opens any, the
    // pages up to its own are there.
    uint32_t got_tok = 0, got_pg = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        tok += add[i];
        pg += open[i];
        if (tok > (uint32_t)p.max_tokens || (open[i] > 0 && pg > count))
            add[i] = open[i] = 0;
        got_tok += add[i];
        got_pg += open[i];
    }
    block_sums(got_tok, got_pg, all_tok, all_pg, s_wave);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = first + i;
        if (i < per && b < B) {
            s_tok[b] = got_tok;
            s_pg[b] = got_pg;
            s_len[b] = (uint32_t)len[i];
            if (one) {
                p.token_start[b] = (int32_t)got_tok;
                p.seq_lens_out[b] = len[i] + (int32_t)add[i];
            }
        }
        got_tok += add[i];
        got_pg += open[i];
    }
    if (tid == 0) {
        s_tok[B] = all_tok;
        s_pg[B] = all_pg;
        if (one) {
            p.token_start[B] = (int32_t)all_tok;
            p.free_count_out[0] = (int32_t)(count - all_pg);
        }
    }
    __syncthreads();
    for (uint32_t x = blockIdx.x * kPageThreads + tid; x < all_pg; x += gridDim.x * kPageThreads) {
        const int b = find(s_pg, B, x);
        p.block_table[(size_t)b * p.max_blocks + blocks_of((int)s_len[b]) + (x - s_pg[b])] = p.free_pages[count - 1 - x];
    }
    const uint32_t from = blockIdx.x * slots_per_block, to = min(from + slots_per_block, (uint32_t)p.max_tokens);
    for (uint32_t x = from + tid; x < to; x += kPageThreads) {
        int32_t slot = -1;
        if (x < all_tok) {
            const int b = find(s_tok, B, x);
            const uint32_t had = blocks_of((int)s_len[b]);
            const int pos = (int)(s_len[b] + (x - s_tok[b]));
            const uint32_t blk = (uint32_t)pos / kPageSize;
            // (an opened page from the stack, not through the table that is being written)
            const int32_t page = blk < had ? p.block_table[(size_t)b * p.max_blocks + blk]
                                           : p.free_pages[count - 1 - (s_pg[b] + blk - had)];
            slot = slot_in(page, pos, p.num_pages);
        }
        p.slots[x] = slot;
    }
}

// The slot map of many tokens, after extend_pages_kernel: kSlotTokens per workgroup.
constexpr int kSlotThreads = 256;
constexpr int kSlotTokens = 1024;
__global__ __launch_bounds__(kSlotThreads) void fill_slots_kernel(PageParams p)
{
    extern __shared__ uint32_t s_dyn[];
    const int B = p.batch;
    for (int b = threadIdx.x; b <= B; b += kSlotThreads)
        s_dyn[b] = (uint32_t)p.token_start[b];
    __syncthreads();
    const uint32_t all = s_dyn[B];
#pragma unroll
    for (int k = 0; k < kSlotTokens / kSlotThreads; ++k) {
        const uint32_t x = blockIdx.x * (uint32_t)kSlotTokens + k * kSlotThreads + threadIdx.x;
        if (x >= (uint32_t)p.max_tokens)
            return;
        int32_t slot = -1;
        if (x < all) {
            const int b = find(s_dyn, B, x);
            const int pos = p.seq_lens_out[b] - (int)(s_dyn[b + 1] - x);
            slot = slot_in(p.block_table[(size_t)b * p.max_blocks + pos / kPageSize], pos, p.num_pages);
        }
        p.slots[x] = slot;
    }
}

template <int PER>
__global__ __launch_bounds__(kPageThreads) void release_pages_kernel(PageParams p)
{
    extern __shared__ uint32_t s_dyn[];
    __shared__ uint32_t s_wave[kPageWaves][2];
    const int B = p.batch, tid = threadIdx.x;
    uint32_t *const s_pg = s_dyn;   // [B + 1] pages given back by the requests before
    const int per = PER == 1 ? 1 : (B + kPageThreads - 1) / kPageThreads, first = tid * per;
    const int most = p.max_blocks * kPageSize;
    const uint32_t count = stack_size(p);
    int len[PER];
    uint32_t back[PER];
    uint32_t pg = 0, none = 0, all, all_none;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = first + i;
        const bool in = i < per && b < B;
        len[i] = in ? p.seq_lens[b] : 0;
        const bool done = in && p.finished[b] != 0 && len[i] >= 0 && len[i] <= most;
        back[i] = done ? blocks_of(len[i]) : 0u;
        len[i] = done ? 0 : len[i];
        pg += back[i];
    }
    block_sums(pg, none, all, all_none, s_wave);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = first + i;
        if (i < per && b < B) {
            s_pg[b] = pg;
            if (blockIdx.x == 0)
                p.seq_lens_out[b] = len[i];
        }
        pg += back[i];
    }
    const uint32_t room = (uint32_t)p.num_pages - count;   // (pages given back twice do not fit)
    if (tid == 0) {
        s_pg[B] = all;
        if (blockIdx.x == 0)
            p.free_count_out[0] = (int32_t)(count + min(all, room));
    }
    __syncthreads();
    // (a request's last block first)
    for (uint32_t x = blockIdx.x * kPageThreads + tid; x < min(all, room); x += gridDim.x * kPageThreads) {
        const int b = find(s_pg, B, x);
        p.free_pages[count + x] = p.block_table[(size_t)b * p.max_blocks + (s_pg[b + 1] - 1 - x)];
    }
}

// Entries of the slot map, or of the block table, per workgroup, at least: one per
// thread (66000 tokens of 96 requests 5.4 us, with four 8.4). Workgroups at most, one per
// CU. Where one workgroup has to do everything, it makes the slot map too up to
// this many entries.
constexpr uint32_t kItemsPerBlock = kPageThreads;
constexpr uint32_t kMostBlocks = 256;
constexpr uint32_t kAloneSlots = 4 * kPageThreads;

// Neither the lengths nor the count is updated in place.
bool apart(const PageParams &p) { return p.seq_lens_out != p.seq_lens && p.free_count_out != p.free_count; }

}  // namespace

// (One request per thread where that is enough: the code for eight is four times
// as long, and a first pass through it is instruction fetches.)
// Call with 1024 requests of 1000 tokens: 9.7 us, with one workgroup for the
// pages and a second launch 63; 96 of 1365: 5.0 and 13.4; 8192 of 100: 23 and 85.
hipError_t launch_extend_pages(const PageParams &p, hipStream_t stream)
{
    const uint32_t tokens = (uint32_t)p.max_tokens;
    const uint32_t each = apart(p) ? std::max(kItemsPerBlock, (tokens + kMostBlocks - 1) / kMostBlocks) : kAloneSlots;
    const bool one_launch = apart(p) || tokens <= kAloneSlots;
    const uint32_t blocks = one_launch && tokens > 0 ? (tokens + each - 1) / each : 1;
    hipLaunchKernelGGL(p.batch <= kPageThreads ? extend_pages_kernel<1> : extend_pages_kernel<kMostPer>, dim3(blocks),
                       dim3(kPageThreads), sizeof(uint32_t) * (3 * (size_t)p.batch + 2), stream, p,
                       one_launch ? each : 0u);
    hipError_t e = hipGetLastError();
    if (one_launch || e != hipSuccess)
        return e;
    hipLaunchKernelGGL(fill_slots_kernel, dim3((tokens + kSlotTokens - 1) / kSlotTokens), dim3(kSlotThreads),
                       sizeof(uint32_t) * ((size_t)p.batch + 1), stream, p);
    return hipGetLastError();
}

hipError_t launch_release_pages(const PageParams &p, hipStream_t stream)
{
    const uint64_t pages = (uint64_t)p.batch * (uint64_t)p.max_blocks;   // at most
    const uint64_t blocks = apart(p) ? std::min<uint64_t>(kMostBlocks, pages / kItemsPerBlock + 1) : 1;
    hipLaunchKernelGGL(p.batch <= kPageThreads ? release_pages_kernel<1> : release_pages_kernel<kMostPer>,
                       dim3((unsigned)blocks), dim3(kPageThreads), sizeof(uint32_t) * ((size_t)p.batch + 1), stream, p);
    return hipGetLastError();
}

}  // namespace sl
