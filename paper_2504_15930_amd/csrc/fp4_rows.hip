// Rows into and out of the 4-bit cache (the record of fp4_unit.h).
//
// Quantise-on-write. A row is cut into blocks of 32 elements; with a = max |x|
// of a block, its scale is the smallest power of two under which a rounds to at
// most 6, E2M1's largest value: a < 7 2^e. On the bits of a (bf16: 8 exponent,
// 7 mantissa bits) adding 0x20 carries into the exponent exactly when the
// mantissa is 1.75 or more, so the scale byte is ((bits + 0x20) >> 7) - 2, kept
// within 1 .. 252 (2^-126, so that it is a normal fp32, and 2^125, whose 6 is
// the largest code value that bf16 holds). Elements are rounded to the nearest
// code, ties to the even one, saturating at 6; so every stored value is within
// half a step of its element. A block that holds a NaN or an infinity gets the
// scale byte 255 and zero codes, and reads as NaN. Rows do not depend on each
// other, so nothing is read before it is written.
//
// Eight elements per thread: a 16-byte load, four conversions
// (v_cvt_scalef32_pk_fp4_bf16), and a 4-byte store of codes; a block is four
// neighbouring threads, whose maximum takes two DPP moves.
//
// Bound by memory where there are many rows (the writer stores 68 bytes for 256
// read, D = 128): 12322 tokens of 8 KV heads, 64 MB, in 15.5 us, 4.1 TB/s, read back
// in 15.6 (a large copy: 5.1 TB/s); by the launch where there are few (96 rows 3.1
// and 2.5 us).
#include "fp4_unit.h"
#include "wave_ops.h"

namespace sl {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

constexpr int kRowThreads = 256;
constexpr int kPer = 8;   // elements of a row per thread
// From this many elements of K and V on (4096 workgroups with one row per thread),
// rows per thread: fewer workgroups to start.
constexpr long long kManyRowElements = 4ll << 20;
constexpr int kRowsPerThread = 4;

// Which element run of which rows a thread has: `part` 0 .. D/8 - 1 of the key
// (which 0) or value row of the (token, KV head) numbers first, first + kUnits, ...
template <int D, int ROWS>
struct RowPart {
    static constexpr int kParts = D / kPer;
    static constexpr int kUnits = kRowThreads / (2 * kParts);
    int first, which, part;
    __device__ __forceinline__ RowPart()
    {
        const int at = threadIdx.x;
        part = at % kParts;
        which = at / kParts % 2;
        first = (int)blockIdx.x * (kUnits * ROWS) + at / (2 * kParts);
    }
    __device__ __forceinline__ int unit(int i) const { return first + i * kUnits; }
};

// Maximum over the four threads of a block (neighbouring lanes).
__device__ __forceinline__ uint32_t quad_lanes_max(uint32_t x)
{
    const uint32_t y = lane_from<0xb1, 0xf>(x, 0u);   // lanes 1 0 3 2
    x = x > y ? x : y;
    const uint32_t z = lane_from<0x4e, 0xf>(x, 0u);   // lanes 2 3 0 1
    return x > z ? x : z;
}

__device__ __forceinline__ uint32_t scale_of(uint32_t top)   // of the block's largest magnitude bits
{
    if (top >= 0x7f80u)
        return 255u;
    const int s = (int)((top + 0x20u) >> 7) - 2;
    return (uint32_t)(s < 1 ? 1 : s > 252 ? 252 : s);
}

// Where the eight codes of a part go: one dword for keys and for values of D =
// 128, two halves for values of D = 64 (runs of four elements, 8 bytes apart).
template <int D>
__device__ __forceinline__ int code_at(int which, int t, int part)
{
    using L = Fp4Layout<D>;
    return which ? L::v_code(t, part * kPer / (D / 16)) : L::k_code(t, part / 4) + 4 * (part % 4);
}
template <int D>
__device__ __forceinline__ int scale_at(int which, int t, int part)
{
    using L = Fp4Layout<D>;
    return which ? L::v_scale(t, part / 4) : L::k_scale(t, part / 4);
}

template <int D>
__device__ __forceinline__ void store_part(uint8_t *rec, int which, int t, int part, u32x4_t x)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = x[i] & 0x7fffu, hi = x[i] >> 16 & 0x7fffu;
        top = max(top, max(lo, hi));
    }
    const uint32_t s = scale_of(quad_lanes_max(top));
    uint32_t codes = 0;
    if (s != 255u) {
        const float scale = e8m0(s);
        // (copies: a bit cast of a vector's element takes its first one here)
        const uint32_t w0 = x[0], w1 = x[1], w2 = x[2], w3 = x[3];
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, w0), scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, w1), scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, w2), scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2_t, w3), scale, 3);
    }
    uint8_t *const at = rec + code_at<D>(which, t, part);
    if (D == 64 && which) {
        *reinterpret_cast<uint16_t *>(at) = (uint16_t)codes;
        *reinterpret_cast<uint16_t *>(at + 4 * Fp4Layout<D>::kRun) = (uint16_t)(codes >> 16);
    } else {
        *reinterpret_cast<uint32_t *>(at) = codes;
    }
    if (part % 4 == 0)
        rec[scale_at<D>(which, t, part)] = (uint8_t)s;
}

template <int D>
__device__ __forceinline__ u32x4_t load_part(const uint8_t *rec, int which, int t, int part)
{
    const uint8_t *const at = rec + code_at<D>(which, t, part);
    uint32_t codes;
    if (D == 64 && which)
        codes = *reinterpret_cast<const uint16_t *>(at) |
                (uint32_t)*reinterpret_cast<const uint16_t *>(at + 4 * Fp4Layout<D>::kRun) << 16;
    else
        codes = *reinterpret_cast<const uint32_t *>(at);
    const float scale = e8m0(rec[scale_at<D>(which, t, part)]);
    return u32x4_t{fp4x2_to_bf16<0>(codes, scale), fp4x2_to_bf16<1>(codes, scale), fp4x2_to_bf16<2>(codes, scale),
                   fp4x2_to_bf16<3>(codes, scale)};
}

// Slot of row t: of a slot map, or of a decode step's new token (append). Negative: none.
__device__ __forceinline__ int slot_of(const Fp4RowParams &p, int t)
{
    if (p.slots)
        return p.slots[t];
    const int L = p.seq_lens[t];
    if (L <= 0 || L > p.max_blocks * kPageSize)
        return -1;
    const int page = p.block_table[(size_t)t * p.max_blocks + (L - 1) / kPageSize];
    return page < 0 || page >= p.num_pages ? -1 : page * kPageSize + (L - 1) % kPageSize;
}

// Token of a unit, unit / num_kv_heads (fewer than 2^27 units).
__device__ __forceinline__ int token_of(const Fp4RowParams &p, int unit)
{
    return p.heads_inverse ? (int)__umulhi((uint32_t)unit, p.heads_inverse)
                           : (int)((uint32_t)unit / (uint32_t)p.num_kv_heads);
}

template <int D>
__device__ __forceinline__ size_t record_at(const Fp4RowParams &p, int slot, int g)
{
    return ((size_t)(slot / kPageSize) * p.num_kv_heads + g) * Fp4Layout<D>::kBytes;
}

// ROWS rows per thread, all of their loads under way before the first store.
template <int D, int ROWS>
__global__ __launch_bounds__(kRowThreads) void fp4_store_kernel(Fp4RowParams p)
{
    const RowPart<D, ROWS> r;
    const int units = p.rows * p.num_kv_heads;
    u32x4_t x[ROWS];
    int slot[ROWS], g[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int unit = min(r.unit(i), units - 1), t = token_of(p, unit);
        g[i] = unit - t * p.num_kv_heads;
        x[i] = *reinterpret_cast<const u32x4_t *>((r.which ? p.v_rows : p.k_rows) + (size_t)unit * D + kPer * r.part);
        slot[i] = r.unit(i) < units ? slot_of(p, t) : -1;
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        if (slot[i] >= 0 && slot[i] < p.num_pages * kPageSize)
            store_part<D>(p.pages + record_at<D>(p, slot[i], g[i]), r.which, slot[i] % kPageSize, r.part, x[i]);
}

template <int D, int ROWS>
__global__ __launch_bounds__(kRowThreads) void fp4_load_kernel(Fp4RowParams p)
{
    const RowPart<D, ROWS> r;
    const int units = p.rows * p.num_kv_heads;
    int slot[ROWS], g[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int unit = min(r.unit(i), units - 1), t = token_of(p, unit);
        g[i] = unit - t * p.num_kv_heads;
        slot[i] = p.slots[t];
    }
    u32x4_t x[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const bool in = slot[i] >= 0 && slot[i] < p.num_pages * kPageSize;
        const uint32_t none = slot[i] < 0 ? 0u : 0x7fc07fc0u;
        x[i] = u32x4_t{none, none, none, none};
        if (in)
            x[i] = load_part<D>(p.pages + record_at<D>(p, slot[i], g[i]), r.which, slot[i] % kPageSize, r.part);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        if (r.unit(i) < units)
            *reinterpret_cast<u32x4_t *>((r.which ? p.v_out : p.k_out) + (size_t)r.unit(i) * D + kPer * r.part) = x[i];
}

template <int D, int ROWS>
hipError_t launch(const Fp4RowParams &p, hipStream_t stream)
{
    const long long units = (long long)p.rows * p.num_kv_heads, per = RowPart<D, ROWS>::kUnits * ROWS;
    const dim3 grid((unsigned)((units + per - 1) / per)), block(kRowThreads);
    if (p.k_rows)
        hipLaunchKernelGGL((fp4_store_kernel<D, ROWS>), grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL((fp4_load_kernel<D, ROWS>), grid, block, 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_fp4_rows(const Fp4RowParams &rows, int head_dim, hipStream_t stream)
{
    Fp4RowParams p = rows;
    // exact for units below 2^32 / heads (inverse_of(1) does not fit)
    p.heads_inverse = p.num_kv_heads > 1 && p.num_kv_heads <= 32 ? inverse_of(p.num_kv_heads) : 0;
    const bool many = (long long)p.rows * p.num_kv_heads * head_dim >= kManyRowElements;
    if (head_dim == 128)
        return many ? launch<128, kRowsPerThread>(p, stream) : launch<128, 1>(p, stream);
    if (head_dim == 64)
        return many ? launch<64, kRowsPerThread>(p, stream) : launch<64, 1>(p, stream);
    return hipErrorInvalidValue;
}

}  // namespace sl
