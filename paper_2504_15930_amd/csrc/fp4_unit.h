#ifndef SL_FP4_UNIT_H
#define SL_FP4_UNIT_H
// The 4-bit cache's record: one page-head tile (16 tokens of one KV head), its
// key rows and its value rows, 17 D bytes. Rows are cut into blocks of 32
// consecutive elements; a block is 32 E2M1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6
// with a sign) and one E8M0 scale byte s, and stands for e2m1(code) 2^(s - 127)
// (NaN where s is 255).
//
//   bytes                     what (t: token's slot, c: block, d: element)
//   0 .. 8 D                  K codes: 16 bytes per (block, token), [c][t]
//   8 D .. 16 D               V codes: [t / 4][16 runs of D / 16 elements][t % 4]
//   16 D .. 16 D + D / 2      K scales: [c][t]
//   16 D + D / 2 .. 17 D      V scales: [t / 4][c][t % 4]
// with a byte holding an even element in its low half and the next in its high
// half. The order is that of the attention's matrix operands: with lane = n +
// 16 quad, 16 bytes of K per lane (D = 128) are block `quad` of token n, and 16
// bytes of V are elements 8 n .. 8 n + 7 of tokens 4 quad .. 4 quad + 3, so both
// stream as whole 1 KB runs, the scales of the tile lie beside them, and a
// record of D = 128 is 17 whole cache lines. A token owns whole bytes of it, so
// rows are written one by one, without reading their neighbours.
#include <hip/hip_runtime.h>

#include "sl_internal.h"

namespace sl {
namespace {

template <int D>
struct Fp4Layout {
    static constexpr int kBytes = 17 * D;       // fp4_record_bytes
    static constexpr int kBlocks = D / 32;      // per row
    static constexpr int kV = 8 * D;            // first byte of the V codes
    static constexpr int kRun = D / 32;         // bytes of one token's run of D / 16 value elements
    __host__ __device__ static constexpr int k_code(int t, int block) { return 256 * block + 16 * t; }
    __host__ __device__ static constexpr int v_code(int t, int run)
    {
        return kV + 4 * kRun * (16 * (t / 4) + run) + kRun * (t % 4);
    }
    __host__ __device__ static constexpr int k_scale(int t, int block) { return 16 * D + 16 * block + t; }
    __host__ __device__ static constexpr int v_scale(int t, int block)
    {
        return 16 * D + D / 2 + 4 * (kBlocks * (t / 4) + block) + t % 4;
    }
};

// 2^(s - 127) of the scale byte s in x's low byte: as the fp32 whose exponent
// field it is (the conversion below reads 255 as NaN and 0 as 2^-127).
__device__ __forceinline__ float e8m0(uint32_t x) { return __builtin_bit_cast(float, (x & 0xffu) << 23); }

// The same of byte B of x, in one instruction. (Left to itself the compiler takes
// a shift and a mask.)
template <int B>
__device__ __forceinline__ float e8m0_byte(uint32_t x)
{
    float f;
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_%3"
        : "=v"(f)
        : "v"(23), "v"(x), "i"(B));
    return f;
}

// The two codes of byte B of x, times `scale`, as a bf16 pair (low half: the
// low code), exact.
template <int B>
__device__ __forceinline__ uint32_t fp4x2_to_bf16(uint32_t x, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, B));
}
// (for a byte that unrolling makes a constant)
__device__ __forceinline__ uint32_t fp4x2_to_bf16_at(uint32_t x, float scale, int b)
{
    return b == 0   ? fp4x2_to_bf16<0>(x, scale)
           : b == 1 ? fp4x2_to_bf16<1>(x, scale)
           : b == 2 ? fp4x2_to_bf16<2>(x, scale)
                    : fp4x2_to_bf16<3>(x, scale);
}

}  // namespace
}  // namespace sl

#endif  // SL_FP4_UNIT_H
