#ifndef SL_UNIT_OPS_H
#define SL_UNIT_OPS_H
// What the decode workers share whatever the cache holds: operand types, the
// softmax state of a unit, cross-lane steps, buffer resources.
#include "sl_internal.h"
#include "wave_ops.h"

namespace sl {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_inff();
// A partial state l = sum 2^(s - m), acc = sum 2^(s - m) v is exact for any
// reference m. The running maximum is raised only when a score exceeds it by
// more than this slack (base-2 units), which bounds the weights by 2^8 and
// leaves the accumulators untouched on most tiles after a unit's first.
constexpr float kRescaleSlack = 8.0f;
constexpr int kRawBufferWord3 = 0x00020000;  // untyped 32-bit buffer resource (CDNA3/4)

// Two fp32 -> packed bf16 pair, round to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    f32x2_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

// Max / sum over the lanes n, n + 16, n + 32, n + 48 of a column.
// (The gfx950 lane-swap builtins would avoid the LDS crossbar here, but this
// compiler folds max(h[0], h[1]) of their two results to one of them, so the
// plain shuffles are used.)
__device__ __forceinline__ float quad_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16, kWave));
    return fmaxf(x, __shfl_xor(x, 32, kWave));
}
__device__ __forceinline__ float quad_sum(float x)
{
    x += __shfl_xor(x, 16, kWave);
    return x + __shfl_xor(x, 32, kWave);
}

// K/V pages are read exactly once per call: stream them with non-temporal loads
// so they do not displace reusable lines in L2 / the Infinity Cache (measured on
// MI355X: random 4 KB tiles reach ~6.8 TB/s this way, ~6.0 TB/s with plain loads).
constexpr int kCachePolicyStream = 2;   // NT

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *base, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, kRawBufferWord3);
}

template <int D>
struct Piece {
    f32x4_t acc[D / 16];
    float m;   // running max of this lane's head, base-2 units
    float l;   // this lane's share of the sum of (bf16-rounded) weights
};

template <int D>
__device__ __forceinline__ void reset(Piece<D> &st)
{
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
        st.acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    st.m = kNegInf;
    st.l = 0.f;
}

// The state as the epilogues take it.
template <int D>
__device__ __forceinline__ Piece<D> &finished(Piece<D> &st, int)
{
    return st;
}

}  // namespace
}  // namespace sl

#endif  // SL_UNIT_OPS_H
