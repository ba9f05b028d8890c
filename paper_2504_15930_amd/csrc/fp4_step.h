#ifndef SL_FP4_STEP_H
#define SL_FP4_STEP_H
// The online softmax over tiles of a 4-bit cache (fp4_unit.h has the record):
// loads, one step of one to four tiles, and the running state.
//
// Scores as for a bf16 cache: the key codes are widened to bf16 with their
// block's power of two, exactly (v_cvt_scalef32_pk_bf16_fp4 takes two elements,
// neighbours in a row), and enter v_mfma_f32_16x16x32_bf16. (The matrix
// instruction that takes E2M1 with E8M0 scales as they are would save the
// widening, but its sums drop what lies 2^-13 below the largest product.)
//
// Values. A widening gives a pair of neighbouring elements of one token, and the
// value product sums over tokens, so its operand wants pairs of tokens of one
// element. Two forms:
//   all 16 columns (HALF false): rows 0-1 and 2-3 of a lane's four tokens are
//   interleaved by v_perm, one per operand register, as for E4M3.
//   HALF, at most eight query heads: the pair stays as it is and the product runs
//   over (token, parity of the element), 32 for a tile of 16 tokens. Columns 0-7
//   and 8-15 both stand for heads 0-7 (the query rows are loaded twice, so every
//   lane has its head's scores), the first with the weights of even elements and
//   zeros for odd ones, the others the other way round. Half of the operand is
//   zeros in place of the columns that would be empty, the permutes are gone (16
//   of some 70 vector instructions per tile of D = 128), and the accumulators are
//   half as many: unit_fp4_kernel with D = 128 has four wavefronts per SIMD in place
//   of three (114 registers, not 160). The streams have as many as without it, one with
//   D = 128 (280 and 320) and two with D = 64.
//
// The sum of the weights comes out of the matrix product too: a row of ones times
// the weights. They enter rounded to bf16 as they do the value product, so the
// normalisation cancels that rounding.
#include "fp4_unit.h"
#include "unit_ops.h"

namespace sl {
namespace {

template <int D>
struct Fp4Tile {
    static constexpr int KW = D / 32;
    static constexpr int VW = D / 32;
    uint32_t k[KW];
    uint32_t v[VW];
    uint32_t ks;   // the scale byte of the lane's key elements
    uint32_t vs;   // those of its value elements in rows 4 quad + r, byte r
};

// Issue the loads of the record at `address`: codes as operands lie in it, and the
// lane's scales. `read` false: zeros, nothing is read. (A tile that the step lacks
// is read all the same, from the step's first record: its address comes ready out
// of a lane, where an index and a size of its own would cost ten scalar
// instructions per tile.)
template <int D, int POLICY>
__device__ __forceinline__ void issue_record(Fp4Tile<D> &t, uint64_t address, bool read, int n, int quad, int lane)
{
    using L = Fp4Layout<D>;
    const __amdgpu_buffer_rsrc_t rec = buffer_of(reinterpret_cast<const void *>(address), read ? (uint32_t)L::kBytes : 0u);
    if constexpr (D == 128) {
        const u32x4_t k = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rec, 16 * lane, 0, POLICY));
        const u32x4_t v =
            __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rec, L::kV + 16 * lane, 0, POLICY));
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            t.k[c] = k[c];
            t.v[c] = v[c];
        }
    } else {   // half a block of 32 key elements per lane
        const u32x2_t k = __builtin_bit_cast(
            u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(rec, L::k_code(n, quad >> 1) + 8 * (quad & 1), 0, POLICY));
        const u32x2_t v =
            __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(rec, L::kV + 8 * lane, 0, POLICY));
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            t.k[c] = k[c];
            t.v[c] = v[c];
        }
    }
    t.ks = __builtin_amdgcn_raw_buffer_load_b8(rec, L::k_scale(n, D == 128 ? quad : quad >> 1), 0, POLICY);
    t.vs = __builtin_bit_cast(
        uint32_t, __builtin_amdgcn_raw_buffer_load_b32(rec, L::v_scale(4 * quad, n * (D / 16) / 32), 0, POLICY));
}

// Score-MFMA A operand of k-step s: dword s of the lane's codes.
template <int D>
__device__ __forceinline__ bf16x8_t k_operand(const Fp4Tile<D> &t, float scale, int s)
{
    return __builtin_bit_cast(bf16x8_t, u32x4_t{fp4x2_to_bf16<0>(t.k[s], scale), fp4x2_to_bf16<1>(t.k[s], scale),
                                                fp4x2_to_bf16<2>(t.k[s], scale), fp4x2_to_bf16<3>(t.k[s], scale)});
}

// Elements 2c and 2c + 1 of row r (of the lane's four tokens).
template <int D>
__device__ __forceinline__ uint32_t v_pair(const Fp4Tile<D> &t, int r, int c, float scale)
{
    return D == 128 ? fp4x2_to_bf16_at(t.v[r], scale, c) : fp4x2_to_bf16_at(t.v[r / 2], scale, 2 * (r % 2) + c);
}

// A unit's running state. acc[i], not HALF: as Piece's. HALF: acc[c] of lane
// (n, quad) holds elements 2c + n / 8 of the runs 4 quad + r of head n % 8.
template <int D, bool HALF>
struct Fp4State {
    f32x4_t acc[HALF ? D / 32 : D / 16];
    f32x4_t l;   // the head's sum of weights, four times
    float m;
    float ref;   // what a step's exponents are first taken against: m, or kBelowAll where |m| >= kWideScore
};

// An exponent in one fma, the exact product of score and factor minus m, has m's own
// rounding error in it, since m is a rounded product: half a unit of its last place.
// Below 2^24 that is at most half a binary order for all tokens alike, and cancels;
// from 2^31 on it is 2^7 and more, and every weight would overflow or vanish. From
// 2^24 on the product is therefore rounded before the subtraction. Such scores are
// rare: a step meets them by comparing against kBelowAll, which no score is below and
// so always sends it where the maximum is raised, and the step has no other branch.
constexpr float kWideScore = 16777216.0f;
constexpr float kBelowAll = -3.4028234663852886e38f;

template <int D, bool HALF>
__device__ __forceinline__ void reset(Fp4State<D, HALF> &st)
{
#pragma unroll
    for (f32x4_t &a : st.acc)
        a = f32x4_t{0.f, 0.f, 0.f, 0.f};
    st.l = f32x4_t{0.f, 0.f, 0.f, 0.f};
    st.m = st.ref = kNegInf;
}

template <int D, bool HALF>
__device__ __forceinline__ Piece<D> finished(const Fp4State<D, HALF> &st, int quad)
{
    Piece<D> out;
    if constexpr (HALF) {   // lanes n < 8 fetch the odd elements from n + 8 (row_ror:8)
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                out.acc[2 * c][r] = st.acc[c][r];
                out.acc[2 * c + 1][r] = lane_from<0x128, 0xf>(st.acc[c][r], 0.0f);
            }
    } else {
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
            out.acc[i] = st.acc[i];
    }
    out.m = st.m;
    out.l = quad == 0 ? st.l[0] : 0.0f;   // (the epilogues add the four quads up)
    return out;
}

// Scores are q . k times |scale|; a negative one turns the query's signs.
__device__ __forceinline__ uint32_t fp4_sign(float scale) { return scale < 0.0f ? 0x80008000u : 0u; }

// One step over the first NT tiles; `valid` = live tokens of the step, 1 .. 16 NT
// (any number with NT > 1 where the first tile has one). mul = |scale| log2(e).
template <int D, int NT, bool HALF, class T, int N>
__device__ __forceinline__ void fp4_step(Fp4State<D, HALF> &st, const T (&t)[N], const bf16x8_t (&qop)[D / 32], float mul,
                                         int valid, int n, int quad)
{
    static_assert(HALF || NT == 1 || NT % 2 == 0, "one tile, or pairs of tiles, per step");
    const bool partial = valid < kPageSize * NT;
    auto dead = [&](int u, int r) { return kPageSize * u + 4 * quad + r >= valid; };
    // In a step of four tiles the compiler makes two copies of the code by itself; in
    // a smaller one it keeps the masks under branches, and their comparisons, if it
    // can, before them, in every step. There every branch has its own `valid`. (Two
    // copies written out took 170 registers for 110 in unit_fp4_kernel of D = 128:
    // 512 x 1..256 tokens, 64/8 heads, 26 -> 35 us.)
    constexpr bool kBranches = NT < 4;
    auto own = [&](int v) {
        if (kBranches)
            asm volatile("" : "+s"(v));
        return v;
    };
    f32x4_t s4[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u)
        s4[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int u = 0; u < NT; ++u)
            s4[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k_operand<D>(t[u], e8m0(t[u].ks), s), qop[s], s4[u],
                                                            0, 0, 0);
    // Exponents relative to the running maximum as it is: |scale| log2(e) and the
    // subtraction in one fma. They show whether the maximum has to be raised, which
    // compute_step asks of the scaled scores; then they are formed again, for large
    // scores in two roundings (kWideScore).
    // (Every score is read here, before any branch: this compiler has let a branch
    // over a few instructions lead from a matrix product to the first reader of its
    // result without the wait states in between.)
    float x[NT][4];
    auto exponents = [&](const auto &y, float factor, float from) {
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                x[u][r] = __builtin_fmaf(y[u][r], factor, -from);
    };
    auto mask = [&](auto &y) {
        if (partial) {
            const int live = own(valid) - 4 * quad;
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    y[u][r] = kPageSize * u + r >= live ? kNegInf : y[u][r];
        }
    };
    auto largest = [&](const auto &y) {
        float top = fmaxf(fmaxf(y[0][0], y[0][1]), fmaxf(y[0][2], y[0][3]));
#pragma unroll
        for (int u = 1; u < NT; ++u)
            top = fmaxf(top, fmaxf(fmaxf(y[u][0], y[u][1]), fmaxf(y[u][2], y[u][3])));
        return top;
    };
    // (An instruction written out: out of a branch the compiler first makes every value canonical.)
    auto largest_of = [&](const float(&y)[NT][4]) {
        auto max3 = [](float a, float b, float c) {
            float top;
            asm("v_max3_f32 %0, %1, %2, %3" : "=v"(top) : "v"(a), "v"(b), "v"(c));
            return top;
        };
        float top = y[0][0];
#pragma unroll
        for (int i = 1; i < 4 * NT; i += 2)
            top = max3(top, y[i / 4][i % 4], i + 1 < 4 * NT ? y[(i + 1) / 4][(i + 1) % 4] : y[i / 4][i % 4]);
        return top;
    };
    exponents(s4, mul, st.ref);
    mask(x);
    if (__builtin_amdgcn_ballot_w64(largest_of(x) > kRescaleSlack) != 0) {
        mask(s4);
        const float mx = quad_max(largest(s4) * mul);
        if (mx > st.m + kRescaleSlack) {
            const float alpha = __builtin_amdgcn_exp2f(st.m - mx);   // 0 on a unit's first tile
#pragma unroll
            for (f32x4_t &a : st.acc)
                a *= alpha;
            st.l *= alpha;
            st.m = mx;
            st.ref = __builtin_fabsf(mx) < kWideScore ? mx : kBelowAll;
        }
        float factor = mul;
        const bool wide = st.ref != st.m;
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(wide) != 0, 0)) {
            factor = wide ? 1.0f : mul;
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    s4[u][r] = wide ? s4[u][r] * mul : s4[u][r];
        }
        exponents(s4, factor, st.m);
        mask(x);   // (a factor of zero made a masked score's NaN)
    }
    float p[NT][4];
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            p[u][r] = __builtin_amdgcn_exp2f(x[u][r]);
    // A dead token's codes are finite, its scale need not be: 1 in its place, by a
    // selection, or a byte put into the scales before.
    uint32_t vs[NT];
    if (kBranches) {
#pragma unroll
        for (int u = 0; u < NT; ++u)
            vs[u] = t[u].vs;
        if (partial) {
            const int live = own(valid) - 4 * quad;
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    vs[u] = kPageSize * u + r >= live ? (vs[u] & ~(0xffu << 8 * r)) | 127u << 8 * r : vs[u];
        }
    }
    auto v_scale = [&](int u, int r) {
        const uint32_t from = kBranches ? vs[u] : t[u].vs;
        const float s = r == 0   ? e8m0_byte<0>(from)
                        : r == 1 ? e8m0_byte<1>(from)
                        : r == 2 ? e8m0_byte<2>(from)
                                 : e8m0_byte<3>(from);
        return !kBranches && partial && dead(u, r) ? 1.0f : s;
    };
    constexpr uint32_t kOnes = 0x3f803f80u;
    const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, u32x4_t{kOnes, kOnes, kOnes, kOnes});
    if constexpr (HALF) {
        // v_perm selectors: a weight alone in the low half (even elements' columns) or the high one.
        const uint32_t first = n < 8 ? 0x0c0c0100u : 0x01000c0cu, second = n < 8 ? 0x0c0c0302u : 0x03020c0cu;
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const uint32_t p01 = pack_bf16(p[u][0], p[u][1]), p23 = pack_bf16(p[u][2], p[u][3]);
            const bf16x8_t b = __builtin_bit_cast(
                bf16x8_t, u32x4_t{__builtin_amdgcn_perm(0u, p01, first), __builtin_amdgcn_perm(0u, p01, second),
                                  __builtin_amdgcn_perm(0u, p23, first), __builtin_amdgcn_perm(0u, p23, second)});
            st.l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, b, st.l, 0, 0, 0);
            float scale[4];
#pragma unroll
            for (int r = 0; r < 4; ++r)
                scale[r] = v_scale(u, r);
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t a[4];
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    a[r] = v_pair<D>(t[u], r, c, scale[r]);
                st.acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8_t, u32x4_t{a[0], a[1], a[2], a[3]}), b, st.acc[c], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int u0 = 0; u0 < NT; u0 += 2) {   // two tiles in one product where there are two
            constexpr int P = NT == 1 ? 1 : 2;
            uint32_t w[4] = {0u, 0u, 0u, 0u};
            float scale[P][4];
#pragma unroll
            for (int k = 0; k < P; ++k) {
                w[2 * k] = pack_bf16(p[u0 + k][0], p[u0 + k][1]);
                w[2 * k + 1] = pack_bf16(p[u0 + k][2], p[u0 + k][3]);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    scale[k][r] = v_scale(u0 + k, r);
            }
            auto add = [&](f32x4_t &acc, const uint32_t (&a)[4]) {
                if constexpr (P == 1)
                    acc = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(i16x4_t, u32x2_t{a[0], a[1]}),
                                                                    __builtin_bit_cast(i16x4_t, u32x2_t{w[0], w[1]}),
                                                                    acc, 0, 0, 0);
                else
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8_t, u32x4_t{a[0], a[1], a[2], a[3]}),
                        __builtin_bit_cast(bf16x8_t, u32x4_t{w[0], w[1], w[2], w[3]}), acc, 0, 0, 0);
            };
            const uint32_t one[4] = {kOnes, kOnes, kOnes, kOnes};
            add(st.l, one);
#pragma unroll
            for (int i = 0; i < D / 16; i += 2) {
                uint32_t a0[4], a1[4];   // operands of elements i and i + 1
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    uint32_t x[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        x[r] = v_pair<D>(t[u0 + k], r, i / 2, scale[k][r]);
                    a0[2 * k] = __builtin_amdgcn_perm(x[1], x[0], 0x05040100u);
                    a1[2 * k] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);
                    a0[2 * k + 1] = __builtin_amdgcn_perm(x[3], x[2], 0x05040100u);
                    a1[2 * k + 1] = __builtin_amdgcn_perm(x[3], x[2], 0x07060302u);
                }
                add(st.acc[i], a0);
                add(st.acc[i + 1], a1);
            }
        }
    }
}

}  // namespace
}  // namespace sl

#endif  // SL_FP4_STEP_H
