// Device side of the 4-bit layers: one wavefront's walk over units of 16 rows and 128 kept columns.
//
//   acc[row][n] += scale[row][g] * ( sum_c (code[row][c] - 8) x[n][c]  -  (zero[row][g] - 8) sum_c x[n][c] )
//
// over the columns c of each scale group g.  The code less 8 is exact in fp16 and in 8 bits, the products of a group are
// summed by the matrix cores in fp32 (int32 for 8-bit inputs, exact), and the scale multiplies the finished sum: no
// weight is ever rounded.  The second sum, for layers with zero points, is a matrix product with ones, which leaves it in
// the accumulator's own layout.  Groups do not cross units.
//
// A unit's columns of x are staged in LDS by the wavefront that multiplies them (16 bytes per lane), so the wavefronts of
// a workgroup need no barrier until their sums meet.
#pragma once

#include <type_traits>

#include "pivot_device.h"
#include "pivot_quant.h"

namespace pivot {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int   i32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef signed char i8x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// A load that is known to go to device memory: pointers that come out of tables in memory or LDS would otherwise be
// followed by the slower loads that also ask LDS.
template <typename V>
__device__ __forceinline__ V gload(const void* p) {
    return *(const __attribute__((address_space(1))) V*)p;
}

// Eight codes of a word, less 8, as fp16: a nibble put into the mantissa of 1024 (of 64 * 16, for the second nibble of a
// byte) is an exact integer, and one packed operation takes off the offset.  9 operations for 8 weights.
__device__ __forceinline__ f16x8 q_dequant(uint32_t w) {
    const uint32_t v = w >> 8;
    const f16x2 c0 = {(_Float16)-1032.f, (_Float16)-1032.f}, c1 = {(_Float16)-72.f, (_Float16)-72.f},
                r = {(_Float16)0.0625f, (_Float16)0.0625f};
    const f16x2 a = __builtin_bit_cast(f16x2, (w & 0x000f000fu) | 0x64006400u) + c0;
    const f16x2 b = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (w & 0x00f000f0u) | 0x64006400u), r, c1);
    const f16x2 c = __builtin_bit_cast(f16x2, (v & 0x000f000fu) | 0x64006400u) + c0;
    const f16x2 d = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v & 0x00f000f0u) | 0x64006400u), r, c1);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// ... and as 8-bit integers, times 16: the code less 8 is the code's nibble with its top bit turned over, in two's
// complement, and in the upper half of a byte it needs no sign extension.
__device__ __forceinline__ i32x2 q_dequant8(uint32_t w) {
    const uint32_t s = w ^ 0x88888888u;
    return i32x2{(int)((s << 4) & 0xf0f0f0f0u), (int)(s & 0xf0f0f0f0u)};
}

// Rows of x as a kernel's launch gives them.
struct QSource {
    const void* x; long long ld; const int32_t* pcol; int K; int vec;   // pcol NULL: columns as they lie; vec: 16-byte (8-byte) pieces may be loaded whole
};

template <bool Q8> struct QElem { typedef _Float16 type; static constexpr int kBytes = 2, kRow = kQBlk * 2 + 16; };
template <> struct QElem<true>  { typedef int8_t type;   static constexpr int kBytes = 1, kRow = kQBlk + 16; };

// Eight columns of x, block-space columns col..col+7 of one row.  idx: their natural columns (pcol given).
template <bool Q8>
__device__ __forceinline__ void q_load8(const QSource& s, long long row, int col, const i32x4 (&idx)[2], typename QElem<Q8>::type (&v)[8]) {
    typedef typename QElem<Q8>::type E;
    const E* p = reinterpret_cast<const E*>(s.x) + row * s.ld;
    if (s.pcol) {
        #pragma unroll
        for (int i = 0; i < 8; ++i) { const int c = idx[i >> 2][i & 3]; v[i] = c >= 0 ? gload<E>(p + c) : E(0); }
    } else if (s.vec && col + 8 <= s.K) {
        if (Q8) *reinterpret_cast<u32x2*>(v) = gload<u32x2>(p + col);
        else    *reinterpret_cast<u32x4*>(v) = gload<u32x4>(p + col);
    } else {
        #pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < s.K ? gload<E>(p + col + i) : E(0);
    }
}

// Stores eight staged columns (8 * c8 .. of the unit) at `row`: fp16 as they are, 8-bit in nibble order.
template <bool Q8>
__device__ __forceinline__ void q_store8(char* row, int c8, const typename QElem<Q8>::type (&v)[8]) {
    if (Q8) {
        union { int8_t b[8]; u32x2 u; } o;
        #pragma unroll
        for (int i = 0; i < 8; ++i) o.b[2 * (i & 3) + (i >> 2)] = (int8_t)v[i];
        *reinterpret_cast<u32x2*>(row + q_byte_pos(8 * c8)) = o.u;
    } else {
        *reinterpret_cast<u32x4*>(row + 16 * c8) = *reinterpret_cast<const u32x4*>(v);
    }
}

// Codes and scales of one unit, per lane.
template <int GPK, bool ZP>
struct QUnit {
    u32x4 w; f16x4 s[GPK]; i8x4 z[ZP ? GPK : 1];
    __device__ __forceinline__ void load(const u32x4* codes, const uint16_t* scales, const int8_t* zoff, size_t unit, int lane) {
        w = gload<u32x4>(codes + unit * 64 + lane);
        #pragma unroll
        for (int g = 0; g < GPK; ++g) {
            const size_t at = (unit * GPK + g) * kQStrip + 4 * (lane >> 4);
            s[g] = gload<f16x4>(scales + at);
            if (ZP) z[g] = gload<i8x4>(zoff + at);
        }
    }
};

// One unit times NT * 16 rows of x staged at `xs` (rows of QElem::kRow bytes).  nrow[t]: byte offset of this lane's row in
// column tile t.  Q8 inputs come out 16 times too large (the caller scales).
template <bool Q8, int GPK, bool ZP, int NT, int RS>
__device__ __forceinline__ void q_multiply(const QUnit<GPK, ZP> (&u)[RS], const char* xs, const int (&nrow)[NT], int lane, f32x4 (&acc)[RS][NT]) {
    typedef typename std::conditional<Q8, i32x4, f32x4>::type part_t;
    const int kg = lane >> 4;
    #pragma unroll
    for (int g = 0; g < GPK; ++g) {
        part_t part[RS][NT] = {}, sum[NT] = {};
        constexpr int SPG = 4 / GPK;    // 32-column steps per group
        if (!Q8) {
            #pragma unroll
            for (int j = g * SPG; j < (g + 1) * SPG; ++j) {
                f16x8 a[RS];
                #pragma unroll
                for (int r = 0; r < RS; ++r) a[r] = q_dequant(u[r].w[j]);
                #pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const f16x8 b = *reinterpret_cast<const f16x8*>(xs + nrow[t] + 64 * j + 16 * kg);
                    #pragma unroll
                    for (int r = 0; r < RS; ++r) part[r][t] = __builtin_bit_cast(part_t, __builtin_amdgcn_mfma_f32_16x16x32_f16(a[r], b, __builtin_bit_cast(f32x4, part[r][t]), 0, 0, 0));
                    if (ZP) {
                        const _Float16 o = (_Float16)1.f;
                        sum[t] = __builtin_bit_cast(part_t, __builtin_amdgcn_mfma_f32_16x16x32_f16(f16x8{o, o, o, o, o, o, o, o}, b, __builtin_bit_cast(f32x4, sum[t]), 0, 0, 0));
                    }
                }
            }
        } else if (GPK == 4) {
            i32x2 a[RS];
            #pragma unroll
            for (int r = 0; r < RS; ++r) a[r] = q_dequant8(u[r].w[g]);
            #pragma unroll
            for (int t = 0; t < NT; ++t) {
                const long b = *reinterpret_cast<const long*>(xs + nrow[t] + 64 * (g >> 1) + 16 * kg + 8 * (g & 1));
                #pragma unroll
                for (int r = 0; r < RS; ++r) part[r][t] = __builtin_bit_cast(part_t, __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a[r]), b, __builtin_bit_cast(i32x4, part[r][t]), 0, 0, 0));
                if (ZP) sum[t] = __builtin_bit_cast(part_t, __builtin_amdgcn_mfma_i32_16x16x32_i8(0x0101010101010101L, b, __builtin_bit_cast(i32x4, sum[t]), 0, 0, 0));
            }
        } else {
            #pragma unroll
            for (int m = g * SPG / 2; m < (g + 1) * SPG / 2; ++m) {
                i32x4 a[RS];
                #pragma unroll
                for (int r = 0; r < RS; ++r) {
                    const i32x2 lo = q_dequant8(u[r].w[2 * m]), hi = q_dequant8(u[r].w[2 * m + 1]);
                    a[r] = i32x4{lo[0], lo[1], hi[0], hi[1]};
                }
                #pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const i32x4 b = *reinterpret_cast<const i32x4*>(xs + nrow[t] + 64 * m + 16 * kg);
                    #pragma unroll
                    for (int r = 0; r < RS; ++r) part[r][t] = __builtin_bit_cast(part_t, __builtin_amdgcn_mfma_i32_16x16x64_i8(a[r], b, __builtin_bit_cast(i32x4, part[r][t]), 0, 0, 0));
                    if (ZP) { const int o = 0x01010101; sum[t] = __builtin_bit_cast(part_t, __builtin_amdgcn_mfma_i32_16x16x64_i8(i32x4{o, o, o, o}, b, __builtin_bit_cast(i32x4, sum[t]), 0, 0, 0)); }
                }
            }
        }
        #pragma unroll
        for (int r = 0; r < RS; ++r)
            #pragma unroll
            for (int t = 0; t < NT; ++t)
                #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float p;
                    if (ZP) p = Q8 ? (float)((int)part[r][t][i] - 16 * (int)u[r].z[g][i] * (int)sum[t][i]) : (float)part[r][t][i] - (float)u[r].z[g][i] * (float)sum[t][i];
                    else    p = (float)part[r][t][i];
                    acc[r][t][i] = __builtin_fmaf((float)u[r].s[g][i], p, acc[r][t][i]);
                }
    }
}

}  // namespace pivot
