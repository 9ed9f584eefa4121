// Device side of the 4-bit layers: one wavefront's walk over units of 16 rows and 128 kept columns.
//
//   acc[row][n] += scale[row][g] * sum_c (code[row][c] - zero[row][g]) x[n][c]       over the columns c of each scale group g
//
// The code less its zero point is exact in fp16 and in 8 bits, the products of a group are summed by the matrix cores in
// fp32 (int32 for 8-bit inputs, exact), and the scale multiplies the finished sum: no weight is ever rounded.  Groups do
// not cross units.
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
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// A load that is known to go to device memory: pointers that come out of tables in memory or LDS would otherwise be
// followed by the slower loads that also ask LDS.
template <typename V>
__device__ __forceinline__ V gload(const void* p) {
    return *(const __attribute__((address_space(1))) V*)p;
}

// ... at a byte offset per lane from an address that is the same for all of them: held in scalar registers.
template <typename V>
__device__ __forceinline__ V gload(const void* base, uint32_t offset) {
    return *(const __attribute__((address_space(1))) V*)((const __attribute__((address_space(1))) char*)base + offset);
}

// The number of this wavefront in its workgroup, known to be the same in all its lanes.
__device__ __forceinline__ int q_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// The zero point of a row's group, as the two forms of dequantisation take it off.
struct QZero16 { f16x2 near, far; };    // of codes put into the mantissa of 1024, of 64 * 16
__device__ __forceinline__ QZero16 q_zero16(uint32_t z) {
    const f16x2 v = __builtin_bit_cast(f16x2, (z | (z << 16)) | 0x64006400u);             // 1024 + z
    const _Float16 o = (_Float16)960.f;
    return QZero16{-v, f16x2{o, o} - v};                                                  // -(1024 + z), -(64 + z)
}

// Eight codes of a word less their zero point, as fp16: a nibble put into the mantissa of 1024 (of 64 * 16, for the second
// nibble of a byte) is an exact integer, and one packed operation takes off the offset with the zero point.  9 operations
// for 8 weights.
__device__ __forceinline__ f16x8 q_dequant(uint32_t w, const QZero16& z) {
    const uint32_t v = w >> 8;
    const f16x2 r = {(_Float16)0.0625f, (_Float16)0.0625f};
    const f16x2 a = __builtin_bit_cast(f16x2, (w & 0x000f000fu) | 0x64006400u) + z.near;
    const f16x2 b = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (w & 0x00f000f0u) | 0x64006400u), r, z.far);
    const f16x2 c = __builtin_bit_cast(f16x2, (v & 0x000f000fu) | 0x64006400u) + z.near;
    const f16x2 d = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v & 0x00f000f0u) | 0x64006400u), r, z.far);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// ... as 8-bit integers.  Without zero points they come out times 16 (kQ8Factor puts that right): the code less 8 is the
// nibble with its top bit turned over, in two's complement, and in the upper half of a byte it needs no sign extension.
// With them, 128 + code less the zero point never borrows from the next byte.
template <bool ZP> constexpr float kQ8Factor = ZP ? 1.f : 0.0625f;
template <bool ZP>
__device__ __forceinline__ i32x2 q_dequant8(uint32_t w, uint32_t zzzz) {
    if (ZP) {
        const uint32_t lo = ((w & 0x0f0f0f0fu) | 0x80808080u) - zzzz, hi = (((w >> 4) & 0x0f0f0f0fu) | 0x80808080u) - zzzz;
        return i32x2{(int)(lo ^ 0x80808080u), (int)(hi ^ 0x80808080u)};
    }
    const uint32_t s = w ^ 0x88888888u;
    return i32x2{(int)((s << 4) & 0xf0f0f0f0u), (int)(s & 0xf0f0f0f0u)};
}

// Rows of x as a kernel's launch gives them.
struct QSource {
    const void* x; long long ld; const int32_t* pcol; int K; int vec;   // pcol NULL: columns as they lie; vec: 16-byte (8-byte) pieces may be loaded whole
};

template <bool Q8> struct QElem { typedef _Float16 type; static constexpr int kBytes = 2, kRow = kQBlk * 2 + 16; };
template <> struct QElem<true>  { typedef int8_t type;   static constexpr int kBytes = 1, kRow = kQBlk + 16; };

// Eight columns of x, block-space columns col..col+7 of one row, as they lie.  idx: their natural columns (pcol given).
template <bool Q8> using q_eight = typename std::conditional<Q8, u32x2, u32x4>::type;
template <bool Q8>
__device__ __forceinline__ q_eight<Q8> q_load8(const QSource& s, long long row, int col, const i32x4 (&idx)[2]) {
    typedef typename QElem<Q8>::type E;
    const E* p = reinterpret_cast<const E*>(s.x) + row * s.ld;
    if (!s.pcol && s.vec && col + 8 <= s.K) return gload<q_eight<Q8>>(p + col);
    union { E v[8]; q_eight<Q8> u; } o;
    #pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = s.pcol ? idx[i >> 2][i & 3] : (col + i < s.K ? col + i : -1);
        o.v[i] = c >= 0 ? gload<E>(p + c) : E(0);
    }
    return o.u;
}

// Eight 8-bit values in nibble order: columns 0,4,1,5 and 2,6,3,7.
__device__ __forceinline__ u32x2 q_nibble_order(u32x2 v) {
    return u32x2{__builtin_amdgcn_perm(v[1], v[0], 0x05010400u), __builtin_amdgcn_perm(v[1], v[0], 0x07030602u)};
}

// Stores eight staged columns (8 * c8 .. of the unit) at `row`: fp16 as they are, 8-bit in nibble order.
template <bool Q8>
__device__ __forceinline__ void q_store8(char* row, int c8, q_eight<Q8> v) {
    if constexpr (Q8) *reinterpret_cast<u32x2*>(row + q_byte_pos(8 * c8)) = q_nibble_order(v);
    else *reinterpret_cast<u32x4*>(row + 16 * c8) = v;
}

// Codes, scales and zero points of one unit, per lane: the scales of the four rows that the lane's accumulators are, the
// zero points of the row whose codes it holds (a byte per group).
template <int GPK, bool ZP>
struct QUnit {
    u32x4 w; f16x4 s[GPK]; uint32_t z;
    __device__ __forceinline__ void load(const u32x4* codes, const uint16_t* scales, const uint8_t* zeros, size_t unit, uint32_t lane) {
        w = gload<u32x4>(codes + unit * 64, lane * 16);
        const uint16_t* sp = scales + unit * (kQStrip * GPK);
        const uint32_t so = (lane >> 4) * (8 * GPK);
        if constexpr (GPK == 1) s[0] = gload<f16x4>(sp, so);
        else {
            #pragma unroll
            for (int g = 0; g < GPK; g += 2) {
                const f16x8 v = gload<f16x8>(sp, so + 8 * g);
                s[g] = f16x4{v[0], v[1], v[2], v[3]};
                s[g + 1] = f16x4{v[4], v[5], v[6], v[7]};
            }
        }
        if constexpr (ZP) {
            const uint8_t* zp = zeros + unit * (kQStrip * GPK);
            const uint32_t zo = (lane & 15) * GPK;
            if constexpr (GPK == 1) z = gload<uint8_t>(zp, zo);
            else if constexpr (GPK == 2) z = gload<uint16_t>(zp, zo);
            else z = gload<uint32_t>(zp, zo);
        }
    }
    __device__ __forceinline__ uint32_t zero(int g) const { return ZP ? (z >> (8 * g)) & 255u : 8u; }
};

// Where the matrix instructions take x from.  Staged in LDS: rows of QElem::kRow bytes.  f16(t, j): columns 32 j .. of
// column tile t; q64(t, m): columns 64 m ..; q32(t, j): columns 32 j ...
template <bool Q8, int NT>
struct QRows {
    const char* xs; const int (&nrow)[NT]; int lane;      // nrow[t]: byte offset of this lane's row in column tile t
    __device__ __forceinline__ f16x8 f16(int t, int j) const { return *reinterpret_cast<const f16x8*>(xs + nrow[t] + 64 * j + 16 * (lane >> 4)); }
    __device__ __forceinline__ i32x4 q64(int t, int m) const { return *reinterpret_cast<const i32x4*>(xs + nrow[t] + 64 * m + 16 * (lane >> 4)); }
    __device__ __forceinline__ long  q32(int t, int j) const { return *reinterpret_cast<const long*>(xs + nrow[t] + 64 * (j >> 1) + 16 * (lane >> 4) + 8 * (j & 1)); }
};
// In registers, from the fragment-order copy of x: chunks of 32 columns, in each the batch rows side by side, their eight
// columns per lane group in order (8 bits: in nibble order).
template <bool Q8, int NT>
struct QFrag {
    typename std::conditional<Q8, u32x2, u32x4>::type v[NT][4];
    __device__ __forceinline__ void load(const char* chunk, const int (&at)[NT], int j) {
        #pragma unroll
        for (int t = 0; t < NT; ++t) v[t][j] = gload<typename std::conditional<Q8, u32x2, u32x4>::type>(chunk, at[t]);
    }
    __device__ __forceinline__ f16x8 f16(int t, int j) const { if constexpr (!Q8) return __builtin_bit_cast(f16x8, v[t][j]); else return f16x8{}; }
    __device__ __forceinline__ i32x4 q64(int t, int m) const { if constexpr (Q8) return i32x4{(int)v[t][2 * m][0], (int)v[t][2 * m][1], (int)v[t][2 * m + 1][0], (int)v[t][2 * m + 1][1]}; else return i32x4{}; }
    __device__ __forceinline__ long  q32(int t, int j) const { if constexpr (Q8) return __builtin_bit_cast(long, v[t][j]); else return 0; }
};

// RS units of the same columns times NT * 16 rows of x.  Q8 inputs come out 1 / kQ8Factor times too large.
template <bool Q8, int GPK, bool ZP, int NT, int RS, typename X>
__device__ __forceinline__ void q_multiply(const QUnit<GPK, ZP> (&u)[RS], const X& x, f32x4 (&acc)[RS][NT]) {
    typedef typename std::conditional<Q8, i32x4, f32x4>::type part_t;
    #pragma unroll
    for (int g = 0; g < GPK; ++g) {
        part_t part[RS][NT] = {};
        constexpr int SPG = 4 / GPK;    // 32-column steps per group
        if constexpr (!Q8) {
            QZero16 z[RS];
            #pragma unroll
            for (int r = 0; r < RS; ++r) z[r] = q_zero16(u[r].zero(g));
            #pragma unroll
            for (int j = g * SPG; j < (g + 1) * SPG; ++j) {
                f16x8 a[RS];
                #pragma unroll
                for (int r = 0; r < RS; ++r) a[r] = q_dequant(u[r].w[j], z[r]);
                #pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const f16x8 b = x.f16(t, j);
                    #pragma unroll
                    for (int r = 0; r < RS; ++r) part[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[r], b, part[r][t], 0, 0, 0);
                }
            }
        } else {
            uint32_t zzzz[RS];
            #pragma unroll
            for (int r = 0; r < RS; ++r) zzzz[r] = u[r].zero(g) * 0x01010101u;
            if constexpr (GPK == 4) {
                i32x2 a[RS];
                #pragma unroll
                for (int r = 0; r < RS; ++r) a[r] = q_dequant8<ZP>(u[r].w[g], zzzz[r]);
                #pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const long b = x.q32(t, g);
                    #pragma unroll
                    for (int r = 0; r < RS; ++r) part[r][t] = __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a[r]), b, part[r][t], 0, 0, 0);
                }
            } else {
                #pragma unroll
                for (int m = g * SPG / 2; m < (g + 1) * SPG / 2; ++m) {
                    i32x4 a[RS];
                    #pragma unroll
                    for (int r = 0; r < RS; ++r) {
                        const i32x2 lo = q_dequant8<ZP>(u[r].w[2 * m], zzzz[r]), hi = q_dequant8<ZP>(u[r].w[2 * m + 1], zzzz[r]);
                        a[r] = i32x4{lo[0], lo[1], hi[0], hi[1]};
                    }
                    #pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const i32x4 b = x.q64(t, m);
                        #pragma unroll
                        for (int r = 0; r < RS; ++r) part[r][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[r], b, part[r][t], 0, 0, 0);
                    }
                }
            }
        }
        #pragma unroll
        for (int r = 0; r < RS; ++r)
            #pragma unroll
            for (int t = 0; t < NT; ++t)
                #pragma unroll
                for (int i = 0; i < 4; ++i) acc[r][t][i] = __builtin_fmaf((float)u[r].s[g][i], (float)part[r][t][i], acc[r][t][i]);
    }
}

// What a wavefront of the rows forms walks over: blocks kb, kb + W, ... below kb1 of a block row (numbered from its first);
// unit of block kb and strip r: unit0 + r * nkb + kb.  pieces NULL: every tile is kept.
struct QWalk {
    const u32x4* codes; const uint16_t* scales; const uint8_t* zeros; const int32_t* pieces;
    size_t unit0; int nkb, kb, kb1, bw_log2;
};

// The rows forms' loop: a turn is two units, two blocks of one strip or one block of two strips (RS = 2).  Sixteen lanes
// take the columns of a block, eight each; the groups of sixteen that a block has take its rows of x in turn.  FAST: x is
// read as it lies in whole pieces of eight columns (no gather, K a multiple of 8, aligned rows).  Then, while a turn is
// multiplied, the next one's codes, scales and first four rows of x are on their way: every load of a turn is issued
// whatever the sizes (past the end the last block's, once more), since behind a load that may or may not have been issued
// the compiler can only wait for all of them.
template <bool Q8, int GPK, bool ZP, int RS, bool FAST, int W, typename Row>
__device__ __forceinline__ void q_walk_rows(const QWalk& k, const QSource& x, int rows, Row row_of, char* xs, f32x4 (&acc)[RS][1]) {
    typedef typename QElem<Q8>::type E;
    constexpr int P = 2 / RS, ROW = QElem<Q8>::kRow, STEP = W * P, G = 4 / P, AHEAD = FAST ? 4 / G : 0;
    struct Turn { QUnit<GPK, ZP> u[P][RS]; q_eight<Q8> v[2]; int col; i32x4 idx[2]; };
    const int lane = threadIdx.x & 63, sp = (lane >> 4) % P, sub = (lane >> 4) / P, c = 8 * (lane & 15), in = c & ((1 << k.bw_log2) - 1);
    const int nrow[1] = {min(lane & 15, rows - 1) * ROW}, last = k.kb1 - 1;
    auto piece_of = [&](int kb) -> int {              // where this lane's columns of the turn at kb begin, K and more: nowhere
        const int s = min(kb + sp * W, last);
        const int piece = k.pieces ? gload<int>(k.pieces + (s << (7 - k.bw_log2)) + (c >> k.bw_log2)) : (s << 7) + c - in;
        return piece < 0 ? x.K : piece + in;
    };
    auto columns = [&](int n, const Turn& t) -> q_eight<Q8> {
        if constexpr (FAST) {
            const q_eight<Q8> v = gload<q_eight<Q8>>(reinterpret_cast<const E*>(x.x) + row_of(n) * x.ld + min(t.col, x.K - 8));
            return t.col < x.K ? v : q_eight<Q8>{};
        } else return q_load8<Q8>(x, row_of(n), t.col, t.idx);
    };
    auto fetch = [&](Turn& t, int kb, int col) {
        t.col = col;
        if constexpr (!FAST) {
            t.idx[0] = t.idx[1] = i32x4{-1, -1, -1, -1};
            if (x.pcol && col < x.K) { t.idx[0] = gload<i32x4>(x.pcol + col); t.idx[1] = gload<i32x4>(x.pcol + col + 4); }
        }
        #pragma unroll
        for (int p = 0; p < P; ++p)
            #pragma unroll
            for (int r = 0; r < RS; ++r) t.u[p][r].load(k.codes, k.scales, k.zeros, k.unit0 + (size_t)r * k.nkb + min(kb + p * W, last), lane);
        #pragma unroll
        for (int i = 0; i < AHEAD; ++i) t.v[i] = columns(min(sub + G * i, rows - 1), t);
    };
    auto multiply = [&](const Turn& t, int kb) {
        char* mine = xs + (sp * rows + sub) * ROW;
        #pragma unroll
        for (int i = 0; i < AHEAD; ++i) if (sub + G * i < rows) q_store8<Q8>(mine + G * i * ROW, lane & 15, t.v[i]);
        for (int n = G * AHEAD; n + sub < rows; n += G) q_store8<Q8>(mine + n * ROW, lane & 15, columns(n + sub, t));
        wave_lds_sync();
        #pragma unroll
        for (int p = 0; p < P; ++p)
            if (p == 0 || kb + p * W < k.kb1) {
                const QRows<Q8, 1> b{xs + p * rows * ROW, nrow, lane};
                q_multiply<Q8, GPK, ZP, 1, RS>(t.u[p], b, acc);
                __builtin_amdgcn_sched_barrier(0);       // one unit at a time: several side by side cost registers that wavefronts need
            }
        wave_lds_sync();
    };
    if (k.kb >= k.kb1) return;
    Turn t0, t1;
    const int c0 = piece_of(k.kb);
    int c1 = piece_of(k.kb + STEP);
    fetch(t0, k.kb, c0);
    for (int kb = k.kb;;) {
        const int c2 = piece_of(kb + 2 * STEP);
        fetch(t1, kb + STEP, c1);
        multiply(t0, kb);
        kb += STEP;
        if (kb >= k.kb1) break;
        c1 = piece_of(kb + 2 * STEP);
        fetch(t0, kb + STEP, c2);
        multiply(t1, kb);
        kb += STEP;
        if (kb >= k.kb1) break;
    }
}

}  // namespace pivot
