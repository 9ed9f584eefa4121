// Root-mean-square norm of rows with the residual's addition in front, output in fp32, fp16 or 8 bits with a scale per row.
//
//     h = x + res,   out = weight * h / sqrt(mean(h^2) + eps);   8 bits: max |out| / 127 is one step
//
// TPR threads share a row, eight neighbouring columns each at a time, and keep weight * h (or both) in registers between the two
// passes (sum of squares and largest weight * h, then the outputs); what of a row does not fit there is read a second
// time.  8192x4096, residual and output fp16: 51 us = 5.2 TB/s, what a copy reaches; fp32 into fp32 95 us = 5.6; fp32 into 8
// bits 84 us = 5.2; fp16 into 8 bits 61 us = 3.8, where the vector units are busy 68 % of the time with 45 instructions a column.
// One row of 4096: 3.2 us, 3.5 into 8 bits, 5.2 in block order: launch, one trip, two reductions, stores.  Rows of up to 16384
// columns are kept whole, their loads out together (64x9203 fp32 into fp16 5.8 -> 5.3 us, 2048x16000 fp16 into 8 bits 69 -> 64,
// but 8192x4096 fp32 into 8 bits 81 -> 84).  In block order 8192x4096 fp16 into fp16 takes 104 us, into 8 bits 102.
// The 8-bit codes depend on weight * h / max alone, which is computed in 64 bits: in 32 bits about one code in
// 10^5 would fall to the other side of the middle between two.
#include <algorithm>
#include <type_traits>

#include "pivot_quant_core.h"

namespace pivot {

namespace {

// Vectors of eight that need no more alignment than their elements have.
typedef float    f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef _Float16 f16x8_any __attribute__((ext_vector_type(8), aligned(2)));

// Eight neighbouring elements as they lie in memory, the first `n` of them real (the others 0).  Loading and converting are
// apart, so that no load of a row waits for another.
struct NormRaw { u32x4 a, b; };
// (the weaker alignment of a type is lost where the type is a template's argument, so this is no gload)
__device__ __forceinline__ u32x4 norm_load16(const void* p) {
    typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
    return *(const __attribute__((address_space(1))) u32x4_any*)p;
}
__device__ __forceinline__ void norm_load(const void* p, int type, long long at, int n, NormRaw& r) {
    const char* q = reinterpret_cast<const char*>(p) + at * (type == PIVOT_F32 ? 4 : 2);
    if (n >= 8) {
        r.a = norm_load16(q);
        if (type == PIVOT_F32) r.b = norm_load16(q + 16);
        return;
    }
    #pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t v = 0;
        if (i < n) v = type == PIVOT_F32 ? gload<uint32_t>(q + 4 * i) : gload<uint16_t>(q + 2 * i);
        if (type == PIVOT_F32) { if (i < 4) r.a[i & 3] = v; else r.b[i & 3] = v; }
        else r.a[i >> 1] = i & 1 ? r.a[i >> 1] | v << 16 : v;
    }
}
__device__ __forceinline__ void norm_floats(const NormRaw& r, int type, float (&v)[8]) {
    if (type == PIVOT_F32) {
        #pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, (uint32_t)(i < 4 ? r.a[i & 3] : r.b[i & 3]));
    } else {
        const f16x8 h = __builtin_bit_cast(f16x8, r.a);
        #pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
    }
}

__device__ __forceinline__ void norm_store(void* p, int type, long long at, int n, const float (&v)[8]) {
    if (type == PIVOT_F32) {
        float* q = reinterpret_cast<float*>(p) + at;
        if (n >= 8) {
            *reinterpret_cast<f32x4_any*>(q) = f32x4_any{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_any*>(q + 4) = f32x4_any{v[4], v[5], v[6], v[7]};
        } else
            #pragma unroll
            for (int i = 0; i < 8; ++i) if (i < n) q[i] = v[i];
    } else {
        _Float16* q = reinterpret_cast<_Float16*>(p) + at;
        if (n >= 8) {
            f16x8_any o;
            #pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (_Float16)v[i];
            *reinterpret_cast<f16x8_any*>(q) = o;
        } else
            #pragma unroll
            for (int i = 0; i < 8; ++i) if (i < n) q[i] = (_Float16)v[i];
    }
}

template <int CTRL>
__device__ __forceinline__ double dpp64(double v) {
    const long long b = __builtin_bit_cast(long long, v);
    const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xF, 0xF, false), hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xF, 0xF, false);
    return __builtin_bit_cast(double, (long long)(((unsigned long long)hi << 32) | lo));
}
__device__ __forceinline__ double lane64(double v, int l) {
    const long long b = __builtin_bit_cast(long long, v);
    const unsigned lo = __builtin_amdgcn_readlane((int)b, l), hi = __builtin_amdgcn_readlane((int)(b >> 32), l);
    return __builtin_bit_cast(double, (long long)(((unsigned long long)hi << 32) | lo));
}
// Over the 64 lanes, in every one of them: rows of sixteen by lane permutes, then the four rows.
template <typename Op>
__device__ __forceinline__ double wave64(double v, Op op) {
    v = op(v, dpp64<0xB1>(v));
    v = op(v, dpp64<0x4E>(v));
    v = op(v, dpp64<0x141>(v));
    v = op(v, dpp64<0x140>(v));
    return op(op(lane64(v, 0), lane64(v, 16)), op(lane64(v, 32), lane64(v, 48)));
}

// v * inv to the nearest integer, ties to even: the low word of the product + 1.5 * 2^52.  The product is rounded before the
// addition, so that what lies in the middle between two codes stays there.
__device__ __forceinline__ int code_of(double v, double inv) {
    #pragma clang fp contract(off)
    const double p = v * inv;
    return (int)__builtin_bit_cast(long long, p + 6755399441055744.0);
}

}  // namespace

// WIDE: h and weight * h in 64 bits, for 8-bit rows and where an input is fp32: its sums and products may leave the range of
// fp32 where the output does not.  Rows of fp16 stay far inside it as long as h / rms is formed first; 64 bits would cost them
// more than the memory hides (8192x4096 fp16 into fp16 51 -> 58 us, 100000x300 83 -> 106; fp32 into fp32 93 -> 95).
template <bool Q8, bool WIDE, bool ORDER, int TPR, int KEEP>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_kernel(NormLaunch a) {
    constexpr int NT = TPR < 256 ? 256 : TPR, NW = TPR / 64;
    typedef typename std::conditional<WIDE, double, float>::type H;
    static_assert(WIDE || !Q8, "8-bit codes are computed in 64 bits");
    __shared__ double s_sum[NT / 64], s_most[NT / 64];
    extern __shared__ __align__(16) char s_row[];       // the output row, where it is put together there
    const int tid = threadIdx.x % TPR, lane = threadIdx.x & 63, wave = q_wave();
    const long long row = a.row0 + (long long)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
    if (TPR < 256 && row >= a.rows) return;             // (whole wavefronts: no barrier below for TPR = 64)
    const long long xo = row * a.ldx, ro = row * a.ldr, so = row * a.ldro, oo = row * a.ldo;
    const int es = Q8 ? 1 : (a.otype == PIVOT_F32 ? 4 : 2);
    // rows in a layer's block order are put together in LDS: single elements all over a row would be a line each to the
    // memory system
    char* mine = s_row + (threadIdx.x / TPR) * ((a.cols * es + 15) & ~15);
    int place[ORDER ? KEEP : 1][8];
    if (ORDER)
        #pragma unroll
        for (int k = 0; k < KEEP; ++k)
            #pragma unroll
            for (int i = 0; i < 8; ++i) { const int c = (tid + k * TPR) * 8 + i; place[k][i] = c < a.cols ? gload<int>(a.order + c) : 0; }

    struct Piece { NormRaw x, r, w; };
    auto fetch = [&](int c, Piece& p) {
        const int n = a.cols - c;
        norm_load(a.x, a.xtype, xo + c, n, p.x);
        if (a.res) norm_load(a.res, a.rtype, ro + c, n, p.r);
        if (a.weight) norm_load(a.weight, PIVOT_F32, c, n, p.w);
    };
    double sum = 0.0, most = 0.0;
    float bad = 0.f;                                    // NaN once anything is infinite or NaN
    // weight * h of a piece (not WIDE: h, and the weights); the sums on the first pass, what goes back to the residual on the
    // last one
    auto combine = [&](int c, const Piece& p, H (&hw)[8], float (&pw)[8], bool first, bool last) {
        float back[8], px[8], pr[8] = {};
        norm_floats(p.x, a.xtype, px);
        if (a.res) norm_floats(p.r, a.rtype, pr);
        if (a.weight) norm_floats(p.w, PIVOT_F32, pw);
        else
            #pragma unroll
            for (int i = 0; i < 8; ++i) pw[i] = 1.f;
        #pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = px[i], r = pr[i], w = pw[i];
            const H h = (H)x + (H)r;
            back[i] = x + r;
            hw[i] = WIDE ? h * (H)w : h;
            if (first) {
                sum = __builtin_fma((double)h, (double)h, sum);
                if constexpr (Q8) {
                    most = __builtin_fmax(most, __builtin_fabs(hw[i]));
                    bad = __builtin_fmaf(x, 0.f, __builtin_fmaf(r, 0.f, __builtin_fmaf(w, 0.f, bad)));
                }
            }
        }
        if (last && a.res_out) norm_store(a.res_out, a.rtype, so + c, a.cols - c, back);
    };
    H keep[KEEP][8];
    float kept_w[KEEP][8];
    {
        Piece p[KEEP];
        #pragma unroll
        for (int k = 0; k < KEEP; ++k) if ((tid + k * TPR) * 8 < a.cols) fetch((tid + k * TPR) * 8, p[k]);
        #pragma unroll
        for (int k = 0; k < KEEP; ++k) if ((tid + k * TPR) * 8 < a.cols) combine((tid + k * TPR) * 8, p[k], keep[k], kept_w[k], true, true);
    }
    for (int c = (tid + KEEP * TPR) * 8; c < a.cols; c += TPR * 8) {
        Piece p;
        H hw[8];
        float pw[8];
        fetch(c, p);
        combine(c, p, hw, pw, true, false);
    }
    if (Q8 && bad != bad) most = __builtin_inf();
    sum = wave64(sum, [](double u, double v) { return u + v; });
    if (Q8) most = wave64(most, [](double u, double v) { return __builtin_fmax(u, v); });
    if (NW > 1) {
        if (lane == 0) { s_sum[wave] = sum; s_most[wave] = most; }
        __syncthreads();
        if (Q8) {
            #pragma unroll
            for (int w = 0; w < NW; ++w) most = __builtin_fmax(most, s_most[w]);
        }
        if (!Q8 || wave == 0) {
            sum = 0.0;
            #pragma unroll
            for (int w = 0; w < NW; ++w) sum += s_sum[w];
        }
    }
    const bool fine = most > 0.0 && most < __builtin_inf();
    const double inv = Q8 && fine ? 127.0 / most : 0.0;
    H rs = 0;
    if (!Q8) rs = (H)(1.0 / sqrt(sum / a.cols + (double)a.eps));
    else if (tid == 0)                                   // the only use of it: the codes do not depend on the sum
        a.scale[row] = fine ? (float)(most / sqrt(sum / a.cols + (double)a.eps) / 127.0) : (most == 0.0 ? 0.f : __builtin_nanf(""));
    auto finish = [&](int c, const H (&hw)[8], const float (&pw)[8], const int* at) {
        const int n = a.cols - c;
        if constexpr (Q8) {
            int code[8];
            #pragma unroll
            for (int i = 0; i < 8; ++i) {
                code[i] = fine ? code_of(hw[i], inv) : 0;
            }
            int8_t* q = reinterpret_cast<int8_t*>(a.out) + oo;
            if (ORDER) {
                int8_t* to = a.lds_rows ? reinterpret_cast<int8_t*>(mine) : q;
                #pragma unroll
                for (int i = 0; i < 8; ++i) if (i < n) to[at ? at[i] : a.order[c + i]] = (int8_t)code[i];
            } else if (n >= 8) {
                typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
                auto four = [&](int i) { return (code[i] & 255u) | (code[i + 1] & 255u) << 8 | (code[i + 2] & 255u) << 16 | (uint32_t)code[i + 3] << 24; };
                *reinterpret_cast<u32x2_any*>(q + c) = u32x2_any{four(0), four(4)};
            } else
                #pragma unroll
                for (int i = 0; i < 8; ++i) if (i < n) q[c + i] = (int8_t)code[i];
        } else {
            float v[8];
            #pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = WIDE ? (float)(hw[i] * rs) : (float)(hw[i] * rs) * pw[i];
            if (!ORDER) norm_store(a.out, a.otype, oo + c, n, v);
            else {
                char* to = a.lds_rows ? mine : reinterpret_cast<char*>(a.out) + oo * es;
                #pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < n) {
                        const int d = at ? at[i] : a.order[c + i];
                        if (a.otype == PIVOT_F32) reinterpret_cast<float*>(to)[d] = v[i];
                        else reinterpret_cast<_Float16*>(to)[d] = (_Float16)v[i];
                    }
            }
        }
    };
    #pragma unroll
    for (int k = 0; k < KEEP; ++k) if ((tid + k * TPR) * 8 < a.cols) finish((tid + k * TPR) * 8, keep[k], kept_w[k], ORDER ? place[k] : nullptr);
    for (int c = (tid + KEEP * TPR) * 8; c < a.cols; c += TPR * 8) {
        Piece p;
        H hw[8];
        float pw[8];
        fetch(c, p);
        combine(c, p, hw, pw, false, true);
        finish(c, hw, pw, nullptr);
    }
    if (ORDER && a.lds_rows) {
        if (NW > 1) __syncthreads(); else wave_lds_sync();
        char* q = reinterpret_cast<char*>(a.out) + oo * es;
        const int bytes = a.cols * es;
        typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
        for (int b = tid * 16; b < bytes; b += TPR * 16) {
            if (b + 16 <= bytes) { const u32x4 v = *reinterpret_cast<const u32x4*>(mine + b); *reinterpret_cast<u32x4_any*>(q + b) = u32x4_any{v[0], v[1], v[2], v[3]}; }
            else for (int i = b; i < bytes; ++i) q[i] = mine[i];
        }
    }
}

namespace {

template <bool Q8, bool WIDE, bool ORDER>
int norm_go(NormLaunch a) {
    hipStream_t st = reinterpret_cast<hipStream_t>(a.stream);
    auto go = [&](auto k, int per, int threads) {
        const size_t row = align_up((size_t)a.cols * (a.otype == PIVOT_Q8 ? 1 : elem_size(a.otype)), 16) * per;
        a.lds_rows = ORDER && row <= 60 * 1024;          // (longer rows: element by element)
        const long long blocks = ((long long)a.rows + per - 1) / per;
        constexpr long long kMost = 1 << 21;             // (a launch has less than 2^32 threads)
        for (long long b = 0; b < blocks; b += kMost) {
            a.row0 = (int)(b * per);
            hipLaunchKernelGGL(k, dim3((unsigned)std::min(kMost, blocks - b)), dim3(threads), a.lds_rows ? row : 0, st, a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) { set_error("launch failed: %s", hipGetErrorString(e)); return PIVOT_E_HIP; }
        }
        return PIVOT_OK;
    };
    const bool many = a.rows >= 512;                      // rows enough to fill the device with few threads each
    if (a.cols <= 64 * 8 && (many || a.cols <= 64)) return go(norm_kernel<Q8, WIDE, ORDER, 64, 1>, 4, 256);
    if (a.cols <= 256 * 8) return go(norm_kernel<Q8, WIDE, ORDER, 256, 1>, 1, 256);
    if (a.cols <= 512 * 8 && many) return go(norm_kernel<Q8, WIDE, ORDER, 512, 1>, 1, 512);
    return a.cols <= 1024 * 8 ? go(norm_kernel<Q8, WIDE, ORDER, 1024, 1>, 1, 1024) : go(norm_kernel<Q8, WIDE, ORDER, 1024, 2>, 1, 1024);
}

}  // namespace

int launch_norm(const NormLaunch& a) {
    if (a.otype == PIVOT_Q8) return a.order ? norm_go<true, true, true>(a) : norm_go<true, true, false>(a);
    if (a.xtype == PIVOT_F32 || (a.res && a.rtype == PIVOT_F32)) return a.order ? norm_go<false, true, true>(a) : norm_go<false, true, false>(a);
    return a.order ? norm_go<false, false, true>(a) : norm_go<false, false, false>(a);
}

}  // namespace pivot
