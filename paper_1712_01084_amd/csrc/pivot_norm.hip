// Root-mean-square norm of rows with the residual's addition in front, output in fp32, fp16 or 8 bits with a scale per row.
//
//     h = x + res,   out = weight * h / sqrt(mean(h^2) + eps);   8 bits: max |out| / 127 is one step
//
// TPR threads share a row and keep it in registers between the two passes (sum of squares and largest weight * h, then
// the outputs); rows too long for that are read a second time.  The 8-bit codes depend on weight * h / max alone, which is
// computed in 64 bits: in 32 bits about one code in 10^5 would fall to the other side of the middle between two.
#include "pivot_quant_core.h"

namespace pivot {

namespace {

// Eight (V = 8: neighbouring, aligned) or single elements as floats.
template <int V>
__device__ __forceinline__ void norm_load(const void* p, int type, long long at, float (&v)[V]) {
    if (type == PIVOT_F32) {
        const float* q = reinterpret_cast<const float*>(p) + at;
        if (V == 8) {
            const f32x4 a = *reinterpret_cast<const f32x4*>(q), b = *reinterpret_cast<const f32x4*>(q + 4);
            #pragma unroll
            for (int i = 0; i < V; ++i) v[i] = i < 4 ? a[i & 3] : b[i & 3];
        } else v[0] = q[0];
    } else {
        const _Float16* q = reinterpret_cast<const _Float16*>(p) + at;
        if (V == 8) {
            const f16x8 a = *reinterpret_cast<const f16x8*>(q);
            #pragma unroll
            for (int i = 0; i < V; ++i) v[i] = (float)a[i];
        } else v[0] = (float)q[0];
    }
}

template <int V>
__device__ __forceinline__ void norm_store(void* p, int type, long long at, const float (&v)[V]) {
    if (type == PIVOT_F32) {
        float* q = reinterpret_cast<float*>(p) + at;
        if (V == 8) {
            *reinterpret_cast<f32x4*>(q) = f32x4{v[0], v[1 % V], v[2 % V], v[3 % V]};
            *reinterpret_cast<f32x4*>(q + 4) = f32x4{v[4 % V], v[5 % V], v[6 % V], v[7 % V]};
        } else q[0] = v[0];
    } else {
        _Float16* q = reinterpret_cast<_Float16*>(p) + at;
        if (V == 8) {
            f16x8 o;
            #pragma unroll
            for (int i = 0; i < V; ++i) o[i] = (_Float16)v[i];
            *reinterpret_cast<f16x8*>(q) = o;
        } else q[0] = (_Float16)v[0];
    }
}

// The larger of two, a NaN being larger than anything.
__device__ __forceinline__ double most_of(double m, double o) { return (o > m || o != o) ? o : m; }

}  // namespace

template <bool Q8, int V, int TPR>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_kernel(NormLaunch a) {
    constexpr int NT = TPR < 256 ? 256 : TPR, NW = TPR / 64, KEEP = V == 8 ? 2 : 4;
    __shared__ double s_sum[NT / 64], s_most[NT / 64];
    const int tid = threadIdx.x % TPR, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long row = (long long)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
    if (TPR < 256 && row >= a.rows) return;             // (whole wavefronts: no barrier below for TPR = 64)
    const long long xo = row * a.ldx, ro = row * a.ldr, so = row * a.ldro, oo = row * a.ldo;
    float kx[KEEP][V], kr[KEEP][V], kw[KEEP][V];
    double sum = 0.0, most = 0.0;
    auto fetch = [&](int c, float (&x)[V], float (&r)[V], float (&w)[V]) {
        norm_load<V>(a.x, a.xtype, xo + c, x);
        if (a.res) norm_load<V>(a.res, a.rtype, ro + c, r);
        else for (int i = 0; i < V; ++i) r[i] = 0.f;
        if (a.weight) norm_load<V>(a.weight, PIVOT_F32, c, w);
        else for (int i = 0; i < V; ++i) w[i] = 1.f;
    };
    auto measure = [&](const float (&x)[V], const float (&r)[V], const float (&w)[V]) {
        #pragma unroll
        for (int i = 0; i < V; ++i) {
            const double h = (double)x[i] + (double)r[i];
            sum += h * h;
            if (Q8) most = most_of(most, fabs(h * (double)w[i]));
        }
    };
    #pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        const int c = (tid + k * TPR) * V;
        if (c < a.cols) { fetch(c, kx[k], kr[k], kw[k]); }
    }
    #pragma unroll
    for (int k = 0; k < KEEP; ++k)
        if ((tid + k * TPR) * V < a.cols) measure(kx[k], kr[k], kw[k]);
    for (int c = (tid + KEEP * TPR) * V; c < a.cols; c += TPR * V) {
        float x[V], r[V], w[V];
        fetch(c, x, r, w);
        measure(x, r, w);
    }
    #pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        sum += __shfl_xor(sum, m, 64);
        if (Q8) most = most_of(most, __shfl_xor(most, m, 64));
    }
    if (NW > 1) {
        if (lane == 0) { s_sum[wave] = sum; s_most[wave] = most; }
        __syncthreads();
        sum = 0.0; most = 0.0;
        #pragma unroll
        for (int w = 0; w < NW; ++w) { sum += s_sum[w]; if (Q8) most = most_of(most, s_most[w]); }
    }
    const double rstd = 1.0 / sqrt(sum / a.cols + (double)a.eps);
    const bool fine = most > 0.0 && most < __builtin_inf();
    const double inv = fine ? 127.0 / most : 0.0;
    if (Q8 && tid == 0) a.scale[row] = fine ? (float)(most * rstd / 127.0) : (most == 0.0 ? 0.f : __builtin_nanf(""));
    const float rs = (float)rstd;
    auto finish = [&](int c, const float (&x)[V], const float (&r)[V], const float (&w)[V]) {
        if (a.res_out) {
            float h[V];
            #pragma unroll
            for (int i = 0; i < V; ++i) h[i] = x[i] + r[i];
            norm_store<V>(a.res_out, a.rtype, so + c, h);
        }
        if (Q8) {
            union { int8_t b[8]; uint2 u; } o;
            #pragma unroll
            for (int i = 0; i < V; ++i) {
                const double hw = ((double)x[i] + (double)r[i]) * (double)w[i];
                o.b[i] = fine ? (int8_t)__double2int_rn(hw * inv) : (int8_t)0;
            }
            int8_t* q = reinterpret_cast<int8_t*>(a.out) + oo;
            if (a.order) { for (int i = 0; i < V; ++i) q[a.order[c + i]] = o.b[i]; }
            else if (V == 8) *reinterpret_cast<uint2*>(q + c) = o.u;
            else q[c] = o.b[0];
        } else {
            float v[V];
            #pragma unroll
            for (int i = 0; i < V; ++i) v[i] = (x[i] + r[i]) * w[i] * rs;
            if (a.order) {
                for (int i = 0; i < V; ++i) {
                    const float one[1] = {v[i]};
                    norm_store<1>(a.out, a.otype, oo + a.order[c + i], one);
                }
            } else norm_store<V>(a.out, a.otype, oo + c, v);
        }
    };
    #pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        const int c = (tid + k * TPR) * V;
        if (c < a.cols) finish(c, kx[k], kr[k], kw[k]);
    }
    for (int c = (tid + KEEP * TPR) * V; c < a.cols; c += TPR * V) {
        float x[V], r[V], w[V];
        fetch(c, x, r, w);
        finish(c, x, r, w);
    }
}

namespace {

template <bool Q8, int V>
int norm_go(const NormLaunch& a) {
    hipStream_t st = reinterpret_cast<hipStream_t>(a.stream);
    if (a.cols <= 64 * V)       hipLaunchKernelGGL((norm_kernel<Q8, V, 64>), dim3((a.rows + 3) / 4), dim3(256), 0, st, a);
    else if (a.cols <= 512 * V) hipLaunchKernelGGL((norm_kernel<Q8, V, 256>), dim3(a.rows), dim3(256), 0, st, a);
    else                        hipLaunchKernelGGL((norm_kernel<Q8, V, 1024>), dim3(a.rows), dim3(1024), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("launch failed: %s", hipGetErrorString(e)); return PIVOT_E_HIP; }
    return PIVOT_OK;
}

bool whole(const void* p, int type, int64_t ld, int rows) {     // whether rows are whole pieces of eight
    const int piece = type == PIVOT_Q8 ? 8 : 16, es = type == PIVOT_Q8 ? 1 : elem_size(type);
    return !p || (reinterpret_cast<uintptr_t>(p) % piece == 0 && (rows == 1 || ld * es % piece == 0));
}

}  // namespace

int launch_norm(const NormLaunch& a) {
    const bool v8 = a.cols % 8 == 0 && whole(a.x, a.xtype, a.ldx, a.rows) && whole(a.res, a.rtype, a.ldr, a.rows) && whole(a.res_out, a.rtype, a.ldro, a.rows) &&
                    whole(a.weight, PIVOT_F32, 0, 1) && (a.order || whole(a.out, a.otype, a.ldo, a.rows));
    if (a.otype == PIVOT_Q8) return v8 ? norm_go<true, 8>(a) : norm_go<true, 1>(a);
    return v8 ? norm_go<false, 8>(a) : norm_go<false, 1>(a);
}

}  // namespace pivot
