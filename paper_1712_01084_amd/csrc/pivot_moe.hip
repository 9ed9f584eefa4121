// A mixture-of-experts layer for up to 16 tokens, three launches:
//
//   router   one workgroup per expert: its logit for every token; the last one to arrive ranks them, takes the softmax and
//            writes down which experts are in use, by which tokens
//   up       one workgroup per expert in use and strip of 16 rows (8 gate rows and their 8 up rows): silu(gate) * up,
//            stored in the block order of the expert's down layer as fp16 value and remainder times 2^11 (22 bits, so
//            that this boundary costs the result nothing an fp32 sum would keep)
//   down     one workgroup per strip of 16 outputs: all experts in use, one after the other, their sums weighted and added
//            in the accumulators.  The tokens are the columns of the matrix instruction in every expert, so no expert's
//            output is ever stored and nothing is added across workgroups
//
// The weights of an expert in use are read once, whatever the number of its tokens.
#include <algorithm>
#include <type_traits>

#include "pivot_quant_core.h"

namespace pivot {

namespace {

constexpr int kRouterThreads = 256;

template <typename T>
__device__ __forceinline__ void router_load8(const T* p, int c, int D, bool vec, float (&v)[8]) {
    if (vec) {
        if constexpr (sizeof(T) == 2) {
            const f16x8 a = *reinterpret_cast<const f16x8*>(p + c);
            #pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
        } else {
            const f32x4 a = *reinterpret_cast<const f32x4*>(p + c), b = *reinterpret_cast<const f32x4*>(p + c + 4);
            #pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < 4 ? a[i & 3] : b[i & 3];
        }
    } else {
        #pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < D ? (float)p[c + i] : 0.f;
    }
}

template <typename RT>
__global__ void __launch_bounds__(kRouterThreads) moe_router_kernel(MoeLaunch a, int vec) {
    __shared__ float s_red[kRouterThreads / 64][kMoeMaxTokens];
    __shared__ float s_logit[kMoeMaxTokens][kMoeMaxExperts];
    __shared__ int   s_sel[kMoeMaxTokens][kMoeMaxTopK];
    __shared__ float s_w[kMoeMaxTokens][kMoeMaxTopK];
    __shared__ int   s_base[kRouterThreads / 64], s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, e = blockIdx.x, T = a.tokens, E = a.E, K = a.top_k;
    const RT* w = reinterpret_cast<const RT*>(a.router) + (long long)e * a.D;
    const _Float16* x = reinterpret_cast<const _Float16*>(a.x);
    float acc[kMoeMaxTokens] = {};
    for (int c = tid * 8; c < a.D; c += kRouterThreads * 8) {
        float wv[8];
        router_load8(w, c, a.D, vec, wv);
        #pragma unroll
        for (int t = 0; t < kMoeMaxTokens; ++t) {
            if (t < T) {
                float xv[8];
                router_load8(x + t * a.ldx, c, a.D, vec, xv);
                #pragma unroll
                for (int i = 0; i < 8; ++i) acc[t] = __builtin_fmaf(wv[i], xv[i], acc[t]);
            }
        }
    }
    #pragma unroll
    for (int t = 0; t < kMoeMaxTokens; ++t) {
        if (t < T) {
            const float s = group_sum<64>(acc[t]);
            if (lane == 0) s_red[wave][t] = s;
        }
    }
    __syncthreads();
    if (tid < T) {
        float s = 0.f;
        #pragma unroll
        for (int q = 0; q < kRouterThreads / 64; ++q) s += s_red[q][tid];
        if (a.router_bias) s += a.router_bias[e];
        agent_store(a.logits + tid * E + e, s);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the logits are out before the arrival is counted
    __syncthreads();
    if (tid == 0) {
        const int last = __hip_atomic_fetch_add(&a.route->ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(E - 1);
        if (last) __hip_atomic_store(&a.route->ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = last;
    }
    __syncthreads();
    if (!s_last) return;

    // ---- the last workgroup: ranks, weights, and who uses what
    for (int i = tid; i < T * E; i += kRouterThreads) s_logit[i / E][i % E] = agent_load(a.logits + i);
    if (tid < kMoeMaxTokens * kMoeMaxTopK) { (&s_sel[0][0])[tid] = -1; (&s_w[0][0])[tid] = 0.f; }
    __syncthreads();
    const float ninf = -__builtin_inff();
    for (int t = wave; t < T; t += kRouterThreads / 64) {
        float v[4], m = ninf;
        int any_nan = 0;
        #pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] = lane + 64 * q < E ? s_logit[t][lane + 64 * q] : ninf;
            any_nan |= v[q] != v[q];
            m = fmaxf(m, v[q]);
        }
        any_nan = __any(any_nan);
        #pragma unroll
        for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
        int rank[4] = {};
        if (any_nan) {                                   // the first top_k experts, with weights that are NaN
            #pragma unroll
            for (int q = 0; q < 4; ++q) { rank[q] = lane + 64 * q; if (rank[q] < E) v[q] = __builtin_nanf(""); }
        } else {
            for (int j = 0; j < E; ++j) {
                const float o = s_logit[t][j];
                #pragma unroll
                for (int q = 0; q < 4; ++q) rank[q] += (o > v[q] || (o == v[q] && j < lane + 64 * q)) ? 1 : 0;
            }
        }
        float p[4], s = 0.f;
        bool chosen[4];
        #pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool real = lane + 64 * q < E && v[q] != ninf;
            chosen[q] = real && rank[q] < K;
            p[q] = real ? expf(v[q] - m) : 0.f;
            if (real && (chosen[q] || !a.renormalise)) s += p[q];
        }
        s = group_sum<64>(s);
        #pragma unroll
        for (int q = 0; q < 4; ++q)
            if (chosen[q]) { s_sel[t][rank[q]] = lane + 64 * q; s_w[t][rank[q]] = p[q] / s; }
    }
    __syncthreads();
    if (tid < T * K) {
        const int t = tid / K, j = tid % K;
        a.route->sel[t][j] = s_sel[t][j];
        a.route->sel_w[t][j] = s_w[t][j];
        if (a.ids) a.ids[tid] = s_sel[t][j];
        if (a.weights) a.weights[tid] = s_w[t][j];
    }
    // experts in use, in ascending order: thread e counts expert e's tokens
    int n = 0;
    if (tid < E)
        for (int i = 0; i < T * K; ++i) n += s_sel[i / K][i % K] == tid;
    const unsigned long long used = __ballot(n > 0);
    if (lane == 0) s_base[wave] = __popcll(used);
    __syncthreads();
    int at = __popcll(used & ((1ull << lane) - 1)), total = 0;
    #pragma unroll
    for (int q = 0; q < kRouterThreads / 64; ++q) { if (q < wave) at += s_base[q]; total += s_base[q]; }
    if (tid == 0) a.route->n = total;
    if (n > 0) {
        a.route->expert[at] = tid;
        a.route->ntok[at] = n;
        int m = 0;
        for (int t = 0; t < kMoeMaxTokens; ++t) {
            int row = -1;
            float share = 0.f;
            if (t < T)
                for (int j = 0; j < K; ++j)
                    if (s_sel[t][j] == tid) { row = t * K + j; share = s_w[t][j]; }
            a.route->hrow[at][t] = row;
            a.route->share[at][t] = share;
            if (row >= 0) a.route->tok[at][m++] = t;
        }
    }
}

template <int GPK, bool ZP, int P, int W>
__global__ void __launch_bounds__(W * 64) moe_up_kernel(MoeLaunch a, int vec) {
    constexpr int ROW = QElem<false>::kRow;
    extern __shared__ __align__(16) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int act = blockIdx.y, strip = blockIdx.x;
    if (act >= a.route->n) return;
    const int e = a.route->expert[act], ntok = a.route->ntok[act], T = a.tokens;
    const MoeExpert& ex = a.experts[e];
    const int sb = a.bh[0] / kQStrip, br = strip / sb, bw_log2 = 31 - __clz(a.bw[0]);
    const int kb0 = ex.kb_ptr[0][br], nkb = ex.kb_ptr[0][br + 1] - kb0;
    const size_t unit0 = (size_t)kb0 * sb + (size_t)(strip % sb) * nkb;
    const u32x4* codes = reinterpret_cast<const u32x4*>(ex.codes[0]); const uint16_t* scales = ex.scales[0]; const int8_t* zoff = ex.zoff[0];
    const int32_t* pieces = ex.pieces[0] + ((size_t)kb0 << (7 - bw_log2));
    const QSource x{a.x, a.ldx, ex.pcol, a.D, vec};
    char* xs = smem + wave * (P * T * ROW);
    const int nrow[1] = {min(lane & 15, ntok - 1) * ROW};
    f32x4 acc[1][1] = {};
    const int sp = (lane >> 4) % P, c8 = lane & 15;
    for (int kb = wave; kb < nkb; kb += W * P) {
        QUnit<GPK, ZP> u[P][1];
        #pragma unroll
        for (int p = 0; p < P; ++p)
            if (kb + p * W < nkb) u[p][0].load(codes, scales, zoff, unit0 + kb + p * W, lane);
        const int skb = kb + sp * W;
        if (skb < nkb) {
            const int c = 8 * c8, piece0 = gload<int>(pieces + (skb << (7 - bw_log2)) + (c >> bw_log2));
            const int col = piece0 < 0 ? a.D : piece0 + (c & ((1 << bw_log2) - 1));
            i32x4 idx[2] = {i32x4{-1, -1, -1, -1}, i32x4{-1, -1, -1, -1}};
            if (x.pcol && piece0 >= 0) { idx[0] = gload<i32x4>(x.pcol + col); idx[1] = gload<i32x4>(x.pcol + col + 4); }
            for (int m = (lane >> 4) / P; m < ntok; m += 4 / P) {
                __align__(16) _Float16 v[8];
                q_load8<false>(x, a.route->tok[act][m], col, idx, v);
                q_store8<false>(xs + (sp * T + m) * ROW, c8, v);
            }
        }
        wave_lds_sync();
        #pragma unroll
        for (int p = 0; p < P; ++p)
            if (kb + p * W < nkb) q_multiply<false, GPK, ZP, 1, 1>(u[p], xs + p * T * ROW, nrow, lane, acc);
        wave_lds_sync();
    }
    __syncthreads();
    float* red = reinterpret_cast<float*>(smem);
    #pragma unroll
    for (int i = 0; i < 4; ++i) red[wave * 256 + (lane & 15) * 16 + 4 * (lane >> 4) + i] = acc[0][0][i];
    __syncthreads();
    if (tid < 8 * ntok) {
        const int m = tid / 8, u = tid % 8, r = strip * 16 + 2 * u, dst = ex.hdst[strip * 8 + u];
        float g = 0.f, v = 0.f;
        #pragma unroll
        for (int w = 0; w < W; ++w) { g += red[w * 256 + m * 16 + 2 * u]; v += red[w * 256 + m * 16 + 2 * u + 1]; }
        g += ex.bias[0][r];
        v += ex.bias[0][r + 1];
        const float h = g / (1.f + expf(-g)) * v;
        const _Float16 hi = (_Float16)h;
        // what fp16 leaves of h, 2^11 times: again fp16; nothing where h is beyond the range
        const _Float16 lo = fabsf((float)hi) < __builtin_inff() ? (_Float16)((h - (float)hi) * 2048.f) : (_Float16)0.f;
        if (dst >= 0) {
            _Float16* out = reinterpret_cast<_Float16*>(a.h) + (size_t)a.route->hrow[act][a.route->tok[act][m]] * a.F_pad + dst;
            out[0] = hi;
            out[(size_t)T * a.top_k * a.F_pad] = lo;
        }
    }
}

// An expert in use, for one strip of its down layer.
struct DownExpert { const u32x4* codes; const uint16_t* scales; const int8_t* zoff; const int32_t* pieces; };

template <int GPK, bool ZP, int P, int W>
__global__ void __launch_bounds__(W * 64) moe_down_kernel(MoeLaunch a) {
    static_assert(P == 2 || P == 4, "the staging takes two planes of P units with four groups of lanes");
    constexpr int ROW = QElem<false>::kRow;
    extern __shared__ __align__(16) char smem[];
    __shared__ DownExpert s_ex[kMoeMaxActive];
    __shared__ int s_cum[kMoeMaxActive + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, T = a.tokens, n_act = a.route->n;
    const int strip = blockIdx.x, sb = a.bh[1] / kQStrip, br = strip / sb, bw_log2 = 31 - __clz(a.bw[1]);
    if (wave == 0) {                                    // block counts of the experts in use, and their running sum
        int run = 0;
        for (int base = 0; base < n_act; base += 64) {
            const int i = base + lane;
            int nkb = 0;
            if (i < n_act) {
                const MoeExpert& ex = a.experts[a.route->expert[i]];
                const int kb0 = ex.kb_ptr[1][br];
                nkb = ex.kb_ptr[1][br + 1] - kb0;
                const size_t unit0 = (size_t)kb0 * sb + (size_t)(strip % sb) * nkb;
                s_ex[i] = DownExpert{reinterpret_cast<const u32x4*>(ex.codes[1]) + unit0 * 64, ex.scales[1] + unit0 * GPK * kQStrip,
                                     ZP ? ex.zoff[1] + unit0 * GPK * kQStrip : nullptr, ex.pieces[1] + ((size_t)kb0 << (7 - bw_log2))};
            }
            int s = nkb;
            #pragma unroll
            for (int d = 1; d < 64; d <<= 1) { const int o = __shfl_up(s, d, 64); if (lane >= d) s += o; }
            if (i < n_act) s_cum[i + 1] = run + s;
            run += __shfl(s, 63, 64);
        }
        if (lane == 0) s_cum[0] = 0;
    }
    __syncthreads();
    const int units = s_cum[n_act];
    char* xs = smem + wave * (P * 2 * T * ROW);
    const int n = min(lane & 15, T - 1);
    f32x4 total = {};
    int cur = 0;
    for (int u0 = wave; u0 < units; u0 += W * P) {
        QUnit<GPK, ZP> u[P][1];
        int act[P], kb[P];
        #pragma unroll
        for (int p = 0; p < P; ++p) {
            const int g = u0 + p * W;
            if (g < units) {
                while (g >= s_cum[cur + 1]) ++cur;
                act[p] = __builtin_amdgcn_readfirstlane(cur);
                kb[p] = __builtin_amdgcn_readfirstlane(g - s_cum[cur]);
                const DownExpert ex = s_ex[act[p]];
                u[p][0].load(ex.codes, ex.scales, ex.zoff, kb[p], lane);
            } else { act[p] = -1; kb[p] = 0; }
        }
        const int c = 8 * (lane & 15);
        #pragma unroll
        for (int q = 0; q < P / 2; ++q) {
            // lane groups 0 and 1: the two units of this turn, plane 0; groups 2 and 3: plane 1
            const int sel = (lane >> 4) & 1, plane = lane >> 5, p = 2 * q + sel;
            const int sa = sel ? act[2 * q + 1] : act[2 * q], skb = sel ? kb[2 * q + 1] : kb[2 * q];
            if (sa >= 0) {
                const int piece0 = gload<int>(s_ex[sa].pieces + (skb << (7 - bw_log2)) + (c >> bw_log2));
                const int col = piece0 < 0 ? a.F : piece0 + (c & ((1 << bw_log2) - 1));
                const QSource h{a.h + (size_t)plane * T * a.top_k * a.F_pad, a.F_pad, nullptr, a.F, 1};
                const int ntok = a.route->ntok[sa];
                const i32x4 none[2] = {};
                for (int m = 0; m < ntok; ++m) {
                    const int t = a.route->tok[sa][m];
                    __align__(16) _Float16 v[8];
                    q_load8<false>(h, a.route->hrow[sa][t], col, none, v);
                    q_store8<false>(xs + ((p * 2 + plane) * T + t) * ROW, lane & 15, v);
                }
            }
        }
        wave_lds_sync();
        #pragma unroll
        for (int p = 0; p < P; ++p)
            if (act[p] >= 0) {
                const int nrow[2] = {(p * 2 * T + n) * ROW, ((p * 2 + 1) * T + n) * ROW};
                f32x4 part[1][2] = {};
                q_multiply<false, GPK, ZP, 2, 1>(u[p], xs, nrow, lane, part);
                // tokens that do not use the expert: whatever their column held is dropped
                const bool mine = a.route->hrow[act[p]][n] >= 0;
                const float share = a.route->share[act[p]][n];
                #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float s = __builtin_fmaf(part[0][1][i], 1.f / 2048.f, part[0][0][i]);
                    total[i] = mine ? __builtin_fmaf(share, s, total[i]) : total[i];
                }
            }
        wave_lds_sync();
    }
    __syncthreads();
    float* red = reinterpret_cast<float*>(smem);
    #pragma unroll
    for (int i = 0; i < 4; ++i) red[wave * 256 + (lane & 15) * 16 + 4 * (lane >> 4) + i] = total[i];
    __syncthreads();
    for (int i = tid; i < 16 * T; i += W * 64) {
        const int t = i / 16, r = strip * 16 + i % 16, dst = a.prow_down[r];
        if (dst < 0) continue;
        float s = 0.f;
        #pragma unroll
        for (int w = 0; w < W; ++w) s += red[w * 256 + i];
        for (int j = 0; j < a.top_k; ++j) {
            const int e = a.route->sel[t][j];
            if (e >= 0) s = __builtin_fmaf(a.route->sel_w[t][j], a.experts[e].bias[1][r], s);
        }
        a.y[t * a.ldy + dst] = s;
    }
}

int launched() {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("launch failed: %s", hipGetErrorString(e)); return PIVOT_E_HIP; }
    return PIVOT_OK;
}

int reserve(const void* k, size_t smem) {
    if (smem > 64 * 1024 && hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != hipSuccess) {
        (void)hipGetLastError();
        set_error("cannot reserve %zu bytes of LDS", smem);
        return PIVOT_E_HIP;
    }
    return PIVOT_OK;
}

template <int GPK, bool ZP, int P>
int up_go(const MoeLaunch& L, int vec) {
    constexpr int W = 8;
    auto k = moe_up_kernel<GPK, ZP, P, W>;
    const size_t smem = std::max((size_t)W * P * L.tokens * QElem<false>::kRow, (size_t)W * 1024);
    int rc = reserve(reinterpret_cast<const void*>(k), smem);
    if (rc != PIVOT_OK) return rc;
    hipLaunchKernelGGL(k, dim3(L.nstrips[0], std::min(L.E, L.tokens * L.top_k)), dim3(W * 64), smem, reinterpret_cast<hipStream_t>(L.stream), L, vec);
    return launched();
}

template <int GPK, bool ZP, int P>
int down_go(const MoeLaunch& L, int) {
    constexpr int W = 8;
    auto k = moe_down_kernel<GPK, ZP, P, W>;
    const size_t smem = std::max((size_t)W * P * 2 * L.tokens * QElem<false>::kRow, (size_t)W * 1024);
    int rc = reserve(reinterpret_cast<const void*>(k), smem);
    if (rc != PIVOT_OK) return rc;
    hipLaunchKernelGGL(k, dim3(L.nstrips[1]), dim3(W * 64), smem, reinterpret_cast<hipStream_t>(L.stream), L);
    return launched();
}

#define PIVOT_MOE_PICK(go, which)                                                                       \
    (L.zeros[which] ? (L.gpk[which] == 1 ? PIVOT_MOE_P(go, 1, true) : L.gpk[which] == 2 ? PIVOT_MOE_P(go, 2, true) : PIVOT_MOE_P(go, 4, true)) \
                    : (L.gpk[which] == 1 ? PIVOT_MOE_P(go, 1, false) : L.gpk[which] == 2 ? PIVOT_MOE_P(go, 2, false) : PIVOT_MOE_P(go, 4, false)))
#define PIVOT_MOE_P(go, gpk, zp) (L.tokens <= 4 ? go<gpk, zp, 4>(L, vec) : go<gpk, zp, 2>(L, vec))

}  // namespace

int launch_moe(const MoeLaunch& L) {
    hipStream_t st = reinterpret_cast<hipStream_t>(L.stream);
    const int vec = reinterpret_cast<uintptr_t>(L.x) % 16 == 0 && (L.ldx % 8 == 0 || L.tokens == 1), rvec = vec && L.D % 8 == 0;
    if (L.router_type == PIVOT_F16) hipLaunchKernelGGL(moe_router_kernel<_Float16>, dim3(L.E), dim3(kRouterThreads), 0, st, L, rvec);
    else                            hipLaunchKernelGGL(moe_router_kernel<float>, dim3(L.E), dim3(kRouterThreads), 0, st, L, rvec);
    int rc = launched();
    if (rc != PIVOT_OK) return rc;
    rc = PIVOT_MOE_PICK(up_go, 0);
    if (rc != PIVOT_OK) return rc;
    return PIVOT_MOE_PICK(down_go, 1);
}

}  // namespace pivot
