// A mixture-of-experts layer for up to 16 tokens, three launches:
//
//   router   one workgroup per expert: its logit for every token; the last one to arrive ranks them, takes the softmax and
//            writes down which experts are in use, by which tokens
//   up       one workgroup per expert in use and strip of 16 rows (8 gate rows and their 8 up rows): silu(gate) * up,
//            stored in fp32, in the block order of the expert's down layer
//   down     one workgroup per strip of 16 outputs: all experts in use, one after the other, their sums weighted and added
//            in the accumulators.  The matrix instruction takes an activation as two fp16 numbers (see moe_down_kernel).  The tokens are the columns of the matrix instruction in every expert, so no expert's
//            output is ever stored and nothing is added across workgroups
//
// The weights of an expert in use are read once, whatever the number of its tokens.
//
// Us in a replayed graph, router / up / down: 1 token through 2 of 8 experts of 4096-8192-4096 (104 MB) 39 = 5 / 17 / 17,
// reading alone 14.5 and 8.4 for the two layers; 16 tokens through 51 of 64 experts of 2048-1408-2048 (242 MB) 89 = 9 / 42 / 44,
// reading alone 33 and 17; 4 tokens through 6.5 of 16 pruned experts 28.3 = 5 / 13 / 11, where the trips from the
// router's list to the first weights count, four or five before each of the two layers streams.  In the down layers the vector
// units are busy 71 and 76 % of the time (dequantising, and the activations into two fp16 numbers), in the gate/up layers 62 and 66.
#include <algorithm>
#include <type_traits>

#include "pivot_quant_core.h"

namespace pivot {

namespace {

constexpr int kRouterThreads = 1024;

template <bool VEC, typename T>
__device__ __forceinline__ void router_load8(const T* p, int c, int D, float (&v)[8]) {
    if constexpr (VEC) {
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

// The largest of 64 lanes (no NaNs), in every lane.
template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
    return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false)));
}
__device__ __forceinline__ float lane_of(float v, int l) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l));
}
__device__ __forceinline__ float wave_max(float v) {
    v = dpp_max<0x140>(dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(v))));
    return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
// ... of sixteen neighbouring lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
    return dpp_max<0x140>(dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(v))));
}
__device__ __forceinline__ float wave_sum(float v) {
    v = group_sum<16>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

// 16 wavefronts: TP tokens (the number of tokens, to the next power of two), 16 / TP wavefronts to each for the logit of
// expert blockIdx.x; in the last workgroup to arrive a wavefront per token for the choice, NQ experts to
// a lane.  ONE: a single workgroup, an expert per wavefront in turn, which saves the logits' way through memory.
// VEC: rows of x and of the router's matrix are whole 16-byte pieces (a template, so that a loop's loads go out together: 16
// tokens, 64 experts, 2048 columns 11.2 -> 9.0 us).
template <typename RT, int TP, int NQ, bool ONE, bool VEC>
__global__ void __launch_bounds__(kRouterThreads) moe_router_kernel(MoeLaunch a) {
    constexpr int S = 16 / TP, NW = sizeof(MoeExpert) / 8, NE = (64 * NQ * NW + kRouterThreads - 1) / kRouterThreads;
    __shared__ float s_red[16], s_logit[ONE ? TP : 1][ONE ? 64 * NQ : 1];
    __shared__ int   s_sel[kMoeMaxTokens][kMoeMaxTopK];
    __shared__ float s_w[kMoeMaxTokens][kMoeMaxTopK];
    __shared__ int   s_mask[kMoeMaxExperts], s_at[kMoeMaxExperts], s_base[4], s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = q_wave(), e = blockIdx.x, T = a.tokens, E = a.E, K = a.top_k;
    // the experts' layers, which the last workgroup will put beside what it finds, are asked for now
    unsigned long long layers[NE];
    #pragma unroll
    for (int i = 0; i < NE; ++i) layers[i] = tid + i * kRouterThreads < E * NW ? gload<unsigned long long>((const unsigned long long*)a.experts + tid + i * kRouterThreads) : 0;
    if constexpr (!ONE) {
        const int t = wave % TP;
        const RT* w = reinterpret_cast<const RT*>(a.router) + (long long)e * a.D;
        const _Float16* x = reinterpret_cast<const _Float16*>(a.x) + t * a.ldx;
        float acc = 0.f;
        if (t < T)
            #pragma unroll 4
            for (int c = ((wave / TP) * 64 + lane) * 8; c < a.D; c += S * 512) {
                float wv[8], xv[8];
                router_load8<VEC>(w, c, a.D, wv);
                router_load8<VEC>(x, c, a.D, xv);
                #pragma unroll
                for (int i = 0; i < 8; ++i) acc = __builtin_fmaf(wv[i], xv[i], acc);
            }
        acc = wave_sum(acc);
        if (lane == 0) s_red[wave] = acc;
    } else {
        for (int e1 = wave; e1 < E; e1 += 16) {
            const RT* w = reinterpret_cast<const RT*>(a.router) + (long long)e1 * a.D;
            float acc[TP] = {};
            #pragma unroll 2
            for (int c = lane * 8; c < a.D; c += 512) {
                float wv[8];
                router_load8<VEC>(w, c, a.D, wv);
                #pragma unroll
                for (int t = 0; t < TP; ++t)
                    if (t < T) {
                        float xv[8];
                        router_load8<VEC>(reinterpret_cast<const _Float16*>(a.x) + t * a.ldx, c, a.D, xv);
                        #pragma unroll
                        for (int i = 0; i < 8; ++i) acc[t] = __builtin_fmaf(wv[i], xv[i], acc[t]);
                    }
            }
            #pragma unroll
            for (int t = 0; t < TP; ++t) {
                const float s = wave_sum(acc[t]);
                if (lane == 0 && t < T) s_logit[t][e1] = s + (a.router_bias ? a.router_bias[e1] : 0.f);
            }
        }
    }
    __syncthreads();
    if (!ONE && tid < T) {
        float s = 0.f;
        #pragma unroll
        for (int q = 0; q < S; ++q) s += s_red[q * TP + tid];
        if (a.router_bias) s += a.router_bias[e];
        agent_store(a.logits + tid * E + e, s);
    }
    if (!ONE && wave == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the logits are out before the arrival is counted
    if (!ONE && tid == 0) {
        const int last = __hip_atomic_fetch_add(&a.route->ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(E - 1);
        if (last) __hip_atomic_store(&a.route->ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = last;
    }
    if (tid < kMoeMaxExperts) s_mask[tid] = 0;
    if (tid < kMoeMaxTokens * kMoeMaxTopK) { (&s_sel[0][0])[tid] = -1; (&s_w[0][0])[tid] = 0.f; }
    __syncthreads();
    if (!ONE && !s_last) return;

    // ---- the last workgroup: who uses what
    if (wave < T) {
        const float ninf = -__builtin_inff();
        const int t = wave;
        float v[NQ];
        int nan = 0;
        #pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const int i = lane + 64 * q;
            v[q] = i < E ? (ONE ? s_logit[t][i] : agent_load(a.logits + t * E + i)) : ninf;
            nan |= v[q] != v[q];
        }
        if (__any(nan)) {                                // the first top_k experts, with weights that are NaN
            if (lane < K) { s_sel[t][lane] = lane; s_w[t][lane] = __builtin_nanf(""); atomicOr(&s_mask[lane], 1 << t); }
        } else {
            float m = 0.f, s = 0.f, all = 0.f, mine = 0.f;   // mine: lane j's weight of choice j
            int chosen = -1, n = 0;
            for (int j = 0; j < K; ++j) {
                float top = v[0];
                #pragma unroll
                for (int q = 1; q < NQ; ++q) top = fmaxf(top, v[q]);
                top = wave_max(top);
                if (top == ninf) break;
                if (j == 0) {
                    m = top;
                    #pragma unroll
                    for (int q = 0; q < NQ; ++q) all += v[q] == ninf ? 0.f : expf(v[q] - m);
                }
                int at = -1;                             // the lowest index among equals
                #pragma unroll
                for (int q = NQ - 1; q >= 0; --q) {
                    const unsigned long long b = __ballot(v[q] == top);
                    if (b) at = 64 * q + __builtin_ctzll(b);
                }
                #pragma unroll
                for (int q = 0; q < NQ; ++q) if (lane + 64 * q == at) v[q] = ninf;
                const float p = expf(top - m);
                s += p;
                if (lane == j) { mine = p; chosen = at; }
                ++n;
            }
            if (!a.renormalise) s = wave_sum(all);
            if (lane < n) { s_sel[t][lane] = chosen; s_w[t][lane] = mine / s; atomicOr(&s_mask[chosen], 1 << t); }
        }
    }
    __syncthreads();
    // experts in use, in ascending order
    int mask = 0, at = 0, total = 0;
    unsigned long long used = 0;
    if (tid < kMoeMaxExperts) {
        mask = s_mask[tid];
        used = __ballot(mask != 0);
        if (lane == 0) s_base[wave] = __popcll(used);
    }
    __syncthreads();
    #pragma unroll
    for (int q = 0; q < 4; ++q) { if (q < wave) at += s_base[q]; total += s_base[q]; }
    at += __popcll(used & ((1ull << lane) - 1));
    if (tid < kMoeMaxExperts) s_at[tid] = at;
    if (mask) {
        unsigned long long tok = 0;
        for (int left = mask, m = 0; left; left &= left - 1, ++m) tok |= (unsigned long long)__builtin_ctz(left) << (4 * m);
        a.route->active[at].ntok = __popc(mask);
        a.route->active[at].mask = mask;
        a.route->active[at].tok = tok;
    }
    if (tid == 0) a.route->n = total;
    __syncthreads();
    if (tid < T * K) {
        const int t = tid / K, j = tid % K, ex = s_sel[t][j];
        const float w = s_w[t][j];
        a.route->sel[t][j] = ex;
        a.route->sel_w[t][j] = w;
        if (a.ids) a.ids[tid] = ex;
        if (a.weights) a.weights[tid] = w;
        if (ex >= 0) {
            MoeActive& act = a.route->active[s_at[ex]];
            const int m = __popc(s_mask[ex] & ((1 << t) - 1));
            act.hrow[m] = tid;
            act.share[t] = w;
        }
    }
    #pragma unroll
    for (int i = 0; i < NE; ++i) {
        const int at = tid + i * kRouterThreads, ex = at / NW;
        if (at < E * NW && s_mask[ex]) reinterpret_cast<unsigned long long*>(&a.route->active[s_at[ex]].ex)[at % NW] = layers[i];
    }
}

// gridDim.y: experts in use, at most; blockIdx.x: RS strips of a block row.  As the rows form of a layer, the rows of x
// being the expert's tokens.  Four wavefronts of at most 128 registers, so that four workgroups share a compute unit and one
// streams while another sets out (eight wavefronts of 170 registers: 22.3 us where this takes 17.5).
template <int GPK, bool ZP, int RS, bool FAST, int W>
__global__ void __launch_bounds__(W * 64, 4) moe_up_kernel(MoeLaunch a, int vec) {
    constexpr int N = 256 * RS;
    extern __shared__ __align__(16) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = q_wave(), T = a.tokens;
    const MoeActive& act = a.route->active[blockIdx.y];
    const MoeExpert& ex = act.ex;
    const int n_act = a.route->n, ntok = act.ntok, whole = ex.whole[0];
    const unsigned long long tok = act.tok;
    if ((int)blockIdx.y >= n_act) return;
    const int strip = blockIdx.x * RS, sb = a.bh[0] / kQStrip, br = strip / sb, bw_log2 = 31 - __clz(a.bw[0]);
    const int kb0 = whole ? br * whole : ex.kb_ptr[0][br], nkb = whole ? whole : ex.kb_ptr[0][br + 1] - kb0;
    // what the end needs is asked for now
    const int em = tid / (8 * RS), eu = tid % (8 * RS);
    int dst = -1, hrow = 0;
    float bg = 0.f, bu = 0.f;
    if (em < ntok) {
        dst = gload<int>(ex.hdst + strip * 8 + eu);
        hrow = act.hrow[em];
        bg = gload<float>(ex.bias[0] + strip * 16 + 2 * eu);
        bu = gload<float>(ex.bias[0] + strip * 16 + 2 * eu + 1);
    }
    f32x4 acc[RS][1] = {};
    const QWalk k{reinterpret_cast<const u32x4*>(ex.codes[0]), ex.scales[0], ex.zeros[0], whole ? nullptr : ex.pieces[0] + ((size_t)kb0 << (7 - bw_log2)),
                  (size_t)kb0 * sb + (size_t)(strip % sb) * nkb, nkb, wave, nkb, bw_log2};
    q_walk_rows<false, GPK, ZP, RS, FAST, W>(k, QSource{a.x, a.ldx, ex.pcol, a.D, vec}, ntok, [&](int m) { return (int)(tok >> (4 * m)) & 15; },
                                           smem + wave * (2 * T * QElem<false>::kRow), acc);
    __syncthreads();
    float* red = reinterpret_cast<float*>(smem);
    #pragma unroll
    for (int r = 0; r < RS; ++r)
        #pragma unroll
        for (int i = 0; i < 4; ++i) red[wave * N + (lane & 15) * (16 * RS) + 16 * r + 4 * (lane >> 4) + i] = acc[r][0][i];
    __syncthreads();
    if (blockIdx.x == 0)                                 // the columns that fill up the down layer's last tile
        for (int i = tid; i < ntok * (a.F_pad - a.F); i += W * 64)
            a.h[(size_t)act.hrow[i / (a.F_pad - a.F)] * a.F_pad + a.F + i % (a.F_pad - a.F)] = 0.f;
    static_assert(8 * RS * kMoeMaxTokens <= W * 64, "a thread has one unit of one token");
    if (em < ntok && dst >= 0) {
        #pragma unroll
        for (int w = 0; w < W; ++w) { bg += red[w * N + em * 16 * RS + 2 * eu]; bu += red[w * N + em * 16 * RS + 2 * eu + 1]; }
        a.h[(size_t)hrow * a.F_pad + dst] = bg / (1.f + expf(-bg)) * bu;
    }
}

// blockIdx.x: a strip of outputs; the units of all experts in use are one list, which the wavefronts of the strip's
// gridDim.y workgroups take in turn, P at a time.  Sixteen wavefronts share what a workgroup looks up first, and most strips
// need no hand-over (four wavefronts and parts in their place: 41.5 and 115 us for the layers above where this takes 39.6 and
// 91).  NT = 2: values and remainders of h are two column tiles; NT = 1 (up to 8 tokens): columns 0-7 and 8-15 of one.
//
// A token's activations under a unit are staged by the sixteen lanes that load them as 2^s h = value + remainder / 2^11, both
// fp16, s such that the largest of the unit's 128 lies in [2^14, 2^15); 2^-s multiplies the unit's sums.  The remainder of an
// activation in [2^e, 2^(e+1)) is at most half a step of the value, 2^(e-11), and half a step of the remainder 2^(e-23): the
// pair is off by one step of fp32 at most, or by 2^-50 of the largest activation (half the remainder's subnormal step) where
// that is more.  A single fp16 would be off by 2^-11.
//
// rows that a wavefront stages: at least the values and remainders of all tokens in one unit
template <int NT> constexpr int kDownRows = 16 * NT;
template <int GPK, bool ZP, int NT, int W>
__global__ void __launch_bounds__(W * 64, 4) moe_down_kernel(MoeLaunch a) {
    constexpr int ROW = QElem<false>::kRow, P = 2;       // (two units a turn: the list of rows is split in two)
    struct Down { const u32x4* codes; const uint16_t* scales; const uint8_t* zeros; const int32_t* pieces; };
    extern __shared__ __align__(16) char smem[];
    __shared__ Down s_ex[kMoeMaxActive];
    __shared__ int s_cum[kMoeMaxActive + 1], s_mask[kMoeMaxActive];
    __shared__ float s_share[kMoeMaxActive][kMoeMaxTokens];
    __shared__ uint8_t s_hrow[kMoeMaxActive][kMoeMaxTokens];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = q_wave(), T = a.tokens, n_act = a.route->n, parts = gridDim.y, step = W * parts;
    const int bound = min(a.E, T * a.top_k);            // at most so many experts in use: the loads that follow need not wait for n_act
    const int strip = blockIdx.x, sb = a.bh[1] / kQStrip, br = strip / sb, bw_log2 = 31 - __clz(a.bw[1]);
    if (wave == 0) {                                    // block counts of the experts in use, and their running sum
        int run = 0;
        for (int base = 0; base < bound; base += 64) {
            const int i = base + lane;
            int nkb = 0;
            const MoeExpert ex = a.route->active[min(i, bound - 1)].ex;
            const int its = a.route->active[min(i, bound - 1)].mask;
            if (i < n_act) {
                const int whole = ex.whole[1], kb0 = whole ? br * whole : ex.kb_ptr[1][br];
                nkb = whole ? whole : ex.kb_ptr[1][br + 1] - kb0;
                const size_t unit0 = (size_t)kb0 * sb + (size_t)(strip % sb) * nkb;
                s_ex[i] = Down{reinterpret_cast<const u32x4*>(ex.codes[1]) + unit0 * 64, ex.scales[1] + unit0 * GPK * kQStrip,
                               ZP ? ex.zeros[1] + unit0 * GPK * kQStrip : nullptr, whole ? nullptr : ex.pieces[1] + ((size_t)kb0 << (7 - bw_log2))};
                s_mask[i] = its;
            }
            int s = nkb;
            #pragma unroll
            for (int d = 1; d < 64; d <<= 1) { const int o = __shfl_up(s, d, 64); if (lane >= d) s += o; }
            if (i < n_act) s_cum[i + 1] = run + s;
            run += __shfl(s, 63, 64);
        }
        if (lane == 0) s_cum[0] = 0;
    } else {
        for (int i = tid - 64; i < bound * kMoeMaxTokens; i += (W - 1) * 64) {   // (of unused entries too: what they hold is not used)
            const MoeActive& act = a.route->active[i / kMoeMaxTokens];
            s_share[i / kMoeMaxTokens][i % kMoeMaxTokens] = act.share[i % kMoeMaxTokens];
            s_hrow[i / kMoeMaxTokens][i % kMoeMaxTokens] = (uint8_t)act.hrow[i % kMoeMaxTokens];
        }
    }
    __syncthreads();
    const int units = s_cum[n_act];
    // what the end needs is asked for now: this thread's output, its experts' biases
    static_assert(16 * kMoeMaxTokens <= W * 64, "a thread has one output");
    int e_dst = -1;
    float e_bias = 0.f;
    if (tid < 16 * T) {
        e_dst = a.prow_down[strip * 16 + tid % 16];
        for (int j = 0; j < a.top_k; ++j) {
            const int e = a.route->sel[tid / 16][j];
            if (e >= 0) e_bias = __builtin_fmaf(a.route->sel_w[tid / 16][j], gload<float>(a.experts[e].bias[1] + strip * 16 + tid % 16), e_bias);
        }
    }
    char* xs = smem + wave * (kDownRows<NT> * ROW);
    // this lane's column: a token, its value or (second half of a single tile) its remainder
    const int n = NT == 1 ? (lane & 7) : (lane & 15), second = NT == 1 ? (lane >> 3) & 1 : 0;
    f32x4 total[NT] = {};
    int cur = 0;
    // A turn: P units, the tokens of both as one list of which the first eight are asked for ahead.  As in the rows form every load is issued whatever the sizes: past the end the last unit's.
    constexpr int NX = 2;
    struct Turn { QUnit<GPK, ZP> u[P][1]; f32x4 v[NX][2]; int act[P], kb[P], mask[P], off[P + 1]; };
    const int c = 8 * (lane & 15), in = c & ((1 << bw_log2) - 1), slot = lane >> 4;
    auto column = [&](int act, int kb) {                // where this lane's columns of a block begin, F_pad and more: nowhere
        const int32_t* pieces = s_ex[act].pieces;
        const int piece = pieces ? gload<int>(pieces + (kb << (7 - bw_log2)) + (c >> bw_log2)) : (kb << 7) + c - in;
        return piece < 0 ? a.F_pad : piece + in;
    };
    auto load = [&](int act, int m, int col, f32x4 (&v)[2]) {              // of token m of the expert's
        const float* p = a.h + (size_t)s_hrow[act][m] * a.F_pad + min(col, a.F_pad - 8);   // (columns between F and F_pad hold zeros)
        v[0] = gload<f32x4>(p);
        v[1] = gload<f32x4>(p + 4);
        if (col >= a.F_pad) v[0] = v[1] = f32x4{};
    };
    auto stage = [&](const f32x4 (&v)[2], char* row, int ntok) {           // the remainders: ntok rows on; behind the values: 2^-s
        uint32_t most = 0;                              // as integers magnitudes are in order, infinities and NaNs last
        #pragma unroll
        for (int i = 0; i < 8; ++i) { const float f = v[i >> 2][i & 3]; most = max(most, __builtin_bit_cast(uint32_t, f) & 0x7fffffffu); }
        most = row16_max(most);
        const bool odd = most >= 0x7f800000u;           // (the unit's sums are infinite or NaN: no remainders)
        const int e = min(max((int)(most >> 23), 15), 254);                // 2^-s and 2^s are both normal numbers
        const float up = __builtin_bit_cast(float, (uint32_t)(268 - e) << 23);     // 2^(141 - e), e - 127 the exponent
        f16x8 hi, lo;
        #pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = v[i >> 2][i & 3] * up;
            hi[i] = (_Float16)x;
            lo[i] = odd ? (_Float16)0.f : (_Float16)((x - (float)hi[i]) * 2048.f);
        }
        q_store8<false>(row, lane & 15, __builtin_bit_cast(u32x4, hi));
        q_store8<false>(row + ntok * ROW, lane & 15, __builtin_bit_cast(u32x4, lo));
        if ((lane & 15) == 0) *reinterpret_cast<float*>(row + 2 * kQBlk) = __builtin_bit_cast(float, (uint32_t)(e - 14) << 23);
    };
    auto fetch = [&](Turn& t, int u0) {
        t.off[0] = 0;
        #pragma unroll
        for (int p = 0; p < P; ++p) {
            const int g = min(u0 + p * step, units - 1);
            while (g >= s_cum[cur + 1]) ++cur;
            t.act[p] = __builtin_amdgcn_readfirstlane(cur);
            t.kb[p] = __builtin_amdgcn_readfirstlane(g - s_cum[cur]);
            t.mask[p] = u0 + p * step < units ? __builtin_amdgcn_readfirstlane(s_mask[cur]) : 0;
            t.off[p + 1] = t.off[p] + __popc(t.mask[p]);
        }
        int act[NX], at[NX], col[NX];                   // this lane's token in each place of the list
        #pragma unroll
        for (int q = 0; q < NX; ++q) {
            const int i = max(0, min(slot + 4 * q, t.off[P] - 1));
            const bool first = i < t.off[1];
            act[q] = first ? t.act[0] : t.act[1];
            at[q] = first ? i : i - t.off[1];
            col[q] = column(act[q], first ? t.kb[0] : t.kb[1]);
        }
        #pragma unroll
        for (int p = 0; p < P; ++p) t.u[p][0].load(s_ex[t.act[p]].codes, s_ex[t.act[p]].scales, s_ex[t.act[p]].zeros, t.kb[p], lane);
        #pragma unroll
        for (int q = 0; q < NX; ++q) load(act[q], at[q], col[q], t.v[q]);
    };
    auto multiply_unit = [&](const Turn& t, int p, int at) {
        const int mask = t.mask[p], ntok = __popc(mask);
        const bool mine = (mask >> n) & 1;
        const int m = mine ? __popc(mask & ((1 << n) - 1)) : 0;
        int nrow[NT];
        #pragma unroll
        for (int q = 0; q < NT; ++q) nrow[q] = (at + m + (q + second) * ntok) * ROW;
        f32x4 part[1][NT] = {};
        const QRows<false, NT> x{xs, nrow, lane};
        q_multiply<false, GPK, ZP, NT, 1>(t.u[p], x, part);
        // tokens that do not use the expert: what their column held is dropped
        const float share = s_share[t.act[p]][n], down = *reinterpret_cast<const float*>(xs + (at + m) * ROW + 2 * kQBlk);
        #pragma unroll
        for (int q = 0; q < NT; ++q)
            #pragma unroll
            for (int i = 0; i < 4; ++i) total[q][i] = mine ? __builtin_fmaf(share, part[0][q][i] * down, total[q][i]) : total[q][i];
    };
    auto multiply = [&](const Turn& t) {
        const bool ahead = t.off[P] <= 4 * NX;
        if (ahead)
            #pragma unroll
            for (int q = 0; q < NX; ++q) {
                const int i = slot + 4 * q;
                const bool first = i < t.off[1];        // (before the second unit's rows: the first one's values and remainders)
                if (i < t.off[P]) stage(t.v[q], xs + (first ? i : t.off[1] + i) * ROW, first ? t.off[1] : t.off[P] - t.off[1]);
            }
        #pragma unroll
        for (int p = 0; p < P; ++p)
            if (t.mask[p]) {
                if (!ahead) {                           // many tokens on few experts: a unit's at a time
                    const int ntok = __popc(t.mask[p]), col = column(t.act[p], t.kb[p]);
                    for (int m = slot; m < ntok; m += 4) {
                        f32x4 v[2];
                        load(t.act[p], m, col, v);
                        stage(v, xs + m * ROW, ntok);
                    }
                }
                wave_lds_sync();
                multiply_unit(t, p, ahead ? 2 * t.off[p] : 0);
                __builtin_amdgcn_sched_barrier(0);
                wave_lds_sync();
            }
    };
    int u0 = wave + W * blockIdx.y;
    if (u0 < units) {
        Turn t0, t1;
        fetch(t0, u0);
        while (true) {
            fetch(t1, u0 + step * P);
            multiply(t0);
            u0 += step * P;
            if (u0 >= units) break;
            fetch(t0, u0 + step * P);
            multiply(t1);
            u0 += step * P;
            if (u0 >= units) break;
        }
    }
    __syncthreads();
    float* red = reinterpret_cast<float*>(smem);        // [wave][tile][column][row]
    #pragma unroll
    for (int t = 0; t < NT; ++t)
        #pragma unroll
        for (int i = 0; i < 4; ++i) red[(wave * NT + t) * 256 + (lane & 15) * 16 + 4 * (lane >> 4) + i] = total[t][i];
    __syncthreads();
    auto sum_of = [&](int i) {
        float s = 0.f, lo = 0.f;
        #pragma unroll
        for (int w = 0; w < W; ++w) { s += red[w * NT * 256 + i]; lo += red[w * NT * 256 + i + (NT == 1 ? 128 : 256)]; }
        return __builtin_fmaf(lo, 1.f / 2048.f, s);
    };
    float* mine = a.partials + (size_t)strip * parts * 16 * T;
    if (parts > 1) {                                    // handed over as the pieces of a block row of a layer are
        if (tid < 16 * T) agent_store(mine + blockIdx.y * 16 * T + tid, sum_of(tid));
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            uint32_t* tk = a.tickets + (size_t)strip * kQTicketStride;
            const int last = __hip_atomic_fetch_add(tk, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(parts - 1);
            if (last) __hip_atomic_store(tk, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = last;
        }
        __syncthreads();
        if (!s_last) return;
    }
    if (e_dst >= 0) {                                   // (of the first 16 T threads)
        float s = 0.f;
        if (parts > 1) { for (int q = 0; q < parts; ++q) s += agent_load(mine + q * 16 * T + tid); }
        else s = sum_of(tid);
        a.y[tid / 16 * a.ldy + e_dst] = s + e_bias;
    }
}

int launched() {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("launch failed: %s", hipGetErrorString(e)); return PIVOT_E_HIP; }
    return PIVOT_OK;
}

template <int GPK, bool ZP>
int up_go(const MoeLaunch& L, int vec) {
    auto go = [&](auto k, int rs, int w) {
        const size_t smem = std::max((size_t)w * 2 * L.tokens * QElem<false>::kRow, (size_t)w * 1024 * rs);
        const int rc = reserve_lds(reinterpret_cast<const void*>(k), smem);
        if (rc != PIVOT_OK) return rc;
        hipLaunchKernelGGL(k, dim3(L.nstrips[0] / rs, std::min(L.E, L.tokens * L.top_k)), dim3(w * 64), smem, reinterpret_cast<hipStream_t>(L.stream), L, vec);
        return launched();
    };
    const int most = std::min(2, L.bh[0] / kQStrip), active = std::min(L.E, L.tokens * L.top_k);
    int rs = 1;
    while (rs < most && L.nstrips[0] * active / (2 * rs) >= 512) rs *= 2;
    if (!(L.gather == 0 && vec && L.D % 8 == 0)) return rs == 1 ? go(moe_up_kernel<GPK, ZP, 1, false, 4>, 1, 4) : go(moe_up_kernel<GPK, ZP, 2, false, 4>, 2, 4);
    return rs == 1 ? go(moe_up_kernel<GPK, ZP, 1, true, 4>, 1, 4) : go(moe_up_kernel<GPK, ZP, 2, true, 4>, 2, 4);
}

template <int GPK, bool ZP>
int down_go(const MoeLaunch& L, int) {
    auto go = [&](auto k, int w, int rows) {
        // Workgroups of a strip: until there is one for every compute unit, with at least two units to a wavefront.
        const int units = L.down_blocks * std::min(L.E, L.tokens * L.top_k);
        int parts = 1;
        while (parts < kMoeMaxParts && L.nstrips[1] * parts < 256 && units >= 4 * w * parts) parts *= 2;
        const size_t smem = (size_t)w * rows * QElem<false>::kRow;      // more than the sums'
        const int rc = reserve_lds(reinterpret_cast<const void*>(k), smem);
        if (rc != PIVOT_OK) return rc;
        hipLaunchKernelGGL(k, dim3(L.nstrips[1], parts), dim3(w * 64), smem, reinterpret_cast<hipStream_t>(L.stream), L);
        return launched();
    };
    return L.tokens <= 8 ? go(moe_down_kernel<GPK, ZP, 1, 16>, 16, kDownRows<1>) : go(moe_down_kernel<GPK, ZP, 2, 16>, 16, kDownRows<2>);
}

template <typename RT, bool VEC>
int router_go(const MoeLaunch& L) {
    auto go = [&](auto k, int grid) {
        hipLaunchKernelGGL(k, dim3(grid), dim3(kRouterThreads), 0, reinterpret_cast<hipStream_t>(L.stream), L);
        return launched();
    };
    auto many = [&](auto nq) {
        constexpr int NQ = decltype(nq)::value;
        if (L.tokens == 1) return go(moe_router_kernel<RT, 1, NQ, false, VEC>, L.E);
        if (L.tokens == 2) return go(moe_router_kernel<RT, 2, NQ, false, VEC>, L.E);
        if (L.tokens <= 4) return go(moe_router_kernel<RT, 4, NQ, false, VEC>, L.E);
        if (L.tokens <= 8) return go(moe_router_kernel<RT, 8, NQ, false, VEC>, L.E);
        return go(moe_router_kernel<RT, 16, NQ, false, VEC>, L.E);
    };
    // One workgroup where a lane has at most 8 pieces of 16 bytes to load (16 experts, 512 columns, 1 token 16.5 -> 15.4 us for
    // the layer, 8 experts, 1024 columns 15.5 -> 14.7; with 16 pieces even, with 32 up to 9 us behind).
    const int loads = ((L.E + 15) / 16) * ((L.D + 511) / 512) * (1 + L.tokens);
    if (L.E <= 64 && L.tokens <= 4 && loads <= 8) return L.tokens == 1 ? go(moe_router_kernel<RT, 1, 1, true, VEC>, 1) : go(moe_router_kernel<RT, 4, 1, true, VEC>, 1);
    return L.E <= 64 ? many(std::integral_constant<int, 1>()) : many(std::integral_constant<int, 4>());
}

#define PIVOT_MOE_PICK(go, which)                                                                                          \
    (L.zeros[which] ? (L.gpk[which] == 1 ? go<1, true>(L, vec) : L.gpk[which] == 2 ? go<2, true>(L, vec) : go<4, true>(L, vec)) \
                    : (L.gpk[which] == 1 ? go<1, false>(L, vec) : L.gpk[which] == 2 ? go<2, false>(L, vec) : go<4, false>(L, vec)))

}  // namespace

int launch_moe(const MoeLaunch& L) {
    const int vec = reinterpret_cast<uintptr_t>(L.x) % 16 == 0 && (L.ldx % 8 == 0 || L.tokens == 1), rvec = vec && L.D % 8 == 0;
    int rc = L.router_type == PIVOT_F16 ? (rvec ? router_go<_Float16, true>(L) : router_go<_Float16, false>(L)) : (rvec ? router_go<float, true>(L) : router_go<float, false>(L));
    if (rc != PIVOT_OK) return rc;
    rc = PIVOT_MOE_PICK(up_go, 0);
    if (rc != PIVOT_OK) return rc;
    return PIVOT_MOE_PICK(down_go, 1);
}

}  // namespace pivot
