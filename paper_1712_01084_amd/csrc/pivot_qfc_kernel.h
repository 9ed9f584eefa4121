// The layer kernel of 4-bit plans and its launcher for one type of x (pivot_qfc_f16.hip, pivot_qfc_q8.hip).
#pragma once

#include <algorithm>
#include <type_traits>

#include "pivot_quant_core.h"

namespace pivot {

struct QfcArgs {
    const u32x4* codes; const uint16_t* scales; const int8_t* zoff; const int32_t* chunks; const int32_t* kb_ptr; const int32_t* pieces;
    const int32_t* prow; const float* bias; const float* xscale;
    QSource x;
    float* y; long long ldy; float* partials; uint32_t* tickets;
    int bh, bw_log2, batch, act;
};

// One work item: RS strips of a block row times a piece of its columns, NT * 16 batch columns; blockIdx.x = piece *
// (strips / RS) + strip group.  Wavefront w takes the blocks w, w + W, ... of the piece, P at a time: their codes and
// their columns of x are requested together, then multiplied.  The wavefronts' sums meet in LDS.
template <bool Q8, int GPK, bool ZP, int NT, int RS, int P, int W>
__global__ void __launch_bounds__(W * 64) qfc_kernel(QfcArgs a) {
    constexpr int ROW = QElem<Q8>::kRow, N = 16 * RS * 16 * NT;
    extern __shared__ __align__(16) char smem[];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int groups = a.bh / (kQStrip * RS);
    const int piece = blockIdx.x / groups, sg = blockIdx.x % groups;
    const int32_t* ch = a.chunks + 8 * piece;
    const int br = ch[0], kb0 = ch[1], kb1 = ch[2], first = ch[3], parts = ch[4], slot = ch[5];
    const int rowkb = a.kb_ptr[br], nkb = a.kb_ptr[br + 1] - rowkb;
    // units of a block row: strip-major
    const size_t unit0 = (size_t)rowkb * (a.bh / kQStrip) + (size_t)(sg * RS) * nkb - rowkb;
    char* xs = smem + wave * (P * a.batch * ROW);
    int nrow[NT];
    #pragma unroll
    for (int t = 0; t < NT; ++t) nrow[t] = min(16 * t + (lane & 15), a.batch - 1) * ROW;

    f32x4 acc[RS][NT] = {};
    const int sp = (lane >> 4) % P, c8 = lane & 15;
    for (int kb = kb0 + wave; kb < kb1; kb += W * P) {
        QUnit<GPK, ZP> u[P][RS];
        #pragma unroll
        for (int p = 0; p < P; ++p)
            if (kb + p * W < kb1)
                #pragma unroll
                for (int r = 0; r < RS; ++r) u[p][r].load(a.codes, a.scales, a.zoff, unit0 + (size_t)r * nkb + kb + p * W, lane);
        // staging: sixteen lanes take the columns of a unit, eight each
        const int skb = kb + sp * W;
        if (skb < kb1) {
            const int c = 8 * c8, piece0 = a.pieces[(skb << (7 - a.bw_log2)) + (c >> a.bw_log2)];
            const int col = piece0 < 0 ? a.x.K : piece0 + (c & ((1 << a.bw_log2) - 1));
            i32x4 idx[2] = {};
            if (a.x.pcol) {
                if (piece0 >= 0) { idx[0] = *reinterpret_cast<const i32x4*>(a.x.pcol + col); idx[1] = *reinterpret_cast<const i32x4*>(a.x.pcol + col + 4); }
                else { idx[0] = i32x4{-1, -1, -1, -1}; idx[1] = idx[0]; }
            }
            for (int n = (lane >> 4) / P; n < a.batch; n += 4 / P) {
                __align__(16) typename QElem<Q8>::type v[8];
                q_load8<Q8>(a.x, n, col, idx, v);
                q_store8<Q8>(xs + (sp * a.batch + n) * ROW, c8, v);
            }
        }
        wave_lds_sync();
        #pragma unroll
        for (int p = 0; p < P; ++p)
            if (kb + p * W < kb1) q_multiply<Q8, GPK, ZP, NT, RS>(u[p], xs + p * a.batch * ROW, nrow, lane, acc);
        wave_lds_sync();
    }

    // sums of the wavefronts: red[wave][row][batch column]
    __syncthreads();
    float* red = reinterpret_cast<float*>(smem);
    #pragma unroll
    for (int r = 0; r < RS; ++r)
        #pragma unroll
        for (int t = 0; t < NT; ++t)
            #pragma unroll
            for (int i = 0; i < 4; ++i)
                red[wave * N + (16 * t + (lane & 15)) * (16 * RS) + 16 * r + 4 * (lane >> 4) + i] = acc[r][t][i];
    __syncthreads();
    const int n_out = 16 * RS * a.batch;
    const size_t strip_off = (size_t)sg * n_out, slot_len = (size_t)a.bh * a.batch;
    if (parts > 1) {
        for (int e = tid; e < n_out; e += W * 64) {
            float s = 0.f;
            #pragma unroll
            for (int w = 0; w < W; ++w) s += red[w * N + e];
            agent_store(a.partials + slot * slot_len + strip_off + e, s);
        }
        // Every store of this workgroup is complete before its arrival is counted; the partial sums bypass the caches,
        // so nothing is written back or invalidated.
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            uint32_t* tk = a.tickets + ((size_t)br * (a.bh / kQStrip) + sg * RS) * kQTicketStride;
            const int last = __hip_atomic_fetch_add(tk, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(parts - 1);
            if (last) __hip_atomic_store(tk, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = last;
        }
        __syncthreads();
        if (!s_last) return;
    }
    for (int e = tid; e < n_out; e += W * 64) {
        const int row = br * a.bh + sg * 16 * RS + e % (16 * RS), n = e / (16 * RS), dst = a.prow[row];
        float s = 0.f;
        if (parts > 1) {
            for (int q = 0; q < parts; ++q) s += agent_load(a.partials + (first + q) * slot_len + strip_off + e);
        } else {
            #pragma unroll
            for (int w = 0; w < W; ++w) s += red[w * N + e];
        }
        if (Q8) s *= 0.0625f * a.xscale[n];
        if (dst >= 0) a.y[n * a.ldy + dst] = apply_act(s + a.bias[row], a.act);
    }
}

// Batch columns, strips per wavefront, blocks in flight per wavefront and wavefronts of the form a call takes.
struct QfcForm { int nt, rs, p, w; };

inline QfcForm qfc_form(const QfcHost& h, int batch) {
    const int rs2 = h.d.bh >= 32 ? 2 : 1;
    if (batch <= 4) return {1, 1, 4, 8};
    if (batch <= 16) return {1, 1, 2, 8};
    if (batch <= 32) return {2, rs2, 1, 8};
    return {4, rs2, 1, 4};
}

inline size_t qfc_smem(const QfcForm& f, int batch, int row) {
    return std::max((size_t)f.w * f.p * batch * row, (size_t)f.w * 16 * f.rs * 16 * f.nt * 4);
}

template <bool Q8, int GPK, bool ZP, int NT, int RS, int P, int W>
inline int qfc_go(const QfcArgs& a, int grid, size_t smem, void* stream) {
    auto k = qfc_kernel<Q8, GPK, ZP, NT, RS, P, W>;
    if (smem > 64 * 1024) {
        // asked for on every call: the attribute belongs to the device that is current
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != hipSuccess) {
            (void)hipGetLastError();
            set_error("cannot reserve %zu bytes of LDS", smem);
            return PIVOT_E_HIP;
        }
    }
    hipLaunchKernelGGL(k, dim3(grid), dim3(W * 64), smem, reinterpret_cast<hipStream_t>(stream), a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("launch failed: %s", hipGetErrorString(e)); return PIVOT_E_HIP; }
    return PIVOT_OK;
}

template <bool Q8, int GPK, bool ZP>
inline int qfc_pick(const QfcForm& f, const QfcArgs& a, int grid, size_t smem, void* stream) {
    if (f.nt == 1) return f.p == 4 ? qfc_go<Q8, GPK, ZP, 1, 1, 4, 8>(a, grid, smem, stream) : qfc_go<Q8, GPK, ZP, 1, 1, 2, 8>(a, grid, smem, stream);
    if (f.nt == 2) return f.rs == 2 ? qfc_go<Q8, GPK, ZP, 2, 2, 1, 8>(a, grid, smem, stream) : qfc_go<Q8, GPK, ZP, 2, 1, 1, 8>(a, grid, smem, stream);
    return f.rs == 2 ? qfc_go<Q8, GPK, ZP, 4, 2, 1, 4>(a, grid, smem, stream) : qfc_go<Q8, GPK, ZP, 4, 1, 1, 4>(a, grid, smem, stream);
}

template <bool Q8>
inline int qfc_dispatch(const QfcHost& h, const QfcForm& f, const QfcArgs& a, void* stream) {
    const int grid = h.nchunks * (h.d.bh / (kQStrip * f.rs));
    const size_t smem = qfc_smem(f, a.batch, QElem<Q8>::kRow);
    if (h.has_zeros) {
        if (h.gpk == 1) return qfc_pick<Q8, 1, true>(f, a, grid, smem, stream);
        if (h.gpk == 2) return qfc_pick<Q8, 2, true>(f, a, grid, smem, stream);
        return qfc_pick<Q8, 4, true>(f, a, grid, smem, stream);
    }
    if (h.gpk == 1) return qfc_pick<Q8, 1, false>(f, a, grid, smem, stream);
    if (h.gpk == 2) return qfc_pick<Q8, 2, false>(f, a, grid, smem, stream);
    return qfc_pick<Q8, 4, false>(f, a, grid, smem, stream);
}

int qfc_launch_f16(const QfcHost& h, const QfcForm& f, const QfcArgs& a, void* stream);
int qfc_launch_q8(const QfcHost& h, const QfcForm& f, const QfcArgs& a, void* stream);

}  // namespace pivot
