// The layer kernel of 4-bit plans and its launcher for one type of x (pivot_qfc_f16.hip, pivot_qfc_q8.hip).
#pragma once

#include <algorithm>
#include <type_traits>

#include "pivot_quant_core.h"

namespace pivot {

struct QfcArgs {
    const u32x4* codes; const uint16_t* scales; const uint8_t* zeros; const int32_t* chunks; const int32_t* pieces;
    const int32_t* prow; const float* bias; const float* xscale;
    QSource x;              // rows form: the rows; fragment form: x.x alone
    float* y; long long ldy; float* partials; uint32_t* tickets;
    int bh, bw_log2, batch, act, zero_chunk, whole, row_items;   // whole > 0: every tile is kept, so many blocks in each block row; row_items: items are whole block rows
};

// A work item: RS strips of a block row times a piece of its columns; blockIdx.x = piece * (strips / RS) + strip group.
template <int RS>
struct QfcItem {
    int br, sg, kb0, kb1, first, parts, slot, rowkb, nkb;     // blocks kb0..kb1 are numbered from the row's first
    size_t unit0;           // unit of block kb and strip r of the item: unit0 + r * nkb + kb
    __device__ __forceinline__ explicit QfcItem(const QfcArgs& a) {
        const int groups = a.bh / (kQStrip * RS), piece = blockIdx.x / groups;
        sg = blockIdx.x % groups;
        if (a.whole && a.row_items) {                    // every row as long as the others and in one piece: nothing to look up
            br = first = slot = piece; parts = 1; nkb = a.whole; rowkb = br * nkb; kb0 = rowkb; kb1 = rowkb + nkb;
        } else {
            const int32_t* ch = a.chunks + 8 * piece;
            br = ch[0]; kb0 = ch[1]; kb1 = ch[2]; first = ch[3]; parts = ch[4]; slot = ch[5]; rowkb = ch[6]; nkb = ch[7];
        }
        unit0 = (size_t)rowkb * (a.bh / kQStrip) + (size_t)(sg * RS) * nkb;      // units of a block row: strip-major
        kb0 -= rowkb;
        kb1 -= rowkb;
    }
};

// Sums of the wavefronts, through LDS (W * 16 RS * 16 NT floats at `red`); pieces of a row through memory; bias,
// activation and the scatter through prow.
// What the end of an item needs of memory, asked for at its beginning: where this thread's (first) output goes, its bias.
struct QfcEnd { int dst; float bias; };
template <int RS>
__device__ __forceinline__ QfcEnd qfc_end(const QfcArgs& a, const QfcItem<RS>& it) {
    const int row = it.br * a.bh + it.sg * 16 * RS + threadIdx.x % (16 * RS);
    return QfcEnd{a.prow[row], a.bias[row]};
}

template <bool Q8, bool ZP, int NT, int RS, int W>
__device__ __forceinline__ void qfc_finish(const QfcArgs& a, const QfcItem<RS>& it, const QfcEnd& end, const f32x4 (&acc)[RS][NT], float* red) {
    constexpr int N = 16 * RS * 16 * NT;
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = q_wave();
    __syncthreads();
    #pragma unroll
    for (int r = 0; r < RS; ++r)
        #pragma unroll
        for (int t = 0; t < NT; ++t)
            #pragma unroll
            for (int i = 0; i < 4; ++i)
                red[wave * N + (16 * t + (lane & 15)) * (16 * RS) + 16 * r + 4 * (lane >> 4) + i] = acc[r][t][i];
    __syncthreads();
    const int n_out = 16 * RS * a.batch;
    const size_t strip_off = (size_t)it.sg * n_out, slot_len = (size_t)a.bh * a.batch;
    if (it.parts > 1) {
        for (int e = tid; e < n_out; e += W * 64) {
            float s = 0.f;
            #pragma unroll
            for (int w = 0; w < W; ++w) s += red[w * N + e];
            agent_store(a.partials + it.slot * slot_len + strip_off + e, s);
        }
        // Every store of this workgroup is complete before its arrival is counted; the partial sums bypass the caches,
        // so nothing is written back or invalidated.
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            uint32_t* tk = a.tickets + ((size_t)it.br * (a.bh / kQStrip) + it.sg * RS) * kQTicketStride;
            const int last = __hip_atomic_fetch_add(tk, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(it.parts - 1);
            if (last) __hip_atomic_store(tk, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = last;
        }
        __syncthreads();
        if (!s_last) return;
    }
    for (int e = tid; e < n_out; e += W * 64) {
        const int n = e / (16 * RS);                      // (a thread's outputs are all of one row: 16 * RS divides W * 64)
        float s = 0.f;
        if (it.parts > 1) {
            for (int q = 0; q < it.parts; ++q) s += agent_load(a.partials + (it.first + q) * slot_len + strip_off + e);
        } else {
            #pragma unroll
            for (int w = 0; w < W; ++w) s += red[w * N + e];
        }
        if (Q8) s *= kQ8Factor<ZP> * a.xscale[n];
        s += end.bias;
        if (a.act == PIVOT_ACT_RELU && s < 0.f) s = 0.f;      // (a NaN stays one)
        if (end.dst >= 0) a.y[n * a.ldy + end.dst] = s;
    }
}

// Rows form, up to 16 batch rows: wavefront w takes the blocks w, w + W, ... of the item.  Eight wavefronts per item: sixteen
// were behind (2048x2048 3.9 -> 4.5 us, 4096x4096 4.95 -> 5.06), four only level where there are 1024 items.
// What bounds it: from 8192x8192 on, memory (16384x16384, batch 1 and 4, 138 MB with the scales, 29.5 us = 4.7 TB/s; a
// launch that only reads takes 29.8).  Below, one trip after the other: descriptor, codes and x, the sums' meeting, the
// store (4096x4096, 8.7 MB: 4.7 us, reading alone 3.5; 1000x1020: 4.0).  The operations of a unit, 57 of the vector units
// and 4 matrix instructions, would allow twice the memory's rate.
template <bool Q8, int GPK, bool ZP, int RS, bool FAST, int W>
__global__ void __launch_bounds__(W * 64, 4) qfc_rows_kernel(QfcArgs a) {
    extern __shared__ __align__(16) char smem[];
    const int wave = q_wave();
    const QfcItem<RS> it(a);
    const QfcEnd end = qfc_end(a, it);
    f32x4 acc[RS][1] = {};
    const QWalk k{a.codes, a.scales, a.zeros, a.whole ? nullptr : a.pieces + ((size_t)it.rowkb << (7 - a.bw_log2)), it.unit0, it.nkb, it.kb0 + wave, it.kb1, a.bw_log2};
    q_walk_rows<Q8, GPK, ZP, RS, FAST, W>(k, a.x, a.batch, [](int n) { return n; }, smem + wave * (2 * a.batch * QElem<Q8>::kRow), acc);
    qfc_finish<Q8, ZP, 1, RS, W>(a, it, end, acc, reinterpret_cast<float*>(smem));
}

// Fragment form: x lies in memory as the matrix instructions read it (qfc_gather_kernel), NT * 16 batch columns.  No LDS but
// for the sums.  What bounds it: the copy's launch (2-4 us of the whole) and, from batch 32 on, x out of the L2 caches, which
// every strip reads (4096x4096 fp16 batch 64: 134 MB of x against 9 of weights, 15.5 us), and the words of y, each a request of its
// own (50 % kept, 8-bit, batch 64: 255 thousand beside 300 thousand reads, 8.9 us, vector units busy 20 % of the time); two strips
// per item halve the reads where 256 items are left (16384x8192, batch 64, 80 -> 55 us).
template <bool Q8, int GPK, bool ZP, int NT, int RS, int W>
__global__ void __launch_bounds__(W * 64) qfc_frag_kernel(QfcArgs a) {
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, wave = q_wave();
    const QfcItem<RS> it(a);
    const QfcEnd end = qfc_end(a, it);
    f32x4 acc[RS][NT] = {};
    int at[NT];                                           // this lane's place in a chunk
    #pragma unroll
    for (int t = 0; t < NT; ++t) at[t] = (min(16 * t + (lane & 15), a.batch - 1) * 32 + 8 * (lane >> 4)) * QElem<Q8>::kBytes;
    const int32_t* pieces = a.pieces + ((size_t)it.rowkb << (7 - a.bw_log2));
    constexpr bool AHEAD = NT == 1;                       // more column tiles of x do not fit beside those in use
    struct Turn { QUnit<GPK, ZP> u[RS]; };
    struct Chunks { int c[4]; };
    auto chunks_of = [&](int kb) {                        // the chunk of x under each 32 columns of a block
        Chunks r;
        #pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 32 * j, in = c & ((1 << a.bw_log2) - 1), b = min(kb, it.kb1 - 1);
            const int piece = a.whole ? (b << 7) + c - in : pieces[(b << (7 - a.bw_log2)) + (c >> a.bw_log2)];
            r.c[j] = piece < 0 ? a.zero_chunk : min(a.zero_chunk, (piece + in) >> 5);
        }
        return r;
    };
    auto fetch = [&](Turn& t, int kb) {
        #pragma unroll
        for (int r = 0; r < RS; ++r) t.u[r].load(a.codes, a.scales, a.zeros, it.unit0 + (size_t)r * it.nkb + min(kb, it.kb1 - 1), lane);
    };
    auto fetch_x = [&](QFrag<Q8, NT>& x, const Chunks& ch) {
        #pragma unroll
        for (int j = 0; j < 4; ++j) x.load(reinterpret_cast<const char*>(a.x.x) + (size_t)ch.c[j] * a.batch * 32 * QElem<Q8>::kBytes, at, j);
    };
    // While a block is multiplied, the next one is on its way.  As in the rows form, no load depends on the sizes.
    const int kb0 = it.kb0 + wave;
    if (kb0 < it.kb1) {
        Turn t0, t1;
        QFrag<Q8, NT> x0, x1;
        Chunks c = chunks_of(kb0), d = chunks_of(kb0 + W);
        fetch(t0, kb0);
        if (AHEAD) fetch_x(x0, c);
        for (int kb = kb0;;) {
            if (AHEAD) { c = chunks_of(kb + 2 * W); fetch_x(x1, d); } else { fetch_x(x0, c); c = chunks_of(kb + 2 * W); }
            fetch(t1, kb + W);
            q_multiply<Q8, GPK, ZP, NT, RS>(t0.u, x0, acc);
            kb += W;
            if (kb >= it.kb1) break;
            if (AHEAD) { d = chunks_of(kb + 2 * W); fetch_x(x0, c); } else { fetch_x(x0, d); d = chunks_of(kb + 2 * W); }
            fetch(t0, kb + W);
            q_multiply<Q8, GPK, ZP, NT, RS>(t1.u, AHEAD ? x1 : x0, acc);
            kb += W;
            if (kb >= it.kb1) break;
        }
    }
    qfc_finish<Q8, ZP, NT, RS, W>(a, it, end, acc, reinterpret_cast<float*>(smem));
}

// The form a call takes: rows (frag = 0) or fragment, column tiles, strips per item, rows form: whether x is read as
// it lies; wavefronts of a workgroup.
struct QfcForm { int frag, nt, rs, fast; static constexpr int w = 8; };

inline size_t qfc_smem(const QfcForm& f, int batch, int row) {
    const size_t red = (size_t)f.w * 16 * f.rs * 16 * f.nt * 4;
    return f.frag ? red : std::max((size_t)f.w * 2 * batch * row, red);
}

template <typename K>
inline int qfc_go(K k, const QfcArgs& a, int grid, int w, size_t smem, void* stream) {
    const int rc = reserve_lds(reinterpret_cast<const void*>(k), smem);
    if (rc != PIVOT_OK) return rc;
    hipLaunchKernelGGL(k, dim3(grid), dim3(w * 64), smem, reinterpret_cast<hipStream_t>(stream), a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("launch failed: %s", hipGetErrorString(e)); return PIVOT_E_HIP; }
    return PIVOT_OK;
}

template <bool Q8, int GPK, bool ZP>
inline int qfc_pick(const QfcForm& f, const QfcArgs& a, int grid, size_t smem, void* stream) {
    auto go = [&](auto k) { return qfc_go(k, a, grid, f.w, smem, stream); };
    if (!f.frag) {
        if (!f.fast) return go(qfc_rows_kernel<Q8, GPK, ZP, 1, false, 8>);
        return f.rs == 1 ? go(qfc_rows_kernel<Q8, GPK, ZP, 1, true, 8>) : go(qfc_rows_kernel<Q8, GPK, ZP, 2, true, 8>);
    }
    if (f.nt == 1) {
        if (f.rs == 1) return go(qfc_frag_kernel<Q8, GPK, ZP, 1, 1, 8>);
        return go(qfc_frag_kernel<Q8, GPK, ZP, 1, 2, 8>);
    }
    if (f.nt == 2) return f.rs == 1 ? go(qfc_frag_kernel<Q8, GPK, ZP, 2, 1, 8>) : go(qfc_frag_kernel<Q8, GPK, ZP, 2, 2, 8>);
    return f.rs == 1 ? go(qfc_frag_kernel<Q8, GPK, ZP, 4, 1, 8>) : go(qfc_frag_kernel<Q8, GPK, ZP, 4, 2, 8>);
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
