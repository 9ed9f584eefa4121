// Layers with 4-bit weights: laying the weights out on the device, and the choice of a launch.
#include <algorithm>
#include <mutex>
#include <unordered_map>

#include "pivot_qfc_kernel.h"

namespace pivot {

// What laying out needs.
struct QfcPack {
    u32x4* codes; uint16_t* scales; uint8_t* zeros; const uint8_t* raw_codes; const uint16_t* raw_scales; const uint8_t* raw_zeros;
    const int32_t* row_of_kb; const int32_t* kb_ptr; const int32_t* pieces; int32_t* bad;
    int M, K, bh, bw, group, gpk;
};

int reserve_lds(const void* kernel, size_t bytes) {
    constexpr int kMost = 144 * 1024;                            // leaves 16 KB of a compute unit for what kernels declare
    if (bytes <= 64 * 1024) return PIVOT_OK;
    static std::mutex lock;
    static std::unordered_map<const void*, uint64_t> done;     // a bit per device
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess && bytes <= kMost) {
        const uint64_t bit = dev < 64 ? 1ull << dev : 0;
        std::lock_guard<std::mutex> g(lock);
        try {
            uint64_t& known = done[kernel];
            if (known & bit) return PIVOT_OK;
            e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kMost);
            if (e == hipSuccess) { known |= bit; return PIVOT_OK; }
        } catch (...) {                                          // no memory to note it in
            e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
            if (e == hipSuccess) return PIVOT_OK;
        }
    }
    (void)hipGetLastError();
    set_error("cannot reserve %zu bytes of LDS", bytes);
    return PIVOT_E_HIP;
}

// One wavefront per unit: lane l gathers the 32 codes of row l % 16 that it will multiply, eight neighbouring columns of the
// caller's rows at a time, and the unit's scales.  bad: set where a zero point is above 15.
__global__ void __launch_bounds__(256) qfc_pack_kernel(QfcPack p, int kb0, int kb1) {
    const int lane = threadIdx.x & 63, kb = kb0 + blockIdx.x * 4 + q_wave(), s = blockIdx.y;
    if (kb >= kb1) return;
    const int br = p.row_of_kb[kb], first = p.kb_ptr[br], nkb = p.kb_ptr[br + 1] - first, ppb = kQBlk / p.bw, row0 = br * p.bh + s * kQStrip;
    const size_t unit = (size_t)first * (p.bh / kQStrip) + (size_t)s * nkb + (kb - first);
    const int row = row0 + (lane & 15);
    const long long code_ld = (p.K + 1) / 2, group_ld = (p.K + p.group - 1) / p.group;
    uint32_t w[4];
    #pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = 32 * j + 8 * (lane >> 4), piece = p.pieces[(size_t)kb * ppb + c / p.bw], col = piece + c % p.bw;
        uint32_t v = 0x88888888u;                               // padding: weights of zero
        if (piece >= 0 && row < p.M && col < p.K) {
            const uint8_t* q = p.raw_codes + row * code_ld + col / 2;
            if (col + 8 <= p.K) {
                typedef uint32_t word_any __attribute__((aligned(1)));
                v = *reinterpret_cast<const word_any*>(q);
            } else
                for (int i = 0; i < p.K - col; ++i) v = (v & ~(15u << (4 * i))) | (uint32_t)((q[i / 2] >> (4 * (i & 1))) & 15) << (4 * i);
        }
        // nibble i holds column q_nibble_col(i): the even columns, then the odd ones
        const auto gather = [](uint32_t n) { n &= 0x0f0f0f0fu; n = (n | n >> 4) & 0x00ff00ffu; return (n | n >> 8) & 0xffffu; };
        w[j] = gather(v) | gather(v >> 4) << 16;
    }
    p.codes[unit * 64 + lane] = u32x4{w[0], w[1], w[2], w[3]};
    for (int e = lane; e < p.gpk * kQStrip; e += 64) {
        const int g = e / kQStrip, i = e % kQStrip, r = row0 + i, c = g * (kQBlk / p.gpk);
        const int piece = p.pieces[(size_t)kb * ppb + c / p.bw], col = piece + c % p.bw;
        const bool real = piece >= 0 && r < p.M && col < p.K;
        const long long at = r * group_ld + col / p.group;
        p.scales[((unit * 4 + i / 4) * p.gpk + g) * 4 + i % 4] = real ? p.raw_scales[at] : (uint16_t)0;
        if (p.zeros) {
            const uint8_t z = real ? p.raw_zeros[at] : (uint8_t)8;
            p.zeros[(unit * kQStrip + i) * p.gpk + g] = z;
            if (z > 15) *p.bad = 1;
        }
    }
}
static_assert(q_nibble_col(1) == 2 && q_nibble_col(3) == 6 && q_nibble_col(4) == 1 && q_nibble_col(7) == 7, "the order of the nibbles");

// The bias in block order.
__global__ void __launch_bounds__(256) qfc_bias_kernel(float* bias_p, const float* bias, const int32_t* prow, int M_pad) {
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r < M_pad) bias_p[r] = prow[r] >= 0 ? bias[prow[r]] : 0.f;
}

int launch_qfc_pack(const QfcHost& h, const QfcDev& d, const uint8_t* raw_codes, const uint16_t* raw_scales, const uint8_t* raw_zeros,
                    const float* raw_bias, int32_t* bad) {
    const QfcPack p{reinterpret_cast<u32x4*>(d.codes), d.scales, d.zeros, raw_codes, raw_scales, raw_zeros, d.row_of_kb, d.kb_ptr, d.pieces,
                    bad, h.d.M, h.d.K, h.d.bh, h.d.bw, h.d.group, h.gpk};
    constexpr int kSlice = 1 << 24;                             // (a launch has less than 2^32 threads)
    for (int kb = 0; kb < h.KB; kb += kSlice) {
        const int end = std::min(h.KB, kb + kSlice);
        hipLaunchKernelGGL(qfc_pack_kernel, dim3((end - kb + 3) / 4, h.strips()), dim3(256), 0, nullptr, p, kb, end);
    }
    if (raw_bias) hipLaunchKernelGGL(qfc_bias_kernel, dim3((h.M_pad + 255) / 256), dim3(256), 0, nullptr, d.bias_p, raw_bias, d.prow_pad, h.M_pad);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("laying out the weights failed: %s", hipGetErrorString(e)); return PIVOT_E_HIP; }
    return PIVOT_OK;
}

// Copy of x for the product kernels, eight columns per thread.  frag: chunks of 32 block-space columns, in each the batch
// rows side by side (8 bits: eight columns in nibble order), and one chunk of zeros behind the last; else rows of K_pad
// columns in block order.
template <bool Q8>
__global__ void __launch_bounds__(256) qfc_gather_kernel(QSource x, void* out, int batch, int K_pad, int frag) {
    const int chunks = K_pad / 32, n8 = (frag ? chunks + 1 : chunks) * batch * 4, i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n8) return;
    int n, col;
    if (frag) { n = (i >> 2) % batch; col = ((i >> 2) / batch) * 32 + 8 * (i & 3); }
    else { n = i / (4 * chunks); col = 8 * (i % (4 * chunks)); }
    i32x4 idx[2] = {i32x4{-1, -1, -1, -1}, i32x4{-1, -1, -1, -1}};
    if (x.pcol && col < K_pad) { idx[0] = gload<i32x4>(x.pcol + col); idx[1] = gload<i32x4>(x.pcol + col + 4); }
    q_eight<Q8> v = q_load8<Q8>(x, n, col, idx);      // zeros past the last column
    if constexpr (Q8) if (frag) v = q_nibble_order(v);
    reinterpret_cast<q_eight<Q8>*>(out)[i] = v;
}

// The form of a call.  as_it_lies: x can be read in whole pieces of eight columns; *copy: x is copied first, in block order
// (rows form) or fragment order.  Us, rows form / fragment form with its copy, x as it lies: 4096x4096 batch 5, 8, 16 5.4 /
// 7.8, 5.8 / 7.8, 8.2 / 8.3; beyond that the fragment form reads x once per column tile and the rows form once per strip.
// Where x has to be gathered, a copy costs a launch (1.2 - 1.8 us) and saves a gather per strip: rows form gathering / with
// a copy / fragment form,
//   4096x4096 batch 2, 4     6.7 / 7.5    8.6 / 7.7          (2.1 and 4.2 million elements of x gathered)
//   8192x8192 25 %, 2, 4     8.9 / 8.7   13.0 / 8.8          (2.1 and 4.2)
//   4096x2048 50 %, 4        5.8 / 6.4                       (1.0)
//   2048x2048 50 %, 5, 8     6.3 / 6.6 / 6.6    7.5 / 7.1 / 6.9     (0.7, 1.0)
//   4096x4096, 5, 8, 16      9.8 / 8.1 / 8.8   12.9 / 9.3 / 9.4   24.0 / 11.9 / 10.4
//   512x512, 8, 16           5.1 / 6.3 / 6.2    6.6 / 7.3 / 6.3     (0.1, 0.3)
// Two strips per item wherever 256 items are left, one for every compute unit: x is then staged or read half as often
// (16384x4096 batch 1 12.5 -> 10.4 us, 8192x8192 11.2 -> 9.9, batch 64 29.4 -> 24.7; 4096x4096 batch 64, with 128 items
// instead of 256, 11.6 -> 13.5).
static QfcForm qfc_form(const QfcHost& h, int batch, bool as_it_lies, bool* copy) {
    const int strips = h.nchunks * h.strips();
    const size_t staged = h.units() * kQBlk * batch;                  // elements of x that the rows form stages
    QfcForm f{};
    f.nt = batch <= 16 ? 1 : (batch <= 32 ? 2 : 4);
    if (batch > 16) f.frag = 1;
    else if (as_it_lies) f.frag = batch > 8 && staged > ((size_t)1 << 24);
    else f.frag = batch > 8 && staged > 300000;
    *copy = f.frag || (!as_it_lies && staged > (batch <= 4 ? (size_t)2 << 20 : (size_t)1 << 20));
    f.fast = !f.frag && (as_it_lies || *copy);
    f.rs = h.strips() >= 2 && strips >= 512 && (f.frag || f.fast) ? 2 : 1;
    return f;
}

size_t qfc_copy_bytes(const QfcHost& h, int batch) { return align_up((size_t)(h.K_pad + 32) * batch * 2, 256); }

int launch_qfc(const QfcLaunch& L, std::string* describe) {
    const QfcHost& h = *L.h;
    const bool q8 = L.xtype == PIVOT_Q8, gathered = !(L.block_order || h.identity_cols);
    const int es = q8 ? 1 : 2, piece = 8 * es;
    const bool vec = reinterpret_cast<uintptr_t>(L.x) % piece == 0 && (L.ldx * es % piece == 0 || L.batch == 1);
    bool copy = false;
    const QfcForm f = qfc_form(h, L.batch, !gathered && vec && h.d.K % 8 == 0, &copy);
    if (describe) {
        char buf[160];
        const char *x = q8 ? "true" : "false", *z = h.has_zeros ? "true" : "false";
        if (f.frag) snprintf(buf, sizeof(buf), "pivot::qfc_frag_kernel<%s, %d, %s, %d, %d, %d>", x, h.gpk, z, f.nt, f.rs, f.w);
        else        snprintf(buf, sizeof(buf), "pivot::qfc_rows_kernel<%s, %d, %s, %d, %s, %d>", x, h.gpk, z, f.rs, f.fast ? "true" : "false", f.w);
        *describe = buf;
        return PIVOT_OK;
    }
    const QfcDev& d = *L.d;
    QfcArgs a{};
    a.codes = reinterpret_cast<const u32x4*>(d.codes); a.scales = d.scales; a.zeros = d.zeros; a.chunks = d.chunks; a.pieces = d.pieces;
    a.prow = d.prow_pad; a.bias = d.bias_p; a.xscale = L.xscale;
    a.x = QSource{L.x, L.ldx, gathered ? d.pcol_pad : nullptr, h.d.K, vec};
    a.y = L.y; a.ldy = L.ldy; a.partials = L.partials; a.tickets = L.tickets;
    a.bh = h.d.bh; a.bw_log2 = h.d.bw == 32 ? 5 : (h.d.bw == 64 ? 6 : 7); a.batch = L.batch; a.act = h.d.act; a.zero_chunk = h.K_pad / 32; a.whole = h.whole ? h.max_kb : 0; a.row_items = h.nchunks == h.nbr;
    if (copy) {
        const int blocks = ((h.K_pad / 32 + 1) * L.batch * 4 + 255) / 256;
        hipStream_t st = reinterpret_cast<hipStream_t>(L.stream);
        if (q8) hipLaunchKernelGGL(qfc_gather_kernel<true>, dim3(blocks), dim3(256), 0, st, a.x, L.xcopy, L.batch, h.K_pad, f.frag);
        else    hipLaunchKernelGGL(qfc_gather_kernel<false>, dim3(blocks), dim3(256), 0, st, a.x, L.xcopy, L.batch, h.K_pad, f.frag);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) { set_error("launch failed: %s", hipGetErrorString(e)); return PIVOT_E_HIP; }
        a.x = QSource{L.xcopy, h.K_pad, nullptr, h.K_pad, 1};
    }
    return q8 ? qfc_launch_q8(h, f, a, L.stream) : qfc_launch_f16(h, f, a, L.stream);
}

}  // namespace pivot
