// Layers with 4-bit weights: laying the weights out on the device, and the choice of a launch.
#include "pivot_qfc_kernel.h"

namespace pivot {

// One wavefront per unit: lane l gathers the 32 codes of row l % 16 that it will multiply, and the unit's scales.
__global__ void __launch_bounds__(64) qfc_pack_kernel(u32x4* codes, uint16_t* scales, int8_t* zoff, const uint8_t* raw_codes,
                                                      const uint16_t* raw_scales, const uint8_t* raw_zeros, const int32_t* row_of_kb,
                                                      const int32_t* kb_ptr, const int32_t* pieces, int M, int K, int bh, int bw, int group, int gpk) {
    const int lane = threadIdx.x, kb = blockIdx.x, s = blockIdx.y;
    const int br = row_of_kb[kb], first = kb_ptr[br], nkb = kb_ptr[br + 1] - first, ppb = kQBlk / bw;
    const size_t unit = (size_t)first * (bh / kQStrip) + (size_t)s * nkb + (kb - first);
    const int row = br * bh + s * kQStrip + (lane & 15);
    const long long code_ld = (K + 1) / 2, group_ld = (K + group - 1) / group;
    uint32_t w[4];
    for (int j = 0; j < 4; ++j) {
        w[j] = 0;
        for (int i = 0; i < 8; ++i) {
            const int c = 32 * j + 8 * (lane >> 4) + q_nibble_col(i);
            const int p = pieces[kb * ppb + c / bw], col = p + c % bw;
            uint32_t q = 8;                                     // padding: a weight of zero
            if (p >= 0 && row < M && col < K) q = (raw_codes[row * code_ld + col / 2] >> (4 * (col & 1))) & 15u;
            w[j] |= q << (4 * i);
        }
    }
    codes[unit * 64 + lane] = u32x4{w[0], w[1], w[2], w[3]};
    for (int e = lane; e < gpk * kQStrip; e += 64) {
        const int g = e / kQStrip, r = br * bh + s * kQStrip + e % kQStrip, c = g * (kQBlk / gpk);
        const int p = pieces[kb * ppb + c / bw], col = p + c % bw;
        const bool real = p >= 0 && r < M && col < K;
        scales[(unit * gpk + g) * kQStrip + e % kQStrip] = real ? raw_scales[r * group_ld + col / group] : (uint16_t)0;
        if (zoff) zoff[(unit * gpk + g) * kQStrip + e % kQStrip] = real ? (int8_t)((int)raw_zeros[r * group_ld + col / group] - 8) : (int8_t)0;
    }
}

int launch_qfc_pack(const QfcHost& h, const QfcDev& d, const uint8_t* raw_codes, const uint16_t* raw_scales, const uint8_t* raw_zeros,
                    const int32_t* row_of_kb) {
    if (h.KB == 0) return PIVOT_OK;
    hipLaunchKernelGGL(qfc_pack_kernel, dim3(h.KB, h.strips()), dim3(64), 0, nullptr, reinterpret_cast<u32x4*>(d.codes), d.scales, d.zoff, raw_codes, raw_scales, raw_zeros,
                       row_of_kb, d.kb_ptr, d.pieces, h.d.M, h.d.K, h.d.bh, h.d.bw, h.d.group, h.gpk);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
    if (e != hipSuccess) { set_error("laying out the weights failed: %s", hipGetErrorString(e)); return PIVOT_E_HIP; }
    return PIVOT_OK;
}

int launch_qfc(const QfcLaunch& L, std::string* describe) {
    const QfcHost& h = *L.h;
    const bool q8 = L.xtype == PIVOT_Q8;
    const QfcForm f = qfc_form(h, L.batch);
    if (describe) {
        char buf[160];
        snprintf(buf, sizeof(buf), "pivot::qfc_kernel<%s, %d, %s, %d, %d, %d, %d>", q8 ? "true" : "false", h.gpk, h.has_zeros ? "true" : "false", f.nt, f.rs, f.p, f.w);
        *describe = buf;
        return PIVOT_OK;
    }
    const QfcDev& d = *L.d;
    const int es = q8 ? 1 : 2, piece = 8 * es;
    QfcArgs a{};
    a.codes = reinterpret_cast<const u32x4*>(d.codes); a.scales = d.scales; a.zoff = d.zoff; a.chunks = d.chunks; a.kb_ptr = d.kb_ptr; a.pieces = d.pieces;
    a.prow = d.prow_pad; a.bias = d.bias_p; a.xscale = L.xscale;
    a.x = QSource{L.x, L.ldx, (L.block_order || h.identity_cols) ? nullptr : d.pcol_pad, h.d.K,
                  reinterpret_cast<uintptr_t>(L.x) % piece == 0 && (L.ldx * es % piece == 0 || L.batch == 1)};
    a.y = L.y; a.ldy = L.ldy; a.partials = L.partials; a.tickets = L.tickets;
    a.bh = h.d.bh; a.bw_log2 = h.d.bw == 32 ? 5 : (h.d.bw == 64 ? 6 : 7); a.batch = L.batch; a.act = h.d.act;
    return q8 ? qfc_launch_q8(h, f, a, L.stream) : qfc_launch_f16(h, f, a, L.stream);
}

}  // namespace pivot
