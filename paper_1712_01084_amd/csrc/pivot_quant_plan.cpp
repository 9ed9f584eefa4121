// Host-side plan of a layer with 4-bit weights: pure CPU code, integer work only (the codes are laid out on the device).
#include <algorithm>
#include <new>
#include <numeric>

#include "pivot_quant.h"

namespace pivot {

static bool invert(const int32_t* p, int n, std::vector<int32_t>& inv) {
    inv.assign(n, -1);
    for (int i = 0; i < n; ++i) {
        if (p[i] < 0 || p[i] >= n || inv[p[i]] >= 0) return false;
        inv[p[i]] = i;
    }
    return true;
}

// Work items: whole block rows where they fill the device.  A row in pieces pays a hand-over between workgroups of 0.8 us,
// so it is cut only into pieces of at least 32 blocks (32 KB per strip) and while they leave half of 256 compute units
// idle: us at batch 1, whole / pieces of 64 / 32 / 16 blocks, dense, 2048x4096 4.7 / - / 4.7 / 5.5, 512x16384 9.2 / 7.5 / 6.5 /
// 7.2, 2048x16384 10.4 / 9.0 / 9.5 / 11.0, 3000x16384 10.7 / 11.4 / 12.0 / 15.9.  Or where the longest row has 64 blocks and
// four times the average (then pieces of twice the average, at least 16): 16384x8192, 10 % kept, rows 1 : 30, 10.5 / 10.5 /
// 8.7 / 7.8.
static int choose_chunk_blocks(const QfcHost& h) {
    if (h.d.chunk_blocks > 0) return h.d.chunk_blocks;
    const int strips = std::max(1, h.nbr * h.strips()), most = std::max(1, h.max_kb);
    int parts = 1;
    while (strips * parts * 2 <= 256 && most / (2 * parts) >= 32) parts *= 2;
    int ck = (most + parts - 1) / parts;
    if (most >= 64 && (long long)most * h.nbr >= 4LL * h.KB) ck = std::min(ck, std::max(16, 2 * ((h.KB + h.nbr - 1) / h.nbr)));
    return ck;
}

int build_qfc_host(const pivot_qfc_desc& d, const uint8_t* zeros, int64_t groups, const uint8_t* tile_mask, const int32_t* prow,
                   const int32_t* pcol, const float* bias, QfcHost& h) try {
    auto unsupported = [](const char* m) { set_error("%s", m); return PIVOT_E_UNSUPPORTED; };
    if (d.M < 1 || d.K < 1) { set_error("M and K must be positive"); return PIVOT_E_SHAPE; }
    if (d.M > kQMaxM || d.K > kQMaxK) return unsupported("4-bit layers take at most 2^22 rows and 65535 columns");
    if (d.bh != 16 && d.bh != 32 && d.bh != 64) return unsupported("tile rows of a 4-bit layer must be 16, 32 or 64");
    if (d.bw != 32 && d.bw != 64 && d.bw != 128) return unsupported("tile columns of a 4-bit layer must be 32, 64 or 128");
    if (d.group != 32 && d.group != 64 && d.group != 128) return unsupported("the group of a 4-bit layer must be 32, 64 or 128 columns");
    if (d.act != PIVOT_ACT_NONE && d.act != PIVOT_ACT_RELU) return unsupported("unknown activation");
    if (d.flags & ~PIVOT_QFC_WEIGHTS_ON_DEVICE) return unsupported("unknown flags");
    if (d.chunk_blocks < 0) { set_error("chunk_blocks must not be negative"); return PIVOT_E_SHAPE; }
    if (zeros)
        for (int64_t i = 0; i < groups; ++i)
            if (zeros[i] > 15) { set_error("zero point %d above 15", (int)zeros[i]); return PIVOT_E_SHAPE; }
    h.d = d;
    h.nbr = (d.M + d.bh - 1) / d.bh;
    h.nbc = (d.K + d.bw - 1) / d.bw;
    h.M_pad = h.nbr * d.bh;
    h.K_pad = h.nbc * d.bw;
    h.gpk = kQBlk / std::min(d.group, d.bw);
    h.has_zeros = zeros != nullptr;
    h.prow_pad.assign(h.M_pad, -1);
    h.pcol_pad.assign(h.K_pad, -1);
    h.identity_cols = true;
    for (int r = 0; r < d.M; ++r) h.prow_pad[r] = prow ? prow[r] : r;
    for (int c = 0; c < d.K; ++c) {
        h.pcol_pad[c] = pcol ? pcol[c] : c;
        h.identity_cols = h.identity_cols && h.pcol_pad[c] == c;
    }
    if (!invert(h.prow_pad.data(), d.M, h.invprow)) { set_error("prow is not a permutation of 0..M-1"); return PIVOT_E_NOT_PERMUTATION; }
    if (!invert(h.pcol_pad.data(), d.K, h.invpcol)) { set_error("pcol is not a permutation of 0..K-1"); return PIVOT_E_NOT_PERMUTATION; }
    h.bias_p.assign(h.M_pad, 0.f);
    if (bias)
        for (int r = 0; r < d.M; ++r) h.bias_p[r] = bias[h.prow_pad[r]];

    const int ppb = kQBlk / d.bw;            // pieces per block
    h.row_ptr.assign(h.nbr + 1, 0);
    h.kb_ptr.assign(h.nbr + 1, 0);
    for (int i = 0; i < h.nbr; ++i) {
        int n = 0;
        for (int j = 0; j < h.nbc; ++j)
            if (!tile_mask || tile_mask[(size_t)i * h.nbc + j]) { h.col_idx.push_back(j); h.pieces.push_back(j * d.bw); ++n; }
        const int kb = (n + ppb - 1) / ppb;
        for (int q = n; q < kb * ppb; ++q) h.pieces.push_back(-1);
        h.row_ptr[i + 1] = h.row_ptr[i] + n;
        h.kb_ptr[i + 1] = h.kb_ptr[i] + kb;
        h.max_kb = std::max(h.max_kb, kb);
    }
    h.T = h.row_ptr[h.nbr];
    h.KB = h.kb_ptr[h.nbr];
    h.whole = (int64_t)h.T == (int64_t)h.nbr * h.nbc;

    h.chunk_blocks = choose_chunk_blocks(h);
    struct Chunk { int row, b, e, first, parts, slot; };
    std::vector<Chunk> cs;
    for (int i = 0; i < h.nbr; ++i) {
        const int kb = h.kb_ptr[i + 1] - h.kb_ptr[i], parts = std::max(1, (kb + h.chunk_blocks - 1) / h.chunk_blocks), first = (int)cs.size();
        // pieces of equal length, not full ones and a rest
        for (int q = 0; q < parts; ++q)
            cs.push_back({i, h.kb_ptr[i] + (int)((int64_t)kb * q / parts), h.kb_ptr[i] + (int)((int64_t)kb * (q + 1) / parts), first, parts, first + q});
        h.max_parts = std::max(h.max_parts, parts);
    }
    std::stable_sort(cs.begin(), cs.end(), [](const Chunk& a, const Chunk& b) { return a.e - a.b > b.e - b.b; });
    h.nchunks = (int)cs.size();
    for (const Chunk& c : cs) for (int v : {c.row, c.b, c.e, c.first, c.parts, c.slot, h.kb_ptr[c.row], h.kb_ptr[c.row + 1] - h.kb_ptr[c.row]}) h.chunks.push_back(v);
    return PIVOT_OK;
} catch (const std::bad_alloc&) {
    set_error("out of host memory");
    return PIVOT_E_ALLOC;
}

size_t qfc_ticket_bytes(const QfcHost& h) {
    return h.max_parts > 1 ? (size_t)h.nbr * h.strips() * kQTicketStride * 4 : 0;
}
size_t qfc_partial_bytes(const QfcHost& h, int batch) {
    return h.max_parts > 1 ? align_up((size_t)h.nchunks * h.d.bh * batch * 4, 256) : 0;
}

int moe_mean_blocks(const std::vector<const pivot_qfc_plan_t*>& layers) {
    int64_t blocks = 0, rows = 0;
    for (const pivot_qfc_plan_t* p : layers) { blocks += p->host.KB; rows += p->host.nbr; }
    return rows ? (int)(blocks / rows) : 0;
}

}  // namespace pivot
