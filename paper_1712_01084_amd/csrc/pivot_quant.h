// Layers with 4-bit weights and group scales: the plan, what the launchers see, and what the host side shares with
// the kernels about where a weight lies.  Not part of the public interface.
//
// A block row of nt kept tiles is, without the pruned ones, a dense matrix of bh rows and nt*bw columns whose columns
// are gathered.  It is cut into strips of 16 rows and blocks of kQBlk = 128 columns: one such unit is 1 KB of codes,
// 16 bytes per lane of a wavefront, and feeds four 16x16x32 matrix instructions (two 16x16x64 in 8 bits).  Lane l holds
// row l % 16 and, in word j, the eight columns 32 j + 8 (l / 16) + 0..7.
#pragma once

#include <cstddef>
#include <cstdint>
#include <memory>
#include <string>
#include <vector>

#include "pivot_internal.h"

namespace pivot {

constexpr int kQBlk = 128;              // columns of a unit
constexpr int kQStrip = 16;             // rows of a unit
constexpr int kQUnitBytes = kQBlk * kQStrip / 2;
constexpr int kQMaxK = 65535, kQMaxM = 1 << 22;
constexpr int kQTicketStride = 64;      // words between arrival counters: a cache line pair each

// Which of the eight columns of a word its nibble i holds: with this order two nibbles masked out of a word in place
// are neighbouring columns of a pair of fp16 values, and the low (high) nibbles of its bytes are columns 0,4,1,5
// (2,6,3,7), the order in which 8-bit inputs are staged.
constexpr int q_nibble_col(int i) { return i < 4 ? 2 * i : 2 * (i - 4) + 1; }
// Where column c of a unit lies among 128 staged 8-bit inputs: the two words of a 64-column step that one lane
// multiplies side by side (16 bytes), the eight columns of a word in nibble order.
constexpr int q_byte_pos(int c) {
    return (c & 64) + ((c >> 3) & 3) * 16 + ((c >> 5) & 1) * 8 + 2 * (c & 3) + ((c >> 2) & 1);
}

struct QfcHost {
    pivot_qfc_desc d{};
    int nbr = 0, nbc = 0, M_pad = 0, K_pad = 0, T = 0, KB = 0, nchunks = 0, chunk_blocks = 0, max_parts = 1, max_kb = 0;
    int gpk = 1;                        // scale groups per unit (1, 2, 4)
    bool has_zeros = false, identity_cols = false, whole = false;   // whole: every tile is kept
    std::vector<int32_t> row_ptr, col_idx;
    std::vector<int32_t> kb_ptr;        // [nbr+1] blocks of 128 kept columns before block row i
    std::vector<int32_t> pieces;        // [KB * 128 / bw] first block-space column of each bw columns, -1 = none
    std::vector<int32_t> chunks;        // [nchunks][8]: block row, first block, end, first slot of the row, pieces of the row, slot, the row's first block, its blocks
    std::vector<int32_t> prow_pad, pcol_pad, invprow, invpcol;
    std::vector<float>   bias_p;
    int strips() const { return d.bh / kQStrip; }
    size_t units() const { return (size_t)KB * strips(); }
};

struct QfcDev {
    std::shared_ptr<char> memory;       // freed with the last plan made in the same call
    void*  codes = nullptr;             // [units][64 lanes] 16 bytes; units of block row i: strip-major
    uint16_t* scales = nullptr;         // [units][4 quarters of the strip][gpk][4 rows] fp16
    uint8_t* zeros = nullptr;           // [units][16 rows][gpk], or NULL
    int32_t* kb_ptr = nullptr;
    int32_t* pieces = nullptr;
    int32_t* chunks = nullptr;
    int32_t* prow_pad = nullptr;
    int32_t* pcol_pad = nullptr;        // [K_pad]
    int32_t* invpcol = nullptr;         // [K]
    float*   bias_p = nullptr;
    int32_t* row_of_kb = nullptr;       // [KB] the block row of a block (laying out)
};

int  build_qfc_host(const pivot_qfc_desc& d, const uint8_t* zeros, int64_t groups, const uint8_t* tile_mask, const int32_t* prow,
                    const int32_t* pcol, const float* bias, QfcHost& h);
// Lays the codes and scales out on the device, on the default stream; raw_*: the caller's arrays, there already (raw_bias NULL:
// bias_p stands); *bad is set where a zero point is above 15.
int  launch_qfc_pack(const QfcHost& h, const QfcDev& d, const uint8_t* raw_codes, const uint16_t* raw_scales,
                     const uint8_t* raw_zeros, const float* raw_bias, int32_t* bad);

struct QfcLaunch {
    const QfcHost* h; const QfcDev* d;
    const void* x; int xtype; int64_t ldx; const float* xscale; int block_order;
    float* y; int64_t ldy; int batch;
    float* partials; uint32_t* tickets; void* xcopy;
    void* stream;
};
size_t qfc_ticket_bytes(const QfcHost& h);
size_t qfc_partial_bytes(const QfcHost& h, int batch);
size_t qfc_copy_bytes(const QfcHost& h, int batch);
int    launch_qfc(const QfcLaunch& L, std::string* describe = nullptr);

struct NormLaunch {
    const void* x; int64_t ldx; const void* res; int64_t ldr; void* res_out; int64_t ldro; const float* weight;
    void* out; int64_t ldo; float* scale; const int32_t* order;   // order: [cols] out[c] = natural column order[c], or NULL
    int xtype, rtype, otype, rows, cols; float eps; int lds_rows, row0; void* stream;   // lds_rows, row0: set by the launcher
};
int launch_norm(const NormLaunch& L);

// Lets `kernel` be launched on the current device with more than 64 KB of LDS (asked of the runtime once per device: 1 us).
int reserve_lds(const void* kernel, size_t bytes);

// ---- mixture of experts
constexpr int kMoeMaxTokens = 16, kMoeMaxExperts = 256, kMoeMaxTopK = 8;
constexpr int kMoeMaxActive = kMoeMaxTokens * kMoeMaxTopK;
constexpr int kMoeMaxParts = 8;         // workgroups of a strip of the down layers
// Blocks of a block row, in the mean over all layers.
int moe_mean_blocks(const std::vector<const pivot_qfc_plan_t*>& layers);

// One expert as the kernels see it: its two layers (0 gate/up, 1 down), and where a unit's activation goes in the down
// layer's input.  whole > 0: every tile is kept, `whole` blocks in each block row, so that neither the blocks of a row nor
// their columns have to be looked up.
struct MoeExpert {
    const void* codes[2]; const uint16_t* scales[2]; const uint8_t* zeros[2]; const int32_t* kb_ptr[2]; const int32_t* pieces[2];
    const int32_t* pcol; const int32_t* hdst; const float* bias[2]; int32_t whole[2];
};
// What the router leaves for the two expert kernels.  Experts in use are numbered 0..n-1 in ascending order; the entry of
// one holds its layers too, which saves the kernels behind a trip.
struct MoeActive {
    MoeExpert ex;
    int32_t ntok, mask;                                   // its tokens: how many, a bit each,
    uint64_t tok;                                         // and four bits each, ascending
    int32_t hrow[kMoeMaxTokens];                          // their rows of h
    float   share[kMoeMaxTokens];                         // the expert's weight, by token
};
struct MoeRoute {
    uint32_t ticket; int32_t pad[63];
    int32_t n; int32_t pad2[63];
    int32_t sel[kMoeMaxTokens][kMoeMaxTopK];              // by token: its experts, largest logit first, -1 = none
    float   sel_w[kMoeMaxTokens][kMoeMaxTopK];
    MoeActive active[kMoeMaxActive];
};
struct MoeLaunch {
    const MoeExpert* experts; const void* router; int router_type; const float* router_bias; int renormalise;
    int E, top_k, D, F, F_pad, gather;                      // gather: whether any gate/up layer takes its columns in an order of its own
    int bh[2], bw[2], gpk[2], zeros[2], nstrips[2], down_blocks;   // down_blocks: of a block row, in the mean
    const int32_t* prow_down;
    const void* x; int64_t ldx; float* y; int64_t ldy; int tokens; int32_t* ids; float* weights;
    uint32_t* tickets; float* partials;                   // of the strips of the down layers
    MoeRoute* route; float* logits; float* h;             // h: [tokens * top_k][F_pad]
    void* stream;
};
int launch_moe(const MoeLaunch& L);

}  // namespace pivot

struct pivot_qfc_plan {
    pivot::QfcHost host;
    pivot::QfcDev  dev;
    int device = -1;
};

struct pivot_moe_plan {
    std::vector<const pivot_qfc_plan_t*> gate_up, down;
    int down_blocks = 0;                // moe_mean_blocks of the down layers
    int E = 0, top_k = 0, D = 0, F = 0, router_type = 0, renormalise = 0, gather = 0, device = -1;
    float eps = 0.f;
    char* dev_base = nullptr;
    pivot::MoeExpert* experts = nullptr; void* router = nullptr; float* router_bias = nullptr; float* norm_weight = nullptr;
};
