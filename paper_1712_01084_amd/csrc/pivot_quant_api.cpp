// C ABI of the layers with 4-bit weights, the norm and the mixture of experts: argument checks, device upload, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>
#include <string>

#include "pivot_device_guard.h"
#include "pivot_quant.h"

namespace pivot {
const char* last_error();
}

using namespace pivot;

namespace {

struct DeviceMemory {       // freed unless released
    char* p = nullptr;
    ~DeviceMemory() { if (p) (void)hipFree(p); }
    int get(size_t bytes) {
        void* q = nullptr;
        const hipError_t e = hipMalloc(&q, std::max<size_t>(bytes, 256));
        if (e != hipSuccess) { (void)hipGetLastError(); set_error("hipMalloc(%zu) failed: %s", bytes, hipGetErrorString(e)); return PIVOT_E_ALLOC; }
        p = static_cast<char*>(q);
        return PIVOT_OK;
    }
    char* release() { char* q = p; p = nullptr; return q; }
};

int hip_error(const char* what, hipError_t e) {
    (void)hipGetLastError();
    set_error("%s failed: %s", what, hipGetErrorString(e));
    return PIVOT_E_HIP;
}

int put(void* dst, const void* src, size_t bytes) {
    if (bytes == 0) return PIVOT_OK;
    const hipError_t e = hipMemcpy(dst, src, bytes, hipMemcpyHostToDevice);
    return e == hipSuccess ? PIVOT_OK : hip_error("hipMemcpy to device", e);
}

// Whether `p` is memory of this device.
bool on_device(const void* p, int device) {
    hipPointerAttribute_t at{};
    if (hipPointerGetAttributes(&at, p) != hipSuccess) { (void)hipGetLastError(); return false; }
    return at.type == hipMemoryTypeDevice && at.device == device;
}

// One plan on its way to the device: where its arrays lie in the allocation, and the caller's weights.
struct Upload {
    pivot_qfc_plan_t* p;
    const uint8_t* codes; const uint16_t* scales; const uint8_t* zeros; const float* bias;
    std::vector<int32_t> row_of_kb;
    struct Piece { const void* src; size_t bytes; void** dst; };
    std::vector<Piece> copied, laid_out;
    void arrange() {
        const QfcHost& h = p->host;
        QfcDev& d = p->dev;
        row_of_kb.resize(h.KB);
        for (int i = 0; i < h.nbr; ++i) std::fill(row_of_kb.begin() + h.kb_ptr[i], row_of_kb.begin() + h.kb_ptr[i + 1], i);
        const size_t units = h.units(), ns = units * h.gpk * kQStrip;
        copied = {
            {h.kb_ptr.data(), h.kb_ptr.size() * 4, (void**)&d.kb_ptr},
            {h.pieces.data(), h.pieces.size() * 4, (void**)&d.pieces},
            {h.chunks.data(), h.chunks.size() * 4, (void**)&d.chunks},
            {h.prow_pad.data(), h.prow_pad.size() * 4, (void**)&d.prow_pad},
            {h.pcol_pad.data(), h.pcol_pad.size() * 4, (void**)&d.pcol_pad},
            {h.invpcol.data(), h.invpcol.size() * 4, (void**)&d.invpcol},
            {h.bias_p.data(), h.bias_p.size() * 4, (void**)&d.bias_p},
            {row_of_kb.data(), row_of_kb.size() * 4, (void**)&d.row_of_kb},
        };
        laid_out = {{nullptr, units * kQUnitBytes, &d.codes}, {nullptr, ns * 2, (void**)&d.scales}};
        if (h.has_zeros) laid_out.push_back({nullptr, ns, (void**)&d.zeros});
    }
    static size_t room(const Piece& q) { return align_up(q.bytes + 1, 256); }
};

// Plans of one device, weights and index arrays of all of them in one allocation, the index arrays in one copy.  Weights in host
// memory pass through a second allocation, large enough for one plan, that is freed again.
int upload(std::vector<Upload>& ups, bool there) {
    const int device = ups[0].p->device;
    DeviceGuard g(device);
    if (!g.ok) { set_error("cannot select device %d", device); return PIVOT_E_HIP; }
    size_t image_bytes = 256, total = 0, most_raw = 0;      // the image begins with the word that a bad zero point sets
    for (Upload& u : ups) {
        const QfcHost& h = u.p->host;
        if (there)
            for (const void* q : {(const void*)u.codes, (const void*)u.scales, (const void*)u.zeros, (const void*)u.bias})
                if (q && !on_device(q, device)) { set_error("PIVOT_QFC_WEIGHTS_ON_DEVICE: codes, scales, zeros and bias must be memory of device %d", device); return PIVOT_E_UNSUPPORTED; }
        u.arrange();
        for (const Upload::Piece& q : u.copied) image_bytes += Upload::room(q);
        for (const Upload::Piece& q : u.laid_out) total += Upload::room(q);
        const size_t groups = (size_t)h.d.M * ((h.d.K + h.d.group - 1) / h.d.group);
        if (h.KB > 0) most_raw = std::max(most_raw, align_up((size_t)h.d.M * ((h.d.K + 1) / 2), 256) + align_up(groups * 2, 256) + groups);
    }
    total += image_bytes;
    std::vector<char> image(image_bytes);
    DeviceMemory mem, raw;
    int rc = mem.get(total);
    if (rc == PIVOT_OK && !there && most_raw) rc = raw.get(most_raw);
    if (rc != PIVOT_OK) return rc;
    int32_t* bad = reinterpret_cast<int32_t*>(mem.p);
    size_t off = 256;
    for (Upload& u : ups)
        for (const Upload::Piece& q : u.copied) {
            if (q.bytes) memcpy(image.data() + off, q.src, q.bytes);
            *q.dst = mem.p + off;
            off += Upload::room(q);
        }
    for (Upload& u : ups)
        for (const Upload::Piece& q : u.laid_out) {
            *q.dst = mem.p + off;
            off += Upload::room(q);
        }
    rc = put(mem.p, image.data(), image.size());
    for (Upload& u : ups) {
        const QfcHost& h = u.p->host;
        if (rc == PIVOT_OK && !there && h.KB > 0) {
            if (const hipError_t e = hipStreamSynchronize(nullptr); e != hipSuccess) return hip_error("laying out the weights", e);   // the plan before, from the same memory
            const size_t code_bytes = (size_t)h.d.M * ((h.d.K + 1) / 2), groups = (size_t)h.d.M * ((h.d.K + h.d.group - 1) / h.d.group);
            const size_t o1 = align_up(code_bytes, 256), o2 = o1 + align_up(groups * 2, 256);
            rc = put(raw.p, u.codes, code_bytes);
            if (rc == PIVOT_OK) rc = put(raw.p + o1, u.scales, groups * 2);
            if (rc == PIVOT_OK && u.zeros) rc = put(raw.p + o2, u.zeros, groups);
            u.codes = reinterpret_cast<const uint8_t*>(raw.p);
            u.scales = reinterpret_cast<const uint16_t*>(raw.p + o1);
            if (u.zeros) u.zeros = reinterpret_cast<const uint8_t*>(raw.p + o2);
        }
        if (rc == PIVOT_OK) rc = launch_qfc_pack(h, u.p->dev, u.codes, u.scales, u.zeros, there ? u.bias : nullptr, bad);
    }
    int32_t zero_above_15 = 0;
    const hipError_t e = hipMemcpy(&zero_above_15, bad, sizeof(int32_t), hipMemcpyDeviceToHost);      // waits for all of it
    if (rc == PIVOT_OK && e != hipSuccess) rc = hip_error("laying out the weights", e);
    if (rc == PIVOT_OK && zero_above_15) { set_error("a zero point is above 15"); rc = PIVOT_E_SHAPE; }
    if (rc != PIVOT_OK) return rc;
    const std::shared_ptr<char> shared(mem.release(), [device](char* p) { DeviceGuard g(device); (void)hipFree(p); });
    for (Upload& u : ups) u.p->dev.memory = shared;
    return PIVOT_OK;
}

int need_workspace(const void* ws, size_t have, size_t need) {
    if (need > 0 && (!ws || have < need)) { set_error("workspace too small: need %zu bytes, got %zu", need, ws ? have : (size_t)0); return PIVOT_E_WORKSPACE; }
    if (need > 0 && reinterpret_cast<uintptr_t>(ws) % 16 != 0) { set_error("workspace must be 16-byte aligned"); return PIVOT_E_WORKSPACE; }
    return PIVOT_OK;
}

bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t type_size(int t) { return t == PIVOT_F32 ? 4 : (t == PIVOT_F16 ? 2 : 1); }

int run_norm(const pivot_norm_args& a, const int32_t* order, void* stream) {
    NormLaunch L{};
    L.x = a.x; L.ldx = a.ldx; L.res = a.res; L.ldr = a.ldr; L.res_out = a.res_out; L.ldro = a.ldro; L.weight = a.weight;
    L.out = a.out; L.ldo = a.ldo; L.scale = a.scale; L.order = order;
    L.xtype = a.xtype; L.rtype = a.rtype; L.otype = a.otype; L.rows = a.rows; L.cols = a.cols; L.eps = a.eps; L.stream = stream;
    return launch_norm(L);
}

struct MoeScratch { size_t route, tickets, logits, partials, h, x, total; };   // counters first: their place does not depend on the tokens
MoeScratch moe_scratch(const pivot_moe_plan_t* p, int tokens) {
    MoeScratch s{};
    const size_t strips = p->down[0]->host.M_pad / kQStrip;
    s.tickets = align_up(sizeof(MoeRoute), 256);
    s.logits = s.tickets + strips * kQTicketStride * 4;
    s.partials = s.logits + align_up((size_t)tokens * p->E * 4, 256);
    s.h = s.partials + align_up(strips * kMoeMaxParts * kQStrip * tokens * 4, 256);
    s.x = s.h + align_up((size_t)tokens * p->top_k * p->down[0]->host.K_pad * 4, 256);
    s.total = s.x + (p->norm_weight ? align_up((size_t)tokens * align_up(p->D, 8) * 2, 256) : 0);
    return s;
}

}  // namespace

extern "C" {

int pivot_qfc_plan_many(int n, const pivot_qfc_desc* descs, const uint8_t* const* codes, const void* const* scales,
                        const uint8_t* const* zeros, const uint8_t* const* tile_mask, const int32_t* const* prow, const int32_t* const* pcol,
                        const float* const* bias, pivot_qfc_plan_t** out) try {
    if (n < 1) { set_error("n must be positive"); return PIVOT_E_SHAPE; }
    if (out) std::fill(out, out + n, nullptr);
    if (!descs || !out) { set_error("desc and out are required"); return PIVOT_E_NULL; }
    const int device = descs[0].device;
    const bool there = descs[0].flags & PIVOT_QFC_WEIGHTS_ON_DEVICE;      // (what lies there is not read here)
    std::vector<std::unique_ptr<pivot_qfc_plan_t>> plans;
    std::vector<Upload> ups(n);
    auto build = [&](int i) -> int {
        const pivot_qfc_desc& d = descs[i];
        auto of = [i](auto* list) { return list ? list[i] : nullptr; };
        Upload& u = ups[i];
        u.codes = of(codes); u.scales = static_cast<const uint16_t*>(of(scales)); u.zeros = of(zeros); u.bias = of(bias);
        if (!u.codes || !u.scales) { set_error("codes and scales are required"); return PIVOT_E_NULL; }
        if (d.device != device || d.flags != descs[0].flags) { set_error("device and flags must be the same for all"); return PIVOT_E_UNSUPPORTED; }
        if (there && device < 0) { set_error("PIVOT_QFC_WEIGHTS_ON_DEVICE needs a device"); return PIVOT_E_NO_DEVICE; }
        if (there && (!aligned_to(u.scales, 2) || !aligned_to(u.bias, 4))) { set_error("scales and bias must be aligned to their type"); return PIVOT_E_SHAPE; }
        // (sizes that the builder refuses are not looked through)
        const int64_t groups = d.M > 0 && d.K > 0 && d.group > 0 ? (int64_t)d.M * (((int64_t)d.K + d.group - 1) / d.group) : 0;
        plans.push_back(std::make_unique<pivot_qfc_plan_t>());
        u.p = plans.back().get();
        u.p->device = device;
        const int rc = build_qfc_host(d, there ? nullptr : u.zeros, groups, of(tile_mask), of(prow), of(pcol), there ? nullptr : u.bias, u.p->host);
        if (there) u.p->host.has_zeros = u.zeros != nullptr;
        return rc;
    };
    for (int i = 0; i < n; ++i) {
        const int rc = build(i);
        if (rc != PIVOT_OK) {
            const std::string why = last_error();
            if (n > 1) set_error("layer %d: %s", i, why.c_str());
            return rc;
        }
    }
    if (device >= 0) {
        const int rc = upload(ups, there);
        if (rc != PIVOT_OK) return rc;
    }
    for (int i = 0; i < n; ++i) out[i] = plans[i].release();
    return PIVOT_OK;
} catch (...) { set_error("out of host memory"); return PIVOT_E_ALLOC; }

int pivot_qfc_plan(const pivot_qfc_desc* desc, const uint8_t* codes, const void* scales, const uint8_t* zeros, const uint8_t* tile_mask,
                   const int32_t* prow, const int32_t* pcol, const float* bias, pivot_qfc_plan_t** out) {
    return pivot_qfc_plan_many(1, desc, &codes, &scales, &zeros, &tile_mask, &prow, &pcol, &bias, out);
}

int pivot_qfc_plan_host_view(const pivot_qfc_plan_t* plan, pivot_qfc_view* v) {
    if (!plan || !v) { set_error("plan and view are required"); return PIVOT_E_NULL; }
    const QfcHost& h = plan->host;
    v->M = h.d.M; v->K = h.d.K; v->bh = h.d.bh; v->bw = h.d.bw; v->group = h.d.group; v->act = h.d.act; v->nbr = h.nbr; v->nbc = h.nbc;
    v->M_pad = h.M_pad; v->K_pad = h.K_pad; v->T = h.T; v->blocks = h.KB; v->chunk_blocks = h.chunk_blocks; v->nchunks = h.nchunks;
    v->groups_per_block = h.gpk;
    v->row_ptr = h.row_ptr.data(); v->col_idx = h.col_idx.data(); v->block_ptr = h.kb_ptr.data(); v->pieces = h.pieces.data();
    v->chunks = h.chunks.data();
    return PIVOT_OK;
}

void pivot_qfc_plan_destroy(pivot_qfc_plan_t* plan) {
    delete plan;
}

size_t pivot_qfc_workspace_bytes(const pivot_qfc_plan_t* plan, int batch) {
    if (!plan || batch < 1) return 0;
    return qfc_ticket_bytes(plan->host) + qfc_partial_bytes(plan->host, batch) + qfc_copy_bytes(plan->host, batch);
}

int pivot_qfc_run(const pivot_qfc_plan_t* plan, const void* x_dev, int xtype, int64_t ldx, const float* xscale_dev, float* y_dev, int64_t ldy,
                  int batch, int flags, void* ws_dev, size_t ws_bytes, void* stream) {
    if (!plan) { set_error("plan is NULL"); return PIVOT_E_NULL; }
    if (plan->device < 0) { set_error("host-only plan (device = -1) cannot run"); return PIVOT_E_NO_DEVICE; }
    if (batch < 1 || batch > 64) { set_error("batch %d outside 1..64", batch); return PIVOT_E_SHAPE; }
    if (xtype != PIVOT_F16 && xtype != PIVOT_Q8) { set_error("x of a 4-bit layer is PIVOT_F16 or PIVOT_Q8"); return PIVOT_E_UNSUPPORTED; }
    if (flags & ~PIVOT_QFC_X_BLOCK_ORDER) { set_error("unknown flags"); return PIVOT_E_UNSUPPORTED; }
    if (!x_dev || !y_dev) { set_error("x_dev and y_dev are required"); return PIVOT_E_NULL; }
    if (xtype == PIVOT_Q8 && !xscale_dev) { set_error("xscale_dev is required with PIVOT_Q8"); return PIVOT_E_NULL; }
    if (xtype == PIVOT_F16 && xscale_dev) { set_error("xscale_dev is for PIVOT_Q8"); return PIVOT_E_UNSUPPORTED; }
    const QfcHost& h = plan->host;
    if (ldx < h.d.K || ldy < h.d.M) { set_error("ldx/ldy smaller than K/M"); return PIVOT_E_SHAPE; }
    if (!aligned_to(x_dev, type_size(xtype)) || !aligned_to(y_dev, 4) || !aligned_to(xscale_dev, 4)) { set_error("x, xscale and y must be aligned to their type"); return PIVOT_E_SHAPE; }
    const size_t nt = qfc_ticket_bytes(h), np = qfc_partial_bytes(h, batch);
    int rc = need_workspace(ws_dev, ws_bytes, nt + np + qfc_copy_bytes(h, batch));
    if (rc != PIVOT_OK) return rc;
    DeviceGuard g(plan->device);
    if (!g.ok) { set_error("cannot select device %d", plan->device); return PIVOT_E_HIP; }
    QfcLaunch L{};
    L.h = &h; L.d = &plan->dev; L.x = x_dev; L.xtype = xtype; L.ldx = ldx; L.xscale = xscale_dev; L.block_order = flags & PIVOT_QFC_X_BLOCK_ORDER;
    L.y = y_dev; L.ldy = ldy; L.batch = batch; L.tickets = static_cast<uint32_t*>(ws_dev);
    L.partials = reinterpret_cast<float*>(static_cast<char*>(ws_dev) + nt); L.xcopy = static_cast<char*>(ws_dev) + nt + np; L.stream = stream;
    return launch_qfc(L);
}

int pivot_qfc_run_kernel_name(const pivot_qfc_plan_t* plan, const void* x_dev, int xtype, int64_t ldx, int batch, int flags, char* buf,
                              size_t buf_len) try {
    if (!plan || !buf) { set_error("plan and buf are required"); return PIVOT_E_NULL; }
    if (buf_len == 0) { set_error("buf_len is 0"); return PIVOT_E_SHAPE; }
    if (batch < 1 || batch > 64) { set_error("batch %d outside 1..64", batch); return PIVOT_E_SHAPE; }
    if (xtype != PIVOT_F16 && xtype != PIVOT_Q8) { set_error("x of a 4-bit layer is PIVOT_F16 or PIVOT_Q8"); return PIVOT_E_UNSUPPORTED; }
    if (flags & ~PIVOT_QFC_X_BLOCK_ORDER) { set_error("unknown flags"); return PIVOT_E_UNSUPPORTED; }
    if (ldx < plan->host.d.K) { set_error("ldx smaller than K"); return PIVOT_E_SHAPE; }
    QfcLaunch L{};
    L.h = &plan->host; L.d = &plan->dev; L.x = x_dev; L.xtype = xtype; L.ldx = ldx; L.block_order = flags & PIVOT_QFC_X_BLOCK_ORDER; L.batch = batch;
    std::string name;
    int rc = launch_qfc(L, &name);
    if (rc != PIVOT_OK) return rc;
    const size_t n = std::min(name.size(), buf_len - 1);
    memcpy(buf, name.data(), n);
    buf[n] = 0;
    return PIVOT_OK;
} catch (...) { set_error("out of host memory"); return PIVOT_E_ALLOC; }

int pivot_qfc_kernel_name(const pivot_qfc_plan_t* plan, int xtype, int batch, char* buf, size_t buf_len) {
    return pivot_qfc_run_kernel_name(plan, nullptr, xtype, plan ? (int64_t)align_up(plan->host.d.K, 16) : 0, batch, 0, buf, buf_len);
}

int pivot_norm_run(const pivot_norm_args* args, void* stream) {
    if (!args) { set_error("args is NULL"); return PIVOT_E_NULL; }
    const pivot_norm_args& a = *args;
    if (!a.x || !a.out) { set_error("x and out are required"); return PIVOT_E_NULL; }
    if (a.rows < 1 || a.cols < 1 || a.cols > kQMaxK) { set_error("rows must be positive and cols in 1..65535"); return PIVOT_E_SHAPE; }
    auto real = [](int t) { return t == PIVOT_F32 || t == PIVOT_F16; };
    if (!real(a.xtype) || (a.res && !real(a.rtype)) || !(real(a.otype) || a.otype == PIVOT_Q8)) { set_error("unsupported type"); return PIVOT_E_UNSUPPORTED; }
    if (a.res_out && !a.res) { set_error("res_out needs res"); return PIVOT_E_NULL; }
    if (a.otype == PIVOT_Q8 && !a.scale) { set_error("scale is required with PIVOT_Q8"); return PIVOT_E_NULL; }
    if (a.otype != PIVOT_Q8 && a.scale) { set_error("scale is for PIVOT_Q8"); return PIVOT_E_UNSUPPORTED; }
    if (!(a.eps >= 0.f) || std::isinf(a.eps)) { set_error("eps must be finite and not negative"); return PIVOT_E_SHAPE; }
    if (a.ldx < a.cols || a.ldo < a.cols || (a.res && a.ldr < a.cols) || (a.res_out && a.ldro < a.cols)) { set_error("a row stride is smaller than cols"); return PIVOT_E_SHAPE; }
    if (a.out == a.x || a.out == a.res || a.out == a.res_out || (a.res_out && a.res_out == a.x)) { set_error("out and res_out must not be x, nor out the residual"); return PIVOT_E_UNSUPPORTED; }
    if (a.res_out == a.res && a.res && a.ldro != a.ldr) { set_error("res in place needs ldro = ldr"); return PIVOT_E_SHAPE; }
    if (!aligned_to(a.x, type_size(a.xtype)) || (a.res && !aligned_to(a.res, type_size(a.rtype))) || (a.res_out && !aligned_to(a.res_out, type_size(a.rtype))) ||
        !aligned_to(a.weight, 4) || !aligned_to(a.out, type_size(a.otype)) || !aligned_to(a.scale, 4)) {
        set_error("arrays must be aligned to their type");
        return PIVOT_E_SHAPE;
    }
    const int32_t* order = nullptr;
    if (a.order) {
        if (a.order->device < 0) { set_error("host-only plan (device = -1) cannot run"); return PIVOT_E_NO_DEVICE; }
        if (a.order->host.d.K != a.cols) { set_error("the plan takes %d columns, not %d", a.order->host.d.K, a.cols); return PIVOT_E_SHAPE; }
        if (!a.order->host.identity_cols) order = a.order->dev.invpcol;
    }
    if (!a.order) return run_norm(a, order, stream);
    DeviceGuard g(a.order->device);
    if (!g.ok) { set_error("cannot select device %d", a.order->device); return PIVOT_E_HIP; }
    return run_norm(a, order, stream);
}

// ------------------------------------------------------------------ mixture of experts

int pivot_moe_plan(const pivot_moe_desc* desc, const pivot_qfc_plan_t* const* gate_up, const pivot_qfc_plan_t* const* down, const void* router,
                   const float* router_bias, const float* norm_weight, pivot_moe_plan_t** out) try {
    if (out) *out = nullptr;
    if (!desc || !out || !gate_up || !down || !router) { set_error("desc, gate_up, down, router and out are required"); return PIVOT_E_NULL; }
    const int E = desc->experts, k = desc->top_k;
    if (E < 1 || E > kMoeMaxExperts || k < 1 || k > kMoeMaxTopK || k > E) { set_error("experts must lie in 1..256, top_k in 1..8 and not above experts"); return PIVOT_E_SHAPE; }
    if (desc->router_type != PIVOT_F32 && desc->router_type != PIVOT_F16) { set_error("router_type must be PIVOT_F32 or PIVOT_F16"); return PIVOT_E_UNSUPPORTED; }
    if (desc->flags & ~PIVOT_MOE_RENORMALISE) { set_error("unknown flags"); return PIVOT_E_UNSUPPORTED; }
    if (norm_weight && (!(desc->norm_eps >= 0.f) || std::isinf(desc->norm_eps))) { set_error("norm_eps must be finite and not negative"); return PIVOT_E_SHAPE; }
    for (int e = 0; e < E; ++e) if (!gate_up[e] || !down[e]) { set_error("expert %d is NULL", e); return PIVOT_E_NULL; }
    const QfcHost &u0 = gate_up[0]->host, &d0 = down[0]->host;
    const int D = u0.d.K, F = d0.d.K, device = gate_up[0]->device;
    for (int e = 0; e < E; ++e) {
        const QfcHost &u = gate_up[e]->host, &d = down[e]->host;
        if (u.d.K != D || u.d.M != 2 * F || d.d.K != F || d.d.M != D) { set_error("expert %d: gate_up must be 2F x D and down D x F, the same for all", e); return PIVOT_E_SHAPE; }
        auto alike = [](const QfcHost& a, const QfcHost& b) { return a.d.bh == b.d.bh && a.d.bw == b.d.bw && a.d.group == b.d.group && a.has_zeros == b.has_zeros && a.d.act == PIVOT_ACT_NONE; };
        if (!alike(u, u0) || !alike(d, d0)) { set_error("expert %d: tile shape, group and zero points must be those of expert 0, and no activation", e); return PIVOT_E_UNSUPPORTED; }
        if (gate_up[e]->device != device || down[e]->device != device) { set_error("all experts must be on one device"); return PIVOT_E_UNSUPPORTED; }
        for (int i = 0; i < F; ++i)
            if (u.prow_pad[2 * i] % 2 != 0 || u.prow_pad[2 * i + 1] != u.prow_pad[2 * i] + 1) { set_error("expert %d: gate_up's row permutation parts the gate and the up row of a unit", e); return PIVOT_E_UNSUPPORTED; }
        if (d.prow_pad != d0.prow_pad) { set_error("expert %d: the down layers must share one row permutation", e); return PIVOT_E_UNSUPPORTED; }
    }
    std::unique_ptr<pivot_moe_plan_t> p(new (std::nothrow) pivot_moe_plan_t());
    if (!p) { set_error("out of host memory"); return PIVOT_E_ALLOC; }
    p->gate_up.assign(gate_up, gate_up + E);
    p->down.assign(down, down + E);
    p->down_blocks = moe_mean_blocks(p->down);
    p->E = E; p->top_k = k; p->D = D; p->F = F; p->router_type = desc->router_type; p->renormalise = desc->flags & PIVOT_MOE_RENORMALISE;
    p->device = device; p->eps = desc->norm_eps;
    if (device < 0) { set_error("host-only plan (device = -1) cannot run"); return PIVOT_E_NO_DEVICE; }
    DeviceGuard g(device);
    if (!g.ok) { set_error("cannot select device %d", device); return PIVOT_E_HIP; }
    const int npairs = u0.M_pad / 2;
    const size_t nex = align_up(E * sizeof(MoeExpert), 256), nr = align_up((size_t)E * D * elem_size(desc->router_type), 256),
                 nb = router_bias ? align_up(E * 4, 256) : 0, nn = norm_weight ? align_up((size_t)D * 4, 256) : 0;
    DeviceMemory mem;
    int rc = mem.get(nex + nr + nb + nn + (size_t)E * npairs * 4);
    if (rc != PIVOT_OK) return rc;
    char* at = mem.p;
    p->experts = reinterpret_cast<MoeExpert*>(at); at += nex;
    p->router = at; at += nr;
    if (router_bias) { p->router_bias = reinterpret_cast<float*>(at); at += nb; }
    if (norm_weight) { p->norm_weight = reinterpret_cast<float*>(at); at += nn; }
    int32_t* hdst_dev = reinterpret_cast<int32_t*>(at);
    std::vector<MoeExpert> ex(E);
    std::vector<int32_t> hdst((size_t)E * npairs, -1);
    for (int e = 0; e < E; ++e) {
        const QfcHost &u = gate_up[e]->host, &d = down[e]->host;
        for (int i = 0; i < F; ++i) hdst[(size_t)e * npairs + i] = d.invpcol[u.prow_pad[2 * i] / 2];
        const QfcDev* dev[2] = {&gate_up[e]->dev, &down[e]->dev};
        for (int q = 0; q < 2; ++q) {
            ex[e].codes[q] = dev[q]->codes; ex[e].scales[q] = dev[q]->scales; ex[e].zeros[q] = dev[q]->zeros; ex[e].kb_ptr[q] = dev[q]->kb_ptr;
            ex[e].pieces[q] = dev[q]->pieces; ex[e].bias[q] = dev[q]->bias_p;
            const QfcHost& l = q ? d : u;
            ex[e].whole[q] = l.whole ? l.max_kb : 0;
        }
        p->gather |= !u.identity_cols;
        ex[e].pcol = u.identity_cols ? nullptr : gate_up[e]->dev.pcol_pad;
        ex[e].hdst = hdst_dev + (size_t)e * npairs;
    }
    rc = put(p->experts, ex.data(), E * sizeof(MoeExpert));
    if (rc == PIVOT_OK) rc = put(p->router, router, (size_t)E * D * elem_size(desc->router_type));
    if (rc == PIVOT_OK && router_bias) rc = put(p->router_bias, router_bias, (size_t)E * 4);
    if (rc == PIVOT_OK && norm_weight) rc = put(p->norm_weight, norm_weight, (size_t)D * 4);
    if (rc == PIVOT_OK) rc = put(hdst_dev, hdst.data(), hdst.size() * 4);
    if (rc != PIVOT_OK) return rc;
    p->dev_base = mem.release();
    *out = p.release();
    return PIVOT_OK;
} catch (...) { set_error("out of host memory"); return PIVOT_E_ALLOC; }

void pivot_moe_plan_destroy(pivot_moe_plan_t* plan) {
    if (!plan) return;
    if (plan->dev_base) {
        DeviceGuard g(plan->device);
        (void)hipFree(plan->dev_base);
    }
    delete plan;
}

size_t pivot_moe_workspace_bytes(const pivot_moe_plan_t* plan, int tokens) {
    if (!plan || tokens < 1) return 0;
    return moe_scratch(plan, tokens).total;
}

int pivot_moe_run(const pivot_moe_plan_t* plan, const void* x_dev, int xtype, int64_t ldx, void* res_dev, float* y_dev, int64_t ldy, int tokens,
                  int32_t* ids_dev, float* weights_dev, void* ws_dev, size_t ws_bytes, void* stream) {
    if (!plan) { set_error("plan is NULL"); return PIVOT_E_NULL; }
    if (tokens < 1 || tokens > kMoeMaxTokens) { set_error("tokens %d outside 1..16", tokens); return PIVOT_E_SHAPE; }
    if (!x_dev || !y_dev) { set_error("x_dev and y_dev are required"); return PIVOT_E_NULL; }
    if (xtype != PIVOT_F16 && !(plan->norm_weight && xtype == PIVOT_F32)) { set_error("x is PIVOT_F16, or PIVOT_F32 with a norm"); return PIVOT_E_UNSUPPORTED; }
    if (res_dev && !plan->norm_weight) { set_error("res_dev is for plans with a norm"); return PIVOT_E_UNSUPPORTED; }
    if (ldx < plan->D || ldy < plan->D) { set_error("ldx/ldy smaller than D"); return PIVOT_E_SHAPE; }
    if (!aligned_to(x_dev, type_size(xtype)) || !aligned_to(res_dev, type_size(xtype)) || !aligned_to(y_dev, 4) || !aligned_to(ids_dev, 4) || !aligned_to(weights_dev, 4)) {
        set_error("arrays must be aligned to their type");
        return PIVOT_E_SHAPE;
    }
    const MoeScratch s = moe_scratch(plan, tokens);
    int rc = need_workspace(ws_dev, ws_bytes, s.total);
    if (rc != PIVOT_OK) return rc;
    DeviceGuard g(plan->device);
    if (!g.ok) { set_error("cannot select device %d", plan->device); return PIVOT_E_HIP; }
    char* ws = static_cast<char*>(ws_dev);
    MoeLaunch L{};
    L.x = x_dev; L.ldx = ldx;
    if (plan->norm_weight) {                            // (into fp16, which is what the matrix instructions of the experts take)
        pivot_norm_args n{};
        n.x = x_dev; n.ldx = ldx; n.res = res_dev; n.ldr = ldx; n.res_out = res_dev; n.ldro = ldx; n.weight = plan->norm_weight;
        n.out = ws + s.x; n.ldo = (int64_t)align_up(plan->D, 8); n.xtype = xtype; n.rtype = xtype; n.otype = PIVOT_F16;
        n.rows = tokens; n.cols = plan->D; n.eps = plan->eps;
        rc = run_norm(n, nullptr, stream);
        if (rc != PIVOT_OK) return rc;
        L.x = n.out; L.ldx = n.ldo;
    }
    const QfcHost* hs[2] = {&plan->gate_up[0]->host, &plan->down[0]->host};
    for (int q = 0; q < 2; ++q) {
        L.bh[q] = hs[q]->d.bh; L.bw[q] = hs[q]->d.bw; L.gpk[q] = hs[q]->gpk; L.zeros[q] = hs[q]->has_zeros; L.nstrips[q] = hs[q]->M_pad / kQStrip;
    }
    L.down_blocks = plan->down_blocks;
    L.gather = plan->gather;
    L.experts = plan->experts; L.router = plan->router; L.router_type = plan->router_type; L.router_bias = plan->router_bias; L.renormalise = plan->renormalise;
    L.E = plan->E; L.top_k = plan->top_k; L.D = plan->D; L.F = plan->F; L.F_pad = hs[1]->K_pad; L.prow_down = plan->down[0]->dev.prow_pad;
    L.y = y_dev; L.ldy = ldy; L.tokens = tokens; L.ids = ids_dev; L.weights = weights_dev;
    L.tickets = reinterpret_cast<uint32_t*>(ws + s.tickets); L.partials = reinterpret_cast<float*>(ws + s.partials);
    L.route = reinterpret_cast<MoeRoute*>(ws + s.route); L.logits = reinterpret_cast<float*>(ws + s.logits); L.h = reinterpret_cast<float*>(ws + s.h);
    L.stream = stream;
    return launch_moe(L);
}

}  // extern "C"
