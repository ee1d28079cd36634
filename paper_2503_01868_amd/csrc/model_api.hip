// C ABI of the operators around the mixers: argument validation (before any HIP call) and kernel selection.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "hy_common.hpp"
#include "hy_launch.hpp"
#include "hy_model_checks.hpp"

using namespace hy;

namespace {

hy_status check_glr(int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype) {
    if (B < 0 || L < 0 || D < 0 || group < 1 || D % group != 0 || L > kMostElements) return HY_ERR_SHAPE;
    // (also of what is empty: strides are computed all the same)
    if (!fits(std::max<int64_t>(B, 1), L + 1, std::max<int64_t>(D, 1))) return HY_ERR_SHAPE;
    return known(dtype) ? HY_OK : HY_ERR_DTYPE;
}

GlrShape glr_shape(int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype) {
    GlrShape s{B, L, D, group, static_cast<hy_dtype>(dtype), {}, {}};
    for (int i = 0; i < 5; ++i) {
        s.rstride[i] = i == kGlrG ? D / group : D;
        s.bstride[i] = s.rstride[i] * L;
    }
    return s;
}

hy_status take_strides(GlrShape& s, const int64_t* strides, const int* which, int n) {
    if (!strides) return HY_OK;
    for (int i = 0; i < n; ++i) {
        const int64_t b = strides[2 * i], r = strides[2 * i + 1];
        if (b < 0 || r < 0) return HY_ERR_SHAPE;
        if (!fits(s.B > 1 ? s.B - 1 : 0, b, 1) || !fits(s.L > 1 ? s.L - 1 : 0, r, 1)) return HY_ERR_SHAPE;
        s.bstride[which[i]] = s.B > 1 ? b : 0;
        s.rstride[which[i]] = s.L > 1 ? r : 0;
    }
    return HY_OK;
}

Range glr_range(const GlrShape& s, const void* p, int i) {
    if (empty(s.B, s.L, s.D)) return Range{p, 0};
    const int64_t row = i == kGlrG ? s.D / s.group : s.D;
    return Range{p, ((s.B - 1) * s.bstride[i] + (s.L - 1) * s.rstride[i] + row) * size_of(s.dtype)};
}

// Inputs may be views that begin at any element: how many a lane can load together.
hy_status take_starts(GlrShape& s, const Range* r, int n, int gate) {
    const uintptr_t e = (uintptr_t)size_of(s.dtype);
    for (int i = 0; i < n; ++i) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(r[i].p);
        if (at % e != 0) return HY_ERR_ALIGN;
        if (i != gate || s.group == 1)
            while (at % (s.start_align * e) != 0) s.start_align /= 2;
    }
    return HY_OK;
}

int64_t marks_bytes(const GlrShape& s) { return s.B * ((s.L + kGlrRows - 1) / kGlrRows) * s.D * 4; }

// ---- cross entropy

hy_status check_xent(int64_t N, int64_t V, int64_t D, int32_t dtype) {
    if (N < 0 || V < 1 || D < 1 || !fits(std::max<int64_t>(N, 1), D, 1) || !fits(V, D, 1)) return HY_ERR_SHAPE;
    if (N > (INT64_C(1) << 60) / V) return HY_ERR_SHAPE;  // (logits: a pair is kept of 64 of them)
    return known(dtype) ? HY_OK : HY_ERR_DTYPE;
}

// ---- AdamW

constexpr int64_t kMostChunks = most_workgroups(kAdamwThreads);  // one workgroup each

int64_t chunks_of(int64_t count) { return (count + kAdamwChunk - 1) / kAdamwChunk; }

// The chunks of all tensors; -1: not a valid problem.
int64_t adamw_chunks(const hy_adamw_tensor* t, int64_t n) {
    if (n < 0 || n > INT32_MAX || (n > 0 && !t)) return -1;
    int64_t all = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (t[i].count < 0 || t[i].count > kMostElements) return -1;
        all += chunks_of(t[i].count);
        if (all > kMostChunks) return -1;
    }
    return all;
}

struct Span {
    uintptr_t from, to;
    bool written;
};

// No written span meets another one.
bool apart(std::vector<Span>& s) {
    std::sort(s.begin(), s.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
    uintptr_t any = 0, written = 0;
    for (const Span& x : s) {
        if (x.from < written || (x.written && x.from < any)) return false;
        any = std::max(any, x.to);
        if (x.written) written = std::max(written, x.to);
    }
    return true;
}

hy_status adamw_entries(const hy_adamw_tensor* t, int64_t n, int32_t param, int32_t grad, int32_t bits, bool with_master,
                        std::vector<AdamwEntry>& entries) {
    std::vector<Span> spans;
    int64_t chunk = 0;
    for (int64_t i = 0; i < n; ++i) {
        const int64_t c = t[i].count, e = bits == 8 ? 1 : 4, blocks = (c + kAdamwBlock - 1) / kAdamwBlock * 4;
        const struct {
            const void* p;
            int64_t bytes, element;
            bool written;
        } arrays[7] = {{t[i].param, c * size_of(param), size_of(param), true}, {t[i].grad, c * size_of(grad), size_of(grad), false},
                       {t[i].exp_avg, c * e, e, true}, {t[i].exp_avg_sq, c * e, e, true},
                       {t[i].avg_scale, bits == 8 ? blocks : 0, 4, true}, {t[i].sq_scale, bits == 8 ? blocks : 0, 4, true},
                       {t[i].master, with_master ? c * 4 : 0, 4, true}};
        bool fours = true;
        for (const auto& x : arrays) {
            if (x.bytes == 0) continue;
            const uintptr_t at = reinterpret_cast<uintptr_t>(x.p);
            if (!x.p) return HY_ERR_NULL;
            if (at % (uintptr_t)x.element != 0) return HY_ERR_ALIGN;
            spans.push_back(Span{at, at + (uintptr_t)x.bytes, x.written});
        }
        for (const auto& x : {arrays[0], arrays[1], arrays[2], arrays[3], arrays[6]})
            if (x.bytes > 0 && reinterpret_cast<uintptr_t>(x.p) % (uintptr_t)(4 * x.element) != 0) fours = false;
        entries.push_back(AdamwEntry{t[i].param, t[i].grad, t[i].exp_avg, t[i].exp_avg_sq, t[i].avg_scale, t[i].sq_scale,
                                     t[i].master, c, chunk, t[i].weight_decay, fours});
        chunk += chunks_of(c);
    }
    return apart(spans) ? HY_OK : HY_ERR_ALIGN;
}

hy_status check_adamw_kinds(int32_t param, int32_t grad, int32_t bits, int32_t with_master) {
    if (!known(param) || !known(grad)) return HY_ERR_DTYPE;
    if (bits != 8 && bits != 32) return HY_ERR_UNSUPPORTED;
    return with_master && param == HY_F32 ? HY_ERR_UNSUPPORTED : HY_OK;  // an fp32 parameter is its own master
}

}  // namespace

extern "C" {

int64_t hyena_xent_fwd_workspace_bytes(int64_t N, int64_t V, int64_t D, int32_t dtype) {
    if (check_xent(N, V, D, dtype) != HY_OK) return -1;
    if (N == 0) return 0;
    const XentShape s{N, V, D, static_cast<hy_dtype>(dtype)};
    return xent_served(s, false) ? xent_fwd_workspace_bytes(s) : -1;
}

int64_t hyena_xent_bwd_workspace_bytes(int64_t N, int64_t V, int64_t D, int32_t dtype) {
    if (check_xent(N, V, D, dtype) != HY_OK) return -1;
    if (N == 0) return 0;
    const XentShape s{N, V, D, static_cast<hy_dtype>(dtype)};
    return xent_served(s, true) ? xent_bwd_workspace_bytes(s) : -1;
}

hy_status hyena_xent_fwd(const void* x, const void* w, const int64_t* target, float* loss, float* lse, void* workspace,
                         int64_t workspace_bytes, int64_t N, int64_t V, int64_t D, int32_t dtype, void* hip_stream) {
    hy_status rc = check_xent(N, V, D, dtype);
    if (rc != HY_OK) return rc;
    if (workspace_bytes < 0) return HY_ERR_SHAPE;
    if (N == 0) return HY_OK;
    if (!x || !w || !target || !loss || !lse) return HY_ERR_NULL;
    const XentShape s{N, V, D, static_cast<hy_dtype>(dtype)};
    const int64_t e = size_of(dtype);
    const Range all[5] = {{x, N * D * e}, {w, V * D * e}, {target, N * 8}, {loss, N * 4}, {lse, N * 4}};
    rc = all_aligned(all, 5);
    if (rc == HY_OK) rc = check_disjoint(all, 3, all + 3, 2);
    if (rc == HY_OK && !xent_served(s, false)) return HY_ERR_UNSUPPORTED;
    if (rc == HY_OK) rc = check_workspace(workspace, workspace_bytes, xent_fwd_workspace_bytes(s), all, 5);
    if (rc != HY_OK) return rc;
    XentPtrs p;
    p.x = x, p.w = w, p.target = target, p.loss = loss, p.lse = lse;
    return launch_xent_fwd(p, s, workspace, static_cast<hipStream_t>(hip_stream));
}

hy_status hyena_xent_bwd(const float* dloss, const void* x, const void* w, const int64_t* target, const float* lse, void* dx,
                         void* dw, void* workspace, int64_t workspace_bytes, int64_t N, int64_t V, int64_t D, int32_t dtype,
                         void* hip_stream) {
    hy_status rc = check_xent(N, V, D, dtype);
    if (rc != HY_OK) return rc;
    if (workspace_bytes < 0) return HY_ERR_SHAPE;
    if (!w || !dw || (N > 0 && (!dloss || !x || !target || !lse || !dx))) return HY_ERR_NULL;
    const XentShape s{N, V, D, static_cast<hy_dtype>(dtype)};
    const int64_t e = size_of(dtype);
    const Range all[7] = {{x, N * D * e}, {w, V * D * e}, {target, N * 8}, {dloss, N * 4}, {lse, N * 4}, {dx, N * D * e}, {dw, V * D * e}};
    rc = all_aligned(all, 7);
    if (rc == HY_OK) rc = check_disjoint(all, 5, all + 5, 2);
    if (rc == HY_OK && N > 0 && !xent_served(s, true)) return HY_ERR_UNSUPPORTED;
    if (rc == HY_OK) rc = check_workspace(workspace, workspace_bytes, N > 0 ? xent_bwd_workspace_bytes(s) : 0, all, 7);
    if (rc != HY_OK) return rc;
    XentPtrs p;
    p.dloss = dloss, p.x = x, p.w = w, p.target = target, p.lse_in = lse, p.dx = dx, p.dw = dw;
    return launch_xent_bwd(p, s, workspace, static_cast<hipStream_t>(hip_stream));
}

int64_t hyena_adamw_table_bytes(const hy_adamw_tensor* tensors, int64_t n_tensors) {
    const int64_t chunks = adamw_chunks(tensors, n_tensors);
    return chunks < 0 ? -1 : n_tensors * (int64_t)sizeof(AdamwEntry) + chunks * (int64_t)sizeof(int32_t);
}

hy_status hyena_adamw_table(const hy_adamw_tensor* tensors, int64_t n_tensors, int32_t param, int32_t grad, int32_t bits,
                            int32_t with_master, void* table, int64_t table_bytes, int64_t* chunks) {
    if (!chunks || (n_tensors > 0 && (!tensors || !table))) return HY_ERR_NULL;
    hy_status rc = check_adamw_kinds(param, grad, bits, with_master);
    if (rc != HY_OK) return rc;
    const int64_t all = adamw_chunks(tensors, n_tensors);
    if (all < 0 || table_bytes < hyena_adamw_table_bytes(tensors, n_tensors)) return HY_ERR_SHAPE;
    try {
        std::vector<AdamwEntry> entries;
        rc = adamw_entries(tensors, n_tensors, param, grad, bits, with_master != 0, entries);
        if (rc != HY_OK) return rc;
        *chunks = all;
        if (n_tensors == 0) return HY_OK;
        const size_t head = entries.size() * sizeof(AdamwEntry);
        memcpy(table, entries.data(), head);
        char* owner = static_cast<char*>(table) + head;
        for (int64_t i = 0; i < n_tensors; ++i)
            for (int64_t c = chunks_of(tensors[i].count); c > 0; --c, owner += sizeof(int32_t)) {
                const int32_t me = (int32_t)i;
                memcpy(owner, &me, sizeof me);
            }
    } catch (...) {  // no host memory
        return HY_ERR_SCRATCH;
    }
    return HY_OK;
}

hy_status hyena_adamw_step(const void* table, int64_t n_tensors, int64_t chunks, int32_t param, int32_t grad, int32_t bits,
                           int32_t with_master, double lr, double beta1, double beta2, double eps, int64_t step,
                           const float* grad_scale, void* hip_stream) {
    hy_status rc = check_adamw_kinds(param, grad, bits, with_master);
    if (rc != HY_OK) return rc;
    if (n_tensors < 0 || n_tensors > INT32_MAX || chunks < 0 || chunks > kMostChunks || (n_tensors == 0 && chunks > 0)) return HY_ERR_SHAPE;
    if (step < 1 || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !(eps >= 0)) return HY_ERR_SHAPE;
    if (chunks == 0) return HY_OK;
    if (!table) return HY_ERR_NULL;
    if (!aligned16(table) || reinterpret_cast<uintptr_t>(grad_scale) % 4 != 0) return HY_ERR_ALIGN;
    const AdamwEntry* entries = static_cast<const AdamwEntry*>(table);
    const AdamwHyper h{lr, beta1, beta2, eps, 1.0 - pow(beta1, (double)step), sqrt(1.0 - pow(beta2, (double)step))};
    return launch_adamw(entries, reinterpret_cast<const int32_t*>(entries + n_tensors), grad_scale, h,
                        AdamwShape{chunks, param, grad, bits, with_master != 0}, static_cast<hipStream_t>(hip_stream));
}

int64_t hyena_glr_fwd_workspace_bytes(int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype) {
    if (check_glr(B, L, D, group, dtype) != HY_OK) return -1;
    return empty(B, L, D) ? 0 : glr_fwd_workspace_bytes(glr_shape(B, L, D, group, dtype));
}

int64_t hyena_glr_bwd_workspace_bytes(int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype, int32_t with_marks) {
    if (check_glr(B, L, D, group, dtype) != HY_OK) return -1;
    return empty(B, L, D) ? 0 : glr_bwd_workspace_bytes(glr_shape(B, L, D, group, dtype), with_marks != 0);
}

hy_status hyena_glr_fwd(const void* q, const void* k, const void* v, const void* g, const float* state_in, void* y,
                        float* state_out, float* marks, const int64_t* strides, void* workspace, int64_t workspace_bytes,
                        int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype, void* hip_stream) {
    TuningSnapshot snap;
    hy_status rc = check_glr(B, L, D, group, dtype);
    if (rc != HY_OK) return rc;
    if (!empty(B, L, D) && (!q || !k || !v || !g || !y)) return HY_ERR_NULL;
    if (workspace_bytes < 0) return HY_ERR_SHAPE;
    GlrShape s = glr_shape(B, L, D, group, dtype);
    const int which[4] = {kGlrQ, kGlrK, kGlrV, kGlrG};
    rc = take_strides(s, strides, which, 4);
    if (rc != HY_OK) return rc;
    const int64_t sb = B * D * 4;
    const Range rd[5] = {glr_range(s, q, kGlrQ), glr_range(s, k, kGlrK), glr_range(s, v, kGlrV), glr_range(s, g, kGlrG),
                         {state_in, state_in ? sb : 0}};
    const Range wr[3] = {{y, B * L * D * size_of(dtype)}, {state_out, state_out ? sb : 0}, {marks, marks ? marks_bytes(s) : 0}};
    rc = take_starts(s, rd, 4, 3);
    if (rc == HY_OK) rc = all_aligned(rd + 4, 1);
    if (rc == HY_OK) rc = all_aligned(wr, 3);
    if (rc == HY_OK) rc = check_disjoint(rd, 5, wr, 3);
    if (rc != HY_OK) return rc;
    if (B == 0 || D == 0 || (L == 0 && !state_out)) return HY_OK;
    const Range others[8] = {rd[0], rd[1], rd[2], rd[3], rd[4], wr[0], wr[1], wr[2]};
    rc = check_workspace(workspace, workspace_bytes, L > 0 ? glr_fwd_workspace_bytes(s) : 0, others, 8);
    if (rc != HY_OK) return rc;
    GlrPtrs p;
    p.q = q, p.k = k, p.v = v, p.g = g, p.state_in = state_in;
    p.y = y, p.state_out = state_out, p.marks_out = marks;
    return launch_glr_fwd(p, s, workspace, static_cast<hipStream_t>(hip_stream));
}

hy_status hyena_glr_bwd(const void* dy, const void* q, const void* k, const void* v, const void* g, const float* marks,
                        const float* state_in, const float* dstate_out, void* dq, void* dk, void* dv, void* dg,
                        float* dstate_in, const int64_t* strides, void* workspace, int64_t workspace_bytes, int64_t B, int64_t L,
                        int64_t D, int32_t group, int32_t dtype, void* hip_stream) {
    TuningSnapshot snap;
    hy_status rc = check_glr(B, L, D, group, dtype);
    if (rc != HY_OK) return rc;
    if (!empty(B, L, D) && (!dy || !q || !k || !v || !g || !dq || !dk || !dv || !dg)) return HY_ERR_NULL;
    if (workspace_bytes < 0) return HY_ERR_SHAPE;
    GlrShape s = glr_shape(B, L, D, group, dtype);
    const int which[5] = {kGlrDy, kGlrQ, kGlrK, kGlrV, kGlrG};
    rc = take_strides(s, strides, which, 5);
    if (rc != HY_OK) return rc;
    const int64_t sb = B * D * 4, bytes = B * L * D * size_of(dtype);
    const Range rd[8] = {glr_range(s, dy, kGlrDy), glr_range(s, q, kGlrQ), glr_range(s, k, kGlrK), glr_range(s, v, kGlrV),
                         glr_range(s, g, kGlrG), {marks, marks ? marks_bytes(s) : 0}, {state_in, state_in ? sb : 0},
                         {dstate_out, dstate_out ? sb : 0}};
    const Range wr[5] = {{dq, bytes}, {dk, bytes}, {dv, bytes}, {dg, bytes / group}, {dstate_in, dstate_in ? sb : 0}};
    rc = take_starts(s, rd, 5, 4);
    if (rc == HY_OK) rc = all_aligned(rd + 5, 3);
    if (rc == HY_OK) rc = all_aligned(wr, 5);
    if (rc == HY_OK) rc = check_disjoint(rd, 8, wr, 5);
    if (rc != HY_OK) return rc;
    if (B == 0 || D == 0 || (L == 0 && !dstate_in)) return HY_OK;
    Range others[13];
    for (int i = 0; i < 8; ++i) others[i] = rd[i];
    for (int i = 0; i < 5; ++i) others[8 + i] = wr[i];
    rc = check_workspace(workspace, workspace_bytes, L > 0 ? glr_bwd_workspace_bytes(s, marks != nullptr) : 0, others, 13);
    if (rc != HY_OK) return rc;
    GlrPtrs p;
    p.dy = dy, p.q = q, p.k = k, p.v = v, p.g = g, p.marks = marks, p.state_in = state_in, p.dstate_out = dstate_out;
    p.dq = dq, p.dk = dk, p.dv = dv, p.dg = dg, p.dstate_in = dstate_in;
    return launch_glr_bwd(p, s, workspace, static_cast<hipStream_t>(hip_stream));
}

hy_status hyena_glr_step(const void* q, const void* k, const void* v, const void* g, float* state, void* y, int64_t B, int64_t D,
                         int32_t group, int32_t dtype, void* hip_stream) {
    hy_status rc = check_glr(B, 1, D, group, dtype);
    if (rc != HY_OK) return rc;
    if (!empty(B, 1, D) && (!q || !k || !v || !g || !state || !y)) return HY_ERR_NULL;
    const int64_t bytes = B * D * size_of(dtype);
    const Range rd[4] = {{q, bytes}, {k, bytes}, {v, bytes}, {g, bytes / group}};
    const Range wr[2] = {{y, bytes}, {state, B * D * 4}};
    GlrShape s = glr_shape(B, 1, D, group, dtype);
    rc = take_starts(s, rd, 4, 3);
    if (rc == HY_OK) rc = all_aligned(wr, 2);
    if (rc == HY_OK) rc = check_disjoint(rd, 4, wr, 2);
    if (rc != HY_OK || B == 0 || D == 0) return rc;
    GlrPtrs p;
    p.q = q, p.k = k, p.v = v, p.g = g, p.y = y, p.state_out = state;
    return launch_glr_step(p, s, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
