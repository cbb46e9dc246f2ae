// C ABI of recblr_ops.h: argument checks on the host, before any HIP call, and
// dispatch to the launchers of ops.hpp.
#include "recblr_ops.h"

#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <new>

#include "capi_util.hpp"
#include "ops.hpp"

using namespace recblr;

namespace {

// ------------------------------------------------------------------ AdamW
struct Range {
    uintptr_t lo, hi;
    bool written;
};

// No written range overlaps any other.  The ranges of one kind usually come in the order of
// their addresses; sorting is then a pass without exchanges.
bool ranges_disjoint(Range* r, int64_t n) {
    auto less = [](const Range& a, const Range& b) { return a.lo < b.lo; };
    if (!std::is_sorted(r, r + n, less)) std::sort(r, r + n, less);
    uintptr_t end = 0, written_end = 0;  // furthest end so far, of all and of written ranges
    for (int64_t i = 0; i < n; ++i) {
        if (r[i].lo < (r[i].written ? end : written_end)) return false;
        end = std::max(end, r[i].hi);
        if (r[i].written) written_end = std::max(written_end, r[i].hi);
    }
    return true;
}

// The ranges of a call over `count` tensors, up to six each.
struct Ranges {
    static constexpr int64_t kSmall = 64;
    Range small[6 * kSmall];
    Range* r;
    int64_t used = 0;
    explicit Ranges(int64_t count)
        : r(count > kSmall ? new (std::nothrow) Range[6 * count] : small) {}
    Ranges(const Ranges&) = delete;
    ~Ranges() {
        if (r != small) delete[] r;
    }
    void add(const void* p, size_t bytes, bool written) {
        if (p) r[used++] = Range{(uintptr_t)p, (uintptr_t)p + bytes, written};
    }
    bool disjoint() { return ranges_disjoint(r, used); }
};

// A launch has fewer than 2^32 threads: below this many workgroups of 256.
constexpr int64_t kMaxGroups = (int64_t)1 << 24;
constexpr int64_t kMaxAdamN = ((int64_t)1 << 36) - 4096;  // 4096 elements to a workgroup
constexpr int64_t kMaxTensorCount = (int64_t)1 << 24;

int64_t adam_blocks(int64_t n) { return (n + RECBLR_ADAMW_BLOCK - 1) / RECBLR_ADAMW_BLOCK; }

}  // namespace

extern "C" {

int recblr_adamw_update(const recblr_adamw_tensor* tensors, int64_t count, int state_bits, int io,
                        int64_t step, double lr, double beta1, double beta2, double eps,
                        void* stream) {
    if (io != RECBLR_F32 && io != RECBLR_BF16) return RECBLR_ERR_UNSUPPORTED;
    if (state_bits != 8 && state_bits != 32) return RECBLR_ERR_UNSUPPORTED;
    if (count < 0 || step < 1 || (count > 0 && !tensors)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0))
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (count > kMaxTensorCount) return RECBLR_ERR_UNSUPPORTED;
    if (count == 0) return RECBLR_OK;
    const bool bits8 = state_bits == 8;
    const size_t pe = esz(io), me = bits8 ? 1 : 4;
    Ranges ranges(count);
    if (!ranges.r) return RECBLR_ERR_INVALID_ARGUMENT;
    for (int kind = 0; kind < (bits8 ? 6 : 4); ++kind)
        for (int64_t i = 0; i < count; ++i) {
            const recblr_adamw_tensor& t = tensors[i];
            if (t.n < 0) return RECBLR_ERR_INVALID_ARGUMENT;
            if (t.n > kMaxAdamN) return RECBLR_ERR_UNSUPPORTED;
            if (t.n == 0) continue;
            const void* p = kind == 0 ? t.param : kind == 1 ? t.grad : kind == 2 ? t.m1
                            : kind == 3 ? t.m2 : kind == 4 ? t.scale1 : (const void*)t.scale2;
            const size_t e = kind < 2 ? pe : kind < 4 ? me : 4;
            if (!p || !aligned(p, e)) return RECBLR_ERR_INVALID_ARGUMENT;
            const size_t bytes = kind < 4 ? (size_t)t.n * e : (size_t)adam_blocks(t.n) * 4;
            ranges.add(p, bytes, kind != 1);
        }
    if (!ranges.disjoint()) return RECBLR_ERR_INVALID_ARGUMENT;
    const AdamWHyper h{lr, beta1, beta2, eps, 1.0 / (1.0 - pow(beta1, (double)step)),
                       1.0 / (1.0 - pow(beta2, (double)step))};
    return status_of(launch_adamw(tensors, count, bits8, io_of(io), h, (hipStream_t)stream));
}

int recblr_adamw_moments(const recblr_adamw_tensor* tensors, int64_t count,
                         float* const* m1_out, float* const* m2_out, void* stream) {
    if (count < 0 || (count > 0 && !tensors)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (count > kMaxTensorCount) return RECBLR_ERR_UNSUPPORTED;
    if (count == 0 || (!m1_out && !m2_out)) return RECBLR_OK;
    Ranges ranges(count);
    if (!ranges.r) return RECBLR_ERR_INVALID_ARGUMENT;
    for (int64_t i = 0; i < count; ++i) {
        const recblr_adamw_tensor& t = tensors[i];
        if (t.n < 0) return RECBLR_ERR_INVALID_ARGUMENT;
        if (t.n > kMaxAdamN) return RECBLR_ERR_UNSUPPORTED;
        if (t.n == 0) continue;
        const size_t n = (size_t)t.n, s = (size_t)adam_blocks(t.n) * 4;
        float *a = m1_out ? m1_out[i] : nullptr, *b = m2_out ? m2_out[i] : nullptr;
        if ((m1_out && (!a || !t.m1 || !t.scale1)) || (m2_out && (!b || !t.m2 || !t.scale2)))
            return RECBLR_ERR_INVALID_ARGUMENT;
        for (const void* p : {(const void*)a, (const void*)b, (const void*)t.scale1,
                              (const void*)t.scale2})
            if (!aligned(p, 4)) return RECBLR_ERR_INVALID_ARGUMENT;
        ranges.add(a, 4 * n, true);
        ranges.add(b, 4 * n, true);
        ranges.add(t.m1, n, false);
        ranges.add(t.m2, n, false);
        ranges.add(t.scale1, s, false);
        ranges.add(t.scale2, s, false);
    }
    if (!ranges.disjoint()) return RECBLR_ERR_INVALID_ARGUMENT;
    return status_of(launch_adamw_moments(tensors, count, m1_out, m2_out, (hipStream_t)stream));
}

// ------------------------------------------------------------------ sampling

static int sample_sizes(int64_t B, int64_t V, int io) {
    if (io != RECBLR_F32 && io != RECBLR_BF16) return RECBLR_ERR_UNSUPPORTED;
    if (B < 0 || V < 0) return RECBLR_ERR_INVALID_ARGUMENT;
    if (B >= kMaxGroups || V > ((int64_t)1 << 24)) return RECBLR_ERR_UNSUPPORTED;
    if (B * ((V + 4095) / 4096) >= kMaxGroups) return RECBLR_ERR_UNSUPPORTED;  // one each
    return RECBLR_OK;
}

size_t recblr_sample_workspace_size(int64_t B, int64_t V, int io) {
    if (sample_sizes(B, V, io) != RECBLR_OK) return 0;
    return sample_workspace(B, V, io_of(io));
}

int recblr_sample(const void* logits, const float* u, const float* temperature,
                  const int32_t* top_k, const float* top_p, const float* min_p, int32_t* ids,
                  float* prob, int64_t B, int64_t V, int io, void* ws, size_t ws_bytes,
                  void* stream) {
    int st = sample_sizes(B, V, io);
    if (st) return st;
    if (B == 0) return RECBLR_OK;
    if (!ids || !u || (V > 0 && !logits)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (!aligned(logits, esz(io))) return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t n = (size_t)(B * V) * esz(io), s = (size_t)B * 4;
    for (const void* p : {(const void*)u, (const void*)temperature, (const void*)top_k,
                          (const void*)top_p, (const void*)min_p, (const void*)ids,
                          (const void*)prob})
        if (!aligned(p, 4)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (!disjoint({{ids, s}, {prob, s}}, {{logits, n}, {u, s}, {temperature, s}, {top_k, s},
                                          {top_p, s}, {min_p, s}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t need = sample_workspace(B, V, io_of(io));
    st = check_ws(ws, ws_bytes, need);
    if (st) return st;
    if (!disjoint({{ws, need}}, {{logits, n}, {u, s}, {temperature, s}, {top_k, s}, {top_p, s},
                                 {min_p, s}, {ids, s}, {prob, s}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const SampleArgs a{logits, u, temperature, top_k, top_p, min_p, ids, prob, B, V, io_of(io)};
    return status_of(launch_sample(a, ws, (hipStream_t)stream));
}

// ------------------------------------------------------------------ gated delta rule

struct DeltaBytes {
    size_t q, v, g, state, states;
};
static DeltaBytes delta_bytes(int64_t B, int64_t L, int64_t H, int64_t HV, int64_t Dk, int64_t Dv,
                              int io) {
    const size_t e = esz(io), s = (size_t)(B * HV * Dk * Dv) * 4;
    return DeltaBytes{(size_t)(B * L * H * Dk) * e, (size_t)(B * L * HV * Dv) * e,
                      (size_t)(B * L * HV) * e, s, s * (size_t)((L + 63) / 64)};
}

static int delta_sizes(int64_t B, int64_t L, int64_t H, int64_t HV, int64_t Dk, int64_t Dv,
                       int io) {
    if (io != RECBLR_F32 && io != RECBLR_BF16) return RECBLR_ERR_UNSUPPORTED;
    if (B < 0 || L < 0 || H < 1 || HV < 1 || Dk < 1 || Dv < 1 || HV % H)
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (Dk > 128 || Dv > 128) return RECBLR_ERR_UNSUPPORTED;
    if (B >= kMaxGroups || HV > 4096 || L >= ((int64_t)1 << 31)) return RECBLR_ERR_UNSUPPORTED;
    // A strip of at least 32 columns, and a chunk of 64 steps, may be a workgroup of its own.
    if (B * HV * ((Dv + 31) / 32) >= kMaxGroups || B * HV * ((L + 63) / 64) >= kMaxGroups)
        return RECBLR_ERR_UNSUPPORTED;
    return RECBLR_OK;
}

size_t recblr_delta_workspace_size(int op, int64_t B, int64_t L, int64_t H, int64_t HV,
                                   int64_t Dk, int64_t Dv, int io) {
    if (delta_sizes(B, L, H, HV, Dk, Dv, io) != RECBLR_OK || B == 0 || L == 0) return 0;
    if (op == RECBLR_OP_DELTA_FORWARD)
        return delta_forward_workspace(B, L, HV, (int)Dk, (int)Dv, io_of(io));
    if (op == RECBLR_OP_DELTA_BACKWARD)
        return delta_backward_workspace(B, L, H, HV, (int)Dk, (int)Dv, io_of(io));
    return 0;
}

int recblr_delta_forward(const void* q, const void* k, const void* v, const void* g,
                         const void* beta, const float* h0, void* o, float* hT, float* states,
                         int64_t B, int64_t L, int64_t H, int64_t HV, int64_t Dk, int64_t Dv,
                         float scale, int io, void* ws, size_t ws_bytes, void* stream) {
    int st = delta_sizes(B, L, H, HV, Dk, Dv, io);
    if (st) return st;
    if (B == 0) return RECBLR_OK;
    if (L > 0 && (!q || !k || !v || !g || !beta || !o)) return RECBLR_ERR_INVALID_ARGUMENT;
    const DeltaBytes n = delta_bytes(B, L, H, HV, Dk, Dv, io);
    for (const void* p : {q, k, v, g, beta, (const void*)o})
        if (!aligned(p, esz(io))) return RECBLR_ERR_INVALID_ARGUMENT;
    for (const float* p : {h0, (const float*)hT, (const float*)states})
        if (!aligned(p, 4)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (!disjoint({{o, n.v}, {hT, n.state}, {states, n.states}},
                  {{q, n.q}, {k, n.q}, {v, n.v}, {g, n.g}, {beta, n.g}, {h0, n.state}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t need = recblr_delta_workspace_size(RECBLR_OP_DELTA_FORWARD, B, L, H, HV, Dk, Dv,
                                                    io);
    st = check_ws(ws, ws_bytes, need);
    if (st) return st;
    if (!disjoint({{ws, need}}, {{q, n.q}, {k, n.q}, {v, n.v}, {g, n.g}, {beta, n.g},
                                 {h0, n.state}, {o, n.v}, {hT, n.state}, {states, n.states}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const DeltaFwdArgs a{q, k, v, g, beta, h0, o, hT, states, B, L, (int)H, (int)HV, (int)Dk,
                         (int)Dv, scale, io_of(io)};
    return status_of(launch_delta_forward(a, ws, (hipStream_t)stream));
}

int recblr_delta_backward(const void* q, const void* k, const void* v, const void* g,
                          const void* beta, const float* states, const void* d_o,
                          const float* dhT, void* dq, void* dk, void* dv, void* dg, void* dbeta,
                          float* dh0, int64_t B, int64_t L, int64_t H, int64_t HV, int64_t Dk,
                          int64_t Dv, float scale, int io, void* ws, size_t ws_bytes,
                          void* stream) {
    int st = delta_sizes(B, L, H, HV, Dk, Dv, io);
    if (st) return st;
    if (B == 0) return RECBLR_OK;
    if (L > 0 && (!q || !k || !v || !g || !beta || !states || !d_o || !dq || !dk || !dv || !dg ||
                  !dbeta))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const DeltaBytes n = delta_bytes(B, L, H, HV, Dk, Dv, io);
    for (const void* p : {q, k, v, g, beta, d_o, (const void*)dq, (const void*)dk,
                          (const void*)dv, (const void*)dg, (const void*)dbeta})
        if (!aligned(p, esz(io))) return RECBLR_ERR_INVALID_ARGUMENT;
    for (const float* p : {states, dhT, (const float*)dh0})
        if (!aligned(p, 4)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (!disjoint({{dq, n.q}, {dk, n.q}, {dv, n.v}, {dg, n.g}, {dbeta, n.g}, {dh0, n.state}},
                  {{q, n.q}, {k, n.q}, {v, n.v}, {g, n.g}, {beta, n.g}, {states, n.states},
                   {d_o, n.v}, {dhT, n.state}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t need = recblr_delta_workspace_size(RECBLR_OP_DELTA_BACKWARD, B, L, H, HV, Dk, Dv,
                                                    io);
    st = check_ws(ws, ws_bytes, need);
    if (st) return st;
    if (!disjoint({{ws, need}},
                  {{q, n.q}, {k, n.q}, {v, n.v}, {g, n.g}, {beta, n.g}, {states, n.states},
                   {d_o, n.v}, {dhT, n.state}, {dq, n.q}, {dk, n.q}, {dv, n.v}, {dg, n.g},
                   {dbeta, n.g}, {dh0, n.state}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const DeltaBwdArgs a{q, k, v, g, beta, states, d_o, dhT, dq, dk, dv, dg, dbeta, dh0, B, L,
                         (int)H, (int)HV, (int)Dk, (int)Dv, scale, io_of(io)};
    return status_of(launch_delta_backward(a, ws, (hipStream_t)stream));
}

int recblr_delta_step(const void* q, const void* k, const void* v, const void* g,
                      const void* beta, const float* h_prev, void* o, float* h_next, int64_t B,
                      int64_t H, int64_t HV, int64_t Dk, int64_t Dv, float scale, int io,
                      void* stream) {
    int st = delta_sizes(B, 1, H, HV, Dk, Dv, io);
    if (st) return st;
    if (B == 0) return RECBLR_OK;
    if (!q || !k || !v || !g || !beta || !h_prev || !o || !h_next)
        return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t e = esz(io), nq = (size_t)(B * H * Dk) * e, nv = (size_t)(B * HV * Dv) * e,
                 ng = (size_t)(B * HV) * e, ns = (size_t)(B * HV * Dk * Dv) * 4;
    for (const void* p : {q, k, v, g, beta, (const void*)o})
        if (!aligned(p, e)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (!aligned(h_prev, 4) || !aligned(h_next, 4)) return RECBLR_ERR_INVALID_ARGUMENT;
    // h_next may be h_prev exactly (in-place update) but must not partly overlap it.
    if (h_next != h_prev && overlaps({h_next, ns}, {h_prev, ns}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (!disjoint({{o, nv}, {h_next, ns}}, {{q, nq}, {k, nq}, {v, nv}, {g, ng}, {beta, ng}}) ||
        overlaps({o, nv}, {h_prev, ns}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const DeltaStepArgs a{q, k, v, g, beta, h_prev, o, h_next, B, (int)H, (int)HV, (int)Dk,
                          (int)Dv, scale, io_of(io)};
    return status_of(launch_delta_step(a, (hipStream_t)stream));
}

// ------------------------------------------------------------------ item lookup

static int embed_sizes(int64_t N, int64_t V, int64_t D, int io) {
    if (io != RECBLR_F32 && io != RECBLR_BF16) return RECBLR_ERR_UNSUPPORTED;
    if (N < 0 || V < 0 || D < 1) return RECBLR_ERR_INVALID_ARGUMENT;
    if (D > 4096 || V >= ((int64_t)1 << 31) - 1 || N > ((int64_t)1 << 28))
        return RECBLR_ERR_UNSUPPORTED;
    // The lookup has a workgroup to 512 units of a row or more, sums and joins of runs one of 1,024
    // and 512 threads to 1,024 positions.
    if (N * D > ((int64_t)1 << 33) || V * D > ((int64_t)1 << 40)) return RECBLR_ERR_UNSUPPORTED;
    return RECBLR_OK;
}

size_t recblr_embed_workspace_size(int64_t N, int64_t V, int64_t D, int io) {
    if (embed_sizes(N, V, D, io) != RECBLR_OK) return 0;
    return embed_workspace(N, V, D, io_of(io));
}

int recblr_embed_forward(const void* table, const int32_t* ids, void* out, int64_t N, int64_t V,
                         int64_t D, float scale, int32_t pad_id, int io, void* stream) {
    const int st = embed_sizes(N, V, D, io);
    if (st) return st;
    if (N == 0) return RECBLR_OK;
    if (!ids || !out || (V > 0 && !table)) return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t e = esz(io), n = (size_t)(N * D) * e, t = (size_t)(V * D) * e;
    if (!aligned(table, e) || !aligned(out, e) || !aligned(ids, 4))
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (!disjoint({{out, n}}, {{table, t}, {ids, (size_t)N * 4}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const EmbedArgs a{ids, table, out, N, V, D, scale, pad_id, false, io_of(io)};
    return status_of(launch_embed_forward(a, (hipStream_t)stream));
}

int recblr_embed_backward(const int32_t* ids, const void* dout, void* dtable, int64_t N,
                          int64_t V, int64_t D, float scale, int32_t pad_id, int accumulate,
                          int io, void* ws, size_t ws_bytes, void* stream) {
    int st = embed_sizes(N, V, D, io);
    if (st) return st;
    if (V == 0 || (N == 0 && accumulate)) return RECBLR_OK;
    if (!dtable || (N > 0 && (!ids || !dout))) return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t e = esz(io), n = (size_t)(N * D) * e, t = (size_t)(V * D) * e;
    if (!aligned(dout, e) || !aligned(dtable, e) || !aligned(ids, 4))
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (!disjoint({{dtable, t}}, {{dout, n}, {ids, (size_t)N * 4}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t need = embed_workspace(N, V, D, io_of(io));
    st = check_ws(ws, ws_bytes, need);
    if (st) return st;
    if (!disjoint({{ws, need}}, {{dout, n}, {ids, (size_t)N * 4}, {dtable, t}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const EmbedArgs a{ids, dout, dtable, N, V, D, scale, pad_id, accumulate != 0, io_of(io)};
    return status_of(launch_embed_backward(a, ws, (hipStream_t)stream));
}

// ------------------------------------------------------------------ norms of queries and keys

static int qk_sizes(int64_t N, int64_t H, int64_t HK, int64_t D, int io) {
    if (io != RECBLR_F32 && io != RECBLR_BF16) return RECBLR_ERR_UNSUPPORTED;
    if (N < 0 || H < 1 || HK < 1 || D < 1) return RECBLR_ERR_INVALID_ARGUMENT;
    if (D > 256 || H > 4096 || HK > 4096 || N >= ((int64_t)1 << 31) - 256)
        return RECBLR_ERR_UNSUPPORTED;
    return RECBLR_OK;
}

size_t recblr_qk_norm_workspace_size(int64_t N, int64_t H, int64_t HK, int64_t D, int io) {
    if (qk_sizes(N, H, HK, D, io) != RECBLR_OK || N == 0) return 0;
    return qk_norm_workspace(N, (int)H, (int)HK, (int)D, io_of(io));
}

// What forward and backward check alike, and their common arguments.
static int qk_args(QkNormArgs* a, const void* q, const void* k, int64_t q_pitch, int64_t k_pitch,
                   const float* wq, const float* wk, const int32_t* positions, int64_t N,
                   int64_t H, int64_t HK, int64_t D, int64_t rotate, double base, int norm,
                   float eps, int io) {
    const int st = qk_sizes(N, H, HK, D, io);
    if (st) return st;
    if (rotate < 0 || rotate > D || rotate % 2 || q_pitch < H * D || k_pitch < HK * D)
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (norm != RECBLR_NORM_L2 && norm != RECBLR_NORM_RMS) return RECBLR_ERR_INVALID_ARGUMENT;
    if (!(eps > 0.0f) || !(base > 0.0)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (q_pitch >= ((int64_t)1 << 31) || k_pitch >= ((int64_t)1 << 31))
        return RECBLR_ERR_UNSUPPORTED;
    if (N > 0 && (!q || !k || (rotate > 0 && !positions))) return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t e = esz(io);
    if (!aligned(q, e) || !aligned(k, e) || !aligned(wq, 4) || !aligned(wk, 4) ||
        !aligned(positions, 4))
        return RECBLR_ERR_INVALID_ARGUMENT;
    *a = QkNormArgs{};
    a->x[0] = q;
    a->x[1] = k;
    a->pitch[0] = q_pitch;
    a->pitch[1] = k_pitch;
    a->w[0] = wq;
    a->w[1] = wk;
    a->positions = rotate > 0 ? positions : nullptr;
    a->N = N;
    a->heads[0] = (int)H;
    a->heads[1] = (int)HK;
    a->D = (int)D;
    a->rotate = (int)rotate;
    a->base = base;
    a->share = norm == RECBLR_NORM_RMS ? 1.0f / (float)D : 1.0f;
    a->eps = eps;
    a->io = io_of(io);
    return RECBLR_OK;
}

// Bytes of N tokens of `width` elements that lie `pitch` apart.
static size_t pitched(int64_t N, int64_t pitch, int64_t width, size_t e) {
    return N > 0 ? (size_t)((N - 1) * pitch + width) * e : 0;
}

int recblr_qk_norm_forward(const void* q, const void* k, int64_t q_pitch, int64_t k_pitch,
                           const float* wq, const float* wk, const int32_t* positions,
                           void* q_out, void* k_out, int64_t N, int64_t H, int64_t HK, int64_t D,
                           int64_t rotate, double base, int norm, float eps, int io,
                           void* stream) {
    QkNormArgs a;
    const int st = qk_args(&a, q, k, q_pitch, k_pitch, wq, wk, positions, N, H, HK, D, rotate,
                           base, norm, eps, io);
    if (st) return st;
    if (N == 0) return RECBLR_OK;
    if (!q_out || !k_out || !aligned(q_out, esz(io)) || !aligned(k_out, esz(io)))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t e = esz(io), w = (size_t)D * 4;
    if (!disjoint({{q_out, (size_t)(N * H * D) * e}, {k_out, (size_t)(N * HK * D) * e}},
                  {{q, pitched(N, q_pitch, H * D, e)}, {k, pitched(N, k_pitch, HK * D, e)},
                   {wq, w}, {wk, w}, {a.positions, (size_t)N * 4}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    a.out[0] = q_out;
    a.out[1] = k_out;
    return status_of(launch_qk_norm_forward(a, (hipStream_t)stream));
}

int recblr_qk_norm_backward(const void* q, const void* k, int64_t q_pitch, int64_t k_pitch,
                            const float* wq, const float* wk, const int32_t* positions,
                            const void* dq_out, const void* dk_out, void* dq, void* dk,
                            float* dwq, float* dwk, int64_t N, int64_t H, int64_t HK, int64_t D,
                            int64_t rotate, double base, int norm, float eps, int io, void* ws,
                            size_t ws_bytes, void* stream) {
    QkNormArgs a;
    int st = qk_args(&a, q, k, q_pitch, k_pitch, wq, wk, positions, N, H, HK, D, rotate, base,
                     norm, eps, io);
    if (st) return st;
    // Weights and their gradients come together.
    if ((dwq != nullptr) != (wq != nullptr) || (dwk != nullptr) != (wk != nullptr))
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (!aligned(dwq, 4) || !aligned(dwk, 4)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (N == 0 && !dwq && !dwk) return RECBLR_OK;
    const size_t e = esz(io), w = (size_t)D * 4;
    const size_t nq = (size_t)(N * H * D) * e, nk = (size_t)(N * HK * D) * e;
    if (N > 0) {
        for (const void* p : {dq_out, dk_out, (const void*)dq, (const void*)dk})
            if (!p || !aligned(p, e)) return RECBLR_ERR_INVALID_ARGUMENT;
    }
    if (!disjoint({{dq, nq}, {dk, nk}, {dwq, w}, {dwk, w}},
                  {{q, pitched(N, q_pitch, H * D, e)}, {k, pitched(N, k_pitch, HK * D, e)},
                   {wq, w}, {wk, w}, {a.positions, (size_t)N * 4}, {dq_out, nq}, {dk_out, nk}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t need = dwq || dwk ? recblr_qk_norm_workspace_size(N, H, HK, D, io) : 0;
    st = check_ws(ws, ws_bytes, need);
    if (st) return st;
    if (!disjoint({{ws, need}},
                  {{q, pitched(N, q_pitch, H * D, e)}, {k, pitched(N, k_pitch, HK * D, e)},
                   {wq, w}, {wk, w}, {a.positions, (size_t)N * 4}, {dq_out, nq}, {dk_out, nk},
                   {dq, nq}, {dk, nk}, {dwq, w}, {dwk, w}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    a.dy[0] = dq_out;
    a.dy[1] = dk_out;
    a.out[0] = dq;
    a.out[1] = dk;
    a.dw[0] = dwq;
    a.dw[1] = dwk;
    return status_of(launch_qk_norm_backward(a, ws, (hipStream_t)stream));
}

// ------------------------------------------------------------------ policy loss

static int policy_sizes(int64_t N, int64_t V, int io) {
    if (io != RECBLR_F32 && io != RECBLR_BF16) return RECBLR_ERR_UNSUPPORTED;
    if (N < 0 || V < 0 || (N > 0 && V == 0)) return RECBLR_ERR_INVALID_ARGUMENT;
    // A row may be 1024 threads, or a piece of 2048 items a workgroup.
    if (N >= ((int64_t)1 << 22) || V > ((int64_t)1 << 24)) return RECBLR_ERR_UNSUPPORTED;
    if (N * ((V + 2047) / 2048) >= kMaxGroups) return RECBLR_ERR_UNSUPPORTED;
    return RECBLR_OK;
}

size_t recblr_policy_loss_workspace_size(int64_t N, int64_t V, int io) {
    if (policy_sizes(N, V, io) != RECBLR_OK) return 0;
    return policy_workspace(N, V, io_of(io));
}

int recblr_policy_loss(const void* logits, const int32_t* ids, const float* old_logp,
                       const float* advantage, const float* ref_logp, const float* weight,
                       float* loss, float* logp, void* dlogits, int64_t N, int64_t V,
                       double temperature, double clip_low, double clip_high, double kl, int io,
                       void* ws, size_t ws_bytes, void* stream) {
    int st = policy_sizes(N, V, io);
    if (st) return st;
    // As floats, so that the limits are limits for a caller who has a float too.
    if (!((float)temperature >= 1e-30f && (float)temperature <= 1e30f)) return RECBLR_ERR_INVALID_ARGUMENT;
    for (double x : {clip_low, clip_high, kl})
        if (!(x >= 0.0 && x <= 3.0e38)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (!loss || !aligned(loss, 4)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (N > 0 && (!logits || !ids || !old_logp || !advantage || (kl > 0.0 && !ref_logp)))
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (!aligned(logits, esz(io)) || !aligned(dlogits, esz(io)))
        return RECBLR_ERR_INVALID_ARGUMENT;
    for (const void* p : {(const void*)ids, (const void*)old_logp, (const void*)advantage,
                          (const void*)ref_logp, (const void*)weight, (const void*)logp})
        if (!aligned(p, 4)) return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t n = (size_t)(N * V) * esz(io), s = (size_t)N * 4;
    // dlogits may be logits exactly.
    if (dlogits != logits && overlaps({dlogits, n}, {logits, n}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (!disjoint({{dlogits, n}, {loss, 4}, {logp, s}},
                  {{ids, s}, {old_logp, s}, {advantage, s}, {ref_logp, s}, {weight, s}}) ||
        !disjoint({{loss, 4}, {logp, s}}, {{logits, n}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const size_t need = policy_workspace(N, V, io_of(io));
    st = check_ws(ws, ws_bytes, need);
    if (st) return st;
    if (!disjoint({{ws, need}}, {{logits, n}, {dlogits, n}, {loss, 4}, {logp, s}, {ids, s},
                                 {old_logp, s}, {advantage, s}, {ref_logp, s}, {weight, s}}))
        return RECBLR_ERR_INVALID_ARGUMENT;
    const PolicyArgs a{logits, ids, old_logp, advantage, kl > 0.0 ? ref_logp : nullptr, weight,
                       loss, logp, dlogits, N, V, temperature, clip_low, clip_high, kl,
                       io_of(io)};
    return status_of(launch_policy_loss(a, ws, (hipStream_t)stream));
}

// ------------------------------------------------------------------ Muon

static int muon_sizes(const recblr_muon_tensor* tensors, int64_t count, int io) {
    if (io != RECBLR_F32 && io != RECBLR_BF16) return RECBLR_ERR_UNSUPPORTED;
    if (count < 0 || (count > 0 && !tensors)) return RECBLR_ERR_INVALID_ARGUMENT;
    if (count > ((int64_t)1 << 20)) return RECBLR_ERR_UNSUPPORTED;
    for (int64_t i = 0; i < count; ++i)
        if (tensors[i].rows < 0 || tensors[i].cols < 0) return RECBLR_ERR_INVALID_ARGUMENT;
    constexpr int64_t kSide = (int64_t)1 << 16, kSize = (int64_t)1 << 30;
    for (int64_t i = 0; i < count; ++i) {
        const recblr_muon_tensor& t = tensors[i];
        if (t.rows > kSide || t.cols > kSide || t.rows * t.cols > kSize)
            return RECBLR_ERR_UNSUPPORTED;
    }
    return RECBLR_OK;
}

size_t recblr_muon_workspace_size(const recblr_muon_tensor* tensors, int64_t count, int io) {
    if (muon_sizes(tensors, count, io) != RECBLR_OK) return 0;
    return muon_workspace(tensors, count);
}

int recblr_muon_update(const recblr_muon_tensor* tensors, int64_t count, int io, double lr,
                       double momentum, int nesterov, int steps, double eps, void* ws,
                       size_t ws_bytes, void* stream) {
    int st = muon_sizes(tensors, count, io);
    if (st) return st;
    // 2^12 / eps is held in 64 bits.
    if (!(momentum >= 0.0 && momentum < 1.0) || !(eps >= 1e-300) || steps < 1)
        return RECBLR_ERR_INVALID_ARGUMENT;
    if (steps > 64) return RECBLR_ERR_UNSUPPORTED;
    if (count == 0) return RECBLR_OK;
    const size_t e = esz(io);
    Ranges ranges(count + 1);
    if (!ranges.r) return RECBLR_ERR_INVALID_ARGUMENT;
    for (int kind = 0; kind < 3; ++kind)
        for (int64_t i = 0; i < count; ++i) {
            const recblr_muon_tensor& t = tensors[i];
            const size_t n = (size_t)(t.rows * t.cols);
            if (n == 0) continue;
            const void* p = kind == 0 ? t.param : kind == 1 ? t.grad : (const void*)t.m;
            const size_t each = kind < 2 ? e : 4;
            if (!p || !aligned(p, each)) return RECBLR_ERR_INVALID_ARGUMENT;
            ranges.add(p, n * each, kind != 1);
        }
    const size_t need = muon_workspace(tensors, count);
    st = check_ws(ws, ws_bytes, need);
    if (st) return st;
    if (need) ranges.add(ws, need, true);
    if (!ranges.disjoint()) return RECBLR_ERR_INVALID_ARGUMENT;
    const MuonHyper h{lr, momentum, eps, nesterov != 0, steps};
    return status_of(launch_muon(tensors, count, io_of(io), h, ws, (hipStream_t)stream));
}

}  // extern "C"
