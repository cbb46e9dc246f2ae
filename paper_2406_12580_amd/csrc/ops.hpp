// Launchers behind recblr_ops.h (AdamW, sampling, gated delta rule, item lookup, norms of queries
// and keys, policy loss, Muon): internal
// to librecblr.so, called by capi_ops.cpp after it has checked the arguments.
// Each enqueues on `stream` and returns the launch's status.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "launch.hpp"
#include "recblr_ops.h"

namespace recblr {

// ------------------------------------------------------------------ AdamW
struct AdamWHyper {
    double lr, beta1, beta2, eps, inv_bc1, inv_bc2;  // inv_bc: 1 / (1 - beta^t)
};
hipError_t launch_adamw(const recblr_adamw_tensor* tensors, int64_t count, bool bits8, IoType io,
                        const AdamWHyper& h, hipStream_t stream);
hipError_t launch_adamw_moments(const recblr_adamw_tensor* tensors, int64_t count,
                                float* const* m1_out, float* const* m2_out, hipStream_t stream);

// ------------------------------------------------------------------ sampling
struct SampleArgs {
    const void* logits;
    const float* u;
    const float* temperature;  // these four may be null
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    int32_t* ids;
    float* prob;  // may be null
    int64_t B, V;
    IoType io;
};
size_t sample_workspace(int64_t B, int64_t V, IoType io);
hipError_t launch_sample(const SampleArgs& a, void* ws, hipStream_t stream);

// ------------------------------------------------------------------ gated delta rule
struct DeltaStepArgs {
    const void* q;
    const void* k;
    const void* v;
    const void* g;
    const void* beta;
    const float* h_prev;
    void* o;
    float* h_next;
    int64_t B;
    int H, HV, Dk, Dv;
    float scale;
    IoType io;
};
struct DeltaFwdArgs {
    const void* q;
    const void* k;
    const void* v;
    const void* g;
    const void* beta;
    const float* h0;  // may be null (zero state)
    void* o;
    float* hT;      // may be null
    float* states;  // may be null; [B][HV][ceil(L / 64)][Dk][Dv]
    int64_t B, L;
    int H, HV, Dk, Dv;
    float scale;
    IoType io;
};
size_t delta_forward_workspace(int64_t B, int64_t L, int64_t HV, int Dk, int Dv, IoType io);
hipError_t launch_delta_forward(const DeltaFwdArgs& a, void* ws, hipStream_t stream);

struct DeltaBwdArgs {
    const void* q;
    const void* k;
    const void* v;
    const void* g;
    const void* beta;
    const float* states;
    const void* d_o;
    const float* dhT;  // may be null
    void* dq;
    void* dk;
    void* dv;
    void* dg;
    void* dbeta;
    float* dh0;  // may be null
    int64_t B, L;
    int H, HV, Dk, Dv;
    float scale;
    IoType io;
};
size_t delta_backward_workspace(int64_t B, int64_t L, int64_t H, int64_t HV, int Dk, int Dv,
                                IoType io);
hipError_t launch_delta_backward(const DeltaBwdArgs& a, void* ws, hipStream_t stream);
hipError_t launch_delta_step(const DeltaStepArgs& a, hipStream_t stream);

// Log decays below this count as this: e^-100 of a state is nothing next to what it was in fp32,
// and the running sums of g stay finite, where differences of them are taken.
constexpr float kDeltaMinG = -100.0f;

// The way of delta_split.hip, where it is the faster one: the forward, and the backward's
// recurrence into D and Y.  With ws null these write the workspace's size to *bytes only.
bool delta_split(int64_t heads, int64_t L, int Dk, int Dv, bool backward);
hipError_t launch_delta_split_forward(const DeltaFwdArgs& a, void* ws, size_t* bytes,
                                      hipStream_t stream);
hipError_t launch_delta_split_backward(const DeltaBwdArgs& a, float* D, float* Y, void* ws,
                                       size_t* bytes, hipStream_t stream);

// ------------------------------------------------------------------ item lookup
struct EmbedArgs {
    const int32_t* ids;
    const void* src;  // the table, or dout
    void* dst;        // out, or dtable
    int64_t N, V, D;
    float scale;
    int32_t pad_id;
    bool accumulate;
    IoType io;
};
size_t embed_workspace(int64_t N, int64_t V, int64_t D, IoType io);
hipError_t launch_embed_forward(const EmbedArgs& a, hipStream_t stream);
hipError_t launch_embed_backward(const EmbedArgs& a, void* ws, hipStream_t stream);

// ------------------------------------------------------------------ norms of queries and keys
struct QkNormArgs {
    const void* x[2];  // q, k
    int64_t pitch[2];
    const float* w[2];         // may be null
    const int32_t* positions;  // null where rotate = 0
    const void* dy[2];         // backward
    void* out[2];              // y, or dx
    float* dw[2];              // backward, where w is given
    int64_t N;
    int heads[2], D, rotate;
    double base;
    float share, eps;  // share: 1, or 1 / D
    IoType io;
};
size_t qk_norm_workspace(int64_t N, int H, int HK, int D, IoType io);
hipError_t launch_qk_norm_forward(const QkNormArgs& a, hipStream_t stream);
hipError_t launch_qk_norm_backward(const QkNormArgs& a, void* ws, hipStream_t stream);

// ------------------------------------------------------------------ policy loss
struct PolicyArgs {
    const void* logits;
    const int32_t* ids;
    const float* old_logp;
    const float* advantage;
    const float* ref_logp;  // null where kl = 0
    const float* weight;    // may be null
    float* loss;
    float* logp;    // may be null
    void* dlogits;  // may be null, or logits
    int64_t N, V;
    double temperature, clip_low, clip_high, kl;
    IoType io;
};
size_t policy_workspace(int64_t N, int64_t V, IoType io);
hipError_t launch_policy_loss(const PolicyArgs& a, void* ws, hipStream_t stream);

// ------------------------------------------------------------------ Muon
struct MuonHyper {
    double lr, momentum, eps;
    bool nesterov;
    int steps;
};
size_t muon_workspace(const recblr_muon_tensor* tensors, int64_t count);
hipError_t launch_muon(const recblr_muon_tensor* tensors, int64_t count, IoType io,
                       const MuonHyper& h, void* ws, hipStream_t stream);

#ifdef __HIPCC__
__device__ __forceinline__ float delta_clamp_g(float g) { return g < kDeltaMinG ? kDeltaMinG : g; }
__device__ __forceinline__ float delta_decay(float g) { return expf(delta_clamp_g(g)); }
#endif

}  // namespace recblr
