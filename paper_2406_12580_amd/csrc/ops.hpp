// Launchers behind recblr_ops.h (AdamW, sampling, gated delta rule): internal
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

#ifdef __HIPCC__
__device__ __forceinline__ float delta_clamp_g(float g) { return g < kDeltaMinG ? kDeltaMinG : g; }
__device__ __forceinline__ float delta_decay(float g) { return expf(delta_clamp_g(g)); }
#endif

}  // namespace recblr
