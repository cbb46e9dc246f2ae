// One token of the gated delta rule for a batch (recblr_delta_step):
//   S' = a S_prev,  u = beta (v - S'^T k),  S = S' + k u^T,  o = scale S^T q
// for every value head's state S [Dk][Dv], a = e^g.
//
// The states are what has to move (Dk Dv floats in and out of each head, against some
// Dk + Dv other elements), so the pass is bound by memory.  Columns of S do not mix: a wave
// takes all Dk rows of a strip of columns, holds them in registers between the two sums over
// the rows, and stores the updated ones, so the state is read and written once.  The strip is
// 32 columns wide (16 bytes to a lane, eight rows to a load) or 64 for at most 64 rows, which
// keeps up to 16 loads of a kilobyte in flight per wave.  32768 heads of 64 x 64: 248 us, 4.4 TB/s
// (a copy of 4 GiB: 4.75 as torch does it, 6.2 with 16 bytes to a lane and no loop).  Few heads are bound by the call: 32 of 128 x 128 take 12 us with it.
#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "ops.hpp"

namespace recblr {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

// VEC columns to a lane, LC lanes to a row, IT loads of kWave / LC rows each.
template <typename T, int VEC, int LC, int IT>
__global__ __launch_bounds__(kWave) void delta_step_kernel(DeltaStepArgs a, int strips) {
    constexpr int RPL = kWave / LC;  // rows in a load
    const int lane = threadIdx.x;
    const int64_t head = blockIdx.x / strips;  // b * HV + hv
    const int strip = (int)(blockIdx.x - head * strips);
    const int64_t b = head / a.HV, hv = head - b * a.HV, h = hv / (a.HV / a.H);
    const int n0 = (strip * LC + lane % LC) * VEC, d0 = lane / LC;
    const bool in_n = n0 < a.Dv;  // VEC = 4 only where Dv is a multiple of 4
    const T* q = (const T*)a.q + (b * a.H + h) * a.Dk;
    const T* k = (const T*)a.k + (b * a.H + h) * a.Dk;
    const int64_t base = head * a.Dk * a.Dv;
    const float* sp = a.h_prev + base;
    float* sn = a.h_next + base;
    float S[IT][VEC], kd[IT], qd[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int d = d0 + i * RPL;
        const bool in = d < a.Dk && in_n;
#pragma unroll
        for (int e = 0; e < VEC; ++e) S[i][e] = 0.0f;
        if (in) {
            if constexpr (VEC == 4) {
                const f4 s = __builtin_nontemporal_load((const f4*)(sp + (int64_t)d * a.Dv + n0));
#pragma unroll
                for (int e = 0; e < 4; ++e) S[i][e] = s[e];
            } else {
                S[i][0] = sp[(int64_t)d * a.Dv + n0];
            }
        }
        kd[i] = d < a.Dk ? to_f32(k[d]) : 0.0f;
        qd[i] = d < a.Dk ? to_f32(q[d]) : 0.0f;
    }
    const float al = delta_decay(to_f32(((const T*)a.g)[head]));
    const float beta = to_f32(((const T*)a.beta)[head]);
    float u[VEC], o[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) u[e] = 0.0f;
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            S[i][e] *= al;
            u[e] = fmaf(S[i][e], kd[i], u[e]);
        }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
#pragma unroll
        for (int d = LC; d < kWave; d <<= 1) u[e] += __shfl_xor(u[e], d);
        const float v = in_n ? to_f32(((const T*)a.v)[head * a.Dv + n0 + e]) : 0.0f;
        u[e] = beta * (v - u[e]);
        o[e] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int d = d0 + i * RPL;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            S[i][e] = fmaf(kd[i], u[e], S[i][e]);
            o[e] = fmaf(S[i][e], qd[i], o[e]);
        }
        if (d < a.Dk && in_n) {
            if constexpr (VEC == 4) {
                const f4 s = {S[i][0], S[i][1], S[i][2], S[i][3]};
                __builtin_nontemporal_store(s, (f4*)(sn + (int64_t)d * a.Dv + n0));
            } else {
                sn[(int64_t)d * a.Dv + n0] = S[i][0];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e)
#pragma unroll
        for (int d = LC; d < kWave; d <<= 1) o[e] += __shfl_xor(o[e], d);
    if (d0 == 0 && in_n) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            store((T*)a.o + head * a.Dv + n0 + e, a.scale * o[e]);
    }
}

template <typename T, int VEC, int LC, int IT>
hipError_t launch_variant(const DeltaStepArgs& a, hipStream_t stream) {
    const int strips = (int)((a.Dv + LC * VEC - 1) / (LC * VEC));
    hipLaunchKernelGGL((delta_step_kernel<T, VEC, LC, IT>), dim3((unsigned)(a.B * a.HV * strips)),
                       dim3(kWave), 0, stream, a, strips);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const DeltaStepArgs& a, hipStream_t stream) {
    const bool vec = a.Dv % 4 == 0 && (uintptr_t)a.h_prev % 16 == 0 && (uintptr_t)a.h_next % 16 == 0;
    if (vec && a.Dk <= 32) return launch_variant<T, 4, 8, 4>(a, stream);
    if (vec && a.Dk <= 64 && a.Dv > 32) return launch_variant<T, 4, 16, 16>(a, stream);
    if (vec) return launch_variant<T, 4, 8, 16>(a, stream);
    if (a.Dk <= 32) return launch_variant<T, 1, 32, 16>(a, stream);
    return launch_variant<T, 1, 32, 64>(a, stream);
}

}  // namespace

hipError_t launch_delta_step(const DeltaStepArgs& a, hipStream_t stream) {
    return a.io == IoType::kF32 ? launch_typed<float>(a, stream) : launch_typed<bf16>(a, stream);
}

}  // namespace recblr
