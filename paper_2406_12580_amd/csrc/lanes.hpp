// Scans and sums over the lanes of a wave by DPP moves.
#ifndef RECBLR_LANES_HPP_
#define RECBLR_LANES_HPP_

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "device_common.hpp"

namespace recblr {
namespace lanes {

typedef unsigned long long u64;

// A register of the lanes that a DPP control names (all lanes active), `old` where there is none.
// These moves take a few cycles, a shuffle through the LDS crossbar a hundred.
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t dpp(uint32_t v, uint32_t old) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, kCtrl, kRows, 0xF, false);
}
template <int kCtrl, int kRows>
__device__ __forceinline__ u64 dpp(u64 v, u64 old) {
    return (u64)dpp<kCtrl, kRows>((uint32_t)(v >> 32), (uint32_t)(old >> 32)) << 32 |
           dpp<kCtrl, kRows>((uint32_t)v, (uint32_t)old);
}
template <int kCtrl, int kRows>
__device__ __forceinline__ float dpp(float v, float old) {
    return __uint_as_float(dpp<kCtrl, kRows>(__float_as_uint(v), __float_as_uint(old)));
}
template <int kCtrl, int kRows>
__device__ __forceinline__ double dpp(double v, double old) {
    return __longlong_as_double(
        (long long)dpp<kCtrl, kRows>((u64)__double_as_longlong(v), (u64)__double_as_longlong(old)));
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) {
    return (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ u64 lane_of(u64 v, int lane) {
    return (u64)lane_of((uint32_t)(v >> 32), lane) << 32 | lane_of((uint32_t)v, lane);
}
__device__ __forceinline__ float lane_of(float v, int lane) {
    return __uint_as_float(lane_of(__float_as_uint(v), lane));
}
__device__ __forceinline__ double lane_of(double v, int lane) {
    return __longlong_as_double((long long)lane_of((u64)__double_as_longlong(v), lane));
}
// op over this lane and those below it: shifts by 1, 2, 4 and 8 within the rows of 16, then a
// row's last lane to the next row, and the second row's to the upper half.  `none` changes
// nothing under op.
template <typename V, typename Op>
__device__ __forceinline__ V wave_scan(V v, V none, Op op) {
    v = op(v, dpp<0x111, 0xF>(v, none));
    v = op(v, dpp<0x112, 0xF>(v, none));
    v = op(v, dpp<0x114, 0xF>(v, none));
    v = op(v, dpp<0x118, 0xF>(v, none));
    v = op(v, dpp<0x142, 0xA>(v, none));
    return op(v, dpp<0x143, 0xC>(v, none));
}
template <typename V>
__device__ __forceinline__ V wave_upto(V v) {
    return wave_scan(v, (V)0, [](V a, V b) { return a + b; });
}
template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
    return lane_of(wave_upto(v), kWave - 1);
}

// Sum over the 16 lanes of a row, in all of them: what is turned round by 8, 4, 2 and 1 lanes.
__device__ __forceinline__ float row_sum(float v) {
    v += dpp<0x128, 0xF>(v, 0.0f);
    v += dpp<0x124, 0xF>(v, 0.0f);
    v += dpp<0x122, 0xF>(v, 0.0f);
    return v + dpp<0x121, 0xF>(v, 0.0f);
}

}  // namespace lanes
}  // namespace recblr

#endif  // RECBLR_LANES_HPP_
