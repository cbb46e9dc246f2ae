// Queries and keys of each head, normalised and rotated by their positions, and the gradients
// (recblr_qk_norm_forward, _backward).
//
// Of a head's vector x, with r = 1 / sqrt(s sum x^2 + eps) and u = r x:
//   y = R (w u);   backward, with g = R^T dy and a = w g:
//   dx = r (a - s u (u . a)),   dw = sum over tokens and heads of g u.
// R turns pairs of elements that lie rotate / 2 apart.  An element is read and written once
// (2 e bytes forward, 3 e backward); u and r are formed again in the backward.
//
// A group of lanes takes a token and walks its heads, so that the token's sines and cosines are
// formed once for all of them.  A lane holds 16 bytes of a head and the lane beside it their
// partners; what they trade, and the two sums of a head, are moves between lanes.
// Widths, rotations, pitches or addresses that are no multiples of that take a wave to a token,
// an element at a time.
//
// Bound by memory.  One MI355X: 204,800 tokens of 2 + 2 heads of 64 bf16, 210 MB forward, 45 us
// (4.7 TB/s); backward with weights 57 us (5.5 TB/s) and 5 for the weights' sums.  131,072 of 4 + 2
// heads of 128 fp32, 805 MB: both together 360 us (5.6 TB/s).  Heads read one ahead, and results written
// past the caches, measured the same.  The other widths' kernel, an element at a time: 204,800 tokens
// of 2 + 2 heads of 17 fp32 160 us forward and 206 backward, bound by its instructions, of 100 bf16
// 327 and 447 and of 72, half rotated, 194 and 427, instructions in half of the cycles; bytes would
// take a fifth or less.
#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "lanes.hpp"
#include "ops.hpp"
#include "wave_tile.hpp"

namespace recblr {
namespace {

using wtile::u4v;

constexpr int kNT = 256;
constexpr int kMaxD = 256;

struct Params {
    const void* x[2];
    const void* dy[2];
    void* out[2];
    const float* w[2];
    int64_t pitch[2];  // elements from token to token of x
    const int32_t* positions;
    float* part;  // backward with weights: [groups][2][D]
    int64_t N;
    int heads[2], D, R;
    float share, eps;
    // turns per position of each pair, base^(-2 i / R) / 2 pi
    double rate[kMaxD / 2];
};

// sin and cos of `turns` full turns: whole turns are taken off in 64 bits, so what is left of a
// far position's angle is exact to fp32.  For bf16 by the hardware, which takes turns: it is off by
// up to 2^-23, small angles' sines too, and a result's rounding to bf16 by 2^-9 of it (100,000
// tokens of 4 + 2 heads of 128: 57 us, 61 with fp32's).  fp32 results would be a tenth farther from
// 64 bits (7.3e-8 for 6.6e-8), and the function costs nothing beside twice the bytes.
template <typename T>
__device__ __forceinline__ void turn(double turns, float& sn, float& cs) {
    const float t = (float)(turns - rint(turns));
    if constexpr (sizeof(T) == 4) {
        sincospif(2.0f * t, &sn, &cs);
    } else {
        sn = __builtin_amdgcn_sinf(t);
        cs = __builtin_amdgcn_cosf(t);
    }
}

template <typename T>
struct Eight;  // 16 bytes as floats
template <>
struct Eight<float> {
    static constexpr int VE = 4;
    __device__ __forceinline__ static void get(u4v v, float (&o)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __uint_as_float(v[e]);
    }
    __device__ __forceinline__ static u4v put(const float (&o)[4]) {
        u4v v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(o[e]);
        return v;
    }
};
template <>
struct Eight<bf16> {
    static constexpr int VE = 8;
    __device__ __forceinline__ static void get(u4v v, float (&o)[8]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[2 * e] = bf16_lo(v[e]);
            o[2 * e + 1] = bf16_hi(v[e]);
        }
    }
    __device__ __forceinline__ static u4v put(const float (&o)[8]) {
        u4v v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = bf16_pair(o[2 * e], o[2 * e + 1]);
        return v;
    }
};

// Sums and largest values over the G lanes of a group (a power of two), in all of them.
template <int G>
struct Group {
    int lane;
    template <typename Op>
    __device__ __forceinline__ float over(float v, Op op) const {
        if constexpr (G >= 2) v = op(v, lanes::dpp<0xB1, 0xF>(v, 0.0f));   // lanes 1, 0, 3, 2
        if constexpr (G >= 4) v = op(v, lanes::dpp<0x4E, 0xF>(v, 0.0f));   // 2, 3, 0, 1
        if constexpr (G >= 8) v = op(v, lanes::dpp<0x141, 0xF>(v, 0.0f));  // eight in reverse
        if constexpr (G >= 16) v = op(v, lanes::dpp<0x140, 0xF>(v, 0.0f));  // sixteen in reverse
        if constexpr (G >= 32) v = op(v, wtile::row_partner(v, (lane >> 4) & 1));
        if constexpr (G >= 64) v = op(v, wtile::half_partner(v, lane >> 5));
        return v;
    }
    __device__ __forceinline__ float sum(float v) const {
        return over(v, [](float a, float b) { return a + b; });
    }
    __device__ __forceinline__ float largest(float v) const {
        return over(v, [](float a, float b) { return fmaxf(a, b); });
    }
};
struct Wave {
    __device__ __forceinline__ float sum(float v) const { return lanes::wave_sum(v); }
    __device__ __forceinline__ float largest(float v) const {
        v = lanes::wave_scan(v, 0.0f, [](float a, float b) { return fmaxf(a, b); });
        return lanes::lane_of(v, kWave - 1);
    }
};

// The sum of squares of a group's head, N elements a lane, times p.share, and eps.  Where it leaves
// fp32's range, or comes so near its lower end that squares lose digits, the head is brought near 1
// first: v by 2^-down, eps by its square.  (A head with an infinity or a NaN has none either.)
struct Squares {
    float sum;
    int down;
};
template <int N, typename Lanes>
__device__ __forceinline__ Squares squares_of(const Params& p, float (&v)[N], const Lanes& all) {
    auto sum = [&](float eps) {
        float q = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) q = fmaf(v[e], v[e], q);
        return fmaf(all.sum(q), p.share, eps);
    };
    Squares s{sum(p.eps), 0};
    const bool far = !(s.sum >= 0x1p-90f && s.sum < __builtin_inff());
    // All of the wave: moves between lanes need all of a group.
    if (__builtin_expect(__ballot(far) != 0, 0)) {
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) top = fmaxf(top, fabsf(v[e]));
        top = all.largest(top);
        const int power = (int)(__float_as_uint(top) >> 23) - 127;
        s.down = !far ? 0 : power < -60 ? -60 : power > 126 ? 126 : power;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = ldexpf(v[e], -s.down);
        s.sum = sum(ldexpf(p.eps, -2 * s.down));
    }
    return s;
}
// dx's factor of what squares_of took off x.
template <int N>
__device__ __forceinline__ void bring_back(const Squares& s, float (&v)[N]) {
    if (__builtin_expect(__ballot(s.down != 0) != 0, 0)) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = ldexpf(v[e], -s.down);
    }
}

// Where a lane's 16 bytes of a head lie.  In the rotated part, lanes 2 c and 2 c + 1 have the c-th
// run and its partner, R / 2 further on, so that a load of the wave is whole cache lines (both runs
// in one lane, half of each line at a time: the backward of 204,800 tokens 67 us, not 58).
template <int VE>
struct Place {
    int at, pair;  // first element; of the rotation's pairs
    bool turned, some;
    __device__ __forceinline__ Place(int l, int D, int R) {
        some = l * VE < D;
        turned = l * VE < R;
        pair = (l >> 1) * VE;
        at = turned ? pair + (l & 1) * (R / 2) : l * VE;
    }
};

// v turned by the angle whose sine is sn for the second of a pair, -sn for the first; v as it is
// where not turned.
template <int VE>
__device__ __forceinline__ void rotate(float (&v)[VE], bool turned, const float (&sn)[VE],
                                       const float (&cs)[VE], float sign) {
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        const float other = lanes::dpp<0xB1, 0xF>(v[e], 0.0f);
        const float r = fmaf(v[e], cs[e], sign * sn[e] * other);
        v[e] = turned ? r : v[e];
    }
}

// kMode: 0 forward, 1 backward, 2 backward with the weights' gradients.
template <typename T, int G, int kMode>
__global__ __launch_bounds__(kNT) void head_kernel(Params p) {
    using E = Eight<T>;
    constexpr int VE = E::VE, kGroups = kNT / G;
    const int t = threadIdx.x, l = t % G;
    const Group<G> group{t & 63};
    const Place<VE> at(l, p.D, p.R);
    float w[2][VE], dw[2][VE];
    const bool second = l & 1;
    double rate[VE / 2];  // each lane of a pair forms half of their sines
#pragma unroll
    for (int e = 0; e < VE / 2; ++e)
        rate[e] = at.turned ? p.rate[at.pair + (second ? VE / 2 : 0) + e] : 0.0;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            w[s][e] = at.some && p.w[s] ? p.w[s][at.at + e] : 1.0f;
            dw[s][e] = 0.0f;
        }
    for (int64_t n = (int64_t)blockIdx.x * kGroups + t / G; n < p.N;
         n += (int64_t)gridDim.x * kGroups) {
        float sn[VE], cs[VE];
        const double pos = p.R ? (double)p.positions[n] : 0.0;
#pragma unroll
        for (int e = 0; e < VE / 2; ++e) {
            float s0, c0;
            turn<T>(pos * rate[e], s0, c0);
            const float s1 = lanes::dpp<0xB1, 0xF>(s0, 0.0f), c1 = lanes::dpp<0xB1, 0xF>(c0, 0.0f);
            sn[e] = second ? s1 : -s0;
            cs[e] = second ? c1 : c0;
            sn[VE / 2 + e] = second ? s0 : -s1;
            cs[VE / 2 + e] = second ? c0 : c1;
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const T* x = (const T*)p.x[s] + n * p.pitch[s];
            const int64_t row = n * p.heads[s];
            for (int h = 0; h < p.heads[s]; ++h) {
                const int64_t o = (row + h) * p.D + at.at;
                u4v rx = {0, 0, 0, 0}, rg = {0, 0, 0, 0};
                if (at.some) {
                    rx = *(const u4v*)(x + h * p.D + at.at);
                    if constexpr (kMode > 0) rg = *(const u4v*)((const T*)p.dy[s] + o);
                }
                float v[VE];
                E::get(rx, v);
                const Squares sq = squares_of(p, v, group);
                const float r = 1.0f / sqrtf(sq.sum);
                if constexpr (kMode == 0) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) v[e] *= r * w[s][e];
                    rotate(v, at.turned, sn, cs, 1.0f);
                } else {
                    float g[VE];
                    E::get(rg, g);
                    rotate(g, at.turned, sn, cs, -1.0f);
                    float dot = 0.0f;
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        v[e] *= r;
                        if constexpr (kMode == 2) dw[s][e] = fmaf(g[e], v[e], dw[s][e]);
                        g[e] *= w[s][e];
                        dot = fmaf(g[e], v[e], dot);
                    }
                    dot = group.sum(dot) * p.share;
#pragma unroll
                    for (int e = 0; e < VE; ++e) v[e] = r * fmaf(-dot, v[e], g[e]);
                    bring_back(sq, v);
                }
                if (at.some) *(u4v*)((T*)p.out[s] + o) = E::put(v);
            }
        }
    }
    if constexpr (kMode == 2) {
        // The groups' sums, in their order.
        __shared__ float all[kNT][VE + 1];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < VE; ++e) all[t][e] = dw[s][e];
            __syncthreads();
            for (int i = t; i < G * VE; i += kNT) {
                const int li = i / VE, e = i % VE;
                const Place<VE> to(li, p.D, p.R);
                if (!to.some) continue;
                float sum = 0.0f;
                for (int g = 0; g < kGroups; ++g) sum += all[g * G + li][e];
                p.part[((int64_t)blockIdx.x * 2 + s) * p.D + to.at + e] = sum;
            }
        }
    }
}

// A wave to a token, element lane + 64 j of a head in its j-th place: any width and alignment.
// Partners are read a second time, from the caches.  Forward, seven waves to a SIMD with a few
// registers of constants spilled: 204,800 tokens of 2 + 2 heads of 17 fp32 160 us, of 72 bf16 194;
// six without 170 and 207.
template <typename T, int kMode>
__global__ __launch_bounds__(kNT, kMode ? 5 : 7) void any_kernel(Params p) {
    constexpr int J = kMaxD / kWave;
    const int lane = threadIdx.x & 63, w0 = wave_id(), half = p.R / 2;
    float w[2][J], dw[2][J];
    bool live[J];
    int mate[J];   // the element's partner
    float side[J]; // -1 for the first of a pair, 1 for the second, 0 for one that is not turned
    double rate[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int i = lane + kWave * j;
        live[j] = i < p.D;
        const bool turned = i < p.R;
        side[j] = !turned ? 0.0f : i < half ? -1.0f : 1.0f;
        mate[j] = !turned ? (live[j] ? i : 0) : i < half ? i + half : i - half;
        rate[j] = turned ? p.rate[i < half ? i : i - half] : 0.0;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            w[s][j] = live[j] && p.w[s] ? p.w[s][i] : 1.0f;
            dw[s][j] = 0.0f;
        }
    }
    for (int64_t n = (int64_t)blockIdx.x * 4 + w0; n < p.N; n += (int64_t)gridDim.x * 4) {
        float sn[J], cs[J];
        const double pos = p.R ? (double)p.positions[n] : 0.0;
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (kWave * j < p.R) turn<T>(pos * rate[j], sn[j], cs[j]);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            for (int h = 0; h < p.heads[s]; ++h) {
                const T* x = (const T*)p.x[s] + n * p.pitch[s] + h * p.D;
                const int64_t o = (n * p.heads[s] + h) * p.D;
                const T* dy = (const T*)p.dy[s] + o;
                T* out = (T*)p.out[s] + o;
                float v[J], m[J], g[J];  // of x; partners, of x or dy; of dy
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    v[j] = live[j] ? to_f32(x[lane + kWave * j]) : 0.0f;
                    m[j] = live[j] ? to_f32((kMode ? dy : x)[mate[j]]) : 0.0f;
                    if constexpr (kMode > 0) g[j] = live[j] ? to_f32(dy[lane + kWave * j]) : 0.0f;
                }
                const Squares sq = squares_of(p, v, Wave{});
                const float r = 1.0f / sqrtf(sq.sum);
                float y[J];
                if constexpr (kMode == 0) {
                    const float by = ldexpf(1.0f, -sq.down);
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        y[j] = v[j] * (r * w[s][j]);
                        if (kWave * j >= p.R) continue;
                        const float wm = p.w[s] && live[j] ? p.w[s][mate[j]] : 1.0f;
                        if (side[j] != 0.0f)
                            y[j] = fmaf(y[j], cs[j], side[j] * (m[j] * by * (r * wm) * sn[j]));
                    }
                } else {
                    float dot = 0.0f;
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        if (side[j] != 0.0f) g[j] = fmaf(g[j], cs[j], -side[j] * (m[j] * sn[j]));
                        v[j] *= r;
                        if constexpr (kMode == 2) dw[s][j] = fmaf(g[j], v[j], dw[s][j]);
                        g[j] *= w[s][j];
                        dot = fmaf(g[j], v[j], dot);
                    }
                    dot = lanes::wave_sum(dot) * p.share;
#pragma unroll
                    for (int j = 0; j < J; ++j) y[j] = r * fmaf(-dot, v[j], g[j]);
                    bring_back(sq, y);
                }
#pragma unroll
                for (int j = 0; j < J; ++j)
                    if (live[j]) out[lane + kWave * j] = from_f32<T>(y[j]);
            }
        }
    }
    if constexpr (kMode == 2) {
        __shared__ float all[4][2][kMaxD];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < J; ++j) all[w0][s][lane + kWave * j] = dw[s][j];
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * p.D; i += kNT) {
            const int s = i >= p.D, e = i - s * p.D;
            p.part[((int64_t)blockIdx.x * 2 + s) * p.D + e] =
                ((all[0][s][e] + all[1][s][e]) + all[2][s][e]) + all[3][s][e];
        }
    }
}

// dw: the rows of partial sums, in 64 bits: sixteen runs of rows, then the runs in order.
__global__ __launch_bounds__(1024) void weights_kernel(const float* part, int rows, int D,
                                                       float* dwq, float* dwk) {
    __shared__ double all[16][kWave];
    const int lane = threadIdx.x & 63, w = wave_id();
    const int i = blockIdx.x * kWave + lane, cols = 2 * D;
    const int run = (rows + 15) / 16;
    double s = 0.0;
    if (i < cols) {
        const int end = min(rows, (w + 1) * run);
#pragma unroll 8
        for (int r = w * run; r < end; ++r) s += (double)part[(int64_t)r * cols + i];
    }
    all[w][lane] = s;
    __syncthreads();
    if (w || i >= cols) return;
    for (int k = 1; k < 16; ++k) s += all[k][lane];
    float* to = i < D ? dwq : dwk;
    if (to) to[i < D ? i : i - D] = (float)s;
}

// ------------------------------------------------------------------ launches
// Workgroups: as many as there are tokens to take (with eight to a compute unit that go on,
// 131,072 tokens took 379 us, not 361), as far as a launch has them, fewer than 2^32 threads; rows
// of partial sums four to a compute unit at most.
int64_t groups_of(int64_t tokens_each, int64_t N, bool sums) {
    const int64_t need = (N + tokens_each - 1) / tokens_each;
    const int64_t most = sums ? 1024 : ((int64_t)1 << 32) / kNT - 1;
    return need < most ? need : most;
}

// Lanes to a token's heads, where all runs of 16 bytes are aligned; 0: the other kernel.
int lanes_of(const QkNormArgs& a, bool backward) {
    const int e = (int)io_bytes(a.io), ve = 16 / e;
    if (a.D % (2 * ve) || a.rotate % (2 * ve)) return 0;
    uintptr_t bits = 0;
    for (int s = 0; s < 2; ++s) {
        bits |= (uintptr_t)a.x[s] | (uintptr_t)a.out[s] | (uintptr_t)(a.pitch[s] * e);
        if (backward) bits |= (uintptr_t)a.dy[s];
    }
    if (bits & 15u) return 0;
    int g = 2;  // pairs of lanes
    while (g * ve < a.D) g *= 2;
    return g;
}

template <typename T, int kMode>
void launch(const Params& p, int g, unsigned groups, hipStream_t st) {
    switch (g) {
        case 0: any_kernel<T, kMode><<<groups, kNT, 0, st>>>(p); break;
        case 2: head_kernel<T, 2, kMode><<<groups, kNT, 0, st>>>(p); break;
        case 4: head_kernel<T, 4, kMode><<<groups, kNT, 0, st>>>(p); break;
        case 8: head_kernel<T, 8, kMode><<<groups, kNT, 0, st>>>(p); break;
        case 16: head_kernel<T, 16, kMode><<<groups, kNT, 0, st>>>(p); break;
        case 32: head_kernel<T, 32, kMode><<<groups, kNT, 0, st>>>(p); break;
        default:
            if constexpr (sizeof(T) == 4) head_kernel<T, 64, kMode><<<groups, kNT, 0, st>>>(p);
    }
}

Params params_of(const QkNormArgs& a) {
    Params p{};
    for (int s = 0; s < 2; ++s) {
        p.x[s] = a.x[s];
        p.dy[s] = a.dy[s];
        p.out[s] = a.out[s];
        p.w[s] = a.w[s];
        p.pitch[s] = a.pitch[s];
        p.heads[s] = a.heads[s];
    }
    p.positions = a.positions;
    p.N = a.N;
    p.D = a.D;
    p.R = a.rotate;
    p.share = a.share;
    p.eps = a.eps;
    // Every eighth power as it is, those between by products: a call has up to 128 of them.
    double between[8];
    for (int i = 0; i < 8 && i < a.rotate / 2; ++i) between[i] = pow(a.base, -2.0 * i / a.rotate);
    for (int i = 0; i < a.rotate / 2; i += 8) {
        const double at = pow(a.base, -2.0 * i / a.rotate) / 6.283185307179586476925;
        for (int j = 0; j < 8 && i + j < a.rotate / 2; ++j) p.rate[i + j] = at * between[j];
    }
    return p;
}

}  // namespace

// Rows of partial sums; the fewest tokens to a workgroup are the other kernel's four.
size_t qk_norm_workspace(int64_t N, int H, int HK, int D, IoType io) {
    return (size_t)groups_of(4, N, true) * 2 * D * 4;
}

hipError_t launch_qk_norm_forward(const QkNormArgs& a, hipStream_t st) {
    const Params p = params_of(a);
    const int g = lanes_of(a, false);
    const unsigned groups = (unsigned)groups_of(g ? kNT / g : 4, a.N, false);
    a.io == IoType::kF32 ? launch<float, 0>(p, g, groups, st) : launch<bf16, 0>(p, g, groups, st);
    return hipGetLastError();
}

hipError_t launch_qk_norm_backward(const QkNormArgs& a, void* ws, hipStream_t st) {
    Params p = params_of(a);
    const int g = lanes_of(a, true);
    const bool sums = a.dw[0] || a.dw[1];
    const unsigned groups = (unsigned)groups_of(g ? kNT / g : 4, a.N, sums);
    p.part = (float*)ws;
    if (a.N == 0) {  // no rows to sum
        if (sums)
            weights_kernel<<<(unsigned)((2 * a.D + 63) / 64), 1024, 0, st>>>(p.part, 0, a.D,
                                                                            a.dw[0], a.dw[1]);
    } else if (sums) {
        a.io == IoType::kF32 ? launch<float, 2>(p, g, groups, st)
                             : launch<bf16, 2>(p, g, groups, st);
        weights_kernel<<<(unsigned)((2 * a.D + 63) / 64), 1024, 0, st>>>(p.part, (int)groups, a.D,
                                                                        a.dw[0], a.dw[1]);
    } else {
        a.io == IoType::kF32 ? launch<float, 1>(p, g, groups, st)
                             : launch<bf16, 1>(p, g, groups, st);
    }
    return hipGetLastError();
}

}  // namespace recblr
