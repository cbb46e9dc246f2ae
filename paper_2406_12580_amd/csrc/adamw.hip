// AdamW over a list of tensors in one launch per kMaxTensors of them, with
// float moments or moments in 8-bit codes (recblr_adamw_update).
//
// One element reads and writes 28 bytes with float moments (fp32 I/O) and 16
// with codes.  The tables travel as kernel arguments, so a call is one launch
// for every kMaxTensors tensors and needs no copies.  A workgroup takes kChunk
// consecutive elements of one tensor, found by comparing its number with every
// tensor's first chunk (all scalar).  A wave takes 256 elements at a time, four
// to a lane: with codes that is one block of a scale, whose maximum stays
// within the wave.
//
// With float moments the pass is bound by memory: 134 million fp32 parameters
// take 705 us (5.3 TB/s), bf16 ones 574 us (5.1 TB/s), where a copy of 4 GiB,
// 16 bytes to a lane, reaches 6.2.  With codes it is bound by their arithmetic,
// in 64 bits: 562 us for fp32 parameters and 522 us for bf16 ones, 16 and 10
// bytes an element (2.6 TB/s).  A model's 45 small tensors are two launches of
// 6 us, behind 30 us of the call from Python.
#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "ops.hpp"

namespace recblr {
namespace {

constexpr int kNT = 256;
constexpr int kMaxTensors = 40;  // a table of 40 is 2.8 KB of the 4 KB of kernel arguments
constexpr int kBlock = RECBLR_ADAMW_BLOCK;
constexpr int kChunk = 16 * kBlock;  // four blocks to each of a workgroup's four waves
static_assert(kBlock == 4 * kWave, "a wave covers a block with four elements to a lane");

struct Entry {
    void* p;
    const void* g;
    void* m1;
    void* m2;
    float* s1;
    float* s2;
    int64_t n;
    float wd;      // 1 - lr wd, rounded once from 64 bits
    uint32_t vec;  // all pointers take vector accesses
};
struct Table {
    uint32_t first[kMaxTensors];  // first chunk of each tensor; unused ones 2^32 - 1
    Entry t[kMaxTensors];
};
static_assert(sizeof(Table) <= 3800, "kernel arguments end at 4 KB");

struct Hyper32 {
    float beta1, one_beta1, beta2, one_beta2, eps, lr_bc1, inv_bc2;
};

__device__ __forceinline__ int find(const uint32_t (&first)[kMaxTensors], uint32_t chunk) {
    int at = -1;
#pragma unroll
    for (int i = 0; i < kMaxTensors; ++i) at += chunk >= first[i];
    return at;
}

template <typename T>
__device__ __forceinline__ void load4(const T* p, int64_t i, int64_t n, bool vec, float (&v)[4]) {
    if (vec && i + 4 <= n) {
        unpack_vec<T, 4>(*(const typename VecT<T, 4>::type*)(p + i), v);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = i + k < n ? to_f32(p[i + k]) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int64_t i, int64_t n, bool vec, const float (&v)[4]) {
    if (vec && i + 4 <= n) {
        typename VecT<T, 4>::type w;
        if constexpr (sizeof(T) == 4) {
            w = {v[0], v[1], v[2], v[3]};
        } else {
            w = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        }
        *(typename VecT<T, 4>::type*)(p + i) = w;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) p[i + k] = from_f32<T>(v[k]);
    }
}
// Four codes as the bytes of a word.
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t i, int64_t n, bool vec) {
    if (vec && i + 4 <= n) return *(const uint32_t*)(p + i);
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) w |= (uint32_t)p[i + k] << (8 * k);
    return w;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t i, int64_t n, bool vec,
                                            uint32_t w) {
    if (vec && i + 4 <= n) {
        *(uint32_t*)(p + i) = w;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) p[i + k] = (uint8_t)(w >> (8 * k));
}

// Largest of a wave's values by their bits: for magnitudes that is their order, with NaN
// above infinity, so a NaN stays visible.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, d);
        v = v > o ? v : o;
    }
    return v;
}

// c / 127 squared with its sign, times the scale; ((c + 1) / 256)^4 times the scale.  The
// integer powers are exact, so each value is rounded once or twice in 64 bits.
__device__ __forceinline__ double value1(double s, int c) {
    return s * ((double)(c * (c < 0 ? -c : c)) * (1.0 / 16129.0));
}
__device__ __forceinline__ double value2(double s, int c) {
    const double q = (double)((c + 1) * (c + 1));
    return s * (q * q * 0x1p-32);
}

// A block's scale as the encoders use it: whether it is positive (else all codes are the
// lowest), a power of two that brings tiny and huge ones (and, in 64 bits, the moments with
// them) to where neither they nor their inverse are denormal, and that inverse.
struct Scale {
    float s, inv;
    double up;
    bool some;
    __device__ __forceinline__ explicit Scale(float scale) {
        s = scale;
        some = s > 0.0f;
        const float by = s < 1e-20f ? 0x1p66f : s > 1e20f ? 0x1p-66f : 1.0f;
        up = by;
        inv = fast_rcp(s * by);
    }
};

// Nearest code of m on the root's scale.  Hardware root and reciprocal (an ulp or two) give the
// code to within one; which side of a border between two codes m falls on, s ((c +- 1/2) /
// 127)^2, is decided in 64 bits.  IEEE division and roots here cost 45 instructions more.
__device__ __forceinline__ int code1(double m, const Scale& s) {
    const double a = fabs(m);
    int c = (int)rintf(127.0f * fast_sqrt((float)(a * s.up) * s.inv));
    c = c < 0 ? 0 : c > 127 ? 127 : c;
    const double x = a * 16129.0, up = c + 0.5, dn = c - 0.5;
    const bool more = x > (double)s.s * (up * up), less = x < (double)s.s * (dn * dn);
    c += more && c < 127 ? 1 : less && c > 0 ? -1 : 0;
    c = s.some ? c : 0;
    return m < 0.0 ? -c : c;
}
// The same for v: borders s ((c + 1 +- 1/2) / 256)^4.
__device__ __forceinline__ int code2(double v, const Scale& s) {
    int c = (int)rintf(256.0f * fast_sqrt(fast_sqrt((float)(v * s.up) * s.inv)));
    c = c < 1 ? 1 : c > 256 ? 256 : c;
    const double x = v * 0x1p32;
    const double up = (c + 0.5) * (c + 0.5), dn = (c - 0.5) * (c - 0.5);
    const bool more = x > (double)s.s * (up * up), less = x < (double)s.s * (dn * dn);
    c += more && c < 256 ? 1 : less && c > 1 ? -1 : 0;
    return s.some ? c - 1 : 0;
}

template <typename T>
__global__ __launch_bounds__(kNT) void adamw32_kernel(Table tab, Hyper32 h) {
    const int at = find(tab.first, blockIdx.x);
    const Entry& e = tab.t[at];
    const int64_t n = e.n;
    const bool vec = e.vec != 0;
    const int64_t base =
        (int64_t)(blockIdx.x - tab.first[at]) * kChunk + (int64_t)threadIdx.x * 4;
    T* p = (T*)e.p;
    const T* g = (const T*)e.g;
    float *m1 = (float*)e.m1, *m2 = (float*)e.m2;
#pragma unroll 2
    for (int j = 0; j < kChunk / (4 * kNT); ++j) {
        const int64_t i = base + j * 4 * kNT;
        if (i >= n) break;
        float pv[4], gv[4], a[4], b[4];
        load4(p, i, n, vec, pv);
        load4(g, i, n, vec, gv);
        load4(m1, i, n, vec, a);
        load4(m2, i, n, vec, b);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            a[k] = fmaf(h.beta1, a[k], h.one_beta1 * gv[k]);
            b[k] = fmaf(h.beta2, b[k], h.one_beta2 * gv[k] * gv[k]);
            pv[k] = pv[k] * e.wd - h.lr_bc1 * a[k] / (sqrtf(b[k] * h.inv_bc2) + h.eps);
        }
        store4(p, i, n, vec, pv);
        store4(m1, i, n, vec, a);
        store4(m2, i, n, vec, b);
    }
}

template <typename T>
__global__ __launch_bounds__(kNT) void adamw8_kernel(Table tab, AdamWHyper h, float lr_bc1,
                                                     float inv_bc2, float eps) {
    const int at = find(tab.first, blockIdx.x);
    const Entry& e = tab.t[at];
    const int64_t n = e.n;
    const bool vec = e.vec != 0;
    const int lane = threadIdx.x % kWave;
    const int64_t block0 =
        (int64_t)(blockIdx.x - tab.first[at]) * (kChunk / kBlock) + wave_id();
    T* p = (T*)e.p;
    const T* g = (const T*)e.g;
    uint8_t *c1 = (uint8_t*)e.m1, *c2 = (uint8_t*)e.m2;
    const double ob1 = 1.0 - h.beta1, ob2 = 1.0 - h.beta2;
#pragma unroll 2
    for (int j = 0; j < kChunk / (4 * kNT); ++j) {
        const int64_t block = block0 + j * (kNT / kWave);
        const int64_t i = block * kBlock + lane * 4;
        if (block * kBlock >= n) break;
        float pv[4], gv[4];
        load4(p, i, n, vec, pv);
        load4(g, i, n, vec, gv);
        const uint32_t w1 = load_codes(c1, i, n, vec), w2 = load_codes(c2, i, n, vec);
        const double s1 = e.s1[block], s2 = e.s2[block];
        double m[4], v[4];
        uint32_t top1 = 0, top2 = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const double gd = gv[k];
            m[k] = fma(h.beta1, value1(s1, (int8_t)(w1 >> (8 * k))), ob1 * gd);
            v[k] = fma(h.beta2, value2(s2, (uint8_t)(w2 >> (8 * k))), ob2 * gd * gd);
            pv[k] = pv[k] * e.wd - lr_bc1 * (float)m[k] / (sqrtf((float)v[k] * inv_bc2) + eps);
            // What lies behind the tensor's end has no say in the block's scale.
            const bool in = i + k < n;
            const uint32_t a = in ? __float_as_uint(fabsf((float)m[k])) : 0u;
            const uint32_t b = in ? __float_as_uint((float)v[k]) & 0x7FFFFFFFu : 0u;
            top1 = top1 > a ? top1 : a;
            top2 = top2 > b ? top2 : b;
        }
        store4(p, i, n, vec, pv);
        const float n1 = __uint_as_float(wave_max(top1)), n2 = __uint_as_float(wave_max(top2));
        const Scale e1(n1), e2(n2);
        uint32_t o1 = 0, o2 = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            o1 |= (uint32_t)(uint8_t)code1(m[k], e1) << (8 * k);
            o2 |= (uint32_t)(uint8_t)code2(v[k], e2) << (8 * k);
        }
        store_codes(c1, i, n, vec, o1);
        store_codes(c2, i, n, vec, o2);
        if (lane == 0) {
            e.s1[block] = n1;
            e.s2[block] = n2;
        }
    }
}

// The values of the codes: p is the output of m1 (or null), g's place holds that of m2.
__global__ __launch_bounds__(kNT) void adamw_moments_kernel(Table tab) {
    const int at = find(tab.first, blockIdx.x);
    const Entry& e = tab.t[at];
    const int64_t n = e.n;
    const bool vec = e.vec != 0;
    const int lane = threadIdx.x % kWave;
    const int64_t block0 =
        (int64_t)(blockIdx.x - tab.first[at]) * (kChunk / kBlock) + wave_id();
    float *out1 = (float*)e.p, *out2 = (float*)const_cast<void*>(e.g);
#pragma unroll 2
    for (int j = 0; j < kChunk / (4 * kNT); ++j) {
        const int64_t block = block0 + j * (kNT / kWave);
        const int64_t i = block * kBlock + lane * 4;
        if (block * kBlock >= n) break;
        float v[4];
        if (out1) {
            const uint32_t w = load_codes((const uint8_t*)e.m1, i, n, vec);
            const double s = e.s1[block];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = (float)value1(s, (int8_t)(w >> (8 * k)));
            store4(out1, i, n, vec, v);
        }
        if (out2) {
            const uint32_t w = load_codes((const uint8_t*)e.m2, i, n, vec);
            const double s = e.s2[block];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = (float)value2(s, (uint8_t)(w >> (8 * k)));
            store4(out2, i, n, vec, v);
        }
    }
}

bool takes(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// Fills tables of up to kMaxTensors tensors and fewer than 2^24 chunks, and launches each.
template <typename Fill, typename Launch>
hipError_t in_tables(int64_t count, const recblr_adamw_tensor* tensors, Fill fill, Launch launch) {
    Table tab;
    int used = 0;
    int64_t chunks = 0;
    auto flush = [&]() -> hipError_t {
        if (used == 0) return hipSuccess;
        for (int i = used; i < kMaxTensors; ++i) {
            tab.first[i] = 0xFFFFFFFFu;
            tab.t[i] = Entry{};
        }
        launch(tab, (unsigned)chunks);
        used = 0;
        chunks = 0;
        return hipGetLastError();
    };
    for (int64_t i = 0; i < count; ++i) {
        const int64_t need = (tensors[i].n + kChunk - 1) / kChunk;
        if (need == 0) continue;
        if (used == kMaxTensors || chunks + need >= (1 << 24)) {
            const hipError_t e = flush();
            if (e != hipSuccess) return e;
        }
        tab.first[used] = (uint32_t)chunks;
        fill(tab.t[used], i);
        chunks += need;
        ++used;
    }
    return flush();
}

}  // namespace

hipError_t launch_adamw(const recblr_adamw_tensor* tensors, int64_t count, bool bits8, IoType io,
                        const AdamWHyper& h, hipStream_t stream) {
    const size_t pe = 4 * io_bytes(io);
    const Hyper32 f{(float)h.beta1, (float)(1.0 - h.beta1), (float)h.beta2,
                    (float)(1.0 - h.beta2), (float)h.eps, (float)(h.lr * h.inv_bc1),
                    (float)h.inv_bc2};
    auto fill = [&](Entry& e, int64_t i) {
        const recblr_adamw_tensor& t = tensors[i];
        const size_t me = bits8 ? 4 : 16;
        e = Entry{t.param, t.grad, t.m1, t.m2, t.scale1, t.scale2, t.n,
                  (float)(1.0 - h.lr * t.weight_decay),
                  takes(t.param, pe) && takes(t.grad, pe) && takes(t.m1, me) && takes(t.m2, me)};
    };
    auto launch = [&](const Table& tab, unsigned grid) {
        if (!bits8 && io == IoType::kF32)
            hipLaunchKernelGGL(adamw32_kernel<float>, dim3(grid), dim3(kNT), 0, stream, tab, f);
        else if (!bits8)
            hipLaunchKernelGGL(adamw32_kernel<bf16>, dim3(grid), dim3(kNT), 0, stream, tab, f);
        else if (io == IoType::kF32)
            hipLaunchKernelGGL(adamw8_kernel<float>, dim3(grid), dim3(kNT), 0, stream, tab, h,
                               f.lr_bc1, f.inv_bc2, f.eps);
        else
            hipLaunchKernelGGL(adamw8_kernel<bf16>, dim3(grid), dim3(kNT), 0, stream, tab, h,
                               f.lr_bc1, f.inv_bc2, f.eps);
    };
    return in_tables(count, tensors, fill, launch);
}

hipError_t launch_adamw_moments(const recblr_adamw_tensor* tensors, int64_t count,
                                float* const* m1_out, float* const* m2_out, hipStream_t stream) {
    auto fill = [&](Entry& e, int64_t i) {
        const recblr_adamw_tensor& t = tensors[i];
        float *a = m1_out ? m1_out[i] : nullptr, *b = m2_out ? m2_out[i] : nullptr;
        e = Entry{a, b, t.m1, t.m2, t.scale1, t.scale2, t.n, 1.0f,
                  takes(a, 16) && takes(b, 16) && takes(t.m1, 4) && takes(t.m2, 4)};
    };
    auto launch = [&](const Table& tab, unsigned grid) {
        hipLaunchKernelGGL(adamw_moments_kernel, dim3(grid), dim3(kNT), 0, stream, tab);
    };
    return in_tables(count, tensors, fill, launch);
}

}  // namespace recblr
