// Clipped policy loss with a KL term over rows of logits, and its gradient
// (recblr_policy_loss).
//
// Of a row, with x = (l - max l) / T, S = sum e^x and the chosen item a:
//   logp = x_a - log S;  the row's loss is a function of logp alone, c its derivative;
//   dlogits = (c / T) (onehot(a) - e^x / S).
// So a row needs its maximum and sum before its first output, and every logit again for
// that output: 2 e bytes a logit where the row stays on chip in between.
//
// Rows are read as 16-byte vectors that lie at multiples of 16 bytes (up to seven elements before
// and behind them are one element more of a thread each).  Those of up to 128 KB stay in the
// registers of a wave or a workgroup and are read once; of a longer one a workgroup keeps 128 KB,
// and reads the rest twice, the second time from the last-level cache.  Few long rows are cut into
// pieces: one launch leaves each piece's maximum and sum, a second joins them.
//
// One MI355X: 4096 x 131072 bf16 405 us, 5.3 TB/s of the logits and their gradient, where a large
// copy reaches 4.7 to 6.2; the powers, two a logit, are 200 us of vector issue beside it.  2048 x
// 3416 fp32: 13 us of kernel, 16 of the call from Python.  Rows of which the chip holds more than
// the last-level cache at once come from memory twice: 200 x 1,000,000 bf16 203 us, 3.9 TB/s.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "device_common.hpp"
#include "lanes.hpp"
#include "ops.hpp"
#include "wave_tile.hpp"

namespace recblr {
namespace {

using wtile::u4v;

struct Params {
    const void* logits;
    const int32_t* ids;
    const float* old_logp;
    const float* advantage;
    const float* ref_logp;
    const float* weight;
    float* logp;
    void* dlogits;
    float* row_loss;
    int64_t N, V;
    float k, k_lo;         // log2(e) / T in two parts
    double T, lo, hi, kl;  // temperature; borders of the ratio; the KL term's weight
};

// ------------------------------------------------------------------ a row's loss
struct RowLoss {
    float lp, loss, c;  // c: d loss / d logp, over T
};

// a b as a float: never part of an fma with what is done to it, since others take it as it is.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// Powers of a row: e^((l - M) / T) = 2^(l K - mk), K = log2(e) / T as two floats, k and the
// positive rest k_lo (which keeps -inf what it is): rounded to one, K would move log S by the mean
// of (l - M) / T times 2^-25, and ratios with it.  mk is M k rounded; what that leaves is common to
// all powers of the row, and `shift` gives it back to log S.  Where M k is so large that it would
// be more than 2^-5, the difference is formed first.
struct Powers {
    float M, k, k_lo, mk;
    bool far;
    double shift;
    __device__ __forceinline__ Powers(float M_, float k_, float k_lo_)
        : M(M_), k(k_), k_lo(k_lo_), mk(rounded_product(M_, k_)) {
        far = !(fabsf(mk) < 0x1p20f);
        shift = far ? 0.0
                    : ((double)M * ((double)k + (double)k_lo) - (double)mk) * 0.6931471805599453094;
    }
    __device__ __forceinline__ static float to(float l, float k, float k_lo, float mk) {
        return fast_exp2(fmaf(l, k_lo, fmaf(l, k, -mk)));
    }
    template <bool kFar>
    __device__ __forceinline__ float of(float l) const {
        return kFar ? to(l - M, k, k_lo, 0.0f) : to(l, k, k_lo, mk);
    }
    // f, told which of the two it is.
    template <typename F>
    __device__ __forceinline__ void use(F f) const {
        far ? f(std::true_type{}) : f(std::false_type{});
    }
};

// xa: the chosen item's logit; S: the sum of powers, infinite only by a logit of +inf.  In 64 bits:
// the ratio is the power of a difference of two numbers of ten or so, whose roundings to fp32 were
// most of the loss's error.  A NaN passes every comparison on to a product with it.
__device__ __forceinline__ RowLoss row_loss(const Params& p, int64_t row, float xa,
                                            const Powers& w2, float S) {
    const double sum = S < __builtin_inff() ? (double)S : __builtin_nan("");
    const double lp = ((double)xa - (double)w2.M) / p.T - (log(sum) - w2.shift);
    const double A = p.advantage[row], w = p.weight ? p.weight[row] : 1.0f;
    const double r = exp(lp - (double)p.old_logp[row]);
    const bool gain = A >= 0.0;
    const bool inside = gain ? !(r > p.hi) : !(r < p.lo);
    const double surrogate = inside ? r * A : (gain ? p.hi : p.lo) * A;
    double loss = -surrogate, c = inside ? -surrogate : 0.0;
    if (p.kl > 0.0) {
        const double d = (double)p.ref_logp[row] - lp, up = expm1(d);
        // Both are of d's size, so what is left of d^2 keeps its digits; e^d may be infinite.
        loss += p.kl * (up < __builtin_inf() ? up - d : up);
        c -= p.kl * up;
    }
    return RowLoss{(float)lp, (float)(w * loss), (float)(w * c / p.T)};
}

__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7FC00000u); }

// ------------------------------------------------------------------ pieces of a row
// Elements [0, n) from `base` on: whole vectors at multiples of 16 bytes, `head` elements
// before them and `tail` behind them.  Without VEC a vector is one element.
template <typename T, bool VEC>
struct Span {
    static constexpr int U = VEC ? 16 / (int)sizeof(T) : 1;
    int head, vecs, tail;
    __device__ __forceinline__ Span(const T* base, int64_t n) {
        if constexpr (VEC) {
            const int mis = (int)((uintptr_t)base & 15u);
            head = mis ? (16 - mis) / (int)sizeof(T) : 0;
            if (head > n) head = (int)n;
            vecs = (int)((n - head) / U);
            tail = (int)(n - head - (int64_t)vecs * U);
        } else {
            head = tail = 0;
            vecs = (int)n;
        }
    }
    // The element that thread t has beside its vectors; -1 for none.
    __device__ __forceinline__ int extra(int t) const {
        if constexpr (!VEC) return -1;
        return t < head ? t : t >= 8 && t < 8 + tail ? head + vecs * U + t - 8 : -1;
    }
};

template <typename T, bool VEC>
struct Raw {
    static constexpr int U = Span<T, VEC>::U;
    u4v v;  // without VEC, the element's float in v[0]
    __device__ __forceinline__ void read(const T* body, int i) {
        if constexpr (VEC)
            v = __builtin_nontemporal_load((const u4v*)body + i);
        else
            v[0] = __float_as_uint(to_f32(body[i]));
    }
    __device__ __forceinline__ void none() {  // -inf in every place
        const uint32_t w = VEC && sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
        v = u4v{w, w, w, w};
    }
    __device__ __forceinline__ void keep(const T* body, int i) {
        if constexpr (VEC) v = *((const u4v*)body + i);
        else v[0] = __float_as_uint(to_f32(body[i]));
    }
    // What is done with the row next starts from its words again: left alone, the compiler keeps all
    // of its values as floats from one use to the next, twice the registers.
    __device__ __forceinline__ void packed() {
        if constexpr (VEC && sizeof(T) == 2) asm volatile("" : "+v"(v));
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (!VEC || sizeof(T) == 4) return __uint_as_float(v[e]);
        return e & 1 ? bf16_hi(v[e >> 1]) : bf16_lo(v[e >> 1]);
    }
    __device__ __forceinline__ static void write(T* body, int i, const float (&x)[U]) {
        if constexpr (!VEC) {
            body[i] = from_f32<T>(x[0]);
        } else {
            u4v w;
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(x[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = bf16_pair(x[2 * e], x[2 * e + 1]);
            }
            __builtin_nontemporal_store(w, (u4v*)body + i);
        }
    }
};

// The sum of f(0) .. f(N - 1), N a power of two, by halves: added to a growing sum one by one, small
// powers would be rounded off more often than up, and ratios lie a little too high.
template <int N, typename F>
__device__ __forceinline__ float sum_by_halves(F f, int from = 0) {
    if constexpr (N == 1) return f(from);
    else return sum_by_halves<N / 2>(f, from) + sum_by_halves<N / 2>(f, from + N / 2);
}

// Over the TH threads that share a row; every one of them gets the result.
template <int TH, typename Op>
__device__ __forceinline__ float over_row(float v, float none, float* red, Op op) {
    v = lanes::lane_of(lanes::wave_scan(v, none, op), kWave - 1);
    if constexpr (TH == kWave) return v;
    const int w = wave_id(), lane = threadIdx.x & 63;
    if (lane == 0) red[w] = v;
    __syncthreads();
    v = lane < TH / kWave ? red[lane] : none;
    v = lanes::lane_of(lanes::wave_scan(v, none, op), kWave - 1);
    __syncthreads();
    return v;
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float added(float a, float b) { return a + b; }

// row_loss for the TH threads of a row, by its first wave (16384 rows of 5,000 bf16 64 us; with its
// 64-bit arithmetic in all of them 76).
template <int TH>
__device__ __forceinline__ RowLoss row_loss_of(const Params& p, int64_t row, float xa,
                                               const Powers& pw, float S, float* red) {
    if constexpr (TH == kWave) return row_loss(p, row, xa, pw, S);
    if (wave_id() == 0) {
        const RowLoss r = row_loss(p, row, xa, pw, S);
        if ((threadIdx.x & 63) == 0) red[0] = r.lp, red[1] = r.loss, red[2] = r.c;
    }
    __syncthreads();
    return RowLoss{red[0], red[1], red[2]};
}

// The gradient of elements whose e^x are given: -(c / S) e^x, c more at the chosen one.
template <int U>
__device__ __forceinline__ void gradient(float (&g)[U], float minus, float c, int64_t at) {
#pragma unroll
    for (int e = 0; e < U; ++e) g[e] *= minus;
    if ((uint64_t)at < (uint64_t)U) {
#pragma unroll
        for (int e = 0; e < U; ++e)
            if (e == (int)at) g[e] += c;
    }
}

// ------------------------------------------------------------------ a row in registers
// TH threads a row, NV vectors a thread; TH = 64 puts four rows into a workgroup.
template <typename T, int TH, int NV, bool VEC>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void row_kernel(Params p) {
    constexpr int U = Span<T, VEC>::U, kRows = TH == kWave ? 4 : 1;
    __shared__ float red[16];
    const int t = TH == kWave ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    const int64_t row = (int64_t)blockIdx.x * kRows + (kRows > 1 ? wave_id() : 0);
    if (row >= p.N) return;  // whole waves, and only where a row is one wave's
    const T* base = (const T*)p.logits + row * p.V;
    T* out = p.dlogits ? (T*)p.dlogits + row * p.V : nullptr;
    const Span<T, VEC> sp(base, p.V);
    const int id = p.ids[row], extra = sp.extra(t);
    const T* body = base + sp.head;
    if (id < 0) {
        if (t == 0) {
            p.row_loss[row] = 0.0f;
            if (p.logp) p.logp[row] = 0.0f;
        }
        if (out) {
            const float zeros[U] = {};
            for (int i = t; i < sp.vecs; i += TH) Raw<T, VEC>::write(out + sp.head, i, zeros);
            if (extra >= 0) out[extra] = from_f32<T>(0.0f);
        }
        return;
    }
    const float xa = id < p.V ? to_f32(base[id]) : quiet_nan();
    Raw<T, VEC> x[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        x[j].none();
        if (t + j * TH < sp.vecs) x[j].read(body, t + j * TH);
    }
    float xe = -__builtin_inff(), m = xe;
    if (VEC && extra >= 0) xe = to_f32(base[extra]);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < U; ++e) m = fmaxf(m, x[j].get(e));
    const float M = over_row<TH>(fmaxf(m, xe), -__builtin_inff(), red, larger);
#pragma unroll
    for (int j = 0; j < NV; ++j) x[j].packed();
    const Powers pw(M, p.k, p.k_lo);
    pw.use([&](auto far) {
        constexpr bool kFar = decltype(far)::value;
        const float ee = pw.of<kFar>(xe);
        const float s = ee + sum_by_halves<NV * U>([&](int i) {
            const float v = pw.of<kFar>(x[i / U].get(i % U));
            if constexpr (!VEC || sizeof(T) == 4) x[i / U].v[i % U] = __float_as_uint(v);
            return v;
        });
        const float S = over_row<TH>(s, 0.0f, red, added);
#pragma unroll
        for (int j = 0; j < NV; ++j) x[j].packed();
        const RowLoss r = row_loss_of<TH>(p, row, xa, pw, S, red);
        if (t == 0) {
            p.row_loss[row] = r.loss;
            if (p.logp) p.logp[row] = r.lp;
        }
        if (!out) return;
        const float minus = -r.c / S;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * TH;
            if (i < sp.vecs) {
                float g[U];
#pragma unroll
                for (int e = 0; e < U; ++e)
                    g[e] = !VEC || sizeof(T) == 4 ? __uint_as_float(x[j].v[e])
                                                  : pw.of<kFar>(x[j].get(e));
                gradient<U>(g, minus, r.c, (int64_t)id - sp.head - (int64_t)i * U);
                Raw<T, VEC>::write(out + sp.head, i, g);
            }
        }
        if (extra >= 0) out[extra] = from_f32<T>(ee * minus + (extra == id ? r.c : 0.0f));
    });
}

// ------------------------------------------------------------------ a row against a running maximum
// A thread's running reference and the sum of powers relative to it, over vectors t, t + TH, ... of
// `vecs`; the reference starts at `low`, where nothing that counts can lie beside a row's maximum
// above it.  B vectors at a time, the first KEPT left in `kept`.
template <int TH, int KEPT, typename T, bool VEC>
__device__ __forceinline__ void running_sum(const T* body, int vecs, int t, float k, float k_lo,
                                            Raw<T, VEC> (&kept)[KEPT], float& m, float& mk,
                                            float& s) {
    constexpr int U = Span<T, VEC>::U, B = 4;
    auto read = [&](Raw<T, VEC>* x, int i) {
#pragma unroll
        for (int j = 0; j < B; ++j) {
            x[j].none();
            if (i + j * TH < vecs) x[j].keep(body, i + j * TH);
        }
    };
    auto add = [&](const Raw<T, VEC>* x) {
        float top = m;
#pragma unroll
        for (int j = 0; j < B; ++j)
#pragma unroll
            for (int e = 0; e < U; ++e) top = fmaxf(top, x[j].get(e));
        const float now = rounded_product(top, k);
        s *= fast_exp2(mk - now);
        m = top;
        mk = now;
        s += sum_by_halves<B * U>([&](int i) { return Powers::to(x[i / U].get(i % U), k, k_lo, mk); });
    };
#pragma unroll
    for (int c = 0; c < KEPT; c += B) read(kept + c, t + c * TH);
#pragma unroll
    for (int c = 0; c < KEPT; c += B) {
        add(kept + c);
#pragma unroll
        for (int j = 0; j < B; ++j) kept[c + j].packed();
    }
    for (int i = t + KEPT * TH; i < vecs; i += B * TH) {
        Raw<T, VEC> x[B];
        read(x, i);
        add(x);
    }
}
// The row's powers and, in S, their sum; xe: one element of the thread's beside its vectors.
template <int TH, int KEPT, typename T, bool VEC>
__device__ __forceinline__ Powers sum_of(const T* body, int vecs, int t, float xe, float k,
                                         float k_lo, Raw<T, VEC> (&kept)[KEPT], float* red,
                                         float& S) {
    constexpr int U = Span<T, VEC>::U;
    const float none = -__builtin_inff(), low = -0x1p19f / k;
    float m = fmaxf(low, xe), mk = rounded_product(m, k), s = Powers::to(xe, k, k_lo, mk);
    running_sum<TH, KEPT, T, VEC>(body, vecs, t, k, k_lo, kept, m, mk, s);
    float M = over_row<TH>(m, none, red, larger);
    Powers pw(M, k, k_lo);
    s *= fast_exp2(mk - pw.mk);
    if (M <= low || pw.far) {  // once more, with the maximum first
        m = xe;
        for (int i = t; i < vecs; i += TH) {
            Raw<T, VEC> x;
            x.keep(body, i);
#pragma unroll
            for (int e = 0; e < U; ++e) m = fmaxf(m, x.get(e));
        }
        M = over_row<TH>(m, none, red, larger);
        pw = Powers(M, k, k_lo);
        pw.far = true;
        pw.shift = 0.0;
        s = pw.of<true>(xe);
        for (int i = t; i < vecs; i += TH) {
            Raw<T, VEC> x;
            x.keep(body, i);
            s += sum_by_halves<U>([&](int e) { return pw.of<true>(x.get(e)); });
        }
    }
    S = over_row<TH>(s, 0.0f, red, added);
    return pw;
}

template <typename T, int TH, int KEPT, bool VEC>
__global__ __launch_bounds__(TH) void running_kernel(Params p) {
    constexpr int U = Span<T, VEC>::U, B = 4;  // vectors on their way
    __shared__ float red[16];
    const int64_t row = blockIdx.x;
    const int id = p.ids[row], t = threadIdx.x;
    const T* base = (const T*)p.logits + row * p.V;
    T* out = p.dlogits ? (T*)p.dlogits + row * p.V : nullptr;
    const Span<T, VEC> sp(base, p.V);
    const T* body = base + sp.head;
    const int extra = sp.extra(t);
    if (id < 0) {
        if (t == 0) {
            p.row_loss[row] = 0.0f;
            if (p.logp) p.logp[row] = 0.0f;
        }
        if (out) {
            const float zeros[U] = {};
            for (int i = t; i < sp.vecs; i += TH) Raw<T, VEC>::write(out + sp.head, i, zeros);
            if (extra >= 0) out[extra] = from_f32<T>(0.0f);
        }
        return;
    }
    const float xa = id < p.V ? to_f32(base[id]) : quiet_nan();
    const float xe = VEC && extra >= 0 ? to_f32(base[extra]) : -__builtin_inff();
    float S;
    Raw<T, VEC> kept[KEPT];
    const Powers pw = sum_of<TH, KEPT, T, VEC>(body, sp.vecs, t, xe, p.k, p.k_lo, kept, red, S);
    const RowLoss r = row_loss_of<TH>(p, row, xa, pw, S, red);
    if (t == 0) {
        p.row_loss[row] = r.loss;
        if (p.logp) p.logp[row] = r.lp;
    }
    if (!out) return;
    const float minus = -r.c / S;
    pw.use([&](auto far) {
        constexpr bool kFar = decltype(far)::value;
        auto put = [&](const Raw<T, VEC>& x, int i) {
            float g[U];
#pragma unroll
            for (int e = 0; e < U; ++e) g[e] = pw.of<kFar>(x.get(e));
            gradient<U>(g, minus, r.c, (int64_t)id - sp.head - (int64_t)i * U);
            Raw<T, VEC>::write(out + sp.head, i, g);
        };
#pragma unroll
        for (int c = 0; c < KEPT; ++c)
            if (t + c * TH < sp.vecs) put(kept[c], t + c * TH);
        for (int i0 = t + KEPT * TH; i0 < sp.vecs; i0 += B * TH) {
            Raw<T, VEC> x[B];
#pragma unroll
            for (int j = 0; j < B; ++j)
                if (i0 + j * TH < sp.vecs) x[j].read(body, i0 + j * TH);
#pragma unroll
            for (int j = 0; j < B; ++j)
                if (i0 + j * TH < sp.vecs) put(x[j], i0 + j * TH);
        }
        if (VEC && extra >= 0)
            out[extra] = from_f32<T>(pw.of<kFar>(xe) * minus + (extra == id ? r.c : 0.0f));
    });
}

// ------------------------------------------------------------------ rows in pieces
struct Part {
    float m, s;
};
constexpr int kPieceThreads = 256;

template <typename T, bool VEC>
__global__ __launch_bounds__(kPieceThreads) void part_kernel(Params p, Part* parts, float* chosen,
                                                             int64_t piece, int pieces) {
    constexpr int U = Span<T, VEC>::U, TH = kPieceThreads, B = 4;
    __shared__ float red[16];
    const int64_t row = blockIdx.x / (unsigned)pieces;
    const int64_t from = (int64_t)(blockIdx.x % (unsigned)pieces) * piece;
    const int64_t n = min(piece, p.V - from);
    const int id = p.ids[row], t = threadIdx.x;
    if (id < 0) return;
    const T* base = (const T*)p.logits + row * p.V + from;
    const Span<T, VEC> sp(base, n);
    const T* body = base + sp.head;
    const int extra = sp.extra(t);
    const float none = -__builtin_inff();
    const float xe = VEC && extra >= 0 ? to_f32(base[extra]) : none;
    // The maximum so far and the sum of powers relative to it, B vectors at a time.
    float m = xe, s = xe > none ? 1.0f : xe == none ? 0.0f : xe;  // a NaN stays one
    for (int i = t; i < sp.vecs; i += B * TH) {
        Raw<T, VEC> x[B];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            x[j].none();
            if (i + j * TH < sp.vecs) x[j].read(body, i + j * TH);
        }
        float top = m;
#pragma unroll
        for (int j = 0; j < B; ++j)
#pragma unroll
            for (int e = 0; e < U; ++e) top = fmaxf(top, x[j].get(e));
        const float ref = top == none ? 0.0f : top;  // nothing but -inf so far: powers of 0
        s *= Powers::to(m - ref, p.k, p.k_lo, 0.0f);
        s += sum_by_halves<B * U>(
            [&](int i) { return Powers::to(x[i / U].get(i % U) - ref, p.k, p.k_lo, 0.0f); });
        m = top;
    }
    const float M = over_row<TH>(m, none, red, larger);
    s *= Powers::to(m - (M == none ? 0.0f : M), p.k, p.k_lo, 0.0f);
    const float S = over_row<TH>(s, 0.0f, red, added);
    if (t == 0) {
        parts[blockIdx.x] = Part{M, S};
        if (id >= from && id < from + n) chosen[row] = to_f32(base[id - from]);
    }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(kPieceThreads) void joined_kernel(Params p, const Part* parts,
                                                               const float* chosen, int64_t piece,
                                                               int pieces) {
    constexpr int U = Span<T, VEC>::U, TH = kPieceThreads;
    __shared__ float red[16];
    const int64_t row = blockIdx.x / (unsigned)pieces;
    const int at = (int)(blockIdx.x % (unsigned)pieces);
    const int64_t from = at * piece, n = min(piece, p.V - from);
    const int id = p.ids[row], t = threadIdx.x;
    const T* base = (const T*)p.logits + row * p.V + from;
    T* out = p.dlogits ? (T*)p.dlogits + row * p.V + from : nullptr;
    const Span<T, VEC> sp(base, n);
    const T* body = base + sp.head;
    const int extra = sp.extra(t);
    if (id < 0) {
        if (t == 0 && at == 0) {
            p.row_loss[row] = 0.0f;
            if (p.logp) p.logp[row] = 0.0f;
        }
        if (out) {
            const float zeros[U] = {};
            for (int i = t; i < sp.vecs; i += TH) Raw<T, VEC>::write(out + sp.head, i, zeros);
            if (extra >= 0) out[extra] = from_f32<T>(0.0f);
        }
        return;
    }
    parts += row * pieces;
    const float none = -__builtin_inff();
    float m = none;
    for (int i = t; i < pieces; i += TH) m = fmaxf(m, parts[i].m);
    const float M = over_row<TH>(m, none, red, larger);
    float s = 0.0f;
    for (int i = t; i < pieces; i += TH) {
        const Part q = parts[i];
        if (q.s != 0.0f || M == none) s += q.s * Powers::to(q.m - M, p.k, p.k_lo, 0.0f);
    }
    const float S = over_row<TH>(s, 0.0f, red, added);
    // The pieces' sums are relative to their maxima as they are: nothing to give back to log S.
    Powers pw(M, p.k, p.k_lo);
    const double shift = pw.shift;
    pw.shift = 0.0;
    const RowLoss r =
        row_loss_of<TH>(p, row, id < p.V ? chosen[row] : quiet_nan(), pw, S, red);
    if (t == 0 && at == 0) {
        p.row_loss[row] = r.loss;
        if (p.logp) p.logp[row] = r.lp;
    }
    if (!out) return;
    const float minus = -r.c / S * (float)exp(-shift);
    const int64_t pick = (int64_t)id - from;
    pw.use([&](auto far) {
        constexpr bool kFar = decltype(far)::value;
#pragma unroll 4
        for (int i = t; i < sp.vecs; i += TH) {
            Raw<T, VEC> x;
            x.read(body, i);
            float g[U];
#pragma unroll
            for (int e = 0; e < U; ++e) g[e] = pw.of<kFar>(x.get(e));
            gradient<U>(g, minus, r.c, pick - sp.head - (int64_t)i * U);
            Raw<T, VEC>::write(out + sp.head, i, g);
        }
        if (VEC && extra >= 0)
            out[extra] = from_f32<T>(pw.of<kFar>(to_f32(base[extra])) * minus +
                                     (extra == pick ? r.c : 0.0f));
    });
}

// ------------------------------------------------------------------ sum of the rows
constexpr int kSumThreads = 1024;
constexpr int64_t kSumRows = 16 * kSumThreads;  // rows to a workgroup

// Sums of kSumRows values each, in order of threads; the last launch has one workgroup.
template <typename In>
__global__ __launch_bounds__(kSumThreads) void sum_kernel(const In* v, int64_t n, double* part,
                                                          float* loss) {
    __shared__ double red[kSumThreads / kWave];
    const int64_t from = (int64_t)blockIdx.x * kSumRows;
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < kSumRows / kSumThreads; ++j) {
        const int64_t i = from + j * kSumThreads + threadIdx.x;
        if (i < n) s += (double)v[i];
    }
    s = lanes::wave_sum(s);
    if ((threadIdx.x & 63) == 0) red[wave_id()] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int i = 0; i < kSumThreads / kWave; ++i) s += red[i];
        if (loss)
            *loss = (float)s;
        else
            part[blockIdx.x] = s;
    }
}

// ------------------------------------------------------------------ which way
struct Way {
    int threads, vecs;  // to a row; vectors that a thread keeps
    int64_t piece;      // > 0: elements to a piece of a row instead
};

// Up to 512 vectors of 16 bytes lie in the registers of a wave or of 256 threads and their maximum
// comes before their powers.  Longer rows are summed against a running maximum, the first vectors
// of each thread kept and what is behind them read again, from the last-level cache: 8192 rows of
// 16 KB 48 us (in registers, maximum first, 55), of 32 KB 88 (nothing kept 107), 4096 of 128 KB
// 190 (204), of 256 KB 405 (450; with 512 threads that keep 16, 412, in registers as a whole
// 420).  Few long rows are cut into pieces: 16 x 131072 bf16 22 us.
Way way_of(int64_t N, int64_t V, IoType io, bool vec) {
    const int64_t U = vec ? 16 / (int64_t)io_bytes(io) : 1, n = (V + U - 1) / U;  // vectors
    if (n <= 64 * 4) return {64, n <= 64 ? 1 : n <= 128 ? 2 : 4, 0};
    if (n <= 256 * 4) return {256, n <= 512 ? 2 : 4, 0};
    if (n <= 512 * 24) return {512, n <= 512 * 4 ? 4 : n <= 512 * 8 ? 8 : 16, 0};
    if (N >= 128 || n <= 16384) return {1024, 8, 0};
    // Pieces: about four workgroups to a compute unit, of 2,048 elements or more.
    const int64_t want = (1024 + N - 1) / N;
    int64_t piece = (V + want - 1) / want;
    piece = (piece + 2047) / 2048 * 2048;
    return {0, 0, piece < 65536 ? piece : 65536};
}

// The piece way may be taken with or without vectors: room for the smaller pieces.
int64_t max_pieces(int64_t N, int64_t V, IoType io) {
    int64_t most = 0;
    for (bool vec : {false, true}) {
        const Way w = way_of(N, V, io, vec);
        if (w.piece > 0) most = std::max(most, (V + w.piece - 1) / w.piece);
    }
    return most;
}

struct Layout {
    size_t rows, sums, parts, chosen, bytes;
};
Layout layout(int64_t N, int64_t V, IoType io) {
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    Layout l;
    const int64_t pieces = max_pieces(N, V, io);
    l.rows = 0;
    l.sums = up((size_t)N * 4);
    l.parts = l.sums + up((size_t)((N + kSumRows - 1) / kSumRows) * 8);
    l.chosen = l.parts + up((size_t)(N * pieces) * sizeof(Part));
    l.bytes = l.chosen + (pieces ? up((size_t)N * 4) : 0);
    return l;
}

template <typename T, bool VEC>
void launch_rows(const Params& p, const Way& w, const Layout& l, char* ws, hipStream_t st) {
    if (w.piece > 0) {
        const int pieces = (int)((p.V + w.piece - 1) / w.piece);
        const dim3 grid((unsigned)(p.N * pieces));
        Part* parts = (Part*)(ws + l.parts);
        float* chosen = (float*)(ws + l.chosen);
        part_kernel<T, VEC><<<grid, kPieceThreads, 0, st>>>(p, parts, chosen, w.piece, pieces);
        joined_kernel<T, VEC><<<grid, kPieceThreads, 0, st>>>(p, parts, chosen, w.piece, pieces);
        return;
    }
    const dim3 rows((unsigned)p.N), quads((unsigned)((p.N + 3) / 4));
    if (w.threads == 64) {
        if (w.vecs == 1) row_kernel<T, 64, 1, VEC><<<quads, 256, 0, st>>>(p);
        else if (w.vecs == 2) row_kernel<T, 64, 2, VEC><<<quads, 256, 0, st>>>(p);
        else row_kernel<T, 64, 4, VEC><<<quads, 256, 0, st>>>(p);
    } else if (w.threads == 256) {
        if (w.vecs == 2) row_kernel<T, 256, 2, VEC><<<rows, 256, 0, st>>>(p);
        else running_kernel<T, 256, 4, VEC><<<rows, 256, 0, st>>>(p);
    } else if (w.threads == 512) {
        if (w.vecs == 4) running_kernel<T, 512, 4, VEC><<<rows, 512, 0, st>>>(p);
        else if (w.vecs == 8) running_kernel<T, 512, 8, VEC><<<rows, 512, 0, st>>>(p);
        else running_kernel<T, 512, 16, VEC><<<rows, 512, 0, st>>>(p);
    } else {
        running_kernel<T, 1024, 8, VEC><<<rows, 1024, 0, st>>>(p);
    }
}

}  // namespace

size_t policy_workspace(int64_t N, int64_t V, IoType io) { return layout(N, V, io).bytes; }

hipError_t launch_policy_loss(const PolicyArgs& a, void* ws, hipStream_t st) {
    const Layout l = layout(a.N, a.V, a.io);
    char* w = (char*)ws;
    const double K = 1.4426950408889634 / a.temperature;
    float k = (float)K;
    // For a positive rest, as a float too: of temperatures near 10^30 it may lie below the least one.
    if ((float)(K - (double)k) <= 0.0f) k = std::nextafterf(k, 0.0f);
    const Params p{a.logits, a.ids, a.old_logp, a.advantage, a.ref_logp, a.weight, a.logp,
                   a.dlogits, (float*)(w + l.rows), a.N, a.V, k, (float)(K - (double)k),
                   a.temperature, 1.0 - a.clip_low, 1.0 + a.clip_high, a.kl};
    if (a.N > 0) {
        // Vectors need rows of both tensors to lie alike to 16 bytes.
        const bool vec =
            !a.dlogits || (((uintptr_t)a.logits ^ (uintptr_t)a.dlogits) & 15u) == 0;
        const Way way = way_of(a.N, a.V, a.io, vec);
        if (a.io == IoType::kF32)
            vec ? launch_rows<float, true>(p, way, l, w, st)
                : launch_rows<float, false>(p, way, l, w, st);
        else
            vec ? launch_rows<bf16, true>(p, way, l, w, st)
                : launch_rows<bf16, false>(p, way, l, w, st);
    }
    double* sums = (double*)(w + l.sums);
    const int64_t groups = (a.N + kSumRows - 1) / kSumRows;
    if (groups > 1) {
        sum_kernel<float><<<dim3((unsigned)groups), kSumThreads, 0, st>>>(p.row_loss, a.N, sums,
                                                                         nullptr);
        sum_kernel<double><<<1, kSumThreads, 0, st>>>(sums, groups, nullptr, a.loss);
    } else {
        sum_kernel<float><<<1, kSumThreads, 0, st>>>(p.row_loss, a.N, nullptr, a.loss);
    }
    return hipGetLastError();
}

}  // namespace recblr
