// Pieces shared by the chunked kernels of the gated delta rule (delta_fwd.hip,
// delta_bwd.hip): matrix-core operands from LDS, decays of a chunk, and the inverse of a
// chunk's unit triangular matrix.
//
// A workgroup of four waves works on 64 steps at a time; wave w owns the strip of rows
// 16 w .. 16 w + 15.  All products are of 16 x 16 tiles, whose accumulator gives lane l
// column l % 16 and rows 4 (l / 16) .. + 3, and whose operands give lane l row (or column)
// l % 16.  With g = l / 16, the lane's k are
//   bf16 I/O: v_mfma_f32_16x16x32_bf16, k = 8 g .. 8 g + 7 of 32 (16 bytes),
//   fp32 I/O: four v_mfma_f32_16x16x4_f32, k = 4 g .. 4 g + 3 of 16 (16 bytes; the j-th
//     instruction contracts the j-th value of every lane).
// fp32 I/O is thus multiplied in fp32.  With bf16 I/O the inputs are exact operands, and what
// is computed from them is given as a sum of bf16 planes (x = h + m + l, each the bf16 nearest
// to what the ones before leave), with the products of planes whose indexes add up to less
// than their number: three planes, hence fp32's 24 bits, on the way to a state, which is
// float and lasts (two planes show 3e-6 to 9e-6 against 64 bits there, three 3e-7), and two,
// 16 bits, where the result is rounded to bf16 at once: outputs and gradients are then off by
// 1.7e-3 against 64 bits (2-norm), all of it the last rounding's, and differ from those of 24-bit
// arithmetic by 1.3e-4, last bits that fall to the other side.  Three would take a half more to
// twice the products, and more LDS than the gradient kernel has.
#pragma once

#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "lanes.hpp"
#include "ops.hpp"
#include "wave_tile.hpp"

namespace recblr {
namespace dtile {

using wtile::b8;
using wtile::f4;
using wtile::lds_barrier;

constexpr int C = 64;     // steps of a chunk
constexpr int NT = 256;   // threads
constexpr int TS = 68;    // floats in a row of the triangular matrix in LDS
typedef __bf16 b4 __attribute__((ext_vector_type(4)));

// Keeps the compiler from starting the LDS reads of the following steps of an unrolled loop
// before this one's accumulators are formed (left alone it starts all reads at once, and spills
// what else the wave holds).  No instruction.
__device__ __forceinline__ void step_end(f4& x) { asm volatile("" : "+v"(x) : : "memory"); }

// ------------------------------------------------------------------ operands
struct F32Op {  // fp32: given and computed operands alike
    f4 v;
};
template <int P>
struct Bf16Op {  // P planes
    b8 p[P];
};

template <typename T>
struct Io;
// kChain, kOut: planes of an operand computed for a state, and for an output of type T.
template <>
struct Io<float> {
    using Elem = float;
    using Given = F32Op;
    template <int P>
    using Made = F32Op;
    static constexpr int kChain = 1, kOut = 1, kStep = 16, kPad = 4, kUnit = 4;
};
template <>
struct Io<bf16> {
    using Elem = __bf16;
    using Given = Bf16Op<1>;
    template <int P>
    using Made = Bf16Op<P>;
    static constexpr int kChain = 3, kOut = 2, kStep = 32, kPad = 8, kUnit = 8;
};  // kUnit: elements in 16 bytes

__device__ __forceinline__ f4 mma(f4 c, const F32Op& a, const F32Op& b) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}
template <int PA, int PB>
__device__ __forceinline__ f4 mma(f4 c, const Bf16Op<PA>& a, const Bf16Op<PB>& b) {
    constexpr int N = PA > PB ? PA : PB;
#pragma unroll
    for (int n = N - 1; n >= 0; --n)  // the small products first
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (n - i >= 0 && n - i < PB)
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[n - i], c, 0, 0, 0);
    return c;
}

// The first planes of an operand.
template <int P>
__device__ __forceinline__ F32Op fewer(const F32Op& a) { return a; }
template <int P, int Q>
__device__ __forceinline__ Bf16Op<P> fewer(const Bf16Op<Q>& a) {
    Bf16Op<P> o;
#pragma unroll
    for (int i = 0; i < P; ++i) o.p[i] = a.p[i];
    return o;
}

// Eight floats as planes.
template <int P>
__device__ __forceinline__ Bf16Op<P> split(const float (&x)[8]) {
    Bf16Op<P> o;
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            o.p[p][e] = (__bf16)r[e];
            r[e] -= (float)o.p[p][e];
        }
    return o;
}

// A matrix in LDS whose rows run along the contraction: operand row `row`, k from k0.
__device__ __forceinline__ F32Op given(const float* m, int stride, int row, int k0, int g) {
    return {*(const f4*)(m + row * stride + k0 + 4 * g)};
}
__device__ __forceinline__ Bf16Op<1> given(const __bf16* m, int stride, int row, int k0, int g) {
    return {{*(const b8*)(m + row * stride + k0 + 8 * g)}};
}
// The same of a computed matrix; `plane`: elements from one plane to the next.
template <int P>
__device__ __forceinline__ F32Op made(const float* m, int, int stride, int row, int k0, int g) {
    return given(m, stride, row, k0, g);
}
template <int P>
__device__ __forceinline__ Bf16Op<P> made(const __bf16* m, int plane, int stride, int row, int k0,
                                          int g) {
    Bf16Op<P> o;
#pragma unroll
    for (int i = 0; i < P; ++i)
        o.p[i] = *(const b8*)(m + i * plane + row * stride + k0 + 8 * g);
    return o;
}
// The k order that accumulators of two neighbouring tiles have: 4 g .. of the first, then of
// the second.  An operand made of accumulators is multiplied by one that is read this way.
template <int P>
__device__ __forceinline__ F32Op made_acc(const float* m, int, int stride, int row, int k0, int g) {
    return given(m, stride, row, k0, g);
}
template <int P>
__device__ __forceinline__ Bf16Op<P> made_acc(const __bf16* m, int plane, int stride, int row,
                                              int k0, int g) {
    Bf16Op<P> o;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const __bf16* p = m + i * plane + row * stride + k0 + 4 * g;
        o.p[i] = __builtin_shufflevector(*(const b4*)p, *(const b4*)(p + 16), 0, 1, 2, 3, 4, 5, 6,
                                         7);
    }
    return o;
}
// A matrix whose columns run along the contraction: operand row = column `col0 + l % 16`, k
// from row k0 on, in natural order.
__device__ __forceinline__ F32Op given_t(const float* m, int stride, int k0, int col0, int ll,
                                         int g) {
    const float* p = m + (k0 + 4 * g) * stride + col0 + ll;
    return {{p[0], p[stride], p[2 * stride], p[3 * stride]}};
}
__device__ __forceinline__ Bf16Op<1> given_t(const __bf16* m, int stride, int k0, int col0, int ll,
                                             int g) {
    const __bf16* p = m + (k0 + 8 * g + (ll >> 2)) * stride + col0 + 4 * (ll & 3);
    return {{wtile::tr_pair((const char*)p, (const char*)(p + 4 * stride))}};
}
template <int P>
__device__ __forceinline__ F32Op made_t(const float* m, int, int stride, int k0, int col0, int ll,
                                        int g) {
    return given_t(m, stride, k0, col0, ll, g);
}
template <int P>
__device__ __forceinline__ Bf16Op<P> made_t(const __bf16* m, int plane, int stride, int k0,
                                            int col0, int ll, int g) {
    Bf16Op<P> o;
#pragma unroll
    for (int i = 0; i < P; ++i) o.p[i] = given_t(m + i * plane, stride, k0, col0, ll, g).p[0];
    return o;
}
// As given_t, in the k order of accumulators.
__device__ __forceinline__ F32Op given_t_acc(const float* m, int stride, int k0, int col0, int ll,
                                             int g) {
    return given_t(m, stride, k0, col0, ll, g);
}
__device__ __forceinline__ Bf16Op<1> given_t_acc(const __bf16* m, int stride, int k0, int col0,
                                                 int ll, int g) {
    const __bf16* p = m + (k0 + 4 * g + (ll >> 2)) * stride + col0 + 4 * (ll & 3);
    return {{wtile::tr_pair((const char*)p, (const char*)(p + 16 * stride))}};
}

// Four accumulator values (consecutive k of a row of the operand that they become).
template <int P>
__device__ __forceinline__ void put(float* m, int, int stride, int row, int k0, const f4& v) {
    *(f4*)(m + row * stride + k0) = v;
}
template <int P>
__device__ __forceinline__ void put(__bf16* m, int plane, int stride, int row, int k0,
                                    const f4& v) {
    f4 r = v;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        b4 h;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[e] = (__bf16)r[e];
            r[e] -= (float)h[e];
        }
        *(b4*)(m + i * plane + row * stride + k0) = h;
    }
}

// An operand from accumulators: tile t of fp32, tiles 2 t and 2 t + 1 of bf16.
template <typename T, int P>
__device__ __forceinline__ typename Io<T>::template Made<P> from_acc(const f4* acc, int t) {
    if constexpr (sizeof(T) == 4) {
        return F32Op{acc[t]};
    } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = acc[2 * t + (e >> 2)][e & 3];
        return split<P>(x);
    }
}

// ------------------------------------------------------------------ global memory
// A chunk's rows of one head, as a buffer: row r, element e at byte (r step + e) sizeof(T).
// Accesses outside of the rows that exist read zeros and write nothing, so no branch guards
// them; elements behind a row's end (the next head's) have to be sent out of range by `off`.
constexpr uint32_t kNowhere = 0x7F000000u;  // an offset behind every buffer's end

template <typename T>
struct Rows {
    __amdgpu_buffer_rsrc_t r;
    uint32_t step;  // bytes from row to row
    // rows [t0, t0 + 64) of the `len` rows from base on, `width` elements wide; none from t0 >= len
    __device__ __forceinline__ Rows(const T* base, int64_t t0, int64_t len, int64_t row_elems,
                                    int width) {
        const int64_t left = len - t0;
        const int rows = left < C ? left < 0 ? 0 : (int)left : C;
        step = (uint32_t)(row_elems * sizeof(T));
        r = wtile::rsrc(base + t0 * row_elems,
                        rows > 0 ? (uint32_t)((rows - 1) * row_elems + width) * (uint32_t)sizeof(T)
                                 : 0u);
    }
    __device__ __forceinline__ uint32_t off(int row, int e, int width) const {
        return e < width ? (uint32_t)row * step + (uint32_t)e * (uint32_t)sizeof(T) : kNowhere;
    }
    // Element e of row `row` and of those behind it, by adding r * step (an offset out of range
    // stays there: four rows of the largest tensors are below 2^24 bytes).
    __device__ __forceinline__ uint32_t next(uint32_t o, int r) const { return o + (uint32_t)r * step; }
    // An element as it lies in memory, and its value.  What is read ahead stays raw until it is
    // used: a conversion next to the load makes the wave wait for it there.
    __device__ __forceinline__ uint32_t raw(uint32_t o) const {
        if constexpr (sizeof(T) == 4)
            return __builtin_amdgcn_raw_buffer_load_b32(r, (int)o, 0, 0);
        else
            return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, (int)o, 0, 0);
    }
    __device__ __forceinline__ static float value(uint32_t raw) {
        return __uint_as_float(sizeof(T) == 4 ? raw : raw << 16);
    }
    __device__ __forceinline__ float get(uint32_t o) const { return value(raw(o)); }
    __device__ __forceinline__ void set(uint32_t o, float v) const {
        if constexpr (sizeof(T) == 4)
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, (int)o, 0, 0);
        else
            __builtin_amdgcn_raw_buffer_store_b16((short)from_f32<bf16>(v).bits, r, (int)o, 0, 0);
    }
    // 16 bytes from element e of a row; VEC: rows start at multiples of 16 bytes.
    template <bool VEC>
    __device__ __forceinline__ wtile::u4v get16(int row, int e, int width) const {
        if constexpr (VEC) {
            return __builtin_bit_cast(wtile::u4v, __builtin_amdgcn_raw_buffer_load_b128(
                                                      r, (int)off(row, e, width), 0, 0));
        } else {
            constexpr int U = 16 / sizeof(T);
            wtile::u4v v = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const uint32_t o = off(row, e + i, width);
                if constexpr (sizeof(T) == 4)
                    v[i] = __builtin_amdgcn_raw_buffer_load_b32(r, (int)o, 0, 0);
                else
                    v[i >> 1] |= (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(
                                     r, (int)o, 0, 0)
                                 << (16 * (i & 1));
            }
            return v;
        }
    }
};

// ------------------------------------------------------------------ decays of a chunk
struct Gates {
    double cum[C];  // running sum of g log2(e)
    float eg[C];    // 2^cum_i: decay from the chunk's start through step i
    float el[C];    // 2^(cum_63 - cum_i): decay behind step i up to the chunk's end
    float bt[C];    // beta
    float es[C];    // scale eg
};

// By one wave, a step to a lane.  The sums are kept in 64 bits: what is used of them is
// differences, exact to fp32 however strong the decays before them were.  Steps behind the
// sequence have g = beta = 0.
__device__ __forceinline__ void gates_of_chunk(Gates* gt, float g, float beta, float scale,
                                               int lane) {
    const double s = lanes::wave_upto((double)delta_clamp_g(g) * 1.4426950408889634074);
    const double end = lanes::lane_of(s, C - 1);
    gt->cum[lane] = s;
    gt->eg[lane] = fast_exp2((float)s);
    gt->el[lane] = fast_exp2((float)(end - s));
    gt->bt[lane] = beta;
    gt->es[lane] = scale * gt->eg[lane];
}

// ------------------------------------------------------------------ (I + A)^-1
// A is strictly lower triangular, 64 x 64 floats in `tm` (its tiles on and below the
// diagonal).  Inverses of the diagonal 16 x 16 tiles by substitution, then of twice the size
// at a time: the tile below is -D^-1 B A^-1.  All in fp32 (powers of A, as a Neumann series
// has them, cancel badly where keys are alike).  The tiles (2..3, 0..1) of the result are
// stored at (0..1, 2..3), where zeros belong, since the ones of A are still read by other
// waves.  tile_at gives the place.

// Wave w inverts its own diagonal tile.  Lane column ll; A's rows are read by all lanes alike.
__device__ __forceinline__ void invert_diagonal(float* tm, int w, int ll, int g) {
    float* b = tm + 16 * w * TS + 16 * w;
    wtile::f16v x;  // a vector: selects among an array's elements would put it into memory
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float s = i == ll ? 1.0f : 0.0f;
#pragma unroll
        for (int m = 0; m < i; m += 4) {
            const f4 a = *(const f4*)(b + i * TS + m);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (m + e < i) s = fmaf(-a[e], x[m + e], s);
        }
        x[i] = s;
        // Taken through here, x is formed before the next rows' reads: all 30 of them in flight
        // at once would cost 120 registers.
        if (i % 4 == 3) {
            asm volatile("" : "+v"(s) : : "memory");
            x[i] = s;
        }
    }
    wave_fence();
    // Each group of 16 lanes writes four of the rows.
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float lo = g & 1 ? x[4 + r] : x[r], hi = g & 1 ? x[12 + r] : x[8 + r];
        b[(4 * g + r) * TS + ll] = g & 2 ? hi : lo;
    }
}

// Tile product with B as it lies in memory ([k][column]).
__device__ __forceinline__ f4 tile_mma(f4 c, const float* a, const float* b, int ll, int g) {
    return mma(c, given(a, TS, ll, 0, g), given_t(b, TS, 0, 0, ll, g));
}
__device__ __forceinline__ void tile_put(float* t, const f4& v, int ll, int g) {
#pragma unroll
    for (int r = 0; r < 4; ++r) t[(4 * g + r) * TS + ll] = v[r];
}
__device__ __forceinline__ float* tile(float* tm, int i, int j) { return tm + 16 * i * TS + 16 * j; }

// Waves 0 and 2: the tile (w + 1, w).
__device__ __forceinline__ void invert_merge1(float* tm, int w, int ll, int g) {
    if (w & 1) return;
    const f4 zero = {0, 0, 0, 0};
    const f4 y = tile_mma(zero, tile(tm, w + 1, w), tile(tm, w, w), ll, g);
    f4 t = mma(zero, given(tile(tm, w + 1, w + 1), TS, ll, 0, g), F32Op{y});
    t = -t;
    wave_fence();
    tile_put(tile(tm, w + 1, w), t, ll, g);
}
// Wave w: the tile (2 + w / 2, w % 2).
__device__ __forceinline__ void invert_merge2(float* tm, int w, int ll, int g) {
    const int rb = 2 + (w >> 1), cb = w & 1;
    const f4 zero = {0, 0, 0, 0};
    f4 t = zero;
    for (int k = 2; k <= rb; ++k) {
        f4 y = zero;
        for (int m = cb; m < 2; ++m) y = tile_mma(y, tile(tm, k, m), tile(tm, m, cb), ll, g);
        t = mma(t, given(tile(tm, rb, k), TS, ll, 0, g), F32Op{y});
    }
    t = -t;
    tile_put(tile(tm, cb, rb), t, ll, g);
}
// Where tile (i, j) of the inverse lies.
__device__ __forceinline__ const float* tile_at(const float* tm, int i, int j) {
    return i >= 2 && j < 2 ? tm + 16 * j * TS + 16 * i : tm + 16 * i * TS + 16 * j;
}

// Operand of the inverse's rows 16 i .. (k: columns, step s), and of its transpose.
template <typename T, int P>
__device__ __forceinline__ typename Io<T>::template Made<P> inverse_rows(const float* tm, int i,
                                                                        int s, int ll, int g) {
    if constexpr (sizeof(T) == 4) {
        return given(tile_at(tm, i, s), TS, ll, 0, g);
    } else {
        const float* p = tile_at(tm, i, 2 * s + (g >> 1)) + ll * TS + 8 * (g & 1);
        const f4 a = *(const f4*)p, b = *(const f4*)(p + 4);
        const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        return split<P>(x);
    }
}
template <typename T, int P>
__device__ __forceinline__ typename Io<T>::template Made<P> inverse_cols(const float* tm, int i,
                                                                        int s, int ll, int g) {
    if constexpr (sizeof(T) == 4) {
        return given_t(tile_at(tm, s, i), TS, 0, 0, ll, g);
    } else {
        const float* p = tile_at(tm, 2 * s + (g >> 1), i) + 8 * (g & 1) * TS + ll;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p[e * TS];
        return split<P>(x);
    }
}

}  // namespace dtile
}  // namespace recblr
