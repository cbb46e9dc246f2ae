// Muon: momentum whose update is brought near the closest orthogonal matrix by Newton-Schulz
// products, over a list of matrices (recblr_muon_update).
//
// With X the update over its norm, m x n, m <= n (transposed where it has more rows):
//   A = X X^T,   B = b A + c A^2,   X <- a X + B X,    five times as a rule.
// All is matrix products: 2 m^2 n + 2 m^3 + 2 m^2 n operations a step, of which the first two
// are of symmetric matrices, so half of their tiles do.
//
// Numbers in 22 bits.  What small singular values get by a product's rounding is not small
// next to them: the steps blow it up with them, by up to a^5 = 485.  One bf16 or fp16 operand
// would leave errors of 10% and more; fp32 matrix instructions run at a sixteenth of fp16's
// rate.  Here each operand is a sum of two fp16 numbers, hi = fp16(v) and lo = fp16(v - hi),
// and a product hi hi + hi lo + lo hi, summed in fp32: three fp16 products for fp32's one.
// Singular values stay below 1.21 (the norm is at most 1 at first, and the polynomial a s +
// b s^3 + c s^5 keeps [0, 1.21] in itself), so entries of X, A and B stay below 1.21, 1.46 and
// 3, and are held times 2^12: far from fp16's largest, and what falls below its smallest is
// 2^-36 of the norm.
//
// Small matrices (both sides' tiles and the planes fit a compute unit's LDS, e.g. 128 x 128 or
// 64 x 256): one workgroup does all of it, X in registers as fp32 beside the planes in LDS.
// Larger ones: planes in the workspace, a launch a product over all matrices of the list.
//
// One MI355X, five steps: 14 matrices of up to 128 x 128 in 44 us, 36 of them the largest one's
// products and barriers on its compute unit.  14 of up to 512 x 512 in 218, 17 launches; 200 x 200
// alone takes 108, 6.4 a launch with next to no work.  Two 2048 x 2048, an 8192 x 2048 and a
// 999 x 1501 in 3,050 to 3,130: products at 0.83 to 0.91 PFLOP/s (8192 x 8192 of a library 1.09),
// 150 for momentum, norm and planes, by memory at 5 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.hpp"
#include "lanes.hpp"
#include "ops.hpp"
#include "wave_tile.hpp"

namespace recblr {
namespace {

using wtile::f16v;
using wtile::f4;
using wtile::u4v;
using wtile::u2v;
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kUp = 4096.0f, kDown = 1.0f / 4096.0f;

struct Hyper {
    float mu, one_mu;  // momentum, 1 - momentum
    double eps;
    bool nesterov;
    int steps;
};

__device__ __forceinline__ f16v mfma(h8 a, h8 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
// hi = fp16(v), lo = fp16(v - hi), of N values.
template <typename V, int N>
__device__ __forceinline__ void split(const float (&v)[N], V& hi, V& lo) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < N; e += 2) {  // two to a conversion
        const h2 h = __builtin_convertvector(f2{v[e], v[e + 1]}, h2);
        // v - (float)h as one instruction (64 x 64: 15.4 -> 14.5 us)
        const uint32_t both = __builtin_bit_cast(uint32_t, h);
        float l0, l1;
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(l0) : "v"(both), "v"(v[e]));
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]"
            : "=v"(l1) : "v"(both), "v"(v[e + 1]));
        const h2 l = __builtin_convertvector(f2{l0, l1}, h2);
        hi[e] = h[0], hi[e + 1] = h[1];
        lo[e] = l[0], lo[e + 1] = l[1];
    }
}

// Momentum and update of an element: the one place where both are formed.
__device__ __forceinline__ float next_momentum(const Hyper& h, float m, float g) {
    return fmaf(h.mu, m, h.one_mu * g);
}
__device__ __forceinline__ float update_of(const Hyper& h, float m, float g) {
    return h.nesterov ? fmaf(h.mu, m, h.one_mu * g) : m;
}

// kUp over the norm and eps, as a factor from 1 to 2 and a power of two: it may lie beyond fp32.
struct Inverse {
    float by;
    int power;
    __device__ __forceinline__ void of(double squares, double eps) {
        const double v = (double)kUp / (sqrt(squares) + eps);
        const int e = ilogb(v);
        power = e < -2000 ? -2000 : e > 2000 ? 2000 : e;  // of zero or a NaN: `by` stays what v is
        by = (float)ldexp(v, -power);
    }
    __device__ __forceinline__ float times(float u) const { return ldexpf(u, power) * by; }
};

// Whether four elements of type T and of float from a multiple of four on are one access.
__device__ __forceinline__ bool takes_vectors(const void* g, size_t e, const void* m) {
    return (((uintptr_t)g & (4 * e - 1)) | ((uintptr_t)m & 15)) == 0;
}

// ------------------------------------------------------------------ small matrices
constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / kWave;
constexpr int kSmallLds = 150 * 1024;
constexpr int kMaxSmall = 72;

struct Small {
    void* p;
    const void* g;
    float* m;
    float wd, ls;      // 1 - lr weight_decay; lr scale
    short rows, cols;  // of X: rows <= cols
    short mp, np;      // padded to 32
    int ld;            // columns of the parameter
    int tall;          // X is the transposed
};
struct SmallTable {
    Small t[kMaxSmall];
};
static_assert(sizeof(SmallTable) <= 3800, "kernel arguments end at 4 KB");

// Planes in LDS, high and low: rows of `width` elements, 8 more to keep rows off each other's
// banks.
__host__ __device__ inline int small_stride(int width) { return width + 8; }
size_t small_lds(int mp, int np) {
    return (size_t)4 * mp * (small_stride(np) + small_stride(mp));
}

// A matrix of planes in LDS.
struct Planes {
    _Float16* at;
    int plane, stride;
};
// Operands of a product of 32 x 32 by 16 of the contraction: p of rows (or, of the transposed,
// columns) of one matrix, q of rows of the other.
struct SmallFrags {
    h8 p[2], q[2];
    __device__ __forceinline__ static void row(h8 (&o)[2], const _Float16* a, int plane) {
        o[0] = *(const h8*)a;
        o[1] = *(const h8*)(a + plane);
    }
    __device__ __forceinline__ static void col(h8 (&o)[2], const _Float16* a, int plane,
                                               int stride) {
#pragma unroll
        for (int pl = 0; pl < 2; ++pl, a += plane)
            o[pl] = __builtin_bit_cast(
                h8, wtile::tr_pair((const char*)a, (const char*)(a + 4 * stride)));
    }
};
// The sum over K (a multiple of 32) of p q, the block at (i0, j0).  Operands are read one step
// ahead, among the products.
template <bool kTurned>
__device__ __forceinline__ f16v small_product(const Planes& P, int i0, const Planes& Q, int j0,
                                              int K, int lane) {
    const _Float16* q = Q.at + (j0 + (lane & 31)) * Q.stride + 8 * (lane >> 5);
    const _Float16* p =
        P.at + (kTurned ? (8 * (lane >> 5) + ((lane & 15) >> 2)) * P.stride + i0 +
                              16 * ((lane >> 4) & 1) + 4 * (lane & 3)
                        : (i0 + (lane & 31)) * P.stride + 8 * (lane >> 5));
    f16v acc = {};
    auto read_p = [&](SmallFrags& f, int k) {
        if constexpr (kTurned) SmallFrags::col(f.p, p + k * P.stride, P.plane, P.stride);
        else SmallFrags::row(f.p, p + k, P.plane);
    };
    auto step = [&](const SmallFrags& now, SmallFrags& then, int k) {
        SmallFrags::row(then.q, q + k, Q.plane);
        acc = mfma(now.p[0], now.q[1], acc);
        __builtin_amdgcn_sched_barrier(0);
        read_p(then, k);
        acc = mfma(now.p[1], now.q[0], acc);
        __builtin_amdgcn_sched_barrier(0);
        acc = mfma(now.p[0], now.q[0], acc);
        __builtin_amdgcn_sched_barrier(0);
    };
    SmallFrags a, b;
    SmallFrags::row(a.q, q, Q.plane);
    read_p(a, 0);
    for (int k = 0; k < K; k += 32) {
        step(a, b, k + 16);
        step(b, a, k + 32 < K ? k + 32 : 0);
    }
    return acc;
}
// A block from (i0, j0) on, as rows j of a matrix (i runs along them).
__device__ __forceinline__ void put_block(const Planes& M, int i0, int j0, const float (&v)[16],
                                          int lane) {
    _Float16* p = M.at + (j0 + (lane & 31)) * M.stride + i0 + 4 * (lane >> 5);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float x[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        h4 hi, lo;
        split(x, hi, lo);
        *(h4*)(p + 8 * q) = hi;
        *(h4*)(p + M.plane + 8 * q) = lo;
    }
}

// Walks the n elements of a matrix in the order of memory, V together, kSlots times V to a thread
// before the next ones: read(slot, i) of them, then use(slot, i, row, column).
constexpr int kSlots = 4;
template <int V, typename Read, typename Use>
__device__ __forceinline__ void in_order(int n, int ld, Read read, Use use) {
    constexpr int B = kSlots, kStep = kSmallThreads * V;
    for (int i0 = threadIdx.x * V; i0 < n; i0 += B * kStep) {
#pragma unroll
        for (int j = 0; j < B; ++j)
            if (i0 + j * kStep < n) read(j, i0 + j * kStep);
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int i = i0 + j * kStep, r = i / ld;
            if (i < n) use(j, i, r, i - r * ld);
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ void get(const T* p, float (&v)[V]) {
    if constexpr (V == 1) v[0] = to_f32(*p);
    else unpack_vec<T, V>(*(const typename VecT<T, V>::type*)p, v);
}
template <typename T, int V>
__device__ __forceinline__ void put(T* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = from_f32<T>(v[0]);
    } else if constexpr (sizeof(T) == 4) {
        *(f4*)p = f4{v[0], v[1], v[2], v[3]};
    } else {
        *(u2v*)p = u2v{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    }
}
// The momentum, and the update, in the parameter's order, to LDS; returns its sum of squares.
template <typename T, int V>
__device__ __forceinline__ double small_momentum(const Small& e, const Hyper& h, float* U,
                                                 int stride) {
    float g[kSlots][V], m[kSlots][V];
    double sum = 0.0;
    in_order<V>(
        e.rows * e.cols, e.ld,
        [&](int j, int i) {
            get<T, V>((const T*)e.g + i, g[j]);
            get<float, V>(e.m + i, m[j]);
        },
        [&](int j, int i, int r, int c) {
#pragma unroll
            for (int x = 0; x < V; ++x) {
                m[j][x] = next_momentum(h, m[j][x], g[j][x]);
                const float u = update_of(h, m[j][x], g[j][x]);
                U[r * stride + c + x] = u;
                sum = fma((double)u, (double)u, sum);
            }
            put<float, V>(e.m + i, m[j]);
        });
    return sum;
}
template <typename T, int V>
__device__ __forceinline__ void small_apply(const Small& e, const float* U, int stride) {
    float p[kSlots][V];
    const float ls = e.ls * kDown;
    in_order<V>(
        e.rows * e.cols, e.ld, [&](int j, int i) { get<T, V>((const T*)e.p + i, p[j]); },
        [&](int j, int i, int r, int c) {
#pragma unroll
            for (int x = 0; x < V; ++x)
                p[j][x] = fmaf(-ls, U[r * stride + c + x], p[j][x] * e.wd);
            put<T, V>((T*)e.p + i, p[j]);
        });
}

// X, A and B are held times kUp.  The parameter, the gradient and the momentum are read and
// written in the order of memory, through LDS: a wave's own elements of X lie in 32 rows, and
// reading them from there took 21 of 76 us at 128 x 128.  A wave has a block of 32 x 32 of X, and
// one of A: eight waves of two blocks each read less of LDS and took 51 us where sixteen of one
// take 45 (64 x 64: 26 and 15).
template <typename T>
__global__ __launch_bounds__(kSmallThreads) void small_kernel(SmallTable tab, Hyper h) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ double red[kSmallWaves];
    __shared__ Inverse inverse;
    const Small& e = tab.t[blockIdx.x];
    const int lane = threadIdx.x & 63, w = wave_id();
    const int mp = e.mp, np = e.np, mt = mp / 32;
    Planes X, A;
    X.stride = small_stride(np), X.plane = mp * X.stride, X.at = (_Float16*)smem;
    A.stride = small_stride(mp), A.plane = mp * A.stride, A.at = X.at + 2 * X.plane;
    float* U = (float*)smem;  // the update in the parameter's order, before and after the products
    const int us = e.ld + 1;
    // Columns i0 on, rows j0 on: lane l has row j0 + l % 32 and of the columns
    // 8 (v / 4) + 4 (l / 32) + v % 4.  The same of A.
    const int i0 = w / mt * 32, j0 = w % mt * 32;
    const bool has = i0 < np, has_a = i0 < mp;
    const int row = j0 + (lane & 31), col0 = i0 + 4 * (lane >> 5);
    auto col = [&](int v) { return col0 + 8 * (v >> 2) + (v & 3); };
    auto at = [&](int v) { return (e.tall ? col(v) : row) * us + (e.tall ? row : col(v)); };
    auto in = [&](int v) { return has && row < e.rows && col(v) < e.cols; };
    const bool vec = takes_vectors(e.g, sizeof(T), e.m) && takes_vectors(e.p, sizeof(T), e.m) &&
                     e.ld % 4 == 0;
    double sum = vec ? small_momentum<T, 4>(e, h, U, us) : small_momentum<T, 1>(e, h, U, us);
    sum = lanes::wave_sum(sum);
    if (lane == 0) red[w] = sum;
    __syncthreads();
    if (w == 0) {  // one wave: in all of them its 64-bit arithmetic took 2 us
        sum = 0.0;
        for (int k = 0; k < kSmallWaves; ++k) sum += red[k];
        if (lane == 0) inverse.of(sum, h.eps);
    }
    float x[16], a[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = in(v) ? U[at(v)] : 0.0f;
    __syncthreads();
    const Inverse inv = inverse;
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = inv.times(x[v]);
    if (has) put_block(X, i0, j0, x, lane);
    __syncthreads();
    for (int step = 0; step < h.steps; ++step) {
        if (has_a) {
            const f16v acc = small_product<false>(X, i0, X, j0, np, lane);
#pragma unroll
            for (int v = 0; v < 16; ++v) a[v] = acc[v] * kDown;
            put_block(A, i0, j0, a, lane);
        }
        __syncthreads();
        if (has_a) {
            const f16v acc = small_product<false>(A, i0, A, j0, mp, lane);
#pragma unroll
            for (int v = 0; v < 16; ++v) a[v] = fmaf(kC * kDown, acc[v], kB * a[v]);
        }
        __syncthreads();
        if (has_a) put_block(A, i0, j0, a, lane);
        __syncthreads();
        if (has) {
            const f16v acc = small_product<true>(X, i0, A, j0, mp, lane);
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] = fmaf(kDown, acc[v], kA * x[v]);
        }
        if (step + 1 == h.steps) break;
        __syncthreads();
        if (has) put_block(X, i0, j0, x, lane);
        __syncthreads();
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 16; ++v)
        if (in(v)) U[at(v)] = x[v];
    __syncthreads();
    vec ? small_apply<T, 4>(e, U, us) : small_apply<T, 1>(e, U, us);
}

// ------------------------------------------------------------------ large matrices
constexpr int kNT = 256;
constexpr int kPad = 64;        // sides are padded to it
constexpr int kMaxLarge = 16;   // matrices to a launch
constexpr int kNormChunk = 4096;

// How a matrix of two fp16 numbers an element lies in memory: row by row, 32 elements at a time,
// their high parts and then their low ones, 128 bytes together.  So the 32 of the contraction that
// are multiplied at a time are one whole cache line of a row (as planes apart they were two
// halves of lines, and loads took half as long again).
constexpr int kBK = 32;
__host__ __device__ inline int64_t place(int64_t row, int64_t col, int64_t width) {  // of the high part
    return (row * width + (col & ~(int64_t)31)) * 2 + (col & 31);
}

struct Large {
    void* p;
    const void* g;
    float* m;
    // X and its transposed, twice, and A and B (see place()).
    _Float16 *x[2], *xt[2], *a, *b;
    double* norm;    // partial sums of squares
    int64_t n;       // elements
    float wd, ls;
    int rows, cols;  // of X
    int mp, np;
    int ld, tall;
    int chunks;
};
enum Work { kSquares, kOthers, kChunks, kPacks };  // tiles of symmetric and other products, ...
struct LargeTable {
    int first[4][kMaxLarge];  // the matrices' first work of each kind; unused ones 2^31 - 1
    Large t[kMaxLarge];
    int count, eighths;
};
static_assert(sizeof(LargeTable) <= 3800, "kernel arguments end at 4 KB");

// The matrix that work `at` is of.
template <Work kKind>
__device__ __forceinline__ int find(const LargeTable& tab, int at) {
    int k = 0;
#pragma unroll
    for (int i = 1; i < kMaxLarge; ++i) k += at >= tab.first[kKind][i];
    return __builtin_amdgcn_readfirstlane(k);
}

// Four elements from i on of n, one access where vec (then i is a multiple of four).
template <typename T>
__device__ __forceinline__ void get4(const T* p, int64_t i, int64_t n, bool vec, float (&v)[4]) {
    if (vec && i + 4 <= n) {
        unpack_vec<T, 4>(*(const typename VecT<T, 4>::type*)(p + i), v);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = i + k < n ? to_f32(p[i + k]) : 0.0f;
    }
}
// Momentum, and the sums of squares of the update: 4,096 elements a workgroup (16,384: 12 us in
// place of 8 for three million, the same for 26).
template <typename T>
__global__ __launch_bounds__(kNT) void momentum_kernel(LargeTable tab, Hyper h) {
    constexpr int B = 4;  // accesses of a thread on their way
    __shared__ double red[kNT / kWave];
    const int at = find<kChunks>(tab, blockIdx.x), chunk = blockIdx.x - tab.first[kChunks][at];
    const Large& e = tab.t[at];
    const int64_t from = (int64_t)chunk * kNormChunk + threadIdx.x * 4;
    const T* g = (const T*)e.g;
    const bool vec = takes_vectors(e.g, sizeof(T), e.m);
    double sum = 0.0;
    for (int j0 = 0; j0 < kNormChunk / (4 * kNT); j0 += B) {
        float gv[B][4], mv[B][4];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int64_t i = from + (j0 + j) * 4 * kNT;
            get4(g, i, e.n, vec, gv[j]);
            get4(e.m, i, e.n, vec, mv[j]);
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int64_t i = from + (j0 + j) * 4 * kNT;
#pragma unroll
            for (int x = 0; x < 4; ++x) {  // what lies behind the end is zeros
                mv[j][x] = next_momentum(h, mv[j][x], gv[j][x]);
                const double u = update_of(h, mv[j][x], gv[j][x]);
                sum = fma(u, u, sum);
            }
            if (vec && i + 4 <= e.n) {
                *(f4*)(e.m + i) = f4{mv[j][0], mv[j][1], mv[j][2], mv[j][3]};
            } else {
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (i + x < e.n) e.m[i + x] = mv[j][x];
            }
        }
    }
    sum = lanes::wave_sum(sum);
    if ((threadIdx.x & 63) == 0) red[wave_id()] = sum;
    __syncthreads();
    if (threadIdx.x == 0) e.norm[chunk] = ((red[0] + red[1]) + red[2]) + red[3];
}

// X and its transposed, 64 x 64 elements a workgroup; zeros beyond the matrix.
template <typename T>
__global__ __launch_bounds__(kNT) void pack_kernel(LargeTable tab, Hyper h) {
    __shared__ double red[kNT / kWave];
    __shared__ Inverse inverse;
    __shared__ float tile[64][65];
    const int which = find<kPacks>(tab, blockIdx.x);
    const Large& e = tab.t[which];
    const int t = threadIdx.x, at = blockIdx.x - tab.first[kPacks][which];
    const int across = e.np / 64, r0 = at / across * 64, c0 = at % across * 64;  // of X
    // tile[a][b]: a along the parameter's rows
    const T* g = (const T*)e.g;
    const int pr0 = e.tall ? c0 : r0, pc0 = e.tall ? r0 : c0;
    const int prows = e.tall ? e.cols : e.rows, pcols = e.tall ? e.rows : e.cols;
    const bool vec = takes_vectors(e.g, sizeof(T), e.m) && e.ld % 4 == 0;
    float gv[4][4], mv[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int a = pr0 + 16 * j + (t >> 4), b = pc0 + 4 * (t & 15);
        const int n = a < prows ? pcols : 0;  // elements of the row
        get4(g + (int64_t)a * e.ld, b, n, vec, gv[j]);
        get4(e.m + (int64_t)a * e.ld, b, n, vec, mv[j]);
    }
    double sum = 0.0;
    for (int i = t; i < e.chunks; i += kNT) sum += e.norm[i];
    sum = lanes::wave_sum(sum);
    if ((t & 63) == 0) red[wave_id()] = sum;
    __syncthreads();
    if (t == 0) inverse.of(((red[0] + red[1]) + red[2]) + red[3], h.eps);
    __syncthreads();
    const Inverse inv = inverse;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x)
            tile[16 * j + (t >> 4)][4 * (t & 15) + x] =
                inv.times(update_of(h, mv[j][x], gv[j][x]));
    __syncthreads();
    // Eight elements of a row of X, and of its transposed, at a time.
    auto put = [&](_Float16* to, int a, int b, bool turned) {
        float v[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] = turned ? tile[b + x][a] : tile[a][b + x];
        h8 hi, lo;
        split(v, hi, lo);
        *(h8*)to = hi;
        *(h8*)(to + 32) = lo;
    };
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int a = 32 * j + (t >> 3), b = 8 * (t & 7);
        put(e.x[0] + place(r0 + a, c0 + b, e.np), a, b, e.tall);
        put(e.xt[0] + place(c0 + a, r0 + b, e.mp), a, b, !e.tall);
    }
}

// One product over all matrices: P Q^T with both operands' rows along the contraction.
enum Product { kGram, kPoly, kNext, kLast };  // A = X X^T; B = b A + c A A; X' = a X + B X; the last

__device__ __forceinline__ void to_lds(const _Float16* g, char* l) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)g,
                                     (__attribute__((address_space(3))) void*)l, 16, 0, 0);
}

// Tiles.  A workgroup of WI x WJ waves has a tile of kI rows and kJ columns, a wave FI x FJ blocks
// of 32 x 32.  A slice of 32 of the contraction in LDS: [P, Q][rows][8 chunks of 16 bytes, high
// and low], a row's chunk c at place c ^ (row / 2) % 8, so that 16 rows' reads of one chunk fall on
// different banks.  S slices: S - 1 on their way while one is multiplied.
template <int WI_, int WJ_, int FI_, int FJ_, int S_>
struct Tile {
    static constexpr int WI = WI_, WJ = WJ_, FI = FI_, FJ = FJ_, S = S_;
    static constexpr int kI = 32 * WI * FI, kJ = 32 * WJ * FJ, kNT = kWave * WI * WJ;
    static constexpr int kStage = (kI + kJ) * 128;
    static constexpr int kPieces = kStage / 1024 / (WI * WJ);  // loads of 1 KB, 8 rows, to a wave
    static constexpr int kRow = kJ + 1;  // floats in a row of the epilogue's buffer
    static constexpr int kLds = S * kStage > 64 * kRow * 4 ? S * kStage : 64 * kRow * 4;
};

// Where a lane's pieces of a slice come from: an operand's rows from the tile's first on, `rows`
// of them (those behind are read as the last one).
struct Source {
    const _Float16* p;
    int rows;
};
template <class G>
struct Loads {
    const _Float16* at[G::kPieces];
    int first;
    __device__ __forceinline__ Loads(const Source& P, const Source& Q, int64_t K, int w,
                                     int lane) {
        first = w * G::kPieces;
#pragma unroll
        for (int j = 0; j < G::kPieces; ++j) {
            const int block = (first + j) * 8;  // first row of the piece
            const bool second = block >= G::kI;
            const int row = block - (second ? G::kI : 0) + (lane >> 3);
            const int chunk = (lane & 7) ^ ((row >> 1) & 7);
            const int rows = second ? Q.rows : P.rows, r = row < rows ? row : rows - 1;
            at[j] = (second ? Q.p : P.p) + r * K * 2 + chunk * 8;
        }
    }
    __device__ __forceinline__ void piece(int j, int64_t s, char* lds) const {
        to_lds(at[j] + s * 64, lds + (first + j) * 1024);
    }
};
// Operands of 16 of the contraction.
template <class G>
struct Frags {
    static constexpr int kReads = G::FI + G::FJ, kMfma = 3 * G::FI * G::FJ;
    h8 p[G::FI][2], q[G::FJ][2];
    // The n-th of the reads.
    __device__ __forceinline__ void read(int n, const char* lds, int wi, int wj, int ks,
                                         int lane) {
        if (n < G::FI) one(p[n], lds, wi + 32 * n, ks, lane);
        else one(q[n - G::FI], lds + G::kI * 128, wj + 32 * (n - G::FI), ks, lane);
    }
    __device__ __forceinline__ static void one(h8 (&o)[2], const char* lds, int row0, int ks,
                                               int lane) {
        const int row = row0 + (lane & 31), chunk = 2 * ks + (lane >> 5), f = (row >> 1) & 7;
        o[0] = *(const h8*)(lds + row * 128 + ((chunk ^ f) << 4));
        o[1] = *(const h8*)(lds + row * 128 + (((chunk + 4) ^ f) << 4));
    }
    // The n-th of the products: low times high of every block, high times low, high times high.
    __device__ __forceinline__ void multiply(int n, f16v (&acc)[G::FI][G::FJ]) const {
        const int term = n / (G::FI * G::FJ), i = n / G::FJ % G::FI, j = n % G::FJ;
        acc[i][j] = mfma(p[i][term == 1], q[j][term == 0], acc[i][j]);
    }
};

// Eight elements of a parameter's row from column c on, as far as it has them.
template <typename T>
__device__ __forceinline__ void get8(const T* p, int64_t r, int64_t c, int rows, int cols, int ld,
                                     bool vec, float (&v)[8]) {
    p += r * ld + c;
    if (vec && r < rows && c + 8 <= cols) {
        get<T, 4>(p, *(float(*)[4])v);
        get<T, 4>(p + 4, *(float(*)[4])(v + 4));
    } else {
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] = r < rows && c + x < cols ? to_f32(p[x]) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void put8(T* p, int64_t r, int64_t c, int rows, int cols, int ld,
                                     bool vec, const float (&v)[8]) {
    p += r * ld + c;
    if (vec && r < rows && c + 8 <= cols) {
        put<T, 4>(p, *(const float(*)[4])v);
        put<T, 4>(p + 4, *(const float(*)[4])(v + 4));
    } else {
#pragma unroll
        for (int x = 0; x < 8; ++x)
            if (r < rows && c + x < cols) p[x] = from_f32<T>(v[x]);
    }
}

// Waits until at most N of the wave's loads are on their way.
template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N < 64, "six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
    asm volatile("" ::: "memory");
}

template <typename T, Product kKind, class G>
__global__ __launch_bounds__(G::kNT, 1) void product_kernel(LargeTable tab, int from) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int t = threadIdx.x, lane = t & 63, w = wave_id();
    constexpr bool kSquare = kKind == kGram || kKind == kPoly;
    // Workgroups go to the XCDs in turn.  Where there is one to each compute unit, every XCD takes
    // a run of all tiles, so that a matrix is read by few of them (a fifth faster); else an eighth
    // of each matrix's, so that none has the longest to itself.
    const int per = gridDim.x / 8, b = tab.eighths ? (int)blockIdx.x
                                                   : (int)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
    constexpr Work kWork = kSquare ? kSquares : kOthers;
    const int k = find<kWork>(tab, b);
    const Large& e = tab.t[k];
    const int down = (e.mp + G::kI - 1) / G::kI;
    const int across = kSquare ? down : (e.np + G::kJ - 1) / G::kJ;
    const int tiles = kSquare ? down * (down + 1) / 2 : down * across;
    const int l = b - tab.first[kWork][k], eighth = (tiles + 7) / 8;
    const int at = tab.eighths ? (l & 7) * eighth + (l >> 3) : l;
    if (at >= tiles || (tab.eighths && (l >> 3) >= eighth)) return;
    int ti, tj;  // tile row and column
    if constexpr (kSquare) {
        // Tiles on and below the diagonal, row by row.
        ti = (int)((sqrtf(8.0f * at + 1.0f) - 1.0f) * 0.5f);
        while (ti * (ti + 1) / 2 > at) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= at) ++ti;
        tj = at - ti * (ti + 1) / 2;
    } else {
        // Bands of eight tile rows, column by column.
        const int band = at / (8 * across), in = at - band * 8 * across;
        const int high = down - 8 * band < 8 ? down - 8 * band : 8;
        ti = 8 * band + in % high;
        tj = in / high;
    }
    const int K = kKind == kGram ? e.np : e.mp;
    const int64_t r0 = (int64_t)ti * G::kI, c0 = (int64_t)tj * G::kJ;
    Source P, Q;
    P.p = kKind == kGram ? e.x[from] : kKind == kPoly ? e.a : e.b;
    Q.p = kSquare ? P.p : e.xt[from];
    P.p += 2 * r0 * K;
    Q.p += 2 * c0 * K;
    P.rows = e.mp - (int)r0;
    Q.rows = (kSquare ? e.mp : e.np) - (int)c0;
    const Loads<G> loads(P, Q, K, w, lane);
    const int wi = w / G::WJ * 32 * G::FI, wj = w % G::WJ * 32 * G::FJ;
    f16v acc[G::FI][G::FJ] = {};
    const int slices = K / kBK;
    // Operands are read 16 of the contraction ahead of their products, and loads of a later slice
    // lie among the products: issued together they hold a wave up for as long as half of these.
    using F = Frags<G>;
    F even, odd;
    auto slice_at = [&](int s) { return smem + (s % G::S) * G::kStage; };
    auto known = [&](int s) { return s < slices ? s : slices - 1; };  // the last one again
#pragma unroll
    for (int s = 0; s < G::S; ++s)
#pragma unroll
        for (int j = 0; j < G::kPieces; ++j) loads.piece(j, known(s), slice_at(s));
    wait_loads<(G::S - 1) * G::kPieces>();
    wtile::lds_barrier();
#pragma unroll
    for (int n = 0; n < F::kReads; ++n) even.read(n, slice_at(0), wi, wj, 0, lane);
    for (int s = 0; s < slices; ++s) {
        const char* lds = slice_at(s);
#pragma unroll
        for (int n = 0; n < F::kMfma; ++n) {
#pragma unroll
            for (int r = 0; r < F::kReads; ++r)
                if (r * F::kMfma / F::kReads / 2 == n) odd.read(r, lds, wi, wj, 1, lane);
            even.multiply(n, acc);
            __builtin_amdgcn_sched_barrier(0);
        }
        // Slice s + 1 has arrived; slice s was read, its place is filled again.
        wait_loads<(G::S - 2) * G::kPieces>();
        wtile::lds_barrier();
        const int next = known(s + G::S);
        char* place = slice_at(s);
        lds = slice_at(s + 1);
#pragma unroll
        for (int n = 0; n < F::kMfma; ++n) {
#pragma unroll
            for (int r = 0; r < F::kReads; ++r)
                if (r * F::kMfma / F::kReads / 2 == n) even.read(r, lds, wi, wj, 0, lane);
#pragma unroll
            for (int j = 0; j < G::kPieces; ++j)
                if (j * F::kMfma / G::kPieces == n) loads.piece(j, next, place);
            odd.multiply(n, acc);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    wait_loads<0>();
    // The tile through LDS, 64 rows at a time: what is added read by rows, results written by
    // rows, and again by columns as the transposed.  Eight values of a row, or of a column, to a
    // thread.
    float* buf = (float*)smem;  // [64][kRow]
    const int64_t width = kSquare ? e.mp : e.np;
    _Float16* out = kKind == kGram ? e.a : kKind == kPoly ? e.b : e.x[from ^ 1];
    _Float16* out_t = kSquare ? out : e.xt[from ^ 1];
    const _Float16* add = kKind == kPoly ? e.a : e.x[from];
    constexpr int kAcross = G::kJ / 8, kPasses = 64 * kAcross / G::kNT, kRows = 64 / kPasses;
    constexpr int kPassesT = G::kJ * 8 / G::kNT, kCols = G::kJ / kPassesT;
    const int r1 = t / kAcross, c1 = t % kAcross * 8;  // by rows
    const int c2 = t / 8, r2 = t % 8 * 8;              // by columns
    const bool vec = kKind == kLast && ((uintptr_t)e.p & 15) == 0 &&
                     e.ld % (16 / (int)sizeof(T)) == 0;
    for (int band = 0; band < G::kI / 64; ++band) {
        const int64_t rr = r0 + 64 * band;
        if (rr >= e.mp) break;
        // What is read of memory, ahead of the first write.
        h8 old[kKind == kGram ? 1 : kPasses][2];
        float was[kKind == kLast ? kPasses : 1][8];
        static_assert(kPasses == kPassesT, "a tile has as many rows in a band as wave columns");
        if constexpr (kKind != kGram) {
#pragma unroll
            for (int pass = 0; pass < kPasses; ++pass) {
                if (c0 + c1 >= width) continue;
                const int64_t o = place(rr + pass * kRows + r1, c0 + c1, width);
                old[pass][0] = *(const h8*)(add + o);
                old[pass][1] = *(const h8*)(add + o + 32);
            }
        }
        if constexpr (kKind == kLast) {
#pragma unroll
            for (int pass = 0; pass < kPasses; ++pass) {
                const int64_t r = rr + (e.tall ? r2 : pass * kRows + r1);
                const int64_t c = c0 + (e.tall ? pass * kCols + c2 : c1);
                if (e.tall) get8((const T*)e.p, c, r, e.cols, e.rows, e.ld, vec, was[pass]);
                else get8((const T*)e.p, r, c, e.rows, e.cols, e.ld, vec, was[pass]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G::FI; ++i)
            if ((wi + 32 * i) / 64 == band)
#pragma unroll
                for (int j = 0; j < G::FJ; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        buf[((wi + 32 * i) % 64 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) *
                                G::kRow + wj + 32 * j + (lane & 31)] = acc[i][j][v];
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < kPasses; ++pass) {
            const int r = pass * kRows + r1;
            if (c0 + c1 >= width) continue;
            float* cell = buf + r * G::kRow + c1;
            float v[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] = cell[x];
            if constexpr (kKind == kGram) {
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] *= kDown;
            } else {
                const h8 hi = old[pass][0], lo = old[pass][1];
                constexpr float ka = kKind == kPoly ? kB : kA, kp = kKind == kPoly ? kC : 1.0f;
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    v[x] = fmaf(kp * kDown, v[x], ka * ((float)hi[x] + (float)lo[x]));
            }
            if constexpr (kKind == kLast) {
                if (!e.tall) {
#pragma unroll
                    for (int x = 0; x < 8; ++x) v[x] = fmaf(-e.ls * kDown, v[x], was[pass][x] * e.wd);
                    put8((T*)e.p, rr + r, c0 + c1, e.rows, e.cols, e.ld, vec, v);
                    continue;
                }
            } else {
                h8 hi, lo;
                split(v, hi, lo);
                const int64_t o = place(rr + r, c0 + c1, width);
                *(h8*)(out + o) = hi;
                *(h8*)(out + o + 32) = lo;
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) cell[x] = v[x];
        }
        if (kSquare && ti == tj) continue;        // its own transposed
        if (kKind == kLast && !e.tall) continue;  // nobody reads it
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < kPasses; ++pass) {
            const int c = pass * kCols + c2;
            if (c0 + c >= width) continue;
            float v[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] = buf[(r2 + x) * G::kRow + c];
            if constexpr (kKind == kLast) {
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] = fmaf(-e.ls * kDown, v[x], was[pass][x] * e.wd);
                put8((T*)e.p, c0 + c, rr + r2, e.cols, e.rows, e.ld, vec, v);
            } else {
                const int64_t o = place(c0 + c, rr + r2, e.mp);
                h8 hi, lo;
                split(v, hi, lo);
                *(h8*)(out_t + o) = hi;
                *(h8*)(out_t + o + 32) = lo;
            }
        }
    }
}

// ------------------------------------------------------------------ launches
struct Shape {
    int rows, cols, mp, np;
    bool tall, small;
};
Shape shape_of(const recblr_muon_tensor& t) {
    Shape s;
    s.tall = t.rows > t.cols;
    s.rows = (int)(s.tall ? t.cols : t.rows);
    s.cols = (int)(s.tall ? t.rows : t.cols);
    s.mp = (s.rows + 31) / 32 * 32;
    s.np = (s.cols + 31) / 32 * 32;
    // A block of 32 x 32 to each wave, and the planes in LDS.
    s.small = (int64_t)(s.mp / 32) * (s.np / 32) <= kSmallWaves &&
              small_lds(s.mp, s.np) <= (size_t)kSmallLds;
    if (!s.small) {
        s.mp = (s.rows + kPad - 1) / kPad * kPad;
        s.np = (s.cols + kPad - 1) / kPad * kPad;
    }
    return s;
}
bool nothing(const recblr_muon_tensor& t) { return t.rows == 0 || t.cols == 0; }
size_t align256(size_t n) { return (n + 255) / 256 * 256; }
int chunks_of(int64_t n) { return (int)((n + kNormChunk - 1) / kNormChunk); }
size_t large_bytes(const Shape& s, int64_t n) {
    return 4 * align256((size_t)s.mp * s.np * 4) + 2 * align256((size_t)s.mp * s.mp * 4) +
           align256((size_t)chunks_of(n) * 8);
}

using Tile256 = Tile<2, 4, 4, 2, 2>;
using Tile128 = Tile<2, 2, 2, 2, 4>;       // one to a compute unit
using Tile128Pair = Tile<2, 2, 2, 2, 2>;   // two
using Tile64 = Tile<2, 2, 1, 1, 4>;

int64_t tiles_of(const Large& l, bool square, int side) {
    const int64_t down = (l.mp + side - 1) / side, across = (l.np + side - 1) / side;
    return square ? down * (down + 1) / 2 : down * across;
}

// Which tiles to take.  Their time, from measurements on the whole chip: `fixed` us and `each`
// for 32 of the contraction, `slots` of them at once; where there are more, what is left over at
// the end is counted as half of the shortest.  2000 x 2000 takes 779 us with tiles of 64, 685
// and 770 with the two of 128, 1,807 with 256; 1000 x 1000: 207, 383, 439, 1,111; 4096 x 4096:
// 5,868, 4,350, 4,274, 3,884 (five steps).
struct Choice {
    int side, slots;
    float each, fixed;
};
constexpr Choice kChoices[] = {{64, 512, 0.50f, 4.0f},
                               {128, 256, 0.78f, 6.0f},
                               {128, 512, 1.45f, 8.0f},
                               {256, 256, 2.50f, 28.0f}};
int choose(const LargeTable& tab, bool square, bool gram) {
    int best = 0;
    float least = 0.0f;
    for (int c = 0; c < 4; ++c) {
        const Choice& k = kChoices[c];
        float sum = 0.0f, longest = 0.0f, shortest = 3e38f;
        int64_t n = 0;
        for (int i = 0; i < tab.count; ++i) {
            const Large& l = tab.t[i];
            const float one = k.fixed + k.each * (float)((gram ? l.np : l.mp) / 32);
            const int64_t tiles = tiles_of(l, square, k.side);
            n += tiles;
            sum += one * (float)tiles;
            longest = one > longest ? one : longest;
            shortest = one < shortest ? one : shortest;
        }
        float time = sum / (float)k.slots + 0.5f * shortest;
        if (n <= k.slots || time < longest) time = longest;
        if (c == 0 || time < least) {
            least = time;
            best = c;
        }
    }
    return best;
}

template <typename T, Product kKind, class G>
hipError_t run_product(LargeTable& tab, int from, hipStream_t st) {
    constexpr bool kSquare = kKind == kGram || kKind == kPoly;
    int64_t all = 0;
    for (int i = 0; i < tab.count; ++i) all += tiles_of(tab.t[i], kSquare, G::kI);
    tab.eighths = all > 256;
    int64_t groups = 0;
    for (int i = 0; i < tab.count; ++i) {
        tab.first[kSquare ? kSquares : kOthers][i] = (int)groups;
        const int64_t n = tiles_of(tab.t[i], kSquare, G::kI);
        groups += tab.eighths ? (n + 7) / 8 * 8 : n;
    }
    groups = (groups + 7) / 8 * 8;
    static std::atomic<uint64_t> done{0};
    const auto kernel = product_kernel<T, kKind, G>;
    const hipError_t e = allow_dynamic_lds((const void*)kernel, G::kLds, done);
    if (e != hipSuccess) return e;
    kernel<<<dim3((unsigned)groups), G::kNT, G::kLds, st>>>(tab, from);
    return hipGetLastError();
}
template <typename T, Product kKind>
hipError_t run_product(LargeTable& tab, int choice, int from, hipStream_t st) {
    return choice == 0   ? run_product<T, kKind, Tile64>(tab, from, st)
           : choice == 1 ? run_product<T, kKind, Tile128>(tab, from, st)
           : choice == 2 ? run_product<T, kKind, Tile128Pair>(tab, from, st)
                         : run_product<T, kKind, Tile256>(tab, from, st);
}

template <typename T>
hipError_t run_large(LargeTable& tab, const int (&work)[2], const Hyper& h, hipStream_t st) {
    momentum_kernel<T><<<dim3((unsigned)work[0]), kNT, 0, st>>>(tab, h);
    pack_kernel<T><<<dim3((unsigned)work[1]), kNT, 0, st>>>(tab, h);
    hipError_t e = hipGetLastError();
    const int gram = choose(tab, true, true), poly = choose(tab, true, false),
              next = choose(tab, false, false);
    for (int s = 0; s < h.steps && e == hipSuccess; ++s) {
        const int from = s & 1;
        e = run_product<T, kGram>(tab, gram, from, st);
        if (e == hipSuccess) e = run_product<T, kPoly>(tab, poly, from, st);
        if (e == hipSuccess)
            e = s + 1 < h.steps ? run_product<T, kNext>(tab, next, from, st)
                                : run_product<T, kLast>(tab, next, from, st);
    }
    return e;
}

template <typename T>
hipError_t run(const recblr_muon_tensor* tensors, int64_t count, const MuonHyper& hy, void* ws,
               hipStream_t st) {
    const Hyper h{(float)hy.momentum, (float)(1.0 - hy.momentum), hy.eps, hy.nesterov, hy.steps};
    SmallTable small;
    int smalls = 0;
    size_t lds = 0;
    auto flush_small = [&]() {
        if (!smalls) return hipSuccess;
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_dynamic_lds((const void*)small_kernel<T>, kSmallLds, done);
        if (e != hipSuccess) return e;
        small_kernel<T><<<dim3((unsigned)smalls), kSmallThreads, lds, st>>>(small, h);
        smalls = 0;
        lds = 0;
        return hipGetLastError();
    };
    LargeTable large;
    large.count = 0;
    int work[2] = {0, 0};
    char* at = (char*)ws;
    auto flush_large = [&]() {
        if (!large.count) return hipSuccess;
        // Those with the longest products first: their tiles are the last to end.
        std::stable_sort(large.t, large.t + large.count,
                         [](const Large& a, const Large& b) { return a.np > b.np; });
        for (auto& kind : large.first) std::fill(kind, kind + kMaxLarge, 0x7FFFFFFF);
        for (int i = 0; i < large.count; ++i) {
            Large& l = large.t[i];
            large.first[kChunks][i] = work[0];
            large.first[kPacks][i] = work[1];
            work[0] += l.chunks;
            work[1] += l.mp / 64 * (l.np / 64);
        }
        const hipError_t e = run_large<T>(large, work, h, st);
        large.count = 0;
        for (int& x : work) x = 0;
        at = (char*)ws;  // the next ones' launches come behind these on the stream
        return e;
    };
    for (int64_t i = 0; i < count; ++i) {
        const recblr_muon_tensor& t = tensors[i];
        if (nothing(t)) continue;
        const Shape s = shape_of(t);
        const float wd = (float)(1.0 - hy.lr * t.weight_decay), ls = (float)(hy.lr * t.scale);
        if (s.small) {
            small.t[smalls++] = Small{t.param, t.grad, t.m, wd, ls, (short)s.rows, (short)s.cols,
                                      (short)s.mp, (short)s.np, (int)t.cols, s.tall};
            const size_t need = small_lds(s.mp, s.np);
            lds = need > lds ? need : lds;
            if (smalls == kMaxSmall) {
                const hipError_t e = flush_small();
                if (e != hipSuccess) return e;
            }
            continue;
        }
        Large& l = large.t[large.count++];
        const int64_t n = t.rows * t.cols;
        auto take = [&](size_t bytes) {
            char* p = at;
            at += align256(bytes);
            return p;
        };
        const size_t xb = (size_t)s.mp * s.np * 4, ab = (size_t)s.mp * s.mp * 4;
        l.p = t.param;
        l.g = t.grad;
        l.m = t.m;
        for (int k = 0; k < 2; ++k) {
            l.x[k] = (_Float16*)take(xb);
            l.xt[k] = (_Float16*)take(xb);
        }
        l.a = (_Float16*)take(ab);
        l.b = (_Float16*)take(ab);
        l.chunks = chunks_of(n);
        l.norm = (double*)take((size_t)l.chunks * 8);
        l.n = n;
        l.wd = wd;
        l.ls = ls;
        l.rows = s.rows;
        l.cols = s.cols;
        l.mp = s.mp;
        l.np = s.np;
        l.ld = (int)t.cols;
        l.tall = s.tall;
        if (large.count == kMaxLarge) {
            const hipError_t e = flush_large();
            if (e != hipSuccess) return e;
        }
    }
    const hipError_t e = flush_small();
    return e != hipSuccess ? e : flush_large();
}

}  // namespace

// That of the kMaxLarge large ones, in the order of the list, that take most together.
size_t muon_workspace(const recblr_muon_tensor* tensors, int64_t count) {
    size_t most = 0, n = 0;
    int used = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (nothing(tensors[i])) continue;
        const Shape s = shape_of(tensors[i]);
        if (s.small) continue;
        n += large_bytes(s, tensors[i].rows * tensors[i].cols);
        most = std::max(most, n);
        if (++used == kMaxLarge) used = 0, n = 0;
    }
    return most;
}

hipError_t launch_muon(const recblr_muon_tensor* tensors, int64_t count, IoType io,
                       const MuonHyper& h, void* ws, hipStream_t st) {
    return io == IoType::kF32 ? run<float>(tensors, count, h, ws, st)
                              : run<bf16>(tensors, count, h, ws, st);
}

}  // namespace recblr
