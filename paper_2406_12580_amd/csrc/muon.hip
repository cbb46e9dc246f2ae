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
#include <hip/hip_runtime.h>

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
// The product of two operands of two fp16 numbers each, the small terms first.
__device__ __forceinline__ f16v mma(const h8 (&a)[2], const h8 (&b)[2], f16v c) {
    c = mfma(a[0], b[1], c);
    c = mfma(a[1], b[0], c);
    return mfma(a[0], b[0], c);
}
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// Momentum and update of an element: the one place where both are formed.
__device__ __forceinline__ float next_momentum(const Hyper& h, float m, float g) {
    return fmaf(h.mu, m, h.one_mu * g);
}
__device__ __forceinline__ float update_of(const Hyper& h, float m, float g) {
    return h.nesterov ? fmaf(h.mu, m, h.one_mu * g) : m;
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

// Planes in LDS: rows of `width` elements, 8 more to keep rows off each other's banks.
__host__ __device__ inline int small_stride(int width) { return width + 8; }
size_t small_lds(int mp, int np) {
    return (size_t)4 * mp * (small_stride(np) + small_stride(mp));
}

// k from k0 on of operand row `row`, both planes.
__device__ __forceinline__ void row_operand(h8 (&o)[2], const _Float16* m, int plane, int stride,
                                            int row, int k) {
    o[0] = *(const h8*)(m + row * stride + k);
    o[1] = *(const h8*)(m + plane + row * stride + k);
}
// The same of the transposed: operand row = column col0 + lane % 32.
__device__ __forceinline__ void col_operand(h8 (&o)[2], const _Float16* m, int plane, int stride,
                                            int k0, int col0, int lane) {
    const _Float16* p = m + (k0 + 8 * (lane >> 5) + ((lane & 15) >> 2)) * stride + col0 +
                        16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    o[0] = __builtin_bit_cast(h8, wtile::tr_pair((const char*)p, (const char*)(p + 4 * stride)));
    p += plane;
    o[1] = __builtin_bit_cast(h8, wtile::tr_pair((const char*)p, (const char*)(p + 4 * stride)));
}
// Accumulators of tile (i0, j0), times kUp over their scale, as rows j of a matrix (i runs
// along them): four values at a time.
__device__ __forceinline__ void put_tile(_Float16* m, int plane, int stride, int i0, int j0,
                                         const float (&v)[16], int lane) {
    _Float16* p = m + (j0 + (lane & 31)) * stride + i0 + 4 * (lane >> 5);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        h4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            _Float16 a, b;
            split(v[4 * q + e] * kUp, a, b);
            hi[e] = a;
            lo[e] = b;
        }
        *(h4*)(p + 8 * q) = hi;
        *(h4*)(p + plane + 8 * q) = lo;
    }
}

template <typename T>
__global__ __launch_bounds__(kSmallThreads) void small_kernel(SmallTable tab, Hyper h) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ double red[kSmallWaves];
    const Small& e = tab.t[blockIdx.x];
    const int lane = threadIdx.x & 63, w = wave_id();
    const int mp = e.mp, np = e.np, xs = small_stride(np), as = small_stride(mp);
    const int xplane = mp * xs, aplane = mp * as;
    _Float16* X = (_Float16*)smem;
    _Float16* A = X + 2 * xplane;
    T* param = (T*)e.p;
    const T* grad = (const T*)e.g;
    // Wave w has the tile of X's columns i0 .. + 31 and rows j0 .. + 31: lane l row j0 + l % 32
    // and sixteen columns, 8 (v / 4) + 4 (l / 32) + v % 4.
    const int mt = mp / 32, nt = np / 32;
    const bool has = w < mt * nt, has_a = w < mt * mt;
    const int i0 = has ? w / mt * 32 : 0, j0 = has ? w % mt * 32 : 0;
    const int ai = has_a ? w / mt * 32 : 0, aj = has_a ? w % mt * 32 : 0;
    const int row = j0 + (lane & 31), col0 = i0 + 4 * (lane >> 5);
    auto at = [&](int v) {  // of the parameter
        const int c = col0 + 8 * (v >> 2) + (v & 3);
        return (int64_t)(e.tall ? c : row) * e.ld + (e.tall ? row : c);
    };
    auto in = [&](int v) { return has && row < e.rows && col0 + 8 * (v >> 2) + (v & 3) < e.cols; };
    float x[16];
    double sum = 0.0;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        x[v] = 0.0f;
        if (in(v)) {
            const int64_t i = at(v);
            const float g = to_f32(grad[i]), m = next_momentum(h, e.m[i], g);
            e.m[i] = m;
            x[v] = update_of(h, m, g);
        }
        sum = fma((double)x[v], (double)x[v], sum);
    }
    sum = lanes::wave_sum(sum);
    if (lane == 0) red[w] = sum;
    __syncthreads();
    sum = 0.0;
    for (int k = 0; k < kSmallWaves; ++k) sum += red[k];
    const float inv = (float)(1.0 / (sqrt(sum) + h.eps));
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] *= inv;
    if (has) put_tile(X, xplane, xs, i0, j0, x, lane);
    __syncthreads();
    const int ll = lane & 31, k8 = 8 * (lane >> 5);
    for (int step = 0; step < h.steps; ++step) {
        float a[16];
        f16v acc = {};
        if (has_a) {
            for (int k = 0; k < np; k += 16) {
                h8 p[2], q[2];
                row_operand(p, X, xplane, xs, ai + ll, k + k8);
                row_operand(q, X, xplane, xs, aj + ll, k + k8);
                acc = mma(p, q, acc);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) a[v] = acc[v] * (kDown * kDown);
            put_tile(A, aplane, as, ai, aj, a, lane);
        }
        __syncthreads();
        acc = f16v{};
        if (has_a) {
            for (int k = 0; k < mp; k += 16) {
                h8 p[2], q[2];
                row_operand(p, A, aplane, as, ai + ll, k + k8);
                row_operand(q, A, aplane, as, aj + ll, k + k8);
                acc = mma(p, q, acc);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v)
                a[v] = fmaf(kC * (kDown * kDown), acc[v], kB * a[v]);
        }
        __syncthreads();
        if (has_a) put_tile(A, aplane, as, ai, aj, a, lane);
        __syncthreads();
        acc = f16v{};
        if (has) {
            for (int k = 0; k < mp; k += 16) {
                h8 p[2], q[2];
                col_operand(p, X, xplane, xs, k, i0, lane);
                row_operand(q, A, aplane, as, j0 + ll, k + k8);
                acc = mma(p, q, acc);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] = fmaf(kA, x[v], acc[v] * (kDown * kDown));
        }
        __syncthreads();
        if (has) put_tile(X, xplane, xs, i0, j0, x, lane);
        __syncthreads();
    }
#pragma unroll
    for (int v = 0; v < 16; ++v)
        if (in(v)) {
            const int64_t i = at(v);
            param[i] = from_f32<T>(fmaf(-e.ls, x[v], to_f32(param[i]) * e.wd));
        }
}

// ------------------------------------------------------------------ large matrices
constexpr int kNT = 256;
constexpr int kTile = 128;      // output tile; sides are padded to it
constexpr int kBK = 32;         // contraction a slice
constexpr int kMaxLarge = 16;   // matrices to a launch
constexpr int kNormChunk = 16384;

struct Large {
    void* p;
    const void* g;
    float* m;
    // Planes (hi, then lo): X and its transposed, twice, and A and B.
    _Float16 *x[2], *xt[2], *a, *b;
    double* norm;    // partial sums of squares
    int64_t n;       // elements
    float wd, ls;
    int rows, cols;  // of X
    int mp, np;
    int ld, tall;
    int first_chunk, first_pack, first_a, first_x;  // work before this matrix's, in each launch
    int chunks;
};
struct LargeTable {
    Large t[kMaxLarge];
    int count;
};
static_assert(sizeof(LargeTable) <= 3800, "kernel arguments end at 4 KB");

template <int Large::*kFirst>
__device__ __forceinline__ int find(const LargeTable& tab, int at) {
    int k = 0;
#pragma unroll
    for (int i = 1; i < kMaxLarge; ++i) k += i < tab.count && at >= tab.t[i].*kFirst;
    return __builtin_amdgcn_readfirstlane(k);
}

// Momentum, and the sums of squares of the update.
template <typename T>
__global__ __launch_bounds__(kNT) void momentum_kernel(LargeTable tab, Hyper h) {
    __shared__ double red[kNT / kWave];
    const Large& e = tab.t[find<&Large::first_chunk>(tab, blockIdx.x)];
    const int chunk = blockIdx.x - e.first_chunk;
    const int64_t from = (int64_t)chunk * kNormChunk;
    const T* g = (const T*)e.g;
    double sum = 0.0;
#pragma unroll 8
    for (int j = 0; j < kNormChunk / kNT; ++j) {
        const int64_t i = from + j * kNT + threadIdx.x;
        if (i >= e.n) break;
        const float gv = to_f32(g[i]), m = next_momentum(h, e.m[i], gv);
        e.m[i] = m;
        const double u = update_of(h, m, gv);
        sum = fma(u, u, sum);
    }
    sum = lanes::wave_sum(sum);
    if ((threadIdx.x & 63) == 0) red[wave_id()] = sum;
    __syncthreads();
    if (threadIdx.x == 0) e.norm[chunk] = ((red[0] + red[1]) + red[2]) + red[3];
}

// X and its transposed as planes, 64 x 64 elements a workgroup; zeros beyond the matrix.
template <typename T>
__global__ __launch_bounds__(kNT) void pack_kernel(LargeTable tab, Hyper h) {
    __shared__ double red[kNT / kWave];
    __shared__ float tile[64][65];
    const Large& e = tab.t[find<&Large::first_pack>(tab, blockIdx.x)];
    const int t = threadIdx.x, at = blockIdx.x - e.first_pack;
    const int across = e.np / 64, r0 = at / across * 64, c0 = at % across * 64;  // of X
    double sum = 0.0;
    for (int i = t; i < e.chunks; i += kNT) sum += e.norm[i];
    sum = lanes::wave_sum(sum);
    if ((t & 63) == 0) red[wave_id()] = sum;
    __syncthreads();
    sum = ((red[0] + red[1]) + red[2]) + red[3];
    const float inv = (float)(1.0 / (sqrt(sum) + h.eps)) * kUp;
    const T* g = (const T*)e.g;
    // tile[a][b]: a along the parameter's rows
    const int pr0 = e.tall ? c0 : r0, pc0 = e.tall ? r0 : c0;
    const int prows = e.tall ? e.cols : e.rows, pcols = e.tall ? e.rows : e.cols;
    for (int i = t; i < 64 * 64; i += kNT) {
        const int a = i >> 6, b = i & 63;
        float u = 0.0f;
        if (pr0 + a < prows && pc0 + b < pcols) {
            const int64_t o = (int64_t)(pr0 + a) * e.ld + pc0 + b;
            u = update_of(h, e.m[o], to_f32(g[o])) * inv;
        }
        tile[a][b] = u;
    }
    __syncthreads();
    const int64_t plane = (int64_t)e.mp * e.np;
    for (int i = t; i < 64 * 64; i += kNT) {
        const int a = i >> 6, b = i & 63;
        _Float16 hi, lo;
        split(e.tall ? tile[b][a] : tile[a][b], hi, lo);
        _Float16* x = e.x[0] + (int64_t)(r0 + a) * e.np + c0 + b;
        x[0] = hi;
        x[plane] = lo;
        split(e.tall ? tile[a][b] : tile[b][a], hi, lo);
        x = e.xt[0] + (int64_t)(c0 + a) * e.mp + r0 + b;
        x[0] = hi;
        x[plane] = lo;
    }
}

// One product over all matrices: P Q^T with both operands' rows along the contraction.
enum Product { kGram, kPoly, kNext, kLast };  // A = X X^T; B = b A + c A A; X' = a X + B X; the last

__device__ __forceinline__ void to_lds(const _Float16* g, char* l) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)g,
                                     (__attribute__((address_space(3))) void*)l, 16, 0, 0);
}

// A slice in LDS: [operand][plane][128 rows][4 chunks of 16 bytes], a row's chunk c at place
// c ^ (row / 4) % 4, so that 16 rows' reads of one chunk fall on different banks.
constexpr int kOperand = kTile * kBK * 2;      // bytes of a plane
constexpr int kStage = 4 * kOperand;           // both operands, both planes
constexpr int kLargeLds = 2 * kStage;          // two slices
constexpr int kRowPad = kTile + 4;

// Loads of a slice: 32 pieces of 1 KB, 16 rows each; wave w takes eight.
__device__ __forceinline__ void load_slice(const _Float16* P, int64_t pplane, int pk,
                                           const _Float16* Q, int64_t qplane, int qk, int k0,
                                           char* lds, int w, int lane) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int piece = w * 8 + j;  // operand, plane, block of 16 rows
        const int op = piece >> 4, pl = (piece >> 3) & 1, block = piece & 7;
        const int row = block * 16 + (lane >> 2), chunk = (lane & 3) ^ ((row >> 2) & 3);
        const _Float16* src = op ? Q + pl * qplane + (int64_t)row * qk
                                 : P + pl * pplane + (int64_t)row * pk;
        to_lds(src + k0 + chunk * 8, lds + piece * 1024);
    }
}
__device__ __forceinline__ void slice_operand(h8 (&o)[2], const char* lds, int row, int chunk) {
    const int at = row * 64 + ((chunk ^ ((row >> 2) & 3)) << 4);
    o[0] = *(const h8*)(lds + at);
    o[1] = *(const h8*)(lds + kOperand + at);
}

template <typename T, Product kKind>
__global__ __launch_bounds__(kNT, 2) void product_kernel(LargeTable tab, int from) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int t = threadIdx.x, lane = t & 63, w = wave_id();
    constexpr bool kSquare = kKind == kGram || kKind == kPoly;
    // Workgroups go to the XCDs in turn; each XCD takes a run of tiles.
    const int all = gridDim.x, xcd = blockIdx.x & 7, per = all / 8, more = all % 8;
    const int b = xcd * per + (xcd < more ? xcd : more) + (blockIdx.x >> 3);
    const int k = kSquare ? find<&Large::first_a>(tab, b) : find<&Large::first_x>(tab, b);
    const Large& e = tab.t[k];
    int ti, tj;  // tile row and column
    if constexpr (kSquare) {
        // Tiles on and below the diagonal, row by row.
        const int at = b - e.first_a;
        ti = (int)((sqrtf(8.0f * at + 1.0f) - 1.0f) * 0.5f);
        while (ti * (ti + 1) / 2 > at) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= at) ++ti;
        tj = at - ti * (ti + 1) / 2;
    } else {
        const int at = b - e.first_x, down = e.mp / kTile;
        ti = at % down;
        tj = at / down;
    }
    const int K = kKind == kGram ? e.np : e.mp;
    const int64_t aplane = (int64_t)e.mp * e.mp, xplane = (int64_t)e.mp * e.np;
    const _Float16 *P, *Q;
    int64_t pplane, qplane;
    if constexpr (kKind == kGram) {
        P = Q = e.x[from];
        pplane = qplane = xplane;
    } else if constexpr (kKind == kPoly) {
        P = Q = e.a;
        pplane = qplane = aplane;
    } else {
        P = e.b;
        Q = e.xt[from];
        pplane = aplane;
        qplane = xplane;
    }
    P += (int64_t)ti * kTile * K;
    Q += (int64_t)tj * kTile * K;
    const int wi = (w >> 1) * 64, wj = (w & 1) * 64;
    f16v acc[2][2] = {};
    const int slices = K / kBK;
    load_slice(P, pplane, K, Q, qplane, K, 0, smem, w, lane);
    for (int s = 0; s < slices; ++s) {
        __syncthreads();  // the slice has arrived, and the other half's reads are done
        if (s + 1 < slices)
            load_slice(P, pplane, K, Q, qplane, K, (s + 1) * kBK, smem + ((s + 1) & 1) * kStage,
                       w, lane);
        const char* lds = smem + (s & 1) * kStage;
#pragma unroll
        for (int ks = 0; ks < kBK / 16; ++ks) {
            h8 p[2][2], q[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                slice_operand(p[i], lds, wi + 32 * i + (lane & 31), 2 * ks + (lane >> 5));
                slice_operand(q[i], lds + 2 * kOperand, wj + 32 * i + (lane & 31),
                              2 * ks + (lane >> 5));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = mma(p[i], q[j], acc[i][j]);
        }
    }
    // The tile through LDS, 64 rows at a time: what is added read by rows, results written by
    // rows, and again by columns as the transposed.
    float* buf = (float*)smem;  // [64][kRowPad]
    const int64_t r0 = (int64_t)ti * kTile, c0 = (int64_t)tj * kTile;
    const int64_t width = kSquare ? e.mp : e.np, plane = kSquare ? aplane : xplane;
    _Float16* out = kKind == kGram ? e.a : kKind == kPoly ? e.b : e.x[from ^ 1];
    _Float16* out_t = kSquare ? out : e.xt[from ^ 1];
    const _Float16* add = kKind == kPoly ? e.a : e.x[from];
    for (int half = 0; half < 2; ++half) {
        __syncthreads();
        if ((w >> 1) == half) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        buf[(32 * i + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * kRowPad + wj +
                            32 * j + (lane & 31)] = acc[i][j][v];
        }
        __syncthreads();
        const int64_t rr = r0 + 64 * half;
        // Sixteen rows of eight values a thread at a time.
#pragma unroll
        for (int pass = 0; pass < 4; ++pass) {
            const int r = pass * 16 + (t >> 4), c = (t & 15) * 8;
            float v[8];
#pragma unroll
            for (int x = 0; x < 8; x += 4) *(f4*)(v + x) = *(const f4*)(buf + r * kRowPad + c + x);
            const int64_t o = (rr + r) * width + c0 + c;
            if constexpr (kKind == kGram) {
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] *= kDown;
            } else {
                const h8 hi = *(const h8*)(add + o), lo = *(const h8*)(add + plane + o);
                constexpr float ka = kKind == kPoly ? kB : kA, kp = kKind == kPoly ? kC : 1.0f;
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    v[x] = fmaf(kp * kDown, v[x], ka * ((float)hi[x] + (float)lo[x]));
            }
            if constexpr (kKind == kLast) {
                if (!e.tall && rr + r < e.rows) {
                    T* param = (T*)e.p + (rr + r) * e.ld + c0 + c;
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        if (c0 + c + x < e.cols)
                            param[x] = from_f32<T>(
                                fmaf(-e.ls * kDown, v[x], to_f32(param[x]) * e.wd));
                }
            } else {
                h8 hi, lo;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    _Float16 a, d;
                    split(v[x], a, d);
                    hi[x] = a;
                    lo[x] = d;
                }
                *(h8*)(out + o) = hi;
                *(h8*)(out + plane + o) = lo;
            }
#pragma unroll
            for (int x = 0; x < 8; x += 4) *(f4*)(buf + r * kRowPad + c + x) = *(const f4*)(v + x);
        }
        if constexpr (kSquare)
            if (ti == tj) continue;  // it is its own transposed
        __syncthreads();
        // Rows of the transposed: column c of the 64 rows, eight values a thread.
        const int64_t tw = kSquare ? e.mp : e.mp;
#pragma unroll
        for (int pass = 0; pass < 4; ++pass) {
            const int c = pass * 32 + (t & 31), r = (t >> 5) * 8;
            float v[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] = buf[(r + x) * kRowPad + c];
            if constexpr (kKind == kLast) {
                if (e.tall && c0 + c < e.cols) {
                    T* param = (T*)e.p + (c0 + c) * e.ld + rr + r;
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        if (rr + r + x < e.rows)
                            param[x] = from_f32<T>(
                                fmaf(-e.ls * kDown, v[x], to_f32(param[x]) * e.wd));
                }
            } else {
                const int64_t o = (c0 + c) * tw + rr + r;
                h8 hi, lo;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    _Float16 a, d;
                    split(v[x], a, d);
                    hi[x] = a;
                    lo[x] = d;
                }
                *(h8*)(out_t + o) = hi;
                *(h8*)(out_t + plane + o) = lo;
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
    // A tile of X, and one of A, to each wave, and the planes in LDS.
    s.small = (int64_t)(s.mp / 32) * (s.np / 32) <= kSmallWaves &&
              small_lds(s.mp, s.np) <= (size_t)kSmallLds;
    if (!s.small) {
        s.mp = (s.rows + kTile - 1) / kTile * kTile;
        s.np = (s.cols + kTile - 1) / kTile * kTile;
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

template <typename T>
hipError_t run_large(const LargeTable& tab, const int (&work)[4], const Hyper& h,
                     hipStream_t st) {
    momentum_kernel<T><<<dim3((unsigned)work[0]), kNT, 0, st>>>(tab, h);
    pack_kernel<T><<<dim3((unsigned)work[1]), kNT, 0, st>>>(tab, h);
    int from = 0;
    for (int s = 0; s < h.steps; ++s) {
        const dim3 square((unsigned)work[2]), whole((unsigned)work[3]);
        product_kernel<T, kGram><<<square, kNT, kLargeLds, st>>>(tab, from);
        product_kernel<T, kPoly><<<square, kNT, kLargeLds, st>>>(tab, from);
        if (s + 1 < h.steps)
            product_kernel<T, kNext><<<whole, kNT, kLargeLds, st>>>(tab, from);
        else
            product_kernel<T, kLast><<<whole, kNT, kLargeLds, st>>>(tab, from);
        from ^= 1;
    }
    return hipGetLastError();
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
    int work[4] = {0, 0, 0, 0};
    char* at = (char*)ws;
    auto flush_large = [&]() {
        if (!large.count) return hipSuccess;
        const hipError_t e = run_large<T>(large, work, h, st);
        large.count = 0;
        for (int& x : work) x = 0;
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
        l.first_chunk = work[0];
        l.first_pack = work[1];
        l.first_a = work[2];
        l.first_x = work[3];
        const int mt = s.mp / kTile, nt = s.np / kTile;
        work[0] += l.chunks;
        work[1] += s.mp / 64 * (s.np / 64);
        work[2] += mt * (mt + 1) / 2;
        work[3] += mt * nt;
        if (large.count == kMaxLarge) {
            const hipError_t e = flush_large();
            if (e != hipSuccess) return e;
        }
    }
    const hipError_t e = flush_small();
    return e != hipSuccess ? e : flush_large();
}

}  // namespace

size_t muon_workspace(const recblr_muon_tensor* tensors, int64_t count) {
    size_t n = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (nothing(tensors[i])) continue;
        const Shape s = shape_of(tensors[i]);
        if (!s.small) n += large_bytes(s, tensors[i].rows * tensors[i].cols);
    }
    return n;
}

hipError_t launch_muon(const recblr_muon_tensor* tensors, int64_t count, IoType io,
                       const MuonHyper& h, void* ws, hipStream_t st) {
    return io == IoType::kF32 ? run<float>(tensors, count, h, ws, st)
                              : run<bf16>(tensors, count, h, ws, st);
}

}  // namespace recblr
