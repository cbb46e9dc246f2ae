// Lookup of items in a table, and the table's gradient (recblr_embed_forward, _backward).
//
// The lookup moves 2 D e bytes a position.  The gradient of a row is the sum of dout over the
// positions that name it, D e bytes a position once they are known, and the row itself.
//
// Finding them: positions are sorted by id (stably, so an item's positions stay in order),
// by counting digits of up to 12 bits: each block of positions counts its digits, the counts
// of a digit become each block's first place within it, and the blocks place their positions,
// 64 at a time, a lane's place among the lanes of the same digit by ballots.  The sorted
// positions are cut into pieces of 64, a wave each, whatever items they hold, so a popular
// item spreads over many waves; a run of an item that lies within a piece is its row, and
// runs that go over borders leave partial sums, joined by a second launch in their order.
// Which addition follows which hangs on the ids alone.
//
// Few positions: each wave looks for its position's id among all; the first of an id sums them.
#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "lanes.hpp"
#include "ops.hpp"
#include "wave_tile.hpp"

namespace recblr {
namespace {

using wtile::u4v;

constexpr int kNT = 256;

// ------------------------------------------------------------------ lookup
template <typename T, bool VEC>
__global__ __launch_bounds__(kNT) void lookup_kernel(const T* __restrict__ table,
                                                     const int32_t* __restrict__ ids,
                                                     T* __restrict__ out, int64_t N, int64_t V,
                                                     int D, int units, int rows, float scale,
                                                     int32_t pad_id) {
    constexpr int U = VEC ? 16 / (int)sizeof(T) : 1;
    const int64_t row0 = (int64_t)blockIdx.x * rows;
#pragma unroll 4
    for (int j = threadIdx.x; j < rows * units; j += kNT) {
        const int rl = (int)((unsigned)j / (unsigned)units), u = j - rl * units;
        const int64_t row = row0 + rl;
        if (row >= N) break;
        const int id = ids[row];
        const bool some = id != pad_id && id >= 0 && id < V;
        const float none = id == pad_id ? 0.0f : __uint_as_float(0x7FC00000u);
        T* o = out + row * D + u * U;
        if constexpr (VEC) {
            u4v v = {0, 0, 0, 0};
            if (some) v = *(const u4v*)(table + (int64_t)id * D + u * U);
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = __float_as_uint(some ? __uint_as_float(v[e]) * scale : none);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = bf16_pair(some ? bf16_lo(v[e]) * scale : none,
                                     some ? bf16_hi(v[e]) * scale : none);
            }
            *(u4v*)o = v;
        } else {
            *o = from_f32<T>(some ? to_f32(table[(int64_t)id * D + u]) * scale : none);
        }
    }
}

// ------------------------------------------------------------------ rows of the gradient
// A wave's columns of a row: lane l has VL of them from (64 c + l) VL on.
template <typename T, int VL>
__device__ __forceinline__ void read_row(const T* p, float (&v)[VL]) {
    if constexpr (VL == 1) {
        v[0] = to_f32(*p);
    } else {
        unpack_vec<T, VL>(*(const typename VecT<T, VL>::type*)p, v);
    }
}
template <typename T, int VL>
__device__ __forceinline__ void write_row(T* p, const float (&v)[VL], float scale, bool add) {
    float o[VL];
    if (add)
        read_row<T, VL>(p, o);
    else
#pragma unroll
        for (int e = 0; e < VL; ++e) o[e] = 0.0f;
#pragma unroll
    for (int e = 0; e < VL; ++e) o[e] = add ? fmaf(scale, v[e], o[e]) : scale * v[e];
    if constexpr (VL == 1) {
        *p = from_f32<T>(o[0]);
    } else {
        typename VecT<T, VL>::type w;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < VL; ++e) w[e] = o[e];
        } else if constexpr (VL == 2) {
            w = bf16_pair(o[0], o[1]);
        } else {
            w = {bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3])};
        }
        *(typename VecT<T, VL>::type*)p = w;
    }
}

struct Grad {
    const void* dout;
    void* dtable;
    int D;
    float scale;
    bool add;
};

// ------------------------------------------------------------------ few positions
constexpr int kFew = 1024;

template <typename T, int VL>
__global__ __launch_bounds__(kNT) void few_kernel(const int32_t* __restrict__ ids, int N,
                                                  int64_t V, int32_t pad_id, Grad g) {
    __shared__ int32_t all[kFew];
    for (int i = threadIdx.x; i < N; i += kNT) all[i] = ids[i];
    __syncthreads();
    const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + wave_id();
    if (i >= N) return;
    const int id = all[i];
    if (id == pad_id || id < 0 || id >= V) return;
    for (int j = lane; j - lane < i; j += kWave)
        if (__ballot(j < i && all[j] == id)) return;  // an earlier position has it
    const int col = ((int)blockIdx.y * kWave + lane) * VL;
    const bool live = col < g.D;
    const T* dout = (const T*)g.dout + col;
    float acc[VL] = {};
    for (int j0 = i & ~63; j0 < N; j0 += kWave) {
        const int j = j0 + lane;
        uint64_t m = __ballot(j >= i && j < N && all[j < N ? j : 0] == id);
        while (m) {
            float v[4][VL];  // four rows' reads at once
            int n = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (!m) break;
                const int at = j0 + __builtin_ctzll(m);
                m &= m - 1;
                if (live) read_row<T, VL>(dout + (int64_t)at * g.D, v[k]);
                n = k + 1;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < n)
#pragma unroll
                    for (int e = 0; e < VL; ++e) acc[e] += v[k][e];
        }
    }
    if (live) write_row<T, VL>((T*)g.dtable + (int64_t)id * g.D + col, acc, g.scale, g.add);
}

// ------------------------------------------------------------------ sorting positions by id
constexpr int kMaxBits = 12, kMaxBins = 1 << kMaxBits;
constexpr int kMaxBlocks = 512;
constexpr int kWaves = kNT / kWave;
constexpr int kTile = 2048;  // a block's positions are a multiple of this

// ids of no row sort behind all others, as V.
__device__ __forceinline__ uint32_t key_of(int32_t id, int64_t V, int32_t pad_id) {
    return id == pad_id || id < 0 || id >= V ? (uint32_t)V : (uint32_t)id;
}

struct Sort {
    const int32_t* ids;        // the first pass's keys
    const uint32_t* keys_in;   // later passes'
    const int32_t* pos_in;
    uint32_t* keys;
    int32_t* pos;
    uint32_t* counts;  // [blocks][bins]
    uint32_t* totals;  // [bins]
    int64_t N, V;
    int64_t each;  // positions to a block
    int blocks, bits, shift;
    int32_t pad_id;
};
__device__ __forceinline__ uint32_t sort_key(const Sort& s, int64_t i) {
    return s.ids ? key_of(s.ids[i], s.V, s.pad_id) : s.keys_in[i];
}

// Blocks from s.blocks on fill the table with zeros, 16 bytes at a time.
__global__ __launch_bounds__(kNT) void count_kernel(Sort s, void* fill, int64_t fill_bytes) {
    __shared__ uint32_t bins[kMaxBins];
    const int n = 1 << s.bits;
    if ((int)blockIdx.x >= s.blocks) {
        const int64_t step = (int64_t)(gridDim.x - s.blocks) * kNT * 16;
        int64_t at = ((int64_t)(blockIdx.x - s.blocks) * kNT + threadIdx.x) * 16;
        char* p = (char*)fill;
        const int64_t head = -(int64_t)(uintptr_t)p & 15;  // bytes before the first 16 aligned
        const int64_t body = fill_bytes > head ? (fill_bytes - head) & ~15ll : 0;
        const u4v zero = {0, 0, 0, 0};
        for (; at < body; at += step) *(u4v*)(p + head + at) = zero;
        if (blockIdx.x == (unsigned)s.blocks && threadIdx.x < 32) {
            const int64_t b = threadIdx.x < 16 ? (int64_t)threadIdx.x
                                               : head + body + (int64_t)threadIdx.x - 16;
            if (threadIdx.x < 16 ? b < head && b < fill_bytes : b < fill_bytes) p[b] = 0;
        }
        return;
    }
    for (int i = threadIdx.x; i < n; i += kNT) bins[i] = 0;
    __syncthreads();
    const int64_t from = blockIdx.x * s.each, to = min(s.N, from + s.each);
#pragma unroll 4
    for (int64_t i = from + threadIdx.x; i < to; i += kNT)
        atomicAdd(&bins[sort_key(s, i) >> s.shift & (n - 1)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kNT) s.counts[(int64_t)blockIdx.x * n + i] = bins[i];
}

// counts: each block's first place within its digit; totals: the digits' sizes.  A lane has a
// digit, a wave a run of blocks.
__global__ __launch_bounds__(1024) void offsets_kernel(Sort s) {
    constexpr int kRun = kMaxBlocks / 16;
    __shared__ uint32_t sum[16][kWave];
    const int n = 1 << s.bits, lane = threadIdx.x & 63, w = wave_id();
    const int bin = blockIdx.x * kWave + lane, run = (s.blocks + 15) / 16;
    uint32_t c[kRun], total = 0;
#pragma unroll
    for (int r = 0; r < kRun; ++r) {
        const int b = w * run + r;
        c[r] = r < run && b < s.blocks && bin < n ? s.counts[(int64_t)b * n + bin] : 0;
    }
#pragma unroll
    for (int r = 0; r < kRun; ++r) total += c[r];
    sum[w][lane] = total;
    __syncthreads();
    uint32_t before = 0, whole = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        before += k < w ? sum[k][lane] : 0;
        whole += sum[k][lane];
    }
    if (bin >= n) return;
#pragma unroll
    for (int r = 0; r < kRun; ++r) {
        const int b = w * run + r;
        if (r < run && b < s.blocks) s.counts[(int64_t)b * n + bin] = before;
        before += c[r];
    }
    if (w == 0) s.totals[bin] = whole;
}

__global__ __launch_bounds__(kNT) void place_kernel(Sort s) {
    __shared__ uint32_t next[kWaves][kMaxBins];  // a wave's next place of each digit
    __shared__ uint32_t wsum[kWaves];
    const int n = 1 << s.bits, t = threadIdx.x, lane = t & 63, w = wave_id();
    const uint64_t below = (1ull << lane) - 1;
    for (int i = t; i < kWaves * n; i += kNT) next[i / n][i % n] = 0;
    __syncthreads();
    // A wave's positions are one run of its block's.
    const int64_t from = blockIdx.x * s.each + w * (s.each / kWaves);
    const int64_t to = min(s.N, from + s.each / kWaves);
#pragma unroll 4
    for (int64_t i = from + lane; i < to; i += kWave)
        atomicAdd(&next[w][sort_key(s, i) >> s.shift & (n - 1)], 1u);
    __syncthreads();
    // Digits before a thread's run of digits, then each digit's first place for each wave.
    const int run = (n + kNT - 1) / kNT;
    uint32_t mine = 0;
    for (int k = 0; k < run; ++k)
        if (t * run + k < n) mine += s.totals[t * run + k];
    uint32_t upto = lanes::wave_scan(mine, 0u, [](uint32_t a, uint32_t b) { return a + b; });
    if (lane == kWave - 1) wsum[w] = upto;
    __syncthreads();
    uint32_t at = upto - mine;
    for (int k = 0; k < w; ++k) at += wsum[k];
    for (int k = 0; k < run; ++k) {
        const int d = t * run + k;
        if (d >= n) break;
        uint32_t place = at + s.counts[(int64_t)blockIdx.x * n + d];
        for (int v = 0; v < kWaves; ++v) {
            const uint32_t c = next[v][d];
            next[v][d] = place;
            place += c;
        }
        at += s.totals[d];
    }
    __syncthreads();
    for (int64_t i0 = from; i0 < to; i0 += kWave) {
        const int64_t i = i0 + lane;
        const bool live = i < to;
        const uint32_t key = live ? sort_key(s, i) : 0;
        const uint32_t d = key >> s.shift & (n - 1);
        uint64_t same = __ballot(live);
        for (int b = 0; b < s.bits; ++b) {
            const bool bit = d >> b & 1;
            const uint64_t m = __ballot(bit);
            same &= bit ? m : ~m;
        }
        if (live) {
            const int rank = __popcll(same & below);
            const uint32_t place = next[w][d] + rank;
            wave_fence();
            if ((same >> lane) == 1ull) next[w][d] = place + 1;  // the last of its digit
            s.keys[place] = key;
            s.pos[place] = s.pos_in ? s.pos_in[i] : (int32_t)i;
        }
        wave_fence();
    }
}

// ------------------------------------------------------------------ sums of runs
constexpr int kPiece = 64;

// part: for each piece, the sum of a run that came from before (slot 0) and of one that starts
// here and goes on (slot 1).
template <typename T, int VL>
__global__ __launch_bounds__(kNT) void piece_kernel(const uint32_t* __restrict__ keys,
                                                    const int32_t* __restrict__ pos, int64_t N,
                                                    int64_t V, Grad g, float* part,
                                                    int64_t pieces) {
    const int64_t piece = (int64_t)blockIdx.x * 4 + wave_id();
    if (piece >= pieces) return;
    const int lane = threadIdx.x & 63;
    const int64_t from = piece * kPiece, i = from + lane;
    const uint32_t none = (uint32_t)V;
    const uint32_t key = i < N ? keys[i] : none;
    const uint32_t after = i + 1 < N ? keys[i + 1] : none;
    const int at = i < N ? pos[i] : 0;
    const uint32_t before = from > 0 ? keys[from - 1] : none;
    const int live = __popcll(__ballot(key != none));  // sorted: the first ones
    if (live == 0) return;
    const uint64_t ends = __ballot(key != after);
    bool earlier = lanes::lane_of(key, 0) == before;  // this run came from before
    const int col = ((int)blockIdx.y * kWave + lane) * VL;
    const bool in = col < g.D;
    const T* dout = (const T*)g.dout + col;
    float* slot = part + piece * 2 * g.D + col;
    float acc[VL] = {};
    constexpr int B = 8;
    for (int j0 = 0; j0 < live; j0 += B) {
        float v[B][VL];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int r = __builtin_amdgcn_readlane(at, j0 + j);  // behind the last one: row 0
            if (in) read_row<T, VL>(dout + (int64_t)r * g.D, v[j]);
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            if (j0 + j >= live) break;
#pragma unroll
            for (int e = 0; e < VL; ++e) acc[e] += v[j][e];
            if (ends >> (j0 + j) & 1) {
                const uint32_t k = lanes::lane_of(key, j0 + j);
                if (in) {
                    if (earlier) {
#pragma unroll
                        for (int e = 0; e < VL; ++e) slot[e] = acc[e];
                    } else {
                        write_row<T, VL>((T*)g.dtable + (int64_t)k * g.D + col, acc, g.scale,
                                         g.add);
                    }
                }
                earlier = false;
#pragma unroll
                for (int e = 0; e < VL; ++e) acc[e] = 0.0f;
            }
        }
    }
    if (live == kPiece && !(ends >> 63) && in) {  // goes on
        float* to = earlier ? slot : slot + g.D;
#pragma unroll
        for (int e = 0; e < VL; ++e) to[e] = acc[e];
    }
}

constexpr int kJoin = 512;

// The workgroup of the piece in which a run starts that goes on: its parts in eight runs of
// pieces, then these in order.
template <typename T, int VL>
__global__ __launch_bounds__(kJoin) void join_kernel(const uint32_t* __restrict__ keys, int64_t N,
                                                     int64_t V, Grad g, const float* part,
                                                     int64_t pieces) {
    constexpr int W = kJoin / kWave;
    __shared__ float all[W][kWave * VL];
    const int64_t p = blockIdx.x, last = p * kPiece + kPiece - 1;
    if (last + 1 >= N) return;
    const uint32_t k = keys[last];
    if (k == (uint32_t)V || keys[last + 1] != k) return;
    if (keys[p * kPiece] == k && p > 0 && keys[p * kPiece - 1] == k) return;  // from before
    // The last piece whose first key is k: ever larger steps, then halves.
    int64_t lo = p + 1, step = 1;
    while (lo + step < pieces && keys[(lo + step) * kPiece] == k) {
        lo += step;
        step *= 2;
    }
    int64_t hi = min(pieces, lo + step);  // keys[lo * kPiece] == k, and not at hi
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if (keys[mid * kPiece] == k) lo = mid;
        else hi = mid;
    }
    const int lane = threadIdx.x & 63, w = wave_id();
    const int col = ((int)blockIdx.y * kWave + lane) * VL;
    const bool in = col < g.D;
    const int64_t n = lo - p, run = n <= 16 ? n : (n + W - 1) / W;
    float acc[VL] = {};
    if (in) {
        if (w == 0)
#pragma unroll
            for (int e = 0; e < VL; ++e) acc[e] = part[(p * 2 + 1) * g.D + col + e];
        const int64_t end = min(lo + 1, p + 1 + (w + 1) * run);
#pragma unroll 8
        for (int64_t q = p + 1 + w * run; q < end; ++q)
#pragma unroll
            for (int e = 0; e < VL; ++e) acc[e] += part[q * 2 * g.D + col + e];
    }
    if (run < n) {
#pragma unroll
        for (int e = 0; e < VL; ++e) all[w][lane * VL + e] = acc[e];
        __syncthreads();
        if (w == 0)
            for (int v = 1; v < W; ++v)
#pragma unroll
                for (int e = 0; e < VL; ++e) acc[e] += all[v][lane * VL + e];
    }
    if (w == 0 && in) write_row<T, VL>((T*)g.dtable + (int64_t)k * g.D + col, acc, g.scale, g.add);
}

// ------------------------------------------------------------------ launches
struct Plan {
    int passes, bits, blocks;
    int64_t each, pieces;
    size_t keys[2], pos[2], counts, totals, part, bytes;
};
Plan plan(int64_t N, int64_t V, int64_t D) {
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    Plan p{};
    int all = 1;  // bits of the keys 0 .. V
    while ((V >> all) > 0) ++all;
    p.passes = (all + kMaxBits - 1) / kMaxBits;
    p.bits = (all + p.passes - 1) / p.passes;
    int64_t each = (N + kMaxBlocks - 1) / kMaxBlocks;
    p.each = (each + kTile - 1) / kTile * kTile;
    p.blocks = (int)((N + p.each - 1) / p.each);
    p.pieces = (N + kPiece - 1) / kPiece;
    size_t at = 0;
    for (int i = 0; i < (p.passes > 1 ? 2 : 1); ++i) {
        p.keys[i] = at;
        at += up((size_t)N * 4);
        p.pos[i] = at;
        at += up((size_t)N * 4);
    }
    p.counts = at;
    at += up(((size_t)p.blocks << p.bits) * 4);
    p.totals = at;
    at += up((size_t)4 << p.bits);
    p.part = at;
    at += up((size_t)p.pieces * 2 * D * 4);
    p.bytes = at;
    return p;
}

// Columns of a lane: as many as a wave needs for a row, where rows take accesses that wide.
int columns(const EmbedArgs& a) {
    const uintptr_t bits = (uintptr_t)a.src | (uintptr_t)a.dst;
    int vl = a.D <= 64 ? 1 : a.D <= 128 ? 2 : 4;
    while (vl > 1 && (a.D % vl || bits % (vl * io_bytes(a.io)))) vl /= 2;
    return vl;
}

template <typename T, int VL>
void launch_sums(const EmbedArgs& a, const Plan& pl, char* ws, const Grad& g, hipStream_t st) {
    const unsigned cols = (unsigned)((a.D + kWave * VL - 1) / (kWave * VL));
    if (a.N <= kFew) {
        few_kernel<T, VL><<<dim3((unsigned)((a.N + 3) / 4), cols), kNT, 0, st>>>(
            a.ids, (int)a.N, a.V, a.pad_id, g);
        return;
    }
    const int last = (pl.passes + 1) % 2;  // passes write buffers 0, 1, 0, ...
    const uint32_t* keys = (const uint32_t*)(ws + pl.keys[last]);
    const int32_t* pos = (const int32_t*)(ws + pl.pos[last]);
    float* part = (float*)(ws + pl.part);
    piece_kernel<T, VL><<<dim3((unsigned)((pl.pieces + 3) / 4), cols), kNT, 0, st>>>(
        keys, pos, a.N, a.V, g, part, pl.pieces);
    join_kernel<T, VL><<<dim3((unsigned)pl.pieces, cols), kJoin, 0, st>>>(keys, a.N, a.V, g, part,
                                                                         pl.pieces);
}

}  // namespace

size_t embed_workspace(int64_t N, int64_t V, int64_t D, IoType io) {
    return N <= kFew ? 0 : plan(N, V, D).bytes;
}

hipError_t launch_embed_forward(const EmbedArgs& a, hipStream_t st) {
    const int e = (int)io_bytes(a.io);
    const bool vec =
        (((uintptr_t)a.src | (uintptr_t)a.dst | (uintptr_t)(a.D * e)) & 15u) == 0;
    const int units = vec ? (int)(a.D * e / 16) : (int)a.D;
    const int rows = units >= 4 * kNT ? 1 : 4 * kNT / units;
    const dim3 grid((unsigned)((a.N + rows - 1) / rows));
    auto go = [&](auto kernel, auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        kernel<<<grid, kNT, 0, st>>>((const T*)a.src, a.ids, (T*)a.dst, a.N, a.V, (int)a.D, units,
                                     rows, a.scale, a.pad_id);
    };
    if (a.io == IoType::kF32)
        vec ? go(lookup_kernel<float, true>, (float*)nullptr)
            : go(lookup_kernel<float, false>, (float*)nullptr);
    else
        vec ? go(lookup_kernel<bf16, true>, (bf16*)nullptr)
            : go(lookup_kernel<bf16, false>, (bf16*)nullptr);
    return hipGetLastError();
}

hipError_t launch_embed_backward(const EmbedArgs& a, void* ws, hipStream_t st) {
    char* w = (char*)ws;
    const int64_t bytes = a.accumulate ? 0 : a.V * a.D * (int64_t)io_bytes(a.io);
    // Four 16-byte stores to a thread, at most 8 workgroups to a compute unit.
    int64_t fill = (bytes + kNT * 64 - 1) / (kNT * 64);
    fill = fill < 2048 ? fill : 2048;
    const bool few = a.N <= kFew;
    const Plan pl = plan(a.N > 0 ? a.N : 1, a.V, a.D);
    Sort s{};
    s.N = a.N;
    s.V = a.V;
    s.each = pl.each;
    s.pad_id = a.pad_id;
    if (few && fill > 0) count_kernel<<<dim3((unsigned)fill), kNT, 0, st>>>(s, a.dst, bytes);
    for (int i = 0; !few && i < pl.passes; ++i) {
        s.ids = i ? nullptr : a.ids;
        s.keys_in = (const uint32_t*)(w + pl.keys[(i + 1) % 2]);
        s.pos_in = i ? (const int32_t*)(w + pl.pos[(i + 1) % 2]) : nullptr;
        s.keys = (uint32_t*)(w + pl.keys[i % 2]);
        s.pos = (int32_t*)(w + pl.pos[i % 2]);
        s.counts = (uint32_t*)(w + pl.counts);
        s.totals = (uint32_t*)(w + pl.totals);
        s.blocks = pl.blocks;
        s.bits = pl.bits;
        s.shift = i * pl.bits;
        const int64_t zeros = i ? 0 : fill;
        count_kernel<<<dim3((unsigned)(pl.blocks + zeros)), kNT, 0, st>>>(s, a.dst, bytes);
        offsets_kernel<<<dim3((unsigned)(((1 << pl.bits) + 63) / 64)), 1024, 0, st>>>(s);
        place_kernel<<<dim3((unsigned)pl.blocks), kNT, 0, st>>>(s);
    }
    if (a.N > 0) {
        const Grad g{a.src, a.dst, (int)a.D, a.scale, a.accumulate};
        const int vl = columns(a);
        auto go = [&](auto* t) {
            using T = std::remove_pointer_t<decltype(t)>;
            if (vl == 1) launch_sums<T, 1>(a, pl, w, g, st);
            else if (vl == 2) launch_sums<T, 2>(a, pl, w, g, st);
            else launch_sums<T, 4>(a, pl, w, g, st);
        };
        a.io == IoType::kF32 ? go((float*)nullptr) : go((bf16*)nullptr);
    }
    return hipGetLastError();
}

}  // namespace recblr
