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
// item spreads over many waves; a run of an item that lies within a piece is its row, runs
// that go over the borders of pieces are joined by the workgroup of 16 pieces, and those that
// go over its borders by a second launch, in their order.  Which addition follows which hangs
// on the ids, the width and the alignment alone.
//
// Few positions are not sorted: each wave looks for its position's id among all, and the first of
// an id sums its rows.
//
// One MI355X: 409,600 positions of 64 fp32 over 3,416 items: lookup 19 us, 5.6 TB/s of what it
// writes; gradient 50: counts with the table's zeros 7, offsets 6, places 13, sums 20 (5.3 TB/s),
// joins 5.  524,288 of 128 bf16 over a million items: 48 and 92, of which its two passes of
// digits are 41.  Lookups and sums are bound by memory, the rest by a launch's chain of reads.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.hpp"
#include "lanes.hpp"
#include "ops.hpp"
#include "wave_tile.hpp"

namespace recblr {
namespace {

using wtile::u4v;

constexpr int kNT = 256;

// ------------------------------------------------------------------ lookup
// Four 16-byte accesses to a thread, of whole rows where these are short; results past the caches,
// where they would push the table out.
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
            __builtin_nontemporal_store(v, (u4v*)o);
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
// The same as it lies in memory, and its values.
template <typename T, int VL>
using RawRow = typename VecT<T, VL>::type;
template <typename T, int VL>
__device__ __forceinline__ RawRow<T, VL> raw_row(const T* p) {
    return *(const RawRow<T, VL>*)p;
}
template <typename T, int VL>
__device__ __forceinline__ void put_row(T* p, const float (&o)[VL]) {
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

// A row of the gradient while it is summed: old: what is there already, where it is added to.
template <typename T, int VL>
__device__ __forceinline__ void end_row(const Grad& g, uint32_t k, int col, const float (&acc)[VL],
                                        const float (&old)[VL]) {
    float o[VL];
#pragma unroll
    for (int e = 0; e < VL; ++e) o[e] = g.add ? fmaf(g.scale, acc[e], old[e]) : g.scale * acc[e];
    put_row<T, VL>((T*)g.dtable + (int64_t)k * g.D + col, o);
}

// ------------------------------------------------------------------ few positions
// Every workgroup has all ids in LDS, and each of its waves a position: the first one of an item
// sums the item's rows.  Those that more than kLight positions name are summed by the whole
// workgroup, a wave a run of all positions, and the waves' sums in their order.  Rows of 64 fp32:
// 1,024 positions 7 us, 11 where they all name one item; 4,000 13 to 34, by sorting 31 (a million
// items: 41); 8,192 24 to 64, by sorting 36.
constexpr int kFew = 4096, kFewThreads = 1024, kFewWaves = kFewThreads / kWave, kLight = 64;

// The sum of the rows at row(0) .. row(n - 1), by halves in groups of B.
template <typename T, int VL, typename Row>
__device__ __forceinline__ void add_rows(const T* dout, int D, bool live, int n, Row row,
                                         float (&acc)[VL]) {
    constexpr int B = VL < 4 ? 16 : 8;
    for (int k0 = 0; k0 < n; k0 += B) {
        RawRow<T, VL> raw[B];
#pragma unroll
        for (int k = 0; k < B; ++k) {  // in place of those behind the last one, the first one's again
            const int at = row(k0 + k < n ? k0 + k : k0);
            if (live) raw[k] = raw_row<T, VL>(dout + (int64_t)at * D);
        }
        float v[B][VL];
#pragma unroll
        for (int k = 0; k < B; ++k) {
            unpack_vec<T, VL>(raw[k], v[k]);
#pragma unroll
            for (int e = 0; e < VL; ++e) v[k][e] = k0 + k < n ? v[k][e] : 0.0f;
        }
#pragma unroll
        for (int h = B / 2; h > 0; h /= 2)
#pragma unroll
            for (int k = 0; k < h; ++k)
#pragma unroll
                for (int e = 0; e < VL; ++e) v[k][e] += v[k + h][e];
#pragma unroll
        for (int e = 0; e < VL; ++e) acc[e] += v[0][e];
    }
}

// Zeros to the rows of a run of `each` (at most 32 kFewWaves kWave) that none of the ids in
// all[0 .. N) names, V rows in all.
template <typename T>
__device__ __forceinline__ void clear_others(const int32_t* all, int N, T* table, int64_t V, int D,
                                             int64_t from, int each, uint32_t* named) {
    const int t = threadIdx.x, rows = (int)min((int64_t)each, V - from);
    named[t] = 0;
    __syncthreads();
    for (int k = t; k < N; k += kFewThreads) {
        const int64_t r = all[k] - from;
        if (r >= 0 && r < rows) atomicOr(&named[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    table += from * D;
    auto put = [&](auto zero, int units) {  // of a row
        for (int j = t; j < rows * units; j += kFewThreads) {
            const int r = (int)((unsigned)j / (unsigned)units);
            if (!(named[r >> 5] >> (r & 31) & 1)) ((decltype(zero)*)table)[j] = zero;
        }
    };
    const int bytes = D * (int)sizeof(T);
    if ((((uintptr_t)table | (unsigned)bytes) & 15) == 0) put(u4v{0, 0, 0, 0}, bytes / 16);
    else if constexpr (sizeof(T) == 4) put(0u, D);
    else put((uint16_t)0, D);
}

// Workgroups from `groups` on clear what no id names, `each` rows of the table.
template <typename T, int VL>
__global__ __launch_bounds__(kFewThreads) void few_kernel(const int32_t* __restrict__ ids, int N,
                                                          int64_t V, int32_t pad_id, Grad g,
                                                          int groups, int each) {
    typedef int i4v __attribute__((ext_vector_type(4)));
    extern __shared__ __attribute__((aligned(16))) int32_t all[];  // -1: no row
    __shared__ int32_t found[kFewWaves][kLight], heavy[kFewWaves];
    static_assert(sizeof(found) == 4 * kFewThreads, "a bit for each of 32 rows to a thread");
    __shared__ float part[kFewWaves][kWave * VL];
    const int t = threadIdx.x, lane = t & 63, w = wave_id(), i = blockIdx.x * kFewWaves + w;
    for (int k = t; k < (N + 255) / 256 * 256; k += kFewThreads) {
        const int id = k < N ? ids[k] : -1;
        all[k] = id == pad_id || id < 0 || id >= V ? -1 : id;
    }
    __syncthreads();
    if ((int)blockIdx.x >= groups) {
        if (blockIdx.y == 0)
            clear_others(all, N, (T*)g.dtable, V, g.D, (int64_t)(blockIdx.x - groups) * each, each,
                         (uint32_t*)&found[0][0]);
        return;
    }
    const int col = ((int)blockIdx.y * kWave + lane) * VL;
    const bool live = col < g.D;
    const T* dout = (const T*)g.dout + col;
    const T* table = (const T*)g.dtable + col;
    const uint64_t below = (1ull << lane) - 1;
    const int id = __builtin_amdgcn_readfirstlane(i < N ? all[i] : -1);
    bool first = id >= 0;
    for (int c = 0; first && c < i; c += 256) {  // none before it
        const i4v q = *(const i4v*)(all + c + 4 * lane);
        bool hit = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) hit |= q[e] == id && c + 4 * lane + e < i;
        first = __ballot(hit) == 0;
    }
    int n = 0;
    for (int c = i & ~255; first && n <= kLight && c < N; c += 256) {
        const i4v q = *(const i4v*)(all + c + 4 * lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t m = __ballot(q[e] == id);  // behind the last one is none
            const int at = n + __popcll(m & below);
            if ((m >> lane & 1) && at < kLight) found[w][at] = c + 4 * lane + e;
            n += __popcll(m);
        }
    }
    wave_fence();
    if (lane == 0) heavy[w] = n > kLight ? id : -1;
    float acc[VL] = {}, old[VL] = {};
    if (first && n <= kLight) {
        if (g.add && live) read_row<T, VL>(table + (int64_t)id * g.D, old);
        add_rows<T, VL>(dout, g.D, live, n, [&](int k) { return found[w][k]; }, acc);
        if (live) end_row<T, VL>(g, (uint32_t)id, col, acc, old);
    }
    __syncthreads();
    const int run = ((N + kWave - 1) / kWave + kFewWaves - 1) / kFewWaves * kWave;
    for (int h = 0; h < kFewWaves; ++h) {
        const int item = __builtin_amdgcn_readfirstlane(heavy[h]);
        if (item < 0) continue;
#pragma unroll
        for (int e = 0; e < VL; ++e) acc[e] = 0.0f;
        if (w == 0 && g.add && live) read_row<T, VL>(table + (int64_t)item * g.D, old);
        for (int c = w * run; c < (w + 1) * run && c < N; c += kWave) {
            uint64_t m = __ballot(all[c + lane] == item);
            add_rows<T, VL>(dout, g.D, live, __popcll(m), [&](int) {
                const int at = c + __builtin_ctzll(m);
                m = (m & (m - 1)) ? m & (m - 1) : m;  // the last one stays
                return at;
            }, acc);
        }
#pragma unroll
        for (int e = 0; e < VL; ++e) part[w][lane * VL + e] = acc[e];
        __syncthreads();
        if (w == 0) {
            for (int v = 1; v < kFewWaves; ++v)
#pragma unroll
                for (int e = 0; e < VL; ++e) acc[e] += part[v][lane * VL + e];
            if (live) end_row<T, VL>(g, (uint32_t)item, col, acc, old);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ sorting positions by id
// Where digit d's number lies in LDS: threads walk runs of digits, 16 numbers apart at most.
__host__ __device__ inline int skew(int d) { return d + (d >> 4); }

// 12 bits: 3,416 items in one pass of three launches, a million in two; the counts of eight waves
// still fit LDS (136 KB).
constexpr int kMaxBits = 12, kMaxBins = 1 << kMaxBits;
constexpr int kMaxBlocks = 512;
constexpr int kTile = 2048;  // a block's positions are a multiple of this
constexpr int kPlaceThreads = 512, kWaves = kPlaceThreads / kWave;
constexpr int kEach = kMaxBins / kPlaceThreads;  // digits of a thread

// ids of no row sort behind all others, as V.
__device__ __forceinline__ uint32_t key_of(int32_t id, int64_t V, int32_t pad_id) {
    return id == pad_id || id < 0 || id >= V ? (uint32_t)V : (uint32_t)id;
}

struct Entry {  // 8 bytes together: scattered writes go by their number
    uint32_t key;
    int32_t pos;
};
struct Sort {
    const int32_t* ids;  // the first pass's keys
    const Entry* in;     // later passes'
    Entry* out;
    uint32_t* counts;  // [blocks][bins]
    uint32_t* totals;  // [bins]
    int64_t N, V;
    int64_t each;  // positions to a block
    int blocks, bits, shift;
    int32_t pad_id;
};
__device__ __forceinline__ uint32_t sort_key(const Sort& s, int64_t i) {
    return s.ids ? key_of(s.ids[i], s.V, s.pad_id) : s.in[i].key;
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
    constexpr int B = kTile / kNT;
    const int64_t from = blockIdx.x * s.each + threadIdx.x;
    const int64_t to = min(s.N, (int64_t)(blockIdx.x + 1) * s.each);
    for (int i = threadIdx.x; i < n; i += kNT) bins[i] = 0;
    for (int64_t i0 = from; i0 - threadIdx.x < to; i0 += B * kNT) {
        uint32_t keys[B];
#pragma unroll
        for (int j = 0; j < B; ++j)
            if (i0 + j * kNT < to) keys[j] = sort_key(s, i0 + j * kNT);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < B; ++j)
            if (i0 + j * kNT < to) atomicAdd(&bins[keys[j] >> s.shift & (n - 1)], 1u);
    }
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

// The lanes that have this lane's digit, of kBits bits, among the live ones.
template <int kBits>
__device__ __forceinline__ uint64_t alike(uint32_t d, bool live) {
    const uint64_t all = __ballot(live);
    uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
#pragma unroll
    for (int b = 0; b < kBits; ++b) {
        const uint32_t x = (uint32_t)((int32_t)(d << (31 - b)) >> 31);  // the bit in every place
        const uint64_t m = __ballot(x != 0);
        lo &= ~((uint32_t)m ^ x);
        hi &= ~((uint32_t)(m >> 32) ^ x);
    }
    return (uint64_t)hi << 32 | lo;
}

// kBits: s.bits or more.  200 blocks of 2,048 positions and 4,096 digits in 13 us: first reads,
// the digits' counts of eight waves in LDS, ranks and scattered writes, a third each.
template <int kBits>
__global__ __launch_bounds__(kPlaceThreads) void place_kernel(Sort s) {
    constexpr int TH = kPlaceThreads, B = kTile / (kWaves * kWave);  // positions read together
    extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
    __shared__ uint32_t wsum[TH / kWave];
    const int n = 1 << s.bits, t = threadIdx.x, lane = t & 63, w = wave_id();
    const int room = skew(n);
    uint32_t* next = lds + w * room;  // the wave's next places
    const uint64_t below = (1ull << lane) - 1;
    // A wave's positions are one run of its block's.
    const int64_t from = blockIdx.x * s.each + w * (s.each / kWaves) + lane;
    const int64_t to = min(s.N, from - lane + s.each / kWaves);
    uint32_t keys[B];
#pragma unroll
    for (int j = 0; j < B; ++j) keys[j] = from + j * kWave < to ? sort_key(s, from + j * kWave) : 0;
    // A thread's digits: the block's first places within them, and all of them.
    const int run = (n + TH - 1) / TH;
    const uint32_t* counts = s.counts + (int64_t)blockIdx.x * n;
    uint32_t first[kEach], total[kEach], mine = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const bool in = k < run && t * run + k < n;
        first[k] = in ? counts[t * run + k] : 0;
        total[k] = in ? s.totals[t * run + k] : 0;
    }
    for (int i = 4 * t; i < kWaves * room; i += 4 * TH) *(u4v*)(lds + i) = u4v{0, 0, 0, 0};
    __syncthreads();
#pragma unroll
    for (int j = 0; j < B; ++j)
        if (from + j * kWave < to) atomicAdd(&next[skew(keys[j] >> s.shift & (n - 1))], 1u);
    for (int64_t i = from + B * kWave; i < to; i += kWave)
        atomicAdd(&next[skew(sort_key(s, i) >> s.shift & (n - 1))], 1u);
    // Digits before a thread's run of digits, then each digit's first place for each wave.
#pragma unroll
    for (int k = 0; k < kEach; ++k) mine += total[k];
    const uint32_t upto = lanes::wave_scan(mine, 0u, [](uint32_t a, uint32_t b) { return a + b; });
    if (lane == kWave - 1) wsum[w] = upto;
    __syncthreads();
    uint32_t at = upto - mine;
    for (int k = 0; k < w; ++k) at += wsum[k];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        if (k >= run || t * run + k >= n) break;
        const int d = skew(t * run + k);
        uint32_t c[kWaves], place = at + first[k];
#pragma unroll
        for (int v = 0; v < kWaves; ++v) c[v] = lds[v * room + d];
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            lds[v * room + d] = place;
            place += c[v];
        }
        at += total[k];
    }
    __syncthreads();
    for (int64_t i0 = from; i0 - lane < to; i0 += B * kWave) {
        int32_t pos[B];
        if (i0 != from) {
#pragma unroll
            for (int j = 0; j < B; ++j)
                keys[j] = i0 + j * kWave < to ? sort_key(s, i0 + j * kWave) : 0;
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int64_t i = i0 + j * kWave;
            pos[j] = !s.ids && i < to ? s.in[i].pos : (int32_t)i;
        }
        uint64_t same[B];
#pragma unroll
        for (int j = 0; j < B; ++j)
            same[j] = alike<kBits>(keys[j] >> s.shift & (n - 1), i0 + j * kWave < to);
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int slot = skew(keys[j] >> s.shift & (n - 1));
            if (i0 + j * kWave < to) {
                const uint32_t place = next[slot] + __popcll(same[j] & below);
                wave_fence();
                if ((same[j] >> lane) == 1ull) next[slot] = place + 1;  // the last of its digit
                s.out[place] = Entry{keys[j], pos[j]};
            }
            wave_fence();
        }
    }
}

// ------------------------------------------------------------------ sums of runs
constexpr int kSumWaves = 16, kSumThreads = kSumWaves * kWave;
constexpr int kPiece = 64, kGroup = kSumWaves * kPiece;  // positions to a wave, to a workgroup

// Eight waves to a SIMD: 409,600 rows of 64 fp32 in 20 us, 5.3 TB/s.
// part: for each workgroup, the sum of a run that came from before it (slot 0) and of one that
// starts in it and goes on (slot 1).
template <typename T, int VL>
__global__ __launch_bounds__(kSumThreads, 8) void sum_kernel(const Entry* __restrict__ sorted,
                                                          int64_t N, int64_t V, Grad g,
                                                          float* part) {
    // Of each wave the same two sums, and whether it has them: 1 a run from before that ends here,
    // 2 one that passes through, 4 one that starts here and goes on.
    __shared__ float kept[kSumWaves][2][kWave * VL];
    __shared__ int kinds[kSumWaves];
    const int lane = threadIdx.x & 63, w = wave_id();
    const int64_t from = (int64_t)blockIdx.x * kGroup + w * kPiece, i = from + lane;
    const uint32_t none = (uint32_t)V;
    const Entry mine = i < N ? sorted[i] : Entry{none, 0};
    const uint32_t key = mine.key;
    const uint32_t after = i + 1 < N ? sorted[i + 1].key : none;
    const int at = mine.pos;
    const uint32_t before = from > 0 && from <= N ? sorted[from - 1].key : none;
    const int live = __popcll(__ballot(key != none));  // sorted: the first ones
    const uint64_t ends = __ballot(key != after);
    bool earlier = live > 0 && lanes::lane_of(key, 0) == before;  // the run came from before
    int kind = 0;
    const int col = ((int)blockIdx.y * kWave + lane) * VL;
    const bool in = col < g.D;
    const T* dout = (const T*)g.dout + col;
    T* dtable = (T*)g.dtable + col;
    float acc[VL] = {};
    // Rows of eight positions, and what is there already of the items that end among them, are read
    // before the eight before them are summed and written: reads issued behind a write would be
    // waited for together with it.
    constexpr int B = sizeof(RawRow<T, VL>) <= 4 ? 8 : 32 / (int)sizeof(RawRow<T, VL>);
    struct Rows {  // as they lie in memory: as floats, bf16 rows would halve the waves that fit
        RawRow<T, VL> v[B], old[B];
    };
    auto fetch = [&](Rows& x, int j0) {
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int r = __builtin_amdgcn_readlane(at, (j0 + j) & 63);  // behind the last one: any
            if (in) x.v[j] = raw_row<T, VL>(dout + (int64_t)r * g.D);
        }
        if (g.add)
#pragma unroll
            for (int j = 0; j < B; ++j)
                if (j0 + j < live && (ends >> (j0 + j) & 1) && in)
                    x.old[j] = raw_row<T, VL>(dtable +
                                              (int64_t)lanes::lane_of(key, j0 + j) * g.D);
    };
    auto use = [&](const Rows& x, int j0) {
#pragma unroll
        for (int j = 0; j < B; ++j) {
            if (j0 + j >= live) break;
            float v[VL];
            unpack_vec<T, VL>(x.v[j], v);
#pragma unroll
            for (int e = 0; e < VL; ++e) acc[e] += v[e];
            if (ends >> (j0 + j) & 1) {
                if (earlier) {
                    kind |= 1;
#pragma unroll
                    for (int e = 0; e < VL; ++e) kept[w][0][lane * VL + e] = acc[e];
                } else if (in) {
                    unpack_vec<T, VL>(x.old[j], v);
                    end_row<T, VL>(g, lanes::lane_of(key, j0 + j), col, acc, v);
                }
                earlier = false;
#pragma unroll
                for (int e = 0; e < VL; ++e) acc[e] = 0.0f;
            }
        }
    };
    Rows even, odd;
    if (live > 0) fetch(even, 0);
    for (int j0 = 0; j0 < live; j0 += 2 * B) {
        if (j0 + B < live) fetch(odd, j0 + B);
        use(even, j0);
        if (j0 + 2 * B < live) fetch(even, j0 + 2 * B);
        use(odd, j0 + B);
    }
    if (live == kPiece && !(ends >> 63)) {  // goes on
        kind |= earlier ? 2 : 4;
#pragma unroll
        for (int e = 0; e < VL; ++e) kept[w][earlier ? 0 : 1][lane * VL + e] = acc[e];
    }
    if (lane == 0) kinds[w] = kind;
    __syncthreads();
    // A wave joins the run that starts in it, the first one also the run that came from before.
    const auto join = [&](int u, bool goes, float* slot) {  // from wave u on, acc holds what is before
        for (; goes && u < kSumWaves; ++u) {
#pragma unroll
            for (int e = 0; e < VL; ++e) acc[e] += kept[u][0][lane * VL + e];
            goes = kinds[u] & 2;
        }
        if (goes) {
            if (in)
#pragma unroll
                for (int e = 0; e < VL; ++e) slot[e] = acc[e];
        }
        return goes;
    };
    float* slot = part + (int64_t)blockIdx.x * 2 * g.D + col;
    if (kind & 4) {
        const uint32_t k = lanes::lane_of(key, kPiece - 1);
        float old[VL];
        if (g.add && in) read_row<T, VL>(dtable + (int64_t)k * g.D, old);
#pragma unroll
        for (int e = 0; e < VL; ++e) acc[e] = kept[w][1][lane * VL + e];
        if (!join(w + 1, true, slot + g.D) && in) end_row<T, VL>(g, k, col, acc, old);
    }
    if (w == 0 && (kinds[0] & 3)) {
#pragma unroll
        for (int e = 0; e < VL; ++e) acc[e] = 0.0f;
        if (!join(0, true, slot) && in)
#pragma unroll
            for (int e = 0; e < VL; ++e) slot[e] = acc[e];
    }
}

constexpr int kJoin = 512;

// The workgroup of the group in which a run starts that goes on: its parts in eight runs of
// groups, then these in order.
template <typename T, int VL>
__global__ __launch_bounds__(kJoin) void join_kernel(const Entry* __restrict__ sorted, int64_t N,
                                                     int64_t V, Grad g, const float* part,
                                                     int64_t groups) {
    constexpr int W = kJoin / kWave;
    __shared__ float all[W][kWave * VL];
    const int64_t p = blockIdx.x, last = p * kGroup + kGroup - 1;
    if (last + 1 >= N) return;
    const uint32_t k = sorted[last].key;
    if (k == (uint32_t)V || sorted[last + 1].key != k) return;
    if (sorted[p * kGroup].key == k && p > 0 && sorted[p * kGroup - 1].key == k)
        return;  // from before
    // The last group whose first key is k: ever larger steps, then halves.
    int64_t lo = p + 1, step = 1;
    while (lo + step < groups && sorted[(lo + step) * kGroup].key == k) {
        lo += step;
        step *= 2;
    }
    int64_t hi = min(groups, lo + step);  // k at lo * kGroup, and not at hi
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if (sorted[mid * kGroup].key == k) lo = mid;
        else hi = mid;
    }
    const int lane = threadIdx.x & 63, w = wave_id();
    const int col = ((int)blockIdx.y * kWave + lane) * VL;
    const bool in = col < g.D;
    const int64_t n = lo - p, run = n <= 16 ? n : (n + W - 1) / W;
    float acc[VL] = {}, old[VL] = {};
    if (in) {
        if (w == 0) {
            if (g.add) read_row<T, VL>((const T*)g.dtable + (int64_t)k * g.D + col, old);
#pragma unroll
            for (int e = 0; e < VL; ++e) acc[e] = part[(p * 2 + 1) * g.D + col + e];
        }
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
    if (w == 0 && in) end_row<T, VL>(g, k, col, acc, old);
}

// ------------------------------------------------------------------ launches
struct Plan {
    int passes, bits, blocks;
    int64_t each, groups;
    size_t entries[2], counts, totals, part, bytes;
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
    p.groups = (N + kGroup - 1) / kGroup;
    size_t at = 0;
    for (int i = 0; i < (p.passes > 1 ? 2 : 1); ++i) {
        p.entries[i] = at;
        at += up((size_t)N * sizeof(Entry));
    }
    p.counts = at;
    at += up(((size_t)p.blocks << p.bits) * 4);
    p.totals = at;
    at += up((size_t)4 << p.bits);
    p.part = at;
    at += up((size_t)p.groups * 2 * D * 4);
    p.bytes = at;
    return p;
}

int place_lds(int bits) { return kWaves * skew(1 << bits) * 4; }

template <int kBits>
hipError_t launch_place(const Sort& s, hipStream_t st) {
    static std::atomic<uint64_t> done{0};
    const hipError_t e =
        allow_dynamic_lds((const void*)place_kernel<kBits>, place_lds(kBits), done);
    if (e != hipSuccess) return e;
    place_kernel<kBits><<<dim3((unsigned)s.blocks), kPlaceThreads, place_lds(s.bits), st>>>(s);
    return hipGetLastError();
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
        const int groups = (int)((a.N + kFewWaves - 1) / kFewWaves);
        // Rows that a workgroup clears: 512 of them, of 16 to 256 KB each.
        const int64_t row = a.D * (int64_t)sizeof(T);
        int64_t each = std::min<int64_t>(std::max<int64_t>(a.V * row / 512, 16384), 262144) / row;
        each = std::min<int64_t>(std::max<int64_t>(each, 1), 32 * kFewThreads);
        const int64_t clears = a.accumulate ? 0 : (a.V + each - 1) / each;
        few_kernel<T, VL><<<dim3((unsigned)(groups + clears), cols), kFewThreads,
                            (size_t)(a.N + 255) / 256 * 1024, st>>>(a.ids, (int)a.N, a.V, a.pad_id,
                                                                    g, groups, (int)each);
        return;
    }
    const int last = (pl.passes + 1) % 2;  // passes write buffers 0, 1, 0, ...
    const Entry* sorted = (const Entry*)(ws + pl.entries[last]);
    float* part = (float*)(ws + pl.part);
    const dim3 grid((unsigned)pl.groups, cols);
    sum_kernel<T, VL><<<grid, kSumThreads, 0, st>>>(sorted, a.N, a.V, g, part);
    join_kernel<T, VL><<<grid, kJoin, 0, st>>>(sorted, a.N, a.V, g, part, pl.groups);
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
    if (a.N == 0 && fill > 0) count_kernel<<<dim3((unsigned)fill), kNT, 0, st>>>(s, a.dst, bytes);
    for (int i = 0; !few && i < pl.passes; ++i) {
        s.ids = i ? nullptr : a.ids;
        s.in = (const Entry*)(w + pl.entries[(i + 1) % 2]);
        s.out = (Entry*)(w + pl.entries[i % 2]);
        s.counts = (uint32_t*)(w + pl.counts);
        s.totals = (uint32_t*)(w + pl.totals);
        s.blocks = pl.blocks;
        s.bits = pl.bits;
        s.shift = i * pl.bits;
        const int64_t zeros = i ? 0 : fill;
        count_kernel<<<dim3((unsigned)(pl.blocks + zeros)), kNT, 0, st>>>(s, a.dst, bytes);
        offsets_kernel<<<dim3((unsigned)(((1 << pl.bits) + 63) / 64)), 1024, 0, st>>>(s);
        const hipError_t e = pl.bits <= 6   ? launch_place<6>(s, st)
                             : pl.bits <= 9 ? launch_place<9>(s, st)
                                            : launch_place<kMaxBits>(s, st);
        if (e != hipSuccess) return e;
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
