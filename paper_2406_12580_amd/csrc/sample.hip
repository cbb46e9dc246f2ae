// One item a row from logits (recblr_sample): temperature, top-k, top-p, min-p.
//
// The items that stay are a run of the order (logit falling, index rising), so a row's
// selection is one border: a key, and how many of the items with that very key stay; nothing
// is sorted.  Weights w = exp((l - max) / temperature) are formed in 64 bits and summed as
// integers q = round(w 2^F): such sums are exact in any order, so atomics repeat bit for bit
// and a border falls where 64-bit arithmetic puts it.  Items with q = 0 can neither be chosen
// nor move a border that matters; they take no part.
//
// The border is found on a histogram of counts and weights over kBins equal steps of the logit
// (uniform steps spread the items of usual logits evenly; the bits of a float do not: its
// upper eleven put half of a row in twenty bins, whose atomics then wait for each other).  The
// bin that holds the border is searched further by its keys' own bits, 8 at a time, until one
// key is left; equal keys (frequent in bf16) are one key from the start.
//
// A row of up to kSpan items is one workgroup's, keys and weights in its registers from a
// single read.  A longer one takes a workgroup for each span of kSpan items and six short
// launches: extremes, histogram, the items of the bins that can hold a border, the border
// itself (on those items alone), sums of the spans, and the choice within one span.
#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "ops.hpp"

namespace recblr {
namespace {

constexpr int kNT = 256;
constexpr int kNW = kNT / kWave;
constexpr int kIT = 4;                 // groups of four items to a lane
constexpr int kItems = 4 * kIT;
constexpr int kSpan = kNT * kItems;    // items of a workgroup
constexpr int kBins = 1024;
constexpr int kBPT = kBins / kNT;
constexpr int kFine = 256;             // bins of the further searches

// Order-preserving bits of a float: equal floats (the two zeros among them) have equal keys.
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
constexpr uint32_t kKeyNegInf = 0x007FFFFFu;  // key_of(-inf); a NaN's key lies outside
constexpr uint32_t kKeyPosInf = 0xFF800000u;  // [key_of(-inf), key_of(+inf)]; 0 is no item's

template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
// Sum over the lanes below this one.
template <typename V>
__device__ __forceinline__ V wave_before(V v, int lane) {
    V s = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const V o = __shfl_up(s, d);
        if (lane >= d) s += o;
    }
    return s - v;
}

typedef unsigned long long u64;

// e^x for x in [-46, 0]: x = n ln 2 + t with |t| <= ln 2 / 2, and e^t by its Taylor polynomial
// of degree 12, whose remainder is below 2e-16 of it.
__device__ __forceinline__ double exp_neg(double x) {
    const double n = __builtin_rint(x * 1.4426950408889634074);
    // ln 2 as its nearest double and what that leaves.
    double t = __builtin_fma(n, -0.69314718055994530942, x);
    t = __builtin_fma(n, -2.3190468138462996e-17, t);
    double p = 1.0 / 479001600.0;
    p = __builtin_fma(p, t, 1.0 / 39916800.0);
    p = __builtin_fma(p, t, 1.0 / 3628800.0);
    p = __builtin_fma(p, t, 1.0 / 362880.0);
    p = __builtin_fma(p, t, 1.0 / 40320.0);
    p = __builtin_fma(p, t, 1.0 / 5040.0);
    p = __builtin_fma(p, t, 1.0 / 720.0);
    p = __builtin_fma(p, t, 1.0 / 120.0);
    p = __builtin_fma(p, t, 1.0 / 24.0);
    p = __builtin_fma(p, t, 1.0 / 6.0);
    p = __builtin_fma(p, t, 0.5);
    p = __builtin_fma(p, t, 1.0);
    p = __builtin_fma(p, t, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}

// The nearest integer of x in [0, 2^51]: 2^52 + x has it in its lowest bits.
__device__ __forceinline__ u64 rounded(double x) {
    return (u64)__double_as_longlong(x + 0x1p52) & 0xFFFFFFFFFFFFFull;
}

// What a row asks for, and the measures that its extremes give.
struct Row {
    double inv_t, max, scale;
    float top, bins;     // largest logit; bins to a unit of the logit
    float top_p, min_p;
    int64_t k;
    bool bad, greedy;
    uint32_t hi;

    // Of a row whose largest and smallest keys are hi and lo.
    __device__ __forceinline__ Row(const SampleArgs& a, int64_t row, uint32_t hi_, uint32_t lo,
                                   double scale_) {
        hi = hi_;
        scale = scale_;
        const float temp = a.temperature ? a.temperature[row] : 1.0f;
        bad = hi <= kKeyNegInf || hi >= kKeyPosInf || lo < kKeyNegInf || !(temp == temp);
        top_p = a.top_p ? a.top_p[row] : 1.0f;
        min_p = a.min_p ? fminf(a.min_p[row], 1.0f) : 0.0f;
        greedy = temp <= 0.0f;
        k = a.top_k && a.top_k[row] > 0 ? a.top_k[row] : a.V;
        if (greedy || top_p <= 0.0f) k = 1;
        inv_t = greedy ? 0.0 : 1.0 / (double)temp;
        top = value_of(hi);
        max = (double)top;
        const float range = fminf(46.0f * temp, top - value_of(lo < kKeyNegInf ? hi : lo));
        bins = range > 0.0f && range < 3e38f ? (float)(kBins - 1) / range : 0.0f;
    }
    __device__ __forceinline__ double weight(uint32_t key) const {
        // What lies further down than 46 temperatures (-inf and what is no item among it) weighs
        // e^-46, which no scale up to 2^51 brings to a half.
        return exp_neg(fmax(((double)value_of(key) - max) * inv_t, -46.0));
    }
    __device__ __forceinline__ u64 fixed(uint32_t key) const { return rounded(weight(key) * scale); }
    // Rising as the logit falls: both roundings keep the order.
    __device__ __forceinline__ int bin(uint32_t key) const {
        const float b = (top - value_of(key)) * bins;
        return b < (float)(kBins - 1) ? (int)b : kBins - 1;
    }
    // Whether a border has to be looked for.
    __device__ __forceinline__ bool cuts(int64_t V) const { return k < V || top_p < 1.0f; }
};

struct Border {
    uint32_t key;   // items above it stay,
    uint32_t ties;  // and the first `ties` of those that have it
};

struct Shared {
    uint32_t cnt[kBins];
    u64 mass[kBins];
    uint32_t fine_cnt[kFine];
    u64 fine_mass[kFine];
    uint32_t w32[2][kNW];
    u64 w64[kNW];
    uint32_t lo, hi;
    int at;             // bin found
    uint32_t at_cnt, above_cnt;
    u64 above_mass, at_mass;
};

// Workgroup sums of a count and a weight over lower threads.
__device__ __forceinline__ void block_before(Shared& sm, uint32_t& c, u64& m, int lane, int w) {
    const uint32_t c0 = c;
    const u64 m0 = m;
    c = wave_before(c, lane);
    m = wave_before(m, lane);
    if (lane == kWave - 1) {
        sm.w32[0][w] = c + c0;
        sm.w64[w] = m + m0;
    }
    __syncthreads();
    for (int i = 0; i < w; ++i) {
        c += sm.w32[0][i];
        m += sm.w64[i];
    }
}

// The last bin that holds items and has less than is wanted before it: fewer than want_cnt
// items, or a weight below want_mass.  `cnt`, `mass`: N bins in LDS, N / kNT of them to a
// thread in order, with c and m before the thread's first (whole arrays, base included).
template <int N>
__device__ __forceinline__ void pick(Shared& sm, const uint32_t* cnt, const u64* mass, uint32_t c,
                                     u64 m, bool by_mass, uint64_t want_cnt, double want_mass,
                                     int tid) {
    constexpr int BPT = N / kNT;
    if (tid == 0) sm.at = -1;
    __syncthreads();
    int mine = -1;
    uint32_t c_at = 0;
    u64 m_at = 0;
#pragma unroll
    for (int j = 0; j < BPT; ++j) {
        const int b = tid * BPT + j;
        const uint32_t n = cnt[b];
        if (n && (by_mass ? (double)m < want_mass : c < want_cnt)) {
            mine = b;
            c_at = c;
            m_at = m;
        }
        c += n;
        m += mass[b];
    }
    if (mine >= 0) atomicMax(&sm.at, mine);
    __syncthreads();
    if (mine >= 0 && sm.at == mine) {
        sm.above_cnt = c_at;
        sm.above_mass = m_at;
        sm.at_cnt = cnt[mine];
        sm.at_mass = mass[mine];
    }
    __syncthreads();
}

// How many of `ties` items of weight q stay when `before` lies above them and less than `want`
// may lie before one that stays.
__device__ __forceinline__ uint32_t ties_within(uint32_t ties, u64 q, u64 before, double want) {
    if (q == 0) return ties;
    const double guess = ceil((want - (double)before) / (double)q);
    int64_t n = guess < 1.0 ? 1 : guess > (double)ties ? (int64_t)ties : (int64_t)guess;
    while (n > 1 && !((double)(before + q * (u64)(n - 1)) < want)) --n;
    while (n < (int64_t)ties && (double)(before + q * (u64)n) < want) ++n;
    return (uint32_t)n;
}

// Searches one bin further.  each(f) calls f(key, q) for the items that may be of it, member()
// tells which are; `above` of sm is what lies before the bin and is brought to what lies before
// the key found, which has sm.at_cnt items.
template <typename Each, typename Member>
__device__ __forceinline__ uint32_t refine(Shared& sm, const Row& row, Each each, Member member,
                                           bool by_mass, uint64_t want_cnt, double want_mass,
                                           int tid, int lane, int w) {
    uint32_t from = 0, to = 0xFFFFFFFFu;
    uint32_t base_c = sm.above_cnt;
    u64 base_m = sm.above_mass;
    // Each search leaves at most a 128th of the keys' range: five come down to one key.
    for (int depth = 0; depth < 8; ++depth) {
        __syncthreads();
        if (tid == 0) {
            sm.lo = 0xFFFFFFFFu;
            sm.hi = 0;
        }
        for (int b = tid; b < kFine; b += kNT) {
            sm.fine_cnt[b] = 0;
            sm.fine_mass[b] = 0;
        }
        __syncthreads();
        uint32_t lo = 0xFFFFFFFFu, hi = 0;
        each([&](uint32_t key, u64 q) {
            const bool in = (q != 0) & (key >= from) & (key <= to) & member(key);
            lo = in && key < lo ? key : lo;
            hi = in && key > hi ? key : hi;
        });
        if (lo <= hi) {
            atomicMin(&sm.lo, lo);
            atomicMax(&sm.hi, hi);
        }
        __syncthreads();
        lo = sm.lo;
        hi = sm.hi;
        if (lo > hi) break;
        const int bits = 32 - __clz((int)((hi - lo) | 1u));
        const int shift = bits > 8 ? bits - 8 : 0;
        each([&](uint32_t key, u64 q) {
            if ((q != 0) & (key >= lo) & (key <= hi) & member(key)) {
                const uint32_t b = (hi - key) >> shift;
                atomicAdd(&sm.fine_cnt[b], 1u);
                atomicAdd(&sm.fine_mass[b], q);
            }
        });
        __syncthreads();
        uint32_t c = sm.fine_cnt[tid];
        u64 m = sm.fine_mass[tid];
        block_before(sm, c, m, lane, w);
        pick<kFine>(sm, sm.fine_cnt, sm.fine_mass, c + base_c, m + base_m, by_mass, want_cnt,
                    want_mass, tid);
        if (sm.at < 0) break;
        const uint32_t b = (uint32_t)sm.at;
        base_c = sm.above_cnt;
        base_m = sm.above_mass;
        to = hi - (b << shift);
        from = to - ((1u << shift) - 1) < lo || to < ((1u << shift) - 1) ? lo
                                                                         : to - ((1u << shift) - 1);
        if (from == to) break;
    }
    return to;
}

// The row's border, from the whole histogram in sm (items with q > 0) and the items of the bins
// that may hold it.  All threads return the same.
template <typename Each>
__device__ __forceinline__ Border find_border(Shared& sm, const Row& row, Each each, int tid,
                                              int lane, int w) {
    uint32_t c = 0;
    u64 m = 0;
#pragma unroll
    for (int j = 0; j < kBPT; ++j) {
        c += sm.cnt[tid * kBPT + j];
        m += sm.mass[tid * kBPT + j];
    }
    const uint32_t c0 = c;
    const u64 m0 = m;
    block_before(sm, c, m, lane, w);
    // Totals stand behind the last thread's bins.
    if (tid == kNT - 1) {
        sm.lo = c + c0;
        sm.at_mass = m + m0;
    }
    __syncthreads();
    const uint32_t total = sm.lo;
    u64 above = sm.at_mass;
    __syncthreads();
    Border b{0, 0};
    u64 tie_q = 0;
    if (row.k < (int64_t)total) {
        pick<kBins>(sm, sm.cnt, sm.mass, c, m, false, (uint64_t)row.k, 0.0, tid);
        const int bin = sm.at;
        b.key = refine(sm, row, each, [&](uint32_t key) { return row.bin(key) == bin; }, false,
                       (uint64_t)row.k, 0.0, tid, lane, w);
        b.ties = (uint32_t)(row.k - sm.above_cnt);
        above = sm.above_mass;
        tie_q = row.fixed(b.key);
    }
    if (row.top_p < 1.0f && row.k > 1) {
        const double want = (double)row.top_p * (double)(above + tie_q * (u64)b.ties);
        if ((double)above < want) {
            if (b.ties) b.ties = ties_within(b.ties, tie_q, above, want);
        } else {
            const uint32_t edge = b.key;
            pick<kBins>(sm, sm.cnt, sm.mass, c, m, true, 0, want, tid);
            const int bin = sm.at;
            b.key = refine(sm, row, each,
                           [&](uint32_t key) { return (key > edge) & (row.bin(key) == bin); }, true,
                           0, want, tid, lane, w);
            b.ties = ties_within(sm.at_cnt, row.fixed(b.key), sm.above_mass, want);
        }
    }
    return b;
}

// A span of a row: its keys in order, a wave's 1024 after another's, groups of four to a lane.
template <typename T>
struct Span {
    uint32_t key[kItems];
    __device__ __forceinline__ static int64_t index(int64_t base, int w, int it, int lane) {
        return base + (w * kIT + it) * 256 + lane * 4;
    }
    __device__ __forceinline__ Span(const T* p, int64_t V, int64_t base, int w, int lane) {
        const bool vec = ((uintptr_t)p) % (4 * sizeof(T)) == 0;
#pragma unroll
        for (int it = 0; it < kIT; ++it) {
            const int64_t i = index(base, w, it, lane);
            if (vec && i + 4 <= V) {
                float v[4];
                unpack_vec<T, 4>(*(const typename VecT<T, 4>::type*)(p + i), v);
#pragma unroll
                for (int e = 0; e < 4; ++e) key[4 * it + e] = key_of(v[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    key[4 * it + e] = i + e < V ? key_of(to_f32(p[i + e])) : 0u;
            }
        }
    }
    // Largest and smallest key over the workgroup's items, by all threads; w32 of LDS.
    __device__ __forceinline__ void extremes(uint32_t (&w32)[2][kNW], int w, int lane, uint32_t& hi,
                                             uint32_t& lo) const {
        // What is no item has key 0, which as the smallest wraps to the largest.
        hi = 0;
        lo = 0xFFFFFFFFu;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            hi = key[i] > hi ? key[i] : hi;
            lo = key[i] - 1u < lo ? key[i] - 1u : lo;
        }
        lo = lo == 0xFFFFFFFFu ? lo : lo + 1u;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const uint32_t h = (uint32_t)__shfl_xor((int)hi, d), l = (uint32_t)__shfl_xor((int)lo, d);
            hi = h > hi ? h : hi;
            lo = l < lo ? l : lo;
        }
        if (lane == 0) {
            w32[0][w] = hi;
            w32[1][w] = lo;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kNW; ++i) {
            hi = w32[0][i] > hi ? w32[0][i] : hi;
            lo = w32[1][i] < lo ? w32[1][i] : lo;
        }
    }
};

// The choice within a span whose first item has `before` items of the border's key and a sum of
// `run0` before it.  q of items that stay is left, others' become 0.
template <typename T>
__device__ __forceinline__ void keep(const Span<T>& sp, const Row& row, const Border& b,
                                     uint64_t before, u64 (&q)[kItems], int lane) {
#pragma unroll
    for (int it = 0; it < kIT; ++it) {
        uint32_t tie[4], n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            tie[e] = sp.key[4 * it + e] == b.key && b.key != 0;
            n += tie[e];
        }
        uint64_t mine = 0;
        if (__any((int)n)) {
            const uint32_t lower = wave_before(n, lane);
            mine = before + lower;
            before += (uint32_t)__shfl((int)(lower + n), kWave - 1);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!(sp.key[4 * it + e] > b.key || (tie[e] && mine < b.ties))) q[4 * it + e] = 0;
            mine += tie[e];
        }
    }
}

// A wave's items of the border's key.
template <typename T>
__device__ __forceinline__ uint32_t wave_ties(const Span<T>& sp, const Border& b) {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) n += sp.key[i] == b.key && b.key != 0;
    return wave_sum(n);
}

// The weights of a row's items: min-p's are 0 as well (in a greedy row all weigh the same).
__device__ __forceinline__ u64 weight_of(const Row& row, uint32_t key) {
    if (row.greedy) return key > kKeyNegInf ? (u64)row.scale : 0;
    const double wt = row.weight(key);
    return wt < (double)row.min_p ? 0 : rounded(wt * row.scale);
}

// The item at which the running sum, `run0` before the wave's first item, first exceeds target,
// else the wave's last one with weight; written by the lane that has it.
template <typename T>
__device__ __forceinline__ void choose(const SampleArgs& a, const Span<T>& sp, const Row& row,
                                       const u64 (&q)[kItems], int64_t r, int64_t base, u64 run,
                                       double target, u64 all, int w, int lane) {
    int64_t found = -1, tail = -1;
    uint32_t key_f = 0, key_t = 0;
#pragma unroll
    for (int it = 0; it < kIT; ++it) {
        const u64 own = q[4 * it] + q[4 * it + 1] + q[4 * it + 2] + q[4 * it + 3];
        u64 c = run + wave_before(own, lane);
        run += wave_sum(own);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c += q[4 * it + e];
            if (q[4 * it + e]) {
                tail = Span<T>::index(base, w, it, lane) + e;
                key_t = sp.key[4 * it + e];
                if (found < 0 && (double)c > target) {
                    found = tail;
                    key_f = key_t;
                }
            }
        }
    }
    u64 best = found >= 0 ? (u64)found : ~0ull;
    long long end = (long long)tail;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const u64 o = __shfl_xor(best, d);
        const long long t = __shfl_xor(end, d);
        best = o < best ? o : best;
        end = t > end ? t : end;
    }
    const bool got = best != ~0ull;
    const int64_t id = got ? (int64_t)best : (int64_t)end;
    if (got ? found == id : tail == id) {
        a.ids[r] = (int32_t)id;
        const double wt = row.greedy ? 1.0 : row.weight(got ? key_f : key_t);
        if (a.prob) a.prob[r] = (float)(wt * row.scale / (double)all);
    }
}

__device__ __forceinline__ void none(const SampleArgs& a, int64_t r) {
    a.ids[r] = -1;
    if (a.prob) a.prob[r] = 0.0f;
}

// Which of n consecutive parts holds the choice: the first whose running sum exceeds the
// target, the last one with weight if none does.  Whether a part with `sum`, `from` before it,
// is the one (u below 0 takes the first part with weight).
__device__ __forceinline__ bool is_part(u64 from, u64 sum, u64 all, double target, bool is_last) {
    if (!((double)all > target)) return is_last;
    if (sum == 0 || !((double)(from + sum) > target)) return false;
    return !((double)from > target) || from == 0;
}

// ------------------------------------------------------------------ a row in one workgroup
template <typename T>
__global__ __launch_bounds__(kNT, 3) void sample_row_kernel(SampleArgs a, double scale) {
    __shared__ Shared sm;
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x;
    const Span<T> sp((const T*)a.logits + r * a.V, a.V, 0, w, lane);
    for (int b = tid; b < kBins; b += kNT) {
        sm.cnt[b] = 0;
        sm.mass[b] = 0;
    }
    uint32_t hi, lo;
    sp.extremes(sm.w32, w, lane, hi, lo);
    const Row row(a, r, hi, lo, scale);
    if (row.bad) {
        if (tid == 0) none(a, r);
        return;
    }
    u64 q[kItems];
    Border b{0, 0};
    if (row.k == 1) {
        b = Border{hi, 1};
#pragma unroll
        for (int i = 0; i < kItems; ++i) q[i] = sp.key[i] == hi ? (u64)scale : 0;
    } else {
#pragma unroll
        for (int i = 0; i < kItems; ++i) q[i] = row.fixed(sp.key[i]);
        if (row.cuts(a.V)) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (q[i]) {
                    const int bin = row.bin(sp.key[i]);
                    atomicAdd(&sm.cnt[bin], 1u);
                    atomicAdd(&sm.mass[bin], q[i]);
                }
            __syncthreads();
            auto each = [&](auto f) {
#pragma unroll
                for (int i = 0; i < kItems; ++i) f(sp.key[i], q[i]);
            };
            b = find_border(sm, row, each, tid, lane, w);
        }
        if (row.min_p > 0.0f) {
            // As weight_of, by the weight itself; its q tells unless it is next to min_p's.
            const u64 least = rounded((double)row.min_p * scale);
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                if (q[i] < least) q[i] = 0;
                else if (q[i] <= least + 1 && row.weight(sp.key[i]) < (double)row.min_p) q[i] = 0;
            }
        }
    }
    __syncthreads();
    const uint32_t ties = wave_ties(sp, b);
    if (lane == 0) sm.w32[0][w] = ties;
    __syncthreads();
    uint64_t before = 0;
    for (int i = 0; i < w; ++i) before += sm.w32[0][i];
    keep(sp, row, b, before, q, lane);
    u64 sum = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) sum += q[i];
    sum = wave_sum(sum);
    if (lane == 0) sm.w64[w] = sum;
    __syncthreads();
    u64 all = 0, from = 0;
    int last = 0;
#pragma unroll
    for (int i = 0; i < kNW; ++i) {
        const u64 s = sm.w64[i];
        if (i < w) from += s;
        if (s) last = i;
        all += s;
    }
    const double target = (double)a.u[r] * (double)all;
    if (is_part(from, sum, all, target, w == last))
        choose(a, sp, row, q, r, 0, from, target, all, w, lane);
}

// ------------------------------------------------------------------ a row in several
struct SpanWs {
    uint32_t* ext;    // [B][S][2] extremes of each span
    uint32_t* cnt;    // [B][kBins]
    u64* mass;        // [B][kBins]
    uint32_t* found;  // [B] items in the list
    uint32_t* list;   // [B][V] their keys
    u64* list_q;      // [B][V] and weights
    Border* border;   // [B]
    u64* sum;         // [B][S] weight above the border
    uint32_t* ties;   // [B][S] items with the border's key
};

template <typename T>
__global__ __launch_bounds__(kNT) void sample_extremes_kernel(SampleArgs a, SpanWs ws, int spans) {
    __shared__ uint32_t w32[2][kNW];
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x / (unsigned)spans;
    const int s = (int)(blockIdx.x - (unsigned)r * (unsigned)spans);
    const int64_t base = (int64_t)s * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, a.V, base, w, lane);
    uint32_t hi, lo;
    sp.extremes(w32, w, lane, hi, lo);
    if (tid == 0) {
        ws.ext[2 * blockIdx.x] = hi;
        ws.ext[2 * blockIdx.x + 1] = lo;
    }
    if (s == 0) {
        for (int b = tid; b < kBins; b += kNT) {
            ws.cnt[r * kBins + b] = 0;
            ws.mass[r * kBins + b] = 0;
        }
        if (tid == 0) ws.found[r] = 0;
    }
}

// The row of a workgroup from its spans' extremes.
__device__ __forceinline__ Row row_of(const SampleArgs& a, const SpanWs& ws, int64_t r, int spans,
                                      double scale, uint32_t (&w32)[2][kNW], int tid, int lane,
                                      int w) {
    uint32_t hi = 0, lo = 0xFFFFFFFFu;
    for (int i = tid; i < spans; i += kNT) {
        const uint32_t h = ws.ext[2 * (r * spans + i)], l = ws.ext[2 * (r * spans + i) + 1];
        hi = h > hi ? h : hi;
        lo = l < lo ? l : lo;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint32_t h = (uint32_t)__shfl_xor((int)hi, d), l = (uint32_t)__shfl_xor((int)lo, d);
        hi = h > hi ? h : hi;
        lo = l < lo ? l : lo;
    }
    if (lane == 0) {
        w32[0][w] = hi;
        w32[1][w] = lo;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kNW; ++i) {
        hi = w32[0][i] > hi ? w32[0][i] : hi;
        lo = w32[1][i] < lo ? w32[1][i] : lo;
    }
    __syncthreads();
    return Row(a, r, hi, lo, scale);
}

template <typename T>
__global__ __launch_bounds__(kNT) void sample_histogram_kernel(SampleArgs a, SpanWs ws, int spans,
                                                               double scale) {
    __shared__ uint32_t cnt[kBins];
    __shared__ u64 mass[kBins];
    __shared__ uint32_t w32[2][kNW];
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x / (unsigned)spans;
    const int64_t base = (int64_t)(blockIdx.x - (unsigned)r * (unsigned)spans) * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, a.V, base, w, lane);
    for (int b = tid; b < kBins; b += kNT) {
        cnt[b] = 0;
        mass[b] = 0;
    }
    const Row row = row_of(a, ws, r, spans, scale, w32, tid, lane, w);
    if (row.bad || row.k == 1 || !row.cuts(a.V)) return;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const u64 q = row.fixed(sp.key[i]);
        if (q) {
            const int bin = row.bin(sp.key[i]);
            atomicAdd(&cnt[bin], 1u);
            atomicAdd(&mass[bin], q);
        }
    }
    __syncthreads();
    for (int b = tid; b < kBins; b += kNT)
        if (cnt[b]) {
            atomicAdd(&ws.cnt[r * kBins + b], cnt[b]);
            atomicAdd(&ws.mass[r * kBins + b], mass[b]);
        }
}

// The items of the bins that can hold a border: top-k's bin, and the bins in which top-p's may
// lie, whose share is of a sum that top-k's bin makes uncertain.
template <typename T>
__global__ __launch_bounds__(kNT) void sample_collect_kernel(SampleArgs a, SpanWs ws, int spans,
                                                             double scale) {
    __shared__ Shared sm;
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x / (unsigned)spans;
    const int64_t base = (int64_t)(blockIdx.x - (unsigned)r * (unsigned)spans) * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, a.V, base, w, lane);
    const Row row = row_of(a, ws, r, spans, scale, sm.w32, tid, lane, w);
    if (row.bad || row.k == 1 || !row.cuts(a.V)) return;
    uint32_t c = 0, c0;
    u64 m = 0, m0;
    for (int b = tid; b < kBins; b += kNT) {
        sm.cnt[b] = ws.cnt[r * kBins + b];
        sm.mass[b] = ws.mass[r * kBins + b];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kBPT; ++j) {
        c += sm.cnt[tid * kBPT + j];
        m += sm.mass[tid * kBPT + j];
    }
    c0 = c;
    m0 = m;
    block_before(sm, c, m, lane, w);
    if (tid == kNT - 1) {
        sm.lo = c + c0;
        sm.at_mass = m + m0;
    }
    __syncthreads();
    const uint32_t total = sm.lo;
    u64 least = sm.at_mass, most = least;  // the sum that top-p's share is of
    __syncthreads();
    int k_bin = -1, p_from = 0, p_to = -1;
    if (row.k < (int64_t)total) {
        pick<kBins>(sm, sm.cnt, sm.mass, c, m, false, (uint64_t)row.k, 0.0, tid);
        k_bin = sm.at;
        least = sm.above_mass;
        most = sm.above_mass + sm.at_mass;
        __syncthreads();
    }
    if (row.top_p < 1.0f) {
        pick<kBins>(sm, sm.cnt, sm.mass, c, m, true, 0, (double)row.top_p * (double)least, tid);
        p_from = sm.at < 0 ? 0 : sm.at;  // none: the least sum is 0, any bin may be it
        __syncthreads();
        pick<kBins>(sm, sm.cnt, sm.mass, c, m, true, 0, (double)row.top_p * (double)most, tid);
        p_to = sm.at;
    }
    u64 q[kItems];
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int bin = row.bin(sp.key[i]);
        const bool in = (sp.key[i] > kKeyNegInf) & ((bin == k_bin) | ((bin >= p_from) & (bin <= p_to)));
        q[i] = in ? row.fixed(sp.key[i]) : 0;
        n += q[i] != 0;
    }
    // One addition to the row's counter for the workgroup's items.
    uint32_t at = n;
    u64 unused = 0;
    __syncthreads();
    block_before(sm, at, unused, lane, w);
    if (tid == kNT - 1) sm.hi = at + n ? atomicAdd(&ws.found[r], at + n) : 0u;
    __syncthreads();
    at += sm.hi;
#pragma unroll
    for (int i = 0; i < kItems; ++i)
        if (q[i]) {
            ws.list[r * a.V + at] = sp.key[i];
            ws.list_q[r * a.V + at] = q[i];
            ++at;
        }
}

__global__ __launch_bounds__(kNT) void sample_border_kernel(SampleArgs a, SpanWs ws, int spans,
                                                            double scale) {
    __shared__ Shared sm;
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x;
    const Row row = row_of(a, ws, r, spans, scale, sm.w32, tid, lane, w);
    Border b{0, 0};
    if (!row.bad && row.k == 1) {
        b = Border{row.hi, 1};
    } else if (!row.bad && row.cuts(a.V)) {
        for (int i = tid; i < kBins; i += kNT) {
            sm.cnt[i] = ws.cnt[r * kBins + i];
            sm.mass[i] = ws.mass[r * kBins + i];
        }
        __syncthreads();
        const uint32_t n = ws.found[r];
        const uint32_t* list = ws.list + r * a.V;
        const u64* list_q = ws.list_q + r * a.V;
        b = find_border(sm, row, [&](auto f) {
            for (uint32_t i = tid; i < n; i += kNT) f(list[i], list_q[i]);
        }, tid, lane, w);
    }
    if (tid == 0) ws.border[r] = b;
}

template <typename T>
__global__ __launch_bounds__(kNT) void sample_sums_kernel(SampleArgs a, SpanWs ws, int spans,
                                                          double scale) {
    __shared__ uint32_t w32[2][kNW];
    __shared__ u64 w64[kNW];
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x / (unsigned)spans;
    const int64_t base = (int64_t)(blockIdx.x - (unsigned)r * (unsigned)spans) * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, a.V, base, w, lane);
    const Row row = row_of(a, ws, r, spans, scale, w32, tid, lane, w);
    if (row.bad) return;
    const Border b = ws.border[r];
    u64 sum = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i)
        if (sp.key[i] > b.key) sum += weight_of(row, sp.key[i]);
    sum = wave_sum(sum);
    const uint32_t ties = wave_ties(sp, b);
    if (lane == 0) {
        w64[w] = sum;
        w32[0][w] = ties;
    }
    __syncthreads();
    if (tid == 0) {
        ws.sum[blockIdx.x] = w64[0] + w64[1] + w64[2] + w64[3];
        ws.ties[blockIdx.x] = w32[0][0] + w32[0][1] + w32[0][2] + w32[0][3];
    }
}

template <typename T>
__global__ __launch_bounds__(kNT) void sample_choose_kernel(SampleArgs a, SpanWs ws, int spans,
                                                            double scale) {
    __shared__ Shared sm;
    __shared__ u64 pick_from, pick_all;
    __shared__ uint64_t pick_ties;
    __shared__ int pick_span;
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x;
    const Row row = row_of(a, ws, r, spans, scale, sm.w32, tid, lane, w);
    if (row.bad) {
        if (tid == 0) none(a, r);
        return;
    }
    const Border b = ws.border[r];
    const u64 tie_q = b.key ? weight_of(row, b.key) : 0;
    const u64* sums = ws.sum + r * spans;
    const uint32_t* ties = ws.ties + r * spans;
    // Consecutive spans to a thread.
    const int per = (spans + kNT - 1) / kNT, s0 = tid * per, s1 = s0 + per < spans ? s0 + per : spans;
    uint32_t t_own = 0;
    for (int i = s0; i < s1; ++i) t_own += ties[i];
    uint32_t t_before = t_own;
    u64 unused = 0;
    block_before(sm, t_before, unused, lane, w);
    auto kept_ties = [&](uint32_t before, uint32_t n) {
        const uint32_t left = before < b.ties ? b.ties - before : 0;
        return left < n ? left : n;
    };
    u64 own = 0;
    uint32_t t = t_before;
    for (int i = s0; i < s1; ++i) {
        own += sums[i] + tie_q * kept_ties(t, ties[i]);
        t += ties[i];
    }
    __syncthreads();
    u64 from = own;
    uint32_t unused32 = 0;
    block_before(sm, unused32, from, lane, w);
    if (tid == kNT - 1) pick_all = from + own;
    if (tid == 0) pick_span = -1;
    __syncthreads();
    const u64 all = pick_all;
    const double target = (double)a.u[r] * (double)all;
    t = t_before;
    u64 run = from;
    for (int i = s0; i < s1; ++i) {
        const u64 s = sums[i] + tie_q * kept_ties(t, ties[i]);
        if (is_part(run, s, all, target, s != 0 && run + s == all)) {
            pick_from = run;
            pick_ties = t;
            pick_span = i;
        }
        run += s;
        t += ties[i];
    }
    __syncthreads();
    if (pick_span < 0) return;  // no weight anywhere (not reached: the largest weighs 1)
    const int64_t base = (int64_t)pick_span * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, a.V, base, w, lane);
    u64 q[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) q[i] = sp.key[i] >= b.key ? weight_of(row, sp.key[i]) : 0;
    const uint32_t wt = wave_ties(sp, b);
    if (lane == 0) sm.w32[0][w] = wt;
    __syncthreads();
    uint64_t before = pick_ties;
    for (int i = 0; i < w; ++i) before += sm.w32[0][i];
    keep(sp, row, b, before, q, lane);
    u64 sum = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) sum += q[i];
    sum = wave_sum(sum);
    if (lane == 0) sm.w64[w] = sum;
    __syncthreads();
    u64 before_w = pick_from;
    for (int i = 0; i < w; ++i) before_w += sm.w64[i];
    if (is_part(before_w, sum, all, target, sum != 0 && before_w + sum == all))
        choose(a, sp, row, q, r, base, before_w, target, all, w, lane);
}

// Rows without items.
__global__ void sample_none_kernel(int32_t* ids, float* prob, int64_t B) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= B) return;
    ids[i] = -1;
    if (prob) prob[i] = 0.0f;
}

int64_t spans_of(int64_t V) { return (V + kSpan - 1) / kSpan; }

SpanWs layout(char* p, int64_t B, int64_t V, size_t* bytes) {
    size_t at = 0;
    auto take = [&](size_t n) {
        char* r = p + at;
        at += (n + 255) / 256 * 256;
        return r;
    };
    const size_t rows = (size_t)B, spans = (size_t)spans_of(V);
    SpanWs w;
    w.ext = (uint32_t*)take(rows * spans * 8);
    w.cnt = (uint32_t*)take(rows * kBins * 4);
    w.mass = (u64*)take(rows * kBins * 8);
    w.found = (uint32_t*)take(rows * 4);
    w.list = (uint32_t*)take(rows * (size_t)V * 4);
    w.list_q = (u64*)take(rows * (size_t)V * 8);
    w.border = (Border*)take(rows * sizeof(Border));
    w.sum = (u64*)take(rows * spans * 8);
    w.ties = (uint32_t*)take(rows * spans * 4);
    *bytes = at;
    return w;
}

template <typename T>
hipError_t launch_typed(const SampleArgs& a, double scale, void* p, hipStream_t stream) {
    const dim3 rows((unsigned)a.B), block(kNT);
    if (a.V <= kSpan) {
        hipLaunchKernelGGL(sample_row_kernel<T>, rows, block, 0, stream, a, scale);
        return hipGetLastError();
    }
    const int spans = (int)spans_of(a.V);
    size_t bytes;
    const SpanWs ws = layout((char*)p, a.B, a.V, &bytes);
    const dim3 all((unsigned)(a.B * spans));
    hipLaunchKernelGGL(sample_extremes_kernel<T>, all, block, 0, stream, a, ws, spans);
    hipLaunchKernelGGL(sample_histogram_kernel<T>, all, block, 0, stream, a, ws, spans, scale);
    hipLaunchKernelGGL(sample_collect_kernel<T>, all, block, 0, stream, a, ws, spans, scale);
    hipLaunchKernelGGL(sample_border_kernel, rows, block, 0, stream, a, ws, spans, scale);
    hipLaunchKernelGGL(sample_sums_kernel<T>, all, block, 0, stream, a, ws, spans, scale);
    hipLaunchKernelGGL(sample_choose_kernel<T>, rows, block, 0, stream, a, ws, spans, scale);
    return hipGetLastError();
}

}  // namespace

size_t sample_workspace(int64_t B, int64_t V, IoType) {
    if (V <= kSpan || B == 0) return 0;
    size_t bytes;
    (void)layout(nullptr, B, V, &bytes);
    return bytes;
}

hipError_t launch_sample(const SampleArgs& a, void* ws, hipStream_t stream) {
    if (a.V == 0) {
        hipLaunchKernelGGL(sample_none_kernel, dim3((unsigned)((a.B + 255) / 256)), dim3(256), 0,
                           stream, a.ids, a.prob, a.B);
        return hipGetLastError();
    }
    int log_v = 0;
    while (((int64_t)1 << log_v) < a.V) ++log_v;
    // Sums of V of them stay below 2^62, and one below 2^51.
    const double scale = (double)((uint64_t)1 << (log_v < 11 ? 51 : 62 - log_v));
    return a.io == IoType::kF32 ? launch_typed<float>(a, scale, ws, stream)
                                : launch_typed<bf16>(a, scale, ws, stream);
}

}  // namespace recblr
