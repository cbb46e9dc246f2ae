// One item a row from logits (recblr_sample): temperature, top-k, top-p, min-p.
//
// The items that stay are a run of the order (logit falling, index rising), so a row's
// selection is one border: a logit, and how many of the items with that very logit stay;
// nothing is sorted.  Weights w = exp((l - max) / temperature) are formed in 64 bits and summed as
// integers q = round(w 2^F): such sums are exact in any order, so atomics repeat bit for bit
// and a border falls where 64-bit arithmetic puts it.  Items with q = 0 can neither be chosen
// nor move a border that matters; they take no part.
//
// The border is found on a histogram of counts and weights over kBins equal steps of the logit
// (uniform steps spread the items of usual logits evenly; the bits of a float do not: its
// upper eleven put half of a row in twenty bins, whose atomics then wait for each other).  The
// bin that holds the border has a few items most often, which are compared with one another; a
// fuller one is searched by the floats' own bits, 8 at a time, until few or equal ones are left.
//
// A row of up to kSpan items is one workgroup's, logits and weights in its registers from a
// single read.  A longer one takes a workgroup for each span of kSpan items and six short
// launches: extremes, histogram, the items of the bins that can hold a border, the border
// itself (on those items alone), sums of the spans, and the choice within one span.
//
// What bounds a row is its chain of some twenty short phases with a barrier each, about 15 us, of
// which four workgroups a CU hide a part: 2048 rows of 3416 take 36 us, 64 of 131072 in bf16
// 75 us and 4 of 50000 43 us (memory alone: 6, 3.5 and 0.2 us).  Handing a row's last steps to
// its last workgroup instead of launches of their own took 82 and 41 us for the latter two.
#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "lanes.hpp"
#include "ops.hpp"

namespace recblr {
namespace {

using namespace lanes;

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
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float wave_top(float v) {
    return lane_of(wave_scan(v, -kInf, [](float a, float b) { return fmaxf(a, b); }), kWave - 1);
}
__device__ __forceinline__ float wave_least(float v) {
    return lane_of(wave_scan(v, kInf, [](float a, float b) { return fminf(a, b); }), kWave - 1);
}

// A constant in scalar registers: left to the compiler, those of exp_neg are kept in vector ones.
__device__ __forceinline__ double scalar(double c) {
    asm("" : "+s"(c));
    return c;
}

// e^x for x in [-46, 0]: x = n ln 2 + t with |t| <= ln 2 / 2, and e^t by its Taylor polynomial
// of degree 12, whose remainder is below 2e-16 of it.
__device__ __forceinline__ double exp_neg(double x) {
    const double n = __builtin_rint(x * scalar(1.4426950408889634074));
    // ln 2 as its nearest double and what that leaves.
    double t = __builtin_fma(n, scalar(-0.69314718055994530942), x);
    t = __builtin_fma(n, scalar(-2.3190468138462996e-17), t);
    double p = scalar(1.0 / 479001600.0);
    p = __builtin_fma(p, t, scalar(1.0 / 39916800.0));
    p = __builtin_fma(p, t, scalar(1.0 / 3628800.0));
    p = __builtin_fma(p, t, scalar(1.0 / 362880.0));
    p = __builtin_fma(p, t, scalar(1.0 / 40320.0));
    p = __builtin_fma(p, t, scalar(1.0 / 5040.0));
    p = __builtin_fma(p, t, scalar(1.0 / 720.0));
    p = __builtin_fma(p, t, scalar(1.0 / 120.0));
    p = __builtin_fma(p, t, scalar(1.0 / 24.0));
    p = __builtin_fma(p, t, scalar(1.0 / 6.0));
    p = __builtin_fma(p, t, 0.5);
    p = __builtin_fma(p, t, 1.0);
    p = __builtin_fma(p, t, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}

// The nearest integer of x in [0, 2^51]: 2^52 + x has it in its lowest bits.
__device__ __forceinline__ u64 rounded(double x) {
    return (u64)__double_as_longlong(x + 0x1p52) & 0xFFFFFFFFFFFFFull;
}

// What a row asks for, read before its logits' extremes are known.
struct Ask {
    float temp, top_p, min_p, u;
    int32_t top_k;
    __device__ __forceinline__ Ask(const SampleArgs& a, int64_t row) {
        temp = a.temperature ? a.temperature[row] : 1.0f;
        top_p = a.top_p ? a.top_p[row] : 1.0f;
        min_p = a.min_p ? a.min_p[row] : 0.0f;
        top_k = a.top_k ? a.top_k[row] : 0;
        u = a.u[row];
    }
};

// Whether an item (with weight) is of some bins: its step of the histogram lies in [from, to).
// A NaN is none's; with to a NaN all further ones are the last bin's.
struct Within {
    float top, bins, from, to;
    __device__ __forceinline__ bool operator()(float v) const {
        const float b = (top - v) * bins;
        return (b >= from) & !(b >= to);
    }
    // Makes this not known to be as before: else the steps of all of a lane's items are kept
    // from one use to the next, and spill.
    __device__ __forceinline__ void anew() { asm volatile("" : "+v"(top)); }
};
__device__ __forceinline__ uint32_t key_anew(float v) {
    asm volatile("" : "+v"(v));
    return key_of(v);
}

// That, and the measures that the extremes give.
struct Row {
    double inv_t, max, scale;
    float top, bins;  // largest logit; bins to a unit of the logit
    float top_p, min_p;
    int64_t k;
    bool bad, greedy;

    // Of a row whose largest and smallest logits are hi and lo.
    __device__ __forceinline__ Row(const Ask& ask, int64_t V, float hi, float lo, double scale_) {
        top = hi;
        scale = scale_;
        const float temp = ask.temp;
        bad = !(hi > -kInf && hi < kInf) || !(temp == temp);
        top_p = ask.top_p;
        min_p = ask.min_p > 1.0f ? 1.0f : ask.min_p;  // a NaN stays one, and sets no limit
        greedy = temp <= 0.0f;
        k = ask.top_k > 0 ? ask.top_k : V;
        if (greedy || top_p <= 0.0f) k = 1;
        inv_t = greedy ? 0.0 : 1.0 / (double)temp;
        max = (double)top;
        const float range = fminf(46.0f * temp, top - lo);
        // Finite at both ends of the range's sizes: else the top's step would be 0 times infinity.
        // A range below 3.4e-36 is then the first bins' alone, and at the end one bin's.
        bins = range > 0.0f ? fminf((float)(kBins - 1) / fminf(range, 3e38f), 3e38f) : 0.0f;
    }
    __device__ __forceinline__ double weight(float v) const {
        // What lies further down than 46 temperatures (-inf and what is no item, a NaN, among it)
        // weighs e^-46, which no scale up to 2^51 brings to a half.
        return exp_neg(fmax(((double)v - max) * inv_t, -46.0));
    }
    __device__ __forceinline__ u64 fixed(float v) const { return rounded(weight(v) * scale); }
    // Rising as the logit falls: both roundings keep the order.
    __device__ __forceinline__ int bin(float v) const {
        const float b = (top - v) * bins;
        return b < (float)(kBins - 1) ? (int)b : kBins - 1;
    }
    // Bins from..to; none where from is -1.
    __device__ __forceinline__ Within within(int from, int to) const {
        const float none = __builtin_nanf("");
        return Within{top, bins, from < 0 ? none : (float)from,
                      to < kBins - 1 ? (float)(to + 1) : none};
    }
    // Whether a border has to be looked for.
    __device__ __forceinline__ bool cuts(int64_t V) const { return k < V || top_p < 1.0f; }
};

struct Border {
    float at;       // items above it stay,
    uint32_t ties;  // and the first `ties` of those that have it
};

struct Shared {
    uint32_t cnt[kBins];
    u64 mass[kBins];
    uint32_t fine_cnt[kFine];
    float few[kWave];
    u64 fine_mass[kFine];
    uint32_t w32[kNW];
    float ext[2][kNW];
    u64 w64[kNW];
    uint32_t lo, hi;
    int at;             // bin found
    uint32_t at_cnt, above_cnt;
    u64 above_mass, at_mass;
};

// A count and a weight of each thread become their sums over lower threads; returned are the
// workgroup's.  Holds one barrier; another one has to lie between two calls.
struct Total {
    uint32_t c;
    u64 m;
};
__device__ __forceinline__ Total block_before(Shared& sm, uint32_t& c, u64& m, int lane, int w) {
    const uint32_t ci = wave_upto(c);
    const u64 mi = wave_upto(m);
    if (lane == kWave - 1) {
        sm.w32[w] = ci;
        sm.w64[w] = mi;
    }
    c = ci - c;
    m = mi - m;
    __syncthreads();
    Total t{0, 0};
#pragma unroll
    for (int i = 0; i < kNW; ++i) {
        c += i < w ? sm.w32[i] : 0;
        m += i < w ? sm.w64[i] : 0;
        t.c += sm.w32[i];
        t.m += sm.w64[i];
    }
    return t;
}

// A thread's N consecutive bins of a histogram in LDS: what they hold, then what lies before them.
template <int N>
struct Bins {
    const uint32_t* cnt;
    const u64* mass;
    uint32_t c = 0;
    u64 m = 0;
    __device__ __forceinline__ Bins(const uint32_t* cnt_, const u64* mass_, int tid)
        : cnt(cnt_ + tid * N), mass(mass_ + tid * N) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            c += cnt[j];
            m += mass[j];
        }
    }
    // The bin before which there is less than wanted (want_cnt items, or a weight of want_mass)
    // and with which there is not: it and what lies before it go to sm, by the one thread that
    // has it.  Ends with a barrier.
    __device__ __forceinline__ void pick(Shared& sm, bool by_mass, uint64_t want_cnt,
                                         double want_mass, int tid) const {
        uint32_t cj = c;
        u64 mj = m;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t n = cnt[j];
            const u64 q = mass[j];
            const bool in = by_mass ? (double)mj < want_mass && !((double)(mj + q) < want_mass)
                                    : cj < want_cnt && !(cj + n < want_cnt);
            if (in) {
                sm.at = tid * N + j;
                sm.above_cnt = cj;
                sm.above_mass = mj;
                sm.at_cnt = n;
                sm.at_mass = q;
            }
            cj += n;
            mj += q;
        }
        __syncthreads();
    }
};

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

// Searches one bin further.  each(f) calls f(v, q) for the items that may be of it (all with
// weight; NaN is passed over), those from `from` on that `bin` takes are; `above` of sm is what lies before the bin and is brought to what lies before
// the logit found, which has sm.at_cnt items.
template <typename Each>
__device__ __forceinline__ float refine(Shared& sm, Each each, Within bin, float from, bool by_mass,
                                        uint64_t want_cnt, double want_mass, int tid, int lane,
                                        int w) {
    float to = kInf;
    uint32_t base_c = sm.above_cnt;
    u64 base_m = sm.above_mass;
    // Each search leaves at most a 128th of the keys' range: five come down to one key.
    for (int depth = 0; depth < 8; ++depth) {
        const bool few = sm.at_cnt <= (uint32_t)kWave;
        bin.anew();
        __syncthreads();
        if (few) {
            // The usual case: each item is compared with all others, a lane of the first wave an
            // item.  The border is the lowest logit with less than is wanted before it.
            if (tid < kWave) sm.few[tid] = -kInf;
            if (tid == 0) sm.hi = 0;
            __syncthreads();
            each([&](float v, u64 q) {
                if ((v >= from) & (v <= to) & bin(v)) {
                    const uint32_t i = atomicAdd(&sm.hi, 1u);
                    sm.few[i] = v;
                    sm.fine_mass[i] = q;
                }
            });
            __syncthreads();
            if (tid < kWave) {
                const uint32_t n = sm.hi;
                const float v = sm.few[tid];
                uint32_t c = base_c, same = 0;
                u64 m = base_m;
#pragma unroll 1
                for (uint32_t i = 0; i < n; i += 4) {
#pragma unroll
                    for (uint32_t j = i; j < i + 4; ++j) {  // behind the last: -inf, above none
                        const float o = sm.few[j];
                        const u64 q = sm.fine_mass[j];
                        c += o > v;
                        same += o == v;
                        m += o > v ? q : 0;
                    }
                }
                const bool in =
                    (uint32_t)tid < n && (by_mass ? (double)m < want_mass : c < want_cnt);
                const float least = wave_least(in ? v : kInf);
                if (in && v == least) {  // equal ones write the same
                    sm.above_cnt = c;
                    sm.above_mass = m;
                    sm.at_cnt = same;
                }
                if (tid == 0) sm.few[0] = least;
            }
            __syncthreads();
            return sm.few[0];
        }
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
        each([&](float v, u64) {
            const bool in = (v >= from) & (v <= to) & bin(v);
            const uint32_t key = key_anew(v);
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
        each([&](float v, u64 q) {
            if ((v >= from) & (v <= to) & bin(v)) {
                const uint32_t b = (hi - key_anew(v)) >> shift;
                atomicAdd(&sm.fine_cnt[b], 1u);
                atomicAdd(&sm.fine_mass[b], q);
            }
        });
        __syncthreads();
        Bins<kFine / kNT> bins(sm.fine_cnt, sm.fine_mass, tid);
        block_before(sm, bins.c, bins.m, lane, w);
        bins.c += base_c;
        bins.m += base_m;
        bins.pick(sm, by_mass, want_cnt, want_mass, tid);
        base_c = sm.above_cnt;
        base_m = sm.above_mass;
        const uint32_t last = hi - ((uint32_t)sm.at << shift);  // the bin's keys end with it
        const uint32_t n = 1u << shift;
        const uint32_t first = last - lo < n ? lo : last - n + 1;
        // Between the zeros' keys, which are one number, lies no item's.
        to = value_of(last == 0x7FFFFFFFu ? last - 1 : last);
        from = value_of(first);
        if (first == last) break;
    }
    return to;
}

// The row's border, from the whole histogram in sm (items with q > 0) and the items of the bins
// that may hold it.  All threads return the same.
template <typename Each>
__device__ __forceinline__ Border find_border(Shared& sm, const Row& row, Each each, int tid,
                                              int lane, int w) {
    Bins<kBPT> bins(sm.cnt, sm.mass, tid);
    const Total total = block_before(sm, bins.c, bins.m, lane, w);
    u64 above = total.m;
    Border b{-kInf, 0};
    u64 tie_q = 0;
    if (row.k < (int64_t)total.c) {
        bins.pick(sm, false, (uint64_t)row.k, 0.0, tid);
        b.at = refine(sm, each, row.within(sm.at, sm.at), -kInf, false, (uint64_t)row.k, 0.0, tid,
                      lane, w);
        b.ties = (uint32_t)(row.k - sm.above_cnt);
        above = sm.above_mass;
        tie_q = row.fixed(b.at);
    }
    if (row.top_p < 1.0f && row.k > 1) {
        const double want = (double)row.top_p * (double)(above + tie_q * (u64)b.ties);
        if ((double)above < want) {
            if (b.ties) b.ties = ties_within(b.ties, tie_q, above, want);
        } else {
            const float next = value_of(key_of(b.at) + 1);  // the float above the first border
            __syncthreads();  // what the first search left in sm has been read
            bins.pick(sm, true, 0, want, tid);
            b.at = refine(sm, each, row.within(sm.at, sm.at), next, true, 0, want, tid, lane, w);
            b.ties = ties_within(sm.at_cnt, row.fixed(b.at), sm.above_mass, want);
        }
    }
    return b;
}

// A span of a row: its logits in order, a wave's 1024 after another's, groups of four to a lane.
// What lies behind the row's end is NaN, which no comparison takes; a NaN within the row becomes
// +inf, which spoils the row as well.
template <typename T>
struct Span {
    float v[kItems];
    __device__ __forceinline__ static int index(int base, int w, int it, int lane) {
        return base + (w * kIT + it) * 256 + lane * 4;
    }
    __device__ __forceinline__ Span(const T* p, int V, int base, int w, int lane) {
        const bool vec = ((uintptr_t)p) % (4 * sizeof(T)) == 0;
#pragma unroll
        for (int it = 0; it < kIT; ++it) {
            const int i = index(base, w, it, lane);
            float x[4];
            if (vec && i + 4 <= V) {
                unpack_vec<T, 4>(*(const typename VecT<T, 4>::type*)(p + i), x);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * it + e] = x[e] == x[e] ? x[e] : kInf;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = i + e < V ? to_f32(p[i + e]) : 0.0f;
                    v[4 * it + e] = i + e < V ? (x[e] == x[e] ? x[e] : kInf) : __builtin_nanf("");
                }
            }
        }
    }
    // Between the phases of a kernel: what one has computed from the logits is computed anew by
    // the next, not kept in registers (kept, it spilled).
    __device__ __forceinline__ void phase() {
#pragma unroll
        for (int i = 0; i < kItems; ++i) asm volatile("" : "+v"(v[i]));
    }
    // Largest and smallest logit over the workgroup's items, by all threads; ext of LDS.
    __device__ __forceinline__ void extremes(float (&ext)[2][kNW], int w, int lane, float& hi,
                                             float& lo) const {
        hi = -kInf;
        lo = kInf;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            hi = v[i] > hi ? v[i] : hi;
            lo = v[i] < lo ? v[i] : lo;
        }
        all_extremes(ext, w, lane, hi, lo);
    }
    __device__ __forceinline__ static void all_extremes(float (&ext)[2][kNW], int w, int lane,
                                                        float& hi, float& lo) {
        hi = wave_top(hi);
        lo = wave_least(lo);
        if (lane == 0) {
            ext[0][w] = hi;
            ext[1][w] = lo;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kNW; ++i) {
            hi = fmaxf(hi, ext[0][i]);
            lo = fminf(lo, ext[1][i]);
        }
        hi = lane_of(hi, 0);
        lo = lane_of(lo, 0);
    }
};

// The choice within a span whose first item has `before` items of the border's logit before it:
// q of items that stay is left, others' become 0.
template <typename T>
__device__ __forceinline__ void keep(const Span<T>& sp, const Border& b, uint32_t before,
                                     u64 (&q)[kItems]) {
#pragma unroll
    for (int it = 0; it < kIT; ++it) {
        const float* v = sp.v + 4 * it;
        uint32_t n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) n += v[e] == b.at;
        if (b.ties && __any((int)n)) {
            const uint32_t upto = wave_upto(n);
            uint32_t mine = before + upto - n;
            before += lane_of(upto, kWave - 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool tie = v[e] == b.at;
                if (!(v[e] > b.at || (tie && mine < b.ties))) q[4 * it + e] = 0;
                mine += tie;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!(v[e] > b.at)) q[4 * it + e] = 0;
        }
    }
}

// A wave's items of the border's logit.
template <typename T>
__device__ __forceinline__ uint32_t wave_ties(const Span<T>& sp, const Border& b) {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) n += (uint32_t)__popcll(__ballot(sp.v[i] == b.at));
    return n;
}

// The weights of a row's items: min-p's are 0 as well (in a greedy row all weigh the same).
__device__ __forceinline__ u64 weight_of(const Row& row, float v) {
    if (row.greedy) return v > -kInf ? (u64)row.scale : 0;
    const double wt = row.weight(v);
    return wt < (double)row.min_p ? 0 : rounded(wt * row.scale);
}

// The item at which the running sum, `run0` before the wave's first item, first exceeds target,
// else the wave's last one with weight; written by the lane that has it.
template <typename T>
__device__ __forceinline__ void choose(const SampleArgs& a, const Span<T>& sp, const Row& row,
                                       const u64 (&q)[kItems], int64_t r, int base, u64 run,
                                       double target, u64 all, int w, int lane) {
    int found = -1, tail = -1;
    float v_found = 0.0f, v_tail = 0.0f;
#pragma unroll
    for (int it = 0; it < kIT; ++it) {
        const u64 own = q[4 * it] + q[4 * it + 1] + q[4 * it + 2] + q[4 * it + 3];
        const u64 upto = wave_upto(own);
        u64 c = run + upto - own;
        run += lane_of(upto, kWave - 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c += q[4 * it + e];
            if (q[4 * it + e]) {
                tail = Span<T>::index(base, w, it, lane) + e;
                v_tail = sp.v[4 * it + e];
                if (found < 0 && (double)c > target) {
                    found = tail;
                    v_found = v_tail;
                }
            }
        }
    }
    // Items are fewer than 2^24: their indexes are floats, found or not.
    const float none = 0x1p24f;
    const float best = wave_least(found >= 0 ? (float)found : none);
    const float end = wave_top((float)tail);
    const bool got = best != none;
    const int id = (int)(got ? best : end);
    if (got ? found == id : tail == id) {
        a.ids[r] = id;
        const double wt = row.greedy ? 1.0 : row.weight(got ? v_found : v_tail);
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
__global__ __launch_bounds__(kNT, 4) void sample_row_kernel(SampleArgs a, double scale) {
    __shared__ Shared sm;
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x;
    Span<T> sp((const T*)a.logits + r * a.V, (int)a.V, 0, w, lane);
    const Ask ask(a, r);
    for (int b = tid; b < kBins; b += kNT) {
        sm.cnt[b] = 0;
        sm.mass[b] = 0;
    }
    float hi, lo;
    sp.extremes(sm.ext, w, lane, hi, lo);
    const Row row(ask, a.V, hi, lo, scale);
    if (row.bad) {
        if (tid == 0) none(a, r);
        return;
    }
    sp.phase();
    u64 q[kItems];
    Border b{-kInf, 0};
    if (row.k == 1) {
        b = Border{row.top, 1};
#pragma unroll
        for (int i = 0; i < kItems; ++i) q[i] = sp.v[i] == row.top ? (u64)scale : 0;
    } else {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            q[i] = row.fixed(sp.v[i]);
            sp.v[i] = q[i] ? sp.v[i] : __builtin_nanf("");
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
        sp.phase();
        if (row.cuts(a.V)) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (q[i]) {
                    const int bin = row.bin(sp.v[i]);
                    atomicAdd(&sm.cnt[bin], 1u);
                    atomicAdd(&sm.mass[bin], q[i]);
                }
            __syncthreads();
            auto each = [&](auto f) {
#pragma unroll
                for (int i = 0; i < kItems; ++i) f(sp.v[i], q[i]);
            };
            sp.phase();
            b = find_border(sm, row, each, tid, lane, w);
        }
        if (row.min_p > 0.0f) {
            // As weight_of, by the weight itself; its q tells unless it is next to min_p's.
            const u64 least = rounded((double)row.min_p * scale);
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                if (q[i] < least) q[i] = 0;
                else if (q[i] <= least + 1 && row.weight(sp.v[i]) < (double)row.min_p) q[i] = 0;
            }
        }
    }
    __syncthreads();
    sp.phase();
    const uint32_t ties = wave_ties(sp, b);
    if (lane == 0) sm.w32[w] = ties;
    __syncthreads();
    uint32_t before = 0;
    for (int i = 0; i < w; ++i) before += sm.w32[i];
    keep(sp, b, before, q);
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
    const double target = (double)ask.u * (double)all;
    if (is_part(from, sum, all, target, w == last))
        choose(a, sp, row, q, r, 0, from, target, all, w, lane);
}

// ------------------------------------------------------------------ a row in several
struct SpanWs {
    float* ext;       // [B][S][2] extremes of each span
    uint32_t* cnt;    // [B][kBins]
    u64* mass;        // [B][kBins]
    uint32_t* found;  // [B] items in the list
    float* list;      // [B][V] their logits
    Border* border;   // [B]
    u64* sum;         // [B][S] weight above the border
    uint32_t* ties;   // [B][S] items with the border's logit
};

template <typename T>
__global__ __launch_bounds__(kNT) void sample_extremes_kernel(SampleArgs a, SpanWs ws, int spans) {
    __shared__ float ext[2][kNW];
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x / (unsigned)spans;
    const int s = (int)(blockIdx.x - (unsigned)r * (unsigned)spans);
    const int base = s * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, (int)a.V, base, w, lane);
    float hi, lo;
    sp.extremes(ext, w, lane, hi, lo);
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
                                      double scale, const Ask& ask, float (&ext)[2][kNW], int tid,
                                      int lane, int w) {
    float hi = -kInf, lo = kInf;
    for (int i = tid; i < spans; i += kNT) {
        hi = fmaxf(hi, ws.ext[2 * (r * spans + i)]);
        lo = fminf(lo, ws.ext[2 * (r * spans + i) + 1]);
    }
    Span<float>::all_extremes(ext, w, lane, hi, lo);
    __syncthreads();
    return Row(ask, a.V, hi, lo, scale);
}

template <typename T>
__global__ __launch_bounds__(kNT) void sample_histogram_kernel(SampleArgs a, SpanWs ws, int spans,
                                                               double scale) {
    __shared__ uint32_t cnt[kBins];
    __shared__ u64 mass[kBins];
    __shared__ float ext[2][kNW];
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x / (unsigned)spans;
    const Ask ask(a, r);
    const int base = (int)(blockIdx.x - (unsigned)r * (unsigned)spans) * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, (int)a.V, base, w, lane);
    for (int b = tid; b < kBins; b += kNT) {
        cnt[b] = 0;
        mass[b] = 0;
    }
    const Row row = row_of(a, ws, r, spans, scale, ask, ext, tid, lane, w);
    if (row.bad || row.k == 1 || !row.cuts(a.V)) return;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const u64 q = row.fixed(sp.v[i]);
        if (q) {
            const int bin = row.bin(sp.v[i]);
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

// A row's histogram on its way from memory to LDS, read before the row is known.
struct Fetched {
    uint32_t cnt[kBPT];
    u64 mass[kBPT];
    __device__ __forceinline__ Fetched(const SpanWs& ws, int64_t r, int tid) {
#pragma unroll
        for (int j = 0; j < kBPT; ++j) {
            cnt[j] = ws.cnt[r * kBins + j * kNT + tid];
            mass[j] = ws.mass[r * kBins + j * kNT + tid];
        }
    }
    __device__ __forceinline__ void put(Shared& sm, int tid) const {
#pragma unroll
        for (int j = 0; j < kBPT; ++j) {
            sm.cnt[j * kNT + tid] = cnt[j];
            sm.mass[j * kNT + tid] = mass[j];
        }
        __syncthreads();
    }
};

// The items of the bins that can hold a border: top-k's bin, and the bins in which top-p's may
// lie, whose share is of a sum that top-k's bin makes uncertain.
template <typename T>
__global__ __launch_bounds__(kNT) void sample_collect_kernel(SampleArgs a, SpanWs ws, int spans,
                                                             double scale) {
    __shared__ Shared sm;
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x / (unsigned)spans;
    const Ask ask(a, r);
    const int base = (int)(blockIdx.x - (unsigned)r * (unsigned)spans) * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, (int)a.V, base, w, lane);
    const Fetched hist(ws, r, tid);
    const Row row = row_of(a, ws, r, spans, scale, ask, sm.ext, tid, lane, w);
    if (row.bad || row.k == 1 || !row.cuts(a.V)) return;
    hist.put(sm, tid);
    Bins<kBPT> bins(sm.cnt, sm.mass, tid);
    const Total total = block_before(sm, bins.c, bins.m, lane, w);
    u64 least = total.m, most = least;  // the sum that top-p's share is of
    int k_bin = -1, p_from = -1, p_to = -1;
    if (row.k < (int64_t)total.c) {
        bins.pick(sm, false, (uint64_t)row.k, 0.0, tid);
        k_bin = sm.at;
        least = sm.above_mass;
        most = sm.above_mass + sm.at_mass;
        __syncthreads();
    }
    if (row.top_p < 1.0f) {
        p_from = 0;  // where the least sum is 0, any bin may be it
        if (least > 0) {
            bins.pick(sm, true, 0, (double)row.top_p * (double)least, tid);
            p_from = sm.at;
            __syncthreads();
        }
        bins.pick(sm, true, 0, (double)row.top_p * (double)most, tid);
        p_to = sm.at;
    }
    const auto of_k = row.within(k_bin, k_bin), of_p = row.within(p_from, p_to);
    u64 q[kItems];
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const bool in = (sp.v[i] > -kInf) & (of_k(sp.v[i]) | of_p(sp.v[i]));
        q[i] = in ? row.fixed(sp.v[i]) : 0;
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
            ws.list[r * a.V + at] = sp.v[i];
            ++at;
        }
}

__global__ __launch_bounds__(kNT) void sample_border_kernel(SampleArgs a, SpanWs ws, int spans,
                                                            double scale) {
    __shared__ Shared sm;
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x;
    const Ask ask(a, r);
    // Everything is read at once, the list's first items too: they stay in registers, since the
    // searches go over them up to ten times.
    constexpr int kHeld = 8;
    const Fetched hist(ws, r, tid);
    const uint32_t n = ws.found[r];
    const float* list = ws.list + r * a.V;
    float v[kHeld];
    u64 q[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
        const uint32_t i = tid + j * kNT;
        v[j] = i < n ? list[i] : __builtin_nanf("");
    }
    const Row row = row_of(a, ws, r, spans, scale, ask, sm.ext, tid, lane, w);
    Border b{-kInf, 0};
    if (!row.bad && row.k == 1) {
        b = Border{row.top, 1};
    } else if (!row.bad && row.cuts(a.V)) {
        hist.put(sm, tid);
#pragma unroll
        for (int j = 0; j < kHeld; ++j) q[j] = row.fixed(v[j]);
        b = find_border(sm, row, [&](auto f) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) f(v[j], q[j]);
            for (uint32_t i = tid + kHeld * kNT; i < n; i += kNT) f(list[i], row.fixed(list[i]));
        }, tid, lane, w);
    }
    if (tid == 0) ws.border[r] = b;
}

template <typename T>
__global__ __launch_bounds__(kNT) void sample_sums_kernel(SampleArgs a, SpanWs ws, int spans,
                                                          double scale) {
    __shared__ uint32_t w32[kNW];
    __shared__ float ext[2][kNW];
    __shared__ u64 w64[kNW];
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x / (unsigned)spans;
    const Ask ask(a, r);
    const int base = (int)(blockIdx.x - (unsigned)r * (unsigned)spans) * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, (int)a.V, base, w, lane);
    const Border b = ws.border[r];
    const Row row = row_of(a, ws, r, spans, scale, ask, ext, tid, lane, w);
    if (row.bad) return;
    u64 sum = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i)
        if (sp.v[i] > b.at) sum += weight_of(row, sp.v[i]);
    sum = wave_sum(sum);
    const uint32_t ties = wave_ties(sp, b);
    if (lane == 0) {
        w64[w] = sum;
        w32[w] = ties;
    }
    __syncthreads();
    if (tid == 0) {
        ws.sum[blockIdx.x] = w64[0] + w64[1] + w64[2] + w64[3];
        ws.ties[blockIdx.x] = w32[0] + w32[1] + w32[2] + w32[3];
    }
}

template <typename T>
__global__ __launch_bounds__(kNT) void sample_choose_kernel(SampleArgs a, SpanWs ws, int spans,
                                                            double scale) {
    __shared__ Shared sm;
    __shared__ u64 pick_from, pick_all;
    __shared__ uint32_t pick_ties;
    __shared__ int pick_span;
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t r = blockIdx.x;
    const Ask ask(a, r);
    const Border b = ws.border[r];
    const u64* sums = ws.sum + r * spans;
    const uint32_t* ties = ws.ties + r * spans;
    // Consecutive spans to a thread.
    const int per = (spans + kNT - 1) / kNT, s0 = tid * per, s1 = s0 + per < spans ? s0 + per : spans;
    // The first of them is read ahead: that is all for up to 2^20 items.
    const u64 first_sum = s0 < s1 ? sums[s0] : 0;
    const uint32_t first_ties = s0 < s1 ? ties[s0] : 0;
    auto sum_of = [&](int i) { return i == s0 ? first_sum : sums[i]; };
    auto ties_of = [&](int i) { return i == s0 ? first_ties : ties[i]; };
    const Row row = row_of(a, ws, r, spans, scale, ask, sm.ext, tid, lane, w);
    if (row.bad) {
        if (tid == 0) none(a, r);
        return;
    }
    const u64 tie_q = b.ties ? weight_of(row, b.at) : 0;
    uint32_t t_own = 0;
    for (int i = s0; i < s1; ++i) t_own += ties_of(i);
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
        own += sum_of(i) + tie_q * kept_ties(t, ties_of(i));
        t += ties_of(i);
    }
    __syncthreads();
    u64 from = own;
    uint32_t unused32 = 0;
    block_before(sm, unused32, from, lane, w);
    if (tid == kNT - 1) pick_all = from + own;
    if (tid == 0) pick_span = -1;
    __syncthreads();
    const u64 all = pick_all;
    const double target = (double)ask.u * (double)all;
    t = t_before;
    u64 run = from;
    for (int i = s0; i < s1; ++i) {
        const u64 s = sum_of(i) + tie_q * kept_ties(t, ties_of(i));
        if (is_part(run, s, all, target, s != 0 && run + s == all)) {
            pick_from = run;
            pick_ties = t;
            pick_span = i;
        }
        run += s;
        t += ties_of(i);
    }
    __syncthreads();
    if (pick_span < 0) {  // no weight anywhere (not reached: the largest weighs 1)
        if (tid == 0) none(a, r);
        return;
    }
    const int base = pick_span * kSpan;
    const Span<T> sp((const T*)a.logits + r * a.V, (int)a.V, base, w, lane);
    u64 q[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) q[i] = sp.v[i] >= b.at ? weight_of(row, sp.v[i]) : 0;
    const uint32_t wt = wave_ties(sp, b);
    if (lane == 0) sm.w32[w] = wt;
    __syncthreads();
    uint32_t before = pick_ties;
    for (int i = 0; i < w; ++i) before += sm.w32[i];
    keep(sp, b, before, q);
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
    w.ext = (float*)take(rows * spans * 8);
    w.cnt = (uint32_t*)take(rows * kBins * 4);
    w.mass = (u64*)take(rows * kBins * 8);
    w.found = (uint32_t*)take(rows * 4);
    w.list = (float*)take(rows * (size_t)V * 4);
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
