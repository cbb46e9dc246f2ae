// One item a row from logits (recblr_sample): temperature, top-k, top-p, min-p.
//
// The items that stay are a run of the order (logit falling, index rising), so a row's
// selection is one border: a key, and how many of the items with that very key stay.  The
// border is found by descending the key's 32 bits, 11, 11 and 10 at a time, over a histogram
// in LDS of counts (top-k) or of weights (top-p); nothing is sorted.  Weights are
// w = exp((l - max) / temperature) in 64 bits, summed as integers q = round(w 2^F): such sums
// are exact in any order, so atomics repeat bit for bit and a border falls where 64-bit
// arithmetic puts it.
//
// One workgroup takes one row.  Waves own consecutive spans of the row, so running sums in
// order of the index are a wave's sum, then a lane's.
#include <hip/hip_runtime.h>

#include "device_common.hpp"
#include "ops.hpp"

namespace recblr {
namespace {

constexpr int kBins = 2048;

// Order-preserving bits of a float: equal floats (the two zeros among them) have equal keys.
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
constexpr uint32_t kKeyNegInf = 0x007FFFFFu;  // key_of(-inf); a NaN's key lies outside
constexpr uint32_t kKeyPosInf = 0xFF800000u;  // [key_of(-inf), key_of(+inf)]

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

struct RowParams {
    double inv_t;   // 1 / temperature
    double max;     // largest logit
    double scale;   // 2^F
};
// The weight of a key, as the integer that is summed.
__device__ __forceinline__ double weight(uint32_t key, const RowParams& r) {
    const double x = ((double)value_of(key) - r.max) * r.inv_t;
    return key > kKeyNegInf && x > -45.0 ? exp(x) : 0.0;  // below e^-45 < 2^-63: rounds to 0
}
__device__ __forceinline__ uint64_t fixed(double w, const RowParams& r) {
    return (uint64_t)(w * r.scale + 0.5);
}

template <int NT>
struct Shared {
    uint32_t cnt[kBins];
    unsigned long long mass[kBins];
    uint32_t wave32[2][NT / kWave];
    unsigned long long wave64[NT / kWave];
    int bin;
    uint32_t above32;
    unsigned long long above64, at64;
    uint32_t at32;
};

// A row's keys, IT groups of four to a lane: kept in registers, or read again each time.
template <typename T, int NT, int IT, bool KEEP>
struct Row {
    const T* p;
    int64_t V;
    int64_t span0;   // first element of the wave's span
    int groups;      // groups of 256 elements in a span
    bool vec;
    uint32_t kept[KEEP ? IT * 4 : 1];

    __device__ __forceinline__ int64_t index(int it, int lane) const {
        return span0 + (int64_t)it * 256 + lane * 4;
    }
    __device__ __forceinline__ void read(int it, int lane, uint32_t (&k)[4]) const {
        const int64_t i = index(it, lane);
        if (vec && i + 4 <= V) {
            float v[4];
            unpack_vec<T, 4>(*(const typename VecT<T, 4>::type*)(p + i), v);
#pragma unroll
            for (int e = 0; e < 4; ++e) k[e] = key_of(v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) k[e] = i + e < V ? key_of(to_f32(p[i + e])) : 0u;
        }
    }
    // f(keys of four consecutive elements, group) over the wave's span; 0 stands behind the row.
    template <typename F>
    __device__ __forceinline__ void each(int lane, F f) const {
        if constexpr (KEEP) {
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                const uint32_t k[4] = {kept[4 * it], kept[4 * it + 1], kept[4 * it + 2],
                                       kept[4 * it + 3]};
                f(k, it);
            }
        } else {
            for (int it = 0; it < groups; ++it) {
                uint32_t k[4];
                read(it, lane, k);
                f(k, it);
            }
        }
    }
};

template <typename T, int NT, int IT, bool KEEP>
__global__ __launch_bounds__(NT) void sample_kernel(SampleArgs a, double scale) {
    __shared__ Shared<NT> sm;
    constexpr int NW = NT / kWave;
    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id();
    const int64_t row = blockIdx.x;
    Row<T, NT, IT, KEEP> r;
    r.p = (const T*)a.logits + row * a.V;
    r.V = a.V;
    r.vec = (((uintptr_t)r.p) % (4 * sizeof(T))) == 0;
    r.groups = KEEP ? IT : (int)((a.V + NW * 256 - 1) / (NW * 256));
    r.span0 = (int64_t)w * r.groups * 256;
    if constexpr (KEEP) {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            uint32_t k[4];
            r.read(it, lane, k);
#pragma unroll
            for (int e = 0; e < 4; ++e) r.kept[4 * it + e] = k[e];
        }
    }
    // Largest and smallest key of the row.
    uint32_t hi = 0, lo = 0xFFFFFFFFu;
    r.each(lane, [&](const uint32_t (&k)[4], int it) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool in = r.index(it, lane) + e < a.V;
            hi = in && k[e] > hi ? k[e] : hi;
            lo = in && k[e] < lo ? k[e] : lo;
        }
    });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint32_t h = (uint32_t)__shfl_xor((int)hi, d), l = (uint32_t)__shfl_xor((int)lo, d);
        hi = h > hi ? h : hi;
        lo = l < lo ? l : lo;
    }
    if (lane == 0) {
        sm.wave32[0][w] = hi;
        sm.wave32[1][w] = lo;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        hi = sm.wave32[0][i] > hi ? sm.wave32[0][i] : hi;
        lo = sm.wave32[1][i] < lo ? sm.wave32[1][i] : lo;
    }
    const float temp = a.temperature ? a.temperature[row] : 1.0f;
    if (hi <= kKeyNegInf || hi >= kKeyPosInf || lo < kKeyNegInf || !(temp == temp)) {
        if (tid == 0) {
            a.ids[row] = -1;
            if (a.prob) a.prob[row] = 0.0f;
        }
        return;
    }
    const float top_p = a.top_p ? a.top_p[row] : 1.0f;
    const float min_p = a.min_p ? fminf(a.min_p[row], 1.0f) : 0.0f;
    const bool greedy = temp <= 0.0f;
    int64_t k = a.top_k && a.top_k[row] > 0 ? a.top_k[row] : a.V;
    if (greedy || top_p <= 0.0f) k = 1;
    const RowParams rp{greedy ? 0.0 : 1.0 / (double)temp, (double)value_of(hi), scale};

    // The border: items with a key above it stay, and the first `ties` of those that have it.
    uint32_t border = 0;
    int64_t ties = 0;

    // Descends `hist(digit histogram of the keys with the given upper bits)`; the bin that
    // holds the border is chosen by `pick`.  count: by counts, else by weights.
    auto descend = [&](auto member, bool by_mass, uint64_t want_count, double want_mass,
                       uint64_t& left, uint64_t& mass_above, uint32_t& total) {
        uint32_t prefix = 0;
        int shift = 32;
        mass_above = 0;
        uint64_t count_above = 0;
        for (int round = 0; round < 3; ++round) {
            const int bits = round == 2 ? 10 : 11;
            const int sh = shift - bits;
            for (int b = tid; b < kBins; b += NT) {
                sm.cnt[b] = 0;
                sm.mass[b] = 0;
            }
            if (tid == 0) sm.bin = -1;
            __syncthreads();
            r.each(lane, [&](const uint32_t (&key)[4], int it) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool in = key[e] != 0 && member(key[e]) &&
                                    (round == 0 || (key[e] >> shift) == (prefix >> shift));
                    if (in) {
                        const uint32_t b = (key[e] >> sh) & ((1u << bits) - 1);
                        atomicAdd(&sm.cnt[b], 1u);
                        if (by_mass) {
                            const uint64_t q = fixed(weight(key[e], rp), rp);
                            if (q) atomicAdd(&sm.mass[b], (unsigned long long)q);
                        }
                    }
                }
            });
            __syncthreads();
            // Bins from the highest down, consecutive ones to a thread.
            constexpr int BPT = kBins / NT;
            uint32_t c = 0;
            uint64_t m = 0;
#pragma unroll
            for (int j = 0; j < BPT; ++j) {
                const int b = kBins - 1 - (tid * BPT + j);
                c += sm.cnt[b];
                m += sm.mass[b];
            }
            uint32_t cb = wave_before(c, lane);
            uint64_t mb = wave_before((unsigned long long)m, lane);
            if (lane == kWave - 1) {
                sm.wave32[0][w] = cb + c;
                sm.wave64[w] = mb + m;
            }
            __syncthreads();
            for (int i = 0; i < w; ++i) {
                cb += sm.wave32[0][i];
                mb += sm.wave64[i];
            }
            // The last bin, from the top, that holds items and has less than what is wanted
            // above it.
            int mine = -1;
            uint32_t c_at = 0;
            uint64_t m_at = 0;
#pragma unroll
            for (int j = 0; j < BPT; ++j) {
                const int pos = tid * BPT + j, b = kBins - 1 - pos;
                const uint32_t cnt = sm.cnt[b];
                const bool short_of = by_mass ? (double)(mass_above + mb) < want_mass
                                              : count_above + cb < want_count;
                if (cnt && short_of) {
                    mine = pos;
                    c_at = cb;
                    m_at = mb;
                }
                cb += cnt;
                mb += sm.mass[b];
            }
            if (mine >= 0) atomicMax(&sm.bin, mine);
            __syncthreads();
            if (mine >= 0 && sm.bin == mine) {
                sm.above32 = c_at;
                sm.above64 = m_at;
                sm.at32 = sm.cnt[kBins - 1 - mine];
            }
            __syncthreads();
            const uint32_t digit = (uint32_t)(kBins - 1 - sm.bin);
            prefix |= digit << sh;
            shift = sh;
            count_above += sm.above32;
            mass_above += sm.above64;
            total = sm.at32;
            __syncthreads();
        }
        left = want_count - count_above;
        return prefix;
    };

    // Sum of the weights of the items above the border and of its ties.
    auto sum_above = [&](uint32_t edge) {
        uint64_t s = 0;
        r.each(lane, [&](const uint32_t (&key)[4], int) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (key[e] > edge) s += fixed(weight(key[e], rp), rp);
        });
        s = wave_sum((unsigned long long)s);
        __syncthreads();
        if (lane == 0) sm.wave64[w] = s;
        __syncthreads();
        s = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) s += sm.wave64[i];
        return s;
    };

    uint32_t tie_total = 0;
    if (k == 1) {
        border = hi;
        ties = 1;
    } else {
        if (k < a.V) {
            uint64_t left, m;
            border = descend([](uint32_t) { return true; }, false, (uint64_t)k, 0.0, left, m,
                             tie_total);
            ties = (int64_t)left;
        }
        if (top_p < 1.0f) {
            const uint64_t above = sum_above(border);
            const uint64_t tie_w = ties ? fixed(weight(border, rp), rp) : 0;
            const double want = (double)top_p * (double)(above + tie_w * (uint64_t)ties);
            if ((double)above < want) {
                // The border lies among the ties (or nowhere, if there are none).
                if (tie_w) {
                    int64_t stay = (int64_t)ceil((want - (double)above) / (double)tie_w);
                    stay = stay < 1 ? 1 : stay;
                    while (stay > 1 &&
                           !((double)(above + tie_w * (uint64_t)(stay - 1)) < want)) --stay;
                    while (stay < ties && (double)(above + tie_w * (uint64_t)stay) < want) ++stay;
                    ties = stay < ties ? stay : ties;
                }
            } else {
                const uint32_t edge = border;
                uint64_t left, m;
                border = descend([edge](uint32_t key) { return key > edge; }, true, 0, want, left,
                                 m, tie_total);
                const uint64_t q = fixed(weight(border, rp), rp);
                ties = tie_total;
                if (q) {
                    int64_t stay = (int64_t)ceil((want - (double)m) / (double)q);
                    stay = stay < 1 ? 1 : stay;
                    while (stay > 1 && !((double)(m + q * (uint64_t)(stay - 1)) < want)) --stay;
                    while (stay < ties && (double)(m + q * (uint64_t)stay) < want) ++stay;
                    ties = stay < ties ? stay : ties;
                }
            }
        }
    }

    // How many items with the border's key lie in the spans before this wave's.
    uint32_t seen = 0;
    r.each(lane, [&](const uint32_t (&key)[4], int) {
#pragma unroll
        for (int e = 0; e < 4; ++e) seen += key[e] == border && key[e] != 0;
    });
    seen = wave_sum(seen);
    __syncthreads();
    if (lane == 0) sm.wave32[0][w] = seen;
    __syncthreads();
    int64_t before = 0;
    for (int i = 0; i < w; ++i) before += sm.wave32[0][i];

    // A kept item's weight; `rank` counts the border's items so far in order of the index.
    auto kept_weight = [&](const uint32_t (&key)[4], int64_t& rank, uint64_t (&q)[4],
                           double (&wt)[4]) {
        uint32_t tie[4], n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            tie[e] = key[e] == border && key[e] != 0;
            n += tie[e];
        }
        int64_t mine = 0;
        if (__any(n)) {
            const uint32_t lower = wave_before(n, lane);
            mine = rank + lower;
            rank += __shfl((int)(lower + n), kWave - 1);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool stays = key[e] > border || (tie[e] && mine < ties);
            mine += tie[e];
            wt[e] = 0.0;
            if (stays) {
                wt[e] = greedy ? 1.0 : weight(key[e], rp);
                if (wt[e] < (double)min_p) wt[e] = 0.0;
            }
            q[e] = fixed(wt[e], rp);
        }
    };
    uint64_t sum = 0;
    {
        int64_t rank = before;
        r.each(lane, [&](const uint32_t (&key)[4], int) {
            uint64_t q[4];
            double wt[4];
            kept_weight(key, rank, q, wt);
            sum += q[0] + q[1] + q[2] + q[3];
        });
    }
    sum = wave_sum((unsigned long long)sum);
    if (lane == 0) sm.wave64[w] = sum;
    __syncthreads();
    uint64_t all = 0, from = 0;
    int last = 0;  // the last wave with a kept item
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const uint64_t s = sm.wave64[i];
        if (i < w) from += s;
        if (s) last = i;
        all += s;
    }
    // The wave whose running sum first exceeds u times the whole, or the last one.
    const double target = (double)a.u[row] * (double)all;
    const bool past_before = (double)from > target, past = (double)(from + sum) > target;
    const bool mine = past ? !past_before && sum != 0 : false;
    const bool none = !((double)all > target);
    if (!(none ? w == last : mine)) {
        // A u below 0 takes the first kept item: its wave has nothing before it.
        if (!(target < 0.0 && from == 0 && sum != 0)) return;
    }
    {
        int64_t rank = before;
        uint64_t run = from;
        int64_t found = -1, tail = -1;
        double wf = 0.0, wl = 0.0;
        r.each(lane, [&](const uint32_t (&key)[4], int it) {
            uint64_t q[4];
            double wt[4];
            kept_weight(key, rank, q, wt);
            const uint64_t own = q[0] + q[1] + q[2] + q[3];
            uint64_t c = run + wave_before((unsigned long long)own, lane);
            run += wave_sum((unsigned long long)own);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                c += q[e];
                if (q[e]) {
                    tail = r.index(it, lane) + e;
                    wl = wt[e];
                    if (found < 0 && (double)c > target) {
                        found = tail;
                        wf = wl;
                    }
                }
            }
        });
        // The least index found by any lane; else the greatest kept one.
        const unsigned long long key_f =
            found >= 0 ? (unsigned long long)found : ~0ull;
        unsigned long long best = key_f;
        long long end = (long long)tail;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const unsigned long long o = __shfl_xor(best, d);
            const long long t = __shfl_xor(end, d);
            best = o < best ? o : best;
            end = t > end ? t : end;
        }
        const bool got = best != ~0ull;
        const int64_t id = got ? (int64_t)best : (int64_t)end;
        if (got ? found == id : tail == id) {
            a.ids[row] = (int32_t)id;
            if (a.prob) a.prob[row] = (float)((got ? wf : wl) * scale / (double)all);
        }
    }
}

// Rows without items.
__global__ void sample_none_kernel(int32_t* ids, float* prob, int64_t B) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= B) return;
    ids[i] = -1;
    if (prob) prob[i] = 0.0f;
}

template <typename T, int NT, int IT, bool KEEP>
hipError_t launch_rows(const SampleArgs& a, double scale, hipStream_t stream) {
    hipLaunchKernelGGL((sample_kernel<T, NT, IT, KEEP>), dim3((unsigned)a.B), dim3(NT), 0, stream,
                       a, scale);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const SampleArgs& a, double scale, hipStream_t stream) {
    if (a.V <= 256 * 4 * 4) return launch_rows<T, 256, 4, true>(a, scale, stream);
    if (a.V <= 1024 * 4 * 4) return launch_rows<T, 1024, 4, true>(a, scale, stream);
    return launch_rows<T, 1024, 1, false>(a, scale, stream);
}

}  // namespace

size_t sample_workspace(int64_t, int64_t, IoType) { return 0; }

hipError_t launch_sample(const SampleArgs& a, void*, hipStream_t stream) {
    if (a.V == 0) {
        hipLaunchKernelGGL(sample_none_kernel, dim3((unsigned)((a.B + 255) / 256)), dim3(256), 0,
                           stream, a.ids, a.prob, a.B);
        return hipGetLastError();
    }
    int log_v = 0;
    while (((int64_t)1 << log_v) < a.V) ++log_v;
    const double scale = (double)((uint64_t)1 << (62 - log_v));
    return a.io == IoType::kF32 ? launch_typed<float>(a, scale, stream)
                                : launch_typed<bf16>(a, scale, stream);
}

}  // namespace recblr
