// The gated delta rule for few heads and long sequences.
//
// The one-kernel walk (delta_fwd.hip, the recurrence of delta_bwd.hip) gives a head's strip of
// columns one workgroup, whose every chunk costs some 7 to 9 us of latency: with few strips
// the chip is idle but for those.  Here everything that does not hang on the state is done for
// all chunks at once, so that the walk is left with
//     X = X0 + W S,    S' = e^{c_63} S + Z + K^T diag(f) X
// two products and two exchanges through LDS a chunk.  With T = (I + A)^-1 (delta_fwd.hip):
//   forward:  X = U,  X0 = T diag(beta) V,  W = -T diag(beta e^c) K,  f = e^{c_63 - c},  Z = 0;
//   backward (chunks from the last to the first, S the gradient D):  X = Y,
//     X0 = scale T^T P^T dO,  W = T^T diag(e^{c_63 - c}) K,  f = -beta e^c,
//     Z = scale (diag(e^c) Q)^T dO.
// W and K^T are written as the walk's operands (a lane's 16 bytes next to its neighbour's), X0
// and Z as its accumulators, so that it reads them straight into registers, two chunks ahead.
// The forward's outputs o = scale (diag(e^c) Q S + P U) follow for all chunks at once.
//
// 4 heads, 16384 steps, 128 x 128 bf16: preparation 40 and 65 us (backward), the two walks of
// segments 71 + 76 and 84 + 89 us, joining them 23 us each way, outputs 55 us.  The walks are
// bound by the latency of their two exchanges a chunk, the others by issue.
#include <hip/hip_runtime.h>

#include "delta_tile.hpp"
#include "ops.hpp"

namespace recblr {
namespace {

using namespace dtile;

constexpr int SC = 16;  // columns of the state to a workgroup of the walk

template <typename T>
struct Frag {
    static constexpr int kPlanes = Io<T>::kChain;                      // of W
    static constexpr int kBytes = kWave * 16;                          // one operand, one plane
};
// Bytes of a chunk's W and K^T at DK padded columns: kStep columns are 4 strips of operands.
template <typename T, int DK>
constexpr int kWBytes = 4 * (DK / Io<T>::kStep) * Frag<T>::kPlanes * Frag<T>::kBytes;
template <typename T, int DK>
constexpr int kKBytes = (DK / 16) * (C / Io<T>::kStep) * Frag<T>::kBytes;

struct SplitWs {
    char* W;
    char* KT;
    float* X0;   // [item][strip][wave][lane][4]
    float* Z;    // [item][strip][d tile][lane][4], backward only
    float* f;    // [item][64]
    float* et;   // [item]
    float* bt;   // [item][64], backward only
    float* X;    // [head][L][Dv]
    float* S;    // [item][Dk][Dv]
    float *psi, *phi, *starts;  // of a walk in segments
};

// What the two preparations share: K's chunk and the decays in LDS, the inverse in tm.
template <typename T, int DK>
struct PrepLds {
    using E = typename Io<T>::Elem;
    static constexpr int kChain = Io<T>::kChain;
    static constexpr int kKS = DK + Io<T>::kPad, kUS = C + Io<T>::kPad, kCols = 32;
    static constexpr int kNS = kCols + Io<T>::kPad, kXPlane = kCols * kUS;
    E k[C * kKS];
    E q[C * kKS];       // backward only
    E v[C * kNS];       // columns of V, or of dO
    union {
        E x[kChain * kXPlane];      // P^T dO
        E od[kChain * C * kNS];     // dO times scale e^c
    };
    float tm[C * TS];
    Gates gt;
};

template <typename T, int DK, bool VEC>
__device__ __forceinline__ void stage_rows(typename Io<T>::Elem* to, int stride, const Rows<T>& r,
                                           int cols, int width, int tid) {
    const int ur = cols / Io<T>::kUnit;
    for (int u = tid; u < C * ur; u += NT)
        *(wtile::u4v*)(to + u / ur * stride + u % ur * Io<T>::kUnit) =
            r.template get16<VEC>(u / ur, u % ur * Io<T>::kUnit, width);
}

// A's strip of wave w and the inverse, with the barriers that it takes.
template <typename T, int DK, typename L>
__device__ __forceinline__ void form_inverse(L& sm, int w, int ll, int g) {
    using I = Io<T>;
    const int i = 16 * w + ll;
    const double ci = sm.gt.cum[i];
    const float bi = sm.gt.bt[i];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        f4 M = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < DK / I::kStep; ++s)
            M = mma(M, given(sm.k, L::kKS, 16 * t + ll, s * I::kStep, g),
                    given(sm.k, L::kKS, 16 * w + ll, s * I::kStep, g));
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int j = 16 * t + 4 * g + r;
            M[r] = j < i ? bi * M[r] * fast_exp2((float)(ci - sm.gt.cum[j])) : 0.0f;
        }
        *(f4*)(sm.tm + i * TS + 16 * t + 4 * g) = M;
    }
    wave_fence();
    invert_diagonal(sm.tm, w, ll, g);
    lds_barrier();
    invert_merge1(sm.tm, w, ll, g);
    lds_barrier();
    invert_merge2(sm.tm, w, ll, g);
    lds_barrier();
}

// Rows of the inverse (or of its transpose) with column k times f[k].
template <typename T, bool TRANS>
__device__ __forceinline__ typename Io<T>::template Made<Io<T>::kChain> inverse_scaled(
    const float* tm, const float* f, int i, int s, int ll, int g) {
    if constexpr (sizeof(T) == 4) {
        const f4 v = (TRANS ? inverse_cols<T, 1>(tm, i, s, ll, g) : inverse_rows<T, 1>(tm, i, s, ll, g)).v;
        return F32Op{v * *(const f4*)(f + s * 16 + 4 * g)};
    } else {
        float x[8];
        const float* t = TRANS ? tile_at(tm, 2 * s + (g >> 1), i) + 8 * (g & 1) * TS + ll
                               : tile_at(tm, i, 2 * s + (g >> 1)) + ll * TS + 8 * (g & 1);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = t[TRANS ? e * TS : e] * f[s * 32 + 8 * g + e];
        return split<Io<T>::kChain>(x);
    }
}
// Whether step s holds tiles on the inverse's triangle for strip w.
template <typename T, bool TRANS>
__device__ __forceinline__ bool on_triangle(int w, int s) {
    return TRANS ? (s + 1) * Io<T>::kStep > 16 * w : s * Io<T>::kStep < 16 * (w + 1);
}

// W's strip as operands: rows 16 w .., times sign; and K^T, each wave every fourth of its tiles.
template <typename T, int DK, bool TRANS, typename L>
__device__ __forceinline__ void write_operands(L& sm, const float* f, float sign, char* W, char* KT,
                                               int w, int lane) {
    using I = Io<T>;
    constexpr int NK = DK / I::kStep, NC = C / I::kStep, P = I::kChain, DTL = DK / 16;
    const int ll = lane & 15, g = lane >> 4;
    typename I::template Made<P> inv[NC];
#pragma unroll
    for (int s = 0; s < NC; ++s)
        if (on_triangle<T, TRANS>(w, s)) inv[s] = inverse_scaled<T, TRANS>(sm.tm, f, w, s, ll, g);
#pragma unroll
    for (int k = 0; k < NK; ++k) {
        constexpr int TP = I::kStep / 16;  // tiles to an operand
        f4 acc[TP];
#pragma unroll
        for (int t = 0; t < TP; ++t) {
            acc[t] = f4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < NC; ++s)
                if (on_triangle<T, TRANS>(w, s))
                    acc[t] = mma(acc[t], given_t(sm.k, L::kKS, s * I::kStep,
                                                 k * I::kStep + 16 * t, ll, g), inv[s]);
            acc[t] *= sign;
        }
        const auto op = from_acc<T, P>(acc, 0);
        char* to = W + ((w * NK + k) * P) * Frag<T>::kBytes + lane * 16;
        if constexpr (sizeof(T) == 4) {
            *(f4*)to = op.v;
        } else {
#pragma unroll
            for (int p = 0; p < P; ++p) *(b8*)(to + p * Frag<T>::kBytes) = op.p[p];
        }
    }
    for (int u = w; u < DTL * NC; u += 4) {
        const auto op = given_t(sm.k, L::kKS, u % NC * I::kStep, 16 * (u / NC), ll, g);
        char* to = KT + u * Frag<T>::kBytes + lane * 16;
        if constexpr (sizeof(T) == 4) *(f4*)to = op.v;
        else *(b8*)to = op.p[0];
    }
}

struct Place {
    int64_t head, item;
    int64_t b, t0;
    int h, hv, c;
};
__device__ __forceinline__ Place place_of(unsigned block, int chunks, int H, int HV) {
    Place p;
    const unsigned head = block / (unsigned)chunks;
    p.item = block;
    p.head = head;
    p.c = (int)(block - head * (unsigned)chunks);
    p.b = head / (unsigned)HV;
    p.hv = (int)(head - (unsigned)p.b * (unsigned)HV);
    p.h = p.hv / (HV / H);
    p.t0 = (int64_t)p.c * C;
    return p;
}

struct SplitArgs {
    const void* q;
    const void* k;
    const void* v;    // V, or dO
    const void* g;
    const void* beta;
    int64_t B, L;
    int H, HV, Dk, Dv, chunks, strips;
    float scale;
};

template <typename T, int DK, bool BWD, bool VEC>
__global__ __launch_bounds__(NT) void delta_prep_kernel(SplitArgs a, SplitWs ws) {
    using I = Io<T>;
    using L = PrepLds<T, DK>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    L& sm = *(L*)smem;
    constexpr int NK = DK / I::kStep, NC = C / I::kStep, NTL = L::kCols / 16, DTL = DK / 16;
    constexpr int P = I::kChain;
    const int tid = threadIdx.x, lane0 = tid % kWave, w = wave_id();
    const Place p = place_of(blockIdx.x, a.chunks, a.H, a.HV);
    const int64_t qk_step = (int64_t)a.H * a.Dk, v_step = (int64_t)a.HV * a.Dv;
    const int64_t qk_base = (p.b * a.L * a.H + p.h) * a.Dk;
    stage_rows<T, DK, VEC>(sm.k, L::kKS, Rows<T>((const T*)a.k + qk_base, p.t0, a.L, qk_step, a.Dk),
                           DK, a.Dk, tid);
    if constexpr (BWD)
        stage_rows<T, DK, VEC>(sm.q, L::kKS,
                               Rows<T>((const T*)a.q + qk_base, p.t0, a.L, qk_step, a.Dk), DK,
                               a.Dk, tid);
    if (w == 0) {
        const int64_t t = p.t0 + lane0, at = (p.b * a.L + t) * a.HV + p.hv;
        gates_of_chunk(&sm.gt, t < a.L ? to_f32(((const T*)a.g)[at]) : 0.0f,
                       t < a.L ? to_f32(((const T*)a.beta)[at]) : 0.0f, a.scale, lane0);
        wave_fence();
        // What a step's row of W is made of, in place of es, and the walk's f.
        const float eg = sm.gt.eg[lane0], el = sm.gt.el[lane0], bt = sm.gt.bt[lane0];
        ws.f[p.item * C + lane0] = BWD ? -bt * eg : el;
        if (BWD) ws.bt[p.item * C + lane0] = bt;
        if (lane0 == 0) ws.et[p.item] = sm.gt.eg[C - 1];
        if (!BWD) sm.gt.es[lane0] = bt * eg;
    }
    lds_barrier();
    {
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
        form_inverse<T, DK>(sm, w, ll, g);
        write_operands<T, DK, BWD>(sm, BWD ? sm.gt.el : sm.gt.es, BWD ? 1.0f : -1.0f,
                                   ws.W + p.item * kWBytes<T, DK>, ws.KT + p.item * kKBytes<T, DK>,
                                   w, lane);
    }
    // P^T's strip of rows j = 16 w + ll, columns 16 t + 4 g ...
    f4 PT[4];
    if constexpr (BWD) {
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
        const int j = 16 * w + ll;
        const double cj = sm.gt.cum[j];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            PT[t] = f4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < NK; ++s)
                PT[t] = mma(PT[t], given(sm.q, L::kKS, 16 * t + ll, s * I::kStep, g),
                            given(sm.k, L::kKS, 16 * w + ll, s * I::kStep, g));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + 4 * g + r;
                PT[t][r] = i >= j ? PT[t][r] * fast_exp2((float)(sm.gt.cum[i] - cj)) : 0.0f;
            }
        }
    }
    for (int n0 = 0; n0 < a.Dv; n0 += L::kCols) {
        const int width = a.Dv - n0;
        const Rows<T> rv((const T*)a.v + (p.b * a.L * a.HV + p.hv) * a.Dv + n0, p.t0, a.L, v_step,
                         width);
        lds_barrier();
        stage_rows<T, DK, VEC>(sm.v, L::kNS, rv, L::kCols, width, tid);
        lds_barrier();
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
        f4 X[NTL];
        if constexpr (!BWD) {
#pragma unroll
            for (int j = 0; j < NTL; ++j) X[j] = f4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < NC; ++s)
                if (on_triangle<T, false>(w, s)) {
                    const auto inv = inverse_scaled<T, false>(sm.tm, sm.gt.bt, w, s, ll, g);
#pragma unroll
                    for (int j = 0; j < NTL; ++j)
                        X[j] = mma(X[j], inv, given_t(sm.v, L::kNS, s * I::kStep, 16 * j, ll, g));
                }
        } else {
            // Z first: dO times scale e^c has X's place until it is read.
            for (int u = tid; u < C * L::kCols / 4; u += NT) {
                const int row = u / (L::kCols / 4), n = u % (L::kCols / 4) * 4;
                const float es = sm.gt.es[row];
                f4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = es * (float)sm.v[row * L::kNS + n + e];
                put<P>(sm.od, C * L::kNS, L::kNS, row, n, v);
            }
#pragma unroll
            for (int j = 0; j < NTL; ++j) {
                X[j] = f4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < NC; ++s)
                    X[j] = mma(X[j], from_acc<T, P>(PT, s),
                               given_t_acc(sm.v, L::kNS, s * I::kStep, 16 * j, ll, g));
                X[j] *= a.scale;
            }
            lds_barrier();
            for (int u = w; u < DTL * NTL; u += 4) {
                const int dt = u / NTL, j = u % NTL;
                f4 z = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < NC; ++s)
                    z = mma(z, given_t(sm.q, L::kKS, s * I::kStep, 16 * dt, ll, g),
                            made_t<P>(sm.od, C * L::kNS, L::kNS, s * I::kStep, 16 * j, ll, g));
                const int strip = n0 / SC + j;
                if (strip < a.strips)
                    *(f4*)(ws.Z + (((p.item * a.strips + strip) * DTL + dt) * kWave + lane) * 4) = z;
            }
            lds_barrier();
#pragma unroll
            for (int j = 0; j < NTL; ++j)
                put<P>(sm.x, L::kXPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g, X[j]);
            lds_barrier();
#pragma unroll
            for (int j = 0; j < NTL; ++j) X[j] = f4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < NC; ++s)
                if (on_triangle<T, true>(w, s)) {
                    const auto inv = inverse_cols<T, P>(sm.tm, w, s, ll, g);
#pragma unroll
                    for (int j = 0; j < NTL; ++j)
                        X[j] = mma(X[j], inv, made<P>(sm.x, L::kXPlane, L::kUS, 16 * j + ll,
                                                      s * I::kStep, g));
                }
        }
#pragma unroll
        for (int j = 0; j < NTL; ++j) {
            const int strip = n0 / SC + j;
            if (strip < a.strips)
                *(f4*)(ws.X0 + (((p.item * a.strips + strip) * 4 + w) * kWave + lane) * 4) = X[j];
        }
    }
}

// ------------------------------------------------------------------ the walk
// The walk is linear in the state that it starts from, so a long one is cut into segments of
// consecutive chunks: each segment is first walked from nothing (Psi, its end state) and without
// inputs from the columns of the unit matrix (Phi), the segments' starts follow one from the
// other as S_{i+1} = Phi_i S_i + Psi_i, and then all segments are walked at once.
struct WalkArgs {
    const float* s0;    // may be null; of a cut walk, [head][segment][Dk][Dv]
    float* s_end;       // may be null
    float* S;           // the state before each chunk (behind it, backwards)
    void* dv;           // backward: dV = beta Y
    int64_t L;
    int HV, Dk, Dv, chunks, strips;
    int segments, per;  // chunks of a segment
    float* psi;         // [head][segment][Dk][Dv]
    float* phi;         // [head][segment][Dk][Dk]
};

// PROBE: Psi and Phi of every segment but the last (of a walk, the last in its order); strips
// behind the state's own are Phi's.
template <typename T, int DK, bool BWD, bool PROBE>
__global__ __launch_bounds__(NT, 2) void delta_walk_kernel(WalkArgs a, SplitWs ws) {
    using I = Io<T>;
    using E = typename I::Elem;
    constexpr int P = I::kChain, NK = DK / I::kStep, NC = C / I::kStep, DTL = DK / 16;
    constexpr int SD = DTL < 4 ? 1 : DTL / 4;
    constexpr int kKS = DK + I::kPad, kUS = C + I::kPad;
    constexpr int kSPlane = SC * kKS, kXPlane = SC * kUS;
    __shared__ __attribute__((aligned(16))) E sS[P * kSPlane];
    __shared__ __attribute__((aligned(16))) E sX[P * kXPlane];
    const int lane = threadIdx.x % kWave, ll = lane & 15, g = lane >> 4, w = wave_id();
    // Workgroup: (strip, head, segment), so that the strips of a segment, which read the same W
    // and K^T, are a multiple of eight workgroups apart where there are enough: on one XCD, whose
    // L2 reads them once (strips next to each other: 108 us for 103).
    const int all_strips = PROBE ? a.strips + (a.Dk + SC - 1) / SC : a.strips;
    const int walked = PROBE ? a.segments - 1 : a.segments;
    const unsigned lines = gridDim.x / (unsigned)all_strips;
    const unsigned hs = blockIdx.x % lines;
    const unsigned head = hs / (unsigned)walked;
    const int segment = (int)(hs - head * (unsigned)walked);
    const int at_strip = (int)(blockIdx.x / lines);
    const bool unit = PROBE && at_strip >= a.strips;  // Phi's
    const int strip = unit ? 0 : at_strip;
    const int n0 = (unit ? at_strip - a.strips : strip) * SC;
    const int cols = unit ? a.Dk : a.Dv, width = cols - n0;
    const int first = segment * a.per;
    const int count = first + a.per < a.chunks ? a.per : a.chunks - first;
    const bool has_d = DTL >= 4 || w < DTL;
    const int64_t b = head / (unsigned)a.HV, hv = head - b * a.HV;

    struct In {
        typename I::template Made<P> w[NK];
        typename I::Given kt[SD][NC];
        f4 x0, f, z[SD], bt;
        float et;
    };
    auto fetch = [&](In& in, int c) {
        const int64_t item = (int64_t)head * a.chunks + c;
        const char* W = ws.W + item * kWBytes<T, DK> + (w * NK * P) * Frag<T>::kBytes + lane * 16;
        const char* KT = ws.KT + item * kKBytes<T, DK> + lane * 16;
#pragma unroll
        for (int s = 0; s < NK; ++s) {
            if constexpr (sizeof(T) == 4) {
                in.w[s].v = *(const f4*)(W + s * Frag<T>::kBytes);
            } else {
#pragma unroll
                for (int p = 0; p < P; ++p)
                    in.w[s].p[p] = *(const b8*)(W + (s * P + p) * Frag<T>::kBytes);
            }
        }
        in.x0 = *(const f4*)(ws.X0 + (((item * a.strips + strip) * 4 + w) * kWave + lane) * 4);
        in.f = *(const f4*)(ws.f + item * C + 16 * w + 4 * (lane >> 4));
        in.et = ws.et[item];
        if (PROBE && unit) in.x0 = f4{0, 0, 0, 0};
        if (has_d) {
#pragma unroll
            for (int i = 0; i < SD; ++i) {
                const int dt = w + 4 * i;
#pragma unroll
                for (int s = 0; s < NC; ++s) {
                    if constexpr (sizeof(T) == 4)
                        in.kt[i][s].v = *(const f4*)(KT + (dt * NC + s) * Frag<T>::kBytes);
                    else
                        in.kt[i][s].p[0] = *(const b8*)(KT + (dt * NC + s) * Frag<T>::kBytes);
                }
                if constexpr (BWD) {
                    in.z[i] = *(const f4*)(ws.Z + (((item * a.strips + strip) * DTL + dt) * kWave +
                                                   lane) * 4);
                    if (PROBE && unit) in.z[i] = f4{0, 0, 0, 0};
                }
            }
        }
        if constexpr (BWD && !PROBE) in.bt = *(const f4*)(ws.bt + item * C + 16 * w + 4 * g);
    };

    f4 S[SD];
    auto state_io = [&](const float* p, auto f) {
        const auto r = wtile::rsrc(p, (uint32_t)(a.Dk * cols * 4));
        if (has_d) {
#pragma unroll
            for (int i = 0; i < SD; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t o = ll < width ? (uint32_t)((16 * (w + 4 * i) + 4 * g + e) * cols +
                                                               n0 + ll) * 4
                                                  : kNowhere;
                    f(r, S[i], e, (int)o);
                }
        }
    };
    auto state_store = [&](float* p) {
        state_io(p, [](auto r, f4& s, int e, int o) {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(s[e]), r, o, 0, 0);
        });
    };
    auto state_put = [&] {
        if (has_d) {
#pragma unroll
            for (int i = 0; i < SD; ++i)
                put<P>(sS, kSPlane, kKS, ll, 16 * (w + 4 * i) + 4 * g, S[i]);
        }
    };
    const int64_t state = (int64_t)a.Dk * a.Dv;
    auto chunk_at = [&](int i) { return BWD ? a.chunks - 1 - first - i : first + i; };
    auto step = [&](In& in, int c) {
        f4 x[2] = {in.x0, {0, 0, 0, 0}};
#pragma unroll
        for (int s = 0; s < NK; ++s)
            x[s & 1] = mma(x[s & 1], in.w[s], made_acc<P>(sS, kSPlane, kKS, ll, s * I::kStep, g));
        const f4 X = x[0] + x[1];
        put<P>(sX, kXPlane, kUS, ll, 16 * w + 4 * g, in.f * X);
        lds_barrier();
        if constexpr (!PROBE) state_store(a.S + ((int64_t)head * a.chunks + c) * state);
        if (has_d) {
#pragma unroll
            for (int i = 0; i < SD; ++i) {
                if constexpr (BWD) S[i] = in.et * S[i] + in.z[i];
                else S[i] *= in.et;
#pragma unroll
                for (int s = 0; s < NC; ++s)
                    S[i] = mma(S[i], in.kt[i][s], made<P>(sX, kXPlane, kUS, ll, s * I::kStep, g));
            }
        }
        state_put();
        lds_barrier();
        if constexpr (!PROBE) {
            const Rows<float> rx(ws.X + (int64_t)head * a.L * a.Dv + n0, (int64_t)c * C, a.L, a.Dv,
                                 width);
#pragma unroll
            for (int r = 0; r < 4; ++r) rx.set(rx.off(16 * w + 4 * g + r, ll, width), X[r]);
            if constexpr (BWD) {
                const Rows<T> rv((T*)a.dv + (b * a.L * a.HV + hv) * a.Dv + n0, (int64_t)c * C, a.L,
                                 (int64_t)a.HV * a.Dv, width);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    rv.set(rv.off(16 * w + 4 * g + r, ll, width), in.bt[r] * X[r]);
            }
        }
    };

#pragma unroll
    for (int i = 0; i < SD; ++i) S[i] = f4{0, 0, 0, 0};
    // Two chunks' operands are on their way.  Reads behind the last chunk are of that one again:
    // a read under a condition would have every wait reckon with the branch that has none.
    const int last = count - 1;
    In one, two;
    fetch(one, chunk_at(0));
    fetch(two, chunk_at(last < 1 ? last : 1));
    if (PROBE && unit && has_d) {
#pragma unroll
        for (int i = 0; i < SD; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                S[i][e] = 16 * (w + 4 * i) + 4 * g + e == n0 + ll ? 1.0f : 0.0f;
    }
    const int64_t start = a.segments > 1 ? (int64_t)head * a.segments + segment : (int64_t)head;
    if (!PROBE && a.s0)
        state_io(a.s0 + start * state, [](auto r, f4& s, int e, int o) {
            s[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0));
        });
    state_put();
    lds_barrier();
    for (int i = 0; i < last; i += 2) {
        step(one, chunk_at(i));
        fetch(one, chunk_at(i + 2 < last ? i + 2 : last));
        step(two, chunk_at(i + 1));
        fetch(two, chunk_at(i + 3 < last ? i + 3 : last));
    }
    if (count & 1) step(one, chunk_at(last));
    if constexpr (PROBE) {
        const int64_t at = (int64_t)head * a.segments + segment;
        state_store(unit ? a.phi + at * a.Dk * a.Dk : a.psi + at * state);
    } else {
        if (a.s_end && segment == a.segments - 1) state_store(a.s_end + (int64_t)head * state);
    }
}

// The segments' starts of one head's strip, one from the other.
template <typename T, int DK>
__global__ __launch_bounds__(NT) void delta_join_kernel(WalkArgs a, float* starts) {
    using I = Io<T>;
    using E = typename I::Elem;
    constexpr int P = I::kChain, NK = DK / I::kStep, DTL = DK / 16, SD = DTL < 4 ? 1 : DTL / 4;
    constexpr int kKS = DK + I::kPad, kSPlane = SC * kKS;
    __shared__ __attribute__((aligned(16))) E sS[P * kSPlane];
    const int lane = threadIdx.x % kWave, ll = lane & 15, g = lane >> 4, w = wave_id();
    const unsigned head = blockIdx.x / (unsigned)a.strips;
    const int n0 = (int)(blockIdx.x - head * (unsigned)a.strips) * SC, width = a.Dv - n0;
    const bool has_d = DTL >= 4 || w < DTL;
    const int64_t state = (int64_t)a.Dk * a.Dv;
    f4 S[SD];
    auto offset = [&](int i, int e) {
        return ll < width ? ((16 * (w + 4 * i) + 4 * g + e) * a.Dv + n0 + ll) * 4 : (int)kNowhere;
    };
    auto read = [&](const float* p, int i) {
        const auto r = wtile::rsrc(p, (uint32_t)(state * 4));
        f4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, offset(i, e), 0, 0));
        return v;
    };
#pragma unroll
    for (int i = 0; i < SD; ++i) {
        S[i] = f4{0, 0, 0, 0};
        if (a.s0 && has_d) S[i] = read(a.s0 + (int64_t)head * state, i);
    }
    constexpr int N = I::kStep / 4;  // a lane's values of a step
    const bool vec = a.Dk % N == 0;
    float x[SD][NK][N];
    f4 psi[SD];
    auto fetch = [&](int seg) {
        const int64_t at = (int64_t)head * a.segments + seg;
        const auto phi = wtile::rsrc(a.phi + at * a.Dk * a.Dk, (uint32_t)(a.Dk * a.Dk * 4));
#pragma unroll
        for (int i = 0; i < SD; ++i) {
            psi[i] = read(a.psi + at * state, i);
            const int row = 16 * (w + 4 * i) + ll;
#pragma unroll
            for (int s = 0; s < NK; ++s) {
                const int d0 = s * I::kStep + N * g;
                if (vec) {
                    const int o = d0 < a.Dk ? (row * a.Dk + d0) * 4 : (int)kNowhere;
#pragma unroll
                    for (int e = 0; e < N; e += 4) {
                        const f4 v = __builtin_bit_cast(
                            f4, __builtin_amdgcn_raw_buffer_load_b128(phi, o + 4 * e, 0, 0));
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[i][s][e + j] = v[j];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        x[i][s][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
                            phi, d0 + e < a.Dk ? (row * a.Dk + d0 + e) * 4 : (int)kNowhere, 0, 0));
                }
            }
        }
    };
    if (has_d && a.segments > 1) fetch(0);
    for (int seg = 0; seg < a.segments; ++seg) {
        const int64_t at = (int64_t)head * a.segments + seg;
        if (has_d) {
            const auto r = wtile::rsrc(starts + at * state, (uint32_t)(state * 4));
#pragma unroll
            for (int i = 0; i < SD; ++i) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[i][e]), r, offset(i, e),
                                                          0, 0);
                put<P>(sS, kSPlane, kKS, ll, 16 * (w + 4 * i) + 4 * g, S[i]);
            }
        }
        lds_barrier();
        if (seg + 1 < a.segments && has_d) {
            typename I::template Made<P> op[SD][NK];
#pragma unroll
            for (int i = 0; i < SD; ++i) {
                S[i] = psi[i];
#pragma unroll
                for (int s = 0; s < NK; ++s) {
                    if constexpr (sizeof(T) == 4)
                        op[i][s] = F32Op{{x[i][s][0], x[i][s][1], x[i][s][2], x[i][s][3]}};
                    else
                        op[i][s] = split<P>(x[i][s]);
                }
            }
            // The last one has no Phi; what is read in its place is not used.
            fetch(seg + 2 < a.segments ? seg + 1 : seg);
#pragma unroll
            for (int s = 0; s < NK; ++s) {
                const auto st = made<P>(sS, kSPlane, kKS, ll, s * I::kStep, g);
#pragma unroll
                for (int i = 0; i < SD; ++i) S[i] = mma(S[i], op[i][s], st);
            }
        }
        lds_barrier();
    }
}

// ------------------------------------------------------------------ the outputs
template <typename T, int DK>
struct OutLds {
    using E = typename Io<T>::Elem;
    static constexpr int kOut = Io<T>::kOut, kCols = 32;
    static constexpr int kKS = DK + Io<T>::kPad, kUS = C + Io<T>::kPad, kNS = kCols + Io<T>::kPad;
    static constexpr int kSPlane = DK * kNS, kUPlane = C * kNS;
    E k[C * kKS];
    E s[kOut * kSPlane];  // [d][column]
    E u[kOut * kUPlane];  // [step][column]
    Gates gt;
};

template <typename T, int DK, bool VEC>
__global__ __launch_bounds__(NT) void delta_out_kernel(SplitArgs a, const float* S, const float* U,
                                                       void* out) {
    using I = Io<T>;
    using L = OutLds<T, DK>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    L& sm = *(L*)smem;
    constexpr int NK = DK / I::kStep, NC = C / I::kStep, NTL = L::kCols / 16;
    const int tid = threadIdx.x, lane0 = tid % kWave, w = wave_id();
    const Place p = place_of(blockIdx.x, a.chunks, a.H, a.HV);
    const int64_t qk_step = (int64_t)a.H * a.Dk, v_step = (int64_t)a.HV * a.Dv;
    const int64_t qk_base = (p.b * a.L * a.H + p.h) * a.Dk;
    const Rows<T> rq((const T*)a.q + qk_base, p.t0, a.L, qk_step, a.Dk);
    typename I::Given qw[NK];
    {
        const int ll = lane0 & 15, g = lane0 >> 4;
#pragma unroll
        for (int s = 0; s < NK; ++s)
            qw[s] = __builtin_bit_cast(
                typename I::Given,
                rq.template get16<VEC>(16 * w + ll, s * I::kStep + I::kUnit * g, a.Dk));
    }
    stage_rows<T, DK, VEC>(sm.k, L::kKS, Rows<T>((const T*)a.k + qk_base, p.t0, a.L, qk_step, a.Dk),
                           DK, a.Dk, tid);
    if (w == 0) {
        const int64_t t = p.t0 + lane0, at = (p.b * a.L + t) * a.HV + p.hv;
        gates_of_chunk(&sm.gt, t < a.L ? to_f32(((const T*)a.g)[at]) : 0.0f, 0.0f, a.scale, lane0);
    }
    lds_barrier();
    f4 Pw[4];
    {
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
        const int i = 16 * w + ll;
        const double ci = sm.gt.cum[i];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            Pw[t] = f4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < NK; ++s)
                Pw[t] = mma(Pw[t], given(sm.k, L::kKS, 16 * t + ll, s * I::kStep, g), qw[s]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = 16 * t + 4 * g + r;
                Pw[t][r] = j <= i ? a.scale * Pw[t][r] * fast_exp2((float)(ci - sm.gt.cum[j])) : 0.0f;
            }
        }
    }
    const auto rs = wtile::rsrc(S + p.item * a.Dk * a.Dv, (uint32_t)(a.Dk * a.Dv * 4));
    for (int n0 = 0; n0 < a.Dv; n0 += L::kCols) {
        const int width = a.Dv - n0;
        const Rows<float> ru(U + p.head * a.L * a.Dv + n0, p.t0, a.L, a.Dv, width);
        lds_barrier();
        for (int u = tid; u < DK * L::kCols / 4; u += NT) {
            const int d = u / (L::kCols / 4), n = u % (L::kCols / 4) * 4;
            f4 s;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
                    rs, n + e < width ? (d * a.Dv + n0 + n + e) * 4 : (int)kNowhere, 0, 0));
            put<L::kOut>(sm.s, L::kSPlane, L::kNS, d, n, s);
        }
        for (int u = tid; u < C * L::kCols / 4; u += NT) {
            const int t = u / (L::kCols / 4), n = u % (L::kCols / 4) * 4;
            f4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = ru.get(ru.off(t, n + e, width));
            put<L::kOut>(sm.u, L::kUPlane, L::kNS, t, n, x);
        }
        lds_barrier();
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
        const f4 es = *(const f4*)(sm.gt.es + 16 * w + 4 * g);
        const Rows<T> ro((T*)out + (p.b * a.L * a.HV + p.hv) * a.Dv + n0, p.t0, a.L, v_step, width);
#pragma unroll
        for (int j = 0; j < NTL; ++j) {
            f4 O = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < NK; ++s)
                O = mma(O, qw[s], made_t<L::kOut>(sm.s, L::kSPlane, L::kNS, s * I::kStep, 16 * j,
                                                  ll, g));
            O *= es;
#pragma unroll
            for (int s = 0; s < NC; ++s) {
                // P's columns have the order of accumulators.
                typename I::template Made<L::kOut> ut;
                if constexpr (sizeof(T) == 4) {
                    ut = given_t_acc(sm.u, L::kNS, s * I::kStep, 16 * j, ll, g);
                } else {
#pragma unroll
                    for (int pl = 0; pl < L::kOut; ++pl)
                        ut.p[pl] = given_t_acc(sm.u + pl * L::kUPlane, L::kNS, s * I::kStep, 16 * j,
                                               ll, g).p[0];
                }
                O = mma(O, from_acc<T, L::kOut>(Pw, s), ut);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
                ro.set(ro.off(16 * w + 4 * g + r, 16 * j + ll, width), O[r]);
        }
    }
}

// ------------------------------------------------------------------ launches
size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

// Segments of a walk of `chunks` by `strips` workgroups in all: as many as give every compute
// unit one workgroup (the walk of 16384 steps of 4 heads: 103 us so, 108 us with two), and none
// shorter than 8 chunks (cutting costs each segment a second walk and Phi's columns).
int segments_of(int64_t chunks, int64_t strips) {
    const int64_t most = chunks / 8, want = 256 / strips;
    const int64_t n = most < want ? most : want;
    return n < 3 ? 1 : (int)(n < 64 ? n : 64);
}

// Layout of the workspace; `bytes` in all.
template <typename T, int DK>
SplitWs layout(char* p, int64_t heads, int64_t L, int64_t chunks, int Dk, int Dv, bool bwd,
               bool own_x, bool own_s, size_t* bytes) {
    const size_t items = (size_t)(heads * chunks), strips = (size_t)((Dv + SC - 1) / SC);
    size_t at = 0;
    auto take = [&](size_t n) {
        char* r = p + at;
        at += round_up(n);
        return r;
    };
    SplitWs ws{};
    ws.W = take(items * kWBytes<T, DK>);
    ws.KT = take(items * kKBytes<T, DK>);
    ws.X0 = (float*)take(items * strips * 4 * kWave * 16);
    if (bwd) ws.Z = (float*)take(items * strips * (DK / 16) * kWave * 16);
    ws.f = (float*)take(items * C * 4);
    ws.et = (float*)take(items * 4);
    if (bwd) ws.bt = (float*)take(items * C * 4);
    if (own_x) ws.X = (float*)take((size_t)(heads * L * Dv) * 4);
    if (own_s) ws.S = (float*)take(items * Dk * Dv * 4);
    const int64_t segs = segments_of(chunks, heads * (int64_t)strips);
    if (segs > 1) {
        ws.psi = (float*)take((size_t)(heads * segs) * Dk * Dv * 4);
        ws.phi = (float*)take((size_t)(heads * segs) * Dk * Dk * 4);
        ws.starts = (float*)take((size_t)(heads * segs) * Dk * Dv * 4);
    }
    *bytes = at;
    return ws;
}

template <typename K>
hipError_t lds(K kernel, int bytes, std::atomic<uint64_t>& set) {
    return bytes > 64 * 1024 ? allow_dynamic_lds((const void*)kernel, bytes, set) : hipSuccess;
}

template <typename T, int DK, bool BWD, bool VEC>
hipError_t launch_prep(const SplitArgs& a, const SplitWs& ws, hipStream_t stream) {
    static std::atomic<uint64_t> set{0};
    constexpr int bytes = (int)sizeof(PrepLds<T, DK>);
    const hipError_t e = lds(delta_prep_kernel<T, DK, BWD, VEC>, bytes, set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((delta_prep_kernel<T, DK, BWD, VEC>),
                       dim3((unsigned)(a.B * a.HV * a.chunks)), dim3(NT), bytes, stream, a, ws);
    return hipGetLastError();
}
template <typename T, int DK, bool BWD>
hipError_t launch_walk(WalkArgs a, int64_t heads, const SplitWs& ws, hipStream_t stream) {
    a.segments = segments_of(a.chunks, heads * a.strips);
    a.per = (a.chunks + a.segments - 1) / a.segments;
    a.segments = (a.chunks + a.per - 1) / a.per;
    if (a.segments > 1) {
        a.psi = ws.psi;
        a.phi = ws.phi;
        const int64_t strips = a.strips + (a.Dk + SC - 1) / SC;
        hipLaunchKernelGGL((delta_walk_kernel<T, DK, BWD, true>),
                           dim3((unsigned)(heads * (a.segments - 1) * strips)), dim3(NT), 0, stream,
                           a, ws);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((delta_join_kernel<T, DK>), dim3((unsigned)(heads * a.strips)), dim3(NT),
                           0, stream, a, ws.starts);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.s0 = ws.starts;
    }
    hipLaunchKernelGGL((delta_walk_kernel<T, DK, BWD, false>),
                       dim3((unsigned)(heads * a.segments * a.strips)), dim3(NT), 0, stream, a, ws);
    return hipGetLastError();
}

template <typename T, int DK>
hipError_t forward(const DeltaFwdArgs& a, void* p, size_t* bytes, hipStream_t stream) {
    const int64_t heads = a.B * a.HV, chunks = (a.L + C - 1) / C;
    // The workspace always has room for the states: whether the caller keeps them is not known
    // when its size is asked for.
    SplitWs ws = layout<T, DK>((char*)p, heads, a.L, chunks, a.Dk, a.Dv, false, true, true, bytes);
    if (!p) return hipSuccess;
    if (a.states) ws.S = a.states;
    const int strips = (a.Dv + SC - 1) / SC;
    const SplitArgs s{a.q, a.k, a.v, a.g, a.beta, a.B, a.L, a.H, a.HV, a.Dk, a.Dv, (int)chunks,
                      strips, a.scale};
    const bool vec = a.Dk * sizeof(T) % 16 == 0 && a.Dv * sizeof(T) % 16 == 0 &&
                     (uintptr_t)a.q % 16 == 0 && (uintptr_t)a.k % 16 == 0 &&
                     (uintptr_t)a.v % 16 == 0;
    hipError_t e = vec ? launch_prep<T, DK, false, true>(s, ws, stream)
                       : launch_prep<T, DK, false, false>(s, ws, stream);
    if (e != hipSuccess) return e;
    e = launch_walk<T, DK, false>(WalkArgs{a.h0, a.hT, ws.S, nullptr, a.L, a.HV, a.Dk, a.Dv,
                                           (int)chunks, strips, 1, 0, nullptr, nullptr},
                                  heads, ws, stream);
    if (e != hipSuccess) return e;
    static std::atomic<uint64_t> set[2];
    constexpr int out_bytes = (int)sizeof(OutLds<T, DK>);
    const dim3 grid((unsigned)(heads * chunks));
    if (vec) {
        e = lds(delta_out_kernel<T, DK, true>, out_bytes, set[0]);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((delta_out_kernel<T, DK, true>), grid, dim3(NT), out_bytes, stream, s,
                           ws.S, ws.X, a.o);
    } else {
        e = lds(delta_out_kernel<T, DK, false>, out_bytes, set[1]);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((delta_out_kernel<T, DK, false>), grid, dim3(NT), out_bytes, stream, s,
                           ws.S, ws.X, a.o);
    }
    return hipGetLastError();
}

template <typename T, int DK>
hipError_t backward(const DeltaBwdArgs& a, float* D, float* Y, void* p, size_t* bytes,
                    hipStream_t stream) {
    const int64_t heads = a.B * a.HV, chunks = (a.L + C - 1) / C;
    SplitWs ws = layout<T, DK>((char*)p, heads, a.L, chunks, a.Dk, a.Dv, true, false, false, bytes);
    if (!p) return hipSuccess;
    ws.X = Y;
    ws.S = D;
    const int strips = (a.Dv + SC - 1) / SC;
    const SplitArgs s{a.q, a.k, a.d_o, a.g, a.beta, a.B, a.L, a.H, a.HV, a.Dk, a.Dv, (int)chunks,
                      strips, a.scale};
    const bool vec = a.Dk * sizeof(T) % 16 == 0 && a.Dv * sizeof(T) % 16 == 0 &&
                     (uintptr_t)a.q % 16 == 0 && (uintptr_t)a.k % 16 == 0 &&
                     (uintptr_t)a.d_o % 16 == 0;
    const hipError_t e = vec ? launch_prep<T, DK, true, true>(s, ws, stream)
                             : launch_prep<T, DK, true, false>(s, ws, stream);
    if (e != hipSuccess) return e;
    return launch_walk<T, DK, true>(WalkArgs{a.dhT, a.dh0, ws.S, a.dv, a.L, a.HV, a.Dk,
                                             a.Dv, (int)chunks, strips, 1, 0, nullptr, nullptr},
                                    heads, ws, stream);
}

template <typename F>
hipError_t by_type(IoType io, int Dk, F f) {
    if (io == IoType::kF32) {
        if (Dk <= 32) return f(float{}, std::integral_constant<int, 32>{});
        if (Dk <= 64) return f(float{}, std::integral_constant<int, 64>{});
        return f(float{}, std::integral_constant<int, 128>{});
    }
    if (Dk <= 32) return f(bf16{}, std::integral_constant<int, 32>{});
    if (Dk <= 64) return f(bf16{}, std::integral_constant<int, 64>{});
    return f(bf16{}, std::integral_constant<int, 128>{});
}

}  // namespace

// Which way is the faster one.  What is done here for all chunks at once costs more than the same
// within the one-kernel walk (operands go through memory), so this way gains only what that walk
// leaves idle: where the strips of 16 columns are no more than the two workgroups a compute unit
// that run at once, the heads no more than half of the units, and the chunks enough to pay for two
// or three launches (and, from 65 columns of K on, for the wider operands of the forward).
// One kernel and this way, bf16, forward / gradients with the backward, us:
//   4 heads, 16384 steps, 128 x 128     1625 and 228  /  2287 and 401
//   96 heads, 1000 steps, 64 x 64        120 and  89  /   213 and 180
//   96 heads, 128 steps, 64 x 64          19 and  32  /    39 and  47
//   192 heads, 1000 steps, 64 x 64       121 and 192  /   322 and 379
//   48 heads, 200 steps, 128 x 128        30 and  51  /    82 and  83
//   8192 heads, 200 steps, 64 x 64       619 and 2610 /  2937 and 4872
// Over 1158 sizes of both types the choice is 0.4% slower than always the faster one, at most 1.5
// times (32-bit 128 x 32, 200 steps).
bool delta_split(int64_t heads, int64_t L, int Dk, int Dv, bool backward) {
    const int64_t chunks = (L + C - 1) / C, strips = heads * ((Dv + SC - 1) / SC);
    return chunks >= (Dk > 64 && !backward ? 7 : 4) && heads <= 128 && strips <= 512;
}

hipError_t launch_delta_split_forward(const DeltaFwdArgs& a, void* ws, size_t* bytes,
                                      hipStream_t stream) {
    return by_type(a.io, a.Dk, [&](auto t, auto dk) {
        return forward<decltype(t), decltype(dk)::value>(a, ws, bytes, stream);
    });
}

hipError_t launch_delta_split_backward(const DeltaBwdArgs& a, float* D, float* Y, void* ws,
                                       size_t* bytes, hipStream_t stream) {
    return by_type(a.io, a.Dk, [&](auto t, auto dk) {
        return backward<decltype(t), decltype(dk)::value>(a, D, Y, ws, bytes, stream);
    });
}

}  // namespace recblr
