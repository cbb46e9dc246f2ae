// Backward of the gated delta rule (recblr_delta_backward), 64 steps at a time.
//
// With the forward's notation (delta_fwd.hip), T = (I + A)^-1, X = V - diag(e^c) K S, U = T
// diag(beta) X, G_ij = e^{c_i - c_j}, and D the gradient of the state behind the chunk:
//   dU = scale P^T dO + diag(e^{c_63 - c}) K D,   Y = T^T dU,   dV = diag(beta) Y
//   D_before = e^{c_63} D + scale (diag(e^c) Q)^T dO - (diag(e^c) K)^T dV
// is the recurrence (delta_bwd_state_kernel, walking the chunks backwards as the forward walks
// them forwards; it keeps D and Y of every chunk).  What is left has no order
// (delta_bwd_grad_kernel, a workgroup to a chunk and query head): with F = dO U^T, Z = Y U^T,
//   dQ = scale diag(e^c) dO S^T + (scale F . G)_{j <= i} K
//   a  = -diag(e^c) Y S^T - (Z . G)_{j < i} K
//   b  = (scale F . G)^T_{i >= j} Q - (diag(beta) Z . G)^T_{i > j} K + diag(e^{c_63 - c}) U D^T
//   dK = diag(beta) a + b,   dbeta_i = Y_i.V_i + k_i.a_i
// and dg_t is the sum of the terms that step t's decay is a factor of,
//   W_ij = G_ij (scale F_ij q_i.k_j - beta_i Z_ij k_i.k_j),
//   dg_t = e^{c_63} <S, D> + sum_{i >= t} e^{c_i} (scale q_i.S dO_i - beta_i k_i.S Y_i)
//        + sum_{j < t} e^{c_63 - c_j} k_j.(D U_j) + sum_{i >= t > j} W_ij,
// so that it is as exact, for its size, as they are.  (As a running sum of dL/dc_i = q_i.dQ_i +
// beta_i k_i.a_i - k_i.b_i, which needs no W, it holds terms without that decay, of size one,
// that are meant to cancel: at g = -12 a hundredth of dg was wrong in fp32.)
//
// Both are bound by issue and latency, not by memory.  2048 heads, 200 steps, 64 x 64 bf16: the
// recurrence 313 us, the rest 506 us; 256 heads, 2048 steps fp32: 456 and 916 us (W's products are
// a seventh of the latter, by fp32 instructions).  Strips of the recurrence are 32 columns (its
// operands leave no room for 64).  The rest is eight waves on one chunk, four to a side (rows for
// dQ and a, columns for b), since one wave's half of the products fills 232 registers at 64
// columns of K; from 65 on it takes all 256 and 92 to 160 more in scratch memory.  Two such
// workgroups do not fit a CU's LDS.
#include <hip/hip_runtime.h>

#include "delta_tile.hpp"
#include "ops.hpp"

namespace recblr {
namespace {

using namespace dtile;

struct BwdWs {
    float* D;   // [B * HV][chunks][Dk][Dv]: gradient of the state behind each chunk
    float* Y;   // [B * HV][L][Dv]
    float* dq;  // [B][L][H][Dk] each: sums over value heads so far, where they share a query head
    float* dk;
    void* split;  // the workspace of delta_split.hip
};

// ------------------------------------------------------------------ the recurrence
template <typename T, int DK, int DVT>
struct StateLds {
    using E = typename Io<T>::Elem;
    static constexpr int kChain = Io<T>::kChain;
    static constexpr int kKS = DK + Io<T>::kPad, kUS = C + Io<T>::kPad, kOS = DVT + Io<T>::kPad;
    static constexpr int kDPlane = DVT * kKS, kXPlane = DVT * kUS, kOPlane = C * kOS;
    E k[C * kKS];
    E q[C * kKS];
    E d_o[kOPlane];
    E od[kChain * kOPlane];  // dO times scale e^c
    // [column][d] the gradient D; then [column][step] dU; then -e^c dV
    E x[kChain * (kDPlane > kXPlane ? kDPlane : kXPlane)];
    float tm[C * TS];
    Gates gt;
};

template <typename T, int DK, int DVT, bool VEC>
__global__ __launch_bounds__(NT, 2) void delta_bwd_state_kernel(DeltaBwdArgs a, BwdWs ws,
                                                                int strips) {
    using I = Io<T>;
    using L = StateLds<T, DK, DVT>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    L& sm = *(L*)smem;
    constexpr int NK = DK / I::kStep, NC = C / I::kStep;
    constexpr int NTL = DVT / 16, DTL = DK / 16;
    constexpr int DW = DTL < 4 ? DTL : 4, NWV = 4 / DW;
    constexpr int SD = DTL / DW, SN = NTL / NWV;
    constexpr int KU = C * DK / I::kUnit / NT, UR = DK / I::kUnit;
    constexpr int OU = C * DVT / I::kUnit / NT, OR = DVT / I::kUnit;
    static_assert(KU >= 1 && OU >= 1, "every thread stages");

    const int lane0 = threadIdx.x % kWave, w = wave_id();
    // A head's strips lie apart by the number of heads, which is a multiple of eight where there
    // are many: on one XCD, whose L2 reads K once for all.
    const unsigned heads = gridDim.x / (unsigned)strips;
    const int64_t head = blockIdx.x % heads;
    const int n0 = (int)(blockIdx.x / heads) * DVT;
    const int64_t b = head / a.HV;
    const int hv = (int)(head - b * a.HV), h = hv / (a.HV / a.H);
    const int Dk = a.Dk, Dv = a.Dv, width = Dv - n0;
    const int64_t qk_step = (int64_t)a.H * Dk, v_step = (int64_t)a.HV * Dv;
    const T* qp = (const T*)a.q + (b * a.L * a.H + h) * Dk;
    const T* kp = (const T*)a.k + (b * a.L * a.H + h) * Dk;
    const T* dop = (const T*)a.d_o + (b * a.L * a.HV + hv) * Dv + n0;
    T* dvp = (T*)a.dv + (b * a.L * a.HV + hv) * Dv + n0;
    float* yp = ws.Y + head * a.L * Dv + n0;
    const T* gp = (const T*)a.g + b * a.L * a.HV + hv;
    const T* bp = (const T*)a.beta + b * a.L * a.HV + hv;
    const int chunks = (int)((a.L + C - 1) / C);
    const int wd = w % DW, wn = w / DW;

    f4 D[SD][SN];
    auto state_d = [&](int i, int g) { return 16 * (wd + DW * i) + 4 * g; };
    auto state_n = [&](int j, int ll) { return 16 * (wn + NWV * j) + ll; };
    auto state_io = [&](const float* p, auto f) {
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
        const auto r = wtile::rsrc(p, (uint32_t)(Dk * Dv * 4));
#pragma unroll
        for (int i = 0; i < SD; ++i)
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                const int n = state_n(j, ll);
                const uint32_t o = n < width ? (uint32_t)(state_d(i, g) * Dv + n0 + n) * 4 : kNowhere;
#pragma unroll
                for (int e = 0; e < 4; ++e) f(r, D[i][j], e, (int)(o + (uint32_t)(4 * e * Dv)));
            }
    };
    auto state_store = [&](float* p) {
        state_io(p, [](auto r, f4& s, int e, int o) {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(s[e]), r, o, 0, 0);
        });
    };
    auto state_put = [&] {
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
#pragma unroll
        for (int i = 0; i < SD; ++i)
#pragma unroll
            for (int j = 0; j < SN; ++j)
                put<L::kChain>(sm.x, L::kDPlane, L::kKS, state_n(j, ll), state_d(i, g),
                               D[i][j]);
    };
#pragma unroll
    for (int i = 0; i < SD; ++i)
#pragma unroll
        for (int j = 0; j < SN; ++j) D[i][j] = f4{0, 0, 0, 0};
    if (a.dhT)
        state_io(a.dhT + head * Dk * Dv, [](auto r, f4& s, int e, int o) {
            s[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0));
        });

    wtile::u4v kn[KU], qn[KU], on[OU];
    uint32_t gn = 0, bn = 0;  // raw
    auto fetch = [&](int c) {
        const int tid = wtile::fresh(threadIdx.x);
        const Rows<T> rk(kp, (int64_t)c * C, a.L, qk_step, Dk);
        const Rows<T> rq(qp, (int64_t)c * C, a.L, qk_step, Dk);
        const Rows<T> ro(dop, (int64_t)c * C, a.L, v_step, width);
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int u = tid + i * NT;
            kn[i] = rk.template get16<VEC>(u / UR, u % UR * I::kUnit, Dk);
            qn[i] = rq.template get16<VEC>(u / UR, u % UR * I::kUnit, Dk);
        }
#pragma unroll
        for (int i = 0; i < OU; ++i) {
            const int u = tid + i * NT;
            on[i] = ro.template get16<VEC>(u / OR, u % OR * I::kUnit, width);
        }
        if (w == 0) {
            const Rows<T> rg(gp, (int64_t)c * C, a.L, a.HV, 1), rb(bp, (int64_t)c * C, a.L, a.HV, 1);
            gn = rg.raw(rg.off(lane0, 0, 1));
            bn = rb.raw(rb.off(lane0, 0, 1));
        }
    };
    if (chunks > 0) fetch(chunks - 1);

    for (int c = chunks - 1; c >= 0; --c) {
        state_store(ws.D + (head * chunks + c) * Dk * Dv);
        lds_barrier();  // what the previous chunk had in LDS has been read
        state_put();
        {
            const int tid = wtile::fresh(threadIdx.x);
#pragma unroll
            for (int i = 0; i < KU; ++i) {
                const int u = tid + i * NT, at = u / UR * L::kKS + u % UR * I::kUnit;
                *(wtile::u4v*)(sm.k + at) = kn[i];
                *(wtile::u4v*)(sm.q + at) = qn[i];
            }
#pragma unroll
            for (int i = 0; i < OU; ++i) {
                const int u = tid + i * NT;
                *(wtile::u4v*)(sm.d_o + u / OR * L::kOS + u % OR * I::kUnit) = on[i];
            }
        }
        if (w == 0)
            gates_of_chunk(&sm.gt, Rows<T>::value(gn), Rows<T>::value(bn), a.scale, lane0);
        lds_barrier();
        {
            const int tid = wtile::fresh(threadIdx.x);
#pragma unroll
            for (int i = 0; i < OU; ++i) {
                const int u = tid + i * NT, row = u / OR, n = u % OR * I::kUnit;
                const float es = sm.gt.es[row];
#pragma unroll
                for (int q4 = 0; q4 < I::kUnit / 4; ++q4) {
                    f4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (sizeof(T) == 4)
                            v[e] = es * __uint_as_float(on[i][e]);
                        else
                            v[e] = es * (e & 1 ? bf16_hi(on[i][2 * q4 + e / 2])
                                               : bf16_lo(on[i][2 * q4 + e / 2]));
                    }
                    put<L::kChain>(sm.od, L::kOPlane, L::kOS, row, n + 4 * q4, v);
                }
            }
        }
        fetch(c > 0 ? c - 1 : chunks);  // in any case, as in the forward
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;

        f4 X[NTL];
        {
            // A's strip (lane: row i = 16 w + ll, columns 16 t + 4 g ..), and the strip of P^T
            // (lane: row j = 16 w + ll, columns i = 16 t + 4 g ..) with dU = scale P^T dO + ...
            f4 M[4], PT[4], KD[NTL];
            typename I::Given kw[NK];
#pragma unroll
            for (int s = 0; s < NK; ++s) kw[s] = given(sm.k, L::kKS, 16 * w + ll, s * I::kStep, g);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                M[t] = PT[t] = f4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < NK; ++s) {
                    if (t <= w)
                        M[t] = mma(M[t], given(sm.k, L::kKS, 16 * t + ll, s * I::kStep, g), kw[s]);
                    if (t >= w)
                        PT[t] = mma(PT[t], given(sm.q, L::kKS, 16 * t + ll, s * I::kStep, g), kw[s]);
                }
            }
            const int i = 16 * w + ll;
            const double ci = sm.gt.cum[i];
            const float bi = sm.gt.bt[i];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * t + 4 * g + r;
                    const double diff = ci - sm.gt.cum[j];
                    if (t <= w) M[t][r] = j < i ? bi * M[t][r] * fast_exp2((float)diff) : 0.0f;
                    if (t >= w) PT[t][r] = j >= i ? PT[t][r] * fast_exp2((float)-diff) : 0.0f;
                }
                if (t <= (w | 1)) *(f4*)(sm.tm + i * TS + 16 * t + 4 * g) = M[t];
            }
#pragma unroll
            for (int j = 0; j < NTL; ++j) {
                X[j] = KD[j] = f4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < NK; ++s)
                    KD[j] = mma(KD[j], kw[s], made<L::kChain>(sm.x, L::kDPlane, L::kKS,
                                                              16 * j + ll, s * I::kStep, g));
            }
#pragma unroll
            for (int s = 0; s < NC; ++s)
                if ((s + 1) * I::kStep > 16 * w) {
                    const auto pt = from_acc<T, L::kChain>(PT, s);
#pragma unroll
                    for (int j = 0; j < NTL; ++j)
                        X[j] = mma(X[j], pt, given_t_acc(sm.d_o, L::kOS, s * I::kStep, 16 * j, ll, g));
                }
            const f4 el = *(const f4*)(sm.gt.el + 16 * w + 4 * g);
#pragma unroll
            for (int j = 0; j < NTL; ++j) X[j] = a.scale * X[j] + el * KD[j];
        }
        wave_fence();
        invert_diagonal(sm.tm, w, ll, g);
        lds_barrier();  // D has been read
#pragma unroll
        for (int j = 0; j < NTL; ++j)
            put<L::kChain>(sm.x, L::kXPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g, X[j]);
        invert_merge1(sm.tm, w, ll, g);
        lds_barrier();
        invert_merge2(sm.tm, w, ll, g);
        lds_barrier();
        f4 Y[NTL];
#pragma unroll
        for (int j = 0; j < NTL; ++j) Y[j] = f4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < NC; ++s)
            if ((s + 1) * I::kStep > 16 * w) {
                const auto inv = inverse_cols<T, L::kChain>(sm.tm, w, s, ll, g);
#pragma unroll
                for (int j = 0; j < NTL; ++j)
                    Y[j] = mma(Y[j], inv, made<L::kChain>(sm.x, L::kXPlane, L::kUS, 16 * j + ll,
                                                          s * I::kStep, g));
            }
        lds_barrier();  // dU has been read
        {
            const f4 bt = *(const f4*)(sm.gt.bt + 16 * w + 4 * g);
            const f4 eg = *(const f4*)(sm.gt.eg + 16 * w + 4 * g);
            const Rows<T> rv(dvp, (int64_t)c * C, a.L, v_step, width);
            const Rows<float> ry(yp, (int64_t)c * C, a.L, Dv, width);
#pragma unroll
            for (int j = 0; j < NTL; ++j) {
                const f4 dv = bt * Y[j];
                put<L::kChain>(sm.x, L::kXPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g, -eg * dv);
                const uint32_t ov = rv.off(16 * w + 4 * g, 16 * j + ll, width);
                const uint32_t oy = ry.off(16 * w + 4 * g, 16 * j + ll, width);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    rv.set(rv.next(ov, r), dv[r]);
                    ry.set(ry.next(oy, r), Y[j][r]);
                }
            }
        }
        lds_barrier();
        const float et = sm.gt.eg[C - 1];
#pragma unroll
        for (int i = 0; i < SD; ++i)
#pragma unroll
            for (int j = 0; j < SN; ++j) D[i][j] *= et;
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int i = 0; i < SD; ++i) {
                const int d0 = 16 * (wd + DW * i), k0 = s * I::kStep;
                const auto qt = given_t(sm.q, L::kKS, k0, d0, ll, g);
                const auto kt = given_t(sm.k, L::kKS, k0, d0, ll, g);
#pragma unroll
                for (int j = 0; j < SN; ++j) {
                    D[i][j] = mma(D[i][j], qt, made_t<L::kChain>(sm.od, L::kOPlane, L::kOS, k0,
                                                                 16 * (wn + NWV * j), ll, g));
                    D[i][j] = mma(D[i][j], kt, made<L::kChain>(sm.x, L::kXPlane, L::kUS,
                                                               state_n(j, ll), k0, g));
                }
            }
    }
    if (a.dh0) state_store(a.dh0 + head * Dk * Dv);
}

// ------------------------------------------------------------------ the gradients
// Eight waves: four for b and what it takes (A's inverse first), four for dQ and a.  Waves w
// and 4 + w share a SIMD and the strip of rows 16 w .., whose triangles of F and Z (j <= i for
// the one, i >= j for the other) are five tiles together for every w.
constexpr int GT = 512;

// Columns of the state at a time: what LDS takes.
template <int DK>
constexpr int kGradCols = DK <= 64 ? 64 : 32;

template <typename T, int DK>
struct GradLds {
    using E = typename Io<T>::Elem;
    static constexpr int kOut = Io<T>::kOut, kCols = kGradCols<DK>;
    static constexpr int kKS = DK + Io<T>::kPad, kUS = C + Io<T>::kPad, kNS = kCols + Io<T>::kPad;
    static constexpr int kSPlane = DK * kNS, kRPlane = kCols * kUS, kYPlane = C * kNS;
    E k[C * kKS];
    E q[C * kKS];
    E d_o[C * kNS];
    union {
        struct {
            E s[kOut * kSPlane];  // [d][column]: the state before the chunk
            E d[kOut * kSPlane];  // the gradient behind it
        };
        float dk[C * (DK + 4)];   // b, handed over at the head's end
    };
    E r[kOut * kRPlane];  // [column][step]
    E u[kOut * kYPlane];  // [step][column]
    E y[kOut * kYPlane];
    float tm[C * TS];
    Gates gt;
    float dca[C], dcb[C], db[C], part[8];
    float pairs[4 * C];  // [wave][t]: sums of W over i of the wave's strip, i >= t > j
};

__device__ __forceinline__ float whole(const float* m, int, int at) { return m[at]; }
__device__ __forceinline__ uint32_t raw_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t raw_of(bf16 v) { return v.bits; }
__device__ __forceinline__ float whole(const __bf16* m, int plane, int at) {
    return (float)m[at] + (float)m[at + plane];
}

// GROUPED: several value heads to a query head, whose sums go through the workspace.
template <typename T, int DK, bool VEC, bool GROUPED>
__global__ __launch_bounds__(GT) void delta_bwd_grad_kernel(DeltaBwdArgs a, BwdWs ws) {
    using I = Io<T>;
    using L = GradLds<T, DK>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    L& sm = *(L*)smem;
    constexpr int NTW = L::kCols;
    constexpr int NK = DK / I::kStep, NC = C / I::kStep, NN = NTW / I::kStep;
    constexpr int DTL = DK / 16, NTL = NTW / 16;
    constexpr int UR = DK / I::kUnit, OR = NTW / I::kUnit;
    constexpr int KU = (C * UR + GT - 1) / GT, OU = (C * OR + GT - 1) / GT;
    constexpr int SU = DK * NTW / 4 / GT, YU = C * NTW / 4 / GT;
    static_assert(SU >= 1 && YU >= 1, "every thread stages");

    const int lane0 = threadIdx.x % kWave;
    const int wave = wave_id(), w = wave & 3;
    const bool side_b = wave < 4;
    const int chunks = (int)((a.L + C - 1) / C);
    const int group = GROUPED ? a.HV / a.H : 1;
    const int Dk = a.Dk, Dv = a.Dv;
    const int64_t qk_step = (int64_t)a.H * Dk, v_step = (int64_t)a.HV * Dv;
    // A chunk of a query head.
    struct Item {
        int64_t b, t0, qk_base;
        int h, c;
    };
    auto item_at = [&](unsigned i) {
        const unsigned bh = i / (unsigned)chunks, b = bh / (unsigned)a.H;
        Item o;
        o.c = (int)(i - bh * (unsigned)chunks);
        o.b = b;
        o.h = (int)(bh - b * (unsigned)a.H);
        o.t0 = (int64_t)o.c * C;
        o.qk_base = (o.b * a.L * a.H + o.h) * Dk;
        return o;
    };

    // What a head's columns need of memory, on its way.
    wtile::u4v on[OU], kn[KU], qn[KU];
    f4 sn[SU], dn[SU], yn[YU];
    uint32_t gn = 0, bn = 0, vn[NTL][4];  // raw
    auto fetch = [&](const Item& it, int hv, int n0) {
        const int tid = wtile::fresh(threadIdx.x), lane = tid % kWave;
        const int64_t head = it.b * a.HV + hv;
        const int width = Dv - n0;
        const int64_t v_base = (it.b * a.L * a.HV + hv) * Dv + n0;
        const Rows<T> ro((const T*)a.d_o + v_base, it.t0, a.L, v_step, width);
        const Rows<float> ry(ws.Y + head * a.L * Dv + n0, it.t0, a.L, Dv, width);
        const int64_t at = (head * chunks + it.c) * Dk * Dv;
        const auto rs = wtile::rsrc(a.states + at, (uint32_t)(Dk * Dv * 4));
        const auto rd = wtile::rsrc(ws.D + at, (uint32_t)(Dk * Dv * 4));
#pragma unroll
        for (int i = 0; i < SU; ++i) {
            const int u = tid + i * GT, d = u / (NTW / 4), n = u % (NTW / 4) * 4;
            if constexpr (VEC) {  // Dv is a multiple of four then
                const int o = n < width ? (d * Dv + n0 + n) * 4 : (int)kNowhere;
                sn[i] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(rs, o, 0, 0));
                dn[i] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(rd, o, 0, 0));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int o = n + e < width ? (d * Dv + n0 + n + e) * 4 : (int)kNowhere;
                    sn[i][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, o, 0, 0));
                    dn[i][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rd, o, 0, 0));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < YU; ++i) {
            const int u = tid + i * GT, t = u / (NTW / 4), n = u % (NTW / 4) * 4;
            if constexpr (VEC) {  // Dv is a multiple of four then
                yn[i] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(
                                                   ry.r, (int)ry.off(t, n, width), 0, 0));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) yn[i][e] = ry.get(ry.off(t, n + e, width));
            }
        }
#pragma unroll
        for (int i = 0; i < OU; ++i) {
            const int u = tid + i * GT;
            if (C * OR % GT == 0 || u < C * OR)
                on[i] = ro.template get16<VEC>(u / OR, u % OR * I::kUnit, width);
        }
        if (!side_b) {
            const int ll = lane & 15, g = lane >> 4;
            const Rows<T> rv((const T*)a.v + v_base, it.t0, a.L, v_step, width);
#pragma unroll
            for (int j = 0; j < NTL; ++j) {
                const uint32_t o = rv.off(16 * w + 4 * g, 16 * j + ll, width);
#pragma unroll
                for (int r = 0; r < 4; ++r) vn[j][r] = rv.raw(rv.next(o, r));
            }
        }
        if (wave == 4 && n0 == 0) {
            const int64_t t = it.t0 + lane < a.L ? it.t0 + lane : a.L - 1;
            const int64_t o = (it.b * a.L + t) * a.HV + hv;
            gn = raw_of(((const T*)a.g)[o]);
            bn = raw_of(((const T*)a.beta)[o]);
        }
    };
    auto fetch_qk = [&](const Item& it) {
        const int tid = wtile::fresh(threadIdx.x);
        const Rows<T> rk((const T*)a.k + it.qk_base, it.t0, a.L, qk_step, Dk);
        const Rows<T> rq((const T*)a.q + it.qk_base, it.t0, a.L, qk_step, Dk);
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int u = tid + i * GT;
            if (C * UR % GT == 0 || u < C * UR) {
                kn[i] = rk.template get16<VEC>(u / UR, u % UR * I::kUnit, Dk);
                qn[i] = rq.template get16<VEC>(u / UR, u % UR * I::kUnit, Dk);
            }
        }
    };

    const unsigned items = (unsigned)(a.B * a.H * chunks);  // below 2^31
    Item next = item_at(blockIdx.x);
    fetch_qk(next);
    fetch(next, next.h * group, 0);
    for (unsigned at = blockIdx.x; at < items; at += gridDim.x) {
    const Item it = next;
    const int64_t b = it.b, t0 = it.t0, qk_base = it.qk_base;
    const int h = it.h;
    const bool more = at + gridDim.x < items;
    if (more) next = item_at(at + gridDim.x);
    for (int hv = h * group; hv < (h + 1) * group; ++hv) {
        // Side a: X1 = dO S^T, X2 = Y S^T; side b: X1 = U D^T (lane: column d, rows 16 w + 4 g
        // ..).  F, Z: side a has row i = 16 w + ll and columns j = 16 t + 4 g .., side b column
        // j = 16 w + ll and rows i = 16 t + 4 g ...
        f4 X1[DTL], X2[DTL], F[4], Z[4], yv = {0, 0, 0, 0};
        float sd = 0.0f;
#pragma unroll
        for (int i = 0; i < DTL; ++i) X1[i] = X2[i] = f4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < 4; ++t) F[t] = Z[t] = f4{0, 0, 0, 0};

        for (int n0 = 0; n0 < Dv; n0 += NTW) {
            const int width = Dv - n0;
            lds_barrier();  // the previous columns' operands, or head's decays, have been read
            if (wave == 4 && n0 == 0)
                gates_of_chunk(&sm.gt, t0 + lane0 < a.L ? Rows<T>::value(gn) : 0.0f,
                               t0 + lane0 < a.L ? Rows<T>::value(bn) : 0.0f, a.scale, lane0);
            const int tid = wtile::fresh(threadIdx.x);
            if (n0 == 0 && hv == h * group) {
#pragma unroll
                for (int i = 0; i < KU; ++i) {
                    const int u = tid + i * GT, o = u / UR * L::kKS + u % UR * I::kUnit;
                    if (C * UR % GT == 0 || u < C * UR) {
                        *(wtile::u4v*)(sm.k + o) = kn[i];
                        *(wtile::u4v*)(sm.q + o) = qn[i];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < OU; ++i) {
                const int u = tid + i * GT;
                if (C * OR % GT == 0 || u < C * OR)
                    *(wtile::u4v*)(sm.d_o + u / OR * L::kNS + u % OR * I::kUnit) = on[i];
            }
#pragma unroll
            for (int i = 0; i < SU; ++i) {
                const int u = tid + i * GT, d = u / (NTW / 4), n = u % (NTW / 4) * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (n + e >= width) sn[i][e] = dn[i][e] = 0.0f;
                    sd = fmaf(sn[i][e], dn[i][e], sd);
                }
                put<L::kOut>(sm.s, L::kSPlane, L::kNS, d, n, sn[i]);
                put<L::kOut>(sm.d, L::kSPlane, L::kNS, d, n, dn[i]);
            }
#pragma unroll
            for (int i = 0; i < YU; ++i) {
                const int u = tid + i * GT, t = u / (NTW / 4), n = u % (NTW / 4) * 4;
                put<L::kOut>(sm.y, L::kYPlane, L::kNS, t, n, yn[i]);
            }
            lds_barrier();
            // The next operands' reads are started behind the first use of this one's V.
            auto fetch_next = [&] {
                if (n0 + NTW < Dv) {
                    fetch(it, hv, n0 + NTW);
                } else if (hv + 1 < (h + 1) * group) {
                    fetch(it, hv + 1, 0);
                } else if (more) {
                    fetch_qk(next);
                    fetch(next, next.h * group, 0);
                }
            };

            if (side_b) {
                if (n0 == 0) {
                    const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
                    f4 M[4];
                    const int i = 16 * w + ll;
                    const double ci = sm.gt.cum[i];
                    const float bi = sm.gt.bt[i];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        M[t] = f4{0, 0, 0, 0};
                        if (t <= w) {
#pragma unroll
                            for (int s = 0; s < NK; ++s)
                                M[t] = mma(M[t], given(sm.k, L::kKS, 16 * t + ll, s * I::kStep, g),
                                           given(sm.k, L::kKS, 16 * w + ll, s * I::kStep, g));
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int j = 16 * t + 4 * g + r;
                                M[t][r] = j < i ? bi * M[t][r] *
                                                      fast_exp2((float)(ci - sm.gt.cum[j]))
                                                : 0.0f;
                            }
                        }
                        if (t <= (w | 1)) *(f4*)(sm.tm + i * TS + 16 * t + 4 * g) = M[t];
                    }
                    wave_fence();
                    invert_diagonal(sm.tm, w, ll, g);
                }
            } else {
                const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
                const f4 eg = *(const f4*)(sm.gt.eg + 16 * w + 4 * g);
                const f4 bt = *(const f4*)(sm.gt.bt + 16 * w + 4 * g);
                f4 KS[NTL];
#pragma unroll
                for (int j = 0; j < NTL; ++j) KS[j] = f4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < NK; ++s) {
                    const auto kw = given(sm.k, L::kKS, 16 * w + ll, s * I::kStep, g);
#pragma unroll
                    for (int j = 0; j < NTL; ++j)
                        KS[j] = mma(KS[j], kw, made_t<L::kOut>(sm.s, L::kSPlane, L::kNS,
                                                               s * I::kStep, 16 * j, ll, g));
                    step_end(KS[0]);
                }
#pragma unroll
                for (int j = 0; j < NTL; ++j) {
                    f4 R;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float y = whole(sm.y, L::kYPlane,
                                              (16 * w + 4 * g + r) * L::kNS + 16 * j + ll);
                        const float v = Rows<T>::value(vn[j][r]);
                        yv[r] = fmaf(y, v, yv[r]);
                        R[r] = bt[r] * (v - eg[r] * KS[j][r]);
                    }
                    put<L::kOut>(sm.r, L::kRPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g, R);
                }
            }
            fetch_next();
            lds_barrier();
            if (n0 == 0) {
                const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
                if (side_b) invert_merge1(sm.tm, w, ll, g);
                lds_barrier();
                if (side_b) invert_merge2(sm.tm, w, ll, g);
            }
            if (!side_b) {
                const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
#pragma unroll
                for (int s = 0; s < NN; ++s) {
                    const int k0 = s * I::kStep;
                    const auto ow = given(sm.d_o, L::kNS, 16 * w + ll, k0, g);
                    const auto yw = made<L::kOut>(sm.y, L::kYPlane, L::kNS, 16 * w + ll, k0, g);
#pragma unroll
                    for (int i = 0; i < DTL; ++i) {
                        const auto st = made<L::kOut>(sm.s, L::kSPlane, L::kNS, 16 * i + ll, k0, g);
                        X1[i] = mma(X1[i], ow, st);
                        X2[i] = mma(X2[i], yw, st);
                        if (i & 1) step_end(X2[i]);
                    }
                }
            }
            if (n0 == 0) lds_barrier();
            // U, half of the columns by each side.
            const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
#pragma unroll
            for (int jj = 0; jj < NTL / 2; ++jj) {
                const int j = jj + (side_b ? 0 : NTL / 2);
                f4 U = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < NC; ++s)
                    if (s * I::kStep < 16 * (w + 1))
                        U = mma(U, made<L::kOut>(sm.r, L::kRPlane, L::kUS, 16 * j + ll,
                                                 s * I::kStep, g),
                                inverse_rows<T, L::kOut>(sm.tm, w, s, ll, g));
                put<L::kOut>(sm.u, L::kYPlane, L::kNS, 16 * w + ll, 16 * j + 4 * g, U);
            }
            lds_barrier();
#pragma unroll
            for (int s = 0; s < NN; ++s) {
                const int k0 = s * I::kStep;
                if (side_b) {
                    const auto uw = made<L::kOut>(sm.u, L::kYPlane, L::kNS, 16 * w + ll, k0, g);
#pragma unroll
                    for (int i = 0; i < DTL; ++i) {
                        X1[i] = mma(X1[i], uw, made<L::kOut>(sm.d, L::kSPlane, L::kNS,
                                                             16 * i + ll, k0, g));
                        if (i & 1) step_end(X1[i]);
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (t >= w) {
                            F[t] = mma(F[t], given(sm.d_o, L::kNS, 16 * t + ll, k0, g), uw);
                            Z[t] = mma(Z[t], made<L::kOut>(sm.y, L::kYPlane, L::kNS, 16 * t + ll,
                                                           k0, g), uw);
                            step_end(Z[t]);
                        }
                } else {
                    const auto ow = given(sm.d_o, L::kNS, 16 * w + ll, k0, g);
                    const auto yw = made<L::kOut>(sm.y, L::kYPlane, L::kNS, 16 * w + ll, k0, g);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (t <= w) {
                            const auto ut = made<L::kOut>(sm.u, L::kYPlane, L::kNS, 16 * t + ll,
                                                          k0, g);
                            F[t] = mma(F[t], ut, ow);
                            Z[t] = mma(Z[t], ut, yw);
                            step_end(Z[t]);
                        }
                }
            }
        }
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
        {
            const int own = 16 * w + ll;
            const double co = sm.gt.cum[own];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int o = 16 * t + 4 * g + r;
                    const double diff = co - sm.gt.cum[o];
                    if (side_b) {
                        const float e = o >= own ? fast_exp2((float)-diff) : 0.0f;
                        F[t][r] = o >= own ? a.scale * F[t][r] * e : 0.0f;
                        Z[t][r] = o > own ? -sm.gt.bt[o] * Z[t][r] * e : 0.0f;
                    } else {
                        const float e = o <= own ? fast_exp2((float)diff) : 0.0f;
                        F[t][r] = o <= own ? a.scale * F[t][r] * e : 0.0f;
                        Z[t][r] = o < own ? -Z[t][r] * e : 0.0f;
                    }
                }
        }
        // W's sums over j < t for each t of a row i, then over the rows i >= t of the strip.
        if (!side_b) {
            const int own = 16 * w + ll;
            const float bi = sm.gt.bt[own];
            float before = 0.0f;  // of the tiles so far
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t <= w) {
                    f4 QK = {0, 0, 0, 0}, KK = QK, upto;
#pragma unroll
                    for (int s = 0; s < NK; ++s) {
                        const auto kt = given(sm.k, L::kKS, 16 * t + ll, s * I::kStep, g);
                        QK = mma(QK, kt, given(sm.q, L::kKS, 16 * w + ll, s * I::kStep, g));
                        KK = mma(KK, kt, given(sm.k, L::kKS, 16 * w + ll, s * I::kStep, g));
                    }
                    float sum = 0.0f;  // of the lane's four columns
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        upto[r] = sum;
                        if (16 * t + 4 * g + r < own)
                            sum += fmaf(F[t][r], QK[r], bi * Z[t][r] * KK[r]);
                    }
                    // The row's four lanes lie 16 apart.
                    const float x16 = __shfl_xor(sum, 16), two = sum + x16;
                    const float x32 = __shfl_xor(two, 32);
                    const float base = before + ((g & 1 ? x16 : 0.0f) + (g & 2 ? x32 : 0.0f));
                    before += two + x32;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        upto[r] = lanes::row_sum(16 * t + 4 * g + r <= own ? base + upto[r] : 0.0f);
                    if (ll == 0) *(f4*)(sm.pairs + w * C + 16 * t + 4 * g) = upto;
                    step_end(upto);
                }
        }
        typename I::template Made<L::kOut> fo[NC], zo[NC];
#pragma unroll
        for (int s = 0; s < NC; ++s) {
            fo[s] = from_acc<T, L::kOut>(F, s);
            zo[s] = from_acc<T, L::kOut>(Z, s);
        }
        lds_barrier();  // S and D have been read: b may take their place
        // The value heads of a query head come one after the other: their sum stands in the
        // workspace as float until the last one (written and read by the same lane).
        const bool first = !GROUPED || hv == h * group;
        const bool last = !GROUPED || hv + 1 == (h + 1) * group;
        auto emit = [&](const f4& v, void* out, float* part, int i, int ll, int g) {
            const Rows<T> ro((T*)out + qk_base, t0, a.L, qk_step, Dk);
            const Rows<float> rp(part + qk_base, t0, a.L, qk_step, Dk);
            const uint32_t oo = ro.off(16 * w + 4 * g, 16 * i + ll, Dk);
            const uint32_t op = rp.off(16 * w + 4 * g, 16 * i + ll, Dk);
            f4 x = v;
            if (!first) {
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] += rp.get(rp.next(op, r));
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (last) ro.set(ro.next(oo, r), x[r]);
                else rp.set(rp.next(op, r), x[r]);
            }
        };
        f4 x1 = {0, 0, 0, 0}, x2 = x1, KA[DTL];
        if (side_b) {
            const f4 el = *(const f4*)(sm.gt.el + 16 * w + 4 * g);
#pragma unroll
            for (int i = 0; i < DTL; ++i) {
                const f4 ud = el * X1[i];
                f4 kb = ud;
#pragma unroll
                for (int s = 0; s < NC; ++s) {
                    const int k0 = s * I::kStep;
                    kb = mma(kb, fo[s], given_t_acc(sm.q, L::kKS, k0, 16 * i, ll, g));
                    kb = mma(kb, zo[s], given_t_acc(sm.k, L::kKS, k0, 16 * i, ll, g));
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float kv = (float)sm.k[(16 * w + 4 * g + r) * L::kKS + 16 * i + ll];
                    x1[r] = fmaf(kv, ud[r], x1[r]);
                    sm.dk[(16 * w + 4 * g + r) * (DK + 4) + 16 * i + ll] = kb[r];
                }
                step_end(kb);
            }
        } else {
            const f4 eg = *(const f4*)(sm.gt.eg + 16 * w + 4 * g);
            const f4 bt = *(const f4*)(sm.gt.bt + 16 * w + 4 * g);
#pragma unroll
            for (int i = 0; i < DTL; ++i) {
                f4 q = a.scale * eg * X1[i], ka = -eg * X2[i], kv;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = (16 * w + 4 * g + r) * L::kKS + 16 * i + ll;
                    kv[r] = (float)sm.k[at];
                    x1[r] = fmaf((float)sm.q[at], q[r], fmaf(bt[r] * kv[r], ka[r], x1[r]));
                }
                step_end(x1);
#pragma unroll
                for (int s = 0; s < NC; ++s) {
                    const auto kt = given_t_acc(sm.k, L::kKS, s * I::kStep, 16 * i, ll, g);
                    q = mma(q, fo[s], kt);
                    ka = mma(ka, zo[s], kt);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) x2[r] = fmaf(kv[r], ka[r], x2[r]);
                emit(q, a.dq, ws.dq, i, ll, g);
                KA[i] = bt * ka;
                step_end(KA[i]);
            }
        }
        // The rows' sums: side b's of k.(D U), side a's of the state's terms and of k.a.
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * w + 4 * g + r;
            const float s1 = lanes::row_sum(x1[r]);
            if (side_b) {
                if (ll == 0) sm.dcb[i] = s1;
            } else {
                const float s2 = lanes::row_sum(x2[r]), sy = lanes::row_sum(yv[r]);
                if (ll == 0) {
                    sm.dca[i] = s1;
                    sm.db[i] = sy + s2;
                }
            }
        }
        sd = lanes::wave_sum(sm.gt.eg[C - 1] * sd);
        if (lane == 0) sm.part[wave] = sd;
        lds_barrier();
        if (wave == 0) {
            // A step to a lane: the sums from it on (the last step first, they are a scan) and the
            // sums before it.
            const float from = __shfl(lanes::wave_upto(sm.dca[C - 1 - lane]), C - 1 - lane);
            float s = from + lanes::wave_upto(lane ? sm.dcb[lane - 1] : 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += sm.part[j];
#pragma unroll
            for (int j = 0; j < 4; ++j) s += lane < 16 * (j + 1) ? sm.pairs[j * C + lane] : 0.0f;
            const int64_t t = t0 + lane;
            if (t < a.L) {
                const int64_t at = (b * a.L + t) * a.HV + hv;
                store((T*)a.dg + at, s);
                store((T*)a.dbeta + at, sm.db[lane]);
            }
        }
        if (!side_b) {
#pragma unroll
            for (int i = 0; i < DTL; ++i) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    KA[i][r] += sm.dk[(16 * w + 4 * g + r) * (DK + 4) + 16 * i + ll];
                emit(KA[i], a.dk, ws.dk, i, ll, g);
            }
        }
    }
    }
}

// ------------------------------------------------------------------ launches
template <typename T, int DK, int DVT, bool VEC>
hipError_t launch_state(const DeltaBwdArgs& a, const BwdWs& ws, hipStream_t stream) {
    static std::atomic<uint64_t> lds_set{0};
    constexpr int bytes = (int)sizeof(StateLds<T, DK, DVT>);
    const hipError_t e = allow_dynamic_lds(
        (const void*)delta_bwd_state_kernel<T, DK, DVT, VEC>, bytes, lds_set);
    if (e != hipSuccess) return e;
    const int strips = (a.Dv + DVT - 1) / DVT;
    hipLaunchKernelGGL((delta_bwd_state_kernel<T, DK, DVT, VEC>),
                       dim3((unsigned)(a.B * a.HV * strips)), dim3(NT), bytes, stream, a, ws,
                       strips);
    return hipGetLastError();
}
template <typename T, int DK, bool VEC, bool GROUPED>
hipError_t launch_grad(const DeltaBwdArgs& a, const BwdWs& ws, hipStream_t stream) {
    const int64_t chunks = (a.L + C - 1) / C;
    if (chunks == 0) return hipSuccess;
    static std::atomic<uint64_t> lds_set{0};
    constexpr int bytes = (int)sizeof(GradLds<T, DK>);
    static_assert(bytes <= 160 * 1024, "LDS of a compute unit");
    const hipError_t e =
        allow_dynamic_lds((const void*)delta_bwd_grad_kernel<T, DK, VEC, GROUPED>, bytes, lds_set);
    if (e != hipSuccess) return e;
    // As many workgroups as the chip holds; each takes chunks until there are no more, with the
    // next one's reads on their way.
    const int64_t items = a.B * a.H * chunks, fit = 256 * (160 * 1024 / bytes);
    hipLaunchKernelGGL((delta_bwd_grad_kernel<T, DK, VEC, GROUPED>),
                       dim3((unsigned)(items < fit ? items : fit)), dim3(GT), bytes, stream, a,
                       ws);
    return hipGetLastError();
}

template <typename T, int DK>
hipError_t launch_both(const DeltaBwdArgs& a, const BwdWs& ws, bool vec, hipStream_t stream) {
    size_t bytes;
    const hipError_t e = delta_split(a.B * a.HV, a.L, a.Dk, a.Dv, true)
                             ? launch_delta_split_backward(a, ws.D, ws.Y, ws.split, &bytes, stream)
                         : vec ? launch_state<T, DK, 32, true>(a, ws, stream)
                               : launch_state<T, DK, 32, false>(a, ws, stream);
    if (e != hipSuccess) return e;
    const bool grouped = a.HV > a.H;
    return vec ? grouped ? launch_grad<T, DK, true, true>(a, ws, stream)
                         : launch_grad<T, DK, true, false>(a, ws, stream)
           : grouped ? launch_grad<T, DK, false, true>(a, ws, stream)
                     : launch_grad<T, DK, false, false>(a, ws, stream);
}

template <typename T>
hipError_t launch_typed(const DeltaBwdArgs& a, const BwdWs& ws, hipStream_t stream) {
    const auto at16 = [](const void* p) { return (uintptr_t)p % 16 == 0; };
    const bool vec = a.Dk * sizeof(T) % 16 == 0 && a.Dv * sizeof(T) % 16 == 0 && at16(a.q) &&
                     at16(a.k) && at16(a.d_o);
    if (a.Dk <= 32) return launch_both<T, 32>(a, ws, vec, stream);
    if (a.Dk <= 64) return launch_both<T, 64>(a, ws, vec, stream);
    return launch_both<T, 128>(a, ws, vec, stream);
}

size_t round_up(size_t v) { return (v + 255) / 256 * 256; }
size_t state_bytes(int64_t B, int64_t L, int64_t HV, int Dk, int Dv) {
    return round_up((size_t)(B * HV * ((L + C - 1) / C) * Dk * Dv) * 4);
}

size_t y_bytes(int64_t B, int64_t L, int64_t HV, int Dv) {
    return round_up((size_t)(B * HV * L * Dv) * 4);
}
size_t sum_bytes(int64_t B, int64_t L, int64_t H, int Dk) {
    return round_up((size_t)(B * L * H * Dk) * 4);
}

}  // namespace

size_t delta_backward_workspace(int64_t B, int64_t L, int64_t H, int64_t HV, int Dk, int Dv,
                                IoType io) {
    size_t split = 0;
    if (delta_split(B * HV, L, Dk, Dv, true)) {
        DeltaBwdArgs a{};
        a.B = B;
        a.L = L;
        a.H = (int)H;
        a.HV = (int)HV;
        a.Dk = Dk;
        a.Dv = Dv;
        a.io = io;
        (void)launch_delta_split_backward(a, nullptr, nullptr, nullptr, &split, nullptr);
    }
    return state_bytes(B, L, HV, Dk, Dv) + y_bytes(B, L, HV, Dv) +
           (HV > H ? 2 * sum_bytes(B, L, H, Dk) : 0) + split;
}

hipError_t launch_delta_backward(const DeltaBwdArgs& a, void* ws, hipStream_t stream) {
    char* p = (char*)ws;
    auto take = [&](size_t n) {
        char* r = p;
        p += n;
        return r;
    };
    BwdWs s{};
    s.D = (float*)take(state_bytes(a.B, a.L, a.HV, a.Dk, a.Dv));
    s.Y = (float*)take(y_bytes(a.B, a.L, a.HV, a.Dv));
    if (a.HV > a.H) {
        s.dq = (float*)take(sum_bytes(a.B, a.L, a.H, a.Dk));
        s.dk = (float*)take(sum_bytes(a.B, a.L, a.H, a.Dk));
    }
    s.split = p;
    return a.io == IoType::kF32 ? launch_typed<float>(a, s, stream)
                                : launch_typed<bf16>(a, s, stream);
}

}  // namespace recblr
