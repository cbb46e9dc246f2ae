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
// and, since every factor e^{c_i - c_j} stands with q_i or k_i on one side and k_j on the other,
//   dc_i = q_i.dQ_i + beta_i k_i.a_i - k_i.b_i,
//   dc_63 += e^{c_63} <S, D> + sum_i e^{c_63 - c_i} k_i.(D U_i),    dg_t = sum_{i >= t} dc_i.
#include <hip/hip_runtime.h>

#include "delta_tile.hpp"
#include "ops.hpp"

namespace recblr {
namespace {

using namespace dtile;

struct BwdWs {
    float* D;  // [B * HV][chunks][Dk][Dv]: gradient of the state behind each chunk
    float* Y;  // [B * HV][L][Dv]
};

// ------------------------------------------------------------------ the recurrence
template <typename T, int DK, int DVT>
struct StateLds {
    using E = typename Io<T>::Elem;
    static constexpr int kKS = DK + Io<T>::kPad, kUS = C + Io<T>::kPad, kOS = DVT + Io<T>::kPad;
    static constexpr int kDPlane = DVT * kKS, kXPlane = DVT * kUS;
    E k[C * kKS];
    E q[C * kKS];
    E d_o[C * kOS];
    E d[Io<T>::kPlanes * kDPlane];  // [column][d]
    E x[Io<T>::kPlanes * kXPlane];  // [column][step]: dU, then -dV
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
    const int64_t head = blockIdx.x / strips;
    const int n0 = (int)(blockIdx.x - head * strips) * DVT;
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
            for (int j = 0; j < SN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int n = state_n(j, ll);
                    const uint32_t o = n < width ? (uint32_t)((state_d(i, g) + e) * Dv + n0 + n) * 4
                                                 : kNowhere;
                    f(r, D[i][j], e, (int)o);
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
                put(sm.d, L::kDPlane, L::kKS, state_n(j, ll), state_d(i, g), D[i][j]);
    };
#pragma unroll
    for (int i = 0; i < SD; ++i)
#pragma unroll
        for (int j = 0; j < SN; ++j) D[i][j] = f4{0, 0, 0, 0};
    if (a.dhT)
        state_io(a.dhT + head * Dk * Dv, [](auto r, f4& s, int e, int o) {
            s[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0));
        });
    state_put();

    wtile::u4v kn[KU], qn[KU], on[OU];
    float gn = 0.0f, bn = 0.0f;
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
            const int64_t t = (int64_t)c * C + lane0;
            gn = t < a.L ? to_f32(gp[t * a.HV]) : 0.0f;
            bn = t < a.L ? to_f32(bp[t * a.HV]) : 0.0f;
        }
    };
    if (chunks > 0) fetch(chunks - 1);

    for (int c = chunks - 1; c >= 0; --c) {
        state_store(ws.D + (head * chunks + c) * Dk * Dv);
        lds_barrier();  // the previous chunk's K, Q and dO have been read
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
        if (w == 0) gates_of_chunk(&sm.gt, gn, bn, a.scale, lane0);
        lds_barrier();
        if (c > 0) fetch(c - 1);
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;

        {
            // A's strip (lane: row i = 16 w + ll, columns 16 t + 4 g ..), and the strip of P^T
            // (lane: row j = 16 w + ll, columns i = 16 t + 4 g ..) with dU = scale P^T dO + ...
            f4 M[4], PT[4], X[NTL], KD[NTL];
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
                    KD[j] = mma(KD[j], kw[s], made(sm.d, L::kDPlane, L::kKS, 16 * j + ll,
                                                   s * I::kStep, g));
            }
#pragma unroll
            for (int s = 0; s < NC; ++s)
                if ((s + 1) * I::kStep > 16 * w) {
                    const auto pt = from_acc<T>(PT, s);
#pragma unroll
                    for (int j = 0; j < NTL; ++j)
                        X[j] = mma(X[j], pt, given_t_acc(sm.d_o, L::kOS, s * I::kStep, 16 * j, ll, g));
                }
            const f4 el = *(const f4*)(sm.gt.el + 16 * w + 4 * g);
#pragma unroll
            for (int j = 0; j < NTL; ++j)
                put(sm.x, L::kXPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g,
                    a.scale * X[j] + el * KD[j]);
        }
        wave_fence();
        invert_diagonal(sm.tm, w, ll, g);
        lds_barrier();
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
                const auto inv = inverse_cols<T>(sm.tm, w, s, ll, g);
#pragma unroll
                for (int j = 0; j < NTL; ++j)
                    Y[j] = mma(Y[j], inv, made(sm.x, L::kXPlane, L::kUS, 16 * j + ll,
                                               s * I::kStep, g));
            }
        lds_barrier();  // dU has been read
        {
            const f4 bt = *(const f4*)(sm.gt.bt + 16 * w + 4 * g);
            const Rows<T> rv(dvp, (int64_t)c * C, a.L, v_step, width);
            const Rows<float> ry(yp, (int64_t)c * C, a.L, Dv, width);
#pragma unroll
            for (int j = 0; j < NTL; ++j) {
                const f4 dv = bt * Y[j];
                put(sm.x, L::kXPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g, -dv);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    rv.set(rv.off(16 * w + 4 * g + r, 16 * j + ll, width), dv[r]);
                    ry.set(ry.off(16 * w + 4 * g + r, 16 * j + ll, width), Y[j][r]);
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
                const auto qt = scaled(given_t(sm.q, L::kKS, k0, d0, ll, g), sm.gt.es, k0, g);
                const auto kt = scaled(given_t(sm.k, L::kKS, k0, d0, ll, g), sm.gt.eg, k0, g);
#pragma unroll
                for (int j = 0; j < SN; ++j) {
                    D[i][j] = mma(D[i][j], qt,
                                  given_t(sm.d_o, L::kOS, k0, 16 * (wn + NWV * j), ll, g));
                    D[i][j] = mma(D[i][j], kt,
                                  made(sm.x, L::kXPlane, L::kUS, state_n(j, ll), k0, g));
                }
            }
        state_put();
    }
    if (a.dh0) state_store(a.dh0 + head * Dk * Dv);
}

// ------------------------------------------------------------------ the gradients
constexpr int NTW = 32;  // columns of the state at a time

template <typename T, int DK>
struct GradLds {
    using E = typename Io<T>::Elem;
    static constexpr int kKS = DK + Io<T>::kPad, kUS = C + Io<T>::kPad, kNS = NTW + Io<T>::kPad;
    static constexpr int kSPlane = DK * kNS, kRPlane = NTW * kUS, kYPlane = C * kNS;
    E k[C * kKS];
    E q[C * kKS];
    E d_o[C * kNS];
    E s[Io<T>::kPlanes * kSPlane];  // [d][column]: the state before the chunk
    E d[Io<T>::kPlanes * kSPlane];  // the gradient behind it
    E r[Io<T>::kPlanes * kRPlane];  // [column][step]
    E u[Io<T>::kPlanes * kYPlane];  // [step][column]
    E y[Io<T>::kPlanes * kYPlane];
    float tm[C * TS];
    Gates gt;
    float dc[C], db[C], part[8];
};

__device__ __forceinline__ float sum16(float v) {
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

template <typename T, int DK, bool VEC>
__global__ __launch_bounds__(NT) void delta_bwd_grad_kernel(DeltaBwdArgs a, BwdWs ws) {
    using I = Io<T>;
    using L = GradLds<T, DK>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    L& sm = *(L*)smem;
    constexpr int NK = DK / I::kStep, NC = C / I::kStep, NN = NTW / I::kStep;
    constexpr int DTL = DK / 16, NTL = NTW / 16;
    constexpr int KU = C * DK / I::kUnit / NT, UR = DK / I::kUnit;
    constexpr int OU = C * NTW / I::kUnit / NT, OR = NTW / I::kUnit;

    const int tid = threadIdx.x, lane = tid % kWave, w = wave_id(), ll = lane & 15, g = lane >> 4;
    const int chunks = (int)((a.L + C - 1) / C);
    const int64_t bh = blockIdx.x / chunks;
    const int c = (int)(blockIdx.x - bh * chunks);
    const int64_t b = bh / a.H;
    const int h = (int)(bh - b * a.H), group = a.HV / a.H;
    const int Dk = a.Dk, Dv = a.Dv;
    const int64_t t0 = (int64_t)c * C;
    const int64_t qk_step = (int64_t)a.H * Dk, v_step = (int64_t)a.HV * Dv;
    const int64_t qk_base = (b * a.L * a.H + h) * Dk;

    {
        const Rows<T> rk((const T*)a.k + qk_base, t0, a.L, qk_step, Dk);
        const Rows<T> rq((const T*)a.q + qk_base, t0, a.L, qk_step, Dk);
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int u = tid + i * NT, at = u / UR * L::kKS + u % UR * I::kUnit;
            *(wtile::u4v*)(sm.k + at) = rk.template get16<VEC>(u / UR, u % UR * I::kUnit, Dk);
            *(wtile::u4v*)(sm.q + at) = rq.template get16<VEC>(u / UR, u % UR * I::kUnit, Dk);
        }
    }
    f4 dQ[DTL], dK[DTL];
#pragma unroll
    for (int i = 0; i < DTL; ++i) dQ[i] = dK[i] = f4{0, 0, 0, 0};

    for (int hv = h * group; hv < (h + 1) * group; ++hv) {
        const int64_t head = b * a.HV + hv;
        if (w == 0) {
            const int64_t t = t0 + lane;
            const int64_t at = (b * a.L + t) * a.HV + hv;
            gates_of_chunk(&sm.gt, t < a.L ? to_f32(((const T*)a.g)[at]) : 0.0f,
                           t < a.L ? to_f32(((const T*)a.beta)[at]) : 0.0f, a.scale, lane);
        }
        __syncthreads();
        {
            f4 M[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                M[t] = f4{0, 0, 0, 0};
                if (t <= w) {
#pragma unroll
                    for (int s = 0; s < NK; ++s)
                        M[t] = mma(M[t], given(sm.k, L::kKS, 16 * t + ll, s * I::kStep, g),
                                   given(sm.k, L::kKS, 16 * w + ll, s * I::kStep, g));
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
                    if (t <= w)
                        M[t][r] = j < i ? bi * M[t][r] * fast_exp2((float)(ci - sm.gt.cum[j]))
                                        : 0.0f;
                }
                if (t <= (w | 1)) *(f4*)(sm.tm + i * TS + 16 * t + 4 * g) = M[t];
            }
        }
        wave_fence();
        invert_diagonal(sm.tm, w, ll, g);
        __syncthreads();
        invert_merge1(sm.tm, w, ll, g);
        __syncthreads();
        invert_merge2(sm.tm, w, ll, g);

        const f4 eg = *(const f4*)(sm.gt.eg + 16 * w + 4 * g);
        const f4 bt = *(const f4*)(sm.gt.bt + 16 * w + 4 * g);
        const f4 el = *(const f4*)(sm.gt.el + 16 * w + 4 * g);
        // OS = dO S^T, YS = Y S^T, UD = U D^T (lane: column d, rows 16 w + 4 g ..).
        f4 OS[DTL], YS[DTL], UD[DTL], F1[4], Z1[4], F2[4], Z2[4], yv = {0, 0, 0, 0};
        float sd = 0.0f;
#pragma unroll
        for (int i = 0; i < DTL; ++i) OS[i] = YS[i] = UD[i] = f4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < 4; ++t) F1[t] = Z1[t] = F2[t] = Z2[t] = f4{0, 0, 0, 0};

        for (int n0 = 0; n0 < Dv; n0 += NTW) {
            const int width = Dv - n0;
            const int64_t v_base = (b * a.L * a.HV + hv) * Dv + n0;
            const Rows<T> ro((const T*)a.d_o + v_base, t0, a.L, v_step, width);
            const Rows<T> rv((const T*)a.v + v_base, t0, a.L, v_step, width);
            const Rows<float> ry(ws.Y + head * a.L * Dv + n0, t0, a.L, Dv, width);
            __syncthreads();  // the previous columns' operands have been read
#pragma unroll
            for (int i = 0; i < OU; ++i) {
                const int u = tid + i * NT;
                *(wtile::u4v*)(sm.d_o + u / OR * L::kNS + u % OR * I::kUnit) =
                    ro.template get16<VEC>(u / OR, u % OR * I::kUnit, width);
            }
            {
                const int64_t at = (head * chunks + c) * Dk * Dv;
                const auto rs = wtile::rsrc(a.states + at, (uint32_t)(Dk * Dv * 4));
                const auto rd = wtile::rsrc(ws.D + at, (uint32_t)(Dk * Dv * 4));
#pragma unroll
                for (int i = 0; i < DK * NTW / 4 / NT; ++i) {
                    const int u = tid + i * NT, d = u / (NTW / 4), n = u % (NTW / 4) * 4;
                    f4 s, dd;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int o = n + e < width ? (d * Dv + n0 + n + e) * 4 : (int)kNowhere;
                        s[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, o, 0, 0));
                        dd[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rd, o, 0, 0));
                        sd = fmaf(s[e], dd[e], sd);
                    }
                    put(sm.s, L::kSPlane, L::kNS, d, n, s);
                    put(sm.d, L::kSPlane, L::kNS, d, n, dd);
                }
#pragma unroll
                for (int i = 0; i < C * NTW / 4 / NT; ++i) {
                    const int u = tid + i * NT, t = u / (NTW / 4), n = u % (NTW / 4) * 4;
                    f4 y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = ry.get(ry.off(t, n + e, width));
                    put(sm.y, L::kYPlane, L::kNS, t, n, y);
                }
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NTL; ++j) {
                f4 KS = {0, 0, 0, 0}, R;
#pragma unroll
                for (int s = 0; s < NK; ++s)
                    KS = mma(KS, given(sm.k, L::kKS, 16 * w + ll, s * I::kStep, g),
                             made_t(sm.s, L::kSPlane, L::kNS, s * I::kStep, 16 * j, ll, g));
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float v = rv.get(rv.off(16 * w + 4 * g + r, 16 * j + ll, width));
                    const float y = ry.get(ry.off(16 * w + 4 * g + r, 16 * j + ll, width));
                    yv[r] = fmaf(y, v, yv[r]);
                    R[r] = bt[r] * (v - eg[r] * KS[r]);
                }
                put(sm.r, L::kRPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g, R);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NTL; ++j) {
                f4 U = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < NC; ++s)
                    if (s * I::kStep < 16 * (w + 1))
                        U = mma(U, made(sm.r, L::kRPlane, L::kUS, 16 * j + ll, s * I::kStep, g),
                                inverse_rows<T>(sm.tm, w, s, ll, g));
                put(sm.u, L::kYPlane, L::kNS, 16 * w + ll, 16 * j + 4 * g, U);
            }
            __syncthreads();
#pragma unroll
            for (int s = 0; s < NN; ++s) {
                const int k0 = s * I::kStep;
                const auto ow = given(sm.d_o, L::kNS, 16 * w + ll, k0, g);
                const auto yw = made(sm.y, L::kYPlane, L::kNS, 16 * w + ll, k0, g);
                const auto uw = made(sm.u, L::kYPlane, L::kNS, 16 * w + ll, k0, g);
#pragma unroll
                for (int i = 0; i < DTL; ++i) {
                    const auto st = made(sm.s, L::kSPlane, L::kNS, 16 * i + ll, k0, g);
                    OS[i] = mma(OS[i], ow, st);
                    YS[i] = mma(YS[i], yw, st);
                    UD[i] = mma(UD[i], uw, made(sm.d, L::kSPlane, L::kNS, 16 * i + ll, k0, g));
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if (t <= w) {
                        const auto ut = made(sm.u, L::kYPlane, L::kNS, 16 * t + ll, k0, g);
                        F1[t] = mma(F1[t], ut, ow);
                        Z1[t] = mma(Z1[t], ut, yw);
                    }
                    if (t >= w) {
                        F2[t] = mma(F2[t], given(sm.d_o, L::kNS, 16 * t + ll, k0, g), uw);
                        Z2[t] = mma(Z2[t], made(sm.y, L::kYPlane, L::kNS, 16 * t + ll, k0, g), uw);
                    }
                }
            }
        }
        // Decays: F1, Z1 have row i = 16 w + ll and columns j = 16 t + 4 g ..; F2, Z2 have
        // column j = 16 w + ll and rows i = 16 t + 4 g ...
        {
            const int own = 16 * w + ll;
            const double co = sm.gt.cum[own];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int o = 16 * t + 4 * g + r;
                    const double diff = co - sm.gt.cum[o];
                    if (t <= w) {
                        const float e = fast_exp2((float)diff);
                        F1[t][r] = o <= own ? a.scale * F1[t][r] * e : 0.0f;
                        Z1[t][r] = o < own ? -Z1[t][r] * e : 0.0f;
                    }
                    if (t >= w) {
                        const float e = fast_exp2((float)-diff);
                        F2[t][r] = o >= own ? a.scale * F2[t][r] * e : 0.0f;
                        Z2[t][r] = o > own ? -sm.gt.bt[o] * Z2[t][r] * e : 0.0f;
                    }
                }
        }
        f4 x1 = {0, 0, 0, 0}, x2 = x1, x3 = x1, x4 = x1;
#pragma unroll
        for (int i = 0; i < DTL; ++i) {
            f4 q = a.scale * eg * OS[i], ka = -eg * YS[i], ud = el * UD[i], kb = ud;
#pragma unroll
            for (int s = 0; s < NC; ++s) {
                const int k0 = s * I::kStep;
                if (k0 < 16 * (w + 1)) {
                    const auto kt = given_t_acc(sm.k, L::kKS, k0, 16 * i, ll, g);
                    q = mma(q, from_acc<T>(F1, s), kt);
                    ka = mma(ka, from_acc<T>(Z1, s), kt);
                }
                if (k0 + I::kStep > 16 * w) {
                    kb = mma(kb, from_acc<T>(F2, s), given_t_acc(sm.q, L::kKS, k0, 16 * i, ll, g));
                    kb = mma(kb, from_acc<T>(Z2, s), given_t_acc(sm.k, L::kKS, k0, 16 * i, ll, g));
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = (16 * w + 4 * g + r) * L::kKS + 16 * i + ll;
                const float kv = (float)sm.k[at], qv = (float)sm.q[at];
                x1[r] = fmaf(qv, q[r], x1[r]);
                x2[r] = fmaf(kv, ka[r], x2[r]);
                x3[r] = fmaf(kv, kb[r], x3[r]);
                x4[r] = fmaf(kv, ud[r], x4[r]);
            }
            dQ[i] += q;
            dK[i] += bt * ka + kb;
        }
        float end = 0.0f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float s2 = sum16(x2[r]), db = sum16(yv[r]) + s2;
            const float dc = sum16(x1[r]) + bt[r] * s2 - sum16(x3[r]);
            end += x4[r];
            if (ll == 0) {
                sm.dc[16 * w + 4 * g + r] = dc;
                sm.db[16 * w + 4 * g + r] = db;
            }
        }
        end = fmaf(sm.gt.eg[C - 1], sd, end);
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) end += __shfl_xor(end, d);
        if (lane == 0) sm.part[w] = end;
        __syncthreads();
        if (w == 0) {
            float s = sm.dc[lane] + (lane == C - 1 ? sm.part[0] + sm.part[1] + sm.part[2] + sm.part[3]
                                                   : 0.0f);
#pragma unroll
            for (int d = 1; d < C; d <<= 1) {
                const float o = __shfl_down(s, d);
                if (lane + d < C) s += o;
            }
            const int64_t t = t0 + lane;
            if (t < a.L) {
                const int64_t at = (b * a.L + t) * a.HV + hv;
                store((T*)a.dg + at, s);
                store((T*)a.dbeta + at, sm.db[lane]);
            }
        }
        // The next head's decays are written by wave 0, which has read this one's sums; the
        // others' reads of them are behind the barrier above.
    }
    const Rows<T> rq((T*)a.dq + qk_base, t0, a.L, qk_step, Dk);
    const Rows<T> rk((T*)a.dk + qk_base, t0, a.L, qk_step, Dk);
#pragma unroll
    for (int i = 0; i < DTL; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t o = rq.off(16 * w + 4 * g + r, 16 * i + ll, Dk);
            rq.set(o, dQ[i][r]);
            rk.set(o, dK[i][r]);
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
template <typename T, int DK, bool VEC>
hipError_t launch_grad(const DeltaBwdArgs& a, const BwdWs& ws, hipStream_t stream) {
    const int64_t chunks = (a.L + C - 1) / C;
    if (chunks == 0) return hipSuccess;
    static std::atomic<uint64_t> lds_set{0};
    constexpr int bytes = (int)sizeof(GradLds<T, DK>);
    static_assert(bytes <= 160 * 1024, "LDS of a compute unit");
    const hipError_t e =
        allow_dynamic_lds((const void*)delta_bwd_grad_kernel<T, DK, VEC>, bytes, lds_set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((delta_bwd_grad_kernel<T, DK, VEC>), dim3((unsigned)(a.B * a.H * chunks)),
                       dim3(NT), bytes, stream, a, ws);
    return hipGetLastError();
}

template <typename T, int DK>
hipError_t launch_both(const DeltaBwdArgs& a, const BwdWs& ws, bool vec, hipStream_t stream) {
    const hipError_t e = vec ? launch_state<T, DK, 32, true>(a, ws, stream)
                             : launch_state<T, DK, 32, false>(a, ws, stream);
    if (e != hipSuccess) return e;
    return vec ? launch_grad<T, DK, true>(a, ws, stream) : launch_grad<T, DK, false>(a, ws, stream);
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

}  // namespace

size_t delta_backward_workspace(int64_t B, int64_t L, int64_t HV, int Dk, int Dv, IoType) {
    return state_bytes(B, L, HV, Dk, Dv) + round_up((size_t)(B * HV * L * Dv) * 4);
}

hipError_t launch_delta_backward(const DeltaBwdArgs& a, void* ws, hipStream_t stream) {
    const BwdWs s{(float*)ws, (float*)((char*)ws + state_bytes(a.B, a.L, a.HV, a.Dk, a.Dv))};
    return a.io == IoType::kF32 ? launch_typed<float>(a, s, stream)
                                : launch_typed<bf16>(a, s, stream);
}

}  // namespace recblr
