// Forward of the gated delta rule (recblr_delta_forward), 64 steps at a time.
//
// Within a chunk, with c the running sum of g from its start, S the state there and the
// updates u_i = beta_i (v_i - a_i S_{i-1}^T k_i), the recurrence unrolls to
//   (I + A) U = diag(beta) (V - diag(e^c) K S),  A_ij = beta_i e^{c_i - c_j} k_i.k_j (j < i)
//   O  = scale (diag(e^c) Q S + P U),            P_ij = e^{c_i - c_j} q_i.k_j (j <= i)
//   S' = e^{c_63} S + (diag(e^{c_63 - c}) K)^T U.
// A workgroup walks the chunks of one head's strip of DVT columns (columns of the state do not
// mix) with the state in its accumulators and, as an operand, in LDS.  Q stays in registers
// as the operand of its wave's strip, and so does P, whose accumulators are an operand as they
// are; K and the inverse of I + A go through LDS, and in one place there, one after the other,
// the state, the right-hand side R, and U with the decays up to the chunk's end (so that K is
// an operand of S' as it was given).
//
// What bounds it is the chain of a chunk, some 8 us of products, substitution and hand-overs
// through LDS with seven barriers, of which two workgroups a CU hide a part: 2048 heads, 200
// steps, 64 x 64 bf16 with kept states take 188 us (2.0 TB/s), 256 heads, 2048 steps fp32 395 us
// (77 TFLOP/s, half of what fp32 matrix instructions reach).  Strips are 64 columns where the
// state then fits the registers, as K, its products and the inverse are formed once a strip.
#include <hip/hip_runtime.h>

#include "delta_tile.hpp"
#include "ops.hpp"

namespace recblr {
namespace {

using namespace dtile;

template <typename T, int DK, int DVT>
struct FwdLds {
    using E = typename Io<T>::Elem;
    static constexpr int kChain = Io<T>::kChain, kOut = Io<T>::kOut;
    static constexpr int kKS = DK + Io<T>::kPad, kUS = C + Io<T>::kPad;
    static constexpr int kSPlane = DVT * kKS, kUPlane = DVT * kUS;
    E k[C * kKS];
    // [column][d] the state; then [column][step] R; then the updates times el
    E x[kChain * (kSPlane > kUPlane ? kSPlane : kUPlane)];
    E u[kOut * kUPlane];  // [column][step] the updates
    float tm[C * TS];
    Gates gt;
};

template <typename T, int DK, int DVT, bool VEC>
__global__ __launch_bounds__(NT, 2) void delta_fwd_kernel(DeltaFwdArgs a, int strips) {
    using I = Io<T>;
    using L = FwdLds<T, DK, DVT>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    L& sm = *(L*)smem;
    constexpr int NK = DK / I::kStep;    // contraction steps over d
    constexpr int NC = C / I::kStep;     // over a chunk
    constexpr int NTL = DVT / 16, DTL = DK / 16;
    constexpr int DW = DTL < 4 ? DTL : 4, NWV = 4 / DW;  // waves along d and along the columns
    constexpr int SD = DTL / DW, SN = NTL / NWV;         // state tiles of a wave
    constexpr int KU = C * DK / I::kUnit / NT;           // 16-byte units of K to a thread
    constexpr int UR = DK / I::kUnit;                    // units in a row
    static_assert(KU >= 1, "every thread stages K");

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
    const T* vp = (const T*)a.v + (b * a.L * a.HV + hv) * Dv + n0;
    T* op = (T*)a.o + (b * a.L * a.HV + hv) * Dv + n0;
    const T* gp = (const T*)a.g + b * a.L * a.HV + hv;
    const T* bp = (const T*)a.beta + b * a.L * a.HV + hv;
    const int chunks = (int)((a.L + C - 1) / C);
    const int wd = w % DW, wn = w / DW;

    // The state's tiles: d = 16 (wd + DW i) + 4 g + r, column 16 (wn + NWV j) + ll.
    f4 S[SD][SN];
    auto state_d = [&](int i, int g) { return 16 * (wd + DW * i) + 4 * g; };
    auto state_n = [&](int j, int ll) { return 16 * (wn + NWV * j) + ll; };
    // f(tile, r, offset) for the state at p [Dk][Dv].
    auto state_io = [&](const float* p, auto f) {
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
        const auto r = wtile::rsrc(p, (uint32_t)(Dk * Dv * 4));
#pragma unroll
        for (int i = 0; i < SD; ++i)
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                const int n = state_n(j, ll);
                // Rows behind Dk lie behind the buffer's end.
                const uint32_t o = n < width ? (uint32_t)(state_d(i, g) * Dv + n0 + n) * 4 : kNowhere;
#pragma unroll
                for (int e = 0; e < 4; ++e) f(r, S[i][j], e, (int)(o + (uint32_t)(4 * e * Dv)));
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
                put<L::kChain>(sm.x, L::kSPlane, L::kKS, state_n(j, ll), state_d(i, g),
                               S[i][j]);
    };
#pragma unroll
    for (int i = 0; i < SD; ++i)
#pragma unroll
        for (int j = 0; j < SN; ++j) S[i][j] = f4{0, 0, 0, 0};
    if (a.h0)
        state_io(a.h0 + head * Dk * Dv, [](auto r, f4& s, int e, int o) {
            s[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0));
        });

    wtile::u4v kn[KU], qn[NK];
    uint32_t vn[NTL][4], gn = 0, bn = 0;  // raw
    auto fetch_k = [&](int c) {
        const int tid = wtile::fresh(threadIdx.x);
        const Rows<T> r(kp, (int64_t)c * C, a.L, qk_step, Dk);
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int u = tid + i * NT;
            kn[i] = r.template get16<VEC>(u / UR, u % UR * I::kUnit, Dk);
        }
        if (w == 0) {
            const Rows<T> rg(gp, (int64_t)c * C, a.L, a.HV, 1), rb(bp, (int64_t)c * C, a.L, a.HV, 1);
            gn = rg.raw(rg.off(lane0, 0, 1));
            bn = rb.raw(rb.off(lane0, 0, 1));
        }
    };
    auto fetch_qv = [&](int c) {
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;
        const Rows<T> rq(qp, (int64_t)c * C, a.L, qk_step, Dk);
#pragma unroll
        for (int s = 0; s < NK; ++s)
            qn[s] = rq.template get16<VEC>(16 * w + ll, s * I::kStep + I::kUnit * g, Dk);
        const Rows<T> rv(vp, (int64_t)c * C, a.L, v_step, width);
#pragma unroll
        for (int j = 0; j < NTL; ++j) {
            const uint32_t o = rv.off(16 * w + 4 * g, 16 * j + ll, width);
#pragma unroll
            for (int r = 0; r < 4; ++r) vn[j][r] = rv.raw(rv.next(o, r));
        }
    };
    if (chunks > 0) {
        fetch_k(0);
        fetch_qv(0);
    }

    for (int c = 0; c < chunks; ++c) {
        if (a.states) state_store(a.states + (head * chunks + c) * Dk * Dv);
        lds_barrier();  // the previous chunk's K and updates have been read
        state_put();
        {
            const int tid = wtile::fresh(threadIdx.x);
#pragma unroll
            for (int i = 0; i < KU; ++i) {
                const int u = tid + i * NT;
                *(wtile::u4v*)(sm.k + u / UR * L::kKS + u % UR * I::kUnit) = kn[i];
            }
        }
        if (w == 0) gates_of_chunk(&sm.gt, Rows<T>::value(gn), Rows<T>::value(bn), a.scale, lane0);
        lds_barrier();  // K, the decays and the state's operand are in LDS
        // Read ahead in any case (behind the last chunk out of range, so nothing): under a condition
        // the compiler waits for more than it needs.
        fetch_k(c + 1);
        const int lane = wtile::fresh(lane0), ll = lane & 15, g = lane >> 4;

        // Strips of k k^T and q k^T (lane: row i = 16 w + ll, columns 16 t + 4 g ..), of K S
        // and Q S (lane: column of the state, rows 16 w + 4 g ..).
        f4 P[4], KS[NTL], O[NTL];
        {
            f4 M[4];
            typename I::Given kw[NK], qw[NK];
#pragma unroll
            for (int s = 0; s < NK; ++s) {
                kw[s] = given(sm.k, L::kKS, 16 * w + ll, s * I::kStep, g);
                qw[s] = __builtin_bit_cast(typename I::Given, qn[s]);
            }
            // Each step's operands are read while the one before is multiplied.
            typename I::Given kt[2][NK];
            auto read_k = [&](int t) {
#pragma unroll
                for (int s = 0; s < NK; ++s)
                    kt[t & 1][s] = given(sm.k, L::kKS, 16 * t + ll, s * I::kStep, g);
            };
            read_k(0);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                M[t] = P[t] = f4{0, 0, 0, 0};
                if (t < 3) read_k(t + 1);
#pragma unroll
                for (int s = 0; s < NK; ++s) {
                    M[t] = mma(M[t], kt[t & 1][s], kw[s]);
                    P[t] = mma(P[t], kt[t & 1][s], qw[s]);
                }
                step_end(P[t]);
            }
            typename I::template Made<L::kChain> st[2];
            auto read_s = [&](int u) {
                st[u & 1] = made<L::kChain>(sm.x, L::kSPlane, L::kKS, 16 * (u / NK) + ll,
                                            u % NK * I::kStep, g);
            };
            read_s(0);
#pragma unroll
            for (int u = 0; u < NTL * NK; ++u) {
                const int j = u / NK, s = u % NK;
                if (s == 0) KS[j] = O[j] = f4{0, 0, 0, 0};
                if (u + 1 < NTL * NK) read_s(u + 1);
                KS[j] = mma(KS[j], kw[s], st[u & 1]);
                O[j] = mma(O[j], qw[s], fewer<L::kOut>(st[u & 1]));
                step_end(O[j]);
            }
            const int i = 16 * w + ll;
            const double ci = sm.gt.cum[i];
            const float bi = sm.gt.bt[i];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * t + 4 * g + r;
                    const float e = fast_exp2((float)(ci - sm.gt.cum[j]));
                    P[t][r] = j <= i ? P[t][r] * e : 0.0f;
                    M[t][r] = j < i ? bi * M[t][r] * e : 0.0f;
                }
                *(f4*)(sm.tm + i * TS + 16 * t + 4 * g) = M[t];
            }
        }
        {
            const f4 eg = *(const f4*)(sm.gt.eg + 16 * w + 4 * g);
            const f4 bt = *(const f4*)(sm.gt.bt + 16 * w + 4 * g);
#pragma unroll
            for (int j = 0; j < NTL; ++j) {
#pragma unroll
                for (int r = 0; r < 4; ++r) KS[j][r] = bt[r] * (Rows<T>::value(vn[j][r]) - eg[r] * KS[j][r]);
                O[j] *= eg;
            }
        }
        fetch_qv(c + 1);
        wave_fence();
        invert_diagonal(sm.tm, w, ll, g);
        lds_barrier();  // the state has been read
#pragma unroll
        for (int j = 0; j < NTL; ++j)
            put<L::kChain>(sm.x, L::kUPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g, KS[j]);
        invert_merge1(sm.tm, w, ll, g);
        lds_barrier();
        invert_merge2(sm.tm, w, ll, g);
        lds_barrier();
        f4 U[NTL];
#pragma unroll
        for (int j = 0; j < NTL; ++j) U[j] = f4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < NC; ++s)
            if (s * I::kStep < 16 * (w + 1)) {
                const auto inv = inverse_rows<T, L::kChain>(sm.tm, w, s, ll, g);
#pragma unroll
                for (int j = 0; j < NTL; ++j)
                    U[j] = mma(U[j], inv, made<L::kChain>(sm.x, L::kUPlane, L::kUS, 16 * j + ll,
                                                          s * I::kStep, g));
            }
        lds_barrier();  // R has been read
        {
            const f4 el = *(const f4*)(sm.gt.el + 16 * w + 4 * g);
#pragma unroll
            for (int j = 0; j < NTL; ++j) {
                put<L::kOut>(sm.u, L::kUPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g, U[j]);
                put<L::kChain>(sm.x, L::kUPlane, L::kUS, 16 * j + ll, 16 * w + 4 * g, el * U[j]);
            }
        }
        lds_barrier();
        const float et = sm.gt.eg[C - 1];
#pragma unroll
        for (int i = 0; i < SD; ++i)
#pragma unroll
            for (int j = 0; j < SN; ++j) S[i][j] *= et;
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int i = 0; i < SD; ++i) {
                const auto kt = given_t(sm.k, L::kKS, s * I::kStep, 16 * (wd + DW * i), ll, g);
#pragma unroll
                for (int j = 0; j < SN; ++j)
                    S[i][j] = mma(S[i][j], kt, made<L::kChain>(sm.x, L::kUPlane, L::kUS,
                                                               state_n(j, ll), s * I::kStep, g));
            }
#pragma unroll
        for (int s = 0; s < NC; ++s)
            {
                const auto pw = from_acc<T, L::kOut>(P, s);
#pragma unroll
                for (int j = 0; j < NTL; ++j)
                    O[j] = mma(O[j], pw, made_acc<L::kOut>(sm.u, L::kUPlane, L::kUS, 16 * j + ll,
                                                           s * I::kStep, g));
            }
        const Rows<T> ro(op, (int64_t)c * C, a.L, v_step, width);
#pragma unroll
        for (int j = 0; j < NTL; ++j) {
            const uint32_t o = ro.off(16 * w + 4 * g, 16 * j + ll, width);
#pragma unroll
            for (int r = 0; r < 4; ++r) ro.set(ro.next(o, r), a.scale * O[j][r]);
        }
    }
    if (a.hT) state_store(a.hT + head * Dk * Dv);
}

template <typename T, int DK, int DVT, bool VEC>
hipError_t launch_kernel(const DeltaFwdArgs& a, hipStream_t stream) {
    static std::atomic<uint64_t> lds_set{0};
    constexpr int bytes = (int)sizeof(FwdLds<T, DK, DVT>);
    const hipError_t e =
        allow_dynamic_lds((const void*)delta_fwd_kernel<T, DK, DVT, VEC>, bytes, lds_set);
    if (e != hipSuccess) return e;
    const int strips = (a.Dv + DVT - 1) / DVT;
    hipLaunchKernelGGL((delta_fwd_kernel<T, DK, DVT, VEC>),
                       dim3((unsigned)(a.B * a.HV * strips)), dim3(NT), bytes, stream, a, strips);
    return hipGetLastError();
}

template <typename T, int DK, int DVT>
hipError_t launch_variant(const DeltaFwdArgs& a, hipStream_t stream) {
    const bool vec = a.Dk * sizeof(T) % 16 == 0 && (uintptr_t)a.q % 16 == 0 &&
                     (uintptr_t)a.k % 16 == 0;
    return vec ? launch_kernel<T, DK, DVT, true>(a, stream)
               : launch_kernel<T, DK, DVT, false>(a, stream);
}

template <typename T>
hipError_t launch_typed(const DeltaFwdArgs& a, hipStream_t stream) {
    if (a.Dk <= 32) return a.Dv <= 32 ? launch_variant<T, 32, 32>(a, stream) : launch_variant<T, 32, 64>(a, stream);
    if (a.Dk <= 64) return a.Dv <= 32 ? launch_variant<T, 64, 32>(a, stream) : launch_variant<T, 64, 64>(a, stream);
    return launch_variant<T, 128, 32>(a, stream);
}

}  // namespace

size_t delta_forward_workspace(int64_t B, int64_t L, int64_t HV, int Dk, int Dv, IoType io) {
    if (!delta_split(B * HV, L, Dk, Dv, false)) return 0;
    DeltaFwdArgs a{};
    a.B = B;
    a.L = L;
    a.H = a.HV = (int)HV;
    a.Dk = Dk;
    a.Dv = Dv;
    a.io = io;
    size_t bytes = 0;
    (void)launch_delta_split_forward(a, nullptr, &bytes, nullptr);
    return bytes;
}

hipError_t launch_delta_forward(const DeltaFwdArgs& a, void* ws, hipStream_t stream) {
    size_t bytes;
    if (delta_split(a.B * a.HV, a.L, a.Dk, a.Dv, false))
        return launch_delta_split_forward(a, ws, &bytes, stream);
    return a.io == IoType::kF32 ? launch_typed<float>(a, stream) : launch_typed<bf16>(a, stream);
}

}  // namespace recblr
