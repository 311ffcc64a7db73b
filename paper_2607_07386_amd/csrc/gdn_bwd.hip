// The dense gated delta rule, reverse mode (gfx950); notation as in gdn.hip.
// Sequential part (gdn_adjoint_kernel), chunks last to first, with dS1 the
// gradient of the chunk's last state and G = diag(gamma), C = diag(exp(lambda_63 - lambda)):
//   dE = P^T dY + C K dS1;   dR = T'^T diag(beta) dE = dV;
//   dS0 = gamma_63 dS1 + (G Q)^T dY - (G K)^T dR
// Parallel part (gdn_grads_kernel), per chunk, from S0 and X as the forward saved
// them, dS1 and dR:
//   Z2 = tril(dY X^T), Z = stril(dR X^T), M1 = X dS1^T, M2 = dY S0^T, M3 = dR S0^T,
//   dQ = G M2 + (Z2 . beta_j D) K
//   dK = (Z2 . beta_j D)^T Q + diag(beta) C M1 - G M3 - (Zb + Zb^T) K,  Zb = Z . beta_j D
//   dbeta_j = sum_i (P . Z2 - N . Z)_ij + exp(lambda_63 - lambda_j) <k_j, M1_j>
//   dlog alpha_t = the sum of every term that contains alpha_t: pairs (i, j) with
//   j < t <= i of (P . Z2 - N . Z)_ij beta_j; gamma_i (<q_i, M2_i> - <k_i, M3_i>)
//   for i >= t; beta_j C_j <k_j, M1_j> for j < t; and gamma_63 <S0, dS1>.
// (X, not E, enters, so a token with beta = 0 has its gradient.)  The terms of
// dlog alpha_t all carry alpha_t as a factor and none that does not is added
// and taken off again, so dividing by a small alpha_t loses nothing.
#include <algorithm>

#include "gdn.h"
#include "sdm_internal.h"

namespace {

template <typename VT, int KTN>
__global__ __launch_bounds__(256, 1) void gdn_adjoint_kernel(GdnArgs a) {
    constexpr int NT = GdnIn<VT>::NT, DT = 2 * KTN;
    const int groups = (a.dv + 63) / 64;
    int grp, bh;
    scan_wg_coords<true>(groups, grp, bh);
    const int col0 = (grp * 4 + (threadIdx.x >> 6)) * 16;
    if (col0 >= a.dv) return;
    const int b = bh / a.H, hk = (bh % a.H) / (a.H / a.Hk);
    const int lane = lane_id(), r16 = lane & 15, g = lane >> 4;
    const int col = col0 + r16;
    const bool cv = col < a.dv;
    const int len = gdn_len(a, b), nc = (len + GDN_C - 1) / GDN_C;
    const size_t sbase = (size_t)bh * a.dk * a.dv + col;
    const sdm_f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    sdm_f32x4 S[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = gdn_row(d, 4 * g + r);
            S[d][r] = a.dstateT && cv && row < a.dk ? a.dstateT[sbase + (size_t)row * a.dv] : 0.f;
        }
    const size_t tq0 = (size_t)(b * a.Hk + hk) * a.T, tv0 = (size_t)bh * a.T;
    for (int c = nc - 1; c >= 0; --c) {
        const int t0 = c * GDN_C;
        const size_t ch = (size_t)bh * a.nC + c, ck = (size_t)(b * a.Hk + hk) * a.nC + c;
        const VT* kp = static_cast<const VT*>(a.k) + (tq0 + t0) * a.dk;
        const float* vec = a.vec + ch * GDN_VEC * 64;
        float* o = a.dS + ch * a.dk * a.dv + col;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = gdn_row(d, 4 * g + r);
                if (cv && row < a.dk) o[(size_t)row * a.dv] = S[d][r];
            }
        sdm_f32x4 dE[4], Y[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            dE[m] = zero;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = gdn_row(m, 4 * g + r);
                Y[m][r] = cv && t0 + t < len ? a.dy[(tv0 + t0 + t) * a.dv + col] : 0.f;
            }
        }
#pragma unroll
        for (int kb = 0; kb < KTN; ++kb) {
            const GdnFrag<3> s = gdn_stack(S[2 * kb], S[2 * kb + 1]);
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const int row = gdn_row(m, r16);
                dE[m] = gdn_mm(gdn_row_frag<NT>(kp + (size_t)row * a.dk, kb, a.dk, t0 + row < len), s, dE[m]);
            }
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const v4f en = ld4(vec + GDN_V_END * 64 + gdn_row(m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) dE[m][r] *= en[r];
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const GdnFrag<3> f = gdn_stack(Y[2 * kb], Y[2 * kb + 1]);
#pragma unroll
            for (int m = 0; m < 2 * kb + 2; ++m)
                dE[m] = gdn_mm(gdn_load_frag<3>(a.pf, ch * GDN_BLKS + gdn_up_blk(m, kb)), f, dE[m]);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const v4f be = ld4(vec + GDN_V_BETA * 64 + gdn_row(m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) dE[m][r] *= be[r];
        }
        sdm_f32x4 dR[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) dR[m] = zero;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const GdnFrag<3> f = gdn_stack(dE[2 * kb], dE[2 * kb + 1]);
#pragma unroll
            for (int m = 0; m < 2 * kb + 2; ++m)
                dR[m] = gdn_mm(gdn_load_frag<3>(a.tf, ch * GDN_BLKS + gdn_up_blk(m, kb)), f, dR[m]);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const v4f gam = ld4(vec + GDN_V_GAM * 64 + gdn_row(m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = gdn_row(m, 4 * g + r);
                if (cv && t0 + t < len) a.dvv[(tv0 + t0 + t) * a.dv + col] = dR[m][r];
                dR[m][r] *= -gam[r];
                Y[m][r] *= gam[r];
            }
        }
        const float last = vec[GDN_V_GAM * 64 + 63];
#pragma unroll
        for (int d = 0; d < DT; ++d) S[d] *= last;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const GdnFrag<3> fr = gdn_stack(dR[2 * kb], dR[2 * kb + 1]);
            const GdnFrag<3> fy = gdn_stack(Y[2 * kb], Y[2 * kb + 1]);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                S[d] = gdn_mm(gdn_load_frag<NT>(a.kt, (ck * DT + d) * 2 + kb), fr, S[d]);
                S[d] = gdn_mm(gdn_load_frag<NT>(a.qt, (ck * DT + d) * 2 + kb), fy, S[d]);
            }
        }
    }
    if (a.dstate0) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = gdn_row(d, 4 * g + r);
                if (cv && row < a.dk) a.dstate0[sbase + (size_t)row * a.dv] = S[d][r];
            }
    }
}

// The same walk for bf16 inputs, fragments staged in LDS as in the forward scan.
template <int KTN>
__global__ __launch_bounds__(256, 1) void gdn_adjoint_staged_kernel(GdnArgs a) {
    constexpr int DT = 2 * KTN;
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t* sK = reinterpret_cast<uint16_t*>(smem);       // K [4][KTN]
    uint16_t* sT = sK + 4 * KTN * GDN_FRAG;                 // T'^T [6][3], then P^T
    uint16_t* sP = sT + GDN_BLKS * 3 * GDN_FRAG;
    uint16_t* sKT = sP + GDN_BLKS * 3 * GDN_FRAG;           // K^T [DT][2], then Q^T
    uint16_t* sQT = sKT + 4 * KTN * GDN_FRAG;
    float* sV = reinterpret_cast<float*>(sQT + 4 * KTN * GDN_FRAG);   // [2][gamma, end, beta][64]

    const int groups = (a.dv + 63) / 64;
    int grp, bh;
    scan_wg_coords<true>(groups, grp, bh);
    const int b = bh / a.H, hk = (bh % a.H) / (a.H / a.Hk);
    const int len = gdn_len(a, b), nc = (len + GDN_C - 1) / GDN_C;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id(), r16 = lane & 15, g = lane >> 4;
    const int col = (grp * 4 + w) * 16 + r16;
    const bool cv = col < a.dv;
    const uint32_t co = cv ? col * 4 : GDN_OUT;
    const size_t sn = (size_t)a.dk * a.dv;
    const sdm_f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    sdm_f32x4 S[DT];
    gdn_load_state(S, a.dstateT ? a.dstateT + bh * sn : nullptr, a.dk, a.dv, co);
    const bf16_t* kp = static_cast<const bf16_t*>(a.k) + (size_t)(b * a.Hk + hk) * a.T * a.dk;
    const float* yp = a.dy + (size_t)bh * a.T * a.dv;
    float* dvp = a.dvv + (size_t)bh * a.T * a.dv;
    const size_t ch0 = (size_t)bh * a.nC, ck0 = (size_t)(b * a.Hk + hk) * a.nC;

    u4v rK[KTN], rT[9], rKT[KTN], rQT[KTN];
    float rV, rY[4][4];
    const auto fetch_k = [&](int c) {
        gdn_fetch_rows(rK, kp + (size_t)c * GDN_C * a.dk, w, len - c * GDN_C, a.dk);
        const int which = w == 0 ? GDN_V_GAM : w == 1 ? GDN_V_END : GDN_V_BETA;   // wave 3 repeats wave 2
        rV = a.vec[(ch0 + c) * GDN_VEC * 64 + which * 64 + lane];
    };
    const auto fetch_y = [&](int c) {
        const auto buf = gdn_buf(yp + (size_t)c * GDN_C * a.dv, (size_t)min(len - c * GDN_C, GDN_C) * a.dv * 4);
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) rY[m][r] = gdn_ldf(buf, gdn_row(m, 4 * g + r) * a.dv * 4 + co);
    };
    const auto fetch_t = [&](int c) {
        const uint16_t* src = w < 2 ? a.tf : a.pf;
        gdn_fetch(rT, src + (ch0 + c) * GDN_BLKS * 3 * GDN_FRAG, (w & 1) * 9);
    };
    const auto fetch_kt = [&](int c) {
        gdn_fetch(rKT, a.kt + (ck0 + c) * DT * 2 * GDN_FRAG, w * KTN);
        gdn_fetch(rQT, a.qt + (ck0 + c) * DT * 2 * GDN_FRAG, w * KTN);
    };
    const auto stage_k = [&](int par) {
        gdn_stage(sK, w * KTN, rK);
        if (w < 3) sV[(par * 3 + w) * 64 + lane] = rV;
    };
    const auto stage_t = [&]() { gdn_stage(sT, w * 9, rT); };
    const auto stage_kt = [&]() {
        gdn_stage(sKT, w * KTN, rKT);
        gdn_stage(sQT, w * KTN, rQT);
    };

    if (nc > 0) {
        fetch_k(nc - 1);
        fetch_y(nc - 1);
        fetch_t(nc - 1);
        fetch_kt(nc - 1);
        stage_k((nc - 1) & 1);
        stage_t();
        stage_kt();
        const int c1 = max(nc - 2, 0);
        fetch_k(c1);
        fetch_t(c1);
        fetch_kt(c1);
        __syncthreads();
    }
    for (int c = nc - 1; c >= 0; --c) {
        const int t0 = c * GDN_C, left = len - t0, next = max(c - 2, 0);
        const float* vec = sV + (c & 1) * 3 * 64;
        const auto rbuf = gdn_buf(dvp + (size_t)t0 * a.dv, (size_t)min(left, GDN_C) * a.dv * 4);
        gdn_store_state(S, a.dS + (ch0 + c) * sn, a.dk, a.dv, co);
        sdm_f32x4 dE[4], Y[4], dR[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            dE[m] = dR[m] = zero;
#pragma unroll
            for (int r = 0; r < 4; ++r) Y[m][r] = rY[m][r];
        }
#pragma unroll
        for (int kb = 0; kb < KTN; ++kb) {
            const GdnFrag<3> s = gdn_stack(S[2 * kb], S[2 * kb + 1]);
#pragma unroll
            for (int m = 0; m < 4; ++m) dE[m] = gdn_mm(gdn_load_frag<1>(sK, m * KTN + kb), s, dE[m]);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const v4f en = ld4(vec + 64 + gdn_row(m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) dE[m][r] *= en[r];
        }
        __syncthreads();
        stage_k((c + 1) & 1);
        fetch_y(max(c - 1, 0));
        fetch_k(next);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const GdnFrag<3> f = gdn_stack(Y[2 * kb], Y[2 * kb + 1]);
#pragma unroll
            for (int m = 0; m < 2 * kb + 2; ++m) dE[m] = gdn_mm(gdn_load_frag<3>(sP, gdn_up_blk(m, kb)), f, dE[m]);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const v4f be = ld4(vec + 128 + gdn_row(m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) dE[m][r] *= be[r];
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const GdnFrag<3> f = gdn_stack(dE[2 * kb], dE[2 * kb + 1]);
#pragma unroll
            for (int m = 0; m < 2 * kb + 2; ++m) dR[m] = gdn_mm(gdn_load_frag<3>(sT, gdn_up_blk(m, kb)), f, dR[m]);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const v4f gam = ld4(vec + gdn_row(m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = gdn_row(m, 4 * g + r);
                gdn_stf(rbuf, t * a.dv * 4 + co, dR[m][r]);
                dR[m][r] *= -gam[r];
                Y[m][r] *= gam[r];
            }
        }
        const float last = vec[63];
        __syncthreads();
        stage_t();
        fetch_t(next);
#pragma unroll
        for (int d = 0; d < DT; ++d) S[d] *= last;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const GdnFrag<3> fr = gdn_stack(dR[2 * kb], dR[2 * kb + 1]);
            const GdnFrag<3> fy = gdn_stack(Y[2 * kb], Y[2 * kb + 1]);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                S[d] = gdn_mm(gdn_load_frag<1>(sKT, d * 2 + kb), fr, S[d]);
                S[d] = gdn_mm(gdn_load_frag<1>(sQT, d * 2 + kb), fy, S[d]);
            }
        }
        __syncthreads();
        stage_kt();
        fetch_kt(next);
    }
    if (a.dstate0) gdn_store_state(S, a.dstate0 + bh * sn, a.dk, a.dv, co);
}

template <int KTN>
hipError_t launch_adjoint_staged(const GdnArgs& a, hipStream_t st) {
    const auto kfn = gdn_adjoint_staged_kernel<KTN>;
    constexpr size_t lds = (size_t)(12 * KTN + 36) * GDN_FRAG * 2 + 2 * 3 * 64 * 4;
    hipError_t e = hipFuncSetAttribute((const void*)kfn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    kfn<<<dim3((a.dv + 63) / 64 * a.B * a.H), 256, lds, st>>>(a);
    return hipGetLastError();
}

// ---------------------------------------------------------------- gradients
constexpr int LD = 68;

// One workgroup per (key head, chunk), over the heads that share the key head in
// order (their dq, dk add up in registers, reproducibly).  Wave w holds tokens
// 16w .. 16w+15.  Per 32 columns of d_v the workgroup stages S0, dS1 and X once
// as fragments in LDS; a row of a matrix is the same fragment as an A or a B
// operand, so every product over d_v reads its rows straight from memory.
template <typename VT, int KTN>
__global__ __launch_bounds__(256, 1) void gdn_grads_kernel(GdnArgs a) {
    constexpr int NT = GdnIn<VT>::NT, DT = 2 * KTN;
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t* sS = reinterpret_cast<uint16_t*>(smem);                  // [DT][3] fragments
    uint16_t* sD = sS + DT * 3 * GDN_FRAG;
    uint16_t* sX = sD + DT * 3 * GDN_FRAG;                             // [4][3]
    float* mQ = reinterpret_cast<float*>(smem);                        // after the products, in their place
    float* mB = mQ + 64 * LD;
    constexpr size_t STAGE = (size_t)(2 * DT + 4) * 3 * GDN_FRAG * 2;
    constexpr size_t PAIRS = (size_t)2 * 64 * LD * 4;
    float* mP = reinterpret_cast<float*>(smem + (STAGE > PAIRS ? STAGE : PAIRS));
    float* mN = mP + 64 * LD;
    float* vlh = mN + 64 * LD;
    float *vll = vlh + 64, *vb = vll + 64, *rEnd = vb + 64, *rFrom = rEnd + 64, *rThr = rFrom + 64, *rCol = rThr + 64,
          *rCross = rCol + 64;

    const int c = blockIdx.x, b = blockIdx.y / a.Hk, hk = blockIdx.y % a.Hk, G = a.H / a.Hk;
    const int len = gdn_len(a, b), t0 = c * GDN_C;
    if (t0 >= len) return;
    const int tid = threadIdx.x, lane = lane_id(), w = tid >> 6, r16 = lane & 15, g = lane >> 4;
    const size_t tq = (size_t)(b * a.Hk + hk) * a.T + t0;
    const VT* kp = static_cast<const VT*>(a.k) + tq * a.dk;
    const VT* qp = static_cast<const VT*>(a.q) + tq * a.dk;
    const size_t ck = (size_t)(b * a.Hk + hk) * a.nC + c;
    const sdm_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const int arow = 16 * w + r16;            // the A operands' token
    const bool aok = t0 + arow < len;
    const int dvb = (a.dv + 31) / 32;

    sdm_f32x4 dq[DT], dk[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dq[d] = dk[d] = zero;

    for (int hg = 0; hg < G; ++hg) {
        const int bh = b * a.H + hk * G + hg;
        const size_t ch = (size_t)bh * a.nC + c, tv = (size_t)bh * a.T + t0;
        const float* vec = a.vec + ch * GDN_VEC * 64;
        const float* S0 = a.saved_S + ch * a.dk * a.dv;
        const float* S1 = a.dS + ch * a.dk * a.dv;
        const float* xr = a.saved_X + (tv + arow) * a.dv;
        const float* yr = a.dy + (tv + arow) * a.dv;
        const float* rr = a.dvv + (tv + arow) * a.dv;
        __syncthreads();                      // the previous head's use of LDS
        if (tid < 64) {
            vlh[tid] = vec[GDN_V_LHI * 64 + tid];
            vll[tid] = vec[GDN_V_LLO * 64 + tid];
            vb[tid] = vec[GDN_V_BETA * 64 + tid];
        }
        sdm_f32x4 M1[DT], M2[DT], M3[DT], Z2[4], Z[4];
#pragma unroll
        for (int d = 0; d < DT; ++d) M1[d] = M2[d] = M3[d] = zero;
#pragma unroll
        for (int j = 0; j < 4; ++j) Z2[j] = Z[j] = zero;
        float through = 0.f;
        for (int kb = 0; kb < dvb; ++kb) {
            const GdnFrag<3> fx = gdn_row_frag<3>(xr, kb, a.dv, aok);
            const GdnFrag<3> fy = gdn_row_frag<3>(yr, kb, a.dv, aok);
            const GdnFrag<3> fr = gdn_row_frag<3>(rr, kb, a.dv, aok);
            gdn_store_frag<3>(sX, w, fx);
            for (int d = w; d < DT; d += 4) {
                const int row = gdn_row(d, r16);
                float x0[8], x1[8];
                gdn_row8(S0 + (size_t)row * a.dv, kb, a.dv, row < a.dk, x0);
                gdn_row8(S1 + (size_t)row * a.dv, kb, a.dv, row < a.dk, x1);
#pragma unroll
                for (int i = 0; i < 8; ++i) through = fmaf(x0[i], x1[i], through);
                gdn_store_frag<3>(sS, d, gdn_split(x0));
                gdn_store_frag<3>(sD, d, gdn_split(x1));
            }
            __syncthreads();
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const GdnFrag<3> s0 = gdn_load_frag<3>(sS, d);
                M2[d] = gdn_mm(fy, s0, M2[d]);
                M3[d] = gdn_mm(fr, s0, M3[d]);
                M1[d] = gdn_mm(fx, gdn_load_frag<3>(sD, d), M1[d]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j > w) break;
                const GdnFrag<3> x = gdn_load_frag<3>(sX, j);
                Z2[j] = gdn_mm(fy, x, Z2[j]);
                Z[j] = gdn_mm(fr, x, Z[j]);
            }
            __syncthreads();
        }
        through = wave_sum(through);
        if (lane == 0) rThr[w] = through;
        // rows of M against q and k; dq, dk without the pairs' part
        float gam[4], en[4], be[4], pe[4], pf[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * w + 4 * g + r;
            gam[r] = vec[GDN_V_GAM * 64 + i];
            en[r] = vec[GDN_V_END * 64 + i];
            be[r] = vec[GDN_V_BETA * 64 + i];
            pe[r] = pf[r] = 0.f;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int dc = gdn_row(d, r16);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * w + 4 * g + r;
                const bool ok = dc < a.dk && t0 + i < len;
                const float kv = ok ? to_f32(kp[(size_t)i * a.dk + dc]) : 0.f;
                const float qv = ok ? to_f32(qp[(size_t)i * a.dk + dc]) : 0.f;
                pe[r] = fmaf(kv, M1[d][r], pe[r]);
                pf[r] = fmaf(qv, M2[d][r], fmaf(-kv, M3[d][r], pf[r]));
                dq[d][r] = fmaf(gam[r], M2[d][r], dq[d][r]);
                dk[d][r] += be[r] * en[r] * M1[d][r] - gam[r] * M3[d][r];
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int m = 1; m < 16; m <<= 1) {
                pe[r] += xor_lane_f(pe[r], m);
                pf[r] += xor_lane_f(pf[r], m);
            }
            if (r16 == 0) {
                rEnd[16 * w + 4 * g + r] = en[r] * pe[r];
                rFrom[16 * w + 4 * g + r] = gam[r] * pf[r];
            }
        }
        // the pairs
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int cj = 16 * j + r16;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * w + 4 * g + r;
                float p = 0.f, n = 0.f, q = 0.f;
                if (cj <= i) {
                    const float bd = vb[cj] * gdn_decay(vlh[i], vll[i], vlh[cj], vll[cj]);
                    p = Z2[j][r] * bd;
                    n = cj < i ? Z[j][r] * bd : 0.f;
                    q = a.pm[(ch * 64 + i) * 64 + cj] * Z2[j][r];
                    if (cj < i) q -= a.nm[(ch * 64 + i) * 64 + cj] * Z[j][r];
                }
                mP[i * LD + cj] = p;
                mN[i * LD + cj] = n;
                mQ[i * LD + cj] = q;
            }
        }
        __syncthreads();
        {   // mB[i][t] = sum over j < t of mQ[i][j] beta_j: four threads a row, 16 columns each
            const int i = tid >> 2, s = tid & 3;
            float part = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) part = fmaf(mQ[i * LD + 16 * s + j], vb[16 * s + j], part);
            const float p1 = __shfl(part, (lane & ~3) + 0, 64), p2 = __shfl(part, (lane & ~3) + 1, 64),
                        p3 = __shfl(part, (lane & ~3) + 2, 64);
            float run = s == 0 ? 0.f : s == 1 ? p1 : s == 2 ? p1 + p2 : p1 + p2 + p3;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                mB[i * LD + 16 * s + j] = run;
                run = fmaf(mQ[i * LD + 16 * s + j], vb[16 * s + j], run);
            }
        }
        __syncthreads();
        {   // per token: column sums of mQ, and of mB from the token's own row down
            const int t = tid >> 2, s = tid & 3;
            float cs = 0.f, cr = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int i = 16 * s + j;
                cs += mQ[i * LD + t];
                cr += i >= t ? mB[i * LD + t] : 0.f;
            }
            cs += xor_lane_f(cs, 1);
            cr += xor_lane_f(cr, 1);
            cs += xor_lane_f(cs, 2);
            cr += xor_lane_f(cr, 2);
            if (s == 0) {
                rCol[t] = cs;
                rCross[t] = cr;
            }
        }
        __syncthreads();
        if (w == 0) {
            const bool ok = t0 + lane < len;
            const float end = rEnd[lane], be_end = vb[lane] * end;
            float suf = rFrom[lane], pre = be_end;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const float o = __shfl_down(suf, m, 64), u = __shfl_up(pre, m, 64);
                if (lane + m < 64) suf += o;
                if (lane >= m) pre += u;
            }
            const float before = __shfl_up(pre, 1, 64);
            const float thr = vec[GDN_V_GAM * 64 + 63] * (rThr[0] + rThr[1] + rThr[2] + rThr[3]);
            const float dl = rCross[lane] + suf + (lane ? before : 0.f) + thr;
            if (ok) {
                a.dalpha[tv + lane] = dl / vec[GDN_V_ALPHA * 64 + lane];
                a.dbeta[tv + lane] = rCol[lane] + end;
            }
        }
        // dq += mP K;  dk += mP^T Q - (mN + mN^T) K
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            float xp[8], xt[8], xn[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = 32 * kb + 8 * g + i;
                xp[i] = mP[arow * LD + j];
                xt[i] = mP[j * LD + arow];
                xn[i] = -(mN[arow * LD + j] + mN[j * LD + arow]);
            }
            const GdnFrag<3> fp = gdn_split(xp), ft = gdn_split(xt), fn = gdn_split(xn);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const GdnFrag<NT> k = gdn_load_frag<NT>(a.kt, (ck * DT + d) * 2 + kb);
                const GdnFrag<NT> q = gdn_load_frag<NT>(a.qt, (ck * DT + d) * 2 + kb);
                dq[d] = gdn_mm(fp, k, dq[d]);
                dk[d] = gdn_mm(ft, q, dk[d]);
                dk[d] = gdn_mm(fn, k, dk[d]);
            }
        }
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        const int dc = gdn_row(d, r16);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * w + 4 * g + r;
            if (dc < a.dk && t0 + i < len) {
                a.dq[(tq + i) * a.dk + dc] = dq[d][r];
                a.dkk[(tq + i) * a.dk + dc] = dk[d][r];
            }
        }
    }
}

template <typename VT, int KTN>
hipError_t launch_grads(const GdnArgs& a, hipStream_t st) {
    constexpr size_t stage = (size_t)(4 * KTN + 4) * 3 * GDN_FRAG * 2, pairs = (size_t)2 * 64 * LD * 4;
    constexpr size_t lds = (stage > pairs ? stage : pairs) + pairs + 8 * 64 * 4;
    const auto kfn = gdn_grads_kernel<VT, KTN>;
    hipError_t e = hipFuncSetAttribute((const void*)kfn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    kfn<<<dim3(a.nC, a.B * a.Hk), 256, lds, st>>>(a);
    return hipGetLastError();
}

}  // namespace

#define GDN_PICK(F)                                                      \
    do {                                                                 \
        if (a.dk <= 32) F(1);                                            \
        else if (a.dk <= 64) F(2);                                       \
        else if (a.dk <= 128) F(4);                                      \
        else F(8);                                                       \
    } while (0)

hipError_t sdm_launch_gdn_adjoint(const GdnArgs& a, hipStream_t st) {
    const dim3 grid((a.dv + 63) / 64 * a.B * a.H);
#define F(N)                                                                                 \
    do {                                                                                     \
        if (a.in_dtype == SDM_DT_BF16) return launch_adjoint_staged<N>(a, st);               \
        else gdn_adjoint_kernel<float, N><<<grid, 256, 0, st>>>(a);                          \
    } while (0)
    GDN_PICK(F);
#undef F
    return hipGetLastError();
}

hipError_t sdm_launch_gdn_grads(const GdnArgs& a, hipStream_t st) {
#define F(N) return a.in_dtype == SDM_DT_BF16 ? launch_grads<bf16_t, N>(a, st) : launch_grads<float, N>(a, st)
    GDN_PICK(F);
#undef F
}
