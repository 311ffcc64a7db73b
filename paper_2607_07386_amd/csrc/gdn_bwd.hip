// The dense gated delta rule, reverse mode (gfx950); notation as in gdn.hip.
// Sequential part (gdn_adjoint_halves_kernel), chunks last to first, with dS1 the
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

// Two waves to 16 columns as in the forward scan: half h
// holds tokens 32 h .. + 31 and one half of the state's rows.  dY is read whole by both
// (its part below needs no exchange); F = diag(beta) dE of the last 32 tokens and -G dR
// pass through LDS.  64 streams of 4096 tokens, 128 x 128: 295 to 310 us, 4.7 us a chunk, as the forward that
// keeps its states (316 to 330 us); of its bytes (0.6 GB) the states at the chunks' ends are 0.27 GB.
template <typename VT, int KTN, int NCT_>
struct AdjCfg {
    static constexpr int NT = GdnIn<VT>::NT;
    static constexpr int NCT = NCT_;
    static constexpr int NW = 2 * NCT;
    static constexpr int FPW = 4 * KTN / NW;
    static constexpr int TPW = (18 + NW - 1) / NW;
    static constexpr int XCH = (KTN + 3) * 3;          // S, then F_b, N_a, N_b
    // K's parts are 96 KB: Q^T (turned already for the gradients) and P^T come straight from memory (256 x 128
    // in fp32, 16 streams of 384 tokens: the backward 256 us, 432 by a wave to 16 columns that stages nothing)
    static constexpr bool DIRECT = NT == 3 && KTN == 8;
    static constexpr size_t LDS = (size_t)(4 * KTN * NT * (DIRECT ? 1 : 2) + (DIRECT ? 18 : 36) + NCT * XCH) * GDN_FRAG * 2 + 2 * 3 * 64 * 4;
};

template <typename VT, int KTN, int NCT>
__global__ __launch_bounds__(2 * NCT * 64) void gdn_adjoint_halves_kernel(GdnArgs a) {
    using C = AdjCfg<VT, KTN, NCT>;
    constexpr int NT = C::NT, NW = C::NW, KH = KTN / 2;
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t* sK = reinterpret_cast<uint16_t*>(smem);       // [4][KTN][NT]
    uint16_t* sQ = sK + 4 * KTN * NT * GDN_FRAG;
    uint16_t* sT = sQ + (C::DIRECT ? 0 : 4 * KTN * NT * GDN_FRAG);   // T'^T [6][3]
    uint16_t* sP = sT + GDN_BLKS * 3 * GDN_FRAG;            // P^T
    uint16_t* sX = sP + (C::DIRECT ? 0 : GDN_BLKS * 3 * GDN_FRAG);
    float* sV = reinterpret_cast<float*>(sX + C::NCT * C::XCH * GDN_FRAG);   // [2][gamma, end, beta][64]

    const int groups = (a.dv + 16 * C::NCT - 1) / (16 * C::NCT);
    int grp, bh;
    scan_wg_coords<true>(groups, grp, bh);
    const int b = bh / a.H, hk = (bh % a.H) / (a.H / a.Hk);
    const int len = gdn_len(a, b), nc = (len + GDN_C - 1) / GDN_C;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id(), r16 = lane & 15, g = lane >> 4;
    const int ct = w % C::NCT, h = w / C::NCT;
    const int col = (grp * C::NCT + ct) * 16 + r16;
    const uint32_t co = col < a.dv ? col * 4 : GDN_OUT;
    const size_t sn = (size_t)a.dk * a.dv;
    const sdm_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    uint16_t* xS = sX + ct * C::XCH * GDN_FRAG;             // [KTN][3]
    uint16_t *xF = xS + KTN * 3 * GDN_FRAG, *xA = xF + 3 * GDN_FRAG, *xB = xA + 3 * GDN_FRAG;

    const VT* kp = static_cast<const VT*>(a.k) + (size_t)(b * a.Hk + hk) * a.T * a.dk;
    const VT* qp = static_cast<const VT*>(a.q) + (size_t)(b * a.Hk + hk) * a.T * a.dk;
    const size_t ch0 = (size_t)bh * a.nC;

    sdm_f32x4 S[KTN];
    GdnFrag<3> sf[KH];
    gdn_load_state(S, a.dstateT ? a.dstateT + bh * sn : nullptr, h * KTN, a.dk, a.dv, co);
    const auto give_state = [&]() {
#pragma unroll
        for (int i = 0; i < KH; ++i) {
            sf[i] = gdn_stack(S[2 * i], S[2 * i + 1]);
            gdn_store_frag<3>(xS, h * KH + i, sf[i]);
        }
    };

    GdnAhead<VT, C::FPW> rK, rQ;
    u4v rT[C::TPW], rP[C::TPW];
    float rV, rY[4][4];
    const auto fetch_kq = [&](int c) {
        rK.template fetch<KTN>(kp + (size_t)c * GDN_C * a.dk, w * C::FPW, len - c * GDN_C, a.dk);
        if constexpr (!C::DIRECT) rQ.template fetch<KTN>(qp + (size_t)c * GDN_C * a.dk, w * C::FPW, len - c * GDN_C, a.dk);
        const int which = w == 0 ? GDN_V_GAM : w == 1 ? GDN_V_END : GDN_V_BETA;   // other waves repeat beta
        rV = a.vec[(ch0 + c) * GDN_VEC * 64 + which * 64 + lane];
    };
    float rB = 0.f;                                         // beta where the workgroup has two waves only
    const auto fetch_y = [&](int c) {
        const auto buf = gdn_buf(a.dy + ((size_t)bh * a.T + (size_t)c * GDN_C) * a.dv, (size_t)min(len - c * GDN_C, GDN_C) * a.dv * 4);
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) rY[m][r] = gdn_ldf(buf, gdn_row(m, 4 * g + r) * a.dv * 4 + co);
        if constexpr (NW == 2) rB = a.vec[(ch0 + c) * GDN_VEC * 64 + GDN_V_BETA * 64 + lane];
    };
    const auto fetch_t = [&](int c) { gdn_fetch_turns<NW>(rT, a.tf + (ch0 + c) * 18 * GDN_FRAG, 18, w); };
    const auto fetch_p = [&](int c) {
        if constexpr (!C::DIRECT) gdn_fetch_turns<NW>(rP, a.pf + (ch0 + c) * 18 * GDN_FRAG, 18, w);
    };
    const auto stage_p = [&]() {
        if constexpr (!C::DIRECT) gdn_stage_turns<NW>(sP, 18, w, rP);
    };
    const auto p_frag = [&](int c, int blk) {
        if constexpr (C::DIRECT) return gdn_load_frag<3>(a.pf, (ch0 + c) * GDN_BLKS + blk);
        else return gdn_load_frag<3>(sP, blk);
    };
    const auto q_turned = [&](int c, int dt, int kb) {
        if constexpr (C::DIRECT) return gdn_load_frag<NT>(a.qt, (((size_t)(b * a.Hk + hk) * a.nC + c) * 2 * KTN + dt) * 2 + kb);
        else return gdn_turned_frag<KTN, NT>(sQ, dt, kb);
    };
    const auto stage_kq = [&](int par) {
        rK.stage(sK, w * C::FPW);
        if constexpr (!C::DIRECT) rQ.stage(sQ, w * C::FPW);
        if (w < 3) sV[(par * 3 + w) * 64 + lane] = rV;
        if (NW == 2 && w == 0) sV[(par * 3 + 2) * 64 + lane] = rB;
    };

    if (nc > 0) {
        fetch_kq(nc - 1);
        fetch_y(nc - 1);
        fetch_t(nc - 1);
        fetch_p(nc - 1);
        give_state();
        stage_kq((nc - 1) & 1);
        gdn_stage_turns<NW>(sT, 18, w, rT);
        stage_p();
        const int c1 = max(nc - 2, 0);
        fetch_p(c1);
        fetch_t(c1);
        fetch_kq(c1);
        __syncthreads();
    }
    for (int c = nc - 1; c >= 0; --c) {
        const int left = len - c * GDN_C, next = max(c - 2, 0);
        const float* vec = sV + (c & 1) * 3 * 64;
        const auto rbuf = gdn_buf(a.dvv + ((size_t)bh * a.T + (size_t)c * GDN_C) * a.dv, (size_t)min(left, GDN_C) * a.dv * 4);
        gdn_store_state(S, a.dS + (ch0 + c) * sn, h * KTN, a.dk, a.dv, co);
        sdm_f32x4 dE[2], dR[2], Y[4];
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) Y[m][r] = rY[m][r];
#pragma unroll
        for (int m = 0; m < 2; ++m) dE[m] = dR[m] = zero;
        // dE = C K dS1 + P^T dY of this half's tokens
#pragma unroll
        for (int i = 0; i < KTN; ++i) {
            const int kb = i < KH ? h * KH + i : (1 - h) * KH + i - KH;
            const GdnFrag<3> s = i < KH ? sf[i < KH ? i : 0] : gdn_load_frag<3>(xS, kb);
#pragma unroll
            for (int m = 0; m < 2; ++m) dE[m] = gdn_mm(gdn_load_frag<NT>(sK, (2 * h + m) * KTN + kb), s, dE[m]);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const v4f en = ld4(vec + 64 + gdn_row(2 * h + m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) dE[m][r] *= en[r];
        }
        if (h == 0) {
            const GdnFrag<3> y = gdn_stack(Y[0], Y[1]);
#pragma unroll
            for (int m = 0; m < 2; ++m) dE[m] = gdn_mm(p_frag(c, gdn_up_blk(m, 0)), y, dE[m]);
        }
        {
            const GdnFrag<3> y = gdn_stack(Y[2], Y[3]);
#pragma unroll
            for (int m = 0; m < 2; ++m) dE[m] = gdn_mm(p_frag(c, h ? 4 + m : 2 * m + 1), y, dE[m]);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const v4f be = ld4(vec + 128 + gdn_row(2 * h + m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) dE[m][r] *= be[r];
        }
        const GdnFrag<3> ff = gdn_stack(dE[0], dE[1]);
        if (h == 1) gdn_store_frag<3>(xF, 0, ff);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const v4f gam = ld4(vec + gdn_row(m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) Y[m][r] *= gam[r];
        }
        const GdnFrag<3> y0 = gdn_stack(Y[0], Y[1]), y1 = gdn_stack(Y[2], Y[3]);
        __syncthreads();
        stage_p();
        fetch_y(max(c - 1, 0));
        fetch_p(next);
        // dR = T'^T F
        if (h == 0) {
            const GdnFrag<3> fb = gdn_load_frag<3>(xF, 0);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                dR[m] = gdn_mm(gdn_load_frag<3>(sT, gdn_up_blk(m, 0)), ff, dR[m]);
                dR[m] = gdn_mm(gdn_load_frag<3>(sT, gdn_up_blk(m, 1)), fb, dR[m]);
            }
        } else {
#pragma unroll
            for (int m = 0; m < 2; ++m) dR[m] = gdn_mm(gdn_load_frag<3>(sT, gdn_up_blk(2 + m, 1)), ff, dR[m]);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const v4f gam = ld4(vec + gdn_row(2 * h + m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                gdn_stf(rbuf, gdn_row(2 * h + m, 4 * g + r) * a.dv * 4 + co, dR[m][r]);
                dR[m][r] *= -gam[r];
            }
        }
        const GdnFrag<3> nf = gdn_stack(dR[0], dR[1]);
        gdn_store_frag<3>(h ? xB : xA, 0, nf);
        const float last = vec[63];
        __syncthreads();
        gdn_stage_turns<NW>(sT, 18, w, rT);
        fetch_t(next);
        // dS0 = gamma dS1 + Q^T (G dY) - K^T (G dR)
        {
            const GdnFrag<3> no = gdn_load_frag<3>(h ? xA : xB, 0);
#pragma unroll
            for (int d = 0; d < KTN; ++d) {
                S[d] *= last;
                S[d] = gdn_mm(q_turned(c, h * KTN + d, 0), y0, S[d]);
                S[d] = gdn_mm(q_turned(c, h * KTN + d, 1), y1, S[d]);
                S[d] = gdn_mm(gdn_turned_frag<KTN, NT>(sK, h * KTN + d, h), nf, S[d]);
                S[d] = gdn_mm(gdn_turned_frag<KTN, NT>(sK, h * KTN + d, 1 - h), no, S[d]);
            }
        }
        give_state();
        __syncthreads();
        stage_kq((c + 1) & 1);
        fetch_kq(next);
        __syncthreads();
    }
    if (a.dstate0) gdn_store_state(S, a.dstate0 + bh * sn, h * KTN, a.dk, a.dv, co);
}

template <typename VT, int KTN, int NCT>
hipError_t launch_adjoint_tiles(const GdnArgs& a, hipStream_t st) {
    using C = AdjCfg<VT, KTN, NCT>;
    const auto kfn = gdn_adjoint_halves_kernel<VT, KTN, NCT>;
    hipError_t e = hipFuncSetAttribute((const void*)kfn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::LDS);
    if (e != hipSuccess) return e;
    kfn<<<dim3((a.dv + 16 * C::NCT - 1) / (16 * C::NCT) * a.B * a.H), C::NW * 64, C::LDS, st>>>(a);
    return hipGetLastError();
}
// column tiles to a workgroup as in the forward scan
template <typename VT, int KTN>
hipError_t launch_adjoint(const GdnArgs& a, hipStream_t st) {
    const int64_t tiles = (int64_t)((a.dv + 15) / 16) * a.B * a.H, cus = sdm_device_simds() / 4;
    if constexpr (KTN == 2 || (KTN == 4 && sizeof(VT) == 2)) {
        if (tiles >= 4 * cus) return launch_adjoint_tiles<VT, KTN, 4>(a, st);
        if (tiles >= 2 * cus) return launch_adjoint_tiles<VT, KTN, 2>(a, st);
    }
    return launch_adjoint_tiles<VT, KTN, 1>(a, st);
}

// ---------------------------------------------------------------- gradients
constexpr int LD = 68;
// bytes of the staged fragments, or of what takes their place: two 64x64 matrices and, of bf16
// inputs, the fragments of K and Q
constexpr size_t grads_stage(int ktn, bool bf) {
    const size_t stage = (size_t)(4 * ktn + 4) * 3 * GDN_FRAG * 2,
                 pairs = (size_t)2 * 64 * LD * 4 + (bf ? (size_t)8 * ktn * GDN_FRAG * 2 : 0);
    return stage > pairs ? stage : pairs;
}

// One workgroup per (key head, chunk), over the heads that share the key head in
// order (their dq, dk add up reproducibly).  Eight waves: wave w holds
// tokens 16 (w & 3) .. + 15 and one half (w >> 2) of the columns of d_k.  Per 32 columns of
// d_v the workgroup stages S0, dS1 and X once as fragments in LDS, the next columns'
// values being fetched meanwhile; a row of a matrix is the same fragment as an A or
// a B operand, so every product over d_v reads its rows straight from memory.
// 4096 chunks of 128 x 128: 522 to 550 us for 0.80 GB, 1.5 TB/s.  One workgroup holds a compute unit (105 KB
// of LDS, 183 registers), so its two phases do not overlap another's: timed each by itself, the products
// over d_v take 370 us (290 without the matrix instructions, the loads' pace), the pairs 230.
// bf16 with d_k <= 128 and either type with d_k <= 64 keep all in registers; fp32 spills 113 of them (392 B of scratch a
// lane) for d_k <= 128, bf16 30 (108 B) and fp32 400 (1,500 B) beyond.  64 streams of 1024 tokens, d_v = 128: 143 us
// in bf16 and 286 in fp32 at d_k = 128, 240 and 947 at 256.
template <typename VT, int KTN>
__global__ __launch_bounds__(512, 2) void gdn_grads_kernel(GdnArgs a) {
    constexpr int NT = GdnIn<VT>::NT, DT = 2 * KTN, DH = KTN;   // DH: a wave's tiles of 16 columns of d_k
    constexpr int SR = (DT + 7) / 8;                            // tiles of S0, dS1 that a wave stages
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t* sS = reinterpret_cast<uint16_t*>(smem);                  // [DT][3] fragments
    uint16_t* sD = sS + DT * 3 * GDN_FRAG;
    uint16_t* sX = sD + DT * 3 * GDN_FRAG;                             // [4][3]
    float* mQ = reinterpret_cast<float*>(smem);                        // after the products, in their place
    float* mB = mQ + 64 * LD;
    uint16_t* sK = reinterpret_cast<uint16_t*>(mB + 64 * LD);          // [4][KTN] fragments (bf16)
    uint16_t* sQ = sK + 4 * KTN * GDN_FRAG;
    float* mP = reinterpret_cast<float*>(smem + grads_stage(KTN, NT == 1));
    float* mN = mP + 64 * LD;
    float* sV = mN + 64 * LD;                                          // the chunk's vectors
    const float *vlh = sV + GDN_V_LHI * 64, *vll = sV + GDN_V_LLO * 64, *vb = sV + GDN_V_BETA * 64;
    float *rEnd = sV + GDN_VEC * 64, *rFrom = rEnd + 128, *rThr = rFrom + 128, *rCol = rThr + 64, *rCross = rCol + 64;

    const int c = blockIdx.x, b = blockIdx.y / a.Hk, hk = blockIdx.y % a.Hk, G = a.H / a.Hk;
    const int len = gdn_len(a, b), t0 = c * GDN_C, left = len - t0;
    if (left <= 0) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int w = wave & 3, half = wave >> 2, d0 = half * DH;
    const size_t tq = (size_t)(b * a.Hk + hk) * a.T + t0;
    const size_t ck = (size_t)(b * a.Hk + hk) * a.nC + c;
    const sdm_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const int wk = w >> 1;                    // the 32 tokens that hold the wave's
    const int dvb = (a.dv + 31) / 32;
    const uint32_t rows_bytes = (uint32_t)min(left, GDN_C) * a.dv * 4, st_bytes = (uint32_t)a.dk * a.dv * 4;

    const size_t kq_n = (size_t)min(left, GDN_C) * a.dk;
    const auto bdq = gdn_buf(a.dq + tq * a.dk, kq_n * 4), bdk = gdn_buf(a.dkk + tq * a.dk, kq_n * 4);

    for (int hg = 0; hg < G; ++hg) {
        // Said to change, so that addresses and masks are formed where they are used: the same
        // for every head, they would be kept across the products (and spill, 16 KB a wave).
        int lane = lane_id();
        asm volatile("" : "+v"(lane));
        const int tid = wave * 64 + lane, r16 = lane & 15, g = lane >> 4;
        const int arow = gdn_row(w, r16);     // the A operands' token; in the C layout gdn_row(w, 4 g + r)
        const int bh = b * a.H + hk * G + hg;
        const size_t ch = (size_t)bh * a.nC + c, tv = (size_t)bh * a.T + t0;
        const float* vec = a.vec + ch * GDN_VEC * 64;
        const auto bS = gdn_buf(a.saved_S + ch * a.dk * a.dv, st_bytes), bD = gdn_buf(a.dS + ch * a.dk * a.dv, st_bytes);
        const auto bX = gdn_buf(a.saved_X + tv * a.dv, rows_bytes), bY = gdn_buf(a.dy + tv * a.dv, rows_bytes),
                   bR = gdn_buf(a.dvv + tv * a.dv, rows_bytes);
        // this lane's next 8 values of a row of each matrix
        float xX[8], xY[8], xR[8], xS[SR][8], xD[SR][8];
        const auto fetch = [&](int kb) {
            const uint32_t o = (uint32_t)(arow * a.dv + 32 * kb + 8 * g) * 4;
            const int p = 32 * kb + 8 * g;
            gdn_ld8(bX, o, p, a.dv, xX);
            gdn_ld8(bY, o, p, a.dv, xY);
            gdn_ld8(bR, o, p, a.dv, xR);
#pragma unroll
            for (int i = 0; i < SR; ++i) {
                const int d = wave + 8 * i;
                const uint32_t os = d < DT ? (uint32_t)(gdn_row(d, r16) * a.dv + 32 * kb + 8 * g) * 4 : GDN_OUT;
                gdn_ld8(bS, os, p, a.dv, xS[i]);
                gdn_ld8(bD, os, p, a.dv, xD[i]);
            }
        };
        fetch(0);
        __syncthreads();                      // the previous head's use of LDS
        if (tid < GDN_VEC * 64) sV[tid] = vec[tid];
        sdm_f32x4 M1[DH], M2[DH], M3[DH], Z[4];   // Z: dY X^T in the first half's waves, dR X^T in the second's
#pragma unroll
        for (int d = 0; d < DH; ++d) M1[d] = M2[d] = M3[d] = zero;
#pragma unroll
        for (int j = 0; j < 4; ++j) Z[j] = zero;
        float through = 0.f;
        for (int kb = 0; kb < dvb; ++kb) {
            const GdnFrag<3> fx = gdn_split(xX), fy = gdn_split(xY), fr = gdn_split(xR);
            if (half == 0) gdn_store_frag<3>(sX, w, fx);
#pragma unroll
            for (int i = 0; i < SR; ++i) {
                const int d = wave + 8 * i;
                if (d < DT) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) through = fmaf(xS[i][j], xD[i][j], through);
                    gdn_store_frag<3>(sS, d, gdn_split(xS[i]));
                    gdn_store_frag<3>(sD, d, gdn_split(xD[i]));
                }
            }
            fetch(min(kb + 1, dvb - 1));
            __syncthreads();
#pragma unroll
            for (int d = 0; d < DH; ++d) {
                const GdnFrag<3> s0 = gdn_load_frag<3>(sS, d0 + d);
                M2[d] = gdn_mm(fy, s0, M2[d]);
                M3[d] = gdn_mm(fr, s0, M3[d]);
                M1[d] = gdn_mm(fx, gdn_load_frag<3>(sD, d0 + d), M1[d]);
                __builtin_amdgcn_sched_barrier(0);   // one tile's fragments at a time: all of them would spill
            }
            const GdnFrag<3> fz = half == 0 ? fy : fr;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j >> 1 <= wk) Z[j] = gdn_mm(fz, gdn_load_frag<3>(sX, j), Z[j]);
            __syncthreads();
        }
        __builtin_amdgcn_sched_barrier(0);
        through = wave_sum(through);
        if (lane == 0) rThr[wave] = through;
        // K and Q of a bf16 input: their fragments go to LDS, where they are turned
        constexpr int FPW = KTN / 2;          // fragments of K and of Q that a wave moves
        GdnAhead<bf16_t, FPW> rK, rQ;
        if constexpr (NT == 1) {
            rK.template fetch<KTN>(static_cast<const bf16_t*>(a.k) + tq * a.dk, wave * FPW, left, a.dk);
            rQ.template fetch<KTN>(static_cast<const bf16_t*>(a.q) + tq * a.dk, wave * FPW, left, a.dk);
        }
        if constexpr (NT == 1) {
            rK.stage(sK, wave * FPW);
            rQ.stage(sQ, wave * FPW);
            __syncthreads();
        }
        // K^T, Q^T: columns of tile d0 + d, depths 32 kb on
        const auto kt = [&](int d, int kb) {
            if constexpr (NT == 1) return gdn_turned_frag<KTN>(sK, d0 + d, kb);
            else return gdn_load_frag<3>(a.kt, (ck * DT + d0 + d) * 2 + kb);
        };
        const auto qt = [&](int d, int kb) {
            if constexpr (NT == 1) return gdn_turned_frag<KTN>(sQ, d0 + d, kb);
            else return gdn_load_frag<3>(a.qt, (ck * DT + d0 + d) * 2 + kb);
        };
        // Q K^T (first half's waves) or K K^T of the wave's rows: P and N but for the decays
        sdm_f32x4 pn[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) pn[j] = zero;
#pragma unroll
        for (int kb = 0; kb < KTN; ++kb) {
            GdnFrag<NT> fa;
            if constexpr (NT == 1) fa = gdn_load_frag<1>(half == 0 ? sQ : sK, w * KTN + kb);
            else fa = gdn_row_frag<NT>(static_cast<const VT*>(half == 0 ? a.q : a.k) + (tq + arow) * a.dk, kb, a.dk, arow < left);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j >> 1 > wk) continue;
                GdnFrag<NT> fb;
                if constexpr (NT == 1) {
                    fb = gdn_load_frag<1>(sK, j * KTN + kb);
                } else {
                    const int row = gdn_row(j, r16);
                    fb = gdn_row_frag<NT>(static_cast<const VT*>(a.k) + (tq + row) * a.dk, kb, a.dk, row < left);
                }
                pn[j] = gdn_mm(fa, fb, pn[j]);
            }
        }
        // rows of M against q and k (this wave's own tokens are among the depths that each lane
        // holds of a turned fragment); then dq (in M2) and dk (in M1) without the pairs' part
        const int i0 = gdn_row(w, 4 * g);
        const v4f gam = ld4(sV + GDN_V_GAM * 64 + i0), en = ld4(sV + GDN_V_END * 64 + i0), be = ld4(vb + i0);
        float pe[4] = {0.f, 0.f, 0.f, 0.f}, pf[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < DH; ++d) {
            const GdnFrag<NT> fk = kt(d, wk), fq = qt(d, wk);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float kv = 0.f, qv = 0.f;
#pragma unroll
                for (int x = NT - 1; x >= 0; --x) {
                    kv += (float)(w & 1 ? fk.t[x][4 + r] : fk.t[x][r]);
                    qv += (float)(w & 1 ? fq.t[x][4 + r] : fq.t[x][r]);
                }
                pe[r] = fmaf(kv, M1[d][r], pe[r]);
                pf[r] = fmaf(qv, M2[d][r], fmaf(-kv, M3[d][r], pf[r]));
                M2[d][r] *= gam[r];
                M1[d][r] = be[r] * en[r] * M1[d][r] - gam[r] * M3[d][r];
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
                rEnd[half * 64 + i0 + r] = en[r] * pe[r];
                rFrom[half * 64 + i0 + r] = gam[r] * pf[r];
            }
        }
        // the pairs: P . Z2 in mQ, N . Z in mB
        {
            float *to = half == 0 ? mP : mN, *to2 = half == 0 ? mQ : mB;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int cj = gdn_row(j, r16);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = i0 + r;
                    const bool on = cj < i + (half == 0);
                    const float d = gdn_decay(vlh[i], vll[i], vlh[cj], vll[cj]);   // may overflow above the diagonal
                    const float z = on ? Z[j][r] * d : 0.f;
                    to[i * LD + cj] = z * vb[cj];
                    to2[i * LD + cj] = z * pn[j][r];
                }
            }
        }
        __syncthreads();
        {   // mQ <- P . Z2 - N . Z, mB[i][t] = sum over j < t of mQ[i][j] beta_j: eight threads a row
            const int i = tid >> 3, s = tid & 7;
            float q[8], part = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                q[j] = mQ[i * LD + 8 * s + j] - mB[i * LD + 8 * s + j];
                mQ[i * LD + 8 * s + j] = q[j];
                part = fmaf(q[j], vb[8 * s + j], part);
            }
            float run = part;                 // inclusive over the eight threads, then without this one's
#pragma unroll
            for (int m = 1; m < 8; m <<= 1) {
                const float o = __shfl_up(run, m, 8);
                if (s >= m) run += o;
            }
            run = __shfl_up(run, 1, 8);
            if (s == 0) run = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                mB[i * LD + 8 * s + j] = run;
                run = fmaf(q[j], vb[8 * s + j], run);
            }
        }
        __syncthreads();
        {   // per token: column sums of mQ, and of mB from the token's own row down
            const int t = tid >> 3, s = tid & 7;
            float cs = 0.f, cr = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = s + 8 * j;
                cs += mQ[i * LD + t];
                cr += i >= t ? mB[i * LD + t] : 0.f;
            }
#pragma unroll
            for (int m = 1; m < 8; m <<= 1) {
                cs += xor_lane_f(cs, m);
                cr += xor_lane_f(cr, m);
            }
            if (s == 0) {
                rCol[t] = cs;
                rCross[t] = cr;
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
            for (int d = 0; d < DH; ++d) {
                const GdnFrag<NT> fk = kt(d, kb);
                M2[d] = gdn_mm(fp, fk, M2[d]);
                M1[d] = gdn_mm(ft, qt(d, kb), M1[d]);
                M1[d] = gdn_mm(fn, fk, M1[d]);
            }
        }
        // added to what the heads before left there (this thread's own stores)
#pragma unroll
        for (int d = 0; d < DH; ++d) {
            const int dc = gdn_row(d0 + d, r16);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t o = dc < a.dk ? (uint32_t)((i0 + r) * a.dk + dc) * 4 : GDN_OUT;
                const float q0 = hg ? gdn_ldf(bdq, o) : 0.f, k0 = hg ? gdn_ldf(bdk, o) : 0.f;
                gdn_stf(bdq, o, q0 + M2[d][r]);
                gdn_stf(bdk, o, k0 + M1[d][r]);
            }
        }
        __syncthreads();
        if (wave == 0) {
            const bool ok = lane < left;
            const float end = rEnd[lane] + rEnd[64 + lane], be_end = vb[lane] * end;
            float suf = rFrom[lane] + rFrom[64 + lane], pre = be_end;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const float o = __shfl_down(suf, m, 64), u = __shfl_up(pre, m, 64);
                if (lane + m < 64) suf += o;
                if (lane >= m) pre += u;
            }
            const float before = __shfl_up(pre, 1, 64);
            float thr = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) thr += rThr[i];
            const float dl = rCross[lane] + suf + (lane ? before : 0.f) + sV[GDN_V_GAM * 64 + 63] * thr;
            if (ok) {
                a.dalpha[tv + lane] = dl / sV[GDN_V_ALPHA * 64 + lane];
                a.dbeta[tv + lane] = rCol[lane] + end;
            }
        }
    }
}

template <typename VT, int KTN>
hipError_t launch_grads(const GdnArgs& a, hipStream_t st) {
    constexpr size_t lds = grads_stage(KTN, sizeof(VT) == 2) + (size_t)2 * 64 * LD * 4 + (GDN_VEC + 7) * 64 * 4;
    const auto kfn = gdn_grads_kernel<VT, KTN>;
    hipError_t e = hipFuncSetAttribute((const void*)kfn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    kfn<<<dim3(a.nC, a.B * a.Hk), 512, lds, st>>>(a);
    return hipGetLastError();
}

}  // namespace

#define GDN_PICK(F)                                                      \
    do {                                                                 \
        if (a.dk <= 64) F(2);                                            \
        else if (a.dk <= 128) F(4);                                      \
        else F(8);                                                       \
    } while (0)

hipError_t sdm_launch_gdn_adjoint(const GdnArgs& a, hipStream_t st) {
#define F(N) return a.in_dtype == SDM_DT_BF16 ? launch_adjoint<bf16_t, N>(a, st) : launch_adjoint<float, N>(a, st)
    GDN_PICK(F);
#undef F
}

hipError_t sdm_launch_gdn_grads(const GdnArgs& a, hipStream_t st) {
#define F(N) return a.in_dtype == SDM_DT_BF16 ? launch_grads<bf16_t, N>(a, st) : launch_grads<float, N>(a, st)
    GDN_PICK(F);
#undef F
}
