// The dense gated delta rule, forward (gfx950).  Per stream (b, h) with a state S
// of d_k x d_v values and t = 0 .. T-1 (Sec. 2, Eq. gdn-update; the recurrence
// whose key-value state the sparse table replaces, Sec. 3.1 "Connection to GDN"):
//   S <- alpha_t S;  e_t = beta_t (v_t - S^T k_t);  S <- S + k_t e_t^T;  y_t = S^T q_t
//
// Recurrent form (gdn_step_kernel): few tokens.  One pass over the state, which
// stays in registers; with u = S^T k, w = S^T q of the state before the token,
// y = alpha w + <k, q> e, so a token needs one reduction over the rows.
//
// Chunk form: tokens by 64.  With lambda_i the sum of log alpha up to token i of
// the chunk, gamma_i = exp(lambda_i), D_ij = exp(lambda_i - lambda_j) for j <= i:
//   N = stril(K K^T . D),  P = tril(Q K^T . D),  T' = (I + N diag(beta))^-1
//   X = T' (V - diag(gamma) K S0)          (X_t = v_t - its read-back)
//   E = diag(beta) X
//   Y = diag(gamma) Q S0 + P E
//   S1 = gamma_63 S0 + K^T diag(exp(lambda_63 - lambda)) E
// gdn_prep_kernel makes T' and P of all chunks in parallel; gdn_scan_halves_kernel walks the
// chunks of a stream, two waves to 16 columns of the state.  With few streams segments of the
// sequence run side by side: with V = 0 a segment multiplies its start by Phi, from the zero state it ends
// in Z, so S_{s+1} = Phi_s S_s + Z_s gives every segment's start (gdn_join_kernel).
#include <algorithm>

#include "gdn.h"
#include "sdm_internal.h"

namespace {

// ---------------------------------------------------------------- recurrent
// A workgroup holds 32 columns of one stream: 8 quads of columns x 32 row
// groups, rows rg + 32 i in registers.  One token of 256 streams of 128 x 128: 7.9 us, 4.3 TB/s
// (the state read and written once, a copy's rate being 4.8); of 16 streams 4.0 us, a launch.
template <typename VT, int NR>
__global__ __launch_bounds__(256) void gdn_step_kernel(GdnArgs a) {
    __shared__ float red[2][4][8][9];
    const int bh = blockIdx.y, b = bh / a.H, hk = (bh % a.H) / (a.H / a.Hk);
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    const int cq = lane & 7, rg = (lane >> 3) + 8 * wave;
    const int col = blockIdx.x * 32 + cq * 4;
    const bool cv = col < a.dv;
    const int len = gdn_len(a, b);
    const size_t sbase = (size_t)bh * a.dk * a.dv;
    v4f S[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int r = rg + 32 * i;
        S[i] = a.state0 && cv && r < a.dk ? ld4(a.state0 + sbase + (size_t)r * a.dv + col) : v4zero();
    }
    const size_t tq = (size_t)(b * a.Hk + hk) * a.T, tv = (size_t)bh * a.T;
    const VT* kp = static_cast<const VT*>(a.k) + tq * a.dk;
    const VT* qp = static_cast<const VT*>(a.q) + tq * a.dk;
    const VT* vp = static_cast<const VT*>(a.v) + tv * a.dv + (cv ? col : 0);
    // the next token's values are fetched while this one is reduced (rows past d_k and columns past
    // d_v read the first ones and are taken as zeros)
    VT nk[NR], nq[NR];
    v4f nv;
    float na, nb;
    const auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int r = rg + 32 * i < a.dk ? rg + 32 * i : 0;
            nk[i] = kp[(size_t)t * a.dk + r];
            nq[i] = qp[(size_t)t * a.dk + r];
        }
        nv = ld4v(vp + (size_t)t * a.dv);
        na = a.alpha[tv + t];
        nb = a.beta[tv + t];
    };
    if (len > 0) fetch(0);
    for (int t = 0; t < len; ++t) {
        float kr[NR], qr[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const bool ok = rg + 32 * i < a.dk;
            kr[i] = ok ? to_f32(nk[i]) : 0.f;
            qr[i] = ok ? to_f32(nq[i]) : 0.f;
        }
        const v4f vt = v4sel(cv, nv, v4zero());
        const float al = na, be = nb;
        fetch(min(t + 1, len - 1));
        v4f u = v4zero(), w = v4zero();
        float kq = 0.f;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            u = v4fma(kr[i], S[i], u);
            w = v4fma(qr[i], S[i], w);
            kq = fmaf(kr[i], qr[i], kq);
        }
#pragma unroll
        for (int m = 8; m <= 32; m <<= 1) {
            u += v4shfl_xor(u, m);
            w += v4shfl_xor(w, m);
            kq += xor_lane_f(kq, m);
        }
        float(&rd)[4][8][9] = red[t & 1];   // two of them: one barrier a token
        if (lane < 8) {
            float* p = rd[wave][cq];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] = u[i];
                p[4 + i] = w[i];
            }
            p[8] = kq;
        }
        __syncthreads();
        u = v4zero();
        w = v4zero();
        kq = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float* p = rd[j][cq];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u[i] += p[i];
                w[i] += p[4 + i];
            }
            kq += p[8];
        }
        v4f e, y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = be * (vt[i] - al * u[i]);
            y[i] = fmaf(kq, e[i], al * w[i]);
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            v4f n;
#pragma unroll
            for (int j = 0; j < 4; ++j) n[j] = fmaf(kr[i], e[j], al * S[i][j]);
            S[i] = n;
        }
        if (cv && rg == 0) st4(a.y + (tv + t) * a.dv + col, y);
    }
    if (a.stateT && cv) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int r = rg + 32 * i;
            if (r < a.dk) st4(a.stateT + sbase + (size_t)r * a.dv + col, S[i]);
        }
    }
}

// ---------------------------------------------------------------- prep
constexpr int LD = 68;   // row stride of the 64x64 fp32 matrices in LDS

// one 16x16x16 product of fp32 matrices in LDS: acc += A[ar..][ac..] B[br..][bc..]
__device__ __forceinline__ sdm_f32x4 lds_mm16(const float* A, int ar, int ac, const float* Bm, int br, int bc,
                                              int ldb, sdm_f32x4 acc) {
    const int r = lane_id() & 15, g = lane_id() >> 4;
#pragma unroll
    for (int k = 0; k < 16; k += 4)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(A[(ar + r) * LD + ac + k + g], Bm[(br + k + g) * ldb + bc + r],
                                                   acc, 0, 0, 0);
    return acc;
}

// One workgroup per (stream, chunk).  T' by blocks: the four 16x16 diagonal
// blocks by substitution (a lane per column), then the blocks below them from
// products, T'_21 = -T'_22 A_21 T'_11, first within each half, then between.
// Everything is latency, so what counts is how many workgroups share a compute unit:
// one 64x64 matrix in LDS serves A, then T' in its place, then P (23 KB, five workgroups).
// 8192 chunks of d_k = 128: 122 us, 0.44 GB moved, 3.6 TB/s (329 us with three matrices
// and K^T gathered for the scan, two workgroups).
template <typename VT, int KTN, bool BWD>
__global__ __launch_bounds__(256) void gdn_prep_kernel(GdnArgs a) {
    constexpr int NT = GdnIn<VT>::NT, DT = 2 * KTN;
    constexpr int KF = NT == 1 ? 4 * KTN * GDN_FRAG * 2 : 0, MW = (64 * LD + 32 * 36) * 4;
    __shared__ __align__(16) unsigned char smem[KF > MW ? KF : MW];
    __shared__ float vlh[64], vll[64], vb[64];
    uint16_t* sK = reinterpret_cast<uint16_t*>(smem);       // fragments of K, until M takes their place
    float* M = reinterpret_cast<float*>(smem);
    float* W = M + 64 * LD;
    const int c = blockIdx.x, bh = blockIdx.y, b = bh / a.H, h = bh % a.H;
    const int G = a.H / a.Hk, hk = h / G;
    const int len = gdn_len(a, b), t0 = c * GDN_C;
    if (t0 >= len) return;
    const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const size_t ch = (size_t)bh * a.nC + c;

    // Gram matrices: this wave's 16 rows against the rows of blocks 0 .. w
    const size_t tq = (size_t)(b * a.Hk + hk) * a.T + t0;
    const VT* kp = static_cast<const VT*>(a.k) + tq * a.dk;
    const VT* qp = static_cast<const VT*>(a.q) + tq * a.dk;
    sdm_f32x4 kk[4], qk[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) kk[j] = qk[j] = sdm_f32x4{0.f, 0.f, 0.f, 0.f};
    const int row = 16 * w + r16;
    const bool ok = t0 + row < len;
    const auto gates = [&]() {
        const int t = t0 + lane;
        const bool on = t < len;
        float al = on ? a.alpha[(size_t)bh * a.T + t] : 1.f;
        al = al < GDN_ALPHA_MIN ? GDN_ALPHA_MIN : al;
        const float be = on ? a.beta[(size_t)bh * a.T + t] : 0.f;
        // the logarithm in fp32 (its last bit counts as one more rounding of alpha), the sums
        // and their differences beyond that
        double lam = (double)logf(al);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const double o = __shfl_up(lam, m, 64);
            if (lane >= m) lam += o;
        }
        const double end = __shfl(lam, 63, 64);
        const float hi = (float)lam, lo = (float)(lam - (double)hi), he = (float)(end - lam);
        vlh[lane] = hi;
        vll[lane] = lo;
        vb[lane] = be;
        float* vec = a.vec + ch * GDN_VEC * 64;
        vec[GDN_V_LHI * 64 + lane] = hi;
        vec[GDN_V_LLO * 64 + lane] = lo;
        const float eh = expf(hi);
        vec[GDN_V_GAM * 64 + lane] = fmaf(eh, lo, eh);
        vec[GDN_V_END * 64 + lane] = expf(he);
        vec[GDN_V_BETA * 64 + lane] = be;
        vec[GDN_V_ALPHA * 64 + lane] = al;
    };
    if constexpr (NT == 1) {
        GdnFrag<1> fk[KTN], fq[KTN];
#pragma unroll
        for (int kb = 0; kb < KTN; ++kb) {
            fk[kb] = gdn_row_frag<1>(kp + (size_t)row * a.dk, kb, a.dk, ok);
            fq[kb] = gdn_row_frag<1>(qp + (size_t)row * a.dk, kb, a.dk, ok);
        }
        if (w == 0) gates();      // has one block of the products to do, wave 3 four
#pragma unroll
        for (int kb = 0; kb < KTN; ++kb) gdn_store_frag<1>(sK, w * KTN + kb, fk[kb]);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j > w) break;
#pragma unroll
            for (int kb = 0; kb < KTN; ++kb) {
                const GdnFrag<1> fb = gdn_load_frag<1>(sK, j * KTN + kb);
                kk[j] = gdn_mm(fk[kb], fb, kk[j]);
                qk[j] = gdn_mm(fq[kb], fb, qk[j]);
            }
        }
    } else {
        if (w == 0) gates();
        for (int kb = 0; kb < KTN; ++kb) {
            const GdnFrag<NT> fk = gdn_row_frag<NT>(kp + (size_t)row * a.dk, kb, a.dk, ok);
            const GdnFrag<NT> fq = gdn_row_frag<NT>(qp + (size_t)row * a.dk, kb, a.dk, ok);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j > w) break;
                const int rj = 16 * j + r16;
                const GdnFrag<NT> fb = gdn_row_frag<NT>(kp + (size_t)rj * a.dk, kb, a.dk, t0 + rj < len);
                kk[j] = gdn_mm(fk, fb, kk[j]);
                qk[j] = gdn_mm(fq, fb, qk[j]);
            }
        }
    }
    __syncthreads();
    // M = N diag(beta), zeros above the diagonal; P stays in qk
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int cj = 16 * j + r16;
        const float bj = vb[cj], hj = vlh[cj], lj = vll[cj];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * w + 4 * g + r;
            float n = 0.f, p = 0.f;
            if (j <= w) {
                const float d = gdn_decay(vlh[i], vll[i], hj, lj);   // may overflow above the diagonal
                n = cj < i ? kk[j][r] * d : 0.f;
                p = cj <= i ? qk[j][r] * d : 0.f;
            }
            M[i * LD + cj] = n * bj;
            qk[j][r] = p;
        }
    }
    __syncthreads();
    if (lane < 16) {   // diagonal block w, column `lane`, in place: the lanes read before any of them writes
        const int o = 16 * w;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == lane ? 1.f : 0.f;
#pragma unroll
            for (int l = 0; l < i; ++l) s = fmaf(-M[(o + i) * LD + o + l], x[l], s);
            x[i] = s;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 16; ++i) M[(o + i) * LD + o + lane] = x[i];
    }
    __syncthreads();
    const sdm_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    if (w < 2) {       // W <- A_21 T'_11 within half w
        const sdm_f32x4 t = lds_mm16(M, 32 * w + 16, 32 * w, M, 32 * w, 32 * w, LD, zero);
#pragma unroll
        for (int r = 0; r < 4; ++r) W[(16 * w + 4 * g + r) * 36 + r16] = t[r];
    }
    __syncthreads();
    if (w < 2) {
        const sdm_f32x4 t = lds_mm16(M, 32 * w + 16, 32 * w + 16, W, 16 * w, 0, 36, zero);
#pragma unroll
        for (int r = 0; r < 4; ++r) M[(32 * w + 16 + 4 * g + r) * LD + 32 * w + r16] = -t[r];
    }
    __syncthreads();
    {                  // between the halves: 32x32, a 16x16 tile per wave
        const int ti = w >> 1, tj = w & 1;
        sdm_f32x4 t = lds_mm16(M, 32 + 16 * ti, 0, M, 0, 16 * tj, LD, zero);
        t = lds_mm16(M, 32 + 16 * ti, 16, M, 16, 16 * tj, LD, t);
#pragma unroll
        for (int r = 0; r < 4; ++r) W[(16 * ti + 4 * g + r) * 36 + 16 * tj + r16] = t[r];
        __syncthreads();
        t = lds_mm16(M, 32 + 16 * ti, 32, W, 0, 16 * tj, 36, zero);
        t = lds_mm16(M, 32 + 16 * ti, 48, W, 16, 16 * tj, 36, t);
#pragma unroll
        for (int r = 0; r < 4; ++r) M[(32 + 16 * ti + 4 * g + r) * LD + 16 * tj + r16] = -t[r];
    }
    __syncthreads();
    // fragments of T', then of P (backward: of their transposes), 6 blocks each
    const auto blocks = [&](uint16_t* to) {
        for (int blk = w; blk < GDN_BLKS; blk += 4) {
            int mt, kb;
            if constexpr (BWD) {
                mt = blk < 4 ? blk >> 1 : blk - 2;
                kb = blk < 4 ? blk & 1 : 1;
            } else {
                mt = blk < 2 ? blk : 2 + ((blk - 2) >> 1);
                kb = blk < 2 ? 0 : (blk - 2) & 1;
            }
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int rr = gdn_row(mt, r16), cc = 32 * kb + 8 * g + i;
                x[i] = BWD ? M[cc * LD + rr] : M[rr * LD + cc];
            }
            gdn_store_frag<3>(to, ch * GDN_BLKS + blk, gdn_split(x));
        }
    };
    blocks(a.tf);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) M[(16 * w + 4 * g + r) * LD + 16 * j + r16] = qk[j][r];
    __syncthreads();
    blocks(a.pf);
    // fp32: K^T and Q^T of the key head, rows of d_k, depth = tokens, for the kernels that do not turn K in LDS
    if constexpr (NT == 3 && BWD) {
        if (h % G) return;
        const size_t ck = (size_t)(b * a.Hk + hk) * a.nC + c;
        for (int f = w; f < 2 * DT * 2; f += 4) {
            const int id = f % (DT * 2), dt = id >> 1, kb = id & 1;
            const VT* src = f < DT * 2 ? kp : qp;
            const int d = gdn_row(dt, r16);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int t = 32 * kb + 8 * g + i;
                x[i] = d < a.dk && t0 + t < len ? src[(size_t)t * a.dk + d] : 0.f;
            }
            gdn_store_frag<3>(f < DT * 2 ? a.kt : a.qt, ck * DT * 2 + id, gdn_split(x));
        }
    }
}

// ---------------------------------------------------------------- scan
// Two waves to 16 columns: half h holds tokens 32 h .. + 31 of the
// chunk and one half of the state's rows, so that a chunk's chain of dependent products
// is half as long and twice as many waves share the device.  What a half needs of the
// other (the state's fragments, R and E of the first 32 tokens, E for the update)
// passes through LDS.  The chunk's K, Q, T' and P are fetched into registers a chunk
// ahead and staged once for the workgroup; K^T is K read with the transposing loads.
// 128 streams of 4096 tokens, 128 x 128: 305 us in a short run, 4.8 us a chunk (350 in
// a long one).  Two waves share a SIMD there; a chunk takes each 108 matrix instructions, which
// keep the matrix pipe for 1,720 cycles, and 420 vector ones, and its unit's LDS 4,130 cycles (bank
// conflicts 770): pipes near each other's pace and four barriers between
// dependent stages.  HBM sees 0.62 GB (2.0 TB/s).  16 streams, 128 column tiles in all: 3.5 us a chunk,
// the chain of dependent products.  (A wave to 16 columns took 6.2 us a chunk.)
template <typename VT, int KTN, int NCT_>
struct ScanCfg {
    static constexpr int NT = GdnIn<VT>::NT;
    static constexpr int NCT = NCT_;                   // column tiles of a workgroup
    static constexpr int NW = 2 * NCT;
    static constexpr bool QD = NT == 1 ? KTN == 8 : KTN >= 4;   // Q straight from memory: LDS is full
    // P as well: K's parts are 96 KB, and it leaves 152 KB in all (256 x 128 in fp32, 16 streams of 384
    // tokens: 106 us, 301 by a wave to 16 columns that stages nothing; 64 of 1024: 645, 1087)
    static constexpr bool PD = NT == 3 && KTN == 8;
    static constexpr int FPW = 4 * KTN / NW;           // fragments of K (and Q) that a wave moves
    static constexpr int TPW = (18 + NW - 1) / NW;     // of T' (and P)
    static constexpr int XCH = (KTN + 3) * 3;          // exchanged fragments per column tile: S, then E_a, E'_a, E'_b (R_a)
    static constexpr size_t LDS =
        (size_t)(4 * KTN * NT * (QD ? 1 : 2) + (PD ? 18 : 36) + NCT * XCH) * GDN_FRAG * 2 + 2 * 3 * 64 * 4;
};

// MODE 0: outputs; 1: and what the backward needs; 2: only a segment's end, from the zero state (columns of
// d_v) and from each unit vector with V = 0 (columns of d_k, after those of d_v).
template <typename VT, int KTN, int NCT, int MODE>
__global__ __launch_bounds__(2 * NCT * 64) void gdn_scan_halves_kernel(GdnArgs a) {
    using C = ScanCfg<VT, KTN, NCT>;
    constexpr bool SAVE = MODE == 1, STATE = MODE == 2;
    constexpr int NT = C::NT, NW = C::NW, KH = KTN / 2;     // KH: 32-row blocks of the state per wave
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t* sK = reinterpret_cast<uint16_t*>(smem);       // [4][KTN][NT]
    uint16_t* sT = sK + 4 * KTN * NT * GDN_FRAG;                 // T' [6][3]
    uint16_t* sP = sT + GDN_BLKS * 3 * GDN_FRAG;
    uint16_t* sX = sP + (C::PD ? 0 : GDN_BLKS * 3 * GDN_FRAG);   // exchange, per column tile
    float* sV = reinterpret_cast<float*>(sX + C::NCT * C::XCH * GDN_FRAG);   // [2][gamma, end, beta][64]
    uint16_t* sQ = reinterpret_cast<uint16_t*>(sV + 2 * 3 * 64);             // [4][KTN][NT] unless QD

    const int tiles_v = (a.dv + 15) / 16, tiles = STATE ? tiles_v + (a.dk + 15) / 16 : tiles_v;
    const int groups = (tiles + C::NCT - 1) / C::NCT;
    int grp, stream;
    scan_wg_coords<true>(groups, grp, stream);
    const int BH = a.B * a.H, seg = stream / BH, bh = stream % BH;
    const int b = bh / a.H, hk = (bh % a.H) / (a.H / a.Hk);
    const int len = gdn_len(a, b), cb = seg * a.seg_len, ce = min((len + GDN_C - 1) / GDN_C, cb + a.seg_len);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id(), r16 = lane & 15, g = lane >> 4;
    const int ct = w % C::NCT, h = w / C::NCT;
    const bool unit = STATE && grp * C::NCT + ct >= tiles_v;   // a column of the multiplier
    const int col = (grp * C::NCT + ct - (unit ? tiles_v : 0)) * 16 + r16;
    const bool cv = col < (unit ? a.dk : a.dv);
    // column offsets: fp32, v's type
    const uint32_t co = cv ? col * 4 : GDN_OUT, cov = cv && !unit ? col * sizeof(VT) : GDN_OUT;
    const size_t sn = (size_t)a.dk * a.dv;
    const sdm_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    uint16_t* xS = sX + ct * C::XCH * GDN_FRAG;             // [KTN][3]
    uint16_t *xE = xS + KTN * 3 * GDN_FRAG, *xA = xE + 3 * GDN_FRAG, *xB = xA + 3 * GDN_FRAG;   // xB: R_a until E'_b

    const VT* kp = static_cast<const VT*>(a.k) + (size_t)(b * a.Hk + hk) * a.T * a.dk;
    const VT* qp = static_cast<const VT*>(a.q) + (size_t)(b * a.Hk + hk) * a.T * a.dk;
    const VT* vp = static_cast<const VT*>(a.v) + (size_t)bh * a.T * a.dv;
    const size_t ch0 = (size_t)bh * a.nC;

    sdm_f32x4 S[KTN];                                       // this half's tiles
    GdnFrag<3> sf[KH];                                      // and their fragments
    if constexpr (STATE) {
#pragma unroll
        for (int d = 0; d < KTN; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[d][r] = unit && gdn_row(h * KTN + d, 4 * g + r) == col ? 1.f : 0.f;
    } else {
        // segments side by side: the first one's start is the join's copy, since another segment's
        // workgroup may have stored stateT, which may be state0, before this one begins
        const float* s0 = a.segs > 1 ? a.seg_z + ((size_t)(seg ? seg - 1 : a.segs - 1) * BH + bh) * sn
                                     : a.state0 ? a.state0 + bh * sn : nullptr;
        gdn_load_state(S, s0, h * KTN, a.dk, a.dv, co);
    }
    const auto give_state = [&]() {
#pragma unroll
        for (int i = 0; i < KH; ++i) {
            sf[i] = gdn_stack(S[2 * i], S[2 * i + 1]);
            gdn_store_frag<3>(xS, h * KH + i, sf[i]);
        }
    };

    GdnAhead<VT, C::FPW> rK, rQ;
    u4v rT[C::TPW], rP[C::TPW];
    float rV, rB = 0.f, V[2][4];                            // rB: beta where the workgroup has two waves
    const auto fetch_k = [&](int c) { rK.template fetch<KTN>(kp + (size_t)c * GDN_C * a.dk, w * C::FPW, len - c * GDN_C, a.dk); };
    const auto fetch_q = [&](int c) {
        if constexpr (!C::QD && !STATE) rQ.template fetch<KTN>(qp + (size_t)c * GDN_C * a.dk, w * C::FPW, len - c * GDN_C, a.dk);
        const int which = w == 0 ? GDN_V_GAM : w == 1 ? GDN_V_END : GDN_V_BETA;   // waves 3 on repeat wave 2
        rV = a.vec[(ch0 + c) * GDN_VEC * 64 + which * 64 + lane];
        if constexpr (NW == 2) rB = a.vec[(ch0 + c) * GDN_VEC * 64 + GDN_V_BETA * 64 + lane];
    };
    const auto fetch_v = [&](int c) {
        const int t0 = c * GDN_C;
        const auto buf = gdn_buf(vp + (size_t)t0 * a.dv, (size_t)min(len - t0, GDN_C) * a.dv * sizeof(VT));
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) V[m][r] = gdn_ld1<VT>(buf, gdn_row(2 * h + m, 4 * g + r) * a.dv * sizeof(VT) + cov);
    };
    const auto fetch_t = [&](int c) { gdn_fetch_turns<NW>(rT, a.tf + (ch0 + c) * 18 * GDN_FRAG, 18, w); };
    const auto fetch_p = [&](int c) {
        if constexpr (!C::PD) gdn_fetch_turns<NW>(rP, a.pf + (ch0 + c) * 18 * GDN_FRAG, 18, w);
    };
    const auto stage_p = [&]() {
        if constexpr (!C::PD) gdn_stage_turns<NW>(sP, 18, w, rP);
    };
    const auto p_frag = [&](int c, int blk) {
        if constexpr (C::PD) return gdn_load_frag<3>(a.pf, (ch0 + c) * GDN_BLKS + blk);
        else return gdn_load_frag<3>(sP, blk);
    };
    const auto stage_k = [&]() { rK.stage(sK, w * C::FPW); };
    const auto stage_q = [&](int par) {
        if constexpr (!C::QD && !STATE) rQ.stage(sQ, w * C::FPW);
        if (w < 3) sV[(par * 3 + w) * 64 + lane] = rV;
        if (NW == 2 && w == 0) sV[(par * 3 + 2) * 64 + lane] = rB;
    };

    if (cb < ce) {
        fetch_k(cb);
        fetch_q(cb);
        fetch_v(cb);
        fetch_t(cb);
        if constexpr (!STATE) fetch_p(cb);
        give_state();
        stage_k();
        stage_q(cb & 1);
        gdn_stage_turns<NW>(sT, 18, w, rT);
        if constexpr (!STATE) stage_p();
        const int c1 = min(cb + 1, ce - 1);
        fetch_q(c1);
        fetch_t(c1);
        if constexpr (!STATE) fetch_p(c1);
        fetch_k(c1);
        __syncthreads();
    }
    // (the last chunks fetch and stage once more what nobody reads: without the
    // branches the compiler counts the loads in flight across the loop)
    for (int c = cb; c < ce; ++c) {
        const int t0 = c * GDN_C, left = len - t0, next = min(c + 2, ce - 1);
        const float* vec = sV + (c & 1) * 3 * 64;
        const size_t row0 = (size_t)bh * a.T + t0, rows = min(left, GDN_C);
        const auto ybuf = gdn_buf(a.y + row0 * a.dv, rows * a.dv * 4);
        const auto xbuf = gdn_buf(SAVE ? a.saved_X + row0 * a.dv : nullptr, rows * a.dv * 4);
        if constexpr (SAVE) gdn_store_state(S, a.saved_S + (ch0 + c) * sn, h * KTN, a.dk, a.dv, co);
        // R = V - gamma K S0 and Y = gamma Q S0 of this half's tokens
        sdm_f32x4 R[2], Y[2], X[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) R[m] = Y[m] = X[m] = zero;
        const auto rows_by_state = [&](int kb, const GdnFrag<3>& s) {
#pragma unroll
            for (int m = 0; m < 2; ++m) R[m] = gdn_mm(gdn_load_frag<NT>(sK, (2 * h + m) * KTN + kb), s, R[m]);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                if constexpr (STATE) continue;
                if constexpr (C::QD) {
                    const int row = gdn_row(2 * h + m, r16);
                    Y[m] = gdn_mm(gdn_row_frag<NT>(qp + (size_t)(t0 + row) * a.dk, kb, a.dk, row < left), s, Y[m]);
                } else {
                    Y[m] = gdn_mm(gdn_load_frag<NT>(sQ, (2 * h + m) * KTN + kb), s, Y[m]);
                }
            }
        };
#pragma unroll
        for (int i = 0; i < KH; ++i) rows_by_state(h * KH + i, sf[i]);
#pragma unroll
        for (int i = 0; i < KH; ++i) rows_by_state((1 - h) * KH + i, gdn_load_frag<3>(xS, (1 - h) * KH + i));
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const v4f gam = ld4(vec + gdn_row(2 * h + m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                R[m][r] = fmaf(-gam[r], R[m][r], V[m][r]);   // 0 past the end: K and V are
                Y[m][r] *= gam[r];
            }
        }
        const GdnFrag<3> rf = gdn_stack(R[0], R[1]);
        if (h == 0) gdn_store_frag<3>(xB, 0, rf);
        __syncthreads();
        stage_q((c + 1) & 1);
        fetch_v(min(c + 1, ce - 1));
        fetch_q(next);
        // X = T' R, E = beta X
        if (h == 1) {
            const GdnFrag<3> ra = gdn_load_frag<3>(xB, 0);
#pragma unroll
            for (int m = 0; m < 2; ++m) X[m] = gdn_mm(gdn_load_frag<3>(sT, gdn_low_blk(2 + m, 0)), ra, X[m]);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) X[m] = gdn_mm(gdn_load_frag<3>(sT, h ? 3 + 2 * m : m), rf, X[m]);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const v4f be = ld4(vec + 128 + gdn_row(2 * h + m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (SAVE) gdn_stf(xbuf, gdn_row(2 * h + m, 4 * g + r) * a.dv * 4 + co, X[m][r]);
                X[m][r] *= be[r];
            }
        }
        const GdnFrag<3> ef = gdn_stack(X[0], X[1]);
        if (!STATE && h == 0) gdn_store_frag<3>(xE, 0, ef);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const v4f en = ld4(vec + 64 + gdn_row(2 * h + m, 4 * g));
#pragma unroll
            for (int r = 0; r < 4; ++r) X[m][r] *= en[r];
        }
        const GdnFrag<3> uf = gdn_stack(X[0], X[1]);
        gdn_store_frag<3>(h ? xB : xA, 0, uf);
        const float last = vec[63];
        __syncthreads();
        gdn_stage_turns<NW>(sT, 18, w, rT);
        fetch_t(next);
        // S = gamma S + K^T (C E), then Y += P E
        {
            const GdnFrag<3> uo = gdn_load_frag<3>(h ? xA : xB, 0);
#pragma unroll
            for (int d = 0; d < KTN; ++d) {
                S[d] *= last;
                S[d] = gdn_mm(gdn_turned_frag<KTN, NT>(sK, h * KTN + d, h), uf, S[d]);
                S[d] = gdn_mm(gdn_turned_frag<KTN, NT>(sK, h * KTN + d, 1 - h), uo, S[d]);
            }
        }
        if constexpr (!STATE) {
            if (h == 1) {
                const GdnFrag<3> ea = gdn_load_frag<3>(xE, 0);
#pragma unroll
                for (int m = 0; m < 2; ++m) Y[m] = gdn_mm(p_frag(c, gdn_low_blk(2 + m, 0)), ea, Y[m]);
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) Y[m] = gdn_mm(p_frag(c, h ? 3 + 2 * m : m), ef, Y[m]);
        }
        give_state();
        if constexpr (!STATE) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) gdn_stf(ybuf, gdn_row(2 * h + m, 4 * g + r) * a.dv * 4 + co, Y[m][r]);
        }
        __syncthreads();
        if constexpr (!STATE) stage_p();
        stage_k();
        if constexpr (!STATE) fetch_p(next);
        fetch_k(next);
        __syncthreads();
    }
    if constexpr (STATE) {
        const size_t at = (size_t)seg * BH + bh;
        gdn_store_state(S, unit ? a.seg_phi + at * a.dk * a.dk : a.seg_z + at * sn, h * KTN, a.dk, unit ? a.dk : a.dv, co);
    } else if (seg == a.segs - 1) {
        gdn_store_state(S, a.stateT + bh * sn, h * KTN, a.dk, a.dv, co);
    }
}

// Starts of the segments, one after the other: S_{s+1} = Phi_s S_s + Z_s in Z_s's place.  A workgroup takes
// 16 columns of a stream, its four waves a quarter of the rows each; the state passes from
// segment to segment as fragments in LDS (two of them, one barrier a segment).  Seven joins of 16
// streams: 37 us, each a read of Phi that waits for nothing but is not fetched ahead.
template <int KTN>
__global__ __launch_bounds__(256) void gdn_join_kernel(GdnArgs a) {
    constexpr int N = KTN / 2;               // row tiles of a wave
    __shared__ __align__(16) uint16_t sS[2][KTN * 3 * GDN_FRAG];
    const int bh = blockIdx.y, BH = a.B * a.H;
    const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15;
    const int col = blockIdx.x * 16 + r16;
    const uint32_t co = col < a.dv ? col * 4 : GDN_OUT;
    const size_t sn = (size_t)a.dk * a.dv;
    // pairs of tiles make a fragment, so a wave of one tile (KTN 2) leaves the cutting to waves 0 and 1
    sdm_f32x4 S[KTN == 2 ? 2 : N];
    const int d0 = KTN == 2 ? 2 * w : w * N;
    const bool holds = KTN > 2 || w < 2;
    gdn_load_state(S, a.state0 && holds ? a.state0 + bh * sn : nullptr, d0, a.dk, a.dv, co);
    if (holds) gdn_store_state(S, a.seg_z + ((size_t)(a.segs - 1) * BH + bh) * sn, d0, a.dk, a.dv, co);
    for (int s = 0; s + 1 < a.segs; ++s) {
        uint16_t* f = sS[s & 1];
        const size_t at = (size_t)s * BH + bh;
        if (holds) {
#pragma unroll
            for (int i = 0; i < (KTN == 2 ? 1 : N / 2); ++i)
                gdn_store_frag<3>(f, d0 / 2 + i, gdn_stack(S[2 * i], S[2 * i + 1]));
            gdn_load_state(S, a.seg_z + at * sn, d0, a.dk, a.dv, co);
        }
        __syncthreads();
        if (holds) {
#pragma unroll
            for (int kb = 0; kb < KTN; ++kb) {
                const GdnFrag<3> x = gdn_load_frag<3>(f, kb);
#pragma unroll
                for (int d = 0; d < (KTN == 2 ? 2 : N); ++d) {
                    const int row = gdn_row(d0 + d, r16);
                    S[d] = gdn_mm(gdn_row_frag<3>(a.seg_phi + (at * a.dk + row) * a.dk, kb, a.dk, row < a.dk), x, S[d]);
                }
            }
            gdn_store_state(S, a.seg_z + at * sn, d0, a.dk, a.dv, co);
        }
    }
}

template <typename VT, int KTN, int NCT, int MODE>
hipError_t launch_scan_tiles(const GdnArgs& a, hipStream_t st) {
    using C = ScanCfg<VT, KTN, NCT>;
    const auto kfn = gdn_scan_halves_kernel<VT, KTN, NCT, MODE>;
    hipError_t e = hipFuncSetAttribute((const void*)kfn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)C::LDS);
    if (e != hipSuccess) return e;
    const int tiles = (a.dv + 15) / 16 + (MODE == 2 ? (a.dk + 15) / 16 : 0), segs = MODE == 2 ? a.segs - 1 : a.segs;
    kfn<<<dim3((tiles + C::NCT - 1) / C::NCT * a.B * a.H * segs), C::NW * 64, C::LDS, st>>>(a);
    return hipGetLastError();
}

// Column tiles to a workgroup: as many as leave a workgroup to every compute unit. More
// share one staging of the chunk, but also one LDS, whose reads then set the pace.
constexpr int scan_most(int ktn, bool f32) { return ktn == 2 ? 4 : ktn == 4 ? (f32 ? 2 : 4) : f32 ? 1 : 2; }   // what LDS holds
int scan_nct(int64_t tiles, int most) {
    const int64_t cus = sdm_device_simds() / 4;
    return most >= 4 && tiles >= 4 * cus ? 4 : most >= 2 && tiles >= 2 * cus ? 2 : 1;
}
template <typename VT, int KTN, int MODE>
hipError_t launch_scan_halves(const GdnArgs& a, hipStream_t st) {
    constexpr int MOST = scan_most(KTN, sizeof(VT) == 4);
    const int64_t cols = (a.dv + 15) / 16 + (MODE == 2 ? (a.dk + 15) / 16 : 0);
    const int nct = scan_nct(cols * a.B * a.H * (MODE == 2 ? a.segs - 1 : a.segs), MOST);
    if constexpr (MOST == 4) {
        if (nct == 4) return launch_scan_tiles<VT, KTN, 4, MODE>(a, st);
    }
    if constexpr (MOST >= 2) {
        if (nct == 2) return launch_scan_tiles<VT, KTN, 2, MODE>(a, st);
    }
    return launch_scan_tiles<VT, KTN, 1, MODE>(a, st);
}

template <typename VT, int KTN, bool SAVE>
hipError_t launch_scan(const GdnArgs& a, hipStream_t st) {
    if (a.segs > 1) {
        hipError_t e = launch_scan_halves<VT, KTN, 2>(a, st);
        if (e != hipSuccess) return e;
        gdn_join_kernel<KTN><<<dim3((a.dv + 15) / 16, a.B * a.H), 256, 0, st>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return launch_scan_halves<VT, KTN, SAVE ? 1 : 0>(a, st);
}

// Time of a chunk of `streams` streams of `cols` column tiles each, in chunks of one workgroup of one tile:
// the rounds of workgroups, a compute unit holding one, by what a chunk of two and of four tiles takes.
double scan_chunk_time(int64_t cols, int64_t streams, int most) {
    const int64_t cus = sdm_device_simds() / 4;
    const int nct = scan_nct(cols * streams, most);
    const int64_t wgs = (cols + nct - 1) / nct * streams;
    return (double)((wgs + cus - 1) / cus) * (nct == 4 ? 1.3 : nct == 2 ? 1.1 : 1.0);
}

// Segments of a sequence of nC chunks.  Few streams leave the device idle while chunk follows chunk.  Segments
// side by side first need each one's end, from the zero state and from the unit vectors (d_k / 16 more tiles;
// such a chunk takes 0.65 of the time, 0.35 where Q would come straight from memory), and the joins, two
// chunks' time each; then they run as many times fewer chunks in a row.  Five of 16 chunks or more,
// where that sum is below 0.92 of one pass.  Measured with and without at 390 shapes (either type, d_k
// 64 to 256, d_v 16 to 1024, 1 to 204 streams, 5,120 to 65,536 tokens): the sum is off by 12% in the mean, no
// shape that it takes was slower, and of those it leaves one would gain 16%, three 4%.  16 streams of 65,536 tokens, bf16,
// 128 x 128: 3.8 ms in one, 1.65 in eight; fp32, 256 x 128, 16,384 tokens: 5.1 ms either way, left in one; of
// 24 streams 5.2 and 7.4.
int gdn_segments(int64_t BH, int64_t nC, int dk, int dv, bool f32) {
    const int ktn = dk <= 64 ? 2 : dk <= 128 ? 4 : 8, most = scan_most(ktn, f32);
    const bool direct = f32 ? ktn >= 4 : ktn == 8;
    const int64_t cols = (dv + 15) / 16, tiles = cols * BH, room = tiles > 0 ? 4 * (sdm_device_simds() / 4) / tiles : 0;
    int64_t n = std::min<int64_t>(std::min<int64_t>(room, nC / 16), 64);
    if (n < 5) return 1;
    const int64_t len = (nC + n - 1) / n;
    n = (nC + len - 1) / len;
    const double in_parts = len * ((direct ? 0.35 : 0.65) * scan_chunk_time(cols + (dk + 15) / 16, BH * (n - 1), most) +
                                   scan_chunk_time(cols, BH * n, most)) + 2.0 * (n - 1);
    return in_parts < 0.92 * nC * scan_chunk_time(cols, BH, most) ? (int)n : 1;
}

}  // namespace

GdnWs gdn_ws(int B, int Hk, int H, int T, int dk, int dv, int in_dtype, bool backward) {
    GdnWs w{};
    const size_t nC = ((size_t)T + GDN_C - 1) / GDN_C;
    const size_t n = (size_t)B * H * nC, nk = (size_t)B * Hk * nC;
    const size_t dt = dk <= 64 ? 4 : dk <= 128 ? 8 : 16;
    const bool f32 = in_dtype == SDM_DT_F32;
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += (bytes + 255) & ~(size_t)255;
        return at;
    };
    w.vec = take(n * GDN_VEC * 64 * 4);
    w.tf = take(n * GDN_BLKS * 3 * GDN_FRAG * 2);
    w.pf = take(n * GDN_BLKS * 3 * GDN_FRAG * 2);
    w.segs = backward ? 1 : gdn_segments((int64_t)B * H, (int64_t)nC, dk, dv, f32);
    w.seg_len = (int)((nC + w.segs - 1) / w.segs);
    if (w.seg_len > 0) w.segs = (int)((nC + w.seg_len - 1) / w.seg_len);
    if (w.segs > 1) {
        w.seg_z = take((size_t)w.segs * B * H * dk * dv * 4);
        w.seg_phi = take((size_t)(w.segs - 1) * B * H * dk * dk * 4);
    }
    if (backward) {
        w.kt = take(f32 ? nk * dt * 2 * 3 * GDN_FRAG * 2 : 0);
        w.qt = take(f32 ? nk * dt * 2 * 3 * GDN_FRAG * 2 : 0);
        w.dS = take(n * dk * dv * 4);
    }
    w.total = o;
    return w;
}

#define GDN_PICK_KTN(K)                                  \
    do {                                                 \
        if (a.dk <= 64) K(2);                            \
        else if (a.dk <= 128) K(4);                      \
        else K(8);                                       \
    } while (0)

hipError_t sdm_launch_gdn_step(const GdnArgs& a, hipStream_t st) {
    const dim3 grid((a.dv + 31) / 32, a.B * a.H);
#define GDN_STEP(VT)                                                                       \
    do {                                                                                   \
        if (a.dk <= 64) gdn_step_kernel<VT, 2><<<grid, 256, 0, st>>>(a);                   \
        else if (a.dk <= 128) gdn_step_kernel<VT, 4><<<grid, 256, 0, st>>>(a);             \
        else gdn_step_kernel<VT, 8><<<grid, 256, 0, st>>>(a);                              \
    } while (0)
    if (a.in_dtype == SDM_DT_BF16) GDN_STEP(bf16_t);
    else GDN_STEP(float);
    return hipGetLastError();
}

hipError_t sdm_launch_gdn_prep(const GdnArgs& a, bool backward, hipStream_t st) {
    const dim3 grid(a.nC, a.B * a.H);
    const bool bf = a.in_dtype == SDM_DT_BF16;
#define K(N)                                                                                 \
    do {                                                                                     \
        if (bf && backward) gdn_prep_kernel<bf16_t, N, true><<<grid, 256, 0, st>>>(a);       \
        else if (bf) gdn_prep_kernel<bf16_t, N, false><<<grid, 256, 0, st>>>(a);             \
        else if (backward) gdn_prep_kernel<float, N, true><<<grid, 256, 0, st>>>(a);         \
        else gdn_prep_kernel<float, N, false><<<grid, 256, 0, st>>>(a);                      \
    } while (0)
    GDN_PICK_KTN(K);
#undef K
    return hipGetLastError();
}

hipError_t sdm_launch_gdn_scan(const GdnArgs& a, hipStream_t st) {
    const bool bf = a.in_dtype == SDM_DT_BF16, save = a.saved_S != nullptr;
#define K(N)                                                       \
    do {                                                           \
        if (bf && save) return launch_scan<bf16_t, N, true>(a, st); \
        if (bf) return launch_scan<bf16_t, N, false>(a, st);       \
        if (save) return launch_scan<float, N, true>(a, st);       \
        return launch_scan<float, N, false>(a, st);                \
    } while (0)
    GDN_PICK_KTN(K);
#undef K
}
