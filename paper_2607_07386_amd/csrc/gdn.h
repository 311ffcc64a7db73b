// Shared pieces of the dense gated delta rule's kernels (gfx950): chunk layout,
// workspace, and matrix-core fragments of fp32 values.
//
// Precision.  State, innovations and outputs are fp32, and so is every product:
// an fp32 factor is cut into three bf16 parts of 8 significant bits each (24
// bits together, the value itself but for its last bit's rounding), and the
// products of parts whose orders add up to at most two are summed in fp32 on
// the matrix cores.  A bf16 input is one exact part, so bf16 x fp32 takes three
// products and fp32 x fp32 six; both are cheaper than the fp32 matrix
// instruction, which runs at 1/16 of the bf16 rate.
//
// Layout.  v_mfma_f32_16x16x32_bf16 takes A with row = lane & 15 and depths
// 8 (lane >> 4) + 0..7, B with column = lane & 15 likewise, and returns C with
// column = lane & 15 and rows 4 (lane >> 4) + 0..3.  Tiles of 16 rows come in
// pairs that cover 32 rows, row p of tile m being row gdn_row(m, p) of the matrix:
// lane group g then holds rows 8g .. 8g+7 of the 32 in its two tiles, which is a
// B operand of the next product as it is.  A wave chains state, innovations and
// output without moving a value between lanes.
#pragma once
#include "sdm_common.h"

#define GDN_C 64                   // tokens per chunk
#define GDN_VEC 6                  // per-chunk vectors of GDN_C floats: see below
#define GDN_ALPHA_MIN 1e-20f       // smaller forget gates count as this (their decays are logarithms)

enum { GDN_V_LHI = 0, GDN_V_LLO = 1, GDN_V_GAM = 2, GDN_V_END = 3, GDN_V_BETA = 4, GDN_V_ALPHA = 5 };

// 16x32 blocks (row block, depth block) of a lower and of an upper triangular 64x64 matrix
// that are not zero: lower (0,0) (1,0) (2,0) (2,1) (3,0) (3,1); upper (0,0) (0,1) (1,0) (1,1) (2,1) (3,1).
#define GDN_BLKS 6
__host__ __device__ constexpr int gdn_low_blk(int mt, int kb) { return mt < 2 ? mt : 2 + (mt - 2) * 2 + kb; }
__host__ __device__ constexpr int gdn_up_blk(int mt, int kb) { return mt < 2 ? mt * 2 + kb : 4 + (mt - 2); }

#define GDN_FRAG 512               // bf16 values of one fragment (64 lanes x 8)

struct GdnArgs {
    const void* q;
    const void* k;
    const void* v;
    int in_dtype;
    const float* alpha;
    const float* beta;
    const int32_t* lens;
    int B, Hk, H, T, dk, dv, nC;
    // forward
    const float* state0;
    float* stateT;
    float* y;
    float* saved_S;                // [B, H, nC, dk, dv] states at the chunks' starts, or NULL
    float* saved_X;                // [B, H, T, dv] v - read-back of every token
    // backward
    const float* dy;
    const float* dstateT;
    float *dq, *dkk, *dvv, *dalpha, *dbeta, *dstate0;
    // workspace
    float* vec;                    // [B H nC][GDN_VEC][64]
    uint16_t *tf, *pf;             // fragments of T' and P (forward), of their transposes (backward)
    uint16_t *kt, *qt;             // fragments of K^T, Q^T: [B Hk nC][dk/16][2][NT]
    float* dS;                     // [B H nC][dk][dv] adjoints at the chunks' ends (backward)
    // the forward scan in `segs` segments of `seg_len` chunks each (1: the whole sequence):
    int segs, seg_len;
    float* seg_z;                  // [segs][B H][dk][dv] a segment's end from the zero state, then from its true
                                   // start; in the last place the start of the sequence
    float* seg_phi;                // [segs - 1][B H][dk][dk] what it multiplies its start by
};

struct GdnWs {
    size_t vec, tf, pf, kt, qt, dS, seg_z, seg_phi, total;
    int segs, seg_len;
};
GdnWs gdn_ws(int B, int Hk, int H, int T, int dk, int dv, int in_dtype, bool backward);
hipError_t sdm_launch_gdn_step(const GdnArgs& a, hipStream_t st);
hipError_t sdm_launch_gdn_prep(const GdnArgs& a, bool backward, hipStream_t st);
hipError_t sdm_launch_gdn_scan(const GdnArgs& a, hipStream_t st);
hipError_t sdm_launch_gdn_adjoint(const GdnArgs& a, hipStream_t st);
hipError_t sdm_launch_gdn_grads(const GdnArgs& a, hipStream_t st);

#ifdef __HIP_DEVICE_COMPILE__
#define GDN_DEV __device__ __forceinline__
#else
#define GDN_DEV __device__ inline
#endif

template <int NT>
struct GdnFrag {
    sdm_bf16x8 t[NT];
};

GDN_DEV int gdn_len(const GdnArgs& a, int b) {
    if (!a.lens) return a.T;
    const int n = a.lens[b];
    return __builtin_amdgcn_readfirstlane(n < 0 ? 0 : (n > a.T ? a.T : n));   // one value for the workgroup
}

// upper halves of two words as one word (a in the low half)
GDN_DEV uint32_t gdn_pack_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Row of the matrix that row p of tile m holds (in the C layout p = 4 (lane >> 4) + r).
GDN_DEV int gdn_row(int m, int p) { return 32 * (m >> 1) + 8 * (p >> 2) + 4 * (m & 1) + (p & 3); }

// Eight fp32 values as three bf16 parts, x = t0 + t1 + t2 up to 2^-24 |x|: each part
// is the top 16 bits of what the parts before it leave (the differences are exact).
GDN_DEV GdnFrag<3> gdn_split(const float (&x)[8]) {
    union {
        uint32_t u[4];
        sdm_bf16x8 v;
    } p0, p1, p2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h[2], m[2], l[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float f = x[2 * i + j];
            h[j] = __float_as_uint(f);
            const float r = f - __uint_as_float(h[j] & 0xffff0000u);
            m[j] = __float_as_uint(r);
            l[j] = __float_as_uint(r - __uint_as_float(m[j] & 0xffff0000u));
        }
        p0.u[i] = gdn_pack_hi(h[0], h[1]);
        p1.u[i] = gdn_pack_hi(m[0], m[1]);
        p2.u[i] = gdn_pack_hi(l[0], l[1]);
    }
    GdnFrag<3> f;
    f.t[0] = p0.v;
    f.t[1] = p1.v;
    f.t[2] = p2.v;
    return f;
}

// Two C tiles (rows 0..15 and 16..31 of a depth block) as a B operand.
GDN_DEV GdnFrag<3> gdn_stack(const sdm_f32x4& lo, const sdm_f32x4& hi) {
    const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return gdn_split(x);
}

// c += A B over 32 depths: products of parts of total order <= 2, smallest first.
template <int NA, int NB>
GDN_DEV sdm_f32x4 gdn_mm(const GdnFrag<NA>& a, const GdnFrag<NB>& b, sdm_f32x4 c) {
#pragma unroll
    for (int o = 2; o >= 0; --o)
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (i + j == o) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.t[i], b.t[j], c, 0, 0, 0);
    return c;
}

// Depth block kb of one row of `n` values (n % 4 == 0; zeros past the end or where
// the row is none) in this lane group's depths.
GDN_DEV void gdn_row8(const float* row, int kb, int n, bool ok, float (&x)[8]) {
    const int p = 32 * kb + 8 * (lane_id() >> 4);
    const v4f a = ok && p < n ? ld4(row + p) : v4zero();
    const v4f b = ok && p + 4 < n ? ld4(row + p + 4) : v4zero();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = a[i];
        x[4 + i] = b[i];
    }
}
template <int NT>
GDN_DEV GdnFrag<NT> gdn_row_frag(const float* row, int kb, int n, bool ok) {
    float x[8];
    gdn_row8(row, kb, n, ok, x);
    return gdn_split(x);
}
template <int NT>
GDN_DEV GdnFrag<NT> gdn_row_frag(const bf16_t* row, int kb, int n, bool ok) {
    const int p = 32 * kb + 8 * (lane_id() >> 4);
    union {
        u2v u[2];
        sdm_bf16x8 v;
    } f;
    f.u[0] = ok && p < n ? *reinterpret_cast<const u2v*>(row + p) : u2v{0u, 0u};
    f.u[1] = ok && p + 4 < n ? *reinterpret_cast<const u2v*>(row + p + 4) : u2v{0u, 0u};
    GdnFrag<NT> r;
    r.t[0] = f.v;
    return r;
}

template <int NT>
GDN_DEV GdnFrag<NT> gdn_load_frag(const uint16_t* base, size_t idx) {
    GdnFrag<NT> f;
#pragma unroll
    for (int i = 0; i < NT; ++i)
        f.t[i] = *reinterpret_cast<const sdm_bf16x8*>(base + (idx * NT + i) * GDN_FRAG + lane_id() * 8);
    return f;
}
template <int NT>
GDN_DEV void gdn_store_frag(uint16_t* base, size_t idx, const GdnFrag<NT>& f) {
#pragma unroll
    for (int i = 0; i < NT; ++i)
        *reinterpret_cast<sdm_bf16x8*>(base + (idx * NT + i) * GDN_FRAG + lane_id() * 8) = f.t[i];
}

template <typename VT>
struct GdnIn;
template <>
struct GdnIn<float> {
    static constexpr int NT = 3;
};
template <>
struct GdnIn<bf16_t> {
    static constexpr int NT = 1;
};

// ---- staging of fragments: memory -> registers (a chunk ahead) -> LDS ----
// Buffers of one chunk or one state: a load past `bytes` gives zeros and a store there
// does nothing, so rows past a sequence's end and past d_k need no branch (a branch
// around a store makes the compiler wait for every load in flight at the next use).
// Columns past d_v take GDN_OUT for their offset.
#define GDN_OUT 0x40000000u
GDN_DEV __amdgpu_buffer_rsrc_t gdn_buf(const void* p, size_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}
GDN_DEV float gdn_ldf(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, (int)off, 0, 0));
}
GDN_DEV void gdn_stf(__amdgpu_buffer_rsrc_t r, uint32_t off, float x) {
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), r, (int)off, 0, 0);
}
template <typename VT>
GDN_DEV float gdn_ld1(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    if constexpr (sizeof(VT) == 4) return gdn_ldf(r, off);
    else return __uint_as_float((uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, (int)off, 0, 0) << 16);
}
// eight values of a row from its place p on (zeros past the row's n values)
GDN_DEV void gdn_ld8(__amdgpu_buffer_rsrc_t r, uint32_t off, int p, int n, float (&x)[8]) {
    const v4f a = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(p < n ? off : GDN_OUT), 0, 0));
    const v4f b = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(p + 4 < n ? off + 16 : GDN_OUT), 0, 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = a[i];
        x[4 + i] = b[i];
    }
}
// Fragments first .. first + N - 1 of the [4][KTN] of 64 rows of a matrix of `rows` rows of n
// values (n % 4 == 0): fragment (m, kb), lane row gdn_row(m, lane & 15).  Rows and depths past
// the end are zero.  fp32 values are fetched as they are and cut into parts when staged.
template <typename VT, int N>
struct GdnAhead;
template <int N>
struct GdnAhead<bf16_t, N> {
    u4v r[N];
    template <int KTN>
    GDN_DEV void fetch(const bf16_t* base, int first, int rows, int n) {
        const auto buf = gdn_buf(base, (size_t)min(rows, GDN_C) * n * 2);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int m = (first + i) / KTN, p = 32 * ((first + i) % KTN) + 8 * (lane_id() >> 4);
            const uint32_t o = (uint32_t)(gdn_row(m, lane_id() & 15) * n + p) * 2;
            if (n % 8 == 0) {
                r[i] = __builtin_bit_cast(u4v, __builtin_amdgcn_raw_buffer_load_b128(buf, (int)(p < n ? o : GDN_OUT), 0, 0));
            } else {
                const u2v lo = __builtin_bit_cast(u2v, __builtin_amdgcn_raw_buffer_load_b64(buf, (int)(p < n ? o : GDN_OUT), 0, 0));
                const u2v hi = __builtin_bit_cast(u2v, __builtin_amdgcn_raw_buffer_load_b64(buf, (int)(p + 4 < n ? o + 8 : GDN_OUT), 0, 0));
                r[i] = u4v{lo.x, lo.y, hi.x, hi.y};
            }
        }
    }
    GDN_DEV void stage(uint16_t* lds, int first) const {
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<u4v*>(lds + (first + i) * GDN_FRAG + lane_id() * 8) = r[i];
    }
};
template <int N>
struct GdnAhead<float, N> {
    float r[N][8];
    template <int KTN>
    GDN_DEV void fetch(const float* base, int first, int rows, int n) {
        const auto buf = gdn_buf(base, (size_t)min(rows, GDN_C) * n * 4);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int m = (first + i) / KTN, p = 32 * ((first + i) % KTN) + 8 * (lane_id() >> 4);
            gdn_ld8(buf, (uint32_t)(gdn_row(m, lane_id() & 15) * n + p) * 4, p, n, r[i]);
        }
    }
    GDN_DEV void stage(uint16_t* lds, int first) const {
#pragma unroll
        for (int i = 0; i < N; ++i) gdn_store_frag<3>(lds, first + i, gdn_split(r[i]));
    }
};
// Tiles d0 .. d0 + N - 1 of a state's 16 columns at the lane's column offset `co` (bytes), in the C layout.
template <int N>
GDN_DEV void gdn_load_state(sdm_f32x4 (&S)[N], const float* p, int d0, int dk, int dv, uint32_t co) {
    const auto buf = gdn_buf(p, p ? (size_t)dk * dv * 4 : 0);
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[d][r] = gdn_ldf(buf, gdn_row(d0 + d, 4 * (lane_id() >> 4) + r) * dv * 4 + co);
}
template <int N>
GDN_DEV void gdn_store_state(const sdm_f32x4 (&S)[N], float* p, int d0, int dk, int dv, uint32_t co) {
    const auto buf = gdn_buf(p, (size_t)dk * dv * 4);
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) gdn_stf(buf, gdn_row(d0 + d, 4 * (lane_id() >> 4) + r) * dv * 4 + co, S[d][r]);
}
// Fragments `wave`, `wave` + NW, ... of the n laid out at base (past the end: the last one again).
template <int NW, int N>
GDN_DEV void gdn_fetch_turns(u4v (&r)[N], const uint16_t* base, int n, int wave) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        r[i] = *reinterpret_cast<const u4v*>(base + (size_t)min(wave + NW * i, n - 1) * GDN_FRAG + lane_id() * 8);
}
template <int NW, int N>
GDN_DEV void gdn_stage_turns(uint16_t* lds, int n, int wave, const u4v (&r)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        *reinterpret_cast<u4v*>(lds + min(wave + NW * i, n - 1) * GDN_FRAG + lane_id() * 8) = r[i];
}
// Rows gdn_row(dt, .) of the transpose of a matrix that stands in LDS as the fragments
// [4][KTN] of its 64 rows, depths 32 kb .. 32 kb + 31 (its rows): the transposing read takes
// four rows of four columns from four lanes each, wherever they are.
template <int KTN, int NT = 1>
GDN_DEV GdnFrag<NT> gdn_turned_frag(const uint16_t* lds, int dt, int kb) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    const int l = lane_id(), row = 4 * (l >> 4) + ((l & 15) >> 2);   // row of the source tile
    GdnFrag<NT> r;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        union {
            s4 s[2];
            sdm_bf16x8 v;
        } f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint16_t* p = lds + (((2 * kb + h) * KTN + (dt >> 1)) * NT + x) * GDN_FRAG + ((l & 3) * 16 + row) * 8 + (dt & 1) * 4;
            f.s[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p);
        }
        r.t[x] = f.v;
    }
    return r;
}

// exp(lambda_i - lambda_j), the sums of log alpha held as two floats each (a
// difference of two long sums keeps its digits)
GDN_DEV float gdn_decay(float hi_i, float lo_i, float hi_j, float lo_j) {
    return expf((hi_i - hi_j) + (lo_i - lo_j));
}
