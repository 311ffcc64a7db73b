// Projections (gfx950): y = act(x W^T + bias) + residual and its gradients, the
// products on either side of the layer's recurrence (Sec. 3.1: W_q, W_k, W_v, W_a,
// W_b, W_g before it, W_o and the residual stream after it), reading and writing the
// recurrences' head-major layout.
//   forward   C[m, n] = sum_k x[m, k] w[n, k]
//   dx        C[m, k] = sum_n dz[m, n] w[n, k],   dz = dy act'(z)
//   dw        C[n, k] = sum_m dz[m, n] x[m, k],   dbias[n] = sum_m dz[m, n]
#include <algorithm>

#include "linear.h"
#include "sdm_common.h"
#include "sdm_internal.h"

namespace {

__device__ __forceinline__ int64_t mat_off(const LinMat& m, int i, int j) {
    return (int64_t)(i / m.T) * m.sb + (int64_t)(i % m.T) * m.st + (int64_t)(j / m.d) * m.sh + j % m.d;
}
__device__ __forceinline__ int64_t mat_row(const LinMat& m, int i) {
    return (int64_t)(i / m.T) * m.sb + (int64_t)(i % m.T) * m.st;
}
__device__ __forceinline__ int64_t mat_col(const LinMat& m, int j) { return (int64_t)(j / m.d) * m.sh + j % m.d; }

// round to nearest even
__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ void put(bf16_t* p, float x) { p->bits = bf16_bits(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }

constexpr float kSqrtHalf = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f;
__device__ __forceinline__ float lin_act(float z, int act) {
    if (act == 1) return z * sdm_sigmoid(z);
    if (act == 2) return 0.5f * z * (1.f + erff(z * kSqrtHalf));
    return z;
}
__device__ __forceinline__ float lin_act_slope(float z, int act) {
    if (act == 1) {
        const float s = sdm_sigmoid(z);
        return s * (1.f + z * (1.f - s));
    }
    if (act == 2) return 0.5f * (1.f + erff(z * kSqrtHalf)) + z * expf(-0.5f * z * z) * kInvSqrt2Pi;
    return 1.f;
}

__device__ __forceinline__ float ld_any(const void* p, int dtype, int64_t i) {
    return dtype == SDM_DT_F32 ? static_cast<const float*>(p)[i] : to_f32(static_cast<const bf16_t*>(p)[i]);
}
__device__ __forceinline__ void st_any(void* p, int dtype, int64_t i, float x) {
    if (dtype == SDM_DT_F32) static_cast<float*>(p)[i] = x;
    else put(static_cast<bf16_t*>(p) + i, x);
}

// one value of the result through the epilogue
__device__ __forceinline__ void lin_store(const LinGemm& g, int64_t o, int j, float c) {
    if (g.bias) c += g.bias[j];
    if (g.pre) st_any(g.pre, g.out.dtype, o, c);
    c = lin_act(c, g.act);
    if (g.residual) c += ld_any(g.residual, g.out.dtype, o);
    st_any(const_cast<void*>(g.out.p), g.out.dtype, o, c);
}

typedef unsigned short lin_us8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ void ld8(const void* p, int dtype, int64_t o, float (&x)[8]) {
    if (dtype == SDM_DT_F32) {
        const v4f a = ld4(static_cast<const float*>(p) + o), b = ld4(static_cast<const float*>(p) + o + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
    } else {
        const lin_us8 v = *reinterpret_cast<const lin_us8*>(static_cast<const bf16_t*>(p) + o);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float((uint32_t)v[i] << 16);
    }
}
__device__ __forceinline__ void st8(void* p, int dtype, int64_t o, const float (&x)[8]) {
    if (dtype == SDM_DT_F32) {
        st4(static_cast<float*>(p) + o, v4f{x[0], x[1], x[2], x[3]});
        st4(static_cast<float*>(p) + o + 4, v4f{x[4], x[5], x[6], x[7]});
    } else {
        lin_us8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = bf16_bits(x[i]);
        *reinterpret_cast<lin_us8*>(static_cast<bf16_t*>(p) + o) = v;
    }
}
// Eight neighbouring columns of a row may be moved at once: rows, heads and the row's
// end are multiples of 8 values.
__device__ __forceinline__ bool lin_wide(const LinGemm& g) { return g.J % 8 == 0 && g.out.d % 8 == 0; }

// Columns j .. j+7 of the row at offset `ro`; `b` the bias there.
__device__ __forceinline__ void lin_store8(const LinGemm& g, bool wide, int64_t ro, int j, const float (&b)[8],
                                           float (&c)[8]) {
    if (!wide) {
        for (int i = 0; i < 8 && j + i < g.J; ++i) lin_store(g, ro + mat_col(g.out, j + i), j + i, c[i]);
        return;
    }
    const int64_t o = ro + mat_col(g.out, j);
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] += b[i];
    if (g.pre) st8(g.pre, g.out.dtype, o, c);
    if (g.act == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = lin_act(c[i], 1);
    } else if (g.act == 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = lin_act(c[i], 2);
    }
    if (g.residual) {
        float r[8];
        ld8(g.residual, g.out.dtype, o, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] += r[i];
    }
    st8(const_cast<void*>(g.out.p), g.out.dtype, o, c);
}

// ---------------------------------------------------------------- general kernel
// 128 x 128 x 32 tiles for any sizes, layouts and types: LDS rows are output
// indices, so a factor stored depth-first is turned while it is staged.
constexpr int GT = 128, GK = 32;
template <typename CT>
struct GenTile;
template <>
struct GenTile<bf16_t> {
    static constexpr int LD = GK + 8, PIECE = 8;
};
template <>
struct GenTile<float> {
    static constexpr int LD = GK + 4, PIECE = 4;
};

// PIECE consecutive values along the matrix's columns, as CT (zeros outside)
template <typename CT, typename ST>
__device__ __forceinline__ void gen_load(const LinMat& m, int row, int col, CT (&x)[GenTile<CT>::PIECE]) {
    constexpr int P = GenTile<CT>::PIECE;
    const bool ok = row < m.rows && col < m.cols;
    const ST* p = static_cast<const ST*>(m.p) + (ok ? mat_off(m, row, col) : 0);
#pragma unroll
    for (int i = 0; i < P; i += 4) {
        const v4f v = ok ? ld4v(p + i) : v4zero();
#pragma unroll
        for (int j = 0; j < 4; ++j) put(&x[i + j], v[j]);
    }
}

template <typename CT, typename ST, bool TR>
__device__ __forceinline__ void gen_stage(const LinMat& m, int o0, int r0, CT* lds) {
    constexpr int P = GenTile<CT>::PIECE, LD = GenTile<CT>::LD;
    constexpr int per_row = (TR ? GT : GK) / P, rows = TR ? GK : GT;
    for (int u = threadIdx.x; u < rows * per_row; u += 256) {
        const int r = u / per_row, c = u % per_row * P;
        CT x[P];
        gen_load<CT, ST>(m, (TR ? r0 : o0) + r, (TR ? o0 : r0) + c, x);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if constexpr (TR) lds[(c + i) * LD + r] = x[i];
            else lds[r * LD + c + i] = x[i];
        }
    }
}

template <typename CT, typename AT, typename BT, bool TA, bool TB>
__global__ __launch_bounds__(256) void linear_general_kernel(LinGemm g) {
    constexpr int LD = GenTile<CT>::LD;
    __shared__ __align__(16) CT sA[GT * LD], sB[GT * LD];
    const int i0 = blockIdx.x * GT, j0 = blockIdx.y * GT;
    const int lane = lane_id(), w = threadIdx.x >> 6, r16 = lane & 15, q = lane >> 4;
    const int wi = (w >> 1) * 64, wj = (w & 1) * 64;
    sdm_f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = sdm_f32x4{0.f, 0.f, 0.f, 0.f};
    const int steps = (g.R + GK - 1) / GK, per = (steps + g.split - 1) / g.split;
    const int s0 = blockIdx.z * per, s1 = min(steps, s0 + per);
    for (int s = s0; s < s1; ++s) {
        gen_stage<CT, AT, TA>(g.a, i0, s * GK, sA);
        gen_stage<CT, BT, TB>(g.b, j0, s * GK, sB);
        __syncthreads();
        if constexpr (sizeof(CT) == 2) {
            sdm_bf16x8 fa[4], fb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fa[i] = *reinterpret_cast<const sdm_bf16x8*>(sA + (wi + 16 * i + r16) * LD + 8 * q);
                fb[i] = *reinterpret_cast<const sdm_bf16x8*>(sB + (wj + 16 * i + r16) * LD + 8 * q);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
        } else {
#pragma unroll
            for (int k = 0; k < GK; k += 4) {
                float fa[4], fb[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    fa[i] = sA[(wi + 16 * i + r16) * LD + k + q];
                    fb[i] = sB[(wj + 16 * i + r16) * LD + k + q];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[i], fb[j], acc[i][j], 0, 0, 0);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int oi = i0 + wi + 16 * i + 4 * q + r, oj = j0 + wj + 16 * j + r16;
                if (oi >= g.I || oj >= g.J) continue;
                if (g.split > 1) g.part[((size_t)blockIdx.z * g.I + oi) * g.J + oj] = acc[i][j][r];
                else lin_store(g, mat_off(g.out, oi, oj), oj, acc[i][j][r]);
            }
}

// The partial sums of a split depth, added in order, through the epilogue: eight
// columns of a row per thread.
__global__ __launch_bounds__(256) void linear_join_kernel(LinGemm g) {
    const int j = (blockIdx.x * 32 + (threadIdx.x & 31)) * 8;
    if (j >= g.J) return;
    const bool wide = lin_wide(g);
    const size_t n = (size_t)g.I * g.J;
    float b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = g.bias && j + i < g.J ? g.bias[j + i] : 0.f;
    for (int row = blockIdx.y * 8 + (threadIdx.x >> 5); row < g.I; row += gridDim.y * 8) {
        const float* p = g.part + (size_t)row * g.J + j;
        float c[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < g.split; ++s) {
            if (wide) {
                const v4f u = ld4(p + s * n), v = ld4(p + s * n + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    c[i] += u[i];
                    c[4 + i] += v[i];
                }
            } else {
                for (int i = 0; i < 8 && j + i < g.J; ++i) c[i] += p[s * n + i];
            }
        }
        lin_store8(g, wide, mat_row(g.out, row), j, b, c);
    }
}

// ---------------------------------------------------------------- tiled kernel
// bf16 factors: BM x BN x 64 tiles, WR x WC waves of 32x32x16 matrix instructions.
// The next tile goes straight from memory to LDS while this one is multiplied; a
// factor stored with its output index as the row is [BM][64] there, one stored depth
// first stays [64][BM] and is turned by the transposing LDS reads.  A piece of 16
// bytes stands at its place XOR a function of its row, so that the lanes of a
// read fall on different banks (the pieces of one direct load go to consecutive
// addresses, so the order is chosen by which piece a lane fetches).
typedef float lin_f32x16 __attribute__((ext_vector_type(16)));
typedef short lin_s4 __attribute__((ext_vector_type(4)));

constexpr int BK = 64;
constexpr uint32_t LIN_OUT = 0x80000000u;   // offset of what lies outside a matrix: loads of it give zeros

__device__ __forceinline__ __amdgpu_buffer_rsrc_t lin_buf(const bf16_t* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p), 0, 0x7fffffff, 0x00020000);
}
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, uint32_t off, void* l) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)l, 16, (int)off, 0, 0, 0);
}

// A factor's tile: O output indices x 64 depths.  Each of the NW waves moves O / (8 NW)
// runs of 1 KB.  A lane's places are 32-bit byte offsets from a base that moves along
// the depth, so that a step costs no vector arithmetic where the depth runs evenly
// (offsets_fit() says whether they do; EVEN: 64 depths always follow one another).
template <int O, int NW, bool TR, bool EVEN>
struct LinTile {
    static constexpr int RUNS = O / (8 * NW);
    static constexpr int PPR = (TR ? O : BK) / 8;      // pieces of a row of the tile in LDS
    static constexpr int RPR = 64 / PPR;               // rows of a run
    static constexpr int MASK = PPR / 4 - 1;           // TR: 4 pieces (32 outputs) move together
    const bf16_t* base;      // !TR: start of the first row's sequence; TR: of the matrix
    uint32_t off[RUNS];      // !TR: the lane's rows; TR: the lane's columns

    __device__ __forceinline__ static int swz(int r) { return TR ? 4 * (r & MASK) : r & 7; }
    __device__ __forceinline__ static int run0() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * RUNS; }
    __device__ __forceinline__ static int row() { return lane_id() / PPR; }
    // the piece of its row that the lane fetches: rows of runs differ by 8 or more (!TR)
    __device__ __forceinline__ static int piece(int r) { return (lane_id() % PPR) ^ swz(r); }

    __device__ __forceinline__ void init(const LinMat& m, int o0) {
        base = static_cast<const bf16_t*>(m.p);
        if constexpr (!TR) {
            const int seq = o0 / m.T;
            base += (int64_t)seq * m.sb;
#pragma unroll
            for (int i = 0; i < RUNS; ++i) {
                const int o = o0 + (run0() + i) * RPR + row();
                off[i] = o < m.rows ? (uint32_t)((int64_t)(o / m.T - seq) * m.sb + (int64_t)(o % m.T) * m.st) * 2 : LIN_OUT;
            }
        } else {
#pragma unroll
            for (int i = 0; i < RUNS; ++i) {
                const int c = o0 + piece((run0() + i) * RPR + row()) * 8;
                off[i] = c < m.cols ? (uint32_t)mat_col(m, c) * 2 : LIN_OUT;
            }
        }
    }
    __device__ __forceinline__ void fetch(const LinMat& m, int r0, unsigned char* lds) {
        if constexpr (!TR) {
            if constexpr (EVEN) {
                const auto buf = lin_buf(base + mat_col(m, r0));
                const uint32_t pc = piece(row()) * 16;
#pragma unroll
                for (int i = 0; i < RUNS; ++i) dma16(buf, off[i] + pc, lds + (run0() + i) * 1024);
            } else {
                const int c = r0 + piece(row()) * 8;
                const uint32_t o = c < m.cols ? (uint32_t)mat_col(m, c) * 2 : LIN_OUT;
#pragma unroll
                for (int i = 0; i < RUNS; ++i) dma16(lin_buf(base), (off[i] | o) & LIN_OUT ? LIN_OUT : off[i] + o, lds + (run0() + i) * 1024);
            }
        } else {
            const int seq = r0 / m.T;
            const auto buf = lin_buf(base + (int64_t)seq * m.sb + (int64_t)(r0 - seq * m.T) * m.st);
            if constexpr (EVEN) {
#pragma unroll
                for (int i = 0; i < RUNS; ++i)
                    dma16(buf, off[i] + ((run0() + i) * RPR + row()) * (uint32_t)m.st * 2, lds + (run0() + i) * 1024);
            } else {
#pragma unroll
                for (int i = 0; i < RUNS; ++i) {
                    const int kr = (run0() + i) * RPR + row(), t = r0 - seq * m.T + kr;
                    const int64_t o = (int64_t)(t / m.T) * m.sb + (int64_t)(t % m.T - (r0 - seq * m.T)) * m.st;
                    const uint32_t at = off[i] + (uint32_t)((int)o * 2);
                    dma16(buf, r0 + kr < m.rows && !(off[i] & LIN_OUT) ? at : LIN_OUT, lds + (run0() + i) * 1024);
                }
            }
        }
    }
    // 32 outputs from `o` on, depths 16 kk .. 16 kk + 15: output = lane & 31, 8 depths a lane half
    __device__ __forceinline__ static sdm_bf16x8 frag(const unsigned char* lds, int o, int kk) {
        const int lane = lane_id();
        if constexpr (!TR) {
            const int r = o + (lane & 31), c = (2 * kk + (lane >> 5)) ^ swz(r);
            return *reinterpret_cast<const sdm_bf16x8*>(lds + r * 128 + c * 16);
        } else {
            const int k = 16 * kk + 8 * (lane >> 5) + ((lane & 15) >> 2);
            const int c = o / 8 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            union {
                lin_s4 s[2];
                sdm_bf16x8 v;
            } f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned char* a = lds + (k + 4 * h) * (O * 2) + (c ^ swz(k + 4 * h)) * 16 + (lane & 1) * 8;
                f.s[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) lin_s4*)a);
            }
            return f.v;
        }
    }
};

template <int BM, int BN, int WR, int WC, bool TA, bool TB, bool EVEN>
__global__ __launch_bounds__(WR* WC * 64) void linear_tile_kernel(LinGemm g, int tiles_j) {
    constexpr int NW = WR * WC, MI = BM / WR / 32, NJ = BN / WC / 32;
    __shared__ __align__(1024) unsigned char sA0[BM * BK * 2], sA1[BM * BK * 2], sB0[BN * BK * 2], sB1[BN * BK * 2];
    using TileA = LinTile<BM, NW, TA, EVEN>;
    using TileB = LinTile<BN, NW, TB, EVEN>;

    // Workgroups go to the 8 XCDs in turn: give each a contiguous range of tiles, and walk
    // the range in columns of 8 row tiles, so that an L2 sees few rows and columns at a time.
    const int tiles_i = (g.I + BM - 1) / BM, n = tiles_i * tiles_j;
    int id = blockIdx.x;
    {
        const int q = n / 8, rem = n % 8, x = id % 8;
        id = (x < rem ? x * (q + 1) : rem * (q + 1) + (x - rem) * q) + id / 8;
    }
    const int band = id / (8 * tiles_j), in = id % (8 * tiles_j), bh = min(8, tiles_i - 8 * band);
    const int i0 = (8 * band + in % bh) * BM, j0 = in / bh * BN;

    const int lane = lane_id(), w = threadIdx.x >> 6;
    const int wi = w / WC * (BM / WR), wj = w % WC * (BN / WC);
    lin_f32x16 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const int steps = (g.R + BK - 1) / BK, per = (steps + g.split - 1) / g.split;
    const int s0 = blockIdx.y * per, s1 = min(steps, s0 + per);
    TileA ta;
    TileB tb;
    ta.init(g.a, i0);
    tb.init(g.b, j0);
    const auto fetch = [&](int s, unsigned char* la, unsigned char* lb) {
        ta.fetch(g.a, s * BK, la);
        tb.fetch(g.b, s * BK, lb);
    };
    // fragments one step of 16 depths ahead; the fences keep the scheduler from
    // reading the whole tile ahead, which would spill
    const auto multiply = [&](const unsigned char* la, const unsigned char* lb) {
        sdm_bf16x8 fa[2][MI], fb[2][NJ];
        const auto read = [&](int kk, int z) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) fb[z][j] = TileB::frag(lb, wj + 32 * j, kk);
#pragma unroll
            for (int i = 0; i < MI; ++i) fa[z][i] = TileA::frag(la, wi + 32 * i, kk);
        };
        read(0, 0);
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) {
            if (kk + 1 < BK / 16) read(kk + 1, (kk + 1) & 1);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[kk & 1][i], fb[kk & 1][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (s0 < s1) fetch(s0, sA0, sB0);
    // two buffers by name: the compiler sees which reads a load in flight concerns
    int s = s0;
    for (; s + 1 < s1; s += 2) {
        __syncthreads();
        fetch(s + 1, sA1, sB1);
        multiply(sA0, sB0);
        __syncthreads();
        if (s + 2 < s1) fetch(s + 2, sA0, sB0);
        multiply(sA1, sB1);
    }
    __syncthreads();
    if (s < s1) multiply(sA0, sB0);
    // C: column = lane & 31, rows 8 (e / 4) + 4 (lane >> 5) + e % 4.  32 rows x 64 columns
    // at a time pass through the wave's own 8 KB of LDS, so that a lane ends with eight
    // neighbouring columns of a row (16 bytes of bf16, whole 128-byte lines per row).
    static_assert(NJ == 2, "a wave's tile is 64 columns wide");
    __syncthreads();
    float* sC = reinterpret_cast<float*>(w < NW / 2 ? sA0 + w * 8192 : sA1 + (w - NW / 2) * 8192);
    const bool wide = lin_wide(g);
    const int oj = j0 + wj + 8 * (lane & 7);
    float bias[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) bias[c] = g.bias && g.split == 1 && oj + c < g.J ? g.bias[oj + c] : 0.f;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                sC[(8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * 64 + 32 * j + (lane & 31)] = acc[i][j][e];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 1
        for (int p = 0; p < 4; ++p) {
            const int r = 8 * p + (lane >> 3), oi = i0 + wi + 32 * i + r;
            if (oi >= g.I || oj >= g.J) continue;
            float c[8];
            const v4f u = ld4(sC + r * 64 + 8 * (lane & 7)), v = ld4(sC + r * 64 + 8 * (lane & 7) + 4);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                c[x] = u[x];
                c[4 + x] = v[x];
            }
            if (g.split > 1) {
                float* o = g.part + ((size_t)blockIdx.y * g.I + oi) * g.J + oj;
                if (wide) {
                    st4(o, u);
                    st4(o + 4, v);
                } else {
                    for (int x = 0; x < 8 && oj + x < g.J; ++x) o[x] = c[x];
                }
            } else lin_store8(g, wide, mat_row(g.out, oi), oj, bias, c);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

template <int BM, int BN, int WR, int WC, bool EVEN>
hipError_t launch_tile(const LinGemm& g, hipStream_t st) {
    const int ti = (g.I + BM - 1) / BM, tj = (g.J + BN - 1) / BN;
    const dim3 grid(ti * tj, g.split);
    if (!g.ta && !g.tb) linear_tile_kernel<BM, BN, WR, WC, false, false, EVEN><<<grid, WR * WC * 64, 0, st>>>(g, tj);
    else if (!g.ta) linear_tile_kernel<BM, BN, WR, WC, false, true, EVEN><<<grid, WR * WC * 64, 0, st>>>(g, tj);
    else linear_tile_kernel<BM, BN, WR, WC, true, true, EVEN><<<grid, WR * WC * 64, 0, st>>>(g, tj);
    return hipGetLastError();
}
// whether every 64 depths of a factor follow one another in memory
bool even_depth(const LinMat& m, bool tr, int R) {
    return R % BK == 0 && (tr ? m.T == m.rows || m.T % BK == 0 : m.d == m.cols || m.d % BK == 0);
}

// ---------------------------------------------------------------- dz, dbias
// A workgroup takes 64 columns x `rows` rows: 16 columns-of-four lanes x 16 rows at a time.
constexpr int DZ_ROWS = 256;
template <typename CT>
__global__ __launch_bounds__(256) void linear_dz_kernel(LinMat dy, const void* z, int z_dtype, int act, int ldz,
                                                        CT* dz, float* part) {
    __shared__ float red[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), rg = threadIdx.x >> 6;
    const int m0 = blockIdx.y * DZ_ROWS, m1 = min(dy.rows, m0 + DZ_ROWS);
    float sum = 0.f;
    if (c < ldz) {
        const bool ok = c < dy.cols;
        const int64_t co = ok ? mat_col(dy, c) : 0;
        for (int m = m0 + rg; m < m1; m += 4) {
            float v = 0.f;
            if (ok) {
                const int64_t o = mat_row(dy, m) + co;
                v = ld_any(dy.p, dy.dtype, o);
                if (act) v *= lin_act_slope(ld_any(z, z_dtype, o), act);
                sum += v;
            }
            if (dz) put(dz + (size_t)m * ldz + c, v);
        }
    }
    if (!part) return;
    red[rg][threadIdx.x & 63] = sum;
    __syncthreads();
    if (rg == 0 && c < dy.cols)
        part[(size_t)blockIdx.y * dy.cols + c] =
            red[0][threadIdx.x] + red[1][threadIdx.x] + red[2][threadIdx.x] + red[3][threadIdx.x];
}
__global__ __launch_bounds__(256) void linear_colsum_kernel(const float* part, int parts, int N, float* out) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= N) return;
    float s = 0.f;
    for (int p = 0; p < parts; ++p) s += part[(size_t)p * N + c];
    out[c] = s;
}

__global__ __launch_bounds__(256) void linear_zero_kernel(uint32_t* p, size_t n) {
    for (size_t u = (size_t)blockIdx.x * 256 + threadIdx.x; u < n; u += (size_t)gridDim.x * 256) p[u] = 0u;
}

template <typename CT, typename AT, typename BT>
hipError_t launch_general(const LinGemm& g, hipStream_t st) {
    const dim3 grid((g.I + GT - 1) / GT, (g.J + GT - 1) / GT, g.split);
    if (!g.ta && !g.tb) linear_general_kernel<CT, AT, BT, false, false><<<grid, 256, 0, st>>>(g);
    else if (!g.ta) linear_general_kernel<CT, AT, BT, false, true><<<grid, 256, 0, st>>>(g);
    else linear_general_kernel<CT, AT, BT, true, true><<<grid, 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace

namespace {
// Whether the tiled kernel's 32-bit offsets reach a tile of this factor: rows of `span`
// tokens (and the columns with them) from the start of the first one's sequence.
bool offsets_fit(const LinMat& m, int span) {
    const int64_t seq = m.T == m.rows ? (int64_t)span * m.st + m.cols : (int64_t)(span / m.T + 2) * m.sb;
    return seq * 2 < (int64_t)1 << 31;
}
bool tiled(const LinGemm& g) {
    return g.ctype == SDM_DT_BF16 && g.a.dtype == SDM_DT_BF16 && g.b.dtype == SDM_DT_BF16 &&
           offsets_fit(g.a, 256) && offsets_fit(g.b, 256);
}
}  // namespace

// Tile and split of the depth.  256 x 256 tiles where they fill the device at least
// once, else 128 x 128 ones; the depth is split where even those leave compute units
// free, into parts of 256 depths or more.
LinPlan sdm_linear_plan(int I, int J, int R, int ctype) {
    const int cus = sdm_device_simds() / 4;
    const auto tiles = [&](int64_t t) { return ((I + t - 1) / t) * ((J + t - 1) / t); };
    LinPlan p{};
    p.big = ctype == SDM_DT_BF16 && tiles(256) >= cus;
    const int64_t n = std::max<int64_t>(p.big ? tiles(256) : tiles(128), 1);
    const int64_t want = (2 * cus + n - 1) / n, most = std::max(R / 256, 1);
    p.split = n * 2 > cus ? 1 : (int)std::max<int64_t>(1, std::min(want, most));
    return p;
}

hipError_t sdm_launch_linear(const LinGemm& g, hipStream_t st) {
    hipError_t e;
    if (g.ctype == SDM_DT_F32) e = launch_general<float, float, float>(g, st);
    else if (g.a.dtype == SDM_DT_F32) e = launch_general<bf16_t, float, bf16_t>(g, st);
    else if (g.b.dtype == SDM_DT_F32) e = launch_general<bf16_t, bf16_t, float>(g, st);
    else if (!tiled(g)) e = launch_general<bf16_t, bf16_t, bf16_t>(g, st);
    else {
        const bool even = even_depth(g.a, g.ta, g.R) && even_depth(g.b, g.tb, g.R);
        if (g.big) e = even ? launch_tile<256, 256, 2, 4, true>(g, st) : launch_tile<256, 256, 2, 4, false>(g, st);
        else e = even ? launch_tile<128, 128, 2, 2, true>(g, st) : launch_tile<128, 128, 2, 2, false>(g, st);
    }
    if (e != hipSuccess || g.split <= 1) return e;
    linear_join_kernel<<<dim3((g.J + 255) / 256, std::min((g.I + 7) / 8, 4096)), 256, 0, st>>>(g);
    return hipGetLastError();
}

int sdm_linear_dz_parts(int M) { return (M + DZ_ROWS - 1) / DZ_ROWS; }

hipError_t sdm_launch_linear_dz(const LinMat& dy, const void* z, int z_dtype, int act, int ctype, int ldz, void* dz,
                                float* part, float* dbias, hipStream_t st) {
    const int parts = sdm_linear_dz_parts(dy.rows);
    const dim3 grid((ldz + 63) / 64, parts);
    float* p = dbias ? part : nullptr;
    if (ctype == SDM_DT_F32)
        linear_dz_kernel<float><<<grid, 256, 0, st>>>(dy, z, z_dtype, act, ldz, static_cast<float*>(dz), p);
    else linear_dz_kernel<bf16_t><<<grid, 256, 0, st>>>(dy, z, z_dtype, act, ldz, static_cast<bf16_t*>(dz), p);
    if (dbias) linear_colsum_kernel<<<(dy.cols + 255) / 256, 256, 0, st>>>(part, parts, dy.cols, dbias);
    return hipGetLastError();
}

hipError_t sdm_launch_linear_zero(void* p, size_t words, hipStream_t st) {
    linear_zero_kernel<<<(int)std::min<size_t>((words + 255) / 256, 8192), 256, 0, st>>>(static_cast<uint32_t*>(p), words);
    return hipGetLastError();
}
