// Projections (gfx950): y = act(x W^T + bias) + residual and its gradients, the
// products on either side of the layer's recurrence (Sec. 3.1: W_q, W_k, W_v, W_a,
// W_b, W_g before it, W_o and the residual stream after it), reading and writing the
// recurrences' head-major layout.
//   forward   C[m, n] = sum_k x[m, k] w[n, k]
//   dx        C[m, k] = sum_n dz[m, n] w[n, k],   dz = dy act'(z)
//   dw        C[n, k] = sum_m dz[m, n] x[m, k],   dbias[n] = sum_m dz[m, n]
//
// All three are one kernel over bf16 tiles (linear_tile_kernel), a factor stored depth
// first being turned on its way from LDS.  fp32 factors are cut into three bf16 parts
// each (gdn.h) and multiplied as six products one after the other in the same
// accumulators, which is faster than the fp32 matrix instruction.  Measured: 8192^3 in
// bf16 0.85 ms, 1.29 PFLOP/s (the library's product 1.66); fp32 4096^3 200 TFLOP/s (the
// library's 151); a layer's projection, 16,384 tokens of 2048 to 2048, 126 us (the library 95),
// with SiLU, head-major, 154 us, 0.89 PFLOP/s.
// There the 32 steps of a tile are few beside its start and its epilogue, and 512
// tiles make two rounds of 256 compute units in which neither overlaps the next.
#include <algorithm>

#include "gdn.h"
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

// us of a step of 64 depths (2048 x 2048 outputs, depth 16384, by the tile): a 256 x 256 tile,
// and two 128 x 128 ones that share a compute unit
constexpr double kStepBig = 2.1, kStepSmall = 1.7;

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
    if (g.rest) st_any(g.rest, g.out.dtype, o, c - (float)(__bf16)c);
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
        const bool flat = g.out.d == g.out.cols;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (j + i < g.J) lin_store(g, ro + (flat ? j + i : mat_col(g.out, j + i)), j + i, c[i]);
        return;
    }
    const int64_t o = ro + mat_col(g.out, j);
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] += b[i];
    if (g.pre) st8(g.pre, g.out.dtype, o, c);
    if (g.rest) {
        float r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = c[i] - (float)(__bf16)c[i];
        st8(g.rest, g.out.dtype, o, r);
    }
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

// The partial sums of a split depth, added in order, through the epilogue: eight
// columns of a row per thread.
__global__ __launch_bounds__(256) void linear_join_kernel(LinGemm g) {
    const int j = (blockIdx.x * 32 + (threadIdx.x & 31)) * 8;
    if (j >= g.J) return;
    const bool wide = lin_wide(g);
    const size_t n = (size_t)g.I * LIN_UP8(g.J);
    float b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = g.bias && j + i < g.J ? g.bias[j + i] : 0.f;
    for (int row = blockIdx.y * 8 + (threadIdx.x >> 5); row < g.I; row += gridDim.y * 8) {
        const float* p = g.part + (size_t)row * LIN_UP8(g.J) + j;
        float c[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < g.split; ++s) {
            const v4f u = ld4(p + s * n), v = ld4(p + s * n + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[i] += u[i];
                c[4 + i] += v[i];
            }
        }
        lin_store8(g, wide, mat_row(g.out, row), j, b, c);
    }
}

// ---------------------------------------------------------------- tiled kernel
// bf16 factors: BM x BN x 64 tiles, WR x WC waves of 32x32x16 matrix instructions.  A wave's
// 128 x 64 outputs take six fragments of LDS for eight instructions, 96 of the 128 bytes a cycle
// that LDS gives; its 64 x 64 in the small tile take four for four, all of them, which bounds
// that tile near half the rate (2048^3: 37 us, 0.47 PFLOP/s).
// The next tile goes straight from memory to LDS while this one is multiplied; a
// factor stored with its output index as the row is [BM][64] there, one stored depth
// first stays [64][BM] and is turned by the transposing LDS reads.  A piece of 16
// bytes stands at its place XOR a function of its row, so that the lanes of a
// read fall on different banks (the pieces of one direct load go to consecutive
// addresses, so the order is chosen by which piece a lane fetches).
typedef float lin_f32x16 __attribute__((ext_vector_type(16)));
typedef short lin_s4 __attribute__((ext_vector_type(4)));
__device__ const uint4 lin_zeros = {0u, 0u, 0u, 0u};   // what pieces outside a matrix read

constexpr int BK = 64;
constexpr uint32_t LIN_OUT = 0x80000000u;   // offset of what lies outside a matrix: loads of it give zeros

__device__ __forceinline__ __amdgpu_buffer_rsrc_t lin_buf(const bf16_t* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p), 0, 0x7fffffff, 0x00020000);
}
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, uint32_t off, void* l) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)l, 16, (int)off, 0, 0, 0);
}

__device__ __forceinline__ void dma16g(const void* g, void* l) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)g,
                                     (__attribute__((address_space(3))) void*)l, 16, 0, 0);
}

// A factor's tile: O output indices x 64 depths.  Each of the NW waves moves O / (8 NW)
// runs of 1 KB.  EVEN: 64 depths always follow one another and a lane's places are
// 32-bit byte offsets from a base that moves along the depth, so that a step costs
// no vector arithmetic.  Otherwise a lane forms its addresses at every step.
template <int O, int NW, bool TR, bool EVEN>
struct LinTile {
    static constexpr int RUNS = O / (8 * NW);
    static constexpr int PPR = (TR ? O : BK) / 8;      // pieces of a row of the tile in LDS
    static constexpr int RPR = 64 / PPR;               // rows of a run
    static constexpr int MASK = PPR / 4 - 1;           // TR: 4 pieces (32 outputs) move together
    const bf16_t* base;      // EVEN, !TR: the first row (one sequence) or the start of its sequence; else the matrix
    uint32_t off[RUNS];      // EVEN: the lane's rows (!TR) or columns (TR)
    const bf16_t* at[RUNS];  // !EVEN, !TR: the lane's rows (NULL past the end)

    __device__ __forceinline__ static int swz(int r) { return TR ? 4 * (r & MASK) : r & 7; }
    __device__ __forceinline__ static int run0() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * RUNS; }
    __device__ __forceinline__ static int row() { return lane_id() / PPR; }
    // the piece of its row that the lane fetches: rows of runs differ by 8 or more (!TR)
    __device__ __forceinline__ static int piece(int r) { return (lane_id() % PPR) ^ swz(r); }

    __device__ __forceinline__ void init(const LinMat& m, int o0) {
        base = static_cast<const bf16_t*>(m.p);
        if constexpr (EVEN && !TR) {
            const int seq = o0 / m.T, first = m.T == m.rows ? o0 : 0;   // 32 bits reach from there, not from the matrix
            base += (int64_t)seq * m.sb + (int64_t)first * m.st;
#pragma unroll
            for (int i = 0; i < RUNS; ++i) {
                const int o = o0 + (run0() + i) * RPR + row();
                off[i] = o < m.rows ? (uint32_t)((int64_t)(o / m.T - seq) * m.sb + (int64_t)(o % m.T - first) * m.st) * 2 : LIN_OUT;
            }
        } else if constexpr (EVEN) {
#pragma unroll
            for (int i = 0; i < RUNS; ++i) {
                const int c = o0 + piece((run0() + i) * RPR + row()) * 8;
                off[i] = c < m.cols ? (uint32_t)mat_col(m, c) * 2 : LIN_OUT;
            }
        } else if constexpr (!TR) {
#pragma unroll
            for (int i = 0; i < RUNS; ++i) {
                const int o = o0 + (run0() + i) * RPR + row();
                at[i] = o < m.rows ? base + mat_row(m, o) : nullptr;
            }
        }
    }
    // the tile at depths r0 .. r0 + 63 of the plane `plane` values into the matrix
    __device__ __forceinline__ void fetch(const LinMat& m, int o0, int r0, int64_t plane, unsigned char* lds) {
        if constexpr (EVEN && !TR) {
            const auto buf = lin_buf(base + plane + mat_col(m, r0));
            const uint32_t pc = piece(row()) * 16;
#pragma unroll
            for (int i = 0; i < RUNS; ++i) dma16(buf, off[i] + pc, lds + (run0() + i) * 1024);
        } else if constexpr (EVEN) {
            const auto buf = lin_buf(base + plane + mat_row(m, r0));
#pragma unroll
            for (int i = 0; i < RUNS; ++i)
                dma16(buf, off[i] + ((run0() + i) * RPR + row()) * (uint32_t)m.st * 2, lds + (run0() + i) * 1024);
        } else if constexpr (!TR) {
            const int c = r0 + piece(row()) * 8;
            const bool ok = c < m.cols;
            const int64_t co = ok ? plane + mat_col(m, c) : 0;
#pragma unroll
            for (int i = 0; i < RUNS; ++i)
                dma16g(at[i] && ok ? (const void*)(at[i] + co) : (const void*)&lin_zeros, lds + (run0() + i) * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < RUNS; ++i) {
                const int kr = (run0() + i) * RPR + row(), r = r0 + kr, c = o0 + piece(kr) * 8;
                dma16g(r < m.rows && c < m.cols ? (const void*)(base + plane + mat_off(m, r, c)) : (const void*)&lin_zeros,
                       lds + (run0() + i) * 1024);
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

    const int depth = (g.R + BK - 1) / BK, steps = depth * g.combos, per = (steps + g.split - 1) / g.split;
    const int s0 = blockIdx.y * per, s1 = min(steps, s0 + per);
    TileA ta;
    TileB tb;
    ta.init(g.a, i0);
    tb.init(g.b, j0);
    const auto fetch = [&](int s, unsigned char* la, unsigned char* lb) {
        const int c = g.combos > 1 ? s / depth : 0, r0 = (g.combos > 1 ? s - c * depth : s) * BK;
        const int pa = (g.part_a >> 2 * c) & 3, pb = (g.part_b >> 2 * c) & 3;
        ta.fetch(g.a, i0, r0, pa * g.plane_a, la);
        tb.fetch(g.b, j0, r0, pb * g.plane_b, lb);
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
                float* o = g.part + ((size_t)blockIdx.y * g.I + oi) * LIN_UP8(g.J) + oj;
                st4(o, u);
                st4(o + 4, v);
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

// Whether every 64 depths of a factor follow one another in memory, up to a multiple of
// 64, and 32-bit offsets reach a tile: its rows from the first one, or from the start of that one's
// sequence where there are several; its depths and the columns of every head.
bool even_depth(const LinMat& m, bool tr, int R) {
    const int up = (R + BK - 1) / BK * BK, span = tr ? BK : 256;
    const bool flat = m.T == m.rows;   // one sequence
    const int64_t heads = m.d == m.cols ? m.cols : m.cols / m.d * m.sh;
    const int64_t reach = tr ? span * m.st + heads : (flat ? span * m.st : (span / m.T + 2) * m.sb) + BK;
    if (reach * 2 >= (int64_t)1 << 31) return false;
    return tr ? m.rows >= up && (flat || m.T % BK == 0) : m.cols >= up && (m.d == m.cols || m.d % BK == 0);
}

// ---------------------------------------------------------------- few rows, few outputs
// Up to 64 rows of x (the decode step) or up to 64 outputs (the gates' pre-activations, one a
// head): bound by reading the other factor once.  A workgroup holds 16 rows of that
// one; its 8 waves take the depth in turns of 64 (a row's 128-byte line in bf16) and their
// sums meet in LDS, so a call is one launch, and fp32 values become bf16 parts on the way.
// 16 rows, 2048 x 2048: 6.7 us (8.4 MB of w, 1.3 TB/s; a launch alone takes 4); 16,384 rows, 16
// outputs: 21 us (3.2 TB/s), fp32 35 us (3.9 TB/s).
// eight depths of a row, from offsets o0 and o1 (the second four, which may be another
// head's); zeros where the depth has ended
__device__ __forceinline__ GdnFrag<3> skinny_frag(const float* row, int64_t o0, int64_t o1, bool ok0, bool ok1) {
    const v4f a = v4sel(ok0, ld4(row + o0), v4zero()), b = v4sel(ok1, ld4(row + o1), v4zero());
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return gdn_split(x);
}
__device__ __forceinline__ GdnFrag<1> skinny_frag(const bf16_t* row, int64_t o0, int64_t, bool ok0, bool) {
    u4v v = *reinterpret_cast<const u4v*>(row + o0);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = ok0 ? v[i] : 0u;
    GdnFrag<1> f;
    f.t[0] = __builtin_bit_cast(sdm_bf16x8, v);
    return f;
}

// BT, ST: types of the factor with many rows and of the one with up to 16 MT; X_FLAT: x is [B, T, K];
// X_MANY: the factor with many rows is x.
template <typename BT, typename ST, int MT, bool X_FLAT, bool X_MANY>
__global__ __launch_bounds__(512) void linear_skinny_kernel(LinGemm g) {
    __shared__ float red[8][MT][256];
    const LinMat &big = X_MANY ? g.a : g.b, &few = X_MANY ? g.b : g.a;
    const int nb = X_MANY ? g.I : g.J, nf = X_MANY ? g.J : g.I;
    const int j0 = blockIdx.x * 16, lane = lane_id(), w = threadIdx.x >> 6, r16 = lane & 15, q = lane >> 4;
    // rows past the end repeat the last one: what they give is not stored
    const BT* bp = static_cast<const BT*>(big.p) + mat_row(big, min(j0 + r16, nb - 1));
    const ST* fp[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) fp[m] = static_cast<const ST*>(few.p) + mat_row(few, min(16 * m + r16, nf - 1));
    sdm_f32x4 acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = sdm_f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = w * 64; k0 < g.R; k0 += 512) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = k0 + 32 * h + 8 * q;
            const bool ok0 = k < g.R, ok1 = k + 4 < g.R;
            const int ka = ok0 ? k : 0, kb = ok1 ? k + 4 : 0;
            const int64_t xa = X_FLAT ? ka : mat_col(g.a, ka), xb = X_FLAT ? kb : mat_col(g.a, kb);
            const auto fb = skinny_frag(bp, X_MANY ? xa : ka, X_MANY ? xb : kb, ok0, ok1);
#pragma unroll
            for (int m = 0; m < MT; ++m)
                acc[m] = gdn_mm(skinny_frag(fp[m], X_MANY ? ka : xa, X_MANY ? kb : xb, ok0, ok1), fb, acc[m]);
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[w][m][(4 * q + r) * 16 + r16] = acc[m][r];
    __syncthreads();
    for (int u = threadIdx.x; u < MT * 256; u += 512) {
        // neighbouring threads store neighbouring outputs
        const int f = X_MANY ? u % (16 * MT) : u >> 4, b = X_MANY ? u / (16 * MT) : u & 15;
        float c = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) c += red[i][f >> 4][(f & 15) * 16 + b];
        const int oi = X_MANY ? j0 + b : f, oj = X_MANY ? f : j0 + b;
        if (oi < g.I && oj < g.J) lin_store(g, mat_off(g.out, oi, oj), oj, c);
    }
}

template <typename WT, typename XT, bool X_FLAT>
hipError_t launch_skinny_rows(const LinGemm& g, hipStream_t st) {
    if (g.I <= LIN_SKINNY) {
        const int grid = (g.J + 15) / 16;
        if (g.I <= 16) linear_skinny_kernel<WT, XT, 1, X_FLAT, false><<<grid, 512, 0, st>>>(g);
        else if (g.I <= 32) linear_skinny_kernel<WT, XT, 2, X_FLAT, false><<<grid, 512, 0, st>>>(g);
        else linear_skinny_kernel<WT, XT, 4, X_FLAT, false><<<grid, 512, 0, st>>>(g);
    } else {
        const int grid = (g.I + 15) / 16;
        if (g.J <= 16) linear_skinny_kernel<XT, WT, 1, X_FLAT, true><<<grid, 512, 0, st>>>(g);
        else if (g.J <= 32) linear_skinny_kernel<XT, WT, 2, X_FLAT, true><<<grid, 512, 0, st>>>(g);
        else linear_skinny_kernel<XT, WT, 4, X_FLAT, true><<<grid, 512, 0, st>>>(g);
    }
    return hipGetLastError();
}
template <typename WT, typename XT>
hipError_t launch_skinny(const LinGemm& g, hipStream_t st) {
    return g.a.d == g.a.cols ? launch_skinny_rows<WT, XT, true>(g, st) : launch_skinny_rows<WT, XT, false>(g, st);
}

// The weights' gradient of an fp32 projection with few outputs: dw[n, k] = sum over tokens of dz[m, n] x[m, k]
// is bound by reading x, so x is read once and cut into parts in registers instead of being laid out
// as parts first.  A workgroup takes 64 columns of x, 16 a wave, and `per` tokens by 128; dz's
// fragments (its parts are there for dx) are gathered once for its four waves.  The call with dz, its join
// included: 16,384 x 2048 by 16 63 us (134 MB of x; 148 by tiles), by 64 94 (153 by tiles); 4096 x
// 1024 by 8 23 (53).
constexpr int DWF = 128;
template <int MT>
__global__ __launch_bounds__(256) void linear_dw_few_kernel(LinMat x, const bf16_t* dz, int64_t plane, int ld, int per, int N,
                                                            float* part) {
    __shared__ __align__(16) uint16_t sA[DWF / 32 * MT * 3 * GDN_FRAG];   // [depth block][tile][part]
    const int lane = lane_id(), w = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
    const int k = blockIdx.x * 64 + 16 * w + r16;
    const float* xp = static_cast<const float*>(x.p) + mat_col(x, min(k, x.cols - 1));   // columns past the end are not stored
    const int m1 = min(x.rows, (int)(blockIdx.y + 1) * per);
    sdm_f32x4 acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = sdm_f32x4{0.f, 0.f, 0.f, 0.f};
    for (int m0 = blockIdx.y * per; m0 < m1; m0 += DWF) {
        float xv[DWF / 32][8];
#pragma unroll
        for (int b = 0; b < DWF / 32; ++b)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int m = m0 + 32 * b + 8 * g + i;
                xv[b][i] = m < m1 ? xp[mat_row(x, m)] : 0.f;
            }
        __syncthreads();   // the tokens before
#pragma unroll
        for (int f = 0; f < DWF / 32 * MT * 3 / 4; ++f) {
            const int id = w + 4 * f, p = id % 3, mt = id / 3 % MT, b = id / 3 / MT;
            lin_us8 v;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int m = m0 + 32 * b + 8 * g + i;
                v[i] = m < m1 ? dz[p * plane + (int64_t)m * ld + 16 * mt + r16].bits : (uint16_t)0;
            }
            *reinterpret_cast<lin_us8*>(sA + id * GDN_FRAG + lane * 8) = v;
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < DWF / 32; ++b) {
            const GdnFrag<3> fx = gdn_split(xv[b]);
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[m] = gdn_mm(gdn_load_frag<3>(sA, b * MT + m), fx, acc[m]);
        }
    }
    if (k >= x.cols) return;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int n = 16 * m + 4 * g + r;
            if (n < N) part[((size_t)blockIdx.y * N + n) * LIN_UP8(x.cols) + k] = acc[m][r];
        }
}

// ---------------------------------------------------------------- parts, dz, dbias
// NP = 1: rounded to bf16; NP = 2: its top 16 bits and what they leave, rounded; NP = 3: the
// three bf16 parts of an fp32 value.
template <int NP>
__device__ __forceinline__ void put_parts(bf16_t* p, int64_t plane, const float (&x)[8]) {
    if constexpr (NP == 1) {
        st8(p, SDM_DT_BF16, 0, x);
    } else if constexpr (NP == 2) {
        float hi[8], lo[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            hi[i] = __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
            lo[i] = x[i] - hi[i];
        }
        st8(p, SDM_DT_BF16, 0, hi);
        st8(p + plane, SDM_DT_BF16, 0, lo);
    } else {
        const GdnFrag<3> f = gdn_split(x);
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<sdm_bf16x8*>(p + i * plane) = f.t[i];
    }
}

// An fp32 matrix as bf16 planes [rows][ld], zeros past its end (both multiples of 64).  16,384 x 2048
// head-major in two parts: 42 us, 268 MB (part of it from the caches).
template <int NP>
__global__ __launch_bounds__(256) void linear_parts_kernel(LinMat m, int rows, int ld, bf16_t* out, int64_t plane) {
    const int c = (blockIdx.x * 32 + (threadIdx.x & 31)) * 8;
    if (c >= ld) return;
    const float* src = static_cast<const float*>(m.p);
    const int64_t o0 = c < m.cols ? mat_col(m, c) : 0, o1 = c + 4 < m.cols ? mat_col(m, c + 4) : 0;
    for (int r = blockIdx.y * 8 + (threadIdx.x >> 5); r < rows; r += gridDim.y * 8) {
        float x[8];
        const int64_t ro = r < m.rows ? mat_row(m, r) : 0;
        const v4f a = r < m.rows && c < m.cols ? ld4(src + ro + o0) : v4zero();
        const v4f b = r < m.rows && c + 4 < m.cols ? ld4(src + ro + o1) : v4zero();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
        put_parts<NP>(out + (int64_t)r * ld + c, plane, x);
    }
}

// dz = dy act'(z) as planes [rows][ld] (zeros past M and N) and its column sums over this
// `per` rows: eight columns a thread, 8 rows at a time.  16,384 x 2048 in bf16 with z and what its
// rounding left: 69 us, 3.9 TB/s.
template <int NP>
__global__ __launch_bounds__(256) void linear_dz_kernel(LinMat dy, const void* z, const void* rest, int z_dtype, int act,
                                                        int rows, int per, int ld, bf16_t* dz, int64_t plane,
                                                        float* part) {
    __shared__ float red[8][256];
    const int cl = threadIdx.x & 31, rg = threadIdx.x >> 5, c = (blockIdx.x * 32 + cl) * 8;
    const bool wide = dy.cols % 8 == 0 && dy.d % 8 == 0;
    int64_t cols[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cols[i] = c + i < dy.cols ? mat_col(dy, c + i) : 0;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < ld) {
        const int m1 = min(rows, (int)(blockIdx.y + 1) * per);
        for (int m = blockIdx.y * per + rg; m < m1; m += 8) {
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (m < dy.rows && c < dy.cols) {
                const int64_t ro = mat_row(dy, m);
                if (wide) {
                    ld8(dy.p, dy.dtype, ro + cols[0], x);
                    if (act) {
                        float zz[8];
                        ld8(z, z_dtype, ro + cols[0], zz);
                        if (rest) {
                            float zr[8];
                            ld8(rest, z_dtype, ro + cols[0], zr);
#pragma unroll
                            for (int i = 0; i < 8; ++i) zz[i] += zr[i];
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] *= act == 1 ? lin_act_slope(zz[i], 1) : lin_act_slope(zz[i], 2);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int64_t o = ro + cols[i];   // a column past the end reads the first one
                        x[i] = ld_any(dy.p, dy.dtype, o);
                        if (act) x[i] *= lin_act_slope(ld_any(z, z_dtype, o) + (rest ? ld_any(rest, z_dtype, o) : 0.f), act);
                        x[i] = c + i < dy.cols ? x[i] : 0.f;
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += x[i];
            }
            if (dz) put_parts<NP>(dz + (int64_t)m * ld + c, plane, x);
        }
    }
    if (!part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) red[rg][cl * 8 + i] = sum[i];
    __syncthreads();
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n < dy.cols) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += red[i][threadIdx.x];
        part[(size_t)blockIdx.y * dy.cols + n] = s;
    }
}
// 32 columns a workgroup, its 32 groups of threads taking the parts in turn
__global__ __launch_bounds__(1024) void linear_colsum_kernel(const float* part, int parts, int N, float* out) {
    __shared__ float red[32][32];
    const int cl = threadIdx.x & 31, rg = threadIdx.x >> 5, c = blockIdx.x * 32 + cl;
    float s = 0.f;
    if (c < N)
        for (int p = rg; p < parts; p += 32) s += part[(size_t)p * N + c];
    red[rg][cl] = s;
    __syncthreads();
    if (rg || c >= N) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += red[i][cl];
    out[c] = s;
}

__global__ __launch_bounds__(256) void linear_zero_kernel(uint32_t* p, size_t n) {
    for (size_t u = (size_t)blockIdx.x * 256 + threadIdx.x; u < n; u += (size_t)gridDim.x * 256) p[u] = 0u;
}

}  // namespace

// Tile and split of the depth (`steps` of 64), by the time they take: a 256 x 256 tile has
// a compute unit to itself, two 128 x 128 ones share it; a split depth is joined by a pass
// over the partial sums.
LinPlan sdm_linear_plan(int I, int J, int steps) {
    const int cus = sdm_device_simds() / 4;
    LinPlan best{};
    double t_best = 1e30;
    for (int big = 0; big < 2; ++big) {
        const int t = big ? 256 : 128;
        const int64_t n = (int64_t)((I + t - 1) / t) * ((J + t - 1) / t);
        for (int split = 1; split <= 64 && (split == 1 || steps / split >= 4); split *= 2) {
            const int64_t slots = (int64_t)cus * (big ? 1 : 2), turns = (n * split + slots - 1) / slots;
            double us = turns * (steps + split - 1) / split * (big ? kStepBig : kStepSmall) + (big ? 6.0 : 4.0);
            if (split > 1) us += 4.0 + (double)I * J * split * 8 / 4e6;
            if (us < t_best) {
                t_best = us;
                best.big = big;
                best.split = split;
            }
        }
    }
    return best;
}

hipError_t sdm_launch_linear(const LinGemm& g, hipStream_t st) {
    const bool even = even_depth(g.a, g.ta, g.R) && even_depth(g.b, g.tb, g.R);
    hipError_t e;
    if (g.big) e = even ? launch_tile<256, 256, 2, 4, true>(g, st) : launch_tile<256, 256, 2, 4, false>(g, st);
    else e = even ? launch_tile<128, 128, 2, 2, true>(g, st) : launch_tile<128, 128, 2, 2, false>(g, st);
    if (e != hipSuccess || g.split <= 1) return e;
    linear_join_kernel<<<dim3((g.J + 255) / 256, std::min((g.I + 7) / 8, 4096)), 256, 0, st>>>(g);
    return hipGetLastError();
}

hipError_t sdm_launch_linear_skinny(const LinGemm& g, hipStream_t st) {
    if (g.b.dtype == SDM_DT_F32) return launch_skinny<float, float>(g, st);
    if (g.a.dtype == SDM_DT_F32) return launch_skinny<bf16_t, float>(g, st);
    return launch_skinny<bf16_t, bf16_t>(g, st);
}

// Parts of the tokens for linear_dw_few_kernel: four workgroups to a compute unit, 256 tokens each or more.
int sdm_linear_dw_few_split(int M, int K) {
    const int64_t want = 4 * (sdm_device_simds() / 4) / ((K + 63) / 64), most = ((int64_t)M + 255) / 256;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(want, most), 64));
}
hipError_t sdm_launch_linear_dw_few(const LinMat& x, const void* dz, int64_t plane, int ld, const LinGemm& g, hipStream_t st) {
    const int per = ((x.rows + g.split - 1) / g.split + DWF - 1) / DWF * DWF;
    const dim3 grid((x.cols + 63) / 64, g.split);
    const bf16_t* d = static_cast<const bf16_t*>(dz);
    if (g.I <= 16) linear_dw_few_kernel<1><<<grid, 256, 0, st>>>(x, d, plane, ld, per, g.I, g.part);
    else if (g.I <= 32) linear_dw_few_kernel<2><<<grid, 256, 0, st>>>(x, d, plane, ld, per, g.I, g.part);
    else linear_dw_few_kernel<4><<<grid, 256, 0, st>>>(x, d, plane, ld, per, g.I, g.part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    linear_join_kernel<<<dim3((g.J + 255) / 256, (g.I + 7) / 8), 256, 0, st>>>(g);
    return hipGetLastError();
}

hipError_t sdm_launch_linear_parts(const LinMat& m, int np, int rows, int ld, void* out, hipStream_t st) {
    const dim3 grid((ld + 255) / 256, std::min((rows + 7) / 8, 2048));
    if (np == 3) linear_parts_kernel<3><<<grid, 256, 0, st>>>(m, rows, ld, static_cast<bf16_t*>(out), (int64_t)rows * ld);
    else linear_parts_kernel<2><<<grid, 256, 0, st>>>(m, rows, ld, static_cast<bf16_t*>(out), (int64_t)rows * ld);
    return hipGetLastError();
}

// Rows of a dz workgroup (a multiple of 8): four workgroups to a compute unit where the matrix is
// large enough, 128 rows at most, or as many as a grid's 65,535 blocks of rows need.
static int dz_rows(int rows, int ld) {
    const int64_t want = 4 * (sdm_device_simds() / 4), cb = (ld + 255) / 256;
    const int64_t least = ((int64_t)rows + 65534) / 65535;
    return (int)std::max<int64_t>((least + 7) / 8 * 8, std::min<int64_t>(128, (int64_t)rows * cb / want / 8 * 8));
}
int sdm_linear_dz_parts(int rows, int ld) { return (rows + dz_rows(rows, ld) - 1) / dz_rows(rows, ld); }

hipError_t sdm_launch_linear_dz(const LinMat& dy, const void* z, const void* rest, int z_dtype, int act, int np,
                                int rows, int ld, void* dz, float* part, float* dbias, hipStream_t st) {
    const int per = dz_rows(rows, ld), parts = sdm_linear_dz_parts(rows, ld);
    const dim3 grid((ld + 255) / 256, parts);
    float* p = dbias ? part : nullptr;
    bf16_t* o = static_cast<bf16_t*>(dz);
    const int64_t plane = (int64_t)rows * ld;
    if (np == 3) linear_dz_kernel<3><<<grid, 256, 0, st>>>(dy, z, rest, z_dtype, act, rows, per, ld, o, plane, p);
    else if (np == 2) linear_dz_kernel<2><<<grid, 256, 0, st>>>(dy, z, rest, z_dtype, act, rows, per, ld, o, plane, p);
    else linear_dz_kernel<1><<<grid, 256, 0, st>>>(dy, z, rest, z_dtype, act, rows, per, ld, o, plane, p);
    if (dbias) linear_colsum_kernel<<<(dy.cols + 31) / 32, 1024, 0, st>>>(part, parts, dy.cols, dbias);
    return hipGetLastError();
}

hipError_t sdm_launch_linear_zero(void* p, size_t words, hipStream_t st) {
    linear_zero_kernel<<<(int)std::min<size_t>((words + 255) / 256, 8192), 256, 0, st>>>(static_cast<uint32_t*>(p), words);
    return hipGetLastError();
}
