// Projections: launch arguments shared by the kernels and the C ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

// A matrix of `rows` x `cols` values in memory, flat [B, T, cols] or head-major
// [B, heads, T, cols / heads]:
//   offset(i, j) = (i / T) sb + (i % T) st + (j / d) sh + j % d.
struct LinMat {
    const void* p;
    int dtype;
    int rows, cols;
    int T, d;
    int64_t sb, st, sh;
};
inline LinMat lin_flat(const void* p, int dtype, int rows, int cols, int64_t ld) {
    return {p, dtype, rows, cols, rows > 0 ? rows : 1, cols > 0 ? cols : 1, 0, ld, 0};
}
inline LinMat lin_tokens(const void* p, int dtype, int B, int T, int cols, int heads) {
    if (heads <= 0) return lin_flat(p, dtype, B * T, cols, cols);
    const int d = cols / heads, t = T > 0 ? T : 1;
    return {p, dtype, B * T, cols, t, d, (int64_t)t * cols, d, (int64_t)t * d};
}

// C[i, j] = sum_r A(i, r) B(j, r).  ta: A is stored with r as its row index and i as
// its column index (tb likewise); otherwise the other way round.
struct LinGemm {
    LinMat a, b;
    bool ta, tb;
    int I, J, R;          // output rows, output columns, depth
    // a factor's fp32 values stand as two or three bf16 parts, `plane` values apart; `combos` products of
    // parts are added up, the c-th of parts (part_a >> 2c) & 3 and (part_b >> 2c) & 3 (lin_products)
    int combos;
    uint32_t part_a, part_b;
    int64_t plane_a, plane_b;
    // out = act(C + bias) + residual, pre = C + bias, rest = what pre's rounding to bf16 left; all laid out
    // and typed as `out`
    LinMat out;
    void* pre;
    void* rest;
    const float* bias;
    const void* residual;
    int act;
    // depth split over `split` workgroups: fp32 partial sums [split][I][LIN_UP8(J)], added up by a second launch
    int split;
    bool big;             // 256 x 256 tiles, else 128 x 128
    float* part;
};

// The products of parts of total order <= `order` of a factor of na parts and one of nb, smallest first.
inline void lin_products(LinGemm& g, int na, int nb, int order) {
    g.combos = 0;
    g.part_a = g.part_b = 0;
    for (int o = order; o >= 0; --o)
        for (int i = 0; i < na; ++i) {
            const int j = o - i;
            if (j < 0 || j >= nb) continue;
            g.part_a |= (uint32_t)i << 2 * g.combos;
            g.part_b |= (uint32_t)j << 2 * g.combos;
            ++g.combos;
        }
}

#define LIN_UP8(x) (((x) + 7) / 8 * 8)
struct LinPlan {
    bool big;
    int split;
};
LinPlan sdm_linear_plan(int I, int J, int steps);
// bf16 factors (or planes of parts) of any sizes
hipError_t sdm_launch_linear(const LinGemm& g, hipStream_t st);
// a or b with up to LIN_SKINNY rows, b [J, R], factors of any types; one launch
// The outputs go up to it for an fp32 x, which is read once instead of being laid out as parts
// first (16,384 x 2048 by 64: 82 us, 141 by tiles), and to half of it for a bf16 one (32 outputs:
// 27 us, 26 by tiles; 64: 42, 29).
#define LIN_SKINNY 64
inline bool lin_skinny(int I, int J, bool x_f32) { return I <= LIN_SKINNY || J <= (x_f32 ? LIN_SKINNY : LIN_SKINNY / 2); }
hipError_t sdm_launch_linear_skinny(const LinGemm& g, hipStream_t st);
// an fp32 matrix as np bf16 planes [rows][ld] (2: to 2^-15 of a value, 3: to 2^-24), zeros past its end
hipError_t sdm_launch_linear_parts(const LinMat& m, int np, int rows, int ld, void* out, hipStream_t st);
// dz = dy act'(z) as np planes [rows][ld] (1: rounded), zeros past M and N, and dbias = its column sums
// (through parts [sdm_linear_dz_parts(rows, ld)][N] added in order).  dz and rest may be NULL.
int sdm_linear_dz_parts(int rows, int ld);
hipError_t sdm_launch_linear_dz(const LinMat& dy, const void* z, const void* rest, int z_dtype, int act, int np, int rows, int ld,
                                void* dz, float* part, float* dbias, hipStream_t st);
// dw = dz^T x of an fp32 x with g.I <= LIN_SKINNY outputs, from dz's three planes [..][ld], ld a multiple of 64;
// g: I, J, out, part of g.split = sdm_linear_dw_few_split(M, K)
int sdm_linear_dw_few_split(int M, int K);
hipError_t sdm_launch_linear_dw_few(const LinMat& x, const void* dz, int64_t plane, int ld, const LinGemm& g, hipStream_t st);
hipError_t sdm_launch_linear_zero(void* p, size_t words, hipStream_t st);
