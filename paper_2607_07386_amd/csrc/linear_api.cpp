// C ABI of the projections: host-side validation, workspace sizing and launch.
// Declarations and contracts: include/sdm.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>

#include "linear.h"
#include "sdm.h"
#include "sdm_internal.h"

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
int fail(int status, const char* msg) { return sdm_set_error(status, msg); }
int hip_fail(hipError_t e, const char* where) {
    char m[256];
    snprintf(m, sizeof(m), "%s: %s", where, hipGetErrorString(e));
    return sdm_set_error(SDM_ERR_HIP, m);
}
int check_ws(const void* p, size_t have, size_t need) {
    if (need == 0) return SDM_OK;
    if (!p || !aligned(p, 256)) return fail(SDM_ERR_INVALID_ARG, "workspace must be a 256-byte aligned pointer");
    if (have < need) {
        char m[128];
        snprintf(m, sizeof(m), "workspace too small: %zu < %zu", have, need);
        return fail(SDM_ERR_WORKSPACE, m);
    }
    return SDM_OK;
}
bool valid_dtype(int d) { return d == SDM_F32 || d == SDM_BF16; }

// Sizes, types and head counts shared by the calls.
const char* bad_sizes(int x_dtype, int x_heads, int w_dtype, int act, int B, int T, int K, int N, int y_heads) {
    if (B < 0 || T < 0 || K < 1 || N < 1) return "B, T must be >= 0 and K, N >= 1";
    if (!valid_dtype(x_dtype) || !valid_dtype(w_dtype)) return "dtypes must be SDM_F32 or SDM_BF16";
    if (x_dtype == SDM_BF16 && w_dtype == SDM_F32) return "a bf16 x needs a bf16 w";
    if (act < 0 || act > 2) return "act must be 0 (identity), 1 (SiLU) or 2 (GELU)";
    if (x_heads < 0 || y_heads < 0 || (x_heads && K % x_heads) || (y_heads && N % y_heads))
        return "head counts must divide K and N";
    const int m = w_dtype == SDM_BF16 ? 8 : 4;
    if ((x_heads ? K / x_heads : K) % m || K % m) return "K, and K / x_heads, must be multiples of 16 bytes of w";
    return nullptr;
}
const char* too_large(int B, int T, int K, int N) {
    // 16 rows a workgroup of 512 threads, and a launch holds fewer than 2^32 threads
    if ((int64_t)B * T > (1 << 26)) return "B*T must be <= 2^26";
    if (K > (1 << 24) || N > (1 << 22)) return "K must be <= 2^24, N <= 2^22";
    return nullptr;
}

int up64(int x) { return (x + 63) / 64 * 64; }
int parts_of(int dtype) { return dtype == SDM_F32 ? 3 : 1; }
// Parts of x in the forward.  Two keep 2^-15 of an fp32 x, a 128th of what the rounding of a bf16
// result takes off; an fp32 result gets all three, and so does any with an fp32 w.  16,384 x 2048 head-major by
// 2048 with a residual: 305 to 313 us, 192 where the caller rounds x, that pass included; an fp32 result 418.
int x_parts(int x_dtype, int w_dtype, int y_dtype) {
    return x_dtype == SDM_BF16 ? 1 : w_dtype == SDM_F32 || y_dtype == SDM_F32 ? 3 : 2;
}
// Parts of dz in the backward: all three for fp32 gradients (of an fp32 x, an fp32 w), two for an fp32 dy where the
// gradients are bf16.  From a bf16 dy an activation's dz is rounded to bf16, as a program that holds its
// activations' gradients in bf16 has it: two parts double both products (16,384 x 2048 x 2048 with dbias:
// 353 us, 596 from an fp32 dy) for dx and dw that are rounded to 2^-8 themselves; without an activation it is exact.
int dz_parts(int x_dtype, int w_dtype, int act, int dy_dtype) {
    if (w_dtype == SDM_F32) return 3;
    if (act == 0 && dy_dtype == SDM_BF16) return 1;
    return x_dtype == SDM_F32 ? 3 : dy_dtype == SDM_F32 ? 2 : 1;
}
// the products of dw = dz^T x: to order 2 for an fp32 dw, to order 1 for a bf16 one
void dw_products(LinGemm& g, int x_dtype, int w_dtype, int nz) {
    lin_products(g, nz, w_dtype == SDM_F32 ? 3 : x_dtype == SDM_F32 ? 2 : 1, w_dtype == SDM_F32 ? 2 : 1);
}
int steps_of(int R, int combos) { return (R + 63) / 64 * combos; }

// Offsets into a call's workspace.  fp32 factors enter the products as bf16 planes,
// padded to multiples of 64 both ways.
struct Ws {
    size_t x = 0, w = 0, dz = 0, parts = 0, split = 0, total = 0;
    LinPlan py{}, px{}, pw{};
    bool direct = false;   // dy is dz as it stands
    bool few = false;      // dw reads x as it stands
    size_t take(size_t bytes) {
        const size_t at = total;
        total += align256(bytes);
        return at;
    }
};
size_t planes(int np, int rows, int cols) { return (size_t)np * up64(rows) * up64(cols) * 2; }
size_t split_bytes(const LinPlan& p, int I, int J) { return p.split > 1 ? (size_t)p.split * I * LIN_UP8(J) * 4 : 0; }

Ws fwd_ws(int x_dtype, int w_dtype, int y_dtype, int M, int K, int N) {
    Ws s;
    if (lin_skinny(M, N, x_dtype == SDM_F32)) return s;
    const int np = x_parts(x_dtype, w_dtype, y_dtype);
    if (x_dtype == SDM_F32) s.x = s.take(planes(np, M, K));
    if (w_dtype == SDM_F32) s.w = s.take(planes(3, N, K));
    s.py = sdm_linear_plan(M, N, steps_of(K, w_dtype == SDM_F32 ? 6 : np));
    s.split = s.take(split_bytes(s.py, M, N));
    return s;
}
Ws bwd_ws(int x_dtype, int w_dtype, int act, int dy_dtype, int y_heads, int M, int K, int N) {
    Ws s;
    const int nz = dz_parts(x_dtype, w_dtype, act, dy_dtype);
    s.direct = w_dtype == SDM_BF16 && act == 0 && dy_dtype == SDM_BF16 && y_heads == 0 && N % 8 == 0;
    if (!s.direct) s.dz = s.take(planes(nz, M, N));
    s.few = w_dtype == SDM_F32 && N <= LIN_SKINNY;
    if (x_dtype == SDM_F32 && !s.few) s.x = s.take(planes(w_dtype == SDM_F32 ? 3 : 2, M, K));
    if (w_dtype == SDM_F32) s.w = s.take(planes(3, N, K));
    s.parts = s.take((size_t)sdm_linear_dz_parts(up64(M), up64(N)) * N * 4);
    LinGemm g{};
    lin_products(g, nz, parts_of(w_dtype), 2);
    s.px = sdm_linear_plan(M, K, steps_of(N, g.combos));
    dw_products(g, x_dtype, w_dtype, nz);
    s.pw = sdm_linear_plan(N, K, steps_of(M, g.combos));
    if (s.few) s.pw.split = sdm_linear_dw_few_split(M, K);
    const size_t dw_bytes = s.few ? (size_t)s.pw.split * N * LIN_UP8(K) * 4 : split_bytes(s.pw, N, K);
    s.split = s.take(std::max(split_bytes(s.px, M, K), dw_bytes));
    return s;
}
// planes of a rows x cols matrix: as rows of a factor (depth = columns), or depth first
LinMat plane_mat(const void* p, int rows, int cols, bool depth_rows) {
    LinMat m = lin_flat(p, SDM_BF16, depth_rows ? up64(rows) : rows, depth_rows ? cols : up64(cols), up64(cols));
    return m;
}
int64_t plane_len(int rows, int cols) { return (int64_t)up64(rows) * up64(cols); }

}  // namespace

extern "C" {

size_t sdm_linear_workspace_bytes(int x_dtype, int w_dtype, int B, int T, int K, int N) {
    if (bad_sizes(x_dtype, 0, w_dtype, 0, B, T, K, N, 0) || too_large(B, T, K, N) || (int64_t)B * T == 0) return 0;
    // for either type of y: a depth of more parts may be split otherwise
    return std::max(fwd_ws(x_dtype, w_dtype, SDM_F32, B * T, K, N).total,
                    fwd_ws(x_dtype, w_dtype, w_dtype, B * T, K, N).total);
}

int sdm_linear(const void* x, int x_dtype, int x_heads, const void* w, int w_dtype, const float* bias, int act,
               const void* residual, int B, int T, int K, int N, int y_heads, void* y, int y_dtype, void* z,
               void* z_rest, void* workspace, size_t ws_bytes, void* stream) {
    sdm_set_error(SDM_OK, "");
    if (const char* m = bad_sizes(x_dtype, x_heads, w_dtype, act, B, T, K, N, y_heads))
        return fail(SDM_ERR_INVALID_ARG, m);
    if (const char* m = too_large(B, T, K, N)) return fail(SDM_ERR_UNSUPPORTED, m);
    if (!valid_dtype(y_dtype) || (w_dtype == SDM_F32 && y_dtype != SDM_F32))
        return fail(SDM_ERR_INVALID_ARG, "y_dtype must be w's or SDM_F32");
    if (z_rest && (!z || y_dtype != SDM_BF16)) return fail(SDM_ERR_INVALID_ARG, "z_rest goes with a bf16 z");
    if (residual && y_heads) return fail(SDM_ERR_INVALID_ARG, "a residual needs a flat y (y_heads 0)");
    if ((int64_t)B * T == 0) return SDM_OK;
    if (!x || !w || !y) return fail(SDM_ERR_INVALID_ARG, "null pointer");
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(y, 16) || !aligned(z, 16) || !aligned(z_rest, 16) ||
        !aligned(residual, 16) ||
        !aligned(bias, 4))
        return fail(SDM_ERR_INVALID_ARG, "misaligned pointer (16-byte alignment required)");
    const int rc = check_ws(workspace, ws_bytes, sdm_linear_workspace_bytes(x_dtype, w_dtype, B, T, K, N));
    if (rc != SDM_OK) return rc;
    const int M = B * T;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    hipStream_t st = (hipStream_t)stream;
    LinGemm g{};
    g.a = lin_tokens(x, x_dtype, B, T, K, x_heads);
    g.b = lin_flat(w, w_dtype, N, K, K);
    g.I = M;
    g.J = N;
    g.R = K;
    lin_products(g, x_parts(x_dtype, w_dtype, y_dtype), parts_of(w_dtype), 2);
    g.out = lin_tokens(y, y_dtype, B, T, N, y_heads);
    g.pre = z;
    g.rest = z_rest;
    g.bias = bias;
    g.residual = residual;
    g.act = act;
    g.split = 1;
    SdmProfScope ps(SDM_K_LINEAR, st);
    hipError_t e = hipSuccess;
    if (lin_skinny(M, N, x_dtype == SDM_F32)) {
        e = sdm_launch_linear_skinny(g, st);
        return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_linear launch");
    }
    const Ws L = fwd_ws(x_dtype, w_dtype, y_dtype, M, K, N);
    if (x_dtype == SDM_F32) {
        e = sdm_launch_linear_parts(g.a, x_parts(x_dtype, w_dtype, y_dtype), up64(M), up64(K), ws + L.x, st);
        g.a = plane_mat(ws + L.x, M, K, false);
        g.plane_a = plane_len(M, K);
    }
    if (e == hipSuccess && w_dtype == SDM_F32) {
        e = sdm_launch_linear_parts(g.b, 3, up64(N), up64(K), ws + L.w, st);
        g.b = plane_mat(ws + L.w, N, K, false);
        g.plane_b = plane_len(N, K);
    }
    g.split = L.py.split;
    g.big = L.py.big;
    g.part = reinterpret_cast<float*>(ws + L.split);
    if (e == hipSuccess) e = sdm_launch_linear(g, st);
    return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_linear launch");
}

size_t sdm_linear_bwd_workspace_bytes(int x_dtype, int w_dtype, int act, int dy_dtype, int B, int T, int K, int N,
                                      int y_heads) {
    if (bad_sizes(x_dtype, 0, w_dtype, act, B, T, K, N, y_heads) || too_large(B, T, K, N) || (int64_t)B * T == 0)
        return 0;
    return bwd_ws(x_dtype, w_dtype, act, dy_dtype, y_heads, B * T, K, N).total;
}

int sdm_linear_bwd(const void* x, int x_dtype, int x_heads, const void* w, int w_dtype, const void* z,
                   const void* z_rest, int z_dtype, int act, const void* dy, int dy_dtype, int B, int T, int K, int N, int y_heads, void* dx, void* dw,
                   float* dbias, void* workspace, size_t ws_bytes, void* stream) {
    sdm_set_error(SDM_OK, "");
    if (const char* m = bad_sizes(x_dtype, x_heads, w_dtype, act, B, T, K, N, y_heads))
        return fail(SDM_ERR_INVALID_ARG, m);
    if (const char* m = too_large(B, T, K, N)) return fail(SDM_ERR_UNSUPPORTED, m);
    if (!valid_dtype(dy_dtype) || (act && !valid_dtype(z_dtype)))
        return fail(SDM_ERR_INVALID_ARG, "dtypes must be SDM_F32 or SDM_BF16");
    if (w_dtype == SDM_F32 && (dy_dtype != SDM_F32 || (act && z_dtype != SDM_F32)))
        return fail(SDM_ERR_INVALID_ARG, "an fp32 w needs fp32 z and dy");
    if (act && z_rest && z_dtype != SDM_BF16) return fail(SDM_ERR_INVALID_ARG, "z_rest goes with a bf16 z");
    if (act && !z && (int64_t)B * T > 0) return fail(SDM_ERR_INVALID_ARG, "an activation's gradient needs z");
    if (!dx && !dw && !dbias) return SDM_OK;
    const int M = B * T;
    if (M > 0 && (!x || !w || !dy)) return fail(SDM_ERR_INVALID_ARG, "null pointer");
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(z, 16) || !aligned(z_rest, 16) || !aligned(dy, 16) || !aligned(dx, 16) ||
        !aligned(dw, 16) || !aligned(dbias, 4))
        return fail(SDM_ERR_INVALID_ARG, "misaligned pointer (16-byte alignment required)");
    hipStream_t st = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    if (M == 0) {   // sums over no tokens
        if (dw) e = sdm_launch_linear_zero(dw, (size_t)N * K * (w_dtype == SDM_BF16 ? 2 : 4) / 4, st);
        if (e == hipSuccess && dbias) e = sdm_launch_linear_zero(dbias, N, st);
        return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_linear_bwd launch");
    }
    const Ws L = bwd_ws(x_dtype, w_dtype, act, dy_dtype, y_heads, M, K, N);
    const int rc = check_ws(workspace, ws_bytes, L.total);
    if (rc != SDM_OK) return rc;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const int nz = dz_parts(x_dtype, w_dtype, act, dy_dtype);
    SdmProfScope ps(SDM_K_LINEAR, st);
    if (!L.direct || dbias)
        e = sdm_launch_linear_dz(lin_tokens(dy, dy_dtype, B, T, N, y_heads), z, z_rest, z_dtype, act, nz, up64(M), up64(N),
                                 L.direct || !(dx || dw) ? nullptr : ws + L.dz, reinterpret_cast<float*>(ws + L.parts), dbias, st);
    LinGemm g{};
    lin_products(g, nz, parts_of(w_dtype), 2);
    g.tb = true;
    g.part = reinterpret_cast<float*>(ws + L.split);
    g.plane_a = plane_len(M, N);
    if (e == hipSuccess && dx) {
        g.a = L.direct ? lin_flat(dy, SDM_BF16, M, N, N) : plane_mat(ws + L.dz, M, N, false);
        g.b = lin_flat(w, w_dtype, N, K, K);
        if (w_dtype == SDM_F32) {
            e = sdm_launch_linear_parts(g.b, 3, up64(N), up64(K), ws + L.w, st);
            g.b = plane_mat(ws + L.w, N, K, true);
            g.plane_b = plane_len(N, K);
        }
        g.I = M;
        g.J = K;
        g.R = N;
        g.out = lin_tokens(dx, x_dtype, B, T, K, x_heads);
        g.split = L.px.split;
        g.big = L.px.big;
        if (e == hipSuccess) e = sdm_launch_linear(g, st);
    }
    if (e == hipSuccess && dw) {
        g.a = L.direct ? lin_flat(dy, SDM_BF16, M, N, N) : plane_mat(ws + L.dz, M, N, true);
        g.ta = true;
        dw_products(g, x_dtype, w_dtype, nz);
        g.b = lin_tokens(x, x_dtype, B, T, K, x_heads);
        if (x_dtype == SDM_F32 && !L.few) {
            e = sdm_launch_linear_parts(g.b, w_dtype == SDM_F32 ? 3 : 2, up64(M), up64(K), ws + L.x, st);
            g.b = plane_mat(ws + L.x, M, K, true);
            g.plane_b = plane_len(M, K);
        }
        g.I = N;
        g.J = K;
        g.R = M;
        g.out = lin_flat(dw, w_dtype, N, K, K);
        g.split = L.pw.split;
        g.big = L.pw.big;
        if (e == hipSuccess && L.few) e = sdm_launch_linear_dw_few(g.b, ws + L.dz, plane_len(M, N), up64(N), g, st);
        else if (e == hipSuccess) e = sdm_launch_linear(g, st);
    }
    return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_linear_bwd launch");
}

}  // extern "C"
