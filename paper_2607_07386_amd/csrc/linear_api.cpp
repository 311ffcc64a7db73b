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
    if ((int64_t)B * T > (1 << 30)) return "B*T must be <= 2^30";
    if (K > (1 << 24) || N > (1 << 22)) return "K must be <= 2^24, N <= 2^22";
    return nullptr;
}

struct BwdWs {
    size_t dz, parts, split, total;
    int ldz;
    LinPlan px, pw;
    bool direct;   // dy is dz as it stands
};
BwdWs bwd_ws(int act, int dy_dtype, int w_dtype, int y_heads, int B, int T, int K, int N) {
    BwdWs w{};
    const int M = B * T, m = w_dtype == SDM_BF16 ? 8 : 4;
    w.ldz = (N + m - 1) / m * m;
    w.direct = act == 0 && dy_dtype == w_dtype && y_heads == 0 && N % m == 0;
    w.px = sdm_linear_plan(M, K, N, w_dtype);
    w.pw = sdm_linear_plan(N, K, M, w_dtype);
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += align256(bytes);
        return at;
    };
    w.dz = take(w.direct ? 0 : (size_t)M * w.ldz * (w_dtype == SDM_BF16 ? 2 : 4));
    w.parts = take((size_t)sdm_linear_dz_parts(M) * N * 4);
    w.split = take(std::max(w.px.split > 1 ? (size_t)w.px.split * M * K * 4 : 0,
                            w.pw.split > 1 ? (size_t)w.pw.split * N * K * 4 : 0));
    w.total = o;
    return w;
}

}  // namespace

extern "C" {

size_t sdm_linear_workspace_bytes(int x_dtype, int w_dtype, int B, int T, int K, int N) {
    if (bad_sizes(x_dtype, 0, w_dtype, 0, B, T, K, N, 0) || too_large(B, T, K, N) || (int64_t)B * T == 0) return 0;
    const int s = sdm_linear_plan(B * T, N, K, w_dtype).split;
    return s > 1 ? align256((size_t)s * B * T * N * 4) : 0;
}

int sdm_linear(const void* x, int x_dtype, int x_heads, const void* w, int w_dtype, const float* bias, int act,
               const void* residual, int B, int T, int K, int N, int y_heads, void* y, int y_dtype, void* z,
               void* workspace, size_t ws_bytes, void* stream) {
    sdm_set_error(SDM_OK, "");
    if (const char* m = bad_sizes(x_dtype, x_heads, w_dtype, act, B, T, K, N, y_heads))
        return fail(SDM_ERR_INVALID_ARG, m);
    if (const char* m = too_large(B, T, K, N)) return fail(SDM_ERR_UNSUPPORTED, m);
    if (!valid_dtype(y_dtype) || (w_dtype == SDM_F32 && y_dtype != SDM_F32))
        return fail(SDM_ERR_INVALID_ARG, "y_dtype must be w's or SDM_F32");
    if (residual && y_heads) return fail(SDM_ERR_INVALID_ARG, "a residual needs a flat y (y_heads 0)");
    if ((int64_t)B * T == 0) return SDM_OK;
    if (!x || !w || !y) return fail(SDM_ERR_INVALID_ARG, "null pointer");
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(y, 16) || !aligned(z, 16) || !aligned(residual, 16) ||
        !aligned(bias, 4))
        return fail(SDM_ERR_INVALID_ARG, "misaligned pointer (16-byte alignment required)");
    const int rc = check_ws(workspace, ws_bytes, sdm_linear_workspace_bytes(x_dtype, w_dtype, B, T, K, N));
    if (rc != SDM_OK) return rc;
    LinGemm g{};
    g.a = lin_tokens(x, x_dtype, B, T, K, x_heads);
    g.b = lin_flat(w, w_dtype, N, K, K);
    g.I = B * T;
    g.J = N;
    g.R = K;
    g.ctype = w_dtype;
    g.out = lin_tokens(y, y_dtype, B, T, N, y_heads);
    g.pre = z;
    g.bias = bias;
    g.residual = residual;
    g.act = act;
    const LinPlan pl = sdm_linear_plan(g.I, g.J, g.R, w_dtype);
    g.split = pl.split;
    g.big = pl.big;
    g.part = static_cast<float*>(workspace);
    SdmProfScope ps(SDM_K_LINEAR, (hipStream_t)stream);
    const hipError_t e = sdm_launch_linear(g, (hipStream_t)stream);
    return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_linear launch");
}

size_t sdm_linear_bwd_workspace_bytes(int x_dtype, int w_dtype, int act, int dy_dtype, int B, int T, int K, int N,
                                      int y_heads) {
    if (bad_sizes(x_dtype, 0, w_dtype, act, B, T, K, N, y_heads) || too_large(B, T, K, N) || (int64_t)B * T == 0)
        return 0;
    return bwd_ws(act, dy_dtype, w_dtype, y_heads, B, T, K, N).total;
}

int sdm_linear_bwd(const void* x, int x_dtype, int x_heads, const void* w, int w_dtype, const void* z, int z_dtype,
                   int act, const void* dy, int dy_dtype, int B, int T, int K, int N, int y_heads, void* dx, void* dw,
                   float* dbias, void* workspace, size_t ws_bytes, void* stream) {
    sdm_set_error(SDM_OK, "");
    if (const char* m = bad_sizes(x_dtype, x_heads, w_dtype, act, B, T, K, N, y_heads))
        return fail(SDM_ERR_INVALID_ARG, m);
    if (const char* m = too_large(B, T, K, N)) return fail(SDM_ERR_UNSUPPORTED, m);
    if (!valid_dtype(dy_dtype) || (act && !valid_dtype(z_dtype)))
        return fail(SDM_ERR_INVALID_ARG, "dtypes must be SDM_F32 or SDM_BF16");
    if (w_dtype == SDM_F32 && (dy_dtype != SDM_F32 || (act && z_dtype != SDM_F32)))
        return fail(SDM_ERR_INVALID_ARG, "an fp32 w needs fp32 z and dy");
    if (act && !z && (int64_t)B * T > 0) return fail(SDM_ERR_INVALID_ARG, "an activation's gradient needs z");
    if (!dx && !dw && !dbias) return SDM_OK;
    const int M = B * T;
    if (M > 0 && (!x || !w || !dy)) return fail(SDM_ERR_INVALID_ARG, "null pointer");
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(z, 16) || !aligned(dy, 16) || !aligned(dx, 16) ||
        !aligned(dw, 16) || !aligned(dbias, 4))
        return fail(SDM_ERR_INVALID_ARG, "misaligned pointer (16-byte alignment required)");
    hipStream_t st = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    if (M == 0) {   // sums over no tokens
        if (dw) e = sdm_launch_linear_zero(dw, (size_t)N * K * (w_dtype == SDM_BF16 ? 2 : 4) / 4, st);
        if (e == hipSuccess && dbias) e = sdm_launch_linear_zero(dbias, N, st);
        return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_linear_bwd launch");
    }
    const BwdWs L = bwd_ws(act, dy_dtype, w_dtype, y_heads, B, T, K, N);
    const int rc = check_ws(workspace, ws_bytes, L.total);
    if (rc != SDM_OK) return rc;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    float* split = reinterpret_cast<float*>(ws + L.split);
    SdmProfScope ps(SDM_K_LINEAR, st);
    if (!L.direct || dbias)
        e = sdm_launch_linear_dz(lin_tokens(dy, dy_dtype, B, T, N, y_heads), z, z_dtype, act, w_dtype, L.ldz,
                                 L.direct ? nullptr : ws + L.dz, reinterpret_cast<float*>(ws + L.parts), dbias, st);
    const LinMat dz = L.direct ? lin_flat(dy, w_dtype, M, N, N) : lin_flat(ws + L.dz, w_dtype, M, N, L.ldz);
    const LinMat xm = lin_tokens(x, x_dtype, B, T, K, x_heads);
    if (e == hipSuccess && dx) {
        LinGemm g{};
        g.a = dz;
        g.b = lin_flat(w, w_dtype, N, K, K);
        g.tb = true;
        g.I = M;
        g.J = K;
        g.R = N;
        g.ctype = w_dtype;
        g.out = lin_tokens(dx, x_dtype, B, T, K, x_heads);
        g.split = L.px.split;
        g.big = L.px.big;
        g.part = split;
        e = sdm_launch_linear(g, st);
    }
    if (e == hipSuccess && dw) {
        LinGemm g{};
        g.a = dz;
        g.b = xm;
        g.ta = g.tb = true;
        g.I = N;
        g.J = K;
        g.R = M;
        g.ctype = w_dtype;
        g.out = lin_flat(dw, w_dtype, N, K, K);
        g.split = L.pw.split;
        g.big = L.pw.big;
        g.part = split;
        e = sdm_launch_linear(g, st);
    }
    return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_linear_bwd launch");
}

}  // extern "C"
