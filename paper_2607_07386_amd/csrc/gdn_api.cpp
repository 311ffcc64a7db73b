// C ABI of the dense gated delta rule: host-side validation, workspace sizing
// and launch.  Declarations and contracts: include/sdm.h.
#include <hip/hip_runtime.h>

#include <cstdio>

#include "gdn.h"
#include "sdm.h"
#include "sdm_internal.h"

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

int fail(int status, const char* msg) { return sdm_set_error(status, msg); }
int fail_small(const char* what, size_t have, size_t need) {
    char m[128];
    snprintf(m, sizeof(m), "%s too small: %zu < %zu", what, have, need);
    return sdm_set_error(SDM_ERR_WORKSPACE, m);
}
int hip_fail(hipError_t e, const char* where) {
    char m[256];
    snprintf(m, sizeof(m), "%s: %s", where, hipGetErrorString(e));
    return sdm_set_error(SDM_ERR_HIP, m);
}

bool valid_sizes(int B, int Hk, int H, int T, int d_k, int d_v) {
    return B >= 0 && Hk >= 1 && H >= 1 && H % Hk == 0 && T >= 0 && (int64_t)B * H <= 65535 && d_k >= 4 &&
           d_k % 4 == 0 && d_k <= 256 && d_v >= 4 && d_v % 4 == 0 && d_v <= 4096 && T <= 1 << 30;
}

// Tokens up to which the recurrent form is the faster one, without states to keep for a
// backward: one launch, no workspace, and a pass over the tokens one by one, where the
// chunk form pays for 64 of them.  16 streams of 128 x 128: 17 us at 14 tokens, 18 by
// chunks; 2048 streams: 175, 168; 256 x 256: 22 us at 16 tokens, 31 at 24, 23 by chunks
// (16 streams); 735 us at 24, 950 by chunks (2048 streams).
bool use_step(int T, int d_k, bool training) { return !training && T <= (d_k > 128 ? 20 : 14); }

int check_common(const void* q, const void* k, const void* v, int in_dtype, const float* alpha, const float* beta,
                 const int32_t* lens, int B, int Hk, int H, int T, int d_k, int d_v) {
    if (B < 0 || T < 0 || H < 0 || Hk < 0) return fail(SDM_ERR_INVALID_ARG, "B, Hk, H, T must be >= 0");
    if (Hk < 1 || H < 1 || H % Hk) return fail(SDM_ERR_INVALID_ARG, "H must be a positive multiple of Hk");
    if ((int64_t)B * H > 65535) return fail(SDM_ERR_UNSUPPORTED, "B*H must be <= 65535");
    if (T > 1 << 30) return fail(SDM_ERR_UNSUPPORTED, "T must be <= 2^30");
    if (d_k < 4 || d_k % 4 || d_v < 4 || d_v % 4)
        return fail(SDM_ERR_INVALID_ARG, "d_k and d_v must be positive multiples of 4");
    if (d_k > 256) return fail(SDM_ERR_UNSUPPORTED, "d_k must be <= 256");
    if (d_v > 4096) return fail(SDM_ERR_UNSUPPORTED, "d_v must be <= 4096");
    if (in_dtype != SDM_F32 && in_dtype != SDM_BF16)
        return fail(SDM_ERR_INVALID_ARG, "in_dtype must be SDM_F32 or SDM_BF16");
    if ((int64_t)B * T > 0 && (!q || !k || !v || !alpha || !beta))
        return fail(SDM_ERR_INVALID_ARG, "null input pointer");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(alpha, 4) || !aligned(beta, 4) ||
        !aligned(lens, 4))
        return fail(SDM_ERR_INVALID_ARG, "misaligned pointer (16-byte alignment required)");
    return SDM_OK;
}

int check_buffer(const void* p, size_t have, size_t need, const char* what) {
    if (need == 0) return SDM_OK;
    if (!p || !aligned(p, 256)) {
        char m[128];
        snprintf(m, sizeof(m), "%s must be a 256-byte aligned pointer", what);
        return fail(SDM_ERR_INVALID_ARG, m);
    }
    return have < need ? fail_small(what, have, need) : SDM_OK;
}

GdnArgs make_args(const void* q, const void* k, const void* v, int in_dtype, const float* alpha, const float* beta,
                  const int32_t* lens, int B, int Hk, int H, int T, int d_k, int d_v) {
    GdnArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.in_dtype = in_dtype;
    a.alpha = alpha;
    a.beta = beta;
    a.lens = lens;
    a.B = B;
    a.Hk = Hk;
    a.H = H;
    a.T = T;
    a.dk = d_k;
    a.dv = d_v;
    a.nC = (T + GDN_C - 1) / GDN_C;
    return a;
}

void set_ws(GdnArgs& a, const GdnWs& w, void* workspace) {
    unsigned char* p = static_cast<unsigned char*>(workspace);
    a.vec = reinterpret_cast<float*>(p + w.vec);
    a.tf = reinterpret_cast<uint16_t*>(p + w.tf);
    a.pf = reinterpret_cast<uint16_t*>(p + w.pf);
    a.kt = reinterpret_cast<uint16_t*>(p + w.kt);
    a.qt = reinterpret_cast<uint16_t*>(p + w.qt);
    a.dS = reinterpret_cast<float*>(p + w.dS);
    a.seg_z = reinterpret_cast<float*>(p + w.seg_z);
    a.seg_phi = reinterpret_cast<float*>(p + w.seg_phi);
    a.segs = w.segs;
    a.seg_len = w.seg_len;
}

size_t saved_states(int B, int H, int T, int d_k, int d_v) {
    const size_t nC = ((size_t)T + GDN_C - 1) / GDN_C;
    return align256((size_t)B * H * nC * d_k * d_v * 4);
}

}  // namespace

extern "C" {

size_t sdm_gdn_saved_bytes(int B, int H, int T, int d_k, int d_v) {
    if (!valid_sizes(B, 1, H, T, d_k, d_v)) return 0;
    return saved_states(B, H, T, d_k, d_v) + align256((size_t)B * H * T * d_v * 4);
}

size_t sdm_gdn_fwd_workspace_bytes(int B, int Hk, int H, int T, int d_k, int d_v, int in_dtype, int training) {
    if (!valid_sizes(B, Hk, H, T, d_k, d_v) || use_step(T, d_k, training != 0)) return 0;
    return gdn_ws(B, Hk, H, T, d_k, d_v, in_dtype, false).total;
}

size_t sdm_gdn_bwd_workspace_bytes(int B, int Hk, int H, int T, int d_k, int d_v, int in_dtype) {
    if (!valid_sizes(B, Hk, H, T, d_k, d_v)) return 0;
    return gdn_ws(B, Hk, H, T, d_k, d_v, in_dtype, true).total;
}

int sdm_gdn_fwd(const void* q, const void* k, const void* v, int in_dtype, const float* alpha, const float* beta,
                const int32_t* lens, const float* state0, float* stateT, int B, int Hk, int H, int T, int d_k,
                int d_v, float* y, void* saved, size_t saved_bytes, void* workspace, size_t ws_bytes, void* stream) {
    sdm_set_error(SDM_OK, "");
    int rc = check_common(q, k, v, in_dtype, alpha, beta, lens, B, Hk, H, T, d_k, d_v);
    if (rc != SDM_OK) return rc;
    if (B == 0) return SDM_OK;
    if (!stateT || !aligned(stateT, 16) || !aligned(state0, 16))
        return fail(SDM_ERR_INVALID_ARG, "stateT must be a 16-byte aligned pointer, state0 one or NULL");
    if (T > 0 && (!y || !aligned(y, 16))) return fail(SDM_ERR_INVALID_ARG, "y must be a 16-byte aligned pointer");
    const bool training = saved != nullptr;
    if (training) {
        rc = check_buffer(saved, saved_bytes, sdm_gdn_saved_bytes(B, H, T, d_k, d_v), "saved buffer");
        if (rc != SDM_OK) return rc;
    }
    const size_t need = sdm_gdn_fwd_workspace_bytes(B, Hk, H, T, d_k, d_v, in_dtype, training);
    rc = check_buffer(workspace, ws_bytes, need, "workspace");
    if (rc != SDM_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    GdnArgs a = make_args(q, k, v, in_dtype, alpha, beta, lens, B, Hk, H, T, d_k, d_v);
    a.state0 = state0;
    a.stateT = stateT;
    a.y = y;
    hipError_t e;
    if (use_step(T, d_k, training)) {
        SdmProfScope ps(SDM_K_GDN_STEP, st);
        e = sdm_launch_gdn_step(a, st);
        return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_gdn_fwd launch");
    }
    set_ws(a, gdn_ws(B, Hk, H, T, d_k, d_v, in_dtype, false), workspace);
    if (training) {
        a.saved_S = static_cast<float*>(saved);
        a.saved_X = reinterpret_cast<float*>(static_cast<unsigned char*>(saved) + saved_states(B, H, T, d_k, d_v));
    }
    if (T > 0) {
        SdmProfScope ps(SDM_K_GDN_PREP, st);
        e = sdm_launch_gdn_prep(a, false, st);
        if (e != hipSuccess) return hip_fail(e, "sdm_gdn_fwd launch");
    }
    SdmProfScope ps(SDM_K_GDN_SCAN, st);
    e = sdm_launch_gdn_scan(a, st);
    return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_gdn_fwd launch");
}

int sdm_gdn_bwd(const void* q, const void* k, const void* v, int in_dtype, const float* alpha, const float* beta,
                const int32_t* lens, const void* saved, size_t saved_bytes, const float* dy, const float* dstateT,
                int B, int Hk, int H, int T, int d_k, int d_v, float* dq, float* dk, float* dv, float* dalpha,
                float* dbeta, float* dstate0, void* workspace, size_t ws_bytes, void* stream) {
    sdm_set_error(SDM_OK, "");
    int rc = check_common(q, k, v, in_dtype, alpha, beta, lens, B, Hk, H, T, d_k, d_v);
    if (rc != SDM_OK) return rc;
    if (B == 0) return SDM_OK;
    if (T > 0 && (!dy || !dq || !dk || !dv || !dalpha || !dbeta))
        return fail(SDM_ERR_INVALID_ARG, "null gradient pointer");
    if (!aligned(dy, 16) || !aligned(dstateT, 16) || !aligned(dq, 16) || !aligned(dk, 16) || !aligned(dv, 16) ||
        !aligned(dalpha, 4) || !aligned(dbeta, 4) || !aligned(dstate0, 16))
        return fail(SDM_ERR_INVALID_ARG, "misaligned pointer (16-byte alignment required)");
    rc = check_buffer(saved, saved_bytes, sdm_gdn_saved_bytes(B, H, T, d_k, d_v), "saved buffer");
    if (rc != SDM_OK) return rc;
    const GdnWs w = gdn_ws(B, Hk, H, T, d_k, d_v, in_dtype, true);
    rc = check_buffer(workspace, ws_bytes, w.total, "workspace");
    if (rc != SDM_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    GdnArgs a = make_args(q, k, v, in_dtype, alpha, beta, lens, B, Hk, H, T, d_k, d_v);
    set_ws(a, w, workspace);
    a.saved_S = static_cast<float*>(const_cast<void*>(saved));
    a.saved_X = reinterpret_cast<float*>(static_cast<unsigned char*>(const_cast<void*>(saved)) +
                                         saved_states(B, H, T, d_k, d_v));
    a.dy = dy;
    a.dstateT = dstateT;
    a.dq = dq;
    a.dkk = dk;
    a.dvv = dv;
    a.dalpha = dalpha;
    a.dbeta = dbeta;
    a.dstate0 = dstate0;
    hipError_t e;
    if (T > 0) {
        SdmProfScope ps(SDM_K_GDN_PREP, st);
        e = sdm_launch_gdn_prep(a, true, st);
        if (e != hipSuccess) return hip_fail(e, "sdm_gdn_bwd launch");
    }
    SdmProfScope ps(SDM_K_GDN_BWD, st);
    e = sdm_launch_gdn_adjoint(a, st);
    if (e == hipSuccess && T > 0) e = sdm_launch_gdn_grads(a, st);
    return e == hipSuccess ? SDM_OK : hip_fail(e, "sdm_gdn_bwd launch");
}

}  // extern "C"
