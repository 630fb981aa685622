// extern "C" entry points of include/qtip.h for 8-bit layers and what stands around a layer: argument validation and
// dispatch to the kernel launchers.  Nothing here touches the data.
#include "../../include/qtip.h"
#include "qtip_internal.h"

namespace {

using qtip::aligned, qtip::fail, qtip::hip_fail;

static_assert(QTIP_F16 == qtip::TYPE_F16 && QTIP_BF16 == qtip::TYPE_BF16 && QTIP_F32 == qtip::TYPE_F32 &&
              QTIP_I8 == qtip::TYPE_I8 && QTIP_ROWS_MAX_N == qtip::ROWS_MAX_N &&
              QTIP_MOE_MAX_TOKENS == qtip::MOE_MAX_TOKENS && QTIP_MOE_MAX_EXPERTS == qtip::MOE_MAX_EXPERTS &&
              QTIP_MOE_MAX_TOP_K == qtip::MOE_MAX_TOP_K, "the header's values");

bool is_float_type(int type) { return type == QTIP_F16 || type == QTIP_BF16 || type == QTIP_F32; }
int bytes_of(int type) { return type == QTIP_F32 ? 4 : type == QTIP_I8 ? 1 : 2; }

int check_rows(const char *fn, int rows, int n, const int8_t *signs, int block) {
    if (rows < 1 || n < 1) return fail(QTIP_EINVAL, "%s: rows = %d and n = %d must be positive", fn, rows, n);
    if (n > QTIP_ROWS_MAX_N) return fail(QTIP_EINVAL, "%s: n = %d is above QTIP_ROWS_MAX_N = %d", fn, n, QTIP_ROWS_MAX_N);
    if (!signs) return QTIP_OK;
    if (block < 16 || block > 16384 || (block & (block - 1)))
        return fail(QTIP_EINVAL, "%s: block = %d must be a power of two in [16, 16384]", fn, block);
    if (n % block) return fail(QTIP_EINVAL, "%s: n = %d is not a multiple of block %d", fn, n, block);
    if (!aligned(signs, 4)) return fail(QTIP_EINVAL, "%s: signs must be 4-byte aligned", fn);
    return QTIP_OK;
}

// Rows of `ld` values of `type` each, of which n are used.
int check_matrix(const char *fn, const char *name, const void *p, int64_t ld, int n, int type) {
    if (ld < n) return fail(QTIP_EINVAL, "%s: rows of %s are %lld values apart, less than %d", fn, name, (long long)ld, n);
    if (!aligned(p, bytes_of(type))) return fail(QTIP_EINVAL, "%s: %s must be %d-byte aligned", fn, name, bytes_of(type));
    return QTIP_OK;
}

}  // namespace

extern "C" {

int qtip_quantize_rows_i8(const void *x, const void *up, int type, int rows, int n, int64_t ldx, const int8_t *signs, int block,
                          int8_t *q, int64_t ldq, float *scale, void *stream) {
    const char *fn = "qtip_quantize_rows_i8";
    if (!x || !q || !scale) return fail(QTIP_EINVAL, "%s: NULL pointer", fn);
    if (!is_float_type(type)) return fail(QTIP_EUNSUPPORTED, "%s: type %d is not F16, BF16 or F32", fn, type);
    if (int rc = check_rows(fn, rows, n, signs, block)) return rc;
    if (int rc = check_matrix(fn, "x", x, ldx, n, type)) return rc;
    if (int rc = check_matrix(fn, "up", up, ldx, n, type)) return rc;
    if (int rc = check_matrix(fn, "q", q, ldq, n, QTIP_I8)) return rc;
    if (!aligned(scale, 4)) return fail(QTIP_EINVAL, "%s: scale must be 4-byte aligned", fn);
    hipError_t e = qtip::launch_quantize_rows_i8(x, up, type, rows, n, ldx, signs, block, q, ldq, scale, (hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(fn, e);
    return QTIP_OK;
}

size_t qtip_matmul_i8_workspace(int m, int n, int B) {
    if (m < 1 || m > QTIP_I8_MAX_M || n < 1 || n > QTIP_I8_MAX_N || B < 1 || B > QTIP_I8_MAX_B) return 0;
    return qtip::matmul_i8_workspace(m, n, B);
}

int qtip_matmul_i8(const int8_t *W, int64_t ldw, const float *w_scale, int m, int n, const int8_t *X, int64_t ldx,
                   const float *x_scale, int B, const float *bias, void *Y, int64_t ldy, int y_type, void *workspace,
                   size_t workspace_bytes, void *stream) {
    const char *fn = "qtip_matmul_i8";
    if (!W || !w_scale || !X || !x_scale || !Y) return fail(QTIP_EINVAL, "%s: NULL pointer", fn);
    if (!is_float_type(y_type)) return fail(QTIP_EUNSUPPORTED, "%s: type %d is not F16, BF16 or F32", fn, y_type);
    if (m < 1 || n < 1) return fail(QTIP_EINVAL, "%s: m = %d and n = %d must be positive", fn, m, n);
    if (n > QTIP_I8_MAX_N) return fail(QTIP_EINVAL, "%s: n = %d is above QTIP_I8_MAX_N = %d", fn, n, QTIP_I8_MAX_N);
    if (m > QTIP_I8_MAX_M) return fail(QTIP_EINVAL, "%s: m = %d is above QTIP_I8_MAX_M = %d", fn, m, QTIP_I8_MAX_M);
    if (B < 1 || B > QTIP_I8_MAX_B) return fail(QTIP_EINVAL, "%s: B = %d out of range", fn, B);
    if (int rc = check_matrix(fn, "W", W, ldw, n, QTIP_I8)) return rc;
    if (int rc = check_matrix(fn, "X", X, ldx, n, QTIP_I8)) return rc;
    if (int rc = check_matrix(fn, "Y", Y, ldy, m, y_type)) return rc;
    if (ldw % 16 || ldx % 16 || !aligned(W, 16) || !aligned(X, 16))
        return fail(QTIP_EINVAL, "%s: rows of W and X must begin at multiples of 16 bytes", fn);
    if (ldw > QTIP_I8_MAX_LD || ldx > QTIP_I8_MAX_LD)
        return fail(QTIP_EINVAL, "%s: rows of W or X are more than QTIP_I8_MAX_LD = %d values apart", fn, QTIP_I8_MAX_LD);
    if (!aligned(w_scale, 4) || !aligned(x_scale, 4) || !aligned(bias, 4))
        return fail(QTIP_EINVAL, "%s: scales and bias must be 4-byte aligned", fn);
    const size_t need = qtip::matmul_i8_workspace(m, n, B);
    if (need && (!workspace || !aligned(workspace, 256)))
        return fail(QTIP_EINVAL, "%s: a workspace of %zu bytes, 256-byte aligned, is needed", fn, need);
    if (workspace_bytes < need) return fail(QTIP_EINVAL, "%s: workspace of %zu bytes, %zu needed", fn, workspace_bytes, need);
    hipError_t e = qtip::launch_matmul_i8({W, X, w_scale, x_scale, bias, Y, ldw, ldx, ldy, m, n, B, y_type}, workspace,
                                          (hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(fn, e);
    return QTIP_OK;
}

int qtip_norm_residual(const void *y, int64_t ldy, int y_type, const void *h, int64_t ldh, int h_type, const void *gate,
                       int64_t ldgate, int rows, int n, int norm, const float *post_weight, const float *post_bias,
                       const float *pre_weight, const float *pre_bias, float eps, float res_scale, const int8_t *signs,
                       int block, void *h_out, void *x, int64_t ldx, int x_type, float *x_scale, void *stream) {
    const char *fn = "qtip_norm_residual";
    if (!y && !h) return fail(QTIP_EINVAL, "%s: neither y nor h", fn);
    if (!h_out && !x) return fail(QTIP_EINVAL, "%s: neither h_out nor x: nothing to store", fn);
    if (norm != QTIP_NORM_RMS && norm != QTIP_NORM_LAYER) return fail(QTIP_EUNSUPPORTED, "%s: unknown norm %d", fn, norm);
    if (!is_float_type(y_type) || (h_type != y_type && h_type != QTIP_F32))
        return fail(QTIP_EUNSUPPORTED, "%s: y of type %d and h of type %d (y: F16, BF16 or F32, h: the same or F32)", fn,
                    y_type, h_type);
    if (int rc = check_rows(fn, rows, n, signs, block)) return rc;
    if ((gate || post_weight) && !y) return fail(QTIP_EINVAL, "%s: a gate or a norm behind the block without y", fn);
    if ((post_bias && !post_weight) || (pre_bias && !pre_weight)) return fail(QTIP_EINVAL, "%s: a bias without a weight", fn);
    if (y)
        if (int rc = check_matrix(fn, "y", y, ldy, n, y_type)) return rc;
    if (h || h_out) {
        if (int rc = check_matrix(fn, "h", h, ldh, n, h_type)) return rc;
        if (int rc = check_matrix(fn, "h_out", h_out, ldh, n, h_type)) return rc;
    }
    if (gate)  // (0: one row for all)
        if (int rc = check_matrix(fn, "gate", gate, ldgate == 0 ? n : ldgate, n, y_type)) return rc;
    if (x) {
        if (!is_float_type(x_type) && x_type != QTIP_I8) return fail(QTIP_EUNSUPPORTED, "%s: x of type %d", fn, x_type);
        if (int rc = check_matrix(fn, "x", x, ldx, n, x_type)) return rc;
        if (x_type == QTIP_I8 && (!x_scale || !aligned(x_scale, 4)))
            return fail(QTIP_EINVAL, "%s: x in 8 bits needs x_scale, 4-byte aligned", fn);
    } else if (pre_weight || signs) {
        return fail(QTIP_EINVAL, "%s: a norm or a transform in front of x without x", fn);
    }
    if (!aligned(post_weight, 4) || !aligned(post_bias, 4) || !aligned(pre_weight, 4) || !aligned(pre_bias, 4))
        return fail(QTIP_EINVAL, "%s: weights and biases must be 4-byte aligned", fn);
    if (!(eps >= 0.f)) return fail(QTIP_EINVAL, "%s: eps must not be negative", fn);
    qtip::NormResidual a = {};
    a.y = y, a.h = h, a.gate = gate, a.h_out = h_out, a.x = x;
    a.post = post_weight, a.post_bias = post_bias, a.pre = pre_weight, a.pre_bias = pre_bias;
    a.signs = signs, a.x_scale = x_scale;
    a.ldy = ldy, a.ldh = ldh, a.ldgate = ldgate, a.ldx = ldx;
    a.n = n, a.layer = norm == QTIP_NORM_LAYER, a.x_type = x_type, a.eps = eps, a.res_scale = res_scale;
    hipError_t e = qtip::launch_norm_residual(a, y_type, h_type, rows, block, (hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(fn, e);
    return QTIP_OK;
}

size_t qtip_moe_i8_workspace(int T, int n, int f, int E, int top_k) {
    if (T < 1 || T > QTIP_MOE_MAX_TOKENS || n < 1 || n > QTIP_ROWS_MAX_N || f < 1 || f > QTIP_ROWS_MAX_N || E < 1 || E > QTIP_MOE_MAX_EXPERTS ||
        top_k < 1 || top_k > QTIP_MOE_MAX_TOP_K || top_k > E)
        return 0;
    return qtip::moe_i8_workspace(T, n, f, E, top_k);
}

int qtip_moe_i8(const void *x, int64_t ldx, int type, int T, int n, const void *router, const float *router_bias, int E,
                int top_k, int renormalize, const int8_t *W_up, const float *up_scale, int f, const int8_t *W_down,
                const float *down_scale, void *y, int64_t ldy, int32_t *ids, float *weights, void *workspace,
                size_t workspace_bytes, void *stream) {
    const char *fn = "qtip_moe_i8";
    if (!x || !router || !W_up || !up_scale || !W_down || !down_scale || !y || !workspace)
        return fail(QTIP_EINVAL, "%s: NULL pointer", fn);
    if (type != QTIP_F16 && type != QTIP_BF16) return fail(QTIP_EUNSUPPORTED, "%s: type %d is not F16 or BF16", fn, type);
    if (T < 1 || T > QTIP_MOE_MAX_TOKENS)
        return fail(QTIP_EINVAL, "%s: T = %d must be in [1, QTIP_MOE_MAX_TOKENS = %d]", fn, T, QTIP_MOE_MAX_TOKENS);
    if (E < 1 || E > QTIP_MOE_MAX_EXPERTS)
        return fail(QTIP_EINVAL, "%s: E = %d must be in [1, QTIP_MOE_MAX_EXPERTS = %d]", fn, E, QTIP_MOE_MAX_EXPERTS);
    if (top_k < 1 || top_k > E || top_k > QTIP_MOE_MAX_TOP_K)
        return fail(QTIP_EINVAL, "%s: top_k = %d must be in [1, %d] and no more than E = %d", fn, top_k, QTIP_MOE_MAX_TOP_K, E);
    if (n < 1 || f < 1 || n % 16 || f % 16)
        return fail(QTIP_EINVAL, "%s: n = %d and f = %d must be positive multiples of 16", fn, n, f);
    if (n > QTIP_ROWS_MAX_N || f > QTIP_ROWS_MAX_N)
        return fail(QTIP_EINVAL, "%s: n = %d or f = %d is above QTIP_ROWS_MAX_N = %d", fn, n, f, QTIP_ROWS_MAX_N);
    if (ldx < n || ldy < n) return fail(QTIP_EINVAL, "%s: rows of x and y are less than n = %d values apart", fn, n);
    if (ldx > QTIP_I8_MAX_LD)
        return fail(QTIP_EINVAL, "%s: rows of x are more than QTIP_I8_MAX_LD = %d values apart", fn, QTIP_I8_MAX_LD);
    if (ldx % 8 || !aligned(x, 16) || !aligned(router, 16) || !aligned(W_up, 16) || !aligned(W_down, 16) ||
        !aligned(up_scale, 16) || !aligned(down_scale, 16))
        return fail(QTIP_EINVAL, "%s: rows of x, the router, weights and scales must begin at multiples of 16 bytes", fn);
    if (!aligned(y, 2) || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(router_bias, 4) || !aligned(workspace, 256))
        return fail(QTIP_EINVAL, "%s: y needs 2-byte, ids, weights and router_bias 4-byte, workspace 256-byte alignment", fn);
    const size_t need = qtip::moe_i8_workspace(T, n, f, E, top_k);
    if (workspace_bytes < need) return fail(QTIP_EINVAL, "%s: workspace of %zu bytes, %zu needed", fn, workspace_bytes, need);
    hipError_t e = qtip::launch_moe_i8({x, router, router_bias, W_up, W_down, up_scale, down_scale, y, ids, weights, ldx, ldy, type,
                                        T, n, f, E, top_k, renormalize}, workspace, (hipStream_t)stream);
    if (e != hipSuccess) return hip_fail(fn, e);
    return QTIP_OK;
}

}  // extern "C"
