// C ABI of libmoe_hip (include/moe.h): argument validation on the host, then
// dispatch to the kernel launchers.  Nothing is enqueued when validation fails.
#include "moe_internal.h"
#include "moe_i8.h"
#include "moe_mx.h"

// mean rows per expert up to which AUTO names MID: no crossover, but the range in which it serves
// f = 128
#ifndef MOE_MID_MAX_ROWS
#define MOE_MID_MAX_ROWS 10
#endif

static inline bool dims_ok(int d) { return d >= 64 && d % 64 == 0 && d <= (1 << 20); }
static inline bool tek_ok(int T, int E, int k) {
    return T >= 0 && E >= 1 && E <= MOE_MAX_E && k >= 1 && k <= MOE_MAX_K && k <= E &&
           (long long)T * k < MOE_MAX_N;
}
static inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// Do two byte ranges overlap?
static inline bool ranges_overlap(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return a && b && a0 < b0 + bn && b0 < a0 + an;
}

// AUTO's choice of kernel family (measured crossovers, Mixtral shape and the 16-expert shape,
// Zipf-skewed routing; with balanced routing each kernel stays ahead somewhat longer than its
// limit here):
//   up to 72 routed rows the decode kernels, which stream each active expert once per
//   16-row tile at ~6.5 TB/s;
//   up to MOE_MID_MAX_ROWS rows per expert on average MID, above that GROUPED: the same launches,
//   except that only MID serves f = 128.
int moe_ffn_auto_path(int N, int E, int d, int f) {
    if (N <= 72 && moe_ffn_stream_supported(d, f)) return MOE_FFN_STREAM;
    if ((long long)N <= (long long)MOE_MID_MAX_ROWS * E && moe_ffn_grouped_supported(true, N, E, d, f))
        return MOE_FFN_MID;
    return MOE_FFN_GROUPED;
}

// Argument checks of the four calls of the hot path, without a launch: what moe_layer asks of all four
// before the first of them runs.

static int route_args(const float* logits, int T, int E, int k, const int32_t* idx, const float* weights) {
    if (!tek_ok(T, E, k)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!logits || !idx || !weights) return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(logits) || !moe_aligned16(idx) || !moe_aligned16(weights))
        return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

static int permute_args(const int32_t* idx, int T, int E, int k, const void* x, int d, moe_dtype_t x_dtype,
                        const int32_t* counts, const int32_t* offsets, const int32_t* perm,
                        const int32_t* inv_perm, const void* xg) {
    if (!tek_ok(T, E, k)) return MOE_ERR_INVALID_ARG;
    if (!counts || !offsets) return MOE_ERR_INVALID_ARG;
    if (T > 0 && (!idx || !perm || !inv_perm)) return MOE_ERR_INVALID_ARG;
    if ((x == nullptr) != (xg == nullptr)) return MOE_ERR_INVALID_ARG;
    if (x) {
        if (!dims_ok(d) || (x_dtype != MOE_F32 && x_dtype != MOE_BF16)) return MOE_ERR_INVALID_ARG;
        if (!moe_aligned16(x) || !moe_aligned16(xg)) return MOE_ERR_INVALID_ARG;
    }
    if (!moe_aligned16(idx) || !moe_aligned16(perm) || !moe_aligned16(inv_perm))
        return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

// `path`: the caller's; in its place the kernel family that runs (all-fp32: AUTO).
static int ffn_args(const moe_weights_t* W, const void* xg, moe_dtype_t act_dtype, const int32_t* offsets,
                    int N, const void* workspace, size_t workspace_bytes, const float* yg, int& path) {
    if (!W || N < 0 || N >= MOE_MAX_N) return MOE_ERR_INVALID_ARG;
    if (act_dtype != MOE_F32 && act_dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (path != MOE_FFN_AUTO && path != MOE_FFN_STREAM && path != MOE_FFN_GROUPED &&
        path != MOE_FFN_MID)
        return MOE_ERR_INVALID_ARG;
    if (!offsets) return MOE_ERR_INVALID_ARG;
    if (N == 0) return MOE_OK;
    if (!xg || !yg || !moe_aligned16(xg) || !moe_aligned16(yg)) return MOE_ERR_INVALID_ARG;
    if (!workspace || (((uintptr_t)workspace) & 255u)) return MOE_ERR_WORKSPACE;
    if (workspace_bytes < moe_expert_ffn_workspace(N, W->E, W->d, W->f, act_dtype))
        return MOE_ERR_WORKSPACE;
    bool served;
    if (W->dtype == MOE_F32) {
        served = act_dtype == MOE_F32 && path == MOE_FFN_AUTO && moe_ffn_f32_supported(N, W->E);
    } else if (W->dtype == MOE_MXFP4) {
        if (path == MOE_FFN_AUTO) path = moe_mx_auto_path(N, W->E, W->d, W->f);
        served = path == MOE_FFN_STREAM ? moe_mx_stream_serves(N, W->E, W->d, W->f)
                                        : path == MOE_FFN_GROUPED && moe_mx_gemm_supported(N, W->E, W->d, W->f);
    } else if (W->dtype == MOE_INT8) {
        if (path == MOE_FFN_AUTO) path = moe_i8_auto_path(N, W->E);
        served = moe_i8_ffn_supported(path, N, W->E, W->d, W->f);
        if (served && W->device != moe_current_device()) return MOE_ERR_INVALID_ARG;
    } else {
        if (path == MOE_FFN_AUTO) path = moe_ffn_auto_path(N, W->E, W->d, W->f);
        served = path == MOE_FFN_STREAM ? moe_ffn_stream_serves(N, W->E, W->d, W->f)
                                        : moe_ffn_grouped_supported(path == MOE_FFN_MID, N, W->E, W->d, W->f);
    }
    return served ? MOE_OK : MOE_ERR_UNSUPPORTED;
}

static int combine_args(const float* yg, const int32_t* inv_perm, const float* weights, int T, int k, int d,
                        const float* y) {
    if (T < 0 || k < 1 || k > MOE_MAX_K || (long long)T * k >= MOE_MAX_N || !dims_ok(d))
        return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!yg || !inv_perm || !weights || !y) return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(yg) || !moe_aligned16(y)) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

// Can moe_layer route and batch in one launch?  A few slots; and every workgroup then reads logits and x while others
// write, so calls in which an output lies over one of them keep the two launches.
static bool fused_front(const float* logits, int T, int EL, int E, int k, const void* x, size_t x_bytes, const int32_t* idx,
                        const float* weights, const int32_t* counts, const int32_t* offsets, const int32_t* perm,
                        const int32_t* inv_perm, const void* xg) {
    if (T < 1 || !x || !moe_route_permute_rows_supported(T, EL, k)) return false;
    const size_t n = (size_t)T * k * 4, e = (size_t)E * 4;
    const struct { const void* p; size_t bytes; } out[7] = {{idx, n}, {weights, n}, {counts, e}, {offsets, e + 4},
                                                            {perm, n}, {inv_perm, n}, {xg, x_bytes * k}};
    for (const auto& o : out)
        if (ranges_overlap(logits, (size_t)T * EL * 4, o.p, o.bytes) || ranges_overlap(x, x_bytes, o.p, o.bytes)) return false;
    return true;
}

// The launches of moe_expert_ffn and its variants, arguments checked, `path` as ffn_args left it.  With
// `perm` the batched row i is read as xg[perm[i] / k] (xg is then the token array).  k: experts of a token (1 if that
// is not known): so many are in use at least, which rules of a dispatch may go by.
static int ffn_launch(const moe_weights_t* W, const void* xg, moe_dtype_t act_dtype, const int32_t* perm, int k,
                      const int32_t* offsets, int N, void* workspace, float* yg, int path, hipStream_t s) {
    if (N == 0) return MOE_OK;
    if (W->dtype == MOE_F32)
        return moe_ffn_f32_launch(W, (const float*)xg, perm, k, offsets, N, workspace, yg, s);
    if (W->dtype == MOE_MXFP4)
        return path == MOE_FFN_STREAM ? moe_mx_stream_launch(W, xg, act_dtype, perm, k, offsets, N, workspace, yg, nullptr, s)
                                      : moe_mx_gemm_launch(W, xg, act_dtype, perm, k, offsets, N, workspace, yg, true, nullptr, nullptr, s);
    if (W->dtype == MOE_INT8)
        return moe_i8_ffn_launch(W, xg, act_dtype, perm ? N / k : N, perm, k, offsets, N, workspace, yg, path, s);
    if (path == MOE_FFN_STREAM)
        return moe_ffn_stream_launch(W, xg, act_dtype, perm, k, offsets, N, workspace, yg, nullptr, s);
    return moe_ffn_grouped_launch(path == MOE_FFN_MID, W, xg, act_dtype, perm, k, offsets, N, workspace, yg, s);
}

static int ffn_dispatch(const moe_weights_t* W, const void* xg, moe_dtype_t act_dtype,
                        const int32_t* perm, int k, const int32_t* offsets, int N, void* workspace,
                        size_t workspace_bytes, float* yg, int path, void* stream) {
    const int rc = ffn_args(W, xg, act_dtype, offsets, N, workspace, workspace_bytes, yg, path);
    if (rc != MOE_OK) return rc;
    return ffn_launch(W, xg, act_dtype, perm, k, offsets, N, workspace, yg, path, (hipStream_t)stream);
}

// A routed step over MXFP4 experts; logits null: routed before.
static MxStep mx_step(const float* logits, int T, int k, int32_t* idx, float* weights, int32_t* counts, int32_t* offsets,
                      int32_t* perm, int32_t* inv_perm, void* y, moe_dtype_t y_dtype) {
    MxStep st = {};
    st.logits = logits;
    st.T = T;
    st.k = k;
    st.idx = idx;
    st.weights = weights;
    st.counts = counts;
    st.offsets = offsets;
    st.perm = perm;
    st.inv_perm = inv_perm;
    st.y = y;
    st.y_dtype = y_dtype;
    return st;
}

extern "C" {

const char* moe_status_string(int status) {
    switch (status) {
        case MOE_OK: return "ok";
        case MOE_ERR_INVALID_ARG: return "invalid argument";
        case MOE_ERR_UNSUPPORTED: return "unsupported shape or dtype";
        case MOE_ERR_WORKSPACE: return "workspace missing or too small";
        case MOE_ERR_HIP: return "HIP runtime error";
        default: return "unknown status";
    }
}

int moe_route(const float* logits, int T, int E, int k, int32_t* idx, float* weights,
              void* stream) {
    const int rc = route_args(logits, T, E, k, idx, weights);
    if (rc != MOE_OK || T == 0) return rc;
    return moe_route_launch(logits, T, E, k, idx, weights, (hipStream_t)stream);
}

int moe_permute(const int32_t* idx, int T, int E, int k, const void* x, int d,
                moe_dtype_t x_dtype, int32_t* counts, int32_t* offsets, int32_t* perm,
                int32_t* inv_perm, void* xg, void* stream) {
    const int rc = permute_args(idx, T, E, k, x, d, x_dtype, counts, offsets, perm, inv_perm, xg);
    if (rc != MOE_OK) return rc;
    // T == 0 still writes counts = 0 and offsets = 0.
    return moe_permute_launch(idx, T, E, k, T > 0 ? x : nullptr, d, x_dtype, counts, offsets, perm,
                              inv_perm, xg, (hipStream_t)stream);
}

int moe_weights_pack(const void* w1, const void* w3, const void* w2, int E, int d, int f,
                     moe_dtype_t w_dtype, moe_weights_t** out, void* stream) {
    if (!out) return MOE_ERR_INVALID_ARG;
    *out = nullptr;
    if (!w1 || !w3 || !w2 || E < 1 || E > MOE_MAX_E || !dims_ok(d) || !dims_ok(f))
        return MOE_ERR_INVALID_ARG;
    if (w_dtype != MOE_F32 && w_dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(w1) || !moe_aligned16(w3) || !moe_aligned16(w2)) return MOE_ERR_INVALID_ARG;
    return moe_weights_pack_impl(w1, w3, w2, E, d, f, w_dtype, out, (hipStream_t)stream);
}

static bool mxfp4_dims_ok(int E, int K, int C) {
    return E >= 1 && E <= MOE_MAX_E && K >= MX_BLOCK && K % MX_BLOCK == 0 && K <= (1 << 20) && C >= 1 && C <= (1 << 20);
}

int moe_mxfp4_quantize(const void* w, moe_dtype_t w_dtype, int E, int K, int C, uint8_t* codes, uint8_t* scales,
                       void* stream) {
    if (!mxfp4_dims_ok(E, K, C) || (w_dtype != MOE_F32 && w_dtype != MOE_BF16)) return MOE_ERR_INVALID_ARG;
    if (!w || !codes || !scales || !moe_aligned16(w) || !moe_aligned16(codes) || !moe_aligned16(scales))
        return MOE_ERR_INVALID_ARG;
    const size_t n = (size_t)E * K * C, wb = n * (w_dtype == MOE_BF16 ? 2 : 4);
    if (ranges_overlap(w, wb, codes, n / 2) || ranges_overlap(w, wb, scales, n / MX_BLOCK) ||
        ranges_overlap(codes, n / 2, scales, n / MX_BLOCK))
        return MOE_ERR_INVALID_ARG;
    return moe_mx_quantize_launch(w, w_dtype, E, K, C, codes, scales, (hipStream_t)stream);
}

int moe_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int E, int K, int C, void* w, moe_dtype_t w_dtype,
                         void* stream) {
    if (!mxfp4_dims_ok(E, K, C) || (w_dtype != MOE_F32 && w_dtype != MOE_BF16)) return MOE_ERR_INVALID_ARG;
    if (!w || !codes || !scales || !moe_aligned16(w) || !moe_aligned16(codes) || !moe_aligned16(scales))
        return MOE_ERR_INVALID_ARG;
    const size_t n = (size_t)E * K * C, wb = n * (w_dtype == MOE_BF16 ? 2 : 4);
    if (ranges_overlap(w, wb, codes, n / 2) || ranges_overlap(w, wb, scales, n / MX_BLOCK)) return MOE_ERR_INVALID_ARG;
    return moe_mx_dequantize_launch(codes, scales, E, K, C, w, w_dtype, (hipStream_t)stream);
}

int moe_weights_pack_mxfp4(const uint8_t* w1_codes, const uint8_t* w1_scales, const uint8_t* w3_codes,
                           const uint8_t* w3_scales, const uint8_t* w2_codes, const uint8_t* w2_scales, int E, int d, int f,
                           moe_weights_t** out, void* stream) {
    if (!out) return MOE_ERR_INVALID_ARG;
    *out = nullptr;
    if (E < 1 || E > MOE_MAX_E || !dims_ok(d) || !dims_ok(f)) return MOE_ERR_INVALID_ARG;
    const uint8_t* codes[3] = {w1_codes, w3_codes, w2_codes};
    const uint8_t* scales[3] = {w1_scales, w3_scales, w2_scales};
    for (int i = 0; i < 3; i++)
        if (!codes[i] || !scales[i] || !moe_aligned16(codes[i]) || !moe_aligned16(scales[i])) return MOE_ERR_INVALID_ARG;
    return moe_mx_pack_impl(codes, scales, E, d, f, out, (hipStream_t)stream);
}

// ---- 8-bit integers ----
static bool int8_k_ok(int K) { return K >= 16 && K % 16 == 0 && K <= I8_MAX_K; }
static bool int8_dims_ok(int E, int K, int C) {
    return E >= 1 && E <= MOE_MAX_E && int8_k_ok(K) && C >= 1 && C <= (1 << 20);
}
static bool float_dtype(moe_dtype_t t) { return t == MOE_F32 || t == MOE_BF16; }
static size_t float_bytes(moe_dtype_t t, size_t n) { return n * (t == MOE_BF16 ? 2 : 4); }

// The arguments of the four conversions: n values in floats against their codes and `scales` scales.
static int int8_convert_args(const void* v, moe_dtype_t dtype, size_t n, const int8_t* codes, const float* scales,
                             size_t n_scales) {
    if (!v || !codes || !scales || !moe_aligned16(v) || !moe_aligned16(codes) || !moe_aligned16(scales))
        return MOE_ERR_INVALID_ARG;
    const size_t vb = float_bytes(dtype, n), sb = n_scales * sizeof(float);
    return ranges_overlap(v, vb, codes, n) || ranges_overlap(v, vb, scales, sb) || ranges_overlap(codes, n, scales, sb)
               ? MOE_ERR_INVALID_ARG
               : MOE_OK;
}

int moe_int8_quantize(const void* w, moe_dtype_t w_dtype, int E, int K, int C, int8_t* codes, float* scales, void* stream) {
    if (!int8_dims_ok(E, K, C) || !float_dtype(w_dtype)) return MOE_ERR_INVALID_ARG;
    const int rc = int8_convert_args(w, w_dtype, (size_t)E * K * C, codes, scales, (size_t)E * C);
    return rc != MOE_OK ? rc : moe_i8_quantize_launch(w, w_dtype, E, K, C, codes, scales, (hipStream_t)stream);
}

int moe_int8_dequantize(const int8_t* codes, const float* scales, int E, int K, int C, void* w, moe_dtype_t w_dtype,
                        void* stream) {
    if (!int8_dims_ok(E, K, C) || !float_dtype(w_dtype)) return MOE_ERR_INVALID_ARG;
    const int rc = int8_convert_args(w, w_dtype, (size_t)E * K * C, codes, scales, (size_t)E * C);
    return rc != MOE_OK ? rc : moe_i8_dequantize_launch(codes, scales, E, K, C, w, w_dtype, (hipStream_t)stream);
}

static bool int8_rows_ok(int T, int K) { return T >= 0 && int8_k_ok(K) && (long long)T * K < 1LL << 40; }

int moe_int8_quantize_rows(const void* x, moe_dtype_t x_dtype, int T, int K, int8_t* codes, float* scales, void* stream) {
    if (!int8_rows_ok(T, K) || !float_dtype(x_dtype)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    const int rc = int8_convert_args(x, x_dtype, (size_t)T * K, codes, scales, (size_t)T);
    return rc != MOE_OK ? rc : moe_i8_rows_launch(x, x_dtype, T, K, codes, scales, (hipStream_t)stream);
}

int moe_int8_dequantize_rows(const int8_t* codes, const float* scales, int T, int K, void* x, moe_dtype_t x_dtype,
                             void* stream) {
    if (!int8_rows_ok(T, K) || !float_dtype(x_dtype)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    const int rc = int8_convert_args(x, x_dtype, (size_t)T * K, codes, scales, (size_t)T);
    return rc != MOE_OK ? rc : moe_i8_rows_back_launch(codes, scales, T, K, x, x_dtype, (hipStream_t)stream);
}

int moe_int8_matmul(const int8_t* x_codes, const float* x_scales, int M, const int8_t* w_codes, const float* w_scales, int E,
                    int K, int C, const int32_t* offsets, void* y, moe_dtype_t y_dtype, void* stream) {
    if (!int8_dims_ok(E, K, C) || M < 0 || M >= MOE_MAX_N || !float_dtype(y_dtype) || (!offsets && E != 1))
        return MOE_ERR_INVALID_ARG;
    if (M == 0) return MOE_OK;
    if (!x_codes || !x_scales || !w_codes || !w_scales || !y || !moe_aligned16(x_codes) || !moe_aligned16(x_scales) ||
        !moe_aligned16(w_codes) || !moe_aligned16(w_scales) || !moe_aligned16(y) || (offsets && !moe_aligned16(offsets)))
        return MOE_ERR_INVALID_ARG;
    const size_t yb = float_bytes(y_dtype, (size_t)M * C);
    if (ranges_overlap(y, yb, x_codes, (size_t)M * K) || ranges_overlap(y, yb, x_scales, (size_t)M * 4) ||
        ranges_overlap(y, yb, w_codes, (size_t)E * C * K) || ranges_overlap(y, yb, w_scales, (size_t)E * C * 4) ||
        ranges_overlap(y, yb, offsets, (size_t)(E + 1) * 4))
        return MOE_ERR_INVALID_ARG;
    const int path = moe_i8_auto_path(M, E);
    if (!moe_i8_product_supported(M, E, K, C, false, path)) return MOE_ERR_UNSUPPORTED;
    I8Product p = {};
    p.x = x_codes;
    p.xs = x_scales;
    p.k = 1;
    p.offsets = offsets;
    p.E = E;
    p.N = M;
    p.K = K;
    p.C = C;
    p.w = w_codes;
    p.ws = w_scales;
    p.y = y;
    p.y_bf16 = y_dtype == MOE_BF16;
    return moe_i8_product_launch(p, path, (hipStream_t)stream);
}

int moe_weights_pack_int8(const int8_t* w1_codes, const float* w1_scales, const int8_t* w3_codes, const float* w3_scales,
                          const int8_t* w2_codes, const float* w2_scales, int E, int d, int f, moe_weights_t** out,
                          void* stream) {
    if (!out) return MOE_ERR_INVALID_ARG;
    *out = nullptr;
    if (E < 1 || E > MOE_MAX_E || !dims_ok(d) || !dims_ok(f) || d > I8_MAX_K || f > I8_MAX_K) return MOE_ERR_INVALID_ARG;
    const int8_t* codes[3] = {w1_codes, w3_codes, w2_codes};
    const float* scales[3] = {w1_scales, w3_scales, w2_scales};
    for (int i = 0; i < 3; i++)
        if (!codes[i] || !scales[i] || !moe_aligned16(codes[i]) || !moe_aligned16(scales[i])) return MOE_ERR_INVALID_ARG;
    return moe_i8_pack_impl(codes, scales, E, d, f, out, (hipStream_t)stream);
}

// what moe_layer_int8 keeps beside the expert FFN's scratch: the experts' rows
static size_t i8_layer_rows(int N, int d) { return align256((size_t)N * d * sizeof(float)); }

size_t moe_layer_int8_workspace(int T, int E, int k, int d, int f) {
    if (!tek_ok(T, E, k) || !dims_ok(d) || !dims_ok(f)) return 0;
    return align256(i8_layer_rows(T * k, d) + moe_i8_ffn_workspace(T * k, E, d, f)) + 256;
}

int moe_layer_int8(const moe_weights_t* W, const void* x, moe_dtype_t x_dtype, const float* x_scales, const float* logits,
                   int T, int k, int32_t* idx, float* weights, int32_t* counts, int32_t* offsets, int32_t* perm,
                   int32_t* inv_perm, void* workspace, size_t workspace_bytes, void* y, moe_dtype_t y_dtype, void* stream) {
    if (!W || W->dtype != MOE_INT8) return MOE_ERR_INVALID_ARG;
    const int E = W->E, d = W->d, f = W->f;
    if (!tek_ok(T, E, k) || !counts || !offsets) return MOE_ERR_INVALID_ARG;
    if ((!float_dtype(x_dtype) && x_dtype != MOE_INT8) || !float_dtype(y_dtype)) return MOE_ERR_INVALID_ARG;
    const int N = T * k;
    hipStream_t s = (hipStream_t)stream;
    if (T == 0)
        return moe_permute_launch(idx, 0, E, k, nullptr, d, MOE_F32, counts, offsets, perm, inv_perm, nullptr, s);
    if (!x || !logits || !idx || !weights || !perm || !inv_perm || !y) return MOE_ERR_INVALID_ARG;
    if ((x_dtype == MOE_INT8) != (x_scales != nullptr)) return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(x) || !moe_aligned16(y) || !moe_aligned16(logits) || !moe_aligned16(idx) || !moe_aligned16(weights) ||
        !moe_aligned16(perm) || !moe_aligned16(inv_perm) || (x_scales && !moe_aligned16(x_scales)))
        return MOE_ERR_INVALID_ARG;
    const int path = moe_i8_auto_path(N, E);
    if (!moe_i8_ffn_supported(path, N, E, d, f)) return MOE_ERR_UNSUPPORTED;
    if (!workspace || (((uintptr_t)workspace) & 255u)) return MOE_ERR_WORKSPACE;
    if (workspace_bytes < moe_layer_int8_workspace(T, E, k, d, f)) return MOE_ERR_WORKSPACE;
    const size_t td = (size_t)T * d, n4 = (size_t)N * 4, e4 = (size_t)E * 4;
    const size_t xb = x_dtype == MOE_INT8 ? td : float_bytes(x_dtype, td);
    const struct { const void* p; size_t bytes; } out[8] = {
        {idx, n4}, {weights, n4}, {counts, e4}, {offsets, e4 + 4}, {perm, n4}, {inv_perm, n4},
        {y, float_bytes(y_dtype, td)}, {workspace, workspace_bytes}};
    for (int o = 0; o < 8; o++) {
        const void* p = out[o].p;
        const size_t bytes = out[o].bytes;
        if (ranges_overlap(logits, (size_t)T * E * 4, p, bytes) || ranges_overlap(x, xb, p, bytes) ||
            ranges_overlap(x_scales, (size_t)T * 4, p, bytes))
            return MOE_ERR_INVALID_ARG;
        for (int q = 0; q < o; q++)
            if (ranges_overlap(out[q].p, out[q].bytes, p, bytes)) return MOE_ERR_INVALID_ARG;
    }
    if (W->device != moe_current_device()) return MOE_ERR_INVALID_ARG;

    I8Front fr = {};
    fr.logits = logits;
    fr.T = T;
    fr.k = k;
    fr.idx = idx;
    fr.counts = counts;
    fr.offsets = offsets;
    fr.perm = perm;
    fr.inv_perm = inv_perm;
    fr.weights = weights;
    if (x_dtype == MOE_INT8) {
        fr.codes = (unsigned*)x;
        fr.scales = (float*)x_scales;
    } else {
        fr.x = x;
    }
    return moe_i8_layer_launch(W, fr, x_dtype, workspace, y, y_dtype, path, s);
}

int moe_block_norm(const void* x, moe_dtype_t x_dtype, const void* y, moe_dtype_t y_dtype, int T, int d, int norm_after,
                   const float* gain_after, const float* gate, const float* row_gate, float residual_scale,
                   const float* gain_before, float eps, void* x_out, void* h, moe_dtype_t h_dtype, int8_t* h_codes,
                   float* h_scales, void* stream) {
    if (T < 0 || !dims_ok(d) || !(eps > 0.f) || !(eps < INFINITY) || !float_dtype(x_dtype)) return MOE_ERR_INVALID_ARG;
    if ((y && !float_dtype(y_dtype)) || (h && !float_dtype(h_dtype))) return MOE_ERR_INVALID_ARG;
    if ((!y && (norm_after || gain_after || gate || row_gate)) || (gain_after && !norm_after)) return MOE_ERR_INVALID_ARG;
    if ((h_codes == nullptr) != (h_scales == nullptr) || (h_codes && d > I8_MAX_K)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!x || (!x_out && !h && !h_codes)) return MOE_ERR_INVALID_ARG;
    const size_t td = (size_t)T * d, d4 = (size_t)d * 4, t4 = (size_t)T * 4;
    const struct { const void* p; size_t bytes; } in[6] = {{x, float_bytes(x_dtype, td)}, {y, float_bytes(y_dtype, td)},
                                                           {gain_after, d4}, {gate, d4}, {row_gate, t4}, {gain_before, d4}};
    const struct { const void* p; size_t bytes; } out[4] = {{x_out, float_bytes(x_dtype, td)}, {h, float_bytes(h_dtype, td)},
                                                            {h_codes, td}, {h_scales, t4}};
    for (const auto& i : in)
        if (i.p && !moe_aligned16(i.p)) return MOE_ERR_INVALID_ARG;
    for (int o = 0; o < 4; o++) {
        if (!out[o].p) continue;
        if (!moe_aligned16(out[o].p)) return MOE_ERR_INVALID_ARG;
        for (const auto& i : in)  // (x_out may be x: a thread reads what it writes before it writes it; no other input has that order)
            if (!(o == 0 && x_out == x && &i == in) && ranges_overlap(i.p, i.bytes, out[o].p, out[o].bytes))
                return MOE_ERR_INVALID_ARG;
        for (int q = 0; q < o; q++)
            if (ranges_overlap(out[q].p, out[q].bytes, out[o].p, out[o].bytes)) return MOE_ERR_INVALID_ARG;
    }
    MoeBlockNorm a = {};
    a.x = x;
    a.y = y;
    a.gain_after = gain_after;
    a.gate = gate;
    a.row_gate = row_gate;
    a.gain_before = gain_before;
    a.x_out = x_out;
    a.h = h;
    a.codes = (unsigned*)h_codes;
    a.scales = h_scales;
    a.T = T;
    a.d = d;
    a.residual_scale = residual_scale;
    a.eps = eps;
    a.norm_after = norm_after != 0;
    a.x_bf16 = x_dtype == MOE_BF16;
    a.y_bf16 = y_dtype == MOE_BF16;
    a.h_bf16 = h_dtype == MOE_BF16;
    return moe_block_norm_launch(a, (hipStream_t)stream);
}

int moe_weights_free(moe_weights_t* w) { return moe_weights_free_impl(w); }

size_t moe_weights_bytes(const moe_weights_t* w) { return w ? w->bytes : 0; }

size_t moe_expert_ffn_workspace(int N, int E, int d, int f, moe_dtype_t act_dtype) {
    if (N < 0 || N >= MOE_MAX_N || E < 1 || E > MOE_MAX_E || !dims_ok(d) || !dims_ok(f)) return 0;
    if (act_dtype != MOE_F32 && act_dtype != MOE_BF16) return 0;
    size_t need = moe_ffn_f32_workspace(N, E, d, f);
    const size_t other[5] = {moe_ffn_stream_workspace(N, E, d, f), moe_ffn_grouped_workspace(N, E, d, f),
                             moe_mx_stream_serves(N, E, d, f) ? moe_mx_stream_workspace(N, E, d, f) : 0,
                             moe_mx_gemm_workspace(N, E, d, f), moe_i8_ffn_workspace(N, E, d, f)};
    for (size_t o : other)
        if (o > need) need = o;
    return align256(need) + 256;
}

int moe_expert_ffn_path(const moe_weights_t* W, const void* xg, moe_dtype_t act_dtype,
                        const int32_t* offsets, int N, void* workspace, size_t workspace_bytes,
                        float* yg, int path, void* stream) {
    return ffn_dispatch(W, xg, act_dtype, nullptr, 1, offsets, N, workspace, workspace_bytes, yg,
                        path, stream);
}

int moe_expert_ffn_tokens(const moe_weights_t* W, const void* x, moe_dtype_t act_dtype, int T,
                          int k, const int32_t* perm, const int32_t* offsets, void* workspace,
                          size_t workspace_bytes, float* yg, void* stream) {
    if (!W || !tek_ok(T, W->E, k)) return MOE_ERR_INVALID_ARG;
    if (T > 0 && (!perm || !moe_aligned16(perm))) return MOE_ERR_INVALID_ARG;
    return ffn_dispatch(W, x, act_dtype, perm, k, offsets, T * k, workspace, workspace_bytes, yg,
                        MOE_FFN_AUTO, stream);
}

int moe_expert_ffn(const moe_weights_t* W, const void* xg, moe_dtype_t act_dtype,
                   const int32_t* offsets, int N, void* workspace, size_t workspace_bytes,
                   float* yg, void* stream) {
    return moe_expert_ffn_path(W, xg, act_dtype, offsets, N, workspace, workspace_bytes, yg,
                               MOE_FFN_AUTO, stream);
}

int moe_expert_ffn_tiles(const int32_t* counts, int E, int d, int f, int path, int k, moe_ffn_tiles_t* up,
                         moe_ffn_tiles_t* down) {
    if (!counts || !up || !down || E < 1 || E > MOE_MAX_E || k < 1 || k > MOE_MAX_K || !dims_ok(d) || !dims_ok(f))
        return MOE_ERR_INVALID_ARG;
    long long N = 0;
    for (int e = 0; e < E; e++) {
        if (counts[e] < 0 || (N += counts[e]) >= MOE_MAX_N) return MOE_ERR_INVALID_ARG;
    }
    if (path == MOE_FFN_AUTO) path = moe_ffn_auto_path((int)N, E, d, f);
    if (path != MOE_FFN_STREAM && path != MOE_FFN_GROUPED && path != MOE_FFN_MID) return MOE_ERR_INVALID_ARG;
    *up = *down = moe_ffn_tiles_t{};
    if (path == MOE_FFN_STREAM) return moe_ffn_stream_supported(d, f) ? MOE_OK : MOE_ERR_UNSUPPORTED;
    return moe_ffn_grouped_tiles(path == MOE_FFN_MID, counts, (int)N, E, d, f, k, up, down);
}

int moe_expert_ffn_plan(int N, int E, int d, int f, moe_dtype_t w_dtype, int path,
                        moe_ffn_plan_t* plan) {
    if (!plan || N < 0 || N >= MOE_MAX_N || E < 1 || E > MOE_MAX_E || !dims_ok(d) || !dims_ok(f))
        return MOE_ERR_INVALID_ARG;
    if (w_dtype != MOE_F32 && w_dtype != MOE_BF16 && w_dtype != MOE_MXFP4 && w_dtype != MOE_INT8) return MOE_ERR_INVALID_ARG;
    if (path != MOE_FFN_AUTO && path != MOE_FFN_STREAM && path != MOE_FFN_GROUPED &&
        path != MOE_FFN_MID)
        return MOE_ERR_INVALID_ARG;
    *plan = moe_ffn_plan_t{};
    plan->n_parts = 1;
    if (w_dtype == MOE_MXFP4) {  // the parts of the second projection are added before the call ends
        plan->path = path == MOE_FFN_AUTO ? moe_mx_auto_path(N, E, d, f) : path;
        if (plan->path == MOE_FFN_STREAM) return moe_mx_stream_serves(N, E, d, f) ? MOE_OK : MOE_ERR_UNSUPPORTED;
        return plan->path == MOE_FFN_GROUPED ? moe_mx_gemm_plan(N, E, d, f, plan) : MOE_ERR_UNSUPPORTED;
    }
    if (w_dtype == MOE_INT8) {
        plan->path = path == MOE_FFN_AUTO ? moe_i8_auto_path(N, E) : path;
        return moe_i8_ffn_plan(N, E, d, f, plan);
    }
    if (w_dtype == MOE_F32) {
        if (path != MOE_FFN_AUTO) return MOE_ERR_UNSUPPORTED;
        plan->path = MOE_FFN_AUTO;  // the all-fp32 kernels are no family of their own
        return MOE_OK;
    }
    if (path == MOE_FFN_AUTO) path = moe_ffn_auto_path(N, E, d, f);
    plan->path = path;
    if (path == MOE_FFN_STREAM) {
        if (!moe_ffn_stream_supported(d, f)) return MOE_ERR_UNSUPPORTED;
        plan->n_parts = moe_ffn_stream_parts(N, d, f);
    } else {
        return moe_ffn_grouped_plan(path == MOE_FFN_MID, N, E, d, f, plan);
    }
    return MOE_OK;
}

int moe_expert_ffn_parts(const moe_weights_t* W, const void* xg, moe_dtype_t act_dtype,
                         const int32_t* offsets, int N, void* workspace, size_t workspace_bytes,
                         float* yg_parts, int max_parts, int* n_parts, void* stream) {
    if (!W || !n_parts || max_parts < 1) return MOE_ERR_INVALID_ARG;
    *n_parts = 1;
    if (N < 0 || N >= MOE_MAX_N) return MOE_ERR_INVALID_ARG;
    const bool stream_path = W->dtype == MOE_BF16 && moe_ffn_auto_path(N, W->E, W->d, W->f) == MOE_FFN_STREAM;
    if (!stream_path || N == 0)
        return moe_expert_ffn_path(W, xg, act_dtype, offsets, N, workspace, workspace_bytes,
                                   yg_parts, MOE_FFN_AUTO, stream);
    if (act_dtype != MOE_F32 && act_dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (!offsets || !xg || !yg_parts || !moe_aligned16(xg) || !moe_aligned16(yg_parts))
        return MOE_ERR_INVALID_ARG;
    if (moe_ffn_stream_parts(N, W->d, W->f) > max_parts) return MOE_ERR_INVALID_ARG;
    if (!workspace || (((uintptr_t)workspace) & 255u)) return MOE_ERR_WORKSPACE;
    if (workspace_bytes < moe_expert_ffn_workspace(N, W->E, W->d, W->f, act_dtype))
        return MOE_ERR_WORKSPACE;
    return moe_ffn_stream_launch(W, xg, act_dtype, nullptr, 1, offsets, N, workspace, yg_parts, n_parts,
                                 (hipStream_t)stream);
}

int moe_combine_parts(const float* yg_parts, int n_parts, const int32_t* inv_perm,
                      const float* weights, int T, int k, int d, float* y, int residual,
                      float* yg, void* stream) {
    if (T < 0 || k < 1 || k > MOE_MAX_K || (long long)T * k >= MOE_MAX_N || !dims_ok(d) ||
        n_parts < 1 || n_parts > 1024)
        return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!yg_parts || !inv_perm || !weights || !y) return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(yg_parts) || !moe_aligned16(y) || (yg && !moe_aligned16(yg)))
        return MOE_ERR_INVALID_ARG;
    const size_t slab = (size_t)T * k * d * sizeof(float);
    if (ranges_overlap(y, (size_t)T * d * sizeof(float), yg_parts, slab * n_parts) ||
        ranges_overlap(yg, slab, yg_parts, slab * n_parts))
        return MOE_ERR_INVALID_ARG;
    return moe_combine_parts_launch(yg_parts, n_parts, (size_t)T * k * d, inv_perm, weights, T, k, d,
                                    y, residual != 0, yg, (hipStream_t)stream);
}

int moe_decode_layer(const moe_weights_t* W, const float* x, const float* logits, int T, int k,
                     int32_t* idx, float* weights, int32_t* counts, int32_t* offsets,
                     int32_t* perm, int32_t* inv_perm, float* xg, void* workspace,
                     size_t workspace_bytes, float* yg, float* y, void* stream) {
    if (!W) return MOE_ERR_INVALID_ARG;
    if (!tek_ok(T, W->E, k)) return MOE_ERR_INVALID_ARG;
    if (!x || !logits || !idx || !weights || !counts || !offsets || !perm || !inv_perm || !y)
        return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(x) || !moe_aligned16(y) || !moe_aligned16(logits) || !moe_aligned16(idx) ||
        !moe_aligned16(weights) || (xg && !moe_aligned16(xg)) || (yg && !moe_aligned16(yg)))
        return MOE_ERR_INVALID_ARG;
    const bool mx = W->dtype == MOE_MXFP4;
    if (mx ? !moe_mx_stream_routes(T, W->E, k, W->d, W->f)
           : W->dtype != MOE_BF16 || !moe_ffn_stream_decode_supported(T, W->E, k, W->d, W->f))
        return MOE_ERR_UNSUPPORTED;
    const int N = T * k;
    if (!workspace || (((uintptr_t)workspace) & 255u)) return MOE_ERR_WORKSPACE;
    if (workspace_bytes < moe_expert_ffn_workspace(N, W->E, W->d, W->f, MOE_F32))
        return MOE_ERR_WORKSPACE;
    // every workgroup of the first kernel reads x and logits while one writes the outputs
    const size_t xb = (size_t)T * W->d * sizeof(float), nb = (size_t)N * W->d * sizeof(float);
    if (ranges_overlap(x, xb, xg, nb) || ranges_overlap(x, xb, y, xb) ||
        ranges_overlap(logits, (size_t)T * W->E * 4, weights, (size_t)N * 4))
        return MOE_ERR_INVALID_ARG;
    if (mx) {
        MxStep st = mx_step(logits, T, k, idx, weights, counts, offsets, perm, inv_perm, y, MOE_F32);
        st.xg = xg;
        st.yg = yg;
        return moe_mx_stream_launch(W, x, MOE_F32, nullptr, k, nullptr, N, workspace, nullptr, &st, (hipStream_t)stream);
    }
    const float* parts = nullptr;
    int n_parts = 1;
    size_t stride = 0;
    int rc = moe_ffn_stream_decode_launch(W, x, logits, T, k, idx, weights, counts, offsets, perm,
                                          inv_perm, xg, workspace, y, yg, &parts, &n_parts, &stride,
                                          (hipStream_t)stream);
    if (rc != MOE_OK || n_parts == 0) return rc;  // 0 parts: the second kernel combined already
    return moe_combine_parts_launch(parts, n_parts, stride, inv_perm, weights, T, k, W->d, y, false,
                                    yg, (hipStream_t)stream);
}

int moe_decode_block(const moe_weights_t* W, const float* x_in, const float* gate_sums,
                     int n_shares, float eps, float* logits, int T, int k, int32_t* idx,
                     float* weights, int32_t* counts, int32_t* offsets, int32_t* perm,
                     int32_t* inv_perm, void* workspace, size_t workspace_bytes, float* x_out,
                     const float* w_gate_next, float* gate_sums_next, void* stream) {
    if (!W) return MOE_ERR_INVALID_ARG;
    if (!tek_ok(T, W->E, k) || T < 1) return MOE_ERR_INVALID_ARG;
    if (!x_in || !logits || !idx || !weights || !counts || !offsets || !perm || !inv_perm || !x_out)
        return MOE_ERR_INVALID_ARG;
    if (gate_sums && (n_shares < 1 || !(eps >= 0.f) || !moe_aligned16(gate_sums)))
        return MOE_ERR_INVALID_ARG;
    if (w_gate_next && (!gate_sums_next || !moe_aligned16(gate_sums_next))) return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(x_in) || !moe_aligned16(x_out) || !moe_aligned16(logits) ||
        !moe_aligned16(idx) || !moe_aligned16(weights))
        return MOE_ERR_INVALID_ARG;
    const bool mx = W->dtype == MOE_MXFP4;
    if (mx ? !moe_mx_block_supported(T, W->E, k, W->d, W->f)
           : W->dtype != MOE_BF16 || !moe_ffn_stream_block_supported(T, W->E, k, W->d, W->f))
        return MOE_ERR_UNSUPPORTED;
    if (gate_sums && n_shares > W->d / 16 && n_shares > 1) return MOE_ERR_INVALID_ARG;
    const int N = T * k;
    if (!workspace || (((uintptr_t)workspace) & 255u)) return MOE_ERR_WORKSPACE;
    if (workspace_bytes < moe_expert_ffn_workspace(N, W->E, W->d, W->f, MOE_F32))
        return MOE_ERR_WORKSPACE;
    // x_out may be x_in itself (every element is read and written by the same lane), nothing else
    const size_t xb = (size_t)T * W->d * sizeof(float), lb = (size_t)T * W->E * sizeof(float);
    const size_t share = (size_t)moe_ffn_stream_gate_stride(T, W->E) * sizeof(float);
    const size_t sb_in = share * (size_t)(gate_sums ? n_shares : 0), sb_out = share * (size_t)(W->d / 16);
    if (x_out != x_in && ranges_overlap(x_in, xb, x_out, xb)) return MOE_ERR_INVALID_ARG;
    if (ranges_overlap(logits, lb, weights, (size_t)N * 4) || ranges_overlap(x_out, xb, logits, lb) ||
        ranges_overlap(gate_sums, sb_in, gate_sums_next, sb_out) ||
        ranges_overlap(x_out, xb, gate_sums_next, sb_out) || ranges_overlap(x_out, xb, gate_sums, sb_in) ||
        ranges_overlap(logits, lb, gate_sums_next, sb_out) || ranges_overlap(logits, lb, gate_sums, sb_in))
        return MOE_ERR_INVALID_ARG;
    if (mx) {
        MxStep st = mx_step(gate_sums ? nullptr : logits, T, k, idx, weights, counts, offsets, perm, inv_perm, x_out, MOE_F32);
        st.gate_stride = moe_ffn_stream_gate_stride(T, W->E);
        if (gate_sums) {
            st.gate_sums = gate_sums;
            st.n_shares = n_shares;
            st.eps = eps;
            st.logits_out = logits;
        }
        st.x_in = x_in;
        st.w_gate_next = w_gate_next;
        st.sums_next = gate_sums_next;
        return moe_mx_stream_launch(W, x_in, MOE_F32, nullptr, k, nullptr, N, workspace, nullptr, &st, (hipStream_t)stream);
    }
    return moe_ffn_stream_block_launch(W, x_in, gate_sums, n_shares, eps, logits, T, k, idx, weights,
                                       counts, offsets, perm, inv_perm, workspace, x_out, w_gate_next,
                                       gate_sums_next, (hipStream_t)stream);
}

int moe_combine(const float* yg, const int32_t* inv_perm, const float* weights, int T, int k,
                int d, float* y, void* stream) {
    const int rc = combine_args(yg, inv_perm, weights, T, k, d, y);
    if (rc != MOE_OK || T == 0) return rc;
    return moe_combine_launch(yg, inv_perm, weights, T, k, d, y, (hipStream_t)stream);
}

int moe_layer(const moe_weights_t* W, const void* x, moe_dtype_t x_dtype, int d, const float* logits, int T,
              int E, int k, int path, int32_t* idx, float* weights, int32_t* counts, int32_t* offsets,
              int32_t* perm, int32_t* inv_perm, void* xg, void* workspace, size_t workspace_bytes, float* yg,
              float* y, int* stage, void* stream) {
    if (!stage) return MOE_ERR_INVALID_ARG;
    int rc;
    // every call's arguments, before the first launch
    *stage = 0;
    if ((rc = route_args(logits, T, E, k, idx, weights)) != MOE_OK) return rc;
    *stage = 2;
    if (!W) return MOE_ERR_INVALID_ARG;
    *stage = 1;
    // The rows of xg are gathered with length d and read with length W->d, and ids of W->E and above have no
    // expert.  (Fewer logits than experts: the last experts get no tokens.)
    if (T > 0 && (d != W->d || E > W->E)) return MOE_ERR_INVALID_ARG;
    if ((rc = permute_args(idx, T, W->E, k, x, d, x_dtype, counts, offsets, perm, inv_perm, xg)) != MOE_OK) return rc;
    *stage = 2;
    if ((rc = ffn_args(W, xg, x_dtype, offsets, T * k, workspace, workspace_bytes, yg, path)) != MOE_OK) return rc;
    *stage = 3;
    if ((rc = combine_args(yg, inv_perm, weights, T, k, W->d, y)) != MOE_OK) return rc;

    hipStream_t s = (hipStream_t)stream;
    *stage = 0;
    if (fused_front(logits, T, E, W->E, k, x, (size_t)T * d * (x_dtype == MOE_BF16 ? 2 : 4), idx, weights, counts, offsets,
                    perm, inv_perm, xg)) {
        rc = moe_route_permute_rows_launch(logits, T, E, W->E, k, x, d, x_dtype, idx, weights, counts, offsets, perm,
                                           inv_perm, xg, s);
    } else {
        if (T > 0 && (rc = moe_route_launch(logits, T, E, k, idx, weights, s)) != MOE_OK) return rc;
        *stage = 1;
        rc = moe_permute_launch(idx, T, W->E, k, T > 0 ? x : nullptr, d, x_dtype, counts, offsets, perm, inv_perm, xg, s);
    }
    if (rc != MOE_OK) return rc;
    *stage = 2;
    if ((rc = ffn_launch(W, xg, x_dtype, nullptr, k, offsets, T * k, workspace, yg, path, s)) != MOE_OK) return rc;
    *stage = 3;
    return T == 0 ? MOE_OK : moe_combine_launch(yg, inv_perm, weights, T, k, W->d, y, s);
}

// what moe_layer_mxfp4 keeps besides the expert FFN's scratch: the experts' rows, where the GEMM leaves them
static size_t mx_layer_rows(int N, int d) { return align256((size_t)N * d * sizeof(float)); }

// Does a call of these sizes route in the streaming kernels' prologue?  That saves four launches, some 12 us.  fp32
// rows of an expert are read by passes of 5 over its matrices, so where there are more of them per expert the GEMM is
// faster, unless the matrices are small (96 MiB: between the last two).  Streamed / GEMM, us, 16 tokens where not
// said: fp32, 8 experts (d 4096, f 14336) 4 rows each 164 / 179, 6 each 238 / 180, 8 each 226 / 181; 4 experts
// (f 6400, 167 MB) 5 each (10 tokens) 49 / 69, 6 each (12) 76 / 70, 16 each 96 / 75; one (f 14336, 94 MB) 16 59 / 64;
// 8 experts (d 2048, f 1408, 37 MB) 8 each 29 / 45.  bf16 rows, 16 to a pass: 8 experts (f 14336) 6 each 141 / 157,
// 8 each 168 / 158; 4 (f 6400) 16 each 61 / 63.
static bool mx_layer_routes(int T, int E, int k, int d, int f, bool x_f32) {
    if (!moe_mx_stream_routes(T, E, k, d, f)) return false;
    const size_t experts = (size_t)(T * k < E ? T * k : E), bytes = experts * 3 * d * f / MX_BLOCK * 17;
    return !x_f32 || T * k <= 5 * E || bytes <= (96u << 20);
}

size_t moe_layer_mxfp4_workspace(int T, int E, int k, int d, int f) {
    if (!tek_ok(T, E, k) || !dims_ok(d) || !dims_ok(f)) return 0;
    const int N = T * k;
    size_t need = 0;
    if (moe_mx_stream_routes(T, E, k, d, f) || moe_mx_auto_path(N, E, d, f) == MOE_FFN_STREAM)
        need = moe_mx_stream_workspace(N, E, d, f);
    if (!mx_layer_routes(T, E, k, d, f, true) && moe_mx_auto_path(N, E, d, f) != MOE_FFN_STREAM) {
        const size_t g = mx_layer_rows(N, d) + moe_mx_gemm_workspace(N, E, d, f);
        need = g > need ? g : need;
    }
    return align256(need) + 256;
}

int moe_layer_mxfp4(const moe_weights_t* W, const void* x, moe_dtype_t x_dtype, const float* logits, int T, int k,
                    int32_t* idx, float* weights, int32_t* counts, int32_t* offsets, int32_t* perm, int32_t* inv_perm,
                    void* workspace, size_t workspace_bytes, void* y, moe_dtype_t y_dtype, void* stream) {
    if (!W || W->dtype != MOE_MXFP4) return MOE_ERR_INVALID_ARG;
    const int E = W->E, d = W->d, f = W->f;
    if (!tek_ok(T, E, k) || !counts || !offsets) return MOE_ERR_INVALID_ARG;
    if ((x_dtype != MOE_F32 && x_dtype != MOE_BF16) || (y_dtype != MOE_F32 && y_dtype != MOE_BF16))
        return MOE_ERR_INVALID_ARG;
    const int N = T * k;
    hipStream_t s = (hipStream_t)stream;
    if (T == 0)
        return moe_permute_launch(idx, 0, E, k, nullptr, d, x_dtype, counts, offsets, perm, inv_perm, nullptr, s);
    if (!x || !logits || !idx || !weights || !perm || !inv_perm || !y) return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(x) || !moe_aligned16(y) || !moe_aligned16(logits) || !moe_aligned16(idx) ||
        !moe_aligned16(weights) || !moe_aligned16(perm) || !moe_aligned16(inv_perm))
        return MOE_ERR_INVALID_ARG;
    const bool routes = mx_layer_routes(T, E, k, d, f, x_dtype == MOE_F32);
    const bool streams = routes || moe_mx_auto_path(N, E, d, f) == MOE_FFN_STREAM;
    if (!streams && !moe_mx_gemm_supported(N, E, d, f)) return MOE_ERR_UNSUPPORTED;
    if (!workspace || (((uintptr_t)workspace) & 255u)) return MOE_ERR_WORKSPACE;
    if (workspace_bytes < moe_layer_mxfp4_workspace(T, E, k, d, f)) return MOE_ERR_WORKSPACE;
    // every workgroup of the first launch may read x and logits while one writes the outputs
    const size_t td = (size_t)T * d, n4 = (size_t)N * 4, e4 = (size_t)E * 4;
    const struct { const void* p; size_t bytes; } out[8] = {
        {idx, n4}, {weights, n4}, {counts, e4}, {offsets, e4 + 4}, {perm, n4}, {inv_perm, n4},
        {y, td * (y_dtype == MOE_BF16 ? 2 : 4)}, {workspace, workspace_bytes}};
    for (const auto& o : out)
        if (ranges_overlap(logits, (size_t)T * E * 4, o.p, o.bytes) ||
            ranges_overlap(x, td * (x_dtype == MOE_BF16 ? 2 : 4), o.p, o.bytes))
            return MOE_ERR_INVALID_ARG;

    MxStep st = mx_step(logits, T, k, idx, weights, counts, offsets, perm, inv_perm, y, y_dtype);
    if (routes)
        return moe_mx_stream_launch(W, x, x_dtype, nullptr, k, nullptr, N, workspace, nullptr, &st, s);
    int rc = moe_route_launch(logits, T, E, k, idx, weights, s);
    if (rc == MOE_OK)
        rc = moe_permute_launch(idx, T, E, k, nullptr, 0, x_dtype, counts, offsets, perm, inv_perm, nullptr, s);
    if (rc != MOE_OK) return rc;
    if (streams) {
        st.logits = nullptr;
        return moe_mx_stream_launch(W, x, x_dtype, perm, k, offsets, N, workspace, nullptr, &st, s);
    }
    float* yg = (float*)workspace;
    const float* slabs = nullptr;
    int n_parts = 1;
    rc = moe_mx_gemm_launch(W, x, x_dtype, perm, k, offsets, N, (char*)workspace + mx_layer_rows(N, d), yg,
                            y_dtype == MOE_F32, &slabs, &n_parts, s);
    if (rc != MOE_OK) return rc;
    return moe_mx_combine_launch(slabs, n_parts, (size_t)N * d, inv_perm, weights, T, k, d, y, y_dtype, s);
}

int moe_rmsnorm(const float* x, int T, int d, float eps, float* h, void* stream) {
    if (T < 0 || !dims_ok(d) || !(eps >= 0.f)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!x || !h) return MOE_ERR_INVALID_ARG;
    return moe_rmsnorm_launch(x, T, d, eps, h, (hipStream_t)stream);
}

int moe_router_logits(const float* h, const float* w_gate, int T, int d, int E, float* logits,
                      void* stream) {
    if (T < 0 || !dims_ok(d) || E < 1 || E > MOE_MAX_E) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!h || !w_gate || !logits) return MOE_ERR_INVALID_ARG;
    if (moe_norm_logits_supported(E) && moe_aligned16(h))
        return moe_norm_logits_launch(false, h, w_gate, T, d, E, 0.f, nullptr, logits, nullptr,
                                      (hipStream_t)stream);
    return moe_router_logits_launch(h, w_gate, T, d, E, logits, (hipStream_t)stream);
}

int moe_rmsnorm_router_logits(const float* x, const float* w_gate, int T, int d, int E, float eps,
                              float* h, float* logits, void* stream) {
    if (T < 0 || !dims_ok(d) || E < 1 || E > MOE_MAX_E || !(eps >= 0.f)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!x || !w_gate || !h || !logits || !moe_aligned16(x) || !moe_aligned16(h))
        return MOE_ERR_INVALID_ARG;
    if (!moe_norm_logits_supported(E)) return MOE_ERR_UNSUPPORTED;
    return moe_norm_logits_launch(true, x, w_gate, T, d, E, eps, h, logits, nullptr,
                                  (hipStream_t)stream);
}

int moe_gate_sums(const float* x, const float* w_gate, int T, int d, int E, float* sums,
                  void* stream) {
    if (T < 0 || !dims_ok(d) || E < 1 || E > MOE_MAX_E) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!x || !w_gate || !sums || !moe_aligned16(x) || !moe_aligned16(sums)) return MOE_ERR_INVALID_ARG;
    if (!moe_norm_logits_supported(E)) return MOE_ERR_UNSUPPORTED;
    return moe_norm_logits_launch(true, x, w_gate, T, d, E, 0.f, nullptr, nullptr, sums,
                                  (hipStream_t)stream);
}

size_t moe_gate_sums_stride(int T, int E) {
    if (T < 1 || E < 1 || E > MOE_MAX_E) return 0;
    return (size_t)moe_ffn_stream_gate_stride(T, E);
}

int moe_decode_block_supported(int T, int E, int k, int d, int f, moe_dtype_t w_dtype) {
    if (!tek_ok(T, E, k) || T < 1 || !dims_ok(d) || !dims_ok(f)) return 0;
    if (w_dtype == MOE_MXFP4) return moe_mx_block_supported(T, E, k, d, f) ? 1 : 0;
    return (w_dtype == MOE_BF16 && moe_ffn_stream_block_supported(T, E, k, d, f)) ? 1 : 0;
}

int moe_residual_add(float* x, const float* y, int T, int d, void* stream) {
    if (T < 0 || !dims_ok(d)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!x || !y || !moe_aligned16(x) || !moe_aligned16(y)) return MOE_ERR_INVALID_ARG;
    return moe_residual_add_launch(x, y, T, d, (hipStream_t)stream);
}

int moe_route_permute(const float* logits, int T, int E, int k, const float* x, int d,
                      int32_t* idx, float* weights, int32_t* counts, int32_t* offsets,
                      int32_t* perm, int32_t* inv_perm, float* xg, void* stream) {
    if (!tek_ok(T, E, k) || !dims_ok(d)) return MOE_ERR_INVALID_ARG;
    if (!logits || !x || !idx || !weights || !counts || !offsets || !perm || !inv_perm || !xg)
        return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(x) || !moe_aligned16(xg)) return MOE_ERR_INVALID_ARG;
    if (ranges_overlap(x, (size_t)T * d * sizeof(float), xg, (size_t)T * k * d * sizeof(float)))
        return MOE_ERR_INVALID_ARG;
    if (T < 1 || T > 16 || E > 16) return MOE_ERR_UNSUPPORTED;
    return moe_gate_small_launch(false, x, nullptr, logits, T, d, E, k, 0.f, nullptr, nullptr, idx,
                                 weights, counts, offsets, perm, inv_perm, xg, nullptr, 1, nullptr,
                                 nullptr, 0, nullptr, (hipStream_t)stream);
}

int moe_norm_route_permute(const float* x, const float* w_gate, int T, int d, int E, int k,
                           float eps, float* h, float* logits, int32_t* idx, float* weights,
                           int32_t* counts, int32_t* offsets, int32_t* perm,
                           int32_t* inv_perm, float* xg, void* stream) {
    if (!tek_ok(T, E, k) || !dims_ok(d) || !(eps >= 0.f)) return MOE_ERR_INVALID_ARG;
    if (!x || !w_gate || !h || !logits || !idx || !weights || !counts || !offsets || !perm ||
        !inv_perm || !xg)
        return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(x) || !moe_aligned16(xg) || !moe_aligned16(h) || !moe_aligned16(w_gate))
        return MOE_ERR_INVALID_ARG;
    // every workgroup reads x while workgroup 0 writes h and the workgroups share xg
    const size_t xb = (size_t)T * d * sizeof(float);
    if (ranges_overlap(x, xb, h, xb) || ranges_overlap(x, xb, xg, xb * k))
        return MOE_ERR_INVALID_ARG;
    if (T < 1 || T > 4 || E > 16) return MOE_ERR_UNSUPPORTED;
    return moe_gate_small_launch(true, x, w_gate, nullptr, T, d, E, k, eps, h, logits, idx, weights,
                                 counts, offsets, perm, inv_perm, xg, nullptr, 1, nullptr, nullptr, 0,
                                 nullptr, (hipStream_t)stream);
}

int moe_combine_norm_route_permute(const float* yg_prev, int n_parts_prev,
                                   const int32_t* inv_perm_prev,
                                   const float* weights_prev, int k_prev, const float* x_in,
                                   float* x_out, const float* w_gate, int T, int d, int E, int k,
                                   float eps, float* h, float* logits, int32_t* idx, float* weights,
                                   int32_t* counts, int32_t* offsets, int32_t* perm,
                                   int32_t* inv_perm, float* xg, void* stream) {
    if (!tek_ok(T, E, k) || !dims_ok(d) || !(eps >= 0.f) || k_prev < 1 || k_prev > MOE_MAX_K)
        return MOE_ERR_INVALID_ARG;
    if (!yg_prev || !inv_perm_prev || !weights_prev || !x_in || !x_out || !w_gate || !h || !logits ||
        !idx || !weights || !counts || !offsets || !perm || !inv_perm || !xg)
        return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(x_in) || !moe_aligned16(x_out) || !moe_aligned16(xg) || !moe_aligned16(h) ||
        !moe_aligned16(yg_prev) || !moe_aligned16(w_gate))
        return MOE_ERR_INVALID_ARG;
    if (n_parts_prev < 1) return MOE_ERR_INVALID_ARG;
    // every workgroup reads the inputs while workgroup 0 writes the outputs
    const size_t xb = (size_t)T * d * sizeof(float);
    const size_t ygb = xb * k_prev * n_parts_prev;
    if (ranges_overlap(x_in, xb, x_out, xb) || ranges_overlap(x_in, xb, h, xb) ||
        ranges_overlap(x_in, xb, xg, xb * k) || ranges_overlap(yg_prev, ygb, xg, xb * k) ||
        ranges_overlap(yg_prev, ygb, h, xb) || ranges_overlap(yg_prev, ygb, x_out, xb) ||
        ranges_overlap(inv_perm_prev, (size_t)T * k_prev * 4, inv_perm, (size_t)T * k * 4) ||
        ranges_overlap(weights_prev, (size_t)T * k_prev * 4, weights, (size_t)T * k * 4))
        return MOE_ERR_INVALID_ARG;
    if (T < 1 || T > 4 || E > 16) return MOE_ERR_UNSUPPORTED;
    return moe_gate_small_launch(true, x_in, w_gate, nullptr, T, d, E, k, eps, h, logits, idx,
                                 weights, counts, offsets, perm, inv_perm, xg, yg_prev, n_parts_prev,
                                 inv_perm_prev, weights_prev, k_prev, x_out, (hipStream_t)stream);
}

int moe_combine_residual(const float* yg, const int32_t* inv_perm, const float* weights, int T,
                         int k, int d, float* x, void* stream) {
    if (T < 0 || k < 1 || k > MOE_MAX_K || (long long)T * k >= MOE_MAX_N || !dims_ok(d))
        return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!yg || !inv_perm || !weights || !x) return MOE_ERR_INVALID_ARG;
    if (!moe_aligned16(yg) || !moe_aligned16(x)) return MOE_ERR_INVALID_ARG;
    return moe_combine_residual_launch(yg, inv_perm, weights, T, k, d, x, (hipStream_t)stream);
}

}  // extern "C"
