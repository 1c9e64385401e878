// Matrices and rows in 8-bit integers: symmetric codes in [-127, 127] with one fp32 scale per output
// channel of a matrix and one per row (token).  Layout of the packed handle, the code of a value,
// and what the launchers are told.
//
// A product of codes is exact in the matrix cores' 32-bit integers (127^2 * 2^17 < 2^31), whatever the
// order or split of the sum, so results depend on the codes alone; the scales enter once, at the end.
#pragma once

#include "moe_internal.h"

// The unit of the packed layout is the A operand of one v_mfma_i32_16x16x64_i8: 16 output features by
// 64 reduction indices, lane l of a wavefront feature l % 16 and the 16 indices 16*(l / 16) .. +15, one
// 16-byte chunk at byte 16*l (1 KiB, one coalesced load).
//   w13: [E][f/16][2 (w1,w3)][d/64] fragments, s13: [E][f/16][2][16] fp32
//   w2 : [E][d/16][f/64]                       s2 : [E][d/16][16]
#define I8_FRAG_K 64
#define I8_MAX_K (1 << 17)  // products of a reduction: the sum stays within 32 bits

#ifdef __HIPCC__
typedef int i32x4_t __attribute__((ext_vector_type(4)));

// The scale of a row whose largest magnitude has the bits `top` (as unsigned numbers NaN > inf > finite): top / 127
// rounded to fp32, NaN where the row holds NaN or an infinity.
__device__ __forceinline__ float i8_scale(unsigned top) {
    return top >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float(top) / 127.0f;
}

// v / s to the nearest integer, ties to even, for fp32 v and s.
struct I8Coder {
    float s, half, inv, lift;
    // Rows of tiny values are scaled up by 2^64 first (`lift`), where scales would be subnormal.
    __device__ __forceinline__ explicit I8Coder(float scale) {
        lift = scale < 0x1p-60f ? 0x1p64f : 1.0f;
        s = scale * lift;
        half = 0.5f * s;
        inv = s > 0.0f ? 1.0f / s : 0.0f;  // (zero and NaN rows: codes 0)
    }
    // The quotient by the reciprocal is off by a few parts in 2^24, which is on the wrong side of a border between two
    // codes at times; the remainder v - q*s is exact (v and q*s agree in their leading bits) and says so.
    __device__ __forceinline__ int exact(float v) const {
        v = inv > 0.0f ? v * lift : 0.0f;
        float q = rintf(v * inv);
        const float r = __builtin_fmaf(-q, s, v);
        const bool odd = ((int)q & 1) != 0;
        if (r > half || (r == half && odd && half > 0.0f)) q += 1.0f;
        else if (r < -half || (r == -half && odd && half > 0.0f)) q -= 1.0f;
        return (int)fminf(fmaxf(q, -127.0f), 127.0f);
    }
    // Four codes, packed.  A fused multiply-add with 1.5 * 2^23 rounds to the integer and leaves the code in the low byte;
    // a quotient is off by 127 * 2^-24 at most, so only those within 10^-4 of a border need the above.
    __device__ __forceinline__ unsigned operator()(const float4& v) const {
        const float magic = 12582912.0f, u[4] = {v.x, v.y, v.z, v.w};
        float far = 0.0f;
        unsigned q[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float t = __builtin_fmaf(u[i], inv, magic);
            q[i] = __float_as_uint(t);
            far = fmaxf(far, fabsf(__builtin_fmaf(u[i], inv, magic - t)));
        }
        if (far > 0.4999f || lift != 1.0f || !(inv > 0.0f)) {
#pragma unroll
            for (int i = 0; i < 4; i++) q[i] = (unsigned)exact(u[i]);
        }
        // (the low bytes of the four)
        return __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u) | __builtin_amdgcn_perm(q[3], q[2], 0x04000c0cu);
    }
};

__device__ __forceinline__ unsigned i8_pack4(int a, int b, int c, int d) {
    return (a & 255) | ((b & 255) << 8) | ((c & 255) << 16) | ((unsigned)d << 24);
}

// Sum of code products times the row's and the channel's scale.
__device__ __forceinline__ float i8_value(int sum, float row_scale, float channel_scale) {
    return (float)sum * row_scale * channel_scale;
}
#endif

static inline __host__ __device__ int i8_frags(int K) { return (K + I8_FRAG_K - 1) / I8_FRAG_K; }

// ---- launchers (moe_i8_convert.hip, moe_i8_stream.hip, moe_i8_gemm.hip) --------------------
int moe_i8_quantize_launch(const void* w, moe_dtype_t w_dtype, int E, int K, int C, int8_t* codes, float* scales,
                           hipStream_t s);
int moe_i8_dequantize_launch(const int8_t* codes, const float* scales, int E, int K, int C, void* w, moe_dtype_t w_dtype,
                             hipStream_t s);
int moe_i8_rows_launch(const void* x, moe_dtype_t x_dtype, int T, int K, int8_t* codes, float* scales, hipStream_t s);

// What a layer of a few tokens does before its products, in one launch: routing and batching (N = T*k slots), rows to 8
// bits (x null: they are already).
#define I8_FRONT_SLOTS 512
struct I8Front {
    const float* logits;
    int T, k, E;
    int32_t *idx, *counts, *offsets, *perm, *inv_perm;
    float* weights;
    const void* x;
    int d;
    unsigned* codes;
    float* scales;
};
int moe_i8_front_launch(const I8Front& f, moe_dtype_t x_dtype, hipStream_t s);
int moe_i8_rows_back_launch(const int8_t* codes, const float* scales, int T, int K, void* x, moe_dtype_t x_dtype,
                            hipStream_t s);
int moe_i8_pack_impl(const int8_t* const codes[3], const float* const scales[3], int E, int d, int f, moe_weights** out,
                     hipStream_t s);

// One product: rows x[i], read as x[perm[i] / k] where perm is given, of the experts' segments of `offsets` (null:
// one matrix for all N rows) with the experts' matrices.
struct I8Product {
    const int8_t* x;         // [rows,K]
    const float* xs;         // [rows]
    const int32_t* perm;
    int k;
    const int32_t* offsets;  // [E+1] or null
    int E, N, K, C;          // C: output channels of y
    const int8_t* w;         // packed fragments, or [E][C][K]
    const float* ws;         // scales in the order of the fragments' features, or [E][C]
    bool packed;             // w and ws as above
    bool gated;              // w of pairs (w1, w3): y = silu(x.w1) * (x.w3)
    void* y;                 // [N,C]
    bool y_bf16;
    unsigned* ytop;          // [N][C/16] or null; gated, STREAM: the bits of the largest magnitude of 16 channels of a row
};
int moe_i8_stream_launch(const I8Product& p, hipStream_t s);
bool moe_i8_streams(const I8Product& p, int NR);  // do loads of the matrices (NR fragment rows each) go past the caches?
int moe_i8_product_launch(const I8Product& p, int path, hipStream_t s);  // path: as moe_i8_auto_path names it
bool moe_i8_product_supported(int N, int E, int K, int C, bool gated, int path);

int moe_i8_auto_path(int N, int E);  // MOE_FFN_STREAM or MOE_FFN_GROUPED

// The expert FFN.
size_t moe_i8_ffn_workspace(int N, int E, int d, int f);
bool moe_i8_ffn_supported(int path, int N, int E, int d, int f);
int moe_i8_ffn_plan(int N, int E, int d, int f, moe_ffn_plan_t* plan);  // plan->path given
// x: `rows` rows of fp32 or bf16.
int moe_i8_ffn_launch(const moe_weights* W, const void* x, moe_dtype_t act_dtype, int rows, const int32_t* perm, int k,
                      const int32_t* offsets, int N, void* ws, float* yg, int path, hipStream_t s);

// The gate-weighted sum at the end of a layer.
struct I8Combine {
    const int32_t* inv_perm;
    const float* weights;
    int T, k;
    void* y;
    bool y_bf16;
};
// The second projection of a few rows, h in fp32 with the largest magnitudes that the first one leaves (ytop): yg, or, with c,
// the layer's y.
bool moe_i8_down_small_serves(int N, int K);
int moe_i8_down_small_launch(const moe_weights* W, const float* h, const unsigned* htop, const int32_t* offsets, int N, float* yg,
                             const I8Combine* c, hipStream_t s);
// The layer from routed tokens and logits: offsets, perm and the others of `f` are written; f's x or its codes and scales
// given, the rest filled in here.  ws: the FFN's workspace and [N,d] floats behind it.
int moe_i8_layer_launch(const moe_weights* W, I8Front f, moe_dtype_t x_dtype, void* ws, void* y, moe_dtype_t y_dtype, int path,
                        hipStream_t s);

// The expert FFN of many rows per expert (moe_i8_grouped.hip), from codes.
bool moe_i8_grouped_supported(int N, int E, int d, int f);
size_t moe_i8_grouped_workspace(int N, int E, int d, int f);
int moe_i8_grouped_tile_rows(int N, int E);
int moe_i8_grouped_launch(const moe_weights* W, const int8_t* codes, const float* scales, const int32_t* perm, int k,
                          const int32_t* offsets, int N, void* ws, float* yg, hipStream_t s);
