// Expert matrices in OCP Microscaling MXFP4: four-bit elements (sign, two exponent bits, one
// mantissa bit) with one power-of-two scale for every 32 consecutive elements of a feature's
// reduction.  Layout of the packed handle and the conversion to matrix-core operands, shared
// by the kernels that read it.
//
// Every element value is exact in bf16, and so is its product with the scale (bytes 0 .. 252: from 2^-127,
// subnormal products included, up to 2^125; past them a product may be past the type and is infinite),
// so v_cvt_scalef32_pk_bf16_fp4 turns two codes and the scale into two bf16 operands without a
// rounding: one instruction per two weights is all the 4-bit format costs on the way to the
// bf16 matrix cores.
#pragma once

#include "moe_internal.h"

// The unit of the packed layout is a fragment of 16 output features by 128 reduction indices:
// lane l of a wavefront owns feature l % 16 and the 32 indices 32*(l / 16) .. +31 -- one scale
// block -- as one 16-byte chunk at byte 16*l (1 KiB in all, one coalesced load).  Word j of the
// chunk holds the indices 8j .. 8j+7: the A operand of the fragment's j-th
// v_mfma_f32_16x16x32_bf16, whose B operand is then x[row][32*(l/16) + 8j .. +7].  The products
// of a matrix instruction may be summed in any order of the reduction, so both sides only have
// to agree.  The scales of four consecutive fragments are one 32-bit word per lane.
//   codes : [E][C/16][KS][nmat] fragments,      KS = ceil(K / 128) (indices past K: code 0)
//   scales: [E][C/16][nmat][KW][64 lanes] u32, KW = ceil(KS / 4), byte s = fragment 4w + s
// with nmat = 2 (w1, w3) for the first projection, 1 for the second.  (w1 and w3 side by side: a wave
// that reads both has one stream of addresses.)
#define MX_BLOCK 32
#define MX_FRAG_K 128

static inline __host__ __device__ int mx_frags(int K) { return (K + MX_FRAG_K - 1) / MX_FRAG_K; }
static inline __host__ __device__ int mx_words(int K) { return (mx_frags(K) + 3) / 4; }

#ifdef __HIPCC__
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// The scale of fragment s of a scale word, 2^(byte - 127): the conversion takes the exponent field of a float
// as it is (byte 0, a float of zero, is 2^-127 to it).
__device__ __forceinline__ float mx_scale(unsigned word, int s) {
    return __uint_as_float(((word >> (8 * s)) & 0xFFu) << 23);
}

// Buffer descriptor over the 2 GiB from a wave-uniform p on: a request's address is then one lane
// offset and one scalar.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t mx_rsrc(const void* p) {
    const unsigned long long v = (unsigned long long)p;
    const unsigned lo = __builtin_amdgcn_readfirstlane((int)(unsigned)v);
    const unsigned hi = __builtin_amdgcn_readfirstlane((int)(unsigned)(v >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void*)(((unsigned long long)hi << 32) | lo), 0, (int)0x80000000u, 0x00027000);
}

// What a value's next bf16 part is taken from, behind its part p: nothing where p is infinite or NaN (inf - inf
// would make an infinite value NaN).
__device__ __forceinline__ float mx_rest(float v, float p) { return fabsf(p) < INFINITY ? v - p : 0.f; }

// Eight codes and their scale -> eight bf16 operands, in the order of the codes.
__device__ __forceinline__ bf16x8_t mx_widen8(unsigned codes, float scale) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
#endif

// ---- launchers (moe_mx_convert.hip, moe_mx_stream.hip, moe_mx_gemm.hip) --------------------
int moe_mx_quantize_launch(const void* w, moe_dtype_t w_dtype, int E, int K, int C, uint8_t* codes, uint8_t* scales,
                           hipStream_t s);
int moe_mx_dequantize_launch(const uint8_t* codes, const uint8_t* scales, int E, int K, int C, void* w,
                             moe_dtype_t w_dtype, hipStream_t s);
int moe_mx_pack_impl(const uint8_t* const codes[3], const uint8_t* const scales[3], int E, int d, int f, moe_weights** out,
                     hipStream_t s);

// What the routing of a step and the end of its second projection are told beside the rows.
struct MxStep {
    // gating in the first kernel's prologue (logits or gate_sums given), else null
    const float* logits;      // [T,E]
    const float* gate_sums;   // shares of the gating sums (see moe_decode_block), or null
    int n_shares, gate_stride;
    float eps;
    float* logits_out;        // [T,E] or null
    int T, k;
    int32_t *idx, *counts, *offsets, *perm, *inv_perm;
    float* weights;
    void* xg;                 // [T*k,d] of the activations' type, or null
    // the end of the second projection: the gate-weighted sum of the rows, if y is given
    void* y;                  // [T,d]
    moe_dtype_t y_dtype;
    float* yg;                // [N,d] or null
    const float* x_in;        // [T,d]: y = x_in + sum, or null
    const float* w_gate_next; // [d,E] or null: the next block's gating sums as well
    float* sums_next;         // [d/16][gate_stride]
};

int moe_mx_auto_path(int N, int E, int d, int f);
bool moe_mx_stream_serves(int N, int E, int d, int f);
size_t moe_mx_stream_workspace(int N, int E, int d, int f);
// yg (step == null), or what `step` asks for.  offsets: device, unless step routes.
int moe_mx_stream_launch(const moe_weights* W, const void* x, moe_dtype_t act_dtype, const int32_t* perm, int k,
                         const int32_t* offsets, int N, void* ws, float* yg, const MxStep* step, hipStream_t s);
bool moe_mx_stream_routes(int T, int E, int k, int d, int f);  // may step->logits be given?
bool moe_mx_block_supported(int T, int E, int k, int d, int f);

bool moe_mx_gemm_supported(int N, int E, int d, int f);
size_t moe_mx_gemm_workspace(int N, int E, int d, int f);
int moe_mx_gemm_plan(int N, int E, int d, int f, moe_ffn_plan_t* plan);
int moe_mx_gemm_launch(const moe_weights* W, const void* x, moe_dtype_t act_dtype, const int32_t* perm, int k,
                       const int32_t* offsets, int N, void* ws, float* yg, bool y_f32, const float** slabs, int* n_parts,
                       hipStream_t s);
int moe_mx_combine_launch(const float* yg, int n_parts, size_t part_stride, const int32_t* inv_perm, const float* weights, int T,
                          int k, int d, void* y, moe_dtype_t y_dtype, hipStream_t s);
