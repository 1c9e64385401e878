// Conversion of matrices between fp32 / bf16 and MXFP4, and the one-time repack of converted
// expert matrices into the order the kernels stream them.
//
// Both conversions are bound by memory (the elements' bytes once, 17/32 byte per element for
// codes and scales).  A matrix W [K,C] has its features along the rows and its codes along the
// reduction, so either direction is a transposition: a workgroup takes 64 * V features by 256
// reduction indices, every thread one scale block of V neighbouring features (two where C is
// even), and the 16-byte chunks of codes change hands in LDS, so that global memory sees 256-byte
// rows on one side (bf16) and 128-byte runs of a feature's codes on the other.
#include <new>

#include "moe_mx.h"

#define CV_LANES 64
#define CV_BLOCKS 8   // scale blocks of a tile along the reduction
#define CV_THREADS (CV_LANES * CV_BLOCKS)

// V neighbouring elements as one access
template <bool BF16, int V>
struct CvElems;
template <>
struct CvElems<true, 1> { typedef uint16_t type; };
template <>
struct CvElems<true, 2> { typedef unsigned type; };
template <>
struct CvElems<false, 1> { typedef float type; };
template <>
struct CvElems<false, 2> { typedef float2 type; };

template <bool BF16, int V>
__device__ __forceinline__ void cv_load(const void* w, size_t i, float (&v)[V]) {
    if constexpr (BF16) {
        const unsigned u = *(const typename CvElems<BF16, V>::type*)((const uint16_t*)w + i);
        v[0] = moe_bf16_to_f32(u & 0xFFFFu);
        if constexpr (V == 2) v[1] = __uint_as_float(u & 0xFFFF0000u);
    } else if constexpr (V == 2) {
        const float2 f = *(const float2*)((const float*)w + i);
        v[0] = f.x;
        v[1] = f.y;
    } else {
        v[0] = ((const float*)w)[i];
    }
}

// The scale is 2^(exponent of the largest magnitude - 2), the exponent kept in [-126, 127]: the
// largest element, 6 = 1.5 * 2^2, then has the largest magnitude's exponent.  The division by a
// power of two is exact; v_cvt_scalef32_pk_fp4_f32 rounds to nearest, ties to the even code, and
// saturates.
template <bool BF16, int V>
__global__ __launch_bounds__(CV_THREADS) void mx_quantize_kernel(const void* __restrict__ w, int K, int C, size_t ctiles,
                                                                 uint8_t* __restrict__ codes,
                                                                 uint8_t* __restrict__ scales) {
    constexpr int COLS = CV_LANES * V;
    __shared__ u32x4_t s_codes[CV_BLOCKS][COLS + 1];
    __shared__ uint8_t s_scales[CV_BLOCKS][COLS];
    const int tid = threadIdx.x;
    const size_t e = blockIdx.x / ctiles;
    const int c0 = (int)(blockIdx.x % ctiles) * COLS;
    const int kb = tid / CV_LANES, cl = tid % CV_LANES * V;
    const int KB = K / MX_BLOCK;
    const int b = blockIdx.y * CV_BLOCKS + kb;
    if (b < KB && c0 + cl < C) {
        const size_t at = (e * K + (size_t)b * MX_BLOCK) * C + c0 + cl;
        float v[MX_BLOCK][V];
#pragma unroll
        for (int i = 0; i < MX_BLOCK; i++) cv_load<BF16, V>(w, at + (size_t)i * C, v[i]);
#pragma unroll
        for (int n = 0; n < V; n++) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < MX_BLOCK; i++) top = fmaxf(top, fabsf(v[i][n]));
            int s = (int)(__float_as_uint(top) >> 23) - 2;
            s = s < 1 ? 1 : s;
            const float scale = __uint_as_float((unsigned)s << 23);
            u32x4_t q;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                unsigned o = 0u;
                o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * j][n], v[8 * j + 1][n], scale, 0);
                o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * j + 2][n], v[8 * j + 3][n], scale, 1);
                o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * j + 4][n], v[8 * j + 5][n], scale, 2);
                o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * j + 6][n], v[8 * j + 7][n], scale, 3);
                q[j] = o;
            }
            s_codes[kb][cl + n] = q;
            s_scales[kb][cl + n] = (uint8_t)s;
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < V; n++) {
        const int i = tid + n * CV_THREADS, cc = i / CV_BLOCKS, bb = i % CV_BLOCKS;
        if (c0 + cc < C && (int)blockIdx.y * CV_BLOCKS + bb < KB) {
            const size_t at = (e * C + c0 + cc) * KB + blockIdx.y * CV_BLOCKS + bb;
            *(u32x4_t*)(codes + at * 16) = s_codes[bb][cc];
            scales[at] = s_scales[bb][cc];
        }
    }
}

template <bool BF16, int V>
__global__ __launch_bounds__(CV_THREADS) void mx_dequantize_kernel(const uint8_t* __restrict__ codes,
                                                                   const uint8_t* __restrict__ scales, int K, int C,
                                                                   size_t ctiles, void* __restrict__ w) {
    constexpr int COLS = CV_LANES * V;
    __shared__ u32x4_t s_codes[CV_BLOCKS][COLS + 1];
    __shared__ uint8_t s_scales[CV_BLOCKS][COLS];
    const int tid = threadIdx.x;
    const size_t e = blockIdx.x / ctiles;
    const int c0 = (int)(blockIdx.x % ctiles) * COLS;
    const int KB = K / MX_BLOCK;
#pragma unroll
    for (int n = 0; n < V; n++) {
        const int i = tid + n * CV_THREADS, cc = i / CV_BLOCKS, bb = i % CV_BLOCKS;
        if (c0 + cc < C && (int)blockIdx.y * CV_BLOCKS + bb < KB) {
            const size_t at = (e * C + c0 + cc) * KB + blockIdx.y * CV_BLOCKS + bb;
            s_codes[bb][cc] = *(const u32x4_t*)(codes + at * 16);
            s_scales[bb][cc] = scales[at];
        }
    }
    __syncthreads();
    const int kb = tid / CV_LANES, cl = tid % CV_LANES * V;
    const int b = blockIdx.y * CV_BLOCKS + kb;
    if (b >= KB || c0 + cl >= C) return;
    u32x4_t q[V];
    float scale[V];
#pragma unroll
    for (int n = 0; n < V; n++) {
        q[n] = s_codes[kb][cl + n];
        scale[n] = __uint_as_float((unsigned)s_scales[kb][cl + n] << 23);
    }
    const size_t at = (e * K + (size_t)b * MX_BLOCK) * C + c0 + cl;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        bf16x8_t v[V];
#pragma unroll
        for (int n = 0; n < V; n++) v[n] = mx_widen8(q[n][j], scale[n]);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const size_t o = at + (size_t)(8 * j + i) * C;
            if constexpr (V == 2) {
                if (BF16) *(bf16x2_t*)((__bf16*)w + o) = bf16x2_t{v[0][i], v[1][i]};
                else *(float2*)((float*)w + o) = make_float2((float)v[0][i], (float)v[1][i]);
            } else {
                if (BF16) ((__bf16*)w)[o] = v[0][i];
                else ((float*)w)[o] = (float)v[0][i];
            }
        }
    }
}

static dim3 cv_grid(int E, int K, int C, int V, size_t& ctiles) {
    ctiles = ((size_t)C + CV_LANES * V - 1) / (CV_LANES * V);
    return dim3((unsigned)(E * ctiles), (unsigned)((K / MX_BLOCK + CV_BLOCKS - 1) / CV_BLOCKS));
}

int moe_mx_quantize_launch(const void* w, moe_dtype_t w_dtype, int E, int K, int C, uint8_t* codes, uint8_t* scales,
                           hipStream_t s) {
    size_t ctiles;
    const int V = C % 2 ? 1 : 2;
    const dim3 grid = cv_grid(E, K, C, V, ctiles);
    auto* kernel = w_dtype == MOE_BF16 ? (V == 2 ? mx_quantize_kernel<true, 2> : mx_quantize_kernel<true, 1>)
                                       : (V == 2 ? mx_quantize_kernel<false, 2> : mx_quantize_kernel<false, 1>);
    hipLaunchKernelGGL(kernel, grid, dim3(CV_THREADS), 0, s, w, K, C, ctiles, codes, scales);
    return moe_launch_status();
}

int moe_mx_dequantize_launch(const uint8_t* codes, const uint8_t* scales, int E, int K, int C, void* w,
                             moe_dtype_t w_dtype, hipStream_t s) {
    size_t ctiles;
    const int V = C % 2 ? 1 : 2;
    const dim3 grid = cv_grid(E, K, C, V, ctiles);
    auto* kernel = w_dtype == MOE_BF16 ? (V == 2 ? mx_dequantize_kernel<true, 2> : mx_dequantize_kernel<true, 1>)
                                       : (V == 2 ? mx_dequantize_kernel<false, 2> : mx_dequantize_kernel<false, 1>);
    hipLaunchKernelGGL(kernel, grid, dim3(CV_THREADS), 0, s, codes, scales, K, C, ctiles, w);
    return moe_launch_status();
}

// codes [E][C][K/2] -> fragments [E][C/16][KS][nmat], this launch fills matrix slot `mat`.
// One thread writes one 16-byte chunk; 16 lanes read 16 features' runs of 64 bytes.
__global__ __launch_bounds__(256) void mx_pack_codes_kernel(const uint8_t* __restrict__ src, u32x4_t* __restrict__ dst,
                                                            int E, int K, int C, int nmat, int mat) {
    const size_t KS = (size_t)mx_frags(K), NB = (size_t)C / 16, total = (size_t)E * NB * KS * 64;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
        const int lane = (int)(i & 63);
        const size_t fr = i >> 6, ks = fr % KS, enb = fr / KS;  // enb = e * NB + nb
        const size_t c = enb * 16 + (lane & 15);                // feature, counted through the experts
        const size_t k0 = ks * MX_FRAG_K + MX_BLOCK * (lane >> 4);
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (k0 < (size_t)K) v = *(const u32x4_t*)(src + c * (K / 2) + k0 / 2);
        dst[((enb * KS + ks) * nmat + mat) * 64 + lane] = v;
    }
}

__global__ __launch_bounds__(256) void mx_pack_scales_kernel(const uint8_t* __restrict__ src, unsigned* __restrict__ dst,
                                                             int E, int K, int C, int nmat, int mat) {
    const size_t KW = (size_t)mx_words(K), NB = (size_t)C / 16, total = (size_t)E * NB * KW * 64;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
        const int lane = (int)(i & 63);
        const size_t w = (i >> 6) % KW, enb = (i >> 6) / KW;
        const size_t c = enb * 16 + (lane & 15);
        unsigned v = 0u;
#pragma unroll
        for (int b = 0; b < 4; b++) {
            const size_t blk = (w * 4 + b) * 4 + (lane >> 4);
            if (blk < (size_t)K / MX_BLOCK) v |= (unsigned)src[c * (K / MX_BLOCK) + blk] << (8 * b);
        }
        dst[((enb * nmat + mat) * KW + w) * 64 + lane] = v;
    }
}

int moe_mx_pack_impl(const uint8_t* const codes[3], const uint8_t* const scales[3], int E, int d, int f, moe_weights** out,
                     hipStream_t s) {
    moe_weights* W = new (std::nothrow) moe_weights();
    if (!W) return MOE_ERR_HIP;
    W->E = E;
    W->d = d;
    W->f = f;
    W->dtype = MOE_MXFP4;
    if (hipGetDevice(&W->device) != hipSuccess) {
        (void)hipGetLastError();
        delete W;
        return MOE_ERR_HIP;
    }
    const size_t bytes[4] = {(size_t)E * f / 16 * 2 * mx_frags(d) * 1024, (size_t)E * d / 16 * mx_frags(f) * 1024,
                             (size_t)E * f / 16 * 2 * mx_words(d) * 256, (size_t)E * d / 16 * mx_words(f) * 256};
    void** dst[4] = {&W->w13, &W->w2, &W->s13, &W->s2};
    for (int i = 0; i < 4; i++) {
        if (hipMalloc(dst[i], bytes[i]) != hipSuccess) {
            (void)hipGetLastError();
            for (int j = 0; j < i; j++) (void)hipFree(*dst[j]);
            delete W;
            return MOE_ERR_HIP;
        }
        W->bytes += bytes[i];
    }
    for (int m = 0; m < 3; m++) {
        const bool up = m < 2;
        const int K = up ? d : f, C = up ? f : d;
        hipLaunchKernelGGL(mx_pack_codes_kernel, dim3(4096), dim3(256), 0, s, codes[m],
                           (u32x4_t*)(up ? W->w13 : W->w2), E, K, C, up ? 2 : 1, up ? m : 0);
        hipLaunchKernelGGL(mx_pack_scales_kernel, dim3(1024), dim3(256), 0, s, scales[m],
                           (unsigned*)(up ? W->s13 : W->s2), E, K, C, up ? 2 : 1, up ? m : 0);
    }
    if (moe_launch_status() != MOE_OK) {
        for (int i = 0; i < 4; i++) (void)hipFree(*dst[i]);
        delete W;
        return MOE_ERR_HIP;
    }
    *out = W;
    return MOE_OK;
}
