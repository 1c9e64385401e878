// Conversion of matrices between fp32 / bf16 and MXFP4, and the one-time repack of converted
// expert matrices into the order the kernels stream them.
//
// Both conversions are bound by memory (the elements' bytes once, 17/32 byte per element for
// codes and scales).  A matrix W [K,C] has its features along the rows and its codes along the
// reduction, so either direction is a transposition: a workgroup takes 64 * V features by 256
// reduction indices, every thread one scale block of V neighbouring features (as many as C is a
// multiple of, up to 8 bytes), and the 16-byte chunks of codes change hands in LDS, so that global
// memory sees 512-byte rows on one side and 128-byte runs of a feature's codes on the other.
#include <new>

#include "moe_mx.h"

#define CV_LANES 64
#define CV_BLOCKS 8   // scale blocks of a tile along the reduction
#define CV_THREADS (CV_LANES * CV_BLOCKS)

// V neighbouring elements as one access of 2 .. 8 bytes
template <int BYTES>
struct CvWord;
template <>
struct CvWord<2> { typedef uint16_t type; };
template <>
struct CvWord<4> { typedef unsigned type; };
template <>
struct CvWord<8> { typedef uint2 type; };
template <bool BF16, int V>
union CvElems {
    typename CvWord<(BF16 ? 2 : 4) * V>::type word;
    uint16_t h[V];
    float f[V];
    __device__ __forceinline__ float at(int n) const { return BF16 ? moe_bf16_to_f32(h[n]) : f[n]; }
};

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
        typedef CvElems<BF16, V> Elems;
        Elems v[MX_BLOCK];
#pragma unroll
        for (int i = 0; i < MX_BLOCK; i++)
            v[i].word = *(const decltype(Elems::word)*)((const char*)w + (at + (size_t)i * C) * (BF16 ? 2 : 4));
#pragma unroll
        for (int n = 0; n < V; n++) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < MX_BLOCK; i++) top = fmaxf(top, fabsf(v[i].at(n)));
            int s = (int)(__float_as_uint(top) >> 23) - 2;
            s = s < 1 ? 1 : s;
            const float scale = __uint_as_float((unsigned)s << 23);
            u32x4_t q;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                unsigned o = 0u;
                o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * j].at(n), v[8 * j + 1].at(n), scale, 0);
                o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * j + 2].at(n), v[8 * j + 3].at(n), scale, 1);
                o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * j + 4].at(n), v[8 * j + 5].at(n), scale, 2);
                o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[8 * j + 6].at(n), v[8 * j + 7].at(n), scale, 3);
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
            CvElems<BF16, V> o;
#pragma unroll
            for (int n = 0; n < V; n++) {
                if constexpr (BF16) o.h[n] = __builtin_bit_cast(uint16_t, (__bf16)v[n][i]);
                else o.f[n] = (float)v[n][i];
            }
            *(decltype(o.word)*)((char*)w + (at + (size_t)(8 * j + i) * C) * (BF16 ? 2 : 4)) = o.word;
        }
    }
}

// Features a thread takes.
static int cv_width(int C, bool bf16) { return bf16 && C % 4 == 0 ? 4 : C % 2 == 0 ? 2 : 1; }

static dim3 cv_grid(int E, int K, int C, int V, size_t& ctiles) {
    ctiles = ((size_t)C + CV_LANES * V - 1) / (CV_LANES * V);
    return dim3((unsigned)(E * ctiles), (unsigned)((K / MX_BLOCK + CV_BLOCKS - 1) / CV_BLOCKS));
}

#define CV_PICK(kernel)                                                                                      \
    w_dtype == MOE_BF16 ? (V == 4 ? kernel<true, 4> : V == 2 ? kernel<true, 2> : kernel<true, 1>)            \
                        : (V == 2 ? kernel<false, 2> : kernel<false, 1>)

int moe_mx_quantize_launch(const void* w, moe_dtype_t w_dtype, int E, int K, int C, uint8_t* codes, uint8_t* scales,
                           hipStream_t s) {
    size_t ctiles;
    const int V = cv_width(C, w_dtype == MOE_BF16);
    const dim3 grid = cv_grid(E, K, C, V, ctiles);
    auto* kernel = CV_PICK(mx_quantize_kernel);
    hipLaunchKernelGGL(kernel, grid, dim3(CV_THREADS), 0, s, w, K, C, ctiles, codes, scales);
    return moe_launch_status();
}

int moe_mx_dequantize_launch(const uint8_t* codes, const uint8_t* scales, int E, int K, int C, void* w,
                             moe_dtype_t w_dtype, hipStream_t s) {
    size_t ctiles;
    const int V = cv_width(C, w_dtype == MOE_BF16);
    const dim3 grid = cv_grid(E, K, C, V, ctiles);
    auto* kernel = CV_PICK(mx_dequantize_kernel);
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
