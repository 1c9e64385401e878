// Conversion of rows and matrices between fp32 / bf16 and 8-bit codes, and the one-time repack of
// converted expert matrices into the order the kernels stream them.  All of it is bound by memory.
#include <new>
#include <type_traits>

#include "moe_gate_wave.h"
#include "moe_i8.h"
#include "moe_rows.h"

// ---------------------------------------------------------------------- rows ----
// A workgroup takes a row: V chunks of four values a thread, kept in registers between the largest
// magnitude and the codes, so that the row is read once.  Rows longer than 4 * V * blockDim.x are read twice.
template <bool BF16>
__device__ __forceinline__ float4 i8_load4(const void* x, size_t chunk) {
    if (BF16) {
        const uint2 u = ((const uint2*)x)[chunk];
        return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                           __uint_as_float(u.y & 0xFFFF0000u));
    }
    return ((const float4*)x)[chunk];
}
__device__ __forceinline__ unsigned i8_top4(float4 v) {
    const unsigned m = 0x7FFFFFFFu, a = __float_as_uint(v.x) & m, b = __float_as_uint(v.y) & m, c = __float_as_uint(v.z) & m,
                   d = __float_as_uint(v.w) & m;
    const unsigned p = a > b ? a : b, q = c > d ? c : d;
    return p > q ? p : q;
}

// The largest of the workgroup's `top`, in every thread.
__device__ __forceinline__ unsigned i8_block_top(unsigned top, unsigned* s_top) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const unsigned o = (unsigned)__shfl_xor((int)top, m, 64);
        top = top > o ? top : o;
    }
    const int waves = blockDim.x >> 6;
    if (waves == 1) return top;
    if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int w = 0; w < waves; w++) top = top > s_top[w] ? top : s_top[w];
    return top;
}

// Row t of K4 chunks to codes, by the whole workgroup.
template <bool BF16, int V>
__device__ __forceinline__ void i8_row(const void* x, int t, int K4, unsigned* codes, float* scales, unsigned* s_top) {
    const size_t base = (size_t)t * K4;
    float4 v[V];
    unsigned top = 0u;
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int c = threadIdx.x + i * blockDim.x;
        v[i] = c < K4 ? i8_load4<BF16>(x, base + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < V; i++) {
        const unsigned o = i8_top4(v[i]);
        top = top > o ? top : o;
    }
    for (int c = threadIdx.x + V * blockDim.x; c < K4; c += blockDim.x) {
        const unsigned o = i8_top4(i8_load4<BF16>(x, base + c));
        top = top > o ? top : o;
    }
    const float scale = i8_scale(i8_block_top(top, s_top));
    const I8Coder code(scale);
    if (threadIdx.x == 0) scales[t] = scale;
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int c = threadIdx.x + i * blockDim.x;
        if (c < K4) codes[base + c] = code(v[i]);
    }
    for (int c = threadIdx.x + V * blockDim.x; c < K4; c += blockDim.x) {
        const float4 u = i8_load4<BF16>(x, base + c);
        codes[base + c] = code(u);
    }
}

template <bool BF16, int V>
__global__ __launch_bounds__(1024) void i8_rows_kernel(const void* __restrict__ x, int T, int K4, unsigned* __restrict__ codes,
                                                       float* __restrict__ scales) {
    __shared__ unsigned s_top[16];
    each_row(blockIdx.x, gridDim.x, T, [&](int t) __attribute__((always_inline)) {
        i8_row<BF16, V>(x, t, K4, codes, scales, s_top);
        __syncthreads();
    });
}

// Four chunks of a row a thread: rows of 4096 in bf16 that the last-level cache holds, 4096 / 1024 of them, with 1 / 2 / 4 / 8 chunks
// 33.6 / 18.1 / 16.0 / 18.7 us and 9.7 / 6.8 / 7.2 / 9.9; a wave per row with 16 chunks 22.5 and 16.0.  From memory, with the four that are kept,
// 18.2 .. 21.3 and 8.3 (their bytes: 9.9 and 2.5).
static int i8_row_threads(int K4) {
    int threads = 64;
    while (threads < 1024 && threads * 4 < K4) threads *= 2;
    return threads;
}

int moe_i8_rows_launch(const void* x, moe_dtype_t x_dtype, int T, int K, int8_t* codes, float* scales, hipStream_t s) {
    const dim3 grid((unsigned)(T < (1 << 20) ? T : (1 << 20)));
    auto* kernel = x_dtype == MOE_BF16 ? i8_rows_kernel<true, 4> : i8_rows_kernel<false, 4>;
    hipLaunchKernelGGL(kernel, grid, dim3(i8_row_threads(K / 4)), 0, s, x, T, K / 4, (unsigned*)codes, scales);
    return moe_launch_status();
}

// Workgroup 0 routes and batches, the others take a row each.
template <bool BF16>
__global__ __launch_bounds__(1024) void i8_front_kernel(I8Front f) {
    __shared__ unsigned s_top[16];
    __shared__ int s_idx[I8_FRONT_SLOTS], s_pos[I8_FRONT_SLOTS], s_next[64];
    if (blockIdx.x > 0) {
        i8_row<BF16, 4>(f.x, blockIdx.x - 1, f.d / 4, f.codes, f.scales, s_top);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), N = f.T * f.k;
    gate_route_any(f.logits, f, f.E, wave, blockDim.x >> 6, lane, s_idx, true);
    if (threadIdx.x < 64) s_next[threadIdx.x] = 0;
    __syncthreads();
    if (wave == 0) {
        // places inside the experts' segments, 64 slots at a time: a ballot for each bit of the expert's number finds the
        // slots of the same one
        const unsigned long long below = lane == 0 ? 0ull : ~0ull >> (64 - lane);
        for (int g = 0; g < N; g += 64) {
            const bool live = g + lane < N;
            const int e = live ? s_idx[g + lane] : 0;
            unsigned long long same = __ballot(live);
#pragma unroll
            for (int b = 0; b < 6; b++) {
                const unsigned long long m = __ballot((e >> b) & 1);
                same &= ((e >> b) & 1) ? m : ~m;
            }
            const int rank = __popcll(same & below);
            int at = 0;
            if (live) at = s_next[e] + rank;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (live) {
                if (rank == 0) s_next[e] = at + __popcll(same);
                s_pos[g + lane] = at;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        const int cnt = s_next[lane];  // 0 for lanes >= E
        int inc = cnt;
#pragma unroll
        for (int dlt = 1; dlt < 64; dlt <<= 1) {
            const int v = __shfl_up(inc, dlt, 64);
            if (lane >= dlt) inc += v;
        }
        __builtin_amdgcn_wave_barrier();
        s_next[lane] = inc - cnt;
        if (lane < f.E) {
            f.counts[lane] = cnt;
            f.offsets[lane] = inc - cnt;
        }
        if (lane == f.E - 1) f.offsets[f.E] = inc;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < N; p += blockDim.x) {
        const int pos = s_next[s_idx[p]] + s_pos[p];
        f.perm[pos] = p;
        f.inv_perm[p] = pos;
    }
}

int moe_i8_front_launch(const I8Front& f, moe_dtype_t x_dtype, hipStream_t s) {
    auto* kernel = x_dtype == MOE_BF16 ? i8_front_kernel<true> : i8_front_kernel<false>;
    // a wave routes a token at a time
    int threads = f.x ? i8_row_threads(f.d / 4) : 64;
    const int waves = f.T < 4 ? 4 : f.T < 16 ? f.T : 16;
    threads = threads < 64 * waves ? 64 * waves : threads;
    hipLaunchKernelGGL(kernel, dim3(f.x ? f.T + 1 : 1), dim3(threads), 0, s, f);
    return moe_launch_status();
}

template <bool BF16>
__global__ __launch_bounds__(256) void i8_rows_back_kernel(const unsigned* __restrict__ codes, const float* __restrict__ scales,
                                                           int T, int K4, void* __restrict__ x) {
    each_row(blockIdx.y, gridDim.y, T, [&](int t) __attribute__((always_inline)) {
        const float s = scales[t];
        for (int c = blockIdx.x * 256 + threadIdx.x; c < K4; c += gridDim.x * 256) {
            const size_t at = (size_t)t * K4 + c;
            const int q = (int)codes[at];
            const float4 v = make_float4((float)(q << 24 >> 24) * s, (float)(q << 16 >> 24) * s, (float)(q << 8 >> 24) * s,
                                         (float)(q >> 24) * s);
            if (BF16) {
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                ((bf16x4*)x)[at] = bf16x4{(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
            } else {
                ((float4*)x)[at] = v;
            }
        }
    });
}

int moe_i8_rows_back_launch(const int8_t* codes, const float* scales, int T, int K, void* x, moe_dtype_t x_dtype,
                            hipStream_t s) {
    const int K4 = K / 4;
    const dim3 grid((unsigned)((K4 + 1023) / 1024), (unsigned)(T < 65535 ? T : 65535));
    auto* kernel = x_dtype == MOE_BF16 ? i8_rows_back_kernel<true> : i8_rows_back_kernel<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const unsigned*)codes, scales, T, K4, x);
    return moe_launch_status();
}

// ------------------------------------------------------------------ matrices ----
// W [K,C] has its channels along the rows and its codes along the reduction, so both directions are transpositions.
//
// To codes: a workgroup takes the channels of 64 bytes of a row and all of K.  A thread takes V neighbouring channels of 16
// consecutive indices at a time, all requested at once and, up to HOLD times, kept in registers between the largest
// magnitudes and the codes: such matrices are read once.  The others are read again, from the last-level cache.  The
// two halves of a 128-byte line go to workgroups of one XCD.  Codes leave as 16 bytes a channel, 128 bytes and more of a
// channel side by side.
// Threads and bytes of a row, 8 x 4096 x 14336 in bf16 / in fp32, us: 512 and 64 454 / 701, 512 and 32 475 / 807, 1024 and 64 534 / 660,
// 1024 and 32 506 / 723, 512 and 128 508 / 688 (floor 275 / 458).  Scales and codes in two launches: below, for long reductions; in groups of
// experts that the last-level cache holds 530 to 630.  What bounds it is the access to narrow strips of long rows: a plain
// read of strips of 64 / 128 / 256 bytes runs at 4.1 / 5.5 / 6.1 TB/s.
#define I8_QT 512
#define I8_SEG 64
#define I8_SIDE (128 / I8_SEG)  // strips of a line, on one XCD
template <bool BF16, int V>
struct I8Quant {
    static constexpr int LC = I8_SEG / (V * (BF16 ? 2 : 4));  // lanes across the channels
    static constexpr int RG = I8_QT / LC;                 // groups of 16 indices of a round
    static constexpr int HOLD = BF16 && V < 4 ? 4 : 2;
    static constexpr int BYTES = V * (BF16 ? 2 : 4);      // of a thread's channels in a row
    typedef std::conditional_t<BYTES == 8, uint2, std::conditional_t<BYTES == 4, unsigned, uint16_t>> Word;
    struct Elems {
        Word word;
        __device__ __forceinline__ float at(int n) const {
            unsigned u;
            if constexpr (BYTES == 8) u = BF16 ? (n < 2 ? word.x : word.y) : n == 0 ? word.x : word.y;
            else u = word;
            if constexpr (BF16) return __uint_as_float((n & 1) ? u & 0xFFFF0000u : u << 16);
            else return __uint_as_float(u);
        }
    };
    // sixteen rows of V channels from element `at` on
    static __device__ __forceinline__ void load(const void* w, size_t at, int C, Elems (&v)[16]) {
        const char* p = (const char*)w + at * (BF16 ? 2 : 4);
        const size_t step = (size_t)C * (BF16 ? 2 : 4);
#pragma unroll
        for (int i = 0; i < 16; i++) v[i].word = *(const Word*)(p + i * step);
    }
};

template <bool BF16, int V>
__global__ __launch_bounds__(I8_QT) void i8_quantize_kernel(const void* __restrict__ w, int K, int C, int strips,
                                                            int8_t* __restrict__ codes, float* __restrict__ scales) {
    typedef I8Quant<BF16, V> Q;
    constexpr int LC = Q::LC, HOLD = Q::HOLD;
    __shared__ unsigned s_top[I8_QT / 64][LC * V];
    const size_t e = blockIdx.y;
    const int strip = (blockIdx.x & ~(8 * I8_SIDE - 1)) + (blockIdx.x & 7) * I8_SIDE + ((blockIdx.x >> 3) & (I8_SIDE - 1));
    if (strip >= strips) return;
    const int cl = threadIdx.x % LC, rg0 = threadIdx.x / LC, wave = threadIdx.x >> 6;
    const int c0 = (strip * LC + cl) * V;
    const int c = c0 < C ? c0 : C - V;  // (C is a multiple of V)
    const size_t base = e * K * C + c;
    const int groups = K / 16;
    typename Q::Elems v[HOLD][16];
    unsigned top[V];
#pragma unroll
    for (int n = 0; n < V; n++) top[n] = 0u;
    auto raise = [&](const typename Q::Elems (&u)[16]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; i++)
#pragma unroll
            for (int n = 0; n < V; n++) {
                const unsigned o = __float_as_uint(u[i].at(n)) & 0x7FFFFFFFu;
                top[n] = top[n] > o ? top[n] : o;
            }
    };
#pragma unroll
    for (int h = 0; h < HOLD; h++)
        if (rg0 + h * Q::RG < groups) Q::load(w, base + (size_t)(rg0 + h * Q::RG) * 16 * C, C, v[h]);
#pragma unroll
    for (int h = 0; h < HOLD; h++)
        if (rg0 + h * Q::RG < groups) raise(v[h]);
    for (int g = rg0 + HOLD * Q::RG; g < groups; g += Q::RG) {
        typename Q::Elems u[16];
        Q::load(w, base + (size_t)g * 16 * C, C, u);
        raise(u);
    }
#pragma unroll
    for (int n = 0; n < V; n++) {
#pragma unroll
        for (int m = LC; m < 64; m <<= 1) {
            const unsigned o = (unsigned)__shfl_xor((int)top[n], m, 64);
            top[n] = top[n] > o ? top[n] : o;
        }
        if ((threadIdx.x & 63) < LC) s_top[wave][cl * V + n] = top[n];
    }
    __syncthreads();
    float scale[V];
#pragma unroll
    for (int n = 0; n < V; n++) {
        unsigned t = 0u;
        for (int i = 0; i < I8_QT / 64; i++) t = t > s_top[i][cl * V + n] ? t : s_top[i][cl * V + n];
        scale[n] = i8_scale(t);
        if (rg0 == 0 && c0 < C) scales[e * C + c + n] = scale[n];
    }
    if (c0 >= C) return;
    auto put = [&](int g, const typename Q::Elems (&u)[16]) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < V; n++) {
            const I8Coder code(scale[n]);
            u32x4_t q;
#pragma unroll
            for (int i = 0; i < 4; i++)
                q[i] = code(make_float4(u[4 * i].at(n), u[4 * i + 1].at(n), u[4 * i + 2].at(n), u[4 * i + 3].at(n)));
            *(u32x4_t*)(codes + (e * C + c + n) * K + (size_t)g * 16) = q;
        }
    };
#pragma unroll
    for (int h = 0; h < HOLD; h++)
        if (rg0 + h * Q::RG < groups) put(rg0 + h * Q::RG, v[h]);
    for (int g = rg0 + HOLD * Q::RG; g < groups; g += Q::RG) {
        typename Q::Elems u[16];
        Q::load(w, base + (size_t)g * 16 * C, C, u);
        put(g, u);
    }
}

// Long reductions in two launches.  The scales alone: a workgroup takes the channels of SEG bytes of a row and all of K.
template <bool BF16, int V, int SEG>
__global__ __launch_bounds__(I8_QT) void i8_scales_kernel(const void* __restrict__ w, int K, int C, float* __restrict__ scales) {
    typedef I8Quant<BF16, V> Q;
    constexpr int LC = SEG / Q::BYTES, RG = I8_QT / LC, HOLD = 2;
    __shared__ unsigned s_top[RG][LC * V];
    const size_t e = blockIdx.y;
    const int cl = threadIdx.x % LC, rg = threadIdx.x / LC, groups = K / 16;
    const int c0 = (blockIdx.x * LC + cl) * V, c = c0 < C ? c0 : C - V;  // (C is a multiple of V)
    const size_t base = e * K * C + c;
    unsigned top[V];
#pragma unroll
    for (int n = 0; n < V; n++) top[n] = 0u;
    for (int g = rg; g < groups; g += HOLD * RG) {
        typename Q::Elems v[HOLD][16];
#pragma unroll
        for (int h = 0; h < HOLD; h++)  // (past the end: the last again)
            Q::load(w, base + (size_t)(g + h * RG < groups ? g + h * RG : groups - 1) * 16 * C, C, v[h]);
#pragma unroll
        for (int h = 0; h < HOLD; h++)
#pragma unroll
            for (int i = 0; i < 16; i++)
#pragma unroll
                for (int n = 0; n < V; n++) {
                    const unsigned o = __float_as_uint(v[h][i].at(n)) & 0x7FFFFFFFu;
                    top[n] = top[n] > o ? top[n] : o;
                }
    }
#pragma unroll
    for (int n = 0; n < V; n++) s_top[rg][cl * V + n] = top[n];
    __syncthreads();
    const int ch = blockIdx.x * (LC * V) + threadIdx.x;
    if (threadIdx.x >= LC * V || ch >= C) return;
    unsigned t = 0u;
    for (int i = 0; i < RG; i++) t = t > s_top[i][threadIdx.x] ? t : s_top[i][threadIdx.x];
    scales[e * C + ch] = i8_scale(t);
}

// The codes by the scales: a tile of 64 channels by 256 indices through LDS.  Neighbouring workgroups take the tiles of the same
// channels: those of the same indices would write lines a channel's row apart, 4096 bytes in K = 4096, which share
// memory channels (8 x 4096 x 14336 in bf16: 385 us that way, 300 this way).
#define I8_CODE_K 256
#define I8_CODE_C 64
template <bool BF16, int V>
__global__ __launch_bounds__(512) void i8_codes_kernel(const void* __restrict__ w, const float* __restrict__ scales, int K, int C,
                                                       int8_t* __restrict__ codes) {
    constexpr int LC = I8_CODE_C / V, RG = 512 / LC;
    __shared__ __align__(16) unsigned s_q[I8_CODE_C][I8_CODE_K / 4 + 1];
    const size_t e = blockIdx.z;
    const int c0 = (int)blockIdx.y * I8_CODE_C, k0 = (int)blockIdx.x * I8_CODE_K;
    const int kn = K - k0 < I8_CODE_K ? K - k0 : I8_CODE_K;
    const int cl = threadIdx.x % LC, rg = threadIdx.x / LC;
    const int cc = c0 + cl * V, c = cc < C ? cc : C - V;  // (C is a multiple of V)
    typedef std::conditional_t<BF16, uint16_t, float> T;
    typedef T Vec __attribute__((ext_vector_type(V)));
    constexpr int R = I8_CODE_K / 4 / RG;  // groups of four indices of a thread
    Vec v[R][4];
    const T* p = (const T*)w + (e * K + k0) * C + c;
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int k = (rg + r * RG) * 4 + i;
            v[r][i] = *(const Vec*)(p + (size_t)(k < kn ? k : kn - 1) * C);
        }
#pragma unroll
    for (int n = 0; n < V; n++) {
        const I8Coder code(scales[e * C + c + n]);
#pragma unroll
        for (int r = 0; r < R; r++) {
            float f[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if constexpr (BF16) f[i] = __uint_as_float((unsigned)v[r][i][n] << 16);
                else f[i] = v[r][i][n];
            }
            s_q[cl * V + n][rg + r * RG] = code(make_float4(f[0], f[1], f[2], f[3]));
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < I8_CODE_C * (I8_CODE_K / 16) / 512; i++) {
        const int at = threadIdx.x + i * 512, ch = at / (I8_CODE_K / 16), b = at % (I8_CODE_K / 16);
        if (c0 + ch >= C || b * 16 >= kn) continue;
        u32x4_t q;
#pragma unroll
        for (int j = 0; j < 4; j++) q[j] = s_q[ch][b * 4 + j];
        *(u32x4_t*)(codes + (e * C + c0 + ch) * K + k0 + b * 16) = q;
    }
}

template <bool BF16, int V, int SEG>
static void i8_scales_go(const void* w, int E, int K, int C, float* scales, hipStream_t s) {
    constexpr int wide = SEG / (BF16 ? 2 : 4);
    hipLaunchKernelGGL((i8_scales_kernel<BF16, V, SEG>), dim3((unsigned)((C + wide - 1) / wide), (unsigned)E), dim3(I8_QT), 0, s, w, K, C, scales);
}
template <bool BF16, int V>
static void i8_scales_pick(const void* w, int E, int K, int C, float* scales, hipStream_t s) {
    // wide strips read at 5.2 TB/s, strips of 64 bytes at 4.0; but there have to be enough of them
    if ((long long)E * C * (BF16 ? 2 : 4) >= 128 * 256) i8_scales_go<BF16, V, 256>(w, E, K, C, scales, s);
    else i8_scales_go<BF16, V, 64>(w, E, K, C, scales, s);
}
template <bool BF16, int V>
static void i8_codes_go(const void* w, const float* scales, int E, int K, int C, int8_t* codes, hipStream_t s) {
    const dim3 grid((unsigned)((K + I8_CODE_K - 1) / I8_CODE_K), (unsigned)((C + I8_CODE_C - 1) / I8_CODE_C), (unsigned)E);
    hipLaunchKernelGGL((i8_codes_kernel<BF16, V>), grid, dim3(512), 0, s, w, scales, K, C, codes);
}

int moe_i8_quantize_launch(const void* w, moe_dtype_t w_dtype, int E, int K, int C, int8_t* codes, float* scales,
                           hipStream_t s) {
    const bool bf16 = w_dtype == MOE_BF16;
    const int V = bf16 && C % 4 == 0 ? 4 : C % 2 == 0 ? 2 : 1;
    // One launch keeps 1024 or 2048 indices of a channel in registers and reads the others twice, in narrow strips: one / two
    // launches 8 x 4096 x 14336 in bf16 461 / 477 us, in fp32 715 / 761, 4 x 6144 x 4096 118 / 98 and 167 / 159, 4 x 14336 x 4096
    // 333 / 258 and 470 / 398, 14336 x 1024 131 / 46, 4 x 4096 x 4095 102 / 99.
    if (K > 4096) {
        if (bf16) V == 4 ? i8_scales_pick<true, 4>(w, E, K, C, scales, s) : V == 2 ? i8_scales_pick<true, 2>(w, E, K, C, scales, s)
                                                                                    : i8_scales_pick<true, 1>(w, E, K, C, scales, s);
        else V == 2 ? i8_scales_pick<false, 2>(w, E, K, C, scales, s) : i8_scales_pick<false, 1>(w, E, K, C, scales, s);
        if (bf16) C % 4 == 0 ? i8_codes_go<true, 4>(w, scales, E, K, C, codes, s) : i8_codes_go<true, 1>(w, scales, E, K, C, codes, s);
        else C % 4 == 0 ? i8_codes_go<false, 4>(w, scales, E, K, C, codes, s) : i8_codes_go<false, 1>(w, scales, E, K, C, codes, s);
        return moe_launch_status();
    }
    const int wide = I8_SEG / (bf16 ? 2 : 4), strips = (C + wide - 1) / wide;
    auto* kernel = bf16 ? (V == 4 ? i8_quantize_kernel<true, 4> : V == 2 ? i8_quantize_kernel<true, 2> : i8_quantize_kernel<true, 1>)
                        : (V == 2 ? i8_quantize_kernel<false, 2> : i8_quantize_kernel<false, 1>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(strips + 8 * I8_SIDE - 1) & ~(8u * I8_SIDE - 1), (unsigned)E), dim3(I8_QT), 0, s, w, K, C, strips, codes, scales);
    return moe_launch_status();
}

// From codes: a tile of 64 channels by 256 indices through LDS.
#define I8_CV_C 64
#define I8_CV_K 256
#define I8_CV_PAD 4  // bytes: a channel's row of the tile starts in another bank than its neighbour's
template <bool BF16>
__global__ __launch_bounds__(1024) void i8_dequantize_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales,
                                                             int K, int C, int ctiles, void* __restrict__ w) {
    __shared__ __align__(16) unsigned char s_q[I8_CV_C][I8_CV_K + I8_CV_PAD];
    const size_t e = blockIdx.x / ctiles;
    const int c0 = (int)(blockIdx.x % ctiles) * I8_CV_C, k0 = (int)blockIdx.y * I8_CV_K;
    const int kn = K - k0 < I8_CV_K ? K - k0 : I8_CV_K;
    const int cc = threadIdx.x >> 4, b = (threadIdx.x & 15) * 16;
    if (c0 + cc < C && b < kn) {
        const u32x4_t v = *(const u32x4_t*)(codes + (e * C + c0 + cc) * K + k0 + b);
        unsigned* p = (unsigned*)&s_q[cc][b];
#pragma unroll
        for (int i = 0; i < 4; i++) p[i] = v[i];
    }
    __syncthreads();
    const int cl = threadIdx.x & 63, kg = threadIdx.x >> 6;
    if (c0 + cl >= C) return;
    const float s = scales[e * C + c0 + cl];
    for (int k = kg * 4; k < kn; k += 64) {
        const int q = *(const int*)&s_q[cl][k];
        const float v[4] = {(float)(q << 24 >> 24) * s, (float)(q << 16 >> 24) * s, (float)(q << 8 >> 24) * s, (float)(q >> 24) * s};
        const size_t at = (e * K + k0 + k) * C + c0 + cl;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (BF16) ((__bf16*)w)[at + (size_t)i * C] = (__bf16)v[i];
            else ((float*)w)[at + (size_t)i * C] = v[i];
        }
    }
}

int moe_i8_dequantize_launch(const int8_t* codes, const float* scales, int E, int K, int C, void* w, moe_dtype_t w_dtype,
                             hipStream_t s) {
    const int ctiles = (C + I8_CV_C - 1) / I8_CV_C;
    const dim3 grid((unsigned)(E * ctiles), (unsigned)((K + I8_CV_K - 1) / I8_CV_K));
    auto* kernel = w_dtype == MOE_BF16 ? i8_dequantize_kernel<true> : i8_dequantize_kernel<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(1024), 0, s, codes, scales, K, C, ctiles, w);
    return moe_launch_status();
}

// -------------------------------------------------------------------- handle ----
// codes [E][C][K] -> fragments [E][C/16][nmat][K/64], this launch fills matrix slot `mat`, and the scales beside
// them.  One thread writes one 16-byte chunk, a wave a fragment: sixteen features' 64 bytes.
__global__ __launch_bounds__(256) void i8_pack_kernel(const int8_t* __restrict__ src, const float* __restrict__ scales,
                                                      u32x4_t* __restrict__ dst, float* __restrict__ dscale, int E, int K, int C,
                                                      int nmat, int mat) {
    const size_t KS = (size_t)i8_frags(K), total = (size_t)E * C * KS * 4;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
        const int l = (int)(i & 63), j = l >> 4;
        const size_t ks = (i >> 6) % KS, b = (i >> 6) / KS, c = b * 16 + (l & 15);  // feature, counted through the experts
        const u32x4_t v = *(const u32x4_t*)(src + c * K + ks * I8_FRAG_K + 16 * j);
        dst[((b * nmat + mat) * KS + ks) * 64 + l] = v;
        if (ks == 0 && j == 0) dscale[(b * nmat + mat) * 16 + l] = scales[c];
    }
}

int moe_i8_pack_impl(const int8_t* const codes[3], const float* const scales[3], int E, int d, int f, moe_weights** out,
                     hipStream_t s) {
    moe_weights* W = new (std::nothrow) moe_weights();
    if (!W) return MOE_ERR_HIP;
    W->E = E;
    W->d = d;
    W->f = f;
    W->dtype = MOE_INT8;
    if (hipGetDevice(&W->device) != hipSuccess) {
        (void)hipGetLastError();
        delete W;
        return MOE_ERR_HIP;
    }
    const size_t n = (size_t)E * d * f;
    // (the persistent loop's steps come in fours and read up to three fragments behind the last, times zeros)
    const size_t bytes[4] = {2 * n + 3 * 1024, n + 3 * 1024, (size_t)E * 2 * f * 4, (size_t)E * d * 4};
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
        hipLaunchKernelGGL(i8_pack_kernel, dim3(4096), dim3(256), 0, s, codes[m], scales[m], (u32x4_t*)(up ? W->w13 : W->w2),
                           (float*)(up ? W->s13 : W->s2), E, up ? d : f, up ? f : d, up ? 2 : 1, up ? m : 0);
    }
    if (moe_launch_status() != MOE_OK) {
        for (int i = 0; i < 4; i++) (void)hipFree(*dst[i]);
        delete W;
        return MOE_ERR_HIP;
    }
    *out = W;
    return MOE_OK;
}
