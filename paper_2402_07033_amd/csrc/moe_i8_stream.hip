// Products of a few 8-bit rows with 8-bit matrices: bound by reading each matrix once, a byte per weight.
//
// A workgroup takes up to 16 rows of one expert and FB fragment rows (16 channels each) of its matrix for the whole
// reduction, which its NW waves share; a wave requests 8 steps of 64 indices at once (FB KiB of weights a step), so the
// loads in flight are many.  The waves' sums meet in LDS: sums of integers, the same bits in any order.  Workgroups are
// short and several run on a CU, one's join under the others' loads.
#include <atomic>

#include "moe_frag_pack.h"
#include "moe_i8.h"
#include "moe_i8_value.h"

#define I8S_U 8  // steps requested at once

struct I8StreamArgs {
    I8Product p;
    int NR;   // fragment rows of an expert's matrix
    int KS;   // steps
    int FG;   // groups of FB fragment rows
};

template <int FB, int NW, bool PACKED, bool GATED, bool ONCE>
__global__ __launch_bounds__(64 * NW) void i8_stream_kernel(I8StreamArgs a) {
    constexpr int U = I8S_U;
    __shared__ i32x4_t s_sum[NW][FB][64];
    const I8Product& p = a.p;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    SegInfo si = {0, 0, p.N, 0};
    const int tile = blockIdx.x / a.FG, fr0 = blockIdx.x % a.FG * FB;
    if (p.offsets && !gg_find_block(p.offsets, p.E, p.N, tile, lane, si)) return;
    const int r0 = (tile - si.bbase) * 16, rows = si.rows - r0 < 16 ? si.rows - r0 : 16;

    // operand of a matrix instruction: row (channel) l % 16, indices 16 * (l / 16) .. +15 of the step
    const int rl = lane & 15, cq = lane >> 4, K = p.K;
    const size_t row = si.row0 + r0 + (rl < rows ? rl : rows - 1);
    const int src = p.perm ? p.perm[row] / p.k : (int)row;
    const int8_t* xp = p.x + (size_t)src * K;
    const int8_t* wp[FB];
#pragma unroll
    for (int r = 0; r < FB; r++) {
        if (PACKED) {
            const int fr = fr0 + r < a.NR ? fr0 + r : a.NR - 1;
            wp[r] = p.w + ((size_t)si.e * a.NR + fr) * a.KS * 1024 + lane * 16;
        } else {
            const int c = (fr0 + r) * 16 + rl < p.C ? (fr0 + r) * 16 + rl : p.C - 1;
            wp[r] = p.w + ((size_t)si.e * p.C + c) * K;
        }
    }
    i32x4_t acc[FB];
#pragma unroll
    for (int r = 0; r < FB; r++) acc[r] = i32x4_t{0, 0, 0, 0};
    const int k_lo = wave * a.KS / NW, k_hi = (wave + 1) * a.KS / NW;
    for (int k0 = k_lo; k0 < k_hi; k0 += U) {
        i32x4_t x[U], w[U][FB];
        // (the rows first: they come from a cache, and requests are answered in order)
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int at = (k0 + u) * I8_FRAG_K + cq * 16;
            x[u] = i32x4_t{0, 0, 0, 0};
            if (k0 + u < k_hi && at < K) x[u] = *(const i32x4_t*)(xp + at);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (k0 + u >= k_hi) break;
            int at = (k0 + u) * I8_FRAG_K + cq * 16;
            at = at < K ? at : K - 16;  // (times x's zeros)
#pragma unroll
            for (int r = 0; r < FB; r++)
            {
                const i32x4_t* q = (const i32x4_t*)(wp[r] + (PACKED ? (size_t)(k0 + u) * 1024 : (size_t)at));
                w[u][r] = ONCE ? __builtin_nontemporal_load(q) : *q;
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (k0 + u >= k_hi) break;
#pragma unroll
            for (int r = 0; r < FB; r++) acc[r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][r], x[u], acc[r], 0, 0, 0);
        }
    }
#pragma unroll
    for (int r = 0; r < FB; r++) s_sum[wave][r][lane] = acc[r];
    __syncthreads();
    if (wave >= FB / (GATED ? 2 : 1)) return;
    auto sum = [&](int r) __attribute__((always_inline)) {
        i32x4_t v = s_sum[0][r][lane];
#pragma unroll
        for (int i = 1; i < NW; i++) v += s_sum[i][r][lane];
        return v;
    };
    if (rl >= rows) return;
    const float sx = p.xs[src];
    if (GATED) {
        if (fr0 + 2 * wave >= a.NR) return;
        const unsigned top = i8_put_gated(p, si.e, a.NR, fr0 + 2 * wave, cq, row, sx, sum(2 * wave), sum(2 * wave + 1));
        if (p.ytop) {
            unsigned o = (unsigned)__shfl_xor((int)top, 16, 64);
            o = top > o ? top : o;
            const unsigned q = (unsigned)__shfl_xor((int)o, 32, 64);
            if (cq == 0) p.ytop[row * (a.NR / 2) + fr0 / 2 + wave] = q > o ? q : o;
        }
    } else {
        i8_put(p, si.e, (fr0 + wave) * 16 + 4 * cq, row, sx, sum(wave));
    }
}

// The second projection of at most four rows in all (a token or two): a workgroup takes 16 channels for every row, so that
// nothing is left to add and the gate-weighted sum of a token's rows ends the layer here.  It brings the rows of h to 8
// bits for itself, in LDS, under its first requests of weights: their largest magnitudes come from the first projection, one
// per 16 channels.  A wave takes one expert's rows and a part of the reduction.
#define I8D_ROWS 4
#define I8D_WAVES 16
#define I8D_LDS (144 * 1024)

struct I8DownArgs {
    const float* h;           // [N,K]
    const unsigned* htop;     // [N][K/16]
    const int32_t* offsets;
    int E, N, K, C, KS;
    const int8_t* w;
    const float* ws;
    float* yg;                // [N,C] or null
    void* y;                  // [T,C] or null: with the rows' places and weights
    bool y_bf16;
    const int32_t* inv_perm;
    const float* weights;
    int T, k;
};

__global__ __launch_bounds__(64 * I8D_WAVES) void i8_down_small_kernel(I8DownArgs a) {
    constexpr int U = 8;
    __shared__ i32x4_t s_sum[I8D_WAVES][64];
    __shared__ float s_scale[I8D_ROWS], s_val[I8D_ROWS][16];
    __shared__ unsigned s_top[I8D_WAVES];
    extern __shared__ __align__(16) unsigned char s_x[];  // [N][K + 16]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int K = a.K, stride = K + 16, fb = blockIdx.x;
    // the experts that have rows, four at most, each with 1 / n of the waves
    int lo, cnt;
    gg_segment_of_lane(a.offsets, a.E, a.N, lane, lo, cnt);
    unsigned long long used = __ballot(cnt > 0);
    const int n = __popcll(used), parts = I8D_WAVES / (n > 0 ? n : 1);
    if (n == 0) return;
    const int mine = wave / parts < n ? wave / parts : n - 1, part = wave - mine * parts;
    for (int i = 0; i < mine; i++) used &= used - 1;
    const int e = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(used));
    const int row0 = __builtin_amdgcn_readlane(lo, e), rows = __builtin_amdgcn_readlane(cnt, e);
    const bool idle = part >= parts;
    const int k_lo = idle ? a.KS : part * a.KS / parts, k_hi = idle ? a.KS : (part + 1) * a.KS / parts;
    const int8_t* wp = a.w + ((size_t)e * (a.C / 16) + fb) * a.KS * 1024 + lane * 16;
    // The rows' largest magnitudes and their values: 1 / N of the waves a row, everything requested at once, the weights
    // last (requests are answered in order).
    constexpr int V = 7;  // chunks of four values of a thread at a time
    const int wpr = I8D_WAVES / a.N, hr = wave / wpr < a.N ? wave / wpr : a.N - 1, span = 64 * wpr;
    const int ht = (wave - hr * wpr) * 64 + lane;  // this thread's place among the row's; >= span: none
    const bool none = ht >= span;
    unsigned top = 0u;
    if (!none) {
        const unsigned* tp = a.htop + (size_t)hr * (K / 16);
#pragma unroll 4
        for (int i = ht; i < K / 16; i += span) {
            const unsigned v = tp[i];
            top = top > v ? top : v;
        }
    }
    const float4* hp = (const float4*)a.h + (size_t)hr * (K / 4);
    float4 v[V];
    auto fetch = [&](int at) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < V; i++)
            if (at + i * span < K / 4) v[i] = hp[at + i * span];
    };
    if (!none) fetch(ht);
    i32x4_t w[2][U];
    auto request = [&](int k, i32x4_t (&to)[U]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; u++)  // (past the end: the last again, so that every chunk counts the same requests)
            to[u] = __builtin_nontemporal_load((const i32x4_t*)(wp + (size_t)(k + u < k_hi ? k + u : a.KS - 1) * 1024));
    };
    request(k_lo, w[0]);
    request(k_lo + U, w[1]);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const unsigned o = (unsigned)__shfl_xor((int)top, m, 64);
        top = top > o ? top : o;
    }
    if (lane == 0) s_top[wave] = none ? 0u : top;
    __syncthreads();
    if (wave < a.N) {
        unsigned t = 0u;
        for (int i = 0; i < wpr; i++) t = t > s_top[wave * wpr + i] ? t : s_top[wave * wpr + i];
        if (lane == 0) s_scale[wave] = i8_scale(t);
    }
    __syncthreads();
    if (!none) {
        const I8Coder code(s_scale[hr]);
        for (int at = ht; at < K / 4; at += V * span) {
            if (at > ht) fetch(at);
#pragma unroll
            for (int i = 0; i < V; i++)
                if (at + i * span < K / 4)
                    *(unsigned*)(s_x + hr * stride + (at + i * span) * 4) = code(v[i]);
        }
    }
    __syncthreads();
    const int rl = lane & 15, cq = lane >> 4;
    const unsigned char* xp = s_x + (row0 + (rl < rows ? rl : 0)) * stride + cq * 16;
    i32x4_t acc = {0, 0, 0, 0};
    auto multiply = [&](int k, const i32x4_t (&with)[U]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (k + u >= k_hi) break;
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(with[u], *(const i32x4_t*)(xp + (k + u) * I8_FRAG_K), acc, 0, 0, 0);
        }
    };
    int k = k_lo;
    for (; k + 2 * U < k_hi; k += 2 * U) {
        multiply(k, w[0]);
        request(k + 2 * U, w[0]);
        multiply(k + U, w[1]);
        request(k + 3 * U, w[1]);
    }
    multiply(k, w[0]);
    multiply(k + U, w[1]);
    s_sum[wave][lane] = acc;
    __syncthreads();
    // the first wave of every expert adds its parts
    if (!idle && part == 0 && rl < rows) {
        for (int q = 1; q < parts; q++) acc += s_sum[wave + q][lane];
        const int row = row0 + rl;
        const float sx = s_scale[row];
        const float4 sw = *(const float4*)(a.ws + (size_t)e * a.C + fb * 16 + 4 * cq);
        const float4 v = make_float4(i8_value(acc[0], sx, sw.x), i8_value(acc[1], sx, sw.y), i8_value(acc[2], sx, sw.z),
                                     i8_value(acc[3], sx, sw.w));
        *(float4*)&s_val[row][4 * cq] = v;
        if (a.yg) *(float4*)(a.yg + (size_t)row * a.C + fb * 16 + 4 * cq) = v;
    }
    if (!a.y) return;
    __syncthreads();
    if (threadIdx.x >= (unsigned)a.T * 16) return;
    const int t = threadIdx.x >> 4, c = threadIdx.x & 15;
    float y = 0.f;
    for (int j = 0; j < a.k; j++) y = __builtin_fmaf(a.weights[t * a.k + j], s_val[a.inv_perm[t * a.k + j]][c], y);
    const size_t at = (size_t)t * a.C + fb * 16 + c;
    if (a.y_bf16) ((uint16_t*)a.y)[at] = (uint16_t)moe_bf16_rne(y);
    else ((float*)a.y)[at] = y;
}

// ------------------------------------------------------------------ host ----
template <int NW, bool PACKED, bool GATED>
static void i8_stream_go(I8StreamArgs& a, size_t tiles, hipStream_t s) {
    constexpr int FB = 2;
    a.FG = (a.NR + FB - 1) / FB;
    auto* kernel = moe_i8_streams(a.p, a.NR) ? i8_stream_kernel<FB, NW, PACKED, GATED, true> : i8_stream_kernel<FB, NW, PACKED, GATED, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles * a.FG)), dim3(64 * NW), 0, s, a);
}

// Waves of a workgroup by the reduction, which they share.  us with (channels, waves) (32, 4) / (32, 8) / (16, 8) / (16, 16): second
// projection of one token's two experts (f 14336) 22.3 / 20.2 / 20.4 / 21.4, of 39 experts with f 1408 23.5 / 29.1 / 30.3 / 60.4; first
// projections (32, 4) / (32, 8) / (64, 8): one token (d 4096) 38.1 / 39.7 / 45.5, 39 experts (d 2048) 40.1 / 47.1 / 41.8.
template <bool PACKED, bool GATED>
static void i8_stream_pick(I8StreamArgs& a, size_t tiles, hipStream_t s) {
    if (a.KS > 64) i8_stream_go<8, PACKED, GATED>(a, tiles, s);
    else i8_stream_go<4, PACKED, GATED>(a, tiles, s);
}

int moe_i8_stream_launch(const I8Product& p, hipStream_t s) {
    I8StreamArgs a = {};
    a.p = p;
    a.NR = p.gated ? 2 * (p.C / 16) : (p.C + 15) / 16;
    a.KS = i8_frags(p.K);
    const int used = p.N < p.E ? p.N : p.E;
    const size_t tiles = ((size_t)p.N + 15 * (size_t)used) / 16;
    if (p.gated) i8_stream_pick<true, true>(a, tiles, s);
    else if (p.packed) i8_stream_pick<true, false>(a, tiles, s);
    else i8_stream_pick<false, false>(a, tiles, s);
    return moe_launch_status();
}

bool moe_i8_down_small_serves(int N, int K) { return N <= I8D_ROWS && (size_t)N * (K + 16) <= I8D_LDS - 32 * 1024; }

int moe_i8_down_small_launch(const moe_weights* W, const float* h, const unsigned* htop, const int32_t* offsets, int N, float* yg,
                             const I8Combine* c, hipStream_t s) {
    static std::atomic<bool> ready[MOE_MAX_DEVICES];  // one-time permission for more than 64 KiB of LDS
    const int dev = moe_current_device();
    if (dev < 0) return MOE_ERR_HIP;
    if (!ready[dev].load(std::memory_order_acquire)) {
        MOE_HIP_TRY(hipFuncSetAttribute((const void*)i8_down_small_kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                                        I8D_LDS - 32 * 1024));
        ready[dev].store(true, std::memory_order_release);
    }
    I8DownArgs a = {};
    a.h = h;
    a.htop = htop;
    a.offsets = offsets;
    a.E = W->E;
    a.N = N;
    a.K = W->f;
    a.C = W->d;
    a.KS = i8_frags(W->f);
    a.w = (const int8_t*)W->w2;
    a.ws = (const float*)W->s2;
    a.yg = yg;
    if (c) {
        a.y = c->y;
        a.y_bf16 = c->y_bf16;
        a.inv_perm = c->inv_perm;
        a.weights = c->weights;
        a.T = c->T;
        a.k = c->k;
    }
    hipLaunchKernelGGL(i8_down_small_kernel, dim3((unsigned)(W->d / 16)), dim3(64 * I8D_WAVES), (size_t)N * (W->f + 16), s, a);
    return moe_launch_status();
}
