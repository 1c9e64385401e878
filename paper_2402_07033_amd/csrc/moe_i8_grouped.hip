// Expert FFN in 8 bits for many rows per expert: the grouped GEMM's persistent loop (moe_ffn_grouped.hip) on the integer matrix
// cores.  Per CU and step of 64 indices it moves and multiplies what the bf16 loop does per 32, so it needs half its steps.
//
//   pack   : rows' codes -> B-operand fragments [block of 16 rows][d/64], their scales [block][16]
//   up     : a = x.w1, b = x.w3, h = silu(a)*b in fp32, and per row the largest magnitude of every 32 channels
//   pack h : h to 8 bits as fragments [block][f/64]: the largest magnitudes are known, so h is read once
//   down   : yg = h.w2
#define GG_INT8
#include "moe_ffn_grouped.hip"

// One projection: the persistent GEMM and the fix-up of left-over tiles that were cut along the reduction.  r192: tiles of 192
// rows instead of 256.
template <bool UP>
int i8_gg_launch(gg_int8::GroupedArgs& a, bool r192, unsigned pgrid, hipStream_t s) {
    using namespace gg_int8;
    auto* kernel = r192 ? gg_gemm_kernel<UP, 12, 4, false, GG_U, GG_LA, GG_NS> : gg_gemm_kernel<UP, 16, 4, false, GG_U, GG_LA, GG_NS>;
    const int lds = GG_NS * (r192 ? 12 : 16) * 1024;
    static std::atomic<bool> ready[2][MOE_MAX_DEVICES];  // one-time permission for more than 64 KiB of LDS
    const int dev = moe_current_device();
    if (dev < 0) return MOE_ERR_HIP;
    if (!ready[r192][dev].load(std::memory_order_acquire)) {
        MOE_HIP_TRY(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        ready[r192][dev].store(true, std::memory_order_release);
    }
    hipLaunchKernelGGL(kernel, dim3(pgrid), dim3(GG_THREADS), lds, s, a);
    if (a.split) {
        auto* fix = r192 ? gg_fixup_kernel<UP, 12, 4, false> : gg_fixup_kernel<UP, 16, 4, false>;
        hipLaunchKernelGGL(fix, dim3(GG_FIX_GRID), dim3(256), 0, s, a, (int)(pgrid / 8), GG_U, GG_NS);
    }
    return moe_launch_status();
}

#ifdef GG_SECOND_PROJECTION
template int i8_gg_launch<false>(gg_int8::GroupedArgs&, bool, unsigned, hipStream_t);
#else
extern template int i8_gg_launch<false>(gg_int8::GroupedArgs&, bool, unsigned, hipStream_t);

// Codes [rows,K] -> fragments [block][KS] of the batched rows (row i is x[perm[i] / k] where perm is given), rows past an
// expert's last and indices past K zero; blockIdx.y: a part of the reduction.
#define I8G_PACK_KS 16
__global__ __launch_bounds__(256) void i8_gg_pack_kernel(const int8_t* __restrict__ x, const float* __restrict__ xs,
                                                         const int32_t* __restrict__ perm, int k,
                                                         const int32_t* __restrict__ offsets, int E, int N, int K, int KS,
                                                         u32x4_t* __restrict__ xp, float* __restrict__ xps) {
    SegInfo si;
    const int lane = threadIdx.x & 63, t = lane & 15;
    if (!gg_find_block(offsets, E, N, blockIdx.x, lane, si)) return;
    const int r = (blockIdx.x - si.bbase) * 16 + t;
    const bool live = r < si.rows;
    int src = live ? si.row0 + r : si.row0;
    if (perm) src = perm[src] / k;
    if (blockIdx.y == 0 && threadIdx.x < 16) xps[(size_t)blockIdx.x * 16 + t] = live ? xs[src] : 0.f;
    const int end = (blockIdx.y + 1) * I8G_PACK_KS < KS ? (blockIdx.y + 1) * I8G_PACK_KS : KS;
    for (int ks = blockIdx.y * I8G_PACK_KS + (threadIdx.x >> 6); ks < end; ks += 4) {
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (live && ks * 64 < K) v = *(const u32x4_t*)(x + (size_t)src * K + ks * 64 + (lane >> 4) * 16);
        xp[((size_t)blockIdx.x * KS + ks) * 64 + lane] = v;
    }
}

// h [N,K] fp32 with the largest magnitudes of 32 channels, top [K/32][N] -> fragments and scales.  Four loads of a wave are
// 16 rows of 256 bytes; their codes change hands in the wave's own LDS.
// h is read past the caches: it is larger than they are (8192 rows of 14336: 137 -> 125 us).
#define I8G_H_KS 32
__global__ __launch_bounds__(256) void i8_gg_pack_h_kernel(const float* __restrict__ h, const unsigned* __restrict__ top,
                                                           const int32_t* __restrict__ offsets, int E, int N, int K, int KS,
                                                           u32x4_t* __restrict__ hp, float* __restrict__ hps) {
    __shared__ unsigned s_top[16][16];
    __shared__ __align__(16) unsigned s_q[4][16][16 + 4];
    SegInfo si;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = threadIdx.x & 15;
    if (!gg_find_block(offsets, E, N, blockIdx.x, lane, si)) return;
    const int b0 = (blockIdx.x - si.bbase) * 16, rows = si.rows - b0;  // rows of the block, 16 and more: full
    const size_t row0 = (size_t)si.row0 + b0;
    unsigned m = 0u;
    if (t < rows) {
#pragma unroll 4
        for (int g = threadIdx.x >> 4; g < K / 32; g += 16) {
            const unsigned v = top[(size_t)g * N + row0 + t];
            m = m > v ? m : v;
        }
    }
    s_top[threadIdx.x >> 4][t] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; i++) m = m > s_top[i][t] ? m : s_top[i][t];
    const float scale = i8_scale(m);  // row t's
    if (blockIdx.y == 0 && threadIdx.x < 16) hps[(size_t)blockIdx.x * 16 + t] = scale;
    const int end = (blockIdx.y + 1) * I8G_H_KS < KS ? (blockIdx.y + 1) * I8G_H_KS : KS;
    for (int ks = blockIdx.y * I8G_H_KS + wave; ks < end; ks += 4) {
        float4 v[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {  // row 4i + lane / 16, four channels from 4 * t on
            const int r = 4 * i + (lane >> 4);
            f32x4_t u = {0.f, 0.f, 0.f, 0.f};
            if (r < rows && ks * 64 < K) u = __builtin_nontemporal_load((const f32x4_t*)(h + (row0 + r) * K + ks * 64 + 4 * t));
            v[i] = make_float4(u[0], u[1], u[2], u[3]);
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int r = 4 * i + (lane >> 4);
            const I8Coder code(__shfl(scale, r, 64));
            s_q[wave][r][t] = code(v[i]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const u32x4_t q = *(const u32x4_t*)&s_q[wave][t][4 * (lane >> 4)];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        hp[((size_t)blockIdx.x * KS + ks) * 64 + lane] = q;
    }
}

static inline size_t i8g_align256(size_t v) { return (v + 255) & ~(size_t)255; }

bool moe_i8_grouped_supported(int N, int E, int d, int f) {
    // Tiles of 256 channels; eight steps at least.  A reduction that is no multiple of 256 is filled up with zeros (64 experts,
    // d = 2048, f = 1408, six per token, against the tiles of moe_i8_gemm.hip: at 3952 tokens 434 us against 449, with skewed
    // routing 471 against 509; at 2200 tokens 314 against 279, skewed 331 against 382: the host does not know the routing,
    // and even counts are the rare ones).
    return d % 256 == 0 && f % 128 == 0 && d > 256 && f > 256;
}
// Steps of a reduction: groups of four, the last one's tokens filled with zeros.
static inline int i8g_steps(int K) { return (K + 255) / 256 * 4; }

// fragments and scales of the rows, h, its largest magnitudes, its fragments and scales, pieces of cut tiles
struct I8GroupedSpace {
    size_t xp, xps, h, top, hp, hps, part, bytes;
    int blocks;
};
static I8GroupedSpace i8_grouped_space(int N, int E, int d, int f) {
    I8GroupedSpace w;
    w.blocks = N / 16 + E;
    const size_t rows = (size_t)w.blocks * 16;
    w.xp = 0;
    w.xps = w.xp + i8g_align256(rows * i8g_steps(d) * 64);
    w.h = w.xps + i8g_align256(rows * 4);
    w.top = w.h + i8g_align256((size_t)N * f * 4);
    w.hp = w.top + i8g_align256((size_t)N * (f / 32) * 4);
    w.hps = w.hp + i8g_align256(rows * i8g_steps(f) * 64);
    w.part = w.hps + i8g_align256(rows * 4);
    w.bytes = w.part + (size_t)((moe_num_cus() + 7) / 8 * 8) * 2 * 256 * 256 * 4;
    return w;
}
size_t moe_i8_grouped_workspace(int N, int E, int d, int f) { return i8_grouped_space(N, E, d, f).bytes; }

// Tiles of 192 rows, as in bf16: experts of 97 .. 176 and 233 .. 256 rows on average.
static bool i8_r192(int N, int E) {
    const long long mean = ((long long)N + E - 1) / E;
    return mean <= GG_R192_MAX_ROWS || (mean >= GG_R192_MIN_ROWS2 && mean <= GG_R192_MAX_ROWS2);
}
int moe_i8_grouped_tile_rows(int N, int E) { return i8_r192(N, E) ? 192 : 256; }

int moe_i8_grouped_launch(const moe_weights* W, const int8_t* codes, const float* scales, const int32_t* perm, int k,
                          const int32_t* offsets, int N, void* ws, float* yg, hipStream_t s) {
    const int d = W->d, f = W->f, E = W->E;
    const I8GroupedSpace sp = i8_grouped_space(N, E, d, f);
    char* base = (char*)ws;
    const unsigned pgrid = (unsigned)((moe_num_cus() + 7) / 8 * 8);  // persistent: one per CU
    const bool r192 = i8_r192(N, E);
    hipLaunchKernelGGL(i8_gg_pack_kernel, dim3((unsigned)sp.blocks, (unsigned)((i8g_steps(d) + I8G_PACK_KS - 1) / I8G_PACK_KS)), dim3(256), 0, s,
                       codes, scales, perm, k, offsets, E, N, d, i8g_steps(d), (u32x4_t*)(base + sp.xp), (float*)(base + sp.xps));
    gg_int8::GroupedArgs a = {};
    a.offsets = offsets;
    a.E = E;
    a.N = N;
    a.part = (float*)(base + sp.part);
    a.wfrag = (const u32x4_t*)W->w13;
    a.bfrag = (const u32x4_t*)(base + sp.xp);
    a.out = base + sp.h;
    a.KS = i8g_steps(d);
    a.KS_w = d / 64;
    a.FR = f / 8;
    a.NT = a.FR / 16;
    a.C = f;
    a.split = gg_split_limit(true, a.KS, (int)(pgrid / 8));
    a.bscale = (const float*)(base + sp.xps);
    a.wscale = (const float*)W->s13;
    a.top = (unsigned*)(base + sp.top);
    int rc = i8_gg_launch<true>(a, r192, pgrid, s);
    if (rc != MOE_OK) return rc;
    moe_record_mid_event(s);
    hipLaunchKernelGGL(i8_gg_pack_h_kernel, dim3((unsigned)sp.blocks, (unsigned)((i8g_steps(f) + I8G_H_KS - 1) / I8G_H_KS)), dim3(256), 0, s,
                       (const float*)(base + sp.h), (const unsigned*)(base + sp.top), offsets, E, N, f,
                       i8g_steps(f), (u32x4_t*)(base + sp.hp), (float*)(base + sp.hps));
    a.wfrag = (const u32x4_t*)W->w2;
    a.bfrag = (const u32x4_t*)(base + sp.hp);
    a.out = yg;
    a.KS = i8g_steps(f);
    a.KS_w = f / 64;
    a.FR = d / 16;
    a.NT = a.FR / 16;
    a.C = d;
    a.split = gg_split_limit(false, a.KS, (int)(pgrid / 8));
    a.bscale = (const float*)(base + sp.hps);
    a.wscale = (const float*)W->s2;
    return i8_gg_launch<false>(a, r192, pgrid, s);
}
#endif  // GG_SECOND_PROJECTION
