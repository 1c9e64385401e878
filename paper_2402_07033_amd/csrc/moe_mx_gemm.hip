// Expert FFN over MXFP4 matrices for tens of rows per expert and prompts: a grouped GEMM on the
// bf16 matrix cores.
#include "moe_mx.h"
#include "moe_frag_pack.h"

#define MXG_RB 4  // 16-row blocks of a tile

// Rows as B operands: block b of 16 rows of an expert, [block][KS][4 j][64 lanes] 16-byte chunks,
// lane l of (ks, j): row l % 16, indices ks*128 + 32*(l / 16) + 8j .. +7 (moe_mx.h).  Rows past
// the expert's last and indices past K are zero.
template <bool BF16>
__global__ __launch_bounds__(256) void mx_rows_kernel(const void* __restrict__ x, const int32_t* __restrict__ perm, int k,
                                                      const int32_t* __restrict__ offsets, int E, int N, int K,
                                                      u32x4_t* __restrict__ xp, u32x4_t* __restrict__ hp, int f) {
    SegInfo si;
    if (!gg_find_block(offsets, E, N, blockIdx.x, threadIdx.x & 63, si)) return;
    const int KS = mx_frags(K);
    const int lane = threadIdx.x & 63;
    const int t = lane & 15, kq = lane >> 4;
    const int r = (blockIdx.x - si.bbase) * 16 + t;
    int src = si.row0 + r;
    if (perm && r < si.rows) src = perm[si.row0 + r] / k;
    for (int i = blockIdx.y * 4 + (threadIdx.x >> 6); i < KS * 4; i += 4 * gridDim.y) {
        const int k0 = (i >> 2) * MX_FRAG_K + kq * MX_BLOCK + (i & 3) * 8;
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (r < si.rows && k0 < K) {
            const size_t off = (size_t)src * K + k0;
            if (BF16) {
                v = *(const u32x4_t*)((const uint16_t*)x + off);
            } else {
                const float4 a = *(const float4*)((const float*)x + off);
                const float4 b = *(const float4*)((const float*)x + off + 4);
                v[0] = moe_pack_bf16x2(a.x, a.y);
                v[1] = moe_pack_bf16x2(a.z, a.w);
                v[2] = moe_pack_bf16x2(b.x, b.y);
                v[3] = moe_pack_bf16x2(b.z, b.w);
            }
        }
        xp[((size_t)blockIdx.x * KS * 4 + i) * 64 + lane] = v;
    }
    // the first projection does not reach the indices of h past f
    if (blockIdx.y == 0 && f % MX_FRAG_K && kq * MX_BLOCK >= f % MX_FRAG_K)
        hp[((size_t)blockIdx.x * mx_frags(f) * 4 + (mx_frags(f) - 1) * 4 + (threadIdx.x >> 6)) * 64 + lane] =
            u32x4_t{0u, 0u, 0u, 0u};
}

struct MxGemmArgs {
    const u32x4_t* wfrag;
    const unsigned* wscale;
    const u32x4_t* xp;
    uint16_t* hp;   // up: out
    float* yg;      // down: out
    const int32_t* offsets;
    int E, N, K, C, NB, KS, KW;
    int ftiles;
};

// Tile `t` of RB * 16 rows -> its segment; b: its first block inside the segment.
template <int RB>
__device__ __forceinline__ bool mx_find_tile(const int32_t* offsets, int E, int N, int tile, int lane, SegInfo& si, int& b) {
    int lo, rows;
    gg_segment_of_lane(offsets, E, N, lane, lo, rows);
    const int nb = (rows + 15) / 16, nt = (nb + RB - 1) / RB;
    int ib = nb, it = nt;
#pragma unroll
    for (int dlt = 1; dlt < 64; dlt <<= 1) {
        const int vb = __shfl_up(ib, dlt, 64), vt = __shfl_up(it, dlt, 64);
        if (lane >= dlt) {
            ib += vb;
            it += vt;
        }
    }
    const unsigned long long m = __ballot(tile >= it - nt && tile < it);
    if (m == 0ull) return false;
    const int e = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(m));
    si.e = e;
    si.row0 = __builtin_amdgcn_readlane(lo, e);
    si.rows = __builtin_amdgcn_readlane(rows, e);
    si.bbase = __builtin_amdgcn_readlane(ib - nb, e);
    b = (tile - __builtin_amdgcn_readlane(it - nt, e)) * RB;
    return true;
}

template <int NMAT, int NBU, int RB>
__global__ __launch_bounds__(256) void mx_gemm_kernel(MxGemmArgs a) {
    constexpr int NF = NMAT * NBU;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    SegInfo si;
    int b0;
    if (!mx_find_tile<RB>(a.offsets, a.E, a.N, blockIdx.x / a.ftiles, lane, si, b0)) return;
    const int nblk = (si.rows + 15) / 16 - b0;  // blocks of the tile that are the expert's
    const int nb0 = ((blockIdx.x % a.ftiles) * 4 + wave) * NBU;
    if (nb0 >= a.NB) return;
    const size_t frow = ((size_t)si.e * a.NB + nb0) * NMAT;
    const u32x4_t* xp = a.xp + (size_t)(si.bbase + b0) * a.KS * 4 * 64 + lane;
    f32x4_t acc[NF][RB];
#pragma unroll
    for (int r = 0; r < NF; r++)
#pragma unroll
        for (int b = 0; b < RB; b++) acc[r][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int ks = 0; ks < a.KS; ks++) {
        u32x4_t q[NF];
        float scale[NF];
#pragma unroll
        for (int r = 0; r < NF; r++) {
            q[r] = a.wfrag[((frow + r) * a.KS + ks) * 64 + lane];
            scale[r] = mx_scale(a.wscale[((frow + r) * a.KW + (ks >> 2)) * 64 + lane], ks & 3);
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            bf16x8_t x[RB];
#pragma unroll
            for (int b = 0; b < RB; b++)
                x[b] = __builtin_bit_cast(bf16x8_t, xp[(((size_t)(b < nblk ? b : 0) * a.KS + ks) * 4 + j) * 64]);
#pragma unroll
            for (int r = 0; r < NF; r++) {
                const bf16x8_t w = mx_widen8(q[r][j], scale[r]);
#pragma unroll
                for (int b = 0; b < RB; b++)
                    acc[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[b], acc[r][b], 0, 0, 0);
            }
        }
    }
    const int t = lane & 15, kq = lane >> 4;
#pragma unroll
    for (int b = 0; b < RB; b++) {
        if (b >= nblk) continue;
#pragma unroll
        for (int u = 0; u < NBU; u++) {
            const int c = (nb0 + u) * 16 + 4 * kq;
            if (NMAT == 2) {
                // h as the second projection's operand, rounded to bf16 there as the rows are
                const f32x4_t g = acc[u * NMAT][b], v = acc[u * NMAT + NMAT - 1][b];
                float h[4];
#pragma unroll
                for (int i = 0; i < 4; i++) h[i] = g[i] / (1.0f + __expf(-g[i])) * v[i];
                const size_t chunk = (((size_t)(si.bbase + b0 + b) * mx_frags(a.C) + c / MX_FRAG_K) * 4 + (c % MX_BLOCK) / 8) * 64 +
                                     (c % MX_FRAG_K) / MX_BLOCK * 16 + t;
                *(uint2*)(a.hp + chunk * 8 + c % 8) = make_uint2(moe_pack_bf16x2(h[0], h[1]), moe_pack_bf16x2(h[2], h[3]));
            } else {
                const int row = (b0 + b) * 16 + t;
                if (row < si.rows)
                    *(float4*)(a.yg + (size_t)(si.row0 + row) * a.C + c) =
                        make_float4(acc[u][b][0], acc[u][b][1], acc[u][b][2], acc[u][b][3]);
            }
        }
    }
}

static inline size_t mxg_align256(size_t v) { return (v + 255) & ~(size_t)255; }
static inline size_t mxg_blocks(int N, int E) { return (size_t)N / 16 + E; }

bool moe_mx_gemm_supported(int N, int E, int d, int f) {
    const long long tiles = N / (16 * MXG_RB) + E;
    return tiles * ((d > f ? d : f) / 16) < (1ll << 31);
}

// the rows' and h's operand chunks
size_t moe_mx_gemm_workspace(int N, int E, int d, int f) {
    return mxg_align256(mxg_blocks(N, E) * mx_frags(d) * 4096) + mxg_align256(mxg_blocks(N, E) * mx_frags(f) * 4096);
}

int moe_mx_gemm_plan(int N, int E, int d, int f, moe_ffn_plan_t* plan) {
    if (!moe_mx_gemm_supported(N, E, d, f)) return MOE_ERR_UNSUPPORTED;
    plan->up_tile_rows = plan->down_tile_rows = 16 * MXG_RB;
    plan->up_tile_features = plan->down_tile_features = 256;
    return MOE_OK;
}

int moe_mx_gemm_launch(const moe_weights* W, const void* x, moe_dtype_t act_dtype, const int32_t* perm, int k,
                       const int32_t* offsets, int N, void* ws, float* yg, hipStream_t s) {
    const int E = W->E, d = W->d, f = W->f;
    u32x4_t* xp = (u32x4_t*)ws;
    u32x4_t* hp = (u32x4_t*)((char*)ws + mxg_align256(mxg_blocks(N, E) * mx_frags(d) * 4096));
    const dim3 grid((unsigned)mxg_blocks(N, E), (unsigned)((mx_frags(d) + 7) / 8));
    if (act_dtype == MOE_BF16)
        hipLaunchKernelGGL(mx_rows_kernel<true>, grid, dim3(256), 0, s, x, perm, k, offsets, E, N, d, xp, hp, f);
    else
        hipLaunchKernelGGL(mx_rows_kernel<false>, grid, dim3(256), 0, s, x, perm, k, offsets, E, N, d, xp, hp, f);
    const unsigned rtiles = (unsigned)(N / (16 * MXG_RB) + E);
    MxGemmArgs a = {};
    a.offsets = offsets;
    a.E = E; a.N = N;
    a.wfrag = (const u32x4_t*)W->w13;
    a.wscale = (const unsigned*)W->s13;
    a.xp = xp;
    a.hp = (uint16_t*)hp;
    a.K = d; a.C = f; a.NB = f / 16; a.KS = mx_frags(d); a.KW = mx_words(d);
    a.ftiles = (a.NB + 7) / 8;
    hipLaunchKernelGGL((mx_gemm_kernel<2, 2, MXG_RB>), dim3(rtiles * a.ftiles), dim3(256), 0, s, a);
    moe_record_mid_event(s);
    a.wfrag = (const u32x4_t*)W->w2;
    a.wscale = (const unsigned*)W->s2;
    a.xp = hp;
    a.yg = yg;
    a.K = f; a.C = d; a.NB = d / 16; a.KS = mx_frags(f); a.KW = mx_words(f);
    a.ftiles = (a.NB + 15) / 16;
    hipLaunchKernelGGL((mx_gemm_kernel<1, 4, MXG_RB>), dim3(rtiles * a.ftiles), dim3(256), 0, s, a);
    return moe_launch_status();
}

// y[t,:] = sum_j weights[t,j] * yg[inv_perm[t*k+j],:], rounded once to y's type.
template <bool BF16>
__global__ __launch_bounds__(256) void mx_combine_kernel(const float4* __restrict__ yg, const int32_t* __restrict__ inv_perm,
                                                         const float* __restrict__ weights, int T, int k, int row_chunks,
                                                         void* __restrict__ y) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= row_chunks) return;
    for (int t = blockIdx.y; t < T; t += gridDim.y) {
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int j = 0; j < k; j++) {
            const float w = weights[(size_t)t * k + j];
            const float4 v = yg[(size_t)inv_perm[(size_t)t * k + j] * row_chunks + c];
            acc.x += w * v.x;
            acc.y += w * v.y;
            acc.z += w * v.z;
            acc.w += w * v.w;
        }
        const size_t at = (size_t)t * row_chunks + c;
        if (BF16) ((uint2*)y)[at] = make_uint2(moe_pack_bf16x2(acc.x, acc.y), moe_pack_bf16x2(acc.z, acc.w));
        else ((float4*)y)[at] = acc;
    }
}

int moe_mx_combine_launch(const float* yg, const int32_t* inv_perm, const float* weights, int T, int k, int d, void* y,
                          moe_dtype_t y_dtype, hipStream_t s) {
    const int row_chunks = d / 4;
    const dim3 grid((unsigned)((row_chunks + 255) / 256), (unsigned)(T < 65535 ? T : 65535));
    if (y_dtype == MOE_BF16)
        hipLaunchKernelGGL(mx_combine_kernel<true>, grid, dim3(256), 0, s, (const float4*)yg, inv_perm, weights, T, k,
                           row_chunks, y);
    else
        hipLaunchKernelGGL(mx_combine_kernel<false>, grid, dim3(256), 0, s, (const float4*)yg, inv_perm, weights, T, k,
                           row_chunks, y);
    return moe_launch_status();
}
