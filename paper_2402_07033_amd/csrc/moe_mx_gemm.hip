// Expert FFN over MXFP4 matrices for several rows per expert and prompts: a grouped GEMM on the
// bf16 matrix cores.
//
// The codes are widened to bf16 in the registers of the wave that multiplies with them (exact, one
// instruction per two weights, moe_mx.h): a wave owns four fragment rows (64 features) for all rows
// of its tile, so nothing is widened twice in a workgroup and weights never touch LDS.  The rows
// come as operand chunks (mx_rows_kernel, and the first projection's epilogue for the second) through
// a ring of LDS stages that the workgroup's four waves fill with direct-to-LDS loads, one fragment's
// 128 reduction indices a stage.
//   * tile: up to RBM (2 or 8) blocks of 16 rows of one expert x 256 features; an expert's blocks are dealt
//     evenly to its tiles, and the loop exists once per number of blocks.
//   * two to four workgroups per CU: one's prologue and epilogue run under the other's loop.
//   * a step waits for its stage, meets the other waves at a barrier (which also frees the stage of
//     the step before), requests the operands D steps ahead, and multiplies.
//   * few tiles (second projection): the reduction is cut in S parts, every part a slab of partial
//     sums, which the combine (or mx_sum_kernel) adds in part order.
//   * T bf16 parts per row, by the caller's types alone: a result in fp32 takes fp32 rows and h in three
//     (all 24 bits), one in bf16, which is rounded to 8 bits in the end, in two (16 bits); bf16 rows are
//     one.  Each part is as much matrix work again.  Rounded to one part, bf16 results were off by 2.4e-3
//     against 64 bits instead of their own rounding's 1.7e-3, and 4096 tokens of 2 of 8 experts (d 4096,
//     f 14336) took 2260 us instead of 2840; 1024 fp32 rows for an fp32 result 322 instead of 792.
#include <type_traits>

#include "moe_mx.h"
#include "moe_frag_pack.h"

#define MXG_WAVES 4
#define MXG_NF 4   // fragment rows of a wave
// Steps requested ahead, in stages of LDS (12 .. 64 KiB a workgroup).  More rows are more matrix work under
// which a request may travel, and a third stage of many rows leaves room for one workgroup per CU.  One part,
// the first projection with one step / two, us: 8 experts of 64 rows (d 4096, f 14336) 146 / 126, of 1024 rows
// 1408 / 1549; a third step for single blocks was slower, 8 experts of 10 rows 84 with two, 88 with three, 16
// (f 6400) of 12 rows 81, 86.  Two parts in tiles of 32 rows, the layer: 8 experts of 12 rows 190 / 165, of 75
// rows 356 / 344, of 1024 rows 2980 / 2990.
constexpr int mxg_depth(int T, int RB) { return RB * T > 4 ? 1 : 2; }
constexpr int mxg_lds(int T, int RBM) {
    int most = 0;
    for (int rb = 1; rb <= RBM; rb++) {
        const int b = (mxg_depth(T, rb) + 1) * rb * T * 4096;
        most = b > most ? b : most;
    }
    return most;
}

// Eight fp32 values -> their T bf16 parts.
template <int T>
__device__ __forceinline__ void mx_parts8(const float (&v)[8], u32x4_t (&o)[T]) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = v[i];
#pragma unroll
    for (int t = 0; t < T; t++) {
        bf16x8_t p;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            p[i] = (__bf16)r[i];
            r[i] = mx_rest(r[i], (float)p[i]);
        }
        o[t] = __builtin_bit_cast(u32x4_t, p);
    }
}

// Rows as B operands: block b of 16 rows of an expert, [block][KS][4 j][T][64 lanes] 16-byte chunks,
// lane l of (ks, j): row l % 16, indices ks*128 + 32*(l / 16) + 8j .. +7 (moe_mx.h).  Rows past
// the expert's last and indices past K are zero.  TH: parts of h.
template <bool BF16, int T>
__global__ __launch_bounds__(256) void mx_rows_kernel(const void* __restrict__ x, const int32_t* __restrict__ perm, int k,
                                                      const int32_t* __restrict__ offsets, int E, int N, int K,
                                                      u32x4_t* __restrict__ xp, u32x4_t* __restrict__ hp, int f, int TH) {
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
        u32x4_t v[T];
#pragma unroll
        for (int p = 0; p < T; p++) v[p] = u32x4_t{0u, 0u, 0u, 0u};
        if (r < si.rows && k0 < K) {
            const size_t off = (size_t)src * K + k0;
            if (BF16) {
                v[0] = *(const u32x4_t*)((const uint16_t*)x + off);
            } else {
                const float4 a = *(const float4*)((const float*)x + off);
                const float4 b = *(const float4*)((const float*)x + off + 4);
                const float f8[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                mx_parts8<T>(f8, v);
            }
        }
#pragma unroll
        for (int p = 0; p < T; p++) xp[(((size_t)blockIdx.x * KS * 4 + i) * T + p) * 64 + lane] = v[p];
    }
    // the first projection does not reach the indices of h past f
    if (blockIdx.y == 0 && f % MX_FRAG_K && kq * MX_BLOCK >= f % MX_FRAG_K)
        for (int p = 0; p < TH; p++)
            hp[(((size_t)blockIdx.x * mx_frags(f) * 4 + (mx_frags(f) - 1) * 4 + (threadIdx.x >> 6)) * TH + p) * 64 + lane] =
                u32x4_t{0u, 0u, 0u, 0u};
}

struct MxGemmArgs {
    const u32x4_t* wfrag;
    const unsigned* wscale;
    const u32x4_t* xp;
    uint16_t* hp;   // up: out
    int TH;         // parts of h
    float* yg;      // down: out, slab 0
    size_t part_stride;
    const int32_t* offsets;
    int E, N, C, NB, KS, KW;
    int FT;         // feature tiles
    int S;          // reduction parts
};

struct MxTile {
    SegInfo si;
    int b0, nblk;   // its blocks inside the segment
    int ft, part;
};

// Tile number L of the launch, order expert, then groups of at most 8 row tiles, part and feature
// tile, row tile; false past the end.  `chunk`: tiles of an XCD.
template <int RBM>
__device__ __forceinline__ bool mx_find_tile(const MxGemmArgs& a, int lane, MxTile& ti) {
    int lo, rows;
    gg_segment_of_lane(a.offsets, a.E, a.N, lane, lo, rows);
    const int nb = (rows + 15) / 16, nt = (nb + RBM - 1) / RBM;
    int ib = nb, it = nt;
#pragma unroll
    for (int dlt = 1; dlt < 64; dlt <<= 1) {
        const int vb = __shfl_up(ib, dlt, 64), vt = __shfl_up(it, dlt, 64);
        if (lane >= dlt) {
            ib += vb;
            it += vt;
        }
    }
    const int FS = a.FT * a.S;
    const int total = __builtin_amdgcn_readlane(it, 63) * FS;
    // an XCD takes neighbours of the order, which share operands in its L2
    const int chunk = (total + 7) / 8, me = blockIdx.x >> 3;
    const int L = (blockIdx.x & 7) * chunk + me;
    if (me >= chunk || L >= total) return false;
    const int base = (it - nt) * FS;
    const unsigned long long m = __ballot(L >= base && L < base + nt * FS);
    const int e = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(m));
    ti.si.e = e;
    ti.si.row0 = __builtin_amdgcn_readlane(lo, e);
    ti.si.rows = __builtin_amdgcn_readlane(rows, e);
    ti.si.bbase = __builtin_amdgcn_readlane(ib - nb, e);
    const int tiles = __builtin_amdgcn_readlane(nt, e), blocks = __builtin_amdgcn_readlane(nb, e);
    int r = L - __builtin_amdgcn_readlane(base, e);
    const int grp = r / (8 * FS);
    r -= grp * 8 * FS;
    const int gw = (tiles - grp * 8) < 8 ? (tiles - grp * 8) : 8;
    const int fs = r / gw, rt = grp * 8 + r % gw;
    ti.ft = fs % a.FT;
    ti.part = fs / a.FT;
    const int per = blocks / tiles, more = blocks % tiles;
    ti.b0 = rt * per + (rt < more ? rt : more);
    ti.nblk = per + (rt < more ? 1 : 0);
    return true;
}

// At most n vector-memory requests and no LDS read in flight, then the other waves.
#define MXG_MEET(n)                                                                \
    do {                                                                           \
        __builtin_amdgcn_s_waitcnt(0x0070 | ((n) & 15) | (((n) >> 4) << 14));      \
        asm volatile("" ::: "memory");                                             \
        __builtin_amdgcn_s_barrier();                                              \
        asm volatile("" ::: "memory");                                             \
    } while (0)

// ONCE: most weights of the launch are read by one tile only, and go past L2.
template <int NMAT, int T, bool ONCE, int RB>
__device__ __forceinline__ void mx_gemm_tile(const MxGemmArgs& a, const MxTile& ti, int lane, int wave, unsigned char* smem) {
    constexpr int NF = MXG_NF, D = mxg_depth(T, RB), NS = D + 1;
    constexpr int STAGE = RB * T * 4096;
    constexpr int VREQ = 2 * NF + RB * T;  // requests of a step and wave
    static_assert((D - 1) * VREQ < 64, "the counter of requests");
    const int frow0 = (ti.ft * MXG_WAVES + wave) * NF;  // of the expert's NB * NMAT
    const bool idle = frow0 >= a.NB * NMAT;             // the last feature tile may be short
    const int k_lo = ti.part * a.KS / a.S, k_hi = (ti.part + 1) * a.KS / a.S;
    const size_t row = (size_t)ti.si.e * a.NB * NMAT + (idle ? 0 : frow0);
    const __amdgpu_buffer_rsrc_t rw = mx_rsrc((const char*)a.wfrag + row * a.KS * 1024);
    const __amdgpu_buffer_rsrc_t rs = mx_rsrc((const char*)a.wscale + row * a.KW * 256);
    const __amdgpu_buffer_rsrc_t rx = mx_rsrc((const char*)a.xp + (size_t)(ti.si.bbase + ti.b0) * a.KS * (T * 4096));

    u32x4_t q[NS][NF];
    unsigned sc[NS][NF];
    auto request = [&](int ks, int slot) __attribute__((always_inline)) {
        ks = ks < k_hi ? ks : k_hi - 1;  // (past the end: again, so that every step counts the same)
#pragma unroll
        for (int r = 0; r < NF; r++) {
            const int at = ((r / NMAT * a.KS + ks) * NMAT + r % NMAT) * 1024;
            q[slot][r] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rw, lane * 16, at, ONCE ? 2 : 0));
            sc[slot][r] = __builtin_amdgcn_raw_buffer_load_b32(rs, lane * 4, (r * a.KW + (ks >> 2)) * 256, 0);
        }
#pragma unroll
        for (int i = 0; i < RB * T; i++) {
            const int c = i * MXG_WAVES + wave;  // chunk of the stage: block c / 4T, (j, part) c % 4T
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rx, (__attribute__((address_space(3))) void*)(smem + slot * STAGE + c * 1024), 16, lane * 16,
                ((c / (4 * T)) * a.KS + ks) * (T * 4096) + (c % (4 * T)) * 1024, 0, 0);
        }
    };

    f32x4_t acc[NF][RB];
#pragma unroll
    for (int r = 0; r < NF; r++)
#pragma unroll
        for (int b = 0; b < RB; b++) acc[r][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D; i++) {
        request(k_lo + i, i);
        asm volatile("" ::: "memory");  // (two steps' requests of one scale word stay two)
    }

    auto step = [&](int k, auto slot_, auto more_) __attribute__((always_inline)) {
        constexpr int u = decltype(slot_)::value;
        constexpr bool more = decltype(more_)::value;  // not one of the last D
        // this step's requests have arrived, and every wave has read the stage that is refilled now
        MXG_MEET(more ? (D - 1) * VREQ : 0);
        if (more) request(k + D, (u + D) % NS);
        const u32x4_t* st = (const u32x4_t*)(smem + u * STAGE) + lane;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            // (the largest tile has no registers for two quarters' rows: without this the compiler spills)
            if (RB == 8 && j > 0) __builtin_amdgcn_sched_barrier(0);
            bf16x8_t x[RB][T];
#pragma unroll
            for (int b = 0; b < RB; b++)
#pragma unroll
                for (int t = 0; t < T; t++) x[b][t] = __builtin_bit_cast(bf16x8_t, st[((b * 4 + j) * T + t) * 64]);
#pragma unroll
            for (int r = 0; r < NF; r++) {
                const bf16x8_t w = mx_widen8(q[u][r][j], mx_scale(sc[u][r] >> (8 * (k & 3)), 0));
#pragma unroll
                for (int t = 0; t < T; t++)
#pragma unroll
                    for (int b = 0; b < RB; b++)
                        acc[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[b][t], acc[r][b], 0, 0, 0);
            }
        }
    };
    // The loop has no way out between its steps: every wait for a step's operands would have to cover
    // it.  The steps behind it request nothing: what nobody uses, the compiler leaves out, and the
    // number of requests that a wait counts on would be another.
    using std::integral_constant;
    int k = k_lo;
    for (; k + NS <= k_hi; k += NS) {
        step(k, integral_constant<int, 0>{}, integral_constant<bool, true>{});
        step(k + 1, integral_constant<int, 1>{}, integral_constant<bool, true>{});
        if constexpr (NS > 2) step(k + 2, integral_constant<int, 2>{}, integral_constant<bool, true>{});
        static_assert(NS == 2 || NS == 3, "steps of the ring");
    }
    if (k < k_hi) step(k, integral_constant<int, 0>{}, integral_constant<bool, false>{});
    if constexpr (NS > 2) if (k + 1 < k_hi) step(k + 1, integral_constant<int, 1>{}, integral_constant<bool, false>{});
    // no request for LDS outlives the workgroup
    __builtin_amdgcn_s_waitcnt(0x0070);
    if (idle) return;

    const int t = lane & 15, kq = lane >> 4;
#pragma unroll
    for (int b = 0; b < RB; b++) {
#pragma unroll
        for (int n = 0; n < NF / NMAT; n++) {
            const int c = (frow0 / NMAT + n) * 16 + 4 * kq;
            if (NMAT == 2) {
                // h as the second projection's operand
                const f32x4_t g = acc[n * NMAT][b], v = acc[n * NMAT + NMAT - 1][b];
                float h[4];
#pragma unroll
                for (int i = 0; i < 4; i++) h[i] = g[i] / (1.0f + __expf(-g[i])) * v[i];
                const size_t chunk = (((size_t)(ti.si.bbase + ti.b0 + b) * mx_frags(a.C) + c / MX_FRAG_K) * 4 + (c % MX_BLOCK) / 8) * a.TH;
                uint16_t* dst = a.hp + (chunk * 64 + (c % MX_FRAG_K) / MX_BLOCK * 16 + t) * 8 + c % 8;
                for (int p = 0; p < a.TH; p++) {
                    *(uint2*)(dst + (size_t)p * 512) = make_uint2(moe_pack_bf16x2(h[0], h[1]), moe_pack_bf16x2(h[2], h[3]));
#pragma unroll
                    for (int i = 0; i < 4; i++) h[i] = mx_rest(h[i], moe_bf16_to_f32(moe_bf16_rne(h[i])));
                }
            } else {
                const int rr = (ti.b0 + b) * 16 + t;
                if (rr < ti.si.rows)
                    *(float4*)(a.yg + ti.part * a.part_stride + (size_t)(ti.si.row0 + rr) * a.C + c) =
                        make_float4(acc[n][b][0], acc[n][b][1], acc[n][b][2], acc[n][b][3]);
            }
        }
    }
}

template <int NMAT, int T, int RBM, bool ONCE>
__global__ __launch_bounds__(64 * MXG_WAVES, RBM > 2 ? 2 : T > 1 ? 3 : 4) void mx_gemm_kernel(MxGemmArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    MxTile ti;
    if (!mx_find_tile<RBM>(a, lane, ti)) return;
    if (ti.nblk == 1) mx_gemm_tile<NMAT, T, ONCE, 1>(a, ti, lane, wave, smem);
    else if (ti.nblk == 2) mx_gemm_tile<NMAT, T, ONCE, 2>(a, ti, lane, wave, smem);
    if constexpr (RBM == 8) {
        if (ti.nblk == 3) mx_gemm_tile<NMAT, T, ONCE, 3>(a, ti, lane, wave, smem);
        else if (ti.nblk == 4) mx_gemm_tile<NMAT, T, ONCE, 4>(a, ti, lane, wave, smem);
        else if (ti.nblk == 5) mx_gemm_tile<NMAT, T, ONCE, 5>(a, ti, lane, wave, smem);
        else if (ti.nblk == 6) mx_gemm_tile<NMAT, T, ONCE, 6>(a, ti, lane, wave, smem);
        else if (ti.nblk == 7) mx_gemm_tile<NMAT, T, ONCE, 7>(a, ti, lane, wave, smem);
        else if (ti.nblk == 8) mx_gemm_tile<NMAT, T, ONCE, 8>(a, ti, lane, wave, smem);
    }
}

// yg = slab 0 + slab 1 + ... in that order, up to the last expert's last row.
__global__ __launch_bounds__(256) void mx_sum_kernel(const float4* __restrict__ slabs, size_t n4, int S, float4* __restrict__ yg,
                                                     const int32_t* __restrict__ end, int row4) {
    const size_t covered = (size_t)(*end < 0 ? 0 : *end) * row4, stop = covered < n4 ? covered : n4;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < stop; i += (size_t)gridDim.x * 256) {
        float4 s = slabs[i];
        for (int p = 1; p < S; p++) {
            const float4 v = slabs[(size_t)p * n4 + i];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        yg[i] = s;
    }
}

// ------------------------------------------------------------------ host ----
static inline size_t mxg_align256(size_t v) { return (v + 255) & ~(size_t)255; }
// Blocks of `rows` rows of one expert, at most: min(N, E) experts have rows, and a last block of at least one.
static inline size_t mxg_blocks(int N, int E, int rows = 16) {
    return ((size_t)N + (size_t)(rows - 1) * (N < E ? N : E)) / rows;
}

// Blocks of a tile, at most.  Rows of one part (the first projection of bf16 rows) by the mean rows of an expert in
// use: tiles of 32 rows let four workgroups run on a CU instead of two, and experts of more rows share their weights in
// L2.  The layer in bf16, tiles of 32 rows / of 128, us: 8 experts (d 4096, f 14336) 20 rows each 170 / 171, 25 each
// 171 / 173, 32 each 224 / 212, 40 each 238 / 223, 100 each 409 / 376; 16 (f 6400) 20 each 163 / 163, 30 each 220 / 202;
// 64 (d 2048, f 1408) 10 each 83 / 84, 19 each 89 / 92, 28 each 107 / 100, 39 each 121 / 114.  Rows of several parts are
// the matrix work of a larger tile already.  The layer with two parts of h (and of x), 32 / 64 rows: 8 experts (f 14336)
// 16 each 165 / 174, 25 each 171 / 172, 50 each 254 / 259, 256 each 808 / 896 (1111 / 1204), 1024 each 2840 / 2865
// (4142 / 4121); 64 of 96 each 184 / 196 (230 / 251), of 384 each 545 / 550 (764 / 755).
#define MXG_SMALL_ROWS 25
static int mxg_rbm(int N, int E, int T) { return T > 1 || N <= MXG_SMALL_ROWS * (N < E ? N : E) ? 2 : 8; }

struct MxGemmShape {
    int tu, td;  // parts of the rows and of h
    int S;       // reduction parts of the second projection
};
static MxGemmShape mxg_shape(int N, int E, int d, int f, bool x_f32, bool y_f32) {
    MxGemmShape sh;
    sh.td = y_f32 ? 3 : 2;
    sh.tu = x_f32 ? sh.td : 1;
    // row tiles that there are about: the experts in use, and those of full tiles
    const int rows = 16 * mxg_rbm(N, E, sh.td);
    const int tiles = N / rows + (N < E ? N : E) + (N == 0);
    const int ft = (d / 16 + MXG_WAVES * MXG_NF - 1) / (MXG_WAVES * MXG_NF);
    int S = 512 / (tiles * ft);
    const int most = mx_frags(f) / 8;
    if (S > most) S = most;
    if (S > 8) S = 8;
    sh.S = S < 1 ? 1 : S;
    return sh;
}

bool moe_mx_gemm_supported(int N, int E, int d, int f) {
    const long long tiles = N / 32 + E;
    return tiles * 8 * ((d > f ? d : f) / 16) < (1ll << 31);
}

// the rows' and h's operand chunks, the second projection's slabs
size_t moe_mx_gemm_workspace(int N, int E, int d, int f) {
    const MxGemmShape sh = mxg_shape(N, E, d, f, true, true), sb = mxg_shape(N, E, d, f, false, false);
    const int S = sh.S > sb.S ? sh.S : sb.S;
    return mxg_align256(mxg_blocks(N, E) * mx_frags(d) * 4096 * sh.tu) +
           mxg_align256(mxg_blocks(N, E) * mx_frags(f) * 4096 * sh.td) + (S > 1 ? (size_t)S * N * d * 4 : 0);
}

int moe_mx_gemm_plan(int N, int E, int d, int f, moe_ffn_plan_t* plan) {
    if (!moe_mx_gemm_supported(N, E, d, f)) return MOE_ERR_UNSUPPORTED;
    plan->up_tile_rows = 16 * mxg_rbm(N, E, 1);  // (of bf16 rows; fp32 rows: as the second projection's)
    plan->down_tile_rows = 16 * mxg_rbm(N, E, 3);
    plan->up_tile_features = plan->down_tile_features = MXG_WAVES * MXG_NF * 16;
    return MOE_OK;
}

template <int NMAT, int T, int RBM, bool ONCE>
static void mxg_go(const MxGemmArgs& a, hipStream_t s) {
    const unsigned grid = ((unsigned)mxg_blocks(a.N, a.E, 16 * RBM) * (unsigned)(a.FT * a.S) + 7) / 8 * 8;
    hipLaunchKernelGGL((mx_gemm_kernel<NMAT, T, RBM, ONCE>), dim3(grid), dim3(64 * MXG_WAVES), mxg_lds(T, RBM), s, a);
}
template <int NMAT, int T>
static void mxg_pick(const MxGemmArgs& a, hipStream_t s) {
    const int rbm = mxg_rbm(a.N, a.E, T);
    const bool once = a.N <= 16 * rbm * a.E;
    if constexpr (T == 1)
        if (rbm == 8) return once ? mxg_go<NMAT, T, 8, true>(a, s) : mxg_go<NMAT, T, 8, false>(a, s);
    once ? mxg_go<NMAT, T, 2, true>(a, s) : mxg_go<NMAT, T, 2, false>(a, s);
}

// The result in n_parts slabs of [N,d] floats from *slabs on, where the caller asks for them; else yg.
int moe_mx_gemm_launch(const moe_weights* W, const void* x, moe_dtype_t act_dtype, const int32_t* perm, int k,
                       const int32_t* offsets, int N, void* ws, float* yg, bool y_f32, const float** slabs, int* n_parts,
                       hipStream_t s) {
    const int E = W->E, d = W->d, f = W->f;
    const MxGemmShape sh = mxg_shape(N, E, d, f, act_dtype == MOE_F32, y_f32);
    u32x4_t* xp = (u32x4_t*)ws;
    u32x4_t* hp = (u32x4_t*)((char*)xp + mxg_align256(mxg_blocks(N, E) * mx_frags(d) * 4096 * sh.tu));
    float* parts = (float*)((char*)hp + mxg_align256(mxg_blocks(N, E) * mx_frags(f) * 4096 * sh.td));
    const dim3 grid((unsigned)mxg_blocks(N, E), (unsigned)((mx_frags(d) + 7) / 8));
    if (act_dtype == MOE_BF16)
        hipLaunchKernelGGL((mx_rows_kernel<true, 1>), grid, dim3(256), 0, s, x, perm, k, offsets, E, N, d, xp, hp, f, sh.td);
    else if (sh.tu == 2)
        hipLaunchKernelGGL((mx_rows_kernel<false, 2>), grid, dim3(256), 0, s, x, perm, k, offsets, E, N, d, xp, hp, f, sh.td);
    else
        hipLaunchKernelGGL((mx_rows_kernel<false, 3>), grid, dim3(256), 0, s, x, perm, k, offsets, E, N, d, xp, hp, f, sh.td);
    MxGemmArgs a = {};
    a.offsets = offsets;
    a.E = E; a.N = N;
    a.wfrag = (const u32x4_t*)W->w13;
    a.wscale = (const unsigned*)W->s13;
    a.xp = xp;
    a.hp = (uint16_t*)hp;
    a.TH = sh.td;
    a.C = f; a.NB = f / 16; a.KS = mx_frags(d); a.KW = mx_words(d);
    a.FT = (2 * a.NB + MXG_WAVES * MXG_NF - 1) / (MXG_WAVES * MXG_NF);
    a.S = 1;
    if (sh.tu == 1) mxg_pick<2, 1>(a, s);
    else if (sh.tu == 2) mxg_pick<2, 2>(a, s);
    else mxg_pick<2, 3>(a, s);
    moe_record_mid_event(s);
    a.wfrag = (const u32x4_t*)W->w2;
    a.wscale = (const unsigned*)W->s2;
    a.xp = hp;
    a.yg = sh.S > 1 ? parts : yg;
    a.part_stride = (size_t)N * d;
    a.C = d; a.NB = d / 16; a.KS = mx_frags(f); a.KW = mx_words(f);
    a.FT = (a.NB + MXG_WAVES * MXG_NF - 1) / (MXG_WAVES * MXG_NF);
    a.S = sh.S;
    if (sh.td == 2) mxg_pick<1, 2>(a, s);
    else mxg_pick<1, 3>(a, s);
    if (slabs) {
        *slabs = a.yg;
        *n_parts = sh.S;
    } else if (sh.S > 1) {
        const size_t n4 = (size_t)N * d / 4;
        const size_t blocks = (n4 + 255) / 256;
        hipLaunchKernelGGL(mx_sum_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s,
                           (const float4*)parts, n4, sh.S, (float4*)yg, offsets + E, d / 4);
    }
    return moe_launch_status();
}

// y[t,:] = sum_j weights[t,j] * (the parts of row inv_perm[t*k+j], in order), rounded once to y's type.
template <bool BF16>
__global__ __launch_bounds__(256) void mx_combine_kernel(const float4* __restrict__ yg, int n_parts, size_t part4,
                                                         const int32_t* __restrict__ inv_perm, const float* __restrict__ weights,
                                                         int T, int k, int row_chunks, void* __restrict__ y) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= row_chunks) return;
    for (int t = blockIdx.y; t < T; t += gridDim.y) {
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int j = 0; j < k; j++) {
            const float w = weights[(size_t)t * k + j];
            const float4* p = yg + (size_t)inv_perm[(size_t)t * k + j] * row_chunks + c;
            float4 v = *p;
            for (int i = 1; i < n_parts; i++) {
                const float4 u = p[i * part4];
                v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
            }
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

int moe_mx_combine_launch(const float* yg, int n_parts, size_t part_stride, const int32_t* inv_perm, const float* weights, int T,
                          int k, int d, void* y, moe_dtype_t y_dtype, hipStream_t s) {
    const int row_chunks = d / 4;
    const dim3 grid((unsigned)((row_chunks + 255) / 256), (unsigned)(T < 65535 ? T : 65535));
    auto* kernel = y_dtype == MOE_BF16 ? mx_combine_kernel<true> : mx_combine_kernel<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const float4*)yg, n_parts, part_stride / 4, inv_perm, weights, T, k,
                       row_chunks, y);
    return moe_launch_status();
}
