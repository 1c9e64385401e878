// Products of 8-bit rows with 8-bit matrices on the integer matrix cores: one matrix, or one per expert
// of a batch whose segments only the device knows.  The expert FFN is two of them: the first one's epilogue
// applies silu(a)*b, its rows are brought to 8 bits again, and the second one reads them.
//
//   * tile: up to 16*WT*RB rows of one expert x 16*WF*FB channels (fragment rows of w) for WT x WF waves; an expert's
//     blocks of 16*WT rows are dealt evenly to its tiles, and the loop exists once per number of blocks.
//   * both operands travel through a ring of NS stages of LDS, 64 reduction indices each, which the waves fill
//     with direct-to-LDS loads NS - 1 steps ahead.  Rows (and matrices that are not packed) are read where
//     they lie: four lanes take 64 bytes of a row, and the four chunks are stored rotated by the row, so that
//     the matrix instructions' reads, one chunk of sixteen rows, meet no bank twice.
//   * a step waits for its stage, meets the other waves at a barrier (which also frees the stage of the step
//     before), requests the stage NS - 1 ahead, and multiplies.
#include <atomic>
#include <type_traits>

#include "moe_i8.h"
#include "moe_frag_pack.h"
#include "moe_i8_value.h"
#include "moe_mx.h"

struct I8GemmArgs {
    I8Product p;
    int NR;   // 16-channel fragment rows of an expert's matrix (w1 and w3 counted both)
    int KS;   // steps
    int FT;   // feature tiles
};

struct I8Tile {
    int e, row0, rows;  // the tile's rows of the batch
    int nblk;           // its blocks of 16 * WT rows
    int ft;
};

// Tile number blockIdx.x of the launch, order expert, groups of at most 8 row tiles, feature tile, row tile; an XCD
// takes neighbours of the order, which share operands in its L2.  False past the end.  BR: rows of a block.
template <int BR, int RBM>
__device__ __forceinline__ bool i8_find_tile(const I8GemmArgs& a, int lane, I8Tile& ti) {
    int lo = 0, rows = lane == 0 ? a.p.N : 0;
    if (a.p.offsets) gg_segment_of_lane(a.p.offsets, a.p.E, a.p.N, lane, lo, rows);
    const int nb = (rows + BR - 1) / BR, nt = (nb + RBM - 1) / RBM;
    int it = nt;
#pragma unroll
    for (int dlt = 1; dlt < 64; dlt <<= 1) {
        const int vt = __shfl_up(it, dlt, 64);
        if (lane >= dlt) it += vt;
    }
    const int total = __builtin_amdgcn_readlane(it, 63) * a.FT;
    const int chunk = (total + 7) / 8, me = blockIdx.x >> 3;
    const int L = (blockIdx.x & 7) * chunk + me;
    if (me >= chunk || L >= total) return false;
    const int base = (it - nt) * a.FT;
    const unsigned long long m = __ballot(L >= base && L < base + nt * a.FT);
    const int e = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(m));
    const int lo_e = __builtin_amdgcn_readlane(lo, e), rows_e = __builtin_amdgcn_readlane(rows, e);
    const int tiles = __builtin_amdgcn_readlane(nt, e), blocks = __builtin_amdgcn_readlane(nb, e);
    int r = L - __builtin_amdgcn_readlane(base, e);
    const int grp = r / (8 * a.FT);
    r -= grp * 8 * a.FT;
    const int gw = (tiles - grp * 8) < 8 ? (tiles - grp * 8) : 8;
    const int rt = grp * 8 + r % gw;
    ti.ft = r / gw;
    const int per = blocks / tiles, more = blocks % tiles;
    const int b0 = rt * per + (rt < more ? rt : more);
    ti.e = e;
    ti.nblk = per + (rt < more ? 1 : 0);
    ti.row0 = lo_e + b0 * BR;
    ti.rows = rows_e - b0 * BR < ti.nblk * BR ? rows_e - b0 * BR : ti.nblk * BR;
    return true;
}

// At most n vector-memory requests and no LDS read in flight, then the other waves.
#define I8_MEET(n)                                                                 \
    do {                                                                           \
        __builtin_amdgcn_s_waitcnt(0x0070 | ((n) & 15) | (((n) >> 4) << 14));      \
        asm volatile("" ::: "memory");                                             \
        __builtin_amdgcn_s_barrier();                                              \
        asm volatile("" ::: "memory");                                             \
    } while (0)

// WT x WF waves, RB blocks of 16 rows and FB fragment rows of w each.
template <int WT, int WF, int FB, int NS, int RB, bool PACKED, bool GATED, bool ONCE>
__device__ __forceinline__ void i8_gemm_tile(const I8GemmArgs& a, const I8Tile& ti, int lane, int wave, unsigned char* smem) {
    constexpr int NW = WT * WF, XF = WT * RB, WFR = WF * FB;
    constexpr int XL = (XF + NW - 1) / NW, WL = (WFR + NW - 1) / NW;  // requests of a wave and step
    constexpr int STAGE = (XF + WFR) * 1024, D = NS - 1;
    static_assert((D - 1) * (XL + WL) < 64, "requests");
    const I8Product& p = a.p;
    const int K = p.K;
    const int wt = wave / WF, wf = wave % WF;
    const int fr0 = ti.ft * WFR;

    // where this lane's part of a request lies: a row-major fragment is 16 rows of 64 bytes, lane l row l / 4
    const int chunk = (lane & 3) ^ ((lane >> 4) & 3);
    const int last = K - 16;  // (the last step of a K that is no multiple of 64 reads nothing behind the row)
    const int8_t* xp[XL];
    const int8_t* wp[WL];
#pragma unroll
    for (int i = 0; i < XL; i++) {
        const int f = i * NW + wave < XF ? i * NW + wave : XF - 1;
        int r = f * 16 + (lane >> 2);
        r = ti.row0 + (r < ti.rows ? r : ti.rows - 1);
        const size_t src = p.perm ? p.perm[r] / p.k : r;
        xp[i] = p.x + src * K;
    }
#pragma unroll
    for (int i = 0; i < WL; i++) {
        int fr = fr0 + (i * NW + wave < WFR ? i * NW + wave : WFR - 1);  // (past the last: the last again)
        if (PACKED) {
            fr = fr < a.NR ? fr : a.NR - 1;
            wp[i] = p.w + ((size_t)ti.e * a.NR + fr) * a.KS * 1024 + lane * 16;
        } else {
            int c = fr * 16 + (lane >> 2);
            c = c < p.C ? c : p.C - 1;
            wp[i] = p.w + ((size_t)ti.e * p.C + c) * K;
        }
    }
    auto request = [&](int ks, int slot) __attribute__((always_inline)) {
        // (past the end: the last step's operands again, so that every step counts the same requests)
        const int kc = ks < a.KS ? ks : a.KS - 1;
        int at = kc * I8_FRAG_K + chunk * 16;
        at = at < last ? at : last;
#pragma unroll
        for (int i = 0; i < WL; i++) {
            const int f = i * NW + wave < WFR ? i * NW + wave : WFR - 1;
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void*)(wp[i] + (PACKED ? (size_t)kc * 1024 : (size_t)at)),
                (__attribute__((address_space(3))) void*)(smem + slot * STAGE + f * 1024), 16, 0, ONCE ? 2 : 0);
        }
#pragma unroll
        for (int i = 0; i < XL; i++) {
            const int f = i * NW + wave < XF ? i * NW + wave : XF - 1;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(xp[i] + at),
                                             (__attribute__((address_space(3))) void*)(smem + slot * STAGE + (WFR + f) * 1024),
                                             16, 0, 0);
        }
    };

    i32x4_t acc[FB][RB];
#pragma unroll
    for (int r = 0; r < FB; r++)
#pragma unroll
        for (int b = 0; b < RB; b++) acc[r][b] = i32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < D; i++) {
        request(i, i);
        asm volatile("" ::: "memory");
    }

    // the matrix instruction's operand: row l % 16, chunk l / 16
    const int rl = lane & 15, cq = lane >> 4;
    const int row_major = (rl * 4 + (cq ^ ((rl >> 2) & 3))) * 16;
    const int w_at = PACKED ? lane * 16 : row_major;
    const int tail = K % I8_FRAG_K;  // bytes of the last step, 0: all
    auto step = [&](int k, auto slot_) __attribute__((always_inline)) {
        constexpr int u = decltype(slot_)::value;
        // this step's operands have arrived, and every wave has read the stage that is refilled now
        I8_MEET((D - 1) * (XL + WL));
        request(k + D, (u + D) % NS);
        const unsigned char* st = smem + u * STAGE;
        i32x4_t w[FB], x[RB];
#pragma unroll
        for (int r = 0; r < FB; r++) w[r] = *(const i32x4_t*)(st + (wf * FB + r) * 1024 + w_at);
#pragma unroll
        for (int b = 0; b < RB; b++) x[b] = *(const i32x4_t*)(st + (WFR + wt * RB + b) * 1024 + row_major);
        if (tail && k == a.KS - 1 && cq * 16 >= tail) {
#pragma unroll
            for (int b = 0; b < RB; b++) x[b] = i32x4_t{0, 0, 0, 0};
        }
#pragma unroll
        for (int b = 0; b < RB; b++)
#pragma unroll
            for (int r = 0; r < FB; r++) acc[r][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[r], x[b], acc[r][b], 0, 0, 0);
    };
    using std::integral_constant;
    int k = 0;
    for (; k + NS <= a.KS; k += NS) {
        step(k, integral_constant<int, 0>{});
        step(k + 1, integral_constant<int, 1>{});
        step(k + 2, integral_constant<int, 2>{});
        if constexpr (NS > 3) step(k + 3, integral_constant<int, 3>{});
        static_assert(NS == 3 || NS == 4, "steps of the ring");
    }
    if (k < a.KS) step(k, integral_constant<int, 0>{});
    if (k + 1 < a.KS) step(k + 1, integral_constant<int, 1>{});
    if constexpr (NS > 3) if (k + 2 < a.KS) step(k + 2, integral_constant<int, 2>{});
    // no request for LDS outlives the workgroup
    __builtin_amdgcn_s_waitcnt(0x0070);

    // lane: row l % 16 of a block, four neighbouring channels of a fragment row
    const int frw = fr0 + wf * FB;
#pragma unroll
    for (int b = 0; b < RB; b++) {
        const int rr = (wt * RB + b) * 16 + rl;
        if (rr >= ti.rows) continue;
        const size_t row = ti.row0 + rr;
        const float sx = p.xs[p.perm ? p.perm[row] / p.k : (int)row];
        if (GATED) {
#pragma unroll
            for (int n = 0; n < FB / 2; n++)
                if (frw + 2 * n < a.NR)
                    i8_put_gated(p, ti.e, a.NR, frw + 2 * n, cq, row, sx, acc[GATED ? 2 * n : 0][b], acc[GATED ? 2 * n + 1 : 0][b]);
        } else {
#pragma unroll
            for (int r = 0; r < FB; r++) i8_put(p, ti.e, (frw + r) * 16 + 4 * cq, row, sx, acc[r][b]);
        }
    }
}

template <int WT, int WF, int FB, int NS, int RBM, bool PACKED, bool GATED, bool ONCE>
__global__ __launch_bounds__(64 * WT * WF, 2) void i8_gemm_kernel(I8GemmArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    I8Tile ti;
    if (!i8_find_tile<16 * WT, RBM>(a, lane, ti)) return;
#define I8_TILE(n) if (ti.nblk == n) i8_gemm_tile<WT, WF, FB, NS, n, PACKED, GATED, ONCE>(a, ti, lane, wave, smem)
    I8_TILE(1);
    else I8_TILE(2);
    if constexpr (RBM >= 4) {
        I8_TILE(3);
        else I8_TILE(4);
    }
    if constexpr (RBM >= 8) {
        I8_TILE(5);
        else I8_TILE(6);
        else I8_TILE(7);
        else I8_TILE(8);
    }
#undef I8_TILE
}

// ------------------------------------------------------------------ host ----
static inline size_t i8_align256(size_t v) { return (v + 255) & ~(size_t)255; }

// Tiles of `rows` rows of one expert, at most: min(N, E) experts have rows, and a last tile of at least one.
static inline size_t i8_tiles(int N, int E, int rows) {
    const size_t used = N < E ? N : E;
    return ((size_t)N + (size_t)(rows - 1) * used) / rows;
}

template <int WT, int WF, int FB, int NS, int RBM, bool PACKED, bool GATED, bool ONCE>
static int i8_gemm_go(I8GemmArgs& a, hipStream_t s) {
    a.FT = (a.NR + WF * FB - 1) / (WF * FB);
    const size_t grid = (i8_tiles(a.p.N, a.p.E, 16 * WT * RBM) * a.FT + 7) / 8 * 8;
    constexpr int lds = NS * (WT * RBM + WF * FB) * 1024;
    auto* kernel = i8_gemm_kernel<WT, WF, FB, NS, RBM, PACKED, GATED, ONCE>;
    if (lds > 65536) {
        static std::atomic<bool> ready[MOE_MAX_DEVICES];  // one-time permission for more than 64 KiB of LDS
        const int dev = moe_current_device();
        if (dev < 0) return MOE_ERR_HIP;
        if (!ready[dev].load(std::memory_order_acquire)) {
            MOE_HIP_TRY(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
            ready[dev].store(true, std::memory_order_release);
        }
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * WT * WF), lds, s, a);
    return moe_launch_status();
}

// Tiles, rows x channels: 256 x 256 where they fill the chip and an expert in use has more than 128 rows on average; else 128 x
// 128 where those do; else 32 x 128.  us with 32 x 128 / 128 x 128 / 256 x 256: first projection (d 4096, f 14336) of 8
// experts of 24 rows 159 / 157 / 165, of 64 207 / 175 / 178, of 128 338 / 214 / 204, of 512 1190 / 658 / 518; the second of 24 rows 82 / 83 /
// 104, of 128 185 / 116 / 151, of 512 649 / 317 / 239; one 4096 x 4096 matrix, 77 rows 15 / 22 / 31, 512 28 / 28 / 61, 1024 49 / 30 / 63,
// 4096 193 / 96 / 79.  256 x 224 where that takes less of whole rounds of 256 compute units (by more than the sixteenth that it costs in
// shared operands): 3000 rows (K 4096, C 14336) 225 -> 213 us, 2048 159 -> 149, 4096 (K 2048, C 10000) 131 -> 121, 4096 (K 4096, C 14336)
// 325 -> 312 to 330, by power.  Only for products: w1 and w3 come in pairs of fragment rows.
struct I8Shape {
    int rows, channels;
};
static I8Shape i8_shape(int N, int E, int NR, bool gated) {
    const int used = N < E ? N : E;
    auto fills = [&](int rows, int channels) {
        return ((long long)N / rows + used) * ((NR * 16 + channels - 1) / channels) >= 200;
    };
    if (N > 128 * used && fills(256, 256)) {
        auto cost = [&](int channels) { return (i8_tiles(N, E, 256) * ((NR * 16 + channels - 1) / channels) + 255) / 256 * channels; };
        return {256, !gated && cost(224) * 17 < cost(256) * 16 ? 224 : 256};
    }
    return fills(128, 128) ? I8Shape{128, 128} : I8Shape{32, 128};
}

// A launch has fewer than 2^32 threads.
bool moe_i8_product_supported(int N, int E, int K, int C, bool gated, int path) {
    if (K > I8_MAX_K) return false;
    const int NR = gated ? 2 * (C / 16) : (C + 15) / 16;
    if (path == MOE_FFN_STREAM) return i8_tiles(N, E, 16) * ((NR + 1) / 2) < ((size_t)1 << 32) / 512;
    const I8Shape sh = i8_shape(N, E, NR, gated);
    return (i8_tiles(N, E, sh.rows) * ((NR * 16 + sh.channels - 1) / sh.channels) + 8) < ((size_t)1 << 32) / 512;
}

// ONCE: matrices that most tiles read alone go past the caches (a plain read streams at 6.9 TB/s that way, at 6.0 otherwise).
template <bool PACKED, bool GATED, bool ONCE>
static int i8_gemm_pick(I8GemmArgs& a, hipStream_t s) {
    const I8Shape sh = i8_shape(a.p.N, a.p.E, a.NR, GATED);
    const int rows = sh.rows;
    if (rows == 32) return i8_gemm_go<1, 4, 2, 4, 2, PACKED, GATED, ONCE>(a, s);
    if (rows == 128) return i8_gemm_go<2, 2, 4, 4, 4, PACKED, GATED, ONCE>(a, s);
    if constexpr (!GATED) {
        if (sh.channels == 224) return i8_gemm_go<4, 2, 7, 3, 4, PACKED, false, false>(a, s);
    }
    return i8_gemm_go<2, 4, 4, 3, 8, PACKED, GATED, false>(a, s);
}

// Are the matrices in use too large for the last-level cache to hold from one call to the next?  Then loads past it are faster:
// 128 x 128 tiles, first projection of 8 experts of 24 rows (d 4096, f 14336) 156 -> 147 us, the second 83 -> 72; 64 experts of 28
// rows (d 2048, f 1408) 70 -> 66; but one 4096 x 4096 matrix, which stays, 64 rows 19 -> 23.
bool moe_i8_streams(const I8Product& p, int NR) {
    const size_t used = p.N < p.E ? p.N : p.E;
    return used * NR * 16 * p.K > ((size_t)96 << 20);
}

int moe_i8_product_launch(const I8Product& p, int path, hipStream_t s) {
    if (path == MOE_FFN_STREAM) return moe_i8_stream_launch(p, s);
    I8GemmArgs a = {};
    a.p = p;
    a.NR = p.gated ? 2 * (p.C / 16) : (p.C + 15) / 16;
    a.KS = i8_frags(p.K);
    const bool once = moe_i8_streams(p, a.NR) && p.N <= 128 * (p.N < p.E ? p.N : p.E);
    if (p.gated) return once ? i8_gemm_pick<true, true, true>(a, s) : i8_gemm_pick<true, true, false>(a, s);
    if (p.packed) return once ? i8_gemm_pick<true, false, true>(a, s) : i8_gemm_pick<true, false, false>(a, s);
    return once ? i8_gemm_pick<false, false, true>(a, s) : i8_gemm_pick<false, false, false>(a, s);
}

// ---- the expert FFN: rows to 8 bits, w1 and w3 with silu*mul, h to 8 bits, w2 ----
// workspace: codes and scales of the rows, h in fp32, its codes and scales, or the bits of its largest magnitudes (a few rows)
struct I8FfnSpace {
    size_t xq, xs, h, hq, hs, top, bytes;
};
// Do both projections take the persistent loop?
static bool i8_persistent(int N, int E, int d, int f) {
    return i8_shape(N, E, f / 8, true).rows == 256 && i8_shape(N, E, d / 16, false).rows == 256 && moe_i8_grouped_supported(N, E, d, f);
}

static I8FfnSpace i8_ffn_space(int N, int E, int d, int f) {
    I8FfnSpace w;
    w.xq = 0;
    w.xs = i8_align256((size_t)N * d);
    w.h = w.xs + i8_align256((size_t)N * 4);
    w.hq = w.h + i8_align256((size_t)N * f * 4);
    w.hs = w.hq + i8_align256((size_t)N * f);
    w.top = w.hq;
    w.bytes = w.hs + i8_align256((size_t)N * 4);
    if (i8_persistent(N, E, d, f)) {
        const size_t b = w.h + moe_i8_grouped_workspace(N, E, d, f);
        w.bytes = b > w.bytes ? i8_align256(b) : w.bytes;
    }
    return w;
}
size_t moe_i8_ffn_workspace(int N, int E, int d, int f) {
    return d <= I8_MAX_K && f <= I8_MAX_K ? i8_ffn_space(N, E, d, f).bytes : 0;
}
// STREAM reads a matrix once for every 16 rows, so skewed batches leave it before balanced ones: 8 experts of 4 / 12 / 16 / 20 rows,
// first projection, STREAM 139 / 144 / 151 / 280 us, 128 x 128 tiles 154 / 156 / 155 / 156; 64 experts (d 2048, f 1408) of 8 / 16 / 20 rows
// 60 / 68 / 100 and 65 / 67 / 68; one 4096 x 4096 matrix, which stays in the caches, 32 / 64 rows 9.5 / 15.5 and 14.3 / 14.5.
int moe_i8_auto_path(int N, int E) {
    const int used = N < E ? N : E;
    return N <= (E == 1 ? 32 : 8 * used) ? MOE_FFN_STREAM : MOE_FFN_GROUPED;
}
bool moe_i8_ffn_supported(int path, int N, int E, int d, int f) {
    return (path == MOE_FFN_GROUPED || path == MOE_FFN_STREAM) && moe_i8_product_supported(N, E, d, f, true, path) &&
           moe_i8_product_supported(N, E, f, d, false, path);
}
int moe_i8_ffn_plan(int N, int E, int d, int f, moe_ffn_plan_t* plan) {
    if (!moe_i8_ffn_supported(plan->path, N, E, d, f)) return MOE_ERR_UNSUPPORTED;
    if (plan->path == MOE_FFN_STREAM) return MOE_OK;
    // (the persistent loop's tiles: 256 features in both projections, whatever whole rounds i8_shape would make)
    const I8Shape loop = {moe_i8_grouped_tile_rows(N, E), 256};
    const bool persistent = i8_persistent(N, E, d, f);
    const I8Shape up = persistent ? loop : i8_shape(N, E, f / 8, true), down = persistent ? loop : i8_shape(N, E, d / 16, false);
    plan->up_tile_rows = up.rows;
    plan->up_tile_features = up.channels;
    plan->down_tile_rows = down.rows;
    plan->down_tile_features = down.channels;
    return MOE_OK;
}

// yg, or the layer's y where `c` is given: then yg is scratch.
static int i8_experts(const moe_weights* W, const int8_t* codes, const float* scales, const int32_t* perm, int k,
                      const int32_t* offsets, int N, char* base, const I8FfnSpace& sp, float* yg, const I8Combine* c, int path,
                      hipStream_t s) {
    const int E = W->E, d = W->d, f = W->f;
    if (path == MOE_FFN_GROUPED && i8_persistent(N, E, d, f)) {
        const int rc = moe_i8_grouped_launch(W, codes, scales, perm, k, offsets, N, base + sp.h, yg, s);
        if (rc != MOE_OK || !c) return rc;
        return moe_mx_combine_launch(yg, 1, 0, c->inv_perm, c->weights, c->T, c->k, d, c->y, c->y_bf16 ? MOE_BF16 : MOE_F32, s);
    }
    const bool small = path == MOE_FFN_STREAM && moe_i8_down_small_serves(N, f);
    I8Product up = {};
    up.x = codes;
    up.xs = scales;
    up.perm = perm;
    up.k = k;
    up.offsets = offsets;
    up.E = E;
    up.N = N;
    up.K = d;
    up.C = f;
    up.w = (const int8_t*)W->w13;
    up.ws = (const float*)W->s13;
    up.packed = up.gated = true;
    up.y = base + sp.h;
    up.ytop = small ? (unsigned*)(base + sp.top) : nullptr;
    int rc = moe_i8_product_launch(up, path, s);
    if (rc != MOE_OK) return rc;
    moe_record_mid_event(s);
    if (small) return moe_i8_down_small_launch(W, (const float*)(base + sp.h), up.ytop, offsets, N, c ? nullptr : yg, c, s);
    rc = moe_i8_rows_launch(base + sp.h, MOE_F32, N, f, (int8_t*)(base + sp.hq), (float*)(base + sp.hs), s);
    if (rc != MOE_OK) return rc;
    I8Product down = {};
    down.x = (const int8_t*)(base + sp.hq);
    down.xs = (const float*)(base + sp.hs);
    down.k = 1;
    down.offsets = offsets;
    down.E = E;
    down.N = N;
    down.K = f;
    down.C = d;
    down.w = (const int8_t*)W->w2;
    down.ws = (const float*)W->s2;
    down.packed = true;
    down.y = yg;
    rc = moe_i8_product_launch(down, path, s);
    if (rc != MOE_OK || !c) return rc;
    return moe_mx_combine_launch(yg, 1, 0, c->inv_perm, c->weights, c->T, c->k, d, c->y, c->y_bf16 ? MOE_BF16 : MOE_F32, s);
}

int moe_i8_ffn_launch(const moe_weights* W, const void* x, moe_dtype_t act_dtype, int rows, const int32_t* perm, int k,
                      const int32_t* offsets, int N, void* ws, float* yg, int path, hipStream_t s) {
    const I8FfnSpace sp = i8_ffn_space(N, W->E, W->d, W->f);
    char* base = (char*)ws;
    int8_t* codes = (int8_t*)(base + sp.xq);
    float* scales = (float*)(base + sp.xs);
    const int rc = moe_i8_rows_launch(x, act_dtype, rows, W->d, codes, scales, s);
    return rc != MOE_OK ? rc : i8_experts(W, codes, scales, perm, k, offsets, N, base, sp, yg, nullptr, path, s);
}

int moe_i8_layer_launch(const moe_weights* W, I8Front f, moe_dtype_t x_dtype, void* ws, void* y, moe_dtype_t y_dtype, int path,
                        hipStream_t s) {
    const int N = f.T * f.k;
    const I8FfnSpace sp = i8_ffn_space(N, W->E, W->d, W->f);
    char* base = (char*)ws;
    f.E = W->E;
    f.d = W->d;
    if (f.x) {
        f.codes = (unsigned*)(base + sp.xq);
        f.scales = (float*)(base + sp.xs);
    }
    int rc;
    if (N <= I8_FRONT_SLOTS) {
        rc = moe_i8_front_launch(f, x_dtype, s);
    } else {
        rc = moe_route_launch(f.logits, f.T, f.E, f.k, f.idx, f.weights, s);
        if (rc == MOE_OK)
            rc = moe_permute_launch(f.idx, f.T, f.E, f.k, nullptr, 0, MOE_F32, f.counts, f.offsets, f.perm, f.inv_perm, nullptr, s);
        if (rc == MOE_OK && f.x) rc = moe_i8_rows_launch(f.x, x_dtype, f.T, f.d, (int8_t*)f.codes, f.scales, s);
    }
    if (rc != MOE_OK) return rc;
    const I8Combine c = {f.inv_perm, f.weights, f.T, f.k, y, y_dtype == MOE_BF16};
    return i8_experts(W, (const int8_t*)f.codes, f.scales, f.perm, f.k, f.offsets, N, base, sp, (float*)(base + sp.bytes), &c, path, s);
}
