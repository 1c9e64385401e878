// Decode-sized expert FFN and layer over MXFP4 expert matrices for gfx950.
//
// A few rows per expert are bound by reading each active expert's matrices once, here 17/32
// byte per weight.  A wave streams two rows of fragments (16 features by 128 reduction indices each)
// with 16-byte-per-lane loads, 16 of them in flight, widens the codes to bf16 in registers (exact,
// moe_mx.h), and multiplies them with the rows on v_mfma_f32_16x16x32_bf16, fp32 accumulate; fp32 rows
// are split into three bf16 parts, which hold all 24 bits.  The rows' operands lie in LDS, one copy
// for the workgroup's 16 waves, and a wave takes its features' whole reduction (or part of it), so
// that the waves meet only where the rows change.  (With the reduction split over the waves, the
// rows in registers and the sums joined in LDS behind every 64 KiB the first projection of 2 / 8
// experts took 30.6 / 89 us, 8 of them in those joins.)
//
// A unit is (tile of rows of one expert, reduction part, group of features): 16 columns of w1 and
// w3, or 32 of w2.  The units are dealt to the workgroups in contiguous, equal ranges.
//   up   (x.w1, x.w3 -> silu*mul -> h): one part.  Its prologue may route the tokens and batch
//        them (up to 64 slots).  h is left as its bf16 parts.
//   down (h.w2): P parts.  Every unit leaves its partial sums in slab [part][N][d]; a counter
//        per feature group tells the workgroup that finishes the group's last unit, and that
//        one adds the parts in part order -- and the rows of a token in slot order, weighted,
//        with the residual and the next block's gating sums if asked for.  The sums' order does
//        not depend on who is last, so the result does not either.  The layer is two launches.
#include <atomic>
#include <type_traits>

#include "moe_mx.h"
#include "moe_gate_wave.h"
#include "moe_stream_wave.h"

#define MXS_MAX_TILES 128
#define MXS_WAVES 16
#define MXS_MAX_WORDS 8  // scale words (512 indices each) of a part: 128 KiB of operands for 16 columns
#define MXS_MAX_SLOTS 64
#define MXS_MAX_ROWS 72
#define MXS_DOWN_COLS 32  // features of a unit of the second projection
#define MXS_MAX_SUMS 96   // T * (E + 1) of a block step's gating sums

// Division of wave-uniform numbers below 2^31 by one that the launch fixes: two multiplications (the
// general one takes some thirty vector instructions, and a kernel's first microseconds are its
// prologue's instructions times the four waves of a SIMD).
struct MxDiv {
    unsigned d, m;  // m = floor(2^32 / d), 2^32 - 1 for 1
};
static inline MxDiv mx_divisor(unsigned d) { return MxDiv{d, d > 1 ? (unsigned)(0x100000000ull / d) : 0xFFFFFFFFu}; }
__device__ __forceinline__ unsigned mx_div(unsigned n, const MxDiv& v) {
    const unsigned q = __umulhi(n, v.m);  // the quotient or one less
    return (q + 1) * v.d <= n ? q + 1 : q;
}

struct MxArgs {
    const u32x4_t* wfrag;
    const unsigned* wscale;
    const void* act;          // [rows,K]
    const int32_t* row_perm;  // or null; else row i of the activations is act[row_perm[i] / row_k]
    int row_k;
    const int32_t* offsets;
    float* out;               // up: h [h_parts][N,C] bf16; down: slabs [P][N][C], or yg (finish == FIN_NONE)
    size_t part_stride;
    int E, N, K, C;
    int NB, KS, KW;           // 16-feature blocks, fragments and scale words of a reduction
    int P;                    // reduction parts
    MxDiv by_groups, by_P, by_k, by_N, by_T, by_grid;
    unsigned* counters;       // [n_counters], one per feature group of the second projection:
    int n_counters;           // cleared by up, counted by down
    int finish;
    int h_parts;              // up: bf16 parts of h, 2 or 3
    float* yg;                // FIN_ROWS: out
    MxStep st;
};
enum { FIN_NONE = 0, FIN_ROWS = 1, FIN_LAYER = 2 };

// How a tile's rows become the matrix instructions' 16 operand columns.  An fp32 row is three
// bf16 parts, and 5 rows have all their parts in one instruction (column part * rows + row), which
// are added in the end.  More rows of an expert are more tiles.  h comes as its parts, [parts][N][f],
// already: three where the result is fp32, two (16 bits) where it is bf16.
enum { ROWS_BF16 = 0, ROWS_F32 = 1, ROWS_PARTS3 = 2, ROWS_PARTS2 = 3 };
constexpr int parts_of(int R) { return R == ROWS_BF16 ? 1 : R == ROWS_PARTS2 ? 2 : 3; }
constexpr int rows_of(int R) { return 16 / parts_of(R); }
constexpr bool rows_in_parts(int R) { return R == ROWS_PARTS3 || R == ROWS_PARTS2; }

// Stages the rows [row0, row0 + rows) of reduction words [w0, w1) as operands, 16-byte chunks
// [(word, fragment, j, lane / 16)][column]: indices word*512 + fragment*128 + 32*(lane/16) + 8j .. +7.
// A wave takes one word of one row (or of one part of it) at a time: block b of (row, word).
template <int R>
struct MxStager {
    static constexpr int REGS = R == ROWS_F32 ? 2 : 1;
    const MxArgs& a;
    const int* rowmap;
    const float* row_scale;
    int row0, rows, w0, words, blocks;
    __device__ __forceinline__ MxStager(const MxArgs& args, const int* rm, const float* rs, int r0, int nr, int wa, int wb)
        : a(args), rowmap(rm), row_scale(rs), row0(r0), rows(nr), w0(wa), words(wb - wa),
          blocks((wb - wa) * nr * (rows_in_parts(R) ? parts_of(R) : 1)) {}
    __device__ __forceinline__ void split(int b, int& rr, int& w) const {
        rr = 0;
        w = b;
        while (w >= words) {
            w -= words;
            rr++;
        }
    }
    __device__ __forceinline__ void request(int b, int lane, u32x4_t (&raw)[REGS], float& sc) const {
        int t, w;
        split(b, t, w);
        int part = 0;
        if (rows_in_parts(R))
            while (t >= rows) {
                t -= rows;
                part++;
            }
        int src = row0 + t;
        if (rowmap) src = __builtin_amdgcn_readfirstlane(rowmap[src]);
        else if (a.row_perm) src = (int)mx_div((unsigned)__builtin_amdgcn_readfirstlane(a.row_perm[src]), a.by_k);
        sc = R == ROWS_F32 && row_scale ? row_scale[src] : 1.0f;
        if (rows_in_parts(R)) src += part * a.N;
        const int k0 = (w0 + w) * 512 + lane * 8;
#pragma unroll
        for (int i = 0; i < REGS; i++) raw[i] = u32x4_t{0u, 0u, 0u, 0u};
        if (k0 >= a.K) return;
        const char* p = (const char*)a.act + (size_t)src * a.K * (R == ROWS_F32 ? 4 : 2) + (size_t)k0 * (R == ROWS_F32 ? 4 : 2);
#pragma unroll
        for (int i = 0; i < REGS; i++) raw[i] = *(const u32x4_t*)(p + 16 * i);
    }
    __device__ __forceinline__ void put(int b, int lane, const u32x4_t (&raw)[REGS], float sc, u32x4_t* s_b) const {
#pragma clang fp contract(off)
        int rr, w;
        split(b, rr, w);
        const int nc = rows * parts_of(R);
        // lane: 8-index group of the word; fragment lane / 16, lane group lane / 4 % 4, j lane % 4
        u32x4_t* dst = s_b + (w * 64 + (lane & 48) + (lane & 3) * 4 + ((lane >> 2) & 3)) * nc + rr;
        if (R != ROWS_F32) {
            *dst = raw[0];
            return;
        }
        bf16x8_t o[3];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            // the scaled row is rounded to fp32 before the split, as if it had been stored
            const float v = __uint_as_float(raw[R == ROWS_F32 ? i / 4 : 0][i % 4]) * sc;
            o[0][i] = (__bf16)v;
            const float r = mx_rest(v, (float)o[0][i]);
            o[1][i] = (__bf16)r;
            o[2][i] = (__bf16)(r - (float)o[1][i]);
        }
#pragma unroll
        for (int p = 0; p < 3; p++) dst[p * rows] = __builtin_bit_cast(u32x4_t, o[p]);
    }
};

// Sum of an accumulator over the columns of a row's parts, for lanes of columns < rows.
template <int R>
__device__ __forceinline__ f32x4_t mx_parts_sum(const f32x4_t& v, int rows, int lane) {
    if (R == ROWS_BF16) return v;
    f32x4_t o = v;
#pragma unroll
    for (int p = 1; p < parts_of(R); p++)
#pragma unroll
        for (int i = 0; i < 4; i++) o[i] += __shfl(v[i], (lane & 48) + ((lane + p * rows) & 15), 64);
    return o;
}

// Slabs are written by one workgroup and read by another of the same launch, maybe on another XCD,
// whose L2 is another: both sides go past the caches that the other does not share, so that
// neither has to write back or drop a whole cache (device fences by every wave made the second
// projection of one token 72 us long instead of 28).
#define MXS_SHARED 16  // cache policy of a buffer access: sc1, coherent for the device
__device__ __forceinline__ void mx_store_shared(const __amdgpu_buffer_rsrc_t& r, unsigned at, const f32x4_t& v) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), r, at, 0, MXS_SHARED);
}
__device__ __forceinline__ f32x4_t mx_load_shared(const __amdgpu_buffer_rsrc_t& r, unsigned at) {
    return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, MXS_SHARED));
}

// The groups of `mask` (bit i: group (g0 + i) % groups) are complete: add the parts, and what the
// step asks for beyond them.  All of them at once: one after the other, each waiting for its own
// slabs, the last workgroup of an 8-expert step took 12 us.
__device__ __forceinline__ f32x4_t mx_row_sum(const MxArgs& a, const __amdgpu_buffer_rsrc_t& slabs, int row, size_t col) {
    const unsigned at = (unsigned)(((size_t)row * a.C + col) * 4), stride = (unsigned)(a.part_stride * 4);
    f32x4_t v = mx_load_shared(slabs, at);
    for (int q = 1; q < a.P; q += 4) {  // four requests at a time, added in order
        f32x4_t u[4];
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (q + i < a.P) u[i] = mx_load_shared(slabs, at + (q + i) * stride);
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (q + i < a.P) v += u[i];
    }
    return v;
}

__device__ __forceinline__ void mx_finish(const MxArgs& a, const int* s_group, int n, int tid, float* s_x) {
    constexpr int C4 = MXS_DOWN_COLS / 4;  // 16-byte columns of a group
    const __amdgpu_buffer_rsrc_t slabs = mx_rsrc(a.out);
    if (a.finish == FIN_ROWS) {
        const int end = a.offsets[a.E];  // rows behind the last expert's have no sums
        for (int i = tid; i < n * a.N * C4; i += 64 * MXS_WAVES) {
            const int c4 = i % C4, gi = (int)mx_div(i / C4, a.by_N), row = i / C4 - gi * a.N;
            if (row >= end) continue;
            const size_t col = (size_t)s_group[gi] * MXS_DOWN_COLS + 4 * c4;
            const f32x4_t v = mx_row_sum(a, slabs, row, col);
            *(f32x4_t*)(a.yg + (size_t)row * a.C + col) = v;
        }
        return;
    }
    const MxStep& st = a.st;
    const int T = (int)a.by_T.d;
    for (int i = tid; i < n * T * C4; i += 64 * MXS_WAVES) {
        const int c4 = i % C4, gi = (int)mx_div(i / C4, a.by_T), t = i / C4 - gi * T;
        const size_t col = (size_t)s_group[gi] * MXS_DOWN_COLS + 4 * c4;
        const size_t at = (size_t)t * a.C + col;
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < st.k; j++) {
            const float w = st.weights[t * st.k + j];
            int row = st.inv_perm[t * st.k + j];
            row = row < 0 ? 0 : (row >= a.N ? a.N - 1 : row);
            const f32x4_t v = mx_row_sum(a, slabs, row, col);
            if (st.yg) *(f32x4_t*)(st.yg + (size_t)row * a.C + col) = v;
            acc += w * v;
        }
        if (st.x_in) acc = *(const f32x4_t*)(st.x_in + at) + acc;
        if (st.y_dtype == MOE_BF16)
            *(uint2*)((uint16_t*)st.y + at) = make_uint2(moe_pack_bf16x2(acc[0], acc[1]), moe_pack_bf16x2(acc[2], acc[3]));
        else
            *(f32x4_t*)((float*)st.y + at) = acc;
        if (st.w_gate_next) *(f32x4_t*)(s_x + (size_t)i * 4) = acc;
    }
    if (!st.w_gate_next) return;
    __syncthreads();
    // shares of the next block's gating sums, 16 features each
    const int items = T * (a.E + 1);
    for (int i = tid; i < n * (MXS_DOWN_COLS / 16) * items; i += 64 * MXS_WAVES) {
        const int it = i % items, b = i / items;  // b: 16 features of the list
        const int t = it / (a.E + 1), ex = it % (a.E + 1);
        const int gi = b / (MXS_DOWN_COLS / 16);
        const size_t share = (size_t)s_group[gi] * (MXS_DOWN_COLS / 16) + b % (MXS_DOWN_COLS / 16);
        const float* xs = s_x + ((size_t)gi * T + t) * MXS_DOWN_COLS + b % (MXS_DOWN_COLS / 16) * 16;
        const float* wg = st.w_gate_next + share * 16 * a.E + ex;
        float w[16];
#pragma unroll
        for (int c = 0; c < 16; c++) w[c] = ex == a.E ? xs[c] : wg[(size_t)c * a.E];
        float v = 0.f;
#pragma unroll
        for (int c = 0; c < 16; c++) v = fmaf(xs[c], w[c], v);
        st.sums_next[share * st.gate_stride + it] = v;
    }
    __syncthreads();  // s_x serves the next groups
}

template <bool DOWN, int R, bool GATE>
__global__ __launch_bounds__(64 * MXS_WAVES) void mx_stream_kernel(MxArgs a) {
    extern __shared__ __align__(16) unsigned char s_raw[];
    u32x4_t* s_b = (u32x4_t*)s_raw;  // operands of the rows at hand, see MxStager
    __shared__ u32x4_t s_zero;       // ... of the columns that no row has
    __shared__ int s_tiles[3][MXS_MAX_TILES], s_ntiles;
    __shared__ int s_idx[GATE ? MXS_MAX_SLOTS : 1];
    __shared__ int s_batch[GATE ? 3 : 1][MXS_MAX_SLOTS];
    __shared__ float s_gate[GATE ? 3 : 1][MXS_MAX_SUMS];  // the summed shares, 1/rms per token, the logits
    __shared__ int s_group[64], s_nlast;

    constexpr int THREADS = 64 * MXS_WAVES;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    if (!DOWN)
        for (int i = blockIdx.x * THREADS + tid; i < a.n_counters; i += gridDim.x * THREADS) a.counters[i] = 0u;
    if (tid == 0) s_zero = u32x4_t{0u, 0u, 0u, 0u};

    const int* rowmap = nullptr;
    const float* row_scale = nullptr;
    if (GATE) {
        const MxStep& st = a.st;
        const float* lg = st.logits;
        if (st.gate_sums) {
            // every wave adds its part of the shares, then one the parts, in wave order
            const int items = st.T * (a.E + 1);
            const int per_w = (st.n_shares + MXS_WAVES - 1) / MXS_WAVES;
            const int row0 = wave * per_w;
            const int row1 = (row0 + per_w) < st.n_shares ? (row0 + per_w) : st.n_shares;
            float* s_gpart = (float*)s_raw;  // [MXS_WAVES][MXS_MAX_SUMS]
            for (int it = lane; it < items; it += 64) {
                float v = 0.f;
                for (int r = row0; r < row1; r += 8) {  // eight requests at a time, added in order
                    float u[8];
#pragma unroll
                    for (int i = 0; i < 8; i++) u[i] = r + i < row1 ? st.gate_sums[(size_t)(r + i) * st.gate_stride + it] : 0.f;
#pragma unroll
                    for (int i = 0; i < 8; i++) v += u[i];
                }
                s_gpart[wave * MXS_MAX_SUMS + it] = v;
            }
            __syncthreads();
            if (wave == 0) {
                for (int it = lane; it < items; it += 64) {
                    float v = s_gpart[it];
#pragma unroll
                    for (int w = 1; w < MXS_WAVES; w++) v += s_gpart[w * MXS_MAX_SUMS + it];
                    s_gate[0][it] = v;
                }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                if (lane < st.T) s_gate[1][lane] = 1.0f / sqrtf(s_gate[0][lane * (a.E + 1) + a.E] / (float)a.K + st.eps);
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                if (lane < st.T * a.E) {
                    const int tok = lane / a.E, ex = lane % a.E;
                    const float v = s_gate[0][tok * (a.E + 1) + ex] * s_gate[1][tok];
                    s_gate[2][lane] = v;
                    if (blockIdx.x == 0 && st.logits_out) st.logits_out[lane] = v;
                }
            }
            __syncthreads();
            lg = s_gate[2];
            row_scale = s_gate[1];
        }
        gate_route_any(lg, st, a.E, wave, MXS_WAVES, lane, s_idx, blockIdx.x == 0);
        __syncthreads();
        rowmap = s_batch[1];
    }
    if (wave == 0) {
        int lo = 0, hi = 0;
        if (GATE) {
            int cnt;
            gate_batch_any(s_idx, a.N, a.E, lane, blockIdx.x == 0, a.st, s_batch[0], s_batch[2], lo, cnt);
            if (lane < a.N) s_batch[1][s_batch[0][lane]] = lane / a.st.k;
            hi = lo + cnt;
        } else if (lane < a.E) {
            lo = a.offsets[lane];
            hi = a.offsets[lane + 1];
        }
        const int n = stream_tile_list<rows_of(R), MXS_MAX_TILES>(lo, hi, a.E, a.N, lane, s_tiles[0], s_tiles[1], s_tiles[2]);
        if (lane == 0) s_ntiles = n;
    }
    __syncthreads();
    auto write_xg = [&]() {
        if (GATE && a.st.xg) {
            const int chunks = a.K / (R == ROWS_BF16 ? 8 : 4);
            for (int i = blockIdx.x; i < a.N; i += gridDim.x) {
                const u32x4_t* src = (const u32x4_t*)a.act + (size_t)rowmap[i] * chunks;
                u32x4_t* dst = (u32x4_t*)a.st.xg + (size_t)i * chunks;
                for (int c = tid; c < chunks; c += THREADS) dst[c] = src[c];
            }
        }
    };
    const unsigned n_tiles = (unsigned)__builtin_amdgcn_readfirstlane(s_ntiles);
    const unsigned groups = (unsigned)(DOWN ? a.NB / 2 : a.NB);
    const unsigned total = n_tiles * (unsigned)a.P * groups;  // < 2^31 (host check)
    const unsigned per = mx_div(total, a.by_grid), rem = total - per * gridDim.x;
    const unsigned u_begin = per * blockIdx.x + mx_div(rem * blockIdx.x, a.by_grid);
    const unsigned u_end = per * (blockIdx.x + 1) + mx_div(rem * (blockIdx.x + 1), a.by_grid);
    if (u_begin >= u_end) {  // uniform over the workgroup
        write_xg();
        return;
    }

    // A wave's work is one sequence of words: those of unit u_begin + wave, of the unit 16 further, ...
    // Word i is in register slot i % 2, and word i + 2 is requested when it has been used.
    struct Item {
        unsigned u, seg;  // unit (>= u_end: none), and its tile and part
        int g, row0, rows, word, w0, w1, part;  // words [w0, w1) of the reduction
        const u32x4_t* p;   // the word's first fragment
        const unsigned* q;  // its scales
    };
    constexpr int FSTEP = DOWN ? 64 : 128;  // w1 and w3 lie fragment by fragment side by side, w2's blocks one after the other
    auto first_word = [&](unsigned u) __attribute__((always_inline)) -> Item {
        Item n;
        n.u = u;
        n.seg = mx_div(u, a.by_groups);
        const unsigned tile = mx_div(n.seg, a.by_P);
        n.g = (int)(u - n.seg * groups);
        n.part = (int)(n.seg - tile * (unsigned)a.P);
        n.row0 = __builtin_amdgcn_readfirstlane(s_tiles[1][tile]);
        n.rows = __builtin_amdgcn_readfirstlane(s_tiles[2][tile]);
        n.word = n.w0 = (int)mx_div(n.part * a.KW, a.by_P);
        n.w1 = (int)mx_div((n.part + 1) * a.KW, a.by_P);
        const size_t frow = ((size_t)__builtin_amdgcn_readfirstlane(s_tiles[0][tile]) * groups + (size_t)n.g) * 2;
        n.p = a.wfrag + frow * a.KS * 64 + (size_t)n.word * (4 * FSTEP);
        n.q = a.wscale + (frow * a.KW + n.word) * 64;
        return n;
    };
    auto next_word = [&](const Item& c) __attribute__((always_inline)) -> Item {
        Item n = c;
        if (c.word + 1 < c.w1) {
            n.word++;
            n.p += 4 * FSTEP;
            n.q += 64;
        } else if (c.u + MXS_WAVES < u_end) {
            return first_word(c.u + MXS_WAVES);
        } else {
            n.u = u_end;
        }
        return n;
    };
    u32x4_t buf[2][2][4];
    unsigned sc[2][2];
    // Fragments past the reduction's end are read as the last one again: their operands are zero.  Behind
    // the last word one line of it is read again: a request that may not be made would have every wait
    // for the other slot wait for both.
    auto request = [&](const Item& n, int slot) __attribute__((always_inline)) {
        const bool none = n.u >= u_end;
        const int last = none ? 0 : a.KS - 1 - n.word * 4;
        const size_t row = none ? 0 : DOWN ? (size_t)a.KS * 64 : 64, srow = none ? 0 : (size_t)a.KW * 64;
#pragma unroll
        for (int r = 0; r < 2; r++) {
            sc[slot][r] = __builtin_nontemporal_load(n.q + r * srow + lane);
#pragma unroll
            for (int s = 0; s < 4; s++)
                buf[slot][r][s] = __builtin_nontemporal_load(n.p + r * row + (s < last ? s : last) * FSTEP + lane);
        }
    };

    // Rows first, weights behind them (requests are answered in order, and the first burst of weights
    // takes microseconds), then the rows' operands into LDS.
    unsigned seg = mx_div(u_begin, a.by_groups);
    auto rows_at = [&](unsigned sg) __attribute__((always_inline)) -> MxStager<R> {
        const unsigned tile = mx_div(sg, a.by_P);
        const int part = (int)(sg - tile * (unsigned)a.P);
        return MxStager<R>(a, rowmap, row_scale, __builtin_amdgcn_readfirstlane(s_tiles[1][tile]),
                           __builtin_amdgcn_readfirstlane(s_tiles[2][tile]), (int)mx_div(part * a.KW, a.by_P),
                           (int)mx_div((part + 1) * a.KW, a.by_P));
    };
    Item item[2];
    {
        const MxStager<R> stager = rows_at(seg);
        u32x4_t raw[2][MxStager<R>::REGS];
        float sc1[2];
#pragma unroll
        for (int i = 0; i < 2; i++)
            if (wave + i * MXS_WAVES < stager.blocks) stager.request(wave + i * MXS_WAVES, lane, raw[i], sc1[i]);
        __builtin_amdgcn_sched_barrier(0);
        item[0].u = u_end;
        if (u_begin + wave < u_end) {
            item[0] = first_word(u_begin + wave);
            request(item[0], 0);
            item[1] = next_word(item[0]);
            request(item[1], 1);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2; i++)
            if (wave + i * MXS_WAVES < stager.blocks) stager.put(wave + i * MXS_WAVES, lane, raw[i], sc1[i], s_b);
        for (int b = wave + 2 * MXS_WAVES; b < stager.blocks; b += MXS_WAVES) {
            stager.request(b, lane, raw[0], sc1[0]);
            stager.put(b, lane, raw[0], sc1[0], s_b);
        }
    }
    __syncthreads();
    const unsigned seg_end = mx_div(u_end - 1, a.by_groups);
    auto next_rows = [&]() __attribute__((always_inline)) {  // by all waves alike
        const MxStager<R> stager = rows_at(++seg);
        __syncthreads();
        for (int b = wave; b < stager.blocks; b += MXS_WAVES) {
            u32x4_t raw[MxStager<R>::REGS];
            float s1;
            stager.request(b, lane, raw, s1);
            stager.put(b, lane, raw, s1, s_b);
        }
        __syncthreads();
    };

    f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    // a unit's sums are complete: h, yg or the part's slab
    auto store = [&](const Item& cur) __attribute__((always_inline)) {
        const f32x4_t sa = mx_parts_sum<R>(acc[0], cur.rows, lane), sb = mx_parts_sum<R>(acc[1], cur.rows, lane);
        const int col = lane & 15, kq = lane >> 4;
        if (col >= cur.rows) return;
        const size_t at = (size_t)(cur.row0 + col) * a.C + (size_t)cur.g * (DOWN ? 32 : 16) + 4 * kq;
        if (!DOWN) {
            float h[4];
#pragma unroll
            for (int i = 0; i < 4; i++) h[i] = sa[i] / (1.0f + __expf(-sa[i])) * sb[i];
            for (int p = 0; p < a.h_parts; p++) {
                *(uint2*)((uint16_t*)a.out + (size_t)p * a.N * a.C + at) =
                    make_uint2(moe_pack_bf16x2(h[0], h[1]), moe_pack_bf16x2(h[2], h[3]));
#pragma unroll
                for (int i = 0; i < 4; i++) h[i] = mx_rest(h[i], moe_bf16_to_f32(moe_bf16_rne(h[i])));
            }
        } else if (a.finish == FIN_NONE) {
            *(f32x4_t*)(a.out + at) = sa;
            *(f32x4_t*)(a.out + at + 16) = sb;
        } else {
            const __amdgpu_buffer_rsrc_t slabs = mx_rsrc(a.out);
            const unsigned to = (unsigned)(((size_t)cur.part * a.part_stride + at) * 4);
            mx_store_shared(slabs, to, sa);
            mx_store_shared(slabs, to + 64, sb);
        }
    };
    auto process = [&](auto slot_) __attribute__((always_inline)) {
        constexpr int slot = decltype(slot_)::value;
        const Item cur = item[slot];
        const bool live = cur.u < u_end;
        while (live && seg < cur.seg) next_rows();
        item[slot] = next_word(item[slot ^ 1]);
        if (live) {
            const int nc = cur.rows * parts_of(R), col = lane & 15, kq = lane >> 4;
            // this lane's operands: its column's, or zeros
            const bool used = col < nc;
            const u32x4_t* pb = used ? s_b + (size_t)((cur.word - cur.w0) * 64 + kq) * nc + col : &s_zero;
            const int step = used ? 4 * nc : 0;
#pragma unroll
            for (int s = 0; s < 4; s++) {
                bf16x8_t x[4];
#pragma unroll
                for (int j = 0; j < 4; j++) x[j] = __builtin_bit_cast(bf16x8_t, pb[(s * 4 + j) * step]);
#pragma unroll
                for (int r = 0; r < 2; r++) {
                    const float scale = mx_scale(sc[slot][r], s);
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mx_widen8(buf[slot][r][s][j], scale), x[j], acc[r], 0, 0, 0);
                }
            }
        }
        request(item[slot], slot);
        if (!live || cur.word + 1 < cur.w1) return;
        store(cur);
        acc[0] = acc[1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    };
    while (item[0].u < u_end) {  // (without a way out between the slots, which the waits would have to cover)
        process(std::integral_constant<int, 0>{});
        process(std::integral_constant<int, 1>{});
    }
    while (seg < seg_end) next_rows();
    write_xg();
    if (!DOWN || a.finish == FIN_NONE) return;

    // The slabs' stores have arrived; count the units, and finish the groups whose last unit this was.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const unsigned need = n_tiles * (unsigned)a.P;
    for (unsigned base = u_begin; base < u_end; base += 64) {
        if (wave == 0) {
            bool last = false;
            const unsigned g = base + lane - mx_div(base + lane, a.by_groups) * groups;
            if (base + lane < u_end)
                last = __hip_atomic_fetch_add(a.counters + g, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u == need;
            const unsigned long long m = __ballot(last);
            if (last) s_group[__popcll(m & ((1ull << lane) - 1))] = (int)g;
            if (lane == 0) s_nlast = __popcll(m);
        }
        __syncthreads();
        const int n = s_nlast;
        if (n) mx_finish(a, s_group, n, tid, (float*)s_raw);
        __syncthreads();
    }
}

// ------------------------------------------------------------------ host ----
static inline size_t mx_align256(size_t v) { return (v + 255) & ~(size_t)255; }

// Parts of the second projection: the operands of a part fit in LDS, and few rows (on at most as many
// experts) give every CU four units, of two words at least.
static int mx_parts(int N, int d, int f) {
    const int KW = mx_words(f);
    int P = (KW + MXS_MAX_WORDS - 1) / MXS_MAX_WORDS;
    while (P * 2 <= KW && (long long)N * (d / MXS_DOWN_COLS) * P < 4 * 256) P++;
    return P;
}

bool moe_mx_stream_serves(int N, int E, int d, int f) {
    if (N > MXS_MAX_ROWS || mx_words(d) > MXS_MAX_WORDS || N / rows_of(ROWS_F32) + E > MXS_MAX_TILES) return false;
    if ((long long)mx_parts(N, d, f) * N * d * 4 >= (1ll << 31)) return false;  // (the slabs' offsets)
    return (long long)MXS_MAX_TILES * mx_parts(1, d, f) * ((d > f ? d : f) / 16) < (1ll << 31);
}

// Streaming, or the GEMM: streaming where an expert's rows are one tile of 5 on average.  8 experts of the
// Mixtral shape with 4 rows each 81 + 55 us (both projections), the GEMM 102 + 63 and 12 for rows and sums;
// 6 rows each 142 + 91 and 102 + 62; 32 rows of uneven experts 100 + 68.
int moe_mx_auto_path(int N, int E, int d, int f) {
    return N <= 4 * E && moe_mx_stream_serves(N, E, d, f) ? MOE_FFN_STREAM : MOE_FFN_GROUPED;
}

// counters, h [3][N,f] bf16, the second projection's slabs [P][N,d] fp32
size_t moe_mx_stream_workspace(int N, int E, int d, int f) {
    (void)E;
    return mx_align256((size_t)d / MXS_DOWN_COLS * 4) + mx_align256((size_t)N * f * 6) + (size_t)mx_parts(N, d, f) * N * d * 4;
}

bool moe_mx_stream_routes(int T, int E, int k, int d, int f) {
    return T >= 1 && T <= 16 && T * k <= MXS_MAX_SLOTS && E <= MOE_MAX_E && moe_mx_stream_serves(T * k, E, d, f);
}

bool moe_mx_block_supported(int T, int E, int k, int d, int f) {
    if (!moe_mx_stream_routes(T, E, k, d, f)) return false;
    return T * k <= 4 && E <= 16 && T * (E + 1) <= MXS_MAX_SUMS && T * E <= 64;
}

template <bool DOWN, int R, bool GATE>
static int mx_stream_go(const MxArgs& a, int rows_max, hipStream_t s) {
    const void* fn = (const void*)mx_stream_kernel<DOWN, R, GATE>;
    // operands of a tile's rows, at most; the shares of the gating sums; the finished rows of a block step
    const int rows = rows_max < rows_of(R) ? rows_max : rows_of(R);
    const int words = (a.KW + a.P - 1) / a.P;
    size_t lds = (size_t)words * 1024 * rows * parts_of(R);
    if (GATE && a.st.gate_sums && lds < (size_t)MXS_WAVES * MXS_MAX_SUMS * 4) lds = (size_t)MXS_WAVES * MXS_MAX_SUMS * 4;
    if (DOWN && a.st.w_gate_next && lds < (size_t)64 * 4 * MXS_DOWN_COLS * 4) lds = (size_t)64 * 4 * MXS_DOWN_COLS * 4;
    static std::atomic<bool> attr_set[MOE_MAX_DEVICES];
    const int dev = moe_current_device();
    if (dev < 0) return MOE_ERR_HIP;
    if (!attr_set[dev].load(std::memory_order_relaxed)) {
        MOE_HIP_TRY(hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 136 * 1024));
        attr_set[dev].store(true, std::memory_order_relaxed);
    }
    MxArgs args = a;
    args.by_groups = mx_divisor((unsigned)(DOWN ? a.NB / 2 : a.NB));
    args.by_P = mx_divisor((unsigned)a.P);
    args.by_k = mx_divisor((unsigned)a.row_k);
    args.by_N = mx_divisor((unsigned)a.N);
    args.by_T = mx_divisor((unsigned)(a.finish == FIN_LAYER ? a.N / a.st.k : a.N));
    args.by_grid = mx_divisor((unsigned)moe_num_cus());
    void* params[1] = {(void*)&args};
    MOE_HIP_TRY(hipLaunchKernel(fn, dim3((unsigned)moe_num_cus()), dim3(64 * MXS_WAVES), params, lds, s));
    return moe_launch_status();
}

int moe_mx_stream_launch(const moe_weights* W, const void* x, moe_dtype_t act_dtype, const int32_t* perm, int k,
                         const int32_t* offsets, int N, void* ws, float* yg, const MxStep* step, hipStream_t s) {
    const bool gate = step && (step->logits || step->gate_sums);
    unsigned* counters = (unsigned*)ws;
    uint16_t* h = (uint16_t*)((char*)ws + mx_align256((size_t)W->d / MXS_DOWN_COLS * 4));
    float* slabs = (float*)((char*)h + mx_align256((size_t)N * W->f * 6));
    if (step) offsets = step->offsets;

    MxArgs a = {};
    a.wfrag = (const u32x4_t*)W->w13;
    a.wscale = (const unsigned*)W->s13;
    a.act = x;
    a.row_perm = gate ? nullptr : perm;
    a.row_k = k;
    a.offsets = offsets;
    a.out = (float*)h;
    a.E = W->E; a.N = N; a.K = W->d; a.C = W->f;
    a.NB = W->f / 16; a.KS = mx_frags(W->d); a.KW = mx_words(W->d);
    a.P = 1;
    a.counters = counters;
    a.n_counters = W->d / MXS_DOWN_COLS;
    if (step) a.st = *step;
    // (a bf16 result is rounded to 8 bits in the end)
    a.h_parts = step && step->y_dtype == MOE_BF16 && !step->yg ? 2 : 3;
    // rows of a tile, at most.  (A token uses an expert once, but logits that are NaN may say otherwise.)
    const int rows_max = N;
    int rc;
    if (act_dtype == MOE_BF16)
        rc = gate ? mx_stream_go<false, ROWS_BF16, true>(a, rows_max, s) : mx_stream_go<false, ROWS_BF16, false>(a, rows_max, s);
    else
        rc = gate ? mx_stream_go<false, ROWS_F32, true>(a, rows_max, s) : mx_stream_go<false, ROWS_F32, false>(a, rows_max, s);
    if (rc != MOE_OK) return rc;
    moe_record_mid_event(s);

    a.wfrag = (const u32x4_t*)W->w2;
    a.wscale = (const unsigned*)W->s2;
    a.act = h;
    a.row_perm = nullptr;
    a.K = W->f; a.C = W->d;
    a.NB = W->d / 16; a.KS = mx_frags(W->f); a.KW = mx_words(W->f);
    a.P = mx_parts(N, W->d, W->f);
    a.finish = step ? FIN_LAYER : (a.P > 1 ? FIN_ROWS : FIN_NONE);
    a.out = a.finish == FIN_NONE ? yg : slabs;
    a.part_stride = (size_t)N * W->d;
    a.yg = yg;
    return a.h_parts == 2 ? mx_stream_go<true, ROWS_PARTS2, false>(a, rows_max, s)
                          : mx_stream_go<true, ROWS_PARTS3, false>(a, rows_max, s);
}
