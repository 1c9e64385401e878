// Decode-sized expert FFN and layer over MXFP4 expert matrices for gfx950.
//
// A few rows per expert are bound by reading each active expert's matrices once, here 17/32
// byte per weight.  The plan is that of the bf16 kernels (moe_ffn_stream.hip): a wave streams
// fragments of 16 features by 128 reduction indices with 16-byte-per-lane loads, widens the
// codes to bf16 in registers (exact, moe_mx.h), and multiplies them with the rows on
// v_mfma_f32_16x16x32_bf16, fp32 accumulate; fp32 rows are split into three bf16 parts, which
// hold all 24 bits.  The waves of a workgroup split the reduction, one scale word (four
// fragments, 512 indices) each, and keep their slice of the rows in registers over all
// consecutive units of the same rows; their partial tiles meet in LDS.
//
// A unit is (tile of rows of one expert, reduction part, group of NBU blocks of 16 features); the
// units are dealt to the workgroups in contiguous, equal ranges, and the loads of two units are
// in flight.
//   up   (x.w1, x.w3 -> silu*mul -> h): one part.  Its prologue may route the tokens and batch
//        them (up to 64 slots).  h is fp32, or bf16 where the result is.
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
#define MXS_MAX_WAVES 8
#define MXS_MAX_SLOTS 64

struct MxArgs {
    const u32x4_t* wfrag;
    const unsigned* wscale;
    const void* act;          // [rows,K]
    const int32_t* row_perm;  // or null; else row i of the activations is act[row_perm[i] / row_k]
    int row_k;
    const int32_t* offsets;
    float* out;               // up: h [N,C]; down: slabs [P][N][C], or yg (finish == FIN_NONE)
    size_t part_stride;
    int E, N, K, C;
    int NB, KS, KW;           // 16-feature blocks, fragments and scale words of a reduction
    int P, W;
    unsigned* counters;       // [n_counters], one per feature group of the second projection:
    int n_counters;           // cleared by up, counted by down
    int finish;
    int h_bf16;               // up: h is bf16
    float* yg;                // FIN_ROWS: out
    MxStep st;
};
enum { FIN_NONE = 0, FIN_ROWS = 1, FIN_LAYER = 2 };

// How a tile's rows become the matrix instructions' 16 operand columns.  An fp32 row is three
// bf16 parts, and 5 rows have all their parts in one instruction (columns t, t + 5, t + 10, added
// in the end).  More rows of an expert are more tiles: the registers that hold two operands a row
// would not leave room for two units in flight.
enum { ROWS_BF16 = 0, ROWS_F32 = 1 };
constexpr int rows_of(int R) { return R == ROWS_BF16 ? 16 : 5; }

// The wave's slice of the rows: four fragments' worth of reduction indices from fragment ks0.
template <int R>
__device__ __forceinline__ void mx_load_act(bf16x8_t (&act)[4][4], const void* actp, int K, int row0, int rows,
                                            int ks0, int lane, const int* rowmap, const int32_t* perm, int perm_k,
                                            const float* row_scale) {
#pragma clang fp contract(off)
    const int c = lane & 15, kq = lane >> 4;
    const int t = R == ROWS_BF16 ? c : c % rows_of(R), part = R == ROWS_BF16 ? 0 : c / rows_of(R);
    const bool used = t < rows && part < 3;
    int src_row = row0 + t;
    if (rowmap && used) src_row = rowmap[row0 + t];
    if (perm && used) src_row = perm[row0 + t] / perm_k;
    float sc = 1.0f;
    if (R != ROWS_BF16 && row_scale && used) sc = row_scale[src_row];
#pragma unroll
    for (int s = 0; s < 4; s++) {
        const int k0 = (ks0 + s) * MX_FRAG_K + kq * MX_BLOCK;
        const bool live = used && k0 < K;
        const size_t off = (size_t)src_row * K + k0;
        if (R == ROWS_BF16) {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                u32x4_t v = {0u, 0u, 0u, 0u};
                if (live) v = *(const u32x4_t*)((const uint16_t*)actp + off + 8 * j);
                act[s][j] = __builtin_bit_cast(bf16x8_t, v);
            }
            continue;
        }
        f32x4_t x[8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            x[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (live) x[j] = *(const f32x4_t*)((const float*)actp + off + 4 * j);
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            // the scaled row is rounded to fp32 before the split, as if it had been stored
            bf16x8_t a;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float v = x[2 * j + i / 4][i % 4] * sc;
                const __bf16 hi = (__bf16)v;
                const float r = v - (float)hi;
                const __bf16 mid = (__bf16)r, lo = (__bf16)(r - (float)mid);
                a[i] = part == 0 ? hi : part == 1 ? mid : lo;
            }
            act[s][j] = a;
        }
        // (the requests of more fragments at once would not fit in registers)
        if (s & 1) __builtin_amdgcn_sched_barrier(0);
    }
}

// Sum of one wave's partial tile over the columns of a row's parts, for lanes of columns < rows.
template <int R>
__device__ __forceinline__ f32x4_t mx_parts_sum(const f32x4_t* p, int lane) {
    if (R == ROWS_BF16) return p[lane];
    const int at = (lane & 48) + (lane & 15) % rows_of(R);
    return p[at] + p[at + 5] + p[at + 10];
}

// Slabs are written by one workgroup and read by another of the same launch, maybe on another XCD,
// whose L2 is another: both sides go past the caches that the other does not share, so that
// neither has to write back or drop a whole cache (device fences by every wave made the second
// projection of one token 72 us long instead of 21).
__device__ __forceinline__ void mx_store_shared(float* p, const f32x4_t& v) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    __hip_atomic_store((unsigned long long*)p, __builtin_bit_cast(unsigned long long, f2{v[0], v[1]}), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store((unsigned long long*)p + 1, __builtin_bit_cast(unsigned long long, f2{v[2], v[3]}), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x4_t mx_load_shared(const float* p) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_bit_cast(f2, __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    const f2 b = __builtin_bit_cast(f2, __hip_atomic_load((const unsigned long long*)p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    return f32x4_t{a[0], a[1], b[0], b[1]};
}

// Per-expert batching of N <= 64 slots by one wave, E <= 64: lane p owns slot p and finds the slots
// of its expert with one ballot per bit of the expert's number.  Lane e < E gets its expert's rows
// [lo, lo + cnt); s_pos[p]: the slot's position; s_cnt [64]: scratch.
__device__ __forceinline__ void mx_batch_wave(const int* s_idx, int N, int E, int lane, bool write, const MxStep& st,
                                              int* s_pos, int* s_cnt, int& lo, int& cnt) {
    const bool live = lane < N;
    const int e = live ? s_idx[lane] : 0;
    unsigned long long same = __ballot(live);
#pragma unroll
    for (int b = 0; b < 6; b++) {
        const unsigned long long m = __ballot((e >> b) & 1);
        same &= ((e >> b) & 1) ? m : ~m;
    }
    const int rank = __popcll(same & ((lane == 0) ? 0ull : (~0ull >> (64 - lane))));
    s_cnt[lane] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (live && rank == 0) s_cnt[e] = __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    cnt = s_cnt[lane];
    int inc = cnt;
#pragma unroll
    for (int dlt = 1; dlt < 64; dlt <<= 1) {
        const int v = __shfl_up(inc, dlt, 64);
        if (lane >= dlt) inc += v;
    }
    lo = inc - cnt;
    const int pos = __shfl(lo, e, 64) + rank;
    if (live) {
        s_pos[lane] = pos;
        if (write) {
            st.perm[pos] = lane;
            st.inv_perm[lane] = pos;
        }
    }
    if (write) {
        if (lane < E) {
            st.counts[lane] = cnt;
            st.offsets[lane] = lo;
        }
        if (lane == E - 1) st.offsets[E] = inc;
    }
}

// The workgroup's waves route the tokens, one at a time each: lane e holds expert e's logit, and its
// rank is the number of logits before it (larger, or equal and of a lower expert).  k rounds of a
// contest by exchanges between lanes, as in moe_route, take 2.5 us for 64 experts and k = 6; this
// a fifth.  The weights, which only the writing workgroup needs, are moe_route's to the bit.
__device__ __forceinline__ void mx_route(const float* logits, const MxStep& st, int E, int wave, int W, int lane, int* s_idx,
                                         float* s_top, bool write) {
    for (int t = wave; t < st.T; t += W) {
        const float v = lane < E ? logits[(size_t)t * E + lane] : -INFINITY;
        int rank = 0;
        for (int e = 0; e < E; e++) {
            const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), e));
            rank += (lane > e ? o >= v : o > v) ? 1 : 0;
        }
        if (lane < st.k) s_idx[t * st.k + lane] = 0;  // (logits that are NaN leave ranks out)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (lane < E && rank < st.k) {
            s_idx[t * st.k + rank] = lane;
            s_top[t * st.k + rank] = v;
        }
        if (!write) continue;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const float u = lane < st.k ? expf(s_top[t * st.k + lane] - s_top[t * st.k]) : 0.f;
        float sum = u;
#pragma unroll
        for (int m = 1; m < MOE_MAX_K; m <<= 1) sum += __shfl_xor(sum, m, 64);
        if (lane < st.k) {
            st.idx[(size_t)t * st.k + lane] = s_idx[t * st.k + lane];
            st.weights[(size_t)t * st.k + lane] = u / sum;
        }
    }
}

// The group's rows are complete: add the parts, and what the step asks for beyond them.
template <int NBU>
__device__ void mx_finish(const MxArgs& a, int g, int tid, int threads, float* s_x) {
    constexpr int C4 = NBU * 4;  // float4 columns of the group
    const size_t col0 = (size_t)g * NBU * 16;
    auto row_sum = [&](int row, int c4) -> float4 {
        const float* p = a.out + (size_t)row * a.C + col0 + 4 * c4;
        f32x4_t v = mx_load_shared(p);
        for (int q = 1; q < a.P; q += 4) {  // four requests at a time, added in order
            f32x4_t u[4];
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (q + i < a.P) u[i] = mx_load_shared(p + (size_t)(q + i) * a.part_stride);
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (q + i < a.P) v += u[i];
        }
        return make_float4(v[0], v[1], v[2], v[3]);
    };
    if (a.finish == FIN_ROWS) {
        for (int i = tid; i < a.N * C4; i += threads) {
            const int row = i / C4, c4 = i % C4;
            *(float4*)(a.yg + (size_t)row * a.C + col0 + 4 * c4) = row_sum(row, c4);
        }
        return;
    }
    const MxStep& st = a.st;
    const int T = a.N / st.k;
    for (int i = tid; i < T * C4; i += threads) {
        const int t = i / C4, c4 = i % C4;
        const size_t at = (size_t)t * a.C + col0 + 4 * c4;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int j = 0; j < st.k; j++) {
            const float w = st.weights[t * st.k + j];
            int row = st.inv_perm[t * st.k + j];
            row = row < 0 ? 0 : (row >= a.N ? a.N - 1 : row);
            const float4 v = row_sum(row, c4);
            if (st.yg) *(float4*)(st.yg + (size_t)row * a.C + col0 + 4 * c4) = v;
            acc.x += w * v.x;
            acc.y += w * v.y;
            acc.z += w * v.z;
            acc.w += w * v.w;
        }
        if (st.x_in) {
            float4 xr = *(const float4*)(st.x_in + at);
            xr.x += acc.x; xr.y += acc.y; xr.z += acc.z; xr.w += acc.w;
            acc = xr;
        }
        if (st.y_dtype == MOE_BF16)
            *(uint2*)((uint16_t*)st.y + at) = make_uint2(moe_pack_bf16x2(acc.x, acc.y), moe_pack_bf16x2(acc.z, acc.w));
        else
            *(float4*)((float*)st.y + at) = acc;
        if (st.w_gate_next) *(float4*)(s_x + t * NBU * 16 + 4 * c4) = acc;
    }
    if (!st.w_gate_next) return;
    __syncthreads();
    // the 16 features' shares of the next block's gating sums
    const int items = T * (a.E + 1);
    for (int i = tid; i < NBU * items; i += threads) {
        const int b = i / items, it = i % items;
        const int t = it / (a.E + 1), ex = it % (a.E + 1);
        const float* xs = s_x + t * NBU * 16 + b * 16;
        const float* wg = st.w_gate_next + (col0 + 16 * b) * a.E + ex;
        float v = 0.f;
#pragma unroll
        for (int c = 0; c < 16; c++) v = fmaf(xs[c], ex == a.E ? xs[c] : wg[(size_t)c * a.E], v);
        st.sums_next[((size_t)g * NBU + b) * st.gate_stride + it] = v;
    }
    __syncthreads();  // s_x serves the next group
}

template <int NMAT, int NBU, int R, bool GATE>
__global__ __launch_bounds__(64 * MXS_MAX_WAVES) void mx_stream_kernel(MxArgs a) {
    constexpr bool DOWN = NMAT == 1;
    constexpr int NF = NMAT * NBU;  // fragment rows of a unit
    extern __shared__ __align__(16) unsigned char s_raw[];
    f32x4_t* s_red = (f32x4_t*)s_raw;  // [2][W][NF][64]
    __shared__ int s_tiles[MXS_MAX_WAVES][3][MXS_MAX_TILES];
    __shared__ int s_idx[GATE ? MXS_MAX_SLOTS : 1];
    __shared__ float s_top[GATE ? MXS_MAX_SLOTS : 1];
    __shared__ int s_batch[GATE ? MXS_MAX_WAVES : 1][3][MXS_MAX_SLOTS];
    __shared__ float s_gate[GATE ? 3 : 1][64];  // the summed shares, 1/rms per token, the logits
    __shared__ float s_gpart[GATE ? MXS_MAX_WAVES : 1][GS_MAX_ITEMS];
    __shared__ unsigned long long s_last;

    const int tid = threadIdx.x, lane = tid & 63, threads = blockDim.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int* s_te = s_tiles[wave][0];
    int* s_tr0 = s_tiles[wave][1];
    int* s_trn = s_tiles[wave][2];

    if (!DOWN)
        for (int i = blockIdx.x * threads + tid; i < a.n_counters; i += gridDim.x * threads) a.counters[i] = 0u;

    int lo = 0, hi = 0;
    const int* rowmap = nullptr;
    const float* row_scale = nullptr;
    if (GATE) {
        const MxStep& st = a.st;
        const float* lg = st.logits;
        if (st.gate_sums) {
            // every wave adds its part of the shares, then every wave the parts, in wave order
            const int items = st.T * (a.E + 1);
            const int per_w = (st.n_shares + a.W - 1) / a.W;
            const int row0 = wave * per_w;
            const int row1 = (row0 + per_w) < st.n_shares ? (row0 + per_w) : st.n_shares;
            if (lane < items) s_gpart[wave][lane] = 0.f;
            float* s_rows = (float*)s_red + wave * (GS_WAVE_ROWS * GS_MAX_ITEMS);
            gate_add_shares(st.gate_sums, row0, row1, st.gate_stride, items, lane, s_rows, s_gpart[wave]);
            __syncthreads();
            if (wave == 0) {
                if (lane < items) {
                    float v = s_gpart[0][lane];
                    for (int w = 1; w < a.W; w++) v += s_gpart[w][lane];
                    s_gate[0][lane] = v;
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
        mx_route(lg, st, a.E, wave, a.W, lane, s_idx, s_top, blockIdx.x == 0);
        __syncthreads();
        int cnt;
        int* s_pos = s_batch[wave][0];
        int* s_src = s_batch[wave][1];
        mx_batch_wave(s_idx, a.N, a.E, lane, blockIdx.x == 0 && wave == 0, st, s_pos, s_batch[wave][2], lo, cnt);
        if (lane < a.N) s_src[s_pos[lane]] = lane / st.k;
        hi = lo + cnt;
        rowmap = s_src;
    } else if (lane < a.E) {
        lo = a.offsets[lane];
        hi = a.offsets[lane + 1];
    }
    auto write_xg = [&]() {
        if (GATE && a.st.xg) {
            const int chunks = a.K / (R == ROWS_BF16 ? 8 : 4);
            for (int i = blockIdx.x; i < a.N; i += gridDim.x) {
                const u32x4_t* src = (const u32x4_t*)a.act + (size_t)rowmap[i] * chunks;
                u32x4_t* dst = (u32x4_t*)a.st.xg + (size_t)i * chunks;
                for (int c = tid; c < chunks; c += threads) dst[c] = src[c];
            }
        }
    };
    const int n_tiles = stream_tile_list<rows_of(R), MXS_MAX_TILES>(lo, hi, a.E, a.N, lane, s_te, s_tr0, s_trn);
    const unsigned groups = (unsigned)(a.NB / NBU);
    const unsigned total = (unsigned)n_tiles * (unsigned)a.P * groups;  // < 2^31 (host check)
    const unsigned per = total / gridDim.x, rem = total % gridDim.x;
    const unsigned u_begin = per * blockIdx.x + rem * blockIdx.x / gridDim.x;
    const unsigned u_end = per * (blockIdx.x + 1) + rem * (blockIdx.x + 1) / gridDim.x;
    if (u_begin >= u_end) {  // uniform over the workgroup
        write_xg();
        return;
    }

    struct Unit {
        int tile, part, g, word;
        size_t row;  // fragment row (e, nb, mat) of the unit's first fragment
    };
    auto unit_of = [&](unsigned u) -> Unit {
        Unit n;
        n.g = (int)(u % groups);
        const unsigned tp = u / groups;
        n.part = (int)(tp % (unsigned)a.P);
        n.tile = (int)(tp / (unsigned)a.P);
        n.word = n.part * a.W + wave;
        n.row = ((size_t)s_te[n.tile] * a.NB + (size_t)n.g * NBU) * NMAT;
        return n;
    };
    // Fragments and words past the reduction's end (a wave whose share is short) are read as the
    // last one again: their rows' operands are zero.
    auto ld = [&](const Unit& n, int i) -> u32x4_t {
        int ks = n.word * 4 + (i & 3);
        ks = ks < a.KS ? ks : a.KS - 1;
        return __builtin_nontemporal_load(a.wfrag + ((n.row + (i >> 2)) * a.KS + ks) * 64 + lane);
    };
    auto ld_scale = [&](const Unit& n, int r) -> unsigned {
        const int w = n.word < a.KW ? n.word : a.KW - 1;
        return __builtin_nontemporal_load(a.wscale + ((n.row + r) * a.KW + w) * 64 + lane);
    };

    Unit unit[2];
    u32x4_t buf[2][NF][4];
    unsigned sc[2][NF];
    auto request = [&](int st, int r) __attribute__((always_inline)) {
        sc[st][r] = ld_scale(unit[st], r);
#pragma unroll
        for (int s = 0; s < 4; s++) buf[st][r][s] = ld(unit[st], r * 4 + s);
    };
    unit[0] = unit_of(u_begin);
#pragma unroll
    for (int r = 0; r < NF; r++) request(0, r);
    unit[1] = unit_of(u_begin + 1 < u_end ? u_begin + 1 : u_begin);
    if (u_begin + 1 < u_end) {
#pragma unroll
        for (int r = 0; r < NF; r++) request(1, r);
    }

    bf16x8_t act[4][4];
    int cur_tile = -1, cur_part = -1;
    // unit u, whose loads are in stage st, and the requests of unit u + 2
    auto process = [&](auto stage, unsigned u) __attribute__((always_inline)) {
        constexpr int st = decltype(stage)::value;
        const Unit cur = unit[st];
        const int row0 = s_tr0[cur.tile], rows = s_trn[cur.tile];
        if (cur.tile != cur_tile || cur.part != cur_part) {
            mx_load_act<R>(act, a.act, a.K, row0, rows, cur.word * 4, lane, rowmap, a.row_perm, a.row_k, row_scale);
            cur_tile = cur.tile;
            cur_part = cur.part;
        }
        const bool more = u + 2 < u_end;
        if (more) unit[st] = unit_of(u + 2);
        const int phase = (int)(u - u_begin);  // of the turns and of the two halves of s_red: its parity is st
        f32x4_t* red = s_red + (size_t)(st * a.W + wave) * NF * 64;
#pragma unroll
        for (int r = 0; r < NF; r++) {
            f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 4; s++) {
                const u32x4_t q = buf[st][r][s];
                const float scale = mx_scale(sc[st][r], s);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mx_widen8(q[j], scale), act[s][j], acc, 0, 0, 0);
                }
            }
            if (more) request(st, r);
            red[r * 64 + lane] = acc;
        }
        __syncthreads();
        // the waves take turns at the blocks' sums
#pragma unroll
        for (int b = 0; b < NBU; b++) {
            if (wave != (phase * NBU + b) % a.W) continue;
            f32x4_t sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < a.W; w++) {
                const f32x4_t* p = s_red + (size_t)(st * a.W + w) * NF * 64 + b * NMAT * 64;
                sa += mx_parts_sum<R>(p, lane);
                if (NMAT == 2) sb += mx_parts_sum<R>(p + 64, lane);
            }
            const int t = lane & 15;
            if (t < rows) {
                const size_t at = (size_t)(row0 + t) * a.C + ((size_t)cur.g * NBU + b) * 16 + 4 * (lane >> 4);
                if (NMAT == 2) {
                    float h[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) h[i] = sa[i] / (1.0f + __expf(-sa[i])) * sb[i];
                    if (a.h_bf16)
                        *(uint2*)((uint16_t*)a.out + at) = make_uint2(moe_pack_bf16x2(h[0], h[1]), moe_pack_bf16x2(h[2], h[3]));
                    else
                        *(float4*)(a.out + at) = make_float4(h[0], h[1], h[2], h[3]);
                } else if (a.finish == FIN_NONE) {
                    *(float4*)(a.out + at) = make_float4(sa[0], sa[1], sa[2], sa[3]);
                } else {
                    mx_store_shared(a.out + (size_t)cur.part * a.part_stride + at, sa);
                }
            }
        }
    };
    for (unsigned u = u_begin; u < u_end; u += 2) {
        process(std::integral_constant<int, 0>{}, u);
        if (u + 1 < u_end) process(std::integral_constant<int, 1>{}, u + 1);
    }
    write_xg();
    if (!DOWN || a.finish == FIN_NONE) return;

    // The slabs' stores have arrived; count the units, and finish the groups whose last unit this was.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const unsigned need = (unsigned)n_tiles * (unsigned)a.P;
    for (unsigned base = u_begin; base < u_end; base += 64) {
        if (wave == 0) {
            bool last = false;
            if (base + lane < u_end)
                last = __hip_atomic_fetch_add(a.counters + (base + lane) % groups, 1u, __ATOMIC_RELAXED,
                                              __HIP_MEMORY_SCOPE_AGENT) + 1u == need;
            const unsigned long long m = __ballot(last);
            if (lane == 0) s_last = m;
        }
        __syncthreads();
        unsigned long long m = s_last;
        while (m) {
            const int i = (int)__builtin_ctzll(m);
            m &= m - 1;
            mx_finish<NBU>(a, (int)((base + i) % groups), tid, threads, (float*)s_red);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ host ----
static inline size_t mx_align256(size_t v) { return (v + 255) & ~(size_t)255; }

// Waves and parts of a reduction: every wave takes one scale word of every part.
struct MxSplit {
    int W, P;
};
static MxSplit mx_split(int K, bool parts) {
    const int KW = mx_words(K);
    MxSplit s = {KW, 1};
    if (KW <= MXS_MAX_WAVES || !parts) return s;
    // as many full waves as possible, then the fewest idle ones
    int best = -1;
    for (int w = MXS_MAX_WAVES; w >= 4; w--) {
        const int p = (KW + w - 1) / w;
        const int score = KW * 1000 / (p * w) * 16 + w;
        if (score > best) {
            best = score;
            s.W = w;
            s.P = p;
        }
    }
    return s;
}

bool moe_mx_stream_serves(int N, int E, int d, int f) {
    if (mx_words(d) > MXS_MAX_WAVES || N / rows_of(ROWS_F32) + E > MXS_MAX_TILES) return false;
    return (long long)MXS_MAX_TILES * mx_split(f, true).P * ((d > f ? d : f) / 16) < (1ll << 31);
}

// The rows up to which streaming is taken (16 rows a pass); the GEMM above it.
int moe_mx_auto_path(int N, int E, int d, int f) {
    return N <= 72 && moe_mx_stream_serves(N, E, d, f) ? MOE_FFN_STREAM : MOE_FFN_GROUPED;
}

// counters, h [N,f] fp32, the second projection's slabs [P][N,d] fp32
size_t moe_mx_stream_workspace(int N, int E, int d, int f) {
    (void)E;
    return mx_align256((size_t)d / 16 * 4) + mx_align256((size_t)N * f * 4) + (size_t)mx_split(f, true).P * N * d * 4;
}

bool moe_mx_stream_routes(int T, int E, int k, int d, int f) {
    return T >= 1 && T <= 16 && T * k <= MXS_MAX_SLOTS && E <= MOE_MAX_E && moe_mx_stream_serves(T * k, E, d, f);
}

bool moe_mx_block_supported(int T, int E, int k, int d, int f) {
    if (!moe_mx_stream_routes(T, E, k, d, f)) return false;
    if (T * k > 4 || E > 16 || T * (E + 1) > GS_MAX_ITEMS) return false;
    return d / 16 <= GS_WAVE_ROWS * mx_split(d, false).W;
}

template <int NMAT, int NBU, int R, bool GATE>
static int mx_stream_go(const MxArgs& a, hipStream_t s) {
    const void* fn = (const void*)mx_stream_kernel<NMAT, NBU, R, GATE>;
    size_t lds = (size_t)2 * a.W * NMAT * NBU * 64 * sizeof(f32x4_t);
    if (GATE && lds < (size_t)a.W * GS_WAVE_ROWS * GS_MAX_ITEMS * 4) lds = (size_t)a.W * GS_WAVE_ROWS * GS_MAX_ITEMS * 4;
    // workgroups per CU, per device and number of waves: 0 = not asked yet.  Threads that race
    // here ask the same question and store the same answer.
    static std::atomic<int> occ_cache[MOE_MAX_DEVICES][MXS_MAX_WAVES + 1];
    const int dev = moe_current_device();
    if (dev < 0) return MOE_ERR_HIP;
    int occ = occ_cache[dev][a.W].load(std::memory_order_relaxed);
    if (occ == 0) {
        MOE_HIP_TRY(hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024));
        MOE_HIP_TRY(hipOccupancyMaxActiveBlocksPerMultiprocessor(&occ, fn, 64 * a.W, lds));
        occ = occ < 1 ? 1 : (occ > 4 ? 4 : occ);
        occ_cache[dev][a.W].store(occ, std::memory_order_relaxed);
    }
    MxArgs args = a;
    void* params[1] = {(void*)&args};
    MOE_HIP_TRY(hipLaunchKernel(fn, dim3((unsigned)(moe_num_cus() * occ)), dim3(64 * a.W), params, lds, s));
    return moe_launch_status();
}

int moe_mx_stream_launch(const moe_weights* W, const void* x, moe_dtype_t act_dtype, const int32_t* perm, int k,
                         const int32_t* offsets, int N, void* ws, float* yg, const MxStep* step, hipStream_t s) {
    const MxSplit up_split = mx_split(W->d, false), down_split = mx_split(W->f, true);
    const bool gate = step && (step->logits || step->gate_sums);
    unsigned* counters = (unsigned*)ws;
    float* h = (float*)((char*)ws + mx_align256((size_t)W->d / 16 * 4));
    float* slabs = (float*)((char*)h + mx_align256((size_t)N * W->f * 4));
    if (step) offsets = step->offsets;

    MxArgs a = {};
    a.wfrag = (const u32x4_t*)W->w13;
    a.wscale = (const unsigned*)W->s13;
    a.act = x;
    a.row_perm = gate ? nullptr : perm;
    a.row_k = k;
    a.offsets = offsets;
    a.out = h;
    a.E = W->E; a.N = N; a.K = W->d; a.C = W->f;
    a.NB = W->f / 16; a.KS = mx_frags(W->d); a.KW = mx_words(W->d);
    a.W = up_split.W; a.P = 1;
    a.counters = counters;
    a.n_counters = W->d / 16;  // a feature group is one block at least
    if (step) a.st = *step;
    // A bf16 result is rounded to 8 bits once more, so h is held in as many before it.
    a.h_bf16 = step && step->y && step->y_dtype == MOE_BF16 && !step->yg;
    int rc;
    if (act_dtype == MOE_BF16)
        rc = gate ? mx_stream_go<2, 1, ROWS_BF16, true>(a, s) : mx_stream_go<2, 1, ROWS_BF16, false>(a, s);
    else
        rc = gate ? mx_stream_go<2, 1, ROWS_F32, true>(a, s) : mx_stream_go<2, 1, ROWS_F32, false>(a, s);
    if (rc != MOE_OK) return rc;
    moe_record_mid_event(s);

    a.wfrag = (const u32x4_t*)W->w2;
    a.wscale = (const unsigned*)W->s2;
    a.act = h;
    a.row_perm = nullptr;
    a.K = W->f; a.C = W->d;
    a.NB = W->d / 16; a.KS = mx_frags(W->f); a.KW = mx_words(W->f);
    a.W = down_split.W; a.P = down_split.P;
    a.finish = step ? FIN_LAYER : (a.P > 1 ? FIN_ROWS : FIN_NONE);
    a.out = a.finish == FIN_NONE ? yg : slabs;
    a.part_stride = (size_t)N * W->d;
    a.yg = yg;
    return a.h_bf16 ? mx_stream_go<1, 2, ROWS_BF16, false>(a, s) : mx_stream_go<1, 2, ROWS_F32, false>(a, s);
}
