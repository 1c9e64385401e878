// The norms around a block, with the gate and the residual scale between them, in one launch:
//     u  = y, or y / sqrt(mean(y^2) + eps) * gain_after              the norm after the block
//     x' = x + residual_scale * gate * row_gate * u
//     h  = x' / sqrt(mean(x'^2) + eps) * gain_before                 the norm before the next one
// with h in fp32 or bf16, or in 8 bits with a scale per row, or both.  Bound by memory: x, y, x' and h pass once,
// a row stays in its workgroup's registers between the two sums over it.
//
// The arithmetic is in 64 bits: a code of the 8-bit rows lies next to a border between two codes for one value in
// some ten thousand, and sums of 32 bits would put them on either side.  The vector units do this in a third
// of the time that the bytes take.
#include <type_traits>

#include "moe_i8.h"

// ONCE: read past the caches (4096 rows of 4096, fp32 and bf16 to fp32 and bf16: 47.8 -> 43.5 us; h, which the next kernel reads, is
// left in them: 43.1 otherwise).
template <bool ONCE>
__device__ __forceinline__ float4 bn_load4(const void* p, bool bf16, size_t chunk) {
    if (bf16) {
        typedef unsigned Pair __attribute__((ext_vector_type(2)));
        const Pair* q = (const Pair*)p + chunk;
        const Pair u = ONCE ? __builtin_nontemporal_load(q) : *q;
        return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                           __uint_as_float(u.y & 0xFFFF0000u));
    }
    const f32x4_t* q = (const f32x4_t*)p + chunk;
    const f32x4_t v = ONCE ? __builtin_nontemporal_load(q) : *q;
    return make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void bn_store4(void* p, bool bf16, size_t chunk, const double (&v)[4]) {
    if (bf16) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        ((bf16x4*)p)[chunk] = bf16x4{(__bf16)(float)v[0], (__bf16)(float)v[1], (__bf16)(float)v[2], (__bf16)(float)v[3]};
    } else {
        ((float4*)p)[chunk] = make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
    }
}

// Sum (or maximum) over a wave, in every lane: inside a row of 16 lanes by DPP, across rows by the two lane swaps.
template <bool MAX>
__device__ __forceinline__ double bn_wave(double v) {
    auto join = [](double a, double b) { return MAX ? fmax(a, b) : a + b; };
    auto dpp = [](double a, auto ctrl) {
        const int lo = __double2loint(a), hi = __double2hiint(a);
        return __hiloint2double(__builtin_amdgcn_update_dpp(hi, hi, decltype(ctrl)::value, 0xF, 0xF, false),
                                __builtin_amdgcn_update_dpp(lo, lo, decltype(ctrl)::value, 0xF, 0xF, false));
    };
    v = join(v, dpp(v, std::integral_constant<int, 0xB1>{}));   // quad_perm 1,0,3,2
    v = join(v, dpp(v, std::integral_constant<int, 0x4E>{}));   // quad_perm 2,3,0,1
    v = join(v, dpp(v, std::integral_constant<int, 0x141>{}));  // row_half_mirror
    v = join(v, dpp(v, std::integral_constant<int, 0x140>{}));  // row_mirror
    unsigned lo = (unsigned)__double2loint(v), hi = (unsigned)__double2hiint(v);
    auto a = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), b = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    v = join(__hiloint2double((int)b[0], (int)a[0]), __hiloint2double((int)b[1], (int)a[1]));
    lo = (unsigned)__double2loint(v);
    hi = (unsigned)__double2hiint(v);
    a = __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
    b = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
    return join(__hiloint2double((int)b[0], (int)a[0]), __hiloint2double((int)b[1], (int)a[1]));
}

// The same over the workgroup, in a fixed order; s: a double per wave, not in use by another such call.
template <bool MAX>
__device__ __forceinline__ double bn_block(double v, double* s) {
    v = bn_wave<MAX>(v);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
    for (int w = 1; w < waves; w++) v = MAX ? fmax(v, s[w]) : v + s[w];
    return v;
}

// Chunk c of an optional vector of d floats, ones where it is null: a descriptor of no bytes answers with zeros.
struct BnGain {
    __amdgpu_buffer_rsrc_t r;
    float add;
    __device__ __forceinline__ BnGain(const float* p, int d)
        : r(__builtin_amdgcn_make_buffer_rsrc((void*)p, 0, p ? d * 4 : 0, 0x00027000)), add(p ? 0.f : 1.f) {}
    __device__ __forceinline__ void get(int c, double (&g)[4]) const {
        const u32x4_t u = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, c * 16, 0, 0));
#pragma unroll
        for (int j = 0; j < 4; j++) g[j] = (double)(__uint_as_float(u[j]) + add);
    }
};

// A workgroup takes a row, V chunks of four values a thread: in registers (HELD), or read again for every pass.
template <int V, bool HELD>
__global__ __launch_bounds__(1024) void block_norm_kernel(MoeBlockNorm a) {
    __shared__ double s[3][16];
    const int d4 = a.d / 4, n = blockDim.x, t = blockIdx.x;
    const size_t base = (size_t)t * d4;
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    const BnGain gain_after(a.gain_after, a.d), gate(a.gate, a.d), gain_before(a.gain_before, a.d);
    float4 hx[HELD ? V : 1], hy[HELD ? V : 1];
    double held[HELD ? V : 1][4];  // x', then h
    // f(i, c) for this thread's chunks
    auto each = [&](auto f) __attribute__((always_inline)) {
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                const int c = threadIdx.x + i * n;
                if (c < d4) f(i, c);
            }
        } else {
            for (int c = threadIdx.x; c < d4; c += n) f(0, c);
        }
    };
    auto load_y = [&](int c) __attribute__((always_inline)) { return a.y ? bn_load4<HELD>(a.y, a.y_bf16, base + c) : zero; };
    if (HELD) {
        each([&](int i, int c) __attribute__((always_inline)) { hx[i] = bn_load4<HELD>(a.x, a.x_bf16, base + c); });
        each([&](int i, int c) __attribute__((always_inline)) { hy[i] = load_y(c); });
    }
    double r_after = 1.0;
    if (a.norm_after) {
        double sum = 0.0;
        each([&](int i, int c) __attribute__((always_inline)) {
            const float4 u = HELD ? hy[i] : load_y(c);
            sum += ((double)u.x * u.x + (double)u.y * u.y) + ((double)u.z * u.z + (double)u.w * u.w);
        });
        r_after = 1.0 / sqrt(bn_block<false>(sum, s[0]) / a.d + (double)a.eps);
    }
    const double scale_y = a.y ? (double)a.residual_scale * (a.row_gate ? (double)a.row_gate[t] : 1.0) * r_after : 0.0;
    auto stream = [&](int i, int c, double (&v)[4]) __attribute__((always_inline)) {
        const float4 x = HELD ? hx[i] : bn_load4<HELD>(a.x, a.x_bf16, base + c), y = HELD ? hy[i] : load_y(c);
        const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
        double g[4], q[4];
        gain_after.get(c, g);
        gate.get(c, q);
#pragma unroll
        for (int j = 0; j < 4; j++) v[j] = __builtin_fma((double)ys[j] * g[j] * q[j], scale_y, (double)xs[j]);
    };
    double sum = 0.0;
    each([&](int i, int c) __attribute__((always_inline)) {
        double u[4];
        double(&v)[4] = HELD ? held[i] : u;
        stream(i, c, v);
        if (HELD && a.x_out) bn_store4(a.x_out, a.x_bf16, base + c, v);
        sum += (v[0] * v[0] + v[1] * v[1]) + (v[2] * v[2] + v[3] * v[3]);
    });
    if (a.h || a.codes) {
        const double r = 1.0 / sqrt(bn_block<false>(sum, s[1]) / a.d + (double)a.eps);
        // h of a chunk: left in `held` by the first pass that asks
        auto next = [&](int i, int c, double (&v)[4]) __attribute__((always_inline)) {
            if (!HELD) stream(i, c, v);
            double g[4];
            gain_before.get(c, g);
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] *= r * g[j];
        };
        double top = 0.0;
        unsigned odd = 0u;  // the largest high word: an infinity's or a NaN's is seen in it
        each([&](int i, int c) __attribute__((always_inline)) {
            double u[4];
            double(&v)[4] = HELD ? held[i] : u;
            next(i, c, v);
            if (a.h) bn_store4(a.h, a.h_bf16, base + c, v);
            if (a.codes) {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    top = fmax(top, fabs(v[j]));
                    const unsigned w = (unsigned)__double2hiint(v[j]) & 0x7FFFFFFFu;
                    odd = odd > w ? odd : w;
                }
            }
        });
        if (a.codes) {
            if (__ballot(odd >= 0x7FF00000u) != 0ull) top = INFINITY;
            top = bn_block<true>(top, s[2]);
            const float scale = top < INFINITY ? (float)(top / 127.0) : __uint_as_float(0x7FC00000u);
            if (threadIdx.x == 0) a.scales[t] = scale;
            const double inv = scale > 0.f ? 1.0 / (double)scale : 0.0;
            const bool plain = scale >= 0x1p-126f;  // (a subnormal scale may be too small for the largest values)
            const double magic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low word is the rounded quotient
            each([&](int i, int c) __attribute__((always_inline)) {
                double u[4];
                double(&v)[4] = HELD ? held[i] : u;
                if (!HELD) next(i, c, v);
                int q[4];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    if (plain) q[j] = __double2loint(__builtin_fma(v[j], inv, magic));
                    else q[j] = inv > 0.0 ? (int)fmin(fmax(rint(v[j] * inv), -127.0), 127.0) : 0;
                }
                a.codes[base + c] = i8_pack4(q[0], q[1], q[2], q[3]);
            });
        }
    }
    // rows that are not held: last, when nothing reads x any more (x_out may be x)
    if (!HELD && a.x_out) {
        each([&](int i, int c) __attribute__((always_inline)) {
            double v[4];
            stream(i, c, v);
            bn_store4(a.x_out, a.x_bf16, base + c, v);
        });
    }
}

#define BN_LAUNCH_ROWS (1 << 20)

// Two chunks a thread: a row's requests are all out at once and its passes short.  4096 rows of 4096 (fp32, bf16 -> fp32,
// bf16; cached reads) with 1 / 2 / 4 / 8 chunks a thread (1024 .. 128 threads) 67.7 / 50.7 / 54.7 / 57.5 us, 1000 rows (8-bit codes too) 21.8 /
// 16.4 / 15.2 / 16.8, 301 of 2048 6.7 / 6.0 / 7.9 / 10.8, one 5.6 / 4.8 / 5.1 / 6.9; 2000 of 8192 - / 58.4 / 55.7 / 52.8.
int moe_block_norm_launch(const MoeBlockNorm& a, hipStream_t s) {
    const int d4 = a.d / 4, V = d4 <= 2048 ? 2 : 4;
    const bool held = d4 <= 1024 * V;
    const int waves = held ? (d4 + 64 * V - 1) / (64 * V) : 16;
    auto* kernel = !held ? block_norm_kernel<1, false> : V == 2 ? block_norm_kernel<2, true> : block_norm_kernel<4, true>;
    // (a launch has fewer than 2^32 threads)
    MoeBlockNorm part = a;
    const size_t xb = a.x_bf16 ? 2 : 4, yb = a.y_bf16 ? 2 : 4, hb = a.h_bf16 ? 2 : 4;
    for (int t = 0; t < a.T; t += part.T) {
        const size_t at = (size_t)t * a.d;
        auto step = [&](const void* p, size_t bytes) { return p ? (const char*)p + bytes : nullptr; };
        part.T = a.T - t < BN_LAUNCH_ROWS ? a.T - t : BN_LAUNCH_ROWS;
        part.x = step(a.x, at * xb);
        part.y = step(a.y, at * yb);
        part.row_gate = (const float*)step(a.row_gate, (size_t)t * 4);
        part.x_out = (void*)step(a.x_out, at * xb);
        part.h = (void*)step(a.h, at * hb);
        part.codes = (unsigned*)step(a.codes, at);
        part.scales = (float*)step(a.scales, (size_t)t * 4);
        hipLaunchKernelGGL(kernel, dim3((unsigned)part.T), dim3(64 * waves), 0, s, part);
    }
    return moe_launch_status();
}
