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
#include "moe_i8.h"

__device__ __forceinline__ float4 bn_load4(const void* p, bool bf16, size_t chunk) {
    if (bf16) {
        const uint2 u = ((const uint2*)p)[chunk];
        return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                           __uint_as_float(u.y & 0xFFFF0000u));
    }
    return ((const float4*)p)[chunk];
}
__device__ __forceinline__ void bn_store4(void* p, bool bf16, size_t chunk, const double (&v)[4]) {
    if (bf16) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        ((bf16x4*)p)[chunk] = bf16x4{(__bf16)(float)v[0], (__bf16)(float)v[1], (__bf16)(float)v[2], (__bf16)(float)v[3]};
    } else {
        ((float4*)p)[chunk] = make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
    }
}

// Sum (or maximum) over the workgroup, in every thread, in a fixed order; s: one double per wave.
template <bool MAX>
__device__ __forceinline__ double bn_block(double v, double* s) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const double o = __shfl_xor(v, m, 64);
        v = MAX ? fmax(v, o) : v + o;
    }
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
    for (int w = 1; w < waves; w++) v = MAX ? fmax(v, s[w]) : v + s[w];
    return v;
}

// x' of one chunk.
__device__ __forceinline__ void bn_stream4(const MoeBlockNorm& a, size_t row, int c, double r_after, double row_scale,
                                           const float4& x, const float4& y, double (&v)[4]) {
    const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
    float4 g = make_float4(1.f, 1.f, 1.f, 1.f), t = g;
    if (a.gain_after) g = ((const float4*)a.gain_after)[c];
    if (a.gate) t = ((const float4*)a.gate)[c];
    const float gs[4] = {g.x, g.y, g.z, g.w}, ts[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
    for (int i = 0; i < 4; i++)
        v[i] = a.y ? (double)xs[i] + row_scale * ((double)ys[i] * r_after * (double)gs[i] * (double)ts[i]) : (double)xs[i];
}

// V chunks of four values a thread in registers; longer rows are read again for every pass.
template <int V>
__global__ __launch_bounds__(1024) void block_norm_kernel(MoeBlockNorm a) {
    __shared__ double s[16];
    const int d4 = a.d / 4, n = blockDim.x;
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
        const size_t base = (size_t)t * d4;
        const bool held = d4 <= V * n;
        float4 x[V], y[V];
        double v[V][4];
        if (held) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                const int c = threadIdx.x + i * n;
                x[i] = c < d4 ? bn_load4(a.x, a.x_bf16, base + c) : zero;
                y[i] = c < d4 && a.y ? bn_load4(a.y, a.y_bf16, base + c) : zero;
            }
        }
        double r_after = 1.0;
        if (a.norm_after) {
            double sum = 0.0;
            auto add = [&](const float4& u) __attribute__((always_inline)) {
                sum += (double)u.x * u.x + (double)u.y * u.y + (double)u.z * u.z + (double)u.w * u.w;
            };
            if (held) {
#pragma unroll
                for (int i = 0; i < V; i++) add(y[i]);
            } else {
                for (int c = threadIdx.x; c < d4; c += n) add(bn_load4(a.y, a.y_bf16, base + c));
            }
            r_after = 1.0 / sqrt(bn_block<false>(sum, s) / a.d + (double)a.eps);
        }
        const double row_scale = (double)a.residual_scale * (a.row_gate ? (double)a.row_gate[t] : 1.0);
        double sum = 0.0;
        if (held) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                const int c = threadIdx.x + i * n;
                if (c < d4) {
                    bn_stream4(a, base, c, r_after, row_scale, x[i], y[i], v[i]);
                    if (a.x_out) bn_store4(a.x_out, a.x_bf16, base + c, v[i]);
                } else {
                    v[i][0] = v[i][1] = v[i][2] = v[i][3] = 0.0;
                }
#pragma unroll
                for (int j = 0; j < 4; j++) sum += v[i][j] * v[i][j];
            }
        } else {
            for (int c = threadIdx.x; c < d4; c += n) {
                double u[4];
                bn_stream4(a, base, c, r_after, row_scale, bn_load4(a.x, a.x_bf16, base + c),
                           a.y ? bn_load4(a.y, a.y_bf16, base + c) : zero, u);
#pragma unroll
                for (int j = 0; j < 4; j++) sum += u[j] * u[j];
            }
        }
        if (a.h || a.codes) {
            const double r = 1.0 / sqrt(bn_block<false>(sum, s) / a.d + (double)a.eps);
            auto before = [&](int c, double (&u)[4]) __attribute__((always_inline)) {
                float4 g = make_float4(1.f, 1.f, 1.f, 1.f);
                if (a.gain_before) g = ((const float4*)a.gain_before)[c];
                u[0] *= r * (double)g.x;
                u[1] *= r * (double)g.y;
                u[2] *= r * (double)g.z;
                u[3] *= r * (double)g.w;
            };
            double top = 0.0;
            auto largest = [&](const double (&u)[4]) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const double m = fabs(u[j]);
                    top = m <= top ? top : m == m ? m : INFINITY;  // (NaN counts as infinite)
                }
            };
            auto again = [&](int c, double (&u)[4]) __attribute__((always_inline)) {
                bn_stream4(a, base, c, r_after, row_scale, bn_load4(a.x, a.x_bf16, base + c),
                           a.y ? bn_load4(a.y, a.y_bf16, base + c) : zero, u);
                before(c, u);
            };
            if (held) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const int c = threadIdx.x + i * n;
                    if (c >= d4) continue;
                    before(c, v[i]);
                    if (a.h) bn_store4(a.h, a.h_bf16, base + c, v[i]);
                    largest(v[i]);
                }
            } else if (a.codes) {
                for (int c = threadIdx.x; c < d4; c += n) {
                    double u[4];
                    again(c, u);
                    largest(u);
                }
            }
            double inv = 0.0;
            if (a.codes) {
                top = bn_block<true>(top, s);
                const float scale = top < INFINITY ? (float)(top / 127.0) : __uint_as_float(0x7FC00000u);
                if (threadIdx.x == 0) a.scales[t] = scale;
                inv = scale > 0.f ? 1.0 / (double)scale : 0.0;
            }
            auto code = [&](double u) __attribute__((always_inline)) {
                return inv > 0.0 ? (int)fmin(fmax(rint(u * inv), -127.0), 127.0) : 0;
            };
            if (held) {
                if (a.codes) {
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        const int c = threadIdx.x + i * n;
                        if (c < d4) a.codes[base + c] = i8_pack4(code(v[i][0]), code(v[i][1]), code(v[i][2]), code(v[i][3]));
                    }
                }
            } else {
                for (int c = threadIdx.x; c < d4; c += n) {
                    double u[4];
                    again(c, u);
                    if (a.h) bn_store4(a.h, a.h_bf16, base + c, u);
                    if (a.codes) a.codes[base + c] = i8_pack4(code(u[0]), code(u[1]), code(u[2]), code(u[3]));
                }
            }
        }
        // rows that are not held: last, when nothing reads x and y any more (x_out may be either)
        if (!held && a.x_out) {
            for (int c = threadIdx.x; c < d4; c += n) {
                double u[4];
                bn_stream4(a, base, c, r_after, row_scale, bn_load4(a.x, a.x_bf16, base + c),
                           a.y ? bn_load4(a.y, a.y_bf16, base + c) : zero, u);
                bn_store4(a.x_out, a.x_bf16, base + c, u);
            }
        }
        __syncthreads();
    }
}

int moe_block_norm_launch(const MoeBlockNorm& a, hipStream_t s) {
    const int d4 = a.d / 4;
    int threads = 64;
    while (threads < 1024 && threads * 2 < d4) threads *= 2;
    const dim3 grid((unsigned)(a.T < (1 << 20) ? a.T : (1 << 20)));
    hipLaunchKernelGGL(block_norm_kernel<2>, grid, dim3(threads), 0, s, a);
    return moe_launch_status();
}
