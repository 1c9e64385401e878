// The end of an 8-bit product: a lane's sums, four neighbouring channels of one row, to values.  Every kernel
// family ends in these, so their results are the same bits.  Device code only.
#pragma once

#include "moe_frag_pack.h"
#include "moe_i8.h"

// y[row, c .. c+3] of expert e; channels past C are dropped.
__device__ __forceinline__ void i8_put(const I8Product& p, int e, int c, size_t row, float sx, i32x4_t v) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    if (c >= p.C) return;
    const float* ws = p.ws + (size_t)e * p.C + c;
    const size_t at = row * p.C + c;
    if (p.C % 4 == 0) {
        const float4 sw = *(const float4*)ws;
        const float4 y = make_float4(i8_value(v[0], sx, sw.x), i8_value(v[1], sx, sw.y), i8_value(v[2], sx, sw.z),
                                     i8_value(v[3], sx, sw.w));
        if (p.y_bf16) *(bf16x4*)((__bf16*)p.y + at) = bf16x4{(__bf16)y.x, (__bf16)y.y, (__bf16)y.z, (__bf16)y.w};
        else *(float4*)((float*)p.y + at) = y;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if (c + i >= p.C) continue;
        const float y = i8_value(v[i], sx, ws[i]);
        if (p.y_bf16) ((__bf16*)p.y)[at + i] = (__bf16)y;
        else ((float*)p.y)[at + i] = y;
    }
}

// h = silu(a)*b for a of fragment row fr (w1's) and b of the next one (w3's), NR of them an expert; returns the bits of the
// largest magnitude of the four.
__device__ __forceinline__ unsigned i8_put_gated(const I8Product& p, int e, int NR, int fr, int cq, size_t row, float sx,
                                             i32x4_t a, i32x4_t b) {
    const float* ws = p.ws + ((size_t)e * NR + fr) * 16 + 4 * cq;
    const float4 s1 = *(const float4*)ws, s3 = *(const float4*)(ws + 16);
    const float sa[4] = {s1.x, s1.y, s1.z, s1.w}, sb[4] = {s3.x, s3.y, s3.z, s3.w};
    float h[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float t = i8_value(a[i], sx, sa[i]);
        h[i] = gg_silu(t) * i8_value(b[i], sx, sb[i]);
    }
    *(float4*)((float*)p.y + row * p.C + fr * 8 + 4 * cq) = make_float4(h[0], h[1], h[2], h[3]);
    unsigned top = 0u;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const unsigned m = __float_as_uint(h[i]) & 0x7FFFFFFFu;
        top = top > m ? top : m;
    }
    return top;
}
