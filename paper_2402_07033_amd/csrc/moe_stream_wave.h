// What the weight-streaming kernels (moe_ffn_stream.hip, moe_mx_stream.hip) do by one wave before
// their first weight request: the list of row tiles, and the sums of a block's gating shares.
// Device code only.
#pragma once

#include "moe_internal.h"

#define GS_MAX_ITEMS 32                    // T * (E + 1) of the shares, at most
#define GS_WAVE_ROWS 32                    // shares one wave adds

// Adds the shares [row0, row1) (at most GS_WAVE_ROWS) for one wave with few instructions (the
// first weight request of the kernel waits for this): lane r copies row r into LDS, then lane
// `it` adds column `it` in row order.  s_rows: GS_WAVE_ROWS x GS_MAX_ITEMS floats of this
// wave; s_out[it] receives the totals.
__device__ __forceinline__ void gate_add_shares(const float* __restrict__ sums, int row0, int row1,
                                                int stride, int items, int lane, float* s_rows,
                                                float* s_out) {
    const int nrows = row1 - row0;
    if (lane < nrows) {
        // a share is a whole 128-byte line: all of it is copied, whatever `items`
        const float4* src = (const float4*)(sums + (size_t)(row0 + lane) * stride);
        float4* dst = (float4*)(s_rows + lane * GS_MAX_ITEMS);
        const float4 v0 = src[0], v1 = src[1], v2 = src[2], v3 = src[3], v4 = src[4], v5 = src[5],
                     v6 = src[6], v7 = src[7];
        dst[0] = v0; dst[1] = v1; dst[2] = v2; dst[3] = v3;
        dst[4] = v4; dst[5] = v5; dst[6] = v6; dst[7] = v7;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (lane < items) {
        float v = 0.f;
        for (int r = 0; r < nrows; r++) v += s_rows[r * GS_MAX_ITEMS + lane];
        s_out[lane] = v;
    }
}

// Row tiles of the routed rows, built by every wave for itself: lane e takes expert e's
// row range, a wave scan numbers the tiles, and the lane writes its experts' tiles into the
// wave's own copy of the list in LDS.  No workgroup barrier and no serial walk: the list is
// ready one global-load latency after the kernel starts.  Returns the number of tiles.
// lo, hi: lane e's row range [offsets[e], offsets[e+1]) (anything for lanes >= E).
template <int TR, int MAXT>
__device__ __forceinline__ int stream_tile_list(int lo, int hi, int E, int N, int lane, int* te,
                                                int* tr0, int* trn) {
    if (lane >= E) lo = hi = 0;
    lo = lo < 0 ? 0 : (lo > N ? N : lo);
    hi = hi < lo ? lo : (hi > N ? N : hi);
    const int nt = (hi - lo + TR - 1) / TR;
    int incl = nt;
#pragma unroll
    for (int dlt = 1; dlt < 64; dlt <<= 1) {
        const int v = __shfl_up(incl, dlt, 64);
        if (lane >= dlt) incl += v;
    }
    const int first = incl - nt;
    for (int i = 0; i < nt; i++) {
        const int ti = first + i;
        if (ti < MAXT) {
            const int r = lo + i * TR;
            te[ti] = lane;
            tr0[ti] = r;
            trn[ti] = (hi - r) < TR ? (hi - r) : TR;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int total = __shfl(incl, 63, 64);
    return __builtin_amdgcn_readfirstlane(total < MAXT ? total : MAXT);
}
