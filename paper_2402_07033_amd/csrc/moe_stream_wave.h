// The list of row tiles that the weight-streaming kernels (moe_ffn_stream.hip, moe_mx_stream.hip) make by one wave before
// their first weight request.  Device code only.
#pragma once

#include "moe_internal.h"

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
