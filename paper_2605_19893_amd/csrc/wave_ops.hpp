// Sums, scans and maxima over the 64 lanes of a wavefront.
#pragma once
#include <hip/hip_runtime.h>

namespace ssv {

// Scans of a wavefront through the lane shifts of the vector pipe (a step takes a few clocks, an exchange through LDS a hundred):
// within rows of 16 lanes by 1, 2, 4 and 8, then the last lane of a row to the next row, and of the lower half to the upper.
template <int CTRL, int ROWS, typename V>
__device__ __forceinline__ V lane_shift(V x, V none) {
    constexpr int N = sizeof(V) / 4;
    int from[N], to[N];
    __builtin_memcpy(from, &x, sizeof(V));
    __builtin_memcpy(to, &none, sizeof(V));
#pragma unroll
    for (int k = 0; k < N; ++k) to[k] = __builtin_amdgcn_update_dpp(to[k], from[k], CTRL, ROWS, 0xf, false);
    V y;
    __builtin_memcpy(&y, to, sizeof(V));
    return y;
}
template <typename V, typename Op>
__device__ __forceinline__ V wave_scan(V x, V none, Op op) {
    x = op(x, lane_shift<0x111, 0xf>(x, none));      // row_shr 1, 2, 4, 8
    x = op(x, lane_shift<0x112, 0xf>(x, none));
    x = op(x, lane_shift<0x114, 0xf>(x, none));
    x = op(x, lane_shift<0x118, 0xf>(x, none));
    x = op(x, lane_shift<0x142, 0xa>(x, none));      // row_bcast 15 into rows 1 and 3
    return op(x, lane_shift<0x143, 0xc>(x, none));   // row_bcast 31 into rows 2 and 3
}
template <typename V>
__device__ __forceinline__ V last_lane(V x) {
    constexpr int N = sizeof(V) / 4;
    int w[N];
    __builtin_memcpy(w, &x, sizeof(V));
#pragma unroll
    for (int k = 0; k < N; ++k) w[k] = __builtin_amdgcn_readlane(w[k], 63);
    __builtin_memcpy(&x, w, sizeof(V));
    return x;
}
template <typename V>
__device__ __forceinline__ V wave_incl_scan(V x) {
    return wave_scan(x, V(0), [](V p, V q) { return p + q; });
}
template <typename V>
__device__ __forceinline__ V wave_sum(V x) { return last_lane(wave_incl_scan(x)); }
template <typename V>
__device__ __forceinline__ V wave_max(V x) {      // (x itself in place of a lane that is not there: the maximum does not mind)
    x = max(x, lane_shift<0x111, 0xf>(x, x));
    x = max(x, lane_shift<0x112, 0xf>(x, x));
    x = max(x, lane_shift<0x114, 0xf>(x, x));
    x = max(x, lane_shift<0x118, 0xf>(x, x));
    x = max(x, lane_shift<0x142, 0xa>(x, x));
    return last_lane(max(x, lane_shift<0x143, 0xc>(x, x)));
}

}  // namespace ssv
