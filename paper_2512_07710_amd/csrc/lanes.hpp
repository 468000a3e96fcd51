// Scans over the lanes of a wave.
#pragma once
#include <hip/hip_runtime.h>

namespace moe355 {

// inclusive prefix sum over the wave, by lane shifts
template <int CTRL, int ROWS>
__device__ inline int from_lanes(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ inline int wave_scan(int v) {
    v += from_lanes<0x111, 0xf>(v);                            // row_shr 1, 2, 4, 8: rows of 16 lanes
    v += from_lanes<0x112, 0xf>(v);
    v += from_lanes<0x114, 0xf>(v);
    v += from_lanes<0x118, 0xf>(v);
    v += from_lanes<0x142, 0xa>(v);                            // row_bcast 15, 31: over the rows
    v += from_lanes<0x143, 0xc>(v);
    return v;
}

// sum and maximum over the wave, in every lane; the order of the sum is fixed
template <int CTRL, int ROWS>
__device__ inline float float_from_lanes(float none, float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
__device__ inline float last_lane(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63)); }
__device__ inline float wave_total(float v) {
    v += float_from_lanes<0x111, 0xf>(0.f, v);
    v += float_from_lanes<0x112, 0xf>(0.f, v);
    v += float_from_lanes<0x114, 0xf>(0.f, v);
    v += float_from_lanes<0x118, 0xf>(0.f, v);
    v += float_from_lanes<0x142, 0xa>(0.f, v);
    v += float_from_lanes<0x143, 0xc>(0.f, v);
    return last_lane(v);
}
__device__ inline float wave_largest(float v) {
    v = fmaxf(v, float_from_lanes<0x111, 0xf>(-INFINITY, v));
    v = fmaxf(v, float_from_lanes<0x112, 0xf>(-INFINITY, v));
    v = fmaxf(v, float_from_lanes<0x114, 0xf>(-INFINITY, v));
    v = fmaxf(v, float_from_lanes<0x118, 0xf>(-INFINITY, v));
    v = fmaxf(v, float_from_lanes<0x142, 0xa>(-INFINITY, v));
    v = fmaxf(v, float_from_lanes<0x143, 0xc>(-INFINITY, v));
    return last_lane(v);
}

}  // namespace moe355
