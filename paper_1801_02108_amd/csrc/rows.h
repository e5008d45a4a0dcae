// What the kernels on the rows of a tile stack share (rms_norm.hip, pointwise_i8.hip): a row is a pixel's channels, a stack
// [cap][pixels][C] is cap * pixels of them, and the first min(*count, cap) * pixels are real.
#pragma once
#include "conv_common.h"

namespace sbnet {

__device__ __forceinline__ long long active_rows(const int32_t *count, int cap, int pixels) {
    const int n = min(*count, cap);
    return n > 0 ? (long long)n * pixels : 0;
}

constexpr float kLeastTop = 7.888609052210118e-31f;                  // 2^-100
constexpr uint32_t kInfBits = 0x7f800000u;

// The 8-bit form of a row whose largest magnitude has the bits `top` (as an unsigned number: NaN is above infinity, infinity
// above everything finite).  Below 2^-100 the scale stays where it is: 127 / t must not overflow.
struct RowCode {
    float inv, scale;
};
__device__ __forceinline__ RowCode row_code(uint32_t top) {
    RowCode r;
    if (top >= kInfBits) {                        // NaN in the scale stands for the whole row; its codes are 0
        r.inv = 0.f;
        r.scale = __uint_as_float(0x7fc00000u);
        return r;
    }
    const float t = fmaxf(__uint_as_float(top), kLeastTop);
    r.inv = 127.f / t;
    r.scale = t / 127.f;
    return r;
}
// |v * inv| <= 127 (1 + 2^-23): the nearest whole number is within -127 .. 127.  A row that is not finite has inv = 0.
__device__ __forceinline__ int code_of(float v, float inv) { return inv > 0.f ? (int)rintf(v * inv) : 0; }

}  // namespace sbnet
