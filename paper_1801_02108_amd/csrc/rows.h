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
// Four codes as bytes.  |v * inv| <= 127 (1 + 2^-23) is first rounded to fp32; added to 3 * 2^22 it is rounded to the nearest whole number,
// ties to even, whose lowest byte is that of the sum's bits.  `keep` is 0 for a row that is not finite, else all ones.
__device__ __forceinline__ uint32_t codes4(const float *v, float inv, uint32_t keep) {
#pragma clang fp contract(off)
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float q = v[k] * inv;
        b[k] = __float_as_uint(q + 12582912.f);
    }
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
    return (lo | hi) & keep;
}
__device__ __forceinline__ int8_t code1(float v, float inv, uint32_t keep) {
#pragma clang fp contract(off)
    const float q = v * inv;
    return (int8_t)(__float_as_uint(q + 12582912.f) & keep);
}
__device__ __forceinline__ uint32_t code_keep(uint32_t top) { return top >= kInfBits ? 0u : 0xffffffffu; }

// f over each group of T lanes (8 .. 64, a power of two), the result in every lane, by moves in the vector unit's data path: inside rows of
// 16 lanes a mirror stands for the exchange with the other half, whose lanes all hold the same value by then.
template <int T, typename F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, F f) {
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));              // quad_perm 1 0 3 2
    if (T > 2) v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));   // quad_perm 2 3 0 1
    if (T > 4) v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));  // row_half_mirror
    if (T > 8) v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));  // row_mirror
    if (T > 16) {                                                                                  // rows 0 and 1, 2 and 3
        const auto q = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = f(q[0], q[1]);
    }
    if (T > 32) {
        const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = f(q[0], q[1]);
    }
    return v;
}
struct AddF32 {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }
};
struct MaxU32 {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); }
};
// f over the T threads of a row: lanes of one wave, or the workgroup (`slots`: one word for each of its waves, which the caller does not use
// again before two more barriers)
template <int T, typename F>
__device__ __forceinline__ uint32_t over_row(uint32_t v, F f, uint32_t *slots) {
    if (T <= 64) return over_lanes<T>(v, f);
    v = over_lanes<64>(v, f);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int w = 1; w < T / 64; ++w) v = f(v, slots[w]);
    return v;
}

// ... the sums of two numbers at once
template <int T>
__device__ __forceinline__ void over_row2(float &a, float &b, uint32_t *slots_a, uint32_t *slots_b) {
    constexpr int L = T <= 64 ? T : 64;
    a = __uint_as_float(over_lanes<L>(__float_as_uint(a), AddF32()));
    b = __uint_as_float(over_lanes<L>(__float_as_uint(b), AddF32()));
    if (T <= 64) return;
    if ((threadIdx.x & 63) == 0) {
        slots_a[threadIdx.x >> 6] = __float_as_uint(a);
        slots_b[threadIdx.x >> 6] = __float_as_uint(b);
    }
    __syncthreads();
    a = __uint_as_float(slots_a[0]);
    b = __uint_as_float(slots_b[0]);
#pragma unroll
    for (int w = 1; w < T / 64; ++w) {
        a += __uint_as_float(slots_a[w]);
        b += __uint_as_float(slots_b[w]);
    }
}

// E neighbouring elements of a row: 16 bytes, or one element where rows do not start at multiples of 16 bytes
template <int DT, int E>
struct Piece {
    static constexpr int kWords = E == 1 ? 1 : 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void *p, size_t i) {
        if (E > 1) {
            const uint4 q = *(const uint4 *)((const typename Elem<DT>::T *)p + i);
            w[0] = q.x; w[kWords > 1 ? 1 : 0] = q.y; w[kWords > 2 ? 2 : 0] = q.z; w[kWords > 3 ? 3 : 0] = q.w;
        } else if (DT == SBNET_F32) {
            w[0] = ((const uint32_t *)p)[i];
        } else {
            w[0] = ((const uint16_t *)p)[i];
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = 0;
    }
    __device__ __forceinline__ float get(int e) const {
        if (DT == SBNET_F32) return __uint_as_float(w[e]);
        return e & 1 ? unpack_hi<DT>(w[e >> 1]) : unpack_lo<DT>(w[e >> 1]);
    }
    __device__ __forceinline__ void set(const float *v) {         // rounds to the type
        if (DT == SBNET_F32) {
#pragma unroll
            for (int k = 0; k < kWords; ++k) w[k] = __float_as_uint(v[k]);
        } else if (E == 1) {
            w[0] = pack2<DT>(v[0], 0.f);
        } else {
#pragma unroll
            for (int k = 0; k < kWords; ++k) w[k] = pack2<DT>(v[2 * k], v[E > 1 ? 2 * k + 1 : 0]);
        }
    }
    __device__ __forceinline__ void store(void *p, size_t i) const {
        if (E > 1) *(uint4 *)((typename Elem<DT>::T *)p + i) = make_uint4(w[0], w[kWords > 1 ? 1 : 0], w[kWords > 2 ? 2 : 0], w[kWords > 3 ? 3 : 0]);
        else if (DT == SBNET_F32) ((uint32_t *)p)[i] = w[0];
        else ((uint16_t *)p)[i] = (uint16_t)w[0];
    }
};
// ... of a float32 vector
template <int E>
__device__ __forceinline__ void load_floats(float *v, const float *p, int i) {
#pragma unroll
    for (int e = 0; e < E; e += 4) {
        if (E == 1) { v[0] = p[i]; break; }
        const float4 q = *(const float4 *)(p + i + e);
        v[e] = q.x; v[E > 1 ? e + 1 : 0] = q.y; v[E > 1 ? e + 2 : 0] = q.z; v[E > 1 ? e + 3 : 0] = q.w;
    }
}

}  // namespace sbnet
