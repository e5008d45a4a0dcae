// What the kernels on the rows of a tile stack share (rms_norm.hip, pointwise_i8.hip): a row is a pixel's channels, a stack
// [cap][pixels][C] is cap * pixels of them, and the first min(*count, cap) * pixels are real.
#pragma once
#include "conv_common.h"

namespace sbnet {

__device__ __forceinline__ long long active_rows(const int32_t *count, int cap, int pixels) {
    const int n = min(*count, cap);
    return n > 0 ? (long long)n * pixels : 0;
}

// whether what a call writes holds its count, which the kernels read while others write
inline bool holds_count(const void *q, size_t bytes, const int32_t *count) { return q && ranges_overlap(q, bytes, count, sizeof(int32_t)); }

constexpr float kLeastTop = 7.888609052210118e-31f;                  // 2^-100
constexpr uint32_t kInfBits = 0x7f800000u;

// The 8-bit form of a row whose largest magnitude has the bits `top` (as an unsigned number: NaN is above infinity, infinity
// above everything finite).  Below 2^-100 the scale stays where it is: the reciprocal must not overflow.
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
    r.inv = 127.f * (1.f / t);
    r.scale = t / 127.f;
    return r;
}
// Four codes as bytes.  |v * inv| <= 127 (1 + 2^-21) is first rounded to fp32; added to 3 * 2^22 it is rounded to the nearest whole number,
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

// The rows of a stack that a workgroup has before it: `rows` of them from row `first` on.  What lies behind a row's end is addressed out of the
// buffer's range, which gives zeros and stores nothing without a branch.
template <int DT>
struct Span {
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ Span(const void *stack, long long first, int rows, int C) {
        constexpr int es = DT == SBNET_F32 ? 4 : 2;
        r = __builtin_amdgcn_make_buffer_rsrc((char *)stack + (size_t)first * C * es, 0, stack ? rows * C * es : 0, kBufWord3);
    }
    // place of element i of the span, `left` of them before the row's end
    static __device__ __forceinline__ uint32_t place(uint32_t i, int left) { return left > 0 ? i * (DT == SBNET_F32 ? 4u : 2u) : kOutOfRange; }
};

// 16 neighbouring bytes of a row, for rows that start at multiples of 16 bytes
template <int DT>
struct Piece {
    static constexpr int kType = DT, E = DT == SBNET_F32 ? 4 : 8; // elements
    uint32_t w[4];
    __device__ __forceinline__ void load(const Span<DT> &s, uint32_t i, int left) {
        const uint4 q = buf_load16(s.r, Span<DT>::place(i, left));
        w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
    }
    __device__ __forceinline__ void store(const Span<DT> &s, uint32_t i, int left, bool past_cache = false) const {
        const u32x4 v = {w[0], w[1], w[2], w[3]};
        if (past_cache) __builtin_amdgcn_raw_buffer_store_b128(v, s.r, (int)Span<DT>::place(i, left), 0, 2);      // non-temporal
        else __builtin_amdgcn_raw_buffer_store_b128(v, s.r, (int)Span<DT>::place(i, left), 0, 0);
    }
    __device__ __forceinline__ float get(int e) const {
        if (DT == SBNET_F32) return __uint_as_float(w[e]);
        return e & 1 ? unpack_hi<DT>(w[e >> 1]) : unpack_lo<DT>(w[e >> 1]);
    }
    __device__ __forceinline__ void set(const float *v) {         // rounds to the type
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = DT == SBNET_F32 ? __float_as_uint(v[k]) : pack2<DT>(v[(2 * k) % E], v[(2 * k + 1) % E]);
    }
};

// one element, for the others (16-byte accesses at any address do work, at a lower rate than these: gradients of 28000 rows of 1004 f16 49 us with them, 38
// so).  It is kept as it was loaded: converted at once, every load would be waited for.
template <int DT>
struct Single {
    static constexpr int kType = DT, E = 1;
    uint32_t w;
    __device__ __forceinline__ void load(const Span<DT> &s, uint32_t i, int left) {
        const int at = (int)Span<DT>::place(i, left);
        w = DT == SBNET_F32 ? __builtin_amdgcn_raw_buffer_load_b32(s.r, at, 0, 0) : (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(s.r, at, 0, 0);
    }
    __device__ __forceinline__ void store(const Span<DT> &s, uint32_t i, int left, bool = false) const {
        const int at = (int)Span<DT>::place(i, left);
        if (DT == SBNET_F32) __builtin_amdgcn_raw_buffer_store_b32(w, s.r, at, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b16((unsigned short)w, s.r, at, 0, 0);
    }
    __device__ __forceinline__ float get(int) const { return DT == SBNET_F32 ? __uint_as_float(w) : unpack_lo<DT>(w); }
    __device__ __forceinline__ void set(const float *f) { w = DT == SBNET_F32 ? __float_as_uint(f[0]) : pack2<DT>(f[0], 0.f); }
};

// E neighbouring floats of a vector of n, zeros behind it; with E > 1 n is a multiple of 4
template <int E>
__device__ __forceinline__ void load_floats(float *v, const Span<SBNET_F32> &s, int i, int n) {
    if (E == 1) {
        Single<SBNET_F32> q;
        q.load(s, i, n - i);
        v[0] = q.get(0);
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            Piece<SBNET_F32> q;
            q.load(s, i + e, n - i - e);
            v[e] = q.get(0); v[E > 1 ? e + 1 : 0] = q.get(1); v[E > 1 ? e + 2 : 0] = q.get(2); v[E > 1 ? e + 3 : 0] = q.get(3);
        }
    }
}

}  // namespace sbnet
