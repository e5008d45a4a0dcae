// Root-mean-square norm over a pixel's channels with the residual's addition, its 8-bit form, its gradients, and the row
// quantiser that the 8-bit form shares (sbnet_rms_norm_on_tiles and its neighbours in sbnet.h).
//
//   rms_rows           s = x + residual, r = rsqrt(mean(s^2) + eps), y = s r gain; in 8 bits: y / scale, scale = max|y| / 127
//   rms_backward_rows  with h = s r:  dx = r (gain dy - h mean(gain dy h)) + dsum,  partial sums of dgain = dy h
//   rms_dgain_sum      adds the partial sums in a fixed order
//
// Bound by memory: a row is read once, stays in registers over its sums, and is written once.
#include "rows.h"

namespace sbnet {
namespace {

constexpr int kMaxC = 32768;

enum Form { kNorm, kNormCodes, kCodes };

struct RowArgs {
    const void *x, *res;
    void *sum, *y;               // kNorm
    int8_t *codes;               // kNormCodes, kCodes
    float *scales;
    const float *gain;
    const int32_t *count;
    float eps, inv_c;
    int cap, pixels, C, pitch;
};

__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }

// over the 1024 threads of a workgroup, in a fixed order; `lds` holds 16 values and is free again after the next barrier
template <typename V, typename F>
__device__ __forceinline__ V over_workgroup(V v, F f, V *lds) {
    for (int d = 32; d; d >>= 1) v = f(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < 16; ++w) v = f(v, lds[w]);
    return v;
}

template <int DT, int FORM>
__global__ __launch_bounds__(1024) void rms_rows(RowArgs p) {
    typedef typename Elem<DT>::T T;
    constexpr int P = kMaxC / 1024;
    __shared__ float fl[16];
    __shared__ uint32_t ul[16];
    const long long rows = active_rows(p.count, p.cap, p.pixels);
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        const size_t at = (size_t)row * p.C;
        float s[P], ss = 0.f;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const int c = k * 1024 + threadIdx.x;
            s[k] = 0.f;
            if (c < p.C) {
                s[k] = Elem<DT>::load((const T *)p.x + at + c);
                if (FORM != kCodes && p.res) {
                    T t;
                    Elem<DT>::store(&t, s[k] + Elem<DT>::load((const T *)p.res + at + c));
                    ((T *)p.sum)[at + c] = t;
                    s[k] = Elem<DT>::load(&t);
                }
            }
            ss += s[k] * s[k];
        }
        if (FORM != kCodes) {
            const float r = rsqrtf(over_workgroup(ss, add, fl) * p.inv_c + p.eps);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const int c = k * 1024 + threadIdx.x;
                if (c < p.C) s[k] = s[k] * r * (p.gain ? p.gain[c] : 1.f);
            }
        }
        if (FORM == kNorm) {
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const int c = k * 1024 + threadIdx.x;
                if (c < p.C) Elem<DT>::store((T *)p.y + at + c, s[k]);
            }
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < P; ++k) top = max(top, __float_as_uint(s[k]) & 0x7fffffffu);
            const RowCode rc = row_code(over_workgroup(top, larger, ul));
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const int c = k * 1024 + threadIdx.x;
                if (c < p.pitch) p.codes[(size_t)row * p.pitch + c] = (int8_t)code_of(s[k], rc.inv);
            }
            if (threadIdx.x == 0) p.scales[row] = rc.scale;
        }
    }
}

struct BackArgs {
    const void *s, *dy, *dsum;
    void *dx;
    const float *gain;
    float *part;                 // [workgroups][C]
    const int32_t *count;
    float eps, inv_c;
    int cap, pixels, C;
};

template <int DT>
__global__ __launch_bounds__(1024) void rms_backward_rows(BackArgs p) {
    typedef typename Elem<DT>::T T;
    constexpr int P = kMaxC / 1024;
    __shared__ float fl[2][16];
    const long long rows = active_rows(p.count, p.cap, p.pixels);
    float dg[P];
#pragma unroll
    for (int k = 0; k < P; ++k) dg[k] = 0.f;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        const size_t at = (size_t)row * p.C;
        float s[P], d[P], ss = 0.f, t = 0.f;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const int c = k * 1024 + threadIdx.x;
            s[k] = d[k] = 0.f;
            if (c < p.C) {
                s[k] = Elem<DT>::load((const T *)p.s + at + c);
                d[k] = Elem<DT>::load((const T *)p.dy + at + c);
                t += (p.gain ? p.gain[c] : 1.f) * d[k] * s[k];
            }
            ss += s[k] * s[k];
        }
        const float r = rsqrtf(over_workgroup(ss, add, fl[0]) * p.inv_c + p.eps);
        const float m = over_workgroup(t, add, fl[1]) * p.inv_c * r;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const int c = k * 1024 + threadIdx.x;
            if (c < p.C) {
                const float h = s[k] * r;
                float dx = r * ((p.gain ? p.gain[c] : 1.f) * d[k] - h * m);
                if (p.dsum) dx += Elem<DT>::load((const T *)p.dsum + at + c);
                Elem<DT>::store((T *)p.dx + at + c, dx);
                dg[k] += d[k] * h;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < P; ++k) {
        const int c = k * 1024 + threadIdx.x;
        if (c < p.C) p.part[(size_t)blockIdx.x * p.C + c] = dg[k];
    }
}

__global__ __launch_bounds__(256) void rms_dgain_sum(const float *__restrict__ part, int n, int C, float *__restrict__ dgain) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= C) return;
    float a = 0.f;
    for (int k = 0; k < n; ++k) a += part[(size_t)k * C + c];
    dgain[c] = a;
}

// workgroups of the gradient: each leaves a row of partial sums
int back_grid(long long rows) { return (int)(rows < 512 ? rows : 512); }

sbnet_status check_rows(const char *who, sbnet_dtype dtype, int cap, int pixels, int C, int most) {
    if (!is_float_dtype(dtype)) return fail(SBNET_EUNSUPPORTED, "%s: dtype must be f32, bf16 or f16", who);
    if (cap < 0 || pixels <= 0 || C <= 0) return fail(SBNET_EINVAL, "%s: bad sizes", who);
    if (C > most) return fail(SBNET_EUNSUPPORTED, "%s: more than %d channels", who, most);
    if ((long long)cap * pixels >= (1LL << 31)) return fail(SBNET_EUNSUPPORTED, "%s: too many rows", who);
    return SBNET_OK;
}

// two stacks of the same size either are the same or share nothing
bool clash(const void *a, const void *b, size_t bytes) { return a && b && a != b && ranges_overlap(a, bytes, b, bytes); }

bool eps_ok(float eps) { return eps > 0.f && eps * 0.f == 0.f; }

sbnet_status rows_launch(const char *who, Form form, const void *x, const void *residual, sbnet_dtype dtype, const int32_t *count,
                         int cap, int pixels, int C, const float *gain, float eps, void *sum, void *y, int8_t *codes,
                         float *scales, void *stream) {
    // (an empty stack may have no memory)
    if (!count || (cap != 0 && (!x || (form == kNorm ? !y : !codes || !scales)))) return fail(SBNET_EINVAL, "%s: null pointer", who);
    const sbnet_status st = check_rows(who, dtype, cap, pixels, C, kMaxC);
    if (st != SBNET_OK) return st;
    if (cap != 0 && !residual != !sum) return fail(SBNET_EINVAL, "%s: residual and sum are given together", who);
    if (form != kCodes && !eps_ok(eps)) return fail(SBNET_EINVAL, "%s: eps must be positive and finite", who);
    const int es = elem_bytes(dtype), pitch = (C + 15) / 16 * 16;
    const uintptr_t stacks = (uintptr_t)x | (uintptr_t)residual | (uintptr_t)sum | (uintptr_t)y;
    if (stacks % es || ((uintptr_t)gain | (uintptr_t)scales | (uintptr_t)count) % 4)
        return fail(SBNET_EINVAL, "%s: a pointer is not aligned to its elements", who);
    const size_t rows = (size_t)cap * pixels, bytes = rows * C * es;
    if ((y && y == sum) || clash(y, sum, bytes) || clash(y, x, bytes) || clash(y, residual, bytes) || clash(sum, x, bytes) ||
        clash(sum, residual, bytes))
        return fail(SBNET_EINVAL, "%s: stacks overlap", who);
    if (codes) {
        const void *in[3] = {x, residual, sum};
        for (const void *q : in)
            if (q && (ranges_overlap(codes, rows * pitch, q, bytes) || ranges_overlap(scales, rows * 4, q, bytes)))
                return fail(SBNET_EINVAL, "%s: stacks overlap", who);
        if (ranges_overlap(codes, rows * pitch, scales, rows * 4)) return fail(SBNET_EINVAL, "%s: stacks overlap", who);
    }
    if (cap == 0) return SBNET_OK;
    RowArgs p = {};
    p.x = x; p.res = residual; p.sum = sum; p.y = y; p.codes = codes; p.scales = scales; p.gain = gain; p.count = count;
    p.eps = eps; p.inv_c = 1.f / (float)C; p.cap = cap; p.pixels = pixels; p.C = C; p.pitch = pitch;
    const int grid = (int)(rows < 4096 ? rows : 4096);
    hipStream_t s = (hipStream_t)stream;
#define SBNET_ROWS(DT)                                                                                         \
    do {                                                                                                       \
        if (form == kNorm) hipLaunchKernelGGL((rms_rows<DT, kNorm>), dim3(grid), dim3(1024), 0, s, p);         \
        else if (form == kNormCodes) hipLaunchKernelGGL((rms_rows<DT, kNormCodes>), dim3(grid), dim3(1024), 0, s, p); \
        else hipLaunchKernelGGL((rms_rows<DT, kCodes>), dim3(grid), dim3(1024), 0, s, p);                      \
    } while (0)
    if (dtype == SBNET_F32) SBNET_ROWS(SBNET_F32);
    else if (dtype == SBNET_BF16) SBNET_ROWS(SBNET_BF16);
    else SBNET_ROWS(SBNET_F16);
#undef SBNET_ROWS
    return launch_status(who);
}

}  // namespace
}  // namespace sbnet

using namespace sbnet;

extern "C" sbnet_status sbnet_rms_norm_on_tiles(const void *x, const void *residual, sbnet_dtype dtype, const int32_t *count, int cap,
                                                int pixels, int C, const float *gain, float eps, void *sum, void *y, void *stream) {
    return rows_launch("sbnet_rms_norm_on_tiles", kNorm, x, residual, dtype, count, cap, pixels, C, gain, eps, sum, y, nullptr, nullptr,
                       stream);
}

extern "C" sbnet_status sbnet_rms_norm_i8_on_tiles(const void *x, const void *residual, sbnet_dtype dtype, const int32_t *count, int cap,
                                                   int pixels, int C, const float *gain, float eps, void *sum, int8_t *codes,
                                                   float *scales, void *stream) {
    return rows_launch("sbnet_rms_norm_i8_on_tiles", kNormCodes, x, residual, dtype, count, cap, pixels, C, gain, eps, sum, nullptr, codes,
                       scales, stream);
}

extern "C" sbnet_status sbnet_quantize_i8_on_tiles(const void *x, sbnet_dtype dtype, const int32_t *count, int cap, int pixels, int C,
                                                   int8_t *codes, float *scales, void *stream) {
    return rows_launch("sbnet_quantize_i8_on_tiles", kCodes, x, nullptr, dtype, count, cap, pixels, C, nullptr, 0.f, nullptr, nullptr, codes,
                       scales, stream);
}

extern "C" size_t sbnet_rms_norm_backward_workspace_bytes(int cap, int pixels, int C) {
    if (cap < 0 || pixels <= 0 || C <= 0) return 0;
    const int g = back_grid((long long)cap * pixels);
    return (size_t)(g > 0 ? g : 1) * C * sizeof(float);
}

extern "C" sbnet_status sbnet_rms_norm_backward_on_tiles(const void *s, const void *dy, const void *dsum, sbnet_dtype dtype,
                                                         const int32_t *count, int cap, int pixels, int C, const float *gain, float eps,
                                                         void *dx, float *dgain, void *workspace, size_t workspace_bytes,
                                                         void *stream) {
    const char *who = "sbnet_rms_norm_backward_on_tiles";
    if (!count || !dgain || !workspace || (cap != 0 && (!s || !dy || !dx))) return fail(SBNET_EINVAL, "%s: null pointer", who);
    const sbnet_status st = check_rows(who, dtype, cap, pixels, C, kMaxC);
    if (st != SBNET_OK) return st;
    if (!eps_ok(eps)) return fail(SBNET_EINVAL, "%s: eps must be positive and finite", who);
    const int es = elem_bytes(dtype);
    const uintptr_t stacks = (uintptr_t)s | (uintptr_t)dy | (uintptr_t)dsum | (uintptr_t)dx;
    if (stacks % es || ((uintptr_t)gain | (uintptr_t)dgain | (uintptr_t)count | (uintptr_t)workspace) % 4)
        return fail(SBNET_EINVAL, "%s: a pointer is not aligned to its elements", who);
    const size_t bytes = (size_t)cap * pixels * C * es, need = sbnet_rms_norm_backward_workspace_bytes(cap, pixels, C);
    if (workspace_bytes < need) return fail(SBNET_EINVAL, "%s: workspace too small", who);
    if (clash(dx, s, bytes) || clash(dx, dy, bytes) || clash(dx, dsum, bytes)) return fail(SBNET_EINVAL, "%s: stacks overlap", who);
    const void *in[4] = {s, dy, dsum, dx};
    for (const void *q : in)
        if (q && (ranges_overlap(dgain, (size_t)C * 4, q, bytes) || ranges_overlap(workspace, need, q, bytes)))
            return fail(SBNET_EINVAL, "%s: stacks overlap", who);
    if (ranges_overlap(dgain, (size_t)C * 4, workspace, need)) return fail(SBNET_EINVAL, "%s: workspace overlaps dgain", who);
    BackArgs p = {};
    p.s = s; p.dy = dy; p.dsum = dsum; p.dx = dx; p.gain = gain; p.part = (float *)workspace; p.count = count;
    p.eps = eps; p.inv_c = 1.f / (float)C; p.cap = cap; p.pixels = pixels; p.C = C;
    const int grid = back_grid((long long)cap * pixels);
    hipStream_t q = (hipStream_t)stream;
    if (grid > 0) {
        if (dtype == SBNET_F32) hipLaunchKernelGGL(rms_backward_rows<SBNET_F32>, dim3(grid), dim3(1024), 0, q, p);
        else if (dtype == SBNET_BF16) hipLaunchKernelGGL(rms_backward_rows<SBNET_BF16>, dim3(grid), dim3(1024), 0, q, p);
        else hipLaunchKernelGGL(rms_backward_rows<SBNET_F16>, dim3(grid), dim3(1024), 0, q, p);
        const sbnet_status done = launch_status(who);
        if (done != SBNET_OK) return done;
    }
    hipLaunchKernelGGL(rms_dgain_sum, dim3((C + 255) / 256), dim3(256), 0, q, p.part, grid, C, dgain);
    return launch_status(who);
}
