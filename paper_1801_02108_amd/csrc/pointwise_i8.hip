// Pointwise convolution on tiles in 8-bit integers (sbnet_pointwise_i8_on_tiles): out = act(acc * scale[row] * w_scale[o] +
// bias[o]), acc = sum over the channels of code * weight code, exact in 32 bits (131056 products of at most 2^14).
//
//   i8_quantize_weights  [1][1][Cin][Cout] -> [Cout][pitch] codes and a scale for each output channel
//   i8_pointwise         the product
#include "rows.h"

namespace sbnet {
namespace {

constexpr int kMaxPitch = 131056;

template <int DT>
__global__ __launch_bounds__(256) void i8_quantize_weights(const typename Elem<DT>::T *__restrict__ w, int Cin, int Cout, int pitch,
                                                           int8_t *__restrict__ codes, float *__restrict__ scales) {
    __shared__ uint32_t tops[256];
    const int o = blockIdx.x;
    uint32_t top = 0;
    for (int c = threadIdx.x; c < Cin; c += 256) top = max(top, __float_as_uint(Elem<DT>::load(w + (size_t)c * Cout + o)) & 0x7fffffffu);
    tops[threadIdx.x] = top;
    __syncthreads();
    for (int k = 0; k < 256; ++k) top = max(top, tops[k]);
    const RowCode rc = row_code(top);
    for (int c = threadIdx.x; c < pitch; c += 256)
        codes[(size_t)o * pitch + c] = c < Cin ? code1(Elem<DT>::load(w + (size_t)c * Cout + o), rc.inv, code_keep(top)) : (int8_t)0;
    if (threadIdx.x == 0) scales[o] = rc.scale;
}

struct PointArgs {
    const int8_t *a, *w;
    const float *a_scales, *w_scales, *bias;
    const int32_t *count;
    void *out;
    int cap, pixels, pitch, N, relu;
};

__device__ __forceinline__ float finish(int acc, float a_scale, float w_scale, float bias, int relu) {
    float v = (float)acc * a_scale;
    v = __fadd_rn(__fmul_rn(v, w_scale), bias);
    return relu && v < 0.f ? 0.f : v;             // (a NaN stays one)
}

// 16 x 16 results per workgroup, one per thread, four products per instruction
template <int DT>
__global__ __launch_bounds__(256) void i8_pointwise(PointArgs p) {
    const long long rows = active_rows(p.count, p.cap, p.pixels);
    const long long row = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int o = blockIdx.y * 16 + (threadIdx.x & 15);
    if (row >= rows || o >= p.N) return;
    const int4 *a = (const int4 *)(p.a + (size_t)row * p.pitch), *w = (const int4 *)(p.w + (size_t)o * p.pitch);
    int acc = 0;
    for (int k = 0; k < p.pitch / 16; ++k) {
        const int4 u = a[k], v = w[k];
        acc = __builtin_amdgcn_sdot4(u.x, v.x, acc, false);
        acc = __builtin_amdgcn_sdot4(u.y, v.y, acc, false);
        acc = __builtin_amdgcn_sdot4(u.z, v.z, acc, false);
        acc = __builtin_amdgcn_sdot4(u.w, v.w, acc, false);
    }
    Elem<DT>::store((typename Elem<DT>::T *)p.out + (size_t)row * p.N + o,
                    finish(acc, p.a_scales[row], p.w_scales[o], p.bias ? p.bias[o] : 0.f, p.relu));
}

}  // namespace
}  // namespace sbnet

using namespace sbnet;

extern "C" sbnet_status sbnet_quantize_weights_i8(const void *w_hwio, sbnet_dtype dtype, int Cin, int Cout, int8_t *w_codes,
                                                  float *w_scales, void *stream) {
    const char *who = "sbnet_quantize_weights_i8";
    if (!w_hwio || !w_codes || !w_scales) return fail(SBNET_EINVAL, "%s: null pointer", who);
    if (!is_float_dtype(dtype)) return fail(SBNET_EUNSUPPORTED, "%s: dtype must be f32, bf16 or f16", who);
    if (Cin <= 0 || Cout <= 0) return fail(SBNET_EINVAL, "%s: bad sizes", who);
    if (Cin > kMaxPitch) return fail(SBNET_EUNSUPPORTED, "%s: more than %d input channels", who, kMaxPitch);
    if ((uintptr_t)w_hwio % elem_bytes(dtype) || ((uintptr_t)w_scales & 3) || ((uintptr_t)w_codes & 15))
        return fail(SBNET_EINVAL, "%s: a pointer is not aligned (codes to 16 bytes, others to their elements)", who);
    const int pitch = (Cin + 15) / 16 * 16;
    const size_t wb = (size_t)Cin * Cout * elem_bytes(dtype), cb = (size_t)Cout * pitch, sb = (size_t)Cout * 4;
    if (ranges_overlap(w_hwio, wb, w_codes, cb) || ranges_overlap(w_hwio, wb, w_scales, sb) || ranges_overlap(w_codes, cb, w_scales, sb))
        return fail(SBNET_EINVAL, "%s: arrays overlap", who);
    hipStream_t s = (hipStream_t)stream;
#define SBNET_QW(DT) hipLaunchKernelGGL(i8_quantize_weights<DT>, dim3(Cout), dim3(256), 0, s, (const Elem<DT>::T *)w_hwio, Cin, Cout, \
                                        pitch, w_codes, w_scales)
    if (dtype == SBNET_F32) SBNET_QW(SBNET_F32);
    else if (dtype == SBNET_BF16) SBNET_QW(SBNET_BF16);
    else SBNET_QW(SBNET_F16);
#undef SBNET_QW
    return launch_status(who);
}

extern "C" sbnet_status sbnet_pointwise_i8_on_tiles(const int8_t *codes, const float *scales, const int32_t *count, int cap, int pixels,
                                                    int pitch, const int8_t *w_codes, const float *w_scales, const float *bias,
                                                    int Cout, int relu, sbnet_dtype dtype, void *out, void *stream) {
    const char *who = "sbnet_pointwise_i8_on_tiles";
    if (!count || !w_codes || !w_scales || (cap != 0 && (!codes || !scales || !out))) return fail(SBNET_EINVAL, "%s: null pointer", who);
    if (!is_float_dtype(dtype)) return fail(SBNET_EUNSUPPORTED, "%s: dtype must be f32, bf16 or f16", who);
    if (cap < 0 || pixels <= 0 || pitch <= 0 || Cout <= 0) return fail(SBNET_EINVAL, "%s: bad sizes", who);
    if (pitch % 16) return fail(SBNET_EUNSUPPORTED, "%s: the pitch of the codes must be a multiple of 16", who);
    if (pitch > kMaxPitch) return fail(SBNET_EUNSUPPORTED, "%s: more than %d input channels", who, kMaxPitch);
    if ((long long)cap * pixels >= (1LL << 31)) return fail(SBNET_EUNSUPPORTED, "%s: too many rows", who);
    if (((uintptr_t)codes | (uintptr_t)w_codes | (uintptr_t)out) & 15)
        return fail(SBNET_EINVAL, "%s: codes, w_codes and out must be 16-byte aligned", who);
    if (((uintptr_t)scales | (uintptr_t)w_scales | (uintptr_t)bias | (uintptr_t)count) & 3)
        return fail(SBNET_EINVAL, "%s: a pointer is not aligned to its elements", who);
    const size_t rows = (size_t)cap * pixels, ob = rows * Cout * elem_bytes(dtype);
    if (ranges_overlap(out, ob, codes, rows * pitch) || ranges_overlap(out, ob, scales, rows * 4) ||
        ranges_overlap(out, ob, w_codes, (size_t)Cout * pitch) || ranges_overlap(out, ob, w_scales, (size_t)Cout * 4) ||
        (bias && ranges_overlap(out, ob, bias, (size_t)Cout * 4)))
        return fail(SBNET_EINVAL, "%s: out overlaps an input", who);
    if (cap == 0) return SBNET_OK;
    PointArgs p = {};
    p.a = codes; p.w = w_codes; p.a_scales = scales; p.w_scales = w_scales; p.bias = bias; p.count = count; p.out = out;
    p.cap = cap; p.pixels = pixels; p.pitch = pitch; p.N = Cout; p.relu = relu ? 1 : 0;
    const long long gy = ((long long)Cout + 15) / 16;
    if (gy > 65535) return fail(SBNET_EUNSUPPORTED, "%s: too many output channels", who);
    const dim3 grid((unsigned)((rows + 15) / 16), (unsigned)gy);
    hipStream_t s = (hipStream_t)stream;
    if (dtype == SBNET_F32) hipLaunchKernelGGL(i8_pointwise<SBNET_F32>, grid, dim3(256), 0, s, p);
    else if (dtype == SBNET_BF16) hipLaunchKernelGGL(i8_pointwise<SBNET_BF16>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(i8_pointwise<SBNET_F16>, grid, dim3(256), 0, s, p);
    return launch_status(who);
}
