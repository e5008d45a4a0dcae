// Root-mean-square norm over a pixel's channels with the residual's addition, its 8-bit form, its gradients, and the row
// quantiser that the 8-bit form shares (sbnet_rms_norm_on_tiles and its neighbours in sbnet.h).
//
//   rms_rows           s = x + residual, r = rsqrt(mean(s^2) + eps), y = s r gain; in 8 bits: round(y (127 (1 / t))), scale t / 127,
//                      t = max|y| or 2^-100
//   rms_backward_rows  with h = s r:  dx = r (gain dy - h mean(gain dy h)) + dsum,  partial sums of dgain = dy h
//   rms_dgain_sum      adds the partial sums in a fixed order
//
// Bound by memory: a row is read once, stays in registers over its sums, and is written once.  112640 rows of 256 bf16: with the residual 40 us (5.8 TB/s; a
// large copy reaches 5.0), in 8 bits from 44288 rows of 384 21 to 24 us (5.0 to 5.7 TB/s), without a norm from 142560 of 256 18 to 21 us (5.3 to 6.2 TB/s);
// gradients with the one past the norm 41 us (5.6 TB/s) and 4 for the sums of dgain; 4099 rows of 4096 f32 22 us (6.1 TB/s).
// Of rows of more than 16384 channels a thread holds 32 in 128 registers.  The norm fits (single f32 and bf16 elements: all but 1 to 10 of them; 800 x 32768 bf16
// with the residual 41 us, 5.1 TB/s), the gradients do not: 52 to 312 bytes a lane go through scratch memory (the same rows 77 us, 2.0 TB/s; 1000 x 20001 f16
// by single elements 175, 0.7 TB/s).
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
    int large;                   // the stacks do not stay in the last-level cache
};

// T threads hold a row of up to T * P channels, E of them at a time; the workgroup has 256 threads or, where a wave does not hold a row, one row's.
constexpr int wg_threads(int T) { return T <= 64 ? 256 : T; }

template <class V, int T, int P, int FORM>
__global__ __launch_bounds__(wg_threads(T)) void rms_rows(RowArgs p) {
    constexpr int E = V::E, NV = P / E, RB = wg_threads(T) / T;
    __shared__ uint32_t slots[2][2][16];
    const long long rows = active_rows(p.count, p.cap, p.pixels);
    const int t = threadIdx.x % T;
    const Span<SBNET_F32> gains(p.gain, 0, 1, p.C);
    float gain[P];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * T + t) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) gain[v * E + e] = 1.f;
        if (FORM != kCodes && p.gain) load_floats<E>(gain + v * E, gains, c, p.C);
    }
    int turn = 0;
    for (long long first = (long long)blockIdx.x * RB; first < rows; first += (long long)gridDim.x * RB, turn ^= 1) {
        const long long row = first + threadIdx.x / T;
        if (T <= 64 && row >= rows) break;                        // (a workgroup of one row has no such thread)
        const uint32_t at = threadIdx.x / T * p.C;                // of the rows from `first` on
        const int here = (int)min((long long)RB, rows - first);
        const Span<V::kType> xs(p.x, first, here, p.C), rs(p.res, first, here, p.C), sums(p.sum, first, here, p.C), ys(p.y, first, here, p.C);
        V x[NV], res[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * T + t) * E;
            x[v].load(xs, at + c, p.C - c);
        }
        if (FORM != kCodes && p.res) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * T + t) * E;
                res[v].load(rs, at + c, p.C - c);
            }
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * T + t) * E;
                float sum[E];
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = x[v].get(e) + res[v].get(e);
                x[v].set(sum);
                x[v].store(sums, at + c, p.C - c, p.large);
            }
        }
        float s[P];
#pragma unroll
        for (int k = 0; k < P; ++k) s[k] = x[k / E].get(k % E);
        if (FORM != kCodes) {
            float ss = 0.f;
#pragma unroll
            for (int k = 0; k < P; ++k) ss += s[k] * s[k];
            ss = __uint_as_float(over_row<T>(__float_as_uint(ss), AddF32(), slots[turn][0]));
            const float r = rsqrtf(ss * p.inv_c + p.eps);
#pragma unroll
            for (int k = 0; k < P; ++k) s[k] = s[k] * r * gain[k];
        }
        if (FORM == kNorm) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * T + t) * E;
                x[v].set(s + v * E);
                x[v].store(ys, at + c, p.C - c, p.large);
            }
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < P; ++k) top = max(top, __float_as_uint(s[k]) & 0x7fffffffu);
            top = over_row<T>(top, MaxU32(), slots[turn][1]);
            const RowCode rc = row_code(top);
            const uint32_t keep = code_keep(top);
            int8_t *to = p.codes + (size_t)row * p.pitch;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * T + t) * E;
                if (c >= p.pitch) continue;
                if (E == 1) to[c] = code1(s[v], rc.inv, keep);
                else if (E == 8) *(uint2 *)(to + c) = make_uint2(codes4(s + v * E, rc.inv, keep), codes4(s + v * E + (E == 8 ? 4 : 0), rc.inv, keep));
                else *(uint32_t *)(to + c) = codes4(s + v * E, rc.inv, keep);
            }
            if (t == 0) p.scales[row] = rc.scale;
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

// A thread keeps its channels' sums of dy h over all its rows; the workgroup adds those of its rows' places in ascending order.  With 32 channels a
// thread the gains, and the gradient past the norm until it is added, stay in memory: 512 threads of them then fit their registers, 1024 still do not.
template <class V, int T, int P>
__global__ __launch_bounds__(wg_threads(T)) void rms_backward_rows(BackArgs p) {
    constexpr int E = V::E, NV = P / E, RB = wg_threads(T) / T;
    constexpr bool kKeep = P <= 16;
    __shared__ uint32_t slots[2][3][16];
    __shared__ float sums[RB > 1 ? RB * T * P : 1];
    const long long rows = active_rows(p.count, p.cap, p.pixels);
    const int t = threadIdx.x % T;
    const Span<SBNET_F32> gains(p.gain, 0, 1, p.C);
    float kept[kKeep ? P : 1], dg[P];
    auto load_gain = [&](float *g, int v) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = 1.f;
        if (p.gain) load_floats<E>(g, gains, (v * T + t) * E, p.C);
    };
#pragma unroll
    for (int k = 0; k < P; ++k) dg[k] = 0.f;
    if (kKeep) {
#pragma unroll
        for (int v = 0; v < NV; ++v) load_gain(kept + (kKeep ? v * E : 0), v);
    }
    int turn = 0;
    for (long long first = (long long)blockIdx.x * RB; first < rows; first += (long long)gridDim.x * RB, turn ^= 1) {
        const long long row = first + threadIdx.x / T;
        if (T <= 64 && row >= rows) break;                        // (a workgroup of one row has no such thread)
        const uint32_t at = threadIdx.x / T * p.C;                // of the rows from `first` on
        const int here = (int)min((long long)RB, rows - first);
        const Span<V::kType> xs(p.s, first, here, p.C), ds(p.dy, first, here, p.C), us(p.dsum, first, here, p.C), to(p.dx, first, here, p.C);
        V s[NV], d[NV], past[kKeep ? NV : 1];
        float ss = 0.f, gs = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) s[v].load(xs, at + (v * T + t) * E, p.C - (v * T + t) * E);
#pragma unroll
        for (int v = 0; v < NV; ++v) d[v].load(ds, at + (v * T + t) * E, p.C - (v * T + t) * E);
        if (kKeep && p.dsum) {
#pragma unroll
            for (int v = 0; v < (kKeep ? NV : 1); ++v) past[v].load(us, at + (v * T + t) * E, p.C - (v * T + t) * E);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float g[E];
            if (!kKeep) load_gain(g, v);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float a = s[v].get(e);
                ss += a * a;
                gs += (kKeep ? kept[kKeep ? v * E + e : 0] : g[e]) * d[v].get(e) * a;
            }
        }
        over_row2<T>(ss, gs, slots[turn][0], slots[turn][1]);
        const float r = rsqrtf(ss * p.inv_c + p.eps);
        float m = gs * p.inv_c * r;
        if (r == 0.f) {                                           // the squares pass the range: y = 0 there and so is dx, unless the row holds an infinity
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < P; ++k) top = max(top, __float_as_uint(s[k / E].get(k % E)) & 0x7fffffffu);
            m = over_row<T>(top, MaxU32(), slots[turn][2]) < kInfBits ? 0.f : __uint_as_float(0x7fc00000u);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * T + t) * E;
            V &q = past[kKeep ? v : 0];
            if (!kKeep && p.dsum) q.load(us, at + c, p.C - c);
            float g[E], dx[E];
            if (!kKeep) load_gain(g, v);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float h = s[v].get(e) * r, dy = d[v].get(e);
                dg[v * E + e] += dy * h;
                dx[e] = r * ((kKeep ? kept[kKeep ? v * E + e : 0] : g[e]) * dy - h * m);
                if (p.dsum) dx[e] += q.get(e);
            }
            s[v].set(dx);
            s[v].store(to, at + c, p.C - c);
        }
    }
    float *part = p.part + (size_t)blockIdx.x * p.C;
    if (RB > 1) {
#pragma unroll
        for (int k = 0; k < P; ++k) sums[(threadIdx.x / T) * (T * P) + (k / E * T + t) * E + k % E] = dg[k];
        __syncthreads();
        for (int c = threadIdx.x; c < p.C; c += wg_threads(T)) {
            float a = sums[c];
#pragma unroll
            for (int k = 1; k < RB; ++k) a += sums[k * (T * P) + c];
            part[c] = a;
        }
    } else {
#pragma unroll
        for (int k = 0; k < P; k += E == 1 ? 1 : 4) {
            const int c = (k / E * T + t) * E + k % E;
            if (E == 1) {
                if (c < p.C) part[c] = dg[k];
            } else {
                Piece<SBNET_F32> q;
                q.set(dg + k);
                q.store(Span<SBNET_F32>(part, 0, 1, p.C), c, p.C - c);
            }
        }
    }
}

// dgain[c] = sum over the workgroups' results part[w][c], w < n: 64 channels per workgroup of 16 waves; wave k takes the results
// k, k + 16, ... in ascending order, eight loads in flight, then the 16 sums are added in ascending order
__global__ __launch_bounds__(1024) void rms_dgain_sum(const float *__restrict__ part, int n, int C, float *__restrict__ dgain) {
    __shared__ float slice[16][64];
    const int lane = threadIdx.x & 63, k = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    float acc = 0.f;
    if (c < C) {
        for (int b = k; b < n; b += 128) {
            float a[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int bj = b + 16 * j;
                const float v = part[(size_t)(bj < n ? bj : 0) * C + c];
                a[j] = bj < n ? v : 0.f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) acc += a[j];
        }
    }
    slice[k][lane] = acc;
    __syncthreads();
    if (k == 0 && c < C) {
        float t = slice[0][lane];
#pragma unroll
        for (int i = 1; i < 16; ++i) t += slice[i][lane];
        dgain[c] = t;
    }
}

// Threads and channels per thread by the row's width, f(T, P) as types: lanes of a wave while 16 channels a lane hold the row, a workgroup's threads
// beyond.  (Row quantiser, 3000 rows of 8192: 512 threads of 16 channels 13.8 us, 1024 of 8 16.2; 256 of 32 13.4, but one row then takes 3.4 instead of
// 3.1.  Norm of 14000 rows of 2048: 128 of 16 42.6, 256 of 8 42.2, 64 of 32 41.4, and 23 rows of 2056 in 8 bits 3.8, 3.8 and 4.2.)  From 8193 channels on 512 threads of 32 and 1024 of 16: norm with
// residual of 1500 rows of 16384 bf16 34.6 and 35.4, of 10000 19.8 and 20.2, quantiser 12.6 and 13.2, 9.0 and 10.0; the gradients, for which the split is the
// same, would take 35.7 instead of 42.9, and 45.1 instead of 69.7 by single elements (1700 x 14001 f16).  From 16385 on no other split holds a row.
template <int A, int B> struct Split {
    static constexpr int T = A, P = B;
};
template <typename F>
void by_width(int C, F f) {
    if (C <= 64) f(Split<8, 8>());
    else if (C <= 128) f(Split<16, 8>());
    else if (C <= 256) f(Split<32, 8>());
    else if (C <= 512) f(Split<64, 8>());
    else if (C <= 1024) f(Split<64, 16>());
    else if (C <= 2048) f(Split<128, 16>());
    else if (C <= 4096) f(Split<256, 16>());
    else if (C <= 8192) f(Split<512, 16>());
    else if (C <= 16384) f(Split<512, 32>());
    else f(Split<1024, 32>());
}

// Workgroups of the gradient: each leaves a row of partial sums, so that there are no more than fill the card (112640 x 256 bf16: 512 of 256 threads 44.9
// us, 1024 49.3, 256 60.4; 14000 x 2048: 1024 of 128 threads 40.6, 512 46.5), and from 128 on each has two rows for every place (300 x 8000: 11.4 instead of
// 14.5; 100 x 1000, halved, 6.3 instead of 5.8).
int back_grid(long long rows, int C) {
    int rb = 1, most = 512;
    by_width(C, [&](auto w) {
        constexpr int T = decltype(w)::T;
        rb = wg_threads(T) / T;
        most = wg_threads(T) > 256 ? 256 : 131072 / wg_threads(T);
    });
    const long long want = (rows + rb - 1) / rb;
    if (want <= 3) return want > 0 ? 1 : 0;       // a few rows one after the other end sooner than a second launch (6.3 us a call, 8.5 with it)
    if (want <= 128) return (int)want;
    const long long half = want / 2 > 128 ? (want + 1) / 2 : 128;
    return (int)(half < most ? half : most);
}

sbnet_status check_rows(const char *who, sbnet_dtype dtype, int cap, int pixels, int C, int most) {
    if (!is_float_dtype(dtype)) return fail(SBNET_EUNSUPPORTED, "%s: dtype must be f32, bf16 or f16", who);
    if (cap < 0 || pixels <= 0 || C <= 0) return fail(SBNET_EINVAL, "%s: bad sizes", who);
    if (C > most) return fail(SBNET_EUNSUPPORTED, "%s: more than %d channels", who, most);
    if ((long long)cap * pixels >= (1LL << 31)) return fail(SBNET_EUNSUPPORTED, "%s: too many rows", who);
    return SBNET_OK;
}

// two stacks of the same size either are the same or share nothing
bool clash(const void *a, const void *b, size_t bytes) { return a && b && a != b && ranges_overlap(a, bytes, b, bytes); }

// (of a row of zeros the reciprocal root is eps's alone)
bool eps_ok(float eps) { return eps >= 1.17549435e-38f && eps * 0.f == 0.f; }

template <class V>
void rows_as(Form form, const RowArgs &p, size_t rows, hipStream_t s) {
    by_width(form == kNorm ? p.C : p.pitch, [&](auto w) {         // (the codes fill the padding too)
        constexpr int T = decltype(w)::T, P = decltype(w)::P, RB = wg_threads(T) / T;
        const size_t want = (rows + RB - 1) / RB;
        const int grid = (int)(want < 4096 ? want : 4096);
        if (form == kNorm) hipLaunchKernelGGL((rms_rows<V, T, P, kNorm>), dim3(grid), dim3(wg_threads(T)), 0, s, p);
        else if (form == kNormCodes) hipLaunchKernelGGL((rms_rows<V, T, P, kNormCodes>), dim3(grid), dim3(wg_threads(T)), 0, s, p);
        else hipLaunchKernelGGL((rms_rows<V, T, P, kCodes>), dim3(grid), dim3(wg_threads(T)), 0, s, p);
    });
}
template <class V>
void back_as(const BackArgs &p, int grid, hipStream_t s) {
    by_width(p.C, [&](auto w) {
        constexpr int T = decltype(w)::T, P = decltype(w)::P;
        hipLaunchKernelGGL((rms_backward_rows<V, T, P>), dim3(grid), dim3(wg_threads(T)), 0, s, p);
    });
}
template <int DT>
void rows_go(Form form, bool wide, const RowArgs &p, size_t rows, hipStream_t s) {
    if (wide) rows_as<Piece<DT>>(form, p, rows, s);
    else rows_as<Single<DT>>(form, p, rows, s);
}
template <int DT>
void back_go(bool wide, const BackArgs &p, int grid, hipStream_t s) {
    if (wide) back_as<Piece<DT>>(p, grid, s);
    else back_as<Single<DT>>(p, grid, s);
}

// Whether a call's stacks pass four fifths of the 256 MiB last-level cache: then its results are written past it, for they would be gone before they are read
// again.  (us, through the cache and past it, results to other memory each time, in brackets with a sum of both results behind it.  Norm with residual: 112640 x 256
// bf16, 231 MB, 42.8 and 41.0 (68.7, 69.1); 160000 x 256 60.4 and 58.6 (98.6, 102.2); 250000 x 256 94.1 and 91.3 (155.5, 160.4).  In 8 bits, with the product
// behind it: 160000 x 256 60.7 and 59.7, 250000 x 256 94.9 and 90.7.  Results that go to the same memory every time stay in the cache up to about 300 MB: 130000
// x 256 41.5 and 46.7.  Below the line who reads the results loses more: 44288 x 384 in 8 bits, 119 MB, 26.7 and 22.1 us, with the layer and the norm behind it
// 70.7 and 73.8; 112640 x 256 in 8 bits, 202 MB, 40.4 and 38.9, 101 and 103.)  The stacks count with their capacity: 219 active of 2200 tiles of 324 x 256 take
// 22.5 and, with a norm of the results behind it, 47.6; a list of 219, which goes through the cache, 22.8 and 46.7.
bool large_call(size_t bytes) { return bytes >= ((size_t)1 << 28) / 5 * 4; }

sbnet_status rows_launch(const char *who, Form form, const void *x, const void *residual, sbnet_dtype dtype, const int32_t *count,
                         int cap, int pixels, int C, const float *gain, float eps, void *sum, void *y, int8_t *codes,
                         float *scales, void *stream) {
    // (an empty stack may have no memory)
    if (!count || (cap != 0 && (!x || (form == kNorm ? !y : !codes || !scales)))) return fail(SBNET_EINVAL, "%s: null pointer", who);
    const sbnet_status st = check_rows(who, dtype, cap, pixels, C, kMaxC);
    if (st != SBNET_OK) return st;
    if (cap != 0 && !residual != !sum) return fail(SBNET_EINVAL, "%s: residual and sum are given together", who);
    if (form != kCodes && !eps_ok(eps)) return fail(SBNET_EINVAL, "%s: eps must be a normal number above 0", who);
    const int es = elem_bytes(dtype), pitch = (C + 15) / 16 * 16;
    const uintptr_t stacks = (uintptr_t)x | (uintptr_t)residual | (uintptr_t)sum | (uintptr_t)y;
    if (stacks % es || ((uintptr_t)gain | (uintptr_t)scales | (uintptr_t)count) % 4)
        return fail(SBNET_EINVAL, "%s: a pointer is not aligned to its elements", who);
    const size_t rows = (size_t)cap * pixels, bytes = rows * C * es;
    if ((y && y == sum) || clash(y, sum, bytes) || clash(y, x, bytes) || clash(y, residual, bytes) || clash(sum, x, bytes) ||
        clash(sum, residual, bytes))
        return fail(SBNET_EINVAL, "%s: stacks overlap", who);
    for (const void *q : {(const void *)sum, (const void *)y})
        if (q && gain && ranges_overlap(q, bytes, gain, (size_t)C * 4)) return fail(SBNET_EINVAL, "%s: a stack overlaps gain", who);
    if (codes) {
        if (gain && (ranges_overlap(codes, rows * pitch, gain, (size_t)C * 4) || ranges_overlap(scales, rows * 4, gain, (size_t)C * 4)))
            return fail(SBNET_EINVAL, "%s: a stack overlaps gain", who);
        const void *in[3] = {x, residual, sum};
        for (const void *q : in)
            if (q && (ranges_overlap(codes, rows * pitch, q, bytes) || ranges_overlap(scales, rows * 4, q, bytes)))
                return fail(SBNET_EINVAL, "%s: stacks overlap", who);
        if (ranges_overlap(codes, rows * pitch, scales, rows * 4)) return fail(SBNET_EINVAL, "%s: stacks overlap", who);
    }
    if (holds_count(sum, bytes, count) || holds_count(y, bytes, count) || holds_count(codes, rows * pitch, count) ||
        holds_count(scales, rows * 4, count))
        return fail(SBNET_EINVAL, "%s: a result overlaps count", who);
    if (cap == 0) return SBNET_OK;
    RowArgs p = {};
    p.x = x; p.res = residual; p.sum = sum; p.y = y; p.codes = codes; p.scales = scales; p.gain = gain; p.count = count;
    p.eps = eps; p.inv_c = 1.f / (float)C; p.cap = cap; p.pixels = pixels; p.C = C; p.pitch = pitch;
    p.large = large_call(bytes * (residual ? 3 : 1) + (y ? bytes : rows * pitch));
    // 16-byte accesses where all rows start at multiples of 16 bytes
    const bool wide = ((size_t)C * es | stacks | (uintptr_t)codes | (uintptr_t)gain) % 16 == 0;
    hipStream_t q = (hipStream_t)stream;
    if (dtype == SBNET_F32) rows_go<SBNET_F32>(form, wide, p, rows, q);
    else if (dtype == SBNET_BF16) rows_go<SBNET_BF16>(form, wide, p, rows, q);
    else rows_go<SBNET_F16>(form, wide, p, rows, q);
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
    const int g = back_grid((long long)cap * pixels, C);
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
    if (!eps_ok(eps)) return fail(SBNET_EINVAL, "%s: eps must be a normal number above 0", who);
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
    const size_t cb = (size_t)C * 4;
    if (gain && (ranges_overlap(dx, bytes, gain, cb) || ranges_overlap(dgain, cb, gain, cb) || ranges_overlap(workspace, need, gain, cb)))
        return fail(SBNET_EINVAL, "%s: a result or the workspace overlaps gain", who);
    if (ranges_overlap(dgain, cb, workspace, need)) return fail(SBNET_EINVAL, "%s: workspace overlaps dgain", who);
    if (holds_count(dx, bytes, count) || holds_count(dgain, cb, count) || holds_count(workspace, need, count))
        return fail(SBNET_EINVAL, "%s: a result or the workspace overlaps count", who);
    BackArgs p = {};
    p.s = s; p.dy = dy; p.dsum = dsum; p.dx = dx; p.gain = gain; p.count = count;
    p.eps = eps; p.inv_c = 1.f / (float)C; p.cap = cap; p.pixels = pixels; p.C = C;
    const int grid = back_grid((long long)cap * pixels, C);
    const bool wide = ((size_t)C * es | stacks | (uintptr_t)gain | (uintptr_t)workspace | (uintptr_t)dgain) % 16 == 0;
    p.part = grid == 1 ? dgain : (float *)workspace;              // (one workgroup's sums are the result)
    hipStream_t q = (hipStream_t)stream;
    if (grid > 0) {
        if (dtype == SBNET_F32) back_go<SBNET_F32>(wide, p, grid, q);
        else if (dtype == SBNET_BF16) back_go<SBNET_BF16>(wide, p, grid, q);
        else back_go<SBNET_F16>(wide, p, grid, q);
        const sbnet_status done = launch_status(who);
        if (done != SBNET_OK || grid == 1) return done;
    }
    hipLaunchKernelGGL(rms_dgain_sum, dim3((C + 63) / 64), dim3(1024), 0, q, p.part, grid, C, dgain);
    return launch_status(who);
}
