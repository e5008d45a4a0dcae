// Pointwise convolution on tiles in 8-bit integers (sbnet_pointwise_i8_on_tiles): out = act(acc * scale[row] * w_scale[o] +
// bias[o]), acc = sum over the channels of code * weight code, exact in 32 bits (131056 products of at most 2^14).
//
//   i8_quantize_weights  [1][1][Cin][Cout] -> [Cout][pitch] codes and a scale for each output channel
//   i8_tiles, i8_direct, i8_stream  the product: large, of few rows, of long lists with few weights
#include "rows.h"

namespace sbnet {
namespace {

constexpr int kMaxPitch = 131056, kMaxCout = 1 << 26;

// 32 output channels per workgroup.  Their weights are read twice, 32 neighbouring ones of an input channel at a time, for the largest and for the codes,
// which change rows and columns in LDS: 128 input channels are 128 bytes of an output channel's row.
template <int DT>
__global__ __launch_bounds__(1024) void i8_quantize_weights(const typename Elem<DT>::T *__restrict__ w, int Cin, int Cout, int pitch,
                                                            int8_t *__restrict__ codes, float *__restrict__ scales) {
    __shared__ uint32_t tile[32][33];
    const int ch = threadIdx.x & 31, r = threadIdx.x >> 5;
    const long long o = (long long)blockIdx.x * 32 + ch;
    uint32_t top = 0;
    if (o < Cout)
        for (int c = r; c < Cin; c += 32) top = max(top, __float_as_uint(Elem<DT>::load(w + (size_t)c * Cout + o)) & 0x7fffffffu);
    tile[r][ch] = top;
    __syncthreads();
    for (int k = 0; k < 32; ++k) top = max(top, tile[k][ch]);
    const RowCode rc = row_code(top);
    const uint32_t keep = code_keep(top);
    if (r == 0 && o < Cout) scales[o] = rc.scale;
    const long long oo = (long long)blockIdx.x * 32 + r;          // the channel this thread writes
    for (int c0 = 0; c0 < pitch; c0 += 128) {
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = c0 + 4 * r + k;
            v[k] = o < Cout && c < Cin ? Elem<DT>::load(w + (size_t)c * Cout + o) : 0.f;
        }
        __syncthreads();
        tile[ch][r] = codes4(v, rc.inv, keep);
        __syncthreads();
        if (oo < Cout && c0 + 4 * ch < pitch) *(uint32_t *)(codes + (size_t)oo * pitch + c0 + 4 * ch) = tile[r][ch];
    }
}

struct PointArgs {
    const int8_t *a, *w;
    const float *a_scales, *w_scales, *bias;
    const int32_t *count;
    void *out;
    float least;
    int cap, pixels, pitch, N;
    int wide;                    // rows of out start at multiples of 16 bytes
};

// The result of a sum; `least` is 0 with a ReLU, else -infinity.  (A NaN stays one.)
__device__ __forceinline__ float finish(int acc, float a_scale, float w_scale, float bias, float least) {
#pragma clang fp contract(off)
    const float v = (float)acc * a_scale;
    return __builtin_elementwise_maximum(fmaf(v, w_scale, bias), least);
}

// ---- large products: tiles of BM rows x BN channels through LDS ----------------------------------------------------------
// 32 x 32 x 32 steps of the matrix unit: its first operand is the weights (32 channels), its second the activations (32 rows), 16 bytes of
// codes per lane each, so that a lane's 16 sums are channels of one row.  In LDS both operands are rows of 128 bytes, piece q of row i
// at place q ^ (i / 2 % 8): the 16-byte reads of 16 neighbouring rows fall on different banks.  Row i of 32 weight rows is channel
// 16 (i / 16) + 8 (i / 4 % 2) + 4 (i / 8 % 2) + i % 4, which makes a lane's sums two times 8 neighbouring channels, next to the other half's.
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4;
typedef __attribute__((__vector_size__(16 * sizeof(int)))) int i32x16;
typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ i32x16 mfma_i8(uint4 a, uint4 b, i32x16 c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint4 read16(const lds_byte *p) {
    const u32x4 v = *(const __attribute__((address_space(3))) u32x4 *)p;
    return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ int channel_of_row(int i) { return (i & 16) + 8 * ((i >> 2) & 1) + 4 * ((i >> 3) & 1) + (i & 3); }

// 8 floats from LDS
__device__ __forceinline__ void load8(float *v, const float *p) {
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
        const float4 q = *(const float4 *)(p + e);
        v[e] = q.x; v[e + 1] = q.y; v[e + 2] = q.z; v[e + 3] = q.w;
    }
}

// The results of 8 (4) neighbouring channels of one row, `left` of them there are.  Where rows do not start at multiples of 16 bytes the memory units take
// the same stores at any address: single ones take longer (33280 x 928 x 419 35 us, with eight single stores 69; 112640 x 64 x 250 17 and 64).
typedef uint32_t any_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t any_u32x2 __attribute__((ext_vector_type(2), aligned(2)));
template <int DT>
__device__ __forceinline__ void store8(void *out, size_t at, const float *v, int left) {
    typedef typename Elem<DT>::T T;
    if (left >= 8) {
        if (DT == SBNET_F32) {
            *(any_u32x4 *)((T *)out + at) = (any_u32x4){__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
            *(any_u32x4 *)((T *)out + at + 4) = (any_u32x4){__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
        } else {
            *(any_u32x4 *)((T *)out + at) = (any_u32x4){pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]), pack2<DT>(v[4], v[5]), pack2<DT>(v[6], v[7])};
        }
    } else {
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (k < left) Elem<DT>::store((T *)out + at + k, v[k]);
    }
}
template <int DT>
__device__ __forceinline__ void store4(void *out, size_t at, const float *v, int left) {
    typedef typename Elem<DT>::T T;
    if (left >= 4) {
        if (DT == SBNET_F32) *(any_u32x4 *)((T *)out + at) = (any_u32x4){__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        else *(any_u32x2 *)((T *)out + at) = (any_u32x2){pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3])};
    } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < left) Elem<DT>::store((T *)out + at + k, v[k]);
    }
}

constexpr int kStageK = 128;                      // bytes of a row in a stage

// Waves 0 .. 3 multiply, WM x WN of them, each MF x NF blocks of 32 x 32; waves 4 .. 7 move the operands from memory to LDS, up to two stages ahead,
// across the borders of tiles.  One barrier a stage: before it stage k has been read to the end and stage k + 1 has landed.
// Bound, one workgroup a CU, by the CU's intake (a stage takes about 15 ns a KB: 0.70 us for 256 x 128, whose matrix steps are 0.43), and on the whole card by its
// power (the clock falls to 1.76 GHz).  8192 x 4096 x 8192: 248 to 265 us, 2.1 to 2.2 POP/s; 4096 x 4096 x 4096 65 us.  Moving waves of their own because a wave stands at
// the copies that it asks for: 329 us where the multiplying waves ask.
template <int DT, int WM, int WN, int MF, int NF>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
void i8_tiles(PointArgs p) {
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32;
    constexpr int kStage = (BM + BN) * kStageK, kScales = (BM + 2 * BN) * 4;
    constexpr int kCopies = (BM + BN) / 8 / 4;    // per moving wave and stage, 8 rows each
    constexpr int kScaleCopies = (BM + 2 * BN) / 64, kScaleEach = (kScaleCopies + 3) / 4;
    extern __shared__ __align__(16) char lds[];
    lds_byte *const ldsb = (lds_byte *)lds;
    lds_byte *const scaleb = ldsb + 3 * kStage;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long rows = active_rows(p.count, p.cap, p.pixels);
    const int tm = (int)((rows + BM - 1) / BM), tn = (p.N + BN - 1) / BN, nk = (p.pitch + kStageK - 1) / kStageK;
    // Tiles in bands of 8 along the rows, column by column; workgroups of one die (every eighth) take neighbouring ones, for its cache
    const long long tiles = (long long)tm * tn;
    const int G = gridDim.x;
    const int place = G % 8 == 0 ? (int)(blockIdx.x % 8) * (G / 8) + (int)blockIdx.x / 8 : (int)blockIdx.x;
    const int mine = place < tiles ? (int)((tiles - place + G - 1) / G) : 0;
    const int total = mine * nk;                  // stages
    if (total == 0) return;
    auto tile_at = [&](int j, long long &row0, int &n0) __attribute__((always_inline)) {
        const long long pos = place + (long long)j * G, band = pos / (8LL * tn);
        const int in = (int)(pos - band * 8 * tn), high = min(8, tm - (int)band * 8);
        const int col = in / high;
        row0 = (band * 8 + (in - col * high)) * BM;
        n0 = col * BN;
    };

    if (wave >= 4) {
        const int w = wave - 4;
        uint32_t rel[kCopies];                    // copy w + 4 i of a stage: rows 8 (w + 4 i) ..
        const uint32_t kb = (uint32_t)(((lane & 7) ^ ((w * 4 + (lane >> 4)) & 7)) * 16);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int r = (w + 4 * i) * 8 + (lane >> 3);
            const int src = r < BM ? r : ((r - BM) & ~31) + channel_of_row((r - BM) & 31);
            rel[i] = (uint32_t)src * p.pitch + kb;
        }
        int j = -1, ks = nk;                      // the tile and stage in it that are requested next
        long long row0 = 0;
        int n0 = 0;
        auto move = [&](int k) __attribute__((always_inline)) {
            if (++ks >= nk) {
                ks = 0;
                ++j;
                tile_at(j, row0, n0);
            }
            const uint32_t here = (uint32_t)min((long long)BM, rows - row0), wide = (uint32_t)min(BN, p.N - n0);
            const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a + (size_t)row0 * p.pitch), 0, (int)(here * p.pitch), kBufWord3);
            const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc((void *)(p.w + (size_t)n0 * p.pitch), 0, (int)(wide * p.pitch), kBufWord3);
            const uint32_t k0 = (uint32_t)ks * kStageK;
            lds_byte *to = ldsb + (k % 3) * kStage + w * 1024;
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                // (bytes behind the row's end are the next row's: not fetched, and zero in LDS)
                const uint32_t off = k0 + kb < (uint32_t)p.pitch ? rel[i] + k0 : kOutOfRange;
                if (i * 32 < BM) __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (lds_void *)(to + i * 4096), 16, (int)off, 0, 0, 0);
                else __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void *)(to + i * 4096), 16, (int)off, 0, 0, 0);
            }
            if (ks == 0) {                        // the tile's scales and biases, 64 at a time
                const __amdgpu_buffer_rsrc_t sr = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a_scales + row0), 0, (int)(here * 4), kBufWord3);
                const __amdgpu_buffer_rsrc_t cr = __builtin_amdgcn_make_buffer_rsrc((void *)(p.w_scales + n0), 0, (int)(wide * 4), kBufWord3);
                const __amdgpu_buffer_rsrc_t br = __builtin_amdgcn_make_buffer_rsrc((void *)(p.bias ? p.bias + n0 : p.w_scales), 0,
                                                                                     p.bias ? (int)(wide * 4) : 0, kBufWord3);
                lds_byte *st = scaleb + (j & 3) * kScales;
#pragma unroll
                for (int i = 0; i < kScaleEach; ++i) {
                    const int c = min(w + 4 * i, kScaleCopies - 1);       // (every wave the same number: some do the last one again)
                    if (c < BM / 64) __builtin_amdgcn_raw_ptr_buffer_load_lds(sr, (lds_void *)(st + c * 256), 4, (c * 64 + lane) * 4, 0, 0, 0);
                    else if (c < (BM + BN) / 64)
                        __builtin_amdgcn_raw_ptr_buffer_load_lds(cr, (lds_void *)(st + c * 256), 4, ((c - BM / 64) * 64 + lane) * 4, 0, 0, 0);
                    else __builtin_amdgcn_raw_ptr_buffer_load_lds(br, (lds_void *)(st + c * 256), 4, ((c - (BM + BN) / 64) * 64 + lane) * 4, 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        // until all but the newest stage has landed; a tile's first stage has its scales' copies too
        auto wait = [&](bool newest, bool first) __attribute__((always_inline)) {
            constexpr int A = kCopies, B = kCopies + kScaleEach;
            if (!newest) __builtin_amdgcn_s_waitcnt(0x0F70);
            else if (first) __builtin_amdgcn_s_waitcnt(0x0F70 | (B & 15) | ((B >> 4) << 14));
            else __builtin_amdgcn_s_waitcnt(0x0F70 | (A & 15) | ((A >> 4) << 14));
        };
        move(0);
        if (total > 1) move(1);
        wait(total > 1, ks == 0);
        __builtin_amdgcn_s_barrier();             // stage 0 is there
        if (total > 2) move(2);
        for (int k = 0; k < total; ++k) {
            wait(k + 2 < total, ks == 0);         // stage k + 1
            __builtin_amdgcn_s_barrier();
            if (k + 3 < total) move(k + 3);
        }
    } else {
        const int wm = wave / WN, wn = wave % WN;
        const int l32 = lane & 31, h = lane >> 5;
        uint32_t at[4];                           // this lane's piece of 32 rows at step 0 .. 3 of a stage
#pragma unroll
        for (int s = 0; s < 4; ++s) at[s] = (uint32_t)(l32 * 128 + (((2 * s + h) ^ ((l32 >> 1) & 7)) * 16));
        const lds_byte *abase = ldsb + wm * MF * 4096, *wbase = ldsb + BM * 128 + wn * NF * 4096;
        uint4 fa[2][MF], fw[2][NF];
        auto fetch = [&](int set, const lds_byte *a, const lds_byte *w, int s) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < NF; ++n) fw[set][n] = read16(w + at[s] + n * 4096);
#pragma unroll
            for (int m = 0; m < MF; ++m) fa[set][m] = read16(a + at[s] + m * 4096);
        };
        i32x16 acc[MF][NF];
        auto multiply = [&](int set) __attribute__((always_inline)) {
#pragma unroll
            for (int m = 0; m < MF; ++m)
#pragma unroll
                for (int n = 0; n < NF; ++n) acc[m][n] = mfma_i8(fw[set][n], fa[set][m], acc[m][n]);
        };
        __syncthreads();                          // stage 0
        fetch(0, abase, wbase, 0);
        int k = 0, slot = 0;
        for (int j = 0; j < mine; ++j) {
#pragma unroll
            for (int m = 0; m < MF; ++m)
#pragma unroll
                for (int n = 0; n < NF; ++n)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[m][n][e] = 0;
            for (int ks = 0; ks < nk; ++ks, ++k) {
                const lds_byte *a = abase + slot * kStage, *w = wbase + slot * kStage;
                slot = slot == 2 ? 0 : slot + 1;
                fetch(1, a, w, 1);
                __builtin_amdgcn_sched_barrier(0);
                multiply(0);
                __builtin_amdgcn_sched_barrier(0);
                fetch(0, a, w, 2);
                __builtin_amdgcn_sched_barrier(0);
                multiply(1);
                __builtin_amdgcn_sched_barrier(0);
                fetch(1, a, w, 3);
                __builtin_amdgcn_sched_barrier(0);
                multiply(0);
                __builtin_amdgcn_sched_barrier(0);
                __syncthreads();                  // everything of this stage is in registers; the next one has landed
                if (k + 1 < total) fetch(0, abase + slot * kStage, wbase + slot * kStage, 0);
                __builtin_amdgcn_sched_barrier(0);
                multiply(1);
                __builtin_amdgcn_sched_barrier(0);
            }
            long long row0;
            int n0;
            tile_at(j, row0, n0);
            const float *sc = (const float *)(lds + 3 * kStage + (j & 3) * kScales);
            float as[MF];
#pragma unroll
            for (int m = 0; m < MF; ++m) as[m] = sc[(wm * MF + m) * 32 + l32];
#pragma unroll
            for (int n = 0; n < NF; ++n)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int c = (wn * NF + n) * 32 + 16 * g + 8 * h;
                    if (n0 + c >= p.N) continue;
                    float ws[8], bs[8];
                    load8(ws, sc + BM + c);
                    load8(bs, sc + BM + BN + c);
#pragma unroll
                    for (int m = 0; m < MF; ++m) {
                        const long long row = row0 + (wm * MF + m) * 32 + l32;
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = finish(acc[m][n][8 * g + e], as[m], ws[e], bs[e], p.least);
                        if (row < rows) store8<DT>(p.out, (size_t)row * p.N + n0 + c, v, p.N - n0 - c);
                    }
                }
        }
    }
}

// ---- small products: 16 MT rows x 16 NT channels per workgroup, operands from memory to registers, the channels summed over split between its waves
// 16 x 16 x 64 steps, weights as the first operand again.  Wave w of KS takes the pieces of 128 bytes w, w + KS, ... of every row; the waves' sums
// meet in LDS.  Frag n of NT holds channels 4 NT q + 4 n + r in its row 4 q + r, which gives a lane 4 NT neighbouring channels.
// Bound by latency (few rows: by the weights' bytes): a wave requests U pieces of all its rows and, before it multiplies them, the next U.  (That request is behind
// a branch, so that the waits count it as not made: all of it has landed before the last step of the first U.)  1 x 4096 x 4096: 5.4 us, 2.7 of them
// the launch, 6 TB/s for the rest; 23 x 2056 x 5125 5.8 us; 300 x 368 x 360 4.1 us.
__device__ __forceinline__ i32x4 mfma_i8_16(uint4 a, uint4 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

template <int DT, int MT, int NT, int KS>
__global__ __launch_bounds__(64 * KS) void i8_direct(PointArgs p) {
    constexpr int U = MT + NT <= 2 ? 4 : MT + NT <= 4 ? 2 : 1;
    constexpr int F = MT * NT;                    // fragments of 16 x 16
    __shared__ int4 sums[KS][F][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long rows = active_rows(p.count, p.cap, p.pixels);
    const int tm = (int)((rows + 16 * MT - 1) / (16 * MT));
    // workgroups of one die (every eighth) take neighbouring tiles along the rows: they share weights
    const int G = gridDim.x;
    const int place = G % 8 == 0 ? (int)(blockIdx.x % 8) * (G / 8) + (int)blockIdx.x / 8 : (int)blockIdx.x;
    const int col = place / max(tm, 1), n0 = col * 16 * NT;
    const long long row0 = (long long)(place - col * tm) * (16 * MT);
    if (rows == 0 || n0 >= p.N) return;
    const uint32_t here = (uint32_t)min(16LL * MT, rows - row0), wide = (uint32_t)min(16 * NT, p.N - n0);
    const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a + (size_t)row0 * p.pitch), 0, (int)(here * p.pitch), kBufWord3);
    const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc((void *)(p.w + (size_t)n0 * p.pitch), 0, (int)(wide * p.pitch), kBufWord3);
    // the results this thread finishes: fragment f of 64 lanes, 4 channels of a row
    float as[(F + KS - 1) / KS], ws[(F + KS - 1) / KS][4], bs[(F + KS - 1) / KS][4];
#pragma unroll
    for (int i = 0; i < (F + KS - 1) / KS; ++i) {
        const int f = wave + i * KS, m = f / NT, n = f % NT;
        const int r = m * 16 + l16, c = 4 * NT * q + 4 * n;
        as[i] = f < F && (uint32_t)r < here ? p.a_scales[row0 + r] : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool ok = f < F && c + e < (int)wide;
            ws[i][e] = ok ? p.w_scales[n0 + c + e] : 0.f;
            bs[i][e] = ok && p.bias ? p.bias[n0 + c + e] : 0.f;
        }
    }
    uint32_t arel[MT], wrel[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) arel[m] = (uint32_t)(m * 16 + l16) * p.pitch;
#pragma unroll
    for (int n = 0; n < NT; ++n) wrel[n] = (uint32_t)(4 * NT * (l16 >> 2) + 4 * n + (l16 & 3)) * p.pitch;
    const int pieces = (p.pitch + 127) / 128, mine = wave < pieces ? (pieces - wave + KS - 1) / KS : 0;
    struct Ops { uint4 a[U][2][MT], w[U][2][NT]; };
    auto load = [&](Ops &o, int i) __attribute__((always_inline)) {           // pieces i .. i + U - 1 of this wave; zeros behind the row's end
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint32_t k = (uint32_t)(wave + (i + u) * KS) * 128 + s * 64 + q * 16;
                const bool in = k < (uint32_t)p.pitch;
#pragma unroll
                for (int n = 0; n < NT; ++n) o.w[u][s][n] = buf_load16(wr, in ? wrel[n] + k : kOutOfRange);
#pragma unroll
                for (int m = 0; m < MT; ++m) o.a[u][s][m] = buf_load16(ar, in ? arel[m] + k : kOutOfRange);
            }
    };
    i32x4 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = (i32x4){0, 0, 0, 0};
    auto multiply = [&](const Ops &o) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[m][n] = mfma_i8_16(o.w[u][s][n], o.a[u][s][m], acc[m][n]);
    };
    Ops o0, o1;
    if (mine > 0) load(o0, 0);
    for (int i = 0; i < mine; i += 2 * U) {
        if (i + U < mine) load(o1, i + U);
        multiply(o0);
        if (i + U < mine) {
            if (i + 2 * U < mine) load(o0, i + 2 * U);
            multiply(o1);
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) sums[wave][m * NT + n][lane] = make_int4(acc[m][n][0], acc[m][n][1], acc[m][n][2], acc[m][n][3]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < (F + KS - 1) / KS; ++i) {
        const int f = wave + i * KS, m = f / NT, n = f % NT;
        if (f >= F) break;
        int4 t = sums[0][f][lane];
#pragma unroll
        for (int w = 1; w < KS; ++w) {
            const int4 u = sums[w][f][lane];
            t.x += u.x; t.y += u.y; t.z += u.z; t.w += u.w;
        }
        const int r = m * 16 + l16, c = n0 + 4 * NT * q + 4 * n;
        const float v[4] = {finish(t.x, as[i], ws[i][0], bs[i][0], p.least), finish(t.y, as[i], ws[i][1], bs[i][1], p.least),
                            finish(t.z, as[i], ws[i][2], bs[i][2], p.least), finish(t.w, as[i], ws[i][3], bs[i][3], p.least)};
        if ((uint32_t)r < here) store4<DT>(p.out, (size_t)(row0 + r) * p.N + c, v, p.N - c);
    }
}

// ---- long lists, few weights: all weights lie in LDS, every wave streams rows past them, 16 at a time
// 16 x 16 x 64 steps on 64 channels at a time.  The weights are laid out in LDS as the operand reads take them, 1 KB each, once a workgroup.  Frags 2 s
// and 2 s + 1 hold channels 32 s + 8 q + 4 (n % 2) + r in their rows 4 q + r: a lane's pair is 8 neighbouring channels, and one 16-byte store of
// a wave is 64 bytes of each of 16 rows.
// Bound by memory, which twelve waves a CU keep busy (eight waves of 32 rows: 112640 x 256 x 256 22.0 us instead of 20.2, 142560 x 256 x 64 13.3 and 12.6, which is
// 4.4 TB/s).  A wave requests the next 16 rows before it multiplies these, but it also waits for them there: the loop over the groups stores, and in front of
// it nothing may be outstanding.  So the overlap is between waves, not within one.
//
// Results no wider than the input (in channels) are written past the cache, which is left to the codes, in whole lines: 112640 x 128 x 128 11.9 us and, with a
// pass over the results behind it, 21.5; so 8.9 and 21.0; 142560 x 256 x 64 13.1 and 20.0, 12.0 and 20.0; 112640 x 256 x 256 21.4 and 40.0, 18.7 and 39.3.
// Wider ones gain alone and lose with who reads them: 60000 x 64 x 512 15.8 and 34.0, 14.4 and 35.5.  Short lists neither gain nor lose: 20000 x 256 x 64 4.5
// and 8.4, past the cache 4.4 and 8.3; 12000 x 128 x 128 4.4 and 8.2, 4.6 and 8.3; 40000 x 128 x 128 6.1 and 10.3, 5.2 and 9.8.
constexpr int kStreamWaves = 12;

// lanes 8 .. 15 of each 16 of a with lanes 0 .. 7 of b
__device__ __forceinline__ void swap8(uint32_t &a, uint32_t &b) {
    const uint32_t u = (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)b, 0x128, 0xf, 0xc, false);      // row_ror:8 into the upper eight
    b = (uint32_t)__builtin_amdgcn_update_dpp((int)b, (int)a, 0x128, 0xf, 0x3, false);
    a = u;
}

template <int DT, int KC>
__global__ __launch_bounds__(64 * kStreamWaves, 3) void i8_stream(PointArgs p, int groups) {
    extern __shared__ __align__(16) char lds[];                   // [groups][KC][4] fragments of 1 KB, then scales and biases
    lds_byte *const ldsb = (lds_byte *)lds;
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long rows = active_rows(p.count, p.cap, p.pixels);
    long long row0 = ((long long)wave * gridDim.x + blockIdx.x) * 16;            // (few steps go to as many workgroups)
    const long long stride = (long long)gridDim.x * kStreamWaves * 16;
    if ((long long)blockIdx.x * 16 >= rows) return;
    uint32_t k[KC];
#pragma unroll
    for (int i = 0; i < KC; ++i) k[i] = (uint32_t)(i * 64 + q * 16) < (uint32_t)p.pitch ? (uint32_t)(l16 * p.pitch + i * 64 + q * 16) : kOutOfRange;
    struct Rows {
        uint4 a[KC];
        float scale;
    };
    auto load = [&](Rows &o, long long at) __attribute__((always_inline)) {
        const uint32_t here = (uint32_t)max(0LL, min(16LL, rows - at));
        const __amdgpu_buffer_rsrc_t ar = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a + (size_t)at * p.pitch), 0, (int)(here * p.pitch), kBufWord3);
        const __amdgpu_buffer_rsrc_t sr = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a_scales + at), 0, (int)(here * 4), kBufWord3);
#pragma unroll
        for (int i = 0; i < KC; ++i) o.a[i] = buf_load16(ar, k[i]);
        o.scale = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sr, l16 * 4, 0, 0));
    };
    const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc((void *)p.w, 0, (int)((uint32_t)p.N * p.pitch), kBufWord3);
    for (int f = wave; f < groups * KC * 4; f += kStreamWaves) {
        const int g = f / (KC * 4), i = f / 4 % KC, n = f % 4;
        const uint32_t at = (uint32_t)(i * 64 + q * 16), o = (uint32_t)(g * 64 + (n >> 1) * 32 + (l16 >> 2) * 8 + (n & 1) * 4 + (l16 & 3));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void *)(ldsb + f * 1024), 16,
                                                 (int)(at < (uint32_t)p.pitch ? o * p.pitch + at : kOutOfRange), 0, 0, 0);
    }
    float *const sc = (float *)(lds + groups * KC * 4096);       // [groups][64] scales, then biases
    for (int c = threadIdx.x; c < groups * 64; c += 64 * kStreamWaves) {
        sc[c] = c < p.N ? p.w_scales[c] : 0.f;
        sc[groups * 64 + c] = c < p.N && p.bias ? p.bias[c] : 0.f;
    }
    const bool past_cache = DT != SBNET_F32 && p.wide && p.N <= p.pitch;
    Rows o0, o1;
    load(o0, row0);
    __syncthreads();
    auto step = [&](const Rows &o, long long at) __attribute__((always_inline)) {
        const long long row = at + l16;
        for (int g = 0; g < groups; ++g) {
            const lds_byte *wf = ldsb + g * KC * 4096 + lane * 16;
            i32x4 acc[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) acc[n] = (i32x4){0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < KC; ++i)
#pragma unroll
                for (int n = 0; n < 4; ++n) acc[n] = mfma_i8_16(read16(wf + (i * 4 + n) * 1024), o.a[i], acc[n]);
            float v[2][8];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float ws[8], bs[8];
                load8(ws, sc + g * 64 + s * 32 + q * 8);
                load8(bs, sc + (groups + g) * 64 + s * 32 + q * 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[s][e] = finish(acc[2 * s + (e >> 2)][e & 3], o.scale, ws[e], bs[e], p.least);
            }
            if (past_cache && g * 64 + 64 <= p.N) {               // 128 bytes of each of 8 rows a store
                u32x4 a, b;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t u = pack2<DT>(v[0][2 * w], v[0][2 * w + 1]), t = pack2<DT>(v[1][2 * w], v[1][2 * w + 1]);
                    swap8(u, t);
                    a[w] = u;
                    b[w] = t;
                }
                uint16_t *to = (uint16_t *)p.out + (size_t)(at + (l16 & 7)) * p.N + g * 64 + (l16 >> 3) * 32 + q * 8;
                if (at + (l16 & 7) < rows) __builtin_nontemporal_store(a, (u32x4 *)to);
                if (at + 8 + (l16 & 7) < rows) __builtin_nontemporal_store(b, (u32x4 *)(to + (size_t)8 * p.N));
                continue;
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int c = g * 64 + s * 32 + q * 8;
                if (c < p.N && row < rows) store8<DT>(p.out, (size_t)row * p.N + c, v[s], p.N - c);
            }
        }
    };
    while (row0 < rows) {
        load(o1, row0 + stride);
        step(o0, row0);
        row0 += stride;
        if (row0 >= rows) break;
        load(o0, row0 + stride);
        step(o1, row0);
        row0 += stride;
    }
}

template <int DT, int WM, int WN, int MF, int NF>
sbnet_status tiles_go(const char *who, const PointArgs &p, long long rows, hipStream_t s) {
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32, lds = 3 * (BM + BN) * kStageK + 4 * (BM + 2 * BN) * 4;
    static_assert(lds <= 160 * 1024, "LDS");
    const long long tiles = ((rows + BM - 1) / BM) * (((long long)p.N + BN - 1) / BN);
    const int grid = (int)(tiles < 256 ? tiles : 256);
    (void)hipFuncSetAttribute((const void *)i8_tiles<DT, WM, WN, MF, NF>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    hipLaunchKernelGGL((i8_tiles<DT, WM, WN, MF, NF>), dim3(grid), dim3(512), lds, s, p);
    return launch_status(who);
}

template <int DT, int MT, int NT, int KS>
sbnet_status direct_go(const char *who, const PointArgs &p, long long rows, hipStream_t s) {
    const long long tiles = (rows + 16 * MT - 1) / (16 * MT) * (((long long)p.N + 16 * NT - 1) / (16 * NT));
    hipLaunchKernelGGL((i8_direct<DT, MT, NT, KS>), dim3((unsigned)tiles), dim3(64 * KS), 0, s, p);
    return launch_status(who);
}

constexpr int kLds = 160 * 1024;
size_t stream_lds(int KC, int N) {
    const size_t groups = (N + 63) / 64;
    return groups * (KC * 4096 + 512);
}
template <int DT, int KC>
sbnet_status stream_go(const char *who, const PointArgs &p, long long rows, hipStream_t s) {
    const long long steps = (rows + 15) / 16;
    const size_t lds = stream_lds(KC, p.N);
    // (the same for every layer: another thread's call may come between this one and the launch)
    (void)hipFuncSetAttribute((const void *)i8_stream<DT, KC>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    hipLaunchKernelGGL((i8_stream<DT, KC>), dim3((unsigned)(steps < 256 ? steps : 256)), dim3(64 * kStreamWaves), lds, s, p, (p.N + 63) / 64);
    return launch_status(who);
}

// What a shape of work costs: `channel` ns for each channel summed over and `result` ns at the end, times the rounds of 256 workgroups.  Fitted to 210 products of
// 1 .. 100000 rows and 32 .. 8192 channels on either side, where the smallest estimate is mostly the fastest of the eight or within a tenth of it.
// E.g. (us) 16 x 4096 x 4096: 6.8 with 16 x 16 a workgroup, 9.1 with 32 x 32, 10.9 with 64 x 64; 64 rows: 14.0, 10.7, 11.3; 128: 17.8
// with 32 x 32, 11.8 with 64 x 64, 13.0 with 64 x 128; 512: 20.6, 15.4 and, with 128 x 128, 17.6; 1024: 28, 21.9 with 128 x 128, 27.6
// with 256 x 128; 2048: 39 and 36.5; 256 x 512 x 512: 4.7 with 32 x 32, 5.3 with 64 x 64.
struct Shape {
    int rows, channels;
    float channel, result;
};
constexpr Shape kShapes[] = {{16, 16, 0.95f, 500}, {16, 32, 1.4f, 600}, {32, 16, 1.4f, 600}, {32, 32, 1.85f, 450},
                             {64, 64, 2.0f, 800}, {64, 128, 2.35f, 1000}, {128, 128, 3.15f, 2000}, {256, 128, 5.4f, 4000}};

// `rows` are those of the list's capacity, here and for the streamed lists: a list with few active tiles takes the tile of a full one (64 pixels of 1024 -> 256,
// 55 of 550 tiles active: 8.6 us, a list of 55 5.3; 1024 -> 2048, 14 of 140: 8.7 and 6.6; 324 pixels of 256 -> 64, 219 of 2200: 6.5 and 6.6).
int cheapest(long long rows, int N, int pitch) {
    int best = 0;
    float least = 0.f;
    for (int i = 0; i < 8; ++i) {
        const Shape &s = kShapes[i];
        const long long tiles = ((rows + s.rows - 1) / s.rows) * (((long long)N + s.channels - 1) / s.channels);
        const float cost = (float)((tiles + 255) / 256) * (s.channel * (float)pitch + s.result);
        if (i == 0 || cost < least) {
            best = i;
            least = cost;
        }
    }
    return best;
}

// Lists whose weights fit LDS are streamed from a length on that grows with them: every workgroup loads all.  (us, streamed and the best of the others,
// below the line and above it: 64 -> 64, 4000 rows 4.0 and 4.0, 12000 4.1 and 4.6; 256 -> 128, 8192 5.6 and 4.9, 20000 6.4 and 6.7; 64 -> 256, 6000
// 5.4 and 5.2, 20000 6.7 and 9.4; 256 -> 256, 16000 8.5 and 7.3, 30000 10.2 and 13.1; 64 -> 1024, 8192 12.9 and 9.7, 30000 15.3 and 24.9.  From 385 input
// channels on the rows in flight are fewer: 512 -> 64, 20000 6.8 and 7.2, 512 -> 128, 50000 13.8 and 13.0.)
bool streams(long long rows, int N, int KC) {
    if (KC > 8 || stream_lds(KC <= 4 ? KC : KC <= 6 ? 6 : 8, N) > kLds) return false;
    const long long weights = (long long)KC * N;
    return rows >= (KC <= 6 ? 4000 + 14 * weights : 60 * weights);
}

template <int DT>
sbnet_status pointwise_go(const char *who, const PointArgs &p, long long rows, hipStream_t s) {
    const int KC = (p.pitch + 63) / 64;
    if (streams(rows, p.N, KC)) {
        if (KC == 1) return stream_go<DT, 1>(who, p, rows, s);
        if (KC == 2) return stream_go<DT, 2>(who, p, rows, s);
        if (KC == 3) return stream_go<DT, 3>(who, p, rows, s);
        if (KC == 4) return stream_go<DT, 4>(who, p, rows, s);
        if (KC <= 6) return stream_go<DT, 6>(who, p, rows, s);
        return stream_go<DT, 8>(who, p, rows, s);
    }
    switch (cheapest(rows, p.N, p.pitch)) {
        case 0: return direct_go<DT, 1, 1, 8>(who, p, rows, s);
        case 1: return direct_go<DT, 1, 2, 8>(who, p, rows, s);
        case 2: return direct_go<DT, 2, 1, 8>(who, p, rows, s);
        case 3: return direct_go<DT, 2, 2, 4>(who, p, rows, s);
        case 4: return tiles_go<DT, 2, 2, 1, 1>(who, p, rows, s);
        case 5: return tiles_go<DT, 2, 2, 1, 2>(who, p, rows, s);
        case 6: return tiles_go<DT, 2, 2, 2, 2>(who, p, rows, s);
        default: return tiles_go<DT, 2, 2, 4, 2>(who, p, rows, s);
    }
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
    if (Cout > kMaxCout) return fail(SBNET_EUNSUPPORTED, "%s: more than %d output channels", who, kMaxCout);
    if ((uintptr_t)w_hwio % elem_bytes(dtype) || ((uintptr_t)w_scales & 3) || ((uintptr_t)w_codes & 15))
        return fail(SBNET_EINVAL, "%s: a pointer is not aligned (codes to 16 bytes, others to their elements)", who);
    const int pitch = (Cin + 15) / 16 * 16;
    const size_t wb = (size_t)Cin * Cout * elem_bytes(dtype), cb = (size_t)Cout * pitch, sb = (size_t)Cout * 4;
    if (ranges_overlap(w_hwio, wb, w_codes, cb) || ranges_overlap(w_hwio, wb, w_scales, sb) || ranges_overlap(w_codes, cb, w_scales, sb))
        return fail(SBNET_EINVAL, "%s: arrays overlap", who);
    hipStream_t s = (hipStream_t)stream;
#define SBNET_QW(DT) hipLaunchKernelGGL(i8_quantize_weights<DT>, dim3((Cout + 31LL) / 32), dim3(1024), 0, s, (const Elem<DT>::T *)w_hwio, Cin, Cout, \
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
    if (Cout > kMaxCout) return fail(SBNET_EUNSUPPORTED, "%s: more than %d output channels", who, kMaxCout);
    if ((long long)cap * pixels >= (1LL << 31)) return fail(SBNET_EUNSUPPORTED, "%s: too many rows", who);
    if (((uintptr_t)codes | (uintptr_t)w_codes | (uintptr_t)out) & 15)
        return fail(SBNET_EINVAL, "%s: codes, w_codes and out must be 16-byte aligned", who);
    if (((uintptr_t)scales | (uintptr_t)w_scales | (uintptr_t)bias | (uintptr_t)count) & 3)
        return fail(SBNET_EINVAL, "%s: a pointer is not aligned to its elements", who);
    const size_t rows = (size_t)cap * pixels, ob = rows * Cout * elem_bytes(dtype);
    if (ranges_overlap(out, ob, codes, rows * pitch) || ranges_overlap(out, ob, scales, rows * 4) ||
        ranges_overlap(out, ob, w_codes, (size_t)Cout * pitch) || ranges_overlap(out, ob, w_scales, (size_t)Cout * 4) ||
        (bias && ranges_overlap(out, ob, bias, (size_t)Cout * 4)) || holds_count(out, ob, count))
        return fail(SBNET_EINVAL, "%s: out overlaps an input", who);
    if (cap == 0) return SBNET_OK;
    PointArgs p = {};
    p.a = codes; p.w = w_codes; p.a_scales = scales; p.w_scales = w_scales; p.bias = bias; p.count = count; p.out = out;
    p.cap = cap; p.pixels = pixels; p.pitch = pitch; p.N = Cout; p.least = relu ? 0.f : -INFINITY;
    p.wide = (long long)Cout * elem_bytes(dtype) % 16 == 0;
    hipStream_t s = (hipStream_t)stream;
    if (dtype == SBNET_F32) return pointwise_go<SBNET_F32>(who, p, (long long)rows, s);
    if (dtype == SBNET_BF16) return pointwise_go<SBNET_BF16>(who, p, (long long)rows, s);
    return pointwise_go<SBNET_F16>(who, p, (long long)rows, s);
}
