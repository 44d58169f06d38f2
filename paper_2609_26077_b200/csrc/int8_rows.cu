// Row kernels of the 8-bit integer layer: quantization, restoring, the root-mean-square norm with 8-bit output, and that
// norm's gradients from an 8-bit checkpoint.  All of them are bound by memory: every kernel reads each input and writes
// each output once, rows staying in registers between the passes that a row needs (sum of squares, maximum, codes).
//
// A thread owns groups of eight consecutive columns (16 bytes of a 16-bit type), a warp N * 256 consecutive columns: group i of lane l are
// columns 256 i + 8 l and on, so that a block of 32 (128) columns is 4 (16) neighbouring lanes and its maximum takes 2 (4) shuffles.
#include <math.h>
#include <algorithm>
#include <type_traits>
#include "fmm_ptx.cuh"
#include "int8_internal.h"
#include "int8_shapes.h"

namespace {

#ifdef FMM_DEBUG
__device__ int g_int8_rows_guard;
#endif
#define ROW_STORE_OK(ptr, bytes, code) INT8_STORE_OK(p.ranges, ptr, bytes, code, &g_int8_rows_guard)

// ---------------------------------------------------------------------------------------- eight columns of a row
// Kernels exist for any rows (AL 0), for rows that all start on 16-byte boundaries and have a multiple of eight columns (1: all of a
// thread's eight exist, or none), and for such rows that fill every thread (2: nothing is tested).  Of the first kind a row is read by the
// aligned 16-byte vectors that hold an element of it, and a thread's eight columns are shifted out of two (fp32: three) of them; it is
// written the same way, neighbouring lanes passing on what belongs to the other's vector; so an output in an input's place holds: a
// lane stores its neighbour's columns only with that lane's numbers, and what else a vector held of others is not used.  (1000 rows of 4095 fp16 columns through the
// norm: 19.3 us element by element, 8.3 this way.)  The offset `m` of a row within its vector is the same for all its columns.
template <typename T, int AL> struct Raw8 { uint32_t w[AL ? sizeof(T) * 2 : sizeof(T) * 2 + 4]; };

template <typename T> __device__ __forceinline__ int row_offset(const T* row) { return (int)(((uintptr_t)row & 15) / sizeof(T)); }

// columns [col, col + 8) of a row of which n are left from col on (0 or less: none is read, zeros)
template <typename T, int AL> __device__ __forceinline__ Raw8<T, AL> load8(const T* row, int col, int n)
{
    constexpr int PER = 16 / sizeof(T);
    const int m = AL ? 0 : row_offset(row);
    const uint4* p = reinterpret_cast<const uint4*>(row + col - m);
    Raw8<T, AL> r;
#pragma unroll
    for (int i = 0; i < 8 / PER + (AL ? 0 : 1); ++i) {
        const bool some = AL == 2 || (AL || i == 0 ? n > 0 : i * PER < m + 8 && n > i * PER - m);
        const uint4 v = some ? p[i] : make_uint4(0u, 0u, 0u, 0u);
        r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
    }
    return r;
}
// w[i] = words [shift, shift + N) of w, shift in units of `T` below 16 bytes' worth
template <typename T, int N, int M> __device__ __forceinline__ void shift_words(uint32_t (&w)[M], int shift)
{
    constexpr int TWO = sizeof(T) == 4 ? 2 : 4, ONE = TWO / 2;
#pragma unroll
    for (int i = 0; i + 2 < M; ++i) w[i] = shift & TWO ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i + 1 < M; ++i) w[i] = shift & ONE ? w[i + 1] : w[i];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = shift & 1 ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
    }
}
// the eight numbers, zeros for those behind the row's end.  m: row_offset
template <typename T, int AL> __device__ __forceinline__ void unpack8(const Raw8<T, AL>& r, int m, int n, float (&f)[8])
{
    constexpr int N = sizeof(T) * 2;
    uint32_t w[AL ? N : N + 4];
#pragma unroll
    for (int i = 0; i < (AL ? N : N + 4); ++i) w[i] = r.w[i];
    if constexpr (!AL) shift_words<T, N>(w, m);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(w[i]);
        else {
            const uint16_t h = (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]);
            f[i] = to_float(*reinterpret_cast<const T*>(&h));
        }
    }
    if (!AL && n < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? f[i] : 0.0f;
    }
}
// The N groups of a warp's lanes, from column col on, of which n are left.  Every lane of the warp calls it.
constexpr int GROUP = 256;
template <int AL, int N, typename T, typename P> __device__ __forceinline__ void store_groups(T* row, int col, int n, const float (&f)[N][8], const P& p, int code)
{
    constexpr int W = sizeof(T) * 2;                          // words of a group
    T* q = row + col;
    auto pack = [](const float (&g)[8], uint32_t* w) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(g[i]);
            else w[i] = pack_two<T>(g[2 * i], g[2 * i + 1]);
        }
    };
    auto store_vectors = [&](T* at, const uint32_t* w) {
        if (!ROW_STORE_OK(at, 8 * sizeof(T), code)) return;
#pragma unroll
        for (int i = 0; i < W / 4; ++i) reinterpret_cast<uint4*>(at)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    };
    if constexpr (AL) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t w[W];
            pack(f[i], w);
            if (AL == 2 || n > i * GROUP) store_vectors(q + i * GROUP, w);
        }
    } else {
        // a lane's vectors hold the last m elements of the lane before (lane 0: of lane 31's group before) and the first 8 - m of its own
        const int m = row_offset(row), lane = threadIdx.x & 31;
        uint32_t before[W] = {};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int left = n - i * GROUP;
            T* at = q + i * GROUP;
            auto store_some = [&](int from, int to) {         // elements [from, to) that exist, one by one
                if (from >= min(to, left) || !ROW_STORE_OK(at + from, (min(to, left) - from) * sizeof(T), code)) return;
#pragma unroll
                for (int j = 0; j < 8; ++j) if (j >= from && j < to && j < left) at[j] = from_float<T>(f[i][j]);
            };
            uint32_t w[W + 4 + W];
            uint32_t* own = w + W;
            pack(f[i], own);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                w[j] = __shfl_sync(0xffffffffu, lane == 31 ? before[j] : own[j], (lane + 31) & 31);
                before[j] = own[j];
            }
            if (m == 0) {
                if (left >= 8) store_vectors(at, own); else store_some(0, 8);
            } else {
                if (left >= 8 - m && (i > 0 || lane > 0)) {
                    if constexpr (sizeof(T) == 4) {
                        // 8 - m words on: 4, then 4 - m
#pragma unroll
                        for (int j = 0; j < 2 * W - 4; ++j) w[j] = w[j + 4];
                        shift_words<T, W>(w, 4 - m);
                    } else shift_words<T, W>(w, 8 - m);
                    store_vectors(at - m, w);
                } else store_some(0, 8 - m);
                // the last m elements are the next lane's to store, unless there is none or its vectors are not whole
                if ((i == N - 1 && lane == 31) || left - 8 < 8 - m) store_some(8 - m, 8);
            }
        }
    }
}
// eight codes; vec: 8-byte aligned
__device__ __forceinline__ uint2 load_codes8(const int8_t* p, int n, bool vec)
{
    if (vec && n >= 8) return *reinterpret_cast<const uint2*>(p);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < n) w[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
template <typename P> __device__ __forceinline__ void store_codes8(int8_t* q, uint2 c, int n, bool vec, const P& p, int code)
{
    if (n <= 0 || !ROW_STORE_OK(q, n < 8 ? n : 8, code)) return;
    if (vec && n >= 8) *reinterpret_cast<uint2*>(q) = c;
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) q[i] = (int8_t)((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
    }
}
// code + 128 as the last byte of 2^23 + that, less 2^23 + 128: two instructions at full rate, a conversion has a quarter of it
__device__ __forceinline__ void codes_to_float(uint2 c, float (&f)[8])
{
    const uint32_t w[2] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(__byte_perm(w[i >> 2], 0x4B000000u, 0x7540 | (i & 3))) - 8388736.0f;
}

// ---------------------------------------------------------------------------------------- quantization of a block
// Maxima are taken over the bit patterns of |x|: they order like the numbers, infinities above them and NaN above those, so
// that a block that holds one of these is seen, and gets NaN as its scale.
// (The three-operand maximum of magnitudes, NaN if one is, halves what finding the maximum costs against masks and integer maxima:
// the kernels issue in 2 of 3 cycles.)
__device__ __forceinline__ float abs_max3(float a, float b, float c)
{ float d; asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
__device__ __forceinline__ uint32_t abs_max8(const float (&f)[8])
{
    const float m = abs_max3(abs_max3(f[0], f[1], f[2]), f[3], f[4]);
    return __float_as_uint(abs_max3(m, f[5], abs_max3(f[6], f[7], 0.0f)));
}
struct Scale { float scale, inverse; };
__device__ __forceinline__ Scale block_scale(uint32_t amax_bits, bool pow2)
{
    const float a = __uint_as_float(max(amax_bits, __float_as_uint(1e-12f)));
    Scale s;
    s.scale = __fdiv_rn(a, 127.0f);
    s.inverse = __fdiv_rn(127.0f, a);
    if (pow2) {
        // up to a power of two: the quotient is a normal number, from 2^-47 to below 2^122
        const uint32_t b = (__float_as_uint(s.scale) + 0x007FFFFFu) & 0xFF800000u;
        s.scale = __uint_as_float(b);
        s.inverse = __uint_as_float(0x7F000000u - b);
    }
    if (amax_bits >= 0x7F800000u) { s.scale = __uint_as_float(0x7FC00000u); s.inverse = 0.0f; }      // NaN, whatever the codes
    return s;
}
// Codes of eight numbers.  |x * inverse| <= 127 (1 + 2^-22), so 1.5 * 2^23 + that is rounded at the units, to nearest with
// ties to even, and its low byte is the code: an addition instead of a conversion, which issues at a quarter of the rate.
__device__ __forceinline__ uint2 codes8(const float (&f)[8], float inverse)
{
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(__fadd_rn(__fmul_rn(f[i], inverse), 12582912.0f));
    auto four = [&](int o) { return __byte_perm(__byte_perm(b[o], b[o + 1], 0x0040), __byte_perm(b[o + 2], b[o + 3], 0x0040), 0x5410); };
    return make_uint2(four(0), four(4));
}
template <int N> __device__ __forceinline__ void share_scales(const uint32_t (&m)[N], int lanes, bool pow2, Scale (&s)[N]);

// Maxima of N groups of eight columns to those of the blocks they lie in, a block being `lanes` (4 or 16) neighbouring lanes, and the
// blocks' scales.
template <int N> __device__ __forceinline__ void block_scales(uint32_t (&m)[N], int lanes, bool pow2, Scale (&s)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        m[i] = max(m[i], __shfl_xor_sync(0xffffffffu, m[i], 1));
        m[i] = max(m[i], __shfl_xor_sync(0xffffffffu, m[i], 2));
        if (lanes > 4) {
            m[i] = max(m[i], __shfl_xor_sync(0xffffffffu, m[i], 4));
            m[i] = max(m[i], __shfl_xor_sync(0xffffffffu, m[i], 8));
        }
    }
    share_scales(m, lanes, pow2, s);
}
// The scales of N blocks whose maxima all of `lanes` neighbouring lanes know: they share the divisions out.
template <int N> __device__ __forceinline__ void share_scales(const uint32_t (&m)[N], int lanes, bool pow2, Scale (&s)[N])
{
    static_assert(N == 1 || N == 2 || N == 4, "groups of a thread");
    const int lane = threadIdx.x & 31, k = lane & (lanes - 1), first = lane - k;
    uint32_t mine = m[0];
    if (N > 1) mine = k & 1 ? m[1] : mine;
    if (N > 2) mine = (k & 2 ? (k & 1 ? m[N - 1] : m[N / 2]) : mine);
    if (pow2 || lanes < 2 * N) {
        // lane k: both numbers of group k
        const Scale own = block_scale(mine, pow2);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i].scale = __shfl_sync(0xffffffffu, own.scale, first + i);
            s[i].inverse = __shfl_sync(0xffffffffu, own.inverse, first + i);
        }
    } else {
        // lane k: the scale of group k, lane N + k its inverse
        const bool inverse = k & N, finite = mine < 0x7F800000u;
        const float a = __uint_as_float(max(mine, __float_as_uint(1e-12f)));
        float x = __fdiv_rn(inverse ? 127.0f : a, inverse ? a : 127.0f);
        if (!finite) x = inverse ? 0.0f : __uint_as_float(0x7FC00000u);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i].scale = __shfl_sync(0xffffffffu, x, first + i);
            s[i].inverse = __shfl_sync(0xffffffffu, x, first + N + i);
        }
    }
}

// ---------------------------------------------------------------------------------------- sums over a row's threads
// (`warps` of them, of a block's row; one: no shared memory)
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t* red, int warps)
{
    m = __reduce_max_sync(0xffffffffu, m);
    if (warps > 1) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        m = __reduce_max_sync(0xffffffffu, lane < warps ? red[lane] : 0u);
    }
    return m;
}
// always the same order: lanes by halves, then the warps by halves
template <typename F> __device__ __forceinline__ F warp_sum(F v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float row_sum(float v, float* red, int warps)
{
    v = warp_sum(v);
    if (warps > 1) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = warp_sum(lane < warps ? red[lane] : 0.0f);
    }
    return v;
}
// 1 / sqrt(mean of squares + eps).  One warp takes the last sum, the division and the root (in fp64 a fifth of what a norm issued, by
// all warps)
__device__ __forceinline__ float row_rstd(double v, double* red, float* result, int warps, int cols, double eps)
{
    auto root = [&](double sum) { return (float)(1.0 / sqrt(sum / (double)cols + eps)); };
    v = warp_sum(v);
    if (warps == 1) return root(v);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        v = warp_sum(lane < warps ? red[lane] : 0.0);
        if (lane == 0) *result = root(v);
    }
    __syncthreads();
    return *result;
}
// both numbers of a row's scale, a division by half of the lanes each
__device__ __forceinline__ Scale row_scale(uint32_t amax_bits, bool pow2)
{
    uint32_t m[1] = {amax_bits};
    Scale s[1];
    share_scales(m, 4, pow2, s);
    return s[0];
}

// ---------------------------------------------------------------------------------------- norm / row-wise quantization
struct RowsParams {
    const void* x; const void* residual; const void* gain;
    void* hidden; int8_t* codes; float* scales; float* rstd;
    int8_t* checkpoint; float* checkpoint_scales;
    int64_t ldx, ldr, ldh, ldc, ldk;
    double eps;
    int rows, cols, block;                    // block: of the checkpoint, 0: none
    bool pow2, aligned, vc, vk;               // aligned: AL for x, residual, gain and hidden; vc, vk: of codes and checkpoint, to 8 bytes
    Int8Ranges ranges;
};

template <int AL, int N> __device__ __forceinline__ void checkpoint8(const RowsParams& p, int64_t row, int col, const float (&h)[N][8])
{
    const int shift = p.block == 32 ? 5 : 7, lanes = 1 << (shift - 3), per_row = (p.cols + p.block - 1) >> shift;
    uint32_t m[N];
    Scale s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) m[i] = abs_max8(h[i]);
    block_scales(m, lanes, false, s);
    int8_t* codes = p.checkpoint + row * p.ldk;
    float* scales = p.checkpoint_scales + row * per_row;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = col + i * GROUP, n = AL == 2 ? 8 : p.cols - c;
        if (n <= 0) continue;
        store_codes8(codes + c, codes8(h[i], s[i].inverse), n, AL == 2 || p.vk, p, 2101);
        if ((c & (p.block - 1)) == 0 && ROW_STORE_OK(scales + (c >> shift), 4, 2102)) scales[c >> shift] = s[i].scale;
    }
}

// A row per block of threads, or (SHORT) per warp, four to a block; held in registers, VPT groups of eight columns a thread.  The squares
// are summed in fp64 (they are exact there), so that the reciprocal root does not depend on the order of the sum and codes are the same
// on every machine.
template <typename T, bool NORM, int AL, int VPT, bool SHORT>
__global__ void __launch_bounds__(SHORT ? 128 : 512, !SHORT && AL && sizeof(T) == 2 ? 2 : 1) rows_kernel(const RowsParams p)
{
    __shared__ double red_sum[32];
    __shared__ float rstd_all;
    __shared__ uint32_t red_max[32];
    const int t = threadIdx.x, warps = SHORT ? 1 : blockDim.x / 32, col = ((t >> 5) * VPT * 32 + (t & 31)) * 8;
    const int64_t row = SHORT ? (int64_t)blockIdx.x * 4 + threadIdx.y : (int64_t)blockIdx.x;
    if (SHORT && row >= p.rows) return;                       // whole warps
    auto left = [&](int i) { return AL == 2 ? 8 : p.cols - (col + i * GROUP); };
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const int mx = AL ? 0 : row_offset(x);
    float h[VPT][8];
    Raw8<T, AL> raw[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) raw[i] = load8<T, AL>(x, col + i * GROUP, left(i));
    if constexpr (NORM) {
        if (p.residual) {
            const T* r = static_cast<const T*>(p.residual) + row * p.ldr;
            const int mr = AL ? 0 : row_offset(r);
            Raw8<T, AL> rawr[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) rawr[i] = load8<T, AL>(r, col + i * GROUP, left(i));
            T* hid = static_cast<T*>(p.hidden) + row * p.ldh;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                float b[8];
                unpack8<T, AL>(raw[i], mx, left(i), h[i]);
                unpack8<T, AL>(rawr[i], mr, left(i), b);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = __fadd_rn(h[i][j], b[j]);
            }
            store_groups<AL>(hid, col, p.cols - col, h, p, 2103);
        } else {
#pragma unroll
            for (int i = 0; i < VPT; ++i) unpack8<T, AL>(raw[i], mx, left(i), h[i]);
        }
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) { const double v = (double)h[i][j]; sum = fma(v, v, sum); }
        if (p.block) {
#pragma unroll
            for (int i = 0; i < VPT; i += 2) checkpoint8<AL, 2>(p, row, col + i * GROUP, *reinterpret_cast<const float (*)[2][8]>(&h[i]));
        }
        const T* gain = static_cast<const T*>(p.gain);
        const int mg = AL ? 0 : row_offset(gain);
        const float rstd = row_rstd(sum, red_sum, &rstd_all, warps, p.cols, p.eps);
        if (t == 0 && p.rstd && ROW_STORE_OK(p.rstd + row, 4, 2104)) p.rstd[row] = rstd;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float g[8];
            unpack8<T, AL>(load8<T, AL>(gain, col + i * GROUP, left(i)), mg, left(i), g);       // (the same for all rows: from L1)
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] = __fmul_rn(__fmul_rn(h[i][j], rstd), g[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPT; ++i) unpack8<T, AL>(raw[i], mx, left(i), h[i]);
    }
    // behind the last column: h is 0 there, and 0 * rstd is NaN where rstd is infinite (a row of zeros with eps 0), which is what
    // the row's own zeros are as well
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) m = max(m, abs_max8(h[i]));
    const Scale s = row_scale(row_max(m, red_max, warps), p.pow2);
    int8_t* codes = p.codes + row * p.ldc;
#pragma unroll
    for (int i = 0; i < VPT; ++i) store_codes8(codes + col + i * GROUP, codes8(h[i], s.inverse), left(i), AL == 2 || p.vc, p, 2105);
    if (t == 0 && ROW_STORE_OK(p.scales + row, 4, 2106)) p.scales[row] = s.scale;
}

// Rows without columns: the scale of nothing, 1e-12 / 127 or the power of two above it
__global__ void __launch_bounds__(256) no_columns_kernel(const RowsParams p)
{
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row < p.rows && ROW_STORE_OK(p.scales + row, 4, 2107)) p.scales[row] = block_scale(0u, p.pow2).scale;
}

// Rows that do not fit registers: read again for each pass (from L2, mostly).  hidden may be x or residual, so it is written in the
// last pass.  Every lane goes round as often, as lanes exchange numbers.
template <typename T, bool NORM, int AL>
__global__ void __launch_bounds__(1024) rows_long_kernel(const RowsParams p)
{
    constexpr int NT = 1024;
    __shared__ double red_sum[32];
    __shared__ float rstd_all;
    __shared__ uint32_t red_max[32];
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x, end = (p.cols + 8 * NT - 1) / (8 * NT) * (8 * NT);
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const T* r = NORM && p.residual ? static_cast<const T*>(p.residual) + row * p.ldr : nullptr;
    auto number8 = [&](const T* row, int col, float (&f)[8]) { unpack8<T, AL>(load8<T, AL>(row, col, p.cols - col), AL ? 0 : row_offset(row), p.cols - col, f); };
    auto hidden8 = [&](int col, float (&h)[8]) {
        number8(x, col, h);
        if (r) {
            float b[8];
            number8(r, col, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = __fadd_rn(h[j], b[j]);
        }
    };
    float rstd = 1.0f;
    if constexpr (NORM) {
        double sum = 0.0;
        for (int col = 8 * t; col < end; col += 8 * NT) {
            float h[1][8];
            hidden8(col, h[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) { const double d = (double)h[0][j]; sum = fma(d, d, sum); }
            if (p.block) checkpoint8<AL>(p, row, col, h);
        }
        rstd = row_rstd(sum, red_sum, &rstd_all, NT / 32, p.cols, p.eps);
        if (t == 0 && p.rstd && ROW_STORE_OK(p.rstd + row, 4, 2114)) p.rstd[row] = rstd;
    }
    auto normed8 = [&](int col, float (&h)[8]) {
        if constexpr (NORM) {
            float g[8];
            number8(static_cast<const T*>(p.gain), col, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = __fmul_rn(__fmul_rn(h[j], rstd), g[j]);
        }
    };
    uint32_t m = 0;
    for (int col = 8 * t; col < end; col += 8 * NT) {
        float h[8];
        hidden8(col, h);
        normed8(col, h);
        m = max(m, abs_max8(h));
    }
    const Scale s = row_scale(row_max(m, red_max, NT / 32), p.pow2);
    for (int col = 8 * t; col < end; col += 8 * NT) {
        float h[1][8];
        hidden8(col, h[0]);
        if (r) store_groups<AL>(static_cast<T*>(p.hidden) + row * p.ldh, col, p.cols - col, h, p, 2113);
        normed8(col, h[0]);
        store_codes8(p.codes + row * p.ldc + col, codes8(h[0], s.inverse), p.cols - col, p.vc, p, 2115);
    }
    if (t == 0 && ROW_STORE_OK(p.scales + row, 4, 2116)) p.scales[row] = s.scale;
}

// ---------------------------------------------------------------------------------------- quantization in blocks, restoring
// Nothing is summed over a row, so a row is cut into pieces of 1024 columns, a warp to each: four groups of eight columns a thread, 256
// columns apart, all of them loaded before the first is used.  A block has eight warps, side by side along a row first.
constexpr int FLAT_VPT = 4, FLAT_PIECE = FLAT_VPT * GROUP;

struct BlocksParams {
    const void* x; int8_t* codes; float* scales;
    int64_t ldx, ldc;
    int rows, cols, block;
    bool pow2, vc;
    Int8Ranges ranges;
};

template <typename T, int AL>
__global__ void __launch_bounds__(256, 3) quantize_blocks_kernel(const BlocksParams p)
{
    constexpr int VPT = FLAT_VPT;
    const int shift = p.block == 32 ? 5 : 7, lanes = 1 << (shift - 3), per_row = (p.cols + p.block - 1) >> shift;
    for (int64_t row = (int64_t)blockIdx.x * blockDim.z + threadIdx.z; row < p.rows; row += (int64_t)gridDim.x * blockDim.z) {
        const T* x = static_cast<const T*>(p.x) + row * p.ldx;
        const int mx = AL ? 0 : row_offset(x);
        for (int piece = threadIdx.y * FLAT_PIECE; piece < p.cols; piece += blockDim.y * FLAT_PIECE) {
            const int col = piece + 8 * threadIdx.x;
            auto left = [&](int i) { return AL == 2 ? 8 : p.cols - (col + i * GROUP); };
            Raw8<T, AL> raw[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) raw[i] = load8<T, AL>(x, col + i * GROUP, left(i));
            float f[VPT][8];
            uint32_t m[VPT];
            Scale s[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) { unpack8<T, AL>(raw[i], mx, left(i), f[i]); m[i] = abs_max8(f[i]); }
            block_scales(m, lanes, p.pow2, s);
            int8_t* codes = p.codes + row * p.ldc + col;
            float* scales = p.scales + row * per_row + (col >> shift);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int n = left(i);
                if (n <= 0) continue;
                store_codes8(codes + i * GROUP, codes8(f[i], s[i].inverse), n, AL == 2 || p.vc, p, 2121);
                float* q = scales + (i * GROUP >> shift);
                if ((col & (p.block - 1)) == 0 && ROW_STORE_OK(q, 4, 2122)) *q = s[i].scale;
            }
        }
    }
}

struct RestoreParams {
    const int8_t* codes; const float* scales; void* x;
    int64_t ldc, ldx;
    int rows, cols, block;
    bool vc;
    Int8Ranges ranges;
};
template <typename T, int AL>
__global__ void __launch_bounds__(256) dequantize_kernel(const RestoreParams p)
{
    constexpr int VPT = FLAT_VPT;
    const int per_row = p.block ? (p.cols + p.block - 1) / p.block : 1, shift = p.block == 32 ? 5 : 7;
    for (int64_t row = (int64_t)blockIdx.x * blockDim.z + threadIdx.z; row < p.rows; row += (int64_t)gridDim.x * blockDim.z) {
        const int8_t* codes = p.codes + row * p.ldc;
        const float* scales = p.scales + row * per_row;
        T* x = static_cast<T*>(p.x) + row * p.ldx;
        for (int piece = threadIdx.y * FLAT_PIECE; piece < p.cols; piece += blockDim.y * FLAT_PIECE) {
            const int col = piece + 8 * threadIdx.x;
            auto left = [&](int i) { return AL == 2 ? 8 : p.cols - (col + i * GROUP); };
            uint2 c[VPT];
            float s[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int at = col + i * GROUP;
                c[i] = load_codes8(codes + at, left(i), AL == 2 || p.vc);
                s[i] = left(i) > 0 ? scales[p.block ? at >> shift : 0] : 0.0f;
            }
            float f[VPT][8];
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                codes_to_float(c[i], f[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[i][j] = __fmul_rn(f[i][j], s[i]);
            }
            store_groups<AL>(x, col, p.cols - col, f, p, 2131);
        }
    }
}

// ---------------------------------------------------------------------------------------- what the product of a gradient reads
// Largest magnitude of finite scales that the threads of a block come across, from `first` on in steps of `step` (threads: of a block, 1024 at most)
__device__ __forceinline__ uint32_t finite_scale_max(const float* scales, int rows, int64_t first, int64_t step, int thread, int threads, uint32_t* red)
{
    uint32_t m = 0;
    for (int64_t i = first; i < rows; i += step) {
        const uint32_t b = __float_as_uint(scales[i]) & 0x7FFFFFFFu;
        if (b < 0x7F800000u) m = max(m, b);
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if ((thread & 31) == 0) red[thread >> 5] = m;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, (thread & 31) < threads / 32 ? red[thread & 31] : 0u);
}
// one a block
__global__ void __launch_bounds__(1024) scale_maxima_kernel(const float* __restrict__ scales, int rows, uint32_t* __restrict__ maxima)
{
    __shared__ uint32_t red[32];
    fmmptx::griddep_launch_dependents();
    const uint32_t m = finite_scale_max(scales, rows, (int64_t)blockIdx.x * 1024 + threadIdx.x, (int64_t)gridDim.x * 1024, threadIdx.x, 1024, red);
    if (threadIdx.x == 0) maxima[blockIdx.x] = m;
}

// A part of a number that others follow: cut off towards zero and never the whole of it, so that what is left has its sign and is not zero.
// (An infinity of dY times a part of 0, or minus an infinity from a part of the other sign, would be NaN.)  Infinities and NaN as they are.
template <typename T> __device__ __forceinline__ uint16_t part_below(float v);
template <> __device__ __forceinline__ uint16_t part_below<__nv_bfloat16>(float v)
{
    const uint32_t b = __float_as_uint(v);
    return (uint16_t)((b - ((b & 0x7FFFFFFFu) - 1u < 0x7F7FFFFFu ? 1u : 0u)) >> 16);
}
template <> __device__ __forceinline__ uint16_t part_below<__half>(float v)
{
    const uint16_t h = __half_as_ushort(__float2half_rz(v));
    return (uint16_t)(h - (__half2float(__ushort_as_half(h)) == v && (uint16_t)((h & 0x7FFFu) - 1u) < 0x7BFFu ? 1u : 0u));
}

// A row's pieces as those of dequantize_kernel.  The values are those of fp32; a part is what the parts before it leave, the last one rounded
// to nearest: two of bf16 are 2^-15 off at most, three exact, two of fp16 2^-21 (or 2^-25 in the units that matrix_exponent sets).
// Where the stage needs one part the others are neither written nor read.
struct ValuesParams {
    const int8_t* codes; const float* scales; uint8_t* flags; void* x;
    int64_t ldc, ldx, step;
    int rows, cols, parts, maxima_count;
    bool vc;
    Int8Ranges ranges;
};
// whether a scale of a row's stage is no power of two (warp-collective, two rows a lane)
__device__ __forceinline__ bool inexact_stage(const float* scales, int rows, int64_t row)
{
    const int64_t r = row / INT8_PART_ROWS * INT8_PART_ROWS + (threadIdx.x & 31);
    uint32_t bits = 0;
    if (r < rows) bits = __float_as_uint(scales[r]);
    if (r + 32 < rows) bits |= __float_as_uint(scales[r + 32]);
    return __any_sync(0xffffffffu, bits & 0x007FFFFFu);
}
// `block` of `blocks`, eight warps each: pieces of a row along y of them, rows along the others
template <typename T> __device__ __forceinline__ void values_block(const ValuesParams& p, float factor, int block, int blocks, int y)
{
    constexpr int VPT = FLAT_VPT;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, side = warp & (y - 1), z = 8 / y;
    for (int64_t row = (int64_t)block * z + warp / y; row < p.rows; row += (int64_t)blocks * z) {
        const int8_t* codes = p.codes + row * p.ldc;
        const float scale = p.scales ? p.scales[row] * factor : 1.0f;
        const bool inexact = p.parts > 1 && inexact_stage(p.scales, p.rows, row);
        const int parts = inexact ? p.parts : 1;
        if (p.flags && row % INT8_PART_ROWS == 0 && lane == 0 && side == 0) {
            uint8_t* flag = p.flags + row / INT8_PART_ROWS;
            if (ROW_STORE_OK(flag, 1, 2183)) *flag = inexact;
        }
        T* x = static_cast<T*>(p.x) + row * p.ldx;
        for (int piece = side * FLAT_PIECE; piece < p.cols; piece += y * FLAT_PIECE) {
            const int col = piece + 8 * lane;
            uint2 c[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) c[i] = load_codes8(codes + col + i * GROUP, p.cols - (col + i * GROUP), p.vc);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if (col + i * GROUP >= p.cols) continue;
                float f[8];
                codes_to_float(c[i], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = __fmul_rn(f[j], scale);
                T* q = x + col + i * GROUP;
                for (int part = 1; part < parts; ++part, q += p.step) {
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint16_t h = part_below<T>(f[j]);
                        w[j / 2] = j & 1 ? w[j / 2] | (uint32_t)h << 16 : h;
                        const float held = to_float(*reinterpret_cast<const T*>(&h));
                        if (isfinite(held)) f[j] -= held;
                    }
                    // (columns behind the last, up to a multiple of eight, belong to the row and are not read)
                    if (ROW_STORE_OK(q, 16, 2181)) *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
                }
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = pack_two<T>(f[2 * j], f[2 * j + 1]);
                if (ROW_STORE_OK(q, 16, 2182)) *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
}
// Up to OWN_MAXIMUM rows every block finds the scales' maximum itself, and the first one leaves it for the product: a launch less.
constexpr int OWN_MAXIMUM = 2048;
template <typename T>
__global__ void __launch_bounds__(256) values_kernel(const ValuesParams p, uint32_t* maxima, int y)
{
    __shared__ uint32_t red[32];
    fmmptx::griddep_launch_dependents();                      // (the product, which waits for this grid to end)
    float factor = 1.0f;
    if (maxima) {
        if (p.rows <= OWN_MAXIMUM) {
            uint32_t m = finite_scale_max(p.scales, p.rows, threadIdx.x, 256, threadIdx.x, 256, red);
            if (blockIdx.x == 0 && threadIdx.x == 0) maxima[0] = m;
            factor = power_of_two(maximum_exponent(m));
        } else {
            fmmptx::griddep_wait();
            factor = power_of_two(matrix_exponent(maxima, p.maxima_count));
        }
    }
    values_block<T>(p, factor, blockIdx.x, gridDim.x, y);
}

// The largest finite number of a row comes to lie in [2^14, 2^15) (within what powers of two fp32 holds on both sides).
struct ScaledParams {
    const __nv_bfloat16* x; const float* scales; __half* y; float* inverse;
    int64_t ldx, ldy;
    int rows, cols, warps;                    // warps: of a row
    bool vs;                                  // scales on a 16-byte boundary
    Int8Ranges ranges;
};
__device__ __forceinline__ void scales8(const ScaledParams& p, int col, float (&s)[8])
{
    const float* q = p.scales + col;
    if (p.vs && col + 8 <= p.cols) {
        const float4 a = reinterpret_cast<const float4*>(q)[0], b = reinterpret_cast<const float4*>(q)[1];
        s[0] = a.x; s[1] = a.y; s[2] = a.z; s[3] = a.w; s[4] = b.x; s[5] = b.y; s[6] = b.z; s[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = col + j < p.cols ? q[j] : 0.0f;
    }
}
__device__ __forceinline__ uint32_t finite_max8(const float (&f)[8], uint32_t m)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = __float_as_uint(f[j]) & 0x7FFFFFFFu;
        m = max(m, b < 0x7F800000u ? b : 0u);
    }
    return m;
}
__device__ __forceinline__ int scaled_exponent(uint32_t most) { return most == 0 ? 0 : min(14 - ((int)(most >> 23) - 127), 126); }
__device__ __forceinline__ void store_scaled8(const ScaledParams& p, int64_t row, int col, const float (&f)[8], float factor)
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = pack_two<__half>(__fmul_rn(f[2 * j], factor), __fmul_rn(f[2 * j + 1], factor));
    uint4* q = reinterpret_cast<uint4*>(p.y + row * p.ldy + col);
    if (ROW_STORE_OK(q, 16, 2191)) *q = make_uint4(w[0], w[1], w[2], w[3]);
}

// Rows of up to 4096 (8192) columns: two (four) groups of eight a thread, whose scales stay in registers, one, two, four or eight warps a
// row; the next row is on its way while this one's maximum is found (8192 x 8192: 43 us, 152 with the scales loaded for every row).  With
// two groups a thread the codes' values come in the same launch, from the blocks behind: 20 instead of 23.8 us of the host's time for a
// call.  (With four, which leave room for two blocks an SM, that takes 84 us for 8192 x 8192 of both; apart 43 and 29.)
template <int AL, int VPT>
__global__ void __launch_bounds__(256, VPT == 2 ? 4 : 2) scaled_rows_kernel(const ScaledParams p, const ValuesParams v, int blocks, int y)
{
    using T = __nv_bfloat16;
    __shared__ uint32_t red[2][8];
    fmmptx::griddep_launch_dependents();
    if ((int)blockIdx.x >= blocks) {
        values_block<__half>(v, 1.0f, (int)blockIdx.x - blocks, (int)gridDim.x - blocks, y);
        return;
    }
    const int warps = p.warps, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, side = warp & (warps - 1), per_block = 8 / warps;
    const int first = side * VPT * GROUP + 8 * lane;
    auto left = [&](int i) { return p.cols - (first + i * GROUP); };
    float scale[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) scales8(p, first + i * GROUP, scale[i]);
    Raw8<T, AL> raw[VPT];
    auto fetch = [&](int64_t row) {
        if (row >= p.rows) return;
#pragma unroll
        for (int i = 0; i < VPT; ++i) raw[i] = load8<T, AL>(p.x + row * p.ldx, first + i * GROUP, left(i));
    };
    int parity = 0;
    const int64_t step = (int64_t)blocks * per_block;
    int64_t row = (int64_t)blockIdx.x * per_block + warp / warps;
    fetch(row);
    // (every warp of the block goes round as often: they meet)
    for (int64_t base = (int64_t)blockIdx.x * per_block; base < p.rows; base += step, row += step, parity ^= 1) {
        const bool live = row < p.rows;
        const int m = AL ? 0 : row_offset(p.x + row * p.ldx);
        float f[VPT][8];
        uint32_t most = 0;
        if (live) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                unpack8<T, AL>(raw[i], m, left(i), f[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[i][j] = __fmul_rn(f[i][j], scale[i][j]);
                most = finite_max8(f[i], most);
            }
        }
        fetch(row + step);
        most = __reduce_max_sync(0xffffffffu, most);
        if (warps > 1) {
            if (lane == 0) red[parity][warp] = most;
            __syncthreads();
            most = __reduce_max_sync(0xffffffffu, lane < warps ? red[parity][(warp - side) + lane] : 0u);
        }
        if (!live) continue;
        const int e = scaled_exponent(most);
        if (side == 0 && lane == 0 && ROW_STORE_OK(p.inverse + row, 4, 2192)) p.inverse[row] = power_of_two(-e);
        const float factor = power_of_two(e);
#pragma unroll
        for (int i = 0; i < VPT; ++i) if (left(i) > 0) store_scaled8(p, row, first + i * GROUP, f[i], factor);
    }
    fmmptx::griddep_wait();                                   // what waits for this grid waits for the one before it too, if there is one
}
// Rows that do not fit registers: ROWS of them, four or one, to a block, so that the scales, which are as many bytes as two rows, come from L2
// for all of them; read twice, the second time from L2, mostly.  (4000 x 20000: 60 us, 124 with a row to a block.)
template <int AL, int ROWS>
__global__ void __launch_bounds__(512) scaled_long_kernel(const ScaledParams p)
{
    using T = __nv_bfloat16;
    constexpr int NT = 512;
    __shared__ uint32_t red[ROWS][NT / 32];
    fmmptx::griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t base = (int64_t)blockIdx.x * ROWS;
    auto row = [&](int r) { return p.x + min(base + r, (int64_t)p.rows - 1) * p.ldx; };      // (behind the last: that one again, not stored)
    auto each8 = [&](auto use) {
        for (int col = 8 * threadIdx.x; col < p.cols; col += 8 * NT) {
            float s[8];
            scales8(p, col, s);
            Raw8<T, AL> raw[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) raw[r] = load8<T, AL>(row(r), col, p.cols - col);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                float f[8];
                unpack8<T, AL>(raw[r], AL ? 0 : row_offset(row(r)), p.cols - col, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = __fmul_rn(f[j], s[j]);
                use(r, col, f);
            }
        }
    };
    uint32_t most[ROWS] = {};
    each8([&](int r, int, const float (&f)[8]) { most[r] = finite_max8(f, most[r]); });
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t m = __reduce_max_sync(0xffffffffu, most[r]);
        if (lane == 0) red[r][warp] = m;
    }
    __syncthreads();
    int e[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        e[r] = scaled_exponent(__reduce_max_sync(0xffffffffu, lane < NT / 32 ? red[r][lane] : 0u));
        if (threadIdx.x == 0 && base + r < p.rows && ROW_STORE_OK(p.inverse + base + r, 4, 2194)) p.inverse[base + r] = power_of_two(-e[r]);
    }
    each8([&](int r, int col, const float (&f)[8]) { if (base + r < p.rows) store_scaled8(p, base + r, col, f, power_of_two(e[r])); });
    fmmptx::griddep_wait();                                   // what waits for this grid waits for the one before it too
}

// 16-bit rows of any alignment, copied to rows that a tensor map can read (ldy a multiple of 8, y on a 16-byte boundary); what lies
// behind the last column of y's rows is written as it comes.  (8192 x 8191: 111 us element by element, 34 by shifted vectors.)
struct RealignParams {
    const __half* x; __half* y;
    int64_t ldx, ldy;
    int rows, cols;
    Int8Ranges ranges;
};
__global__ void __launch_bounds__(256) realign_kernel(const RealignParams p)
{
    constexpr int VPT = FLAT_VPT;
    fmmptx::griddep_launch_dependents();
    for (int64_t row = (int64_t)blockIdx.x * blockDim.z + threadIdx.z; row < p.rows; row += (int64_t)gridDim.x * blockDim.z) {
        const __half* x = p.x + row * p.ldx;
        const int m = row_offset(x);
        for (int piece = threadIdx.y * FLAT_PIECE; piece < p.cols; piece += blockDim.y * FLAT_PIECE) {
            const int col = piece + 8 * threadIdx.x;
            Raw8<__half, 0> raw[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) raw[i] = load8<__half, 0>(x, col + i * GROUP, p.cols - (col + i * GROUP));
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if (col + i * GROUP >= p.cols) continue;
                shift_words<__half, 4>(raw[i].w, m);
                uint4* q = reinterpret_cast<uint4*>(p.y + row * p.ldy + col + i * GROUP);
                if (ROW_STORE_OK(q, 16, 2171)) *q = make_uint4(raw[i].w[0], raw[i].w[1], raw[i].w[2], raw[i].w[3]);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------- the norm's gradients
struct BackParams {
    const void* dy; const int8_t* checkpoint; const float* scales; const float* rstd; const void* gain; const void* dresidual;
    void* dx; float* dgain; float* partial;
    int64_t ldy, ldk, ldr, ldx, ldp;          // ldp: of partial, a multiple of 8
    int rows, cols, block, parts;             // parts: rows of `partial`
    bool aligned, vk;                         // aligned: AL for dy, gain, dresidual and dx; vk: of the checkpoint, to 8 bytes
    Int8Ranges ranges;
};

constexpr int BACK_VPT = 2;

// xhat of eight columns: code * (scale * rstd)
__device__ __forceinline__ void xhat8(uint2 codes, float scale, float rstd, float (&f)[8])
{
    codes_to_float(codes, f);
    const float s = scale * rstd;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= s;
}

// Rows are dealt out to groups of threads, a block or (SHORT) a warp, four to a block; each thread has two groups of eight columns.
// It keeps its columns' sums of dy * xhat in registers over all its rows and the block writes them once, as one row of `partial`;
// column_sum_kernel adds those rows up in a fixed order.  128 registers a thread let the next row's loads be in flight while this one
// is summed (NEXT: aligned rows of a 16-bit type; the others' loads are issued together where the row begins).  The gain, the same for
// all rows, comes from L1 each time.
template <typename T, int AL, bool SHORT>
__global__ void __launch_bounds__(SHORT ? 128 : 512, SHORT ? 4 : 1) back_kernel(const BackParams p)
{
    constexpr bool NEXT = AL && sizeof(T) == 2;
    constexpr int RPC = SHORT ? 4 : 1, VPT = BACK_VPT;
    __shared__ float red[2][32];
    __shared__ float4 meet[RPC > 1 ? RPC * VPT * 32 * 2 : 1];
    fmmptx::griddep_launch_dependents();
    const int t = threadIdx.x, warps = SHORT ? 1 : blockDim.x / 32, first = ((t >> 5) * VPT * 32 + (t & 31)) * 8, group = blockIdx.x * RPC + threadIdx.y, groups = gridDim.x * RPC;
    const int shift = p.block == 32 ? 5 : 7, per_row = p.block ? (p.cols + p.block - 1) >> shift : 1;
    float sum[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[i][j] = 0.0f;
    const T* gain = static_cast<const T*>(p.gain);
    const int mg = AL ? 0 : row_offset(gain);
    Raw8<T, AL> dy[VPT];
    uint2 codes[VPT];
    float scale[VPT], rstd = 0.0f;
    auto fetch = [&](int64_t row) {
        rstd = p.rstd[row];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int col = first + i * GROUP, n = AL == 2 ? 8 : p.cols - col;
            dy[i] = load8<T, AL>(static_cast<const T*>(p.dy) + row * p.ldy, col, n);
            codes[i] = load_codes8(p.checkpoint + row * p.ldk + col, n, AL == 2 || p.vk);
            scale[i] = n > 0 ? p.scales[row * per_row + (p.block ? col >> shift : 0)] : 0.0f;
        }
    };
    int parity = 0;
    if (NEXT && group < p.rows) fetch(group);
    for (int64_t row = group; row < p.rows; row += groups, parity ^= 1) {
        if (!NEXT) fetch(row);
        const float rs = rstd;
        const int my = AL ? 0 : row_offset(static_cast<const T*>(p.dy) + row * p.ldy);
        const T* dres = static_cast<const T*>(p.dresidual) + row * p.ldr;
        Raw8<T, AL> add[VPT];
        if (p.dresidual) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) { const int col = first + i * GROUP; add[i] = load8<T, AL>(dres, col, AL == 2 ? 8 : p.cols - col); }
        }
        float out[VPT][8], xh[VPT][8], c = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int col = first + i * GROUP, n = AL == 2 ? 8 : p.cols - col;
            float g[8];
            unpack8<T, AL>(load8<T, AL>(gain, col, n), mg, n, g);
            unpack8<T, AL>(dy[i], my, n, out[i]);
            xhat8(codes[i], scale[i], rs, xh[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum[i][j] = fmaf(out[i][j], xh[i][j], sum[i][j]);
                out[i][j] *= g[j];
                c = fmaf(out[i][j], xh[i][j], c);
            }
        }
        if (NEXT && row + groups < p.rows) fetch(row + groups);
        c = row_sum(c, red[parity], warps) / (float)p.cols;
        T* dx = static_cast<T*>(p.dx) + row * p.ldx;
        const int mr = AL ? 0 : row_offset(dres);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int col = first + i * GROUP, n = AL == 2 ? 8 : p.cols - col;
            float b[8];
            if (p.dresidual) unpack8<T, AL>(add[i], mr, n, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                out[i][j] = rs * (out[i][j] - xh[i][j] * c);
                if (p.dresidual) out[i][j] += b[j];
            }
            if constexpr (AL != 0) store_groups<AL>(dx, col, n, *reinterpret_cast<const float (*)[1][8]>(&out[i]), p, 2141);
        }
        if constexpr (AL == 0) store_groups<AL>(dx, first, p.cols - first, out, p, 2141);
    }
    if constexpr (RPC > 1) {
        // the block's groups meet, in their order
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                meet[((threadIdx.y * VPT + i) * 2 + h) * 32 + t] = make_float4(sum[i][4 * h], sum[i][4 * h + 1], sum[i][4 * h + 2], sum[i][4 * h + 3]);
        __syncthreads();
        if (threadIdx.y > 0) return;
#pragma unroll
        for (int y = 1; y < RPC; ++y)
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 v = meet[((y * VPT + i) * 2 + h) * 32 + t];
                    sum[i][4 * h] += v.x; sum[i][4 * h + 1] += v.y; sum[i][4 * h + 2] += v.z; sum[i][4 * h + 3] += v.w;
                }
    }
    float* q = p.partial + (int64_t)blockIdx.x * p.ldp;
    store_groups<AL == 2 ? 2 : 1>(q, first, p.cols - first, sum, p, 2142);
}

// Rows that do not fit registers: dy and the codes are read twice (the second time from L2, mostly), and the sums of a group live in
// its row of `partial`, which no other group touches.
template <typename T, int AL>
__global__ void __launch_bounds__(1024) back_long_kernel(const BackParams p)
{
    constexpr int NT = 1024;
    __shared__ float red[2][32];
    fmmptx::griddep_launch_dependents();
    const int t = threadIdx.x, part = blockIdx.x, end = (p.cols + 8 * NT - 1) / (8 * NT) * (8 * NT);
    const int per_row = p.block ? (p.cols + p.block - 1) / p.block : 1, shift = p.block == 32 ? 5 : 7;
    float* q = p.partial + (int64_t)part * p.ldp;
    auto number8 = [&](const void* base, int64_t ld, int64_t row, int col, float (&f)[8]) {
        const T* r = static_cast<const T*>(base) + row * ld;
        unpack8<T, AL>(load8<T, AL>(r, col, p.cols - col), AL ? 0 : row_offset(r), p.cols - col, f);
    };
    int parity = 0;
    for (int64_t row = part; row < p.rows; row += gridDim.x, parity ^= 1) {
        const float rs = p.rstd[row];
        auto both8 = [&](int col, float (&d)[8], float (&xh)[8], float (&g)[8]) {
            const int n = p.cols - col;
            number8(p.dy, p.ldy, row, col, d);
            number8(p.gain, 0, 0, col, g);
            xhat8(load_codes8(p.checkpoint + row * p.ldk + col, n, p.vk), n > 0 ? p.scales[row * per_row + (p.block ? col >> shift : 0)] : 0.0f, rs, xh);
        };
        float c = 0.0f;
        for (int col = 8 * t; col < p.cols; col += 8 * NT) {
            float d[8], xh[8], g[8], s[1][8];
            both8(col, d, xh, g);
            if (row == part) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s[0][j] = 0.0f;
            } else unpack8<float, 1>(load8<float, 1>(q, col, p.cols - col), 0, p.cols - col, s[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) { s[0][j] = fmaf(d[j], xh[j], s[0][j]); c = fmaf(d[j] * g[j], xh[j], c); }
            store_groups<1>(q, col, p.cols - col, s, p, 2152);
        }
        c = row_sum(c, red[parity], NT / 32) / (float)p.cols;
        for (int col = 8 * t; col < end; col += 8 * NT) {
            float d[8], xh[8], g[8], b[8], out[1][8];
            both8(col, d, xh, g);
            if (p.dresidual) number8(p.dresidual, p.ldr, row, col, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                out[0][j] = rs * (d[j] * g[j] - xh[j] * c);
                if (p.dresidual) out[0][j] += b[j];
            }
            store_groups<AL>(static_cast<T*>(p.dx) + row * p.ldx, col, p.cols - col, out, p, 2151);
        }
    }
}

// dgain[col] = sum of the rows of partial: 32 columns a block, 32 warps that take every 32nd row, then the warps in order
__global__ void __launch_bounds__(1024) column_sum_kernel(const BackParams p)
{
    __shared__ float red[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    fmmptx::griddep_wait();
    float s = 0.0f;
    if (col < p.cols) {
#pragma unroll 4
        for (int r = warp; r < p.parts; r += 32) s += p.partial[(int64_t)r * p.ldp + col];
    }
    red[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < p.cols) {
        s = 0.0f;
#pragma unroll
        for (int w = 0; w < 32; ++w) s += red[w][lane];
        if (ROW_STORE_OK(p.dgain + col, 4, 2161)) p.dgain[col] = s;
    }
}

// ---------------------------------------------------------------------------------------- launches
fmm_status_t launched() { return cudaGetLastError() == cudaSuccess ? FMM_OK : FMM_ERR_CUDA; }

// behind: set up while the kernel before drains, for which it waits itself
template <typename... P, typename... A> fmm_status_t launch_behind(void (*kernel)(P...), unsigned grid, dim3 block, bool behind, cudaStream_t st, const A&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid); cfg.blockDim = block; cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = behind ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) { cudaGetLastError(); return FMM_ERR_CUDA; }
    return FMM_OK;
}

template <typename T, bool NORM> fmm_status_t launch_rows(const RowsParams& p, cudaStream_t st)
{
    const int groups = (p.cols + 7) / 8;
    const unsigned rows = (unsigned)p.rows;
    const Int8RowForm form = int8_row_form(p.cols);
    const int threads = form.threads;
    const bool full = p.aligned && form.whole && p.vc && (!p.block || p.vk);
    auto launch = [&](auto al) {
        constexpr int AL = decltype(al)::value;
        if (groups <= 64) rows_kernel<T, NORM, AL, 2, true><<<(rows + 3) / 4, dim3(32, 4), 0, st>>>(p);
        else if (groups <= 128) rows_kernel<T, NORM, AL, 4, true><<<(rows + 3) / 4, dim3(32, 4), 0, st>>>(p);
        else if (groups <= 2048) rows_kernel<T, NORM, AL, 4, false><<<rows, threads, 0, st>>>(p);
        else rows_long_kernel<T, NORM, AL ? 1 : 0><<<rows, 1024, 0, st>>>(p);
    };
    if (full) launch(std::integral_constant<int, 2>{});
    else if (p.aligned) launch(std::integral_constant<int, 1>{});
    else launch(std::integral_constant<int, 0>{});
    return launched();
}

// Threads among which a row of the norm's gradients is split (0: long rows), and blocks.  A group of threads has at least four rows, so that
// what it adds to the columns' sums is worth writing out.
struct BackShape { int threads, blocks; };
BackShape back_shape(int64_t rows, int64_t cols)
{
    const int64_t groups = (cols + 7) / 8;
    const int threads = groups <= 1024 ? (int)(groups + 32 * BACK_VPT - 1) / (32 * BACK_VPT) * 32 : 0;
    const int64_t per_sm = threads == 32 ? 4 : threads ? 512 / threads : 1, rows_at_once = threads == 32 ? 4 : 1;
    const int64_t resident = (int64_t)int8_sm_count() * per_sm, by_rows = (rows + 4 * rows_at_once - 1) / (4 * rows_at_once);
    return {threads, (int)(by_rows < 1 ? 1 : by_rows < resident ? by_rows : resident)};
}
int64_t partial_ld(int64_t cols) { return (cols + 7) / 8 * 8; }

template <typename T> fmm_status_t launch_back(const BackParams& p, int threads, cudaStream_t st)
{
    const unsigned blocks = (unsigned)p.parts;
    auto launch = [&](auto al) {
        constexpr int AL = decltype(al)::value;
        if (threads == 32) back_kernel<T, AL, true><<<blocks, dim3(32, 4), 0, st>>>(p);
        else if (threads) back_kernel<T, AL, false><<<blocks, threads, 0, st>>>(p);
        else back_long_kernel<T, AL ? 1 : 0><<<blocks, 1024, 0, st>>>(p);
    };
    // (32-bit rows that fill every thread: 16 bytes more than 128 registers hold, and no faster)
    constexpr int FULL = sizeof(T) == 2 ? 2 : 1;
    if (p.aligned && p.vk && p.cols == 8 * BACK_VPT * threads) launch(std::integral_constant<int, FULL>{});
    else if (p.aligned) launch(std::integral_constant<int, 1>{});
    else launch(std::integral_constant<int, 0>{});
    if (cudaGetLastError() != cudaSuccess) return FMM_ERR_CUDA;
    // set up while the rows are dealt with; it waits for them before its first load
    return launch_behind(column_sum_kernel, (unsigned)(p.cols + 31) / 32, dim3(1024), true, st, p);
}

// eight warps of a block without a reduction: pieces of a row along y, rows along z
dim3 flat_block(int cols)
{
    unsigned y = 1;
    while (y < 8 && y * FLAT_PIECE < (unsigned)cols) y *= 2;
    return dim3(32, y, 8 / y);
}
// (a block per row instead of 32 blocks an SM: 16384 x 8192 bf16 quantized in 77.7 instead of 74.2 us, restored in 68.0 instead of 63.8)
unsigned flat_grid(int rows, dim3 block)
{
    const int64_t most = (int64_t)int8_sm_count() * 32;
    const int64_t need = ((int64_t)rows + block.z - 1) / block.z;
    return (unsigned)(need < most ? need : most);
}

bool dims_ok(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && rows < INT8_MAX_DIM && cols < INT8_MAX_DIM; }
bool block_ok(int block) { return block == 0 || block == 32 || block == 128; }
// a matrix that is read or written: present, rows not overlapping, elements aligned
bool matrix_ok(const void* p, int64_t cols, int64_t ld, int element) { return p && ld >= cols && !((uintptr_t)p & (element - 1)); }

}  // namespace

int int8_scale_maxima_count(int64_t rows)
{
    return rows <= OWN_MAXIMUM ? 1 : (int)std::min<int64_t>((rows + 1023) / 1024, INT8_MAXIMA);
}

static ValuesParams values_params(int parts, const int8_t* codes, int64_t ldc, const float* scales, uint8_t* flags, void* x, int64_t ldx, int64_t step, int64_t rows,
                                  int64_t cols)
{
    ValuesParams p = {codes, scales, flags, x, ldc, ldx, step, (int)rows, (int)cols, parts, int8_scale_maxima_count(rows), int8_aligned(codes, ldc, 8), {}};
    for (int i = 0; i < parts; ++i) int8_add_range(p.ranges, static_cast<char*>(x) + 2 * i * step, rows, ldx, ldx, 2);
    int8_add_range(p.ranges, flags, 1, (rows + INT8_PART_ROWS - 1) / INT8_PART_ROWS, rows, 1);
    return p;
}

fmm_status_t int8_values(fmm_type_t type, int parts, const int8_t* codes, int64_t ldc, const float* scales, uint32_t* maxima, uint8_t* flags, void* x, int64_t ldx,
                         int64_t step, int64_t rows, int64_t cols, cudaStream_t st)
{
    const ValuesParams p = values_params(parts, codes, ldc, scales, flags, x, ldx, step, rows, cols);
    const bool apart = maxima && rows > OWN_MAXIMUM;
    if (apart) {
        scale_maxima_kernel<<<(unsigned)p.maxima_count, 1024, 0, st>>>(scales, (int)rows, maxima);
        if (launched() != FMM_OK) return FMM_ERR_CUDA;
    }
    const dim3 b = flat_block((int)cols);
    return launch_behind(type == FMM_TYPE_BF16 ? values_kernel<__nv_bfloat16> : values_kernel<__half>, flat_grid((int)rows, b), dim3(256), apart, st, p, maxima,
                         (int)b.y);
}

fmm_status_t int8_codes_and_scaled_rows(const int8_t* codes, int64_t ldc, void* values, int64_t ldv, int64_t code_rows, int64_t code_cols, const void* x, int64_t ldx,
                                        const float* scales, void* y, int64_t ldy, float* inverse, int64_t rows, cudaStream_t st)
{
    const int64_t cols = code_rows;
    const ValuesParams v = values_params(1, codes, ldc, nullptr, nullptr, values, ldv, 0, code_rows, code_cols);
    ScaledParams p = {static_cast<const __nv_bfloat16*>(x), scales, static_cast<__half*>(y), inverse, ldx, ldy, (int)rows, (int)cols, 1, int8_aligned(scales, 0, 16), {}};
    int8_add_range(p.ranges, y, rows, ldy, ldy, 2);
    int8_add_range(p.ranges, inverse, 1, rows, rows, 4);
    const dim3 b = flat_block((int)code_cols);
    const unsigned value_blocks = flat_grid((int)code_rows, b);
    const int64_t sms = int8_sm_count();
    const bool aligned = cols % 8 == 0 && int8_aligned(x, ldx * 2, 16);
    const int vpt = cols <= 8 * 2 * GROUP ? 2 : 4, piece = vpt * GROUP;
    const bool fits = cols <= 8 * piece, together = fits && vpt == 2;
    if (!together) {
        const fmm_status_t s = launch_behind(values_kernel<__half>, value_blocks, dim3(256), false, st, v, (uint32_t*)nullptr, (int)b.y);
        if (s != FMM_OK) return s;
    }
    if (!fits) {
        const bool many = rows >= 8 * sms;
        const auto kernel = many ? (aligned ? scaled_long_kernel<1, 4> : scaled_long_kernel<0, 4>) : aligned ? scaled_long_kernel<1, 1> : scaled_long_kernel<0, 1>;
        return launch_behind(kernel, (unsigned)(many ? (rows + 3) / 4 : rows), dim3(512), true, st, p);
    }
    while (p.warps * piece < cols) p.warps *= 2;
    const int64_t per_block = 8 / p.warps;
    const unsigned blocks = (unsigned)std::min((rows + per_block - 1) / per_block, (vpt == 2 ? 4 : 2) * sms);
    const auto kernel = vpt == 2 ? (aligned ? scaled_rows_kernel<1, 2> : scaled_rows_kernel<0, 2>) : aligned ? scaled_rows_kernel<1, 4> : scaled_rows_kernel<0, 4>;
    return launch_behind(kernel, blocks + (together ? value_blocks : 0), dim3(256), !together, st, p, v, (int)blocks, (int)b.y);
}

fmm_status_t int8_realign(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, cudaStream_t st)
{
    RealignParams p = {static_cast<const __half*>(x), static_cast<__half*>(y), ldx, ldy, (int)rows, (int)cols, {}};
    int8_add_range(p.ranges, y, rows, ldy, ldy, 2);
    const dim3 b = flat_block((int)cols);
    realign_kernel<<<flat_grid((int)rows, b), b, 0, st>>>(p);
    return launched();
}

fmm_status_t int8_rows_guard_read(int* code, bool clear)
{
    *code = 0;
#ifdef FMM_DEBUG
    const int zero = 0;
    const cudaError_t e = clear ? cudaMemcpyToSymbol(g_int8_rows_guard, &zero, sizeof(int)) : cudaMemcpyFromSymbol(code, g_int8_rows_guard, sizeof(int));
    if (e != cudaSuccess) { cudaGetLastError(); return FMM_ERR_CUDA; }
#else
    (void)clear;
#endif
    return FMM_OK;
}

extern "C" {

fmm_status_t fmm_int8_quantize(const fmm_int8_quantize_t* a, void* stream)
{
    if (!a || !int8_type_ok(a->type) || !block_ok(a->block) ||
        (a->scale_mode != FMM_INT8_SCALE_AMAX_DIV_127 && a->scale_mode != FMM_INT8_SCALE_POW2)) return FMM_ERR_INVALID_ARG;
    if (!dims_ok(a->rows, a->cols)) return FMM_ERR_SHAPE;
    const int64_t rows = a->rows, cols = a->cols, ldx = a->ldx, ldc = a->ldc;
    const int block = a->block, e = int8_type_bytes(a->type);
    const fmm_type_t type = a->type;
    const void* X = a->x;
    int8_t* codes = a->codes;
    float* scales = a->scales;
    if (rows == 0 || (cols == 0 && block)) return FMM_OK;
    if (!matrix_ok(scales, 1, 1, 4) || (cols > 0 && (!matrix_ok(X, cols, ldx, e) || !matrix_ok(codes, cols, ldc, 1)))) return FMM_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool vx = int8_aligned(X, ldx * e, 16) && cols % 8 == 0, vc = int8_aligned(codes, ldc, 8), pow2 = a->scale_mode == FMM_INT8_SCALE_POW2;
    Int8Ranges ranges = {};
    int8_add_range(ranges, codes, rows, cols, ldc, 1);
    if (block) {
        const int64_t per_row = (cols + block - 1) / block;
        int8_add_range(ranges, scales, rows, per_row, per_row, 4);
        const BlocksParams p = {X, codes, scales, ldx, ldc, (int)rows, (int)cols, block, pow2, vc, ranges};
        const dim3 b = flat_block((int)cols);
        const unsigned grid = flat_grid((int)rows, b);
        auto launch = [&](auto type) {
            using T = decltype(type);
            if (vx && vc && cols % FLAT_PIECE == 0) quantize_blocks_kernel<T, 2><<<grid, b, 0, st>>>(p);
            else if (vx) quantize_blocks_kernel<T, 1><<<grid, b, 0, st>>>(p);
            else quantize_blocks_kernel<T, 0><<<grid, b, 0, st>>>(p);
        };
        if (type == FMM_TYPE_F32) launch(float{});
        else if (type == FMM_TYPE_BF16) launch(__nv_bfloat16{});
        else launch(__half{});
        return launched();
    }
    int8_add_range(ranges, scales, 1, rows, rows, 4);
    RowsParams p = {};
    p.x = X; p.ldx = ldx; p.codes = codes; p.ldc = ldc; p.scales = scales;
    p.rows = (int)rows; p.cols = (int)cols; p.pow2 = pow2; p.aligned = vx; p.vc = vc; p.ranges = ranges;
    if (cols == 0) {
        no_columns_kernel<<<(unsigned)((rows + 255) / 256), 256, 0, st>>>(p);
        return launched();
    }
    if (type == FMM_TYPE_F32) return launch_rows<float, false>(p, st);
    if (type == FMM_TYPE_BF16) return launch_rows<__nv_bfloat16, false>(p, st);
    return launch_rows<__half, false>(p, st);
}

fmm_status_t fmm_int8_dequantize(const fmm_int8_dequantize_t* a, void* stream)
{
    if (!a || !int8_type_ok(a->type) || !block_ok(a->block)) return FMM_ERR_INVALID_ARG;
    if (!dims_ok(a->rows, a->cols)) return FMM_ERR_SHAPE;
    const int64_t rows = a->rows, cols = a->cols, ldx = a->ldx, ldc = a->ldc;
    const int block = a->block, e = int8_type_bytes(a->type);
    const fmm_type_t type = a->type;
    const int8_t* codes = a->codes;
    const float* scales = a->scales;
    void* X = a->x;
    if (rows == 0 || cols == 0) return FMM_OK;
    if (!matrix_ok(codes, cols, ldc, 1) || !matrix_ok(scales, 1, 1, 4) || !matrix_ok(X, cols, ldx, e)) return FMM_ERR_INVALID_ARG;
    Int8Ranges ranges = {};
    int8_add_range(ranges, X, rows, cols, ldx, e);
    const RestoreParams p = {codes, scales, X, ldc, ldx, (int)rows, (int)cols, block, int8_aligned(codes, ldc, 8), ranges};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const dim3 b = flat_block((int)cols);
    const unsigned grid = flat_grid((int)rows, b);
    auto launch = [&](auto type) {
        using T = decltype(type);
        const bool aligned = int8_aligned(X, ldx * e, 16) && cols % 8 == 0;
        if (aligned && p.vc && cols % FLAT_PIECE == 0) dequantize_kernel<T, 2><<<grid, b, 0, st>>>(p);
        else if (aligned) dequantize_kernel<T, 1><<<grid, b, 0, st>>>(p);
        else dequantize_kernel<T, 0><<<grid, b, 0, st>>>(p);
    };
    if (type == FMM_TYPE_F32) launch(float{});
    else if (type == FMM_TYPE_BF16) launch(__nv_bfloat16{});
    else launch(__half{});
    return launched();
}

fmm_status_t fmm_int8_rms_norm(const fmm_int8_rms_norm_t* a, void* stream)
{
    if (!a || !int8_type_ok(a->type) || !block_ok(a->checkpoint_block) ||
        (a->scale_mode != FMM_INT8_SCALE_AMAX_DIV_127 && a->scale_mode != FMM_INT8_SCALE_POW2) || !(a->eps >= 0.0) || isinf(a->eps))
        return FMM_ERR_INVALID_ARG;
    if (!dims_ok(a->rows, a->cols)) return FMM_ERR_SHAPE;
    if (a->rows == 0 || a->cols == 0) return FMM_OK;
    const int e = int8_type_bytes(a->type);
    const int64_t rows = a->rows, cols = a->cols, per_row = a->checkpoint_block ? (cols + a->checkpoint_block - 1) / a->checkpoint_block : 0;
    if (!matrix_ok(a->x, cols, a->ldx, e) || !matrix_ok(a->gain, cols, cols, e) || !matrix_ok(a->codes, cols, a->ldc, 1) || !matrix_ok(a->scales, 1, 1, 4) ||
        ((uintptr_t)a->rstd & 3) || (a->residual && (!matrix_ok(a->residual, cols, a->ldr, e) || !matrix_ok(a->hidden, cols, a->ldh, e))) ||
        (per_row && (!matrix_ok(a->checkpoint, cols, a->ldk, 1) || !matrix_ok(a->checkpoint_scales, 1, 1, 4))))
        return FMM_ERR_INVALID_ARG;
    RowsParams p = {};
    p.x = a->x; p.residual = a->residual; p.gain = a->gain; p.hidden = a->hidden; p.codes = a->codes; p.scales = a->scales; p.rstd = a->rstd;
    p.checkpoint = a->checkpoint; p.checkpoint_scales = a->checkpoint_scales;
    p.ldx = a->ldx; p.ldr = a->ldr; p.ldh = a->ldh; p.ldc = a->ldc; p.ldk = a->ldk;
    p.eps = a->eps; p.rows = (int)rows; p.cols = (int)cols; p.block = a->checkpoint_block; p.pow2 = a->scale_mode == FMM_INT8_SCALE_POW2;
    p.aligned = cols % 8 == 0 && int8_aligned(a->x, a->ldx * e, 16) && int8_aligned(a->gain, 0, 16) &&
                (!a->residual || (int8_aligned(a->residual, a->ldr * e, 16) && int8_aligned(a->hidden, a->ldh * e, 16)));
    p.vc = int8_aligned(a->codes, a->ldc, 8); p.vk = int8_aligned(a->checkpoint, a->ldk, 8);
    if (a->residual) int8_add_range(p.ranges, a->hidden, rows, cols, a->ldh, e);
    int8_add_range(p.ranges, a->codes, rows, cols, a->ldc, 1);
    int8_add_range(p.ranges, a->scales, 1, rows, rows, 4);
    int8_add_range(p.ranges, a->rstd, 1, rows, rows, 4);
    if (per_row) {
        int8_add_range(p.ranges, a->checkpoint, rows, cols, a->ldk, 1);
        int8_add_range(p.ranges, a->checkpoint_scales, rows, per_row, per_row, 4);
    }
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (a->type == FMM_TYPE_F32) return launch_rows<float, true>(p, st);
    if (a->type == FMM_TYPE_BF16) return launch_rows<__nv_bfloat16, true>(p, st);
    return launch_rows<__half, true>(p, st);
}

fmm_status_t fmm_int8_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols, size_t* bytes)
{
    if (!bytes) return FMM_ERR_INVALID_ARG;
    if (!dims_ok(rows, cols)) return FMM_ERR_SHAPE;
    *bytes = (size_t)back_shape(rows, cols).blocks * (size_t)partial_ld(cols) * 4;
    return FMM_OK;
}

fmm_status_t fmm_int8_rms_norm_backward(const fmm_int8_rms_norm_backward_t* a, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!a || !int8_type_ok(a->type) || !block_ok(a->block)) return FMM_ERR_INVALID_ARG;
    if (!dims_ok(a->rows, a->cols)) return FMM_ERR_SHAPE;
    if (a->cols == 0) return FMM_OK;
    const int e = int8_type_bytes(a->type);
    const int64_t rows = a->rows, cols = a->cols;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (!matrix_ok(a->dgain, 1, 1, 4)) return FMM_ERR_INVALID_ARG;
    if (rows == 0) {
        const cudaError_t z = cudaMemsetAsync(a->dgain, 0, (size_t)cols * 4, st);
        if (z != cudaSuccess) cudaGetLastError();
        return z == cudaSuccess ? FMM_OK : FMM_ERR_CUDA;
    }
    if (!matrix_ok(a->dy, cols, a->ldy, e) || !matrix_ok(a->checkpoint, cols, a->ldk, 1) || !matrix_ok(a->checkpoint_scales, 1, 1, 4) ||
        !matrix_ok(a->rstd, 1, 1, 4) || !matrix_ok(a->gain, cols, cols, e) || !matrix_ok(a->dx, cols, a->ldx, e) ||
        (a->dresidual && !matrix_ok(a->dresidual, cols, a->ldr, e)))
        return FMM_ERR_INVALID_ARG;
    const BackShape shape = back_shape(rows, cols);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < (size_t)shape.blocks * (size_t)partial_ld(cols) * 4) return FMM_ERR_WORKSPACE;
    BackParams p = {};
    p.dy = a->dy; p.checkpoint = a->checkpoint; p.scales = a->checkpoint_scales; p.rstd = a->rstd; p.gain = a->gain; p.dresidual = a->dresidual;
    p.dx = a->dx; p.dgain = a->dgain; p.partial = static_cast<float*>(workspace);
    p.ldy = a->ldy; p.ldk = a->ldk; p.ldr = a->ldr; p.ldx = a->ldx;
    p.ldp = partial_ld(cols);
    p.rows = (int)rows; p.cols = (int)cols; p.block = a->block; p.parts = shape.blocks;
    p.aligned = cols % 8 == 0 && int8_aligned(a->dy, a->ldy * e, 16) && int8_aligned(a->gain, 0, 16) && int8_aligned(a->dx, a->ldx * e, 16) &&
                (!a->dresidual || int8_aligned(a->dresidual, a->ldr * e, 16));
    p.vk = int8_aligned(a->checkpoint, a->ldk, 8);
    int8_add_range(p.ranges, a->dx, rows, cols, a->ldx, e);
    int8_add_range(p.ranges, a->dgain, 1, cols, cols, 4);
    int8_add_range(p.ranges, workspace, shape.blocks, p.ldp, p.ldp, 4);
    if (a->type == FMM_TYPE_F32) return launch_back<float>(p, shape.threads, st);
    if (a->type == FMM_TYPE_BF16) return launch_back<__nv_bfloat16>(p, shape.threads, st);
    return launch_back<__half>(p, shape.threads, st);
}

}  // extern "C"
