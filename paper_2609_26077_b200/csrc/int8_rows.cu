// Row kernels of the 8-bit integer layer: quantization, restoring, the root-mean-square norm with 8-bit output, and that
// norm's gradients from an 8-bit checkpoint.  All of them are bound by memory: every kernel reads each input and writes
// each output once, rows staying in registers between the passes that a row needs (sum of squares, maximum, codes).
//
// A thread owns groups of eight consecutive columns (16 bytes of a 16-bit type); group v of a row is thread v mod NT, so
// that a block of 32 (128) columns is 4 (16) neighbouring lanes of one warp and its maximum takes 2 (4) shuffles.
#include <math.h>
#include "int8_internal.h"

namespace {

#ifdef FMM_DEBUG
__device__ int g_int8_rows_guard;
#endif
#define ROW_STORE_OK(ptr, bytes, code) INT8_STORE_OK(p.ranges, ptr, bytes, code, &g_int8_rows_guard)

// ---------------------------------------------------------------------------------------- eight columns of a row
template <typename T> struct Raw8 { uint32_t w[sizeof(T) * 2]; };

// columns [0, n) of p, zeros behind; n may be 0 or less.  vec: p is 16-byte aligned
template <typename T> __device__ __forceinline__ Raw8<T> load8(const T* p, int n, bool vec)
{
    Raw8<T> r;
    if (vec && n >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(p)[i];
            r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
        }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = i < n ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
    } else {
        const uint16_t* s = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = (2 * i < n ? (uint32_t)s[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)s[2 * i + 1] << 16 : 0u);
    }
    return r;
}
template <typename T> __device__ __forceinline__ void unpack8(const Raw8<T>& r, float (&f)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(r.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            T a, b;
            const uint16_t lo = (uint16_t)r.w[i], hi = (uint16_t)(r.w[i] >> 16);
            a = *reinterpret_cast<const T*>(&lo); b = *reinterpret_cast<const T*>(&hi);
            f[2 * i] = to_float(a); f[2 * i + 1] = to_float(b);
        }
    }
}
template <typename T> __device__ __forceinline__ Raw8<T> pack8(const float (&f)[8])
{
    Raw8<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = pack_two<T>(f[2 * i], f[2 * i + 1]);
    }
    return r;
}
template <typename T, typename P> __device__ __forceinline__ void store8(T* q, const float (&f)[8], int n, bool vec, const P& p, int code)
{
    if (n <= 0 || !ROW_STORE_OK(q, (n < 8 ? n : 8) * sizeof(T), code)) return;
    if (vec && n >= 8) {
        const Raw8<T> r = pack8<T>(f);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            reinterpret_cast<uint4*>(q)[i] = make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) q[i] = from_float<T>(f[i]);
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
__device__ __forceinline__ void codes_to_float(uint2 c, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)(int8_t)((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
}

// ---------------------------------------------------------------------------------------- quantization of a block
// Maxima are taken over the bit patterns of |x|: they order like the numbers, infinities above them and NaN above those, so
// that a block that holds one of these is seen, and gets NaN as its scale.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t abs_max8(const float (&f)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs_bits(f[i]));
    return m;
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
// maximum over aligned groups of `lanes` (4, 16 or 32) lanes
__device__ __forceinline__ uint32_t group_max(uint32_t m, int lanes)
{
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    if (lanes > 4) {
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 4));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 8));
    }
    return m;
}

// ---------------------------------------------------------------------------------------- sums over a row's threads
template <int NT> __device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t* red)
{
    m = __reduce_max_sync(0xffffffffu, m);
    if constexpr (NT > 32) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        m = __reduce_max_sync(0xffffffffu, lane < NT / 32 ? red[lane] : 0u);
    }
    return m;
}
// always the same order: lanes by halves, then the warps by halves
template <int NT, typename F> __device__ __forceinline__ F row_sum(F v, F* red)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (NT > 32) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = lane < NT / 32 ? red[lane] : (F)0;
#pragma unroll
        for (int o = NT / 64; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        v = __shfl_sync(0xffffffffu, v, 0);
    }
    return v;
}

// ---------------------------------------------------------------------------------------- norm / row-wise quantization
struct RowsParams {
    const void* x; const void* residual; const void* gain;
    void* hidden; int8_t* codes; float* scales; float* rstd;
    int8_t* checkpoint; float* checkpoint_scales;
    int64_t ldx, ldr, ldh, ldc, ldk;
    double eps;
    int rows, cols, block;                    // block: of the checkpoint, 0: none
    bool pow2, vx, vr, vg, vh, vc, vk;        // which arrays have aligned rows
    Int8Ranges ranges;
};

template <typename T> __device__ __forceinline__ void checkpoint8(const RowsParams& p, int64_t row, int col, const float (&h)[8])
{
    const int lanes = p.block / 8, n = p.cols - col;
    const Scale s = block_scale(group_max(abs_max8(h), lanes), false);
    if (n <= 0) return;
    store_codes8(p.checkpoint + row * p.ldk + col, codes8(h, s.inverse), n, p.vk, p, 2101);
    if ((col / 8) % lanes == 0) {
        float* q = p.checkpoint_scales + row * ((p.cols + p.block - 1) / p.block) + col / p.block;
        if (ROW_STORE_OK(q, 4, 2102)) *q = s.scale;
    }
}

// A row per NT threads, held in registers: VPT groups of eight columns a thread.  The squares are summed in fp64 (they are
// exact there), so that the reciprocal root does not depend on the order of the sum and codes are the same on every machine.
template <typename T, bool NORM, int NT, int VPT>
__global__ void __launch_bounds__(NT == 32 ? 128 : NT) rows_kernel(const RowsParams p)
{
    __shared__ double red_sum[32];
    __shared__ uint32_t red_max[32];
    constexpr int RPC = NT == 32 ? 4 : 1;
    const int t = threadIdx.x;
    int64_t row = (int64_t)blockIdx.x * RPC + threadIdx.y;
    if (RPC > 1 && row >= p.rows) return;                     // whole warps
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    float h[VPT][8];
    Raw8<T> raw[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) { const int col = 8 * (i * NT + t); raw[i] = load8(x + col, p.cols - col, p.vx); }
    if constexpr (NORM) {
        if (p.residual) {
            const T* r = static_cast<const T*>(p.residual) + row * p.ldr;
            Raw8<T> rawr[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) { const int col = 8 * (i * NT + t); rawr[i] = load8(r + col, p.cols - col, p.vr); }
            T* hid = static_cast<T*>(p.hidden) + row * p.ldh;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int col = 8 * (i * NT + t);
                float b[8];
                unpack8(raw[i], h[i]);
                unpack8(rawr[i], b);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = __fadd_rn(h[i][j], b[j]);
                store8(hid + col, h[i], p.cols - col, p.vh, p, 2103);
            }
        } else {
#pragma unroll
            for (int i = 0; i < VPT; ++i) unpack8(raw[i], h[i]);
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) { const int col = 8 * (i * NT + t); raw[i] = load8(static_cast<const T*>(p.gain) + col, p.cols - col, p.vg); }
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) { const double v = (double)h[i][j]; sum = fma(v, v, sum); }
        if (p.block) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) checkpoint8<T>(p, row, 8 * (i * NT + t), h[i]);
        }
        sum = row_sum<NT>(sum, red_sum);
        const float rstd = (float)(1.0 / sqrt(sum / (double)p.cols + p.eps));
        if (t == 0 && p.rstd && ROW_STORE_OK(p.rstd + row, 4, 2104)) p.rstd[row] = rstd;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float g[8];
            unpack8(raw[i], g);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] = __fmul_rn(__fmul_rn(h[i][j], rstd), g[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPT; ++i) unpack8(raw[i], h[i]);
    }
    // behind the last column: h is 0 there, and 0 * rstd is NaN where rstd is infinite (a row of zeros with eps 0), which is what
    // the row's own zeros are as well
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) m = max(m, abs_max8(h[i]));
    m = row_max<NT>(m, red_max);
    const Scale s = block_scale(m, p.pow2);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int col = 8 * (i * NT + t);
        store_codes8(p.codes + row * p.ldc + col, codes8(h[i], s.inverse), p.cols - col, p.vc, p, 2105);
    }
    if (t == 0 && ROW_STORE_OK(p.scales + row, 4, 2106)) p.scales[row] = s.scale;
}

// Rows that do not fit registers: read again for each pass (from L2, mostly).  hidden may be x or residual, so it is written in the
// last pass.
template <typename T, bool NORM>
__global__ void __launch_bounds__(1024) rows_long_kernel(const RowsParams p)
{
    constexpr int NT = 1024;
    __shared__ double red_sum[32];
    __shared__ uint32_t red_max[32];
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x, groups = (p.cols + 7) / 8;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const T* r = NORM && p.residual ? static_cast<const T*>(p.residual) + row * p.ldr : nullptr;
    auto hidden8 = [&](int col, float (&h)[8]) {
        unpack8(load8(x + col, p.cols - col, p.vx), h);
        if (r) {
            float b[8];
            unpack8(load8(r + col, p.cols - col, p.vr), b);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = __fadd_rn(h[j], b[j]);
        }
    };
    float rstd = 1.0f;
    if constexpr (NORM) {
        double sum = 0.0;
        for (int v = t; v < (groups + NT - 1) / NT * NT; v += NT) {          // every lane goes round as often: checkpoint8 shuffles
            float h[8];
            hidden8(8 * v, h);
#pragma unroll
            for (int j = 0; j < 8; ++j) { const double d = (double)h[j]; sum = fma(d, d, sum); }
            if (p.block) checkpoint8<T>(p, row, 8 * v, h);
        }
        sum = row_sum<NT>(sum, red_sum);
        rstd = (float)(1.0 / sqrt(sum / (double)p.cols + p.eps));
        if (t == 0 && p.rstd && ROW_STORE_OK(p.rstd + row, 4, 2114)) p.rstd[row] = rstd;
    }
    auto normed8 = [&](int col, float (&h)[8]) {
        if constexpr (NORM) {
            float g[8];
            unpack8(load8(static_cast<const T*>(p.gain) + col, p.cols - col, p.vg), g);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = __fmul_rn(__fmul_rn(h[j], rstd), g[j]);
        }
    };
    uint32_t m = 0;
    for (int v = t; v < groups; v += NT) {
        float h[8];
        hidden8(8 * v, h);
        normed8(8 * v, h);
        m = max(m, abs_max8(h));
    }
    const Scale s = block_scale(row_max<NT>(m, red_max), p.pow2);
    for (int v = t; v < groups; v += NT) {
        float h[8];
        hidden8(8 * v, h);
        if (r) store8(static_cast<T*>(p.hidden) + row * p.ldh + 8 * v, h, p.cols - 8 * v, p.vh, p, 2113);
        normed8(8 * v, h);
        store_codes8(p.codes + row * p.ldc + 8 * v, codes8(h, s.inverse), p.cols - 8 * v, p.vc, p, 2115);
    }
    if (t == 0 && ROW_STORE_OK(p.scales + row, 4, 2116)) p.scales[row] = s.scale;
}

// ---------------------------------------------------------------------------------------- quantization in blocks
struct BlocksParams {
    const void* x; int8_t* codes; float* scales;
    int64_t ldx, ldc;
    int rows, cols, block;
    bool pow2, vx, vc;
    Int8Ranges ranges;
};
// No row is reduced: a warp takes 256 columns at a time.  blockDim (columns / 8, rows)
template <typename T>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const BlocksParams p)
{
    const int lanes = p.block / 8, per_row = (p.cols + p.block - 1) / p.block, rounds = (p.cols + 255) / 256 * 32;
    for (int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; row < p.rows; row += (int64_t)gridDim.x * blockDim.y) {
        const T* x = static_cast<const T*>(p.x) + row * p.ldx;
#pragma unroll 2
        for (int v = threadIdx.x; v < rounds; v += blockDim.x) {
            const int col = 8 * v, n = p.cols - col;
            float f[8];
            unpack8(load8(x + col, n, p.vx), f);
            const Scale s = block_scale(group_max(abs_max8(f), lanes), p.pow2);
            if (n <= 0) continue;
            store_codes8(p.codes + row * p.ldc + col, codes8(f, s.inverse), n, p.vc, p, 2121);
            if (v % lanes == 0) {
                float* q = p.scales + row * per_row + v / lanes;
                if (ROW_STORE_OK(q, 4, 2122)) *q = s.scale;
            }
        }
    }
}

// ---------------------------------------------------------------------------------------- restoring
struct RestoreParams {
    const int8_t* codes; const float* scales; void* x;
    int64_t ldc, ldx;
    int rows, cols, block;
    bool vc, vx;
    Int8Ranges ranges;
};
template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(const RestoreParams p)
{
    const int per_row = p.block ? (p.cols + p.block - 1) / p.block : 1, groups = (p.cols + 7) / 8, shift = p.block == 32 ? 2 : 4;
    for (int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; row < p.rows; row += (int64_t)gridDim.x * blockDim.y) {
        const int8_t* codes = p.codes + row * p.ldc;
        const float* scales = p.scales + row * per_row;
        T* x = static_cast<T*>(p.x) + row * p.ldx;
#pragma unroll 4
        for (int v = threadIdx.x; v < groups; v += blockDim.x) {
            float f[8];
            const uint2 c = load_codes8(codes + 8 * v, p.cols - 8 * v, p.vc);
            const float s = scales[p.block ? v >> shift : 0];
            codes_to_float(c, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = __fmul_rn(f[j], s);
            store8(x + 8 * v, f, p.cols - 8 * v, p.vx, p, 2131);
        }
    }
}

// ---------------------------------------------------------------------------------------- the norm's gradients
struct BackParams {
    const void* dy; const int8_t* checkpoint; const float* scales; const float* rstd; const void* gain; const void* dresidual;
    void* dx; float* dgain; float* partial;
    int64_t ldy, ldk, ldr, ldx;
    int rows, cols, block, parts;             // parts: rows of `partial`
    bool vy, vk, vg, vr, vx;
    Int8Ranges ranges;
};

// xhat of eight columns: code * scale * rstd
__device__ __forceinline__ void xhat8(uint2 codes, float scale, float rstd, float (&f)[8])
{
    codes_to_float(codes, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = f[j] * scale * rstd;
}

// What a thread holds of a row.
template <typename T, int VPT> struct BackRow {
    Raw8<T> dy[VPT], dresidual[VPT];
    uint2 codes[VPT];
    float scale[VPT], rstd;
};

// Rows are dealt out to `parts` groups of NT threads; a thread keeps its columns' sums of dy * xhat in registers over all rows of its
// group and writes them once, as one row of `partial`; column_sum_kernel adds those rows up in a fixed order.  A row is held as it was
// read and its numbers are formed twice, before and after the sum over the row, so that the next row's loads can be in flight
// meanwhile (NEXT) in 128 registers: with two groups of a 16-bit type a thread.  Otherwise the gain, and dresidual behind the sum,
// are loaded where they are used.
template <typename T, int NT, int VPT>
__global__ void __launch_bounds__(NT == 32 ? 128 : NT) back_kernel(const BackParams p)
{
    constexpr bool NEXT = sizeof(T) == 2 && VPT <= 2;
    __shared__ float red[2][32];
    constexpr int RPC = NT == 32 ? 4 : 1;
    const int t = threadIdx.x, part = blockIdx.x * RPC + threadIdx.y;
    if (RPC > 1 && part >= p.parts) return;                   // whole warps
    const int per_row = p.block ? (p.cols + p.block - 1) / p.block : 1, shift = p.block == 32 ? 2 : 4;
    float sum[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[i][j] = 0.0f;
    auto load_gain = [&](int i) { const int col = 8 * (i * NT + t); return load8(static_cast<const T*>(p.gain) + col, p.cols - col, p.vg); };
    auto load_dresidual = [&](int64_t row, int i) {
        const int col = 8 * (i * NT + t);
        return load8(static_cast<const T*>(p.dresidual) + row * p.ldr + col, p.cols - col, p.vr);
    };
    auto fetch = [&](int64_t row) {
        BackRow<T, VPT> r;
        r.rstd = p.rstd[row];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = i * NT + t, col = 8 * v, n = p.cols - col;
            r.dy[i] = load8(static_cast<const T*>(p.dy) + row * p.ldy + col, n, p.vy);
            r.codes[i] = load_codes8(p.checkpoint + row * p.ldk + col, n, p.vk);
            r.scale[i] = n > 0 ? p.scales[row * per_row + (p.block ? v >> shift : 0)] : 0.0f;
        }
        if (NEXT && p.dresidual) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) r.dresidual[i] = load_dresidual(row, i);
        }
        return r;
    };
    Raw8<T> g[VPT];
    if (NEXT) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) g[i] = load_gain(i);
    }
    BackRow<T, VPT> next;
    if (NEXT && part < p.rows) next = fetch(part);
    int parity = 0;
    for (int64_t row = part; row < p.rows; row += p.parts, parity ^= 1) {
        const BackRow<T, VPT> r = NEXT ? next : fetch(row);
        if (NEXT && row + p.parts < p.rows) next = fetch(row + p.parts);
        float c = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float d[8], gg[8], xh[8];
            unpack8(r.dy[i], d);
            unpack8(NEXT ? g[i] : load_gain(i), gg);
            xhat8(r.codes[i], r.scale[i], r.rstd, xh);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum[i][j] = fmaf(d[j], xh[j], sum[i][j]);
                c = fmaf(d[j] * gg[j], xh[j], c);
            }
        }
        c = row_sum<NT>(c, red[parity]) / (float)p.cols;
        T* dx = static_cast<T*>(p.dx) + row * p.ldx;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int col = 8 * (i * NT + t);
            float d[8], gg[8], xh[8];
            unpack8(r.dy[i], d);
            unpack8(NEXT ? g[i] : load_gain(i), gg);
            xhat8(r.codes[i], r.scale[i], r.rstd, xh);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = r.rstd * (d[j] * gg[j] - xh[j] * c);
            if (p.dresidual) {
                float b[8];
                unpack8(NEXT ? r.dresidual[i] : load_dresidual(row, i), b);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] += b[j];
            }
            store8(dx + col, d, p.cols - col, p.vx, p, 2141);
        }
    }
    float* q = p.partial + (int64_t)part * p.cols;
#pragma unroll
    for (int i = 0; i < VPT; ++i) { const int col = 8 * (i * NT + t); store8(q + col, sum[i], p.cols - col, (p.cols & 3) == 0, p, 2142); }
}

// Rows that do not fit registers: dy and the codes are read twice (the second time from L2, mostly), and the sums of a group live in
// its row of `partial`, which no other group touches.
template <typename T>
__global__ void __launch_bounds__(1024) back_long_kernel(const BackParams p)
{
    constexpr int NT = 1024;
    __shared__ float red[2][32];
    const int t = threadIdx.x, part = blockIdx.x, groups = (p.cols + 7) / 8;
    const int per_row = p.block ? (p.cols + p.block - 1) / p.block : 1, shift = p.block == 32 ? 2 : 4;
    float* q = p.partial + (int64_t)part * p.cols;
    const bool vq = (p.cols & 3) == 0;
    int parity = 0;
    for (int64_t row = part; row < p.rows; row += p.parts, parity ^= 1) {
        const float rs = p.rstd[row];
        auto both8 = [&](int v, float (&d)[8], float (&xh)[8]) {
            const int n = p.cols - 8 * v;
            unpack8(load8(static_cast<const T*>(p.dy) + row * p.ldy + 8 * v, n, p.vy), d);
            xhat8(load_codes8(p.checkpoint + row * p.ldk + 8 * v, n, p.vk), p.scales[row * per_row + (p.block ? v >> shift : 0)], rs, xh);
        };
        auto gain8 = [&](int v, float (&g)[8]) { unpack8(load8(static_cast<const T*>(p.gain) + 8 * v, p.cols - 8 * v, p.vg), g); };
        float c = 0.0f;
        for (int v = t; v < groups; v += NT) {
            float d[8], xh[8], g[8], s[8];
            both8(v, d, xh);
            gain8(v, g);
            if (row == part) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = 0.0f;
            } else unpack8(load8<float>(q + 8 * v, p.cols - 8 * v, vq), s);
#pragma unroll
            for (int j = 0; j < 8; ++j) { s[j] = fmaf(d[j], xh[j], s[j]); c = fmaf(d[j] * g[j], xh[j], c); }
            store8(q + 8 * v, s, p.cols - 8 * v, vq, p, 2152);
        }
        c = row_sum<NT>(c, red[parity]) / (float)p.cols;
        for (int v = t; v < groups; v += NT) {
            float d[8], xh[8], g[8], b[8];
            both8(v, d, xh);
            gain8(v, g);
            if (p.dresidual) unpack8(load8(static_cast<const T*>(p.dresidual) + row * p.ldr + 8 * v, p.cols - 8 * v, p.vr), b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                d[j] = rs * (d[j] * g[j] - xh[j] * c);
                if (p.dresidual) d[j] += b[j];
            }
            store8(static_cast<T*>(p.dx) + row * p.ldx + 8 * v, d, p.cols - 8 * v, p.vx, p, 2151);
        }
    }
}

// dgain[col] = sum of the `parts` rows of partial: 32 columns a block, 32 warps that take every 32nd row, then the warps in order
__global__ void __launch_bounds__(1024) column_sum_kernel(const BackParams p)
{
    __shared__ float red[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < p.cols) {
#pragma unroll 4
        for (int r = warp; r < p.parts; r += 32) s += p.partial[(int64_t)r * p.cols + col];
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

template <typename T, bool NORM> fmm_status_t launch_rows(const RowsParams& p, cudaStream_t st)
{
    const int groups = (p.cols + 7) / 8;
    const unsigned rows = (unsigned)p.rows;
    if (groups <= 64) rows_kernel<T, NORM, 32, 2><<<(rows + 3) / 4, dim3(32, 4), 0, st>>>(p);
    else if (groups <= 256) rows_kernel<T, NORM, 128, 2><<<rows, 128, 0, st>>>(p);
    else if (groups <= 512) rows_kernel<T, NORM, 256, 2><<<rows, 256, 0, st>>>(p);
    else if (groups <= 1024) rows_kernel<T, NORM, 256, 4><<<rows, 256, 0, st>>>(p);
    else if (groups <= 2048) rows_kernel<T, NORM, 512, 4><<<rows, 512, 0, st>>>(p);
    else rows_long_kernel<T, NORM><<<rows, 1024, 0, st>>>(p);
    return launched();
}

// groups of threads among which the rows of the norm's gradients are dealt out, and threads of a group (1024: long rows)
struct BackShape { int threads, parts; };
BackShape back_shape(int64_t rows, int64_t cols)
{
    const int64_t groups = (cols + 7) / 8;
    const int threads = groups <= 64 ? 32 : groups <= 256 ? 128 : groups <= 512 ? 256 : groups <= 2048 ? 512 : 1024;
    const int64_t resident = (int64_t)fmm_sm_count() * (1024 / threads);
    const int64_t by_rows = (rows + 3) / 4;
    return {threads, (int)(by_rows < 1 ? 1 : by_rows < resident ? by_rows : resident)};
}

template <typename T> fmm_status_t launch_back(const BackParams& p, int threads, cudaStream_t st)
{
    const unsigned parts = (unsigned)p.parts, groups = (unsigned)(p.cols + 7) / 8;
    if (threads == 32) back_kernel<T, 32, 2><<<(parts + 3) / 4, dim3(32, 4), 0, st>>>(p);
    else if (threads == 128) back_kernel<T, 128, 2><<<parts, 128, 0, st>>>(p);
    else if (threads == 256) back_kernel<T, 256, 2><<<parts, 256, 0, st>>>(p);
    else if (threads == 512 && groups <= 1024) back_kernel<T, 512, 2><<<parts, 512, 0, st>>>(p);
    else if (threads == 512) back_kernel<T, 512, 4><<<parts, 512, 0, st>>>(p);
    else back_long_kernel<T><<<parts, 1024, 0, st>>>(p);
    column_sum_kernel<<<(unsigned)(p.cols + 31) / 32, 1024, 0, st>>>(p);
    return launched();
}

// blocks of 256 threads for row-parallel kernels without a reduction: columns / 8 along x, rows along y
dim3 flat_block(int cols)
{
    unsigned x = 32;
    while (x < 256 && 8u * x < (unsigned)cols) x *= 2;
    return dim3(x, 256 / x);
}
unsigned flat_grid(int rows, dim3 block)
{
    const int64_t need = ((int64_t)rows + block.y - 1) / block.y, most = (int64_t)fmm_sm_count() * 32;
    return (unsigned)(need < most ? need : most);
}

bool dims_ok(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && rows < INT8_MAX_DIM && cols < INT8_MAX_DIM; }
bool block_ok(int block) { return block == 0 || block == 32 || block == 128; }
// a matrix that is read or written: present, rows not overlapping, elements aligned
bool matrix_ok(const void* p, int64_t cols, int64_t ld, int element) { return p && ld >= cols && !((uintptr_t)p & (element - 1)); }

}  // namespace

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

fmm_status_t fmm_int8_quantize(const void* X, fmm_type_t type, int64_t ldx, int64_t rows, int64_t cols, int block,
                               fmm_int8_scale_t scale_mode, int8_t* codes, int64_t ldc, float* scales, void* stream)
{
    if (!int8_type_ok(type) || !block_ok(block) || (scale_mode != FMM_INT8_SCALE_AMAX_DIV_127 && scale_mode != FMM_INT8_SCALE_POW2)) return FMM_ERR_INVALID_ARG;
    if (!dims_ok(rows, cols)) return FMM_ERR_SHAPE;
    if (rows == 0 || (cols == 0 && block)) return FMM_OK;
    const int e = int8_type_bytes(type);
    if (!matrix_ok(scales, 1, 1, 4) || (cols > 0 && (!matrix_ok(X, cols, ldx, e) || !matrix_ok(codes, cols, ldc, 1)))) return FMM_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool vx = int8_aligned(X, ldx * e, 16), vc = int8_aligned(codes, ldc, 8), pow2 = scale_mode == FMM_INT8_SCALE_POW2;
    Int8Ranges ranges = {};
    int8_add_range(ranges, codes, rows, cols, ldc, 1);
    if (block) {
        const int64_t per_row = (cols + block - 1) / block;
        int8_add_range(ranges, scales, rows, per_row, per_row, 4);
        const BlocksParams p = {X, codes, scales, ldx, ldc, (int)rows, (int)cols, block, pow2, vx, vc, ranges};
        const dim3 b = flat_block((int)cols);
        const unsigned grid = flat_grid((int)rows, b);
        if (type == FMM_TYPE_F32) quantize_blocks_kernel<float><<<grid, b, 0, st>>>(p);
        else if (type == FMM_TYPE_BF16) quantize_blocks_kernel<__nv_bfloat16><<<grid, b, 0, st>>>(p);
        else quantize_blocks_kernel<__half><<<grid, b, 0, st>>>(p);
        return launched();
    }
    int8_add_range(ranges, scales, 1, rows, rows, 4);
    RowsParams p = {};
    p.x = X; p.ldx = ldx; p.codes = codes; p.ldc = ldc; p.scales = scales;
    p.rows = (int)rows; p.cols = (int)cols; p.pow2 = pow2; p.vx = vx; p.vc = vc; p.ranges = ranges;
    if (type == FMM_TYPE_F32) return launch_rows<float, false>(p, st);
    if (type == FMM_TYPE_BF16) return launch_rows<__nv_bfloat16, false>(p, st);
    return launch_rows<__half, false>(p, st);
}

fmm_status_t fmm_int8_dequantize(const int8_t* codes, int64_t ldc, const float* scales, int64_t rows, int64_t cols, int block,
                                 void* X, fmm_type_t type, int64_t ldx, void* stream)
{
    if (!int8_type_ok(type) || !block_ok(block)) return FMM_ERR_INVALID_ARG;
    if (!dims_ok(rows, cols)) return FMM_ERR_SHAPE;
    if (rows == 0 || cols == 0) return FMM_OK;
    const int e = int8_type_bytes(type);
    if (!matrix_ok(codes, cols, ldc, 1) || !matrix_ok(scales, 1, 1, 4) || !matrix_ok(X, cols, ldx, e)) return FMM_ERR_INVALID_ARG;
    Int8Ranges ranges = {};
    int8_add_range(ranges, X, rows, cols, ldx, e);
    const RestoreParams p = {codes, scales, X, ldc, ldx, (int)rows, (int)cols, block, int8_aligned(codes, ldc, 8), int8_aligned(X, ldx * e, 16), ranges};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const dim3 b = flat_block((int)cols);
    const unsigned grid = flat_grid((int)rows, b);
    if (type == FMM_TYPE_F32) dequantize_kernel<float><<<grid, b, 0, st>>>(p);
    else if (type == FMM_TYPE_BF16) dequantize_kernel<__nv_bfloat16><<<grid, b, 0, st>>>(p);
    else dequantize_kernel<__half><<<grid, b, 0, st>>>(p);
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
    p.vx = int8_aligned(a->x, a->ldx * e, 16); p.vr = int8_aligned(a->residual, a->ldr * e, 16); p.vg = int8_aligned(a->gain, 0, 16);
    p.vh = int8_aligned(a->hidden, a->ldh * e, 16); p.vc = int8_aligned(a->codes, a->ldc, 8); p.vk = int8_aligned(a->checkpoint, a->ldk, 8);
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
    *bytes = (size_t)back_shape(rows, cols).parts * (size_t)cols * 4;
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
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < (size_t)shape.parts * (size_t)cols * 4) return FMM_ERR_WORKSPACE;
    BackParams p = {};
    p.dy = a->dy; p.checkpoint = a->checkpoint; p.scales = a->checkpoint_scales; p.rstd = a->rstd; p.gain = a->gain; p.dresidual = a->dresidual;
    p.dx = a->dx; p.dgain = a->dgain; p.partial = static_cast<float*>(workspace);
    p.ldy = a->ldy; p.ldk = a->ldk; p.ldr = a->ldr; p.ldx = a->ldx;
    p.rows = (int)rows; p.cols = (int)cols; p.block = a->block; p.parts = shape.parts;
    p.vy = int8_aligned(a->dy, a->ldy * e, 16); p.vk = int8_aligned(a->checkpoint, a->ldk, 8); p.vg = int8_aligned(a->gain, 0, 16);
    p.vr = int8_aligned(a->dresidual, a->ldr * e, 16); p.vx = int8_aligned(a->dx, a->ldx * e, 16);
    int8_add_range(p.ranges, a->dx, rows, cols, a->ldx, e);
    int8_add_range(p.ranges, a->dgain, 1, cols, cols, 4);
    int8_add_range(p.ranges, workspace, shape.parts, cols, cols, 4);
    if (a->type == FMM_TYPE_F32) return launch_back<float>(p, shape.threads, st);
    if (a->type == FMM_TYPE_BF16) return launch_back<__nv_bfloat16>(p, shape.threads, st);
    return launch_back<__half>(p, shape.threads, st);
}

}  // extern "C"
