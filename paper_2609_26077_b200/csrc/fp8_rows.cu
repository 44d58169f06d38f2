// Quantization to e4m3 with an fp32 scale for each block of 128: along the rows, along the columns, both, or in tiles.
//
// Bound by HBM: a number is read once (2 or 4 bytes) and written as one byte for each form.  A thread block takes 128 x 128 numbers, which
// hold whole blocks of all three forms, so that both forms come from one pass; a thread holds 8 neighbouring columns of every
// second row of its warp, in its input's own type, from the load to the store.  16384 x 8192 bf16: along the rows 68 to 71 us (5.7 to 5.9 TB/s of
// 6.45), both forms 102 (5.3); 8191 columns, whose rows are not on 16-byte boundaries, 110 and 147.
#include <type_traits>
#include "fp8_internal.h"
#include "fmm_ptx.cuh"

namespace {
using namespace fmmptx;

__device__ int g_fp8_rows_status;

struct QuantizeParams {
    int rows, cols, column_blocks;          // column_blocks: blocks of 128 columns
    int groups; const int* offsets;
    int pow2;
    const void* x; long long ldx, step_x;   // step: from one matrix to the next (tiles)
    uint8_t* codes; long long ldc, step_c;
    float* scales; long long lds;
    uint8_t* column_codes; long long ldcc;
    float* column_scales; long long ldcs;
    Int8Ranges ranges;
};

enum Form { ROWS = 1, COLUMNS = 2, TILES = 4 };

// scale and the factor of the codes from the bits of max |x|
struct Scale { float scale, inverse; };
__device__ __forceinline__ Scale make_scale(uint32_t amax, int pow2)
{
    if (amax >= 0x7f800000u) { const float nan = __uint_as_float(0x7fffffffu); return {nan, nan}; }
    const float a = fmaxf(__uint_as_float(amax), 1e-12f);
    float scale = __fdiv_rn(a, 448.0f);
    if (!pow2) return {scale, __fdiv_rn(448.0f, a)};
    const uint32_t bits = __float_as_uint(scale), e = (bits >> 23) + ((bits & 0x7fffffu) ? 1u : 0u);
    return {__uint_as_float(e << 23), __uint_as_float((254u - e) << 23)};
}
// eight codes of eight numbers, each of a pair of columns times its own factors
__device__ __forceinline__ uint2 encode8(const float (&v)[8], const float (&f)[8])
{
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        unpack2(mul2(pack2(v[2 * i], v[2 * i + 1]), pack2(f[2 * i], f[2 * i + 1])), a, b);
        uint16_t r;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
        c[i] = r;
    }
    return make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
}

// eight neighbouring numbers as they lie in memory
template <typename T> struct Eight { uint32_t w[2 * sizeof(T)]; };
template <typename T> __device__ __forceinline__ void to_floats(const Eight<T>& e, float (&f)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(e.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) { f[2 * i] = __uint_as_float(e.w[i] << 16); f[2 * i + 1] = __uint_as_float(e.w[i] & 0xffff0000u); }
            else { const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&e.w[i])); f[2 * i] = g.x; f[2 * i + 1] = g.y; }
        }
    }
}
// Magnitudes as integers, two 16-bit numbers to a word: they are in the same order, and infinities and NaN come last.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b)
{ uint32_t r; asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
template <typename T> __device__ __forceinline__ uint32_t magnitude(uint32_t w) { return w & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu); }
template <typename T> __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) { return sizeof(T) == 4 ? max(a, b) : max_u16x2(a, b); }
// the larger of a word's two
template <typename T> __device__ __forceinline__ uint32_t one_of(uint32_t m) { return sizeof(T) == 4 ? m : max(m >> 16, m & 0xffffu); }
// a magnitude as the bits of a single
template <typename T> __device__ __forceinline__ uint32_t single(uint32_t m)
{
    if constexpr (sizeof(T) == 4) return m;
    else if constexpr (std::is_same<T, __nv_bfloat16>::value) return m << 16;
    else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
}

// A thread's eight numbers of a row, of which `valid` exist (the others are 0), or none if there is no such `row`.  Lanes 0 .. 15 and 16 .. 31 hold a row each, lane after lane.
// Rows that start on a 16-byte boundary come by vectors.  Others do too, by the aligned ones that hold a number of the row: each lane takes its own,
// gets the neighbour's, and shifts.
template <typename T, bool VEC> __device__ __forceinline__ Eight<T> load8(const T* p, int valid, bool row)
{
    constexpr int WORDS = 2 * sizeof(T), VECS = WORDS / 4, E = sizeof(T);
    Eight<T> e = {};
    if (VEC) {
        if (!row) return e;
        if (valid >= 8) {
#pragma unroll
            for (int i = 0; i < VECS; ++i) {
                const uint4 u = reinterpret_cast<const uint4*>(p)[i];
                e.w[4 * i] = u.x; e.w[4 * i + 1] = u.y; e.w[4 * i + 2] = u.z; e.w[4 * i + 3] = u.w;
            }
            return e;
        }
        T* t = reinterpret_cast<T*>(&e);
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < valid) t[i] = p[i];
        return e;
    }
    const uintptr_t from = reinterpret_cast<uintptr_t>(p), end = from + (intptr_t)valid * E;      // of the row, also where it ends before this lane's first
    const uint4* v = reinterpret_cast<const uint4*>(from & ~(uintptr_t)15);
    const int shift = (int)(from & 15);
    uint32_t w[WORDS + 4] = {};
#pragma unroll
    for (int i = 0; i < VECS; ++i)
        if (row && reinterpret_cast<uintptr_t>(v + i) < end) {
            const uint4 u = v[i];
            w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[WORDS + i] = __shfl_down_sync(0xffffffffu, w[i], 1, 16);
    if ((threadIdx.x & 15) == 15 && row && reinterpret_cast<uintptr_t>(v + VECS) < end) {
        const uint4 u = v[VECS];
        w[WORDS] = u.x; w[WORDS + 1] = u.y; w[WORDS + 2] = u.z; w[WORDS + 3] = u.w;
    }
#pragma unroll
    for (int i = 0; i < WORDS + 2; ++i) if (shift & 8) w[i] = w[i + 2];
#pragma unroll
    for (int i = 0; i < WORDS + 1; ++i) if (shift & 4) w[i] = w[i + 1];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        const uint32_t u = E == 4 ? w[i] : __funnelshift_r(w[i], w[i + 1], (shift & 2) * 8);
        const int there = row ? valid - i * 4 / E : 0;                 // of this word's numbers
        e.w[i] = there >= 4 / E ? u : E == 2 && there == 1 ? u & 0xffffu : 0u;
    }
    return e;
}
__device__ __forceinline__ void store8(uint8_t* p, uint2 c, int valid, const Int8Ranges& r, int where)
{
    if (!INT8_STORE_OK(r, p, min(valid, 8), where, &g_fp8_rows_status)) return;
    if (valid >= 8) *reinterpret_cast<uint2*>(p) = c;
    else for (int i = 0; i < valid; ++i) p[i] = (uint8_t)((i < 4 ? c.x : c.y) >> 8 * (i & 3));
}
__device__ __forceinline__ void store_scale(float* p, float s, const Int8Ranges& r, int where)
{
    if (INT8_STORE_OK(r, p, 4, where, &g_fp8_rows_status)) *p = s;
}

// Warp w takes rows 16 w .. 16 w + 15, two at a time.  The maxima of its 16 rows are reduced together, 8 numbers of each of 16 lanes by 8
// exchanges that leave each row's to two lanes, so that a lane divides for one row only; with every lane dividing for every row the kernel took three
// times as long.
template <typename T, int FORM, bool VEC>
__global__ void __launch_bounds__(256, sizeof(T) == 4 && !VEC && FORM == (ROWS | COLUMNS) ? 1 : sizeof(T) == 4 || (!VEC && FORM != ROWS) ? 2 : 3) fp8_quantize_kernel(const __grid_constant__ QuantizeParams p)
{
    constexpr int WORDS = 2 * sizeof(T);
    __shared__ __align__(16) uint32_t meet[8][128];
    __shared__ __align__(16) float factors[128];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int cb = blockIdx.x % p.column_blocks, rb = blockIdx.x / p.column_blocks;
    int first = rb * 128, count = min(128, p.rows - first);
    if (p.groups) {
        const Fp8Group g = fp8_find_group<true>(p.offsets, p.groups, p.rows, 128, rb);
        if (g.group < 0) return;
        first = g.first + (rb - g.before) * 128;
        count = min(128, g.first + g.rows - first);
    }
    const int col = cb * 128 + (tid & 15) * 8, valid = p.cols - col, r0 = warp * 16 + (lane >> 4);
    const T* x = static_cast<const T*>(p.x) + (FORM == TILES ? blockIdx.y * p.step_x : 0);
    if (FORM == ROWS && warp * 16 >= count) return;
    Eight<T> v[8];
    x += (long long)(first + r0) * p.ldx + col;
#pragma unroll
    for (int i = 0; i < 8; ++i, x += 2 * p.ldx) {
        const int r = r0 + 2 * i;
        v[i] = load8<T, VEC>(x, valid, r < count);
    }
    uint32_t cmax[WORDS] = {}, rmax[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < WORDS; ++j) {
            const uint32_t a = magnitude<T>(v[i].w[j]);
            m = most<T>(m, a);
            if (FORM & COLUMNS) cmax[j] = most<T>(cmax[j], a);
        }
        rmax[i] = one_of<T>(m);
    }
    if (FORM & ROWS) {
#pragma unroll
        for (int n = 4, d = 8; n; n >>= 1, d >>= 1) {
            const bool upper = lane & d;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const uint32_t other = __shfl_xor_sync(0xffffffffu, upper ? rmax[i] : rmax[i + n], d);
                rmax[i] = max(upper ? rmax[i + n] : rmax[i], other);
            }
        }
        const uint32_t m = max(rmax[0], __shfl_xor_sync(0xffffffffu, rmax[0], 1));
        const Scale s = make_scale(single<T>(m), p.pow2);
        const int mine = r0 + 2 * (((lane >> 3) & 1) * 4 + ((lane >> 2) & 1) * 2 + ((lane >> 1) & 1));
        if (!(lane & 1) && mine < count) store_scale(p.scales + (long long)cb * p.lds + first + mine, s.scale, p.ranges, 2502);
        uint8_t* q = p.codes + (long long)(first + r0) * p.ldc + col;
#pragma unroll
        for (int i = 0; i < 8; ++i, q += 2 * p.ldc) {
            const float inverse = __shfl_sync(0xffffffffu, s.inverse, (lane & 16) | (i << 1));
            const int r = r0 + 2 * i;
            if (r < count && valid > 0) {
                float f[8], k[8];
                to_floats(v[i], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) k[j] = inverse;
                store8(q, encode8(f, k), valid, p.ranges, 2501);
            }
        }
    }
    if (FORM & COLUMNS) {
#pragma unroll
        for (int j = 0; j < WORDS; ++j) cmax[j] = most<T>(cmax[j], __shfl_xor_sync(0xffffffffu, cmax[j], 16));
        if (lane < 16) {
#pragma unroll
            for (int j = 0; j < WORDS; ++j) meet[warp][lane * WORDS + j] = cmax[j];
        }
        __syncthreads();
        if (tid < 128) {
            uint32_t m = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) m = most<T>(m, meet[w][sizeof(T) == 4 ? tid : tid / 2]);
            if (sizeof(T) == 2) m = tid & 1 ? m >> 16 : m & 0xffffu;
            const Scale s = make_scale(single<T>(m), p.pow2);
            factors[tid] = s.inverse;
            if (cb * 128 + tid < p.cols) store_scale(p.column_scales + (long long)rb * p.ldcs + cb * 128 + tid, s.scale, p.ranges, 2503);
        }
        __syncthreads();
        const float4 ka = *reinterpret_cast<const float4*>(factors + (tid & 15) * 8), kb = *reinterpret_cast<const float4*>(factors + (tid & 15) * 8 + 4);
        const float k[8] = {ka.x, ka.y, ka.z, ka.w, kb.x, kb.y, kb.z, kb.w};
        if (valid > 0) {
            uint8_t* q = p.column_codes + ((long long)rb * 128 + r0) * p.ldcc + col;
#pragma unroll
            for (int i = 0; i < 8; ++i, q += 2 * p.ldcc) {
                float f[8];
                to_floats(v[i], f);
                const int r = r0 + 2 * i;
                store8(q, r < count ? encode8(f, k) : make_uint2(0, 0), valid, p.ranges, 2504);
            }
        }
    }
    if (FORM == TILES) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, rmax[i]);
        m = __reduce_max_sync(0xffffffffu, m);
        if (lane == 0) meet[0][warp] = m;
        __syncthreads();
        m = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) m = max(m, meet[0][w]);
        const Scale s = make_scale(single<T>(m), p.pow2);
        if (tid == 0) store_scale(p.scales + (long long)blockIdx.y * p.lds + blockIdx.x, s.scale, p.ranges, 2505);
        float k[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) k[j] = s.inverse;
        uint8_t* q = p.codes + blockIdx.y * p.step_c + (long long)(first + r0) * p.ldc + col;
#pragma unroll
        for (int i = 0; i < 8; ++i, q += 2 * p.ldc) {
            float f[8];
            to_floats(v[i], f);
            const int r = r0 + 2 * i;
            if (r < count && valid > 0) store8(q, encode8(f, k), valid, p.ranges, 2506);
        }
    }
}

template <int FORM, bool VEC> fmm_status_t launch_type(const QuantizeParams& p, fmm_type_t type, dim3 grid, cudaStream_t st)
{
    if (type == FMM_TYPE_F32) fp8_quantize_kernel<float, FORM, VEC><<<grid, 256, 0, st>>>(p);
    else if (type == FMM_TYPE_BF16) fp8_quantize_kernel<__nv_bfloat16, FORM, VEC><<<grid, 256, 0, st>>>(p);
    else fp8_quantize_kernel<__half, FORM, VEC><<<grid, 256, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? FMM_OK : FMM_ERR_CUDA;
}
template <int FORM> fmm_status_t launch(const QuantizeParams& p, fmm_type_t type, dim3 grid, cudaStream_t st)
{
    const int64_t e = int8_type_bytes(type);
    const bool vec = int8_aligned(p.x, p.ldx * e, 16) && ((p.step_x * e) & 15) == 0;
    return vec ? launch_type<FORM, true>(p, type, grid, st) : launch_type<FORM, false>(p, type, grid, st);
}
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool dim_ok(int64_t n) { return n >= 0 && n < INT8_MAX_DIM; }

}  // namespace

fmm_status_t fp8_rows_guard_read(int* code, bool clear)
{
    const int zero = 0;
    *code = 0;
    if (cudaMemcpyFromSymbol(code, g_fp8_rows_status, sizeof(int)) != cudaSuccess ||
        (clear && cudaMemcpyToSymbol(g_fp8_rows_status, &zero, sizeof(int)) != cudaSuccess)) {
        cudaGetLastError();
        return FMM_ERR_CUDA;
    }
    return FMM_OK;
}

extern "C" {

fmm_status_t fmm_fp8_column_rows(int64_t rows, int64_t groups, int64_t* column_rows)
{
    if (!column_rows) return FMM_ERR_INVALID_ARG;
    if (!dim_ok(rows) || groups < 0 || groups > FMM_FP8_MAX_GROUPS) return FMM_ERR_SHAPE;
    *column_rows = (rows + 127 * (groups > 1 ? groups : 1)) / 128 * 128;
    return FMM_OK;
}

fmm_status_t fmm_fp8_quantize(const fmm_fp8_quantize_t* a, void* stream)
{
    if (!a || !int8_type_ok(a->type) || (a->scale_mode != FMM_FP8_SCALE_AMAX_DIV_448 && a->scale_mode != FMM_FP8_SCALE_POW2)) return FMM_ERR_INVALID_ARG;
    int64_t column_rows = 0;
    const fmm_status_t s = fmm_fp8_column_rows(a->rows, a->groups, &column_rows);
    if (s != FMM_OK) return s;
    if (!dim_ok(a->cols) || !dim_ok(column_rows)) return FMM_ERR_SHAPE;
    const int64_t rows = a->rows, cols = a->cols, e = int8_type_bytes(a->type);
    if (!a->codes && !a->column_codes) return FMM_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return FMM_OK;
    if (!a->x || ((uintptr_t)a->x & (e - 1)) || a->ldx < cols || (a->groups && (!a->offsets || ((uintptr_t)a->offsets & 3)))) return FMM_ERR_INVALID_ARG;
    const unsigned step = a->loose ? 4 : 16;
    if (a->codes && (a->ldc < cols || !int8_aligned(a->codes, a->ldc, 16) || !a->scales || a->lds < rows || !int8_aligned(a->scales, a->lds * 4, step))) return FMM_ERR_INVALID_ARG;
    if (a->column_codes && (a->ldcc < cols || !int8_aligned(a->column_codes, a->ldcc, 16) || !a->column_scales || a->ldcs < cols ||
                            !int8_aligned(a->column_scales, a->ldcs * 4, step))) return FMM_ERR_INVALID_ARG;
    QuantizeParams p = {};
    p.rows = (int)rows; p.cols = (int)cols; p.column_blocks = (int)ceil_div(cols, 128);
    p.groups = (int)a->groups; p.offsets = a->offsets; p.pow2 = a->scale_mode == FMM_FP8_SCALE_POW2;
    p.x = a->x; p.ldx = a->ldx;
    p.codes = a->codes; p.ldc = a->ldc; p.scales = a->scales; p.lds = a->lds;
    p.column_codes = a->column_codes; p.ldcc = a->ldcc; p.column_scales = a->column_scales; p.ldcs = a->ldcs;
    if (a->codes) { int8_add_range(p.ranges, a->codes, rows, cols, a->ldc, 1); int8_add_range(p.ranges, a->scales, p.column_blocks, rows, a->lds, 4); }
    if (a->column_codes) {
        int8_add_range(p.ranges, a->column_codes, column_rows, cols, a->ldcc, 1);
        int8_add_range(p.ranges, a->column_scales, column_rows / 128, cols, a->ldcs, 4);
    }
    const int64_t blocks = column_rows / 128 * p.column_blocks;
    if (blocks > 0x7FFFFFFF) return FMM_ERR_SHAPE;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const dim3 grid((unsigned)blocks);
    if (a->codes && a->column_codes) return launch<ROWS | COLUMNS>(p, a->type, grid, st);
    return a->codes ? launch<ROWS>(p, a->type, grid, st) : launch<COLUMNS>(p, a->type, grid, st);
}

fmm_status_t fmm_fp8_quantize_weight(const fmm_fp8_quantize_weight_t* a, void* stream)
{
    if (!a || !int8_type_ok(a->type) || (a->scale_mode != FMM_FP8_SCALE_AMAX_DIV_448 && a->scale_mode != FMM_FP8_SCALE_POW2)) return FMM_ERR_INVALID_ARG;
    const int64_t count = a->count, rows = a->rows, cols = a->cols, e = int8_type_bytes(a->type);
    if (count < 0 || count > FMM_FP8_MAX_GROUPS || !dim_ok(rows) || !dim_ok(cols)) return FMM_ERR_SHAPE;
    if (count == 0 || rows == 0 || cols == 0) return FMM_OK;
    const int64_t blocks = ceil_div(rows, 128) * ceil_div(cols, 128);
    if (blocks > 0x7FFFFFFF) return FMM_ERR_SHAPE;
    if (!a->x || ((uintptr_t)a->x & (e - 1)) || a->ldx < cols || !a->codes || a->ldc < cols || !int8_aligned(a->codes, a->ldc, 16) || !a->scales ||
        ((uintptr_t)a->scales & 3)) return FMM_ERR_INVALID_ARG;
    if (count > 1 && (a->step_x < (rows - 1) * a->ldx + cols || a->step_c < (rows - 1) * a->ldc + cols || (a->step_c & 15))) return FMM_ERR_INVALID_ARG;
    QuantizeParams p = {};
    p.rows = (int)rows; p.cols = (int)cols; p.column_blocks = (int)ceil_div(cols, 128);
    p.pow2 = a->scale_mode == FMM_FP8_SCALE_POW2;
    p.x = a->x; p.ldx = a->ldx; p.step_x = count > 1 ? a->step_x : 0;
    p.codes = a->codes; p.ldc = a->ldc; p.step_c = count > 1 ? a->step_c : 0;
    p.scales = a->scales; p.lds = blocks;
    int8_add_range(p.ranges, a->codes, 1, (count - 1) * p.step_c + (rows - 1) * a->ldc + cols, 0, 1);
    int8_add_range(p.ranges, a->scales, count, blocks, blocks, 4);
    return launch<TILES>(p, a->type, dim3((unsigned)blocks, (unsigned)count), reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
