// Internal declarations of the 8-bit integer layer (not part of the C ABI).
#pragma once
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>
#include "../../include/fmm_int8.h"
#include "fmm_internal.h"

// Store ranges of a launch, checked in the FMM_DEBUG build only (as FmmGuard, for launches with more than two outputs).
struct Int8Ranges {
#ifdef FMM_DEBUG
    const char* lo[6];
    const char* hi[6];
    int count;
#endif
};
static inline void int8_add_range(Int8Ranges& r, const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t element)
{
#ifdef FMM_DEBUG
    if (!p || rows <= 0 || cols <= 0) return;
    r.lo[r.count] = static_cast<const char*>(p);
    r.hi[r.count++] = static_cast<const char*>(p) + ((rows - 1) * ld + cols) * element;
#else
    (void)r; (void)p; (void)rows; (void)cols; (void)ld; (void)element;
#endif
}
#if defined(FMM_DEBUG) && defined(__CUDACC__)
__device__ __forceinline__ bool int8_store_ok(const Int8Ranges& r, const void* ptr, size_t bytes, int code, int* word)
{
    const char* c = static_cast<const char*>(ptr);
    for (int i = 0; i < r.count; ++i) if (c >= r.lo[i] && c + bytes <= r.hi[i]) return true;
    atomicCAS(word, 0, code);
    return false;
}
#define INT8_STORE_OK(r, ptr, bytes, code, word) int8_store_ok(r, ptr, bytes, code, word)
#else
#define INT8_STORE_OK(r, ptr, bytes, code, word) true
#endif

static inline int int8_type_bytes(fmm_type_t t) { return t == FMM_TYPE_F32 ? 4 : 2; }
static inline bool int8_type_ok(fmm_type_t t) { return t == FMM_TYPE_F32 || t == FMM_TYPE_BF16 || t == FMM_TYPE_F16; }
static inline bool int8_aligned(const void* p, int64_t ld_bytes, unsigned a) { return (((uintptr_t)p | (uintptr_t)ld_bytes) & (a - 1)) == 0; }
// Rows and columns that 32-bit indexes hold with room for a step of any kernel behind them
constexpr int64_t INT8_MAX_DIM = ((int64_t)1 << 31) - 16384;

// SMs of the current device, asked for once per device: the runtime takes 0.7 us for the two calls, a third of a launch
static inline int int8_sm_count()
{
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 1; }
    if (dev >= 64) return fmm_sm_count();
    int n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) { n = fmm_sm_count(); known[dev].store(n, std::memory_order_relaxed); }
    return n;
}

#ifdef __CUDACC__
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <typename T> __device__ __forceinline__ uint32_t pack_two(float a, float b);
template <> __device__ __forceinline__ uint32_t pack_two<__nv_bfloat16>(float a, float b)
{ __nv_bfloat162 v = __floats2bfloat162_rn(a, b); return *reinterpret_cast<uint32_t*>(&v); }
template <> __device__ __forceinline__ uint32_t pack_two<__half>(float a, float b)
{ __half2 v = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t*>(&v); }

// fp16 parts: a power of two for the whole matrix, by which its largest finite scale comes to lie in [128, 256), so that no value leaves
// the range and those 2^-21 of the largest are still normal numbers.  Exponent, from the maxima that int8_values left (warp-collective).
__device__ __forceinline__ int maximum_exponent(uint32_t m) { return m == 0 ? 0 : min(7 - ((int)(m >> 23) - 127), 100); }
__device__ __forceinline__ int matrix_exponent(const uint32_t* maxima, int count)
{
    const int lane = threadIdx.x & 31;
    return maximum_exponent(__reduce_max_sync(0xffffffffu, max(lane < count ? maxima[lane] : 0u, lane + 32 < count ? maxima[lane + 32] : 0u)));
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }      // -126 .. 127
#endif

// int8_rows.cu: the status word of its store checks (FMM_DEBUG build; 0 otherwise)
fmm_status_t int8_rows_guard_read(int* code, bool clear);
// What the product of a gradient reads, in the workspace.  Rows there are ld elements apart, a multiple of 8, on 16-byte boundaries.
//   values: code * scale in fp32, in `parts` matrices of `type`, step elements apart, each holding what the ones before it leave.  By stages of
//   INT8_PART_ROWS rows: where every scale of a stage is a power of two, its first part is the value, the others are not written, and its
//   byte of `flags` is 0, else 1.  flags null: one part.  maxima: null, or room for INT8_MAXIMA maxima of scales, for fp16.
constexpr int INT8_PART_ROWS = 64, INT8_MAXIMA = 64;
int int8_scale_maxima_count(int64_t rows);
fmm_status_t int8_values(fmm_type_t type, int parts, const int8_t* codes, int64_t ldc, const float* scales, uint32_t* maxima, uint8_t* flags, void* x, int64_t ldx,
                         int64_t step, int64_t rows, int64_t cols, cudaStream_t st);
//   the codes (code_rows x code_cols) themselves in fp16, and rows scaled by code_rows scales: y[i][j] = x[i][j] (bf16) * scales[j] in fp16,
//   times a power of two for each row by which its largest finite number comes to lie in [2^14, 2^15); inverse[i]: one over that.
fmm_status_t int8_codes_and_scaled_rows(const int8_t* codes, int64_t ldc, void* values, int64_t ldv, int64_t code_rows, int64_t code_cols, const void* x, int64_t ldx,
                                        const float* scales, void* y, int64_t ldy, float* inverse, int64_t rows, cudaStream_t st);
// 16-bit rows copied to rows on 16-byte boundaries, ldy a multiple of 8
fmm_status_t int8_realign(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, cudaStream_t st);
