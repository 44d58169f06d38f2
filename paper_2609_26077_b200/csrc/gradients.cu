// Global norm of many tensors, and clipping to a largest one.
//
// Bound by HBM: the norm reads every number once, clipping reads it again and writes it.  Tensors are cut into chunks, which the blocks of one
// launch take in turn whatever tensor they belong to, so that many small tensors cost no more than a large one; the list of tensors is an
// argument of the kernel, so that nothing has to be copied to the device first.  Squares and their sums are taken in fp64, where those of all three
// types are exact or rounded to 53 bits and no range ends (268 M bf16 numbers 94 us; the squares of 16 bytes added in fp32 first: 88, and up to a unit more in the
// norm's last place).  Every block leaves its sum in a place of its own; every block of
// the second launch adds them up, in the same order.  268 M fp32 numbers in 24 tensors: norm 161 us (6.7 TB/s), clipping 547 to 553 (5.8); 2 M bf16 numbers in 200
// tensors 10 us, of which two launches are most.
#include <cmath>
#include <algorithm>
#include <memory>
#include <new>
#include "../../include/fmm_gradients.h"
#include "int8_internal.h"

namespace {

struct Entry { const void* x; void* out; long long size; uint32_t first; uint32_t type; };       // first: chunks before it
template <int CAP> struct List {
    int count; uint32_t chunks; int chunk;          // chunk: numbers
    double* sums;                                   // one for each block of the first kernel
    int first_sum, all_sums;                        // of this launch, of all launches of the call
    double max_norm; float* norm;
    Entry e[CAP];
};

constexpr int THREADS = 256, AT_ONCE = 4;

// sum over the block, in thread 0
__device__ __forceinline__ double block_sum(double s, double* meet)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if ((threadIdx.x & 31) == 0) meet[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0;
    if (threadIdx.x == 0)
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) s += meet[w];
    return s;
}

template <typename T> struct Vec { static constexpr int N = 16 / sizeof(T); };
template <typename T> __device__ __forceinline__ void add_squares(double& s, uint4 u)
{
    const T* t = reinterpret_cast<const T*>(&u);
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) { const double f = to_float(t[i]); s = fma(f, f, s); }
}
// numbers before the first boundary of A bytes
template <int A, typename T> __device__ __forceinline__ int head_of(const T* p, int n) { return min((int)((A - ((uintptr_t)p & (A - 1))) & (A - 1)) / (int)sizeof(T), n); }

template <typename T> __device__ __forceinline__ double chunk_squares(const T* p, int n)
{
    double s = 0;
    const int head = head_of<16>(p, n), vecs = (n - head) / Vec<T>::N, tail = head + vecs * Vec<T>::N;
    const uint4* v = reinterpret_cast<const uint4*>(p + head);
    int i = threadIdx.x;
    for (; i + 3 * THREADS < vecs; i += 4 * THREADS) {
        const uint4 a = v[i], b = v[i + THREADS], c = v[i + 2 * THREADS], d = v[i + 3 * THREADS];
        add_squares<T>(s, a); add_squares<T>(s, b); add_squares<T>(s, c); add_squares<T>(s, d);
    }
    for (; i < vecs; i += THREADS) add_squares<T>(s, v[i]);
    if ((int)threadIdx.x < head) { const double f = to_float(p[threadIdx.x]); s = fma(f, f, s); }
    if (tail + (int)threadIdx.x < n) { const double f = to_float(p[tail + threadIdx.x]); s = fma(f, f, s); }
    return s;
}
// What numbers are scaled by: power, 2^-64 where the whole would not be a normal fp32 number (gradients beyond 1e19), else 1, times rest.
struct Factor {
    float power, rest;
    __device__ __forceinline__ float operator()(float x) const { return x * power * rest; }
};
template <typename T> __device__ __forceinline__ uint4 scale16(uint4 u, Factor f)
{
    T* t = reinterpret_cast<T*>(&u);
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) t[i] = from_float<T>(f(to_float(t[i])));
    return u;
}
template <typename T> __device__ __forceinline__ void chunk_scale(const T* p, T* q, int n, Factor f)
{
    if (((uintptr_t)p ^ (uintptr_t)q) & 15) {
        for (int i = threadIdx.x; i < n; i += THREADS) q[i] = from_float<T>(f(to_float(p[i])));
        return;
    }
    // What the warps write fills whole lines, wherever in a buffer a tensor starts (24 tensors of 268M numbers: 567 -> 555 us)
    const int head = head_of<128>(q, n), vecs = (n - head) / Vec<T>::N, tail = head + vecs * Vec<T>::N;
    const uint4* v = reinterpret_cast<const uint4*>(p + head);
    uint4* w = reinterpret_cast<uint4*>(q + head);
    int i = threadIdx.x;
    for (; i + (AT_ONCE - 1) * THREADS < vecs; i += AT_ONCE * THREADS) {
        uint4 u[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) u[j] = v[i + j * THREADS];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) w[i + j * THREADS] = scale16<T>(u[j], f);
    }
    for (; i < vecs; i += THREADS) w[i] = scale16<T>(v[i], f);
    if ((int)threadIdx.x < head) q[threadIdx.x] = from_float<T>(f(to_float(p[threadIdx.x])));
    if (tail + (int)threadIdx.x < n) q[tail + threadIdx.x] = from_float<T>(f(to_float(p[tail + threadIdx.x])));
}
// the entry that a chunk belongs to
template <int CAP> __device__ __forceinline__ int find_entry(const List<CAP>& l, uint32_t c)
{
    int lo = 0, hi = l.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (l.e[mid].first <= c) lo = mid; else hi = mid - 1;
    }
    return lo;
}

template <int CAP> __global__ void __launch_bounds__(THREADS, 4) gradient_squares_kernel(const __grid_constant__ List<CAP> l)
{
    __shared__ double meet[THREADS / 32];
    double s = 0;
    for (uint32_t c = blockIdx.x; c < l.chunks; c += gridDim.x) {
        const Entry& e = l.e[find_entry(l, c)];
        const long long at = (long long)(c - e.first) * l.chunk;
        const int n = (int)min((long long)l.chunk, e.size - at);
        if (e.type == FMM_TYPE_F32) s += chunk_squares(static_cast<const float*>(e.x) + at, n);
        else if (e.type == FMM_TYPE_BF16) s += chunk_squares(static_cast<const __nv_bfloat16*>(e.x) + at, n);
        else s += chunk_squares(static_cast<const __half*>(e.x) + at, n);
    }
    s = block_sum(s, meet);
    if (threadIdx.x == 0) l.sums[l.first_sum + blockIdx.x] = s;
}
__device__ __forceinline__ double sum_all(const double* sums, int n, double* meet)
{
    double s = 0;
    for (int i = threadIdx.x; i < n; i += THREADS) s += sums[i];
    return block_sum(s, meet);
}
__global__ void __launch_bounds__(THREADS) gradient_norm_kernel(const double* sums, int n, float* norm)
{
    __shared__ double meet[THREADS / 32];
    const double s = sum_all(sums, n, meet);
    if (threadIdx.x == 0) *norm = (float)sqrt(s);
}
template <int CAP> __global__ void __launch_bounds__(THREADS, 4) gradient_scale_kernel(const __grid_constant__ List<CAP> l)
{
    __shared__ double meet[THREADS / 32];
    __shared__ Factor shared_factor;
    const double s = sum_all(l.sums, l.all_sums, meet);
    if (threadIdx.x == 0) {
        const double norm = sqrt(s);
        const double f = norm <= l.max_norm ? 1.0 : l.max_norm / norm;        // (a NaN norm: NaN)
        shared_factor = f < 0x1p-64 ? Factor{0x1p-64f, (float)(f * 0x1p64)} : Factor{1.0f, (float)f};
        if (blockIdx.x == 0 && l.first_sum == 0) *l.norm = (float)norm;
    }
    __syncthreads();
    const Factor f = shared_factor;
    // backwards: what the sums read last is in L2
    for (uint32_t b = blockIdx.x; b < l.chunks; b += gridDim.x) {
        const uint32_t c = l.chunks - 1 - b;
        const Entry& e = l.e[find_entry(l, c)];
        if (f.power == 1.0f && f.rest == 1.0f && e.out == e.x) continue;      // (a factor just below 2^-64 has 2^-64 and 1)
        const long long at = (long long)(c - e.first) * l.chunk;
        const int n = (int)min((long long)l.chunk, e.size - at);
        if (e.type == FMM_TYPE_F32) chunk_scale(static_cast<const float*>(e.x) + at, static_cast<float*>(e.out) + at, n, f);
        else if (e.type == FMM_TYPE_BF16) chunk_scale(static_cast<const __nv_bfloat16*>(e.x) + at, static_cast<__nv_bfloat16*>(e.out) + at, n, f);
        else chunk_scale(static_cast<const __half*>(e.x) + at, static_cast<__half*>(e.out) + at, n, f);
    }
}

// ------------------------------------------------------------------------------------------------ host side
// Tensors that a launch's arguments have room for (32 bytes each, of the 32 KB that a launch can have).  A launch copies all of it, whatever is in use, so
// there is a size for each doubling: with 241 tensors a pass takes 18 us in arguments for 256 and 21 in those for 800, with 400 25 and 27.
constexpr int LEAST = 32, MOST = 1000;
constexpr int MOST_BLOCKS = 2048;
constexpr int64_t MOST_NUMBERS = (int64_t)1 << 42;        // of a tensor

int launches_of(int64_t count) { return (int)((count + MOST - 1) / MOST); }
int blocks_of(uint32_t chunks) { return (int)std::min<int64_t>(chunks, std::min(MOST_BLOCKS, int8_sm_count() * 4)); }

bool list_ok(const fmm_gradients_t* g)
{
    if (g->count && (!g->x || !g->sizes || !g->types)) return false;
    for (int64_t i = 0; i < g->count; ++i) {
        if (!int8_type_ok((fmm_type_t)g->types[i]) || g->sizes[i] < 0 || g->sizes[i] > MOST_NUMBERS) return false;
        const uintptr_t a = (uintptr_t)int8_type_bytes((fmm_type_t)g->types[i]) - 1;
        if (g->sizes[i] && (!g->x[i] || ((uintptr_t)g->x[i] & a) || (g->out && (!g->out[i] || ((uintptr_t)g->out[i] & a))))) return false;
    }
    return true;
}
struct Interval { uintptr_t lo, hi; bool out; };
// Whether no tensor is written that another one's output or input shares memory with
bool apart(const fmm_gradients_t* g)
{
    const std::unique_ptr<Interval[]> v(new (std::nothrow) Interval[2 * g->count + 1]);
    if (!v) return false;
    int64_t n = 0;
    bool sorted = true;
    auto add = [&](const void* p, int64_t bytes, bool out) {
        const uintptr_t lo = (uintptr_t)p;
        if (n && lo < v[n - 1].lo) sorted = false;
        v[n++] = {lo, lo + bytes, out};
    };
    for (int64_t i = 0; i < g->count; ++i) if (g->sizes[i]) add(g->out ? g->out[i] : g->x[i], g->sizes[i] * int8_type_bytes((fmm_type_t)g->types[i]), true);
    if (g->out) for (int64_t i = 0; i < g->count; ++i)
        if (g->sizes[i] && g->out[i] != g->x[i]) add(g->x[i], g->sizes[i] * int8_type_bytes((fmm_type_t)g->types[i]), false);
    if (!sorted) std::sort(v.get(), v.get() + n, [](const Interval& a, const Interval& b) { return a.lo < b.lo; });
    uintptr_t any = 0, written = 0;
    for (int64_t k = 0; k < n; ++k) {
        const Interval& i = v[k];
        if (i.lo < (i.out ? any : written)) return false;
        any = std::max(any, i.hi);
        if (i.out) written = std::max(written, i.hi);
    }
    return true;
}

template <int CAP> fmm_status_t run(const fmm_gradients_t* g, bool scale, double max_norm, float* norm, double* sums, cudaStream_t st)
{
    int64_t total = 0;
    for (int64_t i = 0; i < g->count; ++i) total += g->sizes[i];
    // four chunks to a block, where these are 2048 to 32768 numbers
    int chunk = 2048;
    while (chunk < 32768 && total > (int64_t)chunk * int8_sm_count() * 16) chunk *= 2;
    List<CAP> l;
    l.sums = sums; l.max_norm = max_norm; l.norm = norm; l.chunk = chunk;
    int all = 0;
    for (int pass = 0; pass < (scale ? 2 : 1); ++pass) {
        l.all_sums = all;
        l.first_sum = 0;
        int64_t i = 0;
        do {
            l.count = 0;
            uint64_t chunks = 0;
            for (; i < g->count && l.count < CAP; ++i) {
                if (!g->sizes[i]) continue;
                const uint64_t c = ((uint64_t)g->sizes[i] + chunk - 1) / chunk;
                if (chunks + c > 0xffffffffull) return FMM_ERR_SHAPE;
                l.e[l.count++] = {g->x[i], g->out ? g->out[i] : const_cast<void*>(g->x[i]), g->sizes[i], (uint32_t)chunks, g->types[i]};
                chunks += c;
            }
            l.chunks = (uint32_t)chunks;
            const int blocks = std::max(1, blocks_of(l.chunks));
            if (pass == 0) gradient_squares_kernel<CAP><<<blocks, THREADS, 0, st>>>(l);
            else gradient_scale_kernel<CAP><<<blocks, THREADS, 0, st>>>(l);
            l.first_sum += blocks;
        } while (i < g->count);
        all = l.first_sum;
    }
    if (!scale) gradient_norm_kernel<<<1, THREADS, 0, st>>>(sums, all, norm);
    return cudaGetLastError() == cudaSuccess ? FMM_OK : FMM_ERR_CUDA;
}
template <int CAP> fmm_status_t run_sized(const fmm_gradients_t* g, bool scale, double max_norm, float* norm, double* sums, cudaStream_t st)
{
    if constexpr (CAP < MOST) { if (g->count > CAP) return run_sized<(2 * CAP < MOST ? 2 * CAP : MOST)>(g, scale, max_norm, norm, sums, st); }
    return run<CAP>(g, scale, max_norm, norm, sums, st);
}
fmm_status_t gradients(const fmm_gradients_t* g, bool scale, double max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!g || !norm || ((uintptr_t)norm & 3) || g->count < 0 || !(max_norm >= 0) || std::isinf(max_norm)) return FMM_ERR_INVALID_ARG;
    size_t need = 0;
    const fmm_status_t s = fmm_gradient_workspace_bytes(g->count, &need);
    if (s != FMM_OK) return s;
    if (!list_ok(g) || (scale && !apart(g))) return FMM_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need) return FMM_ERR_WORKSPACE;
    double* sums = static_cast<double*>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return run_sized<LEAST>(g, scale, max_norm, norm, sums, st);
}

}  // namespace

extern "C" {

fmm_status_t fmm_gradient_workspace_bytes(int64_t count, size_t* bytes)
{
    if (!bytes) return FMM_ERR_INVALID_ARG;
    if (count < 0 || count > (1 << 20)) return FMM_ERR_SHAPE;
    *bytes = (size_t)std::max(1, launches_of(count)) * MOST_BLOCKS * sizeof(double);
    return FMM_OK;
}
fmm_status_t fmm_gradient_norm(const fmm_gradients_t* g, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    return gradients(g, false, 0.0, norm, workspace, workspace_bytes, stream);
}
fmm_status_t fmm_gradient_clip(const fmm_gradients_t* g, double max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    return gradients(g, true, max_norm, norm, workspace, workspace_bytes, stream);
}

}  // extern "C"
