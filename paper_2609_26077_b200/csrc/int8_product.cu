// Products of the 8-bit integer layer on the tensor cores:
//
//   INT8    C[i][j]  = (sum_k A[i][k] B[j][k]) a_scales[i] b_scales[j] + bias[j]     codes x codes, kind::i8, exact 32-bit sums
//   GRAD_W  dW[j][k] = sum_i dY[i][j] X[i][k]                                        16-bit operands, kind::f16, fp32 sums
//   GRAD_X  dX[i][k] = sum_j dY[i][j] W[j][k]
//
// The tile's rows (TMEM lanes) run along the output's contiguous axis - output channels j of C, input channels k of the gradients - and
// its columns along the other one, so that 32 lanes store 32 neighbouring elements straight from registers, and a product of
// few tokens is a tile of few columns: the weight streams through the side with 128 rows whatever the number of tokens.  (Up to eight
// tokens take a kernel without tiles.)
//
//               rows operand ("R")                  columns operand ("S")
//   INT8        B (N x K), K-major                  A (M x K), K-major
//   GRAD_W      values of X (M x K), row-major      dY (M x N), row-major     contraction over the rows of both
//   GRAD_X      values of W (N x K), row-major      dY (M x N), K-major
//
// An operand whose contraction runs over its rows is loaded as it lies, in boxes of 64 rows x 128 bytes, and handed to the tensor
// cores as MN-major; nothing is transposed in memory.  One pipeline stage is 128 bytes of contraction on both sides (128 codes, 64
// 16-bit numbers), four MMAs.
//
// What a gradient multiplies is in the workspace in 16 bits, but not rounded to them where the output can show it:
//   - The values code * scale, fp32 numbers, are taken apart into 16-bit parts that are multiplied one after the other: three of
//     bf16 (nothing is lost) or two of fp16 (2^-21) for an fp32 output, two for a 16-bit one (bf16: 2^-15).  Where the scales of all 64
//     rows of a stage are powers of two the first part is the value, and the others are left out: such a product takes a third or half of the
//     others' MMAs (weight gradient in fp32, 8192 cubed: 781 and 2170 us).  fp16 parts carry a power of two that keeps them in range,
//     which the output takes out again.
//   - The input gradient of a bf16 dY with a 16-bit output contracts over the scales of W, so that these can go to dY instead: the product of
//     the codes, exact in fp16, and of dY * scale, which fp16 holds to 2^-11 of a number, or 2^-39 of its row's largest.  An eighth of the
//     output's own rounding, in one pass (8192 cubed: 800 us, 1514 with two parts, 759 with values rounded to bf16).
//   - A caller who wants one pass in any case gets values rounded once to dY's type (`rounded`).
//
// The tensor cores add in fp32 by cutting off what does not fit, so the sums of a gradient drift towards zero as the contraction grows: sums of
// positive terms by 2.2e-5 of their size over 8192 terms, 5.7e-5 over 16384, a 16-bit output's rounding over 2^20.  They are therefore
// taken out of the accumulator and added up in registers, rounded to nearest: every CHUNK stages (512 terms) where the output is fp32
// (positive terms: below 1.9e-6; 256 terms would cost powers of two 12 %, 1024 save 1 %), every CHUNK_SHORT (8192 terms, below 3.1e-5)
// where it has 16 bits.
//
// The 8-bit operand is taken to 16 bits in the workspace before the product: 3 bytes a code and part once, against 2 M N K operations.  Doing
// so tile by tile on the way into the tensor cores would take two more passes through shared memory per tile (codes in, 16-bit values
// out), which the product's own operand traffic already fills where the product is large.
#include <math.h>
#include <algorithm>
#include "fmm_gemm_common.cuh"
#include "int8_internal.h"

namespace {

enum Kind { INT8 = 0, GRAD_W = 1, GRAD_X = 2 };

// [0] first bounded wait that gave up, [1] set by the self-test if its wait did not, [2] store outside its range (FMM_DEBUG build)
__device__ int g_int8_product_status[3];

__device__ __forceinline__ uint4 ld_cluster128u(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* tm)
{ asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory"); }
__device__ __forceinline__ void sts32u(uint32_t addr, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }

// warp-collective, as the MMAs of fmm_ptx.cuh
template <int KIND, int NCTA>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
#define INT8_MMA(group, kind) \
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|q, 0xffffffff;\n\t" \
                 "@q tcgen05.mma.cta_group::" group ".kind::" kind " [%0], %1, %2, %3, p;\n\t}" \
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory")
    if (KIND == INT8) { if (NCTA == 1) INT8_MMA("1", "i8"); else INT8_MMA("2", "i8"); }
    else { if (NCTA == 1) INT8_MMA("1", "f16"); else INT8_MMA("2", "f16"); }
#undef INT8_MMA
}
// MN-major operand tile of 16-bit numbers, 128-byte swizzle: boxes of 64 k rows x 64 elements (8 KB), 8-row groups 1024 bytes apart
constexpr int MN_BOX = 64 * 128;
__device__ __forceinline__ uint64_t make_mnmajor_sw128_desc(uint32_t saddr)
{
    return (uint64_t)((saddr & 0x3FFFF) >> 4) | ((uint64_t)(MN_BOX >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
template <bool MN> __device__ __forceinline__ uint64_t make_desc(uint32_t saddr) { return MN ? make_mnmajor_sw128_desc(saddr) : make_kmajor_sw128_desc(saddr); }

struct ProductParams {
    int rows, cols;                 // of the output: contiguous axis, other axis
    int kstages;                    // 128-byte stages of the contraction
    int tiles_r, tiles_c;
    int k_shares;                   // cluster kernel
    int chunk;                      // gradients: stages after which the sums leave the tensor cores' accumulator
    uint32_t idesc;                 // without the tile's dimensions
    const float* r_scales; const float* c_scales; const void* bias;      // INT8; c_scales: gradients too, or null
    const uint8_t* flags; int parts;                // gradients: which stages have `parts` parts (of int8_values; null: none), the others one
    const uint32_t* maxima; int maxima_count;       // fp16 parts: of matrix_exponent, or null
    void* out; long long ldo;
    int out_type, accumulate;
    int behind;                     // launched behind a kernel of the same call: may be set up while that one drains
    Int8Ranges ranges;
};

constexpr int CHUNK = 8, CHUNK_SHORT = 128;
// contraction elements per stage
template <int KIND> constexpr int STAGE_ELEMENTS = KIND == INT8 ? 128 : 64;
template <int KIND> constexpr bool R_MN = KIND != INT8;
template <int KIND> constexpr bool S_MN = KIND == GRAD_W;

// Operand loads of one stage: `n` rows (K-major) or elements (MN-major) from `first`, stage ks of the contraction.
template <bool MN, int ELEMENTS, int N, int NCTA>
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* tm, int first, int ks, uint32_t bar)
{
    if constexpr (MN) {
        static_assert(N % 64 == 0, "whole boxes");
#pragma unroll
        for (int b = 0; b < N / 64; ++b) tma_load_2d<NCTA>(dst + b * MN_BOX, tm, first + 64 * b, ks * ELEMENTS, bar);
    } else tma_load_2d<NCTA>(dst, tm, ks * ELEMENTS, first, bar);
}
// the rows operand: codes, or a part of a gradient's values
template <int KIND, int NCTA>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* tm, int first, int ks, int part, uint32_t bar)
{
    if constexpr (KIND == INT8) load_operand<false, STAGE_ELEMENTS<KIND>, 128, NCTA>(dst, tm, first, ks, bar);
    else {
#pragma unroll
        for (int b = 0; b < 2; ++b) tma_load_3d<NCTA>(dst + b * MN_BOX, tm, first + 64 * b, ks * STAGE_ELEMENTS<KIND>, part, bar);
    }
}
// The loads of stages [ks0, ks1) of the contraction, load(stage, part) each, until one says false.  Groups of PART_GROUP stages: the small parts
// of all of them come before the first, so that what the tensor cores cut off at each addition is a unit of the whole sum in the last pass
// only (fp32 weight gradient, default scales, 8192 terms: 3.8e-6 off with the parts stage by stage in chunks of 16, 4.4e-7 this way).  Flags are
// read a group ahead; `next`: the group's that follows these stages.  Warp-collective.
constexpr int PART_GROUP = 8;
static_assert(CHUNK % PART_GROUP == 0 && CHUNK_SHORT % PART_GROUP == 0, "all parts of a stage are in one chunk");
template <int KIND> struct StageWalk {
    static_assert(KIND == INT8 || STAGE_ELEMENTS<KIND> == INT8_PART_ROWS, "values_kernel goes by the same stages");
    const ProductParams& p;
    uint32_t ahead = 0;
    __device__ __forceinline__ void fetch(int group)
    {
        if (KIND == INT8 || !p.flags) return;
        const int lane = threadIdx.x & 31;
        ahead = lane < PART_GROUP && group + lane < p.kstages ? p.flags[group + lane] : 0u;
    }
    template <typename L> __device__ __forceinline__ bool run(int ks0, int ks1, int next, L&& load)
    {
        if constexpr (KIND != INT8) {
            if (p.flags) {
                for (int group = ks0; group < ks1; group += PART_GROUP) {
                    const uint32_t mask = warp_uniform(__ballot_sync(0xffffffffu, ahead));
                    const int end = min(group + PART_GROUP, ks1);
                    fetch(end < ks1 ? end : next);
                    for (int part = mask ? p.parts - 1 : 0; part >= 0; --part)
                        for (int ks = group; ks < end; ++ks)
                            if ((part == 0 || (mask >> (ks - group) & 1)) && !load(ks, part)) return false;
                }
                return true;
            }
        }
        for (int ks = ks0; ks < ks1; ++ks) if (!load(ks, 0)) return false;
        return true;
    }
};
// The warp that multiplies them need not tell parts apart: it is told how many pipeline stages a chunk of the walk has, and counts the next
// chunk's while this one's are on their way.  (With the parts in its loop it issues the MMAs more slowly, whatever their number: 8192 cubed in
// 856 instead of 764 us.)  Warp-collective.
template <int KIND> struct ChunkStages {
    const ProductParams& p;
    uint32_t inexact = 0;
    __device__ __forceinline__ void look(int from, int to)
    {
        if (KIND == INT8 || !p.flags) return;
        inexact = 0;
        for (int ks = from + (threadIdx.x & 31); ks < to; ks += 32) inexact += p.flags[ks];
    }
    // of the chunk that was looked at last
    __device__ __forceinline__ int count(int stages)
    {
        if (KIND == INT8 || !p.flags) return stages;
        return (int)warp_uniform(stages + (p.parts - 1) * __reduce_add_sync(0xffffffffu, inexact));
    }
};
// what the sums of fp16 parts are multiplied by
__device__ __forceinline__ float part_inverse(const ProductParams& p) { return p.maxima ? power_of_two(-matrix_exponent(p.maxima, p.maxima_count)) : 1.0f; }
// the four MMAs of a stage
template <int KIND, int NCTA>
__device__ __forceinline__ void mma_stage(uint32_t d, uint32_t r_addr, uint32_t s_addr, uint32_t idesc, bool first)
{
    const uint64_t rd = make_desc<R_MN<KIND>>(r_addr), sd = make_desc<S_MN<KIND>>(s_addr);
    constexpr int RSTEP = R_MN<KIND> ? 2048 >> 4 : 32 >> 4, SSTEP = S_MN<KIND> ? 2048 >> 4 : 32 >> 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) mma<KIND, NCTA>(d, rd + RSTEP * j, sd + SSTEP * j, idesc, (!first || j > 0) ? 1u : 0u);
}

// What becomes of a sum.  INT8: acc * lo * hi with the smaller scale first, so that nothing overflows on the way to a result that does
// not (a comparison with NaN keeps both); then the bias.
__device__ __forceinline__ float scaled(uint32_t acc, float a, float b)
{
    const bool first = a <= b;
    return __int2float_rn((int)acc) * (first ? a : b) * (first ? b : a);
}
template <typename T> __device__ __forceinline__ void put_one(const ProductParams& p, long long at, float v)
{
    T* q = static_cast<T*>(p.out) + at;
    if (!INT8_STORE_OK(p.ranges, q, sizeof(T), 2201, &g_int8_product_status[2])) return;
    if (p.accumulate) v += to_float(*q);
    *q = from_float<T>(v);
}
__device__ __forceinline__ float load_bias(const ProductParams& p, int row)
{
    if (!p.bias) return 0.0f;
    if (p.out_type == FMM_TYPE_F32) return static_cast<const float*>(p.bias)[row];
    if (p.out_type == FMM_TYPE_BF16) return to_float(static_cast<const __nv_bfloat16*>(p.bias)[row]);
    return to_float(static_cast<const __half*>(p.bias)[row]);
}
// N columns from col0 of one row of the output, from a thread's registers, `valid` of which exist.  c_scale: shared address of column
// col0's scale (gradients: if there are any; r_scale: their sums' factor, a power of two).  All of them are computed before the first is stored, and whole groups without a test in between: with one the
// columns came one after the other, 75 cycles each (4096 x 4096 x 128: 47.6 us a call, 19.4 without).
template <int KIND, int N>
__device__ __forceinline__ void put_columns(const ProductParams& p, const uint32_t (&v)[N], int row, int col0, int valid, float r_scale, float bias, uint32_t c_scale)
{
    if (row >= p.rows) return;
    float x[N];
    if (KIND == INT8 || p.c_scales) {
        float s[N];
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int j = 0; j < N; j += 4) { const float4 f = lds128(c_scale + 4 * j); s[j] = f.x; s[j + 1] = f.y; s[j + 2] = f.z; s[j + 3] = f.w; }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) s[j] = lds32f(c_scale + 4 * j);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = KIND == INT8 ? scaled(v[j], r_scale, s[j]) + bias : __uint_as_float(v[j]) * s[j];
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = __uint_as_float(v[j]) * r_scale;
    }
    auto each = [&](auto type) {
        using T = decltype(type);
        T* q = static_cast<T*>(p.out) + ((long long)col0 * p.ldo + row);
#ifndef FMM_DEBUG
        if (valid >= N) {
            if (p.accumulate) {
#pragma unroll
                for (int j = 0; j < N; ++j) x[j] += to_float(q[j * p.ldo]);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) q[j * p.ldo] = from_float<T>(x[j]);
            return;
        }
#endif
#pragma unroll
        for (int j = 0; j < N; ++j) if (j < valid) put_one<T>(p, (q - static_cast<T*>(p.out)) + j * p.ldo, x[j]);
    };
    if (p.out_type == FMM_TYPE_F32) each(float{});
    else if (p.out_type == FMM_TYPE_BF16) each(__nv_bfloat16{});
    else each(__half{});
}

// ------------------------------------------------------------------------------------------------ cluster kernel
// One tile of 128 rows x TC columns per cluster of k_shares CTAs, each of which sums a share of the contraction; the shares meet in
// distributed shared memory and are added in ascending order.  For products of few tiles: latency (a launch, the first load, the
// exchange) and, with few columns, the weight's way from memory bound it, so the contraction is cut until the device is full.
// INT8: two CTAs fit an SM; one exchanges or waits for its first operands while the other multiplies.
//   the first 4 (8) warps  drain TMEM, exchange, output: a TMEM lane quadrant (and half of the columns) each
//   the last two           TMA producer, MMA issuer
template <int KIND, int TC>
struct ClusterCfg {
    static constexpr int R_BYTES = 128 * 128, S_BYTES = TC * 128, STAGE_BYTES = R_BYTES + S_BYTES;
    static constexpr int STAGES = (KIND == INT8 ? 98304 : 196608) / STAGE_BYTES;       // INT8: 5, 4, 4, 3 for 16, 32, 64, 128 columns
    static constexpr int OFF_SCALES = STAGES * STAGE_BYTES, OFF_BAR = OFF_SCALES + TC * 4;
    static constexpr int BUFS = KIND == INT8 ? 1 : 2, NUM_BARS = 2 * STAGES + 2 * BUFS;         // accumulators; gradients: a chunk is drained
    static constexpr int SMEM_BYTES = OFF_BAR + NUM_BARS * 8 + 16 + 1024;                       // while the next one is multiplied
    static constexpr int TMEM_COLS = BUFS * TC < 32 ? 32 : BUFS * TC;
    // gradients keep a chunk's sums in registers: twice the warps, one CTA per SM
    static constexpr int OUT_WARPS = KIND == INT8 ? 4 : 8, THREADS = (OUT_WARPS + 2) * 32, CTAS = KIND == INT8 ? 2 : 1;
    static_assert(TMEM_COLS <= 512 / CTAS, "TMEM of an SM");
    static_assert(SMEM_BYTES + 1024 <= 233472 / (KIND == INT8 ? 2 : 1), "shared memory of an SM");
    static_assert(TC * 512 <= OFF_SCALES, "the exchange tile lies inside the operand ring");
};

template <int KIND, int TC>
__global__ void __launch_bounds__(ClusterCfg<KIND, TC>::THREADS, ClusterCfg<KIND, TC>::CTAS)
int8_cluster_kernel(const __grid_constant__ CUtensorMap tmR, const __grid_constant__ CUtensorMap tmS, const ProductParams p)
{
    using C = ClusterCfg<KIND, TC>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;       // the same offset in every CTA of the cluster
    uint8_t* base_ptr = smem_raw + (base - raw_addr);
    const uint32_t bar0 = base + C::OFF_BAR;
    auto bar_full = [&](int s) { return bar0 + 8u * s; };
    auto bar_empty = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
    auto bar_tfull = [&](int b) { return bar0 + 8u * (2 * C::STAGES + b); };
    auto bar_tempty = [&](int b) { return bar0 + 8u * (2 * C::STAGES + C::BUFS + b); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + C::OFF_BAR + C::NUM_BARS * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const Ctl ctl{abort_flag, g_int8_product_status};

    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (warp == C::OUT_WARPS && elect_one()) { prefetch_map(&tmR); prefetch_map(&tmS); }
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
        for (int b = 0; b < C::BUFS; ++b) { mbar_init(bar_tfull(b), 1); mbar_init(bar_tempty(b), C::OUT_WARPS); }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == C::OUT_WARPS + 1) {
        tmem_alloc<1>(smem_u32(tmem_slot), C::TMEM_COLS);
        tmem_relinquish<1>();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = warp_uniform(*tmem_slot);

    const int shares = p.k_shares, rank = shares > 1 ? (int)warp_uniform(cluster_ctarank()) : 0;
    const int tile = (int)(blockIdx.x / (unsigned)shares), tr = tile % p.tiles_r, tc = tile / p.tiles_r;
    const int ks0 = (int)((long long)p.kstages * rank / shares), ks1 = (int)((long long)p.kstages * (rank + 1) / shares);
    const int row0 = tr * 128, col0 = tc * TC;

    if (warp == C::OUT_WARPS) {
        int stage = 0; uint32_t phase = 0;
        StageWalk<KIND> walk{p};
        griddep_wait();
        walk.fetch(ks0);
        walk.run(ks0, ks1, ks0, [&](int ks, int part) {
            if (!mbar_wait_warp(bar_empty(stage), phase ^ 1u, ctl, 2301)) return false;
            if (elect_one()) {
                const uint32_t s = base + stage * C::STAGE_BYTES;
                mbar_expect_tx(bar_full(stage), C::STAGE_BYTES);
                load_rows<KIND, 1>(s, &tmR, row0, ks, part, bar_full(stage));
                load_operand<S_MN<KIND>, STAGE_ELEMENTS<KIND>, TC, 1>(s + C::R_BYTES, &tmS, col0, ks, bar_full(stage));
            }
            if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
            return true;
        });
    } else if (warp == C::OUT_WARPS + 1) {
        int stage = 0, buf = 0; uint32_t phase = 0, bphase = 0;
        griddep_wait();                                      // (the limit of the waits counts from here)
        const uint32_t idesc = p.idesc | ((uint32_t)(TC >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        bool ok = true;
        ChunkStages<KIND> chunk{p};
        chunk.look(ks0, min(ks0 + p.chunk, ks1));
        for (int kc = ks0; kc < ks1 && ok; kc += p.chunk) {
            if (!mbar_wait_warp(bar_tempty(buf), bphase ^ 1u, ctl, 2304)) break;
            tc_fence_after();
            const int end = min(kc + p.chunk, ks1), stages = chunk.count(end - kc);
            chunk.look(end, min(end + p.chunk, ks1));
            for (int i = 0; i < stages; ++i) {
                if (!mbar_wait_warp(bar_full(stage), phase, ctl, 2302)) { ok = false; break; }
                tc_fence_after();
                const uint32_t s = base + stage * C::STAGE_BYTES;
                mma_stage<KIND, 1>(tmem_base + buf * TC, s, s + C::R_BYTES, idesc, i == 0);
                tc_commit<1>(bar_empty(stage));
                if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
            }
            if (ok) tc_commit<1>(bar_tfull(buf));
            if (++buf == C::BUFS) { buf = 0; bphase ^= 1u; }
        }
    } else {
        griddep_wait();
        const uint32_t scales = base + C::OFF_SCALES;
        if (KIND == INT8 || p.c_scales) {
            for (int i = threadIdx.x; i < TC; i += C::OUT_WARPS * 32) sts32u(scales + 4 * i, col0 + i < p.cols ? __float_as_uint(p.c_scales[col0 + i]) : 0u);
            asm volatile("bar.sync 1, %0;" ::"n"(C::OUT_WARPS * 32) : "memory");
        }
        constexpr int CH = TC < 32 ? TC : 32, COLS = TC * 4 / C::OUT_WARPS;      // columns of a warp
        const int quadrant = warp & 3, first = (warp >> 2) * COLS;
        const uint32_t lane_taddr = tmem_base + ((uint32_t)(quadrant * 32) << 16);
        const int valid = min(TC, p.cols - col0), row = row0 + quadrant * 32 + lane;
        // share 1: the output; else a column-major tile of 128 x 4 bytes a column, over the operand ring, once every MMA of this CTA has
        // read its operands
        auto put = [&](const uint32_t (&v)[CH], int c, float r_scale, float bias) {
            if (shares == 1) put_columns<KIND, CH>(p, v, row, col0 + c, valid - c, r_scale, bias, scales + 4 * c);
            else {
#pragma unroll
                for (int j = 0; j < CH; ++j) sts32u(base + (c + j) * 512 + (quadrant * 32 + lane) * 4, v[j]);
            }
        };
        if constexpr (KIND == INT8) {
            float r_scale = 0.0f, bias = 0.0f;
            if (shares == 1 && row < p.rows) { r_scale = p.r_scales[row]; bias = load_bias(p, row); }
            const bool ok = mbar_wait_warp(bar_tfull(0), 0, ctl, 2303);
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < valid && ok; c += CH) {
                uint32_t v[CH];
                if constexpr (CH == 32) tmem_ld32(lane_taddr + c, v); else tmem_ld16(lane_taddr + c, v);
                tmem_ld_wait();
                put(v, c, r_scale, bias);
            }
        } else {
            float sum[COLS / CH][CH];
            const float inverse = part_inverse(p);
            int buf = 0; uint32_t bphase = 0;
            bool ok = true;
            for (int kc = ks0; kc < ks1; kc += p.chunk) {
                if (!mbar_wait_warp(bar_tfull(buf), bphase, ctl, 2303)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < COLS; c += 16) {
                    uint32_t v[16];
                    tmem_ld16(lane_taddr + buf * TC + first + c, v);
                    tmem_ld_wait16(v);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float& s = sum[(c + j) / CH][(c + j) % CH];
                        s = kc == ks0 ? __uint_as_float(v[j]) : s + __uint_as_float(v[j]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_tempty(buf));
                if (++buf == C::BUFS) { buf = 0; bphase ^= 1u; }
            }
#pragma unroll
            for (int i = 0; i < COLS / CH; ++i) {
                uint32_t v[CH];
#pragma unroll
                for (int j = 0; j < CH; ++j) v[j] = __float_as_uint(sum[i][j]);
                if (ok && first + i * CH < valid) put(v, first + i * CH, inverse, 0.0f);
            }
        }
    }
    if (shares > 1) {
        cluster_sync();                                      // every share is in its CTA's shared memory
        if (warp < C::OUT_WARPS && !*abort_flag) {
            const int valid = min(TC, p.cols - col0), row = row0 + 4 * lane;
            const uint32_t scales = base + C::OFF_SCALES;
            float r_scale[4] = {}, bias[4] = {};
            if constexpr (KIND == INT8) {
#pragma unroll
                for (int i = 0; i < 4; ++i) if (row + i < p.rows) { r_scale[i] = p.r_scales[row + i]; bias[i] = load_bias(p, row + i); }
            } else r_scale[0] = r_scale[1] = r_scale[2] = r_scale[3] = part_inverse(p);
            // the tile's columns are dealt out to the cluster's output warps
            for (int c = rank * C::OUT_WARPS + warp; c < valid; c += C::OUT_WARPS * shares) {
                uint4 x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) if (j < shares) x[j] = ld_cluster128u(map_to_cta(base + c * 512 + lane * 16, j));
                uint32_t sum[4] = {x[0].x, x[0].y, x[0].z, x[0].w};
#pragma unroll
                for (int j = 1; j < 8; ++j)
                    if (j < shares) {
                        const uint32_t y[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            sum[i] = KIND == INT8 ? sum[i] + y[i] : __float_as_uint(__uint_as_float(sum[i]) + __uint_as_float(y[i]));
                    }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t one[1] = {sum[i]};
                    put_columns<KIND, 1>(p, one, row + i, col0 + c, 1, r_scale[i], bias[i], scales + 4 * c);
                }
            }
        }
    }
    // ---------------------------------------------------------------------- teardown
    if (*abort_flag) {
        // let copies that are still in flight towards this CTA's shared memory land
        const uint64_t t0 = global_timer();
        while (global_timer() - t0 < 200000ull) __nanosleep(1000);
    }
    tc_fence_before();
    if (shares > 1) cluster_sync_relaxed();                  // the peers no longer read this CTA's shared memory
    else __syncthreads();
    if (warp == C::OUT_WARPS + 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc<1>(tmem_base, C::TMEM_COLS);
    }
}

// ------------------------------------------------------------------------------------------------ persistent kernel
// CTA pairs (cta_group::2) walk tiles of 256 x 256: each CTA loads its 128 rows and half of the columns, so that an operand byte
// from L2 serves 256 multiply-accumulates.  Two TMEM accumulators: a tile is written out while the next one is multiplied.
template <int KIND>
struct PairCfg {
    static constexpr int TC = 256, R_BYTES = 128 * 128, S_BYTES = 128 * 128, STAGE_BYTES = R_BYTES + S_BYTES, STAGES = 6;
    // (scales: every output warp has its own copy of its columns')
    static constexpr int OFF_SCALES = STAGES * STAGE_BYTES, OFF_BAR = OFF_SCALES + 8 * (TC / 2) * 4, NUM_BARS = 2 * STAGES + 4;
    static constexpr int SMEM_BYTES = OFF_BAR + NUM_BARS * 8 + 16 + 1024;
    // warp 0 TMA producer, warp 1 MMA issuer, warps 4..11 output: a TMEM lane quadrant and half of the columns each, the gradients' sums
    // in registers
    static constexpr int OUT_WARPS = 8, OUT_WARP0 = 4, THREADS = (OUT_WARP0 + OUT_WARPS) * 32;
    static constexpr int REGS_AT_LAUNCH = 168, REGS_CTRL = 56, REGS_OUT = 216;
    static_assert(128 * REGS_CTRL + OUT_WARPS * 32 * REGS_OUT <= THREADS * REGS_AT_LAUNCH, "register pool");
    static_assert(SMEM_BYTES <= 232448, "shared memory of a block");
};

template <int KIND>
__global__ void __launch_bounds__(PairCfg<KIND>::THREADS, 1)
int8_pair_kernel(const __grid_constant__ CUtensorMap tmR, const __grid_constant__ CUtensorMap tmS, const ProductParams p)
{
    using C = PairCfg<KIND>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - raw_addr);
    const uint32_t bar0 = base + C::OFF_BAR;
    auto bar_full = [&](int s) { return bar0 + 8u * s; };
    auto bar_empty = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
    auto bar_tfull = [&](int b) { return bar0 + 8u * (2 * C::STAGES + b); };
    auto bar_tempty = [&](int b) { return bar0 + 8u * (2 * C::STAGES + 2 + b); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + C::OFF_BAR + C::NUM_BARS * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const Ctl ctl{abort_flag, g_int8_product_status};

    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rank = (int)warp_uniform(cluster_ctarank());
    const bool leader = rank == 0;
    if (warp == 2 && elect_one()) { prefetch_map(&tmR); prefetch_map(&tmS); }
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(bar_tfull(b), 1); mbar_init(bar_tempty(b), 2 * C::OUT_WARPS); }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc<2>(smem_u32(tmem_slot), 512);
        tmem_relinquish<2>();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();                                          // the peer's barriers are initialised before anyone signals them
    tc_fence_after();
    const uint32_t tmem_base = warp_uniform(*tmem_slot);

    const int units = gridDim.x / 2, unit = blockIdx.x / 2;
    const long long tiles = (long long)p.tiles_r * p.tiles_c;
    // groups of eight tiles of rows, all columns of a group before the next: the tiles in flight share operands in L2
    auto place = [&](long long w, int& tr, int& tc) {
        const long long per = 8ll * p.tiles_c;
        const int g = (int)(w / per), first = 8 * g, rows = min(8, p.tiles_r - first), in = (int)(w - g * per);
        tr = first + in % rows;
        tc = in / rows;
    };

    if (warp < C::OUT_WARP0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_CTRL));
    if (warp == 0) {
        int stage = 0; uint32_t phase = 0;
        bool ok = true;
        StageWalk<KIND> walk{p};
        griddep_wait();
        walk.fetch(0);
        for (long long w = unit; w < tiles && ok; w += units) {
            int tr, tc;
            place(w, tr, tc);
            ok = walk.run(0, p.kstages, 0, [&](int ks, int part) {
                if (!mbar_wait_warp(bar_empty(stage), phase ^ 1u, ctl, 2311)) return false;
                // completion is counted on the even CTA's barrier; only that CTA arms it
                const uint32_t fb = bar_full(stage) & PEER_BIT_MASK;
                if (elect_one()) {
                    const uint32_t s = base + stage * C::STAGE_BYTES;
                    if (leader) mbar_expect_tx(bar_full(stage), 2 * C::STAGE_BYTES);
                    load_rows<KIND, 2>(s, &tmR, (2 * tr + rank) * 128, ks, part, fb);
                    load_operand<S_MN<KIND>, STAGE_ELEMENTS<KIND>, 128, 2>(s + C::R_BYTES, &tmS, (2 * tc + rank) * 128, ks, fb);
                }
                if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                return true;
            });
        }
    } else if (warp == 1) {
        if (leader) {
            int stage = 0, buf = 0; uint32_t phase = 0, bphase = 0;
            griddep_wait();
            const uint32_t idesc = p.idesc | ((uint32_t)(C::TC >> 3) << 17) | ((uint32_t)(256 >> 4) << 24);
            bool ok = true;
            ChunkStages<KIND> chunk{p};
            chunk.look(0, min(p.chunk, p.kstages));
            for (long long w = unit; w < tiles && ok; w += units)
                for (int kc = 0; kc < p.kstages && ok; kc += p.chunk) {
                    if (!mbar_wait_warp(bar_tempty(buf), bphase ^ 1u, ctl, 2312)) { ok = false; break; }
                    tc_fence_after();
                    const int end = min(kc + p.chunk, p.kstages), stages = chunk.count(end - kc), from = end < p.kstages ? end : 0;
                    chunk.look(from, min(from + p.chunk, p.kstages));
                    for (int i = 0; i < stages; ++i) {
                        if (!mbar_wait_warp(bar_full(stage), phase, ctl, 2313)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t s = base + stage * C::STAGE_BYTES;
                        mma_stage<KIND, 2>(tmem_base + buf * C::TC, s, s + C::R_BYTES, idesc, i == 0);
                        tc_commit<2>(bar_empty(stage));
                        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
                    tc_commit<2>(bar_tfull(buf));
                    if (++buf == 2) { buf = 0; bphase ^= 1u; }
                }
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::REGS_OUT));
        constexpr int COLS = C::TC / 2;                      // of a warp
        const int quadrant = warp & 3, half = (warp - C::OUT_WARP0) >> 2;
        const uint32_t lane_taddr = tmem_base + half * COLS + ((uint32_t)(quadrant * 32) << 16);
        int buf = 0; uint32_t bphase = 0;
        bool ok = true;
        griddep_wait();
        const float inverse = KIND == INT8 ? 1.0f : part_inverse(p);
        auto release = [&] {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(bar_tempty(buf) & PEER_BIT_MASK);
            if (++buf == 2) { buf = 0; bphase ^= 1u; }
        };
        uint32_t next_scale[COLS / 32];
        auto fetch_scales = [&](long long w) {
            if (w >= tiles) return;
            int tr, tc;
            place(w, tr, tc);
#pragma unroll
            for (int i = 0; i < COLS / 32; ++i) {
                const int col = tc * C::TC + half * COLS + lane + 32 * i;
                next_scale[i] = col < p.cols ? __float_as_uint(p.c_scales[col]) : 0u;
            }
        };
        if (KIND == INT8 || p.c_scales) fetch_scales(unit);
        for (long long w = unit; w < tiles && ok; w += units) {
            int tr, tc;
            place(w, tr, tc);
            const int row = (2 * tr + rank) * 128 + quadrant * 32 + lane, col0 = tc * C::TC + half * COLS;
            const int valid = min(COLS, p.cols - col0);
            const uint32_t scales = base + C::OFF_SCALES + (warp - C::OUT_WARP0) * COLS * 4;
            if (KIND == INT8 || p.c_scales) {
                // (No warp waits here for another: one whose wait below has run out leaves the loop, and a barrier among the output
                // warps would then have no limit for those whose wait has not.)
                __syncwarp();                                // the tile before is out
#pragma unroll
                for (int i = 0; i < COLS / 32; ++i) sts32u(scales + 4 * (lane + 32 * i), next_scale[i]);
                __syncwarp();
                fetch_scales(w + units);                     // (a tile ahead: 8192 x 8192 x 1024 product in 63.7 instead of 67.4 us)
            }
            if constexpr (KIND == INT8) {
                float r_scale = 0.0f, bias = 0.0f;
                if (row < p.rows) { r_scale = p.r_scales[row]; bias = load_bias(p, row); }
                if (!mbar_wait_warp(bar_tfull(buf), bphase, ctl, 2314)) break;
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < valid; c += 32) {
                    uint32_t v[32];
                    tmem_ld32(lane_taddr + buf * C::TC + c, v);
                    tmem_ld_wait();
                    put_columns<KIND, 32>(p, v, row, col0 + c, valid - c, r_scale, bias, scales + 4 * c);
                }
                release();
            } else {
                float sum[COLS / 32][32];
                for (int kc = 0; kc < p.kstages; kc += p.chunk) {
                    if (!mbar_wait_warp(bar_tfull(buf), bphase, ctl, 2314)) { ok = false; break; }
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < COLS; c += 16) {
                        uint32_t v[16];
                        tmem_ld16(lane_taddr + buf * C::TC + c, v);
                        tmem_ld_wait16(v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            float& s = sum[c / 32][c % 32 + j];
                            s = kc == 0 ? __uint_as_float(v[j]) : s + __uint_as_float(v[j]);
                        }
                    }
                    release();
                }
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < COLS / 32; ++i) {
                    uint32_t v[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(sum[i][j]);
                    if (32 * i < valid) put_columns<KIND, 32>(p, v, row, col0 + 32 * i, valid - 32 * i, inverse, 0.0f, scales + 128 * i);
                }
            }
        }
    }
    // ---------------------------------------------------------------------- teardown
    if (*abort_flag) {
        const uint64_t t0 = global_timer();
        while (global_timer() - t0 < 200000ull) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();                                          // the peer no longer signals this CTA's barriers
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc<2>(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------------ few tokens
// C of up to eight tokens: the weight's way from memory bounds it, and this kernel has nothing to set up (the cluster kernel: barriers,
// TMEM, tensor maps, an exchange; 1 x 8192 x 8192 15.2 us, 14.0 here, 8 x 4096 x 4096 7.7 and 5.4, 1 x 2048 x 2048 5.1 and 2.8).  A block takes
// 16 output channels, its warps share K: 16 of them, where two such blocks an SM hold all channels (1 x 2048 x 8192 6.7 us, with eight 9.6), else
// eight, four blocks an SM, so that they come in one wave or in many (1 x 8192 x 8192 14.0 us, with 16 15.4).  The weight goes from global memory straight into the A fragments of mma.m16n8k32, the tokens into the B fragments:
// a lane loads 16 codes of channel lane / 4, of channel lane / 4 + 8 and of token lane / 4, all at the same place of K, and takes the first
// eight of each for one mma and the others for the next - both sides number the contraction alike, so any numbering will do.  (dp4a
// in place of the mma: as fast for one token, 19.3 us for four of them at 8192 x 8192.)
constexpr int FEW_TOKENS = 8, FEW_CHANNELS = 16, FEW_LOADS = 2;

struct FewParams {
    const int8_t* a; const int8_t* b;
    long long lda, ldb;
    int k;
    ProductParams p;
};

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes of a weight, which is read once: not kept in L1, 256 bytes brought into L2
__device__ __forceinline__ uint4 load_once(const int8_t* p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <int FEW_WARPS>
__global__ void __launch_bounds__(FEW_WARPS * 32, 32 / FEW_WARPS) int8_few_tokens_kernel(const FewParams f)
{
    __shared__ int meet[FEW_WARPS][FEW_TOKENS][FEW_CHANNELS + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const long long n0 = (long long)blockIdx.x * FEW_CHANNELS;
    const int channels = (int)min((long long)FEW_CHANNELS, f.p.rows - n0), tokens = f.p.cols;
    const int8_t* w0 = f.b + (n0 + g) * f.ldb + 16 * q;
    const int8_t* w1 = w0 + 8 * f.ldb;
    const int8_t* x0 = f.a + g * f.lda + 16 * q;
    const bool some0 = g < channels, some1 = g + 8 < channels, some = g < tokens;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    int acc[4] = {0, 0, 0, 0};
    // 64 codes of K a step; a warp takes FEW_LOADS steps at a time, the block's warps side by side
    constexpr int PIECE = 64 * FEW_LOADS;
    for (int k0 = warp * PIECE; k0 < f.k; k0 += FEW_WARPS * PIECE) {
        uint4 u[FEW_LOADS], v[FEW_LOADS], x[FEW_LOADS];
#pragma unroll
        for (int i = 0; i < FEW_LOADS; ++i) {
            const int k = k0 + 64 * i;
            const bool in = k + 16 * q < f.k;
            u[i] = in && some0 ? load_once(w0 + k) : zero;
            v[i] = in && some1 ? load_once(w1 + k) : zero;
            x[i] = in && some ? *reinterpret_cast<const uint4*>(x0 + k) : zero;
        }
#pragma unroll
        for (int i = 0; i < FEW_LOADS; ++i) {
            const int left = f.k - (k0 + 64 * i + 16 * q);
            if (left < 16) {
                // the codes behind the last one may be anything, on either side: zeros on this one
                uint32_t* y = &x[i].x;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = left - 4 * j;
                    y[j] = n >= 4 ? y[j] : n <= 0 ? 0u : y[j] & ((1u << (8 * n)) - 1u);
                }
            }
            mma_s8(acc, u[i].x, v[i].x, u[i].y, v[i].y, x[i].x, x[i].y);
            mma_s8(acc, u[i].z, v[i].z, u[i].w, v[i].w, x[i].z, x[i].w);
        }
    }
    // accumulators: channels g and g + 8 of tokens 2q and 2q + 1
    meet[warp][2 * q][g] = acc[0];
    meet[warp][2 * q + 1][g] = acc[1];
    meet[warp][2 * q][g + 8] = acc[2];
    meet[warp][2 * q + 1][g + 8] = acc[3];
    __syncthreads();
    const int r = threadIdx.x % FEW_CHANNELS, m = threadIdx.x / FEW_CHANNELS;
    if (m < tokens && r < channels) {
        int s = 0;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) s += meet[w][m][r];
        const int row = (int)n0 + r;
        const float y = scaled((uint32_t)s, f.p.r_scales[row], f.p.c_scales[m]) + load_bias(f.p, row);
        const long long at = m * f.p.ldo + row;
        if (f.p.out_type == FMM_TYPE_F32) put_one<float>(f.p, at, y);
        else if (f.p.out_type == FMM_TYPE_BF16) put_one<__nv_bfloat16>(f.p, at, y);
        else put_one<__half>(f.p, at, y);
    }
}

// An empty contraction: C = bias, or 0
__global__ void __launch_bounds__(256) empty_sum_kernel(const ProductParams p)
{
    const long long n = (long long)p.rows * p.cols;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int col = (int)(i / p.rows), row = (int)(i - (long long)col * p.rows);
        const float v = load_bias(p, row);
        const long long at = (long long)col * p.ldo + row;
        if (p.out_type == FMM_TYPE_F32) put_one<float>(p, at, v);
        else if (p.out_type == FMM_TYPE_BF16) put_one<__nv_bfloat16>(p, at, v);
        else put_one<__half>(p, at, v);
    }
}

// ------------------------------------------------------------------------------------------------ host side
struct Operand { const void* p; int64_t rows, cols, ld, parts = 1, step = 0; };        // row-major, cols contiguous; ld and step in elements

template <int KIND, bool MN>
bool make_operand_map(CUtensorMap* tm, const Operand& o, int n)
{
    const CUtensorMapDataType dt = KIND == INT8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
    const int e = KIND == INT8 ? 1 : 2;
    return make_map_2d(tm, dt, e, o.p, (uint64_t)o.cols, (uint64_t)o.rows, MN ? 64 : 128 / e, MN ? 64 : n, CU_TENSOR_MAP_SWIZZLE_128B, (uint64_t)o.ld);
}

// the rows operand: codes, or the parts of a gradient's values
template <int KIND> bool make_rows_map(CUtensorMap* tm, const Operand& o)
{
    if constexpr (KIND == INT8) return make_operand_map<KIND, false>(tm, o, 128);
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.parts}, strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)o.step * 2};
    const cuuint32_t box[3] = {64, 64, 1}, steps[3] = {1, 1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void*>(o.p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The kernel's shared memory limit, raised once per device.
template <typename K> bool raise_smem(K kernel, int bytes, std::atomic<bool>* done)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return false; }
    if (dev < 64 && done[dev].load(std::memory_order_acquire)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) { cudaGetLastError(); return false; }
    if (dev < 64) done[dev].store(true, std::memory_order_release);
    return true;
}

template <typename K>
fmm_status_t launch_kernel(K kernel, unsigned grid, unsigned threads, int smem, unsigned cluster, const CUtensorMap& r, const CUtensorMap& s, const ProductParams& p, cudaStream_t st)
{
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    // behind the kernel that restores its operand; its warps wait for that one before their first load or store.  (The first kernel of
    // a call is launched in full stream order, as everywhere in this library.)
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = p.behind ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, r, s, p) != cudaSuccess) { cudaGetLastError(); return FMM_ERR_CUDA; }
    return FMM_OK;
}

template <int KIND>
fmm_status_t launch_pair(ProductParams p, const Operand& r, const Operand& s, cudaStream_t st)
{
    using C = PairCfg<KIND>;
    static std::atomic<bool> done[64];
    CUtensorMap tmR, tmS;
    if (!make_rows_map<KIND>(&tmR, r) || !make_operand_map<KIND, S_MN<KIND>>(&tmS, s, 128) ||
        !raise_smem(int8_pair_kernel<KIND>, C::SMEM_BYTES, done)) return FMM_ERR_CUDA;
    p.tiles_r = (p.rows + 255) / 256; p.tiles_c = (p.cols + 255) / 256; p.k_shares = 1;
    // as few pairs as finish in the same number of waves
    const int64_t tiles = (int64_t)p.tiles_r * p.tiles_c, most = std::max(1, int8_sm_count() / 2), waves = (tiles + most - 1) / most;
    return launch_kernel(int8_pair_kernel<KIND>, (unsigned)((tiles + waves - 1) / waves * 2), C::THREADS, C::SMEM_BYTES, 2, tmR, tmS, p, st);
}

template <int KIND, int TC>
fmm_status_t launch_cluster(ProductParams p, const Operand& r, const Operand& s, int shares, cudaStream_t st)
{
    using C = ClusterCfg<KIND, TC>;
    static std::atomic<bool> done[64];
    CUtensorMap tmR, tmS;
    if (!make_rows_map<KIND>(&tmR, r) || !make_operand_map<KIND, S_MN<KIND>>(&tmS, s, TC) ||
        !raise_smem(int8_cluster_kernel<KIND, TC>, C::SMEM_BYTES, done)) return FMM_ERR_CUDA;
    p.tiles_r = (p.rows + 127) / 128; p.tiles_c = (p.cols + TC - 1) / TC; p.k_shares = shares;
    const int64_t grid = (int64_t)p.tiles_r * p.tiles_c * shares;
    if (grid > 0x7FFFFFFF) return launch_pair<KIND>(p, r, s, st);       // (the model never chooses so many)
    return launch_kernel(int8_cluster_kernel<KIND, TC>, (unsigned)grid, C::THREADS, C::SMEM_BYTES, (unsigned)shares, tmR, tmS, p, st);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Time models of the two kernels in microseconds (a gradient's with the restoring of its operand), fitted to 3100 timed calls of both with
// every tile width and number of shares: 16 to 2048 tokens, 512 to 16384 channels, K of 512 to 8192; gradients of 64 to 16384 tokens, 128 to 2048
// channels each way.  Cluster kernel: lat + rounds * fixed + the stages of an SM, of a single CTA (`stage` each) or of as many as it
// holds (`shared` each), + what the exchange takes; a share more leaves 2 % more places in the GPCs empty.  CTAs without an exchange
// make room one by one, so their rounds are a fraction.  Pairs: lat + waves of stages, + what a tile's output costs beyond the next
// tile's stages.  The choice takes 1.1 % (gradients 0.1 %) more time than the fastest of these in the mean, at worst 1.31 times it (2048 x
// 512 x 8192: 22.9, 17.4 us).  Beyond the calls of the fit: gradients of 64 to 8192 tokens and 128 to 4096 channels 2.5 % in the mean, at worst 1.38
// times (weight, 6192 x 1656 x 3128: 136, 99 us).  The models know one part a stage; weight gradients of three take 6.5 % more in the mean.
struct ClusterModel { int columns; float lat, stage, shared, fixed; };
struct ProductModel { float pair_lat, pair_stage, pair_tile, exchange, exchange_share; int per_sm, widths; ClusterModel cluster[4]; };
constexpr ProductModel MODEL_INT8 = {6.544f, 0.277f, 2.584f, 2.365f, 0.022f, 2, 4,
    {{16, 0.937f, 0.216f, 0.199f, 1.682f}, {32, 1.818f, 0.242f, 0.251f, 1.138f}, {64, 2.255f, 0.221f, 0.157f, 2.707f}, {128, 2.161f, 0.282f, 0.458f, 2.846f}}};
constexpr ProductModel MODEL_GRAD = {5.718f, 0.348f, 0.852f, 0.617f, 0.223f, 1, 2, {{64, 1.203f, 0.175f, 0.222f, 3.804f}, {128, 1.266f, 0.213f, 0.278f, 4.779f}}};

fmm_status_t launch_few_tokens(const ProductParams& p, const Operand& b, const Operand& a, cudaStream_t st)
{
    const FewParams f = {static_cast<const int8_t*>(a.p), static_cast<const int8_t*>(b.p), a.ld, b.ld, (int)a.cols, p};
    const int64_t blocks = ceil_div(p.rows, FEW_CHANNELS);
    if (blocks <= 2 * int8_sm_count()) int8_few_tokens_kernel<16><<<(unsigned)blocks, 512, 0, st>>>(f);
    else int8_few_tokens_kernel<8><<<(unsigned)blocks, 256, 0, st>>>(f);
    return cudaGetLastError() == cudaSuccess ? FMM_OK : FMM_ERR_CUDA;
}

struct ProductChoice { int columns, shares; };               // columns 256: pairs
ProductChoice choose_product(const ProductModel& m, const ProductParams& p, double bytes, int sms)
{
    const float by_memory = (float)(bytes / 6.2e6);
    const int64_t pair_tiles = ceil_div(p.rows, 256) * ceil_div(p.cols, 256), waves = ceil_div(pair_tiles, std::max(1, sms / 2));
    float best = std::max(m.pair_lat + (float)waves * p.kstages * m.pair_stage + (float)(waves - 1) * m.pair_tile, m.pair_lat + by_memory);
    ProductChoice choice = {256, 1};
    for (int w = 0; w < m.widths; ++w) {
        const ClusterModel& c = m.cluster[w];
        if (w > 0 && p.cols <= m.cluster[w - 1].columns) break;          // a narrower tile holds every column
        const int64_t tiles = ceil_div(p.rows, 128) * ceil_div(p.cols, c.columns);
        for (int shares = 1; shares <= 8 && shares <= p.kstages; ++shares) {
            const float ctas = (float)(tiles * shares), places = sms * m.per_sm * (1.0f - 0.02f * (shares - 1));
            float rounds = std::max(1.0f, ctas / places);
            if (shares > 1) rounds = ceilf(rounds);
            const float stages = (float)ceil_div(p.kstages, shares);
            const float held = shares > 1 ? ceilf(ctas / sms) : ctas / sms, body = std::max(stages * c.stage * rounds, held * stages * c.shared);
            const float time = std::max(c.lat + rounds * c.fixed + body + (shares > 1 ? m.exchange + m.exchange_share * shares : 0.0f), 3.0f + by_memory);
            if (time < best) { best = time; choice = {c.columns, shares}; }
        }
    }
    return choice;
}

// what fmm_int8_force_product_shape set for this host thread; kernel 0: nothing
thread_local fmm_int8_product_shape_t forced_shape;
enum { SHAPE_PAIRS = 1, SHAPE_CLUSTER = 2, SHAPE_FEW = 3 };
constexpr int FEW_SHAPE_COLUMNS = FEW_TOKENS;

template <int KIND> fmm_int8_product_shape_t product_shape(const ProductParams& p, const Operand& r, const Operand& s)
{
    if (forced_shape.kernel) return forced_shape;
    if (KIND == INT8 && p.cols <= FEW_TOKENS) return {SHAPE_FEW, FEW_SHAPE_COLUMNS, 1};
    const int e = KIND == INT8 ? 1 : 2;
    const double bytes = (double)e * ((double)r.rows * r.cols + (double)s.rows * s.cols) + (double)p.rows * p.cols * int8_type_bytes((fmm_type_t)p.out_type);
    const ProductChoice c = choose_product(KIND == INT8 ? MODEL_INT8 : MODEL_GRAD, p, bytes, int8_sm_count());
    return {c.columns == 256 ? SHAPE_PAIRS : SHAPE_CLUSTER, c.columns, c.shares};
}
template <int KIND>
fmm_status_t launch_product(const ProductParams& p, const Operand& r, const Operand& s, cudaStream_t st)
{
    const fmm_int8_product_shape_t c = product_shape<KIND>(p, r, s);
    if (c.kernel == SHAPE_PAIRS) return launch_pair<KIND>(p, r, s, st);
    if constexpr (KIND == INT8) {
        if (c.kernel == SHAPE_FEW) return p.cols <= FEW_TOKENS ? launch_few_tokens(p, r, s, st) : FMM_ERR_SHAPE;
    }
    if (c.kernel != SHAPE_CLUSTER || c.k_shares > p.kstages) return FMM_ERR_SHAPE;
    if constexpr (KIND == INT8) {
        if (c.columns == 16) return launch_cluster<KIND, 16>(p, r, s, c.k_shares, st);
        if (c.columns == 32) return launch_cluster<KIND, 32>(p, r, s, c.k_shares, st);
    }
    if (c.columns == 64) return launch_cluster<KIND, 64>(p, r, s, c.k_shares, st);
    return c.columns == 128 ? launch_cluster<KIND, 128>(p, r, s, c.k_shares, st) : FMM_ERR_SHAPE;
}

fmm_status_t launch_empty(const ProductParams& p, cudaStream_t st)
{
    empty_sum_kernel<<<(unsigned)int8_sm_count() * 8, 256, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? FMM_OK : FMM_ERR_CUDA;
}

// whether a gradient's workspace has a size that can be had at all (and that 64 bits hold)
bool grad_dims_ok(int64_t M, int64_t N, int64_t K)
{
    if (!(M >= 0 && M < INT8_MAX_DIM && N >= 0 && N < INT8_MAX_DIM && K >= 0 && K < INT8_MAX_DIM)) return false;
    return 2.0 * (3.0 * std::max(M, N) * (K + 8) + (double)M * (N + 8)) < 0x1p46;
}
bool dim_ok(int64_t n) { return n >= 0 && n < INT8_MAX_DIM; }
int64_t up_to(int64_t n, int64_t a) { return ceil_div(n, a) * a; }

// What a gradient's product reads and where it lies in the workspace: the values' parts (or codes), what belongs to them (maxima of the scales
// and a flag for each stage, or a factor for each row of dY), and dY where it is not read as it lies.
struct GradPlan {
    bool scaled;                            // the scales go to dY (see the top)
    int parts;
    fmm_type_t operands;                    // type of what is multiplied
    int64_t ld_values, ld_dy;               // elements
    size_t extra, dy, total;                // bytes
};
template <int KIND> GradPlan grad_plan(const fmm_int8_grad_t* a)
{
    const int64_t code_rows = KIND == GRAD_W ? a->M : a->N;
    GradPlan w;
    w.scaled = KIND == GRAD_X && a->type == FMM_TYPE_BF16 && a->out_type == FMM_TYPE_BF16 && !a->rounded;
    w.parts = w.scaled || a->rounded ? 1 : a->type == FMM_TYPE_BF16 && a->out_type == FMM_TYPE_F32 ? 3 : 2;
    w.operands = w.scaled ? FMM_TYPE_F16 : a->type;
    w.ld_values = up_to(a->K, 8);
    w.ld_dy = up_to(a->N, 8);
    w.extra = (size_t)up_to(code_rows * w.ld_values * 2 * w.parts, 256);
    w.dy = w.extra + (size_t)up_to(w.scaled ? a->M * 4 : INT8_MAXIMA * 4 + ceil_div(code_rows, INT8_PART_ROWS), 256);
    w.total = w.dy + (!w.scaled && int8_aligned(a->dy, a->ldy * 2, 16) ? 0 : (size_t)up_to(a->M * w.ld_dy * 2, 256));
    return w;
}

template <int KIND> fmm_status_t grad_workspace_bytes(const fmm_int8_grad_t* a, size_t* bytes)
{
    if (!a || !bytes) return FMM_ERR_INVALID_ARG;
    if (!grad_dims_ok(a->M, a->N, a->K)) return FMM_ERR_SHAPE;
    *bytes = grad_plan<KIND>(a).total;
    return FMM_OK;
}

// Both gradients: what the product reads into the workspace, one product.
template <int KIND>
fmm_status_t grad(const fmm_int8_grad_t* a, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!a || (a->type != FMM_TYPE_BF16 && a->type != FMM_TYPE_F16) || (a->out_type != FMM_TYPE_F32 && a->out_type != a->type)) return FMM_ERR_INVALID_ARG;
    const fmm_type_t type = a->type, out_type = a->out_type;
    const int64_t M = a->M, N = a->N, K = a->K, ldy = a->ldy, ldc = a->ldc, ldo = a->ldo;
    const void* dY = a->dy;
    const int8_t* codes = a->codes;
    const float* scales = a->scales;
    if (!grad_dims_ok(M, N, K)) return FMM_ERR_SHAPE;
    const int64_t code_rows = KIND == GRAD_W ? M : N, contraction = code_rows, cols = KIND == GRAD_W ? N : M;
    if (K == 0 || cols == 0) return FMM_OK;
    const int eo = int8_type_bytes(out_type);
    if (!a->out || ldo < K || ((uintptr_t)a->out & (eo - 1))) return FMM_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    ProductParams p = {};
    p.rows = (int)K; p.cols = (int)cols;
    p.out = a->out; p.ldo = ldo; p.out_type = out_type; p.accumulate = a->accumulate != 0;
    int8_add_range(p.ranges, a->out, cols, K, ldo, eo);
    if (contraction == 0) return a->accumulate ? FMM_OK : launch_empty(p, st);
    if (!dY || ldy < N || ((uintptr_t)dY & 1) || !codes || ldc < K || !scales || ((uintptr_t)scales & 3)) return FMM_ERR_INVALID_ARG;
    const GradPlan w = grad_plan<KIND>(a);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < w.total) return FMM_ERR_WORKSPACE;
    char* base = static_cast<char*>(workspace);
    const int64_t step = code_rows * w.ld_values;
    Operand dy = {dY, M, N, ldy};
    fmm_status_t s = FMM_OK;
    if (w.scaled) {
        float* inverse = reinterpret_cast<float*>(base + w.extra);
        s = int8_codes_and_scaled_rows(codes, ldc, base, w.ld_values, code_rows, K, dY, ldy, scales, base + w.dy, w.ld_dy, inverse, M, st);
        dy = {base + w.dy, M, N, w.ld_dy};
        p.c_scales = inverse;
    } else {
        uint32_t* maxima = type == FMM_TYPE_F16 ? reinterpret_cast<uint32_t*>(base + w.extra) : nullptr;
        uint8_t* flags = w.parts > 1 ? reinterpret_cast<uint8_t*>(base + w.extra) + INT8_MAXIMA * 4 : nullptr;
        s = int8_values(w.operands, w.parts, codes, ldc, scales, maxima, flags, base, w.ld_values, step, code_rows, K, st);
        if (s == FMM_OK && !int8_aligned(dY, ldy * 2, 16)) {
            s = int8_realign(dY, ldy, base + w.dy, w.ld_dy, M, N, st);
            dy = {base + w.dy, M, N, w.ld_dy};
        }
        p.flags = flags; p.maxima = maxima; p.maxima_count = int8_scale_maxima_count(code_rows);
    }
    if (s != FMM_OK) return s;
    p.parts = w.parts;
    p.behind = 1;
    const uint32_t format = w.operands == FMM_TYPE_BF16 ? 1u : 0u;
    p.kstages = (int)ceil_div(contraction, 64);
    p.chunk = out_type == FMM_TYPE_F32 ? CHUNK : CHUNK_SHORT;
    p.idesc = (1u << 4) | (format << 7) | (format << 10) | (1u << 15) | ((KIND == GRAD_W ? 1u : 0u) << 16);
    return launch_product<KIND>(p, {base, code_rows, K, w.ld_values, w.parts, step}, dy, st);
}

}  // namespace

extern "C" {

fmm_status_t fmm_int8_matmul(const fmm_int8_matmul_t* a, void* stream)
{
    if (!a || !int8_type_ok(a->type)) return FMM_ERR_INVALID_ARG;
    const int64_t M = a->M, N = a->N, K = a->K;
    if (!dim_ok(M) || !dim_ok(N) || K < 0 || K > 131071) return FMM_ERR_SHAPE;
    if (M == 0 || N == 0) return FMM_OK;
    const int e = int8_type_bytes(a->type);
    if (!a->c || a->ldc < N || ((uintptr_t)a->c & (e - 1)) || ((uintptr_t)a->bias & (e - 1))) return FMM_ERR_INVALID_ARG;
    ProductParams p = {};
    p.rows = (int)N; p.cols = (int)M;
    p.r_scales = a->b_scales; p.c_scales = a->a_scales; p.bias = a->bias;
    p.out = a->c; p.ldo = a->ldc; p.out_type = a->type;
    int8_add_range(p.ranges, a->c, M, N, a->ldc, e);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (K == 0) return launch_empty(p, st);
    if (!a->a || !a->b || !a->a_scales || !a->b_scales || (((uintptr_t)a->a_scales | (uintptr_t)a->b_scales) & 3) || a->lda < K || a->ldb < K ||
        !int8_aligned(a->a, a->lda, 16) || !int8_aligned(a->b, a->ldb, 16)) return FMM_ERR_INVALID_ARG;
    p.kstages = p.chunk = (int)ceil_div(K, 128);
    p.idesc = (2u << 4) | (1u << 7) | (1u << 10);
    return launch_product<INT8>(p, {a->b, N, K, a->ldb}, {a->a, M, K, a->lda}, st);
}

fmm_status_t fmm_int8_grad_weight_workspace_bytes(const fmm_int8_grad_t* p, size_t* bytes) { return grad_workspace_bytes<GRAD_W>(p, bytes); }
fmm_status_t fmm_int8_grad_input_workspace_bytes(const fmm_int8_grad_t* p, size_t* bytes) { return grad_workspace_bytes<GRAD_X>(p, bytes); }
fmm_status_t fmm_int8_grad_weight(const fmm_int8_grad_t* p, void* workspace, size_t workspace_bytes, void* stream)
{
    return grad<GRAD_W>(p, workspace, workspace_bytes, stream);
}
fmm_status_t fmm_int8_grad_input(const fmm_int8_grad_t* p, void* workspace, size_t workspace_bytes, void* stream)
{
    return grad<GRAD_X>(p, workspace, workspace_bytes, stream);
}

fmm_status_t fmm_int8_product_shape(fmm_int8_product_t which, int64_t M, int64_t N, int64_t K, fmm_type_t out_type, fmm_int8_product_shape_t* shape)
{
    if (!shape || which < FMM_INT8_MATMUL || which > FMM_INT8_GRAD_INPUT || !int8_type_ok(out_type)) return FMM_ERR_INVALID_ARG;
    if (M <= 0 || N <= 0 || K <= 0 || (which == FMM_INT8_MATMUL ? !dim_ok(M) || !dim_ok(N) || K > 131071 : !grad_dims_ok(M, N, K))) return FMM_ERR_SHAPE;
    ProductParams p = {};
    p.out_type = out_type;
    if (which == FMM_INT8_MATMUL) {
        p.rows = (int)N; p.cols = (int)M; p.kstages = (int)ceil_div(K, 128);
        *shape = product_shape<INT8>(p, {nullptr, N, K, K}, {nullptr, M, K, K});
    } else {
        const int64_t contraction = which == FMM_INT8_GRAD_WEIGHT ? M : N;
        p.rows = (int)K; p.cols = (int)(which == FMM_INT8_GRAD_WEIGHT ? N : M); p.kstages = (int)ceil_div(contraction, 64);
        const Operand values = {nullptr, contraction, K, K}, dy = {nullptr, M, N, N};
        *shape = which == FMM_INT8_GRAD_WEIGHT ? product_shape<GRAD_W>(p, values, dy) : product_shape<GRAD_X>(p, values, dy);
    }
    return FMM_OK;
}

fmm_status_t fmm_int8_force_product_shape(const fmm_int8_product_shape_t* shape)
{
    if (!shape) { forced_shape = {}; return FMM_OK; }
    const int c = shape->columns, n = shape->k_shares;
    const bool ok = shape->kernel == SHAPE_PAIRS     ? c == 256 && n == 1
                    : shape->kernel == SHAPE_CLUSTER ? (c == 16 || c == 32 || c == 64 || c == 128) && n >= 1 && n <= 8
                                                     : shape->kernel == SHAPE_FEW && c == FEW_SHAPE_COLUMNS && n == 1;
    if (!ok) return FMM_ERR_INVALID_ARG;
    forced_shape = *shape;
    return FMM_OK;
}

fmm_status_t fmm_int8_status(int* code)
{
    if (!code) return FMM_ERR_INVALID_ARG;
    *code = 0;
    int words[3] = {0, 0, 0}, rows = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(words, g_int8_product_status, sizeof(words)) != cudaSuccess) {
        cudaGetLastError();
        return FMM_ERR_CUDA;
    }
    const fmm_status_t s = int8_rows_guard_read(&rows, false);
    if (s != FMM_OK) return s;
    *code = words[0] ? words[0] : words[2] ? words[2] : rows;
    return words[0] ? FMM_ERR_DEVICE_TIMEOUT : FMM_OK;
}

fmm_status_t fmm_int8_status_clear(void)
{
    const int zero[3] = {0, 0, 0};
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyToSymbol(g_int8_product_status, zero, sizeof(zero)) != cudaSuccess) {
        cudaGetLastError();
        return FMM_ERR_CUDA;
    }
    int unused = 0;
    return int8_rows_guard_read(&unused, true);
}

fmm_status_t fmm_int8_selftest_bounded_wait(int64_t limit_ns, void* stream)
{
    if (limit_ns < 1 || limit_ns > 2000000000) return FMM_ERR_INVALID_ARG;
    int* status = nullptr;
    if (cudaGetSymbolAddress((void**)&status, g_int8_product_status) != cudaSuccess) { cudaGetLastError(); return FMM_ERR_CUDA; }
    return fmm_launch_bounded_wait_selftest(status, (unsigned long long)limit_ns, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
