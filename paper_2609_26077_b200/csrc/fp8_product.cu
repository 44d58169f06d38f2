// Products of e4m3 codes with an fp32 scale for each block of 128 along the contraction, dense or by group:
//
//   MATMUL  out[i][j] = sum_b sa[b][i] sb[j / 128][b] (sum over block b of a[i][k] b[j][k]) + bias[j]
//   GRAD_X  out[i][k] = sum_b sa[b][i] sb[b][k / 128] (sum over block b of a[i][j] b[j][k])
//   GRAD_W  out[j][k] = sum_b sa[b][j] sb[b][k]       (sum over block b of a[i][j] b[i][k])
//
// A block's sum is one accumulation of four tcgen05 instructions (kind::f8f6f4, K = 32) into TMEM; the tensor cores cannot apply a
// factor of fp32, so it leaves TMEM after every block and is added, times its scales, to sums in registers.
//
//              A (the output's rows, TMEM lanes)          B (the output's columns)
//   MATMUL     tokens x K, K-major                        weight N x K, K-major
//   GRAD_X     dy, tokens x N, K-major                    weight N x K, contraction over its rows: MN-major
//   GRAD_W     dy, rows x N, MN-major                     x, rows x K, MN-major
//
// An operand whose contraction runs over its rows is loaded as it lies, in boxes of 128 rows x 128 bytes, and handed to the tensor cores as
// MN-major; nothing is transposed in memory.  A lane of TMEM is a row of the output: in MATMUL and GRAD_X, whose columns share one scale over 128,
// a thread has one factor for a whole block, and its sums take one multiply-add each.
#include <math.h>
#include <string.h>
#include <algorithm>
#include <type_traits>
#include "fmm_gemm_common.cuh"
#include "fp8_internal.h"

namespace {

enum Kind { MATMUL = 0, GRAD_X = 1, GRAD_W = 2 };

// [0] first bounded wait that gave up, [1] set by the self-test if its wait did not, [2] store outside its range (FMM_DEBUG build)
__device__ int g_fp8_product_status[3];

struct ProductParams {
    int rows, cols, depth;          // of the output (of all groups, or of one's: weight gradient), and of the contraction
    int groups; const int* offsets; int tokens;
    const uint8_t* a; long long lda; const float* a_scales; long long lda_scales;
    const uint8_t* b; long long ldb, step_b; const float* b_scales; long long ldb_scales;
    const void* bias;
    void* out; long long ldo, step_out;
    int out_type, accumulate;
    int by_tma;                     // the output's rows can be written by TMA
    int loose;                      // scales along rows and columns that TMA cannot load
    int shares;                     // CTAs (a cluster, single CTAs only) that share a tile's contraction; more than one: a tile to a cluster
    Int8Ranges ranges;
};

template <typename T> __device__ __forceinline__ void put_one(const ProductParams& p, long long at, float v)
{
    T* q = static_cast<T*>(p.out) + at;
    if (!INT8_STORE_OK(p.ranges, q, sizeof(T), 2602, &g_fp8_product_status[2])) return;
    if (p.accumulate) v += to_float(*q);
    *q = from_float<T>(v);
}
__device__ __forceinline__ void put(const ProductParams& p, long long at, float v)
{
    if (p.out_type == FMM_TYPE_F32) put_one<float>(p, at, v);
    else if (p.out_type == FMM_TYPE_BF16) put_one<__nv_bfloat16>(p, at, v);
    else put_one<__half>(p, at, v);
}
__device__ __forceinline__ float load_bias(const ProductParams& p, long long at)
{
    if (!p.bias) return 0.0f;
    if (p.out_type == FMM_TYPE_F32) return static_cast<const float*>(p.bias)[at];
    if (p.out_type == FMM_TYPE_BF16) return to_float(static_cast<const __nv_bfloat16*>(p.bias)[at]);
    return to_float(static_cast<const __half*>(p.bias)[at]);
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* tm)
{ asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory"); }
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* tm, int x, int y, int z, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(tm)), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
// tmem_ld_wait16 for 32 registers
__device__ __forceinline__ void tmem_ld_wait32(uint32_t* r)
{
    tmem_ld_wait16(r);
    asm volatile("" : "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                      "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]) :: "memory");
}
__device__ __forceinline__ void sts128u(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{ asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory"); }
__device__ __forceinline__ float ld_cluster32f(uint32_t addr)
{ float v; asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory"); return v; }
__device__ __forceinline__ void sts32f(uint32_t addr, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }

// sums += block's sums * factor, and += (block's sums * column scales) * row scale
__device__ __forceinline__ void add2(float& a, float& b, uint32_t va, uint32_t vb, float factor)
{ unpack2(fma2(pack2u(va, vb), pack2(factor, factor), pack2(a, b)), a, b); }
__device__ __forceinline__ void add2(float& a, float& b, uint32_t va, uint32_t vb, float fa, float fb, float row)
{ unpack2(fma2(mul2(pack2u(va, vb), pack2(fa, fb)), pack2(row, row), pack2(a, b)), a, b); }

// MN-major operand tile of 8-bit numbers, 128-byte swizzle: rows of 128 elements, 8-row groups 1024 bytes apart (one box: 128 k)
constexpr int BOX = 128 * 128;
__device__ __forceinline__ uint64_t make_mnmajor_desc(uint32_t saddr)
{
    return (uint64_t)((saddr & 0x3FFFF) >> 4) | ((uint64_t)(BOX >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
template <int KIND> constexpr bool A_MN = KIND == GRAD_W;
template <int KIND> constexpr bool B_MN = KIND != MATMUL;

// ------------------------------------------------------------------------------------------------ tiles
struct Tile {
    int group;                      // -1: there are no more
    int row0, row_end;              // first row of the tile, end of the rows that it may write
    int col0;
    int kb0, kbs;                   // blocks of the contraction
};
// The w'th tile: group by group, in a group bands of eight tiles of rows, all columns of a band before the next (the tiles in flight
// share operands in L2).  Warp-collective.
template <int KIND, int TM, int TN> __device__ __forceinline__ Tile find_tile(const ProductParams& p, unsigned w)
{
    const Tile none = {-1, 0, 0, 0, 0, 0};
    const unsigned tiles_c = (unsigned)(p.cols + TN - 1) / TN;
    Tile t;
    unsigned in = w;
    int tiles_r, rows = p.rows, first = 0;
    t.group = 0;
    t.kb0 = 0;
    t.kbs = (p.depth + 127) / 128;
    if (KIND == GRAD_W) {
        tiles_r = (p.rows + TM - 1) / TM;
        const unsigned per = (unsigned)tiles_r * tiles_c, g = w / per;
        if (g >= (unsigned)max(p.groups, 1)) return none;
        if (p.groups) {
            const Fp8Group f = fp8_find_group<false>(p.offsets, p.groups, p.tokens, 128, (int)g);
            t.kb0 = min(f.before, t.kbs);
            t.kbs = min((f.rows + 127) / 128, t.kbs - t.kb0);
            t.group = (int)g;
        }
        in = w - g * per;
    } else {
        if (p.groups) {
            const Fp8Group f = fp8_find_group<true>(p.offsets, p.groups, p.rows, TM, (int)(w / tiles_c));
            if (f.group < 0) return none;
            t.group = f.group;
            first = f.first;
            rows = f.rows;
            in = w - (unsigned)f.before * tiles_c;
        }
        tiles_r = (rows + TM - 1) / TM;
        if (in >= (unsigned)tiles_r * tiles_c) return none;
    }
    const unsigned band = 8 * tiles_c, b = in / band, n = (unsigned)min(8, tiles_r - (int)(8 * b)), rest = in - b * band, c = rest / n;
    t.row0 = first + (int)(8 * b + rest - c * n) * TM;
    t.row_end = first + rows;
    t.col0 = (int)c * TN;
    return t;
}
// Tiles found ahead of their time by a warp of its own (for a role that finds its tile when it needs it, a tile takes 1400 cycles more): a ring of them
// in shared memory.  `ready` counts that warp, `taken` the warps that read.
constexpr int TILE_RING = 4, TILE_BYTES = 32;
struct TileRing {
    uint32_t at, ready, taken;      // shared addresses
    int slot = 0; uint32_t phase = 0;
    __device__ __forceinline__ void next() { if (++slot == TILE_RING) { slot = 0; phase ^= 1u; } }
    __device__ __forceinline__ bool put(const Tile& t, const Ctl& ctl)
    {
        if (!mbar_wait_warp(taken + 8 * slot, phase ^ 1u, ctl, 2614)) return false;
        if ((threadIdx.x & 31) == 0) {
            sts128u(at + TILE_BYTES * slot, t.group, t.row0, t.row_end, t.col0);
            sts128u(at + TILE_BYTES * slot + 16, t.kb0, t.kbs, 0, 0);
            mbar_arrive(ready + 8 * slot);
        }
        __syncwarp();
        next();
        return true;
    }
    // group -1 also where the wait has run out
    __device__ __forceinline__ Tile get(const Ctl& ctl)
    {
        if (!mbar_wait_warp(ready + 8 * slot, phase, ctl, 2615)) return {-1, 0, 0, 0, 0, 0};
        const float4 a = lds128(at + TILE_BYTES * slot), b = lds128(at + TILE_BYTES * slot + 16);
        const Tile t = {__float_as_int(a.x), __float_as_int(a.y), __float_as_int(a.z), __float_as_int(a.w), __float_as_int(b.x), __float_as_int(b.y)};
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(taken + 8 * slot);
        next();
        return t;
    }
};

// ------------------------------------------------------------------------------------------------ output
// A warp's part of a tile: 32 rows from row0, of which those below row_end exist, lane r holding row r; COLS columns from col0.
//   staging  8 KB of the warp's own
// Whole rows of a 16-byte aligned output go out by TMA, which cuts off the columns behind the last; others, and those that are added to what is
// there, by stores of a row at a time, in fp32 up to there so that they are rounded once.
template <int KIND, int COLS>
__device__ __forceinline__ void put_tile(const ProductParams& p, const CUtensorMap& tm, float (&sum)[COLS], int group, int row0, int row_end, int col0, uint32_t staging)
{
    const int lane = threadIdx.x & 31;
    if (row0 >= row_end || col0 >= p.cols) return;
    // what was stored from here before has been read (by the lane that issues the stores)
    if (elect_one()) bulk_wait_read<0>();
    __syncwarp();
    if (p.bias) {
        for (int c = lane; c < COLS; c += 32) sts32f(staging + 4 * c, col0 + c < p.cols ? load_bias(p, (long long)group * p.cols + col0 + c) : 0.0f);
        __syncwarp();
#pragma unroll
        for (int c = 0; c < COLS; c += 4) {
            const float4 b = lds128(staging + 4 * c);
            sum[c] += b.x; sum[c + 1] += b.y; sum[c + 2] += b.z; sum[c + 3] += b.w;
        }
        __syncwarp();
    }
    if (p.by_tma && row0 + 32 <= row_end && COLS >= 64) {
        auto store = [&](int c, int n) {                     // chunks of 128 bytes x 32 rows, swizzled as the tensor map says
            fence_proxy_async();
            __syncwarp();
            if (elect_one()) {
#pragma unroll
                for (int i = 0; i < n; ++i) {
                    const int x = col0 + c + i * (p.out_type == FMM_TYPE_F32 ? 32 : 64);
                    if (x < p.cols) tma_store_3d(&tm, x, row0, KIND == GRAD_W ? group : 0, staging + i * 4096);
                }
                bulk_commit();
            }
        };
        const uint32_t at = staging + lane * 128, turn = lane & 7;
        if (p.out_type == FMM_TYPE_F32) {
#pragma unroll
            for (int c = 0; c < COLS; c += 64) {
                if (c > 0) { if (elect_one()) bulk_wait_read<0>(); __syncwarp(); }
#pragma unroll
                for (int j = 0; j < 64; j += 4)
                    sts128(at + j / 32 * 4096 + (((j % 32) / 4) ^ turn) * 16, make_float4(sum[c + j], sum[c + j + 1], sum[c + j + 2], sum[c + j + 3]));
                store(c, 2);
            }
        } else {
            const bool bf = p.out_type == FMM_TYPE_BF16;
#pragma unroll
            for (int c = 0; c < COLS; c += 8) {
                uint32_t v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = bf ? pack_two<__nv_bfloat16>(sum[c + 2 * j], sum[c + 2 * j + 1]) : pack_two<__half>(sum[c + 2 * j], sum[c + 2 * j + 1]);
                sts128u(at + c / 64 * 4096 + (((c % 64) / 8) ^ turn) * 16, v[0], v[1], v[2], v[3]);
            }
            store(0, COLS / 64);
        }
        return;
    }
    constexpr int PASS = COLS < 64 ? COLS : 64;
    const int rows = min(32, row_end - row0);
    const long long at = (KIND == GRAD_W ? group * p.step_out : 0) + (long long)row0 * p.ldo + col0;
    auto store = [&](auto type) {
        using T = decltype(type);
#pragma unroll
        for (int c = 0; c < COLS; c += PASS) {
#pragma unroll
            for (int j = 0; j < PASS; j += 4) sts128(staging + lane * PASS * 4 + ((j / 4) ^ (lane & 7)) * 16, make_float4(sum[c + j], sum[c + j + 1], sum[c + j + 2], sum[c + j + 3]));
            __syncwarp();
            // lane l writes columns l and l + 32 of one row after the other
            T* q = static_cast<T*>(p.out) + at + c + lane;
            const bool in0 = col0 + c + lane < p.cols, in1 = PASS == 64 && col0 + c + 32 + lane < p.cols;
            const uint32_t word = (lane & 3) * 4;
#pragma unroll 4
            for (int r = 0; r < rows; ++r, q += p.ldo) {
                const uint32_t from = staging + r * PASS * 4 + word;
                float a = lds32f(from + ((lane / 4) ^ (r & 7)) * 16), b = PASS == 64 ? lds32f(from + ((8 + lane / 4) ^ (r & 7)) * 16) : 0.0f;
                const bool w0 = in0 && INT8_STORE_OK(p.ranges, q, sizeof(T), 2601, &g_fp8_product_status[2]);
                const bool w1 = in1 && INT8_STORE_OK(p.ranges, q + 32, sizeof(T), 2601, &g_fp8_product_status[2]);
                if (p.accumulate) {
                    if (w0) a += to_float(q[0]);
                    if (w1) b += to_float(q[32]);
                }
                if (w0) q[0] = from_float<T>(a);
                if (w1) q[32] = from_float<T>(b);
            }
            __syncwarp();
        }
    };
    if (p.out_type == FMM_TYPE_F32) store(float{});
    else if (p.out_type == FMM_TYPE_BF16) store(__nv_bfloat16{});
    else store(__half{});
}

// ------------------------------------------------------------------------------------------------ kernel
// Persistent CTAs, or pairs of them (cta_group::2) that share a tile of 256 x 256: each loads its 128 rows and half of the columns.
// Bound by the way of the sums through the output warps, then by the power limit.  Cycles for a block of a pair's tile, of which the tensor pipe takes 512
// (8192 cubed, 64 blocks a tile, the tiles' output included; product, input gradient, weight gradient):
//   as it is                                                 704    697    1028
//   without the loads from TMEM                              681    696    1040
//   without the multiply-adds                                636    638     698
//   sums left in TMEM for a tile's 64 blocks                 610    609     660
//   one read of the columns' scales a block instead of 32                   904
// 16384 x 8192 x 8192: 880 us in a single call (2.50 PFLOP/s, tensor pipe 73 % of the cycles), 1040 to 1120 in a long run at
// 1.2 to 1.5 GHz; 8192 cubed 506 to 539, input gradient 479 to 525, weight gradient in fp32 647 to 693.  Larger tiles would not let a block be multiplied
// while another leaves TMEM.
// Two TMEM accumulators (narrow tiles: four): a block is multiplied while the ones before it leave TMEM.  What issues the MMAs bounds the loop before the tensor pipe
// does, so it has one barrier to wait for and one to signal for a block: `full` counts the operands of a stage and the warps that have taken the sums
// of an earlier block out of the accumulator that this one will take; `done` says to those warps that their sums are complete and their scales are there, and
// to the producer that the stage is free.  A block's scales, which those warps read and the MMAs do not, have a slot of their own, and a barrier of the CTA
// that reads them.
//   warp 0 TMA producer, warp 1 MMA issuer, warp 2 finds the tiles, warp 3 sees to the scales, warps 4 .. 11 sums and output: a TMEM lane quadrant and
//   half of the columns each
template <int KIND, int NCTA, int TN> struct Cfg {
    static constexpr int TM = 128 * NCTA, A_BYTES = 128 * 128, B_ROWS = TN / NCTA, B_BYTES = B_MN<KIND> ? BOX : B_ROWS * 128, STAGE_BYTES = A_BYTES + B_BYTES;
    static_assert(!B_MN<KIND> || B_ROWS == 128, "an MN-major box is 128 elements wide");
    static constexpr int OUT_WARPS = 8, OUT_WARP0 = 4, THREADS = (OUT_WARP0 + OUT_WARPS) * 32, COLS = TN / 2;
    // columns that a warp takes from TMEM at a time; an even number of times, as they come in two sets of registers by turns
    static constexpr int CH = COLS < 64 ? COLS / 2 : 32;
    static_assert(COLS % (2 * CH) == 0 && (CH == 16 || CH == 32), "pieces of an accumulator");
    // a warp's output on its way out (and its bias): 8 KB.  Scales of a block: of 128 rows from a multiple of four on, weight gradients: of the columns
    static constexpr int STAGING = 8192, ROW_SCALES = 132 * 4, SLOT = KIND == GRAD_W ? 640 + TN * 4 : 640, SLOTS = TN == 256 ? 8 : 12;
    static constexpr int FIXED = OUT_WARPS * STAGING + SLOTS * SLOT + 512;
    static constexpr int MOST = (232448 - 1024 - FIXED) / STAGE_BYTES, STAGES = MOST < 6 ? MOST : 6;
    static constexpr int OFF_STAGING = STAGES * STAGE_BYTES, OFF_SCALES = OFF_STAGING + OUT_WARPS * STAGING, OFF_BAR = OFF_SCALES + SLOTS * SLOT;
    static constexpr int SCALE_BYTES = ROW_SCALES + (KIND == GRAD_W ? TN * 4 : 0);        // that a CTA loads for a block
    static constexpr int NUM_BARS = 2 * STAGES + SLOTS + 2 * TILE_RING, OFF_RING = 320, SMEM_BYTES = OFF_BAR + 512 + 1024;
    // accumulators: as many as TMEM holds, four at most (the waits for one that is taken out would bound narrow tiles)
    static constexpr int BUFS = TN == 256 ? 2 : 4, TMEM_COLS = BUFS * TN;
    static_assert(BUFS <= STAGES, "operands of the block that takes an accumulator next are counted by a barrier that has come round");
    // Block b is loaded when block b - STAGES has been multiplied, for which all warps have left the accumulator of block b - STAGES - BUFS; they may be
    // at its last piece still.
    static_assert(SLOTS > STAGES + BUFS, "scales are not overwritten while they are read");
    static constexpr int REGS_AT_LAUNCH = 168, REGS_CTRL = 56, REGS_OUT = 224;
    static_assert(128 * REGS_CTRL + OUT_WARPS * 32 * REGS_OUT <= THREADS * REGS_AT_LAUNCH, "register pool");
    static_assert(SMEM_BYTES <= 232448 && NUM_BARS * 8 + 16 <= OFF_RING && OFF_RING + TILE_RING * TILE_BYTES <= 512 && STAGES >= 4, "shared memory of a block");
};

template <int KIND, int NCTA, int TN>
__global__ void __launch_bounds__(Cfg<KIND, NCTA, TN>::THREADS, 1)
fp8_product_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmOut,
                   const __grid_constant__ CUtensorMap tmRowScales, const __grid_constant__ CUtensorMap tmColScales, const __grid_constant__ ProductParams p)
{
    using C = Cfg<KIND, NCTA, TN>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - raw_addr);
    const uint32_t bar0 = base + C::OFF_BAR;
    auto bar_full = [&](int s) { return bar0 + 8u * s; };
    auto bar_done = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
    auto bar_scales = [&](int s) { return bar0 + 8u * (2 * C::STAGES + s); };
    const uint32_t bar_ring = bar0 + 8u * (2 * C::STAGES + C::SLOTS);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + C::OFF_BAR + C::NUM_BARS * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const Ctl ctl{abort_flag, g_fp8_product_status};

    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rank = NCTA == 2 ? (int)warp_uniform(cluster_ctarank()) : 0;
    const int shares = NCTA == 1 ? p.shares : 1, share = NCTA == 1 && shares > 1 ? (int)warp_uniform(cluster_ctarank()) : 0;
    const bool leader = rank == 0;
    if (warp == 2 && elect_one()) { prefetch_map(&tmA); prefetch_map(&tmB); }
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) { mbar_init(bar_full(s), 1 + NCTA * C::OUT_WARPS); mbar_init(bar_done(s), 2); }
        for (int s = 0; s < C::SLOTS; ++s) mbar_init(bar_scales(s), 1);
        // the output warps, the producer, the warp of the scales, the issuer
        for (int i = 0; i < TILE_RING; ++i) { mbar_init(bar_ring + 8u * i, 1); mbar_init(bar_ring + 8u * (TILE_RING + i), C::OUT_WARPS + 2 + leader); }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc<NCTA>(smem_u32(tmem_slot), C::TMEM_COLS);
        tmem_relinquish<NCTA>();
    }
    tc_fence_before();
    __syncthreads();
    if (NCTA == 2) cluster_sync();                           // the peer's barriers are initialised before anyone signals them
    tc_fence_after();
    const uint32_t tmem_base = warp_uniform(*tmem_slot);
    const int units = gridDim.x / (NCTA * shares), unit = blockIdx.x / (NCTA * shares);
    TileRing ring = {base + C::OFF_BAR + C::OFF_RING, bar_ring, bar_ring + 8u * TILE_RING};

    if (warp < C::OUT_WARP0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_CTRL));
    if (warp == 0) {
        int stage = 0, slot = 0; uint32_t phase = 0;
        bool ok = true;
        while (ok) {
            const Tile t = ring.get(ctl);
            if (t.group < 0) break;
            const int row = t.row0 + rank * 128, col = t.col0 + rank * C::B_ROWS;
            for (int kb = t.kb0; kb < t.kb0 + t.kbs; ++kb) {
                if (!mbar_wait_warp(bar_done(stage), phase ^ 1u, ctl, 2611)) { ok = false; break; }
                // completion of operands is counted on the even CTA's barrier; only that CTA arms it
                const uint32_t fb = NCTA == 2 ? bar_full(stage) & PEER_BIT_MASK : bar_full(stage);
                if (elect_one()) {
                    const uint32_t s = base + stage * C::STAGE_BYTES;
                    if (leader) mbar_expect_tx(bar_full(stage), NCTA * C::STAGE_BYTES);
                    tma_load_2d<NCTA>(s, &tmA, A_MN<KIND> ? row : kb * 128, A_MN<KIND> ? kb * 128 : row, fb);
                    tma_load_3d<NCTA>(s + C::A_BYTES, &tmB, B_MN<KIND> ? col : kb * 128, B_MN<KIND> ? kb * 128 : col, KIND == GRAD_W ? 0 : t.group, fb);
                    const uint32_t scales = base + C::OFF_SCALES + slot * C::SLOT;
                    if (!p.loose) {
                        mbar_expect_tx(bar_scales(slot), C::SCALE_BYTES);
                        tma_load_2d<1>(scales, &tmRowScales, row & ~3, kb, bar_scales(slot));
                        if (KIND == GRAD_W) tma_load_2d<1>(scales + 640, &tmColScales, t.col0, kb, bar_scales(slot));
                    }
                }
                if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                if (++slot == C::SLOTS) slot = 0;
            }
        }
    } else if (warp == 1) {
        if (leader) {
            int stage = 0, buf = 0; uint32_t phase = 0;
            // fp32 sums of e4m3 operands
            const uint32_t idesc = (1u << 4) | ((A_MN<KIND> ? 1u : 0u) << 15) | ((B_MN<KIND> ? 1u : 0u) << 16) | ((uint32_t)(TN >> 3) << 17) | ((uint32_t)(C::TM >> 4) << 24);
            constexpr int ASTEP = A_MN<KIND> ? 4096 >> 4 : 32 >> 4, BSTEP = B_MN<KIND> ? 4096 >> 4 : 32 >> 4;
            bool ok = true;
            while (ok) {
                const Tile t = ring.get(ctl);
                if (t.group < 0) break;
                for (int kb = 0; kb < t.kbs; ++kb) {
                    if (!mbar_wait_warp(bar_full(stage), phase, ctl, 2612)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t s = base + stage * C::STAGE_BYTES;
                    const uint64_t ad = A_MN<KIND> ? make_mnmajor_desc(s) : make_kmajor_sw128_desc(s);
                    const uint64_t bd = B_MN<KIND> ? make_mnmajor_desc(s + C::A_BYTES) : make_kmajor_sw128_desc(s + C::A_BYTES);
#pragma unroll
                    for (int j = 0; j < 4; ++j) mma_f8f6f4<NCTA>(tmem_base + buf * TN, ad + ASTEP * j, bd + BSTEP * j, idesc, j > 0 ? 1u : 0u);
                    tc_commit<NCTA>(bar_done(stage));
                    if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                    if (++buf == C::BUFS) buf = 0;
                }
            }
        }
    } else if (warp == 2) {
        for (unsigned w = unit;; w += units) {
            Tile t = find_tile<KIND, C::TM, TN>(p, w);
            if (NCTA == 1 && shares > 1 && t.group >= 0) {
                const int from = (int)((long long)t.kbs * share / shares), to = (int)((long long)t.kbs * (share + 1) / shares);
                t.kb0 += from;
                t.kbs = to - from;
            }
            if (!ring.put(t, ctl) || t.group < 0) break;
        }
    } else {
        // A block's scales are there: said to the output warps by an arrival of this warp, which has seen it, beside that of the MMAs, which says nothing of
        // what TMA has copied.  (A wait of each output warp for its scales costs a tenth of the time: 4096 cubed 70 to 76 us instead of 64 to 68.)  Scales
        // that TMA cannot load come by way of this warp's registers (4096 cubed 71 us instead of 68, 8192 cubed 528 instead of 522, weight gradient 709
        // instead of 672); beyond the last row or column: 0, as by TMA.
        int stage = 0, slot = 0; uint32_t phase = 0, slot_phase = 0;
        bool ok = true;
        while (ok) {
            const Tile t = ring.get(ctl);
            if (t.group < 0) break;
            const int row = t.row0 + rank * 128;
            for (int kb = t.kb0; kb < t.kb0 + t.kbs; ++kb) {
                if (p.loose) {
                    const float *rows_from = p.a_scales + kb * p.lda_scales + row + lane, *cols_from = p.b_scales + kb * p.ldb_scales + t.col0 + lane;
                    float r[4] = {}, c[TN / 32] = {};
#pragma unroll
                    for (int i = 0; i < 4; ++i) if (row + 32 * i + lane < p.rows) r[i] = __ldg(rows_from + 32 * i);
                    if (KIND == GRAD_W) {
#pragma unroll
                        for (int i = 0; i < TN / 32; ++i) if (t.col0 + 32 * i + lane < p.cols) c[i] = __ldg(cols_from + 32 * i);
                    }
                    if (!mbar_wait_warp(bar_done(stage), phase ^ 1u, ctl, 2617)) { ok = false; break; }
                    const uint32_t to = base + C::OFF_SCALES + slot * C::SLOT + 4 * lane;
#pragma unroll
                    for (int i = 0; i < 4; ++i) sts32f(to + ((row & 3) + 32 * i) * 4, r[i]);
                    if (KIND == GRAD_W) {
#pragma unroll
                        for (int i = 0; i < TN / 32; ++i) sts32f(to + 640 + 128 * i, c[i]);
                    }
                    __syncwarp();
                } else if (!mbar_wait_warp(bar_scales(slot), slot_phase, ctl, 2616)) { ok = false; break; }
                if (elect_one()) mbar_arrive(bar_done(stage));
                if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                if (++slot == C::SLOTS) { slot = 0; slot_phase ^= 1u; }
            }
        }
    }
    if (NCTA == 1 && shares > 1) { __syncwarp(); cluster_sync(); cluster_sync(); }        // as the output warps below
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::REGS_OUT));
        constexpr int COLS = C::COLS, CH = C::CH;
        const int quadrant = warp & 3, half = (warp - C::OUT_WARP0) >> 2;
        const uint32_t lane_taddr = tmem_base + half * COLS + ((uint32_t)(quadrant * 32) << 16);
        const uint32_t staging = base + C::OFF_STAGING + (warp - C::OUT_WARP0) * C::STAGING;
        int stage = 0, buf = 0, ahead = C::BUFS % C::STAGES; uint32_t phase = 0;          // ahead: stage of the block that takes this one's accumulator next
        bool ok = true;
        auto release = [&](int s) {
            if (lane == 0) { if (NCTA == 2) mbar_arrive_cluster(bar_full(s) & PEER_BIT_MASK); else mbar_arrive(bar_full(s)); }
        };
#pragma unroll
        for (int b = 0; b < C::BUFS; ++b) release(b);
        // The columns' scale of MATMUL and GRAD_X, one for each block: 32 blocks' in the lanes, the next 32's on their way.  (The rows', and the weight
        // gradient's columns', come with the operands: asked for by these warps, a block or two ahead, they cost 100 cycles a block.)
        float scales_now = 0.0f, scales_next = 0.0f;
        auto fetch = [&](const Tile& t, int kb) -> float {
            if (KIND == GRAD_W || t.group < 0 || kb + lane >= t.kbs) return 0.0f;
            const long long blocks_c = (p.cols + 127) / 128, c = min((t.col0 + half * COLS) / 128, (int)blocks_c - 1), all = (p.depth + 127) / 128, b = t.kb0 + kb + lane;
            return __ldg(p.b_scales + t.group * blocks_c * all + (KIND == MATMUL ? c * all + b : b * blocks_c + c));
        };
        int slot = 0;
        Tile t = ring.get(ctl);
        scales_now = fetch(t, 0);
        float sum[COLS];
        while (t.group >= 0) {
#pragma unroll
            for (int c = 0; c < COLS; ++c) sum[c] = 0.0f;
            const uint32_t row_at = (((t.row0 + rank * 128) & 3) + quadrant * 32 + lane) * 4;
            // The next piece of an accumulator is on its way from TMEM while this one is added, also from one block to the next.  (Alone, eight
            // warps take 128 columns in 83 cycles this way, with their multiply-adds in 274 of 256; tcgen05.ld.16x256b takes 520.)
            uint32_t v[2][CH];
            auto load = [&](uint32_t (&r)[CH], int c) {
                tmem_ld16(lane_taddr + buf * TN + c, r);
                if constexpr (CH == 32) tmem_ld16(lane_taddr + buf * TN + c + 16, r + 16);
            };
            auto arrived = [&](uint32_t (&r)[CH]) {
                if constexpr (CH == 32) tmem_ld_wait32(r); else tmem_ld_wait16(r);
            };
            if (t.kbs > 0) {
                if (!mbar_wait_warp(bar_done(stage), phase, ctl, 2613)) { ok = false; break; }
                tc_fence_after();
                load(v[0], 0);
            }
            for (int kb = 0; kb < t.kbs; ++kb) {
                if (KIND != GRAD_W && (kb & 31) == 0) {
                    if (kb) scales_now = scales_next;
                    scales_next = fetch(t, kb + 32);
                }
                const uint32_t cols_at = base + C::OFF_SCALES + slot * C::SLOT + 640 + half * COLS * 4;
                const float row_scale = lds32f(base + C::OFF_SCALES + slot * C::SLOT + row_at);
                const float factor = KIND == GRAD_W ? 0.0f : row_scale * __shfl_sync(0xffffffffu, scales_now, kb & 31);
                if (++slot == C::SLOTS) slot = 0;
#pragma unroll
                for (int i = 0; i < COLS / CH; ++i) {
                    uint32_t (&now)[CH] = v[i & 1], (&then)[CH] = v[(i + 1) & 1];
                    arrived(now);
                    if (i + 1 < COLS / CH) load(then, (i + 1) * CH);
                    else {
                        tc_fence_before();
                        __syncwarp();
                        release(ahead);
                        if (++ahead == C::STAGES) ahead = 0;
                        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                        if (++buf == C::BUFS) buf = 0;
                        if (kb + 1 < t.kbs) {
                            if (!mbar_wait_warp(bar_done(stage), phase, ctl, 2613)) { ok = false; break; }
                            tc_fence_after();
                            load(then, 0);
                        }
                    }
                    const int c = i * CH;
                    if (KIND == GRAD_W) {
#pragma unroll
                        for (int j = 0; j < CH; j += 4) {
                            const float4 f = lds128(cols_at + 4 * (c + j));
                            add2(sum[c + j], sum[c + j + 1], now[j], now[j + 1], f.x, f.y, row_scale);
                            add2(sum[c + j + 2], sum[c + j + 3], now[j + 2], now[j + 3], f.z, f.w, row_scale);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < CH; j += 2) add2(sum[c + j], sum[c + j + 1], now[j], now[j + 1], factor);
                    }
                }
                if (!ok) break;
            }
            if (!ok || (NCTA == 1 && shares > 1)) break;
            const Tile next = ring.get(ctl);
            scales_now = fetch(next, 0);
            put_tile<KIND, COLS>(p, tmOut, sum, t.group, t.row0 + rank * 128 + quadrant * 32, t.row_end, t.col0 + half * COLS, staging);
            t = next;
        }
        if constexpr (NCTA == 1) {
            // The shares meet in distributed shared memory, over the operands (this CTA's MMAs have read them all), and are added in ascending order.
            if (shares > 1) {
                const int row = quadrant * 32 + lane;
                const bool mine = t.group >= 0 && t.row0 + quadrant * 32 < t.row_end;
                const uint32_t at = base + (half * COLS * 128 + row) * 4;
                if (share > 0 && mine) {
#pragma unroll
                    for (int c = 0; c < COLS; ++c) sts32f(at + c * 512, sum[c]);
                }
                __syncwarp();
                cluster_sync();
                if (share == 0 && mine && ok) {
                    for (int other = 1; other < shares; ++other) {
                        const uint32_t from = map_to_cta(at, (uint32_t)other);
#pragma unroll
                        for (int c = 0; c < COLS; c += 16) {
                            float f[16];
#pragma unroll
                            for (int j = 0; j < 16; ++j) f[j] = ld_cluster32f(from + (c + j) * 512);
#pragma unroll
                            for (int j = 0; j < 16; ++j) sum[c + j] += f[j];
                        }
                    }
                    put_tile<KIND, COLS>(p, tmOut, sum, t.group, t.row0 + quadrant * 32, t.row_end, t.col0 + half * COLS, staging);
                }
                __syncwarp();
                cluster_sync();
            }
        }
        __syncwarp();
        if (elect_one()) bulk_wait<0>();
    }
    // ---------------------------------------------------------------------- teardown
    __syncwarp();
    if (*abort_flag) {
        // let copies that are still in flight towards this CTA's shared memory land
        const uint64_t t0 = global_timer();
        while (global_timer() - t0 < 200000ull) __nanosleep(1000);
    }
    tc_fence_before();
    // (with release and acquire: what the odd CTA has signalled of the last blocks has arrived before the even one leaves)
    if (NCTA == 2) cluster_sync(); else __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc<NCTA>(tmem_base, C::TMEM_COLS);
    }
}

// ------------------------------------------------------------------------------------------------ few tokens
// MATMUL of few tokens, dense or by group: the weight's way from memory bounds it, and this kernel has nothing to set up.  A block takes 16 output
// channels of a group, its warps share the blocks of K.  The weight goes from global memory straight into the A fragments of mma.m16n8k32, the
// tokens into the B fragments: a lane loads 2 x 16 codes of channel lane / 4, of channel lane / 4 + 8 and of token lane / 4, all at the same places of
// K, eight of each for one of the four instructions of a block - both sides number the contraction alike, so any numbering will do.
// NT x 8 tokens at a time.  1 x 8192 x 8192 in 15.2 us (4.4 TB/s), 64 experts x 128 rows x 2048 x 4096 in 75 (5.9).  (The weight by way of
// shared memory, three blocks ahead of each warp: 1.7 and 10 us more.)
constexpr int FEW_CHANNELS = 16;

__device__ __forceinline__ void mma_e4m3(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 bytes of a weight, which is read once: not kept in L1, 256 bytes brought into L2
__device__ __forceinline__ uint4 load_once(const uint8_t* p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// the first `left` of 16 codes, zeros behind them (what lies behind the last column may be anything)
__device__ __forceinline__ void cut(uint4& u, int left)
{
    uint32_t* y = &u.x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = left - 4 * j;
        y[j] = n >= 4 ? y[j] : n <= 0 ? 0u : y[j] & ((1u << (8 * n)) - 1u);
    }
}

template <int WARPS, int NT> __global__ void __launch_bounds__(WARPS * 32, (NT == 1 ? 32 : 24) / WARPS) fp8_few_kernel(const __grid_constant__ ProductParams p)
{
    __shared__ float meet[WARPS][8 * NT][FEW_CHANNELS + 1];
    const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3, group = blockIdx.y;
    int first = 0, rows = p.rows;
    if (p.groups) {
        const Fp8Group f = fp8_find_group<false>(p.offsets, p.groups, p.rows, 1, group);
        first = f.first; rows = f.rows;
    }
    const int n0 = blockIdx.x * FEW_CHANNELS, channels = min(FEW_CHANNELS, p.cols - n0), blocks = (p.depth + 127) / 128;
    const float* w_scales = p.b_scales + ((long long)group * ((p.cols + 127) / 128) + n0 / 128) * blocks;
    const bool some0 = g < channels, some1 = g + 8 < channels;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    // a pointer that moves on is 6 % faster than one sum a load (15.8 us), but takes registers that two sets of tokens do not leave
    constexpr bool MOVING = NT == 1;
#pragma unroll 1
    for (int t0 = 0; t0 < rows; t0 += 8 * NT) {
        const uint8_t *w0 = p.b + group * p.step_b + (long long)(n0 + g) * p.ldb + 16 * q + (MOVING ? warp * 128 : 0), *x0[NT];
        // (a lane without a token takes the last one's; what comes of it goes nowhere)
#pragma unroll
        for (int n = 0; n < NT; ++n) x0[n] = p.a + (long long)(first + min(t0 + 8 * n + g, rows - 1)) * p.lda + 16 * q;
        float sum[NT][4] = {};
        // Scales of a block: of the tokens in the first lanes, of the weight in the others, one load (with three 0.8 us more for one token, 8192 x 8192)
        constexpr int TOKENS = 8 * NT;
        const bool token = lane < TOKENS;
        const int scale_step = token ? (int)p.lda_scales : 1;          // (launch_few: below 2^31)
        const float* scale_at = token ? p.a_scales + first + t0 + min(lane, rows - t0 - 1) : w_scales;
#pragma unroll 1
        for (int kb = warp; kb < blocks; kb += WARPS) {
            const float scales = __ldg(scale_at + (long long)kb * scale_step);
            const int left = p.depth - kb * 128 - 16 * q;    // codes of the row from the lane's first on
            uint4 u[2], v[2], x[NT][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool in = left > 64 * i;
                u[i] = in && some0 ? load_once(w0 + ((MOVING ? 0 : kb * 128) + 64 * i)) : zero;
                v[i] = in && some1 ? load_once(w0 + 8 * p.ldb + ((MOVING ? 0 : kb * 128) + 64 * i)) : zero;
#pragma unroll
                for (int n = 0; n < NT; ++n) x[n][i] = in ? __ldg(reinterpret_cast<const uint4*>(x0[n] + (kb * 128 + 64 * i))) : zero;
            }
            float part[NT][4] = {};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (left < 64 * i + 16) {
                    cut(u[i], left - 64 * i);
                    cut(v[i], left - 64 * i);
#pragma unroll
                    for (int n = 0; n < NT; ++n) cut(x[n][i], left - 64 * i);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mma_e4m3(part[n], u[i].x, v[i].x, u[i].y, v[i].y, x[n][i].x, x[n][i].y);
                    mma_e4m3(part[n], u[i].z, v[i].z, u[i].w, v[i].w, x[n][i].z, x[n][i].w);
                }
            }
            if (MOVING) w0 += WARPS * 128;
            const float ws = __shfl_sync(0xffffffffu, scales, TOKENS);
            float xs[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) xs[n][i] = __shfl_sync(0xffffffffu, scales, 8 * n + 2 * q + i);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[n][i] = fmaf(part[n][i], xs[n][i & 1] * ws, sum[n][i]);
        }
        // channels g and g + 8 of tokens 2q and 2q + 1
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            meet[warp][8 * n + 2 * q][g] = sum[n][0];
            meet[warp][8 * n + 2 * q + 1][g] = sum[n][1];
            meet[warp][8 * n + 2 * q][g + 8] = sum[n][2];
            meet[warp][8 * n + 2 * q + 1][g + 8] = sum[n][3];
        }
        __syncthreads();
#pragma unroll 1
        for (int i = threadIdx.x; i < 8 * NT * FEW_CHANNELS; i += WARPS * 32) {
            const int c = i % FEW_CHANNELS, t = i / FEW_CHANNELS;
            if (t0 + t < rows && c < channels) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < WARPS; ++w) s += meet[w][t][c];
                put(p, (long long)(first + t0 + t) * p.ldo + n0 + c, s + load_bias(p, (long long)group * p.cols + n0 + c));
            }
        }
        __syncthreads();
    }
}

// An empty contraction: bias, or 0
__global__ void __launch_bounds__(256) fp8_empty_kernel(const ProductParams p)
{
    for (int i = blockIdx.x; i < p.rows; i += gridDim.x) {
        int group = 0;
        if (p.groups) {
            group = -1;
            int start = min(max(p.offsets[0], 0), p.rows);
            for (int g = 0; g < p.groups; ++g) {
                const int end = min(max(p.offsets[g + 1], start), p.rows);
                if (i >= start && i < end) { group = g; break; }
                start = end;
            }
            if (group < 0) continue;
        }
        for (int j = threadIdx.x; j < p.cols; j += 256) put(p, blockIdx.y * p.step_out + i * p.ldo + j, load_bias(p, (long long)group * p.cols + j));
    }
}

// ------------------------------------------------------------------------------------------------ host side
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool dim_ok(int64_t n) { return n >= 0 && n < INT8_MAX_DIM; }

bool make_map_3d(CUtensorMap* tm, CUtensorMapDataType dt, int64_t e, const void* ptr, int64_t x, int64_t y, int64_t z, int64_t ld, int64_t step, uint32_t box_x, uint32_t box_y)
{
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)x, (cuuint64_t)y, (cuuint64_t)z};
    const cuuint64_t strides[2] = {(cuuint64_t)(ld * e), (cuuint64_t)((z > 1 ? step : ld) * e)};
    const cuuint32_t box[3] = {box_x, box_y, 1}, steps[3] = {1, 1, 1};
    return fn(tm, dt, 3, const_cast<void*>(ptr), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
// tiles that a call has at most (the groups' sizes are on the device)
template <int KIND> int64_t most_tiles(const ProductParams& p, int tm, int tn)
{
    const int64_t tiles_c = ceil_div(p.cols, tn), tiles_r = ceil_div(p.rows, tm);
    if (KIND == GRAD_W) return tiles_r * tiles_c * std::max(p.groups, 1);
    return (p.groups ? std::min<int64_t>(p.rows, p.rows / tm + p.groups) : tiles_r) * tiles_c;
}
template <int KIND, int NCTA, int TN> fmm_status_t launch_tiles(ProductParams p, int shares, cudaStream_t st)
{
    using C = Cfg<KIND, NCTA, TN>;
    static std::atomic<bool> done[64];
    CUtensorMap tmA, tmB, tmOut, tmRowScales, tmColScales;
    const int64_t groups = std::max(p.groups, 1), e = int8_type_bytes((fmm_type_t)p.out_type);
    const CUtensorMapDataType codes = CU_TENSOR_MAP_DATA_TYPE_UINT8;
    const int64_t a_x = KIND == GRAD_W ? p.rows : p.depth, a_y = KIND == GRAD_W ? p.depth : p.rows;
    const int64_t b_x = KIND == MATMUL ? p.depth : p.cols, b_y = KIND == MATMUL ? p.cols : p.depth;
    bool ok = make_map_2d(&tmA, codes, 1, p.a, (uint64_t)a_x, (uint64_t)a_y, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B, (uint64_t)p.lda) &&
              make_map_3d(&tmB, codes, 1, p.b, b_x, b_y, KIND == GRAD_W ? 1 : groups, p.ldb, p.step_b, 128, B_MN<KIND> ? 128 : C::B_ROWS) &&
              raise_smem(fp8_product_kernel<KIND, NCTA, TN>, C::SMEM_BYTES, done);
    if (!p.loose)
        ok = ok && make_map_2d(&tmRowScales, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, p.a_scales, (uint64_t)p.rows, (uint64_t)ceil_div(p.depth, 128), 132, 1, CU_TENSOR_MAP_SWIZZLE_NONE, (uint64_t)p.lda_scales);
    else memset(&tmRowScales, 0, sizeof(tmRowScales));
    if (KIND == GRAD_W && !p.loose)
        ok = ok && make_map_2d(&tmColScales, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, p.b_scales, (uint64_t)p.cols, (uint64_t)ceil_div(p.depth, 128), TN, 1, CU_TENSOR_MAP_SWIZZLE_NONE, (uint64_t)p.ldb_scales);
    else memset(&tmColScales, 0, sizeof(tmColScales));
    p.by_tma = !p.accumulate && int8_aligned(p.out, p.ldo * e, 16) && ((p.step_out * e) & 15) == 0;
#ifdef FMM_DEBUG
    p.by_tma = 0;                                            // every store is checked
#endif
    if (p.by_tma)
        ok = ok && make_map_3d(&tmOut, e == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, e, p.out, p.cols, p.rows, KIND == GRAD_W ? groups : 1, p.ldo, p.step_out,
                               (uint32_t)(128 / e), 32);
    else memset(&tmOut, 0, sizeof(tmOut));
    if (!ok) return FMM_ERR_CUDA;
    // as few units as finish in the same number of waves
    const int64_t tiles = most_tiles<KIND>(p, C::TM, TN);
    if (tiles > 0x7FFFFFFF - 65536) return FMM_ERR_SHAPE;    // (more than an output that memory holds can have)
    const int64_t most = std::max(1, int8_sm_count() / NCTA), waves = ceil_div(tiles, most);
    if (shares > 1 && (NCTA == 2 || tiles * shares > 0x7FFFFFFF)) return FMM_ERR_SHAPE;
    p.shares = shares;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)(shares > 1 ? tiles * shares : (p.groups ? std::min(tiles, most) : ceil_div(tiles, waves)) * NCTA));
    cfg.blockDim = dim3(C::THREADS); cfg.dynamicSmemBytes = C::SMEM_BYTES; cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)(NCTA * shares); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = NCTA * shares > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, fp8_product_kernel<KIND, NCTA, TN>, tmA, tmB, tmOut, tmRowScales, tmColScales, p) != cudaSuccess) { cudaGetLastError(); return FMM_ERR_CUDA; }
    return FMM_OK;
}
fmm_status_t launch_few(const ProductParams& p, cudaStream_t st)
{
    if (p.lda_scales > 0x7FFFFFFF) return FMM_ERR_SHAPE;     // (only where it is forced)
    const int groups = std::max(p.groups, 1);
    const int64_t blocks = ceil_div(p.cols, FEW_CHANNELS) * groups;
    const dim3 grid((unsigned)ceil_div(p.cols, FEW_CHANNELS), (unsigned)groups);
    // as many warps to a block as let one wave hold all blocks: 16, 8, or else four (64 x 128 x 2048 x 4096 83 us, with eight 89; 1 x 8192 x 8192 with
    // eight 16.4, with four 20.4, as measured before other steps); 16 tokens at a time where there are more than eight
    const bool many = p.groups == 0 && p.rows > 8;
    if (blocks <= 2 * int8_sm_count()) { if (many) fp8_few_kernel<16, 2><<<grid, 512, 0, st>>>(p); else fp8_few_kernel<16, 1><<<grid, 512, 0, st>>>(p); }
    else if (blocks <= 4 * int8_sm_count()) { if (many) fp8_few_kernel<8, 2><<<grid, 256, 0, st>>>(p); else fp8_few_kernel<8, 1><<<grid, 256, 0, st>>>(p); }
    else if (many) fp8_few_kernel<4, 2><<<grid, 128, 0, st>>>(p);
    else fp8_few_kernel<4, 1><<<grid, 128, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? FMM_OK : FMM_ERR_CUDA;
}

// A tile's columns (FEW: the kernel for few tokens) and the CTAs that share its contraction; columns 0: none
struct Shape { int columns, shares; };
// what fmm_fp8_force_tile set for this host thread
thread_local Shape forced_shape;
constexpr int FEW = 8, MOST_SHARES = 4;

// Time of a tile shape in microseconds: the launch, and waves of tiles that take `stage` for each block of the contraction and what their output takes
// beside the next tile's blocks: 16-bit numbers and fp32 ones that go out by TMA, and rows that it cannot write.  Fitted to 34000 calls (1 to 16384
// tokens, 64 to 8192 channels, dense and of 2 to 64 groups, whose tiles are counted as if they were alike; weights that L2 does not hold), before the
// scales had a warp of their own.  On 36000 other calls of each kind since then the choice takes 2.4 % (input gradient 1.2 %, weight gradient 1.3 %) more time
// than the fastest of all shapes in the mean, at worst 2.1 times (1.6, 1.8); pairs wherever their tiles fill a third of the device took 5 to 8 % more.
struct TileModel { int columns; float lat, stage, out[3]; };
template <int KIND> constexpr TileModel TILES[3] = {};
template <> constexpr TileModel TILES<MATMUL>[3] = {{256, 4.28f, 0.383f, {1.8f, 2.8f, 3.9f}}, {128, 3.68f, 0.271f, {1.1f, 1.5f, 2.05f}}, {64, 3.50f, 0.187f, {1.4f, 1.6f, 1.8f}}};
template <> constexpr TileModel TILES<GRAD_X>[3] = {{256, 4.41f, 0.383f, {1.6f, 2.6f, 3.8f}}, {128, 3.90f, 0.302f, {0.85f, 1.25f, 2.0f}}, {0, 0, 0, {}}};
template <> constexpr TileModel TILES<GRAD_W>[3] = {{256, 5.13f, 0.550f, {1.45f, 2.55f, 3.6f}}, {128, 4.55f, 0.400f, {0.85f, 1.3f, 1.95f}}, {0, 0, 0, {}}};
// Two or four CTAs that share a contraction: for the exchange, and for the sums of 128 x 128 that the first of them fetches (fitted to 8100 calls; with
// 32 blocks and more they take 0.65 to 0.8 of the time of one).
struct ShareModel { int shares; float lat, sums; };
constexpr ShareModel SHARES[2] = {{2, 0.76f, 2.31f}, {4, 0.95f, 4.93f}};
template <int KIND> Shape choose_shape(const ProductParams& p)
{
    if (forced_shape.columns) return forced_shape;
    // The kernel for few tokens takes 0.5 to 0.75 of the best tiles' time with up to eight tokens, 0.65 with 16 (8192 x 8192: 23.6 us, by tiles 18.6), 0.9
    // to 1.6 with 32.  By group, where all have about as many rows: 0.6 to 0.9 with up to four to a group, with eight 0.75 to 0.9 for small weights (of many
    // groups at worst 2.4, hence 16 of them at most) and 1.05 to 1.2 for large ones.  How the rows are distributed is known on the device alone.  A group's
    // blocks walk over its rows eight at a time and read its weight again for each eight, so that rows which all go to one group take many times as long as
    // by tiles: 64 groups of 2048 x 4096, 128 rows 74 us (by tiles 11), 256 rows 144 (11); 1024 groups of 512 x 512, 4096 rows 392 (22).
    const int64_t weights = (int64_t)std::max(p.groups, 1) * p.cols * p.depth;
    if (KIND == MATMUL && p.lda_scales <= 0x7FFFFFFF && (p.groups ? p.rows <= (weights <= 1 << 24 && p.groups <= 16 ? 8 : 4) * (int64_t)p.groups : p.rows <= 8 || (p.rows <= 16 && weights <= 1 << 25))) return {FEW, 1};
    const float groups = (float)std::max(p.groups, 1);
    const int e = int8_type_bytes((fmm_type_t)p.out_type), out = p.accumulate || !int8_aligned(p.out, p.ldo * e, 16) || ((p.step_out * e) & 15) ? 2 : e == 4;
    Shape best = {};
    float least = 0.0f;
    for (const TileModel& m : TILES<KIND>) {
        if (!m.columns) break;
        const int tm = m.columns == 256 ? 256 : 128, units = std::max(1, int8_sm_count() / (m.columns == 256 ? 2 : 1));
        float rows = (float)ceil_div(p.rows, tm), blocks = (float)ceil_div(p.depth, 128);
        if (KIND == GRAD_W) {
            rows *= groups;
            if (p.groups) blocks = blocks / groups + 0.5f;
        } else if (p.groups) {
            const float each = (float)p.rows / groups;
            rows = std::min((float)p.rows, each < 0.5f * tm ? groups * std::min(1.0f, each) : (float)p.rows / tm + 0.5f * groups);
        }
        const float waves = std::max(1.0f, ceilf(rows * (float)ceil_div(p.cols, m.columns) / units)), time = m.lat + waves * (blocks * m.stage + m.out[out]);
        if (!best.columns || time < least) { best = {m.columns, 1}; least = time; }
        // where the device holds all clusters at once (of four: with 128 of 148 SMs, as a cluster lies in one GPC)
        for (const ShareModel& n : SHARES) {
            if (m.columns == 256 || most_tiles<KIND>(p, tm, m.columns) * n.shares > (n.shares == 4 ? units * 7 / 8 : units) || blocks < 2.0f * n.shares) break;
            const float each = KIND != GRAD_W && p.groups ? (float)p.rows / groups : (float)p.rows, quarters = std::min(4.0f, ceilf(each / 32.0f)) * 0.25f;
            const float shared = m.lat + ceilf(blocks / n.shares) * m.stage + m.out[out] + n.lat + quarters * n.sums * m.columns / 128.0f;
            if (shared < least) { best = {m.columns, n.shares}; least = shared; }
        }
    }
    return best;
}
template <int KIND> fmm_status_t launch_product(const ProductParams& p, cudaStream_t st)
{
    const Shape c = choose_shape<KIND>(p);
    if (c.columns == 256) return launch_tiles<KIND, 2, 256>(p, c.shares, st);
    if (c.columns == 128) return launch_tiles<KIND, 1, 128>(p, c.shares, st);
    if constexpr (KIND == MATMUL) return c.columns == 64 ? launch_tiles<KIND, 1, 64>(p, c.shares, st) : c.shares == 1 ? launch_few(p, st) : FMM_ERR_SHAPE;
    return FMM_ERR_SHAPE;
}

template <int KIND> fmm_status_t product(const fmm_fp8_product_t* a, void* stream)
{
    if (!a || !int8_type_ok(a->type)) return FMM_ERR_INVALID_ARG;
    const int64_t M = a->M, N = a->N, K = a->K, groups = a->groups, count = groups ? groups : 1;
    if (!dim_ok(M) || !dim_ok(N) || !dim_ok(K) || groups < 0 || groups > FMM_FP8_MAX_GROUPS || (KIND == GRAD_W && M % 128)) return FMM_ERR_SHAPE;
    if (KIND == GRAD_W && groups && (a->tokens < 0 || a->tokens > M)) return FMM_ERR_SHAPE;
    const int64_t rows = KIND == GRAD_W ? N : M, cols = KIND == MATMUL ? N : K, depth = KIND == MATMUL ? K : KIND == GRAD_X ? N : M;
    if (rows == 0 || cols == 0) return FMM_OK;
    const int64_t e = int8_type_bytes(a->type);
    if (!a->out || a->ldo < cols || (((uintptr_t)a->out | (uintptr_t)a->bias) & (e - 1)) || (a->bias && KIND != MATMUL)) return FMM_ERR_INVALID_ARG;
    if (groups && (!a->offsets || ((uintptr_t)a->offsets & 3))) return FMM_ERR_INVALID_ARG;
    if (KIND == GRAD_W && count > 1 && a->step_out < (rows - 1) * a->ldo + cols) return FMM_ERR_INVALID_ARG;
    if (depth) {
        const int64_t a_cols = KIND == MATMUL ? K : N, b_rows = KIND == GRAD_W ? M : N;
        if (!a->a || a->lda < a_cols || !int8_aligned(a->a, a->lda, 16) || !a->b || a->ldb < K || !int8_aligned(a->b, a->ldb, 16) || !a->a_scales || !a->b_scales ||
            a->lda_scales < (KIND == GRAD_W ? N : M) || !int8_aligned(a->a_scales, a->lda_scales * 4, a->loose ? 4 : 16)) return FMM_ERR_INVALID_ARG;
        if (KIND == GRAD_W ? a->ldb_scales < K || !int8_aligned(a->b_scales, a->ldb_scales * 4, a->loose ? 4 : 16) : ((uintptr_t)a->b_scales & 3) != 0) return FMM_ERR_INVALID_ARG;
        if (KIND != GRAD_W && count > 1 && (a->step_b < (b_rows - 1) * a->ldb + K || (a->step_b & 15))) return FMM_ERR_INVALID_ARG;
    }
    ProductParams p = {};
    p.rows = (int)rows; p.cols = (int)cols; p.depth = (int)depth;
    p.groups = (int)groups; p.offsets = a->offsets; p.tokens = (int)(KIND == GRAD_W && a->tokens ? a->tokens : M);
    p.a = a->a; p.lda = a->lda; p.a_scales = a->a_scales; p.lda_scales = a->lda_scales;
    p.b = a->b; p.ldb = a->ldb; p.step_b = KIND != GRAD_W && count > 1 ? a->step_b : 0; p.b_scales = a->b_scales; p.ldb_scales = a->ldb_scales;
    p.bias = a->bias; p.out = a->out; p.ldo = a->ldo; p.step_out = KIND == GRAD_W && count > 1 ? a->step_out : 0;
    p.out_type = a->type; p.accumulate = a->accumulate != 0; p.loose = a->loose != 0;
    if (KIND == GRAD_W) int8_add_range(p.ranges, a->out, 1, (count - 1) * p.step_out + (rows - 1) * a->ldo + cols, 0, e);
    else int8_add_range(p.ranges, a->out, rows, cols, a->ldo, e);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (depth == 0) {
        if (p.accumulate && !p.bias) return FMM_OK;
        if (KIND == GRAD_W) p.groups = 0;                    // no row in any group
        fp8_empty_kernel<<<dim3((unsigned)std::min<int64_t>(rows, 8 * int8_sm_count()), KIND == GRAD_W ? (unsigned)count : 1u), 256, 0, st>>>(p);
        return cudaGetLastError() == cudaSuccess ? FMM_OK : FMM_ERR_CUDA;
    }
    return launch_product<KIND>(p, st);
}

}  // namespace

extern "C" {

fmm_status_t fmm_fp8_matmul(const fmm_fp8_product_t* p, void* stream) { return product<MATMUL>(p, stream); }
fmm_status_t fmm_fp8_grad_input(const fmm_fp8_product_t* p, void* stream) { return product<GRAD_X>(p, stream); }
fmm_status_t fmm_fp8_grad_weight(const fmm_fp8_product_t* p, void* stream) { return product<GRAD_W>(p, stream); }

fmm_status_t fmm_fp8_force_tile(int columns, int shares)
{
    if (columns != 0 && columns != FEW && columns != 64 && columns != 128 && columns != 256) return FMM_ERR_INVALID_ARG;
    if (shares < 1 || shares > MOST_SHARES || (shares > 1 && columns != 64 && columns != 128)) return FMM_ERR_INVALID_ARG;
    forced_shape = {columns, shares};
    return FMM_OK;
}

fmm_status_t fmm_fp8_status(int* code)
{
    if (!code) return FMM_ERR_INVALID_ARG;
    *code = 0;
    int words[3] = {0, 0, 0}, rows = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(words, g_fp8_product_status, sizeof(words)) != cudaSuccess) {
        cudaGetLastError();
        return FMM_ERR_CUDA;
    }
    const fmm_status_t s = fp8_rows_guard_read(&rows, false);
    if (s != FMM_OK) return s;
    *code = words[0] ? words[0] : words[2] ? words[2] : rows;
    return words[0] ? FMM_ERR_DEVICE_TIMEOUT : FMM_OK;
}

fmm_status_t fmm_fp8_status_clear(void)
{
    const int zero[3] = {0, 0, 0};
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyToSymbol(g_fp8_product_status, zero, sizeof(zero)) != cudaSuccess) {
        cudaGetLastError();
        return FMM_ERR_CUDA;
    }
    int unused = 0;
    return fp8_rows_guard_read(&unused, true);
}

fmm_status_t fmm_fp8_selftest_bounded_wait(int64_t limit_ns, void* stream)
{
    if (limit_ns < 1 || limit_ns > 2000000000) return FMM_ERR_INVALID_ARG;
    int* status = nullptr;
    if (cudaGetSymbolAddress((void**)&status, g_fp8_product_status) != cudaSuccess) { cudaGetLastError(); return FMM_ERR_CUDA; }
    return fmm_launch_bounded_wait_selftest(status, (unsigned long long)limit_ns, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
