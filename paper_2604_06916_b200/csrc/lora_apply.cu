// Low-rank adapters of many requests beside a shared projection, forward and gradients, in BF16 (sm_100a).
//
// A request is a run of rows with an adapter of its own (or none).  With t = x A^T (rank r <= 64 columns):
//     y += s t B^T;     from dy:  dt = s dy B,  dx += dt A,  dA = dt^T x,  dB = s dy^T t
// All products run on tcgen05 with FP32 sums.  t is held in two BF16 parts (each what the one before left: 2^-17 of a value is lost and not
// 2^-9), dt in three (its product with x is an FP32 result), side by side as one wider operand against the other one; the memory
// traffic is that of x, y and dy all the same.
//
// HBM bound: the adapters' products are r / 2 operations a byte of x, y, dy, far below the tensor cores' rate.  Three kernels, each
// of which streams its large operands through a ring of TMA stages once:
//   shrink  t = x A^T (or dy B): 128 rows a cluster, whose blocks share the columns and add up their sums over one another's shared
//           memory; leaves t's parts
//   outer   dA and dB: 128 columns of x or dy by the columns of dt's or t's parts, summed over an adapter's rows (both operands have
//           the row as their second index: MN-major); row slices of one adapter are added up in order by a last small launch
//   expand  takes t as an operand and walks 64 columns at a time: a stage brings the columns of y and the factor's rows, the
//           product is added to y in the stage's own memory, and a TMA store takes it back
// Which rows and adapter a block has follows from the requests' offsets on the device: the host knows neither, the grid covers the most
// that there can be (a tile of 128 rows for each 128 rows and one more per request) and blocks without a tile leave.
// Everything is summed in a fixed order: equal inputs give equal bits.
//
// Measured (B200, inside a graph; bytes of the operands once, and each kernel by itself): 17003 rows, 3072 -> 9216, rank 32, 127 us = 5.2
// TB/s, 80 % of the copy rate (shrink 25, expand 103: 6.1 TB/s); gradients of 9216 rows 104 us (shrink 39, outer 44, its sum 4, expand
// 25): dy is read twice, which makes 78 us the floor of this form and 52 that of one that could keep dB's sums of all columns beside dt's (a
// megabyte a row slice).  8 requests of one row, 3072 -> 18432, 17.3 us: latency, two launches of 7 to 9 us each.
// What it was before: t's slices through the workspace and summed by every expanding block, 155 and 110 us (the sum over a
// cluster: 127 and 117 with a cluster that left a second wave, 107 without); a stage held until the next store, 152; y written from registers
// in place of TMA, 166.  Stages of 256 bytes a row in place of 128 in shrink are worth 1 us; another order of columns in every
// block, against their reading the factor's same lines at the same time, nothing.
#include "gemm_common.cuh"
#include "quant_math.cuh"
#include "sol_internal.h"

#include <atomic>

namespace sol {
namespace lora {
namespace {

using gemm::loads_held;
using gemm::wait_bounded;

constexpr int kRows = 128;               // rows of a tile
constexpr int kBox = 64;                 // 16-bit columns of a 128-byte swizzled row
constexpr int kMaxRank = 64, kMaxRequests = 1024;
constexpr int kRowBox = kRows * 128;     // bytes of a [128][64] box
constexpr int kFactorBox = 64 * 128;     // bytes of a [64][64] box
constexpr int kStage = kRowBox + kFactorBox;
constexpr int kMaxStages = 8;
constexpr int kShrinkStage = 2 * kStage;    // 128 columns: rows of 256 bytes, which DRAM gives faster than twice 128
constexpr int kMaxCluster = 8;
constexpr int kHalfSmem = 115712, kFullSmem = 232448;     // a block's shared memory where two fit an SM, or one
constexpr int kSlots = 296;              // blocks that are taken to be resident at once: two on each of 148 SMs (above rank 32 expand has one)

struct Requests {
    const int32_t *offsets;    // [requests + 1]
    const int32_t *ids;        // [requests]
    int requests, adapters, rows;
};
struct Item {
    int row0, end, adapter;    // first row of the tile, row behind the request's last
};

__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t *abort_flag, uint32_t *status, uint32_t code) {
    return __all_sync(0xFFFFFFFFu, wait_bounded(bar, parity, abort_flag, status, code));
}
// Rows of request `s`, held to the rows that exist; the adapter, -1 for none.
__device__ __forceinline__ void request(const Requests &q, int s, int &begin, int &end, int &adapter) {
    begin = min(max(__ldg(q.offsets + s), 0), q.rows);
    end = min(max(__ldg(q.offsets + s + 1), begin), q.rows);
    adapter = __ldg(q.ids + s);
    if (adapter < 0 || adapter >= q.adapters) adapter = -1;
}
// The index-th tile of all requests in order; called by a whole warp.  False: there are not so many.
__device__ __forceinline__ bool find_item(const Requests &q, int index, int lane, Item &item) {
    int before = 0;
    for (int s0 = 0; s0 < q.requests; s0 += 32) {
        int begin = 0, end = 0, adapter = -1;
        if (s0 + lane < q.requests) request(q, s0 + lane, begin, end, adapter);
        const int tiles = adapter >= 0 ? (end - begin + kRows - 1) / kRows : 0;
        int upto = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += v;
        }
        const int total = __shfl_sync(0xFFFFFFFFu, upto, 31);
        if (index < before + total) {
            const int src = __ffs(__ballot_sync(0xFFFFFFFFu, before + upto > index)) - 1;
            const int tile = index - before - __shfl_sync(0xFFFFFFFFu, upto - tiles, src);
            item.row0 = __shfl_sync(0xFFFFFFFFu, begin, src) + tile * kRows;
            item.end = __shfl_sync(0xFFFFFFFFu, end, src);
            item.adapter = __shfl_sync(0xFFFFFFFFu, adapter, src);
            return true;
        }
        before += total;
    }
    return false;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t idesc_of(int n, bool a_mn, bool b_mn) {   // BF16 x BF16 -> FP32, M = 128
    return (1u << 4) | (1u << 7) | (1u << 10) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) |
           (static_cast<uint32_t>(kRows >> 4) << 24);
}

// The first 1024 bytes of a block's shared memory (all of it dynamic, so that what follows lies on 1024-byte boundaries as the
// swizzled operands want it): barriers, the tensor memory's address, the flag of waits that ran out, the item.
constexpr int kControl = 1024;
struct Control {
    uint64_t bars[32];
    uint32_t tmem, abort;
    int found;
    Item item;
    int n_runs;
};
static_assert(sizeof(Control) <= kControl, "control block");

// False: the shared memory is not where it has to be (never seen; recorded, nothing is done).
__device__ __forceinline__ bool aligned_block(const uint8_t *smem, uint32_t *status) {
    if ((ptx::smem_u32(smem) & 1023u) == 0) return true;
    if (threadIdx.x == 0) atomicExch(status, 0xDF0u);
    return false;
}
// `count(i)`: arrivals that barrier i waits for.
template <uint32_t kColumns, class Count>
__device__ __forceinline__ void begin_block(Control &c, int n_bars, Count count, int warp) {
    if (threadIdx.x == 0) {
        for (int i = 0; i < n_bars; ++i) ptx::mbar_init(ptx::smem_u32(c.bars + i), count(i));
        c.abort = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc(ptx::smem_u32(&c.tmem), kColumns);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
}
template <uint32_t kColumns>
__device__ __forceinline__ void end_block(volatile uint32_t *abort_flag, int warp, uint32_t tmem) {
    if (*abort_flag) __nanosleep(2000000);   // let copies already in flight land before the block exits
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, kColumns);
    }
}

// The tensor core adds to an FP32 sum with truncation, 2^-25 of it a step on average and always towards zero: a sum is taken out after so
// many stages (32 steps, 2^-20) and goes on in a register, where additions are rounded.
constexpr int kWindow = 8;               // of 64 rows
constexpr int kShrinkWindow = 4;         // of 128 columns

// ------------------------------------------------------------------------------------------------ shrink
struct Shrink {
    Requests q;
    const float *scaling;     // [adapters]; null: t as it is
    uint16_t *parts;          // [rows][n_parts r]: t's parts, each what the ones before it left
    uint32_t *status;
    int n_parts;              // 2 or 3
    int r, r16;               // rank, and the next multiple of 16
    int tiles, per_split;     // 128-column tiles of the long side, and those of a block
    int splits, stages;       // blocks of a cluster, which share the long side
};
__device__ __forceinline__ float4 ld_cluster(uint32_t cluster_addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_addr) : "memory");
    return v;
}

// kFlip: the factor is [long side][r] (dy B: B is [N][r]) and not [r][long side].
template <bool kFlip>
__global__ void __launch_bounds__(192)
shrink_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_f, const Shrink p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    if (!aligned_block(smem, p.status)) return;
    Control &control = *reinterpret_cast<Control *>(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = blockIdx.x % p.splits;
    if (warp == 0) {
        Item it{};
        const bool there = find_item(p.q, blockIdx.x / p.splits, lane, it);
        if (lane == 0) control.item = it, control.found = there;
    }
    __syncthreads();
    if (!control.found) return;
    const Item item = control.item;
    // full, empty: [stage]; sum full, sum empty: [accumulator]
    constexpr int kSumFull = 2 * kMaxStages, kSumEmpty = kSumFull + 2;
    begin_block<128>(control, kSumEmpty + 2, [](int i) { return i >= kSumEmpty ? 4 : 1; }, warp);
    ptx::grid_launch_dependents();
    const uint32_t bars = ptx::smem_u32(control.bars), tmem = control.tmem, ring = ptx::smem_u32(smem) + kControl;
    volatile uint32_t *abort_flag = &control.abort;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (kMaxStages + s); };
    auto bar = [&](int i) { return bars + 8u * i; };
    const int t0 = split * p.per_split, t1 = min(p.tiles, t0 + p.per_split);
    if (warp == 0) {
        if (ptx::elect_one() && !loads_held(p.status)) {
            const uint32_t factor_bytes = kFlip ? kFactorBox : p.r16 * 128;
            for (int t = t0, s = 0, n = 0; t < t1; ++t, ++n, s = s + 1 == p.stages ? 0 : s + 1) {
                if (n >= p.stages && !wait_bounded(empty(s), ((n / p.stages) - 1) & 1u, abort_flag, p.status, 0xD00u | s)) break;
                const uint32_t to = ring + s * kShrinkStage;
                ptx::mbar_arrive_expect_tx(full(s), 2 * (kRowBox + factor_bytes));
#pragma unroll
                for (int h = 0; h < 2; ++h) ptx::tma_load_2d(to + h * kRowBox, &tm_x, (2 * t + h) * kBox, item.row0, full(s));
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t at = to + 2 * kRowBox + h * kFactorBox;
                    if (kFlip) ptx::tma_load_3d(at, &tm_f, 0, (2 * t + h) * kBox, item.adapter, full(s));
                    else ptx::tma_load_3d(at, &tm_f, (2 * t + h) * kBox, 0, item.adapter, full(s));
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (ptx::elect_one()) {
            const uint32_t idesc = idesc_of(p.r16, false, kFlip);
            for (int t = t0, s = 0, n = 0; t < t1; ++t, ++n, s = s + 1 == p.stages ? 0 : s + 1) {
                const int w = n / kShrinkWindow, d = w & 1;
                if (n % kShrinkWindow == 0 && w >= 2 && !wait_bounded(bar(kSumEmpty + d), ((w >> 1) - 1) & 1u, abort_flag, p.status, 0xD18u | d)) break;
                if (!wait_bounded(full(s), (n / p.stages) & 1u, abort_flag, p.status, 0xD10u | s)) break;
                ptx::tc_fence_after_sync();
                const uint32_t from = ring + s * kShrinkStage;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t factor = from + 2 * kRowBox + (i >> 2) * kFactorBox;
                    const uint64_t a = ptx::smem_desc_sw128(from + (i >> 2) * kRowBox) + 2u * (i & 3);
                    const uint64_t b = kFlip ? ptx::smem_desc_sw128_mn(factor + (i & 3) * 2048, kFactorBox, 1024) : ptx::smem_desc_sw128(factor) + 2u * (i & 3);
                    ptx::mma_bf16(tmem + d * kBox, a, b, idesc, n % kShrinkWindow > 0 || i > 0);
                }
                ptx::tc_commit(empty(s));
                if (n % kShrinkWindow == kShrinkWindow - 1 || t + 1 == t1) ptx::tc_commit(bar(kSumFull + d));
            }
        }
        __syncwarp();
    } else {
        const int quad = warp & 3;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        float sum[kMaxRank] = {};
        bool ok = true;
        for (int w = 0; w * kShrinkWindow < t1 - t0; ++w) {
            const int d = w & 1;
            if (!(ok = warp_wait(bar(kSumFull + d), (w >> 1) & 1u, abort_flag, p.status, 0xD20u | d))) break;
            ptx::tc_fence_after_sync();
#pragma unroll
            for (int c = 0; c < kMaxRank; c += 8) {
                if (c >= p.r) continue;
                uint32_t v[8];
                ptx::tmem_ld_32x8(lanes + d * kBox + c, v);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[c + e] += __uint_as_float(v[e]);
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(kSumEmpty + d));
        }
        if (!ok) __nanosleep(2000000);     // copies already in flight land where the sums go, before them
        // this slice's sums, for the cluster: rows of r floats and four that keep them off one another's banks, where the ring was
        const float nan = __uint_as_float(0x7FC00000u);       // what reads a sum that is not whole shall not take it for a result
        float *mine = reinterpret_cast<float *>(smem + kControl) + (quad * 32 + lane) * (p.r + 4);
#pragma unroll
        for (int c = 0; c < kMaxRank; c += 4) {
            if (c < p.r)
                *reinterpret_cast<float4 *>(mine + c) = ok ? make_float4(sum[c], sum[c + 1], sum[c + 2], sum[c + 3]) : make_float4(nan, nan, nan, nan);
        }
    }
    __syncwarp();
    ptx::cluster_sync();
    // every block adds up its share of the rows' pieces of eight columns, slice after slice, and writes both parts
    const float factor = p.scaling != nullptr ? __ldg(p.scaling + item.adapter) : 1.0f;
    const int pieces = p.r >> 3, rows_here = min(kRows, item.end - item.row0);
    for (int i = split + p.splits * threadIdx.x; i < rows_here * pieces; i += p.splits * blockDim.x) {
        const int r = i / pieces, c = 8 * (i - r * pieces);
        float t[8] = {};
        for (int s = 0; s < p.splits; ++s) {
            const uint32_t from = ptx::map_to_cta(ring + 4 * (r * (p.r + 4) + c), s);
            const float4 a = ld_cluster(from), b = ld_cluster(from + 16);
            t[0] += a.x, t[1] += a.y, t[2] += a.z, t[3] += a.w, t[4] += b.x, t[5] += b.y, t[6] += b.z, t[7] += b.w;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] *= factor;
        uint16_t *out = p.parts + static_cast<int64_t>(item.row0 + r) * p.n_parts * p.r + c;
        for (int part = 0; part < p.n_parts; ++part, out += p.r) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = pack_bf16(t[2 * e], t[2 * e + 1]);
                t[2 * e] -= qmath::bf16_lo(w[e]), t[2 * e + 1] -= qmath::bf16_hi(w[e]);
            }
            *reinterpret_cast<uint4 *>(out) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    ptx::cluster_sync();                   // nobody leaves while others read its memory
    end_block<128>(abort_flag, warp, tmem);
}

// ------------------------------------------------------------------------------------------------ expand
struct Expand {
    Requests q;
    const uint16_t *parts;    // [rows][n_parts r]: t's parts, of which the first two are used
    const float *scaling;     // [adapters]; null: it is on t already
    int n_parts;
    uint16_t *y;
    uint32_t *status;
    int64_t ldy;
    int r, r16, stages;
    int columns, chunks, per_slice, slices;    // 64-column chunks of y, and those of a block
};

// kFlip: the factor is [r][columns] (dt A) and not [columns][r].
template <bool kFlip>
__global__ void __launch_bounds__(320, 2)
expand_kernel(const __grid_constant__ CUtensorMap tm_y, const __grid_constant__ CUtensorMap tm_out, const __grid_constant__ CUtensorMap tm_f,
              const Expand p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    if (!aligned_block(smem, p.status)) return ptx::grid_dependency_wait();
    Control &control = *reinterpret_cast<Control *>(smem);
    constexpr int kSums = 4;              // accumulators of 64 columns
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int slice = blockIdx.x % p.slices;
    if (warp == 0) {
        Item it{};
        const bool there = find_item(p.q, blockIdx.x / p.slices, lane, it);
        if (lane == 0) control.item = it, control.found = there;
    }
    __syncthreads();
    if (!control.found) return ptx::grid_dependency_wait();       // a grid without a tile ends behind the one in front of it all the same
    const Item item = control.item;
    // full, empty: [stage]; sum full, sum empty: [accumulator]; t ready
    constexpr int kSumFull = 2 * kMaxStages, kSumEmpty = kSumFull + kSums, kReady = kSumEmpty + kSums, kBars = kReady + 1;
    // a request's last tile may leave warps without rows: they do not take part
    const int quads = min(4, (item.end - item.row0 + 31) / 32);
    begin_block<64 * kSums>(control, kBars,
                            [quads](int i) { return i == kReady ? 8 : (i >= kMaxStages && i < kSumFull) || i >= kSumEmpty ? quads : 1; }, warp);
    ptx::grid_launch_dependents();
    const uint32_t bars = ptx::smem_u32(control.bars), tmem = control.tmem;
    volatile uint32_t *abort_flag = &control.abort;
    auto bar = [&](int i) { return bars + 8u * i; };
    const uint32_t sT = ptx::smem_u32(smem) + kControl;           // t as [128][2 r16], boxes of 64 columns
    const int t_boxes = (2 * p.r16 + kBox - 1) / kBox;
    const uint32_t ring = sT + t_boxes * kRowBox;
    const int c0 = slice * p.per_slice, c1 = min(p.chunks, c0 + p.per_slice);
    if (warp == 0) {
        if (ptx::elect_one() && !loads_held(p.status)) {
            const uint32_t factor_bytes = kFlip ? p.r16 * 128 : kFactorBox;
            for (int c = c0, s = 0, n = 0; c < c1; ++c, ++n, s = s + 1 == p.stages ? 0 : s + 1) {
                if (n == p.stages) ptx::grid_dependency_wait();      // a wait's limit counts from when what it waits for can come
                if (n >= p.stages && !wait_bounded(bar(kMaxStages + s), ((n / p.stages) - 1) & 1u, abort_flag, p.status, 0xD30u | s)) break;
                const uint32_t to = ring + s * kStage;
                ptx::mbar_arrive_expect_tx(bar(s), kRowBox + factor_bytes);
                ptx::tma_load_2d(to, &tm_y, c * kBox, item.row0, bar(s));
                if (kFlip) ptx::tma_load_3d(to + kRowBox, &tm_f, c * kBox, 0, item.adapter, bar(s));
                else ptx::tma_load_3d(to + kRowBox, &tm_f, 0, c * kBox, item.adapter, bar(s));
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (ptx::elect_one()) {
            const uint32_t idesc = idesc_of(kBox, false, kFlip);
            const int half = p.r16 >> 4;          // products for each of t's parts
            ptx::grid_dependency_wait();
            bool ok = wait_bounded(bar(kReady), 0, abort_flag, p.status, 0xD40u);
            for (int c = c0, s = 0, n = 0; ok && c < c1; ++c, ++n, s = s + 1 == p.stages ? 0 : s + 1) {
                const int d = n % kSums;
                if (n >= kSums && !wait_bounded(bar(kSumEmpty + d), ((n / kSums) - 1) & 1u, abort_flag, p.status, 0xD50u | d)) break;
                if (!wait_bounded(bar(s), (n / p.stages) & 1u, abort_flag, p.status, 0xD60u | s)) break;
                ptx::tc_fence_after_sync();
                const uint32_t from = ring + s * kStage + kRowBox;
                for (int i = 0; i < 2 * half; ++i) {
                    const int j = i < half ? i : i - half;
                    const uint64_t a = ptx::smem_desc_sw128(sT + (i >> 2) * kRowBox) + 2u * (i & 3);
                    const uint64_t b = kFlip ? ptx::smem_desc_sw128_mn(from + j * 2048, kFactorBox, 1024) : ptx::smem_desc_sw128(from) + 2u * j;
                    ptx::mma_bf16(tmem + d * kBox, a, b, idesc, i > 0);
                }
                ptx::tc_commit(bar(kSumFull + d));
            }
        }
        __syncwarp();
    } else {
        const int group = (warp - 2) >> 2, quad = warp & 3;
        const int tile_row = quad * 32 + lane, row = item.row0 + tile_row;
        const bool there = row < item.end;
        const float scale = p.scaling != nullptr ? __ldg(p.scaling + item.adapter) : 1.0f;
        const uint32_t sw = static_cast<uint32_t>(tile_row & 7);
        ptx::grid_dependency_wait();
        // t's parts into the operand, each on a multiple of 16 columns, zeros where there is nothing; the two groups take turns
#pragma unroll
        for (int k = 0; k < kMaxRank / 16; ++k) {
            const int c = 8 * group + 16 * k;
            if (c >= p.r16) continue;
            uint4 h = make_uint4(0, 0, 0, 0), l = h;
            if (there && c < p.r) {
                const uint16_t *from = p.parts + static_cast<int64_t>(row) * p.n_parts * p.r + c;
                h = __ldcg(reinterpret_cast<const uint4 *>(from));
                l = __ldcg(reinterpret_cast<const uint4 *>(from + p.r));
            }
            const int ch = c >> 3, cl = (c + p.r16) >> 3;       // 16-byte pieces of the operand's row
            sts128(sT + (ch >> 3) * kRowBox + tile_row * 128 + ((static_cast<uint32_t>(ch & 7) ^ sw) << 4), h);
            sts128(sT + (cl >> 3) * kRowBox + tile_row * 128 + ((static_cast<uint32_t>(cl & 7) ^ sw) << 4), l);
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(kReady));
        // chunks of 64 columns, the two groups in turn
        const bool whole = item.row0 + quad * 32 + 32 <= item.end;         // all of this warp's rows are the request's
        bool ok = true;
        for (int c = c0 + group, n = group; c < c1 && quad < quads; c += 2, n += 2) {
            const int d = n % kSums, s = n % p.stages;
            ok = warp_wait(bar(kSumFull + d), (n / kSums) & 1u, abort_flag, p.status, 0xD70u | d) &&
                 warp_wait(bar(s), (n / p.stages) & 1u, abort_flag, p.status, 0xD80u | s);
            if (!ok) break;
            ptx::tc_fence_after_sync();
            const uint32_t at = ring + s * kStage + tile_row * 128;
            uint16_t *out = p.y + row * p.ldy + c * kBox;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t v[32];
                ptx::tmem_ld_32x32(tmem + (static_cast<uint32_t>(quad * 32) << 16) + d * kBox + 32 * h, v);
                uint4 old[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) old[q] = ptx::lds128(at + ((static_cast<uint32_t>(4 * h + q) ^ sw) << 4));
                ptx::tmem_ld_wait();
                if (h == 1) {
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar(kSumEmpty + d));
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t w[4] = {old[q].x, old[q].y, old[q].z, old[q].w};
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = pack_bf16(fmaf(__uint_as_float(v[q * 8 + 2 * e]), scale, qmath::bf16_lo(w[e])),
                                         fmaf(__uint_as_float(v[q * 8 + 2 * e + 1]), scale, qmath::bf16_hi(w[e])));
                    const uint4 now = make_uint4(o[0], o[1], o[2], o[3]);
                    if (whole) sts128(at + ((static_cast<uint32_t>(4 * h + q) ^ sw) << 4), now);
                    else if (there && c * kBox + 32 * h + 8 * q < p.columns) *reinterpret_cast<uint4 *>(out + 32 * h + 8 * q) = now;
                }
            }
            if (whole) {
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    ptx::tma_store_2d(&tm_out, c * kBox, item.row0 + quad * 32, ring + s * kStage + quad * 32 * 128);
                    ptx::tma_store_commit();
                    ptx::tma_store_wait_read<0>();
                    ptx::mbar_arrive(bar(kMaxStages + s));
                }
            } else {
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar(kMaxStages + s));
            }
        }
        if (lane == 0) ptx::tma_store_wait_all<0>();
    }
    end_block<64 * kSums>(abort_flag, warp, tmem);
}

// ------------------------------------------------------------------------------------------------ outer
struct Outer {
    Requests q;
    const float *scaling;
    float *da, *db;           // [adapters][r][K], [adapters][N][r]; with several row slices those of the workspace's first
    int64_t slice_floats;     // from one row slice's sums to the next's
    uint32_t *status;
    int r, K, N, tiles_x, tiles;    // 128-column tiles of x, and of x and dy
    int slices;               // row slices of an adapter
    int parts_x, parts_dy;    // parts of dt (with x) and of t (with dy)
};
constexpr int kStepRows = 64;
constexpr int kRunBytes = kMaxRequests * 8;
// A stage: 128 columns of x or dy and all parts' columns of dt or t; two blocks an SM.
__host__ __device__ constexpr int outer_stage(int r, int parts) { return (2 + (parts * r + kBox - 1) / kBox) * kFactorBox; }
__host__ __device__ constexpr int outer_stages(int r, int parts) { return (kHalfSmem - kControl - kRunBytes) / outer_stage(r, parts); }

__global__ void __launch_bounds__(192, 2)
outer_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_dy, const __grid_constant__ CUtensorMap tm_dt,
             const __grid_constant__ CUtensorMap tm_t, const Outer p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    if (!aligned_block(smem, p.status)) return ptx::grid_dependency_wait();
    Control &control = *reinterpret_cast<Control *>(smem);
    int2 *runs = reinterpret_cast<int2 *>(smem + kControl);       // this block's rows: [begin, end) of each request of its adapter, cut to the slice
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tile = blockIdx.x % p.tiles, slice = blockIdx.x / p.tiles % p.slices, adapter = blockIdx.x / p.tiles / p.slices;
    const bool of_x = tile < p.tiles_x;
    const int column = (of_x ? tile : tile - p.tiles_x) * 128;
    if (warp == 0) {
        const int lo = static_cast<int>(static_cast<int64_t>(p.q.rows) * slice / p.slices);
        const int hi = static_cast<int>(static_cast<int64_t>(p.q.rows) * (slice + 1) / p.slices);
        int n = 0;
        for (int s0 = 0; s0 < p.q.requests; s0 += 32) {
            int begin = 0, end = 0, a = -1;
            if (s0 + lane < p.q.requests) request(p.q, s0 + lane, begin, end, a);
            begin = max(begin, lo), end = min(end, hi);
            const uint32_t mine = __ballot_sync(0xFFFFFFFFu, a == adapter && begin < end);
            if (mine >> lane & 1u) runs[n + __popc(mine & ((1u << lane) - 1u))] = make_int2(begin, end);
            n += __popc(mine);
        }
        if (lane == 0) control.n_runs = n;
    }
    // full, empty: [stage]; sum full, sum empty: [accumulator].  A sum has a column for every part's; two take turns where they fit
    constexpr int kSumFull = 2 * kMaxStages, kSumEmpty = kSumFull + 2, kColumns = 256;
    const int parts = of_x ? p.parts_x : p.parts_dy, n_columns = (parts * p.r + 15) / 16 * 16, sums = n_columns <= kColumns / 2 ? 2 : 1;
    const int stage_bytes = outer_stage(p.r, parts), stages = outer_stages(p.r, parts);
    begin_block<kColumns>(control, kSumEmpty + 2, [](int i) { return i >= kSumEmpty ? 4 : 1; }, warp);
    ptx::grid_launch_dependents();
    const uint32_t bars = ptx::smem_u32(control.bars), tmem = control.tmem, ring = ptx::smem_u32(smem) + kControl + kRunBytes;
    volatile uint32_t *abort_flag = &control.abort;
    const int n_runs = control.n_runs;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (kMaxStages + s); };
    auto bar = [&](int i) { return bars + 8u * i; };
    int steps = 0;                        // of 64 rows
    for (int run = 0; run < n_runs; ++run) steps += (runs[run].y - runs[run].x + kStepRows - 1) / kStepRows;
    const int u_boxes = (parts * p.r + kBox - 1) / kBox;
    if (warp == 0) {
        ptx::grid_dependency_wait();
        if (ptx::elect_one() && !loads_held(p.status)) {
            const CUtensorMap *tm_z = of_x ? &tm_x : &tm_dy, *tm_u = of_x ? &tm_dt : &tm_t;
            int s = 0, n = 0;
            bool ok = true;
            for (int run = 0; ok && run < n_runs; ++run) {
                for (int row = runs[run].x; row < runs[run].y; row += kStepRows, ++n, s = s + 1 == stages ? 0 : s + 1) {
                    if (n >= stages && !(ok = wait_bounded(empty(s), ((n / stages) - 1) & 1u, abort_flag, p.status, 0xD90u | s))) break;
                    const uint32_t to = ring + s * stage_bytes;
                    ptx::mbar_arrive_expect_tx(full(s), (2 + u_boxes) * kFactorBox);
                    ptx::tma_load_2d(to, tm_z, column, row, full(s));
                    ptx::tma_load_2d(to + kFactorBox, tm_z, column + kBox, row, full(s));
                    for (int b = 0; b < u_boxes; ++b) ptx::tma_load_2d(to + (2 + b) * kFactorBox, tm_u, b * kBox, row, full(s));
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        ptx::grid_dependency_wait();          // the waits' limits count from here
        const uint32_t idesc = idesc_of(n_columns, true, true);
        int s = 0, n = 0;
        bool ok = true;
        for (int run = 0; ok && run < n_runs; ++run) {
            for (int row = runs[run].x; row < runs[run].y; row += kStepRows, ++n, s = s + 1 == stages ? 0 : s + 1) {
                const int w = n / kWindow, d = w % sums;
                if (n % kWindow == 0 && w >= sums && !(ok = warp_wait(bar(kSumEmpty + d), (w / sums - 1) & 1u, abort_flag, p.status, 0xDA8u | d))) break;
                if (!(ok = warp_wait(full(s), (n / stages) & 1u, abort_flag, p.status, 0xDA0u | s))) break;
                const uint32_t from = ring + s * stage_bytes;
                const int rows = runs[run].y - row;
                if (rows < kStepRows) {       // rows that belong to somebody else may hold anything: zeros in their place
                    for (int i = rows * 8 + lane; i < kStepRows * 8; i += 32)
                        for (int b = 0; b < 2 + u_boxes; ++b) sts128(from + b * kFactorBox + i * 16, make_uint4(0, 0, 0, 0));
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                }
                if (ptx::elect_one()) {
                    ptx::tc_fence_after_sync();
#pragma unroll
                    for (int i = 0; i < kStepRows / 16; ++i)
                        ptx::mma_bf16(tmem + d * (kColumns / 2), ptx::smem_desc_sw128_mn(from + i * 2048, kFactorBox, 1024),
                                      ptx::smem_desc_sw128_mn(from + 2 * kFactorBox + i * 2048, kFactorBox, 1024), idesc, n % kWindow > 0 || i > 0);
                    ptx::tc_commit(empty(s));
                    if (n % kWindow == kWindow - 1 || n + 1 == steps) ptx::tc_commit(bar(kSumFull + d));
                }
                __syncwarp();
            }
        }
    } else {
        ptx::grid_dependency_wait();
        const int quad = warp & 3, c = column + quad * 32 + lane;
        const uint32_t lanes_at = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        float v[kMaxRank] = {};
        bool ok = true;
        for (int w = 0; w * kWindow < steps; ++w) {
            const int d = w % sums;
            if (!(ok = warp_wait(bar(kSumFull + d), (w / sums) & 1u, abort_flag, p.status, 0xDB0u | d))) break;
            ptx::tc_fence_after_sync();
#pragma unroll
            for (int j = 0; j < kMaxRank; j += 8) {
                if (j >= p.r) continue;
                uint32_t part[3][8];
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (k < parts) ptx::tmem_ld_32x8(lanes_at + d * (kColumns / 2) + k * p.r + j, part[k]);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float low = parts > 2 ? __uint_as_float(part[1][e]) + __uint_as_float(part[2][e]) : __uint_as_float(part[1][e]);
                    v[j + e] += __uint_as_float(part[0][e]) + low;
                }
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(kSumEmpty + d));
        }
        const float scale = of_x || steps == 0 ? 1.0f : __ldg(p.scaling + adapter);     // no rows: zeros, whatever the scaling holds
        float *out = (of_x ? p.da : p.db) + slice * p.slice_floats;
        if (ok && c < (of_x ? p.K : p.N)) {
#pragma unroll
            for (int j = 0; j < kMaxRank; j += 4) {
                if (j >= p.r) continue;
                if (of_x) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) out[(static_cast<int64_t>(adapter) * p.r + j + e) * p.K + c] = v[j + e];
                } else {
                    *reinterpret_cast<float4 *>(out + (static_cast<int64_t>(adapter) * p.N + c) * p.r + j) =
                        make_float4(v[j] * scale, v[j + 1] * scale, v[j + 2] * scale, v[j + 3] * scale);
                }
            }
        }
    }
    end_block<kColumns>(abort_flag, warp, tmem);
}

// The row slices' sums, in order: dA's values, then dB's.
__global__ void __launch_bounds__(256)
add_slices(const float4 *__restrict__ from, int64_t slice4, int slices, int64_t da4, float4 *da, float4 *db) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    if (i >= slice4) return;
    float4 v = __ldcg(from + i);
    for (int s = 1; s < slices; ++s) {
        const float4 w = __ldcg(from + s * slice4 + i);
        v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
    }
    if (i < da4) da[i] = v;
    else db[i - da4] = v;
}

// ------------------------------------------------------------------------------------------------ host side
// How a call's work is shared out: from its sizes alone.
int64_t items_of(int64_t M, int64_t requests) { return ceil_div(M, kRows) + requests; }     // tiles of rows, at most
struct Slices {
    int chunks, slices, per_slice;         // 64-column chunks of expand's y, and how blocks share them
};
Slices expand_slices(int64_t items, int64_t columns) {
    // the number of slices with the least (waves + 1/2) (chunks of a block + 4): a block's way in and out is worth some four chunks, and half
    // a wave stands for slots that stay empty at the end and behind short requests.  Every number of slices once, with the fewest chunks
    Slices best{static_cast<int>(ceil_div(columns, kBox)), 1, 0};
    double least = 0.0;
    for (int64_t per = best.chunks; per >= 1; --per) {
        const int64_t n = ceil_div(best.chunks, per);
        per = ceil_div(best.chunks, n);
        const double waves = static_cast<double>(items * n) / kSlots, cost = ((waves < 1.0 ? 1.0 : waves) + 0.5) * static_cast<double>(per + 4);
        if (best.per_slice == 0 || cost < least) least = cost, best.slices = static_cast<int>(n), best.per_slice = static_cast<int>(per);
    }
    return best;
}
struct OuterPlan {
    int tiles, tiles_x, slices;
};
OuterPlan outer_plan(int64_t M, int64_t K, int64_t N, int64_t adapters) {
    OuterPlan p;
    p.tiles_x = static_cast<int>(ceil_div(K, 128));
    p.tiles = p.tiles_x + static_cast<int>(ceil_div(N, 128));
    int64_t slices = kSlots / (p.tiles * adapters);
    if (slices > ceil_div(M, 512)) slices = ceil_div(M, 512);
    p.slices = slices < 1 ? 1 : static_cast<int>(slices);
    return p;
}
int64_t pad256(int64_t bytes) { return (bytes + 255) / 256 * 256; }
// t in two parts; dt in three, since the gradient of lora_a is FP32 and two would be what limits it
constexpr int kTParts = 2, kDtParts = 3;
int64_t parts_bytes(int64_t M, int64_t r, int parts) { return pad256(2 * parts * M * r); }

// Allows kernel `kern` `smem` bytes of dynamic shared memory on the current device (asked for once).
template <auto kern>
bool allow_smem(int smem) {
    static bool done[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    if (done[dev]) return true;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    return done[dev] = true;
}
// kAfter: the kernel may come into the SMs while the one in front of it drains, and waits itself for what that one writes.
template <bool kAfter, class... P, class... A>
sol_status_t launch(void (*kern)(P...), int64_t grid, int threads, int smem, int cluster, cudaStream_t stream, A... args) {
    if (grid > 0x7FFFFFFFLL) return SOL_ERR_BAD_SHAPE;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kAfter ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kern, args...) != cudaSuccess) {
        cudaGetLastError();
        return SOL_ERR_CUDA;
    }
    return launch_status();
}
bool rows_map(CUtensorMap *out, const void *base, int64_t cols, int64_t rows, int64_t ld, int box_rows) {
    return make_tmap_2d(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, cols, rows, 2 * ld, kBox, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
}
// A stack of factors [adapters][rows][cols]; boxes of 64 columns.
bool factor_map(CUtensorMap *out, const void *base, int64_t cols, int64_t rows, int64_t adapters, int box_rows) {
    return make_tmap_3d_bf16(out, base, cols, rows, adapters, 2 * cols, 2 * cols * rows, kBox, box_rows);
}

constexpr int kShrinkStages = 4;           // one block an SM

// Blocks that share the long side: as many as leave all clusters resident at once (clusters of some sizes fit the GPU's SM groups worse than
// others: a second wave for one more block costs twice the time), none with fewer than two tiles.
template <bool kFlip>
int shrink_splits(int64_t items, int tiles, int smem) {
    static std::atomic<int> known[64][kMaxCluster + 1];     // by device: clusters of so many blocks that run at once
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 1;
    for (int n = kMaxCluster; n > 1; --n) {
        if (n > tiles / 2) continue;
        int resident = known[dev][n].load(std::memory_order_relaxed);
        if (resident == 0) {
            cudaLaunchConfig_t cfg{};
            cfg.gridDim = dim3(n * 1024);
            cfg.blockDim = dim3(192);
            cfg.dynamicSmemBytes = smem;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = n;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            if (cudaOccupancyMaxActiveClusters(&resident, shrink_kernel<kFlip>, &cfg) != cudaSuccess) {
                cudaGetLastError();
                continue;
            }
            known[dev][n].store(resident, std::memory_order_relaxed);
        }
        if (items <= resident) return n;
    }
    return 1;
}
template <bool kFlip>
sol_status_t launch_shrink(const Requests &q, const void *x, int64_t ldx, const void *factor, int64_t cols, int64_t r, const float *scaling,
                           void *parts, int n_parts, cudaStream_t stream) {
    const int r16 = static_cast<int>(ceil_div(r, 16) * 16), tiles = static_cast<int>(ceil_div(cols, 2 * kBox)), smem = kControl + kShrinkStages * kShrinkStage;
    CUtensorMap tm_x, tm_f;
    if (!rows_map(&tm_x, x, cols, q.rows, ldx, kRows)) return SOL_ERR_CUDA;
    if (!(kFlip ? factor_map(&tm_f, factor, r, cols, q.adapters, kBox) : factor_map(&tm_f, factor, cols, r, q.adapters, r16))) return SOL_ERR_CUDA;
    if (!allow_smem<shrink_kernel<kFlip>>(smem)) return SOL_ERR_CUDA;
    const int64_t items = items_of(q.rows, q.requests);
    const int per = static_cast<int>(ceil_div(tiles, shrink_splits<kFlip>(items, tiles, smem))), splits = static_cast<int>(ceil_div(tiles, per));
    const Shrink p{q, scaling, static_cast<uint16_t *>(parts), device_status_word(), n_parts, static_cast<int>(r), r16, tiles, per, splits, kShrinkStages};
    return launch<false>(shrink_kernel<kFlip>, items * splits, 192, smem, splits, stream, tm_x, tm_f, p);
}
template <bool kFlip>
sol_status_t launch_expand(const Requests &q, const void *parts, int n_parts, const float *scaling, void *y, int64_t ldy, const void *factor, int64_t cols, int64_t r, cudaStream_t stream) {
    const int r16 = static_cast<int>(ceil_div(r, 16) * 16);
    CUtensorMap tm_y, tm_out, tm_f;
    if (!rows_map(&tm_y, y, cols, q.rows, ldy, kRows) || !rows_map(&tm_out, y, cols, q.rows, ldy, 32)) return SOL_ERR_CUDA;
    if (!(kFlip ? factor_map(&tm_f, factor, cols, r, q.adapters, r16) : factor_map(&tm_f, factor, r, cols, q.adapters, kBox))) return SOL_ERR_CUDA;
    const int64_t items = items_of(q.rows, q.requests);
    const Slices plan = expand_slices(items, cols);
    const int t_bytes = static_cast<int>(ceil_div(2 * r16, kBox)) * kRowBox;
    Expand p{q, static_cast<const uint16_t *>(parts), scaling, n_parts, static_cast<uint16_t *>(y), device_status_word(), ldy, static_cast<int>(r), r16,
             0, static_cast<int>(cols), plan.chunks, plan.per_slice, plan.slices};
    // two blocks an SM with four stages up to rank 32, one with eight beyond
    p.stages = ((t_bytes == kRowBox ? kHalfSmem : kFullSmem) - kControl - t_bytes) / kStage;
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    if (!allow_smem<expand_kernel<kFlip>>(kFullSmem)) return SOL_ERR_CUDA;
    return launch<true>(expand_kernel<kFlip>, items * p.slices, 320, kControl + t_bytes + p.stages * kStage, 1, stream, tm_y, tm_out, tm_f, p);
}

}  // namespace

int max_rank() { return kMaxRank; }
int max_requests() { return kMaxRequests; }

size_t workspace_bytes(int64_t M, int64_t K, int64_t N, int64_t r, int64_t adapters, int64_t requests, bool backward) {
    if (!backward) return static_cast<size_t>(parts_bytes(M, r, kTParts));
    (void)requests;
    const int slices = outer_plan(M, K, N, adapters).slices;
    return static_cast<size_t>(parts_bytes(M, r, kDtParts) + (slices > 1 ? 4 * slices * adapters * r * (K + N) : 0));
}

sol_status_t launch_apply(const Call &c, const void *x, int64_t ldx, void *y, int64_t ldy, void *t_out, void *workspace, cudaStream_t stream) {
    const Requests q{c.offsets, c.ids, static_cast<int>(c.requests), static_cast<int>(c.adapters), static_cast<int>(c.M)};
    void *parts = t_out != nullptr ? t_out : workspace;
    const sol_status_t st = launch_shrink<false>(q, x, ldx, c.a, c.K, c.r, nullptr, parts, kTParts, stream);
    if (st != SOL_OK) return st;
    return launch_expand<false>(q, parts, kTParts, c.scaling, y, ldy, c.b, c.N, c.r, stream);
}

sol_status_t launch_backward(const Call &c, const void *dy, int64_t ld_dy, const void *x, int64_t ldx, const void *t, void *dx, int64_t ld_dx,
                             float *da, float *db, void *workspace, cudaStream_t stream) {
    const Requests q{c.offsets, c.ids, static_cast<int>(c.requests), static_cast<int>(c.adapters), static_cast<int>(c.M)};
    const OuterPlan plan = outer_plan(c.M, c.K, c.N, c.adapters);
    uint8_t *dt = static_cast<uint8_t *>(workspace);
    float *sums = reinterpret_cast<float *>(dt + parts_bytes(c.M, c.r, kDtParts));
    sol_status_t st = launch_shrink<true>(q, dy, ld_dy, c.b, c.N, c.r, c.scaling, dt, kDtParts, stream);
    if (st != SOL_OK) return st;
    // the factors' gradients next, while L2 still holds a part of dy
    CUtensorMap tm_x, tm_dy, tm_dt, tm_t;
    if (!rows_map(&tm_x, x, c.K, c.M, ldx, kStepRows) || !rows_map(&tm_dy, dy, c.N, c.M, ld_dy, kStepRows) ||
        !rows_map(&tm_dt, dt, kDtParts * c.r, c.M, kDtParts * c.r, kStepRows) || !rows_map(&tm_t, t, kTParts * c.r, c.M, kTParts * c.r, kStepRows))
        return SOL_ERR_CUDA;
    const int64_t da_floats = c.adapters * c.r * c.K, db_floats = c.adapters * c.r * c.N;
    const bool sliced = plan.slices > 1;
    const Outer p{q, c.scaling, sliced ? sums : da, sliced ? sums + da_floats : db, da_floats + db_floats, device_status_word(), static_cast<int>(c.r),
                  static_cast<int>(c.K), static_cast<int>(c.N), plan.tiles_x, plan.tiles, plan.slices, kDtParts, kTParts};
    if (!allow_smem<outer_kernel>(kHalfSmem)) return SOL_ERR_CUDA;
    st = launch<true>(outer_kernel, static_cast<int64_t>(plan.tiles) * plan.slices * c.adapters, 192, kHalfSmem, 1,
                      stream, tm_x, tm_dy, tm_dt, tm_t, p);
    if (st != SOL_OK) return st;
    if (sliced) {
        const int64_t slice4 = (da_floats + db_floats) / 4;
        st = launch<true>(add_slices, ceil_div(slice4, 256), 256, 0, 1, stream, reinterpret_cast<const float4 *>(sums), slice4, plan.slices,
                          da_floats / 4, reinterpret_cast<float4 *>(da), reinterpret_cast<float4 *>(db));
        if (st != SOL_OK) return st;
    }
    return dx != nullptr ? launch_expand<true>(q, dt, kDtParts, nullptr, dx, ld_dx, c.a, c.K, c.r, stream) : SOL_OK;
}

}  // namespace lora
}  // namespace sol
