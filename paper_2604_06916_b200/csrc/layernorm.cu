// Layer norm with the modulation of a DiT block (or a plain weight), forward and gradients, in BF16 (sm_100a).
//
// The training pass's form of the rollout's norm (which quantizes its output and keeps nothing).  Per row m of sample s:
//     xhat = (x - mean) rstd,  rstd = 1 / sqrt(var + eps);     y = xhat gain + shift,  gain = offset + scale[s]
// and with w = dy gain, the gradients
//     dx = rstd (w - mean(w) - xhat mean(w xhat)),   dscale[s] = sum over the sample's rows of dy xhat,   dshift[s] = sum of dy.
// HBM bound: 4 bytes per element forward, 6 backward.
//
// Forward: a group of warps (one to sixteen, so that a lane holds up to three pieces of eight columns) walks neighbouring rows with
// the row in registers, so mean, variance (of the centred values) and output take one read of x; scale and shift stay in
// registers while the sample lasts and the next row is under way while this one is summed.  Measured (B200, inside a graph): 36864 x 3072,
// eight samples, 75.6 us = 6.0 TB/s, 91 % of the copy rate (a warp per row of its own 113 us: 16 warps per SM, each waiting for its
// one row; two warps 97 us, four 87 us); 333 x 2432 2.8 us.
//
// Gradients: a thread owns the same eight columns of every row that its block walks, so that the sums over rows stay in its
// registers; the two row means go over the block (a group of warps per row, as many groups as fit the block) once per four
// rows, whose successors are under way meanwhile.  A block's sums leave as FP32 partials, which a second launch adds up in FP64 in
// a fixed order: equal inputs give equal bits.  Measured: 9216 x 3072, two samples, 33.5 us = 5.1 TB/s, 77 %; 13287 x 2432 43.2 us.
// Bound by dependences: three warps a scheduler (168 registers a thread) issue every second cycle (at 2432 columns, ten warps, 44 % of
// them), and per instruction a warp waits 1.2 cycles for its own last result, 0.8 for shuffles and shared memory, 0.8 for the arithmetic
// pipe, 0.3 (0.6) at the barrier, 0.4 (0.2) for memory.  A step of four rows is some 560 instructions a warp, half of them taking BF16
// apart and putting it together.  The sum over the blocks is 4 us of it.  Rows through a ring in shared
// memory (24 warps, bulk copies) took 43.6 us: the same instructions and the second reads; without loads ahead 41 us, two
// sets of registers in turn spill (51 us), two blocks an SM with fewer rows a step 43 us.
#include "ptx.cuh"
#include "quant_math.cuh"
#include "sol_internal.h"

#include <atomic>
#include <type_traits>

namespace sol {
namespace norm {
namespace {

using qmath::add2;
using qmath::bf16_hi;
using qmath::bf16_lo;
using qmath::f32x2;
using qmath::f32x2_of_bf16x2;
using qmath::f32x2_split;
using qmath::fma2;
using qmath::mul2;

constexpr int kMaxK = 16384;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack2(uint64_t v) {
    float lo, hi;
    f32x2_split(v, lo, hi);
    return pack_bf16(lo, hi);
}
__device__ __forceinline__ float sum_lanes(uint64_t v) {
    float a, b;
    f32x2_split(v, a, b);
    return a + b;
}
__device__ __forceinline__ uint64_t twice(float f) { return f32x2(f, f); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ uint4 load8(const uint16_t *p) { return __ldcs(reinterpret_cast<const uint4 *>(p)); }
__device__ __forceinline__ uint4 cached8(const uint16_t *p) { return __ldg(reinterpret_cast<const uint4 *>(p)); }

struct Forward {
    const uint16_t *x, *scale, *shift;   // scale, shift: [samples, K], pitch ld_mod, or null
    uint16_t *y;
    float2 *stats;                       // [M] (mean, rstd) or null
    int64_t ldx, ldy, ld_mod;
    uint32_t rows, rows_per_sample;
    int K;
    float offset, eps, inv_k;
};

constexpr int kForwardWarps = 8;

// kWarps warps (a group) share a row and walk neighbouring rows, a lane holds the same kChunks pieces of eight columns of each:
// scale and shift stay in registers while the sample lasts, and the next row is under way while this one is summed.
template <int kWarps, int kChunks>
__global__ void __launch_bounds__(kWarps > kForwardWarps ? 32 * kWarps : 32 * kForwardWarps)
forward_kernel(const Forward p) {
    constexpr int kBlockWarps = kWarps > kForwardWarps ? kWarps : kForwardWarps;
    constexpr int kGroups = kBlockWarps / kWarps, kLanes = 32 * kWarps;
    __shared__ float part[2][kBlockWarps];
    const int lane = threadIdx.x % kLanes, warp = threadIdx.x >> 5, group = threadIdx.x / kLanes;
    const uint64_t groups = static_cast<uint64_t>(gridDim.x) * kGroups, mine = static_cast<uint64_t>(blockIdx.x) * kGroups + group;
    const uint32_t r0 = static_cast<uint32_t>(p.rows * mine / groups), r1 = static_cast<uint32_t>(p.rows * (mine + 1) / groups);
    if (r0 >= r1) return;               // the whole group: its barrier is its own
    const int pieces = p.K >> 3;
    auto load_row = [&](uint4 (&raw)[kChunks], uint32_t m) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
            raw[i] = lane + i * kLanes < pieces ? load8(p.x + m * p.ldx + 8 * (lane + i * kLanes)) : make_uint4(0, 0, 0, 0);
    };
    // the sum over the row's lanes in a fixed order; the two buffers take turns, so one barrier a sum is enough
    auto row_sum = [&](float v, int b) {
        v = warp_sum(v);
        if (kWarps == 1) return v;
        if ((threadIdx.x & 31) == 0) part[b][warp] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(kLanes) : "memory");
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += part[b][group * kWarps + w];
        return s;
    };
    const uint64_t o2 = twice(p.offset);
    uint4 gain[kChunks], shift[kChunks], raw[kChunks];
    uint32_t left = 0;                  // rows of the sample whose scale and shift are held
    load_row(raw, r0);
    for (uint32_t m = r0; m < r1; ++m, --left) {
        if (left == 0) {
            const uint32_t sample = m / p.rows_per_sample;
            left = p.rows_per_sample - (m - sample * p.rows_per_sample);
            const int64_t s = static_cast<int64_t>(sample) * p.ld_mod;
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                const int c = 8 * (lane + i * kLanes);
                gain[i] = p.scale != nullptr && c < p.K ? cached8(p.scale + s + c) : make_uint4(0, 0, 0, 0);
                shift[i] = p.shift != nullptr && c < p.K ? cached8(p.shift + s + c) : make_uint4(0, 0, 0, 0);
            }
        }
        uint4 next[kChunks];
        if (m + 1 < r1) load_row(next, m + 1);
        uint64_t s2 = 0;
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
            s2 = add2(s2, add2(add2(f32x2_of_bf16x2(raw[i].x), f32x2_of_bf16x2(raw[i].y)), add2(f32x2_of_bf16x2(raw[i].z), f32x2_of_bf16x2(raw[i].w))));
        const float mean = row_sum(sum_lanes(s2), 0) * p.inv_k;
        const uint64_t nm = twice(-mean);
        uint64_t q2 = 0;
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            if (lane + i * kLanes < pieces) {
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint64_t d = add2(f32x2_of_bf16x2(w[e]), nm);
                    q2 = fma2(d, d, q2);
                }
            }
        }
        const float rstd = 1.0f / sqrtf(fmaf(row_sum(sum_lanes(q2), 1), p.inv_k, p.eps));
        if (p.stats != nullptr && lane == 0) p.stats[m] = make_float2(mean, rstd);
        uint16_t *y = p.y + m * p.ldy;
        const uint64_t r2 = twice(rstd);
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int c = 8 * (lane + i * kLanes);
            if (lane + i * kLanes < pieces) {
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                const uint32_t gw[4] = {gain[i].x, gain[i].y, gain[i].z, gain[i].w}, bw[4] = {shift[i].x, shift[i].y, shift[i].z, shift[i].w};
                uint32_t out[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint64_t xhat = mul2(add2(f32x2_of_bf16x2(w[e]), nm), r2);
                    out[e] = pack2(fma2(xhat, add2(f32x2_of_bf16x2(gw[e]), o2), f32x2_of_bf16x2(bw[e])));
                }
                *reinterpret_cast<uint4 *>(y + c) = make_uint4(out[0], out[1], out[2], out[3]);
            }
        }
#pragma unroll
        for (int i = 0; i < kChunks; ++i) raw[i] = next[i];
    }
}

// ------------------------------------------------------------------------------------------------ gradients
struct Backward {
    const uint16_t *dy, *x, *scale;
    const float2 *stats;
    uint16_t *dx;
    float *dscale, *dshift;     // [samples, K] or null
    float *partials;            // [items][2][K] where a sample has several pieces
    int64_t ld_dy, ld_x, ld_dx, ld_scale;
    uint32_t rows, rows_per_sample;
    int K, samples, pieces;     // pieces of a sample
    int warps_per_row;
    float offset, inv_k;
};

constexpr int kMaxWarps = 16;           // of a block, at most (twelve where 168 registers a thread are wanted: up to 3072 columns and from 4097 to 6144)
constexpr int kGroupColumns = 256;      // columns of a warp and piece
// Sums of kValues (a power of two up to 32) values over the warp: lane l ends up with that of value l >> (5 - log2 kValues).
template <int kValues>
__device__ __forceinline__ float transpose_sum(float (&v)[kValues], int lane) {
    int n = kValues;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (n > 1) {
            n >>= 1;
            const bool up = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < kValues / 2; ++i)
                if (i < n) {
                    const float keep = up ? v[i + n] : v[i], give = up ? v[i] : v[i + n];
                    v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, o);
                }
        } else {
            v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], o);
        }
    }
    return v[0];
}

// kRows rows a step of a group; kAhead: the next step's rows are under way meanwhile.
template <int kChunks, int kRows, int kWarps, bool kAhead>
__global__ void __launch_bounds__(32 * kWarps, 1)
backward_kernel(const Backward p) {
    constexpr int kValues = 2 * kRows;
    constexpr int kLanesPer = 32 / kValues;                   // lanes that hold one value after the warp's sum
    __shared__ float part[2][kMaxWarps][kValues];             // [buffer][warp]
    __shared__ __align__(16) float across[kMaxWarps * kGroupColumns];   // the groups' sums: eight columns a thread
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per_row = p.warps_per_row;
    const int groups = (blockDim.x >> 5) / per_row, group = warp / per_row, first_warp = group * per_row;
    const int lanes = 32 * per_row, at = threadIdx.x - 32 * first_warp;
    const int columns8 = p.K >> 3;
    const uint32_t stride = groups * kRows;
    struct Step {
        uint4 x[kRows][kChunks], dy[kRows][kChunks];
        float2 stats[kRows];
    };
    const uint64_t o2 = twice(p.offset);
    int buffer = 0;
    int place[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) place[i] = at + i * lanes < columns8 ? 8 * (at + i * lanes) : 0;
    for (int item = blockIdx.x; item < p.samples * p.pieces; item += gridDim.x) {
        const int sample = item / p.pieces, piece = item - sample * p.pieces;
        const uint32_t s0 = static_cast<uint32_t>(sample) * p.rows_per_sample, len = min(p.rows_per_sample, p.rows - s0);
        // the piece's steps, `stride` rows each: all whole but the sample's last one
        const uint64_t steps = (len + stride - 1) / stride;
        const uint32_t t0 = static_cast<uint32_t>(steps * piece / p.pieces), t1 = static_cast<uint32_t>(steps * (piece + 1) / p.pieces);
        const uint32_t end = s0 + len;
        uint64_t gain[kChunks][4], acc_scale[kChunks][4], acc_shift[kChunks][4];
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            uint4 g = make_uint4(0, 0, 0, 0);
            const bool there = at + i * lanes < columns8;
            if (p.scale != nullptr && there) g = cached8(p.scale + static_cast<int64_t>(sample) * p.ld_scale + 8 * (at + i * lanes));
            const uint32_t gw[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                gain[i][e] = there ? add2(f32x2_of_bf16x2(gw[e]), o2) : 0;
                acc_scale[i][e] = acc_shift[i][e] = 0;
            }
        }
        // rows that do not exist read as 0; a lane without columns reads the first ones, which its gain of 0 takes out of the sums
        auto fetch = [&](Step &s, uint32_t base, auto whole) {
            const uint16_t *x = p.x + base * p.ld_x, *dy = p.dy + base * p.ld_dy;
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const bool there = decltype(whole)::value || base + j < end;
                s.stats[j] = there ? __ldg(p.stats + base + j) : make_float2(0.0f, 0.0f);
#pragma unroll
                for (int i = 0; i < kChunks; ++i) {
                    s.x[j][i] = there ? load8(x + j * p.ld_x + place[i]) : make_uint4(0, 0, 0, 0);
                    s.dy[j][i] = there ? load8(dy + j * p.ld_dy + place[i]) : make_uint4(0, 0, 0, 0);
                }
            }
        };
        auto work = [&](const Step &s, uint32_t base, auto whole) {
            float sums[kValues];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                uint64_t s1 = 0, s2 = 0;
                const uint64_t r2 = twice(s.stats[j].y), back = twice(-s.stats[j].x * s.stats[j].y);
#pragma unroll
                for (int i = 0; i < kChunks; ++i) {
                    const uint32_t xw[4] = {s.x[j][i].x, s.x[j][i].y, s.x[j][i].z, s.x[j][i].w};
                    const uint32_t dw[4] = {s.dy[j][i].x, s.dy[j][i].y, s.dy[j][i].z, s.dy[j][i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t d = f32x2_of_bf16x2(dw[e]), dxhat = mul2(d, fma2(f32x2_of_bf16x2(xw[e]), r2, back));
                        s1 = fma2(d, gain[i][e], s1);
                        s2 = fma2(dxhat, gain[i][e], s2);
                        acc_shift[i][e] = add2(acc_shift[i][e], d);
                        acc_scale[i][e] = add2(acc_scale[i][e], dxhat);
                    }
                }
                sums[2 * j] = sum_lanes(s1);
                sums[2 * j + 1] = sum_lanes(s2);
            }
            float total = transpose_sum<kValues>(sums, lane);
            if (per_row > 1) {
                // the two buffers take turns, so one barrier a step is enough
                if (lane % kLanesPer == 0) part[buffer][warp][lane / kLanesPer] = total;
                asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(lanes) : "memory");
                total = 0.0f;
                for (int w = lane % kLanesPer; w < per_row; w += kLanesPer) total += part[buffer][first_warp + w][lane / kLanesPer];
#pragma unroll
                for (int o = 1; o < kLanesPer; o <<= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
                buffer ^= 1;
            }
            total *= p.inv_k;
            uint16_t *out = p.dx + base * p.ld_dx;
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const float mean_w = __shfl_sync(0xFFFFFFFFu, total, 2 * j * kLanesPer);
                const float mean_wx = __shfl_sync(0xFFFFFFFFu, total, (2 * j + 1) * kLanesPer);
                // rstd (w - mean_w - xhat mean_wx), with xhat = x rstd - mean rstd, as d (gain rstd) + x a + b
                const float rstd = s.stats[j].y, a = -rstd * rstd * mean_wx;
                const uint64_t r2 = twice(rstd), a2 = twice(a), b2 = twice(-fmaf(a, s.stats[j].x, rstd * mean_w));
#pragma unroll
                for (int i = 0; i < kChunks; ++i) {
                    const uint32_t xw[4] = {s.x[j][i].x, s.x[j][i].y, s.x[j][i].z, s.x[j][i].w};
                    const uint32_t dw[4] = {s.dy[j][i].x, s.dy[j][i].y, s.dy[j][i].z, s.dy[j][i].w};
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = pack2(fma2(f32x2_of_bf16x2(xw[e]), a2, fma2(f32x2_of_bf16x2(dw[e]), mul2(gain[i][e], r2), b2)));
                    if ((decltype(whole)::value || base + j < end) && at + i * lanes < columns8)
                        *reinterpret_cast<uint4 *>(out + j * p.ld_dx + place[i]) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
        };
        // whole steps, each one's rows asked for while the one before is worked on (where the registers hold both)
        uint32_t base = s0 + t0 * stride + group * kRows, left = t1 - t0;
        const bool tail = left > 0 && base + (left - 1) * stride + kRows > end;     // this group's last step
        if (tail) --left;
        Step next;
        if (kAhead && left > 0) fetch(next, base, std::true_type{});
#pragma unroll 1
        for (; left > 0; --left, base += stride) {
            if constexpr (kAhead) {
                const Step now = next;
                if (left > 1) fetch(next, base + stride, std::true_type{});
                work(now, base, std::true_type{});
            } else {
                fetch(next, base, std::true_type{});
                work(next, base, std::true_type{});
            }
        }
        if (tail) {
            fetch(next, base, std::false_type{});
            work(next, base, std::false_type{});
        }
        // the groups' sums in order of the groups, one of the two gradients at a time
        const bool whole = p.pieces == 1;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float *to = which == 0 ? p.dscale : p.dshift;
            if (to == nullptr) continue;
            to = whole ? to + static_cast<int64_t>(sample) * p.K : p.partials + (2 * static_cast<int64_t>(item) + which) * p.K;
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) f32x2_split(which == 0 ? acc_scale[i][e] : acc_shift[i][e], v[2 * e], v[2 * e + 1]);
                if (groups > 1) {
                    float4 *mine = reinterpret_cast<float4 *>(across) + (group * lanes + at) * 2;
                    mine[0] = make_float4(v[0], v[1], v[2], v[3]);
                    mine[1] = make_float4(v[4], v[5], v[6], v[7]);
                    __syncthreads();
                    if (group == 0) {
                        for (int g = 1; g < groups; ++g) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] += across[(g * lanes + at) * 8 + e];
                        }
                    }
                    __syncthreads();
                }
                const int c = at + i * lanes;
                if (group == 0 && c < columns8) {
                    reinterpret_cast<float4 *>(to + 8 * c)[0] = make_float4(v[0], v[1], v[2], v[3]);
                    reinterpret_cast<float4 *>(to + 8 * c)[1] = make_float4(v[4], v[5], v[6], v[7]);
                }
            }
        }
    }
}

// Sum of a sample's pieces, in FP64 and in order within each of the strips that the threads take.
constexpr int kStrips = 16;
__global__ void __launch_bounds__(32 * kStrips)
reduce_kernel(const float *__restrict__ partials, int K, int pieces, float *dscale, float *dshift) {
    __shared__ double part[kStrips][32];
    const int sample = blockIdx.y, which = blockIdx.z, strip = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + (threadIdx.x & 31);
    float *to = which == 0 ? dscale : dshift;
    ptx::grid_dependency_wait();
    if (to == nullptr) return;
    double v = 0.0;
    if (c < K) {
#pragma unroll 8
        for (int i = strip; i < pieces; i += kStrips) v += partials[(2 * (static_cast<int64_t>(sample) * pieces + i) + which) * K + c];
    }
    part[strip][threadIdx.x & 31] = v;
    __syncthreads();
    if (strip != 0 || c >= K) return;
#pragma unroll
    for (int i = 1; i < kStrips; ++i) v += part[i][threadIdx.x & 31];
    to[static_cast<int64_t>(sample) * K + c] = static_cast<float>(v);
}

constexpr int kMaxItems = 512;      // pieces in all, where a sample has more than one

struct Shape {
    int variant, chunks, rows, warps_per_row, groups;
};
// A thread holds `chunks` pieces of eight columns of `rows` rows, and as many again of the next ones, in what a block of twelve (168
// registers a thread) or sixteen warps (128) leaves it beside the sums and the gain.  Up to 3072 columns as many groups as twelve
// warps make; beyond, one.  Measured (gradients of 28.3 M values, two samples; in brackets other forms' time in terms of this one's, taken at
// 25 to 34 M): 4096 columns 35 us (two pieces, eight warps: 1.2), 6144 43, 8192 41 (two rows with spills: 1.7; four pieces: 2.1), 12288 65 (with
// the next row: 1.2; four pieces: 1.15), 16384 84 (twelve warps and the next row: 1.4): there the sums alone take half the registers.
constexpr int kVariants = 6;
constexpr int kLimit[kVariants] = {3072, 4096, 6144, 8192, 12288, 16384}, kChunksOf[kVariants] = {1, 1, 2, 2, 3, 4}, kRowsOf[kVariants] = {4, 2, 2, 1, 1, 1};
Shape shape_of(int64_t K) {
    Shape s{};
    while (K > kLimit[s.variant]) ++s.variant;
    s.chunks = kChunksOf[s.variant];
    s.rows = kRowsOf[s.variant];
    s.warps_per_row = static_cast<int>(ceil_div(K, kGroupColumns * s.chunks));
    s.groups = s.variant == 0 ? 12 / s.warps_per_row : 1;
    return s;
}
// Pieces of a sample: as many as there are blocks for each sample (rounded down, at least one: where samples are more than half as many as
// blocks, and no multiple of them, some blocks have less to do), none of fewer rows than the groups take in a step.
int pieces_of(int64_t M, int64_t rows_per_sample, const Shape &s, int blocks) {
    const int64_t samples = ceil_div(M, rows_per_sample);
    const int64_t most = ceil_div(rows_per_sample < M ? rows_per_sample : M, s.groups * s.rows);
    int64_t pieces = blocks / samples;
    if (pieces > most) pieces = most;
    return pieces < 1 ? 1 : static_cast<int>(pieces);
}

template <int kWarps, int kChunks>
sol_status_t forward_of(const Forward &p, cudaStream_t stream, const DeviceInfo *dev) {
    constexpr int kBlockWarps = kWarps > kForwardWarps ? kWarps : kForwardWarps;
    static std::atomic<int> known[64];  // by device: blocks per SM that the kernel's registers allow
    int resident = known[dev->device].load(std::memory_order_relaxed);
    if (resident == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, forward_kernel<kWarps, kChunks>, 32 * kBlockWarps, 0) != cudaSuccess) {
            cudaGetLastError();
            return SOL_ERR_CUDA;
        }
        known[dev->device].store(resident, std::memory_order_relaxed);
    }
    const int64_t most = static_cast<int64_t>(resident) * dev->sm_count, want = ceil_div(p.rows, kBlockWarps / kWarps);
    forward_kernel<kWarps, kChunks><<<static_cast<unsigned>(want < most ? want : most), 32 * kBlockWarps, 0, stream>>>(p);
    return launch_status();
}
template <int kWarps>
sol_status_t forward_by_chunks(const Forward &p, cudaStream_t stream, const DeviceInfo *dev) {
    switch (ceil_div(p.K, 256 * kWarps)) {
        case 1: return forward_of<kWarps, 1>(p, stream, dev);
        case 2: return forward_of<kWarps, 2>(p, stream, dev);
        case 3: return forward_of<kWarps, 3>(p, stream, dev);
    }
    if constexpr (kWarps == 16) return forward_of<kWarps, 4>(p, stream, dev);
    return SOL_ERR_BAD_SHAPE;
}

}  // namespace

int max_k() { return kMaxK; }

sol_status_t launch_forward(const void *x, int64_t M, int64_t K, int64_t ldx, const void *scale, const void *shift, int64_t ld_mod,
                            int64_t rows_per_sample, float offset, float eps, void *y, int64_t ldy, float *stats, cudaStream_t stream,
                            const DeviceInfo *dev) {
    const Forward p{static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(scale), static_cast<const uint16_t *>(shift),
                    static_cast<uint16_t *>(y), reinterpret_cast<float2 *>(stats), ldx, ldy, ld_mod, static_cast<uint32_t>(M),
                    static_cast<uint32_t>(rows_per_sample), static_cast<int>(K), scale != nullptr ? offset : 1.0f, eps,
                    1.0f / static_cast<float>(K)};
    if (K <= 768) return forward_by_chunks<1>(p, stream, dev);
    if (K <= 1536) return forward_by_chunks<2>(p, stream, dev);
    if (K <= 3072) return forward_by_chunks<4>(p, stream, dev);
    if (K <= 6144) return forward_by_chunks<8>(p, stream, dev);
    return forward_by_chunks<16>(p, stream, dev);
}

size_t backward_workspace_bytes(int64_t M, int64_t K, int64_t rows_per_sample) {
    const int pieces = pieces_of(M, rows_per_sample, shape_of(K), kMaxItems);
    return pieces == 1 ? 0 : sizeof(float) * 2 * static_cast<size_t>(K) * static_cast<size_t>(pieces) * static_cast<size_t>(ceil_div(M, rows_per_sample));
}

sol_status_t launch_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const float *stats, const void *scale,
                             int64_t ld_scale, int64_t M, int64_t K, int64_t rows_per_sample, float offset, void *dx, int64_t ld_dx, float *dscale, float *dshift,
                             float *partials, cudaStream_t stream, const DeviceInfo *dev) {
    const Shape s = shape_of(K);
    const int64_t samples = ceil_div(M, rows_per_sample);
    const int blocks = dev->sm_count < kMaxItems ? dev->sm_count : kMaxItems;
    const Backward p{static_cast<const uint16_t *>(dy), static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(scale),
                     reinterpret_cast<const float2 *>(stats), static_cast<uint16_t *>(dx), dscale, dshift, partials,
                     ld_dy, ld_x, ld_dx, ld_scale, static_cast<uint32_t>(M), static_cast<uint32_t>(rows_per_sample),
                     static_cast<int>(K), static_cast<int>(samples), pieces_of(M, rows_per_sample, s, blocks), s.warps_per_row,
                     scale != nullptr ? offset : 1.0f, 1.0f / static_cast<float>(K)};
    const int64_t items = samples * p.pieces;
    const unsigned grid = static_cast<unsigned>(items < blocks ? items : blocks), threads = 32u * s.warps_per_row * s.groups;
    auto launch = [&](auto kern) { kern<<<grid, threads, 0, stream>>>(p); };
    switch (s.variant) {
        case 0: launch(backward_kernel<1, 4, 12, true>); break;
        case 1: launch(backward_kernel<1, 2, 16, true>); break;
        case 2: launch(backward_kernel<2, 2, 12, true>); break;
        case 3: launch(backward_kernel<2, 1, 16, true>); break;
        case 4: launch(backward_kernel<3, 1, 16, false>); break;
        default: launch(backward_kernel<4, 1, 16, false>); break;
    }
    const sol_status_t st = launch_status();
    if (st != SOL_OK || p.pieces == 1 || (dscale == nullptr && dshift == nullptr)) return st;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(ceil_div(K, 32)), static_cast<unsigned>(samples), 2);
    cfg.blockDim = dim3(32 * kStrips);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, reduce_kernel, static_cast<const float *>(partials), static_cast<int>(K), p.pieces, dscale, dshift) != cudaSuccess) {
        cudaGetLastError();
        return SOL_ERR_CUDA;
    }
    return launch_status();
}

}  // namespace norm
}  // namespace sol
