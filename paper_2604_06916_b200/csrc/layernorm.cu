// Layer norm with the modulation of a DiT block (or a plain weight), forward and gradients, in BF16 (sm_100a).
//
// The training pass's form of the rollout's norm (which quantizes its output and keeps nothing).  Per row m of sample s:
//     xhat = (x - mean) rstd,  rstd = 1 / sqrt(var + eps);     y = xhat gain + shift,  gain = offset + scale[s]
// and with w = dy gain, the gradients
//     dx = rstd (w - mean(w) - xhat mean(w xhat)),   dscale[s] = sum over the sample's rows of dy xhat,   dshift[s] = sum of dy.
// HBM bound: 4 bytes per element forward, 6 backward.
//
// Forward: a warp (wide rows: four warps) holds a row in registers, so mean, variance (of the centred values) and output
// take one read of x; scale and shift come from the caches.
//
// Gradients: a thread owns the same eight columns of every row that its block walks, so that the sums over rows stay in its
// registers; the two row means go over the block (a group of warps per row, as many groups as fit the block) once per kRows
// rows.  A block's sums leave as FP32 partials, which a second launch adds up in FP64 in a fixed order: equal inputs give
// equal bits.
#include "ptx.cuh"
#include "quant_math.cuh"
#include "sol_internal.h"

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
    const uint16_t *x, *scale, *shift;   // scale, shift: [samples, K] or null
    uint16_t *y;
    float2 *stats;                       // [M] (mean, rstd) or null
    int64_t ldx, ldy;
    uint32_t rows, rows_per_sample;
    int K;
    float offset, eps, inv_k;
};

constexpr int kForwardWarps = 8;

// kWarps warps share a row; a lane holds kChunks pieces of eight columns.
template <int kWarps, int kChunks>
__global__ void __launch_bounds__(32 * kForwardWarps)
forward_kernel(const Forward p) {
    constexpr int kRows = kForwardWarps / kWarps, kLanes = 32 * kWarps;
    __shared__ float part[2][kForwardWarps];
    const int lane = threadIdx.x % kLanes, warp = threadIdx.x >> 5;
    const uint32_t m = blockIdx.x * kRows + threadIdx.x / kLanes;
    const bool there = m < p.rows;
    if (kWarps == 1 && !there) return;
    const int pieces = there ? p.K >> 3 : 0;
    const uint16_t *x = p.x + m * p.ldx;
    uint4 raw[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) raw[i] = lane + i * kLanes < pieces ? load8(x + 8 * (lane + i * kLanes)) : make_uint4(0, 0, 0, 0);
    // the sum over the row's lanes, in a fixed order; buffer b is written once
    auto row_sum = [&](float v, int b) {
        v = warp_sum(v);
        if (kWarps == 1) return v;
        if ((threadIdx.x & 31) == 0) part[b][warp] = v;
        __syncthreads();
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += part[b][warp / kWarps * kWarps + w];
        return s;
    };
    uint64_t s2 = 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        s2 = add2(s2, add2(add2(f32x2_of_bf16x2(raw[i].x), f32x2_of_bf16x2(raw[i].y)), add2(f32x2_of_bf16x2(raw[i].z), f32x2_of_bf16x2(raw[i].w))));
    }
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
    if (!there) return;
    if (p.stats != nullptr && lane == 0) p.stats[m] = make_float2(mean, rstd);
    const int64_t s = static_cast<int64_t>(m / p.rows_per_sample) * p.K;
    uint16_t *y = p.y + m * p.ldy;
    const uint64_t r2 = twice(rstd), o2 = twice(p.offset);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = 8 * (lane + i * kLanes);
        if (lane + i * kLanes < pieces) {
            const uint4 g = p.scale != nullptr ? cached8(p.scale + s + c) : make_uint4(0, 0, 0, 0);
            const uint4 b = p.shift != nullptr ? cached8(p.shift + s + c) : make_uint4(0, 0, 0, 0);
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w}, gw[4] = {g.x, g.y, g.z, g.w}, bw[4] = {b.x, b.y, b.z, b.w};
            uint32_t out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint64_t xhat = mul2(add2(f32x2_of_bf16x2(w[e]), nm), r2);
                out[e] = pack2(fma2(xhat, add2(f32x2_of_bf16x2(gw[e]), o2), f32x2_of_bf16x2(bw[e])));
            }
            *reinterpret_cast<uint4 *>(y + c) = make_uint4(out[0], out[1], out[2], out[3]);
        }
    }
}

// ------------------------------------------------------------------------------------------------ gradients
struct Backward {
    const uint16_t *dy, *x, *scale;
    const float2 *stats;
    uint16_t *dx;
    float *dscale, *dshift;     // [samples, K] or null
    float *partials;            // [items][2][K] where a sample has several pieces
    int64_t ld_dy, ld_x, ld_dx;
    uint32_t rows, rows_per_sample;
    int K, samples, pieces;     // pieces of a sample
    float offset, inv_k;
};

constexpr int kMaxWarps = 16;           // of a block
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

template <int kChunks, int kRows>
__global__ void __launch_bounds__(32 * kMaxWarps, 1)
backward_kernel(const Backward p, int warps_per_row) {
    constexpr int kValues = 2 * kRows;
    constexpr int kLanesPer = 32 / kValues;                   // lanes that hold one value after the warp's sum
    __shared__ float part[2][kMaxWarps][kValues];             // [buffer][warp]
    __shared__ __align__(16) float across[kChunks == 1 ? kMaxWarps * kGroupColumns : 4];   // the groups' sums: eight columns a thread
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int groups = (blockDim.x >> 5) / warps_per_row, group = warp / warps_per_row, first_warp = group * warps_per_row;
    const int lanes = 32 * warps_per_row, at = threadIdx.x - 32 * first_warp;
    const int columns8 = p.K >> 3;
    const uint64_t o2 = twice(p.offset);
    int buffer = 0;
    for (int item = blockIdx.x; item < p.samples * p.pieces; item += gridDim.x) {
        const int sample = item / p.pieces, piece = item - sample * p.pieces;
        const uint32_t s0 = static_cast<uint32_t>(sample) * p.rows_per_sample;
        const uint32_t len = min(p.rows_per_sample, p.rows - s0);
        const uint32_t r0 = s0 + static_cast<uint32_t>(static_cast<uint64_t>(len) * piece / p.pieces);
        const uint32_t r1 = s0 + static_cast<uint32_t>(static_cast<uint64_t>(len) * (piece + 1) / p.pieces);
        uint4 gain[kChunks];
        uint64_t acc_scale[kChunks][4], acc_shift[kChunks][4];
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            gain[i] = make_uint4(0, 0, 0, 0);
            if (p.scale != nullptr && at + i * lanes < columns8) gain[i] = cached8(p.scale + static_cast<int64_t>(sample) * p.K + 8 * (at + i * lanes));
#pragma unroll
            for (int e = 0; e < 4; ++e) acc_scale[i][e] = acc_shift[i][e] = 0;
        }
        // every group takes as many steps: the barrier below is its own, the block's only at the end
        for (uint32_t base = r0 + group * kRows; base < r1; base += groups * kRows) {
            uint4 raw_x[kRows][kChunks], raw_d[kRows][kChunks];
            float2 st[kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const bool there = base + j < r1;
                st[j] = there ? __ldg(p.stats + base + j) : make_float2(0.0f, 0.0f);
#pragma unroll
                for (int i = 0; i < kChunks; ++i) {
                    raw_x[j][i] = raw_d[j][i] = make_uint4(0, 0, 0, 0);
                    if (there && at + i * lanes < columns8) {
                        raw_x[j][i] = load8(p.x + (base + j) * p.ld_x + 8 * (at + i * lanes));
                        raw_d[j][i] = load8(p.dy + (base + j) * p.ld_dy + 8 * (at + i * lanes));
                    }
                }
            }
            float sums[kValues];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const uint64_t r2 = twice(st[j].y), back = twice(-st[j].x * st[j].y);
                uint64_t s1 = 0, s2 = 0;
#pragma unroll
                for (int i = 0; i < kChunks; ++i) {
                    const uint32_t xw[4] = {raw_x[j][i].x, raw_x[j][i].y, raw_x[j][i].z, raw_x[j][i].w};
                    const uint32_t dw[4] = {raw_d[j][i].x, raw_d[j][i].y, raw_d[j][i].z, raw_d[j][i].w};
                    const uint32_t gw[4] = {gain[i].x, gain[i].y, gain[i].z, gain[i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t xhat = fma2(f32x2_of_bf16x2(xw[e]), r2, back), d = f32x2_of_bf16x2(dw[e]);
                        const uint64_t w = mul2(d, add2(f32x2_of_bf16x2(gw[e]), o2));
                        s1 = add2(s1, w);
                        s2 = fma2(w, xhat, s2);
                        acc_shift[i][e] = add2(acc_shift[i][e], d);
                        acc_scale[i][e] = fma2(d, xhat, acc_scale[i][e]);
                    }
                }
                sums[2 * j] = sum_lanes(s1);
                sums[2 * j + 1] = sum_lanes(s2);
            }
            float total = transpose_sum<kValues>(sums, lane);
            if (warps_per_row > 1) {
                if (lane % kLanesPer == 0) part[buffer][warp][lane / kLanesPer] = total;
                asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(lanes) : "memory");
                total = 0.0f;
                for (int w = lane % kLanesPer; w < warps_per_row; w += kLanesPer) total += part[buffer][first_warp + w][lane / kLanesPer];
#pragma unroll
                for (int o = 1; o < kLanesPer; o <<= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
                buffer ^= 1;
            }
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const float mean_w = __shfl_sync(0xFFFFFFFFu, total, 2 * j * kLanesPer) * p.inv_k;
                const float mean_wx = __shfl_sync(0xFFFFFFFFu, total, (2 * j + 1) * kLanesPer) * p.inv_k;
                if (base + j < r1) {
                    const uint64_t r2 = twice(st[j].y), back = twice(-st[j].x * st[j].y);
                    const uint64_t n1 = twice(-mean_w), n2 = twice(-mean_wx);
#pragma unroll
                    for (int i = 0; i < kChunks; ++i) {
                        const uint32_t xw[4] = {raw_x[j][i].x, raw_x[j][i].y, raw_x[j][i].z, raw_x[j][i].w};
                        const uint32_t dw[4] = {raw_d[j][i].x, raw_d[j][i].y, raw_d[j][i].z, raw_d[j][i].w};
                        const uint32_t gw[4] = {gain[i].x, gain[i].y, gain[i].z, gain[i].w};
                        uint32_t out[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint64_t xhat = fma2(f32x2_of_bf16x2(xw[e]), r2, back);
                            const uint64_t w = mul2(f32x2_of_bf16x2(dw[e]), add2(f32x2_of_bf16x2(gw[e]), o2));
                            out[e] = pack2(mul2(r2, add2(w, fma2(xhat, n2, n1))));
                        }
                        if (at + i * lanes < columns8)
                            *reinterpret_cast<uint4 *>(p.dx + (base + j) * p.ld_dx + 8 * (at + i * lanes)) = make_uint4(out[0], out[1], out[2], out[3]);
                    }
                }
            }
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
                const int c = at + i * lanes;
                if (groups > 1) {      // one chunk only: c < lanes
                    float4 *mine = reinterpret_cast<float4 *>(across) + (group * lanes + c) * 2;
                    mine[0] = make_float4(v[0], v[1], v[2], v[3]);
                    mine[1] = make_float4(v[4], v[5], v[6], v[7]);
                    __syncthreads();
                    if (group == 0) {
                        for (int g = 1; g < groups; ++g) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] += across[(g * lanes + c) * 8 + e];
                        }
                    }
                    __syncthreads();
                }
                if (group == 0 && c < columns8) {
                    reinterpret_cast<float4 *>(to + 8 * c)[0] = make_float4(v[0], v[1], v[2], v[3]);
                    reinterpret_cast<float4 *>(to + 8 * c)[1] = make_float4(v[4], v[5], v[6], v[7]);
                }
            }
        }
    }
}

// Sum of a sample's pieces, in FP64 and in order within each of the strips that the threads take.
constexpr int kStrips = 8;
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
#pragma unroll 4
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
    int chunks, warps_per_row, groups, blocks_per_sm;
};
// A thread holds one piece of eight columns of a row up to 4096 columns, two up to 8192, four beyond; blocks of up to sixteen warps.
Shape shape_of(int64_t K) {
    Shape s;
    s.chunks = K <= 4096 ? 1 : K <= 8192 ? 2 : 4;
    s.warps_per_row = static_cast<int>(ceil_div(K, kGroupColumns * s.chunks));
    s.groups = s.chunks > 1 ? 1 : 12 / s.warps_per_row > 0 ? 12 / s.warps_per_row : 1;
    s.blocks_per_sm = 1;
    return s;
}
int rows_of(int chunks) { return chunks == 1 ? 4 : chunks == 2 ? 2 : 1; }
// Pieces of a sample: so many that the blocks all have one, none of fewer rows than the groups take in a step.
int pieces_of(int64_t M, int64_t rows_per_sample, const Shape &s, int blocks) {
    const int64_t samples = ceil_div(M, rows_per_sample);
    const int64_t most = ceil_div(rows_per_sample < M ? rows_per_sample : M, s.groups * rows_of(s.chunks));
    int64_t pieces = blocks / samples;
    if (pieces > most) pieces = most;
    return pieces < 1 ? 1 : static_cast<int>(pieces);
}

template <int kWarps>
sol_status_t forward_of(const Forward &p, cudaStream_t stream) {
    const unsigned grid = static_cast<unsigned>(ceil_div(p.rows, kForwardWarps / kWarps));
    const int chunks = static_cast<int>(ceil_div(p.K, 256 * kWarps));
    auto launch = [&](auto kern) { kern<<<grid, 32 * kForwardWarps, 0, stream>>>(p); };
    if (chunks <= 1) launch(forward_kernel<kWarps, 1>);
    else if (chunks <= 2) launch(forward_kernel<kWarps, 2>);
    else if (chunks <= 4) launch(forward_kernel<kWarps, 4>);
    else if (chunks <= 6) launch(forward_kernel<kWarps, 6>);
    else if (chunks <= 8) launch(forward_kernel<kWarps, 8>);
    else if (chunks <= 10) launch(forward_kernel<kWarps, 10>);
    else if (chunks <= 12) launch(forward_kernel<kWarps, 12>);
    else launch(forward_kernel<kWarps, 16>);
    return launch_status();
}

}  // namespace

int max_k() { return kMaxK; }

sol_status_t launch_forward(const void *x, int64_t M, int64_t K, int64_t ldx, const void *scale, const void *shift,
                            int64_t rows_per_sample, float offset, float eps, void *y, int64_t ldy, float *stats, cudaStream_t stream,
                            const DeviceInfo *dev) {
    const Forward p{static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(scale), static_cast<const uint16_t *>(shift),
                    static_cast<uint16_t *>(y), reinterpret_cast<float2 *>(stats), ldx, ldy, static_cast<uint32_t>(M),
                    static_cast<uint32_t>(rows_per_sample), static_cast<int>(K), scale != nullptr ? offset : 1.0f, eps,
                    1.0f / static_cast<float>(K)};
    (void)dev;
    return K <= 4096 ? forward_of<1>(p, stream) : forward_of<4>(p, stream);
}

size_t backward_workspace_bytes(int64_t M, int64_t K, int64_t rows_per_sample) {
    const int pieces = pieces_of(M, rows_per_sample, shape_of(K), kMaxItems);
    return pieces == 1 ? 0 : sizeof(float) * 2 * static_cast<size_t>(K) * static_cast<size_t>(pieces) * static_cast<size_t>(ceil_div(M, rows_per_sample));
}

sol_status_t launch_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const float *stats, const void *scale, int64_t M,
                             int64_t K, int64_t rows_per_sample, float offset, void *dx, int64_t ld_dx, float *dscale, float *dshift,
                             float *partials, cudaStream_t stream, const DeviceInfo *dev) {
    const Shape s = shape_of(K);
    const int64_t samples = ceil_div(M, rows_per_sample);
    int blocks = s.blocks_per_sm * dev->sm_count;
    if (blocks > kMaxItems) blocks = kMaxItems;
    Backward p{static_cast<const uint16_t *>(dy), static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(scale),
               reinterpret_cast<const float2 *>(stats), static_cast<uint16_t *>(dx), dscale, dshift, partials, ld_dy, ld_x, ld_dx,
               static_cast<uint32_t>(M), static_cast<uint32_t>(rows_per_sample), static_cast<int>(K), static_cast<int>(samples),
               pieces_of(M, rows_per_sample, s, blocks), scale != nullptr ? offset : 1.0f, 1.0f / static_cast<float>(K)};
    const int64_t items = samples * p.pieces;
    const unsigned grid = static_cast<unsigned>(items < blocks ? items : blocks), threads = 32u * s.warps_per_row * s.groups;
    if (s.chunks == 1) backward_kernel<1, 4><<<grid, threads, 0, stream>>>(p, s.warps_per_row);
    else if (s.chunks == 2) backward_kernel<2, 2><<<grid, threads, 0, stream>>>(p, s.warps_per_row);
    else backward_kernel<4, 1><<<grid, threads, 0, stream>>>(p, s.warps_per_row);
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
