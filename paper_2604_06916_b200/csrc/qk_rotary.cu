// RMS norm of the query and key heads and rotary positions, forward and gradients (sm_100a).
//
// Between the fused q/k/v projection of a DiT block and its attention, every head of q and k is normalised
// and its leading columns are turned by position-dependent angles.  Per (token, head) row x of kD values:
//     n  = w x / sqrt(mean(x^2) + eps)                     (no weight: n = x)
//     (a, b) of pair i -> s (a cos t - b sin t), s (b cos t + a sin t),   t = position[axis(i)] * freq[i]
// Pairs are neighbours (2i, 2i+1) or halves (i, i + rotary/2); columns behind the rotated ones keep n.
// The gradients: dn = the inverse turn of dy (times s), dx = (w dn - xhat mean(w dn xhat)) / rms, and
// dw = sum over rows of dn xhat with xhat = x / rms.
//
// HBM bound: 4 bytes per element forward, 6 backward.  A warp owns one token and walks its heads; a lane owns the
// same eight columns of every head (in the half layout four and their four partners), so the angles are formed once
// per token and tensor, each by one lane, and handed round by shuffles while the first heads' loads are under way.
// Four heads per lane are loaded before any is used.  Where tokens are few, up to one warp per four-head group shares a
// token.  Measured (B200, inside a graph, q and k of 24 heads x 128 from a fused projection, norm and three axes): forward,
// 8 x 4608 tokens, 143 us = 6.3 TB/s, 97 % of the copy rate (one warp per token and eight heads, with its index divisions and
// angles for each: 195 us); 333 tokens, 4.0 us.  Gradients, 2 x 4608 tokens, 63 to 65 us = 5.3 TB/s, 81 %: 116 registers
// hold both tensors' loads, sixteen warps per SM wait for memory 2.3 cycles per issued instruction.  Two heads per lane
// with 24 warps take 71 us, with the next ones prefetched 73 us.  38 and 19 heads of 64, 4099 tokens: 24 us with eight heads a
// step (sixteen: 27 us, a token's last step then leaves most lanes idle); q and k share the blocks by their steps (half
// each: 29 us).
//
// Angles: position * freq and the reduction to half a turn are in FP64 (a far position times a frequency has
// more significant bits than FP32 holds), the sine and cosine of the remainder in FP32.  Squares, means and
// products are FP32; the only rounding to 16 bits is the output's.
#include "ptx.cuh"
#include "quant_math.cuh"
#include "sol_internal.h"

namespace sol {
namespace rotary {
namespace {

using qmath::bf16_hi;
using qmath::bf16_lo;

constexpr int kWarps = 8;
constexpr int kUnroll = 4;      // heads per lane in flight

// Lanes of a head: kD / 8; a warp holds kRep heads at a time.
template <int kD>
struct Shape {
    static constexpr int kLanes = kD / 8;
    static constexpr int kRep = 32 / kLanes;
    static constexpr int kPairs = kRep >= 4 ? 1 : 4 / kRep;   // pairs whose angle a lane forms itself
    static constexpr int kHeads = kRep * kUnroll;             // heads of a warp's step
    // The gradients hold two tensors: eight heads a step keep narrow heads from idling lanes at the last step of a token.
    static constexpr int kUnrollBack = kRep >= 8 ? 1 : kRep >= 2 ? 8 / kRep : 4;
    static constexpr int kBackResident = kUnrollBack >= 4 ? 2 : 3;    // blocks per SM that the registers then allow
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Columns of slot `s`: `c0` holds four, `c1` the other four (neighbour layout: c1 = c0 + 4).
template <bool kHalf>
__device__ __forceinline__ void columns(int s, int rot, int &c0, int &c1) {
    if (kHalf && 8 * s < rot) {
        c0 = 4 * s;
        c1 = (rot >> 1) + 4 * s;
    } else {
        c0 = 8 * s;
        c1 = 8 * s + 4;
    }
}

template <bool kHalf>
__device__ __forceinline__ uint4 load8(const uint16_t *row, int c0, int c1) {
    if (!kHalf) return __ldcs(reinterpret_cast<const uint4 *>(row + c0));
    const uint2 a = __ldcs(reinterpret_cast<const uint2 *>(row + c0)), b = __ldcs(reinterpret_cast<const uint2 *>(row + c1));
    return make_uint4(a.x, a.y, b.x, b.y);
}
template <bool kHalf>
__device__ __forceinline__ void store8(uint16_t *row, int c0, int c1, uint4 v) {
    if (!kHalf) {
        *reinterpret_cast<uint4 *>(row + c0) = v;
    } else {
        *reinterpret_cast<uint2 *>(row + c0) = make_uint2(v.x, v.y);
        *reinterpret_cast<uint2 *>(row + c1) = make_uint2(v.z, v.w);
    }
}
// A slot's eight values as four two-lane FP32 registers, the pairs' first members, then their second ones
// (a0 a1, a2 a3, b0 b1, b2 b3): in this order the turn and everything else is two-lane arithmetic in both layouts.
struct Slot {
    uint64_t v[4];
};
template <bool kHalf>
__device__ __forceinline__ Slot unpack(uint4 r) {
    using qmath::f32x2;
    if (kHalf)
        return {{f32x2(bf16_lo(r.x), bf16_hi(r.x)), f32x2(bf16_lo(r.y), bf16_hi(r.y)), f32x2(bf16_lo(r.z), bf16_hi(r.z)),
                 f32x2(bf16_lo(r.w), bf16_hi(r.w))}};
    return {{f32x2(bf16_lo(r.x), bf16_lo(r.y)), f32x2(bf16_lo(r.z), bf16_lo(r.w)), f32x2(bf16_hi(r.x), bf16_hi(r.y)),
             f32x2(bf16_hi(r.z), bf16_hi(r.w))}};
}
template <bool kHalf>
__device__ __forceinline__ uint4 pack(const Slot &s) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) qmath::f32x2_split(s.v[i], f[2 * i], f[2 * i + 1]);
    if (kHalf) return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    return make_uint4(pack_bf16(f[0], f[4]), pack_bf16(f[1], f[5]), pack_bf16(f[2], f[6]), pack_bf16(f[3], f[7]));
}
// Memory column of value `e` of a slot (0..3: first members, 4..7: second ones).
template <bool kHalf>
__device__ __forceinline__ int column_of(int e, int c0, int c1) {
    if (kHalf) return e < 4 ? c0 + e : c1 + e - 4;
    return c0 + 2 * (e & 3) + (e >> 2);
}
__device__ __forceinline__ uint64_t twice(float f) { return qmath::f32x2(f, f); }
__device__ __forceinline__ float sum_lanes(uint64_t v) {
    float a, b;
    qmath::f32x2_split(v, a, b);
    return a + b;
}
// (a, b) -> (a c - b s, b c + a s) for the slot's four pairs.
struct Angles {
    uint64_t c[2], s[2], ns[2];   // ns = -s
};
__device__ __forceinline__ void turn(Slot &x, const uint64_t *c, const uint64_t *s, const uint64_t *ns) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint64_t a = x.v[i], b = x.v[i + 2];
        x.v[i] = qmath::fma2(a, c[i], qmath::mul2(b, ns[i]));
        x.v[i + 2] = qmath::fma2(b, c[i], qmath::mul2(a, s[i]));
    }
}

// The slot's columns of a norm weight (read by every warp: cached).
__device__ __forceinline__ uint4 load_weight(const uint16_t *w, int c0, int c1) {
    const uint2 a = __ldg(reinterpret_cast<const uint2 *>(w + c0)), b = __ldg(reinterpret_cast<const uint2 *>(w + c1));
    return make_uint4(a.x, a.y, b.x, b.y);
}

// Sum over the lanes of one head (a power of two of neighbouring lanes): every lane gets it, in a fixed order.
template <int kLanes>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Cosine and sine (times the scale) of the four pairs of this lane's slot at row m.  Called by whole warps.
template <int kD>
__device__ __forceinline__ Angles angles(const Turn &t, int64_t m, int lane) {
    using S = Shape<kD>;
    const int slot = lane % S::kLanes, rep = lane / S::kLanes;
    const int64_t *pos = t.positions + static_cast<int64_t>(static_cast<uint32_t>(m) % t.position_rows) * t.axes;
    float mc[S::kPairs], ms[S::kPairs];
#pragma unroll
    for (int j = 0; j < S::kPairs; ++j) {
        const int pair = 4 * slot + (rep * S::kPairs + j) % 4;
        mc[j] = 1.0f, ms[j] = 0.0f;
        if (2 * pair < t.rot) {
            const int axis = (pair >= t.axis_end[0]) + (pair >= t.axis_end[1]) + (pair >= t.axis_end[2]);
            const double turns = static_cast<double>(__ldg(pos + axis)) * __ldg(t.freqs + pair) * 0.15915494309189533577;
            const float part = static_cast<float>(turns - rint(turns));   // of a turn, in [-1/2, 1/2]
            sincospif(2.0f * part, &ms[j], &mc[j]);
            mc[j] *= t.scale, ms[j] *= t.scale;
        }
    }
    float cs[4], sn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int src = slot + S::kLanes * (i / S::kPairs);
        cs[i] = __shfl_sync(0xFFFFFFFFu, mc[i % S::kPairs], src);
        sn[i] = __shfl_sync(0xFFFFFFFFu, ms[i % S::kPairs], src);
    }
    using qmath::f32x2;
    return {{f32x2(cs[0], cs[1]), f32x2(cs[2], cs[3])}, {f32x2(sn[0], sn[1]), f32x2(sn[2], sn[3])},
            {f32x2(-sn[0], -sn[1]), f32x2(-sn[2], -sn[3])}};
}

// A warp takes one token and every `parts`-th group of its heads; blockIdx.y picks q or k.
template <int kD, bool kHalf>
__global__ void __launch_bounds__(32 * kWarps)
forward_kernel(const Heads2 both, const Turn t, uint32_t rows, int parts_log2, float eps) {
    using S = Shape<kD>;
    const int lane = threadIdx.x & 31;
    const Heads d = blockIdx.y == 0 ? both.h[0] : both.h[1];
    const uint32_t task = blockIdx.x * kWarps + (threadIdx.x >> 5);
    const uint32_t m = task >> parts_log2;
    if (m >= rows) return;
    int c0, c1;
    columns<kHalf>(lane % S::kLanes, t.rot, c0, c1);
    int h = static_cast<int>(task & ((1u << parts_log2) - 1u)) * S::kHeads + lane / S::kLanes;
    const int step = S::kHeads << parts_log2;
    const int heads = d.heads;
    const uint16_t *x = d.x + m * d.ld_in;
    uint16_t *out = d.out + m * d.ld_out;
    uint4 raw[kUnroll];
    auto fetch = [&]() {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            raw[u] = h + u * S::kRep < heads ? load8<kHalf>(x + (h + u * S::kRep) * kD, c0, c1) : make_uint4(0, 0, 0, 0);
    };
    fetch();
    Angles an;
    if (t.rot > 0) an = angles<kD>(t, m, lane);
    const bool mine = c0 < t.rot;    // this lane's columns are rotated ones (a slot is wholly inside or outside)
    const bool norm = d.weight != nullptr;
    Slot w;
    if (norm) w = unpack<kHalf>(load_weight(d.weight, c0, c1));
    for (; h - lane / S::kLanes < heads; h += step) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            Slot f = unpack<kHalf>(raw[u]);
            if (norm) {   // uniform over the warp
                uint64_t ss = qmath::mul2(f.v[0], f.v[0]);
#pragma unroll
                for (int e = 1; e < 4; ++e) ss = qmath::fma2(f.v[e], f.v[e], ss);
                const uint64_t r = twice(rsqrtf(fmaf(head_sum<S::kLanes>(sum_lanes(ss)), 1.0f / kD, eps)));
#pragma unroll
                for (int e = 0; e < 4; ++e) f.v[e] = qmath::mul2(f.v[e], qmath::mul2(r, w.v[e]));
            }
            if (mine) turn(f, an.c, an.s, an.ns);
            raw[u] = pack<kHalf>(f);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (h + u * S::kRep < heads) store8<kHalf>(out + (h + u * S::kRep) * kD, c0, c1, raw[u]);
        if (h - lane / S::kLanes + step < heads) {
            h += step;
            fetch();
            h -= step;
        }
    }
}

// Gradients.  The first blocks_q blocks take q, the others k; blocks stay and walk the (token, part of its heads) tasks, so that the weight
// gradient collects in registers: per lane over its tasks and then over the lanes that share a column in FP32 (the FP32
// chain: one term per head that the lane holds in each of its tasks, 384 for 8 x 4608 tokens of 24 heads x 128), over the block's warps
// and, in reduce_weight_grads, over the blocks in FP64, all in a fixed order.  No atomics: the result depends on nothing but
// the shape.
template <int kD, bool kHalf>
__global__ void __launch_bounds__(32 * kWarps, Shape<kD>::kBackResident)
backward_kernel(const Grads2 both, const Turn t, uint32_t rows, int blocks_q, int parts_log2, float eps, double *__restrict__ partials) {
    using S = Shape<kD>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool is_q = static_cast<int>(blockIdx.x) < blocks_q;
    const Grads d = is_q ? both.g[0] : both.g[1];
    const uint32_t block = is_q ? blockIdx.x : blockIdx.x - blocks_q, blocks = is_q ? blocks_q : gridDim.x - blocks_q;
    int c0, c1;
    columns<kHalf>(lane % S::kLanes, t.rot, c0, c1);
    const bool mine = c0 < t.rot;
    const bool norm = d.weight != nullptr;
    const int heads = d.heads, step = (S::kRep * S::kUnrollBack) << parts_log2;
    Slot w, acc{};    // 0.0f in both lanes
    if (norm) w = unpack<kHalf>(load_weight(d.weight, c0, c1));
    const uint64_t tasks = static_cast<uint64_t>(rows) << parts_log2;
    for (uint64_t task = static_cast<uint64_t>(block) * kWarps + warp; task < tasks; task += static_cast<uint64_t>(blocks) * kWarps) {
        const uint32_t m = static_cast<uint32_t>(task >> parts_log2);
        const uint16_t *dy = d.dy + m * d.ld_dy, *x = d.x + m * d.ld_x;
        uint16_t *dx = d.dx + m * d.ld_dx;
        int h = static_cast<int>(task & ((1u << parts_log2) - 1u)) * (S::kRep * S::kUnrollBack) + lane / S::kLanes;
        uint4 raw_dy[S::kUnrollBack], raw_x[S::kUnrollBack];
        auto fetch = [&]() {
#pragma unroll
            for (int u = 0; u < S::kUnrollBack; ++u) {
                // a head that does not exist: dy = 0 and x = 1, whose root mean square is not 0 (with eps = 0 as well)
                raw_dy[u] = make_uint4(0, 0, 0, 0);
                raw_x[u] = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
                if (h + u * S::kRep < heads) {
                    raw_dy[u] = load8<kHalf>(dy + (h + u * S::kRep) * kD, c0, c1);
                    if (norm) raw_x[u] = load8<kHalf>(x + (h + u * S::kRep) * kD, c0, c1);
                }
            }
        };
        fetch();
        Angles an;
        if (t.rot > 0) an = angles<kD>(t, m, lane);
        for (; h - lane / S::kLanes < heads; h += step) {
#pragma unroll
            for (int u = 0; u < S::kUnrollBack; ++u) {
                Slot dn = unpack<kHalf>(raw_dy[u]);
                if (mine) turn(dn, an.c, an.ns, an.s);   // the inverse turn
                if (norm) {   // uniform over the warp
                    const Slot x8 = unpack<kHalf>(raw_x[u]);
                    Slot prod;    // dn x
                    uint64_t ss = 0, dot = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        prod.v[e] = qmath::mul2(dn.v[e], x8.v[e]);
                        ss = qmath::fma2(x8.v[e], x8.v[e], ss);
                        dot = qmath::fma2(prod.v[e], w.v[e], dot);
                    }
                    const float r = rsqrtf(fmaf(head_sum<S::kLanes>(sum_lanes(ss)), 1.0f / kD, eps));
                    const float mean = head_sum<S::kLanes>(sum_lanes(dot)) * r * (1.0f / kD);       // mean of w dn xhat
                    const uint64_t r2 = twice(r), back = twice(-(r * r * mean));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {   // heads that do not exist have dn = 0 and a finite r: they add nothing
                        acc.v[e] = qmath::fma2(prod.v[e], r2, acc.v[e]);
                        dn.v[e] = qmath::fma2(qmath::mul2(dn.v[e], w.v[e]), r2, qmath::mul2(x8.v[e], back));
                    }
                }
                raw_dy[u] = pack<kHalf>(dn);
            }
#pragma unroll
            for (int u = 0; u < S::kUnrollBack; ++u)
                if (h + u * S::kRep < heads) store8<kHalf>(dx + (h + u * S::kRep) * kD, c0, c1, raw_dy[u]);
            if (h - lane / S::kLanes + step < heads) {
                h += step;
                fetch();
                h -= step;
            }
        }
    }
    if (partials == nullptr) return;
    // lanes that hold the same columns (FP32), then the warps: one FP64 value per column and block
    __shared__ float part[kWarps][kD];
    float sums[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) qmath::f32x2_split(acc.v[e], sums[2 * e], sums[2 * e + 1]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int o = S::kLanes; o < 32; o <<= 1) sums[e] += __shfl_xor_sync(0xFFFFFFFFu, sums[e], o);
        if (lane < S::kLanes) part[warp][column_of<kHalf>(e, c0, c1)] = sums[e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < kD; c += 32 * kWarps) {
        double v = 0.0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) v += part[i][c];
        partials[static_cast<int64_t>(blockIdx.x) * kD + c] = v;
    }
}

// dw[c] = sum of the blocks' partials, in block order within each of the strips that the threads take.
constexpr int kReduceStrips = 16;
template <int kD>
__global__ void __launch_bounds__(32 * kReduceStrips)
reduce_weight_grads(const double *__restrict__ partials, int blocks_q, int blocks, float *dw_q, float *dw_k) {
    __shared__ double part[kReduceStrips][32];
    float *dw = blockIdx.y == 0 ? dw_q : dw_k;
    ptx::grid_dependency_wait();
    if (dw == nullptr) return;
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), strip = threadIdx.x >> 5;
    double v = 0.0;
#pragma unroll 8
    for (int b = (blockIdx.y == 0 ? 0 : blocks_q) + strip; b < (blockIdx.y == 0 ? blocks_q : blocks); b += kReduceStrips)
        v += partials[static_cast<int64_t>(b) * kD + c];
    part[strip][threadIdx.x & 31] = v;
    __syncthreads();
    if (strip != 0) return;
#pragma unroll
    for (int i = 1; i < kReduceStrips; ++i) v += part[i][threadIdx.x & 31];
    dw[c] = static_cast<float>(v);
}

constexpr int kMaxBackwardBlocks = 1024;

// Warps that share a token, as a power of two: one where the tokens alone fill the GPU's warps, up to one per group of
// heads where they are few.
int split_of(int64_t rows, int heads, int heads_per_step, int64_t fill) {
    int log2 = 0;
    while ((rows << log2) < fill && (heads_per_step << log2) < heads) ++log2;
    return log2;
}

template <int kD>
sol_status_t forward(const Heads2 &h, const Turn &t, int64_t rows, bool half, float eps, cudaStream_t stream, const DeviceInfo *dev) {
    const int heads = h.h[0].heads > h.h[1].heads ? h.h[0].heads : h.h[1].heads;
    const int split = split_of(rows, heads, Shape<kD>::kHeads, 16LL * dev->sm_count);
    const dim3 grid(static_cast<unsigned>(ceil_div(rows << split, kWarps)), h.h[1].heads > 0 ? 2u : 1u);
    auto kern = half ? forward_kernel<kD, true> : forward_kernel<kD, false>;
    kern<<<grid, 32 * kWarps, 0, stream>>>(h, t, static_cast<uint32_t>(rows), split, eps);
    return launch_status();
}

template <int kD>
sol_status_t backward(const Grads2 &g, const Turn &t, int64_t rows, bool half, float eps, double *partials, cudaStream_t stream,
                      const DeviceInfo *dev) {
    constexpr int kHeads = Shape<kD>::kRep * Shape<kD>::kUnrollBack, kBackResident = Shape<kD>::kBackResident;
    const int heads = g.g[0].heads > g.g[1].heads ? g.g[0].heads : g.g[1].heads;
    const int split = split_of(rows, heads, kHeads, 16LL * dev->sm_count);
    // all blocks resident at once, shared out by the steps that q and k take per token
    const int64_t steps_q = ceil_div(g.g[0].heads, kHeads), steps_k = ceil_div(g.g[1].heads, kHeads);
    const int64_t most = kBackResident * dev->sm_count < kMaxBackwardBlocks ? kBackResident * dev->sm_count : kMaxBackwardBlocks;
    const int64_t want = ceil_div(rows << split, kWarps);       // a warp per task
    int64_t blocks_k = 0, blocks_q = most;
    if (steps_k > 0) {
        blocks_k = (most * steps_k + (steps_q + steps_k) / 2) / (steps_q + steps_k);
        if (blocks_k < 1) blocks_k = 1;
        if (blocks_k >= most) blocks_k = most - 1;
        blocks_q = most - blocks_k;
    }
    if (blocks_q > want) blocks_q = want;
    if (blocks_k > want) blocks_k = want;
    const int blocks = static_cast<int>(blocks_q + blocks_k);
    auto kern = half ? backward_kernel<kD, true> : backward_kernel<kD, false>;
    kern<<<blocks, 32 * kWarps, 0, stream>>>(g, t, static_cast<uint32_t>(rows), static_cast<int>(blocks_q), split, eps, partials);
    const sol_status_t st = launch_status();
    if (st != SOL_OK || partials == nullptr) return st;
    // the few blocks of the sum are set up while the last blocks of the gradients drain (programmatic launch)
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(kD / 32, steps_k > 0 ? 2 : 1);
    cfg.blockDim = dim3(32 * kReduceStrips);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, reduce_weight_grads<kD>, static_cast<const double *>(partials), static_cast<int>(blocks_q), blocks,
                           g.g[0].dweight, g.g[1].dweight) != cudaSuccess) {
        cudaGetLastError();
        return SOL_ERR_CUDA;
    }
    return launch_status();
}

}  // namespace

size_t backward_workspace_bytes(int64_t head_dim) { return sizeof(double) * static_cast<size_t>(head_dim) * kMaxBackwardBlocks; }

bool head_dim_ok(int64_t d) { return d == 32 || d == 64 || d == 128 || d == 256; }

sol_status_t launch_forward(const Heads2 &h, const Turn &t, int64_t rows, int64_t head_dim, bool half, float eps,
                            cudaStream_t stream, const DeviceInfo *dev) {
    switch (head_dim) {
        case 32: return forward<32>(h, t, rows, half, eps, stream, dev);
        case 64: return forward<64>(h, t, rows, half, eps, stream, dev);
        case 128: return forward<128>(h, t, rows, half, eps, stream, dev);
        case 256: return forward<256>(h, t, rows, half, eps, stream, dev);
    }
    return SOL_ERR_BAD_SHAPE;
}

sol_status_t launch_backward(const Grads2 &g, const Turn &t, int64_t rows, int64_t head_dim, bool half, float eps,
                             double *partials, cudaStream_t stream, const DeviceInfo *dev) {
    switch (head_dim) {
        case 32: return backward<32>(g, t, rows, half, eps, partials, stream, dev);
        case 64: return backward<64>(g, t, rows, half, eps, partials, stream, dev);
        case 128: return backward<128>(g, t, rows, half, eps, partials, stream, dev);
        case 256: return backward<256>(g, t, rows, half, eps, partials, stream, dev);
    }
    return SOL_ERR_BAD_SHAPE;
}

}  // namespace rotary
}  // namespace sol
