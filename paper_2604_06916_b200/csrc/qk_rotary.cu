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
// HBM bound: 4 bytes per element forward, 6 backward.  A warp owns one token and a few heads of it; a lane
// owns the same eight columns of each of those heads (in the half layout four and their four partners), so
// angles are formed once per warp, each by one lane, and handed round by shuffles; all loads of a warp are
// issued before the angle arithmetic, which runs in their shadow.
//
// Angles: position * freq and the reduction to half a turn are in FP64 (a far position times a frequency has
// more significant bits than FP32 holds), the sine and cosine of the remainder in FP32.  Squares, means and
// products are FP32; the only rounding to 16 bits is the output's.
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
    static constexpr int kHeads = kRep * kUnroll;             // heads of a warp's task
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
__device__ __forceinline__ void unpack8(uint4 v, float (&f)[8]) {
    f[0] = bf16_lo(v.x), f[1] = bf16_hi(v.x), f[2] = bf16_lo(v.y), f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z), f[5] = bf16_hi(v.z), f[6] = bf16_lo(v.w), f[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
// Members of the slot's pair i (0..3) among its eight values.
template <bool kHalf>
__device__ __forceinline__ constexpr int first_of(int i) { return kHalf ? i : 2 * i; }
template <bool kHalf>
__device__ __forceinline__ constexpr int second_of(int i) { return kHalf ? i + 4 : 2 * i + 1; }

// The slot's columns of a norm weight (read by every warp: cached).
template <bool kHalf>
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
__device__ __forceinline__ void angles(const Turn &t, int64_t m, int lane, float (&cs)[4], float (&sn)[4]) {
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
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int src = slot + S::kLanes * (i / S::kPairs);
        cs[i] = __shfl_sync(0xFFFFFFFFu, mc[i % S::kPairs], src);
        sn[i] = __shfl_sync(0xFFFFFFFFu, ms[i % S::kPairs], src);
    }
}

template <int kD, bool kHalf>
__global__ void __launch_bounds__(32 * kWarps)
forward_kernel(const Heads q, const Heads k, const Turn t, uint32_t rows, int groups, float eps) {
    using S = Shape<kD>;
    const int lane = threadIdx.x & 31;
    const uint64_t task = static_cast<uint64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const uint32_t m = static_cast<uint32_t>(task / static_cast<uint32_t>(groups));
    if (m >= rows) return;
    const int first = static_cast<int>(task % static_cast<uint32_t>(groups)) * S::kHeads + lane / S::kLanes;
    int c0, c1;
    columns<kHalf>(lane % S::kLanes, t.rot, c0, c1);
    uint4 raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int h = first + u * S::kRep;
        raw[u] = make_uint4(0, 0, 0, 0);
        if (h < q.heads) raw[u] = load8<kHalf>(q.x + m * q.ld_in + h * kD, c0, c1);
        else if (h < q.heads + k.heads) raw[u] = load8<kHalf>(k.x + m * k.ld_in + (h - q.heads) * kD, c0, c1);
    }
    float cs[4], sn[4];
    const bool turned = t.rot > 0;
    if (turned) angles<kD>(t, m, lane, cs, sn);
    const bool mine = c0 < t.rot;    // this lane's columns are rotated ones (a slot is wholly inside or outside)
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int h = first + u * S::kRep;
        const bool is_q = h < q.heads, live = h < q.heads + k.heads;
        const uint16_t *w = is_q ? q.weight : k.weight;
        float f[8];
        unpack8(raw[u], f);
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
        ss = head_sum<S::kLanes>(ss);
        if (w != nullptr) {
            const float r = 1.0f / sqrtf(fmaf(ss, 1.0f / kD, eps));
            float g[8];
            unpack8(load_weight<kHalf>(w, c0, c1), g);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= r * g[e];
        }
        if (mine) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = f[first_of<kHalf>(i)], b = f[second_of<kHalf>(i)];
                f[first_of<kHalf>(i)] = fmaf(a, cs[i], -(b * sn[i]));
                f[second_of<kHalf>(i)] = fmaf(b, cs[i], a * sn[i]);
            }
        }
        if (live) {
            uint16_t *out = is_q ? q.out + m * q.ld_out + h * kD : k.out + m * k.ld_out + (h - q.heads) * kD;
            store8<kHalf>(out, c0, c1, pack8(f));
        }
    }
}

// Gradients.  Blocks stay and walk the (token, head group) tasks; a task is all of q or all of k, so that the two
// weight gradients collect in registers: per lane over its tasks, per block over the lanes and warps that share a
// column (FP64, fixed order), and reduce_weight_grads adds the blocks up.  No atomics: the result depends on
// nothing but the shape.
template <int kD, bool kHalf>
__global__ void __launch_bounds__(32 * kWarps)
backward_kernel(const Grads q, const Grads k, const Turn t, uint32_t rows, int groups_q, int groups_k, float eps,
                double *__restrict__ partials) {
    using S = Shape<kD>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int c0, c1;
    columns<kHalf>(lane % S::kLanes, t.rot, c0, c1);
    const bool mine = c0 < t.rot;
    const uint32_t groups = static_cast<uint32_t>(groups_q + groups_k);
    const uint64_t tasks = static_cast<uint64_t>(rows) * groups;
    float acc[2][8] = {};
    for (uint64_t task = static_cast<uint64_t>(blockIdx.x) * kWarps + warp; task < tasks;
         task += static_cast<uint64_t>(gridDim.x) * kWarps) {
        const uint32_t m = static_cast<uint32_t>(task / groups);
        const int g = static_cast<int>(task - static_cast<uint64_t>(m) * groups);
        const bool is_q = g < groups_q;
        const Grads &d = is_q ? q : k;
        const int first = (is_q ? g : g - groups_q) * S::kHeads + lane / S::kLanes;
        const bool norm = d.weight != nullptr;
        uint4 raw_dy[kUnroll], raw_x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = first + u * S::kRep;
            raw_dy[u] = raw_x[u] = make_uint4(0, 0, 0, 0);
            if (h < d.heads) {
                raw_dy[u] = load8<kHalf>(d.dy + m * d.ld_dy + h * kD, c0, c1);
                if (norm) raw_x[u] = load8<kHalf>(d.x + m * d.ld_x + h * kD, c0, c1);
            }
        }
        float cs[4], sn[4], w[8];
        if (t.rot > 0) angles<kD>(t, m, lane, cs, sn);
        if (norm) unpack8(load_weight<kHalf>(d.weight, c0, c1), w);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = first + u * S::kRep;
            float dn[8];
            unpack8(raw_dy[u], dn);
            if (mine) {   // the inverse turn
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = dn[first_of<kHalf>(i)], b = dn[second_of<kHalf>(i)];
                    dn[first_of<kHalf>(i)] = fmaf(a, cs[i], b * sn[i]);
                    dn[second_of<kHalf>(i)] = fmaf(b, cs[i], -(a * sn[i]));
                }
            }
            if (norm) {   // uniform over the warp
                float x[8];
                unpack8(raw_x[u], x);
                float ss = 0.0f, dot = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ss = fmaf(x[e], x[e], ss);
                    dot = fmaf(dn[e] * w[e], x[e], dot);
                }
                ss = head_sum<S::kLanes>(ss);
                dot = head_sum<S::kLanes>(dot);
                const float r = 1.0f / sqrtf(fmaf(ss, 1.0f / kD, eps));
                const float mean = dot * r * (1.0f / kD);       // mean of w dn xhat
                const bool live = h < d.heads;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float xhat = x[e] * r;
                    const float c = live ? dn[e] * xhat : 0.0f;
                    if (is_q) acc[0][e] += c;
                    else acc[1][e] += c;
                    dn[e] = r * fmaf(dn[e], w[e], -(xhat * mean));
                }
            }
            if (h < d.heads) store8<kHalf>(d.dx + m * d.ld_dx + h * kD, c0, c1, pack8(dn));
        }
    }
    if (partials == nullptr) return;
    // lanes that hold the same columns, then the warps, then one FP64 value per column and block
    __shared__ float part[kWarps][2][kD];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = acc[s][e];
#pragma unroll
            for (int o = S::kLanes; o < 32; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
            if (lane < S::kLanes) part[warp][s][e < 4 ? c0 + e : c1 + e - 4] = v;
        }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * kD; c += 32 * kWarps) {
        double v = 0.0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) v += part[i][c / kD][c % kD];
        partials[static_cast<int64_t>(blockIdx.x) * (2 * kD) + c] = v;
    }
}

// dw[c] = sum of the blocks' partials, in block order within each of the strips that the threads take.
constexpr int kReduceStrips = 8;
template <int kD>
__global__ void __launch_bounds__(32 * kReduceStrips)
reduce_weight_grads(const double *__restrict__ partials, int blocks, float *dw_q, float *dw_k) {
    __shared__ double part[kReduceStrips][32];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), strip = threadIdx.x >> 5;
    double v = 0.0;
#pragma unroll 8
    for (int b = strip; b < blocks; b += kReduceStrips) v += partials[static_cast<int64_t>(b) * (2 * kD) + c];
    part[strip][threadIdx.x & 31] = v;
    __syncthreads();
    if (strip != 0) return;
#pragma unroll
    for (int i = 1; i < kReduceStrips; ++i) v += part[i][threadIdx.x & 31];
    float *dw = c < kD ? dw_q : dw_k;
    if (dw != nullptr) dw[c % kD] = static_cast<float>(v);
}

constexpr int kMaxBackwardBlocks = 1024;

template <int kD>
sol_status_t forward(const Heads &q, const Heads &k, const Turn &t, int64_t rows, bool half, float eps, cudaStream_t stream) {
    const int groups = static_cast<int>(ceil_div(q.heads + k.heads, Shape<kD>::kHeads));
    const int64_t blocks = ceil_div(rows * groups, kWarps);
    if (blocks > 0x7FFFFFFFLL) return SOL_ERR_BAD_SHAPE;
    auto kern = half ? forward_kernel<kD, true> : forward_kernel<kD, false>;
    kern<<<static_cast<unsigned>(blocks), 32 * kWarps, 0, stream>>>(q, k, t, static_cast<uint32_t>(rows), groups, eps);
    return launch_status();
}

template <int kD>
sol_status_t backward(const Grads &q, const Grads &k, const Turn &t, int64_t rows, bool half, float eps, double *partials,
                      cudaStream_t stream, const DeviceInfo *dev) {
    const int gq = static_cast<int>(ceil_div(q.heads, Shape<kD>::kHeads)), gk = static_cast<int>(ceil_div(k.heads, Shape<kD>::kHeads));
    const int64_t want = ceil_div(rows * (gq + gk), kWarps);
    const int64_t most = 4 * dev->sm_count < kMaxBackwardBlocks ? 4 * dev->sm_count : kMaxBackwardBlocks;
    const int blocks = static_cast<int>(want < most ? want : most);
    auto kern = half ? backward_kernel<kD, true> : backward_kernel<kD, false>;
    kern<<<blocks, 32 * kWarps, 0, stream>>>(q, k, t, static_cast<uint32_t>(rows), gq, gk, eps, partials);
    const sol_status_t st = launch_status();
    if (st != SOL_OK || partials == nullptr) return st;
    reduce_weight_grads<kD><<<2 * kD / 32, 32 * kReduceStrips, 0, stream>>>(partials, blocks, q.dweight, k.dweight);
    return launch_status();
}

}  // namespace

size_t backward_workspace_bytes(int64_t head_dim) { return sizeof(double) * 2 * static_cast<size_t>(head_dim) * kMaxBackwardBlocks; }

bool head_dim_ok(int64_t d) { return d == 32 || d == 64 || d == 128 || d == 256; }

sol_status_t launch_forward(const Heads &q, const Heads &k, const Turn &t, int64_t rows, int64_t head_dim, bool half, float eps,
                            cudaStream_t stream) {
    switch (head_dim) {
        case 32: return forward<32>(q, k, t, rows, half, eps, stream);
        case 64: return forward<64>(q, k, t, rows, half, eps, stream);
        case 128: return forward<128>(q, k, t, rows, half, eps, stream);
        case 256: return forward<256>(q, k, t, rows, half, eps, stream);
    }
    return SOL_ERR_BAD_SHAPE;
}

sol_status_t launch_backward(const Grads &q, const Grads &k, const Turn &t, int64_t rows, int64_t head_dim, bool half, float eps,
                             double *partials, cudaStream_t stream, const DeviceInfo *dev) {
    switch (head_dim) {
        case 32: return backward<32>(q, k, t, rows, half, eps, partials, stream, dev);
        case 64: return backward<64>(q, k, t, rows, half, eps, partials, stream, dev);
        case 128: return backward<128>(q, k, t, rows, half, eps, partials, stream, dev);
        case 256: return backward<256>(q, k, t, rows, half, eps, partials, stream, dev);
    }
    return SOL_ERR_BAD_SHAPE;
}

}  // namespace rotary
}  // namespace sol
