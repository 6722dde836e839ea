// Products of a few BF16 rows with a weight in NVFP4 or MXFP4 (sm_100a):
//     y[m][n] = bf16( T * sum_k act(x[m][k]) * code[n][k] * scale[n][block of k]  + bias[n] )
// The modulation and embedding linears of a DiT block have one row per sample, not per token: the weight is read
// once for a handful of rows, so the weight's bytes are the floor (0.5625 or 0.53 B per element) and the activations
// stay in 16 bits -- no quantizer, no scale pass over x.
//
// One CTA takes 128 output columns (a row group of the chunked scale layout) and a slice of K; a cluster of up to eight
// CTAs covers K and adds its partial sums through distributed shared memory in rank order.  A warp owns sixteen of
// the 128 weight rows (four neighbours of each 32-row quarter, so that its scale bytes are contiguous), and its
// lanes load their weights straight into the A fragments of mma.m16n8k16: the order of K inside a product is free as
// long as x follows it, so lane t of a quad takes 32 consecutive codes (16 bytes) of its two rows per 128 columns,
// i.e. whole scale blocks, and x is laid out in shared memory in the order in which the B fragments want it.
// Codes become FP16 by the hardware conversion, are multiplied by their block's scale, and enter the tensor core:
// dequantizing, not the products, is the work here (measured: 23 T codes/s for the conversion alone, 15 T codes/s with
// scale and mma, against 11.6 T codes/s that HBM delivers; unpacking into BF16 with integer operations: 9 T).
//
// Number formats.  code * block scale has at most six significant bits: exact in FP16 for NVFP4 (2^-10 .. 2688).  MXFP4
// scales are powers of two of any size: they are taken relative to the largest one of the row's slice, 2^13 for that
// one, so every block within 2^36 of it is exact; what lies below is off by at most 2^-25 of 2^-13 of it.  x (after the
// activation) is scaled by a power of two per row and slice so that its largest element is in [2^14, 2^15): BF16 values
// within 2^-29 of the largest stay exact, smaller ones are off by 2^-40 of the largest; an activation's FP32 result is
// rounded to FP16's 11 bits.  Sums are FP32.
#include <cuda_fp16.h>

#include "ptx.cuh"
#include "quant_math.cuh"
#include "sol_internal.h"

namespace sol {
namespace matvec {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kRows = 128;           // weight rows of a CTA
constexpr int kStepK = 128;          // K of a step: 32 codes per lane and row
constexpr int kRing = 4;             // steps whose weights are in registers or on their way
constexpr int kMaxCluster = 8;
constexpr int kPartPitch = kRows + 4;
constexpr int kXExp = 14;            // exponent of the largest scaled |x|
constexpr int kMxExp = 13;           // exponent of the largest relative MXFP4 scale

struct Params {
    const uint16_t *x;
    const uint8_t *wq;
    const uint8_t *wsf;
    const float *wts;        // null: MXFP4
    const uint16_t *bias;    // null: none
    uint16_t *y;
    int64_t ldx, ldy;
    int M, N, K;
    int steps, per_cta;      // 128-column steps of K, and those of one CTA
    int chunks_k;            // scale chunks per row group
    int silu;
};

__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t pair) {
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"(static_cast<uint16_t>(pair)));
    return d;
}
// 2^(kMxExp - below) as a half, in both lanes; 0 below the smallest subnormal.
__device__ __forceinline__ uint32_t mx_scale_half2(int below) {
    const int e = 15 + kMxExp - below;
    const uint32_t h = e > 0 ? static_cast<uint32_t>(e) << 10 : (e > -10 ? 1u << (9 + e) : 0u);
    return h | h << 16;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ld_cluster(uint32_t cluster_addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr) : "memory");
    return v;
}

__device__ __forceinline__ float silu(float v) { return __fdividef(v, 1.0f + __expf(-v)); }

__device__ __forceinline__ void activate8(uint4 r, int act, float (&f)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = qmath::bf16_lo(w[i]);
        f[2 * i + 1] = qmath::bf16_hi(w[i]);
    }
    if (act) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = silu(f[i]);
    }
}

// Shared memory: x of the slice (kTiles * 8 rows, pitch per_cta * 256 + 64 bytes), partial sums, row scales, x scales.
__host__ __device__ constexpr int x_pitch(int per_cta) { return per_cta * (2 * kStepK) + 64; }
constexpr int smem_bytes(int tiles, int per_cta) {
    return 8 * tiles * x_pitch(per_cta) + 8 * tiles * kPartPitch * 4 + kRows * 4 + 8 * tiles * 4;
}

template <bool kMx, int kTiles>
__global__ void __launch_bounds__(kThreads, 2)
matvec_kernel(const Params p) {
    constexpr int kM = 8 * kTiles;              // rows of x in this CTA
    constexpr int kAccs = kTiles == 1 ? 2 : 1;  // independent sums per tile: one chain of products would wait on itself
    extern __shared__ __align__(16) uint8_t smem[];
    const int pitch = x_pitch(p.per_cta);
    float *part = reinterpret_cast<float *>(smem + kM * pitch);
    int *row_ref = reinterpret_cast<int *>(part + kM * kPartPitch);
    float *x_back = reinterpret_cast<float *>(row_ref + kRows);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t rank = ptx::cluster_ctarank();
    const int group = blockIdx.y, m0 = blockIdx.z * kM;
    const int step0 = static_cast<int>(rank) * p.per_cta;
    const int steps = min(p.per_cta, p.steps - step0);
    const int ra = 4 * warp + (g & 3) + 32 * (g >> 2);          // this lane's rows of the group: ra and ra + 64
    const int64_t na = static_cast<int64_t>(group) * kRows + ra;
    const bool live_a = na < p.N, live_b = na + 64 < p.N;
    const uint8_t *qa = p.wq + na * (p.K / 2) + 16 * t, *qb = qa + static_cast<int64_t>(32) * p.K;   // 64 rows of K / 2 bytes
    const uint8_t *sf = p.wsf + static_cast<int64_t>(group) * p.chunks_k * 512 + (ra & 31) * 16 + (ra >> 5) * 4;

    uint4 wa[kRing], wb[kRing];
    uint32_t sa[kRing], sb[kRing];
    auto fetch = [&](int s, uint4 &a, uint4 &b, uint32_t &fa, uint32_t &fb) {
        const int k = (step0 + s) * kStepK + 32 * t;
        a = b = make_uint4(0, 0, 0, 0);
        fa = fb = 0;
        if (s < steps && k < p.K) {
            if (live_a) a = __ldcs(reinterpret_cast<const uint4 *>(qa + (step0 + s) * (kStepK / 2)));
            if (live_b) b = __ldcs(reinterpret_cast<const uint4 *>(qb + (step0 + s) * (kStepK / 2)));
            if (kMx) {
                const uint8_t *c = sf + static_cast<int64_t>(step0 + s) * 512 + t;
                fa = __ldg(c);
                fb = __ldg(c + 8);
            } else {
                const uint8_t *c = sf + static_cast<int64_t>(2 * (step0 + s) + (t >> 1)) * 512 + 2 * (t & 1);
                fa = __ldg(reinterpret_cast<const uint16_t *>(c));
                fb = __ldg(reinterpret_cast<const uint16_t *>(c + 8));
            }
        }
    };
#pragma unroll
    for (int i = 0; i < kRing; ++i) fetch(i, wa[i], wb[i], sa[i], sb[i]);

    // ---- x: a warp per row; largest magnitude of the slice, then scaled halves in fragment order
    const int chunks = steps * (kStepK / 8), live_chunks = min(chunks, (p.K - step0 * kStepK) / 8);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    uint4 xr[kTiles][2];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const int m = warp + 8 * i;
        const uint16_t *row = p.x + (m0 + m) * p.ldx + step0 * kStepK;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = lane + 32 * j;
            xr[i][j] = m0 + m < p.M && c < live_chunks ? __ldg(reinterpret_cast<const uint4 *>(row + 8 * c)) : zero;
        }
    }
    if (kMx && threadIdx.x < kRows) {   // largest scale exponent of each row's slice
        const uint8_t *c = p.wsf + (static_cast<int64_t>(group) * p.chunks_k + step0) * 512 + (threadIdx.x & 31) * 16 + (threadIdx.x >> 5) * 4;
        uint32_t most = 0;
        for (int s = 0; s < steps; ++s) most = __vmaxu4(most, __ldg(reinterpret_cast<const uint32_t *>(c + s * 512)));
        row_ref[threadIdx.x] = static_cast<int>(max(max(most & 255u, most >> 8 & 255u), max(most >> 16 & 255u, most >> 24)));
    }
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const int m = warp + 8 * i;
        const uint16_t *row = p.x + (m0 + m) * p.ldx + step0 * kStepK;
        const bool live = m0 + m < p.M;
        float f[2][8], most = 0.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            activate8(xr[i][j], p.silu, f[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(f[j][e]));
        }
        for (int c = lane + 64; c < live_chunks; c += 32) {   // slices beyond 512 columns
            float v[8];
            activate8(live ? __ldg(reinterpret_cast<const uint4 *>(row + 8 * c)) : zero, p.silu, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[e]));
        }
        const uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));
        // 2^(kXExp - e) with e the exponent of the largest element, held to what FP32 can scale by
        const int e = max(static_cast<int>(bits >> 23) - 127, -100);
        const float up = __uint_as_float(static_cast<uint32_t>(127 + kXExp - min(e, 127)) << 23);
        if (lane == 0) x_back[m] = bits ? __uint_as_float(static_cast<uint32_t>(127 - kXExp + min(e, 127)) << 23) : 0.0f;
        auto put = [&](int c, const float (&v)[8]) {
            // eight columns of lane t' = (c % 16) / 4, word c % 4 of its sixteen bytes
            __half2 h[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) h[q] = __floats2half2_rn(v[2 * q] * up, v[2 * q + 1] * up);
            uint8_t *to = smem + m * pitch + (c >> 4) * (2 * kStepK) + ((c & 3) * 4 + ((c & 15) >> 2)) * 16;
            *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(h);
        };
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (lane + 32 * j < chunks) put(lane + 32 * j, f[j]);
        for (int c = lane + 64; c < chunks; c += 32) {
            float v[8];
            activate8(live && c < live_chunks ? __ldg(reinterpret_cast<const uint4 *>(row + 8 * c)) : zero, p.silu, v);
            put(c, v);
        }
    }
    __syncthreads();

    // ---- products
    float acc[kTiles][kAccs][4] = {};
    const int ref_a = kMx ? row_ref[ra] : 0, ref_b = kMx ? row_ref[ra + 64] : 0;
    const uint32_t xs = ptx::smem_u32(smem) + g * pitch + t * 16;
    auto multiply = [&](int s, const uint4 &a, const uint4 &b, uint32_t fa, uint32_t fb) {
        const uint32_t wa4[4] = {a.x, a.y, a.z, a.w}, wb4[4] = {b.x, b.y, b.z, b.w};
        uint32_t sca[2], scb[2];    // scale pairs of the lane's first and second sixteen codes
        if (kMx) {
            sca[0] = sca[1] = mx_scale_half2(ref_a - static_cast<int>(fa));
            scb[0] = scb[1] = mx_scale_half2(ref_b - static_cast<int>(fb));
        } else {
            const uint32_t ha = e4m3x2_to_half2(fa), hb = e4m3x2_to_half2(fb);
            sca[0] = __byte_perm(ha, ha, 0x1010);
            sca[1] = __byte_perm(ha, ha, 0x3232);
            scb[0] = __byte_perm(hb, hb, 0x1010);
            scb[1] = __byte_perm(hb, hb, 0x3232);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t ha[4], hb[4];
            codes_to_half(wa4[w], ha);
            codes_to_half(wb4[w], hb);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ha[i] = mul_half2(ha[i], sca[w >> 1]);
                hb[i] = mul_half2(hb[i], scb[w >> 1]);
            }
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
                const uint4 xb = ptx::lds128(xs + n * 8 * pitch + s * (2 * kStepK) + w * 64);
                mma_f16(acc[n][0], ha[0], hb[0], ha[1], hb[1], xb.x, xb.y);
                mma_f16(acc[n][kAccs - 1], ha[2], hb[2], ha[3], hb[3], xb.z, xb.w);
            }
        }
    };
    for (int s = 0; s < steps; s += kRing) {
#pragma unroll
        for (int i = 0; i < kRing; ++i) {
            if (s + i < steps) {
                multiply(s + i, wa[i], wb[i], sa[i], sb[i]);
                fetch(s + i + kRing, wa[i], wb[i], sa[i], sb[i]);
            }
        }
    }

    // ---- sums of the slices: every CTA leaves its own, then adds a share of the outputs over the cluster in rank order
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int m = 8 * n + 2 * t + (e & 1), r = ra + (e >> 1) * 64;
            float v = acc[n][0][e];
            if (kAccs == 2) v += acc[n][kAccs - 1][e];
            v *= x_back[m];
            if (kMx) v = scalbnf(v, ((e >> 1) ? ref_b : ref_a) - 127 - kMxExp);
            part[m * kPartPitch + r] = v;
        }
    }
    ptx::cluster_sync();
    const uint32_t ranks = static_cast<uint32_t>(gridDim.x);
    const float T = kMx ? 1.0f : __ldg(p.wts);
    const uint32_t mine = ptx::smem_u32(part);
    for (uint32_t i = rank * kThreads + threadIdx.x; i < kM * (kRows / 2); i += ranks * kThreads) {
        const int m = static_cast<int>(i) / (kRows / 2), r = 2 * (static_cast<int>(i) % (kRows / 2));
        const int n = group * kRows + r;
        if (m0 + m >= p.M || n >= p.N) continue;
        float v0 = 0.0f, v1 = 0.0f;
        for (uint32_t c = 0; c < ranks; ++c) {
            const uint32_t at = ptx::map_to_cta(mine + (m * kPartPitch + r) * 4, c);
            v0 += ld_cluster(at);
            v1 += ld_cluster(at + 4);
        }
        uint32_t b2 = 0;
        if (p.bias != nullptr) b2 = __ldg(reinterpret_cast<const uint32_t *>(p.bias + n));
        const float y0 = fmaf(v0, T, qmath::bf16_lo(b2)), y1 = fmaf(v1, T, qmath::bf16_hi(b2));
        uint32_t o;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(y1), "f"(y0));
        *reinterpret_cast<uint32_t *>(p.y + (m0 + m) * p.ldy + n) = o;
    }
    ptx::cluster_sync();   // no CTA leaves while another may still read its sums
}

template <bool kMx, int kTiles>
sol_status_t launch(const Params &p, int ranks, cudaStream_t stream) {
    auto kern = matvec_kernel<kMx, kTiles>;
    const int smem = smem_bytes(kTiles, p.per_cta);
    static bool configured[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SOL_ERR_CUDA;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess) return SOL_ERR_CUDA;
        configured[dev] = true;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(ranks), static_cast<unsigned>(ceil_div(p.N, kRows)), static_cast<unsigned>(ceil_div(p.M, 8 * kTiles)));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = static_cast<size_t>(smem);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {static_cast<unsigned>(ranks), 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kern, p) != cudaSuccess) {
        cudaGetLastError();
        return SOL_ERR_CUDA;
    }
    return launch_status();
}

template <bool kMx>
sol_status_t launch_rows(const Params &p, int ranks, cudaStream_t stream) {
    if (p.M <= 8) return launch<kMx, 1>(p, ranks, stream);
    if (p.M <= 16) return launch<kMx, 2>(p, ranks, stream);
    if (p.M <= 24) return launch<kMx, 3>(p, ranks, stream);
    return launch<kMx, 4>(p, ranks, stream);
}

}  // namespace

int max_k() { return 24576; }

sol_status_t launch_matvec(const void *x, int64_t ldx, const void *wq, const void *wsf, const float *wts, const void *bias, void *y,
                           int64_t ldy, int64_t M, int64_t N, int64_t K, bool silu, cudaStream_t stream, const DeviceInfo *dev) {
    Params p{};
    p.x = static_cast<const uint16_t *>(x);
    p.wq = static_cast<const uint8_t *>(wq);
    p.wsf = static_cast<const uint8_t *>(wsf);
    p.wts = wts;
    p.bias = static_cast<const uint16_t *>(bias);
    p.y = static_cast<uint16_t *>(y);
    p.ldx = ldx;
    p.ldy = ldy;
    p.M = static_cast<int>(M);
    p.N = static_cast<int>(N);
    p.K = static_cast<int>(K);
    p.steps = static_cast<int>(ceil_div(K, kStepK));
    p.chunks_k = static_cast<int>(ceil_div(K, wts != nullptr ? 64 : 128));
    p.silu = silu ? 1 : 0;
    // Slices of four steps (what a CTA's registers hold at once), shorter where that leaves SMs without a CTA, longer
    // where the cluster is full.
    const int64_t groups = ceil_div(N, kRows);
    int per = kRing;
    while (per > 1 && groups * ceil_div(p.steps, per) < dev->sm_count && ceil_div(p.steps, per - 1) <= kMaxCluster) --per;
    if (ceil_div(p.steps, per) > kMaxCluster) per = static_cast<int>(ceil_div(p.steps, kMaxCluster));
    p.per_cta = per;
    const int ranks = static_cast<int>(ceil_div(p.steps, per));
    return wts != nullptr ? launch_rows<false>(p, ranks, stream) : launch_rows<true>(p, ranks, stream);
}

}  // namespace matvec
}  // namespace sol
