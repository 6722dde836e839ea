// Products of a few BF16 rows with a weight in NVFP4 or MXFP4 (sm_100a):
//     y[m][n] = bf16( T * sum_k act(x[m][k]) * code[n][k] * scale[n][block of k]  + bias[n] )
// The modulation and embedding linears of a DiT block have one row per sample, not per token: the weight is read
// once for a handful of rows, so the weight's bytes are the floor (0.5625 or 0.53 B per element) and the activations
// stay in 16 bits -- no quantizer, no scale pass over x.
//
// Two launches.  prepare_x turns x (after the activation) into FP16 once, in the shared-memory image of the products'
// operand; the products' kernel is launched along with it (programmatic launch) and waits for it only where x enters.
// Up to four rows of K <= 3072 are prepared by every CTA for its own slice instead (two of its warpgroups, while the other
// two convert the first stage): one launch and no workspace, 2.1 to 2.7 us less for a caller without graphs.  Inside a graph
// it is the slower form, by more the more x a CTA prepares (one / two launches, us, 9216 columns; in brackets with weights from HBM):
//     K = 1536: 1 row 7.4 / 7.4 (8.2 / 8.3), 4 rows 7.9 / 7.5 (8.9 / 8.3);   K = 3072: 9.6 / 9.1 (11.4 / 10.3), 10.3 / 9.2 (11.8 / 10.3)
//     K = 4608: 11.5 / 11.0 (13.4 / 12.1), 12.4 / 11.0 (14.4 / 12.1);   2304 columns, K = 8192: 10.4 / 9.6, 11.3 / 9.7
// The bound on K is that of a CTA's slice (the registers that hold x), for a grid without a cluster, whose slice is all of K;
// beyond it the graph would lose up to 2.2 us where the call gains 2.4.  With eight rows the exponentials alone would take a CTA longer
// than its weights.
// One CTA takes 128 output columns (a row group of the chunked scale layout) and a slice of K, one CTA per SM; where the
// columns leave SMs free, a cluster of up to eight CTAs shares K, each adds up its share of the 128 columns in rank order.
// The weight is the M = 128 operand of tcgen05.mma kind::f16 and comes from tensor memory: codes, scales and x
// stream into a ring of 256-column stages by TMA and bulk copies, a thread per weight row converts the codes to FP16
// (cvt.e2m1x2), multiplies by the block scales and leaves them in its TMEM lane; x is the N operand (16 to 64 rows).
// Four warpgroups convert: two share an even stage, two an odd one, while the products of the stage before run.
//
// Measured (B200, inside a graph, one weight again and again, which L2 then holds): NVFP4 1 x 9216 x 3072 9.4 us, 8 x 18432 x
// 3072 11.4 us, MXFP4 24 x 14592 x 2432 12.1 us; 400 MB of weights in turn, so that each comes from HBM: 10.9, 13.1 and 14.5 us
// (floors 2.4, 4.9 and 3.0 us).  A stage takes 800 cycles per SM while stages run; leaving out three quarters of the products
// or of the conversions changes nothing at up to sixteen rows, nor does L2 in place of HBM make up more than 2.4 us of the
// whole.  The rest is the way in (2 to 2.5 us until the first codes arrive, prepare_x beside it) and out (1.5 us from the last
// product to the stores).  Four stages: with eight
// in flight the first one arrives with the last (13.5 us), with two the ring runs dry (16.8 us).  Register tiles and
// mma.sync m16n8k16 in place of tensor memory: 11.5, 23.7 and 28 us; converting for mma.sync costs 2 codes per cycle and
// scheduler and every eight rows of x as much again, tcgen05 takes 64 rows for the price of one.
//
// Number formats.  code * block scale has at most six significant bits: exact in FP16 for NVFP4 (2^-10 .. 2688).  MXFP4
// scales are powers of two of any size: they are taken relative to the largest one of the row's slice, 2^13 for that
// one, so every block within 2^36 of it is exact; what lies below is off by at most 2^-25 of 2^-13 of it.  x (after the
// activation) is scaled by a power of two per row and slice so that its largest element is in [2^14, 2^15): BF16 values
// within 2^-29 of the largest stay exact, smaller ones are off by 2^-40 of the largest (a largest one below 2^-100 is
// scaled by 2^114 all the same); an activation's FP32 result is rounded to FP16's 11 bits.  Sums are FP32; the powers of two
// of x, of the MXFP4 scales and of T are undone together, which stays in FP32's range wherever the slice's sum does.
#include <cuda_fp16.h>

#include "gemm_common.cuh"
#include "quant_math.cuh"
#include "sol_internal.h"

namespace sol {
namespace matvec {
namespace {

using gemm::loads_held;
using gemm::wait_bounded;

constexpr int kConvWarps = 16;       // four warpgroups
constexpr int kProducer = kConvWarps, kIssuer = kConvWarps + 1;
constexpr int kThreads = 32 * (kConvWarps + 2);
constexpr int kRows = 128;           // weight rows of a CTA
constexpr int kStageK = 256;         // K of a stage: 128 bytes of codes per row
constexpr int kMaxStages = 4;
constexpr int kCodeBytes = kRows * kStageK / 2;
constexpr int kSfBytes = kRows * kStageK / 16;
constexpr int kMaxCluster = 8;
constexpr int kXExp = 14;            // exponent of the largest scaled |x|
constexpr int kMxExp = 13;           // exponent of the largest relative MXFP4 scale
constexpr int kMaxXRows = 64;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColA = 0, kColABuf = 128, kColD = 256;   // A: two buffers of a stage; D: kSums of 64 columns
constexpr int kSums = 4;             // sums that products take in turn: one alone would wait for itself
constexpr int kFull = 0, kXFull = kFull + kMaxStages, kEmpty = kXFull + kMaxStages, kAFull = kEmpty + kMaxStages, kAEmpty = kAFull + 2,
              kDone = kAEmpty + 2, kBars = kDone + 1;
constexpr int kMaxSmem = 232448 - 1024;   // dynamic, beside the static arrays

struct Params {
    const uint16_t *x;       // few rows: prepared by every CTA for its slice (kInline)
    int64_t ldx;
    int K, act;
    const uint8_t *ximage;   // FP16 x: [row chunk][64 columns of K][x_rows][128 bytes, 128-byte swizzle], K padded to stages
    const int *x_exp;        // per row: the exponent that undoes its scaling
    const uint8_t *wsf;
    const float *wts;        // null: MXFP4
    const uint16_t *bias;    // null: none
    uint16_t *y;
    uint32_t *status;
    int64_t ldy;
    int M, N;
    int x_rows;              // rows of x in a CTA: 16, 32, 48 or 64
    int stages, per_cta;     // 256-column stages of K, and those of one CTA
    int ring;                // stages in shared memory
    int chunks_k;            // scale chunks per row group
};

__host__ __device__ constexpr int stage_x_bytes(int x_rows) { return x_rows * (2 * kStageK); }
// Shared memory: the code ring, the x ring, the scale ring, the cluster's partial sums [rank][x row][own columns], barriers.
// `x_stages`: stages of x held at once, the ring's or (kInline) the slice's.
__host__ __device__ constexpr int smem_bytes(int x_rows, int ring, int x_stages) {
    return ring * (kCodeBytes + kSfBytes) + x_stages * stage_x_bytes(x_rows) + x_rows * kRows * 4 + 8 * kBars + 16;
}
constexpr int kXWarps = kConvWarps / 2;   // warps that prepare x there
constexpr int kInlineRows = 4;       // rows of x up to which every CTA prepares its slice itself, in one launch
constexpr int kInlineStages = 12;    // ... of K up to so many stages
constexpr bool prepared_inline(int64_t M, int64_t K) { return M <= kInlineRows && K <= kInlineStages * kStageK; }

__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t s, uint32_t *h) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t.reg .b32 t0, t1, t2, t3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 t0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 t1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 t2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 t3, b3;\n\t"
        "mul.rn.f16x2 %0, t0, %5;\n\t"
        "mul.rn.f16x2 %1, t1, %5;\n\t"
        "mul.rn.f16x2 %2, t2, %5;\n\t"
        "mul.rn.f16x2 %3, t3, %5;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w), "r"(s));
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
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t cluster_addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t cluster_addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory");
}
// A bounded wait of a whole warp: if it runs out for one lane, every lane gives up, so the warp stays together.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t *abort_flag, uint32_t *status, uint32_t code) {
    return __all_sync(0xFFFFFFFFu, wait_bounded(bar, parity, abort_flag, status, code));
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

// e - kXExp with e the exponent of the largest element (FP32 bits), held to what FP32 can scale by; and 2^(kXExp - e).
__device__ __forceinline__ int exponent_back(uint32_t bits) { return min(max(static_cast<int>(bits >> 23) - 127, -100), 127) - kXExp; }
__device__ __forceinline__ float scale_up(uint32_t bits) { return __uint_as_float(static_cast<uint32_t>(127 - exponent_back(bits)) << 23); }
// T = t 2^exp with t in [1, 2); a subnormal T: t = T 2^100; zero, infinities and NaN keep their value.
__device__ __forceinline__ float split_scale(float T, int &exp) {
    const uint32_t bits = __float_as_uint(T), field = bits >> 23 & 255u;
    exp = field == 0 ? -100 : field == 255u ? 0 : static_cast<int>(field) - 127;
    return field == 0 ? T * 0x1p100f : field == 255u ? T : __uint_as_float((bits & 0x807FFFFFu) | 0x3F800000u);
}
// v 2^n in two exact steps, for |v| < 2^55 and n from -254 to 240: where the first step overflows or loses bits, the result is
// infinite or zero anyway.
struct PowerOfTwo {
    float a, b;
    __device__ __forceinline__ explicit PowerOfTwo(int n) {
        n = max(n, -252);
        a = __uint_as_float(static_cast<uint32_t>(127 + (n >> 1)) << 23);
        b = __uint_as_float(static_cast<uint32_t>(127 + n - (n >> 1)) << 23);
    }
    __device__ __forceinline__ float times(float v) const { return v * a * b; }
};
__device__ __forceinline__ float largest8(const float (&v)[8], float most) {
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[e]));
    return most;
}
__device__ __forceinline__ uint4 to_half8(const float (&v)[8], float up) {
    uint32_t h[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const __half2 pair = __floats2half2_rn(v[2 * q] * up, v[2 * q + 1] * up);
        h[q] = *reinterpret_cast<const uint32_t *>(&pair);
    }
    return make_uint4(h[0], h[1], h[2], h[3]);
}
// Place of eight columns (chunk c of the slice) of row r in the image: a box of [x_rows][128 bytes] per 64 columns.
__device__ __forceinline__ int64_t image_offset(int c, int r, int x_rows) {
    return static_cast<int64_t>(c >> 3) * (x_rows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
}

// x -> scaled FP16 in the products' layout.  A block per row (rows behind the last are zeros), a thread per eight columns.
constexpr int kPrepThreads = 512;
__global__ void __launch_bounds__(kPrepThreads)
prepare_x(const uint16_t *__restrict__ x, int64_t ldx, int M, int K, int x_rows, int stages, int act, uint8_t *__restrict__ image,
          int *__restrict__ x_exp) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the products' CTAs may start loading weights
    __shared__ uint32_t warp_max[kPrepThreads / 32];
    const int m = blockIdx.x, chunks = stages * (kStageK / 8), live = K / 8;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const uint16_t *row = x + m * ldx;
    constexpr int kHeld = 2;                  // chunks per thread kept from the first pass (rows up to 8192 columns)
    float f[kHeld][8], most = 0.0f;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
        const int c = threadIdx.x + j * kPrepThreads;
        activate8(m < M && c < live ? __ldg(reinterpret_cast<const uint4 *>(row + 8 * c)) : zero, act, f[j]);
        most = largest8(f[j], most);
    }
    for (int c = threadIdx.x + kHeld * kPrepThreads; c < live; c += kPrepThreads) {
        float v[8];
        activate8(m < M ? __ldg(reinterpret_cast<const uint4 *>(row + 8 * c)) : zero, act, v);
        most = largest8(v, most);
    }
    uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));
    if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = bits;
    __syncthreads();
    bits = __reduce_max_sync(0xFFFFFFFFu, warp_max[threadIdx.x & (kPrepThreads / 32 - 1)]);
    const float up = scale_up(bits);
    if (threadIdx.x == 0) x_exp[m] = exponent_back(bits);
    uint8_t *to = image + static_cast<int64_t>(m / x_rows) * (4 * stages) * (x_rows * 128);
    auto put = [&](int c, const float (&v)[8]) { *reinterpret_cast<uint4 *>(to + image_offset(c, m % x_rows, x_rows)) = to_half8(v, up); };
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
        if (threadIdx.x + j * kPrepThreads < chunks) put(threadIdx.x + j * kPrepThreads, f[j]);
    for (int c = threadIdx.x + kHeld * kPrepThreads; c < chunks; c += kPrepThreads) {
        float v[8];
        activate8(m < M && c < live ? __ldg(reinterpret_cast<const uint4 *>(row + 8 * c)) : zero, act, v);
        put(c, v);
    }
}

template <bool kMx, bool kInline>
__global__ void __launch_bounds__(kThreads, 1)
matvec_kernel(const __grid_constant__ CUtensorMap tm_w, const Params p) {
    constexpr int kChunksPerStage = kMx ? 2 : 4;      // 512-byte scale chunks of a stage
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ uint8_t row_most[kMx ? 4 : 1][kRows];
    __shared__ uint32_t warp_most[kXWarps];
    const uint32_t base = ptx::smem_u32(smem_raw);
    const uint32_t x_bytes = static_cast<uint32_t>(stage_x_bytes(p.x_rows));
    const uint32_t s_code = base, s_x = s_code + p.ring * kCodeBytes, s_sf = s_x + (kInline ? p.per_cta : p.ring) * x_bytes;
    const uint32_t s_part = s_sf + p.ring * kSfBytes, bar_base = s_part + p.x_rows * kRows * 4;
    uint8_t *bar_gen = smem_raw + (bar_base - base);
    const float *part = reinterpret_cast<const float *>(smem_raw + (s_part - base));
    uint32_t *tmem_ptr = reinterpret_cast<uint32_t *>(bar_gen + 8 * kBars);
    volatile uint32_t *abort_flag = reinterpret_cast<volatile uint32_t *>(bar_gen + 8 * kBars + 4);
    // sums are missing, this CTA's own or those of another of its cluster: a wait ran out, y is left alone
    volatile uint32_t *failed = abort_flag + 1;
    auto bar = [&](int i) { return bar_base + 8u * i; };

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x, ranks = gridDim.x;   // the cluster is the grid's x extent
    const int group = blockIdx.y, m0 = blockIdx.z * p.x_rows;
    const int stage0 = rank * p.per_cta;
    const int stages = min(p.per_cta, p.stages - stage0);
    const bool aligned = (base & 1023u) == 0;         // what the swizzled operand layout needs

    auto load_codes = [&](int s) {
        const int st = s % p.ring, chunk0 = (stage0 + s) * kChunksPerStage;
        const uint32_t sf_bytes = 512u * static_cast<uint32_t>(min(kChunksPerStage, p.chunks_k - chunk0));
        ptx::mbar_arrive_expect_tx(bar(kFull + st), kCodeBytes + sf_bytes);
        ptx::tma_load_2d(s_code + st * kCodeBytes, &tm_w, (stage0 + s) * (kStageK / 2), group * kRows, bar(kFull + st));
        ptx::bulk_load_1d(s_sf + st * kSfBytes, p.wsf + (static_cast<int64_t>(group) * p.chunks_k + chunk0) * 512, sf_bytes, bar(kFull + st));
    };
    auto load_x = [&](int s) {
        const int st = s % p.ring;
        ptx::mbar_arrive_expect_tx(bar(kXFull + st), x_bytes);
        ptx::bulk_load_1d(s_x + st * x_bytes, p.ximage + (static_cast<int64_t>(blockIdx.z) * p.stages + stage0 + s) * x_bytes, x_bytes, bar(kXFull + st));
    };
    const int first = min(stages, p.ring);
    // few rows of x: the second half of the converting warps prepares them; their loads go out ahead of the codes'
    constexpr int kHeld = kInlineStages * (kStageK / 8) * kInlineRows / (32 * kXWarps);
    const int me = warp - kConvWarps / 2;
    const int per_row = kXWarps >> (p.M > 2 ? 2 : p.M - 1), m = me / per_row;     // warps of a row: 8, 4 or 2
    const int chunks = stages * (kStageK / 8), live = min(chunks, (p.K - stage0 * kStageK) / 8), step = 32 * per_row;
    const int at = (me % per_row) * 32 + lane, id = me * 32 + lane;
    uint4 raw[kInline ? kHeld : 1];
    bool held = false;
    if (kInline && me >= 0 && me < kXWarps) {
        held = loads_held(p.status);
        const uint16_t *xrow = p.x + m * p.ldx + stage0 * kStageK;
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
            raw[j] = m < p.M && at + j * step < live ? __ldg(reinterpret_cast<const uint4 *>(xrow + 8 * (at + j * step))) : make_uint4(0, 0, 0, 0);
    }
    if (warp == kProducer && aligned) {
        if (ptx::elect_one()) {
            ptx::prefetch_tmap(&tm_w);
            for (int i = 0; i < p.ring; ++i) {
                ptx::mbar_init(bar(kFull + i), 1);
                ptx::mbar_init(bar(kXFull + i), kInline ? kXWarps : 1);
                ptx::mbar_init(bar(kEmpty + i), 1);
            }
            for (int i = 0; i < 2; ++i) {
                ptx::mbar_init(bar(kAFull + i), kConvWarps / 2);
                ptx::mbar_init(bar(kAEmpty + i), 1);
            }
            ptx::mbar_init(bar(kDone), 1);
            *abort_flag = 0;
            *failed = 0;
            ptx::fence_mbar_init();
            ptx::fence_proxy_async_smem();
            for (int s = 0; s < first; ++s) load_codes(s);
        }
        __syncwarp();
    }
    if (warp == kIssuer && aligned) {
        ptx::tmem_alloc(ptx::smem_u32(tmem_ptr), kTmemCols);
        ptx::tmem_relinquish();
    }
    if (!aligned && threadIdx.x == 0) atomicExch(p.status, 0xC00u);
    int ref = 0;        // MXFP4: largest scale exponent of this thread's row and slice
    if (kMx && warp < kConvWarps) {
        const uint8_t *c = p.wsf + (static_cast<int64_t>(group) * p.chunks_k + stage0 * kChunksPerStage) * 512 + lane * 16 + (warp & 3) * 4;
        const int n = min(stages * kChunksPerStage, p.chunks_k - stage0 * kChunksPerStage);
        uint32_t most = 0;    // the four warpgroups read a quarter of the row's words each
#pragma unroll 8
        for (int i = warp >> 2; i < n; i += 4) most = __vmaxu4(most, __ldg(reinterpret_cast<const uint32_t *>(c + i * 512)));
        ref = static_cast<int>(max(max(most & 255u, most >> 8 & 255u), max(most >> 16 & 255u, most >> 24)));
        row_most[warp >> 2][(warp & 3) * 32 + lane] = static_cast<uint8_t>(ref);
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    if (kMx && warp < kConvWarps) {
        const int row = (warp & 3) * 32 + lane;
        ref = max(max(row_most[0][row], row_most[1][row]), max(row_most[2][row], row_most[3][row]));
    }
    const uint32_t tmem = aligned ? *tmem_ptr : 0;
    if (ranks > 1) ptx::cluster_arrive();       // this CTA runs: the others may write their sums into it (awaited before the first such write)

    if (!aligned) {
    } else if (warp == kProducer) {
        // ------------------------------------------------------------ loads
        if (ptx::elect_one()) {
            if (!kInline) {
                held = loads_held(p.status);
                ptx::grid_dependency_wait();       // x is prepared
                for (int s = 0; !held && s < first; ++s) load_x(s);
            }
            for (int s = first; !held && s < stages; ++s) {
                if (!wait_bounded(bar(kEmpty + s % p.ring), static_cast<uint32_t>(s / p.ring - 1) & 1u, abort_flag, p.status, 0xC10u)) break;
                load_codes(s);
                if (!kInline) load_x(s);
            }
        }
        __syncwarp();
    } else if (warp == kIssuer) {
        // ------------------------------------------------------------ products
        if (ptx::elect_one()) {
            const uint32_t idesc = (1u << 4) | (static_cast<uint32_t>(p.x_rows >> 3) << 17) | (static_cast<uint32_t>(kRows >> 4) << 24);
            bool ok = true;
            for (int s = 0; s < stages; ++s) {
                const int st = s % p.ring, buf = s & 1;
                ok = wait_bounded(bar(kXFull + (kInline ? 0 : st)), kInline ? 0u : static_cast<uint32_t>(s / p.ring) & 1u, abort_flag, p.status, 0xC20u) &&
                     wait_bounded(bar(kAFull + buf), static_cast<uint32_t>(s >> 1) & 1u, abort_flag, p.status, 0xC21u);
                if (!ok) break;
                ptx::tc_fence_after_sync();
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint64_t b = ptx::smem_desc_sw128(s_x + (kInline ? s : st) * x_bytes + (i >> 2) * (p.x_rows * 128)) + 2u * (i & 3);
                    ptx::mma_bf16_a_tmem(tmem + kColD + (i % kSums) * kMaxXRows, tmem + kColA + buf * kColABuf + 8 * i, b, idesc, s > 0 || i >= kSums);
                }
                ptx::tc_commit(bar(kAEmpty + buf));
                ptx::tc_commit(bar(kEmpty + st));      // the codes were read before they became A
            }
            if (ok) ptx::tc_commit(bar(kDone));
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ codes -> FP16 in TMEM: thread = weight row
        const int half = (warp >> 2) & 1, odd = warp >> 3;
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t t_a = tmem + kColA + odd * kColABuf + half * (kColABuf / 2) + lanes;
        bool ok = true;
        if (kInline && odd) {
            // this slice of x, while the other two warpgroups convert the first stage: the warps of a row find its largest
            // element, every thread scales and places its columns
            for (int i = id; i < chunks * (p.x_rows - kInlineRows); i += 32 * kXWarps)      // rows that never exist
                sts128(s_x + static_cast<uint32_t>(image_offset(i / (p.x_rows - kInlineRows), kInlineRows + i % (p.x_rows - kInlineRows), p.x_rows)), make_uint4(0, 0, 0, 0));
            float f[8], most = 0.0f;
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                if (j * step >= live) break;
                activate8(raw[j], p.act, f);
                most = largest8(f, most);
            }
            const uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));
            if (lane == 0) warp_most[me] = bits;
            asm volatile("bar.sync 1, %0;" ::"n"(32 * kXWarps) : "memory");
            uint32_t row_bits = 0;
            for (int i = 0; i < per_row; ++i) row_bits = max(row_bits, warp_most[m * per_row + i]);
            const float up = scale_up(row_bits);
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                if (at + j * step >= chunks) break;
                activate8(raw[j], p.act, f);
                sts128(s_x + static_cast<uint32_t>(image_offset(at + j * step, m, p.x_rows)), to_half8(f, up));
            }
            for (int i = id; i < chunks * (kInlineRows - kXWarps / per_row); i += 32 * kXWarps)     // rows without warps
                sts128(s_x + static_cast<uint32_t>(image_offset(i % chunks, kXWarps / per_row + i / chunks, p.x_rows)), make_uint4(0, 0, 0, 0));
            ptx::fence_proxy_async_smem();      // the tensor core reads x through the async proxy
            __syncwarp();
            if (lane == 0 && !held) ptx::mbar_arrive(bar(kXFull));
        }
        for (int s = odd; s < stages; s += 2) {
            const int st = s % p.ring;
            if (!warp_wait(bar(kFull + st), static_cast<uint32_t>(s / p.ring) & 1u, abort_flag, p.status, 0xC40u | st)) {
                ok = false;
                break;
            }
            uint4 q[4];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                q[c] = ptx::lds128(s_code + st * kCodeBytes + row * 128 + (((4 * half + c) ^ (row & 7)) << 4));
            uint32_t sf[2] = {0, 0};
            const uint32_t sf_at = s_sf + st * kSfBytes + lane * 16 + (warp & 3) * 4;
#pragma unroll
            for (int c = 0; c < kChunksPerStage / 2; ++c) {   // chunks behind the last are not loaded: their codes are zeros
                const int chunk = half * (kChunksPerStage / 2) + c;
                if ((stage0 + s) * kChunksPerStage + chunk < p.chunks_k) sf[c] = lds32(sf_at + chunk * 512);
            }
            uint32_t h[2][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) {          // 32 codes: two NVFP4 blocks or one MXFP4 block
                uint32_t s0, s1;
                if (kMx) {
                    s0 = s1 = mx_scale_half2(ref - static_cast<int>(sf[0] >> (8 * c) & 255u));
                } else {
                    const uint32_t pair = e4m3x2_to_half2(sf[c >> 1] >> (16 * (c & 1)));
                    s0 = __byte_perm(pair, pair, 0x1010);
                    s1 = __byte_perm(pair, pair, 0x3232);
                }
                uint32_t *to = &h[c >> 1][16 * (c & 1)];
                codes_to_half(q[c].x, s0, to);
                codes_to_half(q[c].y, s0, to + 4);
                codes_to_half(q[c].z, s1, to + 8);
                codes_to_half(q[c].w, s1, to + 12);
            }
            if (s > 1 && !warp_wait(bar(kAEmpty + odd), static_cast<uint32_t>((s >> 1) - 1) & 1u, abort_flag, p.status, 0xC50u | odd)) {
                ok = false;
                break;
            }
            ptx::tc_fence_after_sync();
            ptx::tmem_st_32x32(t_a, h[0]);
            ptx::tmem_st_32x32(t_a + 32, h[1]);
            ptx::tc_wait_st();
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(kAFull + odd));
        }
        // ------------------------------------------------------------ this slice's sums, to the rank that owns the column
        // The scalings of x, of the MXFP4 scales and T's exponent are undone as one power of two: one after the other they
        // may leave FP32's range on the way to a finite sum.
        constexpr int kSteps = kInline ? 1 : kMaxXRows / 32, kStepRows = kInline ? kInlineRows : 8;      // rows of x in each of the four warpgroups
        int undo[kSteps][kStepRows];
        if (!kInline && ok) {
            ptx::grid_dependency_wait();        // returns at once: x_exp was written with the x that is being multiplied
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int c = 8 * (warp >> 2) + 32 * i;
                if (c < p.x_rows) {
                    const int4 *from = reinterpret_cast<const int4 *>(p.x_exp + m0 + c);
                    const int4 a = __ldcg(from), b = __ldcg(from + 1);
                    const int all[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int e = 0; e < kStepRows; ++e) undo[i][e] = all[e];
                }
            }
        }
        int base_exp = ref - 127 - kMxExp;
        if (!kMx) split_scale(__ldg(p.wts), base_exp);
        ok = ok && warp_wait(bar(kDone), 0, abort_flag, p.status, 0xC60u);
        if (kInline) ok = ok && warp_wait(bar(kXFull), 0, abort_flag, p.status, 0xC61u);    // long complete: warp_most is in view
        if (ranks > 1) ptx::cluster_wait();
        if (!ok && lane < ranks) st_cluster(ptx::map_to_cta(bar_base + 8 * kBars + 8, lane), 1u);
        if (ok) {
            if (kInline) {     // the slice's own scaling of each row
#pragma unroll
                for (int r = 0; r < kInlineRows; ++r) {
                    uint32_t bits = 0;
                    for (int i = r * per_row; i < (r + 1) * per_row && i < kXWarps; ++i) bits = max(bits, warp_most[i]);
                    undo[0][r] = exponent_back(bits);
                }
            }
            ptx::tc_fence_after_sync();
            const int own = kRows / ranks;
            const uint32_t to = ptx::map_to_cta(s_part + (rank * p.x_rows * own + row % own) * 4, row / own);
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                const int c = 8 * (warp >> 2) + 32 * j;
                if (c >= (kInline ? kInlineRows : p.x_rows)) break;
                uint32_t d[kSums][8];
#pragma unroll
                for (int i = 0; i < kSums; ++i) ptx::tmem_ld_32x8(tmem + kColD + i * kMaxXRows + lanes + c, d[i]);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < kStepRows; ++e) {
                    float v = __uint_as_float(d[0][e]);
#pragma unroll
                    for (int i = 1; i < kSums; ++i) v += __uint_as_float(d[i][e]);
                    st_cluster(to + (c + e) * own * 4, PowerOfTwo(base_exp + undo[j][e]).times(v));
                }
            }
        }
    }
    if (ranks > 1 && (!aligned || warp >= kConvWarps)) ptx::cluster_wait();
    ptx::tc_fence_before_sync();

    // ---------------------------------------------------------------- own columns: sum over the ranks, scale, bias, store
    const int own = kRows / ranks, pairs = own / 2, rows = min(p.x_rows, p.M - m0);
    const int r = 2 * (threadIdx.x % pairs), n = group * kRows + rank * own + r;
    int t_exp;                          // (already in the sums)
    const float T = kMx ? 1.0f : split_scale(__ldg(p.wts), t_exp);
    uint32_t b2 = 0;
    if (aligned && *abort_flag) __nanosleep(2000000);  // let copies already in flight land before the CTA exits
    if (p.bias != nullptr && n < p.N) b2 = __ldg(reinterpret_cast<const uint32_t *>(p.bias + n));
    if (ranks > 1) ptx::cluster_sync();
    else __syncthreads();
    const bool store = aligned && *failed == 0 && warp < kConvWarps && n < p.N;
    for (int i = threadIdx.x / pairs; store && i < rows; i += 32 * kConvWarps / pairs) {
        float v0 = 0.0f, v1 = 0.0f;
        for (int c = 0; c < ranks; ++c) {
            const float2 v = *reinterpret_cast<const float2 *>(part + (c * p.x_rows + i) * own + r);
            v0 += v.x;
            v1 += v.y;
        }
        const float y0 = fmaf(v0, T, qmath::bf16_lo(b2)), y1 = fmaf(v1, T, qmath::bf16_hi(b2));
        uint32_t o;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(y1), "f"(y0));
        *reinterpret_cast<uint32_t *>(p.y + (m0 + i) * p.ldy + n) = o;
    }
    if (warp == kIssuer && aligned) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, kTmemCols);
    }
}

int x_rows_of(int64_t M) { return M >= kMaxXRows ? kMaxXRows : static_cast<int>(16 * ceil_div(M, 16)); }
int ring_of(int x_rows) {
    int ring = kMaxStages;
    while (smem_bytes(x_rows, ring, ring) > kMaxSmem) --ring;
    return ring;
}

// Most clusters of `ranks` CTAs that the device holds at once (one CTA per SM; clusters do not span GPCs).
template <bool kMx, bool kInline>
int resident_clusters(int dev, int ranks) {
    static int known[64][kMaxCluster + 1] = {};
    if (known[dev][ranks] == 0) {
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(static_cast<unsigned>(ranks));
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = kMaxSmem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {static_cast<unsigned>(ranks), 1, 1};
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, matvec_kernel<kMx, kInline>, &cfg) != cudaSuccess || n < 1) {
            cudaGetLastError();
            n = 1;
        }
        known[dev][ranks] = n;
    }
    return known[dev][ranks];
}

// K is shared by the largest cluster (of two, four or eight CTAs) that still runs in one wave.
template <bool kMx, bool kInline>
bool share_k(Params &p, int &ranks) {
    auto kern = matvec_kernel<kMx, kInline>;
    static bool configured[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem) != cudaSuccess) return false;
        configured[dev] = true;
    }
    const int64_t ctas = ceil_div(p.N, kRows) * ceil_div(p.M, p.x_rows);
    ranks = 1;
    while (2 * ranks <= kMaxCluster && 2 * ranks <= p.stages && ctas <= resident_clusters<kMx, kInline>(dev, 2 * ranks)) ranks *= 2;
    p.per_cta = static_cast<int>(ceil_div(p.stages, ranks));
    while (ranks > 1 && (ranks - 1) * p.per_cta >= p.stages) {    // every rank needs a stage
        ranks /= 2;
        p.per_cta = static_cast<int>(ceil_div(p.stages, ranks));
    }
    return true;
}

template <bool kMx, bool kInline>
sol_status_t launch_products(const CUtensorMap &tm_w, const Params &p, int ranks, cudaStream_t stream) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(ranks), static_cast<unsigned>(ceil_div(p.N, kRows)), static_cast<unsigned>(ceil_div(p.M, p.x_rows)));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = static_cast<size_t>(smem_bytes(p.x_rows, p.ring, kInline ? p.per_cta : p.ring));
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {static_cast<unsigned>(ranks), 1, 1};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kInline ? 1 : 2;
    if (cudaLaunchKernelEx(&cfg, matvec_kernel<kMx, kInline>, tm_w, p) != cudaSuccess) {
        cudaGetLastError();
        return SOL_ERR_CUDA;
    }
    return launch_status();
}

template <bool kMx>
sol_status_t launch(const void *x, int64_t ldx, bool silu, void *workspace, const CUtensorMap &tm_w, Params &p, int64_t K, cudaStream_t stream) {
    int ranks = 1;
    if (prepared_inline(p.M, K)) {
        if (!share_k<kMx, true>(p, ranks)) return SOL_ERR_CUDA;
        p.x = static_cast<const uint16_t *>(x);
        p.ldx = ldx;
        p.K = static_cast<int>(K);
        p.act = silu ? 1 : 0;
        return launch_products<kMx, true>(tm_w, p, ranks, stream);
    }
    if (!share_k<kMx, false>(p, ranks)) return SOL_ERR_CUDA;
    const int64_t row_chunks = ceil_div(p.M, p.x_rows);
    uint8_t *image = static_cast<uint8_t *>(workspace);
    int *x_exp = reinterpret_cast<int *>(image + row_chunks * p.stages * stage_x_bytes(p.x_rows));
    p.ximage = image;
    p.x_exp = x_exp;
    prepare_x<<<static_cast<unsigned>(row_chunks * p.x_rows), kPrepThreads, 0, stream>>>(
        static_cast<const uint16_t *>(x), ldx, p.M, static_cast<int>(K), p.x_rows, p.stages, silu ? 1 : 0, image, x_exp);
    const sol_status_t st = launch_status();
    return st != SOL_OK ? st : launch_products<kMx, false>(tm_w, p, ranks, stream);
}

}  // namespace

size_t workspace_bytes(int64_t M, int64_t K) {
    if (prepared_inline(M, K)) return 0;
    const int x_rows = x_rows_of(M);
    const int64_t chunks = ceil_div(M, x_rows);
    return static_cast<size_t>(chunks * ceil_div(K, kStageK) * stage_x_bytes(x_rows) + chunks * x_rows * 4);
}

sol_status_t launch_matvec(const void *x, int64_t ldx, const void *wq, const void *wsf, const float *wts, const void *bias, void *y,
                           int64_t ldy, int64_t M, int64_t N, int64_t K, bool silu, void *workspace, cudaStream_t stream) {
    Params p{};
    p.wsf = static_cast<const uint8_t *>(wsf);
    p.wts = wts;
    p.bias = static_cast<const uint16_t *>(bias);
    p.y = static_cast<uint16_t *>(y);
    p.status = device_status_word();
    p.ldy = ldy;
    p.M = static_cast<int>(M);
    p.N = static_cast<int>(N);
    p.stages = static_cast<int>(ceil_div(K, kStageK));
    p.chunks_k = static_cast<int>(ceil_div(K, wts != nullptr ? 64 : 128));
    p.x_rows = x_rows_of(M);
    p.ring = ring_of(p.x_rows);
    CUtensorMap tm_w;
    if (!make_tmap_2d(&tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, wq, static_cast<uint64_t>(K / 2), static_cast<uint64_t>(N),
                      static_cast<uint64_t>(K / 2), kStageK / 2, kRows, CU_TENSOR_MAP_SWIZZLE_128B))
        return SOL_ERR_CUDA;
    return wts != nullptr ? launch<false>(x, ldx, silu, workspace, tm_w, p, K, stream) : launch<true>(x, ldx, silu, workspace, tm_w, p, K, stream);
}

}  // namespace matvec
}  // namespace sol
