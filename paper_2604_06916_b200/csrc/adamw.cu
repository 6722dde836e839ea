// One AdamW step over many tensors (sm_100a).  Per element, with t the step and every operation rounded in FP32:
//     m = b1 m + (1 - b1) g;   v = b2 v + (1 - b2) g^2
//     p = p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// The tensors' addresses are the kernel's parameter (up to kTable of them a launch), so a step over a few hundred adapters is one
// launch, from host arrays, and can be captured; the step counter is on the device and counts replays too: every block takes a
// ticket when it has read it, the one with the last ticket writes it back.
//
// States in 8 bits: blocks of 32 values under a power of two (E8M0, as in the MXFP4 tensors), m in E4M3, v in E5M2 (it is a
// square: twice the exponents).  A value keeps three or two mantissa bits, which is coarser than what a step adds to v at b2 = 0.999:
// rounded to nearest, v would stay where it is.  So it is rounded up or down by chance, in proportion (16 random bits a value, by
// hashing seed, step, tensor and place): the average moves as the 32-bit state does.  The powers of two put the block's largest value
// at [2^7, 2^8) of E4M3, [2^14, 2^15) of E5M2, so rounding up never leaves the format.
// The new parameter comes from m and v before they are rounded.
//
// HBM bound: 28 bytes per element in FP32 (30 with the BF16 copy), 16.1 with 8-bit states, 10.1 with BF16 parameters as well.  A thread
// takes eight neighbouring values (16-byte accesses, a block of 32 is four lanes).
#include "ptx.cuh"
#include "quant_math.cuh"
#include "sol_internal.h"

#include <type_traits>

namespace sol {
namespace adamw {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;                        // values of a thread
constexpr int kChunk = kThreads * kVec;        // values of a block at a time
constexpr int kTable = 448, kSmallTable = 16;  // tensors of a launch

struct Hyper {
    double lr, beta1, beta2, decay;
    float b1, c1, b2, c2, eps;                 // c = 1 - b
    const float *lr_scale, *grad_scale;        // device, or null
    long long *state;                          // [0] steps done, [1] tickets
    uint64_t seed;
    uint32_t first_tensor, chunks;
    int count, stochastic, advance;
};
template <int kN>
struct Table {
    Tensor t[kN];
    uint32_t first[kN + 1];                    // chunk that each tensor begins with
};

__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ x >> 16;
}
__device__ __forceinline__ uint32_t mix_word(uint32_t h, uint32_t w) { return mix(h ^ (w + 0x9E3779B9u)); }

__device__ __forceinline__ void load(float (&f)[kVec], const float *p) {
    const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}
__device__ __forceinline__ void load(float (&f)[kVec], const uint16_t *p) {
    const uint4 r = __ldcs(reinterpret_cast<const uint4 *>(p));
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = qmath::bf16_lo(w[i]), f[2 * i + 1] = qmath::bf16_hi(w[i]);
}
__device__ __forceinline__ float one(const float *p) { return *p; }
__device__ __forceinline__ float one(const uint16_t *p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); }
__device__ __forceinline__ void store(float *p, const float (&f)[kVec]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ uint32_t bf16_rn(float f) {
    uint16_t r;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(f));
    return r;
}

// kMantissa 3: E4M3, values 2^120 times those of the FP32 number with the code's bits on top; 2: E5M2, 2^112 times.
template <int kMantissa>
struct Format {
    static constexpr int kDrop = 23 - kMantissa;
    static constexpr uint32_t kTop = kMantissa == 3 ? 7 : 14;          // exponent of a block's largest value
    static constexpr float kUp = kMantissa == 3 ? 0x1p120f : 0x1p112f, kDown = kMantissa == 3 ? 0x1p-120f : 0x1p-112f;
};
// The 7-bit code of y in [0, 2^kTop+1): to nearest, or up or down by chance.  By chance: scaled down so that its bits are the
// code's, further down (exact but for subnormal codes, where what lies below a 2^-kDrop of a step is rounded), plus the noise's 16
// bits below the code's, in the middle of what they stand for.
template <int kMantissa>
__device__ __forceinline__ uint32_t round_code(float y, uint32_t noise16, bool stochastic) {
    using F = Format<kMantissa>;
    if (stochastic) return (__float_as_uint(__fmul_rn(y, F::kDown)) + (noise16 << (F::kDrop - 16)) + (1u << (F::kDrop - 17))) >> F::kDrop;
    uint16_t r;
    if constexpr (kMantissa == 3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(y));
    else asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(y));
    return r;
}
template <int kMantissa>
__device__ __forceinline__ void decode(float (&f)[kVec], uint2 codes, uint32_t e) {
    using F = Format<kMantissa>;
    const float scale = __uint_as_float(e << 23);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const uint32_t c = (i < 4 ? codes.x : codes.y) >> (8 * (i & 3));
        const float size = __fmul_rn(__fmul_rn(__uint_as_float((c & 127u) << F::kDrop), F::kUp), scale);
        f[i] = __uint_as_float(((c & 127u) == 127u ? 0x7FC00000u : __float_as_uint(size)) | (c & 128u) << 24);
    }
}
// The codes of a thread's eight values and the exponent byte of its block (lanes 4i .. 4i+3); values that are not finite become
// NaN and do not count for the block.
template <int kMantissa>
__device__ __forceinline__ uint2 encode(const float (&f)[kVec], uint32_t &e, const uint32_t (&noise)[kVec], int noise_shift, bool stochastic) {
    using F = Format<kMantissa>;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const uint32_t b = __float_as_uint(f[i]) & 0x7FFFFFFFu;
        most = max(most, b < 0x7F800000u ? b : 0u);
    }
    most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
    most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
    e = max(most >> 23, F::kTop + 1u) - F::kTop;
    const float inv = __uint_as_float((254u - e) << 23);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const uint32_t b = __float_as_uint(f[i]), size = b & 0x7FFFFFFFu;
        const uint32_t c = round_code<kMantissa>(__fmul_rn(__uint_as_float(size), inv), (noise[i] >> noise_shift) & 0xFFFFu, stochastic) & 127u;
        w[i >> 2] |= ((size < 0x7F800000u ? c : 127u) | b >> 31 << 7) << (8 * (i & 3));
    }
    return make_uint2(w[0], w[1]);
}

template <int kN, bool kP16, bool kG16, bool k8>
__global__ void __launch_bounds__(kThreads)
step_kernel(const __grid_constant__ Table<kN> table, const __grid_constant__ Hyper h) {
    using P = typename std::conditional<kP16, uint16_t, float>::type;
    using G = typename std::conditional<kG16, uint16_t, float>::type;
    using S = typename std::conditional<k8, uint8_t, float>::type;
    constexpr bool kNoise = kP16 || k8;
    __shared__ float coefficients[3];      // 1 - lr decay, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    __shared__ uint32_t hash;              // of seed and step
    if (threadIdx.x == 0) {
        const long long t = *reinterpret_cast<volatile long long *>(h.state) + 1;
        // b^t by squaring, in FP64
        double p1 = 1.0, p2 = 1.0, q1 = h.beta1, q2 = h.beta2;
        for (unsigned long long n = t; n != 0; n >>= 1) {
            if (n & 1) p1 *= q1, p2 *= q2;
            q1 *= q1, q2 *= q2;
        }
        const double lr = h.lr_scale != nullptr ? h.lr * *h.lr_scale : h.lr;
        coefficients[0] = static_cast<float>(1.0 - lr * h.decay);
        coefficients[1] = static_cast<float>(lr / (1.0 - p1));
        coefficients[2] = static_cast<float>(1.0 / sqrt(1.0 - p2));
        hash = mix_word(mix_word(mix_word(mix_word(0u, static_cast<uint32_t>(h.seed)), static_cast<uint32_t>(h.seed >> 32)),
                                 static_cast<uint32_t>(t)), static_cast<uint32_t>(t >> 32));
        if (h.advance) {
            unsigned long long *ticket = reinterpret_cast<unsigned long long *>(h.state + 1);
            __threadfence();
            if (atomicAdd(ticket, 1ull) == gridDim.x - 1) {    // every block has read the counter
                h.state[0] = t;
                *ticket = 0;
            }
        }
    }
    __syncthreads();
    const float keep = coefficients[0], size = coefficients[1], root = coefficients[2];
    const float grad_scale = h.grad_scale != nullptr ? __ldg(h.grad_scale) : 1.0f;
    for (uint32_t chunk = blockIdx.x; chunk < h.chunks; chunk += gridDim.x) {
        int lo = 0, hi = h.count;          // the last tensor that begins at or before this chunk
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (table.first[mid] <= chunk) lo = mid;
            else hi = mid;
        }
        const Tensor &t = table.t[lo];
        const int64_t i0 = static_cast<int64_t>(chunk - table.first[lo]) * kChunk + threadIdx.x * kVec;
        const int64_t left = t.n - i0;     // a thread without values still takes part in its block's maximum
        float p[kVec], g[kVec], m[kVec], v[kVec];
        uint2 cm = make_uint2(0, 0), cv = make_uint2(0, 0);
        uint32_t em = 0, ev = 0;
        P *pp = static_cast<P *>(t.param) + i0;
        const G *gp = static_cast<const G *>(t.grad) + i0;
        S *mp = static_cast<S *>(t.m) + i0, *vp = static_cast<S *>(t.v) + i0;
        if (left >= kVec) {
            load(p, pp);
            load(g, gp);
            if constexpr (k8) {
                cm = __ldcs(reinterpret_cast<const uint2 *>(mp));
                cv = __ldcs(reinterpret_cast<const uint2 *>(vp));
            } else {
                load(m, mp);
                load(v, vp);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                p[i] = g[i] = m[i] = v[i] = 0.0f;
                if (i < left) {
                    p[i] = one(pp + i);
                    g[i] = one(gp + i);
                    if constexpr (k8) {
                        (i < 4 ? cm.x : cm.y) |= static_cast<uint32_t>(mp[i]) << (8 * (i & 3));
                        (i < 4 ? cv.x : cv.y) |= static_cast<uint32_t>(vp[i]) << (8 * (i & 3));
                    } else {
                        m[i] = mp[i];
                        v[i] = vp[i];
                    }
                }
            }
        }
        if constexpr (k8) {
            if (left > 0) {
                em = static_cast<const uint8_t *>(t.m_scale)[i0 >> 5];
                ev = static_cast<const uint8_t *>(t.v_scale)[i0 >> 5];
            }
            decode<3>(m, cm, em);
            decode<2>(v, cv, ev);
        }
        uint32_t noise[kVec] = {};
        if (kNoise && h.stochastic) {
            uint32_t base = mix_word(hash, h.first_tensor + lo);
            if (i0 >> 32) base = mix(base ^ static_cast<uint32_t>(i0 >> 32));
#pragma unroll
            for (int i = 0; i < kVec; ++i) noise[i] = mix(base ^ (static_cast<uint32_t>(i0) + i));
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float gi = __fmul_rn(g[i], grad_scale);
            m[i] = __fadd_rn(__fmul_rn(m[i], h.b1), __fmul_rn(gi, h.c1));
            v[i] = __fadd_rn(__fmul_rn(v[i], h.b2), __fmul_rn(__fmul_rn(gi, gi), h.c2));
            float r;
            asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v[i]));
            p[i] = fmaf(p[i], keep, -__fdividef(m[i] * size, fmaf(r, root, h.eps)));
        }
        uint32_t short_p[kVec];
        if constexpr (kP16) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const uint32_t b = __float_as_uint(p[i]);
                const bool by_chance = h.stochastic && (b & 0x7F800000u) != 0x7F800000u;
                short_p[i] = by_chance ? (b + (noise[i] * 0x9E3779B1u >> 16)) >> 16 : bf16_rn(p[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) short_p[i] = bf16_rn(p[i]);
        }
        if constexpr (k8) {
            if (left < kVec) {
#pragma unroll
                for (int i = 0; i < kVec; ++i)
                    if (i >= left) m[i] = v[i] = 0.0f;        // behind the end: nothing that counts for the block
            }
            cm = encode<3>(m, em, noise, 0, h.stochastic);
            cv = encode<2>(v, ev, noise, 16, h.stochastic);
            if (left > 0 && (threadIdx.x & 3) == 0) {
                static_cast<uint8_t *>(t.m_scale)[i0 >> 5] = static_cast<uint8_t>(em);
                static_cast<uint8_t *>(t.v_scale)[i0 >> 5] = static_cast<uint8_t>(ev);
            }
        }
        uint16_t *copy = kP16 ? nullptr : static_cast<uint16_t *>(t.copy);
        if (left >= kVec) {
            const uint4 packed = make_uint4(short_p[0] | short_p[1] << 16, short_p[2] | short_p[3] << 16, short_p[4] | short_p[5] << 16,
                                            short_p[6] | short_p[7] << 16);
            if constexpr (kP16) *reinterpret_cast<uint4 *>(pp) = packed;
            else store(pp, p);
            if (copy != nullptr) *reinterpret_cast<uint4 *>(copy + i0) = packed;
            if constexpr (k8) {
                *reinterpret_cast<uint2 *>(mp) = cm;
                *reinterpret_cast<uint2 *>(vp) = cv;
            } else {
                store(mp, m);
                store(vp, v);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                if (i >= left) continue;
                if constexpr (kP16) pp[i] = static_cast<uint16_t>(short_p[i]);
                else pp[i] = p[i];
                if (copy != nullptr) copy[i0 + i] = static_cast<uint16_t>(short_p[i]);
                if constexpr (k8) {
                    mp[i] = static_cast<uint8_t>((i < 4 ? cm.x : cm.y) >> (8 * (i & 3)));
                    vp[i] = static_cast<uint8_t>((i < 4 ? cv.x : cv.y) >> (8 * (i & 3)));
                } else {
                    mp[i] = m[i];
                    vp[i] = v[i];
                }
            }
        }
    }
}

template <int kN, bool kP16, bool kG16, bool k8>
sol_status_t launch_table(const Tensor *tensors, Hyper h, cudaStream_t stream, const DeviceInfo *dev) {
    Table<kN> table;
    uint64_t chunks = 0;
    for (int i = 0; i < h.count; ++i) {
        table.t[i] = tensors[i];
        table.first[i] = static_cast<uint32_t>(chunks);
        chunks += static_cast<uint64_t>(ceil_div(tensors[i].n, kChunk));
        if (chunks > 0xFFFFFFFFull) return SOL_ERR_BAD_SHAPE;
    }
    for (int i = h.count; i <= kN; ++i) table.first[i] = static_cast<uint32_t>(chunks);
    for (int i = h.count; i < kN; ++i) table.t[i] = Tensor{};
    h.chunks = static_cast<uint32_t>(chunks);
    static int resident = 0;
    if (resident == 0 && cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, step_kernel<kN, kP16, kG16, k8>, kThreads, 0) != cudaSuccess) {
        cudaGetLastError();
        return SOL_ERR_CUDA;
    }
    const int64_t most = static_cast<int64_t>(resident) * dev->sm_count;
    const int64_t grid = static_cast<int64_t>(chunks) < most ? static_cast<int64_t>(chunks) : most;
    step_kernel<kN, kP16, kG16, k8><<<static_cast<unsigned>(grid < 1 ? 1 : grid), kThreads, 0, stream>>>(table, h);
    return launch_status();
}

template <bool kP16, bool kG16, bool k8>
sol_status_t launch_all(const Tensor *tensors, int64_t count, Hyper h, cudaStream_t stream, const DeviceInfo *dev) {
    int64_t first = 0;
    do {
        h.first_tensor = static_cast<uint32_t>(first);
        h.count = static_cast<int>(count - first < kTable ? count - first : kTable);
        h.advance = first + h.count == count;
        const sol_status_t st = h.count <= kSmallTable ? launch_table<kSmallTable, kP16, kG16, k8>(tensors + first, h, stream, dev)
                                                       : launch_table<kTable, kP16, kG16, k8>(tensors + first, h, stream, dev);
        if (st != SOL_OK) return st;
        first += h.count;
    } while (first < count);
    return SOL_OK;
}

}  // namespace

sol_status_t launch_step(const Tensor *tensors, int64_t count, const sol_adamw_options_t &o, int64_t *state, cudaStream_t stream,
                         const DeviceInfo *dev) {
    Hyper h{};
    h.lr = o.lr, h.beta1 = o.beta1, h.beta2 = o.beta2, h.decay = o.weight_decay;
    h.b1 = static_cast<float>(o.beta1), h.c1 = static_cast<float>(1.0 - o.beta1);
    h.b2 = static_cast<float>(o.beta2), h.c2 = static_cast<float>(1.0 - o.beta2);
    h.eps = static_cast<float>(o.eps);
    h.lr_scale = o.lr_scale, h.grad_scale = o.grad_scale;
    h.state = reinterpret_cast<long long *>(state);
    h.seed = o.seed, h.stochastic = o.stochastic != 0;
    const bool e = o.state_bits == 8;
    if (o.param_bf16) {
        if (o.grad_bf16) return e ? launch_all<true, true, true>(tensors, count, h, stream, dev) : launch_all<true, true, false>(tensors, count, h, stream, dev);
        return e ? launch_all<true, false, true>(tensors, count, h, stream, dev) : launch_all<true, false, false>(tensors, count, h, stream, dev);
    }
    if (o.grad_bf16) return e ? launch_all<false, true, true>(tensors, count, h, stream, dev) : launch_all<false, true, false>(tensors, count, h, stream, dev);
    return e ? launch_all<false, false, true>(tensors, count, h, stream, dev) : launch_all<false, false, false>(tensors, count, h, stream, dev);
}

}  // namespace adamw
}  // namespace sol
