// One AdamW step over many tensors (sm_100a).  Per element in FP32, with t the step:
//     m = b1 m + (1 - b1) g;   v = b2 v + (1 - b2) g^2          (every operation rounded)
//     p = p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// In the second line root and quotient are approximate instructions (2^-22 each) and products are fused with their sums: that touches the
// last places of an update, which is itself far below the parameter; the moments, which are compared bit for bit, are not approximate.
// The tensors' addresses are the kernel's parameter (up to kTable of them a launch), so a step over a few hundred adapters is one
// launch, from host arrays, and can be captured; the step counter is on the device and counts replays too: every block takes a
// ticket when it has read it, the one with the last ticket writes it back.
//
// States in 8 bits: blocks of 32 values under a power of two (E8M0, as in the MXFP4 tensors), m in E4M3, v in E5M2 (it is a
// square: twice the exponents).  A value keeps three or two mantissa bits, which is coarser than what a step adds to v at b2 = 0.999:
// rounded to nearest, v would stay where it is.  So it is rounded up or down by chance, in proportion (16 random bits a value, by
// hashing seed, step, tensor and place): the average moves as the 32-bit state does.  The hash's mixer is a published one of two products
// and three shifts, lowbias32 (C. Wellons' hash-prospector).  The powers of two put the block's largest value at [2^7, 2^8) of E4M3,
// [2^14, 2^15) of E5M2, so rounding up never leaves the format.
// The new parameter comes from m and v before they are rounded.
//
// HBM bound in FP32: 28 bytes per element (30 with the BF16 copy); 18.1 with 8-bit states and a copy; 10.1 with BF16 parameters and
// gradients as well, where issuing is the bound (62 instructions a value: hash 9, encoding 14, decoding and the parameter's rounding 3,
// the update 9).  A thread takes eight neighbouring values (a block of 32 is four lanes); FP32 goes in 32-byte accesses where the addresses
// allow it (304 tensors of 60 M values 304 us, with 16-byte ones 324).
// Measured (B200, inside a graph): 60 M FP32 values in 304 tensors with the BF16 copy 301 us = 6.0 TB/s, 91 % of the copy
// rate; 8-bit states 193 us = 5.6 TB/s; 71 M BF16 values with 8-bit states 179 us = 4.0 TB/s; 2 tensors of 98304 values 3.7 us.
// Neighbouring chunks for a block in place of every gridDim-th one: 226 us (8-bit states); loads a chunk ahead: 194 and 200 us (fewer
// blocks fit); every operation and conversion by itself, without the hardware's 8-bit conversions and byte permutes: 259 and 310 us;
// products one an instruction: 186 us on BF16 values; steps two by two 176 us, four by four 202 us.
#include "ptx.cuh"
#include "quant_math.cuh"
#include "sol_internal.h"

#include <atomic>
#include <type_traits>

namespace sol {
namespace adamw {
namespace {

using qmath::f32x2;
using qmath::f32x2_split;
using qmath::mul2;

constexpr int kThreads = 256;
constexpr int kVec = 8;                        // values of a thread
constexpr int kStep = kThreads * kVec;         // values of a block at a time
constexpr int kSteps = 4;                      // of a chunk, where it has more than one
constexpr int kTable = 448, kSmallTable = 16;  // tensors of a launch

struct Hyper {
    double lr, beta1, beta2, decay;
    float b1, c1, b2, c2, eps;                 // c = 1 - b
    const float *lr_scale, *grad_scale;        // device, or null
    long long *state;                          // [0] steps done, [1] tickets
    uint64_t seed;
    uint32_t first_tensor, chunks;
    int steps;                                 // of a chunk: a power of two
    int count, advance, tiny_eps;
};
template <int kN>
struct Table {
    Tensor t[kN];
    uint32_t first[kN + 1];                    // chunk that each tensor begins with
};

__device__ __forceinline__ uint32_t mix_rest(uint32_t x) {
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ x >> 16;
}
__device__ __forceinline__ uint32_t mix(uint32_t x) { return mix_rest(x ^ x >> 16); }
__device__ __forceinline__ uint32_t mix_word(uint32_t h, uint32_t w) { return mix(h ^ (w + 0x9E3779B9u)); }

// FP32 in one 32-byte access where the tensor's addresses allow it (`wide`): half an access a sector costs 7 % of the rate.
__device__ __forceinline__ void load(uint32_t (&w)[8], const float *p, bool wide) {
    if (!wide) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p)), b = __ldcs(reinterpret_cast<const uint4 *>(p) + 1);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
        return;
    }
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void load(uint32_t (&w)[4], const uint16_t *p, bool) {
    const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p));
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
}
__device__ __forceinline__ void load(uint32_t (&w)[2], const uint8_t *p, bool) {
    const uint2 a = __ldcs(reinterpret_cast<const uint2 *>(p));
    w[0] = a.x, w[1] = a.y;
}
// The same from a tensor's last values, 0 behind them.
template <int kWords, class T>
__device__ __forceinline__ void load_some(uint32_t (&w)[kWords], const T *p, int64_t left) {
    constexpr int kPer = 4 / sizeof(T);
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        w[i] = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (i * kPer + e >= left) continue;
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(p[i]);
            else w[i] |= static_cast<uint32_t>(p[i * kPer + e]) << (8 * sizeof(T) * e);
        }
    }
}
template <bool k16, int kWords>
__device__ __forceinline__ void unpack(float (&f)[kVec], const uint32_t (&w)[kWords]) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        if constexpr (k16) f[i] = i & 1 ? qmath::bf16_hi(w[i / 2]) : qmath::bf16_lo(w[i / 2]);
        else f[i] = __uint_as_float(w[i]);
    }
}
__device__ __forceinline__ void store(float *p, const float (&f)[kVec], bool wide) {
    if (!wide) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
        return;
    }
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]),
                 "f"(f[5]), "f"(f[6]), "f"(f[7])
                 : "memory");
}
// kMantissa 3: E4M3, values 2^120 times those of the FP32 number with the code's bits on top; 2: E5M2, 2^112 times.
template <int kMantissa>
struct Format {
    static constexpr int kDrop = 23 - kMantissa;
    static constexpr uint32_t kTop = kMantissa == 3 ? 7 : 14;          // exponent of a block's largest value
    static constexpr float kDown = kMantissa == 3 ? 0x1p-120f : 0x1p-112f;
};
// A block's eight codes of a thread and its exponent byte -> FP32.  The codes go through FP16, which holds both formats exactly (E5M2 is its
// upper byte), NaN and sign included.
__device__ __forceinline__ void halves_to_float(uint32_t pair, float scale, float *f) {
    float lo, hi;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(pair));
    f[0] = __fmul_rn(lo, scale);
    f[1] = __fmul_rn(hi, scale);
}
template <int kMantissa>
__device__ __forceinline__ void decode(float (&f)[kVec], uint2 codes, uint32_t e) {
    const float scale = __uint_as_float(e << 23);
#pragma unroll
    for (int i = 0; i < kVec; i += 2) {
        const uint32_t word = i < 4 ? codes.x : codes.y;
        uint32_t pair;
        if constexpr (kMantissa == 3) {
            const uint16_t two = static_cast<uint16_t>(word >> (8 * (i & 2)));
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(pair) : "h"(two));
        } else {
            pair = __byte_perm(word, 0, (i & 2) ? 0x3424 : 0x1404);     // codes into the upper bytes
        }
        halves_to_float(pair, scale, f + i);
    }
}
__device__ __forceinline__ bool finite_bits(uint32_t b) { return (b & 0x7F800000u) != 0x7F800000u; }

// The codes of a thread's eight values and the exponent byte of its block (lanes 4i .. 4i+3).  To nearest by the hardware's conversion.
// By chance: y scaled down so that its FP32 bits are the code's, further down (exact but for subnormal codes, where what lies below
// 2^-kDrop of a step is rounded), plus the noise's 16 bits below the code's, in the middle of what they leave open.  `odd`: some value
// of the warp is not finite; such values become NaN and do not count for the block.
template <int kMantissa, bool kChance>
__device__ __forceinline__ uint2 encode(const float (&f)[kVec], uint32_t &e, const uint32_t (&noise)[kVec], bool odd) {
    using F = Format<kMantissa>;
    float most = 0.0f;
    if (!odd) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) most = fmaxf(most, fabsf(f[i]));
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) most = fmaxf(most, finite_bits(__float_as_uint(f[i])) ? fabsf(f[i]) : 0.0f);
    }
    most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
    most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
    e = max(__float_as_uint(most) >> 23, F::kTop + 1u) - F::kTop;
    uint32_t c[kVec];                      // the code in the uppermost byte
    if constexpr (kChance) {
        // 2^(127 - e) and the format's 2^-120 (2^-112) in one factor where FP32 has it
        constexpr uint32_t kOne = kMantissa == 3 ? 134u : 142u;
        if (__all_sync(0xFFFFFFFFu, e < kOne)) {
            const float down = __uint_as_float((kOne - e) << 23);
#pragma unroll
            for (int i = 0; i < kVec; ++i) c[i] = __float_as_uint(__fmul_rn(fabsf(f[i]), down));
        } else {
            const float inv = __uint_as_float((254u - e) << 23);
#pragma unroll
            for (int i = 0; i < kVec; ++i) c[i] = __float_as_uint(__fmul_rn(__fmul_rn(fabsf(f[i]), inv), F::kDown));
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            // everything shifted so that the code is the uppermost byte: the noise is the two bytes below, a half of its last bit the third
            const uint32_t r = __byte_perm(noise[i], 0x80u, kMantissa == 3 ? 0x5104 : 0x5324);
            c[i] = (c[i] << (24 - F::kDrop)) + r;
        }
    } else {
        const float inv = __uint_as_float((254u - e) << 23);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float y = __fmul_rn(fabsf(f[i]), inv);
            uint16_t r;
            if constexpr (kMantissa == 3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(y));
            else asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(y));
            c[i] = static_cast<uint32_t>(r) << 24;
        }
    }
    if (odd) {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (!finite_bits(__float_as_uint(f[i]))) c[i] = 0x7F000000u;
    }
    if constexpr (kMantissa == 3) {        // squares have no sign
#pragma unroll
        for (int i = 0; i < kVec; ++i) c[i] = (c[i] & 0x7FFFFFFFu) | (__float_as_uint(f[i]) & 0x80000000u);
    }
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x73), __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x73), 0x5410);
    return make_uint2(w[0], w[1]);
}

template <int kN, bool kP16, bool kG16, bool k8, bool kChance>
__global__ void __launch_bounds__(kThreads, 4)
step_kernel(const __grid_constant__ Table<kN> table, const __grid_constant__ Hyper h) {
    using P = typename std::conditional<kP16, uint16_t, float>::type;
    using G = typename std::conditional<kG16, uint16_t, float>::type;
    using S = typename std::conditional<k8, uint8_t, float>::type;
    constexpr bool kNoise = (kP16 || k8) && kChance, kOdd = kP16 || k8;
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
    const uint64_t gs2 = f32x2(grad_scale, grad_scale), b1 = f32x2(h.b1, h.b1), c1 = f32x2(h.c1, h.c1), b2 = f32x2(h.b2, h.b2), c2 = f32x2(h.c2, h.c2);
    for (uint32_t chunk = blockIdx.x; chunk < h.chunks; chunk += gridDim.x) {
        int lo = 0, hi = h.count;          // the last tensor that begins at or before the chunk
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (table.first[mid] <= chunk) lo = mid;
            else hi = mid;
        }
        // everything that is the block's: addresses of the chunk, so that a thread has 32-bit offsets only
        const Tensor &t = table.t[lo];
        const int64_t base = static_cast<int64_t>(chunk - table.first[lo]) * kStep * h.steps;
        P *const p0 = static_cast<P *>(t.param) + base;
        const G *const g0 = static_cast<const G *>(t.grad) + base;
        S *const m0 = static_cast<S *>(t.m) + base, *const v0 = static_cast<S *>(t.v) + base;
        uint8_t *const ms0 = k8 ? static_cast<uint8_t *>(t.m_scale) + (base >> 5) : nullptr, *const vs0 = k8 ? static_cast<uint8_t *>(t.v_scale) + (base >> 5) : nullptr;
        uint16_t *const copy0 = kP16 || t.copy == nullptr ? nullptr : static_cast<uint16_t *>(t.copy) + base;
        const int here = static_cast<int>(min(t.n - base, static_cast<int64_t>(kStep) * h.steps));
        const bool wide = ((kP16 ? 0 : reinterpret_cast<uintptr_t>(p0)) | (kG16 ? 0 : reinterpret_cast<uintptr_t>(g0)) |
                           (k8 ? 0 : reinterpret_cast<uintptr_t>(m0) | reinterpret_cast<uintptr_t>(v0))) % 32 == 0;
        uint32_t noise_base = 0;
        if (kNoise) {
            noise_base = mix_word(hash, h.first_tensor + lo);
            if (base >> 32) noise_base = mix(noise_base ^ static_cast<uint32_t>(base >> 32));
            noise_base ^= static_cast<uint32_t>(base);
        }
        // kWhole: all threads have eight values; the others' way, value by value, is compiled apart
        auto step = [&](auto whole, uint32_t i0) {
            constexpr bool kWhole = decltype(whole)::value;
            const int left = here - static_cast<int>(i0);      // a thread without values still takes part in its block's maximum
            uint32_t rp[kVec * sizeof(P) / 4], rg[kVec * sizeof(G) / 4], rm[kVec * sizeof(S) / 4], rv[kVec * sizeof(S) / 4];
            uint32_t em = 0, ev = 0;
            if (kWhole || left >= kVec) {
                load(rp, p0 + i0, wide);
                load(rg, g0 + i0, wide);
                load(rm, m0 + i0, wide);
                load(rv, v0 + i0, wide);
            } else {
                load_some(rp, p0 + i0, left);
                load_some(rg, g0 + i0, left);
                load_some(rm, m0 + i0, left);
                load_some(rv, v0 + i0, left);
            }
            if (k8 && (kWhole || left > 0)) em = ms0[i0 >> 5], ev = vs0[i0 >> 5];
            float p[kVec], g[kVec], m[kVec], v[kVec];
            unpack<kP16>(p, rp);
            unpack<kG16>(g, rg);
            uint2 cm = make_uint2(rm[0], rm[1]), cv = make_uint2(rv[0], rv[1]);
            if constexpr (k8) {
                decode<3>(m, cm, em);
                decode<2>(v, cv, ev);
            } else {
                unpack<false>(m, rm);
                unpack<false>(v, rv);
            }
            uint32_t noise[kVec] = {};
            if (kNoise) {
                // the place's bits are the chunk's, the thread's and i's; mix's first step moves none of i's
                uint32_t x = noise_base ^ i0;
                x ^= x >> 16;
#pragma unroll
                for (int i = 0; i < kVec; ++i) noise[i] = mix_rest(x ^ i);
            }
            // products two an instruction, sums one by one: a two-lane sum behind two-lane products would be made one operation with one
            // rounding, and the definition has two
#pragma unroll
            for (int i = 0; i < kVec; i += 2) {
                const uint64_t gi = mul2(f32x2(g[i], g[i + 1]), gs2);
                float a0, a1, g0, g1;
                f32x2_split(mul2(f32x2(m[i], m[i + 1]), b1), a0, a1);
                f32x2_split(mul2(gi, c1), g0, g1);
                m[i] = __fadd_rn(a0, g0), m[i + 1] = __fadd_rn(a1, g1);
                f32x2_split(mul2(f32x2(v[i], v[i + 1]), b2), a0, a1);
                f32x2_split(mul2(mul2(gi, gi), c2), g0, g1);
                v[i] = __fadd_rn(a0, g0), v[i + 1] = __fadd_rn(a1, g1);
            }
            if (h.tiny_eps) {                  // squares below FP32's normal range count
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    float r;
                    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v[i]));
                    p[i] = fmaf(p[i], keep, -__fdividef(m[i] * size, fmaf(r, root, h.eps)));
                }
            } else {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    float r, q;
                    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v[i]));
                    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q) : "f"(fmaf(r, root, h.eps)));
                    p[i] = fmaf(p[i], keep, -(m[i] * size) * q);
                }
            }
            // is a value not finite?  Then v is not (m is only with it), or p is not
            uint32_t largest = 0;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                if (k8) largest = max(largest, __float_as_uint(v[i]));         // a square's bits, or a NaN's of either sign
                if (kP16) largest = max(largest, __float_as_uint(p[i]) & 0x7FFFFFFFu);
            }
            const bool odd = kOdd && __any_sync(0xFFFFFFFFu, largest >= 0x7F800000u);
            uint32_t packed_p[kVec / 2];
            if (kP16 && kChance) {
                uint32_t b[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) b[i] = __float_as_uint(p[i]) + (noise[i] * 0x9E3779B1u >> 16);
                if (odd) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i)
                        if (!finite_bits(__float_as_uint(p[i]))) b[i] = __float_as_uint(p[i]) | (__float_as_uint(p[i]) << 9 ? 0x400000u : 0u);
                }
#pragma unroll
                for (int i = 0; i < kVec; i += 2) packed_p[i / 2] = __byte_perm(b[i], b[i + 1], 0x7632);
            } else {
#pragma unroll
                for (int i = 0; i < kVec; i += 2) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(packed_p[i / 2]) : "f"(p[i + 1]), "f"(p[i]));
            }
            if constexpr (k8) {
                if (!kWhole && left < kVec) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i)
                        if (i >= left) m[i] = v[i] = 0.0f;        // behind the end: nothing that counts for the block
                }
                cm = encode<3, kChance>(m, em, noise, odd);
                cv = encode<2, kChance>(v, ev, noise, odd);
                if ((kWhole || left > 0) && (threadIdx.x & 3) == 0) ms0[i0 >> 5] = static_cast<uint8_t>(em), vs0[i0 >> 5] = static_cast<uint8_t>(ev);
            }
            if (kWhole || left >= kVec) {
                const uint4 packed = make_uint4(packed_p[0], packed_p[1], packed_p[2], packed_p[3]);
                if constexpr (kP16) *reinterpret_cast<uint4 *>(p0 + i0) = packed;
                else store(p0 + i0, p, wide);
                if (copy0 != nullptr) *reinterpret_cast<uint4 *>(copy0 + i0) = packed;
                if constexpr (k8) {
                    *reinterpret_cast<uint2 *>(m0 + i0) = cm;
                    *reinterpret_cast<uint2 *>(v0 + i0) = cv;
                } else {
                    store(m0 + i0, m, wide);
                    store(v0 + i0, v, wide);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    if (i >= left) continue;
                    const uint16_t short_p = static_cast<uint16_t>(packed_p[i / 2] >> (16 * (i & 1)));
                    if constexpr (kP16) p0[i0 + i] = short_p;
                    else p0[i0 + i] = p[i];
                    if (copy0 != nullptr) copy0[i0 + i] = short_p;
                    if constexpr (k8) {
                        m0[i0 + i] = static_cast<uint8_t>((i < 4 ? cm.x : cm.y) >> (8 * (i & 3)));
                        v0[i0 + i] = static_cast<uint8_t>((i < 4 ? cv.x : cv.y) >> (8 * (i & 3)));
                    } else {
                        m0[i0 + i] = m[i];
                        v0[i0 + i] = v[i];
                    }
                }
            }
        };
#pragma unroll 1
        for (int from = 0; from < here; from += kStep) {
            if (from + kStep <= here) step(std::true_type{}, from + threadIdx.x * kVec);
            else step(std::false_type{}, from + threadIdx.x * kVec);
        }
    }
}

template <int kN, bool kP16, bool kG16, bool k8, bool kChance>
sol_status_t launch_table(const Tensor *tensors, Hyper h, cudaStream_t stream, const DeviceInfo *dev) {
    static std::atomic<int> known[64];     // by device: blocks per SM
    int resident = known[dev->device].load(std::memory_order_relaxed);
    if (resident == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, step_kernel<kN, kP16, kG16, k8, kChance>, kThreads, 0) != cudaSuccess) {
            cudaGetLastError();
            return SOL_ERR_CUDA;
        }
        known[dev->device].store(resident, std::memory_order_relaxed);
    }
    const int64_t most = static_cast<int64_t>(resident) * dev->sm_count;
    // chunks of four steps share the looking for the tensor and its addresses (71 M BF16 values 179 us, with one step 184); with FP32
    // parameters and 8-bit states one step is faster all the same (193 us, four 213), and where blocks would not get eight chunks each
    int64_t values = 0;
    for (int i = 0; i < h.count; ++i) values += tensors[i].n;
    h.steps = !(k8 && !kP16) && values >= 8 * most * kSteps * kStep ? kSteps : 1;
    Table<kN> table;
    uint64_t chunks = 0;
    for (int i = 0; i < h.count; ++i) {
        table.t[i] = tensors[i];
        table.first[i] = static_cast<uint32_t>(chunks);
        chunks += static_cast<uint64_t>(ceil_div(tensors[i].n, kStep * h.steps));
        if (chunks > 0xFFFF0000ull) return SOL_ERR_BAD_SHAPE;
    }
    for (int i = h.count; i <= kN; ++i) table.first[i] = static_cast<uint32_t>(chunks);
    for (int i = h.count; i < kN; ++i) table.t[i] = Tensor{};
    h.chunks = static_cast<uint32_t>(chunks);
    const int64_t grid = static_cast<int64_t>(chunks) < most ? static_cast<int64_t>(chunks) : most;
    step_kernel<kN, kP16, kG16, k8, kChance><<<static_cast<unsigned>(grid < 1 ? 1 : grid), kThreads, 0, stream>>>(table, h);
    return launch_status();
}

template <bool kP16, bool kG16, bool k8, bool kChance>
sol_status_t launch_all(const Tensor *tensors, int64_t count, Hyper h, cudaStream_t stream, const DeviceInfo *dev) {
    int64_t first = 0;
    do {
        h.first_tensor = static_cast<uint32_t>(first);
        h.count = static_cast<int>(count - first < kTable ? count - first : kTable);
        h.advance = first + h.count == count;
        const sol_status_t st = h.count <= kSmallTable ? launch_table<kSmallTable, kP16, kG16, k8, kChance>(tensors + first, h, stream, dev)
                                                       : launch_table<kTable, kP16, kG16, k8, kChance>(tensors + first, h, stream, dev);
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
    h.tiny_eps = o.eps < 1e-9;               // a root below 2^-63 (times its bias correction) is then more than eps' last place
    h.lr_scale = o.lr_scale, h.grad_scale = o.grad_scale;
    h.state = reinterpret_cast<long long *>(state);
    h.seed = o.seed;
    auto all = [&](auto p16, auto g16, auto e8, auto chance) {
        // rounding by chance is for what is held in fewer bits
        constexpr bool kChance = decltype(chance)::value && (decltype(p16)::value || decltype(e8)::value);
        return launch_all<decltype(p16)::value, decltype(g16)::value, decltype(e8)::value, kChance>(tensors, count, h, stream, dev);
    };
    auto pick = [](bool v, auto next) { return v ? next(std::true_type{}) : next(std::false_type{}); };
    return pick(o.param_bf16 != 0, [&](auto p16) {
        return pick(o.grad_bf16 != 0, [&](auto g16) {
            return pick(o.state_bits == 8, [&](auto e8) { return pick(o.stochastic != 0, [&](auto chance) { return all(p16, g16, e8, chance); }); });
        });
    });
}

}  // namespace adamw
}  // namespace sol
