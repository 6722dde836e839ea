// C-ABI entry points: argument validation, size queries, device checks, TMA descriptor
// encoding.  Every compute step runs in the kernels of quantize.cu and gemm.cu.
#include "sol_internal.h"
#include "gemm_common.cuh"

#include <cmath>
#include <cstddef>
#include <mutex>

namespace sol {

__device__ DeviceStatusBlock g_status_block = {0u, 0u, kDefaultWaitLimitCycles};

namespace {

std::mutex g_mutex;
DeviceInfo g_devices[64];
uint32_t *g_status_ptr[64] = {};

using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                   const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                   CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                   CUtensorMapFloatOOBfill);
EncodeTiledFn g_encode = nullptr;

EncodeTiledFn encode_fn() {
    std::lock_guard<std::mutex> lock(g_mutex);
    if (g_encode == nullptr) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) == cudaSuccess &&
            qres == cudaDriverEntryPointSuccess)
            g_encode = reinterpret_cast<EncodeTiledFn>(fn);
    }
    return g_encode;
}

}  // namespace

const DeviceInfo *current_device_info() {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    std::lock_guard<std::mutex> lock(g_mutex);
    DeviceInfo &d = g_devices[dev];
    if (!d.ok) {
        cudaDeviceProp prop;
        if (cudaGetDeviceProperties(&prop, dev) != cudaSuccess) return nullptr;
        d.device = dev;
        d.sm_count = prop.multiProcessorCount;
        d.cc_major = prop.major;
        d.cc_minor = prop.minor;
        void *sym = nullptr;
        if (cudaGetSymbolAddress(&sym, g_status_block) != cudaSuccess) return nullptr;
        g_status_ptr[dev] = static_cast<uint32_t *>(sym);
        d.ok = true;
    }
    return &d;
}

sol_status_t check_arch(const DeviceInfo **info_out) {
    const DeviceInfo *d = current_device_info();
    if (d == nullptr) {
        cudaGetLastError();
        return SOL_ERR_CUDA;
    }
    if (d->cc_major != 10) return SOL_ERR_UNSUPPORTED_ARCH;
    *info_out = d;
    return SOL_OK;
}

uint32_t *device_status_word() {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    return g_status_ptr[dev];
}

bool make_tmap_2d(CUtensorMap *out, CUtensorMapDataType dtype, uint32_t elem_bytes, const void *base,
                  uint64_t inner, uint64_t outer, uint64_t pitch_bytes, uint32_t box_inner, uint32_t box_outer,
                  CUtensorMapSwizzle swizzle) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    (void)elem_bytes;
    cuuint64_t dims[2] = {inner, outer};
    cuuint64_t strides[1] = {pitch_bytes};
    cuuint32_t box[2] = {box_inner, box_outer};
    cuuint32_t estr[2] = {1, 1};
    return fn(out, dtype, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_tmap_3d_bf16(CUtensorMap *out, const void *base, uint64_t d0, uint64_t d1, uint64_t d2, uint64_t pitch1_bytes,
                       uint64_t pitch2_bytes, uint32_t box0, uint32_t box1) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    cuuint64_t dims[3] = {d0, d1, d2};
    cuuint64_t strides[2] = {pitch1_bytes, pitch2_bytes};
    cuuint32_t box[3] = {box0, box1, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_tmap_sf(CUtensorMap *out, const void *base, uint64_t chunks_k, uint64_t row_chunks,
                  uint32_t box_row_chunks, uint32_t box_k_chunks) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    cuuint64_t dims[3] = {128, chunks_k, row_chunks};
    cuuint64_t strides[2] = {512, 512 * chunks_k};
    cuuint32_t box[3] = {128, box_k_chunks, box_row_chunks};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void *>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

bool shape_ok(int64_t rows, int64_t K) {
    // the streaming kernels index their tiles (128 rows x 256 elements) and 32 KB pieces with a one-dimensional grid
    return rows > 0 && K > 0 && K % 32 == 0 && rows <= (1LL << 30) && K <= (1LL << 24) &&
           ceil_div(rows, 128) * ceil_div(K, 256) <= 0x7FFFFFFFLL && ceil_div(rows * (K / 8), 2048) <= 0x7FFFFFFFLL;
}

// Host description of the rotary positions -> the kernels' form.  Device pointers are not followed.
sol_status_t make_turn(const sol_rotary_t *r, int64_t head_dim, rotary::Turn *t) {
    *t = rotary::Turn{};
    if (r == nullptr) return SOL_OK;
    if (r->positions == nullptr || r->freqs == nullptr) return SOL_ERR_NULL_POINTER;
    if (r->axes < 1 || r->axes > 4 || r->position_rows < 1 || r->position_rows > 0x7FFFFFFFLL || !std::isfinite(r->scale))
        return SOL_ERR_BAD_SHAPE;
    if (r->layout != SOL_ROTARY_INTERLEAVED && r->layout != SOL_ROTARY_HALF) return SOL_ERR_BAD_LAYOUT;
    int64_t rot = 0;
    for (int i = 0; i < 4; ++i) {
        if (i < r->axes) {
            if (r->axis_dims[i] <= 0 || r->axis_dims[i] % 2 != 0 || r->axis_dims[i] > head_dim) return SOL_ERR_BAD_SHAPE;
            rot += r->axis_dims[i];
        }
        if (i < 3) t->axis_end[i] = i < r->axes - 1 ? static_cast<int>(rot / 2) : 0x7FFFFFFF;
    }
    if (rot % 8 != 0 || rot > head_dim) return SOL_ERR_BAD_SHAPE;
    if ((reinterpret_cast<uintptr_t>(r->positions) & 7u) || (reinterpret_cast<uintptr_t>(r->freqs) & 7u)) return SOL_ERR_ALIGNMENT;
    t->positions = r->positions;
    t->freqs = r->freqs;
    t->position_rows = static_cast<uint32_t>(r->position_rows);
    t->axes = static_cast<int>(r->axes);
    t->rot = static_cast<int>(rot);
    t->scale = r->scale;
    return SOL_OK;
}

bool aligned8(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

size_t align256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

}  // namespace
}  // namespace sol

using namespace sol;

extern "C" {

const char *sol_status_string(sol_status_t status) {
    switch (status) {
        case SOL_OK: return "SOL_OK";
        case SOL_ERR_NULL_POINTER: return "SOL_ERR_NULL_POINTER";
        case SOL_ERR_BAD_SHAPE: return "SOL_ERR_BAD_SHAPE";
        case SOL_ERR_ALIGNMENT: return "SOL_ERR_ALIGNMENT";
        case SOL_ERR_WORKSPACE_TOO_SMALL: return "SOL_ERR_WORKSPACE_TOO_SMALL";
        case SOL_ERR_UNSUPPORTED_ARCH: return "SOL_ERR_UNSUPPORTED_ARCH";
        case SOL_ERR_CUDA: return "SOL_ERR_CUDA";
        case SOL_ERR_TIMEOUT: return "SOL_ERR_TIMEOUT";
        case SOL_ERR_BAD_LAYOUT: return "SOL_ERR_BAD_LAYOUT";
    }
    return "SOL_ERR_UNKNOWN";
}

size_t sol_nvfp4_data_bytes(int64_t rows, int64_t K) {
    if (!shape_ok(rows, K)) return 0;
    return static_cast<size_t>(rows) * static_cast<size_t>(K / 2);
}

size_t sol_nvfp4_scale_bytes(int64_t rows, int64_t K, sol_sf_layout_t layout) {
    if (!shape_ok(rows, K)) return 0;
    if (layout == SOL_SF_ROW_MAJOR) return static_cast<size_t>(rows) * static_cast<size_t>(K / 16);
    if (layout == SOL_SF_SWIZZLED_128x4)
        return static_cast<size_t>(ceil_div(rows, 128)) * static_cast<size_t>(ceil_div(K, 64)) * 512;
    return 0;
}

size_t sol_nvfp4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (!shape_ok(M, K) || N <= 0) return 0;
    return align256(sol_nvfp4_data_bytes(M, K)) + align256(sol_nvfp4_scale_bytes(M, K, SOL_SF_SWIZZLED_128x4)) + 256;
}

sol_status_t sol_amax_bf16(const void *x, int64_t rows, int64_t K, int64_t ld, float *tensor_scale_out,
                           void *stream) {
    if (x == nullptr || tensor_scale_out == nullptr) return SOL_ERR_NULL_POINTER;
    if (!shape_ok(rows, K) || ld < K) return SOL_ERR_BAD_SHAPE;
    if (!aligned16(x) || ld % 8 != 0 || (reinterpret_cast<uintptr_t>(tensor_scale_out) & 3u)) return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_amax(x, rows, K, ld, tensor_scale_out, static_cast<cudaStream_t>(stream), dev);
}

sol_status_t nvfp4_quantize(const void *x_bf16, int64_t M, int64_t K, int64_t ldx, const float *tensor_scale,
                            void *q_out, void *sf_out, sol_sf_layout_t layout, void *stream) {
    if (x_bf16 == nullptr || tensor_scale == nullptr || q_out == nullptr || sf_out == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!shape_ok(M, K) || ldx < K) return SOL_ERR_BAD_SHAPE;
    if (layout != SOL_SF_ROW_MAJOR && layout != SOL_SF_SWIZZLED_128x4) return SOL_ERR_BAD_LAYOUT;
    if (!aligned16(x_bf16) || !aligned16(q_out) || !aligned16(sf_out) || ldx % 8 != 0 ||
        (reinterpret_cast<uintptr_t>(tensor_scale) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_quantize(x_bf16, M, K, ldx, tensor_scale, q_out, sf_out, layout, static_cast<cudaStream_t>(stream));
}

sol_status_t nvfp4_quantize_weight(const void *w_bf16, int64_t N, int64_t K, int64_t ldw, void *q_out,
                                   void *sf_out, float *tensor_scale_out, sol_sf_layout_t layout, void *stream) {
    if (w_bf16 == nullptr || tensor_scale_out == nullptr || q_out == nullptr || sf_out == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!shape_ok(N, K) || ldw < K) return SOL_ERR_BAD_SHAPE;
    if (layout != SOL_SF_ROW_MAJOR && layout != SOL_SF_SWIZZLED_128x4) return SOL_ERR_BAD_LAYOUT;
    if (!aligned16(w_bf16) || !aligned16(q_out) || !aligned16(sf_out) || ldw % 8 != 0 ||
        (reinterpret_cast<uintptr_t>(tensor_scale_out) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    st = launch_amax(w_bf16, N, K, ldw, tensor_scale_out, s, dev);
    if (st != SOL_OK) return st;
    return launch_quantize(w_bf16, N, K, ldw, tensor_scale_out, q_out, sf_out, layout, s);
}

static sol_status_t check_requantize_lora(const void *w, const void *a, const void *b, const void *merged,
                                          const void *q, const void *sf, const float *ts, int64_t ldw, int64_t lda,
                                          int64_t ldb, int64_t N, int64_t K, int64_t r, sol_sf_layout_t layout) {
    if (w == nullptr || a == nullptr || b == nullptr || merged == nullptr || q == nullptr || sf == nullptr ||
        ts == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!shape_ok(N, K) || ldw < K || lda < K || r < 1 || r > lora_max_rank() || ldb < r || N > 65535LL * 64)
        return SOL_ERR_BAD_SHAPE;
    if (layout != SOL_SF_ROW_MAJOR && layout != SOL_SF_SWIZZLED_128x4) return SOL_ERR_BAD_LAYOUT;
    if (!aligned16(w) || !aligned16(a) || !aligned16(merged) || !aligned16(q) || !aligned16(sf) || ldw % 8 != 0 ||
        lda % 8 != 0 || (reinterpret_cast<uintptr_t>(b) & 1u) || (reinterpret_cast<uintptr_t>(ts) & 3u))
        return SOL_ERR_ALIGNMENT;
    return SOL_OK;
}

sol_status_t nvfp4_requantize_lora(const void *w_bf16, int64_t ldw, const void *lora_a, int64_t lda,
                                   const void *lora_b, int64_t ldb, int64_t N, int64_t K, int64_t r, float scaling,
                                   void *merged_bf16, void *q_out, void *sf_out, float *tensor_scale_out,
                                   sol_sf_layout_t layout, void *stream) {
    sol_status_t st = check_requantize_lora(w_bf16, lora_a, lora_b, merged_bf16, q_out, sf_out, tensor_scale_out, ldw,
                                            lda, ldb, N, K, r, layout);
    if (st != SOL_OK) return st;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    MergeGroup mg = {};
    mg.w[0] = static_cast<const uint16_t *>(w_bf16);
    mg.a[0] = static_cast<const uint16_t *>(lora_a);
    mg.b[0] = static_cast<const uint16_t *>(lora_b);
    mg.out[0] = static_cast<uint16_t *>(merged_bf16);
    mg.scale_words[0] = tensor_scale_out;
    st = launch_lora_merge(mg, 1, ldw, lda, ldb, N, K, r, scaling, s);
    if (st != SOL_OK) return st;
    return launch_quantize_from_amax(merged_bf16, N, K, K, tensor_scale_out, q_out, sf_out, layout, s);
}

sol_status_t nvfp4_requantize_lora_batch(int64_t count, const void *const *w_list, const void *const *a_list,
                                         const void *const *b_list, void *const *q_list, void *const *sf_list,
                                         float *const *ts_list, int64_t N, int64_t K, int64_t r, float scaling,
                                         void *merged_bf16, int64_t merged_matrices, sol_sf_layout_t layout,
                                         void *stream) {
    if (count < 0 || merged_matrices < 1) return SOL_ERR_BAD_SHAPE;
    if (count == 0) return SOL_OK;
    if (w_list == nullptr || a_list == nullptr || b_list == nullptr || q_list == nullptr || sf_list == nullptr ||
        ts_list == nullptr)
        return SOL_ERR_NULL_POINTER;
    // validate every matrix before the first launch: an error status means nothing was launched
    for (int64_t i = 0; i < count; ++i) {
        const sol_status_t st = check_requantize_lora(w_list[i], a_list[i], b_list[i], merged_bf16, q_list[i],
                                                      sf_list[i], ts_list[i], K, K, r, N, K, r, layout);
        if (st != SOL_OK) return st;
    }
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t group = merged_matrices < kMaxGroup ? merged_matrices : kMaxGroup;
    for (int64_t i0 = 0; i0 < count; i0 += group) {
        const int n = static_cast<int>(count - i0 < group ? count - i0 : group);
        MergeGroup mg = {};
        QuantGroup qg = {};
        for (int i = 0; i < n; ++i) {
            uint16_t *merged = static_cast<uint16_t *>(merged_bf16) + static_cast<int64_t>(i) * N * K;
            mg.w[i] = static_cast<const uint16_t *>(w_list[i0 + i]);
            mg.a[i] = static_cast<const uint16_t *>(a_list[i0 + i]);
            mg.b[i] = static_cast<const uint16_t *>(b_list[i0 + i]);
            mg.out[i] = merged;
            mg.scale_words[i] = ts_list[i0 + i];
            qg.x[i] = merged;
            qg.scale_words[i] = ts_list[i0 + i];
            qg.q[i] = static_cast<uint8_t *>(q_list[i0 + i]);
            qg.sf[i] = static_cast<uint8_t *>(sf_list[i0 + i]);
        }
        st = launch_lora_merge(mg, n, K, K, r, N, K, r, scaling, s);
        if (st != SOL_OK) return st;
        st = launch_quantize_group(qg, n, N, K, layout, s);
        if (st != SOL_OK) return st;
    }
    return SOL_OK;
}

static sol_status_t check_linear_common(const void *bias, const void *y, int64_t M, int64_t N, int64_t K,
                                        int64_t ldy) {
    if (!shape_ok(M, K) || N <= 0 || N % 8 != 0 || N > (1LL << 24) || ldy < N) return SOL_ERR_BAD_SHAPE;
    if (!aligned16(y) || ldy % 8 != 0 || (bias != nullptr && !aligned16(bias))) return SOL_ERR_ALIGNMENT;
    return SOL_OK;
}

sol_status_t nvfp4_linear(const void *xq, const void *xsf, const float *x_tscale, const void *wq, const void *wsf,
                          const float *w_tscale, const void *bias_bf16, void *y_bf16, int64_t M, int64_t N,
                          int64_t K, int64_t ldy, void *stream) {
    if (xq == nullptr || xsf == nullptr || x_tscale == nullptr || wq == nullptr || wsf == nullptr ||
        w_tscale == nullptr || y_bf16 == nullptr)
        return SOL_ERR_NULL_POINTER;
    sol_status_t st = check_linear_common(bias_bf16, y_bf16, M, N, K, ldy);
    if (st != SOL_OK) return st;
    if (!aligned16(xq) || !aligned16(xsf) || !aligned16(wq) || !aligned16(wsf) ||
        (reinterpret_cast<uintptr_t>(x_tscale) & 3u) || (reinterpret_cast<uintptr_t>(w_tscale) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_gemm_nvfp4(xq, xsf, x_tscale, wq, wsf, w_tscale, bias_bf16, y_bf16, M, N, K, ldy,
                             static_cast<cudaStream_t>(stream), dev);
}

sol_status_t bf16_linear(const void *x_bf16, const void *w_bf16, const void *bias_bf16, void *y_bf16, int64_t M,
                         int64_t N, int64_t K, int64_t ldx, int64_t ldw, int64_t ldy, void *stream) {
    if (x_bf16 == nullptr || w_bf16 == nullptr || y_bf16 == nullptr) return SOL_ERR_NULL_POINTER;
    sol_status_t st = check_linear_common(bias_bf16, y_bf16, M, N, K, ldy);
    if (st != SOL_OK) return st;
    if (ldx < K || ldw < K) return SOL_ERR_BAD_SHAPE;
    if (!aligned16(x_bf16) || !aligned16(w_bf16) || ldx % 8 != 0 || ldw % 8 != 0) return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_gemm_bf16(x_bf16, w_bf16, bias_bf16, y_bf16, M, N, K, ldx, ldw, ldy,
                            static_cast<cudaStream_t>(stream), dev);
}

sol_status_t nvfp4_linear_quantized_out(const void *xq, const void *xsf, const float *x_tscale, const void *wq,
                                        const void *wsf, const float *w_tscale, const void *bias_bf16,
                                        sol_activation_t activation, const float *out_tscale, void *hq_out,
                                        void *hsf_out, float *amax_out, int64_t M, int64_t N, int64_t K, void *stream) {
    if (xq == nullptr || xsf == nullptr || x_tscale == nullptr || wq == nullptr || wsf == nullptr ||
        w_tscale == nullptr || out_tscale == nullptr || hq_out == nullptr || hsf_out == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!shape_ok(M, K) || N <= 0 || N % 64 != 0 || N > (1LL << 24)) return SOL_ERR_BAD_SHAPE;
    if (activation != SOL_ACT_NONE && activation != SOL_ACT_GELU_TANH) return SOL_ERR_BAD_LAYOUT;
    if (!aligned16(xq) || !aligned16(xsf) || !aligned16(wq) || !aligned16(wsf) || !aligned16(hq_out) ||
        !aligned16(hsf_out) || (bias_bf16 != nullptr && !aligned16(bias_bf16)) ||
        (reinterpret_cast<uintptr_t>(x_tscale) & 3u) || (reinterpret_cast<uintptr_t>(w_tscale) & 3u) ||
        (reinterpret_cast<uintptr_t>(out_tscale) & 3u) || (reinterpret_cast<uintptr_t>(amax_out) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return gemm::launch_pair256_nvfp4_quant_out(xq, xsf, x_tscale, wq, wsf, w_tscale, bias_bf16,
                                                activation == SOL_ACT_GELU_TANH ? 1 : 0, out_tscale, hq_out, hsf_out,
                                                reinterpret_cast<uint32_t *>(amax_out), M, N, K,
                                                static_cast<cudaStream_t>(stream), dev);
}

size_t sol_mxfp4_scale_bytes(int64_t rows, int64_t K, sol_sf_layout_t layout) {
    if (!shape_ok(rows, K)) return 0;
    if (layout == SOL_SF_ROW_MAJOR) return static_cast<size_t>(rows) * static_cast<size_t>(K / 32);
    if (layout == SOL_SF_SWIZZLED_128x4)
        return static_cast<size_t>(ceil_div(rows, 128)) * static_cast<size_t>(ceil_div(K, 128)) * 512;
    return 0;
}

sol_status_t mxfp4_quantize(const void *x_bf16, int64_t rows, int64_t K, int64_t ldx, void *q_out, void *sf_out,
                            sol_sf_layout_t layout, void *stream) {
    if (x_bf16 == nullptr || q_out == nullptr || sf_out == nullptr) return SOL_ERR_NULL_POINTER;
    if (!shape_ok(rows, K) || ldx < K) return SOL_ERR_BAD_SHAPE;
    if (layout != SOL_SF_ROW_MAJOR && layout != SOL_SF_SWIZZLED_128x4) return SOL_ERR_BAD_LAYOUT;
    if (!aligned16(x_bf16) || !aligned16(q_out) || !aligned16(sf_out) || ldx % 8 != 0) return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_mxfp4_quantize(x_bf16, rows, K, ldx, q_out, sf_out, layout, static_cast<cudaStream_t>(stream));
}

sol_status_t mxfp4_linear(const void *xq, const void *xsf, const void *wq, const void *wsf, const void *bias_bf16,
                          void *y_bf16, int64_t M, int64_t N, int64_t K, int64_t ldy, void *stream) {
    if (xq == nullptr || xsf == nullptr || wq == nullptr || wsf == nullptr || y_bf16 == nullptr)
        return SOL_ERR_NULL_POINTER;
    sol_status_t st = check_linear_common(bias_bf16, y_bf16, M, N, K, ldy);
    if (st != SOL_OK) return st;
    if (!aligned16(xq) || !aligned16(xsf) || !aligned16(wq) || !aligned16(wsf)) return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return gemm::launch_pair256_mxfp4(xq, xsf, wq, wsf, bias_bf16, y_bf16, M, N, K, ldy,
                                      static_cast<cudaStream_t>(stream), dev);
}

sol_status_t mxfp4_linear_quantized_out(const void *xq, const void *xsf, const void *wq, const void *wsf,
                                        const void *bias_bf16, sol_activation_t activation, void *hq_out, void *hsf_out,
                                        float *amax_out, int64_t M, int64_t N, int64_t K, void *stream) {
    if (xq == nullptr || xsf == nullptr || wq == nullptr || wsf == nullptr || hq_out == nullptr || hsf_out == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!shape_ok(M, K) || N <= 0 || N % 128 != 0 || N > (1LL << 24)) return SOL_ERR_BAD_SHAPE;
    if (activation != SOL_ACT_NONE && activation != SOL_ACT_GELU_TANH) return SOL_ERR_BAD_LAYOUT;
    if (!aligned16(xq) || !aligned16(xsf) || !aligned16(wq) || !aligned16(wsf) || !aligned16(hq_out) ||
        !aligned16(hsf_out) || (bias_bf16 != nullptr && !aligned16(bias_bf16)) ||
        (reinterpret_cast<uintptr_t>(amax_out) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return gemm::launch_pair256_mxfp4_quant_out(xq, xsf, wq, wsf, bias_bf16, activation == SOL_ACT_GELU_TANH ? 1 : 0,
                                                hq_out, hsf_out, reinterpret_cast<uint32_t *>(amax_out), M, N, K,
                                                static_cast<cudaStream_t>(stream), dev);
}

sol_status_t mxfp4_linear_split_out(const void *xq, const void *xsf, const void *wq, const void *wsf,
                                    const void *bias_bf16, void *y_bf16, int64_t ldy, int64_t n_split,
                                    sol_activation_t activation, void *hq_dest, void *hsf_dest, int64_t dest_K,
                                    int64_t dest_col0, float *amax_out, int64_t M, int64_t N, int64_t K, void *stream) {
    if (xq == nullptr || xsf == nullptr || wq == nullptr || wsf == nullptr || y_bf16 == nullptr || hq_dest == nullptr ||
        hsf_dest == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!shape_ok(M, K) || N <= 0 || N > (1LL << 24) || n_split <= 0 || n_split >= N || n_split % 256 != 0 ||
        (N - n_split) % 128 != 0 || ldy < n_split || dest_K <= 0 || dest_K % 128 != 0 || dest_col0 < 0 ||
        dest_col0 % 128 != 0 || dest_col0 + (N - n_split) > dest_K)
        return SOL_ERR_BAD_SHAPE;
    if (activation != SOL_ACT_NONE && activation != SOL_ACT_GELU_TANH) return SOL_ERR_BAD_LAYOUT;
    if (!aligned16(xq) || !aligned16(xsf) || !aligned16(wq) || !aligned16(wsf) || !aligned16(y_bf16) ||
        !aligned16(hq_dest) || !aligned16(hsf_dest) || ldy % 8 != 0 || (bias_bf16 != nullptr && !aligned16(bias_bf16)) ||
        (reinterpret_cast<uintptr_t>(amax_out) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return gemm::launch_pair256_mxfp4_split_out(xq, xsf, wq, wsf, bias_bf16, y_bf16, ldy, n_split,
                                                activation == SOL_ACT_GELU_TANH ? 1 : 0, hq_dest, hsf_dest, dest_K,
                                                dest_col0, reinterpret_cast<uint32_t *>(amax_out), M, N, K,
                                                static_cast<cudaStream_t>(stream), dev);
}

sol_status_t mxfp4_quantize_into(const void *x_bf16, int64_t M, int64_t K, int64_t ldx, void *q_dest, void *sf_dest,
                                 int64_t dest_K, int64_t dest_col0, void *stream) {
    if (x_bf16 == nullptr || q_dest == nullptr || sf_dest == nullptr) return SOL_ERR_NULL_POINTER;
    if (!shape_ok(M, K) || ldx < K || K % 128 != 0 || dest_K <= 0 || dest_K % 128 != 0 || dest_col0 < 0 ||
        dest_col0 % 128 != 0 || dest_col0 + K > dest_K)
        return SOL_ERR_BAD_SHAPE;
    if (!aligned16(x_bf16) || !aligned16(q_dest) || !aligned16(sf_dest) || ldx % 8 != 0) return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_mxfp4_quantize_into(x_bf16, M, K, ldx, q_dest, sf_dest, dest_K, dest_col0,
                                      static_cast<cudaStream_t>(stream));
}

sol_status_t solrl_select_contrastive(const float *rewards, const uint64_t *seeds, int64_t P, int64_t N, int64_t K,
                                      int32_t *idx_out, uint64_t *seeds_out, float *advantages_out, void *stream) {
    if (rewards == nullptr || idx_out == nullptr || (seeds_out != nullptr && seeds == nullptr)) return SOL_ERR_NULL_POINTER;
    if (P <= 0 || P > 0x7FFFFFFF || N <= 0 || N > selection_max_candidates() || K <= 0 || K % 2 != 0 || K > N)
        return SOL_ERR_BAD_SHAPE;
    if ((reinterpret_cast<uintptr_t>(rewards) & 3u) || (reinterpret_cast<uintptr_t>(idx_out) & 3u) ||
        (reinterpret_cast<uintptr_t>(seeds) & 7u) || (reinterpret_cast<uintptr_t>(seeds_out) & 7u) ||
        (reinterpret_cast<uintptr_t>(advantages_out) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_select_contrastive(rewards, seeds, P, N, K, idx_out, seeds_out, advantages_out,
                                     static_cast<cudaStream_t>(stream));
}

sol_status_t solrl_rank_consistency(const float *rewards_ref, const float *rewards_proxy, int64_t P, int64_t N,
                                    int64_t k, int64_t *counts_out, float *metrics_out, void *stream) {
    if (rewards_ref == nullptr || rewards_proxy == nullptr || counts_out == nullptr) return SOL_ERR_NULL_POINTER;
    if (P <= 0 || P > 0x7FFFFFFF || N < 2 || 2 * N > selection_max_candidates() || k <= 0 || k > N)
        return SOL_ERR_BAD_SHAPE;
    if ((reinterpret_cast<uintptr_t>(rewards_ref) & 3u) || (reinterpret_cast<uintptr_t>(rewards_proxy) & 3u) ||
        (reinterpret_cast<uintptr_t>(counts_out) & 7u) || (reinterpret_cast<uintptr_t>(metrics_out) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_rank_consistency(rewards_ref, rewards_proxy, P, N, k, counts_out, metrics_out,
                                   static_cast<cudaStream_t>(stream));
}

sol_status_t nvfp4_linear_split_out(const void *xq, const void *xsf, const float *x_tscale, const void *wq,
                                    const void *wsf, const float *w_tscale, const void *bias_bf16, void *y_bf16,
                                    int64_t ldy, int64_t n_split, sol_activation_t activation, const float *out_tscale,
                                    void *hq_dest, void *hsf_dest, int64_t dest_K, int64_t dest_col0, float *amax_out,
                                    int64_t M, int64_t N, int64_t K, void *stream) {
    if (xq == nullptr || xsf == nullptr || x_tscale == nullptr || wq == nullptr || wsf == nullptr ||
        w_tscale == nullptr || y_bf16 == nullptr || out_tscale == nullptr || hq_dest == nullptr || hsf_dest == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!shape_ok(M, K) || N <= 0 || N > (1LL << 24) || n_split <= 0 || n_split >= N || n_split % 256 != 0 ||
        (N - n_split) % 64 != 0 || ldy < n_split || dest_K <= 0 || dest_K % 64 != 0 || dest_col0 < 0 ||
        dest_col0 % 64 != 0 || dest_col0 + (N - n_split) > dest_K)
        return SOL_ERR_BAD_SHAPE;
    if (activation != SOL_ACT_NONE && activation != SOL_ACT_GELU_TANH) return SOL_ERR_BAD_LAYOUT;
    if (!aligned16(xq) || !aligned16(xsf) || !aligned16(wq) || !aligned16(wsf) || !aligned16(y_bf16) ||
        !aligned16(hq_dest) || !aligned16(hsf_dest) || ldy % 8 != 0 || (bias_bf16 != nullptr && !aligned16(bias_bf16)) ||
        (reinterpret_cast<uintptr_t>(x_tscale) & 3u) || (reinterpret_cast<uintptr_t>(w_tscale) & 3u) ||
        (reinterpret_cast<uintptr_t>(out_tscale) & 3u) || (reinterpret_cast<uintptr_t>(amax_out) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return gemm::launch_pair256_nvfp4_split_out(xq, xsf, x_tscale, wq, wsf, w_tscale, bias_bf16, y_bf16, ldy, n_split,
                                                activation == SOL_ACT_GELU_TANH ? 1 : 0, out_tscale, hq_dest, hsf_dest,
                                                dest_K, dest_col0, reinterpret_cast<uint32_t *>(amax_out), M, N, K,
                                                static_cast<cudaStream_t>(stream), dev);
}

sol_status_t nvfp4_quantize_into(const void *x_bf16, int64_t M, int64_t K, int64_t ldx, const float *tensor_scale,
                                 void *q_dest, void *sf_dest, int64_t dest_K, int64_t dest_col0, void *stream) {
    if (x_bf16 == nullptr || tensor_scale == nullptr || q_dest == nullptr || sf_dest == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!shape_ok(M, K) || ldx < K || K % 64 != 0 || dest_K <= 0 || dest_K % 64 != 0 || dest_col0 < 0 ||
        dest_col0 % 64 != 0 || dest_col0 + K > dest_K)
        return SOL_ERR_BAD_SHAPE;
    if (!aligned16(x_bf16) || !aligned16(q_dest) || !aligned16(sf_dest) || ldx % 8 != 0 ||
        (reinterpret_cast<uintptr_t>(tensor_scale) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_quantize_into(x_bf16, M, K, ldx, tensor_scale, q_dest, sf_dest, dest_K, dest_col0,
                                static_cast<cudaStream_t>(stream));
}

sol_status_t nvfp4_layernorm_quantize(const void *x_bf16, int64_t M, int64_t K, int64_t ldx, const void *scale_bf16,
                                      const void *shift_bf16, int64_t rows_per_sample, float eps,
                                      const float *tensor_scale, void *q_out, void *sf_out, float *amax_out,
                                      void *stream) {
    if (x_bf16 == nullptr || scale_bf16 == nullptr || shift_bf16 == nullptr || tensor_scale == nullptr ||
        q_out == nullptr || sf_out == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!shape_ok(M, K) || K % 64 != 0 || K > layernorm_max_k() || ldx < K || rows_per_sample <= 0 || !(eps >= 0.0f))
        return SOL_ERR_BAD_SHAPE;
    if (!aligned16(x_bf16) || !aligned16(scale_bf16) || !aligned16(shift_bf16) || !aligned16(q_out) ||
        !aligned16(sf_out) || ldx % 8 != 0 || (reinterpret_cast<uintptr_t>(tensor_scale) & 3u) ||
        (reinterpret_cast<uintptr_t>(amax_out) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_layernorm_quantize(x_bf16, M, K, ldx, scale_bf16, shift_bf16, rows_per_sample, eps, tensor_scale,
                                     q_out, sf_out, reinterpret_cast<uint32_t *>(amax_out),
                                     static_cast<cudaStream_t>(stream));
}

sol_status_t sol_attention_bf16(const void *q, const void *k, const void *v, void *out, int64_t batch, int64_t seq_q,
                                int64_t seq_kv, int64_t heads, int64_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                int64_t ld_out, void *stream) {
    if (q == nullptr || k == nullptr || v == nullptr || out == nullptr) return SOL_ERR_NULL_POINTER;
    if (head_dim != 64 && head_dim != 128) return SOL_ERR_BAD_SHAPE;
    const int64_t cols = heads * head_dim;
    if (batch <= 0 || seq_q <= 0 || seq_kv <= 0 || heads <= 0 || batch > 65535 || heads > 65535 ||
        seq_q > (1LL << 24) || seq_kv > (1LL << 24) || ld_q < cols || ld_k < cols || ld_v < cols || ld_out < cols)
        return SOL_ERR_BAD_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || ld_q % 8 != 0 || ld_k % 8 != 0 ||
        ld_v % 8 != 0 || ld_out % 8 != 0)
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    const attn::Stream b{q, k, v, out, seq_q, seq_kv, ld_q, ld_k, ld_v, ld_out};
    return attn::launch_attention(nullptr, b, batch, heads, head_dim, nullptr, static_cast<cudaStream_t>(stream));
}

sol_status_t sol_attention_nvfp4_out(const void *q, const void *k, const void *v, int64_t batch, int64_t seq_q,
                                     int64_t seq_kv, int64_t heads, int64_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                     const float *out_tscale, void *q_dest, void *sf_dest, int64_t dest_K,
                                     int64_t dest_col0, float *amax_out, void *stream) {
    if (q == nullptr || k == nullptr || v == nullptr || out_tscale == nullptr || q_dest == nullptr || sf_dest == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (head_dim != 64 && head_dim != 128) return SOL_ERR_BAD_SHAPE;
    const int64_t cols = heads * head_dim;
    if (batch <= 0 || seq_q <= 0 || seq_kv <= 0 || heads <= 0 || batch > 65535 || heads > 65535 ||
        seq_q > (1LL << 24) || seq_kv > (1LL << 24) || ld_q < cols || ld_k < cols || ld_v < cols || dest_K <= 0 ||
        dest_K % 64 != 0 || dest_col0 < 0 || dest_col0 % 64 != 0 || dest_col0 + cols > dest_K || dest_K > (1LL << 24) ||
        batch * seq_q > (1LL << 30))
        return SOL_ERR_BAD_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_dest) || !aligned16(sf_dest) || ld_q % 8 != 0 ||
        ld_k % 8 != 0 || ld_v % 8 != 0 || (reinterpret_cast<uintptr_t>(out_tscale) & 3u) ||
        (reinterpret_cast<uintptr_t>(amax_out) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    const attn::Stream b{q, k, v, nullptr, seq_q, seq_kv, ld_q, ld_k, ld_v, cols};
    const attn::QuantDest qd{q_dest, sf_dest, out_tscale, reinterpret_cast<uint32_t *>(amax_out), dest_K, dest_col0};
    return attn::launch_attention(nullptr, b, batch, heads, head_dim, &qd, static_cast<cudaStream_t>(stream));
}

sol_status_t sol_attention_bf16_joint(const sol_attention_stream_t *first, const sol_attention_stream_t *second,
                                      int64_t batch, int64_t heads, int64_t head_dim, void *stream) {
    if (first == nullptr || second == nullptr) return SOL_ERR_NULL_POINTER;
    if (head_dim != 64 && head_dim != 128) return SOL_ERR_BAD_SHAPE;
    const sol_attention_stream_t *both[2] = {first, second};
    const int64_t cols = heads * head_dim;
    if (batch <= 0 || heads <= 0 || batch > 65535 || heads > 65535) return SOL_ERR_BAD_SHAPE;
    for (const sol_attention_stream_t *s : both) {
        if (s->q == nullptr || s->k == nullptr || s->v == nullptr || s->out == nullptr) return SOL_ERR_NULL_POINTER;
        if (s->seq <= 0 || s->seq > (1LL << 24) || s->ld_q < cols || s->ld_k < cols || s->ld_v < cols || s->ld_out < cols)
            return SOL_ERR_BAD_SHAPE;
        if (!aligned16(s->q) || !aligned16(s->k) || !aligned16(s->v) || !aligned16(s->out) || s->ld_q % 8 != 0 ||
            s->ld_k % 8 != 0 || s->ld_v % 8 != 0 || s->ld_out % 8 != 0)
            return SOL_ERR_ALIGNMENT;
    }
    if (first->seq % 256 != 0) return SOL_ERR_BAD_SHAPE;  // the first stream must fill whole query-tile pairs
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    const attn::Stream a{first->q, first->k, first->v, first->out, first->seq, first->seq,
                         first->ld_q, first->ld_k, first->ld_v, first->ld_out};
    const attn::Stream b{second->q, second->k, second->v, second->out, second->seq, second->seq,
                         second->ld_q, second->ld_k, second->ld_v, second->ld_out};
    return attn::launch_attention(&a, b, batch, heads, head_dim, nullptr, static_cast<cudaStream_t>(stream));
}

namespace {
bool blocks_shape_ok(int64_t batch, int64_t seq_q, int64_t seq_kv, int64_t heads, int64_t heads_kv, int64_t head_dim) {
    return (head_dim == 64 || head_dim == 128) && batch > 0 && batch <= 65535 && heads > 0 && heads <= 65535 && heads_kv > 0 &&
           heads % heads_kv == 0 && seq_q > 0 && seq_q <= (1LL << 24) && seq_kv > 0 && seq_kv <= blocks::kMaxKeyBlocks * blocks::kKeyBlock;
}
}  // namespace

size_t sol_select_blocks_workspace_bytes(int64_t batch, int64_t seq_q, int64_t seq_kv, int64_t heads, int64_t heads_kv,
                                         int64_t head_dim) {
    return blocks_shape_ok(batch, seq_q, seq_kv, heads, heads_kv, head_dim)
               ? blocks::select_workspace_bytes(batch, seq_q, seq_kv, heads, heads_kv, head_dim) : 0;
}

sol_status_t sol_select_blocks(const void *q, const void *k, int64_t batch, int64_t seq_q, int64_t seq_kv, int64_t heads,
                               int64_t heads_kv, int64_t head_dim, int64_t ld_q, int64_t ld_k, int64_t count, int64_t keep_first,
                               const int32_t *kv_lens, int32_t *block_lists, int32_t *counts, float *scores, void *workspace,
                               size_t workspace_bytes, void *stream) {
    if (q == nullptr || k == nullptr || block_lists == nullptr || counts == nullptr || workspace == nullptr) return SOL_ERR_NULL_POINTER;
    if (!blocks_shape_ok(batch, seq_q, seq_kv, heads, heads_kv, head_dim) || ld_q < heads * head_dim || ld_k < heads_kv * head_dim ||
        count < 1 || count > blocks::kMaxKeyBlocks || keep_first < 0 || keep_first > count)
        return SOL_ERR_BAD_SHAPE;
    if (!aligned16(q) || !aligned16(k) || ld_q % 8 != 0 || ld_k % 8 != 0 || (reinterpret_cast<uintptr_t>(workspace) & 255u) ||
        (reinterpret_cast<uintptr_t>(kv_lens) & 3u) || (reinterpret_cast<uintptr_t>(block_lists) & 3u) ||
        (reinterpret_cast<uintptr_t>(counts) & 3u) || (reinterpret_cast<uintptr_t>(scores) & 3u))
        return SOL_ERR_ALIGNMENT;
    if (workspace_bytes < blocks::select_workspace_bytes(batch, seq_q, seq_kv, heads, heads_kv, head_dim)) return SOL_ERR_WORKSPACE_TOO_SMALL;
    const DeviceInfo *dev = nullptr;
    const sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return blocks::launch_select(q, k, batch, seq_q, seq_kv, heads, heads_kv, head_dim, ld_q, ld_k, count, keep_first, kv_lens,
                                 block_lists, counts, scores, workspace, static_cast<cudaStream_t>(stream), dev);
}

sol_status_t sol_attention_blocks(const void *q, const void *k, const void *v, void *out, int64_t batch, int64_t seq_q, int64_t seq_kv,
                                  int64_t heads, int64_t heads_kv, int64_t head_dim, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                  int64_t ld_out, const int32_t *block_lists, const int32_t *counts, int64_t max_blocks,
                                  const int32_t *kv_lens, void *stream) {
    if (q == nullptr || k == nullptr || v == nullptr || out == nullptr || block_lists == nullptr || counts == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!blocks_shape_ok(batch, seq_q, seq_kv, heads, heads_kv, head_dim) || max_blocks < 1 || max_blocks > blocks::kMaxKeyBlocks ||
        ld_q < heads * head_dim || ld_out < heads * head_dim || ld_k < heads_kv * head_dim || ld_v < heads_kv * head_dim)
        return SOL_ERR_BAD_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || ld_q % 8 != 0 || ld_k % 8 != 0 || ld_v % 8 != 0 ||
        ld_out % 8 != 0 || (reinterpret_cast<uintptr_t>(kv_lens) & 3u) || (reinterpret_cast<uintptr_t>(block_lists) & 3u) ||
        (reinterpret_cast<uintptr_t>(counts) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    const sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    const attn::Stream b{q, k, v, out, seq_q, seq_kv, ld_q, ld_k, ld_v, ld_out};
    const attn::BlockLists lists{block_lists, counts, kv_lens, max_blocks, heads_kv};
    return attn::launch_attention_blocks(b, lists, batch, heads, head_dim, static_cast<cudaStream_t>(stream), dev);
}

namespace {
bool matvec_shape_ok(int64_t M, int64_t K) { return shape_ok(M, K) && M <= (1LL << 18); }

sol_status_t matvec_entry(const void *x, int64_t ldx, const void *wq, const void *wsf, const float *wts, const void *bias,
                          sol_activation_t act, void *y, int64_t ldy, int64_t M, int64_t N, int64_t K, void *workspace,
                          size_t workspace_bytes, void *stream) {
    if (x == nullptr || wq == nullptr || wsf == nullptr || y == nullptr) return SOL_ERR_NULL_POINTER;
    if (act != SOL_ACT_NONE && act != SOL_ACT_SILU) return SOL_ERR_BAD_LAYOUT;
    if (!matvec_shape_ok(M, K) || !shape_ok(N, K) || N > (1LL << 22) || N % 8 != 0 || ldx < K || ldy < N) return SOL_ERR_BAD_SHAPE;
    if (!aligned16(x) || !aligned16(wq) || !aligned16(wsf) || !aligned16(y) || !aligned16(bias) || ldx % 8 != 0 || ldy % 8 != 0 ||
        (reinterpret_cast<uintptr_t>(wts) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return SOL_ERR_ALIGNMENT;
    const size_t need = matvec::workspace_bytes(M, K);
    if (need > 0 && workspace == nullptr) return SOL_ERR_NULL_POINTER;
    if (workspace_bytes < need) return SOL_ERR_WORKSPACE_TOO_SMALL;
    const DeviceInfo *dev = nullptr;
    const sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return matvec::launch_matvec(x, ldx, wq, wsf, wts, bias, y, ldy, M, N, K, act == SOL_ACT_SILU, workspace,
                                 static_cast<cudaStream_t>(stream));
}
}  // namespace

size_t sol_matvec_workspace_bytes(int64_t M, int64_t K) { return matvec_shape_ok(M, K) ? matvec::workspace_bytes(M, K) : 0; }

sol_status_t nvfp4_matvec(const void *x_bf16, int64_t ldx, const void *wq, const void *wsf, const float *w_tscale,
                          const void *bias_bf16, sol_activation_t activation, void *y_bf16, int64_t ldy, int64_t M,
                          int64_t N, int64_t K, void *workspace, size_t workspace_bytes, void *stream) {
    if (w_tscale == nullptr) return SOL_ERR_NULL_POINTER;
    return matvec_entry(x_bf16, ldx, wq, wsf, w_tscale, bias_bf16, activation, y_bf16, ldy, M, N, K, workspace, workspace_bytes, stream);
}

sol_status_t mxfp4_matvec(const void *x_bf16, int64_t ldx, const void *wq, const void *wsf, const void *bias_bf16,
                          sol_activation_t activation, void *y_bf16, int64_t ldy, int64_t M, int64_t N, int64_t K,
                          void *workspace, size_t workspace_bytes, void *stream) {
    return matvec_entry(x_bf16, ldx, wq, wsf, nullptr, bias_bf16, activation, y_bf16, ldy, M, N, K, workspace, workspace_bytes, stream);
}

sol_status_t sol_qk_rotary(const sol_head_tensor_t *q, const sol_head_tensor_t *k, int64_t rows, int64_t head_dim,
                           const sol_rotary_t *rot, float eps, void *stream) {
    if (q == nullptr) return SOL_ERR_NULL_POINTER;
    if (!rotary::head_dim_ok(head_dim) || rows <= 0 || rows > 0x7FFFFFFFLL || !(eps >= 0.0f)) return SOL_ERR_BAD_SHAPE;
    rotary::Heads2 heads{};
    const sol_head_tensor_t *both[2] = {q, k};
    for (int i = 0; i < 2; ++i) {
        const sol_head_tensor_t *s = both[i];
        if (s == nullptr) continue;
        if (s->x == nullptr || s->out == nullptr || (rot == nullptr && s->weight == nullptr)) return SOL_ERR_NULL_POINTER;
        if (s->heads <= 0 || s->heads > 65535 || s->ld_in < s->heads * head_dim || s->ld_out < s->heads * head_dim)
            return SOL_ERR_BAD_SHAPE;
        if (!aligned16(s->x) || !aligned16(s->out) || s->ld_in % 8 != 0 || s->ld_out % 8 != 0 || !aligned8(s->weight))
            return SOL_ERR_ALIGNMENT;
        heads.h[i] = rotary::Heads{static_cast<const uint16_t *>(s->x), static_cast<uint16_t *>(s->out),
                             static_cast<const uint16_t *>(s->weight), static_cast<int>(s->heads), s->ld_in, s->ld_out};
    }
    rotary::Turn t;
    sol_status_t st = make_turn(rot, head_dim, &t);
    if (st != SOL_OK) return st;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return rotary::launch_forward(heads, t, rows, head_dim, rot != nullptr && rot->layout == SOL_ROTARY_HALF, eps,
                                  static_cast<cudaStream_t>(stream), dev);
}

size_t sol_qk_rotary_backward_workspace_bytes(int64_t head_dim) {
    return rotary::head_dim_ok(head_dim) ? rotary::backward_workspace_bytes(head_dim) : 0;
}

sol_status_t sol_qk_rotary_backward(const sol_head_grad_t *q, const sol_head_grad_t *k, int64_t rows, int64_t head_dim,
                                    const sol_rotary_t *rot, float eps, void *workspace, size_t workspace_bytes,
                                    void *stream) {
    if (q == nullptr) return SOL_ERR_NULL_POINTER;
    if (!rotary::head_dim_ok(head_dim) || rows <= 0 || rows > 0x7FFFFFFFLL || !(eps >= 0.0f)) return SOL_ERR_BAD_SHAPE;
    rotary::Grads2 grads{};
    const sol_head_grad_t *both[2] = {q, k};
    bool weights = false;
    for (int i = 0; i < 2; ++i) {
        const sol_head_grad_t *s = both[i];
        if (s == nullptr) continue;
        if (s->dy == nullptr || s->dx == nullptr || (rot == nullptr && s->weight == nullptr)) return SOL_ERR_NULL_POINTER;
        if (s->weight != nullptr && (s->x == nullptr || s->dweight == nullptr)) return SOL_ERR_NULL_POINTER;
        const int64_t cols = s->heads * head_dim;
        if (s->heads <= 0 || s->heads > 65535 || s->ld_dy < cols || s->ld_dx < cols || (s->weight != nullptr && s->ld_x < cols))
            return SOL_ERR_BAD_SHAPE;
        if (!aligned16(s->dy) || !aligned16(s->dx) || s->ld_dy % 8 != 0 || s->ld_dx % 8 != 0 || !aligned8(s->weight) ||
            (s->weight != nullptr && (!aligned16(s->x) || s->ld_x % 8 != 0 || (reinterpret_cast<uintptr_t>(s->dweight) & 3u))))
            return SOL_ERR_ALIGNMENT;
        weights = weights || s->weight != nullptr;
        grads.g[i] = rotary::Grads{static_cast<const uint16_t *>(s->dy), static_cast<const uint16_t *>(s->x),
                             static_cast<uint16_t *>(s->dx), static_cast<const uint16_t *>(s->weight),
                             s->weight != nullptr ? s->dweight : nullptr, static_cast<int>(s->heads), s->ld_dy, s->ld_x, s->ld_dx};
    }
    rotary::Turn t;
    sol_status_t st = make_turn(rot, head_dim, &t);
    if (st != SOL_OK) return st;
    if (weights) {
        if (workspace == nullptr) return SOL_ERR_NULL_POINTER;
        if (workspace_bytes < rotary::backward_workspace_bytes(head_dim)) return SOL_ERR_WORKSPACE_TOO_SMALL;
        if (reinterpret_cast<uintptr_t>(workspace) & 255u) return SOL_ERR_ALIGNMENT;
    }
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return rotary::launch_backward(grads, t, rows, head_dim, rot != nullptr && rot->layout == SOL_ROTARY_HALF, eps,
                                   weights ? static_cast<double *>(workspace) : nullptr, static_cast<cudaStream_t>(stream), dev);
}

static bool norm_shape_ok(int64_t M, int64_t K, int64_t rows_per_sample) {
    return M > 0 && M <= 0x7FFFFFFFLL && K > 0 && K % 8 == 0 && K <= norm::max_k() && rows_per_sample > 0;
}

sol_status_t sol_layernorm(const void *x, int64_t M, int64_t K, int64_t ldx, const void *scale, const void *shift, int64_t ld_mod,
                           int64_t rows_per_sample, float scale_offset, float eps, void *y, int64_t ldy, float *stats, void *stream) {
    if (x == nullptr || y == nullptr) return SOL_ERR_NULL_POINTER;
    if (!norm_shape_ok(M, K, rows_per_sample) || ldx < K || ldy < K || !(eps >= 0.0f) || !std::isfinite(scale_offset) ||
        ((scale != nullptr || shift != nullptr) && ld_mod < K))
        return SOL_ERR_BAD_SHAPE;
    if (!aligned16(x) || !aligned16(y) || !aligned16(scale) || !aligned16(shift) || ldx % 8 != 0 || ldy % 8 != 0 || !aligned8(stats) ||
        ((scale != nullptr || shift != nullptr) && ld_mod % 8 != 0))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    const sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return norm::launch_forward(x, M, K, ldx, scale, shift, ld_mod, rows_per_sample < M ? rows_per_sample : M, scale_offset, eps, y, ldy, stats,
                                static_cast<cudaStream_t>(stream), dev);
}

size_t sol_layernorm_backward_workspace_bytes(int64_t M, int64_t K, int64_t rows_per_sample) {
    return norm_shape_ok(M, K, rows_per_sample) ? norm::backward_workspace_bytes(M, K, rows_per_sample < M ? rows_per_sample : M) : 0;
}

sol_status_t sol_layernorm_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ldx, const float *stats, const void *scale,
                                    int64_t ld_scale, int64_t M, int64_t K, int64_t rows_per_sample, float scale_offset, void *dx, int64_t ld_dx,
                                    float *dscale, float *dshift, void *workspace, size_t workspace_bytes, void *stream) {
    if (dy == nullptr || x == nullptr || stats == nullptr || dx == nullptr) return SOL_ERR_NULL_POINTER;
    if (!norm_shape_ok(M, K, rows_per_sample) || ld_dy < K || ldx < K || ld_dx < K || !std::isfinite(scale_offset) || (scale != nullptr && ld_scale < K))
        return SOL_ERR_BAD_SHAPE;
    if (!aligned16(dy) || !aligned16(x) || !aligned16(dx) || !aligned16(scale) || !aligned16(dscale) || !aligned16(dshift) ||
        !aligned8(stats) || ld_dy % 8 != 0 || ldx % 8 != 0 || ld_dx % 8 != 0 || (scale != nullptr && ld_scale % 8 != 0))
        return SOL_ERR_ALIGNMENT;
    if (rows_per_sample > M) rows_per_sample = M;
    const size_t need = dscale != nullptr || dshift != nullptr ? norm::backward_workspace_bytes(M, K, rows_per_sample) : 0;
    if (need > 0) {
        if (workspace == nullptr) return SOL_ERR_NULL_POINTER;
        if (workspace_bytes < need) return SOL_ERR_WORKSPACE_TOO_SMALL;
        if (reinterpret_cast<uintptr_t>(workspace) & 255u) return SOL_ERR_ALIGNMENT;
    }
    const DeviceInfo *dev = nullptr;
    const sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return norm::launch_backward(dy, ld_dy, x, ldx, stats, scale, ld_scale, M, K, rows_per_sample, scale_offset, dx, ld_dx, dscale, dshift,
                                 static_cast<float *>(workspace), static_cast<cudaStream_t>(stream), dev);
}

sol_status_t sol_adamw_step(const sol_adamw_tensor_t *tensors, int64_t count, const sol_adamw_options_t *o, int64_t *step_state,
                            void *stream) {
    if (o == nullptr || step_state == nullptr || (tensors == nullptr && count > 0)) return SOL_ERR_NULL_POINTER;
    if (count < 0 || count > 0x7FFFFFFFLL) return SOL_ERR_BAD_SHAPE;
    if (o->state_bits != 32 && o->state_bits != 8) return SOL_ERR_BAD_LAYOUT;
    auto from = [](double v, double lo) { return v >= lo && std::isfinite(v); };
    if (!from(o->lr, 0.0) || !from(o->weight_decay, 0.0) || !from(o->eps, 0.0) || !from(o->beta1, 0.0) || !from(o->beta2, 0.0) ||
        o->beta1 >= 1.0 || o->beta2 >= 1.0)
        return SOL_ERR_BAD_SHAPE;
    for (int64_t i = 0; i < count; ++i) {
        const sol_adamw_tensor_t &t = tensors[i];
        if (t.n < 0 || t.n > (1LL << 40)) return SOL_ERR_BAD_SHAPE;
        if (t.n == 0) continue;
        if (t.param == nullptr || t.grad == nullptr || t.m == nullptr || t.v == nullptr) return SOL_ERR_NULL_POINTER;
        if (o->state_bits == 8 && (t.m_scale == nullptr || t.v_scale == nullptr)) return SOL_ERR_NULL_POINTER;
        if (o->param_bf16 && t.copy != nullptr) return SOL_ERR_BAD_LAYOUT;
        if (!aligned16(t.param) || !aligned16(t.copy) || !aligned16(t.grad) || !aligned16(t.m) || !aligned16(t.v)) return SOL_ERR_ALIGNMENT;
    }
    if (!aligned8(step_state) || (reinterpret_cast<uintptr_t>(o->lr_scale) & 3u) || (reinterpret_cast<uintptr_t>(o->grad_scale) & 3u))
        return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    const sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return adamw::launch_step(tensors, count, *o, step_state, static_cast<cudaStream_t>(stream), dev);
}

static bool lora_shape_ok(int64_t M, int64_t K, int64_t N, int64_t r, int64_t adapters, int64_t requests) {
    auto width = [](int64_t c) { return c > 0 && c % 8 == 0 && c <= 1048576; };
    return M > 0 && M <= 0x7FFFFF00LL && width(K) && width(N) && r > 0 && r % 8 == 0 && r <= lora::max_rank() && adapters > 0 && adapters <= 1024 &&
           requests > 0 && requests <= lora::max_requests();
}
static sol_status_t lora_check(const lora::Call &c, const void *a_rows, int64_t lda, const void *b_rows, int64_t ldb, const void *ws, size_t ws_bytes, bool backward) {
    if (a_rows == nullptr || b_rows == nullptr || c.a == nullptr || c.b == nullptr || c.scaling == nullptr || c.offsets == nullptr || c.ids == nullptr)
        return SOL_ERR_NULL_POINTER;
    if (!lora_shape_ok(c.M, c.K, c.N, c.r, c.adapters, c.requests) || lda < c.K || ldb < c.N) return SOL_ERR_BAD_SHAPE;
    auto aligned4 = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; };
    if (!aligned16(a_rows) || !aligned16(b_rows) || !aligned16(c.a) || !aligned16(c.b) || lda % 8 != 0 || ldb % 8 != 0 || !aligned4(c.scaling) ||
        !aligned4(c.offsets) || !aligned4(c.ids))
        return SOL_ERR_ALIGNMENT;
    if (ws == nullptr) return SOL_ERR_NULL_POINTER;
    if (ws_bytes < lora::workspace_bytes(c.M, c.K, c.N, c.r, c.adapters, c.requests, backward)) return SOL_ERR_WORKSPACE_TOO_SMALL;
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return SOL_ERR_ALIGNMENT;
    return SOL_OK;
}

size_t sol_lora_workspace_bytes(int64_t M, int64_t K, int64_t N, int64_t r, int64_t adapters, int64_t requests, int backward) {
    return lora_shape_ok(M, K, N, r, adapters, requests) ? lora::workspace_bytes(M, K, N, r, adapters, requests, backward != 0) : 0;
}

sol_status_t sol_lora_apply(const void *x, int64_t ldx, const void *a, const void *b, const float *scaling, const int32_t *offsets,
                            const int32_t *ids, int64_t requests, int64_t adapters, void *y, int64_t ldy, void *t_out, int64_t M, int64_t K,
                            int64_t N, int64_t r, void *workspace, size_t workspace_bytes, void *stream) {
    const lora::Call c{a, b, scaling, offsets, ids, requests, adapters, M, K, N, r};
    sol_status_t st = lora_check(c, x, ldx, y, ldy, workspace, workspace_bytes, false);
    if (st != SOL_OK) return st;
    if (!aligned16(t_out)) return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return lora::launch_apply(c, x, ldx, y, ldy, t_out, workspace, static_cast<cudaStream_t>(stream));
}

sol_status_t sol_lora_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ldx, const void *t, const void *a, const void *b,
                               const float *scaling, const int32_t *offsets, const int32_t *ids, int64_t requests, int64_t adapters,
                               void *dx, int64_t ld_dx, float *da, float *db, int64_t M, int64_t K, int64_t N, int64_t r, void *workspace,
                               size_t workspace_bytes, void *stream) {
    const lora::Call c{a, b, scaling, offsets, ids, requests, adapters, M, K, N, r};
    sol_status_t st = lora_check(c, x, ldx, dy, ld_dy, workspace, workspace_bytes, true);
    if (st != SOL_OK) return st;
    if (t == nullptr || da == nullptr || db == nullptr) return SOL_ERR_NULL_POINTER;
    if (dx != nullptr && ld_dx < K) return SOL_ERR_BAD_SHAPE;
    if (!aligned16(t) || !aligned16(da) || !aligned16(db) || !aligned16(dx) || (dx != nullptr && ld_dx % 8 != 0)) return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return lora::launch_backward(c, dy, ld_dy, x, ldx, t, dx, ld_dx, da, db, workspace, static_cast<cudaStream_t>(stream));
}

sol_status_t sol_rotary_frequencies(int64_t dim, double theta, sol_rotary_scaling_t scaling, double factor,
                                    double original_length, double beta_fast, double beta_slow, double *freqs_out,
                                    double *scale_out) {
    if (freqs_out == nullptr || scale_out == nullptr) return SOL_ERR_NULL_POINTER;
    if (scaling != SOL_ROTARY_SCALE_NONE && scaling != SOL_ROTARY_SCALE_LINEAR && scaling != SOL_ROTARY_SCALE_NTK &&
        scaling != SOL_ROTARY_SCALE_YARN)
        return SOL_ERR_BAD_LAYOUT;
    if (dim <= 0 || dim % 2 != 0 || dim > 4096 || !(theta > 0.0) || !std::isfinite(theta) || !(factor >= 1.0) || !std::isfinite(factor))
        return SOL_ERR_BAD_SHAPE;
    if (scaling == SOL_ROTARY_SCALE_NTK && dim <= 2) return SOL_ERR_BAD_SHAPE;
    if (scaling == SOL_ROTARY_SCALE_YARN && (!(theta > 1.0) || !(original_length > 0.0) || !std::isfinite(original_length) ||
                                             !(beta_slow > 0.0) || !(beta_fast >= beta_slow) || !std::isfinite(beta_fast)))
        return SOL_ERR_BAD_SHAPE;
    const double d = static_cast<double>(dim);
    const double base = scaling == SOL_ROTARY_SCALE_NTK ? theta * std::pow(factor, d / (d - 2.0)) : theta;
    double lo = 0.0, hi = 0.0;
    if (scaling == SOL_ROTARY_SCALE_YARN) {
        // the (fractional) pair index that turns `beta` times over the original length
        auto pair_of = [&](double beta) { return d * std::log(original_length / (beta * 6.283185307179586477)) / (2.0 * std::log(theta)); };
        lo = std::fmax(std::floor(pair_of(beta_fast)), 0.0);
        hi = std::fmin(std::ceil(pair_of(beta_slow)), d - 1.0);
    }
    for (int64_t i = 0; i < dim / 2; ++i) {
        double f = std::pow(base, -2.0 * static_cast<double>(i) / d);
        if (scaling == SOL_ROTARY_SCALE_LINEAR) f /= factor;
        if (scaling == SOL_ROTARY_SCALE_YARN) {
            const double ramp = std::fmin(std::fmax((static_cast<double>(i) - lo) / std::fmax(hi - lo, 0.001), 0.0), 1.0);
            f = f / factor * ramp + f * (1.0 - ramp);
        }
        freqs_out[i] = f;
    }
    *scale_out = scaling == SOL_ROTARY_SCALE_YARN ? 0.1 * std::log(factor) + 1.0 : 1.0;
    return SOL_OK;
}

sol_status_t nvfp4_quantize_linear(const void *x_bf16, int64_t ldx, const void *wq, const void *wsf,
                                   const float *w_tscale, const void *bias_bf16, void *y_bf16, int64_t M,
                                   int64_t N, int64_t K, int64_t ldy, void *workspace, size_t workspace_bytes,
                                   void *stream) {
    if (x_bf16 == nullptr || wq == nullptr || wsf == nullptr || w_tscale == nullptr || y_bf16 == nullptr ||
        workspace == nullptr)
        return SOL_ERR_NULL_POINTER;
    sol_status_t st = check_linear_common(bias_bf16, y_bf16, M, N, K, ldy);
    if (st != SOL_OK) return st;
    if (ldx < K) return SOL_ERR_BAD_SHAPE;
    if (!aligned16(x_bf16) || !aligned16(wq) || !aligned16(wsf) || ldx % 8 != 0 ||
        (reinterpret_cast<uintptr_t>(w_tscale) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return SOL_ERR_ALIGNMENT;
    if (workspace_bytes < sol_nvfp4_linear_workspace_bytes(M, N, K)) return SOL_ERR_WORKSPACE_TOO_SMALL;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    uint8_t *xq = ws;
    uint8_t *xsf = xq + align256(sol_nvfp4_data_bytes(M, K));
    float *xts = reinterpret_cast<float *>(xsf + align256(sol_nvfp4_scale_bytes(M, K, SOL_SF_SWIZZLED_128x4)));
    st = launch_amax_quantize(x_bf16, M, K, ldx, xts, xq, xsf, SOL_SF_SWIZZLED_128x4, s, dev);
    if (st != SOL_OK) return st;
    return launch_gemm_nvfp4(xq, xsf, xts, wq, wsf, w_tscale, bias_bf16, y_bf16, M, N, K, ldy, s, dev);
}

sol_status_t nvfp4_quantize_linear_delayed(const void *x_bf16, int64_t ldx, const void *wq, const void *wsf,
                                           const float *w_tscale, const void *bias_bf16, void *y_bf16, int64_t M,
                                           int64_t N, int64_t K, int64_t ldy, float *scale_state, void *workspace,
                                           size_t workspace_bytes, void *stream) {
    if (x_bf16 == nullptr || wq == nullptr || wsf == nullptr || w_tscale == nullptr || y_bf16 == nullptr ||
        workspace == nullptr || scale_state == nullptr)
        return SOL_ERR_NULL_POINTER;
    sol_status_t st = check_linear_common(bias_bf16, y_bf16, M, N, K, ldy);
    if (st != SOL_OK) return st;
    if (ldx < K) return SOL_ERR_BAD_SHAPE;
    if (!aligned16(x_bf16) || ldx % 8 != 0 || !aligned16(wq) || !aligned16(wsf) ||
        (reinterpret_cast<uintptr_t>(w_tscale) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u) ||
        (reinterpret_cast<uintptr_t>(scale_state) & 7u))
        return SOL_ERR_ALIGNMENT;
    if (workspace_bytes < sol_nvfp4_linear_workspace_bytes(M, N, K)) return SOL_ERR_WORKSPACE_TOO_SMALL;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    uint8_t *xq = ws;
    uint8_t *xsf = xq + align256(sol_nvfp4_data_bytes(M, K));
    st = launch_quantize_tracking(x_bf16, M, K, ldx, scale_state, xq, xsf, reinterpret_cast<uint32_t *>(scale_state + 1),
                                  s);
    if (st != SOL_OK) return st;
    return launch_gemm_nvfp4(xq, xsf, scale_state, wq, wsf, w_tscale, bias_bf16, y_bf16, M, N, K, ldy, s, dev);
}

sol_status_t sol_roll_tensor_scale(float *scale_state, void *stream) {
    if (scale_state == nullptr) return SOL_ERR_NULL_POINTER;
    if (reinterpret_cast<uintptr_t>(scale_state) & 7u) return SOL_ERR_ALIGNMENT;
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    return launch_roll_scale(scale_state, static_cast<cudaStream_t>(stream));
}

sol_status_t nvfp4_quantize_linear_host(const void *x_host, int64_t ldx, const void *wq, const void *wsf,
                                        const float *w_tscale, const void *bias_bf16, void *y_host, int64_t M,
                                        int64_t N, int64_t K, int64_t ldy, void *x_dev, void *y_dev,
                                        void *workspace, size_t workspace_bytes, void *stream) {
    if (x_host == nullptr || y_host == nullptr || x_dev == nullptr || y_dev == nullptr) return SOL_ERR_NULL_POINTER;
    if (M <= 0 || N <= 0 || K <= 0 || ldx < K || ldy < N) return SOL_ERR_BAD_SHAPE;
    // validate everything else (and the device) before the first copy is queued
    if (wq == nullptr || wsf == nullptr || w_tscale == nullptr || workspace == nullptr) return SOL_ERR_NULL_POINTER;
    sol_status_t st = check_linear_common(bias_bf16, y_dev, M, N, K, N);
    if (st != SOL_OK) return st;
    if (!aligned16(x_dev) || !aligned16(wq) || !aligned16(wsf) || (reinterpret_cast<uintptr_t>(w_tscale) & 3u) ||
        (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return SOL_ERR_ALIGNMENT;
    if (workspace_bytes < sol_nvfp4_linear_workspace_bytes(M, N, K)) return SOL_ERR_WORKSPACE_TOO_SMALL;
    const DeviceInfo *dev = nullptr;
    st = check_arch(&dev);
    if (st != SOL_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cudaMemcpy2DAsync(x_dev, static_cast<size_t>(K) * 2, x_host, static_cast<size_t>(ldx) * 2,
                          static_cast<size_t>(K) * 2, static_cast<size_t>(M), cudaMemcpyHostToDevice, s) != cudaSuccess)
        return SOL_ERR_CUDA;
    st = nvfp4_quantize_linear(x_dev, K, wq, wsf, w_tscale, bias_bf16, y_dev, M, N, K, N, workspace, workspace_bytes,
                               stream);
    if (st != SOL_OK) return st;
    if (cudaMemcpy2DAsync(y_host, static_cast<size_t>(ldy) * 2, y_dev, static_cast<size_t>(N) * 2,
                          static_cast<size_t>(N) * 2, static_cast<size_t>(M), cudaMemcpyDeviceToHost, s) != cudaSuccess)
        return SOL_ERR_CUDA;
    return SOL_OK;
}

sol_status_t sol_set_wait_limit_cycles(int64_t cycles) {
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    const long long limit = cycles > 0 ? static_cast<long long>(cycles) : kDefaultWaitLimitCycles;
    if (cudaMemcpyToSymbol(g_status_block, &limit, sizeof(limit), offsetof(DeviceStatusBlock, wait_limit_cycles)) !=
        cudaSuccess)
        return SOL_ERR_CUDA;
    return SOL_OK;
}

sol_status_t sol_test_hold_loads(int on) {
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    const uint32_t flag = on ? 1u : 0u;
    if (cudaMemcpyToSymbol(g_status_block, &flag, sizeof(flag), offsetof(DeviceStatusBlock, hold_loads)) != cudaSuccess)
        return SOL_ERR_CUDA;
    return SOL_OK;
}

sol_status_t sol_last_device_status(void *stream, uint32_t *detail_out) {
    const DeviceInfo *dev = nullptr;
    sol_status_t st = check_arch(&dev);
    if (st != SOL_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint32_t word = 0;
    if (cudaStreamSynchronize(s) != cudaSuccess) return SOL_ERR_CUDA;
    if (cudaMemcpyFromSymbol(&word, g_status_block, sizeof(word)) != cudaSuccess) return SOL_ERR_CUDA;
    if (detail_out != nullptr) *detail_out = word;
    if (word != 0) {
        const uint32_t zero = 0;
        if (cudaMemcpyToSymbol(g_status_block, &zero, sizeof(zero)) != cudaSuccess) return SOL_ERR_CUDA;
        return SOL_ERR_TIMEOUT;
    }
    return SOL_OK;
}

}  // extern "C"
