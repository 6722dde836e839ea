// Choosing key blocks for block-sparse attention (sm_100a).  Per batch element and head:
//     pq[i] = mean of the query rows of block i (256 tokens), pk[j] = mean of the key rows of block j (128 tokens)
//     score[i][j] = pq[i] . pk[j];  each query block keeps the `count` key blocks of the highest score
// (the first keep_first blocks whatever their score; among equal scores the lower index), ascending.
//
// pool_kernel reads q and k once and is HBM bound; everything behind it works on 1/128 of the data.  Means and scores
// are FP64: a list of indices has no tolerance, and near the cut two scores may differ by less than FP32 resolves.
// Sums of up to 256 BF16 values are exact in FP64 unless their exponents span 37 bits, so the lists do not depend
// on the order of the sums.  A BF16 value becomes FP64 by shifting its bits into the upper word (which scales it by
// 2^-896, undone once per mean): two or three integer operations in place of a conversion instruction, which issues
// at a quarter of the rate of the additions.
#include "ptx.cuh"
#include "sol_internal.h"

namespace sol {
namespace blocks {
namespace {

constexpr int kPoolWarps = 8;
constexpr int kPoolColumns = 256;      // columns of a pooling CTA: 16 bytes per lane
constexpr int kRowsInFlight = 8;       // rows a warp loads before it adds any

// FP64 of the two BF16 halves of a word, times 2^-896 (upper words; the lower ones are zero).
__device__ __forceinline__ double scaled_hi(uint32_t w) {
    return __hiloint2double((static_cast<int>(w) >> 3) & static_cast<int>(0x8FFFE000u), 0);
}
__device__ __forceinline__ double scaled_lo(uint32_t w) { return scaled_hi(w << 16); }

struct PoolTensor {
    const uint16_t *x;
    double *out;              // q: [batch, heads, blocks, head_dim]; k: [batch, heads, head_dim, blocks]
    const int32_t *lens;      // per batch element, or null
    int64_t ld, batch_stride; // elements
    int seq, heads, blocks, rows_per_block, column_chunks;
    bool transposed;
};

struct PoolParams {
    PoolTensor q, k;
    int q_ctas;               // CTAs of q along x; the rest pool k
    int head_dim_log2;
};

__device__ __forceinline__ int valid_rows(const int32_t *lens, int b, int seq) {
    return lens == nullptr ? seq : min(max(__ldg(lens + b), 0), seq);
}

__global__ void __launch_bounds__(32 * kPoolWarps)
pool_kernel(const PoolParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ double part[kPoolWarps][kPoolColumns];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, b = blockIdx.y;
    const bool is_q = static_cast<int>(blockIdx.x) < p.q_ctas;
    const PoolTensor t = is_q ? p.q : p.k;
    const int unit = is_q ? blockIdx.x : blockIdx.x - p.q_ctas;
    const int blk = unit / t.column_chunks, c0 = unit % t.column_chunks * kPoolColumns;
    const int columns = t.heads << p.head_dim_log2;
    const int row0 = blk * t.rows_per_block, rows = min(t.rows_per_block, valid_rows(t.lens, b, t.seq) - row0);
    const int c = c0 + 8 * lane;
    const bool live = c < columns;       // columns are a multiple of 64: a lane is wholly inside or outside
    const uint16_t *x = t.x + b * t.batch_stride + static_cast<int64_t>(row0) * t.ld + c;
    double acc[8] = {};
    for (int r0 = warp; r0 < rows; r0 += kPoolWarps * kRowsInFlight) {
        uint4 v[kRowsInFlight];
#pragma unroll
        for (int i = 0; i < kRowsInFlight; ++i) {
            const int r = r0 + i * kPoolWarps;
            v[i] = live && r < rows ? __ldg(reinterpret_cast<const uint4 *>(x + r * t.ld)) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kRowsInFlight; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                acc[2 * e] += scaled_lo(w[e]);
                acc[2 * e + 1] += scaled_hi(w[e]);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[warp][8 * lane + e] = acc[e];
    __syncthreads();
    const int col = c0 + threadIdx.x;
    if (col >= columns) return;
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kPoolWarps; ++w) sum += part[w][threadIdx.x];
    const double mean = rows > 0 ? sum * 0x1p896 / static_cast<double>(rows) : 0.0;
    const int head = col >> p.head_dim_log2, d = col & ((1 << p.head_dim_log2) - 1);
    const int64_t bh = static_cast<int64_t>(b) * t.heads + head;
    if (t.transposed) t.out[((bh << p.head_dim_log2) + d) * t.blocks + blk] = mean;
    else t.out[((bh * t.blocks + blk) << p.head_dim_log2) + d] = mean;
}

struct SelectParams {
    const double *pq, *pk;
    const int32_t *kv_lens;
    int32_t *blocks, *counts;
    float *scores;            // null: not asked for
    int heads, group, q_blocks, k_blocks, seq_kv, head_dim, count, keep_first;
};

// A warp per query block: scores of all key blocks as ordered 64-bit keys in shared memory, the smallest kept key by a
// binary search over its bits, the list by ballots.
__global__ void select_kernel(const SelectParams p) {
    extern __shared__ unsigned long long keys_all[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int qb = blockIdx.x * (blockDim.x >> 5) + warp, head = blockIdx.y, b = blockIdx.z;
    if (qb >= p.q_blocks) return;
    unsigned long long *keys = keys_all + static_cast<int64_t>(warp) * p.k_blocks;
    ptx::grid_dependency_wait();
    const int valid = (valid_rows(p.kv_lens, b, p.seq_kv) + kKeyBlock - 1) / kKeyBlock;     // a prefix of the key blocks
    const int64_t row = (static_cast<int64_t>(b) * p.heads + head) * p.q_blocks + qb;
    const double *q = p.pq + row * p.head_dim;
    const double *k = p.pk + (static_cast<int64_t>(b) * (p.heads / p.group) + head / p.group) * p.head_dim * p.k_blocks;
    auto score_of_key = [](unsigned long long key) {
        const unsigned long long bits = key >> 63 ? key & 0x7FFFFFFFFFFFFFFFull : ~key;
        return __longlong_as_double(static_cast<long long>(bits));
    };
    for (int j0 = 0; j0 < valid; j0 += 32) {
        const int j = j0 + lane;
        double s = 0.0;
        if (j < valid) {
#pragma unroll 8
            for (int d = 0; d < p.head_dim; ++d) s = fma(__ldcg(q + d), __ldcg(k + static_cast<int64_t>(d) * p.k_blocks + j), s);
            const unsigned long long bits = static_cast<unsigned long long>(__double_as_longlong(s + 0.0));   // -0 is 0
            keys[j] = bits >> 63 ? ~bits : bits | 0x8000000000000000ull;
        }
    }
    __syncwarp();
    const int forced = min(p.keep_first, min(valid, p.count)), wanted = min(p.count, valid);
    // among the blocks behind the forced ones: the largest key that at least `wanted - forced` of them reach
    unsigned long long cut = 0;
    if (wanted < valid && wanted > forced) {
        for (int bit = 63; bit >= 0; --bit) {
            const unsigned long long trial = cut | 1ull << bit;
            int reach = 0;
            for (int j0 = forced; j0 < valid; j0 += 32)
                reach += __popc(__ballot_sync(0xFFFFFFFFu, j0 + lane < valid && keys[j0 + lane] >= trial));
            if (reach >= wanted - forced) cut = trial;
        }
    }
    int above = 0;      // blocks strictly above the cut; the rest of the list are the lowest-numbered ones at it
    for (int j0 = forced; j0 < valid; j0 += 32)
        above += __popc(__ballot_sync(0xFFFFFFFFu, j0 + lane < valid && keys[j0 + lane] > cut));
    int at_cut = wanted - forced - above, written = 0;
    int32_t *list = p.blocks + row * p.count;
    float *out_scores = p.scores == nullptr ? nullptr : p.scores + row * p.count;
    for (int j0 = 0; j0 < valid; j0 += 32) {
        const int j = j0 + lane;
        const bool behind = j < valid && j >= forced && wanted > forced;
        const bool tie = behind && keys[j] == cut;
        const uint32_t ties = __ballot_sync(0xFFFFFFFFu, tie), below = (1u << lane) - 1u;
        const bool take = j < forced || (behind && keys[j] > cut) || (tie && __popc(ties & below) < at_cut);
        const uint32_t taken = __ballot_sync(0xFFFFFFFFu, take);
        if (take) {
            const int at = written + __popc(taken & below);
            list[at] = j;
            if (out_scores != nullptr) out_scores[at] = static_cast<float>(score_of_key(keys[j]));
        }
        written += __popc(taken);
        at_cut -= min(at_cut, __popc(ties));
    }
    for (int i = written + lane; i < p.count; i += 32) {
        list[i] = -1;
        if (out_scores != nullptr) out_scores[i] = -INFINITY;
    }
    if (lane == 0) p.counts[row] = written;
}

constexpr int kSelectWarps = 4;
constexpr int kMaxSelectSmem = kMaxKeyBlocks * 8;

}  // namespace

size_t select_workspace_bytes(int64_t batch, int64_t seq_q, int64_t seq_kv, int64_t heads, int64_t heads_kv, int64_t head_dim) {
    return static_cast<size_t>(batch * head_dim * (heads * ceil_div(seq_q, kQueryBlock) + heads_kv * ceil_div(seq_kv, kKeyBlock))) * sizeof(double);
}

sol_status_t launch_select(const void *q, const void *k, int64_t batch, int64_t seq_q, int64_t seq_kv, int64_t heads, int64_t heads_kv,
                           int64_t head_dim, int64_t ld_q, int64_t ld_k, int64_t count, int64_t keep_first, const int32_t *kv_lens,
                           int32_t *blocks, int32_t *counts, float *scores, void *workspace, cudaStream_t stream) {
    const int nq = static_cast<int>(ceil_div(seq_q, kQueryBlock)), nk = static_cast<int>(ceil_div(seq_kv, kKeyBlock));
    double *pq = static_cast<double *>(workspace), *pk = pq + batch * heads * nq * head_dim;
    PoolParams pool{};
    pool.q = PoolTensor{static_cast<const uint16_t *>(q), pq, nullptr, ld_q, seq_q * ld_q, static_cast<int>(seq_q), static_cast<int>(heads), nq,
                        kQueryBlock, static_cast<int>(ceil_div(heads * head_dim, kPoolColumns)), false};
    pool.k = PoolTensor{static_cast<const uint16_t *>(k), pk, kv_lens, ld_k, seq_kv * ld_k, static_cast<int>(seq_kv), static_cast<int>(heads_kv), nk,
                        kKeyBlock, static_cast<int>(ceil_div(heads_kv * head_dim, kPoolColumns)), true};
    pool.q_ctas = nq * pool.q.column_chunks;
    pool.head_dim_log2 = head_dim == 128 ? 7 : 6;
    const int64_t ctas = pool.q_ctas + static_cast<int64_t>(nk) * pool.k.column_chunks;
    if (ctas > 0x7FFFFFFFLL) return SOL_ERR_BAD_SHAPE;
    pool_kernel<<<dim3(static_cast<unsigned>(ctas), static_cast<unsigned>(batch)), 32 * kPoolWarps, 0, stream>>>(pool);
    const sol_status_t st = launch_status();
    if (st != SOL_OK) return st;

    SelectParams p{};
    p.pq = pq;
    p.pk = pk;
    p.kv_lens = kv_lens;
    p.blocks = blocks;
    p.counts = counts;
    p.scores = scores;
    p.heads = static_cast<int>(heads);
    p.group = static_cast<int>(heads / heads_kv);
    p.q_blocks = nq;
    p.k_blocks = nk;
    p.seq_kv = static_cast<int>(seq_kv);
    p.head_dim = static_cast<int>(head_dim);
    p.count = static_cast<int>(count);
    p.keep_first = static_cast<int>(keep_first);
    // several query blocks per CTA share the key means in L1 as long as their keys leave room for more CTAs
    const int warps = nk <= 512 ? kSelectWarps : 1;
    static bool configured[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SOL_ERR_CUDA;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSelectSmem) != cudaSuccess) return SOL_ERR_CUDA;
        configured[dev] = true;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(ceil_div(nq, warps)), static_cast<unsigned>(heads), static_cast<unsigned>(batch));
    cfg.blockDim = dim3(static_cast<unsigned>(32 * warps));
    cfg.dynamicSmemBytes = static_cast<size_t>(warps) * nk * sizeof(double);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, select_kernel, static_cast<const SelectParams &>(p)) != cudaSuccess) {
        cudaGetLastError();
        return SOL_ERR_CUDA;
    }
    return launch_status();
}

}  // namespace blocks
}  // namespace sol
