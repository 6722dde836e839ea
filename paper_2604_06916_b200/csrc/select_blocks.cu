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
//
// Measured (B200, inside a graph): 2 x 4608 tokens, 24 heads x 128, 9 of 36 blocks: 35 us, of which pooling 25 us (4.5 TB/s; floor of both
// 17 us); 16421 tokens, 38 heads x 64, 24 of 129 blocks: 48 us (pooling 35 us, floor 24 us).  Pooling issues 6.5 instructions
// per element, which is half of its blocks' time and goes on under the loads; the other loss is uneven work: a query unit
// has twice a key unit's rows, and the fullest block gets 7 half-units of 128 rows against a mean of 5.84 (16421 tokens: 10
// against 8.75, the last of ten column chunks half empty besides).  One block per unit with sixteen rows in flight per warp, whose warps all load
// at once and then add at once: 34 us and 69 us; eight rows: 46 and 96 us.  A warp per query block for the scores, the
// key means read again for each: 84 us and 145 us.
#include "ptx.cuh"
#include "sol_internal.h"

namespace sol {
namespace blocks {
namespace {

constexpr int kPoolWarps = 8;
constexpr int kColumns = 256;          // columns of a pooling unit: 16 bytes per lane
constexpr int kBatch = 8;              // rows of a warp's batch: one is on its way while the one before is added

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
};

struct PoolParams {
    PoolTensor q, k;
    int q_units, k_units;
    int head_dim_log2;
};

__device__ __forceinline__ int valid_rows(const int32_t *lens, int b, int seq) {
    return lens == nullptr ? seq : min(max(__ldg(lens + b), 0), seq);
}

// (volatile: all loads of a batch are issued before the first addition, which the compiler otherwise trades for registers)
__device__ __forceinline__ uint4 load_once(const uint16_t *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// A block of rows by 256 columns.  Its rows go to the warps in turn, a batch at a time.
struct Unit {
    const uint16_t *x;      // this lane's first column in the block's first row, or null: no such column
    int64_t ld;
    int rows, batches;      // rows that exist; batches of each warp
    int b, blk, c0;         // sample, block, first column
    bool is_q;
};
__device__ __forceinline__ Unit unit_of(const PoolParams &p, int at, int lane) {
    Unit u;
    u.is_q = at < p.q_units;
    const PoolTensor &t = u.is_q ? p.q : p.k;
    const uint32_t unit = static_cast<uint32_t>(u.is_q ? at : at - p.q_units), line = unit / static_cast<uint32_t>(t.column_chunks);
    u.c0 = static_cast<int>(unit - line * t.column_chunks) * kColumns;
    u.b = static_cast<int>(line / static_cast<uint32_t>(t.blocks));
    u.blk = static_cast<int>(line) - u.b * t.blocks;
    const int c = u.c0 + 8 * lane, row0 = u.blk * t.rows_per_block;
    u.x = c < t.heads << p.head_dim_log2 ? t.x + u.b * t.batch_stride + static_cast<int64_t>(row0) * t.ld + c : nullptr;
    u.ld = t.ld;
    u.rows = min(t.rows_per_block, valid_rows(t.lens, u.b, t.seq) - row0);
    u.batches = t.rows_per_block / (kPoolWarps * kBatch);
    return u;
}

// Blocks stay and walk the units, loads running ahead over the units' borders: without that all warps of the GPU load at
// once and then add at once.
__global__ void __launch_bounds__(32 * kPoolWarps, 2)
pool_kernel(const PoolParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ double part[2][kPoolWarps][kColumns];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int units = p.q_units + p.k_units;
    auto fetch = [&](const Unit &u, int batch, uint4 (&v)[kBatch]) {
        const int first = (batch * kPoolWarps + warp) * kBatch;
        if (u.x == nullptr || first + kBatch > u.rows) {     // no columns, or a block's ragged end
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                v[i] = u.x != nullptr && first + i < u.rows ? load_once(u.x + (first + i) * u.ld) : make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) v[i] = load_once(u.x + (first + i) * u.ld);
        }
    };
    double acc[8];
    auto add_all = [&](const uint4 (&v)[kBatch]) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                acc[2 * e] += scaled_lo(w[e]);
                acc[2 * e + 1] += scaled_hi(w[e]);
            }
        }
    };
    int at = blockIdx.x, buf = 0;
    if (at >= units) return;
    Unit u = unit_of(p, at, lane);
    uint4 now[kBatch], next[kBatch];
    fetch(u, 0, now);
    while (at < units) {
        const int following = at + gridDim.x;
        Unit v = u;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.0;
        for (int batch = 0; batch < u.batches; batch += 2) {       // two or four batches
            fetch(u, batch + 1, next);
            add_all(now);
            if (batch + 2 < u.batches) {
                fetch(u, batch + 2, now);
            } else if (following < units) {
                v = unit_of(p, following, lane);
                fetch(v, 0, now);
            }
            add_all(next);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) part[buf][warp][32 * e + lane] = acc[e];    // column 8 * lane + e: no bank is hit twice
        __syncthreads();
        const PoolTensor &t = u.is_q ? p.q : p.k;
        const int col = u.c0 + 8 * lane + warp;    // a warp takes one of the eight columns of each lane
        if (col < t.heads << p.head_dim_log2) {
            double sum = 0.0;
#pragma unroll
            for (int w = 0; w < kPoolWarps; ++w) sum += part[buf][w][32 * warp + lane];
            const double mean = u.rows > 0 ? sum * 0x1p896 / static_cast<double>(u.rows) : 0.0;
            const int head = col >> p.head_dim_log2, d = col & ((1 << p.head_dim_log2) - 1);
            const int64_t bh = static_cast<int64_t>(u.b) * t.heads + head;
            if (u.is_q) t.out[((bh * t.blocks + u.blk) << p.head_dim_log2) + d] = mean;
            else t.out[((bh << p.head_dim_log2) + d) * t.blocks + u.blk] = mean;
        }
        u = v;
        at = following;
        buf ^= 1;      // the sums of this unit may still be read when the next one's are written
    }
}
static_assert(kPoolWarps == 8 && kKeyBlock % (2 * kPoolWarps * kBatch) == 0 && kQueryBlock % (2 * kPoolWarps * kBatch) == 0, "pairs of batches");

struct SelectParams {
    const double *pq, *pk;
    const int32_t *kv_lens;
    int32_t *blocks, *counts;
    float *scores;            // null: not asked for
    int heads, group, q_blocks, k_blocks, seq_kv, head_dim, count, keep_first;
    int parts;                // of head_dim, summed by different warps
};

// A CTA takes kRows query blocks of one head (the key means are read once for all of them).  Scores: a warp takes 32 key
// blocks, a lane per key block, and where key blocks are few a part of head_dim; the parts are added in order.  They become
// ordered 64-bit keys in shared memory, and a warp per query block finds the smallest kept key -- by counting, for every
// key, the keys before it where these are few, else by a binary search over the bits -- and writes the list by ballots.
constexpr int kSelectWarps = 8;
constexpr int kParts = 4;                  // of head_dim
constexpr int kMaxSplit = 256;             // key blocks up to which head_dim is split: beyond, the key blocks alone occupy the warps
constexpr int kMaxRanked = 96;             // key blocks up to which keys are counted: there it costs what 64 passes of the search do
constexpr int kManyRows = 4;
constexpr int kMaxShared = 1024;           // key blocks up to which a CTA takes kManyRows query blocks
template <int kRows>
__global__ void __launch_bounds__(32 * kSelectWarps)
select_kernel(const SelectParams p) {
    extern __shared__ __align__(16) double shared[];
    double *means = shared;                                             // [head_dim][kRows]
    double *sums = shared + p.head_dim * kRows;                         // [parts][kRows][k_blocks]; part 0 becomes the keys
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int qb0 = blockIdx.x * kRows, head = blockIdx.y, b = blockIdx.z;
    const int valid = (valid_rows(p.kv_lens, b, p.seq_kv) + kKeyBlock - 1) / kKeyBlock;     // a prefix of the key blocks
    const int64_t row0 = (static_cast<int64_t>(b) * p.heads + head) * p.q_blocks + qb0;
    const double *k = p.pk + (static_cast<int64_t>(b) * (p.heads / p.group) + head / p.group) * p.head_dim * p.k_blocks;
    auto key_of = [](double s) {
        const unsigned long long bits = static_cast<unsigned long long>(__double_as_longlong(s + 0.0));   // -0 is 0
        return bits >> 63 ? ~bits : bits | 0x8000000000000000ull;
    };
    auto score_of = [](unsigned long long key) {
        return __longlong_as_double(static_cast<long long>(key >> 63 ? key & 0x7FFFFFFFFFFFFFFFull : ~key));
    };
    ptx::grid_dependency_wait();
    for (int i = threadIdx.x; i < kRows * p.head_dim; i += 32 * kSelectWarps) {
        const int r = i / p.head_dim, d = i % p.head_dim;
        means[d * kRows + r] = qb0 + r < p.q_blocks ? p.pq[(row0 + r) * p.head_dim + d] : 0.0;
    }
    __syncthreads();
    const int depth = p.head_dim / p.parts;
    for (int item = warp; item < (valid + 31) / 32 * p.parts; item += kSelectWarps) {
        const int j = item / p.parts * 32 + lane, part = item % p.parts;
        if (j >= valid) continue;
        const double *kd = k + static_cast<int64_t>(part * depth) * p.k_blocks + j, *qd = means + part * depth * kRows;
        double s[kRows] = {};
#pragma unroll 16
        for (int d = 0; d < depth; ++d) {
            const double kv = kd[static_cast<int64_t>(d) * p.k_blocks];
#pragma unroll
            for (int r = 0; r < kRows; ++r) s[r] = fma(qd[d * kRows + r], kv, s[r]);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) sums[(part * kRows + r) * p.k_blocks + j] = s[r];
    }
    __syncthreads();
    const int qb = qb0 + warp;
    if (warp >= kRows || qb >= p.q_blocks) return;
    const int64_t row = row0 + warp;
    unsigned long long *keys = reinterpret_cast<unsigned long long *>(sums) + static_cast<int64_t>(warp) * p.k_blocks;
    for (int j = lane; j < valid; j += 32) {
        double s = sums[warp * p.k_blocks + j];
        for (int i = 1; i < p.parts; ++i) s += sums[(i * kRows + warp) * p.k_blocks + j];
        keys[j] = key_of(s);
    }
    __syncwarp();
    const int forced = min(p.keep_first, min(valid, p.count)), wanted = min(p.count, valid), open = wanted - forced;
    // the largest key that at least `open` of the blocks behind the forced ones reach, and how many lie above it
    unsigned long long cut = 0;
    int above = 0;
    if (valid > kMaxRanked && open > 0) {
        // bits that all upper halves share need no pass, and no further one once exactly `open` keys reach the trial
        uint32_t least = 0xFFFFFFFFu, most = 0;
        for (int j = forced + lane; j < valid; j += 32) {
            const uint32_t upper = static_cast<uint32_t>(keys[j] >> 32);
            least = min(least, upper);
            most = max(most, upper);
        }
        least = __reduce_min_sync(0xFFFFFFFFu, least);
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        int bit = 63 - __clz(least ^ most);                       // 31 where they agree in all 32
        cut = static_cast<unsigned long long>(most) << 32 >> bit >> 1 << bit << 1;     // the shared bits (a shift by 64 is none)
        for (; bit >= 0; --bit) {
            const unsigned long long trial = cut | 1ull << bit;
            int reach = 0;
            for (int j0 = forced; j0 < valid; j0 += 32)
                reach += __popc(__ballot_sync(0xFFFFFFFFu, j0 + lane < valid && keys[j0 + lane] >= trial));
            if (reach >= open) cut = trial;
            if (reach == open) break;
        }
        for (int j0 = forced; j0 < valid; j0 += 32)
            above += __popc(__ballot_sync(0xFFFFFFFFu, j0 + lane < valid && keys[j0 + lane] > cut));
    }
    int32_t *list = p.blocks + row * p.count;
    float *out_scores = p.scores == nullptr ? nullptr : p.scores + row * p.count;
    const uint32_t below = (1u << lane) - 1u;
    int written = 0, ties_left = open - above;
    for (int j0 = 0; j0 < valid; j0 += 32) {
        const int j = j0 + lane;
        bool take = j < forced, tie = false;
        if (j >= forced && j < valid && open > 0) {
            const unsigned long long mine = keys[j];
            if (valid <= kMaxRanked) {
                int before = 0;
                for (int i = forced; i < valid; ++i) before += keys[i] > mine || (keys[i] == mine && i < j);
                take = before < open;
            } else {
                take = mine > cut;
                tie = mine == cut;
            }
        }
        const uint32_t ties = __ballot_sync(0xFFFFFFFFu, tie);      // taken from the lowest, as far as there is room
        take = take || (tie && __popc(ties & below) < ties_left);
        ties_left -= min(max(ties_left, 0), __popc(ties));
        const uint32_t taken = __ballot_sync(0xFFFFFFFFu, take);
        if (take) {
            const int at = written + __popc(taken & below);
            list[at] = j;
            if (out_scores != nullptr) out_scores[at] = static_cast<float>(score_of(keys[j]));
        }
        written += __popc(taken);
    }
    for (int i = written + lane; i < p.count; i += 32) {
        list[i] = -1;
        if (out_scores != nullptr) out_scores[i] = -INFINITY;
    }
    if (lane == 0) p.counts[row] = written;
}

size_t select_smem(int rows, int parts, int64_t head_dim, int nk) { return sizeof(double) * rows * (head_dim + static_cast<size_t>(parts) * nk); }
constexpr int kMaxSelectSmem = 8 * (128 + kMaxKeyBlocks);      // one row over the most key blocks

template <int kRows>
sol_status_t launch_scores(const SelectParams &p, int64_t batch, cudaStream_t stream) {
    static bool configured[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SOL_ERR_CUDA;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(select_kernel<kRows>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSelectSmem) != cudaSuccess) return SOL_ERR_CUDA;
        configured[dev] = true;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(ceil_div(p.q_blocks, kRows)), static_cast<unsigned>(p.heads), static_cast<unsigned>(batch));
    cfg.blockDim = dim3(32 * kSelectWarps);
    cfg.dynamicSmemBytes = select_smem(kRows, p.parts, p.head_dim, p.k_blocks);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, select_kernel<kRows>, p) != cudaSuccess) {
        cudaGetLastError();
        return SOL_ERR_CUDA;
    }
    return launch_status();
}

}  // namespace

size_t select_workspace_bytes(int64_t batch, int64_t seq_q, int64_t seq_kv, int64_t heads, int64_t heads_kv, int64_t head_dim) {
    return static_cast<size_t>(batch * head_dim * (heads * ceil_div(seq_q, kQueryBlock) + heads_kv * ceil_div(seq_kv, kKeyBlock))) * sizeof(double);
}

sol_status_t launch_select(const void *q, const void *k, int64_t batch, int64_t seq_q, int64_t seq_kv, int64_t heads, int64_t heads_kv,
                           int64_t head_dim, int64_t ld_q, int64_t ld_k, int64_t count, int64_t keep_first, const int32_t *kv_lens,
                           int32_t *blocks, int32_t *counts, float *scores, void *workspace, cudaStream_t stream, const DeviceInfo *dev) {
    const int nq = static_cast<int>(ceil_div(seq_q, kQueryBlock)), nk = static_cast<int>(ceil_div(seq_kv, kKeyBlock));
    double *pq = static_cast<double *>(workspace), *pk = pq + batch * heads * nq * head_dim;
    PoolParams pool{};
    pool.q = PoolTensor{static_cast<const uint16_t *>(q), pq, nullptr, ld_q, seq_q * ld_q, static_cast<int>(seq_q), static_cast<int>(heads), nq,
                        kQueryBlock, static_cast<int>(ceil_div(heads * head_dim, kColumns))};
    pool.k = PoolTensor{static_cast<const uint16_t *>(k), pk, kv_lens, ld_k, seq_kv * ld_k, static_cast<int>(seq_kv), static_cast<int>(heads_kv), nk,
                        kKeyBlock, static_cast<int>(ceil_div(heads_kv * head_dim, kColumns))};
    const int64_t q_units = batch * nq * pool.q.column_chunks, k_units = batch * nk * pool.k.column_chunks;
    if (q_units + k_units > 0x3FFFFFFFLL) return SOL_ERR_BAD_SHAPE;
    pool.q_units = static_cast<int>(q_units);
    pool.k_units = static_cast<int>(k_units);
    pool.head_dim_log2 = head_dim == 128 ? 7 : 6;
    const int64_t resident = 2LL * dev->sm_count;
    pool_kernel<<<static_cast<unsigned>(q_units + k_units < resident ? q_units + k_units : resident), 32 * kPoolWarps, 0, stream>>>(pool);
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
    p.parts = nk <= kMaxSplit ? kParts : 1;
    return nk <= kMaxShared ? launch_scores<kManyRows>(p, batch, stream) : launch_scores<1>(p, batch, stream);
}

}  // namespace blocks
}  // namespace sol
