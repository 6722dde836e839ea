// Block-sparse attention (sm_100a): softmax(q k^T / sqrt(d)) v where each block of 256 queries of a head attends to a list
// of key blocks of 128 tokens.  Products, softmax and roundings are those of the dense kernel, tile for tile.
//
// One CTA per SM, which stays and walks the items (256 query rows of one head of one sample): over a handful of key tiles the
// way into an item (list, Q and the first K, the first scores) and out of it (last product, output) would otherwise cost a
// third of its time.  The next item's list is counted, and its Q and keys are loaded, under the current one.
//
// Per item two query tiles of 128 rows share the K and V tiles (two-stage rings that run on from item to item).  Step
// N = 2 J + t is key tile J (numbered through all items) with query tile t:
//     S = Q_t K_J^T            tcgen05.mma kind::f16, 128 x 128 x d; one score tile serves all steps in turn
//     softmax                  a thread per query row takes the row into registers -- the score tile is then free and the
//                              next step's scores, the other query tile's, are issued -- and forms p = exp2(s c - m)
//     O_t = alpha O_t + P V    P as packed BF16 in a place of its own per query tile; O rescaled when the maximum moved
// So the two query tiles take turns, one's exponentials under the other's loads and maxima, and the scores of a query
// tile's next step are there when it asks.  TMEM: O_0, O_1 (d columns each), P_0, P_1 (64 each), S (128).
//
// Warps: 0..3 and 4..7 = softmax / output of query tile 0 and 1 (one warp per TMEM lane quadrant), 8 = TMA producer, 9 = TMEM
// owner and MMA issuer, 10 = counts the list of the next item; their warpgroup leaves registers to the other two.  Every
// mbarrier wait is bounded, and a warp that works together gives up together.
//
// Measured on B200: 4 x 4608 tokens, 24 heads of 128, 9 of 36 blocks 271 us in a loop of calls (960 TFLOP/s, 58 % of the measured
// BF16 rate) and 229 to 256 us inside a graph, by the clock that the board holds; 2 x 4429, 38 heads of 64, 8 blocks 153 and
// 151 us; 1 x 1536, 24 heads of 128, 4 of 12 blocks 16.4 and 13.8 us.  A key tile takes 3 030 cycles for both query tiles (d =
// 128; clock readings of a tracing copy), of which the products are 2 048 and the rest is the way of a score row through its
// thread; the tensor pipe is busy 59 % of a block's time (d = 64: 30 %).  An item costs 3 000 to 3 800 cycles more: last product,
// output, next first scores.  A CTA per item instead, with the same steps, takes 12.8 us on the smallest case (nothing to
// overlap there, and a plainer way in) but 157 and 234 us on the others.
// Tried without gain: sixteen softmax warps, two threads per row (345 us on the first case); P in two halves (277); three-input
// maxima; two score tiles for d = 64 in phase (179 instead of 159) or one ahead (159); scores of 64 keys at a time (269);
// the next item's Q pulled into L2 ahead (152 and 232 instead of 151 and 231); rows stored by the threads instead of by TMA
// (1 % slower); an item's output after the next item's first exponentials (within 0.5 %).
#include "gemm_common.cuh"
#include "quant_math.cuh"
#include "sol_internal.h"

namespace sol {
namespace attn {
namespace {

using gemm::loads_held;
using gemm::wait_bounded;

constexpr int kBQ = 128, kQTiles = 2, kBKV = 128;
constexpr int kBox = 128 * 128;         // bytes of a [128 rows][64 BF16] box
constexpr int kStages = 2;              // K ring and V ring
constexpr int kWarpsPerTile = 4;
constexpr int kProducer = kQTiles * kWarpsPerTile, kIssuer = kProducer + 1, kCounter = kProducer + 2;      // warp indexes
constexpr int kThreads = 32 * (kProducer + 4);             // whole warpgroups: registers are handed over between them
// 384 threads start with 168 registers each, 64512 in all; 256 x 208 + 128 x 80 = 63488.
constexpr int kSoftmaxRegisters = 208, kOtherRegisters = 80;
static_assert(kSoftmaxRegisters * 32 * kProducer + kOtherRegisters * 128 <= 168 * kThreads, "registers that the block has");
constexpr int kOutBox = 32 * 128;       // bytes of a warp's [32 rows][64 BF16] output box
constexpr float kLazyLog2 = 8.0f;       // slack of the softmax reference maximum, in powers of two
constexpr uint32_t kTmemCols = 512, kColScores = 384;
constexpr int kFirstKeys = 8;           // first keys of the latest tiles, handed from the producer to the softmax
// barriers: Q and O [query tile]; rings [stage]; pairs [query tile][odd key tile]; item information [odd item]
constexpr int kQFull = 0, kQEmpty = 2, kKFull = 4, kKEmpty = 6, kVFull = 8, kVEmpty = 10, kSOf = 12, kLoadOf = 16, kPOf = 20, kPvOf = 24,
              kOEmpty = 28, kInfoFull = 30, kInfoEmpty = 32, kNumBars = 34;
struct Shared {                         // behind the tiles
    uint64_t bars[kNumBars];
    uint32_t tmem, abort_flag;
    int tiles[2], keys[2];              // of an item, by its parity
    int first_key[kFirstKeys];
};
constexpr int smem_bytes(int head_dim) {
    return (kQTiles + 2 * kStages) * (head_dim / 64) * kBox + kQTiles * kWarpsPerTile * kOutBox + static_cast<int>(sizeof(Shared));
}
static_assert(smem_bytes(128) <= 232448, "shared memory budget");

struct Params {
    const int32_t *blocks, *counts, *kv_lens;   // kv_lens null: every sample has seq_kv keys
    uint32_t *status;
    int seq_q, seq_kv, heads, group, q_blocks, max_blocks, items;
    float scale_log2;      // log2(e) / sqrt(d)
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

template <int kD>
__global__ void __launch_bounds__(kThreads, 1)
attention_blocks_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o, const Params p) {
    constexpr int kBoxes = kD / 64;
    constexpr int kTile = kBoxes * kBox;    // bytes of a [128][kD] BF16 tile
    constexpr uint32_t kColP = 2 * kD;
    static_assert(kColP + 128 <= kColScores, "tensor memory");
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t smem_base = ptx::smem_u32(smem_raw);
    if (smem_base & 1023u) {  // the swizzled operand layout needs 1024-byte alignment
        if (threadIdx.x == 0) atomicExch(p.status, 0xB00u);
        return;
    }
    const uint32_t sQ = smem_base, sK = sQ + kQTiles * kTile, sV = sK + kStages * kTile, sOut = sV + kStages * kTile;
    Shared &sh = *reinterpret_cast<Shared *>(smem_raw + (sOut - smem_base) + kQTiles * kWarpsPerTile * kOutBox);
    const uint32_t bar_base = ptx::smem_u32(sh.bars);
    auto bar = [&](int i) { return bar_base + 8u * i; };
    auto pair = [](int kind, int t, int J) { return kind + 2 * t + (J & 1); };            // barrier of key tile J
    auto phase = [](int J) { return static_cast<uint32_t>(J >> 1) & 1u; };                // its parity; rings likewise
    volatile uint32_t *abort_flag = &sh.abort_flag;
    volatile int *tiles_of = sh.tiles, *keys_of = sh.keys, *first_key_of = sh.first_key;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    struct Item { int q_block, head, batch; };
    auto item_of = [&](int w) {
        const int line = w / p.q_blocks, batch = line / p.heads;
        return Item{w - line * p.q_blocks, line - batch * p.heads, batch};
    };
    auto keys_of_sample = [&](int batch) { return p.kv_lens == nullptr ? p.seq_kv : min(max(__ldg(p.kv_lens + batch), 0), p.seq_kv); };
    if (threadIdx.x == 0) {
        for (int i = 0; i < kNumBars; ++i) {
            const bool of_tile = (i >= kLoadOf && i < kPvOf) || (i >= kOEmpty && i < kInfoFull);
            ptx::mbar_init(bar(i), of_tile ? kWarpsPerTile : i >= kInfoEmpty ? 1 + kQTiles * kWarpsPerTile : 1);
        }
        *abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
        ptx::prefetch_tmap(&tm_q);
        ptx::prefetch_tmap(&tm_k);
        ptx::prefetch_tmap(&tm_v);
        ptx::prefetch_tmap(&tm_o);
    }
    if (warp == kIssuer) {
        ptx::tmem_alloc(ptx::smem_u32(&sh.tmem), kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t *>(&sh.tmem);

    auto wait1 = [&](int b, uint32_t parity, uint32_t code) { return wait_bounded(bar(b), parity, abort_flag, p.status, code); };
    auto wait32 = [&](int b, uint32_t parity, uint32_t code) { return __all_sync(0xFFFFFFFFu, wait1(b, parity, code)) != 0; };
    // Items are numbered i = 0, 1, ... per CTA; `full` counts those with keys, J their key tiles.
    auto info_full = [&](int i) { return kInfoFull + (i & 1); };

    if (warp >= kProducer) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegisters));
        if (warp == kCounter) {
            // ------------------------------------------------------------ lists ahead: keys of the sample, entries that name some
            for (int w = blockIdx.x, i = 0; w < p.items; w += gridDim.x, ++i) {
                const Item it = item_of(w);
                const int32_t *from = p.blocks + static_cast<int64_t>(w) * p.max_blocks;
                int next = lane < p.max_blocks ? __ldg(from + lane) : -1;       // not after the count: one latency, not two
                const int keys = keys_of_sample(it.batch);
                const int named = min(max(__ldg(p.counts + w), 0), p.max_blocks), existing = (keys + kBKV - 1) / kBKV;
                int kept = 0;
                for (int e0 = 0; e0 < named; e0 += 32) {
                    const bool keep = e0 + lane < named && next >= 0 && next < existing;
                    if (e0 + 32 + lane < named) next = __ldg(from + e0 + 32 + lane);
                    kept += __popc(__ballot_sync(0xFFFFFFFFu, keep));
                }
                if (!wait32(kInfoEmpty + (i & 1), phase(i) ^ 1u, 0xB01u)) break;
                if (lane == 0) {
                    tiles_of[i & 1] = kept;
                    keys_of[i & 1] = keys;
                    ptx::mbar_arrive(bar(info_full(i)));
                }
                __syncwarp();
            }
        } else if (warp == kProducer) {
            // ------------------------------------------------------------ TMA producer
            if (ptx::elect_one()) {
                const bool held = loads_held(p.status);     // looked at with the first list: one latency, not two
                bool ok = true;
                int J = 0, full = 0;
                for (int w = blockIdx.x; ok && w < p.items; w += gridDim.x) {
                    const Item it = item_of(w);
                    const int32_t *from = p.blocks + static_cast<int64_t>(w) * p.max_blocks;
                    int next = __ldg(from);
                    const int keys = keys_of_sample(it.batch), named = held ? 0 : min(max(__ldg(p.counts + w), 0), p.max_blocks);
                    const int existing = (keys + kBKV - 1) / kBKV;
                    const int xq = it.head * kD, xkv = it.head / p.group * kD;
                    bool first = true;
                    for (int e = 0; ok && e < named; ++e) {
                        const int entry = next;
                        if (e + 1 < named) next = __ldg(from + e + 1);
                        if (entry < 0 || entry >= existing) continue;        // names no keys
                        const int key0 = entry * kBKV, st = J & 1;
                        auto load_q = [&](int t) {      // the tile's last scores of the item before are done
                            if (full > 0 && !wait1(kQEmpty + t, static_cast<uint32_t>(full - 1) & 1u, 0xB03u)) return false;
                            ptx::mbar_arrive_expect_tx(bar(kQFull + t), kTile);
#pragma unroll
                            for (int bx = 0; bx < kBoxes; ++bx)
                                ptx::tma_load_3d(sQ + t * kTile + bx * kBox, &tm_q, xq + 64 * bx, (it.q_block * kQTiles + t) * kBQ, it.batch, bar(kQFull + t));
                            return true;
                        };
                        if (first && !(ok = load_q(0))) break;
                        if (!(ok = wait1(kKEmpty + st, phase(J) ^ 1u, 0xB10u | st))) break;
                        first_key_of[J % kFirstKeys] = key0;
                        ptx::mbar_arrive_expect_tx(bar(kKFull + st), kTile);
#pragma unroll
                        for (int bx = 0; bx < kBoxes; ++bx)
                            ptx::tma_load_3d(sK + st * kTile + bx * kBox, &tm_k, xkv + 64 * bx, key0, it.batch, bar(kKFull + st));
                        if (first && !(ok = load_q(1))) break;
                        if (!(ok = wait1(kVEmpty + st, phase(J) ^ 1u, 0xB20u | st))) break;
                        ptx::mbar_arrive_expect_tx(bar(kVFull + st), kTile);
#pragma unroll
                        for (int bx = 0; bx < kBoxes; ++bx)
                            ptx::tma_load_3d(sV + st * kTile + bx * kBox, &tm_v, xkv + 64 * bx, key0, it.batch, bar(kVFull + st));
                        full += first ? 1 : 0;
                        first = false;
                        ++J;
                    }
                }
            }
            __syncwarp();
        } else if (warp == kIssuer) {
            // ------------------------------------------------------------ MMA issuer
            if (ptx::elect_one()) {
                // BF16 x BF16 -> FP32, M = 128; scores N = 128 keys, output N = kD with B MN-major (bit 16: V is [kv][d])
                constexpr uint32_t idesc_base = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(128 >> 4) << 24);
                constexpr uint32_t idesc_qk = idesc_base | (static_cast<uint32_t>(kBKV >> 3) << 17);
                constexpr uint32_t idesc_pv = idesc_base | (static_cast<uint32_t>(kD >> 3) << 17) | (1u << 16);
                // step n of an item whose key tiles start at J0 and which `full` items with keys precede
                struct Work { int J0, steps, full; };
                // S = Q_t K^T, 16 elements of d per instruction; the score tile is free once the step before has been loaded
                auto scores = [&](const Work &k, int n) {
                    const int t = n & 1, J = k.J0 + (n >> 1), st = J & 1, N = 2 * k.J0 + n - 1;
                    if (n < 2 && !wait1(kQFull + t, static_cast<uint32_t>(k.full) & 1u, 0xB31u)) return false;
                    if (t == 0 && !wait1(kKFull + st, phase(J), 0xB41u)) return false;
                    if (N >= 0 && !wait1(pair(kLoadOf, N & 1, N >> 1), phase(N >> 1), 0xB40u)) return false;
                    ptx::tc_fence_after_sync();
#pragma unroll
                    for (int c = 0; c < kD / 16; ++c) {
                        const uint64_t a = ptx::smem_desc_sw128(sQ + t * kTile + (c >> 2) * kBox) + 2u * (c & 3);
                        const uint64_t b = ptx::smem_desc_sw128(sK + st * kTile + (c >> 2) * kBox) + 2u * (c & 3);
                        ptx::mma_bf16(tmem_base + kColScores, a, b, idesc_qk, c > 0);
                    }
                    ptx::tc_commit(bar(pair(kSOf, t, J)));
                    if (t == 1) ptx::tc_commit(bar(kKEmpty + st));
                    if (n >= k.steps - 2) ptx::tc_commit(bar(kQEmpty + t));
                    return true;
                };
                // O_t += P V, 16 keys (8 columns of packed P) per instruction
                auto product = [&](const Work &k, int n) {
                    const int t = n & 1, J = k.J0 + (n >> 1), st = J & 1;
                    if (!wait1(pair(kPOf, t, J), phase(J), 0xB60u | t)) return false;
                    if (t == 0 && !wait1(kVFull + st, phase(J), 0xB70u)) return false;
                    if (n < 2 && k.full > 0 && !wait1(kOEmpty + t, static_cast<uint32_t>(k.full - 1) & 1u, 0xB71u)) return false;   // the item before has been read
                    ptx::tc_fence_after_sync();
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const uint64_t b = ptx::smem_desc_sw128_mn(sV + st * kTile + c * 2048, kBox, 1024);
                        ptx::mma_bf16_a_tmem(tmem_base + kD * t, tmem_base + kColP + 64 * t + 8 * c, b, idesc_pv, n > 1 || c > 0);
                    }
                    ptx::tc_commit(bar(pair(kPvOf, t, J)));
                    if (t == 1) ptx::tc_commit(bar(kVEmpty + st));
                    return true;
                };
                bool ok = true;
                int J0 = 0, full = 0;
                for (int w = blockIdx.x, i = 0; ok && w < p.items; w += gridDim.x, ++i) {
                    if (!(ok = wait1(info_full(i), phase(i), 0xB30u))) break;
                    const int tiles = tiles_of[i & 1];
                    ptx::mbar_arrive(bar(kInfoEmpty + (i & 1)));
                    if (tiles == 0) continue;
                    const Work k{J0, 2 * tiles, full};
                    // Each step's scores when the tile is free, then the product whose P is the next to arrive.  The last two
                    // products do not wait for the next item's first scores: the softmax warps need them to go on, and the
                    // information of a later item needs the softmax warps (several empty lists in a row).
                    for (int n = 0; ok && n < k.steps; ++n) ok = scores(k, n) && (n < 2 || product(k, n - 2));
                    ok = ok && product(k, k.steps - 2) && product(k, k.steps - 1);
                    J0 += tiles;
                    ++full;
                }
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegisters));
        // ------------------------------------------------------------ softmax and output: thread = query row
        const int t = warp / kWarpsPerTile, quad = warp & 3;
        const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
        const uint32_t t_out = tmem_base + kD * t + lanes, t_s = tmem_base + kColScores + lanes, t_p = tmem_base + kColP + 64 * t + lanes;
        const uint32_t s_out = sOut + warp * kOutBox;
        const uint32_t sw = static_cast<uint32_t>(lane & 7);
        bool ok = true;
        int J = 0;
        for (int w = blockIdx.x, i = 0; ok && w < p.items; w += gridDim.x, ++i) {
            if (!wait32(info_full(i), phase(i), 0xB80u)) break;
            const int tiles = tiles_of[i & 1], keys = keys_of[i & 1];
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(kInfoEmpty + (i & 1)));
            float m = -INFINITY, l = 0.0f;
            for (int j = 0; j < tiles; ++j, ++J) {
                if (!(ok = wait32(pair(kSOf, t, J), phase(J), 0xB82u | t))) break;
                ptx::tc_fence_after_sync();
                uint32_t s[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) ptx::tmem_ld_32x32(t_s + 32 * c, s[c]);
                ptx::tmem_ld_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar(pair(kLoadOf, t, J)));
                const int valid = keys - first_key_of[J % kFirstKeys];    // keys of this tile that exist (>= 1)
                if (valid < kBKV) {  // keys that do not exist score -inf
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (c * 32 + e >= valid) s[c][e] = 0xFF800000u;
                    if (t == 0 && keys < p.seq_kv) {
                        // Value rows behind the length may hold anything, and 0 times NaN is NaN: they are cleared before P is
                        // handed over, which the issuer waits for before it uses V for either query tile.  (Rows behind
                        // seq_kv arrive as zeros.)
                        const int st = J & 1;
                        if (!(ok = wait32(kVFull + st, phase(J), 0xB90u | st))) break;
                        for (int c = valid * 8 + quad * 32 + lane; c < kBKV * 8; c += 32 * kWarpsPerTile) {
#pragma unroll
                            for (int bx = 0; bx < kBoxes; ++bx) sts128(sV + st * kTile + bx * kBox + c * 16, 0, 0, 0, 0);
                        }
                        ptx::fence_proxy_async_smem();
                    }
                }
                float mx8[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) mx8[e] = __uint_as_float(s[0][e]);
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (c + e > 0) mx8[k] = fmaxf(mx8[k], __uint_as_float(s[c][e + k]));
                const float mx = fmaxf(fmaxf(fmaxf(mx8[0], mx8[1]), fmaxf(mx8[2], mx8[3])),
                                       fmaxf(fmaxf(mx8[4], mx8[5]), fmaxf(mx8[6], mx8[7])));
                // The reference maximum m only follows the row maximum when that has grown by more than 2^8: until then the
                // probabilities are up to 256 times larger (exact in FP32 and BF16 alike, l carries the same factor) and O, which
                // lives in TMEM, does not have to be rescaled.
                const float m_tile = mx * p.scale_log2;
                const bool move = m_tile > m + kLazyLog2;
                const float m_new = move ? m_tile : m;
                const float alpha = move ? ex2(m - m_new) : 1.0f;   // 0 on the first tile (m = -inf)
                float sum = 0.0f;
                const uint64_t c2 = qmath::f32x2(p.scale_log2, p.scale_log2), nm2 = qmath::f32x2(-m_new, -m_new);
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        // s c - m for two scores in one two-lane FMA (each lane rounded as the scalar form would be)
                        float x0, x1;
                        qmath::f32x2_split(qmath::fma2(qmath::f32x2(__uint_as_float(s[c][e]), __uint_as_float(s[c][e + 1])), c2, nm2), x0, x1);
                        const float p0 = ex2(x0), p1 = ex2(x1);
                        sum += p0 + p1;
                        s[c][e >> 1] = pack_bf16(p0, p1);  // 16 words per 32 keys, packed in place
                    }
                l = fmaf(l, alpha, sum);
                m = m_new;
                if (j > 0) {      // O may be rescaled, and P's place written, once the product before is done
                    if (!(ok = wait32(pair(kPvOf, t, J - 1), phase(J - 1), 0xBA8u | t))) break;
                    ptx::tc_fence_after_sync();
                    if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
                        for (int c = 0; c < kD / 32; ++c) {
                            uint32_t o[32];
                            ptx::tmem_ld_32x32(t_out + 32 * c, o);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                            ptx::tmem_st_32x32(t_out + 32 * c, o);
                        }
                    }
                }
                // P row: keys 2c and 2c+1 in column c
#pragma unroll
                for (int c = 0; c < 4; ++c) ptx::tmem_st_32x16(t_p + 16 * c, s[c]);
                ptx::tc_wait_st();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar(pair(kPOf, t, J)));
            }
            if (!ok) break;
            if (tiles > 0) {
                if (!(ok = wait32(pair(kPvOf, t, J - 1), phase(J - 1), 0xBA0u | t))) break;
                ptx::tc_fence_after_sync();
            }
            const float inv = 1.0f / l;
            const Item it = item_of(w);
            const int row0 = (it.q_block * kQTiles + t) * kBQ + quad * 32;
#pragma unroll
            for (int bx = 0; bx < kBoxes; ++bx) {     // 64 columns at a time through the warp's box
                if (lane == 0) ptx::tma_store_wait_read<0>();     // the store before has left the box
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t o[32];
                    if (tiles > 0) {
                        ptx::tmem_ld_32x32(t_out + 64 * bx + 32 * c, o);
                        ptx::tmem_ld_wait();
                    }
                    if (bx == kBoxes - 1 && c == 1 && tiles > 0) {      // O_t may be overwritten
                        ptx::tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(bar(kOEmpty + t));
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[e] = tiles > 0 ? pack_bf16(__uint_as_float(o[8 * q + 2 * e]) * inv, __uint_as_float(o[8 * q + 2 * e + 1]) * inv)
                                             : 0u;                       // no key is listed
                        sts128(s_out + lane * 128 + ((static_cast<uint32_t>(4 * c + q) ^ sw) << 4), v[0], v[1], v[2], v[3]);
                    }
                }
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (row0 < p.seq_q) ptx::tma_store_3d(&tm_o, it.head * kD + 64 * bx, row0, it.batch, s_out);   // clipped at the last row
                    ptx::tma_store_commit();
                }
            }
        }
        if (lane == 0) ptx::tma_store_wait_all<0>();
        __syncwarp();
    }

    // ---------------------------------------------------------------- teardown
    if (*abort_flag) __nanosleep(2000000);  // let copies already in flight land before the CTA exits
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == kIssuer) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
}

template <int kD>
sol_status_t launch(const CUtensorMap (&tm)[4], const Params &p, cudaStream_t stream, const DeviceInfo *dev) {
    constexpr int smem = smem_bytes(kD);
    static bool configured[64] = {};
    if (!configured[dev->device]) {
        if (cudaFuncSetAttribute(attention_blocks_kernel<kD>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return SOL_ERR_CUDA;
        configured[dev->device] = true;
    }
    const unsigned grid = static_cast<unsigned>(p.items < dev->sm_count ? p.items : dev->sm_count);
    attention_blocks_kernel<kD><<<grid, kThreads, smem, stream>>>(tm[0], tm[1], tm[2], tm[3], p);
    return launch_status();
}

}  // namespace

sol_status_t launch_attention_blocks(const Stream &s, const BlockLists &lists, int64_t batch, int64_t heads, int64_t head_dim,
                                     cudaStream_t stream, const DeviceInfo *dev) {
    const int64_t q_blocks = ceil_div(s.seq_q, kQTiles * kBQ);
    if (q_blocks * heads * batch > 0x3FFFFFFFLL) return SOL_ERR_BAD_SHAPE;
    CUtensorMap tm[4];
    auto make = [&](CUtensorMap *t, const void *base, int64_t h, int64_t seq, int64_t ld, uint32_t box_rows) {
        return make_tmap_3d_bf16(t, base, static_cast<uint64_t>(h * head_dim), static_cast<uint64_t>(seq), static_cast<uint64_t>(batch),
                                 static_cast<uint64_t>(ld) * 2, static_cast<uint64_t>(seq) * ld * 2, 64, box_rows);
    };
    if (!make(tm, s.q, heads, s.seq_q, s.ld_q, kBQ) || !make(tm + 1, s.k, lists.heads_kv, s.seq_kv, s.ld_k, kBKV) ||
        !make(tm + 2, s.v, lists.heads_kv, s.seq_kv, s.ld_v, kBKV) || !make(tm + 3, s.out, heads, s.seq_q, s.ld_out, 32))
        return SOL_ERR_CUDA;
    Params p{};
    p.blocks = lists.blocks;
    p.counts = lists.counts;
    p.kv_lens = lists.kv_lens;
    p.status = device_status_word();
    p.seq_q = static_cast<int>(s.seq_q);
    p.seq_kv = static_cast<int>(s.seq_kv);
    p.heads = static_cast<int>(heads);
    p.group = static_cast<int>(heads / lists.heads_kv);
    p.q_blocks = static_cast<int>(q_blocks);
    p.max_blocks = static_cast<int>(lists.max_blocks);
    p.items = static_cast<int>(q_blocks * heads * batch);
    p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(head_dim));
    return head_dim == 128 ? launch<128>(tm, p, stream, dev) : launch<64>(tm, p, stream, dev);
}

}  // namespace attn
}  // namespace sol
