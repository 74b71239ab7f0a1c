// The per-query term of the backward of attention over token sequences where the caller has no fp32 output,
//     Delta_i = sum_j P_ij (dout_i . v_j) / sum_j P_ij,
// from the probabilities in fp32.  dout_i . out_i with an output that was rounded to bf16, of probabilities that were rounded to bf16, is subtracted
// from nearly equal numbers in rows of few large probabilities: with scores of standard deviation 4, dq and dk were off by 0.5 to 0.8 %, now by
// 0.23 % (what the roundings of dS and of the results leave).  (The sum of the same probabilities below: a row with one key has Delta = dP.)
//
// An item is 128 queries of a head: S = Q K^T and dP = dO V^T of one key tile after the other go to tensor memory (2 x 256 columns, in turn), sixteen
// warps read both, a row per thread and a quarter of the columns per warp.  lse is known, so that there is no reference to look for and nothing
// to rescale.  The grid is persistent and the items go round by turns, back and forth (the longest come first), so that every warp knows them
// without being told.  Bound by the special-function unit, one exponential per pair: causal, 8 heads of 64, 4 096 tokens 26 us, 32 768 tokens with the
// penalty on distance 1.19 ms (the unit alone 1.07); 64 documents of 512-2 048 tokens, 16 heads on 4, with all options 0.67 ms.  (Two blocks of
// eight such warps per SM, 128 columns at a time, an item each: 59 us, 1.35 and 1.18 ms.)
//
//   warp 0  TMA producer: Q and dO of an item, K and V through a ring     warp 1  issues the MMAs     warp 3  adds an item's sums up, writes Delta
//   warps 4-19  probabilities and sums
#pragma once

#include "attn_position.cuh"
#include "attn_terms.cuh"

namespace gt {
namespace {

using namespace sm100;
using namespace position;

struct DeltaParams {
    const int32_t* cu_seqlens;
    const int32_t* prefix;
    const float* slopes;
    const float* lse;        // [H,T]
    uint4* ext;              // rows of folded terms; the second half of a (query, head) row is written
    uint32_t* status;
    const int4* list;        // as the main kernel's; item = entry {document, block, first row, rows} * heads + head
    int32_t n_items;
    int32_t n_graphs, n_total, n_heads, group, causal;
    int32_t by_work;         // without a list: the same block of all documents, then the next (else document after document)
    int32_t blocks;          // ... of the longest document
    float c1, to_tanh, cap2;
};

constexpr int kDeltaThreads = 640, kDeltaWarps = 16, kDeltaStages = 3;
template <int D>
struct DeltaSmem {
    static constexpr int kRowBytes = D * 2, kTileBytes = 128 * kRowBytes, kPair = 2 * kTileBytes;
    static constexpr int kQ = 0;                                     // [2 items] Q, dO
    static constexpr int kK = 2 * kPair;                             // [kDeltaStages] K, V
    static constexpr int kSums = kK + kDeltaStages * kPair;          // [2 items][4 column groups][128 rows] {sum P dP, sum P}
    static constexpr int kBars = kSums + 2 * 4 * 128 * 8;
    static constexpr int kMisc = kBars + 24 * 8;
    static constexpr int kDynamic = kMisc + 16 + 1024;               // slack for the 1024-byte alignment
    static_assert(kBars % 8 == 0 && kMisc % 16 == 0 && kDynamic <= 227 * 1024, "aligned, and within an SM");
};

template <int D, bool kCap, bool kSlope>
__global__ void __launch_bounds__(kDeltaThreads, 1)
position_delta_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                      const __grid_constant__ CUtensorMap tmap_do, const DeltaParams p)
{
    using L = DeltaSmem<D>;
    constexpr int kTile = 128;
    enum {
        kQFull = 0, kQEmpty = 2,                      // [2 items]
        kKvFull = 4, kKvEmpty = kKvFull + kDeltaStages,
        kScores = kKvEmpty + kDeltaStages,            // [2]  S and dP of a key tile are in tensor memory
        kRead = kScores + 2,                          // [2]  they have been read: an arrival per warp
        kSumsFull = kRead + 2, kSumsEmpty = kSumsFull + 2,       // [2 items]
        kBarriers = kSumsEmpty + 2
    };
    static_assert(kBarriers <= 24);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint64_t* bars = (uint64_t*)(smem + L::kBars);
    uint32_t* misc = (uint32_t*)(smem + L::kMisc);       // [0] TMEM base, [1] abort flag
    float2* sums = (float2*)(smem + L::kSums);
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    volatile uint32_t* abort_flag = &misc[1];
    if (tid == 0) {
        misc[1] = 0u;
        for (int i = 0; i < kBarriers; ++i) mbar_init(bar(i), (i >= kRead && i < kRead + 4) ? kDeltaWarps : 1);      // kRead, kSumsFull
        fence_mbar_init();
        prefetch_tensormap(&tmap_q);
        prefetch_tensormap(&tmap_k);
        prefetch_tensormap(&tmap_v);
        prefetch_tensormap(&tmap_do);
    }
    if (warp == 2) { tmem_alloc(smem_u32(&misc[0]), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = misc[0];
    grid_wait();

    // The items of this block, in turn; a turn may have none (n_kv 0), or there are no more (head -1).
    struct Item { int32_t head, node0, n, prefix, q0, n_kv; };
    auto item_of = [&](int turn) -> Item {
        const int32_t index = turn * (int32_t)gridDim.x + ((turn & 1) != 0 ? (int32_t)(gridDim.x - 1 - blockIdx.x) : (int32_t)blockIdx.x);
        Item it{-1, 0, 0, 0, 0, 0};
        if (turn * (int64_t)gridDim.x >= p.n_items) return it;
        it.head = 0;
        if (index >= p.n_items) return it;
        it.head = index % p.n_heads;
        const int32_t row = index / p.n_heads;
        int32_t g, block;
        if (p.list) {
            const int4 entry = p.list[row];
            g = entry.x;
            block = entry.y;
            it.node0 = entry.z;
            it.n = entry.x < 0 ? 0 : entry.w;
        } else {
            block = p.by_work ? row / p.n_graphs : row % p.blocks;
            g = p.by_work ? row % p.n_graphs : row / p.blocks;
            it.node0 = p.cu_seqlens ? p.cu_seqlens[g] : 0;
            it.n = p.cu_seqlens ? p.cu_seqlens[g + 1] - it.node0 : p.n_total;
        }
        const int32_t n_tiles = (it.n + kTile - 1) / kTile;
        if (block >= n_tiles) return it;
        it.prefix = p.prefix ? p.prefix[g] : 0;
        const int32_t q_tile = p.causal ? n_tiles - 1 - block : block;
        it.q0 = q_tile * kTile;
        it.n_kv = p.causal ? max(q_tile + 1, (min(it.n, it.prefix) + kTile - 1) / kTile) : n_tiles;
        return it;
    };
    // A wait by a whole warp, with one answer for all of its lanes.
    auto wait = [&](int i, uint32_t parity, uint32_t site) -> bool { return __all_sync(0xffffffffu, mbar_wait(bar(i), parity, abort_flag, p.status, site)); };

    if (warp == 0) {
        int c = 0, k = 0;                                    // key tiles and items so far
        bool good = true;                                    // no wait has been given up
        for (int turn = 0; good; ++turn) {
            const Item it = item_of(turn);
            if (it.head < 0) break;
            if (it.n_kv == 0) continue;
            if (k >= 2 && !wait(kQEmpty + (k & 1), ((k >> 1) & 1) ^ 1, 400)) break;
            if (lane == 0) {
                uint8_t* to = smem + L::kQ + (k & 1) * L::kPair;
                mbar_arrive_expect_tx(bar(kQFull + (k & 1)), L::kPair);
                tma_load_3d(smem_u32(to), &tmap_q, bar(kQFull + (k & 1)), 0, it.head, it.node0 + it.q0);
                tma_load_3d(smem_u32(to + L::kTileBytes), &tmap_do, bar(kQFull + (k & 1)), 0, it.head, it.node0 + it.q0);
            }
            const int kv_head = it.head / p.group;
            for (int s = 0; s < it.n_kv && good; ++s, ++c) {
                const int st = c % kDeltaStages;
                if (c >= kDeltaStages) good = wait(kKvEmpty + st, ((c / kDeltaStages) & 1) ^ 1, 401);
                if (good && lane == 0) {
                    uint8_t* to = smem + L::kK + st * L::kPair;
                    mbar_arrive_expect_tx(bar(kKvFull + st), L::kPair);
                    tma_load_3d(smem_u32(to), &tmap_k, bar(kKvFull + st), 0, kv_head, it.node0 + s * kTile);
                    tma_load_3d(smem_u32(to + L::kTileBytes), &tmap_v, bar(kKvFull + st), 0, kv_head, it.node0 + s * kTile);
                }
                __syncwarp();
            }
            ++k;
        }
    } else if (warp == 1) {
        constexpr uint32_t idesc = make_idesc_bf16(128, 128, false, false);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint64_t desc_q0 = make_smem_desc(smem_u32(smem + L::kQ), L::kRowBytes, 0), desc_k0 = make_smem_desc(smem_u32(smem + L::kK), L::kRowBytes, 0);
        int c = 0, k = 0;
        bool good = true;
        for (int turn = 0; good; ++turn) {
            const Item it = item_of(turn);
            if (it.head < 0) break;
            if (it.n_kv == 0) continue;
            good = wait(kQFull + (k & 1), (k >> 1) & 1, 410);
            const uint64_t dq = advance_desc(desc_q0, (k & 1) * L::kPair), ddo = advance_desc(dq, L::kTileBytes);
            for (int s = 0; s < it.n_kv && good; ++s, ++c) {
                const int st = c % kDeltaStages, b = c & 1;
                good = wait(kKvFull + st, (c / kDeltaStages) & 1, 411);
                if (good && c >= 2) good = wait(kRead + b, ((c >> 1) & 1) ^ 1, 412);
                if (!good) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t dk = advance_desc(desc_k0, st * L::kPair), dv = advance_desc(dk, L::kTileBytes);
#pragma unroll
                    for (int e = 0; e < D / 16; ++e) mma_ss(tm + b * 256, advance_desc(dq, e * 32), advance_desc(dk, e * 32), idesc, e > 0);
#pragma unroll
                    for (int e = 0; e < D / 16; ++e) mma_ss(tm + b * 256 + 128, advance_desc(ddo, e * 32), advance_desc(dv, e * 32), idesc, e > 0);
                    mma_commit(bar(kKvEmpty + st));
                    mma_commit(bar(kScores + b));
                    if (s == it.n_kv - 1) mma_commit(bar(kQEmpty + (k & 1)));
                }
                __syncwarp();
            }
            ++k;
        }
    } else if (warp == 3) {
        int k = 0;
        for (int turn = 0;; ++turn) {
            const Item it = item_of(turn);
            if (it.head < 0) break;
            if (it.n_kv == 0) continue;
            // (an item may last as long as a document of millions of tokens does)
            if (!__all_sync(0xffffffffu, item_wait(bar(kSumsFull + (k & 1)), (k >> 1) & 1, abort_flag, p.status, 430))) break;
            for (int r = lane; r < 128; r += 32) {
                const float2* of = sums + (k & 1) * 512 + r;
                const float delta = (of[0].x + of[128].x + of[256].x + of[384].x) / (of[0].y + of[128].y + of[256].y + of[384].y);
                uint4 e = make_uint4(0u, 0u, 0u, 0u);
                fold_term(-delta, e.x, e.y);
                if (it.q0 + r < it.n) p.ext[2 * ((size_t)(it.node0 + it.q0 + r) * p.n_heads + it.head) + 1] = e;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kSumsEmpty + (k & 1)));
            ++k;
        }
    } else if (warp >= 4) {
        const int grp = (warp - 4) >> 2, r = ((warp & 3) << 5) | lane;
        const uint32_t t0 = tmem + grp * 32 + ((uint32_t)((warp & 3) * 32) << 16);
        const uint64_t c1c1 = both(p.c1);
        [[maybe_unused]] const uint64_t to_tanh2 = both(p.to_tanh), cap22 = both(p.cap2);
        int c = 0, k = 0;
        bool good = true;
        Item next = item_of(0);                              // (fetched an item ahead)
        for (int turn = 1; good; ++turn) {
            const Item it = next;
            if (it.head < 0) break;
            next = item_of(turn);
            if (it.n_kv == 0) continue;
            const int32_t q = it.q0 + r;                                                    // this thread's query
            const bool counts = q < it.n;
            const int32_t limit = counts ? row_limit(p.causal, q, it.prefix, it.n) : 0;
            const uint64_t shift = both(counts ? -kLog2e * p.lse[(size_t)it.head * p.n_total + it.node0 + q] : 0.f);
            [[maybe_unused]] const float slope2 = kSlope ? p.slopes[it.head] * kLog2e : 0.f;
            uint64_t sum = both(0.f), mass = sum;
            for (int s = 0; s < it.n_kv; ++s, ++c) {
                const uint32_t tS = t0 + (c & 1) * 256;
                const int32_t kv0 = s * kTile + grp * 32;
                const int valid = limit - kv0;                        // columns that this thread's row sees (may be <= 0)
                [[maybe_unused]] const float ahead = (float)(kv0 - q);
                good = wait(kScores + (c & 1), (c >> 1) & 1, 420);
                if (!good) break;
                tc_fence_after();
                // 16 columns' scores less lse, in log2 units, but for the penalty
                auto scores = [&](const uint32_t (&sr)[16], float (&x)[16]) {
                    float top = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const uint64_t raw = pack_u32x2(sr[i], sr[i + 1]);
                        if constexpr (kCap) {
                            const uint64_t y = mul_f32x2(raw, to_tanh2), yy = mul_f32x2(y, y);
                            float u0, u1;
                            unpack_f32x2(yy, u0, u1);
                            top = max3(top, u0, u1);
                            unpack_f32x2(fma_f32x2(mul_f32x2(y, tanh_ratio(yy)), cap22, shift), x[i], x[i + 1]);
                        } else {
                            unpack_f32x2(fma_f32x2(raw, c1c1, shift), x[i], x[i + 1]);
                        }
                    }
                    if constexpr (kCap)
                        if (__any_sync(0xffffffffu, counts && !(top <= kTanhReach))) {          // beyond the polynomial's reach
#pragma unroll
                            for (int i = 0; i < 16; i += 2) {
                                float y0, y1;
                                unpack_f32x2(mul_f32x2(pack_u32x2(sr[i], sr[i + 1]), to_tanh2), y0, y1);
                                unpack_f32x2(fma_f32x2(pack_f32x2(tanh_any(y0), tanh_any(y1)), cap22, shift), x[i], x[i + 1]);
                            }
                        }
                };
                auto add = [&](int at, float (&x)[16], const uint32_t (&dp)[16], auto rag) {
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        float d0 = __uint_as_float(dp[i]), d1 = __uint_as_float(dp[i + 1]);
                        if constexpr (kSlope) {
                            x[i] = fmaf(-slope2, fabsf(ahead + (float)(at + i)), x[i]);
                            x[i + 1] = fmaf(-slope2, fabsf(ahead + (float)(at + i + 1)), x[i + 1]);
                        }
                        if constexpr (decltype(rag)::value) {           // (what a row does not see has no say, whatever it is)
                            if (at + i >= valid) { x[i] = -INFINITY; d0 = 0.f; }
                            if (at + i + 1 >= valid) { x[i + 1] = -INFINITY; d1 = 0.f; }
                        }
                        const uint64_t pr = pack_f32x2(ex2_approx(x[i]), ex2_approx(x[i + 1]));
                        mass = add_f32x2(mass, pr);
                        sum = fma_f32x2(pr, pack_f32x2(d0, d1), sum);
                    }
                };
                auto read = [&]() {                                    // all that this warp wants of the tile is in registers
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(kRead + (c & 1)));
                };
                auto pass = [&](auto rag) {
                    uint32_t sr[16], d0[16], d1[16];
                    float x[16];
                    tmem_ld16(tS, sr);
                    tmem_wait_ld();
                    tmem_ld16(tS + 128, d0);
                    scores(sr, x);
                    tmem_wait_ld();
                    tmem_ld16(tS + 16, sr);
                    tmem_ld16(tS + 144, d1);
                    add(0, x, d0, rag);
                    tmem_wait_ld();
                    read();
                    scores(sr, x);
                    add(16, x, d1, rag);
                };
                if (!__any_sync(0xffffffffu, valid < 32)) pass(Tag<false>{});
                else if (__any_sync(0xffffffffu, valid > 0)) pass(Tag<true>{});
                else read();
            }
            if (!good) break;
            if (k >= 2 && !wait(kSumsEmpty + (k & 1), ((k >> 1) & 1) ^ 1, 421)) break;
            float a, b, d, e;
            unpack_f32x2(sum, a, b);
            unpack_f32x2(mass, d, e);
            sums[(k & 1) * 512 + grp * 128 + r] = make_float2(a + b, d + e);
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kSumsFull + (k & 1)));
            ++k;
        }
    }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag) __nanosleep(200000);                // let copies that may still be in flight land
    if (warp == 2) tmem_dealloc(tmem, 512);
}

template <int D, bool kCap, bool kSlope>
gt_status launch_delta(const CUtensorMap (&maps)[6], const DeltaParams& p, cudaStream_t s)
{
    auto kern = position_delta_kernel<D, kCap, kSlope>;
    static std::atomic<uint64_t> granted{0};
    const gt_status st = grant_smem(kern, granted, DeltaSmem<D>::kDynamic);
    if (st != GT_OK) return st;
    return launch_overlapped(kern, dim3((unsigned)std::min(p.n_items, sm_count())), kDeltaThreads, DeltaSmem<D>::kDynamic, s, maps[0], maps[1], maps[2], maps[3], p);
}

}  // namespace
}  // namespace gt
