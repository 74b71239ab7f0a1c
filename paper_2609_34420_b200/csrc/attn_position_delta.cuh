// The per-query term of the backward of attention over token sequences where the caller has no fp32 output,
//     Delta_i = sum_j P_ij (dout_i . v_j) / sum_j P_ij,
// from the probabilities in fp32.  dout_i . out_i with an output that was rounded to bf16, of probabilities that were rounded to bf16, is subtracted
// from nearly equal numbers in rows of few large probabilities: with scores of standard deviation 4, dq and dk were off by 0.5 to 0.8 %, now by
// 0.23 % (what the roundings of dS and of the results leave).  (The sum of the same probabilities below: a row with one key has Delta = dP.)
//
// A block has 128 queries of a head and walks over the key tiles that they see: S = Q K^T and dP = dO V^T go to tensor memory (128 columns each),
// eight warps read both, a row per thread and half of the columns per warp.  lse is known, so that there is no reference to look for and nothing
// to rescale.  Two blocks per SM: one's MMAs run while the other's exponentials do.  Bound by the special-function unit: one exponential per pair.
//
//   warp 0  TMA producer: Q and dO, then K and V through a 2-stage ring      warp 1  issues the MMAs      warps 4-11  probabilities and sums
#pragma once

#include "attn_position.cuh"

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
    const int4* list;        // as the main kernel's; entry = {document, block, first row, rows}
    int32_t n_graphs, n_total, n_heads, group, causal;
    int32_t by_work;         // without a list: the same block of all documents, then the next (else document after document)
    int32_t blocks;          // ... of the longest document
    float c1, to_tanh, cap2;
};

constexpr int kDeltaThreads = 384;
constexpr float kLargestTerm = 0x1.fdp127f;      // rounds to a finite bf16

__device__ __forceinline__ void split3_bf16(float v, uint32_t& w01, uint32_t& w2)
{
    const __nv_bfloat16 hi = __float2bfloat16_rn(v);
    const float r1 = v - __bfloat162float(hi);
    const __nv_bfloat16 mid = __float2bfloat16_rn(r1);
    const __nv_bfloat16 lo = __float2bfloat16_rn(r1 - __bfloat162float(mid));
    w01 = (uint32_t)__bfloat16_as_ushort(hi) | ((uint32_t)__bfloat16_as_ushort(mid) << 16);
    w2 = (uint32_t)__bfloat16_as_ushort(lo);
}

template <int D>
struct DeltaSmem {
    static constexpr int kRowBytes = D * 2, kTileBytes = 128 * kRowBytes;
    static constexpr int kQ = 0, kDo = kTileBytes;
    static constexpr int kK = 2 * kTileBytes, kV = kK + kTileBytes, kStage = 2 * kTileBytes;       // [2 stages] at stride kStage
    static constexpr int kSums = kK + 2 * kStage;                    // [2 halves][128 rows] {sum P dP, sum P}
    static constexpr int kBars = kSums + 2 * 128 * 8;
    static constexpr int kMisc = kBars + 8 * 8;
    static constexpr int kDynamic = kMisc + 16 + 1024;               // slack for the 1024-byte alignment
};

template <int D, bool kCap, bool kSlope>
__global__ void __launch_bounds__(kDeltaThreads, 2)
position_delta_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                      const __grid_constant__ CUtensorMap tmap_do, const DeltaParams p)
{
    using L = DeltaSmem<D>;
    constexpr int kTile = 128;
    enum { kQFull = 0, kKvFull = 1, kKvEmpty = 3, kScores = 5, kRead = 6 };        // kKv*: [2 stages]
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
        for (int i = 0; i < kRead; ++i) mbar_init(bar(i), 1);
        mbar_init(bar(kRead), 8);                            // one arrival per warp
        fence_mbar_init();
        prefetch_tensormap(&tmap_q);
        prefetch_tensormap(&tmap_k);
        prefetch_tensormap(&tmap_v);
        prefetch_tensormap(&tmap_do);
    }
    if (warp == 2) { tmem_alloc(smem_u32(&misc[0]), 256); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = misc[0];
    grid_wait();

    const int32_t head = (int32_t)(blockIdx.x % (uint32_t)p.n_heads), row = (int32_t)(blockIdx.x / (uint32_t)p.n_heads);
    int32_t g, block, node0, n;
    if (p.list) {
        const int4 entry = p.list[row];
        g = entry.x;
        block = entry.y;
        node0 = entry.z;
        n = entry.x < 0 ? 0 : entry.w;
    } else {
        block = p.by_work ? row / p.n_graphs : row % p.blocks;
        g = p.by_work ? row % p.n_graphs : row / p.blocks;
        node0 = p.cu_seqlens ? p.cu_seqlens[g] : 0;
        n = p.cu_seqlens ? p.cu_seqlens[g + 1] - node0 : p.n_total;
    }
    const int32_t n_tiles = (n + kTile - 1) / kTile;
    const bool exists = block < n_tiles;
    const int32_t prefix = exists && p.prefix ? p.prefix[g] : 0;
    const int32_t q_tile = p.causal ? n_tiles - 1 - block : block, q0 = q_tile * kTile;       // (causal: the longest first)
    const int32_t n_kv = !exists ? 0 : p.causal ? max(q_tile + 1, (min(n, prefix) + kTile - 1) / kTile) : n_tiles;

    if (warp == 0) {
        const int kv_head = head / p.group;
        bool good = n_kv > 0;                                // no wait has been given up
        if (good && lane == 0) {
            mbar_arrive_expect_tx(bar(kQFull), 2 * L::kTileBytes);
            tma_load_3d(smem_u32(smem + L::kQ), &tmap_q, bar(kQFull), 0, head, node0 + q0);
            tma_load_3d(smem_u32(smem + L::kDo), &tmap_do, bar(kQFull), 0, head, node0 + q0);
        }
        for (int s = 0; s < n_kv && good; ++s) {
            const int st = s & 1;
            if (s >= 2) good = __all_sync(0xffffffffu, mbar_wait(bar(kKvEmpty + st), ((s >> 1) & 1) ^ 1, abort_flag, p.status, 400));
            if (good && lane == 0) {
                mbar_arrive_expect_tx(bar(kKvFull + st), 2 * L::kTileBytes);
                tma_load_3d(smem_u32(smem + L::kK + st * L::kStage), &tmap_k, bar(kKvFull + st), 0, kv_head, node0 + s * kTile);
                tma_load_3d(smem_u32(smem + L::kV + st * L::kStage), &tmap_v, bar(kKvFull + st), 0, kv_head, node0 + s * kTile);
            }
            __syncwarp();
        }
    } else if (warp == 1) {
        constexpr uint32_t idesc = make_idesc_bf16(128, 128, false, false);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint64_t desc_q = make_smem_desc(smem_u32(smem + L::kQ), L::kRowBytes, 0), desc_do = make_smem_desc(smem_u32(smem + L::kDo), L::kRowBytes, 0);
        const uint64_t desc_k0 = make_smem_desc(smem_u32(smem + L::kK), L::kRowBytes, 0), desc_v0 = make_smem_desc(smem_u32(smem + L::kV), L::kRowBytes, 0);
        bool good = n_kv > 0 && __all_sync(0xffffffffu, mbar_wait(bar(kQFull), 0, abort_flag, p.status, 410));
        for (int s = 0; s < n_kv && good; ++s) {
            const int st = s & 1;
            good = __all_sync(0xffffffffu, mbar_wait(bar(kKvFull + st), (s >> 1) & 1, abort_flag, p.status, 411));
            if (good && s > 0) good = __all_sync(0xffffffffu, mbar_wait(bar(kRead), (s - 1) & 1, abort_flag, p.status, 412));
            if (!good) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t dk = advance_desc(desc_k0, st * L::kStage), dv = advance_desc(desc_v0, st * L::kStage);
#pragma unroll
                for (int e = 0; e < D / 16; ++e) mma_ss(tm, advance_desc(desc_q, e * 32), advance_desc(dk, e * 32), idesc, e > 0);
#pragma unroll
                for (int e = 0; e < D / 16; ++e) mma_ss(tm + 128, advance_desc(desc_do, e * 32), advance_desc(dv, e * 32), idesc, e > 0);
                mma_commit(bar(kKvEmpty + st));
                mma_commit(bar(kScores));
            }
            __syncwarp();
        }
    } else if (warp >= 4) {
        const int hf = (warp - 4) >> 2, r = ((warp & 3) << 5) | lane;
        const uint32_t tS = tmem + hf * 64 + ((uint32_t)((warp & 3) * 32) << 16), tDp = tS + 128;
        const int32_t q = q0 + r, limit = row_limit(p.causal, q, prefix, n);        // this thread's query
        const bool counts = exists && q < n;
        const float lse2 = counts ? p.lse[(size_t)head * p.n_total + node0 + q] * kLog2e : 0.f;
        [[maybe_unused]] const float slope2 = kSlope && exists ? p.slopes[head] * kLog2e : 0.f;
        const uint64_t c1c1 = both(p.c1), shift = both(-lse2);
        [[maybe_unused]] const uint64_t to_tanh2 = both(p.to_tanh), cap22 = both(p.cap2);
        uint64_t sum = both(0.f), mass = sum;
        for (int s = 0; s < n_kv; ++s) {
            if (!__all_sync(0xffffffffu, mbar_wait(bar(kScores), s & 1, abort_flag, p.status, 420))) break;
            tc_fence_after();
            const int32_t kv0 = s * kTile + hf * 64;
            const int valid = counts ? limit - kv0 : 0;       // columns that this thread's row sees (may be <= 0)
            [[maybe_unused]] const float ahead = (float)(kv0 - q);
            auto pass = [&](auto rag) {
#pragma unroll
                for (int c = 0; c < 64; c += 16) {
                    uint32_t sr[16], dp[16];
                    tmem_ld16(tS + c, sr);
                    tmem_ld16(tDp + c, dp);
                    tmem_wait_ld();
                    [[maybe_unused]] bool far = false;        // a score beyond the reach of tanh's polynomial
                    if constexpr (kCap) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float y = __uint_as_float(sr[i]) * p.to_tanh;
                            if (!decltype(rag)::value || c + i < valid) far |= !(y * y <= kTanhReach);
                        }
                        far = __any_sync(0xffffffffu, far && counts);
                    }
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const uint64_t raw = pack_u32x2(sr[i], sr[i + 1]);
                        uint64_t x;
                        if constexpr (kCap) {
                            const uint64_t y = mul_f32x2(raw, to_tanh2);
                            if (far) {
                                float y0, y1;
                                unpack_f32x2(y, y0, y1);
                                x = fma_f32x2(pack_f32x2(tanh_any(y0), tanh_any(y1)), cap22, shift);
                            } else {
                                x = fma_f32x2(mul_f32x2(y, tanh_ratio(mul_f32x2(y, y))), cap22, shift);
                            }
                        } else {
                            x = fma_f32x2(raw, c1c1, shift);
                        }
                        float lo, hi;
                        unpack_f32x2(x, lo, hi);
                        if constexpr (kSlope) {
                            lo = fmaf(-slope2, fabsf(ahead + (float)(c + i)), lo);
                            hi = fmaf(-slope2, fabsf(ahead + (float)(c + i + 1)), hi);
                        }
                        if constexpr (decltype(rag)::value) {           // (what a row does not see has no say, whatever it is)
                            if (c + i >= valid) { lo = -INFINITY; dp[i] = 0u; }
                            if (c + i + 1 >= valid) { hi = -INFINITY; dp[i + 1] = 0u; }
                        }
                        const uint64_t pr = pack_f32x2(ex2_approx(lo), ex2_approx(hi));
                        mass = add_f32x2(mass, pr);
                        sum = fma_f32x2(pr, pack_u32x2(dp[i], dp[i + 1]), sum);
                    }
                }
            };
            if (__any_sync(0xffffffffu, valid < 64)) {
                if (__any_sync(0xffffffffu, valid > 0)) pass(Tag<true>{});
            } else {
                pass(Tag<false>{});
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kRead));
        }
        float a, b, c, d;
        unpack_f32x2(sum, a, b);
        unpack_f32x2(mass, c, d);
        sums[hf * 128 + r] = make_float2(a + b, c + d);
    }

    tc_fence_before();
    __syncthreads();
    const bool given_up = *abort_flag != 0u;
    if (given_up) __nanosleep(200000);                   // let copies that may still be in flight land
    if (warp == 2) tmem_dealloc(tmem, 256);
    if (tid < 128 && q0 + tid < n && n_kv > 0 && !given_up) {
        const float2 x = sums[tid], y = sums[128 + tid];
        const float delta = (x.x + y.x) / (x.y + y.y);
        uint4 e = make_uint4(0u, 0u, 0u, 0u);
        if (fabsf(delta) < kLargestTerm) split3_bf16(-delta, e.x, e.y);       // (a NaN, too, would reach the rows that share a tile)
        p.ext[2 * ((size_t)(node0 + q0 + tid) * p.n_heads + head) + 1] = e;
    }
}

template <int D, bool kCap, bool kSlope>
gt_status launch_delta(const CUtensorMap (&maps)[6], const DeltaParams& p, unsigned blocks, cudaStream_t s)
{
    auto kern = position_delta_kernel<D, kCap, kSlope>;
    static std::atomic<uint64_t> granted{0};
    const gt_status st = grant_smem(kern, granted, DeltaSmem<D>::kDynamic);
    if (st != GT_OK) return st;
    return launch_overlapped(kern, dim3(blocks), kDeltaThreads, DeltaSmem<D>::kDynamic, s, maps[0], maps[1], maps[2], maps[3], p);
}

}  // namespace
}  // namespace gt
