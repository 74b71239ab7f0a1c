// gt_position_attn_bwd: gradient of attention over packed token sequences with respect to q, k and v (formulas: the header).
//
// An item of work is one query head and one tile of 128 keys, for which a CTA walks over the query tiles that see any of them.  The grid
// is persistent: a CTA takes one item after the other, and its warps run through them as through one long row of query tiles, so that the
// next item's rows arrive, and its first scores are made, while the last one's dK and dV are written.  Scores are recomputed
// TRANSPOSED (S^T = K Q^T, thread = key = TMEM lane), so that P^T and dS^T can go straight back to tensor memory as the A operands of
// dV += P^T dO and dK += dS^T Q; dS^T is also written to shared memory (MN-major A operand) for dQ_i = dS K, which is added to an fp32
// accumulator in global memory.  A mask is a range of queries for every key, so a thread compares column numbers with two bounds.
//
// The per-query terms are folded into the MMAs: a pre-pass (without the forward's fp32 output another one, attn_position_delta.cuh, for Delta) writes for
// every (query, head) a row of 16 bf16 with -lse sqrt(d) and -Delta, each split into three bf16 terms (24 mantissa bits); one extra K = 16 step against a constant tile of ones adds them.  With
// capped scores the tanh comes between the product and lse, so that only Delta is folded and lse is read from shared memory.
//
// A query tile is two halves of 64 queries with a TMEM stage, MMAs and barriers of their own; while one half's MMAs run, the other
// half's warps compute.  Three helper warps issue the MMAs; each accumulator and each part of a TMEM stage belongs to one of them, so
// every reuse of tensor memory follows, in that thread's issue order, the MMA that reads the old contents.
//
//   warp 0        fetches the items; TMA producer: K and V of an item; Q_i, dO_i and the per-query rows through a 2-stage ring
//   warps 1, 3, 2 MMA issuers: dV and the next S^T; dK and the next dP^T; dQ (which also clears what lies behind the document)
//   warps 4-19    softmax: warps 4-11 own queries [0,64) of every tile, warps 12-19 queries [64,128); within a half, four warps per 32
//                 query columns
//   warps 20-23   dQ reducer: TMEM -> shared memory -> TMA reduce-add into the fp32 accumulator; dV and dK of an item
//
// TMEM columns, half g: S^T/P^T [128g, 128g+64)  dP^T/dS^T [128g+64, 128g+128);
//               dV [256,320)  dK [320,384)  dQ [384,448)  K [448,480)  V [480,512) (bf16 pairs).
#include <math.h>

#include <algorithm>
#include <cmath>

#include "attn_position.cuh"
#include "attn_position_delta.cuh"
#include "attn_terms.cuh"

namespace gt {
namespace {

using namespace sm100;
using namespace position;

constexpr int kTile = 128;
constexpr int kHalf = 64;                   // queries per TMEM stage
constexpr int kStages = 2;
constexpr int kThreads = 768;
constexpr int kSoftmaxWarps = 16;
constexpr int kExtCols = 16;                // bf16 per (query, head) row of folded terms
constexpr int kExtTileBytes = kTile * kExtCols * 2;

struct PositionBwdParams {
    const int32_t* cu_seqlens;
    const int32_t* prefix;
    const float* slopes;
    const float* lse;        // [H,T]
    __nv_bfloat16* dk;
    __nv_bfloat16* dv;
    int64_t dk_row, dv_row;  // elements from a row to the next
    float* dk_acc;           // [T,G,D] fp32 (workspace, zeroed) where several items add to a key's row, else nullptr
    float* dv_acc;
    uint32_t* status;
    uint32_t* next_item;     // counts the items that have been taken beyond the grid's first ones; 0 before and after the kernel
    const int4* list;        // packed batch: work list; item = entry * heads + head (nullptr: heads, then documents and tiles)
    int32_t n_items;
    int32_t parts;           // without a list: items that share the queries of a key tile (then dk_acc and dv_acc are used)
    int32_t by_work;         // without a list: the same tile of all documents, then the next (else document after document)
    int32_t blocks;          // ... of the longest document
    int32_t n_graphs;
    int32_t n_total;
    int32_t n_heads;
    int32_t group;           // query heads per key head
    int32_t causal;
    int32_t whole;           // rows of dk and dv begin at whole sectors
    int32_t early_release;   // let the next kernel start its set-up while this one runs
    float c1;                // log2(e) / sqrt(d)
    float ds_scale;          // of dk and dq: 1 / sqrt(d), with a cap its negative
    float to_tanh;           // 1 / (sqrt(d) cap)
    float cap2;              // cap log2(e)
};

enum Barrier {
    kBarItemFull = 0,                        // [2]  an item's description
    kBarItemEmpty = kBarItemFull + 2,        // [2]  all warps that work on it are done with it
    kBarKFull = kBarItemEmpty + 2,           // [2]  K of an item
    kBarKEmpty = kBarKFull + 2,              // [2]  commit behind the item's last dQ MMA
    kBarVFull = kBarKEmpty + 2,              //      V of an item
    kBarVEmpty,                              //      4 warp arrivals, V rows copied to tensor memory; commit behind the item's first dP^T MMAs
    kBarQdoFull,                             // [2]  Q_i, dO_i and the per-query rows of tile i
    kBarStageEmpty = kBarQdoFull + kStages,  // [2]  commits behind the last MMAs that read Q_i / dO_i
    kBarSFull = kBarStageEmpty + kStages,    // [2]  per half: S^T of the next tile is in tensor memory
    kBarDpFull = kBarSFull + 2,              // [2]  per half: dP^T of the next tile
    kBarPReady = kBarDpFull + 2,             // [2]  per half: 8 warp arrivals, P^T stored
    kBarDsReady = kBarPReady + 2,            // [2]  per half: 8 warp arrivals, dS^T stored (tensor and shared memory)
    kBarDqFull = kBarDsReady + 2,
    kBarDqFree,
    kBarKvTmem,                              //      8 warp arrivals: K and V rows copied to tensor memory
    kBarKvDone,                              //      commits behind the item's last S^T and dP^T MMAs, which read them there
    kBarQClear,                              //      the rows of a Q and a dO tile behind the document are cleared
    kBarFinal,                               //      dV and dK of an item
    kBarAccFree,                             //      4 warp arrivals: they have been read
    kNumBarriers
};
constexpr int kNbDqStaged = 4, kNbDqStagingFree = 5, kNbDqItem = 6;       // named barriers

template <int D>
struct Smem {
    static constexpr int kRowBytes = D * 2;
    static constexpr int kTileBytes = 128 * kRowBytes;
    static constexpr int kK = 0;                                    // [2 items]
    static constexpr int kV = kK + 2 * kTileBytes;
    static constexpr int kOnes = kV + kTileBytes;                   // two constant groups of 8 x 16 bf16 (256 B each)
    static constexpr int kStageBytes = 2 * kTileBytes;              // Q_i then dO_i
    static constexpr int kQ = kOnes + 1024;                         // [kStages] at stride kStageBytes
    static constexpr int kDo = kQ + kTileBytes;                     // [kStages] at stride kStageBytes
    static constexpr int kExt = kQ + kStages * kStageBytes;         // [kStages] per-query rows
    static constexpr int kStg = kExt + kStages * kExtTileBytes;     // dQ staging, two buffers of 128 rows x 32 floats
    static constexpr int kDs = kStg + 2 * 16384;                    // dS^T: 2 atoms x 128 rows x 128 bytes
    static constexpr int kLse = kDs + 32768;                        // [softmax warps][32] float
    static constexpr int kItems = kLse + kSoftmaxWarps * 128;       // [2] Item
    static constexpr int kBars = kItems + 2 * 32;
    static constexpr int kMisc = kBars + (kNumBarriers + 1) / 2 * 16;
    static constexpr int kDynamic = kMisc + 16 + 1024;              // slack for the 1024-byte alignment
    static_assert(kOnes % 1024 == 0 && kQ % 1024 == 0 && kExt % 1024 == 0 && kStg % 1024 == 0 && kDs % 1024 == 0 && kLse % 16 == 0 &&
                  kItems % 16 == 0 && kBars % 16 == 0 && kMisc % 16 == 0 && kDynamic <= 227 * 1024, "aligned, and within an SM");
};

struct alignas(16) Item {
    int32_t node0, n, head, kv0;           // n = 0: there are no more
    int32_t prefix, q_lo, q_hi, pad;       // queries [q_lo, q_hi): those that see a key of the tile, in whole tiles, or a part of them
    __device__ __forceinline__ int32_t q_tiles() const { return (q_hi - q_lo + kTile - 1) / kTile; }
    // rows of the last query tile, and of the key tile, that are the document's, if rows of another one follow in it, else 0
    __device__ __forceinline__ int32_t ragged(int32_t n_total) const { return q_hi == n && node0 + n < n_total ? n % kTile : 0; }
    __device__ __forceinline__ int32_t ragged_keys(int32_t n_total) const { return kv0 + kTile > n && node0 + n < n_total ? n % kTile : 0; }
};

// register budget: the CTA is launched with 768 x 80 registers; after the re-split it holds
// 128 x 48 + 512 x 96 + 128 x 48 = 61440 (an increase can only draw on what the CTA owns)
__device__ __forceinline__ void setmaxnreg_inc_96() { asm volatile("setmaxnreg.inc.sync.aligned.u32 96;"); }
__device__ __forceinline__ void setmaxnreg_dec_48() { asm volatile("setmaxnreg.dec.sync.aligned.u32 48;"); }

template <int D, bool kCap, bool kSlope>
__global__ void __launch_bounds__(kThreads, 1)
position_bwd_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                    const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ CUtensorMap tmap_do,
                    const __grid_constant__ CUtensorMap tmap_ext, const __grid_constant__ CUtensorMap tmap_dq,
                    const PositionBwdParams p)
{
    using L = Smem<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint64_t* bars = (uint64_t*)(smem + L::kBars);
    uint32_t* misc = (uint32_t*)(smem + L::kMisc);
    Item* items = (Item*)(smem + L::kItems);
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    volatile uint32_t* abort_flag = &misc[1];
    if (tid == 0) {
        misc[1] = 0u;
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(kBarItemFull + s), 1);
            mbar_init(bar(kBarItemEmpty + s), 3 + kSoftmaxWarps + 4);
            mbar_init(bar(kBarKFull + s), 1);
            mbar_init(bar(kBarKEmpty + s), 1);
            mbar_init(bar(kBarQdoFull + s), 1);
            mbar_init(bar(kBarStageEmpty + s), 2);
            mbar_init(bar(kBarSFull + s), 1);
            mbar_init(bar(kBarDpFull + s), 1);
            mbar_init(bar(kBarPReady + s), kSoftmaxWarps / 2);       // one arrival per warp
            mbar_init(bar(kBarDsReady + s), kSoftmaxWarps / 2);
        }
        mbar_init(bar(kBarVFull), 1);
        mbar_init(bar(kBarVEmpty), 5);
        mbar_init(bar(kBarDqFull), 1);
        mbar_init(bar(kBarDqFree), 4);
        mbar_init(bar(kBarKvTmem), 8);
        mbar_init(bar(kBarKvDone), 2);
        mbar_init(bar(kBarQClear), 1);
        mbar_init(bar(kBarFinal), 2);
        mbar_init(bar(kBarAccFree), 4);
        fence_mbar_init();
        prefetch_tensormap(&tmap_q);
        prefetch_tensormap(&tmap_k);
        prefetch_tensormap(&tmap_v);
        prefetch_tensormap(&tmap_do);
        prefetch_tensormap(&tmap_ext);
        prefetch_tensormap(&tmap_dq);
    }
    if (warp == 2) { tmem_alloc(smem_u32(&misc[0]), 512); tmem_relinquish(); }
    if (tid < 32) {
        // 8 rows x 32 bytes per group in the 32-byte swizzle: the 16-byte half that holds columns 0..7 sits
        // first in rows 0-3 and second in rows 4-7.  Group 0: ones in columns 0..2 (multiplies the -lse terms),
        // group 1: ones in columns 8..10 (the -Delta terms).
        const int grp_ = tid >> 4, row = (tid >> 1) & 7, phys_half = tid & 1;
        const int logical_half = phys_half ^ (row >> 2);
        const bool has_ones = logical_half == grp_;
        *(uint4*)(smem + L::kOnes + tid * 16) = has_ones ? make_uint4(0x3f803f80u, 0x00003f80u, 0u, 0u) : make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async_smem();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = misc[0];
    grid_wait();
    if (p.early_release) grid_release();
    constexpr uint32_t kColDv = 256, kColDk = 320, kColDq = 384, kColK = 448, kColV = 480;

    // Item number k of this CTA; false: there are no more.  give_back: the calling warp is done with its description.
    auto take = [&](int k) -> bool {
        const bool had = item_wait(bar(kBarItemFull + (k & 1)), (k >> 1) & 1, abort_flag, p.status, 300);
        return goes_on(had, items[k & 1].n, abort_flag, warp_any);
    };
    auto give_back = [&](int k) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kBarItemEmpty + (k & 1)));
    };

    if (warp < 4) {
        setmaxnreg_dec_48();
        if (warp == 0) {
            // ------------------------------ items and TMA producer ------------------------------
            // The CTA's own number, then what the counter gives, as late as can be: when the last rows of the item before are on their way.
            int32_t index = (int32_t)blockIdx.x;
            int c = 0;                                       // query tiles so far
            bool good = true;                                // no wait has been given up (then the items are only counted to their end)
            for (int k = 0;; ++k) {
                Item item{};
                while (item.n == 0) {
                    if (index < 0) {
                        uint32_t taken = (uint32_t)p.n_items;
                        if (lane == 0 && (int32_t)gridDim.x < p.n_items) {
                            taken = atomicAdd(p.next_item, 1u);
                            // every item beyond the first ones is counted once, and every CTA's vain attempt: the last one leaves 0
                            if (taken == (uint32_t)p.n_items - 1u) *p.next_item = 0u;
                        }
                        index = (int32_t)(gridDim.x + __shfl_sync(0xffffffffu, taken, 0));
                    }
                    if (index >= p.n_items) break;
                    int32_t g, tile, part = 0;
                    if (p.list) {
                        const int4 entry = p.list[index / p.n_heads];
                        g = entry.x;
                        tile = entry.y;
                        item.node0 = entry.z;
                        item.n = entry.x < 0 ? 0 : entry.w;
                    } else {
                        int32_t row = index / p.n_heads;
                        part = row % p.parts;
                        row /= p.parts;
                        tile = p.by_work ? row / p.n_graphs : row % p.blocks;
                        g = p.by_work ? row % p.n_graphs : row / p.blocks;
                        item.node0 = p.cu_seqlens ? p.cu_seqlens[g] : 0;
                        item.n = p.cu_seqlens ? p.cu_seqlens[g + 1] - item.node0 : p.n_total;
                    }
                    item.head = index % p.n_heads;
                    index = -1;
                    item.kv0 = tile * kTile;
                    if (item.kv0 >= item.n) {
                        item.n = 0;
                    } else {
                        item.prefix = p.prefix ? p.prefix[g] : 0;
                        item.q_lo = p.causal && item.kv0 >= item.prefix ? item.kv0 : 0;
                        item.q_hi = item.n;
                        if (p.parts > 1) {
                            const int32_t each = (item.q_tiles() + p.parts - 1) / p.parts * kTile;
                            item.q_lo += part * each;
                            item.q_hi = min(item.n, item.q_lo + each);
                            if (item.q_lo >= item.n) item.n = 0;
                        }
                    }
                }
                if (k >= 2 && good) good = !warp_any(!item_wait(bar(kBarItemEmpty + (k & 1)), ((k >> 1) & 1) ^ 1, abort_flag, p.status, 301));
                if (good && lane == 0) {
                    items[k & 1] = item;
                    mbar_arrive(bar(kBarItemFull + (k & 1)));
                }
                __syncwarp();
                if (item.n == 0) break;
                if (!good) continue;
                const int kv_head = item.head / p.group;
                auto wait = [&](int i, uint32_t parity, uint32_t site) { good = good && !warp_any(!mbar_wait(bar(i), parity, abort_flag, p.status, site)); };
                if (k >= 2) wait(kBarKEmpty + (k & 1), ((k >> 1) & 1) ^ 1, 302);
                if (good && lane == 0) {
                    mbar_arrive_expect_tx(bar(kBarKFull + (k & 1)), L::kTileBytes);
                    tma_load_3d(smem_u32(smem + L::kK + (k & 1) * L::kTileBytes), &tmap_k, bar(kBarKFull + (k & 1)), 0, kv_head, item.node0 + item.kv0);
                }
                if (k >= 1) wait(kBarVEmpty, (k - 1) & 1, 303);
                if (good && lane == 0) {
                    mbar_arrive_expect_tx(bar(kBarVFull), L::kTileBytes);
                    tma_load_3d(smem_u32(smem + L::kV), &tmap_v, bar(kBarVFull), 0, kv_head, item.node0 + item.kv0);
                }
                const int n_q = item.q_tiles();
                for (int i = 0; i < n_q; ++i, ++c) {
                    const int s = c & 1;
                    if (c >= 2) wait(kBarStageEmpty + s, ((c >> 1) & 1) ^ 1, 310);
                    if (good && lane == 0) {
                        const int32_t row = item.node0 + item.q_lo + i * kTile;
                        mbar_arrive_expect_tx(bar(kBarQdoFull + s), 2 * L::kTileBytes + kExtTileBytes);
                        tma_load_3d(smem_u32(smem + L::kQ + s * L::kStageBytes), &tmap_q, bar(kBarQdoFull + s), 0, item.head, row);
                        tma_load_3d(smem_u32(smem + L::kDo + s * L::kStageBytes), &tmap_do, bar(kBarQdoFull + s), 0, item.head, row);
                        tma_load_3d(smem_u32(smem + L::kExt + s * kExtTileBytes), &tmap_ext, bar(kBarQdoFull + s), 0, item.head, row);
                    }
                    __syncwarp();
                }
            }
        } else if (warp == 1 || warp == 3) {
            // ------------------------------- MMA issuers -------------------------------
            // warp 1: on "P^T(i) of a half stored": dV += P^T dO_i, then S^T of the next tile over the P^T just read
            // warp 3: on "dS^T(i) of a half stored": dK += dS^T Q_i, then dP^T of the next tile over that dS^T
            const bool on_p = warp == 1;
            constexpr uint32_t idesc_in = make_idesc_bf16(128, kHalf, false, false);   // S^T, dP^T of 64 queries
            constexpr uint32_t idesc_ts = make_idesc_bf16(128, D, false, true);        // A in TMEM, B MN-major
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
            // constant A operand of the extra K step: every 8-row group reads the same 256 bytes (group stride 0)
            const uint64_t desc_ones = make_smem_desc_stride(smem_u32(smem + L::kOnes + (on_p ? 0 : 256)), kExtCols * 2, 0, 0);
            const int acc_b_off = on_p ? L::kDo : L::kQ;       // B of the accumulating MMA: dO_i (dV) / Q_i (dK)
            const int in_b_off = on_p ? L::kQ : L::kDo;        // B of the next input MMA:   Q (S^T)  / dO (dP^T)
            const uint32_t acc_col = on_p ? kColDv : kColDk;
            const uint32_t reg_off = on_p ? 0 : kHalf;          // S^T/P^T or dP^T/dS^T part of a TMEM stage
            const uint32_t in_a_col = on_p ? kColK : kColV;
            const int bar_ready = on_p ? kBarPReady : kBarDsReady, bar_full = on_p ? kBarSFull : kBarDpFull;
            // (S^T - lse sqrt(d)) or (dP^T - Delta) of a half tile.  An item's first tile takes K and V from shared memory: it can go while the
            // softmax warps are still at the item before.
            auto issue_input = [&](int c, int sub, int k, bool begins) {
                const int s = c & 1;
                const uint64_t db = make_smem_desc(smem_u32(smem + in_b_off + s * L::kStageBytes) + sub * kHalf * L::kRowBytes, L::kRowBytes, 0);
                const uint64_t dext = make_smem_desc(smem_u32(smem + L::kExt + s * kExtTileBytes) + sub * kHalf * kExtCols * 2, kExtCols * 2, 0);
                const uint32_t d = tm + sub * 128 + reg_off;
                if (begins) {
                    const uint64_t da = make_smem_desc(smem_u32(smem + (on_p ? L::kK + (k & 1) * L::kTileBytes : L::kV)), L::kRowBytes, 0);
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) mma_ss(d, advance_desc(da, ks * 32), advance_desc(db, ks * 32), idesc_in, ks > 0);
                } else {
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks)         // A = K or V from tensor memory: 8 packed columns per K step
                        mma_ts(d, tm + in_a_col + ks * 8, advance_desc(db, ks * 32), idesc_in, ks > 0);
                }
                if (!kCap || !on_p) mma_ss(d, desc_ones, dext, idesc_in, 1u);
                mma_commit(bar(bar_full + sub));
            };
            int c = 0, cleared = 0;                             // query tiles, and ragged ones, so far
            for (int k = 0; take(k); ++k) {
                const int n_q = items[k & 1].q_tiles();
                const bool ragged = items[k & 1].ragged(p.n_total) != 0;
                give_back(k);
                auto wait_tile = [&](int i) {
                    mbar_wait(bar(kBarQdoFull + ((c + i) & 1)), ((c + i) >> 1) & 1, abort_flag, p.status, 321);
                    if (ragged && i == n_q - 1) mbar_wait(bar(kBarQClear), cleared & 1, abort_flag, p.status, 322);
                };
                if (on_p) mbar_wait(bar(kBarKFull + (k & 1)), (k >> 1) & 1, abort_flag, p.status, 325);
                else mbar_wait(bar(kBarVFull), k & 1, abort_flag, p.status, 326);
                wait_tile(0);
                tc_fence_after();
                if (elect_one()) {
                    issue_input(c, 0, k, true);
                    issue_input(c, 1, k, true);
                    if (!on_p) mma_commit(bar(kBarVEmpty));
                }
                __syncwarp();
                mbar_wait(bar(kBarKvTmem), k & 1, abort_flag, p.status, 320);
                if (n_q == 1 && elect_one()) mma_commit(bar(kBarKvDone));
                __syncwarp();
                if (k > 0) mbar_wait(bar(kBarAccFree), (k - 1) & 1, abort_flag, p.status, 324);
                bool acc_started = false;           // the first MMA into the accumulator overwrites it
                for (int i = 0; i < n_q; ++i) {
                    const int s = (c + i) & 1;
                    if (i + 1 < n_q) wait_tile(i + 1);
#pragma unroll
                    for (int sub = 0; sub < 2; ++sub) {
                        mbar_wait(bar(bar_ready + sub), (c + i) & 1, abort_flag, p.status, 323);
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t t_a = tm + sub * 128 + reg_off;
                            const uint64_t db = make_smem_desc(smem_u32(smem + acc_b_off + s * L::kStageBytes) + sub * kHalf * L::kRowBytes, L::kRowBytes, 0);
#pragma unroll
                            for (int ks = 0; ks < kHalf / 16; ++ks)     // A: bf16 pairs of query group ks/2 at the start of its 32 columns
                                mma_ts(tm + acc_col, t_a + (ks >> 1) * 32 + (ks & 1) * 8,
                                       advance_desc(db, ks * 16 * L::kRowBytes), idesc_ts, (acc_started || ks > 0) ? 1u : 0u);
                            if (sub == 1) {
                                mma_commit(bar(kBarStageEmpty + s));    // this issuer's reads of Q_i / dO_i are done (the other one commits too)
                                if (i + 1 == n_q) mma_commit(bar(kBarFinal));
                            }
                            if (i + 1 < n_q) issue_input(c + i + 1, sub, k, false);
                            if (i + 2 == n_q && sub == 1) mma_commit(bar(kBarKvDone));
                        }
                        __syncwarp();
                        acc_started = true;
                    }
                }
                c += n_q;
                cleared += ragged ? 1 : 0;
            }
        } else {
            // ------------------- dQ issuer; clears what lies behind the document in K, Q and dO -------------------
            constexpr uint32_t idesc_dq = make_idesc_bf16(128, D, true, true);         // A and B MN-major
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
            const uint64_t da = make_smem_desc(smem_u32(smem + L::kDs), 128, 16384);
            int c = 0;
            for (int k = 0; take(k); ++k) {
                const int n_q = items[k & 1].q_tiles();
                const int q_rows = items[k & 1].ragged(p.n_total), k_rows = items[k & 1].ragged_keys(p.n_total);
                give_back(k);
                uint8_t* const s_k = smem + L::kK + (k & 1) * L::kTileBytes;
                const uint64_t desc_k = make_smem_desc(smem_u32(s_k), L::kRowBytes, 0);
                mbar_wait(bar(kBarKFull + (k & 1)), (k >> 1) & 1, abort_flag, p.status, 330);
                if (k_rows != 0) clear_rows(s_k, k_rows, L::kRowBytes);
                auto clear_tile = [&](int at) {                // tile number `at`, the item's last one, before any MMA reads it
                    mbar_wait(bar(kBarQdoFull + (at & 1)), (at >> 1) & 1, abort_flag, p.status, 331);
                    clear_rows(smem + L::kQ + (at & 1) * L::kStageBytes, q_rows, L::kRowBytes);
                    clear_rows(smem + L::kDo + (at & 1) * L::kStageBytes, q_rows, L::kRowBytes);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(kBarQClear));
                };
                fence_proxy_async_smem();
                __syncwarp();
                if (q_rows != 0 && n_q == 1) clear_tile(c);
                for (int i = 0; i < n_q; ++i, ++c) {
                    if (q_rows != 0 && i == n_q - 2) clear_tile(c + 1);
                    // dQ_i = dS K once both halves have stored dS^T(i) and the reducer has drained dQ_{i-1}
                    mbar_wait(bar(kBarDsReady + 0), c & 1, abort_flag, p.status, 332);
                    mbar_wait(bar(kBarDsReady + 1), c & 1, abort_flag, p.status, 333);
                    mbar_wait(bar(kBarDqFree), (c & 1) ^ 1, abort_flag, p.status, 334);
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            mma_ss(tm + kColDq, advance_desc(da, ks * 2048), advance_desc(desc_k, ks * 16 * L::kRowBytes), idesc_dq, ks > 0);
                        mma_commit(bar(kBarDqFull));
                        if (i + 1 == n_q) mma_commit(bar(kBarKEmpty + (k & 1)));
                    }
                    __syncwarp();
                }
            }
        }
    } else if (warp < 20) {
        // ================================ softmax warps ================================
        setmaxnreg_inc_96();
        const int half = (warp - 4) >> 3;               // query half of every tile = TMEM stage
        const int grp = (warp - 4) >> 2;                // query-column group: columns [32 grp, 32 grp + 32) of the tile
        const int r = ((warp & 3) << 5) | lane;         // key row within the tile = TMEM lane
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + half * 128 + (grp & 1) * 32 + lane_off;
        const uint32_t tDp = tS + kHalf;
        const uint64_t c1c1 = both(p.c1);
        [[maybe_unused]] const uint64_t to_tanh2 = both(p.to_tanh), cap22 = both(p.cap2);
        [[maybe_unused]] float* s_lse = (float*)(smem + L::kLse) + (warp - 4) * 32;
        uint8_t* ds_row = smem + L::kDs + half * 16384 + r * 128;

        // K (warps 4-7) and V (warps 8-11) rows of item k -> tensor memory, where they stay as the A operands of S^T = K Q^T and
        // dP^T = V dO^T, once all MMAs that read the last item's there are done
        auto copy_kv = [&](int k) {
            if (warp >= 12) return;
            if (k > 0) mbar_wait(bar(kBarKvDone), (k - 1) & 1, abort_flag, p.status, 345);
            if (warp < 8) mbar_wait(bar(kBarKFull + (k & 1)), (k >> 1) & 1, abort_flag, p.status, 344);
            else mbar_wait(bar(kBarVFull), k & 1, abort_flag, p.status, 346);
            tc_fence_after();
            const uint8_t* src = smem + (warp < 8 ? L::kK + (k & 1) * L::kTileBytes : L::kV) + r * L::kRowBytes;
            uint32_t w[D / 2];
#pragma unroll
            for (int e = 0; e < D / 8; ++e) {
                const int phys = D == 64 ? (e ^ (r & 7)) : (e ^ ((r >> 1) & 3));     // 128-byte / 64-byte swizzle
                const uint4 v4 = *(const uint4*)(src + (phys << 4));
                w[4 * e] = v4.x; w[4 * e + 1] = v4.y; w[4 * e + 2] = v4.z; w[4 * e + 3] = v4.w;
            }
            const uint32_t dst = tmem + (warp < 8 ? kColK : kColV) + lane_off;
            if constexpr (D == 64) tmem_st32(dst, w); else tmem_st16(dst, w);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (warp >= 8) mbar_arrive(bar(kBarVEmpty));
                mbar_arrive(bar(kBarKvTmem));
            }
        };

        int c = 0;                                      // query tiles so far
        for (int k = 0; take(k); ++k) {
        copy_kv(k);
        const int32_t n = items[k & 1].n, q_lo = items[k & 1].q_lo;
        const int32_t key = items[k & 1].kv0 + r, key0 = key - lane;                        // this thread's key, the warp's first one
        // queries [from, to) see the key
        [[maybe_unused]] const int32_t prefix = items[k & 1].prefix;
        const int32_t from = p.causal && key >= prefix ? key : 0, to = key < n ? n : 0;
        const int32_t last_from = p.causal && key0 + 31 >= prefix ? key0 + 31 : 0;               // largest `from` of the warp
        [[maybe_unused]] const float slope2 = kSlope ? p.slopes[items[k & 1].head] * kLog2e : 0.f;
        // (steep penalties: made for every element wherever a key's own query is, see kSteep)
        [[maybe_unused]] const bool linear = p.causal && key0 >= prefix && fabsf(slope2) <= kSteep;
        // lse of the warp's queries, a lane each, fetched a tile ahead
        [[maybe_unused]] const float* lse_row = p.lse + (size_t)items[k & 1].head * p.n_total + items[k & 1].node0;
        [[maybe_unused]] auto fetch_lse = [&](int i) -> float {
            const int32_t q = q_lo + i * kTile + grp * 32 + lane;
            return q < n ? -kLog2e * lse_row[q] : 0.f;
        };
        [[maybe_unused]] float next_lse = kCap ? fetch_lse(0) : 0.f;
        const int n_q = items[k & 1].q_tiles();
        give_back(k);

        for (int i = 0; i < n_q; ++i, ++c) {
            const int32_t q0 = q_lo + i * kTile + grp * 32;                     // the group's first query
            const bool masked = q0 < last_from || q0 + 32 > n || key0 + 32 > n;     // some pair of the warp's may not count
            // bit e: this thread's key is seen by the group's query e
            const uint32_t seen = (to - q0 >= 32 ? 0xffffffffu : to > q0 ? (1u << (to - q0)) - 1u : 0u) &
                                  (from - q0 >= 32 ? 0u : from > q0 ? 0xffffffffu << (from - q0) : 0xffffffffu);
            // Penalty on distance: linear in the column where all queries lie behind the keys (or masked ones before them do not matter) or
            // all before; else made for every element.
            const bool behind = q0 >= key0 + 31 || linear, before = q0 + 31 <= key0;
            [[maybe_unused]] const bool mixed = kSlope && !before && !behind;
            [[maybe_unused]] const float step_slope = behind ? -slope2 : slope2;
            if constexpr (kCap) {
                __syncwarp();
                s_lse[lane] = next_lse;
                if (i + 1 < n_q) next_lse = fetch_lse(i + 1);
                __syncwarp();
            }
            float pr[32];                            // P^T, then dS^T (capped scores: P^T (1 - tanh^2) in between)
            uint32_t pk[16];
            mbar_wait(bar(kBarSFull + half), c & 1, abort_flag, p.status, 340);
            tc_fence_after();

            // ---------------- P^T = exp2((S^T - lse sqrt(d)) c1), or exp2(cap log2(e) tanh(S^T / cap) - lse log2(e)) ----------------
            float top_u = 0.f;
            auto probabilities = [&](auto masked_, auto general) {        // general: any score, any distance
                uint32_t sa[16], sb[16];
                tmem_ld16(tS, sa);
                [[maybe_unused]] const float ahead = (float)(q0 - key);         // the first query's distance
                [[maybe_unused]] uint64_t away = pack_f32x2(step_slope * ahead, fmaf(step_slope, ahead, step_slope));
                auto chunk = [&](int rnd, const uint32_t (&sv)[16]) {
                    [[maybe_unused]] float4 nl;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const int e = rnd * 16 + i;
                        [[maybe_unused]] uint64_t add = both(0.f), t;
                        uint64_t x;
                        if constexpr (kCap) {
                            if (e % 4 == 0) nl = *(const float4*)(s_lse + e);
                            add = e % 4 == 0 ? pack_f32x2(nl.x, nl.y) : pack_f32x2(nl.z, nl.w);
                        }
                        if constexpr (kSlope && decltype(general)::value) {
                            add = add_f32x2(add, pack_f32x2(-slope2 * fabsf(ahead + (float)e), -slope2 * fabsf(ahead + (float)(e + 1))));
                        } else if constexpr (kSlope) {
                            if (e > 0) away = add_f32x2(away, both(2.0f * step_slope));
                            add = kCap ? add_f32x2(add, away) : away;
                        }
                        const uint64_t raw = pack_u32x2(sv[i], sv[i + 1]);
                        if constexpr (kCap) {
                            const uint64_t u = mul_f32x2(raw, to_tanh2);
                            float u0, u1;
                            if constexpr (decltype(general)::value) {
                                unpack_f32x2(u, u0, u1);
                                t = pack_f32x2(tanh_any(u0), tanh_any(u1));
                            } else {
                                const uint64_t uu = mul_f32x2(u, u);
                                unpack_f32x2(uu, u0, u1);
                                top_u = max3(top_u, u0, u1);
                                t = mul_f32x2(u, tanh_ratio(uu));
                            }
                            x = fma_f32x2(t, cap22, add);
                        } else if constexpr (kSlope) {
                            x = fma_f32x2(raw, c1c1, add);
                        } else {
                            x = mul_f32x2(raw, c1c1);
                        }
                        float lo, hi;
                        unpack_f32x2(x, lo, hi);
                        lo = ex2_approx(lo);
                        hi = ex2_approx(hi);
                        if constexpr (decltype(masked_)::value) {
                            if (!(seen & (1u << e))) lo = 0.f;
                            if (!(seen & (2u << e))) hi = 0.f;
                        }
                        pk[e >> 1] = pack_bf16x2(lo, hi);
                        if constexpr (kCap) {
                            // -P (1 - tanh^2): the sign goes into the scale of dq and dk
                            unpack_f32x2(mul_f32x2(pack_f32x2(lo, hi), fma_f32x2(t, t, both(-1.f))), pr[e], pr[e + 1]);
                        } else {
                            pr[e] = lo;
                            pr[e + 1] = hi;
                        }
                    }
                };
                if constexpr (!kCap) tmem_ld16(tS + 16, sb);
                tmem_wait_ld();
                if constexpr (kCap) tmem_ld16(tS + 16, sb);      // (fewer registers at a time)
                chunk(0, sa);
                if constexpr (kCap) tmem_wait_ld();
                chunk(1, sb);
            };
            if (mixed) probabilities(Tag<true>{}, Tag<true>{});
            else {
                if (masked) probabilities(Tag<true>{}, Tag<false>{});
                else probabilities(Tag<false>{}, Tag<false>{});
                if constexpr (kCap)
                    if (__any_sync(0xffffffffu, !(top_u <= kTanhReach))) probabilities(Tag<true>{}, Tag<true>{});
            }
            tmem_st16(tS, pk);                      // P^T of this group: 16 packed columns at the start of its range
            uint32_t dpa[16], dpb[16];
            mbar_wait(bar(kBarDpFull + half), c & 1, abort_flag, p.status, 341);
            tc_fence_after();
            tmem_ld16(tDp, dpa);
            tmem_ld16(tDp + 16, dpb);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarPReady + half));    // dV of this half and the next S^T can go
            tmem_wait_ld();

            // ---------------- dS^T = P^T o (dP^T - Delta) ----------------
            auto ds_round = [&](int rnd, const uint32_t (&dp)[16], auto foreign) {
#pragma unroll
                for (int k = 0; k < 16; k += 2) {
                    const int e = rnd * 16 + k;
                    float lo, hi;
                    unpack_f32x2(mul_f32x2(pack_f32x2(pr[e], pr[e + 1]), pack_u32x2(dp[k], dp[k + 1])), lo, hi);
                    if constexpr (decltype(foreign)::value) {      // (0 x NaN: dP of a row of V that is another document's)
                        if (key >= n) lo = hi = 0.f;
                    }
                    pk[e >> 1] = pack_bf16x2(lo, hi);
                }
            };
            if (key0 + 32 > n) {
                ds_round(0, dpa, Tag<true>{});
                ds_round(1, dpb, Tag<true>{});
            } else {
                ds_round(0, dpa, Tag<false>{});
                ds_round(1, dpb, Tag<false>{});
            }
            tmem_st16(tDp, pk);
            // dQ of the previous tile has read the dS^T tile in shared memory
            if (c > 0) mbar_wait(bar(kBarDqFull), (c - 1) & 1, abort_flag, p.status, 342);
#pragma unroll
            for (int c8 = 0; c8 < 4; ++c8)
                *(uint4*)(ds_row + ((((grp & 1) * 4 + c8) ^ (r & 7)) << 4)) = make_uint4(pk[4 * c8], pk[4 * c8 + 1], pk[4 * c8 + 2], pk[4 * c8 + 3]);
            tmem_wait_st();
            fence_proxy_async_smem();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarDsReady + half));
        }

        }
    } else {
        // ================================ dQ reducer ================================
        // dQ_i (fp32, 128 x D) goes TMEM -> registers -> one of two staging buffers in 128-byte-swizzled rows of 32 floats, and from there to
        // the fp32 accumulator with TMA reduce-add.  An SM's reduce engine moves about 19 bytes per clock, so a buffer is only waited for
        // when it comes round again.
        setmaxnreg_dec_48();
        const int r = ((warp & 3) << 5) | lane;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        int c = 0;
        for (int k = 0;; ++k) {
            const bool had = item_wait(bar(kBarItemFull + (k & 1)), (k >> 1) & 1, abort_flag, p.status, 304);
            if (!goes_on(had, items[k & 1].n, abort_flag, [&](bool x) { return named_barrier_or(kNbDqItem, 128, x); })) break;
            const int n_q = items[k & 1].q_tiles();
            const int32_t n_own = items[k & 1].n - items[k & 1].q_lo, row0 = items[k & 1].node0 + items[k & 1].q_lo, col0 = items[k & 1].head * D;
            for (int i = 0; i < n_q; ++i, ++c) {
                mbar_wait(bar(kBarDqFull), c & 1, abort_flag, p.status, 350);
                tc_fence_after();
                const bool own = i * kTile + r < n_own;             // rows behind the document get zeros, whatever K holds
#pragma unroll
                for (int e = 0; e < D / 32; ++e) {
                    uint8_t* stg = smem + L::kStg + ((c * (D / 32) + e) & 1) * 16384;
                    uint32_t o[32];
                    tmem_ld32(tmem + kColDq + e * 32 + lane_off, o);
                    tmem_wait_ld();
                    if (e == D / 32 - 1) { tc_fence_before(); __syncwarp(); if (lane == 0) mbar_arrive(bar(kBarDqFree)); }
                    if (warp == 20 && elect_one()) bulk_wait_group_read1();        // the reduce that last used this buffer has read it
                    named_barrier_sync(kNbDqStagingFree, 128);
                    uint8_t* row = stg + r * 128;
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        *(uint4*)(row + ((q ^ (r & 7)) << 4)) = own ? make_uint4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]) : make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async_smem();
                    named_barrier_sync(kNbDqStaged, 128);
                    if (warp == 20) {
                        if (elect_one()) {
                            tma_reduce_add_2d(&tmap_dq, smem_u32(stg), col0 + e * 32, row0 + i * kTile);
                            bulk_commit_group();
                        }
                        __syncwarp();
                    }
                }
            }
            // The item's dV and dK, from here, so that the softmax warps go on with the next one.
            const int32_t key = items[k & 1].kv0 + r, node = items[k & 1].node0 + key, kv_head = items[k & 1].head / p.group;
            const bool mine = key < items[k & 1].n;
            give_back(k);
            mbar_wait(bar(kBarFinal), k & 1, abort_flag, p.status, 343);
            tc_fence_after();
#pragma unroll
            for (int e = 0; e < 2 * D; e += 16) {
                uint32_t o[16];
                tmem_ld16(tmem + (e < D ? kColDv + e : kColDk + e - D) + lane_off, o);
                tmem_wait_ld();
                if (e == 2 * D - 16) { tc_fence_before(); __syncwarp(); if (lane == 0) mbar_arrive(bar(kBarAccFree)); }
                const int col = e < D ? e : e - D;
                if (mine && p.dk_acc != nullptr) {
                    float4* dst = (float4*)((e < D ? p.dv_acc : p.dk_acc) + ((size_t)node * (p.n_heads / p.group) + kv_head) * D + col);
#pragma unroll
                    for (int i = 0; i < 4; ++i) red_add_f32x4(dst + i, o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                } else if (mine) {
                    const float mul = e < D ? 1.0f : p.ds_scale;
                    __nv_bfloat16* row = e < D ? p.dv + (int64_t)node * p.dv_row : p.dk + (int64_t)node * p.dk_row;
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = pack_bf16x2(__uint_as_float(o[2 * i]) * mul, __uint_as_float(o[2 * i + 1]) * mul);
                    store_sector(row + kv_head * D + col, p.whole, w);
                }
                __syncwarp();
            }
        }
        if (warp == 20 && elect_one()) bulk_wait_group0();      // all adds have landed before the CTA retires
    }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag) __nanosleep(200000);
    if (warp == 2) tmem_dealloc(tmem, 512);
}

struct PrepareParams {
    const float* out_f32;      // the forward's output before its rounding; nullptr: another kernel writes -Delta
    const __nv_bfloat16* dout;
    const float* lse;
    uint4* ext;
    float4* acc;               // the fp32 accumulators, cleared
    int4* list;                // packed batch: work list of the main kernel, made by the last blocks
    const int32_t* cu_seqlens;
    size_t n_acc;              // float4s of them
    int32_t n_total, n_graphs, n_heads, by_work;
    uint32_t row_blocks;       // thread blocks that work on rows
    float sqrt_d;
};

// What the main kernel wants done before it, in one launch.  Row blocks: for every row (t, h), ext[t][h][0..2] = three-term bf16 split of
// -lse sqrt(d), ext[t][h][8..10] = that of -Delta, Delta = sum_c dO[t,h,c] O[t,h,c] (without the fp32 O: zeros, for position_delta_kernel), zeros elsewhere; and their share of the accumulators
// is cleared.  A thread owns a row and adds its products in channel order; the rows reach it through shared memory, because 32 lanes that each walk along a row of their own ask the L1 for every line eight
// times.  16-byte chunk c of row r lies at chunk c ^ (r & 7): eight neighbouring rows' chunks lie in different banks (D = 32: c ^ (r & 3)).
constexpr int kPrepareThreads = 256, kPrepareRows = 128;
template <int D>
__global__ void __launch_bounds__(kPrepareThreads) position_prepare_kernel(const PrepareParams p)
{
    constexpr int kChunks = D / 8, kSwz = kChunks - 1;
    __shared__ __align__(16) uint8_t s_do[kPrepareRows * 2 * D], s_o[kPrepareRows * 4 * D];
    grid_wait();
    grid_release();
    if (blockIdx.x >= p.row_blocks) {
        const int32_t w = (int32_t)((blockIdx.x - p.row_blocks) * (kPrepareThreads / 32) + (threadIdx.x >> 5));
        if (w < p.n_graphs) write_list<kTile>(p.list, p.n_total / kTile + p.n_graphs, p.cu_seqlens, p.n_graphs, w, p.by_work);
        return;
    }
    const size_t n_rows = (size_t)p.n_total * p.n_heads, row0 = (size_t)blockIdx.x * kPrepareRows;
    const int rows = (int)(row0 + kPrepareRows < n_rows ? kPrepareRows : n_rows - row0);
    auto stage = [&](uint8_t* dst, const void* src, auto chunks_) {
        constexpr int chunks = decltype(chunks_)::value ? 2 * kChunks : kChunks, kEach = kPrepareRows * chunks / kPrepareThreads;
        const uint4* from = (const uint4*)src + row0 * chunks;
        uint4 x[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = (int)threadIdx.x + i * kPrepareThreads;
            if (e < rows * chunks) x[i] = from[e];
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = (int)threadIdx.x + i * kPrepareThreads, r = e / chunks, c = e % chunks;
            if (e < rows * chunks) *(uint4*)(dst + r * chunks * 16 + ((c ^ (r & kSwz)) << 4)) = x[i];
        }
    };
    for (size_t i = (size_t)blockIdx.x * kPrepareThreads + threadIdx.x; i < p.n_acc; i += (size_t)p.row_blocks * kPrepareThreads)
        p.acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    const int r = (int)threadIdx.x;
    const size_t row = row0 + r;
    float acc = 0.f;
    if (p.out_f32 != nullptr) {
        stage(s_do, p.dout, Tag<false>{});
        stage(s_o, p.out_f32, Tag<true>{});
        __syncthreads();
        if (r >= rows) return;
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const uint4 b = *(const uint4*)(s_do + r * 2 * D + ((i ^ (r & kSwz)) << 4));
            const uint32_t bw[4] = {b.x, b.y, b.z, b.w};
            const float4 a0 = *(const float4*)(s_o + r * 4 * D + (((2 * i) ^ (r & kSwz)) << 4));
            const float4 a1 = *(const float4*)(s_o + r * 4 * D + (((2 * i + 1) ^ (r & kSwz)) << 4));
            const float a[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                acc += a[2 * k] * __uint_as_float(bw[k] << 16);
                acc += a[2 * k + 1] * __uint_as_float(bw[k] & 0xffff0000u);
            }
        }
    }
    if (r >= rows) return;
    uint4 e0 = make_uint4(0u, 0u, 0u, 0u), e1 = make_uint4(0u, 0u, 0u, 0u);
    fold_term(-p.lse[(row % p.n_heads) * p.n_total + row / p.n_heads] * p.sqrt_d, e0.x, e0.y);
    fold_term(-acc, e1.x, e1.y);
    p.ext[2 * row] = e0;
    p.ext[2 * row + 1] = e1;
}

struct FinishParams {
    const float4* acc[3];      // dq, and with shared key heads dk, dv
    __nv_bfloat16* to[3];
    int64_t row[3];            // elements from a row to the next
    float mul[3];
    uint32_t vecs[3];          // groups of four channels in a row
    const int32_t* cu_seqlens;
    int32_t n_total, n_graphs;
};

// The fp32 sums, scaled and rounded once; a tensor per blockIdx.y, four groups of four channels a thread.
constexpr int kFinishThreads = 256, kFinishEach = 4;
__global__ void __launch_bounds__(kFinishThreads) position_finish_kernel(const __grid_constant__ FinishParams p)
{
    grid_wait();
    grid_release();
    const int of = blockIdx.y;
    const uint32_t vecs = p.vecs[of];
    const uint64_t all = (uint64_t)p.n_total * vecs, end = p.cu_seqlens ? (uint64_t)p.cu_seqlens[p.n_graphs] * vecs : all;
    const uint64_t at = (uint64_t)blockIdx.x * (kFinishThreads * kFinishEach) + threadIdx.x;
    const float4* acc = p.acc[of];
    const float m = p.mul[of];
    float4 v[kFinishEach];
#pragma unroll
    for (int i = 0; i < kFinishEach; ++i)
        if (at + i * kFinishThreads < end) v[i] = __ldcs(acc + at + i * kFinishThreads);
#pragma unroll
    for (int i = 0; i < kFinishEach; ++i) {
        const uint64_t idx = at + i * kFinishThreads;
        if (idx >= end) continue;
        const uint64_t t = all >> 32 ? idx / vecs : (uint32_t)idx / vecs;
        *(uint2*)(p.to[of] + (int64_t)t * p.row[of] + 4 * (int64_t)(idx - t * vecs)) = make_uint2(pack_bf16x2(v[i].x * m, v[i].y * m), pack_bf16x2(v[i].z * m, v[i].w * m));
    }
}

struct Workspace {
    size_t list_off, ext_off, acc_off, kv_bytes, total;
};

Workspace workspace_of(const gt_batch* b, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim)
{
    Workspace w{};
    const size_t rows = (size_t)b->n_total * n_heads;
    w.list_off = kHeaderBytes;
    w.ext_off = w.list_off + list_bytes(b, kTile);
    w.acc_off = w.ext_off + align_up(rows * kExtCols * 2, 256);
    w.kv_bytes = (size_t)b->n_total * n_kv_heads * head_dim * sizeof(float);
    w.total = w.acc_off + align_up(rows * head_dim * sizeof(float) + 2 * w.kv_bytes, 256);
    return w;
}

// Items that share the queries of a key tile, where the longest one would hold up the rest: a query tile takes about 1.8 us, an item's fill
// and drain 2, sums of dk and dv in memory 4 and 6 for every million of their elements (where heads share keys there are such sums
// anyway).  One item -> this many, causal, 8 heads of 64 if not said otherwise: 4 096 tokens, 2 heads 59 -> 40 us, all pairs 61 -> 44;
// 3 000 tokens, all pairs 107 -> 92; 2 048 tokens 38.7 -> 38.0; but 4 096 tokens 65 -> 79 and 8 192 tokens 200 -> 226, which stay with one.
inline int32_t parts_of(const gt_batch* b, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, bool causal)
{
    const double tiles = (b->max_seqlen + kTile - 1) / kTile, m = (double)b->n_graphs * n_heads, sms = sm_count();
    const double sums = n_heads > n_kv_heads ? 1.0 : 4.0 + 6e-6 * b->n_total * n_kv_heads * head_dim;
    int32_t best = 1;
    double least = 1e30;
    for (int32_t parts = 1; parts <= 4 && parts <= tiles; parts *= 2) {
        const double longest = std::ceil(tiles / parts), all = m * tiles * (causal ? (tiles + 1) / 2 : tiles) / sms, waves = std::ceil(m * tiles * parts / sms);
        const double us = 1.8 * (causal ? std::max(longest, all) : std::max(all, waves * longest)) + 2.0 * waves + sums * (parts / 2);
        if (us < 0.95 * least) { least = us; best = parts; }
    }
    return best;
}

template <int D, bool kCap, bool kSlope>
gt_status launch(const CUtensorMap (&maps)[6], PositionBwdParams p, const gt_batch* batch, cudaStream_t s)
{
    auto kern = position_bwd_kernel<D, kCap, kSlope>;
    static std::atomic<uint64_t> granted{0};
    const gt_status st = grant_smem(kern, granted, Smem<D>::kDynamic);
    if (st != GT_OK) return st;
    const dim3 grid((unsigned)std::min(p.n_items, sm_count()));
    p.early_release = p.n_items <= sm_count();
    return launch_overlapped(kern, grid, kThreads, Smem<D>::kDynamic, s, maps[0], maps[1], maps[2], maps[3], maps[4], maps[5], p);
}

}  // namespace
}  // namespace gt

extern "C" size_t gt_position_attn_bwd_workspace(const gt_batch* batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim)
{
    if (gt::position::validate(batch, n_heads, n_kv_heads, head_dim, nullptr, 0, 0.f) != GT_OK) return 0;
    return gt::workspace_of(batch, n_heads, n_kv_heads, head_dim).total;
}

extern "C" gt_status gt_position_attn_bwd(const void* q, const void* k, const void* v, const void* out, const float* out_f32,
                                          const void* dout, const float* lse, const float* slopes, const int32_t* prefix,
                                          const gt_batch* batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                          const gt_row_strides* strides, int32_t causal, float cap,
                                          void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace gt;
    gt_status st = position::validate(batch, n_heads, n_kv_heads, head_dim, prefix, causal, cap);
    if (st != GT_OK) return st;
    if (!q || !k || !v || (!out && !out_f32) || !dout || !lse || !dq || !dk || !dv) return GT_ERR_INVALID_ARG;
    if (misaligned16(q) || misaligned16(k) || misaligned16(v) || misaligned16(out) || misaligned16(out_f32) || misaligned16(dout) || misaligned16(dq) || misaligned16(dk) ||
        misaligned16(dv))
        return GT_ERR_INVALID_ARG;
    const gt_row_strides given = strides ? *strides : gt_row_strides{};
    const int64_t in[6] = {given.q, given.k, given.v, given.dq, given.dk, given.dv};
    int64_t row[6];
    for (int i = 0; i < 6; ++i)
        if (!position::row_stride(in[i], i % 3 == 0 ? n_heads : n_kv_heads, head_dim, &row[i])) return GT_ERR_INVALID_ARG;
    const Workspace w = workspace_of(batch, n_heads, n_kv_heads, head_dim);
    if (workspace == nullptr || misaligned16(workspace) || workspace_bytes < w.total) return GT_ERR_WORKSPACE;
    if (sm_count() <= 0) return GT_ERR_NO_DEVICE;
    uint8_t* ws = (uint8_t*)workspace;
    const int32_t T = batch->n_total;
    float* dq_acc = (float*)(ws + w.acc_off);
    CUtensorMap maps[6];
    if ((st = encode_rows_map(&maps[0], q, T, n_heads, head_dim, row[0])) != GT_OK) return st;
    if ((st = encode_rows_map(&maps[1], k, T, n_kv_heads, head_dim, row[1])) != GT_OK) return st;
    if ((st = encode_rows_map(&maps[2], v, T, n_kv_heads, head_dim, row[2])) != GT_OK) return st;
    if ((st = encode_thd_map(&maps[3], dout, T, n_heads, head_dim)) != GT_OK) return st;
    if ((st = encode_thd_map(&maps[4], ws + w.ext_off, T, n_heads, kExtCols)) != GT_OK) return st;
    if ((st = encode_dq_map(&maps[5], dq_acc, T, n_heads, head_dim)) != GT_OK) return st;
    PositionBwdParams p{};
    p.cu_seqlens = batch->cu_seqlens;
    p.prefix = prefix;
    p.slopes = slopes;
    p.lse = lse;
    p.dk = (__nv_bfloat16*)dk;
    p.dv = (__nv_bfloat16*)dv;
    p.dk_row = row[4];
    p.dv_row = row[5];
    p.whole = position::whole_sectors(dk) && position::whole_sectors(dv) && row[4] % 16 == 0 && row[5] % 16 == 0;
    p.parts = batch->n_graphs > 1 && list_saves(batch, kTile, n_heads, 0) ? 1 : parts_of(batch, n_heads, n_kv_heads, head_dim, causal != 0);
    const bool sums = n_heads > n_kv_heads || p.parts > 1;
    if (sums) {
        p.dk_acc = dq_acc + (size_t)T * n_heads * head_dim;
        p.dv_acc = p.dk_acc + (size_t)T * n_kv_heads * head_dim;
    }
    p.status = (uint32_t*)workspace;
    p.next_item = (uint32_t*)workspace + kNextBackward;
    p.n_graphs = batch->n_graphs;
    p.blocks = (batch->max_seqlen + kTile - 1) / kTile;
    p.by_work = batch->n_graphs == 1 || list_by_work(batch, causal, (size_t)T * n_heads * head_dim * 8);
    int64_t n_items = (int64_t)((batch->max_seqlen + kTile - 1) / kTile) * batch->n_graphs * n_heads * p.parts;
    if (batch->n_graphs > 1 && list_saves(batch, kTile, n_heads, 0)) {
        p.list = (const int4*)(ws + w.list_off);
        n_items = (int64_t)list_entries(batch, kTile) * n_heads;
    }
    if (n_items > 0x7fff0000) return GT_ERR_UNSUPPORTED;
    p.n_items = (int32_t)n_items;
    p.n_total = T;
    p.n_heads = n_heads;
    p.group = n_heads / n_kv_heads;
    p.causal = causal != 0;
    const float scale = 1.0f / sqrtf((float)head_dim);
    p.ds_scale = cap > 0.f ? -scale : scale;
    p.c1 = kLog2e * scale;
    p.to_tanh = cap > 0.f ? scale / cap : 0.f;
    p.cap2 = cap * kLog2e;
    cudaStream_t s = (cudaStream_t)stream;

    PrepareParams pre{};
    pre.out_f32 = out_f32;
    pre.dout = (const __nv_bfloat16*)dout;
    pre.lse = lse;
    pre.ext = (uint4*)(ws + w.ext_off);
    pre.acc = (float4*)dq_acc;
    pre.list = const_cast<int4*>(p.list);
    pre.cu_seqlens = batch->cu_seqlens;
    pre.n_acc = ((size_t)T * n_heads * head_dim * sizeof(float) + (sums ? 2 * w.kv_bytes : 0)) / 16;
    pre.n_total = T;
    pre.n_graphs = batch->n_graphs;
    pre.n_heads = n_heads;
    pre.by_work = p.by_work;
    pre.row_blocks = (uint32_t)(((size_t)T * n_heads + kPrepareRows - 1) / kPrepareRows);
    pre.sqrt_d = sqrtf((float)head_dim);
    const uint32_t list_blocks = p.list ? (uint32_t)((batch->n_graphs + kPrepareThreads / 32 - 1) / (kPrepareThreads / 32)) : 0;
    auto prepare = head_dim == 64 ? position_prepare_kernel<64> : position_prepare_kernel<32>;
    if ((st = launch_overlapped(prepare, dim3(pre.row_blocks + list_blocks), kPrepareThreads, 0, s, pre)) != GT_OK) return st;

    if (out_f32 == nullptr) {
        DeltaParams d{};
        d.cu_seqlens = batch->cu_seqlens;
        d.prefix = prefix;
        d.slopes = slopes;
        d.lse = lse;
        d.ext = pre.ext;
        d.status = p.status;
        d.list = p.list;
        d.n_items = p.n_items / p.parts;
        d.n_graphs = batch->n_graphs;
        d.n_total = T;
        d.n_heads = n_heads;
        d.group = p.group;
        d.causal = p.causal;
        d.by_work = p.by_work;
        d.blocks = p.blocks;
        d.c1 = p.c1;
        d.to_tanh = p.to_tanh;
        d.cap2 = p.cap2;
        st = position::pick(head_dim == 64, cap > 0.f, slopes != nullptr, [&](auto wide, auto capped, auto sloped) {
            return launch_delta<decltype(wide)::value ? 64 : 32, decltype(capped)::value, decltype(sloped)::value>(maps, d, s);
        });
        if (st != GT_OK) return st;
    }
    st = position::pick(head_dim == 64, cap > 0.f, slopes != nullptr, [&](auto wide, auto capped, auto sloped) {
        return launch<decltype(wide)::value ? 64 : 32, decltype(capped)::value, decltype(sloped)::value>(maps, p, batch, s);
    });
    if (st != GT_OK) return st;

    FinishParams f{};
    const float* acc[3] = {dq_acc, p.dk_acc, p.dv_acc};
    void* const to[3] = {dq, dk, dv};
    for (int i = 0; i < 3; ++i) {
        f.acc[i] = (const float4*)acc[i];
        f.to[i] = (__nv_bfloat16*)to[i];
        f.row[i] = row[3 + i];
        f.mul[i] = i < 2 ? p.ds_scale : 1.0f;
        f.vecs[i] = (uint32_t)((i == 0 ? n_heads : n_kv_heads) * head_dim / 4);
    }
    f.cu_seqlens = batch->cu_seqlens;
    f.n_total = T;
    f.n_graphs = batch->n_graphs;
    const uint64_t blocks = ((uint64_t)T * f.vecs[0] + kFinishThreads * kFinishEach - 1) / (kFinishThreads * kFinishEach);
    if (blocks > 0x7fffffffull) return GT_ERR_UNSUPPORTED;
    return launch_overlapped(position_finish_kernel, dim3((unsigned)blocks, sums ? 3u : 1u), kFinishThreads, 0, s, f);
}
