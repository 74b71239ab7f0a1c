// gt_position_attn_fwd: attention over packed token sequences,
//     out_i = sum_j softmax_j(S_i)_j v_j,   S_ij = cap tanh(q_i . k_j / (sqrt(d) cap)) - slopes[h] |i - j|,
// over the keys that the document, the causal order and the prefix leave a query.  Positions are indices, so nothing but q, k and v is read.
//
// The grid is persistent: a CTA takes one item of work (a head and one or two 128-row query tiles of a document) after the other, and its
// warps run through them as through one long row of key tiles.  The next item's rows are fetched, and its first scores made, while the
// last one's outputs are still written; with a CTA per item, 64 causal documents of 512-2 048 tokens spent 40 % of the time on filling and
// draining (551 -> 460 us).
//
//   warp 0      TMA producer: Q (two items' worth) and K, V through 2-stage rings
//   warp 1      issues S_t = Q_t K^T for both query tiles
//   warp 2      fetches the items
//   warp 3      issues O_t += P_t V (A from TMEM, B = V as MN-major); clears what lies behind the document in its last V tile
//   warps 4-19  softmax: 8 warps per query tile, 4 per half of the 128 key columns (thread = query row = TMEM lane, 64 scores)
//
// The key tiles come from the diagonal down to the document's beginning, then the ones behind the diagonal: with a penalty on distance
// the scores fall along that way, so that a row's reference stays in reach.  A causal item of two tiles begins with a key tile that only
// the second one sees; the first one skips that step.  Where a document has an odd number of tiles, its first one is an item of its own.
//
// Softmax: a tile is exponentiated against the row's reference at once (0 at first), without a look at its maximum; the tile's row sum
// tells whether the reference was out of reach, and only then it is redone with the maximum first.  References are whole numbers in log2
// units, so rescale factors are exact.  The capped score's polynomial is tried and redone in the same way.
//
// TMEM columns: three score buffers [0,128) [128,256) [256,384), used in turn by the steps (key tile, query tile), so that the S MMA of
// a step never waits for a softmax; P overwrites the part of a buffer that its own thread has read; O_0 [384,448), O_1 [448,512).
#include <math.h>

#include <algorithm>
#include <cmath>

#include "attn_position.cuh"

namespace gt {
namespace {

using namespace sm100;
using namespace position;

constexpr int kTile = 128;                    // rows of a query tile, keys of a key tile
constexpr int kStages = 2;                    // of the K ring and of the V ring
constexpr int kCols = 64;                     // score columns of a softmax thread
constexpr int kCW = 16;                       // columns per TMEM load
constexpr float kSumThreshold = 0x1p24f;       // tile row sum above which the reference is raised
// Scores of a capped row lie within cap log2(e) of 0 at the diagonal, so that against a reference of half of that the largest P is between 2^-108 and
// 2^37: sums, products with v of up to 2^60 and their sums stay within fp32, and nothing that counts is lost below.
constexpr float kBoundedCap = 50.0f, kLeastBoundedCap = 0.01f;       // (below, the scaled coefficients leave fp32)
// Every eighth pair of exponentials is a polynomial's (ex2_pair), which takes load off the special-function unit (77 % busy without) and adds
// to the issue slots: 16 384 tokens, 8 heads of 64, all pairs 768 -> 710 us (every sixth 746, every fourth 749, every third 790), causal 372 ->
// 344, causal with the fp32 output 428 -> 409; with the penalty on distance 411 -> 407, and with both 457 -> 475, so not there.  (Back to back, at the
// 1.76 GHz that the power limit leaves; a few passes at 1 965 MHz: causal 303.)
constexpr int kEx2Every = 8;
constexpr float kPeekReach = 24.0f;            // log2 units within which a row's first scores leave the starting reference as it is

struct PositionFwdParams {
    const int32_t* cu_seqlens;
    const int32_t* prefix;
    const float* slopes;
    __nv_bfloat16* out;        // [T,H,D]
    float* out_f32;            // [T,H,D] fp32, or nullptr
    float* lse;                // [H,T]
    uint32_t* status;
    uint32_t* next_item;       // counts the items that have been taken beyond the grid's first ones; 0 before and after the kernel
    const int4* list;          // packed batch: work list; item = entry * heads + head (nullptr: heads, then documents and blocks)
    int32_t n_items;
    int32_t halves_from;       // without a list: rows of items (all heads of a block) from this one on are halved
    int32_t by_work;           // without a list: the same block of all documents, then the next (else document after document)
    int32_t blocks;            // ... of the longest document
    int32_t n_graphs;
    int32_t n_total;
    int32_t n_heads;
    int32_t group;             // query heads per key head
    int32_t causal;
    int32_t whole;             // out and out_f32 begin at a whole sector
    int32_t early_release;     // let the next kernel start its set-up while this one runs
    float c1;                  // log2(e) / sqrt(d)
    float to_tanh;             // 1 / (sqrt(d) cap)
    float cap2;                // cap log2(e)
    float reference;           // kCapForm 1: of all rows, a whole number
    float tanh[6];             //   coefficients of tanh(s / cap2) cap2 / s as a polynomial in s^2
    float reach;               //   s^2 up to which it holds
};

enum Barrier {
    kBarItemFull = 0,                     // [2]  an item's description
    kBarItemEmpty = kBarItemFull + 2,     // [2]  all warps that work on it have read it
    kBarFetch = kBarItemEmpty + 2,        //      the next item is soon wanted
    kBarQFull = kBarFetch + 1,            // [2]
    kBarQEmpty = kBarQFull + 2,           // [2]  commit behind the item's last S MMAs
    kBarKFull = kBarQEmpty + 2,           // [kStages]
    kBarKEmpty = kBarKFull + kStages,     // [kStages]  commit behind the S MMAs of the key tile
    kBarVFull = kBarKEmpty + kStages,     // [kStages]
    kBarVEmpty = kBarVFull + kStages,     // [kStages]  commit behind the PV MMAs of the key tile
    kBarBufFree = kBarVEmpty + kStages,   // [3]  per score buffer: P consumed by its PV MMA
    kBarSFull = kBarBufFree + 3,          // [2 tiles][2 parities of the tile's steps]
    kBarPFull = kBarSFull + 4,            // [2 tiles][2 parities]
    kBarODone = kBarPFull + 4,            // [2 tiles][2 parities]
    kNumBarriers = kBarODone + 4
};

template <int D>
struct Smem {
    static constexpr int kRowBytes = D * 2;
    static constexpr int kTileBytes = 128 * kRowBytes;
    static constexpr int kQ = 0;
    static constexpr int kK = kQ + 4 * kTileBytes;               // Q: [2 items][2 tiles]
    static constexpr int kV = kK + kStages * kTileBytes;
    static constexpr int kXchg = kV + kStages * kTileBytes;      // [2 tiles][max | sum][2 halves][128 rows] float
    static constexpr int kBars = kXchg + 2 * 512 * 4;
    static constexpr int kItems = (kBars + kNumBarriers * 8 + 15) / 16 * 16;      // [2] Item
    static constexpr int kMisc = kItems + 2 * 32;
    static constexpr int kDynamic = kMisc + 16 + 1024;           // slack for the 1024-byte alignment
    static_assert(kXchg % 16 == 0 && kBars % 8 == 0 && kItems % 16 == 0 && kMisc % 16 == 0 && kDynamic <= 227 * 1024, "aligned, and within an SM");
};

struct alignas(16) Item {
    int32_t node0, n, head, prefix;        // n = 0: there are no more
    int32_t first, tiles, pad[2];          // the item's query tiles
};

// What follows from an item: its query tiles and the key tiles that they see.
struct Span {
    int32_t q0, tiles, diagonal, n_kv, skip;
    __device__ __forceinline__ void set(const Item& item, bool causal)
    {
        tiles = item.tiles;
        q0 = item.first * kTile;
        diagonal = item.first + tiles - 1;
        n_kv = causal ? max(diagonal + 1, (min(item.n, item.prefix) + kTile - 1) / kTile) : (item.n + kTile - 1) / kTile;
        // key tiles that the first query tile does not see: the item's first one, or none
        skip = tiles == 2 && causal && item.prefix <= diagonal * kTile ? 1 : 0;
    }
    __device__ __forceinline__ int32_t key_tile(int32_t s) const { return s <= diagonal ? diagonal - s : s; }
    __device__ __forceinline__ int32_t steps() const { return tiles * n_kv - skip; }
};

constexpr int kNbPair = 2;                    // named barriers: + 4 t + lane quarter, the two warps that share 32 query rows

// register budget with two tiles: the CTA is launched with 640 x 96 registers and shares out 128 x 56 + 512 x 104 = 60416 <= 61440
__device__ __forceinline__ void setmaxnreg_dec_56() { asm volatile("setmaxnreg.dec.sync.aligned.u32 56;"); }

// kTiles = 1: items of one query tile, for grids that end sooner with them (one_tile_blocks).
// kCapForm: 0 no cap; 1 a cap of kLeastBoundedCap to kBoundedCap; 2 any cap.  With the second form no score can be out of reach of a reference of half the
// cap, so that nothing is redone, and P takes the place of the scores chunk by chunk; the registers that this frees are what hides the
// polynomial's latency (causal 16 384 tokens, cap 30: 640 -> 530 us; with coefficients
// made for the scores themselves, and whole sectors per store, 490).
// kExact (with the fp32 output): O is divided by the sum of the probabilities as the MMA reads them, rounded to bf16, so that their
// rounding cancels where a row has few large ones; lse is that of the unrounded ones all the same.  The backward subtracts dout . out from
// dout . v_j, two nearly equal numbers in such rows: with scores of standard deviation 4, dq was off by 0.6 % (out rounded to bf16 and
// divided by the unrounded sum), by 0.45 % without either, and by 0.27 % with both.  (A backward without it makes Delta itself: attn_position_delta.cuh.)
template <int D, int kCapForm, bool kSlope, int kTiles, bool kExact>
__global__ void __launch_bounds__(128 + 256 * kTiles, 1)
position_fwd_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                    const __grid_constant__ CUtensorMap tmap_v, const PositionFwdParams p)
{
    using L = Smem<D>;
    constexpr bool kCap = kCapForm != 0, kBounded = kCapForm == 1;
    constexpr int kBuffers = kTiles + 1, kReaders = 3 + 8 * kTiles;          // kReaders: warps that work on an item
    constexpr uint32_t kOCol = 384;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint64_t* bars = (uint64_t*)(smem + L::kBars);
    uint32_t* misc = (uint32_t*)(smem + L::kMisc);       // [0] TMEM base, [1] abort flag
    Item* items = (Item*)(smem + L::kItems);
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    volatile uint32_t* abort_flag = &misc[1];
    if (tid == 0) {
        misc[1] = 0u;
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(kBarItemFull + s), 1);
            mbar_init(bar(kBarItemEmpty + s), kReaders);
            mbar_init(bar(kBarQFull + s), 1);
            mbar_init(bar(kBarQEmpty + s), 1);
        }
        mbar_init(bar(kBarFetch), 1);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bar(kBarKFull + s), 1);
            mbar_init(bar(kBarKEmpty + s), 1);
            mbar_init(bar(kBarVFull + s), 1);
            mbar_init(bar(kBarVEmpty + s), 1);
        }
        for (int b = 0; b < 3; ++b) mbar_init(bar(kBarBufFree + b), 1);
        for (int t = 0; t < 4; ++t) {
            mbar_init(bar(kBarSFull + t), 1);
            mbar_init(bar(kBarPFull + t), 8);                // one arrival per warp
            mbar_init(bar(kBarODone + t), 1);
        }
        fence_mbar_init();
        prefetch_tensormap(&tmap_q);
        prefetch_tensormap(&tmap_k);
        prefetch_tensormap(&tmap_v);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&misc[0]), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = misc[0];
    grid_wait();
    if (p.early_release) grid_release();

    // Item number k of this CTA, read by whole warps; false: there are no more.
    auto take = [&](int k, Item& item) -> bool {
        const bool had = item_wait(bar(kBarItemFull + (k & 1)), (k >> 1) & 1, abort_flag, p.status, 200);
        item = items[k & 1];
        if (!goes_on(had, item.n, abort_flag, warp_any)) return false;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kBarItemEmpty + (k & 1)));
        return true;
    };

    if (warp < 4) {
        if constexpr (kTiles == 2) setmaxnreg_dec_56();
        if (warp == 2) {
            // ---- the items: the CTA's own number, then what the counter gives, as late as its latency allows: the longest items come
            // first, and who takes the short ones of the end is decided by who is done (two items ahead: causal 16 384 tokens 441 us, now 370) ----
            int32_t index = (int32_t)blockIdx.x;
            bool good = true;                                // no wait has been given up (then the items are only counted to their end)
            for (int k = 0;; ++k) {
                if (k > 0 && good) good = !warp_any(!item_wait(bar(kBarFetch), (k - 1) & 1, abort_flag, p.status, 203));
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
                    int32_t g, block, part = -1;              // part: of a block that is halved
                    if (p.list) {
                        const int4 entry = p.list[index / p.n_heads];
                        g = entry.x;
                        block = entry.y;
                        item.node0 = entry.z;
                        item.n = entry.x < 0 ? 0 : entry.w;
                    } else {
                        int32_t row = index / p.n_heads;
                        if (kTiles == 2 && row >= p.halves_from) {
                            part = (row - p.halves_from) & 1;
                            row = p.halves_from + (row - p.halves_from) / 2;
                        }
                        block = p.by_work ? row / p.n_graphs : row % p.blocks;
                        g = p.by_work ? row % p.n_graphs : row / p.blocks;
                        item.node0 = p.cu_seqlens ? p.cu_seqlens[g] : 0;
                        item.n = p.cu_seqlens ? p.cu_seqlens[g + 1] - item.node0 : p.n_total;
                    }
                    item.head = index % p.n_heads;
                    index = -1;
                    // blocks of kTiles query tiles, counted from the document's end
                    const int32_t n_tiles = (item.n + kTile - 1) / kTile, n_blocks = (n_tiles + kTiles - 1) / kTiles, odd = n_blocks * kTiles - n_tiles;
                    const int32_t q_block = p.causal ? n_blocks - 1 - block : block;
                    item.first = max(0, q_block * kTiles - odd);
                    item.tiles = kTiles == 2 && odd && q_block == 0 ? 1 : kTiles;
                    if (part >= 0) {
                        if (part == 1 && item.tiles == 1) block = n_blocks;       // (there is no other half)
                        item.first += part;
                        item.tiles = 1;
                    }
                    if (block >= n_blocks) item.n = 0;
                    else item.prefix = p.prefix ? p.prefix[g] : 0;
                }
                if (k >= 2 && good) good = !warp_any(!item_wait(bar(kBarItemEmpty + (k & 1)), ((k >> 1) & 1) ^ 1, abort_flag, p.status, 201));
                if (good && lane == 0) {
                    items[k & 1] = item;
                    mbar_arrive(bar(kBarItemFull + (k & 1)));
                }
                __syncwarp();
                if (item.n == 0) break;
            }
        } else if (warp == 0) {
            Item item;
            Span span;
            int c = 0;                                       // key tiles so far
            bool good = true;                                // no wait has been given up
            for (int k = 0; take(k, item); ++k) {
                span.set(item, p.causal);
                const int kv_head = item.head / p.group;
                if (k >= 2) good &= mbar_wait(bar(kBarQEmpty + (k & 1)), ((k >> 1) & 1) ^ 1, abort_flag, p.status, 210);
                if (good && lane == 0) {
                    mbar_arrive_expect_tx(bar(kBarQFull + (k & 1)), span.tiles * L::kTileBytes);
                    for (int t = 0; t < span.tiles; ++t)
                        tma_load_3d(smem_u32(smem + L::kQ + (2 * (k & 1) + t) * L::kTileBytes), &tmap_q, bar(kBarQFull + (k & 1)), 0, item.head,
                                    item.node0 + span.q0 + t * kTile);
                }
                const int32_t fetch = max(0, span.n_kv - 6);
                for (int s = 0; s < span.n_kv; ++s, ++c) {
                    if (s == fetch && lane == 0) mbar_arrive(bar(kBarFetch));
                    const int st = c % kStages;
                    const int32_t row = item.node0 + span.key_tile(s) * kTile;
                    if (c >= kStages) good &= mbar_wait(bar(kBarKEmpty + st), ((c / kStages) & 1) ^ 1, abort_flag, p.status, 211);
                    if (good && lane == 0) {
                        mbar_arrive_expect_tx(bar(kBarKFull + st), L::kTileBytes);
                        tma_load_3d(smem_u32(smem + L::kK + st * L::kTileBytes), &tmap_k, bar(kBarKFull + st), 0, kv_head, row);
                    }
                    if (c >= kStages) good &= mbar_wait(bar(kBarVEmpty + st), ((c / kStages) & 1) ^ 1, abort_flag, p.status, 212);
                    if (good && lane == 0) {
                        mbar_arrive_expect_tx(bar(kBarVFull + st), L::kTileBytes);
                        tma_load_3d(smem_u32(smem + L::kV + st * L::kTileBytes), &tmap_v, bar(kBarVFull + st), 0, kv_head, row);
                    }
                    __syncwarp();
                }
            }
        } else if (warp == 1) {
            constexpr uint32_t idesc_s = make_idesc_bf16(128, 128, false, false);
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
            const uint64_t desc_q0 = make_smem_desc(smem_u32(smem + L::kQ), L::kRowBytes, 0);
            const uint64_t desc_k0 = make_smem_desc(smem_u32(smem + L::kK), L::kRowBytes, 0);
            Item item;
            Span span;
            int c = 0, step = 0;                             // key tiles, and score tiles, so far
            int own[2][2] = {{-4, -4}, {-4, -4}}, done[2] = {0, 0};      // each query tile's last two steps, and how many there were
            for (int k = 0; take(k, item); ++k) {
                span.set(item, p.causal);
                mbar_wait(bar(kBarQFull + (k & 1)), (k >> 1) & 1, abort_flag, p.status, 220);
                for (int s = 0; s < span.n_kv; ++s, ++c) {
                    const int ks = c % kStages;
                    mbar_wait(bar(kBarKFull + ks), (c / kStages) & 1, abort_flag, p.status, 221);
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        if (t >= span.tiles || (t == 0 && s < span.skip)) continue;
                        const int b = step % kBuffers;
                        if (step >= kBuffers) mbar_wait(bar(kBarBufFree + b), (step / kBuffers - 1) & 1, abort_flag, p.status, 222);
                        // A tile's softmax may be one step behind, not two (see "one step apart" below): its last step but one has been through
                        // its PV MMA.  Mostly that follows from the buffers; not where an item has one tile only.
                        const int last_but_one = own[t][0], parity = done[t] & 1;
                        if (step - last_but_one < kBuffers) mbar_wait(bar(kBarBufFree + last_but_one % kBuffers), (last_but_one / kBuffers) & 1, abort_flag, p.status, 223);
                        own[t][0] = own[t][1];
                        own[t][1] = step;
                        ++done[t];
                        ++step;
                        tc_fence_after();
                        if (elect_one()) {
                            const uint64_t da = advance_desc(desc_q0, (2 * (k & 1) + t) * L::kTileBytes), db = advance_desc(desc_k0, ks * L::kTileBytes);
#pragma unroll
                            for (int e = 0; e < D / 16; ++e)
                                mma_ss(tm + b * 128, advance_desc(da, e * 32), advance_desc(db, e * 32), idesc_s, e > 0);
                            mma_commit(bar(kBarSFull + 2 * t + parity));
                            if (t == span.tiles - 1) {
                                mma_commit(bar(kBarKEmpty + ks));
                                if (s == span.n_kv - 1) mma_commit(bar(kBarQEmpty + (k & 1)));
                            }
                        }
                        __syncwarp();
                    }
                }
            }
        } else {
            constexpr uint32_t idesc_o = make_idesc_bf16(128, D, false, true);
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
            const uint64_t desc_v0 = make_smem_desc(smem_u32(smem + L::kV), L::kRowBytes, 0);
            Item item;
            Span span;
            int c = 0, step = 0, own[2] = {0, 0};            // key tiles, score tiles and each query tile's so far
            for (int k = 0; take(k, item); ++k) {
                span.set(item, p.causal);
                // the document's last V tile, if rows of another one follow in it
                const int32_t ragged_tile = item.n % kTile != 0 && item.node0 + item.n < p.n_total ? item.n / kTile : -1;
                for (int s = 0; s < span.n_kv; ++s, ++c) {
                    const int vs = c % kStages;
                    mbar_wait(bar(kBarVFull + vs), (c / kStages) & 1, abort_flag, p.status, 230);
                    if (span.key_tile(s) == ragged_tile) {
                        clear_rows(smem + L::kV + vs * L::kTileBytes, item.n - ragged_tile * kTile, L::kRowBytes);
                        fence_proxy_async_smem();
                        __syncwarp();
                    }
                    const uint64_t dv = advance_desc(desc_v0, vs * L::kTileBytes);
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        if (t >= span.tiles || (t == 0 && s < span.skip)) continue;
                        const int b = step % kBuffers;
                        const uint32_t begun = s > (t == 0 ? span.skip : 0) ? 1u : 0u;
                        mbar_wait(bar(kBarPFull + 2 * t + (own[t] & 1)), (own[t] >> 1) & 1, abort_flag, p.status, 231);
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int e = 0; e < kTile / 16; ++e)      // P of key half hf sits at the start of that half's score columns
                                mma_ts(tm + kOCol + t * 64, tm + b * 128 + (e / 4) * kCols + (e % 4) * 8, advance_desc(dv, e * 16 * L::kRowBytes), idesc_o,
                                       e > 0 ? 1u : begun);
                            mma_commit(bar(kBarODone + 2 * t + (own[t] & 1)));
                            mma_commit(bar(kBarBufFree + b));
                            if (t == span.tiles - 1) mma_commit(bar(kBarVEmpty + vs));
                        }
                        __syncwarp();
                        ++step;
                        ++own[t];
                    }
                }
            }
        }
    } else {
        // =================================== softmax warps ===================================
        if constexpr (kTiles == 2) setmaxnreg_inc_104();
        const int sw = warp - 4;
        const int t = sw >> 3, hf = (sw >> 2) & 1;
        const int r = ((warp & 3) << 5) | lane;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        constexpr int kOC = D / 2;                       // output columns per thread
        const uint32_t tO = tmem + kOCol + t * 64 + hf * kOC + lane_off;
        const uint32_t pair_bar = kNbPair + t * 4 + (warp & 3);
        float* xchg = (float*)(smem + L::kXchg) + t * 512;
        const uint64_t c1c1 = both(p.c1);
        [[maybe_unused]] const uint64_t to_tanh2 = both(p.to_tanh);

        int step0 = 0, own = 0;                 // score tiles, and this query tile's, so far
        for (int k = 0;; ++k) {
        // (the item is read again where its results are written, and given back behind that: fewer registers in between)
        const bool had = item_wait(bar(kBarItemFull + (k & 1)), (k >> 1) & 1, abort_flag, p.status, 202);
        if (!goes_on(had, items[k & 1].n, abort_flag, [&](bool x) { return named_barrier_or(pair_bar, 64, x); })) break;
        Span span;
        span.set(items[k & 1], p.causal);
        const int32_t first = t == 0 ? span.skip : 0, diagonal = span.diagonal, step_by = span.tiles;
        int32_t key_tile = span.key_tile(first), left = t < span.tiles ? span.n_kv - first : 0;       // left: steps
        int step = step0 + (span.tiles == 2 ? 2 * first + t - span.skip : 0);
        step0 += span.steps();
        if (left > 0) {
        const int32_t q = span.q0 + t * kTile + r;                                     // this thread's query
        const int32_t limit = row_limit(p.causal, q, items[k & 1].prefix, items[k & 1].n);
        const bool counts = q < items[k & 1].n;
        bool begins = true;
        float m = kBounded ? p.reference : 0.f, l = 0.f;
        [[maybe_unused]] float l_rounded = 0.f;
        [[maybe_unused]] bool wide = false;              // a score was out of the polynomial's reach
        [[maybe_unused]] const float slope2 = kSlope ? p.slopes[items[k & 1].head] * kLog2e : 0.f;
        // (a negative slope favours the farthest key that the row sees: the bound on the scores moves along)
        if (kBounded && kSlope && slope2 < 0.f) m -= slope2 * (float)max(q, limit - 1 - q);
        // (steep penalties: made for every element wherever a row's own key is, see kSteep)
        [[maybe_unused]] const int32_t linear_from = kSlope ? fabsf(slope2) > kSteep ? INT32_MAX : items[k & 1].prefix : 0;

        uint32_t sa[kCW], sb[kCW];              // score chunks, alternating
        uint32_t tS = 0;                        // this thread's score columns of the current step
        auto load_chunk = [&](int c, uint32_t (&sr)[kCW]) { tmem_ld16(tS + c * kCW, sr); };
        // first chunk of a step's scores: fetched at the end of the step before, behind the P store
        auto begin_step = [&]() {
            const int b = step % kBuffers;
            tS = tmem + b * 128 + hf * kCols + lane_off;
            mbar_wait(bar(kBarSFull + 2 * t + (own & 1)), (own >> 1) & 1, abort_flag, p.status, 250);
            tc_fence_after();
            load_chunk(0, sa);
        };
        begin_step();

        for (;;) {
            const int32_t kv0 = key_tile * kTile + hf * kCols;         // this thread's first key
            const int valid = limit - kv0;                             // columns that this thread's row sees (may be <= 0)
            const bool ragged = __any_sync(0xffffffffu, valid < kCols);
            [[maybe_unused]] const int32_t row0 = q - lane;
            // Penalty on distance.  Where no key lies behind the query (or, for masked ones, it does not matter) it is linear in the
            // column: (key - query) slope.  Otherwise keys behind all of the warp's rows have it the other way round, and in between
            // a distance is made for every element.
            const bool before = kv0 + kCols - 1 <= row0 || (p.causal && kv0 >= linear_from), behind = kv0 >= row0 + 31;
            [[maybe_unused]] const bool mixed = kSlope && !before && !behind;
            [[maybe_unused]] const float step_slope = before ? slope2 : -slope2, ahead = (float)(kv0 - q);       // ahead: the first key's distance
            [[maybe_unused]] uint32_t pk[32];      // P of this thread's columns, bf16 pairs
            float tile_sum = 0.f;
            [[maybe_unused]] uint64_t rounded2 = 0;
            bool loaded = true;                    // chunk 0 is already on its way
            bool exact = false;                    // take the tile maximum first

            // Is the starting reference in reach of the first tile?  Four of the thread's first 16 scores tell.
            if (!kBounded && begins) {
                tmem_wait_ld();
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = __uint_as_float(sa[4 * i]) * p.c1;
                    if constexpr (kCap) x = fminf(fmaxf(x, -p.cap2), p.cap2);
                    if constexpr (kSlope) x -= slope2 * fabsf(ahead + (float)(4 * i));
                    if (4 * i < valid) top = fmaxf(top, x);
                }
                exact = named_barrier_or(pair_bar, 64, valid > 0 && counts && !(fabsf(top) <= kPeekReach));   // (a half without valid columns has no say)
            }

            // Scores of eight consecutive columns in log2 units, plus `add`; general: any score, any distance.
            float top_u = 0.f;
            [[maybe_unused]] auto scaled_ratio = [&](uint64_t u) {
                uint64_t r = fma_f32x2(both(p.tanh[5]), u, both(p.tanh[4]));
#pragma unroll
                for (int i = 3; i >= 0; --i) r = fma_f32x2(r, u, both(p.tanh[i]));
                return r;
            };
            auto scores8 = [&](const uint32_t* sr, int col, float add, auto rag, auto general, float (&x)[8]) {
                uint64_t a = both(add);
                if constexpr (kSlope && !decltype(general)::value) {
                    const float at = fmaf(step_slope, ahead + (float)col, add);
                    a = pack_f32x2(at, at + step_slope);
                }
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const uint64_t raw = pack_u32x2(sr[i], sr[i + 1]);
                    uint64_t y;
                    if constexpr (kSlope && !decltype(general)::value)
                        if (i > 0) a = add_f32x2(a, both(2.0f * step_slope));
                    if constexpr (kCap && decltype(general)::value) {
                        float u0, u1, a0, a1;
                        unpack_f32x2(mul_f32x2(raw, to_tanh2), u0, u1);
                        unpack_f32x2(a, a0, a1);
                        y = pack_f32x2(fmaf(p.cap2, tanh_any(u0), a0), fmaf(p.cap2, tanh_any(u1), a1));
                    } else if constexpr (kCap) {
                        // (kBounded: u is the score itself, in log2 units, and the polynomial's coefficients are made for that)
                        const uint64_t u = mul_f32x2(raw, kBounded ? c1c1 : to_tanh2), uu = mul_f32x2(u, u);
                        float u0, u1;
                        unpack_f32x2(uu, u0, u1);
                        if constexpr (decltype(rag)::value) {
                            if (col + i >= valid) u0 = 0.f;
                            if (col + i + 1 >= valid) u1 = 0.f;
                        }
                        top_u = max3(top_u, u0, u1);
                        y = kBounded ? fma_f32x2(u, scaled_ratio(uu), a) : fma_f32x2(mul_f32x2(raw, c1c1), tanh_ratio(uu), a);
                    } else {
                        y = fma_f32x2(raw, c1c1, a);
                    }
                    unpack_f32x2(y, x[i], x[i + 1]);
                    if constexpr (kSlope)
                        if constexpr (decltype(general)::value) {
                            x[i] = fmaf(-slope2, fabsf(ahead + (float)(col + i)), x[i]);
                            x[i + 1] = fmaf(-slope2, fabsf(ahead + (float)(col + i + 1)), x[i + 1]);
                        }
                }
            };

            if constexpr (kBounded) {
                uint64_t sum2 = pack_f32x2(0.f, 0.f);
                rounded2 = sum2;
                auto chunk = [&](int c, const uint32_t (&sr)[kCW], auto rag) {
                    float x[kCW];
                    uint32_t w[kCW / 2];
                    top_u = 0.f;
#pragma unroll
                    for (int e = 0; e < kCW; e += 8) scores8(sr + e, c * kCW + e, -m, rag, Tag<false>{}, *(float (*)[8])(x + e));
                    if (__any_sync(0xffffffffu, counts && !(top_u <= p.reach)) || mixed) {
#pragma unroll
                        for (int e = 0; e < kCW; e += 8) scores8(sr + e, c * kCW + e, -m, rag, Tag<true>{}, *(float (*)[8])(x + e));
                    }
#pragma unroll
                    for (int i = 0; i < kCW; i += 2) {
                        if constexpr (decltype(rag)::value) {
                            if (c * kCW + i >= valid) x[i] = -INFINITY;
                            if (c * kCW + i + 1 >= valid) x[i + 1] = -INFINITY;
                        }
                        const float lo = ex2_approx(x[i]), hi = ex2_approx(x[i + 1]);
                        sum2 = add_f32x2(sum2, pack_f32x2(lo, hi));
                        w[i >> 1] = pack_bf16x2(lo, hi);
                        if constexpr (kExact) rounded2 = add_f32x2(rounded2, pack_u32x2(w[i >> 1] << 16, w[i >> 1] & 0xffff0000u));
                    }
                    tmem_st8(tS + c * (kCW / 2), w);             // over columns of chunks that are in registers, or were
                };
                auto pass = [&](auto rag) {
                    tmem_wait_ld(); load_chunk(1, sb); chunk(0, sa, rag);
                    tmem_wait_ld(); load_chunk(2, sa); chunk(1, sb, rag);
                    tmem_wait_ld(); load_chunk(3, sb); chunk(2, sa, rag);
                    tmem_wait_ld(); chunk(3, sb, rag);
                };
                if (ragged) pass(Tag<true>{});
                else pass(Tag<false>{});
                float lo, hi;
                unpack_f32x2(sum2, lo, hi);
                tile_sum = lo + hi;
            } else for (;;) {
                if (exact) {
                    // ---- classical way: tile maximum, new reference, rescale of l and O ----
                    float mx = -INFINITY;
                    auto max_chunk = [&](int c, const uint32_t (&sr)[kCW]) {
#pragma unroll
                        for (int e = 0; e < kCW; e += 8) {
                            float x[8];
                            scores8(sr + e, c * kCW + e, 0.f, Tag<false>{}, Tag<true>{}, x);
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (c * kCW + e + i < valid) mx = fmaxf(mx, x[i]);
                        }
                    };
                    if (!loaded) load_chunk(0, sa);
                    tmem_wait_ld(); load_chunk(1, sb); max_chunk(0, sa);
                    tmem_wait_ld(); load_chunk(2, sa); max_chunk(1, sb);
                    tmem_wait_ld(); load_chunk(3, sb); max_chunk(2, sa);
                    tmem_wait_ld(); max_chunk(3, sb);
                    loaded = false;
                    xchg[hf * 128 + r] = mx;
                    named_barrier_sync(pair_bar, 64);
                    mx = fmaxf(mx, xchg[(hf ^ 1) * 128 + r]);
                    const float m_new = begins ? ceilf(mx) : fmaxf(m, ceilf(mx));
                    const float alpha = begins ? 0.f : ex2_approx(m - m_new);      // (there is nothing yet; a first reference far below 0 would give infinity)
                    l *= alpha;
                    if constexpr (kExact) l_rounded *= alpha;
                    if (!begins) {
                        mbar_wait(bar(kBarODone + 2 * t + ((own - 1) & 1)), ((own - 1) >> 1) & 1, abort_flag, p.status, 251);
                        tc_fence_after();
                        uint32_t o[kOC];
                        if constexpr (kOC == 32) tmem_ld32(tO, o); else tmem_ld16(tO, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < kOC; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                        if constexpr (kOC == 32) tmem_st32(tO, o); else tmem_st16(tO, o);
                    }
                    m = m_new;
                }

                // ---- P = 2^(score - m), row sum ----
                uint64_t sum2 = pack_f32x2(0.f, 0.f);
                rounded2 = sum2;
                auto exp_chunk = [&](int c, const uint32_t (&sr)[kCW], auto rag, auto general) {
#pragma unroll
                    for (int e = 0; e < kCW; e += 8) {
                        float x[8];
                        scores8(sr + e, c * kCW + e, -m, rag, general, x);
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            if constexpr (decltype(rag)::value) {
                                if (c * kCW + e + i >= valid) x[i] = -INFINITY;
                                if (c * kCW + e + i + 1 >= valid) x[i + 1] = -INFINITY;
                            }
                            float lo, hi;
                            // (never behind the classical way: a NaN would not come through)
                            if (!decltype(rag)::value && !(kSlope && kExact) && ((c * kCW + e + i) / 2) % kEx2Every == kEx2Every - 1) {
                                ex2_pair(pack_f32x2(x[i], x[i + 1]), lo, hi);
                            } else {
                                lo = ex2_approx(x[i]);
                                hi = ex2_approx(x[i + 1]);
                            }
                            sum2 = add_f32x2(sum2, pack_f32x2(lo, hi));
                            const uint32_t w = pk[(c * kCW + e + i) >> 1] = pack_bf16x2(lo, hi);
                            if constexpr (kExact) rounded2 = add_f32x2(rounded2, pack_u32x2(w << 16, w & 0xffff0000u));
                        }
                    }
                };
                auto exp_pass = [&](auto rag, auto general) {
                    if (!loaded) load_chunk(0, sa);
                    tmem_wait_ld(); load_chunk(1, sb); exp_chunk(0, sa, rag, general);
                    tmem_wait_ld(); load_chunk(2, sa); exp_chunk(1, sb, rag, general);
                    tmem_wait_ld(); load_chunk(3, sb); exp_chunk(2, sa, rag, general);
                    tmem_wait_ld(); exp_chunk(3, sb, rag, general);
                };
                if (mixed || (kCap && (exact || wide))) exp_pass(Tag<true>{}, Tag<kCap || kSlope>{});
                else if (ragged || exact) exp_pass(Tag<true>{}, Tag<false>{});
                else exp_pass(Tag<false>{}, Tag<false>{});
                loaded = false;
                {
                    float lo, hi;
                    unpack_f32x2(sum2, lo, hi);
                    tile_sum = lo + hi;
                }
                if (exact) break;
                // reference too low for some row of this pair of warps?  Also catches inf / NaN, and scores near the cap.
                // (Rows behind the document have no say.)
                const bool beyond = kCap && !wide && counts && !(top_u <= kTanhReach);
                if (!named_barrier_or(pair_bar, 64, (counts && !(tile_sum <= kSumThreshold)) || beyond)) break;
                if (kCap && !wide && named_barrier_or(pair_bar, 64, beyond)) wide = true;       // from now on, with the tanh of any score
                else exact = true;
            }
            l += tile_sum;
            if constexpr (kExact) {
                float lo, hi;
                unpack_f32x2(rounded2, lo, hi);
                l_rounded += lo + hi;
            }

            // P over the first half of this thread's own score columns
            if constexpr (!kBounded) tmem_st32(tS, pk);
            tmem_wait_st();
            tc_fence_before();
            // Warps of a tile can be one step apart (nothing in the speculative pass waits for the previous PV MMA), so odd and even steps
            // have barriers of their own: a parity wait can only tell two states apart.  Two steps apart they are never: the S MMA waits
            // for the PV MMA of the last step but one.
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarPFull + 2 * t + (own & 1)));
            ++own;
            step += step_by;
            begins = false;
            if (--left == 0) break;
            key_tile = key_tile > diagonal ? key_tile + 1 : key_tile > 0 ? key_tile - 1 : diagonal + 1;
            begin_step();
        }

        // ---- epilogue: O / l, LSE ----
        mbar_wait(bar(kBarODone + 2 * t + ((own - 1) & 1)), ((own - 1) >> 1) & 1, abort_flag, p.status, 252);
        tc_fence_after();
        xchg[256 + hf * 128 + r] = l;
        if constexpr (kExact) xchg[hf * 128 + r] = l_rounded;
        named_barrier_sync(pair_bar, 64);
        l += xchg[256 + (hf ^ 1) * 128 + r];
        if constexpr (kExact) l_rounded += xchg[(hf ^ 1) * 128 + r];
        uint32_t o[kOC];
        if constexpr (kOC == 32) tmem_ld32(tO, o); else tmem_ld16(tO, o);
        tmem_wait_ld();
        if (counts) {
            const int32_t node = items[k & 1].node0 + q, h = items[k & 1].head;
            float x[kOC];
            if constexpr (kExact) {
#pragma unroll
                for (int i = 0; i < kOC; ++i) x[i] = __uint_as_float(o[i]) / l_rounded;      // (a row with one key gets that key's value to the bit)
                float* dst32 = p.out_f32 + ((size_t)node * p.n_heads + h) * D + hf * kOC;
#pragma unroll
                for (int i = 0; i < kOC; i += 8) {
                    const uint32_t w[8] = {__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]), __float_as_uint(x[i + 3]),
                                           __float_as_uint(x[i + 4]), __float_as_uint(x[i + 5]), __float_as_uint(x[i + 6]), __float_as_uint(x[i + 7])};
                    store_sector(dst32 + i, p.whole, w);
                }
            } else {
                const float inv_l = 1.0f / l;
#pragma unroll
                for (int i = 0; i < kOC; ++i) x[i] = __uint_as_float(o[i]) * inv_l;
            }
            __nv_bfloat16* dst = p.out + ((size_t)node * p.n_heads + h) * D + hf * kOC;
#pragma unroll
            for (int i = 0; i < kOC; i += 16) {
                const uint32_t w[8] = {pack_bf16x2(x[i], x[i + 1]), pack_bf16x2(x[i + 2], x[i + 3]), pack_bf16x2(x[i + 4], x[i + 5]), pack_bf16x2(x[i + 6], x[i + 7]),
                                       pack_bf16x2(x[i + 8], x[i + 9]), pack_bf16x2(x[i + 10], x[i + 11]), pack_bf16x2(x[i + 12], x[i + 13]), pack_bf16x2(x[i + 14], x[i + 15])};
                store_sector(dst + i, p.whole, w);
            }
            if (hf == 0) p.lse[(size_t)h * p.n_total + node] = (m + log2f(l)) * kLn2;
        }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kBarItemEmpty + (k & 1)));
        }
    }

    // ---- teardown ----
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) __nanosleep(200000);    // let copies that may still be in flight land
    if (warp == 1) tmem_dealloc(tmem, 512);
}

// Work list of a packed batch, a warp per document.
constexpr int kListThreads = 128;
__global__ void __launch_bounds__(kListThreads) position_list_kernel(int4* list, int32_t entries, const int32_t* cu_seqlens, int32_t n_graphs, bool by_work)
{
    grid_wait();
    grid_release();
    const int32_t w = (int32_t)((blockIdx.x * blockDim.x + threadIdx.x) >> 5);
    if (w < n_graphs) write_list<2 * kTile>(list, entries, cu_seqlens, n_graphs, w, by_work);
}
constexpr size_t kListMinSaved = 256;        // empty items that the list has to save: it costs a launch

// Blocks of one query tile, a CTA for each, or of two?  A key tile takes about 1.0 us with one query tile and 1.4 us with two, so that two are
// faster where the grid fills the device; the longest block (causal: the last one) has to be through all the same.
inline bool one_tile_blocks(const gt_batch* b, int32_t n_heads, bool causal)
{
    const double tiles = (b->max_seqlen + kTile - 1) / kTile, pairs = (b->max_seqlen + 2 * kTile - 1) / (2 * kTile);
    const double m = (double)b->n_graphs * n_heads, sms = sm_count();
    const double one = causal ? std::max(tiles, m * tiles * (tiles + 1) / 2 / sms) : std::ceil(m * tiles / sms) * tiles;
    const double two = causal ? std::max(tiles, m * pairs * (pairs + 1) / sms) : std::ceil(m * pairs / sms) * tiles;
    return 1.0 * one < 1.4 * two;
}
// Blocks of one long document, all of one length, that are halved so that the grid's last wave is one of halves.
inline int32_t halved_blocks(int32_t blocks, int32_t n_heads)
{
    const int64_t all = (int64_t)blocks * n_heads, whole = all / sm_count() * sm_count() / n_heads;       // blocks in full waves
    return 2 * (all - whole * n_heads) <= sm_count() ? (int32_t)(blocks - whole) : 0;
}

template <int D, int kCapForm, bool kSlope, bool kExact>
gt_status launch(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, PositionFwdParams p, const gt_batch* batch, int32_t rows,
                 cudaStream_t s)
{
    const bool one = rows == kTile;
    auto kern = one ? position_fwd_kernel<D, kCapForm, kSlope, 1, kExact> : position_fwd_kernel<D, kCapForm, kSlope, 2, kExact>;
    static std::atomic<uint64_t> granted[2] = {};
    const gt_status st = grant_smem(kern, granted[one], Smem<D>::kDynamic);
    if (st != GT_OK) return st;
    const dim3 grid((unsigned)std::min(p.n_items, sm_count()));
    p.early_release = p.n_items <= sm_count();
    return launch_overlapped(kern, grid, 128 + 2 * rows, Smem<D>::kDynamic, s, tq, tk, tv, p);
}

}  // namespace
}  // namespace gt

extern "C" size_t gt_position_attn_fwd_workspace(const gt_batch* batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim)
{
    if (gt::position::validate(batch, n_heads, n_kv_heads, head_dim, nullptr, 0, 0.f) != GT_OK) return 0;
    return gt::kHeaderBytes + gt::list_bytes(batch, 2 * gt::kTile);
}

extern "C" gt_status gt_position_attn_fwd(const void* q, const void* k, const void* v, const float* slopes, const int32_t* prefix,
                                          const gt_batch* batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                          const gt_row_strides* strides, int32_t causal, float cap, void* out, float* lse, float* out_f32,
                                          void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace gt;
    gt_status st = position::validate(batch, n_heads, n_kv_heads, head_dim, prefix, causal, cap);
    if (st != GT_OK) return st;
    if (!q || !k || !v || !out || !lse) return GT_ERR_INVALID_ARG;
    if (misaligned16(q) || misaligned16(k) || misaligned16(v) || misaligned16(out) || misaligned16(out_f32)) return GT_ERR_INVALID_ARG;
    int64_t sq, sk, sv;
    if (!position::row_stride(strides ? strides->q : 0, n_heads, head_dim, &sq) || !position::row_stride(strides ? strides->k : 0, n_kv_heads, head_dim, &sk) ||
        !position::row_stride(strides ? strides->v : 0, n_kv_heads, head_dim, &sv))
        return GT_ERR_INVALID_ARG;
    if (workspace == nullptr || misaligned16(workspace) || workspace_bytes < gt_position_attn_fwd_workspace(batch, n_heads, n_kv_heads, head_dim))
        return GT_ERR_WORKSPACE;
    if (sm_count() <= 0) return GT_ERR_NO_DEVICE;
    CUtensorMap tq, tk, tv;
    if ((st = encode_rows_map(&tq, q, batch->n_total, n_heads, head_dim, sq)) != GT_OK) return st;
    if ((st = encode_rows_map(&tk, k, batch->n_total, n_kv_heads, head_dim, sk)) != GT_OK) return st;
    if ((st = encode_rows_map(&tv, v, batch->n_total, n_kv_heads, head_dim, sv)) != GT_OK) return st;
    PositionFwdParams p{};
    p.cu_seqlens = batch->cu_seqlens;
    p.prefix = prefix;
    p.slopes = slopes;
    p.out = (__nv_bfloat16*)out;
    p.out_f32 = out_f32;
    p.whole = position::whole_sectors(out) && position::whole_sectors(out_f32);
    p.lse = lse;
    p.status = (uint32_t*)workspace;
    p.next_item = (uint32_t*)workspace + kNextForward;
    p.n_total = batch->n_total;
    p.n_heads = n_heads;
    p.group = n_heads / n_kv_heads;
    p.causal = causal != 0;
    p.c1 = kLog2e / sqrtf((float)head_dim);
    p.to_tanh = cap > 0.f ? 1.0f / (sqrtf((float)head_dim) * cap) : 0.f;
    p.cap2 = cap * kLog2e;
    cudaStream_t s = (cudaStream_t)stream;
    p.n_graphs = batch->n_graphs;
    const int32_t rows = one_tile_blocks(batch, n_heads, causal != 0) ? kTile : 2 * kTile;
    const int32_t blocks = (batch->max_seqlen + rows - 1) / rows;
    p.blocks = blocks;
    p.by_work = batch->n_graphs == 1 || list_by_work(batch, causal, (size_t)batch->n_total * n_kv_heads * head_dim * 4);
    int64_t n_items = (int64_t)blocks * batch->n_graphs * n_heads;
    p.halves_from = blocks * batch->n_graphs;
    if (rows == 2 * kTile && batch->n_graphs == 1 && !causal) {
        const int32_t halved = halved_blocks(blocks, n_heads);
        p.halves_from -= halved;
        n_items += (int64_t)halved * n_heads;
    }
    if (batch->n_graphs > 1 && rows == 2 * kTile && list_saves(batch, rows, n_heads, kListMinSaved)) {
        int4* list = (int4*)((uint8_t*)workspace + kHeaderBytes);
        p.list = list;
        n_items = (int64_t)list_entries(batch, rows) * n_heads;
        const unsigned blocks = (unsigned)((batch->n_graphs + kListThreads / 32 - 1) / (kListThreads / 32));
        if ((st = launch_overlapped(position_list_kernel, dim3(blocks), kListThreads, 0, s, list, (int32_t)list_entries(batch, rows), batch->cu_seqlens,
                                    batch->n_graphs, p.by_work != 0)) != GT_OK)
            return st;
    }
    if (n_items > 0x7fff0000) return GT_ERR_UNSUPPORTED;
    p.n_items = (int32_t)n_items;
    const bool bounded = cap <= kBoundedCap && cap >= kLeastBoundedCap;
    p.reference = bounded ? floorf(0.5f * p.cap2) : 0.f;
    const float coefficients[6] = {position::kTanh0, position::kTanh1, position::kTanh2, position::kTanh3, position::kTanh4, position::kTanh5};
    for (int i = 0; i < 6; ++i) p.tanh[i] = bounded ? (float)(coefficients[i] * std::pow((double)p.cap2, -2.0 * i)) : 0.f;
    p.reach = position::kTanhReach * p.cap2 * p.cap2;
    auto go = [&](auto wide, auto capped, auto sloped) {
        constexpr int D = decltype(wide)::value ? 64 : 32;
        constexpr bool kCap = decltype(capped)::value, kSlope = decltype(sloped)::value;
        auto exact = [&](auto exact_) {
            constexpr bool kExact = decltype(exact_)::value;
            return bounded ? launch<D, kCap ? 1 : 0, kSlope, kExact>(tq, tk, tv, p, batch, rows, s) : launch<D, kCap ? 2 : 0, kSlope, kExact>(tq, tk, tv, p, batch, rows, s);
        };
        return out_f32 ? exact(Tag<true>{}) : exact(Tag<false>{});
    };
    return position::pick(head_dim == 64, cap > 0.f, slopes != nullptr, go);
}
