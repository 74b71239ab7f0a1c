// What the forward and the backward of attention over token sequences share: which keys a query sees, the capped score, argument
// checks.
#pragma once

#include <cuda_bf16.h>

#include "attn_common.cuh"
#include "sm100_primitives.cuh"

namespace gt {
namespace position {

// tanh(y) = y P(y^2) for |y| <= 1: the polynomial of degree 5 in y^2 whose largest relative error on that range is least (by the
// exchange method of Remez), 5.9e-7.  A score x has |x| < cap nearly always, so that its tanh takes FMAs only and the special-function
// unit is left to the exponentials; a warp that meets a larger score takes its tile again with tanh_any.  (tanh.approx.f32 is off by
// 2^-11 relative: a score of 20 by 0.01, its probability by 1 %.)
constexpr float kTanhReach = 1.0f;                 // of y^2
constexpr float kTanh0 = 9.999994136e-01f, kTanh1 = -3.332904238e-01f, kTanh2 = 1.328143388e-01f, kTanh3 = -5.160567400e-02f,
                kTanh4 = 1.674311506e-02f, kTanh5 = -3.067060327e-03f;

template <bool B> struct Tag { static constexpr bool value = B; };

__device__ __forceinline__ uint64_t both(float x) { return sm100::pack_f32x2(x, x); }

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}

// 32 bytes, a whole sector, in one store where the address allows it (`whole`: of all that a kernel writes): 32 lanes that each write a row of
// their own in pieces of 16 bytes send every sector to the L2 twice.
__device__ __forceinline__ void store_sector(void* at, bool whole, const uint32_t (&w)[8])
{
    if (whole)
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    else {
        ((uint4*)at)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        ((uint4*)at)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}
inline bool whole_sectors(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }

// P(u) of two arguments u = y^2.
__device__ __forceinline__ uint64_t tanh_ratio(uint64_t u)
{
    uint64_t r = sm100::fma_f32x2(both(kTanh5), u, both(kTanh4));
    r = sm100::fma_f32x2(r, u, both(kTanh3));
    r = sm100::fma_f32x2(r, u, both(kTanh2));
    r = sm100::fma_f32x2(r, u, both(kTanh1));
    return sm100::fma_f32x2(r, u, both(kTanh0));
}
constexpr float kEx2_0 = 9.999992614e-01f, kEx2_1 = 6.931218147e-01f, kEx2_2 = 2.402474483e-01f, kEx2_3 = 5.591786032e-02f, kEx2_4 = 9.570101911e-03f;
// 2^x of two arguments without the special-function unit: with n the whole number next to x, 2^(x - n) is a polynomial of degree 4 (by the
// exchange method; off by at most 2.6e-6 relative, a thousandth of what a probability loses to bf16) and n goes into the
// exponent by an integer addition.  x is held within [-126, 127]: below, the result is as good as 0; above, and for a NaN, it is far beyond
// what a sum of a tile may be.
__device__ __forceinline__ void ex2_pair(uint64_t x, float& lo, float& hi)
{
    float a, b;
    sm100::unpack_f32x2(x, a, b);
    asm("max.NaN.f32 %0, %0, 0fC2FC0000;\n\tmin.NaN.f32 %0, %0, 0f42FE0000;" : "+f"(a));
    asm("max.NaN.f32 %0, %0, 0fC2FC0000;\n\tmin.NaN.f32 %0, %0, 0f42FE0000;" : "+f"(b));
    x = sm100::pack_f32x2(a, b);
    const uint64_t t = sm100::add_f32x2(x, both(0x1.8p23f));
    const uint64_t f = sm100::fma_f32x2(sm100::add_f32x2(t, both(-0x1.8p23f)), both(-1.f), x);
    uint64_t r = sm100::fma_f32x2(both(kEx2_4), f, both(kEx2_3));
    r = sm100::fma_f32x2(r, f, both(kEx2_2));
    r = sm100::fma_f32x2(r, f, both(kEx2_1));
    r = sm100::fma_f32x2(r, f, both(kEx2_0));
    float t0, t1, r0, r1;
    sm100::unpack_f32x2(t, t0, t1);
    sm100::unpack_f32x2(r, r0, r1);
    lo = __uint_as_float(__float_as_uint(r0) + (__float_as_uint(t0) << 23));
    hi = __uint_as_float(__float_as_uint(r1) + (__float_as_uint(t1) << 23));
}

// tanh(y) of any y: the polynomial within its reach, beyond it 1 - 2 / (1 + e^2y), which is off by 3e-7.
__device__ __forceinline__ float tanh_any(float y)
{
    const float u = y * y;
    float p = fmaf(kTanh5, u, kTanh4), r;
    p = fmaf(p, u, kTanh3);
    p = fmaf(p, u, kTanh2);
    p = fmaf(p, u, kTanh1);
    p = fmaf(p, u, kTanh0) * y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + sm100::ex2_approx(y * (2.0f * kLog2e))));
    return u <= kTanhReach ? p : fmaf(-2.0f, r, 1.0f);
}

// A penalty that is carried from column to column loses 2^-24 of the largest one on the way at each step; on the score of a query's own key, which has
// none, that leaves up to 2^-20 of a slope (backward 2^-16).  Slopes above this (in log2 units; usual ones are below 1) are multiplied out there.
constexpr float kSteep = 64.0f;

// Words of the workspace's header that no other call uses: counters of the persistent kernels, 0 between calls.
constexpr int kNextForward = 16, kNextBackward = 17;

// A query at position i of a document of n tokens sees the document's keys [0, row_limit).
__device__ __forceinline__ int32_t row_limit(bool causal, int32_t i, int32_t prefix, int32_t n) { return causal ? min(n, max(i + 1, prefix)) : n; }

// Work list of a packed batch, by_work: the blocks with the most keys (in the backward: queries) come first, whatever their document;
// block j of a causal document of b blocks has work b - j.  Otherwise (write_work_list) document after document.
template <int kRows>
__device__ __forceinline__ void write_list(int4* list, int32_t entries, const int32_t* __restrict__ cu_seqlens, int32_t n_graphs, int32_t g, bool by_work)
{
    if (!by_work) {
        write_work_list<kRows>(list, entries, cu_seqlens, n_graphs, g);
        return;
    }
    const int lane = threadIdx.x & 31;
    const int32_t c0 = cu_seqlens[g], n = cu_seqlens[g + 1] - c0, blocks = (n + kRows - 1) / kRows;
    int32_t other[kListSorted / 32];                       // a lane's documents' blocks
    int32_t all = 0;
#pragma unroll
    for (int i = 0; i < kListSorted / 32; ++i) {
        const int j = lane + 32 * i;
        other[i] = j < n_graphs ? (cu_seqlens[j + 1] - cu_seqlens[j] + kRows - 1) / kRows : 0;
        all += other[i];
    }
    all = __reduce_add_sync(0xffffffffu, all);
    for (int32_t block = 0; block < blocks; ++block) {
        const int32_t work = blocks - block;
        int32_t before = 0;                                // entries with more work, and with as much of a document before this one
#pragma unroll
        for (int i = 0; i < kListSorted / 32; ++i) before += max(0, other[i] - work) + (lane + 32 * i < g && other[i] >= work ? 1 : 0);
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) list[before] = make_int4(g, block, c0, n);
    }
    if (g == 0)
        for (int32_t i = all + lane; i < entries; i += 32) list[i] = make_int4(-1, 0, 0, 0);
}

// The longest blocks first end soonest, but they walk through all documents at once: only where what the blocks read again (and, in the
// backward, add to) stays in the L2.  64 causal documents of 1 300 tokens, 16 heads of 64: backward 1 345 us and 7.5 GB from and to memory
// by work, 1 052 us and 1.7 GB document after document.
inline bool list_by_work(const gt_batch* b, int32_t causal, size_t bytes) { return causal && b->n_graphs <= kListSorted && bytes <= (size_t)64 << 20; }

// go(Tag<wide>, Tag<capped>, Tag<sloped>) for three values that are known when the program runs.
template <typename Go>
gt_status pick(bool wide, bool capped, bool sloped, Go go)
{
    auto third = [&](auto a, auto b) { return sloped ? go(a, b, Tag<true>{}) : go(a, b, Tag<false>{}); };
    auto second = [&](auto a) { return capped ? third(a, Tag<true>{}) : third(a, Tag<false>{}); };
    return wide ? second(Tag<true>{}) : second(Tag<false>{});
}

constexpr float kMaxCap = 1e6f;
constexpr int64_t kMaxRowStride = (int64_t)1 << 38;

inline gt_status validate(const gt_batch* batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, const int32_t* prefix, int32_t causal,
                          float cap)
{
    const gt_status st = validate_batch(batch);
    if (st != GT_OK) return st;
    if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0) return GT_ERR_INVALID_ARG;
    if (cap != 0.f && !(cap >= 1.f / kMaxCap && cap <= kMaxCap)) return GT_ERR_INVALID_ARG;
    if (!causal && prefix != nullptr) return GT_ERR_INVALID_ARG;
    if (head_dim != 32 && head_dim != 64) return GT_ERR_UNSUPPORTED;
    if (n_heads > 65535 || batch->n_graphs > 65535) return GT_ERR_UNSUPPORTED;
    return GT_OK;
}

// Elements from a row of a [T, heads, d] bf16 tensor to the next; 0: packed.  TMA copies and 16-byte accesses want whole 16 bytes.
inline bool row_stride(int64_t given, int32_t heads, int32_t head_dim, int64_t* stride)
{
    *stride = given == 0 ? (int64_t)heads * head_dim : given;
    return *stride >= (int64_t)heads * head_dim && *stride % 8 == 0 && *stride <= kMaxRowStride;
}

// A wait that may last as long as an item of work does (a document of millions of tokens: a good part of a second), unlike those for a tile.
__device__ __forceinline__ bool item_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* status, uint32_t site)
{
#pragma unroll 1
    for (uint32_t it = 0; it < 64u * sm100::kWaitIterations; ++it) {
        if (sm100::mbar_try_wait(bar, parity)) return true;
        if ((it & 255u) == 255u && *abort_flag) return false;
    }
    return sm100::mbar_wait(bar, parity, abort_flag, status, site);
}

// Whether a warp goes on to an item of n rows: not behind the last one (n 0), and not once a wait was given up, its own for the item (`had`) or
// another warp's.  The flag may be raised between two looks at it, so all that go on together have one look: `any` is true for all of them if
// it is for one, the lanes of a warp, or the warps that meet in named barriers on the way.  (One that left on its own would be waited for without end.)
// The warp that fetches the items writes no description any more once it has given up waiting for its place: others may still work by the old one.
template <typename Any>
__device__ __forceinline__ bool goes_on(bool had, int32_t n, const volatile uint32_t* abort_flag, Any any)
{
    return !any(!had || n <= 0 || *abort_flag != 0u);
}
__device__ __forceinline__ bool warp_any(bool x) { return __any_sync(0xffffffffu, x); }

// Rows [first, 128) of a tile in shared memory are cleared by the calling warp, for MMAs that read the tile afterwards: what lies behind
// a document's last row belongs to another one, and 0 x NaN is NaN.
__device__ __forceinline__ void clear_rows(uint8_t* tile, int first, int row_bytes)
{
    for (int at = first * row_bytes + (int)(threadIdx.x & 31) * 16; at < 128 * row_bytes; at += 512) *(uint4*)(tile + at) = make_uint4(0u, 0u, 0u, 0u);
}

}  // namespace position
}  // namespace gt
