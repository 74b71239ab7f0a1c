// gt_rotary: rotation of pairs of channels of the queries and keys by position x frequency, and its transpose (the gradient).
//
//     (a, b) -> scale (a cos w - b sin w, a sin w + b cos w),   w = position * frequency[pair]
//
// Bound by memory: every row is read and written once.  A warp has a token.  Lane i makes the cosine and sine of pair i (a head has 32
// pairs at most), the lanes pass them on through shared memory, and then every lane keeps those of its own 16-byte pieces in registers
// while it walks over the heads, 32 bytes at a time, of q and of k.
//
// The angle is reduced in fp64: turns = position * frequency / 2 pi, less the next whole number, is off by 2^-52 of itself, 5e-7 rad at
// position 2^31; in fp32 a position of a million would leave nothing of it.  What is left goes to sincospi in fp32.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "attn_common.cuh"

namespace gt {
namespace {

struct RotaryParams {
    const uint8_t* x[2];       // q, k
    uint8_t* y[2];
    int64_t x_row[2];          // bytes from a token's row to the next
    int64_t y_row[2];
    const double* frequencies;
    const int32_t* positions;
    const int32_t* cu_seqlens;
    int32_t n_total, n_graphs;
    int32_t heads[2];
    int32_t rot_dim;
    int32_t copy;              // channels behind rot_dim have to be copied (some output is not in place)
    float scale, sin_scale;
};

constexpr int kThreads = 256, kTokens = kThreads / 32;
constexpr double kTurn = 0.15915494309189533577;         // 1 / 2 pi

template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen(float v) { return v; }
template <> __device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float widen(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half narrow(float v) { return __float2half_rn(v); }

template <typename T> struct alignas(16) Piece { T v[16 / sizeof(T)]; };

// The document that token t belongs to: the last one that begins at or before it (those without tokens lie before); by whole warps.
__device__ __forceinline__ int32_t document_start(const int32_t* __restrict__ cu_seqlens, int32_t n_graphs, int32_t t)
{
    const int lane = threadIdx.x & 31;
    int32_t lo = 0, n = n_graphs, start = 0;               // it is one of [lo, lo + n)
    for (;;) {
        const int32_t step = (n + 31) / 32, x = lane * step;
        const int32_t begin = x < n ? cu_seqlens[lo + x] : 0x7fffffff;
        const int32_t last = __popc(__ballot_sync(0xffffffffu, begin <= t)) - 1;          // (lane 0's begins there)
        start = __shfl_sync(0xffffffffu, begin, last);
        if (step == 1) return start;
        lo += last * step;
        n = min(step, n - last * step);
    }
}

// Cosine and sine of pair `lane` at token t, scaled.
__device__ __forceinline__ float2 turn_of(const RotaryParams& p, int32_t t)
{
    const int lane = threadIdx.x & 31;
    const int32_t position = p.positions ? p.positions[t] : p.cu_seqlens ? t - document_start(p.cu_seqlens, p.n_graphs, t) : t;
    if (lane >= p.rot_dim / 2) return make_float2(1.f, 0.f);
    double turns = (double)position * (p.frequencies[lane] * kTurn);
    turns -= rint(turns);
    float s, c;
    sincospif((float)(2.0 * turns), &s, &c);
    return make_float2(c * p.scale, s * p.sin_scale);
}

// Rows, and in the layout of halves the rotated channels of each half, come in whole pieces of 16 bytes.  A lane has the same two pieces of
// every head that it meets: two neighbours, or (halves) the same piece of both halves.
template <typename T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const RotaryParams p)
{
    constexpr int kVec = 16 / sizeof(T), kUnits = D / (2 * kVec), kHeads = 32 / kUnits;       // elements of a piece, lanes per head, heads at a time
    constexpr int kUnroll = 4;
    __shared__ float2 s_turn[kTokens][D / 2];
    grid_wait();
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * kTokens + warp;
    if (t >= p.n_total) return;
    const int unit = lane % kUnits, all = p.heads[0] + p.heads[1];
    const int half_pieces = p.rot_dim / 2 / kVec;             // halves: pieces per half
    const bool rotated = kInterleaved ? unit * kVec < p.rot_dim / 2 : unit < half_pieces;
    int at0, at1;                                              // first elements of the lane's pieces within a head
    if (kInterleaved) { at0 = unit * 2 * kVec; at1 = at0 + kVec; }
    else if (rotated) { at0 = unit * kVec; at1 = at0 + p.rot_dim / 2; }
    else { at0 = p.rot_dim + (unit - half_pieces) * 2 * kVec; at1 = at0 + kVec; }
    const bool mine = rotated || p.copy;
    auto where = [&](int h, int64_t* from, int64_t* to) -> int {
        const int of = h < p.heads[0] ? 0 : 1, head = h - (of ? p.heads[0] : 0);
        *from = t * p.x_row[of] + (int64_t)head * D * (int)sizeof(T);
        *to = t * p.y_row[of] + (int64_t)head * D * (int)sizeof(T);
        return of;
    };
    Piece<T> a[kUnroll], b[kUnroll];
    auto load = [&](int h0) {
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const int h = h0 + i * kHeads;
            if (h >= all || !mine) continue;
            int64_t from, to;
            const uint8_t* src = p.x[where(h, &from, &to)] + from;
            a[i] = *(const Piece<T>*)(src + at0 * sizeof(T));
            b[i] = *(const Piece<T>*)(src + at1 * sizeof(T));
        }
    };
    load(lane / kUnits);
    if (p.cu_seqlens && t >= p.cu_seqlens[p.n_graphs]) return;
    const float2 turn = turn_of(p, (int32_t)t);
    if (lane < D / 2) s_turn[warp][lane] = turn;
    __syncwarp();
    if (!mine) return;
    float2 cs[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) cs[i] = s_turn[warp][rotated ? unit * kVec + i : 0];
    for (int h0 = lane / kUnits; h0 < all; h0 += kUnroll * kHeads) {
        if (h0 != lane / kUnits) load(h0);
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const int h = h0 + i * kHeads;
            if (h >= all) continue;
            if (rotated) {
                if (kInterleaved) {
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        T* pair = e < kVec / 2 ? &a[i].v[2 * e] : &b[i].v[2 * e - kVec];
                        if (unit * kVec + e < p.rot_dim / 2) {
                            const float x = widen(pair[0]), y = widen(pair[1]);
                            pair[0] = narrow<T>(x * cs[e].x - y * cs[e].y);
                            pair[1] = narrow<T>(x * cs[e].y + y * cs[e].x);
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        const float x = widen(a[i].v[e]), y = widen(b[i].v[e]);
                        a[i].v[e] = narrow<T>(x * cs[e].x - y * cs[e].y);
                        b[i].v[e] = narrow<T>(x * cs[e].y + y * cs[e].x);
                    }
                }
            }
            int64_t from, to;
            uint8_t* dst = p.y[where(h, &from, &to)] + to;
            *(Piece<T>*)(dst + at0 * sizeof(T)) = a[i];
            *(Piece<T>*)(dst + at1 * sizeof(T)) = b[i];
        }
    }
}

// Any even number of rotated channels, rows at any element's address: lane i has pair i of every head.
template <typename T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) rotary_any_kernel(const RotaryParams p)
{
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * kTokens + (threadIdx.x >> 5);
    const int32_t end = p.cu_seqlens ? p.cu_seqlens[p.n_graphs] : p.n_total;
    if (t >= end) return;
    const float2 cs = turn_of(p, (int32_t)t);
    const int half = p.rot_dim / 2, i0 = kInterleaved ? 2 * lane : lane, i1 = kInterleaved ? i0 + 1 : i0 + half;
    for (int h = 0; h < p.heads[0] + p.heads[1]; ++h) {
        const int of = h < p.heads[0] ? 0 : 1, head = h - (of ? p.heads[0] : 0);
        const T* x = (const T*)(p.x[of] + t * p.x_row[of]) + (int64_t)head * D;
        T* y = (T*)(p.y[of] + t * p.y_row[of]) + (int64_t)head * D;
        if (lane < half) {
            const float a = widen(x[i0]), b = widen(x[i1]);
            y[i0] = narrow<T>(a * cs.x - b * cs.y);
            y[i1] = narrow<T>(a * cs.y + b * cs.x);
        }
        if (p.copy)
            for (int c = p.rot_dim + lane; c < D; c += 32) y[c] = x[c];
    }
}

template <typename T, int D>
gt_status launch_rotary(const RotaryParams& p, bool pieces, bool interleaved, cudaStream_t s)
{
    const dim3 grid((unsigned)((p.n_total + kTokens - 1) / kTokens));
    auto kern = pieces ? (interleaved ? rotary_kernel<T, D, true> : rotary_kernel<T, D, false>)
                       : (interleaved ? rotary_any_kernel<T, D, true> : rotary_any_kernel<T, D, false>);
    return launch_overlapped(kern, grid, kThreads, 0, s, p);
}

}  // namespace
}  // namespace gt

extern "C" gt_status gt_rotary(const void* q, const void* k, const double* frequencies, const int32_t* positions,
                               const gt_batch* batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t rot_dim,
                               gt_dtype dtype, int32_t interleaved, float scale, int32_t inverse,
                               int64_t q_stride, int64_t k_stride, int64_t q_out_stride, int64_t k_out_stride,
                               void* q_out, void* k_out, void* stream)
{
    using namespace gt;
    gt_status st = validate_batch(batch);
    if (st != GT_OK) return st;
    if (n_heads < 1 || n_kv_heads < 0 || !q || !q_out || !frequencies || (n_kv_heads > 0 && (!k || !k_out))) return GT_ERR_INVALID_ARG;
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > head_dim) return GT_ERR_INVALID_ARG;
    if (dtype != GT_BF16 && dtype != GT_FP16 && dtype != GT_FP32) return GT_ERR_INVALID_ARG;
    if (head_dim != 32 && head_dim != 64) return GT_ERR_UNSUPPORTED;
    if (n_heads > 65535 || n_kv_heads > 65535) return GT_ERR_UNSUPPORTED;
    const int size = dtype == GT_FP32 ? 4 : 2;
    RotaryParams p{};
    p.x[0] = (const uint8_t*)q; p.x[1] = (const uint8_t*)k;
    p.y[0] = (uint8_t*)q_out; p.y[1] = (uint8_t*)k_out;
    p.heads[0] = n_heads; p.heads[1] = n_kv_heads;
    const int64_t given[4] = {q_stride, k_stride, q_out_stride, k_out_stride};
    bool pieces = interleaved || rot_dim % (32 / size) == 0;
    for (int i = 0; i < 4; ++i) {
        const int of = i & 1;
        const int64_t packed = (int64_t)p.heads[of] * head_dim, row = given[i] == 0 ? packed : given[i];
        if (p.heads[of] == 0) continue;
        if (row < packed || row > ((int64_t)1 << 38)) return GT_ERR_INVALID_ARG;
        (i < 2 ? p.x_row : p.y_row)[of] = row * size;
        const void* base = i < 2 ? (const void*)p.x[of] : (const void*)p.y[of];
        if (reinterpret_cast<uintptr_t>(base) % size != 0) return GT_ERR_INVALID_ARG;
        pieces = pieces && !misaligned16(base) && row * size % 16 == 0;
    }
    for (int of = 0; of < 2; ++of)
        if (p.heads[of] > 0 && (p.x[of] != p.y[of] || p.x_row[of] != p.y_row[of])) p.copy = 1;
    for (int of = 0; of < 2; ++of)
        if (p.heads[of] > 0 && p.x[of] == p.y[of] && p.x_row[of] != p.y_row[of]) return GT_ERR_INVALID_ARG;      // rows over one another's
    if (sm_count() <= 0) return GT_ERR_NO_DEVICE;
    p.frequencies = frequencies;
    p.positions = positions;
    p.cu_seqlens = batch->cu_seqlens;
    p.n_total = batch->n_total;
    p.n_graphs = batch->n_graphs;
    p.rot_dim = rot_dim;
    p.scale = scale;
    p.sin_scale = inverse ? -scale : scale;
    cudaStream_t s = (cudaStream_t)stream;
    if (head_dim == 64)
        return dtype == GT_BF16 ? launch_rotary<__nv_bfloat16, 64>(p, pieces, interleaved, s)
             : dtype == GT_FP16 ? launch_rotary<__half, 64>(p, pieces, interleaved, s) : launch_rotary<float, 64>(p, pieces, interleaved, s);
    return dtype == GT_BF16 ? launch_rotary<__nv_bfloat16, 32>(p, pieces, interleaved, s)
         : dtype == GT_FP16 ? launch_rotary<__half, 32>(p, pieces, interleaved, s) : launch_rotary<float, 32>(p, pieces, interleaved, s);
}

extern "C" gt_status gt_rotary_frequencies(int32_t rot_dim, double base, gt_rotary_scaling scaling, double factor,
                                           double original_length, double low, double high, double* frequencies_host)
{
    if (!frequencies_host || rot_dim < 2 || rot_dim % 2 != 0 || !(base > 0.0) || !isfinite(base)) return GT_ERR_INVALID_ARG;
    if (scaling != GT_ROTARY_PLAIN && (!(factor > 0.0) || !isfinite(factor))) return GT_ERR_INVALID_ARG;
    switch (scaling) {
        case GT_ROTARY_PLAIN: factor = 1.0; break;
        case GT_ROTARY_LINEAR: break;
        case GT_ROTARY_BASE:
            if (rot_dim == 2) return GT_ERR_INVALID_ARG;
            base *= pow(factor, (double)rot_dim / (rot_dim - 2));
            factor = 1.0;
            break;
        case GT_ROTARY_PARTS:
            if (!(original_length > 0.0) || !isfinite(original_length) || !(low >= 0.0) || !(high > low) || !isfinite(high)) return GT_ERR_INVALID_ARG;
            break;
        default: return GT_ERR_INVALID_ARG;
    }
    for (int32_t i = 0; i < rot_dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / rot_dim);
        double kept = 0.0;                                    // share of the frequency that is not scaled
        if (scaling == GT_ROTARY_PARTS) {
            const double r = original_length * f * gt::kTurn;     // turns within the original length
            kept = r <= low ? 0.0 : r >= high ? 1.0 : (r - low) / (high - low);
        }
        frequencies_host[i] = f * ((1.0 - kept) / factor + kept);
    }
    return GT_OK;
}
