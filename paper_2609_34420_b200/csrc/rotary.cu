// gt_rotary: rotation of pairs of channels of the queries and keys by position x frequency, and its transpose (the gradient).
//
//     (a, b) -> scale (a cos w - b sin w, a sin w + b cos w),   w = position * frequency[pair]
//
// Bound by memory: every row is read and written once.  A block has some consecutive tokens: it makes the cosines and sines of their
// pairs once for all heads, into shared memory, while its first rows are on their way, and then rotates 32 bytes of a head at a time.
//
// The angle is reduced in fp64: turns = position * frequency / 2 pi, less the next whole number, is off by at most 3 x 2^-53 of itself (three
// roundings), 7.2e-7 rad at an angle of 2^31; in fp32 a position of a million would leave nothing of it.  What is left, half a turn at most, goes to
// sincospi in fp32, whose rounding is off by up to 2^-25 pi, 9.4e-8 rad.
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
    int32_t tokens;            // of a block
    int32_t step_tokens, step_heads;       // from a thread's piece to its next: so many tokens and heads further
    int32_t copy;              // channels behind rot_dim have to be copied (some output is not in place)
    float scale, sin_scale;
};

constexpr int kThreads = 256, kMaxTokens = 32;
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

// (As one vector: element by element, 83 863 rows of 16 + 4 heads of 64 in bf16 took 93 us, not 70.)
template <typename T> __device__ __forceinline__ Piece<T> load_piece(const uint8_t* at)
{
    const uint4 v = *(const uint4*)at;
    return *(const Piece<T>*)&v;
}
template <typename T> __device__ __forceinline__ void store_piece(uint8_t* at, const Piece<T>& v) { *(uint4*)at = *(const uint4*)&v; }

// First row of the document that row t belongs to: the last one that begins at or before it (those without rows lie before).
__device__ __forceinline__ int32_t document_start(const int32_t* __restrict__ cu_seqlens, int32_t n_graphs, int32_t t)
{
    int32_t lo = 0, n = n_graphs;                          // it is one of [lo, lo + n)
    while (n > 1) {
        const int32_t step = n / 2;
        if (cu_seqlens[lo + step] <= t) { lo += step; n -= step; } else n = step;
    }
    return cu_seqlens[lo];
}
__device__ __forceinline__ int32_t position_of(const RotaryParams& p, int32_t t)
{
    return p.positions ? p.positions[t] : p.cu_seqlens ? t - document_start(p.cu_seqlens, p.n_graphs, t) : t;
}

// Cosine and sine of a pair at a position, scaled.
__device__ __forceinline__ float2 turn_of(const RotaryParams& p, int32_t position, double frequency)
{
    double turns = (double)position * (frequency * kTurn);
    turns -= rint(turns);
    float s, c;
    sincospif((float)(2.0 * turns), &s, &c);
    return make_float2(c * p.scale, s * p.sin_scale);
}

// Rows, and in the layout of halves the rotated channels of each half, come in whole pieces of 16 bytes.  A thread takes two pieces of a
// head at a time: two neighbours, or (halves) the same piece of both halves.
template <typename T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const RotaryParams p)
{
    constexpr int kVec = 16 / sizeof(T), kUnits = D / (2 * kVec);       // elements of a piece, pairs of pieces in a head
    constexpr int kAhead = 2;
    __shared__ int32_t s_position[kMaxTokens];
    __shared__ __align__(16) float2 s_turn[kMaxTokens][D / 2];
    grid_wait();
    grid_release();
    const int tid = threadIdx.x, unit = tid % kUnits, all = p.heads[0] + p.heads[1], half = p.rot_dim / 2;
    const int64_t t0 = (int64_t)blockIdx.x * p.tokens;
    int tokens = (int)min((int64_t)p.tokens, (int64_t)p.n_total - t0);
    const bool rotated = unit * kVec < half, mine = rotated || p.copy;
    int at0 = unit * (kInterleaved ? 2 * kVec : kVec), at1 = kInterleaved ? at0 + kVec : at0 + half;      // the thread's pieces within a head
    if (!kInterleaved && !rotated) {
        at0 = p.rot_dim + (unit * kVec - half) * 2;
        at1 = at0 + kVec;
    }
    Piece<T> a[kAhead], b[kAhead];
    int token = tid / kUnits / all, head = tid / kUnits - token * all;        // of the next piece to load, and of the next to store
    int out_token = token, out_head = head;
    auto advance = [&](int& tk, int& hd) {
        tk += p.step_tokens;
        hd += p.step_heads;
        if (hd >= all) { hd -= all; ++tk; }
    };
    auto load = [&](int i) {
        if (mine && token < tokens) {
            const bool second = head >= p.heads[0];
            const uint8_t* src = (second ? p.x[1] : p.x[0]) + (t0 + token) * (second ? p.x_row[1] : p.x_row[0]) +
                                 (head - (second ? p.heads[0] : 0)) * (D * (int)sizeof(T));
            a[i] = load_piece<T>(src + at0 * (int)sizeof(T));
            b[i] = load_piece<T>(src + at1 * (int)sizeof(T));
        }
        advance(token, head);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(i);
    if (p.cu_seqlens) tokens = (int)min((int64_t)tokens, (int64_t)p.cu_seqlens[p.n_graphs] - t0);
    if (tokens <= 0) return;
    if (tid < tokens) s_position[tid] = position_of(p, (int32_t)t0 + tid);
    __syncthreads();
    for (int e = tid; e < tokens * (D / 2); e += kThreads) {
        const int pair = e % (D / 2);
        if (pair < half) s_turn[e / (D / 2)][pair] = turn_of(p, s_position[e / (D / 2)], p.frequencies[pair]);
    }
    __syncthreads();
    if (!mine) return;
    while (out_token < tokens) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (out_token < tokens) {
                if (rotated) {
                    float2 cs[kVec];
#pragma unroll
                    for (int e = 0; e < kVec; e += 2) *(float4*)&cs[e] = *(const float4*)&s_turn[out_token][unit * kVec + e];
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        T* x = kInterleaved ? (e < kVec / 2 ? &a[i].v[2 * e] : &b[i].v[2 * e - kVec]) : &a[i].v[e];
                        T* y = kInterleaved ? x + 1 : &b[i].v[e];
                        const float u = widen(*x), w = widen(*y);
                        if (!kInterleaved || unit * kVec + e < half) {
                            *x = narrow<T>(u * cs[e].x - w * cs[e].y);
                            *y = narrow<T>(u * cs[e].y + w * cs[e].x);
                        }
                    }
                }
                const bool second = out_head >= p.heads[0];
                uint8_t* dst = (second ? p.y[1] : p.y[0]) + (t0 + out_token) * (second ? p.y_row[1] : p.y_row[0]) +
                               (out_head - (second ? p.heads[0] : 0)) * (D * (int)sizeof(T));
                store_piece<T>(dst + at0 * (int)sizeof(T), a[i]);
                store_piece<T>(dst + at1 * (int)sizeof(T), b[i]);
            }
            advance(out_token, out_head);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(i);
    }
}

// Any even number of rotated channels, rows at any element's address: lane i has pair i of every head.
template <typename T, int D, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) rotary_any_kernel(const RotaryParams p)
{
    grid_wait();
    grid_release();
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int32_t end = p.cu_seqlens ? min(p.n_total, p.cu_seqlens[p.n_graphs]) : p.n_total;
    if (t >= end) return;
    const int half = p.rot_dim / 2, i0 = kInterleaved ? 2 * lane : lane, i1 = kInterleaved ? i0 + 1 : i0 + half;
    const float2 cs = turn_of(p, position_of(p, (int32_t)t), lane < half ? p.frequencies[lane] : 0.0);
    for (int h = 0; h < p.heads[0] + p.heads[1]; ++h) {
        const bool second = h >= p.heads[0];
        const int head = h - (second ? p.heads[0] : 0);
        const T* x = (const T*)((second ? p.x[1] : p.x[0]) + t * (second ? p.x_row[1] : p.x_row[0])) + head * D;
        T* y = (T*)((second ? p.y[1] : p.y[0]) + t * (second ? p.y_row[1] : p.y_row[0])) + head * D;
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
gt_status launch_rotary(RotaryParams p, bool pieces, bool interleaved, cudaStream_t s)
{
    if (!pieces) {
        auto kern = interleaved ? rotary_any_kernel<T, D, true> : rotary_any_kernel<T, D, false>;
        return launch_overlapped(kern, dim3((unsigned)(((int64_t)p.n_total + kThreads / 32 - 1) / (kThreads / 32))), kThreads, 0, s, p);
    }
    // Four pairs of pieces per thread (eight: 57 730 rows of 8 + 8 heads of 32 in fp32 41.2 us, not 38.2), fewer where that leaves less than two
    // blocks per SM.  Two of them are on their way at a time (one, or four: 71 -> 74 and 76 us for the rows above).
    const int all = p.heads[0] + p.heads[1], units = D * (int)sizeof(T) / 32, heads = kThreads / units;
    int64_t tokens = 4 * heads / all;
    while (tokens > 1 && (p.n_total + tokens - 1) / tokens < 2 * sm_count()) tokens /= 2;
    p.tokens = (int32_t)(tokens < 1 ? 1 : tokens > kMaxTokens ? kMaxTokens : tokens);
    p.step_tokens = heads / all;
    p.step_heads = heads % all;
    auto kern = interleaved ? rotary_kernel<T, D, true> : rotary_kernel<T, D, false>;
    return launch_overlapped(kern, dim3((unsigned)(((int64_t)p.n_total + p.tokens - 1) / p.tokens)), kThreads, 0, s, p);
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
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > head_dim || reinterpret_cast<uintptr_t>(frequencies) % 8 != 0) return GT_ERR_INVALID_ARG;
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
    if (scaling != GT_ROTARY_PLAIN && (!(factor > 0.0) || !isfinite(factor) || !isfinite(1.0 / factor))) return GT_ERR_INVALID_ARG;
    switch (scaling) {
        case GT_ROTARY_PLAIN: factor = 1.0; break;
        case GT_ROTARY_LINEAR: break;
        case GT_ROTARY_BASE:
            if (rot_dim == 2) return GT_ERR_INVALID_ARG;
            base *= pow(factor, (double)rot_dim / (rot_dim - 2));
            if (!(base > 0.0) || !isfinite(base)) return GT_ERR_INVALID_ARG;
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
        if (!isfinite(frequencies_host[i])) return GT_ERR_INVALID_ARG;
    }
    return GT_OK;
}
