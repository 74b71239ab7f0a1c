// The per-query terms that the backward kernels fold into their MMAs, as three bf16 each (24 mantissa bits).
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace gt {

constexpr float kLargestTerm = 0x1.fdp127f;      // rounds to a finite bf16

// bf16 bits of v's terms, {first, second} in w01 and {third, 0} in w2.  A v that is not finite, or that bf16 does not hold, is taken for zero: its
// row may share a tile with rows of another graph, which meet it multiplied by zero.
__device__ __forceinline__ void fold_term(float v, uint32_t& w01, uint32_t& w2)
{
    if (!(fabsf(v) < kLargestTerm)) v = 0.f;
    const __nv_bfloat16 hi = __float2bfloat16_rn(v);
    const float r1 = v - __bfloat162float(hi);
    const __nv_bfloat16 mid = __float2bfloat16_rn(r1);
    const __nv_bfloat16 lo = __float2bfloat16_rn(r1 - __bfloat162float(mid));
    w01 = (uint32_t)__bfloat16_as_ushort(hi) | ((uint32_t)__bfloat16_as_ushort(mid) << 16);
    w2 = (uint32_t)__bfloat16_as_ushort(lo);
}

}  // namespace gt
