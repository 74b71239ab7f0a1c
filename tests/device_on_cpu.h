// What the library's device code uses of its compiler, for host threads in the place of the lanes of one warp: enough for the parts that are
// tested on the CPU.
#pragma once

#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <barrier>
#include <cstring>
#include <random>
#include <thread>
#include <vector>

using std::max;
using std::min;
struct Index { unsigned x; };
static thread_local Index threadIdx, blockIdx, blockDim;
static std::barrier<> g_step(32);
static int g_values[32];
template <typename T> static T __reduce_add_sync(unsigned, T v)
{
    g_values[threadIdx.x] = (int)v;
    g_step.arrive_and_wait();
    int sum = 0;
    for (int x : g_values) sum += x;
    g_step.arrive_and_wait();
    return (T)sum;
}
unsigned __ballot_sync(unsigned, bool);
int __popc(unsigned);
unsigned atomicCAS(uint32_t*, unsigned, unsigned);
size_t __cvta_generic_to_shared(const void*);
static float __uint_as_float(uint32_t x) { float r; memcpy(&r, &x, 4); return r; }
static uint32_t __float_as_uint(float x) { uint32_t r; memcpy(&r, &x, 4); return r; }
static bool __any_sync(unsigned mask, bool x) { return __reduce_add_sync(mask, x ? 1 : 0) != 0; }

#include "attn_position.cuh"
