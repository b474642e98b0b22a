// Shared by the kernels over rows of logits (qn_logprobs.cu, qn_distill.cu): argument checks, reductions, the order of
// logits.
#pragma once

#include <math.h>

#include "qn_device.cuh"
#include "qn_host.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ---- host ----------------------------------------------------------------------------------------------------------

inline size_t dtype_size(qn_dtype t) { return t == QN_F32 ? 4 : 2; }

// Shape, type, temperature and the base pointer of a matrix of logits; the device that holds it.
inline bool check_logits(int64_t rows, int64_t vocab, qn_dtype dtype, const void* logits, int64_t row_stride,
                         double temperature, int* dev) {
    if (!logits || rows < 1 || vocab < 1 || vocab > INT32_MAX || row_stride < vocab) return false;
    if (dtype != QN_F32 && dtype != QN_BF16) return false;
    if (row_stride > INT64_MAX / 8 / rows || reinterpret_cast<uintptr_t>(logits) % dtype_size(dtype)) return false;
    const float inv = static_cast<float>(1.0 / temperature);
    if (!(temperature > 0.0) || !isfinite(inv) || !(inv > 0.0f)) return false;
    return device_of(logits, dev);
}

// A small array beside the logits: aligned to its element type and on their device; NULL passes.
inline bool check_array(const void* p, size_t elem, int dev) {
    return !p || (reinterpret_cast<uintptr_t>(p) % elem == 0 && on_device(p, dev));
}

inline size_t matrix_bytes(int64_t rows, int64_t vocab, int64_t row_stride, qn_dtype dtype) {
    return static_cast<size_t>((rows - 1) * row_stride + vocab) * dtype_size(dtype);
}

// dlogits takes the place of the logits (same pointer and stride) or does not touch them.
inline bool check_gradient(int64_t rows, int64_t vocab, qn_dtype dtype, const void* logits, int64_t row_stride,
                           const void* dlogits, int64_t dlogits_stride, int dev) {
    if (dlogits_stride < vocab || dlogits_stride > INT64_MAX / 8 / rows) return false;
    if (!check_array(dlogits, dtype_size(dtype), dev)) return false;
    if (dlogits == logits && (dlogits_stride == row_stride || rows == 1)) return true;
    return !overlaps(dlogits, matrix_bytes(rows, vocab, dlogits_stride, dtype), logits,
                     matrix_bytes(rows, vocab, row_stride, dtype));
}

// ---- device --------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A logit whose place the gradient may take in the same launch: an ordinary load, not one through the read-only path.
__device__ __forceinline__ float load_rw(const float* p) { return *p; }
__device__ __forceinline__ float load_rw(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// Order of logits as unsigned integers: larger for a larger logit, equal for -0 and +0.  -inf is 0x007fffff.
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
constexpr uint32_t kOrderMasked = 0x007fffffu;

// One key for a logit and its index: larger for a larger logit and, among equals, for a lower index.  0 is no entry.
__device__ __forceinline__ uint64_t key_of(float z, uint32_t i) {
    return (static_cast<uint64_t>(order_of(z)) << 32) | (0xffffffffu - i);
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return 0xffffffffu - static_cast<uint32_t>(key); }
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t o = static_cast<uint32_t>(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}

__device__ __forceinline__ float add_op(float a, float b) { return a + b; }
__device__ __forceinline__ double add_op(double a, double b) { return a + b; }
__device__ __forceinline__ float max_op(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ uint64_t max_op(uint64_t a, uint64_t b) { return a > b ? a : b; }

template <typename V, V (*op)(V, V)>
__device__ __forceinline__ V warp_reduce(V x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = op(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}

// Sums of four values over the CTA, in a fixed order, with one pair of barriers.
template <int NT>
__device__ __forceinline__ float4 block_sum4(float4 x, float4* scratch) {
    x.x = warp_reduce<float, add_op>(x.x);
    x.y = warp_reduce<float, add_op>(x.y);
    x.z = warp_reduce<float, add_op>(x.z);
    x.w = warp_reduce<float, add_op>(x.w);
    if constexpr (NT == 32) return x;
    __syncthreads();  // scratch may still be read from the last use
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    x = scratch[0];
#pragma unroll
    for (int w = 1; w < NT / 32; ++w) {
        const float4 y = scratch[w];
        x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
    }
    return x;
}

// Over the CTA, in a fixed order; every thread gets the result.  `scratch`: one V for each warp.
template <typename V, V (*op)(V, V)>
__device__ __forceinline__ V block_reduce(V x, V* scratch) {
    x = warp_reduce<V, op>(x);
    __syncthreads();  // scratch may still be read from the last use
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    x = scratch[0];
    for (int w = 1; w < (int)(blockDim.x >> 5); ++w) x = op(x, scratch[w]);
    return x;
}

}  // namespace
