// Shared by the kernels over rows of logits (qn_logprobs.cu, qn_distill.cu): argument checks, reductions, the order of
// logits.
#pragma once

#include <math.h>

#include "qn_device.cuh"
#include "qn_host.h"

namespace {

using namespace qn;

constexpr float kLn2 = 0.6931471805599453f;

// ---- host ----------------------------------------------------------------------------------------------------------

inline size_t dtype_size(qn_dtype t) { return t == QN_F32 ? 4 : 2; }

// Shape, type, temperature and the base pointer of a matrix of logits; the device that holds it.
inline bool check_logits(int64_t rows, int64_t vocab, qn_dtype dtype, const void* logits, int64_t row_stride,
                         double temperature, int* dev) {
    if (!logits || rows < 1 || vocab < 1 || vocab > INT32_MAX - 64 || row_stride < vocab) return false;
    if (dtype != QN_F32 && dtype != QN_BF16) return false;
    if (row_stride > INT64_MAX / 8 / rows || reinterpret_cast<uintptr_t>(logits) % dtype_size(dtype)) return false;
    // 1 / T and log2(e) / T, which the kernels get in 32 bits
    const float inv = static_cast<float>(1.0 / temperature), scale = static_cast<float>(1.4426950408889634 / temperature);
    if (!(temperature > 0.0) || !(inv > 0.0f) || !isfinite(scale)) return false;
    return device_of(logits, dev);
}

// A small array beside the logits: aligned to its element type and on their device; NULL passes.
inline bool check_array(const void* p, size_t elem, int dev) {
    return !p || (reinterpret_cast<uintptr_t>(p) % elem == 0 && on_device(p, dev));
}

inline size_t matrix_bytes(int64_t rows, int64_t vocab, int64_t row_stride, qn_dtype dtype) {
    return static_cast<size_t>((rows - 1) * row_stride + vocab) * dtype_size(dtype);
}

// dlogits takes the place of the logits (same pointer and stride) or does not touch them: the two lie apart, or their rows
// lie between one another's (same stride).
inline bool check_gradient(int64_t rows, int64_t vocab, qn_dtype dtype, const void* logits, int64_t row_stride,
                           const void* dlogits, int64_t dlogits_stride, int dev) {
    if (dlogits_stride < vocab || dlogits_stride > INT64_MAX / 8 / rows) return false;
    if (!check_array(dlogits, dtype_size(dtype), dev)) return false;
    if (dlogits == logits && (dlogits_stride == row_stride || rows == 1)) return true;
    if (!overlaps(dlogits, matrix_bytes(rows, vocab, dlogits_stride, dtype), logits,
                  matrix_bytes(rows, vocab, row_stride, dtype)))
        return true;
    if (dlogits_stride != row_stride) return false;
    // elements from some row of the logits to the next row of dlogits
    const int64_t apart = (reinterpret_cast<intptr_t>(dlogits) - reinterpret_cast<intptr_t>(logits)) /
                          static_cast<int64_t>(dtype_size(dtype));
    const int64_t next = (apart % row_stride + row_stride) % row_stride;
    return next >= vocab && next <= row_stride - vocab;
}

// A launch whose set-up may overlap the end of the stream's last kernel (see start_after_last), as clusters of `ctas`.
struct EarlyLaunch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    EarlyLaunch(int64_t grid, int threads, size_t shared, int ctas, cudaStream_t st) {
        cfg.gridDim = dim3(static_cast<unsigned>(grid));
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = shared;
        cfg.stream = st;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = ctas;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = ctas > 1 ? 2 : 1;
    }
};

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

template <typename V, V (*op)(V, V)>
__device__ __forceinline__ V warp_reduce(V x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = op(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}

// Sums of two values over a CTA of NT threads, in a fixed order, with one pair of barriers.
template <int NT>
__device__ __forceinline__ float2 block_sum2(float2 x, float2* scratch) {
    x.x = warp_reduce<float, add_op>(x.x);
    x.y = warp_reduce<float, add_op>(x.y);
    __syncthreads();  // scratch may still be read from the last use
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    x = scratch[0];
#pragma unroll
    for (int w = 1; w < NT / 32; ++w) {
        const float2 y = scratch[w];
        x.x += y.x, x.y += y.y;
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

// ---- pairs of fp32 (one instruction for two) ---------------------------------------------------------------------

typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 exp2_pair(f32x2 d) {
    float lo, hi;
    unpack2(d, lo, hi);
    return pack2(exp2_approx(lo), exp2_approx(hi));
}
// d_i where e_i d_i is wanted: below kFarBelow, -inf included, e_i is 0 already, and a number that is no larger than needed
// takes the place of d_i, so that its product with an upstream gradient stays finite.  NaN does not stay, but e_i keeps it.
constexpr float kFarBelow = -256.0f;
__device__ __forceinline__ f32x2 finite_pair(f32x2 d) {
    float lo, hi;
    unpack2(d, lo, hi);
    return pack2(fmaxf(lo, kFarBelow), fmaxf(hi, kFarBelow));
}

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

template <typename T>
struct Lanes;
template <>
struct Lanes<float> {
    __device__ static __forceinline__ f32x2 pair(const uint4& v, int i) {
        return i == 0 ? pack2(__uint_as_float(v.x), __uint_as_float(v.y)) : pack2(__uint_as_float(v.z), __uint_as_float(v.w));
    }
    // each element or, if that is larger, `floor`; NaN stays
    __device__ static __forceinline__ uint4 at_least(const uint4& v, float floor) {
        return make_uint4(__float_as_uint(max_nan(__uint_as_float(v.x), floor)), __float_as_uint(max_nan(__uint_as_float(v.y), floor)),
                          __float_as_uint(max_nan(__uint_as_float(v.z), floor)), __float_as_uint(max_nan(__uint_as_float(v.w), floor)));
    }
    // the elements whose bit is set become -inf
    __device__ static __forceinline__ uint4 without(const uint4& v, uint32_t bits) {
        return make_uint4(bits & 1 ? 0xff800000u : v.x, bits & 2 ? 0xff800000u : v.y, bits & 4 ? 0xff800000u : v.z,
                          bits & 8 ? 0xff800000u : v.w);
    }
    __device__ static __forceinline__ uint4 masked4() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    // running maximum of a thread, several elements side by side; NaN if there is one
    struct Max {
        float m = -INFINITY;
        __device__ __forceinline__ void start(float x) { m = x; }
        __device__ __forceinline__ void take(const uint4& v) {
            m = max_nan(max_nan(m, max_nan(__uint_as_float(v.x), __uint_as_float(v.y))),
                        max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
        }
        __device__ __forceinline__ float get() const { return m; }
    };
};
template <>
struct Lanes<__nv_bfloat16> {
    __device__ static __forceinline__ f32x2 pair(const uint4& v, int i) {
        const uint32_t w = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
        return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    __device__ static __forceinline__ uint4 at_least(const uint4& v, float floor) {
        Max f;
        f.start(floor);
        return make_uint4(Max::max2(v.x, f.m), Max::max2(v.y, f.m), Max::max2(v.z, f.m), Max::max2(v.w, f.m));
    }
    __device__ static __forceinline__ uint32_t without2(uint32_t w, uint32_t bits) {
        if (bits & 1) w = (w & 0xffff0000u) | 0xff80u;
        if (bits & 2) w = (w & 0xffffu) | 0xff800000u;
        return w;
    }
    __device__ static __forceinline__ uint4 without(const uint4& v, uint32_t bits) {
        return make_uint4(without2(v.x, bits), without2(v.y, bits >> 2), without2(v.z, bits >> 4), without2(v.w, bits >> 6));
    }
    __device__ static __forceinline__ uint4 masked4() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    struct Max {
        uint32_t m = 0xff80ff80u;
        __device__ __forceinline__ void start(float x) {
            asm("cvt.rn.bf16x2.f32 %0, %1, %1;" : "=r"(m) : "f"(x));
        }
        __device__ static __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
            uint32_t r;
            asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            return r;
        }
        __device__ __forceinline__ void take(const uint4& v) {
            m = max2(max2(m, max2(v.x, v.y)), max2(v.z, v.w));
        }
        __device__ __forceinline__ float get() const {
            return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
        }
    };
};

template <typename T>
__device__ __forceinline__ T masked();
template <>
__device__ __forceinline__ float masked<float>() { return -INFINITY; }
template <>
__device__ __forceinline__ __nv_bfloat16 masked<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80u); }

__device__ __forceinline__ float warp_max_f32(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));  // of numbers, if there are any
    return r;
}

// ---- clusters ------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_remote(const void* mine, uint32_t cta) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(mine)), "r"(cta));
    return at;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Store into the same variable of another CTA of the cluster.
__device__ __forceinline__ void store_remote(const float4* mine, uint32_t cta, float4 x) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(map_remote(mine, cta)), "f"(x.x), "f"(x.y),
                 "f"(x.z), "f"(x.w)
                 : "memory");
}
__device__ __forceinline__ void store_remote(const uint64_t* mine, uint32_t cta, uint64_t x) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(map_remote(mine, cta)), "l"(x) : "memory");
}

// For kernels launched with EarlyLaunch: nothing is read or written before the stream's last kernel has ended; and from
// `let_next_start` on the next such kernel may be set up beside this one (it too waits for this one's end).
__device__ __forceinline__ void start_after_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- geometry ------------------------------------------------------------------------------------------------------

// A CTA's slice of a row: the row's vectors [first, first + count).
template <typename T>
struct Slice {
    static constexpr int kVec = Storage<T>::kVec;
    int32_t vocab, phase;  // elements from the 16-byte boundary to the row's first
    int32_t first, count;

    __device__ __forceinline__ Slice(const T* row, int32_t vocab_, int32_t per_cta, uint32_t rank) {
        vocab = vocab_;
        phase = static_cast<int32_t>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        const int32_t all = (phase + vocab + kVec - 1) / kVec;
        first = static_cast<int32_t>(rank) * per_cta;
        count = max(0, min(per_cta, all - first));
    }
    // row index of the slice's element 0 (negative in a row's first vector)
    __device__ __forceinline__ int32_t origin() const { return first * kVec - phase; }
    __device__ __forceinline__ bool holds(int32_t i) const {
        const int32_t at = i - origin();
        return i >= 0 && at >= 0 && at < count * kVec;
    }
    // vectors of the slice that lie wholly inside the row: [full_begin, full_end), slice-relative
    __device__ __forceinline__ int32_t full_begin() const { return first == 0 && phase > 0 ? 1 : 0; }
    __device__ __forceinline__ int32_t full_end() const {
        return max(full_begin(), min(count, (phase + vocab) / kVec - first));
    }
};

}  // namespace
