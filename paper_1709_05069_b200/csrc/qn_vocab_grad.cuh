// The kernel behind the calls that give the gradient of a row of logits: the row is read once, its softmax statistics are
// taken, and the gradient is written, with the row in shared memory between the two.
//
// A cluster of C CTAs takes a row; each holds a slice of at most 192 KB.  A row is seen as 16-byte vectors that start at the
// 16-byte boundary at or below its first element, so that whatever its alignment all but its first and last vector move as
// one bulk copy; what those two hold outside the row is filled with -inf.  Each CTA takes its slice's maximum and sums
// relative to it, tells the other CTAs (stores into their shared memory, one cluster barrier), and joins the C partials in
// rank order, so every CTA arrives at the same numbers.  Two passes over shared memory before that barrier and one after
// it cost about 3/128 of a cycle a byte, an eighth of what the bytes take from and to HBM.
//
// An operator Op brings the few elements of a row that are special (a given token, alternatives, a teacher's list):
//   Params, Shared        arguments; its shared memory
//   begin                 reads them; false if the row is padding (its gradient is 0 and it is not read)
//   before_sums           after the slice has arrived: may take elements out of the sums (by -inf in their place)
//   Partial / sums        what a CTA tells the others
//   finish                from the joined partials to the coefficients: gradient_i = e_i (c0 + c1 d_i) with
//                         d_i = (z_i - m) log2(e) / T, e_i = 2^d_i
//   fix                   the special elements' gradients, one after the other
#pragma once

#include "qn_vocab.cuh"

namespace {

using namespace qn;

constexpr int kMaxCluster = 8;

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
// -inf becomes a number that a zero can be multiplied with; NaN does too, but e_i keeps it.
__device__ __forceinline__ f32x2 finite_pair(f32x2 d) {
    float lo, hi;
    unpack2(d, lo, hi);
    return pack2(fmaxf(lo, -1e30f), fmaxf(hi, -1e30f));
}

template <typename T>
struct Lanes;
template <>
struct Lanes<float> {
    __device__ static __forceinline__ f32x2 pair(const uint4& v, int i) {
        return i == 0 ? pack2(__uint_as_float(v.x), __uint_as_float(v.y)) : pack2(__uint_as_float(v.z), __uint_as_float(v.w));
    }
    // running maximum of a thread, several elements side by side; NaN is passed over (the sums keep it)
    struct Max {
        float m = -INFINITY;
        __device__ __forceinline__ void take(const uint4& v) {
            m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(v.x), __uint_as_float(v.y))),
                      fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
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
    struct Max {
        uint32_t m = 0xff80ff80u;
        __device__ static __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
            uint32_t r;
            asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            return r;
        }
        __device__ __forceinline__ void take(const uint4& v) {
            m = max2(max2(m, max2(v.x, v.y)), max2(v.z, v.w));
        }
        __device__ __forceinline__ float get() const {
            return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
        }
    };
};

template <typename T>
__device__ __forceinline__ T masked();
template <>
__device__ __forceinline__ float masked<float>() { return -INFINITY; }
template <>
__device__ __forceinline__ __nv_bfloat16 masked<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80u); }

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
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Store into the same variable of the CTA of rank `to`.
__device__ __forceinline__ void store_remote(void* mine, uint32_t to, float x) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(mine)), "r"(to));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory");
}

// Before a barrier after which a bulk copy may write what this thread wrote.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- geometry ------------------------------------------------------------------------------------------------------

// A CTA's slice of a row: vectors [first, first + count) of the row, in shared memory.
template <typename T>
struct Slice {
    static constexpr int kVec = Storage<T>::kVec;
    uint4* data;
    int32_t vocab, phase;  // elements from the 16-byte boundary to the row's first
    int32_t first, count;

    __device__ __forceinline__ void set(const T* row, int32_t vocab_, int32_t per_cta, uint32_t rank, uint4* data_) {
        data = data_;
        vocab = vocab_;
        phase = static_cast<int32_t>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        const int32_t all = (phase + vocab + kVec - 1) / kVec;
        first = static_cast<int32_t>(rank) * per_cta;
        count = max(0, min(per_cta, all - first));
    }
    __device__ __forceinline__ T* elements() const { return reinterpret_cast<T*>(data); }
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

// Writes the slice's part of a row of zeros.
template <typename T, int NT>
__device__ __forceinline__ void write_zeros(T* out, const Slice<T>& s) {
    const int32_t lo = max(0, s.origin()), hi = min(s.vocab, s.origin() + s.count * Slice<T>::kVec);
    if (lo >= hi) return;
    constexpr int kVec = Slice<T>::kVec;
    const int32_t head = min(hi - lo, static_cast<int32_t>((16 - (reinterpret_cast<uintptr_t>(out + lo) & 15)) / sizeof(T)) % kVec);
    if (static_cast<int>(threadIdx.x) < head) Storage<T>::store1(out + lo + threadIdx.x, 0.0f);
    const int32_t n = (hi - lo - head) / kVec;
    for (int j = threadIdx.x; j < n; j += NT) stg_stream16(out + lo + head + j * kVec, make_uint4(0, 0, 0, 0));
    const int32_t tail = lo + head + n * kVec + threadIdx.x;
    if (tail < hi && static_cast<int>(threadIdx.x) < kVec) Storage<T>::store1(out + tail, 0.0f);
}

// Copies the slice's elements to a row whose alignment is another than the slice's.
template <int NT>
__device__ __forceinline__ void write_shifted(float* out, const Slice<float>& s) {
    const int32_t lo = max(0, s.origin()), hi = min(s.vocab, s.origin() + s.count * 4);
    const float* from = s.elements() - s.origin();
    for (int i = lo + threadIdx.x; i < hi; i += NT) out[i] = from[i];
}
template <int NT>
__device__ __forceinline__ void write_shifted(__nv_bfloat16* out, const Slice<__nv_bfloat16>& s) {
    const int32_t lo = max(0, s.origin()), hi = min(s.vocab, s.origin() + s.count * 8);
    if (lo >= hi) return;
    const uint16_t* from = reinterpret_cast<const uint16_t*>(s.data) - s.origin();
    uint16_t* to = reinterpret_cast<uint16_t*>(out);
    const int32_t head = (reinterpret_cast<uintptr_t>(to + lo) & 2) ? 1 : 0;
    if (head && threadIdx.x == 0) to[lo] = from[lo];
    const int32_t words = (hi - lo - head) / 2;
    for (int w = threadIdx.x; w < words; w += NT) {
        const int32_t i = lo + head + 2 * w;
        *reinterpret_cast<uint32_t*>(to + i) = from[i] | (static_cast<uint32_t>(from[i + 1]) << 16);
    }
    const int32_t tail = lo + head + 2 * words;
    if (tail < hi && threadIdx.x == 0) to[tail] = from[tail];
}

// Coefficients of e_i and e_i d_i in the gradient, and the maximum they are relative to.
struct Gradient {
    float m, c0, c1;
};

template <typename T, int NT, typename Op>
__global__ void __launch_bounds__(NT) row_gradient_kernel(const typename Op::Params p, const int32_t per_cta) {
    constexpr int kVec = Storage<T>::kVec, kPairs = kVec / 2;
    extern __shared__ __align__(128) uint4 slice_data[];
    __shared__ typename Op::Shared sh;
    __shared__ typename Op::Partial inbox[2][kMaxCluster];
    __shared__ __align__(8) uint64_t bar;
    __shared__ int abort;
    __shared__ Gradient result;
    const uint32_t ctas = cluster_size(), rank = cluster_rank();
    const int tid = threadIdx.x;
    if (ctas > 1) cluster_arrive();  // waited for before the first store into another CTA
    if (tid == 0) {
        abort = 0;
        mbar_init(&bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    uint32_t parity = 0;
    int turn = 0;
    bool first_row = true;
    for (int64_t r = blockIdx.x / ctas; r < p.rows; r += gridDim.x / ctas) {
        const T* row = static_cast<const T*>(p.logits) + r * p.row_stride;
        T* out = p.dlogits ? static_cast<T*>(p.dlogits) + r * p.dlogits_stride : nullptr;
        Slice<T> s;
        s.set(row, p.vocab, per_cta, rank, slice_data);
        if (!Op::template begin<NT>(p, sh, r)) {
            if (out) write_zeros<T, NT>(out, s);
            if (rank == 0 && tid == 0) Op::nothing(p, r);
            __syncthreads();  // the operator's shared memory is free for the next row
            continue;
        }

        // the slice: whole vectors as one bulk copy, the row's ends by elements
        const T* base = row - s.phase + static_cast<int64_t>(s.first) * kVec;
        const int32_t fb = s.full_begin(), fe = s.full_end();
        if (tid == 0 && fe > fb) {
            mbar_arrive_expect_tx(&bar, static_cast<uint32_t>(fe - fb) * 16u);
            bulk_load(s.data + fb, base + fb * kVec, static_cast<uint32_t>(fe - fb) * 16u, &bar);
        }
        if (tid < 2 * kVec) {
            const int32_t j = tid < kVec ? 0 : s.count - 1;
            const int32_t e = j * kVec + tid % kVec;
            const bool end = j >= 0 && (j < fb || j >= fe);
            if (s.count > 0 && end) {
                const int32_t i = s.origin() + e;
                s.elements()[e] = i >= 0 && i < s.vocab ? row[i] : masked<T>();
            }
        }
        if (fe > fb) {
            if (!mbar_wait<false>(&bar, parity, &abort)) mbar_wait<false>(&bar, parity, &abort);
            parity ^= 1;
        }
        __syncthreads();
        Op::template before_sums<T, NT>(p, sh, s);  // ends with a barrier
        typename Lanes<T>::Max top;
        for (int j = tid; j < s.count; j += NT) top.take(s.data[j]);
        const float m_all = Op::template slice_max<T, NT>(p, sh, s, top.get());
        const float m = m_all == -INFINITY ? 0.0f : m_all;
        f32x2 sum = 0, moment = 0;
        const f32x2 minus_m = pack2(-m, -m), scale = pack2(p.scale, p.scale);
        if (Op::moments(p)) {
            for (int j = tid; j < s.count; j += NT) {
                const uint4 v = s.data[j];
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const f32x2 d = mul2(add2(Lanes<T>::pair(v, i), minus_m), scale), e = exp2_pair(d);
                    sum = add2(sum, e);
                    moment = fma2(e, finite_pair(d), moment);
                }
            }
        } else {
            for (int j = tid; j < s.count; j += NT) {
                const uint4 v = s.data[j];
#pragma unroll
                for (int i = 0; i < kPairs; ++i)
                    sum = add2(sum, exp2_pair(mul2(add2(Lanes<T>::pair(v, i), minus_m), scale)));
            }
        }
        float s0, s1, e0, e1;
        unpack2(sum, s0, s1);
        unpack2(moment, e0, e1);
        typename Op::Partial mine = Op::template sums<T, NT>(p, sh, s, m_all, s0 + s1, e0 + e1);
        if (abort) mine.poison();
        // every CTA's partial to every CTA, by the first warp; the buffers alternate, so that the next row's partials do
        // not meet a slower CTA that still reads this row's
        if (ctas > 1) {
            if (first_row) cluster_wait();
            first_row = false;
            if (tid < static_cast<int>(ctas)) {  // `mine` is the same in every thread
                constexpr int kWords = sizeof(typename Op::Partial) / 4;
                const float* words = reinterpret_cast<const float*>(&mine);
                float* slot = reinterpret_cast<float*>(&inbox[turn][rank]);
#pragma unroll
                for (int i = 0; i < kWords; ++i) store_remote(slot + i, tid, words[i]);
            }
            __syncwarp();
            cluster_arrive();
            cluster_wait();
        } else {
            if (tid == 0) inbox[turn][0] = mine;
        }
        if (tid == 0) result = Op::finish(p, sh, inbox[turn], static_cast<int>(ctas), r, rank == 0);
        turn ^= 1;
        fence_async();
        __syncthreads();
        if (!out) continue;
        const Gradient g = result;

        const bool aligned = (reinterpret_cast<uintptr_t>(out) & 15) / sizeof(T) == static_cast<uintptr_t>(s.phase);
        T* out_base = out - s.phase + static_cast<int64_t>(s.first) * kVec;
        const f32x2 minus = pack2(-g.m, -g.m), c0 = pack2(g.c0, g.c0), c1 = pack2(g.c1, g.c1);
        const bool moments = Op::moments(p);
        for (int j = tid; j < s.count; j += NT) {
            const uint4 v = s.data[j];
            float x[kVec];
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                const f32x2 d = mul2(add2(Lanes<T>::pair(v, i), minus), scale), e = exp2_pair(d);
                const f32x2 y = moments ? mul2(e, fma2(finite_pair(d), c1, c0)) : mul2(e, c0);
                unpack2(y, x[2 * i], x[2 * i + 1]);
            }
            const uint4 w = Storage<T>::pack(x);
            if (aligned && j >= fb && j < fe) {
                stg_stream16(out_base + j * kVec, w);
            } else if (aligned) {
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const int32_t i = s.origin() + j * kVec + e;
                    if (i >= 0 && i < s.vocab) Storage<T>::store1(out + i, x[e]);
                }
            } else {
                s.data[j] = w;
            }
        }
        __syncthreads();
        if (aligned) {
            Op::template fix<T, NT>(p, sh, s, g, [&](int32_t i, float x) { Storage<T>::store1(out + i, x); });
        } else {
            Op::template fix<T, NT>(p, sh, s, g, [&](int32_t i, float x) { Storage<T>::store1(s.elements() + (i - s.origin()), x); });
            __syncthreads();
            write_shifted<NT>(out, s);
        }
        fence_async();
        __syncthreads();  // shared memory is free for the next row
    }
    if (ctas > 1 && first_row) cluster_wait();
}

// ---- host ----------------------------------------------------------------------------------------------------------

// CTAs a row and vectors a CTA.
struct RowSplit {
    int ctas, per_cta;
};
inline RowSplit split_row(int64_t rows, int64_t vocab, int vec) {
    const int64_t all = (vocab + 2 * vec - 2) / vec;  // vectors, whatever the alignment
    auto per = [&](int c) { return (all + c - 1) / c; };
    int c = 1;
    while (c < kMaxCluster && per(c) * 16 > 72 * 1024) c *= 2;
    while (c < kMaxCluster && rows * c < 2 * qn_sm_count() && per(c) > 512) c *= 2;
    return {c, static_cast<int>(per(c))};
}

template <typename T, int NT, typename Op>
cudaError_t launch_gradient_nt(const typename Op::Params& p, RowSplit split, cudaStream_t st) {
    auto kernel = row_gradient_kernel<T, NT, Op>;
    const size_t smem = static_cast<size_t>(split.per_cta) * 16;
    static bool raised[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!raised[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
        if (e != cudaSuccess) return e;
        raised[dev] = true;
    }
    const int64_t clusters = p.rows < INT32_MAX / kMaxCluster ? p.rows : INT32_MAX / kMaxCluster;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(clusters * split.ctas));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split.ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p, static_cast<int32_t>(split.per_cta));
}

template <typename T, typename Op>
cudaError_t launch_gradient(const typename Op::Params& p, cudaStream_t st) {
    const RowSplit split = split_row(p.rows, p.vocab, Storage<T>::kVec);
    if (split.per_cta >= 1024) return launch_gradient_nt<T, 256, Op>(p, split, st);
    if (split.per_cta >= 256) return launch_gradient_nt<T, 128, Op>(p, split, st);
    return launch_gradient_nt<T, 32, Op>(p, split, st);
}

}  // namespace
