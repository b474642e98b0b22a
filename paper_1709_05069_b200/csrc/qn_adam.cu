// qn_adam_*: plans, the norm of the gradients, and what the states stand for.  The step is in qn_adam_step.cu.
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <new>

#include "qn_adam.cuh"

namespace {

// ---- the norm ------------------------------------------------------------------------------------------------------

// Sum of squares in 64 bits: each CTA's in a fixed order, and the CTAs' sums in theirs, by the last one to come.  (In 64 bits since a
// clip coefficient that differs in its last bit would be other codes in 8-bit states.)  Bound by memory: 2^28 bf16 gradients 88 us =
// 6.1 TB/s; two conversions and two fused operations in 64 bits for two elements are half of what that pipe can do meanwhile.
template <typename G>
__global__ void __launch_bounds__(kThreads) adam_norm_kernel(const Tensors all, double* partials, unsigned* ticket, double* sumsq) {
    __shared__ double scratch[kThreads / 32];
    __shared__ int found;
    __shared__ bool last;
    const Turns turns(all.pieces, 32, 8);
    start_after_last();
    let_next_start();
    double sum = 0.0;
#pragma unroll 1
    for (int turn = 0; turn < turns.count; ++turn) {
        const int64_t lo = turns.lo(turn), hi = turns.hi(turn);
        __syncthreads();
        if (hi > lo) find_tensor(all, lo, &found);
        __syncthreads();
        int tensor = found;
#pragma unroll 1
        for (int64_t piece = lo; piece < hi; ++tensor) {
            const int64_t first = all.first[tensor], from = piece, to = min(hi, all.first[tensor + 1]);
            const G* grad = static_cast<const G*>(all.records[tensor].grad);
            piece = to;
            if (to == from || !grad) continue;
            const int64_t begin = (from - first) * kPiece, end = min(all.records[tensor].numel, (to - first) * kPiece);
            // eight elements a thread from the first vector on; a few by themselves before it and after the last
            constexpr int kBytes = kOctet * sizeof(G);
            const int64_t head = (kBytes - reinterpret_cast<uintptr_t>(grad + begin) % kBytes) % kBytes / sizeof(G), full = min(begin + head, end);
            const int64_t whole = (end - full) / kOctet * kOctet;
            const auto add_one = [&](int64_t i) {
                const double g = Storage<G>::load1(grad + i);
                sum += g * g;
            };
            if (begin + threadIdx.x < full) add_one(begin + threadIdx.x);
            if (full + whole + threadIdx.x < end) add_one(full + whole + threadIdx.x);
#pragma unroll 4
            for (int64_t at = full + threadIdx.x * kOctet; at < full + whole; at += kPiece) {
                uint32_t raw[sizeof(G) == 4 ? 8 : 4];
                load8(grad + at, raw);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float a, b;
                    unpack2(two_of(raw, q), a, b);
                    sum += static_cast<double>(a) * a;
                    sum += static_cast<double>(b) * b;
                }
            }
        }
    }
    sum = block_reduce<double, add_op>(sum, scratch);
    if (threadIdx.x == 0) {
        partials[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kThreads) sum += __ldcg(partials + i);
    sum = block_reduce<double, add_op>(sum, scratch);
    if (threadIdx.x == 0) {
        *ticket = 0;
        *sumsq = sum;
    }
}

// ---- what codes stand for -------------------------------------------------------------------------------------------
// Bound by memory: 2^28 elements to bf16 282 us = 5.8 TB/s, two thirds of it written; 25.6 million whose codes lie off vectors
// 32 us = 4.8 TB/s (a code a lane 52 us).  Six CTAs on an SM: with five, which the compiler would take, 313 and 35 us.

__device__ __forceinline__ void store_value(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_value(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Eight codes at any address, from the words that they lie in: up to three bytes before them and four behind are read too.
__device__ __forceinline__ void load_codes(const uint8_t* p, uint32_t (&x)[2]) {
    const uint32_t shift = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) % 4 * 8;
    const uint32_t* words = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(3));
    const uint32_t a = words[0], b = words[1], c = words[2];
    x[0] = __funnelshift_r(a, b, shift);
    x[1] = __funnelshift_r(b, c, shift);
}

template <typename T, typename S>
__global__ void __launch_bounds__(kThreads, 6) adam_state_kernel(const Tensors all, T* m_out, T* root_out) {
    __shared__ int found;
    const Turns turns(all.pieces, 8, 32);
    start_after_last();
    let_next_start();
#pragma unroll 1
    for (int turn = 0; turn < turns.count; ++turn) {
        const int64_t lo = turns.lo(turn), hi = turns.hi(turn);
        __syncthreads();
        if (hi > lo) find_tensor(all, lo, &found);
        __syncthreads();
        int tensor = found;
#pragma unroll 1
        for (int64_t piece = lo; piece < hi; ++tensor) {
            const Record r = all.records[tensor];
            const int64_t first = all.first[tensor], from = piece, to = min(hi, all.first[tensor + 1]);
            piece = to;
            if (to == from) continue;
            const S *m_at = static_cast<const S*>(r.m), *v_at = static_cast<const S*>(r.v);
            T *m_to = m_out ? m_out + r.octet * kOctet : nullptr, *root_to = root_out ? root_out + r.octet * kOctet : nullptr;
            const int64_t begin = (from - first) * kPiece, whole = (r.numel + QN_ADAM_BLOCK - 1) / QN_ADAM_BLOCK * QN_ADAM_BLOCK;
            const int64_t end = min(whole, (to - first) * kPiece);
            int64_t i = begin + threadIdx.x;
            const auto off = [](const void* p, uint32_t size) { return reinterpret_cast<uintptr_t>(p) & (8u * size - 1u); };
            const auto value = [&](int64_t at, uint32_t m_code, uint32_t v_code, float& m, float& root) {
                m = m_value(m_code, r.m_scale[at / QN_ADAM_BLOCK]);
                root = root_value(v_code, r.v_scale[at / QN_ADAM_BLOCK]);
            };
            const auto put = [&](int64_t at, float m, float root) {
                if (m_to) store_value(m_to + at, m);
                if (root_to) store_value(root_to + at, root);
            };
            const bool vectors = (off(r.m, sizeof(S)) | off(r.v, sizeof(S))) == 0;
            if ((off(m_out, sizeof(T)) | off(root_out, sizeof(T))) == 0 && (vectors || sizeof(S) == 1)) {
                // eight at a time; off vectors those with more of the tensor on both sides (see load_codes)
                const int64_t low = vectors || begin > 0 ? begin : kOctet;
                const int64_t full = min(end, vectors ? r.numel / kOctet * kOctet : (r.numel - 4) / kOctet * kOctet);
                if (low > begin && threadIdx.x < kOctet) {
                    float m = 0.0f, root = 0.0f;
                    if constexpr (sizeof(S) == 1)
                        if (threadIdx.x < r.numel) value(threadIdx.x, m_at[threadIdx.x], v_at[threadIdx.x], m, root);
                    put(threadIdx.x, m, root);
                }
                const auto octets = [&](auto on_vectors) {
                    constexpr bool kVectors = decltype(on_vectors)::value;
#pragma unroll 2
                    for (int64_t a = begin + threadIdx.x * kOctet; a < full; a += kPiece) {
                        if (!kVectors && a < low) continue;
                        f32x2 m2[4], r2[4];
                        float m[8], root[8];
                        uint32_t m_raw[sizeof(S) == 1 ? 2 : 8], v_raw[sizeof(S) == 1 ? 2 : 8];
                        if constexpr (sizeof(S) == 1) {
                            if (kVectors) load8(m_at + a, m_raw), load8(v_at + a, v_raw);
                            else load_codes(m_at + a, m_raw), load_codes(v_at + a, v_raw);
                        } else {
                            load8(m_at + a, m_raw), load8(v_at + a, v_raw);
                        }
                        if constexpr (sizeof(S) == 1) {
                            m_values(m_raw, m2);
                            root_values(v_raw, r2);
                            const f32x2 m_unit = both(power_of(r.m_scale[a / QN_ADAM_BLOCK])), r_unit = both(root_unit(r.v_scale[a / QN_ADAM_BLOCK]));
#pragma unroll
                            for (int q = 0; q < 4; ++q) m2[q] = mul2(m2[q], m_unit), r2[q] = mul2(r2[q], r_unit);
                        } else {
#pragma unroll
                            for (int q = 0; q < 4; ++q) m2[q] = two_of(m_raw, q), r2[q] = two_of(v_raw, q);
                        }
#pragma unroll
                        for (int q = 0; q < 4; ++q) unpack2(m2[q], m[2 * q], m[2 * q + 1]), unpack2(r2[q], root[2 * q], root[2 * q + 1]);
                        if constexpr (sizeof(S) == 4)
#pragma unroll
                            for (float& x : root) x = __fsqrt_rn(x);
                        if (m_to) store8(m_to + a, m);
                        if (root_to) store8(root_to + a, root);
                    }
                };
                if (vectors) octets(std::true_type());
                else if constexpr (sizeof(S) == 1) octets(std::false_type());
                i = max(low, full) + threadIdx.x;
            }
            // element by element, eight loads of each under way together
#pragma unroll 1
            for (; i + 7 * kThreads < min(end, r.numel); i += 8 * kThreads) {
                S m[8], v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) m[e] = m_at[i + e * kThreads], v[e] = v_at[i + e * kThreads];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float a, b;
                    if constexpr (sizeof(S) == 1) value(i + e * kThreads, m[e], v[e], a, b);
                    else a = m[e], b = __fsqrt_rn(v[e]);
                    put(i + e * kThreads, a, b);
                }
            }
#pragma unroll 1
            for (; i < end; i += kThreads) {
                float m = 0.0f, root = 0.0f;
                if (i < r.numel) {
                    if constexpr (sizeof(S) == 1) value(i, m_at[i], v_at[i], m, root);
                    else m = m_at[i], root = __fsqrt_rn(v_at[i]);
                }
                put(i, m, root);
            }
        }
    }
}

// ---- other gradients -------------------------------------------------------------------------------------------------

constexpr int kPointers = 256;
struct Pointers {
    const void* at[kPointers];
};
__global__ void adam_grads_kernel(Record* records, const __grid_constant__ Pointers p, int first, int count) {
    const int i = threadIdx.x;
    if (i < count) records[first + i].grad = p.at[i];
}

// ---- host ------------------------------------------------------------------------------------------------------------

bool add_range(std::vector<std::pair<uintptr_t, uintptr_t>>& ranges, const void* p, size_t bytes, size_t align, int dev) {
    if (!p || !check_array(p, align, dev)) return false;
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    ranges.emplace_back(at, at + bytes);
    return true;
}

// A gradient is read only: it may lie anywhere but in what a step writes.
bool check_grad(const qn_adam_plan& h, const void* p, int64_t numel) {
    const size_t size = dtype_size(h.grad);
    if (!check_array(p, size, h.device)) return false;
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p), hi = lo + numel * size;
    const auto next = std::upper_bound(h.written.begin(), h.written.end(), std::make_pair(lo, ~uintptr_t(0)));
    if (next != h.written.end() && next->first < hi) return false;
    return next == h.written.begin() || (next - 1)->second <= lo;
}

qn_status create(int32_t count, const qn_adam_tensor* tensors, qn_dtype param, qn_dtype grad, int32_t state, qn_adam_handle* out) {
    qn_adam_plan h;
    h.count = count;
    h.param = param;
    h.grad = grad;
    h.eight = state == QN_STATE_8BIT;
    std::vector<Record> records(count);
    std::vector<int64_t> first(count + 1);
    bool found = false;
    for (int32_t i = 0; i < count; ++i) {
        const qn_adam_tensor& t = tensors[i];
        if (t.numel < 0 || t.numel > (int64_t(1) << 40) || h.places > (int64_t(1) << 42)) return QN_ERR_INVALID;
        if (!(t.weight_decay >= 0.0) || !(t.lr_scale >= 0.0) || !isfinite(t.weight_decay) || !isfinite(t.lr_scale))
            return QN_ERR_INVALID;
        records[i] = Record{t.numel, h.places / kOctet, t.param, t.grad, t.master, t.m, t.v, t.m_scale, t.v_scale, t.weight_decay, t.lr_scale};
        h.numel.push_back(t.numel);
        first[i] = h.pieces;
        if (t.numel == 0) continue;
        const int64_t blocks = (t.numel + QN_ADAM_BLOCK - 1) / QN_ADAM_BLOCK;
        if (!found) {
            if (!t.param || !device_of(t.param, &h.device)) return QN_ERR_INVALID;
            h.master = t.master != nullptr;
            if (h.master && param != QN_BF16) return QN_ERR_INVALID;
            found = true;
        }
        if (h.master != (t.master != nullptr) || h.eight != (t.m_scale != nullptr) || h.eight != (t.v_scale != nullptr))
            return QN_ERR_INVALID;
        const size_t each = h.eight ? 1 : 4;
        if (!add_range(h.written, t.param, t.numel * dtype_size(param), dtype_size(param), h.device) ||
            (h.master && !add_range(h.written, t.master, t.numel * 4, 4, h.device)) ||
            !add_range(h.written, t.m, t.numel * each, each, h.device) ||
            !add_range(h.written, t.v, t.numel * each, each, h.device) ||
            (h.eight && (!add_range(h.written, t.m_scale, blocks, 1, h.device) ||
                         !add_range(h.written, t.v_scale, blocks, 1, h.device))))
            return QN_ERR_INVALID;
        h.places += blocks * QN_ADAM_BLOCK;
        h.pieces += (t.numel + kPiece - 1) / kPiece;
    }
    first[count] = h.pieces;
    std::sort(h.written.begin(), h.written.end());
    for (size_t i = 1; i < h.written.size(); ++i)
        if (h.written[i].first < h.written[i - 1].second) return QN_ERR_INVALID;
    for (int32_t i = 0; i < count; ++i)
        if (records[i].numel && records[i].grad && !check_grad(h, records[i].grad, records[i].numel)) return QN_ERR_INVALID;
    if (h.device < 0 && cudaGetDevice(&h.device) != cudaSuccess) return QN_ERR_CUDA;
    DeviceGuard guard(h.device);
    if (!guard.ok) return QN_ERR_CUDA;
    const size_t record_bytes = count * sizeof(Record), first_bytes = first.size() * sizeof(int64_t);
    const size_t partial_bytes = static_cast<size_t>(kMostCtas) * qn_sm_count() * sizeof(double);
    if (cudaMalloc(&h.block, record_bytes + first_bytes + partial_bytes + 64) != cudaSuccess) {
        cudaGetLastError();
        return QN_ERR_ALLOC;
    }
    char* at = static_cast<char*>(h.block);
    h.records = reinterpret_cast<Record*>(at);
    h.first = reinterpret_cast<int64_t*>(at += record_bytes);
    h.partials = reinterpret_cast<double*>(at += first_bytes);
    h.tickets = reinterpret_cast<unsigned*>(at += partial_bytes);
    // blocking copies from this call's own memory: nothing is left to do when it returns
    if ((record_bytes && cudaMemcpy(h.records, records.data(), record_bytes, cudaMemcpyHostToDevice) != cudaSuccess) ||
        cudaMemcpy(h.first, first.data(), first_bytes, cudaMemcpyHostToDevice) != cudaSuccess ||
        cudaMemset(h.tickets, 0, 64) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
        cudaGetLastError();
        cudaFree(h.block);
        return QN_ERR_CUDA;
    }
    *out = new (std::nothrow) qn_adam_plan(std::move(h));
    if (!*out) {
        cudaFree(h.block);
        return QN_ERR_ALLOC;
    }
    return QN_OK;
}

}  // namespace

extern "C" qn_status qn_adam_create(int32_t count, const qn_adam_tensor* tensors, qn_dtype param, qn_dtype grad, int32_t state,
                                    qn_adam_handle* out) {
    if (!out) return QN_ERR_INVALID;
    *out = nullptr;
    if (count < 0 || count > (1 << 20) || (count && !tensors)) return QN_ERR_INVALID;
    if ((param != QN_F32 && param != QN_BF16) || (grad != QN_F32 && grad != QN_BF16)) return QN_ERR_INVALID;
    if (state != QN_STATE_F32 && state != QN_STATE_8BIT) return QN_ERR_INVALID;
    try {
        return create(count, tensors, param, grad, state, out);
    } catch (...) {  // host memory
        return QN_ERR_ALLOC;
    }
}

extern "C" qn_status qn_adam_destroy(qn_adam_handle h) {
    if (!h) return QN_ERR_INVALID;
    {
        DeviceGuard guard(h->device);
        cudaFree(h->block);  // waits for what uses it
    }
    delete h;
    return QN_OK;
}

extern "C" int64_t qn_adam_places(qn_adam_handle h) { return h ? h->places : 0; }

extern "C" qn_status qn_adam_grads(qn_adam_handle h, const void* const* grads, void* cuda_stream) {
    if (!h || (h->count && !grads)) return QN_ERR_INVALID;
    for (int32_t i = 0; i < h->count; ++i)
        if (h->numel[i] && grads[i] && !check_grad(*h, grads[i], h->numel[i])) return QN_ERR_INVALID;
    DeviceGuard guard(h->device);
    if (!guard.ok) return QN_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    for (int32_t first = 0; first < h->count; first += kPointers) {
        Pointers p;
        const int here = std::min(kPointers, h->count - first);
        for (int i = 0; i < kPointers; ++i) p.at[i] = i < here ? grads[first + i] : nullptr;
        adam_grads_kernel<<<1, kPointers, 0, st>>>(h->records, p, first, here);
        if (cudaGetLastError() != cudaSuccess) return QN_ERR_CUDA;
    }
    return QN_OK;
}

extern "C" qn_status qn_adam_norm(qn_adam_handle h, double* sumsq, void* cuda_stream) {
    if (!h || !sumsq || !check_array(sumsq, 8, h->device)) return QN_ERR_INVALID;
    DeviceGuard guard(h->device);
    if (!guard.ok) return QN_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    static Resident resident[2];
    nvtxRangePushA("qn:adam_norm");
    const cudaError_t e = h->grad == QN_F32 ? launch_over(adam_norm_kernel<float>, resident[0], 0, *h, st, h->partials, h->tickets + 1, sumsq)
                                            : launch_over(adam_norm_kernel<__nv_bfloat16>, resident[1], 0, *h, st, h->partials, h->tickets + 1, sumsq);
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}

extern "C" qn_status qn_adam_state(qn_adam_handle h, qn_dtype dtype, void* m, void* root, void* cuda_stream) {
    if (!h || (dtype != QN_F32 && dtype != QN_BF16)) return QN_ERR_INVALID;
    const size_t size = dtype_size(dtype), bytes = h->places * size;
    if (!check_array(m, size, h->device) || !check_array(root, size, h->device)) return QN_ERR_INVALID;
    if (m && root && overlaps(m, bytes, root, bytes)) return QN_ERR_INVALID;
    for (const auto& range : h->written)
        for (const void* p : {m, root})
            if (p && overlaps(p, bytes, reinterpret_cast<const void*>(range.first), range.second - range.first)) return QN_ERR_INVALID;
    if (h->pieces == 0 || (!m && !root)) return QN_OK;
    DeviceGuard guard(h->device);
    if (!guard.ok) return QN_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:adam_state");
    const auto by_type = [&](auto t) {
        using T = decltype(t);
        static Resident resident[2];
        T *m_out = static_cast<T*>(m), *root_out = static_cast<T*>(root);
        return h->eight ? launch_over(adam_state_kernel<T, uint8_t>, resident[1], 0, *h, st, m_out, root_out)
                        : launch_over(adam_state_kernel<T, float>, resident[0], 0, *h, st, m_out, root_out);
    };
    const cudaError_t e = dtype == QN_F32 ? by_type(float()) : by_type(__nv_bfloat16());
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
