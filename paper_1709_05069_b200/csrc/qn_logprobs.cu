// qn_logprobs and qn_logprobs_backward: log probabilities over a vocabulary and their gradient.
//
// Forward: one CTA takes a row.  The maximum m, then S = sum e_i and E = sum e_i d_i with d_i = (z_i - m) log2(e) / T and
// e_i = 2^d_i.  z - m is formed before the scale, so that a row of the type's lowest values does not overflow and large
// logits lose nothing to the product's rounding.  lse = m / T + ln S, H = ln S - ln 2 * E / S.
// Backward: an operator of the row-gradient kernel.
#include <nvtx3/nvToolsExt.h>

#include "qn_vocab_grad.cuh"

namespace {

using namespace qn;

constexpr int kThreads = 256;

struct LogprobParams {
    const void* logits;
    int64_t row_stride, rows;
    int32_t vocab, k;
    const int64_t* tokens;
    float inv_t, scale;  // 1 / T, log2(e) / T
    float *logprob, *lse, *entropy;
    int64_t* top_token;
    float* top_logprob;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const LogprobParams p) {
    __shared__ float scratch[kThreads / 32];
    __shared__ uint64_t scratch_key[kThreads / 32];
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T* z = static_cast<const T*>(p.logits) + r * p.row_stride;
        float m = -INFINITY;
        for (int i = threadIdx.x; i < p.vocab; i += kThreads) m = fmaxf(m, Storage<T>::load1(z + i));
        m = block_reduce<float, max_op>(m, scratch);
        const bool empty = m == -INFINITY;
        if (empty) m = 0.0f;
        float s = 0.0f, e = 0.0f;
        for (int i = threadIdx.x; i < p.vocab; i += kThreads) {
            const float zi = Storage<T>::load1(z + i);
            const float d = (zi - m) * p.scale, x = exp2_approx(d);
            s += x;
            if (x != 0.0f) e += x * d;  // 0 * -inf
        }
        s = block_reduce<float, add_op>(s, scratch);
        e = block_reduce<float, add_op>(e, scratch);
        const float log_s = logf(s);  // -inf for an empty row, NaN for a row without a distribution
        const bool bad = s != s;
        if (threadIdx.x == 0) {
            if (p.lse) p.lse[r] = m * p.inv_t + log_s;
            if (p.entropy) p.entropy[r] = s == 0.0f ? 0.0f : log_s - kLn2 * (e / s);
            if (p.logprob) {
                const int64_t t = p.tokens[r];
                float out = 0.0f;
                if (t >= p.vocab || (t >= 0 && bad)) out = NAN;
                else if (t >= 0) out = empty ? -INFINITY : (Storage<T>::load1(z + t) - m) * p.inv_t - log_s;
                p.logprob[r] = out;
            }
        }
        uint64_t last = ~0ull;
        for (int j = 0; j < p.k; ++j) {
            uint64_t best = 0;
            if (last != 0 && !bad)
                for (int i = threadIdx.x; i < p.vocab; i += kThreads) {
                    const float zi = Storage<T>::load1(z + i);
                    const uint64_t key = key_of(zi, i);
                    if (zi > -INFINITY && key < last && key > best) best = key;
                }
            last = block_reduce<uint64_t, max_op>(best, scratch_key);
            if (threadIdx.x == 0) {
                p.top_token[r * p.k + j] = last ? (int64_t)key_index(last) : -1;
                p.top_logprob[r * p.k + j] =
                    bad ? NAN : last ? (key_value(last) - m) * p.inv_t - log_s : -INFINITY;
            }
        }
    }
}

struct BackwardParams {
    const void* logits;
    int64_t row_stride, rows;
    int32_t vocab, k;
    const int64_t* tokens;
    float inv_t, scale;  // 1 / T, log2(e) / T
    const float *d_logprob, *d_lse, *d_entropy;
    const int64_t* top_token;
    const float* d_top;
    void* dlogits;
    int64_t dlogits_stride;
};

// dz_i = 1/T [ p_i (a + b ln p_i) + sparse_i ],  a = d_lse - sum of the sparse terms - d_H H,  b = -d_H.
// The sums leave out one maximal element: S = 1 + s, ln S = log1p(s).  For a row whose maximum has nearly all the
// probability, H and ln p then keep their relative accuracy (s is small and all of H comes from it).
struct Backward {
    using Params = BackwardParams;
    struct Shared {
        int32_t pos[QN_TOP_MAX + 1];  // sparse terms: 0 the given token, 1..k the alternatives; -1 for none
        float add[QN_TOP_MAX + 1], z[QN_TOP_MAX + 1];
        float4 scratch[32];
        float scratch_max[32];
        float total;
        int owner, skipped;
    };
    struct Partial {
        float m, s, e;  // a slice's maximum; sums of e_i and e_i d_i over the rest of it
        __device__ void poison() { s = NAN; }
    };
    __device__ static __forceinline__ bool moments(const Params& p) { return p.d_entropy != nullptr; }
    __device__ static void nothing(const Params&, int64_t) {}

    template <int NT>
    __device__ static bool begin(const Params& p, Shared& sh, int64_t r) {
        float sum = 0.0f;
        bool any = false;
        for (int j = threadIdx.x; j <= p.k; j += NT) {
            float mine = 0.0f;
            int64_t at = -1;
            if (j == 0) {
                if (p.d_logprob) {
                    at = p.tokens[r];
                    if (at >= 0) mine = p.d_logprob[r];
                }
                any = (p.d_lse && p.d_lse[r] != 0.0f) || (p.d_entropy && p.d_entropy[r] != 0.0f);
                sh.owner = NT;
            } else if (p.d_top) {
                at = p.top_token[r * p.k + j - 1];
                if (at >= 0) mine = p.d_top[r * p.k + j - 1];
            }
            if (at >= p.vocab) mine = NAN;
            sh.pos[j] = at >= 0 && at < p.vocab ? static_cast<int32_t>(at) : -1;
            sh.add[j] = mine;
            sum += mine;
            any = any || mine != 0.0f;
        }
        const float total = block_sum4<NT>(make_float4(sum, 0.0f, 0.0f, 0.0f), sh.scratch).x;
        if (threadIdx.x == 0) sh.total = total;
        return __syncthreads_or(any);
    }

    template <typename T, int NT>
    __device__ static void before_sums(const Params& p, Shared& sh, const Slice<T>& s) {
        for (int j = threadIdx.x; j <= p.k; j += NT)
            if (s.holds(sh.pos[j])) sh.z[j] = load_rw(s.elements() + (sh.pos[j] - s.origin()));
        __syncthreads();
    }

    // The slice's maximum.  One element that has it (the first of the first thread that has one) leaves the sums.
    template <typename T, int NT>
    __device__ static float slice_max(const Params&, Shared& sh, const Slice<T>& s, float mine) {
        const float m = block_reduce<float, max_op>(mine, sh.scratch_max);
        if (m == -INFINITY) return m;
        if (mine == m) atomicMin(&sh.owner, static_cast<int>(threadIdx.x));
        __syncthreads();
        if (sh.owner == static_cast<int>(threadIdx.x)) {
            int at = s.count * Slice<T>::kVec;
            for (int j = threadIdx.x; j < s.count; j += NT) {
#pragma unroll
                for (int e = 0; e < Slice<T>::kVec; ++e)
                    if (Storage<T>::get(s.data[j], e) == m) at = min(at, j * Slice<T>::kVec + e);
            }
            sh.skipped = at;
            if (at < s.count * Slice<T>::kVec) s.elements()[at] = masked<T>();
        }
        asm volatile("" ::: "memory");  // the owner itself reads the vector next, and no other thread does
        return m;
    }

    template <typename T, int NT>
    __device__ static Partial sums(const Params&, Shared& sh, const Slice<T>& s, float m, float sum, float moment) {
        const float4 x = block_sum4<NT>(make_float4(sum, moment, 0.0f, 0.0f), sh.scratch);
        if (m != -INFINITY && sh.owner == static_cast<int>(threadIdx.x) && sh.skipped < s.count * Slice<T>::kVec)
            Storage<T>::store1(s.elements() + sh.skipped, m);
        return {m, x.x, x.y};
    }

    __device__ static Gradient finish(const Params& p, Shared& sh, const Partial* part, int n, int64_t r, bool) {
        float m = -INFINITY;
        for (int c = 0; c < n; ++c) m = fmaxf(m, part[c].m);
        float s = 0.0f, e = 0.0f;
        bool left_out = false;
        for (int c = 0; c < n; ++c) {
            const Partial x = part[c];
            if (x.m == -INFINITY) {
                s += x.s;  // 0, or NaN where the slice holds one
            } else if (x.m == m && !left_out) {
                left_out = true;
                s += x.s, e += x.e;
            } else {
                const float d = (x.m - m) * p.scale, f = exp2_approx(d);
                s += f * (1.0f + x.s);
                if (f != 0.0f) e += f * (x.e + d * (1.0f + x.s));
            }
        }
        if (m == INFINITY) s = NAN;
        if (m == -INFINITY && s == 0.0f) return {0.0f, 0.0f, 0.0f};  // empty
        const float d_lse = p.d_lse ? p.d_lse[r] : 0.0f, d_h = p.d_entropy ? p.d_entropy[r] : 0.0f;
        // a + b ln p_i = d_lse - total - d_h (H + ln p_i), with H = ln S - ln 2 e / S and ln p_i = ln 2 d_i - ln S: ln S cancels
        const float unit = p.inv_t / (1.0f + s);
        return {m, unit * (d_lse - sh.total + d_h * (kLn2 * e / (1.0f + s))), -unit * d_h * kLn2};
    }

    template <typename T, int NT, typename Store>
    __device__ static void fix(const Params& p, Shared& sh, const Slice<T>& s, const Gradient& g, Store store) {
        for (int j = threadIdx.x; j <= p.k; j += NT) {
            const int32_t at = sh.pos[j];
            if (!s.holds(at)) continue;
            bool first = true;
            float extra = 0.0f;
            for (int i = 0; i <= p.k; ++i) {  // a token that occurs more than once is written once, by its first entry
                if (sh.pos[i] != at) continue;
                if (i < j) first = false;
                extra += sh.add[i];
            }
            const float d = (sh.z[j] - g.m) * p.scale;
            if (first) store(at, exp2_approx(d) * (g.c0 + g.c1 * fmaxf(d, -1e30f)) + extra * p.inv_t);
        }
    }
};

inline unsigned row_grid(int64_t rows) { return static_cast<unsigned>(rows < INT32_MAX ? rows : INT32_MAX); }

}  // namespace

extern "C" qn_status qn_logprobs(int64_t rows, int64_t vocab, qn_dtype dtype, const void* logits, int64_t row_stride,
                                 const int64_t* tokens, double temperature, float* logprob, float* lse, float* entropy,
                                 int32_t k, int64_t* top_token, float* top_logprob, void* cuda_stream) {
    if (rows == 0) return QN_OK;
    int dev = -1;
    if (!check_logits(rows, vocab, dtype, logits, row_stride, temperature, &dev)) return QN_ERR_INVALID;
    if (k < 0 || k > QN_TOP_MAX || (k > 0) != (top_token != nullptr) || (k > 0) != (top_logprob != nullptr))
        return QN_ERR_INVALID;
    if (rows > INT64_MAX / 8 / (QN_TOP_MAX + 1)) return QN_ERR_INVALID;
    if ((logprob && !tokens) || (!logprob && !lse && !entropy && !k)) return QN_ERR_INVALID;
    if (!check_array(tokens, 8, dev) || !check_array(logprob, 4, dev) || !check_array(lse, 4, dev) ||
        !check_array(entropy, 4, dev) || !check_array(top_token, 8, dev) || !check_array(top_logprob, 4, dev))
        return QN_ERR_INVALID;
    const size_t in_bytes = matrix_bytes(rows, vocab, row_stride, dtype);
    float* const vectors[] = {logprob, lse, entropy};
    for (float* v : vectors)
        if (v && overlaps(v, rows * 4, logits, in_bytes)) return QN_ERR_INVALID;
    if (k && (overlaps(top_token, rows * k * 8, logits, in_bytes) || overlaps(top_logprob, rows * k * 4, logits, in_bytes)))
        return QN_ERR_INVALID;
    DeviceGuard guard(dev);
    if (!guard.ok) return QN_ERR_CUDA;
    const LogprobParams p{logits, row_stride, rows, static_cast<int32_t>(vocab), k, tokens,
                          static_cast<float>(1.0 / temperature), static_cast<float>(1.4426950408889634 / temperature),
                          logprob, lse, entropy, top_token, top_logprob};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:logprobs");
    if (dtype == QN_F32) logprobs_kernel<float><<<row_grid(rows), kThreads, 0, st>>>(p);
    else logprobs_kernel<__nv_bfloat16><<<row_grid(rows), kThreads, 0, st>>>(p);
    nvtxRangePop();
    return cudaGetLastError() == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}

extern "C" qn_status qn_logprobs_backward(int64_t rows, int64_t vocab, qn_dtype dtype, const void* logits,
                                          int64_t row_stride, const int64_t* tokens, double temperature,
                                          const float* d_logprob, const float* d_lse, const float* d_entropy,
                                          int32_t k, const int64_t* top_token, const float* d_top_logprob,
                                          void* dlogits, int64_t dlogits_stride, void* cuda_stream) {
    if (rows == 0) return QN_OK;
    int dev = -1;
    if (!check_logits(rows, vocab, dtype, logits, row_stride, temperature, &dev)) return QN_ERR_INVALID;
    if (!dlogits || vocab > QN_GRAD_MAX_VOCAB || k < 0 || k > QN_TOP_MAX || rows > INT64_MAX / 8 / (QN_TOP_MAX + 1)) return QN_ERR_INVALID;
    if (!d_logprob && !d_lse && !d_entropy && !d_top_logprob) return QN_ERR_INVALID;
    if ((d_logprob && !tokens) || (k > 0) != (d_top_logprob != nullptr) || (k > 0 && !top_token))
        return QN_ERR_INVALID;
    if (!check_array(tokens, 8, dev) || !check_array(d_logprob, 4, dev) || !check_array(d_lse, 4, dev) ||
        !check_array(d_entropy, 4, dev) ||
        !check_array(top_token, 8, dev) || !check_array(d_top_logprob, 4, dev))
        return QN_ERR_INVALID;
    if (!check_gradient(rows, vocab, dtype, logits, row_stride, dlogits, dlogits_stride, dev)) return QN_ERR_INVALID;
    DeviceGuard guard(dev);
    if (!guard.ok) return QN_ERR_CUDA;
    const BackwardParams p{logits,    row_stride, rows,      static_cast<int32_t>(vocab), k, tokens,
                           static_cast<float>(1.0 / temperature), static_cast<float>(1.4426950408889634 / temperature),
                           d_logprob, d_lse, d_entropy, top_token, d_top_logprob, dlogits, dlogits_stride};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:logprobs_backward");
    const cudaError_t e = dtype == QN_F32 ? launch_gradient<float, Backward>(p, st)
                                          : launch_gradient<__nv_bfloat16, Backward>(p, st);
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
