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

// dz_i = 1/T [ p_i (a - d_H (ln p_i + H)) + sparse_i ],  a = d_lse - sum of the sparse terms.
// With E = sum e_i d_i, H = ln S - ln 2 E / S and ln p_i = ln 2 d_i - ln S: in their sum ln S cancels, and
// ln p_i + H = ln 2 (d_i - E / S) keeps its relative accuracy in rows whose maximum has nearly all the probability.
template <bool kEntropy>
struct Backward {
    using Params = BackwardParams;
    static constexpr bool kMoments = kEntropy;
    static constexpr bool kListMessage = false, kMask = false;
    struct Shared {
        int32_t pos[QN_TOP_MAX + 1];  // sparse terms: 0 the given token, 1..k the alternatives; -1 for none
        float add[QN_TOP_MAX + 1], z[QN_TOP_MAX + 1];
        float total, d_lse, d_h;
        Gradient g;
    };
    __device__ static void without(const Params&, int64_t, float) {}
    __device__ static __forceinline__ int entries(const Params& p) { return p.k + 1; }
    struct Extra {
        __device__ __forceinline__ void take(const Params&, const Shared&, int, float) {}
    };

    static constexpr int kMine = QN_TOP_MAX / 32 + 1;  // sparse terms a lane
    struct Fetched {
        int64_t at[kMine];
        float x[kMine], d_lse, d_h;
    };
    __device__ static __forceinline__ Fetched fetch(const Params& p, int64_t r) {
        Fetched f;
        const bool row = r < p.rows;
        f.d_lse = row && p.d_lse ? p.d_lse[r] : 0.0f;
        f.d_h = kEntropy && row ? p.d_entropy[r] : 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int j = (threadIdx.x & 31) + 32 * i;
            f.at[i] = -1;
            f.x[i] = 0.0f;
            if (row && j == 0 && p.d_logprob) f.at[i] = p.tokens[r], f.x[i] = p.d_logprob[r];
            if (row && j >= 1 && j <= p.k) f.at[i] = p.top_token[r * p.k + j - 1], f.x[i] = p.d_top[r * p.k + j - 1];
        }
        return f;
    }
    // a sparse term's gradient: none for an absent token, NaN for one that is not in the vocabulary
    __device__ static __forceinline__ float term(const Params& p, const Fetched& f, int i) {
        return f.at[i] < 0 ? 0.0f : f.at[i] >= p.vocab ? NAN : f.x[i];
    }

    __device__ static __forceinline__ bool wanted(const Params& p, const Fetched& f) {
        bool any = f.d_lse != 0.0f || f.d_h != 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) any = any || term(p, f, i) != 0.0f;
        return __any_sync(0xffffffffu, any);
    }

    __device__ static __forceinline__ void begin(const Params& p, Shared& sh, const Fetched& f) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int j = (threadIdx.x & 31) + 32 * i;
            if (j > p.k) continue;
            sh.pos[j] = f.at[i] >= 0 && f.at[i] < p.vocab ? static_cast<int32_t>(f.at[i]) : -1;
            sh.add[j] = term(p, f, i);
            sum += sh.add[j];
        }
        sum = warp_reduce<float, add_op>(sum);
        if ((threadIdx.x & 31) == 0) sh.total = sum, sh.d_lse = f.d_lse, sh.d_h = f.d_h;
        __syncwarp();
    }

    // messages: a warp's maximum, sums of e_i and e_i d_i
    template <int kWarps>
    __device__ static __forceinline__ void join(const Params& p, Shared& sh, const float4* in, int ctas) {
        const int lane = threadIdx.x & 31;
        float m = -INFINITY;
#pragma unroll 1
        for (int i = lane; i < ctas * kWarps; i += 32) m = fmaxf(m, in[i].x);
        m = warp_max_f32(m);
        float s = 0.0f, e = 0.0f;
#pragma unroll 1
        for (int i = lane; i < ctas * kWarps; i += 32) {
            const float4 v = in[i];
            const float d = v.x == m || v.x == -INFINITY ? 0.0f : (v.x - m) * p.scale, f = exp2_approx(d);
            s += f * v.y;  // masked elements only: 0, or NaN where there is one
            if (kEntropy && f != 0.0f) e += f * (v.z + d * v.y);
        }
        s = warp_reduce<float, add_op>(s);
        if constexpr (kEntropy) e = warp_reduce<float, add_op>(e);
        if (m == INFINITY) s = NAN;
        Gradient g = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (s != 0.0f) {  // not empty
            const float unit = p.inv_t / s;
            g.m = m == -INFINITY ? 0.0f : m;
            g.c0 = unit * (sh.d_lse - sh.total + sh.d_h * (kLn2 * e / s));
            g.c1 = -unit * sh.d_h * kLn2;
        }
        if (lane == 0) sh.g = g;
    }

    template <typename T>
    __device__ static void fix(const Params& p, const Shared& sh, const Slice<T>& s, T* out, int64_t, bool) {
        const Gradient g = sh.g;
#pragma unroll 1
        for (int j = threadIdx.x & 31; j <= p.k; j += 32) {
            const int32_t at = sh.pos[j];
            if (!s.holds(at)) continue;
            bool first = true;
            float extra = 0.0f;
#pragma unroll 1
            for (int i = 0; i <= p.k; ++i) {  // a token that occurs more than once is written once, by its first entry
                if (sh.pos[i] != at) continue;
                if (i < j) first = false;
                extra += sh.add[i];
            }
            const float d = (sh.z[j] - g.m) * p.scale;
            if (first) Storage<T>::store1(out + at, exp2_approx(d) * (g.c0 + g.c1 * fmaxf(d, -1e30f)) + extra * p.inv_t);
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
    const cudaError_t e =
        d_entropy ? (dtype == QN_F32 ? launch_gradient<float, Backward<true>>(p, st)
                                     : launch_gradient<__nv_bfloat16, Backward<true>>(p, st))
                  : (dtype == QN_F32 ? launch_gradient<float, Backward<false>>(p, st)
                                     : launch_gradient<__nv_bfloat16, Backward<false>>(p, st));
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
