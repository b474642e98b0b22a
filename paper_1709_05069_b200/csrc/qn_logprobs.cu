// qn_logprobs and qn_logprobs_backward: log probabilities over a vocabulary and their gradient.
//
// One CTA takes a row.  Forward: the maximum m, then S = sum e_i and E = sum e_i d_i with d_i = (z_i - m) log2(e) / T and
// e_i = 2^d_i.  z - m is formed before the scale, so that a row of the type's lowest values does not overflow and large
// logits lose nothing to the product's rounding.  lse = m / T + ln S, H = ln S - ln 2 * E / S.
#include <nvtx3/nvToolsExt.h>

#include "qn_vocab.cuh"

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
    float inv_t;
    const float *d_logprob, *d_lse, *d_entropy;
    const int64_t* top_token;
    const float* d_top;
    void* dlogits;
    int64_t dlogits_stride;
};

// dz_i = 1/T [ p_i (a + b ln p_i) + sparse_i ].  The row is written without its sparse terms (the given token and the
// alternatives); then those few elements are written again whole, from logits fetched before (dlogits may be the logits).
template <typename T>
__global__ void __launch_bounds__(kThreads) logprobs_backward_kernel(const BackwardParams p) {
    __shared__ float scratch[kThreads / 32];
    __shared__ uint64_t scratch_key[kThreads / 32];
    __shared__ int32_t pos[QN_TOP_MAX + 1];
    __shared__ float add[QN_TOP_MAX + 1];
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T* z = static_cast<const T*>(p.logits) + r * p.row_stride;
        T* out = static_cast<T*>(p.dlogits) + r * p.dlogits_stride;
        __syncthreads();  // pos and add of the last row
        // thread j's sparse term: 0 the given token, 1..k the alternatives
        const int j = threadIdx.x;
        float mine = 0.0f;
        int64_t at = -1;
        if (j == 0 && p.d_logprob) {
            at = p.tokens[r];
            if (at >= 0) mine = p.d_logprob[r];
        } else if (j >= 1 && j <= p.k && p.d_top) {
            at = p.top_token[r * p.k + j - 1];
            if (at >= 0) mine = p.d_top[r * p.k + j - 1];
        }
        if (at >= p.vocab) mine = NAN;
        if (j <= p.k) {
            pos[j] = at >= 0 && at < p.vocab ? (int32_t)at : -1;
            add[j] = mine;
        }
        const float total = block_reduce<float, add_op>(mine, scratch);
        const float d_lse = p.d_lse ? p.d_lse[r] : 0.0f, d_h = p.d_entropy ? p.d_entropy[r] : 0.0f;
        const bool none = !__syncthreads_or(mine != 0.0f) && d_lse == 0.0f && d_h == 0.0f;
        // ln p_i = (z_i - m) / T - ln S with ln S = log1p(sum over all but the maximum): for a row whose maximum has
        // nearly all the probability, ln p and H keep their relative accuracy
        uint64_t best = 0;
        if (!none)
            for (int i = threadIdx.x; i < p.vocab; i += kThreads) best = max_op(best, key_of(load_rw(z + i), i));
        best = block_reduce<uint64_t, max_op>(best, scratch_key);
        float m = key_value(best);
        const bool empty = m == -INFINITY;
        if (empty) m = 0.0f;
        float s = 0.0f, e = 0.0f;
        if (!none)
            for (int i = threadIdx.x; i < p.vocab; i += kThreads) {
                const float zi = load_rw(z + i);
                if (i == (int)key_index(best)) continue;
                const float d = (zi - m) * p.inv_t, x = exp2_approx(d * kLog2e);
                s += x;
                if (x != 0.0f) e += x * d;
            }
        s = block_reduce<float, add_op>(s, scratch);
        e = block_reduce<float, add_op>(e, scratch);
        const float log_s = m - m != 0.0f ? NAN : log1pf(s), h = log_s - e / (1.0f + s);
        const float a = d_lse - total - d_h * h, b = -d_h;
        auto grad = [&](float zi, float extra) {
            const float lp = fmaf(zi - m, p.inv_t, -log_s);
            const float pr = empty ? 0.0f : exp2_approx(lp * kLog2e);
            return (pr * (a + b * fmaxf(lp, -1e30f)) + extra) * p.inv_t;
        };
        float zj = 0.0f, extra = 0.0f;
        bool first = false;
        if (j <= p.k && pos[j] >= 0 && !none) {
            first = true;
            for (int i = 0; i <= p.k; ++i) {
                if (pos[i] != pos[j]) continue;
                if (i < j) first = false;
                extra += add[i];
            }
            if (first) zj = load_rw(z + pos[j]);
        }
        __syncthreads();  // every sparse logit is fetched before the row may be overwritten
        for (int i = threadIdx.x; i < p.vocab; i += kThreads)
            Storage<T>::store1(out + i, none ? 0.0f : grad(load_rw(z + i), 0.0f));
        __syncthreads();
        if (first) Storage<T>::store1(out + pos[j], grad(zj, extra));
    }
}

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
                           static_cast<float>(1.0 / temperature), d_logprob, d_lse, d_entropy, top_token,
                           d_top_logprob, dlogits, dlogits_stride};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:logprobs_backward");
    if (dtype == QN_F32) logprobs_backward_kernel<float><<<row_grid(rows), kThreads, 0, st>>>(p);
    else logprobs_backward_kernel<__nv_bfloat16><<<row_grid(rows), kThreads, 0, st>>>(p);
    nvtxRangePop();
    return cudaGetLastError() == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
