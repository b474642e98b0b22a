// qn_distill: a student's loss against a teacher's top logits, and its gradient.
//
// One CTA takes a row.  With e_i = 2^((z_i - m) log2(e) / T) and the student's sums kept apart for the list (S_l) and the
// rest (S_r), S = S_l + S_r: p_k = e_k / S, and the mass off the list p_r = S_r / S comes without a subtraction.
#include <nvtx3/nvToolsExt.h>

#include "qn_vocab.cuh"

namespace {

using namespace qn;

constexpr int kThreads = 256;

struct DistillParams {
    const void* logits;
    int64_t row_stride, rows;
    int32_t vocab, k;
    const int64_t* token;
    const void* value;
    int32_t value_bf16, logprobs;
    float inv_t, scale;  // 1 / T, log2(e) / T
    const float* weight;
    float* loss;
    void* dlogits;
    int64_t dlogits_stride;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) distill_kernel(const DistillParams p) {
    __shared__ float scratch[kThreads / 32];
    __shared__ double scratch_sum[kThreads / 32];
    __shared__ int32_t list[QN_TOP_MAX];
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T* z = static_cast<const T*>(p.logits) + r * p.row_stride;
        T* out = p.dlogits ? static_cast<T*>(p.dlogits) + r * p.dlogits_stride : nullptr;
        const float w = p.weight ? p.weight[r] : 1.0f;
        __syncthreads();  // list of the last row
        // thread j's entry of the teacher's list
        const int j = threadIdx.x;
        const int64_t at = j < p.k ? p.token[r * p.k + j] : -1;
        const bool here = at >= 0 && at < p.vocab;
        if (j < p.k) list[j] = here ? (int32_t)at : -1;
        const bool wrong = __syncthreads_or(at >= p.vocab);
        const int named = __syncthreads_count(here);
        float v = -INFINITY;
        if (here) {
            v = p.value_bf16 ? Storage<__nv_bfloat16>::load1(static_cast<const __nv_bfloat16*>(p.value) + r * p.k + j)
                             : __ldg(static_cast<const float*>(p.value) + r * p.k + j);
        }
        float logq = v, q_rest = 0.0f;
        bool none = named == 0 && !wrong;
        if (p.logprobs) {
            // what is left of 1 may be far smaller than 1: the list is added up in 64 bits
            const double sum = block_reduce<double, add_op>(exp((double)v), scratch_sum);
            if (named < p.vocab) q_rest = sum != sum ? NAN : (float)fmax(0.0, 1.0 - sum);
        } else {
            const float top = block_reduce<float, max_op>(v, scratch);
            if (top == -INFINITY && !__syncthreads_or(v != v)) none = none || !wrong;
            const float d = top == -INFINITY ? -INFINITY : (v - top) * p.inv_t;
            logq = d - logf(block_reduce<float, add_op>(v != v ? NAN : expf(d), scratch));
        }
        if (w == 0.0f || none) {
            if (threadIdx.x == 0) p.loss[r] = 0.0f;
            if (out)
                for (int i = threadIdx.x; i < p.vocab; i += kThreads) Storage<T>::store1(out + i, 0.0f);
            continue;
        }
        const float q = wrong ? NAN : here ? expf(logq) : 0.0f;
        const float mass = block_reduce<float, add_op>(q, scratch) + q_rest;

        const float zj = here ? load_rw(z + at) : -INFINITY;
        float m = -INFINITY;
        for (int i = threadIdx.x; i < p.vocab; i += kThreads) m = fmaxf(m, load_rw(z + i));
        m = block_reduce<float, max_op>(m, scratch);
        const bool empty = m == -INFINITY;
        if (empty) m = 0.0f;
        float rest = 0.0f;
        for (int i = threadIdx.x; i < p.vocab; i += kThreads) {
            bool on = false;
            for (int a = 0; a < p.k; ++a) on = on || list[a] == i;
            if (!on) rest += exp2_approx((load_rw(z + i) - m) * p.scale);
        }
        rest = block_reduce<float, add_op>(rest, scratch);
        const float ej = here ? exp2_approx((zj - m) * p.scale) : 0.0f;
        const float s = rest + block_reduce<float, add_op>(ej, scratch);
        const float log_s = logf(s);
        // q ln q - q ln p, nothing where the teacher has nothing
        float term = wrong ? NAN : q > 0.0f ? q * (logq - ((zj - m) * p.inv_t - log_s)) : q;
        if (empty) term = q > 0.0f ? INFINITY : q;
        if (j == 0 && q_rest > 0.0f) term += q_rest * (logf(q_rest) - (empty ? -INFINITY : logf(rest) - log_s));
        if (j == 0 && q_rest != q_rest) term = NAN;
        const float loss = block_reduce<float, add_op>(term, scratch);
        if (threadIdx.x == 0) p.loss[r] = loss;
        if (!out) continue;
        const float unit = w * p.inv_t;
        const float on_coef = empty ? 0.0f : mass / s;
        const float off_coef = empty ? 0.0f : on_coef - (q_rest > 0.0f && rest > 0.0f ? q_rest / rest : 0.0f);
        __syncthreads();  // every logit of the list is fetched before the row may be overwritten
        for (int i = threadIdx.x; i < p.vocab; i += kThreads)
            Storage<T>::store1(out + i, unit * off_coef * exp2_approx((load_rw(z + i) - m) * p.scale));
        __syncthreads();
        if (here) Storage<T>::store1(out + at, empty ? 0.0f : unit * (on_coef * ej - q));
    }
}

}  // namespace

extern "C" qn_status qn_distill(int64_t rows, int64_t vocab, qn_dtype dtype, const void* logits, int64_t row_stride,
                                int32_t k, const int64_t* teacher_token, qn_dtype teacher_dtype,
                                const void* teacher_value, int32_t teacher, double temperature, const float* weight,
                                float* loss, void* dlogits, int64_t dlogits_stride, void* cuda_stream) {
    if (rows == 0) return QN_OK;
    int dev = -1;
    if (!check_logits(rows, vocab, dtype, logits, row_stride, temperature, &dev)) return QN_ERR_INVALID;
    if (vocab > QN_GRAD_MAX_VOCAB || k < 1 || k > QN_TOP_MAX || rows > INT64_MAX / 8 / QN_TOP_MAX) return QN_ERR_INVALID;
    if (!teacher_token || !teacher_value || !loss) return QN_ERR_INVALID;
    if (teacher_dtype != QN_F32 && teacher_dtype != QN_BF16) return QN_ERR_INVALID;
    if (teacher != QN_TEACHER_LOGITS && teacher != QN_TEACHER_LOGPROBS) return QN_ERR_INVALID;
    if (!check_array(teacher_token, 8, dev) || !check_array(teacher_value, dtype_size(teacher_dtype), dev) ||
        !check_array(weight, 4, dev) || !check_array(loss, 4, dev))
        return QN_ERR_INVALID;
    if (overlaps(loss, rows * 4, logits, matrix_bytes(rows, vocab, row_stride, dtype))) return QN_ERR_INVALID;
    if (dlogits && !check_gradient(rows, vocab, dtype, logits, row_stride, dlogits, dlogits_stride, dev))
        return QN_ERR_INVALID;
    DeviceGuard guard(dev);
    if (!guard.ok) return QN_ERR_CUDA;
    const DistillParams p{logits, row_stride, rows, static_cast<int32_t>(vocab), k, teacher_token, teacher_value,
                          teacher_dtype == QN_BF16, teacher == QN_TEACHER_LOGPROBS,
                          static_cast<float>(1.0 / temperature), static_cast<float>(1.4426950408889634 / temperature),
                          weight, loss, dlogits, dlogits_stride};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const unsigned grid = static_cast<unsigned>(rows < INT32_MAX ? rows : INT32_MAX);
    nvtxRangePushA("qn:distill");
    if (dtype == QN_F32) distill_kernel<float><<<grid, kThreads, 0, st>>>(p);
    else distill_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(p);
    nvtxRangePop();
    return cudaGetLastError() == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
