// qn_distill: a student's loss against a teacher's top logits, and its gradient.
//
// An operator of the row-gradient kernel.  With e_i = 2^((z_i - m) log2(e) / T) and the student's sums kept apart for the list (S_l) and the
// rest (S_r), S = S_l + S_r: p_k = e_k / S, and the mass off the list p_r = S_r / S comes without a subtraction.
#include <nvtx3/nvToolsExt.h>

#include "qn_vocab_grad.cuh"

namespace {

using namespace qn;

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

struct Distill {
    using Params = DistillParams;
    struct Shared {
        int32_t pos[QN_TOP_MAX];  // the teacher's list; -1 for an absent token
        float q[QN_TOP_MAX], z[QN_TOP_MAX];
        float4 scratch[32];
        double scratch_sum[32];
        float scratch_max[32];
        float q_sum, q_log_q, q_rest, weight;
        float on, unit;  // gradient on the list: on * e_k - unit * q_k
    };
    struct Partial {
        float m, rest, list, dot, q;  // a slice's maximum; sums of e_i off and on the list; sums of q_k u_k and q_k
        __device__ void poison() { rest = NAN; }
    };
    __device__ static __forceinline__ bool moments(const Params&) { return false; }
    __device__ static void nothing(const Params& p, int64_t r) { p.loss[r] = 0.0f; }

    template <int NT>
    __device__ static bool begin(const Params& p, Shared& sh, int64_t r) {
        const float w = p.weight ? p.weight[r] : 1.0f;
        if (w == 0.0f) return false;
        constexpr int kMine = (QN_TOP_MAX + NT - 1) / NT;
        float v[kMine];
        int named = 0;
        bool wrong = false, finite = false;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int j = threadIdx.x + i * NT;
            v[i] = -INFINITY;
            if (j >= p.k) continue;
            const int64_t at = p.token[r * p.k + j];
            const bool here = at >= 0 && at < p.vocab;
            sh.pos[j] = here ? static_cast<int32_t>(at) : -1;
            wrong = wrong || at >= p.vocab;
            if (!here) continue;
            ++named;
            v[i] = p.value_bf16 ? Storage<__nv_bfloat16>::load1(static_cast<const __nv_bfloat16*>(p.value) + r * p.k + j)
                                : __ldg(static_cast<const float*>(p.value) + r * p.k + j);
            finite = finite || v[i] != -INFINITY;
        }
        wrong = __syncthreads_or(wrong);
        // a row without a teacher: no token at all, or (logits) none that weighs anything
        if (!wrong && !__syncthreads_or(p.logprobs ? named > 0 : finite)) return false;
        float top = 0.0f, log_norm = 0.0f, inv = 1.0f;
        if (!p.logprobs) {
            top = -INFINITY;
#pragma unroll
            for (int i = 0; i < kMine; ++i) top = fmaxf(top, v[i]);
            top = block_reduce<float, max_op>(top, sh.scratch_max);
            if (top == -INFINITY) top = 0.0f;
            inv = p.inv_t;
            double norm = 0.0;
#pragma unroll
            for (int i = 0; i < kMine; ++i) norm += exp(static_cast<double>((v[i] - top) * inv));
            log_norm = static_cast<float>(log(block_reduce<double, add_op>(norm, sh.scratch_sum)));
        }
        // what is left of 1 may be far smaller than 1: the list is added up in 64 bits
        double q_sum = 0.0;
        float q_log_q = 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int j = threadIdx.x + i * NT;
            if (j >= p.k) continue;
            const float log_q = (v[i] - top) * inv - log_norm;
            const double q = exp(static_cast<double>(log_q));
            q_sum += q;
            if (q != 0.0) q_log_q += static_cast<float>(q) * log_q;
            sh.q[j] = static_cast<float>(q);
        }
        q_sum = block_reduce<double, add_op>(q_sum, sh.scratch_sum);
        const float4 x = block_sum4<NT>(make_float4(q_log_q, static_cast<float>(named), 0.0f, 0.0f), sh.scratch);
        if (threadIdx.x == 0) {
            sh.weight = w;
            sh.q_sum = wrong ? NAN : static_cast<float>(q_sum);
            sh.q_log_q = x.x;
            sh.q_rest = 0.0f;
            if (p.logprobs && x.y < static_cast<float>(p.vocab))
                sh.q_rest = q_sum != q_sum ? NAN : static_cast<float>(fmax(0.0, 1.0 - q_sum));
        }
        __syncthreads();
        return true;
    }

    // The list leaves the sums: its logits are kept, and masked in the slice.
    template <typename T, int NT>
    __device__ static void before_sums(const Params& p, Shared& sh, const Slice<T>& s) {
        for (int j = threadIdx.x; j < p.k; j += NT)
            if (s.holds(sh.pos[j])) sh.z[j] = load_rw(s.elements() + (sh.pos[j] - s.origin()));
        __syncthreads();
        for (int j = threadIdx.x; j < p.k; j += NT)
            if (s.holds(sh.pos[j])) s.elements()[sh.pos[j] - s.origin()] = masked<T>();
        __syncthreads();
    }

    template <typename T, int NT>
    __device__ static float slice_max(const Params& p, Shared& sh, const Slice<T>& s, float mine) {
        for (int j = threadIdx.x; j < p.k; j += NT)
            if (s.holds(sh.pos[j])) mine = fmaxf(mine, sh.z[j]);
        return block_reduce<float, max_op>(mine, sh.scratch_max);
    }

    template <typename T, int NT>
    __device__ static Partial sums(const Params& p, Shared& sh, const Slice<T>& s, float m, float sum, float) {
        const float ref = m == -INFINITY ? 0.0f : m;
        float list = 0.0f, dot = 0.0f, q = 0.0f;
        for (int j = threadIdx.x; j < p.k; j += NT) {
            if (!s.holds(sh.pos[j])) continue;
            const float d = sh.z[j] - ref;
            list += exp2_approx(d * p.scale);
            if (sh.q[j] > 0.0f) dot += sh.q[j] * (d * p.inv_t);
            q += sh.q[j];
        }
        const float4 x = block_sum4<NT>(make_float4(sum, list, dot, q), sh.scratch);
        return {m, x.x, x.y, x.z, x.w};
    }

    __device__ static Gradient finish(const Params& p, Shared& sh, const Partial* part, int n, int64_t r, bool first) {
        float m = -INFINITY;
        for (int c = 0; c < n; ++c) m = fmaxf(m, part[c].m);
        float rest = 0.0f, list = 0.0f, dot = 0.0f;
        for (int c = 0; c < n; ++c) {
            const Partial x = part[c];
            const float f = x.m == m || x.m == -INFINITY ? 1.0f : exp2_approx((x.m - m) * p.scale);
            rest += f * x.rest, list += f * x.list;  // a masked slice's are 0, or NaN where it holds one
            dot += x.dot;
            if (x.q > 0.0f && x.m != m) dot += x.q * ((x.m - m) * p.inv_t);
        }
        const float s = m == INFINITY ? NAN : rest + list, q_rest = sh.q_rest, mass = sh.q_sum + q_rest;
        const bool empty = s == 0.0f;
        const float log_s = logf(s);
        if (first) {
            // sum q (ln q - ln p) with ln p = u - m/T - ln S
            float loss = empty ? INFINITY : sh.q_log_q - dot + sh.q_sum * log_s;
            if (!empty && q_rest != 0.0f) loss += q_rest * (logf(q_rest) - (logf(rest) - log_s));
            p.loss[r] = mass != mass ? NAN : loss;
        }
        sh.unit = empty ? 0.0f : sh.weight * p.inv_t;
        sh.on = empty ? 0.0f : sh.unit * (mass / s);
        const float off = q_rest > 0.0f && rest > 0.0f ? mass / s - q_rest / rest : mass / s;
        return {m == -INFINITY ? 0.0f : m, empty ? 0.0f : sh.unit * off, 0.0f};
    }

    template <typename T, int NT, typename Store>
    __device__ static void fix(const Params& p, Shared& sh, const Slice<T>& s, const Gradient& g, Store store) {
        for (int j = threadIdx.x; j < p.k; j += NT)
            if (s.holds(sh.pos[j]))
                store(sh.pos[j], sh.on * exp2_approx((sh.z[j] - g.m) * p.scale) - sh.unit * sh.q[j]);
    }
};

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
    nvtxRangePushA("qn:distill");
    const cudaError_t e = dtype == QN_F32 ? launch_gradient<float, Distill>(p, st)
                                          : launch_gradient<__nv_bfloat16, Distill>(p, st);
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
