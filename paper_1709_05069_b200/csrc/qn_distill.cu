// qn_distill: a student's loss against a teacher's top logits, and its gradient.
//
// An operator of the row-gradient kernels.  With e_i = 2^((z_i - m) log2(e) / T) and the student's sums kept apart for the
// list (S_l) and the rest (S_r), S = S_l + S_r: p_k = e_k / S, and the mass off the list p_r = S_r / S comes without a
// subtraction (its relative error would be that of S times S / S_r).  S_r is kept relative to the largest logit off the list,
// m_r, and so is the gradient there: in a row whose list leads by more than 87 T, S_r relative to m would be 0, where
// ln p_r = (m_r - m) / T + ln S_r - ln S and the softmax over the rest, e_i / S_r, are ordinary numbers.
// The list's own sums, 1 - sum q and the loss are in 64 bits.
// One launch gives the loss and the gradient; what bounds it and what it measured is in qn_vocab_grad.cuh.
#include <nvtx3/nvToolsExt.h>

#include "qn_vocab_grad.cuh"

namespace {

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

// Out of line: it is called for every entry of the list, and instruction cache is scarce in this kernel.
__device__ __noinline__ double exp64(double x) { return exp(x); }
__device__ __noinline__ double log64(double x) { return log(x); }

constexpr float kNothing = 1442.695f;  // log2(e) * 1000

struct Distill {
    using Params = DistillParams;
    static constexpr bool kMoments = false, kMask = true;
    static constexpr bool kAlone = true;  // it may be called without a gradient to write
    static constexpr int kMine = QN_TOP_MAX / 32;  // entries of the list a lane
    struct Shared {
        int32_t pos[QN_TOP_MAX];  // the teacher's list; -1 for an absent token
        float q[QN_TOP_MAX], z[QN_TOP_MAX];
        double q_total, q_log_q;  // of the q as rounded to 32 bits
        float q_sum, q_rest, q_noise, weight;  // q_noise: what rounding of the values may leave of 1 - sum q
        float list_m, list_s;  // of the list's logits: the largest, sum of e_k relative to it
        bool lost;             // the student masks a token that the teacher does not, however little it weighs
        Gradient g;             // off the list: relative to m_rest
        float m, m_rest;        // the largest of the row (0 if it is empty), and of what is off the list
        float rest, s;          // the sums relative to these
    };
    __device__ static void without(const Params& p, int64_t r, float loss) { p.loss[r] = loss; }
    __device__ static __forceinline__ int entries(const Params& p) { return p.k; }

    struct Fetched {
        int64_t at[kMine];
        float v[kMine], z[kMine], weight;
    };
    __device__ static __forceinline__ Fetched fetch(const Params& p, int64_t r) {
        Fetched f;
        const bool row = r < p.rows;
        f.weight = row && p.weight ? p.weight[r] : 1.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int j = (threadIdx.x & 31) + 32 * i;
            const int64_t entry = r * p.k + j;
            f.at[i] = -1;
            f.v[i] = -INFINITY;
            if (!row || j >= p.k) continue;
            f.at[i] = p.token[entry];
            f.v[i] = p.value_bf16 ? Storage<__nv_bfloat16>::load1(static_cast<const __nv_bfloat16*>(p.value) + entry)
                                  : __ldg(static_cast<const float*>(p.value) + entry);
        }
        return f;
    }

    template <typename T>
    __device__ static __forceinline__ void gather(const Params& p, int64_t r, Fetched& f) {
        const T* row = static_cast<const T*>(p.logits) + r * p.row_stride;
#pragma unroll
        for (int i = 0; i < kMine; ++i) f.z[i] = f.at[i] >= 0 && f.at[i] < p.vocab ? load_rw(row + f.at[i]) : -INFINITY;
    }

    // false: weight 0, or no teacher (no token at all, or of logits none that weighs anything)
    __device__ static __forceinline__ bool wanted(const Params& p, const Fetched& f) {
        bool any = false;
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            any = any || f.at[i] >= p.vocab || (f.at[i] >= 0 && (p.logprobs || f.v[i] != -INFINITY));
        return __any_sync(0xffffffffu, any) && f.weight != 0.0f;
    }

    __device__ static __forceinline__ void begin(const Params& p, Shared& sh, const Fetched& f) {
        const int lane = threadIdx.x & 31;
        float v[kMine];
        int named = 0;
        bool wrong = false;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int j = lane + 32 * i;
            const bool here = f.at[i] >= 0 && f.at[i] < p.vocab;
            v[i] = here ? f.v[i] : -INFINITY;
            wrong = wrong || f.at[i] >= p.vocab;
            named += here;
            if (j < p.k) sh.pos[j] = here ? static_cast<int32_t>(f.at[i]) : -1;
        }
        named = __reduce_add_sync(0xffffffffu, named);
        wrong = __any_sync(0xffffffffu, wrong);
        float top = 0.0f, inv = 1.0f;
        double log_norm = 0.0;
        if (!p.logprobs) {
            top = -INFINITY;
#pragma unroll
            for (int i = 0; i < kMine; ++i) top = fmaxf(top, v[i]);
            top = warp_reduce<float, max_op>(top);
            if (top == -INFINITY) top = 0.0f;
            inv = p.inv_t;
            double norm = 0.0;
#pragma unroll
            for (int i = 0; i < kMine; ++i) norm += exp64((static_cast<double>(v[i]) - top) * inv);
            log_norm = log64(warp_reduce<double, add_op>(norm));
        }
        // what is left of 1 may be far smaller than 1: the list is added up in 64 bits
        double q_sum = 0.0;
        double q_total = 0.0, q_log_q = 0.0;
        bool lost = false;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int j = lane + 32 * i;
            if (j >= p.k) continue;
            const double log_q = (static_cast<double>(v[i]) - top) * inv - log_norm, q = exp64(log_q);
            q_sum += q;
            lost = lost || (q > 0.0 && f.z[i] == -INFINITY);
            const float q32 = static_cast<float>(q);
            if (q32 != 0.0f) q_log_q += q32 * log_q;
            q_total += q32;
            sh.q[j] = q32;
        }
        float list_m = -INFINITY, list_s = 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) list_m = fmaxf(list_m, f.z[i]);
        list_m = warp_max_f32(list_m);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (f.at[i] < 0 || f.at[i] >= p.vocab) continue;
            list_s += exp2_approx((f.z[i] - (list_m == -INFINITY ? 0.0f : list_m)) * p.scale);
            sh.z[lane + 32 * i] = f.z[i];
        }
        list_s = warp_reduce<float, add_op>(list_s);
        q_sum = warp_reduce<double, add_op>(q_sum);
        q_total = warp_reduce<double, add_op>(q_total);
        q_log_q = warp_reduce<double, add_op>(q_log_q);
        lost = __any_sync(0xffffffffu, lost);
        if (lane == 0) {
            sh.weight = f.weight;
            sh.lost = lost;
            sh.list_m = list_m;
            sh.list_s = list_s;
            sh.q_sum = wrong ? NAN : static_cast<float>(q_sum);
            sh.q_total = q_total;
            sh.q_log_q = q_log_q;
            sh.q_rest = 0.0f;
            sh.q_noise = static_cast<float>(q_total - q_log_q) * (p.value_bf16 ? 0x1p-9f : 0x1p-18f);
            if (p.logprobs && named < p.vocab) sh.q_rest = q_sum != q_sum ? NAN : static_cast<float>(fmax(0.0, 1.0 - q_sum));
        }
        __syncwarp();
    }

    // messages: a warp's maximum and sum of e_i off the list
    template <int kWarps>
    __device__ static __forceinline__ void join(const Params& p, Shared& sh, const float4* in, int ctas) {
        const int lane = threadIdx.x & 31, all = ctas * kWarps;
        float m_rest = -INFINITY;
#pragma unroll 1
        for (int i = lane; i < all; i += 32) m_rest = fmaxf(m_rest, in[i].x);
        m_rest = warp_max_f32(m_rest);
        const float m = fmaxf(m_rest, sh.list_m);
        float rest = 0.0f;
#pragma unroll 1
        for (int i = lane; i < all; i += 32) {
            const float4 v = in[i];
            // of masked elements only: 0, or NaN where there is one
            rest += v.y * (v.x == m_rest || v.x == -INFINITY ? 1.0f : exp2_approx((v.x - m_rest) * p.scale));
        }
        rest = warp_reduce<float, add_op>(rest);
        const float rest_at = m_rest == m || m_rest == -INFINITY ? 1.0f : exp2_approx((m_rest - m) * p.scale);
        const float list = sh.list_s * (sh.list_m == m || sh.list_m == -INFINITY ? 1.0f : exp2_approx((sh.list_m - m) * p.scale));
        const float s = m == INFINITY ? NAN : rest * rest_at + list;
        // (as good as) nothing is left off the list, by masks of -inf or of a very low number: then the teacher's rest is what its
        // values' rounding left, if it is no more than that
        const bool nothing = rest == 0.0f || (m_rest - m) * p.scale < -kNothing;
        const float q_rest = nothing && sh.q_rest <= sh.q_noise ? 0.0f : sh.q_rest, mass = sh.q_sum + q_rest;
        Gradient g = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (s != 0.0f) {
            g.m = m_rest == -INFINITY ? 0.0f : m_rest;
            g.unit = sh.weight * p.inv_t;
            g.on = g.unit * __fdividef(mass, s);
            g.c0 = g.on * rest_at;
            if (q_rest > 0.0f && rest > 0.0f) g.c0 -= g.unit * __fdividef(q_rest, rest);
        }
        __syncwarp();
        if (sh.q_sum != sh.q_sum) g.on = g.c0 = NAN;  // also in an empty row
        if (lane == 0) sh.g = g, sh.q_rest = q_rest, sh.m = m == -INFINITY ? 0.0f : m, sh.m_rest = m_rest, sh.rest = rest, sh.s = s;
    }

    template <typename T>
    __device__ static void fix(const Params& p, const Shared& sh, const Slice<T>& s, T* out, int64_t r, bool first) {
        const Gradient g = sh.g;
        const float m = sh.m;
        if (out)
#pragma unroll 1
            for (int j = threadIdx.x & 31; j < p.k; j += 32)
                if (s.holds(sh.pos[j]))
                    Storage<T>::store1(out + sh.pos[j], g.on * exp2_approx((sh.z[j] - m) * p.scale) - g.unit * sh.q[j]);
        if (!first) return;
        // sum q (ln q - ln p) with ln p = ln 2 s (z - m) - ln S: the small difference of these sums, so in 64 bits
        double dot = 0.0;
        for (int j = threadIdx.x & 31; j < p.k; j += 32)
            if (sh.pos[j] >= 0 && sh.q[j] > 0.0f) dot += sh.q[j] * (static_cast<double>(sh.z[j]) - m);
        dot = warp_reduce<double, add_op>(dot);
        if ((threadIdx.x & 31) == 0) {
            const double log_s = log64(static_cast<double>(sh.s));
            double loss = INFINITY;
            if (sh.s != 0.0f && !sh.lost) {
                loss = sh.q_log_q - 0.6931471805599453 * p.scale * dot + sh.q_total * log_s;
                if (sh.q_rest != 0.0f) {
                    const double log_rest = log64(static_cast<double>(sh.rest)) +
                                            0.6931471805599453 * p.scale * (static_cast<double>(sh.m_rest) - m);
                    loss += sh.q_rest * (logf(sh.q_rest) - log_rest + log_s);
                }
            }
            p.loss[r] = sh.q_sum + sh.q_rest != sh.q_sum + sh.q_rest ? NAN : static_cast<float>(loss);
        }
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
