// qn_distill: a student's loss against a teacher's top logits, and its gradient.
//
// An operator of the row-gradient kernel.  With e_i = 2^((z_i - m) log2(e) / T) and the student's sums kept apart for the list (S_l) and the
// rest (S_r), S = S_l + S_r: p_k = e_k / S, and the mass off the list p_r = S_r / S comes without a subtraction.
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

struct Distill {
    using Params = DistillParams;
    static constexpr bool kMoments = false, kListMessage = true, kMask = true;
    static constexpr int kMine = QN_TOP_MAX / 32;  // entries of the list a lane
    struct Shared {
        int32_t pos[QN_TOP_MAX];  // the teacher's list; -1 for an absent token
        float q[QN_TOP_MAX], z[QN_TOP_MAX];
        float q_sum, q_log_q, q_rest, weight;
        Gradient g;
        float rest, s, dot;  // of the row, relative to its maximum
    };
    __device__ static void without(const Params& p, int64_t r, float loss) { p.loss[r] = loss; }
    __device__ static __forceinline__ int entries(const Params& p) { return p.k; }

    struct Fetched {
        int64_t at[kMine];
        float v[kMine], weight;
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
        float top = 0.0f, log_norm = 0.0f, inv = 1.0f;
        if (!p.logprobs) {
            top = -INFINITY;
#pragma unroll
            for (int i = 0; i < kMine; ++i) top = fmaxf(top, v[i]);
            top = warp_reduce<float, max_op>(top);
            if (top == -INFINITY) top = 0.0f;
            inv = p.inv_t;
            double norm = 0.0;
#pragma unroll
            for (int i = 0; i < kMine; ++i) norm += exp64(static_cast<double>((v[i] - top) * inv));
            log_norm = static_cast<float>(log(warp_reduce<double, add_op>(norm)));
        }
        // what is left of 1 may be far smaller than 1: the list is added up in 64 bits
        double q_sum = 0.0;
        float q_log_q = 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int j = lane + 32 * i;
            if (j >= p.k) continue;
            const float log_q = (v[i] - top) * inv - log_norm;
            const double q = exp64(static_cast<double>(log_q));
            q_sum += q;
            if (q != 0.0) q_log_q += static_cast<float>(q) * log_q;
            sh.q[j] = static_cast<float>(q);
        }
        q_sum = warp_reduce<double, add_op>(q_sum);
        q_log_q = warp_reduce<float, add_op>(q_log_q);
        if (lane == 0) {
            sh.weight = f.weight;
            sh.q_sum = wrong ? NAN : static_cast<float>(q_sum);
            sh.q_log_q = q_log_q;
            sh.q_rest = 0.0f;
            if (p.logprobs && named < p.vocab) sh.q_rest = q_sum != q_sum ? NAN : static_cast<float>(fmax(0.0, 1.0 - q_sum));
        }
        __syncwarp();
    }

    // Of the list's entries in a warp's chunks: the largest logit; sums of e_k and q_k u_k relative to it; sum of q_k.
    struct Extra {
        float m = -INFINITY, list = 0.0f, dot = 0.0f, q = 0.0f;
        __device__ __forceinline__ void down_to(const Params& p, float to) {
            if (!(to > m)) return;
            const float d = m - to;  // -inf at first, with nothing in the sums
            list *= exp2_approx(d * p.scale);
            if (q > 0.0f) dot += q * (d * p.inv_t);
            m = to;
        }
        __device__ __forceinline__ void take(const Params& p, const Shared& sh, int k, float z) {
            down_to(p, z);
            const float d = z - (m == -INFINITY ? 0.0f : m), qk = sh.q[k];
            list += exp2_approx(d * p.scale);
            if (qk > 0.0f) dot += qk * (d * p.inv_t);
            q += qk;
        }
        __device__ __forceinline__ float4 message(const Params& p) {
            down_to(p, warp_max_f32(m));
            return make_float4(m, warp_reduce<float, add_op>(list), warp_reduce<float, add_op>(dot),
                               warp_reduce<float, add_op>(q));
        }
    };

    // messages: of a CTA's warps, their maximum and sum of e_i; then of each what Extra has
    template <int kWarps>
    __device__ static __forceinline__ void join(const Params& p, Shared& sh, const float4* in, int ctas) {
        const int lane = threadIdx.x & 31, all = ctas * (2 * kWarps);
        float m = -INFINITY;
#pragma unroll 1
        for (int i = lane; i < all; i += 32) m = fmaxf(m, in[i].x);
        m = warp_max_f32(m);
        float rest = 0.0f, list = 0.0f, dot = 0.0f;
#pragma unroll 1
        for (int i = lane; i < all; i += 32) {
            const float4 v = in[i];
            const float f = v.x == m || v.x == -INFINITY ? 1.0f : exp2_approx((v.x - m) * p.scale);
            if (i % (2 * kWarps) < kWarps) {
                rest += f * v.y;  // masked elements only: 0, or NaN where there is one
            } else {
                list += f * v.y;
                dot += v.z;
                if (v.w > 0.0f && v.x != m) dot += v.w * ((v.x - m) * p.inv_t);
            }
        }
        rest = warp_reduce<float, add_op>(rest);
        list = warp_reduce<float, add_op>(list);
        dot = warp_reduce<float, add_op>(dot);
        const float s = m == INFINITY ? NAN : rest + list, q_rest = sh.q_rest, mass = sh.q_sum + q_rest;
        Gradient g = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (s != 0.0f) {
            g.m = m == -INFINITY ? 0.0f : m;
            g.unit = sh.weight * p.inv_t;
            g.on = g.unit * __fdividef(mass, s);
            g.c0 = q_rest > 0.0f && rest > 0.0f ? g.on - g.unit * __fdividef(q_rest, rest) : g.on;
        }
        if (lane == 0) sh.g = g, sh.rest = rest, sh.s = s, sh.dot = dot;
    }

    template <typename T>
    __device__ static void fix(const Params& p, const Shared& sh, const Slice<T>& s, T* out, int64_t r, bool first) {
        const Gradient g = sh.g;
        if (out)
#pragma unroll 1
            for (int j = threadIdx.x & 31; j < p.k; j += 32)
                if (s.holds(sh.pos[j]))
                    Storage<T>::store1(out + sh.pos[j], g.on * exp2_approx((sh.z[j] - g.m) * p.scale) - g.unit * sh.q[j]);
        if (first && (threadIdx.x & 31) == 0) {
            // sum q (ln q - ln p) with ln p = u - m/T - ln S
            const float log_s = logf(sh.s);
            float loss = sh.s == 0.0f ? INFINITY : sh.q_log_q - sh.dot + sh.q_sum * log_s;
            if (sh.s != 0.0f && sh.q_rest != 0.0f) loss += sh.q_rest * (logf(sh.q_rest) - (logf(sh.rest) - log_s));
            p.loss[r] = sh.q_sum + sh.q_rest != sh.q_sum + sh.q_rest ? NAN : loss;
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
