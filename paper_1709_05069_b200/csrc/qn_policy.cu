// qn_policy: clipped policy loss of given tokens with a KL term and an entropy bonus, and its gradient, from the logits.
//
// An operator of the row-gradient kernels: the loss of a row is a function f of its token's log probability,
// l = u_t - lse, less b times the row's entropy H, so that with p = softmax(u)
//     dL/dz_i = 1/T [ f'(l) (1[i = t] - p_i) + b p_i (ln p_i + H) ]
// has the form e_i (c0 + c1 d_i) and one more term at the token.  What a separate loss would read and write between the log
// probabilities and their backward pass, and the second pass over the row, fall away: a row is read once and its
// gradient written once.  As in qn_logprobs_backward ln p_i + H = ln 2 (d_i - E / S).
// What bounds it is in qn_vocab_grad.cuh.  Measured (the bytes alone at a copy's rate): 4096 x 131072 bf16 400 us (328); 2047 x 100003
// bf16 with entropy, every eighth row padding 172 us (117); 61 x 20011 fp32 5.4 us of kernel, 11 us a call.  The log
// probabilities, a separate loss and their backward pass would read the logits twice.  Rows off 16 bytes: 2047 x 100003 bf16 without padding
// 171 us where 2047 x 100000 takes 160 (125), with entropy 192 and 173.  The loss alone: 4096 x 131072 bf16 201 us (164), with entropy 242;
// 2047 x 100003 107 (63), with entropy 123; 2047 x 100000 88 and 101.
#include <nvtx3/nvToolsExt.h>

#include "qn_vocab_grad.cuh"

namespace {

struct PolicyParams {
    const void* logits;
    int64_t row_stride, rows;
    int32_t vocab;
    const int64_t* tokens;
    float inv_t, scale;  // 1 / T, log2(e) / T
    const float *old_logprob, *ref_logprob, *advantage, *weight;
    float low, high, dual, kl, bonus;  // bounds of the ratio; dual 0: none
    float *loss, *logprob, *entropy;
    void* dlogits;
    int64_t dlogits_stride;
};

// Loss and slope of a token with log probability l.  A token that the policy masks has the ratio 0, and no slope.
__device__ __forceinline__ float2 surrogate(const PolicyParams& p, float l, float old, float ref, float advantage) {
    const bool gone = l == -INFINITY;
    const float ratio = gone && old == old ? 0.0f : expf(l - old);
    float loss = 0.0f, slope = 0.0f;
    if (advantage != 0.0f) {
        const float free = -advantage * ratio, held = -advantage * fminf(fmaxf(ratio, p.low), p.high);
        loss = free >= held ? free : held;
        slope = free >= held ? free : 0.0f;
        const float most = -advantage * p.dual;
        if (p.dual > 0.0f && advantage < 0.0f && loss > most) loss = most, slope = 0.0f;
    }
    if (ratio != ratio || advantage != advantage) loss = slope = NAN;
    if (p.kl != 0.0f) {
        const float y = gone && ref == -INFINITY ? 0.0f : ref - l, k = expm1f(y);
        loss += p.kl * (y == INFINITY ? INFINITY : k - y);
        slope -= p.kl * k;
        if (y != y) slope = NAN;
    }
    return make_float2(loss, gone && loss == loss ? 0.0f : slope);
}

template <bool kEntropy>
struct Policy {
    using Params = PolicyParams;
    static constexpr bool kMoments = kEntropy;
    static constexpr bool kMask = false, kAlone = true;
    static constexpr int kMine = 1;
    struct Shared {
        int32_t pos[1];  // the token; -1 if it is not in the vocabulary
        float z, old, ref, advantage, weight;
        float l, h, slope;
        Gradient g;
    };
    __device__ static void without(const Params& p, int64_t r, float x) {
        p.loss[r] = x;
        if (p.logprob) p.logprob[r] = x;
        if (p.entropy) p.entropy[r] = x;
    }
    __device__ static __forceinline__ int entries(const Params&) { return 1; }

    struct Fetched {
        int64_t at;
        float z, old, ref, advantage, weight;
    };
    __device__ static __forceinline__ Fetched fetch(const Params& p, int64_t r) {
        Fetched f = {-1, -INFINITY, 0.0f, 0.0f, 0.0f, 1.0f};
        if (r < p.rows) {
            f.at = p.tokens[r];
            f.old = p.old_logprob[r];
            f.advantage = p.advantage[r];
            if (p.kl != 0.0f) f.ref = p.ref_logprob[r];
            if (p.weight) f.weight = p.weight[r];
        }
        return f;
    }
    template <typename T>
    __device__ static __forceinline__ void gather(const Params& p, int64_t r, Fetched& f) {
        const T* row = static_cast<const T*>(p.logits) + r * p.row_stride;
        f.z = f.at >= 0 && f.at < p.vocab ? load_rw(row + f.at) : -INFINITY;
    }
    __device__ static __forceinline__ bool wanted(const Params&, const Fetched& f) { return f.at >= 0 && f.weight != 0.0f; }
    __device__ static __forceinline__ void begin(const Params& p, Shared& sh, const Fetched& f) {
        if ((threadIdx.x & 31) == 0) {
            sh.pos[0] = f.at < p.vocab ? static_cast<int32_t>(f.at) : -1;
            sh.z = f.z;
            sh.old = f.old;
            sh.ref = f.ref;
            sh.advantage = f.advantage;
            sh.weight = f.weight;
        }
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
        float l = -INFINITY, h = 0.0f, slope = 0.0f;
        if (s != 0.0f) {  // not empty
            g.m = m == -INFINITY ? 0.0f : m;
            g.unit = sh.weight * p.inv_t;
            const float log_s = logf(s), mean = kEntropy ? kLn2 * e / s : 0.0f;
            l = (sh.z - g.m) * p.inv_t - log_s;
            h = log_s - mean;
            slope = surrogate(p, l, sh.old, sh.ref, sh.advantage).y;
            const float unit = g.unit / s;
            g.c0 = unit * -(slope + p.bonus * mean);
            g.c1 = unit * p.bonus * kLn2;
        }
        __syncwarp();
        if (sh.pos[0] < 0) l = slope = g.c0 = NAN;  // also in an empty row
        if (lane == 0) sh.g = g, sh.l = l, sh.h = h, sh.slope = slope;
    }

    template <typename T>
    __device__ static void fix(const Params& p, const Shared& sh, const Slice<T>& s, T* out, int64_t r, bool first) {
        if ((threadIdx.x & 31) != 0) return;
        const Gradient g = sh.g;
        const int32_t at = sh.pos[0];
        if (out && s.holds(at)) {
            const float d = (sh.z - g.m) * p.scale;
            Storage<T>::store1(out + at, exp2_approx(d) * (g.c0 + g.c1 * fmaxf(d, kFarBelow)) + g.unit * sh.slope);
        }
        if (!first) return;
        const float loss = surrogate(p, sh.l, sh.old, sh.ref, sh.advantage).x;
        p.loss[r] = p.bonus != 0.0f ? loss - p.bonus * sh.h : loss;
        if (p.logprob) p.logprob[r] = sh.l;
        if (p.entropy) p.entropy[r] = sh.l != sh.l && at < 0 ? NAN : sh.h;
    }
};

}  // namespace

extern "C" qn_status qn_policy(int64_t rows, int64_t vocab, qn_dtype dtype, const void* logits, int64_t row_stride,
                               const int64_t* tokens, double temperature, const float* old_logprob, const float* ref_logprob,
                               const float* advantage, const float* weight, double clip_low, double clip_high, double dual,
                               double kl, double entropy_bonus, float* loss, float* logprob, float* entropy, void* dlogits,
                               int64_t dlogits_stride, void* cuda_stream) {
    if (rows == 0) return QN_OK;
    int dev = -1;
    if (!check_logits(rows, vocab, dtype, logits, row_stride, temperature, &dev)) return QN_ERR_INVALID;
    if (vocab > QN_GRAD_MAX_VOCAB || rows > INT64_MAX / 64) return QN_ERR_INVALID;
    if (!tokens || !old_logprob || !advantage || !loss || (kl != 0.0 && !ref_logprob)) return QN_ERR_INVALID;
    if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0) || !(dual == 0.0 || dual > 1.0) || !isfinite(dual)) return QN_ERR_INVALID;
    if (!(kl >= 0.0) || !isfinite(static_cast<float>(kl)) || !isfinite(static_cast<float>(entropy_bonus))) return QN_ERR_INVALID;
    if (!check_array(tokens, 8, dev) || !check_array(old_logprob, 4, dev) || !check_array(ref_logprob, 4, dev) ||
        !check_array(advantage, 4, dev) || !check_array(weight, 4, dev) || !check_array(loss, 4, dev) ||
        !check_array(logprob, 4, dev) || !check_array(entropy, 4, dev))
        return QN_ERR_INVALID;
    if (dlogits && !check_gradient(rows, vocab, dtype, logits, row_stride, dlogits, dlogits_stride, dev)) return QN_ERR_INVALID;
    // what is written touches nothing else, but that the gradient may take the place of the logits
    float* const outputs[] = {loss, logprob, entropy};
    const float* const inputs[] = {old_logprob, ref_logprob, advantage, weight};
    if (dlogits) {
        if (overlaps_rows(tokens, rows * 8, dlogits, rows, vocab, dlogits_stride, dtype)) return QN_ERR_INVALID;
        for (const float* in : inputs)
            if (in && overlaps_rows(in, rows * 4, dlogits, rows, vocab, dlogits_stride, dtype)) return QN_ERR_INVALID;
    }
    for (int i = 0; i < 3; ++i) {
        if (!outputs[i]) continue;
        if (overlaps(outputs[i], rows * 4, logits, matrix_bytes(rows, vocab, row_stride, dtype)) ||
            (dlogits && overlaps(outputs[i], rows * 4, dlogits, matrix_bytes(rows, vocab, dlogits_stride, dtype))) ||
            overlaps(outputs[i], rows * 4, tokens, rows * 8))
            return QN_ERR_INVALID;
        for (const float* in : inputs)
            if (in && overlaps(outputs[i], rows * 4, in, rows * 4)) return QN_ERR_INVALID;
        for (int k = 0; k < i; ++k)
            if (outputs[k] && overlaps(outputs[i], rows * 4, outputs[k], rows * 4)) return QN_ERR_INVALID;
    }
    DeviceGuard guard(dev);
    if (!guard.ok) return QN_ERR_CUDA;
    const PolicyParams p{logits, row_stride, rows, static_cast<int32_t>(vocab), tokens,
                         static_cast<float>(1.0 / temperature), static_cast<float>(1.4426950408889634 / temperature),
                         old_logprob, ref_logprob, advantage, weight,
                         static_cast<float>(1.0 - clip_low), static_cast<float>(1.0 + clip_high), static_cast<float>(dual),
                         static_cast<float>(kl), static_cast<float>(entropy_bonus), loss, logprob, entropy, dlogits, dlogits_stride};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:policy");
    const bool moments = p.bonus != 0.0f || entropy;
    const cudaError_t e = dtype == QN_F32 ? (moments ? launch_gradient<float, Policy<true>>(p, st) : launch_gradient<float, Policy<false>>(p, st))
                                          : (moments ? launch_gradient<__nv_bfloat16, Policy<true>>(p, st)
                                                     : launch_gradient<__nv_bfloat16, Policy<false>>(p, st));
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
