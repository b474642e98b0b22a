// qn_preference: preference loss of pairs of sequences from their tokens' log ratios, and its gradient.
//
//     S = sum_t w_t (l_t - ref_t) over a sequence (/ sum_t w_t),  R = beta S,  h = R_chosen - R_rejected - margin,  L = L(h)
//     dL/dl_t = weight L'(h) (+-beta) w_t (/ sum_t w_t)
// A cluster of CTAs takes a pair: each thread adds up its tokens of both sequences, the CTAs exchange four sums through
// distributed shared memory, every CTA works out the same two coefficients, and each thread writes the gradients of
// its own tokens, whose weights it has kept.  So each token is read once and written once, 16 bytes, and there is one launch.
// Sums and the pair's numbers are in 64 bits: h is the small difference of sums over thousands of tokens.
#include <nvtx3/nvToolsExt.h>

#include "qn_vocab.cuh"

namespace {

constexpr int kMaxCluster = 8;
constexpr int kKept = 8;  // tokens whose weights a thread keeps; it reads those of longer pairs again (from L2, mostly)

struct PreferenceParams {
    int64_t pairs, tokens;
    const float* logprob;
    const void* ref;
    const float* weight;
    const int64_t* offsets;
    const float* pair_weight;
    int32_t kind, normalise, split;
    double beta, margin, smoothing;
    float *loss, *reward, *d_logprob;
};

// What counts of a token: its weight, and its weighted log ratio.  A token of weight 0 counts for nothing whatever it
// holds; nor does one that both sides mask.
struct Token {
    float weight;
    double ratio;
};
template <typename R, bool kRef>
__device__ __forceinline__ Token token_at(const PreferenceParams& p, int64_t i) {
    Token t;
    t.weight = p.weight ? __ldg(p.weight + i) : 1.0f;
    const float l = __ldg(p.logprob + i), ref = kRef ? Storage<R>::load1(static_cast<const R*>(p.ref) + i) : 0.0f;
    if (kRef && l == -INFINITY && ref == -INFINITY) t.weight = 0.0f;
    t.ratio = t.weight == 0.0f ? 0.0 : t.weight * (static_cast<double>(l) - static_cast<double>(ref));
    return t;
}

__device__ __noinline__ double softplus(double x) { return log1p(exp(-fabs(x))) + fmax(x, 0.0); }
__device__ __noinline__ double sigmoid(double x) { return 1.0 / (1.0 + exp(-x)); }

// Loss and slope at h.
__device__ __forceinline__ double2 preference(const PreferenceParams& p, double h) {
    if (h != h) return make_double2(h, h);
    if (p.kind == QN_PREFERENCE_HINGE) return make_double2(fmax(0.0, 1.0 - h), h < 1.0 ? -1.0 : 0.0);
    if (p.kind == QN_PREFERENCE_SQUARED) {
        const double x = (h - 0.5) / p.beta;
        return make_double2(x * x, 2.0 * x / p.beta);
    }
    const double keep = 1.0 - p.smoothing;
    double2 r = make_double2(keep * softplus(-h), -keep * sigmoid(-h));
    if (p.smoothing != 0.0) r.x += p.smoothing * softplus(h), r.y += p.smoothing * sigmoid(h);
    return r;
}

template <int NT, typename R, bool kRef>
__global__ void __launch_bounds__(NT) preference_kernel(const PreferenceParams p) {
    __shared__ double warp_sums[NT / 32][4];
    __shared__ uint64_t inbox[kMaxCluster][4];
    __shared__ float coefficient[2];
    const uint32_t ctas = cluster_size(), rank = cluster_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    start_after_last();
    let_next_start();
    if (ctas > 1) cluster_arrive();  // waited for before the first store into another CTA
    const int64_t pair = blockIdx.x / ctas;
    const int64_t chosen = p.split ? pair : 2 * pair, rejected = p.split ? p.pairs + pair : 2 * pair + 1;
    const float unit = p.pair_weight ? p.pair_weight[pair] : 1.0f;
    int64_t begin[2], length[2];
    bool wrong = false;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int64_t a = p.offsets[s ? rejected : chosen], b = p.offsets[(s ? rejected : chosen) + 1];
        const bool good = a >= 0 && a <= b && b <= p.tokens;
        begin[s] = good ? a : 0;
        length[s] = good ? b - a : 0;
        wrong = wrong || !good;
    }
    const int64_t all = length[0] + length[1], stride = static_cast<int64_t>(ctas) * NT, first = rank * NT + tid;
    const auto place = [&](int64_t j) { return j < length[0] ? begin[0] + j : begin[1] + (j - length[0]); };
    if (unit == 0.0f) {  // padding
        if (p.d_logprob)
            for (int64_t j = first; j < all; j += stride) p.d_logprob[place(j)] = 0.0f;
        if (rank == 0 && tid == 0) {
            p.loss[pair] = 0.0f;
            if (p.reward) p.reward[chosen] = p.reward[rejected] = 0.0f;
        }
        __syncwarp();
        if (ctas > 1) cluster_wait();
        return;
    }
    double sums[4] = {0.0, 0.0, 0.0, 0.0};  // weighted ratios of the chosen and of the rejected, weights of both
    float kept[kKept];
    const auto add = [&](int64_t j, const Token& t) {
        const bool second = j >= length[0];
        sums[0] += second ? 0.0 : t.ratio, sums[1] += second ? t.ratio : 0.0;
        if (p.normalise) sums[2] += second ? 0.0 : t.weight, sums[3] += second ? t.weight : 0.0;
    };
    {
        Token t[kKept];
#pragma unroll
        for (int k = 0; k < kKept; ++k) {
            const int64_t j = first + k * stride;
            t[k] = Token{0.0f, 0.0};
            if (j < all) t[k] = token_at<R, kRef>(p, place(j));
        }
#pragma unroll
        for (int k = 0; k < kKept; ++k) {
            add(first + k * stride, t[k]);
            kept[k] = t[k].weight;
        }
    }
#pragma unroll 4
    for (int64_t j = first + kKept * stride; j < all; j += stride) add(j, token_at<R, kRef>(p, place(j)));
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const double x = warp_reduce<double, add_op>(sums[q]);
        if (lane == 0) warp_sums[warp][q] = x;
    }
    __syncthreads();
    if (warp == 0) {
        double x = 0.0;
        if (lane < 4)
#pragma unroll 1
            for (int w = 0; w < NT / 32; ++w) x += warp_sums[w][lane];
        __syncwarp();
        if (ctas == 1) {
            if (lane < 4) inbox[0][lane] = __double_as_longlong(x);
        } else {
            cluster_wait();
            if (lane < 4)
                for (uint32_t c = 0; c < ctas; ++c) store_remote(&inbox[rank][lane], c, __double_as_longlong(x));
        }
        __syncwarp();
    }
    if (ctas > 1) {
        if (warp != 0) cluster_wait();
        cluster_arrive();
        cluster_wait();
    }
    if (tid == 0) {
        double total[4] = {0.0, 0.0, 0.0, 0.0};
        for (uint32_t c = 0; c < ctas; ++c)
            for (int q = 0; q < 4; ++q) total[q] += __longlong_as_double(inbox[c][q]);
        double each[2], reward[2];
        for (int s = 0; s < 2; ++s) {
            each[s] = !p.normalise ? p.beta : total[2 + s] != 0.0 ? p.beta / total[2 + s] : 0.0;
            reward[s] = each[s] == 0.0 ? 0.0 : each[s] * total[s];
        }
        const double2 l = preference(p, wrong ? NAN : reward[0] - reward[1] - p.margin);
        coefficient[0] = static_cast<float>(unit * l.y * each[0]);
        coefficient[1] = static_cast<float>(-unit * l.y * each[1]);
        if (rank == 0) {
            p.loss[pair] = static_cast<float>(l.x);
            if (p.reward) {
                p.reward[chosen] = wrong ? NAN : static_cast<float>(reward[0]);
                p.reward[rejected] = wrong ? NAN : static_cast<float>(reward[1]);
            }
        }
    }
    __syncthreads();
    if (!p.d_logprob) return;
    const float c0 = coefficient[0], c1 = coefficient[1];
    const auto write = [&](int64_t j, float weight) { p.d_logprob[place(j)] = weight == 0.0f ? 0.0f : weight * (j < length[0] ? c0 : c1); };
#pragma unroll
    for (int k = 0; k < kKept; ++k)
        if (first + k * stride < all) write(first + k * stride, kept[k]);
#pragma unroll 4
    for (int64_t j = first + kKept * stride; j < all; j += stride) write(j, token_at<R, kRef>(p, place(j)).weight);
}

template <int NT, typename R, bool kRef>
cudaError_t launch_preference(const PreferenceParams& p, int ctas, cudaStream_t st) {
    const EarlyLaunch launch(p.pairs * ctas, NT, 0, ctas, st);
    return cudaLaunchKernelEx(&launch.cfg, preference_kernel<NT, R, kRef>, p);
}

template <typename R, bool kRef>
cudaError_t launch_preference(const PreferenceParams& p, cudaStream_t st) {
    // By the mean length of a pair (the lengths themselves are on the device): CTAs until the device is full or each has 512
    // tokens, and threads for eight tokens each.
    const int64_t mean = p.tokens / p.pairs;
    int ctas = 1;
    while (2 * ctas <= kMaxCluster && p.pairs * 2 * ctas <= 2 * qn_sm_count() && mean > 512 * ctas) ctas *= 2;
    const int64_t per_cta = mean / ctas;
    if (per_cta <= 512) return launch_preference<64, R, kRef>(p, ctas, st);
    if (per_cta <= 2048) return launch_preference<256, R, kRef>(p, ctas, st);
    return launch_preference<1024, R, kRef>(p, ctas, st);
}

}  // namespace

extern "C" qn_status qn_preference(int64_t pairs, int64_t tokens, const float* logprob, qn_dtype ref_dtype,
                                   const void* ref_logprob, const float* weight, const int64_t* offsets, int32_t split,
                                   const float* pair_weight, int32_t kind, double beta, double margin, double smoothing,
                                   int32_t normalise, float* loss, float* reward, float* d_logprob, void* cuda_stream) {
    if (pairs == 0) return QN_OK;
    if (pairs < 0 || pairs > INT32_MAX / kMaxCluster || tokens < 0 || tokens > (int64_t(1) << 56)) return QN_ERR_INVALID;
    if (!offsets || !loss || (tokens && !logprob)) return QN_ERR_INVALID;
    if (ref_dtype != QN_F32 && ref_dtype != QN_BF16) return QN_ERR_INVALID;
    if (kind != QN_PREFERENCE_LOGISTIC && kind != QN_PREFERENCE_HINGE && kind != QN_PREFERENCE_SQUARED) return QN_ERR_INVALID;
    if (!(beta > 0.0) || !isfinite(beta) || !isfinite(margin) || !(smoothing >= 0.0 && smoothing <= 1.0)) return QN_ERR_INVALID;
    int dev = -1;
    if (!device_of(loss, &dev)) return QN_ERR_INVALID;
    const size_t ref_size = dtype_size(ref_dtype);
    if (!check_array(logprob, 4, dev) || !check_array(ref_logprob, ref_size, dev) || !check_array(weight, 4, dev) ||
        !check_array(offsets, 8, dev) || !check_array(pair_weight, 4, dev) || !check_array(loss, 4, dev) ||
        !check_array(reward, 4, dev) || !check_array(d_logprob, 4, dev))
        return QN_ERR_INVALID;
    // what is written touches nothing else
    const struct { const void* at; size_t bytes; } arrays[] = {
        {loss, size_t(pairs) * 4}, {reward, size_t(pairs) * 8}, {d_logprob, size_t(tokens) * 4},
        {logprob, size_t(tokens) * 4}, {ref_logprob, size_t(tokens) * ref_size}, {weight, size_t(tokens) * 4},
        {offsets, size_t(2 * pairs + 1) * 8}, {pair_weight, size_t(pairs) * 4}};
    for (int i = 0; i < 3; ++i)
        for (int k = i + 1; k < 8; ++k)
            if (arrays[i].at && arrays[k].at && overlaps(arrays[i].at, arrays[i].bytes, arrays[k].at, arrays[k].bytes)) return QN_ERR_INVALID;
    DeviceGuard guard(dev);
    if (!guard.ok) return QN_ERR_CUDA;
    const PreferenceParams p{pairs, tokens, logprob, ref_logprob, weight, offsets, pair_weight, kind, normalise != 0, split != 0,
                             beta, margin, smoothing, loss, reward, d_logprob};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:preference");
    const cudaError_t e = !ref_logprob ? launch_preference<float, false>(p, st)
                          : ref_dtype == QN_F32 ? launch_preference<float, true>(p, st) : launch_preference<__nv_bfloat16, true>(p, st);
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
