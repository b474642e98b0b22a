// qn_preference: preference loss of pairs of sequences from their tokens' log ratios, and its gradient.
//
//     S = sum_t w_t (l_t - ref_t) over a sequence (/ sum_t w_t),  R = beta S,  h = R_chosen - R_rejected - margin,  L = L(h)
//     dL/dl_t = weight L'(h) (+-beta) w_t (/ sum_t w_t)
// A cluster of CTAs takes a pair: each thread adds up its tokens of both sequences, the CTAs exchange four sums through
// distributed shared memory, every CTA works out the same two coefficients, and each thread writes the gradients of
// its own tokens, whose weights it has kept.  So each token is read once and written once, 16 bytes, and there is one launch.
// Sums and the pair's numbers are in 64 bits: h is the small difference of sums over thousands of tokens.
//
// Bound by latency: offsets, a pair's tiles one after the other, the exchange, exp and a division in 64 bits, the writes.
// Measured, us of kernel in a graph: 4 pairs of 64 tokens at most 3.8; 1024 pairs, 2.4 million tokens 11.7 (the bytes alone
// 5.8); 12 pairs, 2.2 million tokens 13.3 (4.7), with CTAs on all SMs only by clusters of 16.  Steps on the way, the last two
// of these: tokens of both sequences in one index, a select for each sum, 39 and 21; conditions around loads, which then wait for
// one another, 18 and 21; tiles without conditions 14 and 15; weights of four tiles in shared memory instead of two in
// registers 11.7 and 13.3.  Thousands of short pairs are bound by the numbers of each pair, which one thread works out while the
// others of its block wait: a warp a pair, and the eight pairs of a block by eight threads side by side, 4096 pairs of 72
// tokens 14.2 -> 9.4 (4096 of 580 tokens would go from 14.2 to 16.7, 12 of 80 from 3.8 to 4.9: these stay).  These kernels spill
// 24 (no reference), 216 (fp32) and 252 bytes (bf16) a thread.  The shape goes by the mean length, so that a long sequence among thousands
// of short ones is one warp's: 4096 pairs of 72 tokens with one sequence of 60 000 take 288 us.
// The loss alone: 1024 pairs, 2.4 million tokens 9.8 us; 12 pairs, 2.2 million tokens 10.2; 4096 pairs of 72 tokens 8.1.
#include <nvtx3/nvToolsExt.h>

#include "qn_vocab.cuh"

namespace {

constexpr int kMaxCluster = 16;
constexpr int kEach = 8;  // tokens of a tile a thread
constexpr int kKept = 4;  // tiles whose weights a thread keeps (in shared memory); it reads those of longer pairs again (from L2, mostly)

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

// A tile of a sequence: NT * kEach tokens from l, ref and weight on (`count` of them there), NT apart for a thread.  Its weights, and
// what it adds to the sums.  A token of weight 0 counts for nothing whatever it holds; nor does one that both sides mask.
template <typename R>
struct Sequence {
    const float *l, *weight;
    const R* ref;
    float* d;
    int64_t length;
};
template <int NT, typename R, bool kRef>
struct Tile {
    float l[kEach], ref[kEach], weight[kEach];
    // Loads without conditions, so that all are under way together: in a part of a tile, of its last token for those that are not
    // there.  Where a warp has a pair, most tiles are short ones: what no thread has a token for is left out.
    static __device__ __forceinline__ bool some(int k, int count) { return NT > 32 || k * NT < count; }
    template <bool kWhole>
    __device__ __forceinline__ void load(const Sequence<R>& s, int64_t at, int count, bool all) {
        const float *l_at = s.l + at, *weight_at = s.weight + at;
        const R* ref_at = s.ref + at;
        const int tid = NT > 32 ? threadIdx.x : threadIdx.x % NT;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            l[k] = ref[k] = weight[k] = 0.0f;
            if (!kWhole && !some(k, count)) continue;
            const int i = kWhole ? k * NT + tid : min(k * NT + tid, count - 1);
            l[k] = all ? __ldg(l_at + i) : 0.0f;
            ref[k] = kRef && all ? Storage<R>::load1(ref_at + i) : 0.0f;
            weight[k] = s.weight ? __ldg(weight_at + i) : 1.0f;
        }
        if (!kWhole)
#pragma unroll
            for (int k = 0; k < kEach; ++k)
                if (k * NT + tid >= count) weight[k] = 0.0f;
    }
    // all: not the weights alone
    __device__ __forceinline__ Tile(const Sequence<R>& s, int64_t at, int count, bool all = true) {
        if (count == NT * kEach) load<true>(s, at, count, all);
        else load<false>(s, at, count, all);
    }
    // True if a token counts for nothing although its weight is not 0.
    __device__ __forceinline__ bool add(double& ratios, double& weights, int count, bool normalise) {
        float most = 0.0f;  // of the magnitudes; NaN if there is one
#pragma unroll
        for (int k = 0; k < kEach; ++k) asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(most) : "f"(l[k]), "f"(ref[k]));
        bool dead = false;
        if (!(most < INFINITY)) dead = clean();
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            if (!some(k, count)) break;
            const double w = weight[k];  // products of numbers in 32 bits are exact in 64
            ratios += w * static_cast<double>(l[k]);
            if (kRef) ratios -= w * static_cast<double>(ref[k]);
            if (normalise) weights += w;
        }
        return dead;
    }
    // What does not count becomes 0.
    __device__ __forceinline__ bool clean() {
        bool dead = false;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const bool both = kRef && weight[k] != 0.0f && l[k] == -INFINITY && ref[k] == -INFINITY;
            dead = dead || both;
            if (both) weight[k] = 0.0f;
            if (weight[k] == 0.0f) l[k] = ref[k] = 0.0f;
        }
        return dead;
    }
    __device__ static __forceinline__ void write(const Sequence<R>& s, int64_t at, int count, const float (&w)[kEach], float coefficient) {
        const int tid = NT > 32 ? threadIdx.x : threadIdx.x % NT;
        float* d = s.d + at + tid;
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (k * NT + tid < count) d[k * NT] = w[k] == 0.0f ? 0.0f : w[k] * coefficient;
    }
};

// Loss and slope at h; the slope is needed first (the gradients wait for it), so that the two come apart.  e = exp(-|h|).
__device__ __forceinline__ double slope_at(const PreferenceParams& p, double h, double& e) {
    e = 0.0;
    if (h != h) return h;
    if (p.kind == QN_PREFERENCE_HINGE) return h < 1.0 ? -1.0 : 0.0;
    if (p.kind == QN_PREFERENCE_SQUARED) return 2.0 * ((h - 0.5) / p.beta) / p.beta;
    e = exp(-fabs(h));
    const double large = 1.0 / (1.0 + e), small = e * large;  // sigmoid(|h|), sigmoid(-|h|)
    const double up = h > 0.0 ? large : small, down = h > 0.0 ? small : large;
    return p.smoothing * up - (1.0 - p.smoothing) * down;
}
__device__ __forceinline__ double loss_at(const PreferenceParams& p, double h, double e) {
    if (h != h) return h;
    if (p.kind == QN_PREFERENCE_HINGE) return fmax(0.0, 1.0 - h);
    if (p.kind == QN_PREFERENCE_SQUARED) return ((h - 0.5) / p.beta) * ((h - 0.5) / p.beta);
    const double low = log1p(e), keep = 1.0 - p.smoothing;
    double loss = keep != 0.0 ? keep * (low + fmax(-h, 0.0)) : 0.0;
    if (p.smoothing != 0.0) loss += p.smoothing * (low + fmax(h, 0.0));
    return loss;
}

// Pairs of a CTA: short ones are a warp each.
template <int NT>
constexpr int kPairs = NT == 32 ? 8 : 1;

template <int NT, typename R, bool kRef>
__global__ void __launch_bounds__(NT * kPairs<NT>, 1024 / (NT * kPairs<NT>)) preference_kernel(const PreferenceParams p) {
    __shared__ double warp_sums[NT / 32][4];
    __shared__ uint64_t inbox[kMaxCluster][4];
    __shared__ float coefficient[2];
    const uint32_t ctas = NT == 32 ? 1 : cluster_size(), rank = NT == 32 ? 0 : cluster_rank();
    const int tid = NT > 32 ? threadIdx.x : threadIdx.x % NT, warp = tid >> 5, lane = tid & 31;
    start_after_last();
    let_next_start();
    if (ctas > 1) cluster_arrive();  // waited for before the first store into another CTA
    const int64_t mine = NT == 32 ? blockIdx.x * static_cast<int64_t>(kPairs<NT>) + threadIdx.x / NT : blockIdx.x / ctas;
    const bool there = NT > 32 || mine < p.pairs;
    const int64_t pair = there ? mine : p.pairs - 1;
    const int64_t chosen = p.split ? pair : 2 * pair, rejected = p.split ? p.pairs + pair : 2 * pair + 1;
    const float unit = !there ? 0.0f : p.pair_weight ? p.pair_weight[pair] : 1.0f;
    Sequence<R> sequence[2];
    bool wrong = false;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int64_t a = p.offsets[s ? rejected : chosen], b = p.offsets[(s ? rejected : chosen) + 1];
        const bool good = a >= 0 && a <= b && b <= p.tokens;
        const int64_t begin = good ? a : 0;
        sequence[s] = Sequence<R>{p.logprob + begin, p.weight ? p.weight + begin : nullptr, kRef ? static_cast<const R*>(p.ref) + begin : nullptr,
                                  p.d_logprob + (p.d_logprob ? begin : 0), good ? b - a : 0};
        wrong = wrong || !good;
    }
    // tiles of the chosen sequence, then those of the rejected one, in turn for the CTAs
    constexpr int kTile = NT * kEach;
    const int64_t tiles0 = (sequence[0].length + kTile - 1) / kTile, tiles = tiles0 + (sequence[1].length + kTile - 1) / kTile;
    const auto each_tile = [&](auto&& with) {
        int turn = 0;
#pragma unroll 1
        for (int64_t t = rank; t < tiles; t += ctas, turn = turn < kKept ? turn + 1 : turn) with(t, turn);
    };
    struct Place {
        int s;
        int64_t at;
        int count;
    };
    const auto place = [&](int64_t t) {
        const int s = t >= tiles0;
        const int64_t at = (s ? t - tiles0 : t) * kTile;
        return Place{s, at, static_cast<int>(min((s ? sequence[1].length : sequence[0].length) - at, static_cast<int64_t>(kTile)))};
    };
    if (unit == 0.0f) {  // padding
        if (p.d_logprob && there)
            each_tile([&](int64_t t, int) {
                const Place x = place(t);
                const float none[kEach] = {};
                Tile<NT, R, kRef>::write(x.s ? sequence[1] : sequence[0], x.at, x.count, none, 0.0f);
            });
        if (rank == 0 && tid == 0 && there) {
            p.loss[pair] = 0.0f;
            if (p.reward) p.reward[chosen] = p.reward[rejected] = 0.0f;
        }
        if (NT > 32) {
            __syncwarp();
            if (ctas > 1) cluster_wait();
            return;
        }
    }
    double sums[4] = {0.0, 0.0, 0.0, 0.0};  // weighted ratios of the chosen and of the rejected, weights of both
    extern __shared__ float shared[];
    float* kept = shared + (NT > 32 ? 0 : threadIdx.x / NT) * (kKept * kEach * NT);  // [tile][token of a thread][thread]: each thread its own
    bool dead = false;
    const auto add = [&](const Place& x, Tile<NT, R, kRef>& tile) {
        double ratios = 0.0, weights = 0.0;
        dead = tile.add(ratios, weights, x.count, p.normalise) || dead;
        if (x.s) sums[1] += ratios, sums[3] += weights;
        else sums[0] += ratios, sums[2] += weights;
    };
    if (NT > 32 || unit != 0.0f) each_tile([&](int64_t t, int turn) {
        const Place x = place(t);
        Tile<NT, R, kRef> tile(x.s ? sequence[1] : sequence[0], x.at, x.count);
        add(x, tile);
        if (turn < kKept)
#pragma unroll
            for (int e = 0; e < kEach; ++e) kept[(turn * kEach + e) * NT + tid] = tile.weight[e];
    });
    const int count = p.normalise ? 4 : 2;
    double h = 0.0, e = 0.0;
    float c0 = 0.0f, c1 = 0.0f;
    const auto settle = [&](const double (&total)[4], float unit, bool wrong, int64_t chosen, int64_t rejected) {  // by one thread
        double each[2], reward[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            each[s] = !p.normalise ? p.beta : total[2 + s] != 0.0 ? p.beta / total[2 + s] : 0.0;
            reward[s] = each[s] == 0.0 ? 0.0 : each[s] * total[s];
        }
        h = wrong ? NAN : reward[0] - reward[1] - p.margin;
        const double slope = unit * slope_at(p, h, e);
        c0 = static_cast<float>(slope * each[0]);
        c1 = static_cast<float>(-slope * each[1]);
        if (rank == 0 && p.reward) {
            p.reward[chosen] = wrong ? NAN : static_cast<float>(reward[0]);
            p.reward[rejected] = wrong ? NAN : static_cast<float>(reward[1]);
        }
    };
    if constexpr (NT == 32) {
        // the pairs' numbers side by side, by as many threads of the first warp
        __shared__ double totals[kPairs<NT>][4];
        __shared__ float units[kPairs<NT>], coefficients[kPairs<NT>][2];
        __shared__ bool wrongs[kPairs<NT>];
        const int group = threadIdx.x / NT;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const double x = q < count ? warp_reduce<double, add_op>(sums[q]) : 0.0;
            if (lane == q) totals[group][q] = x;
        }
        if (lane == 0) units[group] = unit, wrongs[group] = wrong;
        __syncthreads();
        const int64_t theirs = blockIdx.x * static_cast<int64_t>(kPairs<NT>) + lane;
        const bool one = group == 0 && lane < kPairs<NT> && units[lane % kPairs<NT>] != 0.0f;
        if (one) {
            const double total[4] = {totals[lane][0], totals[lane][1], totals[lane][2], totals[lane][3]};
            settle(total, units[lane], wrongs[lane], p.split ? theirs : 2 * theirs, p.split ? p.pairs + theirs : 2 * theirs + 1);
            coefficients[lane][0] = c0, coefficients[lane][1] = c1;
        }
        __syncthreads();
        if (one) p.loss[theirs] = static_cast<float>(loss_at(p, h, e));
        if (unit == 0.0f) return;
        c0 = coefficients[group][0], c1 = coefficients[group][1];
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (q >= count) break;
            const double x = warp_reduce<double, add_op>(sums[q]);
            if (lane == 0) warp_sums[warp][q] = x;
        }
        __syncthreads();
        if (warp == 0) {
            double mine = 0.0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (q >= count) break;
                const double x = warp_reduce<double, add_op>(lane < NT / 32 ? warp_sums[lane][q] : 0.0);
                if (lane == q) mine = x;
            }
            __syncwarp();
            if (ctas == 1) {
                if (lane < 4) inbox[0][lane] = __double_as_longlong(mine);
            } else {
                cluster_wait();
                if (lane < 4)
                    for (uint32_t c = 0; c < ctas; ++c) store_remote(&inbox[rank][lane], c, __double_as_longlong(mine));
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
            settle(total, unit, wrong, chosen, rejected);
            coefficient[0] = c0, coefficient[1] = c1;
        }
        __syncthreads();
        c0 = coefficient[0], c1 = coefficient[1];
    }
    if (p.d_logprob) {
        each_tile([&](int64_t t, int turn) {
            const Place x = place(t);
            if (turn < kKept) {
                float weight[kEach];
#pragma unroll
                for (int e = 0; e < kEach; ++e) weight[e] = kept[(turn * kEach + e) * NT + tid];
                Tile<NT, R, kRef>::write(x.s ? sequence[1] : sequence[0], x.at, x.count, weight, x.s ? c1 : c0);
            } else {
                Tile<NT, R, kRef> tile(x.s ? sequence[1] : sequence[0], x.at, x.count, dead);
                if (dead) tile.clean();
                Tile<NT, R, kRef>::write(x.s ? sequence[1] : sequence[0], x.at, x.count, tile.weight, x.s ? c1 : c0);
            }
        });
    }
    if (NT > 32 && rank == 0 && tid == 0) p.loss[pair] = static_cast<float>(loss_at(p, h, e));
}

template <int NT>
constexpr int kShared = NT * kPairs<NT> * kEach * kKept * 4;

// How many clusters of 16 fit on the device at once (asked for once on each); such clusters need a permission.
template <int NT, typename R, bool kRef>
cudaError_t large_clusters(int* fit) {
    static int known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (known[dev] == 0) {
        int found = 0;
        const EarlyLaunch launch(kMaxCluster, NT, kShared<NT>, kMaxCluster, nullptr);
        cudaError_t e = cudaFuncSetAttribute(preference_kernel<NT, R, kRef>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(preference_kernel<NT, R, kRef>, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared<NT>);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&found, preference_kernel<NT, R, kRef>, &launch.cfg);
        if (e != cudaSuccess) return e;
        known[dev] = found < 1 ? -1 : found;
    }
    *fit = known[dev];
    return cudaSuccess;
}

template <int NT, typename R, bool kRef>
cudaError_t launch_preference(const PreferenceParams& p, int ctas, cudaStream_t st) {
    if (kShared<NT> > (48 << 10)) {
        const cudaError_t e = cudaFuncSetAttribute(preference_kernel<NT, R, kRef>, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared<NT>);
        if (e != cudaSuccess) return e;
    }
    const EarlyLaunch launch((p.pairs + kPairs<NT> - 1) / kPairs<NT> * ctas, NT * kPairs<NT>, kShared<NT>, ctas, st);
    return cudaLaunchKernelEx(&launch.cfg, preference_kernel<NT, R, kRef>, p);
}

template <typename R, bool kRef>
cudaError_t launch_preference(const PreferenceParams& p, cudaStream_t st) {
    // Threads for a pair, by its mean length (the lengths themselves are on the device): one for each eight tokens, as long as half of
    // the threads that the device has (more do not fit beside their registers) are enough for all pairs.
    const int64_t mean = p.tokens / p.pairs, room = 1024 * static_cast<int64_t>(qn_sm_count()) / p.pairs;
    const int64_t threads = mean / kEach < room ? mean / kEach : room;
    if (threads >= 128 * kMaxCluster) {
        int fit = 0;
        const cudaError_t e = large_clusters<512, R, kRef>(&fit);
        if (e != cudaSuccess) return e;
        if (p.pairs <= fit) return launch_preference<512, R, kRef>(p, kMaxCluster, st);
    }
    int ctas = 1;
    while (ctas < 8 && p.pairs * ctas < qn_sm_count() && threads >= 128 * ctas) ctas *= 2;
    const int64_t each = threads / ctas;
    // a warp a pair: short ones, of which there are more than there is room for blocks of 64 threads (8 an SM are their fair share)
    if (mean < 32 * kEach && p.pairs > 8 * static_cast<int64_t>(qn_sm_count())) return launch_preference<32, R, kRef>(p, ctas, st);
    if (each < 96) return launch_preference<64, R, kRef>(p, ctas, st);
    if (each < 192) return launch_preference<128, R, kRef>(p, ctas, st);
    if (each < 384) return launch_preference<256, R, kRef>(p, ctas, st);
    return launch_preference<512, R, kRef>(p, ctas, st);
}

}  // namespace

extern "C" qn_status qn_preference(int64_t pairs, int64_t tokens, const float* logprob, qn_dtype ref_dtype,
                                   const void* ref_logprob, const float* weight, const int64_t* offsets, int32_t split,
                                   const float* pair_weight, int32_t kind, double beta, double margin, double smoothing,
                                   int32_t normalise, float* loss, float* reward, float* d_logprob, void* cuda_stream) {
    if (pairs == 0) return QN_OK;
    if (pairs < 0 || pairs > INT32_MAX / 8 || tokens < 0 || tokens > (int64_t(1) << 56)) return QN_ERR_INVALID;
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
