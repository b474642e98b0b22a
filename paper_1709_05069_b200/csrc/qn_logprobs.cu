// qn_logprobs and qn_logprobs_backward: log probabilities over a vocabulary and their gradient.
//
// Forward: one pass over the row by a CTA (or, where there are few rows, by a cluster of up to 8 whose results its first
// CTA joins), 256 threads with 16-byte loads straight to registers, a batch of four ahead of its use, and four CTAs on an SM
// (8192 x 131072 bf16 with 64 alternatives, compared in one run: 461 us; two batches ahead and three CTAs 519, none and five
// 471).  Each thread
// keeps a running maximum m, S = sum e_i and E = sum e_i d_i with d_i = (z_i - m) log2(e) / T and e_i = 2^d_i; z - m is
// formed before the scale, so that large logits lose nothing to the product's rounding.  At the end
// lse = m / T + ln S, H = ln S - ln 2 E / S.
//
// The k largest logits come out of the same pass: the k-th largest of the threads' maxima is a lower bound of the k-th
// largest logit, and nearly a tight one (of 256 maxima and k = 64, 74 logits are expected at or above it).  Each thread has
// also left the maxima of its batches in shared memory, so only the batches that hold such a logit are read again (from
// L2); what is found is ranked by counting.  Where that finds too many (equal logits, or the large ones in few threads) or
// too few, a slower selection that is exact for everything takes over.  The bound comes from a histogram of the maxima's float
// order, which stretches towards 0: where the largest is well above 0 and the k-th near it or below, the bound is searched bit by
// bit instead (33 counts over the CTA).  With logits as a language model gives them that is no row for k up to 20, 28 to 99 % of
// rows for k = 64 (131072 to 8192 tokens), and every row for k = 128.
//
// Measured on a B200: 8192 x 131072 bf16 with 64 alternatives 492 to 505 us a call at SM clocks of 1.79 to 1.76 GHz (66 % of a copy's rate):
// 9.7 instructions an element keep the issue slots 56 % busy, and behind the pass come the barriers of the alternatives.  One
// token of 32768 with 8 alternatives 8.3 us in a graph, 3.0 without alternatives.  More CTAs a row than fit at once (96 x
// 131072 in clusters of 8): 29 us against 17.  At 64 registers the forms with alternatives spill 36 (bf16) and 60 bytes.
//
// Backward: an operator of the row-gradient kernel.
#include <nvtx3/nvToolsExt.h>

#include "qn_vocab_grad.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;          // vectors of a thread at a time
constexpr int kGroups = 16;        // groups of batches whose maxima a thread keeps
constexpr int kCandidates = 1024;  // logits at or above the bound
constexpr int kHot = 2048;         // groups that hold one
constexpr int kBins = 256;         // of the threads' maxima, from the row's on down, 64 bins to a factor of 2
constexpr int kBinShift = 17;
constexpr int kTopCluster = 8;
// Logits below this are passed over as if masked in the main pass (their probability is 0 beside any that is not, and a
// product with 0 stays 0); a slice whose maximum is not well above it, or as large, is done again by slice_slow.
constexpr float kFloor = -0x1p66f;

struct LogprobParams {
    const void* logits;
    int64_t row_stride, rows;
    int32_t vocab, k, per_cta;
    const int64_t* tokens;
    float inv_t, scale;  // 1 / T, log2(e) / T
    float *logprob, *lse, *entropy;
    int64_t* top_token;
    float* top_logprob;
};

struct LogprobShared {
    float2 sums[kThreads / 32];
    float max[kThreads / 32];
    float4 part[kTopCluster];  // of the cluster's CTAs: maximum, S, E
    int32_t count, hot_count;
    uint32_t bound;
    int32_t bins[kBins];
    uint32_t hot[kHot];
    uint64_t candidate[kCandidates];
    uint64_t best[QN_TOP_MAX * kTopCluster];  // the CTAs' alternatives, largest first
    float group_max[kGroups][kThreads];
};

// A row's vector j of a slice, element by element; -inf outside the row.
template <typename T>
__device__ __noinline__ uint4 load_edge(const T* row, int32_t origin, int32_t vocab) {
    float x[Storage<T>::kVec];
#pragma unroll
    for (int e = 0; e < Storage<T>::kVec; ++e)
        x[e] = origin + e >= 0 && origin + e < vocab ? Storage<T>::load1(row + origin + e) : -INFINITY;
    return Storage<T>::pack(x);
}

// Vector j of a slice (-inf outside of it).
template <typename T>
__device__ __forceinline__ uint4 load_vector(const T* row, const Slice<T>& s, int32_t fb, int32_t fe, int32_t j) {
    if (j >= fb && j < fe) return ldg_stream16(row + (s.origin() + j * Slice<T>::kVec));
    return j < s.count ? load_edge(row, s.origin() + j * Slice<T>::kVec, s.vocab) : Lanes<T>::masked4();
}

// Gives the k largest of n distinct keys to `put(place, key)`, and 0 for the places that are left.  All threads, after a
// barrier.
template <typename Put>
__device__ __forceinline__ void rank_keys(const uint64_t* key, int n, int k, Put put) {
#pragma unroll 1
    for (int i = threadIdx.x; i < n || i < k; i += kThreads) {
        if (i < n) {
            const uint64_t mine = key[i];
            int above = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) above += key[j] > mine;
            if (above < k) put(above, mine);
        } else {
            put(i, 0);
        }
    }
}

// At most kCandidates logits of a slice, the k largest among them, whatever it holds: in steps of a logit for each thread,
// those above the k-th of what there is.  A step past the end of the largest rows leaves 32 bits, here and in slice_slow.
template <typename T>
__device__ __noinline__ void select_slow(const T* row, const Slice<T> s, int k, LogprobShared& sh, uint64_t* out) {
    const int32_t lo = max(0, s.origin()), hi = min(s.vocab, s.origin() + s.count * Slice<T>::kVec);
    uint64_t least = static_cast<uint64_t>(kOrderMasked) << 32 | 0xffffffffu;  // above every masked logit
    __syncthreads();  // every thread has read the count that sent it here
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
#pragma unroll 1
    for (int64_t i0 = lo; i0 < hi; i0 += kThreads) {
        const int64_t i = i0 + threadIdx.x;
        const uint64_t key = i < hi ? key_of(Storage<T>::load1(row + i), static_cast<uint32_t>(i)) : 0;
        if (key > least) sh.candidate[atomicAdd(&sh.count, 1)] = key;
        __syncthreads();
        if (sh.count > kCandidates - kThreads) {
            rank_keys(sh.candidate, sh.count, k, [&](int at, uint64_t x) { out[at] = x; });
            __syncthreads();
            least = out[k - 1];  // there are more than k
            for (int j = threadIdx.x; j < k; j += kThreads) sh.candidate[j] = out[j];
            if (threadIdx.x == 0) sh.count = k;
            __syncthreads();
        }
        __syncthreads();
    }
}

// The sums of a slice whose distances from kFloor could come out infinite or 0 (see there; or by an extreme temperature).
template <typename T>
__device__ __noinline__ float4 slice_slow(const T* row, const Slice<T> s, float scale, LogprobShared& sh) {
    const int32_t lo = max(0, s.origin()), hi = min(s.vocab, s.origin() + s.count * Slice<T>::kVec);
    float m = -INFINITY;
#pragma unroll 1
    for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) m = fmaxf(m, Storage<T>::load1(row + i));
    m = block_reduce<float, max_op>(m, sh.max);
    const float ref = m == -INFINITY ? 0.0f : m;
    double sum = 0.0, moment = 0.0;
#pragma unroll 1
    for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
        const float d = (Storage<T>::load1(row + i) - ref) * scale, e = exp2_approx(d);
        sum += e;
        if (e != 0.0f) moment += e * d;
    }
    const float2 x = block_sum2<kThreads>(make_float2(static_cast<float>(sum), static_cast<float>(moment)), sh.sums);
    return make_float4(m, x.x, x.y, 0.0f);
}

// The k-th largest of the threads' maxima (as orders), or less; kFloor's order if fewer than k are above that.
__device__ __noinline__ uint32_t search_bound(uint32_t mine, int k) {
    const uint32_t floor = order_of(kFloor);
    if (__syncthreads_count(mine > floor) < k) return floor;
    uint32_t bound = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t next = bound | 1u << bit;
        if (__syncthreads_count(mine >= next) >= k) bound = next;
    }
    return max(bound, floor + 1);
}

template <typename T, bool kTop>
__global__ void __launch_bounds__(kThreads, 4) logprobs_kernel(const LogprobParams p) {
    constexpr int kVec = Storage<T>::kVec, kPairs = kVec / 2;
    extern __shared__ __align__(16) unsigned char shared_bytes[];
    LogprobShared& sh = *reinterpret_cast<LogprobShared*>(shared_bytes);
    const uint32_t ctas = cluster_size(), rank = cluster_rank();
    const int tid = threadIdx.x;
    start_after_last();
    if (ctas > 1) cluster_arrive();  // waited for before the first store into another CTA
    for (int64_t r = blockIdx.x / ctas; r < p.rows; r += gridDim.x / ctas) {
        const T* row = static_cast<const T*>(p.logits) + r * p.row_stride;
        const Slice<T> s(row, p.vocab, p.per_cta, rank);
        const int32_t fb = s.full_begin(), fe = s.full_end();
        const int batches = (s.count + kThreads * kBatch - 1) / (kThreads * kBatch);
        const int per_group = (batches + kGroups - 1) / kGroups;
        auto load = [&](int b, uint4* v) {
            const int32_t j0 = b * (kThreads * kBatch);
            if (j0 >= fb && j0 + kThreads * kBatch <= fe) {
                const T* at = row + s.origin() + (j0 + tid) * kVec;
#pragma unroll
                for (int q = 0; q < kBatch; ++q) v[q] = ldg_stream16(at + q * (kThreads * kVec));
            } else {
#pragma unroll
                for (int q = 0; q < kBatch; ++q) v[q] = load_vector(row, s, fb, fe, j0 + q * kThreads + tid);
            }
        };
        // the given token's logit, long before it is needed
        int64_t token = -1;
        float token_z = 0.0f;
        if (p.logprob && tid == 0 && rank == 0) {
            token = p.tokens[r];
            if (token >= 0 && token < p.vocab) token_z = Storage<T>::load1(row + token);
        }
        if (kTop) {
            if (tid == 0) sh.count = 0, sh.hot_count = 0;
            for (int i = tid; i < kBins; i += kThreads) sh.bins[i] = 0;
        }
        float m = kFloor, group_top = kFloor;
        float sum = 0.0f;
        f32x2 moment = 0;
        const f32x2 scale = pack2(p.scale, p.scale);
        int left = per_group, group = 0;
        auto take = [&](uint4* v) {
            typename Lanes<T>::Max top;
            top.start(kFloor);
#pragma unroll
            for (int q = 0; q < kBatch; ++q) {
                v[q] = Lanes<T>::at_least(v[q], kFloor);
                top.take(v[q]);
            }
            const float most = top.get();
            if (!(most <= m)) {  // a new maximum, or NaN (then m and all sums become NaN)
                const float d = (m - most) * p.scale, f = exp2_approx(d);
                moment = f != 0.0f ? mul2(pack2(f, f), add2(moment, pack2(sum * d, 0.0f))) : 0;
                sum *= f;
                m = most;
            }
            if (kTop) {
                group_top = fmaxf(group_top, most);
                if (--left == 0) {
                    sh.group_max[group++][tid] = group_top;
                    left = per_group, group_top = kFloor;
                }
            }
            // a batch by itself first: beside a term of 1, one below 2^-24 would be lost, and a thousand of them add up (the
            // moment has no such term: d is 0 there)
            const f32x2 minus = pack2(-m, -m);
            f32x2 part;
#pragma unroll
            for (int q = 0; q < kBatch; ++q)
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const f32x2 d = mul2(add2(Lanes<T>::pair(v[q], i), minus), scale), e = exp2_pair(d);
                    part = q + i == 0 ? e : add2(part, e);
                    moment = fma2(e, d, moment);
                }
            float lo, hi;
            unpack2(part, lo, hi);
            sum += lo + hi;
        };
        uint4 a[kBatch], b[kBatch];
        if (batches > 0) load(0, a);
#pragma unroll 1
        for (int i = 0; i < batches; i += 2) {
            if (i + 1 < batches) load(i + 1, b);
            take(a);
            if (i + 1 >= batches) break;
            if (i + 2 < batches) load(i + 2, a);
            take(b);
        }
        let_next_start();
        if (kTop && left != per_group) sh.group_max[group++][tid] = group_top;
        // elements outside the slice were counted at the floor: in a slice with anything above it they are 0

        const int warp = tid >> 5, lane = tid & 31;
        const float wm = warp_max_f32(m);
        if (lane == 0) sh.max[warp] = wm;
        __syncthreads();
        float4 part = make_float4(kFloor, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) part.x = fmaxf(part.x, sh.max[w]);
        {
            const float d = (m - part.x) * p.scale, f = exp2_approx(d);
            float e0, e1;
            unpack2(moment, e0, e1);
            float2 x = make_float2(f * sum, f != 0.0f ? f * fmaf(sum, d, e0 + e1) : 0.0f);
            x.x = warp_reduce<float, add_op>(x.x);
            x.y = warp_reduce<float, add_op>(x.y);
            if (lane == 0) sh.sums[warp] = x;
        }
        const uint32_t most = order_of(part.x), mine = order_of(m);
        if (kTop && m > kFloor) atomicAdd(&sh.bins[min((most - mine) >> kBinShift, kBins - 1u)], 1);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) part.y += sh.sums[w].x, part.z += sh.sums[w].y;
        const bool slow = part.x <= kFloor / 2 || part.x >= -kFloor || !(p.scale > 1e-15f && p.scale < 1e15f);
        if (slow) part = slice_slow(row, s, p.scale, sh);
        if (!(part.y == part.y)) part.x = INFINITY;  // NaN somewhere
        const uint64_t* found = sh.candidate;
        int n = 0;
        if (kTop) {
            bool exact = slow;
            if (!exact) {
                if (warp == 0) {
                    // the bin in which the k-th largest maximum lies
                    constexpr int kPer = kBins / 32;
                    int c[kPer], total = 0;
#pragma unroll
                    for (int i = 0; i < kPer; ++i) c[i] = sh.bins[lane * kPer + i], total += c[i];
                    int before = total;
#pragma unroll
                    for (int o = 1; o < 32; o *= 2) {
                        const int up = __shfl_up_sync(0xffffffffu, before, o);
                        if (lane >= o) before += up;
                    }
                    const uint32_t reached = __ballot_sync(0xffffffffu, before >= p.k);
                    before -= total;
                    if (reached == 0) {
                        if (lane == 0) sh.bound = 0;
                    } else if (lane == __ffs(reached) - 1) {
                        int bin = lane * kPer - 1;
#pragma unroll
                        for (int i = 0; i < kPer; ++i)
                            if (before < p.k) before += c[i], ++bin;
                        const uint32_t depth = static_cast<uint32_t>(bin + 1) << kBinShift;
                        // the last bin has no lower end
                        sh.bound = bin < kBins - 1 ? max(most - depth + 1, order_of(kFloor) + 1) : 0;
                    }
                }
                __syncthreads();
                uint32_t bound = sh.bound;
                if (bound == 0) bound = search_bound(mine, p.k);
                const bool all = bound == order_of(kFloor);  // fewer than k threads have anything above the floor
                const uint32_t above = all ? kOrderMasked : bound - 1;
                auto collect = [&](int32_t j) {
                    const uint4 v = load_vector(row, s, fb, fe, j);
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        const float z = Storage<T>::get(v, e);
                        if (order_of(z) > above) {
                            const int at = atomicAdd(&sh.count, 1);
                            if (at < kCandidates) sh.candidate[at] = key_of(z, s.origin() + j * kVec + e);
                        }
                    }
                };
                if (all) {
#pragma unroll 1
                    for (int j = tid; j < s.count; j += kThreads) collect(j);
                } else {
                    if (mine > above)
#pragma unroll 1
                        for (int g = 0; g < group; ++g)
                            if (order_of(sh.group_max[g][tid]) > above) {
                                const int h = atomicAdd(&sh.hot_count, 1);
                                if (h < kHot) sh.hot[h] = g << 16 | tid;
                            }
                    __syncthreads();
                    const int hot = sh.hot_count, vectors = per_group * kBatch;
                    exact = hot > kHot;
#pragma unroll 1
                    for (int h = tid; !exact && h < hot * vectors; h += kThreads) {
                        const uint32_t id = sh.hot[h / vectors];
                        const int32_t j = ((id >> 16) * vectors + h % vectors) * kThreads + (id & 0xffff);
                        if (j < s.count) collect(j);
                    }
                }
                __syncthreads();
                exact = exact || sh.count > kCandidates;
            }
            if (exact) select_slow(row, s, p.k, sh, sh.best);
            n = sh.count;
        }
        if (ctas > 1) {  // to the cluster's first CTA; there is one row for each cluster then
            cluster_wait();
            if (tid == 0) store_remote(&sh.part[rank], 0, part);
            if (kTop) rank_keys(found, n, p.k, [&](int at, uint64_t x) { store_remote(&sh.best[rank * p.k + at], 0, x); });
            cluster_arrive();
            cluster_wait();
            if (rank != 0) return;
            float top = -INFINITY;
            for (uint32_t q = 0; q < ctas; ++q) top = fmaxf(top, sh.part[q].x);
            part = make_float4(top, 0.0f, 0.0f, 0.0f);
            for (uint32_t q = 0; q < ctas; ++q) {
                const float4 x = sh.part[q];
                const float d = x.x == top || x.x == -INFINITY ? 0.0f : (x.x - top) * p.scale, f = exp2_approx(d);
                part.y += f * x.y;
                if (f != 0.0f) part.z += f * fmaf(x.y, d, x.z);
            }
            if (kTop) {
                // a bound of the k-th largest of all: the largest of the CTAs' k-th; or, as together they have k that large,
                // the smallest of their (k / CTAs)-th
                const int share = (p.k + ctas - 1) / ctas;
                uint64_t low = ~0ull, high = 1;
                for (uint32_t q = 0; q < ctas; ++q) {
                    low = min(low, sh.best[q * p.k + share - 1]);
                    high = max(high, sh.best[q * p.k + p.k - 1]);
                }
                const uint64_t bound = max(low, high);
                if (tid == 0) sh.count = 0;
                __syncthreads();
                for (int i = tid; i < p.k * static_cast<int>(ctas); i += kThreads)
                    if (sh.best[i] >= bound) sh.candidate[atomicAdd(&sh.count, 1)] = sh.best[i];
                __syncthreads();
                n = sh.count;
            }
        }
        const bool bad = part.x == INFINITY, empty = part.x == -INFINITY;
        const float top = empty ? 0.0f : part.x, log_s = bad ? NAN : logf(part.y);
        if (tid == 0) {
            if (p.lse) p.lse[r] = bad ? NAN : top * p.inv_t + log_s;
            if (p.entropy) p.entropy[r] = empty ? 0.0f : log_s - kLn2 * (part.z / part.y);
            if (p.logprob) {
                float out = 0.0f;
                if (token >= p.vocab || (token >= 0 && bad)) out = NAN;
                else if (token >= 0) out = empty ? -INFINITY : (token_z - top) * p.inv_t - log_s;
                p.logprob[r] = out;
            }
        }
        if (kTop) {
            rank_keys(found, n, p.k, [&](int at, uint64_t key) {
                p.top_token[r * p.k + at] = key && !bad ? static_cast<int64_t>(key_index(key)) : -1;
                p.top_logprob[r * p.k + at] = bad ? NAN : key ? (key_value(key) - top) * p.inv_t - log_s : -INFINITY;
            });
        }
        __syncthreads();
    }
}

template <typename T, bool kTop>
cudaError_t launch_logprobs(LogprobParams& p, cudaStream_t st) {
    auto kernel = logprobs_kernel<T, kTop>;
    constexpr int kVec = Storage<T>::kVec;
    const int64_t all = (static_cast<int64_t>(p.vocab) + 2 * kVec - 2) / kVec;  // vectors, whatever the alignment
    int ctas = 1;
    while (ctas < kTopCluster && p.rows * 2 * ctas <= 4 * qn_sm_count() && all / ctas > 2 * kThreads) ctas *= 2;
    p.per_cta = static_cast<int32_t>((all + ctas - 1) / ctas);
    int dev = 0;
    static bool raised[64];
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!raised[dev]) {
        const cudaError_t e =
            cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(LogprobShared));
        if (e != cudaSuccess) return e;
        raised[dev] = true;
    }
    const int64_t most = INT32_MAX / kTopCluster;
    const EarlyLaunch launch((p.rows < most ? p.rows : most) * ctas, kThreads, sizeof(LogprobShared), ctas, st);
    return cudaLaunchKernelEx(&launch.cfg, kernel, p);
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
    static constexpr bool kMask = false, kAlone = false;
    struct Shared {
        int32_t pos[QN_TOP_MAX + 1];  // sparse terms: 0 the given token, 1..k the alternatives; -1 for none
        float add[QN_TOP_MAX + 1], z[QN_TOP_MAX + 1];
        float total, d_lse, d_h;  // total: NaN if a token is not in the vocabulary
        bool wrong;               // one is
        Gradient g;
    };
    __device__ static void without(const Params&, int64_t, float) {}
    __device__ static __forceinline__ int entries(const Params& p) { return p.k + 1; }

    static constexpr int kMine = QN_TOP_MAX / 32 + 1;  // sparse terms a lane
    struct Fetched {
        int64_t at[kMine];
        float x[kMine], z[kMine], d_lse, d_h;
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
    template <typename T>
    __device__ static __forceinline__ void gather(const Params& p, int64_t r, Fetched& f) {
        const T* row = static_cast<const T*>(p.logits) + r * p.row_stride;
#pragma unroll
        for (int i = 0; i < kMine; ++i) f.z[i] = f.at[i] >= 0 && f.at[i] < p.vocab ? load_rw(row + f.at[i]) : -INFINITY;
    }
    // a sparse term's gradient: none for an absent token, NaN for one that is not in the vocabulary
    __device__ static __forceinline__ float term(const Params& p, const Fetched& f, int i) {
        return f.at[i] < 0 ? 0.0f : f.at[i] >= p.vocab ? NAN : f.x[i];
    }

    __device__ static __forceinline__ bool wanted(const Params& p, const Fetched& f) {
        bool any = f.d_lse != 0.0f || f.d_h != 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) any = any || (f.at[i] >= 0 && f.x[i] != 0.0f);
        return __any_sync(0xffffffffu, any);
    }

    __device__ static __forceinline__ void begin(const Params& p, Shared& sh, const Fetched& f) {
        float sum = 0.0f;
        bool wrong = false;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int j = (threadIdx.x & 31) + 32 * i;
            wrong = wrong || f.at[i] >= p.vocab;
            if (j > p.k) continue;
            sh.pos[j] = f.at[i] >= 0 && f.at[i] < p.vocab ? static_cast<int32_t>(f.at[i]) : -1;
            sh.add[j] = term(p, f, i);
            sh.z[j] = f.z[i];
            sum += sh.add[j];
        }
        sum = warp_reduce<float, add_op>(sum);
        wrong = __any_sync(0xffffffffu, wrong);
        if ((threadIdx.x & 31) == 0) sh.total = sum, sh.d_lse = f.d_lse, sh.d_h = f.d_h, sh.wrong = wrong;
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
        if (sh.wrong) g.c0 = NAN;  // also in an empty row
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
            if (first) Storage<T>::store1(out + at, exp2_approx(d) * (g.c0 + g.c1 * fmaxf(d, kFarBelow)) + extra * p.inv_t);
        }
    }
};

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
    LogprobParams p{logits, row_stride, rows, static_cast<int32_t>(vocab), k, 0, tokens,
                    static_cast<float>(1.0 / temperature), static_cast<float>(1.4426950408889634 / temperature),
                    logprob, lse, entropy, top_token, top_logprob};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:logprobs");
    const cudaError_t e = dtype == QN_F32 ? (k ? launch_logprobs<float, true>(p, st) : launch_logprobs<float, false>(p, st))
                                          : (k ? launch_logprobs<__nv_bfloat16, true>(p, st)
                                               : launch_logprobs<__nv_bfloat16, false>(p, st));
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}

extern "C" qn_status qn_logprobs_backward(int64_t rows, int64_t vocab, qn_dtype dtype, const void* logits,
                                          int64_t row_stride, const int64_t* tokens, double temperature,
                                          const float* d_logprob, const float* d_lse, const float* d_entropy,
                                          int32_t k, const int64_t* top_token, const float* d_top_logprob,
                                          void* dlogits, int64_t dlogits_stride, void* cuda_stream) {
    if (rows == 0) return QN_OK;
    int dev = -1;
    if (!check_logits(rows, vocab, dtype, logits, row_stride, temperature, &dev)) return QN_ERR_INVALID;
    if (!dlogits || vocab > QN_GRAD_MAX_VOCAB || k < 0 || k > QN_TOP_MAX) return QN_ERR_INVALID;
    if (rows > INT64_MAX / 8 / (QN_TOP_MAX + 1)) return QN_ERR_INVALID;
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
