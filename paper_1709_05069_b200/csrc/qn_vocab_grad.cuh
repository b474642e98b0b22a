// The kernel behind the calls that give the gradient of a row of logits: the row is read once, its softmax statistics are
// taken, and the gradient is written, with the row in shared memory between the two.
//
// Two forms: the pipeline here, for many long rows, and row_gradient_small_kernel below, for everything else.
//
// A cluster of C CTAs takes a row; each holds a slice of up to 128 KB (80 KB where rows do not start and end on 16 bytes), and
// of up to 192 KB where eight of those are not enough.  A row is seen as 16-byte vectors that start at the 16-byte boundary at or below its first element, so that whatever its
// alignment all but its first and last vector move as bulk copies; what those two hold outside the row is filled with -inf.
//
// There is one CTA on an SM, it stays, and its warps are stages of a pipeline over chunks of 4 KB in a ring of 48:
//   list warps     a row each: read the few elements of it that are special (a given token, alternatives, a teacher's list),
//                  work out what depends on them alone, and sort those by chunk that must not be added
//   copy warp      brings the slices of the coming rows in
//   sum warps      a chunk each: take out what must not be added, and add e_i = 2^d_i, d_i = (z_i - m) log2(e) / T, relative
//                  to a running maximum m of each thread; at the end of a slice each sends its maximum and sums to every
//                  CTA of the cluster (asynchronous stores into shared memory that count on a barrier there)
//   join warp      from all messages, in the same order in every CTA, to the row's coefficients
//   write warps    a chunk each: e_i times the coefficient; give the chunk back
//   end warp       when a row has been written, its special elements' gradients, and the row's loss
// So HBM is read and written at the same time, and the exchange of one row passes while others are summed and written.
//
// Measured on a B200, 4096 x 131072 bf16 with a list of 64 tokens: 417 to 423 us at SM clocks of 1.82 to 1.79 GHz under the power
// cap, 78 % of the rate of a plain copy (fp32, 1024 x 262144: 426 to 432 us near 1.95 GHz, 76 %; clusters of 8 leave 28 of the 148 SMs without
// work).  The time follows the SM clock, but no unit is full: 14.5 instructions an element (17 with an entropy gradient) keep
// the issue slots 51 to 58 % busy, the two exp2 of an element their unit 53 %, and DRAM is active in half of its cycles (1024
// rows; the stages wait for one another).  Whatever adds instructions adds time: a quarter of the exp2 as a polynomial on the
// FMA pipe made 469 us of 441, a vote for every chunk's wait 1.5 %.  Keeping e_i in registers between the two (one exp2) needs
// loops unrolled over them, and those ran out of the instruction cache: 883 us.  One lane that issued all copies took 470
// cycles for each: 526 us.  28 warps of seven roles share 72 registers a thread: with a gradient, 32 to 144 bytes of a thread
// are spilled, most where an entropy gradient meets rows that do not lie on 16 bytes.
//
// An operator Op brings:
//   Params, Shared        arguments; what the warps tell one another of a row
//   Fetched, fetch        a row's special elements as a lane of a list warp loads them, two rows ahead of their use
//   gather                their logits (of the whole row, also outside the slice), a row ahead
//   wanted                false if the row is padding: its gradient is 0, and the pipeline does not read it
//   begin                 list warp: what depends on the special elements alone, and their places (Shared::pos)
//   kMask                 whether the special elements leave the sums and the maximum
//   join                  from all messages to Shared::g
//   fix                   end warp: the special elements' gradients, and the row's loss
#pragma once

#include "qn_vocab.cuh"

namespace {

constexpr int kMaxCluster = 8;
constexpr int kChunk = 256;      // vectors in a chunk
constexpr int kSlots = 48;       // chunks in the ring
constexpr int kListWarps = 2;
constexpr int kLists = 6;  // rows between the list warps' beginning and the end warp's end of them
// Warps that sum and that write.  Measured for 4096 x 131072 bf16 with a list of 64 tokens (at the time), us: 8 / 8 468,
// 10 / 13 449, 11 / 12 440; 28 warps are the most that leave 72 registers for each.
template <bool kWrite>
struct Roles {
    static constexpr int kSum = 11, kWriting = kWrite ? 12 : 0;  // the same sums with and without a gradient
    static constexpr int kThreads = 32 * (kSum + kWriting + 3 + kListWarps);
};

// ---- clusters ------------------------------------------------------------------------------------------------------

// 16 bytes into the same variable of another CTA, counted on the same barrier of that CTA.
__device__ __forceinline__ void store_async(const void* mine, const uint64_t* bar, uint32_t cta, float4 x) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                     map_remote(mine, cta)),
                 "f"(x.x), "f"(x.y), "f"(x.z), "f"(x.w), "r"(map_remote(bar, cta))
                 : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// A bounded wait.  Its slow part is out of line (instruction cache), and leaves the warp suspended for up to 20 us at a time
// instead of polling: with polls in their place half of the instructions that the SM issued were those of waiting warps.
__device__ __noinline__ bool wait_slow(uint64_t* bar, uint32_t parity, volatile int* abort) {
    const uint64_t began = global_timer_ns();
    for (uint32_t it = 0; it < kWaitLimit; ++it) {
        uint32_t passed;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(passed)
            : "r"(smem_u32(bar)), "r"(parity), "r"(20000u)
            : "memory");
        if (passed) return true;
        if (*abort) return false;
        if (global_timer_ns() - began > kWaitLimitNs) break;
    }
    *abort = 1;
    return false;
}
__device__ __forceinline__ bool wait_lane(uint64_t* bar, uint32_t parity, volatile int* abort) {
    return mbar_try(bar, parity) || wait_slow(bar, parity, abort);
}
// With one answer for all lanes of the warp, so that they leave together.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
    return __all_sync(0xffffffffu, mbar_try(bar, parity)) || __all_sync(0xffffffffu, wait_slow(bar, parity, abort));
}

// A lane's wait for the copy of one item, where the last item in that slot may still be on its way.  A parity cannot tell the
// phase before from the one after, so the slot also says which item it was last issued for.  That is read before the barrier:
// once it is this item, the phase before has ended.
__device__ __noinline__ bool wait_copy_slow(uint64_t* bar, uint32_t parity, volatile uint32_t* issued, uint32_t item, volatile int* abort) {
    const uint64_t began = global_timer_ns();
    for (uint32_t it = 0; it < kWaitLimit; ++it) {
        const bool known = *issued == item;
        if (!wait_slow(bar, parity, abort)) return false;
        if (known) return true;
        __nanosleep(64);
        if (*abort) return false;
        if (global_timer_ns() - began > kWaitLimitNs) break;
    }
    *abort = 1;
    return false;
}
__device__ __forceinline__ bool wait_copy(uint64_t* bar, uint32_t parity, volatile uint32_t* issued, uint32_t item, volatile int* abort) {
    const uint32_t last = *issued;
    const bool here = mbar_try(bar, parity) && last == item;
    return here || wait_copy_slow(bar, parity, issued, item, abort);
}

// Before an arrival after which a bulk copy may write what this thread wrote.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- when a wait ran out (kSlots and kLists are those of the ring and of the lists) ---------------------------------------
//
// No CTA may leave while another one may still send into its shared memory, nor while a copy or a message into it is on its way.
// Those that were waited for have arrived, and once its warps are through with all rows, all have.  So every warp simply ends,
// but for the join warp: it keeps the CTA until all other threads of the cluster have ended or have come to the same barrier
// (every wait is bounded, so that they do).  If a wait ran out, the copy warp first waits for its copies, and the join warp after
// the barrier for the messages that were sent: one after the other, until none has come within the limit.

// Copy warp: waits for the last copy into each slot, of the items before `begun` and of the lanes of `mask` after it.
__device__ __noinline__ void wait_copies(uint64_t* full, uint32_t begun, uint32_t mask, volatile int* late) {
    const uint32_t lane = threadIdx.x & 31;
#pragma unroll 1
    for (uint32_t i = lane; i < kSlots && i < begun; i += 32) {
        const uint32_t item = begun - 1 - i;
        if (i < kSlots - 32 || !(mask >> (kSlots - 1 - i) & 1)) wait_slow(&full[item % kSlots], item / kSlots & 1, late);
    }
    if (mask >> lane & 1) wait_slow(&full[(begun + lane) % kSlots], (begun + lane) / kSlots & 1, late);
}

// Join warp: waits for the messages of row u (`bytes`, if `expected` announced already), and of those after it.
__device__ __noinline__ void wait_messages(uint64_t* heard, uint32_t u, bool expected, uint32_t bytes, volatile int* late) {
    do {
        if (!expected && (threadIdx.x & 31) == 0) mbar_arrive_expect_tx(&heard[u % kLists], bytes);
        __syncwarp();
        expected = false;
    } while (wait(&heard[u % kLists], u / kLists & 1, late) && ++u);
}

// ---- writing -------------------------------------------------------------------------------------------------------

// Writes one value over the slice's part of a row, by NT threads.
template <typename T, int NT>
__device__ __noinline__ void write_constant(T* out, const Slice<T> s, int tid, float x) {
    const int32_t lo = max(0, s.origin()), hi = min(s.vocab, s.origin() + s.count * Slice<T>::kVec);
    if (lo >= hi) return;
    constexpr int kVec = Slice<T>::kVec;
    const int32_t head = min(hi - lo, static_cast<int32_t>((16 - (reinterpret_cast<uintptr_t>(out + lo) & 15)) / sizeof(T)) % kVec);
    if (tid < head) Storage<T>::store1(out + lo + tid, x);
    const int32_t n = (hi - lo - head) / kVec;
    float xs[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) xs[e] = x;
    const uint4 w = Storage<T>::pack(xs);
#pragma unroll 1
    for (int j = tid; j < n; j += NT) stg_stream16(out + lo + head + j * kVec, w);
    const int32_t tail = lo + head + n * kVec + tid;
    if (tail < hi && tid < kVec) Storage<T>::store1(out + tail, x);
}

// Loads of logits whose place the gradient may take.
__device__ __forceinline__ uint4 load_stream(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p)
                 : "memory");
    return v;
}
template <typename T>
__device__ __noinline__ uint4 load_edge_rw(const T* row, int32_t origin, int32_t vocab) {
    float x[Storage<T>::kVec];
#pragma unroll
    for (int e = 0; e < Storage<T>::kVec; ++e) x[e] = origin + e >= 0 && origin + e < vocab ? load_rw(row + origin + e) : -INFINITY;
    return Storage<T>::pack(x);
}

// The elements of one vector that lie inside the row, one at a time.
template <typename T>
__device__ __noinline__ void write_edge(T* out, int32_t origin, int32_t vocab, uint4 w) {
#pragma unroll 1
    for (int e = 0; e < Storage<T>::kVec; ++e) {
        if (origin + e >= 0 && origin + e < vocab) Storage<T>::store1(out + origin + e, Storage<T>::get(w, 0));
        if (sizeof(T) == 4) w = make_uint4(w.y, w.z, w.w, 0);
        else w = make_uint4(w.x >> 16 | w.y << 16, w.y >> 16 | w.z << 16, w.z >> 16 | w.w << 16, w.w >> 16);
    }
}
// 32 vectors of a warp, one run of the row from element `at` on, to a row that is not aligned as they are: through shared
// memory to pieces of 4 bytes.
__device__ __forceinline__ void write_run(float* out, int32_t at, const uint4* run) {
    const int lane = threadIdx.x & 31;
    const float* from = reinterpret_cast<const float*>(run);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[at + lane + 32 * i] = from[lane + 32 * i];
}
__device__ __forceinline__ void write_run(__nv_bfloat16* out_, int32_t at, const uint4* run) {
    const int lane = threadIdx.x & 31;
    const uint32_t* from = reinterpret_cast<const uint32_t*>(run);
    uint16_t* out = reinterpret_cast<uint16_t*>(out_) + at;
    if (reinterpret_cast<uintptr_t>(out) & 2) {
        uint32_t* words = reinterpret_cast<uint32_t*>(out + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int w = lane + 32 * i;
            const uint32_t x = from[w];
            if (w == 0) out[0] = static_cast<uint16_t>(x);
            if (w == 127) out[255] = static_cast<uint16_t>(x >> 16);
            else words[w] = x >> 16 | from[w + 1] << 16;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(out)[lane + 32 * i] = from[lane + 32 * i];
    }
}

// gradient_i = e_i (c0 + c1 d_i) with e_i and d_i relative to m; on and unit: for Op::fix.
struct Gradient {
    float m, c0, c1;
    float on, unit;
};

// Elements [begin, end) of a row, as far as they are in [0, vocab), from 16-byte aligned shared memory to an output that is
// not aligned as they are, by one warp: 16-byte stores, put together from 4-byte pieces.
template <typename T>
__device__ __forceinline__ void write_run(T* out, int32_t begin, int32_t end, int32_t vocab, const T* from) {
    constexpr int kVec = Storage<T>::kVec;
    const int lane = threadIdx.x & 31;
    const int32_t lo = max(0, begin), hi = min(vocab, end);
    const int32_t head = min(hi - lo, static_cast<int32_t>((16 - (reinterpret_cast<uintptr_t>(out + lo) & 15)) / sizeof(T)) % kVec);
    const int32_t first = lo + head, vectors = (hi - first) / kVec;
    const int32_t skip = first - begin;  // elements of `from` before the first vector
    const uint32_t* words = reinterpret_cast<const uint32_t*>(from) + (sizeof(T) == 4 ? skip : skip / 2);
    const bool odd = sizeof(T) == 2 && skip % 2;
    if (lane < head) out[lo + lane] = from[lo - begin + lane];
#pragma unroll 2
    for (int j = lane; j < vectors; j += 32) {
        uint32_t w[5];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = words[4 * j + i];
        if (odd) {
            w[4] = words[4 * j + 4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
        }
        stg_stream16(out + first + j * kVec, make_uint4(w[0], w[1], w[2], w[3]));
    }
    const int32_t tail = first + vectors * kVec + lane;
    if (tail < hi) out[tail] = from[tail - begin];
}

// The rows of a cluster.  In every turn the n clusters take the next n rows, moved on by `rotation` (< n) from the last turn,
// so that one of them goes through the rows in a stride without small factors: padding at every s-th row then falls to all
// clusters alike.
struct Walk {
    int64_t base;
    uint32_t at, n, rotation;
    __device__ __forceinline__ int64_t row() const { return base + at; }
    __device__ __forceinline__ void next(int turns = 1) {
        for (int t = 0; t < turns; ++t) {
            base += n;
            at += rotation;
            if (at >= n) at -= n;
        }
    }
};

// kAligned: every row of the gradient starts as far from a 16-byte boundary as its row of logits.
// kEdges: rows may start or end elsewhere than on 16 bytes.
template <typename T, typename Op, bool kAligned, bool kEdges, bool kWrite>
__global__ void __launch_bounds__(Roles<kWrite>::kThreads, 1)
    row_gradient_kernel(const typename Op::Params p, const int32_t per_cta, const uint32_t rotation) {
    constexpr int kSumWarps = Roles<kWrite>::kSum, kWriteWarps = Roles<kWrite>::kWriting;
    constexpr int kVec = Storage<T>::kVec, kPairs = kVec / 2;
    constexpr int kMessages = kSumWarps;
    constexpr bool moments = Op::kMoments;
    extern __shared__ __align__(128) uint4 ring[];
    __shared__ typename Op::Shared lists[kLists];
    __shared__ __align__(16) float4 inbox[kLists][kMaxCluster * kMessages];
    __shared__ __align__(16) uint4 edges[kLists][2];  // a slice's first and last vector, where they reach past the row
    // a row's special elements in the order of their chunks, and where each chunk's begin
    __shared__ uint8_t order[kLists][QN_TOP_MAX + 32], chunk_begin[kLists][64];
    // full: a chunk has arrived; empty: it has been written.  By row: ready: begun; done: summed and written.  retired: its
    // special elements too.  By row that is wanted: heard: all messages; joined: coefficients
    __shared__ uint64_t full[kSlots], empty[kSlots], ready[kLists], done[kLists], heard[kLists], joined[kLists], retired[kLists];
    __shared__ uint32_t issued[kWrite ? 1 : kSlots];  // the item that each slot's last copy is of (see wait_copy)
    __shared__ bool wanted[kLists];
    __shared__ int abort, late[2];  // a wait ran out; one after that did, of the copy warp or of the join warp
    const uint32_t ctas = cluster_size(), rank = cluster_rank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (!kWrite && threadIdx.x < kSlots) issued[threadIdx.x] = ~0u;
    if (threadIdx.x == 0) {
        abort = late[0] = late[1] = 0;
#pragma unroll 1
        for (int i = 0; i < kSlots; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
#pragma unroll 1
        for (int i = 0; i < kLists; ++i) {
            mbar_init(&ready[i], 1), mbar_init(&done[i], kSumWarps + kWriteWarps + 2), mbar_init(&retired[i], 1);
            mbar_init(&heard[i], 1), mbar_init(&joined[i], 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (ctas > 1) cluster_sync();  // every CTA's barriers are there before the first store into it
    const Walk walk{0, blockIdx.x / ctas, gridDim.x / ctas, rotation};
    auto row_of = [&](int64_t r) { return static_cast<const T*>(p.logits) + r * p.row_stride; };
    auto out_of = [&](int64_t r) { return static_cast<T*>(p.dlogits) + r * p.dlogits_stride; };
    auto slice_of = [&](int64_t r) { return Slice<T>(row_of(r), p.vocab, per_cta, rank); };
    auto chunks_of = [](const Slice<T>& s) { return (s.count + kChunk - 1) / kChunk; };
    // rounds of a ring: item n is in slot n % size, and is the (n / size)-th there
    auto wait_item = [&](uint64_t* bars, uint32_t n, uint32_t size) { return wait(&bars[n % size], n / size & 1, &abort); };
    // by each lane for itself, where a vote is dear: for every chunk, and on the way to a row's coefficients (votes for these took
    // 2 to 4 %)
    auto wait_alone = [&](uint64_t* bars, uint32_t n, uint32_t size) { return wait_lane(&bars[n % size], n / size & 1, &abort); };
    // A CTA sends a row's messages once it has joined the row before the last.  So whoever has heard all of row u knows that
    // every CTA has joined u - 2, and may send u + 2: four sets of messages never meet
    auto may_send = [&](uint32_t u) { return u < 2 || wait_alone(joined, u - 2, kLists); };
    auto send = [&](uint32_t u, int index, float4 msg) {
        if (lane < static_cast<int>(ctas))
            store_async(&inbox[u % kLists][rank * kMessages + index], &heard[u % kLists], lane, msg);
    };

    uint32_t n = 0;     // chunks so far
    uint32_t turn = 0;  // rows so far
    uint32_t u = 0;     // wanted rows so far
    if (warp < kSumWarps) {
        uint32_t one_before = 0, two_before = 0;  // the first item of the wanted row before, and of the one before that
        Walk rows = walk;
#pragma unroll 1
        for (int64_t r; (r = rows.row()) < p.rows; rows.next(), ++turn) {
            const int li = turn % kLists;
            if (!wait_alone(ready, turn, kLists)) return;
            if (wanted[li]) {
                const Slice<T> s = slice_of(r);
                const int chunks = chunks_of(s);
                const f32x2 scale = pack2(p.scale, p.scale);
                const int32_t fb = s.full_begin(), fe = s.full_end();
                typename Op::Shared& sh = lists[li];
                float m = -INFINITY;
                f32x2 sum = 0, moment = 0;
                bool patched = false;  // a bulk copy may only write there again after a fence
                // Copies land in any order, and warps go at their own pace: at an item one may meet a slot whose last item, 48
                // before, is still on its way, and take its arrival for the item's own (see wait_copy).  Not so once the row of
                // that one has been joined; the sum warp knows it of all rows before `known`, that is, of items before
                // `sure` - 48.  With a gradient a slot is given back after its row's join, so that to wait for that first
                // costs nothing; without one the slot says what it holds.
                uint32_t known = u < 2 ? 0 : u - 2, sure = two_before + kSlots;
                // chunk c is for worker c % kSumWarps; which warp that is moves on from row to row
                const int worker = (warp + kSumWarps - turn % kSumWarps) % kSumWarps;
#pragma unroll 1
                for (int c = worker; c < chunks; c += kSumWarps) {
                    const uint32_t slot = (n + c) % kSlots;
                    if constexpr (kWrite) {
                        while (n + c >= sure) {
                            if (!wait_alone(joined, known, kLists)) return;
                            sure = (++known == u ? n : one_before) + kSlots;
                        }
                        if (!wait_alone(full, n + c, kSlots)) return;
                    } else if (n + c < sure) {
                        if (!wait_alone(full, n + c, kSlots)) return;
                    } else {
                        if (!wait_copy(&full[slot], (n + c) / kSlots & 1, &issued[slot], n + c, &abort)) return;
                    }
                    if constexpr (Op::kMask) {
                        const int begin = chunk_begin[li][c], end = chunk_begin[li][c + 1];
                        if (begin < end) {
                            T* first = reinterpret_cast<T*>(ring + slot * kChunk) - (s.origin() + c * (kChunk * kVec));
#pragma unroll 1
                            for (int i = begin + lane; i < end; i += 32) first[sh.pos[order[li][i]]] = masked<T>();
                            patched = true;
                            __syncwarp();
                        }
                    }
                    const uint4* data = ring + slot * kChunk + lane;
                    const int count = min(kChunk, s.count - c * kChunk) - lane;
#pragma unroll 1
                    for (int j = 0; j < kChunk; j += 128, data += 128) {
                        uint4 v[4];
                        if (c * kChunk >= fb && (c + 1) * kChunk <= fe) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) v[q] = data[32 * q];
                        } else {
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const int k = c * kChunk + j + 32 * q + lane;
                                v[q] = j + 32 * q >= count ? Lanes<T>::masked4() : kEdges && k < fb ? edges[li][0] : kEdges && k >= fe ? edges[li][1] : data[32 * q];
                            }
                        }
                        typename Lanes<T>::Max top;
#pragma unroll
                        for (int q = 0; q < 4; ++q) top.take(v[q]);
                        const float most = top.get();
                        if (!(most <= m)) {  // a new maximum, or NaN (then m and all sums become NaN)
                            const float d = (m - most) * p.scale, f = exp2_approx(d);
                            const f32x2 f2 = pack2(f, f);
                            if (moments) moment = f != 0.0f ? mul2(f2, fma2(sum, pack2(d, d), moment)) : 0;
                            sum = mul2(sum, f2);
                            m = most;
                        }
                        // four vectors by themselves first: beside a term of 1, one below 2^-24 would be lost, and a thousand
                        // of them add up (the moment has no such term: d is 0 there)
                        const float ref = m == -INFINITY ? 0.0f : m;
                        const f32x2 minus = pack2(-ref, -ref);
                        f32x2 part;
#pragma unroll
                        for (int q = 0; q < 4; ++q)
#pragma unroll
                            for (int i = 0; i < kPairs; ++i) {
                                const f32x2 d = mul2(add2(Lanes<T>::pair(v[q], i), minus), scale), e = exp2_pair(d);
                                part = q + i == 0 ? e : add2(part, e);
                                if constexpr (moments) moment = fma2(e, finite_pair(d), moment);
                            }
                        sum = add2(sum, part);
                    }
                    if (!kWrite) {  // nobody else needs the chunk
                        if (patched) fence_async();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&empty[slot]);
                    }
                }
                // a lane that left alone has set `abort`: then the sums are not those of the row, and the message says NaN
                const int left_alone = *static_cast<volatile int*>(&abort);
                two_before = one_before, one_before = n;
                n += chunks;
                if (patched) fence_async();
                // the warp's message: its maximum, and sums relative to it
                float s0, s1;
                unpack2(sum, s0, s1);
                const float wm = warp_max_f32(m);
                const float down = m == wm || m == -INFINITY ? 0.0f : (m - wm) * p.scale, f = exp2_approx(down);
                float4 msg = make_float4(wm, f * (s0 + s1), 0.0f, 0.0f);
                if constexpr (moments) {
                    float e0, e1;
                    unpack2(moment, e0, e1);
                    if (f != 0.0f) msg.z = f * (e0 + e1) + down * msg.y;
                    msg.z = warp_reduce<float, add_op>(msg.z);
                }
                msg.y = warp_reduce<float, add_op>(msg.y);
                msg.y = left_alone ? NAN : msg.y;
                if (!may_send(u)) return;
                send(u, worker, msg);
                ++u;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&done[li]);
        }
        return;
    }
    if constexpr (kWrite) if (warp < kSumWarps + kWriteWarps) {
        constexpr int NT = 32 * kWriteWarps;
        const int w = warp - kSumWarps, tid = threadIdx.x - 32 * kSumWarps;
        Walk rows = walk;
#pragma unroll 1
        for (int64_t r; (r = rows.row()) < p.rows; rows.next(), ++turn) {
            const int li = turn % kLists;
            const bool ok = wait_alone(ready, turn, kLists) && (!wanted[li] || wait_alone(joined, u, kLists));
            if (!__all_sync(0xffffffffu, ok)) {  // a wait ran out: what is left becomes NaN
#pragma unroll 1
                for (; (r = rows.row()) < p.rows; rows.next()) write_constant<T, NT>(out_of(r), slice_of(r), tid, NAN);
                return;
            }
            const Slice<T> s = slice_of(r);
            if (!wanted[li]) {
                write_constant<T, NT>(out_of(r), s, tid, 0.0f);
            } else {
                ++u;
                const int chunks = chunks_of(s);
                T* out = out_of(r);
                const Gradient g = lists[li].g;
                const f32x2 minus = pack2(-g.m, -g.m), scale = pack2(p.scale, p.scale);
                const f32x2 c0 = pack2(g.c0, g.c0), c1 = pack2(g.c1, g.c1);
                const int32_t fb = s.full_begin(), fe = s.full_end();
#pragma unroll 1
                for (int c = (w + kWriteWarps - turn % kWriteWarps) % kWriteWarps; c < chunks; c += kWriteWarps) {
                    const uint32_t slot = (n + c) % kSlots;
                    wait_alone(full, n + c, kSlots);  // it has been: this thread sees the chunk too
                    const uint4* data = ring + slot * kChunk + lane;
                    auto gradient = [&](const uint4& v) {
                        float y[kVec];
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) {
                            const f32x2 d = mul2(add2(Lanes<T>::pair(v, i), minus), scale), e = exp2_pair(d);
                            unpack2(moments ? mul2(e, fma2(finite_pair(d), c1, c0)) : mul2(e, c0), y[2 * i], y[2 * i + 1]);
                        }
                        return Storage<T>::pack(y);
                    };
                    const int32_t at = s.origin() + (c * kChunk + lane) * kVec;
                    if (kAligned && c * kChunk >= fb && (c + 1) * kChunk <= fe) {
                        T* to = out + at;
#pragma unroll 1
                        for (int q = 0; q < kChunk / 32; q += 4, data += 128, to += 128 * kVec) {
#pragma unroll
                            for (int h = 0; h < 4; ++h) stg_stream16(to + 32 * kVec * h, gradient(data[32 * h]));
                        }
                    } else if (!kAligned) {
                        // the gradient in place of the chunk, and the chunk, one run of the row, from there
                        uint4* in_place = ring + slot * kChunk + lane;
                        const int count = min(kChunk, s.count - c * kChunk);
                        if (c * kChunk >= fb && (c + 1) * kChunk <= fe) {
#pragma unroll 1
                            for (int q = 0; q < kChunk / 32; q += 4, in_place += 128) {
#pragma unroll
                                for (int h = 0; h < 4; ++h) in_place[32 * h] = gradient(in_place[32 * h]);
                            }
                        } else {
#pragma unroll 1
                            for (int j = lane; j < count; j += 32, in_place += 32) {
                                const int k = c * kChunk + j;
                                *in_place = gradient(k < fb ? edges[li][0] : k >= fe ? edges[li][1] : *in_place);
                            }
                        }
                        __syncwarp();
                        write_run(out, s.origin() + c * (kChunk * kVec), s.origin() + (c * kChunk + count) * kVec, s.vocab,
                                  reinterpret_cast<const T*>(ring + slot * kChunk));
                        fence_async();
                    } else {
                        const int count = min(kChunk, s.count - c * kChunk);
#pragma unroll 1
                        for (int q = 0; 32 * q < count; ++q) {
                            const int j = 32 * q + lane, k = c * kChunk + j;
                            if (j >= count) break;
                            const uint4 x = gradient(kEdges && k < fb ? edges[li][0] : kEdges && k >= fe ? edges[li][1] : data[32 * q]);
                            if (k >= fb && k < fe) stg_stream16(out + at + 32 * q * kVec, x);
                            else write_edge(out, at + 32 * q * kVec, s.vocab, x);
                        }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&empty[slot]);
                }
                n += chunks;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&done[li]);
        }
        return;
    }
    if (warp == kSumWarps + kWriteWarps) {
        // ---- copy warp
        Walk rows = walk;
#pragma unroll 1
        for (int64_t r; (r = rows.row()) < p.rows; rows.next(), ++turn) {
            if (!wait_item(ready, turn, kLists)) return wait_copies(full, n, 0, &late[0]);
            const bool want = wanted[turn % kLists];
            __syncwarp();
            if (lane == 0) mbar_arrive(&done[turn % kLists]);
            if (!want) continue;
            const T* row = row_of(r);
            const Slice<T> s = slice_of(r);
            const T* base = row + s.origin();
            const int32_t fb = s.full_begin(), fe = s.full_end(), chunks = chunks_of(s);
            // a chunk for each lane, issued as its slot comes free (one lane issuing all took 470 cycles a chunk, a third of
            // what HBM delivers)
#pragma unroll 1
            for (int c0 = 0; c0 < chunks; c0 += 32) {
                const int c = c0 + lane;
                const uint32_t slot = (n + c) % kSlots, parity = ((n + c) / kSlots & 1) ^ 1;
                uint4* to = ring + slot * kChunk;
                const int32_t j0 = c * kChunk, j1 = min(j0 + kChunk, s.count), b0 = max(j0, fb), b1 = min(j1, fe);
                const uint32_t group = __ballot_sync(0xffffffffu, c < chunks);
                uint32_t pending = group;
                while (pending) {
                    const uint32_t first = n + c0 + __ffs(pending) - 1;  // slots come free in about this order
                    if (!wait(&empty[first % kSlots], (first / kSlots & 1) ^ 1, &abort))
                        return wait_copies(full, n + c0, group & ~pending, &late[0]);
                    const bool mine = (pending >> lane & 1) && mbar_try(&empty[slot], parity);
                    if (mine) {
                        if (b1 > b0) {
                            const uint32_t bytes = static_cast<uint32_t>(b1 - b0) * 16u;
                            mbar_expect_tx(&full[slot], bytes);
                            bulk_load(to + (b0 - j0), base + static_cast<int64_t>(b0) * kVec, bytes, &full[slot]);
                        }
                        if constexpr (!kWrite) *static_cast<volatile uint32_t*>(&issued[slot]) = n + c;
                        mbar_arrive(&full[slot]);
                    }
                    pending &= ~__ballot_sync(0xffffffffu, mine);
                }
                __syncwarp();
            }
            n += chunks;
        }
        return;
    }
    if (warp == kSumWarps + kWriteWarps + 1) {
        // ---- join warp
        bool expected = false;
        Walk rows = walk;
#pragma unroll 1
        for (; rows.row() < p.rows; rows.next(), ++turn) {
            const int li = turn % kLists;
            if (!wait_item(ready, turn, kLists)) break;
            if (wanted[li]) {
                const int set = u % kLists;
                if (lane == 0) mbar_arrive_expect_tx(&heard[set], ctas * (kMessages * 16u));
                __syncwarp();
                expected = true;
                if (!wait_item(heard, u, kLists)) break;
                expected = false;
                Op::template join<kSumWarps>(p, lists[li], inbox[set], static_cast<int>(ctas));
                __syncwarp();
                if (lane == 0) mbar_arrive(&joined[set]);
                ++u;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&done[li]);
        }
        __syncwarp();
        if (ctas > 1) {
            cluster_sync();
            if (abort) wait_messages(heard, u, expected, ctas * (kMessages * 16u), &late[1]);
        }
        return;
    }
    if (warp == kSumWarps + kWriteWarps + 2) {
        // ---- end warp: what is left to do of a row once the others are through with it
        Walk rows = walk;
#pragma unroll 1
        for (int64_t r; (r = rows.row()) < p.rows; rows.next(), ++turn) {
            const int li = turn % kLists;
            if (!wait_item(done, turn, kLists)) break;
            if (wanted[li]) Op::template fix<T>(p, lists[li], slice_of(r), kWrite ? out_of(r) : nullptr, r, rank == 0);
            else if (rank == 0 && lane == 0) Op::without(p, r, 0.0f);
            __syncwarp();
            if (lane == 0) mbar_arrive(&retired[li]);
        }
        if (rank == 0 && lane == 0)  // a wait ran out, if any rows are left
#pragma unroll 1
            for (; rows.row() < p.rows; rows.next()) Op::without(p, rows.row(), NAN);
        return;
    }
    // ---- list warps
    turn = warp - (kSumWarps + kWriteWarps + 3);
    Walk rows = walk;
    rows.next(turn);
    Walk ahead = rows;
    ahead.next(kListWarps);
    typename Op::Fetched next = Op::fetch(p, rows.row()), later = Op::fetch(p, ahead.row());
    Op::template gather<T>(p, rows.row(), next);
    // an element of the first or last vector of a slice, where that reaches past the row
    auto edge_of = [&](int64_t r) {
        if (!kEdges || r >= p.rows || lane >= 2 * kVec) return masked<T>();
        const Slice<T> s = slice_of(r);
        const int32_t i = s.origin() + (lane < kVec ? lane : (s.count - 2) * kVec + lane);
        return s.count > 0 && i >= 0 && i < s.vocab ? row_of(r)[i] : masked<T>();
    };
    T edge = edge_of(rows.row());
#pragma unroll 1
    for (int64_t r; (r = rows.row()) < p.rows; rows.next(kListWarps), turn += kListWarps) {
        const int li = turn % kLists;
        typename Op::Shared& sh = lists[li];
        if (turn >= kLists && !wait_item(retired, turn - kLists, kLists)) return;
        const typename Op::Fetched now = next;
        next = later;
        const int64_t following = ahead.row();
        ahead.next(kListWarps);
        Op::template gather<T>(p, following, next);
        later = Op::fetch(p, ahead.row());
        const T edge_now = edge;
        edge = edge_of(following);
        const bool want = Op::wanted(p, now);
        if (want) {
            Op::begin(p, sh, now);
            if (kEdges && lane < 2 * kVec) reinterpret_cast<T*>(edges[li])[lane] = edge_now;
            if constexpr (Op::kMask) {
                // the special elements in this slice by chunk: how many each has, where it begins, and each element's place
                const Slice<T> s = slice_of(r);
                chunk_begin[li][lane] = chunk_begin[li][lane + 32] = 0;
                __syncwarp();
                int in[Op::kMine], place[Op::kMine];
#pragma unroll
                for (int i = 0; i < Op::kMine; ++i) {
                    const int k = lane + 32 * i, pos = k < Op::entries(p) ? sh.pos[k] : -1;
                    in[i] = s.holds(pos) ? (pos - s.origin()) / (kChunk * kVec) : -1;
                    place[i] = 0;
                    if (!__any_sync(0xffffffffu, in[i] >= 0)) continue;
                    const uint32_t same = __match_any_sync(0xffffffffu, in[i]);
                    if (in[i] >= 0) place[i] = chunk_begin[li][in[i] + 1] + __popc(same & ((1u << lane) - 1));
                    __syncwarp();
                    if (in[i] >= 0 && (same >> lane) == 1) chunk_begin[li][in[i] + 1] += __popc(same);  // the last of its chunk
                    __syncwarp();
                }
                int a = chunk_begin[li][lane], b = chunk_begin[li][lane + 32];
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const int up = __shfl_up_sync(0xffffffffu, a, o), up2 = __shfl_up_sync(0xffffffffu, b, o);
                    if (lane >= o) a += up, b += up2;
                }
                b += __shfl_sync(0xffffffffu, a, 31);
                __syncwarp();
                chunk_begin[li][lane] = static_cast<uint8_t>(a);
                chunk_begin[li][lane + 32] = static_cast<uint8_t>(b);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < Op::kMine; ++i)
                    if (in[i] >= 0) order[li][chunk_begin[li][in[i]] + place[i]] = static_cast<uint8_t>(lane + 32 * i);
#pragma unroll
                for (int i = 0; i < Op::kMine; ++i) {  // and in the edges
                    if (!kEdges || in[i] < 0) continue;
                    const int32_t at = sh.pos[lane + 32 * i] - s.origin(), last = at - (s.count - 1) * kVec;
                    if (at < kVec) reinterpret_cast<T*>(edges[li])[at] = masked<T>();
                    if (last >= 0) reinterpret_cast<T*>(edges[li])[kVec + last] = masked<T>();
                }
            }
        }
        if (lane == 0) wanted[li] = want;
        __syncwarp();
        if (lane == 0) mbar_arrive(&ready[li]);
    }
}

// ---- small problems --------------------------------------------------------------------------------------------------

// The same for problems whose time is latency: a CTA (of a cluster, where there are few rows or long ones) takes a slice of up
// to 32 KB straight into registers, its first warp the special elements meanwhile; sums, exchange, gradient, end.  One
// launch, no stage that waits for another, up to 32 CTAs on an SM.  Measured (when it was built), us: one row of 8192 fp32 5.6 (the pipeline:
// 9.0), 128 x 8192 bf16 6.5 (9.2), 1024 x 8192 fp32 backward 13.4 = 77 % of a copy's rate (21).
constexpr int kSmallVectors = 8;  // of a thread

template <typename T, int NT, typename Op, bool kAligned>
__global__ void __launch_bounds__(NT, 1024 / NT) row_gradient_small_kernel(const typename Op::Params p, const int32_t per_cta) {
    constexpr int kVec = Storage<T>::kVec, kPairs = kVec / 2;
    constexpr int kWarps = NT / 32;
    constexpr bool moments = Op::kMoments;
    __shared__ typename Op::Shared sh;
    __shared__ __align__(16) float4 inbox[kMaxCluster];
    __shared__ __align__(16) uint4 stage[kAligned ? 1 : kWarps][32];
    __shared__ float4 warp_sums[kWarps];
    __shared__ float warp_max[kWarps];
    __shared__ __align__(4) uint8_t special[Op::kMask ? NT * kSmallVectors : 1];  // which elements of a vector leave them; set by words
    __shared__ bool want;
    const uint32_t ctas = cluster_size(), rank = cluster_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    start_after_last();
    if (ctas > 1) cluster_arrive();  // waited for before the first store into another CTA
    const int64_t r = blockIdx.x / ctas;
    const T* row = static_cast<const T*>(p.logits) + r * p.row_stride;
    T* out = p.dlogits ? static_cast<T*>(p.dlogits) + r * p.dlogits_stride : nullptr;
    const Slice<T> s(row, p.vocab, per_cta, rank);
    const int32_t fb = s.full_begin(), fe = s.full_end();
    uint4 v[kSmallVectors];
#pragma unroll
    for (int q = 0; q < kSmallVectors; ++q) {
        const int32_t j = q * NT + tid;
        v[q] = Lanes<T>::masked4();
        if (j >= fb && j < fe) v[q] = load_stream(row + s.origin() + j * kVec);
        else if (j < s.count) v[q] = load_edge_rw(row, s.origin() + j * kVec, s.vocab);
    }
    if (Op::kMask) {
        for (int i = tid; i < NT * kSmallVectors / 4; i += NT) reinterpret_cast<uint32_t*>(special)[i] = 0;
        __syncthreads();
    }
    if (warp == 0) {
        typename Op::Fetched now = Op::fetch(p, r);
        Op::template gather<T>(p, r, now);
        const bool wanted = Op::wanted(p, now);
        if (wanted) Op::begin(p, sh, now);
        if (lane == 0) want = wanted;
        __syncwarp();
        if (Op::kMask && wanted)
#pragma unroll 1
            for (int k = lane; k < Op::entries(p); k += 32)
                if (s.holds(sh.pos[k])) {
                    const int at = sh.pos[k] - s.origin(), bit = at / kVec * 8 + at % kVec;
                    atomicOr(reinterpret_cast<uint32_t*>(special) + bit / 32, 1u << bit % 32);
                }
    }
    let_next_start();
    if (Op::kMask) {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kSmallVectors; ++q) {
            const uint32_t bits = special[q * NT + tid];
            if (bits) v[q] = Lanes<T>::without(v[q], bits);
        }
    }
    typename Lanes<T>::Max top;
#pragma unroll
    for (int q = 0; q < kSmallVectors; ++q) top.take(v[q]);
    const float mine = top.get();  // NaN if there is one: then all of the row becomes NaN
    {
        const float wm = mine != mine ? INFINITY : mine;
        const float x = warp_max_f32(wm);
        if (lane == 0) warp_max[warp] = x;
    }
    __syncthreads();
    if (!want) {
        if (out) write_constant<T, NT>(out, s, tid, 0.0f);
        if (rank == 0 && tid == 0) Op::without(p, r, 0.0f);
        if (ctas > 1) cluster_wait();
        return;
    }
    float m = warp_max[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m = fmaxf(m, warp_max[w]);
    const float ref = m == -INFINITY ? 0.0f : m;
    const f32x2 minus = pack2(-ref, -ref), scale = pack2(p.scale, p.scale);
    f32x2 sum = 0, moment = 0;
#pragma unroll
    for (int q = 0; q < kSmallVectors; ++q) {
        if (q * NT >= s.count) break;
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const f32x2 d = mul2(add2(Lanes<T>::pair(v[q], i), minus), scale), e = exp2_pair(d);
            sum = add2(sum, e);
            if constexpr (moments) moment = fma2(e, finite_pair(d), moment);
        }
    }
    float s0, s1, e0, e1;
    unpack2(sum, s0, s1);
    unpack2(moment, e0, e1);
    float4 x = make_float4(m, s0 + s1, e0 + e1, 0.0f);
    x.y = warp_reduce<float, add_op>(x.y);
    if constexpr (moments) x.z = warp_reduce<float, add_op>(x.z);
    if (lane == 0) warp_sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
        x = warp_sums[0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) x.y += warp_sums[w].y, x.z += warp_sums[w].z;
        if (ctas == 1) {
            if (lane == 0) inbox[0] = x;
        } else {
            cluster_wait();
            if (lane < static_cast<int>(ctas)) store_remote(&inbox[rank], lane, x);
        }
        __syncwarp();
    }
    if (ctas > 1) {
        if (warp != 0) cluster_wait();
        cluster_arrive();
        cluster_wait();
    }
    if (warp == 0) Op::template join<1>(p, sh, inbox, static_cast<int>(ctas));
    __syncthreads();
    if (out) {
        const Gradient g = sh.g;
        const f32x2 minus_m = pack2(-g.m, -g.m), c0 = pack2(g.c0, g.c0), c1 = pack2(g.c1, g.c1);
#pragma unroll
        for (int q = 0; q < kSmallVectors; ++q) {
            if (q * NT >= s.count) break;
            const int32_t j = q * NT + tid, at = s.origin() + j * kVec, j0 = j - lane;
            float y[kVec];
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                const f32x2 d = mul2(add2(Lanes<T>::pair(v[q], i), minus_m), scale), e = exp2_pair(d);
                unpack2(moments ? mul2(e, fma2(finite_pair(d), c1, c0)) : mul2(e, c0), y[2 * i], y[2 * i + 1]);
            }
            const uint4 w = Storage<T>::pack(y);
            if (kAligned) {
                if (j >= fb && j < fe) stg_stream16(out + at, w);
                else if (j < s.count) write_edge(out, at, s.vocab, w);
            } else if (j0 >= fb && j0 + 32 <= fe) {
                __syncwarp();
                stage[warp][lane] = w;
                __syncwarp();
                write_run(out, at - lane * kVec, stage[warp]);
            } else if (j < s.count) {
                write_edge(out, at, s.vocab, w);
            }
        }
        __syncthreads();  // the special elements are written after the others
    }
    if (warp == 0) Op::template fix<T>(p, sh, s, out, r, rank == 0);
}

// ---- host ----------------------------------------------------------------------------------------------------------

template <typename T, typename Op, bool kAligned, bool kEdges, bool kWrite>
cudaError_t launch_gradient_pipeline(const typename Op::Params& p, int64_t all, cudaStream_t st) {
    auto kernel = row_gradient_kernel<T, Op, kAligned, kEdges, kWrite>;
    // CTAs a row: slices of up to 128 KB (80 KB of rows that are not aligned), of up to 192 KB where 8 of them are not enough;
    // where there are few rows, more and smaller ones, down to a chunk for every sum warp.  Measured with slices of up to 128,
    // 96 and 72 KB, us (when this was chosen): 4096 x 131072 bf16 386, 400, 417; 2047 x 100003 bf16 175, 160, 160 (156 with 80).
    constexpr int kGood = (kEdges ? 20 : 32) * kChunk;
    int ctas = 1;
    while (ctas < kMaxCluster && (all + ctas - 1) / ctas > kGood) ++ctas;
    while (2 * ctas <= kMaxCluster && p.rows * 2 * ctas <= qn_sm_count() && all / ctas > Roles<kWrite>::kSum * kChunk) ctas *= 2;
    const int per_cta = static_cast<int>((all + ctas - 1) / ctas);
    if (per_cta > kSlots * kChunk) return cudaErrorInvalidValue;
    constexpr int kBytes = kSlots * kChunk * 16;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(Roles<kWrite>::kThreads);
    cfg.dynamicSmemBytes = kBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    // clusters that fit on the device at once, by cluster size; asked for once
    static int fit[64][kMaxCluster + 1];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    int& clusters = fit[dev][ctas];
    if (clusters == 0) {
        int found = 0;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&found, kernel, &cfg);
        if (e != cudaSuccess) return e;
        if (found < 1) return cudaErrorInvalidConfiguration;
        clusters = found;
    }
    cfg.gridDim = dim3(static_cast<unsigned>((p.rows < clusters ? p.rows : clusters) * ctas));
    uint32_t stride = static_cast<uint32_t>(clusters);
    while (stride % 2 == 0 || stride % 3 == 0 || stride % 5 == 0 || stride % 7 == 0) ++stride;
    return cudaLaunchKernelEx(&cfg, kernel, p, static_cast<int32_t>(per_cta), (stride - static_cast<uint32_t>(clusters)) % static_cast<uint32_t>(clusters));
}

// Every row starts on 16 bytes.
template <typename T, typename Params>
bool rows_aligned(const Params& p) {
    return reinterpret_cast<uintptr_t>(p.logits) % 16 == 0 && (p.rows == 1 || p.row_stride % Storage<T>::kVec == 0);
}

// Vectors that a row may span, whatever its alignment.
template <typename T, typename Params>
int64_t row_vectors(const Params& p) {
    constexpr int kVec = Storage<T>::kVec;
    return (static_cast<int64_t>(p.vocab) + (rows_aligned<T>(p) ? kVec - 1 : 2 * kVec - 2)) / kVec;
}

template <typename T, int NT, typename Op, bool kAligned>
cudaError_t launch_gradient_small(const typename Op::Params& p, int ctas, cudaStream_t st) {
    const EarlyLaunch launch(p.rows * ctas, NT, 0, ctas, st);
    const int per_cta = static_cast<int>((row_vectors<T>(p) + ctas - 1) / ctas);
    return cudaLaunchKernelEx(&launch.cfg, row_gradient_small_kernel<T, NT, Op, kAligned>, p, static_cast<int32_t>(per_cta));
}

template <typename T, typename Op, bool kAligned>
cudaError_t launch_gradient_aligned(const typename Op::Params& p, cudaStream_t st) {
    const int64_t all = row_vectors<T>(p);
    int ctas = 1;
    while (ctas <= kMaxCluster && all > ctas * 256 * kSmallVectors) ++ctas;
    // Rows in flight one by one against the pipeline.  Measured, us (rows x vocab, small kernel / pipeline; the list has 32
    // tokens): bf16 128 x 131072 20 / 22, 1024 x 32000 36 / 36, 8192 x 32000 260 / 207, 1024 x 131072 134 / 115,
    // 8192 x 8192 87 / 118; fp32 128 x 32000 9.7 / 14, 1024 x 32000 71 / 53, 1024 x 8192 17 / 21, 8192 x 8192 129 / 116;
    // one row of 8192: 5 / 9.  So: all logits more than 64 MB, in rows of more than 32 KB.
    const int64_t bytes = p.vocab * static_cast<int64_t>(sizeof(T));
    if (ctas > kMaxCluster || p.rows > INT32_MAX / kMaxCluster || (bytes > (32 << 10) && p.rows > (64 << 20) / bytes))
    {
        // rows that start and end on 16 bytes have no vectors that reach past them
        const bool edges = !rows_aligned<T>(p) || p.vocab % Storage<T>::kVec != 0;
        if constexpr (!Op::kAlone) {
            if (!kAligned) return launch_gradient_pipeline<T, Op, false, true, true>(p, all, st);
            return edges ? launch_gradient_pipeline<T, Op, true, true, true>(p, all, st)
                         : launch_gradient_pipeline<T, Op, true, false, true>(p, all, st);
        } else {
            if (!p.dlogits)
                return edges ? launch_gradient_pipeline<T, Op, true, true, false>(p, all, st)
                             : launch_gradient_pipeline<T, Op, true, false, false>(p, all, st);
            if (!kAligned) return launch_gradient_pipeline<T, Op, false, true, true>(p, all, st);
            return edges ? launch_gradient_pipeline<T, Op, true, true, true>(p, all, st)
                         : launch_gradient_pipeline<T, Op, true, false, true>(p, all, st);
        }
    }
    // few rows: more CTAs, down to a vector a thread; many: no more threads than a row has work for
    while (2 * ctas <= kMaxCluster && p.rows * 2 * ctas <= 2 * qn_sm_count() && all > ctas * 256) ctas *= 2;
    const bool many = p.rows * ctas > 4 * qn_sm_count();
    if (all <= 64 || (many && all <= 64 * kSmallVectors)) return launch_gradient_small<T, 64, Op, kAligned>(p, ctas, st);
    return launch_gradient_small<T, 256, Op, kAligned>(p, ctas, st);
}

template <typename T, typename Op>
cudaError_t launch_gradient(const typename Op::Params& p, cudaStream_t st) {
    const auto off = [](const void* at) { return reinterpret_cast<uintptr_t>(at) % 16; };
    const bool aligned = !p.dlogits || (off(p.logits) == off(p.dlogits) &&
                                        (p.rows == 1 || (p.row_stride - p.dlogits_stride) * sizeof(T) % 16 == 0));
    return aligned ? launch_gradient_aligned<T, Op, true>(p, st) : launch_gradient_aligned<T, Op, false>(p, st);
}

}  // namespace
