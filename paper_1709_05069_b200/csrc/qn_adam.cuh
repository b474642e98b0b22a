// Shared by the kernels of qn_adam_*: a plan's tensors and who works on which of them, the numbers that round by chance, and
// the states in 8 bits.
//
// States in 8 bits.  A block is 32 elements of a tensor; its scale is a power of two, 2^(s - 127), that puts the block's
// largest magnitude in [128, 256) (s = 0: the block is zero).  With a power of two the scaling is exact, so that a code depends
// on its own element and the binade of the block's maximum alone.  m is held in E4M3 (as in torch.float8_e4m3fn), and r = sqrt(v)
// in 4 bits of exponent and 4 of fraction: the root has half of v's range in binades, and one more bit of fraction in place of
// the sign that it does not need.  Both have steps of 2^-9 and 2^-10 below 2^-6, so that a block spans 2^17 in m and
// 2^36 in v.  A moving average with b2 = 0.999 moves by 1/2000 of r a step where codes are 1/16 apart: rounded to
// nearest it would stand still, so codes are rounded up or down with the probabilities that keep the mean.  A root that is not 0
// is never rounded to 0, which would leave m' / eps as the next step.  The arithmetic that leads to a code is in 32
// bits, each operation rounded by itself (no fused ones), so that the codes are the same wherever they are computed.
#pragma once

#include <utility>
#include <vector>

#include <cuda_fp16.h>

#include "qn_vocab.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kOctet = 8;                  // elements that share a hash
constexpr int kPiece = kThreads * kOctet;  // elements that a CTA has in hand at a time
constexpr int kMostCtas = 8;               // on an SM

struct Record {
    int64_t numel, octet;  // octet: the tensor's first place, in units of eight
    void* param;
    const void* grad;
    float* master;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    double decay, lr_scale;
};

// The tensors as pieces, one after the other: tensor t has those from first[t] to first[t + 1].
struct Tensors {
    const Record* records;
    const int64_t* first;
    int32_t count;
    int64_t pieces;
};

// ---- a CTA's share -----------------------------------------------------------------------------------------------------

// A CTA's turns at runs of pieces, the CTAs one after the other: `each` pieces in a run, so that all have as many turns and pieces, give
// or take one.  Within a run addresses only move on, but for the ends of tensors; the shorter the runs, the nearer to one another
// in memory the CTAs are.  Measured with runs of whole shares, and of at least 32, 8 and 4 pieces (at most 8, 32 and 64 turns),
// us for 2^28 parameters: the step with 32-bit states and master copies 1331, 1281, 1237, 1228; with 8-bit states, whose copies ahead end
// with a run, 573, 571, 615, 673 (for 2^27 fp32 parameters with runs of whole shares, 32 and 16 pieces 549, 532, 519); the norm 88, 88,
// 94, 107; the states' values 315, 295, 286, 294.
struct Turns {
    int64_t pieces, each;
    int32_t count;
    __device__ __forceinline__ Turns(int64_t pieces_, int run, int most_turns) : pieces(pieces_) {
        const int64_t most = pieces / (gridDim.x * static_cast<int64_t>(run));
        count = static_cast<int32_t>(most < 1 ? 1 : most > most_turns ? most_turns : most);
        each = (pieces + gridDim.x * count - 1) / (static_cast<int64_t>(gridDim.x) * count);
    }
    __device__ __forceinline__ int64_t lo(int turn) const { return min(pieces, (static_cast<int64_t>(turn) * gridDim.x + blockIdx.x) * each); }
    __device__ __forceinline__ int64_t hi(int turn) const { return min(pieces, lo(turn) + each); }
};
// The tensor of one piece: by all threads, each looks at some of the tensors.
__device__ __forceinline__ void find_tensor(const Tensors& all, int64_t piece, int* found) {
#pragma unroll 1
    for (int t = threadIdx.x; t < all.count; t += kThreads)
        if (all.first[t] <= piece && piece < all.first[t + 1]) *found = t;
}

// ---- random numbers ------------------------------------------------------------------------------------------------

// A hash of 32 bits by multiplication and shifts; the shifts 15, 13 and 16 between products are those of the last steps of the published
// hash XXH32.  The multipliers are the first 32 bits of the fractions of sqrt(3), sqrt(5) and sqrt(7), made odd, and for what is counted up
// Knuth's for multiplicative hashing, the prime 2654435761 next to the golden ratio's fraction; the means, pairwise correlations and
// two-dimensional histograms of what comes out were looked at.
constexpr uint32_t kGolden = 0x9E3779B1u, kMix1 = 0xBB67AE85u, kMix2 = 0x3C6EF373u, kMix3 = 0xA54FF53Bu;

__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 15;
    x *= kMix1;
    x ^= x >> 13;
    x *= kMix2;
    return x ^ (x >> 16);
}
// One number for each step, from all bits of the seed and of the step.
__device__ __forceinline__ uint32_t step_key(uint32_t seed_low, uint32_t seed_high, int64_t step) {
    const uint32_t key = mix(mix(seed_low) + seed_high);
    return mix(mix(key + static_cast<uint32_t>(step) * kGolden) + static_cast<uint32_t>(step >> 32));
}
// One for each eight elements, and one for each of them: the upper half of the latter rounds m, the lower half r, and the upper
// half of its product with another number theta.
__device__ __forceinline__ uint32_t octet_word(uint32_t key, uint32_t octet) { return mix(octet * kGolden + key); }
__device__ __forceinline__ uint32_t element_word(uint32_t octet, uint32_t j) {
    uint32_t y = octet + j * kGolden;
    y = (y ^ (y >> 15)) * kMix3;
    return y ^ (y >> 16);
}

// ---- 8 bits --------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float power_of(uint32_t exponent) { return __uint_as_float(exponent << 23); }

// The scale of a block whose largest finite magnitude has these bits.
__device__ __forceinline__ uint32_t scale_of(uint32_t most) {
    return most == 0 ? 0u : static_cast<uint32_t>(max(static_cast<int>(most >> 23) - 7, 1));
}
__device__ __forceinline__ float up_by(uint32_t scale) { return power_of(scale ? 254u - scale : 127u); }

// |x| 2^-e as a number whose exponent field is the code's: 2^-6, the codes' smallest normal number, becomes the
// smallest normal number in 32 bits, so that what lies below falls on equal steps by itself.  The bits below the code's
// are the chance to be rounded up.
__device__ __forceinline__ uint32_t magnitude_bits(float x, float up) {
    return __float_as_uint(__fmul_rn(__fmul_rn(fabsf(x), up), 0x1p-120f));
}
constexpr uint32_t kInfinity = 0x7f800000u;
__device__ __forceinline__ uint32_t m_code(float m, float up, uint32_t word) {
    const uint32_t bits = __float_as_uint(m);
    if ((bits & 0x7fffffffu) >= kInfinity) return 0x7fu;  // NaN
    const uint32_t chance = ((word >> 12) & 0xffff0u) | 8u;
    return ((magnitude_bits(m, up) + chance) >> 20) | (bits >> 24 & 0x80u);  // -0 has its sign too, as in the packed ways
}
__device__ __forceinline__ uint32_t root_code(float r, float up, uint32_t word) {
    if (__float_as_uint(r) >= kInfinity) return 0xffu;  // the largest
    const uint32_t chance = ((word << 3) & 0x7fff8u) | 4u;
    return max((magnitude_bits(r, up) + chance) >> 19, r > 0.0f ? 1u : 0u);
}
__device__ __forceinline__ float m_value(uint32_t code, uint32_t scale) {
    const float x = __uint_as_float((code & 0x7fu) << 20) * 0x1p120f * power_of(scale);
    return (code & 0x7fu) == 0x7fu ? NAN : code & 0x80u ? -x : x;
}
__device__ __forceinline__ float root_value(uint32_t code, uint32_t scale) {
    return __uint_as_float(code << 19) * 0x1p120f * power_of(scale);
}
// Bits of a magnitude, 0 where it is not finite: the maximum of these makes a block's scale.
__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t bits = __float_as_uint(x) & 0x7fffffffu;
    return bits < kInfinity ? bits : 0u;
}

// ---- eight elements of a thread ----------------------------------------------------------------------------------------

// What is written back in place is read with ordinary loads: by the thread that writes it.
__device__ __forceinline__ void load8(const void* p, uint32_t (&x)[8]) {
    asm volatile("ld.global.L1::no_allocate.v8.u32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void load8(const void* p, uint32_t (&x)[4]) {
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void load8(const void* p, uint32_t (&x)[2]) {
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]),
                 "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = Storage<__nv_bfloat16>::pack(x);
}
// Elements 2 q and 2 q + 1 of eight in 32 bits, or in 16.
__device__ __forceinline__ f32x2 two_of(const uint32_t (&x)[8], int q) { return pack2(__uint_as_float(x[2 * q]), __uint_as_float(x[2 * q + 1])); }
__device__ __forceinline__ f32x2 two_of(const uint32_t (&x)[4], int q) {
    return pack2(__uint_as_float(x[q] << 16), __uint_as_float(x[q] & 0xffff0000u));
}

__device__ __forceinline__ f32x2 both(float x) { return pack2(x, x); }

// What two codes of m (in the lower bytes), or of a root (in bytes 0 and 2), stand for, but for the scale; a root's 2^8 too small: a
// half has the same kind of fraction with five bits of exponent, so that a code moved up by 6 is one.
__device__ __forceinline__ f32x2 m_values(uint32_t codes) {
    uint32_t halves;
    asm("{\n .reg .b16 lo;\n cvt.u16.u32 lo, %1;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n}" : "=r"(halves) : "r"(codes));
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&halves));
    return pack2(x.x, x.y);
}
__device__ __forceinline__ f32x2 root_values(uint32_t codes) {
    const uint32_t halves = codes << 6;
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&halves));
    return pack2(x.x, x.y);
}
__device__ __forceinline__ float root_unit(uint32_t scale) { return scale ? power_of(min(scale + 8u, 254u)) : 0.0f; }
__device__ __forceinline__ void m_values(const uint32_t (&codes)[2], f32x2 (&m)[4]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) m[q] = m_values(codes[q / 2] >> (16 * (q & 1)));
}
__device__ __forceinline__ void root_values(const uint32_t (&codes)[2], f32x2 (&r)[4]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) r[q] = root_values(__byte_perm(codes[q / 2], 0, q & 1 ? 0x4342 : 0x4140));
}

}  // namespace

// ---- a plan ------------------------------------------------------------------------------------------------------------

struct qn_adam_plan {
    int device = -1;
    int32_t count = 0;
    qn_dtype param = QN_F32, grad = QN_F32;
    bool master = false, eight = false;
    int64_t places = 0, pieces = 0;
    void* block = nullptr;  // device memory: records, first pieces, partial sums, tickets
    Record* records = nullptr;
    int64_t* first = nullptr;
    double* partials = nullptr;
    unsigned* tickets = nullptr;  // of the step, of the norm
    std::vector<int64_t> numel;
    std::vector<std::pair<uintptr_t, uintptr_t>> written;  // in order

    Tensors tensors() const { return Tensors{records, first, count, pieces}; }
};

namespace {

// As many CTAs as are on the device at once (asked for once on each), or one for each piece.
struct Resident {
    int on[64];
};
template <typename... P, typename... A>
cudaError_t launch_over(void (*kernel)(P...), Resident& known, size_t shared, const qn_adam_plan& h, cudaStream_t st, A... args) {
    if (h.device < 0 || h.device >= 64) return cudaErrorInvalidDevice;
    int& resident = known.on[h.device];
    if (resident == 0) {
        int found = 0;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(shared));
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&found, kernel, kThreads, shared);
        if (e != cudaSuccess) return e;
        resident = found < 1 ? 1 : found > kMostCtas ? kMostCtas : found;
    }
    const int64_t most = static_cast<int64_t>(resident) * qn_sm_count(), ctas = h.pieces < most ? h.pieces : most;
    const EarlyLaunch launch(ctas < 1 ? 1 : ctas, kThreads, shared, 1, st);
    return cudaLaunchKernelEx(&launch.cfg, kernel, h.tensors(), args...);
}

}  // namespace
