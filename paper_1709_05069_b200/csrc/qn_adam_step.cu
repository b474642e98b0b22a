// qn_adam_step: AdamW over the tensors of one parameter vector, with states in 32 bits or in 8.
//
// Per element, with g~ = c g (c: the clip coefficient times grad_scale) and t the number of this step:
//     m' = b1 m + (1 - b1) g~        v' = b2 v + (1 - b2) g~^2        r' = sqrt(v')
//     theta' = theta (1 - lr wd) - lr / (1 - b1^t) m' / (r' / sqrt(1 - b2^t) + eps)
// Nothing is reused, so the floor is the bytes: each array once in and once out.
//
// CTAs stay and take turns at runs of pieces (see Turns), backwards: the last gradients that qn_adam_norm has read are the
// first to be read again, from L2.  A thread has eight elements, in vectors of 8 to 32 bytes, and works on two at a time
// (packed fp32).  Where tensors do not lie on such vectors, states in 8 bits go by way of shared memory, where they do, and
// states in 32 bits an element a lane, eight for each thread; so does, with both, what is left of a piece where a tensor ends.
//
// Measured on a B200 (a copy: 6.54 TB/s), bytes of the floor over time:
//   states in 32 bits: bound by memory.  2^28 bf16 parameters with master copies (28 bytes an element) 1195 to 1210 us = 6.3 to 6.2 TB/s,
//       without (22 bytes) 913 us = 6.5 TB/s to nearest and by chance, 25.6 million fp32 ones 118 us = 6.1 TB/s; off vectors 4.4 to
//       5.1 TB/s: four-byte accesses.  With two CTAs on an SM and 88 registers 3 % less than with three and 80.
//   states in 8 bits: 57 instructions an element, of which 27 go to the integer and comparison pipe; three quarters of the issue
//       slots, two thirds of that pipe.  2^28 bf16 parameters 557 to 578 us = 4.9 to 4.7 TB/s, to nearest 528 us, with master copies
//       895 us = 4.8 TB/s, 2^27 fp32 ones 500 us (bf16 gradients: 394 us) = 4.3 (4.8) TB/s; off vectors 80 instructions, 2^27 bf16 ones
//       428 us = 3.2 TB/s, 25.6 million fp32 ones 107 us (an element a lane 93, 558 and 120).
//       What the packed way does not take is slow, elements with v' = 0 above all: 2^27 bf16 parameters 266 us, with one of 64 elements or
//       all without history 1150 us, with every other 1024 elements 885 us; off vectors, where a warp's 256 elements go together, 400 us, 3.0
//       and 1.6 ms.
//   Steps on the way (2^28 bf16, 8 bits): an element a lane 4.3 ms; eight elements a thread in vectors 1106 us (81
//       instructions, two CTAs on an SM); the root by one correction instead of a call, reciprocals, codes put together from
//       upper bytes 763; runs instead of chunks 726; copies ahead through shared memory 581 (three slots 619, six 605); turns,
//       folded constants and slots by name 578.  The same constants from shared memory instead of registers changed nothing;
//       nor did, off vectors, fewer instructions for the copies and for the ends of a warp's codes (107 and 439 us).
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <type_traits>

#include "qn_adam.cuh"

namespace {

struct Hyper {
    double lr, log_beta1, log_beta2, max_norm, grad_scale;
    float beta1, rest1, beta2, rest2, eps, minus_zero;
    uint32_t seed_low, seed_high;
};

// What is the same for all elements of a step.
struct Common {
    int64_t t;
    double lr, speed;           // learning rate, and lr / (1 - b1^t)
    float coefficient, spread;  // spread: 1 / sqrt(1 - b2^t)
    uint32_t key;
    bool skip;  // the gradients' norm is not finite
};
struct Setting {
    Hyper h;
    Common c;
};

// By four threads, since each part is a chain of operations in 64 bits.
__device__ __forceinline__ void make_common(const Hyper& h, const int64_t* step, const float* lr, const double* sumsq, Common& c) {
    const int part = threadIdx.x / 32;
    if (threadIdx.x % 32 != 0 || part > 3) return;
    if (part == 2) {
        double coefficient = h.grad_scale;
        c.skip = false;
        if (sumsq) {
            const double norm = sqrt(*sumsq) * fabs(h.grad_scale);
            c.skip = !isfinite(norm);
            if (h.max_norm > 0.0 && norm > h.max_norm) coefficient *= h.max_norm / norm;
        }
        c.coefficient = static_cast<float>(coefficient);
        return;
    }
    const int64_t t = *step + 1;
    if (part == 0) {
        c.lr = lr ? static_cast<double>(*lr) : h.lr;
        c.speed = c.lr / -expm1(static_cast<double>(t) * h.log_beta1);
        c.t = t;
    } else if (part == 1) {
        c.spread = static_cast<float>(1.0 / sqrt(-expm1(static_cast<double>(t) * h.log_beta2)));
    } else {
        c.key = step_key(h.seed_low, h.seed_high, t);
    }
}

// The same for all elements of a tensor.
struct Rates {
    float keep, speed;  // 1 - lr wd, lr / (1 - b1^t)
    // 1 / sqrt(1 - b2^t) and eps in units of speed: speed / (r spread + eps) as one reciprocal.  For a speed of 0 they are infinite, and for
    // r > 0 the step is 0, as it should be.
    float spread, eps;
    __device__ __forceinline__ Rates(const Hyper& h, const Common& c, const Record& r)
        : keep(static_cast<float>(1.0 - c.lr * r.lr_scale * r.decay)), speed(static_cast<float>(c.speed * r.lr_scale)),
          spread(c.spread / speed), eps(h.eps / speed) {}
};

// Where a run of a tensor's elements begins, and how many there are.  S: float, or uint8_t for codes.
template <typename P, typename G, bool kMaster, typename S>
struct Part {
    P* param;
    const G* grad;
    float* master;
    S *m, *v;
    uint8_t *m_scale, *v_scale;
    uint32_t octet;  // the first one's place (its low half: the hash takes no more)
    int32_t count;
    __device__ __forceinline__ Part(const Record& r, int64_t begin, int64_t count_)
        : param(static_cast<P*>(r.param) + begin), grad(static_cast<const G*>(r.grad) + begin),
          master(kMaster ? r.master + begin : nullptr), m(static_cast<S*>(r.m) + begin), v(static_cast<S*>(r.v) + begin),
          m_scale(r.m_scale + begin / QN_ADAM_BLOCK), v_scale(r.v_scale + begin / QN_ADAM_BLOCK),
          octet(static_cast<uint32_t>(r.octet + begin / kOctet)), count(static_cast<int32_t>(count_)) {}
    __device__ __forceinline__ float theta(int i) const { return kMaster ? master[i] : load_rw(param + i); }
    // every array at a multiple of eight of its elements
    __device__ __forceinline__ bool whole_vectors() const {
        const auto off = [](const void* p, uint32_t size) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & (8u * size - 1u); };
        return (off(param, sizeof(P)) | off(grad, sizeof(G)) | (kMaster ? off(master, 4) : 0u) | off(m, sizeof(S)) | off(v, sizeof(S))) == 0;
    }
};

// ---- one element -------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct Element {
    float theta, m, root;
};
// One element with states in 8 bits, whatever it is; m and v: before the step.  The same operations as those of the packed way below,
// so that an element does not depend on which way its neighbours need.  Only here a root may be 0 or so small that what is left, eps in
// units of speed, is below 2^-126, which the reciprocal takes for 0: speed then stays outside (it is above 1, and r spread + eps is
// 2^-126 at least).
__device__ __forceinline__ Element stepped(const Hyper& h, const Common& c, const Rates& rates, float theta, float g, float m, float v) {
    Element e;
    g = __fmul_rn(g, c.coefficient);
    e.m = __fadd_rn(__fmul_rn(m, h.beta1), __fmul_rn(g, h.rest1));
    e.root = __fsqrt_rn(__fadd_rn(__fmul_rn(v, h.beta2), __fmul_rn(__fmul_rn(g, g), h.rest2)));
    const float down = e.root == 0.0f ? -rates.eps : __fmaf_rn(-e.root, rates.spread, -rates.eps);
    const float kept = __fmul_rn(theta, rates.keep);
    if (fabsf(down) < 0x1p-126f) e.theta = __fmaf_rn(__fmul_rn(e.m, rates.speed), rcp_approx(-__fmaf_rn(e.root, c.spread, h.eps)), kept);
    else e.theta = __fmaf_rn(e.m, rcp_approx(down), kept);
    return e;
}

__device__ __forceinline__ uint32_t chance_bits(float x, uint32_t word) {  // the upper 16 bits are the result's
    const uint32_t bits = __float_as_uint(x);
    return x == x ? bits + ((word * kMix2) >> 16) : 0x7fff0000u;
}
// Rounded to nearest, or (kChance) up or down with the probabilities that keep the mean.
template <bool kChance>
__device__ __forceinline__ void store_param(float* p, float x, uint32_t) { *p = x; }
template <bool kChance>
__device__ __forceinline__ void store_param(__nv_bfloat16* p, float x, uint32_t word) {
    *p = kChance ? __ushort_as_bfloat16(static_cast<unsigned short>(chance_bits(x, word) >> 16)) : __float2bfloat16_rn(x);
}

// Element i from memory, with states in 8 bits, whose block had the scales m_scale and v_scale.
template <typename P, typename G, bool kMaster>
__device__ __forceinline__ Element element_at(const Setting& set, const Rates& rates, const Part<P, G, kMaster, uint8_t>& p, int i,
                                              uint32_t m_scale, uint32_t v_scale) {
    const float root = root_value(p.v[i], v_scale);
    return stepped(set.h, set.c, rates, p.theta(i), Storage<G>::load1(p.grad + i), m_value(p.m[i], m_scale), __fmul_rn(root, root));
}

// ---- eight elements, packed ----------------------------------------------------------------------------------------------

// A product that is rounded before it is added to anything: the compiler makes one fused operation of a packed product and a
// packed sum (seen where the two cancel).  This one adds -0, which changes nothing, from an argument, so that the compiler does
// not know it.
__device__ __forceinline__ f32x2 product(f32x2 a, f32x2 b, f32x2 minus_zero) { return fma2(a, b, minus_zero); }

// theta' from m' and -r', two elements.
__device__ __forceinline__ f32x2 moved(const Hyper& h, const Common& c, const Rates& rates, f32x2 theta, f32x2 m, f32x2 minus_r) {
    float d0, d1;
    unpack2(fma2(minus_r, both(c.spread), both(-h.eps)), d0, d1);
    return fma2(mul2(m, both(rates.speed)), pack2(rcp_approx(d0), rcp_approx(d1)), mul2(theta, both(rates.keep)));
}

// States in 32 bits: theta, m and v before and after.
__device__ __forceinline__ void step_pairs(const Hyper& h, const Common& c, const Rates& rates, f32x2 (&theta)[4], f32x2 (&m)[4],
                                           f32x2 (&v)[4], const f32x2 (&grad)[4]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x2 g = mul2(grad[q], both(c.coefficient));
        m[q] = fma2(m[q], both(h.beta1), mul2(g, both(h.rest1)));
        v[q] = fma2(v[q], both(h.beta2), mul2(mul2(g, g), both(h.rest2)));
        float v0, v1, r0, r1;
        unpack2(v[q], v0, v1);
        asm("sqrt.approx.f32 %0, %1;" : "=f"(r0) : "f"(v0));
        asm("sqrt.approx.f32 %0, %1;" : "=f"(r1) : "f"(v1));
        theta[q] = moved(h, c, rates, theta[q], m[q], pack2(-r0, -r1));
    }
}

// max(a, |b|, |c|), NaN if there is one; min(a, |b|, |c|)
__device__ __forceinline__ float largest(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float least(float a, float b, float c) {
    float r;
    asm("min.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The root of a number in [kLow, kHigh] rounded to nearest: s + e / (2 sqrt(v)) with the exact remainder e = v - s^2 (Markstein's
// correction of a root): qn_selftest_roots compares it with the library's root at every one of these numbers.  Numbers come and go
// with their signs changed, which spares the negations.
constexpr float kLow = 0x1p-100f, kHigh = 0x1p30f;
__device__ __forceinline__ f32x2 minus_roots(f32x2 minus_v) {
    float v0, v1, y0, y1;
    unpack2(minus_v, v0, v1);
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y0) : "f"(-v0));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y1) : "f"(-v1));
    const f32x2 y = pack2(y0, y1), s = mul2(minus_v, y);
    return fma2(fma2(s, s, minus_v), mul2(y, both(0.5f)), s);
}

// States in 8 bits: the codes' values become m' and -r'.  They may come without their scales: then keep_m is beta1 times the scale's
// power of two, and keep_v -beta2 times that of r, squared: products with powers of two are exact, so that they may come before the rounding or after it.  (Where
// keep_v underflows, what it stands for is below 2^-126, and below half a step of any v' that stays here; where keep_m may,
// the caller does not come here: see tiny_scale.)  top_m: the largest m'; top_v: the largest v'.  False where this way is not
// the right one: a second moment is 0, or very small, or something is very large or not a number.
__device__ __forceinline__ bool moments(const Hyper& h, const Common& c, f32x2 (&m)[4], f32x2 (&r)[4], const f32x2 (&keep_m)[4],
                                        const f32x2 (&keep_v)[4], const f32x2 (&grad)[4], float& top_m, float& top_v) {
    const f32x2 none = both(h.minus_zero);
    float low_v = INFINITY;
    top_m = top_v = 0.0f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x2 g = mul2(grad[q], both(c.coefficient));
        m[q] = add2(product(m[q], keep_m[q], none), product(g, both(h.rest1), none));
        const f32x2 minus_v = add2(product(mul2(r[q], r[q]), keep_v[q], none), product(mul2(g, g), both(-h.rest2), none));
        float m0, m1, v0, v1;
        unpack2(m[q], m0, m1);
        unpack2(minus_v, v0, v1);
        top_m = largest(top_m, m0, m1);
        top_v = largest(top_v, v0, v1);
        low_v = least(low_v, v0, v1);
        r[q] = minus_roots(minus_v);
    }
    return low_v >= kLow && top_v <= kHigh && top_m <= kHigh;
}
__device__ __forceinline__ float keep_of_m(const Hyper& h, uint32_t scale) { return h.beta1 * power_of(scale); }
__device__ __forceinline__ float keep_of_v(const Hyper& h, uint32_t scale) {
    const float unit = root_unit(scale);
    return unit * unit * -h.beta2;
}
// keep_of_m may not be exact: a small scale, but not that of a block of zeros.  From scale 9 on it is above 2^-126 with a beta1 of 2^-8 and
// more; a smaller one, but for 0, comes with a minus_zero of NaN, so that no element goes the packed way and a step takes several times as
// long.  (Bounds that follow from beta1 cost all others: 2^28 bf16 parameters 557 -> 578 us.)
__device__ __forceinline__ bool tiny_scale(uint32_t scale) { return scale - 1u < 8u; }
float minus_zero_for(float beta1) { return beta1 > 0.0f && beta1 < 0x1p-8f ? NAN : -0.0f; }

// 2^-e / 2^120 (see magnitude_bits; below kHigh this is a number, and one product does for the two there) from the exponent
// field of a block's largest finite magnitude, which is not 0 (m: may be 0).
__device__ __forceinline__ float up_root(uint32_t field) { return power_of(261u - field) * 0x1p-120f; }
__device__ __forceinline__ float up_m(uint32_t field) { return up_root(max(field, 8u)); }
// Of the root, from v.  (The root of the largest v is the largest root, and does not round up to a power of two.)
__device__ __forceinline__ uint32_t root_field(float v) { return ((__float_as_uint(v) >> 23) + 127u) >> 1; }

// Codes of two elements in the upper bytes: (bits + chance) moved up, a half of the chance's step added on the way; m's sign from m.
// `word`: element_word, `upper` its upper half (which its last step does not change).
__device__ __forceinline__ uint32_t m_byte(float z, float m, uint32_t upper) {
    return (((__float_as_uint(z) + upper * 16u) * 16u + 128u) & 0x7fffffffu) | (__float_as_uint(m) & 0x80000000u);
}
__device__ __forceinline__ uint32_t root_byte(float z, uint32_t word) {
    return max(__float_as_uint(z) + (word & 0xffffu) * 8u, (1u << 19) - 4u) * 32u + 128u;
}
__device__ __forceinline__ uint32_t upper_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// theta', codes, and theta' rounded by chance (in the upper halves), of two elements.
template <bool kChance>
struct Coded {
    uint32_t m[2], r[2], theta[2];
    f32x2 theta2;
    // ups: what m and -r are multiplied by
    __device__ __forceinline__ Coded(const Hyper& h, const Common& c, const Rates& rates, f32x2 theta_, f32x2 m_, f32x2 minus_r, f32x2 ups_m,
                                     f32x2 ups_r, const uint32_t (&octets)[2], const uint32_t (&places)[2]) {
        float zm[2], zr[2], m1[2], t[2];
        float d0, d1;
        unpack2(fma2(minus_r, both(rates.spread), both(-rates.eps)), d0, d1);
        theta2 = fma2(m_, pack2(rcp_approx(d0), rcp_approx(d1)), mul2(theta_, both(rates.keep)));
        unpack2(mul2(m_, ups_m), zm[0], zm[1]);
        unpack2(mul2(minus_r, ups_r), zr[0], zr[1]);
        unpack2(m_, m1[0], m1[1]);
        unpack2(theta2, t[0], t[1]);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t y = octets[k] + places[k];
            y = (y ^ (y >> 15)) * kMix3;
            const uint32_t upper = y >> 16;
            y ^= upper;
            m[k] = m_byte(zm[k], m1[k], upper);
            r[k] = root_byte(zr[k], y);
            theta[k] = __float_as_uint(t[k]) + (kChance ? (y * kMix2) >> 16 : 0u);
        }
    }
};

// ---- tensors on vectors ----------------------------------------------------------------------------------------------------

// Eight elements from i on, with states in 32 bits.
template <bool kChance, typename P, typename G, bool kMaster>
__device__ __forceinline__ void step_octet(const Hyper& h, const Common& c, const Rates& rates, const Part<P, G, kMaster, float>& p, int i) {
    const uint32_t word = kChance ? octet_word(c.key, p.octet + i / kOctet) : 0;
    uint32_t graw[sizeof(G) == 4 ? 8 : 4], traw[kMaster || sizeof(P) == 4 ? 8 : 4], mraw[8], vraw[8];
    load8(p.grad + i, graw);
    if constexpr (kMaster) load8(p.master + i, traw);
    else load8(p.param + i, traw);
    load8(p.m + i, mraw);
    load8(p.v + i, vraw);
    f32x2 theta[4], m[4], v[4], g[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) theta[q] = two_of(traw, q), m[q] = two_of(mraw, q), v[q] = two_of(vraw, q), g[q] = two_of(graw, q);
    step_pairs(h, c, rates, theta, m, v, g);
    float t1[8], m1[8], v1[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) unpack2(theta[q], t1[2 * q], t1[2 * q + 1]), unpack2(m[q], m1[2 * q], m1[2 * q + 1]), unpack2(v[q], v1[2 * q], v1[2 * q + 1]);
    store8(p.m + i, m1);
    store8(p.v + i, v1);
    if constexpr (kMaster) store8(p.master + i, t1);
    if constexpr (kChance) {
        uint32_t x[8];
#pragma unroll
        for (int e = 0; e < kOctet; ++e) x[e] = chance_bits(t1[e], element_word(word, e));
        *reinterpret_cast<uint4*>(p.param + i) = make_uint4(__byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632),
                                                            __byte_perm(x[4], x[5], 0x7632), __byte_perm(x[6], x[7], 0x7632));
    } else {
        store8(p.param + i, t1);
    }
}

// Eight elements with states in 8 bits, as they lie in memory.
template <typename P, typename G, bool kMaster>
struct Raw {
    uint32_t theta[kMaster || sizeof(P) == 4 ? 8 : 4], grad[sizeof(G) == 4 ? 8 : 4], m[2], v[2];
    uint32_t m_scale, v_scale;
};

// The way of these elements through shared memory.  What a thread has under way in registers (some 40 bytes of an octet) is a
// third of what it takes to cover the latency of a loaded memory, 2.5 us, so each thread copies its own eight elements of
// the next pieces into slots of its own: asynchronously, and with nobody to wait for but itself.  (Threads of a warp that copy for
// one another, so that each copy is of whole sectors, have to wait for one another: 2^27 fp32 parameters 523 -> 557 us.)
// Slots: four, or three where an element takes so much that CTAs would be lost (two: 579 us).
template <typename P, typename G, bool kMaster>
constexpr int kSlotsOf = (kMaster || sizeof(P) == 4) && sizeof(G) == 4 ? 3 : 4;
template <typename P, typename G, bool kMaster>
struct Slots {
    static constexpr int kSlots = kSlotsOf<P, G, kMaster>;
    static constexpr int kTheta = kMaster || sizeof(P) == 4 ? 2 : 1, kGrad = sizeof(G) == 4 ? 2 : 1;  // units of 16 bytes
    struct Slot {
        uint4 theta[kTheta][kThreads], grad[kGrad][kThreads];
        uint2 m[kThreads], v[kThreads];
    };
    Slot slot[kSlots];

    __device__ static __forceinline__ void copy(uint4* to, const void* from) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
    }
    __device__ static __forceinline__ void copy(uint2* to, const void* from) {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(to)), "l"(from) : "memory");
    }
    // Each call is a group, also if there is nothing to copy.
    __device__ __forceinline__ void fetch(const Part<P, G, kMaster, uint8_t>& p, int s, int i, bool any) {
        const int tid = threadIdx.x;
        Slot& to = slot[s];
        if (any) {
            const char* at = kMaster ? reinterpret_cast<const char*>(p.master + i) : reinterpret_cast<const char*>(p.param + i);
#pragma unroll
            for (int k = 0; k < kTheta; ++k) copy(&to.theta[k][tid], at + 16 * k);
#pragma unroll
            for (int k = 0; k < kGrad; ++k) copy(&to.grad[k][tid], reinterpret_cast<const char*>(p.grad + i) + 16 * k);
            copy(&to.m[tid], p.m + i);
            copy(&to.v[tid], p.v + i);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // All groups but the last kSlots - 2 have arrived.
    __device__ static __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 2) : "memory"); }
    __device__ __forceinline__ void take(int s, Raw<P, G, kMaster>& raw) const {
        const int tid = threadIdx.x;
        const Slot& from = slot[s];
#pragma unroll
        for (int k = 0; k < kTheta; ++k) {
            const uint4 x = from.theta[k][tid];
            raw.theta[4 * k] = x.x, raw.theta[4 * k + 1] = x.y, raw.theta[4 * k + 2] = x.z, raw.theta[4 * k + 3] = x.w;
        }
#pragma unroll
        for (int k = 0; k < kGrad; ++k) {
            const uint4 x = from.grad[k][tid];
            raw.grad[4 * k] = x.x, raw.grad[4 * k + 1] = x.y, raw.grad[4 * k + 2] = x.z, raw.grad[4 * k + 3] = x.w;
        }
        const uint2 a = from.m[tid], b = from.v[tid];
        raw.m[0] = a.x, raw.m[1] = a.y, raw.v[0] = b.x, raw.v[1] = b.y;
    }
};

// For eight elements that are out of the ordinary, from memory again: the bits of the largest finite m' and the exponent field
// of the largest finite r'; and the step.
template <typename P, typename G, bool kMaster>
__device__ __noinline__ uint2 largest_of_any(const Setting* set, const Rates rates, const Part<P, G, kMaster, uint8_t> p, int i, uint32_t m_scale,
                                              uint32_t v_scale) {
    uint2 top = {0, 0};
#pragma unroll 1
    for (int e = i; e < i + kOctet; ++e) {
        const Element x = element_at(*set, rates, p, e, m_scale, v_scale);
        top.x = max(top.x, finite_bits(x.m));
        top.y = max(top.y, finite_bits(x.root) >> 23);
    }
    return top;
}
template <bool kChance, typename P, typename G, bool kMaster>
__device__ __noinline__ void step_any(const Setting* set, const Rates rates, const Part<P, G, kMaster, uint8_t> p, int i, uint32_t m_scale,
                                      uint32_t v_scale, uint32_t ms, uint32_t vs) {
    const uint32_t word = octet_word(set->c.key, p.octet + i / kOctet);
#pragma unroll 1
    for (int e = i; e < i + kOctet; ++e) {
        const uint32_t w = element_word(word, e - i);
        const Element x = element_at(*set, rates, p, e, m_scale, v_scale);
        p.m[e] = static_cast<uint8_t>(m_code(x.m, up_by(ms), w));
        p.v[e] = static_cast<uint8_t>(root_code(x.root, up_by(vs), w));
        if constexpr (kMaster) p.master[e] = x.theta;
        store_param<kChance>(p.param + e, x.theta, w);
    }
}

// 256 elements of a warp from i on, or as many as there are, whatever they are: a block at a time.
template <bool kChance, typename P, typename G, bool kMaster>
__device__ __noinline__ void step_lanes_any(const Setting* set, const Rates rates, const Part<P, G, kMaster, uint8_t> p, int i) {
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int base = i; base < min(i + 256, p.count); base += 32) {
        const int e = base + lane, block = base / QN_ADAM_BLOCK;
        Element x = {0.0f, 0.0f, 0.0f};
        if (e < p.count) {
            const float root = root_value(p.v[e], p.v_scale[block]);
            x = stepped(set->h, set->c, rates, p.theta(e), Storage<G>::load1(p.grad + e), m_value(p.m[e], p.m_scale[block]), __fmul_rn(root, root));
        }
        const uint32_t ms = scale_of(__reduce_max_sync(0xffffffffu, finite_bits(x.m)));
        const uint32_t vs = scale_of(__reduce_max_sync(0xffffffffu, finite_bits(x.root)));
        const uint32_t word = element_word(octet_word(set->c.key, p.octet + e / kOctet), e % kOctet);
        if (e < p.count) {
            p.m[e] = static_cast<uint8_t>(m_code(x.m, up_by(ms), word));
            p.v[e] = static_cast<uint8_t>(root_code(x.root, up_by(vs), word));
            if constexpr (kMaster) p.master[e] = x.theta;
            store_param<kChance>(p.param + e, x.theta, word);
        }
        if (lane == 0) p.m_scale[block] = static_cast<uint8_t>(ms), p.v_scale[block] = static_cast<uint8_t>(vs);
    }
}

// A piece of a tensor that does not lie on vectors, in shared memory.  Numbers in 32 bits are copied word by word, so that there they
// lie on vectors; those in 16 bits too, but for half a word; codes and scales in as many whole units of 16 bytes as it
// takes.  (The tensor has more elements on both sides of the piece.)
template <typename P, typename G, bool kMaster>
struct Window {
    using Theta = typename std::conditional<kMaster, float, P>::type;
    static constexpr int kScales = kPiece / QN_ADAM_BLOCK;
    template <typename X>
    static constexpr int units() { return kPiece * sizeof(X) / 16 + (sizeof(X) == 2); }
    struct Slot {
        uint4 theta[units<Theta>()], grad[units<G>()], m[kPiece / 16 + 1], v[kPiece / 16 + 1], m_scale[kScales / 16 + 1], v_scale[kScales / 16 + 1];
    };
    static constexpr int kSlots = kSlotsOf<P, G, kMaster>;
    Slot slot[kSlots];
    uint4 out[sizeof(P) == 2 ? kThreads : 1];

    __device__ static __forceinline__ uint32_t misplaced(const void* p, uint32_t unit) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) % unit; }
    template <int N>
    __device__ static __forceinline__ void copy_units(uint4 (&to)[N], const uint8_t* from) {
        const uint8_t* at = from - misplaced(from, 16);
        const int units = N - (at == from), j = threadIdx.x;
        static_assert(N <= kThreads, "a unit for a thread");
        if (j < units) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(&to[j])), "l"(at + 16 * j) : "memory");
    }
    template <typename X>
    __device__ static __forceinline__ void copy_words(uint4 (&to)[units<X>()], const X* from) {
        constexpr int kWords = kPiece * sizeof(X) / 4;
        const char* at = reinterpret_cast<const char*>(from) - misplaced(from, 4) + 4 * threadIdx.x;
        const uint32_t into = smem_u32(to) + 4 * threadIdx.x;
#pragma unroll
        for (int k = 0; k < kWords; k += kThreads)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(into + 4 * k), "l"(at + 4 * k) : "memory");
        if (sizeof(X) == 2 && misplaced(from, 4) && threadIdx.x == 0)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(into + 4 * kWords), "l"(at + 4 * kWords) : "memory");
    }
    // By all threads; each call is a group, also if there is nothing to copy.
    __device__ __forceinline__ void fetch(const Part<P, G, kMaster, uint8_t>& p, int s, int i, bool any) {
        if (any) {
            if constexpr (kMaster) copy_words<Theta>(slot[s].theta, p.master + i);
            else copy_words<Theta>(slot[s].theta, p.param + i);
            copy_words<G>(slot[s].grad, p.grad + i);
            copy_units(slot[s].m, p.m + i);
            copy_units(slot[s].v, p.v + i);
            copy_units(slot[s].m_scale, p.m_scale + i / QN_ADAM_BLOCK);
            copy_units(slot[s].v_scale, p.v_scale + i / QN_ADAM_BLOCK);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ static __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 2) : "memory"); }

    // This thread's eight elements.  (`p`: for where its arrays begin within units, which is the same for all pieces.)
    __device__ static __forceinline__ void take8(const uint4* from, const float*, uint32_t (&x)[8]) {
        const uint4 a = from[2 * threadIdx.x], b = from[2 * threadIdx.x + 1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    }
    __device__ static __forceinline__ void take8(const uint4* from, const __nv_bfloat16* at, uint32_t (&x)[4]) {
        const uint4 a = from[threadIdx.x];
        const uint32_t next = from[threadIdx.x + 1].x, shift = 8 * misplaced(at, 4);
        x[0] = __funnelshift_r(a.x, a.y, shift), x[1] = __funnelshift_r(a.y, a.z, shift);
        x[2] = __funnelshift_r(a.z, a.w, shift), x[3] = __funnelshift_r(a.w, next, shift);
    }
    __device__ static __forceinline__ void take8(const uint4* from, const uint8_t* at, uint32_t (&x)[2]) {
        const uint32_t* words = reinterpret_cast<const uint32_t*>(from) + misplaced(at, 16) / 4 + 2 * threadIdx.x;
        const uint32_t a = words[0], b = words[1], c = words[2], shift = 8 * misplaced(at, 4);
        x[0] = __funnelshift_r(a, b, shift), x[1] = __funnelshift_r(b, c, shift);
    }
    __device__ __forceinline__ void take(int s, const Part<P, G, kMaster, uint8_t>& p, Raw<P, G, kMaster>& raw) const {
        const Slot& from = slot[s];
        if constexpr (kMaster) take8(from.theta, p.master, raw.theta);
        else take8(from.theta, p.param, raw.theta);
        take8(from.grad, p.grad, raw.grad);
        take8(from.m, p.m, raw.m);
        take8(from.v, p.v, raw.v);
        const int block = threadIdx.x * kOctet / QN_ADAM_BLOCK;
        raw.m_scale = reinterpret_cast<const uint8_t*>(from.m_scale)[misplaced(p.m_scale, 16) + block];
        raw.v_scale = reinterpret_cast<const uint8_t*>(from.v_scale)[misplaced(p.v_scale, 16) + block];
    }
    // 256 elements of a warp, eight of each thread, to `to`: by way of shared memory, so that the stores of a warp lie together.
    __device__ __forceinline__ void write_f32(int s, float* to, const uint32_t (&x)[8]) {
        const int lane = threadIdx.x % 32;
        uint4* mine = slot[s].theta + 2 * threadIdx.x;  // nobody else has read this
        mine[0] = make_uint4(x[0], x[1], x[2], x[3]);
        mine[1] = make_uint4(x[4], x[5], x[6], x[7]);
        __syncwarp();
        const float* from = reinterpret_cast<const float*>(mine - 2 * lane) + lane;
#pragma unroll
        for (int k = 0; k < 8; ++k) to[32 * k + lane] = from[32 * k];
    }
    __device__ __forceinline__ void write_bf16(__nv_bfloat16* to, uint4 x) {
        const int lane = threadIdx.x % 32;
        const uint32_t off = misplaced(to, 4), before = __shfl_up_sync(0xffffffffu, x.w, 1);
        out[threadIdx.x] = make_uint4(__funnelshift_l(before, x.x, 8 * off), __funnelshift_l(x.x, x.y, 8 * off),
                                      __funnelshift_l(x.y, x.z, 8 * off), __funnelshift_l(x.z, x.w, 8 * off));
        __syncwarp();
        const uint32_t* from = reinterpret_cast<const uint32_t*>(out + (threadIdx.x - lane)) + lane;
        uint32_t* words = reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(to) - off) + lane;
        // the halves of words at both ends by themselves
        if (off && lane == 0) to[0] = __ushort_as_bfloat16(static_cast<unsigned short>(x.x));
        else words[0] = from[0];
#pragma unroll
        for (int k = 1; k < 4; ++k) words[32 * k] = from[32 * k];
        if (off && lane == 31) to[255] = __ushort_as_bfloat16(static_cast<unsigned short>(x.w >> 16));
    }
};
// Eight codes of each thread, at any address: in words, but for what is left of them at both ends of the warp's 256.
__device__ __forceinline__ void write_codes(uint8_t* to, uint2 x) {
    const int lane = threadIdx.x % 32;
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(to)) % 4, before = __shfl_up_sync(0xffffffffu, x.y, 1);
    uint32_t* words = reinterpret_cast<uint32_t*>(to - off);
    if (off == 0 || lane != 0) words[0] = __funnelshift_l(before, x.x, 8 * off);
    words[1] = __funnelshift_l(x.x, x.y, 8 * off);
    if (off != 0) {
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            if (lane == 0 && k + off < 4) to[k] = static_cast<uint8_t>(x.x >> (8 * k));
            if (lane == 31 && k + off >= 4) to[4 + k] = static_cast<uint8_t>(x.y >> (8 * k));
        }
    }
}
// Eight elements from i on; all threads of a warp, four of which have a block.  `window`: if the tensor does not lie on vectors, which
// is what writes it then; elements out of the ordinary send the whole warp the other way.
template <bool kChance, bool kVectors, typename P, typename G, bool kMaster>
__device__ __forceinline__ void step_octet(const Setting* set, const Hyper& h, const Common& c, const Rates& rates,
                                           const Part<P, G, kMaster, uint8_t>& p, int i, const Raw<P, G, kMaster>& raw,
                                           Window<P, G, kMaster>* window, int slot) {
    f32x2 m[4], r[4], g[4];
    float top_m, top_v;
    const f32x2 keep_m = both(keep_of_m(h, raw.m_scale)), keep_v = both(keep_of_v(h, raw.v_scale));
    const f32x2 keeps_m[4] = {keep_m, keep_m, keep_m, keep_m}, keeps_v[4] = {keep_v, keep_v, keep_v, keep_v};
    m_values(raw.m, m);
    root_values(raw.v, r);
#pragma unroll
    for (int q = 0; q < 4; ++q) g[q] = two_of(raw.grad, q);
    bool odd = !moments(h, c, m, r, keeps_m, keeps_v, g, top_m, top_v) || tiny_scale(raw.m_scale);
    uint32_t most_m = __float_as_uint(top_m), field_r = root_field(top_v);
    const int warp_first = i - static_cast<int>(threadIdx.x % 32) * kOctet;
    if (!kVectors && __any_sync(0xffffffffu, odd)) return step_lanes_any<kChance, P, G, kMaster>(set, rates, p, warp_first);
    if (kVectors && odd) {
        const uint2 top = largest_of_any<P, G, kMaster>(set, rates, p, i, raw.m_scale, raw.v_scale);
        most_m = top.x, field_r = top.y;
    }
#pragma unroll
    for (int o = 1; o < 4; o *= 2) {
        most_m = max(most_m, __shfl_xor_sync(0xffffffffu, most_m, o));
        field_r = max(field_r, __shfl_xor_sync(0xffffffffu, field_r, o));
    }
    // another one's element may be too large for this one's way
    if (kVectors) odd = odd || most_m > __float_as_uint(kHigh) || field_r > (__float_as_uint(kHigh) >> 23);
    const uint32_t ms = scale_of(most_m), vs = scale_of(field_r << 23);
    const auto write_scales = [&] {  // all four have read the old ones
        if ((i / kOctet) % 4 != 0) return;
        p.m_scale[i / QN_ADAM_BLOCK] = static_cast<uint8_t>(ms);
        p.v_scale[i / QN_ADAM_BLOCK] = static_cast<uint8_t>(vs);
    };
    if (kVectors) write_scales();
    const f32x2 ups_m = both(up_m(most_m >> 23)), ups_r = both(-up_root(field_r));
    const uint32_t word = octet_word(c.key, p.octet + i / kOctet), octets[2] = {word, word};
    uint32_t a[8], b[8], x[8];
    f32x2 not_finite = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t places[2] = {2 * q * kGolden, (2 * q + 1) * kGolden};
        const Coded<kChance> two(h, c, rates, two_of(raw.theta, q), m[q], r[q], ups_m, ups_r, octets, places);
        if (kChance) not_finite = fma2(two.theta2, 0, not_finite);  // 0, or NaN
#pragma unroll
        for (int k = 0; k < 2; ++k) a[2 * q + k] = two.m[k], b[2 * q + k] = two.r[k], x[2 * q + k] = two.theta[k];
    }
    if (kChance) {
        float n0, n1;
        unpack2(not_finite, n0, n1);
        odd = odd || n0 + n1 != 0.0f;
    }
    const uint2 m_codes = make_uint2(upper_bytes(a[0], a[1], a[2], a[3]), upper_bytes(a[4], a[5], a[6], a[7]));
    const uint2 v_codes = make_uint2(upper_bytes(b[0], b[1], b[2], b[3]), upper_bytes(b[4], b[5], b[6], b[7]));
    if constexpr (!kVectors) {
        if (kChance && __any_sync(0xffffffffu, odd)) return step_lanes_any<kChance, P, G, kMaster>(set, rates, p, warp_first);
        write_scales();
        write_codes(p.m + i, m_codes);
        write_codes(p.v + i, v_codes);
        if constexpr (kMaster || sizeof(P) == 4) window->write_f32(slot, kMaster ? p.master + warp_first : reinterpret_cast<float*>(p.param + warp_first), x);
        if constexpr (sizeof(P) == 2) {
            float t1[8];
#pragma unroll
            for (int e = 0; e < kOctet; ++e) t1[e] = __uint_as_float(x[e]);
            window->write_bf16(p.param + warp_first,
                               kChance ? make_uint4(__byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632),
                                                    __byte_perm(x[4], x[5], 0x7632), __byte_perm(x[6], x[7], 0x7632))
                                       : Storage<__nv_bfloat16>::pack(t1));
        }
        return;
    }
    if (odd) return step_any<kChance, P, G, kMaster>(set, rates, p, i, raw.m_scale, raw.v_scale, ms, vs);
    *reinterpret_cast<uint2*>(p.m + i) = m_codes;
    *reinterpret_cast<uint2*>(p.v + i) = v_codes;
    if constexpr (kChance) {
        *reinterpret_cast<uint4*>(p.param + i) = make_uint4(__byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632),
                                                            __byte_perm(x[4], x[5], 0x7632), __byte_perm(x[6], x[7], 0x7632));
    } else {
        float t1[8];
#pragma unroll
        for (int e = 0; e < kOctet; ++e) t1[e] = __uint_as_float(x[e]);
        if constexpr (kMaster) store8(p.master + i, t1);
        store8(p.param + i, t1);
    }
}

// ---- other tensors -----------------------------------------------------------------------------------------------------------

// 256 elements of a warp, from i on: element i + 32 j + lane is lane's j-th.  States in 32 bits.
template <bool kChance, typename P, typename G, bool kMaster>
__device__ __forceinline__ void step_lanes(const Hyper& h, const Common& c, const Rates& rates, const Part<P, G, kMaster, float>& p, int i) {
    const int lane = threadIdx.x & 31;
    const uint32_t octet = kChance ? octet_word(c.key, p.octet + i / kOctet + lane) : 0;  // of the warp's lane-th eight
    float t[8], m[8], v[8], g[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = i + 32 * j + lane;
        t[j] = m[j] = v[j] = g[j] = 0.0f;
        if (e < p.count) t[j] = p.theta(e), m[j] = p.m[e], v[j] = p.v[e], g[j] = Storage<G>::load1(p.grad + e);
    }
    f32x2 t2[4], m2[4], v2[4], g2[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
        t2[q] = pack2(t[2 * q], t[2 * q + 1]), m2[q] = pack2(m[2 * q], m[2 * q + 1]), v2[q] = pack2(v[2 * q], v[2 * q + 1]), g2[q] = pack2(g[2 * q], g[2 * q + 1]);
    step_pairs(h, c, rates, t2, m2, v2, g2);
#pragma unroll
    for (int q = 0; q < 4; ++q) unpack2(t2[q], t[2 * q], t[2 * q + 1]), unpack2(m2[q], m[2 * q], m[2 * q + 1]), unpack2(v2[q], v[2 * q], v[2 * q + 1]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = i + 32 * j + lane;
        const uint32_t word = kChance ? element_word(__shfl_sync(0xffffffffu, octet, 4 * j + lane / 8), lane % 8) : 0;
        if (e >= p.count) continue;
        p.m[e] = m[j], p.v[e] = v[j];
        if constexpr (kMaster) p.master[e] = t[j];
        store_param<kChance>(p.param + e, t[j], word);
    }
}

// The same with states in 8 bits.
template <bool kChance, typename P, typename G, bool kMaster>
__device__ __forceinline__ void step_lanes(const Setting* set, const Hyper& h, const Common& c, const Rates& rates,
                                           const Part<P, G, kMaster, uint8_t>& p, int i) {
    if (i >= p.count) return;
    const int lane = threadIdx.x & 31, at = i + lane, block = i / QN_ADAM_BLOCK;
    // elements that are not there are ordinary ones that count for nothing and are not written
    const auto here = [&](int j) { return at + 32 * j < p.count; };
    const auto last_block = [&](int b) { return min(b, (p.count - 1) / QN_ADAM_BLOCK); };
    const f32x2 beta1 = both(h.beta1), minus_beta2 = both(-h.beta2);
    const f32x2 keep_m[4] = {beta1, beta1, beta1, beta1}, keep_v[4] = {minus_beta2, minus_beta2, minus_beta2, minus_beta2};
    f32x2 m[4], r[4], g[4];
    float t[8];
    uint32_t codes[8][2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = at + 32 * j;
        codes[j][0] = 0, codes[j][1] = 0x80, t[j] = 0.0f;
        if (here(j)) codes[j][0] = p.m[e], codes[j][1] = p.v[e], t[j] = p.theta(e);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int e = at + 64 * q, b0 = last_block(block + 2 * q), b1 = last_block(block + 2 * q + 1);
        g[q] = pack2(here(2 * q) ? Storage<G>::load1(p.grad + e) : 1.0f, here(2 * q + 1) ? Storage<G>::load1(p.grad + e + 32) : 1.0f);
        m[q] = mul2(m_values(codes[2 * q][0] + codes[2 * q + 1][0] * 256u), pack2(power_of(p.m_scale[b0]), power_of(p.m_scale[b1])));
        r[q] = mul2(root_values(codes[2 * q][1] + codes[2 * q + 1][1] * 65536u), pack2(root_unit(p.v_scale[b0]), root_unit(p.v_scale[b1])));
    }
    float top_m, top_v;
    const bool odd = !moments(h, c, m, r, keep_m, keep_v, g, top_m, top_v);
    if (__any_sync(0xffffffffu, odd)) return step_lanes_any<kChance, P, G, kMaster>(set, rates, p, i);
    const uint32_t octet = octet_word(c.key, p.octet + i / kOctet + lane);  // of the warp's lane-th eight
    const uint32_t place = (lane % 8) * kGolden, places[2] = {place, place};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float m1[2], r1[2], t1[2];
        uint32_t most_m[2], most_r[2], octets[2];
        unpack2(m[q], m1[0], m1[1]);
        unpack2(r[q], r1[0], r1[1]);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            most_m[k] = __reduce_max_sync(0xffffffffu, here(2 * q + k) ? __float_as_uint(m1[k]) & 0x7fffffffu : 0u);
            most_r[k] = __reduce_max_sync(0xffffffffu, here(2 * q + k) ? __float_as_uint(r1[k]) & 0x7fffffffu : 0u);
            octets[k] = __shfl_sync(0xffffffffu, octet, 4 * (2 * q + k) + lane / 8);
        }
        const Coded<kChance> two(h, c, rates, pack2(t[2 * q], t[2 * q + 1]), m[q], r[q], pack2(up_m(most_m[0] >> 23), up_m(most_m[1] >> 23)),
                                 pack2(-up_root(most_r[0] >> 23), -up_root(most_r[1] >> 23)), octets, places);
        unpack2(two.theta2, t1[0], t1[1]);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int e = at + 64 * q + 32 * k;
            if (!here(2 * q + k)) continue;
            p.m[e] = static_cast<uint8_t>(two.m[k] >> 24);
            p.v[e] = static_cast<uint8_t>(two.r[k] >> 24);
            if constexpr (kMaster) p.master[e] = t1[k];
            if constexpr (kChance) {
                const uint32_t x = t1[k] == t1[k] ? two.theta[k] : 0x7fff0000u;
                p.param[e] = P(__ushort_as_bfloat16(static_cast<unsigned short>(x >> 16)));
            } else {
                store_param<false>(p.param + e, t1[k], 0);
            }
            if (lane == 0) {
                p.m_scale[block + 2 * q + k] = static_cast<uint8_t>(scale_of(most_m[k]));
                p.v_scale[block + 2 * q + k] = static_cast<uint8_t>(scale_of(most_r[k]));
            }
        }
    }
}

// ---- the kernel ----------------------------------------------------------------------------------------------------------------

// By one thread of a CTA that has read the step's number: the last to come here counts it, and leaves the ticket as it was.
__device__ __forceinline__ void count_step(int64_t* step, int64_t t, unsigned* ticket) {
    __threadfence();
    if (atomicAdd(ticket, 1u) == gridDim.x - 1) {
        *ticket = 0;
        *step = t;
    }
}

constexpr int64_t kMostPieces = 1 << 19;  // of a run: its elements are counted in 32 bits

template <typename P, typename G, bool kMaster, typename S, bool kChance>
__global__ void __launch_bounds__(kThreads, sizeof(S) == 4 ? 2 : 3) adam_step_kernel(const Tensors all, const Hyper h, int64_t* step, const float* lr,
                                                             const double* sumsq, unsigned* ticket) {
    extern __shared__ __align__(16) unsigned char shared[];
    __shared__ Setting set;
    __shared__ int found;
    // the fewer copies ahead an element leaves room for, the shorter the runs (see Turns)
    constexpr int kTurns = sizeof(S) == 4 ? 32 : kMaster || sizeof(P) == 4 ? 16 : 8;
    const Turns turns(all.pieces, 256 / kTurns, kTurns);
    int64_t lo = turns.lo(turns.count - 1), hi = turns.hi(turns.count - 1);
    start_after_last();
    let_next_start();
    if (hi > lo) find_tensor(all, hi - 1, &found);
    __syncthreads();
    int tensor = found;
    if (hi > lo && all.records[tensor].grad) {
        // the first piece, on its way to L2 while the step's numbers are worked out
        const Record r = all.records[tensor];
        const int64_t i = (hi - 1 - all.first[tensor]) * kPiece + threadIdx.x * kOctet;
        if (i < r.numel) {
            const Part<P, G, kMaster, S> p(r, i, 0);
            const auto warm = [](const void* at) { asm volatile("prefetch.global.L2 [%0];" ::"l"(at)); };
            warm(p.grad), warm(p.m), warm(p.v);
            if constexpr (kMaster) warm(p.master);
            else warm(p.param);
        }
    }
    make_common(h, step, lr, sumsq, set.c);
    if (threadIdx.x == 0) set.h = h;
    __syncthreads();
    const Common c = set.c;
    if (c.skip) return;
    if (threadIdx.x == 0) count_step(step, c.t, ticket);
#pragma unroll 1
    for (int turn = turns.count - 1;;) {
#pragma unroll 1
        for (int64_t piece = hi; piece > lo;) {
            const Record r = all.records[tensor];
            const int64_t first = all.first[tensor], from = max(max(lo, first), piece - kMostPieces), to = piece;
            piece = from;
            if (piece == first) --tensor;
            if (to == from || !r.grad) continue;
            const Rates rates(h, c, r);
            const int64_t begin = (from - first) * kPiece;
            const Part<P, G, kMaster, S> p(r, begin, min(r.numel - begin, (to - from) * kPiece));
            const int last = static_cast<int>(to - from - 1) * kPiece;
            const bool vectors = p.whole_vectors();
            const int mine = static_cast<int>(threadIdx.x / 32) * 256;  // of this warp in a piece
            if constexpr (sizeof(S) == 4) {
                int base = last;
                // element by element, all or what is left of a piece where the tensor ends
#pragma unroll 1
                for (; base >= 0 && (!vectors || base + kPiece > p.count); base -= kPiece) step_lanes<kChance>(h, c, rates, p, base + mine);
#pragma unroll 1
                for (int i = base + static_cast<int>(threadIdx.x) * kOctet; i >= 0; i -= kPiece) step_octet<kChance>(h, c, rates, p, i);
            } else {
                // pieces from `top` down to `low` go through shared memory: whole ones, and off vectors those with more of the tensor on
                // both sides.  The others come first.
                int top = last;
                const int low = !vectors && begin == 0 ? kPiece : 0;
                while (top >= 0 && (vectors ? top + kPiece > p.count : begin + top + kPiece + 16 * QN_ADAM_BLOCK > r.numel)) top -= kPiece;
#pragma unroll 1
                for (int base = last; base >= 0; base -= kPiece) {
                    if (base <= top && base >= low) base = low;
                    else step_lanes<kChance>(&set, h, c, rates, p, base + mine);
                }
                constexpr int kSlots = kSlotsOf<P, G, kMaster>;
                int base = top, slot = 0;
                if (!vectors) {
                    Window<P, G, kMaster>& window = *reinterpret_cast<Window<P, G, kMaster>*>(shared);
#pragma unroll 1
                    for (int k = 0; k < kSlots - 1; ++k) window.fetch(p, k, base - k * kPiece, base - k * kPiece >= low);
#pragma unroll 1
                    for (; base >= low; base -= kPiece) {
                        window.wait();
                        __syncthreads();  // all have their copies, and are through with the slot that is filled next
                        const int ahead = base - (kSlots - 1) * kPiece;
                        window.fetch(p, slot == 0 ? kSlots - 1 : slot - 1, ahead, ahead >= low);
                        Raw<P, G, kMaster> raw;
                        window.take(slot, p, raw);
                        step_octet<kChance, false>(&set, h, c, rates, p, base + static_cast<int>(threadIdx.x) * kOctet, raw, &window, slot);
                        slot = slot == kSlots - 1 ? 0 : slot + 1;
                    }
                } else {
                    Slots<P, G, kMaster>& slots = *reinterpret_cast<Slots<P, G, kMaster>*>(shared);
                    int i = base + static_cast<int>(threadIdx.x) * kOctet;
                    // scales are bytes at any address, and come through registers
                    uint32_t m_scale[kSlots], v_scale[kSlots];
                    const auto fetch = [&](int k, int to) {
                        const int at = i - k * kPiece;
                        slots.fetch(p, to, at, base >= k * kPiece);
                        const int block = max(at, 0) / QN_ADAM_BLOCK;
                        m_scale[to] = p.m_scale[block], v_scale[to] = p.v_scale[block];
                    };
#pragma unroll
                    for (int k = 0; k < kSlots - 1; ++k) fetch(k, k);
#pragma unroll 1
                    while (base >= 0) {
#pragma unroll
                        for (int s = 0; s < kSlots; ++s) {
                            if (base < 0) break;
                            Raw<P, G, kMaster> raw;
                            slots.wait();
                            slots.take(s, raw);
                            raw.m_scale = m_scale[s], raw.v_scale = v_scale[s];
                            fetch(kSlots - 1, s == 0 ? kSlots - 1 : s - 1);
                            step_octet<kChance, true, P, G, kMaster>(&set, h, c, rates, p, i, raw, nullptr, 0);
                            base -= kPiece, i -= kPiece;
                        }
                    }
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                __syncthreads();  // before the slots are filled again
            }
        }
        if (--turn < 0) return;
        lo = turns.lo(turn), hi = turns.hi(turn);
        __syncthreads();
        if (hi > lo) find_tensor(all, hi - 1, &found);
        __syncthreads();
        tensor = found;
    }
}

// How many of the numbers with the bits first to last have another root the packed way.
__global__ void roots_kernel(uint32_t first, uint32_t last, unsigned long long* differ) {
    unsigned count = 0;
    for (uint64_t bits = first + 2ull * (blockIdx.x * blockDim.x + threadIdx.x); bits <= last; bits += 2ull * gridDim.x * blockDim.x) {
        const float v0 = __uint_as_float(static_cast<uint32_t>(bits)), v1 = __uint_as_float(static_cast<uint32_t>(bits) + 1u);
        float r0, r1;
        unpack2(minus_roots(pack2(-v0, -v1)), r0, r1);
        count += __float_as_uint(-r0) != __float_as_uint(__fsqrt_rn(v0));
        count += bits < last && __float_as_uint(-r1) != __float_as_uint(__fsqrt_rn(v1));
    }
    count = __reduce_add_sync(0xffffffffu, count);
    if (threadIdx.x % 32 == 0 && count) atomicAdd(differ, static_cast<unsigned long long>(count));
}

template <typename P, typename G, bool kMaster, bool kChance>
cudaError_t launch_step(const qn_adam_plan& h, const Hyper& hyper, int64_t* step, const float* lr, const double* sumsq, cudaStream_t st) {
    static Resident resident[2];
    constexpr size_t kShared = std::max(sizeof(Slots<P, G, kMaster>), sizeof(Window<P, G, kMaster>));
    return h.eight ? launch_over(adam_step_kernel<P, G, kMaster, uint8_t, kChance>, resident[1], kShared, h, st, hyper, step, lr, sumsq, h.tickets)
                   : launch_over(adam_step_kernel<P, G, kMaster, float, kChance>, resident[0], 0, h, st, hyper, step, lr, sumsq, h.tickets);
}

}  // namespace

extern "C" qn_status qn_adam_step(qn_adam_handle h, int64_t* step, double lr, const float* lr_device, double beta1, double beta2,
                                  double eps, const double* sumsq, double max_norm, double grad_scale, int32_t rounding,
                                  uint64_t seed, void* cuda_stream) {
    if (!h || !step || !check_array(step, 8, h->device) || !check_array(lr_device, 4, h->device) || !check_array(sumsq, 8, h->device))
        return QN_ERR_INVALID;
    if (!lr_device && !(lr >= 0.0 && isfinite(lr))) return QN_ERR_INVALID;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return QN_ERR_INVALID;
    if (!(static_cast<float>(eps) >= 0x1p-126f) || !isfinite(static_cast<float>(eps))) return QN_ERR_INVALID;
    if (max_norm != max_norm || (max_norm > 0.0 && !sumsq) || !isfinite(grad_scale)) return QN_ERR_INVALID;
    if (rounding != QN_ROUND_NEAREST && rounding != QN_ROUND_STOCHASTIC) return QN_ERR_INVALID;
    DeviceGuard guard(h->device);
    if (!guard.ok) return QN_ERR_CUDA;
    const Hyper hyper{lr, log(beta1), log(beta2), max_norm, grad_scale,
                      static_cast<float>(beta1), static_cast<float>(1.0 - beta1), static_cast<float>(beta2), static_cast<float>(1.0 - beta2),
                      static_cast<float>(eps), minus_zero_for(static_cast<float>(beta1)), static_cast<uint32_t>(seed),
                      static_cast<uint32_t>(seed >> 32)};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:adam_step");
    const auto by_grad = [&](auto grad) {
        using G = decltype(grad);
        if (h->param == QN_F32) return launch_step<float, G, false, false>(*h, hyper, step, lr_device, sumsq, st);
        if (h->master) return launch_step<__nv_bfloat16, G, true, false>(*h, hyper, step, lr_device, sumsq, st);
        if (rounding == QN_ROUND_NEAREST) return launch_step<__nv_bfloat16, G, false, false>(*h, hyper, step, lr_device, sumsq, st);
        return launch_step<__nv_bfloat16, G, false, true>(*h, hyper, step, lr_device, sumsq, st);
    };
    const cudaError_t e = h->grad == QN_F32 ? by_grad(float()) : by_grad(__nv_bfloat16());
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}

extern "C" qn_status qn_selftest_roots(int64_t first, int64_t last, int64_t* differ, void* cuda_stream) {
    if (first < 0 || last < first || last >= 0x7f800000 || !differ || reinterpret_cast<uintptr_t>(differ) % 8) return QN_ERR_INVALID;
    int dev = -1;
    if (!device_of(differ, &dev)) return QN_ERR_INVALID;
    DeviceGuard guard(dev);
    if (!guard.ok) return QN_ERR_CUDA;
    roots_kernel<<<4 * qn_sm_count(), kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        static_cast<uint32_t>(first), static_cast<uint32_t>(last), reinterpret_cast<unsigned long long*>(differ));
    return cudaGetLastError() == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
