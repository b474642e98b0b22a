// qn_adam_*: AdamW over the tensors of one parameter vector, with states in 32 bits or in 8, and the gradients' norm.
//
// Per element, with g~ = c g (c: the clip coefficient times grad_scale) and t the number of this step:
//     m' = b1 m + (1 - b1) g~        v' = b2 v + (1 - b2) g~^2        r' = sqrt(v')
//     theta' = theta (1 - lr wd) - lr / (1 - b1^t) m' / (r' / sqrt(1 - b2^t) + eps)
// Nothing is reused, so the floor is the bytes: each array once in and once out.
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
#include <cuda_fp16.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "qn_vocab.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kOctet = 8;  // elements that share a hash
constexpr int kPiece = kThreads * kOctet;  // elements that a CTA has in hand at a time

struct Record {
    int64_t numel, octet;  // octet: the tensor's first place, in units of eight
    void* param;
    const void* grad;
    float* master;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    double decay, lr_scale;
};

// A CTA's share of a turn: `pieces` pieces of a tensor from piece `first` on (fewer where it ends).
struct Chunk {
    int32_t tensor, first;
};

struct Hyper {
    double lr, log_beta1, log_beta2, max_norm, grad_scale;
    float beta1, rest1, beta2, rest2, eps, minus_zero;
    uint32_t seed_low, seed_high;
    int32_t stochastic;
};

// ---- random numbers ------------------------------------------------------------------------------------------------

// A hash of 32 bits by multiplication and shifts.  The multipliers are the fractions of sqrt(3), sqrt(5) and sqrt(6) and of
// the golden ratio, made odd; the means, pairwise correlations and two-dimensional histograms of what comes out were looked at.
constexpr uint32_t kGolden = 0x9E3779B1u, kMix1 = 0xBB67AE85u, kMix2 = 0x3C6EF373u, kMix3 = 0xA54FF53Bu;

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
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
// One for each eight elements, and one for each of them.
__device__ __forceinline__ uint32_t octet_word(uint32_t key, int64_t octet) {
    return mix(static_cast<uint32_t>(octet) * kGolden + key);
}
__device__ __forceinline__ uint32_t element_word(uint32_t octet, uint32_t j) {
    uint32_t y = octet + j * kGolden;
    y = (y ^ (y >> 15)) * kMix3;
    return y ^ (y >> 16);
}

// ---- 8 bits --------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float power_of(uint32_t exponent) { return __uint_as_float(exponent << 23); }

// The scale of a block whose largest finite magnitude has these bits.
__device__ __forceinline__ uint32_t scale_of(uint32_t most) {
    return most == 0 ? 0u : static_cast<uint32_t>(min(max(static_cast<int>(most >> 23) - 7, 1), 247));
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
    return ((magnitude_bits(m, up) + chance) >> 20) | (m < 0.0f ? 0x80u : 0u);
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

// ---- the step ------------------------------------------------------------------------------------------------------

// What is the same for all elements of a step.
struct Common {
    double lr, speed;  // learning rate, and lr / (1 - b1^t)
    float coefficient, spread;  // spread: 1 / sqrt(1 - b2^t)
    uint32_t key;
    bool skip;  // the gradients' norm is not finite
};

__device__ __forceinline__ Common common_of(const Hyper& h, const int64_t* step, const float* lr, const double* sumsq) {
    Common c;
    const int64_t t = *step + 1;
    c.lr = lr ? static_cast<double>(*lr) : h.lr;
    c.speed = c.lr / -expm1(static_cast<double>(t) * h.log_beta1);
    c.spread = static_cast<float>(1.0 / sqrt(-expm1(static_cast<double>(t) * h.log_beta2)));
    double coefficient = h.grad_scale;
    c.skip = false;
    if (sumsq) {
        const double norm = sqrt(*sumsq) * fabs(h.grad_scale);
        c.skip = !isfinite(norm);
        if (h.max_norm > 0.0 && norm > h.max_norm) coefficient *= h.max_norm / norm;
    }
    c.coefficient = static_cast<float>(coefficient);
    c.key = step_key(h.seed_low, h.seed_high, t);
    return c;
}

// The same for all elements of a tensor.
struct Rates {
    float keep, speed;  // 1 - lr wd, lr / (1 - b1^t)
    __device__ __forceinline__ Rates(const Common& c, const Record& r)
        : keep(static_cast<float>(1.0 - c.lr * r.lr_scale * r.decay)), speed(static_cast<float>(c.speed * r.lr_scale)) {}
};

struct Element {
    float theta, m, root;
};
// v: the second moment before the step.
__device__ __forceinline__ Element stepped(const Hyper& h, const Common& c, const Rates& rates, float theta, float g, float m, float& v) {
    Element e;
    g = __fmul_rn(g, c.coefficient);
    e.m = __fadd_rn(__fmul_rn(m, h.beta1), __fmul_rn(g, h.rest1));
    v = __fadd_rn(__fmul_rn(v, h.beta2), __fmul_rn(__fmul_rn(g, g), h.rest2));
    e.root = __fsqrt_rn(v);
    // 2 ulp of the step are far below the rounding of theta
    e.theta = theta * rates.keep - __fdividef(e.m * rates.speed, e.root * c.spread + h.eps);
    return e;
}

__device__ __forceinline__ void store_param(float* p, float x, uint32_t, bool) { *p = x; }
// Rounded to nearest, or up or down with the probabilities that keep the mean.
__device__ __forceinline__ uint32_t chance_bits(float x, uint32_t word) {  // the upper 16 bits are the result's
    const uint32_t bits = __float_as_uint(x);
    return x == x ? bits + ((word * kMix2) >> 16) : 0x7fff0000u;
}
__device__ __forceinline__ void store_param(__nv_bfloat16* p, float x, uint32_t word, bool stochastic) {
    *p = stochastic ? __ushort_as_bfloat16(static_cast<unsigned short>(chance_bits(x, word) >> 16)) : __float2bfloat16_rn(x);
}

// ---- eight elements of a thread ----------------------------------------------------------------------------------------

// In place arrays are read with ordinary loads: the same thread writes them back.
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    asm volatile("ld.global.L1::no_allocate.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = Storage<__nv_bfloat16>::get(v, e);
}
__device__ __forceinline__ uint2 load8(const uint8_t* p) {
    uint2 v;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]),
                 "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = Storage<__nv_bfloat16>::pack(x);
}

// Eight codes of m, or of a root, and back.
__device__ __forceinline__ void m_values(uint2 codes, uint32_t scale, float (&m)[8]) {
    const float unit = power_of(scale);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t two = (q < 2 ? codes.x : codes.y) >> (16 * (q & 1));
        uint32_t halves;
        asm("{\n .reg .b16 lo;\n cvt.u16.u32 lo, %1;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n}" : "=r"(halves) : "r"(two));
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&halves));
        m[2 * q] = x.x * unit;
        m[2 * q + 1] = x.y * unit;
    }
}
// A half has the same kind of fraction with five bits of exponent: a code moved up by 6 is one, 2^8 too small.
__device__ __forceinline__ void root_values(uint2 codes, uint32_t scale, float (&r)[8]) {
    const float unit = scale ? power_of(min(scale + 8u, 254u)) : 0.0f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t word = q < 2 ? codes.x : codes.y;
        const uint32_t halves = __byte_perm(word, 0, q & 1 ? 0x3424 : 0x1404) >> 2;
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&halves));
        r[2 * q] = x.x * unit;
        r[2 * q + 1] = x.y * unit;
    }
}

template <bool k8>
struct Octet {
    float theta[8], m[8], v[8];  // v: r with states in 8 bits
};

__device__ __forceinline__ f32x2 both(float x) { return pack2(x, x); }
// A product that is rounded before it is added to anything: the compiler makes one fused operation of a packed product and a
// packed sum (seen where the two cancel).  This one adds -0, which changes nothing, from an argument, so that the compiler does not know it.
__device__ __forceinline__ f32x2 product(f32x2 a, f32x2 b, f32x2 minus_zero) { return fma2(a, b, minus_zero); }

template <bool k8>
__device__ __forceinline__ void step_octet(const Hyper& h, const Common& c, const Rates& rates, Octet<k8>& o, const float (&grad)[8]) {
    const f32x2 coefficient = both(c.coefficient), beta1 = both(h.beta1), rest1 = both(h.rest1), beta2 = both(h.beta2),
                rest2 = both(h.rest2), keep = both(rates.keep), speed = both(-rates.speed), spread = both(c.spread), eps = both(h.eps);
    const f32x2 none = both(h.minus_zero);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x2 g = mul2(pack2(grad[2 * q], grad[2 * q + 1]), coefficient);
        const f32x2 m = add2(product(pack2(o.m[2 * q], o.m[2 * q + 1]), beta1, none), product(g, rest1, none));
        f32x2 v = pack2(o.v[2 * q], o.v[2 * q + 1]);
        if (k8) v = mul2(v, v);
        v = add2(product(v, beta2, none), product(mul2(g, g), rest2, none));
        float v0, v1, r0, r1, i0, i1;
        unpack2(v, v0, v1);
        if (k8) {
            r0 = __fsqrt_rn(v0), r1 = __fsqrt_rn(v1);
            o.v[2 * q] = r0, o.v[2 * q + 1] = r1;
        } else {
            asm("sqrt.approx.f32 %0, %1;" : "=f"(r0) : "f"(v0));
            asm("sqrt.approx.f32 %0, %1;" : "=f"(r1) : "f"(v1));
            o.v[2 * q] = v0, o.v[2 * q + 1] = v1;
        }
        unpack2(fma2(pack2(r0, r1), spread, eps), i0, i1);
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(i0) : "f"(i0));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(i1) : "f"(i1));
        const f32x2 theta = fma2(mul2(m, speed), pack2(i0, i1), mul2(pack2(o.theta[2 * q], o.theta[2 * q + 1]), keep));
        unpack2(m, o.m[2 * q], o.m[2 * q + 1]);
        unpack2(theta, o.theta[2 * q], o.theta[2 * q + 1]);
    }
}

// The largest magnitude of eight; NaN if there is one.
__device__ __forceinline__ float largest(const float (&x)[8]) {
    float a = fabsf(x[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) a = max_nan(a, fabsf(x[e]));
    return a;
}
__device__ __noinline__ float largest_finite(float a, float b) {
    return fmaxf(__uint_as_float(finite_bits(a)), __uint_as_float(finite_bits(b)));
}
// Of a block: four threads with eight elements each.
__device__ __forceinline__ uint32_t block_scale(float mine) {
    uint32_t bits = __float_as_uint(mine);
    bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 1));
    bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 2));
    return scale_of(bits);
}
__device__ __forceinline__ uint32_t pack_bytes(const uint32_t* x) {
    return __byte_perm(__byte_perm(x[0], x[1], 0x0040), __byte_perm(x[2], x[3], 0x0040), 0x5410);
}

// The last CTA to come here counts the step and leaves the ticket as it was.
__device__ __forceinline__ void count_step(int64_t* step, unsigned* ticket) {
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(ticket, 1u) == gridDim.x - 1) {
            *ticket = 0;
            *step += 1;
        }
    }
}

// Every array of the tensor lies at a multiple of eight of its elements.
template <typename P, typename G, bool kMaster, bool k8>
__device__ __forceinline__ bool whole_vectors(const Record& r) {
    const auto off = [](const void* p, uint32_t size) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & (8u * size - 1u); };
    return (off(r.param, sizeof(P)) | off(r.grad, sizeof(G)) | (kMaster ? off(r.master, 4) : 0u) | off(r.m, k8 ? 1 : 4) | off(r.v, k8 ? 1 : 4)) == 0;
}

// Eight elements from i on (fewer where the tensor ends), of a tensor whose arrays are aligned; all threads of a warp.
template <typename P, typename G, bool kMaster, bool k8>
__device__ __forceinline__ void step_vector(const Hyper& h, const Common& c, const Rates& rates, const Record& r, int64_t i, bool stochastic) {
    const int here = static_cast<int>(max(min(r.numel - i, static_cast<int64_t>(kOctet)), static_cast<int64_t>(0)));
    Octet<k8> o;
    float g[8];
    uint2 mc = {0, 0}, vc = {0, 0};
    uint32_t ms = 0, vs = 0;
    if (here == kOctet) {
        load8(static_cast<const G*>(r.grad) + i, g);
        if constexpr (kMaster) load8(r.master + i, o.theta);
        else load8(static_cast<const P*>(r.param) + i, o.theta);
        if constexpr (k8) {
            mc = load8(static_cast<const uint8_t*>(r.m) + i), vc = load8(static_cast<const uint8_t*>(r.v) + i);
        } else {
            load8(static_cast<const float*>(r.m) + i, o.m);
            load8(static_cast<const float*>(r.v) + i, o.v);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kOctet; ++e) {
            g[e] = o.theta[e] = 0.0f;
            if constexpr (!k8) o.m[e] = o.v[e] = 0.0f;
            if (e >= here) continue;
            g[e] = Storage<G>::load1(static_cast<const G*>(r.grad) + i + e);
            o.theta[e] = kMaster ? r.master[i + e] : load_rw(static_cast<const P*>(r.param) + i + e);
            if constexpr (k8) {
                const uint32_t a = static_cast<const uint8_t*>(r.m)[i + e], b = static_cast<const uint8_t*>(r.v)[i + e];
                (e < 4 ? mc.x : mc.y) |= a << (8 * (e & 3));
                (e < 4 ? vc.x : vc.y) |= b << (8 * (e & 3));
            } else {
                o.m[e] = static_cast<const float*>(r.m)[i + e];
                o.v[e] = static_cast<const float*>(r.v)[i + e];
            }
        }
    }
    if constexpr (k8) {
        if (here) ms = r.m_scale[i / QN_ADAM_BLOCK], vs = r.v_scale[i / QN_ADAM_BLOCK];
        m_values(mc, ms, o.m);
        root_values(vc, vs, o.v);
    }
    step_octet<k8>(h, c, rates, o, g);
    const uint32_t word = k8 || stochastic ? octet_word(c.key, r.octet + i / kOctet) : 0;
    if constexpr (k8) {
        float top_m = largest(o.m), top_r = largest(o.v);
        const bool odd = !(top_m < INFINITY) || !(top_r < INFINITY);  // something is not finite
        if (odd) {
            top_m = top_r = 0.0f;
#pragma unroll
            for (int e = 0; e < kOctet; ++e) top_m = largest_finite(top_m, o.m[e]), top_r = largest_finite(top_r, o.v[e]);
        }
        ms = block_scale(top_m);
        vs = block_scale(top_r);
        const float up_m = up_by(ms), up_r = up_by(vs);
        uint32_t a[8], b[8];
#pragma unroll
        for (int e = 0; e < kOctet; ++e) {
            const uint32_t w = element_word(word, e);
            a[e] = ((magnitude_bits(o.m[e], up_m) + (((w >> 12) & 0xffff0u) | 8u)) >> 20) | (o.m[e] < 0.0f ? 0x80u : 0u);
            b[e] = max((magnitude_bits(o.v[e], up_r) + (((w << 3) & 0x7fff8u) | 4u)) >> 19, min(__float_as_uint(o.v[e]), 1u));
        }
        if (odd) {
#pragma unroll
            for (int e = 0; e < kOctet; ++e) {
                const uint32_t w = element_word(word, e);
                a[e] = m_code(o.m[e], up_m, w), b[e] = root_code(o.v[e], up_r, w);
            }
        }
        mc = make_uint2(pack_bytes(a), pack_bytes(a + 4));
        vc = make_uint2(pack_bytes(b), pack_bytes(b + 4));
        if (here && (i / kOctet) % 4 == 0) {
            r.m_scale[i / QN_ADAM_BLOCK] = static_cast<uint8_t>(ms);
            r.v_scale[i / QN_ADAM_BLOCK] = static_cast<uint8_t>(vs);
        }
    }
    if (here == kOctet) {
        if constexpr (k8) {
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(r.m) + i) = mc;
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(r.v) + i) = vc;
        } else {
            store8(static_cast<float*>(r.m) + i, o.m);
            store8(static_cast<float*>(r.v) + i, o.v);
        }
        if constexpr (kMaster) store8(r.master + i, o.theta);
        if constexpr (sizeof(P) == 2) {
            if (stochastic) {
                uint32_t x[8];
#pragma unroll
                for (int e = 0; e < kOctet; ++e) x[e] = chance_bits(o.theta[e], element_word(word, e));
                *reinterpret_cast<uint4*>(static_cast<P*>(r.param) + i) =
                    make_uint4(__byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632), __byte_perm(x[4], x[5], 0x7632), __byte_perm(x[6], x[7], 0x7632));
                return;
            }
        }
        store8(static_cast<P*>(r.param) + i, o.theta);
        return;
    }
#pragma unroll
    for (int e = 0; e < kOctet; ++e) {
        if (e >= here) continue;
        if constexpr (k8) {
            static_cast<uint8_t*>(r.m)[i + e] = static_cast<uint8_t>((e < 4 ? mc.x : mc.y) >> (8 * (e & 3)));
            static_cast<uint8_t*>(r.v)[i + e] = static_cast<uint8_t>((e < 4 ? vc.x : vc.y) >> (8 * (e & 3)));
        } else {
            static_cast<float*>(r.m)[i + e] = o.m[e];
            static_cast<float*>(r.v)[i + e] = o.v[e];
        }
        if constexpr (kMaster) r.master[i + e] = o.theta[e];
        store_param(static_cast<P*>(r.param) + i + e, o.theta[e], element_word(word, e), stochastic);
    }
}

template <typename P, typename G, bool kMaster, bool k8>
__global__ void __launch_bounds__(kThreads) adam_step_kernel(const Record* records, const Chunk* chunks, int count, int pieces,
                                                             const Hyper h, int64_t* step, const float* lr,
                                                             const double* sumsq, unsigned* ticket) {
    __shared__ Common shared;
    if (threadIdx.x == 0) shared = common_of(h, step, lr, sumsq);
    __syncthreads();
    const Common c = shared;
    if (c.skip) return;
    const bool stochastic = h.stochastic && !kMaster && sizeof(P) == 2;
    for (int at = count - 1 - static_cast<int>(blockIdx.x); at >= 0; at -= gridDim.x) {
        const Chunk chunk = chunks[at];
        const Record r = records[chunk.tensor];
        if (!r.grad) continue;
        const Rates rates(c, r);
        const int64_t begin = static_cast<int64_t>(chunk.first) * kPiece;
        const int64_t end = min(r.numel, begin + static_cast<int64_t>(pieces) * kPiece);
        if (whole_vectors<P, G, kMaster, k8>(r)) {  // eight elements a thread
            for (int64_t base = begin; base < end; base += kPiece) {
                const int64_t i = base + threadIdx.x * kOctet;
                step_vector<P, G, kMaster, k8>(h, c, rates, r, i, stochastic);
            }
            continue;
        }
        // an element a lane: a warp has one block of 32
        for (int64_t base = begin + (threadIdx.x & ~31u); base < end; base += kThreads) {
            const int64_t i = base + (threadIdx.x & 31);
            const bool here = i < end;
            const uint32_t word = k8 || stochastic ? element_word(octet_word(c.key, r.octet + i / kOctet), i % kOctet) : 0;
            float theta = 0.0f, g = 0.0f, m = 0.0f, v = 0.0f;
            if (here) {
                theta = kMaster ? r.master[i] : load_rw(static_cast<const P*>(r.param) + i);
                g = Storage<G>::load1(static_cast<const G*>(r.grad) + i);
                if constexpr (k8) {
                    m = m_value(static_cast<const uint8_t*>(r.m)[i], r.m_scale[base / QN_ADAM_BLOCK]);
                    v = root_value(static_cast<const uint8_t*>(r.v)[i], r.v_scale[base / QN_ADAM_BLOCK]);
                    v = __fmul_rn(v, v);
                } else {
                    m = static_cast<const float*>(r.m)[i];
                    v = static_cast<const float*>(r.v)[i];
                }
            }
            const Element e = stepped(h, c, rates, theta, g, m, v);
            if constexpr (k8) {
                const uint32_t ms = scale_of(__reduce_max_sync(0xffffffffu, here ? finite_bits(e.m) : 0u));
                const uint32_t vs = scale_of(__reduce_max_sync(0xffffffffu, here ? finite_bits(e.root) : 0u));
                if (here) {
                    static_cast<uint8_t*>(r.m)[i] = static_cast<uint8_t>(m_code(e.m, up_by(ms), word));
                    static_cast<uint8_t*>(r.v)[i] = static_cast<uint8_t>(root_code(e.root, up_by(vs), word));
                    if ((threadIdx.x & 31) == 0) {
                        r.m_scale[base / QN_ADAM_BLOCK] = static_cast<uint8_t>(ms);
                        r.v_scale[base / QN_ADAM_BLOCK] = static_cast<uint8_t>(vs);
                    }
                }
            } else if (here) {
                static_cast<float*>(r.m)[i] = e.m;
                static_cast<float*>(r.v)[i] = v;
            }
            if (here) {
                if constexpr (kMaster) r.master[i] = e.theta;
                store_param(static_cast<P*>(r.param) + i, e.theta, word, stochastic);
            }
        }
    }
    count_step(step, ticket);
}

// ---- the norm ------------------------------------------------------------------------------------------------------

// Sum of squares in 64 bits: each CTA's in a fixed order, and the CTAs' sums in theirs, by the last one to come.
template <typename G>
__global__ void __launch_bounds__(kThreads) adam_norm_kernel(const Record* records, const Chunk* chunks, int count, int pieces,
                                                             double* partials, unsigned* ticket, double* sumsq) {
    __shared__ double scratch[kThreads / 32];
    __shared__ bool last;
    double sum = 0.0;
    for (int at = blockIdx.x; at < count; at += gridDim.x) {
        const Chunk chunk = chunks[at];
        const int64_t numel = records[chunk.tensor].numel;
        const G* grad = static_cast<const G*>(records[chunk.tensor].grad);
        if (!grad) continue;
        const int64_t begin = static_cast<int64_t>(chunk.first) * kPiece;
        const int64_t end = min(numel, begin + static_cast<int64_t>(pieces) * kPiece);
        int64_t i = begin + threadIdx.x;
        if (reinterpret_cast<uintptr_t>(grad) % (kOctet * sizeof(G)) == 0) {  // eight elements a thread
#pragma unroll 4
            for (int64_t at8 = begin + threadIdx.x * kOctet; at8 + kOctet <= end; at8 += kPiece) {
                float g[kOctet];
                load8(grad + at8, g);
#pragma unroll
                for (int e = 0; e < kOctet; ++e) sum += static_cast<double>(g[e]) * g[e];
            }
            i = end - (end - begin) % kOctet + threadIdx.x;
        }
#pragma unroll 1
        for (; i < end; i += kThreads) {
            const double g = Storage<G>::load1(grad + i);
            sum += g * g;
        }
    }
    sum = block_reduce<double, add_op>(sum, scratch);
    if (threadIdx.x == 0) {
        partials[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kThreads) sum += __ldcg(partials + i);
    sum = block_reduce<double, add_op>(sum, scratch);
    if (threadIdx.x == 0) {
        *ticket = 0;
        *sumsq = sum;
    }
}

// ---- what codes stand for -------------------------------------------------------------------------------------------

__device__ __forceinline__ void store_value(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_value(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <typename T, bool k8>
__global__ void __launch_bounds__(kThreads) adam_state_kernel(const Record* records, const Chunk* chunks, int count, int pieces, T* m_out, T* root_out) {
    for (int at = blockIdx.x; at < count; at += gridDim.x) {
        const Chunk chunk = chunks[at];
        const Record r = records[chunk.tensor];
        const int64_t begin = static_cast<int64_t>(chunk.first) * kPiece;
        const int64_t whole = (r.numel + QN_ADAM_BLOCK - 1) / QN_ADAM_BLOCK * QN_ADAM_BLOCK;
        const int64_t end = min(whole, begin + static_cast<int64_t>(pieces) * kPiece);
        int64_t i = begin + threadIdx.x;
        T *m_to = m_out ? m_out + r.octet * kOctet : nullptr, *root_to = root_out ? root_out + r.octet * kOctet : nullptr;
        const uintptr_t places = (reinterpret_cast<uintptr_t>(m_out) | reinterpret_cast<uintptr_t>(root_out)) % (kOctet * sizeof(T));
        if (places == 0 && (reinterpret_cast<uintptr_t>(r.m) | reinterpret_cast<uintptr_t>(r.v)) % (kOctet * (k8 ? 1 : 4)) == 0) {
            const int64_t full = min(end, r.numel / kOctet * kOctet);
#pragma unroll 2
            for (int64_t a = begin + threadIdx.x * kOctet; a < full; a += kPiece) {
                float m[8], root[8];
                if constexpr (k8) {
                    m_values(load8(static_cast<const uint8_t*>(r.m) + a), r.m_scale[a / QN_ADAM_BLOCK], m);
                    root_values(load8(static_cast<const uint8_t*>(r.v) + a), r.v_scale[a / QN_ADAM_BLOCK], root);
                } else {
                    load8(static_cast<const float*>(r.m) + a, m);
                    load8(static_cast<const float*>(r.v) + a, root);
#pragma unroll
                    for (int e = 0; e < 8; ++e) root[e] = __fsqrt_rn(root[e]);
                }
                if (m_to) store8(m_to + a, m);
                if (root_to) store8(root_to + a, root);
            }
            i = max(begin, full) + threadIdx.x;
        }
#pragma unroll 1
        for (; i < end; i += kThreads) {
            float m = 0.0f, root = 0.0f;
            if (i < r.numel) {
                if constexpr (k8) {
                    m = m_value(static_cast<const uint8_t*>(r.m)[i], r.m_scale[i / QN_ADAM_BLOCK]);
                    root = root_value(static_cast<const uint8_t*>(r.v)[i], r.v_scale[i / QN_ADAM_BLOCK]);
                } else {
                    m = static_cast<const float*>(r.m)[i];
                    root = __fsqrt_rn(static_cast<const float*>(r.v)[i]);
                }
            }
            if (m_to) store_value(m_to + i, m);
            if (root_to) store_value(root_to + i, root);
        }
    }
}

// ---- other gradients -------------------------------------------------------------------------------------------------

constexpr int kPointers = 256;
struct Pointers {
    const void* at[kPointers];
};
__global__ void adam_grads_kernel(Record* records, const __grid_constant__ Pointers p, int first, int count) {
    const int i = threadIdx.x;
    if (i < count) records[first + i].grad = p.at[i];
}

}  // namespace

struct qn_adam_plan {
    int device = -1;
    int32_t count = 0;
    qn_dtype param = QN_F32, grad = QN_F32;
    bool master = false, eight = false;
    int64_t places = 0;
    int32_t chunks = 0, pieces = 1, most_ctas = 1;
    void* block = nullptr;  // device memory: records, chunks, partial sums, tickets
    Record* records = nullptr;
    Chunk* chunk = nullptr;
    double* partials = nullptr;
    unsigned* tickets = nullptr;  // of the step, of the norm
    std::vector<int64_t> numel;
    std::vector<std::pair<uintptr_t, uintptr_t>> written;  // in order
};

namespace {

constexpr int kMostCtas = 8;  // on an SM

bool add_range(std::vector<std::pair<uintptr_t, uintptr_t>>& ranges, const void* p, size_t bytes, size_t align, int dev) {
    if (!p || !check_array(p, align, dev)) return false;
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    ranges.emplace_back(at, at + bytes);
    return true;
}

// A gradient is read only: it may lie anywhere but in what a step writes.
bool check_grad(const qn_adam_plan& h, const void* p, int64_t numel) {
    const size_t size = dtype_size(h.grad);
    if (!check_array(p, size, h.device)) return false;
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p), hi = lo + numel * size;
    const auto next = std::upper_bound(h.written.begin(), h.written.end(), std::make_pair(lo, ~uintptr_t(0)));
    if (next != h.written.end() && next->first < hi) return false;
    return next == h.written.begin() || (next - 1)->second <= lo;
}

// As many CTAs as are on the device at once (asked for once), or one for each chunk.
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), int& resident, const qn_adam_plan& h, cudaStream_t st, A... args) {
    if (resident == 0) {
        int found = 0;
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&found, kernel, kThreads, 0);
        if (e != cudaSuccess) return e;
        resident = std::max(1, std::min(found, kMostCtas));
    }
    kernel<<<std::max(1, std::min(h.chunks, resident * qn_sm_count())), kThreads, 0, st>>>(args...);
    return cudaGetLastError();
}

qn_status create(int32_t count, const qn_adam_tensor* tensors, qn_dtype param, qn_dtype grad, int32_t state, qn_adam_handle* out) {
    qn_adam_plan h;
    h.count = count;
    h.param = param;
    h.grad = grad;
    h.eight = state == QN_STATE_8BIT;
    std::vector<Record> records(count);
    int64_t pieces = 0;
    bool first = true;
    for (int32_t i = 0; i < count; ++i) {
        const qn_adam_tensor& t = tensors[i];
        if (t.numel < 0 || t.numel > (int64_t(1) << 40) || h.places > (int64_t(1) << 50)) return QN_ERR_INVALID;
        if (!(t.weight_decay >= 0.0) || !(t.lr_scale >= 0.0) || !isfinite(t.weight_decay) || !isfinite(t.lr_scale))
            return QN_ERR_INVALID;
        Record& r = records[i];
        r = Record{t.numel, h.places / kOctet, t.param, t.grad, t.master, t.m, t.v, t.m_scale, t.v_scale, t.weight_decay, t.lr_scale};
        h.numel.push_back(t.numel);
        if (t.numel == 0) continue;
        const int64_t blocks = (t.numel + QN_ADAM_BLOCK - 1) / QN_ADAM_BLOCK;
        if (first) {
            if (!t.param || !device_of(t.param, &h.device)) return QN_ERR_INVALID;
            h.master = t.master != nullptr;
            if (h.master && param != QN_BF16) return QN_ERR_INVALID;
            first = false;
        }
        if (h.master != (t.master != nullptr) || h.eight != (t.m_scale != nullptr) || h.eight != (t.v_scale != nullptr))
            return QN_ERR_INVALID;
        const size_t each = h.eight ? 1 : 4;
        if (!add_range(h.written, t.param, t.numel * dtype_size(param), dtype_size(param), h.device) ||
            (h.master && !add_range(h.written, t.master, t.numel * 4, 4, h.device)) ||
            !add_range(h.written, t.m, t.numel * each, each, h.device) ||
            !add_range(h.written, t.v, t.numel * each, each, h.device) ||
            (h.eight && (!add_range(h.written, t.m_scale, blocks, 1, h.device) ||
                         !add_range(h.written, t.v_scale, blocks, 1, h.device))))
            return QN_ERR_INVALID;
        h.places += blocks * QN_ADAM_BLOCK;
        pieces += (t.numel + kPiece - 1) / kPiece;
    }
    std::sort(h.written.begin(), h.written.end());
    for (size_t i = 1; i < h.written.size(); ++i)
        if (h.written[i].first < h.written[i - 1].second) return QN_ERR_INVALID;
    for (int32_t i = 0; i < count; ++i)
        if (records[i].numel && records[i].grad && !check_grad(h, records[i].grad, records[i].numel)) return QN_ERR_INVALID;
    if (h.device < 0 && cudaGetDevice(&h.device) != cudaSuccess) return QN_ERR_CUDA;
    DeviceGuard guard(h.device);
    if (!guard.ok) return QN_ERR_CUDA;
    h.most_ctas = kMostCtas * qn_sm_count();
    h.pieces = pieces > 4 * static_cast<int64_t>(h.most_ctas) ? 4 : 1;
    std::vector<Chunk> chunks;
    for (int32_t i = 0; i < count; ++i) {
        const int64_t all = (records[i].numel + kPiece - 1) / kPiece;
        if (all > INT32_MAX - 8) return QN_ERR_INVALID;
        for (int64_t p = 0; p < all; p += h.pieces) chunks.push_back(Chunk{i, static_cast<int32_t>(p)});
    }
    if (chunks.size() > static_cast<size_t>(INT32_MAX / 2)) return QN_ERR_INVALID;
    h.chunks = static_cast<int32_t>(chunks.size());
    const size_t record_bytes = count * sizeof(Record), chunk_bytes = chunks.size() * sizeof(Chunk);
    const size_t partial_bytes = h.most_ctas * sizeof(double);
    if (cudaMalloc(&h.block, record_bytes + chunk_bytes + partial_bytes + 64) != cudaSuccess) {
        cudaGetLastError();
        return QN_ERR_ALLOC;
    }
    char* at = static_cast<char*>(h.block);
    h.records = reinterpret_cast<Record*>(at);
    h.partials = reinterpret_cast<double*>(at += record_bytes);
    h.chunk = reinterpret_cast<Chunk*>(at += partial_bytes);
    h.tickets = reinterpret_cast<unsigned*>(at += chunk_bytes);
    // blocking copies from this call's own memory: nothing is left to do when it returns
    if ((record_bytes && cudaMemcpy(h.records, records.data(), record_bytes, cudaMemcpyHostToDevice) != cudaSuccess) ||
        (chunk_bytes && cudaMemcpy(h.chunk, chunks.data(), chunk_bytes, cudaMemcpyHostToDevice) != cudaSuccess) ||
        cudaMemset(h.tickets, 0, 64) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
        cudaGetLastError();
        cudaFree(h.block);
        return QN_ERR_CUDA;
    }
    *out = new (std::nothrow) qn_adam_plan(std::move(h));
    if (!*out) {
        cudaFree(h.block);
        return QN_ERR_ALLOC;
    }
    return QN_OK;
}

template <typename P, typename G, bool kMaster>
cudaError_t launch_step(const qn_adam_plan& h, const Hyper& hyper, int64_t* step, const float* lr, const double* sumsq, cudaStream_t st) {
    static int resident[2];
    const auto run = [&](auto kernel, int& r) {
        return launch(kernel, r, h, st, static_cast<const Record*>(h.records), static_cast<const Chunk*>(h.chunk), h.chunks, h.pieces, hyper, step, lr, sumsq, h.tickets);
    };
    return h.eight ? run(adam_step_kernel<P, G, kMaster, true>, resident[1]) : run(adam_step_kernel<P, G, kMaster, false>, resident[0]);
}

}  // namespace

extern "C" qn_status qn_adam_create(int32_t count, const qn_adam_tensor* tensors, qn_dtype param, qn_dtype grad, int32_t state,
                                    qn_adam_handle* out) {
    if (!out) return QN_ERR_INVALID;
    *out = nullptr;
    if (count < 0 || count > (1 << 24) || (count && !tensors)) return QN_ERR_INVALID;
    if ((param != QN_F32 && param != QN_BF16) || (grad != QN_F32 && grad != QN_BF16)) return QN_ERR_INVALID;
    if (state != QN_STATE_F32 && state != QN_STATE_8BIT) return QN_ERR_INVALID;
    try {
        return create(count, tensors, param, grad, state, out);
    } catch (...) {  // host memory
        return QN_ERR_ALLOC;
    }
}

extern "C" qn_status qn_adam_destroy(qn_adam_handle h) {
    if (!h) return QN_ERR_INVALID;
    {
        DeviceGuard guard(h->device);
        cudaFree(h->block);  // waits for what uses it
    }
    delete h;
    return QN_OK;
}

extern "C" int64_t qn_adam_places(qn_adam_handle h) { return h ? h->places : 0; }

extern "C" qn_status qn_adam_grads(qn_adam_handle h, const void* const* grads, void* cuda_stream) {
    if (!h || (h->count && !grads)) return QN_ERR_INVALID;
    for (int32_t i = 0; i < h->count; ++i)
        if (h->numel[i] && grads[i] && !check_grad(*h, grads[i], h->numel[i])) return QN_ERR_INVALID;
    DeviceGuard guard(h->device);
    if (!guard.ok) return QN_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    for (int32_t first = 0; first < h->count; first += kPointers) {
        Pointers p;
        const int here = std::min(kPointers, h->count - first);
        for (int i = 0; i < kPointers; ++i) p.at[i] = i < here ? grads[first + i] : nullptr;
        adam_grads_kernel<<<1, kPointers, 0, st>>>(h->records, p, first, here);
        if (cudaGetLastError() != cudaSuccess) return QN_ERR_CUDA;
    }
    return QN_OK;
}

extern "C" qn_status qn_adam_norm(qn_adam_handle h, double* sumsq, void* cuda_stream) {
    if (!h || !sumsq || !check_array(sumsq, 8, h->device)) return QN_ERR_INVALID;
    DeviceGuard guard(h->device);
    if (!guard.ok) return QN_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:adam_norm");
    static int resident[2];
    const auto run = [&](auto kernel, int& r) {
        return launch(kernel, r, *h, st, static_cast<const Record*>(h->records), static_cast<const Chunk*>(h->chunk), h->chunks, h->pieces, h->partials, h->tickets + 1, sumsq);
    };
    const cudaError_t e = h->grad == QN_F32 ? run(adam_norm_kernel<float>, resident[0]) : run(adam_norm_kernel<__nv_bfloat16>, resident[1]);
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}

extern "C" qn_status qn_adam_step(qn_adam_handle h, int64_t* step, double lr, const float* lr_device, double beta1, double beta2,
                                  double eps, const double* sumsq, double max_norm, double grad_scale, int32_t rounding,
                                  uint64_t seed, void* cuda_stream) {
    if (!h || !step || !check_array(step, 8, h->device) || !check_array(lr_device, 4, h->device) || !check_array(sumsq, 8, h->device))
        return QN_ERR_INVALID;
    if (!lr_device && !(lr >= 0.0 && isfinite(lr))) return QN_ERR_INVALID;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(static_cast<float>(eps) >= 0x1p-126f) || !isfinite(static_cast<float>(eps)))
        return QN_ERR_INVALID;
    if (max_norm != max_norm || (max_norm > 0.0 && !sumsq) || !isfinite(grad_scale)) return QN_ERR_INVALID;
    if (rounding != QN_ROUND_NEAREST && rounding != QN_ROUND_STOCHASTIC) return QN_ERR_INVALID;
    DeviceGuard guard(h->device);
    if (!guard.ok) return QN_ERR_CUDA;
    const Hyper hyper{lr, log(beta1), log(beta2), max_norm, grad_scale,
                      static_cast<float>(beta1), static_cast<float>(1.0 - beta1), static_cast<float>(beta2), static_cast<float>(1.0 - beta2),
                      static_cast<float>(eps), -0.0f, static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32), rounding == QN_ROUND_STOCHASTIC};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:adam_step");
    const auto by_grad = [&](auto grad) {
        using G = decltype(grad);
        if (h->param == QN_F32) return launch_step<float, G, false>(*h, hyper, step, lr_device, sumsq, st);
        if (h->master) return launch_step<__nv_bfloat16, G, true>(*h, hyper, step, lr_device, sumsq, st);
        return launch_step<__nv_bfloat16, G, false>(*h, hyper, step, lr_device, sumsq, st);
    };
    const cudaError_t e = h->grad == QN_F32 ? by_grad(float()) : by_grad(__nv_bfloat16());
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}

extern "C" qn_status qn_adam_state(qn_adam_handle h, qn_dtype dtype, void* m, void* root, void* cuda_stream) {
    if (!h || (dtype != QN_F32 && dtype != QN_BF16)) return QN_ERR_INVALID;
    const size_t size = dtype_size(dtype), bytes = h->places * size;
    if (!check_array(m, size, h->device) || !check_array(root, size, h->device)) return QN_ERR_INVALID;
    if (m && root && overlaps(m, bytes, root, bytes)) return QN_ERR_INVALID;
    for (const auto& range : h->written)
        for (const void* p : {m, root})
            if (p && overlaps(p, bytes, reinterpret_cast<const void*>(range.first), range.second - range.first)) return QN_ERR_INVALID;
    if (h->chunks == 0 || (!m && !root)) return QN_OK;
    DeviceGuard guard(h->device);
    if (!guard.ok) return QN_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nvtxRangePushA("qn:adam_state");
    const auto by_type = [&](auto t) {
        using T = decltype(t);
        static int resident[2];
        const auto run = [&](auto kernel, int& r) {
            return launch(kernel, r, *h, st, static_cast<const Record*>(h->records), static_cast<const Chunk*>(h->chunk), h->chunks, h->pieces, static_cast<T*>(m), static_cast<T*>(root));
        };
        return h->eight ? run(adam_state_kernel<T, true>, resident[1]) : run(adam_state_kernel<T, false>, resident[0]);
    };
    const cudaError_t e = dtype == QN_F32 ? by_type(float()) : by_type(__nv_bfloat16());
    nvtxRangePop();
    return e == cudaSuccess ? QN_OK : QN_ERR_CUDA;
}
