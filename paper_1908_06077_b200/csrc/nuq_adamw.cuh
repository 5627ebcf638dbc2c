// The AdamW step's arithmetic, shared by the kernels over lists of tensors and by the decoder that applies it.
#pragma once
#include "nuq_common.cuh"

struct nuq_control;

namespace nuq {

// What a step needs besides its tensors.
struct AdamwParams {
    float beta1, rest1, beta2, rest2, eps;       // rest: 1 - beta
    float lr;
    float scale;                                 // multiplies the gradients
    float first, second;                         // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    float log1, log2;                            // ln beta: with a control record the powers are formed on the device
    uint32_t t;                                  // the step's number, its lower 32 bits
    const nuq_control* control;
    uint32_t round_keys[20];                     // Philox4x32-10 key schedule of the seed, as in EncodeParams
};

// The decoder's sums applied at once: see SumParams.
struct AdamwSum {
    float* acc;              // where they are stored too, or nullptr
    float *w, *m, *v;
    float decay;             // lr weight_decay
    AdamwParams step;
};

// The step is m / (root second / first + eps / first).
struct AdamwFactors {
    float scale, root_factor, eps, lr_factor;
    uint32_t t;
    bool taken;
};

constexpr float kMostRate = 0x1p40f;             // the largest learning rate
__device__ __forceinline__ AdamwFactors adamw_factors(const AdamwParams& P) {
    AdamwFactors f;
    float first = P.first, second = P.second;
    f.scale = P.scale;
    f.lr_factor = 1.0f;
    f.t = P.t;
    f.taken = true;
    if (P.control != nullptr) {                  // (the record's fields by their places, see nuq_control)
        const uint4 a = *reinterpret_cast<const uint4*>(P.control), b = *(reinterpret_cast<const uint4*>(P.control) + 1);
        const uint32_t begun = reinterpret_cast<const uint32_t*>(P.control)[9];                  // (ControlRecord::begun)
        const uint64_t step = (uint64_t)a.x | (uint64_t)a.y << 32;
        f.t = a.x;
        f.scale = P.scale * __uint_as_float(a.w);
        f.lr_factor = __uint_as_float(b.x);
        const float lr = P.lr * f.lr_factor;
        f.taken = f.lr_factor >= 0.0f && lr <= kMostRate && b.y == 0u && step != 0u && (begun != 0u || __uint_as_float(a.w) != 0.0f);
        // 1 - beta^t = -expm1(t ln beta): no cancellation, a relative error of a few 2^-24 whatever t is
        const float t = (float)step;
        first = lr / -expm1f(t * P.log1);
        second = 1.0f / sqrtf(-expm1f(t * P.log2));
    }
    // (a learning rate of 0, or as good as that: a denominator that is infinite also for a root of 0)
    const bool moves = first > 0x1p-96f;
    f.root_factor = moves ? second / first : 0x1p126f;
    f.eps = moves ? P.eps / first : __uint_as_float(0x7f800000u);
    return f;
}

// What multiplies w.  decay: lr weight_decay, finite, as is the factor; their product need not be, and 0 stays 0 all the same.
__device__ __forceinline__ float adamw_keep(const AdamwFactors& f, float decay) { return fmaxf(1.0f - f.lr_factor * decay, -0x1.fffffep127f); }

// The moments of an element.  Each product is rounded before it is added, so that what is rounded to 8 bits afterwards is
// the same number for whoever computes it from the formula in fp32.
// (One element at a time: two in a register pair take half the instructions, but those run on one of the two multiply-add pipes
// only, the one that the integer products of the random bits need, and their constants have to be moved to registers first.
// 2^28 elements with 8-bit states: in pairs 836 us, so 802, both before the other steps.)
__device__ __forceinline__ float moment1(const AdamwParams& P, float g, float m) { return __fadd_rn(__fmul_rn(m, P.beta1), __fmul_rn(g, P.rest1)); }
__device__ __forceinline__ float moment2(const AdamwParams& P, float g, float v) { return __fadd_rn(__fmul_rn(v, P.beta2), __fmul_rn(__fmul_rn(g, g), P.rest2)); }

// sqrt(v), correctly rounded for v from 2^-100 to the largest number: an estimate of 1 / sqrt(v) within a few units of its last place,
// and one step of Newton's method for s^2 = v, whose remainder v - s^2 is exact in a fused operation (P. Markstein, Computation
// of elementary functions on the IBM RISC System/6000 processor, IBM J. Res. Dev. 34, 1990: the sum of s and the remainder's
// part is within a little more than half a unit, so a wrong rounding needs a root next to the middle between two numbers).  That
// it happens for no v rests on a comparison with __fsqrt_rn for every one of them, which the tests repeat.  Below, the remainder
// would be lost; 0 and infinity give NaN: those are the caller's to find.
constexpr float kLeastRoot = 0x1p-100f;
__device__ __forceinline__ float ordinary_root(float v) {
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(v));
    const float s = __fmul_rn(v, y);
    return __fmaf_rn(__fmaf_rn(-s, s, v), __fmul_rn(y, 0.5f), s);
}
// sqrt(v) within two units of its last place, for all v: where nothing but the step depends on it.
__device__ __forceinline__ float root_estimate(float v) {
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(v));
    return y;
}
__device__ __forceinline__ float reciprocal_estimate(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 1 / x, correctly rounded for x from 2^-100 to 2^126: the same, for 1 / y = x.  By Markstein's theorem (there) an estimate within one
// unit of its last place is enough, except perhaps for an x whose mantissa is all ones; here too the tests compare every x, with __frcp_rn.
__device__ __forceinline__ float reciprocal(float x) {
    const float y = reciprocal_estimate(x);
    return __fmaf_rn(y, __fmaf_rn(-x, y, 1.0f), y);
}
// The largest of three numbers, NaN if one is; the smallest of those that are numbers.
__device__ __forceinline__ float largest3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float smallest3(float a, float b, float c) {
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// w from the new moments.  keep: 1 - lr weight_decay; root: sqrt(v).  The quotient is a product with an estimate of the reciprocal: within
// 3 units of its last place, and the step is far smaller than what it is subtracted from.  (A denominator below 2^-126 counts
// as 0.)
__device__ __forceinline__ float adamw_value(const AdamwFactors& f, float keep, float w, float m, float root) {
    return __fmaf_rn(keep, w, -__fmul_rn(m, reciprocal_estimate(__fmaf_rn(root, f.root_factor, f.eps))));
}

}  // namespace nuq
