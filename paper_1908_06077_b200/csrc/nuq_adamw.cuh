// The AdamW step's arithmetic, shared by the kernels over lists of tensors and by the decoder that applies it.
#pragma once
#include "nuq_common.cuh"

struct nuq_control;

namespace nuq {

// What a step needs besides its tensors.  The control record's fields by their place in it (see nuq_control in the header).
struct AdamwParams {
    float lr, beta1, rest1, beta2, rest2, eps;   // rest: 1 - beta
    float scale;                                 // multiplies the gradients
    float first, second;                         // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    float log1, log2;                            // ln beta: with a control record the powers are formed on the device
    uint32_t t;                                  // the step's number, its lower 32 bits
    const nuq_control* control;
    uint32_t round_keys[20];                     // Philox4x32-10 key schedule of the seed, as in EncodeParams
};

struct AdamwFactors {
    float scale, first, second, lr_factor;
    uint32_t t;
    bool taken;
};

__device__ __forceinline__ AdamwFactors adamw_factors(const AdamwParams& P) {
    AdamwFactors f;
    f.scale = P.scale;
    f.first = P.first;
    f.second = P.second;
    f.lr_factor = 1.0f;
    f.t = P.t;
    f.taken = true;
    if (P.control != nullptr) {
        const uint4 a = *reinterpret_cast<const uint4*>(P.control), b = *(reinterpret_cast<const uint4*>(P.control) + 1);
        const uint64_t step = (uint64_t)a.x | (uint64_t)a.y << 32;
        f.t = a.x;
        f.scale = P.scale * __uint_as_float(a.w);
        f.lr_factor = __uint_as_float(b.x);
        f.taken = b.y == 0u && step != 0u;
        // 1 - beta^t = -expm1(t ln beta): no cancellation, a relative error of a few 2^-24 whatever t is
        const float t = (float)step;
        f.first = P.lr * f.lr_factor / -expm1f(t * P.log1);
        f.second = 1.0f / sqrtf(-expm1f(t * P.log2));
    }
    return f;
}

// The moments of an element: each product is rounded before it is added, so that what is rounded to 8 bits afterwards is
// the same number for whoever computes it from the formula in fp32.
__device__ __forceinline__ void adamw_moments(const AdamwParams& P, float g, float& m, float& v) {
    m = __fadd_rn(__fmul_rn(m, P.beta1), __fmul_rn(g, P.rest1));
    v = __fadd_rn(__fmul_rn(v, P.beta2), __fmul_rn(__fmul_rn(g, g), P.rest2));
}
// root: sqrt(v).  keep: 1 - lr weight_decay
__device__ __forceinline__ float adamw_value(const AdamwParams& P, const AdamwFactors& f, float keep, float w, float m, float root) {
    return __fmaf_rn(keep, w, -__fdiv_rn(__fmul_rn(m, f.first), __fmaf_rn(root, f.second, P.eps)));
}

}  // namespace nuq
