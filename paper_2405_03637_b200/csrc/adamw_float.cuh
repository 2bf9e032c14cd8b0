// AdamW in IEEE single operations, in the order of Algorithm 2: shared by the comparator with float states and the
// multi-tensor step.
#pragma once
#include "host_common.cuh"

namespace collage {

struct Fp32Scalars {
    float b1, c1, b2, c2, bc1, bc2, neg_a, lam, eps;
    uint32_t flags;
};

inline Fp32Scalars fp32_scalars(const collage_hyper_t* hyper, uint64_t step) {
    const double t = static_cast<double>(step);
    Fp32Scalars k;
    k.b1 = static_cast<float>(hyper->beta1);
    k.c1 = static_cast<float>(1.0 - hyper->beta1);
    k.b2 = static_cast<float>(hyper->beta2);
    k.c2 = static_cast<float>(1.0 - hyper->beta2);
    k.bc1 = static_cast<float>(1.0 - std::pow(hyper->beta1, t));
    k.bc2 = static_cast<float>(1.0 - std::pow(hyper->beta2, t));
    k.neg_a = -static_cast<float>(hyper->lr);
    k.lam = static_cast<float>(hyper->weight_decay);
    k.eps = static_cast<float>(hyper->eps);
    k.flags = hyper->flags & COLLAGE_FLAG_EPS_INSIDE_SQRT;
    return k;
}

// The update of a parameter of value w, lines 8-12; m and v are updated in place.
__device__ __forceinline__ float adamw_fp32_delta(float& m, float& v, float w, float g, const Fp32Scalars& k) {
    m = __fadd_rn(__fmul_rn(k.b1, m), __fmul_rn(k.c1, g));
    v = __fadd_rn(__fmul_rn(k.b2, v), __fmul_rn(k.c2, __fmul_rn(g, g)));
    const float mhat = __fdiv_rn(m, k.bc1);
    const float vhat = __fdiv_rn(v, k.bc2);
    const float den = (k.flags & 1u) ? __fsqrt_rn(__fadd_rn(vhat, k.eps)) : __fadd_rn(__fsqrt_rn(vhat), k.eps);
    const float u = __fadd_rn(__fdiv_rn(mhat, den), __fmul_rn(k.lam, w));
    return __fmul_rn(k.neg_a, u);
}
// One parameter: Algorithm 2 lines 8-13 in float.  Returns the update; w is the stored float
// parameter (master weight, or the widened bfloat16 parameter), updated in place.
__device__ __forceinline__ float adamw_fp32_element(float& m, float& v, float& w, float g, const Fp32Scalars& k) {
    const float delta = adamw_fp32_delta(m, v, w, g, k);
    w = __fadd_rn(w, delta);
    return delta;
}

__device__ __forceinline__ uint16_t to_bf16_rn(float x) {
    uint16_t h;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(x));
    return h;
}
__device__ __forceinline__ float from_bf16(uint16_t h) { return __uint_as_float(static_cast<uint32_t>(h) << 16); }

}  // namespace collage
