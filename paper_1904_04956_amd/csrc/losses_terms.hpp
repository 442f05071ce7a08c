// What a frame's loss is made of, for the kernels that end its sums.
#pragma once
#include "common.hpp"
#include "losses.hpp"

namespace blstm {
namespace {

constexpr float LOG2E = 1.44269504f, LN2 = 0.693147181f;

// Two floats rounded to bf16, in one instruction.
__device__ __forceinline__ unsigned pack2(float lo, float hi) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2_t{lo, hi}), bf16x2_t));
}

// a b, rounded, and no part of a multiply-add.  The exponent of a sum's term is fmaf(u, k, -r) with r the rounded product of the reference and k: the
// same r in every term, so that its rounding (2^-24 of u over the temperature) cancels, as long as sums are brought to another r by the
// difference of the two.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

struct PolicyTerms { float loss, g; };
__device__ __forceinline__ PolicyTerms policy_terms(const PolicyArgs& p, long long m, float lp) {
    const float A = p.advantage[m];
    float loss = 0.0f, g = 0.0f;
    if (A != 0.0f) {                                     // (an infinite ratio times an advantage of zero is no number)
        const float r = p.old_logp ? expf(lp - p.old_logp[m]) : 1.0f;
        const float inner = r * A, outer = fminf(fmaxf(r, 1.0f - p.clip_low), 1.0f + p.clip_high) * A;
        loss = inner > outer ? -outer : -inner;          // (a NaN ratio stays one)
        const bool cut = (A > 0.0f && r > 1.0f + p.clip_high) || (A < 0.0f && r < 1.0f - p.clip_low);
        g = cut ? 0.0f : -inner;
    }
    if (p.ref_logp) {
        const float d = p.ref_logp[m] - lp, e = expm1f(d);
        loss += p.kl_weight * (e - d);
        g -= p.kl_weight * e;
    }
    return {loss, g};
}

}  // namespace
}  // namespace blstm
