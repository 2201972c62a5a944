// Exponentials of a split softmax, for decode attention whose results stay finite for scores and values of any size.
#pragma once

#include "common.h"

namespace ihip {

constexpr float kSoftmaxLowest = -3.4028234e38f;     // stand-in for -inf in maxima: no score is below it
// Exponentials are taken against a score (a maximum of some while ago) and times 2^-26, and the reference moves where eight of them add up
// to more than 2^-20: their products with values, which go up to 6 * 2^125, have finite sums over a million keys, and products with the
// smallest values that are appended, 2^-101, keep 2^-149 and with it 22 bits.  Scores are not scaled before the reference is taken off: of a
// large score and a reference that were rounded apart, the difference would be large as well.
constexpr float kSoftmaxShift = 26.f, kSoftmaxMaxSum = 0x1p-20f;
__device__ inline float softmax_exp(float score, float ref, float scale_log2e) { return __builtin_amdgcn_exp2f(fmaf(score - ref, scale_log2e, -kSoftmaxShift)); }
// of what was taken against `from`, where `to` is the reference
__device__ inline float softmax_weight(float from, float to, float scale_log2e) { return __builtin_amdgcn_exp2f((from - to) * scale_log2e); }
__device__ inline float softmax_lse(float ref, float sum, float scale_log2e)
{
    return sum == 0.f ? -INFINITY : fmaf(ref, scale_log2e, log2f(sum * 0x1p26f)) * 0.69314718055994530942f;
}

}  // namespace ihip
