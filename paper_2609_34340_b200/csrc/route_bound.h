// How far a router key in 32 bits can be from its definition.  It compiles as plain C++, too.
#pragma once

#ifdef __CUDACC__
#define VP_BOUND __host__ __device__ __forceinline__
#else
#define VP_BOUND inline
#endif

// Twice a bound of a score's error, relative to the largest score of the token (softmax) or to 1 (sigmoid).  In units of 2^-24:
//   The exponential of -d is off by d for each of the argument's difference and its product with log2 e, 0.23 d for that constant, and 4.
//   Softmax: that for the score itself; its mean under the softmax for the sum (the mean of d is below 3.4 with 256 experts, 4.5 with 1,024), with an
//   addition per value of a lane and five across lanes; 2 for the reciprocal, 1 for the product.  Where d is 0 that is most: per_lane + 16 + 2.23
//   times the mean.  (With one constant for all sizes, 32, 16,384 tokens of 256 experts in groups took 17.4 us instead of 16.6: more tokens for
//   the comparison in 64 bits.)
//   Sigmoid: ds = s (1 - s) d(exp) / exp, below 1.3; 1 for the sum and 2 for the reciprocal: below 5.
VP_BOUND float twice_score_error(bool sigmoid, int per_lane) {
    return sigmoid ? 2e-6f : (per_lane + (per_lane <= 8 ? 24 : 27)) * 1.2e-7f;
}
