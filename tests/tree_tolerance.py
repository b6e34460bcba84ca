"""How far tree attention over the 8-bit cache may be from its definition: fp32 outputs, all kernels.

Inside the kernels:
  * Values (E4M3) and 16-bit weights multiply exactly; weights are rounded to f16, half a step 2^-11 relative, in the numerator
    and in the sum of weights: 2 * 2^-11.  Below 2^-14 of the reference a weight is off by up to 2^-25 of it instead, at every
    token; the reference is a token's score, so the sum of weights is at least 1 in these units: T * 2^-25 * max |v|, twice.
  * The query is not rounded to 16 bits: a bf16 value is two E4M3 terms after its row was scaled to a largest magnitude in
    [128, 256) (up to 64 columns), exact but for what lies below E4M3's smallest step, 2^-9, i.e. 2^-10 / 128 = 2^-17 of the
    row's largest; or f16 (more columns), exact but for 2^-25 below 2^-14.
  * Scores are sums of exact products in fp32 by the tensor core.  Terms down to 2^-23 of the largest were measured to
    survive beside it, wherever they stand; so an instruction of 32 terms onto an accumulator loses at most 33 * 2^-24 of the
    largest partial sum, and there are at most 8 of them (16 terms and 8 of them with f16): 264 * 2^-24 of sum |q_d k_d|.
    Factors and exponents in fp32 add 2^-22 of the score: 2^-15.8 together.
  * A score error of e changes a weight by a factor of exp(e), and a quotient of two sums of weights by exp(2 e) at most.
  * Exponentials (2^-22), fp32 sums of weights and values (T / 16 accumulations of 2^-23) and the merge: 2^-12 covers T up to 10^4.
"""
import numpy as np


def tolerance(q, k, v, mag, spread, scale):
    """q [n, G, D], k and v [T, D] of one sequence and kv head; mag [n, G, D] and spread [n, G] as oracle.spec_oracle gives them."""
    q_err = np.maximum(2.0 ** -17 * np.abs(q).max(-1), 2.0 ** -25)                       # [n, G], of any dim
    score = 2.0 ** -15.8 * spread + q_err * np.abs(k).sum(-1).max(initial=0.0) * scale
    relative = 2 * 2.0 ** -11 + 2.0 ** -12 + np.expm1(2 * score)
    return relative[..., None] * mag + 2 * 2.0 ** -25 * k.shape[0] * np.abs(v).max(initial=0.0)
