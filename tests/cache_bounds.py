"""The bound that the cache's attention kernels claim for o, without the slack of cache_util's (which lets weights of bf16 pass)."""
import numpy as np

HALF_FP16, HALF_BF16, HALF_FP32 = 2.0 ** -11, 2.0 ** -8, 2.0 ** -24     # half a step, relative to the value


def tight(ref, spread, reach, wide, n, D, largest):
    """|o - ref| at most.  ref, spread [.., D], reach, wide [..] as the model's attend gives them; n keys; largest = max |v| of the sequence.

    * A score's error is e_s as in cache_util.check_attention: fp32 sums of D exact products, the query's two 8-bit numbers, 2^-21 for the exponential.
    * A weight is rounded to fp16: 2^-11 of itself, or 2^-25 where it is below the normal numbers.  The largest one is 2^7 at least (chunks; 2^15 for
      tokens), and the sum is no smaller, so the latter is 2^-32 after division, for each of n keys.
    * o is a mean of V, which is exact, under the rounded weights, whose own sum divides it: errors of weights count for |v| and for |o|, and
      dividing by 1 - 2^-11 instead of 1 adds a 2^-10th of them.
    * Sums in fp32 of n terms, of products and of weights: 2 n 2^-24.
    * o is rounded to bf16 at the end: 2^-8 of what it then is."""
    e_s = (D + 8) * HALF_FP32 * reach + 2.0 ** -21 * wide + 2.0 ** -21
    mass = spread + np.abs(ref)
    before = (HALF_FP16 + e_s[..., None]) * mass * (1 + 2.0 ** -9) + n * 2.0 ** -32 * (largest + np.abs(ref)) + 2 * n * HALF_FP32 * mass
    return before * (1 + HALF_BF16) + HALF_BF16 * np.abs(ref)
