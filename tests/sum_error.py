"""How far sums of products may be off as a whole: bounds that a sum or an operand in too few bits does not meet, where the worst
case of K roundings, which grows with K times the sum of magnitudes, hides them from a few thousand products on.

For K independent products of zero mean, s = sqrt(sum (x w)^2) is the size of a sum, and of its first i products
s sqrt(i / K).

f32 multiply-adds.  A rounding is off by at most 2^-24 of the partial sum, evenly spread: 2^-24 / sqrt 3 on average.  One chain of K
of them, the longest that a kernel can make: sqrt(sum_i i / K / 3) = sqrt(K / 6) of 2^-24 s, and one rounding more at the end.

Tensor cores.  A step adds `products` products to the sum and may cut the result instead of rounding it, 2^-23 of the partial sum
and always towards zero, so that errors add up: over S = K / products steps sum_i sqrt(i / S) = 2/3 S of 2^-23 s.  S of 2^-23 s
leaves half as much again for products that are cut where they are lined up, and for partial sums handed over; 32 steps more
for sums of few."""
import numpy as np


def fma_bound(K):
    return 2.0 ** -24 * (np.sqrt(K / 6) + 1)


def tensor_bound(K, products):
    return 2.0 ** -23 * (K / products + 32)


def off(got, exact, x, w):
    """(root mean square, largest) error in units of s; arrays of numpy or torch in 64 bits, x [R, K], w [N, K]."""
    e = (got - exact) / ((x * x) @ (w * w).T) ** 0.5
    return float((e * e).mean()) ** 0.5, float(abs(e).max())
