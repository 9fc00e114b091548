"""Acceptance bounds of the parity checks, in one place (tests/ and bench.py use these and nothing else).

Notation: Y the oracle's fp64 result, A = sum_k |w x| the oracle's absolute sum (the contract's tolerance
scale), K the row length.  Everything here is numpy on the oracle's outputs; nothing of the method's
arithmetic lives in this file.

1. TOL: the benchmark contract's criterion, |y_gpu - Y| <= 2e-3 * A.
2. arithmetic_bound: what the arithmetic itself allows for ANY shape.  fp32 accumulation in any order is
   within K * 2^-23 * A of the exact sum, and rounding the result to bf16 (8 significant bits) adds at most
   half an ulp <= 2^-8 * |y|.  For short or same-sign rows |y| is close to A and that rounding alone exceeds
   TOL * A (a single product, K = 1, can be off by 0.39 % of itself in any bf16 output), so the contract's
   criterion is asserted where it is attainable (K >= 512 and all benchmark configurations: long mixed-sign
   sums) and this bound everywhere.
3. swiglu_bound: y = silu(g) * u with g, u two products.  silu' lies in [-0.1, 1.1], so an error dg in g and
   du in u moves y by at most 1.1 |u| dg + |silu(g)| du + 1.1 dg du; the combination itself takes a few fp32
   roundings, and the result one bf16 rounding.
4. rmsnorm_commute_bound: the fused calls' definition rounds x * r * g to bf16; the kernels round x * g and
   apply the scalar r to the fp32 sum.  Both roundings are within half an ulp (2^-8 relative) of the same
   exact value, so an activation differs by at most 2^-7 of itself and the sum by at most 2^-7 * sum |w xn|
   (worst case: both roundings opposed on every term; independent errors add in quadrature, so long rows
   stay far inside TOL * A, which the callers assert as well for K >= 512).
"""
import numpy as np

TOL = 2e-3


def arithmetic_bound(A, Y, K):
    return (K + 8) * 2.0 ** -23 * A + 2.0 ** -8 * (np.abs(Y) + (K + 8) * 2.0 ** -23 * A)


def swiglu_bound(G, U, Ag, Au, silu_G, want, K):
    """G, U: the two fp64 products; Ag, Au: their absolute sums; silu_G = silu(G); want = silu(G) * U."""
    dg, du = (K + 8) * 2.0 ** -23 * Ag, (K + 8) * 2.0 ** -23 * Au
    inner = 1.1 * np.abs(U) * dg + np.abs(silu_G) * du + 1.1 * dg * du + 8 * 2.0 ** -23 * np.abs(want)
    return inner + 2.0 ** -8 * (np.abs(want) + inner)


def swiglu_contract_bound(U, Ag, Au, silu_G, want):
    """The contract's 2e-3 * A on each product, carried through the combination, plus the bf16 rounding."""
    return TOL * (1.1 * np.abs(U) * Ag + np.abs(silu_G) * Au) + 2.0 ** -8 * np.abs(want)


def rmsnorm_commute_bound(A_product):
    """A_product: sum_k |w xn| of the product alone (without a residual)."""
    return 2.0 ** -7 * A_product


def attention_lse_bound(size, tokens, head_dim):
    """Log-sum-exp of attention over `tokens` tokens in fp32.  size: the largest |scale| sum_d |q_d k_d| among them.  A score is a sum
    of head_dim products that are exact in fp32, then multiplied by a block's scale and by scale * log2(e) and brought to base 2 less
    the maximum: (head_dim + 24) roundings of at most 2^-23 * size.  The exponential is good to 2^-21 of itself, and a sum of
    `tokens` positive terms to tokens * 2^-23; the last logarithm, and adding the maximum, are a few roundings more (2^-20 of 1 + size)."""
    return (head_dim + 24) * 2.0 ** -23 * size + 2.0 ** -21 + tokens * 2.0 ** -23 + 2.0 ** -20 * (1 + size)


def attention_bound(out, spread, size, tokens, head_dim):
    """Attention output in bf16.  out: the fp64 result; spread: sum p |v| / sum p.  Every p is off by d, the score's error and the
    exponential's (attention_lse_bound bounds both), in the numerator and in the sum that divides it; p times V's scale, or V times its
    scale, or both are rounded to bf16 once (2^-8 each) before the second product, whose fp32 sum of `tokens` terms adds
    tokens * 2^-23; the result is rounded once more."""
    d = attention_lse_bound(size, tokens, head_dim)[..., None]
    inner = (2 * d * (1 + d) + 2 * 2.0 ** -8 + (tokens + 8) * 2.0 ** -23) * spread
    return inner + 2.0 ** -8 * (np.abs(out) + inner)
