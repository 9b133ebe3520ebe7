"""How precise attention over pages in 4 bits and adapters have to be as a whole, where bounds on single outputs leave room for every rounding at its worst.

Rounding to u = 2^-11 (fp16) leaves a relative error of u / sqrt(3) times sqrt(ln 2 / 1.5) = 1.9e-4 of the norm where mantissas are spread evenly in their logarithm, and
up to u / sqrt(3) = 2.8e-4 where the values lie just above a power of two.  Outputs are rounded once; probabilities with their value's scale once, and as
many independent terms they leave the same relative error of a sum whose terms cancel as much as these do.  Together 2.7e-4, at most 4.0e-4: NORM16.

Rounded to bf16 the output's own error hides everything else; but a value that is off by e of the norm before it is rounded lands beside the rounded 64-bit one in
|e| / spacing of all cases, the spacing 2^-7 / 1.44 of the value.  For values of a normal distribution, with c = 184 E|e| where the two are equal, that is
c (2 / pi)^(1/2) E1(c^2 / 2) / 2 + P(|x| < c): 0.10 for one rounding to fp16 (E|e| = 0.8 * 1.9e-4, c = 0.028: 0.028 * 0.8 * 3.6 + 0.02) and 0.14 at the most (2.8e-4), 0.45 for one
to bf16 (c = 0.22: 0.22 * 0.8 * 1.6 + 0.17).  BESIDE: 0.2.

A projection with adapters: weights of the shared product as fp16, inner values as fp16 of their row's power of two, the output: three such errors at the most,
ADAPTERS16 = 2.8e-4 sqrt(3).  silu(gate) up: those of both (silu's slope times gate is at most 1.1 of it or so), less an output: GATED16 = 2.8e-4 sqrt(5) 1.1."""
import torch

NORM16, BESIDE = 4.0e-4, 0.2
ADAPTERS16, GATED16 = 4.9e-4, 6.9e-4


def norm_error(out, want):
    return float((out.double() - want).norm() / want.norm())


def beside(out, want):
    """Share of the outputs that are not the 64-bit value, rounded."""
    return float((out != want.to(out.dtype)).double().mean())


def precise(out, want):
    return norm_error(out, want) <= NORM16 if out.dtype == torch.float16 else beside(out, want) <= BESIDE
