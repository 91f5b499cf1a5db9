"""How far a state, a reverse-time state and ds may be from 64 bits where the calls with a decay return them to fp32's accuracy.

In the mean square a rounding is off by 0.43 of its largest error 2^-24 (mantissas of all sizes), and errors of either sign
add up as their squares.  An element of a state is a sum of n terms k_j g^(n-1-j) / |k_j| v_jc.  A term has met some eight
roundings: the norm's sum and root, the decay's logarithm, product and power, the weight, and what an operand's parts leave,
2^-27 in three bfloat16 parts and (2^-12)^2 = 2^-24 in two of fp16.  The sum takes at most one rounding a term, of partial sums
whose mean square is half the whole's.  Relative to the state's 2-norm that is

    0.43 2^-24 sqrt(8 + n / 2).

ds of a head is the sum of <H, G>, two such matrices, over the chunks (off by sqrt(2) times that, relative to the root of the sum
of its terms' squares: <dH, G> of errors dH that are independent of G is to <H, G> as |dH| to |H|), of whose dk dv products per
chunk each of 64 lanes or more adds its own one after the other.  Both are allowed twice this.
"""
import torch

import decay_reference as ref

ROUNDING = 0.43 * 2.0 ** -24


def state_bound(n):
    return 2 * ROUNDING * (8 + n / 2) ** 0.5


def ds_bound(n, dk, dv, chunk):
    in_lane = dk * dv / 64 * -(-n // chunk)
    return 2 * ROUNDING * (2 * (8 + n / 2) + in_lane / 2) ** 0.5


def state_error(got, want):
    """The largest of the relative errors in 2-norm of the heads' matrices."""
    got, want = got.detach().cpu().double().flatten(2), want.flatten(2)
    return float(((got - want).norm(dim=-1) / want.norm(dim=-1)).max())


def ds_terms(x, log_decay):
    """[B, H]: the root of the sum of the squares of g^(i-j) (qh_i . kh_j) (dO_i . v_j), j <= i."""
    qh, kh = ref.unit(x["Q"].double(), 1e-6)[0], ref.unit(x["K"].double(), 1e-6)[0]
    w = ref.weights(log_decay, x["Q"].shape[2])
    p, a = qh @ kh.transpose(-1, -2) * w, x["dO"].double() @ x["V"].double().transpose(-1, -2)
    return (p * a).flatten(2).norm(dim=-1)


def ds_error(got, want, terms):
    """Root mean square over the heads ([B, H]) of the error relative to the terms."""
    return float((((got.detach().cpu().double() - want) / terms) ** 2).mean().sqrt())
