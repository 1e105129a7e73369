"""Norms of the errors of the gated delta rule's results, for each row and head: what tests/delta_reference.py bounds number by number for
the worst case, here as roundings add up when they fall at random, which is some hundred times closer.

A group is a row's and head's numbers of one result (all steps and columns).  Its error's norm is held against the norm of the group,
or, where that is more, the root mean square of all groups' norms (a group of few numbers can be small by chance).

Limits.  A sum of n products of random signs makes an error of 0.28 sqrt(n) 2^-24 of its result: roundings of 0.4 2^-24 (the root mean
square of a rounding of at most 2^-24) of partial sums that grow with the root of their number.  A result comes of at most n = dk + dv + 2 C
products (C = 32 steps of a chunk, or T) in some five sums behind one another (the products with the state, the substitution, the chunk's own
products, the state's update, twice backwards), whose errors add up as squares: sqrt(5) 0.28 sqrt(n) 2^-24 = 0.63 sqrt(n) 2^-24, and
as much again from a state that took in L steps, C at a time: a factor of sqrt(1 + L / C).  Decays add a relative error of at most 4 2^-24
(the rounding of an exponent of up to 6 binary digits, and of exp2 itself).  What is left over of terms that are larger than their sum has their
errors: estimated from the terms' sizes, a factor of up to six (dlog_decay, the inner product of two states, is in a chunk a sum over
its steps of terms as large as itself: sqrt(32)).  So 32-bit results: 4 sqrt(n (1 + L / C)) 2^-24.

bf16 results are rounded once: of 1024 numbers or more (Gaussian or Laplacian, of any size) that is 0.00155 to 0.0018 of their norm, less than 2^-9, and of fewer
at most 2^-8; what enters the last products as two bf16 terms leaves out 2^-16 of each of three factors, 2^-13 with terms that are larger than
their sum.  A second rounding to bf16 on the way, 0.0023 in all, does not pass.
"""
import math

CHUNK = 32
BY_STATE = ("state", "dstate0")


def groups(name, a):
    """Norms of [N, heads]."""
    if name in BY_STATE:
        return a.flatten(2).norm(dim=-1)
    return a.norm(dim=0) if a.dim() == 3 else a.norm(dim=-1).norm(dim=0)


def limit(name, y, dk, dv, length, bf16, T):
    C = min(CHUNK, T)
    lim = 4 * math.sqrt((dk + dv + 2 * C) * (1 + min(length, T) / C)) * 2.0 ** -24
    if bf16 and name in ("o", "dq", "dk", "dv"):
        lim += 2.0 ** -13 + (2.0 ** -9 if T * y.shape[-1] >= 1024 else 2.0 ** -8)
    return lim


def over(name, x, y, dk, dv, length, bf16, T):
    """The largest of the groups' errors, in parts of the limit."""
    x, y = x.double(), y.double()
    assert x.shape == y.shape, name
    size = groups(name, y)
    size = size.clamp(min=size.square().mean().sqrt().item())
    off = groups(name, x - y)
    return (off / (limit(name, y, dk, dv, length, bf16, T) * size + 1e-37)).nan_to_num(nan=math.inf).max().item()


def check(got, want, dk, dv, length, bf16, T):
    for name, y in want.items():
        part = over(name, got[name], y, dk, dv, length, bf16, T)
        assert part <= 1.0, "%s: %.2f of the limit" % (name, part)
