"""Shared by the tests of the operators."""

def between(got, want, bound):
    """Whether got is the rounding to its type of something within `bound` of `want` (rounding is monotone)."""
    lo, hi = (want - bound).float().to(got.dtype), (want + bound).float().to(got.dtype)
    return bool(((got >= lo) & (got <= hi)).all())
