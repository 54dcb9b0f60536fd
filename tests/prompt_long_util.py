"""A bound for prompt attention over many keys that a single wrong tile of V does not keep."""
from prompt_util import attention  # noqa: F401


def check_long(out, want, where):
    """Over n keys of similar weight the output is about n^(-1/2) of a value, and bounds that let every weight err the same way let more than that pass.
    Here the errors that count are independent from key to key: the weights' rounding to bf16, at most 2^-8 of each, so that a value's error exceeds six times
    2^-8 sqrt(sum p^2 v^2) in one of exp(18) / 2 = 3e7 at most (Hoeffding), and its 2-norm over thousands of them is within the norm of these bounds with nothing
    to multiply.  The output's own rounding is at most 2^-8 of it.  Logits, sums and the division are 32-bit: a logit of up to 2^6 binary orders is off by 2^-17
    at most (128 products added in 2^-24 steps), a weight as much, sums of pieces less: 2^-12 of either is more than all of them together."""
    o, _, _, p2 = want
    err = (out.double() - o).abs()
    tol = 6 * 2.0 ** -8 * p2 + 2.0 ** -8 * o.abs() + 2.0 ** -12 * (p2 + o.abs())
    assert (err <= tol).all(), (where, float((err - tol).max()))
    norm = float((p2.square() + o.square()).sum().sqrt())
    assert float(err.norm()) <= (2.0 ** -8 + 2.0 ** -12) * norm, (where, "2-norm", float(err.norm()) / norm)
