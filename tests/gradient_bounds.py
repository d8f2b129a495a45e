"""How far gradients of attention may be off as a whole, besides value by value: bounds that an error of a few per cent
does not pass, where those of single values are as wide as many of the values.

The roundings to bf16 are of p or ds as a matrix operand, of the output that rowsum(dout out) takes, with its own p and
result, and of the gradient itself.  Each moves a value by at most 2^-8 of it, spread evenly: 2^-8 / sqrt(3) = 0.00226 in the
root mean square, and different values are moved independently of each other, so that a sum of products with random factors is
off by as much of its own size.
* dv: p and the result, 0.0032.
* dq, dk: ds and the result, 0.0032; and p times what the row sums are off.  The latter is 0.0032 (its p and result) of
  |out|, while ds is p times the difference of dout v from its mean, |v| in size, which is larger than |out| where more than two keys
  weigh: 0.0032 at most.  Together 0.0045.
Sums in 32 bits add 2^-14.  With room for rows that see one or two keys: 0.006."""
import torch

BOUND = 0.006


def share(got, want):
    """The size of the error, of the size of what should be."""
    got, want = got.cpu().double(), want.cpu().double()
    return float((got - want).norm() / want.norm())


def along(gradient, value, at):
    """Whether a gradient of `value` at `at` is as long as the value's central difference along it, in 64 bits, says.  Along
    itself an error of 0.006 of its size changes the product by as much of its square, and nothing cancels."""
    g = gradient.cpu().double()
    n = float(g.norm())
    if n == 0:
        return False
    step = 1e-5
    by = float((value(at + step * g / n) - value(at - step * g / n)) / (2 * step))
    return abs(by - n) <= BOUND * n * 1.01 + 1e-6
