"""Newton-Schulz steps in 64 bits, on the CPU, with a bound of what the kernels'
arithmetic may differ from them by in the 2-norm of a matrix.

One product C = X Y of length k.  Its values go in as pairs of fp16 numbers: a
pair is within 2^-22 of its value, the left-out product of low parts is below
2^-22 of the product, so every term is within 3 * 2^-22 (high parts alone:
2 * 2^-11).  The terms' errors are independent: their sum stays within three
times that of sqrt(sum x^2 y^2).  Summing 3 k terms (k) in float32 rounds each
running sum by at most 2^-24 of itself; those roundings too add up as their
square root's number, and a running sum is at most |C| and three times
sqrt(sum x^2 y^2) more.  Entry by entry, with R = sqrt((X o X)(Y o Y)):

  |dC| <= (9 * 2^-22 + 6 sqrt(3 k) 2^-24) R + 2 sqrt(3 k) 2^-24 |C|

(high parts alone: 6 * 2^-11 for the first term).  A step's own error follows
from dA, d(A A), the rounding of B (2^-22, alone 2^-11, and 2^-24 three times)
and d(B X), and an error of X grows by no more than the largest |p'| on the
singular values' range, p(v) = a v + b v^3 + c v^5 (the Lipschitz constant of
X -> p(X) in this norm)."""
import torch

U32 = 2.0 ** -24


def _product(x, y, pair):
    c, k = x @ y, x.shape[1]
    r = (x.square() @ y.square()).sqrt()
    root = (3 * k) ** 0.5 * U32
    d = ((9 * 2.0 ** -22 if pair else 6 * 2.0 ** -11) + 6 * root) * r + 2 * root * c.abs()
    return c, float(d.norm())


def steps_of(m, coefficients, steps, eps, pairs):
    """(X, bound of |error|) of one matrix after `steps` steps; pairs: of each step, whether its products take both parts."""
    a, b, c = coefficients
    m = m.double()
    tall = m.shape[0] > m.shape[1]
    x = (m.t() if tall else m).contiguous()
    norm = float(x.norm())
    x = x / (norm + eps) if norm + eps > 0 else x * 0
    err = 2 * U32 * float(x.norm())
    for pair in pairs[:steps]:
        s = float(torch.linalg.matrix_norm(x, 2)) + err
        g, dg = _product(x, x.t(), pair)
        gg, dgg = _product(g, g, pair)
        p = b * g + c * gg
        g2 = s * s
        dp = abs(b) * dg + abs(c) * (dgg + 2 * g2 * dg) + ((2.0 ** -22 if pair else 2.0 ** -11) + 3 * U32) * float(p.norm()) + \
            4 * U32 * (abs(b) * float(g.norm()) + abs(c) * float(gg.norm()))
        px, dpx = _product(p, x, pair)
        new = a * x + px
        own = dp * s + dpx + 4 * U32 * (abs(a) * float(x.norm()) + float(px.norm()))
        v = torch.linspace(0, s, 2001, dtype=torch.float64)
        slope = float((a + 3 * b * v ** 2 + 5 * c * v ** 4).abs().max())
        err = slope * err + own
        x = new
    return (x.t() if tall else x).contiguous(), err


def check(got, m, coefficients, steps, eps, what):
    """A result against 64 bits: pairs everywhere for float32; for bf16, whose rounding counts too, from the step on before
    which alike singular values would be sqrt(0.14), and in the last two."""
    f32, n = got.dtype == torch.float32, min(m.shape)
    want, bound = steps_of(m, coefficients, steps, eps,
                           [f32 or k + 2 >= steps or coefficients[0] < 1 or coefficients[0] ** (2 * k) > 0.14 * n for k in range(steps)])
    g = got.detach().cpu().double()
    assert g.shape == want.shape and torch.isfinite(g).all(), what
    bound += (U32 if f32 else 2.0 ** -8) * float(want.norm()) + 1e-37
    off = float((g - want).norm())
    assert off <= bound, "%s: off by %.3g, %.3g allowed, of %.3g" % (what, off, bound, float(want.norm()))
    return off, bound
