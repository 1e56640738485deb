"""A sharper bound for several Newton-Schulz steps than the largest slope to the
power of their number: what each step's own errors become by the end.

In exact arithmetic the singular vectors of X stay the same from step to step.
In their basis a small error d of X goes through a step X -> p(X) pair by pair,
with x and y the singular values of the pair (0 beside the last one, for rows and
columns outside X's space):

  d_ij + d_ji  times  (p(x) - p(y)) / (x - y)
  d_ij - d_ji  times  (p(x) + p(y)) / (x + y)

so that the largest product of such factors bounds what becomes of an error that
lies anywhere (`spread`).  An error of the polynomial's matrix, D X, has d_ij =
D_ij y, d_ji = D_ji x, and becomes at most max sqrt((F^2 + G^2) / 2 (x^2 + y^2))
|D| with the products F and G of the two factors (`inside`): what small singular
values multiply up starts as small as they are.

A step's own errors are those of ortho_ref, every product on pairs.  Rows and
columns of zeros stay zeros exactly, since every term of their sums is zero, and
are left out.  Of second order, b X X^T X and c (X X^T)^2 X leave at most 3 |b| s +
10 |c| s^3, below 56 |error| of the first a step for s up to 1.22 and the
coefficients here: less than a ninth while an error's singular values are below
2^-9, a factor of 1.7 over five steps; the bound is taken twice."""
import torch

from ortho_ref import U32, _product


def _live(m):
    m = m[m.abs().amax(1) > 0]
    return m[:, m.abs().amax(0) > 0]


def bound_of(m, coefficients, steps, eps):
    """Bound of |error| (2-norm) of one matrix's float32 update after `steps` steps, before the rounding of the result."""
    a, b, c = coefficients
    m = m.double()
    x = _live(m.t() if m.shape[0] > m.shape[1] else m)
    x = x / (float(x.norm()) + eps)
    sizes, own = [], []
    v = torch.cat((torch.linalg.svdvals(x), torch.zeros(1, dtype=torch.float64)))
    own.append((0.0, 2 * U32 * float(x.norm())))
    for _ in range(steps):
        sizes.append(v)
        g, dg = _product(x, x.t(), True)
        gg, dgg = _product(g, g, True)
        p = b * g + c * gg
        dp = abs(b) * dg + abs(c) * (dgg + 2 * float(v[0]) ** 2 * dg) + (2.0 ** -22 + 3 * U32) * float(p.norm()) + \
            4 * U32 * (abs(b) * float(g.norm()) + abs(c) * float(gg.norm()))
        px, dpx = _product(p, x, True)
        own.append((dp, dpx + 4 * U32 * (abs(a) * float(x.norm()) + float(px.norm()))))
        x, v = a * x + px, v * (a + v ** 2 * (b + c * v ** 2))
        assert float(v.abs().max()) <= 1.22 and 3 * abs(b) * 1.22 + 10 * abs(c) * 1.22 ** 3 <= 56, "second order"
    total, f, g = own[-1][0] * float(sizes[-1].abs().max()) + own[-1][1], 1.0, 1.0
    # backwards, with the factors of the steps behind each step's own errors
    for k in range(steps - 1, -1, -1):
        y = sizes[k][:, None]
        z = sizes[k][None, :]
        even, odd = a + b * (y * y + z * z) + c * (y ** 4 + (y * z) ** 2 + z ** 4), b * y * z + c * (y ** 3 * z + y * z ** 3)
        f, g = f * (even + odd), g * (even - odd)
        f[-1, -1] = g[-1, -1] = 0.0   # (no pair: only rows or only columns are left over)
        spread = float(torch.maximum(f.abs(), g.abs()).max())
        inside = 0.0
        if k > 0:
            # (D X is made from the step's X before it, the factors take what comes out)
            before = sizes[k - 1]
            inside = float((0.5 * (f * f + g * g) * (before[:, None] ** 2 + before[None, :] ** 2)).sqrt().max())
        total += own[k][0] * inside + own[k][1] * spread
    return 2 * total
