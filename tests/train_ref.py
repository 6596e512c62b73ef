"""Training of 16-bit experts in 64 bits, with bounds of how far results in 32 and 16 bits may be away.

Bounds count: eps / 2 of the type for each rounding (2^-11 for fp16, at least half its smallest step, 2^-25), (n + 8) 2^-23 of the sum of magnitudes for a sum of n products
in 32 bits, and (8 + |a|) 2^-22 for the exponential, the quotient and the products around it."""
import torch

HALF, TINY = 2.0 ** -11, 2.0 ** -25


def sums(n):
    return (n + 8) * 2.0 ** -23


def rounded(v, err):
    """Error of a value with error ``err`` once it is rounded to fp16."""
    return err + HALF * (v.abs() + err) + TINY


class Ref:
    """x [T,d], w1, w3 [E,f,d], w2 [E,d,f], all fp16; groups: for each expert (pairs, in grouped order); gates [T k] in 64 bits."""

    def __init__(self, x, w1, w3, w2, groups, gates, k):
        self.x, self.w = x.double(), [(a.double(), b.double(), c.double()) for a, b, c in zip(w1, w3, w2)]
        self.groups, self.g, self.k = groups, gates, k

    def forward(self):
        """Rows a, u in grouped order and out, each as (value, bound)."""
        T, d = self.x.shape
        out, e_out = torch.zeros_like(self.x), torch.zeros_like(self.x)
        kept = []
        for (w1, w3, w2), p in zip(self.w, self.groups):
            x, g = self.x[p // self.k], self.g[p][:, None]
            a, u = x @ w1.t(), x @ w3.t()
            ea, eu = sums(d) * (x.abs() @ w1.abs().t()), sums(d) * (x.abs() @ w3.abs().t())
            kept.append((a, u, rounded(a, ea), rounded(u, eu)))
            z = a * torch.sigmoid(a)
            h = z * u
            eh = rounded(h, 1.1 * ea * (u.abs() + eu) + z.abs() * eu + (8 + a.abs()) * 2.0 ** -22 * h.abs())
            y = h @ w2.t()
            ey = eh @ w2.abs().t() + sums(h.shape[1]) * (h.abs() @ w2.abs().t())
            out.index_add_(0, p // self.k, g * y)
            e_out.index_add_(0, p // self.k, g.abs() * ey + 4 * 2.0 ** -23 * (g * y).abs())
        a, u, ea, eu = (torch.cat(v) for v in zip(*kept))
        return (a, ea), (u, eu), (out, rounded(out, e_out))

    def backward(self, a, u, d_out):
        """From kept rows a, u (fp16): dict of (value, bound): d_x, d_gate [T k], w1, w3, w2 (lists over the experts); none of them rounded at the end."""
        T, d = self.x.shape
        zero = lambda: (torch.zeros_like(self.x), torch.zeros_like(self.x))  # noqa: E731
        d_x, e_x = zero()
        d_g, e_g = torch.zeros_like(self.g), torch.zeros_like(self.g)
        r = dict(w1=[], w3=[], w2=[])
        at = 0
        for (w1, w3, w2), p in zip(self.w, self.groups):
            n, f = len(p), w1.shape[0]
            A, U = a[at: at + n].double(), u[at: at + n].double()
            at += n
            t = p // self.k
            x, do, g = self.x[t], d_out.double()[t], self.g[p][:, None]
            s = torch.sigmoid(A)
            z, slope, near = A * s, s * (1 + A * (1 - s)), (8 + A.abs()) * 2.0 ** -22
            h = z * U
            q = do @ w2
            eq = sums(d) * (do.abs() @ w2.abs())
            d_g[p] = (q * h).sum(1)
            e_g[p] = (eq * h.abs() + (q * h).abs() * (near + sums(f))).sum(1)
            da, du, gh = g * q * U * slope, g * q * z, g * h
            eda = rounded(da, 1.1 * (g * U).abs() * eq + near * (g * q * U).abs())
            edu = rounded(du, (g * z).abs() * eq + near * du.abs())
            egh = rounded(gh, near * gh.abs())
            d_x.index_add_(0, t, da @ w1 + du @ w3)
            e_x.index_add_(0, t, (eda + sums(2 * f) * da.abs()) @ w1.abs() + (edu + sums(2 * f) * du.abs()) @ w3.abs())
            r["w1"].append((da.t() @ x, (eda + sums(n) * da.abs()).t() @ x.abs()))
            r["w3"].append((du.t() @ x, (edu + sums(n) * du.abs()).t() @ x.abs()))
            r["w2"].append((do.t() @ gh, do.abs().t() @ (egh + sums(n) * gh.abs())))
        e_x += 8 * 2.0 ** -23 * d_x.abs()
        return dict(r, d_x=(d_x, e_x), d_gate=(d_g, e_g))


def assert_within(got, value, bound, what, half=False):
    """Every element within its bound (half: and the rounding of the result to fp16), and all of them together within 2e-3."""
    got = got.double().reshape(value.shape)
    if half:
        bound = rounded(value, bound)
    assert torch.isfinite(got).all(), what
    over = (got - value).abs() - bound * (1 + 1e-6) - 1e-30
    assert float(over.max()) <= 0, f"{what}: {float(over.max()):.3g} past its bound, value {float(value.reshape(-1)[over.argmax()]):.3g}"
    norm = float(value.norm())
    if norm > 0 and float(value.abs().max()) > 1e-3:
        off = float((got - value).norm()) / norm
        assert off <= 2e-3, f"{what}: {off:.3g} off"
