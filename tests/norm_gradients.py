"""The gradients of a norm before and after a block, from the formulas in 64 bits, and
how far fp32 arithmetic may be from them.

u = 2^-24.  A row's sum of D terms is taken by threads of 8 to 32 terms each, then over
up to 64 lanes by halves and up to 16 waves: 32 + 6 + 16 roundings deep at most, with 10
for what is formed from it C = 64 u, relative to the sum of the terms' magnitudes.

The mean m is off by d, |d| <= C mean|x|, the same for all elements of a row.  The
centred squares' mean is then off by d^2 alone, since the centred elements' sum is 0:
r = 1 / sqrt(...) is off by rho = C + (d r)^2, relative, however large the mean, and
N(x) = xh by E = r d + (rho + C) |xh|.
  mean(u xh): the terms' roundings C mean(|u| (|xh| + r d)), the mean's error r d |mean(u)|
  and r's, rho |mean(u xh)|: A.
  g = r (u - mean(u) - xh mean(u xh)): r (C (|u| + mean|u| + |xh mean(u xh)|) + E |mean(u xh)|
  + |xh| A) + rho |g|, and where u is off by du, r (du + mean(du) + |xh| mean(du |xh|)).
Sums over tokens are at most 64 rows and 64 partial sums deep with the terms' own errors:
2 C.  A gate's factor and its slope are 2^-20 off (2^-16 in 16 bits) of their terms' sizes."""
import torch

C = 64 * 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}


def mean(x):
    return x.mean(1, keepdim=True)


class Normed:
    """N(x) of a row, what its gradient needs, and their errors.  `wrong` names a mistake."""

    def __init__(self, x, kind, eps, wrong=""):
        x, self.layer, self.wrong = x.double(), kind == "layer", wrong
        self.d = C * mean(x.abs()) if self.layer else torch.zeros_like(x[:, :1])
        c = x - mean(x) if self.layer and wrong != "uncentred" else x
        self.r = (mean(c.square()) + eps).rsqrt()
        self.xh = c * self.r
        self.rho = C + (self.d * self.r) ** 2
        self.off = self.r * self.d + (self.rho + C) * self.xh.abs()

    def back(self, u, du):
        """The gradient of x from u, that of N(x), which is du off; its error."""
        m = mean(u) if self.layer and self.wrong != "no mean" else torch.zeros_like(self.r)
        along = mean(u * self.xh)
        part = along * 0 if self.wrong == "no part along" else along
        g = self.r * (u - m - self.xh * part)
        xh = self.xh.abs()
        a = C * mean(u.abs() * (xh + self.r * self.d)) + self.r * self.d * mean(u).abs() + self.rho * along.abs()
        err = self.r * (C * (u.abs() + mean(u.abs()) + xh * along.abs()) + self.off * along.abs() + xh * a
                        + du + mean(du) + xh * mean(du * xh)) + self.rho * g.abs()
        return g, err


def gate_of(g, act, dtype):
    """a(g), its slope and both errors."""
    if g is None:
        return (torch.tensor(v, dtype=torch.float64) for v in (1.0, 0.0, 0.0, 0.0))
    g = g.double()
    if act == "none":
        return g, torch.ones_like(g), torch.zeros_like(g), torch.zeros_like(g)
    s = torch.sigmoid(g)
    u = 2.0 ** (-20 if dtype == torch.float32 else -16)
    if act == "sigmoid":
        return s, s * (1 - s), u * s, u * s * (1 - s)
    return g * s, s * (1 + g * (1 - s)), u * (g * s).abs(), u * s * (1 + g.abs() * (1 - s))


def gradients(s, kind, eps, act, scale, form, wrong=""):
    """{name: (gradient, error before its rounding)} of `form` for s's out, b, dy, dout, gate, weight and next."""
    got, d = {}, s["dout"].double()
    ed = torch.zeros_like(d)
    if form != "after":
        n, dy, w = Normed(s["out"], kind, eps, wrong), s["dy"].double(), s["next"].double()
        g, eg = n.back(dy * w, 2.0 ** -24 * (dy * w).abs())
        d, ed = d + g, eg + C * (d.abs() + g.abs())
        got["dh"] = d, ed
        terms = dy * n.xh
        got["dnext"] = terms.sum(0), 2 * C * terms.abs().sum(0) + (dy.abs() * n.off).sum(0)
    if form != "before":
        n, w = Normed(s["b"], kind, eps, wrong), s["weight"].double()
        gate = s["gate"]
        a, slope, ea, es = gate_of(gate, act, None if gate is None else gate.dtype)
        e, ee = scale * d, abs(scale) * ed + C * (scale * d).abs()
        ev = w.abs() * (ee * a.abs() + e.abs() * ea) + C * (w * e * a).abs()
        got["db"] = n.back(w * e * a, ev)
        terms = e * a * n.xh
        got["dweight"] = terms.sum(0), 2 * C * terms.abs().sum(0) + ((ee * a.abs() + e.abs() * ea) * n.xh.abs() + (e * a).abs() * n.off).sum(0)
        if gate is not None:
            terms = e * slope * w * n.xh
            errs = w.abs() * ((ee * slope.abs() + e.abs() * es) * n.xh.abs() + (e * slope).abs() * n.off) + C * terms.abs()
            got["dgate"] = (terms, errs) if gate.dim() == 2 else (terms.sum(0), 2 * C * terms.abs().sum(0) + errs.sum(0))
    return got


def excess(got, want, err, dtype=None):
    """|got - want| over what it may be, element by element; terms of second order double it."""
    dtype = got.dtype if dtype is None else dtype
    return (got.double() - want).abs() / (2 * (err + U[dtype] * want.abs()) + TINY[dtype])


def inputs(n, dim, dtype, residual, gate, device, seed, offset):
    """Rows of h (given as `out`) and b `offset` away from 0, the gradients around 0."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device=device)  # noqa: E731
    s = {"out": (3 * normal(n, dim) + offset).to(residual), "b": (1.5 * normal(n, dim) + offset).to(dtype),
         "dy": (0.5 * normal(n, dim)).to(dtype), "dout": (0.5 * normal(n, dim)).to(residual),
         "weight": 1 + 0.3 * normal(dim), "next": 1 + 0.3 * normal(dim), "gate": None}
    if gate == "vector":
        s["gate"] = 3 * normal(dim)
    elif gate == "matrix":
        s["gate"] = (3 * normal(n, dim)).to(dtype)
    return s


# n, dim, kind, offset
CASES = [(9, 1000, "layer", 300.0), (3, 16384, "layer", 300.0), (1, 16384, "layer", 0.0), (4, 9216, "layer", 30.0), (3, 10241, "rms", 0.0),
         (40, 40, "layer", 300.0), (40, 5, "layer", 30.0), (9, 1001, "rms", 300.0), (6, 8192, "layer", 300.0)]
EPS, SCALE = 1e-5, 0.75
