"""Values in float64 with a first-order bound of how far the same arithmetic in 32 bits may be off, element by element.

Every operation adds the roundings of its own result: 2^-24 of it (a sum of n terms: n + 16 of them, of the sum of its terms' sizes, more than any order of
adding needs) and passes on what its operands are off by.  `rounded` adds the rounding to a type of fewer bits, half a step: 2^-8 in bf16."""
import torch

E32 = 2.0 ** -24
TINY = 1e-35      # relative errors mean nothing below 2^-126


def unit(dt):
    return {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 0.0}[dt]


class Ball:
    def __init__(self, v, e=None):
        self.v = v.double() if isinstance(v, torch.Tensor) else v
        self.e = torch.zeros_like(self.v) if e is None else e

    @staticmethod
    def of(x):
        if isinstance(x, Ball):
            return x
        x = torch.as_tensor(x, dtype=torch.float64, device="cuda")
        return Ball(x, E32 * x.abs())      # scales and eps are floats in the calls: 0.8 becomes 0.8 (1 + 2^-26.4), which moves 0.8 h by as much

    def _made(self, v, e):
        return Ball(v, e + E32 * v.abs())

    def __add__(self, o):
        o = Ball.of(o)
        return self._made(self.v + o.v, self.e + o.e)

    def __sub__(self, o):
        o = Ball.of(o)
        return self._made(self.v - o.v, self.e + o.e)

    def __mul__(self, o):
        o = Ball.of(o)
        return self._made(self.v * o.v, self.e * o.v.abs() + o.e * self.v.abs() + self.e * o.e)

    __radd__, __rmul__ = __add__, __mul__

    def __matmul__(self, o):
        k = self.v.shape[-1]
        size = self.v.abs() @ o.v.abs()
        return Ball(self.v @ o.v, self.e @ o.v.abs() + self.v.abs() @ o.e + self.e @ o.e + E32 * (k + 16) * size)

    def t(self):
        return Ball(self.v.t(), self.e.t())

    def sum(self, dim, keepdim=False):
        n = self.v.shape[dim]
        return Ball(self.v.sum(dim, keepdim=keepdim), self.e.sum(dim, keepdim=keepdim) + E32 * (n + 16) * self.v.abs().sum(dim, keepdim=keepdim))

    def mean(self):
        n = self.v.shape[-1]
        s = self.sum(-1, True)
        return self._made(s.v / n, s.e / n + E32 * s.v.abs() / n)

    def rsqrt(self):
        """Of values above 0, with the roundings of a root and a division."""
        v = self.v.rsqrt()
        return Ball(v, 0.5 * self.e * v ** 3 + 4 * E32 * v)

    def rounded(self, dt):
        return Ball(self.v, self.e + unit(dt) * (self.v.abs() + self.e))


def within(name, got, want, dt=None):
    """got (rounded once more to dt, its own type) against a Ball: everything finite, in its bounds."""
    want = want.rounded(dt or got.dtype)
    got = got.double()
    assert got.shape == want.v.shape, (name, got.shape, want.v.shape)
    assert got.isfinite().all() or not want.v.isfinite().all(), f"{name}: not finite"
    over = (got - want.v).abs() - want.e - TINY
    assert over.numel() == 0 or over.max() <= 0, f"{name}: {over.max().item():.3g} beyond its bound"
