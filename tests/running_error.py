"""Values in 64 bits beside a bound of how far off a computation in 32 bits may be: each operation hands on its operands' errors and adds
its own rounding, u = 2^-24 of the result (a chain of n additions: n u of the sum of the absolute values, in whatever order).  And tensors on the GPU whose surroundings are NaN."""
import math

import torch

U32 = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


class Run:
    def __init__(self, v, e=0.0):
        self.v = torch.as_tensor(v).double()
        self.e = torch.as_tensor(e).double().expand(self.v.shape)

    @staticmethod
    def of(x):
        return x if isinstance(x, Run) else Run(x)

    def __add__(self, o):
        o = Run.of(o)
        v = self.v + o.v
        return Run(v, self.e + o.e + U32 * (v.abs() + self.e + o.e))

    def __neg__(self):
        return Run(-self.v, self.e)

    def __sub__(self, o):
        return self + -Run.of(o)

    def __mul__(self, o):
        o = Run.of(o)
        v = self.v * o.v
        e = self.v.abs() * o.e + self.e * o.v.abs() + self.e * o.e
        return Run(v, e + U32 * (v.abs() + e))

    def __getitem__(self, k):
        return Run(self.v[k], self.e[k])

    def view(self, *s):
        return Run(self.v.reshape(*s), self.e.reshape(*s))

    def sum(self, dim, chain, keepdim=False):
        return Run(self.v.sum(dim, keepdim=keepdim), (self.e + chain * U32 * (self.v.abs() + self.e)).sum(dim, keepdim=keepdim))

    def mean(self, chain):
        """Over the last axis; the division as a product with a rounded 1 / n."""
        n = self.v.shape[-1]
        s = self.sum(-1, chain, keepdim=True)
        v = s.v / n
        return Run(v, s.e / n + 3 * U32 * v.abs())

    def rsqrt(self):
        """1 / sqrt(v), both to one unit in the last place or better."""
        v = self.v ** -0.5
        return Run(v, v * (0.5 * self.e / self.v + 6 * U32))

    def sigmoid(self):
        """1 / (1 + 2^(-v log2 e)): the exponent's rounding shows as 2 |v| u of the exponential, which as that function and the reciprocal
        is good to a unit in the last place (2 u).  The slope is at most 1/4, and of either tail at most the value itself."""
        s = torch.sigmoid(self.v)
        return Run(s, s * (1 - s) * (1.1 * self.e + U32 * (2 * self.v.abs() + 3)) + 4 * U32 * s + 1e-38)

    def silu(self):
        return self * self.sigmoid()

    def silu_slope(self):
        """s (1 + v (1 - s)); the error that v brings along goes by the slope's own, at most 1/2."""
        s = Run(self.v).sigmoid()
        r = s * (Run(1.0) + Run(self.v) * (Run(1.0) - s))
        return Run(r.v, r.e + 0.5 * self.e)


def within(got, ref, io="f32"):
    """got (rounded once more where io is bf16) lies within ref's bound."""
    got = got.detach().double().cpu()
    assert got.shape == ref.v.shape, (got.shape, ref.v.shape)
    bound = ref.e + (HALF_STEP[io] * (ref.v.abs() + ref.e) if io != "f32" else 0.0) + 1e-37
    off = (got - ref.v).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), "%d of %d beyond the bound, worst %.3g times it" % (
        int(bad.sum()), bad.numel(), float((off / bound)[bad].nan_to_num(nan=math.inf).max()))


def scan(a, a_off, u, u_off, h0):
    """States before every step of h = a h + u over axis 1 and the one after the last, however the steps are grouped: each step of either
    grouping rounds its product, its sum and the product of its factors, all of them at most the scan of the absolute values."""
    before, off, size = [], [], []
    h, e, s = h0.double(), torch.zeros_like(h0).double(), h0.double().abs()
    for t in range(a.shape[1]):
        before.append(h), off.append(e), size.append(s)
        grown = a[:, t] * s + u[:, t].abs()
        e = (a[:, t] + a_off[:, t]) * e + a_off[:, t] * s + u_off[:, t] + 4 * U32 * grown
        h, s = a[:, t] * h + u[:, t], grown
    both = lambda v: torch.stack(v, 1) if v else torch.zeros(a.shape).double()  # noqa: E731
    return Run(both(before), both(off)), both(size), Run(h, e)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, scale=1.0, io="f32"):
    return (scale * torch.randn(*shape, generator=g)).to(TYPES[io])


def wide(t, extra, lead=0):
    """t on the GPU as a column slice of a buffer that is wider by `extra`, `lead` columns in; what is around it is NaN."""
    buf = torch.full(t.shape[:-1] + (t.shape[-1] + extra,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[..., lead:lead + t.shape[-1]]
    v.copy_(t)
    return v


def blank(shape, io, extra=0, lead=0):
    return wide(torch.full(shape, float("nan"), dtype=TYPES[io]), extra, lead)


def nans(*shape):
    return torch.full(shape, float("nan"), device="cuda")


def workspace(n):
    return torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")


def cuda(t):
    return None if t is None else t.cuda()
