"""64-bit forms of the 8-bit layer's operators and what their tests share.  The formulas are written out from
their definitions in NumPy; nothing here calls the library."""
import math

import numpy as np

TYPES = ("f32", "f16", "bf16")
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
#: half a unit in the last place relative to the value, and the smallest step of the type's subnormal numbers / 2
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
#: Relative error of the binary32 arithmetic between an exact sum and the stored value, against the magnitudes
#: that enter it: the conversion, two scalings, the bias and the final product are rounded (5 * 2^-24), the
#: exponential of an argument up to |x| contributes 2 + 1.2 |x| units (|x| <= 30 here), the quotient 2: below 2^-18.
ARITH = 2.0 ** -18


def torch_type(kind):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[kind]


def size(kind):
    return 4 if kind == "f32" else 2


def erf(x):
    return np.vectorize(math.erf, otypes=[np.float64])(x)


def act(x, kind):
    if kind == "relu":
        return np.maximum(x, 0)
    if kind == "gelu":
        return 0.5 * x * (1 + erf(x / math.sqrt(2)))
    if kind == "gelu_tanh":
        return 0.5 * x * (1 + np.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    if kind == "silu":
        return x / (1 + np.exp(-x))
    return x


def slope(x, kind):
    if kind == "relu":
        return (x > 0).astype(np.float64)
    if kind == "gelu":
        return 0.5 * (1 + erf(x / math.sqrt(2))) + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = np.tanh(c * (x + 0.044715 * x ** 3))
        return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * c * (1 + 3 * 0.044715 * x * x)
    if kind == "silu":
        e = 1 / (1 + np.exp(-x))
        return e * (1 + x * (1 - e))
    return np.ones_like(x)


def rounded(x, kind):
    """x (float64) rounded to the type, as float64 -- for inputs that have to be representable."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch_type(kind)).double().numpy()


class Matrix:
    """A rows x cols matrix on the GPU inside a larger poisoned buffer: pitch `ld` elements, base `shift` elements
    from a 256-byte boundary.  `unchanged()` says whether everything outside the matrix still holds the poison."""

    def __init__(self, rows, cols, kind, ld=None, shift=0, values=None):
        import torch
        self.rows, self.cols, self.ld, self.shift = rows, cols, ld or cols, shift
        dt = torch.int8 if kind == "s8" else (torch.uint8 if kind == "u8" else torch_type(kind))
        self.n = max(rows, 1) * self.ld + shift + 64
        self.buf = torch.full((self.n,), 77, dtype=dt, device="cuda")
        self.view = self.buf[shift:shift + max(rows, 1) * self.ld].view(max(rows, 1), self.ld)[:rows, :cols]
        if values is not None:
            self.view.copy_(torch.from_numpy(np.ascontiguousarray(values)).to(dt))

    @property
    def ptr(self):
        return self.buf.data_ptr() + self.shift * self.buf.element_size()

    def get(self):
        return self.view.double().cpu().numpy()

    def unchanged(self):
        import torch
        mask = torch.ones(self.n, dtype=torch.bool, device="cuda")
        mask[self.shift:self.shift + max(self.rows, 1) * self.ld].view(max(self.rows, 1), self.ld)[:self.rows, :self.cols] = False
        return bool((self.buf[mask] == 77).all())


def vector(values):
    import torch
    return None if values is None else torch.from_numpy(np.asarray(values, dtype=np.float32)).cuda()


def codes(rng, rows, cols, unsigned=False):
    return rng.integers(0, 256, (rows, cols)).astype(np.uint8) if unsigned else rng.integers(-128, 128, (rows, cols)).astype(np.int8)


def scales(rng, n, mean):
    return ((rng.random(n) + 0.5) * mean).astype(np.float32)


def sums(a, b):
    """The exact integer sums A B^T as float64 (every partial sum is below 2^53)."""
    return a.astype(np.float64) @ b.astype(np.float64).T


def check(got, want, magnitude, kind, what=""):
    tol = ROUND[kind] * np.abs(want) * (1 + ARITH) + TINY[kind] + ARITH * magnitude
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        i = tuple(int(v) for v in np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d off; first at %s: got %r want %r tol %r" % (
            what, int(bad.sum()), bad.size, i, got[i], want[i], tol[i]))
