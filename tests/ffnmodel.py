"""The experts' products in 64 bits, with how far a kernel that rounds as
include/topoep_ffn.h says may be off, element by element.

u is half a step of the 16-bit type.  A sum of n products in 32 bits is off by at
most n 2^-24 of the sum of their magnitudes.  sigmoid(z) is off by (2 |z| + 8)
2^-24 of itself (the exponential's argument is rounded to 32 bits).  Bounds
are first order; FIRST covers what is left of higher orders."""
import torch

E32 = 2.0 ** -24
FIRST = 1.02
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounded(value, off, dtype):
    """The bound of a value after one rounding to dtype."""
    return FIRST * (off + half_step(dtype) * (value.abs() + off)) + SMALLEST[dtype]


class Block:
    """One block's forward pass for rows x with weights w, in 64 bits, and bounds."""

    def __init__(self, x, w, up, down, dtype):
        self.dtype, self.x, self.w, self.up, self.down = dtype, x.double(), w.double()[:, None], up.double(), down.double()
        x, up, down, w = self.x, self.up, self.down, self.w
        H, I = x.shape[1], down.shape[1]
        self.a, mag = x @ up.t(), x.abs() @ up.abs().t()
        self.g, self.u = self.a[:, :I], self.a[:, I:]
        off = H * E32 * mag
        self.eg, self.eu = off[:, :I], off[:, I:]
        self.s = torch.sigmoid(self.g)
        self.es = (2 * self.g.abs() + 8) * E32
        self.act = self.g * self.s
        self.h0 = self.act * self.u
        self.eh0 = (1.1 * self.eg * (self.u.abs() + self.eu) + self.act.abs() * self.eu
                    + self.h0.abs() * (self.es + 4 * E32) + 1e-30)
        self.h = w * self.h0
        self.eh = rounded(self.h, w.abs() * self.eh0, dtype)
        self.y = self.h @ down.t()
        self.ey = self.eh @ down.abs().t() + I * E32 * ((self.h.abs() + self.eh) @ down.abs().t())

    def back(self, dy):
        """(value, bound) before the last rounding of dx, up, down and the rows' weights."""
        x, up, down, w, dy = self.x, self.up, self.down, self.w, dy.double()
        n, H, I = x.shape[0], x.shape[1], down.shape[1]
        dh, edh = dy @ down, H * E32 * (dy.abs() @ down.abs())
        slope = self.s * (1.0 + self.g * (1.0 - self.s))
        dg, du = w * dh * self.u * slope, w * dh * self.act
        more = (2 * self.es + 12 * E32)
        edg = w.abs() * (edh * (self.u * slope).abs() + dh.abs() * (1.1 * self.eu + 0.5 * self.u.abs() * self.eg)
                         + (dh * self.u).abs() * more * (1.0 + self.g.abs()) * self.s) + 1e-30
        edu = w.abs() * (edh * self.act.abs() + dh.abs() * (1.1 * self.eg + self.act.abs() * more)) + 1e-30
        da = torch.cat([dg, du], 1)
        eda = rounded(da, torch.cat([edg, edu], 1), self.dtype)
        mda = da.abs() + eda
        dx = da @ up
        edx = eda @ up.abs() + 2 * I * E32 * (mda @ up.abs())
        dup = da.t() @ x
        edup = eda.t() @ x.abs() + n * E32 * (mda.t() @ x.abs())
        ddown = dy.t() @ self.h
        eddown = dy.abs().t() @ self.eh + n * E32 * (dy.abs().t() @ (self.h.abs() + self.eh))
        dw = (dh * self.h0).sum(1)
        edw = (edh * self.h0.abs() + dh.abs() * self.eh0).sum(1) + (I + 8) * E32 * (dh * self.h0).abs().sum(1)
        return {"x": (dx, edx), "up": (dup, edup), "down": (ddown, eddown), "weights": (dw, FIRST * edw)}


def layer(x, ids, weights, up, down, slot=None, dout=None, dtype=None):
    """A routed layer in 64 bits on the CPU: {name: (value, bound)} of out and, with dout, the gradients."""
    x, ids, weights, up, down = (t.detach().cpu() for t in (x, ids, weights, up, down))
    dtype = dtype or x.dtype
    T, k = ids.shape
    L = up.shape[0]
    of = ids.long()
    slot = torch.arange(L) if slot is None else slot.detach().cpu().long()
    of = torch.where((of >= 0) & (of < len(slot)), slot[of.clamp(0, len(slot) - 1)], -1)
    zero = lambda *s: [torch.zeros(s, dtype=torch.float64), torch.zeros(s, dtype=torch.float64)]  # noqa: E731
    got = {"out": zero(*x.shape), "mag": zero(*x.shape)}
    if dout is not None:
        dout = dout.detach().cpu()
        got.update(x=zero(*x.shape), weights=zero(T, k), up=zero(*up.shape), down=zero(*down.shape))
    for e in range(L):
        t, j = (of == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        b = Block(x[t], weights[t, j], up[e], down[e], dtype)
        for i, v in enumerate((b.y, b.ey + k * E32 * b.y.abs())):
            got["out"][i].index_add_(0, t, v)
        if dout is not None:
            back = b.back(dout[t])
            for i in range(2):
                extra = back["x"][i] + (k * E32 * back["x"][0].abs() if i else 0)
                got["x"][i].index_add_(0, t, extra)
                got["weights"][i][t, j] = back["weights"][i]
                got["up"][i][e], got["down"][i][e] = back["up"][i], back["down"][i]
    got.pop("mag")
    return {n: (v, e if n == "weights" else rounded(v, e, dtype)) for n, (v, e) in got.items()}


def dense(x, up, down, dout=None):
    ids = torch.zeros((x.shape[0], 1), dtype=torch.int32)
    ones = torch.ones((x.shape[0], 1))
    got = layer(x, ids, ones, up[None], down[None], None, dout)
    got.pop("weights", None)
    return {n: (v[0], e[0]) if n in ("up", "down") else (v, e) for n, (v, e) in got.items()}


def within(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert bool(torch.isfinite(got).all()), what
    off = (got - want).abs()
    over = off > bound
    assert not over.any(), "%s: %d values off, %.3f times their bound" % (what, over.sum(), (off / bound)[over].max())
