"""Plain fp64 forms of the operators on the full cache, in numpy, and the tensors their tests build."""
from __future__ import annotations

import numpy as np


def rotate(x, pos, freq, layout=0, amplitude=1.0, transpose=False):
    """x fp64 [n, heads, d], pos [n]; layout 0: pairs (j, j + r/2), 1: pairs (2j, 2j + 1)."""
    h = len(freq)
    angle = np.asarray(pos, dtype=np.float64)[:, None] * np.asarray(freq, dtype=np.float64)
    turn = amplitude * np.exp((-1j if transpose else 1j) * angle)[:, None, :]
    first, second = (slice(0, h), slice(h, 2 * h)) if layout == 0 else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
    y = np.array(x, dtype=np.float64)
    z = (y[..., first] + 1j * y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


# A rotated element's error: its angle is rounded to fp32 as a fraction of a turn in [-1/2, 1/2], off by 2^-26 turns = 9.4e-8; cosine
# and sine by at most 2 units of 2^-24 each, their product with the amplitude, the two products and the sum by 2^-24 each:
# (9.4e-8 + 5 * 2^-24) * amplitude * (|a| + |b|) < 4e-7 * ...; then half a step of the element type, eps / 2 relative.
def rotation_bound(x, want, freq, layout, amplitude, half_step):
    h = len(freq)
    first, second = (slice(0, h), slice(h, 2 * h)) if layout == 0 else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
    mag = np.zeros_like(want)
    a = np.abs(x)
    mag[..., first] = mag[..., second] = a[..., first] + a[..., second]
    err = 4e-7 * abs(amplitude) * mag
    return err + half_step * (np.abs(want) + err)


def half_step(dtype):
    import torch

    return torch.finfo(dtype).eps / 2


def f64(t):
    return t.detach().double().cpu().numpy()


def frequencies(r, base=500000.0):
    return [base ** (-2.0 * j / r) for j in range(r // 2)]


def attention(q, K, V, S=0, W=0):
    """One problem: q [Hq, d], K, V [Hkv, len, d] fp64.  Returns out [Hq, d], lse [Hq]; W > 0: only the first S and the last W tokens."""
    Hq, d = q.shape
    Hkv, n, _ = K.shape
    out, lse = np.zeros((Hq, d)), np.full(Hq, -np.inf)
    t = np.arange(n)
    if W:
        t = t[(t < S) | (t >= n - W)]
    if not len(t):
        return out, lse
    for h in range(Hq):
        k, v = K[h // (Hq // Hkv)][t], V[h // (Hq // Hkv)][t]
        x = k @ q[h] / np.sqrt(d)
        m = x.max()
        w = np.exp(x - m)
        out[h], lse[h] = w @ v / w.sum(), m + np.log(w.sum())
    return out, lse


class Pages:
    """A paged cache on the GPU: pools in head- or token-major pages, a shuffled block table, the problems' dense views."""

    def __init__(self, gen, P, Hkv, d, cap, page, dtype, order="heads", spare=3, fill=None):
        import torch

        self.page, self.per = page, -(-cap // page)
        n = P * self.per + spare
        shape = (n, Hkv, page, d) if order == "heads" else (n, page, Hkv, d)
        self.K, self.V = (torch.randn(shape, generator=gen, device="cuda").to(dtype) if fill is None else torch.full(shape, fill, device="cuda", dtype=dtype)
                          for _ in range(2))
        if order == "tokens":
            self.K, self.V = self.K.transpose(1, 2), self.V.transpose(1, 2)
        self.table = torch.randperm(n, generator=gen, device="cuda")[: P * self.per].to(torch.int32).reshape(P, self.per)

    def dense(self, x):
        """[P, Hkv, per * page, d] fp64 of a pool."""
        got = x[self.table.long()]  # [P, per, Hkv, page, d]
        P, per, Hkv, page, d = got.shape
        return f64(got.transpose(1, 2).reshape(P, Hkv, per * page, d))
