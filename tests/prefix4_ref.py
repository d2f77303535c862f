"""A prefix in 4 bits, from its definition, for the tests: rounding to 4 bits, what stored rows stand for, rows
turned by positions of several axes."""
from __future__ import annotations

import numpy as np
import torch

SIZES = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def pack64(y):
    """y [..., d] (float64 on the host): (elements [..., d / 2], scales [..., d / 32]), uint8.  Each element by its
    distance from every size."""
    y = y.double().cpu().unflatten(-1, (-1, 32))
    most = y.abs().amax(-1, keepdim=True)  # (NaN where there is one)
    f, k = np.frexp(most.numpy())  # most = f 2^k, f in [0.5, 1)
    e = np.clip(np.where(most.numpy() > 0, k - 3 + (f >= 0.875), -125), -125, 125)
    unit = torch.from_numpy(np.ldexp(1.0, e))
    far = ((y.abs() / unit)[..., None] - SIZES).abs()  # [..., 32, 8]
    far[..., 1::2] *= 1 + 2.0 ** -50  # (of two equally near the even code)
    code = far.argmin(-1).to(torch.uint8)
    code |= torch.signbit(y).to(torch.uint8) << 3
    # (past fp32 counts as infinite)
    bad = ~(most < 2.0 ** 128)
    code = torch.where(bad, torch.zeros_like(code), code).flatten(-2)
    scales = torch.where(bad, torch.full_like(bad, 255, dtype=torch.uint8), torch.from_numpy(e + 127).to(torch.uint8))
    return code[..., 0::2] | (code[..., 1::2] << 4), scales.squeeze(-1)


def values64(elements, scales):
    """What 4-bit rows stand for: float64 [..., d] on the host."""
    elements, scales = elements.cpu().long(), scales.cpu().double()
    code = torch.stack([elements % 16, elements // 16], -1).flatten(-2)
    unit = torch.where(scales == 255, torch.nan, torch.exp2(scales - 127))
    return SIZES[code % 8] * (1 - 2 * (code // 8)) * unit.repeat_interleave(32, -1)


def turn_axes(x, pos, freq, axis, interleaved):
    """x [..., n, H, d], pos [n][axes], axis [r / 2]: float64, pair by pair."""
    x, pos, r = x.double().cpu(), np.asarray(pos, np.float64), 2 * len(freq)
    f = np.asarray(freq.double().cpu())
    y = x.clone()
    for i in range(r // 2):
        a = torch.from_numpy(pos[:, int(axis[i])] * f[i])[:, None]
        c, s = torch.cos(a), torch.sin(a)
        i0, i1 = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        y[..., i0] = x[..., i0] * c - x[..., i1] * s
        y[..., i1] = x[..., i1] * c + x[..., i0] * s
    return y


def random_rows(gen, shape):
    """Rows in 4 bits whose blocks have units from 2^-4 to 2^1."""
    y = torch.randn(shape, generator=gen).double()
    blocks = y.unflatten(-1, (-1, 32))
    blocks *= torch.exp2(torch.randint(-2, 2, (*blocks.shape[:-1], 1), generator=gen).double())
    return [t.cuda() for t in pack64(y)]


class Prefix4:
    """A random prefix of ``length`` positions in 4-bit pages with other pages around it; k and v are
    (elements, scales)."""

    def __init__(self, gen, rng, layers, kv_heads, dim, length, page, extra=0):
        self.page, self.length = page, length
        used = max(1, -(-(length + extra) // page))
        n = used + 3
        self.pages = rng.permutation(n)[:used].astype(np.int32)
        shape = (n, layers, kv_heads, page, dim)
        self.k, self.v = random_rows(gen, shape), random_rows(gen, shape)

    def packed(self, pool, layer, a, e):
        """(elements, scales) of positions a .. e - 1, [positions][Hkv][..], host."""
        at = torch.arange(a, e)
        page = torch.from_numpy(self.pages).long()[at // self.page]
        return [t.cpu()[page, layer, :, at % self.page] for t in pool]

    def rows(self, pool, layer, upto=None):
        """[Hkv][positions][d] of a layer, in order of position (host, float64)."""
        return values64(*self.packed(pool, layer, 0, self.length if upto is None else upto)).transpose(0, 1)

    def attach(self, dec, length=None):
        dec.set_prefix4(self.k[0], self.k[1], self.v[0], self.v[1], self.pages, self.length if length is None else length)
