"""The shared prefix in 64 bits, from its definition, for the tests: rotation, attention over an
interval of positions and a trie's path, and the error bounds of the kernels' arithmetic."""
from __future__ import annotations

import numpy as np
import torch

HALF_BF16, HALF_F32 = 2.0 ** -8, 2.0 ** -24  # half a rounding step, relative to the value


def half_step(dtype):
    return HALF_BF16 if dtype == torch.bfloat16 else HALF_F32


def turn(x, pos, freq, interleaved):
    """x [..., n, H, d], pos [n], freq [r/2] (float32 values): float64, element by element."""
    x, r = x.double().cpu(), 2 * len(freq)
    a = np.asarray(pos, np.float64)[:, None] * np.asarray(freq.double().cpu())
    c, s = torch.from_numpy(np.cos(a))[:, None], torch.from_numpy(np.sin(a))[:, None]
    y = x.clone()
    for i in range(r // 2):
        i0, i1 = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        y[..., i0] = x[..., i0] * c[..., i] - x[..., i1] * s[..., i]
        y[..., i1] = x[..., i1] * c[..., i] + x[..., i0] * s[..., i]
    return y


def turn_error(x, freq, interleaved, dtype):
    """Bound on the error of a stored rotation: cos and sin within 2^-22 (their argument, in half
    turns, is rounded once, and either function to a few units), two products and a sum within 3
    half steps of fp32, and the last rounding."""
    x, r = x.double().cpu().abs(), 2 * len(freq)
    size = x.clone()
    for i in range(r // 2):
        i0, i1 = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        size[..., i0] = size[..., i1] = x[..., i0] + x[..., i1]
    return size * (2.0 ** -21 + half_step(dtype))


def attend(q, k, v, seen, scale, dtype):
    """q [n][Hq][d], k / v [Hkv][m][d], seen [n][m]: (out [n][Hq][d], bound on the kernels' error).

    The bound.  A score is a sum of d products in fp32 (any order: at most d half steps of the sum of
    their sizes), scaled in two more roundings; the exponential is good to 2 half steps plus the
    score's error.  bf16: the weights are rounded to bf16 in numerator and denominator alike, so an
    error e_i of weight i moves the output by p_i e_i (v_i - o).  The sums over the keys: chains of at
    most m / 32 + 64 additions.  Then the last rounding."""
    n, Hq, d = q.shape
    Hkv = k.shape[0]
    G = Hq // Hkv
    out, tol = torch.zeros(n, Hq, d, dtype=torch.float64), torch.zeros(n, Hq, d, dtype=torch.float64)
    q, k, v, seen = q.double().cpu(), k.double().cpu(), v.double().cpu(), seen.cpu()
    h = half_step(dtype)
    for i in range(n):
        at = torch.nonzero(seen[i]).view(-1)
        if len(at) == 0:
            continue
        for g in range(Hkv):
            qi, kk, vv = q[i, g * G:(g + 1) * G], k[g, at], v[g, at]
            s = qi @ kk.t() * scale
            p = torch.softmax(s, -1)
            o = p @ vv
            size = (qi.abs() @ kk.abs().t()).max() * scale
            score = (d + 4) * HALF_F32 * size * 1.5 + 4 * HALF_F32
            chain = (len(at) / 32 + 64) * HALF_F32
            spread = torch.stack([(p[j][:, None] * (vv - o[j]).abs()).sum(0) for j in range(G)])
            weights = (h if dtype == torch.bfloat16 else 0.0) + 2 * score
            out[i, g * G:(g + 1) * G] = o
            tol[i, g * G:(g + 1) * G] = (weights * 1.01) * spread + 2 * chain * (p @ vv.abs()) + h * 1.01 * o.abs() + 1e-30
    return out, tol


def grow(rng, prompt, steps, b, keep_dead=False):
    """A trie after ``steps`` steps of b beams, as td_load_state takes it."""
    parent, depth = list(range(-1, prompt - 1)), list(range(prompt))
    leaves = [prompt - 1]
    for s in range(steps):
        pick = [leaves[int(r)] for r in rng.integers(0, len(leaves), b)]
        leaves = list(range(len(parent), len(parent) + b))
        parent += pick
        depth += [prompt + s] * b
    bits = [0] * len(parent)
    for i, n in enumerate(leaves):
        while n >= 0:
            bits[n] |= 1 << i
            n = parent[n]
    mask = np.array(bits, np.uint64)
    old = np.arange(len(parent)) if keep_dead else np.nonzero(mask)[0]
    slot = np.full(len(parent) + 1, -1, np.int32)
    slot[old] = np.arange(len(old))
    n, nl = len(old), len(leaves)
    return dict(n_nodes=n, n_live=nl, next_id=len(parent), kv_pending=0, step=steps, node_id=old.astype(np.int32),
                parent_slot=slot[np.array(parent)[old]], token=np.zeros(n, np.int32),
                depth=np.array(depth, np.int32)[old], mask=mask[old], leaf_slot=np.arange(n - nl, n, dtype=np.int32),
                leaf_score=-np.arange(nl).astype(np.float32))


def path_of(state, slot):
    """The node's stored ancestors and itself."""
    seen = np.zeros(state["n_nodes"], bool)
    while slot >= 0:
        seen[slot] = True
        slot = int(state["parent_slot"][slot])
    return seen


class Prefix:
    """A random prefix of ``length`` positions in a paged pool with other pages around it."""

    def __init__(self, gen, rng, layers, kv_heads, dim, dtype, length, page, extra=0):
        self.page, self.length = page, length
        used = max(1, -(-(length + extra) // page))
        n = used + 3
        self.pages = rng.permutation(n)[:used].astype(np.int32)
        shape = (n, layers, kv_heads, page, dim)
        self.k = torch.randn(shape, generator=gen).to(dtype).cuda()
        self.v = torch.randn(shape, generator=gen).to(dtype).cuda()

    def rows(self, pool, layer, upto=None):
        """[Hkv][positions][d] of a layer, in order of position (host, as stored)."""
        n = self.length if upto is None else upto
        got = pool[:, layer].cpu()
        if n == 0:
            return got[0][:, :0]
        return torch.stack([got[self.pages[p // self.page], :, p % self.page] for p in range(n)], 1)

    def attach(self, dec, length=None):
        dec.set_prefix(self.k, self.v, self.pages, self.length if length is None else length)


def check(got, want, tol, what):
    got = got.double().cpu()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(((got - want).abs() - tol)[bad].max()) if bad.any() else 0.0,
                           [int(x) for x in torch.nonzero(bad)[0]], float(got[tuple(torch.nonzero(bad)[0])]),
                           float(want[tuple(torch.nonzero(bad)[0])]))
