"""Stores whose workgroups take several rows each (few heads, thousands of rows), against 64 bits: pages of the
context's type, the tries' pools, one position per row and several axes, and millions of tokens."""
import numpy as np
import pytest
import torch

import paper_2502_00085_amd.binding as B
from gpu_harness import log
from prefix4_ref import pack64, turn_axes
from prefix_ref import check, grow, turn_error

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
L = 3  # layers, of which two are stored


def freqs(r, base=10000.0):
    return (base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().cuda()


def randn(gen, shape, dt):
    return torch.randn(shape, generator=gen).to(dt).cuda()


def rope_of(rng, r, inter, axes):
    """(frequencies, the axis of each pair, what the call takes)."""
    f = freqs(r)
    if axes == 0:
        return f, np.zeros(r // 2, int), B.Rope(f, inter)
    axis = rng.integers(0, axes, r // 2)
    axis[-1] = axes - 1
    return f, axis, B.RopeAxes(f, axis, inter)


# (a workgroup has as many rows as its 256 threads have units for, at most 8, and one of 1,024 of the call's rows)
@pytest.mark.parametrize("axes,form", [(0, "own"), (3, "positions"), (2, "shift"), (4, "own")])
@pytest.mark.parametrize("dtype,D,Hq,Hkv,r,inter,page,pos,n", [
    ("bf16", 64, 2, 1, 64, False, 64, 70, 4203),  # 8 rows
    ("bf16", 128, 4, 2, 64, True, 16, 3, 2101),   # 4
    ("f32", 32, 1, 1, 32, False, 128, 0, 4100),   # 8
    ("f32", 96, 3, 1, 48, True, 32, 33, 1600)])   # 3
def test_pages(dtype, D, Hq, Hkv, r, inter, page, pos, n, axes, form):
    log(f"pages {dtype} d={D} r={r} inter={inter} page={page} pos={pos} n={n} axes={axes} {form}")
    gen, rng, dt = torch.Generator().manual_seed(11), np.random.default_rng(11), DT[dtype]
    dec = B.TrieDecoder(1, 1, 4, 100, L, Hq, Hkv, D, dtype=dtype)
    used = -(-(pos + n) // page)
    table = rng.permutation(used + 2)[:used]
    k_pages, v_pages = (randn(gen, (used + 2, L, Hkv, page, D), dt) for _ in range(2))
    before = k_pages.clone(), v_pages.clone()
    dec.set_prefix(k_pages, v_pages, table, 0)
    k, v, q = (randn(gen, (2, n, h, D), dt) for h in (Hkv, Hkv, Hq))
    out = torch.full_like(q, 7.0)
    f, axis, rope = rope_of(rng, r, inter, axes)
    where, more = np.repeat(np.arange(pos, pos + n)[:, None], max(1, axes), 1), {}
    if form == "positions":
        where = rng.integers(-50, 5000, (n, axes))
        more["positions"] = torch.from_numpy(where.astype(np.int32)).cuda()
    elif form == "shift":
        shift = rng.integers(-900, 50, (1, axes))
        where = where + shift
        more["shift"] = torch.from_numpy(shift.astype(np.int32)).cuda()
    dec.prefix_store(1, 2, pos, k, v, q, out, rope, **more)
    check(out, turn_axes(q, where, f, axis, inter), turn_error(q, f, inter, dt), "q")
    at = torch.arange(pos, pos + n)
    pg, row = torch.from_numpy(table).long()[at // page], at % page
    stored = torch.stack([k_pages.cpu()[pg, 1 + l, :, row] for l in range(2)])
    check(stored, turn_axes(k, where, f, axis, inter), turn_error(k, f, inter, dt), "k")
    assert torch.equal(torch.stack([v_pages.cpu()[pg, 1 + l, :, row] for l in range(2)]), v.cpu())
    own = torch.zeros(k_pages.shape[:4], dtype=torch.bool)
    for l in range(2):
        own[pg, 1 + l, :, row] = True
    assert torch.equal(k_pages.cpu()[~own], before[0].cpu()[~own]) and torch.equal(v_pages.cpu()[~own], before[1].cpu()[~own])
    assert dec.status() == 0
    dec.close()


# rows of several tries in one workgroup: the number of a trie's rows is no multiple of the workgroup's
@pytest.mark.parametrize("axes,form", [(0, "own"), (3, "positions"), (2, "shift")])
@pytest.mark.parametrize("what,dtype,D,Hq,Hkv,r,inter,T,n,S", [
    ("nodes", "bf16", 64, 2, 1, 64, False, 9, 457, 40),  # 8 rows
    ("nodes", "f32", 32, 2, 2, 16, True, 5, 421, 0),     # 4
    ("leaves", "bf16", 96, 2, 1, 48, False, 300, 7, 17),  # 4
    ("leaves", "f32", 64, 1, 1, 64, True, 521, 3, 1000)])  # 3
def test_tries(what, dtype, D, Hq, Hkv, r, inter, T, n, S, axes, form):
    log(f"tries {what} {dtype} d={D} r={r} inter={inter} T={T} n={n} S={S} axes={axes} {form}")
    gen, rng, dt = torch.Generator().manual_seed(12), np.random.default_rng(12), DT[dtype]
    b = n if what == "leaves" else 4
    kinds = [grow(rng, 40, 3, b), grow(rng, 3, 5, b), grow(rng, 1, 0, b)] if what == "leaves" else \
            [grow(rng, 500, 0, b), grow(rng, 90, 30, b, keep_dead=True), grow(rng, 1, 2, b)]
    cap = max(s["n_nodes"] for s in kinds) + b
    dec = B.TrieDecoder(T, b, cap, 100, L, Hq, Hkv, D, dtype=dtype)
    tries = [kinds[int(i)] for i in rng.integers(0, 3, T)]
    for t, s in enumerate(tries):
        dec.load_state(t, s)
    if S:
        shape = ((S + 15) // 16, L, Hkv, 16, D)
        pages = torch.zeros(shape, dtype=dt, device="cuda"), torch.zeros(shape, dtype=dt, device="cuda")
        dec.set_prefix(*pages, range(shape[0]), S)
    dec.k_pool.copy_(randn(gen, tuple(dec.k_pool.shape), dt))
    dec.v_pool.copy_(randn(gen, tuple(dec.v_pool.shape), dt))
    kb, vb = dec.k_pool.cpu().clone(), dec.v_pool.cpu().clone()
    slots = np.full((T, n), -1, np.int64)
    for t, s in enumerate(tries):  # (leaves: those that live; nodes: some, in any order, with gaps)
        if what == "leaves":
            slots[t, :s["n_live"]] = s["leaf_slot"]
        else:
            some = rng.permutation(s["n_nodes"])[:int(rng.integers(1, n + 1))]
            slots[t, np.sort(rng.permutation(n)[:len(some)])] = some
    k, v, q = (randn(gen, (2, T, n, h, D), dt) for h in (Hkv, Hkv, Hq))
    out = torch.full_like(q, 3.0)
    f, axis, rope = rope_of(rng, r, inter, axes)
    depth = np.stack([np.where(x >= 0, s["depth"][np.maximum(x, 0)], 0) for x, s in zip(slots, tries)])
    where, more = np.repeat((S + depth)[..., None], max(1, axes), 2), {}
    if form == "positions":
        where = rng.integers(-50, 5000, (T, n, axes))
        more["positions"] = torch.from_numpy(where.astype(np.int32)).cuda()
    elif form == "shift":
        shift = rng.integers(-900, 50, (T, axes))
        where = where + shift[:, None]
        more["shift"] = torch.from_numpy(shift.astype(np.int32)).cuda()
    dec.store_kv(1, 2, k, v, q, out, rope, None if what == "leaves" else torch.from_numpy(slots.astype(np.int32)).cuda(), **more)
    some = torch.from_numpy(slots.reshape(-1) >= 0)
    flat = where.reshape(T * n, -1)
    q, k, v, out = (x.flatten(1, 2) for x in (q, k, v, out))
    assert bool((out.cpu()[:, ~some] == 0).all())
    want = turn_axes(q, flat, f, axis, inter)
    check(out.cpu()[:, some], want[:, some], turn_error(q, f, inter, dt)[:, some], "q")
    t = torch.arange(T).repeat_interleave(n)[some]
    slot = torch.from_numpy(slots.reshape(-1))[some]
    stored = torch.stack([dec.k_pool.cpu()[t, 1 + l, :, slot] for l in range(2)])
    check(stored, turn_axes(k, flat, f, axis, inter)[:, some], turn_error(k, f, inter, dt)[:, some], "k")
    assert torch.equal(torch.stack([dec.v_pool.cpu()[t, 1 + l, :, slot] for l in range(2)]), v.cpu()[:, some])
    own = torch.zeros(dec.k_pool.shape[:4], dtype=torch.bool)
    for l in range(2):
        own[t, 1 + l, :, slot] = True
    assert torch.equal(dec.k_pool.cpu()[~own], kb[~own]) and torch.equal(dec.v_pool.cpu()[~own], vb[~own])
    assert dec.status() == 0
    dec.close()


@pytest.mark.parametrize("axes", [0, 3])
@pytest.mark.parametrize("kind", ["4 bits", "plain"])
def test_millions_of_tokens(kind, axes):
    """Rows at every place of a workgroup's eight, at the ends and anywhere in a call of over four million."""
    n, page, D = 2 ** 22 + 5, 65536, 32
    log(f"{kind} n={n} axes={axes}")
    gen, rng, dt = torch.Generator(device="cuda").manual_seed(13), np.random.default_rng(13), torch.bfloat16
    used = -(-n // page)
    table = rng.permutation(used + 1)[:used]
    shape = (used + 1, 1, 1, page)
    widths, t = ((D // 2, D // 32, D // 2, D // 32), torch.uint8) if kind == "4 bits" else ((D, D), dt)
    pages = [torch.zeros(shape + (w,), dtype=t, device="cuda") for w in widths]
    dec = B.TrieDecoder(1, 1, 4, 100, 1, 1, 1, D)
    (dec.set_prefix4 if kind == "4 bits" else dec.set_prefix)(*pages, table, 0)
    k, v, q = (torch.randn((1, n, 1, D), generator=gen, device="cuda").to(dt) for _ in range(3))
    f, axis, rope = rope_of(rng, D, False, axes)
    out, more = torch.empty_like(q), {}
    if axes:
        given = torch.randint(-10000, 2 ** 22, (n, axes), generator=gen, device="cuda", dtype=torch.int32)
        more["positions"] = given
    dec.prefix_store(0, 1, 0, k, v, q, out, rope, **more)
    at = torch.from_numpy(np.unique(np.concatenate([np.arange(40), np.arange(n - 40, n), rng.integers(0, n, 4000)])))
    assert {int(x) % 8 for x in at} == set(range(8))
    where = given.cpu()[at].numpy() if axes else at.numpy()[:, None]
    k, v, q, out = (x[:, at.cuda()].cpu() for x in (k, v, q, out))
    check(out, turn_axes(q, where, f, axis, False), turn_error(q, f, False, dt), "q")
    pg, row = torch.from_numpy(table).long()[at // page].cuda(), (at % page).cuda()
    got = [p[pg, 0, 0, row].cpu() for p in pages]
    want = turn_axes(k, where, f, axis, False)[0, :, 0]
    if kind == "4 bits":
        assert all(torch.equal(a, b) for a, b in zip(got, pack64(want) + pack64(v[0, :, 0])))
    else:
        check(got[0], want, turn_error(k, f, False, dt)[0, :, 0], "k")
        assert torch.equal(got[1], v[0, :, 0])
    assert dec.status() == 0
    dec.close()
