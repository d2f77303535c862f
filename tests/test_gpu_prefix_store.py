"""trie_store_kv and trie_prefix_store against 64 bits: rotations, pages, rows that are no nodes,
strides, and that everything else in the pools stays as it was."""
import numpy as np
import pytest
import torch

import paper_2502_00085_amd.binding as B
from gpu_harness import log
from prefix_ref import Prefix, check, grow, turn, turn_error

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def freqs(r, base=10000.0):
    return (base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().cuda()


def randn(gen, shape, dt):
    return torch.randn(shape, generator=gen).to(dt).cuda()


@pytest.mark.parametrize("dtype,D,Hq,Hkv,r,inter,page,pos,n", [
    ("bf16", 128, 8, 2, 128, False, 64, 0, 200), ("bf16", 128, 4, 4, 64, True, 16, 37, 1), ("bf16", 96, 3, 3, 96, False, 16, 31, 34),
    ("f32", 64, 4, 1, 32, True, 32, 100, 65), ("f32", 96, 2, 2, 48, False, 128, 5, 130), ("f32", 32, 7, 1, 16, False, 16, 0, 17),
    ("bf16", 256, 2, 1, 256, True, 256, 250, 9), ("f32", 256, 2, 1, 256, False, 16, 1, 16), ("bf16", 32, 64, 8, 16, True, 16, 3, 40),
    ("bf16", 64, 4, 2, 0, False, 16, 7, 50), ("f32", 160, 5, 5, 80, True, 64, 60, 8)])
def test_prefix_store(dtype, D, Hq, Hkv, r, inter, page, pos, n):
    log(f"prefix store {dtype} d={D} r={r} inter={inter} page={page} pos={pos} n={n}")
    gen, rng, dt, L = torch.Generator().manual_seed(1), np.random.default_rng(1), DT[dtype], 3
    dec = B.TrieDecoder(1, 1, 4, 100, L, Hq, Hkv, D, dtype=dtype)
    p = Prefix(gen, rng, L, Hkv, D, dt, pos + n, page)
    p.attach(dec, 0)
    before = p.k.clone(), p.v.clone()
    k, v, q = randn(gen, (2, n, Hkv, D), dt), randn(gen, (2, n, Hkv, D), dt), randn(gen, (2, n, Hq, D), dt)
    out = torch.full_like(q, 7.0)
    rope = B.Rope(freqs(r), inter) if r else None
    dec.prefix_store(1, 2, pos, k, v, q, out, rope)
    where = np.arange(pos, pos + n)
    f = freqs(r) if r else torch.zeros(0)
    check(out, turn(q, where, f, inter), turn_error(q, f, inter, dt), "q")
    want_k = turn(k, where, f, inter)
    for l in range(2):
        got = p.rows(p.k, 1 + l)[:, pos:].transpose(0, 1)
        check(got, want_k[l], turn_error(k[l], f, inter, dt), f"k layer {l}")
        assert torch.equal(p.rows(p.v, 1 + l)[:, pos:].transpose(0, 1), v[l].cpu())
    # every other row is as it was
    own = torch.zeros(p.k.shape[:4], dtype=torch.bool, device="cuda")
    for x in where:
        own[int(p.pages[x // page]), 1:3, :, x % page] = True
    assert torch.equal(p.k[~own], before[0][~own]) and torch.equal(p.v[~own], before[1][~own])
    assert dec.status() == 0
    dec.close()


@pytest.mark.parametrize("pos", [100_003, 1_000_000, 2 ** 24 + 1])
def test_far_positions(pos):
    """Angles of a million radians and more: the turn is still that of the exact product."""
    gen, D = torch.Generator().manual_seed(2), 32
    dec = B.TrieDecoder(1, 1, 4, 100, 1, 1, 1, D, dtype="f32")
    n_table = pos // 65536 + 1
    k_pages = torch.zeros((n_table, 1, 1, 65536, D), device="cuda")
    v_pages = torch.zeros_like(k_pages)
    dec.set_prefix(k_pages, v_pages, range(n_table), 0)
    k, q = randn(gen, (1, 5, 1, D), torch.float32), randn(gen, (1, 5, 1, D), torch.float32)
    out, f = torch.empty_like(q), freqs(32, 1.5)
    dec.prefix_store(0, 1, pos, k, k, q, out, B.Rope(f))
    where = np.arange(pos, pos + 5)
    check(out, turn(q, where, f, False), turn_error(q, f, False, torch.float32), "q")
    got = k_pages.view(-1, D)[pos:pos + 5][None, :, None]
    check(got, turn(k, where, f, False), turn_error(k, f, False, torch.float32), "k")
    dec.close()


@pytest.mark.parametrize("dtype,D,Hq,Hkv,inter,S", [("bf16", 128, 8, 2, False, 70), ("f32", 64, 3, 1, True, 0), ("bf16", 96, 4, 4, True, 1)])
def test_store_nodes_and_leaves(dtype, D, Hq, Hkv, inter, S):
    """Ragged tries; rows with no node (-1, past the last, far past it), tries of fewer live leaves than
    beams; slices of a fused projection; queries alone and K/V alone."""
    log(f"node store {dtype} d={D} S={S}")
    gen, rng, dt, L, T, b, r = torch.Generator().manual_seed(3), np.random.default_rng(3), DT[dtype], 2, 3, 4, 32
    dec = B.TrieDecoder(T, b, 64, 100, L, Hq, Hkv, D, dtype=dtype)
    tries = [grow(rng, 9, 5, b, keep_dead=True), grow(rng, 17, 0, b), grow(rng, 1, 3, 2)]
    for t, s in enumerate(tries):
        dec.load_state(t, s)
    if S:
        Prefix(gen, rng, L, Hkv, D, dt, S, 16).attach(dec)
    dec.k_pool.copy_(randn(gen, tuple(dec.k_pool.shape), dt))
    dec.v_pool.copy_(randn(gen, tuple(dec.v_pool.shape), dt))
    f = freqs(r)
    rope = B.Rope(f, inter)
    for form in ("nodes", "leaves"):
        n = 11 if form == "nodes" else b
        slots = np.full((T, n), -1, np.int64)
        if form == "nodes":
            slots[0, [0, 3, 4, 10]] = [0, tries[0]["n_nodes"] - 1, 9, 5]
            slots[1, :9] = np.arange(16, 7, -1)
            slots[1, 9:] = [tries[1]["n_nodes"], 2 ** 31 - 1]
            slots[2, 5] = 0
        else:
            for t, s in enumerate(tries):
                slots[t, :s["n_live"]] = s["leaf_slot"]
        qs = torch.from_numpy(slots.astype(np.int32)).cuda() if form == "nodes" else None
        fused = randn(gen, (1, T, n, (Hq + 2 * Hkv) * D + 16), dt)
        q = fused[..., :Hq * D].unflatten(-1, (Hq, D))
        k = fused[..., Hq * D:(Hq + Hkv) * D].unflatten(-1, (Hkv, D))
        v = fused[..., (Hq + Hkv) * D:(Hq + 2 * Hkv) * D].unflatten(-1, (Hkv, D))
        for parts in ("all", "q", "kv"):
            kb, vb, out = dec.k_pool.clone(), dec.v_pool.clone(), torch.full((1, T, n, Hq, D), 3.0, dtype=dt, device="cuda")
            dec.store_kv(1, 1, None if parts == "q" else k, None if parts == "q" else v, None if parts == "kv" else q,
                         None if parts == "kv" else out, rope, qs)
            own = torch.zeros(dec.k_pool.shape[:4], dtype=torch.bool)
            for t, s in enumerate(tries):
                for j, slot in enumerate(slots[t]):
                    if not 0 <= slot < s["n_nodes"]:
                        if parts != "kv":
                            assert bool((out[0, t, j] == 0).all())
                        continue
                    at = [S + int(s["depth"][slot])]
                    if parts != "kv":
                        check(out[0, t, j:j + 1], turn(q[0, t, j:j + 1], at, f, inter), turn_error(q[0, t, j:j + 1], f, inter, dt), "q")
                    if parts != "q":
                        check(dec.k_pool[t, 1, :, slot][None], turn(k[0, t, j:j + 1], at, f, inter),
                              turn_error(k[0, t, j:j + 1], f, inter, dt), "k")
                        assert torch.equal(dec.v_pool[t, 1, :, slot], v[0, t, j])
                        own[t, 1, :, slot] = True
            own = own.cuda()
            assert torch.equal(dec.k_pool[~own], kb[~own]) and torch.equal(dec.v_pool[~own], vb[~own])
            if parts == "kv":
                assert bool((out == 3.0).all())
    assert dec.status() == 0
    dec.close()


def test_queries_in_place():
    gen = torch.Generator().manual_seed(4)
    dec = B.TrieDecoder(1, 2, 40, 100, 1, 4, 2, 64, dtype="bf16")
    dec.init_prompt([30], torch.zeros((1, 30), dtype=torch.int32, device="cuda"))
    q, f = randn(gen, (1, 1, 30, 4, 64), torch.bfloat16), freqs(64)
    want, tol = turn(q[0, 0], np.arange(30), f, False), turn_error(q[0, 0], f, False, torch.bfloat16)
    qs = torch.arange(30, dtype=torch.int32, device="cuda")[None]
    dec.store_kv(0, 1, None, None, q, q, B.Rope(f), qs)
    check(q[0, 0], want, tol, "q")
    dec.close()


@pytest.mark.parametrize("dtype,D,window,gc", [("bf16", 128, 0, 1), ("bf16", 64, 40, 3), ("f32", 64, 40, 1), ("f32", 96, 0, 4),
                                               ("bf16", 128, 25, 1)])
def test_stored_leaves_are_what_the_attention_stores(dtype, D, window, gc):
    """store_kv (no rotation) and then the attention without k_new, layer by layer, against the
    attention that stores k_new itself: pools, outputs and states, bit for bit, over steps that
    collect and move rows."""
    gen, dt, L, T, b, Hq, Hkv, V = torch.Generator().manual_seed(5), DT[dtype], 3, 2, 5, 8, 2, 60
    decs = [B.TrieDecoder(T, b, 220, V, L, Hq, Hkv, D, window, dtype, gc_interval=gc) for _ in range(2)]
    plen = [33, 60]
    pk, pv = randn(gen, tuple(decs[0].k_pool.shape), dt), randn(gen, tuple(decs[0].k_pool.shape), dt)
    for d in decs:
        d.k_pool.copy_(pk)
        d.v_pool.copy_(pv)
        d.init_prompt(plen, torch.zeros((T, 60), dtype=torch.int32, device="cuda"))
    sel = [[torch.zeros((T, b), dtype=x, device="cuda") for x in (torch.int32, torch.int32, torch.float32, torch.float32)] for _ in decs]
    for step in range(14):
        q, k, v = (randn(gen, (L, T, b, h, D), dt) for h in (Hq, Hkv, Hkv))
        logits = (torch.randn((T, b, V), generator=gen) * 3).cuda()
        out = [torch.zeros_like(q) for _ in decs]
        new = step > 0
        for l in range(L):
            decs[0].attn_decode(l, 1, q[l], k[l] if new else None, v[l] if new else None, out[0][l], 0.1)
            if new:
                decs[1].store_kv(l, 1, k[l:l + 1], v[l:l + 1])
            decs[1].attn_decode(l, 1, q[l], None, None, out[1][l], 0.1)
        assert torch.equal(out[0], out[1]), step
        for d, s in zip(decs, sel):
            d.topk_append(logits, *s)
        for t in range(T):
            a, c = decs[0].read_state(t), decs[1].read_state(t)
            assert a["n_nodes"] == c["n_nodes"] and a["base"] == c["base"] and np.array_equal(a["mask"], c["mask"])
            n = a["n_nodes"] - a["n_live"]
            for x, y in ((decs[0].k_pool, decs[1].k_pool), (decs[0].v_pool, decs[1].v_pool)):
                assert torch.equal(x[t], y[t]), (step, t)
            assert n > 0
    assert [d.status() for d in decs] == [0, 0]
    for d in decs:
        d.close()


def test_store_call_order():
    gen, dt = torch.Generator().manual_seed(6), torch.bfloat16
    dec = B.TrieDecoder(1, 2, 60, 50, 2, 2, 1, 64)
    dec.init_prompt([20], torch.zeros((1, 20), dtype=torch.int32, device="cuda"))
    q, k = randn(gen, (2, 1, 2, 2, 64), dt), randn(gen, (2, 1, 2, 1, 64), dt)
    out = torch.zeros_like(q)
    sel = [torch.zeros((1, 2), dtype=x, device="cuda") for x in (torch.int32, torch.int32, torch.float32, torch.float32)]
    dec.store_kv(0, 2, k, k)  # nothing pending: the live leaf's rows again
    dec.attn_decode(0, 2, q, None, None, out, 0.1)
    dec.topk_append(torch.randn((1, 2, 50), generator=gen).cuda(), *sel)
    qs = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    with pytest.raises(B.TdError) as e:
        dec.store_kv(0, 2, k, k, qslots=qs)
    assert e.value.status == B.TD_ESTATE
    dec.store_kv(0, 2, None, None, q, out)  # queries alone: the rows stay pending
    with pytest.raises(B.TdError) as e:
        dec.attn_decode(0, 1, q[0], None, None, out[0], 0.1)
    assert e.value.status == B.TD_EINVAL
    dec.store_kv(0, 1, k[:1], k[:1])
    dec.attn_decode(0, 1, q[0], None, None, out[0], 0.1)
    with pytest.raises(B.TdError):
        dec.attn_decode(0, 2, q, None, None, out, 0.1)
    with pytest.raises(B.TdError) as e:
        dec.topk_append(torch.zeros((1, 2, 50), device="cuda"), *sel)
    assert e.value.status == B.TD_ESTATE
    dec.attn_decode(0, 2, q, k, k, out, 0.1)  # (stores both layers' rows)
    dec.append_prune(sel[0], sel[1], sel[2])
    assert dec.status() == 0
    dec.close()


def test_rows_given_again_for_stored_layers():
    """k_new / v_new of layers whose rows store_kv has stored (rotated) are refused while other layers are
    pending too: nothing is overwritten.  Layers that the attention stored take them again, as ever."""
    gen, dt, L = torch.Generator().manual_seed(8), torch.bfloat16, 3
    dec = B.TrieDecoder(1, 2, 60, 50, L, 2, 1, 64)
    dec.init_prompt([20], torch.zeros((1, 20), dtype=torch.int32, device="cuda"))
    rope = B.Rope(freqs(64))
    q, k, v = (randn(gen, (L, 1, 2, h, 64), dt) for h in (2, 1, 1))
    out = torch.zeros_like(q)
    sel = [torch.zeros((1, 2), dtype=x, device="cuda") for x in (torch.int32, torch.int32, torch.float32, torch.float32)]

    def refused(l, n):
        pools = dec.k_pool.clone(), dec.v_pool.clone()
        with pytest.raises(B.TdError) as e:
            dec.attn_decode(l, n, q[l:l + n], k[l:l + n], v[l:l + n], out[l:l + n], 0.1)
        assert e.value.status == B.TD_EINVAL
        assert torch.equal(pools[0], dec.k_pool) and torch.equal(pools[1], dec.v_pool)

    dec.attn_decode(0, L, q, None, None, out, 0.1)
    for step in range(2):
        dec.topk_append(torch.randn((1, 2, 50), generator=gen).cuda(), *sel)
        dec.store_kv(0, 2, k[:2], v[:2], rope=rope)
        for l, n in ((0, 1), (1, 1), (0, 2)):
            refused(l, n)
        dec.attn_decode(0, 2, q[:2], None, None, out[:2], 0.1)
        refused(0, 1)  # (read by the attention, and still store_kv's)
        if step == 0:
            dec.attn_decode(2, 1, q[2], k[2], v[2], out[2], 0.1)
        else:
            dec.store_kv(2, 1, k[2:], v[2:], rope=rope)
        refused(2, 1)  # (nothing is pending any more)
        refused(0, L)
    dec.topk_append(torch.randn((1, 2, 50), generator=gen).cuda(), *sel)
    for _ in range(2):
        dec.attn_decode(0, 1, q[0], k[0], v[0], out[0], 0.1)
    dec.store_kv(0, 1, k[:1], v[:1], rope=rope)
    refused(0, 1)
    dec.attn_decode(1, 2, q[1:], k[1:], v[1:], out[1:], 0.1)
    assert dec.status() == 0
    dec.close()
