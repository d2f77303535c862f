"""A run as a program makes it: a shared prefix prefilled in chunks, ragged prompts behind it, then
decode steps that collect and move rows - every row stored by the calls that rotate, layer by layer.
Checked in 64 bits: the stored rows of every node against its raw ones at its position, and every
output against attention over the stored rows that it may see."""
import numpy as np
import pytest
import torch

import paper_2502_00085_amd.binding as B
from gpu_harness import log
from prefix_ref import attend, check, path_of, turn, turn_error

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype,D,Hq,Hkv,inter,window,gc,page", [
    ("bf16", 128, 8, 2, False, 0, 1, 16), ("bf16", 64, 4, 4, True, 45, 1, 32), ("bf16", 96, 6, 2, False, 70, 3, 64),
    ("f32", 64, 4, 2, False, 0, 4, 16), ("f32", 96, 2, 1, True, 30, 1, 16)])
def test_run(dtype, D, Hq, Hkv, inter, window, gc, page):
    gen, rng, dt = torch.Generator().manual_seed(11), np.random.default_rng(11), DT[dtype]
    T, b, L, V, S, steps = 2, 4, 2, 50, 75, 9
    plen = [21, 34]
    scale = 1.0 / D ** 0.5
    freq = (10000.0 ** (-torch.arange(0, 32, 2, dtype=torch.float64) / 32)).float().cuda()
    rope = B.Rope(freq, inter)
    dec = B.TrieDecoder(T, b, 120, V, L, Hq, Hkv, D, window, dtype, gc_interval=gc)

    def raw(*lead):
        return [torch.randn(lead + (h, D), generator=gen).to(dt).cuda() for h in (Hq, Hkv, Hkv)]

    def seen_by(q, k, v, seen, out, what):
        at = torch.nonzero(seen).view(-1)
        want, tol = attend(q[None], k[:, at], v[:, at], torch.ones(1, len(at), dtype=torch.bool), scale, dt)
        check(out[None], want, tol, what)

    # the prefix, in chunks of odd sizes
    n_pages = -(-S // page) + 2
    pages = rng.permutation(n_pages)[:-(-S // page)]
    kp = torch.full((n_pages, L, Hkv, page, D), float("nan"), dtype=dt, device="cuda")
    vp = kp.clone()
    dec.set_prefix(kp, vp, pages, S)
    pq, pk, pv = raw(L, S)
    pout, prot = torch.empty_like(pq), torch.empty_like(pq)
    for a, e in ((0, 33), (33, 34), (34, S)):
        for l in range(L):
            dec.prefix_store(l, 1, a, pk[l:l + 1, a:e].contiguous(), pv[l:l + 1, a:e].contiguous(), pq[l:l + 1, a:e].contiguous(),
                             rq := torch.empty((1, e - a, Hq, D), dtype=dt, device="cuda"), rope)
            dec.prefix_attn(l, 1, a, rq, ro := torch.empty_like(rq), scale)
            prot[l, a:e], pout[l, a:e] = rq[0], ro[0]
    pos = np.arange(S)
    prefix = []
    for l in range(L):
        k, v = (torch.stack([x[int(pages[p // page]), l, :, p % page] for p in pos], 1).cpu() for x in (kp, vp))
        check(k.transpose(0, 1), turn(pk[l], pos, freq, inter), turn_error(pk[l], freq, inter, dt), "prefix k")
        assert torch.equal(v.transpose(0, 1), pv[l].cpu())
        check(prot[l], turn(pq[l], pos, freq, inter), turn_error(pq[l], freq, inter, dt), "prefix q")
        prefix.append((k, v))
        for j in (0, 32, 33, 34, 60, S - 1):
            seen_by(prot[l, j], k, v, (torch.arange(S) <= j) & (torch.arange(S) > j - (window or S)), pout[l, j], ("prefix", l, j))

    # the prompts
    most = max(plen)
    dec.init_prompt(plen, torch.zeros((T, most), dtype=torch.int32, device="cuda"))
    qs = torch.full((T, most), -1, dtype=torch.int32, device="cuda")
    for t, n in enumerate(plen):
        qs[t, :n] = torch.arange(n, device="cuda")
    q, k, v = raw(L, T, most)
    raws = [[{j: (k[l, t, j], v[l, t, j]) for j in range(plen[t])} for t in range(T)] for l in range(L)]
    rot, out = torch.empty_like(q), torch.zeros_like(q)
    for l in range(L):
        dec.store_kv(l, 1, k[l:l + 1], v[l:l + 1], q[l:l + 1], rot[l:l + 1], rope, qs)
        if dtype == "bf16":
            dec.tree_attn(l, 1, qs, rot[l], out[l], scale)

    def nodes(l, t, st):
        """Keys and values the trie's node n sees: the prefix's, then the stored nodes'."""
        at = slice(st["base"], st["base"] + st["n_nodes"])
        kk, vv = dec.k_pool[t, l, :, at].cpu(), dec.v_pool[t, l, :, at].cpu()
        own = [raws[l][t][int(i)] for i in st["node_id"]]
        rk = torch.stack([x[0] for x in own])
        check(kk.transpose(0, 1), turn(rk, S + st["depth"], freq, inter), turn_error(rk, freq, inter, dt), ("k", l, t))
        assert torch.equal(vv.transpose(0, 1), torch.stack([x[1] for x in own]).cpu())
        return torch.cat([prefix[l][0], kk], 1), torch.cat([prefix[l][1], vv], 1)

    def sees(st, n):
        d = st["depth"]
        seen = torch.cat([torch.ones(S, dtype=torch.bool), torch.from_numpy(path_of(st, n))])
        if window:
            at = torch.cat([torch.arange(S), torch.from_numpy(S + d)])
            seen &= S + int(d[n]) - at < window
        return seen

    for t in range(T):
        st = dec.read_state(t)
        for l in range(L):
            kk, vv = nodes(l, t, st)
            check(rot[l, t, :plen[t]], turn(q[l, t, :plen[t]], S + np.arange(plen[t]), freq, inter),
                  turn_error(q[l, t, :plen[t]], freq, inter, dt), "prompt q")
            if dtype == "bf16":
                for j in (0, 1, 13, plen[t] - 1):
                    seen_by(rot[l, t, j], kk, vv, sees(st, j), out[l, t, j], ("prompt", l, t, j))

    # the steps
    sel = [torch.zeros((T, b), dtype=x, device="cuda") for x in (torch.int32, torch.int32, torch.float32, torch.float32)]
    for step in range(steps):
        log(f"run {dtype} d={D} W={window} g={gc} step {step}")
        q, k, v = raw(L, T, b)
        rot, out = torch.empty_like(q), torch.empty_like(q)
        for l in range(L):
            if step == 0:  # (the prompt's last token: its row is stored, its query comes again)
                dec.store_kv(l, 1, None, None, q[l:l + 1], rot[l:l + 1], rope)
            else:
                dec.store_kv(l, 1, k[l:l + 1], v[l:l + 1], q[l:l + 1], rot[l:l + 1], rope)
            dec.attn_decode(l, 1, rot[l], None, None, out[l], scale)
        for t in range(T):
            st = dec.read_state(t)
            if step:
                for l in range(L):
                    for j in range(b):
                        raws[l][t][int(st["node_id"][st["leaf_slot"][j]])] = (k[l, t, j], v[l, t, j])
            assert st["kv_pending"] == 0
            for l in range(L):
                kk, vv = nodes(l, t, st)
                for j in range(b):
                    if j >= st["n_live"]:
                        assert bool((out[l, t, j] == 0).all()) and bool((rot[l, t, j] == 0).all())
                        continue
                    leaf = int(st["leaf_slot"][j])
                    check(rot[l, t, j][None], turn(q[l, t, j][None], [S + int(st["depth"][leaf])], freq, inter),
                          turn_error(q[l, t, j][None], freq, inter, dt), "q")
                    seen_by(rot[l, t, j], kk, vv, sees(st, leaf), out[l, t, j], (step, l, t, j))
        dec.topk_append((torch.randn((T, b, V), generator=gen) * 3).cuda(), *sel)
    assert dec.status() == 0
    dec.close()
