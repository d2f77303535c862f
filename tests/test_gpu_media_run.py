"""A run as a program with images makes it: a shared prefix of text and images prefilled in chunks into 4-bit or
plain pages, prompts that hold images of their own behind it, then decode steps that collect and move rows, whose
text continues where the images end - every row stored by the calls that turn by several axes, layer by layer, and
a captured step among them.  Checked in 64 bits: the stored rows of every node against its raw ones at its
positions, and every output against attention over the stored rows that it may see."""
import numpy as np
import pytest
import torch

import paper_2502_00085_amd.binding as B
from gpu_harness import log
from prefix4_ref import pack64, turn_axes, values64
from prefix_ref import attend, check, path_of, turn_error

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def scene(rng, n, start):
    """Positions (time, row, column) of n tokens of text and images from ``start`` on, and the next text's."""
    out = []
    while len(out) < n:
        for _ in range(int(rng.integers(1, 6))):
            out.append([start] * 3)
            start += 1
        t, h, w = (int(x) for x in rng.integers(1, 4, 3))
        out += [[start + a, start + b, start + c] for a in range(t) for b in range(h) for c in range(w)]
        start += max(t, h, w)
    out = np.array(out[:n])
    return out, int(out.max()) + 1


@pytest.mark.parametrize("dtype,D,Hq,Hkv,inter,window,gc,page,four", [
    ("bf16", 128, 8, 2, False, 0, 1, 16, True), ("bf16", 64, 4, 4, True, 45, 1, 32, True), ("bf16", 96, 6, 2, False, 70, 3, 64, True),
    ("f32", 64, 4, 2, False, 0, 4, 16, True), ("f32", 96, 2, 1, True, 30, 1, 16, True), ("bf16", 64, 8, 2, False, 0, 1, 16, False)])
def test_run(dtype, D, Hq, Hkv, inter, window, gc, page, four):
    gen, rng, dt = torch.Generator().manual_seed(21), np.random.default_rng(21), DT[dtype]
    T, b, L, V, S, steps = 2, 4, 2, 50, 75, 7
    plen = [21, 34]
    scale = 1.0 / D ** 0.5
    freq = (10000.0 ** (-torch.arange(0, 32, 2, dtype=torch.float64) / 32)).float().cuda()
    axis = np.array([0, 1, 2, 1, 0, 2, 2, 1, 0, 0, 1, 2, 2, 2, 1, 0])
    rope = B.RopeAxes(freq, axis, inter)
    dec = B.TrieDecoder(T, b, 120, V, L, Hq, Hkv, D, window, dtype, gc_interval=gc)

    def raw(*lead):
        return [torch.randn(lead + (h, D), generator=gen).to(dt).cuda() for h in (Hq, Hkv, Hkv)]

    def dev(x):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()

    def turned(x, pos):
        return turn_axes(x, pos, freq, axis, inter), turn_error(x, freq, inter, dt)

    def seen_by(q, k, v, seen, out, what):
        at = torch.nonzero(seen).view(-1)
        want, tol = attend(q[None], k[:, at], v[:, at], torch.ones(1, len(at), dtype=torch.bool), scale, dt)
        check(out[None], want, tol, what)

    # the prefix, in chunks of odd sizes
    used = -(-S // page)
    pages = rng.permutation(used + 2)[:used]
    if four:
        pools = [torch.full((used + 2, L, Hkv, page, D // per), 255, dtype=torch.uint8, device="cuda") for per in (2, 32, 2, 32)]
        dec.set_prefix4(*pools, pages, S)
    else:
        pools = [torch.full((used + 2, L, Hkv, page, D), float("nan"), dtype=dt, device="cuda") for _ in range(2)]
        dec.set_prefix(*pools, pages, S)
    where, after = scene(rng, S, 0)
    assert after < S  # (images take fewer positions than tokens)
    pq, pk, pv = raw(L, S)
    pout, prot = torch.empty_like(pq), torch.empty_like(pq)
    for a, e in ((0, 33), (33, 34), (34, S)):
        at = dev(where[a:e])
        for l in range(L):
            rq = torch.empty((1, e - a, Hq, D), dtype=dt, device="cuda")
            dec.prefix_store(l, 1, a, pk[l:l + 1, a:e], pv[l:l + 1, a:e], pq[l:l + 1, a:e], rq, rope, positions=at)
            dec.prefix_attn(l, 1, a, rq, ro := torch.empty_like(rq), scale)
            prot[l, a:e], pout[l, a:e] = rq[0], ro[0]
    kb, vb = torch.empty_like(pk), torch.empty_like(pv)
    dec.prefix_load(0, L, 0, kb, vb)
    prefix = []
    for l in range(L):
        want, tol = turned(pk[l], where)
        if four:
            assert torch.equal(kb[l].double().cpu(), values64(*pack64(want)))
            assert torch.equal(vb[l].double().cpu(), values64(*pack64(pv[l])))
        else:
            check(kb[l], want, tol, "prefix k")
            assert torch.equal(vb[l], pv[l])
        check(prot[l], *turned(pq[l], where), "prefix q")
        k, v = kb[l].double().cpu().transpose(0, 1), vb[l].double().cpu().transpose(0, 1)
        prefix.append((k, v))
        for j in (0, 32, 33, 34, 60, S - 1):
            seen_by(prot[l, j], k, v, (torch.arange(S) <= j) & (torch.arange(S) > j - (window or S)), pout[l, j], ("prefix", l, j))

    # the prompts
    most = max(plen)
    dec.init_prompt(plen, torch.zeros((T, most), dtype=torch.int32, device="cuda"))
    qs = torch.full((T, most), -1, dtype=torch.int32, device="cuda")
    given, shift = np.zeros((T, most, 3), int), np.zeros((T, 3), int)
    for t, n in enumerate(plen):
        qs[t, :n] = torch.arange(n, device="cuda")
        given[t, :n - 1], end = scene(rng, n - 1, after)
        given[t, n - 1] = end  # (the last token is text)
        shift[t] = end - (S + n - 1)
    node_pos = [{j: given[t, j] for j in range(plen[t])} for t in range(T)]
    q, k, v = raw(L, T, most)
    raws = [[{j: (k[l, t, j], v[l, t, j]) for j in range(plen[t])} for t in range(T)] for l in range(L)]
    rot, out = torch.empty_like(q), torch.zeros_like(q)
    for l in range(L):
        dec.store_kv(l, 1, k[l:l + 1], v[l:l + 1], q[l:l + 1], rot[l:l + 1], rope, qs, positions=dev(given))
        if dtype == "bf16":
            dec.tree_attn(l, 1, qs, rot[l], out[l], scale)

    def nodes(l, t, st):
        """Keys and values the trie's node n sees: the prefix's, then the stored nodes'."""
        at = slice(st["base"], st["base"] + st["n_nodes"])
        kk, vv = dec.k_pool[t, l, :, at].cpu(), dec.v_pool[t, l, :, at].cpu()
        own = [raws[l][t][int(i)] for i in st["node_id"]]
        rk = torch.stack([x[0] for x in own])
        check(kk.transpose(0, 1), *turned(rk, np.stack([node_pos[t][int(i)] for i in st["node_id"]])), ("k", l, t))
        assert torch.equal(vv.transpose(0, 1), torch.stack([x[1] for x in own]).cpu())
        return torch.cat([prefix[l][0], kk.double()], 1), torch.cat([prefix[l][1], vv.double()], 1)

    def sees(st, n):
        d = st["depth"]
        seen = torch.cat([torch.ones(S, dtype=torch.bool), torch.from_numpy(path_of(st, n))])
        if window:  # (by where rows are stored, not by their positions)
            at = torch.cat([torch.arange(S), torch.from_numpy(S + d)])
            seen &= S + int(d[n]) - at < window
        return seen

    for t in range(T):
        st = dec.read_state(t)
        for l in range(L):
            kk, vv = nodes(l, t, st)
            check(rot[l, t, :plen[t]], *turned(q[l, t, :plen[t]], given[t, :plen[t]]), "prompt q")
            assert bool((rot[l, t, plen[t]:] == 0).all())
            if dtype == "bf16":
                for j in (0, 1, 13, plen[t] - 1):
                    seen_by(rot[l, t, j], kk, vv, sees(st, j), out[l, t, j], ("prompt", l, t, j))

    # the steps
    sel = [torch.zeros((T, b), dtype=x, device="cuda") for x in (torch.int32, torch.int32, torch.float32, torch.float32)]
    moved = dev(shift)
    q, k, v = raw(L, T, b)
    rot, out = torch.empty_like(q), torch.empty_like(q)

    def step_calls(first):
        for l in range(L):
            dec.store_kv(l, 1, None if first else k[l:l + 1], None if first else v[l:l + 1], q[l:l + 1], rot[l:l + 1], rope, shift=moved)
            dec.attn_decode(l, 1, rot[l], None, None, out[l], scale)

    for step in range(steps):
        log(f"media run {dtype} d={D} W={window} g={gc} step {step}")
        for x, y in zip((q, k, v), raw(L, T, b)):
            x.copy_(y)
        rot.fill_(9.0), out.fill_(9.0)
        step_calls(step == 0)  # (at first the prompt's last token: its row is stored, its query comes again)
        for t in range(T):
            st = dec.read_state(t)
            if step:
                for j in range(b):
                    leaf = int(st["leaf_slot"][j])
                    node = int(st["node_id"][leaf])
                    node_pos[t][node] = S + int(st["depth"][leaf]) + shift[t]
                    for l in range(L):
                        raws[l][t][node] = (k[l, t, j].clone(), v[l, t, j].clone())
            assert st["kv_pending"] == 0
            for l in range(L):
                kk, vv = nodes(l, t, st)
                for j in range(b):
                    if j >= st["n_live"]:
                        assert bool((out[l, t, j] == 0).all()) and bool((rot[l, t, j] == 0).all())
                        continue
                    leaf = int(st["leaf_slot"][j])
                    pos = (S + int(st["depth"][leaf]) + shift[t])[None]
                    assert step or int(pos[0, 0]) == int(given[t, plen[t] - 1, 0])
                    check(rot[l, t, j][None], *turned(q[l, t, j][None], pos), "q")
                    seen_by(rot[l, t, j], kk, vv, sees(st, leaf), out[l, t, j], (step, l, t, j))
        dec.topk_append((torch.randn((T, b, V), generator=gen) * 3).cuda(), *sel)
    # the last leaves, by the same calls captured and replayed on other inputs and shifts, with eager calls between
    step_calls(False)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step_calls(False)
    for i in range(3):
        for x, y in zip((q, k, v), raw(L, T, b)):
            x.copy_(y)
        moved.copy_(dev(shift + i))
        rot.fill_(9.0), out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (rot, out, dec.k_pool, dec.v_pool)]
        step_calls(False)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (rot, out, dec.k_pool, dec.v_pool))), i
        for t in range(T):
            st = dec.read_state(t)
            for j in range(b):
                pos = (S + int(st["depth"][int(st["leaf_slot"][j])]) + shift[t] + i)[None]
                check(rot[0, t, j][None], *turned(q[0, t, j][None], pos), "q replayed")
    assert dec.status() == 0
    dec.close()
