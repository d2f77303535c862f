"""Shared prefix, whole outputs against 64 bits where a call runs as several launches (workspaces that hold
only a part of its layers or queries), NaN and infinity in the tries' own rows beside a prefix, and captured
stores and prompts."""
import numpy as np
import pytest
import torch

import paper_2502_00085_amd.binding as B
from gpu_harness import log
from prefix_ref import HALF_F32, Prefix, attend, check, half_step, path_of, turn, turn_error
from test_gpu_prefix_attn import Batch, randn

pytestmark = pytest.mark.gpu


def attend_all(q, k, v, seen, scale, dtype):
    """prefix_ref.attend for many rows at once, on the device: q [n][Hq][d], k / v [Hkv][m][d], seen [n][m]
    (a key or more in every row).  The same bound, with sum p |v - o| <= sum p |v| + |o|."""
    n, Hq, d = q.shape
    G = Hq // k.shape[0]
    h = half_step(dtype)
    out = torch.empty((n, Hq, d), dtype=torch.float64, device="cuda")
    tol = torch.empty_like(out)
    chain = (seen.sum(1).double() / 32 + 64)[:, None] * HALF_F32
    for x in range(Hq):
        qi, kk, vv = q[:, x].double(), k[x // G].double(), v[x // G].double()
        s = torch.matmul(qi, kk.t().contiguous()).mul_(scale).masked_fill_(~seen, -torch.inf)
        p = torch.softmax(s, -1)
        o = torch.matmul(p, vv)
        size = torch.matmul(qi.abs(), kk.abs().t().contiguous()).masked_fill_(~seen, 0.0).amax(1, keepdim=True) * scale
        score = (d + 4) * HALF_F32 * size * 1.5 + 4 * HALF_F32
        around = torch.matmul(p, vv.abs())
        out[:, x] = o
        tol[:, x] = ((h if dtype == torch.bfloat16 else 0.0) + 2 * score) * 1.01 * (around + o.abs()) + 2 * chain * around + h * 1.01 * o.abs() + 1e-30
    return out, tol


def stored_prefix(p, layer):
    """K and V of the prefix's positions in order, on the device: [Hkv][positions][d] each."""
    at = torch.arange(p.length, device="cuda")
    page = torch.from_numpy(p.pages).cuda().long()[at // p.page]
    return [pool[page, layer, :, at % p.page].transpose(0, 1) for pool in (p.k, p.v)]


def check_nodes(dec, prefix, layer, trie, state, slots, q, out, scale, what):
    """Rows `out` of the live nodes at `slots`, every one, over the prefix and their own paths (no window)."""
    n, base = state["n_nodes"], state["base"]
    own = [pool[trie, layer, :, base:base + n] for pool in (dec.k_pool, dec.v_pool)]
    k, v = (torch.cat(x, 1) for x in zip(stored_prefix(prefix, layer), own))
    seen = torch.from_numpy(np.stack([np.r_[np.ones(prefix.length, bool), path_of(state, int(x))] for x in slots])).cuda()
    want, tol = attend_all(q, k, v, seen, scale, q.dtype)
    check(out, want.cpu(), tol.cpu(), what)


@pytest.mark.parametrize("L,D,Hq,Hkv,S,page,prompts", [
    (2, 128, 64, 4, 100, 64, (1100, 900)),  # 1,024 queries of a layer per launch, and the other 76
    (17, 64, 64, 64, 70, 16, (500,))])      # 8 layers per launch, 8, and 1
def test_prompts_in_several_launches(L, D, Hq, Hkv, S, page, prompts):
    bt = Batch("bf16", D, Hq, Hkv, S, page, [(n, 0) for n in prompts], 1, L=L)
    most = max(prompts)
    slots = np.full((bt.T, most), -1, np.int32)
    for t, n in enumerate(prompts):
        slots[t, :n] = np.arange(n)
    q = randn(bt.gen, (L, bt.T, most, Hq, D), bt.dt)
    out = torch.full_like(q, float("nan"))
    bt.dec.tree_attn(0, L, torch.from_numpy(slots).cuda(), q, out, bt.scale)
    for l in range(L):
        log(f"prompts layer {l}")
        for t, n in enumerate(prompts):
            assert bool((out[l, t, n:] == 0).all())
            check_nodes(bt.dec, bt.prefix, l, t, dict(bt.tries[t], base=0), range(n), q[l, t, :n], out[l, t, :n], bt.scale, (l, t))
    assert bt.dec.status() == 0


def test_drafts_in_several_launches():
    """15 layers per launch: the newest nodes of 16 tries, some without a query."""
    L, D, Hq, Hkv, n = 18, 64, 64, 8, 15
    bt = Batch("bf16", D, Hq, Hkv, 75, 32, [(20 + t, 2) for t in range(16)], 5, L=L)
    slots = np.full((16, n), -1, np.int32)
    for t, s in enumerate(bt.tries):
        m = n - t % 3
        slots[t, :m] = np.arange(s["n_nodes"] - m, s["n_nodes"])
    q = randn(bt.gen, (L, 16, n, Hq, D), bt.dt)
    out = torch.full_like(q, float("nan"))
    bt.dec.tree_attn(0, L, torch.from_numpy(slots).cuda(), q, out, bt.scale)
    for l in range(L):
        log(f"drafts layer {l}")
        for t, s in enumerate(bt.tries):
            m = n - t % 3
            assert bool((out[l, t, m:] == 0).all())
            check_nodes(bt.dec, bt.prefix, l, t, dict(s, base=0), slots[t, :m], q[l, t, :m], out[l, t, :m], bt.scale, (l, t))
    assert bt.dec.status() == 0


def test_decode_in_several_launches():
    """fp32, a layer of 34 MB of records per launch."""
    L, D, Hq, Hkv, b = 3, 256, 64, 8, 32
    bt = Batch("f32", D, Hq, Hkv, 70, 16, [(2 + t % 3, 1) for t in range(16)], b, L=L)
    q = randn(bt.gen, (L, 16, b, Hq, D), bt.dt)
    out = torch.full_like(q, float("nan"))
    bt.dec.attn_decode(0, L, q, None, None, out, bt.scale)
    for l in range(L):
        for t, s in enumerate(bt.tries):
            check_nodes(bt.dec, bt.prefix, l, t, dict(s, base=0), s["leaf_slot"], q[l, t], out[l, t], bt.scale, (l, t))
    assert bt.dec.status() == 0


@pytest.mark.parametrize("gc", [1, 2])
def test_steps_in_several_launches(gc):
    """Decode steps that collect and move rows, 15 layers per launch, the leaves' rows stored by the call: the
    pools are those of one-layer calls, bit for bit, and every output is right."""
    gen, rng = torch.Generator().manual_seed(13), np.random.default_rng(13)
    L, T, b, Hq, Hkv, D, V, dt = 20, 16, 16, 64, 8, 64, 200, torch.bfloat16
    decs = [B.TrieDecoder(T, b, 160, V, L, Hq, Hkv, D, gc_interval=gc) for _ in range(2)]
    prefix = Prefix(gen, rng, L, Hkv, D, dt, 40, 16)
    pk, pv = (randn(gen, tuple(decs[0].k_pool.shape), dt) for _ in range(2))
    plen = [9 + t for t in range(T)]
    for d in decs:
        d.k_pool.copy_(pk)
        d.v_pool.copy_(pv)
        d.init_prompt(plen, torch.zeros((T, max(plen)), dtype=torch.int32, device="cuda"))
        prefix.attach(d)
    sel = [[torch.zeros((T, b), dtype=x, device="cuda") for x in (torch.int32, torch.int32, torch.float32, torch.float32)] for _ in decs]
    moved = 0
    for step in range(5):
        log(f"steps g={gc} step {step}")
        q, k, v = (randn(gen, (L, T, b, h, D), dt) for h in (Hq, Hkv, Hkv))
        if step == 0:
            k = v = None
        out = [torch.full_like(q, float("nan")) for _ in decs]
        decs[0].attn_decode(0, L, q, k, v, out[0], 0.125)
        for l in range(L):
            decs[1].attn_decode(l, 1, q[l], None if k is None else k[l], None if v is None else v[l], out[1][l], 0.125)
        assert torch.equal(decs[0].k_pool, decs[1].k_pool) and torch.equal(decs[0].v_pool, decs[1].v_pool), step
        states = [decs[0].read_state(t) for t in range(T)]
        for l in (0, 14, 15, L - 1):
            for t, st in enumerate(states):
                for o in out:
                    assert bool((o[l, t, st["n_live"]:] == 0).all())
                    check_nodes(decs[0], prefix, l, t, st, st["leaf_slot"], q[l, t, :st["n_live"]], o[l, t, :st["n_live"]], 0.125, (step, l, t))
        for o in out:
            assert bool(torch.isfinite(o).all())
        logits = (torch.randn((T, b, V), generator=gen) * 3).cuda()
        for d, s in zip(decs, sel):
            d.topk_append(logits, *s)
        moved += sum(st["n_nodes"] + b > decs[0].read_state(t)["n_nodes"] for t, st in enumerate(states))
    assert moved > 0  # (some appends collected nodes)
    assert [d.status() for d in decs] == [0, 0]
    for d in decs:
        d.close()


# 32, 64 and 128 query rows per block in the launch that also takes the tries' nodes; ranks past 32
@pytest.mark.parametrize("D,Hq,Hkv,b,tries", [(128, 8, 2, 4, [(70, 5)]), (64, 8, 2, 8, [(30, 6), (90, 3)]), (96, 4, 1, 40, [(50, 3), (129, 2)]),
                                              (128, 16, 4, 40, [(100, 3)])])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_bad_rows_of_the_tries(D, Hq, Hkv, b, tries, bad):
    """NaN or infinities in K and V of dead nodes, of slots past the last node and of nodes that one beam
    sees, where the prefix's launch takes the tries' nodes: the other beams are as exact as ever, and that
    beam's rows are not finite."""
    log(f"bad rows d={D} b={b} bad={bad}")
    bt = Batch("bf16", D, Hq, Hkv, 150, 32, tries, b, dead=True)
    hit = []
    for t, s in enumerate(bt.tries):
        n, nl = s["n_nodes"], s["n_live"]
        owner = (nl - 1, 0)[t % 2]
        rows = [int(x) for x in np.nonzero(s["mask"] == 0)[0]] + list(range(n, bt.dec.k_pool.shape[3]))
        assert rows[0] < n  # (there are dead nodes)
        rows += [int(x) for x in np.nonzero(s["mask"] == np.uint64(1 << owner))[0]]  # (its leaf at least)
        hit.append(owner)
        bt.dec.k_pool[t, :, :, rows, ::3] = bad
        bt.dec.v_pool[t, :, :, rows] = bad
    q = randn(bt.gen, (1, bt.T, b, Hq, D), bt.dt)
    out = torch.full_like(q, 5.0)
    bt.dec.attn_decode(0, 1, q, None, None, out, bt.scale)
    for t, s in enumerate(bt.tries):
        for j in range(b):
            if j == hit[t]:
                assert not bool(torch.isfinite(out[0, t, j]).any()), (t, j)
            else:
                want, tol = bt.expect(q[0, t, j], 0, t, int(s["leaf_slot"][j]))
                check(out[0, t, j][None], want, tol, (t, j))
    assert bt.dec.status() == 0


@pytest.mark.parametrize("splits", ["1", "2", ""])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_bad_rows_past_the_nodes(monkeypatch, splits, bad):
    """Slots that hold no node may hold anything, in every launch that takes the tries' nodes."""
    if splits:  # (a launch of its own, unsplit or not)
        monkeypatch.setenv("TD_ATTN_SPLITS", splits)
    bt = Batch("bf16", 128, 8, 2, 150, 32, [(70, 5), (33, 3)], 4)
    for t, s in enumerate(bt.tries):
        bt.dec.k_pool[t, :, :, s["n_nodes"]:] = bad
        bt.dec.v_pool[t, :, :, s["n_nodes"]:] = bad
    bt.decode()
    slots = np.stack([np.r_[np.arange(s["n_nodes"] - 9, s["n_nodes"]), [s["n_nodes"], -1]] for s in bt.tries])
    bt.tree(slots)
    most = min(s["n_nodes"] for s in bt.tries)
    bt.tree(np.stack([np.arange(s["n_nodes"] - most, s["n_nodes"]) for s in bt.tries]), sample=0.2)


def test_graph_of_prompts_and_stores():
    """Captured stores (of the prefix and of nodes) and prompts (both layouts), replayed behind prefixes of other
    lengths with eager work between: each replay is what the eager calls give."""
    dt, L, T = torch.bfloat16, 2, 2
    bt = Batch("bf16", 128, 8, 2, 200, 32, [(60, 3), (45, 2)], 4, L=L)
    most = max(s["n_nodes"] for s in bt.tries)
    slots = np.full((T, most), -1, np.int32)
    for t, s in enumerate(bt.tries):
        slots[t, :s["n_nodes"]] = np.arange(s["n_nodes"])
    qs = torch.from_numpy(slots).cuda()
    few = qs[:, 30:39].contiguous()
    q, k, v = (randn(bt.gen, (L, T, most, h, 128), dt) for h in (8, 2, 2))
    fq = randn(bt.gen, (L, T, 9, 8, 128), dt)
    pk, pv = (randn(bt.gen, (L, 50, 2, 128), dt) for _ in range(2))
    rope = B.Rope(torch.linspace(1.0, 0.01, 64, device="cuda"))
    rot, out, fout = torch.empty_like(q), torch.empty_like(q), torch.empty_like(fq)

    def step():
        bt.dec.prefix_store(0, L, 10, pk, pv, rope=rope)
        bt.dec.store_kv(0, L, k, v, q, rot, rope, qs)
        bt.dec.tree_attn(0, L, qs, rot, out, bt.scale)
        bt.dec.tree_attn(0, L, few, fq, fout, bt.scale)

    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    longer = Prefix(bt.gen, bt.rng, L, 2, 128, dt, 700, 64)
    for name, p, length in (("same", bt.prefix, 200), ("longer", longer, 700), ("shorter", bt.prefix, 90), ("none seen", longer, 0), ("same again", bt.prefix, 200)):
        p.attach(bt.dec, length)
        results = []
        for run in (graph.replay, step, graph.replay):
            for x in (rot, out, fout):
                x.fill_(9.0)
            p.k[:, :, :, 5] = 1.0  # (eager work between)
            run()
            torch.cuda.synchronize()
            results.append([x.clone() for x in (rot, bt.dec.k_pool, bt.dec.v_pool, p.k, p.v, out, fout)])
        for i, (a, e, c) in enumerate(zip(*results)):
            assert torch.equal(a, c), (name, i)
            if i < 5:
                assert torch.equal(a, e), (name, i)
            else:  # (eager calls may split otherwise)
                assert float((a.float() - e.float()).abs().max()) <= 4 * 2.0 ** -8 * float(e.float().abs().max()), (name, i)
    assert bt.dec.status() == 0


def test_a_row_alone():
    """attend_all (above) against prefix_ref.attend: the same values."""
    gen = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(x, generator=gen).to(torch.bfloat16) for x in ((4, 6, 32), (2, 50, 32), (2, 50, 32)))
    seen = torch.ones(4, 50, dtype=torch.bool)
    seen[1, 20:] = False
    seen[2, :49] = False
    a, _ = attend(q, k, v, seen, 0.2, torch.bfloat16)
    c, _ = attend_all(q.cuda(), k.cuda(), v.cuda(), seen.cuda(), 0.2, torch.bfloat16)
    assert float((a - c.cpu()).abs().max()) < 1e-12


def test_graph_behind_a_shorter_table():
    """Captured calls, replayed when the table has become shorter or the prefix is detached: positions that
    it no longer has are not stored (the sticky status says so) and not seen, nodes are at their depths."""
    gen, rng, dt = torch.Generator().manual_seed(21), np.random.default_rng(21), torch.bfloat16
    dec = B.TrieDecoder(1, 2, 40, 50, 1, 4, 2, 64)
    dec.init_prompt([9], torch.zeros((1, 9), dtype=torch.int32, device="cuda"))
    full = Prefix(gen, rng, 1, 2, 64, dt, 100, 16)
    full.attach(dec)
    k, v, q = randn(gen, (1, 30, 2, 64), dt), randn(gen, (1, 30, 2, 64), dt), randn(gen, (1, 30, 4, 64), dt)
    lk, lq = randn(gen, (1, 1, 2, 2, 64), dt), randn(gen, (1, 1, 2, 4, 64), dt)
    rope = B.Rope(torch.linspace(1.0, 0.01, 32, device="cuda"))
    rot, out, lrot, lout = torch.empty_like(q), torch.empty_like(q), torch.empty_like(lq), torch.empty_like(lq)

    def step():
        dec.prefix_store(0, 1, 40, k, v, q, rot, rope)
        dec.prefix_attn(0, 1, 40, rot, out, 0.125)
        dec.store_kv(0, 1, lk, lk, lq, lrot, rope)
        dec.attn_decode(0, 1, lrot, None, None, lout, 0.125)

    step()
    torch.cuda.synchronize()
    assert dec.status() == 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    for room in (48, 16, 0, 112):
        if room:
            dec.set_prefix(full.k, full.v, full.pages[:room // 16], min(100, room))
        else:
            dec.set_prefix(None)
        full.k.fill_(0.5)
        full.v.copy_(randn(gen, tuple(full.v.shape), dt))
        for x in (rot, out, lrot, lout):
            x.fill_(9.0)
        before = full.v.clone()
        for _ in range(2):
            graph.replay()
        n = min(30, max(0, room - 40))  # positions of the call that the table still has
        assert dec.status() == (0 if n == 30 else B.TD_EINVAL)
        assert dec.status() == 0
        stored = torch.zeros(full.v.shape[:4], dtype=torch.bool, device="cuda")
        for j in range(n):
            stored[int(full.pages[(40 + j) // 16]), :, :, (40 + j) % 16] = True
            assert torch.equal(full.v[int(full.pages[(40 + j) // 16]), 0, :, (40 + j) % 16], v[0, j])
        assert torch.equal(full.v[~stored], before[~stored])
        assert bool((rot[:, n:] == 0).all()) and not bool((rot[:, :n] == 0).all(-1).any())
        kk, vv = (torch.stack([x[int(full.pages[p // 16]), 0, :, p % 16] for p in range(room)], 1) if room else x[0, 0][:, :0] for x in (full.k, full.v))
        for j in (0, 7, 8, 29):
            m = min(40 + j + 1, room)
            if m == 0:
                assert bool((out[0, j] == 0).all())
                continue
            want, tol = attend(rot[0, j:j + 1], kk[:, :m], vv[:, :m], torch.ones(1, m, dtype=torch.bool), 0.125, dt)
            check(out[0, j:j + 1], want, tol, (room, j))
        at = min(100, room)
        ok, ov = (torch.cat([a[:, :at], pool[0, 0, :, :9]], 1) for a, pool in ((kk, dec.k_pool), (vv, dec.v_pool)))
        want, tol = attend(lrot[0, 0, :1], ok, ov, torch.ones(1, at + 9, dtype=torch.bool), 0.125, dt)
        check(lout[0, 0, :1], want, tol, room)
        check(lrot[0, 0, :1], turn(lq[0, 0, :1], [at + 8], rope.freq, False), turn_error(lq[0, 0, :1], rope.freq, False, dt), room)
    dec.close()
