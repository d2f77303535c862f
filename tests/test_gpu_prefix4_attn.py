"""Attention over a shared prefix in 4 bits against 64 bits: decode steps, drafts, prompts and the prefix's own
causal prefill, over types, head dims and layouts, lengths from one position, windows, pages that end inside
a tile, blocks that are NaN in what a row does not see, calls of several launches, captured calls."""
import numpy as np
import pytest
import torch

import paper_2502_00085_amd.binding as B
import test_gpu_prefix_attn as plain
from gpu_harness import log
from prefix4_ref import Prefix4, pack64, values64
from prefix_ref import Prefix, check, path_of
from test_gpu_prefix_attn import randn
from test_gpu_prefix_edges import attend_all

pytestmark = pytest.mark.gpu


class Batch(plain.Batch):
    """T tries behind one prefix in 4 bits."""

    def __init__(self, dtype, D, Hq, Hkv, S, page=16, *a, **kw):
        super().__init__(dtype, D, Hq, Hkv, S, page, *a, **kw)
        self.prefix = Prefix4(self.gen, self.rng, self.L, Hkv, D, S, page)
        self.prefix.attach(self.dec)


class Chunk(plain.Chunk):
    def __init__(self, dtype, D, Hq, Hkv, pos, n, page, window=0, L=1, seed=9, spare=0):
        super().__init__(dtype, D, Hq, Hkv, pos, n, page, window, L, seed, spare)
        self.prefix = Prefix4(self.gen, self.rng, L, Hkv, D, pos + n, page, spare)
        self.prefix.attach(self.dec, 0)


# lengths around the tile of 64 keys, head dims of every kernel, 32, 64 and more rows per KV head
@pytest.mark.parametrize("S", [1, 15, 64, 65, 200, 777])
@pytest.mark.parametrize("dtype,D,Hq,Hkv,b,T,page", [("bf16", 128, 8, 2, 3, 2, 16), ("bf16", 64, 4, 4, 2, 1, 64), ("bf16", 96, 6, 2, 5, 3, 32),
                                                     ("f32", 64, 4, 1, 3, 2, 16), ("f32", 128, 8, 1, 5, 4, 128), ("bf16", 128, 16, 2, 8, 5, 64)])
def test_decode(dtype, D, Hq, Hkv, b, T, page, S):
    log(f"decode4 {dtype} d={D} {Hq}/{Hkv} b={b} T={T} S={S}")
    Batch(dtype, D, Hq, Hkv, S, page, [(5 + 30 * t, 4) for t in range(T)], b).decode(sample=0.5 if T > 2 else None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 96, 160, 192, 224, 256])
@pytest.mark.parametrize("T,b", [(1, 2), (2, 12), (3, 40)])
def test_decode_other_head_dims(dtype, D, T, b):
    log(f"decode4 {dtype} d={D} T={T} b={b}")
    Batch(dtype, D, 3, 1, 330, 32, [(7, 2)] * T, b).decode(sample=0.2)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 96)])
@pytest.mark.parametrize("S", [100, 2000])
def test_decode_vector_alu_kernel(dtype, D, S):
    Batch(dtype, D, 4, 2, S, 16, [(9, 3), (70, 2)], 4, attn_impl=B.TD_ATTN_VALU).decode()


def test_splits_forced(monkeypatch):
    monkeypatch.setenv("TD_ATTN_SPLITS", "5")
    Batch("bf16", 128, 8, 2, 500, 64, [(90, 3), (300, 2)], 4).decode()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("bf16", 32), ("f32", 64)])
@pytest.mark.parametrize("window", [1, 6, 40, 64, 100, 300])
def test_decode_window(dtype, D, window):
    """Tries of several depths behind 130 positions: the window ends in the trie, in the prefix, before it."""
    Batch(dtype, D, 8, 2, 130, 16, [(3, 2), (33, 1), (90, 4), (1, 0)], 4, window=window, dead=True).decode()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_decode_window_tries_of_other_depths(dtype, D):
    Batch(dtype, D, 4, 2, 300, 32, [(1 + 13 * i, 1 + i % 3) for i in range(13)], 2, window=90).decode()
    Batch(dtype, D, 4, 2, 40, 16, [(90, 2), (80, 1)], 3, window=64).decode()  # (nothing for any)


def test_one_live_leaf_and_many_layers():
    bt = Batch("bf16", 128, 8, 2, 300, 64, [(12, 0), (40, 3)], 6, L=5)
    q, out = bt.decode(sample=0.3)
    # layer by layer and in uneven ranges: the same sums in other splits
    for calls in ([(l, 1) for l in range(5)], [(0, 3), (3, 2)]):
        other = torch.empty_like(out)
        for l, n in calls:
            bt.dec.attn_decode(l, n, q[l:l + n], None, None, other[l:l + n], bt.scale)
        assert float((other.float() - out.float()).abs().max()) <= 2 * 2.0 ** -8 * float(out.float().abs().max())


def test_layers_past_the_workspace():
    """Records of a layer of 34 MB: the call runs as several launches."""
    Batch("f32", 256, 64, 8, 70, 16, [(2, 1)] * 16, 32, L=3).decode(sample=0.002)


# where the tries' own nodes go: in the prefix's launch (32, 64 and 128 rows to a block), in a launch whose epilogue
# merges the records, in split launches and a merge
@pytest.mark.parametrize("D,Hq,Hkv,b,tries,S,L", [(128, 8, 2, 4, [(300, 6), (20, 2)], 1500, 1), (128, 8, 2, 6, [(200, 6), (20, 2)], 1500, 1),
                                                  (128, 8, 2, 16, [(100, 3), (20, 2), (64, 1)], 1500, 1), (64, 16, 4, 16, [(200, 8)] * 12, 130, 4),
                                                  (96, 8, 8, 3, [(1500, 4), (90, 2)], 40, 1), (96, 8, 8, 30, [(150, 4), (90, 2)], 400, 1),
                                                  (128, 8, 1, 40, [(30, 2), (64, 1)], 300, 1), (64, 24, 2, 30, [(50, 1)] * 2, 900, 1),
                                                  (64, 4, 4, 20, [(150, 4), (90, 2)], 400, 1), (128, 32, 8, 40, [(30, 3), (64, 1)], 700, 2)])
def test_where_the_nodes_go(D, Hq, Hkv, b, tries, S, L):
    Batch("bf16", D, Hq, Hkv, S, 64, tries, b, L=L, dead=True).decode(sample=0.05 if len(tries) > 3 else 0.3)


@pytest.mark.parametrize("dtype,D", [("bf16", 96), ("bf16", 128), ("bf16", 160), ("bf16", 256), ("f32", 96), ("f32", 192), ("f32", 224)])
@pytest.mark.parametrize("off", [1, 3])
def test_scales_at_any_address(dtype, D, off):
    """Scale bytes that begin at an odd address."""
    bt = Batch(dtype, D, 4, 2, 200, 16, [(9, 2), (20, 1)], 3)
    p = bt.prefix
    keep = []
    for name in ("k", "v"):
        e, s = getattr(p, name)
        moved = torch.zeros(s.numel() + 8, dtype=torch.uint8, device="cuda")[off:off + s.numel()].view(s.shape)
        moved.copy_(s)
        keep.append(s)
        setattr(p, name, (e, moved))
    p.attach(bt.dec)
    for s in keep:
        s.fill_(255)  # (no longer read)
    bt.decode()


def test_fp32_chunk_in_several_launches():
    """More blocks of rows than a launch takes: two launches over the queries.  Rows at either side of the border,
    of the ends, and some between."""
    D, Hkv, G, n, W, page = 32, 8, 8, 530_000, 50, 4096
    dec = B.TrieDecoder(1, 1, 4, 100, 1, Hkv * G, Hkv, D, W, "f32")
    gen, rng = torch.Generator().manual_seed(5), np.random.default_rng(5)
    n_pages = -(-n // page)
    e = [torch.randint(0, 256, (n_pages, 1, Hkv, page, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    s = [torch.randint(124, 128, (n_pages, 1, Hkv, page, 1), dtype=torch.uint8, device="cuda") for _ in range(2)]
    dec.set_prefix4(e[0], s[0], e[1], s[1], range(n_pages), n)
    q = torch.empty((1, n, Hkv * G, D), device="cuda").normal_()
    out = torch.full_like(q, 9.0)
    dec.prefix_attn(0, 1, 0, q, out, 0.2)
    assert dec.status() == 0
    border = (1 << 20) // Hkv * 32 // G
    assert 0 < border < n
    at = [0, 1, 49, 50, border - 1, border, border + 1, n - 1] + [int(x) for x in rng.integers(0, n, 12)]
    for j in at:
        lo = max(0, j - W + 1)
        k, v = (values64(x[lo // page:j // page + 1, 0].transpose(1, 2).flatten(0, 1)[lo % page:lo % page + j - lo + 1],
                         y[lo // page:j // page + 1, 0].transpose(1, 2).flatten(0, 1)[lo % page:lo % page + j - lo + 1]).transpose(0, 1)
                for x, y in zip(e, s))
        want, tol = plain.attend(q[0, j:j + 1], k, v, torch.ones(1, j - lo + 1, dtype=torch.bool), 0.2, torch.float32)
        check(out[0, j:j + 1], want, tol, j)
    assert not bool((out == 9.0).all(-1).any())
    dec.close()


def test_leaves_stored_by_the_call():
    """The leaves' rows with the attention call, beside a prefix in 4 bits."""
    bt = Batch("bf16", 128, 8, 2, 500, 64, [(30, 3), (20, 2)], 4, L=2)
    gen, dt = bt.gen, bt.dt
    sel = [torch.zeros((2, 4), dtype=x, device="cuda") for x in (torch.int32, torch.int32, torch.float32, torch.float32)]
    bt.dec.topk_append(randn(gen, (2, 4, 100), torch.float32), *sel)
    q, k, v = (randn(gen, (2, 2, 4, h, 128), dt) for h in (8, 2, 2))
    out = torch.empty_like(q)
    bt.dec.attn_decode(0, 2, q, k, v, out, bt.scale)
    for t in range(2):
        st = bt.dec.read_state(t)
        assert st["base"] == 0
        bt.tries[t] = st
        for l in range(2):
            for j in range(4):
                slot = int(st["leaf_slot"][j])
                assert torch.equal(bt.dec.k_pool[t, l, :, slot], k[l, t, j])
                want, tol = bt.expect(q[l, t, j], l, t, slot)
                check(out[l, t, j][None], want, tol, (l, t, j))


# drafts (the decode layout) and prompts (the prefill-shaped kernels, short and long key ranges)
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 4, 1), (96, 6, 6)])
@pytest.mark.parametrize("S,window", [(1, 0), (333, 0), (100, 50), (40, 90)])
def test_drafts(D, Hq, Hkv, S, window):
    bt = Batch("bf16", D, Hq, Hkv, S, 32, [(30, 4), (50, 2)], 4, window=window, dead=True)
    slots = np.full((2, 9), -1)
    for t, s in enumerate(bt.tries):
        slots[t, 1:8] = np.arange(s["n_nodes"] - 7, s["n_nodes"])
    slots[1, 0], slots[0, 8] = 12, 2 ** 31 - 1
    bt.tree(slots)


@pytest.mark.parametrize("D,Hq,Hkv,prompts", [(128, 16, 2, (50, 33)), (64, 4, 1, (150, 90)), (96, 12, 2, (64, 65, 7)), (128, 8, 1, (640, 70))])
@pytest.mark.parametrize("S,window", [(1, 0), (500, 0), (130, 60)])
def test_prompts(D, Hq, Hkv, prompts, S, window):
    log(f"prompts4 d={D} S={S} W={window}")
    bt = Batch("bf16", D, Hq, Hkv, S, 64, [(p, 0) for p in prompts], 2, window=window)
    slots = np.full((len(prompts), max(prompts)), -1)
    for t, p in enumerate(prompts):
        slots[t, :p] = np.arange(p)
    bt.tree(slots, sample=0.15)


@pytest.mark.parametrize("L,D,Hq,Hkv,S,prompts", [(2, 128, 64, 4, 100, (1100, 900)), (17, 64, 64, 64, 70, (500,))])
def test_prompts_in_several_launches(L, D, Hq, Hkv, S, prompts):
    """Workspaces that hold only a part of a call's queries, or layers: every row."""
    bt = Batch("bf16", D, Hq, Hkv, S, 64, [(n, 0) for n in prompts], 1, L=L)
    most = max(prompts)
    slots = np.full((bt.T, most), -1, np.int32)
    for t, n in enumerate(prompts):
        slots[t, :n] = np.arange(n)
    q = randn(bt.gen, (L, bt.T, most, Hq, D), bt.dt)
    out = torch.full_like(q, float("nan"))
    bt.dec.tree_attn(0, L, torch.from_numpy(slots).cuda(), q, out, bt.scale)
    for l in range(L):
        log(f"prompts4 layer {l}")
        for t, n in enumerate(prompts):
            s = bt.tries[t]
            k, v = (torch.cat([bt.prefix.rows(pool, l).cuda(), own[t, l, :, :s["n_nodes"]].double()], 1)
                    for pool, own in ((bt.prefix.k, bt.dec.k_pool), (bt.prefix.v, bt.dec.v_pool)))
            seen = torch.from_numpy(np.stack([np.r_[np.ones(S, bool), path_of(s, x)] for x in range(n)])).cuda()
            want, tol = attend_all(q[l, t, :n], k, v, seen, bt.scale, bt.dt)
            check(out[l, t, :n], want.cpu(), tol.cpu(), (l, t))
            assert bool((out[l, t, n:] == 0).all())
    assert bt.dec.status() == 0


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 128, 4, 1), ("bf16", 64, 2, 2), ("bf16", 96, 7, 1), ("f32", 64, 4, 2), ("f32", 128, 2, 1),
                                            ("bf16", 256, 2, 1), ("f32", 160, 1, 1), ("bf16", 32, 3, 3), ("f32", 96, 5, 1), ("f32", 32, 9, 1)])
@pytest.mark.parametrize("pos,n,page,window", [(0, 1, 16, 0), (0, 70, 16, 0), (63, 2, 64, 0), (500, 9, 32, 0), (129, 200, 64, 0), (100, 150, 16, 33),
                                               (700, 3, 128, 64)])
def test_prefix_prefill(dtype, D, Hq, Hkv, pos, n, page, window):
    log(f"chunk4 {dtype} d={D} pos={pos} n={n} W={window}")
    c = Chunk(dtype, D, Hq, Hkv, pos, n, page, window)
    c.verify(c.run(), c.rng.permutation(n)[:24])


def test_prefix_prefill_layers_and_splits():
    c = Chunk("bf16", 128, 8, 2, 3000, 40, 64, L=3)
    c.verify(c.run(), [0, 17, 39])


@pytest.mark.parametrize("dtype,D,Hq,Hkv,pos,n,window,L", [("bf16", 64, 16, 8, 5, 700, 100, 3), ("bf16", 128, 32, 8, 90, 1024, 0, 2),
                                                           ("bf16", 96, 32, 32, 0, 1800, 0, 1), ("f32", 64, 16, 8, 0, 1024, 0, 1)])
def test_prefix_prefill_two_blocks_per_cu(dtype, D, Hq, Hkv, pos, n, window, L):
    """Launches whose blocks are ordered to even out the CUs: every block of every layer is taken."""
    c = Chunk(dtype, D, Hq, Hkv, pos, n, 64, window, L)
    out = c.run()
    assert not (out == 5.0).all(-1).any()
    step = 128 * Hkv // Hq
    c.verify(out, range(step // 2, n, step))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("bf16", 96), ("bf16", 256), ("f32", 64), ("f32", 256)])
@pytest.mark.parametrize("n,G", [(90, 4), (20, 1), (13, 4)])
def test_what_a_row_does_not_see(dtype, D, n, G):
    """A chunk whose last keys have blocks of NaN in K and V: earlier rows do not see them and are as exact as
    ever; rows that see them are not finite.  So are pages past the end and other pages."""
    c = Chunk(dtype, D, G, 1, 40, n, 32, spare=70)
    p = c.prefix
    last = c.pos + n - 1
    first_bad = last - 5
    for pos in (first_bad, last):
        p.k[1][int(p.pages[pos // 32]), :, :, pos % 32, ::3] = 255
        p.v[1][int(p.pages[pos // 32]), :, :, pos % 32] = 255
    other = np.setdiff1d(np.arange(p.k[0].shape[0]), p.pages)
    for pool in (p.k, p.v):
        for pos in range(last + 1, len(p.pages) * 32):
            pool[1][int(p.pages[pos // 32]), :, :, pos % 32] = 255
        pool[1][other] = 255
    out = c.run()
    c.verify(out, range(first_bad - c.pos))
    assert not bool(torch.isfinite(out[0, first_bad - c.pos:]).all(-1).any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_hides_bad_rows(dtype):
    bt = Batch(dtype, 64, 4, 2, 150, 16, [(3, 2), (40, 1)], 4, window=60)
    p = bt.prefix
    for pos in range(0, 150 + 4 - 60):  # before the shallower trie's window
        p.v[1][int(p.pages[pos // 16]), :, :, pos % 16] = 255
    # (the deeper trie's rows see none of positions up to 150 + 40 - 60)
    for pos in range(150 + 4 - 60, 150 + 40 - 60):
        p.v[1][int(p.pages[pos // 16]), :, :, pos % 16, 0] = 255
    q = randn(bt.gen, (1, 2, 4, 4, 64), bt.dt)
    out = torch.empty_like(q)
    bt.dec.attn_decode(0, 1, q, None, None, out, bt.scale)
    s = bt.tries[1]
    for j in range(4):
        want, tol = bt.expect(q[0, 1, j], 0, 1, int(s["leaf_slot"][j]))
        check(out[0, 1, j][None], want, tol, j)
    assert not bool(torch.isfinite(out[0, 0, :, :, :32]).any()) and bool(torch.isfinite(out[0, 0, :, :, 32:]).all())


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_large_scores(dtype, D):
    """Scores over hundreds of powers of two, rising and falling along the keys."""
    bt = Batch(dtype, D, 4, 1, 400, 32, [(6, 2), (30, 2)], 4)
    for pos in range(400):
        bt.prefix.k[1][int(bt.prefix.pages[pos // 32]), :, :, pos % 32] += 2 * min(pos, 399 - pos) // 50
    bt.decode()


def test_graph_reads_the_attached_prefix():
    """Captured stores and attention, replayed behind the same, a longer, a shorter and no prefix, and one of the
    other kind, with eager work between: each replay is what the eager calls give, or sees nothing of the
    prefix and says so."""
    dt = torch.bfloat16
    bt = Batch("bf16", 128, 8, 2, 200, 32, [(20, 3), (35, 2)], 4, L=2)
    q, k, v = (randn(bt.gen, (2, 2, 4, h, 128), dt) for h in (8, 2, 2))
    rope = B.Rope(torch.linspace(1.0, 0.01, 64, device="cuda"))
    pc = randn(bt.gen, (2, 5, 8, 128), dt)
    rot, out, chunk = torch.empty_like(q), torch.empty_like(q), torch.empty_like(pc)

    def step():
        bt.dec.store_kv(0, 2, k, v, q, rot, rope)
        bt.dec.attn_decode(0, 2, rot, None, None, out, bt.scale)
        bt.dec.prefix_attn(0, 2, 30, pc, chunk, bt.scale)

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    longer = Prefix4(bt.gen, bt.rng, 2, 2, 128, 1111, 64)
    other = Prefix(bt.gen, bt.rng, 2, 2, 128, dt, 150, 32)
    tol = 4 * 2.0 ** -8  # (eager calls may split otherwise)
    for name, attach in (("same", lambda: None), ("longer", lambda: longer.attach(bt.dec)), ("shorter", lambda: bt.prefix.attach(bt.dec, 70)),
                         ("none", lambda: longer.attach(bt.dec, 0)), ("same again", lambda: bt.prefix.attach(bt.dec))):
        attach()
        for x in (rot, out, chunk):
            x.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (rot, out, chunk, bt.dec.k_pool)]
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], rot) and torch.equal(got[3], bt.dec.k_pool), name
        for a, c in ((got[1], out), (got[2], chunk)):
            assert float((a.float() - c.float()).abs().max()) <= tol * float(c.float().abs().max()), name
        assert bt.dec.status() == 0, name
    # a prefix of the other kind: the replay has its positions for the rows, and none of its keys
    other.attach(bt.dec)
    graph.replay()
    torch.cuda.synchronize()
    assert bt.dec.status() == B.TD_EINVAL
    turned, alone = rot.clone(), out.clone()
    assert bool((chunk == 0).all())
    bt.dec.store_kv(0, 2, k, v, q, rot, rope)
    assert torch.equal(turned, rot)
    bt.dec.set_prefix(None)
    bt.dec.attn_decode(0, 2, rot, None, None, out, bt.scale)
    assert float((alone.float() - out.float()).abs().max()) <= tol * float(out.float().abs().max())
    assert bt.dec.status() == 0
    bt.prefix.attach(bt.dec)
    graph.replay()
    torch.cuda.synchronize()
    got = out.clone()
    step()
    assert float((got.float() - out.float()).abs().max()) <= tol * float(out.float().abs().max())
    assert bt.dec.status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_kinds_in_turn(dtype):
    """Prefixes of both kinds, attached one after the other to one context: each as if it were the only one.  The
    plain one holds what the 4-bit one stands for: the same outputs but for the order of sums."""
    dt = plain.DT[dtype]
    bt = Batch(dtype, 64, 4, 2, 300, 32, [(20, 3), (35, 2)], 4, L=2)
    same = Prefix(bt.gen, bt.rng, 2, 2, 64, dt, 300, 16)
    q = randn(bt.gen, (2, 2, 4, 4, 64), dt)
    outs = []
    for i in range(4):
        if i % 2:
            same.attach(bt.dec)
        else:
            bt.prefix.attach(bt.dec)
            k, v = torch.empty((2, 300, 2, 64), dtype=dt, device="cuda"), torch.empty((2, 300, 2, 64), dtype=dt, device="cuda")
            bt.dec.prefix_load(0, 2, 0, k, v)
            same.attach(bt.dec)
            bt.dec.prefix_store(0, 2, 0, k, v)
            bt.prefix.attach(bt.dec)
        outs.append(torch.full_like(q, 9.0))
        bt.dec.attn_decode(0, 2, q, None, None, outs[-1], bt.scale)
    assert torch.equal(outs[2], outs[0]) and torch.equal(outs[3], outs[1])
    # (the same sums in another order: two roundings of either output and of its weights)
    h = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -16
    assert float((outs[1].float() - outs[0].float()).abs().max()) <= 4 * h * float(outs[0].float().abs().max())
    bt.prefix.attach(bt.dec)
    bt.decode()


def test_another_stream():
    bt = Batch("bf16", 128, 8, 2, 900, 64, [(20, 3)] * 4, 4)
    q = randn(bt.gen, (1, 4, 4, 8, 128), torch.bfloat16)
    want = torch.empty_like(q)
    bt.dec.attn_decode(0, 1, q, None, None, want, bt.scale)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.empty_like(q)
    side.wait_stream(torch.cuda.current_stream())
    bt.dec.attn_decode(0, 1, q, None, None, out, bt.scale, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


def test_kernel_events():
    """The attention's events bracket every launch of a call."""
    bt = Batch("bf16", 128, 8, 2, 900, 64, [(150, 3), (90, 2)], 4, L=2)
    q, out = randn(bt.gen, (2, 2, 4, 8, 128), bt.dt), torch.empty((2, 2, 4, 8, 128), dtype=bt.dt, device="cuda")
    cq = randn(bt.gen, (2, 50, 8, 128), bt.dt)
    for call in (lambda: bt.dec.attn_decode(0, 2, q, None, None, out, bt.scale),
                 lambda: bt.dec.prefix_attn(0, 2, 800, cq, torch.empty_like(cq), bt.scale)):
        call()
        ev = B.KernelEvents()
        B.td_set_kernel_events(bt.dec.ctx, B.TD_PHASE_ATTN, ev.start, ev.stop)
        call()
        assert 0.0 < ev.elapsed_ms() < 50.0
        ev.close()


def test_a_cache_past_32_bits():
    """A pool whose last pages' rows lie past 2^32 bytes and elements: the prefix is in them."""
    n_pages, D, page, S = 1100, 256, 16384, 700
    e = torch.zeros((n_pages, 1, 2, page, D // 2), dtype=torch.uint8, device="cuda")  # 4.6 GB
    s = torch.full((n_pages, 1, 2, page, D // 32), 255, dtype=torch.uint8, device="cuda")
    gen, rng = torch.Generator().manual_seed(3), np.random.default_rng(3)
    c = Chunk("bf16", D, 4, 2, S - 30, 30, page)
    small = c.prefix
    dec = c.dec
    for src, dst in ((small.k[0], e), (small.k[1], s)):
        dst[n_pages - 1] = src[int(small.pages[0])]
    dec.set_prefix4(e, s, e, s, (n_pages - 1,), 0)
    out = c.run()
    k = small.rows(small.k, 0, S)
    for j in (0, 7, 29):
        p = c.pos + j
        want, tol = plain.attend(c.q[0, j:j + 1], k[:, :p + 1], k[:, :p + 1], torch.ones(1, p + 1, dtype=torch.bool), c.scale, c.dt)
        check(out[0, j:j + 1], want, tol, j)
    rows = randn(gen, (1, 3, 2, D), c.dt)
    dec.prefix_store(0, 1, S, rows, rows)  # (k and v share the pages here)
    back = torch.empty_like(rows), torch.empty_like(rows)
    dec.prefix_load(0, 1, S, *back)
    want = values64(*pack64(rows[0]))
    assert torch.equal(back[0][0].double().cpu(), want) and torch.equal(back[1][0].double().cpu(), want)
    assert bool((s[:n_pages - 1] == 255).all())
    dec.close()
