"""Attention over a shared prefix against 64 bits: decode steps, drafts, prompts and the prefix's own
causal prefill, over types, head dims and layouts, lengths from one position, windows that hide part or
all of the prefix, pages that end inside a tile, NaN and infinity in what a row does not see."""
import numpy as np
import pytest
import torch

import paper_2502_00085_amd.binding as B
from gpu_harness import log
from prefix_ref import Prefix, attend, check, grow, path_of

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def randn(gen, shape, dt):
    return torch.randn(shape, generator=gen).to(dt).cuda()


class Batch:
    """T tries behind one prefix, with the outputs and bounds of any of their nodes' queries."""

    def __init__(self, dtype, D, Hq, Hkv, S, page=16, tries=((20, 4),), b=3, L=1, window=0, seed=7, dead=False, attn_impl=0, cap=None):
        self.gen, self.rng, self.dt = torch.Generator().manual_seed(seed), np.random.default_rng(seed), DT[dtype]
        self.L, self.W, self.S, self.b, self.T, self.shape = L, window, S, b, len(tries), (Hq, Hkv, D)
        self.tries = [grow(self.rng, p, n, b, dead) for p, n in tries]
        cap = cap or max(s["n_nodes"] for s in self.tries) + 2 * b
        self.dec = B.TrieDecoder(self.T, b, cap, 100, L, Hq, Hkv, D, window, dtype, attn_impl)
        self.dec.k_pool.copy_(randn(self.gen, tuple(self.dec.k_pool.shape), self.dt))
        self.dec.v_pool.copy_(randn(self.gen, tuple(self.dec.v_pool.shape), self.dt))
        for t, s in enumerate(self.tries):
            self.dec.load_state(t, s)
        self.prefix = Prefix(self.gen, self.rng, L, Hkv, D, self.dt, S, page)
        self.prefix.attach(self.dec)
        self.scale = 1.0 / D ** 0.5

    def expect(self, q, l, t, slot):
        """Query q [Hq][d] of the node: over what it sees."""
        s, p = self.tries[t], self.prefix
        depth = s["depth"]
        pos = self.S + int(depth[slot])
        lo = max(0, pos - self.W + 1) if self.W else 0
        nodes = path_of(s, slot)
        if self.W:
            nodes &= depth[slot] - depth < self.W
        seen = torch.cat([torch.arange(self.S) >= lo, torch.from_numpy(nodes)])
        if (l, t) not in self.__dict__.setdefault("cache", {}):
            n = s["n_nodes"]
            self.cache[l, t] = [torch.cat([p.rows(pool, l), own[t, l, :, :n].cpu()], 1)
                                for pool, own in ((p.k, self.dec.k_pool), (p.v, self.dec.v_pool))]
        k, v = self.cache[l, t]
        at = torch.nonzero(seen).view(-1)  # (hidden rows may hold anything)
        return attend(q[None], k[:, at], v[:, at], torch.ones(1, len(at), dtype=torch.bool), self.scale, self.dt)

    def decode(self, sample=None, calls=None):
        Hq, Hkv, D = self.shape
        q = randn(self.gen, (self.L, self.T, self.b, Hq, D), self.dt)
        out = torch.full_like(q, 5.0)
        for l, n in calls or [(0, self.L)]:
            self.dec.attn_decode(l, n, q[l:l + n], None, None, out[l:l + n], self.scale)
        for l in range(self.L):
            for t, s in enumerate(self.tries):
                for j in range(self.b):
                    if j >= s["n_live"]:
                        assert bool((out[l, t, j] == 0).all())
                    elif sample is None or self.rng.random() < sample:
                        want, tol = self.expect(q[l, t, j], l, t, int(s["leaf_slot"][j]))
                        check(out[l, t, j][None], want, tol, (l, t, j))
        assert self.dec.status() == 0
        return q, out

    def tree(self, slots, sample=None):
        Hq, Hkv, D = self.shape
        slots = np.asarray(slots)
        q = randn(self.gen, (self.L, self.T, slots.shape[1], Hq, D), self.dt)
        out = torch.full_like(q, 5.0)
        self.dec.tree_attn(0, self.L, torch.from_numpy(slots.astype(np.int32)).cuda(), q, out, self.scale)
        for l in range(self.L):
            for t, s in enumerate(self.tries):
                for j, slot in enumerate(slots[t]):
                    if not 0 <= slot < s["n_nodes"] or s["mask"][slot] == 0:
                        assert bool((out[l, t, j] == 0).all()), (l, t, j)
                    elif sample is None or self.rng.random() < sample:
                        want, tol = self.expect(q[l, t, j], l, t, int(slot))
                        check(out[l, t, j][None], want, tol, (l, t, j))


# lengths around the tile of 64 keys, head dims of every kernel, 32, 64 and more rows per KV head
@pytest.mark.parametrize("S", [1, 15, 64, 65, 200, 777])
@pytest.mark.parametrize("dtype,D,Hq,Hkv,b,T,page", [("bf16", 128, 8, 2, 3, 2, 16), ("bf16", 64, 4, 4, 2, 1, 64), ("bf16", 96, 6, 2, 5, 3, 32),
                                                     ("f32", 64, 4, 1, 3, 2, 16), ("f32", 128, 8, 1, 5, 4, 128), ("bf16", 128, 16, 2, 8, 5, 64)])
def test_decode(dtype, D, Hq, Hkv, b, T, page, S):
    log(f"decode {dtype} d={D} {Hq}/{Hkv} b={b} T={T} S={S}")
    Batch(dtype, D, Hq, Hkv, S, page, [(5 + 30 * t, 4) for t in range(T)], b).decode(sample=0.5 if T > 2 else None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 160, 192, 224, 256])
@pytest.mark.parametrize("T,b", [(1, 2), (2, 12), (3, 40)])
def test_decode_other_head_dims(dtype, D, T, b):
    log(f"decode {dtype} d={D} T={T} b={b}")
    Batch(dtype, D, 3, 1, 130, 32, [(7, 2)] * T, b).decode(sample=0.2)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 96)])
@pytest.mark.parametrize("S", [100, 2000])
def test_decode_vector_alu_kernel(dtype, D, S):
    Batch(dtype, D, 4, 2, S, 16, [(9, 3), (70, 2)], 4, attn_impl=B.TD_ATTN_VALU).decode()


def test_splits_forced(monkeypatch):
    monkeypatch.setenv("TD_ATTN_SPLITS", "5")
    Batch("bf16", 128, 8, 2, 500, 64, [(90, 3), (300, 2)], 4).decode()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("window", [1, 6, 40, 64, 100, 300])
def test_decode_window(dtype, D, window):
    """Tries of several depths behind 130 positions: the window ends in the trie, in the prefix, before it."""
    Batch(dtype, D, 8, 2, 130, 16, [(3, 2), (33, 1), (90, 4), (1, 0)], 4, window=window, dead=True).decode()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64), ("bf16", 32)])
def test_decode_window_tries_of_other_depths(dtype, D):
    """Tries of one row block at other depths: the window leaves some of them nothing of the prefix, others a
    part; few tries and more than a block takes the headers of."""
    Batch(dtype, D, 4, 2, 100, 16, [(5, 2), (60, 2), (1, 1), (200, 1)], 3, window=64).decode()
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


def test_zero_length_prefix_is_none():
    bt = Batch("bf16", 128, 8, 2, 64, 64, [(20, 3)], 4)
    q = randn(bt.gen, (1, 1, 4, 8, 128), torch.bfloat16)
    outs = []
    for attach in (lambda: bt.prefix.attach(bt.dec, 0), lambda: bt.dec.set_prefix(None)):
        attach()
        outs.append(torch.empty_like(q))
        bt.dec.attn_decode(0, 1, q, None, None, outs[-1], bt.scale)
    assert torch.equal(*outs)


# drafts (the decode layout) and prompts (the prefill-shaped kernels, short and long key ranges)
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 4, 1), (96, 6, 6)])
@pytest.mark.parametrize("S,window", [(1, 0), (100, 0), (333, 0), (100, 50), (40, 90)])
def test_drafts(D, Hq, Hkv, S, window):
    bt = Batch("bf16", D, Hq, Hkv, S, 32, [(30, 4), (50, 2)], 4, window=window, dead=True)
    slots = np.full((2, 9), -1)
    for t, s in enumerate(bt.tries):
        slots[t, 1:8] = np.arange(s["n_nodes"] - 7, s["n_nodes"])
    slots[1, 0], slots[0, 8] = 12, 2 ** 31 - 1
    bt.tree(slots)


@pytest.mark.parametrize("D,Hq,Hkv,prompts", [(128, 16, 2, (50, 33)), (64, 4, 1, (150, 90)), (96, 12, 2, (64, 65, 7)), (128, 8, 1, (640, 70))])
@pytest.mark.parametrize("S,window", [(1, 0), (130, 0), (500, 0), (130, 60)])
def test_prompts(D, Hq, Hkv, prompts, S, window):
    log(f"prompts d={D} S={S} W={window}")
    bt = Batch("bf16", D, Hq, Hkv, S, 64, [(p, 0) for p in prompts], 2, window=window)
    slots = np.full((len(prompts), max(prompts)), -1)
    for t, p in enumerate(prompts):
        slots[t, :p] = np.arange(p)
    bt.tree(slots, sample=0.15)


def test_prompts_past_the_workspace():
    """73 MB of records for a layer: several launches over queries, then over layers."""
    bt = Batch("bf16", 128, 64, 4, 100, 64, [(1100, 0), (900, 0)], 1, L=2)
    slots = np.stack([np.arange(1100), np.where(np.arange(1100) < 900, np.arange(1100), -1)])
    bt.tree(slots, sample=0.002)
    bt = Batch("bf16", 64, 64, 64, 70, 16, [(500, 0)], 1, L=17)
    bt.tree(np.arange(500)[None], sample=0.0005)


class Chunk:
    def __init__(self, dtype, D, Hq, Hkv, pos, n, page, window=0, L=1, seed=9, spare=0):
        self.gen, self.rng, self.dt = torch.Generator().manual_seed(seed), np.random.default_rng(seed), DT[dtype]
        self.pos, self.n, self.W, self.L, self.shape = pos, n, window, L, (Hq, Hkv, D)
        self.dec = B.TrieDecoder(1, 1, 4, 100, L, Hq, Hkv, D, window, dtype)
        self.prefix = Prefix(self.gen, self.rng, L, Hkv, D, self.dt, pos + n, page, spare)
        self.prefix.attach(self.dec, 0)
        self.scale = 1.0 / D ** 0.5
        self.q = randn(self.gen, (L, n, Hq, D), self.dt)

    def run(self):
        out = torch.full_like(self.q, 5.0)
        self.dec.prefix_attn(0, self.L, self.pos, self.q, out, self.scale)
        return out

    def verify(self, out, rows=None):
        for l in range(self.L):
            k, v = self.prefix.rows(self.prefix.k, l), self.prefix.rows(self.prefix.v, l)
            for j in rows if rows is not None else range(self.n):
                p = self.pos + j
                lo = max(0, p - self.W + 1) if self.W else 0
                want, tol = attend(self.q[l, j:j + 1], k[:, lo:p + 1], v[:, lo:p + 1],
                                   torch.ones(1, p + 1 - lo, dtype=torch.bool), self.scale, self.dt)
                check(out[l, j:j + 1], want, tol, (l, j))


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 128, 4, 1), ("bf16", 64, 2, 2), ("bf16", 96, 7, 1), ("f32", 64, 4, 2), ("f32", 128, 2, 1),
                                            ("bf16", 256, 2, 1), ("f32", 160, 1, 1), ("bf16", 32, 3, 3)])
@pytest.mark.parametrize("pos,n,page,window", [(0, 1, 16, 0), (0, 70, 16, 0), (63, 2, 64, 0), (500, 9, 32, 0), (129, 200, 64, 0), (100, 150, 16, 33),
                                               (700, 3, 128, 64)])
def test_prefix_prefill(dtype, D, Hq, Hkv, pos, n, page, window):
    log(f"chunk {dtype} d={D} pos={pos} n={n} W={window}")
    c = Chunk(dtype, D, Hq, Hkv, pos, n, page, window)
    c.verify(c.run(), c.rng.permutation(n)[:24])


def test_prefix_prefill_layers_and_splits():
    c = Chunk("bf16", 128, 8, 2, 3000, 40, 64, L=3)
    c.verify(c.run(), [0, 17, 39])


@pytest.mark.parametrize("dtype,D,Hq,Hkv,pos,n,window,L", [
    ("bf16", 64, 16, 8, 0, 700, 0, 3),    # 264 blocks, an odd number per XCD, of 3 layers
    ("bf16", 64, 16, 8, 5, 700, 100, 3),
    ("bf16", 128, 32, 8, 90, 1024, 0, 2),  # 512
    ("bf16", 96, 32, 32, 0, 1800, 0, 1),   # 480
    ("f32", 64, 16, 8, 0, 1024, 0, 1)])    # 128 in 4 splits
def test_prefix_prefill_two_blocks_per_cu(dtype, D, Hq, Hkv, pos, n, window, L):
    """Launches whose blocks are ordered to even out the CUs: every block of every layer is taken."""
    c = Chunk(dtype, D, Hq, Hkv, pos, n, 64, window, L)
    out = c.run()
    assert not (out == 5.0).all(-1).any()
    step = 128 * Hkv // Hq
    c.verify(out, range(step // 2, n, step))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("bf16", 256), ("f32", 64), ("f32", 256)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,G", [(90, 4), (20, 1), (13, 4)])
def test_what_a_row_does_not_see(dtype, D, bad, n, G):
    """A chunk whose last keys hold NaN or infinities in K and V: earlier rows do not see them and are
    as exact as ever; rows that see them are not finite.  So are pages past the end and other pages."""
    c = Chunk(dtype, D, G, 1, 40, n, 32, spare=70)
    p = c.prefix
    last = c.pos + n - 1
    first_bad = last - 5
    for pos in (first_bad, last):
        p.k[int(p.pages[pos // 32]), :, :, pos % 32, ::3] = bad
        p.v[int(p.pages[pos // 32]), :, :, pos % 32, 1::2] = bad
    for pos in range(last + 1, len(p.pages) * 32):
        p.k[int(p.pages[pos // 32]), :, :, pos % 32] = bad
        p.v[int(p.pages[pos // 32]), :, :, pos % 32] = bad
    other = np.setdiff1d(np.arange(p.k.shape[0]), p.pages)
    p.k[other] = bad
    p.v[other] = bad
    out = c.run()
    c.verify(out, range(first_bad - c.pos))
    assert not bool(torch.isfinite(out[0, first_bad - c.pos:]).all(-1).any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_hides_bad_rows(dtype):
    bt = Batch(dtype, 64, 4, 2, 150, 16, [(3, 2), (40, 1)], 4, window=60)
    p = bt.prefix
    for pos in list(range(0, 150 + 4 - 60)):  # before the shallower trie's window
        p.v[int(p.pages[pos // 16]), :, :, pos % 16] = float("nan")
    # (the deeper trie's rows see none of positions up to 150 + 40 - 60)
    for pos in range(150 + 4 - 60, 150 + 40 - 60):
        p.v[int(p.pages[pos // 16]), :, :, pos % 16, 0] = float("inf")
    q = randn(bt.gen, (1, 2, 4, 4, 64), bt.dt)
    out = torch.empty_like(q)
    bt.dec.attn_decode(0, 1, q, None, None, out, bt.scale)
    s = bt.tries[1]
    for j in range(4):
        want, tol = bt.expect(q[0, 1, j], 0, 1, int(s["leaf_slot"][j]))
        check(out[0, 1, j][None], want, tol, j)
    assert not bool(torch.isfinite(out[0, 0, :, :, 0]).any()) and bool(torch.isfinite(out[0, 0, :, :, 1:]).all())


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_large_scores(dtype, D):
    """Scores over hundreds of powers of two, rising and falling along the keys."""
    bt = Batch(dtype, D, 4, 1, 400, 32, [(6, 2), (30, 2)], 4)
    ramp = torch.linspace(0.1, 30.0, 400, device="cuda")
    for pos in range(400):
        bt.prefix.k[int(bt.prefix.pages[pos // 32]), :, :, pos % 32] *= float(ramp[2 * min(pos, 399 - pos)])
    bt.decode()


def test_graph_reads_the_attached_prefix():
    """Captured store and attention, replayed behind the same, a longer, a shorter and no prefix, with
    eager work between: each replay is what the eager calls give."""
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
    longer = Prefix(bt.gen, bt.rng, 2, 2, 128, dt, 1111, 64)
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
        tol = 4 * 2.0 ** -8  # (eager calls may split otherwise)
        assert torch.equal(got[0], rot) and torch.equal(got[3], bt.dec.k_pool), name
        for a, c in ((got[1], out), (got[2], chunk)):
            assert float((a.float() - c.float()).abs().max()) <= tol * float(c.float().abs().max()), name
    assert bt.dec.status() == 0


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


# where the tries' own nodes go: in the prefix's launch (short tries and prefixes), in a launch whose
# epilogue merges the records (many units), in split launches and a merge; leaves stored by the call
@pytest.mark.parametrize("D,Hq,Hkv,b,tries,S,L", [(128, 8, 2, 4, [(300, 6), (20, 2)], 1500, 1), (64, 16, 4, 16, [(200, 8)] * 12, 130, 4),
                                                  (96, 8, 8, 3, [(1500, 4), (90, 2)], 40, 1), (128, 32, 8, 40, [(30, 3), (64, 1)], 700, 2)])
@pytest.mark.parametrize("pending", [False, True])
def test_where_the_nodes_go(D, Hq, Hkv, b, tries, S, L, pending):
    bt = Batch("bf16", D, Hq, Hkv, S, 64, tries, b, L=L, dead=True)
    if pending:  # the leaves' rows come with the call: the same rows, loaded as pending
        k = torch.zeros((L, bt.T, b, Hkv, D), dtype=bt.dt, device="cuda")
        v = torch.zeros_like(k)
        for t, s in enumerate(bt.tries):
            for j, n in enumerate(s["leaf_slot"]):
                k[:, t, j], v[:, t, j] = bt.dec.k_pool[t, :, :, int(n)], bt.dec.v_pool[t, :, :, int(n)]
        keep = bt.dec.k_pool.clone(), bt.dec.v_pool.clone()
        for t, s in enumerate(bt.tries):
            s["kv_pending"] = 1
        bt.dec.close()
        bt.dec = B.TrieDecoder(bt.T, b, keep[0].shape[3], 100, L, Hq, Hkv, D)
        for t, s in enumerate(bt.tries):
            bt.dec.load_state(t, s)
        bt.dec.k_pool.copy_(keep[0])
        bt.dec.v_pool.copy_(keep[1])
        for t, s in enumerate(bt.tries):
            for n in s["leaf_slot"]:
                bt.dec.k_pool[t, :, :, int(n)] = bt.dec.v_pool[t, :, :, int(n)] = 7.0
        bt.prefix.attach(bt.dec)
        q = randn(bt.gen, (L, bt.T, b, Hq, D), bt.dt)
        out = torch.empty_like(q)
        bt.dec.attn_decode(0, L, q, k, v, out, bt.scale)
        assert torch.equal(bt.dec.k_pool, keep[0]) and torch.equal(bt.dec.v_pool, keep[1])
        again = torch.empty_like(q)
        bt.dec.attn_decode(0, L, q, None, None, again, bt.scale)
        assert float((again.float() - out.float()).abs().max()) <= 4 * 2.0 ** -8 * float(out.float().abs().max())
    bt.decode(sample=0.05 if len(tries) > 2 else 0.3)


def test_kernel_events():
    """The attention's events bracket every launch of a call, beside a prefix too."""
    bt = Batch("bf16", 128, 8, 2, 900, 64, [(150, 3), (90, 2)], 4, L=2)
    q, out = randn(bt.gen, (2, 2, 4, 8, 128), bt.dt), torch.empty((2, 2, 4, 8, 128), dtype=bt.dt, device="cuda")
    qs = torch.arange(90, dtype=torch.int32, device="cuda").repeat(2, 1)
    tq = randn(bt.gen, (2, 2, 90, 8, 128), bt.dt)
    cq = randn(bt.gen, (2, 50, 8, 128), bt.dt)
    for call in (lambda: bt.dec.attn_decode(0, 2, q, None, None, out, bt.scale),
                 lambda: bt.dec.tree_attn(0, 2, qs, tq, torch.empty_like(tq), bt.scale),
                 lambda: bt.dec.tree_attn(0, 2, qs[:, -7:].contiguous(), tq[:, :, :7].contiguous(), torch.empty_like(tq[:, :, :7].contiguous()), bt.scale),
                 lambda: bt.dec.prefix_attn(0, 2, 800, cq, torch.empty_like(cq), bt.scale)):
        call()
        ev = B.KernelEvents()
        B.td_set_kernel_events(bt.dec.ctx, B.TD_PHASE_ATTN, ev.start, ev.stop)
        call()
        assert 0.0 < ev.elapsed_ms() < 50.0
        ev.close()


def test_refusals():
    dec = B.TrieDecoder(2, 2, 40, 50, 2, 4, 2, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    dt = torch.bfloat16
    kp = torch.zeros((4, 2, 2, 16, 64), dtype=dt, device="cuda")
    q, k = torch.zeros((2, 5, 4, 64), dtype=dt, device="cuda"), torch.zeros((2, 5, 2, 64), dtype=dt, device="cuda")

    def refused(status, fn, *a, **kw):
        with pytest.raises(B.TdError) as e:
            fn(*a, **kw)
        assert e.value.status == status, e.value

    refused(B.TD_ESTATE, dec.prefix_store, 0, 2, 0, k, k)
    refused(B.TD_ESTATE, dec.prefix_attn, 0, 2, 0, q, q.clone(), 0.1)
    nodes = torch.zeros((2, 2, 2, 2, 64), dtype=dt, device="cuda")
    refused(B.TD_ESTATE, dec.store_kv, 0, 2, nodes, nodes)  # no prompts yet
    for pages, length in (((4,), 1), ((-1,), 1), ((0, 0), 1), ((), 0), ((0, 1), 33), ((0, 1), -1), ((0, 1, 2, 3, 1), 3)):
        refused(B.TD_EINVAL, dec.set_prefix, kp, kp, pages, length)
    refused(B.TD_EINVAL, dec.set_prefix, torch.zeros((1, 2, 2, 24, 64), dtype=dt, device="cuda"),
            torch.zeros((1, 2, 2, 24, 64), dtype=dt, device="cuda"), (0,), 1)
    refused(B.TD_EINVAL, dec.set_prefix, torch.zeros((1, 2, 2, 8, 64), dtype=dt, device="cuda"),
            torch.zeros((1, 2, 2, 8, 64), dtype=dt, device="cuda"), (0,), 1)
    for wrong in (kp.float(), kp[:, :1].contiguous(), kp.transpose(0, 1)):
        with pytest.raises(ValueError):
            dec.set_prefix(wrong, wrong, (0,), 1)
    refused(B.TD_ESTATE, dec.prefix_store, 0, 2, 0, k, k)  # (no refused prefix was attached)
    dec.set_prefix(kp, kp.clone(), (2, 0), 10)
    for layer, n, pos in ((0, 3, 0), (-1, 2, 0), (1, 2, 0), (0, 2, -1), (0, 2, 28), (0, 2, 2 ** 31 - 1)):
        refused(B.TD_EINVAL, B.trie_prefix_store, dec.ctx, dec.dims, layer, n, pos, k[:1].expand(n, -1, -1, -1).contiguous(),
                k[:1].expand(n, -1, -1, -1).contiguous())
        refused(B.TD_EINVAL, dec.prefix_attn, layer, n, pos, q[:1].expand(n, -1, -1, -1).contiguous(),
                torch.empty((n, 5, 4, 64), dtype=dt, device="cuda"), 0.1)
    freq = torch.ones(32, device="cuda")
    for n in (0, 4, 12, 40):
        refused(B.TD_EINVAL, dec.prefix_store, 0, 2, 0, k, k, rope=B.Rope(torch.ones(n, device="cuda")))
    refused(B.TD_EINVAL, dec.prefix_store, 0, 2, 0, k, None)
    refused(B.TD_EINVAL, dec.prefix_store, 0, 2, 0, k, k, q)
    refused(B.TD_EINVAL, dec.prefix_store, 0, 2, 0, k, k, None, q)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        refused(B.TD_EINVAL, dec.prefix_attn, 0, 2, 0, q, q.clone(), scale)
    for bad in (k.float(), k[:, :4], k.transpose(2, 3).contiguous(), k.transpose(1, 2).contiguous().transpose(1, 2), k.cpu()):
        with pytest.raises(ValueError):
            dec.prefix_store(0, 2, 0, bad, k, rope=B.Rope(freq))
    with pytest.raises(ValueError):
        dec.prefix_store(0, 2, 0, k, k, q, q[:, :4])
    refused(B.TD_EINVAL, dec.prefix_store, 0, 2, 0, torch.zeros((2, 5, 132), dtype=dt, device="cuda")[..., :128].unflatten(-1, (2, 64)), k)
    flat = torch.zeros(2 * 5 * 128 + 8, dtype=dt, device="cuda")
    refused(B.TD_EINVAL, dec.prefix_store, 0, 2, 0, flat[4:4 + 1280].view(2, 5, 2, 64), k)
    dec.init_prompt([5, 7], torch.zeros((2, 7), **i32))
    with pytest.raises(ValueError):
        dec.store_kv(0, 2, nodes, nodes, qslots=torch.zeros((1, 2), **i32))
    with pytest.raises(ValueError):
        dec.store_kv(0, 2, nodes, nodes, qslots=torch.zeros((2, 2), dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        dec.store_kv(0, 2, nodes[:, :, :1], nodes[:, :, :1])
    assert dec.status() == 0
    dec.close()
