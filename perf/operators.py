"""Performance cases of the shared prefix: the rows that a model's forward pass stores, rotated to
their positions, and the attention of a batch of tries over one prefix that all of them share.

Kinds of case (``case["kind"]``):

* ``leaves``: the K/V rows of every live leaf into the tries' pools, keys and queries rotated
  to the leaves' positions (a decode step).
* ``prompts``: the same for the stored nodes of ragged prompts (a prefill).
* ``prefix``: n tokens into the paged cache of the prefix, from position ``pos`` on.
* ``decode``: the attention of a decode step, every live leaf over the prefix and its own path.
* ``queries``: the attention of stored nodes over the prefix and their own paths: the prompts'
  prefill, or draft nodes.
* ``chunk``: the causal attention of n tokens of the prefix over the prefix up to themselves.

A model calls these layer by layer (``calls = "layer"``); "all" is one call over every layer.
K, V and Q are N(0, 1), as in this repository's workloads.  ``own`` says whether ``run`` makes the
library's calls or computes the same in plain torch operations.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------
def _case(kind, layers, q_heads, kv_heads, head_dim, dtype="bf16", **kw):
    c = dict(kind=kind, layers=layers, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, tries=1,
             beams=1, prompt=1, prompt_min=1, steps=0, window=0, page=64, length=0, pos=0, n=0, queries=0,
             rotary=head_dim, interleaved=False, base=10000.0, calls="layer")
    c.update(kw)
    if "prompt_min" not in kw:
        c["prompt_min"] = c["prompt"]
    return c


def listed():
    return [
        # the smallest step: one fp32 layer, three beams of one request
        _case("leaves", 1, 4, 4, 64, "f32", name="leaves_tiny", beams=3, prompt=32, steps=4, length=16, page=16),
        # a serving batch's step, one call per layer
        _case("leaves", 4, 32, 8, 128, name="leaves_batch16", tries=16, beams=16, prompt=256, prompt_min=100, steps=4,
              length=8192, base=500000.0),
        # the prompts of a serving batch, ragged
        _case("prompts", 2, 32, 8, 128, name="prompts_ragged", tries=8, prompt=1024, prompt_min=301, length=4096,
              base=500000.0),
        # a long shared prefix stored in one call per layer
        _case("prefix", 2, 32, 8, 128, name="prefix_8k", n=8192, base=500000.0),
        # a later chunk far into a long prefix, small pages, part of the head rotated, by neighbours
        _case("prefix", 1, 16, 2, 64, "f32", name="prefix_far", pos=100003, n=777, page=16, rotary=32, interleaved=True),
        # the smallest attention: fp32, a short prefix
        _case("decode", 1, 4, 4, 64, "f32", name="decode_tiny", tries=2, beams=3, prompt=32, steps=4, length=64, page=16),
        # a small batch at the Llama-3.1-8B shape, a layer at a time
        _case("decode", 4, 32, 8, 128, name="decode_batch4", tries=4, beams=8, prompt=256, prompt_min=90, steps=16,
              length=4096),
        # a serving batch: 16 requests of 16 beams over a long system prompt
        _case("decode", 4, 32, 8, 128, name="decode_batch16", tries=16, beams=16, prompt=512, prompt_min=128, steps=32,
              length=8192, calls="all"),
        # few beams over a very long document, multi-head attention at head_dim 96
        _case("decode", 1, 32, 32, 96, name="decode_document", tries=2, beams=4, prompt=64, steps=8, length=50001, page=128),
        # a sliding window that ends inside the prefix
        _case("decode", 4, 32, 8, 128, name="decode_window", tries=4, beams=8, prompt=700, prompt_min=300, steps=20,
              length=6000, window=4096, page=32),
        # the prompts' prefill behind a shared prefix
        _case("queries", 2, 32, 8, 128, name="prompts_prefill", tries=4, prompt=512, prompt_min=380, length=4096, queries=512),
        # a chunk of the prefix's own prefill
        _case("chunk", 2, 32, 8, 128, name="prefix_prefill", pos=6144, n=2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["leaves", "prompts", "prefix", "decode", "decode", "decode", "queries", "queries", "chunk"])
    kv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 4, 7, 8) if g * kv <= 64])
    dtype = "f32" if kind != "queries" and rng.random() < 0.25 else "bf16"
    dim = rng.choice([64, 96, 128, 128] if kind == "queries" or rng.random() < 0.8 else [32, 160, 192, 256])
    esz = 4 if dtype == "f32" else 2
    c = _case(kind, _log_int(rng, 1, 4), heads, kv, dim, dtype, page=rng.choice([16, 32, 64, 64, 128, 256]),
              interleaved=rng.random() < 0.3, base=rng.choice([10000.0, 500000.0]), calls=rng.choice(["layer", "all"]))
    c["rotary"] = rng.choice([dim, dim, 16 * max(1, dim // 32)])
    row = 2 * c["layers"] * kv * dim * esz  # K + V of a position, all layers
    if kind in ("prefix", "chunk"):
        c["n"] = _log_int(rng, 1, 6000)
        c["pos"] = 0 if rng.random() < 0.3 else _log_int(rng, 1, 30000 if kind == "prefix" else 12000)
        most = int(2.5e8 / row)  # positions
        c["n"] = max(1, min(c["n"], most // 2))
        c["pos"] = max(0, min(c["pos"], most - c["n"]))
        if kind == "chunk":
            flops = 4.0 * dim * heads * c["layers"] * (c["pos"] + c["n"] / 2)
            c["n"] = max(1, min(c["n"], int((4e10 if dtype == "f32" else 2.2e11) / flops)))
            c["window"] = rng.choice([0, 0, 0, _log_int(rng, 8, 4000)])
        return c
    c["tries"] = _log_int(rng, 1, 16)
    c["length"] = _log_int(rng, 1, 20000)
    c["window"] = rng.choice([0, 0, 0, _log_int(rng, 8, 8000)]) if kind in ("decode", "queries") else 0
    c["beams"] = _log_int(rng, 1, 24)
    c["steps"] = rng.randrange(1, 40)
    c["prompt"] = _log_int(rng, 1, 1200 if kind == "prompts" else 800)
    if kind in ("prompts", "queries") and rng.random() < 0.6:
        c["beams"], c["steps"] = 1, 0
        c["queries"] = c["prompt"]
    elif kind == "queries":
        c["queries"] = _log_int(rng, 1, 40)
    c["prompt"] = max(1, min(c["prompt"], int(1.5e8 / (row * c["tries"])) - c["steps"] * c["beams"]))
    c["prompt_min"] = max(1, int(c["prompt"] * rng.choice([1.0, 0.3])))
    c["length"] = max(1, min(c["length"], int(2.0e8 / row)))
    if kind in ("decode", "queries"):
        owners = c["tries"] * (c["queries"] or c["beams"])
        flops = 4.0 * dim * heads * c["layers"] * owners
        c["length"] = max(1, min(c["length"], int((2e10 if dtype == "f32" or dim not in (64, 96, 128) else 1.3e11) / flops)))
    return c


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _normal(gen, shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=gen)


def _trie(rng, prompt, steps, b):
    """The trie of one request after ``steps`` decode steps of b beams (the parent of rank r drawn
    with weight 1/(r+1)), nodes on no live path collected, in the layout of td_state."""
    weight = 1.0 / (np.arange(b) + 1.0)
    parent, depth = list(range(-1, prompt - 1)), list(range(prompt))
    leaves = [prompt - 1]
    for s in range(steps):
        w = weight[:len(leaves)]
        chosen = [leaves[r] for r in rng.choice(len(leaves), size=b, p=w / w.sum())]
        leaves = list(range(len(parent), len(parent) + b))
        parent += chosen
        depth += [prompt + s] * b
    bits = [(1 << len(leaves)) - 1] * prompt + [0] * (len(parent) - prompt)
    for i, leaf in enumerate(leaves):
        while leaf >= prompt:
            bits[leaf] |= 1 << i
            leaf = parent[leaf]
    mask = np.array(bits, np.uint64)
    old = np.nonzero(mask)[0]
    slot = np.full(len(parent) + 1, -1, np.int32)  # (the last entry: the parent of the root)
    slot[old] = np.arange(len(old))
    n, nl = len(old), len(leaves)
    return dict(n_nodes=n, n_live=nl, next_id=len(parent), kv_pending=0, step=steps, node_id=old.astype(np.int32),
                parent_slot=slot[np.array(parent)[old]], token=rng.integers(0, 1000, n).astype(np.int32),
                depth=np.array(depth, np.int32)[old], mask=mask[old], leaf_slot=np.arange(n - nl, n, dtype=np.int32),
                leaf_score=-np.sort(rng.random(nl) * 8.0 + 20.0).astype(np.float32))


def _inputs(c, seed):
    """Every input of the case, from the seed alone."""
    gen, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    L, T, Hq, Hkv, D, ps = c["layers"], c["tries"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    kind = c["kind"]
    x = dict(pages=np.zeros(0, np.int32))
    # the prefix's pages lie anywhere in a pool that holds others' pages too
    stored = c["pos"] + c["n"] if kind in ("prefix", "chunk") else c["length"] if kind in ("decode", "queries") else 0
    if stored:
        used = (stored + ps - 1) // ps
        n_pages = used + 1 + used // 8
        x["pages"] = rng.permutation(n_pages)[:used].astype(np.int32)
        x["k_pages"] = _normal(gen, (n_pages, L, Hkv, ps, D), dt)
        x["v_pages"] = _normal(gen, (n_pages, L, Hkv, ps, D), dt)
    if kind in ("prefix", "chunk"):
        lead = (L, c["n"])
    else:
        lengths = [int(n) for n in np.linspace(c["prompt"], c["prompt_min"], T)]
        x["tries"] = [_trie(rng, n, c["steps"], c["beams"]) for n in lengths]
        x["slots"] = c["prompt"] + (c["steps"] + 1) * c["beams"]
        rows = c["beams"]
        if kind in ("prompts", "queries"):  # the newest nodes, or all of them
            rows = min(c["queries"] or x["slots"], c["prompt"] + c["steps"])
            qs = np.full((T, rows), -1, np.int32)
            for t, s in enumerate(x["tries"]):
                n = min(rows, s["n_nodes"])
                qs[t, :n] = np.arange(s["n_nodes"] - n, s["n_nodes"])
            x["qslots"] = torch.from_numpy(qs).cuda()
        x["k_pool"] = _normal(gen, (T, L, Hkv, x["slots"], D), dt)
        x["v_pool"] = _normal(gen, (T, L, Hkv, x["slots"], D), dt)
        lead = (L, T, rows)
    x["q"] = _normal(gen, lead + (Hq, D), dt)
    if kind in ("leaves", "prompts", "prefix"):
        x["k"], x["v"] = _normal(gen, lead + (Hkv, D), dt), _normal(gen, lead + (Hkv, D), dt)
        r = c["rotary"]
        x["freq"] = (c["base"] ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().cuda()
    return x


def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    st = dict(case=c, x=x, scale=1.0 / math.sqrt(c["head_dim"]), out=torch.zeros_like(x["q"]))
    L, Hq, Hkv, D = c["layers"], c["q_heads"], c["kv_heads"], c["head_dim"]
    if not own:
        if "tries" in x:
            st["tables"] = _tables(c, x)
        if len(x["pages"]):
            st["table"] = torch.from_numpy(x["pages"]).cuda().long()
        return st
    import paper_2502_00085_amd.binding as B
    T, b = c["tries"], c["beams"]
    dec = B.TrieDecoder(T, b, x.get("slots", b + 1), 1000, L, Hq, Hkv, D, c["window"], c["dtype"])
    if "tries" in x:
        dec.k_pool.copy_(x.pop("k_pool"))
        dec.v_pool.copy_(x.pop("v_pool"))
        for t, s in enumerate(x["tries"]):
            dec.load_state(t, s)
    if len(x["pages"]):
        dec.set_prefix(x["k_pages"], x["v_pages"], x["pages"], c["length"] or c["pos"] + c["n"])
    elif c["length"]:  # (the stores of nodes need the prefix's length, not its rows)
        n = (c["length"] + 15) // 16
        x["k_pages"] = torch.zeros((n, L, Hkv, 16, D), dtype=x["q"].dtype, device="cuda")
        dec.set_prefix(x["k_pages"], x["k_pages"], range(n), c["length"])
    if "freq" in x:
        st["rope"] = B.Rope(x["freq"], c["interleaved"])
    st["dec"] = dec
    return st


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    c, x, dec, out = st["case"], st["x"], st["dec"], st["out"]
    kind, L = c["kind"], c["layers"]
    for l, n in [(0, L)] if c["calls"] == "all" else [(l, 1) for l in range(L)]:
        s = slice(l, l + n)
        if kind in ("leaves", "prompts"):
            dec.store_kv(l, n, x["k"][s], x["v"][s], x["q"][s], out[s], st["rope"], x.get("qslots"))
        elif kind == "prefix":
            dec.prefix_store(l, n, c["pos"], x["k"][s], x["v"][s], x["q"][s], out[s], st["rope"])
        elif kind == "decode":
            dec.attn_decode(l, n, x["q"][s], None, None, out[s], st["scale"])
        elif kind == "queries":
            dec.tree_attn(l, n, x["qslots"], x["q"][s], out[s], st["scale"])
        else:
            dec.prefix_attn(l, n, c["pos"], x["q"][s], out[s], st["scale"])
    if kind == "prefix":
        return dict(q=out, k_pages=x["k_pages"], v_pages=x["v_pages"])
    if kind in ("leaves", "prompts"):
        return dict(q=out, k_pool=dec.k_pool, v_pool=dec.v_pool)
    return out


def _tables(c, x):
    """Per trie, on the device: the slot and depth of each query, and which nodes it sees."""
    tables = []
    for t, s in enumerate(x["tries"]):
        slots = x["qslots"][t] if "qslots" in x else torch.from_numpy(s["leaf_slot"]).cuda()
        at = torch.nonzero(slots >= 0).view(-1)
        slots = slots[at].long()
        depth = torch.from_numpy(s["depth"]).cuda()
        mask = torch.from_numpy(s["mask"].view(np.int64)).cuda()
        seen = ((mask[None] & mask[slots][:, None]) == mask[slots][:, None]) & (depth[None] <= depth[slots][:, None])
        if c["window"]:
            seen &= depth[slots][:, None] - depth[None] < c["window"]
        tables.append((at, slots, depth[slots], seen))
    return tables


def _rotate(x, pos, freq, interleaved):
    """x [..., n, H, d] at positions pos [n], in 32 bits (the angles in 64)."""
    a = pos.double()[:, None] * freq.double()
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
    r = 2 * freq.numel()
    y = x.float().clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    u, w = y[..., first].clone(), y[..., second].clone()
    y[..., first], y[..., second] = u * cos - w * sin, w * cos + u * sin
    return y.to(x.dtype)


def _attend(q, parts, scale):
    """q [n][Hq][d]; parts: (k, v [Hkv][m][d], seen [n][m]): softmax attention over all of them, in 32
    bits; zeros for a query that sees nothing."""
    n, Hq, D = q.shape
    Hkv = parts[0][0].shape[0]
    G = Hq // Hkv
    qf = q.float().view(n, Hkv, G, D).transpose(0, 1).reshape(Hkv, n * G, D)
    k, v = (torch.cat([p[i].float() for p in parts], 1) for i in (0, 1))
    seen = torch.cat([p[2] for p in parts], 1)
    s = torch.bmm(qf, k.transpose(1, 2).contiguous()).mul_(scale).view(Hkv, n, G, -1)
    s.masked_fill_(~seen[None, :, None, :], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp_min(-3e38))
    o = torch.bmm(p.view(Hkv, n * G, -1), v).view(Hkv, n, G, D)
    o = o / p.sum(-1, keepdim=True)
    o = torch.where(seen.any(1)[None, :, None, None], o, torch.zeros_like(o))
    return o.transpose(0, 1).reshape(n, Hq, D).to(q.dtype)


def _run_plain(st):
    c, x, out = st["case"], st["x"], st["out"]
    kind, S, W = c["kind"], c["length"], c["window"]
    if kind == "prefix":
        pos = torch.arange(c["pos"], c["pos"] + c["n"], device="cuda")
        out.copy_(_rotate(x["q"], pos, x["freq"], c["interleaved"]))
        page, off = st["table"][pos // c["page"]], pos % c["page"]
        x["k_pages"][page, :, :, off] = _rotate(x["k"], pos, x["freq"], c["interleaved"]).transpose(0, 1)
        x["v_pages"][page, :, :, off] = x["v"].transpose(0, 1)
        return dict(q=out, k_pages=x["k_pages"], v_pages=x["v_pages"])
    if kind in ("leaves", "prompts"):
        out.zero_()
        for t, (at, slots, depth, _) in enumerate(st["tables"]):
            pos = S + depth
            out[:, t, at] = _rotate(x["q"][:, t, at], pos, x["freq"], c["interleaved"])
            x["k_pool"][t, :, :, slots] = _rotate(x["k"][:, t, at], pos, x["freq"], c["interleaved"]).transpose(1, 2)
            x["v_pool"][t, :, :, slots] = x["v"][:, t, at].transpose(1, 2)
        return dict(q=out, k_pool=x["k_pool"], v_pool=x["v_pool"])
    out.zero_()
    for l in range(c["layers"]):
        # the prefix's rows of the layer in order of position: [Hkv][positions][d]
        k, v = (x[m][st["table"], l].transpose(0, 1).flatten(1, 2) for m in ("k_pages", "v_pages"))
        at_pos = torch.arange(k.shape[1], device="cuda")
        if kind == "chunk":
            for j in range(0, c["n"], 256):
                pos = c["pos"] + torch.arange(j, min(j + 256, c["n"]), device="cuda")[:, None]
                seen = (at_pos <= pos) & ((pos - at_pos < W) if W else True)
                out[l, j:j + 256] = _attend(x["q"][l, j:j + 256], [(k, v, seen)], st["scale"])
            continue
        for t, (at, slots, depth, seen) in enumerate(st["tables"]):
            n = seen.shape[1]
            for j in range(0, len(at), 256):
                part = slice(j, j + 256)
                before = at_pos < S
                if W:
                    before = before & (S + depth[part][:, None] - at_pos < W)
                before = before.expand(len(at[part]), -1)
                out[l, t, at[part]] = _attend(x["q"][l, t, at[part]],
                                              [(k, v, before), (x["k_pool"][t, l, :, :n], x["v_pool"][t, l, :, :n], seen[part])],
                                              st["scale"])
    return out


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    c = case
    L, Hq, Hkv, D, W, S = (c[k] for k in ("layers", "q_heads", "kv_heads", "head_dim", "window", "length"))
    esz = 4 if c["dtype"] == "f32" else 2
    row, qrow, kind = 2.0 * L * Hkv * D * esz, 1.0 * L * Hq * D * esz, c["kind"]
    lengths = [int(n) for n in np.linspace(c["prompt"], c["prompt_min"], c["tries"])]
    if kind in ("leaves", "prompts", "prefix"):
        rows = c["n"] if kind == "prefix" else c["tries"] * c["beams"] if kind == "leaves" else sum(
            n + c["steps"] for n in lengths) if not c["queries"] else sum(min(c["queries"], n + c["steps"]) for n in lengths)
        return {"bytes": 2.0 * rows * (row + qrow), "flops": 3.0 * rows * L * (Hq + Hkv) * c["rotary"]}
    seen = lambda n: min(n, W) if W else n  # noqa: E731
    if kind == "chunk":
        keys = [seen(c["pos"] + j + 1) for j in range(c["n"])]
        return {"bytes": row * min(c["pos"] + c["n"], keys[0] + c["n"] - 1) + 2 * qrow * c["n"], "flops": 4.0 * D * Hq * L * sum(keys)}
    by, fl, most = 0.0, 0.0, 0
    for P in lengths:
        n = P + c["steps"]  # nodes on a leaf's path
        rows = c["beams"] if kind == "decode" else min(c["queries"], n)
        depths = [n - 1] * rows if kind == "decode" else range(n - rows, n)
        by += row * (min(n, seen(n) + rows - 1) + (rows - 1 if kind == "decode" and c["steps"] else 0)) + 2 * qrow * rows
        fl += 4.0 * D * Hq * L * sum(seen(S + d + 1) for d in depths)
        most = max(most, min(S, max(0, W - 1 - min(depths))) if W else S)
    return {"bytes": by + row * most, "flops": fl}


# ---------------------------------------------------------------------------------------------
# the same in 64 bits, row by row from the definition
# ---------------------------------------------------------------------------------------------
def _turn64(x, pos, freq, interleaved):
    """The rotation as a product of complex numbers."""
    half = freq.numel()
    y = x.double()
    turned = y[..., :2 * half]
    z = turned.unflatten(-1, (half, 2)) if interleaved else turned.unflatten(-1, (2, half)).transpose(-1, -2)
    angle = pos.double()[:, None, None] * freq.double()
    z = torch.view_as_complex(z.contiguous()) * torch.polar(torch.ones_like(angle), angle)
    z = torch.view_as_real(z)
    z = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, y[..., 2 * half:]], -1)


def _soft64(q, k, v, seen, scale):
    """One KV head: q [n][G][d], k / v [m][d], seen [n][m]."""
    s = torch.matmul(q.double(), k.double().t().contiguous()) * scale
    s = s.masked_fill(~seen[:, None], -math.inf)
    return torch.matmul(torch.nan_to_num(torch.softmax(s, -1)), v.double())


def exact(case, seed):
    c = case
    if work(c)["flops"] > 3e12:
        return None
    x = _inputs(c, seed)
    kind, S, W, ps, G = c["kind"], c["length"], c["window"], c["page"], c["q_heads"] // c["kv_heads"]
    pages = torch.from_numpy(x["pages"]).cuda().long()
    if kind == "prefix":
        pos = torch.arange(c["pos"], c["pos"] + c["n"], device="cuda")
        res = dict(q=_turn64(x["q"], pos, x["freq"], c["interleaved"]), k_pages=x["k_pages"].double(),
                   v_pages=x["v_pages"].double())
        k = _turn64(x["k"], pos, x["freq"], c["interleaved"])
        for i in range(c["pos"] // ps, (c["pos"] + c["n"] - 1) // ps + 1):  # page by page
            a, e = max(i * ps, c["pos"]), min((i + 1) * ps, c["pos"] + c["n"])
            for name, rows in (("k_pages", k), ("v_pages", x["v"].double())):
                res[name][pages[i], :, :, a - i * ps:e - i * ps] = rows[:, a - c["pos"]:e - c["pos"]].transpose(1, 2)
        return res
    q = x["q"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    if kind in ("leaves", "prompts"):
        res = dict(q=out, k_pool=x["k_pool"].double(), v_pool=x["v_pool"].double())
        for t, s in enumerate(x["tries"]):
            slots = x["qslots"][t].tolist() if "qslots" in x else s["leaf_slot"].tolist()
            rows = [j for j, n in enumerate(slots) if n >= 0]
            slots = [slots[j] for j in rows]
            pos = torch.tensor([S + int(s["depth"][n]) for n in slots], device="cuda")
            out[:, t, rows] = _turn64(q[:, t, rows], pos, x["freq"], c["interleaved"])
            k = _turn64(x["k"][:, t, rows], pos, x["freq"], c["interleaved"])
            res["k_pool"][t, :, :, slots] = k.transpose(1, 2)
            res["v_pool"][t, :, :, slots] = x["v"][:, t, rows].double().transpose(1, 2)
        return res
    stored = S or c["pos"] + c["n"]
    where = torch.arange(stored, device="cuda")
    if kind == "chunk":
        for l in range(c["layers"]):
            for g in range(c["kv_heads"]):
                k, v = (x[m][pages[where // ps], l, g, where % ps] for m in ("k_pages", "v_pages"))
                for j in range(0, c["n"], 512):
                    pos = torch.arange(c["pos"] + j, c["pos"] + min(j + 512, c["n"]), device="cuda")[:, None]
                    seen = (where <= pos) & (where > pos - W if W else where >= 0)
                    out[l, j:j + 512, g * G:(g + 1) * G] = _soft64(q[l, j:j + 512, g * G:(g + 1) * G], k, v, seen, 1.0 / math.sqrt(c["head_dim"]))
        return out
    for t, s in enumerate(x["tries"]):
        n = s["n_nodes"]
        up = np.zeros((n, n), bool)  # up[i]: node i's ancestors and itself
        for i in range(n):
            if s["parent_slot"][i] >= 0:
                up[i] = up[s["parent_slot"][i]]
            up[i, i] = True
        slots = x["qslots"][t].cpu().numpy() if "qslots" in x else s["leaf_slot"]
        rows = np.nonzero(slots >= 0)[0]
        pos = torch.from_numpy(s["depth"][slots[rows]]).cuda()[:, None] + S
        node_pos = torch.from_numpy(s["depth"]).cuda() + S
        seen = torch.cat([(where >= 0).expand(len(rows), -1), torch.from_numpy(up[slots[rows]]).cuda()], 1)
        if W:
            seen = seen & (pos - torch.cat([where, node_pos]) < W)
        for l in range(c["layers"]):
            for g in range(c["kv_heads"]):
                k, v = (torch.cat([x[m][pages[where // ps], l, g, where % ps], x[p][t, l, g, :n]])
                        for m, p in (("k_pages", "k_pool"), ("v_pages", "v_pool")))
                for j in range(0, len(rows), 512):
                    r = rows[j:j + 512]
                    out[l, t, r, g * G:(g + 1) * G] = _soft64(q[l, t, r, g * G:(g + 1) * G], k, v, seen[j:j + 512],
                                                              1.0 / math.sqrt(c["head_dim"]))
    return out
