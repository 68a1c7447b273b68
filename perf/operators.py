"""The operators that verify a tree of drafted tokens against a paged cache, at the sizes a server has.

- ``rope``     rotary positions applied to the query and key heads inside a fused projection's rows
               (half and interleaved pairs, part of the head, scaled frequencies), forward and backward.
- ``append``   the same on a step's queries and keys, with the new keys and values written to the pages.
- ``fork``     beams: the copies of earlier beams are dropped, every sequence is forked again, and each one
               gets room for new tokens; shared partial pages are copied then.
- ``commit``   a step taken back, its room reserved again, and the accepted path of its tree moved together.
- ``copy``     a list of pages copied over all layers (moves between arenas, explicit copies).
- ``attend``   attention of every node of a tree (or of a chain: prompts and single tokens) over the pages.
- ``tree``     ancestor masks and depths of the drafted trees, then the walk along the target's choices.

Pools are [layers][pages][kv heads][page size][head dim]; a sequence's page table is in arbitrary order, as
it is once pages have been freed and taken again. Head counts, head sizes and context lengths are those of
this repository's drafters and workloads, or generic ones.
"""
import math

import numpy as np
import torch

own = False

LENS_8B = "2668,2687,3853,1355"      # the benchmark's ragged batch


def listed():
    return [
        # the four prompts of the benchmark's batch: q and k heads of a fused QKV projection
        dict(name="rope_prompt", kind="rope", rows=10563, hq=32, hkv=8, hd=128, rot=128, layout="half", dtype="bf16",
             scaling="none", factor=1.0, theta=1e6, start=0, backward=False),
        # fp32, interleaved pairs in half of each head, scaled far beyond the trained length, the gradient's pass
        dict(name="rope_part_f32", kind="rope", rows=601, hq=4, hkv=2, hd=64, rot=32, layout="interleaved", dtype="f32",
             scaling="yarn", factor=16.0, theta=1e6, start=100000, backward=True),
        # one layer's new tokens of a step: trees of 16 nodes in four sequences
        dict(name="append_8b_b4", kind="append", lens=LENS_8B, counts="16,16,16,16", hq=32, hkv=8, hd=128, page=64,
             layers=2, rot=128, layout="half", dtype="bf16", theta=1e6),
        # eight prompts searched with four beams each, tokens of all 36 layers in a page
        dict(name="fork_beams", kind="fork", lens="161,530,77,300,95,640,211,333", ways=3, grow=5, layers=36, hkv=8, hd=128,
             page=64, dtype="bf16"),
        # after verification: accepted paths of 64-node trees in 16 sequences, all 36 layers
        dict(name="commit_b16", kind="commit", lens=",".join(str(90 + 37 * b) for b in range(16)), nodes=64, layers=36,
             hkv=8, hd=128, page=16, dtype="bf16"),
        # one token of one user (latency)
        dict(name="attend_token_b1", kind="attend", lens="2048", counts="1", nodes=1, chain=True, hq=32, hkv=8, hd=128, page=16,
             dtype="bf16"),
        # the benchmark's batch, trees of up to 16 nodes
        dict(name="attend_tree_b4", kind="attend", lens=LENS_8B, counts="16,16,13,16", nodes=16, chain=False, hq=32, hkv=8, hd=128,
             page=64, dtype="bf16"),
        # head_dim 64, eight query heads per kv head, long contexts, odd trees
        dict(name="attend_tree_hd64", kind="attend", lens="8192,8187", counts="33,29", nodes=33, chain=False, hq=64, hkv=8, hd=64,
             page=32, dtype="bf16"),
        # large trees over long contexts: the most cache that is read and the most products
        dict(name="attend_tree_long", kind="attend", lens=",".join(["32768"] * 8), counts=",".join(["64"] * 8), nodes=64,
             chain=False, hq=32, hkv=8, hd=128, page=64, dtype="bf16"),
        # the fp32 drafter's heads, a short cache
        dict(name="attend_tiny_f32", kind="attend", lens="600,35,0", counts="8,7,8", nodes=8, chain=False, hq=4, hkv=2, hd=64, page=16,
             dtype="f32"),
        # one user's tree of a block of 16
        dict(name="tree_b1", kind="tree", batch=1, nodes=16, ragged=False, vocab=151936),
        # a full batch of large trees
        dict(name="tree_b64", kind="tree", batch=64, nodes=255, ragged=True, vocab=151936),
    ]


# ---------------------------------------------------------------------------------- cases of the ranges

def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _join(v):
    return ",".join(str(x) for x in v)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _spread(rng, batch, lo, hi):
    """Lengths of a batch: all near one length drawn on a logarithmic scale."""
    top = _log(rng, max(lo, 1), hi)
    return [rng.randint(max(lo, top // 3), top) for _ in range(batch)]


def _heads(rng, dtype):
    if rng.random() < 0.5:
        return (4, 2, 64) if dtype == "f32" else rng.choice([(32, 8, 128), (64, 8, 64)])
    hkv = rng.choice([1, 2, 4, 8])
    return hkv * rng.choice([1, 2, 3, 4, 5, 7, 8]), hkv, rng.choice([64, 128])


def draw(rng):
    while True:
        c = _draw(rng)
        if _cost(c) <= max(_cost(x) for x in listed()):
            return c


def _cost(c):
    """Seconds at about 6 TB/s or 1.5 PFLOP/s, whichever is more; fp32 products on the CUDA cores."""
    w = work(c)
    return max(w["bytes"] / 6e12, w["flops"] / (1.5e15 if c.get("dtype") == "bf16" else 2e13))


def _draw(rng):
    kind = rng.choice(["rope", "rope", "append", "append", "fork", "commit", "copy", "attend", "attend", "attend", "attend", "tree"])
    if kind == "tree":
        return dict(kind=kind, batch=_log(rng, 1, 64), nodes=_log(rng, 1, 255), ragged=rng.random() < 0.5, vocab=_log(rng, 4001, 201088))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    hq, hkv, hd = _heads(rng, dtype)
    if kind == "rope":
        rot = hd if rng.random() < 0.6 else rng.choice([16, 32, hd // 2])
        scaling = rng.choice(["none", "linear", "ntk", "yarn"])
        return dict(kind=kind, rows=_log(rng, 1, 12000), hq=hq, hkv=hkv, hd=hd, rot=rot, layout=rng.choice(["half", "interleaved"]),
                    dtype=dtype, scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 16.0]),
                    theta=rng.choice([1e4, 1e6]), start=rng.choice([0, 0, _log(rng, 100, 1000000)]), backward=rng.random() < 0.4)
    page = rng.choice([16, 32, 64, 128])
    if kind == "append":
        batch = _log(rng, 1, 32)
        lens = _spread(rng, batch, 0, 4096)
        counts = [rng.randint(0, 3) if rng.random() < 0.1 else n for n in _spread(rng, batch, 1, max(1, 4096 // batch))]
        if sum(counts) == 0:
            counts[0] = 1
        return dict(kind=kind, lens=_join(lens), counts=_join(counts), hq=hq, hkv=hkv, hd=hd, page=page, layers=rng.randint(1, 2),
                    rot=hd if rng.random() < 0.7 else hd // 2, layout=rng.choice(["half", "interleaved"]), dtype=dtype,
                    theta=rng.choice([1e4, 1e6]))
    layers = rng.randint(1, 40)
    if kind == "fork":
        batch = _log(rng, 1, 12)
        return dict(kind=kind, lens=_join(_spread(rng, batch, 1, 600)), ways=rng.randint(1, 4), grow=rng.randint(1, 40), layers=layers,
                    hkv=hkv, hd=hd, page=page, dtype=dtype)
    if kind == "commit":
        batch = _log(rng, 1, 32)
        return dict(kind=kind, lens=_join(_spread(rng, batch, 0, 700)), nodes=_log(rng, 1, 128), layers=layers, hkv=hkv, hd=hd,
                    page=page, dtype=dtype)
    if kind == "copy":
        return dict(kind=kind, pairs=_log(rng, 1, 64), layers=layers, hkv=hkv, hd=hd, page=page, dtype=dtype)
    batch = _log(rng, 1, 48)
    lens = _spread(rng, batch, 0, max(1, min(65536, 262144 // batch)))
    chain = rng.random() < 0.3
    nodes = 1 if chain and rng.random() < 0.5 else _log(rng, 1, 200)
    counts = [nodes if rng.random() < 0.7 else rng.randint(0, nodes) for _ in range(batch)]
    if max(counts) == 0:
        counts[0] = nodes
    return dict(kind=kind, lens=_join(lens), counts=_join(counts), nodes=nodes, chain=chain, hq=hq, hkv=hkv, hd=hd, page=page, dtype=dtype)


# ------------------------------------------------------------------------------------------------ inputs

class _Rand:
    """Named streams of samples on the GPU, each a function of (seed, name) alone."""

    def __init__(self, seed):
        self.seed = seed

    def _hash(self, name):
        h = 1469598103934665603
        for ch in "%d/%s" % (self.seed, name):
            h = (h ^ ord(ch)) * 1099511628211 % (1 << 63)
        return h

    def normal(self, name, shape, dtype, scale=1.0):
        g = torch.Generator(device="cuda").manual_seed(self._hash(name))
        t = torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=g)
        return t if scale == 1.0 else t.mul_(scale)

    def host(self, name):
        return np.random.RandomState(self._hash(name) % (1 << 32))


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int32), device="cuda")


def _up(a, b):
    return -(-a // b)


def _frequencies(c):
    """Angle per position of each pair, and the factor on the rotated values (scalings by their papers' formulas)."""
    rot, theta, f, kind = c["rot"], c["theta"], c.get("factor", 1.0), c.get("scaling", "none")
    if kind == "ntk":
        theta = theta * f ** (rot / (rot - 2.0))
    inv = [theta ** (-2.0 * j / rot) for j in range(rot // 2)]
    if kind == "linear":
        return [x / f for x in inv], 1.0
    if kind == "yarn":      # pairs that turn more than 32 times in 4096 positions stay, those under one turn stretch
        at = [rot * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(theta)) for turns in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot // 2 - 1)
        keep = [1.0 - min(max((j - lo) / max(hi - lo, 1e-3), 0.0), 1.0) for j in range(rot // 2)]
        return [x * k + x / f * (1.0 - k) for x, k in zip(inv, keep)], 0.1 * math.log(f) + 1.0
    return inv, 1.0


def _phase(inv):
    """Turns per position in units of 2^-64."""
    return torch.tensor([int(round(x / (2.0 * math.pi) * 2.0 ** 64)) % (1 << 63) for x in inv], dtype=torch.int64, device="cuda")


def _parents(rng, batch, nodes):
    """Random trees, node 0 the root: a node hangs on one of the eight before it."""
    i = np.arange(nodes)
    back = np.floor(rng.rand(batch, nodes) * np.minimum(i, 8)).astype(np.int64)
    p = i - 1 - back
    p[:, 0] = -1
    return p.astype(np.int32)


def _ancestors(parents):
    """[batch][nodes][nodes] truth: node j is node i or above it (host, in preparing inputs)."""
    batch, n = parents.shape
    a = np.zeros((batch, n, n), bool)
    rows = np.arange(batch)
    for i in range(n):
        a[:, i, i] = True
        above = parents[:, i] >= 0
        a[above, i] |= a[rows[above], parents[above, i]]
    return a


def _words(a):
    """Truth values packed into 32-bit words along the last axis, the lowest bit first."""
    n = a.shape[-1]
    w = np.zeros(a.shape[:-1] + (_up(n, 32) * 32,), np.uint64)
    w[..., :n] = a
    return (w.reshape(a.shape[:-1] + (-1, 32)) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)


def _cache(c, r, lens, held, slots, spare):
    """Pools and tables: sequence b has `held[b]` pages, its pages anywhere in the pool; what is free holds old values."""
    pages = sum(held) + spare
    shape = (c.get("layers", 1), pages, c["hkv"], c["page"], c["hd"])
    s = {"k": r.normal("k", shape, _dtype(c)), "v": r.normal("v", shape, _dtype(c))}
    order = r.host("pages").permutation(pages).astype(np.int32)
    width = max(held) + max(4, c.get("width", 4))
    table = np.full((slots, width), -1, np.int32)
    refs = np.zeros(pages, np.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        refs[order[at:at + n]] = 1
        at += n
    free = np.zeros(pages, np.int32)
    free[:spare] = order[at:]
    full = np.zeros(slots, np.int32)
    full[:len(lens)] = lens
    have = np.zeros(slots, np.int32)
    have[:len(held)] = held
    s.update(table=_i32(table), lens=_i32(full), held=_i32(have), refs=_i32(refs), free=_i32(free), n_free=_i32([spare]))
    return s


def _handle(c, s, nodes):
    """The framework's cache around those pools and tables, as a server keeps it."""
    import paper_2606_02091_gb300 as lib
    s["lib"] = lib
    s["cache"] = lib.PagedCache(k=s["k"], v=s["v"], table=s["table"], lens=s["lens"], held=s["held"], refs=s["refs"], free=s["free"],
                                n_free=s["n_free"], n_q_heads=c.get("hq", c["hkv"]), max_nodes=nodes)


def prepare(case, seed):
    c, r = case, _Rand(seed)
    kind = c["kind"]
    if kind == "tree":
        h = r.host("tree")
        batch, n = c["batch"], c["nodes"]
        parents = _parents(h, batch, n)
        counts = h.randint(max(1, n // 2), n + 1, batch) if c["ragged"] else np.full(batch, n)
        tokens = h.randint(0, c["vocab"], (batch, n))
        choice = h.randint(0, c["vocab"], (batch, n))       # the target's token after each node:
        for i in range(1, n):                               # with luck the token of one of its children
            agree = h.rand(batch) < 0.7
            choice[agree, parents[agree, i]] = tokens[agree, i]
        s = {"kind": kind, "parents": _i32(parents), "counts": _i32(counts), "tokens": _i32(tokens), "choice": _i32(choice),
             "mask": _i32(np.zeros((batch, n, _up(n, 32)))), "depth": _i32(np.zeros((batch, n))), "accept": _i32(np.zeros(batch)),
             "path": _i32(np.zeros((batch, n))), "next": _i32(np.zeros(batch))}
        if own:
            import paper_2606_02091_gb300 as lib
            s["lib"] = lib
        return s
    if kind == "rope":
        inv, magnitude = _frequencies(c)
        heads = c["hq"] + c["hkv"]
        rows = r.normal("x", (c["rows"], heads + c["hkv"], c["hd"]), _dtype(c))
        s = {"kind": kind, "x": rows[:, :heads], "phase": _phase(inv), "magnitude": magnitude, "layout": c["layout"],
             "backward": c["backward"], "out": torch.zeros((c["rows"], heads, c["hd"]), dtype=_dtype(c), device="cuda")}
        s["positions"] = _i32(c["start"] + np.arange(c["rows"]) % max(1, c["rows"] // 4 + 1))
        if own:
            import paper_2606_02091_gb300 as lib
            s["lib"] = lib
        return s
    page = c["page"]
    if kind == "append":
        lens, counts = _ints(c["lens"]), _ints(c["counts"])
        batch, n = len(lens), max(counts)
        s = _cache(c, r, lens, [_up(a + b, page) for a, b in zip(lens, counts)], batch, 3)
        qkv = r.normal("qkv", (batch, n, c["hq"] + 2 * c["hkv"], c["hd"]), _dtype(c))
        s.update(kind=kind, q=qkv[:, :, :c["hq"]], kn=qkv[:, :, c["hq"]:c["hq"] + c["hkv"]], vn=qkv[:, :, c["hq"] + c["hkv"]:],
                 counts=_i32(counts), total=sum(counts), phase=_phase(_frequencies(c)[0]), layout=c["layout"],
                 out=torch.zeros((batch, n, c["hq"], c["hd"]), dtype=_dtype(c), device="cuda"))
        s["layer"] = c["layers"] - 1
        parents = _parents(r.host("tree"), batch, n)
        depth = np.zeros((batch, n), np.int64)
        for i in range(1, n):
            depth[:, i] = depth[np.arange(batch), parents[:, i]] + 1
        s["depth"] = _i32(depth)
        if own:
            _handle(c, s, min(n, 1024))
        return s
    if kind == "fork":
        lens = _ints(c["lens"])
        n, ways, grow = len(lens), c["ways"], c["grow"]
        spare = n * (1 + ways) * (2 + _up(grow, page))
        s = _cache(dict(c, width=2 + _up(grow, page)), r, lens, [_up(a, page) for a in lens], n * (1 + ways), spare)
        s.update(kind=kind, src=_i32(np.repeat(np.arange(n), ways)), dst=_i32(n + np.arange(n * ways)),
                 back=_i32(lens + [0] * (n * ways)), grow=_i32([grow] * (n * (1 + ways))))
    elif kind == "commit":
        lens, n = _ints(c["lens"]), c["nodes"]
        h = r.host("tree")
        batch = len(lens)
        s = _cache(c, r, lens, [_up(a + n, page) for a in lens], batch, 5)
        parents = _parents(h, batch, n)
        path = np.full((batch, n), -1, np.int32)
        accept = np.zeros(batch, np.int32)
        for b in range(batch):      # from a random node up to the root
            at, up = int(h.randint(n)), []
            while at >= 0:
                up.append(at)
                at = parents[b, at]
            accept[b] = len(up)
            path[b, :len(up)] = up[::-1]
        s.update(kind=kind, accept=_i32(accept), path=_i32(path), back=_i32(lens), grow=_i32([n] * batch), most=int(accept.max()))
    elif kind == "copy":
        n = c["pairs"]
        s = _cache(c, r, [], [2 * n], 1, 1)
        order = r.host("pairs").permutation(2 * n)
        s.update(kind=kind, src=_i32(order[:n]), dst=_i32(order[n:]))
    else:
        lens, counts = _ints(c["lens"]), _ints(c["counts"])
        batch, n = len(lens), c["nodes"]
        s = _cache(c, r, lens, [_up(a + b, page) for a, b in zip(lens, counts)], batch, 3)
        s.update(kind=kind, counts=_i32(counts), q=r.normal("q", (batch, n, c["hq"], c["hd"]), _dtype(c), 1.5),
                 out=torch.zeros((batch, n, c["hq"], c["hd"]), dtype=_dtype(c), device="cuda"),
                 lse=torch.zeros((batch, n, c["hq"]), dtype=torch.float32, device="cuda"), width=max(max(_up(a + b, page) for a, b in zip(lens, counts)), 1))
        s["mask"] = None if c["chain"] else _i32(_words(_ancestors(_parents(r.host("tree"), batch, n))))
    if own:
        _handle(c, s, c.get("nodes", 1))
    return s


# ---------------------------------------------------------------------------------------- one pass

def run(state):
    return _own(state) if own else _PLAIN[state["kind"]](state)


_POOLS = ("k", "v", "table", "lens", "held", "refs", "free", "n_free")


def _own(s):
    kind, cache, lib = s["kind"], s.get("cache"), s["lib"]
    if kind == "rope":
        lib.rope(s["x"], s["positions"], s["phase"], s["out"], layout=s["layout"], magnitude=s["magnitude"], backward=s["backward"])
        return s["out"]
    if kind == "append":
        cache.append(s["layer"], s["q"], s["kn"], s["vn"], s["counts"], s["phase"], s["out"], depth=s["depth"], layout=s["layout"])
        return {"q": s["out"], "k": s["k"], "v": s["v"]}
    if kind == "fork":
        cache.truncate(s["back"])
        cache.fork(s["src"], s["dst"])
        cache.reserve(s["grow"])
        return {n: s[n] for n in _POOLS}
    if kind == "commit":
        cache.truncate(s["back"])
        cache.reserve(s["grow"])
        cache.commit(s["accept"], s["path"])
        return {n: s[n] for n in _POOLS}
    if kind == "copy":
        cache.copy_pages(s["src"], s["dst"])
        return {"k": s["k"], "v": s["v"]}
    if kind == "attend":
        cache.attend(0, s["q"], s["counts"], s["out"], mask=s["mask"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    lib.tree_plan(s["parents"], s["counts"], s["mask"], s["depth"])
    lib.tree_accept(s["tokens"], s["parents"], s["choice"], s["counts"], s["accept"], s["path"], s["next"])
    return {n: s[n] for n in ("mask", "depth", "accept", "path", "next")}


# The plain forms: elementary torch operations, arithmetic in 32 bits, rounded once.

def _turn(x, positions, phase, layout, magnitude=1.0, sign=1.0):
    """x [rows][heads][hd], positions [rows]."""
    turns = (positions.long()[:, None] * phase).float() * 2.0 ** -64
    cos = (torch.cos(turns * (2.0 * math.pi)) * magnitude)[:, None]
    sin = (torch.sin(turns * (2.0 * math.pi)) * (magnitude * sign))[:, None]
    half = phase.numel()
    y = x.float()
    if layout == "half":
        a, b = y[..., :half], y[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., 2 * half:]], -1).to(x.dtype)


def _plain_rope(s):
    return _turn(s["x"], s["positions"], s["phase"], s["layout"], s["magnitude"], -1.0 if s["backward"] else 1.0)


def _plain_append(s):
    batch, n, hq, hd = s["q"].shape
    page = s["k"].shape[3]
    i = torch.arange(n, device="cuda")
    there = (i < s["counts"][:, None]).flatten()
    rows = torch.argsort(~there, stable=True)[:s["total"]]
    b, i = rows // n, rows % n
    at = s["lens"].long()[b] + s["depth"].long()[b, i]
    slot = s["lens"].long()[b] + i
    ids = s["table"].long()[b, slot // page]
    s["out"][b, i] = _turn(s["q"][b, i], at, s["phase"], s["layout"])
    s["k"][s["layer"], ids, :, slot % page] = _turn(s["kn"][b, i], at, s["phase"], s["layout"])
    s["v"][s["layer"], ids, :, slot % page] = s["vn"][b, i]
    return {"q": s["out"], "k": s["k"], "v": s["v"]}


def _put(to, index, values, where):
    """to[index] = values where `where`; `to` one-dimensional, the indexes distinct."""
    wide = torch.cat([to, to[:1]])
    wide[torch.where(where, index, to.numel())] = values
    to.copy_(wide[:-1])


def _plain_trim(s, keep):
    """Give back the pages of sequence b from number keep[b] on."""
    slots, width = s["table"].shape
    i = torch.arange(width, device="cuda")
    gone = ((i >= keep[:, None]) & (i < s["held"][:, None])).flatten()
    ids = s["table"].long().clamp(min=0).flatten()
    s["refs"] -= torch.zeros_like(s["refs"]).scatter_add(0, ids, gone.int())
    none = gone & (s["refs"][ids] == 0)
    entry = torch.arange(slots * width, device="cuda")
    last = torch.full_like(s["refs"], -1, dtype=torch.int64).scatter_reduce(0, ids, torch.where(none, entry, -1), "amax")
    push = none & (last[ids] == entry)
    count = push.long().cumsum(0)
    _put(s["free"], s["n_free"].long() + count - 1, ids.int(), push)
    s["n_free"] += count[-1:].int()
    s["table"].copy_(torch.where(gone.view(slots, width), -1, s["table"]))
    s["held"].copy_(torch.minimum(s["held"], keep.int()))


def _plain_truncate(s):
    page = s["k"].shape[3]
    s["lens"].copy_(torch.minimum(s["lens"], s["back"]))
    _plain_trim(s, (s["lens"] + page - 1) // page)


def _plain_reserve(s, grow):
    page, width = s["k"].shape[3], s["table"].shape[1]
    lens, held, refs, table = s["lens"].long(), s["held"].long(), s["refs"].long(), s["table"].long()
    new = (lens + grow + page - 1) // page - held
    new = torch.where(grow > 0, new.clamp(min=0), 0)
    tail = table.gather(1, (lens // page).clamp(max=width - 1)[:, None])[:, 0]
    part = (grow > 0) & (lens % page != 0)
    same = (tail[:, None] == tail) & part[:, None] & part
    rank = torch.tril(same, -1).sum(1)
    copy = part & (refs[tail.clamp(min=0)] - rank > 1)
    need = new + copy
    first = need.cumsum(0) - need
    top = s["n_free"].long()
    i = torch.arange(width, device="cuda")
    # the copy of the tail page comes first, then the new pages in order
    fresh = (i >= held[:, None]) & (i < (held + new)[:, None])
    at = first[:, None] + copy[:, None] + i - held[:, None]
    at = torch.where(copy[:, None] & (i == (lens // page)[:, None]), first[:, None], at)
    take = fresh | (copy[:, None] & (i == (lens // page)[:, None]))
    ids = s["free"].long()[(top - 1 - at).clamp(min=0, max=s["free"].numel() - 1)]
    moved = copy[:, None] & (i == (lens // page)[:, None])
    dst = torch.where(moved, ids, 0).sum(1)
    # a sequence without a copy "copies" its own first page onto itself
    home = table[:, 0].clamp(min=0)
    src, dst = torch.where(copy, tail, home), torch.where(copy, dst, home)
    kept = (torch.arange(page, device="cuda") < (lens % page)[:, None])[:, None, :, None]     # the page's tokens
    for pool in (s["k"], s["v"]):
        pool[:, dst] = torch.where(kept, pool[:, src], pool[:, dst])
    s["refs"] -= torch.zeros_like(s["refs"]).scatter_add(0, tail.clamp(min=0), copy.int())
    s["refs"] += torch.zeros_like(s["refs"]).scatter_add(0, torch.where(take, ids, 0).flatten(), take.int().flatten())
    s["table"].copy_(torch.where(take, ids, table))
    s["held"].copy_(held + new)
    s["n_free"] -= need.sum().int()


def _plain_fork(s):
    _plain_truncate(s)
    page = s["k"].shape[3]
    src, dst = s["src"].long(), s["dst"].long()
    keep = (s["lens"][src] + page - 1) // page
    i = torch.arange(s["table"].shape[1], device="cuda")
    share = i < keep[:, None]
    rows = torch.where(share, s["table"][src], -1)
    s["refs"] += torch.zeros_like(s["refs"]).scatter_add(0, rows.long().clamp(min=0).flatten(), share.int().flatten())
    s["table"][dst] = rows
    s["held"][dst] = keep
    s["lens"][dst] = s["lens"][src]
    _plain_reserve(s, s["grow"].long())
    return {n: s[n] for n in _POOLS}


def _plain_commit(s):
    _plain_truncate(s)
    _plain_reserve(s, s["grow"].long())
    page, lens = s["k"].shape[3], s["lens"].long()
    j = torch.arange(s["most"], device="cuda")
    there = j < s["accept"][:, None]
    # past the accepted path a row is moved onto itself
    from_ = lens[:, None] + torch.where(there, s["path"][:, :s["most"]].long(), 0)
    to = lens[:, None] + torch.where(there, j, 0)
    batch = torch.arange(lens.numel(), device="cuda")[:, None]
    table = s["table"].long()
    for pool in (s["k"], s["v"]):
        rows = pool[:, table[batch, from_ // page], :, from_ % page]
        root = pool[:, table[batch, lens[:, None] // page], :, lens[:, None] % page]
        rows = torch.where(there[:, :, None, None, None], rows, root)
        pool[:, table[batch, to // page], :, to % page] = rows
    s["lens"] += s["accept"]
    _plain_trim(s, (s["lens"] + page - 1) // page)
    return {n: s[n] for n in _POOLS}


def _plain_copy(s):
    src, dst = s["src"].long(), s["dst"].long()
    s["k"][:, dst] = s["k"][:, src]
    s["v"][:, dst] = s["v"][:, src]
    return {"k": s["k"], "v": s["v"]}


def _plain_attend(s):
    q = s["q"]
    batch, n, hq, hd = q.shape
    hkv, page = s["k"].shape[2:4]
    g, ids = hq // hkv, s["table"][:, :s["width"]].long().clamp(min=0)
    k, v = (p[0][ids].float().transpose(1, 2).reshape(batch, hkv, -1, hd) for p in (s["k"], s["v"]))
    keys = k.shape[2]
    i, j = torch.arange(n, device="cuda"), torch.arange(keys, device="cuda")
    lens, counts = s["lens"].long(), s["counts"].long()
    t = j - lens[:, None]                                    # number of the tree's node, negative in the context
    inside = (t < counts[:, None])[:, None, :] & (i < counts[:, None])[:, :, None]
    if s["mask"] is None:
        seen = t[:, None, :] <= i[:, None]
    else:
        at = t.clamp(0, n - 1)
        words = s["mask"].gather(2, (at // 32)[:, None, :].expand(batch, n, keys))
        seen = ((words >> (at % 32)[:, None, :]) & 1).bool() | (t < 0)[:, None, :]
    seen = (seen & inside)[:, None, :, None, :]              # [batch][1][n][1][keys]
    v = torch.where((t < counts[:, None])[:, None, :, None], v, 0.0)
    x = q.float().view(batch, n, hkv, g, hd).transpose(1, 2).reshape(batch, hkv, n * g, hd)
    score = (x @ k.transpose(2, 3)).view(batch, hkv, n, g, keys) * (hd ** -0.5)
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    o = (p.view(batch, hkv, n * g, keys) @ v).view(batch, hkv, n, g, hd) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    return {"out": o.transpose(1, 2).reshape(batch, n, hq, hd).to(q.dtype), "lse": lse.transpose(1, 2).reshape(batch, n, hq)}


def _plain_tree(s):
    batch, n = s["parents"].shape
    i = torch.arange(n, device="cuda")
    there = i < s["counts"][:, None]
    parent = torch.where(there, s["parents"], -1).long()
    # the node itself and its parent, squared until every ancestor is reached
    above = (parent[:, :, None] == i).float() + torch.eye(n, device="cuda")
    for _ in range((n - 1).bit_length()):
        above = (above @ above).clamp(max=1.0)
    above = above * there[:, :, None] * there[:, None, :]
    bits = torch.zeros((batch, n, -(-n // 32) * 32), dtype=torch.int64, device="cuda")
    bits[:, :, :n] = above.long()
    words = (bits.view(batch, n, -1, 32) << torch.arange(32, device="cuda")).sum(-1)
    mask = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
    depth = (above.sum(-1).int() - 1).clamp(min=0)
    up = parent.clamp(min=0)
    match = there & (parent >= 0) & (s["tokens"] == s["choice"].gather(1, up))
    first = torch.full((batch, n), n, device="cuda").scatter_reduce(1, up, torch.where(match, i, n), "amin")
    ok = (match & (first.gather(1, up) == i)) | (i == 0)
    on = ((above @ (~ok).float()[:, :, None])[:, :, 0] == 0) & there & (above[:, :, 0] > 0)
    accept = on.sum(1).int()
    path = torch.full((batch, n + 1), -1, dtype=torch.int32, device="cuda")
    path.scatter_(1, torch.where(on, depth.long(), n), torch.where(on, i, -1).int())
    end = torch.where(on, i, 0).amax(1, keepdim=True)
    following = torch.where(accept > 0, s["choice"].gather(1, end)[:, 0], -1)
    return {"mask": mask, "depth": depth, "accept": accept, "path": path[:, :n], "next": following}


_PLAIN = {"rope": _plain_rope, "append": _plain_append, "fork": _plain_fork, "commit": _plain_commit, "copy": _plain_copy,
          "attend": _plain_attend, "tree": _plain_tree}


# ------------------------------------------------------------------------------------------- work

def work(case):
    c = case
    if c["kind"] == "tree":
        n, w = c["batch"] * c["nodes"], _up(c["nodes"], 32)
        return {"bytes": n * (4 * 3 + 4 * w + 4 + 4) + 12 * c["batch"], "flops": n}
    e = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "rope":
        n = c["rows"] * (c["hq"] + c["hkv"])
        return {"bytes": 2 * e * n * c["hd"] + 4 * c["rows"] + 4 * c["rot"], "flops": 3 * n * c["rot"]}
    row = 2 * c["hkv"] * c["hd"] * e        # a token's key and value of one layer
    if c["kind"] == "append":
        n = sum(_ints(c["counts"]))
        return {"bytes": 2 * n * (row + c["hq"] * c["hd"] * e) + 8 * n, "flops": 3 * n * (c["hq"] + c["hkv"]) * c["rot"]}
    if c["kind"] == "copy":
        return {"bytes": 2 * c["pairs"] * c["layers"] * c["page"] * row, "flops": 0}
    if c["kind"] == "fork":     # a partial page that `ways` + 1 sequences share is copied `ways` times, its tokens only
        part = sum(x % c["page"] for x in _ints(c["lens"]))
        return {"bytes": 2 * c["ways"] * part * c["layers"] * row + 64, "flops": 0}
    if c["kind"] == "commit":   # a path's nodes but the root move: a random node of these trees is about nodes / 8 deep
        deep = max(1, c["nodes"] // 8)
        return {"bytes": 2 * len(_ints(c["lens"])) * deep * c["layers"] * row, "flops": 0}
    lens, counts = _ints(c["lens"]), _ints(c["counts"])
    keys = sum(a + b for a, b in zip(lens, counts) if b)
    rows = sum(counts) * c["hq"]
    pairs = sum(b * (a + 1) for a, b in zip(lens, counts)) * c["hq"]
    return {"bytes": keys * row + rows * (2 * c["hd"] * e + 4) + (0 if c["chain"] else 4 * sum(counts) * _up(c["nodes"], 32)),
            "flops": 4 * pairs * c["hd"]}


# ------------------------------------------------------------------------------------------ exact

def _whirl(x, angle, layout, magnitude, sign):
    """x [rows][heads][hd] in 64 bits as complex numbers times magnitude e^(i sign angle)."""
    r = 2 * angle.shape[1]
    z = torch.polar(torch.full_like(angle, magnitude), sign * angle)[:, None]
    y = x.double().clone()
    if layout == "half":
        t = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * z
        y[..., :r // 2], y[..., r // 2:r] = t.real, t.imag
    else:
        t = torch.view_as_complex(y[..., :r].reshape(y.shape[0], y.shape[1], r // 2, 2).contiguous()) * z
        y[..., :r] = torch.view_as_real(t).reshape(y.shape[0], y.shape[1], r)
    return y


def _exact_pages(c, s):
    """The page calls one sequence at a time, on the host's copies of the tables; the pools in 64 bits."""
    page = c["page"]
    table, lens, held, refs, free = ([list(r) for r in s["table"].tolist()], s["lens"].tolist(), s["held"].tolist(),
                                     s["refs"].tolist(), s["free"].tolist()[:int(s["n_free"])])
    k, v = s["k"].double(), s["v"].double()

    def drop(b, keep):
        for i in range(keep, held[b]):
            p = table[b][i]
            refs[p] -= 1
            if refs[p] == 0:
                free.append(p)
            table[b][i] = -1
        held[b] = min(held[b], keep)

    for b, n in enumerate(s["back"].tolist()):
        lens[b] = min(lens[b], n)
        drop(b, -(-lens[b] // page))
    if c["kind"] == "fork":
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            n = -(-lens[a] // page)
            table[b][:n] = table[a][:n]
            for p in table[a][:n]:
                refs[p] += 1
            lens[b], held[b] = lens[a], n
    for b, n in enumerate(s["grow"].tolist()):
        if not n:
            continue
        if lens[b] % page and refs[table[b][lens[b] // page]] > 1:
            old, new = table[b][lens[b] // page], free.pop()
            rows = lens[b] % page
            k[:, new, :, :rows], v[:, new, :, :rows] = k[:, old, :, :rows], v[:, old, :, :rows]
            refs[old], refs[new], table[b][lens[b] // page] = refs[old] - 1, 1, new
        while held[b] * page < lens[b] + n:
            table[b][held[b]] = free.pop()
            refs[table[b][held[b]]] = 1
            held[b] += 1
    if c["kind"] == "commit":
        for b, n in enumerate(s["accept"].tolist()):
            for j, node in enumerate(s["path"][b, :n].tolist()):
                x, y = lens[b] + node, lens[b] + j
                px, py = table[b][x // page], table[b][y // page]
                k[:, py, :, y % page] = k[:, px, :, x % page].clone()
                v[:, py, :, y % page] = v[:, px, :, x % page].clone()
    return dict({n: None for n in _POOLS}, k=k, v=v)


def exact(case, seed):
    c = case
    if c["kind"] == "tree":
        return None
    s = prepare(case, seed)
    if c["kind"] in ("fork", "commit"):
        return _exact_pages(c, s)
    if c["kind"] == "copy":
        k, v = s["k"].double(), s["v"].double()
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            k[:, b], v[:, b] = s["k"][:, a].double(), s["v"][:, a].double()
        return {"k": k, "v": v}
    if c["kind"] == "rope":
        inv, magnitude = _frequencies(c)
        angle = s["positions"].double()[:, None] * torch.tensor(inv, dtype=torch.float64, device="cuda")
        return _whirl(s["x"], angle, c["layout"], magnitude, -1.0 if c["backward"] else 1.0)
    lens, counts, page, hkv, hd = _ints(c["lens"]), _ints(c["counts"]), c["page"], c["hkv"], c["hd"]
    table = s["table"].long()
    if c["kind"] == "append":
        inv = torch.tensor(_frequencies(c)[0], dtype=torch.float64, device="cuda")
        q, k, v = s["out"].double(), s["k"].double(), s["v"].double()
        for b, n in enumerate(counts):
            angle = (lens[b] + s["depth"][b, :n]).double()[:, None] * inv
            q[b, :n] = _whirl(s["q"][b, :n], angle, c["layout"], 1.0, 1.0)
            at = torch.arange(lens[b], lens[b] + n, device="cuda")
            k[s["layer"], table[b, at // page], :, at % page] = _whirl(s["kn"][b, :n], angle, c["layout"], 1.0, 1.0)
            v[s["layer"], table[b, at // page], :, at % page] = s["vn"][b, :n].double()
        return {"q": q, "k": k, "v": v}
    if sum(a * b for a, b in zip(lens, counts)) * c["hq"] * hd * 4.0 > 6e12:
        return None     # too long in 64 bits
    g = c["hq"] // hkv
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    above = _ancestors(_parents(_Rand(seed).host("tree"), len(lens), c["nodes"])) if not c["chain"] else None
    for b, n in enumerate(counts):
        if not n:
            continue
        total = lens[b] + n
        at = torch.arange(total, device="cuda")
        seen = torch.ones((n, total), dtype=torch.bool, device="cuda")
        seen[:, lens[b]:] = torch.tril(torch.ones((n, n), dtype=torch.bool, device="cuda")) if c["chain"] else \
            torch.from_numpy(above[b, :n, :n].copy()).cuda()
        for h in range(hkv):
            key = s["k"][0][table[b, at // page], h, at % page].double()
            value = s["v"][0][table[b, at // page], h, at % page].double()
            for m in range(h * g, h * g + g):
                z = (s["q"][b, :n, m].double() @ key.T / hd ** 0.5).masked_fill(~seen, -math.inf)
                lse[b, :n, m] = z.logsumexp(-1)
                out[b, :n, m] = z.softmax(-1) @ value
    return {"out": out, "lse": lse}
