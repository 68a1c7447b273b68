"""A step of a server that samples several continuations of a prompt, and the training of the same heads.

- ``norm``    the root-mean-square norm of every query and key head with the rotary positions in the same pass: forward
              alone, forward and backward (training), and with a step's new keys and values written to the pages.
- ``shared``  attention of a batch over a paged cache in which groups of sequences share their leading pages (samples and
              beams of one prompt): which sequences share is found from the page tables, then `layers` layers attend.
- ``sample``  drafted blocks and trees kept or redrawn by the target's probabilities, from given random numbers.

Pools are [layers][pages][kv heads][page size][head dim]; pages lie in arbitrary order, as they do once pages have been
freed and taken again. Head counts, head sizes, context lengths and vocabularies are those of this repository's drafters
and workloads, or generic ones.
"""
import math

import numpy as np
import torch

own = False

LENS_8B = "2668,2687,3853,1355"      # the benchmark's ragged batch
EPS = 1e-6


def listed():
    return [
        # the four prompts of the benchmark's batch: q and k heads of a fused QKV projection
        dict(name="norm_prompt", kind="norm", mode="forward", rows=10563, hq=32, hkv=8, hd=128, rot=128, layout="half", dtype="bf16",
             theta=1e6, start=0),
        # a training step's rows: both directions, and the gains' gradients over all rows and heads
        dict(name="norm_train", kind="norm", mode="train", rows=8192, hq=32, hkv=8, hd=128, rot=128, layout="half", dtype="bf16",
             theta=1e6, start=0),
        # one layer's new tokens of a step on their way into the pages: trees of 16 nodes in four sequences (latency)
        dict(name="norm_pages_b4", kind="norm", mode="pages", lens=LENS_8B, nodes=16, hq=32, hkv=8, hd=128, page=64, rot=128, layout="half",
             dtype="bf16", theta=1e6),
        # the fp32 drafter's heads, interleaved pairs in half of each head, far positions, both directions
        dict(name="norm_train_f32", kind="norm", mode="train", rows=601, hq=4, hkv=2, hd=64, rot=32, layout="interleaved", dtype="f32",
             theta=1e6, start=100000),
        # sixteen samples of one prompt, a token each (latency)
        dict(name="shared_samples", kind="shared", prefixes="4096", ways=16, own="40-300", nodes=1, ragged=False, chain=True, hq=32, hkv=8,
             hd=128, page=16, layers=2, dtype="bf16"),
        # eight samples of a long prompt of odd length, drafted trees of 16 nodes
        dict(name="shared_trees", kind="shared", prefixes="8187", ways=8, own="100-900", nodes=16, ragged=True, chain=False, hq=32, hkv=8,
             hd=128, page=64, layers=2, dtype="bf16"),
        # the benchmark's four prompts with four beams each, short drafted chains, head_dim 64
        dict(name="shared_beams_hd64", kind="shared", prefixes=LENS_8B, ways=4, own="1-200", nodes=5, ragged=True, chain=True, hq=64, hkv=8,
             hd=64, page=32, layers=2, dtype="bf16"),
        # a full server: four long documents, sixteen questions to each, small trees
        dict(name="shared_long", kind="shared", prefixes="32768,32768,30001,32768", ways=16, own="256-2048", nodes=4, ragged=False, chain=False,
             hq=32, hkv=8, hd=128, page=64, layers=2, dtype="bf16"),
        # the fp32 drafter's heads, two prompts, three beams each
        dict(name="shared_f32", kind="shared", prefixes="600,300", ways=3, own="0-35", nodes=8, ragged=True, chain=False, hq=4, hkv=2, hd=64,
             page=16, layers=2, dtype="f32"),
        # one user's drafted block of 16 (latency)
        dict(name="sample_block_b1", kind="sample", mode="drawn", batch=1, nodes=16, ways=1, vocab=151936, ragged=False),
        # a full batch of drafted blocks
        dict(name="sample_block_b64", kind="sample", mode="drawn", batch=64, nodes=16, ways=1, vocab=151936, ragged=False),
        # trees whose siblings were drawn without replacement
        dict(name="sample_tree_b16", kind="sample", mode="distinct", batch=16, nodes=40, ways=4, vocab=201088, ragged=True),
    ]


# ---------------------------------------------------------------------------------- cases of the ranges

def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _heads(rng, dtype):
    if rng.random() < 0.5:
        return (4, 2, 64) if dtype == "f32" else rng.choice([(32, 8, 128), (64, 8, 64)])
    hkv = rng.choice([1, 2, 4, 8])
    return hkv * rng.choice([1, 2, 3, 4, 5, 7, 8]), hkv, rng.choice([64, 128])


def draw(rng):
    dearest = {}
    for x in listed():
        dearest[x["kind"]] = max(dearest.get(x["kind"], 0.0), _cost(x))
    while True:
        c = _draw(rng)
        if _cost(c) <= dearest[c["kind"]] and _size(c) <= 1 << 30:
            return c


def _cost(c):
    """Seconds at about 6 TB/s or 1.5 PFLOP/s, whichever is more; fp32 products on the CUDA cores."""
    w = work(c)
    return max(w["bytes"] / 6e12, w["flops"] / (1.5e15 if c.get("dtype") == "bf16" else 2e13))


def _size(c):
    """Elements of the largest tensor: scores, or probabilities."""
    if c["kind"] == "shared":
        return len(_ints(c["prefixes"])) * c["ways"] * c["nodes"] * c["hq"] * max(a + b for a, b in zip(*_lengths(c)))
    return c["batch"] * c["nodes"] * c["vocab"] if c["kind"] == "sample" else 0


def _draw(rng):
    kind = rng.choice(["norm", "norm", "shared", "shared", "shared", "sample", "sample"])
    if kind == "sample":
        chain = rng.random() < 0.4
        nodes = rng.randint(1, 32) if chain else _log(rng, 2, 64)
        return dict(kind=kind, mode=rng.choice(["drawn", "distinct", "picked"]), batch=_log(rng, 1, 64), nodes=nodes,
                    ways=1 if chain else rng.randint(2, 6), vocab=_log(rng, 2001, 201088), ragged=rng.random() < 0.5)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    hq, hkv, hd = _heads(rng, dtype)
    if kind == "norm":
        mode = rng.choice(["forward", "train", "pages"])
        hd = hd if mode == "pages" else rng.choice([hd, hd, 96, 256])
        rot = hd if rng.random() < 0.6 else rng.choice([16, 32, hd // 2])
        c = dict(kind=kind, mode=mode, hq=hq, hkv=hkv, hd=hd, rot=rot, layout=rng.choice(["half", "interleaved"]), dtype=dtype,
                 theta=rng.choice([1e4, 1e6]))
        if mode == "pages":
            batch = _log(rng, 1, 32)
            top = _log(rng, 1, 4096)
            return dict(c, page=rng.choice([16, 32, 64, 128]), nodes=_log(rng, 1, max(1, 2048 // batch)),
                        lens=",".join(str(rng.randint(top // 3, top)) for _ in range(batch)))
        return dict(c, rows=_log(rng, 1, 12000), start=rng.choice([0, 0, _log(rng, 100, 1000000)]))
    groups = _log(rng, 1, 6)
    top = _log(rng, 40, 65536)
    width = _log(rng, 1, 2000)
    return dict(kind=kind, prefixes=",".join(str(rng.randint(max(1, top // 2), top)) for _ in range(groups)), ways=_log(rng, 1, 24),
                own="%d-%d" % (rng.randint(0, width), width), nodes=rng.choice([1, 1, _log(rng, 2, 64)]), ragged=rng.random() < 0.5,
                chain=rng.random() < 0.5, hq=hq, hkv=hkv, hd=hd, page=rng.choice([16, 32, 64, 128]), layers=rng.randint(1, 3), dtype=dtype)


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

    def gpu(self, name):
        return torch.Generator(device="cuda").manual_seed(self._hash(name))

    def normal(self, name, shape, dtype, scale=1.0):
        t = torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=self.gpu(name))
        return t if scale == 1.0 else t.mul_(scale)

    def host(self, name):
        return np.random.RandomState(self._hash(name) % (1 << 32))


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int32), device="cuda")


def _up(a, b):
    return -(-a // b)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _frequencies(c):
    """Angle per position of each pair."""
    return [c["theta"] ** (-2.0 * j / c["rot"]) for j in range(c["rot"] // 2)]


def _phase(inv):
    """Turns per position in units of 2^-64."""
    return torch.tensor([int(round(x / (2.0 * math.pi) * 2.0 ** 64)) % (1 << 63) for x in inv], dtype=torch.int64, device="cuda")


def _parents(rng, batch, nodes, reach=8):
    """Random trees, node 0 the root: a node hangs on one of the `reach` before it."""
    i = np.arange(nodes)
    back = np.floor(rng.rand(batch, nodes) * np.minimum(i, reach)).astype(np.int64)
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


def _lengths(c):
    """A shared case's lengths: of every sequence's context, and its nodes."""
    prefixes, ways = _ints(c["prefixes"]), c["ways"]
    lo, hi = (int(x) for x in c["own"].split("-"))
    batch = len(prefixes) * ways
    lens = [prefixes[b // ways] + lo + (hi - lo) * (7 * b % batch) // max(1, batch - 1) for b in range(batch)]
    counts = [max(1, c["nodes"] - (3 * b % max(1, c["nodes"] // 2 + 1) if c["ragged"] else 0)) for b in range(batch)]
    return lens, counts


def _pool(c, r, rows, refs_of):
    """Pools and tables: sequence b holds the pages that rows[b] numbers, in arbitrary order in the pool."""
    pages = 1 + max(max(x, default=0) for x in rows) + 3
    shape = (c.get("layers", 1), pages, c["hkv"], c["page"], c["hd"])
    order = r.host("pages").permutation(pages).astype(np.int32)
    table = np.full((len(rows), max(len(x) for x in rows) + 2), -1, np.int32)
    refs = np.zeros(pages, np.int32)
    for b, x in enumerate(rows):
        table[b, :len(x)] = order[x]
    refs[order[:len(refs_of)]] = refs_of
    free = np.zeros(pages, np.int32)
    free[:pages - len(refs_of)] = order[len(refs_of):]
    return {"k": r.normal("k", shape, _dtype(c)), "v": r.normal("v", shape, _dtype(c)), "table": _i32(table), "refs": _i32(refs),
            "held": _i32([len(x) for x in rows]), "free": _i32(free), "n_free": _i32([pages - len(refs_of)])}


def _handle(c, s, nodes):
    """The framework's cache around those pools and tables, as a server keeps it."""
    s["cache"] = s["lib"].PagedCache(k=s["k"], v=s["v"], table=s["table"], lens=s["lens"], held=s["held"], refs=s["refs"], free=s["free"],
                                     n_free=s["n_free"], n_q_heads=c["hq"], max_nodes=nodes)


def prepare(case, seed):
    s = _PREPARE[case["kind"]](case, _Rand(seed))
    s["kind"] = case["kind"]
    if own:
        import paper_2606_02091_gb300 as lib
        s["lib"] = lib
        if "table" in s:
            _handle(case, s, min(case["nodes"], 1024))
            if s["kind"] == "shared":       # the division of the work and partial results
                s["work"] = s["cache"].shared_work(s["q"].shape[1], s["q"].shape[2])
        elif s["kind"] == "norm":
            s["work"] = lib.qk_norm_rope_work(case["hd"])
    return s


def _prepare_norm(c, r):
    hq, hkv, hd, t = c["hq"], c["hkv"], c["hd"], _dtype(c)
    s = {"mode": c["mode"], "layout": c["layout"], "phase": _phase(_frequencies(c)),
         "q_gain": 1.0 + 0.1 * r.normal("q_gain", (hd,), torch.float32), "k_gain": 1.0 + 0.1 * r.normal("k_gain", (hd,), torch.float32)}
    s["q_gain"], s["k_gain"] = s["q_gain"].to(t), s["k_gain"].to(t)
    if c["mode"] == "pages":
        lens, n, page = _ints(c["lens"]), c["nodes"], c["page"]
        batch = len(lens)
        need = [_up(a + n, page) for a in lens]
        first = np.cumsum([0] + need)
        pool = _pool(c, r, [list(range(first[b], first[b + 1])) for b in range(batch)], [1] * int(first[-1]))
        qkv = r.normal("qkv", (batch, n, hq + 2 * hkv, hd), t, 1.3)
        parents = _parents(r.host("tree"), batch, n)
        depth = np.zeros((batch, n), np.int64)
        for i in range(1, n):
            depth[:, i] = depth[np.arange(batch), parents[:, i]] + 1
        return dict(s, **pool, lens=_i32(lens), counts=_i32([n] * batch), depth=_i32(depth), q=qkv[:, :, :hq], kn=qkv[:, :, hq:hq + hkv],
                    vn=qkv[:, :, hq + hkv:], q_out=torch.zeros((batch, n, hq, hd), dtype=t, device="cuda"))
    rows = c["rows"]
    qkv = r.normal("x", (rows, hq + 2 * hkv, hd), t, 1.3)
    s.update(q=qkv[:, :hq], kn=qkv[:, hq:hq + hkv], positions=_i32(c["start"] + np.arange(rows) % max(1, rows // 4 + 1)),
             q_out=torch.zeros((rows, hq, hd), dtype=t, device="cuda"), k_out=torch.zeros((rows, hkv, hd), dtype=t, device="cuda"))
    if c["mode"] == "train":
        s.update(dq_out=r.normal("dq", (rows, hq, hd), t), dk_out=r.normal("dk", (rows, hkv, hd), t),
                 dq=torch.zeros((rows, hq, hd), dtype=t, device="cuda"), dk=torch.zeros((rows, hkv, hd), dtype=t, device="cuda"),
                 dq_gain=torch.zeros(hd, device="cuda"), dk_gain=torch.zeros(hd, device="cuda"))
    return s


def _prepare_shared(c, r):
    prefixes, ways, page, n, t = _ints(c["prefixes"]), c["ways"], c["page"], c["nodes"], _dtype(c)
    lens, counts = _lengths(c)
    batch = len(lens)
    rows, refs = [], []
    for b in range(batch):
        if b % ways == 0:       # the prompt's whole pages, which all of its samples hold
            whole = prefixes[b // ways] // page
            lead = list(range(len(refs), len(refs) + whole))
            refs += [ways] * whole
        more = _up(lens[b] + counts[b], page) - len(lead)
        rows.append(lead + list(range(len(refs), len(refs) + more)))
        refs += [1] * more
    s = _pool(c, r, rows, refs)
    # what the plain form goes by: tokens that each group shares, and the most that a sequence has beside them
    common = [p // page * page for p in prefixes]
    s.update(lens=_i32(lens), counts=_i32(counts), q=r.normal("q", (c["layers"], batch, n, c["hq"], c["hd"]), t, 1.5), ways=ways, common=_i32(common),
             longest=max(common), widest=max(lens[b] + counts[b] - common[b // ways] for b in range(batch)),
             out=torch.zeros((c["layers"], batch, n, c["hq"], c["hd"]), dtype=t, device="cuda"))
    s["mask"] = None if c["chain"] else _i32(_words(_ancestors(_parents(r.host("tree"), batch, n))))
    return s


def _tree_of(c, h):
    """Parents and counts of a sample case's trees: nodes hang on one of the `ways` open places of the last few nodes."""
    batch, n = c["batch"], c["nodes"]
    parents = np.full((batch, n), -1, np.int32)
    i = np.arange(n)
    if c["ways"] == 1:
        parents[:, 1:] = i[1:] - 1
    else:               # level order: node i's parent is node (i - 1) / w, with a width w of its own for every tree
        w = h.randint(2, c["ways"] + 1, (batch, 1))
        parents[:, 1:] = (i[None, 1:] - 1) // w
    counts = h.randint(max(1, n // 2), n + 1, batch) if c["ragged"] else np.full(batch, n)
    return parents, counts


def _prepare_sample(c, r):
    batch, n, vocab, ways = c["batch"], c["nodes"], c["vocab"], c["ways"]
    h = r.host("tree")
    parents, counts = _tree_of(c, h)
    # a drafter's distributions and a target that agrees with them for the most part
    z = r.normal("draft", (batch, n, vocab), torch.float32, 5.0)
    target = torch.softmax(z + r.normal("target", (batch, n, vocab), torch.float32, 0.7), -1)
    draft = z.softmax(-1)[:, :max(1, n - 1)]
    del z
    rank = np.zeros((batch, n), np.int64)       # of a node among its siblings
    for i in range(1, n):
        rank[:, i] = (parents[:, :i] == parents[:, i:i + 1]).sum(1)
    flat = draft.reshape(-1, vocab)
    if c["mode"] == "picked":
        drafted = flat.topk(ways).indices
    elif c["mode"] == "distinct" and ways > 1:
        gumbel = torch.empty_like(flat).exponential_(generator=r.gpu("gumbel"))
        drafted = (flat / gumbel).topk(ways).indices
        del gumbel
    else:
        drafted = torch.multinomial(flat, ways, replacement=True, generator=r.gpu("draws"))
    up, at = torch.from_numpy(np.maximum(parents, 0)).cuda().long(), torch.from_numpy(rank).cuda()
    drafted = drafted.view(batch, draft.shape[1], ways)
    tokens = drafted[torch.arange(batch, device="cuda")[:, None], up.clamp(max=draft.shape[1] - 1), at].int()
    s = {"mode": c["mode"], "tokens": tokens, "parents": _i32(parents), "counts": _i32(counts), "target": target,
         "draft": None if c["mode"] == "picked" else draft, "u": torch.rand((batch, n), device="cuda", generator=r.gpu("u")),
         "ways": ways,
         "accept": _i32(np.zeros(batch)), "path": _i32(np.zeros((batch, n))), "next": _i32(np.zeros(batch))}
    return s


_PREPARE = {"norm": _prepare_norm, "shared": _prepare_shared, "sample": _prepare_sample}


# ---------------------------------------------------------------------------------------- one pass

def run(state):
    return _OWN[state["kind"]](state) if own else _PLAIN[state["kind"]](state)


def _own_norm(s):
    if s["mode"] == "pages":
        s["cache"].append(0, s["q"], s["kn"], s["vn"], s["counts"], s["phase"], s["q_out"], depth=s["depth"], layout=s["layout"],
                          q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS)
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    s["lib"].qk_norm_rope(s["q"], s["kn"], s["positions"], s["phase"], s["q_gain"], s["k_gain"], s["q_out"], s["k_out"], eps=EPS,
                          layout=s["layout"])
    if s["mode"] == "forward":
        return {"q": s["q_out"], "k": s["k_out"]}
    s["lib"].qk_norm_rope_backward(s["q"], s["kn"], s["dq_out"], s["dk_out"], s["positions"], s["phase"], s["q_gain"], s["k_gain"], s["dq"],
                                   s["dk"], s["dq_gain"], s["dk_gain"], s["work"], eps=EPS, layout=s["layout"])
    return {"q": s["q_out"], "k": s["k_out"], "dq": s["dq"], "dk": s["dk"], "dq_gain": s["dq_gain"], "dk_gain": s["dk_gain"]}


def _own_shared(s):
    layers, _, n = s["q"].shape[:3]
    s["cache"].share_plan(s["counts"], n, s["work"])        # once for all layers of a step
    for layer in range(layers):
        s["cache"].attend_shared(layer, s["q"][layer], s["out"][layer], s["work"], mask=s["mask"])
    return s["out"]


def _own_sample(s):
    s["lib"].tree_sample(s["tokens"], s["parents"], s["counts"], s["target"], s["draft"], s["u"], s["accept"], s["path"], s["next"],
                         distinct=s["mode"] == "distinct")
    return {"accept": s["accept"], "path": s["path"], "next": s["next"]}


_OWN = {"norm": _own_norm, "shared": _own_shared, "sample": _own_sample}


# The plain forms: elementary torch operations, arithmetic in 32 bits (64 where decisions hang on it), rounded once.

def _turned(y, positions, phase, layout, sign=1.0):
    """y [rows][heads][hd] fp32, positions [rows]."""
    turns = ((positions.long()[:, None] * phase).double() * 2.0 ** -64).float()
    cos, sin = torch.cos(turns * (2.0 * math.pi))[:, None], torch.sin(turns * (2.0 * math.pi))[:, None] * sign
    half = phase.numel()
    if layout == "half":
        a, b = y[..., :half], y[..., half:2 * half]
        z = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        z = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([z, y[..., 2 * half:]], -1)


def _normed(x, gain):
    x = x.float()
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()


def _gradient(x, dy, gain, s):
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    dz = _turned(dy.float(), s["positions"], s["phase"], s["layout"], -1.0)
    a = dz * gain.float()
    dx = r * (a - x * r.square() * (a * x).mean(-1, keepdim=True))
    return dx.to(dy.dtype), (dz * x * r).sum((0, 1))


def _plain_norm(s):
    q, k, t = s["q"], s["kn"], s["q"].dtype
    if s["mode"] == "pages":
        batch, n, hq, hd = q.shape
        page = s["k"].shape[3]
        i = torch.arange(n, device="cuda")
        at = (s["lens"][:, None] + s["depth"]).flatten()
        slot = (s["lens"][:, None] + i).long()
        ids = s["table"].long().gather(1, slot // page)
        turn = lambda x, gain: _turned(_normed(x.flatten(0, 1), gain), at, s["phase"], s["layout"]).to(t).view(x.shape)  # noqa: E731
        s["q_out"].copy_(turn(q, s["q_gain"]))
        s["k"][0, ids, :, slot % page] = turn(k, s["k_gain"])
        s["v"][0, ids, :, slot % page] = s["vn"]
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    got = {"q": _turned(_normed(q, s["q_gain"]), s["positions"], s["phase"], s["layout"]).to(t),
           "k": _turned(_normed(k, s["k_gain"]), s["positions"], s["phase"], s["layout"]).to(t)}
    if s["mode"] == "train":
        got["dq"], got["dq_gain"] = _gradient(q, s["dq_out"], s["q_gain"], s)
        got["dk"], got["dk_gain"] = _gradient(k, s["dk_out"], s["k_gain"], s)
    return got


def _plain_shared(s):
    layers, batch, n, hq, hd = s["q"].shape
    hkv, page, ways = s["k"].shape[2], s["k"].shape[3], s["ways"]
    groups, g, long, wide = batch // ways, hq // hkv, s["longest"], s["widest"]
    table, common = s["table"].long().clamp(min=0), s["common"].long()
    rows = torch.arange(batch, device="cuda")[:, None]
    lead = torch.arange(long, device="cuda")
    mine = common.repeat_interleave(ways)[:, None] + torch.arange(wide, device="cuda")      # positions beside the shared ones
    t = mine - s["lens"].long()[:, None]                                                    # tree numbers, negative in the context
    i = torch.arange(n, device="cuda")
    there = t < s["counts"][:, None]
    if s["mask"] is None:
        seen = t[:, None, :] <= i[:, None]
    else:
        at = t.clamp(0, n - 1)
        words = s["mask"].gather(2, (at // 32)[:, None, :].expand(batch, n, wide))
        seen = ((words >> (at % 32)[:, None, :]) & 1).bool() | (t < 0)[:, None, :]
    valid = (i < s["counts"][:, None])[:, :, None]
    seen = (seen & there[:, None, :] & valid)[:, None, :, None, :]                          # [batch][1][n][1][wide]
    seen_lead = ((lead < common.repeat_interleave(ways)[:, None])[:, None, :] & valid)[:, None, :, None, :]
    mine = mine.clamp(max=table.shape[1] * page - 1)
    outs = []
    for layer in range(layers):
        x = s["q"][layer].float().view(batch, n, hkv, g, hd).transpose(1, 2)                # [batch][hkv][n][g][hd]
        y = x.reshape(groups, ways, hkv, n * g, hd).transpose(1, 2).reshape(groups, hkv, ways * n * g, hd)
        k1, v1 = (p[layer][table[::ways][:, lead // page], :, lead % page].float().transpose(1, 2) for p in (s["k"], s["v"]))
        k2, v2 = (p[layer][table[rows, mine // page], :, mine % page].float().transpose(1, 2) for p in (s["k"], s["v"]))
        split = lambda z: z.view(groups, hkv, ways, n, g, -1).transpose(1, 2).reshape(batch, hkv, n, g, -1)  # noqa: E731
        a = torch.where(seen_lead, split(y @ k1.transpose(2, 3)) * hd ** -0.5, -math.inf)
        b = (x.reshape(batch, hkv, n * g, hd) @ k2.transpose(2, 3)).view(batch, hkv, n, g, wide)
        b = torch.where(seen, b * hd ** -0.5, -math.inf)
        top = torch.maximum(a.amax(-1, keepdim=True) if long else torch.full_like(b[..., :1], -math.inf), b.amax(-1, keepdim=True))
        top = torch.where(top == -math.inf, 0.0, top)
        a, b = torch.exp(a - top), torch.exp(b - top)
        total = a.sum(-1, keepdim=True) + b.sum(-1, keepdim=True)
        a = a.view(groups, ways, hkv, n * g, long).transpose(1, 2).reshape(groups, hkv, ways * n * g, long)
        o = split(a @ v1) + (b.view(batch, hkv, n * g, wide) @ v2).view(batch, hkv, n, g, hd)
        o = o / torch.where(total == 0, 1.0, total)
        outs.append(o.transpose(1, 2).reshape(batch, n, hq, hd).to(s["q"].dtype))
    return torch.stack(outs)


def _plain_sample(s):
    """All nodes of all trees at once, one rank of children after another; then the nodes whose ancestors were all kept."""
    parents, target, draft, ways = s["parents"].long(), s["target"], s["draft"], s["ways"]
    batch, n, vocab = target.shape
    b, i = torch.arange(batch, device="cuda")[:, None], torch.arange(n, device="cuda")
    there = (i < s["counts"][:, None]) & (i > 0)
    up = torch.where(there, parents, -1)
    rank = torch.tril(up[:, :, None] == up[:, None, :], -1).sum(2)
    child = torch.full((batch, n * ways + 1), n, device="cuda")     # [node][rank]: the child's number, n for none
    child.scatter_(1, torch.where(there, up * ways + rank, n * ways), i.expand(batch, n))
    child = child[:, :-1].view(batch, n, ways)
    x = torch.cat([s["tokens"].long(), torch.zeros_like(up[:, :1])], 1).gather(1, child.flatten(1)).view(child.shape)
    u = torch.cat([s["u"], s["u"][:, :1]], 1).gather(1, child.flatten(1)).view(child.shape).double()
    p = target.gather(2, x).double()
    shift, mass, left = p.new_zeros((batch, n)), p.new_ones((batch, n)), p.new_ones((batch, n))     # F, W, Q
    kept = torch.full((batch, n), n, device="cuda")                 # the child that is kept
    if draft is not None:
        draft = torch.cat([draft, draft[:, :1]], 1)[:, :n] if draft.shape[1] < n else draft
        q = draft.gather(2, x).double()
    for r in range(ways):
        turn = (child[:, :, r] < n) & (kept == n)
        if draft is None:
            before = (x[:, :, :r] == x[:, :, r:r + 1]).any(2)
            w = torch.where(before, 0.0, p[:, :, r])
            keep = turn & (u[:, :, r] * mass < w)
            mass = torch.where(turn & ~keep, mass - w, mass)
        else:
            share = torch.where(left > 0, q[:, :, r] / left, 0.0)
            keep = turn & (u[:, :, r] * share * mass < (p[:, :, r] - shift * q[:, :, r]).clamp(min=0))
            drop = turn & ~keep
            shift = torch.where(drop, shift + torch.where(left > 0, mass / left, 0.0), shift)
            if s["mode"] == "distinct":
                left = torch.where(drop, left - q[:, :, r], left)
            if r + 1 < ways:
                mass = torch.where(drop, (target.double() - shift[:, :, None] * draft).clamp(min=0).sum(2), mass)
        kept = torch.where(keep, child[:, :, r], kept)
    # a node and its parent, squared until every ancestor is reached
    above = (up[:, :, None] == i).float() + torch.eye(n, device="cuda")
    for _ in range((n - 1).bit_length()):
        above = (above @ above).clamp(max=1.0)
    chosen = (there & (kept.gather(1, up.clamp(min=0)) == i)) | (i == 0)
    on = (above @ (~chosen).float()[:, :, None])[:, :, 0] == 0
    end = torch.where(on, i, 0).amax(1, keepdim=True)
    row = target[b, end][:, 0].double()
    if draft is None:
        gone = torch.zeros((batch, vocab + 1), dtype=torch.bool, device="cuda")
        gone.scatter_(1, torch.where(child[b, end][:, 0] < n, x[b, end][:, 0], vocab), True)
        w = torch.where(gone[:, :vocab], 0.0, row)
    else:
        w = (row - shift[b, end] * draft[b, end][:, 0]).clamp(min=0)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, row)
    upto = w.cumsum(1)
    following = (upto <= s["u"][:, :1].double() * upto[:, -1:]).sum(1)
    path = torch.full((batch, n + 1), -1, dtype=torch.int32, device="cuda")
    path.scatter_(1, torch.where(on, on.long().cumsum(1) - 1, n), torch.where(on, i, -1).int())
    return {"accept": on.sum(1).int(), "path": path[:, :n].contiguous(), "next": following.int()}


_PLAIN = {"norm": _plain_norm, "shared": _plain_shared, "sample": _plain_sample}


# ------------------------------------------------------------------------------------------- work

def work(case):
    c = case
    if c["kind"] == "sample":
        # of each sequence the rows at which its walk ends, read once; the trees, their numbers and the answer
        rows = 1 if c["mode"] == "picked" else 2
        return {"bytes": c["batch"] * (rows * 4 * c["vocab"] + c["nodes"] * (4 * 4 + 2 * 4) + 12), "flops": 3 * c["batch"] * c["vocab"]}
    e = 4 if c["dtype"] == "f32" else 2
    hq, hkv, hd = c["hq"], c["hkv"], c["hd"]
    if c["kind"] == "norm":
        if c["mode"] == "pages":
            n = len(_ints(c["lens"])) * c["nodes"]
            return {"bytes": 2 * n * (hq + 2 * hkv) * hd * e + 8 * n, "flops": n * (hq + hkv) * (4 * hd + 3 * c["rot"])}
        n = c["rows"] * (hq + hkv)
        passes = 2 if c["mode"] == "forward" else 2 + 3        # backward: x, dy and dx
        return {"bytes": passes * n * hd * e + 4 * c["rows"], "flops": n * (4 * hd + 3 * c["rot"]) * (1 if c["mode"] == "forward" else 4)}
    lens, counts = _lengths(c)
    ways, page = c["ways"], c["page"]
    common = [p // page * page for p in _ints(c["prefixes"])]
    keys = sum(common) + sum(a + b - common[i // ways] for i, (a, b) in enumerate(zip(lens, counts)))
    pairs = sum(b * (a + 1) for a, b in zip(lens, counts)) * hq
    return {"bytes": c["layers"] * (keys * 2 * hkv * hd * e + sum(counts) * hq * 2 * hd * e), "flops": c["layers"] * 4 * pairs * hd}


# ------------------------------------------------------------------------------------------ exact

def _whirl(y, angle, layout, sign):
    """y [rows][heads][hd] in 64 bits, pairs as complex numbers times e^(i sign angle)."""
    r = 2 * angle.shape[1]
    z = torch.polar(torch.ones_like(angle), sign * angle)[:, None]
    y = y.clone()
    if layout == "half":
        t = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * z
        y[..., :r // 2], y[..., r // 2:r] = t.real, t.imag
    else:
        t = torch.view_as_complex(y[..., :r].reshape(y.shape[0], y.shape[1], r // 2, 2).contiguous()) * z
        y[..., :r] = torch.view_as_real(t).reshape(y.shape[0], y.shape[1], r)
    return y


def _exact_norm(c, s):
    inv = torch.tensor(_frequencies(c), dtype=torch.float64, device="cuda")

    def forward(x, gain, angle):
        x = x.double()
        return _whirl(gain.double() * x / (x.pow(2).sum(-1, keepdim=True) / c["hd"] + EPS).sqrt(), angle, c["layout"], 1.0)

    def backward(x, dy, gain, angle):
        # from the Jacobian of x / |x|_rms: (1 - n n^T) / rms with n = x / (sqrt(hd) rms)
        x, dz = x.double(), _whirl(dy.double(), angle, c["layout"], -1.0)
        rms = (x.pow(2).sum(-1, keepdim=True) / c["hd"] + EPS).sqrt()
        n, a = x / rms, dz * gain.double()
        return (a - n * (a * n).sum(-1, keepdim=True) / c["hd"]) / rms, (dz * n).flatten(0, 1).sum(0)

    if c["mode"] != "pages":
        angle = s["positions"].double()[:, None] * inv
        got = {"q": forward(s["q"], s["q_gain"], angle), "k": forward(s["kn"], s["k_gain"], angle)}
        if c["mode"] == "train":
            got["dq"], got["dq_gain"] = backward(s["q"], s["dq_out"], s["q_gain"], angle)
            got["dk"], got["dk_gain"] = backward(s["kn"], s["dk_out"], s["k_gain"], angle)
        return got
    page, table = c["page"], s["table"].long()
    q, k, v = s["q_out"].double(), s["k"].double(), s["v"].double()
    for b, m in enumerate(_ints(c["lens"])):
        angle = (m + s["depth"][b]).double()[:, None] * inv
        q[b] = forward(s["q"][b], s["q_gain"], angle)
        at = torch.arange(m, m + c["nodes"], device="cuda")
        k[0, table[b, at // page], :, at % page] = forward(s["kn"][b], s["k_gain"], angle)
        v[0, table[b, at // page], :, at % page] = s["vn"][b].double()
    return {"q": q, "k": k, "v": v}


def _exact_shared(c, s, seed):
    """Every sequence by itself over all of its own keys: what is shared makes no difference to a row."""
    lens, counts = _lengths(c)
    if sum(a * b for a, b in zip(lens, counts)) * c["hq"] * c["hd"] * 4.0 * c["layers"] > 6e12:
        return None     # too long in 64 bits
    page, hkv, hd, g = c["page"], c["hkv"], c["hd"], c["hq"] // c["hkv"]
    table, out = s["table"].long(), torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    above = None if c["chain"] else _ancestors(_parents(_Rand(seed).host("tree"), len(lens), c["nodes"]))
    for b, n in enumerate(counts):
        total = lens[b] + n
        at = torch.arange(total, device="cuda")
        seen = torch.ones((n, total), dtype=torch.bool, device="cuda")
        seen[:, lens[b]:] = torch.tril(torch.ones((n, n), dtype=torch.bool, device="cuda")) if c["chain"] else \
            torch.from_numpy(above[b, :n, :n].copy()).cuda()
        for layer in range(c["layers"]):
            key, value = (p[layer][table[b, at // page], :, at % page].double().permute(1, 2, 0) for p in (s["k"], s["v"]))
            q = s["q"][layer, b, :n].double().view(n, hkv, g, hd).permute(1, 2, 0, 3).reshape(hkv, g * n, hd)
            z = (q @ key).view(hkv, g, n, total).div(math.sqrt(hd)).masked_fill(~seen, -math.inf).softmax(-1)
            o = z.view(hkv, g * n, total) @ value.transpose(1, 2)
            out[layer, b, :n] = o.view(hkv, g, n, hd).permute(2, 0, 1, 3).reshape(n, c["hq"], hd)
    return out


def _exact_sample(c, s):
    """The walk, one sequence after another, on the host: the residual is subtracted step by step, as its definition says."""
    batch, n = c["batch"], c["nodes"]
    tokens, parents, counts, u = (s[x].cpu().numpy() for x in ("tokens", "parents", "counts", "u"))
    u = u.astype(np.float64)
    accept, path, following = np.zeros(batch, np.int32), np.full((batch, n), -1, np.int32), np.zeros(batch, np.int32)
    for b in range(batch):
        at, walk = 0, [0]
        while True:
            p = s["target"][b, at].cpu().numpy().astype(np.float64)
            children = [i for i in range(at + 1, counts[b]) if parents[b, i] == at]
            q = s["draft"][b, at].cpu().numpy().astype(np.float64) if s["draft"] is not None and children else None
            w, mass, left, found = p.copy(), 1.0, 1.0, -1
            for i in children:
                x = tokens[b, i]
                if q is None:
                    if u[b, i] * mass < w[x]:
                        found = i
                        break
                    mass -= w[x]
                    w[x] = 0.0
                    continue
                if u[b, i] * mass * (q[x] / left if left > 0 else 0.0) < w[x]:
                    found = i
                    break
                if left > 0:
                    w = np.maximum(w - mass * (q / left), 0.0)
                mass = w.sum()
                if c["mode"] == "distinct":
                    left -= q[x]
            if found < 0:
                break
            at = found
            walk.append(at)
        if not w.sum() > 0:
            w = p
        upto = np.cumsum(w)
        accept[b], following[b] = len(walk), np.searchsorted(upto, u[b, 0] * upto[-1], side="right")
        path[b, :len(walk)] = walk
    return {"accept": torch.from_numpy(accept), "path": torch.from_numpy(path), "next": torch.from_numpy(following)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(case, s)
    if case["kind"] == "shared":
        return _exact_shared(case, s, seed)
    return _exact_sample(case, s)
