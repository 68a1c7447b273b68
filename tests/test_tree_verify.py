"""Verification of drafted trees over a paged cache: rotary positions, the pages, the tree's attention, ancestor
bits and acceptance, each against a plain implementation in 64 bits (or of whole numbers), and their refusals."""
import ctypes
import math
import types

import numpy as np
import pytest
import torch

import paper_2606_02091_gb300 as P
from paper_2606_02091_gb300 import _lib

EPS32 = 2.0 ** -24      # half a unit in the last place of 1.0 in fp32
EPS16 = 2.0 ** -8       # the same in bf16 (eight significant bits)


def i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int32)).cuda()


def up(a, b):
    return -(-a // b)


# ------------------------------------------------------------------------------------------ plain forms

def frequencies(rot, theta, scaling="none", factor=1.0, trained=4096, fast=32.0, slow=1.0):
    if scaling == "ntk":
        theta = theta * factor ** (rot / (rot - 2.0))
    inv = theta ** (-2.0 * np.arange(rot // 2) / rot)
    if scaling == "linear":
        inv = inv / factor
    if scaling == "yarn":
        at = [rot * math.log(trained / (t * 2 * math.pi)) / (2 * math.log(theta)) for t in (fast, slow)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot // 2 - 1)
        mix = np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 1e-3), 0, 1)
        inv = inv * (1 - mix) + inv / factor * mix
    return inv, 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0


def turn(x, pos, inv, layout, magnitude=1.0, sign=1.0):
    """float64 [rows][heads][hd] at positions [rows]."""
    a = np.asarray(pos, np.float64)[:, None] * inv
    c, s = magnitude * np.cos(a)[:, None], magnitude * sign * np.sin(a)[:, None]
    r, y = 2 * len(inv), x.copy()
    i, j = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


def ancestors(parents):
    n = len(parents)
    a = np.zeros((n, n), bool)
    for i in range(n):
        a[i, i] = True
        if parents[i] >= 0:
            a[i] |= a[parents[i]]
    return a


def words(a):
    """[..., n] truth values as int32 words, lowest bit first."""
    n = a.shape[-1]
    w = np.zeros(a.shape[:-1] + (up(n, 32) * 32,), np.uint64)
    w[..., :n] = a
    return (w.reshape(a.shape[:-1] + (-1, 32)) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)


def random_parents(rng, n, reach=6):
    return np.array([-1] + [int(rng.integers(max(0, i - reach), i)) for i in range(1, n)], np.int32)


def host(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------ a cache to test on

class Paged:
    """A cache whose sequences hold `lens[b]` tokens and room for `counts[b]` more on pages in random order;
    every slot that holds no token, and every free page, is NaN."""

    def __init__(self, rng, lens, counts, *, hq, hkv, hd, page, dtype, layers=1, nodes=None, spare=3, scale=1.0):
        self.t = torch.float32 if dtype == "f32" else torch.bfloat16
        self.lens, self.counts, self.page, self.hq, self.hkv, self.hd = list(lens), list(counts), page, hq, hkv, hd
        held = [up(a + b, page) for a, b in zip(lens, counts)]
        pages = sum(held) + spare
        order = rng.permutation(pages)
        table = np.full((len(lens), max(held + [1]) + 2), -1, np.int32)
        refs = np.zeros(pages, np.int32)
        k = np.full((layers, pages, hkv, page, hd), np.nan, np.float32)
        v = k.copy()
        at = 0
        for b in range(len(lens)):
            ids = order[at:at + held[b]]
            at += held[b]
            table[b, :held[b]] = ids
            refs[ids] = 1
            for s in range(lens[b] + counts[b]):
                k[:, ids[s // page], :, s % page] = scale * rng.standard_normal((layers, hkv, hd))
                v[:, ids[s // page], :, s % page] = rng.standard_normal((layers, hkv, hd))
        free = np.zeros(pages, np.int32)
        free[:spare] = order[at:]
        self.k, self.v = (torch.from_numpy(x).to(self.t).cuda() for x in (k, v))
        self.table = table
        self.cache = P.PagedCache(k=self.k, v=self.v, table=i32(table), lens=i32(lens), held=i32(held), refs=i32(refs), free=i32(free),
                                  n_free=i32([spare]), n_q_heads=hq, max_nodes=nodes or max(counts + [1]))

    def rows(self, pool, b, layer=0):
        """[tokens and nodes][hkv][hd] of sequence b in 64 bits."""
        n = self.lens[b] + self.counts[b]
        s = np.arange(n)
        return host(pool[layer])[self.table[b, s // self.page], :, s % self.page].reshape(n, self.hkv, self.hd)


def attend_reference(p, q, seen, scale, layer=0):
    """out, lse and a bound on the difference of a result in fp32 arithmetic, per sequence b: seen[b] [n][keys].

    The bound: a score is a sum of hd products, off by at most (hd + 4) eps sum |q k|; that, the exponentials
    (2^-21 relative) and the sums over the keys move a weight by a relative 2 delta + (keys + 64) eps. In bf16
    each weight and the result are rounded once more."""
    batch, n = q.shape[:2]
    out, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    bound, lse_bound = np.zeros(q.shape), np.zeros(q.shape[:3])
    g = p.hq // p.hkv
    for b in range(batch):
        k, v = p.rows(p.k, b, layer), p.rows(p.v, b, layer)
        for i in range(min(n, p.counts[b])):
            see = seen[b][i]
            if not see.any():
                continue
            kk, vv, qq = k[see], v[see], q[b, i].reshape(p.hkv, g, p.hd)
            z = np.einsum("hgd,khd->hgk", qq, kk) * scale
            delta = (p.hd + 4) * EPS32 * scale * np.einsum("hgd,khd->hgk", np.abs(qq), np.abs(kk)).max(-1)
            w = np.exp(z - z.max(-1, keepdims=True))
            total = w.sum(-1, keepdims=True)
            w /= total
            o, mean = np.einsum("hgk,khd->hgd", w, vv), np.einsum("hgk,khd->hgd", w, np.abs(vv))
            rel = 2 * delta + (z.shape[-1] + 64) * EPS32
            out[b, i] = o.reshape(p.hq, p.hd)
            lse[b, i] = (z.max(-1) + np.log(total[..., 0])).reshape(p.hq)
            bound[b, i] = (rel[..., None] * mean).reshape(p.hq, p.hd)
            lse_bound[b, i] = rel.reshape(p.hq) + 4 * EPS32 * (np.abs(lse[b, i]) + np.abs(z).max(-1).reshape(p.hq))
            if p.t == torch.bfloat16:
                bound[b, i] += EPS16 * 1.01 * (mean.reshape(p.hq, p.hd) + np.abs(out[b, i]))
    return out, lse, bound, lse_bound


def run_attend(p, q, mask=None, scale=None, layer=0, counts=None):
    batch, n = q.shape[:2]
    out = torch.full((batch, n, p.hq, p.hd), 7.0, dtype=p.t, device="cuda")
    lse = torch.full((batch, n, p.hq), 7.0, dtype=torch.float32, device="cuda")
    p.cache.attend(layer, q, i32(counts if counts is not None else p.counts), out, mask=mask, scale=scale, lse=lse)
    assert p.cache.error() == 0
    return out, lse


def check_attend(p, q, seen, mask, scale=None, layer=0):
    out, lse = run_attend(p, q, mask, scale, layer)
    want, wlse, bound, lbound = attend_reference(p, host(q), seen, p.hd ** -0.5 if scale is None else scale, layer)
    assert np.all(np.abs(host(out) - want) <= bound + 1e-30)
    empty = np.isneginf(wlse)
    assert np.array_equal(np.isneginf(host(lse)), empty)
    assert np.all(np.abs(host(lse)[~empty] - wlse[~empty]) <= lbound[~empty])


def queries(rng, p, batch, n, fused=False):
    """q [batch][n][hq][hd], as a part of a wider projection's rows where `fused`."""
    wide = p.hq + (2 * p.hkv if fused else 0)
    return torch.from_numpy(rng.standard_normal((batch, n, wide, p.hd)).astype(np.float32)).to(p.t).cuda()[:, :, :p.hq]


def tree_masks(rng, lens, counts, n):
    """Bits of random trees, and which keys every node sees."""
    a = np.zeros((len(lens), n, n), bool)
    for b, c in enumerate(counts):
        if c:
            a[b, :c, :c] = ancestors(random_parents(rng, c))
    seen = [np.concatenate([np.ones((n, x), bool), a[b, :, :counts[b]]], 1) for b, x in enumerate(lens)]
    return i32(words(a)), seen


def chain_seen(lens, counts, n):
    return [np.concatenate([np.ones((n, x), bool), np.tril(np.ones((n, max(n, c)), bool))[:, :c]], 1) for x, c in zip(lens, counts)]


# ------------------------------------------------------------------------------------------ attention

ATTEND = [
    # lens, counts, hq, hkv, hd, page
    ([37], [1], 8, 2, 64, 16),                          # one token
    ([0, 5, 63, 64, 65], [1, 1, 1, 1, 1], 4, 4, 128, 16),    # empty cache; around a tile's end; no sharing of heads
    ([130, 0, 17], [7, 3, 5], 6, 2, 128, 32),           # three query heads per kv head
    ([100, 95, 200], [16, 13, 16], 8, 2, 128, 64),      # 64 rows
    ([61, 60, 59], [5, 4, 6], 5, 1, 64, 128),           # five heads on one; trees across a tile's end
    ([12, 0, 3], [0, 9, 2], 14, 2, 64, 16),             # a sequence without nodes
    ([200, 31], [33, 40], 16, 2, 128, 16),              # more than 256 rows per kv head
    ([40, 127, 128], [70, 65, 3], 4, 1, 64, 32),        # mask rows of three words
    ([1500, 700, 2], [9, 2, 9], 8, 1, 128, 64),         # keys cut into several runs
    ([5, 300], [130, 129], 2, 1, 64, 64),               # trees longer than a tile
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,counts,hq,hkv,hd,page", ATTEND)
def test_attend_matches_the_definition(lens, counts, hq, hkv, hd, page, dtype):
    rng = np.random.default_rng(sum(lens) + hq)
    p = Paged(rng, lens, counts, hq=hq, hkv=hkv, hd=hd, page=page, dtype=dtype, layers=2)
    n = max(counts)
    q = queries(rng, p, len(lens), n, fused=True)
    mask, seen = tree_masks(rng, lens, counts, n)
    check_attend(p, q, seen, mask, layer=1)
    check_attend(p, q, chain_seen(lens, counts, n), None, scale=0.2)


@pytest.mark.gpu
@pytest.mark.parametrize("nodes,hq,hkv", [(1, 8, 8), (3, 16, 4), (2, 64, 1), (20, 12, 4), (40, 8, 1), (257, 4, 2), (1024, 2, 2)])
def test_attend_for_many_shapes_of_rows(nodes, hq, hkv):
    """Row counts per kv head on both sides of every kernel's tile, up to the largest tree; n_max above the counts."""
    rng = np.random.default_rng(nodes)
    lens, counts = [70, 3], [nodes, max(1, nodes - 1)]
    p = Paged(rng, lens, counts, hq=hq, hkv=hkv, hd=64, page=16, dtype="bf16")
    q = queries(rng, p, 2, nodes)
    mask, seen = tree_masks(rng, lens, counts, nodes)
    check_attend(p, q, seen, mask)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,hq,hkv,hd,batch,top", [(1, 16, 8, 64, 40, 900), (2, 16, 4, 128, 60, 1300), (5, 32, 8, 64, 24, 1100),
                                                        (18, 32, 4, 128, 30, 1500), (34, 32, 4, 64, 20, 2500), (70, 32, 8, 128, 12, 1500)])
def test_runs_that_cross_from_pair_to_pair(nodes, hq, hkv, hd, batch, top, dtype):
    """So many sequences and heads that a CTA's share of the keys spans several of them, some of them whole; lengths
    from nothing on, some sequences without nodes. Three launches follow one another without a wait."""
    rng = np.random.default_rng(nodes)
    lens = [int(x) for x in rng.integers(0, top, batch)]
    lens[1] = 0
    counts = [int(x) for x in rng.integers(1, nodes + 1, batch)]
    counts[2] = 0
    p = Paged(rng, lens, counts, hq=hq, hkv=hkv, hd=hd, page=32, dtype=dtype, nodes=nodes)
    q = queries(rng, p, batch, nodes)
    mask, seen = tree_masks(rng, lens, counts, nodes)
    n = i32(counts)
    outs = [torch.empty_like(q) for _ in range(3)]
    for o in outs:
        p.cache.attend(0, q, n, o, mask=mask)
    check_attend(p, q, seen, mask)
    out, _ = run_attend(p, q, mask)
    assert all(torch.equal(o, out) for o in outs)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,hq,hd,batch", [(31, 32, 128, 1), (60, 32, 128, 2), (64, 64, 128, 3), (120, 64, 64, 2)])
def test_more_rows_than_the_joining_launch_holds_at_once(nodes, hq, hd, batch, dtype):
    """Few enough (sequence, kv head) pairs that CTAs share their keys, so many rows that each of the join's forms walks
    them: 992, 3840, 12288 and 15360. One sequence has fewer nodes, one no key but its own nodes'."""
    rng = np.random.default_rng(nodes)
    lens, counts = [450, 0, 301][:batch], [nodes, nodes, nodes // 3][:batch]
    p = Paged(rng, lens, counts, hq=hq, hkv=4, hd=hd, page=64, dtype=dtype)
    q = queries(rng, p, batch, nodes)
    mask, seen = tree_masks(rng, lens, counts, nodes)
    check_attend(p, q, seen, mask)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes", [4, 40])
def test_rows_that_see_nothing_are_zero(dtype, nodes):
    rng = np.random.default_rng(3)
    lens, counts = [0, 20], [nodes, nodes]
    p = Paged(rng, lens, counts, hq=8, hkv=2, hd=64, page=16, dtype=dtype)
    a = np.zeros((2, nodes, nodes), bool)
    a[0, 2, 0] = a[0, 2, 3] = True        # in sequence 0 only node 2 sees anything
    seen = [np.concatenate([np.ones((nodes, x), bool), a[b]], 1) for b, x in enumerate(lens)]
    q = queries(rng, p, 2, nodes)
    check_attend(p, q, seen, i32(words(a)))
    out, lse = run_attend(p, q, i32(words(a)))
    assert not host(out)[0, [0, 1, 3]].any() and np.isneginf(host(lse)[0, [0, 1, 3]]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,hq,hkv", [(9, 2, 2), (9, 8, 2), (16, 8, 1), (70, 8, 2)])
def test_unseen_infinities_and_nans_stay_out(dtype, nodes, hq, hkv):
    """Node 1's key and value are NaN and infinite: rows that do not see it are as if it were finite, those that
    do take the infinities' sum. The slots behind the last node are NaN already."""
    rng = np.random.default_rng(nodes + hq)
    lens, counts = [75, 64], [nodes, nodes - 2]
    p = Paged(rng, lens, counts, hq=hq, hkv=hkv, hd=64, page=16, dtype=dtype)
    q = queries(rng, p, 2, nodes)
    mask, seen = tree_masks(rng, lens, counts, nodes)
    clean, clean_lse = run_attend(p, q, mask)
    where = [(p.table[b, (x + 1) // 16], (x + 1) % 16) for b, x in enumerate(lens)]
    for page, off in where:
        p.v[0, page, :, off, 3] = math.inf
        p.v[0, page, :, off, 4] = math.nan
        p.v[0, page, :, off, 63] = -math.inf
    out, lse = run_attend(p, q, mask)
    sees = np.stack([np.pad(s[:, x + 1], (0, 0)) & (np.arange(nodes) < c) for s, x, c in zip(seen, lens, counts)])
    o, c = host(out), host(clean)
    assert np.array_equal(o[~sees], c[~sees]) and np.array_equal(host(lse), host(clean_lse))
    assert sees.any() and np.isposinf(o[sees][..., 3]).all() and np.isnan(o[sees][..., 4]).all() and np.isneginf(o[sees][..., 63]).all()
    rest = [e for e in range(64) if e not in (3, 4, 63)]
    assert np.array_equal(o[sees][..., rest], c[sees][..., rest])
    for page, off in where:                 # the key as well: scores of rows that see it are NaN
        p.k[0, page, :, off] = math.nan
    out, lse = run_attend(p, q, mask)
    assert np.array_equal(host(out)[~sees], c[~sees]) and np.array_equal(host(lse)[~sees], host(clean_lse)[~sees])
    assert np.isnan(host(out)[sees]).all() and np.isnan(host(lse)[sees]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,hq,hkv", [(3, 4, 2), (16, 8, 1), (70, 8, 2)])
def test_unseen_infinities_and_nans_stay_out_of_wide_heads(dtype, nodes, hq, hkv):
    """The same at head_dim 128, where a tile's rows lie in two parts: odd values in both, at their ends."""
    rng = np.random.default_rng(nodes)
    lens, counts = [117, 64], [nodes, nodes - 2]
    p = Paged(rng, lens, counts, hq=hq, hkv=hkv, hd=128, page=32, dtype=dtype)
    q = queries(rng, p, 2, nodes)
    mask, seen = tree_masks(rng, lens, counts, nodes)
    clean, clean_lse = run_attend(p, q, mask)
    for b, x in enumerate(lens):        # a node in the middle
        node = (counts[b] - 1) // 2
        page, off = p.table[b, (x + node) // 32], (x + node) % 32
        for e, value in ((0, math.inf), (63, math.nan), (64, -math.inf), (70, math.nan), (127, math.inf)):
            p.v[0, page, :, off, e] = value
    out, lse = run_attend(p, q, mask)
    sees = np.stack([s[:, x + (c - 1) // 2] & (np.arange(nodes) < c) for s, x, c in zip(seen, lens, counts)])
    o, c = host(out), host(clean)
    assert np.array_equal(o[~sees], c[~sees]) and np.array_equal(host(lse), host(clean_lse))
    assert sees.any() and np.isposinf(o[sees][..., [0, 127]]).all() and np.isneginf(o[sees][..., 64]).all()
    assert np.isnan(o[sees][..., [63, 70]]).all()
    rest = [e for e in range(128) if e not in (0, 63, 64, 70, 127)]
    assert np.array_equal(o[sees][..., rest], c[sees][..., rest])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,nodes,hq,hkv,hd,batch,keys", [("bf16", 9, 32, 8, 128, 12, 4000), ("bf16", 40, 64, 8, 64, 6, 1500), ("bf16", 70, 32, 8, 128, 6, 1500),
                                                              ("bf16", 3, 16, 8, 128, 20, 2600), ("f32", 5, 8, 4, 64, 12, 1500)])
def test_scores_that_go_on_growing(dtype, nodes, hq, hkv, hd, batch, keys):
    """Scores spread over tens of powers of two, in runs of several tiles: rows whose maximum is raised long after
    their first keys, when their output has to be scaled down where it is."""
    rng = np.random.default_rng(nodes)
    lens, counts = [keys - 37 * b for b in range(batch)], [nodes - b % 2 for b in range(batch)]
    p = Paged(rng, lens, counts, hq=hq, hkv=hkv, hd=hd, page=64, dtype=dtype, scale=20.0)
    q = queries(rng, p, batch, nodes)
    late = 0
    for b in range(batch):          # rows with a tile 2^8 above the four before it
        k = p.rows(p.k, b)[:lens[b] // 128 * 128]
        z = np.einsum("hgd,khd->hgk", host(q)[b, 0].reshape(hkv, hq // hkv, hd), k) * hd ** -0.5 / math.log(2)
        top = z.reshape(hq, -1, 128).max(-1)
        late += sum(any(row[t] > row[t - 4:t].max() + 8 for t in range(4, len(row))) for row in top)
    assert late > hq * batch // 10
    mask, seen = tree_masks(rng, lens, counts, nodes)
    check_attend(p, q, seen, mask)


@pytest.mark.gpu
@pytest.mark.parametrize("nodes,hq,hkv,hd,lens", [(1024, 8, 2, 128, [300, 0]), (1000, 12, 4, 64, [33]), (1024, 64, 1, 64, [70]), (600, 8, 2, 128, [2000])])
def test_chunks_of_many_query_groups(nodes, hq, hkv, hd, lens):
    """Chunks of a prompt with more than 2048 query rows per kv head, up to more groups of them than the GPU has SMs:
    chains and trees."""
    rng = np.random.default_rng(nodes + hq)
    counts = [nodes - 3 * b for b in range(len(lens))]
    p = Paged(rng, lens, counts, hq=hq, hkv=hkv, hd=hd, page=64, dtype="bf16")
    q = queries(rng, p, len(lens), nodes)
    check_attend(p, q, chain_seen(lens, counts, nodes), None)
    mask, seen = tree_masks(rng, lens, counts, nodes)
    check_attend(p, q, seen, mask)


@pytest.mark.gpu
@pytest.mark.parametrize("nodes", [1, 8, 64])
def test_attend_is_the_same_on_every_run(nodes):
    rng = np.random.default_rng(5)
    lens, counts = [3000, 17, 900], [nodes] * 3
    p = Paged(rng, lens, counts, hq=8, hkv=2, hd=128, page=64, dtype="bf16")
    q = queries(rng, p, 3, nodes)
    mask, _ = tree_masks(rng, lens, counts, nodes)
    first = run_attend(p, q, mask)
    for _ in range(3):
        again = run_attend(p, q, mask)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_the_softmax_streams_meet_between_tensor_memory_fences():
    """With up to 128 query rows a stream reads the output that the other one has waited for. The memory model orders
    that only where a barrier stands between a fence before it and one after it; no run can show one that is missing, so
    this reads the source: every barrier of the two streams is the one that has both."""
    import os
    import re
    src = open(os.path.join(os.path.dirname(P.__file__), "csrc", "tree_attention_tc.cu")).read()
    src = re.sub(r"//[^\n]*", "", src)
    barriers = [m.start() for m in re.finditer(r"bar\.(sync|arrive)", src)]
    fenced = re.search(r'tc_fence_before\(\);\s*asm volatile\("bar\.sync 1, 256;" ::: "memory"\);\s*tc_fence_after\(\);', src)
    assert len(barriers) == 1 and fenced and fenced.start() < barriers[0] < fenced.end()


@pytest.mark.gpu
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens", [[0, 1], [129, 300], [40000, 511], [70000, 70000]])
def test_the_streams_join_over_runs_of_any_length(lens, hd):
    """Up to 128 query rows per kv head: runs of one tile (a single stream), of two, and of many."""
    rng = np.random.default_rng(lens[0] + hd)
    p = Paged(rng, lens, [20, 17], hq=4, hkv=1, hd=hd, page=128, dtype="bf16")
    q = queries(rng, p, 2, 20)
    mask, seen = tree_masks(rng, lens, [20, 17], 20)
    check_attend(p, q, seen, mask)
    first, _ = run_attend(p, q, mask)
    for _ in range(20):
        assert torch.equal(run_attend(p, q, mask)[0], first)


@pytest.mark.gpu
@pytest.mark.parametrize("nodes", [2, 40])
def test_attend_reaches_past_32_bit_offsets(nodes):
    """A pool of more than 2^32 bytes per layer and 2^31 elements: the pages in use lie at its end."""
    rng = np.random.default_rng(6)
    hq, hkv, hd, page, pages = 16, 8, 128, 128, 20000
    pool = [torch.empty((1, pages, hkv, page, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = np.array([[pages - 1, 3, pages - 2, -1]], np.int32)
    n_keys = 2 * page + 40 + nodes
    for t in pool:
        for i in table[0, :3]:
            t[0, int(i)] = torch.from_numpy(rng.standard_normal((hkv, page, hd)).astype(np.float32)).cuda()
    p = object.__new__(Paged)
    p.t, p.lens, p.counts, p.page, p.hq, p.hkv, p.hd = torch.bfloat16, [n_keys - nodes], [nodes], page, hq, hkv, hd
    p.cache = P.PagedCache(k=pool[0], v=pool[1], table=i32(table), lens=i32(p.lens), held=i32([3]),
                           refs=torch.zeros(pages, dtype=torch.int32, device="cuda"),
                           free=torch.zeros(pages, dtype=torch.int32, device="cuda"), n_free=i32([0]), n_q_heads=hq, max_nodes=nodes)
    # the reference reads a small copy of the three pages
    p.k, p.v = (t[:, [pages - 1, 3, pages - 2]] for t in pool)
    p.table = np.array([[0, 1, 2]])
    q = queries(rng, p, 1, nodes)
    mask, seen = tree_masks(rng, p.lens, p.counts, nodes)
    check_attend(p, q, seen, mask)


@pytest.mark.gpu
def test_attend_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(7)
    lens, counts = [100, 65], [5, 5]
    p = Paged(rng, lens, counts, hq=8, hkv=2, hd=64, page=16, dtype="bf16")
    q = queries(rng, p, 2, 5)
    mask, _ = tree_masks(rng, lens, counts, 5)
    want, _ = run_attend(p, q, mask)
    s = torch.cuda.Stream()
    n = i32(counts)
    out = torch.zeros_like(want)
    s.wait_stream(torch.cuda.current_stream())
    p.cache.attend(0, q, n, out, mask=mask, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.cache.attend(0, q, n, out, mask=mask)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    # the graph follows the lengths on the device
    p.cache.lens.copy_(i32([40, 3]))
    p.lens = [40, 3]
    g.replay()
    torch.cuda.synchronize()
    short, _ = run_attend(p, q, mask)
    assert torch.equal(out, short) and not torch.equal(out, want)


@pytest.mark.gpu
def test_attend_stays_within_the_pages_a_sequence_holds():
    """Lengths and counts beyond the pages held, and page numbers that do not exist, read nothing."""
    rng = np.random.default_rng(8)
    for dtype in ("bf16", "f32"):
        p = Paged(rng, [40, 20], [8, 8], hq=4, hkv=2, hd=64, page=16, dtype=dtype, nodes=8)
        q = queries(rng, p, 2, 8)
        p.cache.lens.copy_(i32([40000, 20]))       # three pages hold 48 keys
        out, _ = run_attend(p, q, counts=[8, 9999])
        assert not torch.isnan(out[1]).any()
        p.cache.held.copy_(i32([0, 2]))
        out, lse = run_attend(p, q)
        assert not out[0].any() and torch.isneginf(lse[0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes", [1, 4, 30, 70])
@pytest.mark.parametrize("number", [-1, 10 ** 6])
def test_attend_reports_pages_that_do_not_exist(nodes, number, dtype):
    """A page number in the table that no page has: reported, its keys and values read as zeros, other sequences as ever."""
    rng = np.random.default_rng(nodes)
    lens = [100, 60]
    p = Paged(rng, lens, [nodes, nodes], hq=8, hkv=2, hd=64, page=16, dtype=dtype)
    q = queries(rng, p, 2, nodes)
    mask, seen = tree_masks(rng, lens, [nodes, nodes], nodes)
    check_attend(p, q, seen, mask)
    p.k[0, p.table[0, 2]] = 0
    p.v[0, p.table[0, 2]] = 0
    want, want_lse = run_attend(p, q, mask)
    p.cache.table[0, 2] = number
    out, lse = torch.empty_like(want), torch.empty_like(want_lse)
    p.cache.attend(0, q, i32([nodes, nodes]), out, mask=mask, lse=lse)
    assert p.cache.error() == P.DEVERR_PAGE
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    p.cache.table[0, 2] = int(p.table[0, 2])
    out, _ = run_attend(p, q, mask)
    assert torch.equal(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes", [8, 24, 72])
def test_attend_over_a_length_beyond_the_pages_sees_the_keys_that_exist(nodes, dtype):
    rng = np.random.default_rng(nodes)
    held = up(40 + nodes, 16)
    p = Paged(rng, [40, 20], [16 * held - 40, nodes], hq=4, hkv=2, hd=64, page=16, dtype=dtype, nodes=nodes)
    q = queries(rng, p, 2, nodes)
    p.cache.lens.copy_(i32([40000, 20]))
    mask, seen = tree_masks(rng, [16 * held, 20], [0, nodes], nodes)
    out, lse = run_attend(p, q, mask, counts=[nodes, nodes])
    want, wlse, bound, lbound = attend_reference(p, host(q), seen, 64 ** -0.5)
    assert np.all(np.abs(host(out) - want) <= bound) and np.all(np.abs(host(lse) - wlse) <= lbound)


# ------------------------------------------------------------------------------------------ rotary positions

ROPE = [
    # rows, heads, hd, rot, layout, scaling, start
    (1, 1, 64, 64, "half", "none", 0),
    (7, 5, 128, 128, "half", "linear", 100000),
    (33, 40, 128, 64, "half", "yarn", 900000),
    (9, 3, 64, 32, "interleaved", "ntk", 131071),
    (130, 8, 64, 64, "interleaved", "yarn", 5),
    (5, 3, 80, 20, "half", "none", 77),             # no multiple of 16
    (5, 3, 80, 22, "interleaved", "linear", 77),
    (4, 2, 7, 6, "half", "none", 3),                # an odd head
    (3000, 12, 128, 128, "half", "none", 2 ** 30),  # rows enough for several heads per thread
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,hd,rot,layout,scaling,start", ROPE)
def test_rope_matches_the_definition(rows, heads, hd, rot, layout, scaling, start, dtype):
    rng = np.random.default_rng(rows * hd)
    factor = 1.0 if scaling == "none" else 8.0
    inv, magnitude = frequencies(rot, 1e4, scaling, factor)
    phase, m = P.rope_phases(rot, 1e4, scaling, factor)
    assert abs(m - magnitude) <= 1e-6
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.from_numpy(rng.standard_normal((rows, heads + 2, hd)).astype(np.float32)).to(t).cuda()[:, 1:heads + 1]
    pos = np.minimum(start + rng.integers(0, 50, rows), 2 ** 31 - 1)
    pos[0] = -pos[0]
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    both = np.abs(host(x)[..., a]) + np.abs(host(x)[..., b])
    # cosine and sine of an angle that is off by 2^-24 of pi and their own roundings: 6 eps; a product and a sum: 2
    bound = np.zeros((rows, heads, hd))
    bound[..., a] = bound[..., b] = 8 * EPS32 * magnitude * both
    # the plain angle's own rounding in 64 bits
    bound[..., :rot] += magnitude * np.abs(pos).max() * 2.0 ** -51 * 4
    for backward in (False, True):
        want = turn(host(x), pos, inv, layout, magnitude, -1.0 if backward else 1.0)
        out = torch.full((rows, heads, hd), 7.0, dtype=t, device="cuda")
        P.rope(x, i32(pos), phase, out, layout=layout, magnitude=m, backward=backward)
        off = np.abs(host(out) - want)
        assert np.all(off <= bound + (EPS16 * 1.01 * np.abs(want) if dtype == "bf16" else 0))
        assert torch.equal(out[..., rot:], x[..., rot:])
        # in place, and [heads][rows] order: the same bits
        y = x.clone()
        P.rope(y, i32(pos), phase, y, layout=layout, magnitude=m, backward=backward)
        turned = torch.zeros((heads, rows, hd), dtype=t, device="cuda").transpose(0, 1)
        P.rope(x, i32(pos), phase, turned, layout=layout, magnitude=m, backward=backward)
        assert torch.equal(y, out) and torch.equal(turned, out)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_backward_is_the_gradient(layout):
    """Against differences: the map is linear, so f(x + d) - f(x - d) = 2 J d for any d."""
    rng = np.random.default_rng(11)
    rows, heads, hd, rot = 6, 3, 64, 32
    phase, m = P.rope_phases(rot, 1e4, "yarn", 4.0)
    pos = i32(rng.integers(0, 5000, rows))
    x, d, g = (torch.from_numpy(rng.standard_normal((rows, heads, hd)).astype(np.float32)).cuda() for _ in range(3))

    def f(z, backward=False):
        out = torch.empty_like(z)
        P.rope(z, pos, phase, out, layout=layout, magnitude=m, backward=backward)
        return out.double()

    difference = (f(x + d) - f(x - d)) / 2
    lhs, rhs = (difference * g.double()).sum().item(), (f(g, True) * d.double()).sum().item()
    # 2 x 1152 products of numbers of size 4, each off by 8 eps
    assert abs(lhs - rhs) <= 1152 * 2 * 8 * EPS32 * 16


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_rope_phases_are_the_frequencies(scaling):
    from paper_2606_02091_gb300 import build
    build.build()
    inv, magnitude = frequencies(64, 1e6, scaling, 1.0 if scaling == "none" else 16.0)
    phase, m = P.rope_phases(64, 1e6, scaling, 1.0 if scaling == "none" else 16.0, device="cpu")
    got = phase.numpy().astype(np.float64) / 2.0 ** 64 * 2 * math.pi
    assert np.all(np.abs(got - inv) <= 1e-14 * inv + 2.0 ** -60) and abs(m - magnitude) < 1e-6


@pytest.mark.parametrize("rot,theta,scaling,factor", [(128, 1e6, "none", 1.0), (64, 1e4, "linear", 3.0), (128, 1e4, "ntk", 16.0), (128, 5e5, "yarn", 7.0)])
def test_rope_phases_are_as_exact_as_stated(raw, rot, theta, scaling, factor):
    """Every phase within 2^-50 of itself and one unit: an angle within position x 2^-52 turns, at int32's ends 2^-21."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
    base, f = Decimal(theta), Decimal(factor)
    if scaling == "ntk":
        base *= f ** (Decimal(rot) / (rot - 2))
    exact = [base ** (Decimal(-2 * j) / rot) for j in range(rot // 2)]
    if scaling == "linear":
        exact = [x / f for x in exact]
    if scaling == "yarn":
        at = [rot * (Decimal(4096) / (t * 2 * pi)).ln() / (2 * base.ln()) for t in (32, 1)]
        lo, hi = math.floor(at[0]), math.ceil(at[1])
        mix = [min(max(Decimal(j - lo) / (hi - lo), Decimal(0)), Decimal(1)) for j in range(rot // 2)]
        exact = [x * (1 - m) + x / f * m for x, m in zip(exact, mix)]
    phase, _ = P.rope_phases(rot, theta, scaling, factor, device="cpu")
    off = [abs(Decimal(p) - x / (2 * pi) * 2 ** 64) for p, x in zip(phase.tolist(), exact)]
    assert all(o <= x / (2 * pi) * 2 ** 14 + 1 for o, x in zip(off, exact))
    assert max(off) * 2 ** 31 / 2 ** 64 <= Decimal(2) ** -21


@pytest.mark.parametrize("rot,theta,trained,factor,fast,slow", [
    (128, 1e4, 131072, 4.0, 32.0, 1.0),     # the last pair still turns twice: the mix ends beyond it
    (64, 1e4, 10 ** 7, 16.0, 32.0, 1.0),    # every pair turns 32 times: all keep their frequency
    (64, 1e4, 100, 2.0, 32.0, 1.0),         # the first pair turns 16 times: the mix begins before it
    (64, 1e6, 3, 8.0, 32.0, 1.0),           # no pair turns once: all stretch
    (4, 1e4, 4096, 4.0, 32.0, 1.0),         # two pairs, neither at an end
    (128, 1e6, 32768, 4.0, 32.0, 1.0),
    (2, 1e4, 4096, 4.0, 32.0, 1.0),
])
def test_yarn_goes_by_the_turns_of_each_pair(raw, rot, theta, trained, factor, fast, slow):
    """Frequencies from the turns that pairs make within the trained positions, pairs counted past the head's at both ends."""
    def turns(j):
        return trained * theta ** (-2.0 * j / rot) / (2 * math.pi)

    lo = next(j for j in range(4 * rot, -4 * rot, -1) if turns(j) >= fast)
    hi = next(j for j in range(-4 * rot, 4 * rot) if turns(j) <= slow)
    assert lo < hi
    phase, m = P.rope_phases(rot, theta, "yarn", factor, trained, fast, slow, device="cpu")
    got = phase.numpy().astype(np.float64) / 2.0 ** 64 * 2 * math.pi
    for j in range(rot // 2):
        inv = theta ** (-2.0 * j / rot)
        stretch = (j - lo) / (hi - lo) if lo < j < hi else float(turns(j) < fast)
        want = inv * (1 - stretch) + inv / factor * stretch
        assert abs(got[j] - want) <= 1e-13 * want + 2.0 ** -60
        if turns(j) >= fast:
            assert abs(got[j] - inv) <= 1e-13 * inv + 2.0 ** -60
        if turns(j) <= slow:
            assert abs(got[j] - inv / factor) <= 1e-13 * inv + 2.0 ** -60
    assert abs(m - (0.1 * math.log(factor) + 1.0)) < 1e-6


# ------------------------------------------------------------------------------------------ append

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot,layout,depths", [(64, "half", True), (32, "interleaved", True), (64, "interleaved", False), (20, "half", True), (0, "half", False)])
def test_append_rotates_and_writes_the_pages(rot, layout, depths, dtype):
    rng = np.random.default_rng(rot)
    lens, counts = [0, 15, 16, 40], [5, 3, 0, 9]
    p = Paged(rng, lens, counts, hq=6, hkv=2, hd=64, page=16, dtype=dtype, layers=2)
    n = 9
    qkv = torch.from_numpy(rng.standard_normal((4, n, 10, 64)).astype(np.float32)).to(p.t).cuda()
    q, k, v = qkv[:, :, :6], qkv[:, :, 6:8], qkv[:, :, 8:]
    depth = np.stack([np.arange(n) // 2 for _ in lens])
    out = torch.full((4, n, 6, 64), 7.0, dtype=p.t, device="cuda")
    k0, v0 = p.k.clone(), p.v.clone()
    phase = P.rope_phases(rot, 1e4)[0] if rot else None
    p.cache.append(1, q, k, v, i32(counts), phase, out, depth=i32(depth) if depths else None, layout=layout)
    assert p.cache.error() == 0
    inv = frequencies(rot, 1e4)[0] if rot else np.zeros(0)
    kw, vw = host(k0), host(v0)
    for b, c in enumerate(counts):
        pos = lens[b] + (depth[b, :c] if depths else np.arange(c))
        want = turn(host(q)[b, :c], pos, inv, layout)
        bound = 16 * EPS32 * np.abs(host(q)[b]).max() + (EPS16 * 1.01 * np.abs(want) if dtype == "bf16" else 0)
        assert np.all(np.abs(host(out)[b, :c] - want) <= bound)
        assert (host(out)[b, c:] == 7.0).all()
        keys = turn(host(k)[b, :c], pos, inv, layout)
        for i in range(c):
            at = p.table[b, (lens[b] + i) // 16], (lens[b] + i) % 16
            kw[1, at[0], :, at[1]], vw[1, at[0], :, at[1]] = keys[i], host(v)[b, i]
    got = host(p.k)
    assert np.array_equal(np.isnan(got), np.isnan(kw)) and np.array_equal(host(p.v), vw, equal_nan=True)
    assert np.array_equal(got[0], kw[0], equal_nan=True)
    bound = 16 * EPS32 * 5 + (EPS16 * 1.01 * np.abs(kw) if dtype == "bf16" else 0)
    assert not np.any(np.abs(got - kw) > bound)
    # queries in place, and keys and values alone
    p.cache.append(1, q, k, v, i32(counts), phase, q, depth=i32(depth) if depths else None, layout=layout)
    for b, c in enumerate(counts):
        assert torch.equal(q[b, :c], out[b, :c])
    p.cache.append(0, None, k, v, i32(counts), phase, None, depth=i32(depth) if depths else None, layout=layout)
    for b, c in enumerate(counts):
        for i in range(c):
            page, off = p.table[b, (lens[b] + i) // 16], (lens[b] + i) % 16
            assert torch.equal(p.k[0, page, :, off], p.k[1, page, :, off]) and torch.equal(p.v[0, page, :, off], p.v[1, page, :, off])


@pytest.mark.gpu
def test_a_page_that_is_still_shared_is_not_written():
    """Two sequences share a partly filled page; without a reserve neither append nor commit may touch it."""
    c = P.PagedCache.allocate(n_layers=1, n_pages=8, page_size=16, n_q_heads=1, n_kv_heads=1, head_dim=64, max_batch=2, max_pages=3, max_nodes=8)
    c.k.zero_(), c.v.zero_()
    c.reserve(i32([10, 0]))
    c.commit(i32([10, 0]), i32([np.arange(10), np.arange(10)]))
    c.fork(i32([0]), i32([1]))
    k0, table = c.k.clone(), c.table.clone()
    x = torch.ones((2, 3, 1, 64), dtype=c.dtype, device="cuda")
    c.append(0, None, x, x, i32([0, 3]), None, None)
    assert c.error() == P.DEVERR_PAGE and torch.equal(c.k, k0)
    c.commit(i32([0, 2]), i32([[0, 1, 2], [0, 2, -1]]))
    assert c.error() == P.DEVERR_TREE and torch.equal(c.k, k0) and c.lens.tolist() == [10, 10] and torch.equal(c.table, table)
    c.reserve(i32([0, 3]))          # sequence 1 gets its copy, and sequence 0 keeps the page
    c.append(0, None, x, x, i32([0, 3]), None, None)
    c.commit(i32([0, 2]), i32([[0, 1, 2], [0, 2, -1]]))
    assert c.error() == 0 and c.lens.tolist() == [10, 12] and torch.equal(c.k[0, table[0, 0]], k0[0, table[0, 0]])
    c.append(0, None, x, x, i32([3, 0]), None, None)        # its own now
    assert c.error() == 0 and (c.k[0, table[0, 0], :, 10:13] == 1).all()


@pytest.mark.gpu
def test_append_beyond_the_pages_is_left_out():
    rng = np.random.default_rng(1)
    p = Paged(rng, [30], [2], hq=2, hkv=2, hd=64, page=16, dtype="bf16")
    k0 = p.k.clone()
    k = torch.ones((1, 5, 2, 64), dtype=torch.bfloat16, device="cuda")
    p.cache.append(0, None, k, k, i32([5]), None, None)
    assert p.cache.error() == P.DEVERR_CAPACITY
    same = torch.eq(p.k, k0) | (torch.isnan(p.k) & torch.isnan(k0))
    same[0, p.table[0, 1], :, 14:16] = True
    assert same.all() and (p.k[0, p.table[0, 1], :, 14:16] == 1).all()


# ------------------------------------------------------------------------------------------ pages

class Model:
    """The page calls, one sequence at a time, on Python lists; `rows[page]` is what its slots hold."""

    def __init__(self, batch, pages, page):
        self.page, self.free, self.refs = page, list(range(pages - 1, -1, -1)), [0] * pages
        self.stack = list(self.free)
        self.table, self.lens = [[] for _ in range(batch)], [0] * batch
        self.rows = [[None] * page for _ in range(pages)]

    def _push(self, p):
        self.free.append(p)
        self.stack[len(self.free) - 1] = p

    def reserve(self, n):
        before = (list(self.free), list(self.refs), [list(t) for t in self.table], [list(r) for r in self.rows])
        try:
            for b, x in enumerate(n):
                if x <= 0:
                    continue
                if self.lens[b] % self.page:
                    i = self.lens[b] // self.page
                    old = self.table[b][i]
                    if self.refs[old] > 1:
                        new = self.free.pop()
                        self.refs[old] -= 1
                        self.refs[new], self.table[b][i] = 1, new
                        self.rows[new][:self.lens[b] % self.page] = self.rows[old][:self.lens[b] % self.page]
                while len(self.table[b]) * self.page < self.lens[b] + x:
                    new = self.free.pop()
                    self.refs[new] = 1
                    self.table[b].append(new)
            return True
        except IndexError:
            self.free, self.refs, self.table, self.rows = before
            return False

    def trim(self, b):
        keep = up(self.lens[b], self.page)
        for p in self.table[b][keep:]:
            self.refs[p] -= 1
            if self.refs[p] == 0:
                self._push(p)
        del self.table[b][keep:]

    def truncate(self, n):
        for b, x in enumerate(n):
            self.lens[b] = min(self.lens[b], max(x, 0))
            self.trim(b)

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.table[b] = self.table[a][:up(self.lens[a], self.page)]
            self.lens[b] = self.lens[a]
            for p in self.table[b]:
                self.refs[p] += 1

    def slot(self, b, s):
        return self.table[b][s // self.page], s % self.page

    def commit(self, accept, paths):
        for b, a in enumerate(accept):
            for j, x in enumerate(paths[b][:a]):
                p, o = self.slot(b, self.lens[b] + x)
                r = self.rows[p][o]
                p, o = self.slot(b, self.lens[b] + j)
                self.rows[p][o] = r
            self.lens[b] += a
        for b in range(len(accept)):
            self.trim(b)


def check_pages(c, m):
    torch.cuda.synchronize()
    assert c.lens.tolist() == m.lens and c.held.tolist() == [len(t) for t in m.table]
    table = c.table.tolist()
    for b, t in enumerate(m.table):
        assert table[b][:len(t)] == t and all(x == -1 for x in table[b][len(t):])
    n = int(c.n_free)
    assert n == len(m.free) and c.free.tolist()[:n] == m.free and c.refs.tolist() == m.refs
    k, v = c.k.float().cpu().numpy(), c.v.float().cpu().numpy()
    at = [m.slot(b, s) for b in range(len(m.lens)) for s in range(m.lens[b])]
    if at:
        page, off = np.array(at).T
        want = np.array([m.rows[p][o] for p, o in at])[:, None] + np.arange(c.n_layers)
        for pool, sign in ((k, 1), (v, -1)):
            assert (pool[:, page, :, off] == sign * want[:, :, None, None]).all()      # [slots][layers][heads][elements]


@pytest.mark.gpu
@pytest.mark.parametrize("page,dtype,seed", [(16, "f32", 0), (32, "f32", 1), (16, "bf16", 2), (128, "f32", 3)])
def test_pages_follow_the_model_through_random_calls(page, dtype, seed):
    rng = np.random.default_rng(seed)
    batch, pages, layers, nodes = 6, 40 if page < 128 else 16, 3, 24
    c = P.PagedCache.allocate(n_layers=layers, n_pages=pages, page_size=page, n_q_heads=2, n_kv_heads=2, head_dim=64, max_batch=batch,
                              max_pages=12, max_nodes=nodes, dtype=dtype)
    m = Model(batch, pages, page)
    mark, full = 0, 0
    for step in range(60):
        idle = [b for b in range(batch) if not m.table[b] and m.lens[b] == 0]
        busy = [b for b in range(batch) if m.lens[b] > 0]
        if step % 7 == 3 and idle and busy:       # fork: one source for several, or several
            dst = [int(x) for x in rng.permutation(idle)[:int(rng.integers(1, len(idle) + 1))]]
            src = [int(rng.choice(busy)) for _ in dst]
            c.fork(i32(src), i32(dst))
            m.fork(src, dst)
            assert c.error() == 0
            check_pages(c, m)
            continue
        if step % 7 == 5:
            n = [int(rng.choice([0, m.lens[b] // 2, m.lens[b], m.lens[b] - 1, 10 ** 6])) for b in range(batch)]
            c.truncate(i32(n))
            m.truncate(n)
            assert c.error() == 0
            check_pages(c, m)
            continue
        n = [int(rng.integers(0, nodes + 1)) if m.lens[b] + nodes <= 12 * page else 0 for b in range(batch)]
        c.reserve(i32(n))
        if not m.reserve(n):
            assert c.error() == P.DEVERR_CAPACITY
            full += 1
            check_pages(c, m)
            cut = [m.lens[b] // 3 for b in range(batch)]
            c.truncate(i32(cut))
            m.truncate(cut)
            check_pages(c, m)
            continue
        assert c.error() == 0
        # every new slot gets a mark of its own (numbers that bf16 holds exactly)
        new = np.zeros((batch, nodes), np.float32)
        for b in range(batch):
            for i in range(n[b]):
                mark = mark % 120 + 1
                p, o = m.slot(b, m.lens[b] + i)
                m.rows[p][o] = mark
                new[b, i] = mark
        for layer in range(layers):
            x = torch.from_numpy(new).cuda()[:, :, None, None] + layer
            x = x.expand(batch, nodes, 2, 64).to(c.dtype).contiguous()
            c.append(layer, None, x, -x, i32(n), None, None)
        paths = np.full((batch, nodes), -1, np.int64)
        accept = []
        for b in range(batch):
            a = int(rng.integers(0, n[b] + 1))
            chosen = np.sort(rng.permutation(n[b])[:a])
            if a and rng.random() < 0.7:
                chosen[0] = 0
            paths[b, :a] = chosen
            accept.append(a)
        c.commit(i32(accept), i32(paths))
        m.commit(accept, paths.tolist())
        assert c.error() == 0
        check_pages(c, m)
    assert full or page > 16


@pytest.mark.gpu
def test_pages_by_the_thousand():
    """More pages in one call than a CTA has threads: taken, given back in order, taken again."""
    c = P.PagedCache.allocate(n_layers=1, n_pages=3000, page_size=16, n_q_heads=1, n_kv_heads=1, head_dim=64, max_batch=3, max_pages=1300,
                              max_nodes=1, dtype="f32")
    m = Model(3, 3000, 16)
    for n in ([20000, 5, 17000], [0, 20800, 9000], [16, 16, 20001]):
        c.reserve(i32(n))
        assert m.reserve(n) and c.error() == 0
        check_pages(c, m)
        c.truncate(i32([0, 0, 0]))
        m.truncate([0, 0, 0])
        assert c.error() == 0
        check_pages(c, m)


@pytest.mark.gpu
def test_copy_pages():
    c = P.PagedCache.allocate(n_layers=3, n_pages=9, page_size=32, n_q_heads=3, n_kv_heads=3, head_dim=64, max_batch=1, max_pages=4, max_nodes=4)
    c.k.normal_()
    c.v.normal_()
    k, v = c.k.clone(), c.v.clone()
    c.copy_pages(i32([0, 4, 0, 8]), i32([7, 1, 2, 3]))
    k[:, [7, 1, 2, 3]], v[:, [7, 1, 2, 3]] = k[:, [0, 4, 0, 8]], v[:, [0, 4, 0, 8]]
    assert torch.equal(c.k, k) and torch.equal(c.v, v) and c.error() == 0
    c.copy_pages(i32([0, 9, -1]), i32([5, 6, 4]))
    k[:, 5], v[:, 5] = k[:, 0], v[:, 0]
    assert torch.equal(c.k, k) and torch.equal(c.v, v) and c.error() == P.DEVERR_PAGE


@pytest.mark.gpu
def test_page_calls_report_what_cannot_be():
    c = P.PagedCache.allocate(n_layers=1, n_pages=8, page_size=16, n_q_heads=1, n_kv_heads=1, head_dim=64, max_batch=4, max_pages=3, max_nodes=8)
    m = Model(4, 8, 16)
    n = [20, 0, 0, 0]
    c.reserve(i32(n)), m.reserve(n)
    c.append(0, None, torch.zeros((1, 20, 1, 64), dtype=c.dtype, device="cuda"), torch.zeros((1, 20, 1, 64), dtype=c.dtype, device="cuda"),
             i32([20]), None, None)
    path = np.arange(20)[None]
    for p, r in ((m.slot(0, s), s) for s in range(20)):
        m.rows[p[0]][p[1]] = 0
    c.commit(i32([20]), i32(path))
    m.commit([20], path.tolist())
    c.k.zero_(), c.v.zero_()
    check_pages(c, m)
    # forks: out of range, into a sequence that holds pages, the same dst twice, a src that is also a dst
    c.fork(i32([0, 4, 0, -1]), i32([0, 1, 9, 2]))
    assert c.error() == P.DEVERR_PAGE
    check_pages(c, m)
    c.fork(i32([0, 0, 0]), i32([1, 1, 2]))
    m.fork([0], [2])
    assert c.error() == P.DEVERR_PAGE
    check_pages(c, m)
    # more columns than the table has; a negative count; more pages than there are: nothing is taken
    for n in ([40, 1, 0, 0], [1, -1, 0, 0], [0, 40, 5, 40]):
        c.reserve(i32(n))
        assert c.error() == P.DEVERR_CAPACITY
        check_pages(c, m)
    # accepted lengths and paths that no tree has commit nothing, the others go on
    n = [2, 3, 0, 3]
    c.reserve(i32(n)), m.reserve(n)
    c.commit(i32([-1, 3, 1, 9]), i32([[0, 1, 2, -1, -1, -1, -1, -1], [0, 2, 2, -1, -1, -1, -1, -1], [99, 0, 0, 0, 0, 0, 0, 0], [0] * 8]))
    assert c.error() == P.DEVERR_TREE
    m.commit([0, 0, 0, 0], [[]] * 4)
    check_pages(c, m)


@pytest.mark.gpu
@pytest.mark.parametrize("told", [-1, -1500, 2001, 4000])
def test_a_free_count_that_cannot_be_stays_inside_the_stack(told):
    """*n_free below zero or above the pool: reported, nothing taken, and nothing written outside the stack (which
    lies between values that would do as page numbers)."""
    pages = 2000
    around = torch.full((3 * pages,), 5, dtype=torch.int32, device="cuda")
    free = around[pages:2 * pages]
    free.copy_(torch.arange(pages - 1, -1, -1, dtype=torch.int32))
    pool = [torch.zeros((1, pages, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    c = P.PagedCache(k=pool[0], v=pool[1], table=i32(np.full((2, pages), -1)), lens=i32([0, 0]), held=i32([0, 0]), refs=i32([0] * pages),
                     free=free, n_free=i32([pages]), n_q_heads=1, max_nodes=1)
    c.reserve(i32([1300 * 16, 5]))
    assert c.error() == 0
    before = [t.clone() for t in (c.table, c.held, c.refs, around)]
    c.n_free.fill_(told)
    c.reserve(i32([0, 1200 * 16]))
    assert c.error() == P.DEVERR_PAGE and int(c.n_free) == told
    assert all(torch.equal(a, b) for a, b in zip((c.table, c.held, c.refs, around), before))
    c.truncate(i32([0, 0]))             # 1301 pages come back: to an empty stack, or to one that is full
    assert c.error() == P.DEVERR_PAGE and int(c.n_free) == (1301 if told < 0 else pages)
    assert (around[:pages] == 5).all() and (around[2 * pages:] == 5).all()
    assert not c.refs.any() and (c.table == -1).all() and c.held.tolist() == [0, 0]
    if told < 0:
        assert free[:1301].tolist() == list(range(1301))      # as they were taken


@pytest.mark.gpu
@pytest.mark.parametrize("at,number", [(0, -1), (0, 1 << 20), (1100, -7), (1100, 2000)])
def test_free_pages_that_do_not_exist_are_not_taken(at, number):
    c = P.PagedCache.allocate(n_layers=1, n_pages=2000, page_size=16, n_q_heads=1, n_kv_heads=1, head_dim=64, max_batch=2, max_pages=1300,
                              max_nodes=1)
    c.free[2000 - 1 - at] = number      # the one that would be taken at-th
    before = [t.clone() for t in (c.table, c.held, c.refs, c.free, c.n_free)]
    c.reserve(i32([7, 1200 * 16]))
    assert c.error() == P.DEVERR_PAGE
    assert all(torch.equal(a, b) for a, b in zip((c.table, c.held, c.refs, c.free, c.n_free), before))


# ------------------------------------------------------------------------------------------ trees

@pytest.mark.gpu
@pytest.mark.parametrize("n,batch,reach", [(1, 1, 1), (5, 3, 2), (16, 4, 4), (32, 2, 32), (33, 3, 8), (255, 5, 8), (300, 2, 1), (1024, 2, 300)])
def test_tree_plan_and_accept(n, batch, reach):
    rng = np.random.default_rng(n)
    counts = rng.integers(0, n + 1, batch)
    counts[0] = n
    parents = np.stack([random_parents(rng, n, reach) for _ in range(batch)])
    if n > 4:
        parents[:, 4] = -1                          # a second branch straight behind the context: never accepted
    tokens, choice = rng.integers(0, 3, (batch, n)), rng.integers(0, 3, (batch, n))     # few tokens: equal siblings, ties
    mask = torch.full((batch, n, up(n, 32)), 7, dtype=torch.int32, device="cuda")
    depth, path = (torch.full((batch, n), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    accept, nxt = (torch.full((batch,), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    P.tree_plan(i32(parents), i32(counts), mask, depth)
    P.tree_accept(i32(tokens), i32(parents), i32(choice), i32(counts), accept, path, nxt)
    for b in range(batch):
        c = counts[b]
        a = np.zeros((n, n), bool)
        a[:c, :c] = ancestors(parents[b, :c])
        assert np.array_equal(mask[b].cpu().numpy(), words(a))
        assert np.array_equal(depth[b].cpu().numpy(), np.maximum(a.sum(1) - 1, 0))
        walk = [0] if c else []
        while walk:
            child = [i for i in range(walk[-1] + 1, c) if parents[b, i] == walk[-1] and tokens[b, i] == choice[b, walk[-1]]]
            if not child:
                break
            walk.append(child[0])
        assert accept[b].item() == len(walk) and path[b].tolist() == walk + [-1] * (n - len(walk))
        assert nxt[b].item() == (choice[b, walk[-1]] if walk else -1)


@pytest.mark.gpu
def test_a_chain_is_accepted_as_a_block_is():
    """tree_accept on chains against verify_accept."""
    rng = np.random.default_rng(2)
    batch, B = 5, 8
    drafts, target = rng.integers(0, 2, (batch, B - 1)), rng.integers(0, 2, (batch, B))
    target[1, :-1] = drafts[1]
    lib = P.DFlare(d=64, n_draft_layers=1, n_target_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=64, ffn=64, vocab=16, block=B,
                   max_batch=batch, max_ctx=64, max_fuse_rows=batch, dtype="f32")
    lib.reset(batch)
    acc, nxt, acc2, nxt2 = (torch.zeros(batch, dtype=torch.int32, device="cuda") for _ in range(4))
    lib.verify_accept(i32(drafts), i32(target), acc, nxt)
    tokens = np.concatenate([np.full((batch, 1), 9), drafts], 1)
    parents = np.tile(np.arange(B) - 1, (batch, 1))
    path = torch.zeros((batch, B), dtype=torch.int32, device="cuda")
    P.tree_accept(i32(tokens), i32(parents), i32(target), i32([B] * batch), acc2, path, nxt2)
    assert torch.equal(acc, acc2) and torch.equal(nxt, nxt2)


@pytest.mark.gpu
def test_impossible_trees_are_reported():
    """The C calls' error word: parents at or after their node, a root with a parent, counts out of range."""
    L = _lib.load()
    for parents, count in (([[-1, 1, 0]], 3), ([[0, 0, 0]], 3), ([[-1, -2, 0]], 3), ([[-1, 0, 1]], 4), ([[-1, 0, 1]], -1)):
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        mask, depth, z = (torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(3))
        p, c = i32(parents), i32([count])
        s = torch.cuda.current_stream().cuda_stream
        assert L.dflare_tree_plan(p.data_ptr(), c.data_ptr(), 1, 3, mask.data_ptr(), depth.data_ptr(), err.data_ptr(), s) == 0
        assert err.item() == P.DEVERR_TREE
        err.zero_()
        P.tree_plan(p, c, mask.view(1, 3), depth, error=err)
        assert err.item() == P.DEVERR_TREE
        err.zero_()
        acc, nxt = i32([0]), i32([0])
        assert L.dflare_tree_accept(z.data_ptr(), p.data_ptr(), z.data_ptr(), c.data_ptr(), 1, 3, acc.data_ptr(), depth.data_ptr(),
                                    nxt.data_ptr(), err.data_ptr(), s) == 0
        assert err.item() == P.DEVERR_TREE


# ------------------------------------------------------------------------------------------ steps

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd,page,n", [(4, 2, 64, 16, 7), (8, 2, 128, 32, 20), (16, 2, 64, 16, 40)])
def test_steps_of_a_server(hq, hkv, hd, page, n, dtype):
    """A prompt read in two chunks and forked, then steps of plan, reserve, append and attend per layer, accept and
    commit: every attention against the definition over the rows in the pages, and the rows against a list of what
    was accepted."""
    rng = np.random.default_rng(n)
    batch, layers, prompt = 3, 2, 45
    c = P.PagedCache.allocate(n_layers=layers, n_pages=60, page_size=page, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, max_batch=batch,
                              max_pages=16, max_nodes=max(n, 30), dtype=dtype)
    for t in (c.k, c.v):
        t.fill_(math.nan)
    phase, magnitude = P.rope_phases(hd, 1e4)
    view = object.__new__(Paged)
    view.t, view.page, view.hq, view.hkv, view.hd, view.k, view.v = c.dtype, page, hq, hkv, hd, c.k, c.v
    kept = [[[np.zeros((0, hkv, hd)), np.zeros((0, hkv, hd))] for _ in range(layers)] for _ in range(batch)]

    def one_pass(counts, width, depth, mask, seen):
        """A layer at a time; returns the nodes' rows as they lie in the pages."""
        view.table, view.lens, view.counts = c.table.cpu().numpy(), c.lens.tolist(), counts
        rows = [[None] * layers for _ in range(batch)]
        for layer in range(layers):
            qkv = torch.from_numpy(rng.standard_normal((batch, width, hq + 2 * hkv, hd)).astype(np.float32)).to(c.dtype).cuda()
            q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
            c.append(layer, q, k, v, i32(counts), phase, q, depth=depth, magnitude=magnitude)
            check_attend(types.SimpleNamespace(**view.__dict__, cache=c, rows=view.rows), q, seen, mask, layer=layer)
            for b in range(batch):
                for i, pool in enumerate((c.k, c.v)):
                    got = view.rows(pool, b, layer)
                    assert np.array_equal(got[:view.lens[b]], kept[b][layer][i])
                rows[b][layer] = [view.rows(pool, b, layer)[view.lens[b]:] for pool in (c.k, c.v)]
        return rows

    def accept(rows, paths):
        for b in range(batch):
            for layer in range(layers):
                kept[b][layer] = [np.concatenate([old, new[paths[b]]]) for old, new in zip(kept[b][layer], rows[b][layer])]

    for chunk in (30, prompt - 30):
        counts = [chunk, 0, 0]
        c.reserve(i32(counts))
        rows = one_pass(counts, chunk, None, None, chain_seen(c.lens.tolist(), counts, chunk))
        c.commit(i32(counts), i32(np.tile(np.arange(chunk), (batch, 1))))
        accept(rows, [list(range(chunk)), [], []])
    c.fork(i32([0, 0]), i32([1, 2]))
    kept[1], kept[2] = ([list(x) for x in kept[0]] for _ in range(2))
    for step in range(3):
        counts = [n, max(n - 3, 1), n // 2]
        parents = np.stack([random_parents(rng, n) for _ in range(batch)])
        tokens, choice = rng.integers(0, 2, (batch, n)), rng.integers(0, 2, (batch, n))
        mask, depth = torch.zeros((batch, n, up(n, 32)), dtype=torch.int32, device="cuda"), torch.zeros((batch, n), dtype=torch.int32, device="cuda")
        acc, nxt, path = i32([0] * batch), i32([0] * batch), torch.zeros_like(depth)
        P.tree_plan(i32(parents), i32(counts), mask, depth)
        c.reserve(i32(counts))
        above = np.zeros((batch, n, n), bool)
        for b, x in enumerate(counts):
            above[b, :x, :x] = ancestors(parents[b, :x])
        seen = [np.concatenate([np.ones((n, x), bool), above[b, :, :counts[b]]], 1) for b, x in enumerate(c.lens.tolist())]
        rows = one_pass(counts, n, depth, mask, seen)
        P.tree_accept(i32(tokens), i32(parents), i32(choice), i32(counts), acc, path, nxt)
        c.commit(acc, path)
        accept(rows, [path[b, :x].tolist() for b, x in enumerate(acc.tolist())])
        assert c.error() == 0 and c.lens.tolist() == [len(kept[b][0][0]) for b in range(batch)]
    assert min(c.lens.tolist()) > prompt


# ------------------------------------------------------------------------------------------ refusals (host)

@pytest.fixture(scope="module")
def raw():
    from paper_2606_02091_gb300 import build
    build.build()
    return _lib.load()


FAKE = ctypes.c_void_p(256)       # never dereferenced: the checks come first


def cache_config(**kw):
    base = dict(n_layers=2, n_pages=16, page_size=16, n_q_heads=8, n_kv_heads=2, head_dim=64, max_batch=4, max_pages=8, max_nodes=16, dtype=0)
    base.update(kw)
    return _lib.CacheConfig(**base)


@pytest.mark.parametrize("field,value", [
    ("n_layers", 0), ("n_layers", 257), ("n_pages", 0), ("page_size", 8), ("page_size", 48), ("page_size", 256), ("n_q_heads", 7),
    ("n_q_heads", 0), ("n_q_heads", 130), ("n_kv_heads", 0), ("n_kv_heads", 129), ("head_dim", 96), ("max_batch", 0), ("max_batch", 257),
    ("max_pages", 0), ("max_pages", 1 << 21), ("max_nodes", 0), ("max_nodes", 1025), ("dtype", 2)])
def test_cache_create_refuses_bad_configs(raw, field, value):
    out = ctypes.c_void_p()
    b = _lib.CacheBuffers(*[256] * 8)
    assert raw.dflare_cache_create(ctypes.byref(cache_config(**{field: value})), ctypes.byref(b), ctypes.byref(out)) == _lib.DFLARE_EINVAL
    assert not out and raw.dflare_last_error(None).startswith(b"invalid cache config")


def test_cache_create_leaves_room_for_the_division_of_the_work(raw):
    """The key tiles of all sequences and heads, divided among up to 760 CTAs and rounded up, stay below 2^31."""
    out = ctypes.c_void_p()
    for batch, hkv, max_pages, fits in ((256, 8, 1048573, False), (256, 8, 1048572, True), (255, 8, 1048573, True)):
        tiles = batch * hkv * (max_pages + 1)
        assert tiles < 2 ** 31 and fits == (tiles <= 2 ** 31 - 1 - 4096)
        g = cache_config(max_batch=batch, n_kv_heads=hkv, n_q_heads=hkv, max_pages=max_pages, page_size=32)
        # (no buffers: what fits is refused for those)
        assert raw.dflare_cache_create(ctypes.byref(g), None, ctypes.byref(out)) == _lib.DFLARE_EINVAL
        assert raw.dflare_last_error(None).startswith(b"dflare_cache_create: a buffer" if fits else b"invalid cache config")


def test_cache_create_refuses_bad_buffers(raw):
    out = ctypes.c_void_p()
    g = cache_config()
    for i in range(8):
        b = [256] * 8
        b[i] = None
        assert raw.dflare_cache_create(ctypes.byref(g), ctypes.byref(_lib.CacheBuffers(*b)), ctypes.byref(out)) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_create(ctypes.byref(g), ctypes.byref(_lib.CacheBuffers(*([264] + [256] * 7))), ctypes.byref(out)) == _lib.DFLARE_EINVAL
    assert b"aligned" in raw.dflare_last_error(None)
    assert raw.dflare_cache_create(ctypes.byref(g), None, ctypes.byref(out)) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_create(None, None, ctypes.byref(out)) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_create(ctypes.byref(g), None, None) == _lib.DFLARE_EINVAL


def test_null_caches_are_refused(raw):
    bits = ctypes.c_uint32()
    assert raw.dflare_cache_destroy(None) == _lib.DFLARE_OK
    assert raw.dflare_cache_error(None, ctypes.byref(bits), None) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_reserve(None, FAKE, 1, None) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_truncate(None, FAKE, 1, None) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_commit(None, FAKE, FAKE, 1, 1, None) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_fork(None, FAKE, FAKE, 1, None) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_copy_pages(None, FAKE, FAKE, 1, None) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_append(None, 0, None, 0, FAKE, 64, FAKE, 64, None, 0, None, FAKE, 1, 1, None, 0, 0, 1.0, None) == _lib.DFLARE_EINVAL
    assert raw.dflare_cache_attend(None, 0, FAKE, 512, None, FAKE, 1, 1, 1.0, FAKE, None, None) == _lib.DFLARE_EINVAL


def test_tree_and_rope_calls_refuse_bad_arguments(raw):
    E = _lib.DFLARE_EINVAL
    assert raw.dflare_tree_plan(None, FAKE, 1, 1, FAKE, FAKE, None, None) == E
    assert raw.dflare_tree_plan(FAKE, FAKE, 0, 1, FAKE, FAKE, None, None) == E
    assert raw.dflare_tree_plan(FAKE, FAKE, 1, 1025, FAKE, FAKE, None, None) == E
    assert raw.dflare_tree_accept(FAKE, FAKE, FAKE, FAKE, 1, 0, FAKE, FAKE, FAKE, None, None) == E
    assert raw.dflare_tree_accept(FAKE, FAKE, None, FAKE, 1, 1, FAKE, FAKE, FAKE, None, None) == E
    good = [FAKE, 64, 64, ctypes.c_void_p(512), 64, 64, FAKE, FAKE, 1, 1, 64, 64, 0, 1.0, 0, 0, None]
    for i, v in ((0, None), (3, None), (6, None), (7, None), (8, 0), (9, 0), (10, 1), (11, 65), (11, 3), (11, 0), (12, 2), (13, math.inf), (15, 2),
                 (1, -1), (5, -1)):
        bad = list(good)
        bad[i] = v
        assert raw.dflare_rope(*bad) == E, i
    bad = list(good)
    bad[8], bad[4] = 2, 32                      # rows of the output would overlap
    assert raw.dflare_rope(*bad) == E
    bad = list(good)
    bad[3], bad[4] = FAKE, 128                  # in place with other strides
    assert raw.dflare_rope(*bad) == E
    ph, m = (ctypes.c_uint64 * 512)(), ctypes.c_float()
    for kw in (dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=1026), dict(scaling=4), dict(theta=1.0), dict(theta=math.inf),
               dict(scaling=1, factor=0.5), dict(scaling=2, rot_dim=2), dict(scaling=3, trained=0.0), dict(scaling=3, beta_fast=1.0)):
        base = dict(rot_dim=64, scaling=0, theta=1e4, factor=2.0, trained=4096.0, beta_fast=32.0, beta_slow=1.0)
        base.update(kw)
        assert raw.dflare_rope_phases(ctypes.byref(_lib.RopeConfig(**base)), ph, ctypes.byref(m)) == E, kw
    assert raw.dflare_rope_phases(None, ph, ctypes.byref(m)) == E


def test_the_binding_structs_follow_the_header():
    import os
    import re
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dflare.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    for struct, mirror in (("dflare_rope_config", _lib.RopeConfig), ("dflare_cache_config", _lib.CacheConfig),
                           ("dflare_cache_buffers", _lib.CacheBuffers)):
        body = re.search(r"typedef struct \{([^}]*)\}\s*" + struct + ";", src).group(1)
        assert re.findall(r"(\w+)\s*;", body) == [f for f, _ in mirror._fields_], struct


@pytest.mark.gpu
def test_the_binding_refuses_wrong_tensors():
    rng = np.random.default_rng(0)
    p = Paged(rng, [5, 6], [2, 2], hq=4, hkv=2, hd=64, page=16, dtype="bf16")
    c, n = p.cache, i32([2, 2])
    q = queries(rng, p, 2, 2)
    out = torch.empty_like(q)
    cases = [
        (ValueError, lambda: c.attend(0, q.float(), n, out)), (ValueError, lambda: c.attend(0, q[:, :, :3], n, out)),
        (ValueError, lambda: c.attend(0, q, n.long(), out)), (ValueError, lambda: c.attend(0, q, n[:1], out)),
        (ValueError, lambda: c.attend(0, q.cpu(), n, out)), (ValueError, lambda: c.attend(0, q.transpose(1, 2).contiguous().transpose(1, 2), n, out)),
        (ValueError, lambda: c.attend(0, q, n, out[:, :, :2])), (ValueError, lambda: c.attend(0, q, n, out, mask=i32([1]))),
        (ValueError, lambda: c.attend(0, q, n, out, lse=torch.zeros(3, device="cuda"))),
        (P.DFlareError, lambda: c.attend(1, q, n, out)), (P.DFlareError, lambda: c.attend(0, q, n, out, scale=0.0)),
        (P.DFlareError, lambda: c.attend(0, q, n, out, scale=math.nan)), (P.DFlareError, lambda: c.attend(0, q, n, out, scale=-1.0)),
        (P.DFlareError, lambda: c.attend(0, queries(rng, p, 2, 3), n, torch.empty((2, 3, 4, 64), dtype=p.t, device="cuda"))),
        (ValueError, lambda: c.append(0, q, q[:, :, :2], q, n, None, out)), (ValueError, lambda: c.append(0, q, q[:, :, :2], q[:, :, :2], n, None, None)),
        (P.DFlareError, lambda: c.append(2, None, q[:, :, :2], q[:, :, :2], n, None, None)),
        (ValueError, lambda: c.append(0, None, q[:, :, :2], q[:, :, :2], n, None, None, layout="thirds")),
        (P.DFlareError, lambda: c.reserve(i32([1] * 5))), (P.DFlareError, lambda: c.truncate(i32([1] * 5))),
        (ValueError, lambda: c.commit(n, i32([0, 1]))), (ValueError, lambda: c.commit(n[:1], i32([[0], [0]]))),
        (ValueError, lambda: c.fork(i32([0, 1]), i32([1]))), (P.DFlareError, lambda: c.copy_pages(i32([0] * 99), i32([1] * 99))),
        (ValueError, lambda: P.rope(q[0], n, P.rope_phases(64)[0], out[0].float())), (ValueError, lambda: P.rope(q[0], n, P.rope_phases(64)[0].int(), out[0])),
        (ValueError, lambda: P.rope(q[0], n[:1], P.rope_phases(64)[0], out[0])), (P.DFlareError, lambda: P.rope(q[0], n, P.rope_phases(66)[0], out[0])),
        (ValueError, lambda: P.rope_phases(64, scaling="cubic")), (P.DFlareError, lambda: P.rope_phases(63)),
        (ValueError, lambda: P.tree_plan(n, n, n, n)), (ValueError, lambda: P.tree_plan(i32([[-1, 0]]), n, i32([0]), n)),
    ]
    for k, (kind, call) in enumerate(cases):
        with pytest.raises(kind):
            call()
            pytest.fail(f"case {k} was accepted")
    assert c.error() == 0


class Elsewhere:
    """A tensor as the binding sees one, on a device of one's choice; its memory is never looked at."""

    is_cuda = True

    def __init__(self, shape, dtype, index):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, f"cuda:{index}"
        self._index, self._plain = index, torch.empty(shape, dtype=dtype, device="meta")

    def get_device(self):
        return self._index

    def data_ptr(self):
        return 4096

    def __getattr__(self, name):        # dim, numel, stride, is_contiguous
        return getattr(self._plain, name)


def there(shape, dtype, index):
    return Elsewhere(shape, getattr(torch, dtype), index)


class Taken:
    """The library's calls, taken down."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if not name.startswith("dflare_"):
            raise AttributeError(name)
        return lambda *a: self.calls.append((name, a)) or 0


DEVICE_CALLS = {
    # the tensors of a call, and the call; b, n, hq, hkv, hd = 2, 3, 4, 2, 64
    "reserve": (dict(n_new=((2,), "int32")), lambda c, t, s: c.reserve(**t, stream=s)),
    "truncate": (dict(new_len=((2,), "int32")), lambda c, t, s: c.truncate(**t, stream=s)),
    "fork": (dict(src=((2,), "int32"), dst=((2,), "int32")), lambda c, t, s: c.fork(**t, stream=s)),
    "copy_pages": (dict(src=((2,), "int32"), dst=((2,), "int32")), lambda c, t, s: c.copy_pages(**t, stream=s)),
    "commit": (dict(accept_len=((2,), "int32"), path=((2, 3), "int32")), lambda c, t, s: c.commit(**t, stream=s)),
    "append": (dict(q=((2, 3, 4, 64), "bfloat16"), k=((2, 3, 2, 64), "bfloat16"), v=((2, 3, 2, 64), "bfloat16"), n_new=((2,), "int32"),
                    phase=((32,), "int64"), q_out=((2, 3, 4, 64), "bfloat16"), depth=((2, 3), "int32")), lambda c, t, s: c.append(0, **t, stream=s)),
    "attend": (dict(q=((2, 3, 4, 64), "bfloat16"), n_nodes=((2,), "int32"), out=((2, 3, 4, 64), "bfloat16"), mask=((2, 3, 1), "int32"),
                    lse=((2, 3, 4), "float32")), lambda c, t, s: c.attend(0, **t, stream=s)),
    "rope": (dict(x=((6, 4, 64), "bfloat16"), positions=((6,), "int32"), phase=((32,), "int64"), out=((6, 4, 64), "bfloat16")),
             lambda c, t, s: P.rope(**t, stream=s)),
    "tree_plan": (dict(parents=((2, 3), "int32"), n_nodes=((2,), "int32"), mask=((2, 3, 1), "int32"), depth=((2, 3), "int32"),
                       error=((1,), "int32")), lambda c, t, s: P.tree_plan(**t, stream=s)),
    "tree_accept": (dict(tokens=((2, 3), "int32"), parents=((2, 3), "int32"), choice=((2, 3), "int32"), n_nodes=((2,), "int32"),
                         accept_len=((2,), "int32"), path=((2, 3), "int32"), next_token=((2,), "int32"), error=((1,), "int32")),
                    lambda c, t, s: P.tree_accept(**t, stream=s)),
}


@pytest.mark.parametrize("name", sorted(DEVICE_CALLS))
def test_the_binding_keeps_to_one_device(name, monkeypatch):
    """A cache's calls run on its device and that device's current stream, whatever the current device is; the other
    calls on the current device. Any tensor or stream of another device is refused before the library is called."""
    from types import SimpleNamespace
    from paper_2606_02091_gb300 import paged
    lib = Taken()
    monkeypatch.setattr(_lib, "load", lambda: lib)
    monkeypatch.setattr(paged, "_device", lambda: 0)
    monkeypatch.setattr(paged, "_raw_stream", lambda device: 1000 + device)
    home = 0 if name in ("rope", "tree_plan", "tree_accept") else 1
    c = object.__new__(P.PagedCache)
    c.__dict__.update(_cache=ctypes.c_void_p(), _L=lib, device_index=1, n_layers=1, n_pages=8, n_kv_heads=2, page_size=16, head_dim=64,
                      max_batch=2, max_pages=3, n_q_heads=4, max_nodes=8, dtype=torch.bfloat16)
    shapes, call = DEVICE_CALLS[name]
    call(c, {x: there(*y, home) for x, y in shapes.items()}, None)
    assert len(lib.calls) == 1 and lib.calls[0][1][-1] == 1000 + home
    call(c, {x: there(*y, home) for x, y in shapes.items()}, SimpleNamespace(device_index=home, cuda_stream=77))
    assert len(lib.calls) == 2 and lib.calls[1][1][-1] == 77
    with pytest.raises(ValueError, match="stream"):
        call(c, {x: there(*y, home) for x, y in shapes.items()}, SimpleNamespace(device_index=1 - home, cuda_stream=77))
    for away in shapes:
        tensors = {x: there(*y, 1 - home if x == away else home) for x, y in shapes.items()}
        with pytest.raises(ValueError, match=f"cuda:{home}"):
            call(c, tensors, None)
    assert len(lib.calls) == 2
    if home:
        c.error()
        assert lib.calls[2][1][-1] == 1001


def test_a_cache_has_its_memory_on_one_device(monkeypatch):
    lib = Taken()
    monkeypatch.setattr(_lib, "load", lambda: lib)
    shapes = dict(k=((1, 8, 2, 16, 64), "bfloat16"), v=((1, 8, 2, 16, 64), "bfloat16"), table=((2, 3), "int32"), lens=((2,), "int32"),
                  held=((2,), "int32"), refs=((8,), "int32"), free=((8,), "int32"), n_free=((1,), "int32"))
    for away in shapes:
        with pytest.raises(ValueError, match="cuda:"):
            P.PagedCache(**{x: there(*y, 1 if x == away else 0) for x, y in shapes.items()}, n_q_heads=4, max_nodes=8)
    with pytest.raises(ValueError, match="CUDA tensor"):
        P.PagedCache(**{x: torch.zeros(y[0], dtype=getattr(torch, y[1])) for x, y in shapes.items()}, n_q_heads=4, max_nodes=8)
    assert not lib.calls


# ------------------------------------------------------------------------------------------ all of it together

@pytest.mark.gpu
@pytest.mark.parametrize("plant", [0.0, 0.7])
def test_the_example_decodes_what_plain_decoding_does(plant):
    from examples import tree_verify as example
    prompt = [(7 * i * i + 3) % example.VOCAB for i in range(37)]
    out, plain, lengths = example.decode(prompt, [5, 6, 7], 8, plant)
    assert all(o == p[:len(o)] for o, p in zip(out, plain))
    if plant:       # the walk takes first and second choices, deep ones among them
        assert max(map(max, lengths)) >= 4 and min(map(min, lengths)) >= 1
