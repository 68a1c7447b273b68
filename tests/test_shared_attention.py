"""Attention of a batch whose sequences share leading pages: against the definition in 64 bits, the groups that are found,
workspaces, and a server's steps of sampling over forked sequences; and refusals."""
import ctypes
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2606_02091_gb300 as P
from paper_2606_02091_gb300 import _lib
from tests.test_tree_verify import FAKE, Paged, Taken, ancestors, attend_reference, chain_seen, host, i32, queries, random_parents, there, tree_masks, up, words


class Shared(Paged):
    """Sequences of (prompt, its pages that are shared, own tokens, nodes): those of one prompt hold the same pages, of the prompt
    `base`, if any, the first `base` pages are everyone's. Slots that hold no token are NaN."""

    def __init__(self, rng, seqs, *, hq, hkv, hd, page, dtype, base=0, layers=1, nodes=None, spare=3):
        self.t = torch.float32 if dtype == "f32" else torch.bfloat16
        self.page, self.hq, self.hkv, self.hd = page, hq, hkv, hd
        self.lens = [(base + s) * page + own for _, s, own, _ in seqs]
        self.counts = [c for *_, c in seqs]
        lead, rows, refs = {}, [], []

        def new(n):
            refs.extend([0] * n)
            return list(range(len(refs) - n, len(refs)))

        common = new(base)
        for (prompt, s, own, c) in seqs:
            pages = lead.setdefault(prompt, [])
            pages += new(s - len(pages)) if s > len(pages) else []
            rows.append(common + pages[:s] + new(up(own + c, page)))
            for x in rows[-1]:
                refs[x] += 1
        pages = len(refs) + spare
        order = rng.permutation(pages)
        self.table = np.full((len(seqs), max(len(r) for r in rows) + 2), -1, np.int32)
        k = np.full((layers, pages, hkv, page, hd), np.nan, np.float32)
        v = k.copy()
        done = set()
        for b, r in enumerate(rows):
            self.table[b, :len(r)] = order[r]
            for i, x in enumerate(r):
                tokens = min(max(self.lens[b] + self.counts[b] - i * page, 0), page)
                if x in done:
                    continue
                done.add(x)
                k[:, order[x], :, :tokens] = rng.standard_normal((layers, hkv, tokens, hd))
                v[:, order[x], :, :tokens] = rng.standard_normal((layers, hkv, tokens, hd))
        counts = np.zeros(pages, np.int32)
        counts[order[:len(refs)]] = refs
        free = np.zeros(pages, np.int32)
        free[:spare] = order[len(refs):]
        self.k, self.v = (torch.from_numpy(x).to(self.t).cuda() for x in (k, v))
        self.cache = P.PagedCache(k=self.k, v=self.v, table=i32(self.table), lens=i32(self.lens), held=i32([len(r) for r in rows]),
                                  refs=i32(counts), free=i32(free), n_free=i32([spare]), n_q_heads=hq, max_nodes=nodes or max(self.counts + [1]))


def run_shared(p, q, mask=None, scale=None, layer=0, work=None, lse=True):
    batch, n = q.shape[:2]
    out = torch.full((batch, n, p.hq, p.hd), 7.0, dtype=p.t, device="cuda")
    logs = torch.full((batch, n, p.hq), 7.0, dtype=torch.float32, device="cuda")
    groups = torch.full((batch, 2), 77, dtype=torch.int32, device="cuda")
    if work is None:
        work = p.cache.shared_work(batch, n)
        p.cache.share_plan(i32(p.counts), n, work, groups=groups)
    p.cache.attend_shared(layer, q, out, work, mask=mask, scale=scale, lse=logs if lse else None)
    assert p.cache.error() == 0
    return out, logs, groups.cpu().numpy()


def check_shared(p, q, seen, mask, scale=None, layer=0):
    out, lse, groups = run_shared(p, q, mask, scale, layer)
    want, wlse, bound, lbound = attend_reference(p, host(q), seen, p.hd ** -0.5 if scale is None else scale, layer)
    off = np.abs(host(out) - want) - bound
    assert not (off > 1e-30).any() and not np.isnan(off).any(), (off.max(), groups.tolist())
    empty = np.isneginf(wlse)
    assert np.array_equal(np.isneginf(host(lse)), empty)
    assert np.all(np.abs(host(lse)[~empty] - wlse[~empty]) <= lbound[~empty])
    return groups


CASES = [
    # base, sequences (prompt, shared pages, own tokens, nodes), hq, hkv, hd, page, groups there must be
    (0, [(0, 70, 3, 1), (0, 70, 40, 1), (0, 70, 0, 1)], 8, 2, 64, 16, [3]),                        # single tokens; nothing but the node of one's own
    (0, [(0, 20, 5, 3), (0, 20, 77, 5), (1, 18, 30, 5), (1, 18, 1, 2)], 6, 2, 128, 64, [2, 2]),    # two prompts
    (0, [(0, 9, 127, 16), (0, 9, 128, 16), (0, 9, 129, 13)], 8, 2, 128, 128, [3]),                 # around a tile's end
    (0, [(0, 40, 10, 33), (0, 40, 200, 40), (1, 0, 60, 2), (0, 40, 3, 1)], 16, 2, 128, 32, None),  # more than 256 rows; another between
    (0, [(0, 30, 9, 4), (1, 1, 20, 4), (2, 1, 3, 4), (2, 1, 9, 4)], 4, 1, 64, 64, [1]),            # shared too little: by themselves
    (20, [(0, 12, 5, 4), (0, 12, 8, 4), (0, 12, 1, 3), (1, 20, 2, 4), (1, 20, 9, 1)], 14, 2, 64, 32, None),   # a system prompt under the prompts
    (0, [(0, 33, 4, 2), (0, 33, 9, 0), (0, 33, 12, 2), (2, 0, 0, 0), (0, 33, 50, 1)], 8, 1, 128, 32, [3]),    # some without nodes
    (0, [(0, 200, 70, 70), (0, 200, 65, 65), (0, 200, 1, 3)], 4, 1, 64, 32, [3]),                  # mask rows of three words
    (0, [(0, 17, 5, 9), (0, 16, 40, 9), (0, 19, 2, 9)], 8, 8, 64, 128, [3]),                       # shared to different depths; one head each
    (0, [(0, 3, 0, 1)], 64, 1, 128, 16, [1]),                                                      # alone
    (0, [(i // 12, 40 + i // 12, 7 * i, 1 + i % 2) for i in range(24)], 16, 2, 64, 16, [12, 12]),      # few rows of many sequences
    (0, [(i // 9, 11, 300 - 11 * i, (1, 0, 3, 4)[i % 4]) for i in range(18)], 12, 4, 128, 64, None),
    (0, [(i, 2, 40 * i, 2) for i in range(20)], 32, 4, 128, 16, []),                                # as many, with nothing shared
    (0, [(0, 100, 0, 1) for i in range(140)], 8, 4, 64, 16, [140]),                                 # a group of more than 128 sequences
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("base,seqs,hq,hkv,hd,page,groups", CASES)
def test_attend_shared_matches_the_definition(base, seqs, hq, hkv, hd, page, groups, dtype):
    rng = np.random.default_rng(len(seqs) + hq + page)
    p = Shared(rng, seqs, hq=hq, hkv=hkv, hd=hd, page=page, dtype=dtype, layers=2, base=base)
    n = max(p.counts)
    q = queries(rng, p, len(seqs), n, fused=True)
    mask, seen = tree_masks(rng, p.lens, p.counts, n)
    got = check_shared(p, q, seen, mask, layer=1)
    check_shared(p, q, chain_seen(p.lens, p.counts, n), None, scale=0.2)
    sizes = [((got[:, 0] == b) & (got[:, 1] > 0)).sum() for b in range(len(seqs))]
    if groups is not None:
        assert [x for x in sizes if x] == [x for x in groups if x > 1]


def best_saving(lens, counts, table, page, heads):
    """The most that any division into groups of neighbours saves, in keys, and what a given one does."""
    act = [b for b, c in enumerate(counts) if c]

    def shared(x, y):
        most = min(lens[x], lens[y]) // page
        same = table[x, :most] == table[y, :most]
        return int(np.argmin(same)) if not same.all() else most

    near = [0] + [shared(act[i - 1], act[i]) for i in range(1, len(act))]
    cost = [16 + 8 * counts[b] * heads for b in act]
    value = lambda i, j: max((j - i - 1) * min(near[i + 1:j]) * page - 128 - sum(cost[i:j]), 0) if j - i > 1 else 0     # noqa: E731
    best = [0]
    for j in range(1, len(act) + 1):
        best.append(max(best[i] + value(i, j) for i in range(j)))

    def of(groups):
        total = 0
        for lead in act:
            mine = [i for i, b in enumerate(act) if groups[b, 0] == lead and groups[b, 1] > 0]
            if mine:
                i, j = mine[0], mine[-1] + 1
                assert mine == list(range(i, j)) and act[i] == lead and len(mine) > 1
                assert all(groups[act[x], 1] == min(near[i + 1:j]) for x in mine)
                total += value(i, j)
        assert all(groups[b, 0] == b or groups[b, 1] > 0 for b in range(len(counts)))
        return total

    return best[-1], of


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(6))
def test_groups_save_the_most(seed):
    """Random batches, sequences that share prompts to random depths among them, some without nodes, up to 256."""
    rng = np.random.default_rng(seed)
    batch = [3, 17, 40, 64, 150, 256][seed]
    prompts = np.sort(rng.integers(0, max(2, batch // 5), batch)) if seed % 2 else rng.integers(0, 3, batch)
    depth = {x: int(rng.integers(0, 90)) for x in range(300)}
    top = [2, 9, 3, 30, 2, 12][seed]
    seqs = [(int(x), int(max(0, depth[int(x)] - rng.integers(0, 3))), int(rng.integers(0, 40)), int(rng.integers(0, top + 1))) for x in prompts]
    p = Shared(rng, seqs, hq=2, hkv=1, hd=64, page=16, dtype="bf16", base=int(rng.integers(0, 8)), nodes=top)
    work, groups = p.cache.shared_work(batch, top), torch.full((batch, 2), 77, dtype=torch.int32, device="cuda")
    p.cache.share_plan(i32(p.counts), top, work, groups=groups)
    most, of = best_saving(p.lens, p.counts, p.table, 16, 2)
    assert of(groups.cpu().numpy()) == most and p.cache.error() == 0
    q = queries(rng, p, batch, top)
    mask, seen = tree_masks(rng, p.lens, p.counts, top)
    check_shared(p, q, seen, mask)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,hq,hkv,hd,prompts,ways,pages", [(1, 16, 8, 64, 5, 9, 60), (2, 16, 4, 128, 2, 24, 90), (5, 32, 8, 64, 4, 6, 40),
                                                                 (18, 32, 4, 128, 3, 8, 50), (40, 16, 2, 128, 1, 14, 70), (3, 8, 1, 128, 1, 2, 600)])
def test_runs_that_cross_from_unit_to_unit(nodes, hq, hkv, hd, prompts, ways, pages, dtype):
    """Units of all lengths and several blocks of rows, whole and cut; three launches follow one another without a wait."""
    rng = np.random.default_rng(nodes)
    seqs = [(x, pages - 3 * x, int(rng.integers(0, 700)), int(rng.integers(0 if nodes > 1 else 1, nodes + 1))) for x in range(prompts) for _ in range(ways)]
    seqs[0] = seqs[0][:3] + (nodes,)
    p = Shared(rng, seqs, hq=hq, hkv=hkv, hd=hd, page=32, dtype=dtype)
    q = queries(rng, p, len(seqs), nodes)
    mask, seen = tree_masks(rng, p.lens, p.counts, nodes)
    check_shared(p, q, seen, mask)
    work = p.cache.shared_work(len(seqs), nodes)
    p.cache.share_plan(i32(p.counts), nodes, work)
    outs = [torch.empty_like(q) for _ in range(3)]
    for o in outs:
        p.cache.attend_shared(0, q, o, work, mask=mask)
    out, _, _ = run_shared(p, q, mask, lse=False)
    assert all(torch.equal(o, out) for o in outs)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,more", [(3, 0), (3, 12), (40, 0)])     # (few rows; few of each sequence; many)
def test_rows_that_see_none_of_their_own_keys(dtype, nodes, more):
    """Masks without a bit: a row has the shared keys alone, or, without a context, none at all."""
    rng = np.random.default_rng(nodes)
    p = Shared(rng, [(0, 200, 0, nodes), (0, 200, 0, nodes), (1, 0, 0, nodes)] + [(2, 9, 40, nodes)] * more, hq=8, hkv=2, hd=64, page=16, dtype=dtype)
    a = np.zeros((3 + more, nodes, nodes), bool)
    a[0, 1, 0] = True
    seen = [np.concatenate([np.ones((nodes, x), bool), a[b]], 1) for b, x in enumerate(p.lens)]
    q = queries(rng, p, 3 + more, nodes)
    groups = check_shared(p, q, seen, i32(words(a)))
    assert groups[:2].tolist() == [[0, 200], [0, 200]]
    out, lse, _ = run_shared(p, q, i32(words(a)))
    assert not host(out)[2].any() and np.isneginf(host(lse)[2]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,hd,more", [(4, 64, 0), (4, 64, 9), (4, 128, 20), (16, 128, 0), (70, 64, 0)])
def test_unseen_infinities_and_nans_stay_out(dtype, nodes, hd, more):
    """Node 1's key and value are NaN and infinite in each sequence of a group: rows that do not see it have the same bits."""
    rng = np.random.default_rng(nodes)
    many = 3 + more
    p = Shared(rng, [(0, 250, 17 + 9 * i, nodes - 2 * (i == 1)) for i in range(many)], hq=8, hkv=2, hd=hd, page=16, dtype=dtype)
    q = queries(rng, p, many, nodes)
    mask, seen = tree_masks(rng, p.lens, p.counts, nodes)
    clean, clean_lse, groups = run_shared(p, q, mask)
    assert groups[:, 1].tolist() == [250] * many
    for b, x in enumerate(p.lens):
        page, off = p.table[b, (x + 1) // 16], (x + 1) % 16
        p.v[0, page, :, off, 3], p.v[0, page, :, off, hd - 1] = math.inf, math.nan
    out, lse, _ = run_shared(p, q, mask)
    sees = np.stack([s[:, x + 1] & (np.arange(nodes) < c) for s, x, c in zip(seen, p.lens, p.counts)])
    o, c = host(out), host(clean)
    rest = [e for e in range(hd) if e not in (3, hd - 1)]
    assert np.array_equal(o[~sees], c[~sees]) and np.array_equal(host(lse), host(clean_lse))
    assert np.isposinf(o[sees][..., 3]).all() and np.isnan(o[sees][..., hd - 1]).all() and np.array_equal(o[sees][..., rest], c[sees][..., rest])
    for b, x in enumerate(p.lens):
        p.k[0, p.table[b, (x + 1) // 16], :, (x + 1) % 16] = math.nan
    out, lse, _ = run_shared(p, q, mask)
    assert np.array_equal(host(out)[~sees], c[~sees]) and np.isnan(host(out)[sees]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("nodes", [1, 20])
def test_long_shared_contexts_past_32_bit_offsets(nodes):
    """A pool of 4.5 GB, whose last pages lie behind 2^31 elements, against attention without sharing on the same pages; each
    is within the bound of one result (keys + 64) eps, and twice the rounding of weights and results."""
    rng = np.random.default_rng(nodes)
    page, hkv, hd, pages, layers = 128, 8, 128, 4200, 4
    lens = [128 * 300 + 5, 128 * 300 + 700, 128 * 300]
    held = [up(x + nodes, page) for x in lens]
    table = np.full((3, max(held)), -1, np.int32)
    lead = np.arange(pages - 300, pages)
    at = pages - 300
    for b in range(3):
        own = held[b] - 300
        at -= own
        table[b, :held[b]] = np.concatenate([lead, np.arange(at, at + own)])
    refs = np.zeros(pages, np.int32)
    for b in range(3):
        refs[table[b, :held[b]]] += 1
    k = torch.randn((layers, pages, hkv, page, hd), dtype=torch.bfloat16, device="cuda")
    v = torch.randn((layers, pages, hkv, page, hd), dtype=torch.bfloat16, device="cuda")
    assert k.numel() > 2 ** 31
    c = P.PagedCache(k=k, v=v, table=i32(table), lens=i32(lens), held=i32(held), refs=i32(refs), free=i32(np.zeros(pages)), n_free=i32([0]), n_q_heads=32,
                     max_nodes=nodes)
    q = torch.randn((3, nodes, 32, hd), dtype=torch.bfloat16, device="cuda")
    counts, out, want, work = i32([nodes] * 3), torch.empty_like(q), torch.empty_like(q), c.shared_work(3, nodes)
    groups = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    c.share_plan(counts, nodes, work, groups=groups)
    c.attend_shared(layers - 1, q, out, work)
    c.attend(layers - 1, q, counts, want)
    assert c.error() == 0 and groups.tolist() == [[0, 300]] * 3
    a, w = host(out), host(want)
    # a weight's rounding moves a result by 2^-8 of its share; |v| below 6 and 38400 keys of like weights: the mean of |v| is below 1
    bound = 2 * (2.0 ** -8 * 1.02 * (1.0 + np.abs(w)) + (40000 + 64) * 2.0 ** -24)
    assert np.all(np.abs(a - w) <= bound) and np.abs(a - w).mean() < 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("n,more,dtype", [(6, 0, "bf16"), (3, 38, "bf16"), (9, 8, "bf16"), (3, 0, "f32")])       # (each of the kernels, and two together)
def test_on_another_stream_in_graphs_and_with_two_workspaces(n, more, dtype):
    rng = np.random.default_rng(12)
    seqs = [(0, 80, 30, n), (0, 80, 9, n), (1, 20, 4, n), (1, 20, 33, n)] + [(2 + i // 8, 30, 7 * i, n) for i in range(more)]
    batch = len(seqs)
    p = Shared(rng, seqs, hq=16, hkv=4, hd=128, page=16, dtype=dtype, layers=2)
    mask, _ = tree_masks(rng, p.lens, p.counts, n)
    q, q2 = queries(rng, p, batch, n), queries(rng, p, batch, n)
    want, want2 = run_shared(p, q, mask)[0], run_shared(p, q2, mask, layer=1)[0]
    counts = i32(p.counts)

    def step(q, out, work, layer, stream=None):
        p.cache.share_plan(counts, n, work, stream=stream)
        p.cache.attend_shared(layer, q, out, work, mask=mask, stream=stream)

    torch.cuda.synchronize()
    side, out, out2 = torch.cuda.Stream(), torch.zeros_like(want), torch.zeros_like(want)
    works = [p.cache.shared_work(batch, n) for _ in range(3)]
    torch.cuda.synchronize()
    step(q, out, works[0], 0, side)
    step(q2, out2, works[1], 1)         # at the same time
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(out2, want2)
    graphs = []
    for x, o, layer, work in ((q, out, 0, works[2]), (q2, out2, 1, works[2])):      # graphs that take turns on one workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(x, o, work, layer)
        graphs.append(g)
    for _ in range(3):
        out.zero_()
        out2.zero_()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out2, want2)
    # the lengths that the graph reads are those of the replay: shorter contexts, of which some share a page less
    p.cache.lens.add_(-4)
    p.cache.attend(0, q, counts, want, mask=mask)
    graphs[0].replay()
    torch.cuda.synchronize()
    assert p.cache.error() == 0 and (host(out) - host(want)).__abs__().max() <= 2 * 2.0 ** -8 * 1.02 * (4 + np.abs(host(want)).max())


@pytest.mark.gpu
@pytest.mark.parametrize("n,more,dtype", [(6, 0, "bf16"), (3, 38, "bf16"), (9, 8, "bf16"), (3, 0, "f32")])       # (each of the kernels, and two together)
def test_a_replayed_plan_goes_by_the_lengths_that_it_finds(n, more, dtype):
    """The plan and the attention in one graph: after the lengths change a replay gives the bits of the plain calls at the new lengths,
    which are those of the definition, and not the ones before."""
    rng = np.random.default_rng(17)
    seqs = [(0, 80, 30, n), (0, 80, 9, n), (1, 20, 4, n), (1, 20, 33, n)] + [(2 + i // 8, 30, 5 + 7 * i, n) for i in range(more)]
    batch = len(seqs)
    p = Shared(rng, seqs, hq=16, hkv=4, hd=128, page=16, dtype=dtype)
    mask, seen = tree_masks(rng, p.lens, p.counts, n)
    q, out, counts, work = queries(rng, p, batch, n), torch.zeros((batch, n, 16, 128), dtype=p.t, device="cuda"), i32(p.counts), p.cache.shared_work(batch, n)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.cache.share_plan(counts, n, work)
        p.cache.attend_shared(0, q, out, work, mask=mask)
    g.replay()
    before = out.clone()
    p.cache.lens.sub_(4)        # (of which some share a page less)
    p.lens = [x - 4 for x in p.lens]
    g.replay()
    a = [s[:, 4:] for s in seen]        # four tokens of the context less: node j's key is where node j - 4's was
    want, _, bound, _ = attend_reference(p, host(q), a, p.hd ** -0.5)
    off = np.abs(host(out) - want) - bound
    assert p.cache.error() == 0 and not (off > 1e-30).any() and not np.isnan(off).any(), off.max()
    # (of the four keys that are gone the heaviest, for the row and head that give it most, has several times the bound: of 1300 keys a weight
    # of e^3 / 1300 / e^0.5 = 0.009 and more for one of 48 rows and heads, and the bound is 2 2^-8 of the mean |v|, 0.006)
    assert (np.abs(host(before) - want) > bound).any((1, 2, 3)).all()
    fresh = torch.zeros_like(out)
    p.cache.attend_shared(0, q, fresh, work, mask=mask)
    assert torch.equal(fresh, out)
    again, _, _ = run_shared(p, q, mask)
    assert torch.equal(again, out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd,page,n", [(4, 2, 64, 16, 7), (32, 4, 128, 32, 12)])
def test_a_forked_cache_against_the_definition(hq, hkv, hd, page, n, dtype):
    """Steps of sampled trees over forked sequences, each layer's attention against the definition over the keys that the tables name, within the
    bound of a result's own arithmetic."""
    rng = np.random.default_rng(18 + n)
    layers, batch = 2, 5
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    make = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(t).cuda()     # noqa: E731
    c = P.PagedCache.allocate(n_layers=layers, n_pages=300, page_size=page, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, max_batch=batch, max_pages=60,
                              max_nodes=n, dtype=dtype)
    lens = i32([page * 22 + 3, 0, 0, page * 25, 0])
    c.reserve(lens)
    most = page * 25
    for layer in range(layers):
        c.append(layer, None, make(batch, most, hkv, hd), make(batch, most, hkv, hd), lens, None, None)
    c.commit(lens, i32(np.tile(np.arange(most), (batch, 1))))
    c.fork(i32([0, 0, 3]), i32([1, 2, 4]))
    work, groups = c.shared_work(batch, n), torch.zeros((batch, 2), dtype=torch.int32, device="cuda")
    for step in range(3):
        counts = [int(x) for x in rng.integers(1, n + 1, batch)]
        parents = np.stack([random_parents(rng, n, 3) for _ in range(batch)])
        nodes = i32(counts)
        mask, depth = torch.zeros((batch, n, up(n, 32)), dtype=torch.int32, device="cuda"), torch.zeros((batch, n), dtype=torch.int32, device="cuda")
        P.tree_plan(i32(parents), nodes, mask, depth)
        c.reserve(nodes)
        c.share_plan(nodes, n, work, groups=groups)
        most, of = best_saving(c.lens.tolist(), counts, c.table.cpu().numpy(), page, hq // hkv)
        assert of(groups.cpu().numpy()) == most     # (where a member costs more than it saves it is by itself)
        view = SimpleNamespace(lens=c.lens.tolist(), counts=counts, page=page, hq=hq, hkv=hkv, hd=hd, table=c.table.cpu().numpy(), k=c.k, v=c.v, t=t)
        view.rows = lambda pool, b, layer=0: Paged.rows(view, pool, b, layer)     # noqa: B023
        seen = [np.concatenate([np.ones((n, x), bool), ancestors(par)[:, :m]], 1) for x, par, m in zip(view.lens, parents, counts)]
        for layer in range(layers):
            q, k, v = make(batch, n, hq, hd), make(batch, n, hkv, hd), make(batch, n, hkv, hd)
            out = torch.zeros_like(q)
            c.append(layer, None, k, v, nodes, None, None)
            c.attend_shared(layer, q, out, work, mask=mask)
            want, _, bound, _ = attend_reference(view, host(q), seen, hd ** -0.5, layer)
            for b, m in enumerate(counts):
                off = np.abs(host(out)[b, :m] - want[b, :m]) - bound[b, :m]
                assert not (off > 1e-30).any() and not np.isnan(off).any(), (step, layer, b, off.max())
        accept = i32([int(rng.integers(1, m + 1)) for m in counts])
        c.commit(accept, i32(np.tile(np.arange(n), (batch, 1))))
        assert c.error() == 0


@pytest.mark.gpu
def test_a_workspace_without_the_plan_is_reported_and_nothing_written():
    rng = np.random.default_rng(13)
    p = Shared(rng, [(0, 40, 3, 2), (0, 40, 9, 2)], hq=8, hkv=2, hd=64, page=16, dtype="bf16", nodes=4)
    q, out = queries(rng, p, 2, 2), torch.full((2, 2, 8, 64), 7.0, dtype=p.t, device="cuda")
    work = p.cache.shared_work(2, 4)
    for _ in range(2):      # no plan, and one for more nodes
        p.cache.attend_shared(0, q, out, work)
        assert p.cache.error() == _lib.DEVERR_PLAN and (out == 7).all()
        p.cache.share_plan(i32(p.counts), 4, work)
    # plans of caches with longer tables, other pages, other heads
    for kw in (dict(seqs=[(0, 90, 3, 2), (0, 90, 9, 2)]), dict(page=32), dict(hq=4), dict(hkv=4)):
        other = Shared(rng, **{**dict(seqs=[(0, 40, 3, 2), (0, 40, 9, 2)], hq=8, hkv=2, hd=64, page=16, dtype="bf16", nodes=4), **kw})
        more = other.cache.shared_work(2, 2)
        other.cache.share_plan(i32(other.counts), 2, more)
        room = torch.zeros(max(more.numel(), p.cache.shared_work(2, 2).numel()), dtype=torch.uint8, device="cuda")
        room[:more.numel()] = more
        p.cache.attend_shared(0, q, out, room)
        assert p.cache.error() == _lib.DEVERR_PLAN and (out == 7).all()
    p.cache.share_plan(i32(p.counts), 2, work)
    p.cache.attend_shared(0, q, out, work)
    assert p.cache.error() == 0 and not (out == 7).any()
    with pytest.raises(ValueError, match="bytes"):
        p.cache.attend_shared(0, q, out, work[:1024])


@pytest.mark.gpu
@pytest.mark.parametrize("batch,n,hkv", [(2, 2, 2), (6, 8, 4), (80, 1, 2)])      # (bf16: few rows, many, a list each for own and shared keys)
@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_a_plan_of_another_type_or_head_size_is_reported(dtype, hd, batch, n, hkv):
    """The lists of work, and where everything lies, go by them: a plan of another kind of cache is not used, either way round."""
    rng = np.random.default_rng(15)
    make = lambda t, d: Shared(rng, [(0, 40, 3, n)] * batch, hq=2 * hkv, hkv=hkv, hd=d, page=16, dtype=t, nodes=n)     # noqa: E731
    p = make(dtype, hd)
    q = queries(rng, p, batch, n)
    out, need = torch.full_like(q, 7.0), p.cache.shared_work(batch, n).numel()
    for t, d in (("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)):
        if (t, d) == (dtype, hd):
            continue
        other = make(t, d)
        more = other.cache.shared_work(batch, n)
        other.cache.share_plan(i32(other.counts), n, more)
        room = torch.zeros(max(more.numel(), need), dtype=torch.uint8, device="cuda")
        room[:more.numel()] = more
        p.cache.attend_shared(0, q, out, room)
        assert p.cache.error() == _lib.DEVERR_PLAN and (out == 7).all(), (t, d)
        p.cache.share_plan(i32(p.counts), n, room)
        p.cache.attend_shared(0, q, out, room)
        assert p.cache.error() == 0 and not (out == 7).any()
        out.fill_(7.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_do_not_exist_and_pages_that_are_missing(dtype):
    """A shared page number that does not exist ends the shared part; its keys read as zeros and it is reported, as without
    sharing. A length beyond the pages: the keys that exist."""
    rng = np.random.default_rng(14)
    p = Shared(rng, [(0, 60, 3, 2), (0, 60, 9, 2)], hq=8, hkv=2, hd=64, page=16, dtype=dtype)
    q, counts = queries(rng, p, 2, 2), i32([2, 2])
    p.cache.table[:, 50] = 10 ** 6
    out, want, work, groups = torch.zeros_like(q), torch.zeros_like(q), p.cache.shared_work(2, 2), torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    p.cache.share_plan(counts, 2, work, groups=groups)
    p.cache.attend_shared(0, q, out, work)
    assert p.cache.error() == _lib.DEVERR_PAGE and groups.tolist() == [[0, 50]] * 2
    p.cache.attend(0, q, counts, want)
    assert p.cache.error() == _lib.DEVERR_PAGE
    limit = 2 * ((2.0 ** -8 * 1.02 * (1 + np.abs(host(want)).max())) if dtype == "bf16" else 1200 * 2.0 ** -24 * 4)
    assert np.abs(host(out) - host(want)).max() <= limit
    p.cache.table.copy_(i32(p.table))
    p.cache.lens.copy_(i32([10 ** 6, 2 ** 31 - 1]))
    p.k.copy_(p.k.nan_to_num(0.5))
    p.v.copy_(p.v.nan_to_num(0.5))
    p.cache.share_plan(counts, 2, work, groups=groups)
    p.cache.attend_shared(0, q, out, work)
    p.cache.attend(0, q, counts, want)
    assert p.cache.error() == 0 and groups.tolist() == [[0, 60]] * 2 and np.abs(host(out) - host(want)).max() <= limit


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd,page,n", [(4, 2, 64, 16, 7), (8, 2, 128, 32, 12)])
def test_steps_of_a_sampling_server(hq, hkv, hd, page, n, dtype):
    """Two prompts, forked into three and two continuations; per step and layer normed and rotated heads into the pages, shared
    attention, sampled acceptance, commit. Every piece against the plain calls on a twin without sharing: its own pages with the same
    tokens."""
    rng = np.random.default_rng(n)
    layers, vocab, batch = 2, 300, 5
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    make = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(t).cuda()     # noqa: E731
    new = lambda: P.PagedCache.allocate(n_layers=layers, n_pages=900, page_size=page, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, max_batch=batch,     # noqa: E731
                                        max_pages=100, max_nodes=n, dtype=dtype)
    c, twin = new(), new()
    phase, eps = P.rope_phases(hd, 1e4)[0], 1e-6
    qg, kg = (1 + 0.1 * make(hd)).to(t), (1 + 0.1 * make(hd)).to(t)
    # prompts of the leaders 0 and 3
    lens = [page * 42 + 3, 0, 0, page * 60, 0]
    most = max(lens)
    kp, vp = make(layers, batch, most, hkv, hd), make(layers, batch, most, hkv, hd)
    for x in (1, 2):
        kp[:, x], vp[:, x] = kp[:, 0], vp[:, 0]
    kp[:, 4], vp[:, 4] = kp[:, 3], vp[:, 3]
    for cache, mine in ((c, lens), (twin, [lens[0], lens[0], lens[0], lens[3], lens[3]])):
        for at in range(0, most, 1000):     # (a commit takes 1024 tokens at most)
            end = min(at + 1000, most)
            chunk = i32(np.clip(np.array(mine) - at, 0, end - at))
            cache.reserve(chunk)
            for layer in range(layers):
                cache.append(layer, None, kp[layer, :, at:end].contiguous(), vp[layer, :, at:end].contiguous(), chunk, phase, None, k_gain=kg, eps=eps)
            cache.commit(chunk, i32(np.tile(np.arange(end - at), (batch, 1))))
    c.fork(i32([0, 0, 3]), i32([1, 2, 4]))
    assert c.error() == 0 and twin.error() == 0 and torch.equal(c.lens, twin.lens)
    work, groups = c.shared_work(batch, n), torch.zeros((batch, 2), dtype=torch.int32, device="cuda")
    for step in range(4):
        counts = [int(x) for x in rng.integers(1, n + 1, batch)]
        parents = np.stack([random_parents(rng, n, 3) for _ in range(batch)])
        nodes, par = i32(counts), i32(parents)
        mask, depth = torch.zeros((batch, n, up(n, 32)), dtype=torch.int32, device="cuda"), torch.zeros((batch, n), dtype=torch.int32, device="cuda")
        P.tree_plan(par, nodes, mask, depth)
        c.reserve(nodes)
        twin.reserve(nodes)
        c.share_plan(nodes, n, work, groups=groups)
        assert groups.tolist() == [[0, 42]] * 3 + [[3, 60]] * 2
        for layer in range(layers):
            qkv = make(batch, n, hq + 2 * hkv, hd)
            q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
            turned, same = torch.zeros((batch, n, hq, hd), dtype=t, device="cuda"), torch.zeros((batch, n, hq, hd), dtype=t, device="cuda")
            c.append(layer, q, k, v, nodes, phase, turned, depth=depth, q_gain=qg, k_gain=kg, eps=eps)
            # the same heads normed and turned apart, and stored as they are
            at = (twin.lens[:, None] + depth).int().flatten()
            kk = torch.zeros((batch * n, hkv, hd), dtype=t, device="cuda")
            P.qk_norm_rope(qkv.view(batch * n, -1, hd)[:, :hq], qkv.view(batch * n, -1, hd)[:, hq:hq + hkv], at, phase, qg, kg,
                           same.view(batch * n, hq, hd), kk, eps=eps)
            twin.append(layer, None, kk.view(batch, n, hkv, hd), v, nodes, None, None)
            out, plain = torch.zeros_like(turned), torch.zeros_like(turned)
            c.attend_shared(layer, turned, out, work, mask=mask)
            twin.attend(layer, turned, nodes, plain, mask=mask)
            for b in range(batch):
                assert torch.equal(turned[b, :counts[b]], same[b, :counts[b]])
            limit = 2 * (2.0 ** -8 * 1.02 * (4 + np.abs(host(plain)).max()) if dtype == "bf16" else 5000 * 2.0 ** -24 * 5)
            assert np.abs(host(out) - host(plain)).max() <= limit
        p, d = (torch.softmax(torch.from_numpy(2 * rng.standard_normal((batch, n, vocab))).float().cuda(), -1) for _ in range(2))
        tokens = torch.multinomial(d.view(-1, vocab), 1).view(batch, n).int()
        tokens = torch.gather(tokens, 1, par.clamp(min=0).long()).contiguous() if step % 2 else tokens
        u = torch.from_numpy(rng.random((batch, n)).astype(np.float32)).cuda()
        accept, path, following = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((batch,), (batch, n), (batch,)))
        P.tree_sample(tokens, par, nodes, p, d, u, accept, path, following)
        c.commit(accept, path)
        twin.commit(accept, path)
        assert c.error() == 0 and twin.error() == 0 and torch.equal(c.lens, twin.lens) and (following >= 0).all()
    for b in range(batch):      # the same tokens' keys and values, wherever their pages lie
        s = np.arange(int(c.lens[b]))
        for pool, other in ((c.k, twin.k), (c.v, twin.v)):
            x = pool[:, c.table[b].long()[s // page], :, s % page]
            y = other[:, twin.table[b].long()[s // page], :, s % page]
            assert torch.equal(x, y)


def test_the_streams_meet_before_one_of_them_goes_on_to_a_second_unit():
    """A stream without a tile of the first unit would arrive twice at the barrier of the queries, which counts arrivals only. No run can
    show that for certain, so this reads the source: between the first arrival and the loop over the units the streams meet."""
    import os
    import re
    src = open(os.path.join(os.path.dirname(P.__file__), "csrc", "tree_attention_tc.cu")).read()
    src = re.sub(r"//[^\n]*", "", src)
    first, loop = src.index("q_there();"), src.index("while (more) {")
    assert first < loop and re.search(r"if \(alternate\(p\)\) streams_meet\(\);", src[first:loop])


@pytest.mark.gpu
@pytest.mark.parametrize("hd,nodes", [(128, 24), (64, 24), (64, 40)])
def test_units_of_one_tile_one_after_another(hd, nodes):
    """Single tokens with up to 128 keys of their own beside one tree: every CTA goes through several units of one tile, of which one
    softmax stream has none, from its first on. Queries of one call must not show in the next one's."""
    rng = np.random.default_rng(nodes + hd)
    seqs = [(i // 8, 20, int(rng.integers(0, 120)), 1) for i in range(119)] + [(90, 0, 30, nodes)]
    p = Shared(rng, seqs, hq=32, hkv=8, hd=hd, page=16, dtype="bf16")
    mask, seen = tree_masks(rng, p.lens, p.counts, nodes)
    work = p.cache.shared_work(len(seqs), nodes)
    p.cache.share_plan(i32(p.counts), nodes, work)
    for _ in range(4):
        q = queries(rng, p, len(seqs), nodes)
        want, _, bound, _ = attend_reference(p, host(q), seen, hd ** -0.5)
        shared, plain = torch.empty_like(q), torch.empty_like(q)
        p.cache.attend_shared(0, q, shared, work, mask=mask)
        p.cache.attend(0, q, i32(p.counts), plain, mask=mask)
        for out in (shared, plain):
            off = np.abs(host(out) - want) - bound
            assert not (off > 1e-30).any() and not np.isnan(off).any(), off.max()
    assert p.cache.error() == 0


# ------------------------------------------------------------------------------------------ refusals (host)

@pytest.fixture(scope="module")
def raw():
    from paper_2606_02091_gb300 import build
    build.build()
    return _lib.load()


def test_null_caches_are_refused(raw):
    E, size = _lib.DFLARE_EINVAL, ctypes.c_size_t()
    assert raw.dflare_cache_shared_bytes(None, 1, 1, ctypes.byref(size)) == E
    assert raw.dflare_cache_share_plan(None, FAKE, 1, 1, FAKE, None, None) == E
    assert raw.dflare_cache_attend_shared(None, 0, FAKE, 512, None, 1, 1, 1.0, FAKE, None, FAKE, None) == E


@pytest.mark.gpu
def test_bad_arguments_are_refused(raw):
    rng = np.random.default_rng(0)
    p = Shared(rng, [(0, 4, 5, 2), (0, 4, 6, 2)], hq=4, hkv=2, hd=64, page=16, dtype="bf16")
    E, c, size = _lib.DFLARE_EINVAL, p.cache._cache, ctypes.c_size_t()
    for args in ((c, 0, 2), (c, 3, 2), (c, 2, 0), (c, 2, 3)):
        assert raw.dflare_cache_shared_bytes(*args, ctypes.byref(size)) == E
        assert raw.dflare_cache_share_plan(args[0], FAKE, *args[1:], FAKE, None, None) == E
        assert raw.dflare_cache_attend_shared(args[0], 0, FAKE, 256, None, *args[1:], 1.0, FAKE, None, FAKE, None) == E
    odd = ctypes.c_void_p(256 + 64)
    assert raw.dflare_cache_share_plan(c, FAKE, 2, 2, odd, None, None) == E and raw.dflare_cache_share_plan(c, None, 2, 2, FAKE, None, None) == E
    good = [c, 0, FAKE, 256, None, 2, 2, 1.0, FAKE, None, FAKE, None]
    for i, v in ((1, 1), (1, -1), (2, None), (2, ctypes.c_void_p(264)), (3, 255), (3, 260), (7, 0.0), (7, math.nan), (7, math.inf), (8, None),
                 (8, ctypes.c_void_p(264)), (10, None), (10, odd)):
        bad = list(good)
        bad[i] = v
        assert raw.dflare_cache_attend_shared(*bad) == E, i
    assert p.cache.error() == 0


def test_the_binding_keeps_to_one_device_and_refuses_wrong_tensors(monkeypatch):
    from paper_2606_02091_gb300 import paged
    lib = Taken()
    monkeypatch.setattr(paged, "_device", lambda: 0)
    monkeypatch.setattr(paged, "_raw_stream", lambda device: 1000 + device)
    c = object.__new__(P.PagedCache)
    c.__dict__.update(_cache=ctypes.c_void_p(), _L=lib, device_index=1, n_layers=1, n_pages=8, n_kv_heads=2, page_size=16, head_dim=64,
                      max_batch=2, max_pages=3, n_q_heads=4, max_nodes=8, dtype=torch.bfloat16, _sizes={(2, 3): 4096})
    work = ((4096,), "uint8")
    calls = {
        "plan": (dict(n_nodes=((2,), "int32"), work=work, groups=((2, 2), "int32")), lambda t, s: c.share_plan(n=3, **t, stream=s)),
        "attend": (dict(q=((2, 3, 4, 64), "bfloat16"), out=((2, 3, 4, 64), "bfloat16"), work=work, mask=((2, 3, 1), "int32"), lse=((2, 3, 4), "float32")),
                   lambda t, s: c.attend_shared(0, **t, stream=s)),
    }
    for name, (shapes, call) in calls.items():
        good = {x: there(*y, 1) for x, y in shapes.items()}
        before = len(lib.calls)
        call(good, None)
        call(good, SimpleNamespace(device_index=1, cuda_stream=77))
        assert [a[-1] for _, a in lib.calls[before:]] == [1001, 77]
        with pytest.raises(ValueError, match="stream"):
            call(good, SimpleNamespace(device_index=0, cuda_stream=77))
        for away, (shape, dtype) in shapes.items():
            with pytest.raises(ValueError, match="cuda:1"):
                call(dict(good, **{away: there(shape, dtype, 0)}), None)
            with pytest.raises(ValueError):
                call(dict(good, **{away: there(shape, "float64", 1)}), None)
            if away != "n_nodes":       # (the batch goes by it)
                with pytest.raises(ValueError):
                    call(dict(good, **{away: there((1,) * len(shape), dtype, 1)}), None)
        assert len(lib.calls) == before + 2
