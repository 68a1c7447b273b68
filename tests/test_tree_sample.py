"""Sampled acceptance in drafted trees from given probabilities and random numbers, against the definition in 64 bits and
against the target's distribution, and its refusals."""
import ctypes
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2606_02091_gb300 as P
from paper_2606_02091_gb300 import _lib
from tests.test_tree_verify import FAKE, Taken, i32, random_parents, there

MODES = ["drawn", "distinct", "picked"]


def walk(tokens, parents, count, p, q, u, distinct):
    """The definition for one tree, the residual taken step by step: nodes on the walk, and the next token."""
    u = np.nan_to_num(np.clip(u.astype(np.float64), 0.0, 1.0 - 2.0 ** -24), nan=0.0)
    at, path = 0, [0]
    while True:
        w, W, Q, kept = p[at].astype(np.float64), 1.0, 1.0, None
        for i in (j for j in range(at + 1, count) if parents[j] == at):
            x = tokens[i]
            if q is None:
                if u[i] * W < w[x]:
                    kept = i
                    break
                W -= w[x]
                w[x] = 0.0
                continue
            row = q[at].astype(np.float64)
            if u[i] * W * (row[x] / Q if Q > 0 else 0.0) < w[x]:
                kept = i
                break
            if Q > 0:
                w = np.maximum(w - W / Q * row, 0.0)
            W = w.sum()
            if distinct:
                Q -= row[x]
        if kept is None:
            break
        at = kept
        path.append(at)
    if not w.sum() > 0:
        w = p[at].astype(np.float64)
    upto = np.cumsum(w)
    return path, int(np.searchsorted(upto, u[0] * upto[-1], side="right"))


def softmax(z):
    z = np.exp(z - z.max(-1, keepdims=True))
    return (z / z.sum(-1, keepdims=True)).astype(np.float32)


def draw_children(rng, parents, q, mode):
    """Tokens of every tree's nodes, as a drafter chooses them."""
    batch, n = parents.shape
    tokens = np.zeros((batch, n), np.int32)
    for b in range(batch):
        for at in range(n):
            kids = [i for i in range(at + 1, n) if parents[b, i] == at]
            if not kids:
                continue
            row = q[b, at].astype(np.float64)
            if mode == "drawn":
                tokens[b, kids] = rng.choice(len(row), len(kids), p=row / row.sum())
            elif mode == "distinct":
                tokens[b, kids] = np.argsort(-(np.log(np.maximum(row, 1e-300)) + rng.gumbel(size=len(row))))[:len(kids)]
            else:
                tokens[b, kids] = np.argsort(-row)[:len(kids)]
    return tokens


def make(rng, batch, n, vocab, mode, reach, spread=2.0, apart=0.7):
    z = spread * rng.standard_normal((batch, n, vocab))
    p, q = softmax(z + apart * rng.standard_normal(z.shape)), softmax(z)
    parents = np.stack([random_parents(rng, n, reach) for _ in range(batch)])
    return draw_children(rng, parents, q, mode), parents, p, q, rng.random((batch, n)).astype(np.float32)


def call(tokens, parents, counts, p, q, u, mode, **kw):
    batch, n = parents.shape
    out = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((batch,), (batch, n), (batch,))]
    err = i32([0])
    P.tree_sample(i32(tokens), i32(parents), i32(counts), torch.from_numpy(p).cuda(), None if mode == "picked" else torch.from_numpy(q).cuda(),
                  torch.from_numpy(u).cuda(), *out, distinct=mode == "distinct", error=err, **kw)
    return [x.cpu().numpy() for x in out] + [int(err)]


def check(tokens, parents, counts, p, q, u, mode):
    accept, path, following, err = call(tokens, parents, counts, p, q, u, mode)
    assert err == 0
    lengths = []
    for b, c in enumerate(counts):
        if c == 0:
            assert accept[b] == 0 and following[b] == -1 and (path[b] == -1).all()
            continue
        want, token = walk(tokens[b], parents[b], c, p[b], None if mode == "picked" else q[b], u[b], mode == "distinct")
        assert path[b, :accept[b]].tolist() == want and (path[b, accept[b]:] == -1).all() and following[b] == token, b
        lengths.append(len(want))
    return lengths


# Whole numbers have to be equal. The running sums are good to 2^-40 of the whole, so a token differs with a probability of
# 2^-40 for each of its vocabulary's borders at most: 10^-6 over all these cases.
CASES = [
    # batch, n, vocab, reach (1: chains)
    (1, 1, 1, 1), (3, 2, 2, 1), (5, 7, 5, 3), (2, 16, 1000, 1), (40, 9, 333, 4), (3, 12, 4096, 5), (1, 30, 20011, 3), (9, 16, 8191, 1),
    (2, 8, 70000, 2), (1, 5, 131072, 8), (160, 6, 130, 3), (310, 4, 2049, 2), (1, 64, 6000, 6), (1, 1024, 40, 300),
]


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("batch,n,vocab,reach", CASES)
def test_walks_match_the_definition(batch, n, vocab, reach, mode):
    rng = np.random.default_rng(batch * 1000 + n + vocab)
    data = make(rng, batch, n, vocab, mode if vocab >= n else "drawn", reach)
    counts = rng.integers(1, n + 1, batch)
    counts[0] = n
    if batch > 2:
        counts[1] = 0
    check(data[0], data[1], counts, *data[2:], mode)


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("apart", [0.0, 0.05, 4.0])
def test_drafts_that_agree_and_that_do_not(apart, mode):
    """Equal distributions: everything drawn is kept, and after siblings nothing is left of the residual."""
    rng = np.random.default_rng(3)
    data = make(rng, 24, 14, 500, mode, 3, 3.0, apart)
    lengths = check(data[0], data[1], [14] * 24, *data[2:], mode)
    if apart == 0.0 and mode != "picked":       # u q < p = q
        assert min(lengths) >= 2


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
def test_residuals_far_below_one(mode):
    """One token has nearly all of the mass, so that what rejections leave is 10^-6 of it."""
    rng = np.random.default_rng(4)
    tokens, parents, p, q, u = make(rng, 30, 10, 3000, mode, 3)
    for x in (p, q):
        x *= np.float32(1e-6)
        x[..., 17] = 1.0 - 1e-6
    tokens[:, 1::2] = 17 if mode != "distinct" else tokens[:, 1::2]
    u[:, ::3] = 1.0 - 2.0 ** -24
    check(tokens, parents, [10] * 30, p, q, u, mode)


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
def test_random_numbers_at_the_ends_of_their_range(mode):
    rng = np.random.default_rng(5)
    tokens, parents, p, q, u = make(rng, 12, 9, 700, mode, 3)
    p[:, :, :3] = 0.0           # no token of weight zero may come out, whatever u_0
    p[:, :, -2:] = 0.0
    for b, x in enumerate((0.0, 1.0, -1.0, math.nan, math.inf, 2.0 ** -149)):
        u[2 * b] = x
        u[2 * b + 1, 0] = x
    check(tokens, parents, [9] * 12, p, q, u, mode)
    following = call(tokens, parents, [1] * 12, p, q, u, mode)[2]
    assert all(p[b, 0, x] > 0 for b, x in enumerate(following))


@pytest.mark.gpu
def test_a_run_of_weightless_tokens_where_the_sum_is_reached():
    """u_0 = 1/2, and the weight before a run of zeros is within 2^-46 of that behind it, on either side: the token before the run or
    the one behind it, by the rounding of running sums (2^-40), but none of the run, nor token 0, which weighs nothing either."""
    rng = np.random.default_rng(15)
    batch, vocab = 6000, 64
    p, ends = np.zeros((batch, 1, vocab), np.float32), []
    for b in range(batch):
        k = int(rng.integers(2, 14))        # the run: 4 k .. 4 k + 3
        p[b, 0, 1:4 * k] = np.ldexp((2 ** 23 + rng.integers(0, 2 ** 23, 4 * k - 1)).astype(np.float64), -28 - rng.integers(0, 30, 4 * k - 1))
        rest, at = math.fsum(p[b, 0].tolist()) * (1 + (int(rng.integers(0, 33)) - 16) * 2.0 ** -51), 4 * k + 4
        while rest > 0 and at < min(4 * k + 8, vocab):
            v = np.float32(rest)
            p[b, 0, at] = v if v <= rest else np.nextafter(v, np.float32(0))
            rest -= float(p[b, 0, at])
            at += 1
        ends.append((4 * k - 1, 4 * k + 4))
    zero = np.zeros((batch, 1), np.int32)
    accept, path, following, err = call(zero, zero - 1, [1] * batch, p, p, np.full((batch, 1), 0.5, np.float32), "picked")
    assert err == 0 and (accept == 1).all() and (path == 0).all()
    missed = [(b, int(x)) for b, (x, e) in enumerate(zip(following, ends)) if x not in e]
    assert not missed, (len(missed), missed[:5])


@pytest.mark.gpu
def test_many_rejected_siblings_leave_the_token_that_the_target_prefers():
    """Token 20 has the only p above q, and up to 40 drafts of others are rejected: the residual is token 20's, smaller each time,
    down to less than half a step of p and to nothing, where p counts and u_0 = 1/4 is token 20's again."""
    rng = np.random.default_rng(16)
    vocab, n = 64, 41
    counts = np.tile(np.arange(2, n + 1), 25)
    batch = len(counts)
    p, q = np.zeros((batch, n, vocab), np.float32), np.zeros((batch, n, vocab), np.float32)
    qx = rng.uniform(0.3, 0.95, batch)
    px = qx * (1 + (1 / qx - 1) * rng.uniform(0.01, 0.99, batch))
    p[:, 0, 20], q[:, 0, 20] = px, qx
    p[:, 0, 41:49], q[:, 0, 41:49] = (1 - px[:, None]) / 8, (1 - qx[:, None]) / 8
    tokens, parents = np.tile(41 + np.arange(n, dtype=np.int32) % 8, (batch, 1)), np.zeros((batch, n), np.int32)
    parents[:, 0] = -1
    u = np.full((batch, n), 1 - 2.0 ** -24, np.float32)
    u[:, 0] = 0.25
    accept, path, following, err = call(tokens, parents, counts, p, q, u, "drawn")
    assert err == 0 and (accept == 1).all() and (path[:, 1:] == -1).all()
    assert (following == 20).all(), sorted(set(zip(following[following != 20].tolist(), counts[following != 20].tolist())))[:8]


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
def test_every_token_has_the_targets_distribution(mode):
    """65535 trees of one kind: how often each pair (first token, second token) follows the root, against the target's
    probabilities, within five standard deviations for each of 36 (a chance of 2 10^-5 in all)."""
    rng = np.random.default_rng(6)
    batch, vocab, n = 65535, 6, 7
    parents = np.tile(np.array([-1, 0, 0, 0, 1, 1, 2], np.int32), (batch, 1))
    q0, p0 = softmax(rng.standard_normal((1 + vocab, vocab))), softmax(rng.standard_normal((1 + vocab, vocab)))

    def children(rows, many):
        if mode == "picked":
            return np.argsort(-rows, 1)[:, :many]
        if mode == "distinct":
            return np.argsort(-(np.log(rows) + rng.gumbel(size=rows.shape)), 1)[:, :many]
        return np.stack([(rng.random((len(rows), 1)) > rows.astype(np.float64).cumsum(1)[:, :-1]).sum(1) for _ in range(many)], 1)

    tokens = np.zeros((batch, n), np.int32)
    tokens[:, 1:4] = children(np.tile(q0[:1], (batch, 1)), 3)
    tokens[:, 4:6] = children(q0[1 + tokens[:, 1]], 2)
    tokens[:, 6] = children(q0[1 + tokens[:, 2]], 1)[:, 0]
    rows = np.concatenate([np.zeros((batch, 1), int), 1 + tokens[:, 1:]], 1)      # a node's distribution goes by its token
    u = rng.random((batch, n)).astype(np.float32)
    accept, path, following, err = call(tokens, parents, [n] * batch, p0[rows], q0[rows], u, mode)
    assert err == 0
    b = np.arange(batch)
    first = np.where(accept > 1, tokens[b, path[:, 1]], following)
    # where the walk ended at the root, the second token is drawn here
    own = (rng.random((batch, 1)) > p0[1 + first].astype(np.float64).cumsum(1)[:, :-1]).sum(1)
    second = np.where(accept > 2, tokens[b, path[:, 2]], np.where(accept == 2, following, own))
    for x in range(vocab):
        for y in range(vocab):
            want = float(p0[0, x]) * float(p0[1 + x, y])
            got = ((first == x) & (second == y)).mean()
            assert abs(got - want) <= 5 * math.sqrt(want / batch) + 1e-5, (x, y)
    assert 1.2 < accept.mean() < 3


@pytest.mark.gpu
def test_rows_that_no_walk_needs_are_not_looked_at():
    """A chain whose third node is rejected: all rows but the one it hangs on, and the tokens' own places, are NaN."""
    rng = np.random.default_rng(7)
    tokens, parents, p, q, u = make(rng, 1, 8, 900, "drawn", 1)
    u[:, 1:3], u[:, 3] = 0.0, 1.0 - 2.0 ** -24
    p[0, 2, tokens[0, 3]] = 1e-9
    want, token = walk(tokens[0], parents[0], 8, p[0], q[0], u[0], False)
    assert want == [0, 1, 2]
    for row in (0, 1, 3, 4, 5, 6, 7):
        keep = [tokens[0, row + 1]] if row < 7 else []
        for x in (p, q):
            values = x[0, row, keep].copy()
            x[0, row] = math.nan
            x[0, row, keep] = values
    accept, path, following, err = call(tokens, parents, [8], p, q, u, "drawn")
    assert err == 0 and path[0, :accept[0]].tolist() == want and following[0] == token


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
def test_values_that_weigh_nothing(mode):
    """Infinities, NaN and negative values of the rows where a walk ends: as if they were zero."""
    rng = np.random.default_rng(8)
    tokens, parents, p, q, u = make(rng, 6, 4, 3001, mode, 2)
    clean = p.copy()
    free = [x for x in range(3001) if x not in tokens]
    spots = rng.choice(free, 40, replace=False)
    clean[:, :, spots] = 0.0
    p[:, :, spots] = rng.choice([math.inf, -math.inf, math.nan, -1.0], 40).astype(np.float32)
    want = call(tokens, parents, [4] * 6, clean, q, u, mode)
    got = call(tokens, parents, [4] * 6, p, q, u, mode)
    assert all(np.array_equal(a, b) for a, b in zip(want, got))


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("vocab", [1000, 3001])
def test_probabilities_that_are_none_count_as_zero(vocab, mode):
    """Infinities, NaN and negative values in either's rows, of drafted tokens too: the walk of the rows with zeros there."""
    rng = np.random.default_rng(vocab)
    batch, n = 60, 7
    tokens, parents, p, q, u = make(rng, batch, n, vocab, mode, 4)
    u[:, 1:] = np.maximum(u[:, 1:], rng.random((batch, n - 1)).astype(np.float32))      # more rejections, and so more sums
    odd = np.array([math.inf, -math.inf, math.nan, -1.0, -1e-3, -0.0], np.float32)
    clean = [p.copy(), q.copy()]
    for x, c in zip((p, q), clean):
        spots = rng.random(x.shape) < 0.05
        for b in range(batch):
            for i in range(1, n):
                spots[b, parents[b, i], tokens[b, i]] = rng.random() < 0.3
        c[spots] = 0.0
        x[spots] = rng.choice(odd, spots.sum())
    want = call(tokens, parents, [n] * batch, *clean, u, mode)
    got = call(tokens, parents, [n] * batch, p, q, u, mode)
    assert want[3] == 0 and all(np.array_equal(a, b) for a, b in zip(want, got))
    check(tokens, parents, [n] * batch, *clean, u, mode)


@pytest.mark.gpu
def test_what_cannot_be_is_reported():
    rng = np.random.default_rng(9)
    tokens, parents, p, q, u = make(rng, 5, 6, 50, "drawn", 2)
    bad = tokens.copy()
    bad[0, 1], bad[1, 2] = 50, -3                       # not kept
    u[0] = u[1] = 0.0
    accept, path, following, err = call(bad, parents, [6] * 5, p, q, u, "drawn")
    assert err == _lib.DEVERR_TOKEN and 1 not in path[0] and 2 not in path[1] and ((0 <= following) & (following < 50)).all()
    bad = tokens.copy()
    bad[:, 0] = 10 ** 9                                 # the root's is not looked at
    assert call(bad, parents, [6] * 5, p, q, u, "drawn")[3] == 0
    zero = p.copy()
    zero[2] = 0.0
    accept, path, following, err = call(tokens, parents, [6] * 5, zero, q, u, "drawn")
    assert err == _lib.DEVERR_TOKEN and accept[2] == 1 and following[2] == 0
    twisted = parents.copy()
    twisted[3, 0], twisted[4, 2] = 0, 4
    got = call(tokens, twisted, [6, 6, 6, 6, 6], p, q, u, "drawn")
    want = call(tokens, np.where(np.arange(6) == 2, np.where(np.arange(5)[:, None] == 4, -1, parents), parents), [6] * 5, p, q, u, "drawn")
    assert got[3] == _lib.DEVERR_TREE and want[3] == 0 and all(np.array_equal(a, b) for a, b in zip(got[:3], want[:3]))
    got, want = call(tokens, parents, [7, -1, 6, 6, 6], p, q, u, "drawn"), call(tokens, parents, [6, 0, 6, 6, 6], p, q, u, "drawn")
    assert got[3] == _lib.DEVERR_TREE and all(np.array_equal(a, b) for a, b in zip(got[:3], want[:3]))


@pytest.mark.gpu
def test_a_draft_with_more_rows_and_odd_addresses():
    """Rows that begin 4 bytes past a 16-byte boundary, and a draft with rows for leaves too: the same answers."""
    rng = np.random.default_rng(10)
    batch, n, vocab = 7, 9, 5000
    tokens, parents, p, q, u = make(rng, batch, n, vocab, "drawn", 3)
    want = call(tokens, parents, [n] * batch, p, q, u, "drawn")
    less = call(tokens, parents, [n] * batch, p, np.ascontiguousarray(q[:, :n - 1]), u, "drawn")
    part = torch.from_numpy(q).cuda()[:, :n - 1]        # a part of a tensor with more rows
    out = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((batch,), (batch, n), (batch,))]
    P.tree_sample(i32(tokens), i32(parents), i32([n] * batch), torch.from_numpy(p).cuda(), part, torch.from_numpy(u).cuda(), *out)
    assert not part.is_contiguous() and all(np.array_equal(a, b.cpu().numpy()) for a, b in zip(want, out))
    room = torch.zeros(batch * n * vocab + 1, device="cuda")[1:]
    room.copy_(torch.from_numpy(p).cuda().flatten())
    out = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((batch,), (batch, n), (batch,))]
    P.tree_sample(i32(tokens), i32(parents), i32([n] * batch), room.view(batch, n, vocab), torch.from_numpy(q).cuda(), torch.from_numpy(u).cuda(), *out)
    assert all(np.array_equal(a, b) and np.array_equal(a, c.cpu().numpy()) for a, b, c in zip(want, less, out))


@pytest.mark.gpu
def test_rows_past_32_bit_offsets():
    """Probabilities of 18 GB: the last sequences' rows lie behind 2^32 elements. Rows that no walk visits are left as they come."""
    rng = np.random.default_rng(12)
    batch, n, vocab = 41, 500, 220000
    target, draft = (torch.empty((batch, n, vocab), device="cuda") for _ in range(2))
    assert target[:-1].numel() > 2 ** 32
    tokens, parents, p, q, u = make(rng, 1, 4, vocab, "drawn", 1)
    wide = lambda x, fill: np.concatenate([np.tile(x, (batch, 1)), np.full((batch, n - 4), fill, x.dtype)], 1)     # noqa: E731
    for b in (0, 39, 40):
        target[b, :4], draft[b, :4] = torch.from_numpy(p[0]).cuda(), torch.from_numpy(q[0]).cuda()
    counts = np.zeros(batch, np.int32)
    counts[[0, 39, 40]] = 4
    out = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((batch,), (batch, n), (batch,))]
    P.tree_sample(i32(wide(tokens, 0)), i32(wide(parents, -1)), i32(counts), target, draft, torch.from_numpy(wide(u, 0.5)).cuda(), *out)
    want, token = walk(tokens[0], parents[0], 4, p[0], q[0], u[0], False)
    for b in (0, 39, 40):
        assert out[1][b, :int(out[0][b])].tolist() == want and int(out[2][b]) == token


@pytest.mark.gpu
def test_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(11)
    batch, n, vocab = 5, 12, 30000
    data = [make(rng, batch, n, vocab, "distinct", 3) for _ in range(3)]
    dev = [[i32(t), i32(par), torch.from_numpy(p).cuda(), torch.from_numpy(q).cuda(), torch.from_numpy(u).cuda()] for t, par, p, q, u in data]
    want = [call(t, par, [n] * batch, p, q, u, "distinct") for t, par, p, q, u in data]
    counts = i32([n] * batch)
    now = [x.clone() for x in dev[0]]
    new = lambda: [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((batch,), (batch, n), (batch,))]     # noqa: E731
    out, other = new(), new()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    P.tree_sample(now[0], now[1], counts, now[2], now[3], now[4], *other, distinct=True, stream=side)
    side.synchronize()
    assert all(np.array_equal(a, b.cpu().numpy()) for a, b in zip(want[0], other))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.tree_sample(now[0], now[1], counts, now[2], now[3], now[4], *out, distinct=True)
    for k in (2, 1, 0):
        for a, b in zip(now, dev[k]):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(a, b.cpu().numpy()) for a, b in zip(want[k], out))


def test_whichever_cta_gives_up_the_tree_has_no_result():
    """A wait among a tree's CTAs may give up in one of them and not in the others, which then store a walk and a token. No call makes a
    wait give up, so this reads the source: every CTA stores its results, then arrives at the cluster's last barrier; those that
    gave up wait there for all of them, and then store that there is no result, whatever their rank."""
    import os
    import re
    src = open(os.path.join(os.path.dirname(P.__file__), "csrc", "tree_sample.cu")).read()
    src = re.sub(r"//[^\n]*", "", src)
    end = src[src.index("const bool gave_up"):src.index("constexpr int kTreeCost")]
    results, last = end[:end.index("cluster_arrive();")], end[end.index("cluster_arrive();"):]
    assert "if (rank == 0 && !gave_up)" in results and "a.accept_len[b] = steps;" in results and "cluster_wait" not in results
    after = last[last.index("if (gave_up) {"):]
    assert "steps" not in last and "rank" not in last and last.index("cluster_arrive();") < last.index("if (gave_up) {")
    where = [after.index(x) for x in ("cluster_wait();", "DFLARE_DEVERR_TIMEOUT", "a.accept_len[b] = 0;", "a.next_token[b] = -1;", "a.path[")]
    assert where == sorted(where)


# ------------------------------------------------------------------------------------------ refusals (host)

@pytest.fixture(scope="module")
def raw():
    from paper_2606_02091_gb300 import build
    build.build()
    return _lib.load()


def test_bad_arguments_are_refused(raw):
    good = [FAKE, FAKE, FAKE, FAKE, FAKE, 4, FAKE, 2, 5, 100, 0, FAKE, FAKE, FAKE, None, None]
    for i, v in ((0, None), (1, None), (2, None), (3, None), (6, None), (11, None), (12, None), (13, None), (5, 3), (7, 0), (7, 65536), (8, 0),
                 (8, 1025), (9, 0), (9, (1 << 28) + 1), (10, 2), (10, -1)):
        bad = list(good)
        bad[i] = v
        assert raw.dflare_tree_sample(*bad) == _lib.DFLARE_EINVAL, i


def test_the_binding_keeps_to_one_device_and_refuses_wrong_tensors(monkeypatch):
    from paper_2606_02091_gb300 import paged
    lib = Taken()
    monkeypatch.setattr(_lib, "load", lambda: lib)
    monkeypatch.setattr(paged, "_device", lambda: 0)
    monkeypatch.setattr(paged, "_raw_stream", lambda device: 1000 + device)
    shapes = dict(tokens=((2, 3), "int32"), parents=((2, 3), "int32"), n_nodes=((2,), "int32"), target=((2, 3, 50), "float32"),
                  draft=((2, 2, 50), "float32"), u=((2, 3), "float32"), accept_len=((2,), "int32"), path=((2, 3), "int32"),
                  next_token=((2,), "int32"), error=((1,), "int32"))
    good = {x: there(*y, 0) for x, y in shapes.items()}
    P.tree_sample(**good)
    P.tree_sample(**dict(good, draft=None), distinct=True, stream=SimpleNamespace(device_index=0, cuda_stream=77))
    assert [a[-1] for _, a in lib.calls] == [1000, 77] and lib.calls[1][1][4:6] == (None, 0) and lib.calls[0][1][10] == 0 and lib.calls[1][1][10] == 1
    with pytest.raises(ValueError, match="stream"):
        P.tree_sample(**good, stream=SimpleNamespace(device_index=1, cuda_stream=77))
    for x, (shape, dtype) in shapes.items():
        with pytest.raises(ValueError, match="cuda:0"):
            P.tree_sample(**dict(good, **{x: there(shape, dtype, 1)}))
        with pytest.raises(ValueError):
            P.tree_sample(**dict(good, **{x: there(shape, "float64", 0)}))
        if x not in ("n_nodes", "error"):
            with pytest.raises(ValueError):
                P.tree_sample(**dict(good, **{x: there((1,) * len(shape), dtype, 0)}))
    for x, shape in (("target", (2, 3, 49)), ("draft", (2, 2, 49)), ("draft", (3, 2, 50)), ("u", (2, 4))):
        with pytest.raises(ValueError):
            P.tree_sample(**dict(good, **{x: there(shape, "float32", 0)}))
    part = there((2, 2, 50), "float32", 0)
    for strides, fits in (((150, 50, 1), True), ((120, 50, 1), False), ((150, 75, 1), False), ((100, 1, 2), False)):
        part._plain = torch.empty(900, device="meta").as_strided((2, 2, 50), strides)
        if fits:
            P.tree_sample(**dict(good, draft=part))
            assert lib.calls.pop()[1][5] == 3
        else:
            with pytest.raises(ValueError, match="rows"):
                P.tree_sample(**dict(good, draft=part))
    assert len(lib.calls) == 2
