"""The norm of query and key heads with the rotary positions in the same pass, forward, backward and on the way into the
pages of a cache, against a plain implementation in 64 bits, and its refusals."""
import ctypes
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2606_02091_gb300 as P
from paper_2606_02091_gb300 import _lib
from tests.test_tree_verify import EPS16, EPS32, FAKE, Paged, Taken, frequencies, host, i32, there, turn

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------ plain forms

def forward(x, gain, pos, inv, layout, magnitude, eps):
    """float64 [rows][heads][hd]; and what of it fp32 arithmetic may miss."""
    hd = x.shape[-1]
    r = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    z = x * r * gain
    y = turn(z, pos, inv, layout, magnitude)
    # hd products and sums under a root, the root, a division, two products: (hd / 2 + 8) eps of z. Cosines and
    # sines and their two products and sum: 8 eps of both elements of a pair; the plain angle's own rounding.
    bound = (hd / 2 + 8) * EPS32 * np.abs(z)
    if len(inv):
        both = pairs(np.abs(z), inv, layout)
        bound[..., :2 * len(inv)] = magnitude * both * ((hd / 2 + 16) * EPS32 + np.abs(pos).max() * 2.0 ** -51)
    return y, bound


def yarn(rot, theta, factor, trained=4096, fast=32.0, slow=1.0):
    """Frequencies by the turns of each pair within the trained positions, pairs counted past the head's at both ends
    (rot 6 has three, and the mix of the last two ends at the fifth), and the factor on the values."""
    j = np.arange(-4 * rot, 4 * rot)
    turns = trained * theta ** (-2.0 * j / rot) / (2 * math.pi)
    lo, hi = j[turns >= fast].max(), j[turns <= slow].min()
    j = np.arange(rot // 2)
    inv, mix = theta ** (-2.0 * j / rot), np.clip((j - lo) / (hi - lo), 0, 1)
    return inv * (1 - mix) + inv / factor * mix, 0.1 * math.log(factor) + 1.0


def pairs(v, inv, layout):
    """The sum of each pair, at both of its places."""
    h = len(inv)
    i, j = (slice(0, h), slice(h, 2 * h)) if layout == "half" else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
    out = np.empty(v.shape[:-1] + (2 * h,))
    out[..., i] = out[..., j] = v[..., i] + v[..., j]
    return out


def backward(x, dy, gain, pos, inv, layout, magnitude, eps):
    """dx and the gain's gradient in 64 bits, and their bounds."""
    hd = x.shape[-1]
    r = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    dz = turn(dy, pos, inv, layout, magnitude, -1.0)
    ez = np.zeros(x.shape)
    if len(inv):
        ez[..., :2 * len(inv)] = magnitude * pairs(np.abs(dy), inv, layout) * (8 * EPS32 + np.abs(pos).max() * 2.0 ** -51)
    a = dz * gain
    dx = r * (a - x * r ** 2 * (a * x).mean(-1, keepdims=True))
    mean = np.abs(a * x).mean(-1, keepdims=True)
    # r by (hd / 2 + 6) eps, three times; the mean by hd eps; a handful of products
    bound = r * ((np.abs(a) + np.abs(x) * r ** 2 * mean) * (2.5 * hd + 32) * EPS32 + np.abs(gain) * ez
                 + np.abs(x) * r ** 2 * (np.abs(gain * x) * ez).mean(-1, keepdims=True))
    terms = np.abs(dz * x * r)
    many = x.shape[0] * x.shape[1]
    dgain_bound = terms.sum((0, 1)) * (many + hd / 2 + 10) * EPS32 + (ez * np.abs(x) * r).sum((0, 1))
    return dx, (dz * x * r).sum((0, 1)), bound, dgain_bound


def within(got, want, bound, dtype):
    off, allowed = np.abs(host(got) - want), bound + (EPS16 * 1.01 * (np.abs(want) + bound) if dtype == "bf16" else 0) + 1e-37
    assert not (off > allowed).any(), (off - allowed).max()


CASES = [
    # rows, hq, hkv, hd, rot, layout, start, eps
    (1, 1, 1, 16, 16, "half", 0, 1e-6),
    (1, 32, 8, 128, 128, "half", 70000, 1e-6),
    (7, 5, 3, 128, 64, "half", 100000, 1e-5),
    (33, 9, 2, 64, 32, "interleaved", 5, 1e-6),
    (12, 4, 4, 96, 96, "interleaved", 900000, 1e-6),    # six of a head's eight threads
    (12, 4, 1, 256, 0, "half", 0, 1e-6),                # no rotation
    (5, 3, 2, 512, 256, "half", 9, 0.0),
    (2500, 32, 8, 128, 128, "half", 3, 1e-6),           # several heads of a row per thread
    (1201, 15, 5, 64, 64, "interleaved", 3, 1e-6),
    (6, 3, 2, 80, 20, "half", 77, 1e-6),                # no multiples of 16
    (300, 3, 2, 10, 6, "interleaved", 77, 1e-6),
    (4, 2, 1, 7, 4, "half", 3, 1e-6),                   # an odd head
    (9, 2, 1, 1024, 64, "half", 3, 1e-6),
    (5, 2, 1, 2, 2, "half", 3, 1e-6),
]


def inputs(rng, rows, hq, hkv, hd, dtype):
    """q and k as parts of a projection's rows, gains, the gradients of the results."""
    t = TYPES[dtype]
    make = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(t).cuda()     # noqa: E731
    qkv = make(rows, hq + 2 * hkv, hd)
    return (qkv[:, :hq], qkv[:, hq:hq + hkv], (1 + 0.2 * make(hd)).to(t), (1 + 0.2 * make(hd)).to(t), make(rows, hq, hd), make(rows, hkv, hd))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,hq,hkv,hd,rot,layout,start,eps", CASES)
def test_both_directions_match_the_definition(rows, hq, hkv, hd, rot, layout, start, eps, dtype):
    rng = np.random.default_rng(rows * hd + rot)
    t = TYPES[dtype]
    q, k, qg, kg, dq, dk = inputs(rng, rows, hq, hkv, hd, dtype)
    pos = start + rng.integers(0, 50, rows)
    pos[0] = -pos[0]
    inv, magnitude = yarn(rot, 1e4, 4.0) if rot > 2 else (np.ones(rot // 2), 1.0)
    phase, m = P.rope_phases(rot, 1e4, "yarn" if rot > 2 else "none", 4.0) if rot else (None, 1.0)
    at = i32(pos) if rot else None
    magnitude = magnitude if rot else 1.0
    new = lambda h: torch.full((rows, h, hd), 7.0, dtype=t, device="cuda")     # noqa: E731
    qo, ko = new(hq), new(hkv)
    P.qk_norm_rope(q, k, at, phase, qg, kg, qo, ko, eps=eps, layout=layout, magnitude=m)
    for x, g, y in ((q, qg, qo), (k, kg, ko)):
        want, bound = forward(host(x), host(g), pos, inv, layout, magnitude, eps)
        within(y, want, bound, dtype)
    # the queries alone, in place, and [heads][rows] order: the same bits
    q2, turned = q.clone(), torch.zeros((hq, rows, hd), dtype=t, device="cuda").transpose(0, 1)
    P.qk_norm_rope(q2, None, at, phase, qg, None, q2, None, eps=eps, layout=layout, magnitude=m)
    P.qk_norm_rope(q, None, at, phase, qg, None, turned, None, eps=eps, layout=layout, magnitude=m)
    assert torch.equal(q2, qo) and torch.equal(turned, qo)

    dqo, dko, work = new(hq), new(hkv), P.qk_norm_rope_work(hd).fill_(math.nan)
    dqg, dkg = (torch.full((hd,), math.nan, device="cuda") for _ in range(2))
    P.qk_norm_rope_backward(q, k, dq, dk, at, phase, qg, kg, dqo, dko, dqg, dkg, work, eps=eps, layout=layout, magnitude=m)
    for x, dy, g, dx, dg in ((q, dq, qg, dqo, dqg), (k, dk, kg, dko, dkg)):
        want, want_gain, bound, gain_bound = backward(host(x), host(dy), host(g), pos, inv, layout, magnitude, eps)
        within(dx, want, bound, dtype)
        assert np.all(np.abs(host(dg) - want_gain) <= gain_bound + 1e-37)
    # again, in place of the results' gradients: the same bits, the gains' gradients among them
    a, b, gains = dq.clone(), dk.clone(), [torch.zeros(hd, device="cuda") for _ in range(2)]
    P.qk_norm_rope_backward(q, k, a, b, at, phase, qg, kg, a, b, *gains, work, eps=eps, layout=layout, magnitude=m)
    assert torch.equal(a, dqo) and torch.equal(b, dko) and torch.equal(gains[0], dqg) and torch.equal(gains[1], dkg)
    a = dq.clone()
    P.qk_norm_rope_backward(q, None, a, None, at, phase, qg, None, a, None, gains[0], None, work, eps=eps, layout=layout, magnitude=m)
    assert torch.equal(a, dqo)
    assert np.all(np.abs(host(gains[0]) - host(dqg)) <= 2 * backward(host(q), host(dq), host(qg), pos, inv, layout, magnitude, eps)[3] + 1e-37)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_backward_is_the_limit_of_differences(layout):
    """Along random directions, against differences of the plain forward map in 64 bits: these are off by h^2 of the third
    derivative (below 10 for inputs of size 1) and 2^-52 / h of the sum."""
    rng = np.random.default_rng(5)
    rows, hq, hkv, hd, rot, eps, h = 6, 3, 2, 32, 16, 1e-3, 1e-5
    q, k, qg, kg, dq, dk = inputs(rng, rows, hq, hkv, hd, "f32")
    pos = rng.integers(0, 5000, rows)
    inv, phase = frequencies(rot, 1e4)[0], P.rope_phases(rot, 1e4)[0]
    dx, dy, dg, dkg = (torch.zeros(x.shape, device="cuda") for x in (q, k, qg, kg))
    P.qk_norm_rope_backward(q, k, dq, dk, i32(pos), phase, qg, kg, dx, dy, dg, dkg, P.qk_norm_rope_work(hd), eps=eps, layout=layout)
    for x, gain, up, got, got_gain in ((q, qg, dq, dx, dg), (k, kg, dk, dy, dkg)):
        x, gain, up = host(x), host(gain), host(up)
        f = lambda x, gain: (forward(x, gain, pos, inv, layout, 1.0, eps)[0] * up).sum()     # noqa: E731
        bound, gain_bound = backward(x, up, gain, pos, inv, layout, 1.0, eps)[2:]
        for _ in range(4):
            d, e = rng.standard_normal(x.shape), rng.standard_normal(gain.shape)
            slack = x.size * (10 * h * h + 2.0 ** -52 / h * 16)
            assert abs((f(x + h * d, gain) - f(x - h * d, gain)) / (2 * h) - (host(got) * d).sum()) <= (bound * np.abs(d)).sum() + slack
            assert abs((f(x, gain + h * e) - f(x, gain - h * e)) / (2 * h) - (host(got_gain) * e).sum()) <= (gain_bound * np.abs(e)).sum() + slack


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_beside_the_call_stay_and_odd_values_stay_in_their_heads(dtype):
    """Results into the middle of wider rows; a head of infinities, one of NaN and one of zeros do not reach others."""
    rng = np.random.default_rng(8)
    q, _, qg, _, dq, _ = inputs(rng, 9, 6, 1, 64, dtype)
    q = q.clone()
    phase, pos = P.rope_phases(32, 1e4)[0], i32(range(9))
    clean, wide = torch.zeros_like(q), torch.full((9, 10, 64), 7.0, dtype=q.dtype, device="cuda")
    P.qk_norm_rope(q, None, pos, phase, qg, None, clean, None)
    q[2, 1], q[2, 3], q[4, 0] = math.inf, math.nan, 0.0
    P.qk_norm_rope(q, None, pos, phase, qg, None, wide[:, 2:8], None)
    got = wide[:, 2:8]
    keep = torch.ones((9, 6), dtype=torch.bool, device="cuda")
    keep[2, 1] = keep[2, 3] = keep[4, 0] = False
    assert torch.equal(got[keep], clean[keep]) and not got[4, 0].any() and got[2, 3].isnan().all()
    assert (wide[:, :2] == 7).all() and (wide[:, 8:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset,row", [(1, 0), (0, 3), (4, 5)])
def test_odd_addresses_and_strides(offset, row, dtype):
    """Heads that begin off a 16-byte boundary, or rows an odd number of elements apart, of everything a call reads and writes."""
    rng = np.random.default_rng(offset + row)
    rows, heads, hd, t = 37, 3, 64, TYPES[dtype]
    pos, phase, inv = rng.integers(0, 900, rows), P.rope_phases(32, 1e4)[0], frequencies(32, 1e4)[0]
    gain = (1 + 0.2 * torch.from_numpy(rng.standard_normal(hd).astype(np.float32)).to(t)).cuda()

    def odd():
        wide = torch.from_numpy(rng.standard_normal(rows * (heads * hd + row) + offset).astype(np.float32)).to(t).cuda()
        return wide[offset:].view(rows, heads * hd + row)[:, :heads * hd].view(rows, heads, hd)

    x, dy, out, dx = odd(), odd(), odd(), odd()
    P.qk_norm_rope(x, None, i32(pos), phase, gain, None, out, None)
    want, bound = forward(host(x), host(gain), pos, inv, "half", 1.0, 1e-6)
    within(out, want, bound, dtype)
    dg = torch.zeros(hd, device="cuda")
    P.qk_norm_rope_backward(x, None, dy, None, i32(pos), phase, gain, None, dx, None, dg, None, P.qk_norm_rope_work(hd))
    want, want_gain, bound, gain_bound = backward(host(x), host(dy), host(gain), pos, inv, "half", 1.0, 1e-6)
    within(dx, want, bound, dtype)
    assert np.all(np.abs(host(dg) - want_gain) <= gain_bound)


@pytest.mark.gpu
def test_a_broadcast_input_and_gradient():
    """A row stride of zero: the same head for every row, its gradients one after another."""
    rng = np.random.default_rng(9)
    q, _, qg, _, dq, _ = inputs(rng, 1, 4, 1, 64, "f32")
    rows = 40
    x, dy, out = q.expand(rows, 4, 64), dq.expand(rows, 4, 64), torch.zeros((rows, 4, 64), device="cuda")
    phase, pos, work, dg = P.rope_phases(64, 1e4)[0], rng.integers(0, 99, rows), P.qk_norm_rope_work(64), torch.zeros(64, device="cuda")
    P.qk_norm_rope_backward(x, None, dy, None, i32(pos), phase, qg, None, out, None, dg, None, work)
    want, gain, bound, gain_bound = backward(np.array(host(x)), np.array(host(dy)), host(qg), pos, frequencies(64, 1e4)[0], "half", 1.0, 1e-6)
    within(out, want, bound, "f32")
    assert np.all(np.abs(host(dg) - gain) <= gain_bound)


@pytest.mark.gpu
def test_rows_past_32_bit_offsets():
    """4.6 GB of heads: the last rows against the same rows in a call of their own, and a wide stride between few rows."""
    rows, hq, hd = 450000, 40, 128
    x = torch.randn((rows, hq, hd), dtype=torch.bfloat16, device="cuda")
    assert x[:-99].numel() > 2 ** 31
    gain, phase, pos = torch.ones(hd, dtype=torch.bfloat16, device="cuda"), P.rope_phases(hd, 1e4)[0], torch.arange(rows, dtype=torch.int32, device="cuda")
    out, few = torch.empty_like(x), torch.empty_like(x[:99])
    P.qk_norm_rope(x, None, pos, phase, gain, None, out, None)
    P.qk_norm_rope(x[-99:], None, pos[-99:].contiguous(), phase, gain, None, few, None)
    assert torch.equal(out[-99:], few)
    far = x[::150000][:, :2]        # rows 768 million elements apart
    three, want = torch.zeros((3, 2, hd), dtype=x.dtype, device="cuda"), torch.zeros((3, 2, hd), dtype=x.dtype, device="cuda")
    P.qk_norm_rope(far, None, pos[:3], phase, gain, None, three, None)
    P.qk_norm_rope(far.contiguous(), None, pos[:3], phase, gain, None, want, None)
    assert far.stride(0) == 150000 * hq * hd and torch.equal(three, want)


@pytest.mark.gpu
def test_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(10)
    q, k, qg, kg, dq, dk = inputs(rng, 700, 8, 2, 64, "bf16")
    phase, pos, work = P.rope_phases(64, 1e4)[0], i32(range(700)), P.qk_norm_rope_work(64)

    def buffers():
        return [torch.zeros_like(x.contiguous()) for x in (q, k, q, k)] + [torch.zeros(64, device="cuda") for _ in range(2)]

    def step(o, work, stream=None):
        P.qk_norm_rope(q, k, pos, phase, qg, kg, o[0], o[1], stream=stream)
        P.qk_norm_rope_backward(q, k, dq, dk, pos, phase, qg, kg, o[2], o[3], o[4], o[5], work, stream=stream)

    plain, other, graphed = buffers(), buffers(), buffers()
    step(plain, work)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step(other, P.qk_norm_rope_work(64), side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(graphed, work)
    for x in graphed:
        x.zero_()
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(plain, other, graphed))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,rot,layout,depths", [(64, 64, "half", True), (128, 32, "interleaved", True), (64, 20, "half", False), (128, 0, "half", False)])
def test_append_norms_and_writes_the_pages(hd, rot, layout, depths, dtype):
    rng = np.random.default_rng(rot + hd)
    lens, counts = [0, 15, 16, 40], [5, 3, 0, 9]
    p = Paged(rng, lens, counts, hq=6, hkv=2, hd=hd, page=16, dtype=dtype, layers=2)
    n = 9
    make = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(p.t).cuda()     # noqa: E731
    qkv, qg, kg = make(4, n, 10, hd), (1 + 0.2 * make(hd)).to(p.t), (1 + 0.2 * make(hd)).to(p.t)
    q, k, v = qkv[:, :, :6], qkv[:, :, 6:8], qkv[:, :, 8:]
    depth = np.stack([np.arange(n) // 2 for _ in lens])
    out = torch.full((4, n, 6, hd), 7.0, dtype=p.t, device="cuda")
    kw, vw = host(p.k), host(p.v)
    bound = np.zeros(kw.shape)
    phase, inv = (P.rope_phases(rot, 1e4)[0], frequencies(rot, 1e4)[0]) if rot else (None, np.zeros(0))
    kws = dict(depth=i32(depth) if depths else None, layout=layout, q_gain=qg, k_gain=kg, eps=1e-5)
    p.cache.append(1, q, k, v, i32(counts), phase, out, **kws)
    assert p.cache.error() == 0
    for b, c in enumerate(counts):
        if not c:
            continue
        pos = lens[b] + (depth[b, :c] if depths else np.arange(c))
        want, off = forward(host(q)[b, :c], host(qg), pos, inv, layout, 1.0, 1e-5)
        within(out[b, :c], want, off, dtype)
        keys, off = forward(host(k)[b, :c], host(kg), pos, inv, layout, 1.0, 1e-5)
        for i in range(c):
            page, at = p.table[b, (lens[b] + i) // 16], (lens[b] + i) % 16
            kw[1, page, :, at], vw[1, page, :, at], bound[1, page, :, at] = keys[i], host(v)[b, i], off[i]
    for b, c in enumerate(counts):
        assert (host(out)[b, c:] == 7.0).all()
    got = host(p.k)
    assert np.array_equal(host(p.v), vw, equal_nan=True) and np.array_equal(np.isnan(got), np.isnan(kw))
    limit = bound * (1 + EPS16) + (EPS16 * 1.01 * np.abs(kw) if dtype == "bf16" else 0)
    limit[0] = 0
    same = np.isnan(kw) | (np.abs(got - kw) <= np.where(bound > 0, limit, 0))
    assert same.all()
    # keys and values alone, in the other layer: the same bits
    p.cache.append(0, None, k, v, i32(counts), phase, None, **dict(kws, q_gain=None))
    for b, c in enumerate(counts):
        for i in range(c):
            page, at = p.table[b, (lens[b] + i) // 16], (lens[b] + i) % 16
            assert torch.equal(p.k[0, page, :, at], p.k[1, page, :, at]) and torch.equal(p.v[0, page, :, at], p.v[1, page, :, at])


@pytest.mark.gpu
def test_a_normed_append_beyond_the_pages_is_left_out():
    rng = np.random.default_rng(1)
    p = Paged(rng, [20], [4], hq=2, hkv=1, hd=64, page=16, dtype="bf16")
    p.cache.lens.copy_(i32([30]))
    x = torch.from_numpy(rng.standard_normal((1, 4, 2, 64)).astype(np.float32)).to(p.t).cuda()
    k0, out, one = p.k.clone(), torch.zeros_like(x), torch.ones(64, dtype=p.t, device="cuda")
    p.cache.append(0, x, x[:, :, :1], x[:, :, 1:], i32([4]), None, out, q_gain=one, k_gain=one)
    assert p.cache.error() == _lib.DEVERR_CAPACITY
    wrote = [(p.table[0, 1], 14), (p.table[0, 1], 15)]
    for page, at in wrote:
        k0[0, page, :, at] = p.k[0, page, :, at]
    assert torch.equal(k0.nan_to_num(9.0), p.k.nan_to_num(9.0)) and out.abs().sum(-1).min() > 0


# ------------------------------------------------------------------------------------------ refusals (host)

@pytest.fixture(scope="module")
def raw():
    from paper_2606_02091_gb300 import build
    build.build()
    return _lib.load()


def heads(**kw):
    base = dict(x=256, x_row=512, x_head=64, dy=4096, dy_row=512, dy_head=64, out=8192, out_row=512, out_head=64, gain=256, dgain=256, heads=8)
    base.update(kw)
    return _lib.QkHeads(**base)


def test_the_struct_follows_the_header():
    import os
    import re
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dflare.h")).read()
    assert _lib.QK_NORM_WORK_ROWS == int(re.search(r"DFLARE_QK_NORM_WORK_ROWS (\d+)", src).group(1))
    body = re.search(r"typedef struct \{([^}]*)\}\s*dflare_qk_heads;", re.sub(r"/\*.*?\*/", "", src, flags=re.S)).group(1)
    assert re.findall(r"(\w+)\s*[;,]", body) == [f for f, _ in _lib.QkHeads._fields_]


def test_bad_arguments_are_refused(raw):
    E, ref = _lib.DFLARE_EINVAL, ctypes.byref
    good = [ref(heads()), ref(heads()), FAKE, FAKE, 4, 64, 64, 0, 1.0, 1e-6, 0, None]
    for i, v in ((0, None), (2, None), (3, None), (4, 0), (4, (1 << 24) + 1), (5, 1), (5, 1025), (6, 3), (6, 66), (6, -2), (7, 2), (8, math.inf),
                 (9, -1.0), (9, math.nan), (10, 2)):
        bad = list(good)
        bad[i] = v
        assert raw.dflare_qk_norm_rope(*bad) == E, i
        assert raw.dflare_qk_norm_rope_backward(*bad[:10], FAKE, *bad[10:]) == E, i
    assert raw.dflare_qk_norm_rope_backward(*good[:10], None, *good[10:]) == E
    for kw in (dict(heads=0), dict(heads=4097), dict(x=None), dict(out=None), dict(gain=None), dict(x_row=-1), dict(x_head=-64), dict(out_row=32),
               dict(out_head=32), dict(out=256, out_row=1024)):
        for i in (0, 1):
            bad = list(good)
            bad[i] = ref(heads(**kw))
            assert raw.dflare_qk_norm_rope(*bad) == E, kw
    for kw in (dict(dy=None), dict(dgain=None), dict(dy_row=-1), dict(dy=8192, dy_row=1024)):
        bad = list(good)
        bad[0] = ref(heads(**kw))
        assert raw.dflare_qk_norm_rope_backward(*bad[:10], FAKE, *bad[10:]) == E, kw
    bad = list(good)
    bad[0], bad[4] = ref(heads(heads=4096, out_row=4096 * 64)), 1 << 24
    assert raw.dflare_qk_norm_rope(*bad) == E
    assert raw.dflare_cache_append_normed(None, 0, None, 0, FAKE, 64, FAKE, 64, None, 0, None, FAKE, 1e-6, None, FAKE, 1, 1, None, 0, 0, 1.0, None) == E


@pytest.mark.parametrize("rows,n,row,head", [(4, 2, 64, 64), (4, 2, 64, 128), (4, 2, 127, 64), (4, 2, 64, 255), (2, 3, 191, 64), (1 << 24, 4096, 4096, 64)])
def test_results_that_overlap_are_refused(raw, rows, n, row, head):
    # (4 rows span 3 * 64 + 64 = 256 elements, 2 heads 128, 3 heads 192)
    for i in (0, 1):
        args = [ctypes.byref(heads()), ctypes.byref(heads()), FAKE, FAKE, rows, 64, 64, 0, 1.0, 1e-6, 0, None]
        args[i] = ctypes.byref(heads(heads=n, out_row=row, out_head=head))
        assert raw.dflare_qk_norm_rope(*args) == _lib.DFLARE_EINVAL
        assert b"overlap" in raw.dflare_last_error(None)
        assert raw.dflare_qk_norm_rope_backward(*args[:10], FAKE, *args[10:]) == _lib.DFLARE_EINVAL


def test_results_of_queries_and_keys_that_overlap_are_refused(raw):
    """Both are worked on at the same time: a place that is written for one is nothing of the other's, and a gain that both share has
    two gradients."""
    key = dict(x=1 << 20, dy=2 << 20, out=3 << 20, dgain=4096)

    def said(q, k, backward):
        args = [ctypes.byref(heads(**q)), ctypes.byref(heads(**dict(key, **k))), FAKE, FAKE, 4, 64, 64, 0, 1.0, 1e-6, 0, None]
        call = raw.dflare_qk_norm_rope_backward if backward else raw.dflare_qk_norm_rope
        # (without a workspace the backward call is refused, but for what is asked before that)
        assert call(*(args[:10] + [None] + args[10:] if backward else args)) == _lib.DFLARE_EINVAL
        return raw.dflare_last_error(None)

    for q, k in (({}, dict(out=8192)), ({}, dict(x=8192)), (dict(x=3 << 20), {})):
        for backward in (False, True):
            assert b"overlap" in said(q, k, backward), (q, k)
    for q, k in (({}, dict(dy=8192)), (dict(dy=3 << 20), {}), ({}, dict(dgain=256)), ({}, dict(dgain=256 + 252)), (dict(dgain=4096 + 252), {})):
        assert b"overlap" in said(q, k, True), (q, k)
    # parts of one projection's rows, in place, and gradients side by side
    for q, k in (({}, {}), (dict(x=1 << 16, out=1 << 16), dict(x=(1 << 16) + 128, out=(1 << 16) + 128)), ({}, dict(dgain=256 + 256))):
        assert b"NULL" in said(q, k, True), (q, k)


def test_the_binding_keeps_to_one_device_and_refuses_wrong_tensors(monkeypatch):
    from paper_2606_02091_gb300 import paged
    lib = Taken()
    monkeypatch.setattr(_lib, "load", lambda: lib)
    monkeypatch.setattr(paged, "_device", lambda: 0)
    monkeypatch.setattr(paged, "_raw_stream", lambda device: 1000 + device)
    c = object.__new__(P.PagedCache)
    c.__dict__.update(_cache=ctypes.c_void_p(), _L=lib, device_index=1, n_layers=1, n_pages=8, n_kv_heads=2, page_size=16, head_dim=64,
                      max_batch=2, max_pages=3, n_q_heads=4, max_nodes=8, dtype=torch.bfloat16)
    b = "bfloat16"
    q, k, g = ((6, 4, 64), b), ((6, 2, 64), b), ((64,), b)
    gain32, pos, phase = ((64,), "float32"), ((6,), "int32"), ((32,), "int64")
    both = dict(q=q, k=k, positions=pos, phase=phase, q_gain=g, k_gain=g)
    calls = {
        "forward": (dict(both, q_out=q, k_out=k), lambda t, s: P.qk_norm_rope(**t, stream=s), 0),
        "backward": (dict(both, dq_out=q, dk_out=k, dq=q, dk=k, dq_gain=gain32, dk_gain=gain32, work=((_lib.QK_NORM_WORK_ROWS * 64,), "float32")),
                     lambda t, s: P.qk_norm_rope_backward(**t, stream=s), 0),
        "append": (dict(q=((2, 3, 4, 64), b), k=((2, 3, 2, 64), b), v=((2, 3, 2, 64), b), n_new=((2,), "int32"), phase=phase, q_out=((2, 3, 4, 64), b),
                        depth=((2, 3), "int32"), q_gain=g, k_gain=g), lambda t, s: c.append(0, **t, stream=s), 1),
    }
    for name, (shapes, call, home) in calls.items():
        before = len(lib.calls)
        good = {x: there(*y, home) for x, y in shapes.items()}
        call(good, None)
        call(good, SimpleNamespace(device_index=home, cuda_stream=77))
        assert [a[-1] for _, a in lib.calls[before:]] == [1000 + home, 77], name
        assert lib.calls[-1][0] == {"forward": "dflare_qk_norm_rope", "backward": "dflare_qk_norm_rope_backward", "append": "dflare_cache_append_normed"}[name]
        with pytest.raises(ValueError, match="stream"):
            call(good, SimpleNamespace(device_index=1 - home, cuda_stream=77))
        for away, (shape, dtype) in shapes.items():
            with pytest.raises(ValueError, match=f"cuda:{home}"):
                call(dict(good, **{away: there(shape, dtype, 1 - home)}), None)
            with pytest.raises(ValueError):
                call(dict(good, **{away: there(shape, "float64", home)}), None)
            if away != "phase":     # (a shorter one turns fewer elements)
                with pytest.raises(ValueError):
                    call(dict(good, **{away: there((1,) * len(shape), dtype, home)}), None)
        assert len(lib.calls) == before + 2
    shapes, call, _ = calls["append"]
    good = {x: there(*y, 1) for x, y in shapes.items()}
    for gone in (dict(k_gain=None), dict(q_gain=None)):
        with pytest.raises(ValueError, match="gain"):
            call(dict(good, **gone), None)
    good = {x: there(*y, 0) for x, y in calls["forward"][0].items()}
    for gone in (dict(positions=None), dict(phase=None)):
        with pytest.raises(ValueError, match="go together"):
            calls["forward"][1](dict(good, **gone), None)
