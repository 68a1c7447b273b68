"""Speculative decoding with drafted trees, from the drafter to the target's cache.

A small target model with random weights keeps its keys and values in a PagedCache. A DFlare drafter proposes a block
of tokens; every position's second choice hangs beside its first one, which makes a tree. One pass of the target over
the tree's nodes (rotary positions, pages, tree attention per layer) gives its choice after each of them; the walk
along those choices is accepted, its rows move together in the cache, and the accepted positions' hidden states go
back to the drafter. The prompt is read once and forked into several sequences, which then go on from different
tokens. Run:

    python examples/tree_verify.py

It prints the accepted lengths and checks the tokens against plain decoding, one token at a time.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_02091_gb300 import DFlare, PagedCache, rope_phases, tree_accept, tree_plan  # noqa: E402

D, LAYERS, HQ, HKV, HD, FFN, VOCAB, BLOCK = 256, 3, 8, 2, 64, 512, 512, 6
PAGE, PAGES, MAX_LEN = 16, 128, 256


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def norm(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


class Target:
    """A decoder with random fp32 weights whose attention runs on the paged cache."""

    def __init__(self, batch, max_nodes, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape, scale=1.0):
            return torch.randn(shape, device="cuda", generator=g) * scale

        self.embed = w(VOCAB, D)
        self.qkv = w(LAYERS, (HQ + 2 * HKV) * HD, D, scale=2.0 * D ** -0.5)
        self.o = w(LAYERS, D, HQ * HD, scale=(HQ * HD) ** -0.5)
        self.up, self.down = w(LAYERS, FFN, D, scale=D ** -0.5), w(LAYERS, D, FFN, scale=FFN ** -0.5)
        self.phase, self.magnitude = rope_phases(HD, theta=1e4)
        self.cache = PagedCache.allocate(n_layers=LAYERS, n_pages=PAGES, page_size=PAGE, n_q_heads=HQ, n_kv_heads=HKV, head_dim=HD,
                                         max_batch=batch, max_pages=MAX_LEN // PAGE, max_nodes=max_nodes, dtype="f32")

    def forward(self, tokens, n_nodes, depth=None, mask=None):
        """tokens [batch][n] behind every sequence's cache -> logits [batch][n][VOCAB], hidden [LAYERS][batch][n][D]."""
        batch, n = tokens.shape
        x = self.embed[tokens.long()]
        hidden = []
        self.cache.reserve(n_nodes)
        for i in range(LAYERS):
            qkv = (norm(x) @ self.qkv[i].T).view(batch, n, HQ + 2 * HKV, HD)
            q, k, v = qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HKV], qkv[:, :, HQ + HKV:]
            self.cache.append(i, q, k, v, n_nodes, self.phase, q, depth=depth, magnitude=self.magnitude)
            out = torch.empty((batch, n, HQ, HD), device="cuda")
            self.cache.attend(i, q, n_nodes, out, mask=mask)
            x = x + out.view(batch, n, -1) @ self.o[i].T
            x = x + torch.nn.functional.silu(norm(x) @ self.up[i].T) @ self.down[i].T
            hidden.append(x)
        return norm(x) @ self.embed.T, torch.stack(hidden)


class Drafter:
    """A DFlare drafter of two layers with random weights, beside the target's embedding."""

    def __init__(self, target, batch, rows, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dq, dkv = HQ * HD, HKV * HD

        def w(*shape):
            return 0.02 * torch.randn(shape, device="cuda", generator=g)

        self.lib = DFlare(d=D, n_draft_layers=2, n_target_layers=LAYERS, n_q_heads=HQ, n_kv_heads=HKV, head_dim=HD, ffn=FFN,
                          vocab=VOCAB, block=BLOCK, max_batch=batch, max_ctx=MAX_LEN, max_fuse_rows=rows, dtype="f32")
        ones = torch.ones((2, D), device="cuda")
        self.lib.set_weights(dict(fuse_logits=w(2, LAYERS), fuse_norm=ones, w_kv_ctx=w(2, 2 * dkv, D), attn_norm=ones,
                                  w_qkv=w(2, dq + 2 * dkv, D), w_o=w(2, D, dq), mlp_norm=ones, w_gate=w(2, FFN, D), w_up=w(2, FFN, D),
                                  w_down=w(2, D, FFN), final_norm=ones[0].clone(), embed=target.embed, lm_head=target.embed))
        self.lib.reset(batch)
        self.tokens = torch.zeros((batch, BLOCK - 1), dtype=torch.int32, device="cuda")
        self.logits = torch.zeros((batch, BLOCK - 1, VOCAB), device="cuda")

    def draft(self, last):
        """The two best tokens of every position, [batch][BLOCK - 1][2]."""
        self.lib.draft_block(last, self.tokens, self.logits)
        return self.logits.topk(2, -1).indices.int()


def comb(batch):
    """The tree of every step: node 0, then two nodes per position, both below the position's first one before."""
    parents = [-1]
    for k in range(1, BLOCK):
        parents += [0 if k == 1 else 2 * k - 3] * 2
    return ints([parents] * batch)


def decode(prompt, firsts, steps, plant=0.0, seed=0):
    """Greedy decoding of `steps` tree steps from one prompt, one sequence for every token of `firsts` behind it. With
    probability `plant` a position's second choice is replaced by the token that the target will choose (found by
    plain decoding), so that the walk through the tree has branches to take. Returns the sequences' tokens, the same by
    plain decoding, and the accepted lengths."""
    batch, nodes = len(firsts), 2 * BLOCK - 1
    plain = plain_decode(prompt, firsts, steps * BLOCK, seed)
    target = Target(batch, max(nodes, len(prompt)), seed)
    drafter = Drafter(target, batch, batch * max(len(prompt), BLOCK))
    cache = target.cache
    # the prompt once, in sequence 0, then forked
    n = ints([len(prompt)] + [0] * (batch - 1))
    tokens = ints([prompt] + [[0] * len(prompt)] * (batch - 1))
    _, hidden = target.forward(tokens, n)
    cache.commit(n, torch.arange(len(prompt), dtype=torch.int32, device="cuda").repeat(batch, 1))
    if batch > 1:
        cache.fork(ints([0] * (batch - 1)), ints(list(range(1, batch))))
    drafter.lib.fuse_context(hidden[:, :1].repeat(1, batch, 1, 1), ints([len(prompt)] * batch))

    parents, count = comb(batch), ints([nodes] * batch)
    mask = torch.zeros((batch, nodes, (nodes + 31) // 32), dtype=torch.int32, device="cuda")
    depth, path = torch.zeros((batch, nodes), dtype=torch.int32, device="cuda"), torch.zeros((batch, nodes), dtype=torch.int32, device="cuda")
    accept, last = ints([0] * batch), ints(firsts)
    coin = torch.Generator().manual_seed(seed)
    out, lengths = [[f] for f in firsts], []
    tree_plan(parents, count, mask, depth)
    for _ in range(steps):
        pairs = drafter.draft(last)
        if plant:
            for b in range(batch):
                for k in range(BLOCK - 1):
                    if torch.rand((), generator=coin) < plant:
                        want = plain[b][len(out[b]) + k] if len(out[b]) + k < len(plain[b]) else 0
                        pairs[b, k, int(torch.rand((), generator=coin) < 0.5)] = want
        tokens = torch.cat([last[:, None], pairs.flatten(1)], 1).contiguous()
        logits, hidden = target.forward(tokens, count, depth, mask)
        choice = logits.argmax(-1).int()
        tree_accept(tokens, parents, choice, count, accept, path, last)
        cache.commit(accept, path)
        rows = path[:, :BLOCK].long().clamp(min=0)
        accepted = hidden.gather(2, rows[None, :, :, None].expand(LAYERS, batch, BLOCK, D))
        drafter.lib.fuse_context(accepted.contiguous(), accept)
        lengths.append(accept.tolist())
        for b in range(batch):
            out[b] += [int(tokens[b, i]) for i in path[b, 1:lengths[-1][b]].tolist()] + [int(last[b])]
    assert cache.error() == 0 and drafter.lib.device_error() == 0
    return out, plain, lengths


def plain_decode(prompt, firsts, steps, seed=0):
    """The same target, one token at a time, every sequence with its own copy of the prompt."""
    batch = len(firsts)
    target = Target(batch, len(prompt), seed)
    n = ints([len(prompt)] * batch)
    target.forward(ints([prompt] * batch), n)
    target.cache.commit(n, torch.arange(len(prompt), dtype=torch.int32, device="cuda").repeat(batch, 1))
    one, first_row = ints([1] * batch), ints([[0]] * batch)
    tokens, out = ints(firsts)[:, None], [[f] for f in firsts]
    for _ in range(steps):
        logits, _ = target.forward(tokens.contiguous(), one)
        target.cache.commit(one, first_row)
        tokens = logits.argmax(-1).int()
        for b in range(batch):
            out[b].append(int(tokens[b, 0]))
    assert target.cache.error() == 0
    return out


def main():
    prompt = [(7 * i * i + 3) % VOCAB for i in range(37)]
    for plant in (0.0, 0.7):
        out, plain, lengths = decode(prompt, [5, 6, 7], 12, plant)
        same = all(o == p[:len(o)] for o, p in zip(out, plain))
        print("second choices planted with probability %.1f: accepted lengths %s; tokens as by plain decoding: %s" % (plant, lengths, same))
        if not same:
            raise SystemExit(1)


if __name__ == "__main__":
    main()
