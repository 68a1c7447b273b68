// How the paged attention divides its work, shared by its kernels.
//
// The query rows of one kv head are n * G (row r: node r / G, query head r % G of the group), cut into
// groups of QT rows. For one group index qg the work is the list of all (sequence, kv head) pairs that have
// such rows, each with ceil(keys / KT) key tiles; the group's CTAs take equal runs of that list, wherever they
// begin and end, so contexts of any lengths load the CTAs evenly. A pair counts EXTRA tiles beyond its own for
// what beginning and ending it costs. The groups share the CTAs in proportion to their lists (trees of a batch
// differ, and so does the number of sequences that reach a group); groups with equal lists read the same keys at
// about the same time, once from HBM.
// Rows whose keys lie in one run are written by that CTA; rows whose keys several CTAs read leave partial
// results (at most two per CTA: of the pair it begins in and of the pair it ends in) that a second launch
// joins in a fixed order.
#pragma once
#include "common.cuh"
#include "paged.h"
#include "umma.cuh"

namespace dfl {

// 2^x, relative error about 2^-22; 2^-inf = 0
__device__ __forceinline__ float pow2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}

// What memory says of sequence b, and what follows: nodes, tokens, and keys that exist (tokens and nodes as
// far as the sequence's pages reach). In two steps, so that the loads can be under way long before their use.
struct TreeRaw {
    int n, held, len;
};
__device__ __forceinline__ TreeRaw tree_raw(const TreeArgs& a, int b) { return {a.n_nodes[b], a.pg.held[b], a.pg.lens[b]}; }
__device__ __forceinline__ void tree_lengths(const TreeArgs& a, const TreeRaw& x, int& n, int& ctx, int& keys) {
    n = min(max(x.n, 0), a.n_max);
    const long long room = (long long)min(max(x.held, 0), a.pg.max_pages) * a.pg.ps;
    ctx = max(x.len, 0);
    keys = (int)min((long long)ctx + n, room);
    ctx = min(ctx, keys);
}

// key tiles of a sequence (0: it has no query rows, or no keys) and its query groups
__device__ __forceinline__ int tree_tiles(const TreeArgs& a, const TreeRaw& raw, int QT, int KT, int& groups) {
    int n, ctx, keys;
    tree_lengths(a, raw, n, ctx, keys);
    const int tiles = n ? (int)(((long long)keys + KT - 1) / KT) : 0;
    groups = tiles ? (n * a.G + QT - 1) / QT : 0;
    return tiles;
}
__device__ __forceinline__ int tree_cost(int tiles, int extra) { return tiles ? tiles + extra : 0; }
// length of a run; below `least` it would cost more in joining than it saves
__device__ __forceinline__ int tree_run(int total, int C, int least) { return max((total + C - 1) / C, least); }

// The groups' lists and their parts of the grid. Up to kShares groups share the CTAs by their lists, one CTA for
// every group that has rows and the others in proportion; more groups share them evenly.
constexpr int kShares = 8;
struct TreeCosts {
    int list[kShares];      // of one kv head
};
// A warp adds up the groups' lists; seq(b, cost, groups) says what sequence b has.
template <class F>
__device__ __forceinline__ TreeCosts tree_costs(const TreeArgs& a, int lane, F seq) {
    TreeCosts c;
#pragma unroll
    for (int g = 0; g < kShares; ++g) c.list[g] = 0;
    for (int b = lane; b < a.batch; b += 32) {
        int cost, groups;
        seq(b, cost, groups);
#pragma unroll
        for (int g = 0; g < kShares; ++g) c.list[g] += groups > g ? cost : 0;
    }
#pragma unroll
    for (int g = 0; g < kShares; ++g) {
        if (g >= a.QG) break;
        c.list[g] = __reduce_add_sync(0xffffffffu, c.list[g]);
    }
    return c;
}
// Lane g of the warp gets group g's first CTA and how many it has (up to kShares groups).
__device__ __forceinline__ void tree_shares(const TreeArgs& a, const TreeCosts& c, int lane, int& first, int& many) {
    float all = 0.f, own = 0.f;
    int some = 0;
#pragma unroll
    for (int g = 0; g < kShares; ++g) {
        if (g >= a.QG) break;
        all += (float)c.list[g];
        some += c.list[g] > 0;
        if (lane == g) own = (float)c.list[g];
    }
    // rounded down with room to spare, so that the parts never add up to more than there is
    many = own > 0.f ? 1 + (int)__fmul_rn(__fmul_rn((float)max(a.C - some, 0), 0.999999f), __fdiv_rn(own, all)) : 0;
    first = many;
#pragma unroll
    for (int o = 1; o < kShares; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, first, o);
        if (lane >= o) first += x;
    }
    first -= many;
}

// The query group of this CTA, its run [v0, v1) of the group's list, and cum[0 .. batch] (cost of one kv head before
// sequence b) in shared memory. All threads of the CTA call it; it ends with a barrier. An empty run: nothing to do.
template <int QT, int KT, int EXTRA, int LEAST>
__device__ __forceinline__ void tree_runs(const TreeArgs& a, int32_t* cum, int& qg, int& v0, int& v1) {
    __shared__ int mine[3];     // group, this CTA's number in it, its CTAs
    const int tid = threadIdx.x;
    if (tid < 32) {
        int cost = 0, groups = 0, g = 0, c = blockIdx.x, C = a.C;       // (cost, groups: of sequence tid)
        if (a.QG > kShares) {
            C = max(a.C / a.QG, 1);
            g = blockIdx.x / C;
            c = blockIdx.x % C;
            if (g >= a.QG) C = 0;
        } else if (a.QG > 1) {
            const TreeCosts costs = tree_costs(a, tid, [&](int b, int& x, int& many) {
                x = tree_cost(tree_tiles(a, tree_raw(a, b), QT, KT, many), EXTRA);
                if (b == tid) {
                    cost = x;
                    groups = many;
                }
            });
            int first, many;
            tree_shares(a, costs, tid, first, many);
            const unsigned here = __ballot_sync(0xffffffffu, (int)blockIdx.x >= first && (int)blockIdx.x < first + many);
            g = here ? __ffs(here) - 1 : 0;
            c -= __shfl_sync(0xffffffffu, first, g);
            C = here ? __shfl_sync(0xffffffffu, many, g) : 0;
        }
        if (tid == 0) {
            mine[0] = g;
            mine[1] = c;
            mine[2] = C;
        }
        int base = 0;
        for (int b0 = 0; b0 < a.batch; b0 += 32) {
            const int b = b0 + tid;
            if (b0 || a.QG == 1 || a.QG > kShares) {
                groups = 0;
                cost = b < a.batch ? tree_cost(tree_tiles(a, tree_raw(a, b), QT, KT, groups), EXTRA) : 0;
            }
            int v = groups > g ? cost : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, v, o);
                if (tid >= o) v += x;
            }
            if (b < a.batch) cum[b + 1] = base + v;
            base += __shfl_sync(0xffffffffu, v, 31);
        }
        if (tid == 0) cum[0] = 0;
    }
    __syncthreads();
    qg = mine[0];
    const int total = mine[2] ? cum[a.batch] * a.pg.hkv : 0, per = tree_run(total, max(mine[2], 1), LEAST);
    v0 = (int)min((long long)mine[1] * per, (long long)total);
    v1 = (int)min((long long)v0 + per, (long long)total);
}

// A run's part of one pair: tiles [lo, hi) of the `tiles` of kv head h of sequence b; the pair's place in the
// list is `start`.
struct TreePair {
    int b, h, start, tiles, lo, hi;
    __device__ __forceinline__ bool partial() const { return lo != 0 || hi != tiles; }
};
// The next part from place v on (v moves behind its pair); false at the end of the run.
template <int EXTRA>
__device__ __forceinline__ bool tree_pair(const TreeArgs& a, const int32_t* cum, int& v, int v1, TreePair& p) {
    const int hkv = a.pg.hkv;
    while (v < v1) {
        int lo = 0, hi = a.batch;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cum[mid] * hkv <= v) lo = mid; else hi = mid;
        }
        const int cost = cum[lo + 1] - cum[lo];
        p.b = lo;
        p.tiles = cost - EXTRA;
        p.h = (v - cum[lo] * hkv) / cost;
        p.start = cum[lo] * hkv + p.h * cost;
        p.lo = v - p.start;
        p.hi = min(v1 - p.start, p.tiles);
        v = p.start + cost;
        if (p.lo < p.tiles) return true;
    }
    return false;
}

// The same from a plan's items: v counts them, cum is not looked at.
template <int EXTRA>
__device__ __forceinline__ bool tree_pair(const TreeArgs& a, const int32_t*, int& v, int v1, TreeItem& p) {
    if (v >= v1) return false;
    const int4* from = reinterpret_cast<const int4*>(a.items + v++);
    int4* to = reinterpret_cast<int4*>(&p);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(TreeItem) / 16); ++i) to[i] = __ldg(from + i);
    return true;
}
// Whether a workspace holds a plan for this call's sizes, and a cache's of this type and these sizes: every number in it then fits.
__device__ __forceinline__ bool plan_fits(const TreeArgs& a) {
    const int4* head = reinterpret_cast<const int4*>(a.head);
    const int4 x = head[0], y = head[1];        // (all of it in one trip)
    return ((x.x ^ a.kind) | (x.y ^ a.batch) | (x.z ^ a.n_max) | (x.w ^ a.pg.max_pages) | (y.x ^ a.pg.hkv) | (y.y ^ a.pg.ps) | (y.z ^ a.G)) == 0;
}
// This CTA's items; false (and reported) where there is no such plan.
__device__ __forceinline__ bool tree_items(const TreeArgs& a, int& v, int& v1) {
    const int2 run = a.runs[blockIdx.x];
    const bool ok = plan_fits(a);
    v = ok ? run.x : 0;
    v1 = ok ? run.y : 0;
    if (!ok && threadIdx.x == 0 && blockIdx.x == 0) atomicOr(a.pg.err, DFLARE_DEVERR_PLAN);
    return ok;
}
// Lengths of a pair: what memory has to say of it, and what follows
__device__ __forceinline__ TreeRaw pair_raw(const TreeArgs& a, const TreePair& p) { return tree_raw(a, p.b); }
__device__ __forceinline__ TreeRaw pair_raw(const TreeArgs&, const TreeItem& p) { return {p.nodes, p.keys, p.ctx}; }
template <bool SHARED>
__device__ __forceinline__ void pair_lengths(const TreeArgs& a, const TreeRaw& x, int& n, int& ctx, int& keys) {
    if constexpr (SHARED) {
        n = x.n;
        keys = x.held;
        ctx = x.len;
    } else {
        tree_lengths(a, x, n, ctx, keys);
    }
}
// the query row of a pair's node, in rows of q
__device__ __forceinline__ size_t query_row(const TreeArgs& a, const TreePair& p, int node) { return (size_t)p.b * a.n_max + node; }
__device__ __forceinline__ size_t query_row(const TreeArgs& a, const TreeItem& p, int node) {
    return (size_t)(p.first >= 0 ? p.first + node : __ldg(a.map + ~p.first + node));
}
// the node that a row's mask goes by (a group's rows have none: all of its keys are context)
__device__ __forceinline__ int mask_node(const TreePair&, int node) { return node; }
__device__ __forceinline__ int mask_node(const TreeItem& p, int node) { return p.first >= 0 ? node : 0; }
__device__ __forceinline__ int first_page(const TreePair&) { return 0; }
__device__ __forceinline__ int first_page(const TreeItem& p) { return p.page0; }

// Bounded wait, inline (a call would keep the compiler from giving a kernel's other threads their registers).
__device__ __forceinline__ bool wait_inline(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* err) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
#pragma unroll 1
    while (true) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*abort_flag) return false;
        if (globaltimer_ns() - t0 > kTimeoutNs) {
            *abort_flag = 1;
            atomicOr(err, DFLARE_DEVERR_TIMEOUT);
            return false;
        }
    }
}

// Pages for the warp that streams tiles by TMA: lane x looks up the page of box x (`rows` tokens, a divisor of the tile)
// from tile `base` of a pair on, so that one trip to the table serves 32 boxes. What memory says is looked at only when
// the boxes are due: the first group's copies would wait for the second's pages. A slot without a page takes a plane of
// the tensor map outside the pool, which reads as zero: boxes past the pages held, and, reported, those of a held page
// whose number does not exist.
struct BoxPage {
    int held, page, at, h;
};
__device__ __forceinline__ BoxPage box_page(const TreeArgs& a, const TreePair& p, int base, int KT, int rows, int lane) {
    const int at = (int)(((unsigned)(base * KT) + (unsigned)(lane * rows)) / (unsigned)a.pg.ps);
    return {a.pg.held[p.b], at < a.pg.max_pages ? a.pg.table[(size_t)p.b * a.pg.max_pages + at] : -1, at, p.h};
}
__device__ __forceinline__ BoxPage box_page(const TreeArgs& a, const TreeItem& p, int base, int KT, int rows, int lane) {
    const int at = (int)(((unsigned)(base * KT) + (unsigned)(lane * rows)) / (unsigned)a.pg.ps);
    return {p.held, at < p.held ? a.pg.table[(size_t)p.b * a.pg.max_pages + p.page0 + at] : -1, at, p.h};
}
__device__ __forceinline__ int box_plane(const TreeArgs& a, const BoxPage& x) {
    if (x.at < x.held && x.page >= 0 && x.page < a.pg.pages) return (a.layer * a.pg.pages + x.page) * a.pg.hkv + x.h;
    if (x.at < x.held) atomicOr(a.pg.err, DFLARE_DEVERR_PAGE);
    return (int)min(0x7fffffffLL, (long long)a.pg.layers * a.pg.pages * a.pg.hkv);
}
// f(first tile, tiles, planes of their boxes) for groups of tiles (of one pair, as many as have 32 boxes) of the run from
// pair p on, in order, while it says true; false if it did not. The whole warp calls this and f. planes: [2][32] in
// shared memory; a group's stay as they are until the warp is through with f for the next group.
template <int EXTRA, class P, class F>
__device__ __forceinline__ bool each_group(const TreeArgs& a, const int32_t* cum, int& v, int v1, P p, int KT, int rows, int lane,
                                           int (*planes)[32], F f) {
    const int many = 32 / (KT / rows);
    int base = p.lo, buf = 0;
    BoxPage found = box_page(a, p, base, KT, rows, lane);
    bool ok = true;
    for (bool more = true; more && ok; buf ^= 1) {
        const int n = min(many, p.hi - base), from = base;
        planes[buf][lane] = box_plane(a, found);
        __syncwarp();
        base += n;
        if (base == p.hi) {
            more = tree_pair<EXTRA>(a, cum, v, v1, p);
            base = p.lo;
        }
        if (more) found = box_page(a, p, base, KT, rows, lane);
        ok = f(from, n, planes[buf]);
    }
    return ok;
}

// Infinite and NaN bf16 values of a 16-byte piece become 0; whether there were any. (An exponent of all ones plus
// its lowest bit carries into the sign's place.)
__device__ __forceinline__ bool drop_odd(uint4& v) {
    auto carry = [](uint32_t w) { return (w & 0x7f807f80u) + 0x00800080u; };
    if (!((carry(v.x) | carry(v.y) | carry(v.z) | carry(v.w)) & 0x80008000u)) return false;
    uint32_t* e = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t c = carry(e[q]);
        e[q] &= (c & 0x8000u ? 0xffff0000u : ~0u) & (c & 0x80000000u ? 0xffffu : ~0u);
    }
    return true;
}

// row / G for the rows of a kv head (below 2^24, as G <= 64): a multiplication by the rounded-up reciprocal
__device__ __forceinline__ int group_of(const TreeArgs& a, int row) { return a.G == 1 ? row : (int)__umulhi((unsigned)row, a.G_inv); }

// 64 bits of a node's mask row from bit x >= 0 on
__device__ __forceinline__ uint64_t mask_bits(const int32_t* row, int words, int x) {
    const int i = x >> 5, s = x & 31;
    const uint32_t w0 = i < words ? (uint32_t)row[i] : 0u, w1 = i + 1 < words ? (uint32_t)row[i + 1] : 0u;
    const uint32_t w2 = s && i + 2 < words ? (uint32_t)row[i + 2] : 0u;
    return (uint64_t)__funnelshift_r(w0, w1, s) | ((uint64_t)__funnelshift_r(w1, w2, s) << 32);
}
__device__ __forceinline__ uint64_t low_bits(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }

// Which of the keys [k0, k0 + 64) node `node` of sequence b sees (bit t: key k0 + t).
__device__ __forceinline__ uint64_t tree_seen(const TreeArgs& a, int b, int node, int ctx, int keys, int k0) {
    const int rel = k0 - ctx;           // tree number of key k0
    uint64_t v = low_bits(-rel);        // the context's keys
    if (a.mask) {
        const int32_t* row = a.mask + ((size_t)b * a.n_max + node) * a.words;
        if (rel >= 0) v = mask_bits(row, a.words, rel);
        else if (rel > -64) v |= mask_bits(row, a.words, 0) << -rel;
    } else {
        v |= low_bits(node + 1 - rel);
    }
    return v & low_bits(keys - k0);
}

// The same for 32 keys with the first four words of the node's mask row held in registers, so that a tile at
// the end of the context does not wait for memory that is busy with keys (more words: read when needed).
struct SeenRow {
    uint32_t w[4];
};
__device__ __forceinline__ SeenRow seen_row(const TreeArgs& a, int b, int node) {
    SeenRow r;
    const int32_t* row = a.mask + ((size_t)b * a.n_max + node) * a.words;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = a.mask && i < a.words ? (uint32_t)row[i] : 0u;
    return r;
}
__device__ __forceinline__ uint32_t seen_word(const TreeArgs& a, const SeenRow& r, int b, int node, int i) {
    uint32_t v = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) v = i == x ? r.w[x] : v;
    if (i >= 4 && i < a.words) v = (uint32_t)a.mask[((size_t)b * a.n_max + node) * a.words + i];
    return v;
}
__device__ __forceinline__ uint32_t low_bits32(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t seen32(const TreeArgs& a, const SeenRow& r, int b, int node, int ctx, int keys, int k0) {
    const int rel = k0 - ctx;
    uint32_t v;
    if (a.mask) v = __funnelshift_r(seen_word(a, r, b, node, rel >> 5), seen_word(a, r, b, node, (rel >> 5) + 1), rel & 31);
    else v = low_bits32(node + 1 - rel);
    return (v | low_bits32(-rel)) & low_bits32(keys - k0);
}

// f(value address) for every node in odd[] (one bit per node) that `node` sees, in the layer's values of kv head h
template <class P, class F>
__device__ __forceinline__ void each_odd(const TreeArgs& a, const uint32_t* odd, const P& p, int node, int ctx, int keys, F f) {
    for (int word = 0; word < a.words; ++word) {
        uint32_t bits = odd[word];
        while (bits) {
            const int key = ctx + word * 32 + __ffs(bits) - 1;
            bits &= bits - 1;
            if (!(tree_seen(a, p.b, node, ctx, keys, key) & 1)) continue;
            const int page = a.pg.table[(size_t)p.b * a.pg.max_pages + first_page(p) + key / a.pg.ps];
            f(((((size_t)a.layer * a.pg.pages + page) * a.pg.hkv + p.h) * a.pg.ps + key % a.pg.ps) * a.pg.hd);
        }
    }
}

}  // namespace dfl
