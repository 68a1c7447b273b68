// How the paged attention divides its work, shared by its kernels.
//
// The query rows of one kv head are n * G (row r: node r / G, query head r % G of the group), cut into
// groups of QT rows. For one group index qg the work is the list of all (sequence, kv head) pairs that have
// such rows, each with ceil(keys / KT) key tiles; C CTAs take equal runs of that list, wherever they begin
// and end, so contexts of any lengths load the CTAs evenly. The CTAs of different qg with the same place in
// the list are neighbours in the grid: they read the same keys at about the same time, once from HBM.
// Rows whose keys lie in one run are written by that CTA; rows whose keys several CTAs read leave partial
// results (at most two per CTA: of the pair it begins in and of the pair it ends in) that a second launch
// joins in a fixed order.
#pragma once
#include "common.cuh"
#include "paged.h"

namespace dfl {

// tiles up to sequence b (exclusive), per query group; behind them the run length and the lengths
struct TreePlan {
    int32_t* cum;       // [QG][batch + 1]
    int32_t* per;       // [QG]
};
__host__ __device__ inline size_t tree_plan_ints(int QG, int batch) { return (size_t)QG * (batch + 2); }
__device__ __forceinline__ TreePlan tree_plan_of(const TreeArgs& a) { return {a.plan, a.plan + (size_t)a.QG * (a.batch + 1)}; }

// keys of sequence b that exist: its tokens and its nodes, as far as its pages reach
__device__ __forceinline__ void tree_lengths(const TreeArgs& a, int b, int& n, int& ctx, int& keys) {
    n = min(max(a.n_nodes[b], 0), a.n_max);
    const long long room = (long long)min(max(a.pg.held[b], 0), a.pg.max_pages) * a.pg.ps;
    ctx = max(a.pg.lens[b], 0);
    keys = (int)min((long long)ctx + n, room);
    ctx = min(ctx, keys);
}

// The run [t0, t1) of this CTA, and cum[0 .. batch] (tiles of one kv head before sequence b) in shared
// memory. All threads of the CTA call it; it ends with a barrier. The first CTA of each group writes the
// division down for the joining launch.
template <int QT, int KT, int MIN>
__device__ __forceinline__ void tree_runs(const TreeArgs& a, int qg, int c, int32_t* cum, int& t0, int& t1) {
    const int tid = threadIdx.x;
    if (tid < 32) {
        int base = 0;
        for (int b0 = 0; b0 < a.batch; b0 += 32) {
            const int b = b0 + tid;
            int tiles = 0;
            if (b < a.batch) {
                int n, ctx, keys;
                tree_lengths(a, b, n, ctx, keys);
                if (n * a.G > qg * QT) tiles = (int)(((long long)keys + KT - 1) / KT);
            }
            int v = tiles;
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
    const int total = cum[a.batch] * a.pg.hkv;
    // a run below MIN tiles costs more in joining than it saves
    const int per = max((total + a.C - 1) / a.C, MIN);
    t0 = (int)min((long long)c * per, (long long)total);
    t1 = (int)min((long long)t0 + per, (long long)total);
    if (c == 0) {
        const TreePlan p = tree_plan_of(a);
        for (int b = tid; b <= a.batch; b += blockDim.x) p.cum[(size_t)qg * (a.batch + 1) + b] = cum[b];
        if (tid == 0) p.per[qg] = per;
    }
}

// The (sequence, kv head) pair that tile t of the list belongs to.
struct TreeItem {
    int b, h;        // sequence, kv head
    int start;       // its first tile in the list
    int tiles;
};
__device__ __forceinline__ TreeItem tree_item(const int32_t* cum, int batch, int hkv, int t) {
    int lo = 0, hi = batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cum[mid] * hkv <= t) lo = mid; else hi = mid;
    }
    TreeItem it;
    it.b = lo;
    it.tiles = cum[lo + 1] - cum[lo];
    const int in = t - cum[lo] * hkv;
    it.h = in / it.tiles;
    it.start = cum[lo] * hkv + it.h * it.tiles;
    return it;
}

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

}  // namespace dfl
