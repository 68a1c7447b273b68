// Attention of a batch whose sequences share leading pages (samples and beams of one prompt): a shared page's keys are
// read for a block of the group's rows (16 of a kv head by the warp-level and the fp32 kernel, 256 by the tcgen05 one), not for each
// sequence. The blocks of a group run side by side, so that HBM gives a key that L2 can hold once: 16 single tokens over 4096 shared keys, four
// blocks per kv head, read 28.7 MB of DRAM a layer, of which 27.9 are all keys and values, shared and own.
//
// The keys of a row are those that its group shares and the sequence's own, two disjoint sets; with o, m, l the weighted
// values, the maximum (log2 units) and the sum over each,
//   out = (o_s 2^(m_s - M) + o_o 2^(m_o - M)) / (l_s 2^(m_s - M) + l_o 2^(m_o - M)),   M = max(m_s, m_o),
// just as the parts of a row whose keys several CTAs read are joined. So a group's rows against its shared keys are one
// more "sequence" (without a mask: shared pages hold context only), and each sequence keeps the keys behind those.
//
// A plan, made once per step for all layers, lists this work: units (sequence or group, kv head, block of query rows), each
// with what its key tiles cost and what beginning and ending it does. The CTAs take equal runs of the list. A unit that lies in one run is
// one item; others are cut where a run ends. Partial rows lie in the workspace: two blocks per CTA (of the units cut
// at its run's ends), and one row per query row and part for units that are whole but not all of the row's keys.
//
// Which sequences share: neighbours (sequences without nodes left out) are compared page by page, and neighbours are put into
// groups by what that saves: a group of n that shares s pages saves (n - 1) s of them. The best division is found
// exactly, by best(j) = max over i of best(i) + saving(i .. j - 1).
#include <math.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "common.cuh"
#include "paged.h"
#include "tree_sched.cuh"

namespace dfl {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanRuns = 2048;         // CTAs of a call's kernels, at most

// Query rows per kv head of a whole batch up to which the warp-level kernel has them, 16 at a time. Measured over 91 drawn calls, against
// attention without sharing: 0.84 and 0.76 of its time with 16 rows and fewer (two sets, geometric means), 0.83 with up to 32, 0.79
// with 64, 0.78 with 128, and 0.78 with 512, but eight trees of 16 over 8187 shared tokens then take 102 us for 31.
constexpr int kFewRows = 128;
// Costs of the tcgen05 kernel's work.
constexpr int kTileCost = 4, kWideTileCost = 6, kUnitCost = 14;

constexpr int log2_of(int v) { return v > 1 ? 1 + log2_of(v / 2) : 0; }

// What a plan and the launches that follow it agree on, from the call's sizes alone.
struct WorkLists {
    // fp32: one list. bf16: the warp-level kernel's, where rows are few; a list of own keys for it and one of shared keys for the tcgen05
    // kernel, where a sequence's rows fit one block of the first and there are own units for every SM; the tcgen05 kernel's of both. Measured,
    // a layer with one list and with two: single tokens of 132 sequences, 64/8 heads of 64, own 300 keys behind 240 shared ones 65.2 and
    // 34.7 us, of 88 behind 1250 34.6 and 23.1; 64 sequences of four nodes, own 1150 keys behind 32768 154 and 161; two nodes of 27
    // sequences, 28/4 heads (108 own units) 16.3 and 21.9.
    WorkList list[2];           // of own keys, of shared ones (the same, where there is one)
    int many;
};
struct Layout {
    bool ok;                    // everything fits its numbers
    WorkLists work;
    int own_rows, lead_rows;    // rows of one kv head among the whole units' partial results
    int rows0;                  // the first of those
    size_t runs[2], items[2], map, seqs, ml, o, bytes;      // offsets
};
Layout layout_of(const dflare_cache* c, int batch, int n_max) {
    const dflare_cache_config& g = c->cfg;
    const int G = g.n_q_heads / g.n_kv_heads, sms = c->num_sms;
    Layout y{};
    const long long rows = (long long)batch * n_max * G;
    const WorkList f32{log2_of(kFRows), log2_of(kFKeys), f32_ctas_per_sm(g.head_dim) * sms, 1, 1, kFExtra, kFLeast, 0, false};
    const WorkList mma{log2_of(kMmaRows), log2_of(kMmaKeys), 2 * sms, 1, 1, kMmaExtra, mma_least(g.head_dim), 0, false};
    const WorkList tc{8, log2_of(kTcKeys), sms, kTileCost, kWideTileCost, kUnitCost, kWideTileCost, 0, true};
    y.work.many = 1;
    if (g.dtype == DFLARE_F32) {
        y.work.list[0] = y.work.list[1] = f32;
    } else if (rows <= kFewRows) {
        y.work.list[0] = y.work.list[1] = mma;
    } else if (n_max * G <= kMmaRows && (long long)batch * g.n_kv_heads >= sms) {
        y.work.list[0] = mma;
        y.work.list[1] = tc;
        y.work.many = 2;
    } else {
        y.work.list[0] = y.work.list[1] = tc;
    }
    const long long most = 0x7fffffffLL - 4096;
    y.ok = true;
    long long part = 0, units[2];
    for (int l = 0; l < y.work.many; ++l) {
        WorkList& w = y.work.list[l];
        const long long QT = 1LL << w.qt, own = (long long)batch * (((long long)n_max * G + QT - 1) >> w.qt), lead = ((rows + QT - 1) >> w.qt) + batch / 2;
        units[l] = ((y.work.many == 1 || l == 0 ? own : 0) + (l == y.work.many - 1 ? lead : 0)) * g.n_kv_heads;
        const long long cost = (((long long)g.max_pages * g.page_size + (1LL << w.kt) - 1) >> w.kt) * w.weight2 + w.extra;
        if (units[l] * cost > most) y.ok = false;
        w.slot0 = (int)part;
        part += 2LL * w.C * QT;
    }
    if (y.work.many == 1) y.work.list[1] = y.work.list[0];
    const long long own_rows = ((long long)n_max * G + 31) / 32 * 32, lead_rows = (rows / 32 + batch + 1) * 32;
    const long long rows0 = part;
    part += (batch * own_rows + lead_rows) * g.n_kv_heads;
    if (part > most || y.work.list[0].C + (y.work.many > 1 ? y.work.list[1].C : 0) > kPlanRuns) y.ok = false;
    if (!y.ok) return y;
    y.own_rows = (int)own_rows;
    y.lead_rows = (int)lead_rows;
    y.rows0 = (int)rows0;
    auto place = [&](size_t bytes) {
        const size_t at = y.bytes;
        y.bytes += (bytes + 127) / 128 * 128;
        return at;
    };
    place(sizeof(SharedHead));
    y.seqs = place(sizeof(TreeSeq) * batch);
    y.map = place(sizeof(int32_t) * (size_t)batch * n_max);
    for (int l = 0; l < y.work.many; ++l) {
        y.runs[l] = place(sizeof(int2) * y.work.list[l].C);
        y.items[l] = place(sizeof(TreeItem) * (size_t)(units[l] + y.work.list[l].C));
    }
    y.ml = place(sizeof(float2) * (size_t)part);
    y.o = place(sizeof(float) * (size_t)part * g.head_dim);
    return y;
}

struct PlanArgs {
    PagesView pg;
    const int32_t* n_nodes;
    SharedHead* head;
    int kind;
    int2* runs[2];
    TreeItem* items[2];
    int32_t* map;
    TreeSeq* seqs;
    int32_t* groups;            // optional output
    WorkLists work;
    int batch, n_max, G, own_rows, lead_rows, rows0;
};

// Rows among the partial results: blocks of the CTAs, then of whole units the sequences' own, then the groups'.
__device__ __forceinline__ int own_row(const PlanArgs& a, int b) { return a.rows0 + b * a.pg.hkv * a.own_rows; }
__device__ __forceinline__ int lead_row(const PlanArgs& a, int b, int node0) {
    return own_row(a, a.batch) + (int)((long long)node0 * a.G / 32 + b) * 32;
}
__device__ __forceinline__ void lengths_of(const PlanArgs& a, int b, int& n, int& held, int& ctx, int& keys) {
    n = min(max(a.n_nodes[b], 0), a.n_max);
    held = min(max(a.pg.held[b], 0), a.pg.max_pages);
    const long long room = (long long)held * a.pg.ps;
    const int len = max(a.pg.lens[b], 0);
    keys = (int)min((long long)len + n, room);
    ctx = min(len, keys);
}

// The first kMaxSeqs threads, which have a sequence each.
__device__ __forceinline__ void seq_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kMaxSeqs) : "memory"); }
// Inclusive sums over them, of two numbers at once; tmp holds 8 pairs.
__device__ __forceinline__ int2 plan_scan(int2 v, int2* tmp, int2* total) {
    constexpr int W = kMaxSeqs / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
        if (lane >= o) {
            v.x += x;
            v.y += y;
        }
    }
    seq_barrier();
    if (lane == 31) tmp[warp] = v;
    seq_barrier();
    *total = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const int2 t = tmp[w];
        if (w < warp) {
            v.x += t.x;
            v.y += t.y;
        }
        total->x += t.x;
        total->y += t.y;
    }
    return v;
}

// Pages that sequence b and the one before it that has nodes both hold in the same places, full of context (a warp; the same in
// every lane). One trip to memory where that is sequence b - 1 and they are up to 512.
__device__ __forceinline__ int pages_shared(const PlanArgs& a, int b) {
    constexpr int U = 16;
    const int lane = threadIdx.x & 31;
    const int32_t *x = a.pg.table + (size_t)max(b - 1, 0) * a.pg.max_pages, *y = a.pg.table + (size_t)b * a.pg.max_pages;
    int v[U], w[U];
    auto load = [&](int at) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int i = at + k * 32 + lane;
            v[k] = i < a.pg.max_pages ? x[i] : -1;
            w[k] = i < a.pg.max_pages ? y[i] : -1;
        }
    };
    load(0);
    int n, held, ctx, keys, n2, held2, ctx2, keys2, p = -1;
    lengths_of(a, b, n, held, ctx, keys);
    lengths_of(a, max(b - 1, 0), n2, held2, ctx2, keys2);
    for (int top = b - 1; top >= 0 && p < 0; top -= 32) {
        const unsigned has = __ballot_sync(0xffffffffu, top - lane >= 0 && a.n_nodes[max(top - lane, 0)] > 0);
        if (has) p = top - (__ffs(has) - 1);
    }
    if (p < 0 || n == 0) return 0;
    if (p != b - 1) {
        lengths_of(a, p, n2, held2, ctx2, keys2);
        x = a.pg.table + (size_t)p * a.pg.max_pages;
        load(0);
    }
    const int most = min(ctx, ctx2) / a.pg.ps;
    for (int at = 0;;) {       // up to the first that differs
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int i = at + k * 32 + lane;
            const unsigned differ = __ballot_sync(0xffffffffu, i >= most || v[k] != w[k] || v[k] < 0 || v[k] >= a.pg.pages);
            if (differ) return at + k * 32 + __ffs(differ) - 1;
        }
        at += U * 32;
        load(at);
    }
}

// What a group saves of which `many` share `tokens`, in keys, `costs` being the sum of its members' costs: a member's rows leave and
// join one more partial result each, a group is one more unit. Measured with 32/8 heads of 128, a layer over groups of 4
// that share 512 and 1024 tokens, together and apart: 16 groups, single tokens 32.2 and 37.1 us together, 43.2 and 59.3 apart; trees
// of 16 nodes 52.9 and 59.0, 49.7 and 63.4; 4 groups, trees of 16 19.2 and 22.0, 17.4 and 20.8; 8 groups of 2 over 128 tokens, single
// tokens 14.3 and 13.2, over 256 14.2 and 14.7.
constexpr float kGroupCost = 128.f, kMemberCost = 16.f, kRowCost = 8.f;
__device__ __forceinline__ float saving(float many, float tokens, float costs) { return fmaxf(fmaf(many - 1.f, tokens, -(costs + kGroupCost)), 0.f); }

// The places s .. e - 1 are one group that shares `pages`, or one by itself (a warp).
struct Groups {
    int *first, *members, *pages;       // by place: of its group, the first place, how many (at the first), what they share
    __device__ __forceinline__ void put(int s, int e, int shared) const {
        const int lane = threadIdx.x & 31;
        for (int i = s + lane; i < e; i += 32) {
            first[i] = s;
            pages[i] = e - s > 1 ? shared : 0;
        }
        if (lane == 0) members[s] = e - s;
    }
};
// Sequences s .. e - 1 (by place) of which all neighbours share the same number of pages: all are one group, or none are.
// (False: that is not so, as neighbours share differently or a member costs more than it saves.) costs: sums of what the places
// before each cost.
__device__ __forceinline__ bool divide_even(const int* share, const int* costs, int s, int e, int ps, const Groups& groups) {
    const int lane = threadIdx.x & 31;
    int low = 0x7fffffff, high = 0, dear = 0;
    for (int i = s + lane; i < e; i += 32) {
        if (i > s) {
            low = min(low, share[i]);
            high = max(high, share[i]);
        }
        dear = max(dear, costs[i + 1] - costs[i]);
    }
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    dear = __reduce_max_sync(0xffffffffu, dear);
    const float tokens = (float)low * (float)ps;
    if (e - s > 1 && (low != high || (float)dear >= tokens)) return false;
    if (e - s > 1 && saving((float)(e - s), tokens, (float)(costs[e] - costs[s])) > 0.f) {
        groups.put(s, e, low);
    } else {
        for (int i = s + lane; i < e; i += 32) {
            groups.first[i] = i;
            groups.pages[i] = 0;
        }
    }
    return true;
}
// The same where they differ, up to 32: a warp finds the best division, lane i holding best(i).
__device__ __forceinline__ void divide_few(const int* share, const int* costs, int s, int e, int ps, const Groups& groups) {
    const int lane = threadIdx.x & 31, many = e - s;
    const int before = costs[min(s + lane, e)], upto = costs[min(s + lane + 1, e)];
    const int mine = lane < many ? share[s + lane] : 0;
    const float tokens = (float)mine * (float)ps;
    float best = 0.f, size = (float)-lane, least_f = INFINITY;      // size: of the group that begins here
    int least = 0x7fffffff, from = 0, pages = 0;
    for (int j = 1; j <= many; ++j) {
        size += 1.f;
        const int next = __shfl_sync(0xffffffffu, mine, j - 1);
        const float next_f = __shfl_sync(0xffffffffu, tokens, j - 1);
        if (lane < j - 1) {
            least = min(least, next);
            least_f = fminf(least_f, next_f);
        }
        const float spent = (float)(__shfl_sync(0xffffffffu, upto, j - 1) - before);
        const float v = best + (lane < j - 1 ? saving(size, least_f, spent) : 0.f);
        // (not negative: their bits are in order; of equal ones the shortest group)
        const unsigned bits = lane < j ? __float_as_uint(v) + 1u : 0u, top = __reduce_max_sync(0xffffffffu, bits);
        const int at = 31 - __clz(__ballot_sync(0xffffffffu, bits == top));
        const int shared = __shfl_sync(0xffffffffu, least, at);
        if (lane == j - 1) {
            from = at;
            pages = shared;
        }
        if (lane == j) best = __uint_as_float(top - 1u);
    }
    for (int j = many; j > 0;) {
        const int at = __shfl_sync(0xffffffffu, from, j - 1), shared = __shfl_sync(0xffffffffu, pages, j - 1);
        groups.put(s + at, s + j, shared);
        j = at;
    }
}
// The same for more, with best (e - s + 1 numbers), from and shared_by (e - s each, by place) in shared memory: lane l looks at
// groups that begin at l, l + 32, ...
__device__ __forceinline__ void divide_many(const int* share, const int* costs, int s, int e, int ps, const Groups& groups, float* best, int* from, int* shared_by) {
    const int lane = threadIdx.x & 31, many = e - s;
    int least[kMaxSeqs / 32];
#pragma unroll
    for (int k = 0; k < kMaxSeqs / 32; ++k) least[k] = 0x7fffffff;
    if (lane == 0) best[0] = 0.f;
    __syncwarp();
    for (int j = 1; j <= many; ++j) {
        float top = -1.f;
        int at = 0, pages = 0;
        const int next = share[s + j - 1];
#pragma unroll
        for (int k = 0; k < kMaxSeqs / 32; ++k) {
            const int i = lane + 32 * k;
            if (32 * k >= j) break;
            if (i < j - 1) least[k] = min(least[k], next);
            if (i < j) {
                const float v = best[i] + (i < j - 1 ? saving((float)(j - i), (float)least[k] * (float)ps, (float)(costs[s + j] - costs[s + i])) : 0.f);
                if (v > top) {
                    top = v;
                    at = i;
                    pages = least[k];
                }
            }
        }
        const unsigned bits = top < 0.f ? 0u : __float_as_uint(top) + 1u, most = __reduce_max_sync(0xffffffffu, bits);
        const int last = __reduce_max_sync(0xffffffffu, bits == most ? at : -1);
        if (bits == most && at == last) {
            best[j] = top;
            from[j - 1] = at;
            shared_by[j - 1] = pages;
        }
        __syncwarp();
    }
    for (int j = many; j > 0; j = from[j - 1]) groups.put(s + from[j - 1], s + j, shared_by[j - 1]);
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A cluster with a warp for every sequence, which finds what it shares with the one before it; the first CTA goes on from there.
// Segments: sequence b's own keys, and the keys shared by the group that b leads; one after the other in one list of work, or in a
// list each (place_of).
__global__ void __launch_bounds__(kPlanThreads) tree_shared_plan_kernel(const __grid_constant__ PlanArgs a) {
    __shared__ int same[kMaxSeqs];
    __shared__ int share[kMaxSeqs], costs[kMaxSeqs + 1], begins[kMaxSeqs + 1], from[kMaxSeqs], shared_by[kMaxSeqs], active[kMaxSeqs];
    __shared__ float best[2 * kMaxSeqs];
    __shared__ int group_first[kMaxSeqs], group_members[kMaxSeqs], group_pages[kMaxSeqs];       // by place
    __shared__ int pages_of[kMaxSeqs], node0[kMaxSeqs + 1], nodes_of[kMaxSeqs];                 // by sequence
    __shared__ int n_of[kMaxSeqs], held_of[kMaxSeqs], ctx_of[kMaxSeqs], keys_of[kMaxSeqs];
    __shared__ int seg_start[2 * kMaxSeqs], seg_unit[2 * kMaxSeqs], seg_tiles[2 * kMaxSeqs], seg_blocks[2 * kMaxSeqs], seg_weight[2 * kMaxSeqs];
    __shared__ int2 tmp[kMaxSeqs / 32];
    __shared__ int total_cost[2], total_units[2];       // of the lists
    auto place_of = [&](int b, int which) { return a.work.many == 1 ? 2 * b + which : which * kMaxSeqs + b; };
    __shared__ int first_of[kPlanRuns], last_of[kPlanRuns];        // of the runs of both lists: units
    const bool alone = gridDim.x == 1;
    if (!alone) cluster_arrive();       // (every CTA of the cluster has begun before one writes to another)
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = cluster_rank();
    int n = 0, held = 0, ctx = 0, keys = 0;
    if (tid < a.batch && rank == 0) lengths_of(a, tid, n, held, ctx, keys);
    for (int x = tid; x < kPlanRuns; x += kPlanThreads) {
        first_of[x] = 0x7fffffff;
        last_of[x] = -1;
    }
    const int b0 = (int)rank * (kPlanThreads / 32) + warp, found = b0 < a.batch ? pages_shared(a, b0) : 0;
    if (alone) {
        if (lane == 0 && b0 < a.batch) same[b0] = found;
        __syncthreads();
    } else {
        cluster_wait();
        if (lane == 0 && b0 < a.batch) {
            uint32_t at;
            asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(same + b0)));
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(found) : "memory");
        }
        cluster_arrive();
        cluster_wait();
        if (rank != 0) return;
    }
    if (tid < kMaxSeqs) {       // a thread for every sequence, up to the list of segments
        int2 total;
        if (tid < a.batch) {
            n_of[tid] = n;
            held_of[tid] = held;
            ctx_of[tid] = ctx;
            keys_of[tid] = keys;
        }
        // the sequences that have nodes, in order of their places, and those that share nothing with the one before
        const bool begin = n > 0 && same[tid] == 0;
        const int2 at = plan_scan(make_int2(n > 0, begin), tmp, &total);
        const int place = at.x - 1, m = total.x, runs = total.y;
        const int cost_upto = plan_scan(make_int2(n > 0 ? (int)kMemberCost + (int)kRowCost * n * a.G : 0, 0), tmp, &total).x;
        if (n > 0) {
            active[place] = tid;
            share[place] = same[tid];
            costs[place + 1] = cost_upto;
        }
        if (tid == 0) costs[0] = 0;
        if (begin) begins[at.y - 1] = place;
        if (tid == 0) begins[runs] = m;
        seq_barrier();
        const Groups groups{group_first, group_members, group_pages};
        for (int r = warp; r < runs; r += kMaxSeqs / 32) {
            const int s = begins[r], e = begins[r + 1];
            if (divide_even(share, costs, s, e, a.pg.ps, groups)) continue;
            if (e - s <= 32) divide_few(share, costs, s, e, a.pg.ps, groups);
            else divide_many(share, costs, s, e, a.pg.ps, groups, best + s + r, from + s, shared_by + s);
        }
        seq_barrier();
        const int first = n > 0 ? group_first[place] : 0, pages = n > 0 ? group_pages[place] : 0, lead = n > 0 ? active[first] : tid;
        const bool grouped = pages > 0;
        if (tid < a.batch) {
            pages_of[tid] = pages;
            if (a.groups) {
                a.groups[2 * tid] = lead;
                a.groups[2 * tid + 1] = pages;
            }
        }
        const int upto = plan_scan(make_int2(grouped ? n : 0, 0), tmp, &total).x;
        if (tid < a.batch) node0[tid] = upto - (grouped ? n : 0);
        if (tid == 0) node0[a.batch] = total.x;
        seq_barrier();
        // segments: own of sequence tid, and its group's where it leads one
        int tiles[2] = {0, 0}, blocks[2] = {0, 0}, weight[2] = {a.work.list[0].weight1, a.work.list[1].weight1}, cost[2], units[2];
        const int own_keys = keys - pages * a.pg.ps;
        auto segment_of = [&](int which, int count, int many) {
            const WorkList& w = a.work.list[which];
            tiles[which] = (count + (1 << w.kt) - 1) >> w.kt;
            blocks[which] = (many * a.G + (1 << w.qt) - 1) >> w.qt;
            if (many * a.G > 128) weight[which] = w.weight2;
        };
        if (n > 0 && own_keys > 0) segment_of(0, own_keys, n);
        if (grouped && first == place) {        // its group's nodes lie before those of the next active one
            const int after = place + group_members[place], nodes = (after < m ? node0[active[after]] : node0[a.batch]) - node0[tid];
            nodes_of[tid] = nodes;
            segment_of(1, pages * a.pg.ps, nodes);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            units[i] = blocks[i] * a.pg.hkv;
            cost[i] = units[i] * (tiles[i] * weight[i] + a.work.list[i].extra);
        }
        int2 all_cost, all_units;
        const int2 c = plan_scan(make_int2(cost[0], cost[1]), tmp, &all_cost), u = plan_scan(make_int2(units[0], units[1]), tmp, &all_units);
#pragma unroll
        for (int i = 0; i < 2; ++i) {       // (past the batch: empty, where the list ends)
            const int e = place_of(tid, i);
            const bool one = a.work.many == 1;
            seg_start[e] = (one ? c.x + c.y - (i ? 0 : cost[0]) : i ? c.y : c.x - cost[0]) - (i || one ? cost[1] : 0);
            seg_unit[e] = (one ? u.x + u.y - (i ? 0 : units[0]) : i ? u.y : u.x - units[0]) - (i || one ? units[1] : 0);
            seg_tiles[e] = tiles[i];
            seg_blocks[e] = blocks[i];
            seg_weight[e] = weight[i];
        }
        if (tid == 0) {
            total_cost[0] = a.work.many == 1 ? all_cost.x + all_cost.y : all_cost.x;
            total_units[0] = a.work.many == 1 ? all_units.x + all_units.y : all_units.x;
            total_cost[1] = all_cost.y;
            total_units[1] = all_units.y;
        }
        seq_barrier();
        if (tid < a.batch) {
            const int e = place_of(lead, 1);
            TreeSeq s;
            s.n = n;
            s.start = seg_start[place_of(tid, 0)];
            s.tiles = tiles[0];
            s.blocks = blocks[0];
            s.lead_start = seg_start[e];
            s.lead_tiles = grouped ? seg_tiles[e] : 0;
            s.lead_blocks = seg_blocks[e];
            s.node0 = node0[tid] - node0[lead];
            s.row = own_row(a, tid);
            s.lead_row = lead_row(a, lead, node0[lead]);
            s.weight = weight[0];
            s.lead_weight = seg_weight[e];
            a.seqs[tid] = s;
        }
    }
    __syncthreads();
    if (tid == 0) {
        a.head->kind = a.kind;
        a.head->batch = a.batch;
        a.head->n_max = a.n_max;
        a.head->max_pages = a.pg.max_pages;
        a.head->hkv = a.pg.hkv;
        a.head->ps = a.pg.ps;
        a.head->G = a.G;
    }
    for (int b = warp; b < a.batch; b += kPlanThreads / 32)
        for (int i = lane; i < node0[b + 1] - node0[b]; i += 32) a.map[node0[b] + i] = b * a.n_max + i;
    {       // the lists, each by its part of the threads
        const int threads = kPlanThreads / a.work.many, list = tid / threads, me = tid - list * threads;
        const WorkList& L = a.work.list[list];
        const int all = total_cost[list], all_units = total_units[list], per = max((all + L.C - 1) / L.C, L.least);
        if (me == 0) a.head->per[list] = per;
        // the last of the list's segments that begins at or before x and is not empty
        auto segment = [&](const int* begin, int x) {
            int lo = list * kMaxSeqs, hi = a.work.many == 1 ? 2 * a.batch : lo + a.batch;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (begin[mid] <= x) lo = mid; else hi = mid;
            }
            return lo;
        };
        // The items of run c are numbers u + c for its units u: the list of units and the list of runs advance together.
        int* const firsts = first_of + (list ? a.work.list[0].C : 0);
        int* const lasts = last_of + (list ? a.work.list[0].C : 0);
        // Items by units, `share` threads for each, where there are few.
        int share_log = 0;
        while (((long long)all_units << (share_log + 1)) <= threads && share_log < 5) ++share_log;
        for (int x = me; x < all_units << share_log; x += threads) {
            const int u = x >> share_log, e = segment(seg_unit, u), idx = u - seg_unit[e];
            const int b = a.work.many == 1 ? e >> 1 : e & (kMaxSeqs - 1), which = a.work.many == 1 ? e & 1 : list;
            const int t = seg_tiles[e], bl = seg_blocks[e], w = seg_weight[e], start = seg_start[e] + idx * (t * w + L.extra);
            const int c0 = start / per, c1 = (start + (t - 1) * w) / per;
            TreeItem it;
            it.b = b;
            it.h = bl == 1 ? idx : idx / bl;
            it.row0 = (idx - it.h * bl) << L.qt;
            int whole;          // where its rows go if the unit is one item
            if (which) {
                it.page0 = 0;
                it.held = pages_of[b];
                it.ctx = it.keys = pages_of[b] * a.pg.ps;
                it.first = ~node0[b];
                it.nodes = nodes_of[b];
                whole = lead_row(a, b, node0[b]) + it.h * a.lead_rows + it.row0;
            } else {
                it.page0 = pages_of[b];
                it.held = held_of[b] - it.page0;
                it.ctx = ctx_of[b] - it.page0 * a.pg.ps;
                it.keys = keys_of[b] - it.page0 * a.pg.ps;
                it.first = b * a.n_max;
                it.nodes = n_of[b];
                whole = pages_of[b] ? own_row(a, b) + it.h * a.own_rows + it.row0 : -1;
            }
            for (int c = c0 + (x & ((1 << share_log) - 1)); c <= c1; c += 1 << share_log) {
                const long long v0 = (long long)c * per;
                // (a tile is in the run that its place is in)
                it.lo = c == c0 ? 0 : ((int)(v0 - start) + w - 1) / w;
                it.hi = c == c1 ? t : ((int)(v0 + per - start) + w - 1) / w;
                it.dst = c0 == c1 ? whole : L.slot0 + ((2 * c + (start < v0 ? 0 : 1)) << L.qt);
                a.items[list][u + c] = it;
                atomicMin(&firsts[c], u);
                atomicMax(&lasts[c], u);
            }
        }
        __syncthreads();
        for (int c = me; c < L.C; c += threads) a.runs[list][c] = lasts[c] < 0 ? make_int2(0, 0) : make_int2(firsts[c] + c, lasts[c] + 1 + c);
    }
}

// Rows whose keys several items read, each of them in the order own keys, shared keys; and rows that none did. As
// tree_join_kernel, RW rows to a warp or PW warps to a row, with what the plan says of a row's sequence.
template <int PW> constexpr int kJoinThreads = PW > 4 ? 32 * PW : 128;
constexpr int join_blocks(int HD, int RW) { return HD == 64 ? 6 : RW == 1 ? 5 : 4; }

template <class T, int HD, int RW, int PW>
__global__ void __launch_bounds__(kJoinThreads<PW>, PW > 4 ? 2 : join_blocks(HD, RW)) tree_shared_join_kernel(const __grid_constant__ TreeArgs a, const __grid_constant__ WorkLists work) {
    static_assert(RW == 1 || PW == 1, "several rows per warp or several warps per row");
    constexpr int LPR = 32 / RW, E = HD / LPR, V = E < 4 ? E : 4, J = RW == 4 ? 4 : 8, ROWS = kJoinThreads<PW> / 32 / PW * RW;
    __shared__ float others[PW > 1 ? kJoinThreads<PW> / 32 : 1][HD + 2];     // of a row's warps: output, maximum, sum
    const int lane = threadIdx.x & 31, l = lane % LPR, warp = threadIdx.x >> 5, pw = warp % PW;
    // the plan is older than the kernel before this one, which let this one start after its own wait
    const bool ok = plan_fits(a);
    const int per0 = ok ? a.head->per[0] : 1, per1 = ok ? a.head->per[work.many - 1] : 1;
    const WorkList &L0 = work.list[0], &L1 = work.list[1];
    bool begun = false;
    const unsigned rows = (unsigned)a.batch * a.n_max * a.hq, step = gridDim.x * ROWS;
    unsigned row = blockIdx.x * ROWS + warp / PW * RW + lane / LPR;
    // (the CTA's warps go round together: with several to a row they meet)
    for (unsigned base = blockIdx.x * ROWS; base < rows; base += step, row += step) {
        const bool there = ok && row < rows;
        const int head = row % a.hq, node = row / a.hq % a.n_max, b = there ? row / a.hq / a.n_max : 0;
        const int h = head / a.G, g = head - h * a.G;
        const TreeSeq s = a.seqs[b];
        const bool some = there && node < s.n;
        // own parts, then the group's: how many, the CTA of the first, the unit's place in the list, and the row
        const int r0 = node * a.G + g, r1 = (s.node0 + node) * a.G + g;
        const int u0 = s.start + (h * s.blocks + (r0 >> L0.qt)) * (s.tiles * s.weight + L0.extra), c0 = u0 / per0;
        const int u1 = s.lead_start + (h * s.lead_blocks + (r1 >> L1.qt)) * (s.lead_tiles * s.lead_weight + L1.extra), c1 = u1 / per1;
        const int n0 = some && s.tiles ? (u0 + (s.tiles - 1) * s.weight) / per0 - c0 + 1 : 0;
        const int n1 = some && s.lead_tiles ? (u1 + (s.lead_tiles - 1) * s.lead_weight) / per1 - c1 + 1 : 0;
        const bool written = n0 == 1 && s.lead_tiles == 0;
        const int whole = written ? 0 : n0 + n1, parts = (whole - pw + PW - 1) / PW;       // this warp's: pw, pw + PW, ...
        if (!begun) pdl_wait();
        begun = true;
        const int most = __reduce_max_sync(0xffffffffu, parts);
        auto at = [&](int k) -> size_t {
            const int i = pw + k * PW;
            const bool own = i < n0;
            const int c = own ? c0 + i : c1 + i - n0, u = own ? u0 : u1, r = own ? r0 : r1, per = own ? per0 : per1, qt = own ? L0.qt : L1.qt;
            if ((own ? n0 : n1) == 1)
                return own ? (size_t)s.row + (size_t)h * a.own_rows + r : (size_t)s.lead_row + (size_t)h * a.lead_rows + r;
            return (size_t)(own ? L0.slot0 : L1.slot0) + (((size_t)c * 2 + (u < c * per ? 0 : 1)) << qt) + (r & ((1 << qt) - 1));
        };
        float acc[E], x[J][E], m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
        auto load = [&](int i) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const bool in = i + j < parts, blocks = pw + (i + j) * PW < n0 ? L0.blocks : L1.blocks;
                const size_t row = in ? at(i + j) : 0;
#pragma unroll
                for (int g = 0; g < E / V; ++g) {
                    const int e = (g * LPR + l) * V;
                    // the tcgen05 kernel's rows lie in blocks of 32 rows x 32 elements, 16-byte pieces swizzled
                    const float* src = a.part_o + (!blocks ? row * HD + e
                                                           : (row & ~(size_t)31) * HD + (e >> 5) * 1024 + (row & 31) * 32 +
                                                                 ((((e & 31) >> 2) ^ (int)(row & 7)) << 2) + (e & 3));
                    if constexpr (V == 4) {
                        const float4 v = in ? *reinterpret_cast<const float4*>(src) : make_float4(0.f, 0.f, 0.f, 0.f);
                        x[j][4 * g] = v.x; x[j][4 * g + 1] = v.y; x[j][4 * g + 2] = v.z; x[j][4 * g + 3] = v.w;
                    } else {
                        const float2 v = in ? *reinterpret_cast<const float2*>(src) : make_float2(0.f, 0.f);
                        x[j][0] = v.x; x[j][1] = v.y;
                    }
                }
            }
        };
        load(0);
        float2 v = l < parts ? a.part_ml[at(l)] : make_float2(-INFINITY, 0.f);
        m = v.x;
        for (int i = LPR + l; i < parts; i += LPR) m = fmaxf(m, a.part_ml[at(i)].x);
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float ref = m == -INFINITY ? 0.f : m;
        float w = exp2f(v.x - ref);
        sum = v.y * w;
        for (int i = 0; i < most; i += J) {
            if (i) {
                load(i);
                if (i % LPR == 0) {
                    v = i + l < parts ? a.part_ml[at(i + l)] : make_float2(-INFINITY, 0.f);
                    w = exp2f(v.x - ref);
                    sum = fmaf(v.y, w, sum);
                }
            }
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const float wj = __shfl_sync(0xffffffffu, w, i % LPR + j, LPR);
                if (i + j >= parts) continue;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = fmaf(wj, x[j][e], acc[e]);
            }
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if constexpr (PW > 1) {
            // the row's warps' results against their common maximum: each adds up its part of the elements
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) others[warp][l * E + e] = acc[e];
            if (l == 0) {
                others[warp][HD] = m;
                others[warp][HD + 1] = sum;
            }
            __syncthreads();
            if (pw == 0) {
                float top = m;
#pragma unroll
                for (int q = 1; q < PW; ++q) top = fmaxf(top, others[warp + q][HD]);
                const float ref = top == -INFINITY ? 0.f : top;
                float f = exp2f(m - ref);
                sum *= f;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] *= f;
#pragma unroll
                for (int q = 1; q < PW; ++q) {
                    f = exp2f(others[warp + q][HD] - ref);
                    sum = fmaf(others[warp + q][HD + 1], f, sum);
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = fmaf(others[warp + q][l * E + e], f, acc[e]);
                }
                m = top;
            }
        }
        if (!there || written || pw) continue;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        T* out = static_cast<T*>(a.out) + (size_t)row * HD;
#pragma unroll
        for (int g = 0; g < E / V; ++g) {
            const int e = (g * LPR + l) * V;
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int y = 0; y < V; y += 2)
                    *reinterpret_cast<uint32_t*>(out + e + y) = two_bf16(acc[g * V + y] * inv, acc[g * V + y + 1] * inv);
            } else {
#pragma unroll
                for (int y = 0; y < V; ++y) out[e + y] = acc[g * V + y] * inv;
            }
        }
        if (a.lse && l == 0) a.lse[row] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.69314718055994531f;
    }
}

template <int R, int P>
struct JoinForm {
    static constexpr int RW = R, PW = P;
};
template <class T, int HD>
cudaError_t launch_join(const dflare_cache* c, const TreeArgs& a, const WorkLists& work, cudaStream_t s) {
    const long long rows = (long long)a.batch * a.n_max * a.hq;
    auto go = [&](auto form) {
        constexpr int RW = decltype(form)::RW, PW = decltype(form)::PW;
        constexpr int per = kJoinThreads<PW> / 32 / PW * RW;
        const long long most = (long long)c->num_sms * (PW > 4 ? 2 : join_blocks(HD, RW));
        return launch_kernel(true, tree_shared_join_kernel<T, HD, RW, PW>, dim3((unsigned)std::min((rows + per - 1) / per, most)), dim3(kJoinThreads<PW>), 0, s, a, work);
    };
    // Measured, a layer: 512 rows 17.1 us with a warp for each (four parts at a time 18.4); 4096 rows 31.0 with one for two, 32.5 for
    // four, 35.8 for each; 8192 rows 157 for two, 154 for four.
    if (rows < 256) return go(JoinForm<1, 8>());
    if (rows < 1024) return go(JoinForm<1, 4>());
    if (rows < 4096) return go(JoinForm<1, 1>());
    if (rows < 8192) return go(JoinForm<2, 1>());
    return go(JoinForm<4, 1>());
}

dflare_status refuse(const char* call, const char* m) {
    noalloc_set_error(std::string(call) + ": " + m);
    return DFLARE_EINVAL;
}
// the sizes that the three calls share; nullptr: nothing is wrong
const char* check_sizes(const dflare_cache* c, int batch, int n_max) {
    if (batch < 1 || batch > c->cfg.max_batch) return "batch must be in [1, max_batch]";
    if (n_max < 1 || n_max > c->cfg.max_nodes) return "n_max must be in [1, max_nodes]";
    return nullptr;
}

}  // namespace
}  // namespace dfl

using namespace dfl;

extern "C" {

dflare_status dflare_cache_shared_bytes(dflare_cache* c, int batch, int n_max, size_t* bytes) {
    const char* call = "dflare_cache_shared_bytes";
    if (!c || !bytes) return refuse(call, "NULL argument");
    if (const char* m = check_sizes(c, batch, n_max)) return refuse(call, m);
    const Layout y = layout_of(c, batch, n_max);
    if (!y.ok) return refuse(call, "more work than one call takes");
    *bytes = y.bytes;
    return DFLARE_OK;
}

dflare_status dflare_cache_share_plan(dflare_cache* c, const int32_t* n_nodes_dev, int batch, int n_max, void* work_dev,
                                      int32_t* groups_dev, void* stream) {
    const char* call = "dflare_cache_share_plan";
    if (!c || !n_nodes_dev || !work_dev) return refuse(call, "NULL argument");
    if (const char* m = check_sizes(c, batch, n_max)) return refuse(call, m);
    if (reinterpret_cast<uintptr_t>(work_dev) & 127u) return refuse(call, "the workspace must be 128-byte aligned");
    const Layout y = layout_of(c, batch, n_max);
    if (!y.ok) return refuse(call, "more work than one call takes");
    char* work = static_cast<char*>(work_dev);
    PlanArgs a{};
    a.pg = c->view;
    a.n_nodes = n_nodes_dev;
    a.head = reinterpret_cast<SharedHead*>(work);
    a.kind = plan_kind(c->cfg);
    for (int l = 0; l < y.work.many; ++l) {
        a.runs[l] = reinterpret_cast<int2*>(work + y.runs[l]);
        a.items[l] = reinterpret_cast<TreeItem*>(work + y.items[l]);
    }
    a.map = reinterpret_cast<int32_t*>(work + y.map);
    a.seqs = reinterpret_cast<TreeSeq*>(work + y.seqs);
    a.groups = groups_dev;
    a.batch = batch;
    a.n_max = n_max;
    a.G = c->cfg.n_q_heads / c->cfg.n_kv_heads;
    a.work = y.work;
    a.rows0 = y.rows0;
    a.own_rows = y.own_rows, a.lead_rows = y.lead_rows;
    DeviceGuard guard(c->device);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int ctas = (batch + kPlanThreads / 32 - 1) / (kPlanThreads / 32);
    static_assert(kMaxSeqs <= 8 * (kPlanThreads / 32), "a cluster of up to eight CTAs has a warp for every sequence");
    const cudaError_t e = launch_cluster(true, ctas, tree_shared_plan_kernel, dim3(ctas), dim3(kPlanThreads), 0, s, a);
    if (e == cudaSuccess) return DFLARE_OK;
    noalloc_set_error(std::string(call) + ": " + cudaGetErrorString(e));
    return DFLARE_ECUDA;
}

dflare_status dflare_cache_attend_shared(dflare_cache* c, int layer, const void* q_dev, long long q_row, const int32_t* mask_dev,
                                         int batch, int n_max, float scale, void* out_dev, float* lse_dev, void* work_dev,
                                         void* stream) {
    const char* call = "dflare_cache_attend_shared";
    if (!c || !q_dev || !out_dev || !work_dev) return refuse(call, "NULL argument");
    const dflare_cache_config& g = c->cfg;
    if (layer < 0 || layer >= g.n_layers) return refuse(call, "layer out of range");
    if (const char* m = check_sizes(c, batch, n_max)) return refuse(call, m);
    if (!(scale > 0.f) || !std::isfinite(scale)) return refuse(call, "scale must be positive and finite");
    if (q_row < (long long)g.n_q_heads * g.head_dim || q_row % 8 != 0) return refuse(call, "q_row must hold a row and be a multiple of 8");
    if ((reinterpret_cast<uintptr_t>(q_dev) | reinterpret_cast<uintptr_t>(out_dev)) & 15u) return refuse(call, "q and out must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(work_dev) & 127u) return refuse(call, "the workspace must be 128-byte aligned");
    const Layout y = layout_of(c, batch, n_max);
    if (!y.ok) return refuse(call, "more work than one call takes");
    char* work = static_cast<char*>(work_dev);
    TreeArgs a{};
    a.pg = c->view;
    a.q = q_dev;
    a.q_row = q_row;
    a.mask = mask_dev;
    a.out = out_dev;
    a.lse = lse_dev;
    a.part_o = reinterpret_cast<float*>(work + y.o);
    a.part_ml = reinterpret_cast<float2*>(work + y.ml);
    a.layer = layer;
    a.batch = batch;
    a.n_max = n_max;
    a.words = (n_max + 31) / 32;
    a.hq = g.n_q_heads;
    a.G = g.n_q_heads / g.n_kv_heads;
    a.G_inv = a.G > 1 ? 0xffffffffu / (uint32_t)a.G + 1u : 0u;
    a.QG = 1;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.head = reinterpret_cast<const SharedHead*>(work);
    a.kind = plan_kind(g);
    a.map = reinterpret_cast<const int32_t*>(work + y.map);
    a.seqs = reinterpret_cast<const TreeSeq*>(work + y.seqs);
    a.own_rows = y.own_rows;
    a.lead_rows = y.lead_rows;
    DeviceGuard guard(c->device);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool f32 = g.dtype == DFLARE_F32, wide = g.head_dim == 128;
    cudaError_t e = cudaSuccess;
    for (int l = 0; l < y.work.many && e == cudaSuccess; ++l) {
        a.runs = reinterpret_cast<const int2*>(work + y.runs[l]);
        a.items = reinterpret_cast<const TreeItem*>(work + y.items[l]);
        a.C = y.work.list[l].C;
        a.follows = l > 0;
        e = f32 ? launch_shared_f32(c, a, s) : y.work.list[l].blocks ? launch_shared_tc(c, a, s) : launch_shared_mma(c, a, s);
    }
    if (e == cudaSuccess) e = f32 ? (wide ? launch_join<float, 128>(c, a, y.work, s) : launch_join<float, 64>(c, a, y.work, s))
                                  : (wide ? launch_join<bf16, 128>(c, a, y.work, s) : launch_join<bf16, 64>(c, a, y.work, s));
    if (e == cudaSuccess) return DFLARE_OK;
    noalloc_set_error(std::string(call) + ": " + cudaGetErrorString(e));
    return DFLARE_ECUDA;
}

}  // extern "C"
