// Attention of a batch whose sequences share leading pages (samples and beams of one prompt): a shared page's keys are
// read once for all rows of the group, not once per sequence.
//
// The keys of a row are those that its group shares and the sequence's own, two disjoint sets; with o, m, l the weighted
// values, the maximum (log2 units) and the sum over each,
//   out = (o_s 2^(m_s - M) + o_o 2^(m_o - M)) / (l_s 2^(m_s - M) + l_o 2^(m_o - M)),   M = max(m_s, m_o),
// just as the parts of a row whose keys several CTAs read are joined. So a group's rows against its shared keys are one
// more "sequence" (without a mask: shared pages hold context only), and each sequence keeps the keys behind those.
//
// A plan, made once per step for all layers, lists this work: units (sequence or group, kv head, block of query rows), each
// with its key tiles and kExtra more for beginning and ending it. The CTAs take equal runs of the list. A unit that lies in one run is
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

constexpr int kSameThreads = 256;
constexpr int kPlanThreads = 1024;

// What a plan and the launches that follow it agree on, from the call's sizes alone.
struct Layout {
    bool ok;                    // everything fits its numbers
    int QT, KT, extra, least, C;
    int own_rows, lead_rows;    // rows of one kv head among the whole units' partial results
    size_t runs, items, map, seqs, ml, o, bytes;    // offsets
};
Layout layout_of(const dflare_cache* c, int batch, int n_max) {
    const dflare_cache_config& g = c->cfg;
    const int G = g.n_q_heads / g.n_kv_heads;
    Layout y{};
    const long long rows = (long long)batch * n_max * G;
    if (g.dtype == DFLARE_F32) {
        y.QT = kFRows, y.KT = kFKeys, y.extra = kFExtra, y.least = kFLeast, y.C = f32_ctas_per_sm(g.head_dim) * c->num_sms;
    } else {
        // (blocks of 128 rows where no group can have more)
        y.QT = rows <= 128 ? 128 : 256, y.KT = kTcKeys, y.extra = kTcExtra, y.least = kTcLeast, y.C = c->num_sms;
    }
    const long long own = (long long)batch * (((long long)n_max * G + y.QT - 1) / y.QT), lead = (rows + y.QT - 1) / y.QT + batch / 2;
    const long long units = (own + lead) * g.n_kv_heads, tiles = ((long long)g.max_pages * g.page_size + y.KT - 1) / y.KT + y.extra;
    const long long own_rows = ((long long)n_max * G + 31) / 32 * 32, lead_rows = (rows / 32 + batch + 1) * 32;
    const long long part = 2LL * y.C * y.QT + (batch * own_rows + lead_rows) * g.n_kv_heads;
    const long long most = 0x7fffffffLL - 4096;
    y.ok = units * tiles <= most && part <= most;
    if (!y.ok) return y;
    y.own_rows = (int)own_rows;
    y.lead_rows = (int)lead_rows;
    auto place = [&](size_t bytes) {
        const size_t at = y.bytes;
        y.bytes += (bytes + 127) / 128 * 128;
        return at;
    };
    place(sizeof(SharedHead));
    y.runs = place(sizeof(int2) * y.C);
    y.seqs = place(sizeof(TreeSeq) * batch);
    y.map = place(sizeof(int32_t) * (size_t)batch * n_max);
    y.items = place(sizeof(TreeItem) * (size_t)(units + y.C));
    y.ml = place(sizeof(float2) * (size_t)part);
    y.o = place(sizeof(float) * (size_t)part * g.head_dim);
    return y;
}

struct PlanArgs {
    PagesView pg;
    const int32_t* n_nodes;
    SharedHead* head;
    int2* runs;
    TreeItem* items;
    int32_t* map;
    TreeSeq* seqs;
    int32_t* groups;            // optional output
    int batch, n_max, G, QT, KT, extra, least, C, own_rows, lead_rows;
};

__device__ __forceinline__ void lengths_of(const PlanArgs& a, int b, int& n, int& held, int& ctx, int& keys) {
    n = min(max(a.n_nodes[b], 0), a.n_max);
    held = min(max(a.pg.held[b], 0), a.pg.max_pages);
    const long long room = (long long)held * a.pg.ps;
    const int len = max(a.pg.lens[b], 0);
    keys = (int)min((long long)len + n, room);
    ctx = min(len, keys);
}

// Pages that sequence b (a CTA each) and the one before it that has nodes both hold in the same places, full of context.
__global__ void __launch_bounds__(kSameThreads) tree_same_kernel(const PlanArgs a) {
    __shared__ int before;
    pdl_wait();
    pdl_trigger();
    const int b = blockIdx.x, tid = threadIdx.x;
    if (tid == 0) before = -1;
    __syncthreads();
    int n, held, ctx, keys, same = 0;
    lengths_of(a, b, n, held, ctx, keys);
    if (tid < b && a.n_nodes[tid] > 0) atomicMax(&before, tid);
    __syncthreads();
    const int p = before;
    if (p >= 0 && n > 0) {
        int n2, held2, ctx2, keys2;
        lengths_of(a, p, n2, held2, ctx2, keys2);
        const int most = min(ctx, ctx2) / a.pg.ps;
        const int32_t *x = a.pg.table + (size_t)p * a.pg.max_pages, *y = a.pg.table + (size_t)b * a.pg.max_pages;
        constexpr int U = 4;
        for (;;) {      // U x 256 pages at a time, up to the first that differs
            int u = U * kSameThreads;
#pragma unroll
            for (int k = U - 1; k >= 0; --k) {
                const int i = same + k * kSameThreads + tid;
                const bool equal = i < most && x[i] == y[i] && x[i] >= 0 && x[i] < a.pg.pages;
                if (!equal) u = k * kSameThreads + tid;
            }
            __shared__ int least;
            if (tid == 0) least = U * kSameThreads;
            __syncthreads();
            u = __reduce_min_sync(0xffffffffu, u);
            if ((tid & 31) == 0) atomicMin(&least, u);
            __syncthreads();
            u = least;
            __syncthreads();
            same += u;
            if (u < U * kSameThreads) break;
        }
    }
    if (tid == 0) a.head->same[b] = same;
}

// inclusive sums over a CTA of kPlanThreads; tmp holds 32 ints
__device__ __forceinline__ int plan_scan(int v, int* tmp, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    __syncthreads();
    if (lane == 31) tmp[warp] = v;
    __syncthreads();
    int t = tmp[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, t, o);
        if (lane >= o) t += x;
    }
    *total = __shfl_sync(0xffffffffu, t, 31);
    const int base = __shfl_sync(0xffffffffu, t, max(warp - 1, 0));
    return v + (warp ? base : 0);
}

// What a group of `many` that shares `pages` saves, in keys: less what one more unit and the joining of its rows cost, in keys
// that could be read meanwhile.
constexpr int kGroupCost = 512, kMemberCost = 64;
__device__ __forceinline__ float saving(const PlanArgs& a, int many, int pages) {
    return fmaxf((float)(many - 1) * (float)pages * (float)a.pg.ps - (float)(kGroupCost + kMemberCost * many), 0.f);
}

// One CTA. Segment 2 b is sequence b's own keys, 2 b + 1 the keys shared by the group that b leads.
__global__ void __launch_bounds__(kPlanThreads) tree_shared_plan_kernel(const PlanArgs a) {
    __shared__ int active[kMaxSeqs], share[kMaxSeqs], from[kMaxSeqs + 1], shared_by[kMaxSeqs + 1], nodes_of[kMaxSeqs];
    __shared__ float best[kMaxSeqs + 1];
    __shared__ int pages_of[kMaxSeqs], node0[kMaxSeqs + 1], members[kMaxSeqs];
    __shared__ int seg_start[2 * kMaxSeqs], seg_unit[2 * kMaxSeqs], seg_tiles[2 * kMaxSeqs], seg_blocks[2 * kMaxSeqs];
    __shared__ int tmp[32];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31;
    int n = 0, held = 0, ctx = 0, keys = 0, total;
    if (tid < a.batch) {
        lengths_of(a, tid, n, held, ctx, keys);
        pages_of[tid] = 0;
        members[tid] = 0;
    }
    // the sequences that have nodes, in order
    const int place = plan_scan(n > 0, tmp, &total) - 1, m = total;
    if (n > 0) {
        active[place] = tid;
        share[place] = place ? a.head->same[tid] : 0;
    }
    __syncthreads();
    if (tid < 32) {
        // best[j]: of the first j. Lane l looks at groups that begin at i = l, l + 32, ..; least[k]: pages that i .. j - 1 share.
        int least[kMaxSeqs / 32];
#pragma unroll
        for (int k = 0; k < kMaxSeqs / 32; ++k) least[k] = 0x7fffffff;
        if (lane == 0) best[0] = 0.f;
        __syncwarp();
        for (int j = 1; j <= m; ++j) {
            float top = -1.f;
            int at = 0, pages = 0;
            const int next = share[j - 1];
#pragma unroll
            for (int k = 0; k < kMaxSeqs / 32; ++k) {
                const int i = lane + 32 * k;
                if (32 * k >= j) break;
                if (i < j - 1) least[k] = min(least[k], next);
                if (i < j) {
                    const float v = best[i] + (i < j - 1 ? saving(a, j - i, least[k]) : 0.f);
                    if (v > top) {
                        top = v;
                        at = i;
                        pages = least[k];
                    }
                }
            }
            // (not negative where there is one, so their bits are in order; of equal ones the shortest group)
            const unsigned bits = top < 0.f ? 0u : __float_as_uint(top) + 1u, most = __reduce_max_sync(0xffffffffu, bits);
            const int last = __reduce_max_sync(0xffffffffu, bits == most ? at : -1);
            if (bits == most && at == last) {
                best[j] = top;
                from[j] = at;
                shared_by[j] = pages;
            }
            __syncwarp();
        }
        if (lane == 0) {
            for (int j = m; j > 0; j = from[j]) {
                const int i = from[j];
                members[i] = j - i;
                if (j - i > 1) pages_of[i] = shared_by[j];
            }
        }
    }
    __syncthreads();
    // (members and pages_of by place so far; from here on by sequence)
    int lead = tid, pages = 0, many = 0;
    if (n > 0) {
        int i = place;
        while (members[i] == 0) --i;        // (place 0 begins one)
        lead = active[i];
        pages = pages_of[i];
        if (i == place && pages) many = members[i];
    }
    __syncthreads();
    const bool grouped = n > 0 && pages > 0;
    if (tid < a.batch) {
        pages_of[tid] = grouped ? pages : 0;
        a.head->groups[2 * tid] = lead;
        a.head->groups[2 * tid + 1] = grouped ? pages : 0;
        if (a.groups) {
            a.groups[2 * tid] = lead;
            a.groups[2 * tid + 1] = grouped ? pages : 0;
        }
    }
    const int upto = plan_scan(grouped ? n : 0, tmp, &total);
    if (tid < a.batch) node0[tid] = upto - (grouped ? n : 0);
    if (tid == 0) node0[a.batch] = total;
    __syncthreads();
    // segments: own of sequence tid, and its group's where it leads one
    int tiles[2] = {0, 0}, blocks[2] = {0, 0}, end = 0;
    const int skip = grouped ? pages : 0, own_keys = keys - skip * a.pg.ps;
    if (n > 0 && own_keys > 0) {
        tiles[0] = (own_keys + a.KT - 1) / a.KT;
        blocks[0] = (n * a.G + a.QT - 1) / a.QT;
    }
    if (many) {         // this thread's sequence leads: its group's nodes lie before those of the next active one
        const int after = place + many;
        end = after < m ? node0[active[after]] : node0[a.batch];
        nodes_of[tid] = end - node0[tid];
        tiles[1] = (int)(((long long)pages * a.pg.ps + a.KT - 1) / a.KT);
        blocks[1] = ((end - node0[tid]) * a.G + a.QT - 1) / a.QT;
    }
    int cost[2], units[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        units[i] = blocks[i] * a.pg.hkv;
        cost[i] = units[i] * (tiles[i] + a.extra);
    }
    int all, all_units;
    const int cost_upto = plan_scan(cost[0] + cost[1], tmp, &all), unit_upto = plan_scan(units[0] + units[1], tmp, &all_units);
    if (tid < a.batch) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            seg_start[2 * tid + i] = cost_upto - cost[1] - (i ? 0 : cost[0]);
            seg_unit[2 * tid + i] = unit_upto - units[1] - (i ? 0 : units[0]);
            seg_tiles[2 * tid + i] = tiles[i];
            seg_blocks[2 * tid + i] = blocks[i];
        }
    }
    const int per = max((all + a.C - 1) / a.C, a.least);
    if (tid == 0) {
        a.head->batch = a.batch;
        a.head->n_max = a.n_max;
        a.head->per = per;
        a.head->ok = 1;
    }
    __syncthreads();
    // rows of whole units: 2 C blocks of the CTAs, then the sequences' own, then the groups'
    const int own0 = 2 * a.C * a.QT, lead0 = own0 + a.batch * a.pg.hkv * a.own_rows;
    auto lead_row = [&](int b) { return lead0 + (node0[b] * a.G / 32 + b) * 32; };
    if (tid < a.batch) {
        const int e = 2 * lead + 1;
        TreeSeq s{};
        s.n = n;
        s.start = seg_start[2 * tid];
        s.tiles = tiles[0];
        s.blocks = blocks[0];
        s.lead_start = seg_start[e];
        s.lead_tiles = grouped ? seg_tiles[e] : 0;
        s.lead_blocks = seg_blocks[e];
        s.node0 = node0[tid] - node0[lead];
        s.row = own0 + tid * a.pg.hkv * a.own_rows;
        s.lead_row = lead_row(lead);
        a.seqs[tid] = s;
    }
    for (int x = tid; x < a.batch * a.n_max; x += kPlanThreads) {
        const int b = x / a.n_max, i = x - b * a.n_max;
        const int count = (b + 1 < a.batch ? node0[b + 1] : node0[a.batch]) - node0[b];
        if (i < count) a.map[node0[b] + i] = x;
    }
    // The items of run c are numbers u + c for its units u: the list of units and the list of runs advance together. Four threads
    // share a run's units.
    constexpr int kShare = 4;
    for (int x = tid; x < a.C * kShare; x += kPlanThreads) {
        const int c = x / kShare, part = x % kShare;
        const long long v0 = (long long)c * per, v1 = min(v0 + per, (long long)all);
        if (v0 >= v1) {
            if (part == 0) a.runs[c] = make_int2(0, 0);
            continue;
        }
        int lo = 0, hi = 2 * a.batch;       // the last segment that begins at or before v0 and is not empty
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (seg_start[mid] <= v0) lo = mid; else hi = mid;
        }
        while (lo > 0 && seg_blocks[lo] == 0) --lo;
        int e = lo, unit = seg_tiles[e] + a.extra, idx = (int)((v0 - seg_start[e]) / unit);
        long long start = seg_start[e] + (long long)idx * unit;
        if (v0 - start >= seg_tiles[e]) {       // the run begins behind the unit's tiles
            ++idx;
            start += unit;
        }
        int u = seg_unit[e] + idx;
        const int first = u;
        for (; start < v1; ++u, ++idx, start += unit) {
            while (e < 2 * a.batch && idx >= seg_blocks[e] * a.pg.hkv) {    // on to the next segment
                idx = 0;
                ++e;
                if (e < 2 * a.batch) unit = seg_tiles[e] + a.extra;
            }
            if (e >= 2 * a.batch) break;
            if ((u - first) % kShare != part) continue;
            const int b = e >> 1, t = seg_tiles[e], bl = seg_blocks[e];
            TreeItem it;
            it.b = b;
            it.h = idx / bl;
            it.row0 = (idx - it.h * bl) * a.QT;
            it.lo = (int)max(v0 - start, 0LL);
            it.hi = (int)min(v1 - start, (long long)t);
            const bool whole = it.lo == 0 && it.hi == t;
            const int cut = (2 * c + (start < v0 ? 0 : 1)) * a.QT;
            if (e & 1) {
                it.page0 = 0;
                it.held = pages_of[b];
                it.ctx = it.keys = pages_of[b] * a.pg.ps;
                it.first = ~node0[b];
                it.nodes = nodes_of[b];
                it.dst = whole ? lead_row(b) + it.h * a.lead_rows + it.row0 : cut;
            } else {
                int n2, held2, ctx2, keys2;
                lengths_of(a, b, n2, held2, ctx2, keys2);
                it.page0 = pages_of[b];
                it.held = held2 - it.page0;
                it.ctx = ctx2 - it.page0 * a.pg.ps;
                it.keys = keys2 - it.page0 * a.pg.ps;
                it.first = b * a.n_max;
                it.nodes = n2;
                it.dst = !whole ? cut : pages_of[b] ? own0 + (b * a.pg.hkv + it.h) * a.own_rows + it.row0 : -1;
            }
            a.items[u + c] = it;
        }
        if (part == 0) a.runs[c] = make_int2(first + c, u + c);
    }
}

// Rows whose keys several items read, each of them in the order own keys, shared keys; and rows that none did. As
// tree_join_kernel, RW rows to a warp, with what the plan says of a row's sequence.
constexpr int kJoinThreads = 128;
constexpr int join_blocks(int HD, int RW) { return HD == 64 ? 6 : RW == 1 ? 5 : 4; }

template <class T, int HD, int RW>
__global__ void __launch_bounds__(kJoinThreads, join_blocks(HD, RW)) tree_shared_join_kernel(const TreeArgs a, int QT, int extra, bool blocks) {
    constexpr int LPR = 32 / RW, E = HD / LPR, V = E < 4 ? E : 4, J = 4;
    const int lane = threadIdx.x & 31, l = lane % LPR, warp = threadIdx.x >> 5;
    // the plan is older than the kernel before this one, which let this one start after its own wait
    const bool ok = a.head->batch == a.batch && a.head->n_max == a.n_max && a.head->ok;
    const int per = ok ? a.head->per : 1;
    const unsigned rows = (unsigned)a.batch * a.n_max * a.hq, step = gridDim.x * (kJoinThreads / 32) * RW;
    unsigned row = (blockIdx.x * (kJoinThreads / 32) + warp) * RW + lane / LPR;
    for (bool begun = false; !begun || row - lane / LPR < rows; row += step) {
        const bool there = ok && row < rows;
        const int head = row % a.hq, node = row / a.hq % a.n_max, b = there ? row / a.hq / a.n_max : 0;
        const int h = head / a.G, g = head - h * a.G;
        const TreeSeq s = a.seqs[b];
        const bool some = there && node < s.n;
        // own parts, then the group's: how many, the CTA of the first, the unit's place in the list, and the row
        const int r0 = node * a.G + g, r1 = (s.node0 + node) * a.G + g;
        const int u0 = s.start + (h * s.blocks + r0 / QT) * (s.tiles + extra), c0 = u0 / per;
        const int u1 = s.lead_start + (h * s.lead_blocks + r1 / QT) * (s.lead_tiles + extra), c1 = u1 / per;
        const int n0 = some && s.tiles ? (u0 + s.tiles - 1) / per - c0 + 1 : 0;
        const int n1 = some && s.lead_tiles ? (u1 + s.lead_tiles - 1) / per - c1 + 1 : 0;
        const bool written = n0 == 1 && s.lead_tiles == 0;
        const int parts = written ? 0 : n0 + n1;
        if (!begun) pdl_wait();
        begun = true;
        const int most = __reduce_max_sync(0xffffffffu, parts);
        auto at = [&](int i) -> size_t {
            const bool own = i < n0;
            const int c = own ? c0 + i : c1 + i - n0, u = own ? u0 : u1, r = own ? r0 : r1;
            if ((own ? n0 : n1) == 1)
                return own ? (size_t)s.row + (size_t)h * a.own_rows + r : (size_t)s.lead_row + (size_t)h * a.lead_rows + r;
            return ((size_t)c * 2 + (u < c * per ? 0 : 1)) * QT + r % QT;
        };
        float acc[E], x[J][E], m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
        auto load = [&](int i) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const bool in = i + j < parts;
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
        if (!there || written) continue;
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

template <class T, int HD>
cudaError_t launch_join(const dflare_cache* c, const TreeArgs& a, int QT, int extra, bool blocks, cudaStream_t s) {
    const long long rows = (long long)a.batch * a.n_max * a.hq;
    auto go = [&](auto kernel, int RW) {
        const long long per = kJoinThreads / 32 * RW, most = (long long)c->num_sms * join_blocks(HD, RW);
        return launch_kernel(true, kernel, dim3((unsigned)std::min((rows + per - 1) / per, most)), dim3(kJoinThreads), 0, s, a, QT, extra, blocks);
    };
    return rows < 4096 ? go(tree_shared_join_kernel<T, HD, 1>, 1) : go(tree_shared_join_kernel<T, HD, 4>, 4);
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
    a.runs = reinterpret_cast<int2*>(work + y.runs);
    a.items = reinterpret_cast<TreeItem*>(work + y.items);
    a.map = reinterpret_cast<int32_t*>(work + y.map);
    a.seqs = reinterpret_cast<TreeSeq*>(work + y.seqs);
    a.groups = groups_dev;
    a.batch = batch;
    a.n_max = n_max;
    a.G = c->cfg.n_q_heads / c->cfg.n_kv_heads;
    a.QT = y.QT, a.KT = y.KT, a.extra = y.extra, a.least = y.least, a.C = y.C;
    a.own_rows = y.own_rows, a.lead_rows = y.lead_rows;
    DeviceGuard guard(c->device);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = launch_kernel(true, tree_same_kernel, dim3(batch), dim3(kSameThreads), 0, s, a);
    if (e == cudaSuccess) e = launch_kernel(true, tree_shared_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
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
    a.C = y.C;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.head = reinterpret_cast<const SharedHead*>(work);
    a.runs = reinterpret_cast<const int2*>(work + y.runs);
    a.items = reinterpret_cast<const TreeItem*>(work + y.items);
    a.map = reinterpret_cast<const int32_t*>(work + y.map);
    a.seqs = reinterpret_cast<const TreeSeq*>(work + y.seqs);
    a.own_rows = y.own_rows;
    a.lead_rows = y.lead_rows;
    DeviceGuard guard(c->device);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool f32 = g.dtype == DFLARE_F32, wide = g.head_dim == 128;
    cudaError_t e = f32 ? launch_shared_f32(c, a, s) : launch_shared_tc(c, a, y.QT, s);
    if (e == cudaSuccess)
        e = f32 ? (wide ? launch_join<float, 128>(c, a, y.QT, y.extra, false, s) : launch_join<float, 64>(c, a, y.QT, y.extra, false, s))
                : (wide ? launch_join<bf16, 128>(c, a, y.QT, y.extra, true, s) : launch_join<bf16, 64>(c, a, y.QT, y.extra, true, s));
    if (e == cudaSuccess) return DFLARE_OK;
    noalloc_set_error(std::string(call) + ": " + cudaGetErrorString(e));
    return DFLARE_ECUDA;
}

}  // extern "C"
