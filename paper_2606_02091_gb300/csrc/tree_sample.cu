// Sampled acceptance in drafted trees: the target's probabilities p and the drafter's q decide, by given random numbers,
// which drafted child of a node is kept, and what follows where none is.
//
// At a node the walk holds a residual w = max(0, p - F q) with F = 0, its sum W = 1, and the mass Q = 1 that the drafter's
// next draw is from. Child i with token x is kept where u_i (q_x / Q) W < w_x. If it is not, the residual loses the
// drafter's share: w <- max(0, w - (W / Q) q). As q and the shares are not negative, clamping after every step is clamping
// once, so F <- F + W / Q says it all, and only W = sum w needs another look at the rows. Drawn without replacement,
// Q <- Q - q_x. Where no child is left, the next token is the first whose running sum of w exceeds u_0 sum w.
// Drafts that were picked and not drawn (no q) have the residual p without the picked tokens before.
//
// Decisions hang on sums over the vocabulary: fp32 sums of 150000 terms would move them for one call in a hundred.
// They are held as pairs of fp32 numbers (Knuth's two-sum, products by a fused multiply-add: 2^-46), and so is what the
// walk holds: 64-bit arithmetic has 1/64 of the fp32 rate on this GPU (64 blocks of 16 over 151936 tokens 54.5 us with it in the last
// search, 23.7 without; 21.7 since the cluster meets by messages and not barriers).
//
// A cluster of CTAs per tree, each with a part of the vocabulary; all of them walk the same tree in step. What a walk asks
// of a node whose children before it were not asked (u q_x < p_x) is found for all nodes at once while their numbers come
// in. A residual's sum is one pass over the rows by the whole cluster; its parts meet through distributed shared memory.
#include <math.h>

#include <algorithm>
#include <atomic>
#include <string>

#include "common.cuh"
#include "paged.h"
#include "umma.cuh"

namespace dfl {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;

struct SampleArgs {
    const int32_t* tokens;
    const int32_t* parents;
    const int32_t* n_nodes;
    const float* target;        // [batch][n_max][vocab]
    const float* draft;         // [batch][draft_rows][vocab], or null
    const float* u;             // [batch][n_max]
    int32_t* accept_len;
    int32_t* path;
    int32_t* next_token;
    uint32_t* err;
    int n_max, draft_rows, vocab, distinct;
    int part;                   // elements of a warp, a multiple of 4
};

// A sum as two fp32 numbers. `l` takes up what `h` could not hold.
struct Sum {
    float h, l;
};
__device__ __forceinline__ void add(Sum& s, float x, float low) {
    const float t = __fadd_rn(s.h, x), b = __fsub_rn(t, s.h);
    s.l = __fadd_rn(s.l, __fadd_rn(__fadd_rn(__fsub_rn(s.h, __fsub_rn(t, b)), __fsub_rn(x, b)), low));
    s.h = t;
}
__device__ __forceinline__ Sum shuffled(const Sum& s, int o) { return {__shfl_xor_sync(0xffffffffu, s.h, o), __shfl_xor_sync(0xffffffffu, s.l, o)}; }
__device__ __forceinline__ Sum warp_total(Sum s) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const Sum x = shuffled(s, o);
        // (the lower lane's first: both lanes have the same bits)
        Sum a = threadIdx.x & o ? x : s, b = threadIdx.x & o ? s : x;
        add(a, b.h, b.l);
        s = a;
    }
    return s;
}
// inclusive sums over the lanes
__device__ __forceinline__ Sum warp_upto(Sum s) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        Sum x = {__shfl_up_sync(0xffffffffu, s.h, o), __shfl_up_sync(0xffffffffu, s.l, o)};
        if ((threadIdx.x & 31) >= o) {
            add(x, s.h, s.l);
            s = x;
        }
    }
    return s;
}
// products and quotients of such numbers, to 2^-44
__device__ __forceinline__ Sum settled(float h, float l) {
    const float t = __fadd_rn(h, l);
    return {t, __fsub_rn(l, __fsub_rn(t, h))};
}
__device__ __forceinline__ Sum times(const Sum& a, const Sum& b) {
    const float p = __fmul_rn(a.h, b.h);
    return settled(p, __fmaf_rn(a.h, b.l, __fmaf_rn(a.l, b.h, __fmaf_rn(a.h, b.h, -p))));
}
__device__ __forceinline__ Sum over(const Sum& a, const Sum& b) {
    const float inv = __frcp_rn(b.h), q = __fmul_rn(a.h, inv);     // (the remainder makes up for what q lacks)
    const float rest = __fadd_rn(__fmaf_rn(-q, b.h, a.h), __fmaf_rn(-q, b.l, a.l));
    return settled(q, __fmul_rn(rest, inv));
}
__device__ __forceinline__ bool above(const Sum& a, const Sum& b) { return __fadd_rn(__fsub_rn(a.h, b.h), __fsub_rn(a.l, b.l)) > 0.f; }
// (what is left of p by less than half a step of it lies in `l` alone)
__device__ __forceinline__ bool weighs(const Sum& s) { return __fadd_rn(s.h, s.l) > 0.f; }
__device__ __forceinline__ Sum from_lane(const Sum& s, int lane) { return {__shfl_sync(0xffffffffu, s.h, lane), __shfl_sync(0xffffffffu, s.l, lane)}; }
// Of parts that lie one after another behind `base`, one per lane of the first `many`: the first with any weight at which the running
// sum passes goal (where rounding hides it, the last with any), and base is moved up to it. Neighbouring running sums add up
// in different orders, so that the one behind a part without weight may be larger in its last bits.
__device__ __forceinline__ int part_of(const Sum& part, int many, const Sum& goal, Sum& base) {
    const int lane = threadIdx.x & 31;
    const Sum upto = warp_upto(part);
    Sum x = base;
    add(x, upto.h, upto.l);
    const unsigned some = __ballot_sync(0xffffffffu, lane < many && weighs(part)), past = __ballot_sync(0xffffffffu, above(x, goal)) & some;
    const int at = past ? __ffs(past) - 1 : max(31 - __clz(some), 0);
    const Sum before = from_lane(x, max(at - 1, 0));
    if (at) base = before;
    return at;
}

// The residual that the cluster sums up: of node `at`; F as two numbers; gone: picked tokens that are out of it.
struct Residual {
    const float* p;
    const float* q;             // null: F = 0
    float fh, fl;
    const int32_t* gone;
    int n_gone;
};
// A probability that is negative or not finite counts as 0 (as whole numbers, those, with a sign or all of the exponent, are the larger).
__device__ __forceinline__ float counted(float x) { return __float_as_uint(x) < 0x7f800000u ? x : 0.f; }
// p - F q as two numbers where it is positive: there p >= F q in fp32 too, so that the difference's rounding is two subtractions
__device__ __forceinline__ Sum left_of(float p, float q, float fh, float fl) {
    const float ph = __fmul_rn(fh, q), pl = __fmaf_rn(fl, q, __fmaf_rn(fh, q, -ph));
    const float d = __fsub_rn(p, ph);
    return {d, __fsub_rn(__fsub_rn(__fsub_rn(p, d), ph), pl)};
}
// w = max(0, p - F q) added to s (p not finite: w is NaN, and adds nothing)
__device__ __forceinline__ void add_weight(Sum& s, const Residual& r, float p, float q) {
    const Sum w = left_of(p, counted(q), r.fh, r.fl);
    if (weighs(w)) add(s, w.h, w.l);
}
__device__ __forceinline__ void add_plain(Sum& s, float p) { add(s, counted(p), 0.f); }
__device__ __forceinline__ bool is_gone(const Residual& r, int e) {
    for (int g = 0; g < r.n_gone; ++g)
        if (r.gone[g] == e) return true;
    return false;
}
// The sum of the calling warp over elements [e0, e1). vec: the rows are 16-byte aligned, and e0 a multiple of 4.
__device__ __forceinline__ Sum part_sum(const Residual& r, int e0, int e1, bool vec) {
    constexpr int U = 4;
    const int lane = threadIdx.x & 31;
    Sum s[U] = {};
    bool drops = false;
    for (int g = lane; g < r.n_gone; g += 32) drops |= r.gone[g] >= e0 && r.gone[g] < e1;
    drops = __any_sync(0xffffffffu, drops);
    if (vec && !drops) {
        for (int e = e0 + lane * 4; e < e1; e += U * 128) {
            float4 p[U], q[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                // (a row's end is a multiple of 4 where rows are aligned)
                const bool there = e + k * 128 < e1;
                p[k] = there ? __ldg(reinterpret_cast<const float4*>(r.p + e + k * 128)) : make_float4(0.f, 0.f, 0.f, 0.f);
                q[k] = there && r.q ? __ldg(reinterpret_cast<const float4*>(r.q + e + k * 128)) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            if (!r.q) {
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    add_plain(s[k], p[k].x);
                    add_plain(s[k], p[k].y);
                    add_plain(s[k], p[k].z);
                    add_plain(s[k], p[k].w);
                }
                continue;
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                add_weight(s[k], r, p[k].x, q[k].x);
                add_weight(s[k], r, p[k].y, q[k].y);
                add_weight(s[k], r, p[k].z, q[k].z);
                add_weight(s[k], r, p[k].w, q[k].w);
            }
        }
    } else {
        constexpr int N = 8;
        for (int e = e0 + lane; e < e1; e += N * 32) {
            float p[N], q[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const bool there = e + k * 32 < e1;
                p[k] = there ? __ldg(r.p + e + k * 32) : 0.f;
                q[k] = there && r.q ? __ldg(r.q + e + k * 32) : 0.f;
            }
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (!drops || !is_gone(r, e + k * 32)) add_weight(s[k % U], r, p[k], q[k]);
        }
    }
#pragma unroll
    for (int k = 1; k < U; ++k) add(s[0], s[k].h, s[k].l);
    return warp_total(s[0]);
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// The CTAs' sums of one turn go from each to all, 8 bytes that count towards the receiver's barrier: one trip through the cluster, where a
// barrier of the cluster and a read take three (1.0 and 0.4 us against 0.4).
__device__ __forceinline__ void send(const Sum& s, Sum* to, uint64_t* bar, uint32_t rank) {
    uint32_t at, there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(to)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_u32(bar)), "r"(rank));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(at), "f"(s.h), "f"(s.l), "r"(there) : "memory");
}
__device__ __forceinline__ bool received(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Waits for them, up to two seconds.
__device__ __forceinline__ bool receive(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < 64; ++i)
        if (received(bar, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
    while (!received(bar, parity))
        if (globaltimer_ns() - t0 > kTimeoutNs) return false;
    return true;
}

enum { kSum, kLast, kNone };    // what warp 0 asks of the CTA: a residual's sum; the last one, with the token; nothing more
enum { kGoOn, kSearch, kDone, kGaveUp };        // what it found after the cluster's sum: the token is in this CTA's part; nothing more to do

// The token at which the running sum passes goal, in warp w's part [s0, s1) behind base: the CTA's warps sum up sixteenths, and
// warp 0 goes through one of them, 32 elements at a time.
__device__ __forceinline__ void find_token(const Residual& r, int s0, int s1, Sum base, const Sum& goal, Sum* of_warp, int32_t* token) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each = (s1 - s0 + kWarps - 1) / kWarps;
    const Sum mine = part_sum(r, min(s0 + warp * each, s1), min(s0 + (warp + 1) * each, s1), false);
    if (lane == 0) of_warp[warp] = mine;
    __syncthreads();
    if (warp) return;
    const int k = part_of(lane < kWarps ? of_warp[lane] : Sum{0.f, 0.f}, kWarps, goal, base);
    const int end = min(s0 + (k + 1) * each, s1);
    int found = -1;
    for (int e0 = min(s0 + k * each, s1); e0 < end; e0 += 128) {
        float p[4], q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = e0 + i * 32 + lane;
            p[i] = e < end ? __ldg(r.p + e) : 0.f;
            q[i] = e < end && r.q ? __ldg(r.q + e) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = e0 + i * 32 + lane;
            Sum w = {0.f, 0.f};
            if (e < end && !is_gone(r, e)) add_weight(w, r, p[i], q[i]);
            const unsigned some = __ballot_sync(0xffffffffu, weighs(w));
            if (!some) continue;
            const Sum upto = warp_upto(w);
            Sum x = base;
            add(x, upto.h, upto.l);
            const unsigned past = __ballot_sync(0xffffffffu, above(x, goal)) & some;
            found = e0 + i * 32 + (past ? __ffs(past) - 1 : 31 - __clz(some));
            if (past) {
                if (lane == 0) *token = found;
                return;
            }
            base = from_lane(x, 31);
        }
    }
    if (lane == 0) *token = max(found, 0);
}

__global__ void __launch_bounds__(kThreads, 2) tree_sample_kernel(const SampleArgs a) {
    __shared__ int32_t up[kMaxNodes], tok[kMaxNodes], first[kMaxNodes], list[kMaxNodes];
    __shared__ float u[kMaxNodes], px[kMaxNodes], qx[kMaxNodes];
    __shared__ Sum of_warp[2][kWarps];
    __shared__ __align__(8) Sum of_cta[2][kMaxCluster];
    __shared__ __align__(8) uint64_t bars[2];
    __shared__ Residual todo;
    __shared__ int what, steps, found, from_warp;
    __shared__ Sum from_base, goal;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = cluster_rank(), ctas = cluster_size();
    const int b = blockIdx.x / ctas;
    if (tid == 0) {
        mbar_init(smem_u32(bars), 1);
        mbar_init(smem_u32(bars + 1), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cluster_arrive();       // (before anything is sent, every CTA's barriers are there)
    pdl_wait();
    pdl_trigger();
    const float* target = a.target + (size_t)b * a.n_max * a.vocab;
    const float* draft = a.draft ? a.draft + (size_t)b * a.draft_rows * a.vocab : nullptr;
    // (rows past the tree's nodes are fetched with the others, and stay without effect: two trips to memory, not three)
    const int told = a.n_nodes[b];
    for (int i = tid; i < a.n_max; i += kThreads) first[i] = a.n_max;
    __syncthreads();
    bool odd = false, twisted = false;
    for (int i = tid; i < a.n_max; i += kThreads) {
        int p = a.parents[(size_t)b * a.n_max + i];
        const int x = a.tokens[(size_t)b * a.n_max + i];
        const float r = a.u[(size_t)b * a.n_max + i];
        const bool in = x >= 0 && x < a.vocab, wrong = i == 0 ? p != -1 : (p < -1 || p >= i);
        if (wrong) p = -1;
        px[i] = p >= 0 && in ? counted(target[(size_t)p * a.vocab + x]) : 0.f;
        qx[i] = p >= 0 && in && draft ? counted(draft[(size_t)p * a.vocab + x]) : 0.f;
        up[i] = i < told ? p : -1;
        tok[i] = in ? x : -1;
        u[i] = r > 0.f ? fminf(r, 0x1.fffffep-1f) : 0.f;
        if (i < told) {
            odd |= i > 0 && !in;
            twisted |= wrong;
            if (p >= 0) atomicMin(&first[p], i);
        }
    }
    const int n = min(max(told, 0), a.n_max);
    const bool bad = told != n || twisted;
    if (bad && rank == 0 && a.err) atomicOr(a.err, DFLARE_DEVERR_TREE);
    if (odd && rank == 0 && a.err) atomicOr(a.err, DFLARE_DEVERR_TOKEN);
    if (n == 0) {       // (the same in every CTA of the cluster)
        if (rank == 0) {
            if (tid == 0) {
                a.accept_len[b] = 0;
                a.next_token[b] = -1;
            }
            for (int i = tid; i < a.n_max; i += kThreads) a.path[(size_t)b * a.n_max + i] = -1;
        }
        return;
    }
    __syncthreads();

    cluster_wait();
    // ---------------- warp 0 walks; the others sum what it asks for. Every CTA of the cluster finds the same.
    int at = 0, i = first[0], walked = 1, turn = 0;
    const Sum one = {1.f, 0.f}, zero = {0.f, 0.f};
    Sum F = zero, W = one, Q = one;
    bool again = false;         // the last residual was empty: p instead
    bool lost = false;          // a wait gave up
    if (tid == 0 && rank == 0) a.path[(size_t)b * a.n_max] = 0;
    for (;; ++turn) {
        if (warp == 0) {
            int ask = again ? kLast : kNone;
            while (ask == kNone && !lost) {
                if (i >= n) {
                    ask = kLast;
                    break;
                }
                bool keep;
                float w = 0.f;
                if (i == first[at]) {
                    // u q < p, or u < p where drafts were picked: the sign of an fp32 fused product is exact
                    keep = draft ? fmaf(u[i], qx[i], -px[i]) < 0.f : u[i] < px[i];
                    w = px[i];
                } else if (draft) {
                    // u (q / Q) W < p - F q, times Q
                    const Sum rest = left_of(px[i], qx[i], F.h, F.l);
                    const float uq = __fmul_rn(u[i], qx[i]);
                    keep = __fadd_rn(rest.h, rest.l) > 0.f;
                    if (keep && Q.h > 0.f) keep = above(times(settled(rest.h, rest.l), Q), times({uq, __fmaf_rn(u[i], qx[i], -uq)}, W));
                } else {
                    bool before = false;        // the same token was picked before
                    for (int j = at + 1 + lane; j < i; j += 32) before |= up[j] == at && tok[j] == tok[i];
                    w = __any_sync(0xffffffffu, before) ? 0.f : px[i];
                    keep = above({w, 0.f}, times(W, {u[i], 0.f}));
                }
                if (keep) {
                    at = i;
                    i = first[at];
                    if (lane == 0 && rank == 0) a.path[(size_t)b * a.n_max + walked] = at;
                    ++walked;
                    F = zero;
                    W = Q = one;
                    continue;
                }
                int j = n;      // the next child
                for (int j0 = i + 1; j0 < n && j == n; j0 += 32) {
                    const unsigned hit = __ballot_sync(0xffffffffu, j0 + lane < n && up[j0 + lane] == at);
                    if (hit) j = j0 + __ffs(hit) - 1;
                }
                if (draft) {
                    if (Q.h > 0.f) {
                        const Sum more = over(W, Q);
                        add(F, more.h, more.l);
                        F = F.h < 3e38f ? settled(F.h, F.l) : Sum{3e38f, 0.f};
                    }
                    if (a.distinct) {
                        add(Q, -qx[i], 0.f);
                        Q = settled(Q.h, Q.l);
                    }
                    if (j < n) ask = kSum;
                } else {
                    add(W, -w, 0.f);
                    W = settled(W.h, W.l);
                }
                i = j;
            }
            int gone = 0;
            if (!draft && ask == kLast && !again && first[at] < n) {        // the picked tokens
                for (int j0 = at + 1; j0 < n; j0 += 32) {
                    const bool mine = j0 + lane < n && up[j0 + lane] == at;
                    const unsigned hit = __ballot_sync(0xffffffffu, mine);
                    if (mine) list[gone + __popc(hit & ((1u << lane) - 1u))] = tok[j0 + lane];
                    gone += __popc(hit);
                }
            }
            if (lane == 0) {
                const bool less = draft && F.h > 0.f && !again;
                todo.p = target + (size_t)at * a.vocab;
                todo.q = less ? draft + (size_t)at * a.vocab : nullptr;
                todo.fh = less ? F.h : 0.f;
                todo.fl = less ? F.l : 0.f;
                todo.gone = list;
                todo.n_gone = gone;
                what = lost ? kNone : ask;
                steps = walked;
            }
        }
        __syncthreads();
        if (what == kNone) break;
        const Residual r = todo;
        const bool last = what == kLast;
        const bool vec = a.vocab % 4 == 0 && ((reinterpret_cast<uintptr_t>(r.p) | reinterpret_cast<uintptr_t>(r.q)) & 15u) == 0;
        const long long from = ((long long)rank * kWarps + warp) * a.part;
        const int e0 = (int)min(from, (long long)a.vocab), e1 = (int)min(from + a.part, (long long)a.vocab);
        const Sum mine = part_sum(r, e0, e1, vec);
        if (lane == 0) of_warp[turn & 1][warp] = mine;
        __syncthreads();
        if (warp == 0) {
            const Sum own = warp_total(lane < kWarps ? of_warp[turn & 1][lane] : Sum{0.f, 0.f});
            const uint32_t bar = smem_u32(bars + (turn & 1));
            if (lane == 0) mbar_expect_tx(bar, ctas * (uint32_t)sizeof(Sum));
            if (lane < (int)ctas) send(own, &of_cta[turn & 1][rank], bars + (turn & 1), lane);
            // (a slot is written again two turns on, by a CTA that has had this one's sum of the turn between)
            const bool there = __all_sync(0xffffffffu, receive(bar, (uint32_t)(turn >> 1) & 1u));
            const Sum part = lane < (int)ctas ? of_cta[turn & 1][lane] : Sum{0.f, 0.f};
            W = warp_total(part);
            W = settled(W.h, W.l);
            int next = there ? kGoOn : kGaveUp;
            if (last && there) {
                if (!(W.h > 0.f) && !again && (r.q || r.n_gone)) {
                    again = true;
                } else if (!(W.h > 0.f)) {
                    next = kDone;
                    if (rank == 0 && lane == 0) {       // no weight at all
                        a.next_token[b] = 0;
                        if (a.err) atomicOr(a.err, DFLARE_DEVERR_TOKEN);
                    }
                } else {
                    const Sum g = times(W, {u[0], 0.f});
                    Sum base = {0.f, 0.f};
                    next = part_of(part, (int)ctas, g, base) == (int)rank ? kSearch : kDone;
                    if (next == kSearch) {
                        const int w = part_of(lane < kWarps ? of_warp[turn & 1][lane] : Sum{0.f, 0.f}, kWarps, g, base);
                        if (lane == 0) {
                            from_warp = w;
                            from_base = base;
                            goal = g;
                        }
                    }
                }
            }
            lost = !there;
            if (lane == 0) found = next;
        }
        if (!last) continue;        // (the others wait for what is asked next)
        __syncthreads();
        if (found == kSearch) {
            const long long f0 = ((long long)rank * kWarps + from_warp) * a.part;
            find_token(r, (int)min(f0, (long long)a.vocab), (int)min(f0 + a.part, (long long)a.vocab), from_base, goal, of_warp[(turn & 1) ^ 1], a.next_token + b);
        }
        if (found != kGoOn) break;
    }
    const bool gave_up = what == kNone || found == kGaveUp;
    if (rank == 0 && !gave_up) {
        if (tid == 0) a.accept_len[b] = steps;
        for (int x = steps + tid; x < a.n_max; x += kThreads) a.path[(size_t)b * a.n_max + x] = -1;
    }
    __syncwarp();
    cluster_arrive();       // (what it has stored lies behind this)
    if (gave_up) {
        // No CTA that gave up ends while another may still send it its sum. Others may have had all of theirs and
        // stored a walk and a token: the tree has none, whichever CTA it was.
        cluster_wait();
        if (tid == 0) {
            if (a.err) atomicOr(a.err, DFLARE_DEVERR_TIMEOUT);
            a.accept_len[b] = 0;
            a.next_token[b] = -1;
        }
        for (int x = tid; x < a.n_max; x += kThreads) a.path[(size_t)b * a.n_max + x] = -1;
    }
    // (a CTA that has had every other's sum of the last turn is sent no more)
}

// CTAs per tree: those that take the least time by a model of it, waves of clusters x (what a tree costs beside its rows, in elements of a
// row's part, and the part). How many clusters the GPU holds at once depends on its clusters of SMs: of 16 CTAs 14, not
// 304 / 16 (16 trees in clusters of 16 then go in two waves).
constexpr int kTreeCost = 20000;
cudaError_t cluster_for(int batch, int vocab, int* ctas) {
    static std::atomic<int> known[64][kMaxCluster + 1];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    double best = 0.0;
    for (int c = 1; c <= kMaxCluster; ++c) {
        if (c > 1 && vocab < c * kThreads * 4) break;      // less than a load for every thread
        int active = known[dev & 63][c].load(std::memory_order_relaxed);
        if (active == 0) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(c);
            cfg.blockDim = dim3(kThreads);
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = c;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            e = cudaOccupancyMaxActiveClusters(&active, tree_sample_kernel, &cfg);
            if (e != cudaSuccess) return e;
            active = std::max(active, 1);
            known[dev & 63][c].store(active, std::memory_order_relaxed);
        }
        const double cost = (double)((batch + active - 1) / active) * (kTreeCost + (double)vocab / c);
        if (c == 1 || cost < best) {
            best = cost;
            *ctas = c;
        }
    }
    return cudaSuccess;
}

dflare_status refuse(dflare_status st, const std::string& m) {
    noalloc_set_error(m);
    return st;
}

}  // namespace
}  // namespace dfl

using namespace dfl;

extern "C" dflare_status dflare_tree_sample(const int32_t* tokens_dev, const int32_t* parents_dev, const int32_t* n_nodes_dev,
                                            const float* target_dev, const float* draft_dev, int draft_rows, const float* u_dev,
                                            int batch, int n_max, int vocab, int distinct, int32_t* accept_len_dev, int32_t* path_dev,
                                            int32_t* next_token_dev, uint32_t* err_dev, void* stream) {
    auto bad = [](const char* m) { return refuse(DFLARE_EINVAL, std::string("dflare_tree_sample: ") + m); };
    if (!tokens_dev || !parents_dev || !n_nodes_dev || !target_dev || !u_dev || !accept_len_dev || !path_dev || !next_token_dev)
        return bad("NULL argument");
    if (batch < 1 || batch > 65535 || n_max < 1 || n_max > kMaxNodes) return bad("batch must be in [1, 65535], n_max in [1, 1024]");
    if (vocab < 1 || vocab > (1 << 28)) return bad("vocab must be in [1, 2^28]");
    if (draft_dev && draft_rows < n_max - 1) return bad("every node but the last needs a row of the draft's probabilities");
    if (distinct != 0 && distinct != 1) return bad("distinct must be 0 or 1");
    static PerDeviceOnce once;
    cudaError_t e = once([] { return cudaFuncSetAttribute(tree_sample_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1); });
    int ctas = 1;
    if (e == cudaSuccess) e = cluster_for(batch, vocab, &ctas);
    if (e != cudaSuccess) return refuse(DFLARE_ECUDA, std::string("dflare_tree_sample: ") + cudaGetErrorString(e));
    SampleArgs a{tokens_dev, parents_dev, n_nodes_dev, target_dev, draft_dev, u_dev, accept_len_dev, path_dev, next_token_dev, err_dev,
                 n_max, draft_rows, vocab, distinct, 0};
    a.part = ((vocab + ctas * kWarps - 1) / (ctas * kWarps) + 3) / 4 * 4;
    e = launch_cluster(true, ctas, tree_sample_kernel, dim3((unsigned)(batch * ctas)), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), a);
    return e == cudaSuccess ? DFLARE_OK : refuse(DFLARE_ECUDA, std::string("dflare_tree_sample: ") + cudaGetErrorString(e));
}
