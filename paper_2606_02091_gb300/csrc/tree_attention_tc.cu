// Attention of a tree over a paged cache for many query rows per kv head, bf16, on the fifth-generation
// tensor cores (tcgen05). How the keys are divided among the CTAs: tree_sched.cuh; what a row's unseen keys
// must not do: tree_attention.cu.
//
// Per 128-key tile and 128 query rows (M 128: thread r of a softmax warpgroup = query row r = TMEM lane r):
//   S = Q K^T   M 128 x N 128 x K head_dim, Q and K K-major in 128-byte-swizzled shared memory, S in TMEM;
//   softmax     P = 2^(s - m) rounded to bf16 over the first half of S's columns, the row sum from fp32 P;
//   O += P V    M 128 x N head_dim x K 128 with P read from TMEM, V MN-major as TMA wrote it, O in TMEM.
// Two streams, each a softmax warpgroup with its own S/P and O columns and its own (m, l), keep the tensor pipe
// busy while the other's scores are turned into weights. With 128 rows or fewer (NQ = 1) the streams take
// alternate key tiles of the same rows and are joined per row at the end; with more (NQ = 2) each has 128 rows
// of its own and both read every tile, so 256 rows cost one pass over the keys. Over a plan's items a kernel with NQ = 2 does
// either, unit by unit (two layers of 64 sequences of 4 nodes, their own 1150 keys and four shared contexts of 32768: 411 us with one
// stream idle in units of few rows, 377 so).
// m is raised (and O scaled) only when a tile's maximum exceeds it by 2^8: P <= 2^8 carries the same relative
// precision, and O / l does not depend on m.
// Bound by the chain of hand-offs between softmax and MMA (1.7 us per tile of 256 rows against 1.46 us of HBM time):
// measured, 64 nodes over 8 x 32768 keys, 32/8 heads of 128: 200 us in runs of 4 ms, 5.4 TB/s and 1370 TFLOP/s at once;
// 224 us for seconds on end, 4.8 TB/s and 1230 TFLOP/s, under the power cap (1.37 kW) at a median of 1590 MHz. For short
// contexts by latency, 16 nodes over contexts of 1355 to 3853 keys 19.7 us.
// One thread issues all MMAs in the order PV(i), S(i + 2): MMAs of one thread complete in order, so S(i + 2) may
// overwrite the columns of P(i) without a wait, and the barrier of S(i + 2) also says that PV(i) is done.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "paged.h"
#include "tree_sched.cuh"
#include "umma.cuh"

namespace dfl {
namespace {

constexpr int kKeys = kTcKeys;
constexpr int kThreads = 352;       // warps 0-3, 4-7: softmax streams; 8, 10: TMA of K, V; 9: MMA and tensor memory
constexpr float kRaise = 8.0f;      // growth (log2) of a row's maximum that rescales O

template <int HD, int NQ>
struct TcLayout {
    static constexpr uint32_t TB = HD * 256;                        // a 128-key tile of K or V
    static constexpr int NK = HD == 64 ? 4 : 2;                     // K slots
    static constexpr int NV = HD == 64 ? 4 : 2;                     // V slots
    static constexpr uint32_t Q = 0;                                // [NQ][HD / 64][128 rows][128 B]
    static constexpr uint32_t K = NQ * TB;                          // [NK][HD / 64][128][128 B]
    static constexpr uint32_t V = K + NK * TB;
    static constexpr uint32_t BARS = V + NV * TB;
    static constexpr int NBARS = 2 * NK + 2 * NV + 9;
    static constexpr uint32_t ML = BARS + ((NBARS * 8 + 15) & ~15);    // NQ == 1: [2][128] (m, l) of the streams
    static constexpr uint32_t END = (ML + (NQ == 1 ? 2048 : 0) + 15) & ~15u;
    static constexpr uint32_t TURN = END;                           // 4 KB for each softmax warp to turn its rows around
    static constexpr uint32_t BYTES = END + 32768;
};

// MN-major operand (V): 64-element swizzle atoms along N `atom` bytes apart, 8-key groups 1024 bytes apart
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t saddr, uint32_t atom) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(atom >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// D += A B with A (16-bit, two per column) in tensor memory
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
        "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
// the maximum of three
__device__ __forceinline__ float max3(float a, float b, float c) {
    float v;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(a), "f"(b), "f"(c));
    return v;
}
// The softmax streams meet. What either has waited for in tensor memory (O after its last PV) or read there is in order with
// what the other does there next: tcgen05 operations keep the order of a barrier only between its two fences.
__device__ __forceinline__ void streams_meet() {
    tc_fence_before();
    asm volatile("bar.sync 1, 256;" ::: "memory");
    tc_fence_after();
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// SHARED: over the items of a plan (tree_shared.cu) instead of the batch's sequences and kv heads.
template <int HD, int NQ, bool SHARED>
__global__ void __launch_bounds__(kThreads, 1) tree_tc_kernel(const __grid_constant__ CUtensorMap mk,
                                                              const __grid_constant__ CUtensorMap mv, const TreeArgs a) {
    using LY = TcLayout<HD, NQ>;
    using Pair = std::conditional_t<SHARED, TreeItem, TreePair>;
    constexpr int NK = LY::NK, NV = LY::NV, QT = 128 * NQ;
    constexpr uint32_t TB = LY::TB;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int32_t cum[kMaxSeqs + 1];
    __shared__ uint32_t odd[kMaxNodes / 32];    // nodes with an infinite or NaN value
    __shared__ int odd_any;
    __shared__ volatile int abort_flag;
    __shared__ uint32_t tmem_base;
    __shared__ int planes[2][2][32];            // of the K and of the V warp
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t sb = smem_u32(smem), bars = sb + LY::BARS;
    auto kfull = [&](int i) { return bars + 8u * i; };
    auto kempty = [&](int i) { return bars + 8u * (NK + i); };
    auto vfull = [&](int i) { return bars + 8u * (2 * NK + i); };
    auto vempty = [&](int i) { return bars + 8u * (2 * NK + NV + i); };
    auto sfull = [&](int w) { return bars + 8u * (2 * NK + 2 * NV + w); };       // S of stream w in TMEM
    auto pfull = [&](int w) { return bars + 8u * (2 * NK + 2 * NV + 2 + w); };   // its P written, O scaled
    auto ofull = [&](int w) { return bars + 8u * (2 * NK + 2 * NV + 4 + w); };   // its last PV of a pair done
    const uint32_t qfull = bars + 8u * (2 * NK + 2 * NV + 6);                    // Q of a pair in shared memory
    const uint32_t qsent = qfull + 8u;                                           // the first pair's Q is on its way
    const uint32_t drain = qfull + 16u;                                          // after a wait that gave up
    if (tid == 0) {
        for (int i = 0; i < NK; ++i) {
            mbar_init(kfull(i), 1);
            mbar_init(kempty(i), 1);
        }
        for (int i = 0; i < NV; ++i) {
            mbar_init(vfull(i), 1);
            mbar_init(vempty(i), 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(sfull(w), 1);
            mbar_init(pfull(w), 4);
            mbar_init(ofull(w), 1);
        }
        mbar_init(qfull, 8);
        mbar_init(qsent, 8);
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mk)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mv)) : "memory");
        abort_flag = 0;
        odd_any = 0;
    }
    if (tid < kMaxNodes / 32) odd[tid] = 0;
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    // A launch that follows one of the same call does not wait for that to end: what the call reads was there before the first
    // one let this one start, and the two write different rows. It waits at its own end, for the joining launch.
    if (!SHARED || !a.follows) pdl_wait();
    // Dependents start only once this CTA holds its tensor memory: one of theirs that takes tensor memory
    // before its own dependency wait can never hold columns that this CTA waits for. After this kernel's own
    // wait: the joining launch reads the lengths at once.
    pdl_trigger();
    int qg = 0, v, v1;
    if constexpr (SHARED) tree_items(a, v, v1);
    else tree_runs<QT, kKeys, kTcExtra, kTcLeast>(a, cum, qg, v, v1);
    const int v0 = v;
    // Whether the streams take alternate tiles of the same 128 rows: always (NQ = 1), or, from a plan, where a unit has no more.
    auto alternate = [&](const Pair& p) {
        if constexpr (SHARED) return p.nodes * a.G - p.row0 <= 128;
        else return NQ == 1;
    };
    Pair p, after;
    bool more = tree_pair<kTcExtra>(a, cum, v, v1, p);
    auto tS = [&](int w) { return tmem + 128u * w; };
    auto tO = [&](int w) { return tmem + 256u + (uint32_t)HD * w; };

    if (warp == 8 || warp == 10) {
        // ---------------- TMA: K tiles into their ring (warp 8) and V tiles into theirs (warp 10), a box being up to
        // 64 tokens x 64 head dims. In one warp K(i + 1) waits for the slot of V(i), which is free a tile's time later;
        // one thread that polls for either ring's slot slows the softmax warps (64 nodes over 8 x 32768 keys 211 us).
        const bool vs = warp == 10;
        const int N = vs ? NV : NK, rows = min(a.pg.ps, 64), boxes = kKeys / rows;
        const uint32_t full = vs ? vfull(0) : kfull(0), empty = vs ? vempty(0) : kempty(0), ring = sb + (vs ? LY::V : LY::K);
        const CUtensorMap* map = vs ? &mv : &mk;
        int i = 0;
        const bool ok = !more || each_group<kTcExtra>(a, cum, v, v1, p, kKeys, rows, lane, planes[vs], [&](int first, int n, const int* plane) {
            bool fine = true;
            if (elect_one()) {      // (a branch with a single active lane: copies issue from uniform registers)
                for (int tile = first; tile < first + n; ++tile, ++i, plane += boxes) {
                    // After the first K tile the first pair's queries: behind the whole ring they would arrive last
                    // (measured: 3.5 us later, the time in which 152 x 128 KB come from memory).
                    if (i == (vs ? 0 : 1)) fine = wait_inline(qsent, 0, &abort_flag, a.pg.err);
                    const int st = i % N;
                    if (i >= N && fine) fine = wait_inline(empty + 8 * st, (uint32_t)(i / N - 1) & 1u, &abort_flag, a.pg.err);
                    if (!fine) break;
                    const uint32_t bar = full + 8 * st, dst = ring + st * TB;
                    mbar_expect_tx(bar, TB);
                    for (int x = 0; x < boxes; ++x) {
                        const int z = plane[x], y = (tile * kKeys + x * rows) & (a.pg.ps - 1);
#pragma unroll
                        for (int h = 0; h < HD / 64; ++h) tma_load_3d(dst + h * 16384 + x * rows * 128, map, h * 64, y, z, bar);
                    }
                }
            }
            return (bool)__all_sync(0xffffffffu, fine);
        });
        if (!ok) {      // the copies in flight land before the CTA's shared memory is given up (i: the issuing lane's)
            volatile int never = 0;
            for (int j = max(0, i - N); j < i; ++j) wait_inline(full + 8 * (j % N), (uint32_t)(j / N) & 1u, &never, a.pg.err);
        }
        __syncwarp();
    } else if (warp == 9) {
        if (elect_one()) {
            // ---------------- MMA issue. Steps of a pair: with NQ = 2 (tile t, stream w) in the order 2 t + w,
            // with NQ = 1 tile t on stream t % 2. PV(i), then S(i + 2).
            constexpr uint32_t kId = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);
            constexpr uint32_t kIdS = kId | ((128u >> 3) << 17), kIdO = kId | (1u << 16) | (((uint32_t)HD >> 3) << 17);
            bool ok = true;
            uint32_t base = 0;              // tiles of the pairs before this one
            uint32_t ps0 = 0, ps1 = 0;      // P handed over by each stream
            uint32_t pair = 0;
            auto wait = [&](uint32_t bar, uint32_t parity) {
                if (ok) ok = wait_inline(bar, parity & 1u, &abort_flag, a.pg.err);
            };
            // S of tile x of the run by stream w (a constant where it is called, as alt is but for SHARED)
            auto issue_s = [&](uint32_t x, int w, bool alt) {
                const uint32_t st = x % NK;
                if (alt || w == 0) wait(kfull(st), x / NK);
                if (!ok) return;
                tc_fence_after();
                const uint64_t dq = smem_desc(sb + LY::Q + (alt ? 0 : w * TB));
                const uint64_t dk = smem_desc(sb + LY::K + st * TB);
#pragma unroll
                for (int kk = 0; kk < HD / 16; ++kk) {
                    const uint64_t at = (uint64_t)((kk >> 2) * (16384 / 16) + (kk & 3) * 2);
                    umma_bf16(tS(w), dq + at, dk + at, kIdS, kk > 0 ? 1u : 0u);
                }
                umma_commit(sfull(w));
                if (alt || w == 1) umma_commit(kempty(st));
            };
            TreeRaw raw = more ? pair_raw(a, p) : TreeRaw{};
            for (; more; ++pair) {
                const int n = p.hi - p.lo;
                int nodes, ctx, keys;
                pair_lengths<SHARED>(a, raw, nodes, ctx, keys);
                const bool next = tree_pair<kTcExtra>(a, cum, v, v1, after);
                if (next) raw = pair_raw(a, after);
                // PV of tile j of the pair by stream w, then the stream's next S
                const bool alt = alternate(p);
                const int stride = alt ? 2 : 1;
                auto step = [&](int j, int w) {
                    const uint32_t x = base + j, st = x % NV;
                    if (alt || w == 0) wait(vfull(st), x / NV);
                    wait(pfull(w), w ? ps1++ : ps0++);
                    if (!ok) return;
                    tc_fence_after();
                    const uint64_t dv = smem_desc_mn(sb + LY::V + st * TB, 16384);
                    // (weights and values past the last key are not multiplied, up to the 16 of a step)
                    const int ks = min(kKeys / 16, (keys - (p.lo + j) * kKeys + 15) / 16);
#pragma unroll
                    for (int kk = 0; kk < kKeys / 16; ++kk)
                        if (kk < ks) umma_bf16_ts(tO(w), tS(w) + kk * 8, dv + (uint64_t)(kk * 128), kIdO, (j >= stride || kk > 0) ? 1u : 0u);
                    if (alt || w == 1) umma_commit(vempty(st));
                    if (j + stride < n) issue_s(x + stride, w, alt);
                    else umma_commit(ofull(w));
                };
                wait(qfull, pair);
                if (ok) tc_fence_after();
                issue_s(base, 0, alt);
                if (!alt) issue_s(base, 1, alt);
                else if (n > 1) issue_s(base + 1, 1, alt);
                for (int j = 0; j < n && ok; j += stride) {
                    step(j, 0);
                    if (!alt || j + 1 < n) step(alt ? j + 1 : j, 1);
                }
                if (!ok) break;
                base += n;
                more = next;
                p = after;
            }
            // every MMA has completed before the tensor memory is given up: the softmax streams have waited
            // for the last ones, except after a wait that gave up
            if (!ok) {
                umma_commit(drain);
                volatile int never = 0;
                wait_inline(drain, 0, &never, a.pg.err);
            }
        }
        __syncwarp();
    } else {
        // ---------------- softmax stream w (warps 4 w .. 4 w + 3). After a wait that gave up the warps go on
        // without waiting: results are invalid, the error is set, and every barrier still meets. Code that a
        // pair runs once or twice is kept in loops: under the key stream an instruction cache miss takes
        // microseconds too.
        const int w = warp >> 2, r = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        auto row0_of = [&](const Pair& p) {     // the first row of the block
            if constexpr (SHARED) return p.row0;
            else return qg * QT;
        };
        bool ok = true;
        int base = 0, ss = 0, os = 0;
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (ok) ok = __all_sync(0xffffffffu, wait_inline(bar, parity, &abort_flag, a.pg.err));
        };
        // Q of a pair, asynchronously, by `many` threads (this one the who-th), 128 rows from the block's row 128 x half
        // on: pieces of eight elements, swizzled; rows past R are never looked at
        auto load_q = [&](const Pair& p, int R, int half, int who, int many) {
            constexpr int PC = HD / 8;
            const int pc = who % PC, q0 = row0_of(p) + 128 * half;
            const uint32_t dst = sb + LY::Q + (uint32_t)half * TB + (pc >> 3) * 16384;
            const bf16* src = static_cast<const bf16*>(a.q) + (SHARED ? 0 : (size_t)p.b * a.n_max * a.q_row) + (size_t)(p.h * a.G) * HD + pc * 8;
#pragma unroll 4
            for (int lr = who / PC; lr < 128; lr += many / PC) {
                const int rr = q0 + lr, nd = group_of(a, rr);
                if (rr < R)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + lr * 128 + (((pc & 7) ^ (lr & 7)) << 4)),
                                 "l"(src + (SHARED ? query_row(a, p, nd) : (size_t)nd) * a.q_row + (rr - nd * a.G) * HD) : "memory");
            }
        };
        auto q_there = [&]() {      // this thread's part of Q is in shared memory, for the MMAs to read
            asm volatile("cp.async.wait_all;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(qfull);
        };
        TreeRaw raw{};
        int nodes = 0, ctx = 0, keys = 0;
        if (more) {
            raw = pair_raw(a, p);
            pair_lengths<SHARED>(a, raw, nodes, ctx, keys);
            if (!alternate(p)) load_q(p, nodes * a.G, w, r, 128);
            else load_q(p, nodes * a.G, 0, tid, 256);
            __syncwarp();
            if (lane == 0) mbar_arrive(qsent);
            q_there();
            // qfull counts arrivals and not whose they are: without this a stream that has no tile of the first pair would go on to arrive for
            // the second, and the first S could be computed before the other stream's part of Q is there. (A pair ends with the streams
            // meeting, so its successor's Q is complete before one of them can arrive for a third; streams that do not alternate have a tile each.)
            if (alternate(p)) streams_meet();
        }
        while (more) {
            const int n = p.hi - p.lo;
            const int R = nodes * a.G;
            const bool alt = alternate(p);
            const int my_row = row0_of(p) + (alt ? 0 : 128 * w) + r;
            const bool live = my_row < R;
            const bool warp_live = my_row - lane < R;
            const int node = mask_node(p, group_of(a, min(my_row, R - 1)));
            const SeenRow row = seen_row(a, p.b, node);
            more = tree_pair<kTcExtra>(a, cum, v, v1, after);
            if (more) raw = pair_raw(a, after);
            int nodes2 = 0, ctx2 = 0, keys2 = 0;        // the next pair's
            float m = -INFINITY, l = 0.f;
            const int mine = alt ? (n + 1 - w) / 2 : n;      // tiles of this stream
            for (int j = 0; j < mine; ++j, ++ss) {
                const int tile = alt ? 2 * j + w : j;       // of the pair's run
                const int k0 = (p.lo + tile) * kKeys;
                wait(sfull(w), (uint32_t)ss & 1u);
                tc_fence_after();
                // every S of the pair (of this stream, where each has rows of its own) has been computed: the next pair's Q
                if (tile == n - 1 && more) {
                    pair_lengths<SHARED>(a, raw, nodes2, ctx2, keys2);
                    if constexpr (SHARED) {
                        if (alt == alternate(after)) {
                            load_q(after, nodes2 * a.G, alt ? 0 : w, r, 128);
                        } else if (alt) {       // (this stream had the last S that reads either half)
                            load_q(after, nodes2 * a.G, 0, r, 128);
                            load_q(after, nodes2 * a.G, 1, r, 128);
                        } else if (w == 0) {
                            load_q(after, nodes2 * a.G, 0, r, 128);
                        }
                    } else {
                        load_q(after, nodes2 * a.G, NQ == 2 ? w : 0, r, 128);
                    }
                }
                const bool edge = k0 + kKeys > ctx;
                if (edge) {
                    // nodes of the tree, or slots past the last key
                    if (alt || w == 0) {
                        // values: slots past the last key (of those that are multiplied) and infinite or NaN values
                        // of nodes become 0
                        const int x = base + tile, st = x % NV, rows = min(kKeys, (keys - k0 + 15) & ~15);
                        wait(vfull(st), (uint32_t)(x / NV) & 1u);
                        // (a thread's pieces lie 128 / (HD / 8) rows apart in the same place of the swizzle; four at a time)
                        constexpr int PC = HD / 8, STEP = 128 / PC;
                        const int pc = r % PC;
                        for (int kr = max(ctx - k0, 0) + r / PC; kr < rows; kr += 4 * STEP) {
                            uint4* at = reinterpret_cast<uint4*>(smem + LY::V + st * TB + (pc >> 3) * 16384 + kr * 128 + (((pc & 7) ^ (kr & 7)) << 4));
                            uint4 x[4];
#pragma unroll
                            for (int u = 0; u < 4; ++u) x[u] = kr + u * STEP < rows ? at[u * STEP * 8] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                const int key = k0 + kr + u * STEP;
                                bool bad = key >= keys;
                                if (bad) {
                                    x[u] = make_uint4(0u, 0u, 0u, 0u);
                                } else if (drop_odd(x[u])) {
                                    bad = true;
                                    atomicOr(&odd[(key - ctx) >> 5], 1u << ((key - ctx) & 31));
                                    odd_any = 1;
                                }
                                if (bad && kr + u * STEP < rows) at[u * STEP * 8] = x[u];
                            }
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                }
                if (edge && warp_live) {
                    // scores of unseen keys become -inf where they are (in the loop below a branch for it costs
                    // every tile 0.1 us, a second copy of the loop as much in registers)
#pragma unroll 1
                    for (int x = max(ctx - k0, 0) >> 5; x < 4; ++x) {
                        const uint32_t see = seen32(a, row, p.b, node, ctx, keys, k0 + 32 * x);
                        uint32_t s[32];
                        tmem_ld32_async(tS(w) + lanes + 32 * x, s);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[e] = see & (1u << e) ? s[e] : 0xff800000u;
                        tmem_st16(tS(w) + lanes + 32 * x, s);
                        tmem_st16(tS(w) + lanes + 32 * x + 16, s + 16);
                    }
                    tmem_wait_st();
                }
                if (warp_live) {
                    // One read of the row's scores, 32 at a time: weights against the maximum so far, and the
                    // tile's own maximum. Only where that is above the other by 2^8 the scores are read a second
                    // time. A pair's first tile goes by the maximum of its first 32 keys (by that of the first key
                    // alone, rows go on raising theirs: 248 us instead of 203 for 64 nodes over 8 x 32768 keys).
                    uint32_t pw[64];
                    uint64_t sum[2];
                    const uint64_t scale = pack2(a.scale_log2, a.scale_log2);
#pragma unroll 1
                    for (bool again = false;; again = true) {
                        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                        sum[0] = sum[1] = 0ull;
                        uint32_t s[2][32];
                        tmem_ld32_async(tS(w) + lanes, s[0]);
                        tmem_wait_ld();
                        if (__any_sync(0xffffffffu, m == -INFINITY)) {
                            float mx = -INFINITY;
#pragma unroll
                            for (int e = 0; e < 32; e += 2) mx = max3(mx, __uint_as_float(s[0][e]), __uint_as_float(s[0][e + 1]));
                            if (m == -INFINITY) m = mx * a.scale_log2;
                        }
                        const float neg1 = m == -INFINITY ? 0.f : -m;
                        const uint64_t neg = pack2(neg1, neg1);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            if (x) tmem_wait_ld();
                            if (x < 3) tmem_ld32_async(tS(w) + lanes + 32 * (x + 1), s[(x + 1) & 1]);
                            const uint32_t* v = s[x & 1];
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const float s0 = __uint_as_float(v[2 * e]), s1 = __uint_as_float(v[2 * e + 1]);
                                mx4[e & 3] = max3(mx4[e & 3], s0, s1);
                                float p0, p1;
                                unpack2(fma2(pack2(s0, s1), scale, neg), p0, p1);
                                p0 = pow2(p0);
                                p1 = pow2(p1);
                                sum[e & 1] = add2(sum[e & 1], pack2(p0, p1));
                                // (rounded to bf16, relative error 2^-8 at most: the operand type that goes with bf16
                                // values; the sum is of the unrounded ones)
                                pw[16 * x + e] = two_bf16(p0, p1);
                            }
                        }
                        if (again) break;
                        const float mx = fmaxf(max3(mx4[0], mx4[1], mx4[2]), mx4[3]) * a.scale_log2;
                        const bool raise = mx > m + kRaise;      // (also from -inf)
                        if (!__any_sync(0xffffffffu, raise)) break;
                        const float alpha = raise ? pow2(m - mx) : 1.0f;
                        if (j > 0) {    // (the stream's PV before S(i) has completed: its O is at rest)
#pragma unroll 1
                            for (int x = 0; x < HD / 16; ++x) {
                                uint32_t o[16];
                                tmem_ld16_async(tO(w) + lanes + 16 * x, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                                tmem_st16(tO(w) + lanes + 16 * x, o);
                            }
                        }
                        if (raise) {
                            l *= alpha;
                            m = mx;
                        }
                    }
                    // P over the first 64 columns of S, all of which has been read
#pragma unroll
                    for (int x = 0; x < 4; ++x) tmem_st16(tS(w) + lanes + 16 * x, pw + 16 * x);
                    float s0, s1;
                    unpack2(add2(sum[0], sum[1]), s0, s1);
                    l += s0 + s1;
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pfull(w));
            }
            if (more) {
                pair_lengths<SHARED>(a, raw, nodes2, ctx2, keys2);      // (the stream without the last tile too)
                q_there();      // the next pair's first S is computed while this one's rows are written
            }
            if (mine > 0) wait(ofull(w), (uint32_t)os++ & 1u);
            tc_fence_after();
            // ---------------- the pair's rows. NQ = 2: a thread has its row. NQ = 1: the streams swap (m, l)
            // and each joins one half of the head dims of both.
            bool partial;
            size_t part0;       // the block's first row among the partial results
            if constexpr (SHARED) {
                partial = p.dst >= 0;
                part0 = (size_t)max(p.dst, 0);
            } else {
                partial = p.partial();
                part0 = ((size_t)blockIdx.x * 2 + (p.start < v0 ? 0 : 1)) * QT;
            }
            float M = m, L = l, w0 = 1.f, w1 = 0.f;
            const bool two = alt && n > 1;
            if (alt) {
                // (with NQ = 2 there is room for it only where the warps turn their rows around)
                float2 *mine = reinterpret_cast<float2*>(smem + LY::ML) + w * 128 + r, *other = reinterpret_cast<float2*>(smem + LY::ML) + (w ^ 1) * 128 + r;
                if constexpr (NQ == 2) {
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
                    mine = reinterpret_cast<float2*>(smem + LY::TURN + warp * 4096) + lane;
                    other = reinterpret_cast<float2*>(smem + LY::TURN + (warp ^ 4) * 4096) + lane;
                }
                *mine = make_float2(m, l);
                streams_meet();     // (with it, each reads the O that the other has waited for)
                const float2 own = make_float2(m, l), there = *other, x = w ? there : own, y = w ? own : there;
                M = fmaxf(x.x, y.x);
                const float ref = M == -INFINITY ? 0.f : M;
                w0 = pow2(x.x - ref);
                w1 = pow2(y.x - ref);
                L = x.y * w0 + y.y * w1;
                if constexpr (NQ == 2) streams_meet();      // both have read
            } else {
                streams_meet();     // odd nodes noted by stream 0
            }
            const bool odds = odd_any != 0;
            if (warp_live) {
                // Each warp turns its 32 rows around in shared memory, 128 bytes of every row at a time, so that
                // global stores are whole lines.
                const float inv = partial ? 1.f : L == 0.f ? 0.f : 1.f / L;
                if (alt) {
                    w0 *= inv;
                    w1 *= inv;
                } else {
                    w0 = inv;
                }
                uint8_t* turn = smem + LY::TURN + warp * 4096;
                const int rows = min(32, R - (my_row - lane));
                const size_t prow = part0 + (alt ? 0 : 128 * w) + r;
                const size_t orow = ((size_t)p.b * a.n_max + node) * a.hq + p.h * a.G + min(my_row, R - 1) - node * a.G;
                const int CH = alt ? HD / 64 : HD / 32;
                const int col0 = alt ? w * (HD / 2) : 0;
#pragma unroll 1
                for (int x = 0; x < CH; ++x) {
                    const int col = col0 + 32 * x;
                    uint32_t v0[32];
                    float o[32];
                    tmem_ld32_async(tO(alt ? 0 : w) + lanes + col, v0);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(v0[e]) * w0;
                    if (two) {
                        tmem_ld32_async(tO(1) + lanes + col, v0);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = fmaf(__uint_as_float(v0[e]), w1, o[e]);
                    }
                    if (odds && live)       // infinite and NaN values of the nodes that this row sees
                        each_odd(a, odd, p, node, ctx, keys, [&](size_t at) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                const float f = to_f(static_cast<const bf16*>(a.pg.v)[at + col + e]);
                                if (!isfinite(f)) o[e] += f;
                            }
                        });
                    if (partial) {
                        // the block goes out as it lies here (32 rows x 128 bytes, swizzled) by one bulk copy
                        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                        __syncwarp();
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            *reinterpret_cast<float4*>(turn + lane * 128 + ((e ^ (lane & 7)) << 4)) =
                                make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], 4096;" ::"l"(a.part_o + (prow - lane) * HD + (col >> 5) * 1024),
                                         "r"(sb + LY::TURN + warp * 4096)
                                         : "memory");
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                    } else {
                        const int upper = CH > 1 ? x & 1 : 0;       // which half of a row's 128 bytes
                        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                        __syncwarp();
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint4 u;
                            u.x = two_bf16(o[8 * e], o[8 * e + 1]);
                            u.y = two_bf16(o[8 * e + 2], o[8 * e + 3]);
                            u.z = two_bf16(o[8 * e + 4], o[8 * e + 5]);
                            u.w = two_bf16(o[8 * e + 6], o[8 * e + 7]);
                            *reinterpret_cast<uint4*>(turn + lane * 128 + (((4 * upper + e) ^ (lane & 7)) << 4)) = u;
                        }
                        if (upper || CH == 1) {
                            const int pieces = CH > 1 ? 8 : 4;
                            __syncwarp();
#pragma unroll
                            for (int y = 0; y < 8; ++y) {
                                if (y == pieces) break;
                                const int lr = (32 / pieces) * y + lane / pieces, pc = lane % pieces;
                                const uint4 v = *reinterpret_cast<const uint4*>(turn + lr * 128 + ((pc ^ (lr & 7)) << 4));
                                const size_t to = __shfl_sync(0xffffffffu, orow, lr);
                                if (lr < rows)
                                    *reinterpret_cast<uint4*>(static_cast<bf16*>(a.out) + to * HD + col - 32 * upper + pc * 8) = v;
                            }
                            __syncwarp();
                        }
                    }
                }
                if (live && (!alt || w == 0)) {
                    if (partial) a.part_ml[prow] = make_float2(M, L);
                    else if (a.lse) a.lse[orow] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
                }
            }
            // O, the (m, l) exchange and the odd nodes are free for the next pair
            streams_meet();
            if (odds) {
                if (tid < kMaxNodes / 32) odd[tid] = 0;
                if (tid == 0) odd_any = 0;
                streams_meet();
            }
            base += n;
            p = after;
            nodes = nodes2;
            ctx = ctx2;
            keys = keys2;
        }
        // the partial results are in memory before this CTA ends (and with it what the joining launch waits for)
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (SHARED && a.follows) pdl_wait();
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <int HD, int NQ>
cudaError_t launch_tc(dflare_cache* c, TreeArgs& a, cudaStream_t s) {
    static PerDeviceOnce once;
    auto kernel = tree_tc_kernel<HD, NQ, false>;
    cudaError_t e = once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TcLayout<HD, NQ>::BYTES); });
    if (e != cudaSuccess) return e;
    a.QG = (a.n_max * a.G + 128 * NQ - 1) / (128 * NQ);
    a.C = c->num_sms;
    return launch_kernel(true, kernel, dim3(std::max(a.QG, a.C)), dim3(kThreads), TcLayout<HD, NQ>::BYTES, s, c->maps[0], c->maps[1], a);
}

template <int HD>
cudaError_t launch_items(dflare_cache* c, const TreeArgs& a, cudaStream_t s) {
    static PerDeviceOnce once;
    auto kernel = tree_tc_kernel<HD, 2, true>;
    cudaError_t e = once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TcLayout<HD, 2>::BYTES); });
    if (e != cudaSuccess) return e;
    return launch_kernel(true, kernel, dim3(a.C), dim3(kThreads), TcLayout<HD, 2>::BYTES, s, c->maps[0], c->maps[1], a);
}

}  // namespace

cudaError_t launch_tree_attention_tc(dflare_cache* c, TreeArgs& a, int* QT, cudaStream_t s) {
    const bool one = a.n_max * a.G <= 128;
    *QT = one ? 128 : 256;
    if (c->cfg.head_dim == 128) return one ? launch_tc<128, 1>(c, a, s) : launch_tc<128, 2>(c, a, s);
    return one ? launch_tc<64, 1>(c, a, s) : launch_tc<64, 2>(c, a, s);
}

cudaError_t launch_shared_tc(dflare_cache* c, const TreeArgs& a, cudaStream_t s) {
    return c->cfg.head_dim == 128 ? launch_items<128>(c, a, s) : launch_items<64>(c, a, s);
}

}  // namespace dfl
