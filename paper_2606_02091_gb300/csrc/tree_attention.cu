// Attention of a tree of nodes (or one token, or a chunk of a prompt) over a paged cache, for up to 16
// query rows per kv head in bf16, and for any number in fp32; more rows in bf16 go to tree_attention_tc.cu.
// How the keys are divided among the CTAs: tree_sched.cuh.
//
// One pass over the keys with the running maximum m and sum l of the softmax, in log2 units:
//   m' = max(m, max_j s_j),  l' = l 2^(m - m') + sum_j 2^(s_j - m'),  O' = O 2^(m - m') + sum_j 2^(s_j - m') v_j.
// A row's unseen keys get weight 0 by selection, whatever their score. Weight times value is not selected
// (0 x infinity would be NaN), so values that some row must not see are made harmless in shared memory before
// they are multiplied: slots past the last key become 0, and so do infinite and NaN values of tree nodes,
// whose nodes are noted; rows that do see such a node get its values added at the end.
#include <math.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "common.cuh"
#include "paged.h"
#include "tree_sched.cuh"
#include "umma.cuh"

namespace dfl {
namespace {

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// byte offset of 16-byte piece c of row r in a tile of 64 rows stored as [hd / 64][64][128 bytes], swizzled
__device__ __forceinline__ uint32_t tile_at(int r, int c) {
    return (uint32_t)((c >> 3) * 8192 + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}

// the four warps that compute (the fifth streams tiles)
__device__ __forceinline__ void compute_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

constexpr int kKeys = 64;           // keys per tile
constexpr int kRows = 16;
constexpr int kStages = 2;
constexpr int kMmaThreads = 160;
constexpr int kExtra = 3;       // see tree_sched.cuh
// 2 tiles of head_dim 128, 4 of 64: what the stages and a trip to memory hold anyway. Measured at 128 with 1, 2 and 4: 2048
// keys 9.5, 8.6 and 9.6 us, 300 keys 7.5, 7.5 and 9.0; at 64 with 2 and 4: 4096 keys 8.4 and 8.1.
template <int HD>
constexpr int kLeast = 256 / HD;

template <int HD>
struct MmaLayout {
    static constexpr uint32_t TB = HD * 128;                    // a tile of K or V
    static constexpr uint32_t Q = kStages * 2 * TB;             // two pairs' rows, [HD / 64][16][128 B] each
    static constexpr uint32_t SWAP = Q + 2 * kRows * HD * 2;    // [4 owners][3][HD / 32][32 lanes] float4
    static constexpr uint32_t BARS = SWAP + 4 * 3 * HD * 16;
    static constexpr uint32_t BYTES = BARS + 2 * kStages * 8;
};

// bf16, up to 16 query rows per kv head (single tokens, small trees). Four warps take 16 keys of each 64-key tile
// each; a fifth warp streams the tiles' pages by TMA into a ring of stages. Every warp keeps its own running
// maximum and sum; when a pair's keys are done each warp sums up a quarter of the head dims of all four.
// HBM-bound for long contexts (one token over 100000 keys, 8 kv heads of 128: 70 us, 5.9 TB/s); for short ones by
// its chain of latencies, lengths, page table, keys (2048 keys: 8.6 us).
template <int HD>
__global__ void __launch_bounds__(kMmaThreads, 2) tree_mma_kernel(const __grid_constant__ CUtensorMap mk,
                                                                  const __grid_constant__ CUtensorMap mv, const TreeArgs a) {
    using LY = MmaLayout<HD>;
    constexpr uint32_t TB = LY::TB;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int32_t cum[kMaxSeqs + 1];
    __shared__ uint32_t odd[kMaxNodes / 32];    // nodes with an infinite or NaN value
    __shared__ int odd_any;
    __shared__ int abort_flag;
    __shared__ float2 ml[4][kRows];
    __shared__ int planes[2][32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t sb = smem_u32(smem), full = sb + LY::BARS, empty = full + 8 * kStages;
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        abort_flag = 0;
        odd_any = 0;
    }
    if (tid < kMaxNodes / 32) odd[tid] = 0;
    pdl_wait();
    pdl_trigger();      // the joining launch reads the lengths at once: after this kernel's own wait
    int qg, v, v1;
    tree_runs<kRows, kKeys, kExtra, kLeast<HD>>(a, cum, qg, v, v1);
    const int v0 = v;
    TreePair p, after;
    if (!tree_pair<kExtra>(a, cum, v, v1, p)) return;

    if (warp == 4) {
        // ---------------- stream the tiles: a box is up to 64 tokens of a page x 64 head dims
        const int rows = min(a.pg.ps, kKeys), boxes = kKeys / rows;
        int i = 0;
        const bool ok = each_group<kExtra>(a, cum, v, v1, p, kKeys, rows, lane, planes, [&](int first, int n, const int* plane) {
            for (int tile = first; tile < first + n; ++tile, plane += boxes) {
                // the first pair's queries go first: behind the ring's tiles they would arrive after all of them
                if (i == 0) asm volatile("bar.sync 2, 160;" ::: "memory");
                const int st = i % kStages;
                if (i >= kStages && !__all_sync(0xffffffffu, bar_wait(empty + 8 * st, (uint32_t)(i / kStages - 1) & 1u, &abort_flag, a.pg.err)))
                    return false;
                if (elect_one()) {
                    const uint32_t bar = full + 8 * st, kd = sb + st * 2 * TB;
                    mbar_expect_tx(bar, 2 * TB);
                    for (int x = 0; x < boxes; ++x) {
                        const int z = plane[x], y = (tile * kKeys + x * rows) & (a.pg.ps - 1);
#pragma unroll
                        for (int h = 0; h < HD / 64; ++h) {
                            tma_load_3d(kd + h * 8192 + x * rows * 128, &mk, h * 64, y, z, bar);
                            tma_load_3d(kd + TB + h * 8192 + x * rows * 128, &mv, h * 64, y, z, bar);
                        }
                    }
                }
                ++i;
            }
            return true;
        });
        if (!ok && elect_one()) {   // the copies in flight land before the CTA's shared memory is given up
            volatile int never = 0;
            for (int j = max(0, i - kStages); j < i; ++j)
                bar_wait(full + 8 * (j % kStages), (uint32_t)(j / kStages) & 1u, &never, a.pg.err);
        }
        return;
    }

    const int r0 = lane >> 2;                    // this thread's rows r0 and r0 + 8
    const int cp = (lane & 3) * 2;
    // Q of a pair into half `buf` of its memory, asynchronously: rows past R are never looked at
    auto load_q = [&](const TreePair& p, int R, int buf) {
        constexpr int PC = HD / 8;
#pragma unroll
        for (int x = tid; x < kRows * PC; x += 128) {
            const int r = x / PC, pc = x % PC, nd = group_of(a, r);
            if (r < R)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(sb + LY::Q + buf * (kRows * HD * 2) + (pc >> 3) * (kRows * 128) + r * 128 + (((pc & 7) ^ (r & 7)) << 4)),
                             "l"(static_cast<const bf16*>(a.q) + ((size_t)p.b * a.n_max + nd) * a.q_row + (size_t)(p.h * a.G + r - nd * a.G) * HD + pc * 8)
                             : "memory");
        }
    };
    TreeRaw raw = tree_raw(a, p.b);
    int n, ctx, keys;
    tree_lengths(a, raw, n, ctx, keys);
    load_q(p, n * a.G, 0);
    asm volatile("bar.arrive 2, 160;" ::: "memory");
    // After a wait that gave up the warps go on without waiting: the results are invalid and the error is
    // set, and every barrier among the four still meets.
    bool ok = true, more = true;
    int i = 0;
    for (int pair = 0; more; ++pair) {
        const int R = n * a.G;
        int node[2];
        SeenRow row[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            node[half] = group_of(a, min(r0 + 8 * half, R - 1));
            row[half] = seen_row(a, p.b, node[half]);
        }
        more = tree_pair<kExtra>(a, cum, v, v1, after);
        if (more) raw = tree_raw(a, after.b);
        asm volatile("cp.async.wait_all;" ::: "memory");
        compute_barrier();
        uint32_t qa[HD / 16][4];
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
            const int r = lane & 15, pc = kk * 2 + (lane >> 4);
            ldsm4(sb + LY::Q + (pair & 1) * (kRows * HD * 2) + (pc >> 3) * (kRows * 128) + r * 128 + (((pc & 7) ^ (r & 7)) << 4), qa[kk][0], qa[kk][1],
                  qa[kk][2], qa[kk][3]);
        }
        float o[HD / 8][4];
#pragma unroll
        for (int x = 0; x < HD / 8; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        int n2 = 0, ctx2 = 0, keys2 = 0;

        for (int t = p.lo; t < p.hi; ++t, ++i) {
            const int st = i % kStages;
            if (ok) ok = __all_sync(0xffffffffu, bar_wait(full + 8 * st, (uint32_t)(i / kStages) & 1u, &abort_flag, a.pg.err));
            if (more && t == p.lo) {    // the next pair's queries, a pair ahead
                tree_lengths(a, raw, n2, ctx2, keys2);
                load_q(after, n2 * a.G, (pair + 1) & 1);
            }
            const uint32_t sK = sb + st * 2 * TB, sV = sK + TB;
            const int k0 = t * kKeys, kw = k0 + warp * 16;      // this warp's keys: kw .. kw + 15
            const bool edge = k0 + kKeys > ctx;          // nodes of the tree, or slots past the last key
            if (kw < keys) {
                if (kw + 16 > ctx) {
                    // this warp's values: slots past the last key and infinite or NaN values of nodes become 0
#pragma unroll 1
                    for (int x = lane; x < 16 * (HD / 8); x += 32) {
                        const int r = warp * 16 + x / (HD / 8), key = k0 + r;
                        if (key < ctx) continue;
                        uint4* at = reinterpret_cast<uint4*>(smem + st * 2 * TB + TB + tile_at(r, x % (HD / 8)));
                        uint4 v = make_uint4(0u, 0u, 0u, 0u);
                        bool bad = key >= keys;
                        if (!bad) {
                            v = *at;
                            bad = drop_odd(v);
                            if (bad) {
                                atomicOr(&odd[(key - ctx) >> 5], 1u << ((key - ctx) & 31));
                                odd_any = 1;
                            }
                        }
                        if (bad) *at = v;
                    }
                    // (these stores before the stage's next copy)
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                float s[2][4];
#pragma unroll
                for (int x = 0; x < 2; ++x) s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.f;
#pragma unroll
                for (int kk = 0; kk < HD / 16; kk += 2) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        uint32_t b0, b1, b2, b3;
                        ldsm4(sK + tile_at(warp * 16 + x * 8 + (lane & 7), kk * 2 + (lane >> 3)), b0, b1, b2, b3);
                        mma_bf16(s[x], qa[kk], b0, b1);
                        mma_bf16(s[x], qa[kk + 1], b2, b3);
                    }
                }
                if (edge) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t seen = seen32(a, row[half], p.b, node[half], ctx, keys, kw);
#pragma unroll
                        for (int x = 0; x < 2; ++x)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (!((seen >> (x * 8 + cp + e)) & 1u)) s[x][2 * half + e] = -INFINITY;
                    }
                }
                float alpha[2];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float mx = fmaxf(fmaxf(s[0][2 * half], s[0][2 * half + 1]), fmaxf(s[1][2 * half], s[1][2 * half + 1])) * a.scale_log2;
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    const float top = fmaxf(m[half], mx), ref = top == -INFINITY ? 0.f : top;
                    alpha[half] = pow2(m[half] - ref);
                    m[half] = top;
                    float sum = 0.f;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float w = pow2(fmaf(s[x][2 * half + e], a.scale_log2, -ref));
                            s[x][2 * half + e] = w;
                            sum += w;
                        }
                    }
                    l[half] = l[half] * alpha[half] + sum;
                }
                // Weights rounded to bf16 for the product (relative error 2^-8 at most): what the MMA multiplies by bf16
                // values; a second operand with what the rounding lost would double the products. The sum is of unrounded ones.
                const uint32_t pa[4] = {two_bf16(s[0][0], s[0][1]), two_bf16(s[0][2], s[0][3]), two_bf16(s[1][0], s[1][1]), two_bf16(s[1][2], s[1][3])};
                if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                    for (int x = 0; x < HD / 8; ++x) {
                        o[x][0] *= alpha[0];
                        o[x][1] *= alpha[0];
                        o[x][2] *= alpha[1];
                        o[x][3] *= alpha[1];
                    }
                }
#pragma unroll
                for (int x = 0; x < HD / 16; ++x) {
                    uint32_t b0, b1, b2, b3;
                    ldsm4t(sV + tile_at(warp * 16 + (lane & 15), x * 2 + (lane >> 4)), b0, b1, b2, b3);
                    mma_bf16(o[2 * x], pa, b0, b1);
                    mma_bf16(o[2 * x + 1], pa, b2, b3);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + 8 * st);
        }
        // the four lanes of a row hold parts of its sum
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
            if ((lane & 3) == 0) ml[warp][r0 + 8 * half] = make_float2(m[half], l[half]);
        }
        compute_barrier();
        // every warp's output against the common maximum; quarter q of the head dims goes to warp q
        float M[2], L[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float2 x[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) x[w] = ml[w][r0 + 8 * half];
            M[half] = fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x));
            const float ref = M[half] == -INFINITY ? 0.f : M[half];
            L[half] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) L[half] += x[w].y * pow2(x[w].x - ref);
            const float f = pow2(m[half] - ref);
#pragma unroll
            for (int y = 0; y < HD / 8; ++y) {
                o[y][2 * half] *= f;
                o[y][2 * half + 1] *= f;
            }
        }
        const bool odds = odd_any != 0;
        constexpr int QB = HD / 32;      // blocks of eight head dims in a quarter
        float4* swap = reinterpret_cast<float4*>(smem + LY::SWAP);
        float mine[QB][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#pragma unroll
            for (int y = 0; y < QB; ++y) {
                if (q == warp) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) mine[y][e] = o[q * QB + y][e];
                } else {
                    swap[((q * 3 + ((warp - q) & 3) - 1) * QB + y) * 32 + lane] = make_float4(o[q * QB + y][0], o[q * QB + y][1], o[q * QB + y][2], o[q * QB + y][3]);
                }
            }
        }
        compute_barrier();
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
            for (int y = 0; y < QB; ++y) {
                const float4 x = swap[((warp * 3 + w) * QB + y) * 32 + lane];
                mine[y][0] += x.x;
                mine[y][1] += x.y;
                mine[y][2] += x.z;
                mine[y][3] += x.w;
            }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = r0 + 8 * half, col = warp * (HD / 4) + cp;
            if (r >= R) continue;
            if (odds)
                each_odd(a, odd, p, node[half], ctx, keys, [&](size_t at) {
                    for (int y = 0; y < QB; ++y)
                        for (int e = 0; e < 2; ++e) {
                            const float f = to_f(static_cast<const bf16*>(a.pg.v)[at + col + y * 8 + e]);
                            if (!isfinite(f)) mine[y][2 * half + e] += f;
                        }
                });
            if (p.partial()) {
                const size_t row = ((size_t)blockIdx.x * 2 + (p.start < v0 ? 0 : 1)) * kRows + r;
#pragma unroll
                for (int y = 0; y < QB; ++y)
                    *reinterpret_cast<float2*>(a.part_o + row * HD + col + y * 8) = make_float2(mine[y][2 * half], mine[y][2 * half + 1]);
                if (warp == 0 && (lane & 3) == 0) a.part_ml[row] = make_float2(M[half], L[half]);
            } else {
                const size_t row = ((size_t)p.b * a.n_max + node[half]) * a.hq + p.h * a.G + r - node[half] * a.G;
                const float inv = L[half] == 0.f ? 0.f : 1.f / L[half];
#pragma unroll
                for (int y = 0; y < QB; ++y)
                    *reinterpret_cast<uint32_t*>(static_cast<bf16*>(a.out) + row * HD + col + y * 8) =
                        two_bf16(mine[y][2 * half] * inv, mine[y][2 * half + 1] * inv);
                if (a.lse && warp == 0 && (lane & 3) == 0)
                    a.lse[row] = L[half] == 0.f ? -INFINITY : (M[half] + log2f(L[half])) * 0.69314718055994531f;
            }
        }
        if (odds) {     // the next pair starts with none, once every warp has looked
            compute_barrier();
            if (tid < kMaxNodes / 32) odd[tid] = 0;
            if (tid == 0) odd_any = 0;
            compute_barrier();
        }
        p = after;
        n = n2;
        ctx = ctx2;
        keys = keys2;
    }
}

// fp32: 16 query rows per CTA, 32-key tiles by cp.async in two stages, exact fp32 products on the CUDA cores.
// Scores: a thread takes two rows x two keys; output: (16 / RG) rows x four head dims. Bound by the latency of its
// steps at the sizes that fp32 models have (8 nodes over 600 keys 9 us; 16 over 2 x 1000 keys, 32 heads of 128: 45).
constexpr int kFKeys = 32;
constexpr int kFRows = 16;
constexpr int kFThreads = 128;
// CTAs on an SM, as their shared memory allows. Measured at head_dim 64 with 2 and 5: 60 nodes of 16/8 heads over 1000 and 2000
// keys 79 and 53 us, 150 nodes over 40 contexts up to 100 keys 478 and 300, 8 nodes over 600 keys 8.3 and 8.5.
constexpr int f32_ctas(int HD) { return HD == 64 ? 5 : 2; }
constexpr int kFExtra = 0, kFLeast = 1;     // (a tile takes as long as beginning and ending a pair: 13.0 us with 2 and 3, three contexts up to 600)

template <int HD>
struct F32Layout {
    static constexpr int LD = HD + 4;       // rows of Q and K: float4 reads of neighbouring rows hit all banks
    static constexpr int Q = 0, K = kFRows * LD, V = K + 2 * kFKeys * LD, P = V + 2 * kFKeys * HD, A = P + kFRows * (kFKeys + 4);
    static constexpr int FLOATS = A + 2 * kFRows;
};

template <int HD>
__global__ void __launch_bounds__(kFThreads) tree_f32_kernel(const TreeArgs a) {
    using LY = F32Layout<HD>;
    constexpr int LD = LY::LD, PL = kFKeys + 4, DG = HD / 4, RG = kFThreads / DG, RR = kFRows / RG;
    extern __shared__ __align__(16) float fs[];
    __shared__ int32_t cum[kMaxSeqs + 1];
    float *Qs = fs + LY::Q, *Ks = fs + LY::K, *Vs = fs + LY::V, *Ps = fs + LY::P, *As = fs + LY::A;
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_trigger();
    int qg, v, v1;
    tree_runs<kFRows, kFKeys, kFExtra, kFLeast>(a, cum, qg, v, v1);
    const int v0 = v;
    const int ry = tid / 16, kx = tid % 16;         // scores: rows 2 ry, 2 ry + 1, keys kx, kx + 16
    const int rg = tid / DG, dg = tid % DG;         // output: rows rg RR .., head dims 4 dg ..
    TreePair it;
    while (tree_pair<kFExtra>(a, cum, v, v1, it)) {
        int n, ctx, keys;
        tree_lengths(a, tree_raw(a, it.b), n, ctx, keys);
        const int R = n * a.G, base = qg * kFRows;
        const int32_t* table = a.pg.table + (size_t)it.b * a.pg.max_pages;
        auto load = [&](int tile, int st) {
            const int k0 = tile * kFKeys;
            for (int x = tid; x < kFKeys * DG; x += kFThreads) {
                const int r = x / DG, d = x % DG * 4, key = k0 + r;
                const int page = key < keys ? table[key / a.pg.ps] : -1;
                const bool there = page >= 0 && page < a.pg.pages;
                if (key < keys && !there) atomicOr(a.pg.err, DFLARE_DEVERR_PAGE);
                const size_t at = there ? ((((size_t)a.layer * a.pg.pages + page) * a.pg.hkv + it.h) * a.pg.ps + key % a.pg.ps) * HD + d : 0;
                const int bytes = there ? 16 : 0;       // 0: the 16 bytes become zero
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(Ks + (st * kFKeys + r) * LD + d)),
                             "l"(static_cast<const float*>(a.pg.k) + at), "r"(bytes) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(Vs + (st * kFKeys + r) * HD + d)),
                             "l"(static_cast<const float*>(a.pg.v) + at), "r"(bytes) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        load(it.lo, 0);
        for (int x = tid; x < kFRows * DG; x += kFThreads) {
            const int r = x / DG, d = x % DG * 4, rr = base + r;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (rr < R)
                v = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + ((size_t)it.b * a.n_max + rr / a.G) * a.q_row +
                                                     (size_t)(it.h * a.G + rr % a.G) * HD + d);
            *reinterpret_cast<float4*>(Qs + r * LD + d) = v;
        }
        int node[2];
        for (int i = 0; i < 2; ++i) node[i] = min(base + 2 * ry + i, R - 1) / a.G;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[RR][4];
#pragma unroll
        for (int r = 0; r < RR; ++r) o[r][0] = o[r][1] = o[r][2] = o[r][3] = 0.f;
        for (int t = it.lo; t < it.hi; ++t) {
            const int st = (t - it.lo) & 1, k0 = t * kFKeys;
            if (t + 1 < it.hi) {
                load(t + 1, st ^ 1);
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            } else {
                asm volatile("cp.async.wait_group 0;" ::: "memory");
            }
            __syncthreads();
            float s[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
            const float* K = Ks + (st * kFKeys + kx) * LD;
#pragma unroll 8
            for (int d = 0; d < HD; d += 4) {
                const float4 q0 = *reinterpret_cast<const float4*>(Qs + (2 * ry) * LD + d), q1 = *reinterpret_cast<const float4*>(Qs + (2 * ry + 1) * LD + d);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float4 k = *reinterpret_cast<const float4*>(K + j * 16 * LD + d);
                    s[0][j] = fmaf(q0.x, k.x, fmaf(q0.y, k.y, fmaf(q0.z, k.z, fmaf(q0.w, k.w, s[0][j]))));
                    s[1][j] = fmaf(q1.x, k.x, fmaf(q1.y, k.y, fmaf(q1.z, k.z, fmaf(q1.w, k.w, s[1][j]))));
                }
            }
            const bool edge = k0 + kFKeys > ctx;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint64_t seen = edge ? tree_seen(a, it.b, node[i], ctx, keys, k0) : ~0ull;
                const bool see[2] = {((seen >> kx) & 1) != 0, ((seen >> (kx + 16)) & 1) != 0};
                const float x0 = see[0] ? s[i][0] * a.scale_log2 : -INFINITY, x1 = see[1] ? s[i][1] * a.scale_log2 : -INFINITY;
                float mx = fmaxf(x0, x1);
#pragma unroll
                for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                const float top = fmaxf(m[i], mx), ref = top == -INFINITY ? 0.f : top;
                const float alpha = exp2f(m[i] - ref);
                // unseen: minus zero, which the output's sum tells from a weight that is too small
                const float p0 = see[0] ? exp2f(x0 - ref) : -0.f, p1 = see[1] ? exp2f(x1 - ref) : -0.f;
                float sum = p0 + p1;
#pragma unroll
                for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
                l[i] = l[i] * alpha + sum;
                m[i] = top;
                Ps[(2 * ry + i) * PL + kx] = p0;
                Ps[(2 * ry + i) * PL + kx + 16] = p1;
                if (kx == 0) As[2 * ry + i] = alpha;
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < RR; ++r) {
                const float alpha = As[rg * RR + r];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][e] *= alpha;
            }
            const float* V = Vs + st * kFKeys * HD + 4 * dg;
            if (!edge) {
#pragma unroll 4
                for (int k = 0; k < kFKeys; k += 4) {
                    float4 v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float4*>(V + (k + j) * HD);
#pragma unroll
                    for (int r = 0; r < RR; ++r) {
                        const float4 p = *reinterpret_cast<const float4*>(Ps + (rg * RR + r) * PL + k);
                        const float w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            o[r][0] = fmaf(w[j], v[j].x, o[r][0]);
                            o[r][1] = fmaf(w[j], v[j].y, o[r][1]);
                            o[r][2] = fmaf(w[j], v[j].z, o[r][2]);
                            o[r][3] = fmaf(w[j], v[j].w, o[r][3]);
                        }
                    }
                }
            } else {
                for (int k = 0; k < kFKeys; ++k) {
                    const float4 v = *reinterpret_cast<const float4*>(V + k * HD);
#pragma unroll
                    for (int r = 0; r < RR; ++r) {
                        const float w = Ps[(rg * RR + r) * PL + k];
                        if (__float_as_int(w) < 0) continue;
                        o[r][0] = fmaf(w, v.x, o[r][0]);
                        o[r][1] = fmaf(w, v.y, o[r][1]);
                        o[r][2] = fmaf(w, v.z, o[r][2]);
                        o[r][3] = fmaf(w, v.w, o[r][3]);
                    }
                }
            }
            __syncthreads();
        }
        // (m, l) of a row to the threads that hold its output
        if (kx == 0)
            for (int i = 0; i < 2; ++i) {
                As[2 * ry + i] = m[i];
                As[kFRows + 2 * ry + i] = l[i];
            }
        __syncthreads();
        const bool partial = it.partial();
#pragma unroll
        for (int r = 0; r < RR; ++r) {
            const int lr = rg * RR + r, rr = base + lr;
            if (rr >= R) continue;
            const float mr = As[lr], sr = As[kFRows + lr];
            if (partial) {
                const size_t row = ((size_t)blockIdx.x * 2 + (it.start < v0 ? 0 : 1)) * kFRows + lr;
                *reinterpret_cast<float4*>(a.part_o + row * HD + 4 * dg) = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
                if (dg == 0) a.part_ml[row] = make_float2(mr, sr);
            } else {
                const size_t row = ((size_t)it.b * a.n_max + rr / a.G) * a.hq + it.h * a.G + rr % a.G;
                const float inv = sr == 0.f ? 0.f : 1.f / sr;
                *reinterpret_cast<float4*>(static_cast<float*>(a.out) + row * HD + 4 * dg) =
                    make_float4(o[r][0] * inv, o[r][1] * inv, o[r][2] * inv, o[r][3] * inv);
                if (a.lse && dg == 0) a.lse[row] = sr == 0.f ? -INFINITY : (mr + log2f(sr)) * 0.69314718055994531f;
            }
        }
        __syncthreads();
    }
}

// Rows whose keys several CTAs read: their partial results in the order of the keys. Also the rows that no
// CTA had anything for: no keys, or past the tree's nodes. Where rows are few, four warps share a row's parts (PW), of
// which one long context on one kv head leaves 304; where they are many, a warp takes four rows (RW). Measured, the
// whole attention: one token over 100000 keys on one kv head 37 us with a warp per row and 21 with four; 64 nodes over
// 4096 keys (2048 rows) 18.5 with one and 21.7 with one for four rows; 33 nodes at head_dim 64 (4224 rows) 33 and 29.
// The grid is resident at once and walks the rows: a block finds the division of the work once (2.5 us, while the last
// CTAs of the attention still run). With a block for every four rows, and the division for each, 57 nodes over 20
// contexts of 443 to 1112 keys took 23.5 us for 18.5.
constexpr int kJoinThreads = 128;
constexpr int kJoinFew = 1024, kJoinMany = 4096;    // rows below which a row takes four warps, from which on a warp takes four rows

constexpr int join_blocks(int HD, int RW) { return HD == 64 ? 6 : RW == 1 ? 5 : 4; }     // on an SM, as their registers allow

template <class T, int HD, int RW, int PW>
__global__ void __launch_bounds__(kJoinThreads, join_blocks(HD, RW))
    tree_join_kernel(const TreeArgs a, int QT, int KT, int extra, int least, bool blocks) {
    static_assert(RW == 1 || PW == 1, "several rows per warp or several warps per row");
    constexpr int LPR = 32 / RW, E = HD / LPR, V = E < 4 ? E : 4, J = RW == 1 && PW == 1 ? 8 : 4;
    __shared__ float others[PW][HD + 2];    // of a row's warps: output, maximum, sum
    __shared__ int tiles_of[kMaxSeqs], nodes_of[kMaxSeqs], groups_of[kMaxSeqs];
    __shared__ int first_of[kShares], many_of[kShares];     // of the query groups
    // The kernel before this one let it start after its own dependency wait, so the lengths are final here and
    // the division of the work is found while that kernel still runs.
    // Lane l of a row has the elements (g LPR + l) V .. of its groups g; warp pw of a row the parts pw, pw + PW, ...
    const int lane = threadIdx.x & 31, l = lane % LPR, warp = threadIdx.x >> 5, pw = warp % PW;
    for (int x = threadIdx.x; x < a.batch; x += kJoinThreads) {
        const TreeRaw raw = tree_raw(a, x);
        int n, ctx, keys, groups;
        tree_lengths(a, raw, n, ctx, keys);
        tiles_of[x] = tree_tiles(a, raw, QT, KT, groups);
        nodes_of[x] = n;
        groups_of[x] = groups;
    }
    __syncthreads();
    const bool shares = a.QG > 1 && a.QG <= kShares;
    if (shares && warp == 0) {
        const TreeCosts costs = tree_costs(a, lane, [&](int b, int& cost, int& groups) {
            cost = tree_cost(tiles_of[b], extra);
            groups = groups_of[b];
        });
        int first, many;
        tree_shares(a, costs, lane, first, many);
        if (lane < kShares) {
            first_of[lane] = first;
            many_of[lane] = many;
        }
    }
    if (shares) __syncthreads();
    const unsigned rows = (unsigned)a.batch * a.n_max * a.hq, step = gridDim.x * (kJoinThreads / 32 / PW) * RW;
    unsigned row = (blockIdx.x * (kJoinThreads / 32 / PW) + warp / PW) * RW + lane / LPR;
    for (bool begun = false; !begun || row - lane / LPR < rows; row += step) {
        const bool there = row < rows;
        const int head = row % a.hq, node = row / a.hq % a.n_max, b = there ? row / a.hq / a.n_max : 0;
        const int r = node * a.G + head % a.G, qg = r / QT, tiles = tiles_of[b];
        const bool some = there && node < nodes_of[b] && tiles;
        int before = 0, total = 0, first, C;        // the group's list, its CTAs
        for (int x = l; x < a.batch; x += LPR) {
            const int cost = groups_of[x] > qg ? tree_cost(tiles_of[x], extra) : 0;
            total += cost;
            if (x < b) before += cost;
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) {
            total += __shfl_xor_sync(0xffffffffu, total, o);
            before += __shfl_xor_sync(0xffffffffu, before, o);
        }
        if (shares) {
            C = many_of[qg];
            first = first_of[qg];
        } else {
            C = max(a.C / a.QG, 1);
            first = qg * C;
        }
        const int per = tree_run(total * a.pg.hkv, max(C, 1), least);
        const int start = before * a.pg.hkv + head / a.G * tree_cost(tiles, extra);
        const int c0 = start / per;
        int parts = some ? (start + tiles - 1) / per - c0 + 1 : 0;
        const bool written = parts == 1;        // by the CTA that read all of the row's keys
        parts = written ? 0 : (parts - pw + PW - 1) / PW;       // this warp's
        // every warp waits, so this launch does not end before the one it depends on
        if (!begun) pdl_wait();
        begun = true;
        const int most = __reduce_max_sync(0xffffffffu, parts);
        auto at = [&](int i) {
            const int c = c0 + pw + i * PW;
            return ((size_t)(first + c) * 2 + (start < c * per ? 0 : 1)) * QT + r % QT;
        };
        float acc[E], x[J][E], m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
        auto load = [&](int i) {        // parts i .. i + J - 1
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const size_t row = at(min(i + j, max(parts - 1, 0)));
#pragma unroll
                for (int g = 0; g < E / V; ++g) {
                    const int e = (g * LPR + l) * V;
                    // the tcgen05 kernel's rows lie in blocks of 32 rows x 32 elements, 16-byte pieces swizzled
                    const float* src = a.part_o + (!blocks ? row * HD + e
                                                           : (row & ~(size_t)31) * HD + (e >> 5) * 1024 + (row & 31) * 32 +
                                                                 ((((e & 31) >> 2) ^ (int)(row & 7)) << 2) + (e & 3));
                    if constexpr (V == 4) {
                        const float4 v = i + j < parts ? *reinterpret_cast<const float4*>(src) : make_float4(0.f, 0.f, 0.f, 0.f);
                        x[j][4 * g] = v.x; x[j][4 * g + 1] = v.y; x[j][4 * g + 2] = v.z; x[j][4 * g + 3] = v.w;
                    } else {
                        const float2 v = i + j < parts ? *reinterpret_cast<const float2*>(src) : make_float2(0.f, 0.f);
                        x[j][0] = v.x; x[j][1] = v.y;
                    }
                }
            }
        };
        // the first J parts come in together with the (m, l) that weigh them
        load(0);
        float2 v = l < parts ? a.part_ml[at(l)] : make_float2(-INFINITY, 0.f);
        m = v.x;
        for (int i = LPR + l; i < parts; i += LPR) m = fmaxf(m, a.part_ml[at(i)].x);
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float ref = m == -INFINITY ? 0.f : m;
        float w = exp2f(v.x - ref);             // 0 past the last part
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
#pragma unroll
            for (int e = 0; e < E; ++e) others[pw][l * E + e] = acc[e];
            if (l == 0) {
                others[pw][HD] = m;
                others[pw][HD + 1] = sum;
            }
            __syncthreads();
            if (pw == 0) {
                float top = m;
#pragma unroll
                for (int q = 1; q < PW; ++q) top = fmaxf(top, others[q][HD]);
                const float ref = top == -INFINITY ? 0.f : top;
                float f = exp2f(m - ref);
                sum *= f;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] *= f;
#pragma unroll
                for (int q = 1; q < PW; ++q) {
                    f = exp2f(others[q][HD] - ref);
                    sum = fmaf(others[q][HD + 1], f, sum);
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = fmaf(others[q][l * E + e], f, acc[e]);
                }
                m = top;
            }
            __syncthreads();
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

template <class T, int HD>
cudaError_t launch_join(const dflare_cache* c, const TreeArgs& a, int QT, int KT, int extra, int least, bool blocks, cudaStream_t s) {
    const long long rows = (long long)a.batch * a.n_max * a.hq;
    auto go = [&](auto kernel, int RW, int PW) {
        const long long per = kJoinThreads / 32 / PW * RW, most = (long long)c->num_sms * join_blocks(HD, RW);
        return launch_kernel(true, kernel, dim3((unsigned)std::min((rows + per - 1) / per, most)), dim3(kJoinThreads), 0, s, a, QT, KT, extra,
                             least, blocks);
    };
    if (rows < kJoinFew) return go(tree_join_kernel<T, HD, 1, 4>, 1, 4);
    if (rows < kJoinMany) return go(tree_join_kernel<T, HD, 1, 1>, 1, 1);
    return go(tree_join_kernel<T, HD, 4, 1>, 4, 1);
}

template <int HD>
cudaError_t launch_mma(dflare_cache* c, TreeArgs a, cudaStream_t s) {
    static PerDeviceOnce once;
    cudaError_t e = once([] {
        return cudaFuncSetAttribute(tree_mma_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MmaLayout<HD>::BYTES);
    });
    if (e != cudaSuccess) return e;
    a.QG = 1;
    a.C = 2 * c->num_sms;
    e = launch_kernel(true, tree_mma_kernel<HD>, dim3(a.C), dim3(kMmaThreads), MmaLayout<HD>::BYTES, s, c->maps[0], c->maps[1], a);
    return e == cudaSuccess ? launch_join<bf16, HD>(c, a, kRows, kKeys, kExtra, kLeast<HD>, false, s) : e;
}

template <int HD>
cudaError_t launch_f32(dflare_cache* c, TreeArgs a, cudaStream_t s) {
    static PerDeviceOnce once;
    constexpr int bytes = F32Layout<HD>::FLOATS * 4;
    cudaError_t e = once([] { return cudaFuncSetAttribute(tree_f32_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    if (e != cudaSuccess) return e;
    a.QG = (a.n_max * a.G + kFRows - 1) / kFRows;
    a.C = f32_ctas(HD) * c->num_sms;
    e = launch_kernel(true, tree_f32_kernel<HD>, dim3(std::max(a.QG, a.C)), dim3(kFThreads), bytes, s, a);
    return e == cudaSuccess ? launch_join<float, HD>(c, a, kFRows, kFKeys, kFExtra, kFLeast, false, s) : e;
}

template <int HD>
cudaError_t launch_hd(dflare_cache* c, TreeArgs a, cudaStream_t s) {
    if (c->cfg.dtype == DFLARE_F32) return launch_f32<HD>(c, a, s);
    const int R = a.n_max * a.G;
    // Up to kRows rows the warp-level kernel; the tcgen05 kernel, whose tiles have 128 rows, beside it, us: one token over 2048
    // keys 8.8 and 10.9, four nodes over four contexts up to 3853 keys 16.3 and 19.7, 32 tokens over 1000 keys each 30.9 and
    // 38.9, four nodes over 8 x 32768 keys 165 and 167, two nodes of 64/8 heads of 64 over 16 x 700 keys 13.1 and 18.3.
    if (R <= kRows) return launch_mma<HD>(c, a, s);
    int QT;
    const cudaError_t e = launch_tree_attention_tc(c, a, &QT, s);
    return e == cudaSuccess ? launch_join<bf16, HD>(c, a, QT, kTcKeys, kTcExtra, kTcLeast, true, s) : e;
}

}  // namespace

size_t tree_partial_rows(const dflare_cache_config& g, int num_sms) {
    // two partial results per CTA: of 16 rows with several CTAs per SM, or of up to 256 rows with one
    const int R = g.max_nodes * (g.n_q_heads / g.n_kv_heads);
    const int rows = g.dtype == DFLARE_F32 ? f32_ctas(g.head_dim) * kFRows : R <= kRows ? 2 * kRows : R <= 128 ? 128 : 256;
    return (size_t)num_sms * 2 * rows;
}

cudaError_t launch_tree_attention(dflare_cache* c, TreeArgs a, cudaStream_t s) {
    return c->cfg.head_dim == 128 ? launch_hd<128>(c, a, s) : launch_hd<64>(c, a, s);
}

}  // namespace dfl

using namespace dfl;

extern "C" dflare_status dflare_cache_attend(dflare_cache* c, int layer, const void* q_dev, long long q_row,
                                             const int32_t* mask_dev, const int32_t* n_nodes_dev, int batch, int n_max,
                                             float scale, void* out_dev, float* lse_dev, void* stream) {
    auto bad = [](const char* m) {
        noalloc_set_error(std::string("dflare_cache_attend: ") + m);
        return DFLARE_EINVAL;
    };
    if (!c || !q_dev || !n_nodes_dev || !out_dev) return bad("NULL argument");
    const dflare_cache_config& g = c->cfg;
    if (layer < 0 || layer >= g.n_layers) return bad("layer out of range");
    if (batch < 1 || batch > g.max_batch) return bad("batch must be in [1, max_batch]");
    if (n_max < 1 || n_max > g.max_nodes) return bad("n_max must be in [1, max_nodes]");
    if (!(scale > 0.f) || !std::isfinite(scale)) return bad("scale must be positive and finite");
    if (q_row < (long long)g.n_q_heads * g.head_dim || q_row % 8 != 0) return bad("q_row must hold a row and be a multiple of 8");
    if ((reinterpret_cast<uintptr_t>(q_dev) | reinterpret_cast<uintptr_t>(out_dev)) & 15u) return bad("q and out must be 16-byte aligned");
    TreeArgs a{};
    a.pg = c->view;
    a.q = q_dev;
    a.q_row = q_row;
    a.mask = mask_dev;
    a.n_nodes = n_nodes_dev;
    a.out = out_dev;
    a.lse = lse_dev;
    a.part_o = c->part_o;
    a.part_ml = c->part_ml;
    a.layer = layer;
    a.batch = batch;
    a.n_max = n_max;
    a.words = (n_max + 31) / 32;
    a.hq = g.n_q_heads;
    a.G = g.n_q_heads / g.n_kv_heads;
    a.G_inv = a.G > 1 ? 0xffffffffu / (uint32_t)a.G + 1u : 0u;
    a.scale_log2 = scale * 1.4426950408889634f;
    DeviceGuard guard(c->device);
    const cudaError_t e = launch_tree_attention(c, a, static_cast<cudaStream_t>(stream));
    if (e == cudaSuccess) return DFLARE_OK;
    noalloc_set_error(std::string("dflare_cache_attend: ") + cudaGetErrorString(e));
    return DFLARE_ECUDA;
}
