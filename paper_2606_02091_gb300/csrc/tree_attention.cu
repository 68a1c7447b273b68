// Attention of a tree of nodes (or one token, or a chunk of a prompt) over a paged cache, for up to 64
// query rows per kv head in bf16, and for any number in fp32; many rows in bf16 go to tree_attention_tc.cu.
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
// byte offset of 16-byte piece c of row r in a tile of 64 rows stored as [hd / 64][64][128 bytes], swizzled
__device__ __forceinline__ uint32_t tile_at(int r, int c) {
    return (uint32_t)((c >> 3) * 8192 + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}

// the four warps that compute (the fifth streams tiles)
__device__ __forceinline__ void compute_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

constexpr int kKeys = 64;           // keys per tile
constexpr int kStages = 3;
constexpr int kMmaThreads = 160;
constexpr int kMinTiles = 2;

template <int HD>
struct MmaLayout {
    static constexpr uint32_t TB = HD * 128;                    // a tile of K or V
    static constexpr uint32_t SCRATCH = kStages * 2 * TB;       // partial outputs between warps: half of a row's elements
    static constexpr uint32_t BARS = SCRATCH + 64 * HD;
    static constexpr uint32_t BYTES = BARS + 2 * kStages * 8;
};

// bf16, up to 16 WR query rows. Four warps: WR row blocks of 16 x (4 / WR) parts of each 64-key tile; a
// fifth warp's thread streams the tiles' pages by TMA into a ring of stages. Every warp keeps its own running
// maximum and sum; the parts are joined in shared memory when a pair's keys are done.
template <int HD, int WR>
__global__ void __launch_bounds__(kMmaThreads, 2) tree_mma_kernel(const __grid_constant__ CUtensorMap mk,
                                                                  const __grid_constant__ CUtensorMap mv, const TreeArgs a) {
    using LY = MmaLayout<HD>;
    constexpr int QT = 16 * WR, WK = 4 / WR, KW = kKeys / WK;   // rows, key parts, keys per part
    constexpr uint32_t TB = LY::TB;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int32_t cum[kMaxSeqs + 1];
    __shared__ uint32_t odd[kMaxNodes / 32];    // nodes with an infinite or NaN value
    __shared__ int odd_any;
    __shared__ int abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int qg = blockIdx.x % a.QG, c = blockIdx.x / a.QG;
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
    int t0, t1;
    tree_runs<QT, kKeys, kMinTiles>(a, qg, c, cum, t0, t1);
    pdl_trigger();

    if (warp == 4) {
        // ---------------- stream the tiles: box = up to 64 tokens of a page x 64 head dims; slots without
        // a page take a box outside the pool, which reads as zero
        if (elect_one()) {
            const int rows = min(a.pg.ps, kKeys), boxes = kKeys / rows;
            const int nowhere = (int)min(0x7fffffffLL, (long long)a.pg.layers * a.pg.pages * a.pg.hkv);
            bool ok = true;
            int i = 0;
            for (int t = t0; t < t1 && ok;) {
                const TreeItem it = tree_item(cum, a.batch, a.pg.hkv, t);
                const int end = min(t1, it.start + it.tiles);
                const int32_t* table = a.pg.table + (size_t)it.b * a.pg.max_pages;
                const int pages = min(max(a.pg.held[it.b], 0), a.pg.max_pages);
                for (; t < end && ok; ++t, ++i) {
                    const int st = i % kStages;
                    if (i >= kStages && !(ok = bar_wait(empty + 8 * st, (uint32_t)(i / kStages - 1) & 1u, &abort_flag, a.pg.err))) break;
                    const uint32_t bar = full + 8 * st, kd = sb + st * 2 * TB;
                    mbar_expect_tx(bar, 2 * TB);
                    for (int x = 0; x < boxes; ++x) {
                        const long long slot = (long long)(t - it.start) * kKeys + x * rows;
                        const int pi = (int)(slot / a.pg.ps);
                        const int page = pi < pages ? table[pi] : -1;
                        const int z = page >= 0 && page < a.pg.pages ? (a.layer * a.pg.pages + page) * a.pg.hkv + it.h : nowhere;
                        const int y = (int)(slot % a.pg.ps);
                        for (int h = 0; h < HD / 64; ++h) {
                            tma_load_3d(kd + h * 8192 + x * rows * 128, &mk, h * 64, y, z, bar);
                            tma_load_3d(kd + TB + h * 8192 + x * rows * 128, &mv, h * 64, y, z, bar);
                        }
                    }
                }
            }
            if (!ok) {   // the copies in flight land before the CTA's shared memory is given up
                volatile int never = 0;
                for (int j = max(0, i - kStages); j < i; ++j)
                    bar_wait(full + 8 * (j % kStages), (uint32_t)(j / kStages) & 1u, &never, a.pg.err);
            }
        }
        return;
    }

    const int wr = warp % WR, wk = warp / WR;    // row block, key part
    const int r0 = wr * 16 + (lane >> 2);        // this thread's rows r0 and r0 + 8 of the group
    const int cp = (lane & 3) * 2;
    // After a wait that gave up the warps go on without waiting: the results are invalid and the error is
    // set, and every barrier among the four still meets.
    bool ok = true;
    int i = 0;
    for (int t = t0; t < t1;) {
        const TreeItem it = tree_item(cum, a.batch, a.pg.hkv, t);
        const int first = t, end = min(t1, it.start + it.tiles);
        int n, ctx, keys;
        tree_lengths(a, it.b, n, ctx, keys);
        const int R = n * a.G, base = qg * QT;
        // Q fragments straight from global memory: rows past R are zero
        uint32_t qa[HD / 16][4];
        int node[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = base + r0 + 8 * half;
            node[half] = min(r, R - 1) / a.G;
            const bf16* q = static_cast<const bf16*>(a.q) + ((size_t)it.b * a.n_max + node[half]) * a.q_row +
                            (size_t)(it.h * a.G + min(r, R - 1) % a.G) * HD + cp;
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
                qa[kk][half] = r < R ? *reinterpret_cast<const uint32_t*>(q + kk * 16) : 0u;
                qa[kk][2 + half] = r < R ? *reinterpret_cast<const uint32_t*>(q + kk * 16 + 8) : 0u;
            }
        }
        float o[HD / 8][4];
#pragma unroll
        for (int x = 0; x < HD / 8; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

        for (; t < end; ++t, ++i) {
            const int st = i % kStages;
            if (ok) ok = __all_sync(0xffffffffu, bar_wait(full + 8 * st, (uint32_t)(i / kStages) & 1u, &abort_flag, a.pg.err));
            const uint32_t sK = sb + st * 2 * TB, sV = sK + TB;
            const int k0 = (t - it.start) * kKeys;
            const bool edge = k0 + kKeys > ctx;          // nodes of the tree, or slots past the last key
            if (edge) {
                // values: slots past the last key and infinite or NaN values of nodes become 0
                for (int x = tid; x < kKeys * (HD / 8); x += 128) {
                    const int r = x / (HD / 8), key = k0 + r;
                    if (key < ctx) continue;
                    uint4* p = reinterpret_cast<uint4*>(smem + st * 2 * TB + TB + tile_at(r, x % (HD / 8)));
                    uint4 v = key < keys ? *p : make_uint4(0u, 0u, 0u, 0u);
                    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
                    bool bad = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; bad = true; }
                        if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; bad = true; }
                    }
                    if (bad) {
                        atomicOr(&odd[(key - ctx) >> 5], 1u << ((key - ctx) & 31));
                        odd_any = 1;
                    }
                    if (bad || key >= keys) *p = v;
                }
                // (these stores before the stage's next copy)
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                compute_barrier();
            }
            float s[KW / 8][4];
#pragma unroll
            for (int x = 0; x < KW / 8; ++x) s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.f;
#pragma unroll
            for (int kk = 0; kk < HD / 16; kk += 2) {
#pragma unroll
                for (int x = 0; x < KW / 8; ++x) {
                    uint32_t b0, b1, b2, b3;
                    ldsm4(sK + tile_at(wk * KW + x * 8 + (lane & 7), kk * 2 + (lane >> 3)), b0, b1, b2, b3);
                    mma_bf16(s[x], qa[kk], b0, b1);
                    mma_bf16(s[x], qa[kk + 1], b2, b3);
                }
            }
            if (edge) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint64_t seen = tree_seen(a, it.b, node[half], ctx, keys, k0) >> (wk * KW);
#pragma unroll
                    for (int x = 0; x < KW / 8; ++x)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (!((seen >> (x * 8 + cp + e)) & 1)) s[x][2 * half + e] = -INFINITY;
                }
            }
            uint32_t pa[KW / 16][4];
            float alpha[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float mx = -INFINITY;
#pragma unroll
                for (int x = 0; x < KW / 8; ++x) mx = fmaxf(mx, fmaxf(s[x][2 * half] * a.scale_log2, s[x][2 * half + 1] * a.scale_log2));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                const float top = fmaxf(m[half], mx), ref = top == -INFINITY ? 0.f : top;
                alpha[half] = pow2(m[half] - ref);
                m[half] = top;
                float sum = 0.f;
#pragma unroll
                for (int x = 0; x < KW / 8; ++x) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float p = pow2(fmaf(s[x][2 * half + e], a.scale_log2, -ref));
                        s[x][2 * half + e] = p;
                        sum += p;
                    }
                }
                l[half] = l[half] * alpha[half] + sum;
            }
#pragma unroll
            for (int x = 0; x < KW / 16; ++x) {
                pa[x][0] = two_bf16(s[2 * x][0], s[2 * x][1]);
                pa[x][1] = two_bf16(s[2 * x][2], s[2 * x][3]);
                pa[x][2] = two_bf16(s[2 * x + 1][0], s[2 * x + 1][1]);
                pa[x][3] = two_bf16(s[2 * x + 1][2], s[2 * x + 1][3]);
            }
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
            for (int kk = 0; kk < KW / 16; ++kk) {
#pragma unroll
                for (int x = 0; x < HD / 16; ++x) {
                    uint32_t b0, b1, b2, b3;
                    ldsm4t(sV + tile_at(wk * KW + kk * 16 + (lane & 15), x * 2 + (lane >> 4)), b0, b1, b2, b3);
                    mma_bf16(o[2 * x], pa[kk], b0, b1);
                    mma_bf16(o[2 * x + 1], pa[kk], b2, b3);
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
        }
        // join the key parts: parts 1 and 3 into 0 and 2, then 2 into 0
        float* scratch = reinterpret_cast<float*>(smem + LY::SCRATCH);
        if constexpr (WK > 1) {
            __shared__ float2 ml[4][16];
#pragma unroll
            for (int step = 1; step < WK; step *= 2) {
                const bool gives = (wk & (2 * step - 1)) == step, takes = (wk & (2 * step - 1)) == 0;
                float* at = scratch + ((wk / (2 * step)) * WR + wr) * (8 * HD);
                float mine[2] = {1.f, 1.f}, other[2] = {0.f, 0.f};
                if (gives && (lane & 3) == 0) {
                    ml[warp][lane >> 2] = make_float2(m[0], l[0]);
                    ml[warp][(lane >> 2) + 8] = make_float2(m[1], l[1]);
                }
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    if (gives) {
#pragma unroll
                        for (int x = 0; x < HD / 16; ++x) {
                            const float* v = o[part * (HD / 16) + x];
                            *reinterpret_cast<float4*>(at + (x * 32 + lane) * 4) = make_float4(v[0], v[1], v[2], v[3]);
                        }
                    }
                    compute_barrier();
                    if (takes) {
                        if (part == 0) {
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const float2 v = ml[warp + step * WR][(lane >> 2) + 8 * half];
                                const float top = fmaxf(m[half], v.x), ref = top == -INFINITY ? 0.f : top;
                                mine[half] = pow2(m[half] - ref);
                                other[half] = pow2(v.x - ref);
                                m[half] = top;
                                l[half] = l[half] * mine[half] + v.y * other[half];
                            }
                        }
#pragma unroll
                        for (int x = 0; x < HD / 16; ++x) {
                            const float4 v = *reinterpret_cast<const float4*>(at + (x * 32 + lane) * 4);
                            float* w = o[part * (HD / 16) + x];
                            w[0] = w[0] * mine[0] + v.x * other[0];
                            w[1] = w[1] * mine[0] + v.y * other[0];
                            w[2] = w[2] * mine[1] + v.z * other[1];
                            w[3] = w[3] * mine[1] + v.w * other[1];
                        }
                    }
                    compute_barrier();
                }
            }
        }
        if (wk == 0) {
            const bool partial = first != it.start || end != it.start + it.tiles;
            const int slot = it.start < t0 ? 0 : 1;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int r = base + r0 + 8 * half;
                if (r >= R) continue;
                if (odd_any) {
                    // infinite and NaN values of the nodes that this row sees, in this run's part of the keys
                    for (int w = 0; w < a.words; ++w) {
                        uint32_t bits = odd[w];
                        while (bits) {
                            const int j = w * 32 + __ffs(bits) - 1;
                            bits &= bits - 1;
                            if (!(tree_seen(a, it.b, node[half], ctx, keys, ctx + j) & 1)) continue;
                            const int key = ctx + j, page = a.pg.table[(size_t)it.b * a.pg.max_pages + key / a.pg.ps];
                            const bf16* v = static_cast<const bf16*>(a.pg.v) +
                                            ((((size_t)a.layer * a.pg.pages + page) * a.pg.hkv + it.h) * a.pg.ps + key % a.pg.ps) * HD;
                            for (int x = 0; x < HD / 8; ++x)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const float f = to_f(v[x * 8 + cp + e]);
                                    if (!isfinite(f)) o[x][2 * half + e] += f;
                                }
                        }
                    }
                }
                if (partial) {
                    const size_t row = (((size_t)c * a.QG + qg) * 2 + slot) * QT + r0 + 8 * half;
#pragma unroll
                    for (int x = 0; x < HD / 8; ++x)
                        *reinterpret_cast<float2*>(a.part_o + row * HD + x * 8 + cp) = make_float2(o[x][2 * half], o[x][2 * half + 1]);
                    if ((lane & 3) == 0) a.part_ml[row] = make_float2(m[half], l[half]);
                } else {
                    const size_t row = ((size_t)it.b * a.n_max + node[half]) * a.hq + it.h * a.G + r % a.G;
                    const float inv = l[half] > 0.f ? 1.f / l[half] : l[half] == 0.f ? 0.f : l[half];
#pragma unroll
                    for (int x = 0; x < HD / 8; ++x)
                        *reinterpret_cast<uint32_t*>(static_cast<bf16*>(a.out) + row * HD + x * 8 + cp) =
                            two_bf16(o[x][2 * half] * inv, o[x][2 * half + 1] * inv);
                    if (a.lse && (lane & 3) == 0)
                        a.lse[row] = l[half] == 0.f ? -INFINITY : (m[half] + log2f(l[half])) * 0.69314718055994531f;
                }
            }
        }
        // the next pair starts with no odd nodes, once every warp has looked
        compute_barrier();
        if (odd_any) {
            compute_barrier();
            if (tid < kMaxNodes / 32) odd[tid] = 0;
            if (tid == 0) odd_any = 0;
            compute_barrier();
        }
    }
}

// fp32: 16 query rows per CTA, 32-key tiles by cp.async in two stages, exact fp32 products on the CUDA cores.
// Scores: a thread takes two rows x two keys; output: (16 / RG) rows x four head dims.
constexpr int kFKeys = 32;
constexpr int kFRows = 16;
constexpr int kFThreads = 128;
constexpr int kFMinTiles = 2;

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
    const int tid = threadIdx.x, qg = blockIdx.x % a.QG, c = blockIdx.x / a.QG;
    pdl_wait();
    int t0, t1;
    tree_runs<kFRows, kFKeys, kFMinTiles>(a, qg, c, cum, t0, t1);
    pdl_trigger();
    const int ry = tid / 16, kx = tid % 16;         // scores: rows 2 ry, 2 ry + 1, keys kx, kx + 16
    const int rg = tid / DG, dg = tid % DG;         // output: rows rg RR .., head dims 4 dg ..
    for (int t = t0; t < t1;) {
        const TreeItem it = tree_item(cum, a.batch, a.pg.hkv, t);
        const int first = t, end = min(t1, it.start + it.tiles);
        int n, ctx, keys;
        tree_lengths(a, it.b, n, ctx, keys);
        const int R = n * a.G, base = qg * kFRows;
        const int32_t* table = a.pg.table + (size_t)it.b * a.pg.max_pages;
        auto load = [&](int tile, int st) {
            const int k0 = (tile - it.start) * kFKeys;
            for (int x = tid; x < kFKeys * DG; x += kFThreads) {
                const int r = x / DG, d = x % DG * 4, key = k0 + r;
                const int page = key < keys ? table[key / a.pg.ps] : -1;
                const bool there = page >= 0 && page < a.pg.pages;
                const size_t at = there ? ((((size_t)a.layer * a.pg.pages + page) * a.pg.hkv + it.h) * a.pg.ps + key % a.pg.ps) * HD + d : 0;
                const int bytes = there ? 16 : 0;       // 0: the 16 bytes become zero
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(Ks + (st * kFKeys + r) * LD + d)),
                             "l"(static_cast<const float*>(a.pg.k) + at), "r"(bytes) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(Vs + (st * kFKeys + r) * HD + d)),
                             "l"(static_cast<const float*>(a.pg.v) + at), "r"(bytes) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        load(t, 0);
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
        for (; t < end; ++t) {
            const int st = (t - first) & 1, k0 = (t - it.start) * kFKeys;
            if (t + 1 < end) {
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
        const bool partial = first != it.start || end != it.start + it.tiles;
#pragma unroll
        for (int r = 0; r < RR; ++r) {
            const int lr = rg * RR + r, rr = base + lr;
            if (rr >= R) continue;
            const float mr = As[lr], sr = As[kFRows + lr];
            if (partial) {
                const size_t row = (((size_t)c * a.QG + qg) * 2 + (it.start < t0 ? 0 : 1)) * kFRows + lr;
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
// CTA had anything for: no keys, or past the tree's nodes. A warp per row.
constexpr int kJoinThreads = 256;

template <class T, int HD>
__global__ void __launch_bounds__(kJoinThreads) tree_join_kernel(const TreeArgs a, int QT, int KT) {
    constexpr int E = HD / 32;      // elements per lane
    pdl_wait();
    const long long row = (long long)blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= (long long)a.batch * a.n_max * a.hq) return;
    const int head = (int)(row % a.hq), node = (int)(row / a.hq % a.n_max), b = (int)(row / a.hq / a.n_max);
    int n, ctx, keys;
    tree_lengths(a, b, n, ctx, keys);
    float acc[E], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    if (node < n && keys > 0) {
        const int r = node * a.G + head % a.G, qg = r / QT;
        const TreePlan p = tree_plan_of(a);
        const int32_t* cum = p.cum + (size_t)qg * (a.batch + 1);
        const int per = p.per[qg], tiles = cum[b + 1] - cum[b];
        const int start = cum[b] * a.pg.hkv + head / a.G * tiles;
        const int c0 = start / per, c1 = (start + tiles - 1) / per;
        if (c0 == c1) return;       // written by the CTA that read all of them
        auto at = [&](int c) { return (((size_t)c * a.QG + qg) * 2 + (start < c * per ? 0 : 1)) * QT + r % QT; };
        for (int c = c0 + lane; c <= c1; c += 32) m = fmaxf(m, a.part_ml[at(c)].x);
        m = warp_max(m);
        const float ref = m == -INFINITY ? 0.f : m;
        for (int cb = c0; cb <= c1; cb += 32) {
            float w = 0.f, sum = 0.f;
            if (cb + lane <= c1) {
                const float2 v = a.part_ml[at(cb + lane)];
                w = exp2f(v.x - ref);
                sum = v.y * w;
            }
            l += warp_sum(sum);
            const int upto = min(32, c1 - cb + 1);
#pragma unroll 4
            for (int j = 0; j < upto; ++j) {
                const float wj = __shfl_sync(0xffffffffu, w, j);
                const float* src = a.part_o + at(cb + j) * HD + lane * E;
                float x[E];
                if constexpr (E == 4) {
                    const float4 v = *reinterpret_cast<const float4*>(src);
                    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
                } else {
                    const float2 v = *reinterpret_cast<const float2*>(src);
                    x[0] = v.x; x[1] = v.y;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = fmaf(wj, x[e], acc[e]);
            }
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= inv;
    }
    T* out = static_cast<T*>(a.out) + row * HD + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = from_f<T>(acc[e]);
    if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

template <class T, int HD>
cudaError_t launch_join(const TreeArgs& a, int QT, int KT, cudaStream_t s) {
    const long long rows = (long long)a.batch * a.n_max * a.hq;
    return launch_kernel(true, tree_join_kernel<T, HD>, dim3((unsigned)((rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32))),
                         dim3(kJoinThreads), 0, s, a, QT, KT);
}

template <int HD, int WR>
cudaError_t launch_mma(dflare_cache* c, TreeArgs a, cudaStream_t s) {
    static PerDeviceOnce once;
    cudaError_t e = once([] {
        return cudaFuncSetAttribute(tree_mma_kernel<HD, WR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MmaLayout<HD>::BYTES);
    });
    if (e != cudaSuccess) return e;
    a.QG = (a.n_max * a.G + 16 * WR - 1) / (16 * WR);
    a.C = std::max(1, 2 * c->num_sms / a.QG);
    e = launch_kernel(true, tree_mma_kernel<HD, WR>, dim3(a.QG * a.C), dim3(kMmaThreads), MmaLayout<HD>::BYTES, s, c->maps[0], c->maps[1], a);
    return e == cudaSuccess ? launch_join<bf16, HD>(a, 16 * WR, kKeys, s) : e;
}

template <int HD>
cudaError_t launch_f32(dflare_cache* c, TreeArgs a, cudaStream_t s) {
    static PerDeviceOnce once;
    constexpr int bytes = F32Layout<HD>::FLOATS * 4;
    cudaError_t e = once([] { return cudaFuncSetAttribute(tree_f32_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    if (e != cudaSuccess) return e;
    a.QG = (a.n_max * a.G + kFRows - 1) / kFRows;
    a.C = std::max(1, 2 * c->num_sms / a.QG);
    e = launch_kernel(true, tree_f32_kernel<HD>, dim3(a.QG * a.C), dim3(kFThreads), bytes, s, a);
    return e == cudaSuccess ? launch_join<float, HD>(a, kFRows, kFKeys, s) : e;
}

template <int HD>
cudaError_t launch_hd(dflare_cache* c, const TreeArgs& a, cudaStream_t s) {
    if (c->cfg.dtype == DFLARE_F32) return launch_f32<HD>(c, a, s);
    const int R = a.n_max * a.G;
    if (R <= 16) return launch_mma<HD, 1>(c, a, s);
    if (R <= 32) return launch_mma<HD, 2>(c, a, s);
    return launch_mma<HD, 4>(c, a, s);
}

}  // namespace

size_t tree_partial_rows(const dflare_cache_config& g, int num_sms) {
    // two partial results per CTA: 2 CTAs per SM of 16 (fp32) or up to 64 rows
    return (size_t)num_sms * 2 * 2 * (g.dtype == DFLARE_F32 ? kFRows : 64);
}
size_t tree_plan_size(const dflare_cache_config& g) {
    const int R = g.max_nodes * (g.n_q_heads / g.n_kv_heads);
    return tree_plan_ints((R + 15) / 16, g.max_batch);
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
    a.plan = c->plan;
    a.layer = layer;
    a.batch = batch;
    a.n_max = n_max;
    a.words = (n_max + 31) / 32;
    a.hq = g.n_q_heads;
    a.G = g.n_q_heads / g.n_kv_heads;
    a.scale_log2 = scale * 1.4426950408889634f;
    DeviceGuard guard(c->device);
    const cudaError_t e = launch_tree_attention(c, a, static_cast<cudaStream_t>(stream));
    if (e == cudaSuccess) return DFLARE_OK;
    noalloc_set_error(std::string("dflare_cache_attend: ") + cudaGetErrorString(e));
    return DFLARE_ECUDA;
}
