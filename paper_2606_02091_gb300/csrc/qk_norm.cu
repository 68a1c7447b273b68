// Root-mean-square norm of query and key heads with the rotary positions in the same pass: forward, backward, and on
// a step's new tokens on their way into the pages of a cache.
//
// Of one head x with gain g:  r = 1 / sqrt(mean(x^2) + eps),  z = g x r,  y = R z  (R turns the pairs of the rotated
// elements by position * phase and scales them; the other elements stay).
// Backward, from dy:  dz = R^T dy,  a = g dz,  dx = r (a - x r^2 mean(a x)),  dg = sum over rows and heads of dz x r.
// All of it in fp32, y and dx rounded once.
//
// Work: as in rope.cu a thread has 16 elements of a head, and the head's threads (a power of two of them, neighbours in a
// warp) add up their squares by shuffles. A CTA has heads of queries or of keys (or, in an append, values), so that a thread needs one gain.
#include <math.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "common.cuh"
#include "paged.h"
#include "rope.cuh"

namespace dfl {
namespace {

constexpr int kThreads = 256;
constexpr int kStreamCtas = 2;          // CTAs on an SM, as their registers and rings allow (three spill: 50 us instead of 43 for 10563 rows)
constexpr int kWorkRows = DFLARE_QK_NORM_WORK_ROWS;     // CTAs that may leave a sum of gain gradients

// queries, keys, values (values in an append only: copied)
struct Part {
    const void* x;
    long long x_row, x_head;
    const void* dy;                     // backward
    long long dy_row, dy_head;
    void* out;                          // y or dx; keys and values of an append go to the pages
    long long out_row, out_head;
    const void* gain;
    float* dgain;                       // backward, [hd]
    int heads;
    int blocks;                         // CTAs
};
struct NormArgs {
    Part part[3];
    const int32_t* positions;
    const uint64_t* phase;
    float* work;                        // backward: [CTAs][hd]
    int rows, hd, rot;
    float magnitude, eps;
    PagesView pg;
    AppendRows rows_of;
};

template <class T>
__device__ __forceinline__ const T* head_at(const void* base, long long row, long long row_stride, int h, long long head_stride) {
    return static_cast<const T*>(base) + row * row_stride + h * head_stride;
}
// where head h of a part's row goes; null: nowhere
template <class T, bool APPEND>
__device__ __forceinline__ T* out_at(const NormArgs& a, const Part& p, int part, long long row, int h, long long slot) {
    if (!APPEND || part == 0) return static_cast<T*>(p.out) + row * p.out_row + h * p.out_head;
    return slot < 0 ? nullptr : static_cast<T*>(part == 2 ? a.pg.v : a.pg.k) + (slot + (long long)h * a.pg.ps) * a.hd;
}
// A unit's values as eight packed pairs: of neighbours, so that halves turn (0..3 with 4..7) in packed operations, and
// interleaved pairs turn with their own exchange.
template <class T>
__device__ __forceinline__ void values(const Unit<T>& u, uint64_t* v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = get2(u, i);
        v[i] = pack2(f.x, f.y);
    }
}
template <class T>
__device__ __forceinline__ void put(Unit<T>& u, const uint64_t* v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float a, b;
        unpack2(v[i], a, b);
        set2(u, i, a, b);
    }
}
__device__ __forceinline__ uint64_t swapped(uint64_t v) {
    float a, b;
    unpack2(v, a, b);
    return pack2(b, a);
}
__device__ __forceinline__ uint64_t both(float v) { return pack2(v, v); }
__device__ __forceinline__ float sum2(uint64_t v) {
    float a, b;
    unpack2(v, a, b);
    return a + b;
}
// 1 / sqrt(mean + eps), rounded once more than its argument
__device__ __forceinline__ float inverse_rms(float sum_sq, float inv_hd, float eps) { return __frsqrt_rn(fmaf(sum_sq, inv_hd, eps)); }

// What turns a unit: y_i = r (x_i A_i + x_partner(i) B_i), with the gain in it; or y_i = r x_i A_i where nothing turns.
struct Turn {
    uint64_t a[8], b[8];
};
// c, s of the unit's eight pairs; gain
template <bool INTER>
__device__ __forceinline__ void make_turn(Turn& t, bool rotates, const float* c, const float* s, const uint64_t* gain) {
    if (!rotates) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t.a[i] = gain[i];
            t.b[i] = 0ull;
        }
    } else if (INTER) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t.a[i] = mul2(both(c[i]), gain[i]);
            t.b[i] = mul2(pack2(-s[i], s[i]), swapped(gain[i]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t cc = pack2(c[2 * i], c[2 * i + 1]), ss = pack2(s[2 * i], s[2 * i + 1]);
            t.a[i] = mul2(cc, gain[i]);
            t.a[4 + i] = mul2(cc, gain[4 + i]);
            t.b[i] = mul2(pack2(-s[2 * i], -s[2 * i + 1]), gain[4 + i]);
            t.b[4 + i] = mul2(ss, gain[i]);
        }
    }
}
template <bool INTER>
__device__ __forceinline__ uint64_t partner(const uint64_t* v, int i) { return INTER ? swapped(v[i]) : v[i ^ 4]; }

// Sums of gain gradients: a thread's pairs to their places in its group's row; the groups' rows added up in order
__device__ __forceinline__ void leave(float* row, const uint64_t* acc, int e0, int e1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float lo, hi;
        unpack2(acc[i], lo, hi);
        const int e = i < 4 ? e0 + 2 * i : e1 + 2 * i - 8;
        row[e] = lo;
        row[e + 1] = hi;
    }
}
__device__ __forceinline__ void add_up(const float* sums, int groups, const NormArgs& a) {
    for (int e = threadIdx.x; e < a.hd; e += kThreads) {
        float v = 0.f;
        for (int g = 0; g < groups; ++g) v += sums[g * a.hd + e];
        a.work[(size_t)blockIdx.x * a.hd + e] = v;
    }
}

// ---------------- rot and hd multiples of 16, hd up to 512, everything 16-byte aligned
// The list of all (row, 32 / LANES heads) of a part is shared out evenly among its warps. A warp copies its units ahead into shared
// memory, kStages deep and across rows, so that as much as a load's latency asks for is always under way; a thread reads only what it copied
// itself, so its own wait is enough. A row's cosines are worked out once per warp: a unit's eight pairs are shared out among the threads
// that have the same unit of different heads.
// HBM-bound for many rows: 10563 rows of 40 heads of 128 37.6 us, 5.7 TB/s (52 with whole rows of several heads to a thread and loads
// into registers), 8192 rows forward and backward 80 us, 5.3 TB/s; for few by latency, 64 rows 2.9 and 5.8 us.
template <class T, int NA> constexpr int kStages = sizeof(T) * NA > 4 ? 2 : 4;

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// One thread's ring of units: NA arrays (x, or x and dy), kStages deep; pieces of 16 bytes, a warp's side by side.
template <class T, int NA>
struct Ring {
    static constexpr int P = sizeof(T);             // pieces of a unit
    static constexpr int STAGES = kStages<T, NA>;
    static constexpr uint32_t BYTES = STAGES * NA * P * 512;       // of a warp
    uint32_t base;                                  // this thread's first piece
    __device__ __forceinline__ void copy(int stage, int array, const T* p0, const T* p1) const {
        const uint32_t to = base + (stage * NA + array) * (P * 512);
#pragma unroll
        for (int i = 0; i < P; ++i)
            copy16(to + i * 512, reinterpret_cast<const char*>(i < P / 2 ? p0 : p1) + (i % (P / 2)) * 16);
    }
    __device__ __forceinline__ void read(int stage, int array, Unit<T>& u) const {
        const uint32_t at = base + (stage * NA + array) * (P * 512);
#pragma unroll
        for (int i = 0; i < P; ++i)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(u.v[i].x), "=r"(u.v[i].y), "=r"(u.v[i].z), "=r"(u.v[i].w) : "r"(at + i * 512) : "memory");
    }
};

// Cosines and sines of the eight pairs of a thread's unit at `pos`: the G threads that have the unit work out 8 / G each.
template <int LANES>
struct Pairs {
    static constexpr int G = 32 / LANES, M = G >= 8 ? 1 : 8 / G;
    uint64_t phase[M];
    __device__ __forceinline__ void load(const uint64_t* all, int u, int group, bool rotates) {
#pragma unroll
        for (int m = 0; m < M; ++m) phase[m] = rotates ? all[u * 8 + (m * G + group) % 8] : 0ull;
    }
    __device__ __forceinline__ void at(long long pos, float magnitude, int u, float* c, float* s) const {
        float cm[M], sm[M];
#pragma unroll
        for (int m = 0; m < M; ++m) pair_turn(pos, phase[m], 1.f, magnitude, cm[m], sm[m]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int from = u + LANES * (j % G);
            c[j] = __shfl_sync(0xffffffffu, cm[j / G], from);
            s[j] = __shfl_sync(0xffffffffu, sm[j / G], from);
        }
    }
};
template <int LANES>
__device__ __forceinline__ float sum_of_head(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// f(row, head of this thread, whether it is there, stage, issue) for the warp's part of the list of all (row, 32 / LANES heads); next(row)
// before the first of a row; given(row): whether the row is to be read. NA arrays, whose units begin at elements e0 and e1.
template <class T, int NA, int LANES, class Given, class Next, class F>
__device__ __forceinline__ void each_unit(const NormArgs& a, const Part& p, int wid, int warps, const Ring<T, NA>& ring, int group, bool mine, int e0, int e1,
                                          Given given, Next next, F f) {
    constexpr int G = 32 / LANES, S = kStages<T, NA>;
    const int iters = (p.heads + G - 1) / G;
    const long long all = (long long)a.rows * iters;
    const long long n0 = all * wid / warps;
    int left_i = (int)(all * (wid + 1) / warps - n0), left = left_i;
    int row = (int)(n0 / iters), h = (int)(n0 - (long long)row * iters) * G + group;
    int row_i = row, h_i = h, stage_i = 0, stage = 0;
    bool given_i = left_i > 0 && given(row);
    auto issue = [&]() {
        if (left_i > 0) {
            --left_i;
            if (mine && given_i && h_i < p.heads) {
                const T* x = head_at<T>(p.x, row_i, p.x_row, h_i, p.x_head);
                ring.copy(stage_i, 0, x + e0, x + e1);
                if constexpr (NA == 2) {
                    const T* d = head_at<T>(p.dy, row_i, p.dy_row, h_i, p.dy_head);
                    ring.copy(stage_i, 1, d + e0, d + e1);
                }
            }
            h_i += G;
            if (h_i - group >= p.heads) {
                h_i = group;
                ++row_i;
                given_i = left_i > 0 && given(row_i);
            }
        }
        copies_commit();
        stage_i = stage_i + 1 == S ? 0 : stage_i + 1;
    };
#pragma unroll
    for (int i = 0; i < S - 1; ++i) issue();
    for (; left > 0; ++row, h = group) {
        next(row);
        for (; h - group < p.heads && left > 0; h += G, --left) {
            copies_wait<S - 2>();
            f(row, h, mine && h < p.heads, stage, issue);
            stage = stage + 1 == S ? 0 : stage + 1;
        }
    }
    copies_wait<0>();
}

// CTAs of a part, its number among them, and what a thread has of its heads.
struct StreamPlace {
    int part, wid, warps, u, group, e0, e1;
    bool mine, rotates;
};
template <int LANES, bool INTER>
__device__ __forceinline__ StreamPlace stream_place(const NormArgs& a) {
    StreamPlace y;
    const int lane = threadIdx.x & 31;
    int block = blockIdx.x;
    y.part = 0;
    while (y.part < 2 && block >= a.part[y.part].blocks) block -= a.part[y.part++].blocks;
    y.wid = block * (kThreads / 32) + (threadIdx.x >> 5);
    y.warps = a.part[y.part].blocks * (kThreads / 32);
    y.u = lane % LANES;
    y.group = lane / LANES;
    y.mine = y.u < a.hd / 16;
    y.rotates = y.u < a.rot / 16;
    y.e0 = y.rotates && !INTER ? y.u * 8 : y.u * 16;
    y.e1 = y.rotates && !INTER ? a.rot / 2 + y.u * 8 : y.u * 16 + 8;
    return y;
}

// APPEND: a step's new tokens on their way into the pages; values are copied. Rows past a sequence's new tokens are not read.
template <class T, bool INTER, bool APPEND, int LANES>
__global__ void __launch_bounds__(kThreads, kStreamCtas) qk_norm_stream_kernel(const NormArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_wait();
    pdl_trigger();
    const StreamPlace y = stream_place<LANES, INTER>(a);
    const Part& p = a.part[y.part];
    const Ring<T, 1> ring{(uint32_t)__cvta_generic_to_shared(smem) + (threadIdx.x >> 5) * Ring<T, 1>::BYTES + (threadIdx.x & 31) * 16};
    const bool norms = !APPEND || y.part < 2;
    Unit<T> gain{};
    if (y.mine && norms) load_unit(gain, static_cast<const T*>(p.gain) + y.e0, static_cast<const T*>(p.gain) + y.e1);
    Pairs<LANES> pairs;
    pairs.load(a.phase, y.u, y.group, y.rotates && norms);
    const float inv_hd = 1.f / (float)a.hd;
    long long pos = 0, slot = -1;
    bool begun = false, live = true;
    Turn turn;
    each_unit<T, 1, LANES>(a, p, y.wid, y.warps, ring, y.group, y.mine, y.e0, y.e1,
        [&](int row) { return !APPEND || row % a.rows_of.n_max < a.rows_of.n_new[row / a.rows_of.n_max]; },
        [&](int row) {
            uint64_t g[8];
            float c[8], s[8];
            if constexpr (APPEND) {
                live = append_row(a.pg, a.rows_of, row, pos, slot);
            } else if (a.positions && !begun) {
                pos = a.positions[row];
                begun = true;
            }
            pairs.at(pos, a.magnitude, y.u, c, s);
            if (!APPEND && a.positions && row + 1 < a.rows) pos = a.positions[row + 1];     // (a row ahead)
            values(gain, g);
            make_turn<INTER>(turn, y.rotates, c, s, g);
        },
        [&](int row, int h, bool there, int stage, auto issue) {
            Unit<T> x{};
            if (there) ring.read(stage, 0, x);
            issue();
            uint64_t v[8], sq = 0ull;
            values(x, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sq = fma2(v[i], v[i], sq);
            const uint64_t r = both(inverse_rms(sum_of_head<LANES>(sum2(sq)), inv_hd, a.eps));
            if (norms) {
                uint64_t out[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = mul2(v[i], turn.a[i]);
                if (y.rotates) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) out[i] = fma2(partner<INTER>(v, i), turn.b[i], out[i]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = mul2(out[i], r);
                put(x, out);
            }
            T* to = out_at<T, APPEND>(a, p, y.part, row, h, slot);
            if (there && (!APPEND || (live && to))) store_unit(x, to + y.e0, to + y.e1);
        });
}

// R^T of a unit's pairs: y_i = z_i C_i + z_partner(i) S_i
template <bool INTER>
__device__ __forceinline__ void turn_back(uint64_t* z, const float* c, const float* s) {
    if (INTER) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = fma2(swapped(z[i]), pack2(s[i], -s[i]), mul2(z[i], both(c[i])));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t cc = pack2(c[2 * i], c[2 * i + 1]), ss = pack2(s[2 * i], s[2 * i + 1]), ns = pack2(-s[2 * i], -s[2 * i + 1]);
            const uint64_t z0 = z[i], z1 = z[4 + i];
            z[i] = fma2(z1, ss, mul2(z0, cc));
            z[4 + i] = fma2(z0, ns, mul2(z1, cc));
        }
    }
}

template <class T, bool INTER, int LANES>
__global__ void __launch_bounds__(kThreads, kStreamCtas) qk_norm_backward_stream_kernel(const NormArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_wait();
    pdl_trigger();
    const StreamPlace y = stream_place<LANES, INTER>(a);
    const Part& p = a.part[y.part];
    const Ring<T, 2> ring{(uint32_t)__cvta_generic_to_shared(smem) + (threadIdx.x >> 5) * Ring<T, 2>::BYTES + (threadIdx.x & 31) * 16};
    uint64_t w[8], acc[8];
    {
        Unit<T> g{};
        if (y.mine) load_unit(g, static_cast<const T*>(p.gain) + y.e0, static_cast<const T*>(p.gain) + y.e1);
        values(g, w);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0ull;
    Pairs<LANES> pairs;
    pairs.load(a.phase, y.u, y.group, y.rotates);
    const float inv_hd = 1.f / (float)a.hd;
    int pos = 0;
    bool begun = false;
    float c[8], s[8];
    each_unit<T, 2, LANES>(a, p, y.wid, y.warps, ring, y.group, y.mine, y.e0, y.e1, [](int) { return true; },
        [&](int row) {
            if (a.positions) {
                if (!begun) pos = a.positions[row];
                begun = true;
            }
            pairs.at(pos, a.magnitude, y.u, c, s);
            if (a.positions && row + 1 < a.rows) pos = a.positions[row + 1];     // (a row ahead)
        },
        [&](int row, int h, bool there, int stage, auto issue) {
            Unit<T> x{}, d{};
            if (there) {
                ring.read(stage, 0, x);
                ring.read(stage, 1, d);
            }
            issue();
            uint64_t v[8], z[8], sq = 0ull, ax = 0ull;
            values(x, v);
            values(d, z);
            if (y.rotates) turn_back<INTER>(z, c, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sq = fma2(v[i], v[i], sq);
                ax = fma2(mul2(z[i], w[i]), v[i], ax);
            }
            const float all = sum_of_head<LANES>(sum2(sq)), dot = sum_of_head<LANES>(sum2(ax));
            if (!there) return;
            const float r = inverse_rms(all, inv_hd, a.eps);
            const uint64_t rr = both(r), f = both(-(r * r * (dot * inv_hd)));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint64_t n = mul2(v[i], rr);      // x r
                acc[i] = fma2(z[i], n, acc[i]);
                v[i] = fma2(n, f, mul2(mul2(z[i], w[i]), rr));
            }
            put(x, v);
            T* to = static_cast<T*>(p.out) + row * p.out_row + h * p.out_head;
            store_unit(x, to + y.e0, to + y.e1);
        });
    // the CTA's sums in the order of its warps and their groups, over the rings (whose copies have all landed)
    constexpr int groups = kThreads / LANES;
    float* sums = reinterpret_cast<float*>(smem);
    __syncthreads();
    if (y.mine) leave(sums + (threadIdx.x / LANES) * a.hd, acc, y.e0, y.e1);
    __syncthreads();
    add_up(sums, groups, a);
}

// Any hd up to 1024, rot, strides and alignment: a warp per head, which a lane reads twice.
template <class T, bool INTER, bool APPEND>
__global__ void __launch_bounds__(kThreads) qk_norm_any_kernel(const NormArgs a) {
    pdl_wait();
    pdl_trigger();
    const int total = a.part[0].heads + a.part[1].heads + a.part[2].heads, lane = threadIdx.x & 31;
    const long long g = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const long long row = g / total;
    int h = (int)(g - row * total), part = 0;
    if (row >= a.rows) return;
    while (h >= a.part[part].heads) h -= a.part[part++].heads;
    const Part& p = a.part[part];
    long long pos = 0, slot = -1;
    if (APPEND) {
        if (!append_row(a.pg, a.rows_of, (int)row, pos, slot)) return;
    } else if (a.positions) {
        pos = a.positions[row];
    }
    const T* x = head_at<T>(p.x, row, p.x_row, h, p.x_head);
    T* to = out_at<T, APPEND>(a, p, part, row, h, slot);
    if (APPEND && !to) return;
    float sum = 0.f;
    for (int e = lane; e < a.hd; e += 32) sum = fmaf(to_f(x[e]), to_f(x[e]), sum);
    const float r = inv_rms(warp_sum(sum), a.hd, a.eps);      // (every lane has read before any lane writes)
    const T* gain = static_cast<const T*>(p.gain);
    const int half = a.rot / 2;
    if (APPEND && part == 2) {
        for (int e = lane; e < a.hd; e += 32) to[e] = x[e];
        return;
    }
    for (int j = lane; j < half; j += 32) {
        const int i0 = INTER ? 2 * j : j, i1 = INTER ? 2 * j + 1 : half + j;
        float c, s;
        pair_turn(pos, a.phase[j], 1.f, a.magnitude, c, s);
        const float z0 = to_f(x[i0]) * r * to_f(gain[i0]), z1 = to_f(x[i1]) * r * to_f(gain[i1]);
        to[i0] = from_f<T>(z0 * c - z1 * s);
        to[i1] = from_f<T>(z1 * c + z0 * s);
    }
    for (int e = a.rot + lane; e < a.hd; e += 32) to[e] = from_f<T>(to_f(x[e]) * r * to_f(gain[e]));
}

// Backward for any hd up to 1024, rot, strides and alignment: a warp per head, its gain gradients in shared memory (a
// lane's elements are its own).
template <class T, bool INTER>
__global__ void __launch_bounds__(kThreads) qk_norm_backward_any_kernel(const NormArgs a) {
    extern __shared__ float sums[];                 // [warps][hd]
    pdl_wait();
    pdl_trigger();
    const int part = (int)blockIdx.x >= a.part[0].blocks;
    const Part& p = a.part[part];
    const int bid = blockIdx.x - (part ? a.part[0].blocks : 0), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int warps = kThreads / 32;
    float* acc = sums + warp * a.hd;
    for (int e = lane; e < a.hd; e += 32) acc[e] = 0.f;
    __syncwarp();
    const T* gain = static_cast<const T*>(p.gain);
    const int half = a.rot / 2;
    const long long items = (long long)a.rows * p.heads;
    for (long long item = (long long)bid * warps + warp; item < items; item += (long long)p.blocks * warps) {
        const long long row = item / p.heads;
        const int h = (int)(item - row * p.heads);
        const T* x = head_at<T>(p.x, row, p.x_row, h, p.x_head);
        const T* dy = head_at<T>(p.dy, row, p.dy_row, h, p.dy_head);
        T* to = static_cast<T*>(p.out) + row * p.out_row + h * p.out_head;
        const long long pos = a.positions ? a.positions[row] : 0;
        auto turned = [&](int j, float& z0, float& z1, int& i0, int& i1) {      // pair j of dz
            i0 = INTER ? 2 * j : j;
            i1 = INTER ? 2 * j + 1 : half + j;
            float c, s;
            pair_turn(pos, a.phase[j], 1.f, a.magnitude, c, s);
            const float d0 = to_f(dy[i0]), d1 = to_f(dy[i1]);
            z0 = d0 * c + d1 * s;
            z1 = d1 * c - d0 * s;
        };
        float sq = 0.f, ax = 0.f;
        for (int j = lane; j < half; j += 32) {
            float z0, z1;
            int i0, i1;
            turned(j, z0, z1, i0, i1);
            const float x0 = to_f(x[i0]), x1 = to_f(x[i1]);
            sq = fmaf(x0, x0, fmaf(x1, x1, sq));
            ax = fmaf(z0 * to_f(gain[i0]), x0, fmaf(z1 * to_f(gain[i1]), x1, ax));
        }
        for (int e = a.rot + lane; e < a.hd; e += 32) {
            const float v = to_f(x[e]);
            sq = fmaf(v, v, sq);
            ax = fmaf(to_f(dy[e]) * to_f(gain[e]), v, ax);
        }
        const float r = inv_rms(warp_sum(sq), a.hd, a.eps), f = r * r * warp_sum(ax) / (float)a.hd;
        auto put = [&](int e, float z) {
            const float v = to_f(x[e]);
            acc[e] = fmaf(z, v * r, acc[e]);
            to[e] = from_f<T>(r * (z * to_f(gain[e]) - v * f));
        };
        for (int j = lane; j < half; j += 32) {
            float z0, z1;
            int i0, i1;
            turned(j, z0, z1, i0, i1);
            put(i0, z0);
            put(i1, z1);
        }
        for (int e = a.rot + lane; e < a.hd; e += 32) put(e, to_f(dy[e]));
    }
    __syncthreads();
    add_up(sums, warps, a);
}

// The CTAs' sums of a part's gain gradients, in their order: 32 elements per CTA, 32 warps of which each adds up every 32nd
// row, ten at most at a time (with eight warps 3 us more for 302 rows).
constexpr int kGainThreads = 1024;
__global__ void __launch_bounds__(kGainThreads) qk_norm_gain_kernel(const NormArgs a) {
    __shared__ float sums[kGainThreads / 32][32];
    pdl_wait();
    pdl_trigger();
    const Part& p = a.part[blockIdx.y];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    const float* rows = a.work + (size_t)(blockIdx.y ? a.part[0].blocks : 0) * a.hd;
    float v = 0.f;
    if (e < a.hd) {
#pragma unroll 10
        for (int i = warp; i < p.blocks; i += kGainThreads / 32) v += rows[(size_t)i * a.hd + e];
    }
    sums[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && e < a.hd) {
        v = 0.f;
        for (int w = 0; w < kGainThreads / 32; ++w) v += sums[w][lane];
        p.dgain[e] = v;
    }
}

dflare_status refuse(dflare_status st, const std::string& m) {
    noalloc_set_error(m);
    return st;
}

// CTAs of the parts, in proportion to their work, of `most`
void share_blocks(NormArgs& a, const long long* need, long long most) {
    const long long all = std::max<long long>(need[0] + need[1] + need[2], 1);
    for (int i = 0; i < 3; ++i)
        a.part[i].blocks = (int)(all <= most ? need[i] : need[i] ? std::max<long long>(1, (most - 2) * need[i] / all) : 0);
}
template <class T, bool INTER, bool APPEND, int LANES>
cudaError_t launch_stream(NormArgs& a, bool backward, int num_sms, cudaStream_t s) {
    constexpr int warps = kThreads / 32, many = 32 / LANES;
    // iterations, and one for a row's cosines; CTAs by their shares
    long long need[3], units = 0;
    for (int i = 0; i < 3; ++i) {
        need[i] = a.part[i].heads ? (long long)a.rows * ((a.part[i].heads + many - 1) / many + 1) : 0;
        units += need[i];
    }
    if constexpr (!APPEND) {
        if (backward) {
            static PerDeviceOnce once;
            auto kernel = qk_norm_backward_stream_kernel<T, INTER, LANES>;
            constexpr int ring = warps * Ring<T, 2>::BYTES, sums = kThreads * 16 * 4, bytes = ring > sums ? ring : sums;
            const cudaError_t e = once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
            if (e != cudaSuccess) return e;
            // (two iterations for every warp at least: the CTAs' sums have to be added up. 64 rows 5.8 us, with a CTA for every SM 7.7)
            share_blocks(a, need, std::max<long long>(3, std::min<long long>(std::min(kStreamCtas * num_sms, kWorkRows), units / (warps * 2))));
            return launch_kernel(true, kernel, dim3(a.part[0].blocks + a.part[1].blocks), dim3(kThreads), bytes, s, a);
        }
    }
    static PerDeviceOnce once;
    auto kernel = qk_norm_stream_kernel<T, INTER, APPEND, LANES>;
    constexpr int bytes = warps * Ring<T, 1>::BYTES;
    const cudaError_t e = once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    if (e != cudaSuccess) return e;
    share_blocks(a, need, kStreamCtas * num_sms);
    return launch_kernel(true, kernel, dim3(a.part[0].blocks + a.part[1].blocks + a.part[2].blocks), dim3(kThreads), bytes, s, a);
}
template <class T, bool INTER, bool APPEND>
cudaError_t launch_vec(NormArgs& a, bool backward, int num_sms, cudaStream_t s) {
    if (a.hd <= 64) return launch_stream<T, INTER, APPEND, 4>(a, backward, num_sms, s);
    if (a.hd <= 128) return launch_stream<T, INTER, APPEND, 8>(a, backward, num_sms, s);
    if constexpr (APPEND) return cudaErrorInvalidValue;        // (a cache's heads have 64 or 128 elements)
    else return a.hd <= 256 ? launch_stream<T, INTER, APPEND, 16>(a, backward, num_sms, s) : launch_stream<T, INTER, APPEND, 32>(a, backward, num_sms, s);
}

template <class T, bool INTER, bool APPEND>
cudaError_t launch_forward(NormArgs& a, bool vec, int num_sms, cudaStream_t s) {
    if (vec) return launch_vec<T, INTER, APPEND>(a, false, num_sms, s);
    const long long warps = (long long)a.rows * (a.part[0].heads + a.part[1].heads + a.part[2].heads);
    return launch_kernel(true, qk_norm_any_kernel<T, INTER, APPEND>, dim3((unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32))),
                         dim3(kThreads), 0, s, a);
}
template <bool APPEND>
cudaError_t forward(NormArgs& a, int dtype, int layout, bool vec, int num_sms, cudaStream_t s) {
    if (dtype == DFLARE_BF16)
        return layout == DFLARE_ROPE_INTERLEAVED ? launch_forward<bf16, true, APPEND>(a, vec, num_sms, s)
                                                 : launch_forward<bf16, false, APPEND>(a, vec, num_sms, s);
    return layout == DFLARE_ROPE_INTERLEAVED ? launch_forward<float, true, APPEND>(a, vec, num_sms, s)
                                             : launch_forward<float, false, APPEND>(a, vec, num_sms, s);
}

template <class T, bool INTER>
cudaError_t launch_backward(NormArgs& a, bool vec, int num_sms, cudaStream_t s) {
    cudaError_t e;
    if (vec) {
        e = launch_vec<T, INTER, false>(a, true, num_sms, s);
    } else {
        constexpr int warps = kThreads / 32;
        long long need[3];
        for (int i = 0; i < 3; ++i) need[i] = ((long long)a.rows * a.part[i].heads + warps - 1) / warps;
        share_blocks(a, need, std::min(kStreamCtas * num_sms, kWorkRows));     // CTAs that are resident at once
        e = launch_kernel(true, qk_norm_backward_any_kernel<T, INTER>, dim3(a.part[0].blocks + a.part[1].blocks), dim3(kThreads),
                          (size_t)warps * a.hd * sizeof(float), s, a);
    }
    if (e != cudaSuccess) return e;
    return launch_kernel(true, qk_norm_gain_kernel, dim3((a.hd + 31) / 32, a.part[1].heads ? 2 : 1), dim3(kGainThreads), 0, s, a);
}

// What both directions ask of their arguments; nullptr: nothing is wrong.
const char* check_call(const dflare_qk_heads* q, const dflare_qk_heads* k, const int32_t* positions, const uint64_t* phase, int rows,
                       int head_dim, int rot_dim, int layout, float magnitude, float eps, int dtype, bool backward) {
    if (!q) return "NULL argument";
    if (rot_dim && (!positions || !phase)) return "positions and phases go with a rotation";
    if (rows < 1 || rows > (1 << 24) || head_dim < 2 || head_dim > 1024) return "rows must be in [1, 2^24], head_dim in [2, 1024]";
    if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 2) return "rot_dim must be even, in [0, head_dim]";
    if (layout != DFLARE_ROPE_HALF && layout != DFLARE_ROPE_INTERLEAVED) return "unknown layout";
    if (dtype != DFLARE_BF16 && dtype != DFLARE_F32) return "unknown dtype";
    if (!std::isfinite(magnitude)) return "magnitude must be finite";
    if (!(eps >= 0.f) || !std::isfinite(eps)) return "eps must be finite and not negative";
    long long heads = 0;
    for (const dflare_qk_heads* p : {q, k}) {
        if (!p) continue;
        if (p->heads < 1 || p->heads > 4096) return "heads must be in [1, 4096]";
        if (!p->x || !p->out || !p->gain || (backward && (!p->dy || !p->dgain))) return "NULL argument";
        if (p->x_row < 0 || p->x_head < 0 || p->out_row < 0 || p->out_head < 0 || (backward && (p->dy_row < 0 || p->dy_head < 0)) ||
            (rows > 1 && p->out_row < head_dim) || (p->heads > 1 && p->out_head < head_dim))
            return "strides must not be negative, nor overlap in out";
        // (one of the two strides clears all that the other spans; in floating point, where strides of any size fit)
        const double over_heads = (double)p->out_head * (p->heads - 1) + head_dim, over_rows = (double)p->out_row * (rows - 1) + head_dim;
        if (rows > 1 && p->heads > 1 && (double)p->out_row < over_heads && (double)p->out_head < over_rows)
            return "strides must not be negative, nor overlap in out";
        if (p->x == p->out && (p->x_row != p->out_row || p->x_head != p->out_head)) return "in place needs equal strides";
        if (backward && p->dy == p->out && (p->dy_row != p->out_row || p->dy_head != p->out_head)) return "in place needs equal strides";
        heads += p->heads;
    }
    if ((long long)rows * heads * 32 / kThreads > 0x7ffffff0LL) return "too many heads";
    if (q && k) {       // (both are worked on at the same time)
        if (q->out == k->out || q->out == k->x || k->out == q->x || (backward && (q->out == k->dy || k->out == q->dy)))
            return "queries and keys must not overlap where one is written";
        const uintptr_t a = reinterpret_cast<uintptr_t>(q->dgain), b = reinterpret_cast<uintptr_t>(k->dgain);
        if (backward && (a > b ? a - b : b - a) < head_dim * sizeof(float)) return "the gradients of the gains must not overlap";
    }
    return nullptr;
}

Part part_of(const dflare_qk_heads* p) {
    if (!p) return Part{};
    return Part{p->x, p->x_row, p->x_head, p->dy, p->dy_row, p->dy_head, p->out, p->out_row, p->out_head, p->gain, p->dgain, p->heads, 0};
}
bool part_vec(const Part& p, bool backward) {
    if (!p.heads) return true;
    return aligned16(p.x) && even8(p.x_row) && even8(p.x_head) && aligned16(p.out) && even8(p.out_row) && even8(p.out_head) && aligned16(p.gain) &&
           (!backward || (aligned16(p.dy) && even8(p.dy_row) && even8(p.dy_head)));
}
bool dims_vec(int head_dim, int rot_dim) { return head_dim % 16 == 0 && head_dim <= 512 && rot_dim % 16 == 0; }

}  // namespace
}  // namespace dfl

using namespace dfl;

extern "C" {

dflare_status dflare_qk_norm_rope(const dflare_qk_heads* q, const dflare_qk_heads* k, const int32_t* positions_dev,
                                  const uint64_t* phase_dev, int rows, int head_dim, int rot_dim, int layout, float magnitude, float eps,
                                  int dtype, void* stream) {
    if (const char* m = check_call(q, k, positions_dev, phase_dev, rows, head_dim, rot_dim, layout, magnitude, eps, dtype, false))
        return refuse(DFLARE_EINVAL, std::string("dflare_qk_norm_rope: ") + m);
    NormArgs a{};
    a.part[0] = part_of(q);
    a.part[1] = part_of(k);
    a.positions = positions_dev;
    a.phase = phase_dev;
    a.rows = rows;
    a.hd = head_dim;
    a.rot = rot_dim;
    a.magnitude = magnitude;
    a.eps = eps;
    const bool vec = dims_vec(head_dim, rot_dim) && part_vec(a.part[0], false) && part_vec(a.part[1], false);
    const cudaError_t e = forward<false>(a, dtype, layout, vec, std::max(sms_of_current_device(), 1), static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? DFLARE_OK : refuse(DFLARE_ECUDA, std::string("dflare_qk_norm_rope: ") + cudaGetErrorString(e));
}

dflare_status dflare_qk_norm_rope_backward(const dflare_qk_heads* q, const dflare_qk_heads* k, const int32_t* positions_dev,
                                           const uint64_t* phase_dev, int rows, int head_dim, int rot_dim, int layout, float magnitude,
                                           float eps, float* work_dev, int dtype, void* stream) {
    const char* m = check_call(q, k, positions_dev, phase_dev, rows, head_dim, rot_dim, layout, magnitude, eps, dtype, true);
    if (!m && !work_dev) m = "NULL argument";
    if (m) return refuse(DFLARE_EINVAL, std::string("dflare_qk_norm_rope_backward: ") + m);
    NormArgs a{};
    a.part[0] = part_of(q);
    a.part[1] = part_of(k);
    a.positions = positions_dev;
    a.phase = phase_dev;
    a.work = work_dev;
    a.rows = rows;
    a.hd = head_dim;
    a.rot = rot_dim;
    a.magnitude = magnitude;
    a.eps = eps;
    const bool vec = dims_vec(head_dim, rot_dim) && part_vec(a.part[0], true) && part_vec(a.part[1], true);
    const int sms = std::max(sms_of_current_device(), 1);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool inter = layout == DFLARE_ROPE_INTERLEAVED;
    const cudaError_t e = dtype == DFLARE_BF16 ? (inter ? launch_backward<bf16, true>(a, vec, sms, s) : launch_backward<bf16, false>(a, vec, sms, s))
                                               : (inter ? launch_backward<float, true>(a, vec, sms, s) : launch_backward<float, false>(a, vec, sms, s));
    return e == cudaSuccess ? DFLARE_OK : refuse(DFLARE_ECUDA, std::string("dflare_qk_norm_rope_backward: ") + cudaGetErrorString(e));
}

dflare_status dflare_cache_append_normed(dflare_cache* c, int layer, const void* q_dev, long long q_row, const void* k_dev,
                                         long long k_row, const void* v_dev, long long v_row, void* q_out_dev, long long out_row,
                                         const void* q_gain_dev, const void* k_gain_dev, float eps, const int32_t* depth_dev,
                                         const int32_t* n_new_dev, int batch, int n_max, const uint64_t* phase_dev, int rot_dim, int layout,
                                         float magnitude, void* stream) {
    auto bad = [](const char* m) { return refuse(DFLARE_EINVAL, std::string("dflare_cache_append_normed: ") + m); };
    if (!c || !k_dev || !v_dev || !n_new_dev || !k_gain_dev) return bad("NULL argument");
    if (!q_dev != !q_out_dev) return bad("q and q_out go together");
    if (q_dev && !q_gain_dev) return bad("queries need their gain");
    const dflare_cache_config& g = c->cfg;
    if (layer < 0 || layer >= g.n_layers) return bad("layer out of range");
    if (batch < 1 || batch > g.max_batch) return bad("batch must be in [1, max_batch]");
    if (n_max < 1 || n_max > (1 << 20)) return bad("n_max must be in [1, 2^20]");
    if (rot_dim < 0 || rot_dim > g.head_dim || rot_dim % 2 || (rot_dim && !phase_dev))
        return bad("rot_dim must be even, in [0, head_dim], with phases where it is not 0");
    if (layout != DFLARE_ROPE_HALF && layout != DFLARE_ROPE_INTERLEAVED) return bad("unknown layout");
    if (!std::isfinite(magnitude)) return bad("magnitude must be finite");
    if (!(eps >= 0.f) || !std::isfinite(eps)) return bad("eps must be finite and not negative");
    const long long kv = (long long)g.n_kv_heads * g.head_dim, qw = (long long)g.n_q_heads * g.head_dim;
    if (k_row < kv || v_row < kv || (q_dev && (q_row < qw || out_row < qw))) return bad("a row stride is below a row's heads");
    if (q_dev && q_dev == q_out_dev && q_row != out_row) return bad("in place needs equal strides");
    const int hd = g.head_dim;
    if ((long long)batch * n_max * ((q_dev ? g.n_q_heads : 0) + 2 * g.n_kv_heads) * 32 / kThreads > 0x7ffffff0LL) return bad("too many heads");
    NormArgs a{};
    if (q_dev) a.part[0] = Part{q_dev, q_row, hd, nullptr, 0, 0, q_out_dev, out_row, hd, q_gain_dev, nullptr, g.n_q_heads, 0};
    a.part[1] = Part{k_dev, k_row, hd, nullptr, 0, 0, nullptr, 0, 0, k_gain_dev, nullptr, g.n_kv_heads, 0};
    a.part[2] = Part{v_dev, v_row, hd, nullptr, 0, 0, nullptr, 0, 0, nullptr, nullptr, g.n_kv_heads, 0};
    a.phase = phase_dev;
    a.rows = batch * n_max;
    a.hd = hd;
    a.rot = rot_dim;
    a.magnitude = magnitude;
    a.eps = eps;
    a.pg = c->view;
    a.rows_of = AppendRows{depth_dev, n_new_dev, layer, n_max};
    const bool vec = rot_dim % 16 == 0 && part_vec(a.part[0], false) && part_vec(a.part[1], false) && part_vec(a.part[2], false);
    DeviceGuard guard(c->device);
    const cudaError_t e = forward<true>(a, g.dtype, layout, vec, c->num_sms, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? DFLARE_OK : refuse(DFLARE_ECUDA, std::string("dflare_cache_append_normed: ") + cudaGetErrorString(e));
}

}  // extern "C"
