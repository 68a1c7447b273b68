// Rotary positions, alone (dflare_rope) and on a step's queries and keys on their way into the pages of a
// cache (dflare_cache_append).
//
// Angles: a pair's frequency is held as turns per position in units of 2^-64, so position * phase in 64-bit
// integers, which wrap at a whole turn, is the angle's fraction of a turn with no error but the phase's: the phases
// are computed in double precision, so position * 2^-52 turns at most (measured, 2^-55 for the fastest pair).
// In fp32 the product position * inv_freq would be off by up to 0.03 radians at position 10^6; a table of
// cosines for 131072 positions of 64 pairs would be 64 MB that the pages' traffic evicts.
//
// Work: 16 elements of a head ("unit": eight pairs, or 16 elements that are only copied). A thread keeps one
// row's unit and walks over heads, so a cosine and sine serve all its heads. HBM-bound for many rows: 10563 rows of
// 40 bf16 heads of 128, 34.1 us, 6.3 TB/s; a step's few rows are one trip through lengths, page table and rows (3.7 us).
#include <math.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "common.cuh"
#include "paged.h"

namespace dfl {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kBatchHeads = 4;      // heads whose loads are in flight together

struct RopeArgs {
    const void* x[3];          // q (or the only input), k, v
    long long x_row[3], x_head;
    void* out;                 // of x[0]
    long long out_row, out_head;
    const int32_t* positions;  // dflare_rope: [rows]
    const uint64_t* phase;
    int rows, heads;           // heads: of x[0]
    int hd, rot;
    float magnitude, sign;
    // dflare_cache_append
    PagesView pg;
    const int32_t* depth;
    const int32_t* n_new;
    int layer, n_max;
    int slots;                 // threads that share one row's unit
};

__device__ __forceinline__ void pair_turn(long long pos, uint64_t phase, float sign, float magnitude, float& c, float& s) {
    // [-1/2, 1/2) turns; sincospi of twice that
    const float turns = (float)(long long)((uint64_t)pos * phase) * 5.4210108624275222e-20f;
    sincospif(2.0f * turns, &s, &c);
    c *= magnitude;
    s *= magnitude * sign;
}

// row -> position, and whether there is anything to do; slot: where its key and value go (-1: nowhere)
template <bool APPEND>
__device__ __forceinline__ bool row_of(const RopeArgs& a, int row, long long& pos, long long& slot) {
    slot = -1;
    if (!APPEND) {
        pos = a.positions[row];
        return true;
    }
    const int b = row / a.n_max, i = row - b * a.n_max;
    if (i >= a.n_new[b]) return false;
    const int len = a.pg.lens[b];
    pos = (long long)len + (a.depth ? a.depth[row] : i);
    const long long at = (long long)len + i;
    const long long room = (long long)min(a.pg.held[b], a.pg.max_pages) * a.pg.ps;
    uint32_t err = DFLARE_DEVERR_CAPACITY;
    if (len >= 0 && at < room) {
        const int page = a.pg.table[(size_t)b * a.pg.max_pages + at / a.pg.ps];
        err = DFLARE_DEVERR_PAGE;
        // the page that holds the last tokens may still be shared where no room was reserved: it is not written
        if (page >= 0 && page < a.pg.pages && !(at / a.pg.ps == len / a.pg.ps && len % a.pg.ps && a.pg.refs[page] > 1))
            slot = ((long long)a.layer * a.pg.pages + page) * a.pg.hkv * a.pg.ps + at % a.pg.ps;
    }
    if (slot < 0) atomicOr(a.pg.err, err);
    return true;
}

// Where head h of a row is read and written (in an append heads are numbered q, then k, then v), and whether it
// turns; false: nowhere.
template <class T, bool APPEND>
__device__ __forceinline__ bool place_of(const RopeArgs& a, int row, int h, long long slot, const T*& from, T*& to, bool& turn) {
    turn = true;
    if (h < a.heads) {
        from = static_cast<const T*>(a.x[0]) + row * a.x_row[0] + h * a.x_head;
        to = static_cast<T*>(a.out) + row * a.out_row + h * a.out_head;
        return true;
    }
    const bool is_v = h >= a.heads + a.pg.hkv;
    const int g = h - a.heads - (is_v ? a.pg.hkv : 0);
    from = static_cast<const T*>(a.x[is_v ? 2 : 1]) + row * a.x_row[is_v ? 2 : 1] + (long long)g * a.hd;
    to = static_cast<T*>(is_v ? a.pg.v : a.pg.k) + (slot + (long long)g * a.pg.ps) * a.hd;
    turn = !is_v;
    return slot >= 0;
}

// 16 elements of storage in two runs of eight, as loaded; and their values
template <class T> struct Unit { uint4 v[sizeof(T)]; };      // bf16: one 16-byte piece per run, fp32: two
template <class T>
__device__ __forceinline__ void load_unit(Unit<T>& x, const T* p0, const T* p1) {
    constexpr int H = sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < H; ++i) {
        x.v[i] = reinterpret_cast<const uint4*>(p0)[i];
        x.v[H + i] = reinterpret_cast<const uint4*>(p1)[i];
    }
}
template <class T>
__device__ __forceinline__ void store_unit(const Unit<T>& x, T* p0, T* p1) {
    constexpr int H = sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < H; ++i) {
        reinterpret_cast<uint4*>(p0)[i] = x.v[i];
        reinterpret_cast<uint4*>(p1)[i] = x.v[H + i];
    }
}
__device__ __forceinline__ float2 get2(const Unit<bf16>& x, int i) { return __bfloat1622float2(reinterpret_cast<const __nv_bfloat162*>(x.v)[i]); }
__device__ __forceinline__ float2 get2(const Unit<float>& x, int i) { return reinterpret_cast<const float2*>(x.v)[i]; }
__device__ __forceinline__ void set2(Unit<bf16>& x, int i, float a, float b) { reinterpret_cast<__nv_bfloat162*>(x.v)[i] = __floats2bfloat162_rn(a, b); }
__device__ __forceinline__ void set2(Unit<float>& x, int i, float a, float b) { reinterpret_cast<float2*>(x.v)[i] = make_float2(a, b); }

// Vector form: rot and hd multiples of 16, everything 16-byte aligned. A thread's first heads are on their way
// before it works out its cosines, and stay as they were stored until they are turned.
template <class T, bool INTER, bool APPEND>
__global__ void __launch_bounds__(kRopeThreads, sizeof(T) == 2 ? 3 : 2) rope_kernel(const RopeArgs a) {
    pdl_wait();
    pdl_trigger();
    const int units = a.hd / 16, rot_units = a.rot / 16, half = a.rot / 2;
    const int total_heads = a.heads + (APPEND ? 2 * a.pg.hkv : 0);
    const long long t = (long long)blockIdx.x * kRopeThreads + threadIdx.x;
    const int u = (int)(t % units);
    const long long rest = t / units;
    const int h0 = (int)(rest % a.slots);
    const long long row = rest / a.slots;
    if (row >= a.rows) return;
    long long pos, slot;
    if (!row_of<APPEND>(a, (int)row, pos, slot)) return;
    const bool rotates = u < rot_units;
    // the unit's two runs of eight elements
    const int e0 = rotates && !INTER ? u * 8 : u * 16, e1 = rotates && !INTER ? half + u * 8 : u * 16 + 8;
    float c[8], s[8];
    for (int h = h0; h < total_heads; h += a.slots * kBatchHeads) {
        Unit<T> x[kBatchHeads];
#pragma unroll
        for (int k = 0; k < kBatchHeads; ++k) {
            const int hk = h + k * a.slots;
            const T* from;
            T* to;
            bool turn;
            if (hk < total_heads && place_of<T, APPEND>(a, (int)row, hk, slot, from, to, turn)) load_unit(x[k], from + e0, from + e1);
        }
        if (h == h0 && rotates) {
#pragma unroll
            for (int j = 0; j < 8; ++j) pair_turn(pos, a.phase[u * 8 + j], a.sign, a.magnitude, c[j], s[j]);
        }
#pragma unroll
        for (int k = 0; k < kBatchHeads; ++k) {
            const int hk = h + k * a.slots;
            const T* from;
            T* to;
            bool turn;
            if (hk >= total_heads || !place_of<T, APPEND>(a, (int)row, hk, slot, from, to, turn)) continue;
            if (rotates && turn) {
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    if (INTER) {        // pairs are neighbours: two of them in a float2 each
#pragma unroll
                        for (int i = j; i < j + 2; ++i) {
                            const float2 v = get2(x[k], i);
                            set2(x[k], i, v.x * c[i] - v.y * s[i], v.y * c[i] + v.x * s[i]);
                        }
                    } else {            // pairs are eight (here four float2) apart
                        const float2 v = get2(x[k], j / 2), w = get2(x[k], 4 + j / 2);
                        set2(x[k], j / 2, v.x * c[j] - w.x * s[j], v.y * c[j + 1] - w.y * s[j + 1]);
                        set2(x[k], 4 + j / 2, w.x * c[j] + v.x * s[j], w.y * c[j + 1] + v.y * s[j + 1]);
                    }
                }
            }
            store_unit(x[k], to + e0, to + e1);
        }
    }
}

// Any rot, hd, strides and alignment: a thread per pair (or per two copied elements) of a head.
template <class T, bool INTER, bool APPEND>
__global__ void __launch_bounds__(kRopeThreads) rope_any_kernel(const RopeArgs a) {
    pdl_wait();
    pdl_trigger();
    const int half = a.rot / 2, units = half + (a.hd - a.rot + 1) / 2;
    const int total_heads = a.heads + (APPEND ? 2 * a.pg.hkv : 0);
    const long long t = (long long)blockIdx.x * kRopeThreads + threadIdx.x;
    const int u = (int)(t % units);
    const long long rest = t / units;
    const int h = (int)(rest % total_heads);
    const long long row = rest / total_heads;
    if (row >= a.rows) return;
    long long pos, slot;
    if (!row_of<APPEND>(a, (int)row, pos, slot)) return;
    const T* from;
    T* to;
    bool turn;
    if (!place_of<T, APPEND>(a, (int)row, h, slot, from, to, turn)) return;
    const int e0 = u >= half ? a.rot + 2 * (u - half) : INTER ? 2 * u : u;
    const int e1 = u >= half ? e0 + 1 : INTER ? e0 + 1 : half + u;
    const bool two = e1 < a.hd;
    const T a0 = from[e0], a1 = two ? from[e1] : a0;
    if (u < half && turn) {
        float c, s;
        pair_turn(pos, a.phase[u], a.sign, a.magnitude, c, s);
        const float x0 = to_f(a0), x1 = to_f(a1);
        to[e0] = from_f<T>(x0 * c - x1 * s);
        to[e1] = from_f<T>(x1 * c + x0 * s);
    } else {
        to[e0] = a0;
        if (two) to[e1] = a1;
    }
}

dflare_status refuse(dflare_status st, const std::string& m) {
    noalloc_set_error(m);
    return st;
}

template <class T, bool INTER, bool APPEND>
cudaError_t launch_typed(RopeArgs& a, bool vec, int num_sms, cudaStream_t s) {
    const int total_heads = a.heads + (APPEND ? 2 * a.pg.hkv : 0);
    if (vec) {
        // heads per thread: one while that still fits the GPU at once, up to eight where rows are many and
        // a cosine should serve several heads
        const long long units = (long long)a.rows * (a.hd / 16);
        const long long fit = std::max<long long>(1, units * total_heads / ((long long)num_sms * 2048));
        a.slots = (int)((total_heads + std::min<long long>(fit, 8) - 1) / std::min<long long>(fit, 8));
        const long long blocks = (units * a.slots + kRopeThreads - 1) / kRopeThreads;
        return launch_kernel(true, rope_kernel<T, INTER, APPEND>, dim3((unsigned)blocks), dim3(kRopeThreads), 0, s, a);
    }
    const long long threads = (long long)a.rows * total_heads * (a.rot / 2 + (a.hd - a.rot + 1) / 2);
    const long long blocks = (threads + kRopeThreads - 1) / kRopeThreads;
    return launch_kernel(true, rope_any_kernel<T, INTER, APPEND>, dim3((unsigned)blocks), dim3(kRopeThreads), 0, s, a);
}

template <bool APPEND>
cudaError_t launch_rope(RopeArgs& a, int dtype, int layout, bool vec, int num_sms, cudaStream_t s) {
    if (dtype == DFLARE_BF16)
        return layout == DFLARE_ROPE_INTERLEAVED ? launch_typed<bf16, true, APPEND>(a, vec, num_sms, s)
                                                 : launch_typed<bf16, false, APPEND>(a, vec, num_sms, s);
    return layout == DFLARE_ROPE_INTERLEAVED ? launch_typed<float, true, APPEND>(a, vec, num_sms, s)
                                             : launch_typed<float, false, APPEND>(a, vec, num_sms, s);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// elements that keep 16-byte alignment for either type
bool even8(long long n) { return n % 8 == 0; }

int sms_of_current_device() {
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    int n = known[dev & 63].load(std::memory_order_relaxed);
    if (n == 0 && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess)
        known[dev & 63].store(n, std::memory_order_relaxed);
    return n;
}

}  // namespace
}  // namespace dfl

using namespace dfl;

extern "C" {

dflare_status dflare_rope_phases(const dflare_rope_config* g, uint64_t* phase_host, float* magnitude_host) {
    auto bad = [](const char* m) { return refuse(DFLARE_EINVAL, std::string("dflare_rope_phases: ") + m); };
    if (!g || !phase_host || !magnitude_host) return bad("NULL argument");
    if (g->rot_dim < 2 || g->rot_dim > 1024 || g->rot_dim % 2) return bad("rot_dim must be even, in [2, 1024]");
    if (g->scaling < DFLARE_ROPE_PLAIN || g->scaling > DFLARE_ROPE_YARN) return bad("unknown scaling");
    if (!(g->theta > 1.0) || !std::isfinite(g->theta)) return bad("theta must be above 1");
    const bool scaled = g->scaling != DFLARE_ROPE_PLAIN;
    if (scaled && (!(g->factor >= 1.0) || !std::isfinite(g->factor))) return bad("factor must be at least 1");
    if (g->scaling == DFLARE_ROPE_NTK && g->rot_dim == 2) return bad("NTK scaling needs rot_dim above 2");
    if (g->scaling == DFLARE_ROPE_YARN &&
        (!(g->trained >= 1.0) || !std::isfinite(g->trained) || !(g->beta_slow > 0.0) || !(g->beta_fast > g->beta_slow) ||
         !std::isfinite(g->beta_fast)))
        return bad("YARN needs trained >= 1 and beta_fast > beta_slow > 0");
    const double two_pi = 6.283185307179586476925;
    const int half = g->rot_dim / 2;
    double theta = g->theta;
    if (g->scaling == DFLARE_ROPE_NTK) theta *= std::pow(g->factor, g->rot_dim / (g->rot_dim - 2.0));
    // YARN: the (fractional) pair that turns `beta` times within the trained positions. The mix runs from the last pair with
    // beta_fast turns or more to the first with beta_slow or fewer, either of which may lie beyond the head's pairs: ends
    // drawn in to pairs that the head has would change the frequencies of the pairs between.
    auto pair_at = [&](double beta) { return g->rot_dim * std::log(g->trained / (beta * two_pi)) / (2.0 * std::log(theta)); };
    double lo = 0, hi = 0;
    if (g->scaling == DFLARE_ROPE_YARN) {
        lo = std::floor(pair_at(g->beta_fast));
        hi = std::ceil(pair_at(g->beta_slow));
    }
    for (int j = 0; j < half; ++j) {
        double inv = std::pow(theta, -2.0 * j / g->rot_dim);
        if (g->scaling == DFLARE_ROPE_LINEAR) inv /= g->factor;
        if (g->scaling == DFLARE_ROPE_YARN) {
            const double mix = std::min(std::max((j - lo) / std::max(hi - lo, 1.0), 0.0), 1.0);
            inv = inv * (1.0 - mix) + inv / g->factor * mix;
        }
        phase_host[j] = (uint64_t)std::ldexp(inv / two_pi, 64);    // below 2^64 / 6: inv <= 1
    }
    *magnitude_host = g->scaling == DFLARE_ROPE_YARN ? (float)(0.1 * std::log(g->factor) + 1.0) : 1.0f;
    return DFLARE_OK;
}

dflare_status dflare_rope(const void* x_dev, long long x_row, long long x_head, void* out_dev, long long out_row,
                          long long out_head, const int32_t* positions_dev, const uint64_t* phase_dev, int rows, int heads,
                          int head_dim, int rot_dim, int layout, float magnitude, int backward, int dtype, void* stream) {
    auto bad = [](const char* m) { return refuse(DFLARE_EINVAL, std::string("dflare_rope: ") + m); };
    if (!x_dev || !out_dev || !positions_dev || !phase_dev) return bad("NULL argument");
    if (rows < 1 || rows > (1 << 24) || heads < 1 || heads > 4096 || head_dim < 2 || head_dim > 1024)
        return bad("rows must be in [1, 2^24], heads in [1, 4096], head_dim in [2, 1024]");
    if (rot_dim < 2 || rot_dim > head_dim || rot_dim % 2) return bad("rot_dim must be even, in [2, head_dim]");
    if (layout != DFLARE_ROPE_HALF && layout != DFLARE_ROPE_INTERLEAVED) return bad("unknown layout");
    if (dtype != DFLARE_BF16 && dtype != DFLARE_F32) return bad("unknown dtype");
    if (!std::isfinite(magnitude)) return bad("magnitude must be finite");
    if (x_row < 0 || x_head < 0 || (rows > 1 && out_row < head_dim) || (heads > 1 && out_head < head_dim) || out_row < 0 || out_head < 0)
        return bad("strides must not be negative, nor overlap in out");
    if (x_dev == out_dev && (x_row != out_row || x_head != out_head)) return bad("in place needs equal strides");
    if ((long long)rows * heads * head_dim / 2 / kRopeThreads > 0x7ffffff0LL) return bad("too many elements");
    RopeArgs a{};
    a.x[0] = x_dev;
    a.x_row[0] = x_row;
    a.x_head = x_head;
    a.out = out_dev;
    a.out_row = out_row;
    a.out_head = out_head;
    a.positions = positions_dev;
    a.phase = phase_dev;
    a.rows = rows;
    a.heads = heads;
    a.hd = head_dim;
    a.rot = rot_dim;
    a.magnitude = magnitude;
    a.sign = backward ? -1.f : 1.f;
    const bool vec = rot_dim % 16 == 0 && head_dim % 16 == 0 && aligned16(x_dev) && aligned16(out_dev) && even8(x_row) &&
                     even8(x_head) && even8(out_row) && even8(out_head);
    const cudaError_t e = launch_rope<false>(a, dtype, layout, vec, std::max(sms_of_current_device(), 1), static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? DFLARE_OK : refuse(DFLARE_ECUDA, std::string("dflare_rope: ") + cudaGetErrorString(e));
}

dflare_status dflare_cache_append(dflare_cache* c, int layer, const void* q_dev, long long q_row, const void* k_dev,
                                  long long k_row, const void* v_dev, long long v_row, void* q_out_dev, long long out_row,
                                  const int32_t* depth_dev, const int32_t* n_new_dev, int batch, int n_max,
                                  const uint64_t* phase_dev, int rot_dim, int layout, float magnitude, void* stream) {
    auto bad = [](const char* m) { return refuse(DFLARE_EINVAL, std::string("dflare_cache_append: ") + m); };
    if (!c || !k_dev || !v_dev || !n_new_dev) return bad("NULL argument");
    if (!q_dev != !q_out_dev) return bad("q and q_out go together");
    const dflare_cache_config& g = c->cfg;
    if (layer < 0 || layer >= g.n_layers) return bad("layer out of range");
    if (batch < 1 || batch > g.max_batch) return bad("batch must be in [1, max_batch]");
    if (n_max < 1 || n_max > (1 << 20)) return bad("n_max must be in [1, 2^20]");
    if (rot_dim < 0 || rot_dim > g.head_dim || rot_dim % 2 || (rot_dim && !phase_dev))
        return bad("rot_dim must be even, in [0, head_dim], with phases where it is not 0");
    if (layout != DFLARE_ROPE_HALF && layout != DFLARE_ROPE_INTERLEAVED) return bad("unknown layout");
    if (!std::isfinite(magnitude)) return bad("magnitude must be finite");
    const long long kv = (long long)g.n_kv_heads * g.head_dim, qw = (long long)g.n_q_heads * g.head_dim;
    if (k_row < kv || v_row < kv || (q_dev && (q_row < qw || out_row < qw))) return bad("a row stride is below a row's heads");
    if (q_dev && q_dev == q_out_dev && q_row != out_row) return bad("in place needs equal strides");
    RopeArgs a{};
    a.x[0] = q_dev;
    a.x[1] = k_dev;
    a.x[2] = v_dev;
    a.x_row[0] = q_row;
    a.x_row[1] = k_row;
    a.x_row[2] = v_row;
    a.x_head = a.out_head = g.head_dim;
    a.out = q_out_dev;
    a.out_row = out_row;
    a.phase = phase_dev;
    a.rows = batch * n_max;
    a.heads = q_dev ? g.n_q_heads : 0;
    a.hd = g.head_dim;
    a.rot = rot_dim;
    a.magnitude = magnitude;
    a.sign = 1.f;
    a.pg = c->view;
    a.depth = depth_dev;
    a.n_new = n_new_dev;
    a.layer = layer;
    a.n_max = n_max;
    DeviceGuard guard(c->device);
    const bool vec = rot_dim % 16 == 0 && aligned16(k_dev) && aligned16(v_dev) && even8(k_row) && even8(v_row) &&
                     (!q_dev || (aligned16(q_dev) && aligned16(q_out_dev) && even8(q_row) && even8(out_row)));
    const cudaError_t e = launch_rope<true>(a, g.dtype, layout, vec, c->num_sms, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? DFLARE_OK : refuse(DFLARE_ECUDA, std::string("dflare_cache_append: ") + cudaGetErrorString(e));
}

}  // extern "C"
