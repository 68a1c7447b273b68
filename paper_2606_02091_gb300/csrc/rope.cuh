// Rotary positions of a head's elements, and where an append's rows go: shared by the kernels that rotate (rope.cu)
// and that norm and rotate (qk_norm.cu).
#pragma once
#include <algorithm>

#include "common.cuh"
#include "paged.h"

namespace dfl {

__device__ __forceinline__ void pair_turn(long long pos, uint64_t phase, float sign, float magnitude, float& c, float& s) {
    // [-1/2, 1/2) turns; sincospi of twice that
    const float turns = (float)(long long)((uint64_t)pos * phase) * 5.4210108624275222e-20f;
    sincospif(2.0f * turns, &s, &c);
    c *= magnitude;
    s *= magnitude * sign;
}

// Row i of sequence b in an append: its position, and the slot of its key and value in a layer's pool (-1: nowhere, and
// reported). False: the row is past the sequence's new tokens.
struct AppendRows {
    const int32_t* depth;
    const int32_t* n_new;
    int layer, n_max;
};
__device__ __forceinline__ bool append_row(const PagesView& pg, const AppendRows& a, int row, long long& pos, long long& slot) {
    slot = -1;
    const int b = row / a.n_max, i = row - b * a.n_max;
    // (all of them under way before one is looked at)
    const int n_new = a.n_new[b], len = pg.lens[b], held = pg.held[b], depth = a.depth ? a.depth[row] : i;
    if (i >= n_new) return false;
    pos = (long long)len + depth;
    const long long at = (long long)len + i;
    const long long room = (long long)min(held, pg.max_pages) * pg.ps;
    uint32_t err = DFLARE_DEVERR_CAPACITY;
    if (len >= 0 && at < room) {
        const int page = pg.table[(size_t)b * pg.max_pages + at / pg.ps];
        err = DFLARE_DEVERR_PAGE;
        // the page that holds the last tokens may still be shared where no room was reserved: it is not written
        if (page >= 0 && page < pg.pages && !(at / pg.ps == len / pg.ps && len % pg.ps && pg.refs[page] > 1))
            slot = ((long long)a.layer * pg.pages + page) * pg.hkv * pg.ps + at % pg.ps;
    }
    if (slot < 0) atomicOr(pg.err, err);
    return true;
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

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// elements that keep 16-byte alignment for either type
inline bool even8(long long n) { return n % 8 == 0; }

inline int sms_of_current_device() {
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    int n = known[dev & 63].load(std::memory_order_relaxed);
    if (n == 0 && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess)
        known[dev & 63].store(n, std::memory_order_relaxed);
    return n;
}

}  // namespace dfl
