// Pages of a paged cache: taking them from the free stack (with copy on write), sharing, giving back,
// copying, and moving an accepted path's rows together.
//
// Every kernel here lets the next one start as soon as its own dependency wait is over: the next one's launch and
// prologue then overlap, and its own wait still lasts until this one has ended.
// Who holds what is kept in four small integer arrays (page table, pages held, reference counts, free
// stack). One CTA works on them per call, so that the order in which pages are taken and given back, and
// with it every page number, is the same on every run; the bytes are moved by kernels over the whole GPU.
#include <algorithm>
#include <new>
#include <string>

#include "common.cuh"
#include "paged.h"

namespace dfl {
namespace {

constexpr int kMetaThreads = 1024;
constexpr int kCopyThreads = 256;

// Inclusive sums over the CTA's threads (a multiple of 32, at most 1024); `tmp` holds 32 ints.
__device__ __forceinline__ int block_scan(int v, int* tmp, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    __syncthreads();
    if (lane == 31) tmp[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int t = lane < (int)(blockDim.x >> 5) ? tmp[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, t, o);
            if (lane >= o) t += x;
        }
        tmp[lane] = t;
    }
    __syncthreads();
    *total = tmp[31];
    return v + (warp ? tmp[warp - 1] : 0);
}

// the sequence whose entries [first[b], first[b + 1]) hold e, e < first[n]
__device__ __forceinline__ int entry_owner(const int* first, int n, int e) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= e) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int pages_of(int tokens, int ps) { return (tokens + ps - 1) / ps; }

// Whether sequence b can commit `a` nodes of `path`: 0 <= a <= n, numbers increasing from 0 or more, all their slots
// on pages that it holds, and the page with its last tokens its own (it is, once room was reserved). The answer is
// the same in every lane of the calling warp.
__device__ __forceinline__ bool path_fits(const PagesView& pg, int b, const int32_t* path, int a, int n, int len, int held) {
    bool ok = len >= 0 && a >= 0 && a <= n;
    const bool tail = ok && a > 0 && len % pg.ps && len / pg.ps < min(held, pg.max_pages);
    const int page = tail ? pg.table[(size_t)b * pg.max_pages + len / pg.ps] : 0;      // (under way with the path)
    const int room = min(held, pg.max_pages) * pg.ps - len;     // slots behind len
    for (int j = threadIdx.x & 31; ok && j < a; j += 32) {
        const int x = path[j], before = j ? path[j - 1] : -1;
        if (x <= before || x >= room) ok = false;
    }
    if (tail && (page < 0 || page >= pg.pages || pg.refs[page] > 1)) ok = false;
    return __all_sync(0xffffffffu, ok);
}

// lens and the pages past them. Entry e of the call is one page that a sequence lets go, numbered by
// sequence and then by position. All entries take one off their page's count and leave their number with the
// page, where the largest stays; then those whose page has no count left and still holds their number (a page
// that several sequences let go at once is pushed once, where the last of them stands) are pushed in order.
// add != NULL: lens grows by the accepted lengths; else it is cut to new_len. Latency-bound: a chain of four
// trips to memory.
__global__ void __launch_bounds__(kMetaThreads) trim_kernel(const PagesView pg, const int32_t* __restrict__ new_len,
                                                            const int32_t* __restrict__ add,
                                                            const int32_t* __restrict__ path, int path_row,
                                                            int32_t* __restrict__ last, int n) {
    __shared__ int first[kMaxSeqs + 1], from[kMaxSeqs], tmp[32];
    const int tid = threadIdx.x;
    // Behind the moving launch (add), which lets this one start after its own dependency wait and writes nothing that is
    // read here, everything is found out while it moves; only the writes wait for it.
    if (!add) pdl_wait();
    // a count that no stack of `pages` entries has is reported, and taken as empty or full: pushes stay in the array
    const int told = *pg.n_free;
    int top = min(max(told, 0), pg.pages);
    if (told != top && tid == 0) atomicOr(pg.err, DFLARE_DEVERR_PAGE);
    if (add) {
        // a path that does not fit commits nothing (the moving kernel decided the same); from[] holds
        // the new length until the pages are counted
        for (int b = tid >> 5; b < n; b += kMetaThreads / 32) {
            const int len = pg.lens[b], a = add[b];
            const bool fits = path_fits(pg, b, path + (size_t)b * path_row, a, path_row, len, pg.held[b]);
            if ((tid & 31) == 0) {
                from[b] = fits ? len + a : len;
                if (!fits) atomicOr(pg.err, DFLARE_DEVERR_TREE);
            }
        }
        __syncthreads();
    }
    int gone = 0, old = 0, len = 0, keep = 0;
    if (tid < n) {
        old = pg.lens[tid];
        len = add ? from[tid] : min(old, max(new_len[tid], 0));
        const int held = min(max(pg.held[tid], 0), pg.max_pages);
        keep = pages_of(max(len, 0), pg.ps);
        gone = max(held - keep, 0);
        from[tid] = keep;
    }
    int total;
    const int upto = block_scan(gone, tmp, &total);
    if (tid < n) first[tid + 1] = upto;
    if (tid == 0) first[0] = 0;
    __syncthreads();
    auto entry = [&](int e, int* slot) {
        const int b = entry_owner(first, n, e);
        *slot = b * pg.max_pages + from[b] + e - first[b];
        const int p = pg.table[*slot];
        return p >= 0 && p < pg.pages ? p : -1;
    };
    int slot, mine = tid < total ? entry(tid, &slot) : -1;
    if (add) pdl_wait();
    pdl_trigger();
    if (tid < n) {
        if (len != old) pg.lens[tid] = len;
        if (gone) pg.held[tid] = keep;
    }
    if (total == 0) return;
    for (int e = tid; e < total; e += kMetaThreads) {
        const int p = e == tid ? mine : entry(e, &slot);
        if (p >= 0) {
            atomicSub(&pg.refs[p], 1);
            atomicMax(&last[p], e);
        } else {
            atomicOr(pg.err, DFLARE_DEVERR_PAGE);
        }
    }
    __syncthreads();
    for (int e0 = 0; e0 < total; e0 += kMetaThreads) {
        const int e = e0 + tid;
        const int p = e0 == 0 ? mine : e < total ? entry(e, &slot) : -1;
        bool push = false;
        if (p >= 0) {
            const int refs = __ldcg(&pg.refs[p]), winner = __ldcg(&last[p]);
            push = refs == 0 && winner == e;
            if (refs < 0) atomicOr(pg.err, DFLARE_DEVERR_PAGE);
        }
        int pushed;
        const int at = top + block_scan(push ? 1 : 0, tmp, &pushed) - 1;
        if (push && at < pg.pages) pg.free_pages[at] = p;
        top += pushed;
    }
    if (tid == 0) {
        if (top > pg.pages) atomicOr(pg.err, DFLARE_DEVERR_PAGE);
        *pg.n_free = min(top, pg.pages);
    }
    __syncthreads();
    for (int e = tid; e < total; e += kMetaThreads) {
        const int p = entry(e, &slot);
        if (p >= 0) last[p] = -1;
        pg.table[slot] = -1;
    }
}

// Room for n_new tokens. Thread b counts sequence b's pages; "shared at its turn": refs minus the
// sequences before it that share its partly filled page and write to it too is above one (each of those
// has taken a copy by then). The copies go to a list that copy_kernel works off. Nothing is written before the free
// stack is known to hold what is taken: a count that it cannot have, or a page number that does not exist, takes nothing.
__global__ void __launch_bounds__(kMetaThreads) reserve_kernel(const PagesView pg, const int32_t* __restrict__ n_new,
                                                               int32_t* __restrict__ copies, int n) {
    __shared__ int first[kMaxSeqs + 1], held0[kMaxSeqs], tail[kMaxSeqs], copy_of[kMaxSeqs], tmp[32], bad;
    __shared__ int avail[kMetaThreads];     // the first free pages, looked up while the need is counted
    const int tid = threadIdx.x;
    if (tid == 0) bad = 0;
    pdl_wait();
    pdl_trigger();
    const int top = *pg.n_free;
    const bool stack_ok = top >= 0 && top <= pg.pages;
    int grow = 0, len = 0, held = 0, fresh = 0, page = -1;
    if (tid < n) {
        grow = n_new[tid];
        len = pg.lens[tid];
        held = pg.held[tid];
        const bool sane = len >= 0 && held >= 0 && held <= pg.max_pages && pages_of(len, pg.ps) <= held;
        if (grow > 0 && sane) {
            const long long want = ((long long)len + grow + pg.ps - 1) / pg.ps;
            fresh = want > held ? (int)min(want - held, (long long)pg.max_pages + 1) : 0;
            if (want > pg.max_pages) grow = -1;
            if (len % pg.ps) page = pg.table[(size_t)tid * pg.max_pages + len / pg.ps];
            if (page >= pg.pages || (len % pg.ps && page < 0)) grow = -1;
        } else if (!sane) {
            grow = -1;
        }
        tail[tid] = grow > 0 ? page : -1;
        held0[tid] = held;
    }
    auto free_page = [&](int e) { return pg.free_pages[top - 1 - e]; };
    avail[tid] = stack_ok && tid < top ? free_page(tid) : -1;
    __syncthreads();
    if (grow < 0) bad = 1;
    bool copy = false;
    if (grow > 0 && page >= 0) {
        int rank = 0;
        for (int b = 0; b < tid; ++b) rank += tail[b] == page;
        copy = pg.refs[page] - rank > 1;
    }
    int total;
    const int need = grow > 0 ? fresh + (copy ? 1 : 0) : 0;
    const int upto = block_scan(need, tmp, &total);
    if (tid < n) {
        first[tid + 1] = upto;
        copy_of[tid] = copy ? 1 : 0;
    }
    if (tid == 0) first[0] = 0;
    __syncthreads();
    auto taken = [&](int e) { return e < kMetaThreads ? avail[e] : free_page(e); };
    // (a total past 2^31 would need more columns than tables have)
    uint32_t err = !stack_ok ? DFLARE_DEVERR_PAGE : bad || total > top || total < 0 ? DFLARE_DEVERR_CAPACITY : 0u;
    if (!err) {
        bool odd = false;
        for (int e = tid; e < total; e += kMetaThreads) {
            const int p = taken(e);
            odd |= p < 0 || p >= pg.pages;
        }
        if (__syncthreads_or(odd)) err = DFLARE_DEVERR_PAGE;
    }
    if (err) {
        if (tid == 0) {
            copies[0] = 0;
            atomicOr(pg.err, err);
        }
        return;
    }
    int n_copies;
    const int c = block_scan(copy ? 1 : 0, tmp, &n_copies) - 1;
    for (int e = tid; e < total; e += kMetaThreads) {
        const int b = entry_owner(first, n, e);
        const int i = e - first[b] - copy_of[b];       // -1: the copy of the tail page
        const int p = taken(e);
        if (i >= 0) {
            pg.table[(size_t)b * pg.max_pages + held0[b] + i] = p;
            pg.refs[p] = 1;
        }
    }
    if (copy) {
        const int p = taken(first[tid]);
        pg.table[(size_t)tid * pg.max_pages + len / pg.ps] = p;
        pg.refs[p] = 1;
        atomicSub(&pg.refs[page], 1);
        copies[1 + 3 * c] = page;
        copies[2 + 3 * c] = p;
        copies[3 + 3 * c] = len % pg.ps;
    }
    if (tid < n && grow > 0) pg.held[tid] = held + fresh;
    if (tid == 0) {
        copies[0] = n_copies;
        *pg.n_free = top - total;
    }
}

// One CTA per pair: the table row, the counts, and a reference more for every page.
__global__ void __launch_bounds__(128) fork_kernel(const PagesView pg, const int32_t* __restrict__ src,
                                                   const int32_t* __restrict__ dst, int n) {
    __shared__ int clash;
    const int i = blockIdx.x, tid = threadIdx.x;
    if (tid == 0) clash = 0;
    pdl_wait();
    pdl_trigger();
    __syncthreads();
    const int a = src[i], b = dst[i];
    const bool range = a >= 0 && a < pg.max_batch && b >= 0 && b < pg.max_batch;
    bool hit = false;
    for (int j = tid; j < n; j += 128) hit |= dst[j] == a || (j != i && dst[j] == b);
    if (hit) clash = 1;
    __syncthreads();
    const int len = range ? pg.lens[a] : 0, have = range ? pg.held[a] : 0;
    const int keep = pages_of(max(len, 0), pg.ps);
    if (!range || clash || pg.held[b] != 0 || len < 0 || keep > have || keep > pg.max_pages) {
        if (tid == 0) atomicOr(pg.err, DFLARE_DEVERR_PAGE);
        return;
    }
    for (int j = tid; j < keep; j += 128) {
        const int p = pg.table[(size_t)a * pg.max_pages + j];
        pg.table[(size_t)b * pg.max_pages + j] = p;
        if (p >= 0 && p < pg.pages) atomicAdd(&pg.refs[p], 1);
        else atomicOr(pg.err, DFLARE_DEVERR_PAGE);
    }
    __syncthreads();
    if (tid == 0) {
        pg.held[b] = keep;
        pg.lens[b] = len;
    }
}

// Pages copied over all layers and both pools. list != NULL: the pairs and token counts that a reserve left
// behind; else src / dst, whole pages. A work item is one (pair, layer, pool): `hkv` runs of tokens x hd
// elements, which are one run when the whole page moves. HBM-bound: partial pages of 24 forks over 36 layers, 76 MB
// written from 25 MB of sources (three forks read one page, from L2 after the first), 19 us, 5.3 TB/s.
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const PagesView pg, const int32_t* __restrict__ list,
                                                            const int32_t* __restrict__ src,
                                                            const int32_t* __restrict__ dst, int n, int row_units) {
    pdl_wait();
    pdl_trigger();
    const int pairs = list ? list[0] : n;
    const long long items = (long long)pairs * pg.layers * 2;
    const size_t page_units = (size_t)pg.hkv * pg.ps * row_units;     // of 16 bytes
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int pair = (int)(it / (2 * pg.layers)), rest = (int)(it % (2 * pg.layers));
        const int a = list ? list[1 + 3 * pair] : src[pair], b = list ? list[2 + 3 * pair] : dst[pair];
        const int tokens = list ? list[3 + 3 * pair] : pg.ps;
        if (a < 0 || a >= pg.pages || b < 0 || b >= pg.pages) {
            if (threadIdx.x == 0) atomicOr(pg.err, DFLARE_DEVERR_PAGE);
            continue;
        }
        uint4* pool = static_cast<uint4*>((rest & 1) ? pg.v : pg.k) + (size_t)(rest >> 1) * pg.pages * page_units;
        const uint4* from = pool + (size_t)a * page_units;
        uint4* to = pool + (size_t)b * page_units;
        const int run = tokens * row_units, stride = pg.ps * row_units, units = pg.hkv * run;
        for (int u0 = threadIdx.x; u0 < units; u0 += 4 * kCopyThreads) {
            uint4 x[4];
            int at[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int u = u0 + j * kCopyThreads;
                at[j] = u < units ? (run == stride ? u : u / run * stride + u % run) : -1;
                if (at[j] >= 0) x[j] = __ldcs(from + at[j]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (at[j] >= 0) to[at[j]] = x[j];
        }
    }
}

// The accepted path's rows move from slots len + path[j] to len + j. A thread owns 16 bytes of one (layer,
// pool, head) and takes the moves in order, eight loads before their eight stores: path[j] >= j and the
// path increases, so a store never hits a slot that a later move still reads. Half latency, half HBM: 16 paths of
// 64-node trees over 36 layers, 38 MB, 7.5 us.
__global__ void __launch_bounds__(kCopyThreads) move_kernel(const PagesView pg, const int32_t* __restrict__ accept,
                                                            const int32_t* __restrict__ path, int path_row,
                                                            int row_units) {
    __shared__ long long move_from[kMaxNodes], move_to[kMaxNodes];   // where head 0's row lies in a layer, in units of 16 bytes
    __shared__ int n_moves;
    pdl_wait();
    pdl_trigger();
    const int b = blockIdx.y, tid = threadIdx.x;
    path += (size_t)b * path_row;
    const int first = tid < path_row && tid < 32 ? path[tid] : 0;     // under way together with the lengths
    const int len = pg.lens[b], a = accept[b], held = pg.held[b];
    if (tid < 32) {
        int count = 0;
        const int32_t* row = pg.table + (size_t)b * pg.max_pages;
        // the pages of the first 32 moves, wherever the path would read the table's row at all
        auto in_row = [&](int x) { return x >= 0 && len >= 0 && ((unsigned)len + (unsigned)x) / (unsigned)pg.ps < (unsigned)pg.max_pages; };
        const int pa0 = tid < a && in_row(first) ? row[(len + first) / pg.ps] : -1, pb0 = tid < a && in_row(tid) ? row[(len + tid) / pg.ps] : -1;
        if (path_fits(pg, b, path, a, path_row, len, held)) {
            for (int j0 = 0; j0 < a; j0 += 32) {
                const int j = j0 + tid;
                const int x = j >= a ? j : j0 ? path[j] : first;
                bool moves = x != j;
                int pa = 0, pb = 0;
                if (moves) {
                    pa = j0 ? row[(len + x) / pg.ps] : pa0;
                    pb = j0 ? row[(len + j) / pg.ps] : pb0;
                    if (pa < 0 || pa >= pg.pages || pb < 0 || pb >= pg.pages) {
                        atomicOr(pg.err, DFLARE_DEVERR_PAGE);
                        moves = false;
                    }
                }
                const unsigned votes = __ballot_sync(0xffffffffu, moves);
                if (moves) {
                    const int at = count + __popc(votes & ((1u << tid) - 1u));
                    move_from[at] = ((long long)pa * pg.hkv * pg.ps + (len + x) % pg.ps) * row_units;
                    move_to[at] = ((long long)pb * pg.hkv * pg.ps + (len + j) % pg.ps) * row_units;
                }
                count += __popc(votes);
            }
        }
        if (tid == 0) n_moves = count;
    }
    __syncthreads();
    const int n = n_moves;
    const int per_layer = 2 * pg.hkv * row_units;
    const long long u = (long long)blockIdx.x * kCopyThreads + tid;
    if (n == 0 || u >= (long long)per_layer * pg.layers) return;
    const int layer = (int)(u / per_layer), rest = (int)(u % per_layer);
    const int piece = rest % row_units, head = rest / row_units % pg.hkv;
    uint4* mine = static_cast<uint4*>(rest / row_units >= pg.hkv ? pg.v : pg.k) +
                  ((size_t)layer * pg.pages * pg.hkv + head) * pg.ps * row_units + piece;
    for (int j0 = 0; j0 < n; j0 += 8) {
        uint4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j0 + j < n) x[j] = mine[move_from[j0 + j]];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j0 + j < n) mine[move_to[j0 + j]] = x[j];
    }
}

dflare_status refuse(dflare_status st, const std::string& m) {
    noalloc_set_error(m);
    return st;
}
dflare_status done(cudaError_t e, const char* call) {
    if (e == cudaSuccess) return DFLARE_OK;
    return refuse(DFLARE_ECUDA, std::string(call) + ": " + cudaGetErrorString(e));
}

bool check_cache_config(const dflare_cache_config* g, std::string* why) {
    auto bad = [&](const char* m) {
        *why = std::string("invalid cache config: ") + m;
        return false;
    };
    if (!g) return bad("null");
    if (g->n_layers < 1 || g->n_layers > 256) return bad("n_layers must be in [1, 256]");
    if (g->n_pages < 1 || g->n_pages > (1 << 24)) return bad("n_pages must be in [1, 2^24]");
    if (g->page_size != 16 && g->page_size != 32 && g->page_size != 64 && g->page_size != 128)
        return bad("page_size must be 16, 32, 64 or 128");
    if (g->n_kv_heads < 1 || g->n_kv_heads > 128) return bad("n_kv_heads must be in [1, 128]");
    if (g->n_q_heads < 1 || g->n_q_heads % g->n_kv_heads != 0 || g->n_q_heads / g->n_kv_heads > kMaxGroup)
        return bad("n_q_heads must be a positive multiple of n_kv_heads, at most 64 times it");
    if (g->head_dim != 64 && g->head_dim != 128) return bad("head_dim must be 64 or 128");
    if (g->max_batch < 1 || g->max_batch > kMaxSeqs) return bad("max_batch must be in [1, 256]");
    if (g->max_pages < 1 || g->max_pages > (1 << 20)) return bad("max_pages must be in [1, 2^20]");
    if (g->max_nodes < 1 || g->max_nodes > kMaxNodes) return bad("max_nodes must be in [1, 1024]");
    if (g->dtype != DFLARE_BF16 && g->dtype != DFLARE_F32) return bad("dtype must be DFLARE_BF16 or DFLARE_F32");
    // numbers that kernels hold in 32 bits: token slots of a sequence and of the pool, boxes of the tensor
    // maps, and the attention's 32-key tiles over all sequences and heads (with the CTAs they are divided among: the
    // division rounds up, and the run of the last CTA may end that much later)
    if ((long long)g->max_pages * g->page_size > 0x7fffffffLL) return bad("max_pages * page_size must be below 2^31");
    if ((long long)g->n_pages * g->page_size > 0x7fffffffLL) return bad("n_pages * page_size must be below 2^31");
    if ((long long)g->n_layers * g->n_pages * g->n_kv_heads > 0x7fffffffLL)
        return bad("n_layers * n_pages * n_kv_heads must be below 2^31");
    if ((long long)g->max_batch * g->n_kv_heads * ((long long)g->max_pages * g->page_size / 32 + 1) > 0x7fffffffLL - 4096)
        return bad("max_batch * n_kv_heads * (max_pages * page_size / 32 + 1) must be below 2^31 - 4096");
    if ((long long)g->max_batch * g->max_pages > 0x7fffffffLL) return bad("max_batch * max_pages must be below 2^31");
    return true;
}

int row_units(const dflare_cache* c) { return (int)(c->cfg.head_dim * c->esz / 16); }

bool batch_ok(const dflare_cache* c, int batch) { return batch >= 1 && batch <= c->cfg.max_batch; }

}  // namespace
}  // namespace dfl

using namespace dfl;

extern "C" {

dflare_status dflare_cache_create(const dflare_cache_config* cfg, const dflare_cache_buffers* buffers, dflare_cache** out) {
    std::string why;
    if (!out) return refuse(DFLARE_EINVAL, "dflare_cache_create: out is NULL");
    *out = nullptr;
    if (!check_cache_config(cfg, &why)) return refuse(DFLARE_EINVAL, why);
    if (!buffers || !buffers->k || !buffers->v || !buffers->table || !buffers->lens || !buffers->held || !buffers->refs ||
        !buffers->free_pages || !buffers->n_free)
        return refuse(DFLARE_EINVAL, "dflare_cache_create: a buffer is NULL");
    if ((reinterpret_cast<uintptr_t>(buffers->k) | reinterpret_cast<uintptr_t>(buffers->v)) & 15u)
        return refuse(DFLARE_EINVAL, "dflare_cache_create: k and v must be 16-byte aligned");
    dflare_cache* c = new (std::nothrow) dflare_cache;
    if (!c) return refuse(DFLARE_ENOMEM, "dflare_cache_create: host memory");
    c->cfg = *cfg;
    c->esz = cfg->dtype == DFLARE_F32 ? 4 : 2;
    cudaError_t e = cudaGetDevice(&c->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&c->num_sms, cudaDevAttrMultiProcessorCount, c->device);
    auto give_up = [&](dflare_status st, const std::string& m) {
        dflare_cache_destroy(c);
        return refuse(st, m);
    };
    if (e != cudaSuccess) return give_up(DFLARE_ECUDA, std::string("dflare_cache_create: ") + cudaGetErrorString(e));
    c->part_rows = tree_partial_rows(*cfg, c->num_sms);
    if (cudaMalloc(&c->err, sizeof(uint32_t)) != cudaSuccess ||
        cudaMalloc(&c->last, (size_t)cfg->n_pages * sizeof(int32_t)) != cudaSuccess ||
        cudaMalloc(&c->copies, (1 + 3 * kMaxSeqs) * sizeof(int32_t)) != cudaSuccess ||
        cudaMalloc(&c->part_o, c->part_rows * cfg->head_dim * sizeof(float)) != cudaSuccess ||
        cudaMalloc(&c->part_ml, c->part_rows * sizeof(float2)) != cudaSuccess) {
        cudaGetLastError();
        return give_up(DFLARE_ENOMEM, "dflare_cache_create: device memory");
    }
    e = cudaMemset(c->err, 0, sizeof(uint32_t));
    if (e == cudaSuccess) e = cudaMemset(c->last, 0xff, (size_t)cfg->n_pages * sizeof(int32_t));
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return give_up(DFLARE_ECUDA, std::string("dflare_cache_create: ") + cudaGetErrorString(e));
    if (cfg->dtype == DFLARE_BF16) {
        // [layers * pages * kv heads][page size][head dim]; a copy takes up to 64 tokens of 64 head dims
        const uint64_t dims[3] = {(uint64_t)cfg->head_dim, (uint64_t)cfg->page_size,
                                  (uint64_t)cfg->n_layers * cfg->n_pages * cfg->n_kv_heads};
        const uint64_t strides[2] = {(uint64_t)cfg->head_dim * 2, (uint64_t)cfg->head_dim * 2 * cfg->page_size};
        const uint32_t box[3] = {64, (uint32_t)(cfg->page_size < 64 ? cfg->page_size : 64), 1};
        if (!encode_tma_bf16(&c->maps[0], buffers->k, 3, dims, strides, box) ||
            !encode_tma_bf16(&c->maps[1], buffers->v, 3, dims, strides, box))
            return give_up(DFLARE_ECUDA, "dflare_cache_create: tensor map");
    }
    c->view = PagesView{buffers->k, buffers->v, buffers->table, buffers->lens, buffers->held, buffers->refs, buffers->free_pages,
                        buffers->n_free, c->err, cfg->n_layers, cfg->n_pages, cfg->n_kv_heads, cfg->page_size, cfg->head_dim,
                        cfg->max_batch, cfg->max_pages};
    *out = c;
    return DFLARE_OK;
}

dflare_status dflare_cache_destroy(dflare_cache* c) {
    if (!c) return DFLARE_OK;
    DeviceGuard guard(c->device);
    cudaDeviceSynchronize();
    cudaFree(c->err);
    cudaFree(c->last);
    cudaFree(c->copies);
    cudaFree(c->part_o);
    cudaFree(c->part_ml);
    delete c;
    return DFLARE_OK;
}

dflare_status dflare_cache_error(dflare_cache* c, uint32_t* bits_host, void* stream) {
    if (!c || !bits_host) return refuse(DFLARE_EINVAL, "dflare_cache_error: NULL argument");
    DeviceGuard guard(c->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint32_t bits = 0;
    cudaError_t e = cudaMemcpyAsync(&bits, c->err, sizeof bits, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e == cudaSuccess && bits) {
        e = cudaMemsetAsync(c->err, 0, sizeof bits, s);
        if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    }
    if (e != cudaSuccess) return done(e, "dflare_cache_error");
    *bits_host = bits;
    return bits ? refuse(DFLARE_EDEVICE, "dflare_cache_error: a kernel reported an error") : DFLARE_OK;
}

dflare_status dflare_cache_reserve(dflare_cache* c, const int32_t* n_new_dev, int batch, void* stream) {
    if (!c || !n_new_dev) return refuse(DFLARE_EINVAL, "dflare_cache_reserve: NULL argument");
    if (!batch_ok(c, batch)) return refuse(DFLARE_EINVAL, "dflare_cache_reserve: batch must be in [1, max_batch]");
    DeviceGuard guard(c->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = launch_kernel(true, reserve_kernel, dim3(1), dim3(kMetaThreads), 0, s, c->view, n_new_dev, c->copies, batch);
    if (e == cudaSuccess) {
        const int grid = (int)std::min<long long>(2LL * c->cfg.n_layers * batch, 8LL * c->num_sms);
        e = launch_kernel(true, copy_kernel, dim3(grid), dim3(kCopyThreads), 0, s, c->view, c->copies, nullptr, nullptr, 0, row_units(c));
    }
    return done(e, "dflare_cache_reserve");
}

dflare_status dflare_cache_truncate(dflare_cache* c, const int32_t* new_len_dev, int batch, void* stream) {
    if (!c || !new_len_dev) return refuse(DFLARE_EINVAL, "dflare_cache_truncate: NULL argument");
    if (!batch_ok(c, batch)) return refuse(DFLARE_EINVAL, "dflare_cache_truncate: batch must be in [1, max_batch]");
    DeviceGuard guard(c->device);
    return done(launch_kernel(true, trim_kernel, dim3(1), dim3(kMetaThreads), 0, static_cast<cudaStream_t>(stream), c->view,
                              new_len_dev, nullptr, nullptr, 0, c->last, batch), "dflare_cache_truncate");
}

dflare_status dflare_cache_commit(dflare_cache* c, const int32_t* accept_len_dev, const int32_t* path_dev, int path_row,
                                  int batch, void* stream) {
    if (!c || !accept_len_dev || !path_dev) return refuse(DFLARE_EINVAL, "dflare_cache_commit: NULL argument");
    if (!batch_ok(c, batch)) return refuse(DFLARE_EINVAL, "dflare_cache_commit: batch must be in [1, max_batch]");
    if (path_row < 1 || path_row > kMaxNodes) return refuse(DFLARE_EINVAL, "dflare_cache_commit: path_row must be in [1, 1024]");
    DeviceGuard guard(c->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const long long units = 2LL * c->cfg.n_layers * c->cfg.n_kv_heads * row_units(c);
    const int blocks = (int)((units + kCopyThreads - 1) / kCopyThreads);
    cudaError_t e = launch_kernel(true, move_kernel, dim3(blocks, batch), dim3(kCopyThreads), 0, s, c->view, accept_len_dev,
                                  path_dev, path_row, row_units(c));
    if (e == cudaSuccess)
        e = launch_kernel(true, trim_kernel, dim3(1), dim3(kMetaThreads), 0, s, c->view, nullptr, accept_len_dev, path_dev,
                          path_row, c->last, batch);
    return done(e, "dflare_cache_commit");
}

dflare_status dflare_cache_fork(dflare_cache* c, const int32_t* src_dev, const int32_t* dst_dev, int n, void* stream) {
    if (!c || !src_dev || !dst_dev) return refuse(DFLARE_EINVAL, "dflare_cache_fork: NULL argument");
    if (!batch_ok(c, n)) return refuse(DFLARE_EINVAL, "dflare_cache_fork: n must be in [1, max_batch]");
    DeviceGuard guard(c->device);
    return done(launch_kernel(true, fork_kernel, dim3(n), dim3(128), 0, static_cast<cudaStream_t>(stream), c->view, src_dev,
                              dst_dev, n), "dflare_cache_fork");
}

dflare_status dflare_cache_copy_pages(dflare_cache* c, const int32_t* src_dev, const int32_t* dst_dev, int n, void* stream) {
    if (!c || !src_dev || !dst_dev) return refuse(DFLARE_EINVAL, "dflare_cache_copy_pages: NULL argument");
    if (n < 1 || n > c->cfg.n_pages) return refuse(DFLARE_EINVAL, "dflare_cache_copy_pages: n must be in [1, n_pages]");
    DeviceGuard guard(c->device);
    const int grid = (int)std::min<long long>(2LL * c->cfg.n_layers * n, 8LL * c->num_sms);
    return done(launch_kernel(true, copy_kernel, dim3(grid), dim3(kCopyThreads), 0, static_cast<cudaStream_t>(stream), c->view,
                              nullptr, src_dev, dst_dev, n, row_units(c)), "dflare_cache_copy_pages");
}

}  // extern "C"
