// Host-side internals of the paged cache: its handle and the launchers of its attention.
#pragma once
#include "internal.h"

namespace dfl {

constexpr int kMaxSeqs = 256;        // sequences of a paged cache
constexpr int kMaxNodes = 1024;      // nodes of a tree, rows of a chunk
constexpr int kMaxGroup = 64;        // query heads per kv head of the paged attention

// What the kernels see of a cache (passed by value).
struct PagesView {
    void* k;             // [layers][pages][kv heads][page size][head dim]
    void* v;
    int32_t* table;      // [max_batch][max_pages]
    int32_t* lens;
    int32_t* held;
    int32_t* refs;
    int32_t* free_pages;
    int32_t* n_free;
    uint32_t* err;
    int layers, pages, hkv, ps, hd, max_batch, max_pages;
};

}  // namespace dfl

struct dflare_cache {
    dflare_cache_config cfg;
    dfl::PagesView view{};
    int device = 0;
    int num_sms = 0;
    size_t esz = 2;
    uint32_t* err = nullptr;
    int32_t* last = nullptr;       // [pages] scratch of the page counts: -1 between calls
    int32_t* copies = nullptr;     // [1 + 3 * kMaxSeqs]: count, then (source page, page, tokens) of a reserve
    float* part_o = nullptr;       // attention: partial outputs of rows whose keys several CTAs read
    float2* part_ml = nullptr;     // their (maximum in log2 units, sum)
    size_t part_rows = 0;          // rows of part_o
    CUtensorMap maps[2];           // K and V pools (bf16)
};

namespace dfl {

// one launch of the paged attention
struct TreeArgs {
    PagesView pg;
    const void* q;             // [batch][n_max][hq][hd], q_row elements between rows
    long long q_row;
    const int32_t* mask;       // [batch][n_max][words], or null: node j <= i
    const int32_t* n_nodes;
    void* out;                 // [batch][n_max][hq][hd]
    float* lse;                // [batch][n_max][hq], optional
    float* part_o;
    float2* part_ml;
    int layer, batch, n_max, words, hq, G;   // G: query heads per kv head
    uint32_t G_inv;            // 2^32 / G, rounded up (G > 1)
    int QG, C;                 // groups of query rows, and CTAs that share the work (more are launched for more groups)
    float scale_log2;
};

// The tcgen05 kernel's keys per tile, and how its work is divided (see tree_sched.cuh). Measured with 1, 2, 3 and 4 extra
// tiles a pair: 33 nodes at head_dim 64 over 2 x 8192 keys 27.5, 29.3, 27.9 and 29.0 us, 16 nodes over four contexts 21.1, 19.5,
// 19.5 and 19.8, over eight up to 900 keys 16.5, 14.2, 14.8 and 14.8, 90 over three up to 3000 keys 29.8, 27.9, 26.5 and 28.1;
// with runs of at least 1 and 3: 171 nodes over two contexts of 142 and 96 keys 13.1 and 17.4.
constexpr int kTcKeys = 128, kTcExtra = 3, kTcLeast = 1;

cudaError_t launch_tree_attention(dflare_cache* c, TreeArgs a, cudaStream_t s);
// tcgen05 kernel for many query rows per kv head (bf16); sets a.QG, a.C and the rows of a query group
cudaError_t launch_tree_attention_tc(dflare_cache* c, TreeArgs& a, int* QT, cudaStream_t s);
// rows of the partial buffers that any launch of a cache may use
size_t tree_partial_rows(const dflare_cache_config& g, int num_sms);

}  // namespace dfl
