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

// Attention over shared pages (tree_shared.cu): one CTA's part of one unit of work, which is a block of query rows of one kv
// head against a sequence's own keys, or a group's rows against the keys that the group shares.
struct __align__(16) TreeItem {
    int b;               // the table's row
    int h;               // kv head
    int lo, hi;          // key tiles [lo, hi) of the unit's
    int page0, held;     // the first page of the unit's keys in the table's row, and how many count from there
    int ctx, keys;       // of them: tokens, and tokens and nodes (the same number for a group's)
    int nodes;           // whose rows these are: node i's query row is first + i, or map[~first + i] of a group
    int first;
    int row0;            // the block's first row
    int dst;             // its first row among the partial results, or -1: the result itself
};
// What the joining launch has to know of a sequence.
struct __align__(16) TreeSeq {
    int n;               // nodes
    int start, tiles, blocks;                   // own units: the first one's place in the list, tiles of each, blocks of rows
    int lead_start, lead_tiles, lead_blocks;    // its group's (tiles 0: none)
    int node0;           // its first node among the group's
    int row, lead_row;   // rows of whole units among the partial results: of kv head 0 (lead_row: of the group's row 0)
    int weight, lead_weight;    // cost of a tile
};
// The type and head_dim of a plan's cache, on which its lists of work and the places of everything in the workspace depend; never 0.
inline int plan_kind(const dflare_cache_config& g) { return 1 | (int)g.dtype << 1 | g.head_dim << 2; }
// The head of an attend_shared workspace.
struct __align__(16) SharedHead {
    int kind, batch, n_max, max_pages, hkv, ps, G;      // what the plan was made for (kind: plan_kind)
    int per[2];                                         // length of a CTA's run in each list of work
};
// One kernel's list of work: log2 of its rows per block and keys per tile, its CTAs, what a tile of up to 128 rows and one of more costs, and
// a unit beside its tiles, the shortest run, and the first of its CTAs' rows among the partial results.
struct WorkList {
    int qt, kt, C, weight1, weight2, extra, least, slot0;
    bool blocks;         // its rows lie in blocks of 32 rows x 32 elements
};

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
    // attend_shared
    const SharedHead* head;
    int kind;                  // of the plan that it must hold
    const int2* runs;          // [C]: the first and the last item of a CTA, plus one
    const TreeItem* items;
    const int32_t* map;        // query rows of the groups' nodes
    const TreeSeq* seqs;
    int own_rows, lead_rows;   // rows among the partial results between kv heads
    bool follows;              // the kernel before this one is of the same call, and does not write what this one reads
};

// The tcgen05 kernel's keys per tile, and how its work is divided (see tree_sched.cuh). Measured with 1, 2, 3 and 4 extra
// tiles a pair: 33 nodes at head_dim 64 over 2 x 8192 keys 27.5, 29.3, 27.9 and 29.0 us, 16 nodes over four contexts 21.1, 19.5,
// 19.5 and 19.8, over eight up to 900 keys 16.5, 14.2, 14.8 and 14.8, 90 over three up to 3000 keys 29.8, 27.9, 26.5 and 28.1;
// with runs of at least 1 and 3: 171 nodes over two contexts of 142 and 96 keys 13.1 and 17.4.
constexpr int kTcKeys = 128, kTcExtra = 3, kTcLeast = 1;

// The fp32 kernel's: a tile takes as long as beginning and ending a pair: 13.0 us with 2 and 3, three contexts up to 600.
constexpr int kFKeys = 32, kFRows = 16, kFExtra = 0, kFLeast = 1;

cudaError_t launch_tree_attention(dflare_cache* c, TreeArgs a, cudaStream_t s);
// tcgen05 kernel for many query rows per kv head (bf16); sets a.QG, a.C and the rows of a query group
cudaError_t launch_tree_attention_tc(dflare_cache* c, TreeArgs& a, int* QT, cudaStream_t s);
// The warp-level bf16 kernel's.
constexpr int kMmaKeys = 64, kMmaRows = 16, kMmaExtra = 3;
constexpr int mma_least(int head_dim) { return 256 / head_dim; }
// the same kernels over a plan's items, with 256 (tcgen05), kMmaRows (warp level) or kFRows (fp32) rows in a block
cudaError_t launch_shared_mma(dflare_cache* c, const TreeArgs& a, cudaStream_t s);
cudaError_t launch_shared_tc(dflare_cache* c, const TreeArgs& a, cudaStream_t s);
cudaError_t launch_shared_f32(dflare_cache* c, const TreeArgs& a, cudaStream_t s);
int f32_ctas_per_sm(int head_dim);
// rows of the partial buffers that any launch of a cache may use
size_t tree_partial_rows(const dflare_cache_config& g, int num_sms);

}  // namespace dfl
