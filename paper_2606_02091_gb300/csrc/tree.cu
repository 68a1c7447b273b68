// Drafted trees: ancestor bits and depths from parent numbers, and greedy acceptance. Both calls are a few
// hundred bytes to a few hundred kilobytes of integers: bound by latency.
#include <algorithm>
#include <string>

#include "common.cuh"
#include "paged.h"

namespace dfl {
namespace {

constexpr int kTreeThreads = 256;

// The parents of one tree in shared memory, -1 where a parent is impossible; *bad set if one was.
__device__ __forceinline__ void load_parents(const int32_t* __restrict__ parents, int n, int32_t* up, bool* bad) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        int p = parents[i];
        if (i == 0 ? p != -1 : (p < -1 || p >= i)) {
            *bad = true;
            p = -1;
        }
        up[i] = p;
    }
}

// One CTA per tree, rows of ancestor bits in shared memory, a thread per node (two above 512). Every node starts with
// itself and looks one node up; each round it takes over the bits of the node it looks at (whose words end at that
// node's own) and then looks where that one looks, so a branch of depth d is done in log2(d) rounds. Rows are taken
// over while others write theirs: what is read early or late are ancestors of an ancestor either way. Rows go out as
// whole lines. Measured for 64 trees of 255 nodes: walking up edge by edge 11 us (37 for chains).
constexpr int kPlanThreads = 512, kPlanNodes = kMaxNodes / kPlanThreads;

__global__ void __launch_bounds__(kPlanThreads) tree_plan_kernel(const int32_t* __restrict__ parents,
                                                                 const int32_t* __restrict__ n_nodes, int n_max,
                                                                 int words, uint32_t* __restrict__ mask,
                                                                 int32_t* __restrict__ depth, uint32_t* err) {
    extern __shared__ uint32_t rows[];          // [n_max][words | 1]: an odd stride spreads the rows over the banks
    __shared__ int32_t up[kMaxNodes];           // the node looked at, -1: above the top
    __shared__ int16_t edges[kMaxNodes];        // edges up to there; at the end up to the top, plus one
    pdl_wait();
    pdl_trigger();
    const int b = blockIdx.x, tid = threadIdx.x, stride = words | 1;
    const int told = n_nodes[b], n = min(max(told, 0), n_max);
    bool bad = told != n;
    load_parents(parents + (size_t)b * n_max, n, up, &bad);
    if (bad && err) atomicOr(err, DFLARE_DEVERR_TREE);
    for (int i = tid; i < n_max; i += blockDim.x) {
        for (int w = 0; w < words; ++w) rows[i * stride + w] = i < n && (i >> 5) == w ? 1u << (i & 31) : 0u;
        edges[i] = 1;
    }
    bool more = n > 0;
    while (__syncthreads_or(more)) {
        int to[kPlanNodes], len[kPlanNodes];
        more = false;
#pragma unroll
        for (int k = 0; k < kPlanNodes; ++k) {
            const int i = tid + k * kPlanThreads, u = i < n ? up[i] : -1;
            to[k] = -1;
            len[k] = 0;
            if (u < 0) continue;
            uint32_t* mine = rows + i * stride;
            const uint32_t* theirs = rows + u * stride;
#pragma unroll 4
            for (int w = 0; w <= u >> 5; ++w) mine[w] |= theirs[w];
            to[k] = up[u];
            len[k] = edges[i] + edges[u];
            more |= to[k] >= 0;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPlanNodes; ++k) {
            const int i = tid + k * kPlanThreads;
            if (len[k]) {
                edges[i] = (int16_t)len[k];
                up[i] = to[k];
            }
        }
    }
    for (int x = tid; x < n_max * words; x += blockDim.x) {
        const int i = x / words;
        mask[(size_t)b * n_max * words + x] = rows[i * stride + x - i * words];
    }
    for (int i = tid; i < n_max; i += blockDim.x) depth[(size_t)b * n_max + i] = i < n ? edges[i] - 1 : 0;
}

// One CTA per tree. All nodes at once: whether the node's token is what the target chose after its parent,
// and the lowest such child of every node. The walk from the root then reads one number per step.
__global__ void __launch_bounds__(kTreeThreads) tree_accept_kernel(
    const int32_t* __restrict__ tokens, const int32_t* __restrict__ parents, const int32_t* __restrict__ choice,
    const int32_t* __restrict__ n_nodes, int n_max, int32_t* __restrict__ accept_len, int32_t* __restrict__ path,
    int32_t* __restrict__ next_token, uint32_t* err) {
    __shared__ int32_t up[kMaxNodes], child[kMaxNodes], walk[kMaxNodes];
    __shared__ int steps;
    pdl_wait();
    pdl_trigger();
    const int b = blockIdx.x, tid = threadIdx.x;
    const int told = n_nodes[b], n = min(max(told, 0), n_max);
    const int32_t* tok = tokens + (size_t)b * n_max;
    const int32_t* pick = choice + (size_t)b * n_max;
    bool bad = told != n;
    load_parents(parents + (size_t)b * n_max, n, up, &bad);
    for (int i = tid; i < n; i += kTreeThreads) child[i] = n;
    if (bad && err) atomicOr(err, DFLARE_DEVERR_TREE);
    __syncthreads();
    for (int i = tid; i < n; i += kTreeThreads) {
        const int p = up[i];
        if (p >= 0 && tok[i] == pick[p]) atomicMin(&child[p], i);
    }
    __syncthreads();
    if (tid == 0) {
        int a = 0;
        for (int at = 0; at < n; at = child[at]) walk[a++] = at;
        steps = a;
        accept_len[b] = a;
        next_token[b] = a ? pick[walk[a - 1]] : -1;
    }
    __syncthreads();
    for (int i = tid; i < n_max; i += kTreeThreads) path[(size_t)b * n_max + i] = i < steps ? walk[i] : -1;
}

dflare_status refuse(dflare_status st, const std::string& m) {
    noalloc_set_error(m);
    return st;
}

}  // namespace
}  // namespace dfl

using namespace dfl;

extern "C" {

dflare_status dflare_tree_plan(const int32_t* parents_dev, const int32_t* n_nodes_dev, int batch, int n_max,
                               int32_t* mask_dev, int32_t* depth_dev, uint32_t* err_dev, void* stream) {
    if (!parents_dev || !n_nodes_dev || !mask_dev || !depth_dev)
        return refuse(DFLARE_EINVAL, "dflare_tree_plan: NULL argument");
    if (batch < 1 || batch > 65535 || n_max < 1 || n_max > kMaxNodes)
        return refuse(DFLARE_EINVAL, "dflare_tree_plan: batch must be in [1, 65535], n_max in [1, 1024]");
    static PerDeviceOnce once;
    const int words = (n_max + 31) / 32;
    cudaError_t e = once([] {
        return cudaFuncSetAttribute(tree_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxNodes * (kMaxNodes / 32 + 1) * 4);
    });
    if (e == cudaSuccess)
        e = launch_kernel(true, tree_plan_kernel, dim3(batch), dim3(std::min(kPlanThreads, (n_max + 31) / 32 * 32)), (size_t)n_max * (words | 1) * 4, static_cast<cudaStream_t>(stream),
                          parents_dev, n_nodes_dev, n_max, words, reinterpret_cast<uint32_t*>(mask_dev), depth_dev, err_dev);
    return e == cudaSuccess ? DFLARE_OK : refuse(DFLARE_ECUDA, std::string("dflare_tree_plan: ") + cudaGetErrorString(e));
}

dflare_status dflare_tree_accept(const int32_t* tokens_dev, const int32_t* parents_dev, const int32_t* choice_dev,
                                 const int32_t* n_nodes_dev, int batch, int n_max, int32_t* accept_len_dev,
                                 int32_t* path_dev, int32_t* next_token_dev, uint32_t* err_dev, void* stream) {
    if (!tokens_dev || !parents_dev || !choice_dev || !n_nodes_dev || !accept_len_dev || !path_dev || !next_token_dev)
        return refuse(DFLARE_EINVAL, "dflare_tree_accept: NULL argument");
    if (batch < 1 || batch > 65535 || n_max < 1 || n_max > kMaxNodes)
        return refuse(DFLARE_EINVAL, "dflare_tree_accept: batch must be in [1, 65535], n_max in [1, 1024]");
    const cudaError_t e = launch_kernel(true, tree_accept_kernel, dim3(batch), dim3(kTreeThreads), 0, static_cast<cudaStream_t>(stream),
                                        tokens_dev, parents_dev, choice_dev, n_nodes_dev, n_max, accept_len_dev, path_dev,
                                        next_token_dev, err_dev);
    return e == cudaSuccess ? DFLARE_OK : refuse(DFLARE_ECUDA, std::string("dflare_tree_accept: ") + cudaGetErrorString(e));
}

}  // extern "C"
