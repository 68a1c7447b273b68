// Drafted trees: ancestor bits and depths from parent numbers, and greedy acceptance. Both calls are a few
// hundred bytes to a few hundred kilobytes of integers: bound by the latency of a walk up (or down) a branch.
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

// One CTA per tree, a thread per node (and per further node 256 on). A node's ancestors come up in
// decreasing order, so its mask row is finished word by word from the last word down and needs no storage.
__global__ void __launch_bounds__(kTreeThreads) tree_plan_kernel(const int32_t* __restrict__ parents,
                                                                 const int32_t* __restrict__ n_nodes, int n_max,
                                                                 int words, uint32_t* __restrict__ mask,
                                                                 int32_t* __restrict__ depth, uint32_t* err) {
    __shared__ int32_t up[kMaxNodes];
    pdl_wait();
    const int b = blockIdx.x;
    const int told = n_nodes[b], n = min(max(told, 0), n_max);
    bool bad = told != n;
    load_parents(parents + (size_t)b * n_max, n, up, &bad);
    if (bad && err) atomicOr(err, DFLARE_DEVERR_TREE);
    __syncthreads();
    for (int i = threadIdx.x; i < n_max; i += kTreeThreads) {
        uint32_t* row = mask + ((size_t)b * n_max + i) * words;
        int w = words - 1, edges = -1;
        uint32_t bits = 0;
        for (int j = i < n ? i : -1; j >= 0; j = up[j]) {
            while (w > (j >> 5)) {
                row[w--] = bits;
                bits = 0;
            }
            bits |= 1u << (j & 31);
            ++edges;
        }
        while (w >= 0) {
            row[w--] = bits;
            bits = 0;
        }
        depth[(size_t)b * n_max + i] = max(edges, 0);
    }
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
    const cudaError_t e = launch_kernel(true, tree_plan_kernel, dim3(batch), dim3(kTreeThreads), 0, static_cast<cudaStream_t>(stream),
                                        parents_dev, n_nodes_dev, n_max, (n_max + 31) / 32,
                                        reinterpret_cast<uint32_t*>(mask_dev), depth_dev, err_dev);
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
