// Launch interface between the executor (stack.hip) and the operators of drafted tokens (drafts.hip), where these run inside a
// stack's forward: one sequence, fp16, heads of 128, tables by value instead of in device memory.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "ps_internal.h"

namespace ps {

// The nodes of a tree as they travel in a launch's arguments, a byte each: parents + 1 (0: none), and how many ancestors a
// node has (its position is that many behind the context)
struct TreeBytes { uint32_t w[PS_TREE_MAX / 4]; };
struct StackTreeNodes {
    uint32_t n;              // 0: no tree, tokens follow one another
    TreeBytes up, depth;
};
// host parents -> nodes; false (with an error text) where they are no tree
bool make_tree_nodes(const int32_t *parent, uint32_t n, StackTreeNodes *out);

// What every forward does to the queries and keys of its QKV rows in front of the attention
struct StackRotation {
    const float *inv_freq;           // [rot_dim / 2]
    const __half *q_gain, *k_gain;   // [layer][128] or null
    uint32_t rot_dim, pairs, norm;
    float eps;
};
// rows of a QKV buffer (queries, keys, values), in place; token t stands at position ctx (ctx_dev, if not null, has it) + t, or
// + its depth in the tree
hipError_t launch_stack_rotation(const StackRotation &r, uint32_t layer, __half *qkv, uint32_t qkv_w, uint32_t n_q, uint32_t n_kv, uint32_t n_tokens,
                                 uint32_t ctx, const uint32_t *ctx_dev, const StackTreeNodes &tree, hipStream_t st);

// Attention of a tree over a run of kv heads' cache shards (head0 .. head0 + nheads - 1, k_base the first one's K rows, shards
// head_stride bytes apart, K rows [cap][128] then V rows).  Queries, keys and values in place in the QKV rows; the tokens' rows
// are appended at home[kv head] (null: not).  splits: from stack_tree_splits; more than one: records for launch_stack_tree_merge.
struct StackTreeArgs {
    const __half *k_base;
    uint64_t head_stride;
    uint32_t cap, ctx, head0, nheads, n_q, n_kv, splits;
    const __half *qkv;
    uint32_t qkv_w;
    __half *out;             // [tokens][n_q * 128]
    float *part;
    const uint64_t *home;
};
// a function of the whole model's heads, the context and the tree, so that a result does not depend on where a shard lies
uint32_t stack_tree_splits(uint32_t n_q, uint32_t n_kv, uint32_t ctx, uint32_t n_tokens, uint64_t part_bytes);
hipError_t launch_stack_tree(const StackTreeArgs &a, const StackTreeNodes &tree, hipStream_t st);
hipError_t launch_stack_tree_merge(const StackTreeArgs &a, uint32_t n_tokens, hipStream_t st);

// first (0, n) and the parents of a tree (or of a chain of n), as device tables
hipError_t launch_tree_tables(int32_t *first, int32_t *parent, uint32_t n, const StackTreeNodes &tree, hipStream_t st);
// rows ctx + path[i] -> ctx + i of every home's K and V rows [cap][128]
hipError_t launch_stack_keep(const uint64_t *home, uint32_t n_homes, uint32_t cap, uint32_t ctx, uint32_t width, const int32_t *path, const int32_t *count,
                             hipStream_t st);

}  // namespace ps
