// Device helpers for private continuations in pages, shared by the kernels that read and write them.
#pragma once
#include "polykv_internal.hpp"

namespace polykv {

// The pages as the kernels see them; passed by value.
struct PageView {
    uint16_t *K, *V;           // [layers, pages, H, P, D]
    int32_t *table, *lengths;  // [A, max_blocks], [A]
    int D, H, A, pages, P, max_blocks;
    FastDiv div_P;
};

inline PageView page_view(const polykv_pages* p) {
    return PageView{(uint16_t*)p->K_dev, (uint16_t*)p->V_dev, p->table_dev, p->lengths_dev, p->head_dim, p->kv_heads,
                    p->agents,           p->pages,            p->page_tokens, p->max_blocks, FastDiv::by(p->page_tokens)};
}

// Tokens in agent a's pages, and how many of them are its drafts.
__device__ __forceinline__ int tokens_of(const PageView& v, int a) { return min(max(v.lengths[a], 0), v.max_blocks * v.P); }
__device__ __forceinline__ int drafts_of(const int32_t* counts, int a, int nodes, int length) {
    const int n = min(nodes, length);
    return counts != nullptr ? min(max(counts[a], 0), n) : n;
}
// Row (vector of one head, from the layer's first) of head h at offset `off` of page `page`.
__device__ __forceinline__ int page_row(const PageView& v, int page, int h, int off) { return (page * v.H + h) * v.P + off; }

hipError_t launch_pages_resize(const polykv_pages* p, const int32_t* targets, int32_t* slots, int n_slots, int32_t* offsets,
                               hipStream_t s);
hipError_t launch_pages_resize_by_agent(const polykv_pages* p, const int32_t* targets, int32_t* slots, int per_agent, int32_t* granted,
                                        hipStream_t s);
hipError_t launch_pages_write(const polykv_pages* p, const void* K, const void* V, int in_dtype, int tokens, int64_t layer_stride,
                              int64_t token_stride, int64_t head_stride, const int32_t* slots, int layer_begin, int layer_end,
                              hipStream_t s);
hipError_t launch_tree_masks(const int32_t* parents, const int32_t* counts, int agents, int nodes, uint64_t* mask, int32_t* depth,
                             hipStream_t s);
hipError_t launch_pages_accept(const polykv_pages* p, const int32_t* tokens, const int32_t* following, const int32_t* parents,
                               const int32_t* counts, int nodes, int32_t* path, int32_t* accepted, int32_t* next, int32_t* kept,
                               hipStream_t s);

// What pool_attend_tree needs beside the plan of the pool's part.
struct TreePlan {
    const int32_t* counts;
    const uint64_t* mask;
    int words;                 // 64-bit words of a draft's mask
    int layer_begin, layers, nodes, q_heads, G, rows;   // rows = nodes * G of an agent and KV head
    float qscale;
    int nsplit;                // token-range splits of the pages' part
    int merge;                 // 1: the pages' kernel writes partials for the merge kernel, 0: the output
    int wave_rows;             // rows of a wave: 32, or 16 (waves == 1)
    int waves;                 // waves with rows of their own in a workgroup: 1, 2 or 4
    int share;                 // 1 (waves == 1): four waves share the rows
    int row_blocks;            // blocks of rows of an agent and KV head
    FastDiv div_H, div_A, div_G, div_nsplit, div_row_blocks;
    size_t off_ml, off_o, total;   // the pages' partials in the workspace (behind the pool's)
};
// Fills in the splits and the row blocks.
void plan_tree(const PageView& v, int pool_splits, int page_splits, TreePlan* t);   // pool_splits: 0 without a pool
// The pool's partials, to be joined with the pages': [units][nsplit][agents * rows].
struct PoolPart {
    const float *ml, *o;   // nullptr: there is no pool
    int nsplit, rotated;   // rotated: the value sums are in the rotated domain
    SignBits signs;
};
// The pages' part: partials (out == nullptr), or the output, which takes the pool's partials in.
hipError_t launch_attend_pages(const PageView& v, const TreePlan& t, bool bf16, const void* Q, float* ml, float* o, void* out,
                               const PoolPart& pool, hipStream_t s);
// Joins the pool's partials (has_pool) and the pages' and writes the output.
hipError_t launch_tree_merge(const AttendPlan& plan, const TreePlan& t, bool has_pool, const float* pool_ml, const float* pool_o,
                             const float* ml, const float* o, void* out, hipStream_t s);

}  // namespace polykv
