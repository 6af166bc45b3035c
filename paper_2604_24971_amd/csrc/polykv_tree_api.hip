// C ABI of libpolykv: continuations in pages and drafted tokens -- argument validation, planning, dispatch.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "polykv_pages.hpp"

namespace polykv {

static size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

static bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// What every call needs of the description; `tensors`: the call reads or writes K and V.
static int check_pages(const polykv_pages* p, bool tensors, const char* who) {
    if (p == nullptr) {
        set_error("%s: pages is NULL", who);
        return POLYKV_EINVAL;
    }
    if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) {
        set_error("%s: head_dim=%d not supported (64, 128 or 256)", who, p->head_dim);
        return POLYKV_ESHAPE;
    }
    if (p->layers < 1 || p->kv_heads < 1 || (long)p->layers * p->kv_heads > 65535) {
        set_error("%s: layers=%d kv_heads=%d must be >= 1 and layers*kv_heads <= 65535", who, p->layers, p->kv_heads);
        return POLYKV_ESHAPE;
    }
    if (p->page_tokens < 8 || p->page_tokens % 8 != 0 || p->pages < 1 || (int64_t)p->pages * p->page_tokens > (1 << 30) ||
        (int64_t)p->pages * p->page_tokens * p->kv_heads > 0x7FFFFFFF) {
        set_error("%s: %d pages of %d tokens x %d heads: page_tokens must be a multiple of 8, pages * page_tokens at most 2^30 and "
                  "pages * page_tokens * kv_heads less than 2^31", who, p->pages, p->page_tokens, p->kv_heads);
        return POLYKV_ESHAPE;
    }
    if (p->agents < 1 || p->agents > POLYKV_MAX_PAGED_AGENTS || p->max_blocks < 1 ||
        (int64_t)p->max_blocks * p->page_tokens > (1 << 30)) {
        set_error("%s: agents=%d must be in 1 .. %d, max_blocks=%d >= 1 and max_blocks * page_tokens at most 2^30", who, p->agents,
                  POLYKV_MAX_PAGED_AGENTS, p->max_blocks);
        return POLYKV_ESHAPE;
    }
    if (p->dtype != POLYKV_F16 && p->dtype != POLYKV_BF16) {
        set_error("%s: dtype %d is neither POLYKV_F16 nor POLYKV_BF16", who, p->dtype);
        return POLYKV_EINVAL;
    }
    if (p->table_dev == nullptr || p->lengths_dev == nullptr || !aligned(p->table_dev, 4) || !aligned(p->lengths_dev, 4)) {
        set_error("%s: table_dev and lengths_dev must be 4-byte aligned device pointers", who);
        return POLYKV_EINVAL;
    }
    if (tensors && (p->K_dev == nullptr || p->V_dev == nullptr || !aligned(p->K_dev, 16) || !aligned(p->V_dev, 16))) {
        set_error("%s: K_dev and V_dev must be 16-byte aligned device pointers", who);
        return POLYKV_EINVAL;
    }
    return POLYKV_OK;
}

static int check_layers(const polykv_pages* p, int begin, int end, const char* who) {
    if (begin < 0 || end > p->layers || begin >= end) {
        set_error("%s: layer range [%d,%d) outside [0,%d)", who, begin, end, p->layers);
        return POLYKV_ESHAPE;
    }
    return POLYKV_OK;
}

static int check_nodes(int nodes, const char* who) {
    if (nodes < 1 || nodes > POLYKV_MAX_TREE_NODES) {
        set_error("%s: nodes=%d must be in 1 .. %d", who, nodes, POLYKV_MAX_TREE_NODES);
        return POLYKV_ESHAPE;
    }
    return POLYKV_OK;
}

// `sums`: the array that receives the offsets, or what was granted.
static int check_resize(const polykv_pages* pages, const int32_t* targets, const int32_t* slots_dev, int slots, const int32_t* sums,
                        const char* sums_name, const char* who) {
    const int rc = check_pages(pages, false, who);
    if (rc != POLYKV_OK) return rc;
    if (pages->free_dev == nullptr || pages->free_state_dev == nullptr || pages->ticket_dev == nullptr || targets == nullptr) {
        set_error("%s: NULL free list, ticket or targets", who);
        return POLYKV_EINVAL;
    }
    if (!aligned(pages->free_dev, 4) || !aligned(pages->free_state_dev, 4) || !aligned(pages->ticket_dev, 4) || !aligned(targets, 4) || !aligned(slots_dev, 4) ||
        !aligned(sums, 4)) {
        set_error("%s: arrays must be 4-byte aligned", who);
        return POLYKV_EINVAL;
    }
    if (slots_dev != nullptr && (slots < 0 || slots > (1 << 30))) {
        set_error("%s: slots=%d outside [0, 2^30]", who, slots);
        return POLYKV_ESHAPE;
    }
    const void* own[] = {pages->table_dev, pages->lengths_dev, pages->free_dev, pages->free_state_dev, pages->ticket_dev};
    for (const void* p : own)
        if (p == targets || p == slots_dev || p == sums || (slots_dev != nullptr && slots_dev == sums) || targets == slots_dev || targets == sums) {
            set_error("%s: targets, slots and %s must be arrays of their own", who, sums_name);
            return POLYKV_EINVAL;
        }
    return POLYKV_OK;
}

// Both parts' choices, so that pool_attend_tree_workspace() and pool_attend_tree() agree by construction.
static int make_tree_plan(const polykv_pool* pool, const polykv_pages* pages, const polykv_tree_params* prm, AttendPlan* plan,
                          TreePlan* tree) {
    const char* who = "pool_attend_tree";
    if (prm == nullptr) {
        set_error("%s: NULL params", who);
        return POLYKV_EINVAL;
    }
    int rc = check_pages(pages, true, who);
    if (rc == POLYKV_OK) rc = check_nodes(prm->nodes, who);
    if (rc != POLYKV_OK) return rc;
    if (pool != nullptr && (pool->layers != pages->layers || pool->kv_heads != pages->kv_heads || pool->head_dim != pages->head_dim)) {
        set_error("%s: the pool has layers=%d kv_heads=%d head_dim=%d, the pages %d, %d, %d", who, pool->layers, pool->kv_heads,
                  pool->head_dim, pages->layers, pages->kv_heads, pages->head_dim);
        return POLYKV_ESHAPE;
    }
    if (prm->page_splits < 0) {
        set_error("%s: bad page_splits %d", who, prm->page_splits);
        return POLYKV_EINVAL;
    }
    polykv_attend_params a;
    memset(&a, 0, sizeof(a));
    a.agents = pages->agents, a.q_per_agent = prm->nodes, a.q_heads = prm->q_heads;
    a.layer_begin = prm->layer_begin, a.layer_end = prm->layer_end, a.scale = prm->scale;
    a.kernel = prm->kernel, a.splits = prm->splits, a.io_dtype = pages->dtype, a.key_precision = prm->key_precision;
    polykv_pool none;   // without a pool: the same checks, for a pool of one empty tile
    memset(&none, 0, sizeof(none));
    none.layers = pages->layers, none.kv_heads = pages->kv_heads, none.head_dim = pages->head_dim, none.tokens = 1, none.tiles = 1;
    rc = make_plan(pool != nullptr ? pool : &none, &a, plan, who);
    if (rc != POLYKV_OK) return rc;
    plan->partials_only = 1;
    TreePlan& t = *tree;
    memset(&t, 0, sizeof(t));
    t.counts = prm->counts_dev;
    t.mask = prm->mask_dev;
    t.words = (prm->nodes + 63) / 64;
    t.layer_begin = plan->layer_begin, t.layers = plan->layers, t.nodes = prm->nodes, t.q_heads = plan->q_heads, t.G = plan->G;
    t.rows = prm->nodes * plan->G;
    t.qscale = plan->qscale;
    plan_tree(page_view(pages), pool != nullptr ? plan->nsplit : 0, prm->page_splits, &t);
    const int64_t units = (int64_t)t.layers * pages->kv_heads;
    if ((units * pages->agents * t.nsplit + 8) * t.row_blocks > 0x7F000000) {   // (the grid is rounded up by less than 2^23)
        set_error("%s: %lld KV heads x %d agents x %d row blocks x %d splits are more workgroups than supported", who, (long long)units,
                  pages->agents, t.row_blocks, t.nsplit);
        return POLYKV_ESHAPE;
    }
    size_t off = pool != nullptr ? plan->total : 0;
    t.off_ml = t.off_o = off;
    if (t.merge) {
        off = align_up(off + (size_t)units * t.nsplit * plan->R * 2 * sizeof(float), 256);
        t.off_o = off;
        off = align_up(off + (size_t)units * t.nsplit * plan->R * plan->D * sizeof(float), 256);
    }
    t.total = off;
    return POLYKV_OK;
}

}  // namespace polykv

using namespace polykv;

extern "C" {

int polykv_pages_resize(const polykv_pages* pages, const int32_t* targets_dev, int32_t* slots_dev, int slots, int32_t* offsets_dev,
                        void* stream) {
    const char* who = "polykv_pages_resize";
    const int rc = check_resize(pages, targets_dev, slots_dev, slots, offsets_dev, "offsets", who);
    if (rc != POLYKV_OK) return rc;
    return hip_result(launch_pages_resize(pages, targets_dev, slots_dev, slots, offsets_dev, (hipStream_t)stream), who);
}

int polykv_pages_resize_by_agent(const polykv_pages* pages, const int32_t* targets_dev, int32_t* slots_dev, int per_agent,
                                 int32_t* granted_dev, void* stream) {
    const char* who = "polykv_pages_resize_by_agent";
    const int64_t slots = slots_dev != nullptr && pages != nullptr ? (int64_t)per_agent * std::max(pages->agents, 1) : 0;
    if (slots > (1 << 30)) {   // (what else may be wrong with these numbers is looked at below)
        set_error("%s: %d slots for each of %d agents are more than 2^30", who, per_agent, pages->agents);
        return POLYKV_ESHAPE;
    }
    const int rc = check_resize(pages, targets_dev, slots_dev, (int)std::max<int64_t>(slots, -1), granted_dev, "granted", who);
    if (rc != POLYKV_OK) return rc;
    return hip_result(launch_pages_resize_by_agent(pages, targets_dev, slots_dev, slots_dev != nullptr ? per_agent : 0, granted_dev, (hipStream_t)stream), who);
}

int polykv_pages_write(const polykv_pages* pages, const void* K_dev, const void* V_dev, int in_dtype, int tokens, int64_t layer_stride,
                       int64_t token_stride, int64_t head_stride, const int32_t* slots_dev, int layer_begin, int layer_end,
                       void* stream) {
    const char* who = "polykv_pages_write";
    int rc = check_pages(pages, true, who);
    if (rc == POLYKV_OK) rc = check_layers(pages, layer_begin, layer_end, who);
    if (rc != POLYKV_OK) return rc;
    if (in_dtype != pages->dtype && in_dtype != POLYKV_F32) {
        set_error("%s: in_dtype %d is neither the pages' %d nor POLYKV_F32", who, in_dtype, pages->dtype);
        return POLYKV_EINVAL;
    }
    if (tokens < 0 || (int64_t)tokens * (pages->kv_heads * (pages->head_dim / 8)) > 0x7FFFFF00) {
        set_error("%s: tokens=%d must be >= 0 and tokens * kv_heads * head_dim less than 2^34", who, tokens);
        return POLYKV_ESHAPE;
    }
    if (tokens == 0) return POLYKV_OK;
    if (K_dev == nullptr || V_dev == nullptr || slots_dev == nullptr || !aligned(K_dev, 16) || !aligned(V_dev, 16) || !aligned(slots_dev, 4)) {
        set_error("%s: K and V must be 16-byte aligned device pointers, slots a 4-byte aligned one", who);
        return POLYKV_EINVAL;
    }
    const int64_t unit = in_dtype == POLYKV_F32 ? 4 : 8;
    if (layer_stride < 0 || token_stride < 0 || head_stride < 0 || ((layer_stride | token_stride | head_stride) & (unit - 1)) != 0) {
        set_error("%s: strides (%lld, %lld, %lld) must be >= 0 and multiples of 16 bytes", who, (long long)layer_stride,
                  (long long)token_stride, (long long)head_stride);
        return POLYKV_EINVAL;
    }
    return hip_result(launch_pages_write(pages, K_dev, V_dev, in_dtype, tokens, layer_stride, token_stride, head_stride, slots_dev,
                                         layer_begin, layer_end, (hipStream_t)stream),
                      who);
}

int polykv_tree_masks(const int32_t* parents_dev, const int32_t* counts_dev, int agents, int nodes, uint64_t* mask_dev,
                      int32_t* depth_dev, void* stream) {
    const char* who = "polykv_tree_masks";
    const int rc = check_nodes(nodes, who);
    if (rc != POLYKV_OK) return rc;
    if (agents < 1 || agents > POLYKV_MAX_PAGED_AGENTS) {
        set_error("%s: agents=%d must be in 1 .. %d", who, agents, POLYKV_MAX_PAGED_AGENTS);
        return POLYKV_ESHAPE;
    }
    if (parents_dev == nullptr || mask_dev == nullptr || !aligned(parents_dev, 4) || !aligned(counts_dev, 4) || !aligned(mask_dev, 8) ||
        !aligned(depth_dev, 4)) {
        set_error("%s: parents and mask must be device pointers, all arrays aligned to their elements", who);
        return POLYKV_EINVAL;
    }
    const void *in[] = {parents_dev, counts_dev}, *out[] = {mask_dev, depth_dev};
    for (const void* p : in)
        for (const void* q : out)
            if ((p != nullptr && p == q) || (const void*)mask_dev == (const void*)depth_dev) {
                set_error("%s: an output must not be an input", who);
                return POLYKV_EINVAL;
            }
    return hip_result(launch_tree_masks(parents_dev, counts_dev, agents, nodes, mask_dev, depth_dev, (hipStream_t)stream), who);
}

size_t pool_attend_tree_workspace(const polykv_pool* pool, const polykv_pages* pages, const polykv_tree_params* params) {
    AttendPlan plan;
    TreePlan tree;
    if (make_tree_plan(pool, pages, params, &plan, &tree) != POLYKV_OK) return 0;
    return tree.total;
}

int pool_attend_tree(const polykv_pool* pool, const polykv_pages* pages, const void* Q_dev, void* out_dev,
                     const polykv_tree_params* params, void* stream) {
    const char* who = "pool_attend_tree";
    int rc = pool != nullptr ? check_readable(pool, who) : POLYKV_OK;
    if (rc != POLYKV_OK) return rc;
    AttendPlan plan;
    TreePlan tree;
    rc = make_tree_plan(pool, pages, params, &plan, &tree);
    if (rc != POLYKV_OK) return rc;
    if (Q_dev == nullptr || out_dev == nullptr || !aligned(Q_dev, 16) || !aligned(out_dev, 16)) {
        set_error("%s: Q and out must be 16-byte aligned device pointers", who);
        return POLYKV_EINVAL;
    }
    // (in place is fine: rows are read by the workgroups that write them, before they do; other rows need not be)
    const uintptr_t q = (uintptr_t)Q_dev, o_at = (uintptr_t)out_dev;
    const size_t q_bytes = (size_t)plan.layers * plan.H * plan.R * plan.D * 2;
    if (q != o_at && q < o_at + q_bytes && o_at < q + q_bytes) {
        set_error("%s: out must be Q itself or not overlap it", who);
        return POLYKV_EINVAL;
    }
    if (!aligned(params->counts_dev, 4) || !aligned(params->mask_dev, 8)) {
        set_error("%s: counts must be 4-byte and mask 8-byte aligned", who);
        return POLYKV_EINVAL;
    }
    if (tree.total > 0 && (params->workspace_dev == nullptr || !aligned(params->workspace_dev, 256))) {
        set_error("%s: workspace must be a 256-byte aligned device pointer", who);
        return POLYKV_EINVAL;
    }
    if (params->workspace_bytes < tree.total) {
        set_error("%s: workspace has %zu bytes, %zu needed", who, params->workspace_bytes, tree.total);
        return POLYKV_ENOMEM;
    }
    char* ws = reinterpret_cast<char*>(params->workspace_dev);
    const hipStream_t s = (hipStream_t)stream;
    float *ml = reinterpret_cast<float*>(ws + tree.off_ml), *o = reinterpret_cast<float*>(ws + tree.off_o);
    PoolPart part;
    memset(&part, 0, sizeof(part));
    if (pool != nullptr) {
        const hipError_t e = launch_attend(pool, plan, Q_dev, nullptr, nullptr, ws, s);
        if (e != hipSuccess) return hip_result(e, who);
        part.ml = reinterpret_cast<const float*>(ws + plan.off_ml);
        part.o = reinterpret_cast<const float*>(ws + plan.off_o);
        part.nsplit = plan.nsplit;
        part.rotated = plan.vcodec != POLYKV_VALUES_INT8;
        part.signs = plan.signs;
    }
    // One token range per agent and few of the pool: the pages' kernel completes the rows.  Else the partials are joined after it.
    hipError_t e = launch_attend_pages(page_view(pages), tree, pages->dtype == POLYKV_BF16, Q_dev, ml, o, tree.merge ? nullptr : out_dev,
                                       part, s);
    if (e == hipSuccess && tree.merge) e = launch_tree_merge(plan, tree, pool != nullptr, part.ml, part.o, ml, o, out_dev, s);
    return hip_result(e, who);
}

int polykv_pages_accept(const polykv_pages* pages, const int32_t* tokens_dev, const int32_t* following_dev, const int32_t* parents_dev,
                        const int32_t* counts_dev, int nodes, int32_t* path_dev, int32_t* accepted_dev, int32_t* next_dev,
                        int32_t* kept_dev, void* stream) {
    const char* who = "polykv_pages_accept";
    int rc = check_pages(pages, true, who);
    if (rc == POLYKV_OK) rc = check_nodes(nodes, who);
    if (rc != POLYKV_OK) return rc;
    const void* all[] = {tokens_dev, following_dev, parents_dev, path_dev, accepted_dev, next_dev, kept_dev};
    for (const void* p : all)
        if (p == nullptr || !aligned(p, 4)) {
            set_error("%s: all arrays but counts must be given, 4-byte aligned", who);
            return POLYKV_EINVAL;
        }
    const void* in[] = {tokens_dev, following_dev, parents_dev, counts_dev, pages->lengths_dev, pages->table_dev};
    const void* out[] = {path_dev, accepted_dev, next_dev, kept_dev};
    bool own = true;
    for (const void*& q : out) {
        for (const void* p : in) own &= p != q;   // (every layer's workgroups read the inputs)
        for (const void*& p : out) own &= &p == &q || p != q;
    }
    if (!own) {
        set_error("%s: an output must not be an input or another output", who);
        return POLYKV_EINVAL;
    }
    if (!aligned(counts_dev, 4)) {
        set_error("%s: counts must be 4-byte aligned", who);
        return POLYKV_EINVAL;
    }
    return hip_result(launch_pages_accept(pages, tokens_dev, following_dev, parents_dev, counts_dev, nodes, path_dev, accepted_dev,
                                          next_dev, kept_dev, (hipStream_t)stream),
                      who);
}

}  // extern "C"
