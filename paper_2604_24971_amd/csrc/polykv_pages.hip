// Private continuations in pages (gfx950): block tables and slot maps, writes by slot, masks of draft trees, acceptance.
//
// None of them computes anything to speak of.  A step's calls are bound by the latency of one launch and the chain of
// dependent loads in it, prompts' writes by memory.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <algorithm>

#include "polykv_pages.hpp"

namespace polykv {

// ------------------------------------------------------------------------------- block tables ---
// Sums over agents of three numbers at once.  The first is capped: it is only compared with the number of free pages, and
// the sum of what 4,096 agents may ask for does not fit 32 bits.
constexpr uint32_t kNeedCap = 1u << 28;   // above every page number
struct Sums {
    uint32_t need, give, grow;
};
__device__ __forceinline__ Sums add(const Sums& a, const Sums& b) {
    return Sums{min(a.need + b.need, kNeedCap), a.give + b.give, a.grow + b.grow};
}
__device__ __forceinline__ Sums wave_scan(Sums x, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const Sums y = {(uint32_t)__shfl_up((int)x.need, d, 64), (uint32_t)__shfl_up((int)x.give, d, 64),
                        (uint32_t)__shfl_up((int)x.grow, d, 64)};
        if (lane >= d) x = add(y, x);
    }
    return x;
}

struct AgentChange {
    int length, target, have, want;
};
__device__ __forceinline__ AgentChange change_of(const PageView& v, const int32_t* targets, int a) {
    AgentChange c = {0, 0, 0, 0};
    if (a < v.A) {
        int rem;
        const int most = v.max_blocks * v.P;
        c.length = tokens_of(v, a);
        c.target = targets[a];
        if (c.target < 0 || c.target > most) c.target = c.length;
        c.have = v.div_P.divide(c.length, &rem);
        c.have += rem > 0;
        c.want = v.div_P.divide(c.target, &rem);
        c.want += rem > 0;
    }
    return c;
}

// Every workgroup works out the sums over all agents for itself -- 4,096 agents are four rounds -- and then does its share of
// the agents' table entries and of the slots, the agent of a slot by bisection.  Nothing that other workgroups still read is
// written before they are done: the workgroup that is the last to say so writes the lengths and the ring's state (nobody waits
// for anybody; a launch of its own for them took 4.5 us).  Pages that are given back go behind the ring's last, where no page to
// be taken lies, so the two do not have to wait for each other.
// A step of few agents is all latency: 256 threads there (15 agents: 3.0 us if nothing changes, 3.7 to grow by 16 tokens each, 5.3 with
// their slots -- the bisection, then the ring or the table behind it --, 3.6 to shrink; with 1,024 threads about a microsecond more).
// 1,024 agents are one round of sums, the chain of two scans by shuffles, two loops over the waves' sums and four barriers: 5.8 us of the
// launch if nothing changes, 6.4 with the table entries of 600 new tokens each, 9.3 with their 460,000 slots, 6.1 to shrink.
// 4,096 agents are four rounds: 17.2 us whatever is done behind them.
// BY_AGENT: the slot map has n_slots / A entries for every agent and the third output is how far each grew, for callers whose rows
// have places by agent: an agent that got nothing then moves nobody else's slots.
template <int THREADS, bool BY_AGENT>
__global__ __launch_bounds__(THREADS) void pages_resize_kernel(PageView v, const int32_t* __restrict__ targets, int32_t* ring,
                                                               int32_t* state, int32_t* ticket, int32_t* __restrict__ slots, int n_slots,
                                                               int32_t* __restrict__ offsets) {
    extern __shared__ int shared[];
    int* const end_s = shared;                 // where an agent's new tokens end in the slot map
    int* const len_s = shared + v.A;           // its length
    int* const tgt_s = shared + 2 * v.A;       // its length after the call
    int* const at_s = shared + 3 * v.A;        // its first page among those taken, or given back
    __shared__ Sums wave_s[THREADS / 64];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t NP = v.pages;
    // (the ring's state is the caller's memory: whatever it holds, places stay inside the ring)
    const uint32_t first = (uint32_t)max(state[0], 0) % NP;
    const uint32_t count = min((uint32_t)max(state[1], 0), NP);
    Sums before = {0, 0, 0};
    uint32_t taken = 0;
    for (int a0 = 0; a0 < v.A; a0 += THREADS) {
        const int a = a0 + tid;
        AgentChange c = change_of(v, targets, a);
        // what is asked for, whether it is there, and only then what the slots are
        Sums x = {c.want > c.have ? min((uint32_t)(c.want - c.have), kNeedCap) : 0u, 0u, 0u};
        const uint32_t need = x.need;
        x.give = c.have > c.want ? c.have - c.want : 0;
        Sums sum = wave_scan(x, lane);
        if (lane == 63) wave_s[wave] = sum;
        __syncthreads();
        Sums base = before, total = before;
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w == wave) base = total;
            total = add(total, wave_s[w]);
        }
        const Sums upto = add(base, sum);
        __syncthreads();
        const bool granted = need == 0 || upto.need <= count;
        if (!granted) c.target = c.length, c.want = c.have;
        // (pages are asked for in order, and all that come before a granted agent are granted too: the largest sum that was
        // granted is what has been taken)
        const uint32_t grow = c.target > c.length ? c.target - c.length : 0;
        const Sums g = wave_scan(Sums{0u, 0u, grow}, lane);
        uint32_t most = granted && need > 0 ? upto.need : 0;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d, 64));
        if (lane == 63) wave_s[wave] = Sums{most, 0u, g.grow};
        __syncthreads();
        uint32_t grow_base = before.grow, grow_total = before.grow;
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w == wave) grow_base = grow_total;
            grow_total += wave_s[w].grow;
            taken = max(taken, wave_s[w].need);
        }
        __syncthreads();
        if (a < v.A) {
            end_s[a] = (int)(grow_base + g.grow);
            len_s[a] = c.length;
            tgt_s[a] = c.target;
            at_s[a] = (int)(need > 0 ? upto.need - need : upto.give - (c.have > c.want ? c.have - c.want : 0));
        }
        before = Sums{total.need, total.give, grow_total};
    }
    __syncthreads();
    const int grown = v.A > 0 ? end_s[v.A - 1] : 0;

    const int waves = gridDim.x * (THREADS / 64);
    for (int a = blockIdx.x * (THREADS / 64) + wave; a < v.A; a += waves) {
        int rem;
        int have = v.div_P.divide(len_s[a], &rem);
        have += rem > 0;
        int want = v.div_P.divide(tgt_s[a], &rem);
        want += rem > 0;
        int32_t* row = v.table + (size_t)a * v.max_blocks;
        for (int b = have + lane; b < want; b += 64) row[b] = ring[(first + (uint32_t)at_s[a] + (uint32_t)(b - have)) % NP];
        for (int b = want + lane; b < have; b += 64) {
            ring[(first + count + (uint32_t)at_s[a] + (uint32_t)(b - want)) % NP] = row[b];
            row[b] = -1;
        }
    }
    // page and place of an agent's new token t
    auto page_of = [&](int a, int t, int* off) {
        int rem;
        int have = v.div_P.divide(len_s[a], &rem);
        have += rem > 0;
        const int b = v.div_P.divide(t, off);
        return b < have ? v.table[(size_t)a * v.max_blocks + b] : ring[(first + (uint32_t)at_s[a] + (uint32_t)(b - have)) % NP];
    };
    [[maybe_unused]] const uint32_t per_agent = BY_AGENT ? (uint32_t)n_slots / (uint32_t)v.A : 0;
    // four slots of a thread
    for (int i0 = 4 * (blockIdx.x * THREADS + tid); i0 < n_slots; i0 += 4 * gridDim.x * THREADS) {
        int a = 0;
        if (!BY_AGENT && i0 < grown) {   // one bisection, and then on from agent to agent: the first whose tokens end behind i0
            int hi = v.A - 1;
            while (a < hi) {
                const int mid = (a + hi) >> 1;
                if (end_s[mid] > i0) hi = mid;
                else a = mid + 1;
            }
        }
        int page[4], off[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            page[u] = -1, off[u] = 0;
            const int i = i0 + u;
            if constexpr (BY_AGENT) {
                if (i >= n_slots) continue;
                int k;
                a = i / per_agent, k = i - a * per_agent;
                if (k < tgt_s[a] - len_s[a]) page[u] = page_of(a, len_s[a] + k, &off[u]);
            } else {
                if (i >= grown) continue;
                while (a < v.A - 1 && end_s[a] <= i) ++a;
                // (in range for whatever the sums hold)
                page[u] = page_of(a, min(max(tgt_s[a] - (end_s[a] - i), 0), v.max_blocks * v.P - 1), &off[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i0 + u < n_slots) slots[i0 + u] = (uint32_t)page[u] < NP ? page[u] * v.P + off[u] : -1;
    }
    if (offsets != nullptr && blockIdx.x == 0) {
        if constexpr (BY_AGENT) {
            for (int a = tid; a < v.A; a += THREADS) offsets[a] = max(tgt_s[a] - len_s[a], 0);
        } else {
            for (int a = tid; a < v.A; a += THREADS) offsets[a + 1] = end_s[a];
            if (tid == 0) offsets[0] = 0;
        }
    }
    __shared__ int last_s;
    if (gridDim.x > 1) {   // (what this workgroup has read of lengths and state is in LDS and registers by now)
        __syncthreads();
        if (tid == 0) last_s = atomicAdd(ticket, 1) == (int)gridDim.x - 1;
        __syncthreads();
        if (!last_s) return;
        if (tid == 0) *ticket = 0;
    }
    for (int a = tid; a < v.A; a += THREADS) v.lengths[a] = tgt_s[a];
    if (tid == 0) {
        state[0] = (int)((first + taken) % NP);
        state[1] = (int)min(count - min(taken, count) + before.give, NP);
    }
}

template <bool BY_AGENT>
static hipError_t launch_resize(const polykv_pages* p, const int32_t* targets, int32_t* slots, int n_slots, int32_t* offsets,
                                hipStream_t s) {
    const PageView v = page_view(p);
    const int shared = 4 * v.A * (int)sizeof(int);
    if (shared > 48 * 1024) {   // (by call: the attribute belongs to the current device)
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(pages_resize_kernel<1024, BY_AGENT>), hipFuncAttributeMaxDynamicSharedMemorySize, shared);
        if (err != hipSuccess) return err;
    }
    if (slots == nullptr) n_slots = 0;
    if (v.A <= 64 && n_slots <= 4096) {
        launch_kernel(pages_resize_kernel<256, BY_AGENT>, dim3(1), dim3(256), shared, s, {}, v, targets, p->free_dev, p->free_state_dev, p->ticket_dev, slots,
                      n_slots, offsets);
    } else {
        const int by_slots = (n_slots + 4095) / 4096, by_agents = (v.A + 15) / 16;   // a round each: four slots a thread, an agent a wave
        launch_kernel(pages_resize_kernel<1024, BY_AGENT>, dim3(std::min(std::max(by_slots, by_agents), 256)), dim3(1024), shared, s, {}, v, targets, p->free_dev,
                      p->free_state_dev, p->ticket_dev, slots, n_slots, offsets);
    }
    return hipGetLastError();
}

hipError_t launch_pages_resize(const polykv_pages* p, const int32_t* targets, int32_t* slots, int n_slots, int32_t* offsets,
                               hipStream_t s) {
    return launch_resize<false>(p, targets, slots, n_slots, offsets, s);
}
hipError_t launch_pages_resize_by_agent(const polykv_pages* p, const int32_t* targets, int32_t* slots, int per_agent, int32_t* granted,
                                        hipStream_t s) {
    return launch_resize<true>(p, targets, slots, p->agents * per_agent, granted, s);
}

// -------------------------------------------------------------------------------------- write ---
// A thread moves eight elements of a token's keys and the same of its values; consecutive threads take consecutive pieces of
// a head, then the heads of a token.  The slot is not needed before the stores, so that only one latency is waited for.  Bound by
// memory: 7,400 tokens into 32 layers of 8 x 128 numbers (1.9 GB in and out) 346 us, 5.6 TB/s, where a copy of 1 GiB reaches 5.1;
// one layer's drafts of a step of 15 agents 2.4 us, which is one launch.
typedef uint32_t page_uint4 __attribute__((ext_vector_type(4)));
typedef float page_float4 __attribute__((ext_vector_type(4)));
typedef _Float16 page_half8 __attribute__((ext_vector_type(8)));
typedef __bf16 page_bf8 __attribute__((ext_vector_type(8)));
typedef float page_float8 __attribute__((ext_vector_type(8)));

// MODE: 0 the pages' type, 1 fp32 to fp16, 2 fp32 to bfloat16 (to nearest even).
template <int MODE> __device__ __forceinline__ page_uint4 load_piece(const void* src, int64_t at) {
    if constexpr (MODE == 0) {
        return *reinterpret_cast<const page_uint4*>(reinterpret_cast<const uint16_t*>(src) + at);
    } else {
        const page_float4* f = reinterpret_cast<const page_float4*>(reinterpret_cast<const float*>(src) + at);
        const page_float4 lo = f[0], hi = f[1];
        const page_float8 x = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        if constexpr (MODE == 1) return __builtin_bit_cast(page_uint4, __builtin_convertvector(x, page_half8));
        else return __builtin_bit_cast(page_uint4, __builtin_convertvector(x, page_bf8));
    }
}

struct WriteArgs {
    PageView v;
    const void *K, *V;
    const int32_t* slots;
    int64_t layer_stride, token_stride, head_stride;
    int items, layer_begin;     // pieces of a layer
    FastDiv div_token;          // pieces of a token
    int head_shift;             // log2 of the pieces of a head
};

template <int MODE> __global__ __launch_bounds__(256) void pages_write_kernel(WriteArgs w) {
    const int item = blockIdx.x * 256 + threadIdx.x;
    if (item >= w.items) return;
    int piece;
    const int t = w.div_token.divide(item, &piece), l = blockIdx.y;
    const int h = piece >> w.head_shift, c = (piece & ((1 << w.head_shift) - 1)) * 8;
    const int slot = w.slots[t];
    const int64_t from = l * w.layer_stride + t * w.token_stride + h * w.head_stride + c;
    const page_uint4 k = load_piece<MODE>(w.K, from), x = load_piece<MODE>(w.V, from);
    if ((uint32_t)slot >= (uint32_t)w.v.pages * (uint32_t)w.v.P) return;
    int off;
    const int page = w.v.div_P.divide(slot, &off);
    const size_t to = ((size_t)(w.layer_begin + l) * w.v.pages * w.v.H * w.v.P + page_row(w.v, page, h, off)) * w.v.D + c;
    *reinterpret_cast<page_uint4*>(w.v.K + to) = k;
    *reinterpret_cast<page_uint4*>(w.v.V + to) = x;
}

hipError_t launch_pages_write(const polykv_pages* p, const void* K, const void* V, int in_dtype, int tokens, int64_t layer_stride,
                              int64_t token_stride, int64_t head_stride, const int32_t* slots, int layer_begin, int layer_end,
                              hipStream_t s) {
    const int per_token = p->kv_heads * p->head_dim / 8;
    const WriteArgs w = {page_view(p), K, V, slots, layer_stride, token_stride, head_stride, tokens * per_token, layer_begin,
                         FastDiv::by(per_token), p->head_dim == 64 ? 3 : p->head_dim == 128 ? 4 : 5};
    const int mode = in_dtype != POLYKV_F32 ? 0 : p->dtype == POLYKV_F16 ? 1 : 2;
    launch_kernel(mode == 0 ? pages_write_kernel<0> : mode == 1 ? pages_write_kernel<1> : pages_write_kernel<2>,
                  dim3((w.items + 255) / 256, layer_end - layer_begin), dim3(256), 0, s, {}, w);
    return hipGetLastError();
}

// -------------------------------------------------------------------------------------- trees ---
__device__ __forceinline__ int parent_of(const int32_t* parents, int i, int count) {   // an earlier draft, or -1
    const int p = i < count ? parents[i] : -1;
    return p < i ? max(p, -1) : -1;
}

// One workgroup per agent, a thread per draft.  A draft's set and its ancestors' join in rounds: after round k a draft knows the
// 2^k nearest of them and the one they end at, so the deepest tree takes log2(nodes) rounds (a walk from parent to parent takes as
// many as it is deep).  Latency: 15 trees of 16 drafts 2.6 us, 512 of 256 drafts 5.5.
template <int W> __global__ __launch_bounds__(64 * W) void tree_masks_kernel(const int32_t* __restrict__ parents, const int32_t* __restrict__ counts,
                                                                             int nodes, uint64_t* __restrict__ mask, int32_t* __restrict__ depth) {
    __shared__ uint64_t set_s[2][W][64 * W];
    __shared__ int up_s[2][64 * W], depth_s[2][64 * W];
    const int a = blockIdx.x, i = threadIdx.x;
    const int count = counts != nullptr ? min(max(counts[a], 0), nodes) : nodes;
    int up = i < nodes ? parent_of(parents + (size_t)a * nodes, i, count) : -1;
    int above = up >= 0 ? 1 : 0;
    uint64_t set[W];
#pragma unroll
    for (int w = 0; w < W; ++w) set[w] = i < count && (i >> 6) == w ? 1ull << (i & 63) : 0;
    for (int reach = 1, k = 0; reach < nodes; reach <<= 1, k ^= 1) {
#pragma unroll
        for (int w = 0; w < W; ++w) set_s[k][w][i] = set[w];
        up_s[k][i] = up;
        depth_s[k][i] = above;
        __syncthreads();
        if (up >= 0) {
#pragma unroll
            for (int w = 0; w < W; ++w) set[w] |= set_s[k][w][up];
            above += depth_s[k][up];
            up = up_s[k][up];
        }
    }
    if (i < nodes) {
        const size_t at = (size_t)a * nodes + i;
        const int words = (nodes + 63) >> 6;
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (w < words) mask[at * words + w] = set[w];
        if (depth != nullptr) depth[at] = above;
    }
}

hipError_t launch_tree_masks(const int32_t* parents, const int32_t* counts, int agents, int nodes, uint64_t* mask, int32_t* depth,
                             hipStream_t s) {
    const int words = (nodes + 63) / 64;
    const auto kern = words == 1 ? tree_masks_kernel<1> : words == 2 ? tree_masks_kernel<2> : words == 3 ? tree_masks_kernel<3> : tree_masks_kernel<4>;
    launch_kernel(kern, dim3(agents), dim3(64 * words), 0, s, {}, parents, counts, nodes, mask, depth);
    return hipGetLastError();
}

// One workgroup per agent and layer; each works the path out for itself (the layers' first writes it down).
// A draft that continues its parent as the model does enters itself as the parent's successor, the lowest one stays, and the
// path follows the successors from draft 0.  Then a thread moves one 16-byte piece of one head's keys, and of its values, along the
// whole path: a path's k-th draft is k at the least, so what is read for step k lies behind everything written before it, and
// eight steps' pieces are read before they are written.  32 layers of 15 agents with 16 drafts each take 4.0 us, of which the chain of
// dependent loads (length, parent, the model's token, page, row) is most; 24 layers of 64 agents with 100 drafts 15.4, the moves 10 of it.
__global__ __launch_bounds__(256) void pages_accept_kernel(PageView v, const int32_t* __restrict__ tokens, const int32_t* __restrict__ following,
                                                           const int32_t* __restrict__ parents, const int32_t* __restrict__ counts,
                                                           int nodes, int32_t* __restrict__ path, int32_t* __restrict__ accepted,
                                                           int32_t* __restrict__ next, int32_t* __restrict__ kept) {
    __shared__ int successor_s[POLYKV_MAX_TREE_NODES], path_s[POLYKV_MAX_TREE_NODES], n_s;
    __shared__ int from_s[POLYKV_MAX_TREE_NODES], to_s[POLYKV_MAX_TREE_NODES];   // rows of head 0, -1: nothing to move
    const int a = blockIdx.x, l = blockIdx.y, i = threadIdx.x;
    const int length = tokens_of(v, a), count = drafts_of(counts, a, nodes, length), before = length - count;
    const size_t at = (size_t)a * nodes;
    successor_s[i] = INT32_MAX;
    __syncthreads();
    if (i < count) {
        const int up = parent_of(parents + at, i, count);
        if (up >= 0 && tokens[at + i] == following[at + up]) atomicMin(&successor_s[up], i);
    }
    __syncthreads();
    if (i == 0) {
        int n = 0;
        for (int k = 0; k < count; k = successor_s[k]) path_s[n++] = k;   // (a successor is a later draft, so this ends)
        n_s = n;
    }
    __syncthreads();
    const int n = n_s;
    if (i < n) {
        int from_off, to_off;
        const int from_block = v.div_P.divide(before + path_s[i], &from_off), to_block = v.div_P.divide(before + i, &to_off);
        const int32_t* row = v.table + (size_t)a * v.max_blocks;
        const int from_page = row[from_block], to_page = row[to_block];
        const bool move = path_s[i] != i && (uint32_t)from_page < (uint32_t)v.pages && (uint32_t)to_page < (uint32_t)v.pages;
        from_s[i] = move ? page_row(v, from_page, 0, from_off) : -1;
        to_s[i] = move ? page_row(v, to_page, 0, to_off) : -1;
    }
    if (l == 0) {
        if (i < nodes) path[at + i] = i < n ? path_s[i] : -1;
        if (i == 0) {
            accepted[a] = n;
            next[a] = n > 0 ? following[at + path_s[n - 1]] : -1;
            kept[a] = before + n;
        }
    }
    __syncthreads();
    const int pieces = v.H * v.D / 8, per_head = v.D / 8;
    const size_t layer = (size_t)l * v.pages * v.H * v.P * v.D;
    for (int piece = i; piece < pieces; piece += 256) {
        const int h = piece / per_head;
        const size_t at_head = layer + (size_t)h * v.P * v.D + (piece - h * per_head) * 8;
        for (int k0 = 1; k0 < n; k0 += 8) {
            page_uint4 x[8], y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k0 + k < n && from_s[k0 + k] >= 0) {
                    const size_t from = at_head + (size_t)from_s[k0 + k] * v.D;
                    x[k] = *reinterpret_cast<const page_uint4*>(v.K + from);
                    y[k] = *reinterpret_cast<const page_uint4*>(v.V + from);
                }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k0 + k < n && from_s[k0 + k] >= 0) {
                    const size_t to = at_head + (size_t)to_s[k0 + k] * v.D;
                    *reinterpret_cast<page_uint4*>(v.K + to) = x[k];
                    *reinterpret_cast<page_uint4*>(v.V + to) = y[k];
                }
        }
    }
}

hipError_t launch_pages_accept(const polykv_pages* p, const int32_t* tokens, const int32_t* following, const int32_t* parents,
                               const int32_t* counts, int nodes, int32_t* path, int32_t* accepted, int32_t* next, int32_t* kept,
                               hipStream_t s) {
    launch_kernel(pages_accept_kernel, dim3(p->agents, p->layers), dim3(256), 0, s, {}, page_view(p), tokens, following, parents,
                  counts, nodes, path, accepted, next, kept);
    return hipGetLastError();
}

}  // namespace polykv
