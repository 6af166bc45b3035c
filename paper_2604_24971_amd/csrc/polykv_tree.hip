// Attention of drafted tokens over their agent's continuation in pages, and its join with the pool's part (gfx950).
//
// For the rows of one agent and KV head (drafts x query heads of the group) and the tokens t that a row sees,
//   m = max s(t),  l = sum 2^(s(t) - m),  o = sum 2^(s(t) - m) v(t),   s(t) = q . k(t) * scale * log2 e
// over one pass through the tokens: a partial (m, l, o) per row.  Partials of token ranges, and the pool's (whose o is in the
// rotated value domain), join with weights 2^(m - M); the output is o / l.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <mutex>

#include "polykv_layout.hpp"
#include "polykv_pages.hpp"

namespace polykv {

typedef _Float16 tree_half8 __attribute__((ext_vector_type(8)));
typedef _Float16 tree_half2 __attribute__((ext_vector_type(2)));
typedef __bf16 tree_bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 tree_bf2 __attribute__((ext_vector_type(2)));
typedef float tree_float2 __attribute__((ext_vector_type(2)));
typedef float tree_float16 __attribute__((ext_vector_type(16)));
typedef uint32_t tree_uint4 __attribute__((ext_vector_type(4)));

template <bool BF> __device__ __forceinline__ tree_float16 tree_mfma(const tree_uint4& a, const tree_uint4& b, const tree_float16& c) {
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(tree_bf8, a), __builtin_bit_cast(tree_bf8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(tree_half8, a), __builtin_bit_cast(tree_half8, b), c, 0, 0, 0);
}
template <bool BF> __device__ __forceinline__ uint32_t pack2(float x, float y) {   // to nearest even
    const tree_float2 f = {x, y};
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, tree_bf2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, tree_half2));
}
__device__ __forceinline__ float other_half_max(float x) {   // over lanes l and l ^ 32
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Whether one of the two 16-bit numbers is infinite or NaN.
template <bool BF> __device__ __forceinline__ bool any_nonfinite(uint32_t w) {
    constexpr uint32_t exponents = BF ? 0x7F807F80u : 0x7C007C00u, one = BF ? 0x00800080u : 0x04000400u;
    return (((w & exponents) + one) & 0x80008000u) != 0;
}

constexpr int kRaise = 8;   // a row's reference moves when a score is 2^8 times above it

// Tokens [32-token tiles] are the M dimension of the score products and the K dimension of the value products, rows the N
// dimension of both, so that a lane has one row throughout and its probabilities leave the score accumulators in the order
// in which they enter the value products (tokens 8 (i / 4) + 4 h + i % 4 of a tile for i < 16, h = lane / 32).
//   keys    lane (n, h) holds token n's elements 16 j + 8 h .. + 7: a key row's pieces straight from its page, no staging;
//   values  lane (n, h) loads coordinates (D / 32) n .. of the 16 tokens of its half, whole rows at a time, and makes the products'
//           operands (eight tokens of one coordinate) of them by byte permutes in registers: value block e of the products
//           has coordinate (D / 32) m + e in its row m.
// The tile's page numbers are requested two tiles ahead, its keys when the scores of the tile before are done, its values when
// that tile's value products are.  Four waves take the tiles of a token range in turn and are joined through LDS at the end.
template <int D, bool BF, int NT> struct PageTile {
    static constexpr int KJ = D / 16, VW = D / 64;   // key pieces of a lane; dwords of a value row in a lane
    tree_uint4 k[KJ];
    uint32_t v[16][VW];
};

struct TreeArgs {
    PageView v;
    TreePlan t;
    const uint16_t* Q;
    float *ml, *o;
    uint16_t* out;   // not nullptr: the rows are complete, written normalized
};

template <int D, bool BF, int NT>
__global__ __launch_bounds__(256, NT == 2 && D == 128 ? 1 : D == 256 ? 1 : 2) void attend_pages_kernel(TreeArgs g) {
    constexpr int ROWS = 32 * NT, MG = D / 32, KJ = D / 16, VW = D / 64, OSTRIDE = D + 4;
    extern __shared__ __align__(16) float o_s[];   // [4][ROWS][OSTRIDE]
    __shared__ float m_s[4][ROWS], l_s[4][ROWS];
    const PageView& v = g.v;
    const TreePlan& t = g.t;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, n = lane & 31;

    // Workgroup -> (token range of an agent and KV head, row block).  Consecutive workgroups go to the eight dies in turn: the row
    // blocks of a token range follow each other on one die, whose L2 they share.
    int row_block, split, a, kvh;
    const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x;
    const int stream = t.div_row_blocks.divide((int)(block >> 3), &row_block) * 8 + (int)(block & 7);
    if (stream >= t.layers * v.H * v.A * t.nsplit) return;
    const int ua = t.div_nsplit.divide(stream, &split), usel = t.div_A.divide(ua, &a), ls = t.div_H.divide(usel, &kvh);
    const int row0 = row_block * ROWS;

    const int length = tokens_of(v, a), count = drafts_of(t.counts, a, t.nodes, length), before = length - count;
    // the range's tiles; a block of rows that are all behind the agent's drafts sees none
    const int tiles = row0 < count * t.G ? (length + 31) >> 5 : 0;
    const int per_split = ((tiles + t.nsplit - 1) / t.nsplit + 3) & ~3;
    const int t_begin = split * per_split, t_end = min(tiles, t_begin + per_split);
    const int first = t_begin + wave;

    const size_t layer = (size_t)(t.layer_begin + ls) * v.pages * v.H * v.P * D;
    const uint16_t* const Kb = v.K + layer;
    const uint16_t* const Vb = v.V + layer;
    const int32_t* const table = v.table + (size_t)a * v.max_blocks;

    // token of the lane in a tile -> its row among the layer's, -1 if it is not there
    auto page_at = [&](int tile) {
        int off;
        const int b = v.div_P.divide(min(32 * tile + n, length - 1), &off);
        return table[b];
    };
    auto row_at = [&](int tile, int page) {
        int off;
        const int tok = 32 * tile + n;
        (void)v.div_P.divide(tok, &off);
        return tok < length && (uint32_t)page < (uint32_t)v.pages ? page_row(v, page, kvh, off) : -1;
    };
    PageTile<D, BF, NT> x;
    auto load_keys = [&](int row) {
        const uint16_t* src = Kb + (size_t)max(row, 0) * D + 8 * h;
#pragma unroll
        for (int j = 0; j < KJ; ++j) x.k[j] = *reinterpret_cast<const tree_uint4*>(src + 16 * j);
    };
    auto load_values = [&](int row) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {   // tokens 8 q + 4 h .. + 3, which lie in one page
            const int r = __shfl(row, 8 * q + 4 * h, 64);
            const uint16_t* src = Vb + (size_t)max(r, 0) * D + MG * n;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (VW == 1) x.v[4 * q + e][0] = *reinterpret_cast<const uint32_t*>(src + e * D);
                else if constexpr (VW == 2) {
                    const uint2 w = *reinterpret_cast<const uint2*>(src + e * D);
                    x.v[4 * q + e][0] = w.x, x.v[4 * q + e][1] = w.y;
                } else {
                    const tree_uint4 w = *reinterpret_cast<const tree_uint4*>(src + e * D);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.v[4 * q + e][i] = w[i];
                }
            }
        }
    };

    tree_float16 acc[NT][MG];
    float m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt] = -INFINITY, l[nt] = 0.0f;
#pragma unroll
        for (int e = 0; e < MG; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[nt][e][i] = 0.0f;
    }

    if (first < t_end) {
        int row = row_at(first, page_at(first));
        int page = first + 4 < t_end ? page_at(first + 4) : -1;
        load_keys(row);
        load_values(row);
        // ---- the block's queries, lane (n, h): row n's elements 16 j + 8 h .. + 7 (rows past the last repeat it)
        tree_uint4 q[NT][KJ];
        int draft[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            int in_group;
            draft[nt] = t.div_G.divide(min(row0 + 32 * nt + n, t.rows - 1), &in_group);
            const uint16_t* src = g.Q + ((((size_t)ls * v.A + a) * t.nodes + draft[nt]) * t.q_heads + kvh * t.G + in_group) * D + 8 * h;
#pragma unroll
            for (int j = 0; j < KJ; ++j) q[nt][j] = *reinterpret_cast<const tree_uint4*>(src + 16 * j);
        }
        float poison[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) poison[nt] = 0.0f;

        for (int tile = first; tile < t_end; tile += 4) {
            tree_float16 s[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[nt][i] = 0.0f;
#pragma unroll
                for (int j = 0; j < KJ; ++j) s[nt] = tree_mfma<BF>(x.k[j], q[nt][j], s[nt]);
            }
            const int t0 = 32 * tile;
            const uint32_t there = (uint32_t)__ballot(row >= 0);   // (lanes 32 .. 63 repeat the tile's tokens)
            const bool more = tile + 4 < t_end;
            int next_row = -1;
            if (more) {
                next_row = row_at(tile + 4, page);
                load_keys(next_row);
                page = tile + 8 < t_end ? page_at(tile + 8) : -1;
            }

            // ---- tokens that are not there, and drafts that the lane's draft does not see
            if (there != 0xFFFFFFFFu || t0 + 32 > before || row0 + ROWS > count * t.G) {
                uint32_t bad = 0;   // drafts with a value that is not finite
                if (t0 + 32 > before) {
#pragma unroll
                    for (int u = 0; u < 16; ++u) {
                        bool b = false;
#pragma unroll
                        for (int w = 0; w < VW; ++w) b |= any_nonfinite<BF>(x.v[u][w]);
                        const uint64_t lanes = __ballot(b);
                        const int tok = 8 * (u >> 2) + (u & 3);
                        if ((uint32_t)lanes) bad |= 1u << tok;
                        if (lanes >> 32) bad |= 1u << (tok + 4);
                    }
                    bad &= there & ~(before > t0 ? (1u << (before - t0)) - 1 : 0u);
                }
                const uint32_t kept = there & ~bad;
                if (kept != 0xFFFFFFFFu) {   // their values are zeroed: a weight of 0 does not undo a NaN
#pragma unroll
                    for (int u = 0; u < 16; ++u) {
                        const bool keep = (kept >> (8 * (u >> 2) + 4 * h + (u & 3))) & 1;
#pragma unroll
                        for (int w = 0; w < VW; ++w) x.v[u][w] = keep ? x.v[u][w] : 0;
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    uint32_t seen = there;   // bit t: the lane's row sees token t of the tile
                    const int i = draft[nt];
                    if (i >= count) seen = 0;
                    else if (t0 + 32 > before) {
                        uint32_t drafts = 0;   // bit t: token t is a draft that the row sees
                        const int lead = t0 - before;   // the tile's first token as a draft
                        if (t.mask == nullptr) {
                            const int n_seen = i + 1 - lead;   // drafts 0 .. i
                            drafts = n_seen >= 32 ? 0xFFFFFFFFu : n_seen > 0 ? (1u << n_seen) - 1 : 0u;
                        } else {
                            const uint64_t* row_mask = t.mask + ((size_t)a * t.nodes + i) * t.words;
                            if (lead >= 0) {
                                const int w = lead >> 6, by = lead & 63;
                                drafts = w < t.words ? (uint32_t)(row_mask[w] >> by) : 0u;
                                if (by > 32 && w + 1 < t.words) drafts |= (uint32_t)(row_mask[w + 1] << (64 - by));
                            } else {
                                drafts = (uint32_t)row_mask[0] << -lead;
                            }
                        }
                        if (lead < 0) drafts |= (1u << -lead) - 1;   // the tokens before the drafts
                        seen &= drafts;
                    }
                    if (seen & bad) poison[nt] = NAN;
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (!((seen >> (8 * (k >> 2) + 4 * h + (k & 3))) & 1)) s[nt][k] = -INFINITY;
                }
            }

            // ---- probabilities; the row's reference moves only when a score is far above it
            tree_uint4 p[NT][2], p_low[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float top = s[nt][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) top = fmaxf(top, s[nt][i]);
                top = other_half_max(top) * t.qscale;
                if (__ballot(top > m[nt] + kRaise)) {
                    const float m_new = fmaxf(m[nt], top);
                    const float f = m[nt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[nt] - m_new);
                    m[nt] = m_new;
                    l[nt] *= f;
#pragma unroll
                    for (int e = 0; e < MG; ++e) acc[nt][e] *= f;
                }
                const float ref = m[nt] == -INFINITY ? 0.0f : m[nt];   // (a row that has seen nothing yet: weights 0)
                float pr[16], sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    pr[i] = __builtin_amdgcn_exp2f(fmaf(s[nt][i], t.qscale, -ref));
                    sum += pr[i];
                }
                l[nt] += sum;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t w = pack2<BF>(pr[2 * i], pr[2 * i + 1]);
                    p[nt][i >> 2][i & 3] = w;
                    if constexpr (BF)   // what bfloat16's eight bits leave out, as a second term
                        p_low[nt][i >> 2][i & 3] = pack2<BF>(pr[2 * i] - __uint_as_float(w << 16), pr[2 * i + 1] - __uint_as_float(w & 0xFFFF0000u));
                }
            }

            // ---- values
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int e = 0; e < MG; ++e) {
                    tree_uint4 av;
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        av[y] = __builtin_amdgcn_perm(x.v[8 * half + 2 * y + 1][e >> 1], x.v[8 * half + 2 * y][e >> 1],
                                                      e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        acc[nt][e] = tree_mfma<BF>(av, p[nt][half], acc[nt][e]);
                        if constexpr (BF) acc[nt][e] = tree_mfma<BF>(av, p_low[nt][half], acc[nt][e]);
                    }
                }
            if (more) load_values(next_row);
            row = next_row;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) l[nt] += poison[nt];
    }

    // ---- the waves' shares
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = 32 * nt + n;
        const float sum = other_half_sum(l[nt]);
        if (h == 0) m_s[wave][r] = m[nt], l_s[wave][r] = sum;
        float* dst = o_s + (wave * ROWS + r) * OSTRIDE;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int c = 0; c < MG; ++c) {   // coordinates MG (8 q + 4 h) + 4 c ..: accumulator 4 q + j of block e is MG j + e
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = acc[nt][(4 * c + i) % MG][4 * q + (4 * c + i) / MG];
                *reinterpret_cast<float4*>(dst + MG * (8 * q + 4 * h) + 4 * c) = make_float4(y[0], y[1], y[2], y[3]);
            }
    }
    __syncthreads();

    constexpr int TPR = 256 / ROWS, CPT = D / (4 * TPR);   // threads of a row, its groups of four coordinates per thread
    const int rr = tid / TPR, part = tid % TPR, r = row0 + rr;
    float M = m_s[0][rr];
#pragma unroll
    for (int w = 1; w < 4; ++w) M = fmaxf(M, m_s[w][rr]);
    float f[4], L = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        f[w] = m_s[w][rr] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_s[w][rr] - M);
        L += l_s[w][rr] * f[w];
    }
    if (r >= t.rows) return;
    const bool none = M == -INFINITY && L == 0.0f;   // the row has seen no token
    const float inv = L != 0.0f ? 1.0f / L : 0.0f;
    const size_t R = (size_t)v.A * t.rows, prow = ((size_t)usel * t.nsplit + split) * R + (size_t)a * t.rows + r;
    int in_group;
    const int i = t.div_G.divide(r, &in_group);
    const size_t orow = (((size_t)ls * v.A + a) * t.nodes + i) * t.q_heads + kvh * t.G + in_group;
#pragma unroll
    for (int c = 0; c < CPT; ++c) {
        const int at = 4 * (c * TPR + part);
        float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float4 z = *reinterpret_cast<const float4*>(o_s + (w * ROWS + rr) * OSTRIDE + at);
            y[0] = fmaf(z.x, f[w], y[0]), y[1] = fmaf(z.y, f[w], y[1]), y[2] = fmaf(z.z, f[w], y[2]), y[3] = fmaf(z.w, f[w], y[3]);
        }
        if (g.out != nullptr)
            *reinterpret_cast<uint2*>(g.out + orow * D + at) = make_uint2(pack2<BF>(y[0] * inv, y[1] * inv), pack2<BF>(y[2] * inv, y[3] * inv));
        else if (!none)
            *reinterpret_cast<float4*>(g.o + prow * D + at) = make_float4(y[0], y[1], y[2], y[3]);
    }
    if (g.out == nullptr && part == 0) *reinterpret_cast<float2*>(g.ml + prow * 2) = make_float2(M, L);
}

// -------------------------------------------------------------------------------------- merge ---
// One wave per row.  The pool's partials are added in the rotated domain and rotated back, the pages' join behind that.
template <int D, bool BF>
__global__ __launch_bounds__(256) void tree_merge_kernel(AttendPlan p, int nsplit, int page_nsplit, const float* __restrict__ pool_ml,
                                                         const float* __restrict__ pool_o, const float* __restrict__ ml,
                                                         const float* __restrict__ o, uint16_t* __restrict__ out) {
    constexpr int EPL = D / 64;
    const int lane = threadIdx.x & 63;
    const long row_global = ((long)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6), nrows = (long)p.layers * p.H * p.R;
    const bool active = row_global < nrows;   // no early return: the butterflies need the whole wave
    const long rg = active ? row_global : 0;
    const int usel = (int)(rg / p.R), r = (int)(rg - (long)usel * p.R);
    int kvh;
    const int ls = p.div_H.divide(usel, &kvh);
    // (m, l) of a partial, from every lane: the numbers are the same for the whole wave
    auto pool_at = [&](int s) { return *reinterpret_cast<const float2*>(pool_ml + (((size_t)usel * nsplit + s) * p.R + r) * 2); };
    auto page_at = [&](int s) { return *reinterpret_cast<const float2*>(ml + (((size_t)usel * page_nsplit + s) * p.R + r) * 2); };
    float M = -INFINITY;
    for (int s = 0; s < nsplit; ++s) M = fmaxf(M, pool_at(s).x);
    for (int s = 0; s < page_nsplit; ++s) M = fmaxf(M, page_at(s).x);
    float x[EPL], L = 0.0f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = 0.0f;
    for (int s = 0; s < nsplit; ++s) {
        const float2 part = pool_at(s);
        const float w = part.x == -INFINITY ? 0.0f : exp2f(part.x - M);
        L = fmaf(part.y, w, L);
#pragma unroll
        for (int i = 0; i < EPL; ++i) x[i] = fmaf(pool_o[(((size_t)usel * nsplit + s) * p.R + r) * D + lane * EPL + i], w, x[i]);
    }
    if (nsplit > 0 && p.vcodec != POLYKV_VALUES_INT8) {   // (int8 values were never rotated)
        wht_inlane<EPL>(x);
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            x[i] = wht_lane_stage<1>(x[i], lane);
            x[i] = wht_lane_stage<2>(x[i], lane);
            x[i] = wht_lane_stage<4>(x[i], lane);
            x[i] = wht_lane_stage<8>(x[i], lane);
            x[i] = wht_lane_stage<16>(x[i], lane);
            x[i] = wht_lane_stage<32>(x[i], lane);
            x[i] *= (D == 64 ? 0.125f : D == 128 ? 0.08838834764831845f : 0.0625f);
        }
        if (p.signs.on) flip_signs<EPL>(x, sign_word(p.signs, (lane * EPL) >> 5) >> ((lane * EPL) & 31));
    }
    for (int s = 0; s < page_nsplit; ++s) {
        const float2 part = page_at(s);
        if (part.x == -INFINITY && part.y == 0.0f) continue;   // no token: its sums were not written
        const float w = exp2f(part.x - M);
        L = fmaf(part.y, w, L);
#pragma unroll
        for (int i = 0; i < EPL; ++i) x[i] = fmaf(o[(((size_t)usel * page_nsplit + s) * p.R + r) * D + lane * EPL + i], w, x[i]);
    }
    const float inv = L != 0.0f ? 1.0f / L : 0.0f;
    if (active) {
        uint16_t* dst = out + q_row_index(p, ls, kvh, r) * D + lane * EPL;
        if constexpr (EPL == 1) {
            *dst = (uint16_t)pack2<BF>(x[0] * inv, 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < EPL; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = pack2<BF>(x[i] * inv, x[i + 1] * inv);
        }
    }
}

// ----------------------------------------------------------------------------------- launchers ---
void plan_tree(const PageView& v, int page_splits, TreePlan* t) {
    t->row_tiles = t->rows > 32 && v.D != 256 ? 2 : 1;
    t->row_blocks = (t->rows + 32 * t->row_tiles - 1) / (32 * t->row_tiles);
    // Token ranges: workgroups for 512 places, as far as each of a workgroup's four waves keeps two tiles of the longest
    // continuation there can be.
    const long groups = (long)t->layers * v.H * v.A * t->row_blocks, tiles = ((long)v.max_blocks * v.P + 31) / 32;
    long want = page_splits > 0 ? page_splits : (512 + groups - 1) / groups;
    const long most = page_splits > 0 ? (tiles + 3) / 4 : tiles / 8;
    if (want > most) want = most;
    if (want < 1) want = 1;
    t->nsplit = (int)want;
    t->div_H = FastDiv::by(v.H);
    t->div_A = FastDiv::by(v.A);
    t->div_G = FastDiv::by(t->G);
    t->div_nsplit = FastDiv::by(t->nsplit);
    t->div_row_blocks = FastDiv::by(t->row_blocks);
}

// A grid dimension holds 16.7 million workgroups; beyond 2^23 of them the launch gets a second dimension.
static dim3 grid_of(uint64_t workgroups) {
    const uint64_t most = 1u << 23;
    return workgroups <= most ? dim3((uint32_t)workgroups) : dim3((uint32_t)most, (uint32_t)((workgroups + most - 1) / most));
}

template <int D, bool BF, int NT>
static hipError_t launch_pages_one(const TreeArgs& g, dim3 grid, bool main_kernel, hipStream_t s) {
    constexpr int kShared = 4 * 32 * NT * (D + 4) * (int)sizeof(float);
    const auto kern = attend_pages_kernel<D, BF, NT>;
    static std::once_flag configured;
    static hipError_t config_result = hipSuccess;
    std::call_once(configured, [&]() {
        config_result = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kShared);
    });
    if (config_result != hipSuccess) return config_result;
    launch_kernel(kern, grid, dim3(256), kShared, s, main_kernel ? take_kernel_events() : KernelEvents{}, g);
    return hipGetLastError();
}

hipError_t launch_attend_pages(const PageView& v, const TreePlan& t, bool bf16, const void* Q, float* ml, float* o, void* out,
                               bool main_kernel, hipStream_t s) {
    const TreeArgs g = {v, t, (const uint16_t*)Q, ml, o, (uint16_t*)out};
    const uint64_t streams = (uint64_t)t.layers * v.H * v.A * t.nsplit;
    const dim3 grid = grid_of((streams + 7) / 8 * 8 * t.row_blocks);
    if (v.D == 64) {
        if (t.row_tiles == 2) return bf16 ? launch_pages_one<64, true, 2>(g, grid, main_kernel, s) : launch_pages_one<64, false, 2>(g, grid, main_kernel, s);
        return bf16 ? launch_pages_one<64, true, 1>(g, grid, main_kernel, s) : launch_pages_one<64, false, 1>(g, grid, main_kernel, s);
    }
    if (v.D == 128) {
        if (t.row_tiles == 2) return bf16 ? launch_pages_one<128, true, 2>(g, grid, main_kernel, s) : launch_pages_one<128, false, 2>(g, grid, main_kernel, s);
        return bf16 ? launch_pages_one<128, true, 1>(g, grid, main_kernel, s) : launch_pages_one<128, false, 1>(g, grid, main_kernel, s);
    }
    return bf16 ? launch_pages_one<256, true, 1>(g, grid, main_kernel, s) : launch_pages_one<256, false, 1>(g, grid, main_kernel, s);
}

hipError_t launch_tree_merge(const AttendPlan& plan, const TreePlan& t, bool has_pool, const float* pool_ml, const float* pool_o,
                             const float* ml, const float* o, void* out, hipStream_t s) {
    const long nrows = (long)plan.layers * plan.H * plan.R;
    using Kern = decltype(&tree_merge_kernel<64, false>);
    static const Kern table[3][2] = {{tree_merge_kernel<64, false>, tree_merge_kernel<64, true>},
                                     {tree_merge_kernel<128, false>, tree_merge_kernel<128, true>},
                                     {tree_merge_kernel<256, false>, tree_merge_kernel<256, true>}};
    launch_kernel(table[plan.D == 64 ? 0 : plan.D == 128 ? 1 : 2][plan.io_bf16 ? 1 : 0], grid_of((uint64_t)(nrows + 3) / 4), dim3(256), 0, s, {},
                  plan, has_pool ? plan.nsplit : 0, t.nsplit, pool_ml, pool_o, ml, o, (uint16_t*)out);
    return hipGetLastError();
}

}  // namespace polykv
