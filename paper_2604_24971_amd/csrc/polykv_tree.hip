// Attention of drafted tokens over their agent's continuation in pages, and its join with the pool's part (gfx950).
//
// For the rows of one agent and KV head (drafts x query heads of the group) and the tokens t that a row sees,
//   m = max s(t),  l = sum 2^(s(t) - m),  o = sum 2^(s(t) - m) v(t),   s(t) = q . k(t) * scale * log2 e
// over one pass through the tokens: a partial (m, l, o) per row.  Partials of token ranges, and the pool's (whose o is in the
// rotated value domain), join with weights 2^(m - M); the output is o / l.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <algorithm>
#include <type_traits>

#include "polykv_layout.hpp"
#include "polykv_pages.hpp"

namespace polykv {

typedef _Float16 tree_half8 __attribute__((ext_vector_type(8)));
typedef _Float16 tree_half2 __attribute__((ext_vector_type(2)));
typedef __bf16 tree_bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 tree_bf2 __attribute__((ext_vector_type(2)));
typedef float tree_float2 __attribute__((ext_vector_type(2)));
typedef float tree_float4 __attribute__((ext_vector_type(4)));
typedef float tree_float16 __attribute__((ext_vector_type(16)));
typedef uint32_t tree_uint4 __attribute__((ext_vector_type(4)));

// Products of R x R blocks, R = 32 over 16 elements or 16 over 32.
template <int R> struct Block;
template <> struct Block<32> {
    using Acc = tree_float16;
};
template <> struct Block<16> {
    using Acc = tree_float4;
};
template <bool BF, int R>
__device__ __forceinline__ typename Block<R>::Acc tree_mfma(const tree_uint4& a, const tree_uint4& b, const typename Block<R>::Acc& c) {
    if constexpr (BF) {
        const tree_bf8 x = __builtin_bit_cast(tree_bf8, a), y = __builtin_bit_cast(tree_bf8, b);
        if constexpr (R == 32) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
    } else {
        const tree_half8 x = __builtin_bit_cast(tree_half8, a), y = __builtin_bit_cast(tree_half8, b);
        if constexpr (R == 32) return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
    }
}
template <bool BF> __device__ __forceinline__ uint32_t pack2(float x, float y) {   // to nearest even
    const tree_float2 f = {x, y};
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, tree_bf2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, tree_half2));
}
// x of lanes with the bit STEP (32 or 16) clear and set, from every lane of the pair.
template <int STEP> __device__ __forceinline__ float2 both_lanes(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto r = STEP == 32 ? __builtin_amdgcn_permlane32_swap(u, u, false, false) : __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Over the lanes of a row, lane % R.
template <int R> __device__ __forceinline__ float row_max(float x) {
    float2 b = both_lanes<32>(x);
    x = fmaxf(b.x, b.y);
    if constexpr (R == 16) {
        b = both_lanes<16>(x);
        x = fmaxf(b.x, b.y);
    }
    return x;
}
template <int R> __device__ __forceinline__ float row_sum(float x) {
    float2 b = both_lanes<32>(x);
    x = b.x + b.y;
    if constexpr (R == 16) {
        b = both_lanes<16>(x);
        x = b.x + b.y;
    }
    return x;
}
// Sixteen lanes read 8 bytes each, [4][16] numbers of 16 bits (lanes 4 j .. 4 j + 3: row j), and get a column each.
__device__ __forceinline__ uint2 lds_transposed(uint16_t* p) {
    typedef short short4v __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)p));
}
// Whether one of the two 16-bit numbers is infinite or NaN.
template <bool BF> __device__ __forceinline__ bool any_nonfinite(uint32_t w) {
    constexpr uint32_t exponents = BF ? 0x7F807F80u : 0x7C007C00u, one = BF ? 0x00800080u : 0x04000400u;
    return (((w & exponents) + one) & 0x80008000u) != 0;
}

struct TreeArgs {
    PageView v;
    TreePlan t;
    const uint16_t* Q;
    float *ml, *o;   // where partials go
    uint16_t* out;   // not nullptr: the rows are completed here, with the pool's partials if there are any
    PoolPart pool;
};

// Both kernels below work on 32-token tiles, a wave on R = 32 or 16 query rows.  Tokens are the M dimension of the score products
// and the K dimension of the value products, rows the N dimension of both, so that a lane (n = lane % R, g = lane / R) has row n
// throughout, and its probabilities leave the score accumulators in the order in which they enter the value products: score i
// of a lane belongs to token token_of(i).
//   keys    lane (n, g) holds pieces of 8 elements of tokens n (and, with R = 16, 16 + n);
//   values  value block e of the products has coordinates of its own in its rows m = 4 LPR q + 4 g + j (accumulator 4 q + j).
template <int D, int R> struct Shape {
    static constexpr int LPR = 64 / R;             // lanes of a row
    static constexpr int KJ = D / (8 * LPR);       // pieces of a token's key in a lane
    static constexpr int TT = 32 / R;              // score blocks of a tile
    static constexpr int SN = R / 2;               // scores of a lane
    static constexpr int PARTS = SN / 8;           // value products over a tile's tokens
    static constexpr int MG = D / R;               // value blocks
    static constexpr int AN = R * R / 64;          // accumulators of a block in a lane
    __device__ static constexpr int token_of(int i) { return 4 * LPR * (i >> 2) + (i & 3); }   // + 4 g
};

// Where a workgroup is: which agent, KV head, rows and tiles.
struct Place {
    int a, usel, ls, kvh, split, row_block;
    int length, before, count;   // the agent's tokens, those before its drafts, its drafts
    bool inside;                 // (the grid is rounded up)
};
__device__ __forceinline__ Place place_of(const TreeArgs& g) {
    const TreePlan& t = g.t;
    Place p;
    // Workgroup -> (token range of an agent and KV head, row block).  Consecutive workgroups go to the eight dies in turn: the row
    // blocks of a token range follow each other on one die, whose L2 they share.
    const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x;
    const int stream = t.div_row_blocks.divide((int)(block >> 3), &p.row_block) * 8 + (int)(block & 7);
    p.inside = stream < t.layers * g.v.H * g.v.A * t.nsplit;
    const int ua = t.div_nsplit.divide(stream, &p.split);
    p.usel = t.div_A.divide(ua, &p.a);
    p.ls = t.div_H.divide(p.usel, &p.kvh);
    if (p.inside) {
        p.length = tokens_of(g.v, p.a);
        p.count = drafts_of(t.counts, p.a, t.nodes, p.length);
        p.before = p.length - p.count;
    }
    return p;
}

// The queries of a wave's rows from row0 on in operand order (rows past the last repeat it), and the draft of the lane's row.
template <int D, int R> __device__ __forceinline__ int load_queries(const TreeArgs& g, const Place& p, int row0, int lane, tree_uint4 (&q)[Shape<D, R>::KJ]) {
    const TreePlan& t = g.t;
    constexpr int LPR = 64 / R;
    int in_group;
    const int draft = t.div_G.divide(min(row0 + lane % R, t.rows - 1), &in_group);
    const uint16_t* src = g.Q + ((((size_t)p.ls * g.v.A + p.a) * t.nodes + draft) * t.q_heads + p.kvh * t.G + in_group) * D + 8 * (lane / R);
#pragma unroll
    for (int j = 0; j < Shape<D, R>::KJ; ++j) q[j] = *reinterpret_cast<const tree_uint4*>(src + 8 * LPR * j);
    return draft;
}
// Ahead of a loop: otherwise its first product waits for the queries in every round, and with them for all that has been requested
// for the rounds to come.
template <int N> __device__ __forceinline__ void wait_for(tree_uint4 (&q)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+v"(q[j]));
}

// What the lane's draft sees of the drafts: bits of the first 64 of them, requested ahead of the tiles (most trees have no more).
__device__ __forceinline__ uint64_t first_drafts(const TreePlan& t, const Place& p, int draft) {
    if (t.mask == nullptr) return draft >= 63 ? ~0ull : (2ull << draft) - 1;   // drafts 0 .. draft
    return t.mask[((size_t)p.a * t.nodes + draft) * t.words];
}
// Bit t: draft `draft`'s rows see token t0 + t, among the tile's tokens `there`.
__device__ __forceinline__ uint32_t seen_tokens(const TreePlan& t, const Place& p, int draft, uint64_t first, int t0, uint32_t there) {
    if (draft >= p.count) return 0;
    const int lead = t0 - p.before;   // the tile's first token as a draft
    if (lead + 32 <= 0) return there;
    uint32_t drafts;
    if (lead <= 0) {
        drafts = (uint32_t)first << -lead | ((1u << -lead) - 1);   // with the tokens before the drafts
    } else {
        const int w = lead >> 6, by = lead & 63;
        auto word = [&](int i) -> uint64_t {
            if (i == 0) return first;
            if (t.mask == nullptr) return draft >= 64 * i + 63 ? ~0ull : draft >= 64 * i ? (2ull << (draft - 64 * i)) - 1 : 0ull;
            return i < t.words ? t.mask[((size_t)p.a * t.nodes + draft) * t.words + i] : 0ull;
        };
        drafts = (uint32_t)(word(w) >> by);
        if (by > 32) drafts |= (uint32_t)(word(w + 1) << (64 - by));
    }
    return drafts & there;
}

// The scores of a lane.
template <int R> struct Scores {
    typename Block<R>::Acc t[32 / R];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int u = 0; u < 32 / R; ++u)
#pragma unroll
            for (int i = 0; i < R * R / 64; ++i) t[u][i] = 0.0f;
    }
    __device__ __forceinline__ float get(int i) const { return R == 32 ? t[0][i] : t[i >> 2 & (32 / R - 1)][i & 3]; }
    __device__ __forceinline__ void set(int i, float x) {
        if constexpr (R == 32) t[0][i] = x;
        else t[i >> 2][i & 3] = x;
    }
};
template <int D, int R> __device__ __forceinline__ void hide_unseen(Scores<R>& s, uint32_t seen, int g) {
    seen >>= 4 * g;
#pragma unroll
    for (int i = 0; i < Shape<D, R>::SN; ++i)
        if (!((seen >> Shape<D, R>::token_of(i)) & 1)) s.set(i, -INFINITY);
}

// A wave's rows: reference (of the scores in base-2 units), sum and value sums, all relative to the reference.  The reference is
// the maximum of the first tokens that the row sees; it moves when a tile's probabilities sum to more than 2^15 in a lane, a test on
// a sum that is needed anyway, so most tiles go without maxima.
template <int D, int R> struct Rows {
    typename Block<R>::Acc acc[D / R];
    float m, l;

    __device__ __forceinline__ void clear() {
        m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int e = 0; e < D / R; ++e)
#pragma unroll
            for (int i = 0; i < R * R / 64; ++i) acc[e][i] = 0.0f;
    }
};

// Scores -> probabilities in the pages' type, in operand order.  fp16: one term, whose rounding (half a step, 2^-11 of a weight, 2^-25
// below the normal range) is as fine as the output's own; the denominator sums the rounded weights, so that what a weight loses
// it loses on both sides of the fraction (errors 2.7e-4 of the output's rms, 2.1e-4 with weights in fp32; a second term would
// double the value products).  bfloat16's eight bits leave too much out: a second term holds it.
template <bool BF, int R> struct Weights {
    tree_uint4 p[R / 16], low[BF ? R / 16 : 1];
};
template <int D, bool BF, int R> __device__ __forceinline__ Weights<BF, R> weigh(Rows<D, R>& r, const Scores<R>& s, float qscale) {
    constexpr int SN = Shape<D, R>::SN;
    Weights<BF, R> w;
    float sum = 0.0f;
    bool raise = __ballot(r.m == -INFINITY) != 0;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {   // (one copy of the code for both passes: two cost the accumulators' registers)
        if (raise) {
            float top = s.get(0);
            asm volatile("" : "+v"(top));   // (or the maxima are taken for every tile, ahead of the loop)
#pragma unroll
            for (int i = 1; i < SN; ++i) top = fmaxf(top, s.get(i));
            const float m_new = fmaxf(r.m, row_max<R>(top) * qscale);
            const float f = r.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(r.m - m_new);
            r.m = m_new;
            r.l *= f;
#pragma unroll
            for (int e = 0; e < D / R; ++e) r.acc[e] *= f;
        }
        const float ref = r.m == -INFINITY ? 0.0f : r.m;   // (a row that has seen nothing yet: weights 0)
        float x[SN];
#pragma unroll
        for (int i = 0; i < SN; ++i) x[i] = fmaf(s.get(i), qscale, -ref);
        if (__ballot(fabsf(ref) > 65536.0f)) {   // the product's own rounding is more than 2^-8: rounded as it was for the reference
            float by = qscale;
            asm volatile("" : "+v"(by));   // (likewise)
#pragma unroll
            for (int i = 0; i < SN; ++i) x[i] = __fsub_rn(__fmul_rn(s.get(i), by), ref);
        }
#pragma unroll
        for (int i = 0; i < SN; ++i) x[i] = __builtin_amdgcn_exp2f(x[i]);
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < SN / 2; ++i) {
            const uint32_t two = pack2<BF>(x[2 * i], x[2 * i + 1]);
            w.p[i >> 2][i & 3] = two;
            if constexpr (BF) {
                w.low[i >> 2][i & 3] = pack2<BF>(x[2 * i] - __uint_as_float(two << 16), x[2 * i + 1] - __uint_as_float(two & 0xFFFF0000u));
                sum += x[2 * i] + x[2 * i + 1];
            } else {   // (the rounded ones: two at a time)
                const tree_half2 ones = {(_Float16)1.0f, (_Float16)1.0f};
                sum = __builtin_amdgcn_fdot2(__builtin_bit_cast(tree_half2, two), ones, sum, false);
            }
        }
        raise = __ballot(sum > 32768.0f) != 0;
        if (!raise) break;
    }
    r.l += sum;
    return w;
}

// Row r of the agent in Q and out, and among the partials.
__device__ __forceinline__ size_t out_row(const TreeArgs& g, const Place& p, int r) {
    int in_group;
    const int i = g.t.div_G.divide(r, &in_group);
    return (((size_t)p.ls * g.v.A + p.a) * g.t.nodes + i) * g.t.q_heads + p.kvh * g.t.G + in_group;
}
__device__ __forceinline__ size_t partial_row(const TreeArgs& g, const Place& p, int r) {
    return ((size_t)p.usel * g.t.nsplit + p.split) * ((size_t)g.v.A * g.t.rows) + (size_t)p.a * g.t.rows + r;
}

// Up to so many splits of the pool the pages' kernel joins itself; beyond it writes partials and the merge kernel joins all.  Measured,
// joined here and by the merge kernel: one layer of 15 agents with a row each, 16 splits 18.3 and 19.7 us a call; of 4 agents with 4 x 4
// rows, 16 splits, 18.5 and 20.1; of one agent with 70 rows, 42 splits, 29 and 18.
constexpr int kJoinSplits = 16;

constexpr float kRotation(int D) { return D == 64 ? 0.125f : D == 128 ? 0.08838834764831845f : 0.0625f; }

// The pool's partials of a row: maxima and sums of its splits.  The first two are requested ahead of everything else (at head_dim
// 256, whose registers are full, none are).
template <int D> struct PoolSums {
    static constexpr bool AHEAD = D != 256;
    float m0, l0, m1, l1;

    __device__ static __forceinline__ size_t row(const TreeArgs& g, const Place& p, int r, int s) {   // among the partials
        return ((size_t)p.usel * g.pool.nsplit + s) * ((size_t)g.v.A * g.t.rows) + (size_t)p.a * g.t.rows + min(r, g.t.rows - 1);
    }
    __device__ __forceinline__ void request(const TreeArgs& g, const Place& p, int r) {
        m0 = l0 = m1 = l1 = 0.0f;
        if (AHEAD && g.pool.ml != nullptr && g.out != nullptr) {
            const float2 a = load(g, p, r, 0), b = load(g, p, r, min(1, g.pool.nsplit - 1));
            m0 = a.x, l0 = a.y, m1 = b.x, l1 = b.y;
        }
    }
    __device__ static __forceinline__ float2 load(const TreeArgs& g, const Place& p, int r, int s) {
        return *reinterpret_cast<const float2*>(g.pool.ml + row(g, p, r, s) * 2);
    }
    __device__ __forceinline__ void all(const TreeArgs& g, const Place& p, int r, float* M, float* L) const {
        *M = -INFINITY, *L = 0.0f;
        auto take = [&](auto& x, float top) {
            if (top == -INFINITY) return;   // (empty splits so far; the pool is not empty)
            *L *= __builtin_amdgcn_exp2f(*M - top);
            *M = top;
#pragma unroll
            for (const float2& y : x) *L = fmaf(y.y, __builtin_amdgcn_exp2f(y.x - top), *L);
        };
        if (AHEAD) {
            const float2 x[2] = {make_float2(m0, l0), g.pool.nsplit > 1 ? make_float2(m1, l1) : make_float2(-INFINITY, 0.0f)};
            take(x, fmaxf(x[0].x, x[1].x));
        }
        constexpr int B = AHEAD ? 8 : 4;   // are requested before the first is used
#pragma unroll 1
        for (int s0 = AHEAD ? 2 : 0; s0 < g.pool.nsplit; s0 += B) {
            float2 x[B];
            float top = *M;
#pragma unroll
            for (int k = 0; k < B; ++k) x[k] = s0 + k < g.pool.nsplit ? load(g, p, r, s0 + k) : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int k = 0; k < B; ++k) top = fmaxf(top, x[k].x);
            take(x, top);
        }
    }
    // d += the value sums of a row's splits, each times 2^(m - M) * scale; coordinates base + at(i) .. + 3 in d[4 i] .. d[4 i + 3].
    template <int N, class At> __device__ static __forceinline__ void add(const TreeArgs& g, const Place& p, int r, float M, float scale, float (&d)[N], At at) {
        constexpr int PIECE = N < 128 ? N / 4 : N / 8;   // (as far as the registers reach: all of 128 took 68 bytes of scratch a lane)
        auto splits = [&](int s0, auto count) {   // all of a piece are requested before the first is used
            constexpr int B = decltype(count)::value;
#pragma unroll
            for (int i0 = 0; i0 < N / 4; i0 += PIECE) {
                float4 z[B][PIECE];
                float w[B];
#pragma unroll
                for (int k = 0; k < B; ++k) {
                    w[k] = load(g, p, r, s0 + k).x;
                    const float* src = g.pool.o + row(g, p, r, s0 + k) * D;
#pragma unroll
                    for (int i = 0; i < PIECE; ++i) z[k][i] = *reinterpret_cast<const float4*>(src + at(i0 + i));
                }
#pragma unroll
                for (int k = 0; k < B; ++k) {
                    const float f = __builtin_amdgcn_exp2f(w[k] - M) * scale;
#pragma unroll
                    for (int i = 0; i < PIECE; ++i) {
                        float* y = d + 4 * (i0 + i);
                        y[0] = fmaf(z[k][i].x, f, y[0]), y[1] = fmaf(z[k][i].y, f, y[1]), y[2] = fmaf(z[k][i].z, f, y[2]), y[3] = fmaf(z[k][i].w, f, y[3]);
                    }
                }
            }
        };
        int s0 = 0;
        if constexpr (N < 64)   // (as far as the registers reach)
            for (; s0 + 1 < g.pool.nsplit; s0 += 2) splits(s0, std::integral_constant<int, 2>());
        for (; s0 < g.pool.nsplit; ++s0) splits(s0, std::integral_constant<int, 1>());
    }
};

// A wave's rows straight from the registers: partials, or, completed with the pool's, the output.
// A lane has runs of consecutive coordinates of its row, the row's lanes in turn, so the inverse rotation of the pool's part is an
// exchange with each of the row's other lanes and butterflies between registers.
//   permuted operands    block e has coordinates MG m + e: R / (4 LPR) runs of 4 MG, run k from MG (4 LPR k + 4 g)
//   transposed operands  block e has coordinates R e + m: D / (4 LPR) runs of 4, run k from 4 LPR k + 4 g
template <int D, bool BF, int R, bool TR>
__device__ __forceinline__ void store_rows(const TreeArgs& g, const Place& p, const Rows<D, R>& x, const PoolSums<D>& pool, int row0, int lane) {
    constexpr int MG = D / R, LPR = 64 / R, C = TR ? 4 : 4 * MG, RUNS = D / (LPR * C), PER = R / (4 * LPR);   // PER: runs of a block
    const int h = lane / R, r = row0 + lane % R;
    auto first = [&](int k) { return C * (LPR * k + h); };
    float sum = row_sum<R>(x.l);
    const bool any = sum != 0.0f;   // the row has seen a token (its sum is then about 1 at the least)
    // (a row that has seen none may share its wave with rows that have seen values that are not finite)
    auto acc = [&](int k, int c) { return any ? TR ? x.acc[k / PER][4 * (k % PER) + c] : x.acc[c % MG][4 * k + c / MG] : 0.0f; };
    const float m = any ? x.m : -INFINITY;
    if (g.out == nullptr) {
        if (r >= g.t.rows) return;
        const size_t prow = partial_row(g, p, r);
        if (any) {   // (else nobody reads its sums)
#pragma unroll
            for (int k = 0; k < RUNS; ++k)
#pragma unroll
                for (int c = 0; c < C; c += 4)
                    *reinterpret_cast<float4*>(g.o + prow * D + first(k) + c) = make_float4(acc(k, c), acc(k, c + 1), acc(k, c + 2), acc(k, c + 3));
        }
        if (h == 0) *reinterpret_cast<float2*>(g.ml + prow * 2) = make_float2(m, sum);
        return;
    }
    constexpr int N = D / LPR;   // coordinates of a lane
    float y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = 0.0f;
    float weight = 1.0f;
    if (g.pool.ml != nullptr) {
        float M, L;
        pool.all(g, p, r, &M, &L);
        const float top = fmaxf(M, m), scale = g.pool.rotated ? kRotation(D) : 1.0f;
        pool.add(g, p, r, top, scale, y, [&](int i) { return first(4 * i / C) + 4 * i % C; });
        if (g.pool.rotated) {
            wht_inlane<N>(y);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float2 b = both_lanes<32>(y[i]);
                y[i] = lane & 32 ? b.x - b.y : b.x + b.y;
                if constexpr (R == 16) {
                    b = both_lanes<16>(y[i]);
                    y[i] = lane & 16 ? b.x - b.y : b.x + b.y;
                }
            }
            if (g.pool.signs.on) {
                constexpr int W = C < 32 ? C : 32;   // coordinates of one word of signs
#pragma unroll
                for (int k = 0; k < RUNS; ++k)
#pragma unroll
                    for (int c = 0; c < C; c += W)
                        flip_signs<W>(*reinterpret_cast<float(*)[W]>(y + C * k + c), sign_word(g.pool.signs, (first(k) + c) >> 5) >> ((first(k) + c) & 31));
            }
        }
        weight = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top);
        sum = fmaf(sum, weight, L * __builtin_amdgcn_exp2f(M - top));
    }
    if (r >= g.t.rows) return;
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
    uint16_t* const dst = g.out + out_row(g, p, r) * D;
#pragma unroll
    for (int k = 0; k < RUNS; ++k) {
        uint32_t z[C / 2];
#pragma unroll
        for (int c = 0; c < C; c += 2)
            z[c / 2] = pack2<BF>(fmaf(acc(k, c), weight, y[C * k + c]) * inv, fmaf(acc(k, c + 1), weight, y[C * k + c + 1]) * inv);
        if constexpr (TR) {
            *reinterpret_cast<uint2*>(dst + first(k)) = make_uint2(z[0], z[1]);
        } else {
#pragma unroll
            for (int c = 0; c < C; c += 8)
                *reinterpret_cast<uint4*>(dst + first(k) + c) = make_uint4(z[c / 2], z[c / 2 + 1], z[c / 2 + 2], z[c / 2 + 3]);
        }
    }
}

// ---------------------------------------------------------------------------- few rows a head ---
// A wave's keys and values come straight from the pages into registers.  The tile's page numbers are requested two tiles ahead, its
// keys when the scores of the tile before are done, its values when that tile's value products are.  A lane loads MG coordinates
// of the tokens that its scores belong to and makes operands (eight tokens of one coordinate) of them by byte permutes.
// SHARE: the four waves of a workgroup take every fourth tile and are joined through LDS; otherwise a workgroup is one wave.
// Bound by memory where there are many agents and heads: 24 layers x 32 heads x 100 agents, one row over 61 to 121 tokens each (head_dim
// 64), 1.84 GB in 312 us, 5.9 TB/s; 32 layers x 8 heads x 15 agents, 32 rows over 210 to 308 tokens (bfloat16, head_dim 128), 0.64 GB with
// the pool's partials in 129 us, 4.9 TB/s.  By a wave's chain (queries, page, keys, two products, final pass) where there are few: one layer of
// 15 agents 9.2 us.
constexpr int few_waves_per_simd(int D, int R) { return R == 16 ? (D == 64 ? 4 : D == 128 ? 3 : 2) : D == 64 ? 3 : 2; }

template <int D, bool BF, int R, bool SHARE>
__global__ __launch_bounds__(SHARE ? 256 : 64, few_waves_per_simd(D, R)) void attend_pages_few_kernel(TreeArgs g) {
    using S = Shape<D, R>;
    constexpr int MG = S::MG, KJ = S::KJ, SN = S::SN, VW = MG / 2, OSTRIDE = D + 4, STEP = SHARE ? 4 : 1;
    // Head_dim 256: a tile's keys and values and the sums leave no registers for the queries, which wait in LDS (8 layers x 8 heads x 50
    // agents over 300 tokens 143 us, 161 with them in registers and 60 bytes a lane of addresses in scratch).  At 128 the bfloat16 form whose
    // four waves share sixteen rows lacks two registers (12 bytes of scratch, reloaded in every tile; times within 0.5 % either way).
    constexpr bool Q_LDS = D == 256 || (SHARE && BF && D == 128 && R == 16);
    __shared__ tree_uint4 q_own[Q_LDS && !SHARE ? KJ * 64 : 1];
    extern __shared__ __align__(16) float o_s[];   // [4][R][OSTRIDE] (SHARE)
    __shared__ float m_s[SHARE ? 4 : 1][R], l_s[SHARE ? 4 : 1][R];
    const PageView& v = g.v;
    const TreePlan& t = g.t;
    const int tid = threadIdx.x, lane = tid & 63, wave = SHARE ? __builtin_amdgcn_readfirstlane(tid >> 6) : 0;
    const int h = lane / R, n = lane % R;
    // (with SHARE where the wave's sums will be)
    tree_uint4* const q_s = (SHARE ? reinterpret_cast<tree_uint4*>(o_s + wave * R * OSTRIDE) : q_own) + lane;
    const Place pl = place_of(g);
    if (!pl.inside) return;
    const int row0 = pl.row_block * R;
    PoolSums<D> pool;
    pool.request(g, pl, row0 + (SHARE ? tid / (256 / R) : n));
    // the range's tiles; a block of rows that are all behind the agent's drafts sees none
    const int tiles = row0 < pl.count * t.G ? (pl.length + 31) >> 5 : 0;
    const int per_split = ((tiles + t.nsplit - 1) / t.nsplit + STEP - 1) & -STEP;
    const int t_begin = pl.split * per_split, t_end = min(tiles, t_begin + per_split), first = t_begin + wave;

    const size_t layer = (size_t)(t.layer_begin + pl.ls) * v.pages * v.H * v.P * D;
    const uint16_t* const Kb = v.K + layer;
    const uint16_t* const Vb = v.V + layer;
    const int32_t* const table = v.table + (size_t)pl.a * v.max_blocks;
    // lane l looks after token l % 32 of a tile: its page; its row among the layer's, -1 if it is not there
    auto page_at = [&](int tile) {
        int off;
        return table[v.div_P.divide(min(32 * tile + (lane & 31), pl.length - 1), &off)];
    };
    auto row_at = [&](int tile, int page) {
        int off;
        const int tok = 32 * tile + (lane & 31);
        (void)v.div_P.divide(tok, &off);
        return tok < pl.length && (uint32_t)page < (uint32_t)v.pages ? page_row(v, page, pl.kvh, off) : -1;
    };
    tree_uint4 k[S::TT][KJ];
    uint32_t x[SN][VW];
    auto load_keys = [&](int row) {
#pragma unroll
        for (int u = 0; u < S::TT; ++u) {
            const int r = R == 32 ? row : __shfl(row, 16 * u + n, 64);
            const uint16_t* src = Kb + (size_t)max(r, 0) * D + 8 * h;
#pragma unroll
            for (int j = 0; j < KJ; ++j) k[u][j] = *reinterpret_cast<const tree_uint4*>(src + 8 * S::LPR * j);
        }
    };
    auto load_values = [&](int row) {
#pragma unroll
        for (int q = 0; q < SN / 4; ++q) {   // four tokens at a time, which lie in one page
            const uint16_t* src = Vb + (size_t)max(__shfl(row, S::token_of(4 * q) + 4 * h, 64), 0) * D + MG * n;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t* at = reinterpret_cast<const uint32_t*>(src + e * D);
                if constexpr (VW == 1) {
                    x[4 * q + e][0] = at[0];
                } else if constexpr (VW == 2) {
                    const uint2 w = *reinterpret_cast<const uint2*>(at);
                    x[4 * q + e][0] = w.x, x[4 * q + e][1] = w.y;
                } else {
#pragma unroll
                    for (int c = 0; c < VW; c += 4) {
                        const tree_uint4 w = *reinterpret_cast<const tree_uint4*>(at + c);
                        x[4 * q + e][c] = w[0], x[4 * q + e][c + 1] = w[1], x[4 * q + e][c + 2] = w[2], x[4 * q + e][c + 3] = w[3];
                    }
                }
            }
        }
    };

    Rows<D, R> rows;
    rows.clear();
    if (first < t_end) {
        const int first_page = page_at(first);
        tree_uint4 q[KJ];
        const int draft = load_queries<D, R>(g, pl, row0, lane, q);
        const uint64_t see_first = first_drafts(t, pl, draft);
        int row = row_at(first, first_page);
        load_keys(row);
        load_values(row);
        int page = first + STEP < t_end ? page_at(first + STEP) : -1;
        wait_for(q);
        if constexpr (Q_LDS) {   // (each lane's own)
#pragma unroll
            for (int j = 0; j < KJ; ++j) q_s[64 * j] = q[j];
        }
        float poison = 0.0f;
        if (draft >= pl.count) rows.m = 0.0f;   // such a row never sees a token: any reference will do

        for (int tile = first; tile < t_end; tile += STEP) {
            Scores<R> s;
            s.clear();
            int at = 0;
            if constexpr (Q_LDS) asm volatile("" : "+v"(at));   // (or they are read ahead of the loop)
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                const tree_uint4 qj = Q_LDS ? q_s[64 * j + at] : q[j];
#pragma unroll
                for (int u = 0; u < S::TT; ++u) s.t[u] = tree_mfma<BF, R>(k[u][j], qj, s.t[u]);
            }
            const int t0 = 32 * tile;
            const uint32_t there = (uint32_t)__ballot(row >= 0);   // (lanes 32 .. 63 repeat the tile's tokens)
            const bool more = tile + STEP < t_end;
            int next_row = -1;
            if (more) {
                next_row = row_at(tile + STEP, page);
                load_keys(next_row);
                page = tile + 2 * STEP < t_end ? page_at(tile + 2 * STEP) : -1;
            }
            // ---- tokens that are not there, and drafts that the lane's draft does not see
            if (there != 0xFFFFFFFFu || t0 + 32 > pl.before || row0 + R > pl.count * t.G) {
                uint32_t bad = 0;   // drafts with a value that is not finite
                if (t0 + 32 > pl.before) {
#pragma unroll
                    for (int u = 0; u < SN; ++u) {
                        bool b = false;
#pragma unroll
                        for (int w = 0; w < VW; ++w) b |= any_nonfinite<BF>(x[u][w]);
                        const uint64_t lanes = __ballot(b);
#pragma unroll
                        for (int i = 0; i < S::LPR; ++i)
                            if (lanes >> (R * i) & ((1ull << R) - 1)) bad |= 1u << (S::token_of(u) + 4 * i);
                    }
                    bad &= there & ~(pl.before > t0 ? (1u << (pl.before - t0)) - 1 : 0u);
                }
                const uint32_t kept = there & ~bad;
                if (kept != 0xFFFFFFFFu) {   // their values are zeroed: a weight of 0 does not undo a NaN
#pragma unroll
                    for (int u = 0; u < SN; ++u) {
                        const bool keep = (kept >> (S::token_of(u) + 4 * h)) & 1;
#pragma unroll
                        for (int w = 0; w < VW; ++w) x[u][w] = keep ? x[u][w] : 0;
                    }
                }
                const uint32_t seen = seen_tokens(t, pl, draft, see_first, t0, there);
                if (seen & bad) poison = NAN;
                hide_unseen<D, R>(s, seen, h);
            }
            const Weights<BF, R> w = weigh<D, BF, R>(rows, s, t.qscale);
#pragma unroll
            for (int part = 0; part < S::PARTS; ++part)
#pragma unroll
                for (int e = 0; e < MG; ++e) {
                    tree_uint4 a;
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        a[y] = __builtin_amdgcn_perm(x[8 * part + 2 * y + 1][e >> 1], x[8 * part + 2 * y][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
                    rows.acc[e] = tree_mfma<BF, R>(a, w.p[part], rows.acc[e]);
                    if constexpr (BF) rows.acc[e] = tree_mfma<BF, R>(a, w.low[part], rows.acc[e]);
                }
            if (more) load_values(next_row);
            row = next_row;
        }
        rows.l += poison;
        if constexpr (Q_LDS) asm volatile("" ::: "memory");   // (the queries' place takes the sums)
    }
    if constexpr (!SHARE) {
        store_rows<D, BF, R, false>(g, pl, rows, pool, row0, lane);
    } else {
        // ---- the waves' shares
        const float sum = row_sum<R>(rows.l);
        const bool any = sum != 0.0f;   // (as in store_rows)
        if (h == 0) m_s[wave][n] = any ? rows.m : -INFINITY, l_s[wave][n] = sum;
        float* dst = o_s + (wave * R + n) * OSTRIDE;
#pragma unroll
        for (int q = 0; q < S::AN / 4; ++q)
#pragma unroll
            for (int c = 0; c < 4 * MG; c += 4) {
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = any ? rows.acc[(c + i) % MG][4 * q + (c + i) / MG] : 0.0f;
                *reinterpret_cast<float4*>(dst + 4 * MG * (S::LPR * q + h) + c) = make_float4(y[0], y[1], y[2], y[3]);
            }
        __syncthreads();
        // TPR threads of a row, each with groups of four coordinates in turn
        constexpr int TPR = 256 / R, CG = D / (4 * TPR);
        const int rr = tid / TPR, part = tid % TPR, r = row0 + rr;
        float M = m_s[0][rr];
#pragma unroll
        for (int w = 1; w < 4; ++w) M = fmaxf(M, m_s[w][rr]);
        float L = 0.0f, pool_M = -INFINITY, pool_L = 0.0f;
        const bool last = g.out != nullptr, with_pool = last && g.pool.ml != nullptr;
        if (with_pool) {
            pool.all(g, pl, r, &pool_M, &pool_L);
            M = fmaxf(M, pool_M);
        }
        float f[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = m_s[w][rr] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_s[w][rr] - M);
            L += l_s[w][rr] * f[w];
        }
        float y[4 * CG];
#pragma unroll
        for (int i = 0; i < 4 * CG; ++i) y[i] = 0.0f;
        if (with_pool) {
            pool.add(g, pl, r, M, g.pool.rotated ? kRotation(D) : 1.0f, y, [&](int i) { return 4 * (TPR * i + part); });
            if (g.pool.rotated) {
                wht_inlane<4 * CG>(y);
#pragma unroll
                for (int i = 0; i < 4 * CG; ++i) {
                    y[i] = wht_lane_stage<1>(y[i], lane);
                    y[i] = wht_lane_stage<2>(y[i], lane);
                    y[i] = wht_lane_stage<4>(y[i], lane);
                    if constexpr (TPR == 16) y[i] = wht_lane_stage<8>(y[i], lane);
                }
                if (g.pool.signs.on) {
#pragma unroll
                    for (int c = 0; c < CG; ++c) {
                        const int at = 4 * (TPR * c + part);
                        flip_signs<4>(*reinterpret_cast<float(*)[4]>(y + 4 * c), sign_word(g.pool.signs, at >> 5) >> (at & 31));
                    }
                }
            }
            L = fmaf(pool_L, __builtin_amdgcn_exp2f(pool_M - M), L);
        }
        if (r >= t.rows) return;
        const float inv = L != 0.0f ? 1.0f / L : 0.0f;
        const size_t orow = out_row(g, pl, r), prow = partial_row(g, pl, r);
#pragma unroll
        for (int c = 0; c < CG; ++c) {
            const int at = 4 * (TPR * c + part);
            float* d = y + 4 * c;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float4 z = *reinterpret_cast<const float4*>(o_s + (w * R + rr) * OSTRIDE + at);
                d[0] = fmaf(z.x, f[w], d[0]), d[1] = fmaf(z.y, f[w], d[1]), d[2] = fmaf(z.z, f[w], d[2]), d[3] = fmaf(z.w, f[w], d[3]);
            }
            if (last)
                *reinterpret_cast<uint2*>(g.out + orow * D + at) = make_uint2(pack2<BF>(d[0] * inv, d[1] * inv), pack2<BF>(d[2] * inv, d[3] * inv));
            else if (L != 0.0f)   // (a partial of no tokens: nobody reads its sums)
                *reinterpret_cast<float4*>(g.o + prow * D + at) = make_float4(d[0], d[1], d[2], d[3]);
        }
        if (!last && part == 0) *reinterpret_cast<float2*>(g.ml + prow * 2) = make_float2(M, L);
    }
}

// ----------------------------------------------------------------------------- more rows a head ---
// The waves of a workgroup (two or four) have 32 rows each and walk through the tiles together: a tile is fetched once, whole rows
// at a time, by all of them, and handed out through LDS, two tiles deep.  A thread fetches pieces of 16 bytes of a few tokens; what it
// fetches for the tile after the next waits in registers until the tile before is done with.  (Keys straight from the pages as
// operands, as above, are 32-byte pieces of 32 rows per load: four waves that fetch the same tile that way are bound by the L1.)
// 128 rows over 7,194 tokens of 16 agents (4 layers x 8 heads, head_dim 128, 1.9 GB, 0.24 Tflop): 383 us at the fastest, where the loads
// alone take 319 and the arithmetic alone 344.  Two waves a SIMD do not hide all of either behind the other; 64 rows a wave would halve
// the LDS reads, but put a wave's sums into accumulation registers (521 us).
template <int I> using Set = std::integral_constant<int, I>;
constexpr int many_waves_per_simd(int D) { return D == 256 ? 1 : 2; }

template <int D, bool BF, int W>
__global__ __launch_bounds__(64 * W, many_waves_per_simd(D)) void attend_pages_many_kernel(TreeArgs g) {
    constexpr int R = 32;
    using S = Shape<D, R>;
    constexpr int MG = S::MG, KJ = S::KJ;
    constexpr int LPT = D / 8;                    // threads that fetch a token's row
    constexpr int TPP = 64 * W / LPT, NP = 32 / TPP;   // tokens of a pass, passes of a tile
    // Rows in LDS, in halves: 16 bytes more rotate the banks for the keys' operands (16 bytes of each of 32 rows), 64 bytes
    // more for the values' (64 bytes of each of 4 rows).
    constexpr int KS = D + 8, VS = D + 32, TILE = 32 * (KS + VS);
    extern __shared__ __align__(16) uint16_t kv_s[];   // [2 tiles]([32][KS] keys, [32][VS] values)
    __shared__ int flag_s[2][32];                 // of a tile's token: 1 there, 2 a draft with a value that is not finite
    const PageView& v = g.v;
    const TreePlan& t = g.t;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane / R, n = lane % R;
    const Place pl = place_of(g);
    if (!pl.inside) return;
    const int row0 = pl.row_block * R * W;
    const int tiles = row0 < pl.count * t.G ? (pl.length + 31) >> 5 : 0;
    const int per_split = (tiles + t.nsplit - 1) / t.nsplit;
    const int t_begin = pl.split * per_split, t_end = min(tiles, t_begin + per_split);
    const int my_row0 = row0 + wave * R;
    PoolSums<D> pool;
    pool.request(g, pl, my_row0 + n);

    const size_t layer = (size_t)(t.layer_begin + pl.ls) * v.pages * v.H * v.P * D;
    const uint16_t* const Kb = v.K + layer;
    const uint16_t* const Vb = v.V + layer;
    const int32_t* const table = v.table + (size_t)pl.a * v.max_blocks;
    const int my_token = tid / LPT, piece = tid % LPT;   // of a pass
    constexpr int SETS = W == 4 ? 2 : 1;
    int page[NP], page_off[NP];
    tree_uint4 fk[SETS][NP], fv[SETS][NP];
    bool fthere[SETS][NP];
    auto fetch_pages = [&](int tile) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            page[i] = table[v.div_P.divide(min(32 * tile + i * TPP + my_token, pl.length - 1), &page_off[i])];
        }
    };
    auto fetch = [&](int tile, auto set) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            fthere[set][i] = 32 * tile + i * TPP + my_token < pl.length && (uint32_t)page[i] < (uint32_t)v.pages;
            const size_t at = (size_t)(fthere[set][i] ? page_row(v, page[i], pl.kvh, page_off[i]) : 0) * D + 8 * piece;
            fk[set][i] = *reinterpret_cast<const tree_uint4*>(Kb + at);
            fv[set][i] = *reinterpret_cast<const tree_uint4*>(Vb + at);
        }
    };
    auto stage = [&](int tile, auto set) {
        uint16_t* const dst = kv_s + (tile & 1) * TILE;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int tok = i * TPP + my_token;
            bool bad = false;
            if (32 * tile + 32 > pl.before) {
                const bool mine = any_nonfinite<BF>(fv[set][i][0]) || any_nonfinite<BF>(fv[set][i][1]) || any_nonfinite<BF>(fv[set][i][2]) || any_nonfinite<BF>(fv[set][i][3]);
                const uint64_t lanes = __ballot(mine);
                const int group = (lane / LPT) * LPT;   // the lanes that hold the token
                bad = ((lanes >> group) & (LPT == 64 ? ~0ull : (1ull << LPT) - 1)) != 0 && 32 * tile + tok >= pl.before;
            }
            // values that are not there, or not finite, are zeroed: a weight of 0 does not undo a NaN
            const bool keep = fthere[set][i] && !bad;
            const tree_uint4 zero = {0, 0, 0, 0};
            *reinterpret_cast<tree_uint4*>(dst + tok * KS + 8 * piece) = fk[set][i];
            *reinterpret_cast<tree_uint4*>(dst + 32 * KS + tok * VS + 8 * piece) = keep ? fv[set][i] : zero;
            if (piece == 0) flag_s[tile & 1][tok] = (fthere[set][i] ? 1 : 0) | (bad && fthere[set][i] ? 2 : 0);
        }
    };

    Rows<D, R> rows;
    rows.clear();
    if (t_begin < t_end) {   // (the same for all waves)
        // Tile t_begin + i waits for LDS in register set i % SETS.
        auto ask = [&](int tile, auto set) {   // its pages' numbers have been asked for; those of the tile behind it are now
            if (tile < t_end) fetch(tile, set);
            if (tile + 1 < t_end) fetch_pages(tile + 1);
        };
        fetch_pages(t_begin);
        ask(t_begin, Set<0>());
        if constexpr (SETS > 1) ask(t_begin + 1, Set<1>());
        tree_uint4 q[KJ];
        const int draft = load_queries<D, R>(g, pl, my_row0, lane, q);
        const uint64_t see_first = first_drafts(t, pl, draft);
        float poison = 0.0f;
        if (draft >= pl.count) rows.m = 0.0f;   // such a row never sees a token: any reference will do
        stage(t_begin, Set<0>());
        wait_for(q);
        ask(t_begin + SETS, Set<0>());
        __syncthreads();

        auto step = [&](int tile, auto next) {   // `next`: the set with the tile behind it
            uint16_t* const src = kv_s + (tile & 1) * TILE;
            const int t0 = 32 * tile;
            Scores<R> s;
            s.clear();
#pragma unroll
            for (int j = 0; j < KJ; ++j)
#pragma unroll
                for (int u = 0; u < S::TT; ++u)
                    s.t[u] = tree_mfma<BF, R>(*reinterpret_cast<const tree_uint4*>(src + (R * u + n) * KS + 8 * (S::LPR * j + h)), q[j], s.t[u]);
            const int flags = flag_s[tile & 1][lane & 31];
            const uint32_t there = (uint32_t)__ballot(flags & 1);
            if (there != 0xFFFFFFFFu || t0 + 32 > pl.before || my_row0 + R > pl.count * t.G) {
                const uint32_t bad = (uint32_t)__ballot(flags & 2), seen = seen_tokens(t, pl, draft, see_first, t0, there);
                if (seen & bad) poison = NAN;
                hide_unseen<D, R>(s, seen, h);
            }
            const Weights<BF, R> w = weigh<D, BF, R>(rows, s, t.qscale);
            // values: sixteen lanes read 16 coordinates of four tokens and get four tokens of one coordinate each
            uint16_t* const vals = src + 32 * KS + (4 * h + ((lane & 15) >> 2)) * VS + (n & 16) + 4 * (lane & 3);
#pragma unroll
            for (int part = 0; part < S::PARTS; ++part)
#pragma unroll
                for (int e = 0; e < MG; ++e) {
                    uint16_t* const at = vals + S::token_of(8 * part) * VS + R * e;
                    const uint2 lo = lds_transposed(at), hi = lds_transposed(at + S::token_of(4) * VS);
                    const tree_uint4 a = {lo.x, lo.y, hi.x, hi.y};
                    rows.acc[e] = tree_mfma<BF, R>(a, w.p[part], rows.acc[e]);
                    if constexpr (BF) rows.acc[e] = tree_mfma<BF, R>(a, w.low[part], rows.acc[e]);
                }
            if (tile + 1 < t_end) {
                stage(tile + 1, next);
                ask(tile + 1 + SETS, next);
            }
            __syncthreads();
        };
        for (int tile = t_begin; tile < t_end; tile += SETS) {
            step(tile, Set<1 % SETS>());
            if constexpr (SETS > 1)
                if (tile + 1 < t_end) step(tile + 1, Set<0>());
        }
        rows.l += poison;
    }
    store_rows<D, BF, R, true>(g, pl, rows, pool, my_row0, lane);
}

// -------------------------------------------------------------------------------------- merge ---
// One wave per row, or (SHARE) eight that take every eighth partial each.  The pool's partials are added in the rotated domain and
// rotated back, the pages' join behind that; what the eight waves have then is added through LDS.
template <int D, bool BF, bool SHARE>
__global__ __launch_bounds__(SHARE ? 512 : 256) void tree_merge_kernel(AttendPlan p, int nsplit, int page_nsplit, const float* __restrict__ pool_ml,
                                                                       const float* __restrict__ pool_o, const float* __restrict__ ml,
                                                                       const float* __restrict__ o, uint16_t* __restrict__ out) {
    constexpr int EPL = D / 64;
    constexpr int STEP = SHARE ? 8 : 1, B = SHARE ? 8 : 16;   // B partial rows are requested at once
    __shared__ float2 x_s[SHARE ? 8 : 1][SHARE ? D / 2 : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, turn = SHARE ? wave : 0;
    const long block = (long)blockIdx.y * gridDim.x + blockIdx.x, row_global = SHARE ? block : block * 4 + wave;
    const long nrows = (long)p.layers * p.H * p.R;
    const bool active = row_global < nrows;   // no early return: the butterflies need the whole wave
    const long rg = active ? row_global : 0;
    const int usel = (int)(rg / p.R), r = (int)(rg - (long)usel * p.R);
    int kvh;
    const int ls = p.div_H.divide(usel, &kvh);
    // Lane s holds (m, l) of split s: first the maximum over all splits, then sixty-four splits' weights at a time, which are handed
    // out with readlane.
    auto sums_of = [&](const float* base, int n, int s) {
        return s < n ? *reinterpret_cast<const float2*>(base + (((size_t)usel * n + s) * p.R + r) * 2) : make_float2(-INFINITY, 0.0f);
    };
    float M = -INFINITY;
    for (int s0 = 0; s0 < nsplit; s0 += 64) M = fmaxf(M, sums_of(pool_ml, nsplit, s0 + lane).x);
    for (int s0 = 0; s0 < page_nsplit; s0 += 64) M = fmaxf(M, sums_of(ml, page_nsplit, s0 + lane).x);
    M = fmaxf(M, lane_xor<1>(M));
    M = fmaxf(M, lane_xor<2>(M));
    M = fmaxf(M, lane_xor<4>(M));
    M = fmaxf(M, lane_xor<8>(M));
    M = row_max<16>(M);
    float x[EPL], L = 0.0f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = 0.0f;
    auto add = [&](const float* base_ml, const float* base_o, int n) {
        for (int s0 = 0; s0 < n; s0 += 64) {
            const float2 part = sums_of(base_ml, n, s0 + lane);
            const float w = part.x == -INFINITY ? 0.0f : exp2f(part.x - M);   // (a partial of no tokens)
            L = fmaf(part.y, w, L);
            const int cnt = min(64, n - s0);
            const float* src = base_o + (((size_t)usel * n + s0) * p.R + r) * D + lane * EPL;
            for (int k0 = turn; k0 < cnt; k0 += B * STEP) {
                float v[B][EPL], wk[B];
#pragma unroll
                for (int k = 0; k < B; ++k) {
                    const int split = k0 + STEP * k;
                    wk[k] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), min(split, 63)));
                    const bool used = split < cnt && wk[k] != 0.0f;   // (sums that weigh nothing need not have been written)
#pragma unroll
                    for (int i = 0; i < EPL; ++i) v[k][i] = used ? src[(size_t)split * p.R * D + i] : 0.0f;
                }
#pragma unroll
                for (int k = 0; k < B; ++k)
#pragma unroll
                    for (int i = 0; i < EPL; ++i) x[i] = fmaf(v[k][i], wk[k], x[i]);
            }
        }
    };
    add(pool_ml, pool_o, nsplit);
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
            x[i] *= kRotation(D);
        }
        if (p.signs.on) flip_signs<EPL>(x, sign_word(p.signs, (lane * EPL) >> 5) >> ((lane * EPL) & 31));
    }
    add(ml, o, page_nsplit);
    L += lane_xor<1>(L);
    L += lane_xor<2>(L);
    L += lane_xor<4>(L);
    L += lane_xor<8>(L);
    L = row_sum<16>(L);
    const float inv = L != 0.0f ? 1.0f / L : 0.0f;
    uint16_t* const dst = out + q_row_index(p, ls, kvh, r) * D;
    if constexpr (SHARE) {   // (every workgroup has a row)
#pragma unroll
        for (int i = 0; i < EPL; ++i) reinterpret_cast<float*>(x_s[wave])[lane * EPL + i] = x[i];
        __syncthreads();
        if (threadIdx.x < D / 2) {
            float2 y = x_s[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < 8; ++w) y.x += x_s[w][threadIdx.x].x, y.y += x_s[w][threadIdx.x].y;
            reinterpret_cast<uint32_t*>(dst)[threadIdx.x] = pack2<BF>(y.x * inv, y.y * inv);
        }
    } else if (active) {
        if constexpr (EPL == 1) {
            dst[lane] = (uint16_t)pack2<BF>(x[0] * inv, 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < EPL; i += 2) *reinterpret_cast<uint32_t*>(dst + lane * EPL + i) = pack2<BF>(x[i] * inv, x[i + 1] * inv);
        }
    }
}

// ----------------------------------------------------------------------------------- launchers ---
// Which form a call takes, by the rows of an agent and KV head and by how many agents and KV heads there are.  Measured, both sides:
//   four waves share the rows where even so the waves do not fill the SIMDs twice: one layer of 15 agents x 64 rows over 112 tokens and a
//     pool 37.4 us, 40.9 with a wave for 32 rows; all 24 layers of 100 agents with one row each 613 and 433 us;
//   up to 16 rows a wave has 16: that last call 438 us with 32, 396;
//     (at head_dim 256 32 rows do not fit a wave's registers beside keys and values on their way, and a wave always has 16);
//   more than one wave's rows: two or four waves fetch the tiles together, four where two would not leave fewer waves idle: 128
//     rows over 7,194 tokens 414 us, 514 with two; 160 rows over 300 tokens 261 us, 207 with two.
void plan_tree(const PageView& v, int pool_splits, int page_splits, TreePlan* t) {
    const long tiles = ((long)v.max_blocks * v.P + 31) / 32, units = (long)t->layers * v.H * v.A;
    const int row_tiles = (t->rows + 31) / 32;
    t->share = units * row_tiles <= 512 ? 1 : 0;
    t->wave_rows = t->rows <= 16 || v.D == 256 ? 16 : 32;
    t->waves = 1;
    if (!t->share && t->rows > t->wave_rows) {
        t->waves = (row_tiles + 3) / 4 * 4 <= (row_tiles + 1) / 2 * 2 ? 4 : 2;
        t->wave_rows = 32;
    }
    const int rows = t->wave_rows * t->waves;
    t->row_blocks = (t->rows + rows - 1) / rows;
    const long groups = units * t->row_blocks;
    // Token ranges: the count with the least estimated time, in steps of a wave (one tile, about 1.5 us): rounds of workgroups over
    // the places there are (waves that the registers leave room for), times the steps of the longest continuation there can be plus
    // four for the ramp and the final pass; more than one range adds the merge kernel and its partials.
    const int on_simd = t->waves > 1 ? many_waves_per_simd(v.D) : few_waves_per_simd(v.D, t->wave_rows), ways = t->share ? 4 : 1;
    const long places = 256l * (4 * on_simd / (t->share ? 4 : t->waves));
    const long most = std::min((tiles + 3) / 4, 64l);
    auto cost = [&](long n) {
        const double steps = (double)((tiles + n * ways - 1) / (n * ways)) + 4;
        const double rounds = (double)((groups * n + places - 1) / places);
        return rounds * steps + (n > 1 || pool_splits > kJoinSplits ? 6 + n * (double)units * t->rows * v.D * (8 / 4e12 / 1.5e-6) : 0.0);
    };
    long want = 1;
    for (long n = 2; n <= most; ++n)
        if (cost(n) < cost(want)) want = n;
    if (page_splits > 0) want = std::min((long)page_splits, (tiles + 3) / 4);
    t->nsplit = (int)want;
    t->merge = want > 1 || pool_splits > kJoinSplits;
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

using PagesKernel = void (*)(TreeArgs);
struct PagesForm {
    PagesKernel kern;
    int threads, shared;
};
template <int D, bool BF> static PagesForm pages_form(const TreePlan& t) {
    constexpr int kShare = 4 * (D + 4) * (int)sizeof(float), kStage = 2 * 32 * (2 * D + 40) * (int)sizeof(uint16_t);
    if (t.waves == 4) return {attend_pages_many_kernel<D, BF, 4>, 256, kStage};
    if (t.waves == 2) return {attend_pages_many_kernel<D, BF, 2>, 128, kStage};
    if constexpr (D != 256)
        if (t.wave_rows == 32) return t.share ? PagesForm{attend_pages_few_kernel<D, BF, 32, true>, 256, 32 * kShare} : PagesForm{attend_pages_few_kernel<D, BF, 32, false>, 64, 0};
    return t.share ? PagesForm{attend_pages_few_kernel<D, BF, 16, true>, 256, 16 * kShare} : PagesForm{attend_pages_few_kernel<D, BF, 16, false>, 64, 0};
}

hipError_t launch_attend_pages(const PageView& v, const TreePlan& t, bool bf16, const void* Q, float* ml, float* o, void* out,
                               const PoolPart& pool, hipStream_t s) {
    const TreeArgs g = {v, t, (const uint16_t*)Q, ml, o, (uint16_t*)out, pool};
    const uint64_t streams = (uint64_t)t.layers * v.H * v.A * t.nsplit;
    const dim3 grid = grid_of((streams + 7) / 8 * 8 * t.row_blocks);
    const PagesForm f = v.D == 64    ? (bf16 ? pages_form<64, true>(t) : pages_form<64, false>(t))
                        : v.D == 128 ? (bf16 ? pages_form<128, true>(t) : pages_form<128, false>(t))
                                     : (bf16 ? pages_form<256, true>(t) : pages_form<256, false>(t));
    if (f.shared > 48 * 1024) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(f.kern), hipFuncAttributeMaxDynamicSharedMemorySize, f.shared);
        if (err != hipSuccess) return err;
    }
    launch_kernel(f.kern, grid, dim3(f.threads), f.shared, s, take_kernel_events(), g);   // (without a pool: the call's main kernel)
    return hipGetLastError();
}

using MergeKernel = void (*)(AttendPlan, int, int, const float*, const float*, const float*, const float*, uint16_t*);
template <int D> static MergeKernel merge_form(bool bf16, bool share) {
    if (share) return bf16 ? tree_merge_kernel<D, true, true> : tree_merge_kernel<D, false, true>;
    return bf16 ? tree_merge_kernel<D, true, false> : tree_merge_kernel<D, false, false>;
}

// Measured, fastest of ten, eight waves a row and one: 32 rows of head_dim 256 and 75 partials 7.6 and 21.3 us, 256 rows of 128
// and 44 partials 5.1 and 6.7, 2,048 rows and 24 partials 14.7 and 6.5.
constexpr long kMergeShareRows = 512;

hipError_t launch_tree_merge(const AttendPlan& plan, const TreePlan& t, bool has_pool, const float* pool_ml, const float* pool_o,
                             const float* ml, const float* o, void* out, hipStream_t s) {
    const long nrows = (long)plan.layers * plan.H * plan.R;
    const bool share = nrows <= kMergeShareRows;
    launch_kernel(plan.D == 64 ? merge_form<64>(plan.io_bf16, share) : plan.D == 128 ? merge_form<128>(plan.io_bf16, share) : merge_form<256>(plan.io_bf16, share),
                  grid_of(share ? (uint64_t)nrows : (uint64_t)(nrows + 3) / 4), dim3(share ? 512 : 256), 0, s, {}, plan, has_pool ? plan.nsplit : 0, t.nsplit,
                  pool_ml, pool_o, ml, o, (uint16_t*)out);
    return hipGetLastError();
}

}  // namespace polykv
