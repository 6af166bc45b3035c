"""Drafted decoding over continuations in pages, against plain 64-bit implementations (tree_util): block tables, writes, masks,
attention with and without a pool, acceptance, and a step of all of them, eager and in graphs."""
import numpy as np
import pytest
import torch

import tree_util as U
from paper_2604_24971_amd import workloads as W

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def _pk():
    from paper_2604_24971_amd import polykv as pk
    return pk


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t.to(dtype) if dtype is not None else t).cuda()


def rounded(x, dtype):
    """float64 values as the dtype holds them."""
    return torch.from_numpy(np.asarray(x, np.float64)).to(dtype).double().numpy()


class Setup:
    """Pages with the agents' tokens scattered over them; whatever no agent holds is NaN."""

    def __init__(self, rng, lengths, d, H=2, P=16, L=1, dtype=F16, kscale=1.0, MB=None, NP=None):
        pk = _pk()
        self.lengths, self.P, self.d, self.dtype = np.array(lengths, np.int32), P, d, dtype
        MB = MB or max(1, -(-max(lengths) // P) + 1)
        self.table, pages = U.scattered(rng, lengths, P, MB)
        self.K = np.full((L, pages, H, P, d), np.nan)
        self.V = np.full((L, pages, H, P, d), np.nan)
        for a, n in enumerate(lengths):
            for t in range(n):
                at = (slice(None), self.table[a, t // P], slice(None), t % P)
                self.K[at] = rng.standard_normal((L, H, d)) * kscale
                self.V[at] = rng.standard_normal((L, H, d))
        self.K, self.V = rounded(self.K, dtype), rounded(self.V, dtype)
        self.pages = pk.Pages(L, H, d, pages, len(lengths), MB, page_tokens=P, dtype=dtype)
        self.load()

    def load(self):
        self.pages.K.copy_(dev(self.K, self.dtype))
        self.pages.V.copy_(dev(self.V, self.dtype))
        self.pages.table.copy_(dev(self.table))
        self.pages.lengths.copy_(dev(self.lengths))

    def check(self, got, Q, counts, seen, pool=None, **kw):
        out, mag, big = U.attend(Q, self.K, self.V, self.table, self.lengths, counts, seen, pool, **kw)
        vmax = max(np.nanmax(np.abs(self.V), initial=0.0), np.abs(pool[1]).max() if pool is not None else 0.0)
        tokens = int(self.lengths.max()) + (pool[0].shape[2] if pool is not None else 0)
        tol = U.bound(out, mag, big, self.d, self.dtype, tokens, vmax, pool is not None)
        err = np.abs(got.double().cpu().numpy() - out)
        assert np.isfinite(err).all(), "not finite at %s" % (np.argwhere(~np.isfinite(err))[0],)
        assert (err <= tol).all(), "off by %g, %g allowed, at %s" % (err[err > tol].max(), tol[err > tol].min(), np.argwhere(err > tol)[0])


LENGTHS = [0, 1, 2, 7, 8, 9, 31, 32, 33, 63, 65, 96, 127, 128, 129, 161, 300]


def _pool(rng, L, H, d, T, dtype, **kw):
    pk = _pk()
    K = dev(0.3 * rng.standard_normal((L, H, T, d)), dtype)
    V = dev(rng.standard_normal((L, H, T, d)), dtype)
    pool = pk.Pool(L, H, d, T, **kw).bind()
    pool.encode(K, V)
    Kh, Vh = pool.decode(torch.float32)
    return pool, (Kh.double().cpu().numpy(), Vh.double().cpu().numpy())


@pytest.mark.parametrize("d,group,nodes,P,dtype", [
    (64, 1, 1, 16, F16), (64, 3, 5, 8, BF16), (64, 4, 33, 24, F16), (128, 4, 1, 16, BF16), (128, 4, 8, 24, F16), (128, 1, 70, 8, F16),
    (128, 5, 13, 40, BF16), (256, 2, 1, 16, F16), (256, 3, 11, 32, BF16)])
def test_attention_over_pages(d, group, nodes, P, dtype):
    rng = np.random.default_rng(d + 7 * group + nodes)
    A, H = len(LENGTHS), 2
    s = Setup(rng, LENGTHS, d, H=H, P=P, L=2, dtype=dtype)
    Q = rounded(rng.standard_normal((2, A, nodes, H * group, d)), dtype)
    counts = rng.integers(0, nodes + 1, A).astype(np.int32)
    counts[::3] = nodes
    seen = rng.random((A, nodes, nodes)) < 0.5     # any set of drafts, empty ones too: an agent without other tokens sees nothing
    seen[:, ::4] = False
    mask = dev(U.pack(seen))
    kw = dict(counts=dev(counts), mask=mask)
    for splits in (0, 1, 3):
        s.check(s.pages.attend_tree(dev(Q, dtype), page_splits=splits, **kw), Q, counts, seen)
    s.check(s.pages.attend_tree(dev(Q, dtype)), Q, np.full(A, nodes), None)      # neither counts nor mask
    got = s.pages.attend_tree(dev(Q[1:], dtype), layer_begin=1, layer_end=2, scale=0.2, **kw)
    s.check(got, Q[1:], counts, seen, layer_begin=1, scale=0.2)
    pool, dense = _pool(rng, 2, H, d, 75, dtype)
    for splits, page_splits in ((0, 0), (1, 2), (2, 1)):
        got = pool.attend_tree(dev(Q, dtype), s.pages, splits=splits, page_splits=page_splits, **kw)
        s.check(got, Q, counts, seen, pool=dense)
    got = pool.attend_tree(dev(Q[1:], dtype), s.pages, layer_begin=1, layer_end=2, kernel=_pk().KERNEL_VECTOR, **kw)
    s.check(got, Q[1:], counts, seen, pool=dense, layer_begin=1)


@pytest.mark.parametrize("d,dtype,kw", [(128, F16, dict(value_codec=2)), (256, BF16, dict(value_codec=2)), (64, F16, dict(value_codec=1)),
                                        (128, BF16, dict(value_codec=5, sign_seed=77)), (128, F16, dict(key_codec=1)), (64, BF16, dict(sign_seed=3))])
def test_every_kind_of_pool(d, dtype, kw):
    rng = np.random.default_rng(d)
    s = Setup(rng, [40, 0, 65], d, L=2, dtype=dtype)
    pool, dense = _pool(rng, 2, 2, d, 333, dtype, **kw)
    Q = rounded(rng.standard_normal((2, 3, 4, 6, d)), dtype)
    seen = U.reach(U.random_trees(rng, 3, 4), [4, 4, 4])
    for splits in (0, 2):
        s.check(pool.attend_tree(dev(Q, dtype), s.pages, mask=dev(U.pack(seen)), splits=splits), Q, [4, 4, 4], seen, pool=dense)


@pytest.mark.parametrize("d,nodes,dtype", [(64, 3, BF16), (64, 130, F16), (128, 1, F16), (128, 90, BF16), (256, 2, BF16), (256, 87, F16)])
def test_more_partials_than_a_wave_has_lanes(d, nodes, dtype):
    """Calls of few and of many rows whose token ranges, 71 of the pages and up to 96 of the pool, are joined; most hold nothing of
    the shorter agents, and one agent has no token at all."""
    rng = np.random.default_rng(d + nodes)
    s = Setup(rng, [9000, 140, 0], d, H=1, dtype=dtype)
    Q = rounded(rng.standard_normal((1, 3, nodes, 2, d)), dtype)
    counts = np.array([nodes, nodes // 2, 0], np.int32)
    s.check(s.pages.attend_tree(dev(Q, dtype), counts=dev(counts), page_splits=71), Q, counts, None)
    pool, dense = _pool(rng, 1, 1, d, 3100, dtype)
    for page_splits in (2, 71):
        got = pool.attend_tree(dev(Q, dtype), s.pages, counts=dev(counts), splits=96, page_splits=page_splits)
        s.check(got, Q, counts, None, pool=dense)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_many_rows_and_the_largest_trees(dtype):
    rng = np.random.default_rng(5)
    s = Setup(rng, [256, 290, 511], 64, H=1, P=8, dtype=dtype)
    Q = rounded(rng.standard_normal((1, 3, 256, 3, 64)), dtype)
    parents = U.random_trees(rng, 3, 256, near=200)
    counts = np.array([256, 256, 201], np.int32)
    seen = U.reach(parents, counts)
    mask, depth = _pk().tree_masks(dev(parents), dev(counts))
    assert torch.equal(mask.cpu(), torch.from_numpy(U.pack(seen)))
    s.check(s.pages.attend_tree(dev(Q, dtype), mask=mask, counts=dev(counts)), Q, counts, seen)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_rising_and_far_apart_scores(d, dtype):
    """Keys that grow along the tokens: a row's reference moves in every tile, by up to hundreds of powers of two, and for some
    rows the other way round."""
    rng = np.random.default_rng(d + 1)
    s = Setup(rng, [700, 333], d, dtype=dtype)
    for a, n in enumerate(s.lengths):
        for t in range(n):
            s.K[:, s.table[a, t // 16], :, t % 16] *= t / 40.0
    s.K = rounded(s.K, dtype)
    s.load()
    Q = rounded(rng.standard_normal((1, 2, 3, 8, d)) * np.array([1.0, -3.0, 0.01])[:, None, None], dtype)
    for splits in (1, 2):
        s.check(s.pages.attend_tree(dev(Q, dtype), page_splits=splits), Q, [3, 3], None)


@pytest.mark.parametrize("d,nodes,group,dtype", [(64, 8, 2, F16), (64, 30, 1, BF16), (64, 20, 3, F16), (64, 100, 1, BF16), (128, 4, 4, BF16),
                                                 (128, 8, 4, F16), (128, 16, 4, BF16), (128, 32, 4, F16), (256, 8, 2, F16), (256, 24, 2, BF16)])
def test_rising_scores_in_calls_of_many_heads(d, nodes, group, dtype):
    """The same for the forms with rows of their own; scores of many thousands, where a product's rounding matters, among them."""
    pk = _pk()
    rng = np.random.default_rng(d + nodes)
    s = Setup(rng, [nodes + 300, nodes + 77], d, dtype=dtype)
    for a, n in enumerate(s.lengths):
        for t in range(n):
            s.K[:, s.table[a, t // 16], :, t % 16] *= t / 40.0
    s.K = rounded(s.K, dtype)
    s.load()
    layers = 300
    pages = pk.Pages(layers, 2, d, s.K.shape[1], 2, s.table.shape[1], dtype=dtype)
    for name in ("K", "V"):
        getattr(pages, name).copy_(getattr(s.pages, name).expand_as(pages.K))
    pages.table.copy_(dev(s.table))
    pages.lengths.copy_(s.pages.lengths)
    for size in (1.0, -3.0, 0.01, 2e4):
        Q1 = rounded(np.clip(rng.standard_normal((1, 2, nodes, 2 * group, d)) * size, -6e4, 6e4), dtype)     # (finite in fp16)
        got = pages.attend_tree(dev(Q1, dtype).expand(layers, -1, -1, -1, -1).contiguous(), page_splits=1)
        assert torch.equal(got, got[:1].expand_as(got))
        if size < 1e3:
            s.check(got[:1], Q1, [nodes, nodes], None)
        else:   # (one token has all the weight, up to ties within the scores' rounding: the result is some mean of values)
            assert torch.isfinite(got).all() and float(got.abs().max()) <= np.nanmax(np.abs(s.V)) * 1.01


def test_queries_and_values_of_extreme_magnitude():
    rng = np.random.default_rng(11)
    for dtype, big in ((F16, 6e4), (BF16, 1e30)):
        s = Setup(rng, [100, 37], 128, dtype=dtype)
        s.V = rounded(s.V * (big / 8), dtype)
        s.load()
        Q = rounded(rng.standard_normal((1, 2, 2, 4, 128)), dtype)
        s.check(s.pages.attend_tree(dev(Q, dtype)), Q, [2, 2], None)
        Q[...] = 0.0
        s.check(s.pages.attend_tree(dev(Q, dtype)), Q, [2, 2], None)


@pytest.mark.parametrize("d,dtype", [(64, F16), (128, BF16), (256, F16)])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_what_a_draft_does_not_see_has_no_effect(d, dtype, bad):
    """Siblings hold vectors that are not finite: only the drafts that see them are touched."""
    rng = np.random.default_rng(d)
    A, N = 3, 12
    s = Setup(rng, [45, 12, 70], d, dtype=dtype)
    parents = U.random_trees(rng, A, N, near=4)
    seen = U.reach(parents, [N] * A)
    broken = [5, 3, 9]
    for a, i in enumerate(broken):
        t = s.lengths[a] - N + i
        s.K[:, s.table[a, t // 16], :, t % 16] = bad
        s.V[:, s.table[a, t // 16], :, t % 16, ::3] = bad
    s.load()
    Q = rounded(rng.standard_normal((1, A, N, 6, d)), dtype)
    for a, i in enumerate(broken):      # what the 64-bit form computes for rows that do not see it, without it
        t = s.lengths[a] - N + i
        s.K[:, s.table[a, t // 16], :, t % 16] = 0.0
        s.V[:, s.table[a, t // 16], :, t % 16] = 0.0
    touched = np.array([seen[a, :, i] for a, i in enumerate(broken)])
    for splits in (1, 2):
        got = s.pages.attend_tree(dev(Q, dtype), mask=dev(U.pack(seen)), page_splits=splits)
        assert not torch.isfinite(got[:, torch.from_numpy(touched)]).any()
        clean = torch.where(torch.from_numpy(touched).cuda()[None, :, :, None, None], 0.0, got.float())
        want = Q * ~touched[None, :, :, None, None]
        s2 = seen & ~touched[:, :, None]
        out, mag, big = U.attend(want, s.K, s.V, s.table, s.lengths, [N] * A, s2)
        err = np.abs(clean.double().cpu().numpy() - out)[:, ~touched]
        tol = U.bound(out, mag, big, d, dtype, 70, 6.0)[:, ~touched]
        assert (err <= tol).all()


@pytest.mark.parametrize("d,nodes,group", [(64, 2, 3), (128, 5, 4), (128, 20, 4), (256, 3, 4), (256, 40, 2)])
def test_rows_without_drafts_beside_values_that_are_not_finite(d, nodes, group):
    """An agent has fewer drafts than rows, and NaN and infinite vectors before them: its rows without a draft attend the pool
    alone, without one they are 0, and other agents see nothing of it."""
    rng = np.random.default_rng(d + nodes)
    s = Setup(rng, [40, 100, 33], d, dtype=BF16)
    broken = s.table[0, 1]
    s.K[:, broken, :, 3], s.V[:, broken, :, 4:6] = np.nan, np.inf
    s.load()
    Q = rounded(rng.standard_normal((1, 3, nodes, 2 * group, d)), BF16)
    pool, dense = _pool(rng, 1, 2, d, 64, BF16)
    counts = np.array([1, nodes, 0], np.int32)
    for splits in (1, 2):
        for with_pool in (None, dense):
            kw = dict(counts=dev(counts), page_splits=splits)
            got = s.pages.attend_tree(dev(Q, BF16), **kw) if with_pool is None else pool.attend_tree(dev(Q, BF16), s.pages, **kw)
            assert not torch.isfinite(got[0, 0, 0]).any()
            got[0, 0, 0] = 0.0
            lengths, s.lengths = s.lengths, np.array([0, 100, 33], np.int32)
            Q0 = Q.copy()
            got_rest, Q_rest = got[:, 1:], Q0[:, 1:]
            out, mag, big = U.attend(Q_rest, s.K, s.V, s.table[1:], s.lengths[1:], counts[1:], None, with_pool)
            tol = U.bound(out, mag, big, d, BF16, 164, 6.0, with_pool is not None)
            assert (np.abs(got_rest.double().cpu().numpy() - out) <= tol).all()
            alone = U.attend(Q[:, :1, 1:], s.K, s.V, s.table[:1], [0], [0], None, with_pool)
            tol = U.bound(*alone, d, BF16, 164, 6.0, with_pool is not None)
            assert (np.abs(got[:, :1, 1:].double().cpu().numpy() - alone[0]) <= tol).all()
            s.lengths = lengths


@pytest.mark.parametrize("d,nodes,group,dtype", [
    (64, 5, 3, F16), (64, 16, 1, BF16), (64, 30, 1, F16), (64, 10, 3, BF16), (64, 20, 2, F16), (64, 33, 2, BF16), (64, 130, 1, F16),
    (128, 4, 4, F16), (128, 3, 5, BF16), (128, 8, 4, BF16), (128, 25, 1, F16), (128, 13, 4, F16), (128, 41, 4, BF16), (128, 96, 1, F16),
    (256, 8, 2, F16), (256, 16, 2, BF16), (256, 20, 5, F16)])
@pytest.mark.parametrize("page_splits", [1, 2])
def test_calls_of_many_heads(d, nodes, group, dtype, page_splits):
    """Calls with many KV heads, where waves and workgroups have rows of their own: masks of any kind, agents with fewer drafts than
    rows, drafts with values that are not finite, a page that is not there, NaN behind the tokens."""
    pk = _pk()
    rng = np.random.default_rng(7 * d + nodes + group)
    lengths = [nodes, nodes + 1, nodes + 90, 0, nodes + 33, nodes + 130, max(nodes - 1, 1)]
    A = len(lengths)
    layers = 520 // (2 * A) + 1
    s = Setup(rng, lengths, d, P=24, dtype=dtype)
    s.table[5, 1] = -1
    seen = rng.random((A, nodes, nodes)) < 0.5
    seen[:, 1::5] = False
    counts = np.array([nodes, max(nodes - 2, 0), nodes, nodes, nodes // 2, nodes, nodes], np.int32)
    touched = np.zeros((A, nodes), bool)
    for a in (0, 2, 4):      # a draft that some others see
        if counts[a] < 2:
            continue
        i = int(counts[a]) // 2
        t = lengths[a] - counts[a] + i
        s.V[:, s.table[a, t // 24], :, t % 24, 1::2] = np.inf
        touched[a, :counts[a]] = seen[a, :counts[a], i]
    s.load()
    pages = pk.Pages(layers, 2, d, s.K.shape[1], A, s.table.shape[1], page_tokens=24, dtype=dtype)
    for name in ("K", "V"):
        getattr(pages, name).copy_(getattr(s.pages, name).expand_as(pages.K))
    pages.table.copy_(dev(s.table))
    pages.lengths.copy_(s.pages.lengths)
    Q1 = rounded(rng.standard_normal((1, A, nodes, 2 * group, d)), dtype)
    Q = dev(Q1, dtype).expand(layers, -1, -1, -1, -1).contiguous()
    got = pages.attend_tree(Q, counts=dev(counts), mask=dev(U.pack(seen)), page_splits=page_splits)
    same = (got[:1].expand_as(got) == got) | got.isnan()
    assert bool(same.all())
    t = torch.from_numpy(touched).cuda()
    assert not torch.isfinite(got[:, t]).any()
    s.V[~np.isfinite(s.V)] = 0.0
    clean = torch.where(t[None, :, :, None, None], 0.0, got[:1].float()).to(dtype)
    out, mag, big = U.attend(Q1, s.K, s.V, s.table, s.lengths, counts, seen)
    err = np.abs(clean.double().cpu().numpy() - out)[:, ~touched]
    assert (err <= U.bound(out, mag, big, d, dtype, max(lengths), 6.0)[:, ~touched]).all()


def _between_guards(nbytes):
    """Memory with 4 KB of a pattern on both sides: (the whole, the part between)."""
    raw = torch.full((4096 + (nbytes + 255) // 256 * 256 + 4096,), 0x5C, dtype=torch.uint8, device="cuda")
    return raw, raw[4096:4096 + nbytes]


def _untouched(raw, nbytes):
    return bool((raw[:4096] == 0x5C).all()) and bool((raw[4096 + nbytes:] == 0x5C).all())


@pytest.mark.parametrize("d,nodes,group,layers", [(64, 1, 1, 1), (64, 16, 1, 40), (64, 17, 1, 40), (64, 40, 1, 40), (64, 100, 1, 20), (128, 3, 5, 1),
                                                  (128, 1, 5, 40), (128, 5, 5, 40), (128, 9, 5, 40), (128, 20, 5, 20), (256, 1, 3, 40), (256, 7, 3, 20),
                                                  (256, 23, 3, 10)])
def test_writes_stay_inside_the_output_and_the_workspace(d, nodes, group, layers):
    """Every form of the kernel (few rows and many, shared and not), with and without splits and a pool."""
    pk = _pk()
    rng = np.random.default_rng(d + nodes)
    lengths = [nodes, nodes + 70, 9, 150, 33, 64, 200, 31]
    s = Setup(rng, lengths, d, L=1)
    pages = pk.Pages(layers, 2, d, s.K.shape[1], len(lengths), s.table.shape[1], page_tokens=16)
    pages.K.copy_(s.pages.K.expand_as(pages.K))
    pages.V.copy_(s.pages.V.expand_as(pages.V))
    pages.table.copy_(s.pages.table)
    pages.lengths.copy_(s.pages.lengths)
    pool, dense = _pool(rng, 1, 2, d, 70, F16)
    big = pk.Pool(layers, 2, d, 70).bind()
    K, V = pool.decode(F16)
    big.encode(K.expand(layers, -1, -1, -1).contiguous(), V.expand(layers, -1, -1, -1).contiguous())
    Kh, Vh = big.decode(torch.float32, layer_begin=0, layer_end=1)
    dense = Kh.double().cpu().numpy(), Vh.double().cpu().numpy()
    Q1 = rounded(rng.standard_normal((1, len(lengths), nodes, 2 * group, d)), F16)
    Q = dev(Q1, F16).expand(layers, -1, -1, -1, -1).contiguous()
    for p in (None, big):
        for splits in (0, 1, 2):
            need = pages.attend_tree_workspace_bytes(Q, p, page_splits=splits)
            raw_w, ws = _between_guards(max(need, 256))
            raw_o, out = _between_guards(Q.numel() * 2)
            out = out.view(F16).view(Q.shape)
            kw = dict(page_splits=splits, workspace=ws)
            got = pages.attend_tree(Q, out, **kw) if p is None else p.attend_tree(Q, pages, out, **kw)
            torch.cuda.synchronize()
            assert _untouched(raw_w, max(need, 256)) and _untouched(raw_o, Q.numel() * 2)
            assert torch.equal(got, got[:1].expand_as(got))
            s.check(got[:1], Q1, np.full(len(lengths), nodes), None, pool=dense if p is not None else None)


@pytest.mark.parametrize("d,nodes,group,layers,dtype", [(64, 1, 1, 1, F16), (64, 16, 1, 40, BF16), (64, 17, 1, 40, F16), (64, 40, 1, 40, F16),
                                                        (64, 100, 1, 20, BF16), (128, 3, 5, 1, BF16), (128, 5, 1, 40, BF16), (128, 5, 5, 40, F16),
                                                        (128, 20, 5, 20, F16), (256, 1, 3, 1, F16), (256, 1, 3, 40, BF16), (256, 23, 3, 10, F16)])
def test_joining_the_pools_splits(d, nodes, group, layers, dtype):
    """Every form of the kernel with one token range of the pages and one, two, several and more splits of the pool than it joins
    itself; the agents hold a few tokens, or none."""
    pk = _pk()
    rng = np.random.default_rng(d + nodes + 1)
    lengths = [nodes, nodes + 40, 0, 33, nodes + 1, 5, 64, 2]
    s = Setup(rng, lengths, d, L=1, dtype=dtype)
    pages = pk.Pages(layers, 2, d, s.K.shape[1], len(lengths), s.table.shape[1], page_tokens=16, dtype=dtype)
    pages.K.copy_(s.pages.K.expand_as(pages.K))
    pages.V.copy_(s.pages.V.expand_as(pages.V))
    pages.table.copy_(s.pages.table)
    pages.lengths.copy_(s.pages.lengths)
    K = dev(0.3 * rng.standard_normal((1, 2, 700, d)), dtype)
    V = dev(rng.standard_normal((1, 2, 700, d)), dtype)
    pool = pk.Pool(layers, 2, d, 700).bind()
    pool.encode(K.expand(layers, -1, -1, -1).contiguous(), V.expand(layers, -1, -1, -1).contiguous())
    Kh, Vh = pool.decode(torch.float32, layer_begin=0, layer_end=1)
    dense = Kh.double().cpu().numpy(), Vh.double().cpu().numpy()
    Q1 = rounded(rng.standard_normal((1, len(lengths), nodes, 2 * group, d)), dtype)
    Q = dev(Q1, dtype).expand(layers, -1, -1, -1, -1).contiguous()
    for splits in (1, 2, 3, 10, 16, 17):
        got = pool.attend_tree(Q, pages, splits=splits, page_splits=1)
        assert torch.equal(got, got[:1].expand_as(got))
        s.check(got[:1], Q1, np.full(len(lengths), nodes), None, pool=dense)


def test_two_threads_on_one_stream():
    """Calls of different sizes from two threads, on the same stream and pages: each gets what it gets alone."""
    import threading
    rng = np.random.default_rng(6)
    s = Setup(rng, [500, 300, 64], 128, L=2)
    pool, _ = _pool(rng, 2, 2, 128, 700, F16)
    Q = [dev(rng.standard_normal((2, 3, n, 8, 128)), F16) for n in (1, 7)]
    want = [pool.attend_tree(q, s.pages, page_splits=3) for q in Q]
    torch.cuda.synchronize()
    got = [[], []]

    def work(i):
        for _ in range(40):
            got[i].append(pool.attend_tree(Q[i], s.pages, page_splits=3))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(want[i], x) for x in got[i])


def test_pages_that_are_not_there_and_lengths_out_of_range():
    rng = np.random.default_rng(3)
    s = Setup(rng, [100, 64, 33], 128, MB=8)
    s.table[0, 2] = -1
    s.table[1, 0] = 10_000
    s.table[1, 3] = -2_000_000_000
    s.load()
    Q = rounded(rng.standard_normal((1, 3, 2, 4, 128)), F16)
    s.check(s.pages.attend_tree(dev(Q, F16)), Q, [2, 2, 2], None)
    # lengths beyond the table's, negative ones, counts of any size: taken as the nearest bound, entries of -1 are not there
    s.K, s.V = np.nan_to_num(s.K), np.nan_to_num(s.V)       # (behind its 100 tokens agent 0's last page is no longer empty)
    s.load()
    s.pages.lengths.copy_(dev(np.array([2 ** 31 - 1, -5, 33], np.int32)))
    s.lengths = np.array([128, 0, 33], np.int32)
    counts = np.array([1000, 1, -7], np.int32)
    got = s.pages.attend_tree(dev(Q, F16), counts=dev(counts))
    s.check(got, Q, np.array([2, 0, 0]), None)
    assert not got[0, 1:].any()


def test_chain_equals_dense_tails():
    """The same step through pool.attend with dense continuations (fp32) and through pages."""
    pk = _pk()
    rng = np.random.default_rng(9)
    lengths, N, d = [20, 3, 70, 129], 3, 128
    s = Setup(rng, lengths, d, H=2, L=2)
    pool, _ = _pool(rng, 2, 2, d, 500, F16)
    Q = dev(rng.standard_normal((2, 4, N, 8, d)), F16)
    tails = []
    for a, n in enumerate(lengths):
        k, v = np.zeros((2, 2, 130, d)), np.zeros((2, 2, 130, d))
        for t in range(n):
            k[:, :, t], v[:, :, t] = s.K[:, s.table[a, t // 16], :, t % 16], s.V[:, s.table[a, t // 16], :, t % 16]
        tails.append((dev(k, F16), dev(v, F16), n))
    want = pool.attend(Q, tails=tails, tail_causal=True)
    got = pool.attend_tree(Q, s.pages)
    # both are within 2e-3 of the exact result, and the second is rounded
    assert ((got.float() - want).abs() <= 4e-3 + 2.0 ** -11 * want.abs()).all()


def test_offsets_beyond_32_bits():
    """Pages far behind the first 4 GiB of a layer."""
    pk = _pk()
    NP, P, H, d = 70_000, 64, 4, 128
    pages = pk.Pages(1, H, d, NP, 2, 3, page_tokens=P)
    assert pages.K.numel() * 2 > 2 ** 32 and pages.K.numel() < 2 ** 32
    rng = np.random.default_rng(1)
    table = np.array([[NP - 1, 3, NP - 5], [NP - 2, 66_000, 1]], np.int32)
    lengths = np.array([150, 129], np.int32)
    K, V = rounded(rng.standard_normal((1, 279, H, d)), F16), rounded(rng.standard_normal((1, 279, H, d)), F16)
    pages.table.copy_(dev(table))
    pages.lengths.copy_(dev(lengths))
    slots = np.concatenate([table[a, np.arange(n) // P] * P + np.arange(n) % P for a, n in enumerate(lengths)]).astype(np.int32)
    pages.write(dev(K, F16), dev(V, F16), dev(slots))
    Q = rounded(rng.standard_normal((1, 2, 2, 2 * H, d)), F16)
    got = pages.attend_tree(dev(Q, F16))
    small = np.zeros((1, 279, H, 1, d)), np.zeros((1, 279, H, 1, d))      # the same tokens in pages of one
    small[0][:, :, :, 0], small[1][:, :, :, 0] = K, V
    where = np.full((2, 150), -1, np.int32)
    where[0], where[1, :129] = np.arange(150), 150 + np.arange(129)
    out, mag, big = U.attend(Q, *small, where, lengths, [2, 2], None)
    err = np.abs(got.double().cpu().numpy() - out)
    assert (err <= U.bound(out, mag, big, d, F16, 150, 6.0)).all()
    # an accepted path's vectors move across them
    parents = np.array([[-1, 0, 0], [-1, 0, 0]], np.int32)
    tok, fol = np.array([[7, 8, 9], [7, 8, 9]], np.int32), np.array([[9, 0, 5], [8, 1, 0]], np.int32)
    path, n, after, kept = pages.accept(dev(tok), dev(fol), dev(parents))
    assert path.tolist() == [[0, 2, -1], [0, 1, -1]] and after.tolist() == [5, 1] and kept.tolist() == [149, 128]
    assert torch.equal(pages.K[0, NP - 5, :, 148 - 128], dev(K, F16)[0, 149])
    assert torch.equal(pages.V[0, 66_000, :, 127 - 64], dev(V, F16)[0, 150 + 127])


# ------------------------------------------------------------------------------------------------------ tables and slots
def _state(pages):
    return [x.cpu().numpy() for x in (pages.table, pages.lengths, pages.free, pages.free_state)]


@pytest.mark.parametrize("A,P,MB,NP,n_slots", [(1, 8, 4, 4, 40), (3, 16, 9, 20, 100), (64, 24, 7, 200, 4096), (65, 16, 7, 333, 700),
                                               (1025, 8, 12, 5000, 40_000), (4096, 8, 5, 9000, 9001)])
def test_resize_in_many_steps(A, P, MB, NP, n_slots):
    """Agents grow and shrink at random, sometimes beyond what is free or what the table holds."""
    pk = _pk()
    rng = np.random.default_rng(A)
    pages = pk.Pages(1, 1, 64, NP, A, MB, page_tokens=P)
    slots = torch.empty(n_slots, dtype=torch.int32, device="cuda")
    offsets = torch.empty(A + 1, dtype=torch.int32, device="cuda")
    for step in range(8):
        table, lengths, ring, state = _state(pages)
        targets = np.where(rng.random(A) < 0.3, lengths, rng.integers(-2, MB * P + 3, A))
        if step == 3:
            targets = np.zeros(A)
        if step == 5:
            targets = lengths + rng.integers(0, 3, A)
        targets = targets.astype(np.int32)
        want = U.resize(table, lengths, ring, state, targets, P, n_slots)
        if step % 3 == 2:
            pages.resize(dev(targets))
        else:
            pages.resize(dev(targets), slots, offsets)
            np.testing.assert_array_equal(slots.cpu().numpy(), want[4])
            np.testing.assert_array_equal(offsets.cpu().numpy(), want[5])
        for got, ref in zip(_state(pages), want):
            np.testing.assert_array_equal(got, ref)
        # every page is somewhere once
        t, _, ring, (first, count) = _state(pages)
        there = np.concatenate([t[t >= 0], ring[(first + np.arange(count)) % NP]])
        assert sorted(there) == list(range(NP))


def test_resize_with_a_broken_state_stays_inside_its_arrays():
    """Whatever the device arrays hold: table, ring, slots and offsets keep to their bounds (guards on both sides)."""
    pk = _pk()
    rng = np.random.default_rng(2)
    A, MB, NP = 70, 5, 40
    raw = torch.full((10_000,), 0x5C5C5C5C, dtype=torch.int32, device="cuda")
    pages = pk.Pages(1, 1, 64, NP, A, MB, page_tokens=8)
    views, at = [], 1000
    for n in (A * MB, A, NP, 2, 333, A + 1):
        views.append(raw[at:at + n])
        at += n + 500
    inside = torch.zeros_like(raw, dtype=torch.bool)
    for v in views:
        inside[v.storage_offset():v.storage_offset() + v.numel()] = True
    pages._desc.table_dev, pages._desc.lengths_dev, pages._desc.free_dev, pages._desc.free_state_dev = (v.data_ptr() for v in views[:4])
    for _ in range(4):
        for v in views:
            v.copy_(dev(rng.integers(-2 ** 31, 2 ** 31, v.numel()).astype(np.int32)))
        views[1].copy_(dev(rng.integers(-10, 60, A).astype(np.int32)))
        pages.resize(dev(rng.integers(-5, 60, A).astype(np.int32)), views[4], views[5])
        torch.cuda.synchronize()
        assert bool((raw[~inside] == 0x5C5C5C5C).all())


@pytest.mark.parametrize("d,H,P,dtype,src", [(64, 3, 8, F16, F16), (128, 2, 24, BF16, BF16), (256, 1, 16, F16, torch.float32),
                                             (128, 8, 16, BF16, torch.float32)])
def test_write(d, H, P, dtype, src):
    pk = _pk()
    rng = np.random.default_rng(d + H)
    L, NP, n = 3, 11, 37
    pages = pk.Pages(L, H, d, NP, 1, 1, page_tokens=P, dtype=dtype)
    pages.K.fill_(7.0)
    pages.V.fill_(8.0)
    kv = torch.from_numpy(rng.standard_normal((L, n, 2, H, d)) * 3).to(src).cuda()
    slots = rng.permutation(NP * P)[:n].astype(np.int32)
    slots[[0, 5, 9, 36]] = [-1, NP * P, 2 ** 31 - 1, -2 ** 31]
    wantK, wantV = pages.K.clone(), pages.V.clone()
    for i, at in enumerate(slots):
        if 0 <= at < NP * P:
            wantK[:, at // P, :, at % P], wantV[:, at // P, :, at % P] = kv[:, i, 0].to(dtype), kv[:, i, 1].to(dtype)
    pages.write(kv[1:, :, 0], kv[1:, :, 1], dev(slots), layer_begin=1)       # side by side, two of three layers
    assert torch.equal(pages.K[1:], wantK[1:]) and torch.equal(pages.V[1:], wantV[1:])
    assert bool((pages.K[0] == 7).all()) and bool((pages.V[0] == 8).all())
    pages.write(kv[:, :, 0].contiguous(), kv[:, :, 1].contiguous(), dev(slots))
    assert torch.equal(pages.K, wantK) and torch.equal(pages.V, wantV)
    head_major = kv.permute(0, 3, 2, 1, 4).contiguous().permute(0, 3, 2, 1, 4)      # [layers, heads, 2, tokens, d] in memory
    pages.K.fill_(7.0)
    pages.V.fill_(8.0)
    pages.write(head_major[:, :, 0], head_major[:, :, 1], dev(slots))
    assert torch.equal(pages.K, wantK) and torch.equal(pages.V, wantV)
    pages.write(kv[:, :0, 0], kv[:, :0, 1], dev(slots[:0]))                     # nothing
    single = kv[:, 7:8, 0].as_strided((L, 1, H, d), (kv.stride(0), 1, kv.stride(3), 1))     # a stride that nothing is read with
    pages.write(single, kv[:, 7:8, 1], dev(np.array([5], np.int32)))
    assert torch.equal(pages.K[:, 0, :, 5], kv[:, 7, 0].to(dtype)) and torch.equal(pages.V[:, 0, :, 5], kv[:, 7, 1].to(dtype))
    one = kv[:, 3:4, 0].expand(L, 2, H, d)                                       # one token for two slots
    pages.write(one, one, dev(np.array([4, 6], np.int32)))
    assert torch.equal(pages.K[:, 4 // P, :, 4 % P], kv[:, 3, 0].to(dtype)) and torch.equal(pages.V[:, 6 // P, :, 6 % P], kv[:, 3, 0].to(dtype))


# ------------------------------------------------------------------------------------------------------ trees
@pytest.mark.parametrize("A,N", [(1, 1), (3, 2), (5, 63), (4, 64), (2, 65), (3, 128), (2, 129), (2, 193), (7, 256)])
@pytest.mark.parametrize("near", [1, 3, 300])
def test_masks_and_depths(A, N, near):
    pk = _pk()
    rng = np.random.default_rng(A + N)
    parents = U.random_trees(rng, A, N, near)
    odd = rng.random((A, N)) < 0.1      # further roots, and numbers that are no earlier draft
    parents[odd] = rng.choice([-1, -9, N, 2 ** 31 - 1, -2 ** 31], odd.sum())
    parents[0, N // 2] = N // 2
    counts = rng.integers(-1, N + 2, A).astype(np.int32)
    for c, used in ((None, np.full(A, N)), (dev(counts), counts)):
        seen = U.reach(parents, used)
        mask, depth = pk.tree_masks(dev(parents), c)
        np.testing.assert_array_equal(mask.cpu().numpy(), U.pack(seen))
        np.testing.assert_array_equal(depth.cpu().numpy(), np.maximum(seen.sum(-1) - 1, 0))


@pytest.mark.parametrize("d,N,P,dtype", [(64, 1, 8, F16), (128, 7, 16, BF16), (64, 64, 24, F16), (256, 40, 8, BF16), (128, 256, 32, F16)])
def test_accept(d, N, P, dtype):
    rng = np.random.default_rng(N + d)
    lengths = [N, N + 1, N + 37, N + 100, max(N - 1, 0), 0, N + 5, N + 64]
    A = len(lengths)
    s = Setup(rng, lengths, d, H=3, P=P, L=2, dtype=dtype)
    parents = U.random_trees(rng, A, N, near=3)
    parents[1] = np.arange(-1, N - 1)       # a chain, accepted whole
    tokens = rng.integers(0, 3, (A, N)).astype(np.int32)     # few tokens: children that agree twice, and none
    following = rng.integers(0, 3, (A, N)).astype(np.int32)
    tokens[1], following[1] = 5, 5
    counts = np.array([N, N, N, max(N - 2, 0), N, N, 0, N], np.int32)
    path, accepted, after, kept = U.accept(tokens, following, parents, counts, s.lengths)
    Kb, Vb = s.pages.K.clone(), s.pages.V.clone()
    for c in (dev(counts), None):
        if c is None:
            path, accepted, after, kept = U.accept(tokens, following, parents, np.full(A, N), s.lengths)
        s.pages.K.copy_(Kb)
        s.pages.V.copy_(Vb)
        wantK, wantV = Kb.clone(), Vb.clone()
        for a in range(A):
            start = kept[a] - accepted[a]
            for k in range(accepted[a]):
                src, dst = start + path[a, k], start + k
                ps, pd = s.table[a, src // P], s.table[a, dst // P]
                wantK[:, pd, :, dst % P], wantV[:, pd, :, dst % P] = Kb[:, ps, :, src % P], Vb[:, ps, :, src % P]
        got = s.pages.accept(dev(tokens), dev(following), dev(parents), c)
        for x, ref in zip(got, (path, accepted, after, kept)):
            np.testing.assert_array_equal(x.cpu().numpy(), ref)
        assert torch.equal(s.pages.K.view(torch.int16), wantK.view(torch.int16)) and torch.equal(s.pages.V.view(torch.int16), wantV.view(torch.int16))


def test_accept_skips_pages_that_are_not_there():
    rng = np.random.default_rng(0)
    s = Setup(rng, [20, 20], 64, P=8, MB=4)
    s.table[0, 2] = 99
    s.table[1, 1] = -1
    s.load()
    before = s.pages.K.clone()
    N = 12
    parents = np.tile(np.where(np.arange(N) < 10, -1, [0] * 10 + [0, 10]), (2, 1)).astype(np.int32)
    tokens, following = np.full((2, N), 4, np.int32), np.full((2, N), 4, np.int32)
    path, n, _, _ = s.pages.accept(dev(tokens), dev(following), dev(parents))
    assert n.tolist() == [3, 3] and path[0, :4].tolist() == [0, 10, 11, -1]
    # agent 0: both sources lie in the missing page; agent 1: both targets do
    assert torch.equal(s.pages.K.view(torch.int16), before.view(torch.int16))


# ------------------------------------------------------------------------------------------------------ together
class Step:
    """A model-less decode step of three agents over a shared pool: room, masks, writes and attention layer by layer, acceptance,
    and the pages that are not needed go back."""

    def __init__(self, seed, dtype=F16, stream_pool=None):
        pk = _pk()
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.L, self.H, self.G, self.d, self.A, self.N = 2, 2, 3, 128, 3, 9
        r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        self.pool = pk.Pool(self.L, self.H, self.d, 400).bind()
        self.pool.encode(r(self.L, self.H, 400, self.d).to(dtype), r(self.L, self.H, 400, self.d).to(dtype))
        self.pages = pk.Pages(self.L, self.H, self.d, 40, self.A, 8, page_tokens=8, dtype=dtype)
        self.pages.K.zero_()
        self.pages.V.zero_()
        self.counts = torch.tensor([9, 4, 7], dtype=torch.int32, device="cuda")
        self.kept = torch.zeros(self.A, dtype=torch.int32, device="cuda")
        self.target = torch.zeros(self.A, dtype=torch.int32, device="cuda")
        self.slots = torch.empty(self.A * self.N, dtype=torch.int32, device="cuda")
        self.offsets = torch.empty(self.A + 1, dtype=torch.int32, device="cuda")
        self.parents = dev(U.random_trees(np.random.default_rng(seed), self.A, self.N, 3))
        self.tokens = torch.zeros((self.A, self.N), dtype=torch.int32, device="cuda")
        self.following = torch.zeros((self.A, self.N), dtype=torch.int32, device="cuda")
        self.kv = r(self.L, self.A * self.N, 2, self.H, self.d).to(dtype)
        self.Q = r(self.L, self.A, self.N, self.H * self.G, self.d).to(dtype)
        self.out = torch.zeros_like(self.Q)
        self.result = None

    def inputs(self, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(1000 + seed)
        for x in (self.kv, self.Q):
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        for x in (self.tokens, self.following):
            x.copy_(torch.randint(0, 2, x.shape, device="cuda", generator=g))

    def run(self):
        pk = _pk()
        torch.add(self.kept, self.counts, out=self.target)
        self.pages.resize(self.target, self.slots, self.offsets)
        mask, depth = pk.tree_masks(self.parents, self.counts)
        for l in range(self.L):
            self.pages.write(self.kv[l:l + 1, :, 0], self.kv[l:l + 1, :, 1], self.slots, layer_begin=l, layer_end=l + 1)
            self.pool.attend_tree(self.Q[l:l + 1], self.pages, self.out[l:l + 1], counts=self.counts, mask=mask, layer_begin=l, layer_end=l + 1)
        self.result = self.pages.accept(self.tokens, self.following, self.parents, self.counts)
        self.kept.copy_(self.result[3])
        self.pages.resize(self.kept)

    def state(self):
        p = self.pages
        return [x.clone() for x in (self.out, self.kept, self.slots, p.table, p.lengths, p.free, p.free_state, p.K, p.V, *self.result)]


def test_a_step_against_the_plain_forms():
    s = Step(1)
    p = s.pages
    Kd, Vd = s.pool.decode(torch.float32)
    dense = Kd.double().cpu().numpy(), Vd.double().cpu().numpy()
    for step in range(3):
        s.inputs(step)
        was = _state(p)
        table, lengths, ring, state, slots, _ = U.resize(*was, s.kept.cpu().numpy() + s.counts.cpu().numpy(), 8, 27)
        K, V = p.K.double().cpu().numpy(), p.V.double().cpu().numpy()
        kv = s.kv.double().cpu().numpy()
        for i, at in enumerate(slots):
            if at >= 0:
                K[:, at // 8, :, at % 8], V[:, at // 8, :, at % 8] = kv[:, i, 0], kv[:, i, 1]
        counts = s.counts.cpu().numpy()
        seen = U.reach(s.parents.cpu().numpy(), counts)
        Q = s.Q.double().cpu().numpy()
        out, mag, big = U.attend(Q, K, V, table, lengths, counts, seen, dense)
        s.run()
        err = np.abs(s.out.double().cpu().numpy() - out)
        assert (err <= U.bound(out, mag, big, 128, F16, 500, 6.0, pool=True)).all()
        want = U.accept(*(x.cpu().numpy() for x in (s.tokens, s.following, s.parents)), counts, lengths)
        for x, ref in zip(s.result, want):
            np.testing.assert_array_equal(x.cpu().numpy(), ref)
        back = U.resize(table, lengths, ring, state, want[3], 8, 0)
        for got, ref in zip(_state(p), back):
            np.testing.assert_array_equal(got, ref)


def test_captured_steps_follow_the_lengths():
    """One captured step, replayed: lengths, tables and masks are those of the replay.  Two graphs, captured on one stream and
    replayed on two, do not disturb each other, and eager steps run in between."""
    eager, graphed = [Step(1), Step(2)], [Step(1), Step(2)]
    for s in eager + graphed:
        s.inputs(0)
        s.run()
    torch.cuda.synchronize()
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s in graphed:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                s.run()
            graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for step in range(1, 5):
        for s in eager + graphed:
            s.inputs(step)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        for s in eager:
            s.run()
        torch.cuda.synchronize()
        for a, b in zip(eager, graphed):
            for x, y in zip(a.state(), b.state()):
                assert torch.equal(x, y)


def test_what_the_binding_refuses():
    pk = _pk()
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    for bad in (dict(page_tokens=12), dict(agents=5000), dict(head_dim=96), dict(max_blocks=0)):
        kw = dict(dict(layers=1, kv_heads=2, head_dim=64, pages=4, agents=3, max_blocks=2, page_tokens=8), **bad)
        with pytest.raises(pk.PolyKVError):
            pk.Pages(**kw)
    with pytest.raises(TypeError):
        pk.Pages(1, 2, 64, 4, 3, 2, device="cpu")
    with pytest.raises(TypeError):
        pk.Pages(1, 2, 64, 4, 3, 2, dtype=torch.float32)
    p = pk.Pages(1, 2, 64, 4, 3, 2, page_tokens=8)
    Q = torch.zeros((1, 3, 2, 4, 64), dtype=F16, device="cuda")
    for call in (lambda: p.resize(i32(4)), lambda: p.resize(i32(3).long()), lambda: p.resize(i32(6)[::2]), lambda: p.resize(i32(3).cpu()),
                 lambda: p.resize(i32(3), i32(5), i32(3)), lambda: p.attend_tree(Q.to(BF16)), lambda: p.attend_tree(Q, Q.float()),
                 lambda: p.attend_tree(Q, counts=i32(2)), lambda: p.attend_tree(Q, mask=i32(3, 2, 1)),
                 lambda: p.attend_tree(Q.transpose(2, 3).contiguous().transpose(2, 3)), lambda: pk.tree_masks(i32(3, 4).cpu()),
                 lambda: pk.tree_masks(i32(3, 4), i32(4)), lambda: p.accept(i32(3, 4), i32(3, 5), i32(3, 4)),
                 lambda: p.write(Q[:, 0, :, :2].float().half().to(BF16), Q[:, 0, :, :2].to(BF16), i32(2))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: p.attend_tree(Q[:, :2]), lambda: p.attend_tree(Q[0]), lambda: p.attend_tree(Q, Q[:, :, :1]), lambda: p.accept(i32(2, 4), i32(2, 4), i32(2, 4)),
                 lambda: p.attend_tree(Q, layer_begin=1), lambda: p.write(Q[:, 0], Q[:, 0], i32(2)),
                 lambda: p.write(Q[:, 0, :, :2], Q[:, 0, :, :2].contiguous(), i32(2)), lambda: p.write(Q[:, 0, :, :2, ::2], Q[:, 0, :, :2, ::2], i32(2))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(pk.PolyKVError):
        p.attend_tree(torch.zeros((1, 3, 257, 4, 64), dtype=F16, device="cuda"))
    with pytest.raises(pk.PolyKVError):
        pk.Pool(1, 2, 64, 40).attend_tree(Q, p)          # nothing bound


def test_on_another_stream_and_twice():
    """A side stream given by name; the same call again gives the same bits."""
    rng = np.random.default_rng(4)
    s = Setup(rng, [300, 10, 64], 128, L=2)
    pool, _ = _pool(rng, 2, 2, 128, 900, F16)
    Q = dev(rng.standard_normal((2, 3, 4, 8, 128)), F16)
    want = pool.attend_tree(Q, s.pages, page_splits=2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [pool.attend_tree(Q, s.pages, page_splits=2, stream=side) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(want, x) for x in got)


def test_a_captured_stream_that_is_not_the_current_one():
    """A call on a stream by name, which is being captured while another is current: the graph has a workspace of its own, and its
    replays leave alone the one of that stream's eager calls."""
    rng = np.random.default_rng(6)
    s = Setup(rng, [300, 10, 64], 128, L=2)
    pool, _ = _pool(rng, 2, 2, 128, 900, F16)
    Q, other_Q = (dev(rng.standard_normal((2, 3, 4, 8, 128)), F16) for _ in range(2))
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    for known in (True, False):       # with and without an eager workspace of the stream
        s.pages._workspaces.clear()
        want = pool.attend_tree(Q, s.pages, page_splits=2)
        torch.cuda.synchronize()
        if known:
            pool.attend_tree(Q, s.pages, page_splits=2, stream=side)
            torch.cuda.synchronize()
        graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(Q)
        with torch.cuda.stream(side):
            graph.capture_begin()
            with torch.cuda.stream(other):
                pool.attend_tree(Q, s.pages, out, page_splits=2, stream=side)
            graph.capture_end()
        pool.attend_tree(other_Q, s.pages, page_splits=2, stream=side)
        torch.cuda.synchronize()
        eager = s.pages._workspaces[side.cuda_stream]
        eager.fill_(0x5C)
        for _ in range(3):
            out.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(other):
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            assert bool((eager == 0x5C).all())


@pytest.mark.parametrize("d,nodes,group,layers", [(64, 4, 2, 1), (128, 40, 4, 1), (64, 8, 2, 100), (128, 20, 1, 100), (128, 20, 2, 100), (256, 3, 2, 100), (256, 90, 2, 60)])
@pytest.mark.parametrize("page_splits", [1, 2])
def test_in_place(d, nodes, group, layers, page_splits):
    """The output may be the queries themselves, in every form, with and without a pool."""
    rng = np.random.default_rng(d + nodes)
    pages = _pk().Pages(layers, 2, d, 60, 3, 20, dtype=F16)
    g = torch.Generator(device="cuda").manual_seed(1)
    for x in (pages.K, pages.V):
        x.normal_(generator=g)
    pages.table.copy_(dev(rng.permutation(60).astype(np.int32)).view(3, 20))
    pages.lengths.copy_(dev(np.array([310, nodes, 150], np.int32)))
    Q = torch.randn((layers, 3, nodes, 2 * group, d), device="cuda", generator=g).half()
    pool = _pk().Pool(layers, 2, d, 200).bind()
    pool.encode(*(torch.randn((layers, 2, 200, d), device="cuda", generator=g).half() for _ in range(2)))
    for call in (pages.attend_tree, lambda q, out, **kw: pool.attend_tree(q, pages, out, **kw)):
        want = call(Q, torch.empty_like(Q), page_splits=page_splits)
        both = Q.clone()
        assert call(both, both, page_splits=page_splits) is both
        assert torch.equal(both, want)


def test_a_workspace_on_another_device():
    """(The first of its places that the call may look at; one GPU is enough to see that.)"""
    class Elsewhere:
        device, is_cuda, dtype = torch.device("cuda", 1), True, torch.uint8

    p = _pk().Pages(1, 2, 64, 4, 3, 2, page_tokens=8)
    with pytest.raises(ValueError, match="workspace is on cuda:1"):
        p.attend_tree(torch.zeros((1, 3, 2, 4, 64), dtype=F16, device="cuda"), workspace=Elsewhere())
