"""Agents whose continuation could not grow: places and counts by agent, and steps in which some have no drafts."""
import numpy as np
import pytest
import torch

import tree_util as U

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def _pk():
    from paper_2604_24971_amd import polykv as pk
    return pk


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _state(pages):
    return [x.cpu().numpy() for x in (pages.table, pages.lengths, pages.free, pages.free_state)]


def by_agent(was, targets, P, n):
    """The plain resize, its slots spread over rows of n: (state after it, slots [agents, n], granted)."""
    *after, slots, offsets = U.resize(*was, targets, P, int(np.maximum(targets - was[1], 0).sum()) + 1)
    granted = np.diff(offsets).astype(np.int32)
    rows = np.full((len(targets), n), -1, np.int32)
    for a, k in enumerate(granted):
        rows[a, :min(k, n)] = slots[offsets[a]:offsets[a] + min(k, n)]
    return after, rows, granted


@pytest.mark.parametrize("A,P,MB,NP,n", [(1, 8, 4, 4, 40), (3, 16, 9, 20, 5), (64, 24, 7, 200, 64), (65, 16, 7, 333, 1), (300, 8, 12, 2000, 33),
                                         (4096, 8, 5, 9000, 9), (5, 16, 40, 150, 1300)])
def test_places_by_agent(A, P, MB, NP, n):
    pk = _pk()
    rng = np.random.default_rng(A + n)
    pages = pk.Pages(1, 1, 64, NP, A, MB, page_tokens=P)
    raw = torch.full((A * n + 200,), 0x5C5C5C5C, dtype=torch.int32, device="cuda")
    slots, granted = raw[100:100 + A * n].view(A, n), torch.empty(A, dtype=torch.int32, device="cuda")
    refused = 0
    for step in range(8):
        was = _state(pages)
        targets = np.where(rng.random(A) < 0.3, was[1], rng.integers(-2, MB * P + 3, A))
        if step == 3:
            targets = np.zeros(A)
        if step % 2:
            targets = np.where(rng.random(A) < 0.9, was[1] + rng.integers(0, n + 2, A), targets)
        targets = targets.astype(np.int32)
        after, rows, grew = by_agent(was, targets, P, n)
        refused += int(((targets > was[1]) & (grew == 0)).sum())
        if step == 6:
            pages.resize(dev(targets), granted=granted)
        else:
            pages.resize(dev(targets), slots, granted=granted)
            np.testing.assert_array_equal(slots.cpu().numpy(), rows)
        np.testing.assert_array_equal(granted.cpu().numpy(), grew)
        for got, ref in zip(_state(pages), after):
            np.testing.assert_array_equal(got, ref)
        assert bool((raw[:100] == 0x5C5C5C5C).all()) and bool((raw[100 + A * n:] == 0x5C5C5C5C).all())
    assert refused or A < 64


@pytest.mark.parametrize("dtype,graph", [(F16, False), (BF16, False), (F16, True)])
def test_steps_in_which_agents_have_no_room(dtype, graph):
    """Four agents, drafts of each in rows of their own.  Agent 1 is at the end of its block table (targets out of range), and
    after two steps the pages run out.  A refused agent has no drafts in the
    step, keeps its tokens, and nobody's keys and values are moved or overwritten for it."""
    pk = _pk()
    rng = np.random.default_rng(5)
    L, H, G, d, A, N, P, MB, NP = 2, 2, 2, 64, 4, 6, 8, 6, 14
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    pool = pk.Pool(L, H, d, 90).bind()
    pool.encode(r(L, H, 90, d).to(dtype), r(L, H, 90, d).to(dtype))
    dense = tuple(x.double().cpu().numpy() for x in pool.decode(torch.float32))
    pages = pk.Pages(L, H, d, NP, A, MB, page_tokens=P, dtype=dtype)
    for x in (pages.K, pages.V):
        x.copy_(r(*x.shape))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    slots, granted, targets, kept = i32(A, N), i32(A), i32(A), i32(A)
    tokens, following = i32(A, N), i32(A, N)
    parents = dev(U.random_trees(rng, A, N, 2))
    kv, Q = r(2, L, A * N, H, d).to(dtype), r(L, A, N, H * G, d).to(dtype)
    out, result = torch.zeros_like(Q), [i32(A, N), i32(A), i32(A), i32(A)]
    pages.resize(dev(np.array([5, 43, 9, 20], np.int32)))
    kept.copy_(pages.lengths)

    def step():
        torch.add(kept, N, out=targets)
        pages.resize(targets, slots, granted=granted)
        mask, _ = pk.tree_masks(parents, granted)
        pages.write(kv[0], kv[1], slots.view(-1))
        pool.attend_tree(Q, pages, out, counts=granted, mask=mask)
        for x, y in zip(result, pages.accept(tokens, following, parents, granted)):
            x.copy_(y)
        kept.copy_(result[3])
        pages.resize(kept)

    run = step
    if graph:
        mask, _ = pk.tree_masks(parents, granted)
        pool.attend_tree(Q, pages, out, counts=granted, mask=mask)      # (the library is warm)
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
        run = captured.replay
    refused = np.zeros(A, int)
    for i in range(7):
        kv.copy_(r(*kv.shape))
        Q.copy_(r(*Q.shape))
        tokens.copy_(dev(rng.integers(0, 2, (A, N)).astype(np.int32)))
        following.copy_(dev(rng.integers(0, 2, (A, N)).astype(np.int32)))
        was = _state(pages)
        after, rows, grew = by_agent(was, was[1] + N, P, N)
        K, V = pages.K.double().cpu().numpy(), pages.V.double().cpu().numpy()
        new = kv.double().cpu().numpy()
        for j, at in enumerate(rows.reshape(-1)):
            if at >= 0:
                K[:, at // P, :, at % P], V[:, at // P, :, at % P] = new[0, :, j], new[1, :, j]
        seen = U.reach(parents.cpu().numpy(), grew)
        want = U.attend(Q.double().cpu().numpy(), K, V, after[0], after[1], grew, seen, dense)
        run()
        np.testing.assert_array_equal(granted.cpu().numpy(), grew)
        np.testing.assert_array_equal(slots.cpu().numpy(), rows)
        tol = U.bound(*want, d, dtype, 90 + MB * P, 6.0, pool=True)
        assert (np.abs(out.double().cpu().numpy() - want[0]) <= tol).all()
        path = U.accept(*(x.cpu().numpy() for x in (tokens, following, parents)), grew, after[1])
        for x, ref in zip(result, path):
            np.testing.assert_array_equal(x.cpu().numpy(), ref)
        for a in range(A):
            if grew[a] == 0:
                refused[a] += 1
                assert path[1][a] == 0 and path[2][a] == -1 and path[3][a] == was[1][a]
            before = after[1][a] - grew[a]
            for k in range(path[1][a]):     # (the moves, one after the other)
                src, dst = before + path[0][a, k], before + k
                s, t = (after[0][a, x // P] for x in (src, dst))
                K[:, t, :, dst % P], V[:, t, :, dst % P] = K[:, s, :, src % P].copy(), V[:, s, :, src % P].copy()
        assert np.array_equal(pages.K.double().cpu().numpy(), K) and np.array_equal(pages.V.double().cpu().numpy(), V)
        for got, ref in zip(_state(pages), U.resize(*after, path[3], P, 0)):
            np.testing.assert_array_equal(got, ref)
    assert list(refused) == [0, 7, 3, 5]


def test_what_the_binding_refuses():
    pk = _pk()
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    p = pk.Pages(1, 2, 64, 4, 3, 2, page_tokens=8)
    for call in (lambda: p.resize(i32(3), i32(3, 4), granted=i32(4)), lambda: p.resize(i32(3), i32(4, 3), granted=i32(3)),
                 lambda: p.resize(i32(3), i32(3, 8)[:, ::2], granted=i32(3)), lambda: p.resize(i32(3), i32(3, 4).long(), granted=i32(3)),
                 lambda: p.resize(i32(3), granted=i32(3).cpu())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: p.resize(i32(3), i32(12), granted=i32(3)), lambda: p.resize(i32(3), i32(3, 4), i32(4), granted=i32(3))):
        with pytest.raises(ValueError):
            call()
    x = i32(3)
    with pytest.raises(pk.PolyKVError):
        p.resize(x, granted=x)
