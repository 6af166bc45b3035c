"""Plain implementations (numpy, 64 bits) of continuations in pages and of drafted decoding, and inputs for their tests."""
import numpy as np
import torch


def resize(table, lengths, ring, state, targets, P, n_slots):
    """One resize, agent by agent, page by page.  Returns the new (table, lengths, ring, state), slots and offsets."""
    table, lengths, ring = table.copy(), lengths.copy(), ring.copy()
    (A, MB), NP = table.shape, len(ring)
    first, count = (int(x) for x in state)
    asked = taken = given = 0
    slots, offsets = [], [0]
    for a in range(A):
        old, new = int(lengths[a]), int(targets[a])
        if not 0 <= new <= MB * P:
            new = old
        have, want = -(-old // P), -(-new // P)
        if want > have:
            asked += want - have
            if asked > count:
                new = old
            else:
                for b in range(have, want):
                    table[a, b] = ring[(first + taken) % NP]
                    taken += 1
        for b in range(want, have):
            ring[(first + count + given) % NP] = table[a, b]
            table[a, b] = -1
            given += 1
        lengths[a] = new
        slots += [int(table[a, t // P]) * P + t % P for t in range(old, new)]
        offsets.append(len(slots))
    out = np.full(n_slots, -1, np.int32)
    out[:min(n_slots, len(slots))] = slots[:n_slots]
    return table, lengths, ring, np.array([(first + taken) % NP, count - taken + given], np.int32), out, np.array(offsets, np.int32)


def reach(parents, counts):
    """[agents, nodes, nodes] truth values: draft j is draft i or one of its ancestors."""
    A, N = parents.shape
    r = np.zeros((A, N, N), bool)
    for a in range(A):
        for i in range(min(max(int(counts[a]), 0), N)):
            r[a, i, i] = True
            if 0 <= parents[a, i] < i:
                r[a, i] |= r[a, parents[a, i]]
    return r


def pack(seen):
    """Truth values [agents, nodes, nodes] as masks int64 [agents, nodes, words]."""
    A, N, _ = seen.shape
    W = -(-N // 64)
    bits = np.zeros((A, N, W * 64), np.uint64)
    bits[:, :, :N] = seen
    return (bits.reshape(A, N, W, 64) << np.arange(64, dtype=np.uint64)).sum(-1, dtype=np.uint64).view(np.int64)


def accept(tokens, following, parents, counts, lengths):
    A, N = tokens.shape
    path = np.full((A, N), -1, np.int32)
    accepted, after, kept = (np.zeros(A, np.int32) for _ in range(3))
    for a in range(A):
        n = min(max(int(counts[a]), 0), N, int(lengths[a]))
        at, k, last = (0 if n else None), 0, -1
        while at is not None:
            path[a, k], last, k = at, at, k + 1
            at = next((c for c in range(at + 1, n) if parents[a, c] == at and tokens[a, c] == following[a, at]), None)
        accepted[a], after[a], kept[a] = k, following[a, last] if k else -1, lengths[a] - n + k
    return path, accepted, after, kept


def attend(Q, K, V, table, lengths, counts, seen, pool=None, layer_begin=0, scale=None):
    """Q [layers, agents, nodes, q_heads, d]; pages K, V; seen [agents, nodes, nodes] or None (a draft sees what is not
    behind it); pool: (K, V) [layers, heads, tokens, d] of all layers.  Returns the output in 64 bits, the same sums over
    |v|, and the largest sum |q| |k| scale of a row."""
    L, A, N, qh, d = Q.shape
    H, P = K.shape[2], K.shape[3]
    G = qh // H
    scale = d ** -0.5 if scale is None else scale
    out, mag, big = np.zeros(Q.shape), np.zeros(Q.shape), np.zeros(Q.shape[:-1])
    for a in range(A):
        n = int(lengths[a])
        c = min(max(int(counts[a]), 0), N, n)
        see = np.zeros((N, n), bool)
        for i in range(c):
            see[i, :n - c] = True
            see[i, n - c:] = seen[a, i, :c] if seen is not None else np.arange(c) <= i
        pg, off = table[a, np.arange(n) // P], np.arange(n) % P
        there = (pg >= 0) & (pg < K.shape[1])
        see &= there
        for l in range(L):
            for h in range(H):
                k = np.where(there[:, None], K[layer_begin + l, np.where(there, pg, 0), h, off].astype(np.float64), 0.0)
                v = np.where(there[:, None], V[layer_begin + l, np.where(there, pg, 0), h, off].astype(np.float64), 0.0)
                w = see
                if pool is not None:
                    k, v = np.concatenate([pool[0][layer_begin + l, h], k]), np.concatenate([pool[1][layer_begin + l, h], v])
                    w = np.concatenate([np.ones((N, pool[0].shape[2]), bool), see], 1)
                for g in range(G):
                    q = Q[l, a, :, h * G + g].astype(np.float64)
                    for i in range(N):
                        kk, vv = k[w[i]], v[w[i]]
                        if not len(kk):
                            continue
                        s = kk @ q[i] * scale
                        e = np.exp(s - s.max())
                        out[l, a, i, h * G + g] = e @ vv / e.sum()
                        mag[l, a, i, h * G + g] = e @ np.abs(vv) / e.sum()
                        big[l, a, i, h * G + g] = (np.abs(kk) @ np.abs(q[i])).max() * scale
    return out, mag, big


def bound(out, mag, big, d, dtype, tokens, vmax, pool=False):
    """How far a result may be from the 64-bit one.  A probability is rounded by half a step of fp16 (bfloat16: two terms, 2^-17);
    below fp16's normal range by 2^-25, with the row's largest at 1 or above.  A score of d products in fp32 is off by
    (d + 2) 2^-24 of its absolute sum, which enters numerator and denominator; sums over tokens likewise.  The output is rounded
    by half a step.  The pool's part is held to the 2e-3 of its own tests."""
    half = torch.finfo(dtype).eps / 2
    prob = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -16
    inner = mag * (prob + 2 * (d + 2) * 2.0 ** -24 * big[..., None] + 2 * (tokens + 8) * 2.0 ** -24) + tokens * 2.0 ** -25 * vmax
    if pool:
        inner = inner + 2e-3
    tiny = torch.finfo(dtype).tiny * torch.finfo(dtype).eps   # a step below the normal range
    return half * (np.abs(out) + inner) + inner + tiny


def random_trees(rng, A, N, near=8):
    p = np.full((A, N), -1, np.int32)
    for i in range(1, N):
        p[:, i] = i - rng.integers(1, min(i, near) + 1, A)
    return p


def scattered(rng, lengths, P, MB, spare=3):
    """A block table whose pages lie anywhere: (table, pages)."""
    held = [-(-int(n) // P) for n in lengths]
    pages = sum(held) + spare
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((len(held), MB), -1, np.int32)
    at = 0
    for a, n in enumerate(held):
        table[a, :n] = order[at:at + n]
        at += n
    return table, pages
