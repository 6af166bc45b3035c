"""Rows most of whose weight, or a good part of it, lies on many tokens far below the first: probabilities below fp16's normal
range, summed in numerator and denominator."""
import numpy as np
import pytest
import torch

import tree_util as U

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("below", [9.0, 14.5, 16.0, 18.0])
@pytest.mark.parametrize("d,nodes,group,agents,heads,tokens,dtype", [
    (64, 1, 4, 1, 2, 4000, F16), (128, 5, 4, 1, 2, 4000, F16), (256, 2, 2, 1, 2, 4000, F16), (128, 2, 2, 1, 2, 4000, BF16),    # four waves share the rows
    (64, 2, 2, 5, 110, 500, F16), (128, 2, 4, 5, 110, 500, F16), (128, 5, 4, 5, 110, 500, F16), (256, 2, 2, 5, 110, 500, F16),  # a wave has its rows
    (64, 20, 2, 3, 110, 500, F16), (128, 20, 2, 3, 110, 500, F16), (256, 10, 4, 5, 110, 500, F16), (128, 32, 4, 5, 110, 500, F16),  # tiles through LDS
])
def test_many_small_weights_below_a_large_one(below, d, nodes, group, agents, heads, tokens, dtype):
    """The first token's score lies `below` powers of two above all others of the row.  Its values are -1, the others' about 1, so
    that weight lost on one side of the fraction only shows.

    A probability e = 2^(s - m) is off by 2^-11 of itself, below 2^-14 by 2^-25, as one error in numerator and denominator alike:
    sum |error| |v - out| / sum e <= (2^-11 + n 2^-25 / sum e) 2 max|v|.  Scores in fp32: (d + 2) 2^-24 of the largest |q| |k|
    scale, natural units, in the same way.  The sums: n 2^-24 each.  bfloat16: 2^-16 in place of 2^-11 and 2^-25.  The output: half
    a step.  Another reference than the first token's score only makes weights larger."""
    from paper_2604_24971_amd import polykv as pk
    rng = np.random.default_rng(int(10 * below) + d + nodes)
    half = float(torch.finfo(dtype).eps) / 2
    t = lambda x: torch.from_numpy(np.asarray(x)).to(dtype)  # noqa: E731
    n = tokens + nodes
    P, MB = 16, -(-n // 16)
    pages = pk.Pages(1, heads, d, agents * MB, agents, MB, dtype=dtype)
    table = rng.permutation(agents * MB).astype(np.int32).reshape(agents, MB)
    direction = rng.choice([-1.0, 1.0], (heads, d))                 # the queries' of a head
    scale = d ** -0.5
    up = below * np.log(2) / (d * scale)                            # the first key's component along it
    K = (0.02 * rng.standard_normal((agents, n, heads, d))).astype(np.float32)
    K[:, 0] += up * direction
    V = (1.0 + 0.1 * rng.standard_normal((agents, n, heads, d))).astype(np.float32)
    V[:, 0] = -1.0
    K, V = t(K), t(V)
    order = torch.from_numpy(table).long()
    full = torch.zeros((agents * MB, heads, P, d), dtype=dtype)
    for name, x in (("K", K), ("V", V)):
        padded = torch.zeros((agents, MB * P, heads, d), dtype=dtype)
        padded[:, :n] = x
        full[order.reshape(-1)] = padded.view(agents * MB, P, heads, d).transpose(1, 2)
        getattr(pages, name)[0].copy_(full)
    pages.table.copy_(torch.from_numpy(table))
    pages.lengths.fill_(n)
    size = 1.0 + 0.05 * rng.random((agents, nodes, heads, group))
    Q = t(size[..., None] * direction[:, None])                     # [agents, nodes, heads, group, d]
    got = pages.attend_tree(Q.reshape(1, agents, nodes, heads * group, d).cuda(), page_splits=1)
    got = got.view(agents, nodes, heads, group, d).permute(0, 2, 1, 3, 4).double()
    q = Q.permute(0, 2, 1, 3, 4).double().cuda().reshape(agents * heads, nodes * group, d)
    k, v = (x.permute(0, 2, 1, 3).double().cuda().reshape(agents * heads, n, d) for x in (K, V))
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
    i = torch.arange(n, device="cuda")
    draft = torch.arange(nodes * group, device="cuda") // group
    s = torch.where(i <= tokens + draft[:, None], s, -torch.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True))
    L = e.sum(-1, keepdim=True)
    want = (torch.matmul(e, v) / L).view(got.shape)
    lost = float((1 - 1 / L).median())                              # the share of the small weights
    assert lost > tokens * 2.0 ** -below / 4 / (1 + tokens * 2.0 ** -below)
    vmax = float(v.abs().max())
    big = float(torch.matmul(q.abs(), k.abs().transpose(1, 2).contiguous()).max()) * scale
    rel, small = (2.0 ** -11, 2.0 ** -25) if dtype == F16 else (2.0 ** -16, 0.0)
    inner = 2 * vmax * (rel + small * n / L + 2 * (d + 2) * 2.0 ** -24 * big + 2 * n * 2.0 ** -24)
    tol = inner.view(agents, heads, nodes, group, 1) + half * (want.abs() + inner.view(agents, heads, nodes, group, 1))
    err = (got - want).abs()
    assert bool((err <= tol).all()), "off by %g where %g is allowed; small weights are %g of a row" % (float(err.max()), float(tol.min()), lost)
