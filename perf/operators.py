"""Operators of drafted (speculative) decoding over the shared pool, with the agents' private continuations in pages.

A step of N agents, each with up to `nodes` drafted tokens that form a tree:
  resize   block tables and slot maps on the GPU: every agent's continuation grows by its drafts, and shrinks again
  masks    which drafts a draft sees (its ancestors and itself), as bits, and how deep it sits, from the tree's parents
  write    keys and values of new tokens go to their slots in the pages
  attend   softmax attention of every draft over the shared pool, its agent's private tokens and the drafts it sees
  accept   the path of drafts that the model agrees with, and the moves of its keys and values to where they stay

Tensors: pages [layers, pages, kv_heads, page_tokens, head_dim]; block table [agents, max_blocks]; lengths [agents];
queries [layers, agents, nodes, q_heads, head_dim]; masks int64 [agents, nodes, words of 64 drafts].
Shapes and value distributions are those of `paper_2604_24971_amd/workloads.py` and `cases.py`.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
# Lloyd-Max levels of N(0,1) at 3 bits, ascending: the pool's value codebook.
CENTROIDS = (-2.15194570, -1.34390928, -0.75600528, -0.24509418, 0.24509418, 0.75600528, 1.34390928, 2.15194570)


def _case(name, op, **kw):
    return dict({"name": name, "op": op}, **kw)


def listed():
    return [
        # one layer of a model's decode loop: 15 agents, 16 drafts each, in the middle of their answers
        _case("attend-one-layer", "attend", layers=1, kv_heads=8, group=4, head_dim=128, agents=15, nodes=16, tokens=4096,
              private=96, page=16, dtype="f16"),
        # the same step with all layers in one call, bfloat16, longer answers
        _case("attend-all-layers", "attend", layers=32, kv_heads=8, group=4, head_dim=128, agents=15, nodes=8, tokens=4096,
              private=300, page=16, dtype="bf16"),
        # agents that share nothing and hold long contexts of their own, wide trees
        _case("attend-long-private", "attend", layers=4, kv_heads=8, group=4, head_dim=128, agents=16, nodes=32, tokens=0,
              private=7194, page=64, dtype="f16"),
        # plain decoding, one token an agent, no query groups; more agents than dense tails allow
        _case("attend-single-token", "attend", layers=24, kv_heads=32, group=1, head_dim=64, agents=100, nodes=1, tokens=1851,
              private=120, page=24, dtype="f16"),
        # block tables of the step of 15 agents; of a server's many requests, prompts arriving among them
        _case("resize-step", "resize", agents=15, grow=16, private=300, page=16),
        _case("resize-many-requests", "resize", agents=1024, grow=600, private=4096, page=16),
        # the drafts' keys and values of one layer; prompts of several requests in all layers
        _case("write-step", "write", layers=1, kv_heads=8, head_dim=128, agents=15, new=16, page=16, dtype="f16"),
        _case("write-prompts", "write", layers=32, kv_heads=8, head_dim=128, agents=4, new=1851, page=16, dtype="bf16"),
        # the trees of 15 agents; many agents with the largest trees
        _case("masks-step", "masks", agents=15, nodes=16),
        _case("masks-many", "masks", agents=512, nodes=256),
        # the accepted paths of 15 agents; many agents with long drafts
        _case("accept-step", "accept", layers=32, kv_heads=8, head_dim=128, agents=15, nodes=16, private=300, page=16, dtype="bf16"),
        _case("accept-long-drafts", "accept", layers=24, kv_heads=32, head_dim=64, agents=64, nodes=100, private=250, page=24, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend", "resize", "write", "masks", "accept"])
    page = rng.choice([8, 16, 24, 32, 64, 128])
    kv_heads, group, head_dim = rng.choice([(4, 1, 64), (32, 1, 64), (8, 4, 128), (8, 4, 128), (2, 5, 128), (8, 2, 256)])
    dtype = rng.choice(["f16", "bf16"])
    if op == "resize":
        return {"op": op, "agents": _log_int(rng, 1, 1024), "grow": _log_int(rng, 1, 600), "private": _log_int(rng, 1, 4096),
                "page": page}
    if op == "masks":
        return {"op": op, "agents": _log_int(rng, 1, 512), "nodes": _log_int(rng, 1, 256)}
    if op == "write":
        case = {"op": op, "layers": _log_int(rng, 1, 32), "kv_heads": kv_heads, "head_dim": head_dim,
                "agents": _log_int(rng, 1, 64), "new": _log_int(rng, 1, 1851), "page": page, "dtype": dtype}
        most = 32 * 8 * 128 * 4 * 1851
        case["new"] = max(1, min(case["new"], most // (kv_heads * head_dim * case["agents"])))
        case["layers"] = max(1, min(case["layers"], most // (kv_heads * head_dim * case["agents"] * case["new"])))
        return case
    if op == "accept":
        case = {"op": op, "layers": _log_int(rng, 1, 32), "kv_heads": kv_heads, "head_dim": head_dim,
                "agents": _log_int(rng, 1, 64), "nodes": _log_int(rng, 1, 128), "private": _log_int(rng, 1, 500), "page": page,
                "dtype": dtype}
        case["layers"] = max(1, min(case["layers"], 24 * 32 * 64 * 64 * 350 //
                                    (kv_heads * head_dim * case["agents"] * (case["nodes"] + case["private"]))))
        return case
    case = {"op": op, "layers": _log_int(rng, 1, 32), "kv_heads": kv_heads, "group": group, "head_dim": head_dim,
            "agents": _log_int(rng, 1, 100), "nodes": rng.choice([1, 1, 2, 4, _log_int(rng, 1, 64), _log_int(rng, 1, 128)]),
            "tokens": rng.choice([0, _log_int(rng, 100, 7194), _log_int(rng, 100, 7194)]),
            "private": rng.choice([_log_int(rng, 1, 300), _log_int(rng, 1, 7194)]), "page": page, "dtype": dtype}
    # no more scores, private tokens or pool tokens than the listed cases have
    while True:
        rows = case["agents"] * case["nodes"] * group
        ctx = case["private"] + case["nodes"]
        each = kv_heads * max(rows * (case["tokens"] + ctx) / (15 * 8 * 4 * 4400), case["agents"] * ctx * head_dim / (16 * 7226 * 128 / 8),
                              case["tokens"] * head_dim / (4096 * 128))
        most = int(32 * 8 // each)
        if most >= 1:
            case["layers"] = min(case["layers"], most)
            return case
        case["agents"] = max(1, case["agents"] // 2)
        case["private"] = max(1, case["private"] // 2)


# ------------------------------------------------------------------------------------------------ sizes of a case
def _contexts(c):
    # the agents are at different places of their answers: from half of `private` to all of it
    return [c["private"] - (7 * a) % (c["private"] // 2 + 1) for a in range(c["agents"])]


def _counts(c):
    # drafts of each agent: from half of `nodes` to all of them
    return [c["nodes"] - (3 * a) % (c["nodes"] // 2 + 1) for a in range(c["agents"])]


def _new(c):
    # new tokens of each agent, likewise
    return [c["new"] - (5 * a) % (c["new"] // 2 + 1) for a in range(c["agents"])]


def _grown(c):
    # tokens for which each agent's continuation takes room, likewise
    return [c["grow"] - (11 * a) % (c["grow"] // 2 + 1) for a in range(c["agents"])]


def _blocks(tokens, page):
    return -(-tokens // page)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed, device):
    g = torch.Generator(device=device)
    g.manual_seed(1000003 * int(seed) + 7)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _tables(held, max_blocks, spare, g):
    """A block table whose pages lie anywhere, and the free pages: (table, ring of free pages, pages)."""
    used = sum(held)
    pages = used + spare
    order = torch.randperm(pages, generator=g)
    table = torch.full((len(held), max_blocks), -1, dtype=torch.int32)
    at = 0
    for a, n in enumerate(held):
        table[a, :n] = order[at:at + n].int()
        at += n
    free = torch.full((pages,), -1, dtype=torch.int32)
    free[:spare] = order[used:].int()
    return table.to(DEVICE), free.to(DEVICE), pages


def _parents(c, g):
    """Trees in which a node hangs from one of the eight before it; node 0 is the root."""
    i = torch.arange(c["nodes"])
    back = (torch.rand((c["agents"], c["nodes"]), generator=g) * torch.clamp(i, max=8)).long() + 1
    return torch.where(i > 0, i - back, torch.full_like(back, -1)).int()


def _pages(c, lengths, g, cpu):
    """Pages of all layers with the agents' tokens somewhere in them."""
    held = [_blocks(n, c["page"]) for n in lengths]
    table, free, pages = _tables(held, max(held), 3, cpu)
    shape = (c["layers"], pages, c["kv_heads"], c["page"], c["head_dim"])
    K = torch.empty(shape, dtype=DTYPES[c["dtype"]], device=DEVICE)
    V = torch.empty_like(K)
    r = lambda *s: torch.randn(s, device=DEVICE, generator=g)  # noqa: E731
    for l in range(c["layers"]):
        K[l] = r(*shape[1:]) * torch.exp(0.5 * r(1, c["kv_heads"], 1, c["head_dim"]))
        V[l] = r(*shape[1:]) * torch.exp(0.3 * r(pages, c["kv_heads"], c["page"], 1))
    state = _ints([0, 3])
    return {"K": K, "V": V, "table": table, "lengths": _ints(lengths), "free": free, "free_state": state}


def _hadamard(n, dtype):
    i = torch.arange(n, device=DEVICE)
    x = i[:, None] & i[None, :]
    ones = (x[:, :, None] >> torch.arange(8, device=DEVICE) & 1).sum(-1)
    return (1 - 2 * (ones & 1)).to(dtype)


def _pool(c, g):
    """A shared context in the pool's format, and the dense tensors that it is made of: keys as 8-bit codes with an fp16
    scale for 32 of them, values as 3-bit codes of their rotated coordinates.  The dense values are the decoded ones, so
    that what the pool makes of them are these codes."""
    L, H, T, d = c["layers"], c["kv_heads"], c["tokens"], c["head_dim"]
    dt = DTYPES[c["dtype"]]
    r = lambda *s: torch.randn(s, device=DEVICE, generator=g)  # noqa: E731
    s = {"K": torch.empty((L, H, T, d), dtype=dt, device=DEVICE), "V": torch.empty((L, H, T, d), dtype=dt, device=DEVICE),
         "k_codes": torch.empty((L, H, T, d), dtype=torch.int8, device=DEVICE),
         "k_scales": torch.empty((L, H, T, d // 32), dtype=torch.float16, device=DEVICE),
         "v_codes": torch.empty((L, H, T, d), dtype=torch.uint8, device=DEVICE)}
    levels = torch.tensor(CENTROIDS, device=DEVICE)
    rotate = _hadamard(d, torch.float32) / math.sqrt(d)
    for l in range(L):
        gain = torch.exp(0.5 * r(H, 1, d))
        gain = torch.where(torch.rand((H, 1, d), device=DEVICE, generator=g) < 0.01, gain * 8.0, gain)
        K = (r(H, T, d) * gain).to(dt)
        blocks = K.float().view(H, T, d // 32, 32)
        scale = (blocks.abs().amax(-1, keepdim=True) / 127.0).half()
        s["K"][l] = K
        s["k_scales"][l] = scale[..., 0]
        s["k_codes"][l] = torch.round(blocks * (1.0 / scale.float())).view(H, T, d).to(torch.int8)
        code = torch.bucketize(r(H, T, d) * torch.exp(0.3 * r(H, T, 1)), (levels[1:] + levels[:-1]) / 2)
        s["v_codes"][l] = code.to(torch.uint8)
        s["V"][l] = (levels[code] @ rotate).to(dt)
    return s


def prepare(case, seed):
    c = dict(case)
    g, cpu = _gen(seed, DEVICE), _gen(seed, "cpu")
    s = {"case": c}
    if c["op"] == "masks":
        s["parents"], s["counts"] = _parents(c, cpu).to(DEVICE), _ints(_counts(c))
    if c["op"] == "resize":
        now = _contexts(c)
        then = [n + k for n, k in zip(now, _grown(c))]
        held, most = [_blocks(n, c["page"]) for n in now], max(_blocks(n, c["page"]) for n in then)
        # (a few pages too few: the last requests have to wait)
        spare = sum(_blocks(n, c["page"]) for n in then) - sum(held)
        spare = max(1, spare - spare // 16)
        table, free, pages = _tables(held, most, spare, cpu)
        s["pages"] = {"table": table, "lengths": _ints(now), "free": free, "free_state": _ints([0, spare]), "pages": pages}
        s["before"], s["after"] = _ints(now), _ints(then)
        s["slots"] = torch.empty((sum(then) - sum(now) + 5,), dtype=torch.int32, device=DEVICE)
        s["offsets"] = torch.empty((c["agents"] + 1,), dtype=torch.int32, device=DEVICE)
    if c["op"] == "write":
        s["pages"] = _pages(c, _new(c), g, cpu)
        n = sum(_new(c))
        a = torch.repeat_interleave(torch.arange(c["agents"]), torch.tensor(_new(c)))
        t = torch.cat([torch.arange(k) for k in _new(c)])
        slots = s["pages"]["table"].cpu()[a, t // c["page"]] * c["page"] + t % c["page"]
        s["slots"] = torch.cat([slots, torch.full((3,), -1)]).int().to(DEVICE)
        # keys and values as the projection leaves them, side by side for a token; three tokens of padding
        s["kv"] = torch.randn((c["layers"], n + 3, 2, c["kv_heads"], c["head_dim"]), device=DEVICE, generator=g).to(DTYPES[c["dtype"]])
    if c["op"] in ("attend", "accept"):
        counts = _counts(c)
        s["counts"] = _ints(counts)
        s["pages"] = _pages(c, [n + k for n, k in zip(_contexts(c), counts)], g, cpu)
        parents = _parents(c, cpu)
    if c["op"] == "accept":
        tokens = torch.randint(0, 32000, (c["agents"], c["nodes"]), generator=cpu)
        following = torch.randint(0, 32000, (c["agents"], c["nodes"]), generator=cpu)
        # the model mostly goes on as one of the drafts does
        agree = (torch.rand((c["agents"], c["nodes"]), generator=cpu) < 0.8) & (parents >= 0)
        for i in range(c["nodes"]):
            at = parents[:, i].clamp(min=0).long()[:, None]
            following.scatter_(1, at, torch.where(agree[:, i:i + 1], tokens[:, i:i + 1], following.gather(1, at)))
        s["parents"], s["tokens"], s["following"] = (x.int().to(DEVICE) for x in (parents, tokens, following))
    if c["op"] == "attend":
        shape = (c["layers"], c["agents"], c["nodes"], c["kv_heads"] * c["group"], c["head_dim"])
        s["Q"] = torch.randn(shape, device=DEVICE, generator=g).to(DTYPES[c["dtype"]])
        s["out"] = torch.empty_like(s["Q"])
        s["mask"] = _masks(parents.to(DEVICE), s["counts"])[0]
        if c["tokens"]:
            s["pool"] = _pool(c, g)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program of the framework holds instead of the plain tensors: its pages, and the encoded pool."""
    from paper_2604_24971_amd import polykv as pk
    c, p = s["case"], s.get("pages")
    if p is not None:
        pages = p["K"].shape[1] if "K" in p else p["pages"]
        s["pages"] = pk.Pages(c.get("layers", 1), c.get("kv_heads", 1), c.get("head_dim", 64), pages, p["table"].shape[0],
                              p["table"].shape[1], page_tokens=c["page"], dtype=DTYPES[c.get("dtype", "f16")])
        for name, x in p.items():
            if name != "pages":
                getattr(s["pages"], name).copy_(x)
    if "pool" in s:
        pool = pk.Pool(c["layers"], c["kv_heads"], c["head_dim"], c["tokens"]).bind()
        pool.encode(s["pool"]["K"], s["pool"]["V"])
        s["pool"] = pool


# ------------------------------------------------------------------------------------------------ plain forms
def _reach(parents, counts):
    """reach[a, i, j]: draft j is draft i or one of its ancestors.  A parent that is no earlier draft is none."""
    A, N = parents.shape
    i = torch.arange(N, device=parents.device)
    there = i < counts[:, None]
    up = torch.where((parents >= 0) & (parents < i), parents, -1)
    step = (up[:, :, None] == i) & there[:, :, None]
    reach = (step | torch.eye(N, dtype=torch.bool, device=parents.device)) & there[:, :, None]
    for _ in range(max(1, (N - 1).bit_length())):   # paths of twice the length
        reach = torch.bmm(reach.float(), reach.float()) > 0
    return reach


def _masks(parents, counts):
    reach = _reach(parents, counts)
    A, N, _ = reach.shape
    W = -(-N // 64)
    bits = torch.nn.functional.pad(reach, (0, 64 * W - N)).view(A, N, W, 64).long()
    mask = (bits << torch.arange(64, device=parents.device)).sum(-1)
    depth = (reach.sum(-1) - 1).clamp(min=0)
    return mask, depth.int()


def _resize(p, targets, slots, offsets, P):
    NP, (A, MB) = p["pages"], p["table"].shape
    dev = targets.device
    length, target, (first, count) = p["lengths"].long(), targets.long(), p["free_state"].long()
    ok = (target >= 0) & (target <= MB * P)
    target = torch.where(ok, target, length)
    have, want = (length + P - 1) // P, (target + P - 1) // P
    need = (want - have).clamp(min=0)
    granted = (need == 0) | (need.cumsum(0) <= count)
    target, want = torch.where(granted, target, length), torch.where(granted, want, have)
    take, give = (want - have).clamp(min=0), (have - want).clamp(min=0)
    b = torch.arange(MB, device=dev)
    new = (b >= have[:, None]) & (b < want[:, None])
    old = (b >= want[:, None]) & (b < have[:, None])
    fresh = p["free"][(first + (take.cumsum(0) - take - have)[:, None] + b) % NP]
    back = torch.where(old, (first + count + (give.cumsum(0) - give - want)[:, None] + b) % NP, NP)
    ring = torch.cat([p["free"], p["free"][:1]]).scatter(0, back.reshape(-1), p["table"].reshape(-1))
    p["free"].copy_(ring[:NP])
    p["table"].copy_(torch.where(new, fresh, torch.where(old, -1, p["table"])))
    p["lengths"].copy_(target)
    p["free_state"].copy_(torch.stack([(first + take.sum()) % NP, count - take.sum() + give.sum()]))
    if slots is None:
        return
    grow = (target - length).clamp(min=0)
    end = grow.cumsum(0)
    offsets[0] = 0
    offsets[1:] = end
    i = torch.arange(slots.shape[0], device=dev)
    a = torch.searchsorted(end, i, right=True).clamp(max=A - 1)
    t = (length + grow - end)[a] + i
    page = p["table"][a, (t // P).clamp(max=MB - 1)].long()
    slots.copy_(torch.where((i < end[-1]) & (page >= 0) & (page < NP), page * P + t % P, -1))


def _write(p, K, V, slots):
    n, P = p["K"].shape[1], p["K"].shape[3]
    there = (slots >= 0) & (slots < n * P)
    at = slots[there].long()
    p["K"][:, at // P, :, at % P] = K[:, there].transpose(0, 1)
    p["V"][:, at // P, :, at % P] = V[:, there].transpose(0, 1)


def _accept(p, tokens, following, parents, counts):
    P, N = p["K"].shape[3], tokens.shape[1]
    i = torch.arange(N, device=tokens.device)
    count = torch.minimum(counts, p["lengths"]).clamp(min=0)
    there = i < count[:, None]
    up = torch.where((parents >= 0) & (parents < i) & there, parents, -1).long()
    agreed = (up >= 0) & (tokens == following.gather(1, up.clamp(min=0)))
    first = ~((up[:, :, None] == up[:, None, :]) & agreed[:, None, :] & (i < i[:, None])).any(-1)   # of a node's children
    good = (agreed & first) | (i == 0)
    reach = _reach(parents, count)
    taken = there & ~(reach & ~good[:, None, :]).any(-1) & reach[:, :, 0]
    accepted = taken.sum(-1)
    at = torch.where(taken, taken.cumsum(-1) - 1, N)
    path = torch.full((tokens.shape[0], N + 1), -1, dtype=torch.int64, device=tokens.device).scatter(1, at, i.expand_as(at))
    path = path[:, :N]
    last = path.gather(1, (accepted - 1).clamp(min=0)[:, None])[:, 0]
    following = torch.where(accepted > 0, following.gather(1, last.clamp(min=0)[:, None])[:, 0], -1)
    before = p["lengths"] - count
    moved = path >= 0
    a = torch.arange(tokens.shape[0], device=tokens.device)[:, None].expand_as(path)[moved]
    src, dst = (before[:, None] + path)[moved], (before[:, None] + i)[moved]
    ps, pd = p["table"][a, src // P].long(), p["table"][a, dst // P].long()
    p["K"][:, pd, :, dst % P] = p["K"][:, ps, :, src % P]
    p["V"][:, pd, :, dst % P] = p["V"][:, ps, :, src % P]
    return path.int(), accepted.int(), following.int(), (before + accepted).int()


def _attend(s):
    c, p, Q = s["case"], s["pages"], s["Q"]
    L, A, N, _, d = Q.shape
    H, G, P = c["kv_heads"], c["group"], c["page"]
    q = Q.float().view(L, A, N, H, G, d).permute(0, 3, 1, 2, 4, 5).reshape(L, H, A, N * G, d).contiguous() / math.sqrt(d)
    # the private tokens, dense: [layers, kv_heads, agents, tokens, head_dim]
    t = torch.arange(p["table"].shape[1] * P, device=Q.device)
    page = p["table"].long()[:, t // P].clamp(min=0)
    k, v = (p[x][:, page, :, t % P].float().permute(2, 3, 0, 1, 4).contiguous() for x in ("K", "V"))
    before = (p["lengths"] - s["counts"])[:, None]
    draft = (t - before).clamp(0, N - 1)
    word = s["mask"].gather(2, (draft // 64)[:, None, :].expand(A, N, -1))
    seen = (t < before)[:, None, :] | ((t >= before) & (t < p["lengths"][:, None]))[:, None, :] & ((word >> (draft % 64)[:, None, :]) & 1 > 0)
    seen = seen & (torch.arange(N, device=Q.device) < s["counts"][:, None])[:, :, None]
    seen = seen[:, :, None, :].expand(A, N, G, -1).reshape(A, N * G, -1)
    v = torch.where((t < p["lengths"][:, None])[:, :, None], v, 0.0)
    score = (q @ k.transpose(-1, -2)).masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    if "pool" in s:
        w = s["pool"]
        T = c["tokens"]
        levels = torch.tensor(CENTROIDS, device=Q.device)
        pk_ = (w["k_codes"].float().view(L, H, T, d // 32, 32) * w["k_scales"].float()[..., None]).view(L, H, T, d)
        pv = levels[w["v_codes"].int()] @ (_hadamard(d, torch.float32) / math.sqrt(d))
        shared = q.reshape(L, H, A * N * G, d) @ pk_.transpose(-1, -2)
        top = torch.maximum(top, shared.amax(-1).reshape(L, H, A, N * G, 1))
    top = top.masked_fill(top == -math.inf, 0.0)
    e = torch.exp(score - top)
    den, num = e.sum(-1, keepdim=True), e @ v
    if "pool" in s:
        e = torch.exp(shared - top.reshape(L, H, A * N * G, 1))
        den = den + e.sum(-1).reshape(L, H, A, N * G, 1)
        num = num + (e @ pv).reshape(L, H, A, N * G, d)
    out = torch.where(den > 0, num / den, 0.0)
    s["out"].copy_(out.reshape(L, H, A, N, G, d).permute(0, 2, 3, 1, 4, 5).reshape(Q.shape))
    return s["out"]


# ------------------------------------------------------------------------------------------------ a pass
def run(s):
    c = s["case"]
    p = s.get("pages")
    if c["op"] == "masks":
        if own:
            from paper_2604_24971_amd import polykv as pk
            return pk.tree_masks(s["parents"], s["counts"])
        return _masks(s["parents"], s["counts"])
    if c["op"] == "resize":      # the drafts' pages are taken, and go back after the step
        if own:
            p.resize(s["after"], s["slots"], s["offsets"])
            p.resize(s["before"])
            return s["slots"], s["offsets"], p.table, p.lengths, p.free, p.free_state
        _resize(p, s["after"], s["slots"], s["offsets"], c["page"])
        _resize(p, s["before"], None, None, c["page"])
        return s["slots"], s["offsets"], p["table"], p["lengths"], p["free"], p["free_state"]
    if c["op"] == "write":
        K, V = s["kv"][:, :, 0], s["kv"][:, :, 1]
        if own:
            p.write(K, V, s["slots"])
            return p.K, p.V
        _write(p, K, V, s["slots"])
        return p["K"], p["V"]
    if c["op"] == "accept":
        if own:
            path, accepted, following, kept = p.accept(s["tokens"], s["following"], s["parents"], s["counts"])
            return path, accepted, following, kept, p.K, p.V
        return (*_accept(p, s["tokens"], s["following"], s["parents"], s["counts"]), p["K"], p["V"])
    if own:
        if "pool" in s:
            return s["pool"].attend_tree(s["Q"], p, s["out"], counts=s["counts"], mask=s["mask"])
        return p.attend_tree(s["Q"], s["out"], counts=s["counts"], mask=s["mask"])
    return _attend(s)


def work(case):
    c = dict(case)
    if c["op"] == "masks":
        n = c["agents"] * c["nodes"]
        return {"bytes": n * (4 + 4 + 8 * _blocks(c["nodes"], 64)) + 4 * c["agents"], "flops": n}
    if c["op"] == "resize":
        grown = sum(_grown(c))
        # slots and offsets written, lengths and targets read and lengths written, pages taken and given back (the second
        # call has no slots)
        return {"bytes": 4 * grown + 28 * c["agents"] + 4 * 4 * grown / c["page"], "flops": grown}
    vector = 2 * c["layers"] * c["kv_heads"] * c["head_dim"] * 2     # bytes of a token's keys and values
    if c["op"] == "write":
        return {"bytes": sum(_new(c)) * (2 * vector + 4), "flops": 0}
    if c["op"] == "accept":
        # the paths depend on the drafts: in these trees about two of an agent's tokens move
        n = sum(_counts(c))
        return {"bytes": 16 * n + 2 * vector * 2 * c["agents"], "flops": n}
    lengths = [x + k for x, k in zip(_contexts(c), _counts(c))]
    rows = c["layers"] * c["kv_heads"] * c["group"] * c["agents"] * c["nodes"]
    d = c["head_dim"]
    packed = c["layers"] * c["kv_heads"] * c["tokens"] * (d + d // 16 + 3 * d // 8)
    private = sum(n * k for n, k in zip(lengths, _counts(c))) * c["layers"] * c["kv_heads"] * c["group"]
    return {"bytes": packed + sum(lengths) * vector + rows * d * 4, "flops": 4 * d * (rows * c["tokens"] + private)}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    c = dict(case)
    if c["op"] in ("masks", "resize"):
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    p = s["pages"]
    table, P = p["table"].cpu(), c["page"]
    if c["op"] == "write":
        K, V = p["K"].double(), p["V"].double()
        for i, at in enumerate(s["slots"].tolist()):
            if at >= 0:
                K[:, at // P, :, at % P] = s["kv"][:, i, 0].double()
                V[:, at // P, :, at % P] = s["kv"][:, i, 1].double()
        return K, V
    if c["op"] == "accept":
        K, V = p["K"].double(), p["V"].double()
        parents, tokens, following = (s[x].tolist() for x in ("parents", "tokens", "following"))
        for a, (ctx, n) in enumerate(zip(_contexts(c), _counts(c))):
            at, k = 0, 0
            while at is not None:
                src, dst = ctx + at, ctx + k
                for x in (K, V):
                    x[:, table[a, dst // P], :, dst % P] = x[:, table[a, src // P], :, src % P]
                at = next((j for j in range(n) if parents[a][j] == at and tokens[a][j] == following[a][at]), None)
                k += 1
        return None, None, None, None, K, V
    H, G, d = c["kv_heads"], c["group"], c["head_dim"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEVICE)
    mask = s["mask"].cpu().tolist()
    if c["tokens"]:
        w = s["pool"]
        levels = torch.tensor(CENTROIDS, dtype=torch.float64, device=DEVICE)
        turn = torch.ones((1, 1), dtype=torch.float64, device=DEVICE)
        while turn.shape[0] < d:
            turn = torch.cat([torch.cat([turn, turn], 1), torch.cat([turn, -turn], 1)], 0) / math.sqrt(2.0)
    # what each draft sees of its agent's own tokens
    views = []
    for a, (ctx, n) in enumerate(zip(_contexts(c), _counts(c))):
        see = torch.zeros((c["nodes"], ctx + n), dtype=torch.bool)
        for i in range(n):
            see[i, :ctx] = True
            for j in range(n):
                see[i, ctx + j] = (mask[a][i][j // 64] >> (j % 64)) & 1 == 1
        views.append(see.to(DEVICE))
    for l in range(c["layers"]):
        if c["tokens"]:
            key = w["k_codes"][l].double() * w["k_scales"][l].double().repeat_interleave(32, -1)
            value = torch.matmul(levels[w["v_codes"][l].long()], turn)
        for a, see in enumerate(views):
            t = torch.arange(see.shape[1])
            at = table[a, t // P].long().to(DEVICE)
            t = (t % P).to(DEVICE)
            k = p["K"][l].double()[at, :, t].transpose(0, 1).contiguous()      # [heads, tokens, head_dim]
            v = p["V"][l].double()[at, :, t].transpose(0, 1).contiguous()
            q = s["Q"][l, a].double().view(c["nodes"], H, G, d).permute(1, 2, 0, 3).contiguous()
            x = torch.matmul(q, k[:, None].transpose(-1, -2).contiguous()) * d ** -0.5
            x = torch.where(see, x, torch.full_like(x, -math.inf))
            if c["tokens"]:
                x = torch.cat([torch.matmul(q, key[:, None].transpose(-1, -2).contiguous()) * d ** -0.5, x], -1)
                v = torch.cat([value, v], 1)
            x = torch.exp(x - torch.clamp(x.amax(-1, keepdim=True), min=-1e300))
            y = torch.matmul(x, v[:, None]) / torch.clamp(x.sum(-1, keepdim=True), min=1e-300)
            out[l, a] = y.permute(2, 0, 1, 3).reshape(c["nodes"], H * G, d)
    return out
