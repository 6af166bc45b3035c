"""Continuations in pages and drafted decoding: host logic, sizes and refusals.  No kernel is launched."""
import ctypes as C

import pytest

pk = pytest.importorskip("paper_2604_24971_amd.polykv")
lib = pk.lib
P = C.c_void_p(0x10000)      # never dereferenced: every call below ends before a launch


def desc(**kw):
    d = dict(layers=2, kv_heads=2, head_dim=64, pages=10, page_tokens=16, agents=3, max_blocks=4, dtype=pk.F16, K_dev=P, V_dev=P,
             table_dev=P, lengths_dev=0x20000, free_dev=P, free_state_dev=P, ticket_dev=P)
    d.update(kw)
    return pk.PagesDesc(**{k: getattr(v, "value", v) for k, v in d.items()})


def params(**kw):
    d = dict(nodes=4, q_heads=4, layer_begin=0, layer_end=2, scale=0.0)
    d.update(kw)
    return pk.TreeParams(**d)


BAD_PAGES = [(dict(head_dim=96), pk.ESHAPE), (dict(layers=0), pk.ESHAPE), (dict(layers=40000, kv_heads=2), pk.ESHAPE), (dict(page_tokens=12), pk.ESHAPE),
             (dict(page_tokens=0), pk.ESHAPE), (dict(pages=0), pk.ESHAPE), (dict(pages=2 ** 27, page_tokens=16), pk.ESHAPE),
             (dict(pages=2 ** 26, page_tokens=16, kv_heads=4, layers=1), pk.ESHAPE), (dict(agents=0), pk.ESHAPE), (dict(agents=4097), pk.ESHAPE),
             (dict(max_blocks=0), pk.ESHAPE), (dict(max_blocks=2 ** 27), pk.ESHAPE), (dict(dtype=pk.F32), pk.EINVAL), (dict(table_dev=None), pk.EINVAL),
             (dict(lengths_dev=None), pk.EINVAL), (dict(table_dev=0x10002), pk.EINVAL)]


def calls(d, **kw):
    """Every entry point with this description."""
    p = params()
    return {
        "resize": lambda: lib.polykv_pages_resize(d, P, P, 10, P, None),
        "write": lambda: lib.polykv_pages_write(d, P, P, pk.F16, 5, 640, 128, 64, P, 0, 2, None),
        "attend": lambda: lib.pool_attend_tree(None, d, P, P, p, None),
        "accept": lambda: lib.polykv_pages_accept(d, P, P, P, P, 4, *([C.c_void_p(0x30000)] * 4), None),
    }


@pytest.mark.parametrize("bad,code", BAD_PAGES)
def test_descriptions_that_are_refused(bad, code):
    for name, call in calls(C.byref(desc(**bad))).items():
        assert call() == code, name
        assert lib.polykv_last_error()
    assert lib.pool_attend_tree_workspace(None, C.byref(desc(**bad)), C.byref(params())) == 0


def test_no_description():
    for name, call in calls(None).items():
        assert call() == pk.EINVAL, name
    for bad in (dict(K_dev=None), dict(V_dev=None), dict(K_dev=0x10008)):
        for name in ("write", "attend", "accept"):
            assert calls(C.byref(desc(**bad)))[name]() == pk.EINVAL


def test_resize_refusals():
    d = C.byref(desc())
    f = lib.polykv_pages_resize
    assert f(d, None, P, 10, P, None) == pk.EINVAL
    assert f(d, C.c_void_p(0x20000), P, 10, P, None) == pk.EINVAL          # the lengths themselves
    a, b, c = (C.c_void_p(0x40000 + 0x1000 * k) for k in range(3))
    for args in ((a, P, 10, c), (a, b, 10, P), (P, b, 10, c), (a, a, 10, c), (a, b, 10, a), (a, b, 10, b), (a, C.c_void_p(0x20000), 10, c)):
        assert f(d, *args, None) == pk.EINVAL                               # arrays that are also something else
    assert f(d, C.c_void_p(0x10002), b, 10, c, None) == pk.EINVAL
    assert f(d, a, b, -1, c, None) == pk.ESHAPE
    assert f(d, a, b, 2 ** 30 + 1, c, None) == pk.ESHAPE
    assert f(C.byref(desc(free_dev=None)), P, P, 10, P, None) == pk.EINVAL
    assert f(C.byref(desc(free_state_dev=None)), P, P, 10, P, None) == pk.EINVAL
    assert f(C.byref(desc(ticket_dev=None)), P, P, 10, P, None) == pk.EINVAL


def test_write_refusals():
    d = C.byref(desc())
    f = lib.polykv_pages_write
    ok = [d, P, P, pk.F16, 5, 640, 128, 64, P, 0, 2, None]

    def with_(**kw):
        names = ["d", "K", "V", "dtype", "tokens", "ls", "ts", "hs", "slots", "begin", "end", "stream"]
        return f(*(kw.get(n, x) for n, x in zip(names, ok)))

    assert with_(dtype=pk.BF16) == pk.EINVAL
    assert with_(tokens=-1) == pk.ESHAPE
    assert with_(tokens=2 ** 31 - 1) == pk.ESHAPE
    assert with_(K=None) == pk.EINVAL and with_(V=None) == pk.EINVAL and with_(slots=None) == pk.EINVAL
    assert with_(K=C.c_void_p(0x10008)) == pk.EINVAL and with_(slots=C.c_void_p(0x10001)) == pk.EINVAL
    assert with_(hs=-64) == pk.EINVAL and with_(ts=100) == pk.EINVAL and with_(ls=641) == pk.EINVAL
    assert with_(dtype=pk.F32, ts=130) == pk.EINVAL
    for begin, end in ((-1, 2), (0, 3), (1, 1), (2, 1)):
        assert with_(begin=begin, end=end) == pk.ESHAPE
    assert with_(tokens=0, K=None) == pk.OK             # nothing to do, nothing launched


def test_masks_refusals():
    f = lib.polykv_tree_masks
    assert f(None, P, 3, 4, P, P, None) == pk.EINVAL and f(P, P, 3, 4, None, P, None) == pk.EINVAL
    assert f(P, P, 0, 4, P, P, None) == pk.ESHAPE and f(P, P, 4097, 4, P, P, None) == pk.ESHAPE
    assert f(P, P, 3, 0, P, P, None) == pk.ESHAPE and f(P, P, 3, 257, P, P, None) == pk.ESHAPE
    assert f(P, P, 3, 4, C.c_void_p(0x10004), P, None) == pk.EINVAL
    a, b = C.c_void_p(0x40000), C.c_void_p(0x50000)
    for args in ((a, None, 3, 4, a, b), (a, None, 3, 4, b, a), (a, b, 3, 4, P, b), (a, b, 3, 4, b, P), (a, None, 3, 4, P, P)):
        assert f(*args, None) == pk.EINVAL                                  # an output that is an input, or both outputs


def test_accept_refusals():
    d = C.byref(desc())
    out = [C.c_void_p(0x30000 + 0x1000 * k) for k in range(4)]
    f = lib.polykv_pages_accept
    assert f(d, P, P, P, P, 0, *out, None) == pk.ESHAPE and f(d, P, P, P, P, 257, *out, None) == pk.ESHAPE
    for k in range(3):
        assert f(d, *[None if i == k else P for i in range(3)], P, 4, *out, None) == pk.EINVAL
    for k in range(4):
        assert f(d, P, P, P, P, 4, *[None if i == k else x for i, x in enumerate(out)], None) == pk.EINVAL
        assert f(d, P, P, P, P, 4, *[P if i == k else x for i, x in enumerate(out)], None) == pk.EINVAL          # an input
        assert f(d, P, P, P, P, 4, *[C.c_void_p(0x20000) if i == k else x for i, x in enumerate(out)], None) == pk.EINVAL      # lengths


def test_attend_refusals_and_sizes():
    d = C.byref(desc())
    f = lib.pool_attend_tree
    ws = dict(workspace_dev=0x100000, workspace_bytes=1 << 40)
    assert f(None, d, P, P, None, None) == pk.EINVAL
    for bad in (dict(nodes=0), dict(nodes=257), dict(q_heads=3), dict(q_heads=0), dict(layer_begin=-1), dict(layer_end=3), dict(layer_begin=2)):
        assert f(None, d, P, P, C.byref(params(**bad, **ws)), None) == pk.ESHAPE, bad
    for bad in (dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(kernel=9), dict(splits=-1), dict(page_splits=-1),
                dict(key_precision=5), dict(mask_dev=0x10004), dict(counts_dev=0x10001)):
        assert f(None, d, P, P, C.byref(params(**bad, **ws)), None) == pk.EINVAL, bad
    assert f(None, d, None, P, C.byref(params(**ws)), None) == pk.EINVAL and f(None, d, P, None, C.byref(params(**ws)), None) == pk.EINVAL
    assert f(None, d, C.c_void_p(0x10008), P, C.byref(params(**ws)), None) == pk.EINVAL
    # more rows per KV head than a pool takes; more workgroups than a launch takes
    assert f(None, C.byref(desc(agents=4096)), P, P, C.byref(params(nodes=256, q_heads=4, **ws)), None) == pk.ESHAPE
    assert f(None, C.byref(desc(agents=4096, layers=32767, pages=1, max_blocks=2 ** 20)), P, P,
             C.byref(params(nodes=1, layer_end=32767, page_splits=2 ** 19, **ws)), None) == pk.ESHAPE
    # workspace
    h = C.c_void_p()
    assert lib.pool_create(2, 2, 64, 100, C.byref(h)) == pk.OK
    rows = 3 * 4 * 2
    need = lib.pool_attend_tree_workspace(h, d, C.byref(params()))
    assert need >= 2 * 2 * rows * (64 + 2) * 4
    assert lib.pool_attend_tree_workspace(None, d, C.byref(params())) == 0          # complete in one launch
    split = lib.pool_attend_tree_workspace(None, d, C.byref(params(page_splits=2)))
    assert split == 0 or split >= 2 * (2 * 2 * rows * (64 + 2) * 4)
    assert f(h, d, P, P, C.byref(params(**ws)), None) == pk.ESTATE                      # never bound
    assert lib.pool_bind(h, P, 1 << 40) == pk.OK
    assert f(h, d, P, P, C.byref(params(**ws)), None) == pk.ESTATE                      # never encoded
    for other in ((1, 2, 64), (2, 1, 64), (2, 2, 128)):
        h2 = C.c_void_p()
        assert lib.pool_create(*other, 100, C.byref(h2)) == pk.OK
        assert lib.pool_attend_tree_workspace(h2, d, C.byref(params())) == 0
        assert b"the pool has" in lib.polykv_last_error()
        lib.pool_destroy(h2)
    lib.pool_destroy(h)
    d = C.byref(desc(max_blocks=64))
    need = lib.pool_attend_tree_workspace(None, d, C.byref(params(page_splits=4)))
    assert need > 0
    assert f(None, d, P, P, C.byref(params(page_splits=4)), None) == pk.EINVAL
    assert f(None, d, P, P, C.byref(params(page_splits=4, workspace_dev=0x100080, workspace_bytes=need)), None) == pk.EINVAL
    assert f(None, d, P, P, C.byref(params(page_splits=4, workspace_dev=0x100000, workspace_bytes=need - 1)), None) == pk.ENOMEM


def test_a_closed_pool_is_not_an_absent_one():
    """The C calls take a pool of NULL for none; the binding does not hand a closed one on to them."""
    pool = pk.Pool(2, 2, 64, 100)
    pool.close()
    pages = pk.Pages.__new__(pk.Pages)     # (its tensors would be on a GPU; no call gets as far as them)
    for call in (lambda: pool.attend_tree(None, pages), lambda: pages.attend_tree_workspace_bytes(None, pool)):
        with pytest.raises(pk.PolyKVError) as e:
            call()
        assert e.value.status == pk.EINVAL and "closed" in str(e.value)


def test_resize_by_agent_refusals():
    d = C.byref(desc())
    f = lib.polykv_pages_resize_by_agent
    a, b, c = (C.c_void_p(0x40000 + 0x1000 * k) for k in range(3))
    for bad, code in BAD_PAGES:
        assert f(C.byref(desc(**bad)), a, b, 4, c, None) == code
    assert f(None, a, b, 4, c, None) == pk.EINVAL and f(d, None, b, 4, c, None) == pk.EINVAL
    for args in ((C.c_void_p(0x20000), b, 4, c), (a, P, 4, c), (a, b, 4, P), (P, b, 4, c), (a, a, 4, c), (a, b, 4, a), (a, b, 4, b), (a, b, 4, C.c_void_p(0x20000))):
        assert f(d, *args, None) == pk.EINVAL                               # arrays that are also something else
    assert f(d, C.c_void_p(0x10002), b, 4, c, None) == pk.EINVAL and f(d, a, b, 4, C.c_void_p(0x40001), None) == pk.EINVAL
    for per_agent in (-1, -2 ** 31, 2 ** 30 // 3 + 1, 2 ** 31 - 1):
        assert f(d, a, b, per_agent, c, None) == pk.ESHAPE
    assert f(C.byref(desc(free_dev=None)), a, b, 4, c, None) == pk.EINVAL
    assert f(C.byref(desc(free_state_dev=None)), a, b, 4, c, None) == pk.EINVAL
    assert f(C.byref(desc(ticket_dev=None)), a, b, 4, c, None) == pk.EINVAL


def test_refusals_name_the_call():
    """Also those of the planner that pool_attend and pool_attend_tree share."""
    d = C.byref(desc())
    for bad in (dict(scale=-1.0), dict(q_heads=3), dict(kernel=9), dict(layer_end=3), dict(key_precision=5)):
        p = C.byref(params(workspace_dev=0x100000, workspace_bytes=1 << 40, **bad))
        assert lib.pool_attend_tree(None, d, P, P, p, None) != pk.OK
        assert lib.polykv_last_error().startswith(b"pool_attend_tree: "), bad
    h = C.c_void_p()
    assert lib.pool_create(2, 2, 64, 100, C.byref(h)) == pk.OK
    a = pk.AttendParams(agents=1, q_per_agent=1, q_heads=3, layer_end=2)
    assert lib.pool_attend_workspace(h, C.byref(a)) == 0 and lib.polykv_last_error().startswith(b"pool_attend: ")
    lib.pool_destroy(h)


def test_out_that_overlaps_the_queries():
    d = C.byref(desc(max_blocks=64))
    nbytes = 2 * 3 * 4 * 4 * 64 * 2       # layers, agents, drafts, query heads, head_dim
    p = C.byref(params(page_splits=4, workspace_dev=0x100000, workspace_bytes=0))
    at = lambda k: C.c_void_p(0x4000000 + k)  # noqa: E731
    for k in (16, nbytes - 16):
        assert lib.pool_attend_tree(None, d, at(0), at(k), p, None) == pk.EINVAL and b"overlap" in lib.polykv_last_error()
        assert lib.pool_attend_tree(None, d, at(k), at(0), p, None) == pk.EINVAL and b"overlap" in lib.polykv_last_error()
    for k in (0, nbytes):                  # (in place, and side by side: the workspace is what is refused)
        assert lib.pool_attend_tree(None, d, at(0), at(k), p, None) == pk.ENOMEM
        assert lib.pool_attend_tree(None, d, at(k), at(0), p, None) == pk.ENOMEM


def test_accept_outputs_are_arrays_of_their_own():
    table = C.c_void_p(0x60000)
    d = C.byref(desc(table_dev=table))
    out = [C.c_void_p(0x30000 + 0x1000 * k) for k in range(4)]
    for k in range(4):
        for x in (*[out[j] for j in range(4) if j != k], table):
            args = [x if i == k else y for i, y in enumerate(out)]
            assert lib.polykv_pages_accept(d, P, P, P, P, 4, *args, None) == pk.EINVAL


def test_pages_on_the_current_device(monkeypatch):
    """A device without a number is the current one, as it is for every tensor."""
    torch = pytest.importorskip("torch")

    class Asked(Exception):
        pass

    def empty(*_args, device=None, **_kw):
        raise Asked(device)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch, "empty", empty)
    for device, index in (("cuda", 3), ("cuda:1", 1)):
        with pytest.raises(Asked) as e:
            pk.Pages(1, 2, 64, 4, 3, 2, page_tokens=8, device=device)
        assert e.value.args[0] == torch.device("cuda", index)
