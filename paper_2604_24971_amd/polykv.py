"""ctypes binding of libpolykv.so: argument marshalling only -- every step of the hot path runs in
the HIP kernels behind the C ABI declared in include/polykv.h.  torch supplies device memory and
the current stream, nothing else.  Importing this module fails loudly if the library is missing."""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpolykv.so")

OK, EINVAL, ESHAPE, ESTATE, ENOMEM, EHIP = 0, -1, -2, -3, -4, -5
F16, F32, BF16 = 0, 1, 2
_DTYPES = {torch.float16: F16, torch.float32: F32, torch.bfloat16: BF16}
KERNEL_AUTO, KERNEL_VECTOR, KERNEL_MATRIX = 0, 1, 2
KEY_PRECISION_EXACT, KEY_PRECISION_FP16 = 0, 1
VALUES_TQ3, VALUES_TQ3_SCALED, VALUES_INT8 = 0, 1, 2
VALUES_TQ2, VALUES_TQ2_SCALED, VALUES_TQ4, VALUES_TQ4_SCALED = 3, 4, 5, 6
VALUE_BITS = {0: 3, 1: 3, 2: 8, 3: 2, 4: 2, 5: 4, 6: 4}
KEYS_Q8_BLOCK32, KEYS_Q8_TENSOR = 0, 1
MAX_TAIL_AGENTS = 64
STATIC_WORKSPACE_BYTES = 32 << 20
MAX_PAGED_AGENTS, MAX_TREE_NODES = 4096, 256


class PolyKVError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("polykv status %d: %s" % (status, message))
        self.status = status


class AttendParams(C.Structure):
    _fields_ = [
        ("agents", C.c_int), ("q_per_agent", C.c_int), ("q_heads", C.c_int),
        ("layer_begin", C.c_int), ("layer_end", C.c_int), ("scale", C.c_float),
        ("tail_K", C.POINTER(C.c_void_p)), ("tail_V", C.POINTER(C.c_void_p)),
        ("tail_len", C.POINTER(C.c_int)), ("tail_capacity", C.c_int), ("tail_causal", C.c_int),
        ("kernel", C.c_int), ("splits", C.c_int),
        ("workspace_dev", C.c_void_p), ("workspace_bytes", C.c_size_t),
        ("io_dtype", C.c_int), ("key_precision", C.c_int),
    ]


class AttendChoice(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("kernel", "splits", "block_rows", "own_rows", "references", "tails_in_pool_launch")] + \
        [("grid", C.c_int * 3)]


class PagesDesc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("layers", "kv_heads", "head_dim", "pages", "page_tokens", "agents", "max_blocks", "dtype")] + \
        [(n, C.c_void_p) for n in ("K_dev", "V_dev", "table_dev", "lengths_dev", "free_dev", "free_state_dev", "ticket_dev")]


class TreeParams(C.Structure):
    _fields_ = [
        ("nodes", C.c_int), ("q_heads", C.c_int), ("layer_begin", C.c_int), ("layer_end", C.c_int), ("scale", C.c_float),
        ("kernel", C.c_int), ("splits", C.c_int), ("key_precision", C.c_int), ("page_splits", C.c_int),
        ("counts_dev", C.c_void_p), ("mask_dev", C.c_void_p), ("workspace_dev", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libpolykv.so is not built (%s); run `python -m paper_2604_24971_amd.build`" % LIB_PATH)
    lib = C.CDLL(LIB_PATH)
    vp, ip, sz = C.c_void_p, C.c_int, C.c_size_t
    lib.pool_create.argtypes = [ip, ip, ip, ip, C.POINTER(vp)]
    lib.pool_create.restype = ip
    lib.pool_create_codec.argtypes = [ip, ip, ip, ip, ip, C.POINTER(vp)]
    lib.pool_create_codec.restype = ip
    lib.pool_create_codecs.argtypes = [ip, ip, ip, ip, ip, ip, C.POINTER(vp)]
    lib.pool_create_codecs.restype = ip
    lib.pool_set_sign_seed.argtypes = [vp, C.c_uint64]
    lib.pool_set_sign_seed.restype = ip
    lib.pool_destroy.argtypes = [vp]
    lib.pool_destroy.restype = None
    lib.pool_bytes.argtypes = [vp]
    lib.pool_bytes.restype = sz
    lib.pool_bind.argtypes = [vp, vp, sz]
    lib.pool_bind.restype = ip
    lib.pool_encode.argtypes = [vp, vp, vp, vp]
    lib.pool_encode.restype = ip
    lib.pool_append.argtypes = [vp, vp, vp, ip, vp]
    lib.pool_append.restype = ip
    lib.pool_encode_dtype.argtypes = [vp, vp, vp, ip, vp]
    lib.pool_encode_dtype.restype = ip
    lib.pool_append_dtype.argtypes = [vp, vp, vp, ip, ip, vp]
    lib.pool_append_dtype.restype = ip
    lib.pool_length.argtypes = [vp]
    lib.pool_length.restype = ip
    lib.pool_decode_layers.argtypes = [vp, vp, vp, ip, ip, ip, vp]
    lib.pool_decode_layers.restype = ip
    lib.pool_decode.argtypes = [vp, vp, vp, ip, vp]
    lib.pool_decode.restype = ip
    lib.pool_export.argtypes = [vp, vp, vp, vp, vp]
    lib.pool_export.restype = ip
    lib.pool_export_value_scales.argtypes = [vp, vp, vp]
    lib.pool_export_value_scales.restype = ip
    lib.pool_attend_workspace.argtypes = [vp, C.POINTER(AttendParams)]
    lib.pool_attend_workspace.restype = sz
    lib.pool_attend_plan.argtypes = [vp, C.POINTER(AttendParams), C.POINTER(AttendChoice)]
    lib.pool_attend_plan.restype = ip
    lib.pool_attend.argtypes = [vp, vp, vp, C.POINTER(AttendParams), vp]
    lib.pool_attend.restype = ip
    lib.pool_attend_static.argtypes = [vp, vp, vp, C.POINTER(AttendParams), vp]
    lib.pool_attend_static.restype = ip
    pp, tp, i64 = C.POINTER(PagesDesc), C.POINTER(TreeParams), C.c_int64
    lib.polykv_pages_resize.argtypes = [pp, vp, vp, ip, vp, vp]
    lib.polykv_pages_resize.restype = ip
    lib.polykv_pages_resize_by_agent.argtypes = [pp, vp, vp, ip, vp, vp]
    lib.polykv_pages_resize_by_agent.restype = ip
    lib.polykv_pages_write.argtypes = [pp, vp, vp, ip, ip, i64, i64, i64, vp, ip, ip, vp]
    lib.polykv_pages_write.restype = ip
    lib.polykv_tree_masks.argtypes = [vp, vp, ip, ip, vp, vp, vp]
    lib.polykv_tree_masks.restype = ip
    lib.pool_attend_tree_workspace.argtypes = [vp, pp, tp]
    lib.pool_attend_tree_workspace.restype = sz
    # The call enqueues several kernels that share a workspace.  It keeps the interpreter's lock, so that those of two threads
    # on one stream do not mix (it takes a few microseconds and waits for nothing).
    lib.pool_attend_tree = C.PyDLL(LIB_PATH).pool_attend_tree
    lib.pool_attend_tree.argtypes = [vp, pp, vp, vp, tp, vp]
    lib.pool_attend_tree.restype = ip
    lib.polykv_pages_accept.argtypes = [pp, vp, vp, vp, vp, ip, vp, vp, vp, vp, vp]
    lib.polykv_pages_accept.restype = ip
    lib.polykv_codebook.argtypes = [C.POINTER(C.c_float), C.POINTER(C.c_float)]
    lib.polykv_codebook.restype = None
    lib.polykv_codebook_bits.argtypes = [ip, C.POINTER(C.c_float), C.POINTER(C.c_float)]
    lib.polykv_codebook_bits.restype = ip
    lib.polykv_time_next_kernel.argtypes = [vp, vp]
    lib.polykv_time_next_kernel.restype = ip
    lib.polykv_last_error.argtypes = []
    lib.polykv_last_error.restype = C.c_char_p
    return lib


lib = _load()


def _check(rc: int):
    if rc != OK:
        raise PolyKVError(rc, lib.polykv_last_error().decode())


def codebook(bits: int = 3):
    c = (C.c_float * (1 << bits))()
    t = (C.c_float * ((1 << bits) - 1))()
    _check(lib.polykv_codebook_bits(bits, c, t))
    return list(c), list(t)


def time_next_kernel(start: torch.cuda.Event, stop: torch.cuda.Event):
    """polykv_time_next_kernel(start, stop): the next encode / decode / attend call of this thread stamps the two
    events at the begin and end of its main kernel.  The events must have been recorded once before, so
    that torch has created their handles."""
    _check(lib.polykv_time_next_kernel(C.c_void_p(start.cuda_event), C.c_void_p(stop.cuda_event)))


# The handle of the current stream without the Stream object that torch.cuda.current_stream() builds around it, nor the
# look whether CUDA is there: 0.15 instead of 3.6 us, of 5 to 12 us that a call of one or two kernels takes on the host.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_ptr(stream=None) -> int:
    if stream is None:
        if _raw_stream is not None and _get_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_get_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _dev_ptr(t: torch.Tensor, dtype, what: str) -> int:
    if t.is_cuda and t.dtype is dtype and t.is_contiguous():
        return t.data_ptr()
    raise TypeError("%s must be a contiguous CUDA tensor of dtype %s" % (what, dtype))


class Tails:
    """The agents' private continuations, marshalled once: per agent a (K, V) pair of fp16 tensors
    [layers, kv_heads, capacity, head_dim] (or None) that the caller keeps appending to, plus the current
    lengths, which set_lengths() updates in place between decode steps."""

    def __init__(self, pool: "Pool", tensors, lengths=None):
        A = len(tensors)
        if A > MAX_TAIL_AGENTS:
            raise ValueError("at most %d agents can carry private tails" % MAX_TAIL_AGENTS)
        self.agents = A
        self.k = (C.c_void_p * A)()
        self.v = (C.c_void_p * A)()
        self.len = (C.c_int * A)()
        self.capacity = 0
        self.dtype = None            # torch.float16 or torch.bfloat16, the same for every tail
        self._keep = []
        for a, ent in enumerate(tensors):
            if ent is None:
                continue
            Kt, Vt = ent[0], ent[1]
            shape = (pool.layers, pool.kv_heads, Kt.shape[2], pool.head_dim)
            if tuple(Kt.shape) != shape or tuple(Vt.shape) != shape:
                raise ValueError("tail tensors must be [layers, kv_heads, capacity, head_dim]")
            if self.capacity and self.capacity != Kt.shape[2]:
                raise ValueError("all tails must share one capacity")
            self.capacity = Kt.shape[2]
            if self.dtype is None:
                self.dtype = Kt.dtype
            if self.dtype not in (torch.float16, torch.bfloat16):
                raise TypeError("tails must be float16 or bfloat16")
            self.k[a] = _dev_ptr(Kt, self.dtype, "tail K")
            self.v[a] = _dev_ptr(Vt, self.dtype, "tail V")
            self._keep += [Kt, Vt]
            if len(ent) > 2:
                self.len[a] = int(ent[2])
        if lengths is not None:
            self.set_lengths(lengths)

    def set_lengths(self, lengths):
        if len(lengths) != self.agents:
            raise ValueError("one length per agent")
        for a, n in enumerate(lengths):
            self.len[a] = int(n)
        return self


class Pool:
    """pool_create + pool_bind around a torch-owned storage tensor."""

    def __init__(self, layers: int, kv_heads: int, head_dim: int, tokens: int, device="cuda:0",
                 value_codec: int = VALUES_TQ3, sign_seed: int = 0, key_codec: int = KEYS_Q8_BLOCK32):
        self.layers, self.kv_heads, self.head_dim, self.tokens = layers, kv_heads, head_dim, tokens
        self.value_codec = value_codec
        self.key_codec = key_codec
        self.device = torch.device(device)
        h = C.c_void_p()
        _check(lib.pool_create_codecs(layers, kv_heads, head_dim, tokens, key_codec, value_codec, C.byref(h)))
        self._h = h
        if sign_seed:
            _check(lib.pool_set_sign_seed(self._h, sign_seed))
        self.nbytes = lib.pool_bytes(self._h)
        self.storage = None
        self._workspaces = {}   # stream handle -> cached attend workspace

    def bind(self, storage: torch.Tensor | None = None):
        if storage is None:
            storage = torch.empty(self.nbytes, dtype=torch.uint8, device=self.device)
        _check(lib.pool_bind(self._h, _dev_ptr(storage, torch.uint8, "storage"), storage.numel()))
        self.storage = storage
        return self

    def close(self):
        h, self._h = getattr(self, "_h", None), None
        if h and lib is not None:      # `lib` is already gone when the interpreter shuts down
            lib.pool_destroy(h)

    __del__ = close

    def _handle(self, what: str):
        """For the calls whose pool may also be absent: a closed one is not an absent one."""
        if self._h is None:
            raise PolyKVError(EINVAL, "%s: the pool is closed" % what)
        return self._h

    # pool_encode(K, V)
    def encode(self, K: torch.Tensor, V: torch.Tensor, stream=None):
        shape = (self.layers, self.kv_heads, self.tokens, self.head_dim)
        if tuple(K.shape) != shape or tuple(V.shape) != shape:
            raise ValueError("K and V must have shape %s" % (shape,))
        if K.dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("K and V must be float16 or bfloat16")
        _check(lib.pool_encode_dtype(self._h, _dev_ptr(K, K.dtype, "K"), _dev_ptr(V, K.dtype, "V"), _DTYPES[K.dtype],
                                     _stream_ptr(stream)))

    # pool_append(K, V, count)
    def append(self, K: torch.Tensor, V: torch.Tensor, stream=None):
        if K.dim() != 4 or tuple(K.shape) != tuple(V.shape) or \
                tuple(K.shape[:2]) != (self.layers, self.kv_heads) or K.shape[3] != self.head_dim:
            raise ValueError("K and V must be [layers, kv_heads, count, head_dim]")
        if K.dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("K and V must be float16 or bfloat16")
        _check(lib.pool_append_dtype(self._h, _dev_ptr(K, K.dtype, "K"), _dev_ptr(V, K.dtype, "V"),
                                     int(K.shape[2]), _DTYPES[K.dtype], _stream_ptr(stream)))

    @property
    def length(self) -> int:
        return lib.pool_length(self._h)

    # pool_decode(K_out, V_out)
    def decode(self, dtype=torch.float32, K_out=None, V_out=None, stream=None, layer_begin=0, layer_end=None):
        layer_end = self.layers if layer_end is None else layer_end
        shape = (max(layer_end - layer_begin, 0), self.kv_heads, self.length, self.head_dim)
        code = _DTYPES[dtype]
        if K_out is None:
            K_out = torch.empty(shape, dtype=dtype, device=self.device)
        if V_out is None:
            V_out = torch.empty(shape, dtype=dtype, device=self.device)
        if K_out.shape != shape or V_out.shape != shape:
            raise ValueError("decode outputs must have shape %s" % (shape,))
        _check(lib.pool_decode_layers(self._h, _dev_ptr(K_out, dtype, "K_out"), _dev_ptr(V_out, dtype, "V_out"),
                                      code, layer_begin, layer_end, _stream_ptr(stream)))
        return K_out, V_out

    def export(self, stream=None):
        n = (self.layers, self.kv_heads, self.length)
        kc = torch.empty(n + (self.head_dim,), dtype=torch.int8, device=self.device)
        if self.key_codec == KEYS_Q8_TENSOR:     # one scale per layer tensor
            ks = torch.empty((self.layers,), dtype=torch.float16, device=self.device)
        else:
            ks = torch.empty(n + (self.head_dim // 32,), dtype=torch.float16, device=self.device)
        if self.value_codec == VALUES_INT8:      # the int8 value codes themselves
            vp = torch.empty(n + (self.head_dim,), dtype=torch.int8, device=self.device)
        else:
            vp = torch.empty(n + (VALUE_BITS[self.value_codec] * self.head_dim // 8,), dtype=torch.uint8, device=self.device)
        _check(lib.pool_export(self._h, kc.data_ptr(), ks.data_ptr(),
                               vp.data_ptr(), _stream_ptr(stream)))
        return kc, ks, vp

    def export_value_scales(self, stream=None):
        vs = torch.empty((self.layers, self.kv_heads, self.length), dtype=torch.float16, device=self.device)
        _check(lib.pool_export_value_scales(self._h, C.c_void_p(vs.data_ptr()), _stream_ptr(stream)))
        return vs

    def _params(self, Q, q_heads, layer_begin, layer_end, scale, tails, kernel, splits, tail_causal=False,
                key_precision=KEY_PRECISION_EXACT):
        if Q.dim() != 5:
            raise ValueError("Q must be [layers_selected, agents, q_per_agent, q_heads, head_dim]")
        layer_end = self.layers if layer_end is None else layer_end
        Ls, A, nq, qh, d = Q.shape
        if Ls != layer_end - layer_begin or d != self.head_dim or (q_heads is not None and qh != q_heads):
            raise ValueError("Q shape %s does not match the layer range / head_dim" % (tuple(Q.shape),))
        p = AttendParams()
        p.agents, p.q_per_agent, p.q_heads = A, nq, qh
        p.layer_begin, p.layer_end, p.scale = layer_begin, layer_end, float(scale or 0.0)
        p.kernel, p.splits = kernel, splits
        p.key_precision = key_precision
        if Q.dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("Q must be float16 or bfloat16")
        p.io_dtype = _DTYPES[Q.dtype]
        keep = []
        if tails is not None:
            if not isinstance(tails, Tails):
                tails = Tails(self, tails)
            if tails.agents != A:
                raise ValueError("tails must have one entry per agent")
            if tails.dtype is not None and tails.dtype != Q.dtype:
                raise TypeError("Q and the tails must have the same dtype")
            p.tail_K, p.tail_V, p.tail_len = tails.k, tails.v, tails.len    # (arrays become pointers without a cast)
            p.tail_capacity = tails.capacity
            p.tail_causal = 1 if tail_causal else 0
            keep.append(tails)
        return p, keep

    def attend_workspace_bytes(self, Q, **kw):
        p, _keep = self._params(Q, kw.get("q_heads"), kw.get("layer_begin", 0), kw.get("layer_end"),
                                kw.get("scale"), kw.get("tails"), kw.get("kernel", KERNEL_AUTO),
                                kw.get("splits", 0), kw.get("tail_causal", False))
        return lib.pool_attend_workspace(self._h, C.byref(p))

    def attend_plan(self, Q, **kw) -> AttendChoice:
        """What attend(Q, **kw) does; for tests and benchmarks."""
        p, _keep = self._params(Q, kw.get("q_heads"), kw.get("layer_begin", 0), kw.get("layer_end"), kw.get("scale"),
                                kw.get("tails"), kw.get("kernel", KERNEL_AUTO), kw.get("splits", 0),
                                kw.get("tail_causal", False), kw.get("key_precision", KEY_PRECISION_EXACT))
        choice = AttendChoice()
        _check(lib.pool_attend_plan(self._h, C.byref(p), C.byref(choice)))
        return choice

    # pool_attend(Q[agents], out)
    def attend(self, Q: torch.Tensor, out: torch.Tensor | None = None, *, q_heads=None, layer_begin=0,
               layer_end=None, scale=None, tails=None, kernel=KERNEL_AUTO, splits=0, workspace=None,
               stream=None, tail_causal=False, key_precision=KEY_PRECISION_EXACT):
        p, _keep = self._params(Q, q_heads, layer_begin, layer_end, scale, tails, kernel, splits, tail_causal,
                                key_precision)
        sp = _stream_ptr(stream)
        # One cached workspace per stream: calls on different streams may overlap and must not share one.  A call that is being
        # captured gets one of its own from the graph's memory: graphs may be replayed on any streams.
        capturing = workspace is None and _capturing(stream)
        ws = workspace if workspace is not None else None if capturing else self._workspaces.get(sp)
        if ws is None:
            ws = self._grow_workspace(p, sp, stream, keep=not capturing)
        p.workspace_dev = _dev_ptr(ws, torch.uint8, "workspace")
        p.workspace_bytes = ws.numel()
        if out is None:
            out = torch.empty(Q.shape, dtype=torch.float32, device=self.device)
        args = (self._h, _dev_ptr(Q, Q.dtype, "Q"), _dev_ptr(out, torch.float32, "out"), C.byref(p), sp)
        rc = lib.pool_attend(*args)
        if rc == ENOMEM and workspace is None:   # (nothing was launched) the cached one is too small: the size is asked for only then
            ws = self._grow_workspace(p, sp, stream)
            p.workspace_dev, p.workspace_bytes = ws.data_ptr(), ws.numel()
            rc = lib.pool_attend(*args)
        _check(rc)
        return out

    def _grow_workspace(self, p, sp, stream, keep=True):
        need = lib.pool_attend_workspace(self._h, C.byref(p))
        if need == 0:
            _check(lib.pool_attend(self._h, None, None, C.byref(p), None))  # surfaces the shape error
        # From the memory of the stream that uses it: the one it replaces may still be in use there, and goes to later work of
        # that stream only.
        with torch.cuda.stream(stream):
            ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        if keep:
            self._workspaces[sp] = ws
        return ws

    # pool_attend_static(Q[agents], out): no workspace, nothing allocated by the library
    def attend_static(self, Q: torch.Tensor, out: torch.Tensor, *, q_heads=None, layer_begin=0, layer_end=None,
                      scale=None, tails=None, kernel=KERNEL_AUTO, splits=0, stream=None, tail_causal=False,
                      key_precision=KEY_PRECISION_EXACT):
        p, _keep = self._params(Q, q_heads, layer_begin, layer_end, scale, tails, kernel, splits, tail_causal,
                                key_precision)
        _check(lib.pool_attend_static(self._h, _dev_ptr(Q, Q.dtype, "Q"), _dev_ptr(out, torch.float32, "out"),
                                      C.byref(p), _stream_ptr(stream)))
        return out

    # pool_attend_tree(Q[drafts], out): the pool, the agents' pages and the drafts in them
    def attend_tree(self, Q: torch.Tensor, pages: "Pages", out: torch.Tensor | None = None, *, kernel=KERNEL_AUTO, splits=0,
                    key_precision=KEY_PRECISION_EXACT, **kw):
        """Attention of every agent's drafted tokens over this pool, then the agent's tokens in `pages` and the drafts
        among them that a draft sees; the further arguments are Pages.attend_tree()'s."""
        handle = self._handle("attend_tree")
        if self.storage is not None and self.storage.device != pages.device:
            raise ValueError("the pool is on %s, the pages on %s" % (self.storage.device, pages.device))
        return pages._attend_tree(handle, Q, out, kernel=kernel, splits=splits, key_precision=key_precision, **kw)


# Calls act on the current device and on streams of it; an object on another device switches to it for the call.
def _elsewhere(index: int) -> bool:
    return (_get_device() if _get_device is not None and torch.cuda.is_initialized() else torch.cuda.current_device()) != index


def _capturing(stream=None) -> bool:
    """Whether the stream that the call runs on is being captured, which need not be the current one."""
    if stream is None:
        return torch.cuda.is_current_stream_capturing()
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


def _new(shape, dtype, device, stream=None):
    """A tensor from the memory of the stream that the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _ints(t: torch.Tensor, shape, device, what: str) -> int:
    if t.dtype is torch.int32 and t.shape == shape and t.device == device and t.is_contiguous():
        return t.data_ptr()
    raise TypeError("%s must be a contiguous int32 tensor of shape %s on %s" % (what, tuple(shape), device))


def tree_masks(parents: torch.Tensor, counts: torch.Tensor | None = None, mask: torch.Tensor | None = None,
               depth: torch.Tensor | None = None, stream=None):
    """Trees of drafted tokens: parents int32 [agents, nodes], an earlier draft of the same agent or -1; counts int32
    [agents], the drafts of each agent (None: all).  Returns (mask, depth): mask int64 [agents, nodes, ceil(nodes / 64)],
    whose bit j % 64 of word j / 64 says that a draft sees draft j (itself and its ancestors), and depth int32 [agents,
    nodes], the number of a draft's ancestors -- how far its position is from the first draft's."""
    if parents.dim() != 2 or not parents.is_cuda:
        raise TypeError("parents must be a CUDA tensor [agents, nodes]")
    device = parents.device
    if _elsewhere(device.index):
        with torch.cuda.device(device):
            return tree_masks(parents, counts, mask, depth, stream)
    shape = parents.shape
    agents, nodes = shape
    words = (agents, nodes, (nodes + 63) // 64)
    if mask is None:
        mask = _new(words, torch.int64, device, stream)
    elif mask.dtype is not torch.int64 or mask.shape != words or mask.device != device or not mask.is_contiguous():
        raise TypeError("mask must be a contiguous int64 tensor of shape %s on %s" % (words, device))
    if depth is None:
        depth = torch.empty_like(parents) if stream is None else _new(shape, torch.int32, device, stream)
    _check(lib.polykv_tree_masks(_ints(parents, shape, device, "parents"),
                                 _ints(counts, (agents,), device, "counts") if counts is not None else None, agents, nodes,
                                 mask.data_ptr(), _ints(depth, shape, device, "depth"), _stream_ptr(stream)))
    return mask, depth


class Pages:
    """Private continuations of `agents` agents in pages of a common store, the counterpart of Tails for any number of
    agents, lengths on the device and several drafted tokens a step.

      K, V        [layers, pages, kv_heads, page_tokens, head_dim], float16 or bfloat16
      table       int32 [agents, max_blocks]: the pages of an agent's tokens, in order
      lengths     int32 [agents]: tokens in an agent's pages, drafts included
      free, free_state   the ring of free pages, and its first place and how many there are

    Agents start empty and all pages free.  The tensors are the caller's to read, and to write between calls (their
    storage has to stay)."""

    def __init__(self, layers: int, kv_heads: int, head_dim: int, pages: int, agents: int, max_blocks: int, page_tokens: int = 16,
                 dtype=torch.float16, device="cuda:0"):
        if dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("pages must be float16 or bfloat16")
        self.layers, self.kv_heads, self.head_dim = layers, kv_heads, head_dim
        self.pages, self.page_tokens, self.agents, self.max_blocks, self.dtype = pages, page_tokens, agents, max_blocks, dtype
        device = torch.device(device)
        if device.type != "cuda":
            raise TypeError("pages lie in GPU memory, not on %s" % device)
        self.device = torch.device(device.type, device.index if device.index is not None else torch.cuda.current_device())
        shape = (layers, pages, kv_heads, page_tokens, head_dim)
        self.K = torch.empty(shape, dtype=dtype, device=self.device)
        self.V = torch.empty(shape, dtype=dtype, device=self.device)
        self.table = torch.full((agents, max_blocks), -1, dtype=torch.int32, device=self.device)
        self.lengths = torch.zeros((agents,), dtype=torch.int32, device=self.device)
        self.free = torch.arange(pages, dtype=torch.int32, device=self.device)
        self.free_state = torch.tensor([0, pages], dtype=torch.int32, device=self.device)
        self._ticket = torch.zeros((1,), dtype=torch.int32, device=self.device)
        self._desc = PagesDesc(layers, kv_heads, head_dim, pages, page_tokens, agents, max_blocks, _DTYPES[dtype],
                               *(t.data_ptr() for t in (self.K, self.V, self.table, self.lengths, self.free, self.free_state,
                                                         self._ticket)))
        self._ref = C.byref(self._desc)
        # (writing nothing checks the description)
        _check(lib.polykv_pages_write(self._ref, None, None, _DTYPES[dtype], 0, 0, 0, 0, None, 0, layers, None))
        self._index = self.device.index
        self._per_agent, self._per_offset = self.lengths.shape, torch.Size((agents + 1,))
        self._workspaces = {}   # stream handle -> cached attend_tree workspace

    # polykv_pages_resize(targets, slots, offsets), polykv_pages_resize_by_agent(targets, slots, granted)
    def resize(self, targets: torch.Tensor, slots: torch.Tensor | None = None, offsets: torch.Tensor | None = None, stream=None, *,
               granted: torch.Tensor | None = None):
        """Agent a's continuation becomes targets[a] tokens long: pages are taken for it or given back.  An agent for which
        there are no pages, or whose target is out of range, keeps its length.  `slots` (int32, any length) receives the
        places of the tokens that agents grew by, for write(), agent after agent, and -1 behind them; `offsets` (int32
        [agents + 1]) where each agent's begin: rows for write() are packed by them, without those of agents that kept their
        length.

        With `granted` (int32 [agents]) places go by agent: `slots` is [agents, n], entry [a, i] the place of the i-th token
        that agent a grew by and -1 behind them, and granted[a] receives how many these are.  For rows of drafts [agents, n]
        this is the form to use: write() takes slots.view(-1), and tree_masks(), attend_tree() and accept() take `granted`
        as their counts, so that an agent that kept its length has no drafts in the step."""
        if _elsewhere(self._index):
            with torch.cuda.device(self._index):
                return self.resize(targets, slots, offsets, stream, granted=granted)
        if granted is not None:
            if offsets is not None:
                raise ValueError("offsets are those of slots without granted")
            n = 0
            if slots is not None:
                if slots.dim() != 2:
                    raise ValueError("with granted, slots must be [agents, n]")
                n = slots.shape[1]
                slots = _ints(slots, (self.agents, n), self.device, "slots")
            _check(lib.polykv_pages_resize_by_agent(self._ref, _ints(targets, self._per_agent, self.device, "targets"), slots, n,
                                                    _ints(granted, self._per_agent, self.device, "granted"), _stream_ptr(stream)))
            return
        n = 0
        if slots is not None:
            n = slots.numel()
            slots = _ints(slots, (n,), self.device, "slots")
        if offsets is not None:
            offsets = _ints(offsets, self._per_offset, self.device, "offsets")
        _check(lib.polykv_pages_resize(self._ref, _ints(targets, self._per_agent, self.device, "targets"), slots, n, offsets,
                                       _stream_ptr(stream)))

    # polykv_pages_write(K, V, slots)
    def write(self, K: torch.Tensor, V: torch.Tensor, slots: torch.Tensor, layer_begin=0, layer_end=None, stream=None):
        """Keys and values [layers of the range, tokens, kv_heads, head_dim] (the pages' dtype or float32; heads' elements
        contiguous, any other strides of whole 16 bytes, the same for both) into the slots of their tokens."""
        if _elsewhere(self._index):
            with torch.cuda.device(self._index):
                return self.write(K, V, slots, layer_begin, layer_end, stream)
        layer_end = self.layers if layer_end is None else layer_end
        shape, device, dtype = K.shape, self.device, K.dtype
        if len(shape) != 4 or shape != V.shape or shape[0] != layer_end - layer_begin or shape[2] != self.kv_heads or \
                shape[3] != self.head_dim:
            raise ValueError("K and V must be [%d, tokens, %d, %d]" % (layer_end - layer_begin, self.kv_heads, self.head_dim))
        if (dtype is not self.dtype and dtype is not torch.float32) or V.dtype is not dtype or K.device != device or V.device != device:
            raise TypeError("K and V must be %s or float32 tensors on %s" % (self.dtype, device))
        strides = K.stride()
        if strides != V.stride() or strides[3] != 1 or 1 in shape[1:]:   # (a dimension of one element: its stride does not matter)
            strides = [s if n > 1 else 0 for s, n in zip(strides, shape)]
            if strides[3] != 1 or [s if n > 1 else 0 for s, n in zip(V.stride(), shape)] != strides:
                raise ValueError("K and V must have the same strides, 1 along head_dim")
        _check(lib.polykv_pages_write(self._ref, K.data_ptr(), V.data_ptr(), _DTYPES[dtype], shape[1],
                                      strides[0] if shape[0] > 1 else 0, strides[1], strides[2],
                                      _ints(slots, (shape[1],), device, "slots"), layer_begin, layer_end, _stream_ptr(stream)))

    # pool_attend_tree(NULL, Q[drafts], out)
    def attend_tree(self, Q: torch.Tensor, out: torch.Tensor | None = None, **kw):
        """Attention of every agent's drafted tokens (the last counts[a] of its lengths[a] tokens) over the tokens before
        them and the drafts that a draft's mask names.  Q [layers of the range, agents, nodes, q_heads, head_dim] of the
        pages' dtype; the result has its shape and dtype.  counts int32 [agents] (None: `nodes` for every agent); mask int64
        [agents, nodes, ceil(nodes / 64)] as tree_masks() makes it (None: a draft sees itself and all before it).  Rows
        of drafts that an agent does not have see no private token.  `out` may be Q.  page_splits: token ranges of an agent;
        by itself the call takes as many as continuations that fill the block tables need, and 1 is faster where they are much
        shorter."""
        return self._attend_tree(None, Q, out, **kw)

    def _attend_tree(self, pool, Q, out, *, counts=None, mask=None, layer_begin=0, layer_end=None, scale=None, kernel=KERNEL_AUTO,
                     splits=0, page_splits=0, key_precision=KEY_PRECISION_EXACT, workspace=None, stream=None):
        device = self.device
        if _elsewhere(self._index):
            with torch.cuda.device(device):
                return self._attend_tree(pool, Q, out, counts=counts, mask=mask, layer_begin=layer_begin, layer_end=layer_end,
                                         scale=scale, kernel=kernel, splits=splits, page_splits=page_splits,
                                         key_precision=key_precision, workspace=workspace, stream=stream)
        p = self._tree_params(Q, layer_begin, layer_end, scale, kernel, splits, page_splits, key_precision)
        if Q.device != device:
            raise ValueError("Q is on %s, the pages on %s" % (Q.device, device))
        if counts is not None:
            p.counts_dev = _ints(counts, self._per_agent, device, "counts")
        if mask is not None:
            words = (self.agents, p.nodes, (p.nodes + 63) // 64)
            if mask.dtype is not torch.int64 or mask.shape != words or mask.device != device or not mask.is_contiguous():
                raise TypeError("mask must be a contiguous int64 tensor of shape %s on %s" % (words, device))
            p.mask_dev = mask.data_ptr()
        sp = _stream_ptr(stream)
        ref = C.byref(p)
        if out is None:
            out = _new(Q.shape, self.dtype, device, stream)
        elif out.shape != Q.shape or out.device != device:
            raise ValueError("out must have Q's shape %s on %s" % (tuple(Q.shape), device))
        q_ptr, out_ptr = _dev_ptr(Q, self.dtype, "Q"), _dev_ptr(out, self.dtype, "out")
        # One cached workspace per stream: calls on different streams may overlap and must not share one.  A call that is
        # being captured gets one of its own from the graph's memory: graphs may be replayed on any streams.
        own = workspace is None
        capturing = own and _capturing(stream)
        if not own and workspace.device != device:
            raise ValueError("workspace is on %s, the pages on %s" % (workspace.device, device))
        ws = workspace if not own else None if capturing else self._workspaces.get(sp)
        if ws is not None:
            p.workspace_dev, p.workspace_bytes = ws.data_ptr() if own else _dev_ptr(ws, torch.uint8, "workspace"), ws.numel()
            rc = lib.pool_attend_tree(pool, self._ref, q_ptr, out_ptr, ref, sp)
            if rc != ENOMEM or not own:
                _check(rc)
                return out
        ws = _new((max(lib.pool_attend_tree_workspace(pool, self._ref, ref), 256),), torch.uint8, device, stream)
        if not capturing:
            self._workspaces[sp] = ws
        p.workspace_dev, p.workspace_bytes = ws.data_ptr(), ws.numel()
        _check(lib.pool_attend_tree(pool, self._ref, q_ptr, out_ptr, ref, sp))
        return out

    def _tree_params(self, Q, layer_begin, layer_end, scale, kernel, splits, page_splits, key_precision):
        layer_end = self.layers if layer_end is None else layer_end
        if Q.dim() != 5:
            raise ValueError("Q must be [layers_selected, agents, nodes, q_heads, head_dim]")
        n, agents, nodes, q_heads, d = Q.shape
        if n != layer_end - layer_begin or agents != self.agents or d != self.head_dim:
            raise ValueError("Q shape %s does not match the layer range, %d agents and head_dim %d" % (tuple(Q.shape), self.agents, self.head_dim))
        return TreeParams(nodes, q_heads, layer_begin, layer_end, float(scale or 0.0), kernel, splits, key_precision, page_splits)

    def attend_tree_workspace_bytes(self, Q, pool: "Pool | None" = None, *, layer_begin=0, layer_end=None, kernel=KERNEL_AUTO, splits=0,
                                    page_splits=0):
        """Scratch that attend_tree(Q) needs (with a pool: pool.attend_tree(Q, pages)); 0: none."""
        handle = pool._handle("attend_tree_workspace_bytes") if pool is not None else None
        p = self._tree_params(Q, layer_begin, layer_end, None, kernel, splits, page_splits, KEY_PRECISION_EXACT)
        return lib.pool_attend_tree_workspace(handle, self._ref, C.byref(p))

    # polykv_pages_accept(tokens, following, parents)
    def accept(self, tokens: torch.Tensor, following: torch.Tensor, parents: torch.Tensor, counts: torch.Tensor | None = None,
               stream=None):
        """The drafts that the model agrees with: int32 [agents, nodes] the drafted tokens, what the model puts after each
        of them, and the trees.  Draft 0 is accepted; after an accepted draft the first of its children whose token is what
        the model puts there.  Their keys and values move to right behind the tokens before the drafts, in all layers.
        Returns int32 tensors: path [agents, nodes] (-1 behind the accepted drafts), accepted [agents] (how many), following
        [agents] (the model's token after the last of them) and kept [agents] (the lengths with them, for resize())."""
        device, shape = self.device, tokens.shape
        if _elsewhere(self._index):
            with torch.cuda.device(device):
                return self.accept(tokens, following, parents, counts, stream)
        if len(shape) != 2 or shape[0] != self.agents:
            raise ValueError("tokens must be [agents, nodes]")
        inputs = (_ints(tokens, shape, device, "tokens"), _ints(following, shape, device, "following"), _ints(parents, shape, device, "parents"),
                  _ints(counts, self._per_agent, device, "counts") if counts is not None else None)
        # (one tensor each: they outlive each other)
        if stream is None:
            path, accepted, after, kept = torch.empty_like(tokens), *(torch.empty_like(self.lengths) for _ in range(3))
        else:
            path = _new(shape, torch.int32, device, stream)
            accepted, after, kept = (_new(self._per_agent, torch.int32, device, stream) for _ in range(3))
        _check(lib.polykv_pages_accept(self._ref, *inputs, shape[1], path.data_ptr(), accepted.data_ptr(), after.data_ptr(),
                                       kept.data_ptr(), _stream_ptr(stream)))
        return path, accepted, after, kept
