"""Python binding of libhoccl (ctypes).

Argument marshalling only: every step of a collective runs in the HIP
library (``libhoccl.so``, built from ``csrc/`` by ``build.py``; so is
``_tensors.so``, which reads lists of tensors).  PyTorch is
used for device memory and streams; each call passes raw device pointers and
``torch.cuda.current_stream().cuda_stream`` (or the stream given) to the
C ABI declared in ``include/hoccl.h``.

Importing fails loudly when the library has not been built: there is no
fallback implementation.
"""
import collections
import contextlib
import ctypes
import os
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhoccl.so")

for _path in (LIB_PATH, os.path.join(_HERE, "_tensors.so")):
    if not os.path.exists(_path):
        raise ImportError(
            f"{_path} is not built; run `python {os.path.join(_HERE, 'build.py')}` "
            "(or __graft_entry__.build()) first")

from . import _tensors  # noqa: E402  (csrc/tensors.cpp)

_lib = ctypes.CDLL(LIB_PATH)

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_HIP, ERR_NO_MEMORY, ERR_TIMEOUT, ERR_INTERNAL = range(7)
INT32, FP32, BF16, UINT8 = 0, 1, 2, 3
COPY_AUTO, COPY_SDMA, COPY_KERNEL, COPY_HIP = range(4)
REDUCE_RING, REDUCE_DIRECT, REDUCE_AUTO = range(3)
OP_ALLREDUCE, OP_REDUCE_SCATTER, OP_ALLGATHER, OP_SENDRECV, OP_ALLTOALL = range(5)

_DTYPES = {torch.int32: INT32, torch.float32: FP32, torch.bfloat16: BF16}
_COPY_DTYPES = {**_DTYPES, torch.uint8: UINT8}     # the copy-only collectives also move bytes
HOP_FIRST, HOP_MIDDLE, HOP_LAST, HOP_ONLY = range(4)
HOPS = {"first": HOP_FIRST, "middle": HOP_MIDDLE, "last": HOP_LAST, "only": HOP_ONLY}
COPY_PATHS = {"auto": COPY_AUTO, "sdma": COPY_SDMA, "engines": COPY_SDMA,
              "kernel": COPY_KERNEL, "hip": COPY_HIP}
COPY_PATH_NAMES = {COPY_AUTO: "auto", COPY_SDMA: "engines", COPY_KERNEL: "kernel", COPY_HIP: "hip"}
REDUCE_ALGOS = {"ring": REDUCE_RING, "direct": REDUCE_DIRECT, "auto": REDUCE_AUTO}


class Config(ctypes.Structure):
    _fields_ = [("workgroups_per_step", ctypes.c_int),
                ("threads_per_workgroup", ctypes.c_int),
                ("chunk_bytes", ctypes.c_size_t),
                ("copy_streams", ctypes.c_int),
                ("copy_path", ctypes.c_int),
                ("allgather_direct", ctypes.c_int),
                ("allreduce_chunk_groups", ctypes.c_int),
                ("sdma_engines", ctypes.c_int),
                ("reduce_algo", ctypes.c_int),
                ("kernel_timing", ctypes.c_int),
                ("proxy_timeout_ms", ctypes.c_uint),
                ("proxy_handshake", ctypes.c_int),
                ("ring_group_bytes", ctypes.c_size_t),
                ("proxy_wait_limit_us", ctypes.c_uint),
                ("fused_hops", ctypes.c_int),
                ("a2a_schedule", ctypes.c_int),
                ("proxy_slice_bytes", ctypes.c_size_t),
                ("bf16_partials", ctypes.c_int)]


class Stats(ctypes.Structure):
    _fields_ = [("reduce_launches", ctypes.c_int),
                ("copy_ops", ctypes.c_int),
                ("workgroups_per_step", ctypes.c_int),
                ("cus_available", ctypes.c_int),
                ("cus_used_max", ctypes.c_int),
                ("copy_path_used", ctypes.c_int),
                ("hbm_bytes_algorithmic", ctypes.c_ulonglong),
                ("host_enqueue_us", ctypes.c_double),
                ("copy_kernel_launches", ctypes.c_int),
                ("reduce_algo_used", ctypes.c_int),
                ("copy_bytes", ctypes.c_ulonglong)]


class _AdamW(ctypes.Structure):
    _fields_ = [("param_dtype", ctypes.c_int),
                ("grad_dtype", ctypes.c_int),
                ("state_bits", ctypes.c_int),
                ("step", ctypes.c_longlong),
                ("lr", ctypes.c_double),
                ("beta1", ctypes.c_double),
                ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double),
                ("lr_dev", ctypes.c_void_p),
                ("step_dev", ctypes.c_void_p),
                ("grad_scale", ctypes.c_void_p)]


class _Balance(ctypes.Structure):
    _fields_ = [("logits_dtype", ctypes.c_int),
                ("index_bytes", ctypes.c_int),
                ("experts", ctypes.c_int),
                ("topk", ctypes.c_int),
                ("ranks", ctypes.c_int),
                ("max_ranks", ctypes.c_int),
                ("expert_weight", ctypes.c_double),
                ("rank_weight", ctypes.c_double),
                ("traffic_weight", ctypes.c_double)]


_vpp = ctypes.POINTER(ctypes.c_void_p)
_vp = ctypes.c_void_p
_sz = ctypes.c_size_t
_szp = ctypes.POINTER(ctypes.c_size_t)
_i = ctypes.c_int
_SIGS = {
    "hoccl_init": [_i],
    "hoccl_finalize": [],
    "hoccl_set_config": [ctypes.POINTER(Config)],
    "hoccl_get_config": [ctypes.POINTER(Config)],
    "hoccl_get_last_stats": [ctypes.POINTER(Stats)],
    "hoccl_get_kernel_times": [ctypes.POINTER(ctypes.c_float), _i, ctypes.POINTER(_i)],
    "hoccl_allreduce": [_vpp, _vpp, _sz, _i, _i, ctypes.c_void_p],
    "hoccl_reduce_scatter": [_vpp, _vpp, _sz, _i, _i, ctypes.c_void_p],
    "hoccl_reduce_scatter_noalloc": [_vpp, _vpp, _sz, _i, _i, ctypes.c_void_p],
    "hoccl_allgather": [_vpp, _vpp, _sz, _i, _i, ctypes.c_void_p],
    "hoccl_sendrecv": [_vpp, _vpp, ctypes.POINTER(_i), _sz, _i, _i, ctypes.c_void_p],
    "hoccl_alltoall": [_vpp, _vpp, _sz, _i, _i, ctypes.c_void_p],
    "hoccl_alltoallv": [_vpp, _szp, _szp, _vpp, _szp, _i, _i, ctypes.c_void_p],
    "hoccl_ring_hop": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, _sz, _i, _i, ctypes.c_void_p],
    "hoccl_adamw": [_vp, _i, ctypes.POINTER(_AdamW), _vp],
    "hoccl_rmsnorm": [_vp, _vp, _vp, _vp, _vp, _vp, _sz, _sz, ctypes.c_double, _i, _i, _vp],
    "hoccl_rmsnorm_backward_workspace": [_sz, _sz, _i, _szp],
    "hoccl_rmsnorm_backward": [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _sz, _sz, ctypes.c_double, _i, _i, _vp],
    "hoccl_balance_workspace": [_vp, _i, ctypes.POINTER(_Balance), _szp],
    "hoccl_balance_loss": [_vp, _vp, _vp, _i, ctypes.POINTER(_Balance), _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "hoccl_balance_loss_backward": [_vp, _vp, _vp, _i, ctypes.POINTER(_Balance), _vp, _vp, _vp, _vp],
    "hoccl_debug_plan_json": [_i, _sz, _i, _i, ctypes.c_char_p, _sz, _szp],
    "hoccl_debug_schedule_json": [_i, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_i),
                                  ctypes.POINTER(_i), ctypes.c_double, ctypes.c_double,
                                  ctypes.c_char_p, _sz, _szp],
    "hoccl_debug_interleave": [_i, ctypes.POINTER(ctypes.c_double), ctypes.c_double,
                               ctypes.POINTER(_i), _sz, _szp],
    "hoccl_debug_stream_ceiling": [_i, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, _sz,
                                   ctypes.c_void_p],
    "hoccl_ipc_export": [ctypes.c_void_p, ctypes.c_void_p, _szp, _szp],
    "hoccl_ipc_open": [ctypes.c_void_p, _sz, _sz, ctypes.POINTER(ctypes.c_void_p)],
    "hoccl_ipc_close_all": [],
    "hoccl_mailbox_create": [ctypes.c_char_p, ctypes.c_uint, _sz, _vpp],
    "hoccl_mailbox_open": [ctypes.c_char_p, _vpp],
    "hoccl_mailbox_unlink": [ctypes.c_char_p],
    "hoccl_mailbox_close": [ctypes.c_void_p],
    "hoccl_mailbox_post": [ctypes.c_void_p, ctypes.c_uint, ctypes.c_uint, ctypes.c_char_p, _sz],
    "hoccl_mailbox_wait": [ctypes.c_void_p, ctypes.c_uint, ctypes.c_uint, ctypes.c_uint],
    "hoccl_mailbox_read": [ctypes.c_void_p, ctypes.c_uint, ctypes.c_char_p, _sz, _szp],
}
for _name, _args in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = ctypes.c_int
_lib.hoccl_status_string.argtypes = [ctypes.c_int]
_lib.hoccl_status_string.restype = ctypes.c_char_p
_lib.hoccl_last_error_string.argtypes = []
_lib.hoccl_last_error_string.restype = ctypes.c_char_p
_lib.hoccl_sdma_engine_count.argtypes = []
_lib.hoccl_sdma_engine_count.restype = ctypes.c_int


class HocclError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = _lib.hoccl_status_string(status).decode()
        detail = _lib.hoccl_last_error_string().decode()
        super().__init__(f"{where}: {msg}" + (f" ({detail})" if detail else ""))


def _check(status, where):
    if status != OK:
        raise HocclError(status, where)


def lib():
    """The loaded ctypes library (for tests that call the C ABI directly)."""
    return _lib


# ---- configuration -------------------------------------------------------------

def get_config():
    c = Config()
    _check(_lib.hoccl_get_config(ctypes.byref(c)), "hoccl_get_config")
    return {k: getattr(c, k) for k, _ in Config._fields_}


def set_config(**kw):
    """Update configuration fields; copy_path also accepts a name
    ('auto', 'sdma' or 'engines', 'kernel', 'hip') and reduce_algo
    'ring', 'direct' or 'auto'."""
    c = Config()
    _check(_lib.hoccl_get_config(ctypes.byref(c)), "hoccl_get_config")
    for k, v in kw.items():
        if k == "copy_path" and isinstance(v, str):
            v = COPY_PATHS[v]
        if k == "reduce_algo" and isinstance(v, str):
            v = REDUCE_ALGOS[v]
        if not hasattr(c, k):
            raise KeyError(k)
        setattr(c, k, v)
    _check(_lib.hoccl_set_config(ctypes.byref(c)), "hoccl_set_config")


class config:
    """Context manager: temporarily change configuration fields."""

    def __init__(self, **kw):
        self.kw = kw

    def __enter__(self):
        self.saved = get_config()
        set_config(**self.kw)
        return self

    def __exit__(self, *exc):
        set_config(**self.saved)


def last_stats():
    s = Stats()
    _check(_lib.hoccl_get_last_stats(ctypes.byref(s)), "hoccl_get_last_stats")
    return {k: getattr(s, k) for k, _ in Stats._fields_}


def kernel_times():
    """Durations (ms) of the kernel launches of the last call (needs
    kernel_timing=1); waits for them."""
    n = ctypes.c_int(0)
    _check(_lib.hoccl_get_kernel_times(None, 0, ctypes.byref(n)), "hoccl_get_kernel_times")
    buf = (ctypes.c_float * max(1, n.value))()
    _check(_lib.hoccl_get_kernel_times(buf, n.value, ctypes.byref(n)), "hoccl_get_kernel_times")
    return list(buf[:n.value])


def sdma_engine_count():
    return _lib.hoccl_sdma_engine_count()


def init(device=-1):
    _check(_lib.hoccl_init(device), "hoccl_init")


def finalize():
    _check(_lib.hoccl_finalize(), "hoccl_finalize")


def plan_json(op, count, dtype, R):
    import json
    need = ctypes.c_size_t(0)
    _check(_lib.hoccl_debug_plan_json(op, count, dtype, R, None, 0, ctypes.byref(need)),
           "hoccl_debug_plan_json")
    buf = ctypes.create_string_buffer(need.value)
    _check(_lib.hoccl_debug_plan_json(op, count, dtype, R, buf, need.value, ctypes.byref(need)),
           "hoccl_debug_plan_json")
    return json.loads(buf.value.decode())


def schedule(C, node, peer, bw_intra, bw_inter):
    """The paper's collective scheduler on a described topology: returns
    {'T', 'stages', 'tau', 'total'} (see hoccl_debug_schedule_json)."""
    import json
    G = len(node)
    flat = [float(C[u][v]) for u in range(G) for v in range(G)]
    Cm = (ctypes.c_double * (G * G))(*flat)
    nd = (ctypes.c_int * G)(*node)
    pr = (ctypes.c_int * G)(*peer)
    need = ctypes.c_size_t(0)
    _check(_lib.hoccl_debug_schedule_json(G, Cm, nd, pr, bw_intra, bw_inter, None, 0,
                                          ctypes.byref(need)), "hoccl_debug_schedule_json")
    buf = ctypes.create_string_buffer(need.value)
    _check(_lib.hoccl_debug_schedule_json(G, Cm, nd, pr, bw_intra, bw_inter, buf, need.value,
                                          ctypes.byref(need)), "hoccl_debug_schedule_json")
    return json.loads(buf.value.decode())


def interleave(bytes_per_flow, chunk_bytes):
    """Flow-size-aware chunk order on one engine: list of flow indices."""
    F = len(bytes_per_flow)
    b = (ctypes.c_double * max(1, F))(*bytes_per_flow)
    n = ctypes.c_size_t(0)
    _check(_lib.hoccl_debug_interleave(F, b, chunk_bytes, None, 0, ctypes.byref(n)),
           "hoccl_debug_interleave")
    out = (ctypes.c_int * max(1, n.value))()
    _check(_lib.hoccl_debug_interleave(F, b, chunk_bytes, out, n.value, ctypes.byref(n)),
           "hoccl_debug_interleave")
    return list(out[:n.value])


# ---- collectives ---------------------------------------------------------------

def _dtype_of(tensors, copy=False):
    dt = tensors[0].dtype
    table = _COPY_DTYPES if copy else _DTYPES
    if dt not in table:
        raise TypeError(f"unsupported dtype {dt}")
    dev = tensors[0].device
    for t in tensors:
        if t.dtype != dt:
            raise TypeError("all buffers must share one dtype")
        if t.device != dev or t.device.type != "cuda":
            raise ValueError("all buffers must live on the same GPU")
        if not t.is_contiguous():
            raise ValueError("buffers must be contiguous")
    return table[dt]


def _ptrs(tensors):
    return (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _on_send_device(fn):
    """Runs a collective with its buffers' GPU current (and that GPU's
    current stream as the default): the library keeps its streams and
    workspace per device and acts on the current one."""
    import functools

    @functools.wraps(fn)
    def wrapper(send, *args, **kwargs):
        with torch.cuda.device(send[0].device):
            return fn(send, *args, **kwargs)
    return wrapper


@_on_send_device
def allreduce(send, recv=None, stream=None):
    """Sum of the R tensors `send`, written to every tensor of `recv`
    (defaults to in place)."""
    recv = send if recv is None else recv
    dt = _dtype_of(list(send) + list(recv))
    n = send[0].numel()
    if any(t.numel() != n for t in list(send) + list(recv)):
        raise ValueError("all buffers must have the same number of elements")
    _check(_lib.hoccl_allreduce(_ptrs(send), _ptrs(recv), n, dt, len(send), _stream(stream)),
           "hoccl_allreduce")
    return recv


@_on_send_device
def reduce_scatter(send, recv=None, stream=None):
    """send: R tensors of R*n elements; recv[r] receives block r of the sum."""
    R = len(send)
    if send[0].numel() % R:
        raise ValueError("send buffers must hold R * recvcount elements")
    n = send[0].numel() // R
    if recv is None:
        recv = [torch.empty(n, dtype=send[0].dtype, device=send[0].device) for _ in range(R)]
    dt = _dtype_of(list(send) + list(recv))
    if any(t.numel() != R * n for t in send) or any(t.numel() != n for t in recv):
        raise ValueError("buffer sizes do not match")
    _check(_lib.hoccl_reduce_scatter(_ptrs(send), _ptrs(recv), n, dt, R, _stream(stream)),
           "hoccl_reduce_scatter")
    return recv


@_on_send_device
def reduce_scatter_noalloc(send, recv, stream=None):
    """reduce_scatter through the entry point that allocates nothing: the
    ring's partials live in the library's static device scratch.  `recv`
    must be given; the library must be initialised on the device."""
    R = len(send)
    if send[0].numel() % R:
        raise ValueError("send buffers must hold R * recvcount elements")
    n = send[0].numel() // R
    dt = _dtype_of(list(send) + list(recv))
    if any(t.numel() != R * n for t in send) or any(t.numel() != n for t in recv):
        raise ValueError("buffer sizes do not match")
    _check(_lib.hoccl_reduce_scatter_noalloc(_ptrs(send), _ptrs(recv), n, dt, R, _stream(stream)),
           "hoccl_reduce_scatter_noalloc")
    return recv


@_on_send_device
def allgather(send, recv=None, stream=None):
    """send: R tensors of n elements; every recv[r] gets their concatenation."""
    R = len(send)
    n = send[0].numel()
    if recv is None:
        recv = [torch.empty(R * n, dtype=send[0].dtype, device=send[0].device) for _ in range(R)]
    dt = _dtype_of(list(send) + list(recv), copy=True)
    if any(t.numel() != n for t in send) or any(t.numel() != R * n for t in recv):
        raise ValueError("buffer sizes do not match")
    _check(_lib.hoccl_allgather(_ptrs(send), _ptrs(recv), n, dt, R, _stream(stream)),
           "hoccl_allgather")
    return recv


@_on_send_device
def sendrecv(send, recv, peers, stream=None):
    """Rank r sends send[r] to rank peers[r] (-1: nothing).  recv[d] may be
    None for ranks that receive nothing."""
    R = len(send)
    n = send[0].numel()
    live = [t for t in list(send) + list(recv) if t is not None]
    dt = _dtype_of(live, copy=True)
    rp = (ctypes.c_void_p * R)(*[0 if t is None else t.data_ptr() for t in recv])
    pp = (ctypes.c_int * R)(*peers)
    _check(_lib.hoccl_sendrecv(_ptrs(send), rp, pp, n, dt, R, _stream(stream)), "hoccl_sendrecv")
    return recv


@_on_send_device
def alltoall(send, recv=None, stream=None):
    R = len(send)
    if send[0].numel() % R:
        raise ValueError("send buffers must hold R blocks")
    n = send[0].numel() // R
    if recv is None:
        recv = [torch.empty_like(t) for t in send]
    dt = _dtype_of(list(send) + list(recv), copy=True)
    _check(_lib.hoccl_alltoall(_ptrs(send), _ptrs(recv), n, dt, R, _stream(stream)),
           "hoccl_alltoall")
    return recv


@_on_send_device
def alltoallv(send, counts, sdispls, recv, rdispls, stream=None):
    """counts/sdispls/rdispls: R*R element counts and offsets, [s*R + d]."""
    R = len(send)
    dt = _dtype_of(list(send) + list(recv), copy=True)
    S = ctypes.c_size_t * (R * R)
    _check(_lib.hoccl_alltoallv(_ptrs(send), S(*counts), S(*sdispls), _ptrs(recv), S(*rdispls),
                                dt, R, _stream(stream)), "hoccl_alltoallv")
    return recv


IPC_HANDLE_BYTES = 64


def ipc_export(t):
    """(handle bytes, byte offset, allocation bytes) of the allocation that
    holds tensor `t`'s data (hoccl_ipc_export)."""
    h = ctypes.create_string_buffer(IPC_HANDLE_BYTES)
    off, size = ctypes.c_size_t(0), ctypes.c_size_t(0)
    with torch.cuda.device(t.device):
        _check(_lib.hoccl_ipc_export(t.data_ptr(), h, ctypes.byref(off), ctypes.byref(size)),
               "hoccl_ipc_export")
    return h.raw, off.value, size.value


def ipc_open(handle, offset, alloc_bytes):
    """Device address, in this process, of byte `offset` of an allocation
    another process exported (hoccl_ipc_open; cached per handle)."""
    p = ctypes.c_void_p()
    _check(_lib.hoccl_ipc_open(handle, offset, alloc_bytes, ctypes.byref(p)), "hoccl_ipc_open")
    return p.value


def ipc_close_all():
    _check(_lib.hoccl_ipc_close_all(), "hoccl_ipc_close_all")


class Mailbox:
    """A cross-process mailbox (hoccl_mailbox_*): numbered slots of a
    sequence number and a payload in POSIX shared memory.  Given `slots`, it
    creates the object `name`; otherwise it opens an existing one."""

    def __init__(self, name, slots=None, slot_bytes=None):
        self._h = ctypes.c_void_p()
        self.name = name
        if slots is None:
            _check(_lib.hoccl_mailbox_open(name.encode(), ctypes.byref(self._h)), "hoccl_mailbox_open")
        else:
            _check(_lib.hoccl_mailbox_create(name.encode(), slots, slot_bytes, ctypes.byref(self._h)),
                   "hoccl_mailbox_create")
        self._cap = slot_bytes or (1 << 20)
        self._local = threading.local()     # a read buffer per thread

    @staticmethod
    def unlink(name):
        _check(_lib.hoccl_mailbox_unlink(name.encode()), "hoccl_mailbox_unlink")

    def post(self, slot, seq, data=b""):
        _check(_lib.hoccl_mailbox_post(self._h, slot, seq & 0xFFFFFFFF, data, len(data)),
               "hoccl_mailbox_post")

    def wait(self, slot, seq, timeout_ms):
        _check(_lib.hoccl_mailbox_wait(self._h, slot, seq & 0xFFFFFFFF, int(timeout_ms)),
               "hoccl_mailbox_wait")

    def ready(self, slot, seq):
        """Whether the slot has reached `seq` (one look, no waiting)."""
        return _lib.hoccl_mailbox_wait(self._h, slot, seq & 0xFFFFFFFF, 0) == OK

    def read(self, slot):
        loc = self._local
        if not hasattr(loc, "buf"):
            loc.buf, loc.len = ctypes.create_string_buffer(self._cap), ctypes.c_size_t(0)
        _check(_lib.hoccl_mailbox_read(self._h, slot, loc.buf, self._cap, ctypes.byref(loc.len)),
               "hoccl_mailbox_read")
        return loc.buf.raw[:loc.len.value]

    def close(self):
        if self._h:
            _lib.hoccl_mailbox_close(self._h)
            self._h = ctypes.c_void_p()


CEILING_MODES = {"read": 0, "write": 1, "copy": 2, "add": 3, "rmw": 4, "copy_nt": 5, "add_nt": 6}


def stream_ceiling(mode, a=None, b=None, c=None, nbytes=None, stream=None):
    """One launch of a streaming-ceiling kernel (hoccl_debug_stream_ceiling):
    'read' a, 'write' c, 'copy' a -> c, 'add' c = a + b (fp32), 'rmw' c += 1
    (fp32), 'copy_nt' and 'add_nt' with non-temporal stores.  nbytes
    defaults to the size of the first tensor given."""
    m = CEILING_MODES[mode] if isinstance(mode, str) else int(mode)
    ts = [t for t in (a, b, c) if t is not None]
    if nbytes is None:
        nbytes = ts[0].numel() * ts[0].element_size()
    ptr = lambda t: None if t is None else t.data_ptr()
    with torch.cuda.device(ts[0].device):
        _check(_lib.hoccl_debug_stream_ceiling(m, ptr(a), ptr(b), ptr(c), nbytes, _stream(stream)),
               "hoccl_debug_stream_ceiling")


def ring_hop(partial, local, out=None, hop="middle", stream=None):
    """One ring hop of one rank: out = partial + local in the ring fold's
    arithmetic (hoccl_ring_hop).  With bf16 `local`, `partial` and `out`
    are fp32 or bf16 by hop: "first" bf16 -> fp32, "middle" fp32 -> fp32,
    "last" fp32 -> bf16, "only" bf16 -> bf16; int32 and fp32 use their own
    dtype throughout.  `out` defaults to a new tensor and may be `partial`
    (same dtype) for an in-place update."""
    h = HOPS[hop] if isinstance(hop, str) else int(hop)
    dt = _dtype_of([local])
    bf = local.dtype == torch.bfloat16
    want_in = torch.float32 if bf and h in (HOP_MIDDLE, HOP_LAST) else local.dtype
    want_out = torch.float32 if bf and h in (HOP_FIRST, HOP_MIDDLE) else local.dtype
    if out is None:
        out = torch.empty(local.numel(), dtype=want_out, device=local.device)
    for t, want, name in ((partial, want_in, "partial"), (out, want_out, "out")):
        if t.dtype != want:
            raise TypeError(f"{name} must be {want} for this hop, not {t.dtype}")
        if t.device != local.device:
            raise ValueError("all buffers must live on the same GPU")
        if not t.is_contiguous():
            raise ValueError("buffers must be contiguous")
        if t.numel() != local.numel():
            raise ValueError("partial, local and out must have the same number of elements")
    with torch.cuda.device(local.device):
        _check(_lib.hoccl_ring_hop(partial.data_ptr(), local.data_ptr(), out.data_ptr(), local.numel(),
                                   dt, h, _stream(stream)), "hoccl_ring_hop")
    return out


# ---- operators on a rank's shard (include/hoccl.h has their formulas) ---------------

BLOCK = 128                     # values in 8 bits that share a scale
_FLOATS = {torch.float32: FP32, torch.bfloat16: BF16}
_NOWHERE = contextlib.nullcontext()


# The current device and the current stream's handle without the objects and
# checks around them: 3.2 us of a call's 12.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                      lambda index: torch.cuda.current_stream(index).cuda_stream)


def _at(index, stream):
    """The context of a call on GPU `index` (a tensor's get_device()): that
    GPU current and, given a stream, the stream too, so that what the call
    allocates belongs to it."""
    if index < 0:
        raise ValueError("tensors must live on a GPU")
    if stream is None:
        return _NOWHERE if _current_device() == index else torch.cuda.device(index)
    if stream.device.index != index:
        raise ValueError(f"the stream is on {stream.device}, the tensors on GPU {index}")
    return torch.cuda.stream(stream)


def _handle(index, stream):
    return _raw_stream(index) if stream is None else stream.cuda_stream


def _want(t, name, index, dtypes, shape=None):
    """Checks one operand; returns its dtype's code (or None)."""
    dtype = t.dtype
    if dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(map(str, dtypes))}, not {dtype}")
    if t.get_device() != index:
        raise ValueError("all buffers must live on the same GPU")
    if not t.is_contiguous():
        raise ValueError("buffers must be contiguous")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has the shape {tuple(t.shape)}, not {tuple(shape)}")
    return _FLOATS.get(dtype)


def _scalar(t, name, index, dtype):
    if t.numel() != 1:
        raise ValueError(f"{name} must have one element")
    _want(t, name, index, (dtype,))
    return t.data_ptr()


def adamw_state(params, bits=32):
    """(exp_avgs, exp_avg_sqs, exp_avg_scales, exp_avg_sq_scales) of a first
    adamw step over `params`: zeros, fp32 and no scales (None), or in 8 bits
    with the scales of each BLOCK elements."""
    if bits not in (8, 32):
        raise ValueError(f"bits is 8 or 32, not {bits}")

    def zeros(shape_of, dtype):
        return [torch.zeros(shape_of(p), dtype=dtype, device=p.device) for p in params]

    if bits == 32:
        return zeros(lambda p: p.shape, torch.float32), zeros(lambda p: p.shape, torch.float32), None, None
    q = lambda: [t.view(torch.float8_e4m3fn) for t in zeros(lambda p: p.shape, torch.uint8)]
    s = lambda: zeros(lambda p: -(-p.numel() // BLOCK), torch.float32)
    return q(), q(), s(), s()


def adamw(params, grads, exp_avgs, exp_avg_sqs, exp_avg_scales=None, exp_avg_sq_scales=None, *, step, lr,
          betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, copies=None, grad_scale=None, stream=None):
    """One AdamW step over lists of tensors, in place (hoccl_adamw).  All
    params share a dtype (fp32 or bf16), and all grads.  The states are fp32,
    or float8_e4m3fn with their scales (adamw_state makes either).  `copies`:
    bf16 tensors that receive the new parameters.  `step` counts from 1; it
    may be an int32 tensor of one element on the GPU and `lr` an fp32 one,
    which are then read when the work runs.  `grad_scale`: an fp32 tensor of
    one element that multiplies every gradient.  Params may require gradients:
    like torch's own writes in place under no_grad, the step is no part of a
    graph, and a backward pass over a graph that saved what it overwrote is
    refused.  Returns `params`."""
    n = len(params)
    eight = exp_avg_scales is not None
    if eight != (exp_avg_sq_scales is not None):
        raise ValueError("8-bit states need the scales of both")
    if n == 0 or len(grads) != n:
        if len(grads) != n:
            raise ValueError(f"grads has {len(grads)} tensors, params {n}")
        return params
    index, pdt, gdt = params[0].get_device(), params[0].dtype, grads[0].dtype
    if pdt not in _FLOATS or gdt not in _FLOATS:
        raise TypeError(f"params and grads must be fp32 or bf16, not {pdt} and {gdt}")
    states = torch.float8_e4m3fn if eight else torch.float32
    rows = _tensors.table(index, ("params", params, pdt, 1), ("grads", grads, gdt, 1),
                          ("exp_avgs", exp_avgs, states, 1), ("exp_avg_sqs", exp_avg_sqs, states, 1),
                          ("exp_avg_scales", exp_avg_scales, torch.float32, BLOCK) if eight else None,
                          ("exp_avg_sq_scales", exp_avg_sq_scales, torch.float32, BLOCK) if eight else None,
                          None if copies is None else ("copies", copies, torch.bfloat16, 1))
    with _at(index, stream):
        o = _AdamW(_FLOATS[pdt], _FLOATS[gdt], 8 if eight else 32, 0, 0.0, betas[0], betas[1], eps, weight_decay)
        if isinstance(step, torch.Tensor):
            o.step_dev = _scalar(step, "step", index, torch.int32)
        else:
            o.step = step
        if isinstance(lr, torch.Tensor):
            o.lr_dev = _scalar(lr, "lr", index, torch.float32)
        else:
            o.lr = lr
        if grad_scale is not None:
            o.grad_scale = _scalar(grad_scale, "grad_scale", index, torch.float32)
        _check(_lib.hoccl_adamw(rows, len(rows) // 64, ctypes.byref(o), _handle(index, stream)), "hoccl_adamw")
    _tensors.wrote(params, exp_avgs, exp_avg_sqs, exp_avg_scales, exp_avg_sq_scales, copies)
    return params


def _rows(x):
    if x.dim() == 0:
        raise ValueError("rows of at least one dimension are needed")
    hidden = x.shape[-1]
    return (x.numel() // hidden if hidden else 0), hidden


def rmsnorm(x, weight, residual=None, *, eps=1e-6, quantize=False, out=None, residual_out=None, stream=None):
    """RMS norm over the last dimension of x, or of h = x + residual
    (hoccl_rmsnorm).  Returns y, and with a residual (y, h): h is the new
    residual, rounded to the type of x.  With `quantize` y is a pair of
    float8_e4m3fn values, shaped like x, and fp32 scales [..., blocks of
    BLOCK].  `out` (y, or the pair) and `residual_out` default to new tensors;
    y and residual_out may each be x or residual itself.  The results are no
    part of an autograd graph, whatever requires gradients: rmsnorm_backward
    makes them."""
    index = x.get_device()
    dt = _want(x, "x", index, _FLOATS)
    rows, hidden = _rows(x)
    wdt = _want(weight, "weight", index, _FLOATS, (hidden,))
    if residual is not None:
        _want(residual, "residual", index, (x.dtype,), x.shape)
    given = () if out is None else out if quantize else (out,)
    if residual_out is not None:
        given = (*given, residual_out)
    with _at(index, stream):
        q = scale = y = None
        if quantize:
            blocks = x.shape[:-1] + (-(-hidden // BLOCK),)
            if out is None:
                q = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device)
                scale = torch.empty(blocks, dtype=torch.float32, device=x.device)
            else:
                q, scale = out
                _want(q, "out", index, (torch.float8_e4m3fn,), x.shape)
                _want(scale, "the scales of out", index, (torch.float32,), blocks)
        else:
            y = torch.empty_like(x) if out is None else out
            if out is not None:
                _want(y, "out", index, (x.dtype,), x.shape)
        if residual_out is None:
            if residual is not None:
                residual_out = torch.empty_like(x)
        else:
            _want(residual_out, "residual_out", index, (x.dtype,), x.shape)
        if rows:
            _check(_lib.hoccl_rmsnorm(x.data_ptr(), None if residual is None else residual.data_ptr(), weight.data_ptr(),
                                      None if residual_out is None else residual_out.data_ptr(),
                                      (q if quantize else y).data_ptr(), scale.data_ptr() if quantize else None,
                                      rows, hidden, eps, dt, wdt, _handle(index, stream)), "hoccl_rmsnorm")
            if given:
                _tensors.wrote(given)
    y = (q, scale) if quantize else y
    return y if residual is None else (y, residual_out)


def rmsnorm_backward(grad, h, weight, grad_residual=None, *, eps=1e-6, weight_grad=True, out=None, stream=None):
    """(dx, dweight) of rmsnorm at h (x, or the h that it returned), from the
    gradient of y and, if any, that of h from elsewhere
    (hoccl_rmsnorm_backward).  dx is the gradient of x and of the residual, in
    `out` (a new tensor; or grad, grad_residual or h itself); dweight is fp32,
    or None without `weight_grad`."""
    index = h.get_device()
    dt = _want(h, "h", index, _FLOATS)
    rows, hidden = _rows(h)
    wdt = _want(weight, "weight", index, _FLOATS, (hidden,))
    _want(grad, "grad", index, (h.dtype,), h.shape)
    if grad_residual is not None:
        _want(grad_residual, "grad_residual", index, (h.dtype,), h.shape)
    if out is not None:
        _want(out, "out", index, (h.dtype,), h.shape)
    with _at(index, stream):
        dx = torch.empty_like(h) if out is None else out
        dweight = ws = None
        need = ctypes.c_size_t(0)
        if weight_grad:
            dweight = torch.empty(hidden, dtype=torch.float32, device=h.device)
            if hidden:
                _check(_lib.hoccl_rmsnorm_backward_workspace(rows, hidden, dt, ctypes.byref(need)),
                       "hoccl_rmsnorm_backward_workspace")
            ws = torch.empty(need.value, dtype=torch.uint8, device=h.device)
        if hidden:
            _check(_lib.hoccl_rmsnorm_backward(grad.data_ptr(),
                                               None if grad_residual is None else grad_residual.data_ptr(),
                                               h.data_ptr(), weight.data_ptr(), dx.data_ptr(),
                                               dweight.data_ptr() if weight_grad else None,
                                               ws.data_ptr() if weight_grad else None, need.value, rows, hidden, eps,
                                               dt, wdt, _handle(index, stream)), "hoccl_rmsnorm_backward")
            if out is not None:
                _tensors.wrote((out,))
    return dx, dweight


BalanceLoss = collections.namedtuple("BalanceLoss", "loss expert_tokens rank_tokens coef")


def _balance(logits, experts, ranks, weights=(0.0, 0.0, 0.0), max_ranks=0):
    """The options and host arrays of both directions."""
    if not logits or len(logits) != len(experts):
        raise ValueError("logits and experts must be lists of the same length, one tensor a batch")
    dtype, choices = logits[0].dtype, experts[0].dtype
    if dtype not in _FLOATS:
        raise TypeError(f"logits must be fp32 or bf16, not {dtype}")
    if choices not in (torch.int32, torch.int64):
        raise TypeError(f"experts must be int32 or int64, not {choices}")
    if logits[0].dim() != 2 or experts[0].dim() != 2:
        raise ValueError("logits are [tokens, experts], experts [tokens, topk]")
    E, k = logits[0].shape[1], experts[0].shape[1]
    tokens = _tensors.rows("logits", logits, E)
    if _tensors.rows("experts", experts, k) != tokens:
        raise ValueError("logits and experts must have the same tokens")
    index = logits[0].get_device()
    lp, ep = _tensors.read("logits", logits, dtype, index), _tensors.read("experts", experts, choices, index)
    return index, _Balance(_FLOATS[dtype], choices.itemsize, E, k, ranks, max_ranks, *weights), tokens, lp, ep


def balance_loss(logits, experts, ranks=1, *, expert_weight=1.0, rank_weight=0.0, traffic_weight=0.0, max_ranks=None,
                 stream=None):
    """The router's balance loss over lists of batches, one a rank or a
    sequence (hoccl_balance_loss): logits [tokens, E] (fp32 or bf16), experts
    [tokens, topk] (int32 or int64; what is outside [0, E) is no choice, a
    token without a choice is padding), `ranks` ranks of E / ranks experts.
    Returns a BalanceLoss: loss [batches], expert_tokens [batches, E] and
    rank_tokens [batches, ranks] (int32: choices of an expert, tokens sent to
    a rank), and coef, which balance_loss_backward takes.  The loss is no part
    of an autograd graph, whatever requires gradients: balance_loss_backward
    makes them."""
    index, o, tokens, lp, ep = _balance(logits, experts, ranks, (expert_weight, rank_weight, traffic_weight),
                                        0 if max_ranks is None else max_ranks)
    n, E = len(logits), o.experts
    with _at(index, stream):
        need, device, o_ = ctypes.c_size_t(0), logits[0].device, ctypes.byref(o)
        _check(_lib.hoccl_balance_workspace(tokens, n, o_, ctypes.byref(need)), "hoccl_balance_workspace")
        ws = torch.empty(need.value, dtype=torch.uint8, device=device) if need.value else None
        loss = torch.empty(n, dtype=torch.float32, device=device)
        counts = torch.empty(n, E, dtype=torch.int32, device=device)
        sent = torch.empty(n, ranks, dtype=torch.int32, device=device)
        coef = torch.empty(n, E, dtype=torch.float32, device=device)
        _check(_lib.hoccl_balance_loss(lp, ep, tokens, n, o_, loss.data_ptr(), counts.data_ptr(), sent.data_ptr(),
                                       coef.data_ptr(), None if ws is None else ws.data_ptr(), need.value,
                                       _handle(index, stream)), "hoccl_balance_loss")
    return BalanceLoss(loss, counts, sent, coef)


def balance_loss_backward(logits, experts, coef, grad=None, *, stream=None):
    """The gradients of the logits, from balance_loss's coef and the gradient
    of its losses (fp32 [batches]; ones by default)."""
    index, o, tokens, lp, ep = _balance(logits, experts, 1)
    n = len(logits)
    _want(coef, "coef", index, (torch.float32,), (n, o.experts))
    if grad is not None:
        _want(grad, "grad", index, (torch.float32,), (n,))
    with _at(index, stream):
        out = [torch.empty_like(x) for x in logits]
        _check(_lib.hoccl_balance_loss_backward(lp, ep, tokens, n, ctypes.byref(o), coef.data_ptr(),
                                                None if grad is None else grad.data_ptr(),
                                                _tensors.read("out", out, out[0].dtype, index),
                                                _handle(index, stream)), "hoccl_balance_loss_backward")
    return out
