"""ctypes binding of libivf.so (include/ivf.h): argument marshalling only.

Every step of the computation runs in the HIP kernels behind the C ABI; this
module only passes torch device pointers, sizes and the current HIP stream,
and sizes the caller-owned workspace. There is no CPU path: if the library is
not built, or no GPU is present, the calls raise.
"""
from __future__ import annotations

import collections
import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libivf.so")

IVF_OK, IVF_EINVAL, IVF_EUNSUPPORTED, IVF_ENOMEM, IVF_EDEVICE = range(5)
IVF_F32, IVF_U8, IVF_F16, IVF_BF16 = range(4)
IVF_OP_ROUTE, IVF_OP_KMEANS_STEP, IVF_OP_ASSIGN_BUILD, IVF_OP_BUILD_LISTS, IVF_OP_PQ_TRAIN_STEP, IVF_OP_ADC_SCAN = range(6)
(IVF_OPT_FORCE_FALLBACK, IVF_OPT_SAMPLE_RANK, IVF_OPT_PROFILE, IVF_OPT_BUILD_BLOCKS, IVF_OPT_SCREEN_WAVES,
 IVF_OPT_FP32_SCREEN, IVF_OPT_I8_TWO_PLANE_ONLY, IVF_OPT_FORCE_RESCREEN, IVF_OPT_RESCREEN_CAP,
 IVF_OPT_ASSIGN_SLICE, IVF_OPT_S1_ID_ORDER) = range(11)

STATUS_NAMES = {0: "IVF_OK", 1: "IVF_EINVAL", 2: "IVF_EUNSUPPORTED", 3: "IVF_ENOMEM", 4: "IVF_EDEVICE"}

# Exported symbols and their ctypes signatures: (name, restype, argtypes).
_P = ctypes.c_void_p
_I64, _I32, _U64, _INT, _SZ = ctypes.c_int64, ctypes.c_int32, ctypes.c_uint64, ctypes.c_int, ctypes.c_size_t
SIGNATURES = [
    ("ivf_create", _INT, [_INT, _P, ctypes.POINTER(_P)]),
    ("ivf_destroy", None, [_P]),
    ("ivf_last_error", ctypes.c_char_p, [_P]),
    ("ivf_set_stream", _INT, [_P, _P]),
    ("ivf_workspace_bytes", _SZ, [_INT, _I64, _I64, _I32, _I32]),
    ("ivf_set_workspace", _INT, [_P, _P, _SZ]),
    ("ivf_sync", _INT, [_P]),
    ("ivf_route", _INT, [_P, _P, _I64, _P, _I64, _I32, _I32, _P, _P]),
    ("ivf_route_noalloc", _INT, [_P, _P, _I64, _P, _I64, _I32, _I32, _P, _P]),
    ("ivf_kmeans_step", _INT, [_P, _P, _INT, _I64, _P, _I64, _I32, _U64, _I32, _P, _P, _P, _P, _P]),
    ("ivf_assign_build", _INT, [_P, _P, _INT, _I64, _P, _I64, _I32, _P, _P, _P, _P]),
    ("ivf_build_lists", _INT, [_P, _P, _I64, _I64, _P, _P, _P]),
    ("ivf_last_stats", _INT, [_P, ctypes.POINTER(_I64)]),
    ("ivf_set_option", _INT, [_P, _INT, _I64]),
    ("ivf_kernel_times", _INT, [_P, _INT, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_float)]),
    ("ivf_mfma_probe", _INT, [_P, _I32, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_double)]),
    ("ivf_mfma_probe_i8", _INT, [_P, _I32, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_double)]),
    ("ivf_list_major", _INT, [_P, _P, _INT, _I64, _P, _I64, _I32, _P, _P, _I64, _I64, _P, _P]),
    ("ivf_pq_encode", _INT, [_P, _P, _I64, _I32, _I32, _P, _P]),
    ("ivf_assign_graph", _INT, [_P, _P, _INT, _I64, _P, _I64, _I32, _P, _I32, _P, _P, _P, _P]),
    ("ivf_assign_cells", _INT, [_P, _P, _INT, _I64, _P, _I64, _I32, _P, _I64, _P, _P, _I64, _P, _I32, _I32, _P, _P, _P]),
    ("ivf_adc_scan", _INT, [_P, _P, _I64, _I32, _P, _I64, _P, _I32, _P, _P, _I64, _P, _I32, _P, _I32, _P, _P]),
    ("ivf_pq_train_step", _INT, [_P, _P, _I64, _I32, _I32, _P, _U64, _I32, _P, _P, _P]),
    ("ivf_kv_plan", _INT, [_P, _P, _P, _I64, _I32, _P, _I32, _P, _I64, _I64, _P, _P, _P, _P, _P]),
    ("ivf_kv_fork", _INT, [_P, _P, _P, _I64, _P, _I64, _I32, _P, _I32, _P, _I64, _P, _P, _P]),
    ("ivf_kv_copy", _INT, [_P, _P, _P, _P, _P, _I64]),
    ("ivf_kv_reclaim", _INT, [_P, _P, _I64, _I32, _P, _I32, _I64, _I64, _P, _P, _P, _P]),
    ("ivf_kv_reclaim_bytes", _SZ, [_I64, _I32, _I32, _I64, _I64]),
    ("ivf_kv_append", _INT, [_P, _P, _P, _I64, _I64, _P, _I64, _I64, _P, _I64]),
    ("ivf_kv_read", _INT, [_P, _P, _P, _I64, _P, _P, _P, _I64, _P]),
    ("ivf_kv_select", _INT, [_P, _P, _P, _I64, _I64, _I32, _I64, _P, _P, _P, _I64, _I32, _I32, _I32, _I32, _P]),
    ("ivf_kv_attend_bytes", _SZ, [_P, _I32, _I64, _I64, _I32, _I32, _I64]),
    ("ivf_kv_attend", _INT, [_P, _P, _P, _I64, _I64, _I32, _I64, _P, _P, _P, _P, _I64, _I32, _P, _I32,
                             ctypes.c_float, _I64, _P, _P]),
    ("ivf_sample", _INT, [_P, _P, _INT, _I64, _I64, _I64, _P, _P, _P, _P, _P, _P, _P]),
    ("ivf_sample_bytes", _SZ, [_I64, _I64, _I32]),
    ("ivf_kv_attend_terms", _INT, [_P, _P, _P, _I64, _I64, _I32, _I64, _P, _P, _P, _P, _I64, _I32, _P, _I32,
                                   ctypes.c_float, _I64, _P, _P, _P]),
]

_lib = None


class IvfError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, status), message))
        self.status = status


def load_library(path: str = LIB_PATH):
    """Loads libivf.so (after torch, so that both share one HIP runtime)."""
    global _lib
    if _lib is None:
        try:
            import torch  # noqa: F401
        except ImportError:  # pragma: no cover - torch is part of the image
            pass
        if not os.path.exists(path):
            raise RuntimeError("libivf.so is not built (%s); run __graft_entry__.build()" % path)
        lib = ctypes.CDLL(path)
        for name, res, args in SIGNATURES:
            f = getattr(lib, name)
            f.restype = res
            f.argtypes = args
        _lib = lib
    return _lib


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


_raw_stream = None


def _stream_handle(device=None):
    global _raw_stream
    if _raw_stream is None:
        import torch

        # torch.cuda.current_stream() builds a Stream object (3 us); the raw query is 0.1 us
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda device: torch.cuda.current_stream(device).cuda_stream)
    if device is None:
        import torch

        device = torch.cuda.current_device()
    return _raw_stream(device)


class Context:
    """An ivf_ctx bound to a device and to torch's current stream, plus a
    grow-only workspace tensor allocated through torch.

    Calls may be captured into graphs. A graph keeps the address of the
    workspace that its calls were captured with, so a workspace that a capture
    has used lives as long as the context, also where a later call replaces it by
    a larger one, and the context has to outlive its graphs."""

    def __init__(self, device: int = 0):
        import torch

        self.lib = load_library()
        self.device = device
        self._ws = None
        self._ws_captured = False  # a captured call holds its address
        self._ws_streams = set()  # the streams that torch knows to use it
        self._kept = []  # replaced workspaces of captured calls
        h = ctypes.c_void_p()
        if device >= 0:
            with torch.cuda.device(device):
                st = self.lib.ivf_create(device, _stream_handle(), ctypes.byref(h))
        else:
            st = self.lib.ivf_create(device, None, ctypes.byref(h))
        if st != IVF_OK:
            raise IvfError(st, "ivf_create(%d) failed" % device)
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            self.lib.ivf_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def error(self) -> str:
        return (self.lib.ivf_last_error(self.handle) or b"").decode()

    def check(self, st: int, what: str):
        if st != IVF_OK:
            raise IvfError(st, "%s: %s" % (what, self.error()))

    def set_option(self, option: int, value: int):
        self.check(self.lib.ivf_set_option(self.handle, option, value), "ivf_set_option")

    def ensure_workspace(self, nbytes: int):
        import torch

        stream = _stream_handle(self.device)
        if self._ws is None or self._ws.numel() < nbytes:
            if self._ws_captured:
                self._kept.append(self._ws)
            self._ws, self._ws_captured = None, False
            self._ws = torch.empty(max(nbytes, 1 << 20), dtype=torch.uint8, device="cuda:%d" % self.device)
            self._ws_streams = {stream}
        if torch.cuda.is_current_stream_capturing():
            self._ws_captured = True
        elif stream not in self._ws_streams:
            # its memory is handed on only after what this stream does with it
            self._ws.record_stream(torch.cuda.current_stream(self.device))
            self._ws_streams.add(stream)
        self.check(self.lib.ivf_set_workspace(self.handle, _ptr(self._ws), self._ws.numel()),
                   "ivf_set_workspace")

    def bind_stream(self):
        self.check(self.lib.ivf_set_stream(self.handle, _stream_handle()), "ivf_set_stream")

    def bind(self):
        """Binds torch's current stream of the device; the library and the context's handle."""
        # each time: the handle may have been given another stream since
        self.lib.ivf_set_stream(self.handle, _stream_handle(self.device))
        return self.lib, self.handle

    def sync(self):
        self.check(self.lib.ivf_sync(self.handle), "ivf_sync")

    def kernel_times(self):
        """[(kernel name, ms)] of every launch recorded with IVF_OPT_PROFILE on
        since the last read (the read clears the timeline)."""
        n = self.lib.ivf_kernel_times(self.handle, 0, None, None)
        if n < 0:
            raise IvfError(IVF_EDEVICE, "ivf_kernel_times failed")
        names = (ctypes.c_char_p * max(n, 1))()
        ms = (ctypes.c_float * max(n, 1))()
        self.lib.ivf_kernel_times(self.handle, n, names, ms)
        return [(names[i].decode(), float(ms[i])) for i in range(n)]

    def mfma_probe(self, iters: int = 20000):
        """(ms, TFLOP/s) of the fp32 MFMA throughput probe (synchronises)."""
        ms = ctypes.c_float()
        tf = ctypes.c_double()
        self.bind_stream()
        self.check(self.lib.ivf_mfma_probe(self.handle, iters, ctypes.byref(ms), ctypes.byref(tf)),
                   "ivf_mfma_probe")
        return float(ms.value), float(tf.value)

    def mfma_probe_i8(self, iters: int = 20000):
        """(ms, TOP/s) of the int8 MFMA throughput probe (synchronises)."""
        ms = ctypes.c_float()
        tops = ctypes.c_double()
        self.bind_stream()
        self.check(self.lib.ivf_mfma_probe_i8(self.handle, iters, ctypes.byref(ms), ctypes.byref(tops)),
                   "ivf_mfma_probe_i8")
        return float(ms.value), float(tops.value)

    def last_stats(self):
        out = (ctypes.c_int64 * 8)()
        self.check(self.lib.ivf_last_stats(self.handle, out), "ivf_last_stats")
        keys = ("fallback", "refine2", "candidates", "overflow", "sample", "screen_i8", "rescreen", "screen_f16")
        return {k: int(out[i]) for i, k in enumerate(keys)}


def _dtype_code(t):
    import torch

    if t.dtype == torch.uint8:
        return IVF_U8
    if t.dtype == torch.float32:
        return IVF_F32
    raise TypeError("rows must be float32 or uint8, got %s" % t.dtype)


def _device_tensor(t, name):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous device tensor" % name)


def ivf_route(ctx: Context, queries, centroids, nprobe: int, out_ids=None, out_dist=None,
              want_dist: bool = True):
    """Coarse search (Eq. 1 with Eq. 6): ids [Q, nprobe] int32 and squared L2
    distances [Q, nprobe] fp32, ascending (distance, id)."""
    import torch

    _device_tensor(queries, "queries")
    _device_tensor(centroids, "centroids")
    Q, D = queries.shape
    C = centroids.shape[0]
    dev = queries.device
    if out_ids is None:
        out_ids = torch.empty((Q, nprobe), dtype=torch.int32, device=dev)
    if out_dist is None and want_dist:
        out_dist = torch.empty((Q, nprobe), dtype=torch.float32, device=dev)
    ctx.ensure_workspace(ctx.lib.ivf_workspace_bytes(IVF_OP_ROUTE, Q, C, D, nprobe))
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_route(ctx.handle, _ptr(queries), Q, _ptr(centroids), C, D, nprobe,
                                _ptr(out_ids), _ptr(out_dist)), "ivf_route")
    return out_ids, out_dist


def ivf_route_noalloc(ctx: Context, queries, centroids, nprobe: int, out_ids, out_dist=None):
    """ivf_route without a workspace: the library's static device scratch is
    used and nothing is allocated by the call (out_ids / out_dist are the
    caller's). Calls that overlap on one device race."""
    _device_tensor(queries, "queries")
    _device_tensor(centroids, "centroids")
    Q, D = queries.shape
    C = centroids.shape[0]
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_route_noalloc(ctx.handle, _ptr(queries), Q, _ptr(centroids), C, D, nprobe,
                                        _ptr(out_ids), _ptr(out_dist)), "ivf_route_noalloc")
    return out_ids, out_dist


def ivf_kmeans_step(ctx: Context, train, centroids, seed: int = 0, it: int = 0, out_labels=None,
                    out_centroids=None, out_counts=None, out_objective=None, hint_labels=None):
    """One Lloyd iteration: labels [N] int32, new centroids [C, D] fp32,
    counts [C] int64 (before reseeding), objective (device fp64 scalar).
    `hint_labels` (int32 [N], e.g. the previous iteration's labels) only
    changes the speed."""
    import torch

    _device_tensor(train, "train")
    _device_tensor(centroids, "centroids")
    N, D = train.shape
    C = centroids.shape[0]
    dev = train.device
    if out_labels is None:
        out_labels = torch.empty(N, dtype=torch.int32, device=dev)
    if out_centroids is None:
        out_centroids = torch.empty((C, D), dtype=torch.float32, device=dev)
    if out_counts is None:
        out_counts = torch.empty(C, dtype=torch.int64, device=dev)
    if out_objective is None:
        out_objective = torch.empty(2, dtype=torch.float64, device=dev)
    if hint_labels is not None:
        _device_tensor(hint_labels, "hint_labels")
    ctx.ensure_workspace(ctx.lib.ivf_workspace_bytes(IVF_OP_KMEANS_STEP, N, C, D, 0))
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_kmeans_step(ctx.handle, _ptr(train), _dtype_code(train), N, _ptr(centroids),
                                      C, D, seed & (2**64 - 1), it, _ptr(out_labels),
                                      _ptr(out_centroids), _ptr(out_counts), _ptr(out_objective),
                                      _ptr(hint_labels) if hint_labels is not None else None),
              "ivf_kmeans_step")
    return out_labels, out_centroids, out_counts, out_objective


def ivf_assign_build(ctx: Context, base, centroids, out_labels=None, out_counts=None,
                     out_offsets=None, out_perm=None):
    """Full assignment + inverted lists: labels [N], counts [C], offsets [C+1], perm [N]."""
    import torch

    _device_tensor(base, "base")
    _device_tensor(centroids, "centroids")
    N, D = base.shape
    C = centroids.shape[0]
    dev = base.device
    if out_labels is None:
        out_labels = torch.empty(N, dtype=torch.int32, device=dev)
    if out_counts is None:
        out_counts = torch.empty(C, dtype=torch.int64, device=dev)
    if out_offsets is None:
        out_offsets = torch.empty(C + 1, dtype=torch.int64, device=dev)
    if out_perm is None:
        out_perm = torch.empty(N, dtype=torch.int32, device=dev)  # uint32 bit pattern
    ctx.ensure_workspace(ctx.lib.ivf_workspace_bytes(IVF_OP_ASSIGN_BUILD, N, C, D, 0))
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_assign_build(ctx.handle, _ptr(base), _dtype_code(base), N, _ptr(centroids),
                                       C, D, _ptr(out_labels), _ptr(out_counts), _ptr(out_offsets),
                                       _ptr(out_perm)), "ivf_assign_build")
    return out_labels, out_counts, out_offsets, out_perm


def ivf_build_lists(ctx: Context, labels, C: int, out_counts=None, out_offsets=None, out_perm=None):
    """Inverted lists for given labels: counts [C], offsets [C+1], perm [N] (uint32 bits in int32)."""
    import torch

    _device_tensor(labels, "labels")
    N = labels.shape[0]
    dev = labels.device
    if out_counts is None:
        out_counts = torch.empty(C, dtype=torch.int64, device=dev)
    if out_offsets is None:
        out_offsets = torch.empty(C + 1, dtype=torch.int64, device=dev)
    if out_perm is None:
        out_perm = torch.empty(N, dtype=torch.int32, device=dev)
    ctx.ensure_workspace(ctx.lib.ivf_workspace_bytes(IVF_OP_BUILD_LISTS, N, C, 0, 0))
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_build_lists(ctx.handle, _ptr(labels), N, C, _ptr(out_counts),
                                      _ptr(out_offsets), _ptr(out_perm)), "ivf_build_lists")
    return out_counts, out_offsets, out_perm


def ivf_list_major(ctx: Context, base, centroids, offsets, perm, pos0: int = 0, n=None,
                   rows: bool = True, residuals: bool = True, out_rows=None, out_residuals=None):
    """List-major copy base[perm[pos0:pos0+n]] and residuals against each
    position's list centroid (fp32). Returns (rows or None, residuals or None)."""
    import torch

    for t, name in ((base, "base"), (centroids, "centroids"), (offsets, "offsets"), (perm, "perm")):
        _device_tensor(t, name)
    N, D = base.shape
    C = centroids.shape[0]
    if n is None:
        n = N - pos0
    dev = base.device
    if rows and out_rows is None:
        out_rows = torch.empty((n, D), dtype=base.dtype, device=dev)
    if residuals and out_residuals is None:
        out_residuals = torch.empty((n, D), dtype=torch.float32, device=dev)
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_list_major(ctx.handle, _ptr(base), _dtype_code(base), N, _ptr(centroids), C, D,
                                     _ptr(offsets), _ptr(perm), pos0, n,
                                     _ptr(out_rows if rows else None),
                                     _ptr(out_residuals if residuals else None)), "ivf_list_major")
    return (out_rows if rows else None), (out_residuals if residuals else None)


PQ_K = 256


def ivf_pq_encode(ctx: Context, x, codebooks, out_codes=None):
    """PQ codes uint8 [n, M] of fp32 rows x [n, D] with codebooks [M, 256, D/M]."""
    import torch

    _device_tensor(x, "x")
    _device_tensor(codebooks, "codebooks")
    n, D = x.shape
    M = codebooks.shape[0]
    if out_codes is None:
        out_codes = torch.empty((n, M), dtype=torch.uint8, device=x.device)
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_pq_encode(ctx.handle, _ptr(x), n, D, M, _ptr(codebooks), _ptr(out_codes)),
              "ivf_pq_encode")
    return out_codes


def ivf_pq_train_step(ctx: Context, x, codebooks, seed: int = 0, it: int = 0, out_codebooks=None,
                      out_counts=None, out_objective=None):
    """One Lloyd step per subspace: (codebooks [M, 256, D/M], counts int64 [M, 256],
    objectives fp64 [M])."""
    import torch

    _device_tensor(x, "x")
    _device_tensor(codebooks, "codebooks")
    n, D = x.shape
    M = codebooks.shape[0]
    dev = x.device
    if out_codebooks is None:
        out_codebooks = torch.empty_like(codebooks)
    if out_counts is None:
        out_counts = torch.empty((M, PQ_K), dtype=torch.int64, device=dev)
    if out_objective is None:
        out_objective = torch.empty(M, dtype=torch.float64, device=dev)
    ctx.ensure_workspace(ctx.lib.ivf_workspace_bytes(IVF_OP_PQ_TRAIN_STEP, n, M, D, 0))
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_pq_train_step(ctx.handle, _ptr(x), n, D, M, _ptr(codebooks), seed & (2**64 - 1), it,
                                        _ptr(out_codebooks), _ptr(out_counts), _ptr(out_objective)),
              "ivf_pq_train_step")
    return out_codebooks, out_counts, out_objective


def ivf_assign_graph(ctx: Context, rows, centroids, graph, prev, order=None, out_labels=None, out_dist=None,
                     want_dist: bool = True):
    """Nearest of each row's candidates graph[prev[i]] (int32 [C, S]):
    labels int32 [N] and squared distances fp32 [N]. `order` (int32 [N] or
    None) only sets the processing order."""
    import torch

    for t, name in ((rows, "rows"), (centroids, "centroids"), (graph, "graph"), (prev, "prev")):
        _device_tensor(t, name)
    N, D = rows.shape
    C = centroids.shape[0]
    S = graph.shape[1]
    if out_labels is None:
        out_labels = torch.empty(N, dtype=torch.int32, device=rows.device)
    if want_dist and out_dist is None:
        out_dist = torch.empty(N, dtype=torch.float32, device=rows.device)
    ctx.bind_stream()
    if order is not None:
        _device_tensor(order, "order")
    ctx.check(ctx.lib.ivf_assign_graph(ctx.handle, _ptr(rows), _dtype_code(rows), N, _ptr(centroids), C, D,
                                       _ptr(graph), S, _ptr(prev), _ptr(order) if order is not None else None,
                                       _ptr(out_labels), _ptr(out_dist if want_dist else None)),
              "ivf_assign_graph")
    return out_labels, (out_dist if want_dist else None)


def ivf_assign_cells(ctx: Context, rows, centroids, cell, cell_offsets, cell_members, graph=None, hops: int = 0,
                     order=None, out_labels=None, out_dist=None, want_dist: bool = True):
    """Nearest member of each row's coarse cell, then up to `hops` greedy
    moves over graph (int32 [C, S] or None): labels int32 [N] and squared
    distances fp32 [N]. `order` (int32 [N] or None) only sets the processing
    order."""
    import torch

    for t, name in ((rows, "rows"), (centroids, "centroids"), (cell, "cell"), (cell_offsets, "cell_offsets"),
                    (cell_members, "cell_members")):
        _device_tensor(t, name)
    if graph is not None:
        _device_tensor(graph, "graph")
    if order is not None:
        _device_tensor(order, "order")
    N, D = rows.shape
    C = centroids.shape[0]
    G = cell_offsets.shape[0] - 1
    M = cell_members.shape[0]
    S = graph.shape[1] if graph is not None else 0
    if out_labels is None:
        out_labels = torch.empty(N, dtype=torch.int32, device=rows.device)
    if want_dist and out_dist is None:
        out_dist = torch.empty(N, dtype=torch.float32, device=rows.device)
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_assign_cells(ctx.handle, _ptr(rows), _dtype_code(rows), N, _ptr(centroids), C, D,
                                       _ptr(cell), G, _ptr(cell_offsets), _ptr(cell_members) if M else None, M,
                                       _ptr(graph) if graph is not None else None, S, hops,
                                       _ptr(order) if order is not None else None, _ptr(out_labels),
                                       _ptr(out_dist if want_dist else None)), "ivf_assign_cells")
    return out_labels, (out_dist if want_dist else None)


def ivf_adc_scan(ctx: Context, queries, centroids, probes, offsets, perm, codes, codebooks, k: int,
                 out_ids=None, out_dist=None):
    """Residual-PQ ADC scan: each query's k best (approximate distance, row id)
    over its probed lists. Returns (ids [B, k] uint32 bits in int32, dist [B, k])."""
    import torch

    for t, name in ((queries, "queries"), (centroids, "centroids"), (probes, "probes"), (offsets, "offsets"),
                    (perm, "perm"), (codes, "codes"), (codebooks, "codebooks")):
        _device_tensor(t, name)
    B, D = queries.shape
    C = centroids.shape[0]
    P = probes.shape[1]
    N, M = codes.shape
    dev = queries.device
    if out_ids is None:
        out_ids = torch.empty((B, k), dtype=torch.int32, device=dev)
    if out_dist is None:
        out_dist = torch.empty((B, k), dtype=torch.float32, device=dev)
    ctx.ensure_workspace(ctx.lib.ivf_workspace_bytes(IVF_OP_ADC_SCAN, B, P, D, k))
    ctx.bind_stream()
    ctx.check(ctx.lib.ivf_adc_scan(ctx.handle, _ptr(queries), B, D, _ptr(centroids), C, _ptr(probes), P,
                                   _ptr(offsets), _ptr(perm), N, _ptr(codes), M, _ptr(codebooks), k,
                                   _ptr(out_ids), _ptr(out_dist)), "ivf_adc_scan")
    return out_ids, out_dist


# ---- the paged 4-bit key/value cache ------------------------------------------
# The calls of a decoding step are small, so that the checks and allocations here
# weigh as much as the kernels: few attribute reads, and outputs of one call carved
# from one allocation.

class _KvCacheStruct(ctypes.Structure):
    """ivf_kv_cache."""
    _fields_ = [("records", _P), ("summary", _P), ("weight", _P), ("blocks", _I64), ("block_size", _I32),
                ("heads", _I32), ("dim", _I32), ("dtype", _I32)]


class _KvTermsStruct(ctypes.Structure):
    """ivf_kv_terms."""
    _fields_ = [("cap", ctypes.c_float), ("slopes", _P), ("first", _P), ("prefix", _P)]


class KVCache:
    """A paged key/value cache held in 4 bits: `records` uint8 [blocks, heads,
    block_size * dim * 17 / 16], `summary` int8 [blocks, heads, dim] and
    `weight` fp32 [blocks, heads] (layout: ivf_kv_cache in include/ivf.h), for
    keys, values and queries of `dtype` (torch.float16 or torch.bfloat16)."""

    def __init__(self, records, summary, weight, block_size: int, dtype):
        import torch

        for t, name, kind in ((records, "records", torch.uint8), (summary, "summary", torch.int8),
                              (weight, "weight", torch.float32)):
            _device_tensor(t, name)
            if t.dtype != kind:
                raise TypeError("%s must be %s, got %s" % (name, kind, t.dtype))
        codes = {torch.float16: IVF_F16, torch.bfloat16: IVF_BF16}
        if dtype not in codes:
            raise TypeError("the cache's type must be float16 or bfloat16, got %s" % dtype)
        if summary.dim() != 3:
            raise ValueError("summary must be [blocks, heads, dim], got %s" % (tuple(summary.shape),))
        blocks, heads, dim = summary.shape
        if tuple(records.shape) != (blocks, heads, block_size * dim * 17 // 16) or tuple(weight.shape) != (blocks, heads):
            raise ValueError("records %s, summary %s and weight %s do not belong together (block_size %d)" % (
                tuple(records.shape), tuple(summary.shape), tuple(weight.shape), block_size))
        if not records.device == summary.device == weight.device:
            raise ValueError("records, summary and weight must lie on one device")
        self.device = records.get_device()
        self.records, self.summary, self.weight = records, summary, weight
        self.blocks, self.heads, self.dim, self.block_size, self.dtype = blocks, heads, dim, block_size, dtype
        self.struct = _KvCacheStruct(records.data_ptr(), summary.data_ptr(), weight.data_ptr(), blocks, block_size,
                                     heads, dim, codes[dtype])
        self.ref = ctypes.byref(self.struct)
        self._workspace = {}  # bytes that an attention call of given sizes asks for

    @classmethod
    def empty(cls, blocks: int, heads: int, dim: int, block_size: int = 64, dtype=None, device="cuda"):
        """A cache of `blocks` unwritten blocks."""
        import torch

        new = lambda shape, kind: torch.zeros(shape, dtype=kind, device=device)  # noqa: E731
        return cls(new((blocks, heads, block_size * dim * 17 // 16), torch.uint8), new((blocks, heads, dim), torch.int8),
                   new((blocks, heads), torch.float32), block_size, dtype or torch.bfloat16)

    def attend_bytes(self, ctx, *sizes):
        """ivf_kv_attend_bytes for these (query heads, T, B, columns, count, longest)."""
        need = self._workspace.get(sizes)
        if need is None:
            if len(self._workspace) >= 1024:
                self._workspace.clear()
            need = self._workspace[sizes] = ctx.lib.ivf_kv_attend_bytes(self.ref, *sizes)
        return need


KVPlan = collections.namedtuple("KVPlan", "start slots request position info")
KVFork = collections.namedtuple("KVFork", "source to info")
KVReclaim = collections.namedtuple("KVReclaim", "free source to info")


def _grad_enabled():
    import torch

    return torch.is_grad_enabled()


def _rows(ctx, t, name, cache, heads=None):
    """(pointer, token stride, head stride) of rows [tokens, heads, dim]."""
    device = ctx.device
    if cache.device != device:
        raise TypeError("the cache must be on the context's device %d, is on %s" % (device, cache.records.device))
    if t.get_device() != device or t.dtype != cache.dtype:
        raise TypeError("%s must be of the cache's type %s on device %d, got %s on %s" % (
            name, cache.dtype, device, t.dtype, t.device))
    if t.requires_grad and _grad_enabled():
        raise RuntimeError("%s requires a gradient, and the cache's calls have no backward pass: detach it, or call "
                           "under torch.no_grad()" % name)
    shape = t.shape
    if len(shape) != 3 or shape[2] != cache.dim or (heads is not None and shape[1] != heads):
        raise ValueError("%s must be [tokens, %s, %d], got %s" % (name, heads or "heads", cache.dim, tuple(shape)))
    if shape[0] == 0 or shape[1] == 0:
        return None, 0, 0
    st, sh, sd = t.stride()
    if sd != 1:
        raise ValueError("%s: channels must be contiguous" % name)
    return t.data_ptr(), st if shape[0] > 1 else 0, sh if shape[1] > 1 else 0


def _ints(ctx, t, name, shape, kind):
    """The pointer of a contiguous tensor of this type and shape on the context's device."""
    if t.dtype != kind or t.get_device() != ctx.device:
        raise TypeError("%s must be %s on device %d, got %s on %s" % (name, kind, ctx.device, t.dtype, t.device))
    if t.shape != shape:
        raise ValueError("%s must be %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


def ivf_kv_plan(ctx: Context, cached, added, block_size: int, table, free_blocks, tokens: int, want_info: bool = False):
    """Block tables and slots of a batch: requests of cached[b] tokens (int32 [B])
    bring added[b] more, `tokens` in all. Fills `table` (int32 [B, columns]) in
    place with blocks of free_blocks (int32, taken in order) and returns
    KVPlan(start [B + 1], slots int64 [tokens], request [tokens], position
    [tokens], info int64 [4] or None: tokens, blocks asked for, blocks taken, requests
    beyond the table)."""
    import torch

    i32 = torch.int32
    B = cached.shape[0]
    shape = table.shape
    if len(shape) != 2 or shape[0] != B:
        raise ValueError("table must be [%d, columns], got %s" % (B, tuple(shape)))
    if tokens < 0:
        raise ValueError("tokens must be >= 0, got %d" % tokens)
    n_free = free_blocks.numel()
    ins = (_ints(ctx, cached, "cached", (B,), i32), _ints(ctx, added, "added", (B,), i32), B, block_size,
           _ints(ctx, table, "table", shape, i32), shape[1], _ints(ctx, free_blocks, "free_blocks", (n_free,), i32),
           n_free, tokens)
    # slots (two words each) come first: 8-byte aligned; parts without gradients, at half the cost of views
    whole = torch.empty(4 * tokens + B + 1, dtype=i32, device=cached.device)
    slots, request, position, start = torch.unsafe_split_with_sizes(whole, (2 * tokens, tokens, tokens, B + 1))
    info = torch.empty(4, dtype=torch.int64, device=cached.device) if want_info else None
    at = whole.data_ptr()
    lib, handle = ctx.bind()
    st = lib.ivf_kv_plan(handle, *ins, at + 16 * tokens, at, at + 8 * tokens, at + 12 * tokens,
                         info.data_ptr() if want_info else None)
    if st:
        ctx.check(st, "ivf_kv_plan")
    return KVPlan(start, slots.view(torch.int64), request, position, info)


def ivf_kv_fork(ctx: Context, parent, child, cached, block_size: int, table, free_blocks, want_info: bool = False):
    """Requests that go on from another's tokens: rows child (int32 [n]) of `table`
    (int32 [B, columns]) and `cached` (int32 [B]) become those of `parent`, in place, a
    partly filled last block replaced by one of free_blocks (int32, taken in order).
    Returns KVFork(source [n], to [n], info int64 [2] or None): the pairs that
    ivf_kv_copy has to copy, -1 where there is nothing to copy; blocks asked for and
    taken. A row that is a parent is no child in the same call: such forks are left out."""
    import torch

    i32 = torch.int32
    shape = table.shape
    if len(shape) != 2:
        raise ValueError("table must be [requests, columns], got %s" % (tuple(shape),))
    n, n_free = parent.numel(), free_blocks.numel()
    ins = (_ints(ctx, parent, "parent", (n,), i32), _ints(ctx, child, "child", (n,), i32), n,
           _ints(ctx, cached, "cached", shape[:1], i32), shape[0], block_size, _ints(ctx, table, "table", shape, i32),
           shape[1], _ints(ctx, free_blocks, "free_blocks", (n_free,), i32), n_free)
    source, to = torch.unsafe_split_with_sizes(torch.empty(2 * n, dtype=i32, device=table.device), (n, n))
    info = torch.empty(2, dtype=torch.int64, device=table.device) if want_info else None
    lib, handle = ctx.bind()
    st = lib.ivf_kv_fork(handle, *ins, source.data_ptr(), to.data_ptr(), info.data_ptr() if want_info else None)
    if st:
        ctx.check(st, "ivf_kv_fork")
    return KVFork(source, to, info)


def ivf_kv_copy(ctx: Context, cache: KVCache, to, source, source_cache: KVCache | None = None):
    """Copies blocks `source` (int32 [n]) of source_cache (default: the cache
    itself) into blocks `to` (int32 [n]) of cache. Pairs of -1 are skipped."""
    import torch

    other = cache if source_cache is None else source_cache
    for c in (cache, other):
        if c.device != ctx.device:
            raise TypeError("the cache must be on the context's device %d, is on %s" % (ctx.device, c.records.device))
    n = to.numel()
    args = _ints(ctx, to, "to", (n,), torch.int32), _ints(ctx, source, "source", (n,), torch.int32), n
    lib, handle = ctx.bind()
    st = lib.ivf_kv_copy(handle, cache.ref, other.ref, *args)
    if st:
        ctx.check(st, "ivf_kv_copy")


_reclaim_bytes = {}  # workspace of calls of given sizes


def ivf_kv_reclaim(ctx: Context, cached, block_size: int, table, blocks: int, moves: int = 0):
    """The blocks (of `blocks`) that no request holds: request b holds those of the
    first ceil(cached[b] / block_size) columns of its row of `table` (int32 [B, columns]).
    With `moves`, up to so many held blocks are first moved into free ones of lower
    numbers, in `table`. Returns KVReclaim(free [blocks] ascending, -1 behind them,
    source [moves], to [moves]: the pairs that ivf_kv_copy has to copy before the free
    blocks are used, -1 behind them, info int64 [3]: blocks held, moves made, blocks free)."""
    import torch

    i32 = torch.int32
    shape = table.shape
    if len(shape) != 2:
        raise ValueError("table must be [requests, columns], got %s" % (tuple(shape),))
    if moves < 0 or blocks < 1:
        raise ValueError("blocks >= 1 and moves >= 0 are wanted, got %d and %d" % (blocks, moves))
    B, cols = shape
    ins = (_ints(ctx, cached, "cached", (B,), i32), B, block_size, _ints(ctx, table, "table", shape, i32), cols, blocks, moves)
    whole = torch.empty(6 + blocks + 2 * moves, dtype=i32, device=table.device)  # info (two words each) comes first
    info, free, source, to = torch.unsafe_split_with_sizes(whole, (6, blocks, moves, moves))
    sizes = B, block_size, cols, blocks, moves
    need = _reclaim_bytes.get(sizes)  # (goes by sizes alone)
    if need is None:
        if len(_reclaim_bytes) >= 1024:
            _reclaim_bytes.clear()
        need = _reclaim_bytes[sizes] = ctx.lib.ivf_kv_reclaim_bytes(*sizes)
    if need:
        ctx.ensure_workspace(need)
    at = whole.data_ptr()
    lib, handle = ctx.bind()
    st = lib.ivf_kv_reclaim(handle, *ins, at + 24, at + 24 + 4 * blocks, at + 24 + 4 * (blocks + moves), at)
    if st:
        ctx.check(st, "ivf_kv_reclaim")
    return KVReclaim(free, source, to, info.view(torch.int64))


def ivf_kv_append(ctx: Context, cache: KVCache, k, v, slots):
    """Writes keys and values [T, heads, dim] into the cache at slots (int64 [T])."""
    import torch

    T = slots.shape[0]
    kp, kt, kh = _rows(ctx, k, "k", cache, cache.heads)
    vp, vt, vh = _rows(ctx, v, "v", cache, cache.heads)
    if k.shape[0] != T or v.shape[0] != T:
        raise ValueError("k and v must hold one row per slot (%d)" % T)
    lib, handle = ctx.bind()
    st = lib.ivf_kv_append(handle, cache.ref, kp, kt, kh, vp, vt, vh, _ints(ctx, slots, "slots", (T,), torch.int64), T)
    if st:
        ctx.check(st, "ivf_kv_append")


def ivf_kv_read(ctx: Context, cache: KVCache, slots, blocks=None):
    """The cache's values: keys and values [T, heads, dim] at slots (int64 [T])
    and, of `blocks` (int32 [n]), the key means [n, heads, dim] fp32 (else None)."""
    import torch

    if cache.device != ctx.device:
        raise TypeError("the cache must be on the context's device %d, is on %s" % (ctx.device, cache.records.device))
    T = slots.shape[0]
    k = torch.empty(T, cache.heads, cache.dim, dtype=cache.dtype, device=slots.device)
    v = torch.empty_like(k)
    mean, n, p_blocks, p_mean = None, 0, None, None
    if blocks is not None:
        n = blocks.shape[0]
        p_blocks = _ints(ctx, blocks, "blocks", (n,), torch.int32)
        mean = torch.empty(n, cache.heads, cache.dim, dtype=torch.float32, device=slots.device)
        p_mean = mean.data_ptr()
    lib, handle = ctx.bind()
    st = lib.ivf_kv_read(handle, cache.ref, _ints(ctx, slots, "slots", (T,), torch.int64), T, k.data_ptr(), v.data_ptr(),
                         p_blocks, n, p_mean)
    if st:
        ctx.check(st, "ivf_kv_read")
    return k, v, mean


def ivf_kv_select(ctx: Context, cache: KVCache, q, request, position, table, count: int, first: int = 1, last: int = 1):
    """The blocks that the queries q [T, query heads, dim] read: int32 [T, heads,
    count] columns of the request's row of `table`, ascending, -1 behind. The
    first `first` and the last `last` blocks are always among them."""
    import torch

    i32 = torch.int32
    qp, qt, qh = _rows(ctx, q, "q", cache)
    T, Hq, _ = q.shape
    B, cols = table.shape
    out = torch.empty(T, cache.heads, max(count, 0), dtype=i32, device=q.device)
    lib, handle = ctx.bind()
    st = lib.ivf_kv_select(handle, cache.ref, qp, qt, qh, Hq, T, _ints(ctx, request, "request", (T,), i32),
                           _ints(ctx, position, "position", (T,), i32), _ints(ctx, table, "table", (B, cols), i32), B,
                           cols, first, last, count, out.data_ptr())
    if st:
        ctx.check(st, "ivf_kv_select")
    return out


def ivf_kv_attend(ctx: Context, cache: KVCache, q, start, request, position, table, scale: float, longest: int,
                  blocks=None, out=None, out_lse=None, want_lse: bool = True, cap: float = 0.0, slopes=None,
                  first=None, prefix=None):
    """Attention of queries q [T, query heads, dim] over their requests' tokens in
    the cache, or over the selected `blocks` (int32 [T, heads, count]) only:
    outputs like q and the log-sum-exps fp32 [T, query heads]. `longest` is at
    least the largest number of tokens that one request has in the batch. Without
    `blocks`, rows past start[B] (padding of the batch) are left unwritten.

    With `cap` a score x is cap * tanh(x / cap); with `slopes` (fp32 [query heads])
    it then loses slope * |p - j| for the positions p of the query and j of the key;
    with `first` and `prefix` (int32 [T]) a token sees the keys first <= j <= p and
    j < prefix (ivf_kv_terms in include/ivf.h)."""
    import torch

    i32 = torch.int32
    qp, qt, qh = _rows(ctx, q, "q", cache)
    T, Hq, dim = q.shape
    B, cols = table.shape
    p_blocks, count = None, 0
    if blocks is not None:
        count = blocks.shape[-1]
        p_blocks = _ints(ctx, blocks, "blocks", (T, cache.heads, count), i32)
    if out is None:
        out = q.new_empty(T, Hq, dim)
    elif (out.get_device() != ctx.device or not out.is_contiguous() or out.dtype != cache.dtype
          or out.shape != (T, Hq, dim)):
        raise ValueError("out must be contiguous %s %s on the context's device" % ((T, Hq, dim), cache.dtype))
    if out_lse is None:
        if want_lse:
            out_lse = torch.empty(T, Hq, dtype=torch.float32, device=q.device)
    elif (out_lse.get_device() != ctx.device or not out_lse.is_contiguous() or out_lse.dtype != torch.float32
          or out_lse.shape != (T, Hq)):
        raise ValueError("out_lse must be contiguous %s fp32 on the context's device" % ((T, Hq),))
    need = cache.attend_bytes(ctx, Hq, T, B, cols, count, longest)
    if need:
        ctx.ensure_workspace(need)
    args = (cache.ref, qp, qt, qh, Hq, T, _ints(ctx, start, "start", (B + 1,), i32),
            _ints(ctx, request, "request", (T,), i32), _ints(ctx, position, "position", (T,), i32),
            _ints(ctx, table, "table", (B, cols), i32), B, cols, p_blocks, count, scale, longest)
    outs = out.data_ptr(), None if out_lse is None else out_lse.data_ptr()
    if cap or slopes is not None or first is not None or prefix is not None:
        if slopes is not None and slopes.requires_grad and _grad_enabled():
            raise RuntimeError("slopes require a gradient, and the cache's calls have no backward pass: detach them, or "
                               "call under torch.no_grad()")
        terms = _KvTermsStruct(cap, None if slopes is None else _ints(ctx, slopes, "slopes", (Hq,), torch.float32),
                               None if first is None else _ints(ctx, first, "first", (T,), i32),
                               None if prefix is None else _ints(ctx, prefix, "prefix", (T,), i32))
        lib, handle = ctx.bind()
        st = lib.ivf_kv_attend_terms(handle, *args, ctypes.byref(terms), *outs)
    else:
        lib, handle = ctx.bind()
        st = lib.ivf_kv_attend(handle, *args, *outs)
    if st:
        ctx.check(st, "ivf_kv_attend")
    return out, out_lse


# ---- the token that follows ---------------------------------------------------

_logit_types = None
_sample_bytes = {}  # workspace of calls of given sizes on a device


def ivf_sample(ctx: Context, logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
    """The token that follows, for each row of logits [T, V] (fp32, fp16 or bf16,
    V contiguous), drawn by uniform (fp32 [T], in [0, 1)): weights
    exp((x - max) / temperature), of which the first top_k remain (int32 [T], 0: all), of
    those the shortest part that reaches top_p (fp32 [T]), of that those of at least min_p
    (fp32 [T]) times the largest. A temperature (fp32 [T]) of 0 takes the largest logit.
    Returns (tokens int32 [T], their log-probabilities fp32 [T])."""
    import torch

    global _logit_types
    if _logit_types is None:
        _logit_types = {torch.float32: IVF_F32, torch.float16: IVF_F16, torch.bfloat16: IVF_BF16}
    dt = _logit_types.get(logits.dtype)
    if dt is None or logits.get_device() != ctx.device:
        raise TypeError("logits must be float32, float16 or bfloat16 on device %d, got %s on %s" % (
            ctx.device, logits.dtype, logits.device))
    if (logits.requires_grad or (temperature is not None and temperature.requires_grad)) and _grad_enabled():
        raise RuntimeError("logits or temperature require a gradient, and sampling has no backward pass: detach them, or call "
                           "under torch.no_grad()")
    if logits.dim() != 2 or logits.shape[1] < 1:
        raise ValueError("logits must be [T, V] with V >= 1, got %s" % (tuple(logits.shape),))
    T, V = logits.shape
    stride, one = logits.stride()
    if one != 1 and V > 1:
        raise ValueError("logits: a row must be contiguous")
    f32, shape = torch.float32, (T,)
    args = (_ints(ctx, uniform, "uniform", shape, f32),
            None if temperature is None else _ints(ctx, temperature, "temperature", shape, f32),
            None if top_k is None else _ints(ctx, top_k, "top_k", shape, torch.int32),
            None if top_p is None else _ints(ctx, top_p, "top_p", shape, f32),
            None if min_p is None else _ints(ctx, min_p, "min_p", shape, f32))
    token, logprob = torch.unsafe_split_with_sizes(torch.empty(2 * T, dtype=torch.int32, device=logits.device), (T, T))
    logprob = logprob.view(f32)
    sizes = T, V, int(top_k is not None or top_p is not None)
    need = _sample_bytes.get((ctx.device, sizes))
    if need is None:
        if len(_sample_bytes) >= 1024:
            _sample_bytes.clear()
        with torch.cuda.device(ctx.device):  # it goes by the device's compute units
            need = _sample_bytes[ctx.device, sizes] = ctx.lib.ivf_sample_bytes(*sizes)
    if need:
        ctx.ensure_workspace(need)
    lib, handle = ctx.bind()
    st = lib.ivf_sample(handle, logits.data_ptr(), dt, stride if T > 1 else 0, T, V, *args, token.data_ptr(),
                        logprob.data_ptr())
    if st:
        ctx.check(st, "ivf_sample")
    return token, logprob
