"""ctypes binding of libgba (include/gba.h): the same entry points, argument
marshalling only.  Every step of the aggregate-and-apply path runs in the
library's CUDA kernels; there is no Python or CPU fallback, and loading fails
loudly when the library has not been built.

``GBA`` is a small convenience wrapper that passes torch tensors' device
pointers; torch is only used for device memory and streams.
"""
from __future__ import annotations

import ctypes
import os
import re

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgba.so")
HEADER = os.path.join(os.path.dirname(_HERE), "include", "gba.h")

GBA_OK = 0
GBA_E_ARG = -1
GBA_E_ID_RANGE = -2
GBA_E_OOM = -3
GBA_E_CUDA = -4
GBA_E_DEVICE_TIMEOUT = -5
GBA_E_STATE = -6
GBA_E_FULL = -7
STATUS_NAMES = {0: "GBA_OK", -1: "GBA_E_ARG", -2: "GBA_E_ID_RANGE", -3: "GBA_E_OOM",
                -4: "GBA_E_CUDA", -5: "GBA_E_DEVICE_TIMEOUT", -6: "GBA_E_STATE",
                -7: "GBA_E_FULL"}
ADAGRAD, ADAM = 0, 1
DIRECT, MODULO, HASH = 0, 1, 2
F32, BF16, F16 = 0, 1, 2
NO_PAD = -2**63
INT32_MAX = 2**31 - 1
KERNEL_NAMES = ["weights", "sort_hist", "sort_pass", "seg_scan", "row_long", "row_apply",
                "dense", "init", "other"]


class GBAError(RuntimeError):
    def __init__(self, status, msg=""):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class gba_opt_desc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("lr", ctypes.c_float),
                ("adagrad_init_acc", ctypes.c_float), ("beta1", ctypes.c_float),
                ("beta2", ctypes.c_float), ("eps", ctypes.c_float)]


class gba_table_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("dim", ctypes.c_int32), ("id_mode", ctypes.c_int32),
                ("max_ids_per_msg", ctypes.c_int64), ("opt", gba_opt_desc)]


class gba_staleness_desc(ctypes.Structure):
    _fields_ = [("iota", ctypes.c_int32), ("row_staleness", ctypes.c_int32),
                ("sparse_denominator", ctypes.c_int32), ("decay", ctypes.c_int32),
                ("lambda_", ctypes.c_float), ("drop_latest", ctypes.c_int32)]


class gba_sparse_grad(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("n", ctypes.c_int64), ("rows", ctypes.c_void_p)]


class gba_stats_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "steps", "msgs_kept", "msgs_dropped", "dense_stale_sum", "dense_stale_max", "pairs",
        "pairs_dropped", "row_stale_sum", "row_stale_max", "occurrences", "rows_touched",
        "rows_applied", "occurrences_kept")]

    def as_dict(self):
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


class gba_kernel_times_t(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_int64 * len(KERNEL_NAMES)),
                ("ms", ctypes.c_double * len(KERNEL_NAMES))]


class gba_matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("stride", ctypes.c_int64),
                ("cols", ctypes.c_int32), ("type", ctypes.c_int32)]


class gba_grad_part(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("type", ctypes.c_int32), ("out_type", ctypes.c_int32)]


_P = ctypes.c_void_p
_M = ctypes.POINTER(gba_matrix)
_SIGNATURES = {
    "gba_create": (ctypes.c_int, [ctypes.POINTER(gba_table_desc), ctypes.c_int32, ctypes.c_int64,
                                  ctypes.POINTER(gba_opt_desc), ctypes.c_int64, ctypes.c_int32,
                                  ctypes.POINTER(gba_staleness_desc), ctypes.c_uint64, _P,
                                  ctypes.POINTER(_P)]),
    "gba_push": (ctypes.c_int, [_P, ctypes.c_int64, ctypes.POINTER(gba_sparse_grad), _P,
                                ctypes.c_int32]),
    "gba_push_ref": (ctypes.c_int, [_P, ctypes.c_int64, ctypes.POINTER(gba_sparse_grad), _P,
                                    ctypes.c_int32]),
    "gba_try_apply": (ctypes.c_int32, [_P]),
    "gba_pull_version": (ctypes.c_int64, [_P]),
    "gba_sync": (ctypes.c_int, [_P]),
    "gba_get_table": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.POINTER(_P), ctypes.POINTER(_P),
                                     ctypes.POINTER(_P), ctypes.POINTER(_P)]),
    "gba_get_dense": (ctypes.c_int, [_P, ctypes.POINTER(_P), ctypes.POINTER(_P),
                                     ctypes.POINTER(_P)]),
    "gba_stats": (ctypes.c_int, [_P, ctypes.POINTER(gba_stats_t)]),
    "gba_last_error": (ctypes.c_char_p, [_P]),
    "gba_destroy": (None, [_P]),
    "gba_set_timing": (ctypes.c_int, [_P, ctypes.c_int32]),
    "gba_kernel_times": (ctypes.c_int, [_P, ctypes.POINTER(gba_kernel_times_t)]),
    "gba_set_debug": (ctypes.c_int, [_P, ctypes.c_int32]),
    "gba_set_overlap": (ctypes.c_int, [_P, ctypes.c_int32]),
    "gba_join": (ctypes.c_int, [_P]),
    "gba_set_eager_dense": (ctypes.c_int, [_P, ctypes.c_int32]),
    "gba_table_capacity": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.POINTER(ctypes.c_int64)]),
    "gba_lookup_rows": (ctypes.c_int, [_P, ctypes.c_int32, _P, ctypes.c_int64, _P]),
    "gba_pull": (ctypes.c_int, [_P, ctypes.c_int32, _P, ctypes.c_int64, _P]),
    "gba_token_list_create": (ctypes.c_int, [ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(_P)]),
    "gba_fetch_token": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_int64)]),
    "gba_token_list_state": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_int64),
                                            ctypes.POINTER(ctypes.c_int64)]),
    "gba_token_list_destroy": (None, [_P]),
    "gba_debug_segments": (ctypes.c_int, [_P, ctypes.c_int64, _P, _P, _P, _P,
                                          ctypes.POINTER(ctypes.c_int64)]),
    "gba_debug_sorted": (ctypes.c_int, [_P, ctypes.c_int64, _P, _P,
                                        ctypes.POINTER(ctypes.c_int64)]),
    "gba_debug_keep": (ctypes.c_int, [_P, ctypes.c_int32, _P, ctypes.POINTER(ctypes.c_int32)]),
    "gba_debug_set_wait_limit": (ctypes.c_int, [_P, ctypes.c_int64]),
    "gba_debug_withhold_dense_copies": (ctypes.c_int, [_P, ctypes.c_int32]),
    "gba_selftest_wait_timeout": (ctypes.c_int, [ctypes.c_int64, _P]),
    "gba_version_string": (ctypes.c_char_p, []),
    "gba_device_binary_version": (ctypes.c_int32, []),
    "gba_sort_ids_static": (ctypes.c_int, [_P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32,
                                           _P, _P, _P]),
    "gba_worker_create": (ctypes.c_int, [_P, ctypes.POINTER(_P)]),
    "gba_worker_sync": (ctypes.c_int, [_P]),
    "gba_worker_last_error": (ctypes.c_char_p, [_P]),
    "gba_worker_destroy": (None, [_P]),
    "gba_embed": (ctypes.c_int, [_P, _M, ctypes.c_int32, _P, ctypes.c_int64, ctypes.c_float,
                                 ctypes.c_int64, _M]),
    "gba_embed_table": (ctypes.c_int, [_P, _P, ctypes.c_int32, _P, ctypes.c_int64, ctypes.c_float,
                                       ctypes.c_int64, _M]),
    "gba_embed_grad": (ctypes.c_int, [_P, _P, ctypes.c_int64, _M, ctypes.c_int64, ctypes.c_int32,
                                      ctypes.c_float, ctypes.c_int64, _P, _P, _P]),
    "gba_embed_grad_dense": (ctypes.c_int, [_P, _P, ctypes.c_int64, _M, ctypes.c_int32,
                                            ctypes.c_float, ctypes.c_int64, _M, ctypes.c_int32]),
    "gba_grad_norm": (ctypes.c_int, [_P, ctypes.POINTER(gba_grad_part), ctypes.c_int32, _P]),
    "gba_clip_grads": (ctypes.c_int, [_P, ctypes.POINTER(gba_grad_part), ctypes.c_int32,
                                      ctypes.c_float, _P]),
    "gba_layer_norm": (ctypes.c_int, [_P, _M, _P, _P, ctypes.c_int32, ctypes.c_float, _M, _P, _P]),
    "gba_layer_norm_grad": (ctypes.c_int, [_P, _M, _M, _P, ctypes.c_int32, _P, _P, _M, _P, _P]),
}

_lib = None


def header_functions(path: str = HEADER):
    """Names of the functions include/gba.h declares."""
    text = open(path).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(gba_[a-z_0-9]+)\s*\(", text)))


def load(path: str = LIB_PATH):
    """Load libgba.so and declare its signatures (raises if it is missing)."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"libgba.so not built: {path} (run __graft_entry__.build())")
    L = ctypes.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    if path == LIB_PATH:
        _lib = L
    return L


def check(status, h=None, what=""):
    if status < 0:
        msg = what
        if h:
            msg += " " + (load().gba_last_error(h) or b"").decode()
        raise GBAError(status, msg)
    return status


# ---- thin functional wrappers with the ABI's names ------------------------------------

def gba_create(tables, dense_size, dense_opt, global_batch, max_buffered_msgs, staleness,
               init_seed, cuda_stream=None):
    L = load()
    arr = (gba_table_desc * max(1, len(tables)))(*tables)
    h = _P()
    st = check(L.gba_create(arr, len(tables), dense_size,
                            ctypes.byref(dense_opt) if dense_opt is not None else None,
                            global_batch, max_buffered_msgs,
                            ctypes.byref(staleness) if staleness is not None else None,
                            init_seed & (2**64 - 1), cuda_stream, ctypes.byref(h)),
               what="gba_create")
    return h, st


def gba_push(h, token, per_table, dense_grad, local_batch):
    arr = (gba_sparse_grad * max(1, len(per_table)))(*per_table)
    return load().gba_push(h, token, arr, dense_grad, local_batch)


def gba_push_ref(h, token, per_table, dense_grad, local_batch):
    arr = (gba_sparse_grad * max(1, len(per_table)))(*per_table)
    return load().gba_push_ref(h, token, arr, dense_grad, local_batch)


def gba_try_apply(h):
    return load().gba_try_apply(h)


def gba_pull_version(h):
    return load().gba_pull_version(h)


def gba_sync(h):
    return load().gba_sync(h)


def gba_destroy(h):
    load().gba_destroy(h)


# ---- convenience wrapper over torch tensors --------------------------------------------

def opt_desc(kind=ADAGRAD, lr=0.01, init_acc=0.1, beta1=0.9, beta2=0.999, eps=1e-8):
    return gba_opt_desc(kind, lr, init_acc, beta1, beta2, eps)


def gba_for_workload(cfg, max_buf=None, seed=None, overlap=False, **rule):
    """A handle sized for a workload description (a `workload.WorkloadCfg`:
    tables, dense size, optimizers, global batch, tolerance iota), with room
    for max_buf buffered messages (default two global batches)."""
    def od(o):
        return opt_desc(o.kind, o.lr, o.init_acc, o.beta1, o.beta2, o.eps)
    tables = [(tb.rows, tb.dim, tb.id_mode, cfg.max_ids_per_msg(t), od(tb.opt))
              for t, tb in enumerate(cfg.tables)]
    rule = rule or dict(iota=cfg.iota)
    g = GBA(tables, cfg.D, od(cfg.dense_opt), cfg.G, max_buf or 2 * cfg.M,
            seed=cfg.seed if seed is None else seed, **rule)
    if overlap:
        g.set_overlap(True)
    return g


class GBA:
    """One parameter-server state on the current CUDA device."""

    def __init__(self, tables, dense_size, dense_opt, global_batch, max_buffered_msgs,
                 iota=INT32_MAX, row_staleness=0, sparse_denominator=0, seed=0, stream=None,
                 decay=0, lam=1.0, drop_latest=0):
        """tables: list of (rows, dim, id_mode, max_ids_per_msg, gba_opt_desc)."""
        import torch
        self.torch = torch
        self.L = load()
        self.dims = [int(t[1]) for t in tables]
        self.rows = [int(t[0]) for t in tables]
        self.opts = [t[4] for t in tables]
        self.D = int(dense_size)
        self.dense_opt = dense_opt
        descs = [gba_table_desc(int(r), int(d), int(m), int(mx), o) for (r, d, m, mx, o) in tables]
        st = gba_staleness_desc(int(iota), int(row_staleness), int(sparse_denominator),
                                int(decay), float(lam), int(drop_latest))
        if stream is None:
            stream = torch.cuda.current_stream()
        self.stream = stream
        self.h, _ = gba_create(descs, self.D, dense_opt, int(global_batch),
                               int(max_buffered_msgs), st, int(seed),
                               ctypes.c_void_p(stream.cuda_stream))
        self._keep = []  # tensors referenced by pushed-by-reference messages

    def close(self):
        if self.h:
            self.L.gba_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _grads(self, ids, rows):
        out = []
        for t in range(len(self.dims)):
            i, r = ids[t], rows[t]
            n = int(i.numel())
            out.append(gba_sparse_grad(i.data_ptr() if n else None, n,
                                       r.data_ptr() if n else None))
        return out

    def push(self, token, ids, rows, dense, local_batch):
        """Copying push; tensors may live on the device or in (pinned) host memory."""
        return check(gba_push(self.h, int(token), self._grads(ids, rows),
                              dense.data_ptr() if self.D else None, int(local_batch)),
                     self.h, "gba_push")

    def push_ref(self, token, ids, rows, dense, local_batch):
        """Push by reference (device tensors that stay valid until applied)."""
        return check(gba_push_ref(self.h, int(token), self._grads(ids, rows),
                                  dense.data_ptr() if self.D else None, int(local_batch)),
                     self.h, "gba_push_ref")

    def try_apply(self):
        return check(gba_try_apply(self.h), self.h, "gba_try_apply")

    def version(self):
        return int(gba_pull_version(self.h))

    def sync(self):
        return check(gba_sync(self.h), self.h, "gba_sync")

    def table(self, t):
        """Copies (on the device) of table t: w [rows, dim], slot0, slot1, ver."""
        w, s0, s1, v = _P(), _P(), _P(), _P()
        check(self.L.gba_get_table(self.h, t, ctypes.byref(w), ctypes.byref(s0),
                                   ctypes.byref(s1), ctypes.byref(v)), self.h)
        rows = self.capacity(t)
        n = rows * self.dims[t]
        torch = self.torch
        self.sync()
        out = []
        for p, cnt, dt in ((w, n, torch.float32), (s0, n, torch.float32), (s1, n, torch.float32),
                           (v, rows, torch.int32)):
            out.append(None if not p.value else _copy_device(p.value, cnt, dt))
        out[0] = out[0].view(rows, self.dims[t])
        out[1] = out[1].view(rows, self.dims[t])
        if out[2] is not None:
            out[2] = out[2].view(rows, self.dims[t])
        return out

    def table_rows(self, t, rows):
        """w, slot0, slot1, ver of selected rows of table t (device tensors)."""
        w, s0, s1, v = _P(), _P(), _P(), _P()
        check(self.L.gba_get_table(self.h, t, ctypes.byref(w), ctypes.byref(s0),
                                   ctypes.byref(s1), ctypes.byref(v)), self.h)
        self.sync()
        torch = self.torch
        d = self.dims[t]
        cap = self.capacity(t)
        idx = torch.as_tensor(rows, dtype=torch.int64, device="cuda")
        res = []
        for p in (w, s0, s1):
            if not p.value:
                res.append(None)
                continue
            res.append(_gather_rows(p.value, cap, d, idx))
        res.append(_gather_rows(v.value, cap, 1, idx, torch.int32).view(-1))
        return res

    def dense(self):
        w, s0, s1 = _P(), _P(), _P()
        check(self.L.gba_get_dense(self.h, ctypes.byref(w), ctypes.byref(s0), ctypes.byref(s1)),
              self.h)
        self.sync()
        torch = self.torch
        return [None if not p.value else _copy_device(p.value, self.D, torch.float32)
                for p in (w, s0, s1)]

    def stats(self):
        s = gba_stats_t()
        check(self.L.gba_stats(self.h, ctypes.byref(s)), self.h)
        return s.as_dict()

    def pull(self, t, ids):
        """Current rows of table t for the device int64 tensor ids (pull responding)."""
        torch = self.torch
        ids = ids.contiguous()
        out = torch.empty(ids.numel(), self.dims[t], dtype=torch.float32, device=ids.device)
        check(self.L.gba_pull(self.h, int(t), ids.data_ptr() if ids.numel() else None,
                              ids.numel(), out.data_ptr() if ids.numel() else None),
              self.h, "gba_pull")
        return out

    def capacity(self, t):
        """Rows the arrays of table t hold now (slots of a HASH table)."""
        r = ctypes.c_int64()
        check(self.L.gba_table_capacity(self.h, int(t), ctypes.byref(r)), self.h)
        return int(r.value)

    def lookup(self, t, ids):
        """Slots of the device int64 tensor ids in HASH table t (-1: absent)."""
        torch = self.torch
        ids = ids.contiguous()
        out = torch.empty(ids.numel(), dtype=torch.int64, device=ids.device)
        if ids.numel():
            check(self.L.gba_lookup_rows(self.h, int(t), ids.data_ptr(), ids.numel(),
                                         out.data_ptr()), self.h, "gba_lookup_rows")
        return out

    def set_eager_dense(self, on=True):
        check(self.L.gba_set_eager_dense(self.h, int(on)), self.h, "gba_set_eager_dense")

    def join(self):
        """Order the handle's stream after every step enqueued so far."""
        check(self.L.gba_join(self.h), self.h, "gba_join")

    def set_overlap(self, on=True):
        check(self.L.gba_set_overlap(self.h, int(on)), self.h)

    def set_debug(self, on=True):
        check(self.L.gba_set_debug(self.h, int(on)), self.h)

    def set_timing(self, on=True):
        check(self.L.gba_set_timing(self.h, int(on)), self.h)

    def kernel_times(self):
        kt = gba_kernel_times_t()
        check(self.L.gba_kernel_times(self.h, ctypes.byref(kt)), self.h)
        return {KERNEL_NAMES[i]: (int(kt.launches[i]), float(kt.ms[i])) for i in range(len(KERNEL_NAMES))}

    def set_wait_limit(self, ns):
        check(self.L.gba_debug_set_wait_limit(self.h, int(ns)), self.h)

    def withhold_dense_copies(self, on=True):
        check(self.L.gba_debug_withhold_dense_copies(self.h, 1 if on else 0), self.h)

    def segments(self, cap=None):
        """Dedup output of the last step: (table, row, count, kept) numpy arrays."""
        import numpy as np
        n = ctypes.c_int64()
        if cap is None:
            self.L.gba_debug_segments(self.h, 0, None, None, None, None, ctypes.byref(n))
            cap = int(n.value)
        t = np.zeros(cap, np.int32)
        r = np.zeros(cap, np.int64)
        c = np.zeros(cap, np.int64)
        k = np.zeros(cap, np.int64)
        check(self.L.gba_debug_segments(self.h, cap, t.ctypes.data, r.ctypes.data, c.ctypes.data,
                                        k.ctypes.data, ctypes.byref(n)), self.h)
        u = int(n.value)
        return t[:u], r[:u], c[:u], k[:u]

    def sorted_keys(self):
        import numpy as np
        n = ctypes.c_int64()
        self.L.gba_debug_sorted(self.h, 0, None, None, ctypes.byref(n))
        cap = int(n.value)
        keys = np.zeros(cap, np.uint32)
        occ = np.zeros(cap, np.uint32)
        check(self.L.gba_debug_sorted(self.h, cap, keys.ctypes.data, occ.ctypes.data,
                                      ctypes.byref(n)), self.h)
        return keys, occ

    def keep(self, cap=4096):
        import numpy as np
        out = np.zeros(cap, np.int32)
        M = ctypes.c_int32()
        check(self.L.gba_debug_keep(self.h, cap, out.ctypes.data, ctypes.byref(M)), self.h)
        return out[:M.value]


class _DevArray:
    """Minimal __cuda_array_interface__ over library-owned device memory."""

    def __init__(self, ptr, nbytes):
        self.__cuda_array_interface__ = {"shape": (nbytes,), "typestr": "|u1",
                                         "data": (ptr, False), "version": 3}


def _copy_device(ptr, n, dtype):
    import torch
    elem = torch.empty((), dtype=dtype).element_size()
    raw = torch.as_tensor(_DevArray(ptr, n * elem), device="cuda")
    return raw.view(dtype).clone()


def _gather_rows(ptr, rows, d, idx, dtype=None):
    import torch
    dtype = dtype or torch.float32
    elem = torch.empty((), dtype=dtype).element_size()
    raw = torch.as_tensor(_DevArray(ptr, rows * d * elem), device="cuda").view(dtype)
    return raw.view(rows, d).index_select(0, idx).clone()


class TokenList:
    """The token list of Sec. 4.1 / Alg. 2 (see gba_token_list_create)."""

    def __init__(self, repeats, workers):
        self.L = load()
        self.h = _P()
        check(self.L.gba_token_list_create(int(repeats), int(workers), ctypes.byref(self.h)),
              what="gba_token_list_create")

    def fetch(self):
        t = ctypes.c_int64()
        check(self.L.gba_fetch_token(self.h, ctypes.byref(t)), what="gba_fetch_token")
        return int(t.value)

    def state(self):
        q, f = ctypes.c_int64(), ctypes.c_int64()
        check(self.L.gba_token_list_state(self.h, ctypes.byref(q), ctypes.byref(f)))
        return int(q.value), int(f.value)

    def close(self):
        if self.h:
            self.L.gba_token_list_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- a worker's operators -----------------------------------------------------------------

def _refuse(why):
    raise GBAError(GBA_E_ARG, why)


_types = {}  # torch dtype -> gba_dtype


def _type_of(t):
    if not _types:
        import torch
        _types.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    try:
        return _types[t.dtype]
    except KeyError:
        _refuse(f"tensors are float32, bfloat16 or float16, not {t.dtype}")


def _matrix(t):
    """t as a gba_matrix: two dimensions, rows of consecutive elements."""
    shape, strides = t.shape, t.stride()
    if len(shape) != 2 or (strides[1] != 1 and shape[1] > 1):
        _refuse("a matrix has two dimensions, and rows of consecutive elements")
    rows, cols = shape
    if cols > INT32_MAX:
        _refuse("a matrix has too many columns")
    return gba_matrix(t.data_ptr() if rows else None, rows, strides[0] if rows > 1 else max(cols, 1), cols,
                      _type_of(t))


# ctypes keeps an integer's low bits, so what does not fit is refused before it.
def _int64(x):
    if not -2**63 <= x < 2**63:
        _refuse(f"{x} is no 64-bit integer")
    return x


def _pad(pad_id):
    return NO_PAD if pad_id is None else _int64(pad_id)


def _mode(id_mode):
    if id_mode != DIRECT and id_mode != MODULO:
        _refuse("id_mode is neither DIRECT nor MODULO")
    return id_mode


def _rows_of(t):
    """An input of any leading shape as a matrix [n, d]; copied if its rows are not apart or
    their elements not consecutive (an expanded tensor, a transposed one)."""
    if t.dim() != 2:
        t = t.reshape(t.numel() // max(1, t.shape[-1]), t.shape[-1])
    (rows, cols), strides = t.shape, t.stride()
    if (cols > 1 and strides[1] != 1) or (rows > 1 and strides[0] < cols):
        t = t.contiguous()
    return t


class GradParts:
    """A list of gradient tensors (and of what receives them clipped), as the library takes
    it.  It holds the tensors and the addresses that they had when it was made: gradients that
    are made anew (set to None between steps) or given other storage need a new list.  Making one
    costs about 1.2 us a tensor of Python, so it pays to keep it for gradients that stay."""

    def __init__(self, grads, out=None):
        grads = list(grads)
        out = grads if out is None else list(out)
        if len(out) != len(grads):
            _refuse("as many outputs as gradients")
        self.device = (grads[0].get_device() if grads else None)  # checked against the worker's
        for t in (*grads, *out):
            if t.get_device() != self.device or self.device < 0:
                _refuse("gradients and their outputs are on one GPU")
            if not t.is_contiguous():
                _refuse("gradients and their outputs are contiguous")
        for g, o in zip(grads, out):
            if g.numel() != o.numel():
                _refuse("an output has its gradient's size")
        self.tensors = (grads, out)
        self.n = len(grads)
        self.array = (gba_grad_part * max(1, self.n))(*[
            gba_grad_part(g.data_ptr(), o.data_ptr(), g.numel(), _type_of(g), _type_of(o))
            for g, o in zip(grads, out)])


def grad_parts(grads, out=None):
    """The list of a program's gradient tensors, made once for tensors that stay.  out: what
    clipping writes to (default: in place)."""
    return GradParts(grads, out)


class Worker:
    """A worker's operators on one CUDA device: lookups and their gradient, norm and clipping,
    layer norm (see include/gba.h).

    Work is issued on `stream` (default: the current one), on the stream's device.  A call made while another stream
    is current orders the two both ways, so tensors of the current stream can be passed and
    results used there.

    The operators work on the tensors' data: nothing is recorded for autograd, results never
    require gradients, and what is written in place (out, clipped gradients) does not count as a
    change of the tensor there.  Tensors are on the worker's device."""

    def __init__(self, stream=None):
        import torch
        self.torch = torch
        self.L = load()
        self.h = None
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self._raw_stream = self.stream.cuda_stream
        self._device = self.stream.device
        self._index = self._device.index
        h = _P()
        with torch.cuda.device(self._device):
            check(self.L.gba_worker_create(self._raw_stream, ctypes.byref(h)), what="gba_worker_create")
        self.h = h

    def close(self):
        if self.h:
            self.L.gba_worker_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _call(self, name, *args):
        call = getattr(self.L, name)
        if self.torch._C._cuda_getCurrentRawStream(self._index) == self._raw_stream:
            status = call(self.h, *args)
        else:
            now = self.torch.cuda.current_stream(self._device)
            self.stream.wait_stream(now)
            status = call(self.h, *args)
            now.wait_stream(self.stream)
        if status < 0:
            self._check(status, name)

    def _mine(self, *tensors):
        for t in tensors:
            if t is not None and t.get_device() != self._index:
                _refuse("a tensor is not on the worker's GPU")

    def _parts(self, grads):
        p = grads if isinstance(grads, GradParts) else GradParts(grads)
        if p.n and p.device != self._index:
            _refuse("a tensor is not on the worker's GPU")
        return p

    def _new(self, *shape, dtype=None):
        return self.torch.empty(shape, dtype=dtype or self.torch.float32, device=self._device)

    def _check(self, status, name):
        if status < 0:
            raise GBAError(status, name + " " + (self.L.gba_worker_last_error(self.h) or b"").decode())

    def sync(self):
        """Wait for the worker's stream; raises what its kernels reported since the last time."""
        self._check(self.L.gba_worker_sync(self.h), "gba_worker_sync")

    def _ids(self, ids):
        if ids.dtype != self.torch.int64:
            _refuse("ids are int64")
        self._mine(ids)
        return ids.contiguous()

    def _embed_out(self, ids, d, dtype, out):
        if out is None:
            out = self._new(*ids.shape, d, dtype=dtype)
        self._mine(out)
        flat = out if out.dim() == 2 else out.view(ids.numel(), d)
        return out, _matrix(flat)

    def embed(self, weights, ids, scale=1.0, pad_id=None, dtype=None, id_mode=DIRECT, out=None):
        """scale * weights[ids] in dtype (default: the weights'), or into out, in out's type; padding
        gives zeros."""
        ids = self._ids(ids)
        self._mine(weights)
        out, om = self._embed_out(ids, weights.shape[-1], dtype or weights.dtype, out)
        self._call("gba_embed", _matrix(weights), _mode(id_mode), ids.data_ptr(), ids.numel(), scale,
                   _pad(pad_id), om)
        return out

    def embed_table(self, server, t, ids, scale=1.0, pad_id=None, dtype=None, out=None):
        """The same from table t of a server (a GBA), as of every step applied so far."""
        if not 0 <= t < len(server.dims):
            _refuse("no such table")
        ids = self._ids(ids)
        out, om = self._embed_out(ids, server.dims[t], dtype or self.torch.float32, out)
        self._call("gba_embed_table", server.h, t, ids.data_ptr(), ids.numel(), scale,
                   _pad(pad_id), om)
        return out

    def embed_grad(self, ids, grad, rows, scale=1.0, pad_id=None, id_mode=DIRECT):
        """The lookup's gradient as one message's ids and rows: (ids [n], rows [n, d] float32,
        count).  The first `count` (a device int64) entries are the distinct rows in ascending
        order; those after repeat the last one's id with zeros."""
        torch = self.torch
        ids, grad = self._ids(ids), _rows_of(grad)
        self._mine(grad)
        n, d = ids.numel(), grad.shape[1]
        ids_out = self._new(n, dtype=torch.int64)
        rows_out = self._new(n, d)
        count = self._new(dtype=torch.int64)
        self._call("gba_embed_grad", ids.data_ptr(), n, _matrix(grad), _int64(rows), _mode(id_mode), scale,
                   _pad(pad_id), ids_out.data_ptr(), rows_out.data_ptr(),
                   count.data_ptr())
        return ids_out, rows_out, count

    def embed_grad_dense(self, ids, grad, out, scale=1.0, pad_id=None, id_mode=DIRECT, accumulate=False):
        """The lookup's gradient over all rows of the table, into (or added to) out."""
        ids, grad = self._ids(ids), _rows_of(grad)
        self._mine(grad, out)
        self._call("gba_embed_grad_dense", ids.data_ptr(), ids.numel(), _matrix(grad), _mode(id_mode), scale,
                   _pad(pad_id), _matrix(out), int(accumulate))
        return out

    def grad_norm(self, grads):
        """The 2-norm of all the tensors together (a list, or grad_parts of it), on the device."""
        p = self._parts(grads)
        norm = self._new()
        self._call("gba_grad_norm", p.array, p.n, norm.data_ptr())
        return norm

    def clip_grads(self, grads, max_norm):
        """Scales the tensors (a list, or grad_parts of it) by min(1, max_norm / (norm + 1e-6)),
        in place or into the parts' outputs; returns the norm."""
        p = self._parts(grads)
        norm = self._new()
        self._call("gba_clip_grads", p.array, p.n, max_norm, norm.data_ptr())
        return norm

    def _params(self, d, *params):
        at, kind = [], None
        for p in params:
            if p is None:
                at.append(None)
                continue
            self._mine(p)
            if p.numel() != d or not p.is_contiguous():
                _refuse("a parameter has a value per column")
            if kind is not None and kind != _type_of(p):
                _refuse("the parameters of a layer norm have one type")
            kind = _type_of(p)
            at.append(p.data_ptr())
        return at, F32 if kind is None else kind

    def layer_norm(self, x, gamma=None, beta=None, eps=1e-5):
        """(y, mean, rstd) of the rows of x (its last dimension)."""
        self._mine(x)
        rows = _rows_of(x)
        n, d = rows.shape
        y = self._new(n, d, dtype=x.dtype)
        mean, rstd = self._new(n), self._new(n)
        (pg, pb), ptype = self._params(d, gamma, beta)
        self._call("gba_layer_norm", _matrix(rows), pg, pb, ptype, eps, _matrix(y), mean.data_ptr(),
                   rstd.data_ptr())
        return y if x.dim() == 2 else y.view(x.shape), mean, rstd

    def layer_norm_grad(self, dy, x, gamma, mean, rstd):
        """(dx, dgamma, dbeta) from the gradient of layer_norm's y and its mean and rstd."""
        torch = self.torch
        self._mine(dy, x, mean, rstd)
        xr, dr = _rows_of(x), _rows_of(dy)
        n, d = xr.shape
        if mean.numel() != n or rstd.numel() != n or {mean.dtype, rstd.dtype} != {torch.float32}:
            _refuse("mean and rstd are float32, one for each row")
        mean, rstd = mean.contiguous(), rstd.contiguous()
        dx = self._new(n, d, dtype=x.dtype)
        dgamma, dbeta = self._new(d), self._new(d)
        (pg,), ptype = self._params(d, gamma)
        self._call("gba_layer_norm_grad", _matrix(dr), _matrix(xr), pg, ptype, mean.data_ptr(),
                   rstd.data_ptr(), _matrix(dx), dgamma.data_ptr(), dbeta.data_ptr())
        return dx if x.dim() == 2 else dx.view(x.shape), dgamma, dbeta
