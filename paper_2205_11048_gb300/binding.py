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
NORMS = {"none": 0, "rms": 1, "layer": 2}
GATES = {"none": 0, "mul": 1, "sigmoid": 2, "silu": 3}
DECAYS = {"sigmoid": 0, "log": 1}
ROUNDINGS = {"nearest": 0, "chance": 1}
NO_PAD = -2**63
INT32_MAX = 2**31 - 1
LEGACY_STREAM = 1  # cudaStreamLegacy: the default stream by a name that is not NULL
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


class gba_block(ctypes.Structure):
    _fields_ = [("post_norm", ctypes.c_int32), ("pre_norm", ctypes.c_int32), ("gate", ctypes.c_int32),
                ("param_type", ctypes.c_int32), ("post_weight", ctypes.c_void_p), ("post_bias", ctypes.c_void_p),
                ("pre_weight", ctypes.c_void_p), ("pre_bias", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("residual_scale", ctypes.c_float), ("block_scale", ctypes.c_float)]


class gba_block_grads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("post_weight", "post_bias", "pre_weight", "pre_bias")]


class gba_scan(ctypes.Structure):
    _fields_ = [("decay", ctypes.c_int32), ("tied", ctypes.c_int32), ("n_seq", ctypes.c_int64),
                ("lengths", ctypes.c_void_p), ("offsets", ctypes.c_void_p)]


class gba_adamw_part(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("weight", "grad", "m", "v", "m_scale", "v_scale", "copy")] + [
        ("n", ctypes.c_int64), ("type", ctypes.c_int32), ("grad_type", ctypes.c_int32),
        ("copy_type", ctypes.c_int32), ("bits", ctypes.c_int32), ("weight_decay", ctypes.c_float)]


class gba_adamw_desc(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("lr_now", ctypes.c_void_p), ("norm", ctypes.c_void_p),
                ("max_norm", ctypes.c_float), ("rounding", ctypes.c_int32)]


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
    "gba_residual_norm": (ctypes.c_int, [_P, ctypes.POINTER(gba_block), _M, _M, _M, _M, _M, _P]),
    "gba_residual_norm_grad": (ctypes.c_int, [_P, ctypes.POINTER(gba_block), _M, _M, _M, _M, _M, _P, _M, _M, _M,
                                              ctypes.POINTER(gba_block_grads)]),
    "gba_gated_scan": (ctypes.c_int, [_P, ctypes.POINTER(gba_scan), _M, _M, _M, _M, _M]),
    "gba_gated_scan_grad": (ctypes.c_int, [_P, ctypes.POINTER(gba_scan)] + [_M] * 9),
    "gba_adamw": (ctypes.c_int, [_P, ctypes.POINTER(gba_adamw_part), ctypes.c_int32,
                                 ctypes.POINTER(gba_adamw_desc), _P]),
    "gba_adamw_values": (ctypes.c_int, [_P, ctypes.POINTER(gba_adamw_part), ctypes.c_int32, ctypes.POINTER(_P),
                                        ctypes.POINTER(_P)]),
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
    """One parameter-server state on the current CUDA device.  Its work is issued on `stream`
    (default: the current one, the default stream too), so tensors of that stream can be passed,
    and results read, without waiting."""

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
                               ctypes.c_void_p(stream.cuda_stream or LEGACY_STREAM))  # NULL: a stream of its own
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


def _opt(t):
    return None if t is None else _matrix(t)


def _shaped(t, like):
    return t if t is None or t.shape == like.shape else t.view(like.shape)


def _addresses(tensors):
    return (ctypes.c_void_p * max(1, len(tensors)))(*[t.data_ptr() for t in tensors])


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


class ResidualNorm:
    """The parameters of Worker.residual_norm: what it normalises and how, and the tensors of its
    weights and biases (of one type; held, and read where they are when a call runs)."""

    def __init__(self, post_norm="none", pre_norm="none", gate="none", post_weight=None, post_bias=None,
                 pre_weight=None, pre_bias=None, eps=1e-6, residual_scale=1.0, block_scale=1.0):
        try:
            kinds = NORMS[post_norm], NORMS[pre_norm], GATES[gate]
        except (KeyError, TypeError):
            _refuse(f"norms are one of {list(NORMS)}, gates one of {list(GATES)}")
        self.tensors = (post_weight, post_bias, pre_weight, pre_bias)
        there = [p for p in self.tensors if p is not None]
        if pre_norm == "none" and (pre_weight is not None or pre_bias is not None):
            _refuse("parameters of a norm that is not taken")
        for p in there:
            if not p.is_contiguous() or p.numel() != there[0].numel() or _type_of(p) != _type_of(there[0]):
                _refuse("the parameters of a block have a value per column and one type")
            if p.get_device() != there[0].get_device():
                _refuse("the parameters of a block are on one GPU")
        self.pre, self.gate = pre_norm != "none", gate != "none"
        self.cols = there[0].numel() if there else None
        self.device = there[0].get_device() if there else None
        self.block = gba_block(*kinds, _type_of(there[0]) if there else F32,
                               *[None if p is None else p.data_ptr() for p in self.tensors], eps, residual_scale,
                               block_scale)


def residual_norm(**how):
    """A block's norms, gate and residual, made once (see ResidualNorm)."""
    return ResidualNorm(**how)


class Sequences:
    """Where n sequences lie among the rows of a scan: of equal length, one after another; with
    lengths (an int64 tensor of n), the first lengths[i] rows of each of those; with offsets (of
    n + 1), sequence i has the rows offsets[i] up to offsets[i + 1]."""

    def __init__(self, n, lengths=None, offsets=None):
        if not 0 <= n < 2**29:
            _refuse("from 0 to 2^29 - 1 sequences")
        if lengths is not None and offsets is not None:
            _refuse("lengths and offsets")
        for t, many in ((lengths, n), (offsets, n + 1)):
            if t is not None and (str(t.dtype) != "torch.int64" or t.numel() != many or not t.is_contiguous()):
                _refuse("lengths are n and offsets n + 1 int64")
        self.n, self.lengths, self.offsets = n, lengths, offsets


def sequences(n, lengths=None, offsets=None):
    """The sequences of a scan, made once (see Sequences)."""
    return Sequences(n, lengths, offsets)


class AdamWStates:
    """AdamW's states of a list of weights, which it holds: m and v (lists of float32 tensors, or
    of uint8 with 8 bits and their m_scale and v_scale), step (a device int64) and, if given,
    copies of the weights that follow them.  States that are not given start as zeros.  With 8
    bits and rounding "nearest" a state does not follow changes of a few per cent a step, so
    where a weight's gradient gets small beside those of its 256 neighbours its second moment
    stays large; with "chance" states are right on average (see gba_rounding in include/gba.h)."""

    def __init__(self, weights, bits=32, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, copies=None, m=None, v=None,
                 m_scale=None, v_scale=None, step=None, rounding="nearest"):
        import torch
        self.weights = list(weights)
        if bits not in (32, 8):
            _refuse("states have 32 or 8 bits")
        if rounding not in ROUNDINGS or (bits == 32 and rounding != "nearest"):
            _refuse(f"roundings of states in 8 bits are one of {list(ROUNDINGS)}")
        self.rounding = rounding
        self.bits, self.betas, self.eps = bits, (float(betas[0]), float(betas[1])), float(eps)
        n = len(self.weights)
        self.device = self.weights[0].get_device() if n else None
        self.decays = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else list(weight_decay)
        where = self.weights[0].device if n else "cuda"

        def states(given, kind, size):
            if given is None:
                return [torch.zeros(size(w.numel()), dtype=kind, device=where) for w in self.weights]
            given = list(given)
            if len(given) != n or any(t.dtype != kind or t.numel() != size(w.numel())
                                      for t, w in zip(given, self.weights)):
                _refuse("a state has its weight's size, and its own type")
            return given

        def scales(k):
            return (k + 255) // 256

        def same(k):
            return k

        kind = torch.float32 if bits == 32 else torch.uint8
        if bits == 8 and ((m is None) != (m_scale is None) or (v is None) != (v_scale is None)):
            _refuse("8-bit states come with their scales")
        if bits == 32 and (m_scale is not None or v_scale is not None):
            _refuse("scales of states in 32 bits")
        self.m, self.v = states(m, kind, same), states(v, kind, same)
        self.m_scale = states(m_scale, torch.float32, scales) if bits == 8 else None
        self.v_scale = states(v_scale, torch.float32, scales) if bits == 8 else None
        self.copies = None if copies is None else list(copies)
        if len(self.decays) != n or (self.copies is not None and len(self.copies) != n):
            _refuse("a weight decay and a copy for each weight")
        if self.copies is not None and any(c.numel() != w.numel() for c, w in zip(self.copies, self.weights)):
            _refuse("a copy has its weight's size")
        self.step = torch.zeros((), dtype=torch.int64, device=where) if step is None else step
        if self.step.dtype != torch.int64 or self.step.numel() != 1:
            _refuse("step is one int64")
        for t in (*self.weights, *self.m, *self.v, *(self.m_scale or ()), *(self.v_scale or ()), *(self.copies or ()),
                  self.step):
            if t.get_device() < 0 or (n and t.get_device() != self.device):
                _refuse("weights, states and step are on one GPU")
            if not t.is_contiguous():
                _refuse("weights and states are contiguous")
        at = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size())
                    for ts in (self.weights, self.m, self.v, self.m_scale, self.v_scale, self.copies, [self.step])
                    for t in ts or () if t.numel())
        if any(b[0] < a[1] for a, b in zip(at, at[1:])):
            _refuse("weights, states, copies or step overlap (a shared weight is listed once)")

    def parts(self, grads):
        """The list of weights with their gradients, made once for gradients that stay."""
        return AdamWParts(self, grads)


class AdamWParts:
    """What Worker.adamw takes: states and gradients, by their addresses when it was made."""

    def __init__(self, states, grads):
        grads = list(grads)
        if len(grads) != len(states.weights):
            _refuse("as many gradients as weights")
        for g, w in zip(grads, states.weights):
            if g.get_device() != states.device or not g.is_contiguous() or g.numel() != w.numel():
                _refuse("a gradient is contiguous, of its weight's size and on its GPU")
        self.states, self.grads, self.n = states, grads, len(grads)
        self.device = states.step.get_device()

        def at(ts, i):
            return None if ts is None else ts[i].data_ptr()

        self.array = (gba_adamw_part * max(1, self.n))(*[
            gba_adamw_part(w.data_ptr(), g.data_ptr(), at(states.m, i), at(states.v, i), at(states.m_scale, i),
                           at(states.v_scale, i), at(states.copies, i), w.numel(), _type_of(w), _type_of(g),
                           F32 if states.copies is None else _type_of(states.copies[i]), states.bits,
                           states.decays[i])
            for i, (w, g) in enumerate(zip(states.weights, grads))])


def adamw_states(weights, **how):
    """AdamW's states of a list of weights (see AdamWStates)."""
    return AdamWStates(weights, **how)


class Worker:
    """A worker's operators on one CUDA device: lookups and their gradient, norm and clipping,
    layer norm, and those of a block: norms with a gate and the residual, gated scans, AdamW (see
    include/gba.h).

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

    def _block(self, block, x, *others):
        """Rows of x and of the others (None stays None), checked against the block and the worker."""
        if not isinstance(block, ResidualNorm):
            _refuse("a block is made by residual_norm()")
        if block.device is not None and block.device != self._index:
            _refuse("a parameter is not on the worker's GPU")
        self._mine(x, *others)
        if block.cols is not None and block.cols != x.shape[-1]:
            _refuse("a parameter has a value per column")
        for t in others:
            if t is not None and t.shape != x.shape:
                _refuse("tensors of different shapes")
        return [None if t is None else _rows_of(t) for t in (x, *others)]

    def residual_norm(self, block, x, residual=None, gate=None, keep_sum=True, sum_out=None, sum_dtype=None):
        """(y, z, stats): z = residual_scale * residual + block_scale * act(gate) * post_norm(x) and
        y = pre_norm(z), with the parameters of block (None where its pre_norm is none).  z goes to
        sum_out (the residual itself, say); keep_sum=False: it is not kept.  Without a residual z
        has the type sum_dtype (default: x's), else the residual's."""
        rows, res, g, so = self._block(block, x, residual, gate, sum_out)
        if so is not None and (so.data_ptr() != sum_out.data_ptr() or not keep_sum):
            _refuse("sum_out has rows of consecutive elements, and is kept")
        n, d = rows.shape
        y = self._new(n, d, dtype=x.dtype) if block.pre else None
        z = so
        if z is None and keep_sum:
            z = self._new(n, d, dtype=residual.dtype if residual is not None else sum_dtype or x.dtype)
        stats = self._new(n, 4)
        self._call("gba_residual_norm", block.block, _matrix(rows), _opt(res), _opt(g), _opt(z), _opt(y),
                   stats.data_ptr())
        return (_shaped(y, x), sum_out if sum_out is not None else _shaped(z, x), stats)

    def residual_norm_grad(self, block, dy, dz, x, z, stats, gate=None, residual=True):
        """The gradients of residual_norm's inputs and parameters, from those of y and z (dy None
        where block has no pre_norm, dz None for none) and what it took and gave: a dict of dx,
        dresidual (unless residual is False), dgate and dpost_weight, dpost_bias, dpre_weight and
        dpre_bias, each if what it belongs to is there."""
        if not block.pre:
            z = None
        if z is None and dz is None:
            _refuse("neither dy nor dz")
        xr, dyr, dzr, zr, g = self._block(block, x, dy, dz, z, gate)
        self._mine(stats)
        n, d = xr.shape
        if stats.dtype != self.torch.float32 or stats.numel() != 4 * n or not stats.is_contiguous():
            _refuse("stats are those of residual_norm")
        wide = (z if z is not None else dz).dtype
        out = {"dx": self._new(n, d, dtype=x.dtype)}
        if residual:
            out["dresidual"] = self._new(n, d, dtype=wide)
        if gate is not None:
            out["dgate"] = self._new(n, d, dtype=x.dtype)
        sums = gba_block_grads()
        for name, p in zip(("post_weight", "post_bias", "pre_weight", "pre_bias"), block.tensors):
            if p is not None:
                out["d" + name] = t = self._new(d)
                setattr(sums, name, t.data_ptr())
        self._call("gba_residual_norm_grad", block.block, _opt(dyr), _opt(dzr), _matrix(xr), _opt(zr), _opt(g),
                   stats.data_ptr(), _matrix(out["dx"]), _opt(out.get("dresidual")), _opt(out.get("dgate")), sums)
        for k in ("dx", "dresidual", "dgate"):
            if k in out:
                out[k] = _shaped(out[k], x)
        return out

    def _scan(self, seq, decay, tied, x, *others):
        if not isinstance(seq, Sequences):
            _refuse("sequences are made by sequences()")
        if decay not in DECAYS:
            _refuse(f"decays are one of {list(DECAYS)}")
        self._mine(x, seq.lengths, seq.offsets, *others)
        for t in others:
            if t is not None and t.shape != x.shape:
                _refuse("tensors of different shapes")
        desc = gba_scan(DECAYS[decay], int(bool(tied)), seq.n,
                        None if seq.lengths is None else seq.lengths.data_ptr(),
                        None if seq.offsets is None else seq.offsets.data_ptr())
        return desc, [_rows_of(t) for t in (x, *others)]

    def _state(self, t, seq, d):
        if t is None:
            return None
        self._mine(t)
        t = t if t.dim() == 2 else t.view(seq.n, d)
        if tuple(t.shape) != (seq.n, d) or t.dtype != self.torch.float32:
            _refuse("states are float32, a row for each sequence")
        return t

    def gated_scan(self, x, f, seq, decay="sigmoid", tied=True, state=None, state_out=None, dtype=None):
        """(y, last): y = h with h = a h + (1 - a) x (a h + x unless tied) along the sequences of
        the rows of x, from state (default zeros); a = sigmoid(f), or exp(min(f, 0)) with decay
        "log".  last: h after each sequence's last row, into state_out if given (state itself, for
        steps in place).  dtype: of y (x's or float32)."""
        desc, (xr, fr) = self._scan(seq, decay, tied, x, f)
        n, d = xr.shape
        st, so = self._state(state, seq, d), self._state(state_out, seq, d)
        if so is None:
            so = self._new(seq.n, d)
        y = self._new(n, d, dtype=dtype or x.dtype)
        self._call("gba_gated_scan", desc, _matrix(xr), _matrix(fr), _opt(st), _matrix(y), _matrix(so))
        return _shaped(y, x), state_out if state_out is not None else so

    def gated_scan_grad(self, dy, x, f, y, seq, decay="sigmoid", tied=True, state=None, dstate=None):
        """(dx, df, dstate) from the gradients of gated_scan's y and (dstate, default none) of its
        last states; the last is None without a state."""
        desc, (xr, fr, yr, dr) = self._scan(seq, decay, tied, x, f, y, dy)
        n, d = xr.shape
        st, ds = self._state(state, seq, d), self._state(dstate, seq, d)
        dx, df = self._new(n, d, dtype=x.dtype), self._new(n, d, dtype=x.dtype)
        out = None if st is None else self._new(seq.n, d)
        self._call("gba_gated_scan_grad", desc, _matrix(dr), _opt(ds), _matrix(xr), _matrix(fr), _opt(st),
                   _matrix(yr), _matrix(dx), _matrix(df), _opt(out))
        return _shaped(dx, x), _shaped(df, x), out

    def _adamw(self, parts):
        if not isinstance(parts, AdamWParts):
            _refuse("parts are made by AdamWStates.parts()")
        if parts.device != self._index:
            _refuse("a tensor is not on the worker's GPU")
        return parts.states

    def adamw(self, parts, lr, norm=None, max_norm=None):
        """One step of AdamW over the weights of parts (AdamWStates.parts of their gradients), in
        place.  lr: a number, or a device float32 that is read when the call runs.  norm (a device
        float32, of grad_norm say) and max_norm clip the gradients on the way; with a norm that is
        infinite or NaN nothing changes."""
        st, torch = self._adamw(parts), self.torch
        if (norm is None) != (max_norm is None):
            _refuse("norm and max_norm go together")
        now = lr if hasattr(lr, "data_ptr") else None
        for t in (now, norm):
            if t is not None and (t.dtype != torch.float32 or t.numel() != 1):
                _refuse("lr and norm are one float32")
        self._mine(now, norm)
        desc = gba_adamw_desc(0.0 if now is not None else lr, *st.betas, st.eps,
                              None if now is None else now.data_ptr(), None if norm is None else norm.data_ptr(),
                              0.0 if max_norm is None else max_norm, ROUNDINGS[st.rounding])
        self._call("gba_adamw", parts.array, parts.n, desc, st.step.data_ptr())

    def adamw_values(self, parts, m_out=None, v_out=None):
        """The states of parts as float32: (list of m, list of v), into the given lists of tensors."""
        st = self._adamw(parts)
        m_out, v_out = [[self._new(w.numel()) for w in st.weights] if o is None else list(o) for o in (m_out, v_out)]
        for o in (m_out, v_out):
            if len(o) != parts.n:
                _refuse("as many outputs as weights")
            self._mine(*o)
            for t, w in zip(o, st.weights):
                if t.numel() != w.numel() or t.dtype != self.torch.float32 or not t.is_contiguous():
                    _refuse("an output is float32, contiguous and of its weight's size")
        self._call("gba_adamw_values", parts.array, parts.n, _addresses(m_out), _addresses(v_out))
        return m_out, v_out
