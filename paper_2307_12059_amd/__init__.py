"""Python binding of the kgc C ABI (include/kgc.h): argument marshalling only.

Every step of the join runs in the HIP library ``libkgc.so`` built from
``csrc/``; PyTorch is used for device memory and the stream.  There is no CPU
fallback: importing works without a GPU (so the exported symbols can be
checked), but any compute call fails loudly if the library or a device is
missing.

Names follow the C ABI: ``kgc_create``, ``kgc_join``, ``kgc_norms``,
``kgc_get_stats``, ``kgc_last_error``, ``kgc_destroy``, ``kgc_version``, and
for the operators on embedding tables ``kgc_lookup``, ``kgc_lookup_grad``,
``kgc_pack4``, ``kgc_scores4``, ``kgc_adjust``.  The classes ``Join`` and
``Embed`` are thin convenience wrappers around them.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

from . import build as _build

KGC_F32, KGC_BF16 = 0, 1
KGC_PRUNE_AUTO, KGC_PRUNE_OFF, KGC_PRUNE_ON = 0, 1, 2
KGC_OK, KGC_OVERFLOW = 0, 1
KGC_E_INVALID, KGC_E_NOMEM, KGC_E_HIP = -1, -2, -3

EXPORTS = ["kgc_create", "kgc_join", "kgc_join_range", "kgc_join_ab", "kgc_join_se", "kgc_join_blocks", "kgc_top1", "kgc_topk", "kgc_topk_range", "kgc_norms", "kgc_get_stats", "kgc_last_error", "kgc_destroy",
           "kgc_version", "kgc_calibrate_mfma", "kgc_join_static", "kgc_set_stream", "kgc_lookup", "kgc_lookup_grad_bytes", "kgc_lookup_grad",
           "kgc_table4_bytes", "kgc_pack4", "kgc_scores4", "kgc_adjust"]


class kgc_triple(ctypes.Structure):
    _fields_ = [("h", ctypes.c_int32), ("r", ctypes.c_int32), ("t", ctypes.c_int32), ("dist", ctypes.c_float)]


class kgc_config(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("max_d", ctypes.c_int32), ("prune", ctypes.c_int32),
                ("tile_cfg", ctypes.c_int32), ("workspace_bytes", ctypes.c_int64), ("stream", ctypes.c_void_p),
                ("group_radius", ctypes.c_float), ("range_kib", ctypes.c_int32), ("factorised", ctypes.c_int32),
                ("reserved", ctypes.c_int32 * 3)]


class kgc_stats(ctypes.Structure):
    _fields_ = [("triples_total", ctypes.c_uint64), ("tiles_total", ctypes.c_uint64),
                ("tiles_evaluated", ctypes.c_uint64), ("tiles_pruned", ctypes.c_uint64),
                ("pairs_evaluated", ctypes.c_uint64), ("candidates", ctypes.c_uint64),
                ("emitted", ctypes.c_uint64), ("join_launches", ctypes.c_uint64), ("groups", ctypes.c_uint64),
                ("ms_total", ctypes.c_float), ("ms_precompute", ctypes.c_float), ("ms_prune", ctypes.c_float),
                ("ms_join", ctypes.c_float), ("tile_m", ctypes.c_int32), ("tile_n", ctypes.c_int32),
                ("k_padded", ctypes.c_int32), ("relation_batches", ctypes.c_int32), ("join_variant", ctypes.c_int32),
                ("exact_blocks", ctypes.c_int32)]

    def as_dict(self) -> dict:
        return {name: getattr(self, name) for name, _ in self._fields_}


class kgc_adjustment(ctypes.Structure):
    """What kgc_adjust does to scores (include/kgc.h)."""
    _fields_ = [("scores", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("N", ctypes.c_int64),
                ("ld_scores", ctypes.c_int64), ("ld_out", ctypes.c_int64), ("bias", ctypes.c_void_p), ("allowed", ctypes.c_void_p),
                ("masks", ctypes.c_int64), ("ld_allowed", ctypes.c_int64), ("mask_row", ctypes.c_void_p),
                ("known_offsets", ctypes.c_void_p), ("known_ids", ctypes.c_void_p), ("known_count", ctypes.c_int64),
                ("seen_offsets", ctypes.c_void_p), ("seen_ids", ctypes.c_void_p), ("seen_count", ctypes.c_int64),
                ("repeat", ctypes.c_float), ("presence", ctypes.c_float), ("frequency", ctypes.c_float), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int64)]


_lib = None


class kgc_cursor(ctypes.Structure):
    """Where a join over blocks stands (include/kgc.h); all zero to start."""
    _fields_ = [("unit", ctypes.c_uint64), ("units", ctypes.c_uint64), ("need", ctypes.c_uint64), ("reserved", ctypes.c_uint64)]


def library_path() -> str:
    return _build.LIB


def load_library():
    """Load libkgc.so.  It is built first when no built library exists.  A library older than its sources is loaded
    as it is, with a warning (a rebuild takes minutes and the GPU tests must not spend them): run
    ``python -m paper_2307_12059_amd.build`` after a change, or set KGC_REBUILD_STALE=1 to have it done here."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        _build.build()
    elif _build.stale():
        if os.environ.get("KGC_REBUILD_STALE") == "1":
            _build.build()
        else:
            import warnings
            warnings.warn("libkgc.so is older than its sources: loading it as it is (rebuild with "
                          "`python -m paper_2307_12059_amd.build`)", RuntimeWarning, stacklevel=2)
    lib = ctypes.CDLL(_build.LIB)
    vp = ctypes.c_void_p
    lib.kgc_create.restype = ctypes.c_int
    lib.kgc_create.argtypes = [ctypes.POINTER(kgc_config), ctypes.POINTER(vp)]
    lib.kgc_join.restype = ctypes.c_int
    lib.kgc_join.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, vp, ctypes.c_int32, ctypes.c_int32,
                             ctypes.c_float, vp, ctypes.c_uint64, ctypes.POINTER(ctypes.c_uint64)]
    lib.kgc_join_static.restype = ctypes.c_int
    lib.kgc_join_static.argtypes = lib.kgc_join.argtypes
    lib.kgc_join_range.restype = ctypes.c_int
    lib.kgc_join_range.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, vp, ctypes.c_int32, ctypes.c_int32,
                                   ctypes.c_float, ctypes.c_int32, ctypes.c_int32, vp, ctypes.c_uint64,
                                   ctypes.POINTER(ctypes.c_uint64)]
    lib.kgc_join_blocks.restype = ctypes.c_int
    lib.kgc_join_blocks.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
                                    ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(kgc_cursor), vp, ctypes.c_uint64,
                                    ctypes.POINTER(ctypes.c_uint64)]
    lib.kgc_join_se.restype = ctypes.c_int
    lib.kgc_join_se.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
                                vp, ctypes.c_uint64, ctypes.POINTER(ctypes.c_uint64)]
    lib.kgc_join_ab.restype = ctypes.c_int
    lib.kgc_join_ab.argtypes = [vp, vp, vp, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                ctypes.c_float, vp, ctypes.c_uint64, ctypes.POINTER(ctypes.c_uint64)]
    lib.kgc_top1.restype = ctypes.c_int
    lib.kgc_top1.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                             ctypes.POINTER(kgc_triple)]
    lib.kgc_topk.restype = ctypes.c_int
    lib.kgc_topk.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                             ctypes.c_uint64, vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.kgc_topk_range.restype = ctypes.c_int
    lib.kgc_topk_range.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                   ctypes.c_int32, ctypes.c_int32, ctypes.c_uint64, vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.kgc_norms.restype = ctypes.c_int
    lib.kgc_norms.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, vp, ctypes.c_int32, vp, vp]
    lib.kgc_get_stats.restype = ctypes.c_int
    lib.kgc_get_stats.argtypes = [vp, ctypes.POINTER(kgc_stats)]
    lib.kgc_last_error.restype = ctypes.c_char_p
    lib.kgc_last_error.argtypes = [vp]
    lib.kgc_destroy.restype = None
    lib.kgc_destroy.argtypes = [vp]
    lib.kgc_version.restype = ctypes.c_char_p
    lib.kgc_version.argtypes = []
    lib.kgc_calibrate_mfma.restype = ctypes.c_int
    lib.kgc_calibrate_mfma.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(ctypes.c_float)]
    i32, i64, u64, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float
    lib.kgc_set_stream.restype = ctypes.c_int
    lib.kgc_set_stream.argtypes = [vp, vp]
    lib.kgc_lookup.restype = ctypes.c_int
    lib.kgc_lookup.argtypes = [vp, vp, i64, i64, vp, i64, f32, vp, i64, i64, vp, i64, f32, i64, i32, vp, i64, i32]
    lib.kgc_lookup_grad_bytes.restype = u64
    lib.kgc_lookup_grad_bytes.argtypes = [i64, i64, i32]
    lib.kgc_lookup_grad.restype = ctypes.c_int
    lib.kgc_lookup_grad.argtypes = [vp, vp, i32, i64, vp, i64, i64, i32, f32, i32, vp, i32, i64, i64, vp, u64]
    lib.kgc_table4_bytes.restype = u64
    lib.kgc_table4_bytes.argtypes = [i64, i32]
    lib.kgc_pack4.restype = ctypes.c_int
    lib.kgc_pack4.argtypes = [vp, vp, i64, i64, i32, vp, u64, vp]
    lib.kgc_scores4.restype = ctypes.c_int
    lib.kgc_scores4.argtypes = [vp, vp, i64, i32, vp, i32, i64, i64, f32, vp, f32, vp, i32, i64]
    lib.kgc_adjust.restype = ctypes.c_int
    lib.kgc_adjust.argtypes = [vp, ctypes.POINTER(kgc_adjustment)]
    _lib = lib
    return lib


# ---- the C ABI, one Python function per entry point ----
def kgc_version() -> str:
    return load_library().kgc_version().decode()


def kgc_create(cfg: Optional[kgc_config] = None):
    """Returns (code, handle); handle is an opaque integer (None on failure)."""
    out = ctypes.c_void_p()
    rc = load_library().kgc_create(ctypes.byref(cfg) if cfg is not None else None, ctypes.byref(out))
    return rc, (out.value if rc == KGC_OK else None)


def kgc_destroy(handle) -> None:
    if handle:
        load_library().kgc_destroy(ctypes.c_void_p(handle))


def kgc_last_error(handle) -> str:
    return load_library().kgc_last_error(ctypes.c_void_p(handle)).decode()


def kgc_get_stats(handle) -> dict:
    st = kgc_stats()
    rc = load_library().kgc_get_stats(ctypes.c_void_p(handle), ctypes.byref(st))
    if rc != KGC_OK:
        raise RuntimeError("kgc_get_stats failed")
    return st.as_dict()


def kgc_join(handle, E_ptr: int, N: int, d: int, R_ptr: int, R: int, p: int, delta: float, out_ptr: int, cap: int):
    """Raw call on device addresses.  Returns (code, count)."""
    count = ctypes.c_uint64(0)
    rc = load_library().kgc_join(ctypes.c_void_p(handle), ctypes.c_void_p(E_ptr), N, d, ctypes.c_void_p(R_ptr), R, p,
                                 ctypes.c_float(delta), ctypes.c_void_p(out_ptr), cap, ctypes.byref(count))
    return rc, int(count.value)


def kgc_join_static(handle, E_ptr: int, N: int, d: int, R_ptr: int, R: int, p: int, delta: float, out_ptr: int, cap: int):
    """Raw call on device addresses: the dense join with its scratch in the library's static device array.  Returns (code, count)."""
    count = ctypes.c_uint64(0)
    rc = load_library().kgc_join_static(ctypes.c_void_p(handle), ctypes.c_void_p(E_ptr), N, d, ctypes.c_void_p(R_ptr), R, p,
                                        ctypes.c_float(delta), ctypes.c_void_p(out_ptr), cap, ctypes.byref(count))
    return rc, int(count.value)


def kgc_join_range(handle, E_ptr: int, N: int, d: int, R_ptr: int, R: int, p: int, delta: float, r_begin: int,
                   r_end: int, out_ptr: int, cap: int):
    """Raw call on device addresses, relations r_begin <= r < r_end only.  Returns (code, count)."""
    count = ctypes.c_uint64(0)
    rc = load_library().kgc_join_range(ctypes.c_void_p(handle), ctypes.c_void_p(E_ptr), N, d, ctypes.c_void_p(R_ptr), R,
                                       p, ctypes.c_float(delta), r_begin, r_end, ctypes.c_void_p(out_ptr), cap,
                                       ctypes.byref(count))
    return rc, int(count.value)


def kgc_join_ab(handle, A_ptr: int, B_ptr: int, N: int, d: int, R: int, b_per_relation: bool, p: int, delta: float,
                out_ptr: int, cap: int):
    """Raw call on device addresses: the join on caller-supplied connector outputs.  Returns (code, count)."""
    count = ctypes.c_uint64(0)
    rc = load_library().kgc_join_ab(ctypes.c_void_p(handle), ctypes.c_void_p(A_ptr), ctypes.c_void_p(B_ptr), N, d, R,
                                    1 if b_per_relation else 0, p, ctypes.c_float(delta), ctypes.c_void_p(out_ptr), cap,
                                    ctypes.byref(count))
    return rc, int(count.value)


def kgc_join_blocks(handle, E_ptr: int, N: int, d: int, R_ptr: int, R: int, p: int, delta: float, block_rows: int,
                    rel_block: int, cursor: "kgc_cursor", out_ptr: int, cap: int):
    """Raw call on device addresses: the join block by block; ``cursor`` is updated in place.  Returns (code, count)."""
    count = ctypes.c_uint64(0)
    rc = load_library().kgc_join_blocks(ctypes.c_void_p(handle), ctypes.c_void_p(E_ptr), N, d, ctypes.c_void_p(R_ptr), R, p,
                                        ctypes.c_float(delta), block_rows, rel_block, ctypes.byref(cursor),
                                        ctypes.c_void_p(out_ptr), cap, ctypes.byref(count))
    return rc, int(count.value)


def kgc_join_se(handle, E_ptr: int, N: int, d: int, Wl_ptr: int, Wr_ptr: int, R: int, p: int, delta: float, out_ptr: int,
                cap: int):
    """Raw call on device addresses: the structured-embedding join (connectors formed on the device).  Returns (code, count)."""
    count = ctypes.c_uint64(0)
    rc = load_library().kgc_join_se(ctypes.c_void_p(handle), ctypes.c_void_p(E_ptr), N, d, ctypes.c_void_p(Wl_ptr),
                                    ctypes.c_void_p(Wr_ptr), R, p, ctypes.c_float(delta), ctypes.c_void_p(out_ptr), cap,
                                    ctypes.byref(count))
    return rc, int(count.value)


def kgc_top1(handle, E_ptr: int, N: int, d: int, R_ptr: int, R: int, p: int, exclude_self: bool):
    """Raw call on device addresses.  Returns (code, kgc_triple)."""
    out = kgc_triple()
    rc = load_library().kgc_top1(ctypes.c_void_p(handle), ctypes.c_void_p(E_ptr), N, d, ctypes.c_void_p(R_ptr), R, p,
                                 1 if exclude_self else 0, ctypes.byref(out))
    return rc, out


def kgc_topk(handle, E_ptr: int, N: int, d: int, R_ptr: int, R: int, p: int, exclude_self: bool, k: int, out_ptr: int):
    """Raw call on device addresses.  Returns (code, found)."""
    found = ctypes.c_uint64(0)
    rc = load_library().kgc_topk(ctypes.c_void_p(handle), ctypes.c_void_p(E_ptr), N, d, ctypes.c_void_p(R_ptr), R, p,
                                 1 if exclude_self else 0, k, ctypes.c_void_p(out_ptr), ctypes.byref(found))
    return rc, int(found.value)


def kgc_topk_range(handle, E_ptr: int, N: int, d: int, R_ptr: int, R: int, p: int, exclude_self: bool, r_begin: int,
                   r_end: int, k: int, out_ptr: int):
    """Raw call on device addresses.  Returns (code, found)."""
    found = ctypes.c_uint64(0)
    rc = load_library().kgc_topk_range(ctypes.c_void_p(handle), ctypes.c_void_p(E_ptr), N, d, ctypes.c_void_p(R_ptr), R, p,
                                       1 if exclude_self else 0, r_begin, r_end, k, ctypes.c_void_p(out_ptr),
                                       ctypes.byref(found))
    return rc, int(found.value)


def kgc_calibrate_mfma(wave_tile: int, feed: int, ms_target: int, stream: int = 0):
    """Returns (code, TFLOP/s, ms of the timed launch)."""
    tf, ms = ctypes.c_double(0.0), ctypes.c_float(0.0)
    rc = load_library().kgc_calibrate_mfma(wave_tile, feed, ms_target, ctypes.c_void_p(stream), ctypes.byref(tf), ctypes.byref(ms))
    return rc, float(tf.value), float(ms.value)


def kgc_norms(handle, E_ptr: int, N: int, d: int, R_ptr: int, R: int, nB_ptr: int, nA_ptr: int) -> int:
    return load_library().kgc_norms(ctypes.c_void_p(handle), ctypes.c_void_p(E_ptr), N, d, ctypes.c_void_p(R_ptr), R,
                                    ctypes.c_void_p(nB_ptr), ctypes.c_void_p(nA_ptr))


def kgc_set_stream(handle, stream: int) -> int:
    return load_library().kgc_set_stream(handle, stream)


def kgc_lookup(handle, A_ptr: int, Na: int, lda: int, ia_ptr: int, sia: int, sa: float, B_ptr: int, Nb: int, ldb: int, ib_ptr: int,
               sib: int, sb: float, n: int, d: int, out_ptr: int, ldo: int, out_dtype: int) -> int:
    """Raw call on device addresses: rows of one or two tables (B_ptr = ib_ptr = 0: one), scaled and added."""
    return load_library().kgc_lookup(handle, A_ptr, Na, lda, ia_ptr, sia, sa, B_ptr, Nb, ldb, ib_ptr, sib, sb, n, d, out_ptr, ldo,
                                     out_dtype)


def kgc_lookup_grad_bytes(n: int, N: int, d: int) -> int:
    return load_library().kgc_lookup_grad_bytes(n, N, d)


def kgc_lookup_grad(handle, G_ptr: int, g_dtype: int, ldg: int, ids_ptr: int, sid: int, n: int, d: int, scale: float, accumulate: int,
                    dW_ptr: int, dw_dtype: int, N: int, ldw: int, work_ptr: int, work_bytes: int) -> int:
    """Raw call on device addresses: the gradient of a lookup with respect to its table."""
    return load_library().kgc_lookup_grad(handle, G_ptr, g_dtype, ldg, ids_ptr, sid, n, d, scale, accumulate, dW_ptr, dw_dtype, N, ldw,
                                          work_ptr, work_bytes)


def kgc_table4_bytes(N: int, d: int) -> int:
    return load_library().kgc_table4_bytes(N, d)


def kgc_pack4(handle, W_ptr: int, N: int, ldw: int, d: int, table_ptr: int, table_bytes: int, sq_ptr: int) -> int:
    """Raw call on device addresses: a table in 4 bits."""
    return load_library().kgc_pack4(handle, W_ptr, N, ldw, d, table_ptr, table_bytes, sq_ptr)


def kgc_scores4(handle, table_ptr: int, N: int, d: int, x_ptr: int, x_dtype: int, ldx: int, n: int, alpha: float, c_ptr: int, beta: float,
                y_ptr: int, y_dtype: int, ldy: int) -> int:
    """Raw call on device addresses: scores of n queries against every row of a packed table."""
    return load_library().kgc_scores4(handle, table_ptr, N, d, x_ptr, x_dtype, ldx, n, alpha, c_ptr, beta, y_ptr, y_dtype, ldy)


def kgc_adjust(handle, adjustment: "kgc_adjustment") -> int:
    """Raw call: bias, penalties and masks on scores."""
    return load_library().kgc_adjust(handle, ctypes.byref(adjustment))


# ---- convenience wrapper over torch tensors ----
class Join:
    """Owns one kgc handle bound to the current torch stream.

    ``E`` and ``Rv`` are CUDA tensors, float32 or bfloat16 (matching ``dtype``),
    contiguous.  ``join`` returns a dict of numpy arrays ``h, r, t, dist``
    (the first min(count, cap) records), ``count``, ``code`` and ``stats``.
    """

    def __init__(self, dtype: str = "f32", prune: int = KGC_PRUNE_AUTO, tile_cfg: int = 0, max_d: int = 0,
                 workspace_bytes: int = 0, group_radius: float = 0.0, range_kib: int = 0,
                 factorised: bool = False):
        import torch

        if not torch.cuda.is_available():
            raise RuntimeError("kgc needs a GPU: torch.cuda.is_available() is False and there is no CPU fallback")
        cfg = kgc_config()
        cfg.dtype = {"f32": KGC_F32, "bf16": KGC_BF16}[dtype]
        cfg.prune = prune
        cfg.tile_cfg = tile_cfg
        cfg.max_d = max_d
        cfg.workspace_bytes = workspace_bytes
        cfg.group_radius = group_radius
        cfg.range_kib = range_kib
        cfg.factorised = 1 if factorised else 0
        cfg.stream = torch.cuda.current_stream().cuda_stream
        rc, h = kgc_create(cfg)
        if rc != KGC_OK:
            raise RuntimeError(f"kgc_create failed with code {rc}")
        self.handle = h
        self.dtype = dtype
        self._torch = torch

    def close(self):
        if getattr(self, "handle", None):
            kgc_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, E, Rv):
        torch = self._torch
        want = torch.float32 if self.dtype == "f32" else torch.bfloat16
        for x in (E, Rv):
            if not (x.is_cuda and x.is_contiguous() and x.dtype == want and x.dim() == 2):
                raise ValueError("E and Rv must be contiguous 2-D CUDA tensors of the handle's dtype")
        if E.shape[0] and Rv.shape[0] and E.shape[1] != Rv.shape[1]:
            raise ValueError("E and Rv must share d")

    def join(self, E, Rv, p: int, delta: float, cap: int, out=None, fetch: bool = True, r_range=None) -> dict:
        """``r_range = (r_begin, r_end)`` restricts the join to those relations (kgc_join_range)."""
        torch = self._torch
        self._check(E, Rv)
        N, d = E.shape[0], (E.shape[1] if E.shape[0] else Rv.shape[1])
        R = Rv.shape[0]
        if out is None:
            out = torch.empty((max(cap, 1), 4), dtype=torch.int32, device=E.device)
        if r_range is None:
            rc, count = kgc_join(self.handle, E.data_ptr(), N, d, Rv.data_ptr(), R, p, float(delta), out.data_ptr(), cap)
        else:
            rc, count = kgc_join_range(self.handle, E.data_ptr(), N, d, Rv.data_ptr(), R, p, float(delta),
                                       int(r_range[0]), int(r_range[1]), out.data_ptr(), cap)
        if rc < 0:
            raise RuntimeError(f"kgc_join failed with code {rc}: {kgc_last_error(self.handle)}")
        res = {"code": rc, "count": count, "stats": kgc_get_stats(self.handle), "out": out}
        if fetch:
            n = min(count, cap)
            host = out[:n].cpu().numpy()
            res.update({"h": host[:, 0].copy(), "r": host[:, 1].copy(), "t": host[:, 2].copy(),
                        "dist": host[:, 3].copy().view("float32")})
        return res

    def join_ab(self, A, B, p: int, delta: float, cap: int) -> dict:
        """The general form: ``A`` is R x N x d, ``B`` is N x d (shared) or R x N x d (per relation)."""
        torch = self._torch
        if A.dim() != 3 or B.dim() not in (2, 3) or not A.is_contiguous() or not B.is_contiguous():
            raise ValueError("A must be R x N x d and B N x d or R x N x d, contiguous")
        if A.dtype != B.dtype or A.dtype != (torch.float32 if self.dtype == "f32" else torch.bfloat16) or not A.is_cuda or not B.is_cuda:
            raise ValueError("A and B must be CUDA tensors of the handle's dtype")
        R, N, d = A.shape
        per_rel = B.dim() == 3
        if tuple(B.shape[-2:]) != (N, d) or (per_rel and B.shape[0] != R):
            raise ValueError("B does not match A")
        out = torch.empty((max(cap, 1), 4), dtype=torch.int32, device=A.device)
        rc, count = kgc_join_ab(self.handle, A.data_ptr(), B.data_ptr(), N, d, R, per_rel, p, float(delta), out.data_ptr(), cap)
        if rc < 0:
            raise RuntimeError(f"kgc_join_ab failed with code {rc}: {kgc_last_error(self.handle)}")
        n = min(count, cap)
        host = out[:n].cpu().numpy()
        return {"code": rc, "count": count, "stats": kgc_get_stats(self.handle), "h": host[:, 0].copy(),
                "r": host[:, 1].copy(), "t": host[:, 2].copy(), "dist": host[:, 3].copy().view("float32")}

    def join_blocks(self, E, Rv, p: int, delta: float, cap: int, block_rows: int, rel_block: int, cursor=None) -> dict:
        """One call of the join block by block: runs units from ``cursor`` on until the buffer of ``cap`` records is
        full or all are done.  Returns the records of the completed units, ``code``, ``count`` and the updated ``cursor``
        (pass it to the next call while ``code`` is KGC_OVERFLOW)."""
        torch = self._torch
        self._check(E, Rv)
        if cursor is None:
            cursor = kgc_cursor()
        N, d = E.shape
        out = torch.empty((max(cap, 1), 4), dtype=torch.int32, device=E.device)
        rc, count = kgc_join_blocks(self.handle, E.data_ptr(), N, d, Rv.data_ptr(), Rv.shape[0], p, float(delta), block_rows,
                                    rel_block, cursor, out.data_ptr(), cap)
        if rc < 0:
            raise RuntimeError(f"kgc_join_blocks failed with code {rc}: {kgc_last_error(self.handle)}")
        host = out[:count].cpu().numpy()
        return {"code": rc, "count": count, "cursor": cursor, "stats": kgc_get_stats(self.handle), "h": host[:, 0].copy(),
                "r": host[:, 1].copy(), "t": host[:, 2].copy(), "dist": host[:, 3].copy().view("float32")}

    def join_se(self, E, W_lhs, W_rhs, p: int, delta: float, cap: int, fetch: bool = True) -> dict:
        """The structured-embedding join: ``E`` is N x d, ``W_lhs`` and ``W_rhs`` are R x d x d.  ``fetch=False`` leaves
        the records on the device (``out``) and returns counts and stats only."""
        torch = self._torch
        want = torch.float32 if self.dtype == "f32" else torch.bfloat16
        for x in (E, W_lhs, W_rhs):
            if not (x.is_cuda and x.is_contiguous() and x.dtype == want):
                raise ValueError("E, W_lhs and W_rhs must be contiguous CUDA tensors of the handle's dtype")
        N, d = E.shape
        R = W_lhs.shape[0]
        if tuple(W_lhs.shape) != (R, d, d) or tuple(W_rhs.shape) != (R, d, d):
            raise ValueError("W_lhs and W_rhs must be R x d x d")
        out = torch.empty((max(cap, 1), 4), dtype=torch.int32, device=E.device)
        rc, count = kgc_join_se(self.handle, E.data_ptr(), N, d, W_lhs.data_ptr(), W_rhs.data_ptr(), R, p, float(delta),
                                out.data_ptr(), cap)
        if rc < 0:
            raise RuntimeError(f"kgc_join_se failed with code {rc}: {kgc_last_error(self.handle)}")
        if not fetch:
            return {"code": rc, "count": count, "stats": kgc_get_stats(self.handle), "out": out}
        n = min(count, cap)
        host = out[:n].cpu().numpy()
        return {"code": rc, "count": count, "stats": kgc_get_stats(self.handle), "h": host[:, 0].copy(),
                "r": host[:, 1].copy(), "t": host[:, 2].copy(), "dist": host[:, 3].copy().view("float32")}

    def top1(self, E, Rv, p: int, exclude_self: bool = False):
        """The triple with the smallest distance (None when no triple is eligible): dict h, r, t, dist."""
        self._check(E, Rv)
        rc, rec = kgc_top1(self.handle, E.data_ptr(), E.shape[0], E.shape[1], Rv.data_ptr(), Rv.shape[0], p, exclude_self)
        if rc < 0:
            raise RuntimeError(f"kgc_top1 failed with code {rc}: {kgc_last_error(self.handle)}")
        if rec.h < 0:
            return None
        return {"h": int(rec.h), "r": int(rec.r), "t": int(rec.t), "dist": float(rec.dist)}

    def topk(self, E, Rv, p: int, k: int, exclude_self: bool = False, r_range=None) -> dict:
        """The k smallest-distance triples, sorted by (dist, r, h, t) on the host: dict h, r, t, dist, count.
        ``r_range = (r_begin, r_end)`` restricts the search to those relations (one relation: its k best pairs)."""
        import numpy as np
        torch = self._torch
        self._check(E, Rv)
        out = torch.empty((max(k, 1), 4), dtype=torch.int32, device=E.device)
        lo, hi = (0, Rv.shape[0]) if r_range is None else (int(r_range[0]), int(r_range[1]))
        rc, found = kgc_topk_range(self.handle, E.data_ptr(), E.shape[0], E.shape[1], Rv.data_ptr(), Rv.shape[0], p,
                                   exclude_self, lo, hi, k, out.data_ptr())
        if rc < 0:
            raise RuntimeError(f"kgc_topk failed with code {rc}: {kgc_last_error(self.handle)}")
        host = out[:found].cpu().numpy()
        h, r, t, dist = host[:, 0].copy(), host[:, 1].copy(), host[:, 2].copy(), host[:, 3].copy().view("float32")
        order = np.lexsort((t, h, r, dist))
        return {"h": h[order], "r": r[order], "t": t[order], "dist": dist[order], "count": found}

    def norms(self, E, Rv, want_nA: bool = True):
        torch = self._torch
        self._check(E, Rv)
        N, d, R = E.shape[0], E.shape[1], Rv.shape[0]
        nB = torch.empty(N, dtype=torch.float32, device=E.device)
        nA = torch.empty((R, N), dtype=torch.float32, device=E.device) if want_nA else None
        rc = kgc_norms(self.handle, E.data_ptr(), N, d, Rv.data_ptr(), R, nB.data_ptr(),
                       nA.data_ptr() if nA is not None else 0)
        if rc < 0:
            raise RuntimeError(f"kgc_norms failed with code {rc}: {kgc_last_error(self.handle)}")
        return nB, nA


_grad_bytes = functools.lru_cache(maxsize=256)(kgc_lookup_grad_bytes)
_table4_bytes = functools.lru_cache(maxsize=256)(kgc_table4_bytes)
_idle = {}        # handles of closed Embeds, by device and settings: making one takes 70 us, and they hold nothing of a call


class Table4:
    """A table in 4 bits (Embed.pack4): ``data`` as the library lays it out (``kgc_table4_bytes(N, d)`` bytes), ``sq`` the squared norms
    of its ``N`` rows of ``d``."""

    def __init__(self, data, N: int, d: int, sq):
        self.data, self.N, self.d, self.sq = data, N, d, sq


class Embed:
    """Operators on embedding tables over torch tensors: lookups and their gradient, scores of single queries against a table in
    4 bits, and what the caller knows applied to such scores.

    Owns one kgc handle of the current device; ``dtype`` ("f32" or "bf16") is the type of the tables that ``lookup`` and ``pack4``
    read.  Calls are enqueued on torch's current stream, return without waiting and can be captured into graphs; tensors of another
    stream are ordered by the caller, as for torch's own operators.  Tensors are on the handle's device with a last stride of 1, ids are int32 (any stride: a column of an n x 3 array of triples, say); an id that
    names no row is padding.  ``out`` tensors are written in place, count as changed for autograd, and are returned.  Nothing else is
    recorded for autograd, and results never require a gradient, also where arguments do: the gradient of ``lookup`` is ``lookup_grad``.
    """

    def __init__(self, dtype: str = "f32", max_d: int = 0):
        import torch

        if not torch.cuda.is_available():
            raise RuntimeError("kgc needs a GPU: torch.cuda.is_available() is False and there is no CPU fallback")
        self._types = {torch.float32: KGC_F32, torch.bfloat16: KGC_BF16}
        cfg = kgc_config()
        cfg.dtype = {"f32": KGC_F32, "bf16": KGC_BF16}[dtype]
        cfg.max_d = max_d
        self._index = torch.cuda.current_device()
        self.device = torch.device("cuda", self._index)
        self._key = (self._index, dtype, max_d)
        self._stream = None                                   # (set by the first call)
        try:
            self.handle = _idle[self._key].pop()
        except (KeyError, IndexError):
            rc, self.handle = kgc_create(cfg)
            if rc != KGC_OK:
                raise RuntimeError(f"kgc_create failed with code {rc}")
        self.dtype = dtype
        self._table_type = torch.float32 if dtype == "f32" else torch.bfloat16
        self._torch, self._int32, self._lib = torch, torch.int32, load_library()
        # the current device and stream as plain numbers: what torch.cuda's functions wrap, a microsecond less each
        self._current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)
        # torch counts the changes of a tensor, and refuses gradients that were to use what stood there before
        self._changed = torch.autograd.graph.increment_version

    def close(self):
        handle, self.handle = getattr(self, "handle", None), None
        if handle:
            idle = _idle.setdefault(self._key, [])
            if len(idle) < 16:
                idle.append(handle)
            else:
                kgc_destroy(handle)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- arguments --
    def _rows(self, name, x, d=None, dtype=None):
        """Rows, columns and row stride of a 2-D tensor."""
        if x.get_device() != self._index or x.dim() != 2:
            raise ValueError(f"{name} must be a 2-D tensor on {self.device}")
        if (x.dtype not in self._types) if dtype is None else (x.dtype != dtype):
            raise ValueError(f"{name} must be " + ("float32 or bfloat16" if dtype is None else str(dtype)))
        n, cols = x.shape
        if d is not None and cols != d:
            raise ValueError(f"{name} must have {d} columns")
        ld, step = x.stride()
        if step != 1 and cols > 1:
            raise ValueError(f"the last stride of {name} must be 1")
        return n, cols, ld if n > 1 else cols

    def _ids(self, name, x, n=None):
        """Number and stride of a 1-D tensor of ids."""
        if x.get_device() != self._index or x.dtype != self._int32 or x.dim() != 1:
            raise ValueError(f"{name} must be a 1-D int32 tensor on {self.device}")
        m = x.shape[0]
        if n is not None and m != n:
            raise ValueError(f"{name} must hold {n} ids")
        return m, x.stride(0)

    def _floats(self, name, x, N):
        if x.get_device() != self._index or x.dim() != 1 or x.shape[0] != N or x.dtype != self._torch.float32 or not x.is_contiguous():
            raise ValueError(f"{name} must be {N} contiguous floats on {self.device}")
        return x.data_ptr()

    def _out(self, out, rows, cols, out_dtype, default):
        """The output tensor, its row stride and its type's number."""
        if out is None:
            dtype = out_dtype or default
            if dtype not in self._types:
                raise ValueError("out_dtype must be float32 or bfloat16")
            return self._torch.empty((rows, cols), dtype=dtype, device=self.device), cols, self._types[dtype]
        if out_dtype not in (None, out.dtype) or out.shape[0] != rows:
            raise ValueError(f"out must be {rows} x {cols} of out_dtype")
        ld = self._rows("out", out, cols)[2]
        self._changed((out,))
        return out, ld, self._types[out.dtype]

    def _call(self, what, *args):
        if not self.handle:
            raise RuntimeError("the handle is closed")
        torch = self._torch
        if self._current_device() != self._index:
            with torch.cuda.device(self._index):
                return self._call(what, *args)
        stream = self._raw_stream(self._index)
        if stream != self._stream:
            kgc_set_stream(self.handle, stream)
            self._stream = stream
        rc = what(self.handle, *args)
        if rc != KGC_OK:
            raise RuntimeError(f"{what.__name__} failed with code {rc}: {kgc_last_error(self.handle)}")

    # -- training --
    def lookup(self, A, ia, B=None, ib=None, sa: float = 1.0, sb: float = 1.0, out=None, out_dtype=None):
        """``sa * A[ia] + sb * B[ib]`` (``B`` and ``ib`` may be left out): n x d, of ``out_dtype`` (the tables' type by default)."""
        Na, d, lda = self._rows("A", A, None, self._table_type)
        n, sia = self._ids("ia", ia)
        if (B is None) != (ib is None):
            raise ValueError("B and ib go together")
        b = ib_ptr = Nb = ldb = sib = 0
        if B is not None:
            Nb, _, ldb = self._rows("B", B, d, self._table_type)
            sib = self._ids("ib", ib, n)[1]
            if Nb:
                b, ib_ptr = B.data_ptr(), ib.data_ptr()
        out, ldo, kind = self._out(out, n, d, out_dtype, self._table_type)
        self._call(self._lib.kgc_lookup, A.data_ptr(), Na, lda, ia.data_ptr(), sia, sa, b, Nb, ldb, ib_ptr, sib, sb, n, d, out.data_ptr(),
                   ldo, kind)
        return out

    def lookup_grad(self, G, ids, N: Optional[int] = None, out=None, scale: float = 1.0, accumulate: bool = False, out_dtype=None):
        """The gradient of a lookup with respect to a table of ``N`` rows: row v is ``scale`` times the sum of ``G[i]`` over the i
        with ``ids[i] == v``; ``accumulate=True`` adds that to ``out``.  float32 unless ``out`` or ``out_dtype`` says otherwise."""
        n, d, ldg = self._rows("G", G)
        sid = self._ids("ids", ids, n)[1]
        if out is None and (N is None or accumulate):
            raise ValueError("N or out is needed" if not accumulate else "accumulate needs out")
        N = out.shape[0] if N is None else N
        out, ldw, kind = self._out(out, N, d, out_dtype, self._torch.float32)
        size = _grad_bytes(n, N, d)
        work = self._torch.empty(size, dtype=self._torch.uint8, device=self.device) if size else None
        self._call(self._lib.kgc_lookup_grad, G.data_ptr(), self._types[G.dtype], ldg, ids.data_ptr(), sid, n, d, scale,
                   1 if accumulate else 0, out.data_ptr(), kind, N, ldw, work.data_ptr() if size else 0, size)
        return out

    # -- answering --
    def pack4(self, W) -> Table4:
        """A table in 4 bits: e2m1 values with a bfloat16 scale for every 32 dimensions, and the squared norms of its rows."""
        N, d, ldw = self._rows("W", W, None, self._table_type)
        data = self._torch.empty(kgc_table4_bytes(N, d), dtype=self._torch.uint8, device=self.device)
        sq = self._torch.empty(N, dtype=self._torch.float32, device=self.device)
        self._call(self._lib.kgc_pack4, W.data_ptr(), N, ldw, d, data.data_ptr(), data.numel(), sq.data_ptr())
        return Table4(data, N, d, sq)

    def scores4(self, table: Table4, x, alpha: float = 1.0, beta: float = 0.0, c=None, out=None, out_dtype=None):
        """``alpha * x @ W.T + beta * c`` over the values that the table stands for: n x N, float32 unless ``out`` or ``out_dtype``
        says otherwise.  ``alpha=2, beta=-1, c=table.sq`` ranks the entities by the L2 distance of their 4-bit rows from the rows of ``x``."""
        n, d, ldx = self._rows("x", x, table.d)
        N, data = table.N, table.data
        if data.get_device() != self._index or data.dtype != self._torch.uint8 or data.numel() != _table4_bytes(N, d) \
                or not data.is_contiguous():
            raise ValueError(f"the table's data must be {_table4_bytes(N, d)} contiguous bytes on {self.device}")
        out, ldy, kind = self._out(out, n, N, out_dtype, self._torch.float32)
        self._call(self._lib.kgc_scores4, data.data_ptr(), N, d, x.data_ptr(), self._types[x.dtype], ldx, n, alpha,
                   self._floats("c", c, N) if c is not None else 0, beta, out.data_ptr(), kind, ldy)
        return out

    def adjust(self, scores, bias=None, allowed=None, mask_row=None, known=None, seen=None, repeat: float = 1.0,
               presence: float = 0.0, frequency: float = 0.0, out=None):
        """Scores n x N with a bias for every entity, penalties for the entities of ``seen`` and minus infinity for those that are not
        ``allowed`` or ``known`` (include/kgc.h has the formulas).  ``known`` and ``seen`` are (offsets, ids): int64 n + 1 and
        int32; ``allowed`` holds masks of (N + 31) // 32 int32 words, ``mask_row`` the number of each row's mask.  ``out=scores`` works
        in place."""
        torch = self._torch
        n, N, ld = self._rows("scores", scores)
        if out is not None and out.dtype != scores.dtype:
            raise ValueError("out must be of the scores' type")
        out, ld_out, kind = self._out(out, n, N, None, scores.dtype)
        allowed_ptr = masks = ld_allowed = mask_row_ptr = 0
        if allowed is not None:
            words = (N + 31) // 32
            if allowed.get_device() != self._index or allowed.dim() != 2 or allowed.dtype != self._int32 or allowed.shape[1] != words \
                    or (words > 1 and allowed.stride(1) != 1):
                raise ValueError(f"allowed must be masks of {words} int32 words on {self.device}")
            allowed_ptr, masks, ld_allowed = allowed.data_ptr(), allowed.shape[0], allowed.stride(0)
        if mask_row is not None:
            if self._ids("mask_row", mask_row, n)[1] != 1 and n > 1:
                raise ValueError("mask_row must be contiguous")
            mask_row_ptr = mask_row.data_ptr()
        lists = []
        for name, given in (("known", known), ("seen", seen)):
            if given is None:
                lists += (0, 0, 0)
                continue
            offsets, ids = given
            if offsets.get_device() != self._index or offsets.dim() != 1 or offsets.dtype != torch.int64 or offsets.shape[0] != n + 1 \
                    or not offsets.is_contiguous():
                raise ValueError(f"the offsets of {name} must be {n + 1} contiguous int64 on {self.device}")
            count, step = self._ids(name, ids)
            if step != 1 and count > 1:
                raise ValueError(f"the ids of {name} must be contiguous")
            lists += (offsets.data_ptr(), ids.data_ptr(), count)
        self._call(self._lib.kgc_adjust, ctypes.byref(kgc_adjustment(
            scores.data_ptr(), out.data_ptr(), n, N, ld, ld_out, 0 if bias is None else self._floats("bias", bias, N), allowed_ptr, masks,
            ld_allowed, mask_row_ptr, *lists, repeat, presence, frequency, kind, 0)))
        return out
