"""Thin ctypes binding of liblpq.so with the names of include/lpq.h.

Argument marshalling only: every step of the search path runs in the HIP library.
torch is used for device memory (tensors are the caller-owned buffers the C ABI asks
for) and for the stream the work is enqueued on.  There is no CPU fallback: if the
library cannot be loaded, importing the symbols raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch
from torch.autograd import forward_ad

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("LPQ_LIBRARY") or os.path.join(_HERE, "liblpq.so")   # LPQ_LIBRARY: another build of the same ABI

OK, EINVAL, ERANGE, ENOMEM, EDEVICE, ENONFINITE, ESTATE = range(7)
CALIB_MINMAX, CALIB_ABSMAX, CALIB_GAUSS, CALIB_QUANTILE = 0, 1, 2, 3
SCOPE_PER_FEATURE, SCOPE_GLOBAL, SCOPE_SHARED_WIDTH = 0, 1, 2
METRIC_L2SQ, METRIC_IP = 0, 1
TUNE_PATH, TUNE_SPLITS, TUNE_SEED_ROWS, TUNE_DRY_RUN, TUNE_WORK_ORDER, TUNE_WAVE_QUERIES, TUNE_REGION_CAP = 0, 1, 2, 3, 4, 5, 6

CALIB = {"minmax": CALIB_MINMAX, "absmax": CALIB_ABSMAX, "gauss": CALIB_GAUSS, "quantile": CALIB_QUANTILE}
SCOPE = {"per_feature": SCOPE_PER_FEATURE, "global": SCOPE_GLOBAL, "shared_width": SCOPE_SHARED_WIDTH}
METRIC = {"l2sq": METRIC_L2SQ, "ip": METRIC_IP}

_ERR_NAMES = {1: "LPQ_EINVAL", 2: "LPQ_ERANGE", 3: "LPQ_ENOMEM", 4: "LPQ_EDEVICE",
              5: "LPQ_ENONFINITE", 6: "LPQ_ESTATE"}


class LpqError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{_ERR_NAMES.get(code, code)}: {msg}")
        self.code = code


_lib = None


def lib() -> C.CDLL:
    """The loaded library (raises OSError if liblpq.so has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError(f"{LIB_PATH} is missing: run `python -m paper_2110_08919_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i64, i32, f32 = C.c_void_p, C.c_int64, C.c_int, C.c_float
        sig = {
            "lpq_quantizer_create": (i32, [C.POINTER(vp), i32, i32]),
            "lpq_quantizer_destroy": (None, [vp]),
            "lpq_quantizer_calibrate": (i32, [vp, vp, i64, i64, i32, i32, f32, vp]),
            "lpq_quantizer_set_params": (i32, [vp, vp, vp, vp]),
            "lpq_quantizer_get_params": (i32, [vp, vp, vp, vp, vp]),
            "lpq_encode": (i32, [vp, vp, i64, i64, vp, i64, vp, vp]),
            "lpq_index_create": (i32, [C.POINTER(vp), vp, i64]),
            "lpq_index_create_packed": (i32, [C.POINTER(vp), vp, i64]),
            "lpq_index_destroy": (None, [vp]),
            "lpq_index_add_f32": (i32, [vp, vp, i64, i64, vp]),
            "lpq_index_add_i8": (i32, [vp, vp, i64, i64, vp]),
            "lpq_index_size": (i64, [vp]),
            "lpq_index_data": (i32, [vp, C.POINTER(vp), C.POINTER(i64), C.POINTER(vp)]),
            "lpq_search_workspace_bytes": (C.c_size_t, [vp, i64, i32, i32]),
            "lpq_search": (i32, [vp, vp, i64, i64, i32, i32, vp, vp, vp, C.c_size_t, vp]),
            "lpq_search_static": (i32, [vp, vp, i64, i64, i32, i32, vp, vp, vp]),
            "lpq_search_i8": (i32, [vp, vp, i64, i64, i32, i32, vp, vp, vp, C.c_size_t, vp]),
            "lpq_search_f32_workspace_bytes": (C.c_size_t, [i64, i64, i32, i32]),
            "lpq_search_f32": (i32, [vp, i64, i64, vp, i64, i64, i32, i32, i32, vp, vp, vp, C.c_size_t, vp]),
            "lpq_gather_dist_i8": (i32, [vp, vp, i64, i64, vp, i32, i32, vp, vp]),
            "lpq_rerank_f32": (i32, [vp, i64, i64, vp, i64, i64, i32, vp, i32, i32, i32, vp, vp, vp]),
            "lpq_search_overflow_stats": (i32, [vp, i64, i32, i32, vp, C.POINTER(i64), C.POINTER(i64)]),
            "lpq_search_overflow_left": (i32, [vp, i64, i32, i32, vp, C.POINTER(i64)]),
            "lpq_set_tuning": (i32, [i32, i64]),
            "lpq_profile_enable": (i32, [i32]),
            "lpq_profile_read": (i32, [C.POINTER(i64), C.POINTER(C.c_double)]),
            "lpq_profile_read_kind": (i32, [i32, C.POINTER(i64), C.POINTER(C.c_double)]),
            "lpq_search_plan_info": (i32, [i32, i32, i32, i64, i64, i32, C.POINTER(i64), i32]),
            "lpq_search_maxima_info": (i32, [i32, i32, i32, i64, i64, i32, C.POINTER(i64), i32]),
            "lpq_probe_mfma_i8": (i32, [vp, C.c_size_t, i32, C.POINTER(C.c_double), vp]),
            "lpq_probe_scan_core": (i32, [vp, C.c_size_t, i32, C.POINTER(C.c_double), vp]),
            "lpq_probe_stream": (i32, [vp, C.c_size_t, i32, i32, C.POINTER(C.c_double), vp]),
            "lpq_kv_storage_bytes": (i32, [i32, i32, i32, i64, i32, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t), C.POINTER(i32)]),
            "lpq_kv_create": (i32, [C.POINTER(vp), vp, vp, i32, i32, i64, i32, vp, vp, vp]),
            "lpq_kv_destroy": (None, [vp]),
            "lpq_kv_write": (i32, [vp, vp, i64, i64, vp, i64, i64, i32, i64, i64, vp, vp, vp, i64, i64, vp]),
            "lpq_kv_write_rotated": (i32, [vp, vp, i64, i64, vp, i64, i64, i32, i64, i64, vp, vp, vp, i64, i64, vp, vp, i64, i64, i32, i32, vp,
                                           vp, i64, i64, i32, vp, i64, i64, vp]),
            "lpq_kv_read": (i32, [vp, vp, i64, i64, vp, i64, i64, i32, i64, i64, vp, vp, vp, i64, i64, vp]),
            "lpq_kv_select_workspace_bytes": (C.c_size_t, [vp, i64, i64]),
            "lpq_kv_select": (i32, [vp, vp, i64, i64, i64, i32, i64, i32, i32, vp, vp, i64, i64, i32, i32, i32, vp, vp,
                                    C.c_size_t, vp]),
            "lpq_kv_attend_workspace_bytes": (C.c_size_t, [vp, i64, i32, i32, i64, i32]),
            "lpq_kv_attend": (i32, [vp, vp, i64, i64, i64, i32, i64, i32, i32, f32, vp, vp, i64, i64, vp, i32, vp, i64, i64,
                                    i64, vp, vp, C.c_size_t, vp]),
            "lpq_kv_attend_masked_workspace_bytes": (C.c_size_t, [vp, i64, i32, i32, i64, i32, i64, i32, i32]),
            "lpq_kv_attend_masked": (i32, [vp, vp, i64, i64, i64, i32, i64, i32, i32, f32, vp, vp, i64, i64, vp, i32, i64, i32, vp, i64, i64,
                                           vp, i64, i64, i64, vp, vp, C.c_size_t, vp]),
            "lpq_row_codes_bytes": (C.c_size_t, [i64, i32]),
            "lpq_encode_rows": (i32, [vp, i64, i32, i64, i32, vp, vp, vp]),
            "lpq_matmul_i8_workspace_bytes": (C.c_size_t, [i64, i64, i32]),
            "lpq_matmul_i8": (i32, [vp, vp, i64, vp, vp, i64, i32, vp, vp, i64, i32, vp, C.c_size_t, vp]),
            "lpq_linear8_workspace_bytes": (C.c_size_t, [i64, i64, i32]),
            "lpq_linear8": (i32, [vp, i64, i32, i64, vp, vp, i64, i32, vp, vp, i64, vp, C.c_size_t, vp]),
            "lpq_linear8_plan_info": (i32, [i64, i64, i32, C.POINTER(i64), i32]),
            "lpq_last_error": (C.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _check(rc: int):
    if rc != 0:
        raise LpqError(rc, lib().lpq_last_error().decode())


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(t: torch.Tensor) -> int:
    """_stream() on the device of t.  A call of a few microseconds feels that the Stream object costs 2.7 us to make."""
    return _raw_stream(t.get_device()) if _raw_stream is not None else torch.cuda.current_stream(t.device).cuda_stream


# (torch.cuda.current_device() looks first whether there is one)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dev_matrix(t: torch.Tensor, dtype):
    assert t.is_cuda and t.dtype == dtype and t.dim() == 2 and t.stride(1) == 1, "need a row-major device matrix"
    ld = t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])   # a 1-row stride is arbitrary
    return t.data_ptr(), t.shape[0], ld


def set_tuning(key: int, value: int):
    _check(lib().lpq_set_tuning(key, value))


def profile_enable(on: bool):
    _check(lib().lpq_profile_enable(1 if on else 0))


PROFILE_SCAN, PROFILE_SEED = 0, 1


def profile_read(kind=None):
    """(launches, total ms) of all bracketed launches, or of one kind (PROFILE_SCAN / PROFILE_SEED)."""
    n, ms = C.c_int64(0), C.c_double(0.0)
    if kind is None:
        _check(lib().lpq_profile_read(C.byref(n), C.byref(ms)))
    else:
        _check(lib().lpq_profile_read_kind(kind, C.byref(n), C.byref(ms)))
    return n.value, ms.value


PLAN_INFO_COUNT = 35


def search_plan_info(d: int, bits: int, packed: bool, n_items: int, nq: int, k: int):
    """lpq_search_plan_info: the plan of a search as a list of PLAN_INFO_COUNT integers (no device needed)."""
    out = (C.c_int64 * PLAN_INFO_COUNT)()
    _check(lib().lpq_search_plan_info(d, bits, 1 if packed else 0, n_items, nq, k, out, PLAN_INFO_COUNT))
    return list(out)


MAXIMA_INFO_COUNT = 8


def search_maxima_info(d: int, bits: int, packed: bool, n_items: int, nq: int, k: int):
    """lpq_search_maxima_info: how such a search goes by group maxima, MAXIMA_INFO_COUNT zeros where it does not (no device needed)."""
    out = (C.c_int64 * MAXIMA_INFO_COUNT)()
    _check(lib().lpq_search_maxima_info(d, bits, 1 if packed else 0, n_items, nq, k, out, MAXIMA_INFO_COUNT))
    return list(out)


LINEAR8_INFO_COUNT = 4


def linear8_plan_info(m: int, n: int, d: int):
    """lpq_linear8_plan_info: tokens and channels of a workgroup, parts of the features, whether codes are made on the way (no device needed)."""
    out = (C.c_int64 * LINEAR8_INFO_COUNT)()
    _check(lib().lpq_linear8_plan_info(m, n, d, out, LINEAR8_INFO_COUNT))
    return list(out)


def probe_mfma_i8(operands: torch.Tensor = None, iters: int = 50000) -> float:
    """Sustained 1e12 op/s of a register-resident int8 matrix-instruction loop whose operand
    registers are filled from `operands` (a contiguous device tensor; None = zeros)."""
    out = C.c_double(0.0)
    nbytes = 0 if operands is None else operands.numel() * operands.element_size()
    _check(lib().lpq_probe_mfma_i8(_ptr(operands), nbytes, iters, C.byref(out), _stream()))
    return out.value


def probe_scan_core(operands: torch.Tensor = None, stages: int = 12000) -> float:
    """Sustained 1e12 op/s of the batched scan's inner loop alone (no copies, barrier or candidates),
    its LDS ring and query registers filled from `operands` (None = zeros)."""
    out = C.c_double(0.0)
    nbytes = 0 if operands is None else operands.numel() * operands.element_size()
    _check(lib().lpq_probe_scan_core(_ptr(operands), nbytes, stages, C.byref(out), _stream()))
    return out.value


def probe_stream(src: torch.Tensor, mode: int = 0, reps: int = 10) -> float:
    """Sustained 1e9 B/s of reading `src` (contiguous device tensor): mode 0 asynchronous
    global->LDS copies, mode 1 register loads."""
    out = C.c_double(0.0)
    _check(lib().lpq_probe_stream(src.data_ptr(), src.numel() * src.element_size(), mode, reps, C.byref(out), _stream()))
    return out.value


class Quantizer:
    """lpq_quantizer_* : the constants of Equation 1 on the device."""

    def __init__(self, d: int, bits: int = 8):
        h = C.c_void_p()
        _check(lib().lpq_quantizer_create(C.byref(h), d, bits))
        self._h, self.d, self.bits = h, d, bits

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.lpq_quantizer_destroy(self._h)
            self._h = None

    def calibrate(self, x: torch.Tensor, mode="minmax", scope="per_feature", sigma_mult=1.0):
        p, n, ld = _dev_matrix(x, torch.float32)
        assert x.shape[1] == self.d
        _check(lib().lpq_quantizer_calibrate(self._h, p, n, ld, CALIB[mode], SCOPE[scope], sigma_mult, _stream()))
        return self

    def set_params(self, k, s_b, s_e):
        arrs = [torch.as_tensor(a, dtype=torch.float32).contiguous().cpu() for a in (k, s_b, s_e)]
        assert all(a.numel() == self.d for a in arrs)
        _check(lib().lpq_quantizer_set_params(self._h, *[a.data_ptr() for a in arrs]))
        return self

    def get_params(self):
        out = [torch.empty(self.d, dtype=torch.float32) for _ in range(4)]
        _check(lib().lpq_quantizer_get_params(self._h, *[a.data_ptr() for a in out]))
        return tuple(a.numpy() for a in out)  # k, S_b, S_e, m

    def encode(self, x: torch.Tensor, with_norms=False, ld_codes=None):
        p, n, ld = _dev_matrix(x, torch.float32)
        ldc = ld_codes or self.d
        # (a wider stride leaves bytes behind each row that the call does not write)
        codes = (torch.empty if ldc == self.d else torch.zeros)((n, ldc), dtype=torch.int8, device=x.device)
        norms = torch.empty(n, dtype=torch.int32, device=x.device) if with_norms else None
        _check(lib().lpq_encode(self._h, p, n, ld, codes.data_ptr(), ldc, _ptr(norms), _stream()))
        codes = codes[:, :self.d]
        return (codes, norms) if with_norms else codes


class Index:
    """lpq_index_* and lpq_search*: the flat int8 corpus and exhaustive top-k search."""

    def __init__(self, quantizer: Quantizer, capacity: int, packed: bool = False):
        h = C.c_void_p()
        create = lib().lpq_index_create_packed if packed else lib().lpq_index_create
        _check(create(C.byref(h), quantizer._h, capacity))
        self._h, self.d, self.capacity, self.packed = h, quantizer.d, capacity, packed
        self._ws = None

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.lpq_index_destroy(self._h)
            self._h = None

    def add_f32(self, x: torch.Tensor):
        p, n, ld = _dev_matrix(x, torch.float32)
        assert x.shape[1] == self.d
        _check(lib().lpq_index_add_f32(self._h, p, n, ld, _stream()))
        return self

    def add_i8(self, codes: torch.Tensor):
        p, n, ld = _dev_matrix(codes, torch.int8)
        assert codes.shape[1] == self.d
        _check(lib().lpq_index_add_i8(self._h, p, n, ld, _stream()))
        return self

    @property
    def size(self) -> int:
        return lib().lpq_index_size(self._h)

    def data(self):
        """(codes_ptr, ld_codes, norms_ptr): raw device pointers into the index storage."""
        cp, ld, npn = C.c_void_p(), C.c_int64(), C.c_void_p()
        _check(lib().lpq_index_data(self._h, C.byref(cp), C.byref(ld), C.byref(npn)))
        return cp.value, ld.value, npn.value

    def storage(self):
        """Host copies (numpy) of the stored rows, uint8 [size, ld_codes] as they lie in device memory
        (int8 codes, or two nibbles per byte for a packed index), and of the norms int32 [size]."""
        import numpy as np
        cp, ld, npn = self.data()
        torch.cuda.synchronize()
        n = self.size
        rows = torch.empty((n, ld), dtype=torch.uint8, device="cuda")
        norms = torch.empty((n,), dtype=torch.int32, device="cuda")
        hip = C.CDLL("libamdhip64.so")
        hip.hipMemcpy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]
        for dst, src, nb in ((rows, cp, n * ld), (norms, npn, n * 4)):
            rc = hip.hipMemcpy(dst.data_ptr(), src, nb, 3)   # device to device
            if rc:
                raise LpqError(-1, f"hipMemcpy failed with {rc}")
        return np.asarray(rows.cpu()), np.asarray(norms.cpu())

    def workspace_bytes(self, nq: int, k: int, metric="l2sq") -> int:
        return lib().lpq_search_workspace_bytes(self._h, nq, k, METRIC[metric])

    def _workspace(self, nbytes: int, device) -> torch.Tensor:
        if self._ws is None or self._ws.numel() < nbytes or self._ws.device != device:
            self._ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        return self._ws

    def gather_dist(self, qcodes: torch.Tensor, ids: torch.Tensor, metric="l2sq"):
        """int32 [nq, m]: integer distance between query i (int8 codes) and item ids[i, j]."""
        qp, nq, ld = _dev_matrix(qcodes, torch.int8)
        ip, ni, ldi = _dev_matrix(ids, torch.int32)
        assert ni == nq and ldi == ids.shape[1]
        out = torch.empty(ids.shape, dtype=torch.int32, device=ids.device)
        _check(lib().lpq_gather_dist_i8(self._h, qp, nq, ld, ip, ids.shape[1], METRIC[metric], out.data_ptr(),
                                        _stream()))
        return out

    def overflow_stats(self, nq: int, k: int, metric, workspace: torch.Tensor = None):
        """(queries searched again exactly, largest region fill) of the last search in `workspace`
        (default: the index's own workspace, used when search() was given none)."""
        workspace = self._ws if workspace is None else workspace
        a, b = C.c_int64(0), C.c_int64(0)
        _check(lib().lpq_search_overflow_stats(self._h, nq, k, METRIC[metric], workspace.data_ptr(), C.byref(a), C.byref(b)))
        return a.value, b.value

    def overflow_left(self, nq: int, k: int, metric, workspace: torch.Tensor = None):
        """Queries that overflowed again in the second round of the collecting scan of the last search
        (they went through the generic kernel); 0 when there was no second round."""
        workspace = self._ws if workspace is None else workspace
        a = C.c_int64(0)
        _check(lib().lpq_search_overflow_left(self._h, nq, k, METRIC[metric], workspace.data_ptr(), C.byref(a)))
        return a.value

    def search(self, q: torch.Tensor, k: int, metric="l2sq", out=None, workspace=None):
        """q fp32 [nq, d] or int8 codes [nq, d] on the device -> (ids int32, dists int32) [nq, k]."""
        is_codes = q.dtype == torch.int8
        p, nq, ld = _dev_matrix(q, torch.int8 if is_codes else torch.float32)
        ids, dists = out if out is not None else (
            torch.empty((nq, k), dtype=torch.int32, device=q.device),
            torch.empty((nq, k), dtype=torch.int32, device=q.device))
        need = self.workspace_bytes(nq, k, metric)
        ws = workspace if workspace is not None else self._workspace(need, q.device)
        fn = lib().lpq_search_i8 if is_codes else lib().lpq_search
        _check(fn(self._h, p, nq, ld, k, METRIC[metric], ids.data_ptr(), dists.data_ptr(),
                  ws.data_ptr(), ws.numel(), _stream()))
        return ids, dists

    def search_static(self, q: torch.Tensor, k: int, metric="l2sq", out=None):
        """lpq_search_static: fp32 queries, the library's built-in workspace, no allocation inside the call
        (pass `out` to keep this wrapper from allocating the result tensors either)."""
        p, nq, ld = _dev_matrix(q, torch.float32)
        ids, dists = out if out is not None else (
            torch.empty((nq, k), dtype=torch.int32, device=q.device),
            torch.empty((nq, k), dtype=torch.int32, device=q.device))
        _check(lib().lpq_search_static(self._h, p, nq, ld, k, METRIC[metric], ids.data_ptr(), dists.data_ptr(), _stream()))
        return ids, dists


STATIC_WORKSPACE_BYTES = 64 << 20

TYPE_F32, TYPE_F16, TYPE_BF16 = 0, 1, 2
_TYPE = {torch.float32: TYPE_F32, torch.float16: TYPE_F16, torch.bfloat16: TYPE_BF16}


def _no_gradient(why: str, *tensors):
    """Refuses tensors that ask for a gradient, or carry a tangent, which the call would not give or pass on."""
    if torch.is_grad_enabled():
        for t in tensors:
            assert t is None or not t.requires_grad, f"{why}: use torch.no_grad() or detach()"
    if forward_ad._current_level >= 0:           # within dual_level(), with or without gradients enabled
        for t in tensors:
            assert t is None or forward_ad.unpack_dual(t).tangent is None, f"{why}, nor a tangent: use unpack_dual(t).primal"


def _dev_ints(t: torch.Tensor, n: int, device: int):
    assert t.get_device() == device and t.dtype is torch.int32 and t.dim() == 1 and t.shape[0] == n and t.is_contiguous(), \
        f"need {n} contiguous int32 values on the cache's device"
    return t.data_ptr()


class KVCache:
    """lpq_kv_*: keys and values of one layer as codes in pages, and the attention that reads them.

    The quantizers hold the constants of the heads' features one after the other (d = heads * features of a head).
    Storage is three tensors of this object: `k` and `v` [pages, heads, page, row bytes] and the pages' bounds.
    Which pages a sequence has is the caller's to say: `table` int32 [sequences, columns], page numbers in order of
    position, -1 (or anything outside the pool) where there is none.  Everything that a call is given lies on the cache's device, which is the current one;
    the quantizers were made there."""

    def __init__(self, keys: Quantizer, values: Quantizer, heads: int, page: int, pages: int, packed: bool = False,
                 device="cuda"):
        assert heads >= 1 and keys.d % heads == 0, "d of the quantizers must be a multiple of heads"
        assert torch.device(device).type == "cuda", "the cache lies in device memory"
        with torch.cuda.device(device):
            self._create(keys, values, heads, page, pages, packed, device)

    def _create(self, keys, values, heads, page, pages, packed, device):
        row = C.c_int()
        self.heads, self.dim, self.page, self.pages, self.packed = heads, keys.d // heads, page, pages, packed
        _check(lib().lpq_kv_storage_bytes(heads, self.dim, page, pages, 1 if packed else 0, None, None, C.byref(row)))
        shape = (pages, heads, page, row.value // 2 if packed else row.value)
        kind = torch.uint8 if packed else torch.int8
        self.k, self.v = (torch.zeros(shape, dtype=kind, device=device) for _ in range(2))
        self._at = self.k.get_device()
        self._bounds = torch.zeros((pages, heads, 2, row.value), dtype=torch.int8, device=device)
        torch.cuda.current_stream().synchronize()           # calls on any stream find it cleared
        h = C.c_void_p()
        _check(lib().lpq_kv_create(C.byref(h), keys._h, values._h, heads, page, pages, 1 if packed else 0, self.k.data_ptr(),
                                   self.v.data_ptr(), self._bounds.data_ptr()))
        self._h = h

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.lpq_kv_destroy(self._h)
            self._h = None

    @property
    def bounds(self) -> torch.Tensor:
        """int8 [pages, heads, 2, features]: smallest and largest key code of each page."""
        return self._bounds[..., :self.dim]

    def _table(self, table: torch.Tensor):
        assert _current_device() == self._at, "calls go to the current device: make the cache's the current one"
        assert table.get_device() == self._at and table.dtype is torch.int32 and table.dim() == 2, "need a device table int32 [sequences, columns]"
        nseq, columns = table.shape
        ld, inner = table.stride()
        assert inner == 1 or columns == 1, "need the columns of the table side by side"
        return nseq, (table.data_ptr(), ld if nseq > 1 else max(ld, columns), columns)

    def _rows(self, t: torch.Tensor, dtype):
        assert t.get_device() == self._at and t.dtype is dtype and t.dim() == 3, f"need device rows of {dtype}"
        n, heads, dim = t.shape
        by_row, by_head, inner = t.stride()
        assert heads == self.heads and dim == self.dim and (inner == 1 or dim == 1), \
            f"need rows [n, {self.heads}, {self.dim}], features side by side"
        return n, (t.data_ptr(), by_row, by_head)

    def write(self, k: torch.Tensor, v: torch.Tensor, first: torch.Tensor, table: torch.Tensor, starts: torch.Tensor = None):
        """New rows [n, heads, features] (float32, float16 or bfloat16): rows starts[b] .. starts[b + 1] go to positions
        first[b] on of sequence b; without starts one row per sequence."""
        nseq, tab = self._table(table)
        n, keys = self._rows(k, k.dtype)
        same, values = self._rows(v, k.dtype)
        assert n == same, "as many values as keys"
        _check(_lib.lpq_kv_write(self._h, *keys, *values, _TYPE[k.dtype], n, nseq, _dev_ints(first, nseq, self._at),
                                 None if starts is None else _dev_ints(starts, nseq + 1, self._at), *tab, _stream_of(table)))

    def write_rotated(self, k: torch.Tensor, v: torch.Tensor, first: torch.Tensor, table: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor,
                      starts: torch.Tensor = None, positions: torch.Tensor = None, q: torch.Tensor = None, out: torch.Tensor = None,
                      interleaved: bool = False):
        """write() of keys that are turned by their positions' angles on the way, and the queries q [n, query heads, features] of
        the same rows turned with them (returned; out=q: in place; out must not overlap k, v or the angles).  cos, sin: float32 [positions, turned features / 2]; features are
        paired with those half the turned ones further, interleaved: with their neighbours.  positions: int32 [n], where a row
        stands if not at the position it is written to.  Rows, queries and angles that require a gradient are refused."""
        _no_gradient("rotated rows have no gradient here", k, v, q, cos, sin)
        nseq, tab = self._table(table)
        n, keys = self._rows(k, k.dtype)
        same, values = self._rows(v, k.dtype)
        assert n == same, "as many values as keys"
        assert cos.get_device() == self._at and cos.dtype is torch.float32 and cos.dim() == 2 and cos.stride(1) == 1, \
            "need device angles float32 [positions, pairs]"
        count, pairs = cos.shape
        apart = cos.stride(0) if count > 1 else max(cos.stride(0), pairs)
        assert sin.get_device() == self._at and sin.dtype is torch.float32 and sin.shape == cos.shape and sin.stride(1) == 1 \
            and (count == 1 or sin.stride(0) == apart), "need sines laid out as the cosines"
        queries, q_heads = (None, 0, 0), 0
        into = (None, 0, 0)
        if q is not None:
            if out is None:
                out = q.new_empty(q.shape)
            q_heads, queries = self._query_rows(q, n, k.dtype)
            more, into = self._query_rows(out, n, k.dtype)
            assert more == q_heads, "as many heads in the output"
        _check(_lib.lpq_kv_write_rotated(self._h, *keys, *values, _TYPE[k.dtype], n, nseq, _dev_ints(first, nseq, self._at),
                                         None if starts is None else _dev_ints(starts, nseq + 1, self._at), *tab, cos.data_ptr(), sin.data_ptr(), apart, count,
                                         2 * pairs, interleaved, None if positions is None else _dev_ints(positions, n, self._at), *queries, q_heads, *into,
                                         _stream_of(table)))
        return out

    def _query_rows(self, t: torch.Tensor, n: int, dtype):
        assert t.get_device() == self._at and t.dtype is dtype and t.dim() == 3, f"need device queries of {dtype}"
        rows, heads, dim = t.shape
        by_row, by_head, inner = t.stride()
        assert rows == n and dim == self.dim and (inner == 1 or dim == 1), f"need queries [{n}, query heads, {self.dim}], features side by side"
        return heads, (t.data_ptr(), by_row, by_head)

    def read(self, first: torch.Tensor, table: torch.Tensor, starts: torch.Tensor = None, rows: int = None,
             dtype=torch.float32, out=None):
        """Keys and values [rows, heads, features] as they read back, numbered as in write(); zeros where there is nothing, as in
        rows from starts[-1] on."""
        nseq, tab = self._table(table)
        n = nseq if starts is None else rows
        assert n is not None, "with starts, say how many rows"
        k, v = out if out is not None else (
            torch.empty((n, self.heads, self.dim), dtype=dtype, device=table.device),
            torch.empty((n, self.heads, self.dim), dtype=dtype, device=table.device))
        a, keys = self._rows(k, k.dtype)
        b, values = self._rows(v, k.dtype)
        assert a == n and b == n, f"need {n} rows"
        _check(_lib.lpq_kv_read(self._h, *keys, *values, _TYPE[k.dtype], n, nseq, _dev_ints(first, nseq, self._at),
                                None if starts is None else _dev_ints(starts, nseq + 1, self._at), *tab, _stream_of(table)))
        return k, v

    def _queries(self, q: torch.Tensor, nseq: int):
        assert q.get_device() == self._at and q.dtype in _TYPE and q.dim() == 4, "need device queries of float32, float16 or bfloat16"
        n, new, heads, dim = q.shape
        by_seq, by_token, by_head, inner = q.stride()
        assert n == nseq and dim == self.dim and (inner == 1 or dim == 1), \
            f"need queries [{nseq}, new tokens, query heads, {self.dim}], features side by side"
        return new, heads, (q.data_ptr(), by_seq, by_token, by_head)

    @staticmethod
    def _workspace(given: torch.Tensor, need: int, device):
        """The workspace to pass: memory of this call's own unless some was given (calls on several streams do not share any)."""
        if given is not None:
            assert given.is_cuda and given.is_contiguous() and given.device == device, "need a workspace that is one run of the device's memory"
        elif need:
            given = torch.empty(need, dtype=torch.uint8, device=device)
        return (given, None, 0) if given is None else (given, given.data_ptr(), given.numel() * given.element_size())

    def select(self, q: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, n_select: int, keep_first: int = 0,
               keep_last: int = 1, out: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
        """int32 [sequences, heads, n_select]: the pages with the largest bounds of the queries' integer products,
        ascending, -1 at the end."""
        nseq, tab = self._table(table)
        new, q_heads, queries = self._queries(q, nseq)
        if out is None:
            out = torch.empty((nseq, self.heads, n_select), dtype=torch.int32, device=q.device)
        assert out.get_device() == self._at and out.dtype is torch.int32 and out.is_contiguous() and out.shape == (nseq, self.heads, n_select)
        workspace, ws, size = self._workspace(workspace, _lib.lpq_kv_select_workspace_bytes(self._h, nseq, tab[2]), q.device)
        _check(_lib.lpq_kv_select(self._h, *queries, _TYPE[q.dtype], nseq, new, q_heads, _dev_ints(lengths, nseq, self._at), *tab,
                                  n_select, keep_first, keep_last, out.data_ptr(), ws, size, _stream_of(q)))
        return out

    def attend(self, q: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, pages: torch.Tensor = None,
               scale: float = None, out: torch.Tensor = None, return_lse: bool = False, workspace: torch.Tensor = None,
               window: int = None, sinks: int = 0, tree: torch.Tensor = None):
        """Attention of q [sequences, new tokens, query heads, features] over the cache (the last new_tokens positions of
        each length are the queries' own), or over the `pages` that select() names; scale 1 / sqrt(features) by default.
        window: a token sees the last `window` positions up to its own, and the first `sinks`.  tree: bool [sequences, new
        tokens, new tokens] (or without the first axis, for all sequences), which new tokens each sees beside all the
        tokens ahead of them: drafted tokens, themselves and their ancestors.
        A call takes up to 65 536 (new token, query head) pairs of a sequence, 2^22 in all: longer prompts go through it in parts,
        each with the lengths up to its end.
        There is no way back through the codes: queries that require a gradient are refused."""
        _no_gradient("attention over codes has no gradient", q)
        nseq, tab = self._table(table)
        new, q_heads, queries = self._queries(q, nseq)
        if out is None:
            out = q.new_empty(q.shape)
            outputs = (out.data_ptr(), new * q_heads * self.dim, q_heads * self.dim, self.dim)
        else:
            assert out.shape == q.shape and out.dtype is q.dtype
            outputs = self._queries(out, nseq)[2]
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if return_lse else None
        n_select = 0
        if pages is not None:
            n_select = pages.shape[-1]
            assert pages.get_device() == self._at and pages.dtype is torch.int32 and pages.is_contiguous() and pages.shape == (nseq, self.heads, n_select) \
                and n_select > 0, "need contiguous int32 pages [sequences, heads, pages], at least one of them"
        if window is not None or sinks or tree is not None:
            return self._attend_masked(q, queries, nseq, new, q_heads, lengths, tab, pages, n_select, scale, out, outputs, lse, workspace,
                                       window, sinks, tree)
        workspace, ws, size = self._workspace(
            workspace, _lib.lpq_kv_attend_workspace_bytes(self._h, nseq, new, q_heads, tab[2], n_select), q.device)
        _check(_lib.lpq_kv_attend(self._h, *queries, _TYPE[q.dtype], nseq, new, q_heads,
                                  self.dim ** -0.5 if scale is None else scale, _dev_ints(lengths, nseq, self._at), *tab, _ptr(pages), n_select,
                                  *outputs, _ptr(lse), ws, size, _stream_of(q)))
        return (out, lse) if return_lse else out

    def _attend_masked(self, q, queries, nseq, new, q_heads, lengths, tab, pages, n_select, scale, out, outputs, lse, workspace, window, sinks,
                       tree):
        assert window is None or window >= 1, "a window holds one position at least"
        assert 0 <= sinks < 2 ** 31, "sinks are counted from 0"
        mask, by_seq, by_token = None, 0, 0
        if tree is not None:
            assert tree.get_device() == self._at and tree.dtype is torch.bool and tree.shape in ((nseq, new, new), (new, new)) \
                and (tree.stride(-1) == 1 or new == 1), f"need a device tree bool [{nseq}, {new}, {new}], the last axis contiguous"
            mask, by_seq, by_token = tree.data_ptr(), tree.stride(0) if tree.dim() == 3 else 0, tree.stride(-2)
        width = 0 if window is None else min(window, 2 ** 40)
        workspace, ws, size = self._workspace(
            workspace, _lib.lpq_kv_attend_masked_workspace_bytes(self._h, nseq, new, q_heads, tab[2], n_select, width, sinks, mask is not None), q.device)
        _check(_lib.lpq_kv_attend_masked(self._h, *queries, _TYPE[q.dtype], nseq, new, q_heads, self.dim ** -0.5 if scale is None else scale,
                                         _dev_ints(lengths, nseq, self._at), *tab, _ptr(pages), n_select, width, sinks, mask, by_seq, by_token, *outputs,
                                         _ptr(lse), ws, size, _stream_of(q)))
        return out if lse is None else (out, lse)


def _typed_matrix(t: torch.Tensor, what: str):
    assert t.is_cuda and t.dtype in _TYPE and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1), \
        f"need {what} of float32, float16 or bfloat16 on the device, a row's values side by side"
    n, d = t.shape
    return n, d, t.stride(0) if n > 1 else max(t.stride(0), d)


class RowCodes:
    """Rows [n, d] as 8-bit codes with a scale each: what encode_rows() makes and matmul_i8() takes.  `blocks` int8 [ceil(n / 16), 2 ceil(d / 128), 4,
    16, 16] holds code k of row i at [i // 16, k // 64, k % 64 // 16, i % 16, k % 16] (features d on are 0), `scales` float32 [n]; a row reads
    back as codes * scale."""

    def __init__(self, blocks: torch.Tensor, scales: torch.Tensor, d: int):
        assert blocks.is_cuda and blocks.dtype is torch.int8 and blocks.is_contiguous(), "need blocks of device codes"
        assert scales.is_cuda and scales.dtype is torch.float32 and scales.is_contiguous() and scales.dim() == 1 and scales.device == blocks.device, \
            "need a float32 scale for each row, on the codes' device"
        assert d >= 1 and blocks.shape == self.shape(scales.shape[0], d), f"need blocks {self.shape(scales.shape[0], d)}"
        self.blocks, self.scales, self.d, self.n = blocks, scales, d, scales.shape[0]

    @staticmethod
    def shape(n: int, d: int):
        return -(-n // 16), 2 * -(-d // 128), 4, 16, 16

    @property
    def codes(self) -> torch.Tensor:
        """int8 [n, d], a copy."""
        rows = self.blocks.permute(0, 3, 1, 2, 4).reshape(16 * self.blocks.shape[0], -1)
        return rows[:self.n, :self.d].contiguous()

    def float(self) -> torch.Tensor:
        """The rows as they read back, float32 [n, d]."""
        return self.codes.float() * self.scales[:, None]


def encode_rows(x: torch.Tensor) -> RowCodes:
    """lpq_encode_rows of x [n, d] (float32, float16 or bfloat16): each row's largest magnitude becomes 127.  There is no way back through
    the codes: rows that require a gradient are refused."""
    _no_gradient("codes have no gradient", x)
    n, d, ld = _typed_matrix(x, "rows")
    assert lib().lpq_row_codes_bytes(n, d) > 0 or n == 0, f"rows of 1 to 131072 values, not {d}"
    with torch.cuda.device(x.device):
        out = RowCodes(torch.empty(RowCodes.shape(n, d), dtype=torch.int8, device=x.device), torch.empty(n, dtype=torch.float32, device=x.device), d)
        _check(lib().lpq_encode_rows(x.data_ptr(), ld, _TYPE[x.dtype], n, d, out.blocks.data_ptr(), out.scales.data_ptr(), _stream_of(x)))
    return out


def _bias(bias: torch.Tensor, n: int, device):
    if bias is None:
        return None
    assert bias.shape == (n,) and bias.device == device, f"need a bias [{n}] on the weights' device"
    return bias.detach().float().contiguous()


def matmul_i8(a: RowCodes, b: RowCodes, bias: torch.Tensor = None, dtype=torch.bfloat16, out: torch.Tensor = None) -> torch.Tensor:
    """[rows of a, rows of b] of `dtype`: the products of all rows of a with all rows of b (and bias, one for each row of b).  A bias that requires a
    gradient is refused."""
    _no_gradient("products of codes have no gradient", bias)
    assert a.d == b.d, f"rows of {a.d} and of {b.d} codes"
    assert a.blocks.device == b.blocks.device, "both on one device"
    if out is None:
        out = torch.empty((a.n, b.n), dtype=dtype, device=a.blocks.device)
    m, n, ldo = _typed_matrix(out, "an output")
    assert (m, n) == (a.n, b.n) and out.device == a.blocks.device, f"need an output [{a.n}, {b.n}] on the codes' device"
    bias = _bias(bias, n, a.blocks.device)
    with torch.cuda.device(out.device):
        ws, size = _scratch(lib().lpq_matmul_i8_workspace_bytes(m, n, a.d), out.device)
        _check(lib().lpq_matmul_i8(a.blocks.data_ptr(), a.scales.data_ptr(), m, b.blocks.data_ptr(), b.scales.data_ptr(), n, a.d, _ptr(bias),
                                   out.data_ptr(), ldo, _TYPE[out.dtype], _ptr(ws), size, _stream_of(out)))
    return out


def _scratch(need: int, device):
    return (None, 0) if need == 0 else (torch.empty(need, dtype=torch.uint8, device=device), need)


class Linear8:
    """lpq_linear8: y = x w^T + bias with w [channels, d] kept as 8-bit codes (a scale for each channel) and the rows of x made codes on
    the way (a scale for each row).  For serving: weight and bias are taken as they are now, inputs that require a gradient are refused."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor = None):
        self.weight = encode_rows(weight.detach())
        self.d, self.channels, self.device = self.weight.d, self.weight.n, weight.device
        self.bias = _bias(bias, self.channels, self.device)
        if bias is not None and self.bias.data_ptr() == bias.data_ptr():
            self.bias = self.bias.clone()                   # the layer's own, as its codes are
        torch.cuda.current_stream(self.device).synchronize()     # calls on any stream find the codes written
        self._args = self.weight.blocks.data_ptr(), self.weight.scales.data_ptr(), self.channels, self.d, _ptr(self.bias)

    def __call__(self, x: torch.Tensor, out: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
        """x [..., d] of float32, float16 or bfloat16 -> [..., channels] of its type."""
        _no_gradient("codes have no gradient", x)
        assert x.dim() >= 1 and x.shape[-1] == self.d and x.device == self.device, f"need [..., {self.d}] on {self.device}"
        rows = x if x.dim() == 2 else x.reshape(-1, self.d)
        m, _, ldx = _typed_matrix(rows, "rows")
        if out is None:
            out = x.new_empty((*x.shape[:-1], self.channels))
            ldo = self.channels
        else:
            assert out.shape == (*x.shape[:-1], self.channels) and out.dtype is x.dtype and out.device == x.device, "need an output of x's type and rows"
            _, _, ldo = _typed_matrix(out if out.dim() == 2 else out.view(-1, self.channels), "an output")
        if torch.cuda.current_device() != x.get_device():
            with torch.cuda.device(x.device):
                return self._run(rows, m, ldx, out, ldo, workspace)
        return self._run(rows, m, ldx, out, ldo, workspace)

    def _run(self, x, m, ldx, out, ldo, workspace):
        workspace, ws, size = KVCache._workspace(workspace, _lib.lpq_linear8_workspace_bytes(m, self.channels, self.d), x.device)
        _check(_lib.lpq_linear8(x.data_ptr(), ldx, _TYPE[x.dtype], m, *self._args, out.data_ptr(), ldo, ws, size, _stream_of(x)))
        return out


def rerank_f32(x: torch.Tensor, q: torch.Tensor, cand_ids: torch.Tensor, k: int, metric="l2sq"):
    """Exact re-rank of candidate lists int32 [nq, kc] on the fp32 vectors: (ids int32, dists fp32) [nq, k]."""
    xp, n, ldx = _dev_matrix(x, torch.float32)
    qp, nq, ldq = _dev_matrix(q, torch.float32)
    cp, nc, ldc = _dev_matrix(cand_ids, torch.int32)
    assert nc == nq and ldc == cand_ids.shape[1] and q.shape[1] == x.shape[1]
    ids = torch.empty((nq, k), dtype=torch.int32, device=x.device)
    dists = torch.empty((nq, k), dtype=torch.float32, device=x.device)
    _check(lib().lpq_rerank_f32(xp, n, ldx, qp, nq, ldq, x.shape[1], cp, cand_ids.shape[1], k, METRIC[metric],
                                ids.data_ptr(), dists.data_ptr(), _stream()))
    return ids, dists


def search_f32(x: torch.Tensor, q: torch.Tensor, k: int, metric="l2sq"):
    """Exact fp32 search: (ids int32, dists fp32) [nq, k]."""
    xp, n, ldx = _dev_matrix(x, torch.float32)
    qp, nq, ldq = _dev_matrix(q, torch.float32)
    d = x.shape[1]
    assert q.shape[1] == d
    ids = torch.empty((nq, k), dtype=torch.int32, device=x.device)
    dists = torch.empty((nq, k), dtype=torch.float32, device=x.device)
    need = lib().lpq_search_f32_workspace_bytes(n, nq, d, k)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
    _check(lib().lpq_search_f32(xp, n, ldx, qp, nq, ldq, d, k, METRIC[metric], ids.data_ptr(),
                                dists.data_ptr(), ws.data_ptr(), ws.numel(), _stream()))
    return ids, dists
