"""Thin ctypes binding of libsame_lda.so (argument marshalling only).

Every step of the sweep runs in the HIP library; this module converts Python objects to the
plain pointers of the C ABI.  PyTorch appears only as the owner of device memory and streams.
There is no fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import operator
import os
import struct
from ctypes import POINTER, Structure, byref, c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_uint32, c_uint64, c_void_p

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsame_lda.so")

THETA, PHI, NDK, NWK, NK = 0, 1, 2, 3, 4
# Tokens of a nonzero drawn as one multinomial (one task).  Large groups measure fastest (fewer tasks,
# and a nonzero's copies share one scan); m * min(count, this) must stay below 2^24.
DEFAULT_TOKENS_PER_DRAW = 1024
_DTYPES = {THETA: np.float32, PHI: np.float32, NDK: np.uint32, NWK: np.uint32, NK: np.uint64}

EXPORTS = ["same_lda_init", "same_lda_sweep", "same_lda_sweep_poisson", "same_lda_sweep_sampled", "same_lda_loglik", "same_lda_free",
           "same_lda_set_batch", "same_lda_stage_batch", "same_lda_commit_batch", "same_lda_debug_draw_poisson", "same_lda_sddmm",
           "same_lda_vb_exp_elog_beta", "same_lda_vb_estep",
           "same_lda_embed", "same_lda_embed_grad_workspace", "same_lda_embed_grad", "same_lda_dropout", "same_lda_embed_dropout", "same_lda_embed_dropout_grad_workspace", "same_lda_embed_dropout_grad",
           "same_lda_group_size", "same_lda_group_quantize", "same_lda_group_product_workspace", "same_lda_group_product", "same_lda_micro_size", "same_lda_micro_quantize", "same_lda_micro_product",
           "same_lda_get", "same_lda_set", "same_lda_get_pass", "same_lda_set_pass", "same_lda_task_count",
           "same_lda_debug_draw", "same_lda_debug_draw_noalloc", "same_lda_debug_chunk_limit", "same_lda_set_timing", "same_lda_get_timing", "same_lda_selftest",
           "same_lda_synchronize",
           "same_lda_last_error"]


class SameLdaError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"same_lda error {code}: {text}")
        self.code = code


class _Csc(Structure):
    _fields_ = [("D", c_int32), ("V", c_int32), ("nnz", c_int64), ("colptr", c_void_p),
                ("rowidx", c_void_p), ("val", c_void_p), ("on_device", c_int32)]


_lib = None


def load(path: str | None = None) -> ctypes.CDLL:
    """Loads the built library; raises if it is missing (build it with paper_1409_5402_amd.build).  `path` (or the
    environment variable SAME_LDA_LIB) names another build of the same library, e.g. the event-counting build of
    bench.py --mode stats; the first load of a process decides."""
    global _lib
    if _lib is None:
        path = path or os.environ.get("SAME_LDA_LIB") or LIB_PATH
        if not os.path.exists(path):
            raise FileNotFoundError(f"{path} is missing: run paper_1409_5402_amd.build.build() first")
        try:
            import torch  # noqa: F401  (where torch is installed, its HIP runtime must be the one loaded first:
        except ImportError:             # the library then binds to the same runtime as the tensors it is given)
            pass
        L = ctypes.CDLL(path)
        L.same_lda_init.argtypes = [POINTER(c_void_p), POINTER(_Csc), c_int32, c_float, c_float, c_uint64,
                                    c_int32, c_int32, c_void_p]
        L.same_lda_sweep.argtypes = [c_void_p, c_int32, c_float]
        L.same_lda_sweep_sampled.argtypes = [c_void_p, c_int32]
        L.same_lda_sweep_poisson.argtypes = [c_void_p, c_float, c_float]
        L.same_lda_debug_draw_poisson.argtypes = [c_void_p, c_float, c_void_p, c_int32, c_void_p]
        L.same_lda_loglik.argtypes = [c_void_p, POINTER(_Csc), c_int32, c_int32, POINTER(c_double)]
        L.same_lda_free.argtypes = [c_void_p]
        L.same_lda_free.restype = None
        L.same_lda_set_batch.argtypes = [c_void_p, POINTER(_Csc), c_int32]
        L.same_lda_stage_batch.argtypes = [c_void_p, POINTER(_Csc), c_int32, c_int32]
        L.same_lda_commit_batch.argtypes = [c_void_p]
        L.same_lda_get.argtypes = [c_void_p, c_int32, c_void_p, c_size_t, c_int32]
        L.same_lda_set.argtypes = [c_void_p, c_int32, c_void_p, c_size_t, c_int32]
        L.same_lda_get_pass.argtypes = [c_void_p, POINTER(c_int32)]
        L.same_lda_set_pass.argtypes = [c_void_p, c_int32]
        L.same_lda_task_count.argtypes = [c_void_p, POINTER(c_int64)]
        L.same_lda_debug_draw.argtypes = [c_void_p, c_int32, c_void_p, c_int32, c_void_p]
        L.same_lda_debug_draw_noalloc.argtypes = [c_void_p, c_int32, c_void_p, c_int32, c_void_p]
        L.same_lda_debug_chunk_limit.argtypes = [c_void_p, c_int64, POINTER(c_int64)]
        L.same_lda_sddmm.argtypes = [c_void_p, c_void_p, c_int32]
        L.same_lda_vb_exp_elog_beta.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p]
        L.same_lda_vb_estep.argtypes = [c_void_p, c_void_p, c_void_p, c_float, c_int32, c_void_p, c_void_p]
        L.same_lda_embed.argtypes = [c_void_p, c_void_p, c_int32, c_float, c_void_p, c_void_p]
        L.same_lda_embed_grad_workspace.argtypes = [c_void_p, c_void_p, POINTER(c_size_t)]
        L.same_lda_embed_grad.argtypes = [c_void_p, c_void_p, c_int32, c_float, c_int32, c_void_p, c_void_p, c_size_t, c_void_p]
        L.same_lda_dropout.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p]
        L.same_lda_embed_dropout.argtypes = [c_void_p, c_void_p, c_int32, c_float, c_void_p, c_void_p, c_void_p]
        L.same_lda_embed_dropout_grad_workspace.argtypes = [c_void_p, c_void_p, POINTER(c_size_t)]
        L.same_lda_embed_dropout_grad.argtypes = [c_void_p, c_void_p, c_int32, c_float, c_void_p, c_int32, c_void_p, c_void_p, c_size_t, c_void_p]
        L.same_lda_group_size.argtypes = [c_int64, c_int32, c_int32, POINTER(c_size_t), POINTER(c_size_t)]
        L.same_lda_group_quantize.argtypes = [c_void_p, c_void_p, c_void_p]
        L.same_lda_group_product_workspace.argtypes = [c_void_p, c_void_p, POINTER(c_size_t)]
        L.same_lda_group_product.argtypes = [c_void_p, c_void_p, c_float, c_void_p, c_void_p, c_size_t, c_void_p]
        L.same_lda_micro_size.argtypes = [c_int64, c_int32, POINTER(c_size_t), POINTER(c_size_t)]
        L.same_lda_micro_quantize.argtypes = [c_void_p, c_void_p, c_void_p]
        L.same_lda_micro_product.argtypes = [c_void_p, c_void_p, c_float, c_void_p, c_void_p]
        L.same_lda_set_timing.argtypes = [c_void_p, c_int32]
        L.same_lda_get_timing.argtypes = [c_void_p, POINTER(c_double), POINTER(c_int64)]
        L.same_lda_selftest.argtypes = [POINTER(c_int64)]
        L.same_lda_synchronize.argtypes = [c_void_p]
        L.same_lda_last_error.argtypes = [c_void_p]
        L.same_lda_last_error.restype = c_char_p
        for name in EXPORTS:
            if name not in ("same_lda_free", "same_lda_last_error"):
                getattr(L, name).restype = c_int32
        _lib = L
    return _lib


def _is_torch(x) -> bool:
    return type(x).__module__.startswith("torch")


def _csc(D, V, colptr, rowidx, val):
    """Builds the C view of a matrix from three numpy arrays (host) or three torch tensors."""
    keep = []
    if _is_torch(colptr):
        import torch
        dev = colptr.device
        arrs = []
        for a, dt in ((colptr, torch.int32), (rowidx, torch.int32), (val, torch.float32)):
            a = a.to(dtype=dt).contiguous()
            assert a.device == dev
            arrs.append(a)
        keep = arrs
        ptrs = [a.data_ptr() if a.numel() else None for a in arrs]
        on_device = 1 if dev.type == "cuda" else 0
        nnz = int(arrs[1].numel())
    else:
        arrs = [np.ascontiguousarray(colptr, np.int32), np.ascontiguousarray(rowidx, np.int32),
                np.ascontiguousarray(val, np.float32)]
        keep = arrs
        ptrs = [a.ctypes.data if a.size else None for a in arrs]
        on_device = 0
        nnz = int(arrs[1].size)
    c = _Csc(int(D), int(V), nnz, ptrs[0], ptrs[1], ptrs[2], on_device)
    return c, keep


def selftest() -> int:
    """Runs the library's device self-test; returns the number of mismatches (0 = pass)."""
    L = load()
    n = c_int64()
    rc = L.same_lda_selftest(byref(n))
    if rc != 0:
        raise SameLdaError(rc, L.same_lda_last_error(None).decode())
    return n.value


class SameLDA:
    """A SAME Gibbs LDA model resident on the current GPU (one handle of the C library)."""

    def __init__(self, D, V, colptr, rowidx, val, K, alpha, beta, seed, m0, tokens_per_draw=DEFAULT_TOKENS_PER_DRAW, stream=None):
        self._lib = load()
        self._h = c_void_p()
        self.V, self.K, self.D = int(V), int(K), int(D)
        self.nnz = int(rowidx.shape[0])
        if stream is None:
            try:
                import torch
                stream = torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
            except ImportError:
                stream = 0
        c, keep = _csc(D, V, colptr, rowidx, val)
        rc = self._lib.same_lda_init(byref(self._h), byref(c), int(K), float(alpha), float(beta), int(seed),
                                     int(m0), int(tokens_per_draw), c_void_p(stream or None))
        del keep
        if rc != 0:
            raise SameLdaError(rc, self._lib.same_lda_last_error(None).decode())

    def _check(self, rc):
        if rc != 0:
            raise SameLdaError(rc, self._lib.same_lda_last_error(self._h).decode())

    def sweep(self, m, rho=1.0):
        self._check(self._lib.same_lda_sweep(self._h, int(m), float(rho)))

    def sweep_sampled(self, m):
        self._check(self._lib.same_lda_sweep_sampled(self._h, int(m)))

    def sweep_poisson(self, m, rho=1.0):
        self._check(self._lib.same_lda_sweep_poisson(self._h, float(m), float(rho)))

    def set_batch(self, D, colptr, rowidx, val, m_init):
        c, keep = _csc(D, self.V, colptr, rowidx, val)
        self._check(self._lib.same_lda_set_batch(self._h, byref(c), int(m_init)))
        self.D, self.nnz = int(D), int(rowidx.shape[0])
        del keep

    def stage_batch(self, D, colptr, rowidx, val, m_init, sweeps_ahead=0):
        c, keep = _csc(D, self.V, colptr, rowidx, val)
        self._check(self._lib.same_lda_stage_batch(self._h, byref(c), int(m_init), int(sweeps_ahead)))
        self._staged_D, self._staged_nnz = int(D), int(rowidx.shape[0])
        del keep

    def commit_batch(self):
        self._check(self._lib.same_lda_commit_batch(self._h))
        self.D, self.nnz = self._staged_D, self._staged_nnz

    def loglik(self, D, colptr, rowidx, val, foldin_sweeps, m_eval) -> float:
        c, keep = _csc(D, self.V, colptr, rowidx, val)
        out = c_double()
        self._check(self._lib.same_lda_loglik(self._h, byref(c), int(foldin_sweeps), int(m_eval), byref(out)))
        del keep
        return out.value

    def _shape(self, which):
        return {THETA: (self.D, self.K), PHI: (self.V, self.K), NDK: (self.D, self.K),
                NWK: (self.V, self.K), NK: (self.K,)}[which]

    def get(self, which, out=None):
        """A state matrix as a numpy array; ``out``: a contiguous torch tensor of its shape and type (float32 for THETA and
        PHI, int32 for NDK and NWK, int64 for NK) that is filled instead, on the host or the device."""
        if out is not None:
            import torch
            dtype = {np.float32: torch.float32, np.uint32: torch.int32, np.uint64: torch.int64}[_DTYPES[which]]
            if tuple(out.shape) != self._shape(which) or out.dtype != dtype or not out.is_contiguous():
                raise ValueError(f"out must be a contiguous {dtype} tensor of shape {self._shape(which)}")
            nbytes = out.numel() * out.element_size()
            on_device = out.device.type == "cuda"
            torch.autograd.graph.increment_version(out)                 # autograd may have kept what it held
            if on_device:
                torch.cuda.current_stream(out.device).synchronize()     # what is still being done to out ends first
            self._check(self._lib.same_lda_get(self._h, which, out.data_ptr() if nbytes else None, nbytes, 1 if on_device else 0))
            return out
        out = np.empty(self._shape(which), dtype=_DTYPES[which])
        self._check(self._lib.same_lda_get(self._h, which, out.ctypes.data if out.size else None, out.nbytes, 0))
        return out

    def set(self, which, arr):
        """arr: a numpy array (host) or a torch tensor (host or device) of the matrix' shape and dtype."""
        if _is_torch(arr):
            import torch
            t = arr.contiguous()
            assert tuple(t.shape) == self._shape(which) and t.dtype == torch.float32
            nbytes = t.numel() * t.element_size()
            self._check(self._lib.same_lda_set(self._h, which, t.data_ptr() if nbytes else None, nbytes,
                                               1 if t.device.type == "cuda" else 0))
            return
        a = np.ascontiguousarray(arr, dtype=_DTYPES[which])
        assert a.shape == self._shape(which)
        self._check(self._lib.same_lda_set(self._h, which, a.ctypes.data if a.size else None, a.nbytes, 0))

    @property
    def pass_index(self) -> int:
        v = c_int32()
        self._check(self._lib.same_lda_get_pass(self._h, byref(v)))
        return v.value

    @pass_index.setter
    def pass_index(self, v):
        self._check(self._lib.same_lda_set_pass(self._h, int(v)))

    @property
    def task_count(self) -> int:
        v = c_int64()
        self._check(self._lib.same_lda_task_count(self._h, byref(v)))
        return v.value

    def debug_draw(self, m, task_ids) -> np.ndarray:
        ids = np.ascontiguousarray(task_ids, np.int64)
        out = np.zeros((ids.shape[0], self.K), np.uint32)
        self._check(self._lib.same_lda_debug_draw(self._h, int(m), ids.ctypes.data if ids.size else None,
                                                  ids.shape[0], out.ctypes.data if out.size else None))
        return out

    def debug_draw_noalloc(self, m, task_ids) -> np.ndarray:
        ids = np.ascontiguousarray(task_ids, np.int64)
        out = np.zeros((ids.shape[0], self.K), np.uint32)
        self._check(self._lib.same_lda_debug_draw_noalloc(self._h, int(m), ids.ctypes.data if ids.size else None,
                                                          ids.shape[0], out.ctypes.data if out.size else None))
        return out

    def debug_chunk_limit(self, max_chunks: int = -1) -> int:
        """Chunks of the pair-list pool the sweeps may use from now on (negative: all); returns the number in use."""
        n = c_int64(0)
        self._check(self._lib.same_lda_debug_chunk_limit(self._h, int(max_chunks), ctypes.byref(n)))
        return int(n.value)

    def debug_draw_poisson(self, m, task_ids) -> np.ndarray:
        ids = np.ascontiguousarray(task_ids, np.int64)
        out = np.zeros((ids.shape[0], self.K), np.uint32)
        self._check(self._lib.same_lda_debug_draw_poisson(self._h, float(m), ids.ctypes.data if ids.size else None,
                                                          ids.shape[0], out.ctypes.data if out.size else None))
        return out

    def sddmm(self, out=None):
        """mu of every nonzero of the resident matrix; ``out``: a float32 torch tensor on the device (filled
        asynchronously) or None (a numpy array is returned)."""
        if out is not None:
            self._check(self._lib.same_lda_sddmm(self._h, out.data_ptr(), 1))
            return out
        mu = np.zeros(self.nnz, np.float32)
        self._check(self._lib.same_lda_sddmm(self._h, mu.ctypes.data if mu.size else None, 0))
        return mu

    def vb_exp_elog_beta(self, lam, b_out, shift_out):
        """Rows of exp E[log beta] of lambda divided by their largest entry (b_out [V][K]) and the logarithm of that
        entry (shift_out [V]); all float32 torch tensors on the device; asynchronous."""
        self._check(self._lib.same_lda_vb_exp_elog_beta(self._h, lam.data_ptr(), b_out.data_ptr(), shift_out.data_ptr()))
        return b_out, shift_out

    def vb_estep(self, b, shift, alpha: float, iters: int, gamma, log_mu=None):
        """`iters` iterations of the variational E-step on the resident matrix; b [V][K], shift [V] (or None),
        gamma [D][K] (updated in place) and log_mu [nnz] (optional) are float32 torch tensors on the device;
        asynchronous."""
        self._check(self._lib.same_lda_vb_estep(self._h, b.data_ptr(), shift.data_ptr() if shift is not None else None,
                                                float(alpha), int(iters), gamma.data_ptr(),
                                                log_mu.data_ptr() if log_mu is not None else None))
        return gamma

    def set_timing(self, enabled: bool):
        self._check(self._lib.same_lda_set_timing(self._h, 1 if enabled else 0))

    def get_timing(self):
        ms, n = c_double(), c_int64()
        self._check(self._lib.same_lda_get_timing(self._h, byref(ms), byref(n)))
        return ms.value, n.value

    def synchronize(self):
        self._check(self._lib.same_lda_synchronize(self._h))

    def close(self):
        if self._h:
            self._lib.same_lda_free(self._h)
            self._h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- Word tables as an embedding.  These functions take torch tensors on one GPU, run on torch's current stream of that
# GPU and return at once; what a call allocates (outputs, scratch) comes from torch's allocator.  Nothing is recorded for torch's
# autograd: embed_grad is the backward pass of embed.  A call's own time on the host counts where tokens come one by one, so
# operands are checked and passed on in few steps.

MICRO = 3
_pack_rows = struct.Struct("PPqqii").pack          # same_lda_rows, passed by the address of its bytes
_pack_drop = struct.Struct("dQQP").pack            # same_lda_drop
_torch = None
_types = {}                                        # element types by torch's
_library = None


def _setup():
    """torch and the library, at the first call of an operator."""
    global _torch, _types, _library
    import torch
    _types = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    _library = load()
    _torch = torch


class MicroMatrix:
    """A matrix in microscaled four-bit floating point: ``codes`` [rows, 64 * g] and ``scales`` [rows, 4 * g], contiguous
    uint8 tensors on one GPU with g = ceil(width / 128), in the layout that include/same_lda.h describes."""

    __slots__ = ("codes", "scales", "width", "rows")

    def __init__(self, codes, scales, width):
        if _torch is None:
            _setup()
        width = int(width)
        groups = -(-width // 128)
        rows = codes.shape[0]
        if (width < 1 or codes.dtype != _torch.uint8 or scales.dtype != _torch.uint8 or codes.shape != (rows, 64 * groups)
                or scales.shape != (rows, 4 * groups) or not codes.is_contiguous() or not scales.is_contiguous() or codes.device != scales.device):
            raise ValueError(f"rows of {width} elements need contiguous uint8 codes [rows, {64 * groups}] and scales [rows, {4 * groups}] on one device")
        self.codes, self.scales, self.width, self.rows = codes, scales, width, rows

    @property
    def shape(self):
        return (self.rows, self.width)

    @property
    def device(self):
        return self.codes.device

    def get_device(self):
        return self.codes.get_device()

    def __getitem__(self, rows):
        """A range of rows (a slice without a step), not copied."""
        if not isinstance(rows, slice) or rows.step not in (None, 1):
            raise TypeError("a microscaled matrix is sliced by ranges of rows")
        return MicroMatrix(self.codes[rows], self.scales[rows], self.width)


class GroupMatrix:
    """A matrix in grouped four-bit integers, q s + b: ``codes`` [rows, 64 * g] in uint8 and ``scales`` [rows, 128 * g / group, 2] in
    bfloat16 (s and b of every group of `group` = 32, 64 or 128 elements), contiguous tensors on one GPU with g = ceil(width / 128), in
    the layout that include/same_lda.h describes."""

    __slots__ = ("codes", "scales", "width", "group", "rows")

    def __init__(self, codes, scales, width, group):
        if _torch is None:
            _setup()
        width, group = int(width), int(group)
        if group not in (32, 64, 128):
            raise ValueError(f"groups hold 32, 64 or 128 elements, not {group}")
        blocks = -(-width // 128)
        rows, n = codes.shape[0], blocks * (128 // group)
        if (width < 1 or codes.dtype != _torch.uint8 or scales.dtype != _torch.bfloat16 or codes.shape != (rows, 64 * blocks) or scales.shape != (rows, n, 2)
                or not codes.is_contiguous() or not scales.is_contiguous() or codes.device != scales.device):
            raise ValueError(f"rows of {width} elements in groups of {group} need contiguous uint8 codes [rows, {64 * blocks}] and bfloat16 scales [rows, {n}, 2] on one device")
        self.codes, self.scales, self.width, self.group, self.rows = codes, scales, width, group, rows

    @property
    def shape(self):
        return (self.rows, self.width)

    @property
    def device(self):
        return self.codes.device

    def get_device(self):
        return self.codes.get_device()

    def __getitem__(self, rows):
        """A range of rows (a slice without a step), not copied."""
        if not isinstance(rows, slice) or rows.step not in (None, 1):
            raise TypeError("a grouped matrix is sliced by ranges of rows")
        return GroupMatrix(self.codes[rows], self.scales[rows], self.width, self.group)


_CODED = (MicroMatrix, GroupMatrix)


class Dropout:
    """Which elements of a matrix are kept: each with probability 1 - p, by its place, the seed and the step alone, so a backward pass that is
    given the same Dropout repeats the forward pass's choice.  `step`: an integer in [0, 2^56), another one for every call whose
    choice is to be another; or a tensor of one int64 element on the GPU, read when the kernel runs (a captured graph that counts it up
    draws anew in every replay).  p, seed and step stay what they are: another step in a number is another Dropout."""

    __slots__ = ("_p", "_seed", "_step", "_packed")

    def __init__(self, p, seed, step=0):
        p = float(p)
        if not 0.0 <= p <= 1.0:
            raise ValueError(f"the probability {p} is not in [0, 1]")
        seed = operator.index(seed)
        if not 0 <= seed < 1 << 64:
            raise ValueError(f"the seed {seed} is not in [0, 2^64)")
        self._p, self._seed, self._step, self._packed = p, seed, step, None
        if _is_torch(step):
            self._pack()
        else:
            count = operator.index(step)
            if not 0 <= count < 1 << 56:
                raise ValueError(f"the step {count} is not in [0, 2^56)")
            self._packed = _pack_drop(p, seed, count, 0)

    p = property(lambda self: self._p)
    seed = property(lambda self: self._seed)
    step = property(lambda self: self._step)

    def _pack(self) -> bytes:
        """As a same_lda_drop.  A step in a tensor is looked at in every call: its memory may be another one than before."""
        if self._packed is not None:
            return self._packed
        import torch
        step = self._step
        if step.numel() != 1 or step.dtype != torch.int64:
            raise TypeError(f"a step in a tensor is one int64 element, not {step.numel()} of {step.dtype}")
        return _pack_drop(self._p, self._seed, 0, step.data_ptr())

    def _on(self):
        """The operand among a call's that must be on its GPU: the step's tensor, if it is one."""
        return None if self._packed is not None else self._step


def _drop(drop) -> bytes:
    if type(drop) is not Dropout:
        raise TypeError(f"drop is a Dropout, not a {type(drop).__name__}")
    return drop._pack()


def _type_of(dtype) -> int:
    kind = _types.get(dtype)
    if kind is None:
        raise TypeError(f"{dtype} is not one of float32, bfloat16 and float16")
    return kind


def _rows(x) -> bytes:
    """A matrix as a same_lda_rows."""
    if type(x) is MicroMatrix:
        return _pack_rows(x.codes.data_ptr(), x.scales.data_ptr(), x.rows, x.width, x.width, MICRO)
    if type(x) is GroupMatrix:
        return _pack_rows(x.codes.data_ptr(), x.scales.data_ptr(), x.rows, x.width, x.width, x.group)
    kind = _type_of(x.dtype)
    if x.dim() != 2:
        raise ValueError(f"a matrix has two dimensions, not {x.dim()}")
    rows, width = x.shape
    stride, inner = x.stride()
    if inner != 1 and width > 1 or stride < width and rows > 1:
        raise ValueError("the elements of a row must be contiguous and rows must not overlap")
    return _pack_rows(x.data_ptr(), 0, rows, stride if rows > 1 else width, width, kind)


def _not_micro(name, x):
    return TypeError(f"{name} is a MicroMatrix (micro_quantize makes one), not a {type(x).__name__}")


def _gpu(*operands) -> int:
    """The number of the GPU that all operands are on."""
    index = operands[0].get_device()
    for x in operands:
        if x is not None and (x.get_device() != index or index < 0):
            raise ValueError(f"all operands must be on one GPU (got {[str(y.device) for y in operands if y is not None]})")
    return index


def _run(index, call, *arguments):
    """One call of the library on torch's stream of GPU `index`, which is the current one meanwhile."""
    if _torch._C._cuda_getDevice() == index:
        rc = call(*arguments, _torch._C._cuda_getCurrentRawStream(index))
    else:
        with _torch.cuda.device(index):
            rc = call(*arguments, _torch._C._cuda_getCurrentRawStream(index))
    if rc != 0:
        raise SameLdaError(rc, _library.same_lda_last_error(None).decode())


def _token_ids(tokens):
    if _torch is None:
        _setup()
    if tokens.dtype is not _torch.int64 and tokens.dtype is not _torch.int32:
        raise TypeError(f"tokens are int32 or int64, not {tokens.dtype}")
    return tokens if tokens.is_contiguous() else tokens.contiguous()


def _rewritten(out):
    """Tells autograd, as torch's own in-place operations do, that `out` will not hold what it may have kept of it for a backward pass."""
    _torch.autograd.graph.increment_version(out)


def _output(out, shape, rows, width, dtype, default, device):
    """The output of a call, made here where none is given, and its same_lda_rows as `rows` rows of `width`."""
    if out is None:
        kind = _type_of(dtype or default)
        out = _torch.empty(shape, dtype=dtype or default, device=device)
        return out, _pack_rows(out.data_ptr(), 0, rows, width, width, kind)
    if type(out) in _CODED:
        raise TypeError(f"out is a tensor, not a {type(out).__name__}")
    if out.shape != shape or (dtype is not None and out.dtype != dtype):
        raise ValueError(f"out has shape {tuple(out.shape)} and type {out.dtype}, not {tuple(shape)} and {dtype or out.dtype}")
    _rewritten(out)
    return out, _rows(out if out.dim() == 2 else out.view(-1, width))


def embed(table, tokens, scale=1.0, dtype=None, out=None, drop=None):
    """scale * table[tokens]: the rows of `table` (a matrix, a MicroMatrix or a GroupMatrix) for int32 or int64 `tokens` of any shape, in
    `dtype` (default: the table's, float32 for one in four bits).  An id outside the table (padding) gives zeros.  `drop`: a Dropout of the
    result, whose row i is that of the i-th token.  `out`: a tensor of
    shape tokens.shape + (width,) whose leading dimensions can be viewed as one.  The result has no gradient function, also of a table that
    requires a gradient: a step calls embed_grad for it."""
    ids = _token_ids(tokens)
    index = _gpu(ids, table, out)
    t, n, width = _rows(table), ids.numel(), table.shape[1]
    if drop is not None:
        d = _drop(drop)
        _gpu(ids, drop._on())
    out, o = _output(out, (*tokens.shape, width), n, width, dtype, _torch.float32 if type(table) in _CODED else table.dtype, ids.device)
    if drop is None:
        _run(index, _library.same_lda_embed, t, ids.data_ptr() if n else _EMPTY, ids.element_size(), scale, o)
    else:
        _run(index, _library.same_lda_embed_dropout, t, ids.data_ptr() if n else _EMPTY, ids.element_size(), scale, d, o)
    return out


def dropout(x, drop, dtype=None, out=None):
    """x / (1 - p) where `drop` (a Dropout) keeps an element, else 0, for a tensor of one dimension or more as the matrix of its last dimension's
    rows; in `dtype` (default: x's).  The gradient is the same call on the result's gradient.  `out` may be x itself; its leading
    dimensions can be viewed as one.  For autograd the result is a constant."""
    if _torch is None:
        _setup()
    if type(x) in _CODED:
        raise TypeError(f"x is a tensor, not a {type(x).__name__}")
    d = _drop(drop)
    if not x.dim() or not x.shape[-1]:
        raise ValueError(f"x has shape {tuple(x.shape)}, which holds no rows")
    index = _gpu(x, out, drop._on())
    width = x.shape[-1]
    flat, r = _flat_rows(x, x.numel() // width, width)
    out, o = _output(out, x.shape, x.numel() // width, width, dtype, x.dtype, x.device)
    _run(index, _library.same_lda_dropout, r, d, o)
    return out


def _flat_rows(x, rows, width):
    """x as a matrix and its same_lda_rows, copied where its rows are not contiguous or share memory (an expanded tensor)."""
    flat = x if x.dim() == 2 else x.reshape(rows, width)
    try:
        return flat, _rows(flat)
    except ValueError:
        flat = flat.contiguous()
        return flat, _rows(flat)


_EMPTY = 16        # stands for the address of a list of no tokens: not null, never read


def embed_grad(grad, tokens, rows=None, scale=1.0, dtype=None, out=None, accumulate=False, drop=None):
    """The gradient of ``embed(table, tokens, scale)`` with respect to a table of `rows` rows, from that of its result: `grad`
    of shape tokens.shape + (width,), copied first where its rows are not contiguous or share memory (an expanded tensor).  `dtype` (default: grad's) is the result's type.  `out`: where it is written, or added to with
    ``accumulate=True``; `rows` is then out's.  `drop`: the Dropout of the lookup.  Equal numbers of
    one type and shape give equal bits, whatever their strides."""
    ids = _token_ids(tokens)
    if type(grad) in _CODED:
        raise TypeError(f"grad is a tensor, not a {type(grad).__name__}")
    shape = grad.shape
    if not shape or shape[:-1] != tokens.shape:
        raise ValueError(f"grad has shape {tuple(grad.shape)}, tokens {tuple(tokens.shape)}")
    if out is None and (accumulate or rows is None):
        raise ValueError("accumulate needs out" if accumulate else "rows or out must say how many rows the table has")
    index = _gpu(ids, grad, out)
    if drop is not None:
        d = _drop(drop)
        _gpu(ids, drop._on())
    width = shape[-1]
    rows = out.shape[0] if rows is None else int(rows)
    flat, g = _flat_rows(grad, ids.numel(), width)
    out, o = _output(out, (rows, width), rows, width, dtype, grad.dtype, ids.device)
    n = c_size_t()
    if (_library.same_lda_embed_grad_workspace if drop is None else _library.same_lda_embed_dropout_grad_workspace)(g, o, byref(n)):
        raise SameLdaError(-1, _library.same_lda_last_error(None).decode())
    space = _torch.empty(n.value, dtype=_torch.uint8, device=ids.device) if n.value else None
    t, at = ids.data_ptr() if ids.numel() else _EMPTY, space.data_ptr() if n.value else None
    if drop is None:
        _run(index, _library.same_lda_embed_grad, g, t, ids.element_size(), scale, 1 if accumulate else 0, o, at, n.value)
    else:
        _run(index, _library.same_lda_embed_dropout_grad, g, t, ids.element_size(), scale, d, 1 if accumulate else 0, o, at, n.value)
    return out


def micro_quantize(x, out=None) -> MicroMatrix:
    """A matrix in microscaled four-bit floating point (for autograd a constant)."""
    if _torch is None:
        _setup()
    if type(x) in _CODED:
        raise TypeError(f"x is a tensor, not a {type(x).__name__}")
    index = _gpu(x, out)
    r = _rows(x)
    if out is None:
        rows, width = x.shape
        groups = -(-width // 128)
        device = x.device
        out = MicroMatrix.__new__(MicroMatrix)
        out.codes = _torch.empty((rows, 64 * groups), dtype=_torch.uint8, device=device)
        out.scales = _torch.empty((rows, 4 * groups), dtype=_torch.uint8, device=device)
        out.width, out.rows = width, rows
    elif type(out) is not MicroMatrix:
        raise TypeError("out is a MicroMatrix")
    else:
        _rewritten((out.codes, out.scales))
    _run(index, _library.same_lda_micro_quantize, r, _rows(out))
    return out


def micro_dequantize(q, dtype=None, out=None):
    """The numbers that a MicroMatrix stands for, in `dtype` (default: float32; for autograd a constant)."""
    if type(q) is not MicroMatrix:
        raise _not_micro("q", q)
    index = _gpu(q, out)
    out, o = _output(out, q.shape, q.rows, q.width, dtype, _torch.float32, q.codes.device)
    _run(index, _library.same_lda_embed, _rows(q), None, 8, 1.0, o)
    return out


def _rounded_in_the_call(a, b) -> bool:
    """Whether micro_product leaves the rounding of a matrix to the library's call: one launch in place of two, where it takes
    the rows, and above 16 of them by tables that are small (us in the call and before it: 32 x 2000 x 256 7.2, 15.1;
    64 x 60,000 x 256 12.6, 14.8; 64 x 70,000 x 256 13.2, 14.8; 64 x 100,000 x 256 18.1, 14.8; 17 x 50,000 x 900 13.1, 14.7)."""
    rows = a.shape[0]
    return rows <= 64 and a.numel() <= 16384 and (rows <= 16 or -(-rows // 16) * b.rows * b.width <= 1 << 26)


def micro_product(a, b, scale=1.0, dtype=None, out=None):
    """scale * a @ b.T in `dtype` (default: float32) for a MicroMatrix `b`; `a` is a MicroMatrix, or a matrix that is rounded to
    one first.  The result has no gradient function, also where `a` requires a gradient."""
    if type(b) is not MicroMatrix:
        raise _not_micro("b", b)
    if type(a) is GroupMatrix:
        raise TypeError("a is a tensor or a MicroMatrix, not a GroupMatrix")
    if type(a) is not MicroMatrix and not _rounded_in_the_call(a, b):
        a = micro_quantize(a)
    index = _gpu(a, b, out)
    x, rows = _rows(a), a.shape[0]
    out, o = _output(out, (rows, b.rows), rows, b.rows, dtype, _torch.float32, b.codes.device)
    _run(index, _library.same_lda_micro_product, x, _rows(b), scale, o)
    return out


def group_quantize(x, group=64, out=None) -> GroupMatrix:
    """A matrix in grouped four-bit integers, with a step and a base for every `group` = 32, 64 or 128 elements of a row (for
    autograd a constant).  `out`: a GroupMatrix that is written; the group is then out's."""
    if _torch is None:
        _setup()
    if type(x) in _CODED:
        raise TypeError(f"x is a tensor, not a {type(x).__name__}")
    index = _gpu(x, out)
    r = _rows(x)
    if out is None:
        if group not in (32, 64, 128):
            raise ValueError(f"groups hold 32, 64 or 128 elements, not {group}")
        rows, width = x.shape
        blocks = -(-width // 128)
        device = x.device
        out = GroupMatrix.__new__(GroupMatrix)
        out.codes = _torch.empty((rows, 64 * blocks), dtype=_torch.uint8, device=device)
        out.scales = _torch.empty((rows, blocks * (128 // group), 2), dtype=_torch.bfloat16, device=device)
        out.width, out.group, out.rows = width, int(group), rows
    elif type(out) is not GroupMatrix:
        raise TypeError("out is a GroupMatrix")
    else:
        _rewritten((out.codes, out.scales))
    _run(index, _library.same_lda_group_quantize, r, _rows(out))
    return out


def group_dequantize(q, dtype=None, out=None):
    """The numbers that a GroupMatrix stands for, in `dtype` (default: float32; for autograd a constant)."""
    if type(q) is not GroupMatrix:
        raise TypeError(f"q is a GroupMatrix (group_quantize makes one), not a {type(q).__name__}")
    index = _gpu(q, out)
    out, o = _output(out, q.shape, q.rows, q.width, dtype, _torch.float32, q.codes.device)
    _run(index, _library.same_lda_embed, _rows(q), None, 8, 1.0, o)
    return out


def group_product(a, b, scale=1.0, dtype=None, out=None):
    """scale * a @ b.T in `dtype` (default: a's) for a GroupMatrix `b` and a matrix `a`, which is not rounded.  The result has no
    gradient function, also where `a` requires a gradient."""
    if type(b) is not GroupMatrix:
        raise TypeError(f"b is a GroupMatrix (group_quantize makes one), not a {type(b).__name__}")
    if type(a) in _CODED:
        raise TypeError(f"a is a tensor, not a {type(a).__name__}")
    index = _gpu(a, b, out)
    x, rows = _rows(a), a.shape[0]
    out, o = _output(out, (rows, b.rows), rows, b.rows, dtype, a.dtype, b.codes.device)
    t, space, size = _rows(b), None, 0
    if rows > 16 or b.width > 4096:                    # fewer and shorter rows need none
        n = c_size_t()
        if _library.same_lda_group_product_workspace(x, t, byref(n)):
            raise SameLdaError(-1, _library.same_lda_last_error(None).decode())
        size = n.value
        space = _torch.empty(size, dtype=_torch.uint8, device=b.codes.device) if size else None
    _run(index, _library.same_lda_group_product, x, t, scale, o, space.data_ptr() if size else None, size)
    return out
