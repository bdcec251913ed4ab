"""ctypes binding of include/lshbeam.h.  Argument marshalling only."""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "liblshbeam.so")

LSH_F32, LSH_BF16, LSH_F16 = 0, 1, 2
NUM_KERNELS = 5

# every symbol include/lshbeam.h declares
EXPORTED_SYMBOLS = (
    "lsh_build_tables", "lsh_free_tables", "lsh_step_workspace_bytes", "lsh_decode_step",
    "lsh_debug_codes", "lsh_debug_embedding_codes", "lsh_debug_bucket", "lsh_debug_csr",
    "lsh_debug_cuckoo_shape", "lsh_debug_candidates", "lsh_debug_logprobs", "lsh_profiler_create",
    "lsh_profiler_destroy", "lsh_profiler_read", "lsh_decode_step_timed", "lsh_kernel_name",
    "lsh_status_string", "lsh_step_is_fused", "lsh_debug_build_info", "lsh_beam_advance",
    "lsh_beam_backtrace", "lsh_set_option", "lsh_get_option", "lsh_decode_step_static",
    "lsh_static_scratch_bytes", "lsh_debug_counts", "lsh_release_kept",
    "lsh_select_workspace_bytes", "lsh_beam_select", "lsh_cache_workspace_bytes", "lsh_cache_advance", "lsh_cache_write",
    "lsh_attention_workspace_bytes", "lsh_cache_attention",
)

OPTION_AUTO = -1
OPTION_NAMES = ("fused", "fused_grid", "logits_grid", "logits_waves", "logits_hlds", "logits_estage",
                "hlds_rem", "logits_planes", "hlds_rows", "part_rows", "stage_rows", "one_launch", "fused_tile",
                "estage_union", "first_tiles")


class LshBeamError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {_status_string(status)} (status {status})")


class BuildParams(ctypes.Structure):
    _fields_ = [("V", ctypes.c_int32), ("d", ctypes.c_int32), ("ld_e", ctypes.c_int64),
                ("e_dtype", ctypes.c_int32), ("K", ctypes.c_int32), ("P", ctypes.c_int32),
                ("bands", ctypes.c_int32), ("seed", ctypes.c_uint64)]


class BeamParams(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int32), ("B", ctypes.c_int32), ("n_states", ctypes.c_int32),
                ("state_dim", ctypes.c_int32), ("eos", ctypes.c_int32), ("max_len", ctypes.c_int32)]


class StepParams(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int32), ("B", ctypes.c_int32), ("T", ctypes.c_int32),
                ("threshold", ctypes.c_int32), ("full_vocab", ctypes.c_int32)]


class SelectParams(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int32), ("B", ctypes.c_int32), ("N", ctypes.c_int32), ("V", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("ld", ctypes.c_int64), ("allowed_ld", ctypes.c_int64)]


class CacheParams(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int32), ("B", ctypes.c_int32), ("n_blocks", ctypes.c_int32), ("block", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class AttentionParams(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("causal", ctypes.c_int32), ("window", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class _PoolPointers(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class _Rows(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("row", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load liblshbeam.so (built in-tree by `python -m paper_1806_00588_amd.build`).  Raises if
    it is missing: there is no fallback implementation."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} not found: build it with `python -m paper_1806_00588_amd.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    i32p = ctypes.POINTER(ctypes.c_int32)
    lib.lsh_build_tables.argtypes = [vp, vp, ctypes.POINTER(BuildParams), vp, ctypes.POINTER(vp)]
    lib.lsh_free_tables.argtypes = [vp]
    lib.lsh_free_tables.restype = None
    lib.lsh_release_kept.argtypes = []
    lib.lsh_release_kept.restype = None
    lib.lsh_step_workspace_bytes.argtypes = [vp, ctypes.POINTER(StepParams)]
    lib.lsh_step_workspace_bytes.restype = sz
    lib.lsh_decode_step.argtypes = [vp, vp, vp, vp, ctypes.POINTER(StepParams), vp, sz, vp, vp, vp, vp]
    lib.lsh_debug_codes.argtypes = [vp, vp, i32, i32p]
    lib.lsh_debug_embedding_codes.argtypes = [vp, i32, i32, i32p]
    lib.lsh_debug_bucket.argtypes = [vp, i32, i32, i32p, i32, i32p]
    lib.lsh_debug_csr.argtypes = [vp, i32, i32p, i32p, i32p, i32, i32p]
    lib.lsh_debug_cuckoo_shape.argtypes = [vp, i32, i32p, i32p]
    lib.lsh_debug_build_info.argtypes = [vp, i32p, i32p]
    lib.lsh_beam_advance.argtypes = [ctypes.POINTER(BeamParams), i32, vp, vp, vp, ctypes.POINTER(vp),
                                     ctypes.POINTER(vp), vp, vp, vp, vp, vp]
    lib.lsh_beam_advance.restype = i32
    lib.lsh_beam_backtrace.argtypes = [ctypes.POINTER(BeamParams), i32, vp, vp, vp, vp, vp, vp, vp]
    lib.lsh_beam_backtrace.restype = i32
    lib.lsh_debug_build_info.restype = i32
    lib.lsh_debug_candidates.argtypes = [vp, vp, ctypes.POINTER(StepParams), i32, i32p, i32, i32p]
    lib.lsh_debug_counts.argtypes = [vp, vp, ctypes.POINTER(StepParams), i32p]
    lib.lsh_debug_logprobs.argtypes = [vp, vp, ctypes.POINTER(StepParams), i32,
                                       ctypes.POINTER(ctypes.c_float), i32, i32p]
    lib.lsh_decode_step_timed.argtypes = lib.lsh_decode_step.argtypes + [vp]
    lib.lsh_decode_step_static.argtypes = [vp, vp, vp, vp, ctypes.POINTER(StepParams), vp, vp, vp, vp]
    lib.lsh_static_scratch_bytes.argtypes = []
    lib.lsh_static_scratch_bytes.restype = sz
    lib.lsh_profiler_create.argtypes = [i32, ctypes.POINTER(vp)]
    lib.lsh_profiler_destroy.argtypes = [vp]
    lib.lsh_profiler_destroy.restype = None
    lib.lsh_profiler_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double), i32p]
    lib.lsh_set_option.argtypes = [vp, ctypes.c_char_p, i32]
    lib.lsh_get_option.argtypes = [vp, ctypes.c_char_p, i32p]
    lib.lsh_step_is_fused.argtypes = [vp, ctypes.POINTER(StepParams)]
    lib.lsh_kernel_name.argtypes = [i32]
    lib.lsh_kernel_name.restype = ctypes.c_char_p
    lib.lsh_select_workspace_bytes.argtypes = [ctypes.POINTER(SelectParams)]
    lib.lsh_select_workspace_bytes.restype = sz
    lib.lsh_beam_select.argtypes = [ctypes.POINTER(SelectParams), vp, vp, vp, vp, sz, vp, vp, vp, vp, vp]
    lib.lsh_cache_workspace_bytes.argtypes = [ctypes.POINTER(CacheParams)]
    lib.lsh_cache_workspace_bytes.restype = sz
    lib.lsh_cache_advance.argtypes = [ctypes.POINTER(CacheParams), i32] + [vp] * 11 + [sz, vp]
    rows = ctypes.POINTER(_Rows)
    lib.lsh_cache_write.argtypes = [ctypes.POINTER(CacheParams), ctypes.POINTER(_PoolPointers), i32, vp, rows, vp, rows, vp, vp, vp]
    lib.lsh_attention_workspace_bytes.argtypes = [ctypes.POINTER(CacheParams), ctypes.POINTER(AttentionParams)]
    lib.lsh_attention_workspace_bytes.restype = sz
    lib.lsh_cache_attention.argtypes = [ctypes.POINTER(CacheParams), ctypes.POINTER(_PoolPointers), ctypes.POINTER(AttentionParams), vp,
                                        rows, vp, vp, vp, vp, vp, sz, vp, rows, vp, vp]
    lib.lsh_status_string.argtypes = [ctypes.c_int]
    lib.lsh_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _status_string(status: int) -> str:
    try:
        return load_library().lsh_status_string(status).decode()
    except Exception:
        return "?"


def _check(status: int, what: str):
    if status != 0:
        raise LshBeamError(status, what)


def kernel_names():
    lib = load_library()
    return [lib.lsh_kernel_name(i).decode() for i in range(NUM_KERNELS)]


def _i32p(a: np.ndarray):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


_current_raw = None


def _current_stream_ptr() -> int:
    """The current device's current stream.  torch.cuda.current_stream() makes a Stream object on every call (3.0 us of
    a step that takes 7 us to enqueue from C); torch's raw getter takes 0.1 us and is used where this torch has it."""
    global _current_raw
    if _current_raw is None:
        import torch
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is None or device is None:
            _current_raw = lambda: int(torch.cuda.current_stream().cuda_stream)
        else:
            torch.cuda.init()
            _current_raw = lambda: raw(device())
    return _current_raw()


def _stream_ptr(stream) -> int:
    if stream is None:
        return _current_stream_ptr()
    if isinstance(stream, int):  # a raw hipStream_t
        return stream
    return int(stream.cuda_stream)


def _require_cuda(x, name, dtypes):
    if x.is_cuda and x.dtype in dtypes and x.is_contiguous():
        return
    if not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if x.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {x.dtype} not in {dtypes}")
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


class Tables:
    """Owns an lsh_tables handle and keeps the borrowed embedding tensor alive."""

    def __init__(self, handle: int, E, K: int, P: int, W: int, e_dtype: int):
        self._h = handle
        self.E = E
        self.V, self.d = int(E.shape[0]), int(E.shape[1])
        self.K, self.P, self.W, self.e_dtype = K, P, W, e_dtype
        self._prof = None          # lsh_profiler* while profile_begin .. profile_end is open

    @property
    def handle(self) -> int:
        if not self._h:
            raise ValueError("tables already freed")
        return self._h

    def close(self):
        if self._prof:
            load_library().lsh_profiler_destroy(self._prof)
            self._prof = None
        if self._h:
            load_library().lsh_free_tables(self._h)
            self._h = None

    # ---- launch-plan options ------------------------------------------------------------------
    def set_option(self, name: str, value: int = OPTION_AUTO):
        """lsh_set_option: force a launch-plan rule (value >= 0) or restore it (OPTION_AUTO)."""
        _check(load_library().lsh_set_option(self.handle, name.encode(), int(value)),
               f"lsh_set_option({name})")

    def get_option(self, name: str) -> int:
        v = ctypes.c_int32(0)
        _check(load_library().lsh_get_option(self.handle, name.encode(), ctypes.byref(v)),
               f"lsh_get_option({name})")
        return v.value

    def set_options(self, **kw):
        for k, v in kw.items():
            self.set_option(k, v)

    def reset_options(self):
        for k in OPTION_NAMES:
            self.set_option(k, OPTION_AUTO)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- inspection -------------------------------------------------------------------------
    def debug_codes(self, H) -> np.ndarray:
        import torch
        _require_cuda(H, "H", (torch.float32,))
        R = int(H.shape[0])
        out = np.empty((R, self.W), dtype=np.int32)
        _check(load_library().lsh_debug_codes(self.handle, H.data_ptr(), R, _i32p(out)),
               "lsh_debug_codes")
        return out

    def debug_embedding_codes(self, row0: int = 0, n: Optional[int] = None) -> np.ndarray:
        n = self.V - row0 if n is None else n
        out = np.empty((n, self.W), dtype=np.int32)
        _check(load_library().lsh_debug_embedding_codes(self.handle, row0, n, _i32p(out)),
               "lsh_debug_embedding_codes")
        return out

    def debug_bucket(self, band: int, code: int):
        out = np.empty(self.V, dtype=np.int32)
        n = ctypes.c_int32(0)
        _check(load_library().lsh_debug_bucket(self.handle, band, int(code), _i32p(out), self.V,
                                               ctypes.byref(n)), "lsh_debug_bucket")
        return None if n.value < 0 else out[: n.value].copy()

    def debug_csr(self, band: int):
        nk = ctypes.c_int32(0)
        lib = load_library()
        _check(lib.lsh_debug_csr(self.handle, band, ctypes.byref(nk), None, None, 0, None),
               "lsh_debug_csr")
        keys = np.empty(nk.value, dtype=np.int32)
        offs = np.empty(nk.value + 1, dtype=np.int32)
        words = np.empty(self.V, dtype=np.int32)
        _check(lib.lsh_debug_csr(self.handle, band, ctypes.byref(nk), _i32p(keys), _i32p(offs),
                                 nk.value, _i32p(words)), "lsh_debug_csr")
        return keys, offs, words

    def debug_build_info(self):
        """(built on the device?, insertion rounds the device made)"""
        dev, att = ctypes.c_int32(0), ctypes.c_int32(0)
        _check(load_library().lsh_debug_build_info(self.handle, ctypes.byref(dev), ctypes.byref(att)),
               "lsh_debug_build_info")
        return bool(dev.value), att.value

    def debug_cuckoo_shape(self, band: int):
        cap, nk = ctypes.c_int32(0), ctypes.c_int32(0)
        _check(load_library().lsh_debug_cuckoo_shape(self.handle, band, ctypes.byref(cap),
                                                     ctypes.byref(nk)), "lsh_debug_cuckoo_shape")
        return cap.value, nk.value

    def debug_candidates(self, workspace, sp: StepParams, s: int) -> np.ndarray:
        out = np.empty(self.V, dtype=np.int32)
        n = ctypes.c_int32(0)
        _check(load_library().lsh_debug_candidates(self.handle, workspace.data_ptr(),
                                                   ctypes.byref(sp), s, _i32p(out), self.V,
                                                   ctypes.byref(n)), "lsh_debug_candidates")
        return out[: n.value].copy()

    def debug_counts(self, workspace, sp: StepParams) -> np.ndarray:
        """Candidate counts of all sentences of the last step on this workspace."""
        out = np.empty(sp.S, dtype=np.int32)
        _check(load_library().lsh_debug_counts(self.handle, workspace.data_ptr(), ctypes.byref(sp),
                                               _i32p(out)), "lsh_debug_counts")
        return out

    def debug_logprobs(self, workspace, sp: StepParams, s: int, cap: Optional[int] = None):
        cap = self.V if cap is None else cap
        out = np.empty((sp.B, cap), dtype=np.float32)
        n = ctypes.c_int32(0)
        _check(load_library().lsh_debug_logprobs(
            self.handle, workspace.data_ptr(), ctypes.byref(sp), s,
            out.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), cap, ctypes.byref(n)),
            "lsh_debug_logprobs")
        return out[:, : min(n.value, cap)].copy()

    # ---- per-kernel timing ------------------------------------------------------------------
    def profile_begin(self, max_steps: int):
        """Steps made through this object (decode_step, make_step_caller) from now on are timed
        per kernel (lsh_decode_step_timed with a profiler this object owns), up to max_steps."""
        lib = load_library()
        if self._prof:
            lib.lsh_profiler_destroy(self._prof)
            self._prof = None
        out = ctypes.c_void_p(0)
        _check(lib.lsh_profiler_create(max_steps, ctypes.byref(out)), "lsh_profiler_create")
        self._prof = out.value

    def profile_end(self):
        """{kernel name: (mean ms per launch, launches)}; ends the timing."""
        lib = load_library()
        if not self._prof:
            raise ValueError("profile_end without profile_begin")
        ms = (ctypes.c_double * NUM_KERNELS)()
        n = (ctypes.c_int32 * NUM_KERNELS)()
        rc = lib.lsh_profiler_read(self._prof, ms, n)
        lib.lsh_profiler_destroy(self._prof)
        self._prof = None
        _check(rc, "lsh_profiler_read")
        return {name: (ms[i], n[i]) for i, name in enumerate(kernel_names())}


def release_kept():
    """lsh_release_kept: device memory kept for the next build goes back to the driver."""
    load_library().lsh_release_kept()


def build_tables(E, perms, K: int, bands: int, seed: int = 0, stream=None) -> Tables:
    """lsh_build_tables.  E: device tensor [V, d], float32, or bfloat16 / int16 / uint16 holding
    bf16 bit patterns; perms: device int32 [P, K]."""
    import torch
    lib = load_library()
    if E.dtype == torch.float32:
        dt = LSH_F32
    elif E.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        dt = LSH_BF16
    else:
        raise ValueError(f"E: unsupported dtype {E.dtype}")
    _require_cuda(perms, "perms", (torch.int32,))
    if E.dim() != 2 or perms.dim() != 2 or int(perms.shape[1]) != K:
        raise ValueError("E must be [V, d] and perms [P, K]")
    # rows may be pitched (a [:, a:b] view of a wider matrix): unit stride inside a row only
    if not E.is_cuda or int(E.stride(1)) != 1 or int(E.stride(0)) < int(E.shape[1]):
        raise ValueError("E must be a device tensor with contiguous rows (row pitch >= d)")
    bp = BuildParams(int(E.shape[0]), int(E.shape[1]), int(E.stride(0)), dt, K,
                     int(perms.shape[0]), bands, seed)
    out = ctypes.c_void_p(0)
    _check(lib.lsh_build_tables(E.data_ptr(), perms.data_ptr(), ctypes.byref(bp),
                                _stream_ptr(stream), ctypes.byref(out)), "lsh_build_tables")
    return Tables(out.value, E, K, int(perms.shape[0]), bands, dt)


def step_params(S: int, B: int, T: int, threshold: int = 1, full_vocab: bool = False) -> StepParams:
    return StepParams(S, B, T, threshold, 1 if full_vocab else 0)


def step_is_fused(tables: Tables, sp: StepParams) -> bool:
    return bool(load_library().lsh_step_is_fused(tables.handle, ctypes.byref(sp)))


def step_workspace_bytes(tables: Tables, sp: StepParams) -> int:
    return int(load_library().lsh_step_workspace_bytes(tables.handle, ctypes.byref(sp)))


def decode_step(tables: Tables, H, beam_scores, topfreq, sp: StepParams, workspace, out_beam,
                out_word, out_score, stream=None):
    """lsh_decode_step: asynchronous on `stream` (default: torch's current stream)."""
    import torch
    _require_cuda(H, "H", (torch.float32,))
    _require_cuda(beam_scores, "beam_scores", (torch.float32,))
    _require_cuda(out_beam, "out_beam", (torch.int32,))
    _require_cuda(out_word, "out_word", (torch.int32,))
    _require_cuda(out_score, "out_score", (torch.float32,))
    R = sp.S * sp.B
    if H.numel() != R * tables.d or beam_scores.numel() != R:
        raise ValueError("H must be [S*B, d] and beam_scores [S*B]")
    if min(out_beam.numel(), out_word.numel(), out_score.numel()) < R:
        raise ValueError("outputs must hold S*B elements")
    tf_ptr = 0
    if topfreq is not None:
        _require_cuda(topfreq, "topfreq", (torch.int32,))
        if topfreq.numel() < sp.T:
            raise ValueError("topfreq shorter than T")
        tf_ptr = topfreq.data_ptr()
    args = (tables.handle, H.data_ptr(), beam_scores.data_ptr(), tf_ptr, ctypes.byref(sp),
            workspace.data_ptr(), workspace.numel() * workspace.element_size(), out_beam.data_ptr(),
            out_word.data_ptr(), out_score.data_ptr(), _stream_ptr(stream))
    if tables._prof:
        _check(load_library().lsh_decode_step_timed(*args, tables._prof), "lsh_decode_step_timed")
    else:
        _check(load_library().lsh_decode_step(*args), "lsh_decode_step")


def static_scratch_bytes() -> int:
    return int(load_library().lsh_static_scratch_bytes())


def decode_step_static(tables: Tables, H, beam_scores, topfreq, sp: StepParams, out_beam, out_word,
                       out_score, stream=None):
    """lsh_decode_step_static: the step in the library's built-in scratch buffer (no workspace)."""
    import torch
    for x, name, dt in ((H, "H", torch.float32), (beam_scores, "beam_scores", torch.float32),
                        (out_beam, "out_beam", torch.int32), (out_word, "out_word", torch.int32),
                        (out_score, "out_score", torch.float32)):
        _require_cuda(x, name, (dt,))
    R = sp.S * sp.B
    if H.numel() != R * tables.d or beam_scores.numel() != R:
        raise ValueError("H must be [S*B, d] and beam_scores [S*B]")
    if min(out_beam.numel(), out_word.numel(), out_score.numel()) < R:
        raise ValueError("outputs must hold S*B elements")
    tf_ptr = 0
    if topfreq is not None:
        _require_cuda(topfreq, "topfreq", (torch.int32,))
        if topfreq.numel() < sp.T:
            raise ValueError("topfreq shorter than T")
        tf_ptr = topfreq.data_ptr()
    _check(load_library().lsh_decode_step_static(
        tables.handle, H.data_ptr(), beam_scores.data_ptr(), tf_ptr, ctypes.byref(sp),
        out_beam.data_ptr(), out_word.data_ptr(), out_score.data_ptr(), _stream_ptr(stream)),
        "lsh_decode_step_static")


def make_step_caller(tables: Tables, sp: StepParams, workspace, topfreq):
    """Pre-marshalled lsh_decode_step for tight loops: returns
    f(H_ptr, beam_scores_ptr, out_beam_ptr, out_word_ptr, out_score_ptr, stream_ptr) -> None,
    all arguments raw device addresses (ints).  Same entry point, same kernels; only the Python
    argument checking is hoisted out of the loop."""
    lib = load_library()
    fn, fn_timed = lib.lsh_decode_step, lib.lsh_decode_step_timed
    h = ctypes.c_void_p(tables.handle)
    spp = ctypes.pointer(sp)
    ws = ctypes.c_void_p(workspace.data_ptr())
    wsn = ctypes.c_size_t(workspace.numel() * workspace.element_size())
    tf = ctypes.c_void_p(topfreq.data_ptr() if topfreq is not None else 0)
    keep = (tables, sp, workspace, topfreq)

    def call(H_ptr, bs_ptr, ob_ptr, ow_ptr, osc_ptr, stream_ptr, _keep=keep):
        if tables._prof:
            rc = fn_timed(h, H_ptr, bs_ptr, tf, spp, ws, wsn, ob_ptr, ow_ptr, osc_ptr, stream_ptr,
                          tables._prof)
        else:
            rc = fn(h, H_ptr, bs_ptr, tf, spp, ws, wsn, ob_ptr, ow_ptr, osc_ptr, stream_ptr)
        if rc:
            raise LshBeamError(rc, "lsh_decode_step")

    return call


class BeamHistory:
    """Caller-owned device arrays of the beam bookkeeping calls (torch is only the allocator)."""

    def __init__(self, S: int, B: int, max_len: int, n_states: int = 0, state_dim: int = 0, eos: int = -1):
        import torch
        self.bp = BeamParams(S, B, n_states, state_dim, eos, max_len)
        self.backptr = torch.empty((max_len, S, B), dtype=torch.int32, device="cuda")
        self.words = torch.empty((max_len, S, B), dtype=torch.int32, device="cuda")
        self.scores = torch.empty((max_len, S, B), dtype=torch.float32, device="cuda")


def beam_advance(hist: BeamHistory, step: int, out_beam, out_word, out_score, states_in, states_out,
                 next_scores, stream=None) -> None:
    """lsh_beam_advance; states_in / states_out are sequences of device tensors [S*B, state_dim]."""
    n = hist.bp.n_states
    assert len(states_in) == n and len(states_out) == n
    pin = (ctypes.c_void_p * max(n, 1))(*[t.data_ptr() for t in states_in])
    pout = (ctypes.c_void_p * max(n, 1))(*[t.data_ptr() for t in states_out])
    _check(load_library().lsh_beam_advance(ctypes.byref(hist.bp), step, out_beam.data_ptr(),
                                           out_word.data_ptr(), out_score.data_ptr(), pin, pout,
                                           hist.backptr.data_ptr(), hist.words.data_ptr(),
                                           hist.scores.data_ptr(), next_scores.data_ptr(),
                                           _stream_ptr(stream)), "lsh_beam_advance")


def beam_backtrace(hist: BeamHistory, n_steps: int, stream=None):
    """lsh_beam_backtrace -> (tokens [S, max_len] int32, length [S] int32, score [S] fp32), device."""
    import torch
    S, L = hist.bp.S, hist.bp.max_len
    tokens = torch.full((S, L), -1, dtype=torch.int32, device="cuda")
    length = torch.empty(S, dtype=torch.int32, device="cuda")
    score = torch.empty(S, dtype=torch.float32, device="cuda")
    _check(load_library().lsh_beam_backtrace(ctypes.byref(hist.bp), n_steps, hist.backptr.data_ptr(),
                                             hist.words.data_ptr(), hist.scores.data_ptr(),
                                             tokens.data_ptr(), length.data_ptr(), score.data_ptr(),
                                             _stream_ptr(stream)), "lsh_beam_backtrace")
    return tokens, length, score


# ---- selection from the caller's logits, and a paged cache in 8 bits -----------------------------

class _Torch:
    """What the calls below need of torch, looked up once."""

    def __init__(self):
        import torch
        self.i32, self.f32, self.u8 = torch.int32, torch.float32, torch.uint8
        self.types = {torch.float32: LSH_F32, torch.bfloat16: LSH_BF16, torch.float16: LSH_F16}
        torch.cuda.init()
        self.device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


_torch = None


def _t() -> _Torch:
    global _torch
    if _torch is None:
        _torch = _Torch()
    return _torch


def _ptr(x, dtype, n, name, device) -> int:
    """Device address of a contiguous tensor of n elements on the current device: the library launches there, and has no handle
    that says where it was made."""
    if x.dtype is dtype and x.get_device() == device and x.numel() == n and x.is_contiguous():
        return x.data_ptr()
    _require_cuda(x, name, (dtype,))
    if x.numel() != n:
        raise ValueError(f"{name} must have {n} elements, has {x.numel()}")
    raise ValueError(f"{name} must be on the current device")


def _room(x, device):
    """Address and bytes of a workspace."""
    if x.get_device() != device or not x.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the current device")
    return x.data_ptr(), x.numel() * x.element_size()


def select_params(S: int, B: int, V: int, N: Optional[int] = None) -> SelectParams:
    """N: results per sentence, B of them unless given."""
    return SelectParams(S, B, B if N is None else N, V, LSH_F32, V, 0)


def select_workspace_bytes(sp: SelectParams) -> int:
    return int(load_library().lsh_select_workspace_bytes(ctypes.byref(sp)))


def beam_select(sp: SelectParams, logits, beam_scores, workspace, out_beam, out_word, out_score, allowed=None, lse=None,
                stream=None):
    """lsh_beam_select: asynchronous on `stream` (default: torch's current stream).  logits: [S*B, V], float32, bfloat16 or
    float16, unit stride in a row; allowed: int32 bits [S*B, >= ceil(V / 32)], or one row of them for all."""
    t = _t()
    dev, R, V = t.device(), sp.S * sp.B, sp.V
    n = sp.S * sp.N
    dtype = t.types.get(logits.dtype)
    if dtype is None or logits.get_device() != dev or tuple(logits.shape) != (R, V) or (V > 1 and logits.stride(1) != 1):
        raise ValueError(f"logits must be [S*B, V] with contiguous rows on the current device, of {tuple(t.types)}")
    mask, mask_ld = None, 0
    if allowed is not None:
        words = (V + 31) // 32
        if allowed.dtype is not t.i32 or allowed.get_device() != dev or allowed.dim() != 2 or allowed.shape[0] not in (1, R) or (
                allowed.shape[1] < words or (allowed.shape[1] > 1 and allowed.stride(1) != 1)):
            raise ValueError("allowed must be int32 [S*B or 1, >= ceil(V / 32)] with contiguous rows on the current device")
        mask, mask_ld = allowed.data_ptr(), allowed.stride(0) if allowed.shape[0] > 1 else 0
    p = SelectParams(sp.S, sp.B, sp.N, V, dtype, logits.stride(0) if R > 1 else V, mask_ld)
    ws, room = _room(workspace, dev)
    _check(load_library().lsh_beam_select(
        ctypes.byref(p), logits.data_ptr(), _ptr(beam_scores, t.f32, R, "beam_scores", dev), mask, ws, room,
        _ptr(out_beam, t.i32, n, "out_beam", dev), _ptr(out_word, t.i32, n, "out_word", dev), _ptr(out_score, t.f32, n, "out_score", dev),
        None if lse is None else _ptr(lse, t.f32, R, "lse", dev), _stream_ptr(stream)), "lsh_beam_select")


def cache_params(S: int, B: int, n_blocks: int, block: int, max_blocks: int, n_heads: int, head_dim: int) -> CacheParams:
    return CacheParams(S, B, n_blocks, block, max_blocks, n_heads, head_dim)


class CachePool:
    """Caller-owned device memory of one layer of a cache (torch is only the allocator): codes as uint8 k [n_blocks, heads,
    head_dim / 16, block, 16] and v [n_blocks, heads, block / 16, head_dim, 16], scales as float32 [n_blocks, heads].  Tensors
    that are handed in are kept and used as they are."""

    def __init__(self, cp: CacheParams, k=None, v=None, k_scale=None, v_scale=None):
        import torch
        shapes = ((cp.n_blocks, cp.n_heads, cp.head_dim // 16, cp.block, 16), (cp.n_blocks, cp.n_heads, cp.block // 16, cp.head_dim, 16),
                  (cp.n_blocks, cp.n_heads), (cp.n_blocks, cp.n_heads))
        given = []
        for x, shape, name in zip((k, v, k_scale, v_scale), shapes, ("k", "v", "k_scale", "v_scale")):
            dtype = torch.uint8 if name in ("k", "v") else torch.float32
            if x is None:
                x = torch.zeros(shape, dtype=dtype, device="cuda")
            _require_cuda(x, name, (dtype,))
            if tuple(x.shape) != shape:
                raise ValueError(f"{name} must be {shape}, is {tuple(x.shape)}")
            given.append(x)
        self.k, self.v, self.k_scale, self.v_scale = given
        self._shape = (cp.n_blocks, cp.block, cp.n_heads, cp.head_dim)
        if len({x.get_device() for x in given}) != 1:
            raise ValueError("a pool's tensors must be on one device")
        self._device = self.k.get_device()
        self._pointers = _PoolPointers(*[x.data_ptr() for x in given])

    def _of(self, cp: CacheParams, device: int):
        if (cp.n_blocks, cp.block, cp.n_heads, cp.head_dim) != self._shape or device != self._device:
            raise ValueError("the pool was made for other cache parameters, or on another device than the current one")
        return ctypes.byref(self._pointers)


def cache_workspace_bytes(cp: CacheParams) -> int:
    return int(load_library().lsh_cache_workspace_bytes(ctypes.byref(cp)))


def cache_advance(cp: CacheParams, T: int, tables_in, lengths_in, tables_out, lengths_out, slots, copy_from, shared, status, workspace,
                  parents=None, n_new=None, stream=None):
    """lsh_cache_advance: all arrays int32; shared, parents and n_new may be None."""
    t = _t()
    dev, i32, R = t.device(), t.i32, cp.S * cp.B
    n = R * cp.max_blocks
    ws, room = _room(workspace, dev)
    _check(load_library().lsh_cache_advance(
        ctypes.byref(cp), T, None if parents is None else _ptr(parents, i32, R, "parents", dev),
        None if n_new is None else _ptr(n_new, i32, R, "n_new", dev), _ptr(tables_in, i32, n, "tables_in", dev),
        _ptr(lengths_in, i32, R, "lengths_in", dev), _ptr(tables_out, i32, n, "tables_out", dev),
        _ptr(lengths_out, i32, R, "lengths_out", dev), _ptr(slots, i32, R * T, "slots", dev), _ptr(copy_from, i32, R, "copy_from", dev),
        None if shared is None else _ptr(shared, i32, cp.S, "shared", dev), _ptr(status, i32, 2, "status", dev), ws, room,
        _stream_ptr(stream)), "lsh_cache_advance")


def _rows(x, name, R, T, heads, D, dev):
    """lsh_rows of a tensor [R, T, heads, D] with any pitches."""
    t = _t().types.get(x.dtype)
    if t is None or x.get_device() != dev or tuple(x.shape) != (R, T, heads, D):
        raise ValueError(f"{name} must be {(R, T, heads, D)} on the current device, of {tuple(_t().types)}")
    row, token, head, one = x.stride()
    if one != 1:
        raise ValueError(f"{name} must have contiguous heads")
    return _Rows(t, row, token, head)


def cache_write(cp: CacheParams, pool: CachePool, k, v, slots, copy_from=None, stream=None):
    """lsh_cache_write: k, v [S*B, T, n_heads, head_dim] (views into a fused projection, say), slots int32 [S*B, T]."""
    t = _t()
    dev, R, T = t.device(), cp.S * cp.B, k.shape[1] if k.dim() == 4 else 0
    kr, vr = _rows(k, "k", R, T, cp.n_heads, cp.head_dim, dev), _rows(v, "v", R, T, cp.n_heads, cp.head_dim, dev)
    _check(load_library().lsh_cache_write(
        ctypes.byref(cp), pool._of(cp, dev), T, k.data_ptr(), ctypes.byref(kr), v.data_ptr(), ctypes.byref(vr),
        _ptr(slots, t.i32, R * T, "slots", dev), None if copy_from is None else _ptr(copy_from, t.i32, R, "copy_from", dev),
        _stream_ptr(stream)), "lsh_cache_write")


def attention_params(T: int, n_heads: int, scale: float, causal: bool = True, window: int = 0) -> AttentionParams:
    return AttentionParams(T, n_heads, 1 if causal else 0, window, scale)


def attention_workspace_bytes(cp: CacheParams, ap: AttentionParams) -> int:
    return int(load_library().lsh_attention_workspace_bytes(ctypes.byref(cp), ctypes.byref(ap)))


def cache_attention(cp: CacheParams, ap: AttentionParams, pool: CachePool, q, tables, lengths, workspace, out, shared=None, n_new=None,
                    lse=None, stream=None):
    """lsh_cache_attention: q, out [S*B, T, n_heads, head_dim] of one type, lse float32 [S*B, T, n_heads] or None."""
    t = _t()
    dev, i32, R, T, H = t.device(), t.i32, cp.S * cp.B, ap.T, ap.n_heads
    qr, orow = _rows(q, "q", R, T, H, cp.head_dim, dev), _rows(out, "out", R, T, H, cp.head_dim, dev)
    ws, room = _room(workspace, dev)
    _check(load_library().lsh_cache_attention(
        ctypes.byref(cp), pool._of(cp, dev), ctypes.byref(ap), q.data_ptr(), ctypes.byref(qr),
        _ptr(tables, i32, R * cp.max_blocks, "tables", dev), _ptr(lengths, i32, R, "lengths", dev),
        None if n_new is None else _ptr(n_new, i32, R, "n_new", dev), None if shared is None else _ptr(shared, i32, cp.S, "shared", dev),
        ws, room, out.data_ptr(), ctypes.byref(orow), None if lse is None else _ptr(lse, t.f32, R * T * H, "lse", dev),
        _stream_ptr(stream)), "lsh_cache_attention")
