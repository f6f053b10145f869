"""ctypes binding of libcham (argument marshalling only; every step runs in the HIP kernels).

PyTorch is used for device memory and the current stream, nothing else.  The functions carry
the names of the C entry points declared in ``include/cham.h``.  There is no CPU fallback:
if the library is not built, or no GPU is present, calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcham.so")

F_FORCE_EXACT, F_STREAMING, F_RESIDENT, F_NO_MFMA = 1, 2, 4, 8
F_VALUES_BELOW_2048 = 16
F_NORM_GIVEN = 32
TYPE_F32, TYPE_BF16, TYPE_F16, TYPE_I8, TYPE_I32, TYPE_I64 = 0, 1, 2, 16, 17, 18
TERMS = ("total", "policy", "value", "entropy", "kl", "clipped")
OUT_EMPTY, OUT_KEPT, OUT_SYNTH, OUT_DROPPED = 0, 1, 2, 3

EXPORTS = [
    "cham_version", "cham_strerror", "cham_last_hip_error", "cham_sweep_workspace_bytes",
    "cham_kmeans_sweep", "cham_select_k", "cham_select_k_host", "cham_snap_workspace_bytes",
    "cham_snap_centroids", "cham_synth_workspace_bytes", "cham_synthesize", "cham_hash_config",
    "cham_hash_rows", "cham_sweep_knee_workspace_bytes", "cham_kmeans_sweep_knee", "cham_synthesize_table",
    "cham_visited_table_clear", "cham_visited_table_insert_hashes", "cham_visited_table_insert_configs",
    "cham_update_configs", "cham_sweep_path", "cham_sweep_path_kernel", "cham_sweep_kernel", "cham_sweep_passes",
    "cham_static_bytes", "cham_static_init", "cham_kmeans_sweep_static",
    "cham_sweep_workspace_bytes_u16", "cham_sweep_path_u16", "cham_sweep_kernel_u16", "cham_kmeans_sweep_u16", "cham_sweep_knee_workspace_bytes_u16",
    "cham_kmeans_sweep_knee_u16", "cham_snap_workspace_bytes_u16", "cham_snap_centroids_u16",
    "cham_synth_workspace_bytes_u16", "cham_synthesize_u16", "cham_synthesize_table_u16",
    "cham_visited_table_insert_configs_u16", "cham_hash_config_u16", "cham_hash_rows_u16",
    "cham_policy_workspace_bytes", "cham_policy_logp", "cham_policy_loss", "cham_gae_workspace_bytes", "cham_gae",
    "cham_grad_workspace_bytes", "cham_grad_norm", "cham_clip_grads",
]


class ChamError(RuntimeError):
    pass


_FLOAT_TYPES, _ACTION_TYPES = {}, {}                    # torch's types and the library's codes, once torch is there


class _PolicyCoef(C.Structure):
    _fields_ = [(name, C.c_double) for name in ("clip_low", "clip_high", "value", "entropy", "kl", "value_clip")]


_lib = None


def load() -> C.CDLL:
    """Load libcham.so (built in-tree by ``build.build_lib``); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ChamError(f"{LIB_PATH} is not built; run `python -m paper_2001_08743_amd.build`")
        # PyTorch ships its own copy of the HIP runtime: it has to be in the process first, so that the
        # library binds to that same runtime (its kernels then see the device and streams torch uses).
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        lib = C.CDLL(LIB_PATH)
        vp, i32, i64, u64, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_double
        lib.cham_version.restype = i32
        lib.cham_strerror.restype = C.c_char_p
        lib.cham_strerror.argtypes = [i32]
        lib.cham_last_hip_error.restype = i32
        lib.cham_sweep_workspace_bytes.restype = i64
        lib.cham_sweep_workspace_bytes.argtypes = [i64, i32, vp, i32, vp, i32, i32, i32]
        lib.cham_kmeans_sweep.restype = i32
        lib.cham_kmeans_sweep.argtypes = [vp, i64, i32, vp, i32, vp, i32, i32, i32, vp,
                                          vp, vp, vp, vp, vp, vp, vp, i64, i32, vp]
        lib.cham_sweep_path.restype = i32
        lib.cham_sweep_path.argtypes = [i64, i32, vp, i32, vp, i32, i32]
        lib.cham_sweep_path_u16.restype = i32
        lib.cham_sweep_path_u16.argtypes = [i64, i32, vp, i32, vp, i32, i32]
        lib.cham_sweep_path_kernel.restype = C.c_char_p
        lib.cham_sweep_path_kernel.argtypes = [i32]
        for name in ("cham_sweep_kernel", "cham_sweep_kernel_u16"):
            getattr(lib, name).restype = C.c_char_p
            getattr(lib, name).argtypes = [i64, i32, vp, i32, vp, i32, i32]
        lib.cham_sweep_passes.restype = i32
        lib.cham_sweep_passes.argtypes = [vp, i64, i64, i32, vp, i32, vp, i32, i32, vp, vp]
        lib.cham_static_bytes.restype = i64
        lib.cham_static_bytes.argtypes = [i64, i32, vp, i32, vp, i32, i32]
        lib.cham_static_init.restype = i32
        lib.cham_static_init.argtypes = []
        lib.cham_kmeans_sweep_static.restype = i32
        lib.cham_kmeans_sweep_static.argtypes = [vp, i64, i32, vp, i32, vp, i32, i32, i32, vp,
                                                 vp, vp, vp, vp, vp, vp, i32, vp]
        lib.cham_sweep_knee_workspace_bytes.restype = i64
        lib.cham_sweep_knee_workspace_bytes.argtypes = [i64, i32, vp, i32, vp, i32, i32, i32]
        lib.cham_kmeans_sweep_knee.restype = i32
        lib.cham_kmeans_sweep_knee.argtypes = [vp, i64, i32, vp, i32, vp, i32, i32, i32, vp, f64, i32,
                                               vp, vp, vp, vp, vp, vp, vp, vp, i64, i32, vp]
        lib.cham_synthesize_table.restype = i32
        lib.cham_synthesize_table.argtypes = [vp, i64, i32, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, i64, vp,
                                              vp, vp, vp, vp, i64, vp]
        lib.cham_visited_table_clear.restype = i32
        lib.cham_visited_table_clear.argtypes = [vp, i64, vp]
        lib.cham_visited_table_insert_hashes.restype = i32
        lib.cham_visited_table_insert_hashes.argtypes = [vp, i64, vp, i64, vp, vp]
        lib.cham_visited_table_insert_configs.restype = i32
        lib.cham_visited_table_insert_configs.argtypes = [vp, i64, vp, i64, i32, vp, vp, i64, vp, vp]
        lib.cham_update_configs.restype = i32
        lib.cham_update_configs.argtypes = [vp, vp, i64, i32, i32, vp, u64, vp, i64, vp, i64, vp, vp, vp]
        lib.cham_select_k.restype = i32
        lib.cham_select_k.argtypes = [vp, vp, i32, i32, f64, vp, vp]
        lib.cham_select_k_host.restype = i32
        lib.cham_select_k_host.argtypes = [vp, vp, i32, f64]
        lib.cham_snap_workspace_bytes.restype = i64
        lib.cham_snap_workspace_bytes.argtypes = [i64, i32, vp, i32, vp, i32]
        lib.cham_snap_centroids.restype = i32
        lib.cham_snap_centroids.argtypes = [vp, i64, i32, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, i64, i32, vp]
        lib.cham_synth_workspace_bytes.restype = i64
        lib.cham_synth_workspace_bytes.argtypes = [i64, i32, vp, i32, vp, i32]
        lib.cham_synthesize.restype = i32
        lib.cham_synthesize.argtypes = [vp, i64, i32, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, i64, vp,
                                        vp, vp, vp, vp, i64, vp]
        lib.cham_hash_config.restype = u64
        lib.cham_hash_config.argtypes = [vp, i32, u64]
        lib.cham_hash_rows.restype = i32
        lib.cham_hash_rows.argtypes = [vp, i64, i32, vp, u64, vp, vp]
        lib.cham_policy_workspace_bytes.restype = i64
        lib.cham_policy_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
        lib.cham_policy_logp.restype = i32
        lib.cham_policy_logp.argtypes = [vp, i32, i64, i32, i32, i64, i64, vp, i32, i64, vp, vp, vp, vp, i64, vp]
        lib.cham_policy_loss.restype = i32
        lib.cham_policy_loss.argtypes = [vp, i32, i64, i32, i32, i64, i64, vp, i32, i64, vp, vp, vp, vp, vp, vp, vp,
                                         C.POINTER(_PolicyCoef), vp, vp, vp, vp, i64, i64, vp, vp, i64, vp]
        lib.cham_gae_workspace_bytes.restype = i64
        lib.cham_gae_workspace_bytes.argtypes = [i64, i64]
        lib.cham_gae.restype = i32
        lib.cham_gae.argtypes = [i32, i64, i64, vp, i64, i64, vp, i64, i64, vp, i64, i64, vp, vp, f64, f64, vp, vp, i64, i64,
                                 vp, i64, vp]
        lib.cham_grad_workspace_bytes.restype = i64
        lib.cham_grad_workspace_bytes.argtypes = [vp, vp, i32]
        lib.cham_grad_norm.restype = i32
        lib.cham_grad_norm.argtypes = [vp, vp, vp, i32, vp, vp, i64, vp]
        lib.cham_clip_grads.restype = i32
        lib.cham_clip_grads.argtypes = [vp, vp, vp, vp, i32, f64, vp, vp, i64, i32, vp]
        # the entry points for two-byte knobs take the same argument lists
        for name in EXPORTS:
            if name.endswith("_u16"):
                base = getattr(lib, name[:-4])
                getattr(lib, name).restype = base.restype
                getattr(lib, name).argtypes = base.argtypes
        _lib = lib
    return _lib


def _knob_dtypes(sfx: str):
    """(numpy dtype of host rows, torch dtype of device knob buffers) for an entry-point suffix.
    Two-byte knobs live in int16 tensors (same bits as uint16)."""
    torch = _torch()
    return (np.uint8, torch.uint8) if sfx == "" else (np.uint16, torch.int16)


def knobs_to_host(t) -> np.ndarray:
    """Device knob tensor (uint8, or int16 holding uint16 bits) as a numpy array of unsigned values."""
    a = t.cpu().numpy()
    return a.view(np.uint16) if a.dtype == np.int16 else a


def _check(rc: int):
    if rc < 0:
        lib = load()
        msg = lib.cham_strerror(int(rc)).decode()
        raise ChamError(f"libcham error {rc}: {msg} (hip error {lib.cham_last_hip_error()})")
    return rc


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:                           # a GPU that is there stays: asked once, 2 us a call otherwise
        import torch
        if not torch.cuda.is_available():
            raise ChamError("no GPU visible: libcham has no CPU path")
        _FLOAT_TYPES.update({torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16})
        _ACTION_TYPES.update({torch.int8: TYPE_I8, torch.int32: TYPE_I32, torch.int64: TYPE_I64})
        _torch_module = torch
    return _torch_module


def _hp(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _dp(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    torch = _torch()
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _host_lists(task_off, ks):
    to = np.ascontiguousarray(task_off, dtype=np.int64)
    k = np.ascontiguousarray(ks, dtype=np.int32)
    return to, k


def to_soa(rows: np.ndarray, device="cuda:0", pad_to: int = 64):
    """Upload row-major rows [N, d] (uint8, or uint16 for two-byte knobs) as the structure-of-arrays
    matrix X [d, ld] the library reads."""
    torch = _torch()
    dt = np.uint16 if np.asarray(rows).dtype == np.uint16 else np.uint8
    rows = np.ascontiguousarray(rows, dtype=dt)
    n, d = rows.shape
    ld = max(pad_to, (n + pad_to - 1) // pad_to * pad_to)
    host = np.zeros((d, ld), dtype=dt)
    host[:, :n] = rows.T
    if dt == np.uint16:
        host = host.view(np.int16)
    return torch.from_numpy(host).to(device), ld


def cham_version() -> int:
    return int(load().cham_version())


def cham_hash_config(cfg, salt: int = 0) -> int:
    cfg = np.ascontiguousarray(cfg, dtype=np.uint8)
    return int(load().cham_hash_config(_hp(cfg), C.c_int32(cfg.shape[0]), C.c_uint64(int(salt))))


def cham_hash_config_u16(cfg, salt: int = 0) -> int:
    cfg = np.ascontiguousarray(cfg, dtype=np.uint16)
    return int(load().cham_hash_config_u16(_hp(cfg), C.c_int32(cfg.shape[0]), C.c_uint64(int(salt))))


def cham_select_k_host(curve, status=None, threshold: float = 2.5) -> int:
    curve = np.ascontiguousarray(curve, dtype=np.float64)
    st = None if status is None else np.ascontiguousarray(status, dtype=np.int32)
    return int(load().cham_select_k_host(_hp(curve), _hp(st), C.c_int32(len(curve)), C.c_double(threshold)))


def cham_hash_rows(rows_dev, salts_dev=None, salt_all: int = 0, _sfx: str = ""):
    """rows_dev: device uint8 [n, d] row-major; salts_dev: device int64/uint64 [n] or None."""
    torch = _torch()
    assert rows_dev.dtype == _knob_dtypes(_sfx)[1]
    n, d = rows_dev.shape
    out = torch.empty(n, dtype=torch.int64, device=rows_dev.device)
    _check(getattr(load(), "cham_hash_rows" + _sfx)(_dp(rows_dev), C.c_int64(n), C.c_int32(d), _dp(salts_dev),
                                                    C.c_uint64(int(salt_all)), _dp(out), _stream()))
    return out


def cham_hash_rows_u16(rows_dev, salts_dev=None, salt_all: int = 0):
    """rows_dev: device int16 tensor [n, d] holding uint16 knob values, row-major."""
    return cham_hash_rows(rows_dev, salts_dev, salt_all, _sfx="_u16")


def cham_sweep_workspace_bytes(ld, d, task_off, ks, n_iter, flags=0, _sfx: str = "") -> int:
    to, k = _host_lists(task_off, ks)
    fn = getattr(load(), "cham_sweep_workspace_bytes" + _sfx)
    return _check(fn(C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(len(to) - 1),
                     _hp(k), C.c_int32(len(k)), C.c_int32(n_iter), C.c_int32(flags)))


def cham_sweep_knee_workspace_bytes(ld, d, task_off, ks, n_iter, flags=0, _sfx: str = "") -> int:
    to, k = _host_lists(task_off, ks)
    fn = getattr(load(), "cham_sweep_knee_workspace_bytes" + _sfx)
    return _check(fn(C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(len(to) - 1), _hp(k), C.c_int32(len(k)),
                     C.c_int32(n_iter), C.c_int32(flags)))


def cham_sweep_workspace_bytes_u16(ld, d, task_off, ks, n_iter, flags=0) -> int:
    return cham_sweep_workspace_bytes(ld, d, task_off, ks, n_iter, flags, _sfx="_u16")


def cham_sweep_knee_workspace_bytes_u16(ld, d, task_off, ks, n_iter, flags=0) -> int:
    return cham_sweep_knee_workspace_bytes(ld, d, task_off, ks, n_iter, flags, _sfx="_u16")


def cham_kmeans_sweep(X, ld: int, d: int, task_off, ks: Sequence[int], n_iter: int, init_centroids=None,
                      want_labels: bool = False, want_trace: bool = False, flags: int = 0,
                      out: Optional[dict] = None, workspace=None, _sfx: str = ""):
    """Run the sweep; returns a dict of device tensors (centroids, counts, inertia, status, labels, trace)."""
    torch = _torch()
    lib = load()
    assert X.dtype == _knob_dtypes(_sfx)[1]
    to, k = _host_lists(task_off, ks)
    T, n_k, Ksum = len(to) - 1, len(k), int(k.sum())
    dev = X.device
    if out is None:
        out = {}
        out["centroids"] = torch.empty((T, Ksum, d), dtype=torch.float64, device=dev)
        out["counts"] = torch.empty((T, Ksum), dtype=torch.int32, device=dev)
        out["inertia"] = torch.empty((T, n_k), dtype=torch.float64, device=dev)
        out["status"] = torch.empty((T, n_k), dtype=torch.int32, device=dev)
        out["labels"] = torch.zeros((n_k, ld), dtype=torch.uint8, device=dev) if want_labels else None
        out["trace"] = torch.empty((T, n_k, n_iter + 1), dtype=torch.float64, device=dev) if want_trace else None
    if workspace is None:
        nbytes = cham_sweep_workspace_bytes(ld, d, to, k, n_iter, flags, _sfx=_sfx)
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    rc = getattr(lib, "cham_kmeans_sweep" + _sfx)(_dp(X), C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(T), _hp(k), C.c_int32(n_k),
                               C.c_int32(n_iter), C.c_int32(0 if init_centroids is None else 1),
                               _dp(init_centroids), _dp(out["centroids"]), _dp(out["counts"]),
                               _dp(out["inertia"]), _dp(out["status"]), _dp(out.get("labels")),
                               _dp(out.get("trace")), _dp(workspace), C.c_int64(workspace.numel()),
                               C.c_int32(flags), _stream())
    _check(rc)
    out["workspace"] = workspace
    out["koff"] = np.concatenate([[0], np.cumsum(k)]).astype(np.int64)
    return out


def cham_sweep_path(ld: int, d: int, task_off, ks, flags: int = 0, _sfx: str = "") -> int:
    to, k = _host_lists(task_off, ks)
    return _check(getattr(load(), "cham_sweep_path" + _sfx)(C.c_int64(ld), C.c_int32(d), _hp(to),
                                                            C.c_int32(len(to) - 1), _hp(k), C.c_int32(len(k)),
                                                            C.c_int32(flags)))


def cham_sweep_path_u16(ld: int, d: int, task_off, ks, flags: int = 0) -> int:
    return cham_sweep_path(ld, d, task_off, ks, flags, _sfx="_u16")


def cham_sweep_path_kernel(path: int) -> str:
    return load().cham_sweep_path_kernel(C.c_int32(path)).decode()


def cham_sweep_kernel(ld: int, d: int, task_off, ks, flags: int = 0, _sfx: str = "") -> str:
    """Name of the kernel that does the sweep for these arguments."""
    to, k = _host_lists(task_off, ks)
    name = getattr(load(), "cham_sweep_kernel" + _sfx)(C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(len(to) - 1), _hp(k), C.c_int32(len(k)),
                                                       C.c_int32(flags))
    if name is None:
        cham_sweep_path(ld, d, task_off, ks, flags, _sfx)                   # raises the error
        raise ChamError("cham_sweep_kernel: no kernel for these arguments")
    return name.decode()


def cham_sweep_kernel_u16(ld: int, d: int, task_off, ks, flags: int = 0) -> str:
    return cham_sweep_kernel(ld, d, task_off, ks, flags, _sfx="_u16")


def cham_sweep_passes(workspace, ld: int, d: int, task_off, ks, flags: int = 0, passes=None):
    """Labelling passes per (task, k) that the last sweep using ``workspace`` ran; device int32 [T, n_k]."""
    torch = _torch()
    to, k = _host_lists(task_off, ks)
    T, n_k = len(to) - 1, len(k)
    if passes is None:
        passes = torch.empty((T, n_k), dtype=torch.int32, device=workspace.device)
    _check(load().cham_sweep_passes(_dp(workspace), C.c_int64(workspace.numel()), C.c_int64(ld), C.c_int32(d),
                                    _hp(to), C.c_int32(T), _hp(k), C.c_int32(n_k), C.c_int32(flags), _dp(passes),
                                    _stream()))
    return passes


def cham_static_bytes(ld: int, d: int, task_off, ks, flags: int = 0) -> int:
    """What cham_kmeans_sweep_static counts against its limit for these arguments."""
    to, k = _host_lists(task_off, ks)
    return _check(load().cham_static_bytes(C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(len(to) - 1), _hp(k), C.c_int32(len(k)), C.c_int32(flags)))


def cham_static_init() -> None:
    _torch()
    _check(load().cham_static_init())


def cham_kmeans_sweep_static(X, ld: int, d: int, task_off, ks: Sequence[int], n_iter: int, out: dict,
                             init_centroids=None, flags: int = 0):
    """cham_kmeans_sweep on the library's static scratch buffer; ``out`` holds the caller's output tensors
    (centroids, counts, inertia, status and optionally labels, trace).  Nothing is allocated here."""
    to, k = _host_lists(task_off, ks)
    rc = load().cham_kmeans_sweep_static(_dp(X), C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(len(to) - 1), _hp(k),
                                         C.c_int32(len(k)), C.c_int32(n_iter),
                                         C.c_int32(0 if init_centroids is None else 1), _dp(init_centroids),
                                         _dp(out["centroids"]), _dp(out["counts"]), _dp(out["inertia"]),
                                         _dp(out["status"]), _dp(out.get("labels")), _dp(out.get("trace")),
                                         C.c_int32(flags), _stream())
    _check(rc)
    return out


def cham_kmeans_sweep_u16(X, ld: int, d: int, task_off, ks: Sequence[int], n_iter: int, **kw):
    """cham_kmeans_sweep for two-byte knobs: X is a device int16 tensor [d, ld] holding uint16 values."""
    return cham_kmeans_sweep(X, ld, d, task_off, ks, n_iter, _sfx="_u16", **kw)


def cham_kmeans_sweep_knee(X, ld: int, d: int, task_off, ks: Sequence[int], n_iter: int, threshold: float = 2.5,
                           chunk: int = 8, init_centroids=None, want_labels: bool = False,
                           want_trace: bool = False, flags: int = 0, out: Optional[dict] = None, workspace=None,
                           _sfx: str = ""):
    """Run the sweep in chunks and stop every task at its knee; returns the same dict plus ``chosen``."""
    torch = _torch()
    lib = load()
    assert X.dtype == _knob_dtypes(_sfx)[1]
    to, k = _host_lists(task_off, ks)
    T, n_k, Ksum = len(to) - 1, len(k), int(k.sum())
    dev = X.device
    if out is None:
        out = {}
        out["centroids"] = torch.empty((T, Ksum, d), dtype=torch.float64, device=dev)
        out["counts"] = torch.empty((T, Ksum), dtype=torch.int32, device=dev)
        out["inertia"] = torch.empty((T, n_k), dtype=torch.float64, device=dev)
        out["status"] = torch.empty((T, n_k), dtype=torch.int32, device=dev)
        out["chosen"] = torch.empty(T, dtype=torch.int32, device=dev)
        out["labels"] = torch.zeros((n_k, ld), dtype=torch.uint8, device=dev) if want_labels else None
        out["trace"] = torch.empty((T, n_k, n_iter + 1), dtype=torch.float64, device=dev) if want_trace else None
    if workspace is None:
        nbytes = cham_sweep_knee_workspace_bytes(ld, d, to, k, n_iter, flags, _sfx=_sfx)
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    rc = getattr(lib, "cham_kmeans_sweep_knee" + _sfx)(_dp(X), C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(T), _hp(k),
                                    C.c_int32(n_k), C.c_int32(n_iter), C.c_int32(0 if init_centroids is None else 1),
                                    _dp(init_centroids), C.c_double(threshold), C.c_int32(chunk),
                                    _dp(out["centroids"]), _dp(out["counts"]), _dp(out["inertia"]),
                                    _dp(out["status"]), _dp(out["chosen"]), _dp(out.get("labels")),
                                    _dp(out.get("trace")), _dp(workspace), C.c_int64(workspace.numel()),
                                    C.c_int32(flags), _stream())
    _check(rc)
    out["workspace"] = workspace
    out["koff"] = np.concatenate([[0], np.cumsum(k)]).astype(np.int64)
    return out


def cham_kmeans_sweep_knee_u16(X, ld: int, d: int, task_off, ks: Sequence[int], n_iter: int, **kw):
    return cham_kmeans_sweep_knee(X, ld, d, task_off, ks, n_iter, _sfx="_u16", **kw)


def cham_select_k(inertia, status, threshold: float = 2.5, chosen=None):
    torch = _torch()
    T, n_k = inertia.shape
    if chosen is None:
        chosen = torch.empty(T, dtype=torch.int32, device=inertia.device)
    _check(load().cham_select_k(_dp(inertia), _dp(status), C.c_int32(T), C.c_int32(n_k), C.c_double(threshold),
                                _dp(chosen), _stream()))
    return chosen


def cham_snap_centroids(X, ld: int, d: int, task_off, ks, chosen_idx, centroids, flags: int = 0,
                        out: Optional[dict] = None, workspace=None, _sfx: str = ""):
    torch = _torch()
    assert X.dtype == _knob_dtypes(_sfx)[1]
    to, k = _host_lists(task_off, ks)
    T, n_k, kmax = len(to) - 1, len(k), int(k[-1])
    dev = X.device
    if out is None:
        out = dict(labels_sel=torch.zeros(ld, dtype=torch.uint8, device=dev),
                   pick_row=torch.empty((T, kmax), dtype=torch.int32, device=dev),
                   pick_cfg=torch.empty((T, kmax, d), dtype=_knob_dtypes(_sfx)[1], device=dev))
    if workspace is None:
        nbytes = _check(getattr(load(), "cham_snap_workspace_bytes" + _sfx)(
            C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(T), _hp(k), C.c_int32(n_k)))
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    _check(getattr(load(), "cham_snap_centroids" + _sfx)(_dp(X), C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(T), _hp(k),
                                      C.c_int32(n_k), _dp(chosen_idx), _dp(centroids), _dp(out["labels_sel"]),
                                      _dp(out["pick_row"]), _dp(out["pick_cfg"]), _dp(workspace),
                                      C.c_int64(workspace.numel()), C.c_int32(flags), _stream()))
    out["workspace"] = workspace
    return out


def cham_snap_centroids_u16(X, ld: int, d: int, task_off, ks, chosen_idx, centroids, **kw):
    return cham_snap_centroids(X, ld, d, task_off, ks, chosen_idx, centroids, _sfx="_u16", **kw)


def cham_synthesize(X, ld: int, d: int, task_off, cards, valid, ks, chosen_idx, labels_sel, pick_row, pick_cfg,
                    visited, task_salt=None, out: Optional[dict] = None, workspace=None, _sfx: str = ""):
    """visited: device int64/uint64 tensor, sorted ascending as unsigned 64-bit words."""
    torch = _torch()
    assert X.dtype == _knob_dtypes(_sfx)[1] and pick_cfg.dtype == X.dtype
    to, k = _host_lists(task_off, ks)
    T, n_k, kmax = len(to) - 1, len(k), int(k[-1])
    cards = np.ascontiguousarray(cards, dtype=np.uint16).reshape(T, d)
    salts = None if task_salt is None else np.ascontiguousarray(task_salt, dtype=np.uint64)
    dev = X.device
    if out is None:
        out = dict(out_cfg=torch.empty((T, kmax, d), dtype=_knob_dtypes(_sfx)[1], device=dev),
                   out_flag=torch.empty((T, kmax), dtype=torch.uint8, device=dev),
                   out_count=torch.empty(T, dtype=torch.int32, device=dev))
    if workspace is None:
        nbytes = _check(getattr(load(), "cham_synth_workspace_bytes" + _sfx)(
            C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(T), _hp(k), C.c_int32(n_k)))
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    n_vis = 0 if visited is None else int(visited.numel())
    _check(getattr(load(), "cham_synthesize" + _sfx)(_dp(X), C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(T), _hp(cards),
                                  _dp(valid), _hp(k), C.c_int32(n_k), _dp(chosen_idx), _dp(labels_sel),
                                  _dp(pick_row), _dp(pick_cfg), _dp(visited) if n_vis else None,
                                  C.c_int64(n_vis), _hp(salts), _dp(out["out_cfg"]), _dp(out["out_flag"]),
                                  _dp(out["out_count"]), _dp(workspace), C.c_int64(workspace.numel()), _stream()))
    out["workspace"] = workspace
    return out


def cham_synthesize_u16(X, ld: int, d: int, task_off, cards, valid, ks, chosen_idx, labels_sel, pick_row,
                        pick_cfg, visited, **kw):
    return cham_synthesize(X, ld, d, task_off, cards, valid, ks, chosen_idx, labels_sel, pick_row, pick_cfg,
                           visited, _sfx="_u16", **kw)


def cham_synthesize_table(X, ld: int, d: int, task_off, cards, valid, ks, chosen_idx, labels_sel, pick_row,
                          pick_cfg, table, task_salt=None, out: Optional[dict] = None, workspace=None,
                          _sfx: str = ""):
    """cham_synthesize with the visited set held in a device table (int64/uint64 tensor of 2^m slots)."""
    torch = _torch()
    assert X.dtype == _knob_dtypes(_sfx)[1] and pick_cfg.dtype == X.dtype
    to, k = _host_lists(task_off, ks)
    T, n_k, kmax = len(to) - 1, len(k), int(k[-1])
    cards = np.ascontiguousarray(cards, dtype=np.uint16).reshape(T, d)
    salts = None if task_salt is None else np.ascontiguousarray(task_salt, dtype=np.uint64)
    dev = X.device
    if out is None:
        out = dict(out_cfg=torch.empty((T, kmax, d), dtype=_knob_dtypes(_sfx)[1], device=dev),
                   out_flag=torch.empty((T, kmax), dtype=torch.uint8, device=dev),
                   out_count=torch.empty(T, dtype=torch.int32, device=dev))
    if workspace is None:
        nbytes = _check(getattr(load(), "cham_synth_workspace_bytes" + _sfx)(
            C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(T), _hp(k), C.c_int32(n_k)))
        workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    _check(getattr(load(), "cham_synthesize_table" + _sfx)(_dp(X), C.c_int64(ld), C.c_int32(d), _hp(to), C.c_int32(T), _hp(cards),
                                        _dp(valid), _hp(k), C.c_int32(n_k), _dp(chosen_idx), _dp(labels_sel),
                                        _dp(pick_row), _dp(pick_cfg), _dp(table), C.c_int64(table.numel()),
                                        _hp(salts), _dp(out["out_cfg"]), _dp(out["out_flag"]),
                                        _dp(out["out_count"]), _dp(workspace), C.c_int64(workspace.numel()),
                                        _stream()))
    out["workspace"] = workspace
    return out


def cham_synthesize_table_u16(X, ld: int, d: int, task_off, cards, valid, ks, chosen_idx, labels_sel, pick_row,
                              pick_cfg, table, **kw):
    return cham_synthesize_table(X, ld, d, task_off, cards, valid, ks, chosen_idx, labels_sel, pick_row, pick_cfg,
                                 table, _sfx="_u16", **kw)


def cham_visited_table_clear(table):
    _check(load().cham_visited_table_clear(_dp(table), C.c_int64(table.numel()), _stream()))
    return table


def cham_visited_table_insert_hashes(table, hashes, overflow=None):
    _check(load().cham_visited_table_insert_hashes(_dp(table), C.c_int64(table.numel()), _dp(hashes),
                                                   C.c_int64(hashes.numel()), _dp(overflow), _stream()))


def cham_visited_table_insert_configs_u16(table, cfgs, d: int, **kw):
    return cham_visited_table_insert_configs(table, cfgs, d, _sfx="_u16", **kw)


def cham_visited_table_insert_configs(table, cfgs, d: int, flags=None, salts=None, rows_per_salt: int = 1,
                                      overflow=None, _sfx: str = ""):
    assert cfgs.dtype == _knob_dtypes(_sfx)[1]
    n = cfgs.numel() // d
    _check(getattr(load(), "cham_visited_table_insert_configs" + _sfx)(_dp(table), C.c_int64(table.numel()), _dp(cfgs), C.c_int64(n),
                                                    C.c_int32(d), _dp(flags), _dp(salts), C.c_int64(rows_per_salt),
                                                    _dp(overflow), _stream()))


def cham_update_configs(theta, actions, cards, salt: int = 0, seen_table=None, unique_rows=None, n_unique=None,
                        overflow=None):
    """theta [B][d] uint8 (in place), actions [S][B][d] int8, cards [d] (device int16/uint16 tensor)."""
    B, d = theta.shape
    n_steps = actions.shape[0] if actions.dim() == 3 else 1
    _check(load().cham_update_configs(_dp(theta), _dp(actions), C.c_int64(B), C.c_int32(d), C.c_int32(n_steps),
                                      _dp(cards), C.c_uint64(salt), _dp(seen_table),
                                      C.c_int64(0 if seen_table is None else seen_table.numel()), _dp(unique_rows),
                                      C.c_int64(0 if unique_rows is None else unique_rows.shape[0]), _dp(n_unique),
                                      _dp(overflow), _stream()))
    return theta


def _type_of(t, types, what: str) -> int:
    code = types.get(t.dtype)
    if code is None:
        raise ChamError(f"{what}: {t.dtype} is not one of {', '.join(map(str, types))}")
    return code


def _stream_of(t, what: str):
    """(device, its index, its current stream) of a tensor on the current device (kernels are launched there)."""
    torch = _torch()
    index = t.get_device()
    if index < 0 or index != torch._C._cuda_getDevice():
        raise ChamError(f"{what}: on {t.device}, current device cuda:{torch.cuda.current_device()}")
    return t.device, index, torch._C._cuda_getCurrentRawStream(index)


def _addr(t, index: int, what: str, dtype, shape):
    """Address of an optional tensor that has to lie on the device with this index, dense, with this type and shape."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == index and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    raise ChamError(f"{what}: need a dense {dtype} tensor of shape {tuple(shape)} on cuda:{index}, "
                    f"got {t.dtype} {tuple(t.shape)} strides {t.stride()} on {t.device}")


def _scratch(workspace, device, index: int, nbytes, *sizes):
    """The caller's workspace, or one of nbytes(*sizes) bytes; and its address."""
    if workspace is None:
        workspace = _torch().empty(max(nbytes(*sizes), 256), dtype=_torch().uint8, device=device)
    elif workspace.get_device() != index or not workspace.is_contiguous() or workspace.element_size() != 1:
        raise ChamError(f"workspace: need dense bytes on {device}, got {workspace.dtype} strides {workspace.stride()} on {workspace.device}")
    return workspace, workspace.data_ptr()


def _heads(logits, what: str):
    """(R, G, V, ld_r, ld_g) of logits [R, V] or [R, G, V] whose choices are consecutive."""
    shape, stride = logits.shape, logits.stride()
    if len(shape) not in (2, 3) or (stride[-1] != 1 and shape[-1] > 1):
        raise ChamError(f"{what}: need [R, V] or [R, G, V] with consecutive choices, got {tuple(shape)} strides {stride}")
    return (shape[0], 1, shape[1], stride[0], 0) if len(shape) == 2 else (*shape, stride[0], stride[1])


def cham_policy_workspace_bytes(R: int, G: int, V: int, type: int, want_grad: bool) -> int:
    return _check(load().cham_policy_workspace_bytes(R, G, V, type, 1 if want_grad else 0))


def cham_policy_logp(logits, actions, first_action: int = 0, weights=None, out: Optional[dict] = None, workspace=None):
    """Log-probability of the actions and entropy per decision.  logits [R, V] or [R, G, V] (f32, bf16, f16; choices
    consecutive), actions [R] or [R, G] (int8, int32, int64); returns a dict of float tensors logp [R], entropy [R]."""
    torch = _torch()
    dev, index, stream = _stream_of(logits, "logits")
    R, G, V, ld_r, ld_g = _heads(logits, "logits")
    code = _type_of(logits, _FLOAT_TYPES, "logits")
    acts = _addr(actions, index, "actions", actions.dtype, logits.shape[:-1])
    out = dict(out) if out is not None else dict(logp=torch.empty(R, dtype=torch.float32, device=dev), entropy=torch.empty(R, dtype=torch.float32, device=dev))
    workspace, at = _scratch(workspace, dev, index, cham_policy_workspace_bytes, R, G, V, code, False)
    _check(load().cham_policy_logp(logits.data_ptr(), code, R, G, V, ld_r, ld_g, acts, _type_of(actions, _ACTION_TYPES, "actions"), first_action,
                                   _addr(weights, index, "weights", torch.float32, (R,)), _addr(out["logp"], index, "logp", torch.float32, (R,)),
                                   _addr(out.get("entropy"), index, "entropy", torch.float32, (R,)), at, workspace.numel(), stream))
    out["workspace"] = workspace
    return out


def cham_policy_loss(logits, actions, old_logp, advantages, first_action: int = 0, ref_logp=None, weights=None, values=None, old_values=None,
                     returns=None, clip_low: float = 0.2, clip_high: float = 0.2, value_coef: float = 0.0, entropy_coef: float = 0.0,
                     kl_coef: float = 0.0, value_clip: float = 0.2, want_grad: bool = True, out: Optional[dict] = None, workspace=None):
    """Clipped policy loss and its gradients; returns a dict of device tensors: terms [6] (names: TERMS), logp and entropy [R],
    grad_logits (like logits) and grad_values [R] (None without want_grad, or without values).  ``out`` holds the caller's
    tensors under these names; out["grad_logits"] may be the logits themselves."""
    torch = _torch()
    dev, index, stream = _stream_of(logits, "logits")
    R, G, V, ld_r, ld_g = _heads(logits, "logits")
    code = _type_of(logits, _FLOAT_TYPES, "logits")
    f32 = torch.float32
    acts = _addr(actions, index, "actions", actions.dtype, logits.shape[:-1])
    if out is None:
        rows = torch.empty((2, R), dtype=f32, device=dev)
        out = dict(terms=torch.empty(len(TERMS), dtype=f32, device=dev), logp=rows[0], entropy=rows[1],
                   grad_logits=torch.empty(logits.shape, dtype=logits.dtype, device=dev) if want_grad else None,
                   grad_values=torch.empty(R, dtype=f32, device=dev) if want_grad and values is not None else None)
    else:
        out = dict(out)
    grad = out.get("grad_logits") if want_grad else None
    gld_r = gld_g = 0
    if grad is not None:
        if grad.dtype is not logits.dtype or grad.shape != logits.shape or grad.get_device() != index:
            raise ChamError(f"grad_logits: need {logits.dtype} {tuple(logits.shape)} on {dev}, got {grad.dtype} {tuple(grad.shape)} on {grad.device}")
        _, _, _, gld_r, gld_g = _heads(grad, "grad_logits")
    row = (R,)
    rows = (weights, old_logp, advantages, ref_logp, values, old_values, returns, out.get("logp"), out.get("entropy"),
            out.get("grad_values") if want_grad else None)
    at = []
    for i, t in enumerate(rows):                        # as _addr, ten of them a call
        if t is None:
            at.append(None)
        elif t.dtype is f32 and t.get_device() == index and t.shape == row and t.is_contiguous():
            at.append(t.data_ptr())
        else:
            _addr(t, index, _LOSS_ROWS[i], f32, row)
    coef = _PolicyCoef(clip_low, clip_high, value_coef, entropy_coef, kl_coef, value_clip)
    workspace, ws = _scratch(workspace, dev, index, cham_policy_workspace_bytes, R, G, V, code, grad is not None)
    _check(load().cham_policy_loss(
        logits.data_ptr(), code, R, G, V, ld_r, ld_g, acts, _type_of(actions, _ACTION_TYPES, "actions"), first_action, *at[:7], coef,
        _addr(out["terms"], index, "terms", f32, (len(TERMS),)), at[7], at[8], None if grad is None else grad.data_ptr(), gld_r, gld_g, at[9],
        ws, workspace.numel(), stream))
    out["workspace"] = workspace
    return out


_LOSS_ROWS = ("weights", "old_logp", "advantages", "ref_logp", "values", "old_values", "returns", "logp", "entropy", "grad_values")


def _matrix(t, index: int, what: str, dtype, shape):
    """(address, stride of trajectories, stride of steps) of an optional [B, S] tensor of any strides."""
    if t is None:
        return None, 0, 0
    if t.get_device() != index or t.dtype is not dtype or t.shape != shape:
        raise ChamError(f"{what}: need {dtype} {tuple(shape)} on cuda:{index}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return (t.data_ptr(), *t.stride())


def cham_gae_workspace_bytes(B: int, S: int) -> int:
    return _check(load().cham_gae_workspace_bytes(B, S))


def cham_gae(rewards, values, gamma: float, lam: float, dones=None, bootstrap=None, lengths=None, out: Optional[dict] = None, workspace=None):
    """Advantages and returns [B, S] of trajectories; rewards and values [B, S] of one type (f32, bf16, f16), dones uint8
    or bool [B, S], bootstrap float [B], lengths int32 [B].  Any strides: steps that are stored first ([S, B]) are passed as ``t()``.
    ``out`` holds advantages and returns (float, of one layout; returns may be None); without it they are made like
    rewards, zero behind a length."""
    torch = _torch()
    dev, index, stream = _stream_of(rewards, "rewards")
    if rewards.dim() != 2:
        raise ChamError(f"rewards: need [B, S], got {tuple(rewards.shape)}")
    B, S = shape = rewards.shape
    code = _type_of(rewards, _FLOAT_TYPES, "rewards")
    if dones is not None and dones.dtype == torch.bool:
        dones = dones.view(torch.uint8)
    if out is None:
        make = torch.empty if lengths is None else torch.zeros
        pair = make((2, S, B), dtype=torch.float32, device=dev).transpose(1, 2) if rewards.stride(0) < rewards.stride(1) else make((2, B, S), dtype=torch.float32, device=dev)
        out = dict(advantages=pair[0], returns=pair[1])
    else:
        out = dict(out)
    r, r_b, r_s = _matrix(rewards, index, "rewards", rewards.dtype, shape)
    v, v_b, v_s = _matrix(values, index, "values", rewards.dtype, shape)
    d, d_b, d_s = _matrix(dones, index, "dones", torch.uint8, shape)
    adv, o_b, o_s = _matrix(out["advantages"], index, "advantages", torch.float32, shape)
    ret, q_b, q_s = _matrix(out.get("returns"), index, "returns", torch.float32, shape)
    if ret is not None and (q_b, q_s) != (o_b, o_s):
        raise ChamError("returns: need the strides of advantages")
    workspace, at = _scratch(workspace, dev, index, cham_gae_workspace_bytes, B, S)
    _check(load().cham_gae(code, B, S, r, r_b, r_s, v, v_b, v_s, d, d_b, d_s, _addr(bootstrap, index, "bootstrap", torch.float32, (B,)),
                           _addr(lengths, index, "lengths", torch.int32, (B,)), gamma, lam, adv, ret, o_b, o_s,
                           at, workspace.numel(), stream))
    out["workspace"] = workspace
    return out


class GradList:
    """Addresses, sizes and types of a list of dense tensors on one device, for programs that clip the same tensors in every
    step.  It keeps the tensors alive; a tensor whose storage is replaced needs a new list (gradients that are set to None between steps
    are new tensors in the next)."""

    def __init__(self, tensors):
        _torch()
        self.tensors = list(tensors)
        n = len(self.tensors)
        self.n = n
        self.device = self.tensors[0].device if n else None
        codes = []
        for i, t in enumerate(self.tensors):
            if t.device != self.device or not t.is_contiguous():
                raise ChamError(f"tensor {i}: need dense tensors on one device, got strides {t.stride()} on {t.device}")
            codes.append(_type_of(t, _FLOAT_TYPES, f"tensor {i}"))
        self.ptrs = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in self.tensors])
        self.numels = (C.c_int64 * max(n, 1))(*[t.numel() for t in self.tensors])
        spans = sorted((p, p + m * (4 if code == TYPE_F32 else 2)) for p, m, code in zip(self.ptrs, self.numels, codes) if m > 0)
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ChamError("tensors of the list share memory")
        self.types = (C.c_int32 * max(n, 1))(*codes)
        self.sizes = bytes(self.numels) + bytes(self.types)
        self.workspace_bytes = _check(load().cham_grad_workspace_bytes(self.numels, self.types, n))


def _grad_call(grads, norm, workspace):
    torch = _torch()
    grads = grads if isinstance(grads, GradList) else GradList(grads)
    if norm is None:
        norm = torch.empty(1, dtype=torch.float64, device=grads.device if grads.n else "cuda")
    dev, index, stream = _stream_of(norm, "norm")
    if grads.n and grads.device != dev:
        raise ChamError(f"gradients on {grads.device}, current device {dev}")
    workspace, at = _scratch(workspace, dev, index, int, grads.workspace_bytes)
    return grads, norm, _addr(norm, index, "norm", torch.float64, (1,)), workspace, at, stream


def cham_grad_workspace_bytes(grads) -> int:
    return (grads if isinstance(grads, GradList) else GradList(grads)).workspace_bytes


def cham_grad_norm(grads, norm=None, workspace=None):
    """Norm of all tensors of ``grads`` (a GradList or a list of tensors) together; returns a dict: norm (double [1])."""
    grads, norm, norm_at, workspace, at, stream = _grad_call(grads, norm, workspace)
    _check(load().cham_grad_norm(grads.ptrs, grads.numels, grads.types, grads.n, norm_at, at, workspace.numel(), stream))
    return dict(norm=norm, workspace=workspace)


def cham_clip_grads(grads, max_norm: float, out=None, norm=None, norm_given: bool = False, workspace=None):
    """Scales ``grads`` (a GradList or a list of tensors) to a norm of at most max_norm, in place or into the tensors of
    ``out``; norm_given: ``norm`` is read instead of computed.  Returns a dict: norm (double [1], before clipping)."""
    if norm_given and norm is None:
        raise ChamError("norm_given without a norm")
    grads, norm, norm_at, workspace, at, stream = _grad_call(grads, norm, workspace)
    outs = None
    if out is not None:
        out = out if isinstance(out, GradList) else GradList(out)
        if out.sizes != grads.sizes or (out.n and out.device != grads.device):
            raise ChamError("out: need tensors of the same sizes, types and device as the gradients")
        outs = out.ptrs
    _check(load().cham_clip_grads(grads.ptrs, outs, grads.numels, grads.types, grads.n, max_norm, norm_at, at, workspace.numel(),
                                  F_NORM_GIVEN if norm_given else 0, stream))
    return dict(norm=norm, workspace=workspace)


class DeviceWorkload:
    """A workload's inputs resident on the GPU, plus a driver for the whole path."""

    def __init__(self, wl, device="cuda:0"):
        torch = _torch()
        self.wl = wl
        self.device = device
        self.X, self.ld = to_soa(wl.rows, device)
        self.sfx = "_u16" if wl.rows.dtype == np.uint16 else ""      # which family of entry points
        self.d = wl.d
        v = np.zeros(self.ld, dtype=np.uint8)
        v[:wl.n_total] = wl.valid
        self.valid = torch.from_numpy(v).to(device)
        self.visited = None

    def build_visited(self):
        """Hash the visited configurations on the device and sort them (input preparation)."""
        torch = _torch()
        from . import workloads
        wl = self.wl
        if len(wl.visited_cfg):
            host = np.ascontiguousarray(wl.visited_cfg)
            rows = torch.from_numpy(host.view(np.int16) if self.sfx else host).to(self.device)
            salts = torch.from_numpy(wl.salts[wl.visited_task].astype(np.int64)).to(self.device)
            h = cham_hash_rows(rows, salts, _sfx=self.sfx).cpu().numpy().view(np.uint64)
        else:
            h = np.zeros(0, dtype=np.uint64)
        arr = workloads.finalize_visited(h, wl.visited_raw, wl.n_visited)
        self.visited_host = arr
        self.visited = torch.from_numpy(arr.view(np.int64).copy()).to(self.device)
        return self.visited

    def run(self, threshold: Optional[float] = None, flags: int = 0, want_labels: bool = False,
            want_trace: bool = False, bufs: Optional[dict] = None):
        """sweep -> select -> snap -> synthesize on the current stream; no host synchronisation."""
        wl = self.wl
        thr = wl.threshold if threshold is None else threshold
        if self.visited is None:
            self.build_visited()
        b = bufs or {}
        # two-byte knobs: cardinalities of at most 2048 are the caller's promise of values below 2048
        sweep_flags = flags | (F_VALUES_BELOW_2048 if self.sfx and int(np.max(wl.cards)) <= 2048 else 0)
        sw = cham_kmeans_sweep(self.X, self.ld, self.d, wl.task_off, wl.ks, wl.n_iter, flags=sweep_flags,
                               want_labels=want_labels, want_trace=want_trace,
                               out=b.get("sweep"), workspace=b.get("sweep_ws"), _sfx=self.sfx)
        chosen = cham_select_k(sw["inertia"], sw["status"], thr, chosen=b.get("chosen"))
        sn = cham_snap_centroids(self.X, self.ld, self.d, wl.task_off, wl.ks, chosen, sw["centroids"],
                                 flags=flags, out=b.get("snap"), workspace=b.get("snap_ws"), _sfx=self.sfx)
        sy = cham_synthesize(self.X, self.ld, self.d, wl.task_off, wl.cards, self.valid, wl.ks, chosen,
                             sn["labels_sel"], sn["pick_row"], sn["pick_cfg"], self.visited,
                             task_salt=wl.salts, out=b.get("synth"), workspace=b.get("synth_ws"), _sfx=self.sfx)
        return dict(sweep=sw, chosen=chosen, snap=sn, synth=sy)
