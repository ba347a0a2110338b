"""Thin ctypes binding of `libfamilyseer.so` (see include/familyseer.h).

Only argument marshalling lives here: every step of scoring and of the top-k cut runs
in the library's HIP kernels.  PyTorch supplies device memory and the current stream.
The functions carry the names of the C entry points they call.  There is no CPU
fallback: if the library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfamilyseer.so")

FS_OK, FS_EINVAL, FS_ENOMEM, FS_EDEVICE, FS_EUNSUPPORTED = 0, -1, -2, -3, -4
FS_ROWMAJOR, FS_COLBLOCK64 = 0, 1
FS_MAX_TOPK = 16384
FS_MAX_FEATURES = 4096
FS_MAX_TREE_NODES = 65535

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it first (python -m paper_2201_00194_amd.build); "
        "there is no fallback path")

_lib = ctypes.CDLL(LIB_PATH)


class FsError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"familyseer error {code}: {message}")
        self.code = code


class _FsFamily(ctypes.Structure):
    _fields_ = [("model", ctypes.c_void_p), ("features", ctypes.c_void_p),
                ("layout", ctypes.c_int32), ("n_rows", ctypes.c_int64),
                ("prog_off", ctypes.c_void_p), ("n_programs", ctypes.c_int32),
                ("prog_score", ctypes.c_void_p), ("row_score", ctypes.c_void_p),
                ("leaf_idx", ctypes.c_void_p)]


class _FsTopkReq(ctypes.Structure):
    _fields_ = [("score", ctypes.c_void_p), ("n", ctypes.c_int32), ("k", ctypes.c_int32),
                ("out_idx", ctypes.c_void_p), ("out_score", ctypes.c_void_p)]


_i32p = ctypes.POINTER(ctypes.c_int32)
_f32p = ctypes.POINTER(ctypes.c_float)
_lib.fs_last_error.restype = ctypes.c_char_p
_lib.fs_last_error.argtypes = []
_lib.fs_version.restype = ctypes.c_int
_lib.fs_version.argtypes = []
_lib.fs_model_create.restype = ctypes.c_int
_lib.fs_model_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.c_int32,
                                 _i32p, _i32p, _f32p, _i32p, _i32p, _f32p, ctypes.c_float]
_lib.fs_model_destroy.restype = None
_lib.fs_model_destroy.argtypes = [ctypes.c_void_p]
_lib.fs_score_families.restype = ctypes.c_int
_lib.fs_score_families.argtypes = [ctypes.c_int32, ctypes.POINTER(_FsFamily), ctypes.c_void_p]
_lib.fs_topk.restype = ctypes.c_int
_lib.fs_topk.argtypes = [ctypes.c_int32, ctypes.POINTER(_FsTopkReq), ctypes.c_void_p]
_lib.fs_topk_noalloc.restype = ctypes.c_int
_lib.fs_topk_noalloc.argtypes = [ctypes.c_int32, ctypes.POINTER(_FsTopkReq), ctypes.c_void_p]
_lib.fs_pack_colblock64.restype = ctypes.c_int
_lib.fs_pack_colblock64.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32,
                                    ctypes.c_void_p, ctypes.c_void_p]
_lib.fs_colblock64_floats.restype = ctypes.c_int64
_lib.fs_colblock64_floats.argtypes = [ctypes.c_int64, ctypes.c_int32]


_lib.fs_workspace_bytes.restype = ctypes.c_size_t
_lib.fs_workspace_bytes.argtypes = [ctypes.c_int32, ctypes.POINTER(_FsFamily)]
_lib.fs_topk_workspace_bytes.restype = ctypes.c_size_t
_lib.fs_topk_workspace_bytes.argtypes = [ctypes.c_int32, ctypes.POINTER(_FsTopkReq)]
_lib.fs_workspace_reserve.restype = ctypes.c_int
_lib.fs_workspace_reserve.argtypes = [ctypes.c_size_t, ctypes.c_size_t]
_lib.fs_tune_set.restype = ctypes.c_int
_lib.fs_tune_set.argtypes = [ctypes.c_int32, ctypes.c_int32]
_lib.fs_tune_get.restype = ctypes.c_int32
_lib.fs_tune_get.argtypes = [ctypes.c_int32]
(FS_TUNE_LDS_TILES, FS_TUNE_LDS_MODE, FS_TUNE_RANK, FS_TUNE_RANK_TILES, FS_TUNE_VERBOSE,
 FS_TUNE_TRAIN_SLAB_ROWS, FS_TUNE_TRAIN_SORT, FS_TUNE_TRAIN_PACKED, FS_TUNE_LDS_GROUPS,
 FS_TUNE_TREELET, FS_TUNE_TREELET_FORM, FS_TUNE_TRAIN_WORK_MB) = range(12)
FS_TUNE_OPTIONS = 12

_lib.fs_profile_begin.restype = ctypes.c_int
_lib.fs_profile_begin.argtypes = [ctypes.c_int32]
_lib.fs_profile_end.restype = ctypes.c_int
_lib.fs_profile_end.argtypes = [ctypes.POINTER(ctypes.c_double), _i32p]
KERNEL_CLASSES = ("traverse", "segsum", "topk", "pack", "traverse_global", "rank_code",
                  "traverse_rank", "train_hist", "train_split", "train_other")


def _check(rc: int) -> None:
    if rc != FS_OK:
        raise FsError(rc, _lib.fs_last_error().decode("utf-8", "replace"))


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> ctypes.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def fs_version() -> int:
    return int(_lib.fs_version())


def fs_last_error() -> str:
    return _lib.fs_last_error().decode("utf-8", "replace")


class fs_model:
    """Owner of one `fs_model*` (one family's ensemble, device resident)."""

    def __init__(self, n_features: int, tree_off, split_feature, threshold, left, right, value,
                 bias: float = 0.0):
        to = np.ascontiguousarray(tree_off, dtype=np.int32)
        sf = np.ascontiguousarray(split_feature, dtype=np.int32)
        th = np.ascontiguousarray(threshold, dtype=np.float32)
        le = np.ascontiguousarray(left, dtype=np.int32)
        ri = np.ascontiguousarray(right, dtype=np.int32)
        va = np.ascontiguousarray(value, dtype=np.float32)
        n_trees = int(to.shape[0]) - 1
        handle = ctypes.c_void_p()
        rc = _lib.fs_model_create(
            ctypes.byref(handle), int(n_features), n_trees,
            to.ctypes.data_as(_i32p), sf.ctypes.data_as(_i32p), th.ctypes.data_as(_f32p),
            le.ctypes.data_as(_i32p), ri.ctypes.data_as(_i32p), va.ctypes.data_as(_f32p),
            ctypes.c_float(bias))
        _check(rc)
        self._h = handle
        self.n_features = int(n_features)
        self.n_trees = n_trees

    @classmethod
    def from_arrays(cls, m) -> "fs_model":
        """From any object with the fields of `workloads.Model`."""
        return cls(m.n_features, m.tree_off, m.split_feature, m.threshold, m.left, m.right,
                   m.value, m.bias)

    def destroy(self) -> None:
        if getattr(self, "_h", None) is not None and self._h:
            _lib.fs_model_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class Family:
    """Argument bundle for one `fs_family` entry; tensors live on the device."""

    def __init__(self, model: fs_model, features: torch.Tensor, layout: int, n_rows: int,
                 prog_off: torch.Tensor, prog_score: torch.Tensor,
                 row_score: Optional[torch.Tensor] = None,
                 leaf_idx: Optional[torch.Tensor] = None):
        self.model, self.features, self.layout, self.n_rows = model, features, layout, int(n_rows)
        self.prog_off, self.prog_score = prog_off, prog_score
        self.row_score, self.leaf_idx = row_score, leaf_idx
        self.n_programs = int(prog_off.shape[0]) - 1 if prog_off is not None else 0


def _family_array(fams: Sequence[Family]):
    arr = (_FsFamily * max(1, len(fams)))()
    for i, f in enumerate(fams):
        arr[i].model = f.model._h if f.model is not None else None
        arr[i].features = _ptr(f.features)
        arr[i].layout = f.layout
        arr[i].n_rows = f.n_rows
        arr[i].prog_off = _ptr(f.prog_off)
        arr[i].n_programs = f.n_programs
        arr[i].prog_score = _ptr(f.prog_score)
        arr[i].row_score = _ptr(f.row_score)
        arr[i].leaf_idx = _ptr(f.leaf_idx)
    return arr


class PreparedFamilies:
    """A family array marshalled once, for callers that submit the same set repeatedly."""

    def __init__(self, fams: Sequence[Family]):
        self.fams = list(fams)
        self.arr = _family_array(self.fams)
        self.n = len(self.fams)


def fs_score_families(fams, stream: Optional[torch.cuda.Stream] = None) -> None:
    if not isinstance(fams, PreparedFamilies):
        fams = PreparedFamilies(fams)
    _check(_lib.fs_score_families(fams.n, fams.arr, _stream_ptr(stream)))


class TopkRequest:
    def __init__(self, score: Optional[torch.Tensor], n: int, k: int, out_idx: torch.Tensor,
                 out_score: Optional[torch.Tensor] = None):
        self.score, self.n, self.k, self.out_idx, self.out_score = score, int(n), int(k), out_idx, out_score


class PreparedTopk:
    def __init__(self, reqs: Sequence[TopkRequest]):
        self.reqs = list(reqs)
        self.n = len(self.reqs)
        self.arr = (_FsTopkReq * max(1, self.n))()
        for i, r in enumerate(self.reqs):
            self.arr[i].score = _ptr(r.score)
            self.arr[i].n = r.n
            self.arr[i].k = r.k
            self.arr[i].out_idx = _ptr(r.out_idx)
            self.arr[i].out_score = _ptr(r.out_score)


def fs_topk(reqs, stream: Optional[torch.cuda.Stream] = None) -> None:
    if not isinstance(reqs, PreparedTopk):
        reqs = PreparedTopk(reqs)
    _check(_lib.fs_topk(reqs.n, reqs.arr, _stream_ptr(stream)))


def fs_topk_noalloc(reqs, stream: Optional[torch.cuda.Stream] = None) -> None:
    if not isinstance(reqs, PreparedTopk):
        reqs = PreparedTopk(reqs)
    _check(_lib.fs_topk_noalloc(reqs.n, reqs.arr, _stream_ptr(stream)))


def fs_workspace_bytes(fams) -> int:
    if not isinstance(fams, PreparedFamilies):
        fams = PreparedFamilies(fams)
    return int(_lib.fs_workspace_bytes(fams.n, fams.arr))


def fs_topk_workspace_bytes(reqs) -> int:
    if not isinstance(reqs, PreparedTopk):
        reqs = PreparedTopk(reqs)
    return int(_lib.fs_topk_workspace_bytes(reqs.n, reqs.arr))


def fs_workspace_reserve(score_bytes: int, topk_bytes: int) -> None:
    _check(_lib.fs_workspace_reserve(int(score_bytes), int(topk_bytes)))


def fs_tune_set(option: int, value: int) -> None:
    _check(_lib.fs_tune_set(int(option), int(value)))


def fs_tune_get(option: int) -> int:
    return int(_lib.fs_tune_get(int(option)))


def fs_colblock64_floats(n_rows: int, n_features: int) -> int:
    return int(_lib.fs_colblock64_floats(int(n_rows), int(n_features)))


def fs_pack_colblock64(rowmajor: torch.Tensor, n_rows: int, n_features: int,
                       out: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    if out is None:
        out = torch.empty(fs_colblock64_floats(n_rows, n_features), dtype=torch.float32,
                          device=rowmajor.device)
    _check(_lib.fs_pack_colblock64(_ptr(rowmajor), int(n_rows), int(n_features), _ptr(out),
                                   _stream_ptr(stream)))
    return out


def fs_profile_begin(max_records: int) -> None:
    _check(_lib.fs_profile_begin(int(max_records)))


def fs_profile_end() -> dict:
    """{kernel class: (total ms, timed launches)}"""
    ms = (ctypes.c_double * len(KERNEL_CLASSES))()
    cnt = (ctypes.c_int32 * len(KERNEL_CLASSES))()
    _check(_lib.fs_profile_end(ms, cnt))
    return {name: (float(ms[i]), int(cnt[i])) for i, name in enumerate(KERNEL_CLASSES)}


# ---- conveniences for tests and the benchmark (allocation + marshalling only) ---------------

def upload_case(case, layout: int = FS_COLBLOCK64, **kw):
    """One `DeviceFamily` per entry of `case.families`; entries that share a host `Model`
    object share one `fs_model`."""
    models, out = {}, []
    for f in case.families:
        key = id(f.model)
        if key not in models:
            models[key] = fs_model.from_arrays(f.model)
        out.append(DeviceFamily(f, layout=layout, model=models[key], **kw))
    return out


class DeviceFamily:
    """Uploads one `workloads.Family` and allocates its outputs."""

    def __init__(self, fam, layout: int = FS_COLBLOCK64, device: str = "cuda:0",
                 want_row_score: bool = False, want_leaf_idx: bool = False, model=None):
        """`model`: an existing `fs_model` to use (families that share a cost model) instead
        of building one from `fam.model`."""
        dev = torch.device(device)
        self.host = fam
        self.model = model if model is not None else fs_model.from_arrays(fam.model)
        self.n_rows, self.n_programs, self.k = fam.n_rows, fam.n_programs, fam.k
        x = torch.from_numpy(np.ascontiguousarray(fam.features)).to(dev)
        if x.numel() == 0:
            x = torch.zeros(4, dtype=torch.float32, device=dev)
        if layout == FS_COLBLOCK64 and fam.n_rows > 0:
            self.features = fs_pack_colblock64(x, fam.n_rows, fam.model.n_features)
            torch.cuda.synchronize()
            del x
        else:
            self.features = x
        self.layout = layout
        self.prog_off = torch.from_numpy(np.ascontiguousarray(fam.prog_off, dtype=np.int32)).to(dev)
        self.prog_score = torch.full((max(1, fam.n_programs),), float("nan"), dtype=torch.float32,
                                     device=dev)
        self.row_score = (torch.full((max(1, fam.n_rows),), float("nan"), dtype=torch.float32,
                                     device=dev) if want_row_score else None)
        self.leaf_idx = (torch.full((max(1, fam.n_rows * fam.model.n_trees),), -1,
                                    dtype=torch.int16, device=dev) if want_leaf_idx else None)
        self.topk_idx = torch.full((max(1, fam.k),), -7, dtype=torch.int32, device=dev)
        self.topk_score = torch.full((max(1, fam.k),), float("nan"), dtype=torch.float32, device=dev)

    def family(self) -> Family:
        return Family(self.model, self.features, self.layout, self.n_rows, self.prog_off,
                      self.prog_score, self.row_score, self.leaf_idx)

    def topk_request(self) -> TopkRequest:
        return TopkRequest(self.prog_score, self.n_programs, self.k, self.topk_idx, self.topk_score)


# ---- training (familyseer_train.h) -------------------------------------------------------------

FS_TRAIN_MAX_DEPTH = 10
FS_TRAIN_MAX_CUTS = 255


class _FsTrainParams(ctypes.Structure):
    _fields_ = [("max_depth", ctypes.c_int32), ("eta", ctypes.c_float), ("lam", ctypes.c_float),
                ("min_gain", ctypes.c_float), ("min_child_weight", ctypes.c_float),
                ("grad_scale", ctypes.c_float)]


_lib.fs_trainer_create.restype = ctypes.c_int
_lib.fs_trainer_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.c_void_p,
                                   ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int32,
                                   ctypes.c_void_p, _i32p, _f32p, ctypes.c_float, ctypes.c_int32,
                                   ctypes.c_int32, ctypes.c_void_p]
_lib.fs_trainer_destroy.restype = None
_lib.fs_trainer_destroy.argtypes = [ctypes.c_void_p]
_lib.fs_train_boost.restype = ctypes.c_int
_lib.fs_train_boost.argtypes = [ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32,
                                ctypes.POINTER(_FsTrainParams), ctypes.c_void_p]
_lib.fs_trainer_size.restype = ctypes.c_int
_lib.fs_trainer_size.argtypes = [ctypes.c_void_p, _i32p, ctypes.POINTER(ctypes.c_int64), ctypes.c_void_p]
_lib.fs_trainer_export.restype = ctypes.c_int
_lib.fs_trainer_export.argtypes = [ctypes.c_void_p, _i32p, _i32p, _f32p, _i32p, _i32p, _f32p,
                                   ctypes.c_void_p]
_lib.fs_trainer_predictions.restype = ctypes.c_int
_lib.fs_trainer_predictions.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]


def train_params(max_depth: int = 6, eta: float = 0.3, lam: float = 1.0, min_gain: float = 0.0,
                 min_child_weight: float = 1.0, grad_scale: float = float(1 << 20)) -> _FsTrainParams:
    return _FsTrainParams(max_depth, eta, lam, min_gain, min_child_weight, grad_scale)


class fs_trainer:
    """Owner of one `fs_trainer*`: a family's measured programs, binned, and the model so far."""

    def __init__(self, n_features: int, features: torch.Tensor, layout: int, n_rows: int,
                 prog_off: torch.Tensor, n_programs: int, target: torch.Tensor, cut_off, cuts,
                 bias: float = 0.0, max_depth: int = 6, max_trees: int = 64,
                 stream: Optional[torch.cuda.Stream] = None):
        co = np.ascontiguousarray(cut_off, dtype=np.int32)
        cu = np.ascontiguousarray(cuts, dtype=np.float32)
        if cu.size == 0:
            cu = np.zeros(1, np.float32)
        self.handle = ctypes.c_void_p()
        self.n_features, self.n_rows, self.n_programs, self.bias = n_features, n_rows, n_programs, bias
        _check(_lib.fs_trainer_create(ctypes.byref(self.handle), n_features, _ptr(features), layout,
                                      n_rows, _ptr(prog_off), n_programs, _ptr(target),
                                      co.ctypes.data_as(_i32p), cu.ctypes.data_as(_f32p), bias,
                                      max_depth, max_trees, _stream_ptr(stream)))

    @classmethod
    def from_train_set(cls, ts, layout: int = FS_COLBLOCK64, device: str = "cuda:0", **kw):
        dev = torch.device(device)
        x = torch.from_numpy(np.ascontiguousarray(ts.features)).to(dev)
        if layout == FS_COLBLOCK64:
            x = fs_pack_colblock64(x, ts.n_rows, ts.features.shape[1])
        off = torch.from_numpy(np.ascontiguousarray(ts.prog_off, dtype=np.int32)).to(dev)
        y = torch.from_numpy(np.ascontiguousarray(ts.target, dtype=np.float32)).to(dev)
        t = cls(ts.features.shape[1], x, layout, ts.n_rows, off, ts.n_programs, y, ts.cut_off,
                ts.cuts, **kw)
        torch.cuda.synchronize()          # the inputs may be freed once they are binned
        return t

    def size(self, stream: Optional[torch.cuda.Stream] = None):
        nt, nn = ctypes.c_int32(), ctypes.c_int64()
        _check(_lib.fs_trainer_size(self.handle, ctypes.byref(nt), ctypes.byref(nn), _stream_ptr(stream)))
        return int(nt.value), int(nn.value)

    def export(self, stream: Optional[torch.cuda.Stream] = None):
        """(tree_off, split_feature, threshold, left, right, value) as numpy arrays."""
        nt, nn = self.size(stream)
        to = np.zeros(nt + 1, np.int32)
        sf, le, ri = (np.zeros(max(1, nn), np.int32) for _ in range(3))
        th, va = (np.zeros(max(1, nn), np.float32) for _ in range(2))
        _check(_lib.fs_trainer_export(self.handle, to.ctypes.data_as(_i32p), sf.ctypes.data_as(_i32p),
                                      th.ctypes.data_as(_f32p), le.ctypes.data_as(_i32p),
                                      ri.ctypes.data_as(_i32p), va.ctypes.data_as(_f32p),
                                      _stream_ptr(stream)))
        return to, sf[:nn], th[:nn], le[:nn], ri[:nn], va[:nn]

    def predictions(self, stream: Optional[torch.cuda.Stream] = None):
        rows = torch.empty(self.n_rows, dtype=torch.float32, device="cuda")
        progs = torch.empty(self.n_programs, dtype=torch.float32, device="cuda")
        _check(_lib.fs_trainer_predictions(self.handle, _ptr(rows), _ptr(progs), _stream_ptr(stream)))
        return rows, progs

    def destroy(self) -> None:
        if self.handle:
            _lib.fs_trainer_destroy(self.handle)
            self.handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def fs_train_boost(trainers, n_rounds: int, params: _FsTrainParams,
                   stream: Optional[torch.cuda.Stream] = None) -> None:
    arr = (ctypes.c_void_p * max(1, len(trainers)))(*[t.handle for t in trainers])
    _check(_lib.fs_train_boost(len(trainers), arr, n_rounds, ctypes.byref(params), _stream_ptr(stream)))


# ---- population compaction ----------------------------------------------------------------------

class _FsGatherSrc(ctypes.Structure):
    _fields_ = [("features", ctypes.c_void_p), ("prog_off", ctypes.c_void_p),
                ("score", ctypes.c_void_p), ("n_programs", ctypes.c_int32)]


_lib.fs_gather_programs.restype = ctypes.c_int
_lib.fs_gather_programs.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(_FsGatherSrc),
                                    ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64,
                                    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]


def fs_gather_programs(n_features: int, sources, keep: torch.Tensor, n_keep: int,
                       out_features: torch.Tensor, out_row_capacity: int,
                       out_prog_off: torch.Tensor, out_score: Optional[torch.Tensor],
                       status: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """`sources`: sequence of (features, prog_off, score-or-None, n_programs) device tensors."""
    arr = (_FsGatherSrc * max(1, len(sources)))()
    for i, (x, off, sc, n) in enumerate(sources):
        arr[i] = _FsGatherSrc(_ptr(x), _ptr(off), _ptr(sc), n)
    _check(_lib.fs_gather_programs(n_features, len(sources), arr, _ptr(keep), n_keep,
                                   _ptr(out_features), out_row_capacity, _ptr(out_prog_off),
                                   _ptr(out_score), _ptr(status), _stream_ptr(stream)))


def unpack_colblock64(x: torch.Tensor, n_rows: int, n_features: int) -> np.ndarray:
    """Host copy of an FS_COLBLOCK64 buffer as a row-major [n_rows, n_features] array (tests)."""
    tiles = (n_rows + 63) // 64
    a = x[: tiles * n_features * 64].cpu().numpy().reshape(tiles, n_features, 64)
    return np.ascontiguousarray(a.transpose(0, 2, 1).reshape(tiles * 64, n_features)[:n_rows])


# ---- mixtures of family models (familyseer_mixture.h) ---------------------------------------------
#
# The calls take no part in autograd: results have no graph, also of inputs that require a gradient.  Every operator has its
# gradient as a call of its own (fs_..._backward; fs_expert_combine without weights is fs_expert_gather's), to be made by the
# program, as FamilyMixture.gradients does, or from a torch.autograd.Function.  They run on the current GPU.

FS_F32, FS_BF16, FS_F16 = 0, 1, 2
FS_ID_I32, FS_ID_I64, FS_ID_U16 = 0, 1, 2
FS_SCORE_SOFTMAX, FS_SCORE_SIGMOID = 0, 1
FS_MAX_EXPERTS = 1024
FS_MAX_CHOICES = 16
FS_MAX_WIDTH = 1048576

_ELEMENT = {torch.float32: FS_F32, torch.bfloat16: FS_BF16, torch.float16: FS_F16}
_ID = {torch.int32: FS_ID_I32, torch.int64: FS_ID_I64, torch.int16: FS_ID_U16, torch.uint16: FS_ID_U16}


class _FsRouteParams(ctypes.Structure):
    _fields_ = [("n_experts", ctypes.c_int32), ("k", ctypes.c_int32), ("score", ctypes.c_int32),
                ("renormalise", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("top_groups", ctypes.c_int32),
                ("group_best", ctypes.c_int32), ("scale", ctypes.c_float)]


_i32, _i64, _vp, _sz, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
for _name, _result, _args in (
        ("fs_route", ctypes.c_int, [ctypes.POINTER(_FsRouteParams), _i64, _vp, _i32, _i64, _vp, _vp, _vp, _vp]),
        ("fs_route_backward", ctypes.c_int,
         [ctypes.POINTER(_FsRouteParams), _i64, _vp, _i32, _i64, _vp, _vp, _vp, _i64, _vp]),
        ("fs_expert_plan_workspace_bytes", _sz, [_i64, _i32, _i32]),
        ("fs_expert_plan", ctypes.c_int, [_i64, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
        ("fs_expert_gather", ctypes.c_int, [_i64, _i32, _i32, _i32, _vp, _i32, _i64, _vp, _vp, _vp, _i64, _vp]),
        ("fs_expert_combine", ctypes.c_int, [_i64, _i32, _i32, _vp, _i32, _i64, _vp, _vp, _vp, _i64, _vp]),
        ("fs_expert_combine_backward", ctypes.c_int,
         [_i64, _i32, _i32, _i32, _vp, _i32, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _i64, _vp, _vp]),
        ("fs_embed", ctypes.c_int, [_i32, _i32, _vp, _i32, _i64, _i64, _i32, _vp, _i32, _vp, _f32, _vp, _i32, _i64, _vp]),
        ("fs_embed_backward_workspace_bytes", _sz, [_i32, _i32, _i32, _i64, _i32]),
        ("fs_embed_backward", ctypes.c_int,
         [_i32, _i32, _vp, _i32, _i64, _i64, _i32, _vp, _i32, _vp, _f32, _i32, _vp, _i32, _i64, _vp, _sz, _vp])):
    getattr(_lib, _name).restype = _result
    getattr(_lib, _name).argtypes = _args


_INT32_MAX = 2147483647


def _int32(v: int, what: str) -> int:
    """A number for an int32_t: ctypes would pass on its low 32 bits."""
    if not -2147483648 <= v <= _INT32_MAX:
        raise FsError(FS_EINVAL, f"{what}: {v} does not fit 32 bits")
    return v


def _matrix(t: torch.Tensor, what: str, width: Optional[int] = None, rows: Optional[int] = None,
            dtype: Optional[torch.dtype] = None, on: Optional[int] = None):
    """(pointer, element type, row stride) of a matrix argument whose rows' elements are adjacent; `on`: the call's GPU."""
    if on is not None and t.get_device() != on:
        raise FsError(FS_EINVAL, f"{what} is not on the call's GPU")
    kind = _ELEMENT.get(t.dtype)
    if kind is None or t.dim() != 2:
        raise FsError(FS_EINVAL, f"{what} is not a matrix of fp32, bf16 or fp16")
    n, w = t.shape
    if (width is not None and w != width) or (rows is not None and n != rows):
        raise FsError(FS_EINVAL, f"{what} is {(n, w)}, not {(rows, width)}")
    if dtype is not None and t.dtype != dtype:
        raise FsError(FS_EINVAL, f"{what} is {t.dtype}, not {dtype}")
    if w > _INT32_MAX:
        raise FsError(FS_EINVAL, f"{what}: a row of {w} elements")
    step, between = t.stride()
    if between != 1 and w > 1:
        raise FsError(FS_EINVAL, f"{what}: the elements of a row are not adjacent")
    return t.data_ptr(), kind, (step if n > 1 else max(1, w))


def _array(t: Optional[torch.Tensor], what: str, shape, dtype: torch.dtype, on: Optional[int] = None) -> Optional[int]:
    """The pointer of an array argument; `shape`: so many elements, or a shape, which the array has or, laid flat, would have."""
    if t is None:
        return None
    if on is not None and t.get_device() != on:
        raise FsError(FS_EINVAL, f"{what} is not on the call's GPU")
    if type(shape) is tuple:
        fits = t.shape == shape or (t.dim() == 1 and t.numel() == math.prod(shape))
    else:
        fits = t.numel() == shape
    if t.dtype != dtype or not fits or not t.is_contiguous():
        raise FsError(FS_EINVAL, f"{what} is not a contiguous array of {shape} {dtype}")
    return t.data_ptr()


# The current stream's handle without the object around it (0.1 us instead of 2, of 11 that a call takes).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


_gpus = 0        # how many there are, once a call has asked


def _refuse_other_gpus(index: int, stream: Optional[torch.cuda.Stream]) -> None:
    """The library launches on the current GPU, and a default stream's handle names that one's, whichever GPU it was asked of."""
    global _gpus
    _gpus = _gpus or torch.cuda.device_count()
    if _gpus > 1:
        if torch.cuda.current_device() != index:
            raise FsError(FS_EINVAL, f"the tensors are on GPU {index}, which is not the current one")
        if stream is not None and stream.device_index != index:
            raise FsError(FS_EINVAL, f"the stream is GPU {stream.device_index}'s, the tensors are on GPU {index}")


class _Place:
    """Where a call runs, the current GPU: results and working memory are allocated for its stream."""

    __slots__ = ("device", "index", "stream", "ptr")

    def __init__(self, like: torch.Tensor, stream: Optional[torch.cuda.Stream]):
        if not like.is_cuda:
            raise FsError(FS_EINVAL, "the tensors are not on the GPU")
        self.device, self.stream = like.device, stream
        self.index = self.device.index
        if _gpus != 1:
            _refuse_other_gpus(self.index, stream)
        self.ptr = _raw_stream(self.index) if stream is None else stream.cuda_stream

    def empty(self, shape, dtype: torch.dtype) -> torch.Tensor:
        # empty_strided takes 1.3 us, empty 1.65.
        steps = (1,) if len(shape) == 1 else (max(1, shape[1]), 1)
        if self.stream is None:
            return torch.empty_strided(shape, steps, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty_strided(shape, steps, dtype=dtype, device=self.device)

    def matrix(self, out: Optional[torch.Tensor], what: str, rows: int, width: int, dtype: torch.dtype):
        """(the tensor, its pointer, its row stride): `out`, checked, or a new one."""
        if out is None:
            out = self.empty((rows, width), dtype)
            return out, out.data_ptr(), max(1, width)
        ptr, _, stride = _matrix(out, what, width, rows, dtype, self.index)
        return out, ptr, stride

    def array(self, out: Optional[torch.Tensor], what: str, shape, dtype: torch.dtype):
        if out is None:
            out = self.empty(shape, dtype)
            return out, out.data_ptr()
        return out, _array(out, what, shape, dtype, self.index)


def route_params(n_experts: int, k: int, score: int = FS_SCORE_SOFTMAX, renormalise: bool = True, n_groups: int = 1,
                 top_groups: int = 1, group_best: int = 1, scale: float = 1.0) -> _FsRouteParams:
    return _FsRouteParams(_int32(n_experts, "n_experts"), _int32(k, "k"), _int32(score, "score"), _int32(int(renormalise), "renormalise"),
                          _int32(n_groups, "n_groups"), _int32(top_groups, "top_groups"), _int32(group_best, "group_best"), scale)


def fs_route(params: _FsRouteParams, logits: torch.Tensor, bias: Optional[torch.Tensor] = None,
             expert: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None):
    """(expert, weight), int32 and fp32 of [tokens, k], of logits [tokens, n_experts]."""
    at = _Place(logits, stream)
    ptr, typ, stride = _matrix(logits, "logits", params.n_experts, on=at.index)
    n, k = logits.shape[0], params.k
    expert, e_ptr = at.array(expert, "expert", (n, max(k, 0)), torch.int32)
    weight, w_ptr = at.array(weight, "weight", (n, max(k, 0)), torch.float32)
    _check(_lib.fs_route(params, n, ptr, typ, stride, _array(bias, "bias", params.n_experts, torch.float32, at.index), e_ptr, w_ptr,
                         at.ptr))
    return expert, weight


def fs_route_backward(params: _FsRouteParams, logits: torch.Tensor, expert: torch.Tensor, d_weight: torch.Tensor,
                      d_logits: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    at = _Place(logits, stream)
    ptr, typ, stride = _matrix(logits, "logits", params.n_experts, on=at.index)
    n, k = logits.shape[0], params.k
    d_logits, d_ptr, d_stride = at.matrix(d_logits, "d_logits", n, params.n_experts, logits.dtype)
    _check(_lib.fs_route_backward(params, n, ptr, typ, stride, _array(expert, "expert", (n, k), torch.int32, at.index),
                                  _array(d_weight, "d_weight", (n, k), torch.float32, at.index), d_ptr, d_stride, at.ptr))
    return d_logits


class ExpertPlan:
    """Which slot every choice of `expert` [tokens, k] takes: first [n_experts+1], order [tokens*k], place [tokens, k]."""

    def __init__(self, first: torch.Tensor, order: torch.Tensor, place: torch.Tensor):
        self.first, self.order, self.place = first, order, place
        self.n_experts = first.shape[0] - 1
        self.n_tokens, self.k = place.shape

    def _bounds(self, at: _Place):
        """The pointer of first."""
        return _array(self.first, "first", self.n_experts + 1, torch.int32, at.index)

    def _lists(self, at: _Place):
        """The pointers of first and place."""
        return (_array(self.first, "first", self.n_experts + 1, torch.int32, at.index),
                _array(self.place, "place", self.n_tokens * self.k, torch.int32, at.index))


def fs_expert_plan(expert: torch.Tensor, n_experts: int, plan: Optional[ExpertPlan] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> ExpertPlan:
    """`plan`: an ExpertPlan of the same shape whose tensors are written again."""
    at = _Place(expert, stream)
    if expert.dim() != 2:
        raise FsError(FS_EINVAL, "expert is not [tokens, k]")
    n, k = expert.shape
    if k > _INT32_MAX or n_experts > _INT32_MAX:
        raise FsError(FS_EINVAL, f"{k} choices or {n_experts} experts do not fit 32 bits")
    if plan is not None and (plan.n_tokens, plan.k, plan.n_experts) != (n, k, n_experts):
        raise FsError(FS_EINVAL, f"plan is of {(plan.n_tokens, plan.k, plan.n_experts)} tokens, choices and experts, not {(n, k, n_experts)}")
    src = _array(expert, "expert", n * k, torch.int32, at.index)
    old = (None, None, None) if plan is None else (plan.first, plan.order, plan.place)
    first, f_ptr = at.array(old[0], "first", (max(n_experts, 0) + 1,), torch.int32)
    order, o_ptr = at.array(old[1], "order", (n * k,), torch.int32)
    place, p_ptr = at.array(old[2], "place", (n, k), torch.int32)
    need = _lib.fs_expert_plan_workspace_bytes(n, k, n_experts)
    work = at.empty((need,), torch.uint8) if need else None
    _check(_lib.fs_expert_plan(n, k, n_experts, src, f_ptr, o_ptr, p_ptr, _ptr(work), need, at.ptr))
    return ExpertPlan(first, order, place) if plan is None else plan


def fs_expert_gather(x: torch.Tensor, plan: ExpertPlan, out: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Rows x [tokens, width] in the experts' slots: [tokens*k, width]."""
    at = _Place(x, stream)
    ptr, typ, stride = _matrix(x, "x", rows=plan.n_tokens, on=at.index)
    width = x.shape[1]
    out, o_ptr, o_stride = at.matrix(out, "out", plan.n_tokens * plan.k, width, x.dtype)
    _check(_lib.fs_expert_gather(plan.n_tokens, plan.k, plan.n_experts, width, ptr, typ, stride, *plan._lists(at), o_ptr, o_stride, at.ptr))
    return out


def fs_expert_combine(y: torch.Tensor, plan: ExpertPlan, weight: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The slots' rows y [tokens*k, width], weighted, at their tokens: [tokens, width]."""
    at = _Place(y, stream)
    ptr, typ, stride = _matrix(y, "y", rows=plan.n_tokens * plan.k, on=at.index)
    width = y.shape[1]
    out, o_ptr, o_stride = at.matrix(out, "out", plan.n_tokens, width, y.dtype)
    _check(_lib.fs_expert_combine(plan.n_tokens, plan.k, width, ptr, typ, stride, plan._lists(at)[1],
                                  _array(weight, "weight", (plan.n_tokens, plan.k), torch.float32, at.index), o_ptr, o_stride, at.ptr))
    return out


def fs_expert_combine_backward(d_out: torch.Tensor, y: torch.Tensor, plan: ExpertPlan, weight: torch.Tensor,
                               d_y: Optional[torch.Tensor] = None, d_weight: Optional[torch.Tensor] = None,
                               stream: Optional[torch.cuda.Stream] = None):
    """(d_y, d_weight) of a weighted fs_expert_combine."""
    at = _Place(d_out, stream)
    n, k = plan.n_tokens, plan.k
    ptr, typ, stride = _matrix(d_out, "d_out", rows=n, on=at.index)
    width = d_out.shape[1]
    y_ptr, _, y_stride = _matrix(y, "y", width, n * k, d_out.dtype, at.index)
    d_y, o_ptr, o_stride = at.matrix(d_y, "d_y", n * k, width, d_out.dtype)
    d_weight, w_ptr = at.array(d_weight, "d_weight", (n, k), torch.float32)
    _check(_lib.fs_expert_combine_backward(n, k, plan.n_experts, width, ptr, typ, stride, y_ptr, y_stride, *plan._lists(at),
                                           _array(weight, "weight", (n, k), torch.float32, at.index), o_ptr, o_stride, w_ptr, at.ptr))
    return d_y, d_weight


def _id_array(ids: torch.Tensor, col_base: Optional[torch.Tensor], on: Optional[int] = None):
    """(rows, columns, pointer, type, base pointer): ids [rows] are single tokens, [rows, columns] bags."""
    if ids.dim() not in (1, 2) or ids.dtype not in _ID:
        raise FsError(FS_EINVAL, "ids is not [rows] or [rows, columns] of int32, int64 or 16-bit leaf ids")
    if not ids.is_contiguous():
        raise FsError(FS_EINVAL, "ids is not contiguous")
    if on is not None and ids.get_device() != on:
        raise FsError(FS_EINVAL, "ids is not on the call's GPU")
    rows, cols = ids.shape[0], (ids.shape[1] if ids.dim() == 2 else 1)
    if cols > _INT32_MAX:
        raise FsError(FS_EINVAL, f"ids has {cols} columns")
    return rows, cols, ids.data_ptr(), _ID[ids.dtype], _array(col_base, "col_base", cols, torch.int32, on)


def fs_embed(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, col_base: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """[rows, width]: the scaled rows of `table` that ids [rows] name, or the scaled sums of those that ids [rows, columns]
    name.  The result is of the table's type unless `out` (of that type or fp32) is given."""
    at = _Place(table, stream)
    t_ptr, typ, t_stride = _matrix(table, "table", on=at.index)
    rows, cols, i_ptr, i_typ, base = _id_array(ids, col_base, at.index)
    vocab, width = table.shape
    if vocab > _INT32_MAX:
        raise FsError(FS_EINVAL, f"table has {vocab} rows")
    out, o_ptr, o_stride = at.matrix(out, "out", rows, width, table.dtype if out is None else out.dtype)
    o_typ = _ELEMENT[out.dtype]
    _check(_lib.fs_embed(vocab, width, t_ptr, typ, t_stride, rows, cols, i_ptr, i_typ, base, scale, o_ptr, o_typ, o_stride, at.ptr))
    return out


def fs_embed_backward(d_out: torch.Tensor, ids: torch.Tensor, n_vocab: int, scale: float = 1.0,
                      col_base: Optional[torch.Tensor] = None, d_table: Optional[torch.Tensor] = None, accumulate: bool = False,
                      stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The table's gradient [n_vocab, width]: fp32 unless `d_table` (of that type or d_out's) is given; `accumulate` adds to
    what `d_table` holds."""
    at = _Place(d_out, stream)
    if n_vocab > _INT32_MAX:
        raise FsError(FS_EINVAL, f"n_vocab {n_vocab} does not fit 32 bits")
    rows, cols, i_ptr, i_typ, base = _id_array(ids, col_base, at.index)
    ptr, typ, stride = _matrix(d_out, "d_out", rows=rows, on=at.index)
    width = d_out.shape[1]
    if d_table is None and accumulate:
        raise FsError(FS_EINVAL, "accumulate needs a d_table to add to")
    kind = torch.float32 if d_table is None else d_table.dtype
    d_table, t_ptr, t_stride = at.matrix(d_table, "d_table", max(n_vocab, 0), width, kind)
    t_typ = _ELEMENT[d_table.dtype]
    need = _lib.fs_embed_backward_workspace_bytes(n_vocab, width, typ, rows, cols)
    work = at.empty((need,), torch.uint8) if need else None
    _check(_lib.fs_embed_backward(n_vocab, width, ptr, typ, stride, rows, cols, i_ptr, i_typ, base, scale, int(accumulate), t_ptr,
                                  t_typ, t_stride, _ptr(work), need, at.ptr))
    return d_table


# ---- networks as experts (familyseer_experts.h) ----------------------------------------------------
#
# As above: no autograd.  fs_expert_matmul with the other `turned` is the rows' gradient, fs_expert_matmul_backward the weights'.

FS_MAX_I8_WIDTH = 131072
FS_MAX_CLASSES = 1048576
FS_MAX_LISTED = 1024


class _FsDistillParams(ctypes.Structure):
    _fields_ = [("n_classes", ctypes.c_int32), ("k", ctypes.c_int32), ("temperature", ctypes.c_float), ("scale", ctypes.c_float)]


for _name, _result, _args in (
        ("fs_expert_matmul", ctypes.c_int, [_i64, _i32, _i32, _i32, _vp, _i32, _i64, _vp, _vp, _i64, _i64, _i32, _vp, _i32, _i64, _vp]),
        ("fs_expert_matmul_backward_workspace_bytes", _sz, [_i64, _i32, _i32, _i32, _i32]),
        ("fs_expert_matmul_backward", ctypes.c_int,
         [_i64, _i32, _i32, _i32, _vp, _i32, _i64, _vp, _i64, _vp, _i32, _vp, _i32, _i64, _i64, _vp, _sz, _vp]),
        ("fs_quantize_rows", ctypes.c_int, [_i64, _i32, _vp, _i32, _i64, _vp, _i64, _vp, _vp]),
        ("fs_expert_gather_i8", ctypes.c_int, [_i64, _i32, _i32, _i32, _vp, _i32, _i64, _vp, _vp, _vp, _i64, _vp, _vp]),
        ("fs_expert_matmul_i8", ctypes.c_int, [_i64, _i32, _i32, _i32, _vp, _i64, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _i32, _i64, _vp]),
        ("fs_distill_workspace_bytes", _sz, [ctypes.POINTER(_FsDistillParams), _i64, _i32]),
        ("fs_distill", ctypes.c_int,
         [ctypes.POINTER(_FsDistillParams), _i64, _vp, _i32, _i64, _vp, _i32, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
        ("fs_distill_backward", ctypes.c_int,
         [ctypes.POINTER(_FsDistillParams), _i64, _vp, _i32, _i64, _vp, _i32, _vp, _i32, _vp, _vp, _vp, _vp, _i64, _vp, _sz, _vp])):
    getattr(_lib, _name).restype = _result
    getattr(_lib, _name).argtypes = _args


def _bytes_matrix(t: torch.Tensor, what: str, width: Optional[int] = None, rows: Optional[int] = None, on: Optional[int] = None):
    """(pointer, row stride) of a matrix of 8-bit integers."""
    if on is not None and t.get_device() != on:
        raise FsError(FS_EINVAL, f"{what} is not on the call's GPU")
    if t.dtype != torch.int8 or t.dim() != 2:
        raise FsError(FS_EINVAL, f"{what} is not a matrix of int8")
    n, w = t.shape
    if (width is not None and w != width) or (rows is not None and n != rows):
        raise FsError(FS_EINVAL, f"{what} is {(n, w)}, not {(rows, width)}")
    if w > _INT32_MAX:
        raise FsError(FS_EINVAL, f"{what}: a row of {w} elements")
    step, between = t.stride()
    if between != 1 and w > 1:
        raise FsError(FS_EINVAL, f"{what}: the elements of a row are not adjacent")
    return t.data_ptr(), (step if n > 1 else max(1, w))


def _weights(w: torch.Tensor, what: str, n_experts: int, dtype, on: Optional[int] = None):
    """(pointer, rows, columns, row stride, step from expert to expert) of weights [n_experts, rows, columns]."""
    if on is not None and w.get_device() != on:
        raise FsError(FS_EINVAL, f"{what} is not on the call's GPU")
    if w.dim() != 3 or w.dtype not in (dtype if type(dtype) is tuple else (dtype,)):
        raise FsError(FS_EINVAL, f"{what} is {w.dim()}-dimensional of {w.dtype}, not [experts, rows, columns] of {dtype}")
    e, n, c = w.shape
    if e != n_experts:
        raise FsError(FS_EINVAL, f"{what} is of {e} experts, not {n_experts}")
    if n > _INT32_MAX or c > _INT32_MAX:
        raise FsError(FS_EINVAL, f"{what}: matrices of {n} x {c}")
    between, step, adjacent = w.stride()
    if adjacent != 1 and c > 1:
        raise FsError(FS_EINVAL, f"{what}: the elements of a row are not adjacent")
    step = step if n > 1 else max(1, c)
    return w.data_ptr(), n, c, step, (between if e > 1 else n * step)


def _slots_of(plan: ExpertPlan) -> int:
    return plan.n_tokens * plan.k


def fs_expert_matmul(x: torch.Tensor, plan: ExpertPlan, w: torch.Tensor, turned: bool = False, out: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Rows x [slots, in] of `plan`'s slots times their expert's weights w [experts, out, in], or `turned` [experts, in, out]: [slots, out],
    of x's type unless `out` (of that type or fp32) is given.  With w turned, of a result's gradient, it is the rows' gradient."""
    at = _Place(x, stream)
    slots = _slots_of(plan)
    ptr, typ, stride = _matrix(x, "x", rows=slots, on=at.index)
    w_ptr, rows, cols, w_stride, w_step = _weights(w, "w", plan.n_experts, x.dtype, at.index)
    width, out_width = (rows, cols) if turned else (cols, rows)
    if x.shape[1] != width:
        raise FsError(FS_EINVAL, f"x has {x.shape[1]} columns, w takes {width}")
    out, o_ptr, o_stride = at.matrix(out, "out", slots, out_width, x.dtype if out is None else out.dtype)
    _check(_lib.fs_expert_matmul(slots, plan.n_experts, width, out_width, ptr, typ, stride, plan._bounds(at), w_ptr, w_stride, w_step,
                                 int(turned), o_ptr, _ELEMENT[out.dtype], o_stride, at.ptr))
    return out


def fs_expert_matmul_backward(d_y: torch.Tensor, x: torch.Tensor, plan: ExpertPlan, d_w: Optional[torch.Tensor] = None,
                              accumulate: bool = False, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The gradient [experts, out, in] of weights through which x [slots, in] went to results whose gradient is d_y [slots, out] (of turned
    weights: x and d_y change places); fp32 unless `d_w` (of that type or x's) is given; `accumulate` adds to what `d_w` holds."""
    at = _Place(d_y, stream)
    slots = _slots_of(plan)
    g_ptr, typ, g_stride = _matrix(d_y, "d_y", rows=slots, on=at.index)
    x_ptr, _, x_stride = _matrix(x, "x", rows=slots, dtype=d_y.dtype, on=at.index)
    out_width, width = d_y.shape[1], x.shape[1]
    if d_w is None:
        if accumulate:
            raise FsError(FS_EINVAL, "accumulate needs a d_w to add to")
        d_w = at.empty((plan.n_experts * out_width, width), torch.float32).view(plan.n_experts, out_width, width)
    d_ptr, rows, cols, d_stride, d_step = _weights(d_w, "d_w", plan.n_experts, (torch.float32, d_y.dtype), at.index)
    if (rows, cols) != (out_width, width):
        raise FsError(FS_EINVAL, f"d_w is of {(rows, cols)} an expert, not {(out_width, width)}")
    need = _lib.fs_expert_matmul_backward_workspace_bytes(slots, plan.n_experts, width, out_width, typ)
    work = at.empty((need,), torch.uint8) if need else None
    _check(_lib.fs_expert_matmul_backward(slots, plan.n_experts, width, out_width, g_ptr, typ, g_stride, x_ptr, x_stride, plan._bounds(at),
                                          int(accumulate), d_ptr, _ELEMENT[d_w.dtype], d_stride, d_step, _ptr(work), need, at.ptr))
    return d_w


def fs_quantize_rows(x: torch.Tensor, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None):
    """(q, scale): rows x [rows, width] as 8-bit integers, and what each row's are multiplied by, fp32 [rows]."""
    at = _Place(x, stream)
    ptr, typ, stride = _matrix(x, "x", on=at.index)
    n, width = x.shape
    q = at.empty((n, width), torch.int8) if q is None else q
    q_ptr, q_stride = _bytes_matrix(q, "q", width, n, at.index)
    scale, s_ptr = at.array(scale, "scale", (n,), torch.float32)
    _check(_lib.fs_quantize_rows(n, width, ptr, typ, stride, q_ptr, q_stride, s_ptr, at.ptr))
    return q, scale


def fs_expert_gather_i8(x: torch.Tensor, plan: ExpertPlan, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None):
    """(q [tokens*k, width], scale [tokens*k]): rows x [tokens, width] as fs_quantize_rows makes them, in the experts' slots."""
    at = _Place(x, stream)
    ptr, typ, stride = _matrix(x, "x", rows=plan.n_tokens, on=at.index)
    slots, width = _slots_of(plan), x.shape[1]
    q = at.empty((slots, width), torch.int8) if q is None else q
    q_ptr, q_stride = _bytes_matrix(q, "q", width, slots, at.index)
    scale, s_ptr = at.array(scale, "scale", (slots,), torch.float32)
    _check(_lib.fs_expert_gather_i8(plan.n_tokens, plan.k, plan.n_experts, width, ptr, typ, stride, *plan._lists(at), q_ptr, q_stride, s_ptr, at.ptr))
    return q, scale


def fs_expert_matmul_i8(q: torch.Tensor, scale: torch.Tensor, plan: ExpertPlan, w: torch.Tensor, w_scale: torch.Tensor,
                        dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Rows q [slots, in] of int8 times their expert's weights w [experts, out, in] of int8, times both scales, scale [slots] and
    w_scale [experts, out]: [slots, out] of `dtype`, or into `out`."""
    at = _Place(q, stream)
    slots = _slots_of(plan)
    ptr, stride = _bytes_matrix(q, "q", rows=slots, on=at.index)
    w_ptr, out_width, width, w_stride, w_step = _weights(w, "w", plan.n_experts, torch.int8, at.index)
    if q.shape[1] != width:
        raise FsError(FS_EINVAL, f"q has {q.shape[1]} columns, w takes {width}")
    if out is None and dtype not in _ELEMENT:
        raise FsError(FS_EINVAL, f"results of {dtype}")
    out, o_ptr, o_stride = at.matrix(out, "out", slots, out_width, dtype if out is None else out.dtype)
    _check(_lib.fs_expert_matmul_i8(slots, plan.n_experts, width, out_width, ptr, stride, _array(scale, "scale", slots, torch.float32, at.index),
                                    plan._bounds(at), w_ptr, w_stride, w_step,
                                    _array(w_scale, "w_scale", (plan.n_experts, out_width), torch.float32, at.index), o_ptr, _ELEMENT[out.dtype],
                                    o_stride, at.ptr))
    return out


def distill_params(n_classes: int, k: int, temperature: float = 1.0, scale: float = 1.0) -> _FsDistillParams:
    return _FsDistillParams(_int32(n_classes, "n_classes"), _int32(k, "k"), temperature, scale)


def _distill(params: _FsDistillParams, at: _Place, logits, ids, teacher, total):
    """The arguments that both distillation calls begin with, and working memory."""
    ptr, typ, stride = _matrix(logits, "logits", params.n_classes, on=at.index)
    n = logits.shape[0]
    if ids.dtype not in (torch.int32, torch.int64):
        raise FsError(FS_EINVAL, f"ids is {ids.dtype}, neither int32 nor int64")
    if teacher.dtype not in _ELEMENT:
        raise FsError(FS_EINVAL, f"teacher is {teacher.dtype}, not fp32, bf16 or fp16")
    need = _lib.fs_distill_workspace_bytes(params, n, typ)
    work = at.empty((need,), torch.uint8) if need else None
    return n, work, need, (params, n, ptr, typ, stride, _array(ids, "ids", (n, params.k), ids.dtype, at.index), _ID[ids.dtype],
                           _array(teacher, "teacher", (n, params.k), teacher.dtype, at.index), _ELEMENT[teacher.dtype],
                           _array(total, "total", (n,), torch.float32, at.index))


def fs_distill(params: _FsDistillParams, logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, total: Optional[torch.Tensor] = None,
               loss: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Losses [tokens] of student's logits [tokens, n_classes] against the classes `ids` [tokens, k] and logits `teacher` [tokens, k] that a teacher
    gave; with `total` [tokens], the log of the sum of exp(logit / temperature) over all of its classes, the rest counts as a class."""
    at = _Place(logits, stream)
    n, work, need, args = _distill(params, at, logits, ids, teacher, total)
    loss, l_ptr = at.array(loss, "loss", (n,), torch.float32)
    _check(_lib.fs_distill(*args, l_ptr, _ptr(work), need, at.ptr))
    return loss


def fs_distill_backward(params: _FsDistillParams, logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, d_loss: torch.Tensor,
                        total: Optional[torch.Tensor] = None, loss: Optional[torch.Tensor] = None, d_logits: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The logits' gradient of losses whose gradient is d_loss [tokens]; `loss` [tokens], if given, receives the losses too."""
    at = _Place(logits, stream)
    n, work, need, args = _distill(params, at, logits, ids, teacher, total)
    d_logits, d_ptr, d_stride = at.matrix(d_logits, "d_logits", n, params.n_classes, logits.dtype)
    if d_logits.dtype != logits.dtype:
        raise FsError(FS_EINVAL, f"d_logits is {d_logits.dtype}, not {logits.dtype}")
    _check(_lib.fs_distill_backward(*args, _array(d_loss, "d_loss", (n,), torch.float32, at.index), _array(loss, "loss", (n,), torch.float32, at.index),
                                    d_ptr, d_stride, _ptr(work), need, at.ptr))
    return d_logits
