"""Python binding of libhwsel.so (ctypes; the calls on 8-bit matrices, the draws,
their log probabilities, dropout and joins through _binding.so, whose checks in
C++ take 3 us where Python's took 11).

The functions carry the C ABI's names and only marshal arguments: torch
tensors in device memory become raw pointers, the current torch stream
becomes the hipStream_t.  Every step of the scored path runs in the HIP
library; there is no fallback of any kind -- if the library is missing the
call raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhwsel.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "hwsel.h")

HWSEL_OK, HWSEL_EINVAL, HWSEL_EUNSUPPORTED, HWSEL_EHIP = 0, 1, 2, 3


class HwselError(RuntimeError):
    def __init__(self, fn: str, status: int, detail: str):
        super().__init__(f"{fn} -> {status} ({detail})")
        self.status = status


class hwsel_hw_t(C.Structure):
    _fields_ = [(n, C.c_int64) for n in (
        "n_sm", "smem_per_sm", "smem_per_block_max", "smem_reserved", "regs_per_sm",
        "max_regs_per_thread", "max_blocks_per_sm", "max_threads_per_sm", "arch_id",
        "llc_bytes", "hbm_bw_gbps")] + [("peak_gflops", C.c_int64 * 3)]


CAND_FIELDS = ("tile_m", "tile_n", "tile_k", "inst_n", "stages", "cluster_m", "cluster_n", "swizzle",
               "inst_m_div16", "inst_k", "kernel_sched", "epi_sched", "tile_sched")


class hwsel_cands_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in CAND_FIELDS]


class hwsel_forest_t(C.Structure):
    _fields_ = [("n_trees", C.c_int32), ("depth", C.c_int32), ("n_features", C.c_int32),
                ("flags", C.c_uint32), ("base_score", C.c_float), ("node_feature", C.c_void_p),
                ("node_threshold", C.c_void_p), ("leaf_value", C.c_void_p)]


class hwsel_mlp_t(C.Structure):
    _fields_ = [("n_in", C.c_int32), ("h1", C.c_int32), ("h2", C.c_int32), ("h3", C.c_int32),
                ("mean", C.c_void_p), ("inv_std", C.c_void_p), ("W1", C.c_void_p), ("W2", C.c_void_p),
                ("W3", C.c_void_p), ("W4", C.c_void_p), ("b1", C.c_void_p), ("b2", C.c_void_p),
                ("b3", C.c_void_p), ("b4", C.c_void_p)]


class hwsel_cands_out_t(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in CAND_FIELDS]


class hwsel_linear_t(C.Structure):
    _fields_ = [("n_features", C.c_int32), ("bias", C.c_float), ("mean", C.c_void_p), ("inv_std", C.c_void_p),
                ("w", C.c_void_p), ("w_onehot", C.c_void_p)]


class hwsel_fp8_t(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("q", C.c_void_p), ("ld", C.c_int64),
                ("scale", C.c_void_p), ("ld_scale", C.c_int64), ("format", C.c_int32), ("block_rows", C.c_int32)]


class hwsel_sampling_t(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_k", C.c_int32), ("top_p", C.c_float), ("min_p", C.c_float),
                ("temperature_of", C.c_void_p), ("top_k_of", C.c_void_p), ("top_p_of", C.c_void_p),
                ("min_p_of", C.c_void_p)]


class hwsel_matrix_t(C.Structure):
    _fields_ = [("data", C.c_void_p), ("ld", C.c_int64), ("dtype", C.c_int32)]


class hwsel_dropout_t(C.Structure):
    _fields_ = [("seed", C.c_uint64), ("offset", C.c_uint64), ("state", C.c_void_p), ("p", C.c_float)]


class hwsel_join_t(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("w_branch", C.c_void_p), ("w_pre", C.c_void_p),
                ("eps", C.c_float), ("stream_scale", C.c_float), ("branch_scale", C.c_float), ("post_norm", C.c_int32),
                ("gate_sigmoid", C.c_int32), ("gate_cols", C.c_int64), ("dropout", hwsel_dropout_t)]


_lib = None


def lib() -> C.CDLL:
    """Load the HIP library; raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python paper_2609_35587_amd/build.py` (there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        L.hwsel_status_string.restype = C.c_char_p
        L.hwsel_last_error.restype = C.c_char_p
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.hwsel_features.argtypes = [hwsel_hw_t, vp, i32, vp, C.POINTER(hwsel_cands_t), i64, i32, vp, i64, vp]
        L.hwsel_forest_score.argtypes = [C.POINTER(hwsel_forest_t), vp, vp, i64, i64, vp, vp, C.c_size_t, vp]
        L.hwsel_forest_pack_bytes.argtypes = [C.POINTER(hwsel_forest_t), C.POINTER(C.c_size_t)]
        L.hwsel_forest_pack.argtypes = [C.POINTER(hwsel_forest_t), vp, C.c_size_t, vp]
        L.hwsel_forest_pack_host.argtypes = [C.POINTER(hwsel_forest_t), vp, C.c_size_t]
        L.hwsel_forest_workspace_bytes.argtypes = [C.POINTER(hwsel_forest_t), i64, C.POINTER(C.c_size_t)]
        L.hwsel_forest_score_checked.argtypes = [C.POINTER(hwsel_forest_t), vp, vp, i64, i64, vp, vp, C.c_size_t,
                                                 vp, vp, i64, i64, vp]
        L.hwsel_forest_leaves.argtypes = [C.POINTER(hwsel_forest_t), vp, i64, i64, vp, i64, vp, vp]
        L.hwsel_mlp_score.argtypes = [C.POINTER(hwsel_mlp_t), vp, vp, i64, i64, vp, vp]
        L.hwsel_mlp_pack_bytes.argtypes = [C.POINTER(hwsel_mlp_t), C.POINTER(C.c_size_t)]
        L.hwsel_mlp_pack.argtypes = [C.POINTER(hwsel_mlp_t), vp, C.c_size_t, vp]
        L.hwsel_topk_per_problem.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        L.hwsel_regret.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp, vp]
        L.hwsel_linear_score.argtypes = [C.POINTER(hwsel_linear_t), vp, i64, i64, vp, vp]
        sz = C.c_size_t
        L.hwsel_select_forest_workspace_bytes.argtypes = [C.POINTER(hwsel_forest_t), i64, C.POINTER(sz)]
        L.hwsel_select_forest.argtypes = [hwsel_hw_t, vp, i32, vp, C.POINTER(hwsel_cands_t), i64, i32,
                                          C.POINTER(hwsel_forest_t), vp, i32, vp, vp, vp, vp, sz, vp]
        L.hwsel_evaluate_workspace_bytes.argtypes = [i32, C.POINTER(sz)]
        L.hwsel_evaluate.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.hwsel_evaluate_noalloc.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp, vp, vp]
        L.hwsel_static_config_workspace_bytes.argtypes = [i32, i32, C.POINTER(sz)]
        L.hwsel_static_config.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp, sz, vp]
        L.hwsel_catalogue_mask.argtypes = [hwsel_hw_t, vp, i32, C.c_uint32, vp, vp, vp]
        L.hwsel_catalogue_compact.argtypes = [vp, vp, i32, vp, vp, i64, vp]
        L.hwsel_catalogue_candidates.argtypes = [vp, i32, vp, vp, i64, C.POINTER(hwsel_cands_out_t), vp]
        L.hwsel_sample_score.argtypes = [hwsel_hw_t, vp, i32, vp, C.POINTER(hwsel_cands_t), i64, vp, vp]
        fp = C.POINTER(hwsel_fp8_t)
        L.hwsel_fp8_quantise.argtypes = [vp, i32, i64, i32, vp, vp, fp, vp]
        L.hwsel_fp8_dequantise.argtypes = [fp, vp, i32, i64, vp]
        L.hwsel_fp8_transpose.argtypes = [fp, fp, vp]
        L.hwsel_fp8_matmul_workspace_bytes.argtypes = [fp, fp, C.POINTER(sz)]
        L.hwsel_fp8_matmul.argtypes = [fp, fp, vp, i32, vp, i32, i64, vp, sz, vp]
        L.hwsel_fp8_layer.argtypes = [fp, fp, vp, i32, fp, vp, sz, vp]
        L.hwsel_sample_workspace_bytes.argtypes = [i64, i32, i32, C.POINTER(sz)]
        L.hwsel_sample_per_problem.argtypes = [vp, i64, vp, i32, C.POINTER(hwsel_sampling_t), vp, i32, vp, vp, vp, vp,
                                               sz, vp]
        f32, mat, join = C.c_float, C.POINTER(hwsel_matrix_t), C.POINTER(hwsel_join_t)
        L.hwsel_logprob_workspace_bytes.argtypes = [i64, i32, i32, C.POINTER(sz)]
        L.hwsel_logprob_per_problem.argtypes = [vp, i64, vp, i32, f32, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.hwsel_logprob_gradient.argtypes = [vp, i64, vp, i32, f32, vp, vp, vp, i32, vp, vp, vp, vp, vp]
        L.hwsel_dropout.argtypes = [C.POINTER(hwsel_dropout_t), i64, i64, mat, mat, mat, vp]
        L.hwsel_block_join.argtypes = [join, mat, mat, mat, mat, mat, vp]
        L.hwsel_block_join_gradient_workspace_bytes.argtypes = [join, C.POINTER(sz)]
        L.hwsel_block_join_gradient.argtypes = [join, mat, mat, mat, mat, mat, mat, mat, mat, vp, vp, vp, sz, vp]
        _lib = L
    return _lib


_binding = None
# as csrc/binding.cpp lists them
_BOUND = ("hwsel_fp8_quantise", "hwsel_fp8_dequantise", "hwsel_fp8_transpose", "hwsel_fp8_matmul_workspace_bytes",
          "hwsel_fp8_matmul", "hwsel_fp8_layer", "hwsel_sample_workspace_bytes", "hwsel_sample_per_problem",
          "hwsel_logprob_workspace_bytes", "hwsel_logprob_per_problem", "hwsel_logprob_gradient", "hwsel_dropout",
          "hwsel_block_join", "hwsel_block_join_gradient_workspace_bytes", "hwsel_block_join_gradient", "hwsel_last_error")


def _calls():
    """_binding.so, connected to the library; raises if it has not been built."""
    global _binding
    if _binding is None:
        L = lib()
        try:
            from . import _binding as module
        except ImportError as e:
            raise RuntimeError("paper_2609_35587_amd/_binding.so does not load: build it with "
                               f"`python paper_2609_35587_amd/build.py` ({e})") from e
        module.connect(HwselError, *[C.cast(getattr(L, n), C.c_void_p).value for n in _BOUND])
        _binding = module
    return _binding


def _check(fn: str, status: int) -> None:
    if status != HWSEL_OK:
        raise HwselError(fn, status, lib().hwsel_last_error().decode())


def _ptr(t) -> int | None:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:                                      # (0.3 us; 2.7 through a Stream object)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _empty(shape, dtype: torch.dtype, device, stream) -> torch.Tensor:
    """A result or workspace of a call on ``stream``.  torch hands freed memory
    to the next allocation of the same stream without waiting, so on a stream
    other than the current one it is that stream's, noted on the current one."""
    current = None if stream is None else torch.cuda.current_stream(device)
    if current is None or _stream(stream) == current.cuda_stream:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(torch.cuda.ExternalStream(_stream(stream), device=device)):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(current)
    return t


def _dev(t: torch.Tensor, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    return t


def _arg(t, name: str, dtypes, numel: int = 0, like: torch.Tensor | None = None) -> torch.Tensor:
    """A caller-supplied buffer the library reads or writes: a contiguous
    device tensor (on the same device as ``like``) of one of ``dtypes`` with
    at least ``numel`` elements.  Raises ValueError before anything runs."""
    t = _dev(t, name)
    if like is not None and t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, the other operands on {like.device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} has dtype {t.dtype}, expected one of {tuple(dtypes)}")
    if t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, {numel} needed")
    return t


def _matrix(X, name: str, cols: int, like: torch.Tensor | None = None) -> torch.Tensor:
    """A row-major fp32 matrix [R][ld] with ld >= cols (a column slice of a
    wider buffer is fine): rows are read or written ld apart."""
    if not isinstance(X, torch.Tensor) or not X.is_cuda or X.dim() != 2:
        raise ValueError(f"{name} must be a 2-D device tensor")
    if like is not None and X.device != like.device:
        raise ValueError(f"{name} is on {X.device}, the other operands on {like.device}")
    if X.dtype != torch.float32 or X.stride(1) != 1 or X.shape[1] < cols or X.stride(0) < cols:
        raise ValueError(f"{name} must be fp32 [R][>= {cols}] with unit column stride")
    return X


F32, I32, I64 = (torch.float32,), (torch.int32,), (torch.int64,)
U8 = (torch.uint8,)
U16 = (torch.int16, torch.uint16) if hasattr(torch, "uint16") else (torch.int16,)


# ----------------------------------------------------------------------------
# Marshalling helpers (numpy -> device tensors); no arithmetic of the path.
# ----------------------------------------------------------------------------
def to_device(a: np.ndarray, device="cuda") -> torch.Tensor:
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        a = a.view(np.int16)
    elif a.dtype.fields is not None:
        a = a.view(np.uint8).reshape(len(a), -1)
    return torch.from_numpy(a).to(device)


def hw_struct(hw: dict) -> hwsel_hw_t:
    s = hwsel_hw_t()
    for n, _ in hwsel_hw_t._fields_[:-1]:
        setattr(s, n, int(hw[n]))
    for i, v in enumerate(hw["peak_gflops"]):
        s.peak_gflops[i] = int(v)
    return s


# ----------------------------------------------------------------------------
# Entry points
# ----------------------------------------------------------------------------
def hwsel_features(hw: dict, problems: torch.Tensor, seg_offsets: torch.Tensor, cands: dict,
                   n_features: int, X: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """problems: uint8 [P, 16] device records; seg_offsets int64 [P+1];
    cands: name -> device tensor of length R.  Returns X fp32 [R, ld]."""
    P = problems.shape[0]
    R = cands["tile_m"].shape[0]
    if X is None:
        X = _empty((R, n_features), torch.float32, problems.device, stream)
    _matrix(X, "X", n_features, like=problems)
    if X.shape[0] < R:
        raise ValueError(f"X has {X.shape[0]} rows, {R} candidates")
    cs = _cands_struct(cands, R, problems)
    _check("hwsel_features", lib().hwsel_features(
        hw_struct(hw), _ptr(_dev(problems, "problems")), P, _ptr(_dev(seg_offsets, "seg_offsets")),
        C.byref(cs), R, n_features, _ptr(X), X.stride(0), _stream(stream)))
    return X


def _cands_struct(cands: dict, R: int, like: torch.Tensor) -> hwsel_cands_t:
    wide = ("tile_m", "tile_n", "tile_k", "inst_n")
    for n in CAND_FIELDS:
        _arg(cands[n], n, U16 if n in wide else U8, R, like)
    return hwsel_cands_t(*[_ptr(cands[n]) for n in CAND_FIELDS])


def hwsel_sample_score(hw: dict, problems: torch.Tensor, seg_offsets: torch.Tensor, cands: dict,
                       scores: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The analytic sampling score per row (no feature matrix)."""
    P = problems.shape[0]
    R = cands["tile_m"].shape[0]
    if scores is None:
        scores = _empty(R, torch.float32, problems.device, stream)
    _arg(scores, "scores", F32, R, problems)
    cs = _cands_struct(cands, R, problems)
    _check("hwsel_sample_score", lib().hwsel_sample_score(
        hw_struct(hw), _ptr(_dev(problems, "problems")), P, _ptr(_dev(seg_offsets, "seg_offsets")),
        C.byref(cs), R, _ptr(scores), _stream(stream)))
    return scores


def linear_struct(m: dict) -> hwsel_linear_t:
    return hwsel_linear_t(int(m["n_features"]), float(m["bias"]), _ptr(m["mean"]), _ptr(m["inv_std"]),
                          _ptr(m["w"]), _ptr(m["w_onehot"]))


def hwsel_linear_score(lin: dict, X: torch.Tensor, scores: torch.Tensor | None = None,
                       stream=None) -> torch.Tensor:
    R = X.shape[0]
    F = int(lin["n_features"])
    _matrix(X, "X", F)
    if scores is None:
        scores = _empty(R, torch.float32, X.device, stream)
    _arg(scores, "scores", F32, R, X)
    for n in ("mean", "inv_std", "w"):
        _arg(lin[n], n, F32, F, X)
    _arg(lin["w_onehot"], "w_onehot", F32, 12, X)
    s = linear_struct(lin)
    _check("hwsel_linear_score", lib().hwsel_linear_score(C.byref(s), _ptr(X), R, X.stride(0), _ptr(scores),
                                                          _stream(stream)))
    return scores


def forest_struct(f: dict) -> hwsel_forest_t:
    return hwsel_forest_t(int(f["n_trees"]), int(f["depth"]), int(f["n_features"]), int(f["flags"]),
                          float(f["base_score"]), _ptr(f["node_feature"]), _ptr(f["node_threshold"]),
                          _ptr(f["leaf_value"]))


def hwsel_forest_pack_bytes(forest: dict) -> int:
    n = C.c_size_t(0)
    s = forest_struct(forest)
    _check("hwsel_forest_pack_bytes", lib().hwsel_forest_pack_bytes(C.byref(s), C.byref(n)))
    return int(n.value)


def hwsel_forest_pack(forest: dict, packed: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Pack a device-resident forest once; returns the packed image (uint8)."""
    nbytes = hwsel_forest_pack_bytes(forest)
    _forest_arrays(forest)
    if packed is None:
        packed = _empty(nbytes, torch.uint8, forest["node_feature"].device, stream)
    _arg(packed, "packed", U8, nbytes, forest["node_feature"])
    s = forest_struct(forest)
    _check("hwsel_forest_pack", lib().hwsel_forest_pack(C.byref(s), _ptr(packed), packed.numel(),
                                                        _stream(stream)))
    return packed


def _forest_arrays(forest: dict) -> None:
    T, d = int(forest["n_trees"]), int(forest["depth"])
    if not 1 <= d <= 12 or T < 1:
        return                                    # the library rejects the shape itself
    n_int = ((1 << d) - 1) * T
    ref = _arg(forest["node_feature"], "node_feature", U8, n_int)
    _arg(forest["node_threshold"], "node_threshold", F32, n_int, ref)
    _arg(forest["leaf_value"], "leaf_value", F32, (1 << d) * T, ref)


def _packed_image(forest: dict, packed: torch.Tensor, like: torch.Tensor) -> None:
    _arg(packed, "packed", U8, hwsel_forest_pack_bytes(forest), like)


def hwsel_forest_pack_host(forest: dict) -> np.ndarray:
    """The packed image of a forest given as host numpy arrays, built on the
    host (no GPU needed); returns it as uint8 numpy array."""
    arrays = {n: np.ascontiguousarray(forest[n], dt) for n, dt in
              (("node_feature", np.uint8), ("node_threshold", np.float32), ("leaf_value", np.float32))}
    f = dict(forest, **{n: a.ctypes.data for n, a in arrays.items()})
    n = C.c_size_t(0)
    s = forest_struct(f)
    _check("hwsel_forest_pack_bytes", lib().hwsel_forest_pack_bytes(C.byref(s), C.byref(n)))
    image = np.zeros(int(n.value), np.uint8)
    _check("hwsel_forest_pack_host", lib().hwsel_forest_pack_host(C.byref(s), image.ctypes.data, image.size))
    return image


def hwsel_forest_workspace_bytes(forest: dict, R: int) -> int:
    n = C.c_size_t(0)
    s = forest_struct(forest)
    _check("hwsel_forest_workspace_bytes", lib().hwsel_forest_workspace_bytes(C.byref(s), R, C.byref(n)))
    return int(n.value)


def hwsel_forest_score(forest: dict, X: torch.Tensor, scores: torch.Tensor | None = None,
                       packed: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                       stream=None) -> torch.Tensor:
    """Score rows of X.  With ``packed`` (from hwsel_forest_pack) the fast
    path runs and ``workspace`` (allocated here if None) holds its bins and
    partial sums."""
    R = X.shape[0]
    _matrix(X, "X", int(forest["n_features"]))
    _forest_arrays(forest)
    if scores is None:
        scores = _empty(R, torch.float32, X.device, stream)
    _arg(scores, "scores", F32, R, X)
    ws_bytes = 0
    if packed is not None:
        _packed_image(forest, packed, X)
        if workspace is None:
            workspace = _empty(hwsel_forest_workspace_bytes(forest, R), torch.uint8, X.device, stream)
        _arg(workspace, "workspace", U8, 0, X)
        ws_bytes = workspace.numel() * workspace.element_size()
    s = forest_struct(forest)
    _check("hwsel_forest_score", lib().hwsel_forest_score(
        C.byref(s), _ptr(packed), _ptr(X), R, X.stride(0), _ptr(scores), _ptr(workspace), ws_bytes,
        _stream(stream)))
    return scores


def hwsel_forest_score_checked(forest: dict, X: torch.Tensor, packed: torch.Tensor, with_hash: bool = True,
                               leaf_rows: tuple[int, int] | None = None, scores: torch.Tensor | None = None,
                               workspace: torch.Tensor | None = None, stream=None):
    """The packed traversal with its check outputs.  Returns (scores, leaf_hash
    uint64-as-int64 [R] or None, leaf_idx int16 [n][T] for the row range
    ``leaf_rows`` = (row0, n) or None)."""
    R = X.shape[0]
    _matrix(X, "X", int(forest["n_features"]))
    _forest_arrays(forest)
    _packed_image(forest, packed, X)
    if scores is None:
        scores = _empty(R, torch.float32, X.device, stream)
    _arg(scores, "scores", F32, R, X)
    if workspace is None:
        workspace = _empty(hwsel_forest_workspace_bytes(forest, R), torch.uint8, X.device, stream)
    _arg(workspace, "workspace", U8, 0, X)
    lh = _empty(R, torch.int64, X.device, stream) if with_hash else None
    li, row0, n = None, 0, 0
    if leaf_rows is not None:
        row0, n = leaf_rows
        li = _empty((n, int(forest["n_trees"])), torch.int16, X.device, stream)
    s = forest_struct(forest)
    _check("hwsel_forest_score_checked", lib().hwsel_forest_score_checked(
        C.byref(s), _ptr(packed), _ptr(X), R, X.stride(0), _ptr(scores), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(lh), _ptr(li), row0, n, _stream(stream)))
    return scores, lh, li


def hwsel_forest_leaves(forest: dict, X: torch.Tensor, rows: torch.Tensor,
                        leaf_idx: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    n = rows.shape[0]
    _matrix(X, "X", int(forest["n_features"]))
    _forest_arrays(forest)
    _arg(rows, "rows", I64, 0, X)
    if leaf_idx is None:
        leaf_idx = _empty((n, int(forest["n_trees"])), torch.int16, X.device, stream)
    _arg(leaf_idx, "leaf_idx", U16, n * int(forest["n_trees"]), X)
    s = forest_struct(forest)
    _check("hwsel_forest_leaves", lib().hwsel_forest_leaves(
        C.byref(s), _ptr(X), X.shape[0], X.stride(0), _ptr(_dev(rows, "rows")), n, _ptr(leaf_idx),
        _stream(stream)))
    return leaf_idx


def mlp_struct(m: dict) -> hwsel_mlp_t:
    return hwsel_mlp_t(128, 512, 512, 256, *[_ptr(m[n]) for n in
                                             ("mean", "inv_std", "W1", "W2", "W3", "W4", "b1", "b2", "b3", "b4")])


def hwsel_mlp_pack(mlp: dict, packed: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Arrange W1..W3 once for the matrix-core kernel; returns the image."""
    _mlp_arrays(mlp)
    s = mlp_struct(mlp)
    n = C.c_size_t(0)
    _check("hwsel_mlp_pack_bytes", lib().hwsel_mlp_pack_bytes(C.byref(s), C.byref(n)))
    if packed is None:
        packed = _empty(int(n.value), torch.uint8, mlp["W1"].device, stream)
    _arg(packed, "packed", U8, int(n.value), mlp["W1"])
    _check("hwsel_mlp_pack", lib().hwsel_mlp_pack(C.byref(s), _ptr(packed), packed.numel(), _stream(stream)))
    return packed


def _mlp_arrays(mlp: dict) -> None:
    sizes = dict(mean=128, inv_std=128, W1=512 * 128, W2=512 * 512, W3=256 * 512, W4=256, b1=512, b2=512, b3=256,
                 b4=1)
    ref = mlp["W1"]
    for n, k in sizes.items():
        _arg(mlp[n], n, U16 if n.startswith("W") else F32, k, ref)


def hwsel_mlp_score(mlp: dict, X: torch.Tensor, scores: torch.Tensor | None = None,
                    packed: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    R = X.shape[0]
    _matrix(X, "X", 128)
    _mlp_arrays(mlp)
    if scores is None:
        scores = _empty(R, torch.float32, X.device, stream)
    _arg(scores, "scores", F32, R, X)
    if packed is not None:
        n = C.c_size_t(0)
        _check("hwsel_mlp_pack_bytes", lib().hwsel_mlp_pack_bytes(C.byref(mlp_struct(mlp)), C.byref(n)))
        _arg(packed, "packed", U8, int(n.value), X)
    s = mlp_struct(mlp)
    _check("hwsel_mlp_score", lib().hwsel_mlp_score(C.byref(s), _ptr(packed), _ptr(X), R, X.stride(0),
                                                    _ptr(scores), _stream(stream)))
    return scores


def hwsel_topk_per_problem(scores: torch.Tensor, seg_offsets: torch.Tensor, k: int,
                           idx: torch.Tensor | None = None, vals: torch.Tensor | None = None,
                           with_vals: bool = True, stream=None):
    P = seg_offsets.shape[0] - 1
    _arg(scores, "scores", F32)
    _arg(seg_offsets, "seg_offsets", I64, 1, scores)
    if idx is None:
        idx = _empty((P, k), torch.int32, scores.device, stream)
    if vals is None and with_vals:
        vals = _empty((P, k), torch.float32, scores.device, stream)
    _arg(idx, "idx", I32, P * k, scores)
    if vals is not None:
        _arg(vals, "vals", F32, P * k, scores)
    _check("hwsel_topk_per_problem", lib().hwsel_topk_per_problem(
        _ptr(_dev(scores, "scores")), _ptr(_dev(seg_offsets, "seg_offsets")), P, k, _ptr(idx), _ptr(vals),
        _stream(stream)))
    return idx, vals


def hwsel_regret(runtimes: torch.Tensor, seg_offsets: torch.Tensor, idx: torch.Tensor,
                 r1: torch.Tensor | None = None, rk: torch.Tensor | None = None,
                 best: torch.Tensor | None = None, stream=None):
    P, k = idx.shape
    dev = runtimes.device
    _arg(runtimes, "runtimes", F32)
    _arg(seg_offsets, "seg_offsets", I64, P + 1, runtimes)
    _arg(idx, "idx", I32, P * k, runtimes)
    r1 = _empty(P, torch.float32, dev, stream) if r1 is None else r1
    rk = _empty(P, torch.float32, dev, stream) if rk is None else rk
    best = _empty(P, torch.int32, dev, stream) if best is None else best
    _arg(r1, "r1", F32, P, runtimes)
    _arg(rk, "rk", F32, P, runtimes)
    _arg(best, "best", I32, P, runtimes)
    _check("hwsel_regret", lib().hwsel_regret(
        _ptr(_dev(runtimes, "runtimes")), _ptr(_dev(seg_offsets, "seg_offsets")), P, _ptr(_dev(idx, "idx")), k,
        _ptr(r1), _ptr(rk), _ptr(best), _stream(stream)))
    return r1, rk, best


def hwsel_select_forest_workspace_bytes(forest: dict, R: int) -> int:
    n = C.c_size_t(0)
    s = forest_struct(forest)
    _check("hwsel_select_forest_workspace_bytes", lib().hwsel_select_forest_workspace_bytes(C.byref(s), R,
                                                                                            C.byref(n)))
    return int(n.value)


def hwsel_select_forest(hw: dict, problems: torch.Tensor, seg_offsets: torch.Tensor, cands: dict, n_features: int,
                        forest: dict, packed: torch.Tensor, k: int, workspace: torch.Tensor | None = None,
                        idx: torch.Tensor | None = None, vals: torch.Tensor | None = None,
                        scores: torch.Tensor | None = None, with_vals: bool = True, stream=None):
    """Fused features -> packed forest -> top-k; returns (idx, vals, scores)."""
    P = problems.shape[0]
    R = cands["tile_m"].shape[0]
    dev = problems.device
    _forest_arrays(forest)
    _packed_image(forest, packed, problems)
    if workspace is None:
        workspace = _empty(hwsel_select_forest_workspace_bytes(forest, R), torch.uint8, dev, stream)
    _arg(workspace, "workspace", U8, 0, problems)
    if idx is None:
        idx = _empty((P, k), torch.int32, dev, stream)
    if vals is None and with_vals:
        vals = _empty((P, k), torch.float32, dev, stream)
    _arg(idx, "idx", I32, P * k, problems)
    if vals is not None:
        _arg(vals, "vals", F32, P * k, problems)
    if scores is not None:
        _arg(scores, "scores", F32, R, problems)
    cs = _cands_struct(cands, R, problems)
    f = forest_struct(forest)
    _check("hwsel_select_forest", lib().hwsel_select_forest(
        hw_struct(hw), _ptr(_dev(problems, "problems")), P, _ptr(_dev(seg_offsets, "seg_offsets")), C.byref(cs), R,
        n_features, C.byref(f), _ptr(packed), k, _ptr(idx), _ptr(vals), _ptr(scores), _ptr(workspace),
        workspace.numel(), _stream(stream)))
    return idx, vals, scores


HWSEL_EVAL_FIELDS = 9
HWSEL_CATALOGUE_SIZE = 534600


def hwsel_evaluate(runtimes: torch.Tensor, seg_offsets: torch.Tensor, idx: torch.Tensor,
                   workspace: torch.Tensor | None = None, per_group: bool = True, stream=None):
    """Returns (out fp64 [9], regret fp64 [P], rank int32 [P], ybar fp64 [P]);
    the per-group arrays are None unless per_group."""
    P, k = idx.shape
    dev = runtimes.device
    n = C.c_size_t(0)
    _check("hwsel_evaluate_workspace_bytes", lib().hwsel_evaluate_workspace_bytes(P, C.byref(n)))
    _arg(runtimes, "runtimes", F32)
    _arg(seg_offsets, "seg_offsets", I64, P + 1, runtimes)
    _arg(idx, "idx", I32, P * k, runtimes)
    if workspace is None:
        workspace = _empty(int(n.value), torch.uint8, dev, stream)
    _arg(workspace, "workspace", U8, 0, runtimes)
    out = _empty(HWSEL_EVAL_FIELDS, torch.float64, dev, stream)
    reg = rank = ybar = None
    if per_group:
        reg = _empty(P, torch.float64, dev, stream)
        rank = _empty(P, torch.int32, dev, stream)
        ybar = _empty(P, torch.float64, dev, stream)
    _check("hwsel_evaluate", lib().hwsel_evaluate(
        _ptr(_dev(runtimes, "runtimes")), _ptr(_dev(seg_offsets, "seg_offsets")), P, _ptr(_dev(idx, "idx")), k,
        _ptr(out), _ptr(reg), _ptr(rank), _ptr(ybar), _ptr(workspace), workspace.numel(), _stream(stream)))
    return out, reg, rank, ybar


HWSEL_EVAL_NOALLOC_MAX_P = 65536


def hwsel_evaluate_noalloc(runtimes: torch.Tensor, seg_offsets: torch.Tensor, idx: torch.Tensor,
                           out: torch.Tensor | None = None, regret: torch.Tensor | None = None,
                           rank: torch.Tensor | None = None, ybar: torch.Tensor | None = None,
                           per_group: bool = True, stream=None):
    """hwsel_evaluate without a workspace (the library's own scratch array);
    outputs as for hwsel_evaluate.  Output tensors may be passed in."""
    P, k = idx.shape
    dev = runtimes.device
    _arg(runtimes, "runtimes", F32)
    _arg(seg_offsets, "seg_offsets", I64, P + 1, runtimes)
    _arg(idx, "idx", I32, P * k, runtimes)
    if out is None:
        out = _empty(HWSEL_EVAL_FIELDS, torch.float64, dev, stream)
    _arg(out, "out", (torch.float64,), HWSEL_EVAL_FIELDS, runtimes)
    if per_group:
        regret = _empty(P, torch.float64, dev, stream) if regret is None else regret
        rank = _empty(P, torch.int32, dev, stream) if rank is None else rank
        ybar = _empty(P, torch.float64, dev, stream) if ybar is None else ybar
    for n, t, dt in (("regret", regret, (torch.float64,)), ("rank", rank, I32), ("ybar", ybar, (torch.float64,))):
        if t is not None:
            _arg(t, n, dt, P, runtimes)
    _check("hwsel_evaluate_noalloc", lib().hwsel_evaluate_noalloc(
        _ptr(_dev(runtimes, "runtimes")), _ptr(_dev(seg_offsets, "seg_offsets")), P, _ptr(_dev(idx, "idx")), k,
        _ptr(out), _ptr(regret), _ptr(rank), _ptr(ybar), _stream(stream)))
    return out, regret, rank, ybar


def hwsel_static_config(runtimes: torch.Tensor, seg_offsets: torch.Tensor, config_id: torch.Tensor,
                        n_configs: int, workspace: torch.Tensor | None = None, stream=None):
    """Returns (best int32 [2] = (id, count), mean_y fp64 [1]) on the device."""
    P = seg_offsets.shape[0] - 1
    dev = runtimes.device
    n = C.c_size_t(0)
    _check("hwsel_static_config_workspace_bytes",
           lib().hwsel_static_config_workspace_bytes(P, n_configs, C.byref(n)))
    _arg(runtimes, "runtimes", F32)
    _arg(seg_offsets, "seg_offsets", I64, P + 1, runtimes)
    _arg(config_id, "config_id", I32, int(runtimes.numel()), runtimes)
    if workspace is None:
        workspace = _empty(int(n.value), torch.uint8, dev, stream)
    _arg(workspace, "workspace", U8, 0, runtimes)
    best = _empty(2, torch.int32, dev, stream)
    mean_y = _empty(1, torch.float64, dev, stream)
    _check("hwsel_static_config", lib().hwsel_static_config(
        _ptr(_dev(runtimes, "runtimes")), _ptr(_dev(seg_offsets, "seg_offsets")), P,
        _ptr(_dev(config_id, "config_id")), n_configs, _ptr(best), _ptr(mean_y), _ptr(workspace),
        workspace.numel(), _stream(stream)))
    return best, mean_y


def hwsel_catalogue_mask(hw: dict, problems: torch.Tensor, flags: int = 0, mask: torch.Tensor | None = None,
                         stream=None):
    """Returns (mask uint8 [P, 534600], n_valid int64 [P])."""
    P = problems.shape[0]
    dev = problems.device
    if mask is None:
        mask = _empty((P, HWSEL_CATALOGUE_SIZE), torch.uint8, dev, stream)
    _arg(mask, "mask", U8, P * HWSEL_CATALOGUE_SIZE, problems)
    n_valid = _empty(P, torch.int64, dev, stream)
    _check("hwsel_catalogue_mask", lib().hwsel_catalogue_mask(
        hw_struct(hw), _ptr(_dev(problems, "problems")), P, flags, _ptr(mask), _ptr(n_valid), _stream(stream)))
    return mask, n_valid


def hwsel_catalogue_compact(mask: torch.Tensor, n_valid: torch.Tensor, capacity: int,
                            point: torch.Tensor | None = None, stream=None):
    """Returns (seg_offsets int64 [P+1], point int32 [capacity])."""
    P = mask.shape[0]
    dev = mask.device
    _arg(mask, "mask", U8, P * HWSEL_CATALOGUE_SIZE)
    _arg(n_valid, "n_valid", I64, P, mask)
    seg = _empty(P + 1, torch.int64, dev, stream)
    if point is None:
        point = _empty(max(capacity, 1), torch.int32, dev, stream)
    _arg(point, "point", I32, capacity, mask)
    _check("hwsel_catalogue_compact", lib().hwsel_catalogue_compact(
        _ptr(_dev(mask, "mask")), _ptr(_dev(n_valid, "n_valid")), P, _ptr(seg), _ptr(point), capacity,
        _stream(stream)))
    return seg, point


def hwsel_catalogue_candidates(problems: torch.Tensor, seg_offsets: torch.Tensor, R: int,
                               point: torch.Tensor | None = None, out: dict | None = None, stream=None) -> dict:
    """Candidate SoA (name -> device tensor of length R) of catalogue points;
    ``out`` may supply the field tensors (allocated here if None)."""
    P = problems.shape[0]
    dev = problems.device
    wide = ("tile_m", "tile_n", "tile_k", "inst_n")
    if out is None:
        out = {n: _empty(R, torch.int16 if n in wide else torch.uint8, dev, stream) for n in CAND_FIELDS}
    _arg(seg_offsets, "seg_offsets", I64, P + 1, problems)
    if point is not None:
        _arg(point, "point", I32, R, problems)
    for n in CAND_FIELDS:
        t = _dev(out[n], n)
        if t.element_size() != (2 if n in wide else 1) or t.numel() < R or t.device != problems.device:
            raise ValueError(f"{n} must hold at least R elements of {2 if n in wide else 1} byte(s) on "
                             f"{problems.device}")
    s = hwsel_cands_out_t(*[_ptr(out[n]) for n in CAND_FIELDS])
    _check("hwsel_catalogue_candidates", lib().hwsel_catalogue_candidates(
        _ptr(_dev(problems, "problems")), P, _ptr(_dev(seg_offsets, "seg_offsets")), _ptr(point), R, C.byref(s),
        _stream(stream)))
    return out


# ----------------------------------------------------------------------------
# 8-bit matrices with block scales.  An operand is a dict: q uint8 [rows][ld],
# scale uint8 [ceil(rows / block_rows)][ld_scale], rows, cols, format,
# block_rows (see hwsel_fp8_t).
# ----------------------------------------------------------------------------
FP8_E4M3, FP8_E5M2 = 0, 1
FP8_BLOCK = 128


def hwsel_fp8_empty(rows: int, cols: int, format: int = FP8_E4M3, block_rows: int = 1, device="cuda") -> dict:
    """Buffers of an 8-bit [rows][cols] matrix, to be written by an entry point."""
    blocks = -(-cols // FP8_BLOCK)
    return dict(q=torch.empty((rows, blocks * FP8_BLOCK), dtype=torch.uint8, device=device),
                scale=torch.empty((-(-rows // block_rows), -(-blocks // 4) * 4), dtype=torch.uint8, device=device),
                rows=rows, cols=cols, format=format, block_rows=block_rows)


def hwsel_fp8_quantise(X: torch.Tensor, format: int = FP8_E4M3, block_rows: int = 1, transpose: bool = False,
                       mean: torch.Tensor | None = None, inv_std: torch.Tensor | None = None,
                       out: dict | None = None, stream=None) -> dict:
    """X (fp32 or bf16 [R][C]), or X transposed, in 8 bits with a scale for
    each block of 128; standardised on the way if mean and inv_std are given."""
    return (_binding or _calls()).fp8_quantise(X, format, block_rows, transpose, mean, inv_std, out, stream)


def hwsel_fp8_dequantise(m: dict, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
                         stream=None) -> torch.Tensor:
    """The values of an 8-bit matrix in bf16 or fp32."""
    return (_binding or _calls()).fp8_dequantise(m, dtype, out, stream)


def hwsel_fp8_transpose(m: dict, format: int = FP8_E4M3, block_rows: int = 1, out: dict | None = None,
                        stream=None) -> dict:
    """An 8-bit matrix transposed and quantised again along its own rows."""
    return (_binding or _calls()).fp8_transpose(m, format, block_rows, out, stream)


def hwsel_fp8_matmul_workspace_bytes(A: dict, B: dict) -> int:
    return (_binding or _calls()).fp8_matmul_workspace_bytes(A, B)


def hwsel_fp8_matmul(A: dict, B: dict, dtype: torch.dtype = torch.bfloat16, bias: torch.Tensor | None = None,
                     gelu: bool = False, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                     stream=None) -> torch.Tensor:
    """act(A B^T + bias) of 8-bit matrices A [M][K], B [N][K], in bf16 or fp32."""
    return (_binding or _calls()).fp8_matmul(A, B, dtype, bias, gelu, out, workspace, stream)


def hwsel_fp8_layer(A: dict, B: dict, bias: torch.Tensor | None = None, gelu: bool = False, out: dict | None = None,
                    workspace: torch.Tensor | None = None, stream=None) -> dict:
    """act(A B^T + bias) as an 8-bit matrix, the next layer's operand."""
    return (_binding or _calls()).fp8_layer(A, B, bias, gelu, out, workspace, stream)


def hwsel_sample_workspace_bytes(R: int, P: int, n_draws: int) -> int:
    n = C.c_size_t(0)
    _check("hwsel_sample_workspace_bytes", lib().hwsel_sample_workspace_bytes(R, P, n_draws, C.byref(n)))
    return int(n.value)


def hwsel_sample_per_problem(scores: torch.Tensor, seg_offsets: torch.Tensor, u: torch.Tensor, temperature=1.0,
                             top_k=0, top_p=1.0, min_p=0.0, idx: torch.Tensor | None = None,
                             prob: torch.Tensor | None = None, kept: torch.Tensor | None = None,
                             workspace: torch.Tensor | None = None, stream=None):
    """Draws u.shape[1] candidates of every problem from its scores by the
    random numbers u fp32 [P][draws].  Each setting is a number or a device
    tensor [P].  Returns (idx int32 [P][draws], prob fp32 [P][draws], kept
    int32 [P])."""
    return (_binding or _calls()).sample_per_problem(scores, seg_offsets, u, temperature, top_k, top_p, min_p, idx, prob, kept,
                                                     workspace, stream)


def hwsel_logprob_workspace_bytes(R: int, P: int, top: int = 0) -> int:
    n = C.c_size_t(0)
    _check("hwsel_logprob_workspace_bytes", lib().hwsel_logprob_workspace_bytes(R, P, top, C.byref(n)))
    return int(n.value)


def hwsel_logprob_per_problem(scores: torch.Tensor, seg_offsets: torch.Tensor, picks: torch.Tensor | None = None,
                              temperature=1.0, top: int = 0, logp: torch.Tensor | None = None,
                              entropy: torch.Tensor | None = None, norm: torch.Tensor | None = None,
                              top_idx: torch.Tensor | None = None, top_logp: torch.Tensor | None = None,
                              workspace: torch.Tensor | None = None, stream=None):
    """Log probabilities of every problem's candidates picks int32 [P][n] under
    the softmax of its scores at a temperature (a number or a device tensor
    [P]).  Returns (logp fp32 [P][n] or None, entropy fp32 [P], norm fp32
    [P][2], top_idx int32 [P][top] or None, top_logp fp32 [P][top] or None)."""
    return (_binding or _calls()).logprob_per_problem(scores, seg_offsets, picks, temperature, top, logp, entropy, norm,
                                                      top_idx, top_logp, workspace, stream)


def hwsel_logprob_gradient(scores: torch.Tensor, seg_offsets: torch.Tensor, norm: torch.Tensor,
                           picks: torch.Tensor | None = None, d_logp: torch.Tensor | None = None,
                           entropy: torch.Tensor | None = None, d_entropy: torch.Tensor | None = None,
                           temperature=1.0, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The scores' gradient fp32 [R] from those of hwsel_logprob_per_problem's
    logp [P][n] and, given d_entropy [P], of its entropy; norm and entropy as
    that call wrote them."""
    return (_binding or _calls()).logprob_gradient(scores, seg_offsets, norm, picks, d_logp, entropy, d_entropy,
                                                   temperature, out, stream)


def hwsel_dropout(x: torch.Tensor, p: float, seed: int = 0, offset: int = 0, state: torch.Tensor | None = None,
                  residual: torch.Tensor | None = None, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """residual + x with a share p of its elements dropped and the others
    divided by the share kept; the mask is a function of (seed, offset), or of
    the device tensor state int64 [2], and an element's place.  The gradient of
    x is the same call on the result's gradient, without a residual."""
    return (_binding or _calls()).dropout(x, p, seed, offset, state, residual, out, stream)


# ----------------------------------------------------------------------------
# Joins of blocks to a residual stream.  A join is a dict; its keys and what
# they are where they are missing: post_norm False, gate_sigmoid False,
# w_branch None, w_pre None (fp32 [cols]), eps 1e-6, stream_scale 1.0,
# branch_scale 1.0, p 0.0, seed 0, offset 0, state None (see hwsel_join_t).
# ----------------------------------------------------------------------------
def hwsel_block_join(join: dict, x: torch.Tensor, y: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                     dtype: torch.dtype | None = None, x1: torch.Tensor | None = None, z: torch.Tensor | None = None,
                     with_x1: bool = True, with_z: bool = True, stream=None):
    """x1 = stream_scale x + dropout(branch_scale g w_branch norm(y)) and z =
    w_pre norm(x1).  gate: [rows][cols], [rows][1] or None.  z has y's dtype,
    without y `dtype` or x's.  Returns (x1 or None, z or None)."""
    return (_binding or _calls()).block_join(join, x, y, gate, dtype, x1, z, with_x1, with_z, stream)


def hwsel_block_join_gradient_workspace_bytes(rows: int, cols: int) -> int:
    n, j = C.c_size_t(0), hwsel_join_t(rows=rows, cols=cols, eps=1e-6, stream_scale=1.0, branch_scale=1.0)
    _check("hwsel_block_join_gradient_workspace_bytes",
           lib().hwsel_block_join_gradient_workspace_bytes(C.byref(j), C.byref(n)))
    return int(n.value)


def hwsel_block_join_gradient(join: dict, x1: torch.Tensor, y: torch.Tensor | None = None,
                              gate: torch.Tensor | None = None, d_x1: torch.Tensor | None = None,
                              d_z: torch.Tensor | None = None, dx: torch.Tensor | None = None,
                              dy: torch.Tensor | None = None, dgate: torch.Tensor | None = None,
                              dw_branch: torch.Tensor | None = None, dw_pre: torch.Tensor | None = None,
                              workspace: torch.Tensor | None = None, stream=None):
    """Gradients of hwsel_block_join from those of x1 and z (either may be
    None), x1 as it was written.  Returns (dx, dy, dgate, dw_branch, dw_pre),
    None for what the join does not have."""
    return (_binding or _calls()).block_join_gradient(join, x1, y, gate, d_x1, d_z, dx, dy, dgate, dw_branch, dw_pre,
                                                      workspace, stream)


def declared_functions() -> list[str]:
    """Names of the functions include/hwsel.h declares."""
    import re
    text = open(HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(hwsel_[a-z0-9_]+)\s*\(", text)))
