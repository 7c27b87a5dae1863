"""ctypes binding of libscnn.so: argument marshalling only."""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence, Tuple

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(HERE, "libscnn.so")
_lib = None

ABS, SIGNED = 0, 1
FUSE_RELU, FUSE_MAXPOOL2 = 1, 2
FLAG_CAND_OVERFLOW, FLAG_OUT_OVERFLOW, FLAG_BAD_COORD, FLAG_UNSORTED = 1, 2, 4, 8
NNZ_LEN = 4
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}

EXPORTED_SYMBOLS = [
    "scnn_last_error", "scnn_version", "scnn_k_from_rho", "sparse_conv_fwd_max_rows", "sparse_conv_fwd_workspace",
    "sparse_conv_fwd", "attention_topk_workspace", "attention_topk", "sparse_relu_workspace", "sparse_relu",
    "sparse_maxpool_workspace", "sparse_maxpool", "scnn_validate_rows", "scnn_profile_enable",
    "scnn_profile_stage_count", "scnn_set_conv_path", "scnn_calibration_copy", "scnn_profile_stage_name", "scnn_profile_collect",
    "sparse_conv_bwd_workspace", "sparse_conv_bwd", "sparse_to_dense",
    "density_regulariser_workspace", "density_regulariser", "prune_weights", "sparse_conv_fwd_chained",
    "sparse_relu_static_max_rows", "sparse_relu_static", "scnn_last_conv_kernel",
    "linear_fwd_workspace", "linear_fwd", "linear_bwd_workspace", "linear_bwd", "layer_norm_fwd",
    "layer_norm_bwd_workspace", "layer_norm_bwd", "grad_clip_workspace", "grad_clip",
]


class ScnnError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libscnn error {code}: {msg}")
        self.code = code


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libscnn.so.  If it was never built, build it once (tests and the benchmark
    normally find it already built in-tree); a missing compiler is an error, not a fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        from .build import build
        build(force=False)
    L = ctypes.CDLL(_LIB_PATH)
    i32p = ctypes.POINTER(ctypes.c_int32)
    vp, i64, sz, ci, cu, dbl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int, ctypes.c_uint, ctypes.c_double
    L.scnn_last_error.restype = ctypes.c_char_p
    L.scnn_version.restype = ci
    L.scnn_k_from_rho.restype = i64
    L.scnn_k_from_rho.argtypes = [dbl, i64]
    L.sparse_conv_fwd_max_rows.restype = i64
    L.sparse_conv_fwd_max_rows.argtypes = [ci, i32p, ci, i64, i32p]
    L.sparse_conv_fwd_workspace.restype = sz
    L.sparse_conv_fwd_workspace.argtypes = [ci, i32p, ci, i64, ci, ci, i32p, cu, i64]
    L.sparse_conv_fwd.restype = ci
    L.sparse_conv_fwd.argtypes = [ci, i32p, ci, vp, vp, i64, ci, i32p, vp, vp, ci, dbl, ci, cu, vp, vp, i64, i64, vp,
                                  vp, sz, vp]
    L.sparse_conv_bwd_workspace.restype = sz
    L.sparse_conv_bwd_workspace.argtypes = [ci, i32p, ci, i64, ci, ci, i32p, i64]
    L.sparse_conv_bwd.restype = ci
    L.sparse_conv_bwd.argtypes = [ci, i32p, ci, vp, vp, i64, ci, i32p, vp, ci, vp, vp, i64, vp, vp, vp, vp, sz, vp]
    L.attention_topk_workspace.restype = sz
    L.attention_topk_workspace.argtypes = [ci, i32p, ci, i64, ci]
    L.attention_topk.restype = ci
    L.attention_topk.argtypes = [ci, i32p, ci, vp, vp, i64, ci, i64, ci, vp, vp, i64, vp, vp, sz, vp]
    L.sparse_relu_workspace.restype = sz
    L.sparse_relu_workspace.argtypes = [i64, ci]
    L.sparse_relu.restype = ci
    L.sparse_relu.argtypes = [ci, vp, vp, i64, ci, vp, vp, i64, vp, vp, sz, vp]
    L.sparse_relu_static_max_rows.restype = i64
    L.sparse_relu_static_max_rows.argtypes = []
    L.sparse_relu_static.restype = ci
    L.sparse_relu_static.argtypes = [ci, vp, vp, i64, ci, vp, vp, i64, vp, vp]
    L.sparse_maxpool_workspace.restype = sz
    L.sparse_maxpool_workspace.argtypes = [ci, i32p, ci, i64, ci]
    L.sparse_maxpool.restype = ci
    L.sparse_maxpool.argtypes = [ci, i32p, ci, ci, vp, vp, i64, ci, vp, vp, i64, vp, vp, sz, vp]
    L.sparse_to_dense.restype = ci
    L.sparse_to_dense.argtypes = [ci, i32p, ci, vp, vp, i64, vp, ci, vp, vp]
    L.sparse_conv_fwd_chained.restype = ci
    L.sparse_conv_fwd_chained.argtypes = [ci, i32p, ci, vp, vp, i64, vp, ci, i32p, vp, vp, ci, dbl, ci, cu, vp, vp, i64,
                                          i64, vp, vp, sz, vp]
    L.density_regulariser_workspace.restype = sz
    L.density_regulariser_workspace.argtypes = []
    L.density_regulariser.restype = ci
    L.density_regulariser.argtypes = [vp, i64, vp, ci, i64, dbl, dbl, dbl, dbl, dbl, vp, i64, vp, vp, vp, sz, vp]
    L.prune_weights.restype = ci
    L.prune_weights.argtypes = [vp, vp, i64, ctypes.c_float, vp, vp]
    L.linear_fwd_workspace.restype = sz
    L.linear_fwd_workspace.argtypes = [ci, i64, i64, i64]
    L.linear_fwd.restype = ci
    L.linear_fwd.argtypes = [ci, vp, i64, vp, i64, vp, vp, i64, ci, vp, vp, vp, vp, sz, vp]
    L.linear_bwd_workspace.restype = sz
    L.linear_bwd_workspace.argtypes = [ci, i64, i64, i64, ci]
    L.linear_bwd.restype = ci
    L.linear_bwd.argtypes = [ci, vp, i64, vp, i64, vp, i64, ci, vp, vp, vp, vp, vp, vp, sz, vp]
    L.layer_norm_fwd.restype = ci
    L.layer_norm_fwd.argtypes = [ci, vp, i64, vp, i64, vp, vp, dbl, vp, vp, vp, vp]
    L.layer_norm_bwd_workspace.restype = sz
    L.layer_norm_bwd_workspace.argtypes = [ci, i64, i64]
    L.layer_norm_bwd.restype = ci
    L.layer_norm_bwd.argtypes = [ci, vp, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.grad_clip_workspace.restype = sz
    L.grad_clip_workspace.argtypes = [ci, ctypes.POINTER(i64)]
    L.grad_clip.restype = ci
    L.grad_clip.argtypes = [ci, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(i64), ctypes.POINTER(ci), dbl, vp, vp,
                            sz, vp]
    L.scnn_validate_rows.restype = ci
    L.scnn_validate_rows.argtypes = [ci, i32p, ci, vp, i64, vp, sz, vp]
    L.scnn_calibration_copy.restype = ci
    L.scnn_calibration_copy.argtypes = [vp, vp, sz, vp]
    L.scnn_last_conv_kernel.restype = ctypes.c_char_p
    L.scnn_last_conv_kernel.argtypes = []
    L.scnn_set_conv_path.restype = ci
    L.scnn_set_conv_path.argtypes = [ci]
    L.scnn_profile_enable.restype = ci
    L.scnn_profile_enable.argtypes = [ci]
    L.scnn_profile_stage_count.restype = ci
    L.scnn_profile_stage_name.restype = ctypes.c_char_p
    L.scnn_profile_stage_name.argtypes = [ci]
    L.scnn_profile_collect.restype = ci
    L.scnn_profile_collect.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]
    _lib = L
    return L


def _check(L, rc: int):
    if rc != 0:
        raise ScnnError(rc, L.scnn_last_error().decode())


def _i32arr(v: Sequence[int]):
    return (ctypes.c_int32 * len(v))(*[int(x) for x in v])


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dev(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}")
    return t.contiguous()


def k_from_rho(rho_up: float, n_sites: int) -> int:
    return int(load_library().scnn_k_from_rho(float(rho_up), int(n_sites)))


def sparse_conv_fwd_max_rows(extent, batch, nnz_in, ksize) -> int:
    L = load_library()
    r = int(L.sparse_conv_fwd_max_rows(len(extent), _i32arr(extent), int(batch), int(nnz_in), _i32arr(ksize)))
    if r < 0:
        _check(L, r)
    return r


def sparse_conv_fwd_workspace(extent, batch, nnz_in, c_in, c_out, ksize, fuse=0, cand_capacity=0) -> int:
    L = load_library()
    r = int(L.sparse_conv_fwd_workspace(len(extent), _i32arr(extent), int(batch), int(nnz_in), int(c_in), int(c_out),
                                        _i32arr(ksize), int(fuse), int(cand_capacity)))
    if r == 0:
        raise ScnnError(-1, L.scnn_last_error().decode())
    return r


def _finish(out_coords, out_feats, nnz, sync):
    if not sync:
        return out_coords, out_feats, nnz
    n = nnz.cpu()
    rows, flags = int(n[0]), int(n[2])
    if flags & (FLAG_CAND_OVERFLOW | FLAG_OUT_OVERFLOW):
        raise ScnnError(-2, f"capacity exceeded (rows={rows}, candidates={int(n[1])}, flags={flags})")
    return out_coords[:rows], out_feats[:rows], n


def sparse_conv_fwd(extent, batch, coords, feats, ksize, w, bias=None, *, rho_up=1.0, topk_mode=ABS, relu=False,
                    pool=False, out_capacity: Optional[int] = None, cand_capacity: int = 0, workspace=None,
                    out=None, stream=None, sync=True):
    """Forward sparse convolution + attention (+ReLU, +2^d max-pool).  Returns (out_coords, out_feats, nnz)
    where nnz is the int64[4] counter vector (device tensor when sync=False, host tensor otherwise)."""
    L = load_library()
    ndim = len(extent)
    coords = _dev(coords, torch.int32, "coords")
    feats = _dev(feats, torch.float32, "feats")
    w = _dev(w, torch.float32, "w")
    if bias is not None:
        bias = _dev(bias, torch.float32, "bias")
    nnz_in, c_in = feats.shape
    taps, c_in_w, c_out = w.shape
    if c_in_w != c_in or coords.shape != (nnz_in, 1 + ndim):
        raise ValueError("shape mismatch between coords, feats and w")
    t = 1
    for s in ksize:
        t *= int(s)
    if t != taps:
        raise ValueError("w.shape[0] != prod(ksize)")
    if bias is not None and bias.shape != (c_out,):
        raise ValueError("bias must be [c_out]")
    fuse = (FUSE_RELU if relu else 0) | (FUSE_MAXPOOL2 if pool else 0)
    ext, ks = _i32arr(extent), _i32arr(ksize)
    dev = feats.device
    if cand_capacity <= 0:
        cand_capacity = int(L.sparse_conv_fwd_max_rows(ndim, ext, int(batch), nnz_in, ks))
    if out_capacity is None:
        out_capacity = cand_capacity
    need = int(L.sparse_conv_fwd_workspace(ndim, ext, int(batch), nnz_in, c_in, c_out, ks, fuse, cand_capacity))
    if need == 0:
        raise ScnnError(-1, L.scnn_last_error().decode())
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    if out is None:
        out_coords = torch.empty((out_capacity, 1 + ndim), dtype=torch.int32, device=dev)
        out_feats = torch.empty((out_capacity, c_out), dtype=torch.float32, device=dev)
        nnz = torch.zeros(NNZ_LEN, dtype=torch.int64, device=dev)
    else:
        out_coords, out_feats, nnz = out
    rc = L.sparse_conv_fwd(ndim, ext, int(batch), _ptr(coords), _ptr(feats), nnz_in, c_in, ks, _ptr(w), _ptr(bias),
                           c_out, float(rho_up), int(topk_mode), fuse, _ptr(out_coords), _ptr(out_feats),
                           int(out_capacity), int(cand_capacity), _ptr(nnz), _ptr(workspace), workspace.numel(),
                           _stream(stream))
    _check(L, rc)
    return _finish(out_coords, out_feats, nnz, sync)


def sparse_conv_bwd(extent, batch, coords, feats, ksize, w, g_coords, g_feats, *, workspace=None, out=None,
                    stream=None, sync=True):
    """Back-propagation through the convolution (Algorithm 2 with the masks of Eq. 3).
    Returns (bp_data [rows, C_in], bp_filter [T, C_in, C_out], info int64[4])."""
    L = load_library()
    ndim = len(extent)
    coords = _dev(coords, torch.int32, "coords")
    feats = _dev(feats, torch.float32, "feats")
    w = _dev(w, torch.float32, "w")
    g_coords = _dev(g_coords, torch.int32, "g_coords")
    g_feats = _dev(g_feats, torch.float32, "g_feats")
    nnz_in, c_in = feats.shape
    taps, c_in_w, c_out = w.shape
    g_rows = g_feats.shape[0]
    if c_in_w != c_in or coords.shape != (nnz_in, 1 + ndim):
        raise ValueError("shape mismatch between coords, feats and w")
    if g_feats.shape[1] != c_out or g_coords.shape != (g_rows, 1 + ndim):
        raise ValueError("shape mismatch between g_coords, g_feats and w")
    t = 1
    for s in ksize:
        t *= int(s)
    if t != taps:
        raise ValueError("w.shape[0] != prod(ksize)")
    ext, ks = _i32arr(extent), _i32arr(ksize)
    dev = feats.device
    need = int(L.sparse_conv_bwd_workspace(ndim, ext, int(batch), nnz_in, c_in, c_out, ks, g_rows))
    if need == 0:
        raise ScnnError(-1, L.scnn_last_error().decode())
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    if out is None:
        bp_data = torch.empty((nnz_in, c_in), dtype=torch.float32, device=dev)
        bp_filter = torch.empty((taps, c_in, c_out), dtype=torch.float32, device=dev)
        info = torch.zeros(NNZ_LEN, dtype=torch.int64, device=dev)
    else:
        bp_data, bp_filter, info = out
    rc = L.sparse_conv_bwd(ndim, ext, int(batch), _ptr(coords), _ptr(feats), nnz_in, c_in, ks, _ptr(w), c_out,
                           _ptr(g_coords), _ptr(g_feats), g_rows, _ptr(bp_data), _ptr(bp_filter), _ptr(info),
                           _ptr(workspace), workspace.numel(), _stream(stream))
    _check(L, rc)
    if sync:
        info = info.cpu()
    return bp_data, bp_filter, info


def sparse_conv_bwd_workspace(extent, batch, nnz_in, c_in, c_out, ksize, g_rows) -> int:
    L = load_library()
    r = int(L.sparse_conv_bwd_workspace(len(extent), _i32arr(extent), int(batch), int(nnz_in), int(c_in), int(c_out),
                                        _i32arr(ksize), int(g_rows)))
    if r == 0:
        raise ScnnError(-1, L.scnn_last_error().decode())
    return r


class ChainedLayer:
    """One layer of a chain that runs without host reads: buffers sized once from capacities, the input row count
    taken on the device.  `in_capacity` bounds the rows of the input arrays.  Run a chain once eagerly before
    capturing it in a HIP graph: the first launch of a matrix-core kernel sets that kernel's shared-memory attribute,
    which is not a stream operation."""

    def __init__(self, extent, batch, in_capacity, c_in, ksize, w, *, bias=None, rho_up=1.0, topk_mode=ABS,
                 relu=False, pool=False):
        L = load_library()
        self.extent, self.batch, self.ksize = tuple(int(e) for e in extent), int(batch), tuple(int(k) for k in ksize)
        self.ndim = len(self.extent)
        self.w = _dev(w, torch.float32, "w")
        self.bias = None if bias is None else _dev(bias, torch.float32, "bias")
        self.c_in, self.c_out = int(c_in), int(self.w.shape[2])
        self.in_capacity = max(1, int(in_capacity))
        self.rho_up, self.topk_mode = float(rho_up), int(topk_mode)
        self.fuse = (FUSE_RELU if relu else 0) | (FUSE_MAXPOOL2 if pool else 0)
        ext, ks = _i32arr(self.extent), _i32arr(self.ksize)
        self.cand_capacity = int(L.sparse_conv_fwd_max_rows(self.ndim, ext, self.batch, self.in_capacity, ks))
        need = int(L.sparse_conv_fwd_workspace(self.ndim, ext, self.batch, self.in_capacity, self.c_in, self.c_out, ks,
                                               self.fuse, self.cand_capacity))
        if need == 0:
            raise ScnnError(-1, L.scnn_last_error().decode())
        dev = self.w.device
        self.out_extent = tuple((e + 1) // 2 for e in self.extent) if pool else self.extent
        n_out = self.batch
        for e in self.out_extent:
            n_out *= e
        self.out_capacity = min(self.cand_capacity, n_out)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        self.out_coords = torch.empty((self.out_capacity, 1 + self.ndim), dtype=torch.int32, device=dev)
        self.out_feats = torch.empty((self.out_capacity, self.c_out), dtype=torch.float32, device=dev)
        self.nnz = torch.zeros(NNZ_LEN, dtype=torch.int64, device=dev)

    def __call__(self, coords, feats, nnz_in_dev, stream=None):
        """Enqueue the layer; returns (out_coords, out_feats, nnz) -- full-capacity buffers, the count stays on the
        device in nnz[0]."""
        L = load_library()
        if coords.shape[0] > self.in_capacity or feats.shape != (coords.shape[0], self.c_in):
            raise ValueError("input arrays do not fit this layer")
        rc = L.sparse_conv_fwd_chained(self.ndim, _i32arr(self.extent), self.batch, _ptr(coords), _ptr(feats),
                                       coords.shape[0], _ptr(nnz_in_dev), self.c_in, _i32arr(self.ksize), _ptr(self.w),
                                       _ptr(self.bias), self.c_out, self.rho_up, self.topk_mode, self.fuse,
                                       _ptr(self.out_coords), _ptr(self.out_feats), self.out_capacity,
                                       self.cand_capacity, _ptr(self.nnz), _ptr(self.workspace),
                                       self.workspace.numel(), _stream(stream))
        _check(L, rc)
        return self.out_coords, self.out_feats, self.nnz


def attention_topk(extent, batch, coords, resp, k, topk_mode=ABS, *, out_capacity=None, workspace=None, stream=None,
                   sync=True):
    L = load_library()
    ndim = len(extent)
    coords = _dev(coords, torch.int32, "coords")
    resp = _dev(resp, torch.float32, "resp")
    rows, ch = resp.shape
    ext = _i32arr(extent)
    dev = resp.device
    if out_capacity is None:
        out_capacity = rows
    need = int(L.attention_topk_workspace(ndim, ext, int(batch), rows, ch))
    if need == 0:
        raise ScnnError(-1, "attention_topk_workspace: bad arguments")
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    out_coords = torch.empty((out_capacity, 1 + ndim), dtype=torch.int32, device=dev)
    out_feats = torch.empty((out_capacity, ch), dtype=torch.float32, device=dev)
    nnz = torch.zeros(NNZ_LEN, dtype=torch.int64, device=dev)
    rc = L.attention_topk(ndim, ext, int(batch), _ptr(coords), _ptr(resp), rows, ch, int(k), int(topk_mode),
                          _ptr(out_coords), _ptr(out_feats), int(out_capacity), _ptr(nnz), _ptr(workspace),
                          workspace.numel(), _stream(stream))
    _check(L, rc)
    return _finish(out_coords, out_feats, nnz, sync)


def sparse_relu(ndim, coords, feats, *, out_capacity=None, workspace=None, stream=None, sync=True):
    L = load_library()
    coords = _dev(coords, torch.int32, "coords")
    feats = _dev(feats, torch.float32, "feats")
    rows, ch = feats.shape
    dev = feats.device
    if out_capacity is None:
        out_capacity = rows
    need = int(L.sparse_relu_workspace(rows, ch))
    if need == 0:
        raise ScnnError(-1, "sparse_relu_workspace: bad arguments")
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    out_coords = torch.empty((out_capacity, 1 + ndim), dtype=torch.int32, device=dev)
    out_feats = torch.empty((out_capacity, ch), dtype=torch.float32, device=dev)
    nnz = torch.zeros(NNZ_LEN, dtype=torch.int64, device=dev)
    rc = L.sparse_relu(int(ndim), _ptr(coords), _ptr(feats), rows, ch, _ptr(out_coords), _ptr(out_feats),
                       int(out_capacity), _ptr(nnz), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(L, rc)
    return _finish(out_coords, out_feats, nnz, sync)


def sparse_relu_static_max_rows() -> int:
    return int(load_library().sparse_relu_static_max_rows())


def sparse_relu_static(ndim, coords, feats, out_coords, out_feats, nnz, *, stream=None):
    """sparse_relu on the library's own scratch array: every buffer is the caller's, nothing is allocated here."""
    L = load_library()
    coords = _dev(coords, torch.int32, "coords")
    feats = _dev(feats, torch.float32, "feats")
    rows, ch = feats.shape
    rc = L.sparse_relu_static(int(ndim), _ptr(coords), _ptr(feats), rows, ch, _ptr(out_coords), _ptr(out_feats),
                              int(out_feats.shape[0]), _ptr(nnz), _stream(stream))
    _check(L, rc)


def sparse_maxpool(extent, batch, coords, feats, window=2, *, out_capacity=None, workspace=None, stream=None,
                   sync=True):
    L = load_library()
    ndim = len(extent)
    coords = _dev(coords, torch.int32, "coords")
    feats = _dev(feats, torch.float32, "feats")
    rows, ch = feats.shape
    ext = _i32arr(extent)
    dev = feats.device
    if out_capacity is None:
        out_capacity = rows
    need = int(L.sparse_maxpool_workspace(ndim, ext, int(batch), rows, ch))
    if need == 0:
        raise ScnnError(-1, "sparse_maxpool_workspace: bad arguments")
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    out_coords = torch.empty((out_capacity, 1 + ndim), dtype=torch.int32, device=dev)
    out_feats = torch.empty((out_capacity, ch), dtype=torch.float32, device=dev)
    nnz = torch.zeros(NNZ_LEN, dtype=torch.int64, device=dev)
    rc = L.sparse_maxpool(ndim, ext, int(batch), int(window), _ptr(coords), _ptr(feats), rows, ch, _ptr(out_coords),
                          _ptr(out_feats), int(out_capacity), _ptr(nnz), _ptr(workspace), workspace.numel(),
                          _stream(stream))
    _check(L, rc)
    return _finish(out_coords, out_feats, nnz, sync)


def sparse_to_dense(extent, batch, coords, feats, *, rows_dev=None, out=None, stream=None):
    """Dense fp32 [batch, channels, *extent] holding the rows' values, zero elsewhere."""
    L = load_library()
    coords = _dev(coords, torch.int32, "coords")
    feats = _dev(feats, torch.float32, "feats")
    rows, ch = feats.shape
    if out is None:
        out = torch.empty((int(batch), ch, *[int(e) for e in extent]), dtype=torch.float32, device=feats.device)
    _check(L, L.sparse_to_dense(len(extent), _i32arr(extent), int(batch), _ptr(coords), _ptr(feats), rows,
                                _ptr(rows_dev), ch, _ptr(out), _stream(stream)))
    return out


def density_regulariser(out_feats, n_sites_total, rho_up, o, b1, b2, lam, w, *, rows_dev=None, want_grad=True,
                        stream=None):
    """Eq. 4.  Returns (result double[4] = {rho, b, lambda * sum (w + b)^2, entries} on the device, grad_w or None)."""
    L = load_library()
    out_feats = _dev(out_feats, torch.float32, "out_feats")
    w = _dev(w, torch.float32, "w")
    rows, ch = out_feats.shape
    dev = w.device
    grad = torch.empty_like(w) if want_grad else None
    result = torch.zeros(4, dtype=torch.float64, device=dev)
    need = int(L.density_regulariser_workspace())
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _check(L, L.density_regulariser(_ptr(out_feats), rows, _ptr(rows_dev), ch, int(n_sites_total), float(rho_up),
                                    float(o), float(b1), float(b2), float(lam), _ptr(w), w.numel(), _ptr(grad),
                                    _ptr(result), _ptr(ws), need, _stream(stream)))
    return result, grad


def prune_weights(w, warned, eps, *, stream=None):
    """One-warning-shot pruning, in place on w (fp32) and warned (uint8).  Returns counts int64[2] on the device."""
    L = load_library()
    if not (w.is_cuda and warned.is_cuda and w.dtype == torch.float32 and warned.dtype == torch.uint8):
        raise ValueError("w must be a float32 and warned a uint8 GPU tensor")
    if not (w.is_contiguous() and warned.is_contiguous()) or w.numel() != warned.numel():
        raise ValueError("w and warned must be contiguous and of equal size")
    counts = torch.zeros(2, dtype=torch.int64, device=w.device)
    _check(L, L.prune_weights(_ptr(w), _ptr(warned), w.numel(), float(eps), _ptr(counts), _stream(stream)))
    return counts


# Layers on rows of values.  All tensors of a call live on one device, which need not be the current one.  With `stream`
# the call runs there and its new tensors belong to that stream: the caller orders other streams behind it.  No call records
# an autograd graph, whatever its tensors require: gradients come from the _bwd calls.  What a call writes in place does not
# move autograd's version counters.

class _Here:
    """The current device and stream: nothing to change."""

    def __enter__(self):
        pass

    def __exit__(self, *exc):
        pass


_HERE = _Here()


def _on(dev, stream, tensors):
    """Makes `dev`, and `stream` where one is given, current while a call allocates and launches."""
    if stream is None:
        return _HERE if dev.index == torch.cuda.current_device() else torch.cuda.device(dev)
    if stream.device != dev:
        raise ValueError("the stream belongs to another device than the tensors")
    if stream != torch.cuda.current_stream(dev):
        for t in tensors:  # (their memory may not be handed out again before the stream is done with them)
            if t is not None:
                t.record_stream(stream)
    return torch.cuda.stream(stream)


def _at(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _same(t, like: torch.Tensor, shape, name: str, dtype=None):
    """An optional input of a given shape, of like's device and (without dtype) type."""
    if t is None:
        return None
    if t.device != like.device:
        raise ValueError(f"{name} must live on the GPU of the other tensors")
    if t.dtype != (dtype or like.dtype):
        raise ValueError(f"{name} must be {dtype or like.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be of shape {list(shape)}, not {list(t.shape)}")
    return t


def _result(t, like: torch.Tensor, shape, name: str, dtype=None) -> torch.Tensor:
    """An output: the caller's, which must be contiguous, or a new one."""
    if t is None:
        if dtype is not None:
            return like.new_empty(shape, dtype=dtype)
        return torch.empty_like(like) if like.shape == shape else like.new_empty(shape)  # (the cheaper call; like is contiguous)
    if not _same(t, like, shape, name, dtype).is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _rows_of(x: torch.Tensor, name: str) -> Tuple[int, int, int]:
    if not x.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if x.dtype not in DTYPES:
        raise ValueError(f"{name} must be float32, bfloat16 or float16")
    if x.dim() != 2:
        raise ValueError(f"{name} must be [rows, channels]")
    return DTYPES[x.dtype], x.shape[0], x.shape[1]


def _rows_dev(rows_dev, like: torch.Tensor):
    if rows_dev is None:
        return None
    if rows_dev.device != like.device or rows_dev.dtype != torch.int64 or rows_dev.numel() < 1:
        raise ValueError("rows_dev must be an int64 tensor on the GPU of the rows")
    return rows_dev


def _activation(act: str) -> int:
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[act]


@functools.lru_cache(maxsize=4096)
def _need(device: int, query: str, *sizes) -> int:
    """Answer of a workspace query, which depends on its arguments and on the current device (`device`) alone."""
    L = load_library()
    r = int(getattr(L, query)(*sizes))
    if r == 0:
        raise ScnnError(-1, L.scnn_last_error().decode())
    return r


def _ask(query: str, dtype: torch.dtype, *sizes) -> int:
    if dtype not in DTYPES:
        raise ValueError("dtype must be float32, bfloat16 or float16")
    return _need.__wrapped__(-1, query, DTYPES[dtype], *sizes)


def _scratch(workspace, need: int, like: torch.Tensor) -> Optional[torch.Tensor]:
    if workspace is None:
        # (a call that needs the least amount uses none)
        return None if need <= 256 else like.new_empty(need, dtype=torch.uint8)
    if workspace.device != like.device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the GPU of the rows")
    return workspace


def _bytes(workspace) -> int:
    return 0 if workspace is None else workspace.numel()


def _current() -> int:
    """The current device's current stream."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _cont(t: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    return None if t is None else t.contiguous()


def linear_fwd_workspace(dtype: torch.dtype, rows: int, c_in: int, c_out: int) -> int:
    return _ask("linear_fwd_workspace", dtype, int(rows), int(c_in), int(c_out))


def linear_fwd(x, w, bias=None, *, act="none", residual=None, keep_pre=False, rows_dev=None, out=None, pre=None,
               workspace=None, stream=None):
    """out = act(x w + bias) + residual on rows x [rows, c_in], w [c_in, c_out]; act: "none", "relu", "gelu" or "silu".
    Returns out, or (out, pre) with keep_pre (or a tensor given as pre): pre = x w + bias is what linear_bwd needs."""
    L = load_library()
    dt, rows, c_in = _rows_of(x, "x")
    if w.dim() != 2 or w.shape[0] != c_in:
        raise ValueError("w must be [c_in, c_out]")
    c_out = w.shape[1]
    _same(w, x, (c_in, c_out), "w")
    _same(bias, x, (c_out,), "bias")
    _same(residual, x, (rows, c_out), "residual")
    code = _activation(act)
    rows_dev = _rows_dev(rows_dev, x)
    with _on(x.device, stream, (x, w, bias, residual, rows_dev, out, pre, workspace)):
        x, w, bias, residual = x.contiguous(), w.contiguous(), _cont(bias), _cont(residual)
        keep = keep_pre or pre is not None
        out = _result(out, x, (rows, c_out), "out")
        if keep:
            pre = _result(pre, x, (rows, c_out), "pre")
        workspace = _scratch(workspace, _need(x.device.index, "linear_fwd_workspace", dt, rows, c_in, c_out), x)
        _check(L, L.linear_fwd(dt, _at(x), rows, _at(rows_dev), c_in, _at(w), _at(bias), c_out, code, _at(residual),
                               _at(out), _at(pre), _at(workspace), _bytes(workspace), _current()))
    return (out, pre) if keep else out


def linear_bwd_workspace(dtype: torch.dtype, rows: int, c_in: int, c_out: int, act="none") -> int:
    return _ask("linear_bwd_workspace", dtype, int(rows), int(c_in), int(c_out), _activation(act))


def linear_bwd(x, w, g, *, act="none", pre=None, want=(True, True, True), rows_dev=None, out=None, workspace=None,
               stream=None):
    """Gradients of linear_fwd from g [rows, c_out], the gradient of its result (which is the residual's gradient too).
    pre: as linear_fwd gave it (not read with act "none").  Returns (dx, dw, dbias), None where `want` is False; `out`:
    tensors to put them in."""
    L = load_library()
    dt, rows, c_in = _rows_of(x, "x")
    if w.dim() != 2 or w.shape[0] != c_in:
        raise ValueError("w must be [c_in, c_out]")
    c_out = w.shape[1]
    _same(w, x, (c_in, c_out), "w")
    _same(g, x, (rows, c_out), "g")
    code = _activation(act)
    if code and pre is None:
        raise ValueError("the activation's gradient needs pre")
    pre = _same(pre, x, (rows, c_out), "pre") if code else None
    rows_dev = _rows_dev(rows_dev, x)
    dx, dw, dbias = out if out is not None else (None, None, None)
    with _on(x.device, stream, (x, w, g, pre, rows_dev, dx, dw, dbias, workspace)):
        x, w, g, pre = x.contiguous(), w.contiguous(), g.contiguous(), _cont(pre)
        dx = _result(dx, x, (rows, c_in), "dx") if want[0] else None
        dw = _result(dw, x, (c_in, c_out), "dw") if want[1] else None
        dbias = _result(dbias, x, (c_out,), "dbias") if want[2] else None
        workspace = _scratch(workspace, _need(x.device.index, "linear_bwd_workspace", dt, rows, c_in, c_out, code), x)
        _check(L, L.linear_bwd(dt, _at(x), rows, _at(rows_dev), c_in, _at(w), c_out, code, _at(pre), _at(g), _at(dx),
                               _at(dw), _at(dbias), _at(workspace), _bytes(workspace), _current()))
    return dx, dw, dbias


def layer_norm_fwd(x, gamma=None, beta=None, *, eps=1e-5, rows_dev=None, out=None, stream=None):
    """Layer norm over the channels of each row of x [rows, channels].  Returns (out, mean, rstd), the statistics fp32
    [rows], which layer_norm_bwd needs; `out`: three tensors to put them in."""
    L = load_library()
    dt, rows, ch = _rows_of(x, "x")
    _same(gamma, x, (ch,), "gamma")
    _same(beta, x, (ch,), "beta")
    rows_dev = _rows_dev(rows_dev, x)
    y, mean, rstd = out if out is not None else (None, None, None)
    with _on(x.device, stream, (x, gamma, beta, rows_dev, y, mean, rstd)):
        x, gamma, beta = x.contiguous(), _cont(gamma), _cont(beta)
        y = _result(y, x, (rows, ch), "out")
        mean = _result(mean, x, (rows,), "mean", torch.float32)
        rstd = _result(rstd, mean, (rows,), "rstd")
        _check(L, L.layer_norm_fwd(dt, _at(x), rows, _at(rows_dev), ch, _at(gamma), _at(beta), float(eps), _at(y),
                                   _at(mean), _at(rstd), _current()))
    return y, mean, rstd


def layer_norm_bwd_workspace(dtype: torch.dtype, rows: int, channels: int) -> int:
    return _ask("layer_norm_bwd_workspace", dtype, int(rows), int(channels))


def layer_norm_bwd(x, g, gamma, mean, rstd, *, want=(True, True, True), rows_dev=None, out=None, workspace=None,
                   stream=None):
    """Gradients of layer_norm_fwd from g [rows, channels], the gradient of its result; gamma may be None, mean and rstd as
    layer_norm_fwd gave them.  Returns (dx, dgamma, dbeta), None where `want` is False; `out`: tensors to put them in."""
    L = load_library()
    dt, rows, ch = _rows_of(x, "x")
    _same(g, x, (rows, ch), "g")
    _same(gamma, x, (ch,), "gamma")
    _same(mean, x, (rows,), "mean", torch.float32)
    _same(rstd, x, (rows,), "rstd", torch.float32)
    rows_dev = _rows_dev(rows_dev, x)
    dx, dgamma, dbeta = out if out is not None else (None, None, None)
    with _on(x.device, stream, (x, g, gamma, mean, rstd, rows_dev, dx, dgamma, dbeta, workspace)):
        x, g, gamma, mean, rstd = x.contiguous(), g.contiguous(), _cont(gamma), mean.contiguous(), rstd.contiguous()
        dx = _result(dx, x, (rows, ch), "dx") if want[0] else None
        dgamma = _result(dgamma, x, (ch,), "dgamma") if want[1] else None
        dbeta = _result(dbeta, x, (ch,), "dbeta") if want[2] else None
        workspace = _scratch(workspace, _need(x.device.index, "layer_norm_bwd_workspace", dt, rows, ch), x)
        _check(L, L.layer_norm_bwd(dt, _at(x), _at(g), rows, _at(rows_dev), ch, _at(gamma), _at(mean), _at(rstd),
                                   _at(dx), _at(dgamma), _at(dbeta), _at(workspace), _bytes(workspace), _current()))
    return dx, dgamma, dbeta


def _dense(t: torch.Tensor) -> bool:
    """The tensor's entries fill one stretch of memory, in any order of its axes."""
    if t.is_contiguous():
        return True
    step = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
        if stride != step:
            return False
        step *= size
    return True


def _grad_clip(grads, max_norm, outs, workspace, stream):
    """outs: None (the norm alone), the list of gradients itself, or other tensors."""
    L = load_library()
    n = len(grads)
    if n == 0:
        raise ValueError("no gradients")
    like = grads[0]
    where = like.get_device()
    dtypes = [t.dtype for t in grads]
    types = [DTYPES.get(d, -1) for d in dtypes]
    if where < 0 or any([t.get_device() != where for t in grads]):
        raise ValueError("the gradients must live on one GPU")
    if -1 in types:
        raise ValueError("gradients must be float32, bfloat16 or float16")
    plain = all([t.is_contiguous() for t in grads])
    if not plain and not all([_dense(t) for t in grads]):
        raise ValueError("a gradient must fill one stretch of memory")
    if outs is not None and outs is not grads:
        if len(outs) != n:
            raise ValueError("outs must hold a tensor for every gradient")
        alike = all([o.get_device() == where for o in outs]) and [o.dtype for o in outs] == dtypes
        alike = alike and [o.shape for o in outs] == [t.shape for t in grads]
        if not alike or not (all([o.is_contiguous() for o in outs]) if plain else
                             [o.stride() for o in outs] == [t.stride() for t in grads]):
            raise ValueError("an output must be like its gradient (device, type, shape and strides)")
    sizes = [t.numel() for t in grads]
    counts = (ctypes.c_int64 * n)(*sizes)
    src = (ctypes.c_void_p * n)(*[t.data_ptr() for t in grads])
    dst = src if outs is grads else None if outs is None else (ctypes.c_void_p * n)(*[t.data_ptr() for t in outs])
    dev = like.device
    with _on(dev, stream, None if stream is None else (*grads, *(outs or ()), workspace)):
        result = like.new_empty(2, dtype=torch.float64)
        workspace = _scratch(workspace, int(L.grad_clip_workspace(n, counts)), like)
        _check(L, L.grad_clip(n, src, dst, counts, (ctypes.c_int * n)(*types), float(max_norm), _at(result), _at(workspace),
                              _bytes(workspace), _current()))
    return result


def clip_grad_norm(grads, max_norm, *, outs=None, workspace=None, stream=None):
    """Scales all gradients by min(1, max_norm / (norm + 1e-6)), norm = their global 2-norm: in place, or into `outs`.
    Returns double[2] = {norm, scale} on the device."""
    grads = list(grads)
    return _grad_clip(grads, max_norm, grads if outs is None else list(outs), workspace, stream)


def grad_norm(grads, *, workspace=None, stream=None):
    """Global 2-norm of a list of gradients: a double on the device."""
    return _grad_clip(list(grads), float("inf"), None, workspace, stream)[0]


def grad_clip_workspace(counts) -> int:
    """Bytes of workspace of clip_grad_norm and grad_norm for tensors of these numbers of entries."""
    L = load_library()
    r = int(L.grad_clip_workspace(len(counts), (ctypes.c_int64 * len(counts))(*[int(c) for c in counts])))
    if r == 0:
        raise ScnnError(-1, L.scnn_last_error().decode())
    return r


def validate_rows(extent, batch, coords, stream=None) -> None:
    """Raises ScnnError if coords are out of the grid (-1) or not strictly ascending (-4).  Synchronises."""
    L = load_library()
    coords = _dev(coords, torch.int32, "coords")
    ws = torch.empty(256, dtype=torch.uint8, device=coords.device)
    rc = L.scnn_validate_rows(len(extent), _i32arr(extent), int(batch), _ptr(coords), coords.shape[0], _ptr(ws), 256,
                              _stream(stream))
    _check(L, rc)


def profile_enable(on) -> None:
    """Per-stage HIP-event timing of sparse_conv_fwd calls made from this thread: False / 0 = off, True / 1 = every
    stage, 2 = only the convolution stage (two events per call), 3 = the same on every fourth call."""
    _check(load_library(), load_library().scnn_profile_enable(int(on)))


def profile_collect():
    """Waits for the recorded calls; returns ({stage name: total ms}, number of calls)."""
    L = load_library()
    n = L.scnn_profile_stage_count()
    ms = (ctypes.c_double * n)()
    calls = ctypes.c_int64(0)
    _check(L, L.scnn_profile_collect(ms, ctypes.byref(calls)))
    return {L.scnn_profile_stage_name(i).decode(): float(ms[i]) for i in range(n)}, int(calls.value)


def set_conv_path(path: int) -> None:
    """0 = choose the convolution kernel by shape and size, 1 = always the vector kernels, 2 = the fp32 quad kernel where
    it takes the shape, else the pair-list kernel, 3 = the pair-list matrix-core kernel where it takes the shape, 5 = the
    split-operand kernel where it takes the shape."""
    L = load_library()
    _check(L, L.scnn_set_conv_path(int(path)))


def last_conv_kernel() -> str:
    """Convolution kernel launched by this thread's last sparse_conv_fwd call."""
    return load_library().scnn_last_conv_kernel().decode()


def calibration_copy(dst: torch.Tensor, src: torch.Tensor, stream=None) -> None:
    """Plain streaming copy of src into dst (same byte size, a multiple of 16)."""
    L = load_library()
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("size mismatch")
    _check(L, L.scnn_calibration_copy(_ptr(dst), _ptr(src), nbytes, _stream(stream)))
