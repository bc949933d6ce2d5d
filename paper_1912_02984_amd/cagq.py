"""Python binding of the gfx950 CAGQ library (``libcagq.so``).

Argument marshalling only: every step of the path runs in the library's HIP
kernels. Tensors are torch CUDA (HIP) tensors; the library enqueues on the
current torch stream. The names mirror the C ABI in ``include/cagq.h``:
``build_grid``, ``sample_centers``, ``query_context``, ``get_device_status``;
and, on the features of the grouped points, ``group_attention``,
``point_lists``, ``relative_bias`` and their gradients.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Dict, Optional, Sequence

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcagq.so")

OK = 0
ERR_INVALID_ARG = -1
ERR_GRID_TOO_LARGE = -2
ERR_WORKSPACE_TOO_SMALL = -3
ERR_NONFINITE_INPUT = -4
ERR_CAPACITY = -5
ERR_HIP = -6
ERR_CENTER_NOT_OCCUPIED = -7

SAMPLE = {"rvs": 0, "cas": 1, "cas_swap": 2}
QUERY = {"cube": 0, "knn": 1, "knn_ring": 2}
MAX_K = 128
MAX_NV = 64
MAX_RADIUS = 3


class GridDesc(C.Structure):
    _fields_ = [("origin", C.c_float * 3), ("voxel_size", C.c_float * 3),
                ("dims", C.c_int32 * 3), ("n_v", C.c_int32), ("radius", C.c_int32)]


class LayoutC(C.Structure):
    _fields_ = [("total_bytes", C.c_size_t), ("nvox", C.c_size_t), ("vox_lin", C.c_size_t),
                ("vox_count", C.c_size_t), ("vox_off", C.c_size_t), ("pt_list", C.c_size_t)]


class GridC(C.Structure):
    _fields_ = [("B", C.c_int32), ("N", C.c_int32), ("desc", GridDesc), ("points", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class GroupsC(C.Structure):
    _fields_ = [("B", C.c_int32), ("N", C.c_int32), ("M", C.c_int32), ("K", C.c_int32), ("idx", C.c_void_p),
                ("n_valid", C.c_void_p), ("off", C.c_void_p), ("idx_len", C.c_int64), ("points", C.c_void_p),
                ("centers", C.c_void_p)]


class BiasC(C.Structure):
    _fields_ = [("table", C.c_void_p), ("edges", C.c_void_p), ("slope", C.c_void_p), ("buckets", C.c_int32)]


class AttnC(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("H", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("scale", C.c_float),
                ("cap", C.c_float), ("q_row", C.c_int64), ("k_row", C.c_int64), ("v_row", C.c_int64)]


class CagqError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {status_string(code)} ({code})")
        self.code = code


_lib = None


def lib() -> C.CDLL:
    """Load ``libcagq.so``; raises if the library has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_1912_02984_amd.build")
        L = C.CDLL(LIB_PATH)
        P = C.c_void_p
        F3, I3 = C.c_float * 3, C.c_int32 * 3
        L.cagq_desc_from_voxel_size.argtypes = [C.POINTER(F3), C.POINTER(F3), C.POINTER(F3), C.c_int32,
                                                C.c_int32, C.POINTER(GridDesc)]
        L.cagq_desc_from_dims.argtypes = [C.POINTER(F3), C.POINTER(F3), C.POINTER(I3), C.c_int32, C.c_int32,
                                          C.POINTER(GridDesc)]
        L.cagq_workspace_layout.argtypes = [C.c_int32, C.c_int32, C.POINTER(GridDesc), C.POINTER(LayoutC)]
        L.cagq_build_grid_static.argtypes = [P, C.c_int32, C.c_int32, C.POINTER(GridDesc), P, C.POINTER(GridC)]
        L.cagq_build_grid.argtypes = [P, C.c_int32, C.c_int32, C.POINTER(GridDesc), P, C.c_size_t, P,
                                      C.POINTER(GridC)]
        L.cagq_sample_centers.argtypes = [C.POINTER(GridC), C.c_int32, C.c_int32, C.c_uint64, C.c_uint32,
                                          P, P, P]
        L.cagq_query_context.argtypes = [C.POINTER(GridC), P, P, C.c_int32, C.c_int32, C.c_int32,
                                         C.c_uint64, P, P, P, P, P, P, P]
        L.cagq_query_points.argtypes = [C.POINTER(GridC), P, C.c_int32, C.c_int32, C.c_int32, C.c_uint64,
                                        P, P, P, P, P, P]
        L.cagq_context_offsets.argtypes = [C.POINTER(GridC), P, C.c_int32, P, P]
        L.cagq_context_list.argtypes = [C.POINTER(GridC), P, C.c_int32, P, P, C.c_int64, P]
        L.cagq_sample_points.argtypes = [P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_uint64, P, P]
        L.cagq_ball_query.argtypes = [P, C.c_int32, C.c_int32, P, C.c_int32, C.c_int32, C.c_float, P, P, P]
        L.cagq_coverage.argtypes = [C.POINTER(GridC), P, P, C.c_int32, C.c_int32, P, P]
        G, A, Bi, SZ = C.POINTER(GroupsC), C.POINTER(AttnC), C.POINTER(BiasC), C.POINTER(C.c_size_t)
        L.cagq_group_attention_workspace.argtypes = [G, A, Bi, C.c_int32, SZ]
        L.cagq_group_attention.argtypes = [G, A, Bi, P, P, P, P, P, P, C.c_size_t, P]
        L.cagq_point_lists_workspace.argtypes = [G, SZ]
        L.cagq_point_lists.argtypes = [G, P, P, C.c_int64, P, C.c_size_t, P]
        L.cagq_group_attention_backward.argtypes = [G, A, Bi, P, P, C.c_int64, P, P, P, P, P, P, P, P, P, P, P,
                                                    C.c_size_t, P]
        L.cagq_relative_bias.argtypes = [G, Bi, C.c_int32, C.c_int32, P, P]
        L.cagq_relative_bias_workspace.argtypes = [G, Bi, C.c_int32, SZ]
        L.cagq_relative_bias_backward.argtypes = [G, Bi, C.c_int32, C.c_int32, P, P, P, P, C.c_size_t, P]
        L.cagq_get_device_status.argtypes = [C.POINTER(GridC), P]
        L.cagq_status_string.argtypes = [C.c_int]
        L.cagq_status_string.restype = C.c_char_p
        for f in ("cagq_desc_from_voxel_size", "cagq_desc_from_dims", "cagq_workspace_layout", "cagq_build_grid", "cagq_build_grid_static", "cagq_sample_centers",
                  "cagq_query_context", "cagq_query_points", "cagq_context_offsets", "cagq_context_list",
                  "cagq_sample_points", "cagq_ball_query", "cagq_coverage", "cagq_get_device_status",
                  "cagq_group_attention_workspace", "cagq_group_attention", "cagq_point_lists_workspace",
                  "cagq_point_lists", "cagq_group_attention_backward", "cagq_relative_bias",
                  "cagq_relative_bias_workspace", "cagq_relative_bias_backward"):
            getattr(L, f).restype = C.c_int
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().cagq_status_string(int(code)).decode()


def _check(rc: int, what: str):
    if rc != OK:
        raise CagqError(rc, what)


def make_desc(origin: Sequence[float], voxel_size: Sequence[float], dims: Sequence[int],
              n_v: int, radius: int = 1) -> GridDesc:
    d = GridDesc()
    for a in range(3):
        d.origin[a] = float(origin[a])
        d.voxel_size[a] = float(voxel_size[a])
        d.dims[a] = int(dims[a])
    d.n_v = int(n_v)
    d.radius = int(radius)
    return d


def desc_from_voxel_size(lo: Sequence[float], hi: Sequence[float], voxel_size: Sequence[float], n_v: int,
                         radius: int = 1) -> GridDesc:
    """GridDesc of the smallest grid at origin ``lo`` with the given voxel
    size whose voxels hold every point of the box [lo, hi] without clamping."""
    F3 = C.c_float * 3
    d = GridDesc()
    _check(lib().cagq_desc_from_voxel_size(C.byref(F3(*lo)), C.byref(F3(*hi)), C.byref(F3(*voxel_size)),
                                           int(n_v), int(radius), C.byref(d)), "cagq_desc_from_voxel_size")
    return d


def desc_from_dims(lo: Sequence[float], hi: Sequence[float], dims: Sequence[int], n_v: int,
                   radius: int = 1) -> GridDesc:
    """GridDesc at origin ``lo`` with ``dims`` voxels per axis spanning [lo, hi]."""
    F3, I3 = C.c_float * 3, C.c_int32 * 3
    d = GridDesc()
    _check(lib().cagq_desc_from_dims(C.byref(F3(*lo)), C.byref(F3(*hi)), C.byref(I3(*dims)),
                                     int(n_v), int(radius), C.byref(d)), "cagq_desc_from_dims")
    return d


def desc_from_spec(spec) -> GridDesc:
    """GridDesc from an object with origin, voxel_size, dims, n_v, radius."""
    return make_desc(spec.origin, spec.voxel_size, spec.dims, spec.n_v, spec.radius)


def workspace_layout(B: int, N: int, desc: GridDesc) -> LayoutC:
    out = LayoutC()
    _check(lib().cagq_workspace_layout(B, N, C.byref(desc), C.byref(out)), "cagq_workspace_layout")
    return out


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_cur_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_ptr(stream: Optional[torch.cuda.Stream] = None):
    """The HIP stream to launch on: ``stream``, else torch's current stream
    (read as a raw handle: building a Stream object per call costs ~3 us)."""
    if stream is not None:
        return C.c_void_p(stream.cuda_stream)
    if _raw_stream is not None and _cur_device is not None:
        return C.c_void_p(_raw_stream(_cur_device()))
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _need(t: torch.Tensor, dtype, shape, name: str):
    if not t.is_cuda or t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} {tuple(shape)} on the GPU, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


STATIC_WORKSPACE_BYTES = 64 << 20  # CAGQ_STATIC_WORKSPACE_BYTES


@dataclass
class Grid:
    """A built grid: the C record plus the tensors it borrows (workspace is
    None for a grid in the library's own array, cagq_build_grid_static)."""
    rec: GridC
    points: torch.Tensor
    workspace: Optional[torch.Tensor]
    layout: LayoutC

    @property
    def B(self) -> int:
        return self.rec.B

    @property
    def N(self) -> int:
        return self.rec.N

    def _view(self, off: int, count: int, dtype, ws: torch.Tensor) -> torch.Tensor:
        nbytes = count * torch.tensor([], dtype=dtype).element_size()
        return ws[off:off + nbytes].view(dtype)

    def _exposed(self) -> torch.Tensor:
        """The workspace bytes up to the end of the exposed arrays: the
        tensor itself, or a copy out of the library's array."""
        if self.workspace is not None:
            return self.workspace
        L = self.layout
        n = L.pt_list + 4 * self.B * self.N
        out = torch.empty(n, dtype=torch.uint8, device=self.points.device)
        torch.cuda.current_stream().synchronize()
        _check(0 if _hip().hipMemcpy(C.c_void_p(out.data_ptr()), C.c_void_p(self.rec.workspace), C.c_size_t(n),
                                     3) == 0 else ERR_HIP, "hipMemcpy")  # 3: device to device
        return out

    def table(self) -> Dict[str, torch.Tensor]:
        """Views of the occupied-voxel table inside the workspace (uint32 as int32)."""
        B, N, L = self.B, self.N, self.layout
        ws = self._exposed()
        return dict(
            nvox=self._view(L.nvox, B, torch.int32, ws),
            vox_lin=self._view(L.vox_lin, B * N, torch.int32, ws).view(B, N),
            vox_count=self._view(L.vox_count, B * N, torch.int32, ws).view(B, N),
            vox_off=self._view(L.vox_off, B * (N + 1), torch.int32, ws).view(B, N + 1),
            pt_list=self._view(L.pt_list, B * N, torch.int32, ws).view(B, N),
        )


_hip_lib = None


def _hip() -> C.CDLL:
    """The HIP runtime torch has loaded (for copies out of the library's own array)."""
    global _hip_lib
    if _hip_lib is None:
        _hip_lib = C.CDLL("libamdhip64.so")
        _hip_lib.hipMemcpy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]
        _hip_lib.hipMemcpy.restype = C.c_int
    return _hip_lib


def build_grid(points: torch.Tensor, desc: GridDesc, workspace: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> Grid:
    """Voxelize and index a batch ``points`` float32 [B, N, 3] (cagq_build_grid)."""
    if points.dim() != 3 or points.shape[2] != 3:
        raise ValueError("points must be [B, N, 3]")
    B, N = int(points.shape[0]), int(points.shape[1])
    _need(points, torch.float32, (B, N, 3), "points")
    lay = workspace_layout(B, N, desc)
    if workspace is None:
        workspace = torch.empty(lay.total_bytes, dtype=torch.uint8, device=points.device)
    rec = GridC()
    _check(lib().cagq_build_grid(_ptr(points), B, N, C.byref(desc), _ptr(workspace), workspace.numel(),
                                 _stream_ptr(stream), C.byref(rec)), "cagq_build_grid")
    return Grid(rec, points, workspace, lay)


def build_grid_static(points: torch.Tensor, desc: GridDesc, stream: Optional[torch.cuda.Stream] = None) -> Grid:
    """cagq_build_grid into the library's own array (cagq_build_grid_static):
    no workspace, no allocation by the call. A later static build on the same
    GPU overwrites the grid."""
    if points.dim() != 3 or points.shape[2] != 3:
        raise ValueError("points must be [B, N, 3]")
    B, N = int(points.shape[0]), int(points.shape[1])
    _need(points, torch.float32, (B, N, 3), "points")
    lay = workspace_layout(B, N, desc)
    rec = GridC()
    _check(lib().cagq_build_grid_static(_ptr(points), B, N, C.byref(desc), _stream_ptr(stream), C.byref(rec)),
           "cagq_build_grid_static")
    return Grid(rec, points, None, lay)


def sample_centers(grid: Grid, M: int, mode: str, seed: int, beta_q16: int = 0,
                   center_lin: Optional[torch.Tensor] = None, m_valid: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None):
    """M center voxels per cloud by RVS, CAS (greedy) or CAS with the paper's
    challenger / incumbent swaps (cagq_sample_centers; mode "rvs", "cas" or
    "cas_swap")."""
    dev = grid.points.device
    if center_lin is None:
        center_lin = torch.empty((grid.B, M), dtype=torch.int32, device=dev)
    if m_valid is None:
        m_valid = torch.empty((grid.B,), dtype=torch.int32, device=dev)
    _need(center_lin, torch.int32, (grid.B, M), "center_lin")
    _need(m_valid, torch.int32, (grid.B,), "m_valid")
    _check(lib().cagq_sample_centers(C.byref(grid.rec), M, SAMPLE[mode], C.c_uint64(seed & (2**64 - 1)),
                                     C.c_uint32(beta_q16), _ptr(center_lin), _ptr(m_valid),
                                     _stream_ptr(stream)), "cagq_sample_centers")
    return center_lin, m_valid


def alloc_query_outputs(B: int, M: int, K: int, device, want_xyz: bool = True,
                        want_ctx: bool = True) -> Dict[str, torch.Tensor]:
    return dict(
        node_idx=torch.empty((B, M, K), dtype=torch.int32, device=device),
        node_xyz=torch.empty((B, M, K, 3), dtype=torch.float32, device=device) if want_xyz else None,
        n_valid=torch.empty((B, M), dtype=torch.int32, device=device),
        center_xyz=torch.empty((B, M, 3), dtype=torch.float32, device=device),
        center_w=torch.empty((B, M), dtype=torch.int32, device=device),
        ctx_count=torch.empty((B, M), dtype=torch.int32, device=device) if want_ctx else None,
    )


def query_context(grid: Grid, center_lin: torch.Tensor, K: int, mode: str, seed: int,
                  weights: Optional[torch.Tensor] = None, out: Optional[Dict[str, torch.Tensor]] = None,
                  want_xyz: bool = True, want_ctx: bool = True,
                  stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """K node points and the group center per center voxel (cagq_query_context).

    ``weights`` int32/uint32-valued [B, N] or None (all 1). ``center_w`` holds
    uint32 values in an int32 tensor.
    """
    B, M = int(center_lin.shape[0]), int(center_lin.shape[1])
    _need(center_lin, torch.int32, (B, M), "center_lin")
    if weights is not None:
        _need(weights, torch.int32, (grid.B, grid.N), "weights")
    if out is None:
        out = alloc_query_outputs(B, M, K, grid.points.device, want_xyz, want_ctx)
    _check(lib().cagq_query_context(
        C.byref(grid.rec), _ptr(weights), _ptr(center_lin), M, K, QUERY[mode], C.c_uint64(seed & (2**64 - 1)),
        _ptr(out["node_idx"]), _ptr(out.get("node_xyz")), _ptr(out["n_valid"]), _ptr(out["center_xyz"]),
        _ptr(out["center_w"]), _ptr(out.get("ctx_count")), _stream_ptr(stream)), "cagq_query_context")
    return out


def query_points(grid: Grid, centers: torch.Tensor, K: int, mode: str, seed: int,
                 out: Optional[Dict[str, torch.Tensor]] = None, want_xyz: bool = True,
                 stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """Upsampling query: K node points around given center points [B, M, 3]
    (cagq_query_points). Also returns ctx_count and each center's voxel lin."""
    B, M = int(centers.shape[0]), int(centers.shape[1])
    _need(centers, torch.float32, (B, M, 3), "centers")
    dev = grid.points.device
    if out is None:
        out = dict(
            node_idx=torch.empty((B, M, K), dtype=torch.int32, device=dev),
            node_xyz=torch.empty((B, M, K, 3), dtype=torch.float32, device=dev) if want_xyz else None,
            n_valid=torch.empty((B, M), dtype=torch.int32, device=dev),
            ctx_count=torch.empty((B, M), dtype=torch.int32, device=dev),
            center_lin=torch.empty((B, M), dtype=torch.int32, device=dev),
        )
    _check(lib().cagq_query_points(
        C.byref(grid.rec), _ptr(centers), M, K, QUERY[mode], C.c_uint64(seed & (2**64 - 1)),
        _ptr(out["node_idx"]), _ptr(out.get("node_xyz")), _ptr(out["n_valid"]), _ptr(out.get("ctx_count")),
        _ptr(out.get("center_lin")), _stream_ptr(stream)), "cagq_query_points")
    return out


def context_offsets(grid: Grid, center_lin: torch.Tensor, out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """CSR offsets [B*M + 1] (int64) of the centers' context lists."""
    B, M = int(center_lin.shape[0]), int(center_lin.shape[1])
    _need(center_lin, torch.int32, (B, M), "center_lin")
    if out is None:
        out = torch.empty(B * M + 1, dtype=torch.int64, device=grid.points.device)
    _need(out, torch.int64, (B * M + 1,), "ctx_off")
    _check(lib().cagq_context_offsets(C.byref(grid.rec), _ptr(center_lin), M, _ptr(out), _stream_ptr(stream)),
           "cagq_context_offsets")
    return out


def context_list(grid: Grid, center_lin: torch.Tensor, ctx_off: torch.Tensor,
                 out: Optional[torch.Tensor] = None, capacity: Optional[int] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The context lists (int32 point indices) laid out by ``ctx_off``. Without
    ``out`` the total is read back from ``ctx_off`` to size it."""
    B, M = int(center_lin.shape[0]), int(center_lin.shape[1])
    _need(center_lin, torch.int32, (B, M), "center_lin")
    _need(ctx_off, torch.int64, (B * M + 1,), "ctx_off")
    if out is None:
        total = int(ctx_off[-1].item())
        out = torch.empty(max(total, 1), dtype=torch.int32, device=grid.points.device)
        capacity = total
    if capacity is None:
        capacity = int(out.numel())
    _check(lib().cagq_context_list(C.byref(grid.rec), _ptr(center_lin), M, _ptr(ctx_off), _ptr(out),
                                   int(capacity), _stream_ptr(stream)), "cagq_context_list")
    return out


POINTS = {"rps": 0, "fps": 1}


def sample_points(points: torch.Tensor, M: int, mode: str, seed: int = 0, out: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Random / Farthest Point Sampling (comparison methods): [B, M] point indices."""
    B, N = int(points.shape[0]), int(points.shape[1])
    _need(points, torch.float32, (B, N, 3), "points")
    if out is None:
        out = torch.empty((B, M), dtype=torch.int32, device=points.device)
    _check(lib().cagq_sample_points(_ptr(points), B, N, M, POINTS[mode], C.c_uint64(seed & (2**64 - 1)), _ptr(out),
                                    _stream_ptr(stream)), "cagq_sample_points")
    return out


def ball_query(points: torch.Tensor, center_idx: torch.Tensor, K: int, radius2: float,
               out: Optional[Dict[str, torch.Tensor]] = None,
               stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """Ball Query (comparison method): the first K points within the radius."""
    B, N = int(points.shape[0]), int(points.shape[1])
    M = int(center_idx.shape[1])
    _need(points, torch.float32, (B, N, 3), "points")
    _need(center_idx, torch.int32, (B, M), "center_idx")
    if out is None:
        out = dict(node_idx=torch.empty((B, M, K), dtype=torch.int32, device=points.device),
                   n_valid=torch.empty((B, M), dtype=torch.int32, device=points.device))
    _check(lib().cagq_ball_query(_ptr(points), B, N, _ptr(center_idx), M, K, C.c_float(radius2),
                                 _ptr(out["node_idx"]), _ptr(out["n_valid"]), _stream_ptr(stream)),
           "cagq_ball_query")
    return out


def coverage(grid: Grid, node_idx: torch.Tensor, n_valid: torch.Tensor, out: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Occupied voxels [B] holding a valid node point (divide by nvox for the metric)."""
    B, M, K = (int(x) for x in node_idx.shape)
    _need(node_idx, torch.int32, (B, M, K), "node_idx")
    _need(n_valid, torch.int32, (B, M), "n_valid")
    if out is None:
        out = torch.empty(B, dtype=torch.int32, device=node_idx.device)
    _check(lib().cagq_coverage(C.byref(grid.rec), _ptr(node_idx), _ptr(n_valid), M, K, _ptr(out),
                               _stream_ptr(stream)), "cagq_coverage")
    return out


# ---------------------------------------------------------------- operators on point features

FEATURES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}  # CAGQ_F32, CAGQ_BF16, CAGQ_F16
MAX_BUCKETS = 64
MAX_HEADS = 128
MAX_HEAD_DIM = 256


_F32, _I32, _I64, _U8 = torch.float32, torch.int32, torch.int64, torch.uint8


def _on(t: torch.Tensor, dtype, shape, name: str, dev):
    """A contiguous tensor on ``dev``."""
    if t.dtype is not dtype or t.shape != shape or t.device != dev or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} {tuple(shape)} on {dev}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def _empty(like: torch.Tensor, shape, dtype, stream):
    """A tensor whose memory is handed on in the order of the stream it is used on."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _empty_as(like: torch.Tensor, stream):
    """The same for a dense tensor of the shape and type of ``like``."""
    if stream is None and like.is_contiguous():
        return torch.empty_like(like)
    return _empty(like, like.shape, like.dtype, stream)


def _handle(stream: Optional[torch.cuda.Stream], groups) -> int:
    """The HIP stream to launch on; it and the groups have to be on the current device."""
    cur = _cur_device() if _cur_device is not None else torch.cuda.current_device()
    if cur != groups.index:
        raise ValueError(f"groups on {groups.device}, but the current device is cuda:{cur}")
    if stream is None:
        return _raw_stream(cur) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream
    if stream.device_index != cur:
        raise ValueError(f"stream on cuda:{stream.device_index}, but the current device is cuda:{cur}")
    return stream.cuda_stream


def _scratch(workspace: Optional[torch.Tensor], size, args, like: torch.Tensor, stream, what: str):
    """Address and bytes of the workspace given, or of one as large as ``size(*args, pointer)`` says, and its tensor."""
    if workspace is None:
        need = C.c_size_t()
        rc = size(*args, C.byref(need))
        if rc:
            raise CagqError(rc, what)
        if not need.value:
            return None, 0, None
        workspace = _empty(like, need.value, _U8, stream)
    elif workspace.dtype is not _U8 or workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError(f"workspace: expected contiguous torch.uint8 on {like.device}")
    return workspace.data_ptr(), workspace.numel(), workspace


class Groups:
    """Groups of points: what ``query_context``, ``query_points``, ``ball_query`` or ``context_list`` found for
    the ``centers`` [B, M, 3] among the ``points`` [B, N, 3] (float32).

    Fixed groups: ``idx`` int32 [B, M, K], of which the first ``n_valid`` int32 [B, M] slots count (all K where it
    is None). Ragged groups: ``off`` int64 [B*M + 1] and ``idx`` int32 [entries]. An index outside [0, N) is a
    masked slot. The record holds the tensors' addresses: they must keep their storage as long as it is used."""
    __slots__ = ("rec", "idx", "points", "centers", "n_valid", "off", "B", "N", "M", "K", "device", "index")

    def __init__(self, idx: torch.Tensor, points: torch.Tensor, centers: torch.Tensor,
                 n_valid: Optional[torch.Tensor] = None, off: Optional[torch.Tensor] = None):
        dev = points.device
        cur = _cur_device() if _cur_device is not None else torch.cuda.current_device()
        if dev.type != "cuda" or dev.index != cur:
            raise ValueError(f"points on {dev}, but the current device is cuda:{cur}")
        if points.dim() != 3 or centers.dim() != 3:
            raise ValueError("points must be [B, N, 3] and centers [B, M, 3]")
        B, N, _ = points.shape
        M = centers.shape[1]
        _on(points, _F32, (B, N, 3), "points", dev)
        _on(centers, _F32, (B, M, 3), "centers", dev)
        K, nv, of, entries = 0, None, None, 0
        if off is None:
            if idx.dim() != 3 or idx.shape[2] < 1:
                raise ValueError("idx must be [B, M, K], or off be given")
            K = idx.shape[2]
            _on(idx, _I32, (B, M, K), "idx", dev)
            if n_valid is not None:
                _on(n_valid, _I32, (B, M), "n_valid", dev)
                nv = n_valid.data_ptr()
        else:
            if n_valid is not None or idx.dim() != 1:
                raise ValueError("ragged groups have idx [entries] and no n_valid")
            entries = idx.shape[0]
            _on(idx, _I32, (entries,), "idx", dev)
            _on(off, _I64, (B * M + 1,), "off", dev)
            of = off.data_ptr()
        self.idx, self.points, self.centers, self.n_valid, self.off = idx, points, centers, n_valid, off
        self.B, self.N, self.M, self.K, self.device, self.index = B, N, M, K, dev, cur
        self.rec = GroupsC(B, N, M, K, idx.data_ptr(), nv, of, entries, points.data_ptr(), centers.data_ptr())

    @property
    def slots(self) -> int:
        return self.idx.numel()


class RelativeBias:
    """Relative position bias of H heads: ``table`` [3, buckets, H] read by the buckets that the ascending
    ``edges`` [3, buckets - 1] cut each axis into, and ``slope`` [H] times the distance (float32; either may be
    None). What is learned may be given other storage (``table.data = ...``, a module's ``.to``): each call reads
    what ``table`` and ``slope`` hold by then, after the checks made here. ``edges`` must keep theirs."""
    __slots__ = ("rec", "table", "edges", "slope", "H", "device", "table_at", "slope_at")

    def __init__(self, table: Optional[torch.Tensor] = None, edges: Optional[torch.Tensor] = None,
                 slope: Optional[torch.Tensor] = None):
        self.table, self.edges, self.slope = table, edges, slope
        self._make()

    def _make(self):
        table, edges, slope = self.table, self.edges, self.slope
        some = table if table is not None else slope
        if some is None or not some.is_cuda:
            raise ValueError("a bias needs a table or a slope, on the GPU")
        dev, nb, H = some.device, 0, some.shape[-1] if some.dim() else 0
        tp = ep = sp = None
        if table is not None:
            nb = table.shape[1] if table.dim() == 3 else 0
            if not 1 <= nb <= MAX_BUCKETS:
                raise ValueError(f"table must be [3, buckets, H] with 1 to {MAX_BUCKETS} buckets")
            _on(table, _F32, (3, nb, H), "table", dev)
            tp = table.data_ptr()
            if edges is None and nb > 1:
                raise ValueError("a table needs edges [3, buckets - 1]")
        if edges is not None:
            _on(edges, _F32, (3, max(0, nb - 1)), "edges", dev)
            ep = edges.data_ptr()
        if slope is not None:
            _on(slope, _F32, (H,), "slope", dev)
            sp = slope.data_ptr()
        self.H, self.device, self.table_at, self.slope_at = H, dev, tp, sp
        self.rec = BiasC(tp, ep, sp, nb)

    def ref(self):
        """The C record, by reference."""
        t, s = self.table, self.slope
        if (t is not None and t.data_ptr() != self.table_at) or (s is not None and s.data_ptr() != self.slope_at):
            self._make()
        return C.byref(self.rec)


def _row(t: torch.Tensor, name: str) -> int:
    """Elements from one row of ``t`` [B, n, heads, D] to the next; its heads and channels are contiguous, its
    rows evenly spaced (a part of a larger projection, say)."""
    B, n, h, d = t.shape
    if t.is_contiguous():
        return h * d
    sb, sn, sh, sd = t.stride()
    row = sn if n > 1 else sb if B > 1 else h * d
    if (d > 1 and sd != 1) or (h > 1 and sh != d) or (B > 1 and sb != n * row) or row < h * d:
        raise ValueError(f"{name}: rows must be evenly spaced, their heads and channels contiguous, "
                         f"got strides {tuple(t.stride())} for {tuple(t.shape)}")
    return row


def _attn(groups: Groups, q, k, v, bias: Optional[RelativeBias], scale, cap):
    dev, dtype = groups.device, q.dtype
    code = FEATURES.get(dtype)
    if code is None:
        raise ValueError(f"q: features are {', '.join(str(x) for x in FEATURES)}, got {dtype}")
    for t, n, name in ((q, groups.M, "q"), (k, groups.N, "k"), (v, groups.N, "v")):
        if t.dim() != 4 or t.dtype is not dtype or t.device != dev or t.shape[:2] != (groups.B, n):
            raise ValueError(f"{name}: expected {dtype} [{groups.B}, {n}, heads, D] on {dev}, "
                             f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    _, _, H, D = q.shape
    _, _, Hkv, Dk = k.shape
    if v.shape != k.shape or Dk != D or D < 1 or Hkv < 1 or H % Hkv:
        raise ValueError(f"heads of q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not fit")
    if bias is not None and (bias.H != H or bias.device != dev):
        raise ValueError(f"bias: expected {H} heads on {dev}, got {bias.H} on {bias.device}")
    return AttnC(code, H, Hkv, D, D ** -0.5 if scale is None else scale, cap, _row(q, "q"), _row(k, "k"), _row(v, "v"))


def group_attention(groups: Groups, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                    bias: Optional[RelativeBias] = None, scale: Optional[float] = None, cap: float = 0.0,
                    out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Attention of each center over its group (cagq_group_attention): ``q`` [B, M, H, D], ``k`` and ``v``
    [B, N, Hkv, D] of float32, bfloat16 or float16. ``scale`` is D ** -0.5 by default; ``cap`` > 0 caps the scores
    by a tanh. Returns (out [B, M, H, D], lse float32 [B, M, H]), which carry no autograd graph, whatever the inputs
    require: ``group_attention_backward`` makes the gradients."""
    h, b = _handle(stream, groups), None if bias is None else bias.ref()
    a = _attn(groups, q, k, v, bias, scale, cap)
    if out is None:
        out = _empty_as(q, stream)
    else:
        _on(out, q.dtype, q.shape, "out", groups.device)
    if lse is None:
        lse = _empty(q, q.shape[:3], _F32, stream)
    else:
        _on(lse, _F32, q.shape[:3], "lse", groups.device)
    L, g, ab = _lib or lib(), C.byref(groups.rec), C.byref(a)
    p, n, _held = _scratch(workspace, L.cagq_group_attention_workspace, (g, ab, b, 0), q, stream, "cagq_group_attention")
    _check(L.cagq_group_attention(g, ab, b, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                  p, n, h), "cagq_group_attention")
    return out, lse


def point_lists(groups: Groups, off: Optional[torch.Tensor] = None, center: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """The groups turned round (cagq_point_lists): offsets int64 [B*N + 1] and, for each point, the centers whose
    groups hold it, ascending, int32 [slots] (-1 behind the last list)."""
    h = _handle(stream, groups)
    idx, points = groups.idx, groups.B * groups.N
    if off is None:
        off = _empty(idx, points + 1, _I64, stream)
    else:
        _on(off, _I64, (points + 1,), "off", groups.device)
    if center is None:
        center = _empty(idx, idx.numel(), _I32, stream)
    else:
        _on(center, _I32, center.shape, "center", groups.device)
    L, g = _lib or lib(), C.byref(groups.rec)
    p, n, _held = _scratch(workspace, L.cagq_point_lists_workspace, (g,), idx, stream, "cagq_point_lists")
    _check(L.cagq_point_lists(g, off.data_ptr(), center.data_ptr(), center.numel(), p, n, h), "cagq_point_lists")
    return off, center


def group_attention_backward(groups: Groups, lists, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                             lse: torch.Tensor, dout: torch.Tensor, bias: Optional[RelativeBias] = None,
                             scale: Optional[float] = None, cap: float = 0.0,
                             workspace: Optional[torch.Tensor] = None,
                             stream: Optional[torch.cuda.Stream] = None) -> Dict[str, Optional[torch.Tensor]]:
    """Gradients of ``group_attention`` for the gradient ``dout`` of its output (cagq_group_attention_backward),
    with ``lists`` from ``point_lists`` of the same groups: dq, dk, dv of the features' type, dtable and dslope
    float32 (None where the bias has no such part). ``dout`` and ``lse`` must be contiguous."""
    h, b = _handle(stream, groups), None if bias is None else bias.ref()
    a = _attn(groups, q, k, v, bias, scale, cap)
    dev = groups.device
    off, center = lists
    _on(off, _I64, (groups.B * groups.N + 1,), "lists[0]", dev)
    _on(center, _I32, center.shape, "lists[1]", dev)
    _on(lse, _F32, q.shape[:3], "lse", dev)
    _on(dout, q.dtype, q.shape, "dout", dev)
    dq, dk, dv = _empty_as(dout, stream), _empty_as(k, stream), _empty_as(k, stream)
    dtable = dslope = None
    if bias is not None:
        if bias.table is not None:
            dtable = _empty_as(bias.table, stream)
        if bias.slope is not None:
            dslope = _empty_as(bias.slope, stream)
    L, g, ab = _lib or lib(), C.byref(groups.rec), C.byref(a)
    what = "cagq_group_attention_backward"
    p, n, _held = _scratch(workspace, L.cagq_group_attention_workspace, (g, ab, b, 1), q, stream, what)
    _check(L.cagq_group_attention_backward(
        g, ab, b, off.data_ptr(), center.data_ptr(), center.numel(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
        lse.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(dtable), _ptr(dslope), p, n,
        h), what)
    return dict(dq=dq, dk=dk, dv=dv, dtable=dtable, dslope=dslope)


def relative_bias(groups: Groups, bias: RelativeBias, dtype=torch.float32, out: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The relative position bias of every slot (cagq_relative_bias): [B, M, K, H], or [entries, H] of ragged
    groups; 0 in the slots that do not count. It carries no autograd graph: ``relative_bias_backward`` makes the
    gradients."""
    h, b = _handle(stream, groups), bias.ref()
    code = FEATURES.get(dtype)
    if code is None or bias.device != groups.device:
        raise ValueError(f"relative_bias: {dtype} with a bias on {bias.device} for groups on {groups.device}")
    shape = (*groups.idx.shape, bias.H)
    if out is None:
        out = _empty(groups.idx, shape, dtype, stream)
    else:
        _on(out, dtype, shape, "out", groups.device)
    _check((_lib or lib()).cagq_relative_bias(C.byref(groups.rec), b, bias.H, code, out.data_ptr(),
                                              h), "cagq_relative_bias")
    return out


def relative_bias_backward(groups: Groups, bias: RelativeBias, dbias: torch.Tensor,
                           workspace: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None):
    """(dtable, dslope), float32, for the gradient ``dbias`` of ``relative_bias``'s output
    (cagq_relative_bias_backward); None where the bias has no such part."""
    dev, h, b = groups.device, _handle(stream, groups), bias.ref()
    code = FEATURES.get(dbias.dtype)
    if code is None or bias.device != dev:
        raise ValueError(f"relative_bias_backward: {dbias.dtype} with a bias on {bias.device} for groups on {dev}")
    _on(dbias, dbias.dtype, (*groups.idx.shape, bias.H), "dbias", dev)
    dtable = None if bias.table is None else _empty_as(bias.table, stream)
    dslope = None if bias.slope is None else _empty_as(bias.slope, stream)
    L, g = _lib or lib(), C.byref(groups.rec)
    what = "cagq_relative_bias_backward"
    p, n, _held = _scratch(workspace, L.cagq_relative_bias_workspace, (g, b, bias.H), dbias, stream, what)
    _check(L.cagq_relative_bias_backward(g, b, bias.H, code, dbias.data_ptr(), _ptr(dtable), _ptr(dslope), p, n, h), what)
    return dtable, dslope


def get_device_status(grid: Grid, stream: Optional[torch.cuda.Stream] = None) -> int:
    """Synchronises the stream; first device-side error since the grid was built."""
    return int(lib().cagq_get_device_status(C.byref(grid.rec), _stream_ptr(stream)))


def run_layer(points: torch.Tensor, layer, weights: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None):
    """One CAGQ layer (build, sample, query) for a LayerSpec-like object.

    Returns (grid, center_lin, m_valid, query outputs)."""
    g = build_grid(points, desc_from_spec(layer.grid), workspace)
    cl, mv = sample_centers(g, layer.M, layer.sample, layer.seed)
    q = query_context(g, cl, layer.K, layer.query, layer.seed, weights=weights)
    return g, cl, mv, q
