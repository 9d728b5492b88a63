"""torch.Tensor wrappers over the C ABI (argument marshalling only).

Every function allocates its outputs with ``torch.empty`` on the input's
device (unless ``out=`` is given), passes raw device pointers, leading
dimensions and the current HIP stream, and raises on a non-zero status.
All arithmetic happens in libmesorasi.so.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import _lib
from ._lib import F32, BF16, I8, check

_vp = ctypes.c_void_p


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _rows(t: torch.Tensor, width: int | None = None):
    """(pointer, leading dimension) of a [..., rows, C] tensor whose last dim
    is contiguous and whose leading dims collapse to one row index."""
    assert t.stride(-1) == 1, "last dimension must be contiguous"
    ld = t.stride(-2) if t.dim() >= 2 else t.shape[-1]
    # all leading dims must be row-contiguous multiples of ld
    expect = ld * t.shape[-2] if t.dim() >= 2 else None
    for d in range(t.dim() - 3, -1, -1):
        # the stride of a size-1 dimension is never used
        assert t.shape[d] == 1 or t.stride(d) == expect, "leading dimensions must collapse into rows"
        expect *= t.shape[d]
    if width is not None:
        assert t.shape[-1] >= width
    return t.data_ptr(), ld


def _check_xyz(x: torch.Tensor, name: str):
    assert x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 3 and x.shape[-1] == 3, \
        f"{name} must be a contiguous float32 [B, N, 3] tensor"


def fps_workspace_bytes(B: int, N: int, M: int) -> int:
    return int(_lib.lib().mesorasi_fps_workspace(B, N, M))


def fps(xyz: torch.Tensor, M: int, want_xyz: bool = True, out_idx: torch.Tensor | None = None,
        out_xyz: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """ws: a uint8 device tensor of at least fps_workspace_bytes(B, N, M)
    (allocated here when needed and not given); its first 4 bytes read 0
    after the call unless a workgroup gave up waiting (see the C header)."""
    _check_xyz(xyz, "xyz")
    B, N, _ = xyz.shape
    idx = out_idx if out_idx is not None else torch.empty((B, M), dtype=torch.int32, device=xyz.device)
    cxyz = out_xyz if out_xyz is not None else (
        torch.empty((B, M, 3), dtype=torch.float32, device=xyz.device) if want_xyz else None)
    need = fps_workspace_bytes(B, N, M)
    if need and (ws is None or ws.numel() < need):
        ws = torch.empty(need, dtype=torch.uint8, device=xyz.device)
    wp, wn = (ws.data_ptr(), ws.numel()) if need else (None, 0)
    check(_lib.lib().mesorasi_fps(xyz.data_ptr(), B, N, M, idx.data_ptr(), _ptr(cxyz), wp, wn, _stream()), "fps")
    return idx, cxyz


def fps_prefix(idx_prev: torch.Tensor, cxyz_prev: torch.Tensor | None, M: int, out_idx: torch.Tensor | None = None,
               out_xyz: torch.Tensor | None = None, want_xyz: bool = True):
    """The sampling of M points from (idx_prev, cxyz_prev), an earlier
    fps() (or fps_prefix()) output: its first M points (see the C header)."""
    if idx_prev.dtype != torch.int32 or idx_prev.dim() != 2 or not idx_prev.is_contiguous():
        raise ValueError("idx_prev must be a contiguous [B, M_prev] int32 tensor")
    B, Mp = idx_prev.shape
    if cxyz_prev is not None:
        _check_xyz(cxyz_prev, "cxyz_prev")
        if tuple(cxyz_prev.shape[:2]) != (B, Mp):
            raise ValueError("cxyz_prev must be [B, M_prev, 3]")
    idx = out_idx if out_idx is not None else torch.empty((B, M), dtype=torch.int32, device=idx_prev.device)
    cxyz = out_xyz if out_xyz is not None else (
        torch.empty((B, M, 3), dtype=torch.float32, device=idx_prev.device)
        if want_xyz and cxyz_prev is not None else None)
    check(_lib.lib().mesorasi_fps_prefix(idx_prev.data_ptr(), _ptr(cxyz_prev), B, Mp, M, idx.data_ptr(), _ptr(cxyz),
                                         _stream()), "fps_prefix")
    return idx, cxyz


def fps_prefix_levels(idx0: torch.Tensor, cxyz0: torch.Tensor | None, Ms, out_idx=None, out_xyz=None):
    """Nested levels of M[v] points each, all prefixes of (idx0, cxyz0), in
    one launch (mesorasi_fps_prefix_levels).  Returns [(idx, cxyz)] per
    level."""
    if idx0.dtype != torch.int32 or idx0.dim() != 2 or not idx0.is_contiguous():
        raise ValueError("idx0 must be a contiguous [B, M0] int32 tensor")
    B, M0 = idx0.shape
    if cxyz0 is not None:
        _check_xyz(cxyz0, "cxyz0")
    n = len(Ms)
    idx = list(out_idx) if out_idx is not None else [
        torch.empty((B, m), dtype=torch.int32, device=idx0.device) for m in Ms]
    xyz = list(out_xyz) if out_xyz is not None else (
        [torch.empty((B, m, 3), dtype=torch.float32, device=idx0.device) for m in Ms] if cxyz0 is not None
        else [None] * n)
    Mc = (ctypes.c_int64 * max(n, 1))(*Ms)
    ic = (_vp * max(n, 1))(*[t.data_ptr() for t in idx])
    xc = (_vp * max(n, 1))(*[None if t is None else t.data_ptr() for t in xyz])
    check(_lib.lib().mesorasi_fps_prefix_levels(idx0.data_ptr(), _ptr(cxyz0), B, M0, n, ctypes.cast(Mc, _vp),
                                                ctypes.cast(ic, _vp), ctypes.cast(xc, _vp), _stream()),
          "fps_prefix_levels")
    return list(zip(idx, xyz))


def ball_query_workspace_bytes(B: int, N: int, M: int) -> int:
    return int(_lib.lib().mesorasi_ball_query_workspace(B, N, M))


def ball_query(xyz: torch.Tensor, qxyz: torch.Tensor, radius: float, K: int, want_cnt: bool = False,
               out: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """ws: a uint8 device tensor of at least ball_query_workspace_bytes(B, N,
    M) (allocated here when needed and not given)."""
    _check_xyz(xyz, "xyz")
    _check_xyz(qxyz, "qxyz")
    B, N, _ = xyz.shape
    M = qxyz.shape[1]
    nit = out if out is not None else torch.empty((B, M, K), dtype=torch.int32, device=xyz.device)
    cnt = torch.empty((B, M), dtype=torch.int32, device=xyz.device) if want_cnt else None
    need = ball_query_workspace_bytes(B, N, M)
    if need and (ws is None or ws.numel() < need):
        ws = torch.empty(need, dtype=torch.uint8, device=xyz.device)
    wp, wn = (ws.data_ptr(), ws.numel()) if need else (None, 0)
    check(_lib.lib().mesorasi_ball_query(xyz.data_ptr(), qxyz.data_ptr(), B, N, M, float(radius), K, nit.data_ptr(),
                                         _ptr(cnt), wp, wn, _stream()), "ball_query")
    return nit, cnt


def ball_query_grid_workspace_bytes(B: int, N: int) -> int:
    return int(_lib.lib().mesorasi_ball_query_grid_workspace(B, N))


def ball_query_grid_build(xyz: torch.Tensor, radius: float, ws: torch.Tensor | None = None) -> torch.Tensor:
    """Bin the clouds of xyz for ball queries of radius up to `radius`
    (mesorasi_ball_query_grid_build); returns the workspace holding the grid."""
    _check_xyz(xyz, "xyz")
    B, N, _ = xyz.shape
    need = ball_query_grid_workspace_bytes(B, N)
    if ws is None or ws.numel() < need:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=xyz.device)
    check(_lib.lib().mesorasi_ball_query_grid_build(xyz.data_ptr(), B, N, float(radius), ws.data_ptr(), ws.numel(),
                                                    _stream()), "ball_query_grid_build")
    return ws


def ball_query_grid(xyz: torch.Tensor, qxyz: torch.Tensor, radius: float, K: int, grid: torch.Tensor,
                    want_cnt: bool = False, out: torch.Tensor | None = None):
    """ball_query() against a grid from ball_query_grid_build() on the same
    xyz (mesorasi_ball_query_grid): the same result."""
    _check_xyz(xyz, "xyz")
    _check_xyz(qxyz, "qxyz")
    B, N, _ = xyz.shape
    M = qxyz.shape[1]
    nit = out if out is not None else torch.empty((B, M, K), dtype=torch.int32, device=xyz.device)
    cnt = torch.empty((B, M), dtype=torch.int32, device=xyz.device) if want_cnt else None
    check(_lib.lib().mesorasi_ball_query_grid(xyz.data_ptr(), qxyz.data_ptr(), B, N, M, float(radius), K,
                                              nit.data_ptr(), _ptr(cnt), grid.data_ptr(), grid.numel(), _stream()),
          "ball_query_grid")
    return nit, cnt


def knn(ref: torch.Tensor, query: torch.Tensor, K: int, want_dist: bool = False, out: torch.Tensor | None = None):
    """ref [B, N, >=C], query [B, M, >=C] (last dim contiguous, may be
    column slices of wider tensors); C = ref.shape[-1]."""
    assert ref.dtype == torch.float32 and query.dtype == torch.float32
    B, N, C = ref.shape
    M = query.shape[1]
    pr, ldr = _rows(ref)
    pq, ldq = _rows(query)
    nit = out if out is not None else torch.empty((B, M, K), dtype=torch.int32, device=ref.device)
    dist = torch.empty((B, M, K), dtype=torch.float32, device=ref.device) if want_dist else None
    check(_lib.lib().mesorasi_knn(pr, ldr, pq, ldq, B, N, M, C, K, nit.data_ptr(), _ptr(dist), _stream()), "knn")
    return nit, dist


class MLPParams:
    """Weights of one shared MLP on the device, plus the host pointer arrays
    the ABI takes.  W[l] is [C_out, C_in] (torch Linear layout)."""

    def __init__(self, Ws, bs, dtype: int = F32, device="cuda"):
        self.dtype = dtype
        self.dims = [int(Ws[0].shape[1])] + [int(W.shape[0]) for W in Ws]
        self.n = len(Ws)
        self.W32 = [torch.as_tensor(W, dtype=torch.float32).to(device).contiguous() for W in Ws]
        self.b = [None if b is None else torch.as_tensor(b, dtype=torch.float32).to(device).contiguous() for b in bs]
        if dtype == BF16:
            self.W = [cast_bf16(W) for W in self.W32]
        else:
            self.W = self.W32
        self._dims_c = (ctypes.c_int32 * (self.n + 1))(*self.dims)
        self._W_c = (_vp * self.n)(*[W.data_ptr() for W in self.W])
        self._b_c = (_vp * self.n)(*[None if b is None else b.data_ptr() for b in self.b])

    @property
    def c_out(self):
        return self.dims[-1]

    def abi(self):
        return (ctypes.cast(self._dims_c, _vp), ctypes.cast(self._W_c, _vp), ctypes.cast(self._b_c, _vp))


def mlp_workspace_bytes(rows: int, p: MLPParams, pool_group: int = 0) -> int:
    d, _, _ = p.abi()
    return int(_lib.lib().mesorasi_pointwise_mlp_workspace(rows, p.n, d, p.dtype, pool_group))


def pointwise_mlp(x0: torch.Tensor, p: MLPParams, x1: torch.Tensor | None = None, relu_mask: int | None = None,
                  out_dtype: int = F32, pool_group: int = 0, out: torch.Tensor | None = None,
                  ws: torch.Tensor | None = None):
    """MLP on the rows of [x0 | x1].  x0 [..., R, c0], x1 [..., R, c1].
    pool_group > 0 returns the column max over each group of rows."""
    p0, ld0 = _rows(x0)
    c0 = x0.shape[-1]
    if x1 is not None:
        p1, ld1 = _rows(x1)
        c1 = x1.shape[-1]
    else:
        p1, ld1, c1 = None, 0, 0
    rows = math.prod(x0.shape[:-1])
    if relu_mask is None:
        relu_mask = (1 << p.n) - 1
    lead = tuple(x0.shape[:-1])
    if out is None:
        dt = torch.float32 if out_dtype == F32 else torch.bfloat16
        if pool_group:
            out = torch.empty((rows // pool_group, p.c_out), dtype=dt, device=x0.device)
        else:
            out = torch.empty(lead + (p.c_out,), dtype=dt, device=x0.device)
    py, ldy = _rows(out)
    need = mlp_workspace_bytes(rows, p, pool_group)
    if need and (ws is None or ws.numel() < need):
        ws = torch.empty(need, dtype=torch.uint8, device=x0.device)
    wp, wn = (ws.data_ptr(), ws.numel()) if need else (None, 0)
    d, W, b = p.abi()
    check(_lib.lib().mesorasi_pointwise_mlp(p0, c0, ld0, p1, c1, ld1, rows, p.n, d, W, b, relu_mask, p.dtype,
                                            out_dtype, py, ldy, pool_group, wp, wn, _stream()),
          "pointwise_mlp")
    return out


def pointwise_mlp_noalloc(x0: torch.Tensor, p: MLPParams, x1: torch.Tensor | None = None,
                          relu_mask: int | None = None, out_dtype: int = F32, pool_group: int = 0,
                          out: torch.Tensor | None = None):
    """pointwise_mlp through the allocation-free entry point: the library's
    fixed per-GPU scratch array replaces the workspace (calls that overlap
    on one GPU race).  Only `out` is allocated here, when not given."""
    p0, ld0 = _rows(x0)
    c0 = x0.shape[-1]
    if x1 is not None:
        p1, ld1 = _rows(x1)
        c1 = x1.shape[-1]
    else:
        p1, ld1, c1 = None, 0, 0
    rows = math.prod(x0.shape[:-1])
    if relu_mask is None:
        relu_mask = (1 << p.n) - 1
    if out is None:
        dt = torch.float32 if out_dtype == F32 else torch.bfloat16
        shape = (rows // pool_group, p.c_out) if pool_group else tuple(x0.shape[:-1]) + (p.c_out,)
        out = torch.empty(shape, dtype=dt, device=x0.device)
    py, ldy = _rows(out)
    d, W, b = p.abi()
    check(_lib.lib().mesorasi_pointwise_mlp_noalloc(p0, c0, ld0, p1, c1, ld1, rows, p.n, d, W, b, relu_mask,
                                                    p.dtype, out_dtype, py, ldy, pool_group, _stream()),
          "pointwise_mlp_noalloc")
    return out


def aggregate_mlp_supported(p: MLPParams, C: int) -> bool:
    """The fused aggregate-into-MLP form applies: an fp32 MLP of at least two
    layers, inputs <= 160 and outputs <= 128 channels, first layer 3 + C."""
    return (p.dtype == F32 and p.n >= 2 and p.dims[0] == 3 + C and C % 4 == 0
            and all(((d + 15) // 16) * 16 <= 160 for d in p.dims[:-1]) and all(d <= 128 for d in p.dims[1:]))


def aggregate_mlp(cxyz: torch.Tensor, pft: torch.Tensor, nit: torch.Tensor, cidx: torch.Tensor, p: MLPParams,
                  relu_mask: int | None = None, out: torch.Tensor | None = None, agg_out: torch.Tensor | None = None):
    """MLP of module i + 1 on [cxyz | module i's aggregation] with the
    aggregation done in the MLP's loader; agg_out (optional) also receives
    the aggregated rows.  cxyz [B, M, 3], pft [B, N, >=C] float32, nit
    [B, M, K], cidx [B, M]."""
    _check_xyz(cxyz, "cxyz")
    B, M, K = nit.shape
    N, C = pft.shape[1], pft.shape[-1]
    assert pft.dtype == torch.float32 and nit.is_contiguous() and cidx.is_contiguous()
    pp, ldp = _rows(pft)
    if relu_mask is None:
        relu_mask = (1 << p.n) - 1
    if out is None:
        out = torch.empty((B, M, p.c_out), dtype=torch.float32, device=pft.device)
    py, ldy = _rows(out)
    pa, lda = _rows(agg_out) if agg_out is not None else (None, 0)
    d, W, b = p.abi()
    check(_lib.lib().mesorasi_aggregate_mlp(cxyz.data_ptr(), pp, ldp, nit.data_ptr(), cidx.data_ptr(), B, N, M, K, C,
                                            p.n, d, W, b, relu_mask, py, ldy, pa, lda, _stream()), "aggregate_mlp")
    return out


def aggregate_max(pft: torch.Tensor, nit: torch.Tensor, cidx: torch.Tensor | None = None,
                  cfeat: torch.Tensor | None = None, sign: int = -1, relu: bool = False,
                  out: torch.Tensor | None = None):
    """pft [B, N, >=C] float32 or bfloat16; nit [B, M, K] int32;
    cidx [B, M] int32 or cfeat [B, M, >=C] (same dtype as pft)."""
    B, N, C = pft.shape
    M, K = nit.shape[1], nit.shape[2]
    dt = F32 if pft.dtype == torch.float32 else BF16
    pp, ldp = _rows(pft)
    if cfeat is not None:
        assert cfeat.dtype == pft.dtype
        pc, ldc = _rows(cfeat)
    else:
        pc, ldc = None, 0
    if out is None:
        out = torch.empty((B, M, C), dtype=torch.float32, device=pft.device)
    po, ldo = _rows(out)
    assert nit.is_contiguous() and nit.dtype == torch.int32
    check(_lib.lib().mesorasi_aggregate_max(pp, ldp, dt, nit.data_ptr(), B, N, M, K, C, _ptr(cidx), pc, ldc, sign,
                                            1 if relu else 0, po, ldo, _stream()), "aggregate_max")
    return out


def conventional_workspace_bytes(B: int, M: int, K: int, p: MLPParams) -> int:
    d, _, _ = p.abi()
    return int(_lib.lib().mesorasi_conventional_workspace(B, M, K, p.n, d, p.dtype))


def conventional_module(nit: torch.Tensor, p: MLPParams, xyz: torch.Tensor | None = None,
                        feat: torch.Tensor | None = None, cxyz: torch.Tensor | None = None, grouping: int = 0,
                        relu_mask: int | None = None, out: torch.Tensor | None = None,
                        ws: torch.Tensor | None = None):
    """grouping 0: [xyz_j - cxyz_c | feat_j] (PointNet++); grouping 1:
    [f_i | f_j - f_i] with f = feat (DGCNN edge features)."""
    B, M, K = nit.shape
    if grouping == 0:
        N = xyz.shape[1]
    else:
        N = feat.shape[1]
    cf = 0 if feat is None else feat.shape[-1]
    pf, ldf = _rows(feat) if feat is not None else (None, max(cf, 1))
    if relu_mask is None:
        relu_mask = (1 << p.n) - 1
    if out is None:
        out = torch.empty((B, M, p.c_out), dtype=torch.float32, device=nit.device)
    po, ldo = _rows(out)
    need = conventional_workspace_bytes(B, M, K, p)
    if ws is None or ws.numel() < need:
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=nit.device)
    d, W, b = p.abi()
    check(_lib.lib().mesorasi_conventional_module(_ptr(xyz), pf, cf, ldf, _ptr(cxyz), nit.data_ptr(), B, N, M, K,
                                                  grouping, p.n, d, W, b, relu_mask, p.dtype, po, ldo,
                                                  ws.data_ptr(), ws.numel(), _stream()), "conventional_module")
    return out


def ltd_workspace_bytes(B: int, M: int, K: int, p: MLPParams) -> int:
    d, _, _ = p.abi()
    return int(_lib.lib().mesorasi_ltd_workspace(B, M, K, p.n, d, p.dtype))


def ltd_module(p1: torch.Tensor, q: torch.Tensor, nit: torch.Tensor, p: MLPParams, b1: torch.Tensor | None = None,
               relu_mask: int | None = None, out: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """Limited delayed aggregation (Sec. 7.3): p1 [B, N, >=C1] = the first
    layer's product on the input points, q [B, M, >=C1] = its centroid
    term, b1 [C1] the first layer's bias; p = the remaining layers.
    Returns max_k MLP_rest(ReLU(p1[nit] - q + b1)) [B, M, C_out]."""
    B, M, K = nit.shape
    N, C1 = p1.shape[1], p.dims[0]
    pp, ldp = _rows(p1, C1)
    pq, ldq = _rows(q, C1)
    if relu_mask is None:
        relu_mask = (1 << p.n) - 1
    if out is None:
        out = torch.empty((B, M, p.c_out), dtype=torch.float32, device=nit.device)
    po, ldo = _rows(out)
    need = ltd_workspace_bytes(B, M, K, p)
    if ws is None or ws.numel() < need:
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=nit.device)
    d, W, b = p.abi()
    check(_lib.lib().mesorasi_ltd_module(pp, ldp, pq, ldq, _ptr(b1), nit.data_ptr(), B, N, M, K, C1, p.n, d, W, b,
                                         relu_mask, p.dtype, po, ldo, ws.data_ptr(), ws.numel(), _stream()),
          "ltd_module")
    return out


def interpolate3(xyz_dst: torch.Tensor, xyz_src: torch.Tensor, f_src: torch.Tensor,
                 out: torch.Tensor | None = None):
    _check_xyz(xyz_dst, "xyz_dst")
    _check_xyz(xyz_src, "xyz_src")
    B, Nd, _ = xyz_dst.shape
    Ns = xyz_src.shape[1]
    C = f_src.shape[-1]
    ps, lds = _rows(f_src)
    if out is None:
        out = torch.empty((B, Nd, C), dtype=torch.float32, device=f_src.device)
    po, ldo = _rows(out)
    check(_lib.lib().mesorasi_interpolate3(xyz_dst.data_ptr(), xyz_src.data_ptr(), ps, lds, B, Nd, Ns, C, po, ldo,
                                           _stream()), "interpolate3")
    return out


def three_nn(xyz_dst: torch.Tensor, xyz_src: torch.Tensor, out_nit: torch.Tensor | None = None,
             out_dist: torch.Tensor | None = None):
    """The 3 nearest sources of every destination (indices, squared
    distances), as mesorasi_knn with K = 3."""
    _check_xyz(xyz_dst, "xyz_dst")
    _check_xyz(xyz_src, "xyz_src")
    B, Nd, _ = xyz_dst.shape
    Ns = xyz_src.shape[1]
    nit = out_nit if out_nit is not None else torch.empty((B, Nd, 3), dtype=torch.int32, device=xyz_dst.device)
    dist = out_dist if out_dist is not None else torch.empty((B, Nd, 3), dtype=torch.float32, device=xyz_dst.device)
    check(_lib.lib().mesorasi_three_nn(xyz_dst.data_ptr(), xyz_src.data_ptr(), B, Nd, Ns, nit.data_ptr(),
                                       dist.data_ptr(), _stream()), "three_nn")
    return nit, dist


def interpolate3_apply(nit: torch.Tensor, dist: torch.Tensor, f_src: torch.Tensor, out: torch.Tensor | None = None):
    """Inverse-distance interpolation from precomputed 3-NN (three_nn)."""
    assert nit.dtype == torch.int32 and nit.is_contiguous() and dist.dtype == torch.float32 and dist.is_contiguous()
    B, Nd, _ = nit.shape
    Ns, C = f_src.shape[1], f_src.shape[-1]
    ps, lds = _rows(f_src)
    if out is None:
        out = torch.empty((B, Nd, C), dtype=torch.float32, device=f_src.device)
    po, ldo = _rows(out)
    check(_lib.lib().mesorasi_interpolate3_apply(nit.data_ptr(), dist.data_ptr(), ps, lds, B, Nd, Ns, C, po, ldo,
                                                 _stream()), "interpolate3_apply")
    return out


def interpolate3_add(nit: torch.Tensor, dist: torch.Tensor, f_src: torch.Tensor, add: torch.Tensor,
                     relu: bool = True, out: torch.Tensor | None = None):
    """phi(interpolation of f_src from precomputed 3-NN + add), phi = ReLU
    when relu: a feature-propagation first layer whose interpolated part
    was multiplied on the coarse points.  out may be add itself."""
    assert nit.dtype == torch.int32 and nit.is_contiguous() and dist.dtype == torch.float32 and dist.is_contiguous()
    B, Nd, _ = nit.shape
    Ns, C = f_src.shape[1], f_src.shape[-1]
    assert add.shape[:2] == (B, Nd) and add.shape[-1] == C and add.dtype == torch.float32
    ps, lds = _rows(f_src)
    pa, lda = _rows(add)
    if out is None:
        out = torch.empty((B, Nd, C), dtype=torch.float32, device=f_src.device)
    po, ldo = _rows(out)
    check(_lib.lib().mesorasi_interpolate3_add(nit.data_ptr(), dist.data_ptr(), ps, lds, B, Nd, Ns, C, pa, lda,
                                               1 if relu else 0, po, ldo, _stream()), "interpolate3_add")
    return out


def interpolate3_mlp_supported(p: MLPParams, rows: int) -> bool:
    """mesorasi_interpolate3_mlp applies: an fp32 MLP whose layers are all at
    most 128 wide (the register-resident MLP), first layer a multiple of 4,
    and, when the layers' fp32 weights make more than 160 KB, at most one
    32-row tile per wave (8 per compute unit).  This mirrors the library's
    rule."""
    if p.dtype != F32 or p.dims[0] % 4 != 0 or any(d > 128 for d in p.dims):
        return False
    h0 = ((p.dims[0] + 1) // 2 + 15) // 16 * 16     # first-layer k steps, as the library pads them
    cap, off, phases = 160 * 1024, 0, 1
    for l in range(p.n):
        nob = (p.dims[l + 1] + 31) // 32
        steps = h0 if l == 0 else 16 * ((p.dims[l] + 31) // 32)
        size = 4 * (nob * steps * 64 + nob * 32)
        if off + size > cap:
            phases, off = phases + 1, 0
        off += size
    if phases == 1:
        return True
    cus = torch.cuda.get_device_properties(torch.cuda.current_device()).multi_processor_count
    return (rows + 31) // 32 <= 8 * cus


def interpolate3_mlp(nit: torch.Tensor, dist: torch.Tensor, f_src: torch.Tensor, add: torch.Tensor, p: MLPParams,
                     relu: bool = True, relu_mask: int | None = None, out: torch.Tensor | None = None):
    """MLP on the rows phi(interpolation of f_src + add) in one kernel
    (mesorasi_interpolate3_mlp)."""
    assert nit.dtype == torch.int32 and nit.is_contiguous() and dist.dtype == torch.float32 and dist.is_contiguous()
    B, Nd, _ = nit.shape
    Ns = f_src.shape[1]
    assert add.shape[:2] == (B, Nd) and add.shape[-1] == p.dims[0] and f_src.shape[-1] == p.dims[0]
    ps, lds = _rows(f_src)
    pa, lda = _rows(add)
    if out is None:
        out = torch.empty((B, Nd, p.c_out), dtype=torch.float32, device=f_src.device)
    po, ldo = _rows(out)
    d, W, b = p.abi()
    rm = (1 << p.n) - 1 if relu_mask is None else relu_mask
    check(_lib.lib().mesorasi_interpolate3_mlp(nit.data_ptr(), dist.data_ptr(), ps, lds, B, Nd, Ns, pa, lda,
                                               1 if relu else 0, p.n, d, W, b, rm, po, ldo, _stream()),
          "interpolate3_mlp")
    return out


def cast_bf16(x: torch.Tensor) -> torch.Tensor:
    """float32 -> bfloat16 (round to nearest even) on the device."""
    assert x.dtype == torch.float32 and x.is_contiguous()
    y = torch.empty(x.shape, dtype=torch.bfloat16, device=x.device)
    check(_lib.lib().mesorasi_cast_bf16(x.data_ptr(), x.numel(), y.data_ptr(), _stream()), "cast_bf16")
    return y


def edgeconv_fold(W: torch.Tensor, b: torch.Tensor | None):
    """W [C_out, 2C] -> ([W1 - W2 ; W2] [2 C_out, C], [b ; 0])."""
    Cout, C2 = W.shape
    C = C2 // 2
    Wo = torch.empty((2 * Cout, C), dtype=torch.float32, device=W.device)
    bo = torch.empty((2 * Cout,), dtype=torch.float32, device=W.device)
    check(_lib.lib().mesorasi_edgeconv_fold(W.data_ptr(), _ptr(b), C, Cout, Wo.data_ptr(), bo.data_ptr(), _stream()),
          "edgeconv_fold")
    return Wo, bo


def count_out_of_range(idx: torch.Tensor, bound: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """Device int32 scalar: entries of idx outside [0, bound) (debug check)."""
    assert idx.dtype == torch.int32 and idx.is_contiguous()
    count = out if out is not None else torch.empty((), dtype=torch.int32, device=idx.device)
    check(_lib.lib().mesorasi_count_out_of_range(idx.data_ptr(), idx.numel(), int(bound), count.data_ptr(),
                                                 _stream()), "count_out_of_range")
    return count


# ---------------------------------------------------------------------------
# the operators of an attention level
# ---------------------------------------------------------------------------

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_ACTS = {"none": _lib.ACT_NONE, "relu": _lib.ACT_RELU, "silu": _lib.ACT_SILU, "gelu": _lib.ACT_GELU}


def _require(cond, msg: str):
    if not cond:
        raise ValueError(msg)


def _dtype(t: torch.Tensor, name: str) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return dt


def _like(t, x: torch.Tensor, name: str, dtype, shape):
    """t (may be None) is a contiguous tensor of this dtype and shape on x's device."""
    if t is not None and not (t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.device == x.device):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {list(shape)} on {x.device}")


_entry_points: dict = {}


def _entry(name: str):
    fn = _entry_points.get(name)
    if fn is None:
        fn = _entry_points[name] = getattr(_lib.lib(), "mesorasi_" + name)
    return fn


def _call(x: torch.Tensor, where: str, *args):
    """The entry point `where` on x's device, on that device's current stream."""
    if not x.is_cuda:
        raise ValueError(f"{where}: tensors must be on a GPU, not on {x.device}")
    # less host work than torch.cuda's own wrappers, looked up here: a torch built without a GPU has neither
    fn, i, device, stream = _entry(where), x.get_device(), torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    if i == device():
        rc = fn(*args, stream(i))
    else:
        with torch.cuda.device(i):
            rc = fn(*args, stream(i))
    if rc:
        check(rc, where)


def _workspace(x: torch.Tensor, need: int, ws):
    """(pointer, bytes, tensor) of the caller's workspace, or of a new one
    when it is missing or too small."""
    if not need:
        return None, 0, None
    if ws is not None and not (ws.device == x.device and ws.dtype is torch.uint8 and ws.is_contiguous()):
        raise ValueError(f"ws must be a contiguous uint8 tensor on {x.device}")
    if ws is None or ws.numel() < need:
        ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    return ws.data_ptr(), ws.numel(), ws


def _apart(out: torch.Tensor, *inputs):
    """out must not be one of the inputs: other workgroups may still read what one has written."""
    p = out.data_ptr()
    for t in inputs:
        if t.data_ptr() == p and t.numel() and out.numel():
            raise ValueError("out must not be an input")


def _new(x: torch.Tensor, shape, dtype=None) -> torch.Tensor:
    """An uninitialised contiguous tensor on x's device, of x's type unless given."""
    return x.new_empty(shape, dtype=dtype)


def _collapsed(shape, stride, last: int, name: str):
    """The row stride of dimensions 0 .. last, which must collapse into rows;
    None for a single row, whose stride is not used."""
    n, ld = 1, None
    for d in range(last, -1, -1):
        if shape[d] == 1:
            continue
        if ld is None:
            ld = stride[d]
        if stride[d] != ld * n:
            raise ValueError(f"{name}'s leading dimensions must collapse into rows")
        n *= shape[d]
    return ld


def _ld(t: torch.Tensor, name: str):
    """(pointer, leading dimension) of rows of the last dimension."""
    shape = t.shape
    if t.is_contiguous() and len(shape) >= 2:
        return t.data_ptr(), shape[-1]
    stride = t.stride()
    if len(shape) < 2 or (shape[-1] > 1 and stride[-1] != 1):
        raise ValueError(f"{name}'s last dimension must be contiguous")
    ld = _collapsed(shape, stride, len(shape) - 2, name)
    return t.data_ptr(), shape[-1] if ld is None else ld


def group_norm_workspace_bytes(B: int, N: int, C: int, G: int, dtype: int = F32) -> int:
    return int(_lib.lib().mesorasi_group_norm_workspace(B, N, C, G, dtype))


def group_norm(x: torch.Tensor, groups: int, gamma: torch.Tensor | None = None, beta: torch.Tensor | None = None,
               eps: float = 1e-5, act: str = "none", lens: torch.Tensor | None = None,
               out: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """Group norm over each cloud's valid points with an activation ("none",
    "relu", "silu", "gelu").  x [B, N, C] float32 or bfloat16; gamma, beta
    [C] float32; lens [B] int32 (rows from lens[b] on are not read and come
    out 0).  The rows of x and of out are evenly spaced, across
    clouds too.  out: like x, or of the other type (see the C header); it may not
    overlap x, other columns of its rows aside."""
    _require(x.dim() == 3, "x must be [B, N, C]")
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)}")
    B, N, C = x.shape
    dt = dy = _dtype(x, "x")
    _like(gamma, x, "gamma", torch.float32, (C,))
    _like(beta, x, "beta", torch.float32, (C,))
    _like(lens, x, "lens", torch.int32, (B,))
    px, ldx = _ld(x, "x")
    if out is None:
        out = _new(x, (B, N, C))
        py, ldy = out.data_ptr(), C
    else:
        _require(out.shape == x.shape and out.device == x.device, "out must have x's shape and device")
        dy = _dtype(out, "out")
        py, ldy = _ld(out, "out")
        _apart(out, x)
    wp, wn, ws = _workspace(x, _entry("group_norm_workspace")(B, N, C, groups, dt), ws)
    _call(x, "group_norm", px, ldx, dt, B, N, C, groups, _ptr(lens), _ptr(gamma), _ptr(beta), eps, _ACTS[act], py, ldy,
          dy, wp, wn)
    return out


def quantize_int8(x: torch.Tensor, out: torch.Tensor | None = None, scale: torch.Tensor | None = None):
    """Rows in 8 bits with a scale each: (q, scale) of x [..., C] float32 or
    bfloat16.  q [..., C] int8 has rows a multiple of 16 bytes apart, as
    linear_int8 reads them; the bytes behind each row up to the next multiple of
    16 are written as 0, in a given out too.  Neither may overlap x."""
    dt = _dtype(x, "x")
    px, ldx = _ld(x, "x")
    C, lead = x.shape[-1], x.shape[:-1]
    rows = math.prod(lead)
    if out is None:
        out = _new(x, (*lead, (C + 15) // 16 * 16), torch.int8)[..., :C]
    else:
        _require(out.dtype == torch.int8 and out.shape == x.shape and out.device == x.device,
                 "out must be int8 of x's shape, on x's device")
        _apart(out, x)
    if scale is None:
        scale = _new(x, lead, torch.float32)
    else:
        _like(scale, x, "scale", torch.float32, lead)
    pq, ldq = _ld_int8(out, "out")
    _call(x, "quantize_i8", px, ldx, dt, rows, C, pq, ldq, scale.data_ptr())
    return out, scale


def _ld_int8(t: torch.Tensor, name: str):
    """_ld() of 8-bit rows: a single row's leading dimension is its width
    rounded up to 16, within the storage."""
    p, ld = _ld(t, name)
    C = t.shape[-1]
    pad = (C + 15) // 16 * 16
    if ld == C and ld % 16 and t.numel() in (0, C):
        ld = pad
    if pad != C and t.numel() and ld % 16 == 0:
        have = t.untyped_storage().nbytes() - t.storage_offset()
        if (t.numel() // C - 1) * ld + pad > have:
            raise ValueError(f"{name}'s last row must be followed by its padding to 16 bytes")
    return p, ld


def int8_rows(q: torch.Tensor) -> torch.Tensor:
    """int8 rows [..., C] laid out as linear_int8 reads them: a multiple of
    16 bytes apart, zeros behind each."""
    _require(q.dtype == torch.int8, "q must be int8")
    C = q.shape[-1]
    t = torch.zeros(tuple(q.shape[:-1]) + ((C + 15) // 16 * 16,), dtype=torch.int8, device=q.device)
    t[..., :C] = q
    return t[..., :C]


class Int8Params:
    """One layer's weights in 8 bits on the device, laid out for
    linear_int8: Wq [C_out, C_in] int8, w_scale [C_out] float32 (channel o's
    weights are Wq[o] w_scale[o]), bias [C_out] float32 or None."""

    def __init__(self, Wq, w_scale, bias=None, device="cuda"):
        Wq, w_scale = torch.as_tensor(Wq), torch.as_tensor(w_scale)
        _require(Wq.dtype == torch.int8 and Wq.dim() == 2, "Wq must be int8 [C_out, C_in]")
        self.c_out, self.c_in = int(Wq.shape[0]), int(Wq.shape[1])
        _require(w_scale.numel() == self.c_out, "w_scale must hold one scale for each output channel")
        if Wq.is_cuda:
            device = Wq.device
        self.W = int8_rows(Wq.to(device))
        self.ld = (self.c_in + 15) // 16 * 16
        self.w_scale = w_scale.to(device=device, dtype=torch.float32).reshape(-1).contiguous()
        self.bias = None
        if bias is not None:
            self.bias = torch.as_tensor(bias).to(device=device, dtype=torch.float32).reshape(-1).contiguous()
            _require(self.bias.numel() == self.c_out, "bias must hold one value for each output channel")
        self.abi = (self.W.data_ptr(), self.ld, self.w_scale.data_ptr(), _ptr(self.bias), self.c_out)

    @classmethod
    def from_float(cls, W, bias=None, device="cuda"):
        """Float weights [C_out, C_in] brought to 8 bits by quantize_int8's
        rule, a scale for each output channel."""
        W = torch.as_tensor(W, dtype=torch.float32)
        q, s = quantize_int8((W if W.is_cuda else W.to(device)).contiguous())
        return cls(q, s, bias)


def linear_int8_workspace_bytes(rows: int, p: Int8Params, dtype: int = F32) -> int:
    return int(_lib.lib().mesorasi_linear_i8_workspace(rows, p.c_in, p.c_out, dtype))


def linear_int8(x: torch.Tensor, p: Int8Params, x_scale: torch.Tensor | None = None, relu: bool = False,
                out_dtype: torch.dtype | None = None, out: torch.Tensor | None = None,
                ws: torch.Tensor | None = None):
    """A layer's product in 8-bit integers.  x [..., C_in] float32 or
    bfloat16 (brought to 8 bits within the call), or int8 rows of
    quantize_int8() with their x_scale.  out_dtype: float32 (the default) or
    bfloat16.  out may not overlap an input."""
    int8 = x.dtype is torch.int8
    dt = I8 if int8 else _dtype(x, "x")
    *lead, c_in = x.shape
    if c_in != p.c_in:
        raise ValueError(f"x has {c_in} columns, the weights {p.c_in}")
    _require(p.W.device == x.device, "the weights are on another device than x")
    lead = tuple(lead)
    rows = math.prod(lead)
    _require(int8 == (x_scale is not None), "x_scale goes with int8 rows, and only with them")
    if int8:
        _like(x_scale, x, "x_scale", torch.float32, lead)
        px, ldx = _ld_int8(x, "x")
    else:
        px, ldx = _ld(x, "x")
    if out is None:
        out = _new(x, lead + (p.c_out,), out_dtype or torch.float32)
        py, ldy = out.data_ptr(), p.c_out
    else:
        _require(out.shape == lead + (p.c_out,) and out.device == x.device and out_dtype in (None, out.dtype),
                 "out must be [..., C_out] of out_dtype on x's device")
        py, ldy = _ld(out, "out")
        _apart(out, x)
    wp, wn, ws = _workspace(x, _entry("linear_i8_workspace")(rows, c_in, p.c_out, dt), ws)
    _call(x, "linear_i8", px, ldx, dt, _ptr(x_scale), rows, c_in, *p.abi, 1 if relu else 0, py, ldy,
          _dtype(out, "out"), wp, wn)
    return out


class RotaryParams:
    """The angles of rotary positions: sections[a] pairs of a head turn by
    coordinate a, pair i of a section of s by freq = scale base^(-i / s)
    radians per unit, or by the given freq [sum(sections)]."""

    def __init__(self, sections, freq=None, base: float = 10000.0, scale: float = 1.0, interleaved: bool = False,
                 device="cuda"):
        self.sections = [int(s) for s in sections]
        self.interleaved = bool(interleaved)
        if freq is None:
            freq = torch.tensor([scale * base ** (-i / s) for s in self.sections for i in range(s)],
                                dtype=torch.float32)
        freq = torch.as_tensor(freq, dtype=torch.float32)
        self.freq = (freq if freq.is_cuda else freq.to(device)).reshape(-1).contiguous()
        _require(1 <= len(self.sections) <= 4 and min(self.sections) >= 0, "1 to 4 sections of 0 or more pairs")
        _require(self.freq.numel() == sum(self.sections), "freq must hold one value for each pair")
        self._sections_c = (ctypes.c_int32 * len(self.sections))(*self.sections)


def rotary(x: torch.Tensor, pos: torch.Tensor, p: RotaryParams, out: torch.Tensor | None = None):
    """Every head's feature pairs turned by the row's coordinates.  x [..., H,
    D] float32 or bfloat16, heads side by side; pos [..., axes] float32; the
    leading dimensions of each collapse into evenly spaced rows.  out
    may be x, but not overlap an input in another way."""
    dt = _dtype(x, "x")
    shape = x.shape
    _require(len(shape) >= 2, "x must be [..., H, D]")
    *lead, H, D = shape
    axes = len(p.sections)
    if pos.dtype is not torch.float32 or pos.shape != (*lead, axes) or pos.device != x.device:
        raise ValueError(f"pos must be float32 {lead + [axes]} on {x.device}")
    _require(p.freq.device == x.device, "the frequencies are on another device than x")
    px, ldx = _heads(x, "x")
    if out is None:
        out = _new(x, shape)
        py, ldy = out.data_ptr(), H * D
    else:
        _require(out.dtype == x.dtype and out.shape == shape and out.device == x.device, "out must be like x")
        py, ldy = _heads(out, "out")
    pp, ldp = _ld(pos if lead else pos[None], "pos")
    _call(x, "rotary", px, ldx, dt, math.prod(lead), H, D, pp, ldp, axes, p._sections_c, p.freq.data_ptr(),
          1 if p.interleaved else 0, py, ldy)
    return out


def _heads(t: torch.Tensor, name: str):
    """(pointer, leading dimension) of [..., H, D] rows of heads side by side."""
    shape = t.shape
    H, D = shape[-2], shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), H * D
    stride = t.stride()
    if (D > 1 and stride[-1] != 1) or (H > 1 and stride[-2] != D):
        raise ValueError(f"{name}'s heads must lie side by side")
    ld = _collapsed(shape, stride, len(shape) - 3, name)
    return t.data_ptr(), H * D if ld is None else ld


def cross_attention_workspace_bytes(B: int, Nq: int, Nk: int, Hq: int, Hkv: int, D: int, dtype: int = F32) -> int:
    return int(_lib.lib().mesorasi_cross_attention_workspace(B, Nq, Nk, Hq, Hkv, D, dtype))


def _strides(t: torch.Tensor, shape, name: str):
    """Pointer, cloud, point and head strides; those of single entries are not used."""
    b, n, h, c = t.stride()
    if c != 1 and shape[3] > 1:
        raise ValueError(f"{name}'s channels must be contiguous")
    return t.data_ptr(), b if shape[0] > 1 else 0, n if shape[1] > 1 else 0, h if shape[2] > 1 else 0


def cross_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_len: torch.Tensor | None = None,
                    k_mask: torch.Tensor | None = None, scale: float | None = None,
                    out: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """Every query point over the points of another set.  q [B, Nq, Hq, D];
    k, v [B, Nk, Hkv, D], Hq a multiple of Hkv; float32 or bfloat16, any
    strides with contiguous channels (views of one projection, a head-major
    layout transposed, the filled part of a longer buffer).  k_len [B] int32:
    sources from k_len[b] on are not valid; k_mask [B, Nk] bool (its
    clouds may share one row): only the True ones are.  A query without a valid source gives 0.  scale: 1 / sqrt(D)
    unless given.  bfloat16 rounds the weights to its 8 bits where there are many
    rows (see the C header); float32 keeps float32's.  out: like q (its strides
    may differ); it may not overlap q, k or v, other columns of their rows
    aside."""
    qs, ks = q.shape, k.shape
    _require(len(qs) == 4 and len(ks) == 4 and v.shape == ks, "q must be [B, Nq, Hq, D], k and v [B, Nk, Hkv, D]")
    B, Nq, Hq, D = qs
    Nk, Hkv = ks[1], ks[2]
    _require(ks[0] == B and ks[3] == D, "q, k and v must agree in B and D")
    dev, qd = q.device, q.dtype
    _require(k.dtype is qd and v.dtype is qd and k.device == dev and v.device == dev,
             "q, k and v must have one type and device")
    dt = _dtype(q, "q")
    _like(k_len, q, "k_len", torch.int32, (B,))
    mask_ld = 0
    if k_mask is not None:
        if not (k_mask.dtype in (torch.bool, torch.uint8) and k_mask.shape == (B, Nk) and k_mask.device == dev
                and (Nk <= 1 or k_mask.stride(1) == 1)):
            raise ValueError(f"k_mask must be bool [{B}, {Nk}] with contiguous rows on {dev}")
        mask_ld = k_mask.stride(0) if B > 1 else Nk
    if scale is None:
        scale = 1.0 / math.sqrt(D) if D else 1.0
    if out is None:
        out = _new(q, qs)
        po = (out.data_ptr(), max(Nq, 1) * Hq * D, Hq * D, D)
    else:
        _require(out.shape == qs and out.dtype is qd and out.device == dev, "out must be like q")
        po = _strides(out, qs, "out")
        _apart(out, q, k, v)
    wp, wn, ws = _workspace(q, _entry("cross_attention_workspace")(B, Nq, Nk, Hq, Hkv, D, dt), ws)
    _call(q, "cross_attention", *_strides(q, qs, "q"), *_strides(k, ks, "k"), *_strides(v, ks, "v"), dt, B, Nq, Nk,
          Hq, Hkv, D, scale, _ptr(k_len), _ptr(k_mask), mask_ld, *po, wp, wn)
    return out
