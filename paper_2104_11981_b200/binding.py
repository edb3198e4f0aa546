"""Binding of libdecentlam.so: argument marshalling only (ctypes; the training operators' calls, which have up to 22
arguments, go through _calls, a C module that converts them in a tenth of the time).

Every function mirrors the C entry point of the same name (include/decentlam.h).  Tensors are
torch CUDA tensors used purely as device memory; only their data pointers, strides and the
current stream cross the boundary.  A non-zero status raises DecentlamError.  There is no
fallback: if the shared library is missing, importing this module fails.
"""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdecentlam.so")

RING, STATIC_EXP, ONE_PEER_EXP, COMPLETE, CSR_MH, CSR_WEIGHTS, SYM_EXP, MESH = range(8)
G_F32, G_BF16 = 0, 1
DSGD_ATC, DSGD_AWC = 0, 1
NORM_L2, NORM_MAX = 0, 1
MAX_NODES = 2048

STATUS = {0: "DLM_OK", -1: "DLM_ERR_NULL", -2: "DLM_ERR_SHAPE", -3: "DLM_ERR_ALIGN", -4: "DLM_ERR_ALIAS",
          -5: "DLM_ERR_HYPER", -6: "DLM_ERR_KIND", -7: "DLM_ERR_TOPOLOGY", -8: "DLM_ERR_UNSUPPORTED",
          -9: "DLM_ERR_CUDA", -10: "DLM_ERR_WORKSPACE"}


class DecentlamError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        msg = _lib.dlm_status_string(self.status).decode()
        super().__init__(f"{where}: {STATUS.get(self.status, self.status)} ({msg})")


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} not found: build it with `python -m paper_2104_11981_b200.build` "
                      "(there is no CPU fallback)")
_lib = ctypes.CDLL(LIB_PATH)

try:
    from . import _calls  # linked to the library above
except ImportError:  # built for another Python, or where its headers are missing: ctypes makes the same calls, 1 to 2 us slower
    _calls = _lib

_i32p = ctypes.POINTER(ctypes.c_int32)
_f32p = ctypes.POINTER(ctypes.c_float)
_vp = ctypes.c_void_p
_i64 = ctypes.c_int64
_int = ctypes.c_int
_flt = ctypes.c_float


class _held_int(ctypes.c_int):
    """An int parameter whose argument is held to its range instead of cut to 32 bits: too large stays too large."""

    @classmethod
    def from_param(cls, v):
        return _int(min(max(v, -(1 << 31)), (1 << 31) - 1))


_lib.dlm_status_string.argtypes = [_int]
_lib.dlm_status_string.restype = ctypes.c_char_p
_lib.topology_build.argtypes = [_int, _int, _vp, _vp, _vp, ctypes.POINTER(_vp)]
_lib.topology_build_periodic.argtypes = [_int, _int, _int, _vp, _vp, _vp, ctypes.POINTER(_vp)]
_lib.topology_period.argtypes = [_vp, ctypes.POINTER(_int)]
_lib.topology_nodes.argtypes = [_vp, ctypes.POINTER(_int)]
for _name in ("topology_tables_host", "topology_tables_device"):
    getattr(_lib, _name).argtypes = [_vp, _int, ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                     ctypes.POINTER(_i64)]
_lib.topology_destroy.argtypes = [_vp]
for _name in ("decentlam_step", "dmsgd_step"):
    getattr(_lib, _name).argtypes = [_vp, _i64, _int, _i64, _i64, _vp, _vp, _vp, _int, _i64, _flt, _flt, _vp]
_lib.decentlam_step_host_gradients.argtypes = [_vp, _i64, _int, _i64, _i64, _vp, _vp, _vp, _int, _i64, _vp, _i64, _flt,
                                               _flt, _vp]
_lib.dsgd_step.argtypes = [_vp, _i64, _int, _i64, _i64, _vp, _vp, _int, _i64, _flt, _int, _vp]
_lib.topology_shard.argtypes = [_vp, _int, _int, ctypes.POINTER(_vp)]
_lib.topology_shard_destroy.argtypes = [_vp]
_lib.topology_shard_rows.argtypes = [_vp, ctypes.POINTER(_int), ctypes.POINTER(_int), ctypes.POINTER(_int)]
_lib.topology_halo.argtypes = [_vp, _int, ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_int)]
_lib.topology_halo_sends.argtypes = [_vp, _int, _int, ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_int)]
_lib.decentlam_step_sharded.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _int, _i64, _vp, _i64, _vp, _i64, _flt, _flt,
                                        _vp]
_lib.dmsgd_local_sharded.argtypes = [_vp, _i64, _i64, _vp, _vp, _vp, _int, _i64, _flt, _flt, _vp]
_lib.partial_average_sharded.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp]
_lib.pmsgd_step.argtypes = [_int, _i64, _i64, _vp, _vp, _vp, _int, _i64, _flt, _flt, _vp]
_lib.lsq_grad_workspace_bytes.argtypes = [_int, _int, _int]
_lib.lsq_grad_workspace_bytes.restype = _i64
_lib.lsq_grad.argtypes = [_int, _int, _int, _vp, _vp, _vp, _vp, _flt, _vp, _i64, _vp]
_lib.lsq_grad_static.argtypes = [_int, _int, _int, _vp, _vp, _vp, _vp, _flt, _vp]
_lib.lsq_gram_build.argtypes = [_int, _int, _int, _vp, _vp, _flt, _vp, _vp, _vp]
_lib.lsq_grad_gram.argtypes = [_int, _int, _vp, _vp, _vp, _vp, _vp]
_lib.gradients_build.argtypes = [_int, _int, ctypes.POINTER(_i64), ctypes.POINTER(_int), ctypes.POINTER(_vp),
                                 ctypes.POINTER(_i64), ctypes.POINTER(_vp)]
_lib.gradients_layout.argtypes = [_vp, ctypes.POINTER(ctypes.POINTER(_i64)), ctypes.POINTER(_i64)]
_lib.gradients_destroy.argtypes = [_vp]
_lib.gradient_norm.argtypes = [_vp, _held_int, _vp, _vp]
_lib.gradient_clip.argtypes = [_vp, _held_int, _flt, _vp, _vp, _held_int, _i64, _vp]
_lib.layer_norm.argtypes = [_held_int, _i64, _i64, _vp, _held_int, _i64, _vp, _i64, _vp, _i64, _flt, _vp, _i64, _vp, _vp, _vp]
_lib.layer_norm_grad_workspace_bytes.argtypes = [_held_int, _i64, _i64]
_lib.layer_norm_grad_workspace_bytes.restype = _i64
_lib.layer_norm_grad.argtypes = [_held_int, _i64, _i64, _vp, _held_int, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _i64, _vp,
                                 _i64, _held_int, _vp, _i64, _vp]
_lib.policy_loss_workspace_bytes.argtypes = [_held_int, _i64, _i64]
_lib.policy_loss_workspace_bytes.restype = _i64
_lib.policy_loss_grad.argtypes = [_held_int, _i64, _i64, _vp, _held_int, _i64, _vp, _vp, _vp, _vp, _vp, _flt, _flt, _flt, _vp, _vp, _vp,
                                  _i64, _vp, _i64, _vp]
_lib.dlm_launch_count.argtypes = []
_lib.dlm_launch_count.restype = _i64
_lib.dlm_kernel_error.argtypes = [ctypes.POINTER(_int)]
_lib.dlm_set_tuning.argtypes = [_int, _int]

EXPORTS = ["dlm_status_string", "topology_build", "topology_build_periodic", "topology_period", "topology_nodes", "topology_tables_host",
           "topology_tables_device", "topology_destroy", "decentlam_step", "decentlam_step_host_gradients", "dmsgd_step", "dsgd_step", "pmsgd_step",
           "topology_shard", "topology_shard_destroy", "topology_shard_rows", "topology_halo", "topology_halo_sends",
           "decentlam_step_sharded", "dmsgd_local_sharded", "partial_average_sharded",
           "lsq_grad_workspace_bytes", "lsq_grad", "lsq_grad_static", "lsq_gram_build", "lsq_grad_gram",
           "gradients_build", "gradients_layout", "gradients_destroy", "gradient_norm", "gradient_clip", "layer_norm",
           "layer_norm_grad_workspace_bytes", "layer_norm_grad", "policy_loss_workspace_bytes", "policy_loss_grad", "dlm_launch_count", "dlm_kernel_error", "dlm_set_tuning"]


def _check(rc, where):
    if rc != 0:
        raise DecentlamError(rc, where)


def raw():
    """The ctypes library object (for tests that pass deliberately bad arguments)."""
    return _lib


class Topology:
    """Owner of a dlm_topology handle."""

    def __init__(self, handle):
        self.handle = handle

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def destroy(self):
        if getattr(self, "handle", None):
            _lib.topology_destroy(self.handle)
            self.handle = None

    @property
    def period(self):
        v = _int()
        _check(_lib.topology_period(self.handle, ctypes.byref(v)), "topology_period")
        return v.value

    @property
    def n(self):
        v = _int()
        _check(_lib.topology_nodes(self.handle, ctypes.byref(v)), "topology_nodes")
        return v.value

    def tables_host(self, slot=0):
        """(rowptr int32[n+1], col int32[nnz], val float32[nnz]) copies of one slot's CSR tables."""
        import numpy as np
        rp, cp, vp, nnz = _vp(), _vp(), _vp(), _i64()
        _check(_lib.topology_tables_host(self.handle, slot, ctypes.byref(rp), ctypes.byref(cp), ctypes.byref(vp),
                                         ctypes.byref(nnz)), "topology_tables_host")
        n, z = self.n, nnz.value
        rowptr = np.ctypeslib.as_array(ctypes.cast(rp, _i32p), shape=(n + 1,)).copy()
        col = np.ctypeslib.as_array(ctypes.cast(cp, _i32p), shape=(z,)).copy()
        val = np.ctypeslib.as_array(ctypes.cast(vp, _f32p), shape=(z,)).copy()
        return rowptr, col, val

    def tables_device(self, slot=0):
        """Raw device addresses (rowptr, col, val) and nnz of one slot."""
        rp, cp, vp, nnz = _vp(), _vp(), _vp(), _i64()
        _check(_lib.topology_tables_device(self.handle, slot, ctypes.byref(rp), ctypes.byref(cp), ctypes.byref(vp),
                                           ctypes.byref(nnz)), "topology_tables_device")
        return rp.value, cp.value, vp.value, nnz.value


def topology_build(kind, n, rowptr=None, col=None, val=None):
    import numpy as np

    def ptr(a, dt):
        if a is None:
            return None, None
        a = np.ascontiguousarray(a, dtype=dt)
        return a, a.ctypes.data_as(_vp)

    keep_r, pr = ptr(rowptr, np.int32)
    keep_c, pc = ptr(col, np.int32)
    keep_v, pv = ptr(val, np.float32)
    out = _vp()
    _check(_lib.topology_build(kind, n, pr, pc, pv, ctypes.byref(out)), "topology_build")
    return Topology(out)


def topology_build_periodic(kind, n, period, rowptr, col, val=None):
    """Time-varying topology: concatenated CSR of `period` slots (rowptr has period * n + 1 entries)."""
    import numpy as np
    rowptr = np.ascontiguousarray(rowptr, dtype=np.int32)
    col = np.ascontiguousarray(col, dtype=np.int32)
    pv = None
    if val is not None:
        val = np.ascontiguousarray(val, dtype=np.float32)
        pv = val.ctypes.data_as(_vp)
    out = _vp()
    _check(_lib.topology_build_periodic(kind, n, period, rowptr.ctypes.data_as(_vp), col.ctypes.data_as(_vp), pv,
                                        ctypes.byref(out)), "topology_build_periodic")
    return Topology(out)


def _stream_ptr(stream):
    if stream is not None:
        return stream.cuda_stream
    import torch
    # the raw handle of the current stream: building a torch.cuda.Stream object for it costs 3.5 us a call
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _state_args(x, m, g):
    import torch
    assert x.is_cuda and m.is_cuda and g.is_cuda, "device tensors required"
    assert x.dtype == torch.float32 and m.dtype == torch.float32
    assert x.dim() == 2 and m.shape == x.shape and g.shape == x.shape
    assert x.stride(1) == 1 and m.stride(1) == 1 and g.stride(1) == 1 and m.stride(0) == x.stride(0)
    if g.dtype == torch.float32:
        gd = G_F32
    elif g.dtype == torch.bfloat16:
        gd = G_BF16
    else:
        raise TypeError("g must be float32 or bfloat16")
    n, d = x.shape
    return n, d, x.stride(0), _vp(x.data_ptr()), _vp(m.data_ptr()), _vp(g.data_ptr()), gd, g.stride(0)


def decentlam_step(topo, k, x, m, g, beta, gamma, stream=None):
    n, d, ld, px, pm, pg, gd, ldg = _state_args(x, m, g)
    _check(_lib.decentlam_step(topo.handle, k, n, d, ld, px, pm, pg, gd, ldg, beta, gamma, _stream_ptr(stream)),
           "decentlam_step")


def decentlam_step_host_gradients(topo, k, x, m, g_host, staging, chunk_cols, beta, gamma, stream=None):
    """decentlam_step with g in (pinned) host memory: chunked copy overlapped with the update.
    staging: device tensor of g's dtype with at least 2 * n * chunk_cols elements."""
    import torch
    assert not g_host.is_cuda and g_host.dim() == 2 and g_host.stride(1) == 1 and g_host.shape == x.shape
    assert x.is_cuda and m.is_cuda and staging.is_cuda and staging.dtype == g_host.dtype
    n, d = x.shape
    assert staging.numel() >= 2 * n * chunk_cols and m.stride(0) == x.stride(0)
    gd = G_F32 if g_host.dtype == torch.float32 else G_BF16
    _check(_lib.decentlam_step_host_gradients(topo.handle, k, n, d, x.stride(0), _vp(x.data_ptr()), _vp(m.data_ptr()),
                                              _vp(g_host.data_ptr()), gd, g_host.stride(0), _vp(staging.data_ptr()),
                                              chunk_cols, beta, gamma, _stream_ptr(stream)),
           "decentlam_step_host_gradients")


def dmsgd_step(topo, k, x, m, g, beta, gamma, stream=None):
    n, d, ld, px, pm, pg, gd, ldg = _state_args(x, m, g)
    _check(_lib.dmsgd_step(topo.handle, k, n, d, ld, px, pm, pg, gd, ldg, beta, gamma, _stream_ptr(stream)),
           "dmsgd_step")


def dsgd_step(topo, k, x, g, gamma, variant=DSGD_ATC, stream=None):
    import torch
    assert x.is_cuda and g.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and g.shape == x.shape
    assert x.stride(1) == 1 and g.stride(1) == 1
    gd = G_F32 if g.dtype == torch.float32 else G_BF16 if g.dtype == torch.bfloat16 else None
    if gd is None:
        raise TypeError("g must be float32 or bfloat16")
    n, d = x.shape
    _check(_lib.dsgd_step(topo.handle, k, n, d, x.stride(0), _vp(x.data_ptr()), _vp(g.data_ptr()), gd, g.stride(0),
                          gamma, variant, _stream_ptr(stream)), "dsgd_step")


class Shard:
    """Owner of a dlm_shard handle: one rank's share of a topology in a row-sharded run."""

    def __init__(self, handle, period):
        self.handle = handle
        self.period = period

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def destroy(self):
        if getattr(self, "handle", None):
            _lib.topology_shard_destroy(self.handle)
            self.handle = None

    @property
    def rows(self):
        """(row_begin, row_end, max_halo)."""
        lo, hi, mh = _int(), _int(), _int()
        _check(_lib.topology_shard_rows(self.handle, ctypes.byref(lo), ctypes.byref(hi), ctypes.byref(mh)),
               "topology_shard_rows")
        return lo.value, hi.value, mh.value

    @staticmethod
    def _pair(pa, pb, count):
        import numpy as np
        if count == 0:
            return np.zeros(0, np.int32), np.zeros(0, np.int32)
        a = np.ctypeslib.as_array(ctypes.cast(pa, _i32p), shape=(count,)).copy()
        b = np.ctypeslib.as_array(ctypes.cast(pb, _i32p), shape=(count,)).copy()
        return a, b

    def halo(self, slot):
        """(rows, owners): the remote rows this rank receives in `slot` (ascending global indices; rows[t]
        goes to row t of the halo buffers) and the rank owning each."""
        pr, po, c = _vp(), _vp(), _int()
        _check(_lib.topology_halo(self.handle, slot, ctypes.byref(pr), ctypes.byref(po), ctypes.byref(c)), "topology_halo")
        return self._pair(pr, po, c.value)

    def sends(self, slot, peer):
        """(rows, dst_slots): own rows (global indices) that `peer` needs in `slot`, and the halo row of
        the peer each one lands in."""
        pr, pd, c = _vp(), _vp(), _int()
        _check(_lib.topology_halo_sends(self.handle, slot, peer, ctypes.byref(pr), ctypes.byref(pd), ctypes.byref(c)),
               "topology_halo_sends")
        return self._pair(pr, pd, c.value)


def topology_shard(topo, rank, ranks):
    out = _vp()
    _check(_lib.topology_shard(topo.handle, rank, ranks, ctypes.byref(out)), "topology_shard")
    return Shard(out, topo.period)


def _halo_ptr(t):
    return (_vp(t.data_ptr()), t.stride(0)) if t is not None and t.numel() > 0 else (None, 0)


def decentlam_step_sharded(shard, k, x, m, g, halo_x, halo_g, beta, gamma, stream=None):
    """DecentLaM step of one rank: x, m, g are the rank's own rows [n_loc, d]; halo_x, halo_g [halo, d] hold
    the remote neighbours' rows in the order of shard.halo(k % period) (None when the halo is empty)."""
    n, d, ld, px, pm, pg, gd, ldg = _state_args(x, m, g)
    (phx, ldhx), (phg, ldhg) = _halo_ptr(halo_x), _halo_ptr(halo_g)
    _check(_lib.decentlam_step_sharded(shard.handle, k, d, ld, px, pm, pg, gd, ldg, phx, ldhx, phg, ldhg, beta, gamma,
                                       _stream_ptr(stream)), "decentlam_step_sharded")


def dmsgd_local_sharded(shard, x, m, g, beta, gamma, stream=None):
    """First half of a sharded DmSGD step on the rank's own rows: m <- beta m + g, x <- x - gamma m."""
    n, d, ld, px, pm, pg, gd, ldg = _state_args(x, m, g)
    _check(_lib.dmsgd_local_sharded(shard.handle, d, ld, px, pm, pg, gd, ldg, beta, gamma, _stream_ptr(stream)),
           "dmsgd_local_sharded")


def partial_average_sharded(shard, k, x, halo_x, stream=None):
    """Second half: x_i <- x_i + sum_{j != i} w_ij (x_j - x_i) over own rows, remote rows from halo_x."""
    import torch
    assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
    n, d = x.shape
    phx, ldhx = _halo_ptr(halo_x)
    _check(_lib.partial_average_sharded(shard.handle, k, d, x.stride(0), _vp(x.data_ptr()), phx, ldhx,
                                        _stream_ptr(stream)), "partial_average_sharded")


def pmsgd_step(x, m, g, beta, gamma, stream=None):
    n, d, ld, px, pm, pg, gd, ldg = _state_args(x, m, g)
    _check(_lib.pmsgd_step(n, d, ld, px, pm, pg, gd, ldg, beta, gamma, _stream_ptr(stream)), "pmsgd_step")


def lsq_grad_workspace_bytes(n, p, q):
    v = _lib.lsq_grad_workspace_bytes(n, p, q)
    if v < 0:
        raise DecentlamError(v, "lsq_grad_workspace_bytes")
    return int(v)


def lsq_grad(A, b, x, g, scale, workspace, stream=None):
    """g <- scale * A_i^T (A_i x_i - b_i).  A [n,p,q], b [n,p], x [n,q], g [n,q] contiguous fp32 device
    tensors; workspace: uint8 device tensor of at least lsq_grad_workspace_bytes(n, p, q) bytes."""
    n, p, q = A.shape
    assert A.is_contiguous() and b.is_contiguous() and x.is_contiguous() and g.is_contiguous()
    assert b.shape == (n, p) and x.shape == (n, q) and g.shape == (n, q)
    _check(_lib.lsq_grad(n, p, q, _vp(A.data_ptr()), _vp(b.data_ptr()), _vp(x.data_ptr()), _vp(g.data_ptr()),
                         scale, _vp(workspace.data_ptr()), workspace.numel() * workspace.element_size(),
                         _stream_ptr(stream)), "lsq_grad")


LSQ_STATIC_SCRATCH_BYTES = 4 << 20


def lsq_grad_static(A, b, x, g, scale, stream=None):
    """lsq_grad for callers that cannot allocate device scratch: same arguments minus the
    workspace, same result.  The partial sums go to a fixed 4 MiB array inside the library, shared
    by all calls, so calls must not overlap on the GPU; problems whose partial sums do not fit
    raise DecentlamError(DLM_ERR_WORKSPACE)."""
    n, p, q = A.shape
    assert A.is_contiguous() and b.is_contiguous() and x.is_contiguous() and g.is_contiguous()
    assert b.shape == (n, p) and x.shape == (n, q) and g.shape == (n, q)
    _check(_lib.lsq_grad_static(n, p, q, _vp(A.data_ptr()), _vp(b.data_ptr()), _vp(x.data_ptr()),
                                _vp(g.data_ptr()), scale, _stream_ptr(stream)), "lsq_grad_static")


def lsq_gram_build(A, b, scale, H, c, stream=None):
    """H <- scale * A_i^T A_i [n,q,q], c <- scale * A_i^T b_i [n,q] (contiguous fp32 device tensors)."""
    n, p, q = A.shape
    assert A.is_contiguous() and b.is_contiguous() and H.is_contiguous() and c.is_contiguous()
    assert b.shape == (n, p) and H.shape == (n, q, q) and c.shape == (n, q)
    _check(_lib.lsq_gram_build(n, p, q, _vp(A.data_ptr()), _vp(b.data_ptr()), scale, _vp(H.data_ptr()),
                               _vp(c.data_ptr()), _stream_ptr(stream)), "lsq_gram_build")


def lsq_grad_gram(H, c, x, g, stream=None):
    """g <- H_i x_i - c_i with H, c from lsq_gram_build; x, g [n,q] contiguous fp32 device tensors."""
    n, q, _ = H.shape
    assert H.is_contiguous() and c.is_contiguous() and x.is_contiguous() and g.is_contiguous()
    assert H.shape == (n, q, q) and c.shape == (n, q) and x.shape == (n, q) and g.shape == (n, q)
    _check(_lib.lsq_grad_gram(n, q, _vp(H.data_ptr()), _vp(c.data_ptr()), _vp(x.data_ptr()), _vp(g.data_ptr()),
                              _stream_ptr(stream)), "lsq_grad_gram")


_G_DTYPES = {}  # torch dtype -> DLM_G_*, filled on first use so that importing this module does not import torch


def _dtype(t):
    v = _G_DTYPES.get(t.dtype)
    if v is None:
        import torch
        _G_DTYPES.update({torch.float32: G_F32, torch.bfloat16: G_BF16})
        v = _G_DTYPES.get(t.dtype)
        if v is None:
            raise TypeError("float32 or bfloat16 expected")
    return v


class Gradients:
    """Owner of a dlm_gradients handle: n nodes' lists of parameter gradients.  Keeps the tensors alive."""

    def __init__(self, handle, n, tensors, keep):
        self.handle, self.n, self.keep = handle, n, keep
        self.address = handle.value
        po, c = ctypes.POINTER(_i64)(), _i64()
        _check(_lib.gradients_layout(handle, ctypes.byref(po), ctypes.byref(c)), "gradients_layout")
        self.offsets = [po[t] for t in range(tensors)]  # first column of each tensor in a stacked row
        self.columns = c.value                          # width of a stacked row

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def destroy(self):
        if getattr(self, "handle", None):
            _lib.gradients_destroy(self.handle)
            self.handle = self.address = None



def gradients_build(nodes, offsets=None):
    """nodes: one list of gradient tensors per node, the same sizes and types in every node, each contiguous, all on the
    current CUDA device.  offsets: first column of each tensor in a node's stacked row (None: packed without gaps)."""
    n, tensors = len(nodes), len(nodes[0]) if nodes else 0
    sizes, dtypes = [t.numel() for t in nodes[0]] if n else [], [_dtype(t) for t in nodes[0]] if n else []
    if tensors:
        import torch
        home = nodes[0][0].device
        assert home.type == "cuda" and home.index == torch.cuda.current_device(), "gradients on the current CUDA device are expected"
    data = (_vp * max(1, n * tensors))()
    for i, node in enumerate(nodes):
        assert len(node) == tensors, "every node has the same tensors"
        for t, g in enumerate(node):
            assert g.device == home, "gradients on one device are expected"
            assert g.is_contiguous() and g.numel() == sizes[t] and _dtype(g) == dtypes[t]
            data[i * tensors + t] = g.data_ptr()
    assert offsets is None or len(offsets) == tensors
    po = (_i64 * tensors)(*offsets) if offsets is not None else None
    out = _vp()
    _check(_lib.gradients_build(n, tensors, (_i64 * max(1, tensors))(*sizes), (_int * max(1, tensors))(*dtypes), data, po,
                                ctypes.byref(out)), "gradients_build")
    return Gradients(out, n, tensors, [list(node) for node in nodes])


def _check_norms(grads, norms):
    assert norms.is_cuda and _dtype(norms) == G_F32 and norms.is_contiguous() and norms.numel() == grads.n


def gradient_norm(grads, norms, kind=NORM_L2, stream=None):
    """norms[i] <- norm of node i's whole gradient (fp32 device tensor of n elements)."""
    _check_norms(grads, norms)
    _check(_calls.gradient_norm(grads.address, kind, norms.data_ptr(), _stream_ptr(stream)), "gradient_norm")


def gradient_clip(grads, max_norm, norms, g=None, kind=NORM_L2, stream=None):
    """Clip every node's gradient to max_norm by its own norm (written to norms): in place, or (g [n, >= columns],
    fp32 or bf16) gathered into the stacked rows that the update rules read, the tensors left as they are."""
    _check_norms(grads, norms)
    pg, gd, ldg = None, G_F32, 0
    if g is not None:
        n, width = g.shape
        assert g.is_cuda and n == grads.n and width >= grads.columns and (g.stride(1) == 1 or width == 1)
        pg, gd, ldg = g.data_ptr(), _dtype(g), g.stride(0) if n > 1 else width
    _check(_calls.gradient_clip(grads.address, kind, max_norm, norms.data_ptr(), pg, gd, ldg, _stream_ptr(stream)),
           "gradient_clip")


def _node_rows(t, shape, dtype):
    """Row stride of activations [n, rows, c] of this shape and type, whose nodes follow one another."""
    assert t.is_cuda and t.dtype == dtype and t.shape == shape, "a CUDA tensor of the same shape and type is expected"
    n, rows, c = shape
    if t.is_contiguous():
        return c
    s0, s1, s2 = t.stride()
    assert s2 == 1 or c == 1, "unit column stride expected"
    if rows == 1:
        return s0
    assert n == 1 or s0 == rows * s1, "the nodes' rows must be evenly spaced"
    return s1


def _node_vectors(t, n, c):
    """(pointer, row stride) of per-node vectors [n, c] with unit column stride, or of None."""
    if t is None:
        return None, 0
    assert t.is_cuda and t.shape == (n, c), "per-node vectors [n, c] are expected"
    s0, s1 = t.stride()
    assert s1 == 1 or c == 1, "unit column stride expected"
    return t.data_ptr(), s0 if n > 1 else c


def _per_row(t, count):
    """Pointer of a contiguous fp32 tensor of one value per row."""
    assert t.is_cuda and _dtype(t) == G_F32 and t.is_contiguous() and t.numel() == count, "fp32, one value per row"
    return t.data_ptr()


def layer_norm(x, weight, bias, eps, y, mean, rstd, stream=None):
    """y <- (x - mean) rstd weight + bias over the last axis of x [n, rows, c] (fp32 or bf16); weight, bias fp32 [n, c]
    (views of the stacked parameters, for instance; bias may be None); mean, rstd fp32 [n, rows] are written."""
    shape, dtype = x.shape, x.dtype
    n, rows, c = shape
    assert _dtype(weight) == G_F32 and (bias is None or _dtype(bias) == G_F32)
    (pw, ldw), (pb, ldb) = _node_vectors(weight, n, c), _node_vectors(bias, n, c)
    _check(_calls.layer_norm(n, rows, c, x.data_ptr(), _dtype(x), _node_rows(x, shape, dtype), pw, ldw, pb, ldb, eps,
                             y.data_ptr(), _node_rows(y, shape, dtype), _per_row(mean, n * rows), _per_row(rstd, n * rows),
                             _stream_ptr(stream)), "layer_norm")


def layer_norm_grad_workspace_bytes(n, rows, c):
    v = _lib.layer_norm_grad_workspace_bytes(n, rows, c)
    if v < 0:
        raise DecentlamError(v, "layer_norm_grad_workspace_bytes")
    return int(v)


def layer_norm_grad(x, dy, weight, mean, rstd, dx, dweight, dbias, workspace, stream=None):
    """Backward pass of layer_norm: dx of x's shape and type; dweight, dbias [n, c] fp32 or bf16 (views of the stacked
    gradient, for instance; dbias may be None) are overwritten; workspace: uint8 device tensor of at least
    layer_norm_grad_workspace_bytes(n, rows, c) bytes."""
    shape, dtype = x.shape, x.dtype
    n, rows, c = shape
    assert _dtype(weight) == G_F32 and (dbias is None or dbias.dtype == dweight.dtype)
    assert workspace.is_cuda and workspace.is_contiguous()
    pw, ldw = _node_vectors(weight, n, c)
    (pgw, ldgw), (pgb, ldgb) = _node_vectors(dweight, n, c), _node_vectors(dbias, n, c)
    _check(_calls.layer_norm_grad(n, rows, c, x.data_ptr(), _dtype(x), _node_rows(x, shape, dtype), dy.data_ptr(),
                                  _node_rows(dy, shape, dtype), pw, ldw, _per_row(mean, n * rows), _per_row(rstd, n * rows),
                                  dx.data_ptr(), _node_rows(dx, shape, dtype), pgw, ldgw, pgb, ldgb, _dtype(dweight),
                                  workspace.data_ptr(), workspace.nbytes, _stream_ptr(stream)), "layer_norm_grad")


def policy_loss_workspace_bytes(n, rows, vocab):
    v = _lib.policy_loss_workspace_bytes(n, rows, vocab)
    if v < 0:
        raise DecentlamError(v, "policy_loss_workspace_bytes")
    return int(v)


def policy_loss_grad(logits, tokens, weight, advantage, old_logp, ref_logp, clip_low, clip_high, kl_coef, loss, logp,
                     dlogits, workspace, stream=None):
    """Clipped policy loss with a KL term, and its gradient: logits [n, rows, vocab] fp32 or bf16; tokens int64, weight,
    advantage, old_logp, ref_logp (or None) fp32 [n, rows]; loss fp32 [n] and logp fp32 [n, rows] are written, and dlogits
    (of the logits' shape and type; None: no gradient; the logits themselves: in place).  workspace: uint8 device tensor
    of at least policy_loss_workspace_bytes(n, rows, vocab) bytes."""
    import torch
    shape, dtype = logits.shape, logits.dtype
    n, rows, vocab = shape
    count = n * rows
    assert tokens.is_cuda and tokens.dtype == torch.int64 and tokens.is_contiguous() and tokens.numel() == count
    assert workspace.is_cuda and workspace.is_contiguous()
    pd, ldd = (dlogits.data_ptr(), _node_rows(dlogits, shape, dtype)) if dlogits is not None else (None, 0)
    _check(_calls.policy_loss_grad(n, rows, vocab, logits.data_ptr(), _dtype(logits), _node_rows(logits, shape, dtype),
                                   tokens.data_ptr(), _per_row(weight, count), _per_row(advantage, count),
                                   _per_row(old_logp, count), _per_row(ref_logp, count) if ref_logp is not None else None,
                                   clip_low, clip_high, kl_coef, _per_row(loss, n), _per_row(logp, count), pd, ldd,
                                   workspace.data_ptr(), workspace.nbytes, _stream_ptr(stream)), "policy_loss_grad")


def launch_count():
    return int(_lib.dlm_launch_count())


def kernel_error():
    v = _int()
    _check(_lib.dlm_kernel_error(ctypes.byref(v)), "dlm_kernel_error")
    return v.value


def set_tuning(knob, value):
    _check(_lib.dlm_set_tuning(knob, value), "dlm_set_tuning")
