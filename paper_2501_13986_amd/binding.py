"""ctypes binding of libcgtp.so: the functions of include/cgtp.h under the same names.

Argument marshalling only: torch tensors supply device memory (scratch too) and the current stream, every
step of the computation runs in the library's kernels.  There is no fallback: if the shared
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcgtp.so")

CGTP_F32, CGTP_F64 = 0, 1
CGTP_UVU, CGTP_UVW = 0, 1
CGTP_MUL_IR, CGTP_IR_MUL = 0, 1
K_TP_FWD, K_TP_BWD, K_CONV_FWD, K_CONV_BWD, K_CONV_FWD_ATOMIC, K_CONV_BWD_ATOMIC, K_TP_DBL_BWD = 0, 1, 2, 3, 4, 5, 6
K_CONV_DBL_FWD, K_CONV_DBL_BWD = 7, 8
ACT_NONE, ACT_SILU, ACT_GELU, ACT_SIGMOID, ACT_TANH = 0, 1, 2, 3, 4
CGTP_NORM_GATED = 2
STATUS = {0: "CGTP_OK", 1: "CGTP_EINVAL", 2: "CGTP_EUNSUPPORTED", 3: "CGTP_ECOMPILE", 4: "CGTP_ERUNTIME", 5: "CGTP_ENOMEM"}

EXPORTS = [
    "cgtp_plan_create", "cgtp_plan_create_ex", "cgtp_plan_destroy", "cgtp_plan_dim", "cgtp_plan_num_paths", "cgtp_plan_get_path",
    "cgtp_plan_path_nonzeros", "cgtp_plan_flops", "cgtp_plan_source", "cgtp_plan_kernel_info", "cgtp_plan_conv_kernel",
    "tp_forward", "tp_backward", "tp_double_backward", "conv_forward", "conv_forward_static", "conv_backward", "conv_forward_perm", "conv_backward_perm", "conv_double_backward", "conv_double_backward_ws",
    "cgtp_conv_double_workspace_bytes", "conv_forward_atomic", "conv_backward_atomic",
    "cgtp_csr_from_coo", "cgtp_csr_from_coo_async", "cgtp_csr_workspace_bytes", "cgtp_last_error", "cgtp_check_code_object",
    "gated_forward", "gated_backward", "cgtp_gated_workspace_bytes",
    "cgtp_norm_create", "cgtp_norm_destroy", "cgtp_norm_dim", "cgtp_norm_kernel", "cgtp_norm_workspace_bytes", "norm_forward", "norm_backward",
    "grouped_forward", "grouped_backward", "cgtp_grouped_workspace_bytes", "orthogonalise", "cgtp_orthogonalise_workspace_bytes",
]


class CgtpError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class cgtp_options(C.Structure):
    _fields_ = [("struct_size", C.c_int32), ("kahan_conv", C.c_int32)]


class cgtp_path(C.Structure):
    _fields_ = [("ix", C.c_int32), ("iy", C.c_int32), ("iz", C.c_int32), ("mode", C.c_int32), ("coeff", C.c_double)]


_lib = None


def lib() -> C.CDLL:
    """Loads libcgtp.so (built by paper_2501_13986_amd.build) and declares the prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2501_13986_amd.build`")
    L = C.CDLL(LIB_PATH)
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
    L.cgtp_last_error.restype = C.c_char_p
    L.cgtp_check_code_object.argtypes = [C.c_char_p, C.c_char_p, C.c_size_t]
    L.cgtp_plan_create.argtypes = [C.c_char_p, C.c_char_p, C.c_char_p, C.POINTER(cgtp_path), i32, i32, i32, i32, i32, C.c_uint32,
                                   C.POINTER(vp)]
    L.cgtp_plan_create_ex.argtypes = [C.c_char_p, C.c_char_p, C.c_char_p, C.POINTER(cgtp_path), i32, i32, i32, i32, i32, C.c_uint32,
                                      C.POINTER(cgtp_options), C.POINTER(vp)]
    L.cgtp_plan_destroy.argtypes = [vp]
    L.cgtp_plan_dim.argtypes = [vp, i32]
    L.cgtp_plan_dim.restype = i64
    L.cgtp_plan_num_paths.argtypes = [vp]
    L.cgtp_plan_get_path.argtypes = [vp, i32, C.POINTER(cgtp_path), C.POINTER(i32), C.POINTER(i32), C.POINTER(i64)]
    L.cgtp_plan_path_nonzeros.argtypes = [vp, i32, i32, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32), C.POINTER(C.c_double)]
    L.cgtp_plan_flops.argtypes = [vp, i32]
    L.cgtp_plan_flops.restype = i64
    L.cgtp_plan_source.argtypes = [vp, i32]
    L.cgtp_plan_source.restype = C.c_char_p
    L.cgtp_plan_kernel_info.argtypes = [vp, i32, C.POINTER(i32)]
    L.cgtp_plan_conv_kernel.argtypes = [vp, i32, i64, i64]
    L.cgtp_plan_conv_kernel.restype = C.c_char_p
    L.tp_forward.argtypes = [vp, vp, vp, vp, vp, i64, vp]
    L.tp_backward.argtypes = [vp] + [vp] * 7 + [i64, vp]
    L.tp_double_backward.argtypes = [vp] + [vp] * 11 + [i64, vp]
    L.conv_forward.argtypes = [vp, vp, vp, vp, vp, i64, i64, vp, vp, vp]
    L.conv_forward_static.argtypes = [vp, vp, vp, vp, vp, i64, i64, vp, vp, vp]
    L.conv_backward.argtypes = [vp] + [vp] * 7 + [i64, i64, vp, vp, vp, vp, vp]
    L.conv_forward_perm.argtypes = [vp, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp]
    L.conv_backward_perm.argtypes = [vp] + [vp] * 7 + [i64, i64, vp, vp, vp, vp, vp, vp]
    L.conv_double_backward.argtypes = [vp] + [vp] * 11 + [i64, i64, vp, vp, vp, vp, vp]
    L.conv_double_backward_ws.argtypes = [vp] + [vp] * 11 + [i64, i64, vp, vp, vp, vp, vp, C.c_size_t, vp]
    L.cgtp_conv_double_workspace_bytes.argtypes = [vp, i64, i64]
    L.cgtp_conv_double_workspace_bytes.restype = C.c_size_t
    L.conv_forward_atomic.argtypes = [vp, vp, vp, vp, vp, i64, i64, vp, vp, vp]
    L.conv_backward_atomic.argtypes = [vp] + [vp] * 7 + [i64, i64, vp, vp, vp]
    L.cgtp_csr_from_coo.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, vp, vp]
    L.cgtp_csr_workspace_bytes.argtypes = [i64, i64]
    L.cgtp_csr_workspace_bytes.restype = C.c_size_t
    L.cgtp_csr_from_coo_async.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
    L.gated_forward.argtypes = [vp] * 6 + [i64] * 5 + [i32, i32, vp]
    L.gated_backward.argtypes = [vp] * 11 + [i64] * 6 + [i32, i32, vp, C.c_size_t, vp]
    L.cgtp_gated_workspace_bytes.argtypes = [i64, i64, i64, i32]
    L.cgtp_gated_workspace_bytes.restype = C.c_size_t
    L.cgtp_norm_create.argtypes = [C.c_char_p, i32, i32, C.c_double, i32, i32, C.c_uint32, C.POINTER(vp)]
    L.cgtp_norm_destroy.argtypes = [vp]
    L.cgtp_norm_dim.argtypes = [vp, i32]
    L.cgtp_norm_dim.restype = i64
    L.cgtp_norm_kernel.argtypes = [vp, i32, i32]
    L.cgtp_norm_kernel.restype = C.c_char_p
    L.cgtp_norm_workspace_bytes.argtypes = [vp, i64, i64, i32, i32]
    L.cgtp_norm_workspace_bytes.restype = C.c_size_t
    L.norm_forward.argtypes = [vp] * 6 + [i64, i64, vp, vp, C.c_size_t, vp]
    L.norm_backward.argtypes = [vp] * 9 + [i64, i64, vp, vp, C.c_size_t, vp]
    L.grouped_forward.argtypes = [vp] * 4 + [i64] * 5 + [vp, vp, i64, i64, i32, vp]
    L.grouped_backward.argtypes = [vp] * 6 + [i64] * 5 + [vp, vp, i64, i64, i64, i32, vp, C.c_size_t, vp]
    L.cgtp_grouped_workspace_bytes.argtypes = [i64] * 5 + [i32]
    L.cgtp_grouped_workspace_bytes.restype = C.c_size_t
    L.orthogonalise.argtypes = [vp, vp] + [i64] * 7 + [C.POINTER(C.c_double), i32, C.c_double, i32, vp, C.c_size_t, vp]
    L.cgtp_orthogonalise_workspace_bytes.argtypes = [i64] * 3 + [i32]
    L.cgtp_orthogonalise_workspace_bytes.restype = C.c_size_t
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        raise CgtpError(status, lib().cgtp_last_error().decode())


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


_raw_stream = None


def _stream() -> int:
    """The current stream of the current device.  Asked for by its handle: torch.cuda.current_stream() builds a Stream
    object, 2.8 of the 7.7 us that the host needs for a small convolution (the handle 0.2; the C call itself 4.2)."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()   # initialises, or raises without a GPU
        handle, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        _raw_stream = lambda: handle(device())  # noqa: E731
    return _raw_stream()


class Plan:
    """Owns a cgtp_plan.  device=-1: plan + source only; -2: also compile into the kernel cache;
    >= 0: compile and load on that GPU."""

    def __init__(self, irreps_x: str, irreps_y: str, irreps_z: str, paths: Optional[Sequence[Tuple]] = None,
                 mode: int = CGTP_UVU, shared_weights: bool = False, dtype: int = CGTP_F32, device: int = 0,
                 kahan_conv: bool = False, flags: int = CGTP_MUL_IR):
        L = lib()
        arr, n = None, 0
        if paths:
            n = len(paths)
            arr = (cgtp_path * n)()
            for t, q in enumerate(paths):
                q = tuple(q)
                arr[t] = cgtp_path(q[0], q[1], q[2], q[3] if len(q) > 3 else mode, q[4] if len(q) > 4 else 1.0)
        h = C.c_void_p()
        if kahan_conv:
            opt = cgtp_options(C.sizeof(cgtp_options), 1)
            _check(L.cgtp_plan_create_ex(irreps_x.encode(), irreps_y.encode(), irreps_z.encode(), arr, n, mode,
                                         int(shared_weights), dtype, device, flags, C.byref(opt), C.byref(h)))
        else:
            _check(L.cgtp_plan_create(irreps_x.encode(), irreps_y.encode(), irreps_z.encode(), arr, n, mode,
                                      int(shared_weights), dtype, device, flags, C.byref(h)))
        self._h = h
        self.dtype = dtype
        self.dim_x, self.dim_y, self.dim_z, self.n_w = (L.cgtp_plan_dim(h, t) for t in range(4))
        self.num_paths = L.cgtp_plan_num_paths(h)

    def close(self):
        if getattr(self, "_h", None):
            lib().cgtp_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:      # interpreter shutdown: module globals may already be gone
            pass

    def path(self, p: int):
        q, l = cgtp_path(), (C.c_int32 * 3)()
        nnz, woff = C.c_int32(), C.c_int64()
        _check(lib().cgtp_plan_get_path(self._h, p, C.byref(q), l, C.byref(nnz), C.byref(woff)))
        return dict(ix=q.ix, iy=q.iy, iz=q.iz, mode=q.mode, coeff=q.coeff, l=tuple(l), nnz=nnz.value, w_offset=woff.value)

    def path_nonzeros(self, p: int):
        n = lib().cgtp_plan_path_nonzeros(self._h, p, 0, None, None, None, None)
        i, j, k, v = (C.c_int32 * n)(), (C.c_int32 * n)(), (C.c_int32 * n)(), (C.c_double * n)()
        lib().cgtp_plan_path_nonzeros(self._h, p, n, i, j, k, v)
        return [(i[t], j[t], k[t], v[t]) for t in range(n)]

    def flops(self, which: int) -> int:
        return lib().cgtp_plan_flops(self._h, which)

    def source(self, kernel: int) -> Optional[str]:
        s = lib().cgtp_plan_source(self._h, kernel)
        return None if s is None else s.decode()

    def kernel_info(self, kernel: int):
        a = (C.c_int32 * 6)()
        _check(lib().cgtp_plan_kernel_info(self._h, kernel, a))
        return dict(vgprs=a[0], sgprs=a[1], lds=a[2], scratch=a[3], wg=a[4], blocks_per_cu=a[5])

    def conv_kernel(self, kernel: int, V: int, E: int) -> Optional[str]:
        """Name of the kernel that a convolution of this size runs (kernel: K_CONV_FWD, K_CONV_BWD, K_CONV_DBL_BWD)."""
        s = lib().cgtp_plan_conv_kernel(self._h, kernel, V, E)
        return None if s is None else s.decode()


def tp_forward(plan: Plan, x, y, W, z, B: Optional[int] = None):
    _check(lib().tp_forward(plan._h, _ptr(x), _ptr(y), _ptr(W), _ptr(z), x.shape[0] if B is None else B, _stream()))
    return z


def tp_backward(plan: Plan, x, y, W, gz, gx, gy, gW, B: Optional[int] = None):
    _check(lib().tp_backward(plan._h, _ptr(x), _ptr(y), _ptr(W), _ptr(gz), _ptr(gx), _ptr(gy), _ptr(gW),
                             x.shape[0] if B is None else B, _stream()))
    return gx, gy, gW


def tp_double_backward(plan: Plan, x, y, W, gz, La, Lb, LC, Lx, Ly, LW, Lgz, B: Optional[int] = None):
    _check(lib().tp_double_backward(plan._h, _ptr(x), _ptr(y), _ptr(W), _ptr(gz), _ptr(La), _ptr(Lb), _ptr(LC), _ptr(Lx),
                                    _ptr(Ly), _ptr(LW), _ptr(Lgz), x.shape[0] if B is None else B, _stream()))
    return Lx, Ly, LW, Lgz


def conv_forward(plan: Plan, x_nodes, y_edges, W_edges, z_nodes, row_ptr, col):
    V, E = z_nodes.shape[0], y_edges.shape[0]
    _check(lib().conv_forward(plan._h, _ptr(x_nodes), _ptr(y_edges), _ptr(W_edges), _ptr(z_nodes), V, E,
                              _ptr(row_ptr), _ptr(col), _stream()))
    return z_nodes


def conv_forward_static(plan: Plan, x_nodes, y_edges, W_edges, z_nodes, row_ptr, col):
    V, E = z_nodes.shape[0], y_edges.shape[0]
    _check(lib().conv_forward_static(plan._h, _ptr(x_nodes), _ptr(y_edges), _ptr(W_edges), _ptr(z_nodes), V, E,
                                     _ptr(row_ptr), _ptr(col), _stream()))
    return z_nodes


def conv_backward(plan: Plan, x_nodes, y_edges, W_edges, gz_nodes, gx_nodes, gy_edges, gW_edges, row_ptr, col,
                  t_row_ptr, t_perm):
    V, E = x_nodes.shape[0], y_edges.shape[0]
    _check(lib().conv_backward(plan._h, _ptr(x_nodes), _ptr(y_edges), _ptr(W_edges), _ptr(gz_nodes), _ptr(gx_nodes),
                               _ptr(gy_edges), _ptr(gW_edges), V, E, _ptr(row_ptr), _ptr(col), _ptr(t_row_ptr),
                               _ptr(t_perm), _stream()))
    return gx_nodes, gy_edges, gW_edges


def conv_forward_perm(plan: Plan, x_nodes, y_edges, W_edges, z_nodes, row_ptr, col, edge_perm):
    V, E = z_nodes.shape[0], y_edges.shape[0]
    _check(lib().conv_forward_perm(plan._h, _ptr(x_nodes), _ptr(y_edges), _ptr(W_edges), _ptr(z_nodes), V, E,
                                   _ptr(row_ptr), _ptr(col), _ptr(edge_perm), _stream()))
    return z_nodes


def conv_backward_perm(plan: Plan, x_nodes, y_edges, W_edges, gz_nodes, gx_nodes, gy_edges, gW_edges, row_ptr, col,
                       t_row_ptr, t_perm, edge_perm):
    V, E = x_nodes.shape[0], y_edges.shape[0]
    _check(lib().conv_backward_perm(plan._h, _ptr(x_nodes), _ptr(y_edges), _ptr(W_edges), _ptr(gz_nodes), _ptr(gx_nodes),
                                    _ptr(gy_edges), _ptr(gW_edges), V, E, _ptr(row_ptr), _ptr(col), _ptr(t_row_ptr),
                                    _ptr(t_perm), _ptr(edge_perm), _stream()))
    return gx_nodes, gy_edges, gW_edges


def conv_double_backward(plan: Plan, x_nodes, y_edges, W_edges, gz_nodes, La_nodes, Lb_edges, LC_edges, Lx_nodes, Ly_edges,
                         LW_edges, Lgz_nodes, row_ptr, col, t_row_ptr, t_perm):
    """The memory of the one walk is torch's for the time of the call: shared by all plans, given back to its allocator on the
    current stream, part of the graph's pool under torch.cuda.graph.  Where torch has none left the pass goes in two walks, whose
    sums are in another order."""
    V, E = x_nodes.shape[0], y_edges.shape[0]
    L, scratch = lib(), None
    n = L.cgtp_conv_double_workspace_bytes(plan._h, V, E) if E >= 1024 else 0   # the rows of fewer edges fit the plan's workspace
    if n:
        import torch
        try:
            scratch = torch.empty(n, dtype=torch.uint8, device=x_nodes.device)
        except torch.cuda.OutOfMemoryError:
            n = 0
    _check(L.conv_double_backward_ws(plan._h, _ptr(x_nodes), _ptr(y_edges), _ptr(W_edges), _ptr(gz_nodes), _ptr(La_nodes),
                                     _ptr(Lb_edges), _ptr(LC_edges), _ptr(Lx_nodes), _ptr(Ly_edges), _ptr(LW_edges),
                                     _ptr(Lgz_nodes), V, E, _ptr(row_ptr), _ptr(col), _ptr(t_row_ptr), _ptr(t_perm),
                                     _ptr(scratch), n, _stream()))
    return Lx_nodes, Ly_edges, LW_edges, Lgz_nodes


def conv_forward_atomic(plan: Plan, x_nodes, y_edges, W_edges, z_nodes, recv, send):
    V, E = z_nodes.shape[0], y_edges.shape[0]
    _check(lib().conv_forward_atomic(plan._h, _ptr(x_nodes), _ptr(y_edges), _ptr(W_edges), _ptr(z_nodes), V, E,
                                     _ptr(recv), _ptr(send), _stream()))
    return z_nodes


def conv_backward_atomic(plan: Plan, x_nodes, y_edges, W_edges, gz_nodes, gx_nodes, gy_edges, gW_edges, recv, send):
    V, E = x_nodes.shape[0], y_edges.shape[0]
    _check(lib().conv_backward_atomic(plan._h, _ptr(x_nodes), _ptr(y_edges), _ptr(W_edges), _ptr(gz_nodes), _ptr(gx_nodes),
                                      _ptr(gy_edges), _ptr(gW_edges), V, E, _ptr(recv), _ptr(send), _stream()))
    return gx_nodes, gy_edges, gW_edges


def check_code_object(path: str) -> str:
    """The library's check of compiled code on a code object file: the first vector instruction placed where the
    execution mask is empty, or an empty string."""
    buf = C.create_string_buffer(256)
    _check(lib().cgtp_check_code_object(path.encode(), buf, 256))
    return buf.value.decode()


def cgtp_csr_from_coo(recv, send, V: int):
    """recv, send: int64 CUDA tensors [E].  Returns (row_ptr, col, perm, t_row_ptr, t_perm) on the same device."""
    import torch
    E = recv.shape[0]
    dev = recv.device
    row_ptr = torch.empty(V + 1, dtype=torch.int64, device=dev)
    t_row_ptr = torch.empty(V + 1, dtype=torch.int64, device=dev)
    col, perm, t_perm = (torch.empty(E, dtype=torch.int64, device=dev) for _ in range(3))
    _check(lib().cgtp_csr_from_coo(_ptr(recv), _ptr(send), E, V, _ptr(row_ptr), _ptr(col), _ptr(perm), _ptr(t_row_ptr),
                                   _ptr(t_perm), _stream()))
    return row_ptr, col, perm, t_row_ptr, t_perm


def cgtp_csr_workspace_bytes(E: int, V: int) -> int:
    return lib().cgtp_csr_workspace_bytes(E, V)


def cgtp_csr_from_coo_async(recv, send, V: int, out, workspace, bad_flag=None, transpose: bool = True):
    """Asynchronous variant on caller-owned buffers: out = (row_ptr, col, perm, t_row_ptr, t_perm) int64 CUDA tensors
    (t_row_ptr, t_perm ignored when transpose is False), workspace a uint8 CUDA tensor of at least
    cgtp_csr_workspace_bytes(E, V) bytes, bad_flag an optional int32 CUDA tensor [1].  Nothing is allocated or awaited."""
    row_ptr, col, perm, t_row_ptr, t_perm = out
    _check(lib().cgtp_csr_from_coo_async(_ptr(recv), _ptr(send), recv.shape[0], V, _ptr(row_ptr), _ptr(col), _ptr(perm),
                                         _ptr(t_row_ptr) if transpose else 0, _ptr(t_perm) if transpose else 0,
                                         _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(bad_flag), _stream()))
    return out


# ---- layer operators around the convolution ---------------------------------------------------------------------------

def _bad(msg: str):
    raise CgtpError(1, msg)


_torch = None


def _torch_module():
    """torch, without the cost of an import statement in every call (0.3 of the 8 us that the host needs for a small one)."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _operand(t, name: str, shape: Tuple, dtype, device: int, optional: bool = False) -> int:
    """Checks a contiguous operand and returns its address."""
    if t is None:
        return 0 if optional else _bad(f"{name} is missing")
    if t.shape != shape:
        _bad(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype or t.get_device() != device:
        _bad(f"{name}: {t.dtype} on {t.device}, expected {dtype} where x is")
    if not t.is_contiguous():
        _bad(f"{name} must be contiguous")
    return t.data_ptr()


def _row_operand(t, name: str, shape: Tuple, dtype, device: int) -> Tuple[int, int]:
    """The same for rows that may be columns of wider rows: address and elements from one row to the next."""
    if t is None:
        _bad(f"{name} is missing")
    if t.shape != shape:
        _bad(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype or t.get_device() != device:
        _bad(f"{name}: {t.dtype} on {t.device}, expected {dtype} where x is")
    ld, step = t.stride()
    if step != 1 and shape[1] > 1 and shape[0] > 0:
        _bad(f"{name}: the elements of a row must be neighbours")
    return t.data_ptr(), ld if shape[0] > 1 else shape[1]


def _type_and_device(x) -> Tuple[int, int]:
    """The kernels go to the current stream of the current device: data elsewhere is refused, after the other checks (device -1: not
    on a GPU)."""
    torch = _torch_module()
    if x is None:
        _bad("x is missing")
    if x.dtype == torch.float32:
        return CGTP_F32, x.get_device()
    if x.dtype == torch.float64:
        return CGTP_F64, x.get_device()
    _bad(f"float32 or float64 expected, got {x.dtype}")


def _stream_of(x, device: int) -> int:
    if device < 0 or _torch._C._cuda_getDevice() != device:
        current = f"cuda:{_torch._C._cuda_getDevice()}" if _torch.cuda.is_available() else "none"
        _bad(f"tensors are on {x.device}, the current device is {current}")
    return _stream()


def _scratch(n: int, like):
    """Workspace of a call: torch's, given back to its allocator on the current stream, part of the graph's pool under
    torch.cuda.graph."""
    return _torch.empty(n, dtype=_torch.uint8, device=like.device) if n else None


def gated_forward(x, Wg, Wu, out, bg=None, bu=None, act: int = ACT_SILU):
    """out = act(x Wg + bg) * (x Wu + bu).  x [rows, d_in], Wg, Wu [d_in, d_out], bg, bu [d_out] or None, out [rows, d_out]; x and
    out may be columns of wider rows.  out must not overlap an input."""
    dt, dev = _type_and_device(x)
    if x.dim() != 2 or Wg is None or Wg.dim() != 2:
        _bad("x and Wg must have two dimensions")
    (rows, k), n, ty = x.shape, Wg.shape[1], x.dtype
    px, ldx = _row_operand(x, "x", (rows, k), ty, dev)
    po, ldo = _row_operand(out, "out", (rows, n), ty, dev)
    w = (_operand(Wg, "Wg", (k, n), ty, dev), _operand(Wu, "Wu", (k, n), ty, dev), _operand(bg, "bg", (n,), ty, dev, True),
         _operand(bu, "bu", (n,), ty, dev, True))
    st = _stream_of(x, dev)
    _check(lib().gated_forward(px, *w, po, rows, k, n, ldx, ldo, act, dt, st))
    return out


def gated_backward(x, Wg, Wu, gout, gx, gWg, gWu, bg=None, bu=None, gbg=None, gbu=None, act: int = ACT_SILU):
    """Gradients of gated_forward given gout [rows, d_out]; gbg, gbu are given where bg, bu are.  x, gout and gx may be columns of
    wider rows.  No output may overlap an input."""
    dt, dev = _type_and_device(x)
    if x.dim() != 2 or Wg is None or Wg.dim() != 2:
        _bad("x and Wg must have two dimensions")
    (rows, k), n, ty = x.shape, Wg.shape[1], x.dtype
    px, ldx = _row_operand(x, "x", (rows, k), ty, dev)
    pg, ldg = _row_operand(gout, "gout", (rows, n), ty, dev)
    pgx, ldgx = _row_operand(gx, "gx", (rows, k), ty, dev)
    w = (_operand(Wg, "Wg", (k, n), ty, dev), _operand(Wu, "Wu", (k, n), ty, dev), _operand(bg, "bg", (n,), ty, dev, True),
         _operand(bu, "bu", (n,), ty, dev, True))
    g = (_operand(gWg, "gWg", (k, n), ty, dev), _operand(gWu, "gWu", (k, n), ty, dev), _operand(gbg, "gbg", (n,), ty, dev, True),
         _operand(gbu, "gbu", (n,), ty, dev, True))
    st = _stream_of(x, dev)
    L = lib()
    nb = L.cgtp_gated_workspace_bytes(rows, k, n, dt)
    ws = _scratch(nb, x)
    _check(L.gated_backward(px, *w, pg, pgx, *g, rows, k, n, ldx, ldg, ldgx, act, dt, _ptr(ws), nb, st))
    return gx, gWg, gWu, gbg, gbu


class Norm:
    """Owns a cgtp_norm: the group normalisation of rows of `irreps` with activation and gates (include/cgtp.h).  device as for
    Plan; flags: the layout."""

    def __init__(self, irreps: str, groups: int = 1, act: int = ACT_SILU, gated: bool = True, eps: float = 1e-5, dtype: int = CGTP_F32,
                 device: int = 0, flags: int = CGTP_MUL_IR):
        L, h = lib(), C.c_void_p()
        _check(L.cgtp_norm_create(irreps.encode(), groups, act, eps, dtype, device, flags | (CGTP_NORM_GATED if gated else 0), C.byref(h)))
        self._h, self.dtype, self.groups = h, dtype, groups
        self.dim_x, self.dim_y, self.n_w, self.n_b, self.n_stat = (L.cgtp_norm_dim(h, t) for t in range(5))

    def kernel(self, ptr: bool, backward: bool) -> str:
        """Name of the (first) kernel that a call runs; ptr: whether ptr is given."""
        return lib().cgtp_norm_kernel(self._h, ptr, backward).decode()

    def close(self):
        if getattr(self, "_h", None):
            lib().cgtp_norm_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:      # interpreter shutdown: module globals may already be gone
            pass


def _norm_operands(norm: Norm, x, weight, bias, stats, ptr):
    dt, dev = _type_and_device(x)
    if dt != norm.dtype:
        _bad(f"x is {x.dtype}, the normalisation was made for {'float64' if norm.dtype == CGTP_F64 else 'float32'}")
    if x.dim() != 2:
        _bad("x must have two dimensions")
    N, ty = x.shape[0], x.dtype
    S, pp, ps = N, 0, 0
    if ptr is not None:
        if ptr.dtype != _torch.int64 or ptr.dim() != 1 or ptr.shape[0] < 1 or not ptr.is_contiguous() or ptr.get_device() != dev:
            _bad("ptr: a contiguous int64 tensor [samples + 1] on the device of x")
        S, pp = ptr.shape[0] - 1, ptr.data_ptr()
    if stats is not None:
        if stats.numel() != S * norm.n_stat:
            _bad(f"stats: {stats.numel()} numbers, expected {S} * {norm.n_stat}")
        ps = _operand(stats, "stats", stats.shape, ty, dev)
    ops = (_operand(x, "x", (N, norm.dim_x), ty, dev), _operand(weight, "weight", (norm.n_w,), ty, dev),
           _operand(bias, "bias", (norm.n_b,), ty, dev, norm.n_b == 0))
    return N, S, pp, ops, ps, ty, dev


def norm_forward(norm: Norm, x, weight, bias, y, stats=None, ptr=None):
    """x [N, dim_x], weight [n_w], bias [n_b], y [N, dim_y], stats: samples * n_stat numbers, or None where no backward pass follows;
    ptr: int64 [S + 1] or None (every row a sample).  Returns (y, stats).  No output may overlap an input."""
    N, S, pp, ops, ps, ty, dev = _norm_operands(norm, x, weight, bias, stats, ptr)
    py = _operand(y, "y", (N, norm.dim_y), ty, dev)
    st = _stream_of(x, dev)
    L = lib()
    nb = L.cgtp_norm_workspace_bytes(norm._h, N, S, ptr is not None, 0)
    ws = _scratch(nb, x)
    _check(L.norm_forward(norm._h, *ops, py, ps, N, S, pp, _ptr(ws), nb, st))
    return y, stats


def norm_backward(norm: Norm, x, weight, bias, gy, stats, gx, gweight, gbias, ptr=None):
    """Gradients of norm_forward given gy [N, dim_y] and the stats that it wrote.  Returns (gx, gweight, gbias).  No output may overlap
    an input."""
    N, S, pp, ops, ps, ty, dev = _norm_operands(norm, x, weight, bias, stats, ptr)
    out = (_operand(gx, "gx", (N, norm.dim_x), ty, dev), _operand(gweight, "gweight", (norm.n_w,), ty, dev),
           _operand(gbias, "gbias", (norm.n_b,), ty, dev, norm.n_b == 0))
    pg = _operand(gy, "gy", (N, norm.dim_y), ty, dev)
    st = _stream_of(x, dev)
    L = lib()
    nb = L.cgtp_norm_workspace_bytes(norm._h, N, S, ptr is not None, 1)
    ws = _scratch(nb, x)
    _check(L.norm_backward(norm._h, *ops, pg, ps, *out, N, S, pp, _ptr(ws), nb, st))
    return gx, gweight, gbias


# ---- products by kind of row, orthogonalised updates ------------------------------------------------------------------

def _index_operand(t, name: str, size: int, device: int) -> int:
    if t is None:
        return 0
    if t.dtype != _torch.int64 or t.dim() != 1 or t.shape[0] != size or not t.is_contiguous() or t.get_device() != device:
        _bad(f"{name}: a contiguous int64 tensor [{size}] where x is")
    return t.data_ptr()


def _grouped_operands(x, W, ptr, perm, comps: int):
    dt, dev = _type_and_device(x)
    if x.dim() != 2 or W is None or W.dim() != 3:
        _bad("x must have two dimensions, W three")
    if comps < 1:
        _bad("comps must be positive")
    rows, (groups, k, n), ty = x.shape[0], W.shape, x.dtype
    if ptr is None:
        _bad("ptr is missing")
    index = (_index_operand(ptr, "ptr", groups + 1, dev), _index_operand(perm, "perm", rows, dev))
    return rows, groups, k, n, ty, dt, dev, index, _row_operand(x, "x", (rows, comps * k), ty, dev), _operand(W, "W", (groups, k, n), ty, dev)


def grouped_forward(x, W, out, ptr, b=None, perm=None, comps: int = 1):
    """out = x W[g] + b[g] for the rows of each group g: positions ptr[g] .. ptr[g+1] - 1, position p being row perm[p] (or p).  x [rows, comps * d_in],
    W [groups, d_in, d_out], b [groups, d_out] or None, out [rows, comps * d_out]; ptr int64 [groups + 1], perm int64 [rows] or None: row_ptr
    and perm of cgtp_csr_from_coo with the kinds as receivers.  x and out may be columns of wider rows.  Rows of no group keep
    what out holds.  out must not overlap an input."""
    rows, groups, k, n, ty, dt, dev, index, (px, ldx), pw = _grouped_operands(x, W, ptr, perm, comps)
    po, ldo = _row_operand(out, "out", (rows, comps * n), ty, dev)
    pb = _operand(b, "b", (groups, n), ty, dev, True)
    st = _stream_of(x, dev)
    _check(lib().grouped_forward(px, pw, pb, po, rows, k, n, comps, groups, *index, ldx, ldo, dt, st))
    return out


def grouped_backward(x, W, gout, gx, gW, ptr, gb=None, perm=None, comps: int = 1):
    """Gradients of grouped_forward given gout [rows, comps * d_out]: gx like x, gW like W, and gb [groups, d_out] where it is given.  x, gout and gx
    may be columns of wider rows.  Returns (gx, gW, gb).  No output may overlap an input."""
    rows, groups, k, n, ty, dt, dev, index, (px, ldx), pw = _grouped_operands(x, W, ptr, perm, comps)
    pg, ldg = _row_operand(gout, "gout", (rows, comps * n), ty, dev)
    pgx, ldgx = _row_operand(gx, "gx", (rows, comps * k), ty, dev)
    out = (pgx, _operand(gW, "gW", (groups, k, n), ty, dev), _operand(gb, "gb", (groups, n), ty, dev, True))
    st = _stream_of(x, dev)
    L = lib()
    nb = L.cgtp_grouped_workspace_bytes(rows, k, n, comps, groups, dt)
    ws = _scratch(nb, x)
    _check(L.grouped_backward(px, pw, pg, *out, rows, k, n, comps, groups, *index, ldx, ldg, ldgx, dt, _ptr(ws), nb, st))
    return gx, gW, gb


STEPS = ((3.4445, -4.7750, 2.0315),) * 5      # take singular values from 0.002 of the size of a matrix to all of it into 0.68 to 1.21


def _matrices(t, name: str, shape: Tuple, dtype, device: int) -> Tuple[int, int, int]:
    """Address, elements from one row and from one matrix to the next."""
    if t is None:
        _bad(f"{name} is missing")
    if t.shape != shape:
        _bad(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype or t.get_device() != device:
        _bad(f"{name}: {t.dtype} on {t.device}, expected {dtype} where G is")
    stride, ld, step = t.stride()
    if step != 1 and shape[2] > 1 and t.numel() > 0:
        _bad(f"{name}: the elements of a row must be neighbours")
    return t.data_ptr(), ld if shape[1] > 1 else shape[2], stride if shape[0] > 1 else shape[1] * shape[2]


def orthogonalise(G, out, coefficients: Sequence[Sequence[float]] = STEPS, eps: float = 1e-7):
    """out = G [batch, m, n] (or [m, n]) with the singular values of each matrix taken towards one: X = G / (|G| + eps), then for each triple of
    coefficients X <- a X + (b A + c A A) X with A = X X^T.  Rows of G and out may be columns of wider ones.  out must not overlap G."""
    dt, dev = _type_and_device(G)
    if G.dim() == 2:
        orthogonalise(G[None], None if out is None else out[None], coefficients, eps)
        return out
    if G.dim() != 3:
        _bad("G must have two or three dimensions")
    (batch, m, n), ty = G.shape, G.dtype
    pg, ldg, sg = _matrices(G, "G", G.shape, ty, dev)
    po, ldo, so = _matrices(out, "out", G.shape, ty, dev)
    if any(len(t) != 3 for t in coefficients):
        _bad("coefficients: three numbers for each step")
    c = (C.c_double * (3 * len(coefficients)))(*(v for t in coefficients for v in t))
    st = _stream_of(G, dev)
    L = lib()
    nb = L.cgtp_orthogonalise_workspace_bytes(batch, m, n, dt)
    ws = _scratch(nb, G)
    _check(L.orthogonalise(pg, po, batch, m, n, ldg, ldo, sg, so, c, len(coefficients), eps, dt, _ptr(ws), nb, st))
    return out
