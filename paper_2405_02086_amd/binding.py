"""ctypes binding for libmlproj.so (declared in include/mlproj.h).

Argument marshalling only: every step of the projection runs in the HIP kernels.
PyTorch is used for device memory and streams.  There is no CPU fallback: if the
shared library has not been built, every entry point raises.
"""
import ctypes
import os
import struct
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmlproj.so")
SRC_PATHS = [os.path.join(_HERE, "csrc", name) for name in ("mlproj.hip", "heldmulti.hip", "gatedff.hip", "linear.hip", "blocknorm.hip", "w4.hip", "q8.hip")]

L1INF, L11, L12, L1INFINF = 0, 1, 2, 3
_VARIANTS = {"l1inf": L1INF, "l11": L11, "l12": L12, "tri": L1INFINF}

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed-fp32 VALU ops
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


class MlprojError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = lib().mlproj_status_string(status).decode() if _lib is not None else "?"
        super().__init__(f"{where}: {msg} (status {status})")


def build(verbose=False):
    """Compile the translation units csrc/*.hip (with the csrc/*.h they include) for gfx950, side by
    side, and link them into libmlproj.so next to this file."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, "%d.o" % i) for i in range(len(SRC_PATHS))]
        commands = [[hipcc] + HIPCC_FLAGS + ["-c", "-o", o, src] for o, src in zip(objects, SRC_PATHS)]
        running = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for c in commands]
        said = [p.communicate()[0] for p in running]
        link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB_PATH] + objects
        failed = any(p.returncode != 0 for p in running)
        if not failed:
            done = subprocess.run(link, capture_output=True, text=True)
            commands.append(link)
            said.append(done.stdout + done.stderr)
            failed = done.returncode != 0
        if verbose or failed:
            for c, out in zip(commands, said):
                print(" ".join(c))
                print(out)
    if failed:
        raise RuntimeError("hipcc failed building libmlproj.so")
    global _lib
    _lib = None
    return LIB_PATH


_lib = None


def lib():
    """The loaded C library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()'). "
            "There is no CPU fallback.")
    L = ctypes.CDLL(LIB_PATH)
    c_ll, c_sz, c_vp, c_f, c_i = ctypes.c_longlong, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_float, ctypes.c_int
    L.mlproj_version.restype = c_i
    L.mlproj_version.argtypes = []
    L.mlproj_status_string.restype = ctypes.c_char_p
    L.mlproj_status_string.argtypes = [c_i]
    L.mlproj_workspace_bytes.restype = c_i
    L.mlproj_workspace_bytes.argtypes = [c_i, c_ll, c_ll, c_ll, ctypes.POINTER(c_sz)]
    L.mlproj_trace_begin.restype = c_i
    L.mlproj_trace_begin.argtypes = [ctypes.POINTER(c_vp), c_i]
    L.mlproj_trace_end.restype = c_i
    L.mlproj_trace_end.argtypes = []
    L.mlproj_set_l11_sweeps.restype = c_i
    L.mlproj_set_l11_sweeps.argtypes = [c_i]
    L.mlproj_set_search_spin_limit.restype = c_i
    L.mlproj_set_search_spin_limit.argtypes = [c_i]
    L.mlproj_stripe_of_workgroup.restype = c_i
    L.mlproj_stripe_of_workgroup.argtypes = [c_ll, c_ll]
    L.mlproj_multilevel_one_pass.restype = c_i
    L.mlproj_multilevel_one_pass.argtypes = [c_i, c_i, c_ll, c_ll, c_ll, c_i]
    L.mlproj_norm_l1q.restype = c_i
    L.mlproj_norm_l1q.argtypes = [c_vp, c_ll, c_ll, c_i, c_vp, c_sz, c_vp, c_vp, c_vp]
    for name in ("bilevel_proj_l1inf", "bilevel_proj_l11", "bilevel_proj_l12"):
        fn = getattr(L, name)
        fn.restype = c_i
        fn.argtypes = [c_vp, c_vp, c_ll, c_ll, c_f, c_vp, c_sz, c_vp, c_vp, c_vp]
    L.bilevel_proj_l1inf_no_alloc.restype = c_i
    L.bilevel_proj_l1inf_no_alloc.argtypes = [c_vp, c_vp, c_ll, c_ll, c_f, c_vp, c_vp, c_vp]
    L.bilevel_radii.restype = c_i
    L.bilevel_radii.argtypes = [c_i, c_vp, c_ll, c_ll, c_f, c_vp, c_sz, c_vp, c_vp]
    L.bilevel_apply.restype = c_i
    L.bilevel_apply.argtypes = [c_i, c_vp, c_vp, c_ll, c_ll, c_vp, c_sz, c_vp, c_vp]
    L.mlproj_multilevel_workspace_bytes.restype = c_i
    L.mlproj_multilevel_workspace_bytes.argtypes = [c_i, ctypes.POINTER(c_ll), ctypes.POINTER(c_sz)]
    L.multilevel_proj.restype = c_i
    L.multilevel_proj.argtypes = [c_vp, c_vp, c_i, ctypes.POINTER(c_ll), ctypes.POINTER(c_i), c_f, c_vp, c_sz,
                                  c_vp, c_vp, c_vp]
    L.multilevel_proj_p.restype = c_i
    L.multilevel_proj_p.argtypes = [c_i, c_vp, c_vp, c_i, ctypes.POINTER(c_ll), ctypes.POINTER(c_i), c_f, c_vp,
                                    c_sz, c_vp, c_vp, c_vp]
    L.multilevel_proj_stored.restype = c_i
    L.multilevel_proj_stored.argtypes = [c_i, c_i, c_vp, c_vp, c_i, ctypes.POINTER(c_ll), ctypes.POINTER(c_i), c_f,
                                         c_vp, c_sz, c_vp, c_vp, c_vp]
    L.bilevel_proj_pq.restype = c_i
    L.bilevel_proj_pq.argtypes = [c_i, c_i, c_vp, c_vp, c_ll, c_ll, c_f, c_vp, c_sz, c_vp, c_vp, c_vp]
    L.bilevel_proj_stored.restype = c_i
    L.bilevel_proj_stored.argtypes = [c_i, c_i, c_i, c_vp, c_vp, c_ll, c_ll, c_f, c_vp, c_sz, c_vp, c_vp, c_vp, c_vp]
    L.bilevel_proj_batch.restype = c_i
    L.bilevel_proj_batch.argtypes = [c_i, c_i, c_i, c_i, ctypes.POINTER(Problem), c_vp]
    L.multilevel_proj_weighted.restype = c_i
    L.multilevel_proj_weighted.argtypes = [c_i, c_vp, c_vp, c_i, ctypes.POINTER(c_ll), ctypes.POINTER(c_i), c_f, c_vp,
                                           c_vp, c_sz, c_vp, c_vp, c_vp]
    L.bilevel_proj_weighted.restype = c_i
    L.bilevel_proj_weighted.argtypes = [c_i, c_i, c_vp, c_vp, c_ll, c_ll, c_f, c_vp, c_vp, c_sz, c_vp, c_vp, c_vp, c_vp]
    L.trilevel_proj_stored.restype = c_i
    L.trilevel_proj_stored.argtypes = [c_i, c_vp, c_vp, c_ll, c_ll, c_ll, c_f, c_vp, c_sz, c_vp, c_vp, c_vp, c_vp]
    L.trilevel_proj_l1infinf.restype = c_i
    L.trilevel_proj_l1infinf.argtypes = [c_vp, c_vp, c_ll, c_ll, c_ll, c_f, c_vp, c_sz, c_vp, c_vp, c_vp]
    block, norm, w4 = ctypes.POINTER(GatedBlock), ctypes.POINTER(NormBlock), ctypes.POINTER(PackedW4)
    L.mlproj_gated_ff_workspace_bytes.restype = c_i
    L.mlproj_gated_ff_workspace_bytes.argtypes = [c_i, c_ll, c_ll, c_ll, c_i, c_i, ctypes.POINTER(c_sz)]
    L.mlproj_gated_ff_route.restype = c_i
    L.mlproj_gated_ff_route.argtypes = [c_i, c_i, c_ll, c_ll, c_ll]
    L.gated_ff_forward.restype = c_i
    L.gated_ff_forward.argtypes = [c_i, c_i, block, c_vp, c_ll, c_vp, c_vp, c_ll, c_vp, c_sz, c_vp]
    L.gated_ff_backward.restype = c_i
    L.gated_ff_backward.argtypes = [c_i, c_i, block, c_vp, c_ll, c_vp, c_vp, c_ll, c_vp, c_ll, c_vp, c_vp, c_ll, c_vp, c_sz, c_vp]
    linear, drop = ctypes.POINTER(LinearBlock), ctypes.POINTER(DropoutStruct)
    L.mlproj_linear_workspace_bytes.restype = c_i
    L.mlproj_linear_workspace_bytes.argtypes = [c_i, c_ll, c_ll, c_ll, c_i, ctypes.POINTER(c_sz)]
    L.linear_forward.restype = c_i
    L.linear_forward.argtypes = [c_i, c_i, linear, c_vp, c_ll, c_vp, c_ll, c_vp, c_ll, c_vp, c_sz, c_vp]
    L.linear_backward.restype = c_i
    L.linear_backward.argtypes = [c_i, c_i, linear, c_vp, c_ll, c_vp, c_ll, c_vp, c_ll, c_vp, c_ll, c_vp, c_vp, c_sz, c_vp]
    L.dropout_forward.restype = c_i
    L.dropout_forward.argtypes = [c_i, drop, c_ll, c_ll, c_vp, c_ll, c_vp, c_ll, c_vp, c_ll, c_vp]
    L.block_norm_forward.restype = c_i
    L.block_norm_forward.argtypes = [c_i, norm, c_vp, c_ll, c_vp, c_ll, c_vp, c_ll, c_vp]
    L.mlproj_block_norm_workspace_bytes.restype = c_i
    L.mlproj_block_norm_workspace_bytes.argtypes = [c_ll, c_ll, ctypes.POINTER(c_sz)]
    L.block_norm_backward.restype = c_i
    L.block_norm_backward.argtypes = [c_i, norm, c_vp, c_ll, c_vp, c_ll, c_vp, c_ll, c_vp, c_ll, c_vp, c_ll, c_vp, c_vp, c_ll,
                                      c_vp, c_vp, c_sz, c_vp]
    q8 = ctypes.POINTER(PackedQ8)
    L.q8_pack.restype = c_i
    L.q8_pack.argtypes = [c_i, c_i, c_vp, c_ll, q8, c_vp]
    L.block_norm8_forward.restype = c_i
    L.block_norm8_forward.argtypes = [c_i, norm, c_vp, c_ll, c_vp, c_ll, q8, c_vp]
    L.mlproj_q8_workspace_bytes.restype = c_i
    L.mlproj_q8_workspace_bytes.argtypes = [c_ll, c_ll, c_ll, c_i, ctypes.POINTER(c_sz)]
    L.q8_linear.restype = c_i
    L.q8_linear.argtypes = [c_i, c_i, q8, q8, c_vp, c_vp, c_ll, c_vp, c_ll, c_vp, c_sz, c_vp]
    L.q8_gated.restype = c_i
    L.q8_gated.argtypes = [c_i, c_i, q8, q8, q8, c_vp, c_ll, c_vp, c_sz, c_vp]
    L.mlproj_w4_bytes.restype = c_i
    L.mlproj_w4_bytes.argtypes = [c_ll, c_ll, c_i, ctypes.POINTER(c_sz), ctypes.POINTER(c_sz)]
    L.w4_pack.restype = c_i
    L.w4_pack.argtypes = [c_i, c_vp, c_ll, w4, c_vp]
    L.w4_matvec.restype = c_i
    L.w4_matvec.argtypes = [c_i, w4, c_vp, c_ll, c_ll, c_vp, c_ll, c_vp]
    L.w4_gated_matvec.restype = c_i
    L.w4_gated_matvec.argtypes = [c_i, c_i, w4, w4, c_vp, c_ll, c_ll, c_vp, c_ll, c_vp]
    _lib = L
    return L


class Problem(ctypes.Structure):
    """mlproj_problem of include/mlproj.h."""
    _fields_ = [("Y", ctypes.c_void_p), ("X", ctypes.c_void_p), ("n", ctypes.c_longlong), ("m", ctypes.c_longlong),
                ("eta", ctypes.c_float), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("v_out", ctypes.c_void_p), ("u_out", ctypes.c_void_p), ("mask_out", ctypes.c_void_p)]


class GatedBlock(ctypes.Structure):
    """mlproj_gated_block of include/mlproj.h."""
    _fields_ = [("tokens", ctypes.c_longlong), ("n", ctypes.c_longlong), ("m", ctypes.c_longlong),
                ("X", ctypes.c_void_p), ("ldx", ctypes.c_longlong), ("Wg", ctypes.c_void_p), ("Wu", ctypes.c_void_p),
                ("ldw", ctypes.c_longlong), ("mask", ctypes.c_void_p)]


class DropoutStruct(ctypes.Structure):
    """mlproj_dropout of include/mlproj.h."""
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_ulonglong), ("offset", ctypes.c_ulonglong), ("step", ctypes.c_void_p)]


class LinearBlock(ctypes.Structure):
    """mlproj_linear of include/mlproj.h."""
    _fields_ = [("tokens", ctypes.c_longlong), ("n", ctypes.c_longlong), ("m", ctypes.c_longlong),
                ("X", ctypes.c_void_p), ("ldx", ctypes.c_longlong), ("W", ctypes.c_void_p), ("ldw", ctypes.c_longlong),
                ("bias", ctypes.c_void_p), ("dropout", ctypes.POINTER(DropoutStruct))]


class NormBlock(ctypes.Structure):
    """mlproj_norm_block of include/mlproj.h."""
    _fields_ = [("tokens", ctypes.c_longlong), ("n", ctypes.c_longlong), ("b", ctypes.c_void_p), ("ldb", ctypes.c_longlong),
                ("w_post", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("gate_stride", ctypes.c_longlong),
                ("w_pre", ctypes.c_void_p), ("scale", ctypes.c_float), ("eps", ctypes.c_float)]


class PackedQ8(ctypes.Structure):
    """mlproj_q8 of include/mlproj.h."""
    _fields_ = [("rows", ctypes.c_longlong), ("n", ctypes.c_longlong), ("codes", ctypes.c_void_p), ("ld", ctypes.c_longlong),
                ("scales", ctypes.c_void_p), ("lds", ctypes.c_longlong)]


class PackedW4(ctypes.Structure):
    """mlproj_w4 of include/mlproj.h."""
    _fields_ = [("n", ctypes.c_longlong), ("m", ctypes.c_longlong), ("group", ctypes.c_int), ("codes", ctypes.c_void_p),
                ("scales", ctypes.c_void_p)]


EXPORTS = (
    "mlproj_version", "mlproj_status_string", "mlproj_workspace_bytes", "mlproj_trace_begin", "mlproj_trace_end",
    "mlproj_norm_l1q", "bilevel_proj_l1inf", "bilevel_proj_l11", "bilevel_proj_l12",
    "trilevel_proj_l1infinf", "bilevel_radii", "bilevel_apply",
    "mlproj_multilevel_workspace_bytes", "multilevel_proj", "multilevel_proj_p", "bilevel_proj_pq",
    "bilevel_proj_stored", "bilevel_proj_batch", "trilevel_proj_stored", "mlproj_set_l11_sweeps",
    "multilevel_proj_stored", "bilevel_proj_weighted", "multilevel_proj_weighted", "mlproj_set_search_spin_limit",
    "bilevel_proj_l1inf_no_alloc", "mlproj_stripe_of_workgroup", "mlproj_multilevel_one_pass",
    "mlproj_gated_ff_workspace_bytes", "mlproj_gated_ff_route", "gated_ff_forward", "gated_ff_backward",
    "mlproj_linear_workspace_bytes", "linear_forward", "linear_backward", "dropout_forward",
    "block_norm_forward", "mlproj_block_norm_workspace_bytes", "block_norm_backward",
    "q8_pack", "block_norm8_forward", "mlproj_q8_workspace_bytes", "q8_linear", "q8_gated",
    "mlproj_w4_bytes", "w4_pack", "w4_matvec", "w4_gated_matvec",
)


def _check(status, where):
    if status != 0:
        raise MlprojError(status, where)


def set_search_spin_limit(polls):
    """Polls after which the several-workgroup search gives up (0 = at once); returns the old value."""
    before = lib().mlproj_set_search_spin_limit(int(polls))
    if before < 0:
        raise MlprojError(int(before), "mlproj_set_search_spin_limit")
    return int(before)


def set_l11_sweeps(sweeps):
    """Lock-step passes an l1,1 call enqueues before its finishing pass (0 = default); returns the old value."""
    before = lib().mlproj_set_l11_sweeps(int(sweeps))
    if before < 0:
        raise MlprojError(before, "mlproj_set_l11_sweeps")
    return before


def workspace_bytes(variant, d0, d1, d2=1):
    out = ctypes.c_size_t(0)
    v = _VARIANTS.get(variant, variant)
    _check(lib().mlproj_workspace_bytes(v, d0, d1, d2, ctypes.byref(out)), "mlproj_workspace_bytes")
    return out.value


# What a call costs on the host is marshalling: for the smallest matrices it is longer than the kernel.
# Pointers and the radius go to ctypes as plain numbers (the argument types convert them), and the
# current stream is asked for as the handle it is.  A 256 x 128 call: 8.0 -> 6.4 us.
def _ptr(t):
    return None if t is None else t.data_ptr()


_torch = None


def _import_torch():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    c = _import_torch()._C
    return c._cuda_getCurrentRawStream(c._cuda_getDevice())


# What a call allocates itself (scratch, results) it allocates on the stream that it runs on: the allocator hands out and takes
# back memory in the order of the stream it was asked on, and the scratch is given back while the kernels are still to run.
def _empty_like(t, stream=None):
    torch = _import_torch()
    if stream is None:
        return torch.empty_like(t)
    with torch.cuda.stream(stream):
        return torch.empty_like(t)


def _new_empty(like, shape, dtype=None, stream=None):
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with _import_torch().cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


class Workspace:
    """Device scratch for one call at a time, allocated on `stream` (default: the current one); needs no initialisation."""

    def __init__(self, nbytes, device="cuda", stream=None):
        torch = _import_torch()
        nbytes = (int(nbytes) + 255) // 256 * 256
        if stream is None:
            self.buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
        else:
            with torch.cuda.stream(stream):
                self.buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
        assert self.buf.data_ptr() % 256 == 0
        self.nbytes = nbytes

    @classmethod
    def for_call(cls, variant, d0, d1, d2=1, **kw):
        return cls(workspace_bytes(variant, d0, d1, d2), **kw)

    def result(self):
        """Synchronise and decode the mlproj_result record at the head of the workspace."""
        raw = bytes(self.buf[:64].cpu().numpy().tobytes())
        tau, norm, vmax, scale, cap, n_active, inside, iters, sweeps, pending, finished = struct.unpack_from("<dddddIIIIII", raw)
        return {"tau": tau, "norm": norm, "vmax": vmax, "scale": scale, "cap": cap, "n_active": n_active,
                "inside_ball": bool(inside), "search_iters": iters,
                "inner_sweeps": sweeps, "inner_pending": pending, "inner_finished": finished}


def _prep(Y, X, stream=None):
    torch = _import_torch()
    f32 = torch.float32
    assert Y.is_cuda and Y.dtype is f32 and Y.is_contiguous(), "Y: contiguous fp32 device tensor"
    if X is None:
        return _empty_like(Y, stream)
    assert X.is_cuda and X.dtype is f32 and X.is_contiguous() and X.shape == Y.shape
    return X


def _bilevel(name, variant, Y, eta, X, workspace, v_out, u_out, stream):
    assert Y.dim() == 2
    n, m = Y.shape
    X = _prep(Y, X, stream)
    if workspace is None:
        workspace = Workspace.for_call(variant, n, m, device=Y.device, stream=stream)
    st = getattr(lib(), name)(Y.data_ptr(), X.data_ptr(), n, m, eta, workspace.buf.data_ptr(), workspace.nbytes,
                              None if v_out is None else v_out.data_ptr(), None if u_out is None else u_out.data_ptr(),
                              _stream(stream))
    if st != 0:
        _check(st, name)
    return X


def bilevel_proj_l1inf(Y, eta, X=None, workspace=None, v_out=None, u_out=None, stream=None):
    return _bilevel("bilevel_proj_l1inf", L1INF, Y, eta, X, workspace, v_out, u_out, stream)


def bilevel_proj_l1inf_no_alloc(Y, eta, X, v_out=None, u_out=None, stream=None):
    """bilevel_proj_l1inf on the library's built-in scratch buffer: the call allocates nothing,
    so X is the caller's (and there is no workspace to pass)."""
    assert Y.dim() == 2 and X is not None
    n, m = Y.shape
    assert _prep(Y, X) is X
    st = lib().bilevel_proj_l1inf_no_alloc(_ptr(Y), _ptr(X), n, m, ctypes.c_float(eta), _ptr(v_out), _ptr(u_out),
                                           _stream(stream))
    _check(st, "bilevel_proj_l1inf_no_alloc")
    return X


def bilevel_proj_l11(Y, eta, X=None, workspace=None, v_out=None, u_out=None, stream=None):
    return _bilevel("bilevel_proj_l11", L11, Y, eta, X, workspace, v_out, u_out, stream)


def bilevel_proj_l12(Y, eta, X=None, workspace=None, v_out=None, u_out=None, stream=None):
    return _bilevel("bilevel_proj_l12", L12, Y, eta, X, workspace, v_out, u_out, stream)


def bilevel_radii(variant, Y, eta, workspace, v_out=None, stream=None):
    n, m = Y.shape
    v = _VARIANTS.get(variant, variant)
    _check(lib().bilevel_radii(v, _ptr(Y), n, m, ctypes.c_float(eta), _ptr(workspace.buf), workspace.nbytes,
                               _ptr(v_out), _stream(stream)), "bilevel_radii")


def bilevel_apply(variant, Y, X, workspace, u_out=None, stream=None):
    n, m = Y.shape
    v = _VARIANTS.get(variant, variant)
    _check(lib().bilevel_apply(v, _ptr(Y), _ptr(X), n, m, _ptr(workspace.buf), workspace.nbytes,
                               _ptr(u_out), _stream(stream)), "bilevel_apply")
    return X


def trilevel_proj_l1infinf(Y, eta, X=None, workspace=None, v_out=None, u_out=None, stream=None):
    assert Y.dim() == 3
    d0, d1, d2 = Y.shape
    X = _prep(Y, X, stream)
    if workspace is None:
        workspace = Workspace.for_call(L1INFINF, d0, d1, d2, device=Y.device, stream=stream)
    st = lib().trilevel_proj_l1infinf(_ptr(Y), _ptr(X), d0, d1, d2, ctypes.c_float(eta),
                                      _ptr(workspace.buf), workspace.nbytes, _ptr(v_out), _ptr(u_out),
                                      _stream(stream))
    _check(st, "trilevel_proj_l1infinf")
    return X


OUTER_L1, OUTER_L2, OUTER_LINF = 0, 1, 2
_OUTERS = {1: OUTER_L1, 2: OUTER_L2, "inf": OUTER_LINF}


def bilevel_proj_pq(p, q, Y, eta, X=None, workspace=None, v_out=None, u_out=None, stream=None):
    """BP^{p,q}: p in {1, 2, "inf"} (outer), q in {"inf", 1, 2} (per column)."""
    assert Y.dim() == 2
    n, m = Y.shape
    X = _prep(Y, X, stream)
    variant = {"inf": L1INF, 1: L11, 2: L12}[q]
    if workspace is None:
        workspace = Workspace.for_call(variant, n, m, device=Y.device, stream=stream)
    st = lib().bilevel_proj_pq(_OUTERS[p], variant, _ptr(Y), _ptr(X), n, m, ctypes.c_float(eta),
                               _ptr(workspace.buf), workspace.nbytes, _ptr(v_out), _ptr(u_out), _stream(stream))
    _check(st, "bilevel_proj_pq")
    return X


STORE_F32, STORE_BF16, STORE_F16 = 0, 1, 2


def bilevel_proj_stored(Y, eta, q, p=1, X=None, workspace=None, v_out=None, u_out=None, mask_out=None,
                        stream=None):
    """BP^{p,q} on a contiguous fp32, bf16 or fp16 device matrix (X has Y's dtype); mask_out is an
    optional uint8 tensor of m entries that receives 1 for every kept column."""
    import torch
    storages = {torch.float32: STORE_F32, torch.bfloat16: STORE_BF16, torch.float16: STORE_F16}
    assert Y.is_cuda and Y.dim() == 2 and Y.is_contiguous() and Y.dtype in storages
    n, m = Y.shape
    if X is None:
        X = _empty_like(Y, stream)
    assert X.is_cuda and X.dtype == Y.dtype and X.is_contiguous() and X.shape == Y.shape
    assert mask_out is None or (mask_out.dtype == torch.uint8 and mask_out.numel() >= m)
    variant = {"inf": L1INF, 1: L11, 2: L12}[q]
    if workspace is None:
        workspace = Workspace.for_call(variant, n, m, device=Y.device, stream=stream)
    st = lib().bilevel_proj_stored(storages[Y.dtype], _OUTERS[p], variant, _ptr(Y), _ptr(X), n, m,
                                   ctypes.c_float(eta), _ptr(workspace.buf), workspace.nbytes, _ptr(v_out),
                                   _ptr(u_out), _ptr(mask_out), _stream(stream))
    _check(st, "bilevel_proj_stored")
    return X


def bilevel_proj_weighted(Y, eta, q, weights, X=None, workspace=None, v_out=None, u_out=None, mask_out=None,
                          stream=None):
    """BP^{p,q} with the weighted l1 ball {u : sum_j w_j |u_j| <= eta} as outer norm, on a contiguous
    fp32, bf16 or fp16 device matrix; weights is an fp32 device tensor of m positive entries."""
    import torch
    storages = {torch.float32: STORE_F32, torch.bfloat16: STORE_BF16, torch.float16: STORE_F16}
    assert Y.is_cuda and Y.dim() == 2 and Y.is_contiguous() and Y.dtype in storages
    n, m = Y.shape
    assert weights.is_cuda and weights.dtype == torch.float32 and weights.is_contiguous() and weights.numel() == m
    if X is None:
        X = _empty_like(Y, stream)
    assert X.is_cuda and X.dtype == Y.dtype and X.is_contiguous() and X.shape == Y.shape
    assert mask_out is None or (mask_out.dtype == torch.uint8 and mask_out.numel() >= m)
    variant = {"inf": L1INF, 1: L11, 2: L12}[q]
    if workspace is None:
        workspace = Workspace.for_call(variant, n, m, device=Y.device, stream=stream)
    st = lib().bilevel_proj_weighted(storages[Y.dtype], variant, _ptr(Y), _ptr(X), n, m, ctypes.c_float(eta),
                                     _ptr(weights), _ptr(workspace.buf), workspace.nbytes, _ptr(v_out),
                                     _ptr(u_out), _ptr(mask_out), _stream(stream))
    _check(st, "bilevel_proj_weighted")
    return X


def trilevel_proj_stored(Y, eta, X=None, workspace=None, v_out=None, u_out=None, mask_out=None, stream=None):
    """TP^{1,inf,inf} on a contiguous fp32, bf16 or fp16 device tensor of three axes."""
    import torch
    storages = {torch.float32: STORE_F32, torch.bfloat16: STORE_BF16, torch.float16: STORE_F16}
    assert Y.is_cuda and Y.dim() == 3 and Y.is_contiguous() and Y.dtype in storages
    d0, d1, d2 = Y.shape
    if X is None:
        X = _empty_like(Y, stream)
    assert X.is_cuda and X.dtype == Y.dtype and X.is_contiguous() and X.shape == Y.shape
    if workspace is None:
        workspace = Workspace.for_call("tri", d0, d1, d2, device=Y.device, stream=stream)
    st = lib().trilevel_proj_stored(storages[Y.dtype], _ptr(Y), _ptr(X), d0, d1, d2, ctypes.c_float(eta),
                                    _ptr(workspace.buf), workspace.nbytes, _ptr(v_out), _ptr(u_out),
                                    _ptr(mask_out), _stream(stream))
    _check(st, "trilevel_proj_stored")
    return X


class PreparedBatch:
    """The argument block of a bilevel_proj_batch call, marshalled once: a training loop projects
    the same buffers after every step, and filling the block costs more host time than the
    call.  Calling the object enqueues the batch; `.X` lists the output tensors.  It keeps every
    tensor it points to alive.  `stream`: what it allocates itself is for calls on that stream."""

    def __init__(self, Ys, etas, q, p=1, Xs=None, workspaces=None, v_outs=None, u_outs=None, mask_outs=None, stream=None):
        import torch
        storages = {torch.float32: STORE_F32, torch.bfloat16: STORE_BF16, torch.float16: STORE_F16}
        count = len(Ys)
        assert count > 0 and len(etas) == count
        self.variant = {"inf": L1INF, 1: L11, 2: L12}[q]
        self.outer = _OUTERS[p]
        self.count = count
        pick = lambda lst, i: None if lst is None else lst[i]
        self.problems = (Problem * count)()
        self.X = []
        self.keep = [Ys, v_outs, u_outs, mask_outs]   # every buffer the block points to
        for i, Y in enumerate(Ys):
            assert Y.is_cuda and Y.dim() == 2 and Y.is_contiguous() and Y.dtype == Ys[0].dtype and Y.dtype in storages
            n, m = Y.shape
            X = pick(Xs, i)
            if X is None:
                X = _empty_like(Y, stream)
            assert X.is_cuda and X.dtype == Y.dtype and X.is_contiguous() and X.shape == Y.shape
            # every problem needs a workspace of its own
            ws = pick(workspaces, i) or Workspace.for_call(self.variant, n, m, device=Y.device, stream=stream)
            self.keep.append(ws)
            self.X.append(X)
            pr = self.problems[i]
            pr.Y, pr.X, pr.n, pr.m, pr.eta = Y.data_ptr(), X.data_ptr(), n, m, float(etas[i])
            pr.workspace, pr.workspace_bytes = ws.buf.data_ptr(), ws.nbytes
            for field, lst in (("v_out", v_outs), ("u_out", u_outs), ("mask_out", mask_outs)):
                t = pick(lst, i)
                setattr(pr, field, None if t is None else t.data_ptr())
        self.storage = storages[Ys[0].dtype]

    def __call__(self, stream=None):
        st = lib().bilevel_proj_batch(self.storage, self.outer, self.variant, self.count, self.problems,
                                      _stream(stream))
        _check(st, "bilevel_proj_batch")
        return self.X


def bilevel_proj_batch(Ys, etas, q, p=1, Xs=None, workspaces=None, v_outs=None, u_outs=None, mask_outs=None,
                       stream=None):
    """Independent BP^{p,q} projections of the matrices in Ys (same dtype, any shapes) with radii
    etas, through bilevel_proj_batch; returns the list of X tensors.  Optional lists give the
    per-problem X, workspace, v_out, u_out and mask_out."""
    batch = PreparedBatch(Ys, etas, q, p=p, Xs=Xs, workspaces=workspaces, v_outs=v_outs, u_outs=u_outs,
                          mask_outs=mask_outs, stream=stream)
    return batch(stream)


NORM_INF, NORM_L1, NORM_L2 = 0, 1, 2
_NORMS = {"inf": NORM_INF, 1: NORM_L1, 2: NORM_L2}


def multilevel_workspace_bytes(shape):
    dims = (ctypes.c_longlong * len(shape))(*shape)
    out = ctypes.c_size_t(0)
    _check(lib().mlproj_multilevel_workspace_bytes(len(shape), dims, ctypes.byref(out)),
           "mlproj_multilevel_workspace_bytes")
    return out.value


def multilevel_proj(Y, norms, eta, X=None, workspace=None, v_out=None, u_out=None, stream=None, p=1):
    """norms: inner norms, innermost (last axis) first, each "inf", 1 or 2; groups on axis 0;
    p: outermost norm (1, 2 or "inf")."""
    X = _prep(Y, X, stream)
    shape = tuple(Y.shape)
    assert len(norms) == len(shape) - 1
    if workspace is None:
        workspace = Workspace(multilevel_workspace_bytes(shape), device=Y.device, stream=stream)
    dims = (ctypes.c_longlong * len(shape))(*shape)
    nrm = (ctypes.c_int * len(norms))(*[_NORMS[q] for q in norms])
    if p == 1:
        st = lib().multilevel_proj(_ptr(Y), _ptr(X), len(shape), dims, nrm, ctypes.c_float(eta),
                                   _ptr(workspace.buf), workspace.nbytes, _ptr(v_out), _ptr(u_out), _stream(stream))
    else:
        st = lib().multilevel_proj_p(_OUTERS[p], _ptr(Y), _ptr(X), len(shape), dims, nrm, ctypes.c_float(eta),
                                     _ptr(workspace.buf), workspace.nbytes, _ptr(v_out), _ptr(u_out), _stream(stream))
    _check(st, "multilevel_proj")
    return X


def multilevel_proj_stored(Y, norms, eta, p=1, X=None, workspace=None, v_out=None, u_out=None, stream=None):
    """multilevel_proj on a contiguous fp32, bf16 or fp16 device tensor (X has Y's dtype)."""
    import torch
    storages = {torch.float32: STORE_F32, torch.bfloat16: STORE_BF16, torch.float16: STORE_F16}
    assert Y.is_cuda and Y.is_contiguous() and Y.dtype in storages
    if X is None:
        X = _empty_like(Y, stream)
    assert X.is_cuda and X.dtype == Y.dtype and X.is_contiguous() and X.shape == Y.shape
    shape = tuple(Y.shape)
    assert len(norms) == len(shape) - 1
    if workspace is None:
        workspace = Workspace(multilevel_workspace_bytes(shape), device=Y.device, stream=stream)
    dims = (ctypes.c_longlong * len(shape))(*shape)
    nrm = (ctypes.c_int * len(norms))(*[_NORMS[q] for q in norms])
    st = lib().multilevel_proj_stored(storages[Y.dtype], _OUTERS[p], _ptr(Y), _ptr(X), len(shape), dims, nrm,
                                      ctypes.c_float(eta), _ptr(workspace.buf), workspace.nbytes, _ptr(v_out),
                                      _ptr(u_out), _stream(stream))
    _check(st, "multilevel_proj_stored")
    return X


def multilevel_proj_weighted(Y, norms, eta, weights, X=None, workspace=None, v_out=None, u_out=None, stream=None):
    """multilevel_proj_stored with the weighted l1 ball {u : sum_a w_a |u_a| <= eta} as outermost norm;
    weights is an fp32 device tensor with one positive entry per group of axis 0."""
    import torch
    storages = {torch.float32: STORE_F32, torch.bfloat16: STORE_BF16, torch.float16: STORE_F16}
    assert Y.is_cuda and Y.is_contiguous() and Y.dtype in storages
    shape = tuple(Y.shape)
    assert weights.is_cuda and weights.dtype == torch.float32 and weights.is_contiguous() and weights.numel() == shape[0]
    if X is None:
        X = _empty_like(Y, stream)
    assert X.is_cuda and X.dtype == Y.dtype and X.is_contiguous() and X.shape == Y.shape
    assert len(norms) == len(shape) - 1
    if workspace is None:
        workspace = Workspace(multilevel_workspace_bytes(shape), device=Y.device, stream=stream)
    dims = (ctypes.c_longlong * len(shape))(*shape)
    nrm = (ctypes.c_int * len(norms))(*[_NORMS[q] for q in norms])
    st = lib().multilevel_proj_weighted(storages[Y.dtype], _ptr(Y), _ptr(X), len(shape), dims, nrm,
                                        ctypes.c_float(eta), _ptr(weights), _ptr(workspace.buf), workspace.nbytes,
                                        _ptr(v_out), _ptr(u_out), _stream(stream))
    _check(st, "multilevel_proj_weighted")
    return X


def norm_l1q(Y, variant, workspace=None, v_out=None, stream=None):
    """||Y||_{1,q} computed on the device; returns a python float (synchronises)."""
    import torch
    assert Y.dim() == 2 and Y.is_cuda and Y.dtype == torch.float32 and Y.is_contiguous()
    n, m = Y.shape
    v = _VARIANTS.get(variant, variant)
    if workspace is None:
        workspace = Workspace.for_call(v, n, m, device=Y.device, stream=stream)
    out = _new_empty(Y, 1, torch.float64, stream)
    st = lib().mlproj_norm_l1q(_ptr(Y), n, m, v, _ptr(workspace.buf), workspace.nbytes, _ptr(out),
                               _ptr(v_out), _stream(stream))
    _check(st, "mlproj_norm_l1q")
    if stream is not None:
        stream.synchronize()      # (item() waits for the current stream)
    return float(out.item())


# ---------------------------------------------------------------- the pruned feed-forward block

ACT_SILU, ACT_GELU, ACT_RELU, ACT_NONE = 0, 1, 2, 3
_ACTS = {"silu": ACT_SILU, "gelu": ACT_GELU, "relu": ACT_RELU, "none": ACT_NONE, None: ACT_NONE}
_STORAGES = {}


def _storage(dtype):
    if not _STORAGES:
        torch = _import_torch()
        _STORAGES.update({torch.float32: STORE_F32, torch.bfloat16: STORE_BF16, torch.float16: STORE_F16})
    assert dtype in _STORAGES, "fp32, bf16 or fp16"
    return _STORAGES[dtype]


# (One token through a norm is 4 us on the GPU: here too, what a call costs is marshalling, and most tensors are contiguous.)
def _matrix(t, shape, like, what):
    """A device matrix of `shape` and `like`'s dtype whose rows are contiguous; returns its row stride."""
    assert t.dtype is like.dtype and t.is_cuda and t.shape == shape, what
    if t.is_contiguous():
        return shape[1]
    rows, cols = shape
    assert cols <= 1 or t.stride(1) == 1, what + ": the entries of a row must be neighbours"
    return t.stride(0) if rows > 1 else max(cols, t.stride(0))


def _result(t, shape, like, what, stream):
    if t is None:
        if like.shape == shape and like.is_contiguous():
            return _torch.empty_like(like) if stream is None else _empty_like(like, stream), shape[1]
        return _new_empty(like, shape, None, stream), shape[1]
    return t, _matrix(t, shape, like, what)


def gated_ff_workspace_bytes(tokens, n, m, dtype, backward=False, masked=True):
    """Bytes a call of these sizes needs (one of fewer tokens may need more); masked=False: for calls without a mask only, which
    need far less."""
    out = ctypes.c_size_t(0)
    _check(lib().mlproj_gated_ff_workspace_bytes(_storage(dtype), tokens, n, m, int(backward), int(masked), ctypes.byref(out)),
           "mlproj_gated_ff_workspace_bytes")
    return out.value


def gated_ff_route(dtype, product, tokens, n, m):
    """How a product of a block with aligned rows is computed: {"kind", "packed", "parts", "low", "shares"} (see
    mlproj.h)."""
    r = lib().mlproj_gated_ff_route(_storage(dtype), product, tokens, n, m)
    if r < 0:
        _check(r, "mlproj_gated_ff_route")
    return {"kind": r & 15, "packed": bool(r & 16), "parts": bool(r & 32), "low": bool(r & 64), "shares": r >> 8}


def _gated_block(X, Wg, Wu, mask):
    assert X.dim() == 2 and Wg.dim() == 2
    tokens, n = X.shape
    m = Wg.shape[1]
    ldx = _matrix(X, (tokens, n), X, "X")
    ldw = _matrix(Wg, (n, m), X, "Wg")
    assert _matrix(Wu, (n, m), X, "Wu") == ldw, "Wg and Wu: one row stride"
    if mask is not None:
        assert mask.is_cuda and mask.element_size() == 1 and mask.is_contiguous() and mask.numel() == m, "mask: one byte per column"
    return GatedBlock(tokens, n, m, X.data_ptr(), ldx, Wg.data_ptr(), Wu.data_ptr(), ldw, _ptr(mask)), tokens, n, m


def gated_ff(X, Wg, Wu, act="silu", mask=None, H=None, g_out=None, u_out=None, workspace=None, stream=None):
    """H = mask * act(X Wg) * (X Wu): X is tokens x n, the weights n x m, all of one type (fp32, bf16, fp16), rows any
    distance apart.  act: "silu", "gelu" (with erf) or "relu"; mask: the kept-column mask of a projection.
    g_out, u_out: tensors that also receive X Wg and X Wu, for gated_ff_backward."""
    storage = _storage(X.dtype)
    block, tokens, n, m = _gated_block(X, Wg, Wu, mask)
    H, ldh = _result(H, (tokens, m), X, "H", stream)
    ldg = 0
    assert (g_out is None) == (u_out is None), "g_out and u_out: both or neither"
    if g_out is not None:
        ldg = _matrix(g_out, (tokens, m), X, "g_out")
        assert _matrix(u_out, (tokens, m), X, "u_out") == ldg, "g_out and u_out: one row stride"
    if workspace is None:
        workspace = Workspace(gated_ff_workspace_bytes(tokens, n, m, X.dtype, False, mask is not None), device=X.device, stream=stream)
    st = lib().gated_ff_forward(storage, _ACTS[act], ctypes.byref(block), H.data_ptr(), ldh, _ptr(g_out), _ptr(u_out),
                                ldg, workspace.buf.data_ptr(), workspace.nbytes, _stream(stream))
    if st != 0:
        _check(st, "gated_ff_forward")
    return H


def gated_ff_backward(dH, X, Wg, Wu, act="silu", mask=None, G=None, U=None, dX=None, dWg=None, dWu=None, workspace=None,
                      stream=None, need_dx=True, need_dw=True):
    """(dX, dWg, dWu) of gated_ff for the gradient dH of its result.  G, U: what the forward call wrote to g_out and
    u_out; without them they are computed again.  need_dx, need_dw: leave out what is not needed (None comes back)."""
    storage = _storage(X.dtype)
    block, tokens, n, m = _gated_block(X, Wg, Wu, mask)
    ldh = _matrix(dH, (tokens, m), X, "dH")
    assert (G is None) == (U is None), "G and U: both or neither"
    ldg = lddx = lddw = 0
    if G is not None:
        ldg = _matrix(G, (tokens, m), X, "G")
        assert _matrix(U, (tokens, m), X, "U") == ldg, "G and U: one row stride"
    if need_dx:
        dX, lddx = _result(dX, (tokens, n), X, "dX", stream)
    if need_dw:
        dWg, lddw = _result(dWg, (n, m), X, "dWg", stream)
        dWu, ld = _result(dWu, (n, m), X, "dWu", stream)
        assert ld == lddw, "dWg and dWu: one row stride"
    if workspace is None:
        workspace = Workspace(gated_ff_workspace_bytes(tokens, n, m, X.dtype, True, mask is not None), device=X.device, stream=stream)
    st = lib().gated_ff_backward(storage, _ACTS[act], ctypes.byref(block), dH.data_ptr(), ldh, _ptr(G), _ptr(U), ldg,
                                 _ptr(dX) if need_dx else None, lddx, _ptr(dWg) if need_dw else None,
                                 _ptr(dWu) if need_dw else None, lddw, workspace.buf.data_ptr(), workspace.nbytes,
                                 _stream(stream))
    if st != 0:
        _check(st, "gated_ff_backward")
    return (dX if need_dx else None, dWg if need_dw else None, dWu if need_dw else None)


def _vector(t, shape, like, what):
    assert t.dtype is like.dtype and t.is_cuda and t.shape == shape and t.is_contiguous(), what
    return t.data_ptr()


def _fixed(self, name, value):
    """What a structure of the library was made of stays as it is, or the two would differ."""
    if "_ref" in self.__dict__:
        raise AttributeError(f"{type(self).__name__}.{name} is fixed: make another one")
    object.__setattr__(self, name, value)


class Dropout:
    """Dropout whose mask is a function of the place of an entry (mlproj_dropout of include/mlproj.h): D(v) keeps an entry
    with probability 1 - p and divides it by 1 - p.  The same object in a call and in the call of its gradient is the
    same mask; calls with another `offset` (a number of the layer and the step, say) have independent ones.  step: a device tensor
    of one int64 that is added to offset when the kernels run, so that a captured graph's replays differ.  What counts is the sum:
    layers that share a seed and a step take offsets further apart than the step will ever go (layer << 40), or seeds of their
    own.  The object does not change: the next step has one of its own, or advances `step`."""
    __setattr__ = _fixed

    def __init__(self, p, seed, offset=0, step=None):
        if step is not None:
            assert step.is_cuda and step.element_size() == 8 and not step.is_floating_point() and step.numel() == 1, "step: one int64 on the device"
        self.p, self.seed, self.offset, self.step = p, seed, offset, step
        self._struct = DropoutStruct(p, seed & 0xffffffffffffffff, offset & 0xffffffffffffffff, _ptr(step))
        self._ref = ctypes.pointer(self._struct)


def dropout(x, drop, residual=None, y=None, stream=None):
    """y = residual + D(x), rows of x any distance apart; y may be x or residual (in place)."""
    assert x.dim() == 2
    storage, shape = _storage(x.dtype), x.shape
    ldx, ldr = _matrix(x, shape, x, "x"), 0
    if residual is not None:
        ldr = _matrix(residual, shape, x, "residual")
    y, ldy = _result(y, shape, x, "y", stream)
    st = lib().dropout_forward(storage, drop._ref, shape[0], shape[1], x.data_ptr(), ldx, _ptr(residual), ldr, y.data_ptr(), ldy,
                               _stream(stream))
    if st != 0:
        _check(st, "dropout_forward")
    return y


def dropout_backward(dy, drop, dx=None, stream=None):
    """dx = D(dy), the gradient of dropout (the residual's is dy itself); dx may be dy."""
    return dropout(dy, drop, y=dx, stream=stream)


def linear_workspace_bytes(tokens, n, m, dtype, backward=False):
    """Bytes a call of these sizes needs (one of fewer tokens may need more)."""
    out = ctypes.c_size_t(0)
    _check(lib().mlproj_linear_workspace_bytes(_storage(dtype), tokens, n, m, int(backward), ctypes.byref(out)),
           "mlproj_linear_workspace_bytes")
    return out.value


def linear(X, W, bias=None, residual=None, act=None, dropout=None, Y=None, z_out=None, workspace=None, stream=None):
    """Y = residual + D(act(X W + bias)): X is tokens x n, W n x m, all of one type (fp32, bf16, fp16), rows any distance
    apart.  act: None, "silu", "gelu" (with erf) or "relu"; dropout: a Dropout.  z_out: a tensor that also receives
    X W + bias, for linear_backward.  Y may be the residual (in place)."""
    assert X.dim() == 2 and W.dim() == 2
    storage = _storage(X.dtype)
    tokens, n = X.shape
    m = W.shape[1]
    shape = (tokens, m)
    block = LinearBlock(tokens, n, m, X.data_ptr(), _matrix(X, (tokens, n), X, "X"), W.data_ptr(), _matrix(W, (n, m), X, "W"),
                        None if bias is None else _vector(bias, (m,), X, "bias: m entries"), None if dropout is None else dropout._ref)
    ldr = ldz = 0
    if residual is not None:
        ldr = _matrix(residual, shape, X, "residual")
    if z_out is not None:
        ldz = _matrix(z_out, shape, X, "z_out")
    Y, ldy = _result(Y, shape, X, "Y", stream)
    if workspace is None:
        workspace = Workspace(linear_workspace_bytes(tokens, n, m, X.dtype), device=X.device, stream=stream)
    st = lib().linear_forward(storage, _ACTS[act], ctypes.byref(block), _ptr(residual), ldr, Y.data_ptr(), ldy, _ptr(z_out), ldz,
                              workspace.buf.data_ptr(), workspace.nbytes, _stream(stream))
    if st != 0:
        _check(st, "linear_forward")
    return Y


def linear_backward(dY, X, W, Z=None, act=None, dropout=None, dX=None, dW=None, workspace=None, stream=None, need_dx=True,
                    need_dw=True, need_dbias=False):
    """(dX, dW, dbias) of linear for the gradient dY of its result (the residual's gradient is dY itself).  Z: what the forward
    call wrote to z_out, needed with an activation; dropout: the forward call's.  dbias is in fp32; what is not needed is
    None, and then X (for dW) and W (for dX) are not read."""
    assert X.dim() == 2 and W.dim() == 2
    storage = _storage(X.dtype)
    tokens, n = X.shape
    m = W.shape[1]
    shape = (tokens, m)
    block = LinearBlock(tokens, n, m, X.data_ptr(), _matrix(X, (tokens, n), X, "X"), W.data_ptr(), _matrix(W, (n, m), X, "W"), None,
                        None if dropout is None else dropout._ref)
    lddy = _matrix(dY, shape, X, "dY")
    ldz = lddx = lddw = 0
    assert Z is not None or _ACTS[act] == ACT_NONE, "Z: the pre-activations of the forward call"
    if Z is not None:
        ldz = _matrix(Z, shape, X, "Z")
    dX, lddx = _result(dX, (tokens, n), X, "dX", stream) if need_dx else (None, 0)
    dW, lddw = _result(dW, (n, m), X, "dW", stream) if need_dw else (None, 0)
    dbias = _new_empty(X, m, _torch.float32, stream) if need_dbias else None
    if workspace is None:
        workspace = Workspace(linear_workspace_bytes(tokens, n, m, X.dtype, True), device=X.device, stream=stream)
    st = lib().linear_backward(storage, _ACTS[act], ctypes.byref(block), dY.data_ptr(), lddy, _ptr(Z), ldz, _ptr(dX), lddx,
                               _ptr(dW), lddw, _ptr(dbias), workspace.buf.data_ptr(), workspace.nbytes, _stream(stream))
    if st != 0:
        _check(st, "linear_backward")
    return dX, dW, dbias


def _norm_block(z, b, w_post, gate, w_pre, scale, eps):
    shape = z.shape
    tokens, n = shape
    row = (n,)
    pre = None if w_pre is None else _vector(w_pre, row, z, "w_pre: n entries")
    if b is None:
        return NormBlock(tokens, n, None, 0, None, None, 0, pre, scale, eps), shape, False
    ldb = _matrix(b, shape, z, "b")
    post = _vector(w_post, row, z, "w_post: n entries")
    token_gate = gate.dim() == 2
    if token_gate:
        stride, at = _matrix(gate, shape, z, "gate"), gate.data_ptr()
    else:
        stride, at = 0, _vector(gate, row, z, "gate: n entries, or tokens x n")
    return NormBlock(tokens, n, b.data_ptr(), ldb, post, at, stride, pre, scale, eps), shape, token_gate


def block_norm(x, b=None, w_post=None, gate=None, w_pre=None, scale=1.0, eps=1e-6, r=None, y=None, stream=None):
    """(r, y) with r = x + scale * gate * w_post * b / rms(b) and y = w_pre * r / rms(r), rows of n entries.  gate is
    a vector of n entries or a tokens x n matrix.  Without b, r is x itself; without w_pre there is no y.
    r may be x and y may be b (in place)."""
    assert x.dim() == 2
    storage = _storage(x.dtype)
    block, shape, _ = _norm_block(x, b, w_post, gate, w_pre, scale, eps)
    ldx = _matrix(x, shape, x, "x")
    at_r = at_y = None
    ldr = ldy = 0
    if b is None:
        r = x
    else:
        r, ldr = _result(r, shape, x, "r", stream)
        at_r = r.data_ptr()
    if w_pre is None:
        y = None
    else:
        y, ldy = _result(y, shape, x, "y", stream)
        at_y = y.data_ptr()
    st = lib().block_norm_forward(storage, ctypes.byref(block), x.data_ptr(), ldx, at_r, ldr, at_y, ldy, _stream(stream))
    if st != 0:
        _check(st, "block_norm_forward")
    return r, y


def block_norm_workspace_bytes(tokens, n):
    out = ctypes.c_size_t(0)
    _check(lib().mlproj_block_norm_workspace_bytes(tokens, n, ctypes.byref(out)), "mlproj_block_norm_workspace_bytes")
    return out.value


def block_norm_backward(dr, dy, r, b=None, w_post=None, gate=None, w_pre=None, scale=1.0, eps=1e-6, dx=None, db=None,
                        workspace=None, stream=None):
    """(dx, db, dw_post, dgate, dw_pre) of block_norm for the gradients dr (None: zeros) and dy (None without w_pre) of
    its results; r is what it returned.  The gradients of vectors are fp32 sums over the tokens, dgate of a
    tokens x n gate is a matrix like it; what has no input is None.  dx may be dr, db may be b or dy."""
    assert r.dim() == 2
    storage = _storage(r.dtype)
    f32 = _torch.float32
    if b is not None and gate.dim() == 2 and gate.stride(0) == 0 and gate.shape[0] > 1:
        # one row seen by all tokens: to the library a stride of 0 is a gate per channel, whose gradient is one row as well
        if stream is None:
            gate = gate.contiguous()
        else:
            with _torch.cuda.stream(stream):
                gate = gate.contiguous()
    block, shape, token_gate = _norm_block(r, b, w_post, gate, w_pre, scale, eps)
    tokens, n = shape
    ldr = _matrix(r, shape, r, "r")
    lddr = lddy = lddb = ldg = 0
    at_dy = at_db = at_post = at_gate = at_pre = dw_post = dgate = dw_pre = None
    if dr is not None:
        lddr = _matrix(dr, shape, r, "dr")
    dx, lddx = _result(dx, shape, r, "dx", stream)
    if b is None:
        db = None
    else:
        db, lddb = _result(db, shape, r, "db", stream)
        dw_post = _new_empty(r, n, f32, stream)
        if token_gate:
            dgate, ldg = _result(None, shape, r, "dgate", stream)
        else:
            dgate = _new_empty(r, n, f32, stream)
        at_db, at_post, at_gate = db.data_ptr(), dw_post.data_ptr(), dgate.data_ptr()
    if w_pre is not None:
        lddy = _matrix(dy, shape, r, "dy")
        dw_pre = _new_empty(r, n, f32, stream)
        at_dy, at_pre = dy.data_ptr(), dw_pre.data_ptr()
    if workspace is None:
        workspace = Workspace(block_norm_workspace_bytes(tokens, n), device=r.device, stream=stream)
    st = lib().block_norm_backward(storage, ctypes.byref(block), r.data_ptr(), ldr, _ptr(dr), lddr, at_dy, lddy, dx.data_ptr(),
                                   lddx, at_db, lddb, at_post, at_gate, ldg, at_pre, workspace.buf.data_ptr(),
                                   workspace.nbytes, _stream(stream))
    if st != 0:
        _check(st, "block_norm_backward")
    return dx, db, dw_post, dgate, dw_pre


class Q8:
    """A matrix in 8 bits (mlproj_q8 of include/mlproj.h): rows of n entries, each a code times the power of two of its 32
    neighbours.  codes: a float8_e4m3fn tensor of rows x n filled up with zeros to whole blocks of 128, scales: a float8_e8m0fnu
    tensor of rows x one per 32 of those; the rows of either may be further apart (codes by multiples of 16, scales of 4).  The tensors' entries may
    change, the object does not."""
    __setattr__ = _fixed

    def __init__(self, n, codes, scales):
        torch = _import_torch()
        rows, wide = codes.shape
        assert codes.is_cuda and codes.dtype is torch.float8_e4m3fn and wide == -(-n // 128) * 128, "codes: rows x n in whole blocks of 128, e4m3"
        assert scales.is_cuda and scales.dtype is torch.float8_e8m0fnu and scales.shape == (rows, wide // 32), "scales: one e8m0 per 32 codes"
        ld, lds = _matrix(codes, (rows, wide), codes, "codes"), _matrix(scales, (rows, wide // 32), scales, "scales")
        self.rows, self.n, self.codes, self.scales = rows, n, codes, scales
        self._struct = PackedQ8(rows, n, codes.data_ptr(), ld, scales.data_ptr(), lds)
        self._ref = ctypes.byref(self._struct)


def _new_q8(like, rows, n, stream):
    """A Q8 on memory of its own, without the checks of one that is given."""
    torch = _import_torch()
    wide = (n + 127) // 128 * 128
    q = Q8.__new__(Q8)
    codes = _new_empty(like, (rows, wide), torch.float8_e4m3fn, stream)
    scales = _new_empty(like, (rows, wide // 32), torch.float8_e8m0fnu, stream)
    struct = PackedQ8(rows, n, codes.data_ptr(), wide, scales.data_ptr(), wide // 32)
    q.__dict__.update(rows=rows, n=n, codes=codes, scales=scales, _struct=struct, _ref=ctypes.byref(struct))
    return q


def _result_q8(q, rows, n, like, what, stream):
    if q is None:
        return _new_q8(like, rows, n, stream)
    assert q.rows == rows and q.n == n, what
    return q


def q8_pack(A, columns=False, packed=None, stream=None):
    """Packs a device matrix (fp32, bf16, fp16) into a Q8: its rows, or with columns=True its columns, as a weight
    matrix n x m is held (m rows of n)."""
    assert A.dim() == 2
    rows, n = (A.shape[1], A.shape[0]) if columns else A.shape
    lda = _matrix(A, tuple(A.shape), A, "A")
    packed = _result_q8(packed, rows, n, A, "packed: the matrix's size", stream)
    st = lib().q8_pack(_storage(A.dtype), int(columns), A.data_ptr(), lda, packed._ref, _stream(stream))
    if st != 0:
        _check(st, "q8_pack")
    return packed


def block_norm8(x, b=None, w_post=None, gate=None, w_pre=None, scale=1.0, eps=1e-6, r=None, y=None, stream=None):
    """block_norm with y in 8 bits (a Q8), rounded from the y that is not yet rounded to x's type; w_pre is needed."""
    assert x.dim() == 2 and w_pre is not None
    storage = _storage(x.dtype)
    block, shape, _ = _norm_block(x, b, w_post, gate, w_pre, scale, eps)
    ldx, ldr, at_r = _matrix(x, shape, x, "x"), 0, None
    if b is None:
        r = x
    else:
        r, ldr = _result(r, shape, x, "r", stream)
        at_r = r.data_ptr()
    y = _result_q8(y, shape[0], shape[1], x, "y: a Q8 of x's size", stream)
    st = lib().block_norm8_forward(storage, ctypes.byref(block), x.data_ptr(), ldx, at_r, ldr, y._ref, _stream(stream))
    if st != 0:
        _check(st, "block_norm8_forward")
    return r, y


def q8_workspace_bytes(tokens, n, m, gated=False):
    """Bytes a call of these sizes needs (one of fewer tokens may need more)."""
    out = ctypes.c_size_t(0)
    _check(lib().mlproj_q8_workspace_bytes(tokens, n, m, int(gated), ctypes.byref(out)), "mlproj_q8_workspace_bytes")
    return out.value


def _q8_result(out, like, shape, dtype, what, stream):
    if out is None:
        return _new_empty(like, shape, dtype, stream), shape[1]
    return out, _matrix(out, shape, out, what)


def q8_linear(x, W, bias=None, residual=None, act=None, dtype=None, y=None, workspace=None, stream=None):
    """y = residual + act(x W + bias) with x (tokens of n) and W (packed by its columns) Q8s; bias, residual and y of one type:
    `dtype`, or that of the first of them there is, else bf16.  act: None, "silu", "gelu" or "relu".  y may be the residual."""
    torch = _import_torch()
    shape, given = (x.rows, W.rows), y if y is not None else residual if residual is not None else bias
    assert W.n == x.n, "x and W: rows of one length"
    if dtype is None:
        dtype = given.dtype if given is not None else torch.bfloat16
    storage = _storage(dtype)
    y, ldy = _q8_result(y, x.codes, shape, dtype, "y", stream)
    assert y.dtype is dtype, "y: of that type"
    at_bias = None if bias is None else _vector(bias, (W.rows,), y, "bias: one entry per column")
    ldr = 0 if residual is None else _matrix(residual, shape, y, "residual")
    if workspace is None:
        workspace = Workspace(q8_workspace_bytes(x.rows, x.n, W.rows), device=x.codes.device, stream=stream)
    st = lib().q8_linear(storage, _ACTS[act], x._ref, W._ref, at_bias, _ptr(residual), ldr, y.data_ptr(), ldy,
                         workspace.buf.data_ptr(), workspace.nbytes, _stream(stream))
    if st != 0:
        _check(st, "q8_linear")
    return y


def q8_gated(x, Wg, Wu, act="silu", dtype=None, h=None, workspace=None, stream=None):
    """h = act(x Wg) * (x Wu) with x, Wg and Wu Q8s (the weights packed by their columns, of one size); h of `dtype` (bf16)."""
    torch = _import_torch()
    shape = (x.rows, Wg.rows)
    assert Wg.n == x.n and Wu.n == x.n and Wu.rows == Wg.rows, "x, Wg and Wu: rows of one length"
    if dtype is None:
        dtype = h.dtype if h is not None else torch.bfloat16
    storage = _storage(dtype)
    h, ldh = _q8_result(h, x.codes, shape, dtype, "h", stream)
    assert h.dtype is dtype, "h: of that type"
    if workspace is None:
        workspace = Workspace(q8_workspace_bytes(x.rows, x.n, Wg.rows, True), device=x.codes.device, stream=stream)
    st = lib().q8_gated(storage, _ACTS[act], x._ref, Wg._ref, Wu._ref, h.data_ptr(), ldh, workspace.buf.data_ptr(), workspace.nbytes,
                        _stream(stream))
    if st != 0:
        _check(st, "q8_gated")
    return h


def w4_bytes(n, m, group):
    codes, scales = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().mlproj_w4_bytes(n, m, group, ctypes.byref(codes), ctypes.byref(scales)), "mlproj_w4_bytes")
    return codes.value, scales.value


class W4:
    """An n x m weight matrix in 4 bits with one bf16 scale per column and `group` rows (the layout is declared in
    include/mlproj.h); `codes` is a uint8 tensor, `scales` a bf16 tensor, both contiguous."""

    def __init__(self, n, m, group, codes, scales):
        torch = _import_torch()
        code_bytes, scale_bytes = w4_bytes(n, m, group)
        assert codes.is_cuda and codes.dtype == torch.uint8 and codes.is_contiguous() and codes.numel() == code_bytes
        assert scales.is_cuda and scales.dtype == torch.bfloat16 and scales.is_contiguous() and scales.numel() * 2 == scale_bytes
        self.n, self.m, self.group, self.codes, self.scales = n, m, group, codes, scales
        self._struct = PackedW4(n, m, group, codes.data_ptr(), scales.data_ptr())
        self._ref = ctypes.byref(self._struct)


def w4_pack(W, group=128, stream=None):
    """Packs a device matrix (fp32, bf16, fp16) into a W4."""
    torch = _import_torch()
    assert W.dim() == 2
    n, m = W.shape
    ldw = _matrix(W, (n, m), W, "W")
    code_bytes, scale_bytes = w4_bytes(n, m, group)
    packed = W4(n, m, group, _new_empty(W, code_bytes, torch.uint8, stream),
                _new_empty(W, scale_bytes // 2, torch.bfloat16, stream))
    _check(lib().w4_pack(_storage(W.dtype), W.data_ptr(), ldw, packed._ref, _stream(stream)), "w4_pack")
    return packed


def w4_matvec(x, W, y=None, stream=None):
    """y = x W for few tokens (x: tokens x n) and a packed W."""
    storage, tokens = _storage(x.dtype), x.shape[0]
    ldx = _matrix(x, (tokens, W.n), x, "x")
    y, ldy = _result(y, (tokens, W.m), x, "y", stream)
    st = lib().w4_matvec(storage, W._ref, x.data_ptr(), ldx, tokens, y.data_ptr(), ldy, _stream(stream))
    if st != 0:
        _check(st, "w4_matvec")
    return y


def w4_gated_matvec(x, Wg, Wu, act="silu", h=None, stream=None):
    """h = act(x Wg) * (x Wu) for few tokens and packed weights of one size and group."""
    storage, tokens = _storage(x.dtype), x.shape[0]
    ldx = _matrix(x, (tokens, Wg.n), x, "x")
    h, ldh = _result(h, (tokens, Wg.m), x, "h", stream)
    st = lib().w4_gated_matvec(storage, _ACTS[act], Wg._ref, Wu._ref, x.data_ptr(), ldx, tokens, h.data_ptr(), ldh,
                               _stream(stream))
    if st != 0:
        _check(st, "w4_gated_matvec")
    return h


class KernelTrace:
    """Times the kernels inside library calls with HIP events (mlproj_trace_begin / _end).

    with KernelTrace(capacity) as tr: ...calls...; tr.durations_ms() then gives the time
    between consecutive events, i.e. one entry per kernel launched, in launch order.
    """

    def __init__(self, capacity):
        self.hip = ctypes.CDLL("libamdhip64.so")
        self.capacity = capacity
        self.events = (ctypes.c_void_p * capacity)()
        for i in range(capacity):
            ev = ctypes.c_void_p()
            assert self.hip.hipEventCreate(ctypes.byref(ev)) == 0
            self.events[i] = ev
        self.count = 0

    def __enter__(self):
        _check(lib().mlproj_trace_begin(self.events, self.capacity), "mlproj_trace_begin")
        return self

    def __exit__(self, *exc):
        self.count = lib().mlproj_trace_end()
        return False

    def durations_ms(self):
        import torch
        torch.cuda.synchronize()
        out = []
        for i in range(self.count - 1):
            ms = ctypes.c_float()
            assert self.hip.hipEventElapsedTime(ctypes.byref(ms), ctypes.c_void_p(self.events[i]),
                                                ctypes.c_void_p(self.events[i + 1])) == 0
            out.append(ms.value)
        return out

    def close(self):
        for i in range(self.capacity):
            self.hip.hipEventDestroy(ctypes.c_void_p(self.events[i]))
