"""ctypes binding of libshampoo.so: the same entry points as include/shampoo.h
(the tensors of a step and of the training operators go through _marshal.so, csrc/marshal.cpp).

Argument marshalling only -- every step of the optimizer runs in the HIP
kernels of the library.  PyTorch is used for device memory and streams.
The library is loaded on first use and a missing library is an error: there
is no fallback path.
"""
import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libshampoo.so")

GRAD_F32, GRAD_BF16 = 0, 1
GET_L, GET_R, GET_LINV, GET_RINV, GET_A, GET_M, GET_PSH, GET_NORMS, GET_GF, GET_L2, GET_L2INV, GET_L3, GET_L3INV = range(13)
MAX_NDIM = 4
GRAFT_ADAGRAD, GRAFT_SGD, GRAFT_RMSPROP, GRAFT_ADAM = 0, 1, 2, 3
ROOT_EIGH, ROOT_NEWTON = 0, 1
LARGE_DIM_BLOCKING, LARGE_DIM_ADAGRAD, LARGE_DIM_DIAGONAL = 0, 1, 2
MATRIX_CORES_AUTO, MATRIX_CORES_FP32 = 0, 1
STAGE_FACTOR, STAGE_GRAFT, STAGE_ROOT, STAGE_PRECOND, STAGE_UPDATE, STAGE_DIAG, STAGE_FUSED, STAGE_PRECOND2 = range(8)
OUT_IN, IN_OUT = 0, 1
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
STAGE_NAMES = ("factor", "graft", "root", "precond", "update", "diag", "fused", "precond2")

EXPORTS = (
    "shampoo_plan", "shampoo_workspace_bytes", "shampoo_create", "shampoo_step", "shampoo_get",
    "shampoo_status", "shampoo_set_timing", "shampoo_get_timing", "shampoo_destroy",
    "shampoo_root_inverse_workspace_bytes", "shampoo_root_inverse", "shampoo_root_inverse_static",
    "shampoo_root_inverse_warm_workspace_bytes", "shampoo_root_inverse_warm",
    "shampoo_root_inverse_newton_workspace_bytes", "shampoo_root_inverse_newton", "shampoo_jacobi_pair",
    "shampoo_linear_cross_entropy_workspace_bytes", "shampoo_linear_cross_entropy",
    "shampoo_checkpoint_bytes", "shampoo_checkpoint_pack", "shampoo_checkpoint_unpack", "shampoo_checkpoint_activation_grad",
    "shampoo_checkpoint_weight_grad_workspace_bytes", "shampoo_checkpoint_weight_grad",
    "shampoo_residual_norm_forward", "shampoo_residual_norm_backward_workspace_bytes", "shampoo_residual_norm_backward",
    "shampoo_log_probs_workspace_bytes", "shampoo_log_probs", "shampoo_log_probs_grad",
    "shampoo_gradient_norm_workspace_bytes", "shampoo_gradient_norm",
    "shampoo_adamw_workspace_bytes", "shampoo_adamw_create", "shampoo_adamw_step", "shampoo_adamw_get", "shampoo_adamw_set", "shampoo_adamw_destroy",
    "shampoo_strerror",
)


class ShampooConfig(ctypes.Structure):
    _fields_ = [
        ("n_params", ctypes.c_int32),
        ("ndim", ctypes.POINTER(ctypes.c_int32)),
        ("shape", ctypes.POINTER(ctypes.c_int64)),
        ("block_size", ctypes.c_int32),
        ("beta2", ctypes.c_float),
        ("epsilon", ctypes.c_float),
        ("root_exponent", ctypes.c_float),
        ("precondition_frequency", ctypes.c_int32),
        ("start_preconditioning_step", ctypes.c_int32),
        ("graft_epsilon", ctypes.c_float),
        ("momentum", ctypes.c_float),
        ("beta1", ctypes.c_float),
        ("weight_decay", ctypes.c_float),
        ("use_decoupled_weight_decay", ctypes.c_int32),
        ("use_nesterov", ctypes.c_int32),
        ("grafting_type", ctypes.c_int32),
        ("grafting_beta2", ctypes.c_float),
        ("use_bias_correction", ctypes.c_int32),
        ("large_dim_method", ctypes.c_int32),
        ("root_method", ctypes.c_int32),
        ("newton_tolerance", ctypes.c_float),
        ("newton_max_iterations", ctypes.c_int32),
        ("precond_matrix_cores", ctypes.c_int32),
        ("warm_start_roots", ctypes.c_int32),
        ("grad_dtype", ctypes.c_int32),
        ("device", ctypes.c_int32),
    ]


class CrossEntropy(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in (
        "features", "classes", "dtype", "grad_dtype", "w_layout", "has_bias", "gradients")] + [
        (n, ctypes.c_int64) for n in ("ldx", "ldw", "lddx", "lddw")]


class ResidualNorm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("cols", "dtype", "post", "pre")] + [
        ("gates", ctypes.c_int64), ("epsilon", ctypes.c_float), ("scale", ctypes.c_float)] + [
        (n, ctypes.c_void_p) for n in ("w_post", "b_post", "gate", "w_pre", "b_pre")]


class Logits(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("classes", "tokens", "top", "dtype")] + [
        ("inverse_temperature", ctypes.c_float), ("ld", ctypes.c_int64)]


class AdamWConfig(ctypes.Structure):
    _fields_ = [("n_params", ctypes.c_int32), ("numel", ctypes.POINTER(ctypes.c_int64)), ("decay", ctypes.POINTER(ctypes.c_int32))] + [
        (n, ctypes.c_int32) for n in ("state_bits", "param_dtype", "grad_dtype", "device")] + [
        (n, ctypes.c_double) for n in ("beta1", "beta2", "epsilon", "weight_decay")]


_lib = None


def lib():
    """The loaded library (raises OSError if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise OSError(f"{LIB_PATH} not found: build it with `python -m paper_2309_06497_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    cfgp = ctypes.POINTER(ShampooConfig)
    L.shampoo_plan.argtypes = [cfgp, ctypes.POINTER(i64), i64, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    L.shampoo_plan.restype = ctypes.c_int
    L.shampoo_workspace_bytes.argtypes = [cfgp]
    L.shampoo_workspace_bytes.restype = sz
    L.shampoo_create.argtypes = [cfgp, vp, sz, vp, ctypes.POINTER(vp)]
    L.shampoo_create.restype = ctypes.c_int
    L.shampoo_step.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), f32, i64, vp]
    L.shampoo_step.restype = ctypes.c_int
    L.shampoo_get.argtypes = [vp, i32, i32, i32, vp, sz, vp]
    L.shampoo_get.restype = ctypes.c_int
    L.shampoo_status.argtypes = [vp, vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    L.shampoo_status.restype = ctypes.c_int
    L.shampoo_set_timing.argtypes = [vp, i32]
    L.shampoo_set_timing.restype = ctypes.c_int
    L.shampoo_get_timing.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]
    L.shampoo_get_timing.restype = ctypes.c_int
    L.shampoo_destroy.argtypes = [vp]
    L.shampoo_destroy.restype = ctypes.c_int
    L.shampoo_root_inverse_workspace_bytes.argtypes = [i32, i32]
    L.shampoo_root_inverse_workspace_bytes.restype = sz
    L.shampoo_root_inverse.argtypes = [vp, i32, i32, f32, f32, vp, vp, vp, vp, sz, vp]
    L.shampoo_root_inverse.restype = ctypes.c_int
    L.shampoo_root_inverse_warm_workspace_bytes.argtypes = [i32, i32]
    L.shampoo_root_inverse_warm_workspace_bytes.restype = sz
    L.shampoo_root_inverse_warm.argtypes = [vp, i32, i32, f32, f32, vp, vp, vp, vp, i32, vp, vp, sz, vp]
    L.shampoo_root_inverse_warm.restype = ctypes.c_int
    L.shampoo_root_inverse_static.argtypes = [vp, i32, i32, f32, f32, vp, vp, vp, vp]
    L.shampoo_root_inverse_static.restype = ctypes.c_int
    L.shampoo_root_inverse_newton_workspace_bytes.argtypes = [i32, i32]
    L.shampoo_root_inverse_newton_workspace_bytes.restype = sz
    L.shampoo_root_inverse_newton.argtypes = [vp, i32, i32, f32, i32, f32, i32, vp, vp, vp, vp, sz, vp]
    L.shampoo_root_inverse_newton.restype = ctypes.c_int
    L.shampoo_jacobi_pair.argtypes = [ctypes.c_int32] * 4 + [ctypes.POINTER(ctypes.c_int32)] * 2
    L.shampoo_jacobi_pair.restype = ctypes.c_int
    cep, rnp = ctypes.POINTER(CrossEntropy), ctypes.POINTER(ResidualNorm)
    L.shampoo_linear_cross_entropy_workspace_bytes.argtypes = [cep]
    L.shampoo_linear_cross_entropy_workspace_bytes.restype = sz
    L.shampoo_linear_cross_entropy.argtypes = [cep, vp, vp, vp, vp, vp, f32, vp, vp, vp, vp, vp, sz, vp]
    L.shampoo_linear_cross_entropy.restype = ctypes.c_int
    L.shampoo_checkpoint_bytes.argtypes = [i64, i32]
    L.shampoo_checkpoint_bytes.restype = sz
    L.shampoo_checkpoint_pack.argtypes = [vp, i32, i64, i32, i64, vp, sz, vp]
    L.shampoo_checkpoint_pack.restype = ctypes.c_int
    L.shampoo_checkpoint_unpack.argtypes = [vp, sz, i64, i32, i32, vp, i32, i64, vp]
    L.shampoo_checkpoint_unpack.restype = ctypes.c_int
    L.shampoo_checkpoint_activation_grad.argtypes = [vp, sz, i64, i32, i32, vp, i32, i64, vp, i64, vp]
    L.shampoo_checkpoint_activation_grad.restype = ctypes.c_int
    L.shampoo_checkpoint_weight_grad_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i64, i32, i32]
    L.shampoo_checkpoint_weight_grad_workspace_bytes.restype = sz
    L.shampoo_checkpoint_weight_grad.argtypes = [vp, sz, i64, i32, i32, vp, i32, i32, i64, vp, i32, i32, i64, vp, vp, sz, vp]
    L.shampoo_checkpoint_weight_grad.restype = ctypes.c_int
    L.shampoo_residual_norm_forward.argtypes = [rnp, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]
    L.shampoo_residual_norm_forward.restype = ctypes.c_int
    L.shampoo_residual_norm_backward_workspace_bytes.argtypes = [rnp]
    L.shampoo_residual_norm_backward_workspace_bytes.restype = sz
    L.shampoo_residual_norm_backward.argtypes = [rnp, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64] + [vp] * 5 + [vp, sz, vp]
    L.shampoo_residual_norm_backward.restype = ctypes.c_int
    lgp, awp, f64 = ctypes.POINTER(Logits), ctypes.POINTER(AdamWConfig), ctypes.c_double
    L.shampoo_log_probs_workspace_bytes.argtypes = [lgp]
    L.shampoo_log_probs_workspace_bytes.restype = sz
    L.shampoo_log_probs.argtypes = [lgp] + [vp] * 8 + [sz, vp]
    L.shampoo_log_probs.restype = ctypes.c_int
    L.shampoo_log_probs_grad.argtypes = [lgp] + [vp] * 6 + [i64, vp]
    L.shampoo_log_probs_grad.restype = ctypes.c_int
    L.shampoo_gradient_norm_workspace_bytes.argtypes = [i32, ctypes.POINTER(i64)]
    L.shampoo_gradient_norm_workspace_bytes.restype = sz
    L.shampoo_gradient_norm.argtypes = [i32, ctypes.POINTER(vp), ctypes.POINTER(i64), i32, vp, vp, vp, sz, vp]
    L.shampoo_gradient_norm.restype = ctypes.c_int
    L.shampoo_adamw_workspace_bytes.argtypes = [awp]
    L.shampoo_adamw_workspace_bytes.restype = sz
    L.shampoo_adamw_create.argtypes = [awp, vp, sz, vp, ctypes.POINTER(vp)]
    L.shampoo_adamw_create.restype = ctypes.c_int
    L.shampoo_adamw_step.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), f64, i64, vp, f32, vp]
    L.shampoo_adamw_step.restype = ctypes.c_int
    L.shampoo_adamw_get.argtypes = [vp, vp, vp, i32, vp]
    L.shampoo_adamw_get.restype = ctypes.c_int
    L.shampoo_adamw_set.argtypes = [vp, vp, vp, vp]
    L.shampoo_adamw_set.restype = ctypes.c_int
    L.shampoo_adamw_destroy.argtypes = [vp]
    L.shampoo_adamw_destroy.restype = ctypes.c_int
    L.shampoo_strerror.argtypes = [ctypes.c_int]
    L.shampoo_strerror.restype = ctypes.c_char_p
    _lib = L
    return L


class ShampooError(RuntimeError):
    def __init__(self, code):
        self.code = code
        super().__init__(f"libshampoo error {code}: {lib().shampoo_strerror(code).decode()}")


def _check(code):
    if code != 0:
        raise ShampooError(code)


def make_config(shapes, block_size, beta2, epsilon, root_exponent, precondition_frequency,
                start_preconditioning_step=0, graft_epsilon=1e-10, momentum=0.0,
                grad_dtype=GRAD_F32, device=0, beta1=0.0, weight_decay=0.0,
                use_decoupled_weight_decay=True, use_nesterov=False, grafting_type=GRAFT_ADAGRAD,
                use_bias_correction=False, root_method=ROOT_EIGH,
                newton_tolerance=1e-6, newton_max_iterations=100, grafting_beta2=0.999,
                large_dim_method=LARGE_DIM_BLOCKING, precond_matrix_cores=MATRIX_CORES_AUTO,
                warm_start_roots=False):
    """Builds a ShampooConfig; keeps the shape arrays alive on the returned object."""
    n = len(shapes)
    ndim = (ctypes.c_int32 * max(n, 1))(*[len(s) for s in shapes])
    flat = []
    for s in shapes:
        dims = [int(d) for d in s][:MAX_NDIM]
        flat += dims + [1] * (MAX_NDIM - len(dims))
    shape = (ctypes.c_int64 * max(MAX_NDIM * n, 1))(*flat)
    cfg = ShampooConfig(n, ndim, shape, block_size, beta2, epsilon, root_exponent,
                        precondition_frequency, start_preconditioning_step, graft_epsilon,
                        momentum, beta1, weight_decay, 1 if use_decoupled_weight_decay else 0,
                        1 if use_nesterov else 0, grafting_type, grafting_beta2, 1 if use_bias_correction else 0,
                        large_dim_method, root_method, newton_tolerance, newton_max_iterations,
                        precond_matrix_cores, 1 if warm_start_roots else 0, grad_dtype, device)
    cfg._keep = (ndim, shape)
    return cfg


def shampoo_plan(cfg):
    """Returns (table int64 [n_blocks, 12], n_buckets); rows are
    {param, row0, col0, m, n, bucket, slot, flags, s3, d3, s4, d4}.  Host only."""
    nb, nk = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(lib().shampoo_plan(ctypes.byref(cfg), None, 0, ctypes.byref(nb), ctypes.byref(nk)))
    table = np.zeros((max(nb.value, 1), 12), dtype=np.int64)
    _check(lib().shampoo_plan(ctypes.byref(cfg), table.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
                              nb.value, ctypes.byref(nb), ctypes.byref(nk)))
    return table[:nb.value], nk.value


def shampoo_workspace_bytes(cfg):
    return lib().shampoo_workspace_bytes(ctypes.byref(cfg))


def _stream_ptr(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


class Shampoo:
    """Owns the workspace tensor and the library handle for one parameter list."""

    def __init__(self, shapes, block_size, beta2, epsilon, root_exponent, precondition_frequency,
                 start_preconditioning_step=0, graft_epsilon=1e-10, momentum=0.0,
                 grad_dtype=GRAD_F32, device=0, beta1=0.0, weight_decay=0.0,
                 use_decoupled_weight_decay=True, use_nesterov=False, grafting_type=GRAFT_ADAGRAD,
                use_bias_correction=False, root_method=ROOT_EIGH,
                newton_tolerance=1e-6, newton_max_iterations=100, grafting_beta2=0.999,
                large_dim_method=LARGE_DIM_BLOCKING, precond_matrix_cores=MATRIX_CORES_AUTO,
                warm_start_roots=False):
        import torch
        self.shapes = [tuple(s) for s in shapes]
        self.cfg = make_config(self.shapes, block_size, beta2, epsilon, root_exponent,
                               precondition_frequency, start_preconditioning_step, graft_epsilon,
                               momentum, grad_dtype, device, beta1, weight_decay,
                               use_decoupled_weight_decay, use_nesterov, grafting_type,
                               use_bias_correction, root_method, newton_tolerance, newton_max_iterations,
                               grafting_beta2, large_dim_method, precond_matrix_cores, warm_start_roots)
        self.device = torch.device("cuda", device)
        self.grad_dtype = grad_dtype
        nbytes = shampoo_workspace_bytes(self.cfg)
        if nbytes == 0:
            raise ShampooError(lib().shampoo_plan(ctypes.byref(self.cfg), None, 0, None, None) or -2)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.handle = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().shampoo_create(ctypes.byref(self.cfg), ctypes.c_void_p(self.workspace.data_ptr()),
                                        nbytes, _stream_ptr(), ctypes.byref(self.handle)))
        from . import _marshal
        self._marshal = _marshal
        self._stepper = _marshal.make(ctypes.cast(lib().shampoo_step, ctypes.c_void_p).value, self.handle.value, device,
                                      grad_dtype == GRAD_BF16, self.shapes)

    def step(self, params, grads, lr, step):
        """params / grads: lists of contiguous CUDA tensors (float32 / float32-or-bfloat16)."""
        _check(self._marshal.step(self._stepper, params, grads, lr, step) if self.handle else -1)

    def get(self, param, block, which):
        import torch
        s = self.shapes[param]
        table = self.plan()[0]
        rows = table[table[:, 0] == param] if len(table) else table
        if len(rows) == 0:      # 1-D, or a matrix on the diagonal-method path
            shape = tuple(s)
        else:
            if not 0 <= block < len(rows):
                raise ShampooError(-2)
            m, n, flags, d3, d4 = (int(rows[block, k]) for k in (3, 4, 7, 9, 11))
            if flags & 4:        # a block of a tensor parameter: m x n x d3 (x d4), one factor per dimension
                blk = (m, n, d3, d4) if (flags >> 4) == 4 else (m, n, d3)
                dl = blk[-1]     # R / RINV belong to the last dimension
                shape = {GET_L: (m, m), GET_LINV: (m, m), GET_L2: (n, n), GET_L2INV: (n, n),
                         GET_L3: (d3, d3), GET_L3INV: (d3, d3),
                         GET_R: (dl, dl), GET_RINV: (dl, dl), GET_A: blk, GET_M: blk, GET_PSH: blk,
                         GET_NORMS: (2,), GET_GF: blk}[which]
            else:
                lshape = (m,) if flags & 1 else (m, m)
                rshape = (n,) if flags & 2 else (n, n)
                shape = {GET_L: lshape, GET_LINV: lshape, GET_R: rshape, GET_RINV: rshape,
                         GET_A: (m, n), GET_M: (m, n), GET_PSH: (m, n), GET_NORMS: (2,), GET_GF: (m, n)}[which]
        out = torch.empty(shape, dtype=torch.float32, device=self.device)
        _check(lib().shampoo_get(self.handle, param, block, which, ctypes.c_void_p(out.data_ptr()),
                                 out.numel() * 4, _stream_ptr()))
        return out

    def plan(self):
        if not hasattr(self, "_plan"):
            self._plan = shampoo_plan(self.cfg)
        return self._plan

    def status(self):
        a, b = ctypes.c_int64(0), ctypes.c_int64(0)
        _check(lib().shampoo_status(self.handle, _stream_ptr(), ctypes.byref(a), ctypes.byref(b)))
        return {"refreshes": a.value, "failed_roots": b.value}

    def set_timing(self, enable):
        _check(lib().shampoo_set_timing(self.handle, 1 if enable else 0))

    def get_timing(self):
        """{stage name: (total ms, intervals)} since the last call."""
        out = {}
        for st, name in enumerate(STAGE_NAMES):
            ms, cnt = ctypes.c_double(0), ctypes.c_int64(0)
            _check(lib().shampoo_get_timing(self.handle, st, ctypes.byref(ms), ctypes.byref(cnt)))
            out[name] = (ms.value, cnt.value)
        return out

    def destroy(self):
        if self.handle:
            self._stepper = None
            lib().shampoo_destroy(self.handle)
            self.handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# The stand-alone calls take their workspace from torch's allocator and give it back on return,
# while the work is still queued: the allocator hands freed memory to later work of the same
# stream only, and the library's helper streams have joined that stream by then.
def shampoo_root_inverse(a, epsilon, r, want_lambda=False, want_failed=False):
    """a: CUDA float32 tensor [batch, n, n] (symmetric).  Returns X [batch, n, n]
    (and eigenvalues [batch, n], failure flags [batch] on request)."""
    import torch
    assert a.is_cuda and a.dtype == torch.float32 and a.dim() == 3 and a.shape[1] == a.shape[2]
    a = a.contiguous()
    batch, n = a.shape[0], a.shape[1]
    x = torch.empty_like(a)
    lam = torch.empty((batch, n), dtype=torch.float32, device=a.device) if want_lambda else None
    failed = torch.zeros((batch,), dtype=torch.int32, device=a.device) if want_failed else None
    # with eigenvalues the call takes the solver of the warm start, which needs half as much
    size = "shampoo_root_inverse_warm_workspace_bytes" if want_lambda and n > 128 else "shampoo_root_inverse_workspace_bytes"
    nbytes = getattr(lib(), size)(n, batch)
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=a.device)
    with torch.cuda.device(a.device):
        _check(lib().shampoo_root_inverse(
            ctypes.c_void_p(a.data_ptr()), n, batch, epsilon, r, ctypes.c_void_p(x.data_ptr()),
            ctypes.c_void_p(lam.data_ptr()) if lam is not None else None,
            ctypes.c_void_p(failed.data_ptr()) if failed is not None else None,
            ctypes.c_void_p(ws.data_ptr()), ws.numel(), _stream_ptr()))
    res = [x]
    if want_lambda:
        res.append(lam)
    if want_failed:
        res.append(failed)
    return res[0] if len(res) == 1 else tuple(res)


def shampoo_root_inverse_warm(a, epsilon, r, qt, start):
    """shampoo_root_inverse with the eigenvectors kept in qt ([batch, np, np] float32 CUDA tensor,
    np = n rounded up to 64) between calls; start: begin from them.  Returns
    (X, eigenvalues, failed, sweeps)."""
    import torch
    assert a.is_cuda and a.dtype == torch.float32 and a.dim() == 3 and a.shape[1] == a.shape[2]
    a = a.contiguous()
    batch, n = a.shape[0], a.shape[1]
    npad = (n + 63) // 64 * 64
    assert qt.is_cuda and qt.dtype == torch.float32 and tuple(qt.shape) == (batch, npad, npad) and qt.is_contiguous()
    x = torch.empty_like(a)
    lam = torch.empty((batch, n), dtype=torch.float32, device=a.device)
    failed = torch.zeros((batch,), dtype=torch.int32, device=a.device)
    sweeps = torch.zeros((batch,), dtype=torch.int32, device=a.device)
    nbytes = lib().shampoo_root_inverse_warm_workspace_bytes(n, batch)
    if nbytes == 0:
        raise ShampooError(-7)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=a.device)
    with torch.cuda.device(a.device):
        _check(lib().shampoo_root_inverse_warm(
            ctypes.c_void_p(a.data_ptr()), n, batch, epsilon, r, ctypes.c_void_p(x.data_ptr()),
            ctypes.c_void_p(lam.data_ptr()), ctypes.c_void_p(failed.data_ptr()), ctypes.c_void_p(qt.data_ptr()),
            1 if start else 0, ctypes.c_void_p(sweeps.data_ptr()), ctypes.c_void_p(ws.data_ptr()), ws.numel(),
            _stream_ptr()))
    return x, lam, failed, sweeps


def shampoo_root_inverse_static(a, epsilon, r, x, lam=None, failed=None):
    """shampoo_root_inverse without a workspace (the library's fixed scratch array is used):
    a, x: CUDA float32 tensors [batch, n, n]; lam [batch, n] float32 and failed [batch] int32
    optional.  Outputs are written into the tensors given: nothing is allocated here either.
    Asynchronous on the current stream."""
    import torch
    assert a.is_cuda and a.dtype == torch.float32 and a.dim() == 3 and a.shape[1] == a.shape[2] and a.is_contiguous()
    assert x.is_cuda and x.dtype == torch.float32 and x.shape == a.shape and x.is_contiguous()
    batch, n = a.shape[0], a.shape[1]
    assert lam is None or (lam.dtype == torch.float32 and lam.shape == (batch, n) and lam.is_contiguous())
    assert failed is None or (failed.dtype == torch.int32 and failed.shape == (batch,) and failed.is_contiguous())
    with torch.cuda.device(a.device):
        _check(lib().shampoo_root_inverse_static(
            ctypes.c_void_p(a.data_ptr()), n, batch, epsilon, r, ctypes.c_void_p(x.data_ptr()),
            ctypes.c_void_p(lam.data_ptr()) if lam is not None else None,
            ctypes.c_void_p(failed.data_ptr()) if failed is not None else None, _stream_ptr()))


def shampoo_jacobi_pair(s, halves, rnd, k):
    """(p, q), p < q: pair k of round rnd of the eigensolver's sweep over s indices (host only)."""
    p, q = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().shampoo_jacobi_pair(s, int(halves), rnd, k, ctypes.byref(p), ctypes.byref(q)))
    return p.value, q.value


def shampoo_root_inverse_newton(a, epsilon, p, tolerance=1e-6, max_iterations=100, want_iterations=False,
                                want_failed=False):
    """a: CUDA float32 tensor [batch, n, n] (symmetric).  Returns X [batch, n, n], the coupled
    inverse Newton approximation of (a + epsilon I)^(-1/p) (and the iteration counts [batch],
    failure flags [batch] on request)."""
    import torch
    assert a.is_cuda and a.dtype == torch.float32 and a.dim() == 3 and a.shape[1] == a.shape[2]
    a = a.contiguous()
    batch, n = a.shape[0], a.shape[1]
    x = torch.empty_like(a)
    iters = torch.zeros((batch,), dtype=torch.int32, device=a.device) if want_iterations else None
    failed = torch.zeros((batch,), dtype=torch.int32, device=a.device) if want_failed else None
    nbytes = lib().shampoo_root_inverse_newton_workspace_bytes(n, batch)
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=a.device)
    with torch.cuda.device(a.device):
        _check(lib().shampoo_root_inverse_newton(
            ctypes.c_void_p(a.data_ptr()), n, batch, epsilon, p, tolerance, max_iterations,
            ctypes.c_void_p(x.data_ptr()),
            ctypes.c_void_p(iters.data_ptr()) if iters is not None else None,
            ctypes.c_void_p(failed.data_ptr()) if failed is not None else None,
            ctypes.c_void_p(ws.data_ptr()), ws.numel(), _stream_ptr()))
    res = [x]
    if want_iterations:
        res.append(iters)
    if want_failed:
        res.append(failed)
    return res[0] if len(res) == 1 else tuple(res)


# ----------------------------------------------------------------------------
# Operators of a training pass: checks of tensors, outputs and workspaces are csrc/marshal.cpp's.  Like the step they take tensors that
# require gradients and record nothing for automatic differentiation: their results are not part of any graph.
# ----------------------------------------------------------------------------
_ops = None
_codes = {}            # torch's types and the library's
_DTYPES = ()


def _load_ops():
    global _ops, _codes, _DTYPES
    import torch
    from . import _marshal
    L = lib()
    _marshal.use([ctypes.cast(getattr(L, "shampoo_" + name), ctypes.c_void_p).value for name in (
        "linear_cross_entropy_workspace_bytes", "linear_cross_entropy", "checkpoint_bytes", "checkpoint_pack", "checkpoint_unpack",
        "checkpoint_activation_grad", "checkpoint_weight_grad_workspace_bytes", "checkpoint_weight_grad", "residual_norm_forward",
        "residual_norm_backward_workspace_bytes", "residual_norm_backward", "log_probs_workspace_bytes", "log_probs", "log_probs_grad",
        "gradient_norm_workspace_bytes", "gradient_norm", "adamw_step", "adamw_get")])
    _codes = {torch.float32: GRAD_F32, torch.bfloat16: GRAD_BF16}
    _DTYPES = (torch.float32, torch.bfloat16)
    _ops = _marshal
    return _marshal


def _code(dtype):
    assert dtype in _codes, f"float32 or bfloat16, not {dtype}"
    return _codes[dtype]


def _result(r):
    """An operator's tensors; instead of them the library's error code"""
    if r.__class__ is int:
        raise ShampooError(r)
    return r


def shampoo_linear_cross_entropy(x, w, targets, bias=None, weight=None, scale=1.0, grad_dtype=None, gradients=True):
    """Loss of every row, lse(x w^T + bias) - (x w^T + bias)[target], and the gradients of scale * sum(weight * loss).

    x [n, d] and w [v, d]: CUDA, both float32 or both bfloat16; w may be the transposed view of a [d, v] matrix, dw then is one
    too.  targets [n] int64 (outside 0 ... v - 1: ignored), bias [v] and weight [n] float32.  Returns (loss, dx, dw, dbias),
    dbias None without a bias, dw of grad_dtype (default: the type of w); with gradients=False the loss alone."""
    ops = _ops or _load_ops()
    r = _result(ops.cross_entropy(x, w, targets, bias, weight, scale, None if grad_dtype is None else _code(grad_dtype), gradients))
    return r if gradients else r[0]


class Checkpoint:
    """An activation [rows, cols] in 8 bits (codes and shared exponents in one CUDA tensor)."""
    __slots__ = ("packed", "rows", "cols", "code")

    def __init__(self, packed, shape, code):
        self.packed, (self.rows, self.cols), self.code = packed, shape, code

    @property
    def dtype(self):
        """That of the packed matrix"""
        _ops or _load_ops()
        return _DTYPES[self.code]


def shampoo_checkpoint_pack(x):
    """Checkpoint of a CUDA matrix [rows, cols], float32 or bfloat16."""
    return Checkpoint(_result((_ops or _load_ops()).pack(x)), x.shape, _codes[x.dtype])


def shampoo_checkpoint_unpack(c, activation=ACT_NONE, dtype=None):
    """activation(x) [rows, cols] of what a checkpoint holds, in `dtype` (default: that of the packed matrix)."""
    ops = _ops or _load_ops()
    return _result(ops.unpack(c.packed, c.rows, c.cols, activation, c.code if dtype is None else _code(dtype)))


def shampoo_checkpoint_activation_grad(c, dy, activation):
    """dy * activation'(x) for the x that a checkpoint holds."""
    return _result((_ops or _load_ops()).activation_grad(c.packed, c.rows, c.cols, dy, activation))


def shampoo_checkpoint_weight_grad(c, dy, activation=ACT_NONE, grad_dtype=None, out_in=False, bias=False):
    """Gradient of the weight of y = activation(x) W from a checkpoint of x [rows, in] and dy [rows, out]: [in, out], or [out, in]
    with out_in; of grad_dtype (default: the type of dy).  With bias also the column sums of dy, float32."""
    ops = _ops or _load_ops()
    r = _result(ops.weight_grad(c.packed, c.rows, c.cols, dy, activation, None if grad_dtype is None else _code(grad_dtype), out_in, bias))
    return r if bias else r[0]


def shampoo_residual_norm_forward(r, f, post=NORM_RMS, pre=NORM_RMS, w_post=None, b_post=None, gate=None, w_pre=None, b_pre=None,
                                  epsilon=1e-5, scale=1.0, checkpoint=False):
    """r_out = r + scale * gate * norm_post(f) and h = norm_pre(r_out) (None where pre is NORM_NONE).  r, f [rows, cols], float32 or
    bfloat16; weights [cols] and gate [cols] or [gates, cols] (every rows / gates rows share one) float32.  With
    checkpoint also those of r and f, for the backward pass: (r_out, h, r8, f8)."""
    ops = _ops or _load_ops()
    r_out, h, r8, f8 = _result(ops.norm_forward(r, f, post, pre, w_post, b_post, gate, w_pre, b_pre, epsilon, scale, checkpoint))
    if not checkpoint:
        return r_out, h
    code = _codes[r.dtype]
    return r_out, h, Checkpoint(r8, r.shape, code), Checkpoint(f8, r.shape, code)


_NORM_GRADIENTS = ("dr", "df", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")


def shampoo_residual_norm_backward(r, f, dr_out, dh, post=NORM_RMS, pre=NORM_RMS, w_post=None, b_post=None, gate=None, w_pre=None,
                                   b_pre=None, epsilon=1e-5, scale=1.0):
    """Gradients of shampoo_residual_norm_forward from those of r_out (None: zero) and h (None where there is no h); r and f: the
    matrices, or the checkpoints that the forward pass wrote.  Returns a dict of dr, df, and float32 dgate, dw_post, db_post,
    dw_pre, db_pre, None for those of what is not there."""
    ops = _ops or _load_ops()
    if isinstance(r, Checkpoint):
        if not isinstance(f, Checkpoint) or (f.rows, f.cols, f.code) != (r.rows, r.cols, r.code):
            raise AssertionError("checkpoints of one shape and type are needed")
        out = ops.norm_backward(r.packed, f.packed, r.rows, r.cols, r.code, dr_out, dh, post, pre, w_post, b_post, gate, w_pre, b_pre, epsilon, scale)
    else:
        out = ops.norm_backward(r, f, 0, 0, None, dr_out, dh, post, pre, w_post, b_post, gate, w_pre, b_pre, epsilon, scale)
    return dict(zip(_NORM_GRADIENTS, _result(out)))


# ----------------------------------------------------------------------------
# Operators on given logits
# ----------------------------------------------------------------------------
class LogProbs:
    """What shampoo_log_probs returns: log_probs (of the given tokens, in their shape), entropy [n], and where alternatives were asked
    for top_tokens [n, top] int64 and top_log_probs [n, top]; statistics [n, 4] and temperature are the backward pass's."""
    __slots__ = ("log_probs", "entropy", "top_tokens", "top_log_probs", "statistics", "temperature")

    def __init__(self, log_probs, entropy, top_tokens, top_log_probs, statistics, temperature):
        self.log_probs, self.entropy, self.top_tokens, self.top_log_probs = log_probs, entropy, top_tokens, top_log_probs
        self.statistics, self.temperature = statistics, temperature


def shampoo_log_probs(logits, tokens, top=0, temperature=1.0):
    """Log probabilities of given tokens under softmax(logits / temperature), the entropy of every row and its `top` most probable tokens.

    logits [n, v]: CUDA, float32 or bfloat16.  tokens [n] or [n, m] int64, m at most 64 (outside 0 ... v - 1: ignored, log probability 0).  -inf masks a
    token.  Of equal logits the lower token is the more probable one; where fewer than top (at most 64) are left the rest is -1."""
    return LogProbs(*_result((_ops or _load_ops()).log_probs(logits, tokens, top, temperature)), temperature)


def shampoo_log_probs_grad(logits, tokens, forward, d_log_probs, d_entropy=None, out=None):
    """Gradient of the logits from those of `forward`'s log_probs (or None) and entropy (or None); logits and tokens as shampoo_log_probs had them.
    out: where it is written, the logits themselves where they are no longer needed."""
    return _result((_ops or _load_ops()).log_probs_grad(logits, tokens, forward.statistics, forward.temperature, d_log_probs, d_entropy, out))


# ----------------------------------------------------------------------------
# All tensors of a model
# ----------------------------------------------------------------------------
def shampoo_gradient_norm(grads):
    """(norm of all gradients together, norms [n] of each) on their device, float32, from sums in 64 bits.  grads: contiguous CUDA tensors, all float32 or
    all bfloat16."""
    return _result((_ops or _load_ops()).gradient_norm(grads))


class AdamW:
    """AdamW over one list of parameters: owns the workspace tensor, which holds all state, and the library handle.  decay: for every parameter
    whether weight_decay applies to it (default: to all).  Calls on several streams are ordered by the caller."""

    def __init__(self, shapes, beta1=0.9, beta2=0.999, epsilon=1e-8, weight_decay=0.01, decay=None, state_bits=32, param_dtype=GRAD_F32,
                 grad_dtype=GRAD_F32, device=0):
        import torch
        self.shapes = [tuple(int(d) for d in s) for s in shapes]
        n = len(self.shapes)
        sizes = [int(np.prod(s, dtype=object)) for s in self.shapes]
        self.total = sum(sizes)
        numel = (ctypes.c_int64 * max(n, 1))(*sizes)
        flags = None
        if decay is not None:
            if len(decay) != n:
                raise ValueError("one entry of decay per parameter")
            flags = (ctypes.c_int32 * max(n, 1))(*[1 if d else 0 for d in decay])
        self.cfg = AdamWConfig(n, numel, flags, state_bits, param_dtype, grad_dtype, device, beta1, beta2, epsilon, weight_decay)
        self.device, self.param_dtype, self.state_bits = torch.device("cuda", device), param_dtype, state_bits
        self.handle = ctypes.c_void_p()
        nbytes = lib().shampoo_adamw_workspace_bytes(ctypes.byref(self.cfg))
        if nbytes == 0:
            raise ShampooError(lib().shampoo_adamw_create(ctypes.byref(self.cfg), None, 0, None, ctypes.byref(self.handle)))
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        with torch.cuda.device(self.device):
            _check(lib().shampoo_adamw_create(ctypes.byref(self.cfg), ctypes.c_void_p(self.workspace.data_ptr()), nbytes, _stream_ptr(),
                                              ctypes.byref(self.handle)))
        size = 4 * self.total
        self._views = tuple(self.workspace[at:at + size].view(torch.float32) for at in (0, (size + 255) // 256 * 256)) if state_bits == 32 else None
        ops = _ops or _load_ops()
        self._step, self._state = ops.adamw_step, ops.adamw_state
        self._stepper = ops.make(0, self.handle.value, device, grad_dtype == GRAD_BF16, self.shapes)

    def step(self, params, grads, lr, step, copies=None, norm=None, max_norm=float("inf")):
        """One step, 0-based and strictly increasing.  params, grads: lists of contiguous CUDA tensors of the types given; params are updated in place, each
        tensor stands there once.  copies: bfloat16 tensors that get the updated float32 parameters.  norm: that of these gradients, as shampoo_gradient_norm
        returns it: they count as scaled down to max_norm, and nothing changes where it is not finite.  After a launch that failed (code -6) the step does not
        count, but some tensors may have had it: restore them and the state before it is tried again."""
        _check(self._step(self._stepper, params, grads, copies, lr, step, norm, max_norm, self.param_dtype) if self.handle else -1)

    def state(self):
        """(m, v) of all parameters, one behind the other: with 32 bits views of the optimizer's memory, with 8 bits the values that it holds, as
        bfloat16 (which holds them exactly)."""
        if not self.handle:
            raise ShampooError(-1)
        if self.state_bits == 32:
            return self._views
        return _result(self._state(self._stepper, self.total))

    def load(self, m, v):
        """The states of another optimizer, as state() gives them (any floating type)."""
        import torch
        if not self.handle:
            raise ShampooError(-1)
        assert all(x.is_cuda and x.device == self.device and x.numel() == self.total for x in (m, v)), "states of all elements on the optimizer's device"
        m, v = (x.reshape(-1).to(torch.float32).contiguous() for x in (m, v))
        with torch.cuda.device(self.device):
            _check(lib().shampoo_adamw_set(self.handle, ctypes.c_void_p(m.data_ptr()), ctypes.c_void_p(v.data_ptr()), _stream_ptr()))

    def destroy(self):
        if self.handle:
            self._stepper = None
            lib().shampoo_adamw_destroy(self.handle)
            self.handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
