"""Thin ctypes binding of the C ABI in ``include/hf.h``.

Argument marshalling only: every step of the gradient, the curvature products
and CG runs in the HIP kernels of ``libhf.so``.  PyTorch provides the device
memory (the tensors and the workspace) and the stream.  There is no other
backend: without the built library every call raises.
"""

import ctypes
import os

from paper_1606_00511_amd.buildid import source_hash

HERE = os.path.dirname(os.path.abspath(__file__))
# HF_LIB_PATH names another build of the same sources (the host-sanitizer
# build of the CPU tests); by default the in-tree library.
LIB_PATH = os.environ.get("HF_LIB_PATH") or os.path.join(HERE, "libhf.so")

HF_SIGMOID, HF_TANH, HF_RELU = 0, 1, 2
HF_HESSIAN, HF_GAUSS_NEWTON, HF_HYBRID = 0, 1, 2
HF_SOLVER_CG, HF_SOLVER_BICGSTAB = 0, 1
HF_FP32, HF_BF16_INPUTS = 0, 1
HF_OK, HF_EINVAL, HF_ENOMEM, HF_EHIP, HF_ELABEL, HF_ENUMERIC, HF_EWORKSPACE = \
    0, -1, -2, -3, -4, -5, -6

ACTS = {"sigmoid": HF_SIGMOID, "tanh": HF_TANH, "relu": HF_RELU}
MODES = {"hessian": HF_HESSIAN, "gauss_newton": HF_GAUSS_NEWTON}
CURVATURES = {"hessian": HF_HESSIAN, "gauss_newton": HF_GAUSS_NEWTON,
              "hybrid": HF_HYBRID}
SOLVERS = {"cg": HF_SOLVER_CG, "bicgstab": HF_SOLVER_BICGSTAB}
PRECS = {"fp32": HF_FP32, "bf16": HF_BF16_INPUTS}
# HFVocab: the type of rows, matrices and gradients
HF_TYPE_FP32, HF_TYPE_BF16 = 0, 1
TYPES = {"fp32": HF_TYPE_FP32, "bf16": HF_TYPE_BF16}
HF_IGNORE = -100          # a masked label, token or id
HF_VOCAB_MAX, HF_VOCAB_MAX_WIDTH = 1 << 22, 65536
HF_VOCAB_MAX_ROWS, HF_VOCAB_MAX_TOP = 262144, 128
# HFGated: its activations, and what a forward call keeps for the gradient
HF_SILU, HF_GELU, HF_GELU_TANH = 3, 4, 5
GATED_ACTS = dict(ACTS, silu=HF_SILU, gelu=HF_GELU, gelu_tanh=HF_GELU_TANH)
HF_KEEP_NONE, HF_KEEP_FULL, HF_KEEP_CODES = 0, 1, 2
KEEPS = {None: HF_KEEP_NONE, "full": HF_KEEP_FULL, "int8": HF_KEEP_CODES}
HF_GATED_MAX_WIDTH, HF_GATED_MAX_ROWS, HF_GATED_MAX_OUT = 65536, 262144, 1 << 22
HF_CODE_BLOCK = 32

# Every function declared in include/hf.h.
EXPORTS = (
    "hf_create", "hf_destroy", "hf_set_stream", "hf_num_params",
    "hf_workspace_bytes", "hf_set_workspace", "hf_loss_grad", "hf_hvp",
    "hf_cg", "hf_pcg", "hf_fisher_diag", "hf_bicgstab", "hf_pbicgstab", "hf_loss",
    "hf_iterate",
    "hf_set_trace", "hf_build_id", "hf_hvp_noalloc", "hf_check", "hf_last_error",
    "hf_strerror", "hf_prof_enable", "hf_prof_only",
    "hf_prof_reset", "hf_prof_count", "hf_prof_get",
    "hf_vocab_create", "hf_vocab_destroy", "hf_vocab_set_stream",
    "hf_vocab_workspace_bytes", "hf_vocab_set_workspace", "hf_vocab_loss",
    "hf_vocab_loss_grad", "hf_vocab_distill", "hf_vocab_distill_grad",
    "hf_vocab_embed", "hf_vocab_embed_grad", "hf_vocab_check",
    "hf_vocab_last_error",
    "hf_gated_create", "hf_gated_destroy", "hf_gated_set_stream",
    "hf_gated_workspace_bytes", "hf_gated_set_workspace", "hf_gated_forward",
    "hf_gated_grad", "hf_gated_pack", "hf_gated_unpack", "hf_gated_codes",
    "hf_gated_product", "hf_gated_forward_codes", "hf_gated_last_error",
)


class hf_cg_info(ctypes.Structure):
    _fields_ = [
        ("iters", ctypes.c_int32), ("products", ctypes.c_int32),
        ("neg_curv", ctypes.c_int32), ("neg_iter", ctypes.c_int32),
        ("pBp", ctypes.c_double), ("pHp", ctypes.c_double),
        ("gTd", ctypes.c_double), ("rr0", ctypes.c_double),
        ("rr_final", ctypes.c_double), ("status", ctypes.c_int32),
        ("replayed", ctypes.c_int32),
    ]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class hf_iter_params(ctypes.Structure):
    _fields_ = [
        ("solver", ctypes.c_int32), ("curvature", ctypes.c_int32),
        ("damping", ctypes.c_float), ("max_iters", ctypes.c_int32),
        ("rel_tol", ctypes.c_float), ("eta", ctypes.c_float),
        ("armijo_c", ctypes.c_float), ("shrink", ctypes.c_float),
        ("max_backtracks", ctypes.c_int32), ("adapt_damping", ctypes.c_int32),
        ("keep_cap", ctypes.c_int32), ("keep_buf", ctypes.c_void_p),
        ("precondition", ctypes.c_int32), ("precond_exp", ctypes.c_float),
    ]


class hf_iter_info(ctypes.Structure):
    _fields_ = [
        ("solve", hf_cg_info), ("mode_used", ctypes.c_int32),
        ("direction", ctypes.c_int32), ("accepted", ctypes.c_int32),
        ("evals", ctypes.c_int32), ("f0", ctypes.c_double),
        ("f1", ctypes.c_double), ("alpha", ctypes.c_double),
        ("gTd", ctypes.c_double), ("backtrack_iter", ctypes.c_int32),
        ("rho", ctypes.c_double), ("damping_next", ctypes.c_double),
    ]

    def as_dict(self):
        d = {k: getattr(self, k) for k, _ in self._fields_ if k != "solve"}
        d["solve"] = self.solve.as_dict()
        return d


class HFError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("%s: %s" % (strerror(code), msg))
        self.code = code


_lib = None


def lib():
    """Load libhf.so (raises if it has not been built, or if it was built
    from sources other than those beside it)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "libhf.so is not built (%s); run python -m paper_1606_00511_amd.build"
            % LIB_PATH)
    L = ctypes.CDLL(LIB_PATH)
    L.hf_build_id.restype = ctypes.c_char_p
    L.hf_build_id.argtypes = []
    built = L.hf_build_id().decode()
    want = source_hash()
    if built != want:
        raise RuntimeError(
            "libhf.so (%s) was built from other sources (build id %s, sources %s);"
            " rebuild with python -m paper_1606_00511_amd.build"
            % (LIB_PATH, built[:16], want[:16]))
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    F32, D = ctypes.c_float, ctypes.c_double
    sig = {
        "hf_create": (ctypes.c_int, [ctypes.POINTER(I32), I32, I32, I32, I64,
                                     P, ctypes.POINTER(P)]),
        "hf_destroy": (ctypes.c_int, [P]),
        "hf_set_stream": (ctypes.c_int, [P, P]),
        "hf_num_params": (I64, [P]),
        "hf_workspace_bytes": (SZ, [P, I64]),
        "hf_set_workspace": (ctypes.c_int, [P, P, SZ]),
        "hf_loss_grad": (ctypes.c_int, [P, P, P, P, I64, P, P]),
        "hf_hvp": (ctypes.c_int, [P, P, P, P, I64, P, I32, P]),
        "hf_hvp_noalloc": (ctypes.c_int, [P, P, P, P, I64, P, I32, P, P]),
        "hf_cg": (ctypes.c_int, [P, P, P, P, I64, P, F32, I32, F32, I32, P, P,
                                 ctypes.POINTER(hf_cg_info)]),
        "hf_bicgstab": (ctypes.c_int, [P, P, P, P, I64, P, F32, I32, F32, I32, P,
                                       P, ctypes.POINTER(hf_cg_info)]),
        "hf_pcg": (ctypes.c_int, [P, P, P, P, I64, P, F32, I32, F32, I32, P, P, P,
                                  ctypes.POINTER(hf_cg_info)]),
        "hf_pbicgstab": (ctypes.c_int, [P, P, P, P, I64, P, F32, I32, F32, I32, P,
                                        P, P, ctypes.POINTER(hf_cg_info)]),
        "hf_fisher_diag": (ctypes.c_int, [P, P, P, P, I64, P]),
        "hf_loss": (ctypes.c_int, [P, P, P, P, I64, P]),
        "hf_iterate": (ctypes.c_int, [P, P, P, P, I64, P, P, I64,
                                      ctypes.POINTER(hf_iter_params),
                                      ctypes.POINTER(I32), P,
                                      ctypes.POINTER(hf_iter_info)]),
        "hf_set_trace": (ctypes.c_int, [P, P, I32]),
        "hf_build_id": (ctypes.c_char_p, []),
        "hf_check": (ctypes.c_int, [P]),
        "hf_last_error": (ctypes.c_char_p, [P]),
        "hf_strerror": (ctypes.c_char_p, [I32]),
        "hf_prof_enable": (ctypes.c_int, [P, I32]),
        "hf_prof_only": (ctypes.c_int, [P, ctypes.c_char_p]),
        "hf_prof_reset": (ctypes.c_int, [P]),
        "hf_prof_count": (I32, [P]),
        "hf_prof_get": (ctypes.c_int, [P, I32, ctypes.POINTER(ctypes.c_char_p),
                                       ctypes.POINTER(I64), ctypes.POINTER(D),
                                       ctypes.POINTER(D), ctypes.POINTER(D)]),
        "hf_vocab_create": (ctypes.c_int, [I64, I32, I32, I64, P, ctypes.POINTER(P)]),
        "hf_vocab_destroy": (ctypes.c_int, [P]),
        "hf_vocab_set_stream": (ctypes.c_int, [P, P]),
        "hf_vocab_workspace_bytes": (SZ, [P, I64]),
        "hf_vocab_set_workspace": (ctypes.c_int, [P, P, SZ]),
        "hf_vocab_loss": (ctypes.c_int, [P, P, I64, P, I64, P, I64, F32, P, P]),
        "hf_vocab_loss_grad": (ctypes.c_int, [P, P, I64, P, I64, P, I64, F32, P, P,
                                              P, I64, P, I64, I32]),
        "hf_vocab_distill": (ctypes.c_int, [P, P, I64, P, I64, P, I64, P, I64, I32,
                                            F32, I64, F32, P, P]),
        "hf_vocab_distill_grad": (ctypes.c_int, [P, P, I64, P, I64, P, I64, P, I64,
                                                 I32, F32, I64, F32, P, P, P, I64, P,
                                                 I64, I32]),
        "hf_vocab_embed": (ctypes.c_int, [P, P, I64, P, I64, F32, P, I64]),
        "hf_vocab_embed_grad": (ctypes.c_int, [P, P, I64, F32, P, I64, P, I64, I32]),
        "hf_vocab_check": (ctypes.c_int, [P]),
        "hf_vocab_last_error": (ctypes.c_char_p, [P]),
        "hf_gated_create": (ctypes.c_int, [I32, I32, I32, I32, I64, P, ctypes.POINTER(P)]),
        "hf_gated_destroy": (ctypes.c_int, [P]),
        "hf_gated_set_stream": (ctypes.c_int, [P, P]),
        "hf_gated_workspace_bytes": (SZ, [P, I64]),
        "hf_gated_set_workspace": (ctypes.c_int, [P, P, SZ]),
        "hf_gated_forward": (ctypes.c_int, [P] + [P, I64] * 4 + [I64, P, I64, I32, P, I64, P,
                                                                 I64]),
        "hf_gated_grad": (ctypes.c_int, [P] + [P, I64] * 5 + [I32] + [P, I64] * 3 + [I64]
                          + [P, I64] * 4 + [I32]),
        "hf_gated_pack": (ctypes.c_int, [P, P, I64, I64, I64, P, I64, P, I64]),
        "hf_gated_unpack": (ctypes.c_int, [P, P, I64, P, I64, I64, I64, P, I64]),
        "hf_gated_codes": (ctypes.c_int, [P, P, I64, I64, I64, P, I64, P]),
        "hf_gated_product": (ctypes.c_int, [P, P, I64, P, P, I64, P, I64, I64, I64, P, I64]),
        "hf_gated_forward_codes": (ctypes.c_int, [P, P, I64] + [P, I64, P] * 3 + [I64, P, I64]),
        "hf_gated_last_error": (ctypes.c_char_p, [P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def strerror(code):
    return lib().hf_strerror(code).decode()


def _ptr(t, dtype, numel, what):
    """Device pointer of a contiguous CUDA tensor, after checking it."""
    import torch
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError("%s must be a CUDA tensor" % what)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (what, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % what)
    if numel is not None and t.numel() != numel:
        raise ValueError("%s has %d elements, expected %d" % (what, t.numel(), numel))
    return t.data_ptr()


class HFNet:
    """One context of the C library plus its torch-allocated workspace.

    dims: (d_0, ..., d_L); act: "sigmoid" | "tanh" | "relu"; max_batch: the
    largest batch any call will use; prec: "fp32" or "bf16" (bf16 GEMM
    operands, fp32 accumulation); ws_batch: size the workspace for calls of
    up to this many rows only (default max_batch).  Calls run on torch's
    current stream.
    """

    def __init__(self, dims, act, max_batch, device="cuda", prec="fp32",
                 ws_batch=None):
        import torch
        self.dims = tuple(int(d) for d in dims)
        self.act = act
        self.prec = prec
        self.max_batch = int(max_batch)
        L = lib()
        arr = (ctypes.c_int32 * len(self.dims))(*self.dims)
        h = ctypes.c_void_p()
        rc = L.hf_create(arr, len(self.dims), ACTS[act], PRECS[prec],
                         self.max_batch, None, ctypes.byref(h))
        if rc != HF_OK:
            raise HFError(rc, "hf_create rejected dims=%s act=%s max_batch=%d prec=%s"
                          % (self.dims, act, self.max_batch, prec))
        self._h = h
        self._last = None                 # stream of the last call
        self.n = int(L.hf_num_params(h))
        nbytes = int(L.hf_workspace_bytes(
            h, self.max_batch if ws_batch is None else int(ws_batch)))
        if nbytes == 0:
            raise ValueError("ws_batch %s outside [1, %d]" % (ws_batch, self.max_batch))
        self.device = torch.device(device)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self._check(L.hf_set_workspace(h, self.workspace.data_ptr(), nbytes))

    # ------------------------------------------------------------- plumbing
    def _check(self, rc):
        if rc != HF_OK:
            raise HFError(rc, lib().hf_last_error(self._h).decode())
        return rc

    def _stream(self):
        import torch
        current = torch.cuda.current_stream(self.device)
        if current.cuda_stream != self._last:
            # the allocator keeps the workspace until this stream's work is done
            self.workspace.record_stream(current)
            self._last = current.cuda_stream
        self._check(lib().hf_set_stream(self._h, current.cuda_stream))

    def close(self):
        if getattr(self, "_h", None) is not None:
            lib().hf_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, X):
        if X.dim() != 2 or X.shape[1] != self.dims[0]:
            raise ValueError("X must be B x %d" % self.dims[0])
        return int(X.shape[0])

    # -------------------------------------------------------------- the ABI
    def hf_loss_grad(self, W, X, y, loss=None, grad=None):
        import torch
        B = self._rows(X)
        if loss is None:
            loss = torch.empty(1, dtype=torch.float32, device=self.device)
        if grad is None:
            grad = torch.empty(self.n, dtype=torch.float32, device=self.device)
        self._stream()
        self._check(lib().hf_loss_grad(
            self._h, _ptr(W, torch.float32, self.n, "W"),
            _ptr(X, torch.float32, None, "X"), _ptr(y, torch.int32, B, "y"), B,
            _ptr(loss, torch.float32, 1, "loss"),
            _ptr(grad, torch.float32, self.n, "grad")))
        return loss, grad

    def hf_hvp(self, W, X, y, v, mode="hessian", out=None):
        import torch
        B = self._rows(X)
        if out is None:
            out = torch.empty(self.n, dtype=torch.float32, device=self.device)
        self._stream()
        self._check(lib().hf_hvp(
            self._h, _ptr(W, torch.float32, self.n, "W"),
            _ptr(X, torch.float32, None, "X"),
            _ptr(y, torch.int32, B, "y") if y is not None else None, B,
            _ptr(v, torch.float32, self.n, "v"), MODES[mode],
            _ptr(out, torch.float32, self.n, "out")))
        return out

    def hf_cg(self, W, Xc, yc, g, damping, max_iters, mode="hessian",
              rel_tol=0.0, step=None, neg_dir=None):
        return self._solve("hf_cg", W, Xc, yc, g, damping, max_iters, mode,
                           rel_tol, step, neg_dir)

    def hf_bicgstab(self, W, Xc, yc, g, damping, max_iters, mode="hessian",
                    rel_tol=0.0, step=None, neg_dir=None):
        return self._solve("hf_bicgstab", W, Xc, yc, g, damping, max_iters,
                           mode, rel_tol, step, neg_dir)

    def _solve(self, fn, W, Xc, yc, g, damping, max_iters, mode, rel_tol, step,
               neg_dir):
        import torch
        B = self._rows(Xc)
        if step is None:
            step = torch.empty(self.n, dtype=torch.float32, device=self.device)
        if neg_dir is None:
            neg_dir = torch.empty(self.n, dtype=torch.float32, device=self.device)
        info = hf_cg_info()
        self._stream()
        rc = getattr(lib(), fn)(
            self._h, _ptr(W, torch.float32, self.n, "W"),
            _ptr(Xc, torch.float32, None, "Xc"),
            _ptr(yc, torch.int32, B, "yc") if yc is not None else None, B,
            _ptr(g, torch.float32, self.n, "g"), float(damping), int(max_iters),
            float(rel_tol), MODES[mode], _ptr(step, torch.float32, self.n, "step"),
            _ptr(neg_dir, torch.float32, self.n, "neg_dir"), ctypes.byref(info))
        self._check(rc)
        return step, neg_dir, info.as_dict()

    def hf_pcg(self, W, Xc, yc, g, minv, damping, max_iters, mode="hessian",
               rel_tol=0.0, step=None, neg_dir=None):
        """CG preconditioned by diag(minv) = M^-1 (hf_pcg)."""
        return self._psolve("hf_pcg", W, Xc, yc, g, minv, damping, max_iters,
                            mode, rel_tol, step, neg_dir)

    def hf_pbicgstab(self, W, Xc, yc, g, minv, damping, max_iters,
                     mode="hessian", rel_tol=0.0, step=None, neg_dir=None):
        """Bi-CG-STAB preconditioned on the right by diag(minv) = M^-1
        (hf_pbicgstab)."""
        return self._psolve("hf_pbicgstab", W, Xc, yc, g, minv, damping,
                            max_iters, mode, rel_tol, step, neg_dir)

    def _psolve(self, fn, W, Xc, yc, g, minv, damping, max_iters, mode,
                rel_tol, step, neg_dir):
        import torch
        B = self._rows(Xc)
        if step is None:
            step = torch.empty(self.n, dtype=torch.float32, device=self.device)
        if neg_dir is None:
            neg_dir = torch.empty(self.n, dtype=torch.float32, device=self.device)
        info = hf_cg_info()
        self._stream()
        self._check(getattr(lib(), fn)(
            self._h, _ptr(W, torch.float32, self.n, "W"),
            _ptr(Xc, torch.float32, None, "Xc"),
            _ptr(yc, torch.int32, B, "yc") if yc is not None else None, B,
            _ptr(g, torch.float32, self.n, "g"), float(damping), int(max_iters),
            float(rel_tol), MODES[mode], _ptr(minv, torch.float32, self.n, "minv"),
            _ptr(step, torch.float32, self.n, "step"),
            _ptr(neg_dir, torch.float32, self.n, "neg_dir"), ctypes.byref(info)))
        return step, neg_dir, info.as_dict()

    def hf_fisher_diag(self, W, X, y, out=None):
        """(1/B) sum_b grad l_b^2 (hf_fisher_diag)."""
        import torch
        B = self._rows(X)
        if out is None:
            out = torch.empty(self.n, dtype=torch.float32, device=self.device)
        self._stream()
        self._check(lib().hf_fisher_diag(
            self._h, _ptr(W, torch.float32, self.n, "W"),
            _ptr(X, torch.float32, None, "X"), _ptr(y, torch.int32, B, "y"), B,
            _ptr(out, torch.float32, self.n, "out")))
        return out

    def hf_loss(self, W, X, y, loss=None):
        import torch
        B = self._rows(X)
        if loss is None:
            loss = torch.empty(1, dtype=torch.float32, device=self.device)
        self._stream()
        self._check(lib().hf_loss(
            self._h, _ptr(W, torch.float32, self.n, "W"),
            _ptr(X, torch.float32, None, "X"), _ptr(y, torch.int32, B, "y"), B,
            _ptr(loss, torch.float32, 1, "loss")))
        return loss

    def hf_iterate(self, W, X, y, Xc, yc, delta, solver="cg",
                   curvature="hessian", damping=1e-2, max_iters=10, rel_tol=0.0,
                   eta=0.0, armijo_c=1e-4, shrink=0.5, max_backtracks=20,
                   hybrid_state=0, adapt_damping=False, keep=None,
                   precondition=False, precond_exp=0.75):
        """One outer HF iteration; W and delta are updated in place.
        keep: None, or a CUDA float32 tensor of cap x n for the iterates that
        CG-backtracking keeps (cap = keep.shape[0]).  adapt_damping: report
        rho and the next lambda (info["damping_next"]).  precondition:
        the solver (PCG, or Bi-CG-STAB preconditioned on the right) with
        M = (F + lambda)^precond_exp.
        Returns (info dict, the new hybrid state)."""
        import torch
        B = self._rows(X)
        Bc = self._rows(Xc)
        cap, kbuf = 0, None
        if keep is not None:
            if keep.dim() != 2 or keep.shape[1] != self.n:
                raise ValueError("keep must be cap x %d" % self.n)
            cap = int(keep.shape[0])
            kbuf = _ptr(keep, torch.float32, None, "keep")
        prm = hf_iter_params(SOLVERS[solver], CURVATURES[curvature],
                             float(damping), int(max_iters), float(rel_tol),
                             float(eta), float(armijo_c), float(shrink),
                             int(max_backtracks), 1 if adapt_damping else 0,
                             cap, kbuf, 1 if precondition else 0,
                             float(precond_exp))
        hs = ctypes.c_int32(int(hybrid_state))
        info = hf_iter_info()
        self._stream()
        self._check(lib().hf_iterate(
            self._h, _ptr(W, torch.float32, self.n, "W"),
            _ptr(X, torch.float32, None, "X"), _ptr(y, torch.int32, B, "y"), B,
            _ptr(Xc, torch.float32, None, "Xc"),
            _ptr(yc, torch.int32, Bc, "yc") if yc is not None else None, Bc,
            ctypes.byref(prm), ctypes.byref(hs),
            _ptr(delta, torch.float32, self.n, "delta"), ctypes.byref(info)))
        return info.as_dict(), int(hs.value)

    def hf_check(self):
        self._check(lib().hf_check(self._h))

    def set_trace(self, cap):
        """Record the operand and result of the first `cap` curvature
        products of every later solve (hf_set_trace); cap = 0 turns it off.
        Returns the 2 cap x n trace tensor: row 2k the operand v of product
        k, row 2k + 1 the undamped product A v."""
        import torch
        if cap <= 0:
            self._check(lib().hf_set_trace(self._h, None, 0))
            self._trace = None
            return None
        buf = torch.full((2 * int(cap), self.n), float("nan"), dtype=torch.float32,
                         device=self.device)
        self._check(lib().hf_set_trace(self._h, buf.data_ptr(), int(cap)))
        self._trace = buf   # kept alive while tracing is on
        return buf

    # ------------------------------------------------------------ profiling
    def prof_enable(self, on=True):
        self._check(lib().hf_prof_enable(self._h, 1 if on else 0))

    def prof_only(self, name=None):
        """Time only the launches of kernel `name` (None: every kernel)."""
        self._check(lib().hf_prof_only(self._h, name.encode() if name else None))

    def prof_reset(self):
        self._check(lib().hf_prof_reset(self._h))

    def prof_stats(self):
        L = lib()
        out = {}
        for i in range(int(L.hf_prof_count(self._h))):
            name = ctypes.c_char_p()
            launches = ctypes.c_int64()
            ms, fl, by = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
            self._check(L.hf_prof_get(self._h, i, ctypes.byref(name),
                                      ctypes.byref(launches), ctypes.byref(ms),
                                      ctypes.byref(fl), ctypes.byref(by)))
            out[name.value.decode()] = dict(launches=launches.value, ms=ms.value,
                                            flops=fl.value, bytes=by.value)
        return out


class _RowContext:
    """What HFVocab and HFGated share: a context of the C library whose calls
    work on rows, its workspace, and the checks of tensors.  _prefix: of the C
    calls' names."""

    # torch's current device and stream as plain numbers, where it gives them: a
    # stream object takes 1.5 us to make, a small call 10
    _device = _raw_stream = None

    def _open(self, h, ws_rows, device):
        """The context h's workspace for calls of ws_rows rows (None: max_rows)."""
        torch, L = self._torch, lib()
        self._h = h
        self._stream = None               # of the last call
        nbytes = int(getattr(L, self._prefix + "_workspace_bytes")(
            h, self.max_rows if ws_rows is None else int(ws_rows)))
        if nbytes == 0:
            raise ValueError("ws_rows %s outside [1, %d]" % (ws_rows, self.max_rows))
        device = torch.device(device)
        if device.type == "cuda" and device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self.device = device
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        with torch.cuda.device(self.device):
            self._check(getattr(L, self._prefix + "_set_workspace")(
                h, self.workspace.data_ptr(), nbytes))
        self._device = getattr(torch._C, "_cuda_getDevice", None)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

    # ------------------------------------------------------------- plumbing
    def _check(self, rc):
        if rc != HF_OK:
            raise HFError(rc, getattr(lib(), self._prefix + "_last_error")(self._h).decode())
        return rc

    def _call(self, fn, *args):
        cuda, L = self._torch.cuda, lib()
        if self._device() != self.device.index if self._device else \
                cuda.current_device() != self.device.index:
            with cuda.device(self.device):
                return self._call(fn, *args)
        if self._raw_stream:
            stream = self._raw_stream(self.device.index)
        else:
            stream = cuda.current_stream(self.device.index).cuda_stream
        if stream != self._stream:
            self.workspace.record_stream(cuda.current_stream(self.device.index))
            self._stream = None
            self._check(getattr(L, self._prefix + "_set_stream")(self._h, stream))
            self._stream = stream
        return self._check(getattr(L, fn)(self._h, *args))

    def close(self):
        if getattr(self, "_h", None) is not None:
            getattr(lib(), self._prefix + "_destroy")(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _mat(self, t, rows, cols, dtype, what):
        """(pointer, elements between rows) of a rows x cols tensor."""
        if not isinstance(t, self._torch.Tensor) or t.device != self.device:
            raise TypeError("%s must be a tensor on %s" % (what, self.device))
        if t.dtype is not dtype:
            raise TypeError("%s must be %s, got %s" % (what, dtype, t.dtype))
        if t.shape != (rows, cols):
            raise ValueError("%s is %s, expected %d x %d"
                             % (what, tuple(t.shape), rows, cols))
        ld, one = t.stride()
        if cols > 1 and one != 1:
            raise ValueError("the rows of %s must be contiguous" % what)
        if rows <= 1:
            ld = cols
        elif ld < cols:
            raise ValueError("the rows of %s overlap" % what)
        return t.data_ptr(), ld

    def _vec(self, t, n, dtype, what):
        if not isinstance(t, self._torch.Tensor) or t.device != self.device:
            raise TypeError("%s must be a tensor on %s" % (what, self.device))
        if t.dtype != dtype:
            raise TypeError("%s must be %s, got %s" % (what, dtype, t.dtype))
        if t.numel() != n or not t.is_contiguous():
            raise ValueError("%s must be %d contiguous elements" % (what, n))
        return t.data_ptr()

    def _out(self, *shape, dtype=None):
        return self._torch.empty(*shape, dtype=dtype or self.dtype, device=self.device)


class HFVocab(_RowContext):
    """A vocabulary context of the C library plus its torch-allocated
    workspace: the token embedding, and the softmax head over a large
    vocabulary with the loss of hard labels or of a teacher's top logits.

    vocab x width: the matrices; max_rows: the most rows any call will use;
    dtype: "fp32" or "bf16", of the rows, the matrices and their gradients;
    ws_rows: size the workspace for calls of up to this many rows only
    (default max_rows).  Rows may be strided (the last dimension contiguous).
    Labels, tokens and ids are int32, HF_IGNORE where masked.  Calls run on
    torch's current stream of the context's device; the workspace goes back to
    torch's allocator once the work on all of them is done.  A graph that has
    captured calls works in it at every replay: keep the object as long.
    """

    _prefix = "hf_vocab"

    def __init__(self, vocab, width, max_rows, dtype="fp32", device="cuda",
                 ws_rows=None):
        import torch
        self._torch = torch
        self.vocab, self.width = int(vocab), int(width)
        self.max_rows = int(max_rows)
        self.dtype = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
        L = lib()
        h = ctypes.c_void_p()
        rc = L.hf_vocab_create(self.vocab, self.width, TYPES[dtype], self.max_rows,
                               None, ctypes.byref(h))
        if rc != HF_OK:
            raise HFError(rc, "hf_vocab_create rejected vocab=%d width=%d max_rows=%d"
                          % (self.vocab, self.width, self.max_rows))
        self._open(h, ws_rows, device)

    def _rows(self, X, what):
        if X.dim() != 2 or X.shape[1] != self.width:
            raise ValueError("%s must be rows x %d" % (what, self.width))
        return int(X.shape[0])

    def _head(self, fn, X, W, targets, T, denom, loss, row_loss, grad):
        """A head call: targets and their arguments as the C call takes them."""
        f32 = self._torch.float32
        xp, ldx = self._mat(X, T, self.width, self.dtype, "X")
        wp, ldw = self._mat(W, self.vocab, self.width, self.dtype, "W")
        loss = self._out(1, dtype=f32) if loss is None else loss
        row_loss = self._out(T, dtype=f32) if row_loss is None else row_loss
        args = [xp, ldx, wp, ldw, *targets, T, float(denom),
                self._vec(loss, 1, f32, "loss"), self._vec(row_loss, T, f32, "row_loss")]
        if grad is None:
            self._call(fn, *args)
            return loss, row_loss
        dX, dW, need_dX, need_dW, accumulate = grad
        for t, need, what in ((dX, need_dX, "dX"), (dW, need_dW, "dW")):
            if t is not None and not need:
                raise ValueError("%s is given, and need_%s is False" % (what, what))
        if accumulate and dW is None:
            raise ValueError("accumulate needs the dW to add to")
        if dX is None and need_dX:
            dX = self._out(T, self.width)
        if dW is None and need_dW:
            dW = self._out(self.vocab, self.width)
        for t, rows, what in ((dX, T, "dX"), (dW, self.vocab, "dW")):
            args += [None, 0] if t is None else self._mat(t, rows, self.width, self.dtype,
                                                          what)
        self._call(fn, *args, 1 if accumulate else 0)
        return loss, row_loss, dX, dW

    def _list(self, ids, t, T, tau):
        torch = self._torch
        if ids.dim() != 2:
            raise ValueError("ids must be rows x top")
        K = int(ids.shape[1])
        ip, ldi = self._mat(ids, T, K, torch.int32, "ids")
        tp, ldt = self._mat(t, T, K, torch.float32, "t")
        return ip, ldi, tp, ldt, K, float(tau)

    # -------------------------------------------------------------- the ABI
    def hf_vocab_loss(self, X, W, y, denom=0.0, loss=None, row_loss=None):
        """Softmax cross entropy of X W^T: (loss, row losses)."""
        T = self._rows(X, "X")
        y = self._vec(y, T, self._torch.int32, "y")
        return self._head("hf_vocab_loss", X, W, [y], T,
                          denom, loss, row_loss, None)

    def hf_vocab_loss_grad(self, X, W, y, denom=0.0, loss=None, row_loss=None, dX=None,
                           dW=None, need_dX=True, need_dW=True, accumulate=False):
        """hf_vocab_loss and its gradients: (loss, row losses, dX, dW).
        need_dX / need_dW False: that gradient is not computed (None, and none
        may be given).  accumulate: dW += (dW given)."""
        T = self._rows(X, "X")
        y = self._vec(y, T, self._torch.int32, "y")
        return self._head("hf_vocab_loss_grad", X, W, [y], T, denom, loss, row_loss,
                          (dX, dW, need_dX, need_dW, accumulate))

    def hf_vocab_distill(self, X, W, ids, t, tau=1.0, denom=0.0, loss=None,
                         row_loss=None):
        """Divergence from a teacher's top logits t at ids, at temperature
        tau: (loss, row losses)."""
        T = self._rows(X, "X")
        return self._head("hf_vocab_distill", X, W, self._list(ids, t, T, tau), T, denom,
                          loss, row_loss, None)

    def hf_vocab_distill_grad(self, X, W, ids, t, tau=1.0, denom=0.0, loss=None,
                              row_loss=None, dX=None, dW=None, need_dX=True,
                              need_dW=True, accumulate=False):
        """hf_vocab_distill and its gradients: (loss, row losses, dX, dW)."""
        T = self._rows(X, "X")
        return self._head("hf_vocab_distill_grad", X, W, self._list(ids, t, T, tau), T,
                          denom, loss, row_loss, (dX, dW, need_dX, need_dW, accumulate))

    def hf_vocab_embed(self, E, tok, scale=1.0, out=None):
        """scale E[tok], zeros where tok is HF_IGNORE."""
        T = tok.numel()
        out = self._out(T, self.width) if out is None else out
        ep, lde = self._mat(E, self.vocab, self.width, self.dtype, "E")
        op, ldo = self._mat(out, T, self.width, self.dtype, "out")
        self._call("hf_vocab_embed", ep, lde, self._vec(tok, T, self._torch.int32, "tok"),
                   T, float(scale), op, ldo)
        return out

    def hf_vocab_embed_grad(self, tok, dout, scale=1.0, dE=None, accumulate=False):
        """Gradient of hf_vocab_embed with respect to E; accumulate: dE +=
        (dE given)."""
        T = self._rows(dout, "dout")
        if accumulate and dE is None:
            raise ValueError("accumulate needs the dE to add to")
        dE = self._out(self.vocab, self.width) if dE is None else dE
        dp, ldd = self._mat(dout, T, self.width, self.dtype, "dout")
        ep, lde = self._mat(dE, self.vocab, self.width, self.dtype, "dE")
        self._call("hf_vocab_embed_grad", self._vec(tok, T, self._torch.int32, "tok"), T,
                   float(scale), dp, ldd, ep, lde, 1 if accumulate else 0)
        return dE

    def hf_vocab_check(self):
        """Synchronise and raise HFError(HF_ELABEL) for a label, token or id
        outside the vocabulary seen since the last check."""
        self._call("hf_vocab_check")


class HFGated(_RowContext):
    """A context of the gated feed-forward block of the C library plus its
    torch-allocated workspace: Y = (act(X Wg^T) * (X Wu^T)) Wd^T and its
    gradients, activation checkpoints in 8 bits, and products of 8-bit codes.

    width x hidden: X and Y are rows x width, Wg and Wu hidden x width, Wd width
    x hidden; max_rows: the most rows any call will use; act: "silu", "gelu",
    "gelu_tanh", "sigmoid", "tanh" or "relu"; dtype: "fp32" or "bf16", of the
    rows, the matrices and their gradients; ws_rows: size the workspace for
    calls of up to this many rows only (default max_rows).  One context serves
    every layer of these sizes.  Rows may be strided (the last dimension
    contiguous).  Streams, the workspace and graphs as for HFVocab.

    A checkpoint in 8 bits is a pair (codes int8, scale uint8), of a rows x cols
    matrix with a scale byte for every 32 columns; a matrix for products is a
    pair (codes int8, scale fp32) with a scale for every row.
    """

    _prefix = "hf_gated"

    def __init__(self, width, hidden, max_rows, act="silu", dtype="fp32", device="cuda",
                 ws_rows=None):
        import torch
        self._torch = torch
        self.width, self.hidden = int(width), int(hidden)
        self.max_rows = int(max_rows)
        self.dtype = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
        h = ctypes.c_void_p()
        rc = lib().hf_gated_create(self.width, self.hidden, GATED_ACTS[act], TYPES[dtype],
                                   self.max_rows, None, ctypes.byref(h))
        if rc != HF_OK:
            raise HFError(rc, "hf_gated_create rejected width=%d hidden=%d max_rows=%d"
                          % (self.width, self.hidden, self.max_rows))
        self._open(h, ws_rows, device)

    def _rows(self, X, what):
        if X.dim() != 2 or X.shape[1] != self.width:
            raise ValueError("%s must be rows x %d" % (what, self.width))
        return int(X.shape[0])

    def _weights(self, Wg, Wu, Wd, dtype=None):
        dtype, D, F = dtype or self.dtype, self.width, self.hidden
        return (*self._mat(Wg, F, D, dtype, "Wg"), *self._mat(Wu, F, D, dtype, "Wu"),
                *self._mat(Wd, D, F, dtype, "Wd"))

    def _blocks(self, cols):
        return (cols + HF_CODE_BLOCK - 1) // HF_CODE_BLOCK

    def _codes(self, pair, rows, cols, blocks, what):
        """(pointer, ld, pointer, ld) of a checkpoint's codes and scale bytes."""
        codes, scale = pair
        return (*self._mat(codes, rows, cols, self._torch.int8, what),
                *self._mat(scale, rows, blocks, self._torch.uint8, what + "'s scale"))

    def _kept(self, keep, kept, T):
        """(keep, pointer, ld, pointer, ld) of what a forward call keeps."""
        F = self.hidden
        if keep == "int8":
            return (HF_KEEP_CODES, *self._codes(kept, T, 2 * F, 2 * self._blocks(F), "kept"))
        return (HF_KEEP_FULL, *self._mat(kept, T, 2 * F, self.dtype, "kept"), None, 0)

    # -------------------------------------------------------------- the ABI
    def hf_gated_forward(self, X, Wg, Wu, Wd, keep=None, Y=None, kept=None):
        """The block: (Y, kept).  keep: what its gradient will need: None
        (nothing; kept is None), "full" (a rows x 2 hidden tensor: a row's
        X Wg^T and then its X Wu^T) or "int8" (that as a checkpoint, with
        2 ceil(hidden / 32) scale bytes a row)."""
        torch, T, F = self._torch, self._rows(X, "X"), self.hidden
        if keep not in KEEPS:
            raise ValueError("keep is %r, none of None, 'full', 'int8'" % (keep,))
        if keep is None and kept is not None:
            raise ValueError("kept is given, and keep is None")
        Y = self._out(T, self.width) if Y is None else Y
        if keep == "full" and kept is None:
            kept = self._out(T, 2 * F)
        elif keep == "int8" and kept is None:
            kept = (self._out(T, 2 * F, dtype=torch.int8),
                    self._out(T, 2 * self._blocks(F), dtype=torch.uint8))
        k = (HF_KEEP_NONE, None, 0, None, 0) if keep is None else self._kept(keep, kept, T)
        self._call("hf_gated_forward", *self._mat(X, T, self.width, self.dtype, "X"),
                   *self._weights(Wg, Wu, Wd), T,
                   *self._mat(Y, T, self.width, self.dtype, "Y"), *k)
        return Y, kept

    def hf_gated_grad(self, X, Wg, Wu, Wd, kept, dY, dX=None, dWg=None, dWu=None, dWd=None,
                      need_dX=True, need_dW=True, accumulate=False):
        """Gradients of the block: (dX, dWg, dWu, dWd).  kept: what
        hf_gated_forward kept, a tensor or a checkpoint; X: as forward had it,
        or its checkpoint.  need_dX / need_dW False: these are not computed
        (None, and none may be given).  accumulate: dWg, dWu and dWd += (all
        given)."""
        D, F = self.width, self.hidden
        T = self._rows(dY, "dY")
        for given, need, what in ((dX, need_dX, "dX"), (dWg, need_dW, "dW"),
                                  (dWu, need_dW, "dW"), (dWd, need_dW, "dW")):
            if given is not None and not need:
                raise ValueError("%s is given, and need_%s is False" % (what, what))
        if accumulate and (dWg is None or dWu is None or dWd is None):
            raise ValueError("accumulate needs the dWg, dWu and dWd to add to")
        if isinstance(X, (tuple, list)):
            x = self._codes(X, T, D, self._blocks(D), "X")
        else:
            x = (*self._mat(X, T, D, self.dtype, "X"), None, 0)
        k = self._kept("int8" if isinstance(kept, (tuple, list)) else "full", kept, T)
        if dX is None and need_dX:
            dX = self._out(T, D)
        if need_dW:
            dWg = self._out(F, D) if dWg is None else dWg
            dWu = self._out(F, D) if dWu is None else dWu
            dWd = self._out(D, F) if dWd is None else dWd
        outs = []
        for t, rows, cols, what in ((dX, T, D, "dX"), (dWg, F, D, "dWg"), (dWu, F, D, "dWu"),
                                    (dWd, D, F, "dWd")):
            outs += [None, 0] if t is None else self._mat(t, rows, cols, self.dtype, what)
        self._call("hf_gated_grad", *x, *self._weights(Wg, Wu, Wd), *k,
                   *self._mat(dY, T, D, self.dtype, "dY"), T, *outs, 1 if accumulate else 0)
        return dX, dWg, dWu, dWd

    def hf_gated_pack(self, X, codes=None, scale=None):
        """X (any rows x cols) as a checkpoint in 8 bits: (codes, scale)."""
        rows, cols = X.shape
        n = self._blocks(cols)
        codes = self._out(rows, cols, dtype=self._torch.int8) if codes is None else codes
        scale = self._out(rows, n, dtype=self._torch.uint8) if scale is None else scale
        self._call("hf_gated_pack", *self._mat(X, rows, cols, self.dtype, "X"), rows, cols,
                   *self._codes((codes, scale), rows, cols, n, "codes"))
        return codes, scale

    def hf_gated_unpack(self, codes, scale, X=None):
        """The numbers that a checkpoint stands for."""
        rows, cols = codes.shape
        X = self._out(rows, cols) if X is None else X
        self._call("hf_gated_unpack",
                   *self._codes((codes, scale), rows, cols, self._blocks(cols), "codes"),
                   rows, cols, *self._mat(X, rows, cols, self.dtype, "X"))
        return X

    def hf_gated_codes(self, X, codes=None, scale=None):
        """X (any rows x cols) as codes with a scale for each row, for a
        product: (codes, scale)."""
        torch = self._torch
        rows, cols = X.shape
        codes = self._out(rows, cols, dtype=torch.int8) if codes is None else codes
        scale = self._out(rows, dtype=torch.float32) if scale is None else scale
        self._call("hf_gated_codes", *self._mat(X, rows, cols, self.dtype, "X"), rows, cols,
                   *self._mat(codes, rows, cols, torch.int8, "codes"),
                   self._vec(scale, rows, torch.float32, "scale"))
        return codes, scale

    def _coded(self, codes, scale, rows, cols, what):
        return (*self._mat(codes, rows, cols, self._torch.int8, what),
                self._vec(scale, rows, self._torch.float32, what + "'s scale"))

    def hf_gated_product(self, A, sa, B, sb, Y=None):
        """A B^T of codes A (rows x k) and B (channels x k) with the scales sa
        and sb of their rows."""
        T, k = A.shape
        n = B.shape[0]
        Y = self._out(T, n) if Y is None else Y
        self._call("hf_gated_product", *self._coded(A, sa, T, k, "A"),
                   *self._coded(B, sb, n, k, "B"), T, n, k, *self._mat(Y, T, n, self.dtype, "Y"))
        return Y

    def hf_gated_forward_codes(self, X, Wg, Wu, Wd, Y=None):
        """The block with its matrices as pairs (codes, scale) of
        hf_gated_codes."""
        T, D, F = self._rows(X, "X"), self.width, self.hidden
        Y = self._out(T, D) if Y is None else Y
        self._call("hf_gated_forward_codes", *self._mat(X, T, D, self.dtype, "X"),
                   *self._coded(*Wg, F, D, "Wg"), *self._coded(*Wu, F, D, "Wu"),
                   *self._coded(*Wd, D, F, "Wd"), T, *self._mat(Y, T, D, self.dtype, "Y"))
        return Y
