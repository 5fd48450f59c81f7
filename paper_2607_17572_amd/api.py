"""Thin Python binding over the JAGG C ABI (include/jagg.h).

Argument marshalling only: every step of the path runs in libjagg.so.  PyTorch
supplies device memory (tensors) and the HIP stream.  If the library is not
built, every entry point raises instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import asdict, dataclass

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libjagg.so")

F32, BF16 = 0, 1
DGRAD, DGRAD_GELU, WGRAD = 0, 1, 2
E4M3, E5M2 = 0, 1


class _DitConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in (
        "n_double", "n_single", "hidden", "heads", "head_dim", "mlp_hidden", "in_ch", "patch", "lat_h",
        "lat_w", "n_txt", "txt_dim", "t_freq_dim", "block_only", "act_dtype", "grad_dtype", "checkpoint")]


class _GrpoWindow(ctypes.Structure):
    _fields_ = [("v_hat", ctypes.POINTER(ctypes.c_void_p)), ("z", ctypes.POINTER(ctypes.c_void_p)),
                ("t", ctypes.POINTER(ctypes.c_float)), ("sigma", ctypes.POINTER(ctypes.c_float)),
                ("logp_old", ctypes.c_void_p), ("adv", ctypes.c_void_p), ("clip_eps", ctypes.c_float),
                ("adv_clip", ctypes.c_float), ("W", ctypes.c_int), ("v_batch", ctypes.POINTER(ctypes.c_int)),
                ("v_index", ctypes.POINTER(ctypes.c_int))]


class _TensorDesc(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("offset", ctypes.c_size_t), ("numel", ctypes.c_size_t),
                ("rows", ctypes.c_int), ("cols", ctypes.c_int)]


class _Mat8(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("ld", ctypes.c_size_t), ("rows", ctypes.c_int),
                ("k", ctypes.c_int), ("fmt", ctypes.c_int)]


class _Grad(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_size_t), ("dtype", ctypes.c_int)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises RuntimeError if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2607_17572_amd.build.build() "
                               "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, i, f, d = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float, ctypes.c_double
        pcfg, pm8, pg = ctypes.POINTER(_DitConfig), ctypes.POINTER(_Mat8), ctypes.POINTER(_Grad)
        L.jagg_last_error.restype = ctypes.c_char_p
        sig = {
            "dit_param_layout": [pcfg, ctypes.POINTER(sz), ctypes.POINTER(sz), ctypes.POINTER(_TensorDesc), sz],
            "jagg_ctx_create": [pcfg, vp, ctypes.POINTER(vp)],
            "dit_saved_bytes": [vp, i, ctypes.POINTER(sz)],
            "dit_workspace_bytes": [vp, i, ctypes.POINTER(sz)],
            "jagg_ctx_set_workspace": [vp, vp, sz],
            "dit_forward_save": [vp, vp, vp, ctypes.POINTER(f), vp, vp, vp, i],
            "dit_vjp": [vp, vp, vp, i, vp, vp, f],
            "jagg_alpha": [ctypes.POINTER(f), i, ctypes.POINTER(f)],
            "jagg_aggregate": [vp, ctypes.POINTER(vp), ctypes.POINTER(f), i, sz, i, vp, vp],
            "jagg_group_scores": [vp, ctypes.POINTER(vp), sz, i, i, ctypes.POINTER(d)],
            "jagg_group_scores_noalloc": [vp, ctypes.POINTER(vp), sz, i, i, vp],
            "jagg_route": [ctypes.POINTER(d), i, d, d, ctypes.POINTER(ctypes.c_ubyte), ctypes.POINTER(d)],
            "jagg_group_backward": [vp, vp, vp, i, ctypes.POINTER(vp), ctypes.POINTER(f), i, vp, f],
            "perstep_group_backward": [vp, vp, ctypes.POINTER(vp), i, ctypes.POINTER(vp), i, vp, f],
            "jagg_trajectory_backward": [vp, vp, i, i, i, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                         ctypes.POINTER(f), ctypes.POINTER(ctypes.c_ubyte), vp, f],
            "jagg_linear_grad": [vp, i, vp, vp, vp, i, i, i, vp, i, f],
            "jagg_endpoint_backward": [vp, vp, vp, i, ctypes.POINTER(vp), ctypes.POINTER(f), i, i, vp, f],
            "jagg_grad_compare": [vp, vp, vp, sz, i, ctypes.POINTER(d)],
            "jagg_count_nonfinite": [vp, vp, sz, i, ctypes.POINTER(ctypes.c_ulonglong)],
            "jagg_window_quality": [vp, vp, vp, ctypes.POINTER(vp), i, ctypes.POINTER(vp), ctypes.POINTER(f), i, vp, vp,
                                    vp, ctypes.POINTER(d)],
            "jagg_mat8_bytes": [i, i, ctypes.POINTER(sz), ctypes.POINTER(sz), ctypes.POINTER(sz)],
            "jagg_quantize8": [vp, vp, sz, i, i, i, vp, vp, i, pm8, pm8],
            "jagg_matmul8_bytes": [i, i, i, i, ctypes.POINTER(sz)],
            "jagg_matmul8": [vp, pm8, pm8, vp, vp, sz, i, f],
            "jagg_rmsnorm8": [vp, vp, sz, vp, sz, vp, i, i, i, f, vp, sz, pm8, vp],
            "jagg_rmsnorm8_grad_bytes": [i, i, ctypes.POINTER(sz)],
            "jagg_rmsnorm8_grad": [vp, vp, sz, vp, sz, vp, vp, vp, sz, i, i, i, vp, sz, vp, i, f],
            "jagg_grad_norm_bytes": [ctypes.POINTER(sz)],
            "jagg_grad_norm": [vp, pg, i, i, vp],
            "jagg_grad_clip": [vp, pg, pg, i, i, d, vp],
            "jagg_grpo_composites": [vp, ctypes.POINTER(_GrpoWindow), i, vp, vp, vp],
            "jagg_grpo_upstream": [vp, ctypes.POINTER(_GrpoWindow), i, ctypes.POINTER(vp), vp],
            "jagg_grpo_group_backward": [vp, vp, vp, i, ctypes.POINTER(_GrpoWindow), vp, f, vp],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        L.jagg_ctx_destroy.argtypes = [vp]
        L.jagg_ctx_destroy.restype = None
        L.jagg_prof_begin.argtypes = [i]
        L.jagg_prof_begin.restype = ctypes.c_int
        L.jagg_prof_end.argtypes = [ctypes.POINTER(ctypes.c_long), ctypes.POINTER(d), ctypes.POINTER(d)]
        L.jagg_prof_end.restype = ctypes.c_int
        _lib = L
    return _lib


class JaggError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"JAGG status {status}: {msg}")
        self.status = status


def _check(rc: int):
    if rc != 0:
        raise JaggError(rc, lib().jagg_last_error().decode())


@dataclass(frozen=True)
class Config:
    n_double: int
    n_single: int
    hidden: int
    heads: int
    head_dim: int
    mlp_hidden: int
    in_ch: int = 4
    patch: int = 1
    lat_h: int = 4
    lat_w: int = 4
    n_txt: int = 8
    txt_dim: int = 64
    t_freq_dim: int = 256
    block_only: int = 0
    act_dtype: int = F32
    grad_dtype: int = F32
    checkpoint: int = 0

    def c(self) -> _DitConfig:
        return _DitConfig(**{k: int(v) for k, v in asdict(self).items()})

    @property
    def n_img(self) -> int:
        return (self.lat_h // self.patch) * (self.lat_w // self.patch)

    @property
    def n_tok(self) -> int:
        return self.n_txt + self.n_img


def param_layout(cfg: Config):
    """[(name, offset, numel, rows, cols)], flat length."""
    c = cfg.c()
    nt, ne = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().dit_param_layout(ctypes.byref(c), ctypes.byref(nt), ctypes.byref(ne), None, 0))
    arr = (_TensorDesc * nt.value)()
    _check(lib().dit_param_layout(ctypes.byref(c), ctypes.byref(nt), ctypes.byref(ne), arr, nt.value))
    return [(d.name.decode(), d.offset, d.numel, d.rows, d.cols) for d in arr], ne.value


def alpha(t):
    W = len(t)
    tt = (ctypes.c_float * W)(*[float(x) for x in t])
    out = (ctypes.c_float * W)()
    _check(lib().jagg_alpha(tt, W, out))
    return list(out)


def route(n_groups: int, frac: float | None = None, scores=None, tau: float = 0.5):
    """(list of 0/1 per group, realised fraction)."""
    sc = None
    if scores is not None:
        sc = (ctypes.c_double * n_groups)(*[float(x) for x in scores])
    mask = (ctypes.c_ubyte * n_groups)()
    fr = ctypes.c_double()
    _check(lib().jagg_route(sc, n_groups, float(tau), -1.0 if frac is None else float(frac), mask, ctypes.byref(fr)))
    return list(mask), fr.value


PROF_GEMM_FWD, PROF_GEMM_DGRAD, PROF_GEMM_WGRAD = 1, 2, 3
PROF_ATTN_FWD, PROF_ATTN_BWD_KV, PROF_ATTN_BWD_Q, PROF_AGGREGATE = 4, 5, 6, 7
PROF_COMPARE, PROF_UPSTREAM = 8, 9


def prof_begin(cls: int):
    """Arm HIP-event timing of every launch of kernel class ``cls``."""
    _check(lib().jagg_prof_begin(cls))


def prof_end():
    """(launches, total kernel ms, total algorithmic work) of the armed class."""
    n, ms, work = ctypes.c_long(), ctypes.c_double(), ctypes.c_double()
    _check(lib().jagg_prof_end(ctypes.byref(n), ctypes.byref(ms), ctypes.byref(work)))
    return n.value, ms.value, work.value


def _ptrs(tensors):
    return (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


# -------------------------------------------------- arguments of the operators
def _refuse(msg: str):
    raise JaggError(1, msg)


def _dtype_of(t, name: str) -> int:
    torch = _torch()
    dt = t.dtype
    if dt is torch.bfloat16:
        return BF16
    if dt is torch.float32:
        return F32
    _refuse(f"{name} must be bf16 or fp32")


def _vec(t, name: str, n: int, dtype, device):
    """Pointer of a contiguous vector of n elements."""
    if t.dtype is not dtype or t.dim() != 1 or t.numel() != n or not t.is_contiguous() or t.device != device:
        _refuse(f"{name} must be a contiguous vector of {n} elements of {dtype} on {device}")
    return t.data_ptr()


def _rows(t, name: str, rows: int, cols: int, dtype, device):
    """(pointer, row stride) of a matrix whose rows are contiguous."""
    sh = t.shape
    if t.dtype is not dtype or len(sh) != 2 or sh[0] != rows or sh[1] != cols or t.device != device:
        _refuse(f"{name} must be {rows} x {cols} of {dtype} on {device}")
    if t.is_contiguous():
        return t.data_ptr(), cols
    st = t.stride()
    if (cols > 1 and st[1] != 1) or (rows > 1 and st[0] < cols):
        _refuse(f"{name} must have contiguous rows that do not overlap")
    return t.data_ptr(), st[0] if rows > 1 else cols


class Mat8:
    """An 8-bit matrix with one power-of-two scale per block of 128 columns
    (jagg_mat8): ``q`` uint8 [rows][ld], ``scale`` uint8 [ceil(k/512)][rows][4].
    Allocates both on the current CUDA device, or takes given tensors, and keeps
    them; a call refuses a matrix whose memory is no longer where it was."""

    def __init__(self, rows: int, k: int, fmt: int = E4M3, q=None, scale=None):
        torch = _torch()
        ld, nq, ns = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
        _check(lib().jagg_mat8_bytes(rows, k, ctypes.byref(ld), ctypes.byref(nq), ctypes.byref(ns)))
        if fmt not in (E4M3, E5M2):
            _refuse("unknown 8-bit format")
        words = (k + 511) // 512
        if q is None:
            q = torch.empty(rows, ld.value, dtype=torch.uint8, device="cuda")
        if scale is None:
            scale = torch.empty(words, rows, 4, dtype=torch.uint8, device=q.device)
        if q.element_size() != 1 or q.dim() != 2 or q.shape[0] != rows or q.shape[1] < ld.value or not q.is_contiguous():
            _refuse(f"q must be contiguous bytes [{rows}][>= {ld.value}]")
        if scale.element_size() != 1 or tuple(scale.shape) != (words, rows, 4) or not scale.is_contiguous():
            _refuse(f"scale must be contiguous bytes [{words}][{rows}][4]")
        if scale.device != q.device or not q.is_cuda:
            _refuse("q and scale must be on one GPU")
        self.rows, self.k, self.fmt = rows, k, fmt
        self.q, self.scale = q.view(torch.uint8), scale.view(torch.uint8)
        self.device = q.device
        self._at = self.q.data_ptr(), self.scale.data_ptr()
        self._c = _Mat8(*self._at, q.shape[1], rows, k, fmt)

    def _arg(self, device):
        """The C struct for a call on the given device."""
        if self.device != device:
            _refuse("an 8-bit matrix must be on the context's device")
        if (self.q.data_ptr(), self.scale.data_ptr()) != self._at:
            _refuse("the tensors of an 8-bit matrix have moved since it was made")
        return self._c


class GradList:
    """Gradient tensors (each contiguous, bf16 or fp32, of one GPU) as the norm and
    clipping calls take them; a program that keeps its gradients keeps one.  The list
    stands for the memory that the tensors have when it is made, and keeps it: a
    gradient that is made anew, or a tensor given other memory (``set_``, ``.data``),
    needs a new list.  A call refuses a list whose memory itself was moved
    (``resize_`` beyond it)."""

    def __init__(self, tensors):
        self._fill(tensors)
        held = {s.data_ptr(): s for s in (t.untyped_storage() for t in self.tensors)}
        self._held = [(s, p) for p, s in held.items()]

    def _fill(self, tensors):
        self.tensors = list(tensors)
        if not self.tensors:
            _refuse("a gradient list needs a tensor")
        self.device = self.tensors[0].device
        self._c = (_Grad * len(self.tensors))()
        for g, t in zip(self._c, self.tensors):
            if not t.is_cuda or t.device != self.device or not t.is_contiguous():
                _refuse("gradients must be contiguous tensors of one GPU")
            g.data, g.n, g.dtype = t.data_ptr(), t.numel(), _dtype_of(t, "a gradient")
        self.spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in self.tensors if t.numel())
        if any(a[1] > b[0] for a, b in zip(self.spans, self.spans[1:])):
            _refuse("gradients must not overlap")

    def _arg(self):
        for s, p in self._held:
            if s.data_ptr() != p:
                _refuse("the memory of a gradient list has moved since it was made")
        return self._c


def _grads(g) -> GradList:
    if isinstance(g, GradList):
        return g
    one = GradList.__new__(GradList)  # for this call only: the caller holds the memory
    one._fill([g] if _torch().is_tensor(g) else g)
    one._held = ()
    return one


@functools.cache
def _grad_bytes() -> int:
    """Workspace of the norm and clipping calls."""
    n = ctypes.c_size_t()
    _check(lib().jagg_grad_norm_bytes(ctypes.byref(n)))
    return n.value


_NORMS = {2: 0, 2.0: 0, float("inf"): 1}


class Context:
    """One model configuration bound to a HIP stream, with a workspace tensor.  Every call
    runs on that stream, whichever is current."""

    def __init__(self, cfg: Config, stream=None):
        torch = _torch()
        self.cfg = cfg
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        h = ctypes.c_void_p()
        c = cfg.c()
        self.device = self.stream.device
        with torch.cuda.device(self.device):
            _check(lib().jagg_ctx_create(ctypes.byref(c), ctypes.c_void_p(self.stream.cuda_stream), ctypes.byref(h)))
        self._h = h
        self._ws = None
        self._ws_batch = self._ws_bytes = 0
        self._captured, self._ws_of_graphs = False, []
        self.layout, self.n_params = param_layout(cfg)

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _lib is not None:
            _lib.jagg_ctx_destroy(h)
            self._h = None

    @property
    def dtype(self):
        torch = _torch()
        return torch.bfloat16 if self.cfg.act_dtype == BF16 else torch.float32

    @property
    def grad_dtype(self):
        torch = _torch()
        return torch.bfloat16 if self.cfg.grad_dtype == BF16 else torch.float32

    def saved_bytes(self, batch: int) -> int:
        n = ctypes.c_size_t()
        _check(lib().dit_saved_bytes(self._h, batch, ctypes.byref(n)))
        return n.value

    def workspace_bytes(self, batch: int) -> int:
        n = ctypes.c_size_t()
        _check(lib().dit_workspace_bytes(self._h, batch, ctypes.byref(n)))
        return n.value

    def ensure_workspace(self, batch: int):
        if self._ws is not None and self._ws_batch >= batch:
            self._ensure_bytes(0)
            return
        self._ensure_bytes(self.workspace_bytes(batch))
        self._ws_batch = batch

    def _ensure_bytes(self, nb: int):
        """A bound workspace of at least nb bytes (it only grows).  One that a captured call
        used stays for as long as the context, since the graph may hold its address."""
        torch = _torch()
        capturing = torch.cuda.is_current_stream_capturing()
        if self._ws is not None and self._ws_bytes >= nb:
            self._captured |= capturing
            return
        if self._captured:
            self._ws_of_graphs.append(self._ws)
        with torch.cuda.device(self.device), torch.cuda.stream(self.stream):
            ws = torch.empty(nb + 256, dtype=torch.uint8, device=self.device)
        base = ws.data_ptr()
        off = (-base) % 256
        _check(lib().jagg_ctx_set_workspace(self._h, ctypes.c_void_p(base + off), nb))
        self._ws, self._ws_bytes, self._captured = ws, nb, capturing

    def new_saved(self, batch: int):
        torch = _torch()
        return torch.empty(self.saved_bytes(batch), dtype=torch.uint8, device="cuda")

    def forward_save(self, theta, z, t, txt=None, saved=None, batch=None, v_out=None):
        """v = v_theta(z, t); `saved` (uint8 tensor of saved_bytes(batch)) or None (no graph)."""
        torch = _torch()
        B = len(t) if batch is None else batch
        self.ensure_workspace(B)
        if v_out is None:
            v_out = torch.empty_like(z)
        tt = (ctypes.c_float * B)(*[float(x) for x in t])
        _check(lib().dit_forward_save(self._h, theta.data_ptr(), z.data_ptr(), tt,
                                      None if txt is None else txt.data_ptr(), v_out.data_ptr(),
                                      None if saved is None else saved.data_ptr(), B))
        return v_out

    def vjp(self, theta, saved, batch: int, s, dtheta, beta: float = 0.0):
        self.ensure_workspace(batch)
        _check(lib().dit_vjp(self._h, theta.data_ptr(), saved.data_ptr(), batch, s.data_ptr(), dtheta.data_ptr(),
                             float(beta)))
        return dtheta

    def aggregate(self, s_list, t, s_base, s_corr):
        W = len(s_list)
        tt = (ctypes.c_float * W)(*[float(x) for x in t])
        dt = BF16 if s_list[0].dtype == _torch().bfloat16 else F32
        _check(lib().jagg_aggregate(self._h, _ptrs(s_list), tt, W, s_list[0].numel(), dt, s_base.data_ptr(),
                                    s_corr.data_ptr()))
        return s_base, s_corr

    def group_score(self, h_list) -> float:
        self.ensure_workspace(1)
        out = ctypes.c_double()
        dt = BF16 if h_list[0].dtype == _torch().bfloat16 else F32
        _check(lib().jagg_group_scores(self._h, _ptrs(h_list), h_list[0].numel(), len(h_list), dt, ctypes.byref(out)))
        return out.value

    def group_score_noalloc(self, h_list, score_dev):
        """Allocation-free group score: written into score_dev (a device fp64
        tensor of one element) on the stream; needs no workspace."""
        dt = BF16 if h_list[0].dtype == _torch().bfloat16 else F32
        _check(lib().jagg_group_scores_noalloc(self._h, _ptrs(h_list), h_list[0].numel(), len(h_list), dt,
                                               score_dev.data_ptr()))
        return score_dev

    def group_backward(self, theta, saved_pair, batch: int, s_list, t, dtheta, beta: float = 0.0):
        """JAGG: composites + one VJP over the batch-2B endpoint pair."""
        W = len(s_list)
        self.ensure_workspace(2 * batch)
        tt = (ctypes.c_float * W)(*[float(x) for x in t])
        _check(lib().jagg_group_backward(self._h, theta.data_ptr(), saved_pair.data_ptr(), batch, _ptrs(s_list), tt,
                                         W, dtheta.data_ptr(), float(beta)))
        return dtheta

    def endpoint_backward(self, theta, saved, batch: int, s_list, t, endpoint: int, dtheta, beta: float = 0.0):
        """Sequential-graph JAGG: the backward of one endpoint (0: s_base, 1: s_corr)."""
        W = len(s_list)
        self.ensure_workspace(batch)
        tt = (ctypes.c_float * W)(*[float(x) for x in t])
        _check(lib().jagg_endpoint_backward(self._h, theta.data_ptr(), saved.data_ptr(), batch, _ptrs(s_list), tt, W,
                                            int(endpoint), dtheta.data_ptr(), float(beta)))
        return dtheta

    def grad_compare(self, a, b):
        """(a.b, a.a, b.b, cos, rho) over every element of two equal-size device
        tensors: the fp64 sums and the quality figures the library forms from them."""
        self.ensure_workspace(1)
        out = (ctypes.c_double * 5)()
        dt = BF16 if a.dtype == _torch().bfloat16 else F32
        assert a.numel() == b.numel() and a.dtype == b.dtype
        _check(lib().jagg_grad_compare(self._h, a.data_ptr(), b.data_ptr(), a.numel(), dt, out))
        return tuple(out)

    def count_nonfinite(self, x) -> int:
        """Number of NaN / +-Inf elements of a device tensor (fp32 or bf16)."""
        self.ensure_workspace(1)
        out = ctypes.c_ulonglong()
        dt = BF16 if x.dtype == _torch().bfloat16 else F32
        _check(lib().jagg_count_nonfinite(self._h, x.data_ptr(), x.numel(), dt, ctypes.byref(out)))
        return int(out.value)

    def window_quality(self, theta, saved_pair, saved_steps, batch: int, s_list, t, g_jagg, g_exact, g_ablate):
        """(cos_jagg, rho_jagg, cos_ablate, rho_ablate) of one window; the three
        group gradients are left in the given (zero-padded) buffers."""
        W = len(s_list)
        self.ensure_workspace(2 * batch)
        tt = (ctypes.c_float * W)(*[float(x) for x in t])
        out = (ctypes.c_double * 4)()
        _check(lib().jagg_window_quality(self._h, theta.data_ptr(), saved_pair.data_ptr(), _ptrs(saved_steps), batch,
                                         _ptrs(s_list), tt, W, g_jagg.data_ptr(), g_exact.data_ptr(),
                                         g_ablate.data_ptr(), out))
        return tuple(out)

    @staticmethod
    def _grpo_window(v_list, z_list, t, sigma, logp_old, adv, clip_eps, adv_clip):
        """The C struct of one GRPO window; returns (struct, keep-alive list).
        logp_old: device fp64 tensor [W][B]; adv: device fp32 tensor [B].
        An entry of v_list may be (tensor, batch, index): samples index ..
        index + B - 1 of a batch-``batch`` model output."""
        W = len(v_list)
        assert len(z_list) == W + 1 and len(t) == W + 1 and len(sigma) == W
        vt = [x[0] if isinstance(x, tuple) else x for x in v_list]
        B = adv.numel()
        vb = (ctypes.c_int * W)(*[x[1] if isinstance(x, tuple) else B for x in v_list])
        vk = (ctypes.c_int * W)(*[x[2] if isinstance(x, tuple) else 0 for x in v_list])
        vp, zp = _ptrs(vt), _ptrs(z_list)
        tt = (ctypes.c_float * (W + 1))(*[float(x) for x in t])
        sg = (ctypes.c_float * W)(*[float(x) for x in sigma])
        w = _GrpoWindow(vp, zp, tt, sg, logp_old.data_ptr(), adv.data_ptr(), float(clip_eps), float(adv_clip), W,
                        vb, vk)
        return w, [vp, zp, tt, sg, vb, vk]

    def grpo_composites(self, v_list, z_list, t, sigma, logp_old, adv, s_base, s_corr, clip_eps=0.1, adv_clip=5.0,
                        stats=None, batch=None):
        """Phases 2 + 3 fused: composites of the window's GRPO upstream gradients."""
        B = adv.numel() if batch is None else batch
        self.ensure_workspace(1)
        w, keep = self._grpo_window(v_list, z_list, t, sigma, logp_old, adv, clip_eps, adv_clip)
        _check(lib().jagg_grpo_composites(self._h, ctypes.byref(w), B, s_base.data_ptr(), s_corr.data_ptr(),
                                          None if stats is None else stats.data_ptr()))
        return s_base, s_corr

    def grpo_upstream(self, v_list, z_list, t, sigma, logp_old, adv, s_out, clip_eps=0.1, adv_clip=5.0, stats=None,
                      batch=None):
        """Phase 2: the W upstream gradients s_j (written into s_out)."""
        B = adv.numel() if batch is None else batch
        self.ensure_workspace(1)
        w, keep = self._grpo_window(v_list, z_list, t, sigma, logp_old, adv, clip_eps, adv_clip)
        _check(lib().jagg_grpo_upstream(self._h, ctypes.byref(w), B, _ptrs(s_out),
                                        None if stats is None else stats.data_ptr()))
        return s_out

    def grpo_group_backward(self, theta, saved_pair, batch: int, v_list, z_list, t, sigma, logp_old, adv, dtheta,
                            beta: float = 0.0, clip_eps=0.1, adv_clip=5.0, stats=None):
        """Phases 2-4: fused composites into the pair cotangent, one joint VJP."""
        self.ensure_workspace(2 * batch)
        w, keep = self._grpo_window(v_list, z_list, t, sigma, logp_old, adv, clip_eps, adv_clip)
        _check(lib().jagg_grpo_group_backward(self._h, theta.data_ptr(), saved_pair.data_ptr(), batch,
                                              ctypes.byref(w), dtheta.data_ptr(), float(beta),
                                              None if stats is None else stats.data_ptr()))
        return dtheta

    def linear_grad(self, kind: int, dY, other, result, beta: float = 0.0, pre=None):
        """One product of a linear layer's backward (DGRAD, DGRAD_GELU or WGRAD)."""
        torch = _torch()
        rows, n_out = dY.shape
        n_in = other.shape[1]
        rdt = BF16 if result.dtype == torch.bfloat16 else F32
        _check(lib().jagg_linear_grad(self._h, kind, dY.data_ptr(), other.data_ptr(),
                                      None if pre is None else pre.data_ptr(), rows, n_out, n_in, result.data_ptr(),
                                      rdt, float(beta)))
        return result

    # ------------------------------------------- 8-bit linear layers, clipping
    def quantize8(self, x, out: Mat8 = None, out_t: Mat8 = None, tile: bool = False, row_mul=None, col_mul=None):
        """8-bit form of y = x * row_mul[:, None] * col_mul: ``out`` its rows (blocks
        of 128 along a row), ``out_t`` its transpose (blocks along a column), either
        or both; ``tile``: one scale per 128 x 128, the same in both."""
        if x.dim() != 2:
            _refuse("x must be a matrix")
        rows, cols = x.shape
        dt = _dtype_of(x, "x")
        p, ld = _rows(x, "x", rows, cols, x.dtype, self.device)
        rm = None if row_mul is None else _vec(row_mul, "row_mul", rows, _torch().float32, self.device)
        cm = None if col_mul is None else _vec(col_mul, "col_mul", cols, x.dtype, self.device)
        _check(lib().jagg_quantize8(self._h, p, ld, rows, cols, dt, rm, cm, 1 if tile else 0,
                                    None if out is None else out._arg(self.device),
                                    None if out_t is None else out_t._arg(self.device)))
        return out, out_t

    def matmul8(self, a: Mat8, b: Mat8, out, bias=None, beta: float = 0.0):
        """out = beta * out + a b^T + bias (out: [a.rows][b.rows], bf16 or fp32).  The sums
        are fp32, but for large bf16 results: there the 8-bit matrix instructions'."""
        dt = _dtype_of(out, "out")
        p, ld = _rows(out, "out", a.rows, b.rows, out.dtype, self.device)
        ac, bc = a._arg(self.device), b._arg(self.device)
        bp = None if bias is None else _vec(bias, "bias", b.rows, out.dtype, self.device)
        if a.rows > 16:
            nb = ctypes.c_size_t()
            _check(lib().jagg_matmul8_bytes(a.rows, b.rows, a.k, dt, ctypes.byref(nb)))
            if nb.value:
                self._ensure_bytes(nb.value)
        _check(lib().jagg_matmul8(self._h, ac, bc, bp, p, ld, dt, beta))
        return out

    def rmsnorm8(self, x, gain, y: Mat8, residual=None, h=None, rstd=None, eps: float = 1e-6):
        """h = x + residual, y = h / sqrt(mean(h^2) + eps) * gain in 8 bits (E4M3);
        ``h`` and ``rstd`` are written if given (the backward reads both)."""
        if x.dim() != 2:
            _refuse("x must be a matrix")
        rows, cols = x.shape
        dt, dev = _dtype_of(x, "x"), self.device
        p, ld = _rows(x, "x", rows, cols, x.dtype, dev)
        rp, rl = (None, 0) if residual is None else _rows(residual, "residual", rows, cols, x.dtype, dev)
        hp, hl = (None, 0) if h is None else _rows(h, "h", rows, cols, x.dtype, dev)
        _check(lib().jagg_rmsnorm8(self._h, p, ld, rp, rl, _vec(gain, "gain", cols, x.dtype, dev), rows, cols, dt, eps,
                                   hp, hl, y._arg(dev), None if rstd is None else _vec(rstd, "rstd", rows, _torch().float32, dev)))
        return y

    def rmsnorm8_grad(self, dy, h, rstd, gain, dx, dgain, dh=None, beta: float = 0.0):
        """Backward of rmsnorm8: dx (of x and of the residual; dh, the gradient of h
        from elsewhere, is added) and dgain = beta * dgain + its gradient."""
        if h.dim() != 2:
            _refuse("h must be a matrix")
        rows, cols = h.shape
        dt, dev = _dtype_of(h, "h"), self.device
        yp, yl = _rows(dy, "dy", rows, cols, h.dtype, dev)
        hp, hl = _rows(h, "h", rows, cols, h.dtype, dev)
        gp, gl = (None, 0) if dh is None else _rows(dh, "dh", rows, cols, h.dtype, dev)
        xp, xl = _rows(dx, "dx", rows, cols, h.dtype, dev)
        nb = ctypes.c_size_t()
        _check(lib().jagg_rmsnorm8_grad_bytes(rows, cols, ctypes.byref(nb)))
        self._ensure_bytes(nb.value)
        _check(lib().jagg_rmsnorm8_grad(self._h, yp, yl, hp, hl, _vec(rstd, "rstd", rows, _torch().float32, dev),
                                        _vec(gain, "gain", cols, h.dtype, dev), gp, gl, rows, cols, dt, xp, xl,
                                        _vec(dgain, "dgain", cols, dgain.dtype, dev), _dtype_of(dgain, "dgain"), beta))
        return dx, dgain

    def grad_norm(self, grads, out, ord=2):
        """Global norm (2 or inf) of a tensor, a list of tensors or a GradList into
        ``out`` (device fp64 tensor of one element)."""
        g = _grads(grads)
        if g.device != self.device or ord not in _NORMS:
            _refuse("the gradients must be on the context's device, ord 2 or inf")
        p = _vec(out, "out", 1, _torch().float64, self.device)
        self._ensure_bytes(_grad_bytes())
        _check(lib().jagg_grad_norm(self._h, g._arg(), len(g.tensors), _NORMS[ord], p))
        return out

    def clip_grads(self, grads, max_norm: float, out, dst=None, ord=2):
        """Scales the gradients (in place, or into ``dst``, tensors of the same sizes)
        so that their global norm is at most max_norm; out (device fp64 tensor of
        two elements) receives the norm and the factor.  A norm that is not finite
        leaves the values as they are."""
        g = _grads(grads)
        d = None if dst is None else _grads(dst)
        if g.device != self.device or ord not in _NORMS:
            _refuse("the gradients must be on the context's device, ord 2 or inf")
        if d is not None:
            if d.device != self.device or len(d.tensors) != len(g.tensors):
                _refuse("dst must have one tensor on the context's device for each gradient")
            # lists that lie apart as a whole need no closer look
            apart = not g.spans or not d.spans or d.spans[-1][1] <= g.spans[0][0] or g.spans[-1][1] <= d.spans[0][0]
            if not (apart or d is g):
                self._check_dst(g, d)
        p = _vec(out, "out", 2, _torch().float64, self.device)
        self._ensure_bytes(_grad_bytes())
        _check(lib().jagg_grad_clip(self._h, g._arg(), None if d is None else d._arg(), len(g.tensors), _NORMS[ord],
                                    float(max_norm), p))
        return out

    @staticmethod
    def _check_dst(g: GradList, d: GradList):
        own = {a.data_ptr() for a, b in zip(g.tensors, d.tensors)
               if a.data_ptr() == b.data_ptr() and a.dtype is b.dtype and a.numel() == b.numel()}
        both = sorted(g.spans + [s for s in d.spans if s[0] not in own])
        if any(a[1] > b[0] for a, b in zip(both, both[1:])):
            _refuse("dst must not overlap the gradients, but for a tensor's own")

    def trajectory_backward(self, theta, W: int, batch: int, saved_pairs, saved_steps, s_list, t, use_jagg, dtheta,
                            beta: float = 0.0):
        """Whole trajectory: JAGG for the windows use_jagg marks, per step for
        the rest and the T mod W tail.  saved_pairs: one entry per full window
        (None where it takes the per-step backward); saved_steps: one per step
        (None for steps of JAGG windows)."""
        T = len(s_list)
        n = T // W
        any_jagg = any(int(u) for u in use_jagg)
        self.ensure_workspace(2 * batch if any_jagg else batch)
        vp = ctypes.c_void_p
        pairs = (vp * max(n, 1))(*[None if x is None else x.data_ptr() for x in saved_pairs])
        steps = (vp * T)(*[None if x is None else x.data_ptr() for x in saved_steps])
        tt = (ctypes.c_float * T)(*[float(x) for x in t])
        mk = (ctypes.c_ubyte * max(n, 1))(*[int(u) for u in use_jagg])
        _check(lib().jagg_trajectory_backward(self._h, theta.data_ptr(), T, W, batch, pairs, steps, _ptrs(s_list), tt,
                                              mk, dtheta.data_ptr(), float(beta)))
        return dtheta

    def perstep_group_backward(self, theta, saved_list, batch: int, s_list, dtheta, beta: float = 0.0):
        self.ensure_workspace(batch)
        _check(lib().perstep_group_backward(self._h, theta.data_ptr(), _ptrs(saved_list), batch, _ptrs(s_list),
                                            len(s_list), dtheta.data_ptr(), float(beta)))
        return dtheta


# ------------------------------------------------------------------ configs
def config(name: str, **over) -> Config:
    """The five workloads: tiny (C1), block (C2), slice (C3), flux (C4), qwen (C5)."""
    big = dict(hidden=3072, heads=24, head_dim=128, mlp_hidden=12288, in_ch=16, patch=2, t_freq_dim=256,
               act_dtype=BF16, grad_dtype=F32)
    table = {
        "tiny": dict(n_double=2, n_single=0, hidden=64, heads=4, head_dim=16, mlp_hidden=256, in_ch=4, patch=1,
                     lat_h=4, lat_w=4, n_txt=8, txt_dim=64, t_freq_dim=256, act_dtype=F32, grad_dtype=F32),
        "block": dict(big, n_double=1, n_single=0, lat_h=128, lat_w=128, n_txt=512, txt_dim=3072, block_only=1),
        "slice": dict(big, n_double=4, n_single=8, lat_h=64, lat_w=64, n_txt=512, txt_dim=4096),
        "flux": dict(big, n_double=19, n_single=38, lat_h=128, lat_w=128, n_txt=512, txt_dim=4096,
                     grad_dtype=BF16, checkpoint=1),
        "qwen": dict(big, n_double=60, n_single=0, lat_h=128, lat_w=128, n_txt=256, txt_dim=4096, checkpoint=1),
    }
    d = dict(table[name])
    d.update(over)
    return Config(**d)
