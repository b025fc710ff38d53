"""ctypes binding of libzeno.so -- argument marshalling only.

Every step of the Zeno aggregation rule (scores, ranking, trimmed mean) runs in
the CUDA kernels behind the C ABI declared in include/zeno.h; this module turns
torch tensors into device pointers and status codes into exceptions.  There is
no CPU fallback: if the shared library is missing or a call fails, it raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Sequence, Union

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libzeno.so")

MAX_LAYERS = 8
MAX_CANDIDATES = 1024

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(6)
LOSS_SOFTMAX_MLP, LOSS_LEAST_SQUARES, LOSS_SOFTMAX_CNN = 0, 1, 2
FAULT_BIT_FLIP, FAULT_SCALE = 0, 1
F32, BF16 = 0, 1

EXPORTS = (
    "zeno_param_count", "zeno_create", "zeno_destroy", "zeno_score", "zeno_select",
    "zeno_aggregate", "zeno_worker_gradients", "zeno_inject_faults", "zeno_score_partial", "zeno_score_from_sums", "zeno_median", "zeno_krum", "zeno_step", "zeno_step_update", "zeno_run", "zeno_step_host", "zeno_device_status", "zeno_score_lsq_static",
    "zeno_debug_set_wait_limit",
    "zeno_profile", "zeno_profile_read",
    "zeno_last_launch_count",
    "zeno_last_cuda_error", "zeno_last_wait_code", "zeno_status_string",
    "zeno_layer_norm", "zeno_layer_norm_gradient", "zeno_layer_norm_gradient_workspace", "zeno_pack_activations",
    "zeno_dense_gradient", "zeno_dense_gradient_workspace", "zeno_token_logprobs", "zeno_token_gradient",
    "zeno_embed", "zeno_embed_gradient", "zeno_embed_gradient_workspace", "zeno_linear_logprobs", "zeno_linear_logprobs_workspace",
    "zeno_linear_logprobs_gradient", "zeno_linear_logprobs_gradient_workspace",
    "zeno_operator_status", "zeno_debug_set_operator_wait_limit",
)


class ModelDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("param_dtype", ctypes.c_int32),
                ("n_layers", ctypes.c_int32), ("has_bias", ctypes.c_int32),
                ("dims", ctypes.c_int64 * (MAX_LAYERS + 1))]


class Batch(ctypes.Structure):
    _fields_ = [("features", ctypes.c_void_p), ("targets", ctypes.c_void_p),
                ("n_r", ctypes.c_int32)]


class RowsDesc(ctypes.Structure):
    """zeno_rows: where the rows of m groups of activations lie (strides in elements)."""
    _fields_ = [("data", ctypes.c_void_p), ("row", ctypes.c_int64), ("group", ctypes.c_int64)]


class ZenoError(RuntimeError):
    def __init__(self, status: int, what: str, detail: str = ""):
        self.status = status
        super().__init__(f"{what}: status {status} ({status_string(status)}){detail}")


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads libzeno.so; raises if it has not been built (python -m paper_1805_10032_b200.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_1805_10032_b200.build` "
            "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.zeno_param_count.restype = i64
    lib.zeno_param_count.argtypes = [ctypes.POINTER(ModelDesc)]
    lib.zeno_create.restype = i32
    lib.zeno_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(ModelDesc), i32, i32, i32]
    lib.zeno_destroy.restype = i32
    lib.zeno_destroy.argtypes = [vp]
    lib.zeno_score.restype = i32
    lib.zeno_score.argtypes = [vp, vp, vp, i64, i32, ctypes.POINTER(Batch), f32, f32, vp, vp, vp, vp]
    lib.zeno_select.restype = i32
    lib.zeno_select.argtypes = [vp, vp, i32, i32, vp, vp]
    lib.zeno_aggregate.restype = i32
    lib.zeno_aggregate.argtypes = [vp, vp, i64, i32, vp, i32, vp, vp]
    lib.zeno_worker_gradients.restype = i32
    lib.zeno_worker_gradients.argtypes = [vp, vp, vp, vp, i32, i32, vp, vp, i64, vp]
    lib.zeno_inject_faults.restype = i32
    lib.zeno_inject_faults.argtypes = [vp, vp, i64, i32, vp, i32, i32, f32, vp]
    lib.zeno_score_partial.restype = i32
    lib.zeno_score_partial.argtypes = [vp, vp, vp, i64, i32, vp, i32, vp, vp]
    lib.zeno_score_from_sums.restype = i32
    lib.zeno_score_from_sums.argtypes = [vp, vp, vp, i32, i32, f32, f32, vp, vp, vp, vp]
    lib.zeno_median.restype = i32
    lib.zeno_median.argtypes = [vp, vp, i64, i32, vp, vp]
    lib.zeno_krum.restype = i32
    lib.zeno_krum.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp, vp]
    lib.zeno_step.restype = i32
    lib.zeno_step.argtypes = [vp, vp, vp, i64, i32, ctypes.POINTER(Batch), f32, f32, i32, vp, vp, vp, vp]
    lib.zeno_run.restype = i32
    lib.zeno_run.argtypes = [vp, vp, vp, i64, i64, i32, vp, vp, i32, i32, f32, f32, i32, vp, vp, vp]
    lib.zeno_step_update.restype = i32
    lib.zeno_step_update.argtypes = [vp, vp, vp, i64, i32, ctypes.POINTER(Batch), f32, f32, i32, vp, vp, vp, vp]
    lib.zeno_step_host.restype = i32
    lib.zeno_step_host.argtypes = [vp, vp, vp, i64, i32, vp, vp, i32, f32, f32, i32, vp, vp, vp, vp]
    lib.zeno_score_lsq_static.restype = i32
    lib.zeno_score_lsq_static.argtypes = [i32, vp, vp, i64, i64, i32, vp, vp, i32, f32, f32, vp, vp, vp, vp]
    lib.zeno_device_status.restype = i32
    lib.zeno_device_status.argtypes = [vp, vp]
    lib.zeno_debug_set_wait_limit.restype = i32
    lib.zeno_debug_set_wait_limit.argtypes = [vp, ctypes.c_uint32]
    lib.zeno_profile.restype = i32
    lib.zeno_profile.argtypes = [vp, i32]
    lib.zeno_profile_read.restype = i32
    lib.zeno_profile_read.argtypes = [vp, i32, ctypes.POINTER(f32), ctypes.POINTER(ctypes.c_char_p), i32]
    lib.zeno_last_launch_count.restype = i32
    lib.zeno_last_launch_count.argtypes = [vp]
    lib.zeno_last_cuda_error.restype = i32
    lib.zeno_last_cuda_error.argtypes = [vp]
    lib.zeno_last_wait_code.restype = i32
    lib.zeno_last_wait_code.argtypes = [vp]
    lib.zeno_status_string.restype = ctypes.c_char_p
    lib.zeno_status_string.argtypes = [i32]
    rows = ctypes.POINTER(RowsDesc)
    lib.zeno_layer_norm.restype = i32
    lib.zeno_layer_norm.argtypes = [i32, i32, i32, rows, i32, i64, i64, vp, vp, i64, f32, rows, vp, vp, vp]
    lib.zeno_layer_norm_gradient.restype = i32
    lib.zeno_layer_norm_gradient.argtypes = [i32, i32, i32, rows, rows, rows, rows, i32, i64, i64, vp, i64, vp, vp, rows, vp, vp,
                                             i64, vp, i64, vp]
    lib.zeno_layer_norm_gradient_workspace.restype = i64
    lib.zeno_layer_norm_gradient_workspace.argtypes = [i32, i64, i64]
    lib.zeno_pack_activations.restype = i32
    lib.zeno_pack_activations.argtypes = [i32, i32, rows, i32, i64, i64, rows, rows, vp]
    lib.zeno_dense_gradient.restype = i32
    lib.zeno_dense_gradient.argtypes = [i32, i32, i32, rows, rows, rows, i32, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp]
    lib.zeno_dense_gradient_workspace.restype = i64
    lib.zeno_dense_gradient_workspace.argtypes = [i32, rows, rows, i32, i64, i64, i64]
    lib.zeno_operator_status.restype = i32
    lib.zeno_operator_status.argtypes = [i32, vp]
    lib.zeno_debug_set_operator_wait_limit.restype = i32
    lib.zeno_debug_set_operator_wait_limit.argtypes = [ctypes.c_uint32]
    lib.zeno_token_logprobs.restype = i32
    lib.zeno_token_logprobs.argtypes = [i32, i32, rows, i32, i64, i64, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.zeno_token_gradient.restype = i32
    lib.zeno_token_gradient.argtypes = [i32, i32, rows, i32, i64, i64, vp, vp, vp, vp, vp, rows, vp]
    lib.zeno_embed.restype = i32
    lib.zeno_embed.argtypes = [i32, i32, i32, vp, i32, i64, i64, i64, vp, i64, f32, rows, vp]
    lib.zeno_embed_gradient.restype = i32
    lib.zeno_embed_gradient.argtypes = [i32, i32, i32, vp, rows, i32, i64, i64, i64, f32, i32, vp, i64, vp, i64, vp]
    lib.zeno_embed_gradient_workspace.restype = i64
    lib.zeno_embed_gradient_workspace.argtypes = [i32, i64, i64, i64]
    lib.zeno_linear_logprobs.restype = i32
    lib.zeno_linear_logprobs.argtypes = [i32, i32, i32, rows, i32, i64, i64, i64, vp, i64, vp, f32, vp, vp, vp, i64, vp]
    lib.zeno_linear_logprobs_workspace.restype = i64
    lib.zeno_linear_logprobs_workspace.argtypes = [i32, i32, i32, i64, i64, i64, vp, i64]
    lib.zeno_linear_logprobs_gradient.restype = i32
    lib.zeno_linear_logprobs_gradient.argtypes = [i32, i32, i32, rows, i32, i64, i64, i64, vp, i64, vp, f32, vp, vp, rows, vp, i64, vp, i64, vp]
    lib.zeno_linear_logprobs_gradient_workspace.restype = i64
    lib.zeno_linear_logprobs_gradient_workspace.argtypes = [i32, i32, i32, i64, i64, i64, vp, i64, i32]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().zeno_status_string(int(status)).decode()


def make_desc(kind: int, param_dtype: int, dims: Sequence[int], has_bias: bool = True) -> ModelDesc:
    if len(dims) > MAX_LAYERS + 1:
        raise ValueError("too many layers")
    d = ModelDesc()
    d.kind = kind
    d.param_dtype = param_dtype
    # a convolutional network's list starts with the image side: [S, C_0, C_1, .., C_Lc, classes]
    d.n_layers = len(dims) - 2 if kind == LOSS_SOFTMAX_CNN else len(dims) - 1
    d.has_bias = int(has_bias)
    for i, v in enumerate(dims):
        d.dims[i] = int(v)
    return d


def param_count(desc: ModelDesc) -> int:
    return int(load_library().zeno_param_count(ctypes.byref(desc)))


# A step of a small model is over on the GPU in 9 us, so what the binding spends on a call shows: addresses go to
# ctypes as plain integers, the stream is read without building a Stream object, the device object is made once.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


class Zeno:
    """A handle for one model shape on one device (zeno_create / zeno_destroy).

    All tensors are CUDA tensors on the handle's device; outputs are allocated by the
    caller side of this binding with torch (device memory is torch's job here)."""

    def __init__(self, kind: int, param_dtype: int, dims: Sequence[int], has_bias: bool = True,
                 m_max: int = 128, n_r_max: int = 128, device: int = 0):
        self._lib = load_library()
        self.desc = make_desc(kind, param_dtype, dims, has_bias)
        self.kind, self.param_dtype = kind, param_dtype
        self.dims = tuple(int(v) for v in dims)
        self.device = int(device)
        self._torch_device = torch.device("cuda", self.device)
        self.m_max, self.n_r_max = int(m_max), int(n_r_max)
        self._h = ctypes.c_void_p()
        st = self._lib.zeno_create(ctypes.byref(self._h), ctypes.byref(self.desc), self.m_max,
                                   self.n_r_max, self.device)
        if st != OK:
            self._h = ctypes.c_void_p()
            raise ZenoError(st, "zeno_create")
        self.d = param_count(self.desc)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.zeno_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- helpers ------------------------------------------------------------------------
    def _check(self, st: int, what: str):
        if st != OK:
            detail = ""
            if st == ERR_CUDA:
                detail = f" [cudaError {self._lib.zeno_last_cuda_error(self._h)}]"
            if st == ERR_TIMEOUT:
                detail = f" [wait code {self._lib.zeno_last_wait_code(self._h):#x}]"
            raise ZenoError(st, what, detail)

    def _batch(self, features: torch.Tensor, targets: torch.Tensor) -> Batch:
        return Batch(features.data_ptr(), targets.data_ptr(), targets.shape[0])

    def _dev(self):
        return self._torch_device

    @property
    def last_launch_count(self) -> int:
        return int(self._lib.zeno_last_launch_count(self._h))

    def check_device_status(self, stream=None):
        """Synchronises and raises if a kernel gave up on a bounded device-side wait."""
        self._check(self._lib.zeno_device_status(self._h, _stream_ptr(stream)), "zeno_device_status")

    def debug_set_wait_limit(self, polls: int):
        """Test hook: polls a bounded device-side wait may take before it gives up (see zeno.h)."""
        self._check(self._lib.zeno_debug_set_wait_limit(self._h, int(polls)), "zeno_debug_set_wait_limit")

    @property
    def last_wait_code(self) -> int:
        return int(self._lib.zeno_last_wait_code(self._h))

    def profile(self, enable: bool = True):
        self._check(self._lib.zeno_profile(self._h, int(enable)), "zeno_profile")

    def profile_read(self, back: int = 0):
        """[(kernel name, milliseconds)] of the call made `back` calls ago, in launch order."""
        cap = 32
        ms = (ctypes.c_float * cap)()
        names = (ctypes.c_char_p * cap)()
        n = self._lib.zeno_profile_read(self._h, int(back), ms, names, cap)
        if n < 0:
            raise ZenoError(ERR_CUDA, "zeno_profile_read")
        return [(names[i].decode(), float(ms[i])) for i in range(n)]

    # -- the four calls -------------------------------------------------------------------
    def score(self, x, V, features, targets, gamma, rho, m=None, ldv=None, want_losses=True,
              want_norms=True, stream=None):
        """Returns (scores[m], losses[m+1] or None, norms[m] or None) as CUDA float32 tensors."""
        m = V.shape[0] if m is None else m
        ldv = V.stride(0) if ldv is None else ldv
        scores = torch.empty(m, dtype=torch.float32, device=self._dev())
        losses = torch.empty(m + 1, dtype=torch.float32, device=self._dev()) if want_losses else None
        norms = torch.empty(m, dtype=torch.float32, device=self._dev()) if want_norms else None
        b = self._batch(features, targets)
        st = self._lib.zeno_score(self._h, _ptr(x), _ptr(V), int(ldv), int(m), ctypes.byref(b),
                                  float(gamma), float(rho), _ptr(scores), _ptr(losses), _ptr(norms),
                                  _stream_ptr(stream))
        self._check(st, "zeno_score")
        return scores, losses, norms

    def select(self, scores, b, m=None, stream=None):
        """Returns idx[m-b] (int32, rank order)."""
        m = scores.shape[0] if m is None else m
        idx = torch.empty(max(m - b, 0), dtype=torch.int32, device=self._dev())
        st = self._lib.zeno_select(self._h, _ptr(scores), int(m), int(b), _ptr(idx),
                                   _stream_ptr(stream))
        self._check(st, "zeno_select")
        return idx

    def aggregate(self, V, idx, m=None, ldv=None, k=None, out=None, stream=None):
        """Returns out[d] float32 = mean of the rows idx of V."""
        m = V.shape[0] if m is None else m
        ldv = V.stride(0) if ldv is None else ldv
        k = idx.shape[0] if k is None else k
        if out is None:
            out = torch.empty(self.d, dtype=torch.float32, device=self._dev())
        st = self._lib.zeno_aggregate(self._h, _ptr(V), int(ldv), int(m), _ptr(idx), int(k),
                                      _ptr(out), _stream_ptr(stream))
        self._check(st, "zeno_aggregate")
        return out

    def worker_gradients(self, x, features, targets, V, label_flip=None, stream=None):
        """Algorithm 1's worker lines: row i of V <- the gradient at x of worker i's mean loss over its own batch
        (features [m, n, in], targets [m, n]); label_flip: int32 [m] device tensor or None."""
        m, n = features.shape[0], features.shape[1]
        st = self._lib.zeno_worker_gradients(self._h, _ptr(x), _ptr(features), _ptr(targets), int(n), int(m),
                                             _ptr(label_flip), _ptr(V), int(V.stride(0)), _stream_ptr(stream))
        self._check(st, "zeno_worker_gradients")
        return V

    def inject_faults(self, V, faulty, mode, eps=0.0, stream=None):
        """The experiments' failures on the rows `faulty` (int32 device tensor) of V, in place."""
        st = self._lib.zeno_inject_faults(self._h, _ptr(V), int(V.stride(0)), int(V.shape[0]), _ptr(faulty),
                                          int(faulty.shape[0]), int(mode), float(eps), _stream_ptr(stream))
        self._check(st, "zeno_inject_faults")
        return V

    def score_partial(self, x, V, features, m=None, ldv=None, sums=None, stream=None):
        """This handle's column slice of the least-squares score sums: float64 [(m+1), (n_r+1)]."""
        m = V.shape[0] if m is None else m
        ldv = V.stride(0) if ldv is None else ldv
        n_r = features.shape[0]
        if sums is None:
            sums = torch.empty((m + 1, n_r + 1), dtype=torch.float64, device=self._dev())
        st = self._lib.zeno_score_partial(self._h, _ptr(x), _ptr(V), int(ldv), int(m), _ptr(features), int(n_r),
                                          _ptr(sums), _stream_ptr(stream))
        self._check(st, "zeno_score_partial")
        return sums

    def score_from_sums(self, sums, targets, gamma, rho, stream=None):
        """Definition 2's scores from the sums of all slices: returns (scores[m], losses[m+1], norms[m])."""
        m, n_r = sums.shape[0] - 1, sums.shape[1] - 1
        scores = torch.empty(m, dtype=torch.float32, device=self._dev())
        losses = torch.empty(m + 1, dtype=torch.float32, device=self._dev())
        norms = torch.empty(m, dtype=torch.float32, device=self._dev())
        st = self._lib.zeno_score_from_sums(self._h, _ptr(sums), _ptr(targets), int(m), int(n_r), float(gamma),
                                            float(rho), _ptr(scores), _ptr(losses), _ptr(norms), _stream_ptr(stream))
        self._check(st, "zeno_score_from_sums")
        return scores, losses, norms

    def median(self, V, m=None, ldv=None, out=None, stream=None):
        """The marginal median of the candidates (the paper's Median baseline): out[d] float32."""
        m = V.shape[0] if m is None else m
        ldv = V.stride(0) if ldv is None else ldv
        if out is None:
            out = torch.empty(self.d, dtype=torch.float32, device=self._dev())
        self._check(self._lib.zeno_median(self._h, _ptr(V), int(ldv), int(m), _ptr(out), _stream_ptr(stream)),
                    "zeno_median")
        return out

    def krum(self, V, b, m=None, ldv=None, want_out=True, stream=None):
        """Krum_b (the paper's Krum baseline): returns (out[d] or None, k int32[1], sums[m])."""
        m = V.shape[0] if m is None else m
        ldv = V.stride(0) if ldv is None else ldv
        out = torch.empty(self.d, dtype=torch.float32, device=self._dev()) if want_out else None
        k = torch.empty(1, dtype=torch.int32, device=self._dev())
        sums = torch.empty(m, dtype=torch.float32, device=self._dev())
        self._check(self._lib.zeno_krum(self._h, _ptr(V), int(ldv), int(m), int(b), _ptr(out), _ptr(k), _ptr(sums),
                                        _stream_ptr(stream)), "zeno_krum")
        return out, k, sums

    def step(self, x, V, features, targets, gamma, rho, b, m=None, ldv=None, out=None,
             scores=None, idx=None, want_scores=True, want_idx=True, stream=None):
        """Zeno_b: returns (out[d], scores[m] or None, idx[m-b] or None)."""
        m = V.shape[0] if m is None else m
        ldv = V.stride(0) if ldv is None else ldv
        if out is None:
            out = torch.empty(self.d, dtype=torch.float32, device=self._dev())
        if scores is None and want_scores:
            scores = torch.empty(m, dtype=torch.float32, device=self._dev())
        if idx is None and want_idx:
            idx = torch.empty(max(m - b, 0), dtype=torch.int32, device=self._dev())
        bt = self._batch(features, targets)
        st = self._lib.zeno_step(self._h, _ptr(x), _ptr(V), int(ldv), int(m), ctypes.byref(bt),
                                 float(gamma), float(rho), int(b), _ptr(out), _ptr(scores), _ptr(idx),
                                 _stream_ptr(stream))
        self._check(st, "zeno_step")
        return out, scores, idx

    def step_update(self, x, V, features, targets, gamma, rho, b, m=None, ldv=None, out=None,
                    scores=None, idx=None, want_out=True, want_scores=True, want_idx=True, stream=None):
        """Zeno_b followed by the server update x <- x - gamma * average, in place and in the pass that
        forms the average.  Returns (out[d] or None, scores[m] or None, idx[m-b] or None)."""
        m = V.shape[0] if m is None else m
        ldv = V.stride(0) if ldv is None else ldv
        if out is None and want_out:
            out = torch.empty(self.d, dtype=torch.float32, device=self._dev())
        if scores is None and want_scores:
            scores = torch.empty(m, dtype=torch.float32, device=self._dev())
        if idx is None and want_idx:
            idx = torch.empty(max(m - b, 0), dtype=torch.int32, device=self._dev())
        bt = self._batch(features, targets)
        st = self._lib.zeno_step_update(self._h, _ptr(x), _ptr(V), int(ldv), int(m), ctypes.byref(bt),
                                        float(gamma), float(rho), int(b), _ptr(out), _ptr(scores),
                                        _ptr(idx), _stream_ptr(stream))
        self._check(st, "zeno_step_update")
        return out, scores, idx

    def run(self, x, V, features, targets, gamma, rho, b, scores=None, idx=None, stream=None):
        """Algorithm 1's server loop: V [steps, m, ldv], features [steps, n_r, in], targets [steps, n_r];
        x is updated in place.  Returns (scores [steps, m], idx [steps, m - b])."""
        steps, m = V.shape[0], V.shape[1]
        ldv, stride = V.stride(1), V.stride(0)
        n_r = features.shape[1]
        assert features.is_contiguous() and targets.is_contiguous()
        if scores is None:
            scores = torch.empty((steps, m), dtype=torch.float32, device=self._dev())
        if idx is None:
            idx = torch.empty((steps, max(m - b, 0)), dtype=torch.int32, device=self._dev())
        st = self._lib.zeno_run(self._h, _ptr(x), _ptr(V), int(ldv), int(stride), int(m), _ptr(features),
                                _ptr(targets), int(n_r), int(steps), float(gamma), float(rho), int(b),
                                _ptr(scores), _ptr(idx), _stream_ptr(stream))
        self._check(st, "zeno_run")
        return scores, idx

    def step_host(self, x, V, features, targets, gamma, rho, b, out, scores=None, idx=None,
                  m=None, ldv=None, stream=None):
        """Host-memory variant: all tensors are CPU tensors (pinned for asynchronous copies);
        `out` (float32 [d]) is filled on return."""
        m = V.shape[0] if m is None else m
        ldv = V.stride(0) if ldv is None else ldv
        st = self._lib.zeno_step_host(self._h, _ptr(x), _ptr(V), int(ldv), int(m), _ptr(features),
                                      _ptr(targets), int(targets.shape[0]), float(gamma), float(rho),
                                      int(b), _ptr(out), _ptr(scores), _ptr(idx), _stream_ptr(stream))
        self._check(st, "zeno_step_host")
        return out


STATIC_MAX_M, STATIC_MAX_N_R = 64, 32


def score_lsq_static(x, V, A, y, gamma, rho, scores, losses=None, norms=None, m=None, ldv=None,
                     device=0, stream=None):
    """zeno_score_lsq_static: least-squares scores with no allocation anywhere -- the caller passes
    every buffer (CUDA tensors: x [d], V [m, ldv], A [n_r, d], y [n_r], scores [m] float32; losses
    [m+1] and norms [m] optional).  For callers that may not call the CUDA allocator; m <= 64 and
    n_r <= 32.  Calls whose kernels could overlap on the GPU must be ordered by the caller."""
    lib = load_library()
    m = V.shape[0] if m is None else m
    ldv = V.stride(0) if ldv is None else ldv
    st = lib.zeno_score_lsq_static(int(device), _ptr(x), _ptr(V), int(ldv), int(x.shape[0]), int(m),
                                   _ptr(A), _ptr(y), int(y.shape[0]), float(gamma), float(rho),
                                   _ptr(scores), _ptr(losses), _ptr(norms), _stream_ptr(stream))
    if st != OK:
        raise ZenoError(st, "zeno_score_lsq_static")
    return scores


# -- operators of language models -----------------------------------------------------------------------------------------
# No handle: the device is the tensors', the stream its current one unless one is given, and what a call allocates (outputs
# that are not passed in, scratch) belongs to that stream.  Activations are [m, n, columns] -- n tokens of each of m workers or
# models -- or [n, columns]; any strides whose last one is 1, and inputs may be expanded over the groups.  Arguments that do
# not fit raise ValueError, what the library refuses raises ZenoError.  They record nothing for autograd: a backward pass is a call.

SAVED_BLOCK = 128
MAX_TOP = 32
_TYPES = {torch.float32: F32, torch.bfloat16: BF16}


class Saved(NamedTuple):
    """Activations kept in 8 bits: codes (float8_e4m3fn, shaped like the activations; rows start at multiples of 16 bytes)
    and the scales of every 128 columns (float32 [.., ceil(columns / 128)]).  The values are codes * scales."""
    codes: torch.Tensor
    scales: torch.Tensor


class TokenLogprobs(NamedTuple):
    logprobs: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor
    top_idx: Optional[torch.Tensor]
    top_logprobs: Optional[torch.Tensor]


class LinearLogprobs(NamedTuple):
    logprobs: torch.Tensor
    lse: torch.Tensor


# Calls of a few tokens are over on the GPU in a few microseconds, so here too what the binding spends on a call shows: messages are built only for
# a refusal, shapes and strides are read once, devices are compared by their index, empty_like and empty_strided (1.4 and 1.6 us) stand in for empty (2.4).
_DEVICES = [torch.device("cuda", i) for i in range(64)]
_EMPTY, _EMPTY_LIKE = torch.empty_strided, torch.empty_like
_ROWS = RowsDesc


def _refuse(what: str):
    raise ValueError(what)


def _type(t: torch.Tensor, name: str) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        _refuse(f"{name}: float32 or bfloat16 is needed, not {t.dtype}")
    return kind


def _rows(t: torch.Tensor, name: str) -> RowsDesc:
    strides = t.stride()
    if len(strides) == 3:
        group, row, last = strides
    elif len(strides) == 2:
        group, (row, last) = 0, strides
    else:
        _refuse(f"{name}: [m, n, columns] or [n, columns] is needed, not {tuple(t.shape)}")
    if last != 1 and t.shape[-1] > 1:
        _refuse(f"{name}: the last stride has to be 1")
    return _ROWS(t.data_ptr(), row, group)


def _sizes(shape):
    if len(shape) == 3:
        return shape
    if len(shape) != 2:
        _refuse(f"[m, n, columns] or [n, columns] is needed, not {tuple(shape)}")
    return 1, shape[0], shape[1]


def _device(t: torch.Tensor, *others) -> int:
    """The index of the device that all of the tensors (or None) are on."""
    index = t.get_device()
    if index < 0:
        _refuse("CUDA tensors are needed")
    for o in others:
        if o is not None and o.get_device() != index:
            _refuse(f"CUDA tensors on one device are needed, not {t.device} and {o.device}")
    return index


def _per_token(t: torch.Tensor, lead, dtype, name: str):
    if t.dtype != dtype or t.shape != lead or not t.is_contiguous():
        _refuse(f"{name}: contiguous {dtype} {tuple(lead)} is needed")


def _current(index: int, stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream(index).cuda_stream
    return _raw_stream(index)


def _empty(stream, index: int, shape, dtype) -> torch.Tensor:
    """An output or scratch of one to three dimensions, contiguous: memory of the stream that the call runs on."""
    if len(shape) == 2:
        strides = shape[1], 1
    else:
        strides = (1,) if len(shape) == 1 else (shape[1] * shape[2], shape[2], 1)
    if stream is None:
        return _EMPTY(shape, strides, dtype=dtype, device=_DEVICES[index])
    with torch.cuda.stream(stream):
        return _EMPTY(shape, strides, dtype=dtype, device=_DEVICES[index])


def _empty_like(stream, t: torch.Tensor, dtype=None) -> torch.Tensor:
    """The same in the shape of t (and its order of dimensions)."""
    if stream is None:
        return _EMPTY_LIKE(t) if dtype is None else _EMPTY_LIKE(t, dtype=dtype)
    with torch.cuda.stream(stream):
        return _EMPTY_LIKE(t, dtype=dtype)


def _done(st: int, what: str):
    raise ZenoError(st, what)


def _norm_weight(w: torch.Tensor, m: int, cols: int) -> int:
    """Elements between the groups' weights: 0 if they share them."""
    shape = w.shape
    if len(shape) == 1:
        if shape[0] == cols and (cols == 1 or w.stride(0) == 1):
            return 0
    elif len(shape) == 2 and shape[0] == m and shape[1] == cols:
        row, last = w.stride()
        if last == 1 or cols == 1:
            return row if m > 1 else 0
    _refuse(f"weight and bias: [{cols}] or [{m}, {cols}] with a last stride of 1 is needed")


def _alike(t: torch.Tensor, like: torch.Tensor, name: str):
    if t.shape != like.shape or t.dtype != like.dtype:
        _refuse(f"{name}: {like.dtype} {tuple(like.shape)} is needed")


def layer_norm(x, weight, bias=None, eps=1e-5, out=None, want_stats=True, stream=None):
    """zeno_layer_norm: returns (y, mean or None, rstd or None).  weight, bias: [columns], or [m, columns] where every model has its own (of one
    stride: slices of the models' parameter vectors).  out may be x."""
    lib = load_library()
    shape = x.shape
    m, n, cols = _sizes(shape)
    dev = _device(x, weight, bias, out)
    ldw = _norm_weight(weight, m, cols)
    if bias is not None and (bias.dtype != weight.dtype or bias.shape != weight.shape or _norm_weight(bias, m, cols) != ldw):
        _refuse("bias: the type and layout of the weight is needed")
    if out is None:
        out = _empty_like(stream, x)
    else:
        _alike(out, x, "out")
    mean = rstd = None
    if want_stats:
        mean = _empty(stream, dev, shape[:-1], torch.float32)
        rstd = _empty_like(stream, mean)
    st = lib.zeno_layer_norm(dev, _type(x, "x"), _type(weight, "weight"), _rows(x, "x"), m, n, cols, weight.data_ptr(), _ptr(bias), ldw, eps,
                             _rows(out, "out"), _ptr(mean), _ptr(rstd), _current(dev, stream))
    return (out, mean, rstd) if st == OK else _done(st, "zeno_layer_norm")


def _saved_rows(saved, lead, cols: int):
    codes, scales = saved
    if codes.dtype not in (torch.float8_e4m3fn, torch.uint8) or codes.shape != (*lead, cols):
        _refuse(f"codes: float8_e4m3fn {(*lead, cols)} is needed")
    if scales.dtype != torch.float32 or scales.shape != (*lead, -(-cols // SAVED_BLOCK)):
        _refuse(f"scales: float32 {(*lead, -(-cols // SAVED_BLOCK))} is needed")
    return _rows(codes, "codes"), _rows(scales, "scales")


def _gradient_row(t: torch.Tensor, m: int, cols: int, dtype, name: str) -> int:
    """Elements between the groups' gradients."""
    shape = t.shape
    if t.dtype == dtype:
        if len(shape) == 2 and shape[0] == m and shape[1] == cols:
            row, last = t.stride()
            if last == 1 or cols == 1:
                return row
        elif m == 1 and len(shape) == 1 and shape[0] == cols and (cols == 1 or t.stride(0) == 1):
            return cols
    _refuse(f"{name}: {dtype} [{m}, {cols}] with a last stride of 1 is needed")


def layer_norm_gradient(dy, x: Union[torch.Tensor, Saved], weight, mean, rstd, dweight=None, dbias=None, dx=None, want_dx=True,
                        stream=None):
    """zeno_layer_norm_gradient: writes dweight and dbias ([m, columns], for instance V[:, at:at + columns], of one stride) and
    returns dx (None if not wanted).  x: the layer's input, or what pack_activations kept of it.  dx may be dy."""
    lib = load_library()
    shape = dy.shape
    lead = shape[:-1]
    m, n, cols = _sizes(shape)
    x_rows = codes = scales = None
    if isinstance(x, tuple):
        dev = _device(dy, x[0], x[1], weight, mean, rstd, dweight, dbias, dx)
        codes, scales = _saved_rows(x, lead, cols)
    else:
        dev = _device(dy, x, weight, mean, rstd, dweight, dbias, dx)
        _alike(x, dy, "x")
        x_rows = _rows(x, "x")
    _per_token(mean, lead, torch.float32, "mean")
    _per_token(rstd, lead, torch.float32, "rstd")
    ldw = _norm_weight(weight, m, cols)
    ldg = 0
    if dweight is not None:
        ldg = _gradient_row(dweight, m, cols, weight.dtype, "dweight")
    if dbias is not None:
        ldb = _gradient_row(dbias, m, cols, weight.dtype, "dbias")
        if dweight is None:
            ldg = ldb
        elif ldb != ldg and m > 1:
            _refuse("dbias: the stride of dweight is needed")
    if dx is not None:
        _alike(dx, dy, "dx")
    elif want_dx:
        dx = _empty_like(stream, dy)
    nbytes = lib.zeno_layer_norm_gradient_workspace(m, n, cols)
    ws = _empty(stream, dev, (nbytes,), torch.uint8) if nbytes else None
    st = lib.zeno_layer_norm_gradient(dev, _type(dy, "dy"), _type(weight, "weight"), _rows(dy, "dy"), x_rows, codes, scales, m, n, cols,
                                      weight.data_ptr(), ldw, mean.data_ptr(), rstd.data_ptr(), None if dx is None else _rows(dx, "dx"),
                                      _ptr(dweight), _ptr(dbias), ldg, _ptr(ws), nbytes, _current(dev, stream))
    return dx if st == OK else _done(st, "zeno_layer_norm_gradient")


def pack_activations(x, stream=None) -> Saved:
    """zeno_pack_activations: x in 8 bits, for layer_norm_gradient and dense_gradient."""
    lib = load_library()
    shape = x.shape
    lead = shape[:-1]
    m, n, cols = _sizes(shape)
    dev = _device(x)
    codes = _empty(stream, dev, (*lead, -(-cols // 16) * 16), torch.float8_e4m3fn)
    if cols % 16:
        codes = codes[..., :cols]
    scales = _empty(stream, dev, (*lead, -(-cols // SAVED_BLOCK)), torch.float32)
    st = lib.zeno_pack_activations(dev, _type(x, "x"), _rows(x, "x"), m, n, cols, _rows(codes, "codes"), _rows(scales, "scales"), _current(dev, stream))
    return Saved(codes, scales) if st == OK else _done(st, "zeno_pack_activations")


def dense_gradient(dy, saved: Saved, dweight, dbias=None, stream=None):
    """zeno_dense_gradient: the weight gradient of a dense layer, dy^T x for every group, from x as pack_activations kept it.
    dweight: [m, outputs, inputs] (or without m), contiguous per group, for instance
    V[:, at:at + outputs * inputs].unflatten(1, (outputs, inputs)); dbias: [m, outputs]."""
    lib = load_library()
    dy_shape = dy.shape
    m, n, outputs = _sizes(dy_shape)
    inputs = saved[0].shape[-1]
    dev = _device(dy, saved[0], saved[1], dweight, dbias)
    codes, scales = _saved_rows(saved, dy_shape[:-1], inputs)
    shape, strides = dweight.shape, dweight.stride()
    if not (shape == (m, outputs, inputs) or (m == 1 and shape == (outputs, inputs))):
        _refuse(f"dweight: [{m}, {outputs}, {inputs}] is needed")
    if (inputs > 1 and strides[-1] != 1) or (outputs > 1 and strides[-2] != inputs):
        _refuse("dweight: contiguous for every group is needed")
    ldb = 0 if dbias is None else _gradient_row(dbias, m, outputs, dweight.dtype, "dbias")
    kind, dy_rows = _type(dy, "dy"), _rows(dy, "dy")
    nbytes = lib.zeno_dense_gradient_workspace(kind, dy_rows, codes, m, n, inputs, outputs)
    ws = _empty(stream, dev, (nbytes,), torch.uint8) if nbytes else None
    st = lib.zeno_dense_gradient(dev, kind, _type(dweight, "dweight"), dy_rows, codes, scales, m, n, inputs, outputs, dweight.data_ptr(),
                                 strides[0] if len(shape) == 3 else inputs * outputs, _ptr(dbias), ldb, _ptr(ws), nbytes, _current(dev, stream))
    return dweight if st == OK else _done(st, "zeno_dense_gradient")


def token_logprobs(logits, targets=None, top=0, stream=None) -> TokenLogprobs:
    """zeno_token_logprobs: (logprobs or None without targets, entropy, lse, top_idx, top_logprobs (None if top is 0)) of logits [m, n, vocab] or
    [n, vocab]; targets: int32, one outside the vocabulary means none."""
    lib = load_library()
    shape = logits.shape
    lead = shape[:-1]
    m, n, vocab = _sizes(shape)
    dev = _device(logits, targets)
    if targets is not None:
        _per_token(targets, lead, torch.int32, "targets")
    entropy = _empty(stream, dev, lead, torch.float32)
    lse = _empty_like(stream, entropy)
    lp = None if targets is None else _empty_like(stream, entropy)
    idx = top_lp = None
    if top > 0:
        idx = _empty(stream, dev, (*lead, top), torch.int32)
        top_lp = _empty_like(stream, idx, torch.float32)
    st = lib.zeno_token_logprobs(dev, _type(logits, "logits"), _rows(logits, "logits"), m, n, vocab, _ptr(targets), top, _ptr(lp),
                                 entropy.data_ptr(), lse.data_ptr(), _ptr(idx), _ptr(top_lp), _current(dev, stream))
    return TokenLogprobs(lp, entropy, lse, idx, top_lp) if st == OK else _done(st, "zeno_token_logprobs")


def token_gradient(logits, targets, lse, g_logprob, entropy=None, g_entropy=None, out=None, stream=None):
    """zeno_token_gradient: the gradient at the logits from the gradients at token_logprobs's logprobs and (g_entropy) entropy.
    out may be the logits."""
    lib = load_library()
    shape = logits.shape
    lead = shape[:-1]
    m, n, vocab = _sizes(shape)
    dev = _device(logits, targets, lse, g_logprob, entropy, g_entropy, out)
    _per_token(targets, lead, torch.int32, "targets")
    _per_token(lse, lead, torch.float32, "lse")
    _per_token(g_logprob, lead, torch.float32, "g_logprob")
    if g_entropy is not None:
        if entropy is None:
            _refuse("entropy: needed with g_entropy")
        _per_token(entropy, lead, torch.float32, "entropy")
        _per_token(g_entropy, lead, torch.float32, "g_entropy")
    if out is None:
        out = _empty_like(stream, logits)
    else:
        _alike(out, logits, "out")
    st = lib.zeno_token_gradient(dev, _type(logits, "logits"), _rows(logits, "logits"), m, n, vocab, targets.data_ptr(), lse.data_ptr(),
                                 _ptr(entropy), g_logprob.data_ptr(), _ptr(g_entropy), _rows(out, "out"), _current(dev, stream))
    return out if st == OK else _done(st, "zeno_token_gradient")


def _vocabulary(w: torch.Tensor, name: str):
    """(vocab, columns) of a table or of output weights."""
    if len(w.shape) < 2:
        _refuse(f"{name}: [vocab, columns] or [m, vocab, columns] is needed, not {tuple(w.shape)}")
    return w.shape[-2:]


def _matrix(w: torch.Tensor, m: int, rows: int, cols: int, name: str, shared: bool) -> int:
    """Elements between the groups' matrices of contiguous rows: 0 if they share one."""
    shape, strides = w.shape, w.stride()
    if (shape == (rows, cols) and (shared or m == 1)) or shape == (m, rows, cols):
        if (cols == 1 or strides[-1] == 1) and (rows == 1 or strides[-2] == cols):
            return strides[0] if m > 1 and len(shape) == 3 else 0
    _refuse(f"{name}: [{m}, {rows}, {cols}]{f' or [{rows}, {cols}]' if shared or m == 1 else ''}, contiguous for every group, is needed")


def _group_sizes(tokens: torch.Tensor):
    shape = tokens.shape
    if len(shape) == 2:
        return shape
    if len(shape) != 1:
        _refuse(f"tokens: [m, n] or [n] is needed, not {tuple(shape)}")
    return 1, shape[0]


def embed(tokens, table, scale=1.0, dtype=None, out=None, stream=None):
    """zeno_embed: scale * table[tokens], [m, n, columns] of tokens [m, n] or [n, columns] of [n] (int32; one outside the vocabulary: zeros).  table:
    [vocab, columns], or [m, vocab, columns] where every model has its own, for instance P[:, at:at + vocab * columns].unflatten(1, (vocab,
    columns)).  The result's type is out's, dtype, or the table's."""
    lib = load_library()
    m, n = _group_sizes(tokens)
    vocab, cols = _vocabulary(table, "table")
    dev = _device(tokens, table, out)
    _per_token(tokens, tokens.shape, torch.int32, "tokens")
    ldt = _matrix(table, m, vocab, cols, "table", True)
    shape = (*tokens.shape, cols)
    if out is None:
        out = _empty(stream, dev, shape, dtype or table.dtype)
    elif out.shape != shape or (dtype is not None and out.dtype != dtype):
        _refuse(f"out: {dtype or out.dtype} {shape} is needed")
    st = lib.zeno_embed(dev, _type(out, "out"), _type(table, "table"), tokens.data_ptr(), m, n, vocab, cols, table.data_ptr(), ldt, scale, _rows(out, "out"),
                        _current(dev, stream))
    return out if st == OK else _done(st, "zeno_embed")


def embed_gradient(tokens, dy, dtable, scale=1.0, add=False, stream=None):
    """zeno_embed_gradient: writes dtable ([m, vocab, columns], or without m; a slice of V as in embed) from dy, the gradient at embed's result; with
    add, adds to it (tied weights, after linear_logprobs_gradient)."""
    lib = load_library()
    m, n = _group_sizes(tokens)
    vocab, cols = _vocabulary(dtable, "dtable")
    dev = _device(tokens, dy, dtable)
    _per_token(tokens, dy.shape[:-1], torch.int32, "tokens")
    if dy.shape[-1] != cols:
        _refuse(f"dy: rows of {cols} are needed, not {dy.shape[-1]}")
    ldt = _matrix(dtable, m, vocab, cols, "dtable", False)
    nbytes = lib.zeno_embed_gradient_workspace(m, n, vocab, cols)
    ws = _empty(stream, dev, (nbytes,), torch.uint8) if nbytes else None
    st = lib.zeno_embed_gradient(dev, _type(dy, "dy"), _type(dtable, "dtable"), tokens.data_ptr(), _rows(dy, "dy"), m, n, vocab, cols, scale, add,
                                 dtable.data_ptr(), ldt, _ptr(ws), nbytes, _current(dev, stream))
    return dtable if st == OK else _done(st, "zeno_embed_gradient")


def linear_logprobs(x, weight, targets, scale=1.0, stream=None) -> LinearLogprobs:
    """zeno_linear_logprobs: (logprobs, lse) of the targets (int32; one outside the vocabulary: 0 for both) under the logits scale * x @ weight.T, which
    are not kept.  x: [m, n, columns] or [n, columns]; weight: [vocab, columns], or [m, vocab, columns] where every model has its own."""
    lib = load_library()
    shape = x.shape
    m, n, cols = _sizes(shape)
    vocab = _vocabulary(weight, "weight")[0]
    dev = _device(x, weight, targets)
    _per_token(targets, shape[:-1], torch.int32, "targets")
    ldw = _matrix(weight, m, vocab, cols, "weight", True)
    kind, wkind, w = _type(x, "x"), _type(weight, "weight"), weight.data_ptr()
    logprobs = _empty(stream, dev, shape[:-1], torch.float32)
    lse = _empty_like(stream, logprobs)
    nbytes = lib.zeno_linear_logprobs_workspace(kind, wkind, m, n, cols, vocab, w, ldw)
    ws = _empty(stream, dev, (nbytes,), torch.uint8) if nbytes else None
    st = lib.zeno_linear_logprobs(dev, kind, wkind, _rows(x, "x"), m, n, cols, vocab, w, ldw, targets.data_ptr(), scale, logprobs.data_ptr(), lse.data_ptr(),
                                  _ptr(ws), nbytes, _current(dev, stream))
    return LinearLogprobs(logprobs, lse) if st == OK else _done(st, "zeno_linear_logprobs")


def linear_logprobs_gradient(x, weight, targets, lse, g_logprob, dweight=None, dx=None, want_dx=True, scale=1.0, stream=None):
    """zeno_linear_logprobs_gradient: from the gradient at linear_logprobs's logprobs, writes dweight ([m, vocab, columns], or without m; a slice of V
    as in embed; every group its own, also where the weight is shared) and returns dx (None if not wanted)."""
    lib = load_library()
    shape = x.shape
    lead = shape[:-1]
    m, n, cols = _sizes(shape)
    vocab = _vocabulary(weight, "weight")[0]
    dev = _device(x, weight, targets, lse, g_logprob, dweight, dx)
    _per_token(targets, lead, torch.int32, "targets")
    _per_token(lse, lead, torch.float32, "lse")
    _per_token(g_logprob, lead, torch.float32, "g_logprob")
    ldw = _matrix(weight, m, vocab, cols, "weight", True)
    lddw = 0
    if dweight is not None:
        if dweight.dtype != weight.dtype:
            _refuse(f"dweight: {weight.dtype} is needed")
        lddw = _matrix(dweight, m, vocab, cols, "dweight", False)
    if dx is not None:
        _alike(dx, x, "dx")
    elif want_dx:
        dx = _empty_like(stream, x)
    kind, wkind, w = _type(x, "x"), _type(weight, "weight"), weight.data_ptr()
    nbytes = lib.zeno_linear_logprobs_gradient_workspace(kind, wkind, m, n, cols, vocab, w, ldw, dx is not None)
    ws = _empty(stream, dev, (nbytes,), torch.uint8) if nbytes else None
    st = lib.zeno_linear_logprobs_gradient(dev, kind, wkind, _rows(x, "x"), m, n, cols, vocab, w, ldw, targets.data_ptr(), scale, lse.data_ptr(),
                                           g_logprob.data_ptr(), None if dx is None else _rows(dx, "dx"), _ptr(dweight), lddw, _ptr(ws), nbytes,
                                           _current(dev, stream))
    return dx if st == OK else _done(st, "zeno_linear_logprobs_gradient")


def check_operator_status(device: int = 0, stream=None):
    """Synchronises the stream and raises if a kernel of the operators above gave up on a bounded device-side wait (dense_gradient and
    linear_logprobs on the tensor cores, and the latter's gradient, have them) since this stream was last asked: on this stream, or on another one of the device."""
    st = load_library().zeno_operator_status(device, _current(device, stream))
    if st != OK:
        _done(st, "zeno_operator_status")


def debug_set_operator_wait_limit(polls: int):
    """Test hook: polls a bounded device-side wait of the operators may take before it gives up (see zeno.h)."""
    load_library().zeno_debug_set_operator_wait_limit(polls)


def from_workload(w, m_max=None, n_r_max=None, device=0) -> "Zeno":
    """A handle shaped for a synthetic.Workload."""
    kind = {"lsq": LOSS_LEAST_SQUARES, "cnn": LOSS_SOFTMAX_CNN}.get(w.kind, LOSS_SOFTMAX_MLP)
    dt = BF16 if w.dtype == "bf16" else F32
    return Zeno(kind, dt, w.dims, w.has_bias, m_max or w.m, n_r_max or w.n_r, device)
