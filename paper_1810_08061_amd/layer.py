"""A layer's operators, its training's and its answers': the binding of ``include/lstm_dyn_layer.h``.

``LinearAttention`` (a recurrence whose state is a matrix, with a decay for each head:
whole sequences, gradients, one step), ``LayerNorm`` (and its gradients), ``GradClip`` (the norm of
all gradients, and clipping to it; ``AdamW.step`` takes one) and ``TokenSample`` (one token a row
from given random numbers).  As for the operators of ``ops``: every computation runs in the
library's HIP kernels, a handle has one call in flight, a call runs on the current stream, and
``stream=`` is short for ``with torch.cuda.stream(stream)``.  The ``lstm_dyn_*`` functions mirror the C ABI.
"""
from __future__ import annotations

import ctypes
import operator

from . import BF16, F32, _on, ops
from .ops import _call, _create, _dtype, _Handle, _ok, _query, _t


class SampleFilter(ctypes.Structure):
    """lstm_dyn_sample_filter_t"""
    _fields_ = [("temperature", ctypes.c_float), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
                ("top_k", ctypes.c_int32), ("temperatures", ctypes.c_void_p), ("top_ps", ctypes.c_void_p),
                ("min_ps", ctypes.c_void_p), ("top_ks", ctypes.c_void_p)]


# --- C ABI mirrors ----------------------------------------------------------

def lstm_dyn_norm_create(B: int, T_max: int, D: int, dtype: int, eps: float) -> int:
    return _create("lstm_dyn_norm_create", B, T_max, D, dtype, eps)


def lstm_dyn_norm_forward(handle, x, lengths, weight, bias, out_y, stream=0) -> None:
    _call("lstm_dyn_norm_forward", handle, x, lengths, weight, bias, out_y, stream)


def lstm_dyn_norm_backward(handle, x, lengths, weight, dy, dy_dtype, out_dx, d_weight, d_bias, stream=0) -> None:
    _call("lstm_dyn_norm_backward", handle, x, lengths, weight, dy, dy_dtype, out_dx, d_weight, d_bias, stream)


def lstm_dyn_norm_query(handle, what) -> int:
    return _query("lstm_dyn_norm_query", handle, what)


def lstm_dyn_norm_destroy(handle) -> None:
    _call("lstm_dyn_norm_destroy", handle)


def lstm_dyn_check_norm_args(*args) -> int:
    return ops._lib().lstm_dyn_check_norm_args(*args)


def _counts(n):
    return (ctypes.c_longlong * len(n))(*n)


def _addresses(p):
    return None if p is None else (ctypes.c_void_p * len(p))(*p)


def lstm_dyn_clip_create(n) -> int:
    """n: the tensors' numbers of elements."""
    return _create("lstm_dyn_clip_create", _counts(n), len(n))


def lstm_dyn_clip_norm(handle, grads, grad_dtype, grad_scale, max_norm, result, stream=0) -> None:
    """grads: a ctypes array of pointers."""
    _call("lstm_dyn_clip_norm", handle, grads, grad_dtype, grad_scale, max_norm, result, stream)


def lstm_dyn_clip_apply(handle, grads, grad_dtype, result, out, stream=0) -> None:
    _call("lstm_dyn_clip_apply", handle, grads, grad_dtype, result, out, stream)


def lstm_dyn_clip_query(handle, what) -> int:
    return _query("lstm_dyn_clip_query", handle, what)


def lstm_dyn_clip_destroy(handle) -> None:
    _call("lstm_dyn_clip_destroy", handle)


def lstm_dyn_check_clip_args(n, grads=None, grad_dtype=F32, result=0, out=None) -> int:
    return ops._lib().lstm_dyn_check_clip_args(_counts(n), len(n), _addresses(grads), grad_dtype, result, _addresses(out))


def lstm_dyn_adamw_step_clipped(handle, grads, grad_dtype, lr, beta1, beta2, eps, result, step, stream=0) -> None:
    _call("lstm_dyn_adamw_step_clipped", handle, grads, grad_dtype, lr, beta1, beta2, eps, result, step, stream)


def lstm_dyn_sample_create(N: int, V: int, dtype: int) -> int:
    return _create("lstm_dyn_sample_create", N, V, dtype)


def lstm_dyn_sample_step(handle, logits, u, filter, out_token, out_logp, stream=0) -> None:
    """filter: a SampleFilter by reference, or None."""
    _call("lstm_dyn_sample_step", handle, logits, u, filter, out_token, out_logp, stream)


def lstm_dyn_sample_query(handle, what) -> int:
    return _query("lstm_dyn_sample_query", handle, what)


def lstm_dyn_sample_destroy(handle) -> None:
    _call("lstm_dyn_sample_destroy", handle)


def lstm_dyn_check_sample_args(*args) -> int:
    return ops._lib().lstm_dyn_check_sample_args(*args)


def _floats(x):
    return None if x is None else (ctypes.c_float * len(x))(*x)


def lstm_dyn_attend_create(B: int, heads: int, Dk: int, Dv: int, T_max: int, dtype: int, decay) -> int:
    """decay: one number a head."""
    return _create("lstm_dyn_attend_create", B, heads, Dk, Dv, T_max, dtype, _floats(decay))


def lstm_dyn_attend_forward(handle, z, lengths, S0, out_S, out_y, stream=0) -> None:
    _call("lstm_dyn_attend_forward", handle, z, lengths, S0, out_S, out_y, stream)


def lstm_dyn_attend_backward(handle, z, lengths, S0, dy, d_out_S, dz, dS0, stream=0) -> None:
    _call("lstm_dyn_attend_backward", handle, z, lengths, S0, dy, d_out_S, dz, dS0, stream)


def lstm_dyn_attend_step(handle, rows, z, S, out_S, out_y, stream=0) -> None:
    _call("lstm_dyn_attend_step", handle, rows, z, S, out_S, out_y, stream)


def lstm_dyn_attend_query(handle, what) -> int:
    return _query("lstm_dyn_attend_query", handle, what)


def lstm_dyn_attend_destroy(handle) -> None:
    _call("lstm_dyn_attend_destroy", handle)


def lstm_dyn_check_attend_args(B, heads, Dk, Dv, T_max, dtype, decay, *buffers) -> int:
    return ops._lib().lstm_dyn_check_attend_args(B, heads, Dk, Dv, T_max, dtype, _floats(decay), *buffers)


# --- torch convenience wrappers ---------------------------------------------

def _stream(device):
    return ops._stream(device)


class LinearAttention(_Handle):
    """The recurrence S_t = a S_{t-1} + k_t v_t^T, y_t = S_t^T q_t for each row and head, with the
    head's decay a in [0, 1] (decay: one number a head, or one for all).

    z [B, T_max, heads (2 Dk + Dv)] = (q of all heads, k of all heads, v of all heads) in the
    handle's dtype, lengths int32 [B] or None (all T_max), S0 float32 [B, heads, Dk, Dv]; y [B, T_max,
    heads Dv] is in the handle's dtype, the state float32.  Dk and Dv are at most 128."""
    _kind = "attend"

    def __init__(self, B: int, heads: int, Dk: int, Dv: int, T_max: int, decay, dtype="bf16"):
        self.B, self.heads, self.Dk, self.Dv, self.T = B, heads, Dk, Dv, T_max
        self.dtype, self._et = _dtype(dtype)
        self.decay = [float(decay)] * heads if isinstance(decay, (int, float)) else [float(a) for a in decay]
        if len(self.decay) != heads:
            raise ValueError(f"decay must be one number, or one for each of {heads} heads")
        self._device = _t().cuda.current_device()
        self._width, self._out = heads * (2 * Dk + Dv), heads * Dv
        self.handle = lstm_dyn_attend_create(B, heads, Dk, Dv, T_max, self.dtype, self.decay)

    def _inputs(self, z, lengths, S0):
        torch = _t()
        self._check("z", z, self._et, (self.B, self.T, self._width))
        self._check("S0", S0, torch.float32, (self.B, self.heads, self.Dk, self.Dv))
        if lengths is None:
            return 0
        self._check("lengths", lengths, torch.int32, (self.B,))
        return lengths.data_ptr()

    def forward(self, z, lengths, S0, out_S=None, out_y=None, stream=None):
        """Returns (y, zero past each length, and the state after each row's last step); out_S may be S0."""
        if stream is not None:
            with _on(stream):
                return self.forward(z, lengths, S0, out_S, out_y)
        torch = _t()
        L = self._inputs(z, lengths, S0)
        if out_S is None:
            out_S = torch.empty_like(S0)
        else:
            self._check("out_S", out_S, torch.float32, S0.shape)
        if out_y is None:
            out_y = z.new_empty((self.B, self.T, self._out))
        else:
            self._check("out_y", out_y, self._et, (self.B, self.T, self._out))
        _ok(ops._ready.lstm_dyn_attend_forward(self.handle, z.data_ptr(), L, S0.data_ptr(), out_S.data_ptr(),
                                               out_y.data_ptr(), _stream(z.device)), "lstm_dyn_attend_forward")
        return out_y, out_S

    __call__ = forward

    def backward(self, z, lengths, S0, dy, d_out_S=None, stream=None, out=None):
        """The gradients of ``forward`` (which need not have run): a dict of dz (the handle's dtype) and dS0
        float32.  dy in the handle's dtype; d_out_S float32 [B, heads, Dk, Dv] or None.  out: a dict with those
        keys holding caller-owned tensors."""
        if stream is not None:
            with _on(stream):
                return self.backward(z, lengths, S0, dy, d_out_S, None, out)
        torch = _t()
        L = self._inputs(z, lengths, S0)
        self._check("dy", dy, self._et, (self.B, self.T, self._out))
        if d_out_S is not None:
            self._check("d_out_S", d_out_S, torch.float32, S0.shape)
        if out is None:
            out = {"dz": torch.empty_like(z), "dS0": torch.empty_like(S0)}
        else:
            if sorted(out) != ["dS0", "dz"]:
                raise ValueError("out must hold exactly ['dS0', 'dz']")
            self._check("dz", out["dz"], self._et, z.shape)
            self._check("dS0", out["dS0"], torch.float32, S0.shape)
        _ok(ops._ready.lstm_dyn_attend_backward(self.handle, z.data_ptr(), L, S0.data_ptr(), dy.data_ptr(),
                                                d_out_S.data_ptr() if d_out_S is not None else 0,
                                                out["dz"].data_ptr(), out["dS0"].data_ptr(), _stream(z.device)),
            "lstm_dyn_attend_backward")
        return out

    def step(self, z, S, out_S=None, out_y=None, stream=None):
        """One step of any number of rows: z [R, heads (2 Dk + Dv)], S float32 [R, heads, Dk, Dv]; returns
        (y [R, heads Dv], S).  out_S may be S itself."""
        if stream is not None:
            with _on(stream):
                return self.step(z, S, out_S, out_y)
        torch = _t()
        R = S.shape[0]
        self._check("z", z, self._et, (R, self._width))
        self._check("S", S, torch.float32, (R, self.heads, self.Dk, self.Dv))
        if out_S is None:
            out_S = torch.empty_like(S)
        else:
            self._check("out_S", out_S, torch.float32, S.shape)
        if out_y is None:
            out_y = z.new_empty((R, self._out))
        else:
            self._check("out_y", out_y, self._et, (R, self._out))
        _ok(ops._ready.lstm_dyn_attend_step(self.handle, R, z.data_ptr(), S.data_ptr(), out_S.data_ptr(),
                                            out_y.data_ptr(), _stream(z.device)), "lstm_dyn_attend_step")
        return out_y, out_S


class LayerNorm(_Handle):
    """y = (x - mean) / sqrt(var + eps) weight + bias over the last axis of x [B, T_max, D], zero past
    each length, and its gradients.  x and y in the handle's dtype, lengths int32 [B] or None (all
    T_max), weight and bias float32 [D] or None (ones, zeros).  D is at most 32768."""
    _kind = "norm"

    def __init__(self, B: int, T_max: int, D: int, dtype="bf16", eps: float = 1e-5):
        self.B, self.T, self.D, self.eps = B, T_max, D, float(eps)
        self.dtype, self._et = _dtype(dtype)
        self._device = _t().cuda.current_device()
        self.handle = lstm_dyn_norm_create(B, T_max, D, self.dtype, self.eps)

    def _optional(self, name, t, dtype, shape):
        if t is None:
            return 0
        self._check(name, t, dtype, shape)
        return t.data_ptr()

    def forward(self, x, lengths=None, weight=None, bias=None, out_y=None, stream=None):
        """Returns y; out_y may be x itself."""
        if stream is not None:
            with _on(stream):
                return self.forward(x, lengths, weight, bias, out_y)
        torch = _t()
        self._check("x", x, self._et, (self.B, self.T, self.D))
        L = self._optional("lengths", lengths, torch.int32, (self.B,))
        w = self._optional("weight", weight, torch.float32, (self.D,))
        b = self._optional("bias", bias, torch.float32, (self.D,))
        if out_y is None:
            out_y = torch.empty_like(x)
        else:
            self._check("out_y", out_y, self._et, x.shape)
        _ok(ops._ready.lstm_dyn_norm_forward(self.handle, x.data_ptr(), L, w, b, out_y.data_ptr(), _stream(x.device)),
            "lstm_dyn_norm_forward")
        return out_y

    __call__ = forward

    def backward(self, x, lengths, weight, dy, out=None, stream=None):
        """The gradients of ``forward`` (which need not have run): a dict of dx (in dy's type, float32 or
        bfloat16), dweight and dbias float32 [D].  out: a dict with those keys holding caller-owned
        tensors; dx may be dy itself."""
        if stream is not None:
            with _on(stream):
                return self.backward(x, lengths, weight, dy, out)
        torch = _t()
        self._check("x", x, self._et, (self.B, self.T, self.D))
        L = self._optional("lengths", lengths, torch.int32, (self.B,))
        w = self._optional("weight", weight, torch.float32, (self.D,))
        code = BF16 if isinstance(dy, torch.Tensor) and dy.dtype == torch.bfloat16 else F32
        self._check("dy", dy, torch.bfloat16 if code == BF16 else torch.float32, x.shape)
        if out is None:
            like = weight if weight is not None else x.new_empty((self.D,), dtype=torch.float32)
            out = {"dx": torch.empty_like(dy), "dweight": torch.empty_like(like), "dbias": torch.empty_like(like)}
        else:
            if sorted(out) != ["dbias", "dweight", "dx"]:
                raise ValueError("out must hold exactly ['dbias', 'dweight', 'dx']")
            self._check("dx", out["dx"], dy.dtype, x.shape)
            self._check("dweight", out["dweight"], torch.float32, (self.D,))
            self._check("dbias", out["dbias"], torch.float32, (self.D,))
        _ok(ops._ready.lstm_dyn_norm_backward(self.handle, x.data_ptr(), L, w, dy.data_ptr(), code,
                                              out["dx"].data_ptr(), out["dweight"].data_ptr(), out["dbias"].data_ptr(),
                                              _stream(x.device)), "lstm_dyn_norm_backward")
        return out


class GradClip(_Handle):
    """The norm of the gradients of a list of tensors together, and gradients clipped to max_norm.
    params: tensors with the gradients' shapes (the parameters, or the gradients themselves)."""
    _kind = "clip"

    def __init__(self, params, max_norm: float):
        self.shapes = [p.shape for p in params]
        if not self.shapes:
            raise ValueError("params must not be empty")
        self.max_norm = float(max_norm)
        self._device = _t().cuda.current_device()
        self.handle = lstm_dyn_clip_create([s.numel() for s in self.shapes])
        self._pointers = ctypes.c_void_p * len(self.shapes)

    def _grads(self, name, tensors, et):
        if len(tensors) != len(self.shapes):
            raise ValueError(f"{len(self.shapes)} of {name} are needed, got {len(tensors)}")
        addresses, device = [], self._device
        for t, s in zip(tensors, self.shapes):      # (written out: lists are long, calls few microseconds)
            try:
                if t.dtype is et and t.shape == s and t.get_device() == device and t.is_contiguous():
                    addresses.append(t.data_ptr())
                    continue
            except AttributeError:
                pass
            self._check(name, t, et, s)
            addresses.append(t.data_ptr())
        return self._pointers(*addresses)

    def _type(self, grads):
        torch = _t()
        et = grads[0].dtype if grads and isinstance(grads[0], torch.Tensor) else None
        if et not in (torch.float32, torch.bfloat16):
            raise TypeError("gradients must be float32 or bfloat16 device tensors")
        return et, (BF16 if et == torch.bfloat16 else F32)

    def norm(self, grads, grad_scale: float = 1.0, stream=None):
        """float32 [2]: the norm of all gradients (all float32 or all bfloat16) times grad_scale, and the factor that
        clips them, grad_scale min(1, max_norm / norm)."""
        if stream is not None:
            with _on(stream):
                return self.norm(grads, grad_scale)
        grads = list(grads)
        et, code = self._type(grads)
        return self._norm(self._grads("gradients", grads, et), code, grad_scale, grads[0])

    def _norm(self, g, code, grad_scale, like):
        result = like.new_empty((2,), dtype=_t().float32)
        _ok(ops._ready.lstm_dyn_clip_norm(self.handle, g, code, grad_scale, self.max_norm, result.data_ptr(),
                                          _stream(like.device)), "lstm_dyn_clip_norm")
        return result

    def clip(self, grads, grad_scale: float = 1.0, out=None, stream=None):
        """``norm``, and the gradients times its factor: in place, or into the tensors of out."""
        if stream is not None:
            with _on(stream):
                return self.clip(grads, grad_scale, out)
        grads = list(grads)
        et, code = self._type(grads)
        g = self._grads("gradients", grads, et)
        o = g if out is None else self._grads("out", list(out), et)
        result = self._norm(g, code, grad_scale, grads[0])
        _ok(ops._ready.lstm_dyn_clip_apply(self.handle, g, code, result.data_ptr(), o, _stream(result.device)),
            "lstm_dyn_clip_apply")
        return result


class TokenSample(_Handle):
    """One token for each of N rows over a vocabulary of V, from given random numbers."""
    _kind = "sample"

    def __init__(self, N: int, V: int, dtype="bf16"):
        self.N, self.V = N, V
        self.dtype, self._et = _dtype(dtype)
        self._device = _t().cuda.current_device()
        self.handle = lstm_dyn_sample_create(N, V, self.dtype)
        self._filter = SampleFilter()      # read before a call returns
        self._filter_at = ctypes.byref(self._filter)

    def sample(self, logits, u, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
        """Returns (token int32 [N], the log of its probability among the tokens kept, float32 [N]).

        logits [N, V] in the handle's dtype, u float32 [N] in [0, 1).  Each of temperature,
        top_p, min_p (float32) and top_k (int32) is a number, a tensor [N] with one a row, or None
        (1 and no limit).  Kept are the first top_k tokens by logit, of those the shortest start with top_p
        of their probability, of those the ones with at least min_p of the first one's; the token is where the
        running sum of their probabilities by index passes u.  A temperature of zero takes the
        first token.  A row of nothing but -inf (or NaN) gives token -1 and logp -inf."""
        if stream is not None:
            with _on(stream):
                return self.sample(logits, u, temperature, top_k, top_p, min_p)
        torch = _t()
        N = self.N
        self._check("logits", logits, self._et, (N, self.V))
        self._check("u", u, torch.float32, (N,))
        f = self._filter
        f.temperature, f.top_p, f.min_p, f.top_k = 1.0, 1.0, 0.0, 0
        f.temperatures = f.top_ps = f.min_ps = f.top_ks = None
        for name, value in (("temperature", temperature), ("top_p", top_p), ("min_p", min_p), ("top_k", top_k)):
            if value is None:
                continue
            if isinstance(value, torch.Tensor):
                self._check(name, value, torch.int32 if name == "top_k" else torch.float32, (N,))
                setattr(f, name + "s", value.data_ptr())
            elif name == "top_k":       # (a number that the structure's 32 bits do not hold would be cut to its low ones)
                f.top_k = max(0, min(operator.index(value), self.V))
            else:
                setattr(f, name, value)
        token, logp = torch.empty_like(u, dtype=torch.int32), torch.empty_like(u)
        _ok(ops._ready.lstm_dyn_sample_step(self.handle, logits.data_ptr(), u.data_ptr(), self._filter_at,
                                            token.data_ptr(), logp.data_ptr(), _stream(logits.device)),
            "lstm_dyn_sample_step")
        return token, logp
