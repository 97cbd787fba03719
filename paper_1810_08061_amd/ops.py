"""Operators around the time loop: the binding of ``include/lstm_dyn_ops.h``.

``TokenEmbed`` (rows of a token table and the table's gradient), ``GatedScan``
(a gated linear recurrence, its backward pass and its single step), ``AdamW``
(one optimizer step over many tensors) and ``BeamSearch`` (one selection over
beams and vocabulary).  As for ``LstmDyn``: every computation runs in the
library's HIP kernels, torch owns device memory and names streams, a handle has
one call in flight.  A call runs on the current stream; ``stream=`` (a torch stream or
its address) is short for ``with torch.cuda.stream(stream)``: the results belong to
that stream, which waits for no other by itself.  The ``lstm_dyn_*`` functions
mirror the C ABI.
"""
from __future__ import annotations

import ctypes

from . import BF16, F32, OK, LstmDynError, _DTYPES, _load, _on

ERR_BAD_TOKENS = 8
OPS_Q_STATUS, OPS_Q_WORKSPACE_BYTES, OPS_Q_LAUNCHES = range(3)
BEAM_MAX_K, BEAM_MAX_STATES = 32, 8
STATE_BLOCK = 256   # elements that share the exponent of an 8-bit state


class AdamwTensor(ctypes.Structure):
    """lstm_dyn_adamw_tensor_t"""
    _fields_ = [("p", ctypes.c_void_p), ("p_bf16", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("n", ctypes.c_longlong), ("weight_decay", ctypes.c_float)]


class BeamState(ctypes.Structure):
    """lstm_dyn_beam_state_t"""
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("row_bytes", ctypes.c_longlong)]


_ready = None


def _lib():
    global _ready
    if _ready is not None:
        return _ready
    lib = _load()
    P, I, LL = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong
    F, DB = ctypes.c_float, ctypes.c_double
    PP, PLL = ctypes.POINTER(P), ctypes.POINTER(LL)
    for name, args in {
        "scan_create": [PP, I, I, I, I], "scan_forward": [P] * 7, "scan_forward_train": [P] * 7,
        "scan_backward": [P] * 9, "scan_step": [I, I, I] + [P] * 5, "scan_query": [P, I, PLL],
        "scan_destroy": [P], "check_scan_args": [I] * 4 + [P] * 9,
        "embed_create": [PP, I, I, I, I, I], "embed_forward": [P, P, P, P, F, P, P],
        "embed_backward": [P, P, P, P, I, F, P, P], "embed_query": [P, I, PLL], "embed_destroy": [P],
        "check_embed_args": [I] * 5 + [P] * 5 + [I, P],
        "adamw_create": [PP, P, I, I], "adamw_step": [P, P, I, DB, DB, DB, DB, DB, LL, P],
        "adamw_states": [P, P, P, P], "adamw_query": [P, I, PLL], "adamw_destroy": [P],
        "check_adamw_args": [P, I, I, P, I],
        "beam_create": [PP, I, I, I, I], "beam_step": [P, P, P, P, I, P, P, P, P, P, I, P],
        "beam_query": [P, I, PLL], "beam_destroy": [P],
        "check_beam_args": [I] * 4 + [P] * 8 + [I],
    }.items():
        f = getattr(lib, "lstm_dyn_" + name)
        f.argtypes, f.restype = args, I
    _ready = lib
    return lib


# --- C ABI mirrors ----------------------------------------------------------

def _call(name, *args):
    rc = getattr(_ready or _lib(), name)(*args)
    if rc != OK:
        raise LstmDynError(rc, name)


def _ok(rc, name):
    """For the wrappers below, whose calls are few microseconds: the function is called directly."""
    if rc != OK:
        raise LstmDynError(rc, name)


def _create(name, *args) -> int:
    h = ctypes.c_void_p()
    _call(name, ctypes.byref(h), *args)
    return h.value


def _query(name, handle, what) -> int:
    v = ctypes.c_longlong(0)
    _call(name, handle, what, ctypes.byref(v))
    return int(v.value)


def lstm_dyn_scan_create(B: int, H: int, T_max: int, dtype: int) -> int:
    return _create("lstm_dyn_scan_create", B, H, T_max, dtype)


def lstm_dyn_scan_forward(handle, z, lengths, h0, out_h, out_y, stream=0) -> None:
    _call("lstm_dyn_scan_forward", handle, z, lengths, h0, out_h, out_y, stream)


def lstm_dyn_scan_forward_train(handle, z, lengths, h0, out_h, out_y, stream=0) -> None:
    _call("lstm_dyn_scan_forward_train", handle, z, lengths, h0, out_h, out_y, stream)


def lstm_dyn_scan_backward(handle, z, lengths, h0, dy, d_out_h, dz, dh0, stream=0) -> None:
    _call("lstm_dyn_scan_backward", handle, z, lengths, h0, dy, d_out_h, dz, dh0, stream)


def lstm_dyn_scan_step(rows, H, dtype, z, h, out_h, out_y, stream=0) -> None:
    _call("lstm_dyn_scan_step", rows, H, dtype, z, h, out_h, out_y, stream)


def lstm_dyn_scan_query(handle, what) -> int:
    return _query("lstm_dyn_scan_query", handle, what)


def lstm_dyn_scan_destroy(handle) -> None:
    _call("lstm_dyn_scan_destroy", handle)


def lstm_dyn_check_scan_args(*args) -> int:
    return _lib().lstm_dyn_check_scan_args(*args)


def lstm_dyn_embed_create(B: int, T_max: int, V: int, D: int, dtype: int) -> int:
    return _create("lstm_dyn_embed_create", B, T_max, V, D, dtype)


def lstm_dyn_embed_forward(handle, tokens, lengths, table, scale, out_x, stream=0) -> None:
    _call("lstm_dyn_embed_forward", handle, tokens, lengths, table, scale, out_x, stream)


def lstm_dyn_embed_backward(handle, tokens, lengths, dx, dx_dtype, scale, d_table, stream=0) -> None:
    _call("lstm_dyn_embed_backward", handle, tokens, lengths, dx, dx_dtype, scale, d_table, stream)


def lstm_dyn_embed_query(handle, what) -> int:
    return _query("lstm_dyn_embed_query", handle, what)


def lstm_dyn_embed_destroy(handle) -> None:
    _call("lstm_dyn_embed_destroy", handle)


def lstm_dyn_check_embed_args(*args) -> int:
    return _lib().lstm_dyn_check_embed_args(*args)


def lstm_dyn_adamw_create(tensors, state_bits: int) -> int:
    """tensors: a sequence of AdamwTensor."""
    array = (AdamwTensor * len(tensors))(*tensors)
    return _create("lstm_dyn_adamw_create", array, len(tensors), state_bits)


def lstm_dyn_adamw_step(handle, grads, grad_dtype, lr, beta1, beta2, eps, grad_scale, step, stream=0) -> None:
    """grads: a ctypes array of pointers."""
    _call("lstm_dyn_adamw_step", handle, grads, grad_dtype, lr, beta1, beta2, eps, grad_scale, step, stream)


def lstm_dyn_adamw_states(handle, out_m, out_v, stream=0) -> None:
    _call("lstm_dyn_adamw_states", handle, out_m, out_v, stream)


def lstm_dyn_adamw_query(handle, what) -> int:
    return _query("lstm_dyn_adamw_query", handle, what)


def lstm_dyn_adamw_destroy(handle) -> None:
    _call("lstm_dyn_adamw_destroy", handle)


def lstm_dyn_check_adamw_args(tensors, state_bits, grads=None, grad_dtype=F32) -> int:
    array = (AdamwTensor * len(tensors))(*tensors)
    g = None if grads is None else (ctypes.c_void_p * len(grads))(*grads)
    return _lib().lstm_dyn_check_adamw_args(array, len(tensors), state_bits, g, grad_dtype)


def lstm_dyn_beam_create(B: int, K: int, V: int, dtype: int) -> int:
    return _create("lstm_dyn_beam_create", B, K, V, dtype)


def lstm_dyn_beam_step(handle, logits, scores, finished, end, out_scores, out_parent, out_token,
                       out_finished, states, n_states, stream=0) -> None:
    """states: a ctypes array of BeamState, or None."""
    _call("lstm_dyn_beam_step", handle, logits, scores, finished, end, out_scores, out_parent,
          out_token, out_finished, states, n_states, stream)


def lstm_dyn_beam_query(handle, what) -> int:
    return _query("lstm_dyn_beam_query", handle, what)


def lstm_dyn_beam_destroy(handle) -> None:
    _call("lstm_dyn_beam_destroy", handle)


def lstm_dyn_check_beam_args(*args) -> int:
    return _lib().lstm_dyn_check_beam_args(*args)


# --- torch convenience wrappers ---------------------------------------------

_torch = None


def _t():
    """torch, imported at the first handle: importing this module does not need it."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _stream(device):
    return _torch.cuda.current_stream(device).cuda_stream


def _dtype(dtype):
    code = _DTYPES[dtype] if isinstance(dtype, str) else int(dtype)
    return code, (_t().bfloat16 if code == BF16 else _t().float32)


class _Handle:
    """What the operators' wrappers share: a handle, of the device that is current where it is made, the
    checks of tensors, its query and its end."""
    _kind = ""
    handle = None

    def _check(self, name, t, dtype, shape):
        try:
            if t.dtype is dtype and t.shape == shape and t.get_device() == self._device and t.is_contiguous():
                return
        except AttributeError:
            pass
        if not isinstance(t, _t().Tensor) or not t.is_cuda:
            raise TypeError(f"{name} must be a device tensor")
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
        if t.get_device() != self._device:
            raise ValueError(f"{name} must be on the handle's device {self._device}, got {t.get_device()}")
        raise ValueError(f"{name} must be contiguous")

    def query(self, what: int) -> int:
        return _query(f"lstm_dyn_{self._kind}_query", self.handle, what)

    def status(self) -> int:
        """The device status of the calls since the last such query (waits for them)."""
        return self.query(OPS_Q_STATUS)

    def close(self):
        if self.handle:
            handle, self.handle = self.handle, None
            _call(f"lstm_dyn_{self._kind}_destroy", handle)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


class GatedScan(_Handle):
    """The recurrence a = sigmoid(f), h_t = a h_{t-1} + (1 - a) v, y_t = sigmoid(o) h_t over
    z [B, T_max, 3H] = (f, v, o) in the handle's dtype, with lengths int32 [B]
    and h0 float32 [B, H]; y is in the handle's dtype, the state float32."""
    _kind = "scan"

    def __init__(self, B: int, H: int, T_max: int, dtype="bf16"):
        self.B, self.H, self.T = B, H, T_max
        self.dtype, self._et = _dtype(dtype)
        self._device = _torch.cuda.current_device()
        self.handle = lstm_dyn_scan_create(B, H, T_max, self.dtype)

    def _forward(self, call, z, lengths, h0, out_h, out_y, stream):
        if stream is not None:
            with _on(stream):
                return self._forward(call, z, lengths, h0, out_h, out_y, None)
        torch = _torch
        B, T, H = self.B, self.T, self.H
        self._check("z", z, self._et, (B, T, 3 * H))
        self._check("lengths", lengths, torch.int32, (B,))
        self._check("h0", h0, torch.float32, (B, H))
        if out_h is None:
            out_h = torch.empty_like(h0)
        else:
            self._check("out_h", out_h, torch.float32, (B, H))
        if out_y is None:
            out_y = torch.empty((B, T, H), dtype=self._et, device=z.device)
        else:
            self._check("out_y", out_y, self._et, (B, T, H))
        _ok(getattr(_ready, call)(self.handle, z.data_ptr(), lengths.data_ptr(), h0.data_ptr(), out_h.data_ptr(),
                                  out_y.data_ptr(), _stream(z.device)), call)
        return out_y, out_h

    def forward(self, z, lengths, h0, out_h=None, out_y=None, stream=None):
        """Returns (y [B, T_max, H], zero past each length, and the state after each row's last step)."""
        return self._forward("lstm_dyn_scan_forward", z, lengths, h0, out_h, out_y, stream)

    __call__ = forward

    def forward_train(self, z, lengths, h0, out_h=None, out_y=None, stream=None):
        """``forward`` that also keeps what ``backward`` needs."""
        return self._forward("lstm_dyn_scan_forward_train", z, lengths, h0, out_h, out_y, stream)

    def backward(self, z, lengths, h0, dy, d_out_h=None, stream=None, out=None):
        """Gradients after ``forward_train`` with the same z, lengths and h0: a dict of dz
        [B, T_max, 3H] (the handle's dtype) and dh0 float32 [B, H].  dy in the
        handle's dtype; d_out_h float32 [B, H] or None.  out: a dict with those
        keys holding caller-owned tensors."""
        if stream is not None:
            with _on(stream):
                return self.backward(z, lengths, h0, dy, d_out_h, None, out)
        torch = _torch
        B, T, H = self.B, self.T, self.H
        self._check("z", z, self._et, (B, T, 3 * H))
        self._check("lengths", lengths, torch.int32, (B,))
        self._check("h0", h0, torch.float32, (B, H))
        self._check("dy", dy, self._et, (B, T, H))
        if d_out_h is not None:
            self._check("d_out_h", d_out_h, torch.float32, (B, H))
        if out is None:
            out = {"dz": torch.empty_like(z), "dh0": torch.empty_like(h0)}
        else:
            if sorted(out) != ["dh0", "dz"]:
                raise ValueError("out must hold exactly ['dh0', 'dz']")
            self._check("dz", out["dz"], self._et, (B, T, 3 * H))
            self._check("dh0", out["dh0"], torch.float32, (B, H))
        _ok(_ready.lstm_dyn_scan_backward(self.handle, z.data_ptr(), lengths.data_ptr(), h0.data_ptr(),
                                          dy.data_ptr(), d_out_h.data_ptr() if d_out_h is not None else 0,
                                          out["dz"].data_ptr(), out["dh0"].data_ptr(), _stream(z.device)),
            "lstm_dyn_scan_backward")
        return out

    def step(self, z, h, out_h=None, out_y=None, stream=None):
        """One step of any number of rows: z [R, 3H], h float32 [R, H]; returns (y [R, H], h).
        out_h may be h itself."""
        if stream is not None:
            with _on(stream):
                return self.step(z, h, out_h, out_y)
        torch = _torch
        R, H = h.shape[0], self.H
        self._check("z", z, self._et, (R, 3 * H))
        self._check("h", h, torch.float32, (R, H))
        if out_h is None:
            out_h = torch.empty_like(h)
        else:
            self._check("out_h", out_h, torch.float32, (R, H))
        if out_y is None:
            out_y = torch.empty_like(h, dtype=self._et)
        else:
            self._check("out_y", out_y, self._et, (R, H))
        _ok(_ready.lstm_dyn_scan_step(R, H, self.dtype, z.data_ptr(), h.data_ptr(), out_h.data_ptr(),
                                      out_y.data_ptr(), _stream(z.device)), "lstm_dyn_scan_step")
        return out_y, out_h


class TokenEmbed(_Handle):
    """x [B, T_max, D] = scale * table[tokens] for the loop, zero past each length, and the gradient
    of the table.  tokens int32 [B, T_max], lengths int32 [B] or None (all T_max),
    table [V, D] in the handle's dtype.  A token outside [0, V) gives a zero row
    and no gradient, and shows in ``status()``."""
    _kind = "embed"

    def __init__(self, B: int, T_max: int, V: int, D: int, dtype="bf16", scale: float = 1.0):
        self.B, self.T, self.V, self.D, self.scale = B, T_max, V, D, float(scale)
        self.dtype, self._et = _dtype(dtype)
        self._device = _torch.cuda.current_device()
        self.handle = lstm_dyn_embed_create(B, T_max, V, D, self.dtype)

    def _tokens(self, tokens, lengths):
        torch = _torch
        self._check("tokens", tokens, torch.int32, (self.B, self.T))
        if lengths is None:
            return 0
        self._check("lengths", lengths, torch.int32, (self.B,))
        return lengths.data_ptr()

    def forward(self, tokens, lengths, table, out_x=None, stream=None):
        if stream is not None:
            with _on(stream):
                return self.forward(tokens, lengths, table, out_x)
        torch = _torch
        L = self._tokens(tokens, lengths)
        self._check("table", table, self._et, (self.V, self.D))
        if out_x is None:
            out_x = torch.empty((self.B, self.T, self.D), dtype=self._et, device=table.device)
        else:
            self._check("out_x", out_x, self._et, (self.B, self.T, self.D))
        _ok(_ready.lstm_dyn_embed_forward(self.handle, tokens.data_ptr(), L, table.data_ptr(), self.scale,
                                          out_x.data_ptr(), _stream(table.device)), "lstm_dyn_embed_forward")
        return out_x

    __call__ = forward

    def backward(self, tokens, lengths, dx, out=None, stream=None):
        """d_table float32 [V, D] (rows of tokens that do not occur are zero) from dx [B, T_max, D],
        float32 (as ``LstmDyn.backward`` gives it) or bfloat16."""
        if stream is not None:
            with _on(stream):
                return self.backward(tokens, lengths, dx, out)
        torch = _torch
        L = self._tokens(tokens, lengths)
        code = BF16 if isinstance(dx, torch.Tensor) and dx.dtype == torch.bfloat16 else F32
        self._check("dx", dx, torch.bfloat16 if code == BF16 else torch.float32, (self.B, self.T, self.D))
        if out is None:
            out = torch.empty((self.V, self.D), dtype=torch.float32, device=dx.device)
        else:
            self._check("out", out, torch.float32, (self.V, self.D))
        _ok(_ready.lstm_dyn_embed_backward(self.handle, tokens.data_ptr(), L, dx.data_ptr(), code, self.scale,
                                           out.data_ptr(), _stream(dx.device)), "lstm_dyn_embed_backward")
        return out


class AdamW(_Handle):
    """AdamW over a list of float32 tensors, updated in place by one launch for up to 256 of them.

    copies: a list of bfloat16 tensors (or None) that receive the parameters
    rounded, for a model that computes in bf16.  state_bits 32: ``m``, ``v`` float32.
    state_bits 8: ``m`` and ``v`` hold e4m3 codes of m and of sqrt(v), ``m_exp`` and
    ``v_exp`` one exponent byte per 256 elements.  weight_decay: one number, or one per
    tensor.  The handle keeps the tensors' addresses, so they stay where they are."""
    _kind = "adamw"

    def __init__(self, params, copies=None, state_bits: int = 32, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.01, steps_done: int = 0):
        torch = _t()
        self.params = list(params)
        self.copies = list(copies) if copies is not None else [None] * len(self.params)
        if not self.params or len(self.copies) != len(self.params):
            raise ValueError("params must not be empty, and copies be as many")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.bits, self.betas, self.eps, self.steps_done = state_bits, betas, eps, int(steps_done)
        self._device = torch.cuda.current_device()
        wd = [float(weight_decay)] * len(self.params) if isinstance(weight_decay, (int, float)) else list(weight_decay)
        if len(wd) != len(self.params):
            raise ValueError("weight_decay must be one number or one per tensor")
        self.m, self.v, self.m_exp, self.v_exp, rows = [], [], [], [], []
        for i, (p, c) in enumerate(zip(self.params, self.copies)):
            self._check(f"params[{i}]", p, torch.float32, p.shape)
            if c is not None:
                self._check(f"copies[{i}]", c, torch.bfloat16, p.shape)
            n, dev = p.numel(), p.device
            if state_bits == 32:
                self.m.append(torch.zeros(p.shape, dtype=torch.float32, device=dev))
                self.v.append(torch.zeros(p.shape, dtype=torch.float32, device=dev))
            else:
                for codes, exps in ((self.m, self.m_exp), (self.v, self.v_exp)):
                    codes.append(torch.zeros(n, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn))
                    # zero codes: 2^-100, the exponent of a block of zeros
                    exps.append(torch.full(((n + STATE_BLOCK - 1) // STATE_BLOCK,), 27, dtype=torch.uint8, device=dev))
            ptr = lambda t: t.data_ptr() if t is not None and t.numel() else 0
            rows.append(AdamwTensor(ptr(p), ptr(c), ptr(self.m[i]), ptr(self.v[i]),
                                    ptr(self.m_exp[i]) if state_bits == 8 else 0,
                                    ptr(self.v_exp[i]) if state_bits == 8 else 0, n, wd[i]))
        self.handle = lstm_dyn_adamw_create(rows, state_bits)
        self._pointers = ctypes.c_void_p * len(self.params)

    def load_state(self, m, v, m_exp=None, v_exp=None):
        """Copy states kept before (in the layout of the attributes) into this optimizer, on the current stream."""
        for mine, given in ((self.m, m), (self.v, v), (self.m_exp, m_exp or []), (self.v_exp, v_exp or [])):
            if len(mine) != len(given):
                raise ValueError("the states of every tensor are needed")
            for a, b in zip(mine, given):
                if a.shape != b.shape or a.dtype != b.dtype:
                    raise ValueError(f"a state must be {a.dtype} {tuple(a.shape)}, got {b.dtype} {tuple(b.shape)}")
                a.copy_(b)

    def step(self, grads, lr: float, grad_scale: float = 1.0, stream=None):
        """One step from the gradients (all float32 or all bfloat16, in the parameters' shapes), each
        times grad_scale.  The step's number is a value of the call: a captured call repeats it."""
        if stream is not None:
            with _on(stream):
                return self.step(grads, lr, grad_scale)
        torch = _torch
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError(f"{len(self.params)} gradients are needed, got {len(grads)}")
        et = grads[0].dtype if isinstance(grads[0], torch.Tensor) else None
        if et not in (torch.float32, torch.bfloat16):
            raise TypeError("gradients must be float32 or bfloat16 device tensors")
        for g, p in zip(grads, self.params):
            self._check("a gradient", g, et, p.shape)
        _ok(_ready.lstm_dyn_adamw_step(self.handle, self._pointers(*[g.data_ptr() for g in grads]),
                                       BF16 if et == torch.bfloat16 else F32, lr, self.betas[0], self.betas[1],
                                       self.eps, grad_scale, self.steps_done + 1, _stream(grads[0].device)),
            "lstm_dyn_adamw_step")
        self.steps_done += 1

    def states(self, stream=None):
        """What the states stand for, two lists in the parameters' shapes: (m, v), the float32 tensors
        themselves; or with 8 bits (m, sqrt(v)) as bfloat16, which holds their values exactly."""
        if self.bits == 32:
            return self.m, self.v
        if stream is not None:
            with _on(stream):
                return self.states()
        torch = _torch
        m = [torch.empty(p.shape, dtype=torch.bfloat16, device=p.device) for p in self.params]
        v = [torch.empty_like(x) for x in m]
        lstm_dyn_adamw_states(self.handle, self._pointers(*[x.data_ptr() for x in m]),
                              self._pointers(*[x.data_ptr() for x in v]),
                              _stream(self.params[0].device))
        return m, v


class BeamSearch(_Handle):
    """One step of a beam search over B sequences with K beams (at most 32) and a vocabulary of V.
    end: the token that finishes a beam, or None."""
    _kind = "beam"

    def __init__(self, B: int, K: int, V: int, dtype="bf16", end=None):
        self.B, self.K, self.V, self.end = B, K, V, -1 if end is None else int(end)
        self.dtype, self._et = _dtype(dtype)
        self._device = _torch.cuda.current_device()
        self.handle = lstm_dyn_beam_create(B, K, V, self.dtype)
        self._rows = (BeamState * BEAM_MAX_STATES)()

    def step(self, logits, scores, finished, states=(), out_states=None, stream=None):
        """The K best of scores[b, k] + log_softmax(logits[b, k])[j] for every b (a finished beam goes
        on only as itself), and the states' rows in their order.

        logits [B, K, V] in the handle's dtype, scores float32 [B, K], finished
        uint8 [B, K], states: tensors [B, K, ...] of any type (at most 8).  Returns
        (scores, parent int32, token int32, finished, states), all new, the states
        in out_states if given."""
        if stream is not None:
            with _on(stream):
                return self.step(logits, scores, finished, states, out_states)
        torch = _torch
        B, K = self.B, self.K
        self._check("logits", logits, self._et, (B, K, self.V))
        self._check("scores", scores, torch.float32, (B, K))
        self._check("finished", finished, torch.uint8, (B, K))
        if len(states) > BEAM_MAX_STATES:
            raise ValueError(f"at most {BEAM_MAX_STATES} states, got {len(states)}")
        if out_states is None:
            out_states = [torch.empty_like(s) for s in states]
        elif len(out_states) != len(states):
            raise ValueError("out_states must be as many as states")
        rows = self._rows      # read before the call returns
        for i, (s, d) in enumerate(zip(states, out_states)):
            shape = s.shape
            self._check("a state", s, s.dtype, shape)
            self._check("a state's output", d, s.dtype, shape)
            if shape[:2] != (B, K):
                raise ValueError(f"states[{i}] must have shape ({B}, {K}, ...), got {tuple(shape)}")
            row = rows[i]
            row.src, row.dst, row.row_bytes = s.data_ptr(), d.data_ptr(), s.nbytes // (B * K)
        out_scores, done = torch.empty_like(scores), torch.empty_like(finished)
        parent, token = torch.empty_like(scores, dtype=torch.int32), torch.empty_like(scores, dtype=torch.int32)
        _ok(_ready.lstm_dyn_beam_step(self.handle, logits.data_ptr(), scores.data_ptr(), finished.data_ptr(),
                                      self.end, out_scores.data_ptr(), parent.data_ptr(), token.data_ptr(),
                                      done.data_ptr(), self._rows, len(states), _stream(logits.device)),
            "lstm_dyn_beam_step")
        return out_scores, parent, token, done, out_states
