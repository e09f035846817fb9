"""Python binding of the C ABI in include/gwtf_stage.h (ctypes; argument
marshalling only -- the operators run in the HIP library).

The functions carry the C names (``gwtf_stage_create``, ``gwtf_stage_embed``,
``gwtf_stage_embed_grad``, ``gwtf_stage_dropout``, ``gwtf_stage_norm``,
``gwtf_stage_norm_grad``, ``gwtf_stage_logprob``, ``gwtf_stage_logprob_grad``,
``gwtf_stage_destroy``, ``gwtf_stage_last_error``); ``StageOps`` wraps them for
torch device tensors.  PyTorch only provides device memory and the HIP stream.

There is no fallback: if ``libgwtf_mcf.so`` is missing or cannot be loaded,
every entry point raises.
"""
from __future__ import annotations

import ctypes

from .mcf import GwtfError, load_library

GWTF_TYPE_F32 = 0
GWTF_TYPE_F16 = 1
GWTF_TYPE_BF16 = 2
GWTF_TOKEN_I32 = 0
GWTF_TOKEN_I64 = 1
GWTF_NORM_PLAIN = 0
GWTF_NORM_F8_ROW = 1
GWTF_NORM_F8_BLOCK = 2
GWTF_NORM_BLOCK = 128
GWTF_STAGE_MAX_HIDDEN = 16384
GWTF_STAGE_MAX_TOP = 64

_i32, _i64, _u32, _u64, _vp, _f32, _f64 = (ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64,
                                           ctypes.c_void_p, ctypes.c_float, ctypes.c_double)


class gwtf_stage_shape_t(ctypes.Structure):
    _fields_ = [("max_tokens", _i64), ("max_hidden", _i64), ("max_vocab", _i64), ("device", _i32)]


class gwtf_stage_embed_t(ctypes.Structure):
    _fields_ = [("num_tokens", _i64), ("hidden", _i64), ("vocab", _i64), ("type", _i32), ("token_type", _i32),
                ("scale", _f32), ("tokens", _vp), ("table", _vp), ("table_stride", _i64), ("out", _vp),
                ("out_stride", _i64)]


class gwtf_stage_embed_grad_t(ctypes.Structure):
    _fields_ = [("num_tokens", _i64), ("hidden", _i64), ("vocab", _i64), ("type", _i32), ("grad_type", _i32),
                ("token_type", _i32), ("accumulate", _i32), ("scale", _f32), ("tokens", _vp), ("dout", _vp),
                ("dout_stride", _i64), ("grad", _vp), ("grad_stride", _i64)]


class gwtf_stage_dropout_t(ctypes.Structure):
    _fields_ = [("num_tokens", _i64), ("hidden", _i64), ("type", _i32), ("site", _u32), ("seed", _u64), ("p", _f64),
                ("rows", _vp), ("x", _vp), ("x_stride", _i64), ("residual", _vp), ("residual_stride", _i64),
                ("out", _vp), ("out_stride", _i64)]


class gwtf_stage_norm_t(ctypes.Structure):
    _fields_ = [("num_tokens", _i64), ("hidden", _i64), ("type", _i32), ("form", _i32), ("eps", _f32), ("x", _vp),
                ("x_stride", _i64), ("residual", _vp), ("residual_stride", _i64), ("weight", _vp), ("y", _vp),
                ("y_stride", _i64), ("h_out", _vp), ("h_stride", _i64), ("scales", _vp), ("rstd", _vp)]


class gwtf_stage_norm_grad_t(ctypes.Structure):
    _fields_ = [("num_tokens", _i64), ("hidden", _i64), ("type", _i32), ("dy", _vp), ("dy_stride", _i64), ("h", _vp),
                ("h_stride", _i64), ("dh", _vp), ("dh_stride", _i64), ("weight", _vp), ("rstd", _vp), ("dx", _vp),
                ("dx_stride", _i64), ("dweight", _vp)]


class gwtf_stage_logprob_t(ctypes.Structure):
    _fields_ = [("num_tokens", _i64), ("vocab", _i64), ("type", _i32), ("token_type", _i32), ("top", _i32),
                ("logits", _vp), ("logits_stride", _i64), ("targets", _vp), ("logp", _vp), ("entropy", _vp),
                ("lse", _vp), ("top_logp", _vp), ("top_ids", _vp)]


class gwtf_stage_logprob_grad_t(ctypes.Structure):
    _fields_ = [("num_tokens", _i64), ("vocab", _i64), ("type", _i32), ("token_type", _i32), ("logits", _vp),
                ("logits_stride", _i64), ("targets", _vp), ("lse", _vp), ("entropy", _vp), ("dlogp", _vp),
                ("dentropy", _vp), ("dlogits", _vp), ("dlogits_stride", _i64)]


_CALLS = {"embed": gwtf_stage_embed_t, "embed_grad": gwtf_stage_embed_grad_t, "dropout": gwtf_stage_dropout_t,
          "norm": gwtf_stage_norm_t, "norm_grad": gwtf_stage_norm_grad_t, "logprob": gwtf_stage_logprob_t,
          "logprob_grad": gwtf_stage_logprob_grad_t}

_lib = None


def _library():
    """libgwtf_mcf.so with the prototypes of this header."""
    global _lib
    if _lib is None:
        lib = load_library()
        lib.gwtf_stage_create.argtypes = [ctypes.POINTER(gwtf_stage_shape_t), _vp, ctypes.POINTER(_vp)]
        lib.gwtf_stage_create.restype = ctypes.c_int
        lib.gwtf_stage_destroy.argtypes = [_vp]
        lib.gwtf_stage_destroy.restype = None
        lib.gwtf_stage_last_error.argtypes = [_vp]
        lib.gwtf_stage_last_error.restype = ctypes.c_char_p
        for name, args in _CALLS.items():
            fn = getattr(lib, "gwtf_stage_" + name)
            fn.argtypes = [_vp, ctypes.POINTER(args)]
            fn.restype = ctypes.c_int
        _lib = lib
    return _lib


def gwtf_stage_last_error(handle=None) -> str:
    return _library().gwtf_stage_last_error(handle).decode()


def _check(code, handle=None):
    if code:
        raise GwtfError(code, gwtf_stage_last_error(handle))


def gwtf_stage_create(max_tokens: int, max_hidden: int, max_vocab: int, device: int = 0, hip_stream: int = 0):
    """Create a handle; returns an opaque pointer."""
    shape = gwtf_stage_shape_t(max_tokens, max_hidden, max_vocab, device)
    out = _vp()
    _check(_library().gwtf_stage_create(ctypes.byref(shape), hip_stream, ctypes.byref(out)))
    return out


def gwtf_stage_destroy(handle) -> None:
    _library().gwtf_stage_destroy(handle)


def gwtf_stage_embed(handle, args: gwtf_stage_embed_t) -> None:
    _check(_library().gwtf_stage_embed(handle, args), handle)


def gwtf_stage_embed_grad(handle, args: gwtf_stage_embed_grad_t) -> None:
    _check(_library().gwtf_stage_embed_grad(handle, args), handle)


def gwtf_stage_dropout(handle, args: gwtf_stage_dropout_t) -> None:
    _check(_library().gwtf_stage_dropout(handle, args), handle)


def gwtf_stage_norm(handle, args: gwtf_stage_norm_t) -> None:
    _check(_library().gwtf_stage_norm(handle, args), handle)


def gwtf_stage_norm_grad(handle, args: gwtf_stage_norm_grad_t) -> None:
    _check(_library().gwtf_stage_norm_grad(handle, args), handle)


def gwtf_stage_logprob(handle, args: gwtf_stage_logprob_t) -> None:
    _check(_library().gwtf_stage_logprob(handle, args), handle)


def gwtf_stage_logprob_grad(handle, args: gwtf_stage_logprob_grad_t) -> None:
    _check(_library().gwtf_stage_logprob_grad(handle, args), handle)


class StageOps:
    """Operators on a routed microbatch for torch device tensors: the data
    node's first stage (``embed``, ``embed_grad``), the hand-off between stages
    (``norm``, ``norm_grad``), repeatable ``dropout``, and the data node's last
    stage (``logprob``, ``logprob_grad``).

    A row is one token of any microbatch; matrices are two-dimensional tensors
    of float32, float16 or bfloat16 whose columns are adjacent (rows may be
    any distance apart), index vectors contiguous int32 or int64.  New tensors
    are returned unless ``out`` is given; autograd is not involved, gradients
    are calls of their own.  Work runs on ``stream`` (by default
    the current one when the object is made); called on another stream, an
    operator waits for that stream first and that stream waits for it.  Calls
    that are captured into a graph need an object made with the capturing stream.
    """

    def __init__(self, max_tokens: int, max_hidden: int, max_vocab: int, device: int = 0, stream=None):
        import torch

        self.handle = None
        self.torch = torch
        self.device = device
        self.stream = stream if stream is not None else torch.cuda.current_stream(device)
        self._raw = self.stream.cuda_stream
        self._dev = torch.device("cuda", device)
        self._types = {torch.float32: GWTF_TYPE_F32, torch.float16: GWTF_TYPE_F16, torch.bfloat16: GWTF_TYPE_BF16}
        self._tokens = {torch.int32: GWTF_TOKEN_I32, torch.int64: GWTF_TOKEN_I64}
        self._forms = {"none": GWTF_NORM_PLAIN, "row": GWTF_NORM_F8_ROW, "block": GWTF_NORM_F8_BLOCK}
        self._current = torch._C._cuda_getCurrentRawStream  # the current stream without an object for it
        # a small call is bound by its host work: new tensors come from one at
        # hand (1.2 to 1.4 us each, torch.empty with a device 1.6) and calls go
        # to the library's functions directly
        self._f32 = torch.empty(0, dtype=torch.float32, device=self._dev)
        self._i32 = torch.empty(0, dtype=torch.int32, device=self._dev)
        lib = _library()
        self._calls = {name: getattr(lib, "gwtf_stage_" + name) for name in _CALLS}
        self.handle = gwtf_stage_create(max_tokens, max_hidden, max_vocab, device, self._raw)

    # ---- arguments ----

    def _type(self, t, name):
        if not isinstance(t, self.torch.Tensor):
            raise TypeError(f"{name}: expected a torch tensor")
        if t.dim() != 2 or t.dtype not in self._types:
            raise ValueError(f"{name}: need a matrix of float32, float16 or bfloat16, not {t.dtype} {tuple(t.shape)}")
        return self._types[t.dtype]

    def _mat(self, t, shape, dtype, name):
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self.device:
            raise ValueError(f"{name}: need a {dtype} tensor of shape {tuple(shape)} on cuda:{self.device}, "
                             f"not {t.dtype} {tuple(t.shape)} on {t.device}")
        s = t.stride()
        if s[1] != 1 and shape[1] != 1:
            raise ValueError(f"{name}: columns must be adjacent (strides {s})")
        return t.data_ptr(), s[0]

    def _vec(self, t, n, dtype, name):
        if t.dtype is not dtype or t.shape != (n,) or t.get_device() != self.device or not t.is_contiguous():
            raise ValueError(f"{name}: need a contiguous {dtype} tensor of shape ({n},) on cuda:{self.device}, "
                             f"not {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _ids(self, t, name):
        try:
            kind = self._tokens[t.dtype]
        except KeyError:
            raise ValueError(f"{name}: need int32 or int64, not {t.dtype}") from None
        if t.dim() != 1 or t.get_device() != self.device or not t.is_contiguous():
            raise ValueError(f"{name}: need a contiguous vector on cuda:{self.device}")
        return t.data_ptr(), kind

    def _run(self, name, args, tensors):
        if self.handle is None:
            raise RuntimeError("StageOps: closed")
        if self._current(self.device) == self._raw:
            code = self._calls[name](self.handle, args)
            if code:
                _check(code, self.handle)
            return
        here = self.torch.cuda.current_stream(self.device)
        self.stream.wait_stream(here)
        _check(self._calls[name](self.handle, args), self.handle)
        here.wait_stream(self.stream)
        for t in tensors:
            if t is not None:
                t.record_stream(self.stream)

    # ---- the data node's first stage ----

    def embed(self, tokens, table, scale: float = 1.0, out=None):
        """``scale * table[tokens]`` ([N][H]); zeros for a token outside the table."""
        kind = self._type(table, "table")
        ids, idk = self._ids(tokens, "tokens")
        n, (v, h) = tokens.shape[0], table.shape
        tab = self._mat(table, table.shape, table.dtype, "table")
        if out is None:
            out = table.new_empty((n, h))
            to = out.data_ptr(), h
        else:
            to = self._mat(out, (n, h), table.dtype, "out")
        a = gwtf_stage_embed_t(n, h, v, kind, idk, scale, ids, *tab, *to)
        self._run("embed", a, (tokens, table, out))
        return out

    def embed_grad(self, tokens, dout, vocab: int, scale: float = 1.0, dtype=None, out=None, accumulate: bool = False):
        """Gradient [vocab][H] of the table from the gradient [N][H] of
        ``embed``'s result, in ``dtype`` (dout's or float32).  With
        ``accumulate`` it is added to ``out`` and rows of absent tokens stay."""
        kind = self._type(dout, "dout")
        ids, idk = self._ids(tokens, "tokens")
        n, h = tokens.shape[0], dout.shape[1]
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs an existing out tensor")
            out = dout.new_empty((vocab, h), dtype=dtype)
        elif dtype is not None and out.dtype != dtype:
            raise ValueError(f"out: {out.dtype} is not the dtype asked for, {dtype}")
        a = gwtf_stage_embed_grad_t(n, h, vocab, kind, self._type(out, "out"), idk, bool(accumulate), scale, ids,
                                    *self._mat(dout, (n, h), dout.dtype, "dout"),
                                    *self._mat(out, (vocab, h), out.dtype, "out"))
        self._run("embed_grad", a, (tokens, dout, out))
        return out

    # ---- dropout ----

    def dropout(self, x, p: float, seed: int, site: int, rows=None, residual=None, out=None):
        """``residual + x * keep / (1 - p)`` with the mask of (seed, site,
        identity of the row); ``rows``: int64 identities [N], 0, 1, .. by default.
        The gradient is the same call on the gradient, without residual."""
        torch, kind = self.torch, self._type(x, "x")
        if not 0 <= seed < 1 << 64 or not 0 <= site < 1 << 32:
            raise ValueError("seed must fit in 64 bits and site in 32, both >= 0")
        shape, dt = x.shape, x.dtype
        xs = self._mat(x, shape, dt, "x")
        if out is None:
            out = torch.empty_like(x)
            to = out.data_ptr(), shape[1]
        else:
            to = self._mat(out, shape, dt, "out")
        a = gwtf_stage_dropout_t(shape[0], shape[1], kind, site, seed, p,
                                 None if rows is None else self._vec(rows, shape[0], torch.int64, "rows"), *xs,
                                 *((None, 0) if residual is None else self._mat(residual, shape, dt, "residual")), *to)
        self._run("dropout", a, (x, rows, residual, out))
        return out

    # ---- hand-off ----

    def norm(self, x, weight, eps: float = 1e-5, residual=None, quant: str = "none", out=None):
        """RMS norm of ``h = x + residual``: (y, scales, h, rstd).  ``quant``
        "none" gives y in x's type and scales None; "row" and "block" give
        float8_e4m3fn values and float32 scales [N][1] or [N][ceil(H / 128)] with
        y about values * scales.  h is None without a residual (it is x).
        ``out``: the tuple of a former call of the same shapes, overwritten."""
        torch, kind = self.torch, self._type(x, "x")
        form = self._forms[quant]
        shape, dt = x.shape, x.dtype
        n, h = shape
        groups = (n, 1 if form == GWTF_NORM_F8_ROW else -(-h // GWTF_NORM_BLOCK))
        f32, ydt = torch.float32, torch.float8_e4m3fn if form else dt
        xs = self._mat(x, shape, dt, "x")
        if out is None:
            new = self._f32.new_empty
            y, scales = torch.empty_like(x, dtype=ydt), new(groups) if form else None
            hout, rstd = None if residual is None else torch.empty_like(x), new((n,))
            out = y, scales, hout, rstd
            to = y.data_ptr(), h
            ho = (None, 0) if hout is None else (hout.data_ptr(), h)
            sc, rs = scales.data_ptr() if form else None, rstd.data_ptr()
        else:
            y, scales, hout, rstd = out
            to = self._mat(y, shape, ydt, "y")
            ho = (None, 0) if hout is None else self._mat(hout, shape, dt, "h")
            sc = self._mat(scales, groups, f32, "scales")[0] if form else None
            if form and not scales.is_contiguous():
                raise ValueError("scales: must be contiguous")
            rs = None if rstd is None else self._vec(rstd, n, f32, "rstd")
        a = gwtf_stage_norm_t(n, h, kind, form, eps, *xs,
                              *((None, 0) if residual is None else self._mat(residual, shape, dt, "residual")),
                              self._vec(weight, h, dt, "weight"), *to, *ho, sc, rs)
        self._run("norm", a, (x, residual, weight, y, scales, hout, rstd))
        return out

    def norm_grad(self, dy, h, weight, rstd, dh=None, out=None):
        """(dx, dweight) from the gradient of y, ``h`` and ``rstd`` of the
        forward call and ``dh``, the gradient that reaches h directly.
        dx is the residual's gradient too; dweight is float32."""
        kind = self._type(h, "h")
        shape, dt, f32 = h.shape, h.dtype, self.torch.float32
        hs = self._mat(h, shape, dt, "h")
        if out is None:
            dx, dw = out = self.torch.empty_like(h), self._f32.new_empty((shape[1],))
            to, dwp = (dx.data_ptr(), shape[1]), dw.data_ptr()
        else:
            dx, dw = out
            to = self._mat(dx, shape, dt, "dx")
            dwp = None if dw is None else self._vec(dw, shape[1], f32, "dweight")
        a = gwtf_stage_norm_grad_t(shape[0], shape[1], kind, *self._mat(dy, shape, dt, "dy"), *hs,
                                   *((None, 0) if dh is None else self._mat(dh, shape, dt, "dh")),
                                   self._vec(weight, shape[1], dt, "weight"), self._vec(rstd, shape[0], f32, "rstd"),
                                   *to, dwp)
        self._run("norm_grad", a, (dy, h, dh, weight, rstd, dx, dw))
        return out

    # ---- the data node's last stage ----

    def logprob(self, logits, targets=None, top: int = 0):
        """(logp, entropy, lse, top_logp, top_ids) of each row: the log
        probability of its target (None without targets), its entropy, the
        logarithm of its sum of exponentials, and the ``top`` most likely
        tokens, equal ones by ascending index (None with top == 0)."""
        kind = self._type(logits, "logits")
        shape = logits.shape
        n, v = shape
        if not 0 <= top <= GWTF_STAGE_MAX_TOP:
            raise ValueError(f"top: outside [0, {GWTF_STAGE_MAX_TOP}]")
        ids, idk, logp = None, 0, None
        new = self._f32.new_empty
        if targets is not None:
            ids, idk = self._ids(targets, "targets")
            if targets.shape[0] != n:
                raise ValueError(f"targets: need {n} of them")
            logp = new(n)
        # tensors of their own (5.8 us for five): parts of one (4.8) would share its version and its life
        entropy, lse, top_logp, top_ids = new(n), new(n), None, None
        if top:
            top_logp, top_ids = new(n, top), self._i32.new_empty(n, top)
        a = gwtf_stage_logprob_t(n, v, kind, idk, top, *self._mat(logits, shape, logits.dtype, "logits"), ids,
                                 logp.data_ptr() if logp is not None else None, entropy.data_ptr(), lse.data_ptr(),
                                 top_logp.data_ptr() if top else None, top_ids.data_ptr() if top else None)
        self._run("logprob", a, (logits, targets, logp, entropy, lse, top_logp, top_ids))
        return logp, entropy, lse, top_logp, top_ids

    def logprob_grad(self, logits, targets, lse, entropy=None, dlogp=None, dentropy=None, out=None):
        """Gradient [N][V] of logp and entropy with respect to the logits, from
        ``lse`` (and ``entropy``, where ``dentropy`` is given) of the forward
        call.  ``out`` may be ``logits`` itself."""
        kind = self._type(logits, "logits")
        shape, dt, f32 = logits.shape, logits.dtype, self.torch.float32
        n, v = shape
        ids, idk = None, 0
        if dlogp is not None:
            if targets is None:
                raise ValueError("dlogp needs targets")
            ids, idk = self._ids(targets, "targets")
            if targets.shape[0] != n:
                raise ValueError(f"targets: need {n} of them")
        if dentropy is not None and entropy is None:
            raise ValueError("dentropy needs entropy")
        xs = self._mat(logits, shape, dt, "logits")
        if out is None:
            out = self.torch.empty_like(logits)
            to = out.data_ptr(), v
        else:
            to = self._mat(out, shape, dt, "out")
        a = gwtf_stage_logprob_grad_t(n, v, kind, idk, *xs, ids,
                                      self._vec(lse, n, f32, "lse"),
                                      None if dentropy is None else self._vec(entropy, n, f32, "entropy"),
                                      None if dlogp is None else self._vec(dlogp, n, f32, "dlogp"),
                                      None if dentropy is None else self._vec(dentropy, n, f32, "dentropy"), *to)
        self._run("logprob_grad", a, (logits, targets, lse, entropy, dlogp, dentropy, out))
        return out

    def close(self):
        if self.handle is not None:
            gwtf_stage_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()
