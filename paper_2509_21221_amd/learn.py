"""Python binding of the C ABI in include/gwtf_learn.h (ctypes; argument
marshalling only -- the operators run in the HIP library).

The functions carry the C names (``gwtf_learn_create``, ``gwtf_learn_sample``,
``gwtf_learn_list_create``, ``gwtf_learn_list_destroy``,
``gwtf_learn_grad_norm``, ``gwtf_learn_adamw``, ``gwtf_learn_destroy``,
``gwtf_learn_last_error``); ``LearnOps`` wraps them for torch device tensors.
PyTorch only provides device memory and the HIP stream.

There is no fallback: if ``libgwtf_mcf.so`` is missing or cannot be loaded,
every entry point raises.
"""
from __future__ import annotations

import ctypes
import math

from .mcf import GwtfError, load_library
from .stage import GWTF_TYPE_BF16, GWTF_TYPE_F16, GWTF_TYPE_F32

GWTF_UNIFORM_F32 = 0
GWTF_UNIFORM_F64 = 1
GWTF_STATE_F32 = 0
GWTF_STATE_F8 = 1
GWTF_STATE_NONE = 2
GWTF_STATE_BLOCK = 128

_i32, _i64, _u32, _u64, _vp, _f32, _f64 = (ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64,
                                           ctypes.c_void_p, ctypes.c_float, ctypes.c_double)


class gwtf_learn_sample_t(ctypes.Structure):
    _fields_ = [("num_tokens", _i64), ("vocab", _i64), ("type", _i32), ("uniform_type", _i32), ("top_k", _i32),
                ("temperature", _f64), ("top_p", _f64), ("min_p", _f64), ("temperatures", _vp), ("top_ks", _vp),
                ("top_ps", _vp), ("min_ps", _vp), ("logits", _vp), ("logits_stride", _i64), ("u", _vp), ("ids", _vp),
                ("logp", _vp), ("kept", _vp)]


class gwtf_learn_tensor_t(ctypes.Structure):
    _fields_ = [("size", _i64), ("type", _i32), ("grad_type", _i32), ("grad", _vp), ("param", _vp), ("master", _vp),
                ("m", _vp), ("v", _vp), ("m_scale", _vp), ("v_scale", _vp), ("weight_decay", _f32), ("site", _u32)]


class gwtf_learn_grad_norm_t(ctypes.Structure):
    _fields_ = [("list", _vp), ("max_norm", _f64), ("scale", _f64), ("norm", _vp), ("factor", _vp)]


class gwtf_learn_adamw_t(ctypes.Structure):
    _fields_ = [("list", _vp), ("step", _i64), ("step_at", _vp), ("lr", _f64), ("lr_at", _vp), ("beta1", _f64),
                ("beta2", _f64), ("eps", _f64), ("seed", _u64), ("factor", _vp)]


_CALLS = {"sample": gwtf_learn_sample_t, "grad_norm": gwtf_learn_grad_norm_t, "adamw": gwtf_learn_adamw_t}

_lib = None


def _library():
    """libgwtf_mcf.so with the prototypes of this header."""
    global _lib
    if _lib is None:
        lib = load_library()
        lib.gwtf_learn_create.argtypes = [_i32, _vp, ctypes.POINTER(_vp)]
        lib.gwtf_learn_create.restype = ctypes.c_int
        lib.gwtf_learn_destroy.argtypes = [_vp]
        lib.gwtf_learn_destroy.restype = None
        lib.gwtf_learn_last_error.argtypes = [_vp]
        lib.gwtf_learn_last_error.restype = ctypes.c_char_p
        lib.gwtf_learn_list_create.argtypes = [_vp, _i64, ctypes.POINTER(gwtf_learn_tensor_t), _i32, ctypes.POINTER(_vp)]
        lib.gwtf_learn_list_create.restype = ctypes.c_int
        lib.gwtf_learn_list_destroy.argtypes = [_vp]
        lib.gwtf_learn_list_destroy.restype = None
        for name, args in _CALLS.items():
            fn = getattr(lib, "gwtf_learn_" + name)
            fn.argtypes = [_vp, ctypes.POINTER(args)]
            fn.restype = ctypes.c_int
        _lib = lib
    return _lib


def gwtf_learn_last_error(handle=None) -> str:
    return _library().gwtf_learn_last_error(handle).decode()


def _check(code, handle=None):
    if code:
        raise GwtfError(code, gwtf_learn_last_error(handle))


def gwtf_learn_create(device: int = 0, hip_stream: int = 0):
    """Create a handle; returns an opaque pointer."""
    out = _vp()
    _check(_library().gwtf_learn_create(device, hip_stream, ctypes.byref(out)))
    return out


def gwtf_learn_destroy(handle) -> None:
    _library().gwtf_learn_destroy(handle)


def gwtf_learn_list_create(handle, tensors, form: int):
    """Create a list of an array of gwtf_learn_tensor_t; returns an opaque pointer."""
    out = _vp()
    _check(_library().gwtf_learn_list_create(handle, len(tensors), tensors, form, ctypes.byref(out)), handle)
    return out


def gwtf_learn_list_destroy(list_) -> None:
    _library().gwtf_learn_list_destroy(list_)


def gwtf_learn_sample(handle, args: gwtf_learn_sample_t) -> None:
    _check(_library().gwtf_learn_sample(handle, args), handle)


def gwtf_learn_grad_norm(handle, args: gwtf_learn_grad_norm_t) -> None:
    _check(_library().gwtf_learn_grad_norm(handle, args), handle)


def gwtf_learn_adamw(handle, args: gwtf_learn_adamw_t) -> None:
    _check(_library().gwtf_learn_adamw(handle, args), handle)


class Parameters:
    """Tensors of a node's parameters as ``LearnOps.parameters`` has checked
    them: ``params``, ``grads``, ``m``, ``v``, ``m_scales``, ``v_scales``,
    ``master`` (lists, or None where there are none).

    The lists hold the memory that the tensors had when they were given, and
    keep it: gradients are written into the same tensors at every step
    (accumulated after ``zero_grad(set_to_none=False)``, or copied; tensors that
    torch makes anew are not seen), and a parameter that is to live elsewhere needs a new list.
    Lists are made, and given up, outside of stream captures.

    A step moves the versions of ``params`` and ``master``, so that a backward pass
    of a graph that has kept the old values is refused, as after any change in place (a
    replayed capture moves none: it is the graph's owner who orders it)."""

    def __init__(self, owner, lists, form, array, versions=()):
        self.list = None
        self.owner = owner
        self.params, self.grads, self.m, self.v, self.m_scales, self.v_scales, self.master = lists
        self.form = form
        self.tensors = [t for one in lists if one for t in one]
        self.versions = versions  # of what a step writes and a graph may have kept, tensors that carry them
        self.list = gwtf_learn_list_create(owner.handle, array, form)

    def __del__(self):
        try:
            if self.list is not None:
                gwtf_learn_list_destroy(self.list)
                self.list = None
        except Exception:
            pass


class LearnOps:
    """Operators that close a training step, for torch device tensors: answers
    drawn from logits (``sample``), the norm of a node's gradients
    (``grad_norm``) and the AdamW step over its parameters (``adamw``).

    A row of logits is one token of any microbatch, as in ``StageOps``.  Results
    stay on the device: ``grad_norm``'s factor is read there by ``adamw``.  New
    tensors are returned unless ``out`` is given; autograd is not involved.  Work
    runs on ``stream`` (by default the current one when the object is made);
    called on another stream, an operator waits for that stream first and that
    stream waits for it; so do the states that ``parameters`` makes.  Calls that
    are captured into a graph need an object made with the capturing stream; step
    number and learning rate can be device tensors there, which a replay reads anew.
    """

    def __init__(self, device: int = 0, stream=None):
        import torch

        self.handle = None
        self.torch = torch
        self.device = device
        self.stream = stream if stream is not None else torch.cuda.current_stream(device)
        self._raw = self.stream.cuda_stream
        self._dev = torch.device("cuda", device)
        self._types = {torch.float32: GWTF_TYPE_F32, torch.float16: GWTF_TYPE_F16, torch.bfloat16: GWTF_TYPE_BF16}
        self._uniforms = {torch.float32: GWTF_UNIFORM_F32, torch.float64: GWTF_UNIFORM_F64}
        self._current = torch._C._cuda_getCurrentRawStream  # the current stream without an object for it
        self._written = torch.autograd.graph.increment_version
        self._f32 = torch.empty(0, dtype=torch.float32, device=self._dev)
        self._i32 = torch.empty(0, dtype=torch.int32, device=self._dev)
        lib = _library()
        self._calls = {name: getattr(lib, "gwtf_learn_" + name) for name in _CALLS}
        self.handle = gwtf_learn_create(device, self._raw)

    # ---- arguments ----

    def _vec(self, t, n, dtype, name):
        if t.dtype is not dtype or t.shape != (n,) or t.get_device() != self.device or not t.is_contiguous():
            raise ValueError(f"{name}: need a contiguous {dtype} tensor of shape ({n},) on cuda:{self.device}, "
                             f"not {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _setting(self, v, n, dtype, name):
        """(number, pointer) of a setting that is a number or a tensor [N]."""
        if isinstance(v, self.torch.Tensor):
            return 0, self._vec(v, n, dtype, name)
        return v, None

    def _one(self, v, dtype, name):
        """(number, pointer) of a number or a device tensor of one."""
        if isinstance(v, self.torch.Tensor):
            if v.dtype is not dtype or v.numel() != 1 or v.get_device() != self.device:
                raise ValueError(f"{name}: need a number or one {dtype} on cuda:{self.device}")
            return 0, v.data_ptr()
        return v, None

    def _given(self, out):
        """Results that the caller gave have been written."""
        self._written([t for t in out if t is not None and not t.is_inference()])

    def _run(self, name, args, tensors, group=None):
        if self.handle is None:
            raise RuntimeError("LearnOps: closed")
        if self._current(self.device) == self._raw:
            code = self._calls[name](self.handle, args)
            if code:
                _check(code, self.handle)
            return
        here = self.torch.cuda.current_stream(self.device)
        self.stream.wait_stream(here)
        _check(self._calls[name](self.handle, args), self.handle)
        here.wait_stream(self.stream)
        for t in (*tensors, *(group.tensors if group is not None else ())):
            if isinstance(t, self.torch.Tensor):
                t.record_stream(self.stream)

    # ---- the data node's last stage ----

    def sample(self, logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None):
        """(ids, logp, kept) of each row: the token drawn with the row's random
        number ``u`` ([N] float32 or float64 within [0, 1)), the logarithm of its
        share of what could have been drawn, and how many tokens could.
        Settings are numbers, or tensors [N] with one for each row (float32;
        ``top_k`` int32); ``top_k`` 0, ``top_p`` 1 and ``min_p`` 0 leave all,
        ``temperature`` 0 the likeliest.  ``out``: the tuple of a former call."""
        if not isinstance(logits, self.torch.Tensor):
            raise TypeError("logits: expected a torch tensor")
        f32, i32 = self.torch.float32, self.torch.int32
        if logits.dim() != 2 or logits.dtype not in self._types or logits.get_device() != self.device:
            raise ValueError(f"logits: need a matrix of float32, float16 or bfloat16 on cuda:{self.device}, "
                             f"not {logits.dtype} {tuple(logits.shape)} on {logits.device}")
        n, v = logits.shape
        stride, across = logits.stride()
        if across != 1 and v != 1:
            raise ValueError(f"logits: columns must be adjacent (strides {logits.stride()})")
        if not isinstance(u, self.torch.Tensor) or u.dtype not in self._uniforms:
            raise ValueError("u: need a float32 or float64 tensor")
        t, ts = self._setting(temperature, n, f32, "temperature")
        k, ks = self._setting(top_k, n, i32, "top_k")
        p, ps = self._setting(top_p, n, f32, "top_p")
        q, qs = self._setting(min_p, n, f32, "min_p")
        if not 0 <= k < 1 << 31:
            raise ValueError("top_k: outside [0, 2^31)")
        given = out is not None
        if not given:
            ids, logp, kept = out = self._i32.new_empty(n), self._f32.new_empty(n), self._i32.new_empty(n)
            to = ids.data_ptr(), logp.data_ptr(), kept.data_ptr()
        else:
            ids, logp, kept = out
            to = (self._vec(ids, n, i32, "ids"), None if logp is None else self._vec(logp, n, f32, "logp"),
                  None if kept is None else self._vec(kept, n, i32, "kept"))
        a = gwtf_learn_sample_t(n, v, self._types[logits.dtype], self._uniforms[u.dtype], k, t, p, q, ts, ks, ps, qs,
                                logits.data_ptr(), stride, self._vec(u, n, u.dtype, "u"), *to)
        self._run("sample", a, (logits, u, temperature, top_k, top_p, min_p, ids, logp, kept))
        if given:
            self._given(out)
        return out

    # ---- update phase ----

    def _list(self, tensors, like, dtypes, name):
        """The tensors as flat views that keep their memory."""
        tensors = list(tensors)
        if like is not None and len(tensors) != len(like):
            raise ValueError(f"{name}: need {len(like)} of them, not {len(tensors)}")
        out = []
        for i, t in enumerate(tensors):
            if not isinstance(t, self.torch.Tensor):
                raise TypeError(f"{name}[{i}]: expected a torch tensor")
            if t.dtype not in dtypes or t.get_device() != self.device or not t.is_contiguous():
                raise ValueError(f"{name}[{i}]: need a contiguous tensor of {' or '.join(map(str, dtypes))} on "
                                 f"cuda:{self.device}, not {t.dtype} {tuple(t.shape)} {t.stride()} on {t.device}")
            if like is not None and t.numel() != like[i].numel():
                raise ValueError(f"{name}[{i}]: need {like[i].numel()} values, not {t.numel()}")
            out.append(t.detach().view(-1))
        return out

    def _apart(self, written, read):
        """No memory that a step writes belongs to two tensors, or to a gradient."""
        spans = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), name, True) for t, name in written if t.numel()]
        spans += [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), "grads", False) for t in read if t.numel()]
        end, by, was = 0, "", False
        for begin, stop, name, writes in sorted(spans):
            if begin < end and (writes or was):
                raise ValueError(f"{name}: a tensor shares memory with one of {by}")
            if stop > end or begin >= end:
                end, by, was = stop, name, writes

    def parameters(self, params, grads, bits: int = 32, moments=None, scales=None, master=None, weight_decay=0.0, sites=None):
        """A node's parameters for ``grad_norm`` and ``adamw`` (``Parameters``).

        ``params``: contiguous tensors of float32, float16 or bfloat16; ``grads``:
        as many of the same sizes, each of the parameter's type or float32.
        States are float32 (``bits`` 32) or 8 bits with float32 scales; ``moments``
        (m, v) and ``scales`` (m's, v's), lists each, continue with those of a former run
        (m of float8_e4m3fn and v of float8_e5m2, and scales, make ``bits`` 8), else they
        are made as zeros.  ``master``: float32 copies that the step works on,
        True to make them.  ``weight_decay``: a number or one for each tensor;
        ``sites``: numbers of the tensors for 8-bit rounding, their places in the list by
        default.  With ``params`` None the list is for ``grad_norm`` alone."""
        if self.handle is None:
            raise RuntimeError("LearnOps: closed")
        # states are made, and copies taken, in the order of the object's stream: after its pending steps and before the next
        here = self.torch.cuda.current_stream(self.device)
        if here.cuda_stream == self._raw:
            return self._parameters(params, grads, bits, moments, scales, master, weight_decay, sites)
        self.stream.wait_stream(here)
        with self.torch.cuda.stream(self.stream):
            made = self._parameters(params, grads, bits, moments, scales, master, weight_decay, sites)
        here.wait_stream(self.stream)
        return made

    def _parameters(self, params, grads, bits, moments, scales, master, weight_decay, sites):
        torch, types = self.torch, tuple(self._types)
        f32 = torch.float32
        if params is None:
            grads = self._list(grads, None, types, "grads")
            array = (gwtf_learn_tensor_t * len(grads))()
            for a, g in zip(array, grads):
                a.size, a.grad_type, a.grad = g.numel(), self._types[g.dtype], g.data_ptr()
            return Parameters(self, (None, grads, None, None, None, None, None), GWTF_STATE_NONE, array)
        if bits not in (8, 32):
            raise ValueError("bits: 8 or 32")
        given = list(params)
        params = self._list(given, None, types, "params")
        grads = self._list(grads, params, types, "grads")
        for i, (p, g) in enumerate(zip(params, grads)):
            if g.dtype not in (p.dtype, f32):
                raise ValueError(f"grads[{i}]: need {p.dtype} or float32, not {g.dtype}")
        if scales is not None:
            bits = 8
            if moments is None:
                raise ValueError("scales need moments")
        kinds = (torch.float8_e4m3fn, torch.float8_e5m2) if bits == 8 else (f32, f32)
        if moments is None:
            moments = [[torch.zeros(p.shape, dtype=torch.uint8 if bits == 8 else f32, device=self._dev) for p in params]
                       for _ in kinds]
            if bits == 8:
                moments = [[t.view(kind) for t in one] for one, kind in zip(moments, kinds)]
        elif bits == 8 and scales is None:
            raise ValueError("moments in 8 bits need scales")
        m, v = (self._list(one, params, (kind,), name) for one, kind, name in zip(moments, kinds, ("m", "v")))
        ms = vs = None
        if bits == 8:
            blocks = [torch.empty(-(-p.numel() // GWTF_STATE_BLOCK), device="meta") for p in params]
            if scales is None:
                scales = [[torch.ones(b.shape, dtype=f32, device=self._dev) for b in blocks] for _ in kinds]
            ms, vs = (self._list(one, blocks, (f32,), name) for one, name in zip(scales, ("m_scale", "v_scale")))
        if master is True:
            master = [p.to(f32, copy=True) for p in params]
            given += master
        elif master is not None and master is not False:
            copies = list(master)
            master = self._list(copies, params, (f32,), "master")
            given += copies
        else:
            master = None
        # of what a step writes; views of one tensor share its version
        versions = {id(t if t._base is None else t._base): w for t, w in zip(given, [*params, *(master or ())])}
        n = len(params)
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        sites = list(range(n)) if sites is None else list(sites)
        if len(decay) != n or len(sites) != n:
            raise ValueError(f"weight_decay, sites: need {n} of them")
        if any(not 0 <= s < 1 << 32 for s in sites):
            raise ValueError("sites must fit in 32 bits and be >= 0")
        self._apart([(t, name) for one, name in ((params, "params"), (m, "m"), (v, "v"), (ms, "m_scale"), (vs, "v_scale"),
                                                 (master, "master")) if one for t in one], grads)
        array = (gwtf_learn_tensor_t * n)()
        for i, a in enumerate(array):
            p = params[i]
            a.size, a.type, a.grad_type = p.numel(), self._types[p.dtype], self._types[grads[i].dtype]
            a.grad, a.param, a.m, a.v = grads[i].data_ptr(), p.data_ptr(), m[i].data_ptr(), v[i].data_ptr()
            a.master = None if master is None else master[i].data_ptr()
            if bits == 8:
                a.m_scale, a.v_scale = ms[i].data_ptr(), vs[i].data_ptr()
            a.weight_decay, a.site = decay[i], sites[i]
        return Parameters(self, (params, grads, m, v, ms, vs, master), GWTF_STATE_F8 if bits == 8 else GWTF_STATE_F32, array,
                          tuple(t for t in versions.values() if not t.is_inference()))

    def _group(self, group):
        if self.handle is None:
            raise RuntimeError("LearnOps: closed")
        if not isinstance(group, Parameters) or group.owner is not self:
            raise ValueError("need the Parameters of this object's parameters()")
        return group.list

    def grad_norm(self, group, max_norm: float = math.inf, scale: float = 1.0, out=None):
        """(norm, factor), float32 tensors of one: ``scale`` times the norm of
        all gradients of ``group``, and what they are to be multiplied with so
        that it is at most ``max_norm``; NaN where the norm is not finite."""
        given = out is not None
        if not given:
            out = self._f32.new_empty(1), self._f32.new_empty(1)
        norm, factor = out
        f32 = self.torch.float32
        a = gwtf_learn_grad_norm_t(self._group(group), max_norm, scale, None if norm is None else self._vec(norm, 1, f32, "norm"),
                                   None if factor is None else self._vec(factor, 1, f32, "factor"))
        self._run("grad_norm", a, (norm, factor), group)
        if given:
            self._given(out)
        return out

    def adamw(self, group, lr, step, betas=(0.9, 0.999), eps: float = 1e-8, factor=None, seed: int = 0):
        """One AdamW step on all parameters of ``group``, in place.  ``lr`` and
        ``step`` (1 for the first) are numbers or device tensors of one (float32, int64);
        ``factor``: ``grad_norm``'s.  A factor or a device tensor's rate that is not finite, and
        a device tensor's step below 1, leave everything as it was.  ``seed``: of 8-bit states' rounding."""
        table = self._group(group)
        if not 0 <= seed < 1 << 64:
            raise ValueError("seed must fit in 64 bits and be >= 0")
        if factor is not None and not isinstance(factor, self.torch.Tensor):
            raise TypeError("factor: need a device tensor, as grad_norm gives it")
        lr_, lr_at = self._one(lr, self.torch.float32, "lr")
        step_, step_at = self._one(step, self.torch.int64, "step")
        a = gwtf_learn_adamw_t(table, step_, step_at, lr_, lr_at, betas[0], betas[1], eps, seed,
                               None if factor is None else self._one(factor, self.torch.float32, "factor")[1])
        self._run("adamw", a, (lr, step, factor), group)
        self._written(group.versions)

    def close(self):
        if self.handle is not None:
            gwtf_learn_destroy(self.handle)
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
