"""Token-mixing operators: the ABI of include/seqmix.h, and a device-side helper for each.

``seqmix_*`` functions mirror the C ABI (device buffers, streams and errors as in ``binding``).
``LinearAttention``, ``TokenConv`` and ``GateNorm``, and for layers with a cache of keys and values ``SoftmaxAttention``,
``Rotary`` and ``CachePages``, own a descriptor, check the tensors that they
are given and launch on torch's current stream.  All arithmetic happens in the HIP library.
They are forward operators: where gradients are recorded, tensors that require one are refused.
"""
from __future__ import annotations

import ctypes

from . import binding as B
from .binding import Conv2dError, _check, _ptr, _stream

SEQMIX_DECAY_NONE, SEQMIX_DECAY_HEAD, SEQMIX_DECAY_TOKEN = 0, 1, 2
SEQMIX_KERNEL_TOKENS, SEQMIX_KERNEL_CHUNKS = 0, 1
SEQMIX_ACT_NONE, SEQMIX_ACT_SILU, SEQMIX_ACT_SIGMOID, SEQMIX_ACT_LINEAR = 0, 1, 2, 3
SEQMIX_NORM_NONE, SEQMIX_NORM_RMS, SEQMIX_NORM_LAYER = 0, 1, 2
SEQMIX_MAX_HEAD_DIM, SEQMIX_MAX_CONV_WIDTH, SEQMIX_MAX_NORM_WIDTH = 256, 8, 16384
SEQMIX_MASK_FULL, SEQMIX_MASK_CAUSAL, SEQMIX_MASK_TREE = 0, 1, 2
SEQMIX_KERNEL_PROMPT, SEQMIX_KERNEL_STEP = 0, 1
SEQMIX_ROTARY_HALF, SEQMIX_ROTARY_INTERLEAVED = 0, 1
SEQMIX_MAX_PAGE = 65536

# every function the header declares
EXPORTS = ("seqmix_attn_desc_create", "seqmix_attn_desc_destroy", "seqmix_attn_plan_query", "seqmix_attn_reserve",
           "seqmix_attn_fwd", "seqmix_conv_desc_create", "seqmix_conv_desc_destroy", "seqmix_conv_fwd",
           "seqmix_norm_desc_create", "seqmix_norm_desc_destroy", "seqmix_norm_fwd",
           "seqmix_softmax_desc_create", "seqmix_softmax_desc_destroy", "seqmix_softmax_plan_query",
           "seqmix_softmax_reserve", "seqmix_softmax_fwd", "seqmix_rotary_desc_create", "seqmix_rotary_desc_destroy",
           "seqmix_rotary_fwd", "seqmix_pages_desc_create", "seqmix_pages_desc_destroy", "seqmix_pages_fwd")


class seqmix_attn_params(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("seqs", ctypes.c_int64), ("slots", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("qk_heads", ctypes.c_int32), ("dk", ctypes.c_int32),
                ("dv", ctypes.c_int32), ("dtype", ctypes.c_int32), ("o_dtype", ctypes.c_int32),
                ("decay", ctypes.c_int32), ("scale", ctypes.c_float)] + [
        (f"{t}_{d}", ctypes.c_int64) for t in "qkvo" for d in ("row", "head")]


class seqmix_attn_plan_info(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("chunk", ctypes.c_int32), ("segment", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_int64)]


class seqmix_conv_params(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("seqs", ctypes.c_int64), ("slots", ctypes.c_int64),
                ("channels", ctypes.c_int64), ("width", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("act", ctypes.c_int32), ("has_bias", ctypes.c_int32), ("x_row", ctypes.c_int64),
                ("y_row", ctypes.c_int64)]


class seqmix_norm_params(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("width", ctypes.c_int64), ("group", ctypes.c_int64),
                ("gate_run", ctypes.c_int64)] + [
        (n, ctypes.c_int32) for n in ("dtype", "res_dtype", "post", "post_bias", "gate", "gate_first", "residual",
                                      "scale_vec", "pre", "pre_bias")] + [
        (n, ctypes.c_float) for n in ("scale", "post_eps", "pre_eps")] + [
        (n, ctypes.c_int64) for n in ("u_row", "gate_row", "res_row", "y_row", "h_row")]


class seqmix_softmax_params(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("tokens", "seqs", "slots", "key_tokens", "pages", "max_pages")] + [
        (n, ctypes.c_int32) for n in ("page", "heads", "kv_heads", "dk", "dv", "dtype", "mask")] + [
        ("scale", ctypes.c_float)] + [(n, ctypes.c_int64) for n in (
            "q_row", "q_head", "o_row", "o_head", "k_row", "k_head", "k_page", "v_row", "v_head", "v_page")]


class seqmix_softmax_plan_info(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("pack", ctypes.c_int32), ("shares", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_int64)]


class seqmix_rotary_params(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("pages", ctypes.c_int64)] + [
        (n, ctypes.c_int32) for n in ("page", "heads", "kv_heads", "dk", "dv", "rot", "layout", "dtype")] + [
        ("amplitude", ctypes.c_float)] + [(f"{t}_{d}", ctypes.c_int64) for t in ("q", "k", "v", "qo", "ko")
                                          for d in ("row", "head")] + [
        (f"{t}_{d}", ctypes.c_int64) for t in ("kc", "vc") for d in ("row", "head", "page")]


class seqmix_pages_params(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("tokens", "seqs", "slots", "pages", "max_pages")] + [
        ("page", ctypes.c_int32)]


_lib = None
_pycall = None


def load():
    """libconv2d.so with the argument types of this ABI set."""
    global _lib
    if _lib is not None:
        return _lib
    lib = B.load()
    vp = ctypes.c_void_p
    for op, params, nptr in (("attn", seqmix_attn_params, 10), ("conv", seqmix_conv_params, 9),
                             ("norm", seqmix_norm_params, 11), ("softmax", seqmix_softmax_params, 11),
                             ("rotary", seqmix_rotary_params, 11), ("pages", seqmix_pages_params, 11)):
        getattr(lib, f"seqmix_{op}_desc_create").argtypes = [ctypes.POINTER(params), ctypes.POINTER(vp)]
        getattr(lib, f"seqmix_{op}_desc_destroy").argtypes = [vp]
        getattr(lib, f"seqmix_{op}_fwd").argtypes = [vp] * (1 + nptr)
    lib.seqmix_attn_plan_query.argtypes = [vp, ctypes.POINTER(seqmix_attn_plan_info)]
    lib.seqmix_attn_reserve.argtypes = [vp]
    lib.seqmix_softmax_plan_query.argtypes = [vp, ctypes.POINTER(seqmix_softmax_plan_info)]
    lib.seqmix_softmax_reserve.argtypes = [vp]
    for name in EXPORTS:
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _create(op, params):
    d = ctypes.c_void_p()
    name = f"seqmix_{op}_desc_create"
    _check(getattr(load(), name)(ctypes.byref(params), ctypes.byref(d)), name)
    return d.value


def seqmix_attn_desc_create(params: seqmix_attn_params) -> int:
    return _create("attn", params)


def seqmix_attn_desc_destroy(desc: int) -> None:
    _check(load().seqmix_attn_desc_destroy(desc), "seqmix_attn_desc_destroy")


def seqmix_attn_plan_query(desc: int) -> seqmix_attn_plan_info:
    out = seqmix_attn_plan_info()
    _check(load().seqmix_attn_plan_query(desc, ctypes.byref(out)), "seqmix_attn_plan_query")
    return out


def seqmix_attn_reserve(desc: int) -> None:
    _check(load().seqmix_attn_reserve(desc), "seqmix_attn_reserve")


def seqmix_attn_fwd(desc: int, q, k, v, decay, offsets, slot_index, state_in, state_out, o, stream=None) -> None:
    _check(load().seqmix_attn_fwd(desc, _ptr(q), _ptr(k), _ptr(v), _ptr(decay), _ptr(offsets), _ptr(slot_index),
                                  _ptr(state_in), _ptr(state_out), _ptr(o), _stream(stream)), "seqmix_attn_fwd")


def seqmix_conv_desc_create(params: seqmix_conv_params) -> int:
    return _create("conv", params)


def seqmix_conv_desc_destroy(desc: int) -> None:
    _check(load().seqmix_conv_desc_destroy(desc), "seqmix_conv_desc_destroy")


def seqmix_conv_fwd(desc: int, x, w, bias, offsets, slot_index, window_in, window_out, y, stream=None) -> None:
    _check(load().seqmix_conv_fwd(desc, _ptr(x), _ptr(w), _ptr(bias), _ptr(offsets), _ptr(slot_index),
                                  _ptr(window_in), _ptr(window_out), _ptr(y), _stream(stream)), "seqmix_conv_fwd")


def seqmix_norm_desc_create(params: seqmix_norm_params) -> int:
    return _create("norm", params)


def seqmix_norm_desc_destroy(desc: int) -> None:
    _check(load().seqmix_norm_desc_destroy(desc), "seqmix_norm_desc_destroy")


def seqmix_norm_fwd(desc: int, u, post_w, post_b, gate, residual, scale_vec, pre_w, pre_b, y, h, stream=None) -> None:
    _check(load().seqmix_norm_fwd(desc, _ptr(u), _ptr(post_w), _ptr(post_b), _ptr(gate), _ptr(residual),
                                  _ptr(scale_vec), _ptr(pre_w), _ptr(pre_b), _ptr(y), _ptr(h), _stream(stream)),
           "seqmix_norm_fwd")


def seqmix_softmax_desc_create(params: seqmix_softmax_params) -> int:
    return _create("softmax", params)


def seqmix_softmax_desc_destroy(desc: int) -> None:
    _check(load().seqmix_softmax_desc_destroy(desc), "seqmix_softmax_desc_destroy")


def seqmix_softmax_plan_query(desc: int) -> seqmix_softmax_plan_info:
    out = seqmix_softmax_plan_info()
    _check(load().seqmix_softmax_plan_query(desc, ctypes.byref(out)), "seqmix_softmax_plan_query")
    return out


def seqmix_softmax_reserve(desc: int) -> None:
    _check(load().seqmix_softmax_reserve(desc), "seqmix_softmax_reserve")


def seqmix_softmax_fwd(desc: int, q, k, v, offsets, key_offsets, slot_index, lens, table, tree, o, stream=None) -> None:
    _check(load().seqmix_softmax_fwd(desc, *(_ptr(t) for t in (q, k, v, offsets, key_offsets, slot_index, lens, table, tree,
                                                               o)), _stream(stream)), "seqmix_softmax_fwd")


def seqmix_rotary_desc_create(params: seqmix_rotary_params) -> int:
    return _create("rotary", params)


def seqmix_rotary_desc_destroy(desc: int) -> None:
    _check(load().seqmix_rotary_desc_destroy(desc), "seqmix_rotary_desc_destroy")


def seqmix_rotary_fwd(desc: int, q, k, v, position, freqs, q_out, k_out, k_cache, v_cache, place, stream=None) -> None:
    _check(load().seqmix_rotary_fwd(desc, *(_ptr(t) for t in (q, k, v, position, freqs, q_out, k_out, k_cache, v_cache,
                                                              place)), _stream(stream)), "seqmix_rotary_fwd")


def seqmix_pages_desc_create(params: seqmix_pages_params) -> int:
    return _create("pages", params)


def seqmix_pages_desc_destroy(desc: int) -> None:
    _check(load().seqmix_pages_desc_destroy(desc), "seqmix_pages_desc_destroy")


def seqmix_pages_fwd(desc: int, kept, offsets, slot_index, lens, table, free_pages, taken, place, position, admitted,
                     stream=None) -> None:
    _check(load().seqmix_pages_fwd(desc, *(_ptr(t) for t in (kept, offsets, slot_index, lens, table, free_pages, taken, place,
                                                             position, admitted)), _stream(stream)), "seqmix_pages_fwd")


_DTYPES = {"f32": B.CONV2D_F32, "bf16": B.CONV2D_BF16}


def _pick(names, value, what):
    try:
        return names[value]
    except KeyError:
        raise ValueError(f"{what} is one of {', '.join(names)}: got {value!r}") from None


class _Operator:
    """A descriptor, and what each tensor argument of a call has to be, in the order of the C call."""

    op = ""

    def __init__(self, params):
        import torch
        self._torch = torch
        self._td = {B.CONV2D_F32: torch.float32, B.CONV2D_BF16: torch.bfloat16}
        self.params = params
        self.desc = _create(self.op, params)
        self._want = []
        self._call = None
        # torch's stream lookup without its Python wrapper (1 us), where this torch has it
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda dev: torch.cuda.current_stream(dev).cuda_stream)

    def _expect(self, name, dtype, shape, strides=None, out=False):
        if strides is None:
            strides, n = [], 1
            for d in reversed(shape):
                strides.insert(0, n)
                n *= d
        self._want.append((dtype, tuple(shape), tuple(strides), name, out))

    def _ready(self):
        """The checks and the C function as one call of the extension module."""
        global _pycall
        if _pycall is None:
            from . import _seqmix as _pycall  # after torch
        fn = ctypes.cast(getattr(load(), f"seqmix_{self.op}_fwd"), ctypes.c_void_p).value
        like = {d: self._torch.empty(0, dtype=d) for d in {w[0] for w in self._want}}
        self._call = _pycall.make(fn, self.desc, [(like[d], shape, strides, out)
                                             for d, shape, strides, _, out in self._want])
        return self._call

    @staticmethod
    def _has_memory(t):
        try:
            return t.numel() == 0 or t.data_ptr() != 0
        except RuntimeError:
            return False

    def _refuse(self, t, want, dev):
        dtype, shape, strides, name, _ = want
        who = f"{type(self).__name__}: {name}"
        if not isinstance(t, self._torch.Tensor):
            raise TypeError(f"{who} is a tensor or None: got {type(t).__name__}")
        if t.layout is not self._torch.strided:
            what = f"is {t.layout}: arguments are dense"
        elif t.dtype is not dtype or t.shape != shape:
            what = f"is {tuple(t.shape)} {t.dtype}, not {shape} {dtype}"
        elif not t.is_cuda or t.get_device() != dev:
            what = f"is on {t.device}: all arguments are on one GPU"
        elif t.is_neg():
            what = "is a negated view (resolve_neg makes it dense)"
        elif any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), strides)):
            what = f"has strides {t.stride()}, not {strides}"
        elif not self._has_memory(t):
            what = "has no memory of its own (a tensor of a torch transform, or a fake one)"
        else:
            what = "requires a gradient, and there is none of a forward operator: call it under torch.no_grad(), or with x.detach()"
        raise Conv2dError(B.CONV2D_E_INVALID, f"{who} {what}")

    def _launch(self, lead, name, stream, *tensors):
        """Checks the tensors (None: not given) and calls the library with their addresses, on the GPU of `lead`."""
        cuda = self._torch.cuda
        try:
            dev = lead.get_device()
        except AttributeError:
            raise TypeError(f"{type(self).__name__}: {name} is a tensor: got {type(lead).__name__}") from None
        call = self._call or self._ready()
        if dev < 0:  # no GPU, no stream: let the checks say which tensor is wrong
            st = _pycall.run(call, dev, 0, *tensors)
        else:
            raw = self._raw_stream(dev) if stream is None else _stream(stream)
            if dev == cuda.current_device():
                st = _pycall.run(call, dev, raw, *tensors)
            else:
                with cuda.device(dev):
                    st = _pycall.run(call, dev, raw, *tensors)
        if st > 0:
            self._refuse(tensors[st - 1], self._want[st - 1], dev)
        if st:
            raise Conv2dError(st, f"seqmix_{self.op}_fwd")

    def close(self):
        if self.desc:
            desc, self.desc, self._call = self.desc, 0, None
            _check(getattr(load(), f"seqmix_{self.op}_desc_destroy")(desc), f"seqmix_{self.op}_desc_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class LinearAttention(_Operator):
    """seqmix_attn of `tokens` rows in `seqs` sequences.

    q, k: [tokens, qk_heads, dk], v, o: [tokens, heads, dv], strides as given (elements between rows and
    between heads) or dense; decay: fp32 [tokens, heads] ("token"), [heads] ("head") or None ("none");
    states: fp32 [slots, heads, dk, dv]; offsets: int64 [seqs + 1]; slot_index: int32 [seqs].  Of packed sequences the kernels
    are chosen by the average length: single tokens of many requests and long prompts are better two calls.
    """

    op = "attn"

    def __init__(self, *, tokens, seqs, heads, dk, dv, qk_heads=None, slots=None, dtype="bf16", o_dtype=None,
                 decay="token", scale=1.0, q_strides=None, k_strides=None, v_strides=None, o_strides=None):
        qk_heads = heads if qk_heads is None else qk_heads
        slots = seqs if slots is None else slots
        dt = _pick(_DTYPES, dtype, "dtype")
        odt = dt if o_dtype is None else _pick(_DTYPES, o_dtype, "o_dtype")
        kind = _pick({"none": SEQMIX_DECAY_NONE, "head": SEQMIX_DECAY_HEAD, "token": SEQMIX_DECAY_TOKEN}, decay, "decay")
        strides = {n: tuple(s) if s is not None else (h * d, d) for n, s, h, d in (
            ("q", q_strides, qk_heads, dk), ("k", k_strides, qk_heads, dk), ("v", v_strides, heads, dv),
            ("o", o_strides, heads, dv))}
        super().__init__(seqmix_attn_params(
            tokens=tokens, seqs=seqs, slots=slots, heads=heads, qk_heads=qk_heads, dk=dk, dv=dv, dtype=dt, o_dtype=odt,
            decay=kind, scale=scale, **{f"{n}_{d}": s[i] for n, s in strides.items() for i, d in
                                        enumerate(("row", "head"))}))
        td, torch = self._td, self._torch
        for n, h, d in (("q", qk_heads, dk), ("k", qk_heads, dk), ("v", heads, dv)):
            self._expect(n, td[dt], (tokens, h, d), (*strides[n], 1))
        self._expect("decay", torch.float32, (tokens, heads) if decay == "token" else (heads,))
        self._expect("offsets", torch.int64, (seqs + 1,))
        self._expect("slot_index", torch.int32, (seqs,))
        self._expect("state_in", torch.float32, (slots, heads, dk, dv))
        self._expect("state_out", torch.float32, (slots, heads, dk, dv), out=True)
        self._expect("o", td[odt], (tokens, heads, dv), (*strides["o"], 1), out=True)

    def run(self, q, k, v, decay, state_in, state_out, o, offsets=None, slot_index=None, stream=None):
        self._launch(o, "o", stream, q, k, v, decay, offsets, slot_index, state_in, state_out, o)

    def plan(self):
        return seqmix_attn_plan_query(self.desc)

    def reserve(self):
        """Allocate the workspace now (before a graph capture)."""
        seqmix_attn_reserve(self.desc)


class TokenConv(_Operator):
    """seqmix_conv: x, y: [tokens, channels], w: [channels, width], bias: fp32 [channels], windows:
    [slots, width - 1, channels]; offsets and slot_index as for LinearAttention."""

    op = "conv"

    def __init__(self, *, tokens, seqs, channels, width, slots=None, dtype="bf16", act="silu", bias=True, x_row=None,
                 y_row=None):
        slots = seqs if slots is None else slots
        dt = _pick(_DTYPES, dtype, "dtype")
        x_row = channels if x_row is None else x_row
        y_row = channels if y_row is None else y_row
        super().__init__(seqmix_conv_params(
            tokens=tokens, seqs=seqs, slots=slots, channels=channels, width=width, dtype=dt,
            act=_pick({"none": SEQMIX_ACT_NONE, "silu": SEQMIX_ACT_SILU}, act, "act"), has_bias=1 if bias else 0,
            x_row=x_row, y_row=y_row))
        td, torch = self._td[dt], self._torch
        self._expect("x", td, (tokens, channels), (x_row, 1))
        self._expect("w", td, (channels, width))
        self._expect("bias", torch.float32, (channels,))
        self._expect("offsets", torch.int64, (seqs + 1,))
        self._expect("slot_index", torch.int32, (seqs,))
        self._expect("window_in", td, (slots, width - 1, channels))
        self._expect("window_out", td, (slots, width - 1, channels), out=True)
        self._expect("y", td, (tokens, channels), (y_row, 1), out=True)

    def run(self, x, w, bias, window_in, window_out, y, offsets=None, slot_index=None, stream=None):
        self._launch(y, "y", stream, x, w, bias, offsets, slot_index, window_in, window_out, y)


class GateNorm(_Operator):
    """seqmix_norm: u, gate, h: [rows, width], residual, y: [rows, width] in res_dtype; weights and biases fp32:
    post [group], pre and scale_vec [width].  gate_run rows share a row of the gate."""

    op = "norm"

    def __init__(self, *, rows, width, group=None, dtype="bf16", res_dtype=None, post="rms", post_bias=False,
                 gate="none", gate_run=1, gate_first=False, residual=False, scale=1.0, scale_vec=False, pre="none",
                 pre_bias=False, eps=1e-6, pre_eps=None, u_row=None, gate_row=None, res_row=None, y_row=None,
                 h_row=None):
        group = width if group is None else group
        dt = _pick(_DTYPES, dtype, "dtype")
        rdt = dt if res_dtype is None else _pick(_DTYPES, res_dtype, "res_dtype")
        norms = {"none": SEQMIX_NORM_NONE, "rms": SEQMIX_NORM_RMS, "layer": SEQMIX_NORM_LAYER}
        acts = {"none": SEQMIX_ACT_NONE, "silu": SEQMIX_ACT_SILU, "sigmoid": SEQMIX_ACT_SIGMOID,
                "linear": SEQMIX_ACT_LINEAR}
        row = {n: width if r is None else r for n, r in (("u_row", u_row), ("gate_row", gate_row), ("res_row", res_row),
                                                         ("y_row", y_row), ("h_row", h_row))}
        super().__init__(seqmix_norm_params(
            rows=rows, width=width, group=group, gate_run=gate_run, dtype=dt, res_dtype=rdt,
            post=_pick(norms, post, "post"), post_bias=1 if post_bias else 0, gate=_pick(acts, gate, "gate"),
            gate_first=1 if gate_first else 0, residual=1 if residual else 0, scale_vec=1 if scale_vec else 0,
            pre=_pick(norms, pre, "pre"), pre_bias=1 if pre_bias else 0, scale=scale, post_eps=eps,
            pre_eps=eps if pre_eps is None else pre_eps, **row))
        td, torch = self._td, self._torch
        self._expect("u", td[dt], (rows, width), (row["u_row"], 1))
        self._expect("post_w", torch.float32, (group,))
        self._expect("post_b", torch.float32, (group,))
        self._expect("gate", td[dt], (-(-rows // gate_run), width), (row["gate_row"], 1))
        self._expect("residual", td[rdt], (rows, width), (row["res_row"], 1))
        for n in ("scale_vec", "pre_w", "pre_b"):
            self._expect(n, torch.float32, (width,))
        self._expect("y", td[rdt], (rows, width), (row["y_row"], 1), out=True)
        self._expect("h", td[dt], (rows, width), (row["h_row"], 1), out=True)

    def run(self, u, post_w=None, post_b=None, gate=None, residual=None, scale_vec=None, pre_w=None, pre_b=None,
            y=None, h=None, stream=None):
        self._launch(u, "u", stream, u, post_w, post_b, gate, residual, scale_vec, pre_w, pre_b, y, h)


def _strides(given, *sizes):
    """Elements from one to the next of all but the last dimension: as given, or dense."""
    if given is not None:
        return tuple(given)
    dense, n = [], 1
    for d in reversed(sizes[1:]):
        n *= d
        dense.insert(0, n)
    return tuple(dense)


class SoftmaxAttention(_Operator):
    """seqmix_softmax of `tokens` rows in `seqs` sequences.

    q: [tokens, heads, dk], o: [tokens, heads, dv], strides as given (elements between rows and between heads) or dense;
    offsets: int64 [seqs + 1]; slot_index: int32 [seqs]; tree (mask "tree"): int64 [tokens].  Keys and values either
    packed (page 0), k: [key_tokens, kv_heads, dk], v alike, key_offsets: int64 [seqs + 1] (None: the rows of q),
    or in `pages` pages of `page` tokens, k: [pages, page, kv_heads, dk], v alike (three strides), lens: int32 [slots],
    table: int32 [slots, max_pages].  The kernels are chosen by the average number of rows of a sequence: prompts and single
    tokens are better two calls.
    """

    op = "softmax"

    def __init__(self, *, tokens, seqs, heads, dk, dv=None, kv_heads=None, slots=None, dtype="bf16", mask="causal", scale=None,
                 key_tokens=None, page=0, pages=0, max_pages=0, q_strides=None, k_strides=None, v_strides=None,
                 o_strides=None):
        kv_heads = heads if kv_heads is None else kv_heads
        dv = dk if dv is None else dv
        slots = seqs if slots is None else slots
        key_tokens = tokens if key_tokens is None else key_tokens
        dt = _pick(_DTYPES, dtype, "dtype")
        kind = _pick({"full": SEQMIX_MASK_FULL, "causal": SEQMIX_MASK_CAUSAL, "tree": SEQMIX_MASK_TREE}, mask, "mask")
        where = (pages, page) if page else (key_tokens,)
        qs, os_ = _strides(q_strides, tokens, heads, dk), _strides(o_strides, tokens, heads, dv)
        ks, vs = _strides(k_strides, *where, kv_heads, dk), _strides(v_strides, *where, kv_heads, dv)
        super().__init__(seqmix_softmax_params(
            tokens=tokens, seqs=seqs, slots=slots, key_tokens=key_tokens, pages=pages, max_pages=max_pages, page=page,
            heads=heads, kv_heads=kv_heads, dk=dk, dv=dv, dtype=dt, mask=kind,
            scale=dk ** -0.5 if scale is None else scale, q_row=qs[0], q_head=qs[1], o_row=os_[0], o_head=os_[1],
            k_row=ks[-2], k_head=ks[-1], k_page=ks[0] if page else 0, v_row=vs[-2], v_head=vs[-1],
            v_page=vs[0] if page else 0))
        td, torch = self._td[dt], self._torch
        self._expect("q", td, (tokens, heads, dk), (*qs, 1))
        self._expect("k", td, (*where, kv_heads, dk), (*ks, 1))
        self._expect("v", td, (*where, kv_heads, dv), (*vs, 1))
        self._expect("offsets", torch.int64, (seqs + 1,))
        self._expect("key_offsets", torch.int64, (seqs + 1,))
        self._expect("slot_index", torch.int32, (seqs,))
        self._expect("lens", torch.int32, (slots,))
        self._expect("table", torch.int32, (slots, max_pages))
        self._expect("tree", torch.int64, (tokens,))
        self._expect("o", td, (tokens, heads, dv), (*os_, 1), out=True)

    def run(self, q, k, v, o, offsets=None, key_offsets=None, slot_index=None, lens=None, table=None, tree=None, stream=None):
        self._launch(o, "o", stream, q, k, v, offsets, key_offsets, slot_index, lens, table, tree, o)

    def plan(self):
        return seqmix_softmax_plan_query(self.desc)

    def reserve(self):
        """Allocate the workspace now (before a graph capture)."""
        seqmix_softmax_reserve(self.desc)


class Rotary(_Operator):
    """seqmix_rotary: q, q_out: [tokens, heads, dk], k, k_out: [tokens, kv_heads, dk], v: [tokens, kv_heads, dv], strides as
    given or dense (q_out may be q, k_out k); position, place: int32 [tokens]; freqs: float64 [rot / 2]
    (`rotary_frequencies`); caches of `pages` pages of `page` tokens, k_cache: [pages, page, kv_heads, dk], v_cache alike."""

    op = "rotary"

    def __init__(self, *, tokens, heads, kv_heads, dk, dv=None, rot=None, layout="half", dtype="bf16", amplitude=1.0, page=0,
                 pages=0, q_strides=None, k_strides=None, v_strides=None, q_out_strides=None, k_out_strides=None,
                 k_cache_strides=None, v_cache_strides=None):
        dv = dk if dv is None else dv
        rot = dk if rot is None else rot
        dt = _pick(_DTYPES, dtype, "dtype")
        rows = {n: _strides(s, tokens, h, d) for n, s, h, d in (
            ("q", q_strides, heads, dk), ("k", k_strides, kv_heads, dk), ("v", v_strides, kv_heads, dv),
            ("qo", q_out_strides, heads, dk), ("ko", k_out_strides, kv_heads, dk))}
        caches = {n: _strides(s, pages, page, kv_heads, d) for n, s, d in (("kc", k_cache_strides, dk),
                                                                           ("vc", v_cache_strides, dv))}
        super().__init__(seqmix_rotary_params(
            tokens=tokens, pages=pages, page=page, heads=heads, kv_heads=kv_heads, dk=dk, dv=dv, rot=rot,
            layout=_pick({"half": SEQMIX_ROTARY_HALF, "interleaved": SEQMIX_ROTARY_INTERLEAVED}, layout, "layout"),
            dtype=dt, amplitude=amplitude,
            **{f"{n}_{d}": s[i] for n, s in rows.items() for i, d in enumerate(("row", "head"))},
            **{f"{n}_{d}": s[i] for n, s in caches.items() for i, d in enumerate(("page", "row", "head"))}))
        td, torch = self._td[dt], self._torch
        self._expect("q", td, (tokens, heads, dk), (*rows["q"], 1))
        self._expect("k", td, (tokens, kv_heads, dk), (*rows["k"], 1))
        self._expect("v", td, (tokens, kv_heads, dv), (*rows["v"], 1))
        self._expect("position", torch.int32, (tokens,))
        self._expect("freqs", torch.float64, (rot // 2,))
        self._expect("q_out", td, (tokens, heads, dk), (*rows["qo"], 1), out=True)
        self._expect("k_out", td, (tokens, kv_heads, dk), (*rows["ko"], 1), out=True)
        self._expect("k_cache", td, (pages, page, kv_heads, dk), (*caches["kc"], 1), out=True)
        self._expect("v_cache", td, (pages, page, kv_heads, dv), (*caches["vc"], 1), out=True)
        self._expect("place", torch.int32, (tokens,))

    def run(self, q, k, v, position, freqs, q_out, k_out=None, k_cache=None, v_cache=None, place=None, stream=None):
        self._launch(position, "position", stream, q, k, v, position, freqs, q_out, k_out, k_cache, v_cache, place)


def rotary_frequencies(rot, base=10000.0, factor=1.0, trained=None, low=1.0, high=4.0, device="cuda"):
    """float64 [rot / 2]: base ** (-2 i / rot) radians per position, for texts `factor` times longer than trained on.

    Without `trained` all are divided by the factor.  With it (the positions trained on), those that turn less than `low` times
    over them are, those that turn more than `high` times stay as they are, and between them the share grows evenly with the turns."""
    import math

    import torch
    if not low < high:
        raise ValueError(f"low < high: got {low} and {high}")
    f = base ** -(torch.arange(rot // 2, dtype=torch.float64, device=device) * 2 / max(rot, 1))
    if trained is None:
        return f / factor
    keep = ((trained * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
    return f * keep + f / factor * (1 - keep)


class CachePages(_Operator):
    """seqmix_pages of `tokens` new rows in `seqs` sequences: kept, slot_index, admitted: int32 [seqs]; offsets: int64
    [seqs + 1]; lens: int32 [slots], table: int32 [slots, max_pages], free_pages: int32 [pages], taken: int32 [1] (all updated);
    place, position: int32 [tokens].  `empty` makes the four of a pool without requests."""

    op = "pages"

    def __init__(self, *, tokens, seqs, page, pages, max_pages, slots=None):
        slots = seqs if slots is None else slots
        super().__init__(seqmix_pages_params(tokens=tokens, seqs=seqs, slots=slots, pages=pages, max_pages=max_pages,
                                             page=page))
        i32 = self._torch.int32
        self._expect("kept", i32, (seqs,))
        self._expect("offsets", self._torch.int64, (seqs + 1,))
        self._expect("slot_index", i32, (seqs,))
        for n, shape in (("lens", (slots,)), ("table", (slots, max_pages)), ("free_pages", (pages,)), ("taken", (1,)),
                         ("place", (tokens,)), ("position", (tokens,)), ("admitted", (seqs,))):
            self._expect(n, i32, shape, out=True)

    @staticmethod
    def empty(slots, pages, max_pages, device="cuda"):
        """lens, table, free_pages, taken."""
        import torch
        return (torch.zeros(slots, dtype=torch.int32, device=device),
                torch.full((slots, max_pages), -1, dtype=torch.int32, device=device),
                torch.arange(pages, dtype=torch.int32, device=device), torch.zeros(1, dtype=torch.int32, device=device))

    def run(self, kept, lens, table, free_pages, taken, place, position, admitted, offsets=None, slot_index=None, stream=None):
        self._launch(lens, "lens", stream, kept, offsets, slot_index, lens, table, free_pages, taken, place, position, admitted)
