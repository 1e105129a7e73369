"""The operators of a memory block on torch tensors: binding of include/sf_memory.h.

  linear_attention, linear_attention_backward, linear_attention_step
  residual_norm, residual_norm_backward
  gated_ffn, gated_ffn_backward

Argument checks and marshalling only; every operator runs in the library's HIP kernels, on `stream` or the current
stream.  Each function puts its results into `out` (a dict) and returns it.  A program that calls one again and
again keeps that dict: buffers that are there already are written to (they have to fit), and so is the workspace.
"""
import ctypes as C

from . import binding
from .binding import SF_OK, SfError, sf_last_error

SF_DTYPE_FP32, SF_DTYPE_BF16 = 0, 1

EXPORTS = ("sf_linattn_workspace_bytes", "sf_linattn", "sf_linattn_backward", "sf_linattn_step", "sf_resnorm", "sf_resnorm_workspace_bytes",
           "sf_resnorm_backward", "sf_ffn_workspace_bytes", "sf_ffn", "sf_ffn_backward")

_STRIDE = C.c_int64 * 3


class SfLinattnConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("T", C.c_int32), ("N", C.c_int32), ("H", C.c_int32),
                ("Hk", C.c_int32), ("dk", C.c_int32), ("dv", C.c_int32), ("scale", C.c_float),
                ("q_stride", _STRIDE), ("k_stride", _STRIDE), ("v_stride", _STRIDE), ("o_stride", _STRIDE)]


class SfResnormConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("M", C.c_int32), ("D", C.c_int32), ("groups", C.c_int32),
                ("post", C.c_int32), ("pre", C.c_int32), ("gate_act", C.c_int32), ("eps", C.c_float), ("b_stride", C.c_int64),
                ("x_stride", C.c_int64), ("gate_stride", C.c_int64), ("dy_stride", C.c_int64), ("dn_stride", C.c_int64)]


class SfFfnConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("M", C.c_int32), ("D", C.c_int32), ("F", C.c_int32),
                ("act", C.c_int32), ("x_stride", C.c_int64), ("w_gate_stride", C.c_int64), ("w_up_stride", C.c_int64),
                ("w_down_stride", C.c_int64), ("dy_stride", C.c_int64)]


# by their C names
STRUCTS = {"sf_linattn_config": SfLinattnConfig, "sf_resnorm_config": SfResnormConfig, "sf_ffn_config": SfFfnConfig}

_lib = None


def load_library():
    """The library with these entry points' signatures set; raises if it has not been built."""
    global _lib
    if _lib is None:
        L = binding.load_library()
        P = C.c_void_p
        for name, restype, argtypes in (
                ("sf_linattn_workspace_bytes", C.c_int64, [C.POINTER(SfLinattnConfig), C.c_int]),
                ("sf_linattn", C.c_int, [C.POINTER(SfLinattnConfig)] + [P] * 10),
                ("sf_linattn_backward", C.c_int, [C.POINTER(SfLinattnConfig)] + [P] * 14),
                ("sf_linattn_step", C.c_int, [C.POINTER(SfLinattnConfig)] + [P] * 5 + [C.c_int32] + [P] * 4),
                ("sf_resnorm", C.c_int, [C.POINTER(SfResnormConfig)] + [P] * 9),
                ("sf_resnorm_workspace_bytes", C.c_int64, [C.POINTER(SfResnormConfig)]),
                ("sf_resnorm_backward", C.c_int, [C.POINTER(SfResnormConfig)] + [P] * 16),
                ("sf_ffn_workspace_bytes", C.c_int64, [C.POINTER(SfFfnConfig), C.c_int]),
                ("sf_ffn", C.c_int, [C.POINTER(SfFfnConfig)] + [P] * 7),
                ("sf_ffn_backward", C.c_int, [C.POINTER(SfFfnConfig)] + [P] * 11)):
            f = getattr(L, name)
            f.restype, f.argtypes = restype, argtypes
        _lib = L
    return _lib


def _check(rc):
    if rc != SF_OK:
        raise SfError(rc, sf_last_error())


_dtypes = None


def _dtype_of(t):
    """SF_DTYPE_* of a tensor."""
    global _dtypes
    if _dtypes is None:
        torch = binding._torch()
        _dtypes = {torch.float32: SF_DTYPE_FP32, torch.bfloat16: SF_DTYPE_BF16}
    return _dtypes[t.dtype] if t.dtype in _dtypes else _refuse("dtype %s: float32 or bfloat16 is wanted" % t.dtype)


def _refuse(text):
    raise ValueError(text)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _same(name, t, like, shape, dtype=None, dense=True):
    """Checks an argument that has to be on like's device, of `shape`, and (dense) contiguous."""
    if tuple(t.shape) != shape or t.dtype != (like.dtype if dtype is None else dtype) or t.device != like.device:
        _refuse("%s: %s %s on %s, wanted %s %s on %s" % (name, tuple(t.shape), t.dtype, t.device, shape,
                                                        like.dtype if dtype is None else dtype, like.device))
    if dense and not t.is_contiguous():
        _refuse("%s is not contiguous" % name)
    return t


def _result(out, name, shape, dtype, device):
    t = out.get(name)
    if t is None:
        t = out[name] = binding._torch().empty(shape, dtype=dtype, device=device)
    elif tuple(t.shape) != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        _refuse("out[%r] does not fit: %s %s on %s is wanted, contiguous" % (name, shape, dtype, device))
    return t


def _workspace(out, n_bytes, device):
    if n_bytes < 0:
        raise SfError(binding.SF_ERR_SHAPE, sf_last_error())
    if not n_bytes:
        return None
    w = out.get("workspace")
    if w is None or w.numel() < n_bytes or w.device != device:
        torch = binding._torch()
        w = out["workspace"] = torch.empty(n_bytes, dtype=torch.uint8, device=device)
    return w.data_ptr()


def _stream(stream, device):
    return (binding._torch().cuda.current_stream(device) if stream is None else stream).cuda_stream


def _rows(name, t):
    """Strides of a tensor whose last axis is dense (any stride where an axis has one element)."""
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse("%s: the last axis is not dense" % name)
    return t.stride()[:-1]


def _linattn_config(q, k, v, log_decay, scale, steps):
    """steps: the arrays have a time axis in front."""
    if not q.is_cuda:
        _refuse("q is not on the GPU")
    if q.dim() != (4 if steps else 3) or k.dim() != q.dim() or v.dim() != q.dim():
        _refuse("q, k, v: %s, %s, %s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    lead, (H, dk) = tuple(q.shape[:-2]), q.shape[-2:]
    Hk, dv = v.shape[-2:]
    _same("k", k, q, lead + (Hk, dk), dense=False)
    _same("v", v, q, lead + (Hk, dv), dense=False)
    _same("log_decay", log_decay, q, (H,), dtype=binding._torch().float32)
    c = SfLinattnConfig(C.sizeof(SfLinattnConfig), _dtype_of(q), lead[0] if steps else 1, lead[-1], H, Hk, dk, dv,
                        dk ** -0.5 if scale is None else scale)
    for field, name, t in ((c.q_stride, "q", q), (c.k_stride, "k", k), (c.v_stride, "v", v)):
        s = _rows(name, t)
        field[0], field[1], field[2] = s if steps else (0,) + s
    c.o_stride[0], c.o_stride[1], c.o_stride[2] = lead[-1] * H * dv, H * dv, dv
    return c


def _optional(name, t, like, shape, dtype):
    return None if t is None else _same(name, t, like, shape, dtype).data_ptr()


def linear_attention(q, k, v, log_decay, done=None, state0=None, scale=None, out=None, stream=None):
    """Over N trajectories of T steps: q [T,N,H,dk], k [T,N,Hk,dk], v [T,N,Hk,dv] (bf16 or fp32, last axis dense),
    log_decay fp32 [H], done u8 [T,N], state0 fp32 [N,H,dk,dv]; scale: dk ** -0.5.  Results: o [T,N,H,dv],
    state [N,H,dk,dv]."""
    torch = binding._torch()
    out = {} if out is None else out
    c = _linattn_config(q, k, v, log_decay, scale, True)
    T, N, H, dk = q.shape
    d, s = q.device, (N, H, dk, c.dv)
    done = _optional("done", done, q, (T, N), torch.uint8)
    s0 = _optional("state0", state0, q, s, torch.float32)
    o = _result(out, "o", (T, N, H, c.dv), q.dtype, d)
    state = _result(out, "state", s, torch.float32, d)
    L = load_library()
    w = _workspace(out, L.sf_linattn_workspace_bytes(C.byref(c), 0), d)
    _check(L.sf_linattn(C.byref(c), q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), done, s0, o.data_ptr(),
                        state.data_ptr(), w, _stream(stream, d)))
    return out


def linear_attention_backward(q, k, v, log_decay, do, done=None, state0=None, dstate=None, scale=None, out=None, stream=None):
    """Gradients of linear_attention with the same arguments, given those of o (do) and of the final state (dstate, or
    None).  Results: dq, dk, dv, dstate0."""
    torch = binding._torch()
    out = {} if out is None else out
    c = _linattn_config(q, k, v, log_decay, scale, True)
    T, N, H, dk = q.shape
    d, s, f32 = q.device, (N, H, dk, c.dv), torch.float32
    _same("do", do, q, (T, N, H, c.dv), dense=False)
    c.o_stride[0], c.o_stride[1], c.o_stride[2] = _rows("do", do)
    done = _optional("done", done, q, (T, N), torch.uint8)
    s0, ds = _optional("state0", state0, q, s, f32), _optional("dstate", dstate, q, s, f32)
    dq = _result(out, "dq", (T, N, H, dk), q.dtype, d)
    gk = _result(out, "dk", (T, N, c.Hk, dk), q.dtype, d)
    gv = _result(out, "dv", (T, N, c.Hk, c.dv), q.dtype, d)
    ds0 = _result(out, "dstate0", s, f32, d)
    L = load_library()
    w = _workspace(out, L.sf_linattn_workspace_bytes(C.byref(c), 1), d)
    _check(L.sf_linattn_backward(C.byref(c), q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), do.data_ptr(), done,
                                 s0, ds, dq.data_ptr(), gk.data_ptr(), gv.data_ptr(), ds0.data_ptr(), w, _stream(stream, d)))
    return out


def linear_attention_step(q, k, v, log_decay, state_table, env_ids=None, done=None, scale=None, out=None, stream=None):
    """One step of B environments: q [B,H,dk], k [B,Hk,dk], v [B,Hk,dv], done u8 [B]; state_table fp32 [n_env,H,dk,dv] is
    read and overwritten at the rows env_ids (i32 [B], distinct; None: rows 0 .. B-1).  Result: o [B,H,dv]."""
    torch = binding._torch()
    out = {} if out is None else out
    c = _linattn_config(q, k, v, log_decay, scale, False)
    B, H, dk = q.shape
    n_env = state_table.shape[0]
    _same("state_table", state_table, q, (n_env, H, dk, c.dv), torch.float32)
    ids = _optional("env_ids", env_ids, q, (B,), torch.int32)
    done = _optional("done", done, q, (B,), torch.uint8)
    o = _result(out, "o", (B, H, c.dv), q.dtype, q.device)
    _check(load_library().sf_linattn_step(C.byref(c), q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(),
                                          state_table.data_ptr(), n_env, ids, done, o.data_ptr(), _stream(stream, q.device)))
    return out


_NORMS = {"none": 0, "rms": 1, "layer": 2}
_GATES = {"none": 0, "sigmoid": 1, "silu": 2}


def _flat(name, t, like=None):
    """A tensor of rows [..., D] as [M, D] (no copy)."""
    if t.dim() != 2:
        t = t.view(-1, t.shape[-1])
    if like is not None:
        _same(name, t, like, tuple(like.shape), dense=False)
    if t.shape[1] > 1 and t.stride(1) != 1:
        _refuse("%s: the last axis is not dense" % name)
    return t


def _resnorm_config(b, x, gate, post, pre, post_w, pre_w, scale, groups, gate_act, eps):
    """The configuration, b, x and the gate as rows, and the weights' addresses."""
    if not b.is_cuda:
        _refuse("b is not on the GPU")
    b = _flat("b", b)
    for what, how, known in (("post", post, _NORMS), ("pre", pre, _NORMS), ("gate_act", gate_act, _GATES)):
        if how not in known:
            _refuse("%s = %r: one of %s is wanted" % (what, how, ", ".join(known)))
    if (gate is None) != (gate_act == "none"):
        _refuse("a gate and its activation come together")
    M, D = b.shape
    x = None if x is None else _flat("x", x, b)
    gate = None if gate is None else _flat("gate", gate, b)
    f32 = binding._torch().float32
    w = tuple(_optional(n, t, b, (D,), f32) for n, t in (("post_w", post_w), ("scale", scale), ("pre_w", pre_w)))
    c = SfResnormConfig(C.sizeof(SfResnormConfig), _dtype_of(b), M, D, groups, _NORMS[post], _NORMS[pre], _GATES[gate_act], eps,
                        b.stride(0), 0 if x is None else x.stride(0), 0 if gate is None else gate.stride(0), 0, 0)
    return c, b, x, gate, w


def residual_norm(b, x=None, gate=None, post="rms", pre="rms", post_w=None, pre_w=None, scale=None, groups=1, gate_act="none",
                  eps=1e-6, out=None, stream=None):
    """y = x + scale * act(gate) * N_post(b) * post_w and n = N_pre(y) * pre_w over rows [..., D] (bf16 or fp32, last axis
    dense; weights fp32 [D]).  post, pre: "none", "rms" or "layer"; gate_act: "none", "sigmoid" or "silu"; groups: of
    channels that post is taken over (pre "none" then).  Results: y and, with pre, n."""
    out = {} if out is None else out
    shape = tuple(b.shape)
    c, b, x, gate, w = _resnorm_config(b, x, gate, post, pre, post_w, pre_w, scale, groups, gate_act, eps)
    y = _result(out, "y", shape, b.dtype, b.device)
    n = _result(out, "n", shape, b.dtype, b.device) if c.pre else None
    _check(load_library().sf_resnorm(C.byref(c), b.data_ptr(), _ptr(x), _ptr(gate), w[0], w[1], w[2], y.data_ptr(), _ptr(n),
                                     _stream(stream, b.device)))
    return out


def residual_norm_backward(b, dy, dn=None, x=None, gate=None, post="rms", pre="rms", post_w=None, pre_w=None, scale=None, groups=1,
                           gate_act="none", eps=1e-6, out=None, stream=None):
    """Gradients of residual_norm with the same arguments, given those of y (None: zero) and, with pre, of n.  Results: db and,
    for what was given, dx, dgate, dpost_w, dscale, dpre_w (fp32)."""
    out = {} if out is None else out
    shape = tuple(b.shape)
    c, b, x, gate, w = _resnorm_config(b, x, gate, post, pre, post_w, pre_w, scale, groups, gate_act, eps)
    if dn is None and c.pre:
        _refuse("dn is wanted with pre = %r" % pre)
    if dy is None and not c.pre:
        _refuse("dy is wanted")
    if dy is not None:
        dy = _flat("dy", dy, b)
        c.dy_stride = dy.stride(0)
    if dn is not None:
        dn = _flat("dn", dn, b)
        c.dn_stride = dn.stride(0)
    d, f32, D = b.device, binding._torch().float32, (b.shape[1],)
    db = _result(out, "db", shape, b.dtype, d)
    dx = None if x is None else _result(out, "dx", shape, b.dtype, d)
    dgate = None if gate is None else _result(out, "dgate", shape, b.dtype, d)
    dw = [None if t is None else _result(out, n, D, f32, d) for n, t in (("dpost_w", post_w), ("dscale", scale), ("dpre_w", pre_w))]
    L = load_library()
    ws = _workspace(out, L.sf_resnorm_workspace_bytes(C.byref(c)), d) if any(t is not None for t in dw) else None
    _check(L.sf_resnorm_backward(C.byref(c), b.data_ptr(), _ptr(x), _ptr(gate), w[0], w[1], w[2], _ptr(dy), _ptr(dn), _ptr(dx),
                                 db.data_ptr(), _ptr(dgate), _ptr(dw[0]), _ptr(dw[1]), _ptr(dw[2]), ws, _stream(stream, d)))
    return out


_ACTS = {"silu": 0, "gelu": 1, "sigmoid": 2}


def _ffn_config(x, w_gate, w_up, w_down, act):
    if not x.is_cuda:
        _refuse("x is not on the GPU")
    if act not in _ACTS:
        _refuse("act = %r: one of %s is wanted" % (act, ", ".join(_ACTS)))
    x = _flat("x", x)
    if w_gate.dim() != 2:
        _refuse("w_gate: %s" % (tuple(w_gate.shape),))
    (M, D), F = x.shape, w_gate.shape[0]
    for name, w, shape in (("w_gate", w_gate, (F, D)), ("w_up", w_up, (F, D)), ("w_down", w_down, (D, F))):
        _same(name, w, x, shape, dense=False)
        _rows(name, w)
    c = SfFfnConfig(C.sizeof(SfFfnConfig), _dtype_of(x), M, D, F, _ACTS[act], x.stride(0), w_gate.stride(0), w_up.stride(0), w_down.stride(0), 0)
    return c, x


def gated_ffn(x, w_gate, w_up, w_down, act="silu", out=None, stream=None):
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T: x [..., D], w_gate and w_up [F,D], w_down [D,F] (all bf16 or all fp32, last
    axis dense); act: "silu", "gelu" or "sigmoid".  Result: y [..., D]."""
    out = {} if out is None else out
    shape = tuple(x.shape)
    c, x = _ffn_config(x, w_gate, w_up, w_down, act)
    y = _result(out, "y", shape, x.dtype, x.device)
    L = load_library()
    w = _workspace(out, L.sf_ffn_workspace_bytes(C.byref(c), 0), x.device)
    _check(L.sf_ffn(C.byref(c), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), y.data_ptr(), w, _stream(stream, x.device)))
    return out


def gated_ffn_backward(x, w_gate, w_up, w_down, dy, act="silu", out=None, stream=None):
    """Gradients of gated_ffn with the same arguments, given that of y.  Results: dx, dw_gate, dw_up, dw_down."""
    out = {} if out is None else out
    shape, d = tuple(x.shape), x.device
    c, x = _ffn_config(x, w_gate, w_up, w_down, act)
    dy = _flat("dy", dy, x)
    c.dy_stride = dy.stride(0)
    got = [_result(out, n, s, x.dtype, d) for n, s in (("dx", shape), ("dw_gate", (c.F, c.D)), ("dw_up", (c.F, c.D)), ("dw_down", (c.D, c.F)))]
    L = load_library()
    w = _workspace(out, L.sf_ffn_workspace_bytes(C.byref(c), 1), d)
    _check(L.sf_ffn_backward(C.byref(c), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), dy.data_ptr(),
                             *(t.data_ptr() for t in got), w, _stream(stream, d)))
    return out
