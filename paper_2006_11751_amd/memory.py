"""The operators of a memory block on torch tensors: binding of include/sf_memory.h.

  linear_attention, linear_attention_backward, linear_attention_step
  delta_rule, delta_rule_backward, delta_rule_step
  residual_norm, residual_norm_backward
  gated_ffn, gated_ffn_backward
  clip_gradients

Argument checks and marshalling only; every operator runs in the library's HIP kernels, on the tensors' device, on its
current stream or, with `stream`, as if that were current (its order to other streams' work is the caller's; tensors and
results may be dropped right after the call).  Each function puts its results into `out` (a dict) and returns it.  A
program that calls one again and again keeps that dict: buffers that are there already are written to (they have to fit),
and so is the workspace.  One that has become too small stays in the dict, as "workspace_1" and so on, for graphs that
were recorded with it; who has none may take it out.
Calls are short (a policy worker's step takes a few microseconds on the GPU), so what the checks of a call found is kept
by the shapes, strides, types and devices of its arguments, and the checks are made once for each of these.
They are not part of autograd's graph: results carry no history, whether or not an argument requires a gradient, and the
gradients are what the *_backward functions return.
"""
import array
import ctypes as C
import operator

from . import binding
from .binding import SF_OK, SfError, sf_last_error

SF_DTYPE_FP32, SF_DTYPE_BF16 = 0, 1

EXPORTS = ("sf_linattn_workspace_bytes", "sf_linattn", "sf_linattn_backward", "sf_linattn_step",
           "sf_deltarule_workspace_bytes", "sf_deltarule", "sf_deltarule_backward", "sf_deltarule_step", "sf_resnorm",
           "sf_resnorm_workspace_bytes", "sf_resnorm_backward", "sf_ffn_workspace_bytes", "sf_ffn", "sf_ffn_backward",
           "sf_gradclip_workspace_bytes", "sf_gradclip")

_STRIDE = C.c_int64 * 3


class SfLinattnConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("T", C.c_int32), ("N", C.c_int32), ("H", C.c_int32),
                ("Hk", C.c_int32), ("dk", C.c_int32), ("dv", C.c_int32), ("scale", C.c_float),
                ("q_stride", _STRIDE), ("k_stride", _STRIDE), ("v_stride", _STRIDE), ("o_stride", _STRIDE)]


class SfDeltaruleConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("T", C.c_int32), ("N", C.c_int32), ("H", C.c_int32),
                ("Hk", C.c_int32), ("dk", C.c_int32), ("dv", C.c_int32), ("scale", C.c_float),
                ("q_stride", _STRIDE), ("k_stride", _STRIDE), ("v_stride", _STRIDE), ("do_stride", _STRIDE)]


class SfResnormConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("M", C.c_int32), ("D", C.c_int32), ("groups", C.c_int32),
                ("post", C.c_int32), ("pre", C.c_int32), ("gate_act", C.c_int32), ("eps", C.c_float), ("b_stride", C.c_int64),
                ("x_stride", C.c_int64), ("gate_stride", C.c_int64), ("dy_stride", C.c_int64), ("dn_stride", C.c_int64)]


class SfFfnConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("M", C.c_int32), ("D", C.c_int32), ("F", C.c_int32),
                ("act", C.c_int32), ("x_stride", C.c_int64), ("w_gate_stride", C.c_int64), ("w_up_stride", C.c_int64),
                ("w_down_stride", C.c_int64), ("dy_stride", C.c_int64)]


class SfGradclipConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n", C.c_int32), ("max_norm", C.c_float), ("eps", C.c_float)]


# by their C names
STRUCTS = {"sf_linattn_config": SfLinattnConfig, "sf_deltarule_config": SfDeltaruleConfig, "sf_resnorm_config": SfResnormConfig, "sf_ffn_config": SfFfnConfig,
           "sf_gradclip_config": SfGradclipConfig}

_lib = None


def load_library():
    """The library with these entry points' signatures set; raises if it has not been built."""
    global _lib
    if _lib is None:
        L = binding.load_library()
        P = C.c_void_p  # (of a configuration too: its address is taken once, when it is made)
        for name, restype, argtypes in (
                ("sf_linattn_workspace_bytes", C.c_int64, [P, C.c_int]),
                ("sf_linattn", C.c_int, [P] * 11),
                ("sf_linattn_backward", C.c_int, [P] * 15),
                ("sf_linattn_step", C.c_int, [P] * 6 + [C.c_int32] + [P] * 4),
                ("sf_deltarule_workspace_bytes", C.c_int64, [P, C.c_int]),
                ("sf_deltarule", C.c_int, [P] * 12),
                ("sf_deltarule_backward", C.c_int, [P] * 18),
                ("sf_deltarule_step", C.c_int, [P] * 7 + [C.c_int32] + [P] * 4),
                ("sf_resnorm", C.c_int, [P] * 10),
                ("sf_resnorm_workspace_bytes", C.c_int64, [P]),
                ("sf_resnorm_backward", C.c_int, [P] * 17),
                ("sf_ffn_workspace_bytes", C.c_int64, [P, C.c_int]),
                ("sf_ffn", C.c_int, [P] * 8),
                ("sf_ffn_backward", C.c_int, [P] * 12),
                ("sf_gradclip_workspace_bytes", C.c_int64, [C.c_int32, P]),
                ("sf_gradclip", C.c_int, [P] * 8)):
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


def _number(x):
    """A number as what it is now: a plan must not hold a tensor that may change in place."""
    return x if x is None or type(x) is float else float(x)


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


def _optional(name, t, like, shape, dtype):
    if t is not None:
        _same(name, t, like, shape, dtype)


def _rows(name, t):
    """Strides of a tensor whose last axis is dense (any stride where an axis has one element)."""
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse("%s: the last axis is not dense" % name)
    return t.stride()[:-1]


class _Plan:
    """What the checks of a call found: the configuration, the results' shapes and types, the size of the workspace."""
    __slots__ = ("key", "config", "address", "results", "n_bytes", "device", "index")

    def __init__(self, config, results, n_bytes, device):
        if n_bytes < 0:
            raise SfError(binding.SF_ERR_SHAPE, sf_last_error())
        self.config, self.address, self.n_bytes, self.device, self.index = config, C.addressof(config), n_bytes, device, device.index
        torch = binding._torch()
        self.results = [(name, torch.Size(shape), dtype) for name, shape, dtype in results]


_plans = {}  # by key: (function, arguments that are no tensors, what the tensors are)
_last = {}   # by function: the plan it used last


def _plan(name, rest, tensors, build, *args):
    key = [rest]
    for t in tensors:
        if t is None:
            key.append(None)
        else:
            key += (t.shape, t.stride(), t.dtype, t.device)
    plan = _last.get(name)
    if plan is not None and plan.key == key:
        return plan
    whole = (name,) + tuple(key)
    plan = _plans.get(whole)
    if plan is None:
        load_library()
        plan = build(*args)
        plan.key = key
        if len(_plans) >= 1024:
            _plans.clear()
        _plans[whole] = plan
    _last[name] = plan
    return plan


def _results(out, plan):
    """The results' addresses; what is not in `out` is allocated."""
    got = []
    for name, shape, dtype in plan.results:
        t = out.get(name)
        if t is None:
            t = out[name] = binding._torch().empty(shape, dtype=dtype, device=plan.device)
        elif t.shape != shape or t.dtype != dtype or t.device != plan.device or not t.is_contiguous():
            _refuse("out[%r] does not fit: %s %s on %s is wanted, contiguous" % (name, tuple(shape), dtype, plan.device))
        got.append(t.data_ptr())
    return got


def _workspace(out, plan):
    if not plan.n_bytes:
        return None
    w = out.get("workspace")
    if w is None or w.numel() < plan.n_bytes or w.device != plan.device:
        if w is not None:  # (a graph that was recorded with it goes on writing there)
            out["workspace_%d" % (1 + sum(name.startswith("workspace_") for name in out))] = w
        torch = binding._torch()
        w = out["workspace"] = torch.empty(plan.n_bytes, dtype=torch.uint8, device=plan.device)
    elif not w.is_contiguous():
        _refuse("out['workspace'] is not contiguous")
    return w.data_ptr()


# Torch's functions for the current device's index and for the handle of a device's current stream, from the first call on (the
# handle alone: a Stream object of torch costs two microseconds).
def _current_device():
    global _current_device
    _current_device = binding._torch()._C._cuda_getDevice
    return _current_device()


def _stream(index):
    global _stream
    _stream = binding._torch()._C._cuda_getCurrentRawStream
    return _stream(index)


def _elsewhere(stream, plan, call, first, rest, out):
    """call(*first, *rest, out=out) with the tensors' device and, where one is given, `stream` as the current ones, so that what it
    allocates is that stream's.  The allocator is told of every tensor that now has work on it there, and of the stream that was current
    before, for which the results are: memory that is let go of after the call is given out again only when both are done with it."""
    torch = binding._torch()
    if stream is None:
        with torch.cuda.device(plan.device):
            return call(*first, *rest, out=out)
    if stream.device != plan.device:
        _refuse("the stream is on %s, the tensors are on %s" % (stream.device, plan.device))
    before = torch.cuda.current_stream(plan.device)
    with torch.cuda.stream(stream):
        try:
            return call(*first, *rest, out=out)
        finally:
            if stream != before:
                for t in (*first, *rest, *out.values()):
                    for t in t if isinstance(t, (list, tuple)) else (t,):
                        if isinstance(t, torch.Tensor) and t.is_cuda:
                            t.record_stream(stream)
                            t.record_stream(before)


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


def linear_attention(q, k, v, log_decay, done=None, state0=None, scale=None, out=None, stream=None):
    """Over N trajectories of T steps: q [T,N,H,dk], k [T,N,Hk,dk], v [T,N,Hk,dv] (bf16 or fp32, last axis dense),
    log_decay fp32 [H], done u8 [T,N], state0 fp32 [N,H,dk,dv]; scale: dk ** -0.5.  Results: o [T,N,H,dv],
    state [N,H,dk,dv]."""
    out, scale = {} if out is None else out, _number(scale)
    plan = _plan("linear_attention", scale, (q, k, v, log_decay, done, state0), _linattn_plan, q, k, v, log_decay, done, state0, scale)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, linear_attention, (q, k, v, log_decay, done, state0), (scale,), out)
    o, state = _results(out, plan)
    _check(_lib.sf_linattn(plan.address, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), _ptr(done), _ptr(state0), o, state,
                           _workspace(out, plan), _stream(plan.index)))
    return out


def _linattn_plan(q, k, v, log_decay, done, state0, scale):
    torch = binding._torch()
    c = _linattn_config(q, k, v, log_decay, scale, True)
    T, N, H, dk = q.shape
    s = (N, H, dk, c.dv)
    _optional("done", done, q, (T, N), torch.uint8)
    _optional("state0", state0, q, s, torch.float32)
    return _Plan(c, (("o", (T, N, H, c.dv), q.dtype), ("state", s, torch.float32)),
                 _lib.sf_linattn_workspace_bytes(C.addressof(c), 0), q.device)


def linear_attention_backward(q, k, v, log_decay, do, done=None, state0=None, dstate=None, scale=None, out=None, stream=None):
    """Gradients of linear_attention with the same arguments, given those of o (do) and of the final state (dstate, or
    None).  Results: dq, dk, dv, dstate0."""
    out, scale = {} if out is None else out, _number(scale)
    plan = _plan("linear_attention_backward", scale, (q, k, v, log_decay, do, done, state0, dstate), _linattn_back_plan, q, k, v, log_decay, do,
                 done, state0, dstate, scale)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, linear_attention_backward, (q, k, v, log_decay, do, done, state0, dstate), (scale,), out)
    dq, dk, dv, ds0 = _results(out, plan)
    _check(_lib.sf_linattn_backward(plan.address, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), do.data_ptr(), _ptr(done),
                                    _ptr(state0), _ptr(dstate), dq, dk, dv, ds0, _workspace(out, plan), _stream(plan.index)))
    return out


def _linattn_back_plan(q, k, v, log_decay, do, done, state0, dstate, scale):
    torch = binding._torch()
    c = _linattn_config(q, k, v, log_decay, scale, True)
    T, N, H, dk = q.shape
    s, f32 = (N, H, dk, c.dv), torch.float32
    _same("do", do, q, (T, N, H, c.dv), dense=False)
    c.o_stride[0], c.o_stride[1], c.o_stride[2] = _rows("do", do)
    _optional("done", done, q, (T, N), torch.uint8)
    _optional("state0", state0, q, s, f32)
    _optional("dstate", dstate, q, s, f32)
    return _Plan(c, (("dq", (T, N, H, dk), q.dtype), ("dk", (T, N, c.Hk, dk), q.dtype), ("dv", (T, N, c.Hk, c.dv), q.dtype), ("dstate0", s, f32)),
                 _lib.sf_linattn_workspace_bytes(C.addressof(c), 1), q.device)


def linear_attention_step(q, k, v, log_decay, state_table, env_ids=None, done=None, scale=None, out=None, stream=None):
    """One step of B environments: q [B,H,dk], k [B,Hk,dk], v [B,Hk,dv], done u8 [B]; state_table fp32 [n_env,H,dk,dv] is
    read and overwritten at the rows env_ids (i32 [B], distinct; None: rows 0 .. B-1).  Result: o [B,H,dv]."""
    out, scale = {} if out is None else out, _number(scale)
    plan = _plan("linear_attention_step", scale, (q, k, v, log_decay, state_table, env_ids, done), _linattn_step_plan, q, k, v, log_decay,
                 state_table, env_ids, done, scale)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, linear_attention_step, (q, k, v, log_decay, state_table, env_ids, done), (scale,), out)
    o, = _results(out, plan)
    _check(_lib.sf_linattn_step(plan.address, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), state_table.data_ptr(),
                                state_table.shape[0], _ptr(env_ids), _ptr(done), o, _stream(plan.index)))
    return out


def _linattn_step_plan(q, k, v, log_decay, state_table, env_ids, done, scale):
    torch = binding._torch()
    c = _linattn_config(q, k, v, log_decay, scale, False)
    B, H, dk = q.shape
    _same("state_table", state_table, q, (state_table.shape[0], H, dk, c.dv), torch.float32)
    _optional("env_ids", env_ids, q, (B,), torch.int32)
    _optional("done", done, q, (B,), torch.uint8)
    return _Plan(c, (("o", (B, H, c.dv), q.dtype),), 0, q.device)


def _delta_config(q, k, v, log_decay, beta, scale, steps):
    """steps: the arrays have a time axis in front."""
    if not q.is_cuda:
        _refuse("q is not on the GPU")
    if q.dim() != (4 if steps else 3) or k.dim() != q.dim() or v.dim() != q.dim():
        _refuse("q, k, v: %s, %s, %s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    lead, (Hk, dk) = tuple(q.shape[:-2]), q.shape[-2:]
    H, dv = v.shape[-2:]
    _same("k", k, q, lead + (Hk, dk), dense=False)
    _same("v", v, q, lead + (H, dv), dense=False)
    for name, t in (("log_decay", log_decay), ("beta", beta)):
        _same(name, t, q, lead + (H,), dtype=binding._torch().float32)
    c = SfDeltaruleConfig(C.sizeof(SfDeltaruleConfig), _dtype_of(q), lead[0] if steps else 1, lead[-1], H, Hk, dk, dv,
                          dk ** -0.5 if scale is None else scale)
    for field, name, t in ((c.q_stride, "q", q), (c.k_stride, "k", k), (c.v_stride, "v", v)):
        s = _rows(name, t)
        field[0], field[1], field[2] = s if steps else (0,) + s
    return c


def delta_rule(q, k, v, log_decay, beta, done=None, state0=None, scale=None, out=None, stream=None):
    """The gated delta rule over N trajectories of T steps: q, k [T,N,Hk,dk], v [T,N,H,dv] (bf16 or fp32, last axis dense; keys
    of unit length), log_decay and beta fp32 [T,N,H], done u8 [T,N], state0 fp32 [N,H,dk,dv]; scale: dk ** -0.5.  Results:
    o [T,N,H,dv], state [N,H,dk,dv]."""
    out, scale = {} if out is None else out, _number(scale)
    given = (q, k, v, log_decay, beta, done, state0)
    plan = _plan("delta_rule", scale, given, _delta_plan, *given, scale)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, delta_rule, given, (scale,), out)
    o, state = _results(out, plan)
    _check(_lib.sf_deltarule(plan.address, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), beta.data_ptr(), _ptr(done),
                             _ptr(state0), o, state, _workspace(out, plan), _stream(plan.index)))
    return out


def _delta_plan(q, k, v, log_decay, beta, done, state0, scale):
    torch = binding._torch()
    c = _delta_config(q, k, v, log_decay, beta, scale, True)
    s = (c.N, c.H, c.dk, c.dv)
    _optional("done", done, q, (c.T, c.N), torch.uint8)
    _optional("state0", state0, q, s, torch.float32)
    return _Plan(c, (("o", (c.T, c.N, c.H, c.dv), q.dtype), ("state", s, torch.float32)),
                 _lib.sf_deltarule_workspace_bytes(C.addressof(c), 0), q.device)


def delta_rule_backward(q, k, v, log_decay, beta, do, done=None, state0=None, dstate=None, scale=None, out=None, stream=None):
    """Gradients of delta_rule with the same arguments, given those of o (do) and of the final state (dstate, or None).  Results:
    dq, dk, dv, dlog_decay, dbeta, dstate0."""
    out, scale = {} if out is None else out, _number(scale)
    given = (q, k, v, log_decay, beta, do, done, state0, dstate)
    plan = _plan("delta_rule_backward", scale, given, _delta_back_plan, *given, scale)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, delta_rule_backward, given, (scale,), out)
    dq, dk, dv, dld, dbeta, ds0 = _results(out, plan)
    _check(_lib.sf_deltarule_backward(plan.address, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), beta.data_ptr(), do.data_ptr(),
                                      _ptr(done), _ptr(state0), _ptr(dstate), dq, dk, dv, dld, dbeta, ds0, _workspace(out, plan),
                                      _stream(plan.index)))
    return out


def _delta_back_plan(q, k, v, log_decay, beta, do, done, state0, dstate, scale):
    torch = binding._torch()
    c = _delta_config(q, k, v, log_decay, beta, scale, True)
    s, f32 = (c.N, c.H, c.dk, c.dv), torch.float32
    _same("do", do, q, (c.T, c.N, c.H, c.dv), dense=False)
    c.do_stride[0], c.do_stride[1], c.do_stride[2] = _rows("do", do)
    _optional("done", done, q, (c.T, c.N), torch.uint8)
    _optional("state0", state0, q, s, f32)
    _optional("dstate", dstate, q, s, f32)
    return _Plan(c, (("dq", q.shape, q.dtype), ("dk", q.shape, q.dtype), ("dv", v.shape, q.dtype), ("dlog_decay", log_decay.shape, f32),
                     ("dbeta", beta.shape, f32), ("dstate0", s, f32)), _lib.sf_deltarule_workspace_bytes(C.addressof(c), 1), q.device)


def delta_rule_step(q, k, v, log_decay, beta, state_table, env_ids=None, done=None, scale=None, out=None, stream=None):
    """One step of B environments: q, k [B,Hk,dk], v [B,H,dv], log_decay and beta fp32 [B,H], done u8 [B]; state_table fp32
    [n_env,H,dk,dv] is read and overwritten at the rows env_ids (i32 [B], distinct; None: rows 0 .. B-1).  Result: o [B,H,dv]."""
    out, scale = {} if out is None else out, _number(scale)
    given = (q, k, v, log_decay, beta, state_table, env_ids, done)
    plan = _plan("delta_rule_step", scale, given, _delta_step_plan, *given, scale)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, delta_rule_step, given, (scale,), out)
    o, = _results(out, plan)
    _check(_lib.sf_deltarule_step(plan.address, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), beta.data_ptr(),
                                  state_table.data_ptr(), state_table.shape[0], _ptr(env_ids), _ptr(done), o, _stream(plan.index)))
    return out


def _delta_step_plan(q, k, v, log_decay, beta, state_table, env_ids, done, scale):
    torch = binding._torch()
    c = _delta_config(q, k, v, log_decay, beta, scale, False)
    _same("state_table", state_table, q, (state_table.shape[0], c.H, c.dk, c.dv), torch.float32)
    _optional("env_ids", env_ids, q, (c.N,), torch.int32)
    _optional("done", done, q, (c.N,), torch.uint8)
    return _Plan(c, (("o", (c.N, c.H, c.dv), q.dtype),), 0, q.device)


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
    """The configuration, and b as rows."""
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
    for n, t in (("post_w", post_w), ("scale", scale), ("pre_w", pre_w)):
        _optional(n, t, b, (D,), f32)
    c = SfResnormConfig(C.sizeof(SfResnormConfig), _dtype_of(b), M, D, groups, _NORMS[post], _NORMS[pre], _GATES[gate_act], eps,
                        b.stride(0), 0 if x is None else x.stride(0), 0 if gate is None else gate.stride(0), 0, 0)
    return c, b


def residual_norm(b, x=None, gate=None, post="rms", pre="rms", post_w=None, pre_w=None, scale=None, groups=1, gate_act="none",
                  eps=1e-6, out=None, stream=None):
    """y = x + scale * act(gate) * N_post(b) * post_w and n = N_pre(y) * pre_w over rows [..., D] (bf16 or fp32, last axis
    dense; weights fp32 [D]).  post, pre: "none", "rms" or "layer"; gate_act: "none", "sigmoid" or "silu"; groups: of
    channels that post is taken over (pre "none" then).  Results: y and, with pre, n."""
    out = {} if out is None else out
    how = (post, pre, groups, gate_act, _number(eps))
    plan = _plan("residual_norm", how, (b, x, gate, post_w, pre_w, scale), _resnorm_plan, b, x, gate, post_w, pre_w, scale, how)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, residual_norm, (b, x, gate), (post, pre, post_w, pre_w, scale, groups, gate_act, eps), out)
    got = _results(out, plan)
    _check(_lib.sf_resnorm(plan.address, b.data_ptr(), _ptr(x), _ptr(gate), _ptr(post_w), _ptr(scale), _ptr(pre_w), got[0],
                           got[1] if len(got) > 1 else None, _stream(plan.index)))
    return out


def _resnorm_plan(b, x, gate, post_w, pre_w, scale, how):
    c, _ = _resnorm_config(b, x, gate, *how[:2], post_w, pre_w, scale, *how[2:])
    return _Plan(c, [(n, b.shape, b.dtype) for n in (("y", "n") if c.pre else ("y",))], 0, b.device)


def residual_norm_backward(b, dy, dn=None, x=None, gate=None, post="rms", pre="rms", post_w=None, pre_w=None, scale=None, groups=1,
                           gate_act="none", eps=1e-6, out=None, stream=None):
    """Gradients of residual_norm with the same arguments, given those of y (None: zero) and, with pre, of n.  Results: db and,
    for what was given, dx, dgate, dpost_w, dscale, dpre_w (fp32)."""
    out = {} if out is None else out
    how = (post, pre, groups, gate_act, _number(eps))
    given = (b, x, gate, post_w, scale, pre_w)
    plan = _plan("residual_norm_backward", how, (dy, dn) + given, _resnorm_back_plan, dy, dn, given, how)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, residual_norm_backward, (b, dy, dn, x, gate), (post, pre, post_w, pre_w, scale, groups, gate_act, eps), out)
    got = _results(out, plan)
    db, dx, dgate, dpost_w, dscale, dpre_w = got if len(got) == 6 else _spread(got, given)
    _check(_lib.sf_resnorm_backward(plan.address, b.data_ptr(), _ptr(x), _ptr(gate), _ptr(post_w), _ptr(scale), _ptr(pre_w), _ptr(dy), _ptr(dn),
                                    dx, db, dgate, dpost_w, dscale, dpre_w, _workspace(out, plan), _stream(plan.index)))
    return out


def _spread(got, given):
    """The results' addresses at the places of what was given."""
    got = iter(got)
    return [None if t is None else next(got) for t in given]


def _resnorm_back_plan(dy, dn, given, how):
    b, x, gate, post_w, scale, pre_w = given
    c, rows = _resnorm_config(b, x, gate, *how[:2], post_w, pre_w, scale, *how[2:])
    if dn is None and c.pre:
        _refuse("dn is wanted with pre = %r" % how[1])
    if dy is None and not c.pre:
        _refuse("dy is wanted")
    if dy is not None:
        c.dy_stride = _flat("dy", dy, rows).stride(0)
    if dn is not None:
        c.dn_stride = _flat("dn", dn, rows).stride(0)
    f32, names = binding._torch().float32, ("db", "dx", "dgate", "dpost_w", "dscale", "dpre_w")
    results = [(n, b.shape if i < 3 else (c.D,), b.dtype if i < 3 else f32) for i, (n, t) in enumerate(zip(names, given)) if t is not None]
    n_bytes = _lib.sf_resnorm_workspace_bytes(C.addressof(c))
    return _Plan(c, results, n_bytes if n_bytes < 0 or any(t is not None for t in given[3:]) else 0, b.device)


_ACTS = {"silu": 0, "gelu": 1, "sigmoid": 2}


def _ffn_config(x, w_gate, w_up, w_down, act):
    """The configuration, and x as rows."""
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
    plan = _plan("gated_ffn", act, (x, w_gate, w_up, w_down), _ffn_plan, x, w_gate, w_up, w_down, act)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, gated_ffn, (x, w_gate, w_up, w_down), (act,), out)
    y, = _results(out, plan)
    _check(_lib.sf_ffn(plan.address, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), y, _workspace(out, plan),
                       _stream(plan.index)))
    return out


def _ffn_plan(x, w_gate, w_up, w_down, act):
    c, _ = _ffn_config(x, w_gate, w_up, w_down, act)
    return _Plan(c, (("y", x.shape, x.dtype),), _lib.sf_ffn_workspace_bytes(C.addressof(c), 0), x.device)


def gated_ffn_backward(x, w_gate, w_up, w_down, dy, act="silu", out=None, stream=None):
    """Gradients of gated_ffn with the same arguments, given that of y.  Results: dx, dw_gate, dw_up, dw_down."""
    out = {} if out is None else out
    plan = _plan("gated_ffn_backward", act, (x, w_gate, w_up, w_down, dy), _ffn_back_plan, x, w_gate, w_up, w_down, dy, act)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, gated_ffn_backward, (x, w_gate, w_up, w_down, dy), (act,), out)
    dx, dwg, dwu, dwd = _results(out, plan)
    _check(_lib.sf_ffn_backward(plan.address, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), dy.data_ptr(), dx, dwg, dwu, dwd,
                                _workspace(out, plan), _stream(plan.index)))
    return out


def _ffn_back_plan(x, w_gate, w_up, w_down, dy, act):
    c, rows = _ffn_config(x, w_gate, w_up, w_down, act)
    c.dy_stride = _flat("dy", dy, rows).stride(0)
    return _Plan(c, [(n, s, x.dtype) for n, s in (("dx", x.shape), ("dw_gate", (c.F, c.D)), ("dw_up", (c.F, c.D)), ("dw_down", (c.D, c.F)))],
                 _lib.sf_ffn_workspace_bytes(C.addressof(c), 1), x.device)


def _dense(t):
    """Whether a tensor's elements fill its memory, in whatever order of its axes (those of one without elements do)."""
    if t.numel() == 0:
        return True
    size = 1
    for stride, n in sorted((stride, n) for stride, n in zip(t.stride(), t.shape) if n != 1):
        if stride != size:
            return False
        size *= n
    return True


_tensor_facts = None  # of a list's tensors, by functions that map() calls (a list may have hundreds)


def _list_key(name, tensors):
    """What a list of gradients is: the device's index, shapes and types; their strides where tensors are not contiguous."""
    global _tensor_facts
    if _tensor_facts is None:
        T = binding._torch().Tensor
        _tensor_facts = T.get_device, operator.attrgetter("shape"), operator.attrgetter("dtype"), T.is_contiguous
    device, shape, dtype, contiguous = _tensor_facts
    try:
        where = set(map(device, tensors))
        shapes, types = list(map(shape, tensors)), list(map(dtype, tensors))
        strides = None if all(map(contiguous, tensors)) else [None if contiguous(t) else t.stride() for t in tensors]
    except TypeError:
        _refuse("%s: a list of tensors is wanted" % name)
    if len(where) != 1 or min(where) < 0:
        _refuse("%s: %s, tensors on one GPU are wanted" % (name, "an empty list" if not where else "on %s" % ", ".join(
            "the CPU" if i < 0 else "cuda:%d" % i for i in sorted(where))))
    return [where, shapes, types, strides]


class _ListPlan(_Plan):
    __slots__ = ("sizes", "types")


def clip_gradients(grads, max_norm, eps=1e-6, in_place=True, out=None, stream=None):
    """The global norm of a list of gradients (at least one; bf16 or fp32 or both, dense in any order of their axes), and the gradients times
    min(1, max_norm / (norm + eps)): in place, or in_place=False as results.  Results: norm, fp32 [1], before clipping, and unless
    in place grads, a list of tensors like the ones given."""
    out, max_norm, eps = {} if out is None else out, _number(max_norm), _number(eps)
    grads = grads if type(grads) is list else list(grads)
    key = _list_key("grads", grads)
    plan = _last.get("clip_gradients")
    if plan is None or plan.key != key:
        plan = _last["clip_gradients"] = _clip_plan(grads, key)
    if stream is not None or plan.index != _current_device():
        return _elsewhere(stream, plan, clip_gradients, (grads,), (max_norm, eps, in_place), out)
    torch = binding._torch()
    data_ptr = torch.Tensor.data_ptr
    norm, = _results(out, plan)
    pointers = array.array("Q", map(data_ptr, grads))
    results = pointers
    if not in_place:
        to = out.get("grads")
        if to is None:
            to = out["grads"] = [torch.empty_like(g) for g in grads]
        elif len(to) != len(grads) or _list_key("out['grads']", to) != key:
            _refuse("out['grads'] does not fit: %d tensors of the same shapes, types and strides as the gradients are wanted" % len(grads))
        results = array.array("Q", map(data_ptr, to))
    config = SfGradclipConfig(C.sizeof(SfGradclipConfig), len(grads), max_norm, eps)
    _check(_lib.sf_gradclip(C.addressof(config), pointers.buffer_info()[0], plan.sizes, plan.types, results.buffer_info()[0], norm,
                            _workspace(out, plan), _stream(plan.index)))
    return out


def _clip_plan(grads, key):
    load_library()
    types = [_dtype_of(g) for g in grads]
    if key[3] is not None:
        for i, g in enumerate(grads):
            if not _dense(g):
                _refuse("grads[%d] is not dense: %s, strides %s" % (i, tuple(g.shape), g.stride()))
    n = len(grads)
    sizes = (C.c_int64 * n)(*(shape.numel() for shape in key[1]))
    plan = _ListPlan(SfGradclipConfig(), (("norm", (1,), binding._torch().float32),), _lib.sf_gradclip_workspace_bytes(n, sizes), grads[0].device)
    plan.key, plan.sizes, plan.types = key, sizes, (C.c_int32 * n)(*types)
    return plan
