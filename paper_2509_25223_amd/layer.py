"""The operators around a mixing layer (include/rla_layer.h): the short causal
convolution, the selective state-space scan, the residual addition with the norm
before a block and the gated norm after one.

As in the package's other functions, names are the C ABI's, arguments are
checked and marshalled here and every step runs in the library's HIP kernels.
Activations are bf16 or fp32, [B, T, ...] or packed [T, ...] with cu_seqlens (int32
[N + 1], device); their rows may lie further apart than they are wide (slices
of a projection), every other tensor is contiguous.  Parameters, their gradients
and the scan's states are fp32.  Outputs and workspaces are allocated (on
`stream`, if given) unless passed in.  A call runs on its tensors' GPU, whichever
is the current one; a stream has to be that GPU's.
"""
from __future__ import annotations

import ctypes
import functools

from . import RLA_BF16, RLA_F32, RLA_OK, RLAError, load_library

torch = None   # imported with the library, on the first call

RLA_SSM_FORWARD, RLA_SSM_BACKWARD = 0, 1

LAYER_SYMBOLS = ("rla_conv_workspace_size", "rla_conv_forward", "rla_conv_backward", "rla_conv_decode",
                 "rla_ssm_workspace_size", "rla_ssm_forward", "rla_ssm_backward", "rla_ssm_decode",
                 "rla_addnorm_workspace_size", "rla_addnorm_forward", "rla_addnorm_backward",
                 "rla_gatenorm_workspace_size", "rla_gatenorm_forward", "rla_gatenorm_backward")

_i64, _i32, _vp, _f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float


class rla_conv_problem(ctypes.Structure):
    _fields_ = [("batch", _i64), ("seq_len", _i64), ("channels", _i64), ("num_seqs", _i64),
                ("cu_seqlens", _vp), ("x_stride", _i64), ("dy_stride", _i64), ("taps", _i32), ("silu", _i32),
                ("dtype", _i32)]


class rla_ssm_problem(ctypes.Structure):
    _fields_ = [("batch", _i64), ("seq_len", _i64), ("channels", _i64), ("states", _i64), ("groups", _i64),
                ("num_seqs", _i64), ("cu_seqlens", _vp), ("u_stride", _i64), ("delta_stride", _i64),
                ("z_stride", _i64), ("do_stride", _i64), ("b_stride", _i64), ("c_stride", _i64),
                ("softplus", _i32), ("dtype", _i32)]


class rla_addnorm_problem(ctypes.Structure):
    _fields_ = [("rows", _i64), ("width", _i64), ("x_stride", _i64), ("dn_stride", _i64), ("dtype", _i32),
                ("residual_dtype", _i32), ("eps", _f32)]


class rla_gatenorm_problem(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("heads", _i64), ("width", _i64), ("x_stride", _i64), ("gate_stride", _i64),
                ("do_stride", _i64), ("dtype", _i32), ("x_dtype", _i32), ("gate_first", _i32),
                ("weight_per_head", _i32), ("eps", _f32)]


# pointer arguments between the problem and the trailing (workspace, bytes,) stream
_ARGS = {"rla_conv_forward": (6, True), "rla_conv_backward": (10, True), "rla_conv_decode": (6, False),
         "rla_addnorm_forward": (6, False), "rla_addnorm_backward": (10, True),
         "rla_gatenorm_forward": (4, False), "rla_gatenorm_backward": (7, True)}
_PROBLEMS = {"conv": rla_conv_problem, "ssm": rla_ssm_problem, "addnorm": rla_addnorm_problem,
             "gatenorm": rla_gatenorm_problem}


_bound = _stream_of = _current = None


def _lib():
    """The library with this header's functions typed."""
    global _bound, torch, _stream_of, _current
    if _bound is not None:
        return _bound
    import torch as module
    torch = module
    _stream_of = torch._C._cuda_getCurrentRawStream   # of a device, without its object
    _current = torch._C._cuda_getDevice
    lib = load_library()
    for op, problem in _PROBLEMS.items():
        size = getattr(lib, "rla_%s_workspace_size" % op)
        size.argtypes = [ctypes.POINTER(problem)] + ([ctypes.c_int] if op in ("conv", "ssm") else [])
        size.restype = ctypes.c_size_t
        for name, (n, ws) in _ARGS.items():
            if name.startswith("rla_%s_" % op):
                f = getattr(lib, name)
                f.argtypes = [ctypes.POINTER(problem)] + [_vp] * n + ([_vp, ctypes.c_size_t] if ws else []) + [_vp]
                f.restype = ctypes.c_int
    pp = ctypes.POINTER(rla_ssm_problem)
    lib.rla_ssm_forward.argtypes = [pp] + [_vp] * 11 + [ctypes.c_int, _vp, ctypes.c_size_t, _vp]
    lib.rla_ssm_backward.argtypes = [pp] + [_vp] * 20 + [ctypes.c_int, _vp, ctypes.c_size_t, _vp]
    lib.rla_ssm_decode.argtypes = [pp] + [_vp] * 12
    for name in ("rla_ssm_forward", "rla_ssm_backward", "rla_ssm_decode"):
        getattr(lib, name).restype = ctypes.c_int
    _bound = lib
    return lib


# ---------------------------------------------------------------------------
# checks.  A call of a few tokens is bound by the host, so each tensor is looked at
# once, cheaply; the checks that name what is wrong run where that look fails.
# ---------------------------------------------------------------------------

def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream_handle(stream, index):
    if stream is None:
        return _stream_of(index)
    if stream.device_index != index:
        raise ValueError("stream must be on GPU %d" % index)
    return stream.cuda_stream


def _elsewhere(call, index):
    """`call` with GPU `index` the current one, as it has to be where its tensors are
    there: kernels run on the current device, and a default stream's handle (0) is
    that device's."""
    def on_it(*args):
        with torch.cuda.device(index):
            return call(*args)
    return on_it


def _code(name, dt):
    if dt is torch.bfloat16:
        return RLA_BF16
    if dt is torch.float32:
        return RLA_F32
    raise TypeError("%s must be bfloat16 or float32, got %s" % (name, dt))


def _device(name, t):
    index = t.get_device()
    if index < 0:
        raise ValueError("%s must be on a GPU" % name)
    return index


def _need(**given):
    for name, t in given.items():
        if t is None:
            raise ValueError("%s is required" % name)


def _check(name, t, index, shape, dtype):
    """A contiguous tensor of exactly this device, shape and type (None passes)."""
    if t is None or (t.shape == shape and t.dtype is dtype and t.get_device() == index and t.is_contiguous()):
        return
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.get_device() != index:
        raise ValueError("%s must be on GPU %d" % (name, index))
    raise ValueError("%s must be contiguous" % name)


def _rows(name, t, index, shape, lead, dtype):
    """Elements between the rows of an activation whose first `lead` dimensions are
    tokens (0: next to each other).  Rows themselves are contiguous, and evenly
    spaced over all tokens."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        if t.shape != shape:
            raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
        if t.dtype is not dtype:
            raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
        raise ValueError("%s must be on GPU %d" % (name, index))
    if t.is_contiguous():
        return 0
    stride, width = t.stride(), 1
    for d in range(len(shape) - 1, lead - 1, -1):
        if shape[d] != 1 and stride[d] != width:
            raise ValueError("%s: a token's values must be contiguous" % name)
        width *= shape[d]
    step, rows = 0, 1
    for d in range(lead - 1, -1, -1):
        if shape[d] == 1:
            continue
        if rows == 1:
            step = stride[d]
        elif stride[d] != step * rows:
            raise ValueError("%s: tokens must be evenly spaced" % name)
        rows *= shape[d]
    if rows > 1 and step < width:
        raise ValueError("%s: tokens must not overlap" % name)
    return step


# problems by their sizes (never changed after): building one costs as much as passing it
_conv_problem = functools.lru_cache(256)(rla_conv_problem)
_ssm_problem = functools.lru_cache(256)(rla_ssm_problem)
_addnorm_problem = functools.lru_cache(256)(rla_addnorm_problem)
_gatenorm_problem = functools.lru_cache(256)(rla_gatenorm_problem)


def _cu(cu_seqlens, index, lead):
    """(pointer, N) of packed sequences."""
    if cu_seqlens is None:
        return None, 0
    if len(lead) == 2 and lead[0] != 1:
        raise ValueError("cu_seqlens requires packed tokens")
    if cu_seqlens.dtype is not torch.int32 or cu_seqlens.get_device() != index:
        raise TypeError("cu_seqlens must be an int32 tensor on GPU %d" % index)
    if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1 or not cu_seqlens.is_contiguous():
        raise ValueError("cu_seqlens must be contiguous [N + 1]")
    return cu_seqlens.data_ptr(), cu_seqlens.numel() - 1


def _tokens(name, t, inner):
    """(B, T, leading shape) of activations with `inner` dimensions per token."""
    lead = t.shape[:t.dim() - inner]
    if len(lead) == 2:
        return lead[0], lead[1], lead
    if len(lead) == 1:
        return 1, lead[0], lead
    raise ValueError("%s must be [B, T, ...] or [T, ...]" % name)


def _new(like, shape, dtype, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):   # memory of the stream that uses it
        return torch.empty(shape, dtype=dtype, device=like.device)


def _space(like, need, workspace, stream):
    if workspace is None:
        workspace = _new(like, max(need, 1), torch.uint8, stream)
    elif workspace.get_device() != like.get_device() or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous and on %s" % like.device)
    have = workspace.numel() * workspace.element_size()
    if have < need:
        raise ValueError("workspace too small: need %d bytes" % need)
    return workspace, have


def _ok(status, name):
    if status != RLA_OK:
        raise RLAError(status, name)


def _gradients(grads, index, expected):
    """Caller-supplied gradient buffers: every one of `expected`, nothing else."""
    for key in grads:
        if key not in expected:
            raise ValueError("unknown gradient %r" % key)
    for key, (shape, dtype) in expected.items():
        if grads.get(key) is None:
            raise ValueError("grads[%r] is required" % key)
        _check("grads[%s]" % key, grads[key], index, shape, dtype)


# ---------------------------------------------------------------------------
# short causal convolution
# ---------------------------------------------------------------------------

def _conv(x, weight, bias, silu, cu_seqlens, dy=None):
    if x is None or weight is None:
        _need(x=x, weight=weight)
    index = _device("x", x)
    B, T, lead = _tokens("x", x, 1)
    D = x.shape[-1]
    dtype = _code("x", x.dtype)
    if weight.dim() != 2 or not 2 <= weight.shape[1] <= 4:
        raise ValueError("weight must be [%d, taps], 2 to 4 taps" % D)
    taps = weight.shape[1]
    _check("weight", weight, index, (D, taps), torch.float32)
    _check("bias", bias, index, (D,), torch.float32)
    cu, n = _cu(cu_seqlens, index, lead)
    xs = _rows("x", x, index, x.shape, len(lead), x.dtype)
    ds = _rows("dy", dy, index, x.shape, len(lead), x.dtype)
    make = _conv_problem if cu is None else rla_conv_problem
    problem = make(B, T, D, n, cu, xs, ds, taps, 1 if silu else 0, dtype)
    return problem, index, ((B if cu is None else n), taps - 1, D)


def make_conv_problem(x, weight, cu_seqlens=None, silu=False) -> rla_conv_problem:
    """rla_conv_problem for x [B, T, D] / [T, D] and weight [D, taps]."""
    _lib()
    return rla_conv_problem.from_buffer_copy(_conv(x, weight, None, silu, cu_seqlens)[0])


def rla_conv_workspace_size(problem: rla_conv_problem, backward: bool = True) -> int:
    return int(_lib().rla_conv_workspace_size(problem, 1 if backward else 0))


def rla_conv_forward(x, weight, bias=None, silu=False, state=None, cu_seqlens=None, out=None, state_final=None,
                     return_state=True, workspace=None, stream=None):
    """Causal depthwise convolution of x [B, T, D] / [T, D] with weight [D, taps]
    (taps 2 to 4), the last tap on the token itself, then SiLU with `silu`.
    state [N, taps - 1, D]: the inputs before each sequence, oldest first
    (None: zeros).  Returns (y, state_final); the final state is None without
    return_state."""
    lib = _lib()
    problem, index, shape = _conv(x, weight, bias, silu, cu_seqlens)
    _check("state", state, index, shape, x.dtype)
    _check("out", out, index, x.shape, x.dtype)
    _check("state_final", state_final, index, shape, x.dtype)
    if out is None:
        out = _new(x, x.shape, x.dtype, stream)
    if state_final is None and return_state:
        state_final = _new(x, shape, x.dtype, stream)
    ws, have = None, 0
    if cu_seqlens is not None:
        ws, have = _space(x, lib.rla_conv_workspace_size(problem, 0), workspace, stream)
    call = lib.rla_conv_forward if _current() == index else _elsewhere(lib.rla_conv_forward, index)
    _ok(call(problem, x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(state), out.data_ptr(), _ptr(state_final),
             _ptr(ws), have, _stream_handle(stream, index)), "rla_conv_forward")
    return out, state_final


def rla_conv_backward(x, weight, dy, bias=None, silu=False, state=None, dstate_final=None, cu_seqlens=None,
                      grads=None, workspace=None, stream=None):
    """Gradients of <dy, y> + <dstate_final, state_final> for rla_conv_forward:
    a dict of dx, dweight, dbias (with a bias) and dstate (with a state)."""
    lib = _lib()
    problem, index, shape = _conv(x, weight, bias, silu, cu_seqlens, dy)
    if dy is None:
        raise ValueError("dy is required")
    _check("state", state, index, shape, x.dtype)
    _check("dstate_final", dstate_final, index, shape, x.dtype)
    expected = {"dx": (x.shape, x.dtype), "dweight": (weight.shape, torch.float32)}
    if bias is not None:
        expected["dbias"] = (bias.shape, torch.float32)
    if state is not None:
        expected["dstate"] = (shape, x.dtype)
    if grads is None:
        grads = {key: _new(x, s, dt, stream) for key, (s, dt) in expected.items()}
    else:
        _gradients(grads, index, expected)
    ws, have = _space(x, lib.rla_conv_workspace_size(problem, 1), workspace, stream)
    call = lib.rla_conv_backward if _current() == index else _elsewhere(lib.rla_conv_backward, index)
    _ok(call(problem, x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(state), dy.data_ptr(), _ptr(dstate_final),
             grads["dx"].data_ptr(), grads["dweight"].data_ptr(), _ptr(grads.get("dbias")), _ptr(grads.get("dstate")),
             ws.data_ptr(), have, _stream_handle(stream, index)), "rla_conv_backward")
    return grads


def rla_conv_decode(x, weight, bias=None, silu=False, state=None, state_out=None, out=None, stream=None):
    """A few new tokens x [B, T, D] onto the sequences' states [B, taps - 1, D]
    (None: zeros).  Returns (y, state_out); state_out=state updates in place."""
    lib = _lib()
    if x is not None and x.dim() != 3:
        raise ValueError("x must be [B, T, D]")
    problem, index, shape = _conv(x, weight, bias, silu, None)
    _check("state", state, index, shape, x.dtype)
    _check("state_out", state_out, index, shape, x.dtype)
    _check("out", out, index, x.shape, x.dtype)
    if out is None:
        out = _new(x, x.shape, x.dtype, stream)
    if state_out is None:
        state_out = _new(x, shape, x.dtype, stream)
    call = lib.rla_conv_decode if _current() == index else _elsewhere(lib.rla_conv_decode, index)
    _ok(call(problem, x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(state), out.data_ptr(), state_out.data_ptr(),
             _stream_handle(stream, index)), "rla_conv_decode")
    return out, state_out


# ---------------------------------------------------------------------------
# selective state-space scan
# ---------------------------------------------------------------------------

def _ssm(u, delta, A, B, C, D, z, delta_bias, softplus, cu_seqlens, dO=None):
    if u is None or delta is None or A is None or B is None or C is None:
        _need(u=u, delta=delta, A=A, B=B, C=C)
    index = _device("u", u)
    nb, T, lead = _tokens("u", u, 1)
    width, k, dt = u.shape[-1], len(lead), u.dtype
    dtype = _code("u", dt)
    if A.dim() != 2:
        raise ValueError("A must be [%d, states]" % width)
    states = A.shape[1]
    if not 1 <= states <= 64:
        raise ValueError("A must have 1 to 64 states, got %d" % states)
    _check("A", A, index, (width, states), torch.float32)
    # B, C: [..., G, states], or [..., states] for one group
    if B.dim() not in (k + 1, k + 2):
        raise ValueError("B must be [..., states] or [..., groups, states]")
    groups = B.shape[k] if B.dim() == k + 2 else 1
    if groups < 1 or width % groups:
        raise ValueError("B: %d channels are no multiple of %d groups" % (width, groups))
    shape = tuple(lead) + ((groups, states) if B.dim() == k + 2 else (states,))
    us = _rows("u", u, index, u.shape, k, dt)
    ds = _rows("delta", delta, index, u.shape, k, dt)
    bs = _rows("B", B, index, shape, k, dt)
    cs = _rows("C", C, index, shape, k, dt)
    zs = _rows("z", z, index, u.shape, k, dt)
    os_ = _rows("dO", dO, index, u.shape, k, dt)
    _check("D", D, index, (width,), torch.float32)
    _check("delta_bias", delta_bias, index, (width,), torch.float32)
    cu, n = _cu(cu_seqlens, index, lead)
    make = _ssm_problem if cu is None else rla_ssm_problem
    problem = make(nb, T, width, states, groups, n, cu, us, ds, zs, os_, bs, cs, 1 if softplus else 0, dtype)
    return problem, index, ((nb if cu is None else n), width, states)


def make_ssm_problem(u, A, B, cu_seqlens=None, softplus=True) -> rla_ssm_problem:
    """rla_ssm_problem for u [B, T, D] / [T, D], A [D, states] and B [..., groups,
    states] (sizes only: what a workspace depends on)."""
    _lib()
    return rla_ssm_problem.from_buffer_copy(_ssm(u, u, A, B, B, None, None, None, softplus, cu_seqlens)[0])


def rla_ssm_workspace_size(problem: rla_ssm_problem, op: int) -> int:
    return int(_lib().rla_ssm_workspace_size(problem, int(op)))


def rla_ssm_forward(u, delta, A, B, C, D=None, z=None, delta_bias=None, softplus=True, h0=None, cu_seqlens=None,
                    out=None, h_final=None, return_state=True, save_for_backward=False, workspace=None, stream=None):
    """Selective scan of u [.., D] with steps softplus(delta + delta_bias), rates A
    [D, states] (fp32, as used: negative to decay), B and C [.., groups, states] (or
    [.., states]), skip D and gate z: o = (C h + D u) silu(z).  h0, h_final [N, D,
    states] fp32.  Returns (o, h_final).  With save_for_backward the workspace
    (of RLA_SSM_BACKWARD's size) keeps what rla_ssm_backward(use_saved=True) reads."""
    lib = _lib()
    problem, index, shape = _ssm(u, delta, A, B, C, D, z, delta_bias, softplus, cu_seqlens)
    f32 = torch.float32
    _check("h0", h0, index, shape, f32)
    _check("out", out, index, u.shape, u.dtype)
    _check("h_final", h_final, index, shape, f32)
    if save_for_backward and workspace is None:
        raise ValueError("save_for_backward needs a workspace")
    if out is None:
        out = _new(u, u.shape, u.dtype, stream)
    if h_final is None and return_state:
        h_final = _new(u, shape, f32, stream)
    op = RLA_SSM_BACKWARD if save_for_backward else RLA_SSM_FORWARD
    ws, have = _space(u, lib.rla_ssm_workspace_size(problem, op), workspace, stream)
    call = lib.rla_ssm_forward if _current() == index else _elsewhere(lib.rla_ssm_forward, index)
    _ok(call(problem, u.data_ptr(), delta.data_ptr(), A.data_ptr(), B.data_ptr(), C.data_ptr(), _ptr(D), _ptr(z),
             _ptr(delta_bias), _ptr(h0), out.data_ptr(), _ptr(h_final), 1 if save_for_backward else 0, ws.data_ptr(),
             have, _stream_handle(stream, index)), "rla_ssm_forward")
    return out, h_final


def rla_ssm_backward(u, delta, A, B, C, dO, D=None, z=None, delta_bias=None, softplus=True, h0=None, dh_final=None,
                     cu_seqlens=None, grads=None, use_saved=False, workspace=None, stream=None):
    """Gradients of <dO, o> + <dh_final, h_final> for rla_ssm_forward: a dict of
    du, ddelta, dA, dB, dC, and dD, dz, ddelta_bias, dh0 where those inputs are
    given.  use_saved: reads what rla_ssm_forward(save_for_backward=True) left in
    `workspace`."""
    lib = _lib()
    if dO is None:
        raise ValueError("dO is required")
    if use_saved and workspace is None:
        raise ValueError("use_saved needs the workspace of the saving forward call")
    problem, index, shape = _ssm(u, delta, A, B, C, D, z, delta_bias, softplus, cu_seqlens, dO)
    f32 = torch.float32
    _check("h0", h0, index, shape, f32)
    _check("dh_final", dh_final, index, shape, f32)
    expected = {"du": (u.shape, u.dtype), "ddelta": (u.shape, u.dtype), "dA": (A.shape, f32),
                "dB": (B.shape, u.dtype), "dC": (B.shape, u.dtype)}
    if D is not None:
        expected["dD"] = (D.shape, f32)
    if z is not None:
        expected["dz"] = (u.shape, u.dtype)
    if delta_bias is not None:
        expected["ddelta_bias"] = (delta_bias.shape, f32)
    if h0 is not None:
        expected["dh0"] = (shape, f32)
    if grads is None:
        grads = {key: _new(u, s, dt, stream) for key, (s, dt) in expected.items()}
    else:
        _gradients(grads, index, expected)
    ws, have = _space(u, lib.rla_ssm_workspace_size(problem, RLA_SSM_BACKWARD), workspace, stream)
    g = grads
    call = lib.rla_ssm_backward if _current() == index else _elsewhere(lib.rla_ssm_backward, index)
    _ok(call(problem, u.data_ptr(), delta.data_ptr(), A.data_ptr(), B.data_ptr(), C.data_ptr(), _ptr(D), _ptr(z),
             _ptr(delta_bias), _ptr(h0), dO.data_ptr(), _ptr(dh_final), g["du"].data_ptr(), g["ddelta"].data_ptr(),
             g["dA"].data_ptr(), g["dB"].data_ptr(), g["dC"].data_ptr(), _ptr(g.get("dD")), _ptr(g.get("dz")),
             _ptr(g.get("ddelta_bias")), _ptr(g.get("dh0")), 1 if use_saved else 0, ws.data_ptr(), have,
             _stream_handle(stream, index)), "rla_ssm_backward")
    return grads


def rla_ssm_decode(u, delta, A, B, C, D=None, z=None, delta_bias=None, softplus=True, h_in=None, h_out=None,
                   out=None, stream=None):
    """A few new tokens u [B, T, D] onto the states h_in [B, D, states] (None:
    zeros).  Returns (o, h_out); h_out=h_in updates in place."""
    lib = _lib()
    if u is not None and u.dim() != 3:
        raise ValueError("u must be [B, T, D]")
    problem, index, shape = _ssm(u, delta, A, B, C, D, z, delta_bias, softplus, None)
    f32 = torch.float32
    _check("h_in", h_in, index, shape, f32)
    _check("h_out", h_out, index, shape, f32)
    _check("out", out, index, u.shape, u.dtype)
    if out is None:
        out = _new(u, u.shape, u.dtype, stream)
    if h_out is None:
        h_out = _new(u, shape, f32, stream)
    call = lib.rla_ssm_decode if _current() == index else _elsewhere(lib.rla_ssm_decode, index)
    _ok(call(problem, u.data_ptr(), delta.data_ptr(), A.data_ptr(), B.data_ptr(), C.data_ptr(), _ptr(D), _ptr(z),
             _ptr(delta_bias), _ptr(h_in), out.data_ptr(), h_out.data_ptr(), _stream_handle(stream, index)),
        "rla_ssm_decode")
    return out, h_out


# ---------------------------------------------------------------------------
# norms
# ---------------------------------------------------------------------------

def _addnorm(x, residual_dtype, eps, dn=None, name="x"):
    """`x`: the block's output, or (backward without a scale) its stand-in dn."""
    if x is None:
        raise ValueError("%s is required" % name)
    if x.dim() < 1:
        raise ValueError("%s must have rows" % name)
    index = _device(name, x)
    lead = x.dim() - 1
    dtype = _code(name, x.dtype)
    rd = _code("residual_dtype", residual_dtype)
    xs = _rows(name, x, index, x.shape, lead, x.dtype)
    ds = _rows("dn", dn, index, x.shape, lead, x.dtype)
    width = x.shape[-1]
    return _addnorm_problem(x.numel() // width if width else 0, width, xs, ds, dtype, rd, eps), index


def make_addnorm_problem(x, residual_dtype, eps=1e-6) -> rla_addnorm_problem:
    """rla_addnorm_problem for x [.., D] and a residual stream of that type."""
    _lib()
    return rla_addnorm_problem.from_buffer_copy(_addnorm(x, residual_dtype, eps)[0])


def rla_addnorm_workspace_size(problem: rla_addnorm_problem) -> int:
    return int(_lib().rla_addnorm_workspace_size(problem))


def rla_addnorm_forward(x, weight, residual=None, scale=None, eps=1e-6, out=None, residual_out=None,
                        residual_dtype=None, stream=None):
    """The residual stream takes a block's output, and the next block its norm:
    residual_out = residual + scale x, n = RMS(residual_out) weight, over the last
    dimension.  residual None: 0; scale [D] None: 1.  The stream is of residual's
    type (without one: residual_dtype, fp32 by default).  Returns (n, residual_out);
    residual_out=residual updates in place."""
    lib = _lib()
    rd = residual.dtype if residual is not None else residual_out.dtype if residual_out is not None else \
        torch.float32 if residual_dtype is None else residual_dtype
    problem, index = _addnorm(x, rd, eps)
    D = x.shape[-1]
    if weight is None:
        _need(weight=weight)
    _check("weight", weight, index, (D,), torch.float32)
    _check("scale", scale, index, (D,), torch.float32)
    _check("residual", residual, index, x.shape, rd)
    _check("out", out, index, x.shape, x.dtype)
    _check("residual_out", residual_out, index, x.shape, rd)
    if out is None:
        out = _new(x, x.shape, x.dtype, stream)
    if residual_out is None:
        residual_out = _new(x, x.shape, rd, stream)
    call = lib.rla_addnorm_forward if _current() == index else _elsewhere(lib.rla_addnorm_forward, index)
    _ok(call(problem, x.data_ptr(), _ptr(residual), weight.data_ptr(), _ptr(scale), out.data_ptr(),
             residual_out.data_ptr(), _stream_handle(stream, index)), "rla_addnorm_forward")
    return out, residual_out


def rla_addnorm_backward(dn, residual_out, weight, x=None, scale=None, dresidual_out=None, eps=1e-6, grads=None,
                         workspace=None, stream=None):
    """Gradients of <dn, n> + <dresidual_out, residual_out> for rla_addnorm_forward,
    from the stream that it left: a dict of dx, dresidual (of the stream's type),
    dweight, and dscale where scale is given (x is needed then).
    grads["dresidual"] may be dresidual_out."""
    lib = _lib()
    _need(dn=dn, residual_out=residual_out, weight=weight)
    if scale is not None and x is None:
        raise ValueError("x is required with scale")
    rd = residual_out.dtype
    problem, index = _addnorm(dn if x is None else x, rd, eps, dn, "dn" if x is None else "x")
    shape = dn.shape
    D = shape[-1]
    _check("weight", weight, index, (D,), torch.float32)
    _check("scale", scale, index, (D,), torch.float32)
    _check("residual_out", residual_out, index, shape, rd)
    _check("dresidual_out", dresidual_out, index, shape, rd)
    expected = {"dx": (shape, dn.dtype), "dresidual": (shape, rd), "dweight": ((D,), torch.float32)}
    if scale is not None:
        expected["dscale"] = ((D,), torch.float32)
    if grads is None:
        grads = {key: _new(dn, s, dt, stream) for key, (s, dt) in expected.items()}
    else:
        _gradients(grads, index, expected)
    ws, have = _space(dn, lib.rla_addnorm_workspace_size(problem), workspace, stream)
    call = lib.rla_addnorm_backward if _current() == index else _elsewhere(lib.rla_addnorm_backward, index)
    _ok(call(problem, dn.data_ptr(), _ptr(dresidual_out), residual_out.data_ptr(), _ptr(x), weight.data_ptr(),
             _ptr(scale), grads["dx"].data_ptr(), grads["dresidual"].data_ptr(), grads["dweight"].data_ptr(),
             _ptr(grads.get("dscale")), ws.data_ptr(), have, _stream_handle(stream, index)), "rla_addnorm_backward")
    return grads


def _gatenorm(x, gate, weight, gate_first, eps, dO=None):
    if x is None or gate is None or weight is None:
        _need(x=x, gate=gate, weight=weight)
    if x.dim() < 2:
        raise ValueError("x must be [.., heads, width]")
    index = _device("x", x)
    lead = x.dim() - 2
    H, d = x.shape[-2:]
    dtype, xd = _code("gate", gate.dtype), _code("x", x.dtype)
    xs = _rows("x", x, index, x.shape, lead, x.dtype)
    gs = _rows("gate", gate, index, x.shape, lead, gate.dtype)
    ds = _rows("dO", dO, index, x.shape, lead, gate.dtype)
    per_head = weight.dim() == 2
    _check("weight", weight, index, (H, d) if per_head else (d,), torch.float32)
    tokens = x.numel() // (H * d) if H * d else 0
    return _gatenorm_problem(tokens, H, d, xs, gs, ds, dtype, xd, 1 if gate_first else 0, 1 if per_head else 0,
                             eps), index


def make_gatenorm_problem(x, gate, weight, gate_first=False, eps=1e-6) -> rla_gatenorm_problem:
    """rla_gatenorm_problem for x, gate [.., heads, width] and weight [width] or
    [heads, width]."""
    _lib()
    return rla_gatenorm_problem.from_buffer_copy(_gatenorm(x, gate, weight, gate_first, eps)[0])


def rla_gatenorm_workspace_size(problem: rla_gatenorm_problem) -> int:
    return int(_lib().rla_gatenorm_workspace_size(problem))


def rla_gatenorm_forward(x, gate, weight, gate_first=False, eps=1e-6, out=None, stream=None):
    """Gated norm of the heads of a mixer's output x [.., heads, width] (bf16 or fp32;
    with a bf16 gate either): RMS(x) weight silu(gate), or with gate_first
    RMS(x silu(gate)) weight; weight [width], or [heads, width].  Returns o, of
    the gate's type."""
    lib = _lib()
    problem, index = _gatenorm(x, gate, weight, gate_first, eps)
    _check("out", out, index, x.shape, gate.dtype)
    if out is None:
        out = _new(x, x.shape, gate.dtype, stream)
    call = lib.rla_gatenorm_forward if _current() == index else _elsewhere(lib.rla_gatenorm_forward, index)
    _ok(call(problem, x.data_ptr(), gate.data_ptr(), weight.data_ptr(), out.data_ptr(), _stream_handle(stream, index)),
        "rla_gatenorm_forward")
    return out


def rla_gatenorm_backward(dO, x, gate, weight, gate_first=False, eps=1e-6, grads=None, workspace=None, stream=None):
    """Gradients of <dO, o> for rla_gatenorm_forward: a dict of dx (x's type), dgate
    and dweight."""
    lib = _lib()
    if dO is None:
        raise ValueError("dO is required")
    problem, index = _gatenorm(x, gate, weight, gate_first, eps, dO)
    expected = {"dx": (x.shape, x.dtype), "dgate": (x.shape, gate.dtype), "dweight": (weight.shape, weight.dtype)}
    if grads is None:
        grads = {key: _new(x, s, dt, stream) for key, (s, dt) in expected.items()}
    else:
        _gradients(grads, index, expected)
    ws, have = _space(x, lib.rla_gatenorm_workspace_size(problem), workspace, stream)
    call = lib.rla_gatenorm_backward if _current() == index else _elsewhere(lib.rla_gatenorm_backward, index)
    _ok(call(problem, dO.data_ptr(), x.data_ptr(), gate.data_ptr(), weight.data_ptr(), grads["dx"].data_ptr(),
             grads["dgate"].data_ptr(), grads["dweight"].data_ptr(), ws.data_ptr(), have,
             _stream_handle(stream, index)), "rla_gatenorm_backward")
    return grads
