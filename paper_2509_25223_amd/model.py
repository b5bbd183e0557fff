"""The ends of a language model on the mixing layers, and a second recurrent mixer
(include/rla_model.h): embedding lookup, gated linear recurrence, log
probabilities of tokens with entropy and alternatives; each with its gradients.

As in the package's other functions, names are the C ABI's, arguments are
checked and marshalled here and every step runs in the library's HIP kernels.
Activations are bf16 or fp32; their rows may lie further apart than they are wide,
every other tensor is contiguous.  Token ids are int64 or int32.  Parameters,
their gradients, states and statistics are fp32 (an embedding table may be bf16).
Outputs and workspaces are allocated (on `stream`, if given) unless passed
in; a workspace sized for a call serves smaller ones, and outputs lie over no inputs
but where a function says so.  A call runs on its tensors' GPU, whichever is the current one; a stream has
to be that GPU's.
"""
from __future__ import annotations

import ctypes
import functools
import operator

from . import layer as _layer
from .layer import _check, _code, _cu, _device, _elsewhere, _gradients, _need, _new, _ok, _ptr, _rows, _space, _tokens

RLA_GLR_FORWARD, RLA_GLR_BACKWARD = 0, 1
RLA_INDEX_I32, RLA_INDEX_I64 = 0, 1

MODEL_SYMBOLS = ("rla_embed_workspace_size", "rla_embed_forward", "rla_embed_backward",
                 "rla_logprob_workspace_size", "rla_logprob_forward", "rla_logprob_backward",
                 "rla_glr_workspace_size", "rla_glr_forward", "rla_glr_backward", "rla_glr_decode")

_i64, _i32, _vp, _f32, _size = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t


class rla_embed_problem(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("vocab", _i64), ("width", _i64), ("dout_stride", _i64), ("index", _i32),
                ("dtype", _i32), ("table_dtype", _i32), ("scale", _f32)]


class rla_logprob_problem(ctypes.Structure):
    _fields_ = [("rows", _i64), ("vocab", _i64), ("logits_stride", _i64), ("index", _i32), ("dtype", _i32),
                ("top", _i32), ("scale", _f32)]


class rla_glr_problem(ctypes.Structure):
    _fields_ = [("batch", _i64), ("seq_len", _i64), ("channels", _i64), ("num_seqs", _i64), ("cu_seqlens", _vp),
                ("x_stride", _i64), ("r_stride", _i64), ("i_stride", _i64), ("z_stride", _i64), ("do_stride", _i64),
                ("normalize", _i32), ("dtype", _i32)]


_bound = torch = None


def _lib():
    """The library with this header's functions typed."""
    global _bound, torch
    if _bound is not None:
        return _bound
    lib = _layer._lib()
    torch = _layer.torch
    ws = [_vp, _size]
    for op, problem, functions in (
            ("embed", rla_embed_problem, dict(forward=[_vp] * 3, backward=[_vp] * 4 + ws)),
            ("logprob", rla_logprob_problem, dict(forward=[_vp] * 7 + ws, backward=[_vp] * 7)),
            ("glr", rla_glr_problem, dict(forward=[_vp] * 8 + [ctypes.c_int] + ws,
                                          backward=[_vp] * 14 + [ctypes.c_int] + ws, decode=[_vp] * 8))):
        pointer = [ctypes.POINTER(problem)]
        size = getattr(lib, "rla_%s_workspace_size" % op)
        size.argtypes, size.restype = pointer + ([ctypes.c_int] if op == "glr" else []), _size
        for name, args in functions.items():
            f = getattr(lib, "rla_%s_%s" % (op, name))
            f.argtypes, f.restype = pointer + args + [_vp], ctypes.c_int
    _bound = lib
    return lib


def _call(name, index):
    """The C function, run with GPU `index` the current one."""
    f = getattr(_bound, name)
    return f if _layer._current() == index else _elsewhere(f, index)


def _stream(stream, index):
    return _layer._stream_handle(stream, index)


# problems by their sizes (numbers, never changed after): building one costs as much as passing it
_embed_problem = functools.lru_cache(256)(rla_embed_problem)
_logprob_problem = functools.lru_cache(256)(rla_logprob_problem)
_glr_problem = functools.lru_cache(256)(rla_glr_problem)


def _ids(name, t, index, shape=None):
    """The rla_index of contiguous token ids."""
    if t.dtype is not torch.int64 and t.dtype is not torch.int32:
        raise TypeError("%s must be int64 or int32, got %s" % (name, t.dtype))
    _check(name, t, index, t.shape if shape is None else shape, t.dtype)
    return RLA_INDEX_I64 if t.dtype is torch.int64 else RLA_INDEX_I32


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------

def _embed(ids, vocab, width, dtype, table_dtype, scale, dout=None):
    index = _device("ids", ids)
    kind = _ids("ids", ids, index)
    ds = 0 if dout is None else _rows("dout", dout, index, ids.shape + (width,), ids.dim(), dout.dtype)
    return _embed_problem(ids.numel(), vocab, width, ds, kind, dtype, table_dtype, float(scale)), index


def make_embed_problem(ids, table, scale=1.0) -> rla_embed_problem:
    """rla_embed_problem for ids [..] and a table [vocab, width]."""
    _lib()
    code = _code("table", table.dtype)
    return rla_embed_problem.from_buffer_copy(_embed(ids, table.shape[0], table.shape[1], code, code, scale)[0])


def rla_embed_workspace_size(problem: rla_embed_problem) -> int:
    return int(_lib().rla_embed_workspace_size(problem))


def rla_embed_forward(ids, table, scale=1.0, out=None, out_dtype=None, stream=None):
    """Rows scale * table[ids] for ids [..] (int64 or int32) and a table [vocab,
    width], of out's type (without one: out_dtype, by default the table's).  Ids
    outside [0, vocab) give zeros.  Returns out [.., width]."""
    lib = _lib()  # noqa: F841
    if ids is None or table is None:
        _need(ids=ids, table=table)
    if table.dim() != 2:
        raise ValueError("table must be [vocab, width]")
    dt = out.dtype if out is not None else table.dtype if out_dtype is None else out_dtype
    V, D = table.shape
    kind = _code("table", table.dtype)
    problem, index = _embed(ids, V, D, _code("out", dt), kind, scale)
    _check("table", table, index, table.shape, table.dtype)
    shape = ids.shape + (D,)
    _check("out", out, index, shape, dt)
    if out is None:
        out = _new(ids, shape, dt, stream)
    _ok(_call("rla_embed_forward", index)(problem, ids.data_ptr(), table.data_ptr(), out.data_ptr(),
                                          _stream(stream, index)), "rla_embed_forward")
    return out


def rla_embed_backward(ids, dout, vocab, scale=1.0, base=None, dtable=None, workspace=None, stream=None):
    """base (None: 0) plus the table's gradient [vocab, width] (fp32) of <dout, out>
    for rla_embed_forward: sums of dout's rows by id, in the rows' order.
    dtable=base adds in place, and touches the rows of the ids only."""
    lib = _lib()
    if ids is None or dout is None or vocab is None:
        _need(ids=ids, dout=dout, vocab=vocab)
    if dout.dim() != ids.dim() + 1:
        raise ValueError("dout must be [.., width]")
    D, vocab = dout.shape[-1], operator.index(vocab)
    code = _code("dout", dout.dtype)
    problem, index = _embed(ids, vocab, D, code, code, scale, dout)
    _check("base", base, index, (vocab, D), torch.float32)
    _check("dtable", dtable, index, (vocab, D), torch.float32)
    if dtable is None:
        dtable = _new(dout, (vocab, D), torch.float32, stream)
    ws, have = _space(dout, lib.rla_embed_workspace_size(problem), workspace, stream)
    _ok(_call("rla_embed_backward", index)(problem, ids.data_ptr(), dout.data_ptr(), _ptr(base), dtable.data_ptr(),
                                           ws.data_ptr(), have, _stream(stream, index)), "rla_embed_backward")
    return dtable


# ---------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------

def _logprob(logits, targets, top, scale):
    if logits is None:
        raise ValueError("logits is required")
    if logits.dim() < 1:
        raise ValueError("logits must be [.., vocab]")
    index = _device("logits", logits)
    dtype = _code("logits", logits.dtype)
    shape = logits.shape
    V = shape[-1]
    lead = shape[:-1]
    stride = _rows("logits", logits, index, shape, len(lead), logits.dtype)
    kind = RLA_INDEX_I64 if targets is None else _ids("targets", targets, index, lead)
    return _logprob_problem(lead.numel(), V, stride, kind, dtype, top, float(scale)), index, lead


def make_logprob_problem(logits, top=0, scale=1.0) -> rla_logprob_problem:
    """rla_logprob_problem for logits [.., vocab]."""
    _lib()
    return rla_logprob_problem.from_buffer_copy(_logprob(logits, None, operator.index(top), scale)[0])


def rla_logprob_workspace_size(problem: rla_logprob_problem) -> int:
    return int(_lib().rla_logprob_workspace_size(problem))


def rla_logprob_forward(logits, targets=None, scale=1.0, entropy=False, top=0, out=None, lse=None, entropy_out=None,
                        top_logprobs=None, top_ids=None, workspace=None, stream=None):
    """Of the rows z = scale * logits [.., vocab] a dict of
      logprob  z[targets] - lse for targets [..] (None: not computed; a target
               outside [0, vocab) leaves its row out: 0)
      lse      log sum e^z
      entropy  with `entropy`
      top_logprobs, top_ids (int32) [.., top]  the likeliest `top` (up to 64) tokens,
               equal logits by their place; -inf and -1 where fewer have any
    None for what is not asked for.  `out`, `lse`, `entropy_out`, `top_logprobs`,
    `top_ids` are written into if given."""
    lib = _lib()
    top = operator.index(top)
    problem, index, lead = _logprob(logits, targets, top, scale)
    if not 0 <= top <= 64 or top > logits.shape[-1]:
        raise ValueError("top must be 0 to 64, and at most the vocabulary; got %d" % top)
    f32 = torch.float32
    if targets is not None:
        _check("out", out, index, lead, f32)
        if out is None:
            out = _new(logits, lead, f32, stream)
    elif out is not None:
        raise ValueError("targets is required with out")
    _check("lse", lse, index, lead, f32)
    if lse is None:
        lse = _new(logits, lead, f32, stream)
    if entropy or entropy_out is not None:
        _check("entropy_out", entropy_out, index, lead, f32)
        if entropy_out is None:
            entropy_out = _new(logits, lead, f32, stream)
    if top:
        shape = lead + (top,)
        _check("top_logprobs", top_logprobs, index, shape, f32)
        _check("top_ids", top_ids, index, shape, torch.int32)
        if top_logprobs is None:
            top_logprobs = _new(logits, shape, f32, stream)
        if top_ids is None:
            top_ids = _new(logits, shape, torch.int32, stream)
    elif top_logprobs is not None or top_ids is not None:
        raise ValueError("top is required with top_logprobs and top_ids")
    need, ws, have = lib.rla_logprob_workspace_size(problem), None, 0
    if need:
        ws, have = _space(logits, need, workspace, stream)
    _ok(_call("rla_logprob_forward", index)(
        problem, logits.data_ptr(), _ptr(targets), _ptr(out), lse.data_ptr(), _ptr(entropy_out), _ptr(top_logprobs),
        _ptr(top_ids), _ptr(ws), have, _stream(stream, index)), "rla_logprob_forward")
    return {"logprob": out, "lse": lse, "entropy": entropy_out, "top_logprobs": top_logprobs, "top_ids": top_ids}


def rla_logprob_backward(logits, lse, targets=None, dlogprob=None, entropy=None, dentropy=None, scale=1.0, out=None,
                         stream=None):
    """Gradient by the logits of <dlogprob, logprob> + <dentropy, entropy> for
    rla_logprob_forward, from the lse (and, with dentropy, the entropy) that it
    wrote.  out=logits overwrites contiguous logits with it."""
    _lib()
    problem, index, lead = _logprob(logits, targets, 0, scale)
    if lse is None:
        _need(lse=lse)
    f32 = torch.float32
    _check("lse", lse, index, lead, f32)
    if dlogprob is not None:
        if targets is None:
            raise ValueError("targets is required with dlogprob")
        _check("dlogprob", dlogprob, index, lead, f32)
    if dentropy is not None:
        if entropy is None:
            raise ValueError("entropy is required with dentropy")
        _check("dentropy", dentropy, index, lead, f32)
        _check("entropy", entropy, index, lead, f32)
    _check("out", out, index, logits.shape, logits.dtype)
    if out is None:
        out = _new(logits, logits.shape, logits.dtype, stream)
    _ok(_call("rla_logprob_backward", index)(
        problem, logits.data_ptr(), _ptr(targets), lse.data_ptr(), _ptr(entropy), _ptr(dlogprob), _ptr(dentropy),
        out.data_ptr(), _stream(stream, index)), "rla_logprob_backward")
    return out


# ---------------------------------------------------------------------------
# gated linear recurrence
# ---------------------------------------------------------------------------

def _glr(x, r, A, i, z, normalize, cu_seqlens, dO=None):
    if x is None or r is None or A is None:
        _need(x=x, r=r, A=A)
    index = _device("x", x)
    nb, T, lead = _tokens("x", x, 1)
    k, dt, D = len(lead), x.dtype, x.shape[-1]
    dtype = _code("x", dt)
    _check("A", A, index, (D,), torch.float32)
    strides = [_rows(name, t, index, x.shape, k, dt) for name, t in (("x", x), ("r", r), ("i", i), ("z", z), ("dO", dO))]
    cu, n = _cu(cu_seqlens, index, lead)
    make = _glr_problem if cu is None else rla_glr_problem
    return make(nb, T, D, n, cu, *strides, 1 if normalize else 0, dtype), index, ((nb if cu is None else n), D)


def make_glr_problem(x, cu_seqlens=None) -> rla_glr_problem:
    """rla_glr_problem for x [B, T, D] / [T, D] (sizes only: what a workspace
    depends on)."""
    _lib()
    if x is None:
        _need(x=x)
    index = _device("x", x)
    nb, T, lead = _tokens("x", x, 1)
    cu, n = _cu(cu_seqlens, index, lead)
    return rla_glr_problem(nb, T, x.shape[-1], n, cu, 0, 0, 0, 0, 0, 1, _code("x", x.dtype))


def rla_glr_workspace_size(problem: rla_glr_problem, op: int) -> int:
    return int(_lib().rla_glr_workspace_size(problem, int(op)))


def rla_glr_forward(x, r, A, i=None, z=None, normalize=True, h0=None, cu_seqlens=None, out=None, h_final=None,
                    return_state=True, save_for_backward=False, workspace=None, stream=None):
    """Gated linear recurrence of x [B, T, D] / [T, D]: h_t = a_t h_{t-1} + m_t
    sigmoid(i_t) x_t with a_t = exp(A sigmoid(r_t)), A [D] (fp32, as used: negative to
    decay), m_t = sqrt(1 - a_t^2) with normalize, else 1; o = h, or h silu(z).  i
    None: the factor 1.  h0, h_final [N, D] fp32.  Returns (o, h_final).  With
    save_for_backward the workspace (of RLA_GLR_BACKWARD's size) keeps what
    rla_glr_backward(use_saved=True) reads."""
    lib = _lib()
    problem, index, shape = _glr(x, r, A, i, z, normalize, cu_seqlens)
    f32 = torch.float32
    _check("h0", h0, index, shape, f32)
    _check("out", out, index, x.shape, x.dtype)
    _check("h_final", h_final, index, shape, f32)
    if save_for_backward and workspace is None:
        raise ValueError("save_for_backward needs a workspace")
    if out is None:
        out = _new(x, x.shape, x.dtype, stream)
    if h_final is None and return_state:
        h_final = _new(x, shape, f32, stream)
    op = RLA_GLR_BACKWARD if save_for_backward else RLA_GLR_FORWARD
    ws, have = _space(x, lib.rla_glr_workspace_size(problem, op), workspace, stream)
    _ok(_call("rla_glr_forward", index)(
        problem, x.data_ptr(), r.data_ptr(), A.data_ptr(), _ptr(i), _ptr(z), _ptr(h0), out.data_ptr(), _ptr(h_final),
        1 if save_for_backward else 0, ws.data_ptr(), have, _stream(stream, index)), "rla_glr_forward")
    return out, h_final


def rla_glr_backward(x, r, A, dO, i=None, z=None, normalize=True, h0=None, dh_final=None, cu_seqlens=None, grads=None,
                     use_saved=False, workspace=None, stream=None):
    """Gradients of <dO, o> + <dh_final, h_final> for rla_glr_forward: a dict of dx,
    dr, dA, and di, dz, dh0 where those inputs are given.  use_saved: reads what
    rla_glr_forward(save_for_backward=True) left in `workspace`."""
    lib = _lib()
    if dO is None:
        raise ValueError("dO is required")
    if use_saved and workspace is None:
        raise ValueError("use_saved needs the workspace of the saving forward call")
    problem, index, shape = _glr(x, r, A, i, z, normalize, cu_seqlens, dO)
    f32 = torch.float32
    _check("h0", h0, index, shape, f32)
    _check("dh_final", dh_final, index, shape, f32)
    expected = {"dx": (x.shape, x.dtype), "dr": (x.shape, x.dtype), "dA": (A.shape, f32)}
    if i is not None:
        expected["di"] = (x.shape, x.dtype)
    if z is not None:
        expected["dz"] = (x.shape, x.dtype)
    if h0 is not None:
        expected["dh0"] = (shape, f32)
    if grads is None:
        grads = {key: _new(x, s, dt, stream) for key, (s, dt) in expected.items()}
    else:
        _gradients(grads, index, expected)
    ws, have = _space(x, lib.rla_glr_workspace_size(problem, RLA_GLR_BACKWARD), workspace, stream)
    g = grads
    _ok(_call("rla_glr_backward", index)(
        problem, x.data_ptr(), r.data_ptr(), A.data_ptr(), _ptr(i), _ptr(z), _ptr(h0), dO.data_ptr(), _ptr(dh_final),
        g["dx"].data_ptr(), g["dr"].data_ptr(), g["dA"].data_ptr(), _ptr(g.get("di")), _ptr(g.get("dz")),
        _ptr(g.get("dh0")), 1 if use_saved else 0, ws.data_ptr(), have, _stream(stream, index)), "rla_glr_backward")
    return grads


def rla_glr_decode(x, r, A, i=None, z=None, normalize=True, h_in=None, h_out=None, out=None, stream=None):
    """A few new tokens x [B, T, D] onto the states h_in [B, D] (None: zeros).
    Returns (o, h_out); h_out=h_in updates in place, and out may be x, r, i or z."""
    _lib()
    if x is not None and x.dim() != 3:
        raise ValueError("x must be [B, T, D]")
    problem, index, shape = _glr(x, r, A, i, z, normalize, None)
    f32 = torch.float32
    _check("h_in", h_in, index, shape, f32)
    _check("h_out", h_out, index, shape, f32)
    _check("out", out, index, x.shape, x.dtype)
    if out is None:
        out = _new(x, x.shape, x.dtype, stream)
    if h_out is None:
        h_out = _new(x, shape, f32, stream)
    _ok(_call("rla_glr_decode", index)(
        problem, x.data_ptr(), r.data_ptr(), A.data_ptr(), _ptr(i), _ptr(z), _ptr(h_in), out.data_ptr(),
        h_out.data_ptr(), _stream(stream, index)), "rla_glr_decode")
    return out, h_out
