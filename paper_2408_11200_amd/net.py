"""ctypes front end of the operators of include/kan_net.h (block norms, embedding, token log probabilities, distillation, clipped gradients, beam
search): same names as the header.  Argument marshalling only, as in `binding`; `autograd` has the same operators on torch's own terms, all but the
clipping and the beams' as differentiable functions.
"""
import ctypes

import torch

from . import binding
from .binding import KAN_OK, KanError, _on_stream, _ptr, _stream, _workspace

EXPORTS = ["kan_block_norm_forward", "kan_block_norm_workspace_bytes", "kan_block_norm_backward", "kan_embedding_forward",
           "kan_embedding_workspace_bytes", "kan_embedding_backward", "kan_token_logprob_forward", "kan_token_logprob_workspace_bytes",
           "kan_token_logprob_backward", "kan_gradient_norm", "kan_clip_gradients", "kan_clip_workspace_bytes", "kan_token_distill_forward",
           "kan_token_distill_backward", "kan_token_distill_step", "kan_token_distill_workspace_bytes", "kan_beam_select",
           "kan_beam_select_workspace_bytes", "kan_beam_reorder"]

KAN_F32, KAN_BF16 = 0, 1
KAN_NORM_RMS, KAN_NORM_LAYER = 0, 1
KAN_TOP_MAX = 64
KAN_TEACHER_LOGP, KAN_TEACHER_LOGITS = 0, 1
KAN_TEACHER_MAX = 256
KAN_BEAM_MAX = 64
TYPES = {torch.float32: KAN_F32, torch.bfloat16: KAN_BF16}
TYPE_NAMES = {"f32": KAN_F32, "bf16": KAN_BF16}
NORMS = {"rms": KAN_NORM_RMS, "layer": KAN_NORM_LAYER}
TEACHERS = {"logp": KAN_TEACHER_LOGP, "logits": KAN_TEACHER_LOGITS}
PARAMS = ("w_post", "b_post", "gate", "w_pre", "b_pre")


class KanBlockNormDesc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("norm", ctypes.c_int32), ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("gate_rows", ctypes.c_int64), ("stream_type", ctypes.c_int32), ("branch_type", ctypes.c_int32)]


class KanBlockNormParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in PARAMS]


class KanBlockNormGrads(ctypes.Structure):
    _fields_ = [("g" + n, ctypes.c_void_p) for n in PARAMS]


class KanTensorRef(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_int64), ("type", ctypes.c_int32)]


class KanStateRef(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("outer", ctypes.c_int64), ("inner", ctypes.c_int64), ("bytes", ctypes.c_int64),
                ("stride", ctypes.c_int64 * 3), ("out_stride", ctypes.c_int64 * 3)]


F32 = torch.float32
_lib = None


def load():
    """The built library with this header's argument types; raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    lib = binding.load()
    vp, i64, sz, i32, f = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int32, ctypes.c_float
    d, p = ctypes.POINTER(KanBlockNormDesc), ctypes.POINTER(KanBlockNormParams)
    of = {"kan_block_norm_forward": [d, i64, vp, vp, p, vp, vp, vp, vp],
          "kan_block_norm_backward": [d, i64, vp, vp, p, vp, vp, vp, vp, vp, ctypes.POINTER(KanBlockNormGrads), vp, sz, vp],
          "kan_embedding_forward": [i64, i64, i32, vp, vp, i32, f, vp, i32, vp],
          "kan_embedding_backward": [i64, i64, i32, vp, vp, i32, f, vp, i32, vp, sz, vp],
          "kan_token_logprob_forward": [i64, i64, vp, i32, i64, vp, f, i32, vp, vp, vp, vp, vp, vp, sz, vp],
          "kan_token_logprob_backward": [i64, i64, vp, i32, i64, vp, f, vp, vp, vp, vp, vp, vp],
          "kan_gradient_norm": [i32, ctypes.POINTER(KanTensorRef), vp, vp, sz, vp],
          "kan_clip_gradients": [i32, ctypes.POINTER(KanTensorRef), f, vp, vp, sz, vp],
          "kan_token_distill_forward": [i64, i64, vp, i32, i64, i32, vp, vp, i32, i32, f, vp, vp, vp, sz, vp],
          "kan_token_distill_backward": [i64, i64, vp, i32, i64, i32, vp, f, vp, vp, vp, vp],
          "kan_token_distill_step": [i64, i64, vp, i32, i64, i32, vp, vp, i32, i32, f, vp, vp, vp, vp, sz, vp],
          "kan_beam_select": [i64, i32, i64, vp, i32, i64, vp, vp, vp, i64, f, i32, vp, vp, vp, vp, vp, sz, vp],
          "kan_beam_reorder": [i64, i32, i32, vp, i32, ctypes.POINTER(KanStateRef), vp]}
    for name, args in of.items():
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = args
    for name, args in {"kan_block_norm_workspace_bytes": [d, i64], "kan_embedding_workspace_bytes": [i64, i64, i32],
                       "kan_token_logprob_workspace_bytes": [i64, i64, i32], "kan_clip_workspace_bytes": [i32],
                       "kan_token_distill_workspace_bytes": [i64, i64, i32], "kan_beam_select_workspace_bytes": [i64, i32, i64, i32]}.items():
        getattr(lib, name).restype = sz
        getattr(lib, name).argtypes = args
    _lib = lib
    return lib


def _done(rc, where):
    if rc != KAN_OK:
        raise KanError(rc, where)


def _of(t, dtype):
    """The address of a tensor of the operator's type (None: no tensor)."""
    if t is None:
        return None
    assert t.dtype == dtype and t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors of the operator's type only"
    return t.data_ptr()


def _of32(t):
    return _of(t, F32)


def _type(dtype):
    assert dtype in TYPES, "float32 and bfloat16 tensors only"
    return TYPES[dtype]


def _new(shape, dtype, device, stream):
    return _on_stream(torch.empty(shape, dtype=dtype, device=device), stream)


# ---- norms at a block boundary --------------------------------------------------------------

_descs = {}


def block_norm_desc(spec, stream_dtype=torch.float32, branch_dtype=None):
    """KanBlockNormDesc from anything with n, norm, eps, residual_scale, gate_rows, branch."""
    key = (spec.n, spec.norm, spec.eps, spec.residual_scale, spec.gate_rows, stream_dtype, branch_dtype or spec.branch)
    d = _descs.get(key)
    if d is None:
        if len(_descs) >= 1024:
            _descs.clear()
        branch = TYPE_NAMES[spec.branch] if branch_dtype is None else _type(branch_dtype)
        d = _descs[key] = KanBlockNormDesc(spec.n, NORMS[spec.norm], spec.eps, spec.residual_scale, spec.gate_rows, _type(stream_dtype), branch)
    return d


def _norm_call(spec, x, f, p):
    """(rows, type of the branch, addresses of the parameters) of a call whose shapes have been checked."""
    n = spec.n
    assert x.shape[-1] == n and (f is None or f.shape == x.shape), "rows of n channels"
    B = x.numel() // n
    at = []
    for name in PARAMS:
        t = p.get(name)
        if t is None:
            at.append(None)
            continue
        assert t.numel() == (n * -(-B // spec.gate_rows) if name == "gate" and spec.gate_rows > 0 else n), name
        at.append(_of(t, F32))
    return B, f.dtype if f is not None else F32 if spec.branch == "f32" else torch.bfloat16, at


def kan_block_norm_forward(spec, x, f, p, x_out=None, h=None, stats=None, want_h=True, stream=None):
    """(x_out, h); p maps w_post, b_post, gate, w_pre, b_pre to tensors (missing ones: ones and zeros).  f None: x_out is x."""
    lib = load()
    B, branch, at = _norm_call(spec, x, f, p)
    if f is None:
        x_out = None
    elif x_out is None:
        x_out = _new(x.shape, x.dtype, x.device, stream)
    if want_h and h is None:
        h = _new(x.shape, branch, x.device, stream)
    dtype = x.dtype
    assert (x_out is None or x_out.numel() == x.numel()) and (h is None or h.numel() == x.numel()) and (stats is None or stats.numel() == 4 * B), "outputs of the rows"
    _done(lib.kan_block_norm_forward(ctypes.byref(block_norm_desc(spec, dtype, branch)), B, _of(x, dtype), _of(f, branch), ctypes.byref(KanBlockNormParams(*at)),
                                     _of(x_out, dtype), _of(h, branch), _of(stats, F32), _stream(stream)), "kan_block_norm_forward")
    return (x if f is None else x_out), h


def kan_block_norm_workspace_bytes(spec, B):
    return int(load().kan_block_norm_workspace_bytes(ctypes.byref(block_norm_desc(spec, torch.bfloat16)), B))


def kan_block_norm_backward(spec, x, f, p, stats, gx_out, gh, want=None, out=None, ws=None, stream=None):
    """All (or the wanted) gradients, named gx, gf, gw_post, ...; default: of x, of f and of every parameter in p."""
    lib = load()
    B, branch, at = _norm_call(spec, x, f, p)
    dtype = x.dtype
    d = block_norm_desc(spec, dtype, branch)
    if want is None:
        want = ("gx",) if f is None else ("gx", "gf")
        want += tuple(["g" + n for n in (PARAMS[3:] if f is None else PARAMS) if p.get(n) is not None])
    out = dict(out or ())
    for name in want:
        if name not in out:
            if name in ("gx", "gf"):
                out[name] = _new(x.shape, dtype if name == "gx" else branch, x.device, stream)
            else:
                rows = -(-B // spec.gate_rows) if spec.gate_rows > 0 else 1
                out[name] = _new((rows, spec.n) if name == "ggate" else (spec.n,), F32, x.device, stream)
    grads = [out.get("g" + n) for n in PARAMS]
    for name, t in zip(PARAMS, grads):
        assert t is None or t.numel() == (spec.n * -(-B // spec.gate_rows) if name == "gate" and spec.gate_rows > 0 else spec.n), "g" + name
    gx, gf = out.get("gx"), out.get("gf")
    assert all([t is None or t.numel() == x.numel() for t in (gx, gf, gx_out, gh)]) and stats.numel() == 4 * B, "gradients of the rows"
    if ws is None and any([t is not None for t in grads]):
        ws = _workspace(lib.kan_block_norm_workspace_bytes(ctypes.byref(d), B), x.device, stream)
    _done(lib.kan_block_norm_backward(ctypes.byref(d), B, _of(x, dtype), _of(f, branch), ctypes.byref(KanBlockNormParams(*at)), _of(stats, F32),
                                      _of(gx_out, dtype), _of(gh, branch), _of(gx, dtype), _of(gf, branch),
                                      ctypes.byref(KanBlockNormGrads(*[_of(t, F32) for t in grads])), _ptr(ws), 0 if ws is None else ws.numel(),
                                      _stream(stream)), "kan_block_norm_backward")
    return out


# ---- embedding ------------------------------------------------------------------------------

def kan_embedding_forward(ids, table, scale=1.0, y=None, dtype=None, stream=None):
    V, n = table.shape
    if y is None:
        y = _new(tuple(ids.shape) + (n,), dtype or table.dtype, table.device, stream)
    assert y.numel() == ids.numel() * n, "a row for each id"
    _done(load().kan_embedding_forward(ids.numel(), V, n, _of(ids, torch.int64), _ptr(table), _type(table.dtype), scale, _ptr(y), _type(y.dtype),
                                       _stream(stream)), "kan_embedding_forward")
    return y


def kan_embedding_workspace_bytes(T, V, n):
    return int(load().kan_embedding_workspace_bytes(T, V, n))


def kan_embedding_backward(ids, gy, V, scale=1.0, gtable=None, dtype=None, ws=None, stream=None):
    """The gradient of a table of V rows (of `dtype`, default that of gy), every row of it."""
    lib, n, T = load(), gy.shape[-1], ids.numel()
    assert gy.numel() == T * n, "a row for each id"
    if gtable is None:
        gtable = _new((V, n), dtype or gy.dtype, gy.device, stream)
    assert tuple(gtable.shape) == (V, n), "V rows of n channels"
    if ws is None:
        ws = _workspace(lib.kan_embedding_workspace_bytes(T, V, n), gy.device, stream)
    _done(lib.kan_embedding_backward(T, V, n, _of(ids, torch.int64), _ptr(gy), _type(gy.dtype), scale, _ptr(gtable), _type(gtable.dtype), _ptr(ws),
                                     ws.numel(), _stream(stream)), "kan_embedding_backward")
    return gtable


# ---- log probabilities of tokens ------------------------------------------------------------

def _logits(t):
    """(pointer, rows, vocabulary, stride) of two-dimensional logits with dense rows, which may be a slice of wider ones."""
    assert t.is_cuda and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1), "device-resident rows of logits only"
    R, V = t.shape
    stride = t.stride(0) if R > 1 else V
    assert stride >= V, "rows of logits must not overlap"
    return t.data_ptr(), R, V, stride


def kan_token_logprob_workspace_bytes(R, V, top=0):
    return int(load().kan_token_logprob_workspace_bytes(R, V, top))


def kan_token_logprob_forward(logits, ids, temperature=1.0, top=0, out=None, ws=None, stream=None):
    """dict of logp, entropy, stats and, for top > 0, top_ids and top_logp."""
    lib = load()
    at, R, V, stride = _logits(logits)
    assert ids.numel() == R, "one id for each row"
    out, dev = dict(out or {}), logits.device
    for name, shape, dtype in (("logp", (R,), torch.float32), ("entropy", (R,), torch.float32), ("stats", (R, 2), torch.float32)):
        if name not in out:
            out[name] = _new(shape, dtype, dev, stream)
        assert out[name].numel() == R * (2 if name == "stats" else 1), name
    if top > 0:
        for name, dtype in (("top_ids", torch.int64), ("top_logp", torch.float32)):
            if name not in out:
                out[name] = _new((R, top), dtype, dev, stream)
            assert out[name].numel() == R * top, name
    if ws is None:
        need = lib.kan_token_logprob_workspace_bytes(R, V, top)
        ws = _workspace(need, dev, stream) if need else None
    _done(lib.kan_token_logprob_forward(R, V, at, _type(logits.dtype), stride, _of(ids, torch.int64), temperature, top, _of32(out["logp"]),
                                        _of32(out["entropy"]), _of32(out["stats"]), _of(out["top_ids"], torch.int64) if top > 0 else None,
                                        _of32(out["top_logp"]) if top > 0 else None, _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)),
          "kan_token_logprob_forward")
    return out


def kan_token_logprob_backward(logits, ids, fwd, g_logp=None, g_entropy=None, temperature=1.0, glogits=None, stream=None):
    """fwd: what the forward call returned (its stats and entropy)."""
    at, R, V, stride = _logits(logits)
    assert ids.numel() == R and all(t is None or t.numel() == R for t in (g_logp, g_entropy)), "one id and gradient for each row"
    if glogits is None:
        glogits = _new((R, V), logits.dtype, logits.device, stream)
    assert glogits.numel() == R * V, "rows of V gradients"
    _done(load().kan_token_logprob_backward(R, V, at, _type(logits.dtype), stride, _of(ids, torch.int64), temperature, _of32(fwd["stats"]),
                                            _of32(fwd["entropy"]), _of32(g_logp), _of32(g_entropy), _of(glogits, logits.dtype), _stream(stream)),
          "kan_token_logprob_backward")
    return glogits


# ---- norm of all gradients ------------------------------------------------------------------

def _tensor_list(tensors, out):
    assert len(out) == len(tensors) and all(o.dtype == t.dtype and o.shape == t.shape for t, o in zip(tensors, out)), "an output like each tensor"
    refs = (KanTensorRef * max(len(tensors), 1))()
    for r, t, o in zip(refs, tensors, out):
        r.data, r.out, r.count, r.type = _ptr(t), _ptr(o), t.numel(), _type(t.dtype)
    return refs


def kan_clip_workspace_bytes(n):
    return int(load().kan_clip_workspace_bytes(n))


def kan_gradient_norm(tensors, norm=None, ws=None, stream=None):
    lib, refs = load(), _tensor_list(tensors, tensors)
    norm = _new((), torch.float32, tensors[0].device, stream) if norm is None else norm
    ws = _workspace(lib.kan_clip_workspace_bytes(len(tensors)), norm.device, stream) if ws is None else ws
    _done(lib.kan_gradient_norm(len(tensors), refs, _of32(norm), _ptr(ws), ws.numel(), _stream(stream)), "kan_gradient_norm")
    return norm


def kan_clip_gradients(tensors, max_norm, out=None, norm=None, ws=None, stream=None):
    """The norm (device tensor); the tensors scaled in place, or into `out`."""
    lib, refs = load(), _tensor_list(tensors, tensors if out is None else out)
    norm = _new((), torch.float32, tensors[0].device, stream) if norm is None else norm
    ws = _workspace(lib.kan_clip_workspace_bytes(len(tensors)), norm.device, stream) if ws is None else ws
    _done(lib.kan_clip_gradients(len(tensors), refs, max_norm, _of32(norm), _ptr(ws), ws.numel(), _stream(stream)), "kan_clip_gradients")
    return norm


# ---- divergence from a teacher's likely tokens ----------------------------------------------

def _teacher(teacher_ids, values, R):
    """(K, address of the ids, of the values, their type) of a teacher's lists, [R][K]."""
    assert teacher_ids.shape == values.shape and teacher_ids.dim() >= 1 and teacher_ids.shape[-1] > 0, "a value for each id, K of them a row"
    K = teacher_ids.shape[-1]
    assert teacher_ids.numel() == R * K, "a list for each row"
    return K, _of(teacher_ids, torch.int64), _of(values, values.dtype), _type(values.dtype)


def kan_token_distill_workspace_bytes(R, V, K):
    return int(load().kan_token_distill_workspace_bytes(R, V, K))


def _distill_workspace(lib, R, V, K, ws, device, stream):
    if ws is None:
        need = lib.kan_token_distill_workspace_bytes(R, V, K)
        ws = _workspace(need, device, stream) if need else None
    return ws, _ptr(ws), 0 if ws is None else ws.numel()


def kan_token_distill_forward(logits, teacher_ids, values, temperature=1.0, teacher="logp", out=None, ws=None, stream=None):
    """dict of loss and stats.  teacher: what the values are, "logp" (log probabilities, the rest of the vocabulary one outcome more) or "logits"."""
    lib = load()
    at, R, V, stride = _logits(logits)
    K, ids_at, values_at, values_type = _teacher(teacher_ids, values, R)
    out, dev = dict(out or {}), logits.device
    for name, shape in (("loss", (R,)), ("stats", (R, K + 2))):
        if name not in out:
            out[name] = _new(shape, F32, dev, stream)
        assert out[name].numel() == R * (1 if name == "loss" else K + 2), name
    ws, ws_at, ws_bytes = _distill_workspace(lib, R, V, K, ws, dev, stream)
    _done(lib.kan_token_distill_forward(R, V, at, _type(logits.dtype), stride, K, ids_at, values_at, values_type, TEACHERS[teacher], temperature,
                                        _of32(out["loss"]), _of32(out["stats"]), ws_at, ws_bytes, _stream(stream)), "kan_token_distill_forward")
    return out


def kan_token_distill_backward(logits, teacher_ids, fwd, g_loss, temperature=1.0, glogits=None, stream=None):
    """fwd: what the forward call returned (its stats)."""
    at, R, V, stride = _logits(logits)
    K = teacher_ids.shape[-1]
    assert teacher_ids.numel() == R * K and fwd["stats"].numel() == R * (K + 2) and g_loss.numel() == R, "a list and a gradient for each row"
    if glogits is None:
        glogits = _new((R, V), logits.dtype, logits.device, stream)
    assert glogits.numel() == R * V, "rows of V gradients"
    _done(load().kan_token_distill_backward(R, V, at, _type(logits.dtype), stride, K, _of(teacher_ids, torch.int64), temperature, _of32(fwd["stats"]), _of32(g_loss),
                                            _of(glogits, logits.dtype), _stream(stream)), "kan_token_distill_backward")
    return glogits


def kan_token_distill_step(logits, teacher_ids, values, g_loss, temperature=1.0, teacher="logp", loss=None, glogits=None, ws=None, stream=None):
    """(loss, glogits) for weights g_loss of the rows that are known before their losses."""
    lib = load()
    at, R, V, stride = _logits(logits)
    K, ids_at, values_at, values_type = _teacher(teacher_ids, values, R)
    loss = _new((R,), F32, logits.device, stream) if loss is None else loss
    glogits = _new((R, V), logits.dtype, logits.device, stream) if glogits is None else glogits
    assert g_loss.numel() == R and loss.numel() == R and glogits.numel() == R * V, "a weight, a loss and a gradient for each row"
    ws, ws_at, ws_bytes = _distill_workspace(lib, R, V, K, ws, logits.device, stream)
    _done(lib.kan_token_distill_step(R, V, at, _type(logits.dtype), stride, K, ids_at, values_at, values_type, TEACHERS[teacher], temperature, _of32(g_loss),
                                     _of32(loss), _of(glogits, logits.dtype), ws_at, ws_bytes, _stream(stream)), "kan_token_distill_step")
    return loss, glogits


# ---- beam search ----------------------------------------------------------------------------

FLAGS = (torch.bool, torch.uint8)


def _flags(t):
    assert t is None or t.dtype in FLAGS, "flags of type bool or uint8"
    return None if t is None else _of(t, t.dtype)


def kan_beam_select_workspace_bytes(N, B, V, top):
    return int(load().kan_beam_select_workspace_bytes(N, B, V, top))


def kan_beam_select(logits, scores, top=None, ended=None, end_id=-1, rank_scale=None, temperature=1.0, out=None, ws=None, stream=None):
    """dict of scores, tokens, parents, ended: the `top` (default: as many as beams) best continuations of every search.  scores [N][B], logits [N * B][V]."""
    lib = load()
    assert scores.dim() == 2 and scores.shape[1] > 0, "scores: a row of beams for each search"
    at, rows, V, stride = _logits(logits)
    N, B = scores.shape
    assert rows == N * B and all(t is None or t.shape == scores.shape for t in (ended, rank_scale)), "a row of logits, a flag and a scale for each beam"
    top = B if top is None else top
    out, dev = dict(out or {}), logits.device
    for name, dtype in (("scores", F32), ("tokens", torch.int64), ("parents", torch.int64), ("ended", torch.bool)):
        if name not in out:
            out[name] = _new((N, top), dtype, dev, stream)
        assert out[name].numel() == N * top, name
    if ws is None:
        ws = _workspace(lib.kan_beam_select_workspace_bytes(N, B, V, top), dev, stream)
    _done(lib.kan_beam_select(N, B, V, at, _type(logits.dtype), stride, _of32(scores), _flags(ended), _of32(rank_scale), end_id, temperature, top,
                              _of32(out["scores"]), _of(out["tokens"], torch.int64), _of(out["parents"], torch.int64), _flags(out["ended"]), _ptr(ws), ws.numel(),
                              _stream(stream)), "kan_beam_select")
    return out


def _evenly(dims):
    """(count, stride, out stride) of dimensions that lie evenly behind one another; dims: sizes above 1 with the strides of both tensors."""
    count, stride, to = 1, 0, 0
    for n, s, o in reversed(dims):
        if count == 1:
            count, stride, to = n, s, o
        else:
            assert s == stride * count and o == to * count, "states whose dimensions before the rows, and behind them, lie evenly"
            count *= n
    return count, stride, to


def _state(shape, strides, out_strides, size, dim):
    """A KanStateRef's numbers behind its two addresses: rows in dimension `dim`, a contiguous end of a row as one run, what is before and between as one dimension each."""
    dims = [(n, a * size, b * size) for n, a, b in zip(shape, strides, out_strides)]
    before, behind, run = [d for d in dims[:dim] if d[0] != 1], [d for d in dims[dim + 1:] if d[0] != 1], size
    while behind and behind[-1][1] == run == behind[-1][2]:
        run *= behind.pop()[0]
    outer, s0, o0 = _evenly(before)
    inner, s2, o2 = _evenly(behind)
    return outer, inner, run, s0, dims[dim][1], s2, o0, dims[dim][2], o2


def kan_beam_reorder(parents, tensors, beams, out=None, dim=0, stream=None):
    """Row n * top + j of every tensor from its row n * beams + parents[n][j], parents [N][top]: in place, or into the tensors of `out`.  dim: the dimension of the rows."""
    assert parents.dim() == 2 and parents.shape[1] > 0, "parents: a row for each search"
    N, top = parents.shape
    out = tensors if out is None else out
    assert len(out) == len(tensors), "an output for each tensor"
    device, numbers, layouts = parents.device, [], {}       # tensors that lie alike are looked at once
    for t, o in zip(tensors, out):
        assert t.device == device and (o is t or o.device == device), "states on the device of the parents"
        key = (t.shape, t.dtype, t.stride()) + (() if o is t else (o.shape, o.dtype, o.stride()))
        layout = layouts.get(key)
        if layout is None:
            shape, other, d = t.shape, o.shape, dim + t.dim() if dim < 0 else dim
            assert len(shape) == len(other) > d >= 0 and shape[d] == N * beams and other[d] == N * top and o.dtype == t.dtype, "a row of a state for each beam, and an output of its type"
            assert shape[:d] == other[:d] and shape[d + 1:] == other[d + 1:], "an output of a state's shape"
            layout = layouts[key] = _state(shape, t.stride(), o.stride(), t.element_size(), d) if t.numel() and o.numel() else ()
        if layout:
            numbers += (t.data_ptr(), o.data_ptr()) + layout
    refs = (ctypes.c_int64 * max(len(numbers), 1))(*numbers)
    _done(load().kan_beam_reorder(N, beams, top, _of(parents, torch.int64), len(numbers) // 11, ctypes.cast(refs, ctypes.POINTER(KanStateRef)), _stream(stream)),
          "kan_beam_reorder")
    return out
