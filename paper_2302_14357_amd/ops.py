"""Operators of an autoregressive model beside the search (include/tbs.h): products with their epilogue, attention of one
new token over a paged cache, selection over beams and vocabulary, reordering of the cached states.

Each function checks its tensors, makes the outputs and enqueues the kernels on the current stream of the tensors' device; nothing
synchronises.  What the library refuses is a TbsError, a tensor of the wrong type, shape or device a ValueError.
"""

from __future__ import annotations

import ctypes as C

from .tbs import TbsError, _check, load_library  # noqa: F401

_P, _I32, _I64 = C.c_void_p, C.c_int32, C.c_int64

_MAX_CACHES = 128
_ACTS = {"none": 0, "relu": 1, "tanh": 2, "gelu": 3, "silu": 4}


class _Linear(C.Structure):
    _fields_ = ([(n, _P) for n in ("x", "w", "bias", "residual", "out")] + [(n, _I64) for n in ("ld_x", "ld_w", "ld_residual", "ld_out")] +
                [(n, _I32) for n in ("m", "n", "k", "dtype", "out_dtype", "act")])


class _Attend(C.Structure):
    _fields_ = ([(n, _P) for n in ("q", "k_new", "v_new", "k_cache", "v_cache", "tables", "lens", "out", "workspace")] +
                [(n, _I64) for n in ("workspace_bytes", "q_row", "q_head", "k_new_row", "k_new_head", "v_new_row", "v_new_head", "out_row", "out_head",
                                     "k_page", "k_token", "k_head", "v_page", "v_token", "v_head", "ld_tables")] +
                [(n, _I32) for n in ("rows", "heads", "kv_heads", "dim", "page", "pages", "table_width", "max_len", "beams", "dtype")] +
                [("scale", C.c_float)])


class _Select(C.Structure):
    _fields_ = ([(n, _P) for n in ("logits", "scores", "finished", "out_scores", "out_tokens", "out_parents", "out_finished", "workspace")] +
                [(n, _I64) for n in ("workspace_bytes", "ld_logits")] + [(n, _I32) for n in ("rows", "beams", "vocab", "eos", "dtype")])


class _Reorder(C.Structure):
    _fields_ = ([(n, _P) for n in ("parents", "tables", "lens", "finished", "out_tables", "out_lens", "status", "caches")] +
                [(n, _I64) for n in ("cache_page", "cache_token", "cache_head", "ld_tables", "ld_out_tables")] +
                [(n, _I32) for n in ("n_caches", "rows", "beams", "table_width", "pages", "page", "kv_heads", "dim", "dtype", "appended")])


_torch = None
_dtypes = {}
_lib = None


def _library():
    """libtbs and torch, once."""
    global _torch, _lib
    if _lib is None:
        import torch
        L = load_library()
        _torch = torch
        _dtypes.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
        _lib = L
    return _lib


def _want(ok, what):
    if not ok:
        raise ValueError(what)


def _dtype(t, name):
    try:
        return _dtypes[t.dtype]
    except KeyError:
        raise ValueError(f"{name} is {t.dtype}: float32, bfloat16 or float16 is wanted") from None


def _call(fn, args, device):
    """fn(&args, current stream), with the tensors' device current."""
    cuda = _torch.cuda
    if device.index != cuda.current_device():
        with cuda.device(device):
            rc = fn(C.byref(args), cuda.current_stream().cuda_stream)
    else:
        rc = fn(C.byref(args), cuda.current_stream().cuda_stream)
    if rc:
        _check(rc)


def _same_device(first, **others):
    _want(first.is_cuda, "the tensors have to be on the GPU: this library has no CPU path")
    for name, t in others.items():
        _want(t is None or t.device == first.device, f"{name} is on {t.device if t is not None else None}, not on {first.device}")


def _rows(t, name, shape):
    """A 2-D tensor whose rows are contiguous: its row stride (of one row: any)."""
    _want(tuple(t.shape) == shape, f"{name} has shape {tuple(t.shape)}: {shape} is wanted")
    _want(t.stride(1) == 1 or shape[1] == 1, f"{name}: elements of a row have to lie side by side")
    return t.stride(0) if shape[0] > 1 else shape[1]


def linear(x, weight, bias=None, *, act="none", residual=None, out=None, out_dtype=None):
    """act(x @ weight.T + bias) + residual.

    x [..., K] and weight [N, K] in float32, bfloat16 or float16; bias [N] float32; residual and the result [..., N] in x's type or, with
    out_dtype=torch.float32, in float32.  act: "none", "relu", "tanh", "gelu" (by the error function) or "silu".  `out` may be
    `residual`.  Rows of any stride; the sum is float32 and rounded once.
    """
    L = _library()
    torch = _torch
    _want(x.dim() >= 1 and weight.dim() == 2, "x [..., K] and weight [N, K] are wanted")
    n, k = weight.shape
    _want(x.shape[-1] == k, f"x has {x.shape[-1]} columns, weight {k}")
    _want(act in _ACTS, f"act {act!r}: one of {sorted(_ACTS)} is wanted")
    dt = _dtype(x, "x")
    _want(weight.dtype == x.dtype, f"weight is {weight.dtype}, x {x.dtype}")
    _same_device(x, weight=weight, bias=bias, residual=residual, out=out)
    lead = x.shape[:-1]
    x2 = x if x.dim() == 2 else x.reshape(-1, k)
    m = x2.shape[0]
    odt = out_dtype or (out.dtype if out is not None else x.dtype)
    _want(odt == x.dtype or odt == torch.float32, f"the result in {odt}: x's type or float32 is wanted")
    if out is None:
        out = torch.empty((*lead, n), dtype=odt, device=x.device)
    _want(out.dtype == odt and tuple(out.shape) == (*lead, n), f"out has shape {tuple(out.shape)} and {out.dtype}: {(*lead, n)} in {odt} is wanted")
    o2 = out if out.dim() == 2 else out.view(-1, n)
    r2, ld_r = None, 0
    if residual is not None:
        _want(residual.dtype == odt and tuple(residual.shape) == (*lead, n),
              f"residual has shape {tuple(residual.shape)} and {residual.dtype}: {(*lead, n)} in {odt} is wanted")
        r2 = residual if residual.dim() == 2 else residual.reshape(-1, n)
        ld_r = _rows(r2, "residual", (m, n))
    if bias is not None:
        _want(bias.dtype == torch.float32 and tuple(bias.shape) == (n,) and (n == 1 or bias.stride(0) == 1), "bias [N] in float32, contiguous, is wanted")
    if m == 0:
        return out
    a = _Linear(x2.data_ptr(), weight.data_ptr(), bias.data_ptr() if bias is not None else None, r2.data_ptr() if r2 is not None else None,
                o2.data_ptr(), _rows(x2, "x", (m, k)), _rows(weight, "weight", (n, k)), ld_r, _rows(o2, "out", (m, n)), m, n, k, dt, _dtypes[odt],
                _ACTS[act])
    _call(L.tbs_linear, a, x.device)
    return out


def _size(bytes_, device):
    """The workspace of a call: a tensor, or None where none is wanted."""
    if bytes_ < 0:
        _check(int(bytes_))
    return _torch.empty(bytes_, dtype=_torch.uint8, device=device) if bytes_ else None


def _heads(t, name, shape, dtype):
    """[rows, heads, dim] with a head's elements side by side: strides of rows and heads (of one row or head: any)."""
    _want(t.dtype == dtype and tuple(t.shape) == shape, f"{name} has shape {tuple(t.shape)} and {t.dtype}: {shape} in {dtype} is wanted")
    row, head, one = t.stride()
    _want(one == 1, f"{name}: elements of a head have to lie side by side")
    return (row if shape[0] > 1 else shape[1] * shape[2]), (head if shape[1] > 1 else shape[2])


def _cache(t, name, shape, dtype):
    _want(t.dim() == 4 and t.dtype == dtype and (shape is None or t.shape == shape),
          f"{name} has shape {tuple(t.shape)} and {t.dtype}: {tuple(shape) if shape is not None else '[pages, page, heads, dim]'} in {dtype} is wanted")
    page, token, head, one = t.stride()
    _want(one == 1, f"{name}: elements of a head have to lie side by side")
    # (a stride that nothing is reached by says nothing)
    return page if t.shape[0] > 1 else t.numel(), token if t.shape[1] > 1 else t.shape[2] * t.shape[3], head if t.shape[2] > 1 else t.shape[3]


def _ints(t, name, rows):
    _want(t.dtype == _torch.int32 and t.dim() == 1 and t.shape[0] == rows and (rows <= 1 or t.stride(0) == 1),
          f"{name} [{rows}] in int32, contiguous, is wanted")
    return t.data_ptr()


def _flags(t, name, rows):
    if t is None:
        return None
    _want(t.dtype in (_torch.bool, _torch.uint8) and t.dim() == 1 and t.shape[0] == rows and (rows <= 1 or t.stride(0) == 1),
          f"{name} [{rows}] in bool, contiguous, is wanted")
    return t.data_ptr()


def attend_paged(q, k_cache, v_cache, tables, lens, *, k_new=None, v_new=None, scale=None, beams=1, max_len=None, out=None):
    """Attention of one new token per row over a paged cache; the new token's key and value are written to the cache.

    q [rows, heads, dim], k_new and v_new [rows, kv_heads, dim] (both or neither), k_cache and v_cache [pages, page, kv_heads, dim] (any
    strides, a head's elements side by side; a layout [pages, kv_heads, page, dim] is given as its transpose), all in one of float32,
    bfloat16 and float16; tables int32 [rows, table width] of page numbers; lens int32 [rows], the tokens in the cache before this one,
    negative for a row that takes no part.  Returns [rows, heads, dim].  `beams` rows are hypotheses of one utterance and may share
    pages; `max_len` is about the longest row's tokens (default: what a table holds).  include/tbs.h says what holds at the edges.
    """
    L = _library()
    torch = _torch
    dt = _dtype(q, "q")
    _want(q.dim() == 3 and k_cache.dim() == 4, "q [rows, heads, dim] and k_cache [pages, page, kv_heads, dim] are wanted")
    rows, heads, dim = q.shape
    pages, page, kv = k_cache.shape[:3]
    _want(k_cache.shape[3] == dim, f"k_cache has heads of {k_cache.shape[3]}, q of {dim}")
    _same_device(q, k_cache=k_cache, v_cache=v_cache, tables=tables, lens=lens, k_new=k_new, v_new=v_new, out=out)
    _want((k_new is None) == (v_new is None), "k_new and v_new belong together")
    _want(tables.dim() == 2 and tables.dtype == torch.int32 and tables.shape[0] == rows, "tables [rows, table width] in int32 is wanted")
    if out is None:
        out = torch.empty((rows, heads, dim), dtype=q.dtype, device=q.device)
    if rows == 0:
        return out
    shape = (rows, kv, dim)
    a = _Attend(q.data_ptr(), None, None, k_cache.data_ptr(), v_cache.data_ptr(), tables.data_ptr(), _ints(lens, "lens", rows), out.data_ptr(), None, 0,
                *_heads(q, "q", (rows, heads, dim), q.dtype), 0, 0, 0, 0, *_heads(out, "out", (rows, heads, dim), q.dtype),
                *_cache(k_cache, "k_cache", None, q.dtype), *_cache(v_cache, "v_cache", k_cache.shape, q.dtype),
                _rows(tables, "tables", (rows, tables.shape[1])), rows, heads, kv, dim, page, pages, tables.shape[1],
                0 if max_len is None else int(max_len), beams, dt, 0.0 if scale is None else scale)
    if k_new is not None:
        a.k_new, a.v_new = k_new.data_ptr(), v_new.data_ptr()
        a.k_new_row, a.k_new_head = _heads(k_new, "k_new", shape, q.dtype)
        a.v_new_row, a.v_new_head = _heads(v_new, "v_new", shape, q.dtype)
    work = _size(L.tbs_attend_workspace(C.byref(a)), q.device)
    if work is not None:
        a.workspace, a.workspace_bytes = work.data_ptr(), work.numel()
    _call(L.tbs_attend_paged, a, q.device)
    return out


def beam_select(logits, scores, *, beams, finished=None, eos=-1):
    """The `beams` best continuations of every group of `beams` hypotheses: (scores float64, tokens int32, parents int32, finished bool), [rows]
    each and best first in every group.

    logits [rows, vocabulary] in float32, bfloat16 or float16, scores [rows] float64 (natural logarithms), finished [rows] bool.  A
    candidate's score is its hypothesis' plus the logarithm of its softmax; a finished hypothesis stays as it is.  Places without
    a candidate have the score -inf, token and parent -1 and are finished; at the first step give the hypotheses that do not exist
    yet the score -inf.
    """
    L = _library()
    torch = _torch
    dt = _dtype(logits, "logits")
    _want(logits.dim() == 2, "logits [rows, vocabulary] is wanted")
    rows, vocab = logits.shape
    _same_device(logits, scores=scores, finished=finished)
    _want(scores.dtype == torch.float64 and scores.dim() == 1 and scores.shape[0] == rows and (rows <= 1 or scores.stride(0) == 1),
          f"scores [{rows}] in float64, contiguous, is wanted")
    done = _flags(finished, "finished", rows)
    out = (torch.empty(rows, dtype=torch.float64, device=logits.device), torch.empty(rows, dtype=torch.int32, device=logits.device),
           torch.empty(rows, dtype=torch.int32, device=logits.device), torch.empty(rows, dtype=torch.bool, device=logits.device))
    if rows == 0:
        return out
    a = _Select(logits.data_ptr(), scores.data_ptr(), done, *[t.data_ptr() for t in out], None, 0, _rows(logits, "logits", (rows, vocab)), rows, beams,
                vocab, eos, dt)
    work = _size(L.tbs_beam_select_workspace(C.byref(a)), logits.device)
    a.workspace, a.workspace_bytes = work.data_ptr(), work.numel()
    _call(L.tbs_beam_select, a, logits.device)
    return out


def beam_reorder(parents, tables, lens, caches, *, beams, finished=None, appended=True, status=None):
    """The states of beam_select's hypotheses: (tables, lens), new tensors, with the caches' pages that are not full copied in place where several
    hypotheses go on from one.

    parents and finished are beam_select's; tables int32 [rows, table width] and lens int32 [rows] the ones this step ran with; caches the key and
    value caches [pages, page, kv_heads, dim] of every layer (a list of tensors alike in shape, strides and type, or one tensor with
    their number in front).  Full pages are shared, not copied.  `appended`: the step wrote a token per row that took part.
    """
    L = _library()
    torch = _torch
    rows = parents.shape[0]
    _want(tables.dim() == 2 and tables.dtype == torch.int32 and tables.shape[0] == rows, "tables [rows, table width] in int32 is wanted")
    _same_device(parents, tables=tables, lens=lens, finished=finished, status=status)
    width = tables.shape[1]
    n = len(caches)
    _want(n > 0, "caches: one at least is wanted")
    c0 = caches[0]
    dt = _dtype(c0, "caches")
    strides = _cache(c0, "caches", None, c0.dtype)
    shape, given, kind, where = c0.shape, c0.stride(), c0.dtype, parents.device
    for c in caches:
        _want(c.shape == shape and c.stride() == given and c.dtype == kind and c.device == where,
              "the caches have to be alike in shape, strides and type, on the device of the tables")
    ptrs = [c.data_ptr() for c in caches]
    pages, page, kv, dim = shape
    _want(status is None or (status.dtype == torch.int32 and status.numel() == 1), "status: one number in int32 is wanted")
    new_tables = torch.empty((rows, width), dtype=torch.int32, device=parents.device)
    new_lens = torch.empty(rows, dtype=torch.int32, device=parents.device)
    if rows == 0:
        return new_tables, new_lens
    a = _Reorder(_ints(parents, "parents", rows), tables.data_ptr(), _ints(lens, "lens", rows), _flags(finished, "finished", rows), new_tables.data_ptr(),
                 new_lens.data_ptr(), status.data_ptr() if status is not None else None, None, *strides, _rows(tables, "tables", (rows, width)), width, 0,
                 rows, beams, width, pages, page, kv, dim, dt, 1 if appended else 0)
    for i in range(0, n, _MAX_CACHES):   # (every launch writes the same tables)
        some = ptrs[i:i + _MAX_CACHES]
        a.caches, a.n_caches = C.cast((_P * len(some))(*some), _P), len(some)
        if i:
            a.status = None
        _call(L.tbs_beam_reorder, a, parents.device)
    return new_tables, new_lens
