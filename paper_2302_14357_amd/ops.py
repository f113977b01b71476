"""Operators of an autoregressive model beside the search (include/tbs.h): products with their epilogue, attention of one
new token over a paged cache, selection over beams and vocabulary, reordering of the cached states.

Each function checks its tensors, makes the outputs and enqueues the kernels on the current stream of the tensors' device; nothing
synchronises.  They serve and have no gradients: with grad mode on, a tensor that requires one is refused.  What the library refuses is a TbsError, a tensor of the wrong type, shape or device a ValueError.
"""

from __future__ import annotations

import ctypes as C

from .tbs import TbsError, _check, load_library  # noqa: F401

_P, _I32, _I64 = C.c_void_p, C.c_int32, C.c_int64

_ACTS = {"none": 0, "relu": 1, "tanh": 2, "gelu": 3, "silu": 4}


# The C ABI's argument blocks, for callers of libtbs without the binding module.
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


_binding = None


def _load():
    """libtbs and the module that calls it (csrc/ops_binding.cpp), once."""
    global _binding
    load_library()
    try:
        from . import _tbs_ops
    except ImportError as e:
        raise ImportError(f"{e}: build it with `python -m paper_2302_14357_amd.build` (there is no CPU fallback)") from e
    _tbs_ops.raise_by(_check)
    _binding = _tbs_ops
    return _binding


def linear(x, weight, bias=None, *, act="none", residual=None, out=None, out_dtype=None):
    """act(x @ weight.T + bias) + residual.

    x [..., K] and weight [N, K] in float32, bfloat16 or float16; bias [N] float32; residual and the result [..., N] in x's type or, with
    out_dtype=torch.float32, in float32.  act: "none", "relu", "tanh", "gelu" (by the error function) or "silu".  `out` may be
    `residual`, and lie over nothing else that is read (slices of one tensor beside each other are fine).  Rows apart by
    their length or more; the sum is float32 and rounded once.
    """
    code = _ACTS.get(act)
    if code is None:
        raise ValueError(f"act {act!r}: one of {sorted(_ACTS)} is wanted")
    f32 = None
    if out_dtype is not None:
        f32 = out_dtype.itemsize == 4 and out_dtype.is_floating_point
        if not f32 and out_dtype != x.dtype:
            raise ValueError(f"the result in {out_dtype}: x's type or float32 is wanted")
    return (_binding or _load()).linear(x, weight, bias, code, residual, out, f32)


def attend_paged(q, k_cache, v_cache, tables, lens, *, k_new=None, v_new=None, scale=None, beams=1, max_len=None, out=None):
    """Attention of one new token per row over a paged cache; the new token's key and value are written to the cache.

    q [rows, heads, dim], k_new and v_new [rows, kv_heads, dim] (both or neither), k_cache and v_cache [pages, page, kv_heads, dim] (any
    strides, a head's elements side by side; a layout [pages, kv_heads, page, dim] is given as its transpose), all in one of float32,
    bfloat16 and float16; tables int32 [rows, table width] of page numbers; lens int32 [rows], the tokens in the cache before this one,
    negative for a row that takes no part.  Returns [rows, heads, dim] (`out`, which may be `q`).  `beams` rows are hypotheses of one utterance and may share
    pages; `max_len` is about the longest row's tokens (default: what a table holds).  include/tbs.h says what holds at the edges.
    """
    return (_binding or _load()).attend_paged(q, k_cache, v_cache, tables, lens, k_new, v_new, scale, beams, max_len, out)


def beam_select(logits, scores, *, beams, finished=None, eos=-1):
    """The `beams` best continuations of every group of `beams` hypotheses: (scores float64, tokens int32, parents int32, finished bool), [rows]
    each and best first in every group.

    logits [rows, vocabulary] in float32, bfloat16 or float16, scores [rows] float64 (natural logarithms), finished [rows] bool.  A
    candidate's score is its hypothesis' plus the logarithm of its softmax; a finished hypothesis stays as it is.  Places without
    a candidate have the score -inf, token and parent -1 and are finished; at the first step give the hypotheses that do not exist
    yet the score -inf.
    """
    return (_binding or _load()).beam_select(logits, scores, beams, finished, eos)


def beam_reorder(parents, tables, lens, caches, *, beams, finished=None, appended=True, status=None):
    """The states of beam_select's hypotheses: (tables, lens), new tensors, with the caches' pages that are not full copied in place where several
    hypotheses go on from one.

    parents and finished are beam_select's; tables int32 [rows, table width] and lens int32 [rows] the ones this step ran with; caches the key and
    value caches [pages, page, kv_heads, dim] of every layer (a list of tensors alike in shape, strides and type, or one tensor with
    their number in front).  Full pages are shared, not copied.  `appended`: the step wrote a token per row that took part.  `status`
    (int32, one number) counts hypotheses that had to be dropped; include/tbs.h says when.  Their places, and those of their children, have the length -1:
    where `(lens == -1) & ~finished`, give the score -inf before the next beam_select.
    """
    return (_binding or _load()).beam_reorder(parents, tables, lens, caches, beams, finished, appended, status)
