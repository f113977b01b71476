"""What the operators of an autoregressive model refuse before they touch a GPU, through the C ABI and the Python functions."""

import ctypes as C

import pytest


def _ops():
    from paper_2302_14357_amd import ops
    return ops.load_library(), ops


P = 1 << 20   # an aligned address that nothing may look at


def _linear(ops, **kw):
    a = ops._Linear(x=P, w=P, bias=P, out=P, ld_x=64, ld_w=64, ld_out=32, m=3, n=32, k=64, dtype=1, out_dtype=1, act=0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [dict(x=None), dict(w=None), dict(out=None), dict(m=-1), dict(n=0), dict(k=0), dict(k=2**31 - 1), dict(ld_x=63), dict(ld_w=63),
                                 dict(ld_out=31), dict(residual=P, ld_residual=31), dict(dtype=3), dict(dtype=-1), dict(out_dtype=2), dict(act=5),
                                 dict(act=-1), dict(x=P + 1), dict(bias=P + 2), dict(out=P + 1), dict(residual=P + 1, ld_residual=32)])
def test_linear_refuses(bad):
    L, ops = _ops()
    assert L.tbs_linear(C.byref(_linear(ops, **bad)), None) == -1


# x [6, 64] by rows of 256 bytes, w [32, 64], out [6, 32] by rows of 128, in bf16, each in memory of its own; what lies over the result
A, B, D, R, W = (P * i for i in (2, 3, 4, 5, 6))


@pytest.mark.parametrize("bad", [dict(out=A, ld_out=128), dict(out=A + 64, ld_out=128), dict(out=A + 126, ld_out=128), dict(out=A - 62, ld_out=128), dict(out=A - 256 * 5 - 62, ld_out=128),
                                 dict(out=A + 256 * 5, ld_out=128), dict(out=A + 126), dict(out=A - 5 * 64 - 62), dict(out=A + 5 * 256 + 126), dict(out=B), dict(out=B - 62, m=1),
                                 dict(out=B + 64 * 2 * 32 - 2), dict(out=B, ld_out=64), dict(out=W + 126), dict(out=W - 6 * 64 + 2), dict(residual=D, ld_residual=64),
                                 dict(residual=D + 2, ld_residual=32), dict(residual=D + 62, ld_residual=32), dict(residual=D - 6 * 64 + 2, ld_residual=32),
                                 dict(residual=D + 62, ld_residual=100, m=1), dict(residual=D - 4, ld_residual=33)])
def test_linear_refuses_a_result_over_what_it_reads(bad):
    L, ops = _ops()
    kw = dict(x=A, ld_x=128, m=6, w=B, out=D, bias=W, n=32, k=64)
    assert L.tbs_linear(C.byref(_linear(ops, **{**kw, **bad})), None) == -1


def test_linear_of_no_rows():
    L, ops = _ops()
    assert L.tbs_linear(C.byref(_linear(ops, m=0, x=None, out=None)), None) == 0
    assert L.tbs_linear(None, None) == -1


def _attend(ops, **kw):
    a = ops._Attend(q=P, k_new=P, v_new=P, k_cache=P, v_cache=P, tables=P, lens=P, out=P, workspace=P, workspace_bytes=1 << 40, q_row=512, q_head=64,
                    k_new_row=128, k_new_head=64, v_new_row=128, v_new_head=64, out_row=512, out_head=64, k_page=2048, k_token=128, k_head=64, v_page=2048,
                    v_token=128, v_head=64, ld_tables=10, rows=4, heads=8, kv_heads=2, dim=64, page=16, pages=50, table_width=10, max_len=0, beams=2, dtype=1)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [dict(q=None), dict(k_cache=None), dict(v_cache=None), dict(tables=None), dict(lens=None), dict(out=None), dict(k_new=None),
                                 dict(v_new=None), dict(rows=-1), dict(rows=65536, beams=1), dict(heads=7), dict(heads=0), dict(kv_heads=0), dict(dim=0),
                                 dict(dim=12), dict(dim=264), dict(page=0), dict(page=65537), dict(pages=0), dict(table_width=0), dict(ld_tables=9),
                                 dict(beams=0), dict(beams=3), dict(max_len=-1), dict(dtype=3), dict(q=P + 1), dict(k_cache=P + 1), dict(out=P + 1),
                                 dict(table_width=1 << 20, page=2048, ld_tables=1 << 20), dict(out_row=63), dict(out_head=63), dict(k_head=63),
                                 dict(v_token=63), dict(k_page=-1), dict(v_page=8), dict(workspace=None, rows=2, table_width=4096, ld_tables=4096),
                                 dict(workspace=P + 8, rows=2, table_width=4096, ld_tables=4096),
                                 dict(workspace_bytes=16, rows=2, table_width=4096, ld_tables=4096)])
def test_attend_refuses(bad):
    L, ops = _ops()
    assert L.tbs_attend_paged(C.byref(_attend(ops, **bad)), None) == -1


def test_attend_of_no_rows_and_its_workspace():
    L, ops = _ops()
    assert L.tbs_attend_paged(C.byref(_attend(ops, rows=0)), None) == 0
    assert L.tbs_attend_paged(None, None) == -1 and L.tbs_attend_workspace(None) == -1
    assert L.tbs_attend_workspace(C.byref(_attend(ops, dim=12))) == -1
    long = dict(table_width=4096, ld_tables=4096)
    assert L.tbs_attend_workspace(C.byref(_attend(ops, **long))) > 0          # four rows over 65536 tokens are split
    assert L.tbs_attend_workspace(C.byref(_attend(ops, max_len=30, **long))) == 0   # ... not over 30
    assert L.tbs_attend_workspace(C.byref(_attend(ops, rows=8192, **long))) == 0    # ... nor where the rows fill the chip


def _select(ops, **kw):
    a = ops._Select(logits=P, scores=P, out_scores=P, out_tokens=P, out_parents=P, out_finished=P, workspace=P, workspace_bytes=1 << 40, ld_logits=1000, rows=10,
                    beams=5, vocab=1000, eos=0, dtype=0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [dict(logits=None), dict(scores=None), dict(out_scores=None), dict(out_tokens=None), dict(out_parents=None),
                                 dict(out_finished=None), dict(workspace=None, vocab=4000, ld_logits=4000), dict(workspace_bytes=64, vocab=4000, ld_logits=4000),
                                 dict(workspace=P + 4, vocab=4000, ld_logits=4000), dict(ld_logits=999),
                                 dict(rows=-5), dict(rows=11), dict(rows=65540), dict(beams=0), dict(beams=33, rows=33), dict(vocab=0), dict(vocab=524289, ld_logits=524289),
                                 dict(dtype=3), dict(logits=P + 2)])
def test_select_refuses(bad):
    L, ops = _ops()
    assert L.tbs_beam_select(C.byref(_select(ops, **bad)), None) == -1


def test_select_of_no_rows():
    L, ops = _ops()
    assert L.tbs_beam_select(C.byref(_select(ops, rows=0)), None) == 0
    assert L.tbs_beam_select_workspace(C.byref(_select(ops, rows=0))) == 0
    assert L.tbs_beam_select_workspace(C.byref(_select(ops))) == 0                      # a vocabulary of 1000 needs none
    assert L.tbs_beam_select_workspace(C.byref(_select(ops, vocab=4000, ld_logits=4000))) > 0
    assert L.tbs_beam_select(None, None) == -1 and L.tbs_beam_select_workspace(None) == -1


def _reorder(ops, **kw):
    ptrs = (C.c_void_p * 129)(*([P] * 129))
    a = ops._Reorder(parents=P, tables=P, lens=P, out_tables=2 * P, out_lens=2 * P, caches=C.cast(ptrs, C.c_void_p), cache_page=2048, cache_token=128,
                     cache_head=64, ld_tables=10, ld_out_tables=10, n_caches=2, rows=10, beams=5, table_width=10, pages=200, page=16, kv_heads=2, dim=64, dtype=1,
                     appended=1)
    for k, v in kw.items():
        setattr(a, k, v)
    a.keep = ptrs
    return a


@pytest.mark.parametrize("bad", [dict(parents=None), dict(tables=None), dict(lens=None), dict(out_tables=None), dict(out_lens=None), dict(caches=None),
                                 dict(n_caches=-1), dict(n_caches=129), dict(rows=-5), dict(rows=11), dict(beams=0), dict(beams=33, rows=33),
                                 dict(table_width=0), dict(ld_tables=9), dict(ld_out_tables=9), dict(pages=0), dict(page=0), dict(page=65537),
                                 dict(kv_heads=0), dict(dim=0), dict(dtype=7), dict(appended=2), dict(cache_page=-1), dict(cache_token=63), dict(cache_head=63),
                                 dict(out_tables=P), dict(out_tables=P + 396), dict(out_lens=P + 36)])
def test_reorder_refuses(bad):
    L, ops = _ops()
    assert L.tbs_beam_reorder(C.byref(_reorder(ops, **bad)), None) == -1


def test_reorder_of_no_rows():
    L, ops = _ops()
    assert L.tbs_beam_reorder(C.byref(_reorder(ops, rows=0)), None) == 0
    assert L.tbs_beam_reorder(None, None) == -1


def test_tensors_that_do_not_fit():
    import torch
    from paper_2302_14357_amd import attend_paged, beam_reorder, beam_select, linear
    x, w = torch.zeros(3, 8), torch.zeros(4, 8)
    for args, kw in [((x, w), {}),                                              # not on a GPU
                     ((x, torch.zeros(4, 9)), {}), ((x, w.half()), {}), ((x, w), dict(act="softplus")), ((x.int(), w.int()), {})]:
        with pytest.raises(ValueError):
            linear(*args, **kw)
    cache = torch.zeros(5, 4, 2, 8)
    with pytest.raises(ValueError):
        attend_paged(torch.zeros(2, 4, 8), cache, cache, torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        beam_select(x, torch.zeros(3, dtype=torch.float64), beams=3)
    with pytest.raises(ValueError):
        beam_reorder(torch.zeros(3, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), [cache], beams=3)


def test_tensors_that_require_a_gradient():
    """None of the operators has a gradient, so a call that would lose one is refused; without grad mode it is a call like another (here: not on a GPU)."""
    import torch
    from paper_2302_14357_amd import attend_paged, beam_reorder, beam_select, linear
    x, w, b, r = torch.zeros(3, 8), torch.zeros(4, 8), torch.zeros(4), torch.zeros(3, 4)
    q, cache, kn = torch.zeros(2, 4, 8), torch.zeros(5, 4, 2, 8), torch.zeros(2, 2, 8)
    tables, lens = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    leaf = lambda t: t.clone().requires_grad_()   # noqa: E731
    calls = [lambda f: linear(f(x), w, b, residual=r), lambda f: linear(x, f(w), b, residual=r), lambda f: linear(x, w, f(b), residual=r), lambda f: linear(x, w, b, residual=f(r)),
             lambda f: linear(x, w, out=f(r)), lambda f: attend_paged(f(q), cache, cache, tables, lens), lambda f: attend_paged(q, f(cache), cache, tables, lens),
             lambda f: attend_paged(q, cache, f(cache), tables, lens), lambda f: attend_paged(q, cache, cache, tables, lens, k_new=f(kn), v_new=kn),
             lambda f: attend_paged(q, cache, cache, tables, lens, k_new=kn, v_new=f(kn)), lambda f: beam_select(f(x), torch.zeros(3, dtype=torch.float64), beams=3),
             lambda f: beam_select(x, f(torch.zeros(3, dtype=torch.float64)), beams=3), lambda f: beam_reorder(lens, tables, lens, [cache, f(cache)], beams=2),
             lambda f: beam_reorder(lens, tables, lens, f(torch.zeros(2, 5, 4, 2, 8)), beams=2)]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call(leaf)
        for f in (leaf, lambda t: t):
            with torch.no_grad(), pytest.raises(ValueError) as e:
                call(f)
            assert "gradient" not in str(e.value)
        with pytest.raises(ValueError) as e:
            call(lambda t: t)
        assert "gradient" not in str(e.value)


def test_reorder_appended_that_is_no_truth_value():
    import torch
    from paper_2302_14357_amd import beam_reorder
    row, tables = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="appended"):
        beam_reorder(row, tables, row, [torch.zeros(5, 4, 2, 8)], beams=2, appended=torch.zeros(2))
