"""What the operators that bring prompts into the cache refuse before they touch a GPU, through the C ABI and the Python functions."""

import ctypes as C

import pytest


def _ops():
    from paper_2302_14357_amd import ops
    return ops.load_library(), ops


P = 1 << 20   # an aligned address that nothing may look at
A, B, D, E = (P << i for i in (1, 2, 3, 4))


def _set(a, kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _tables(ops, **kw):
    return _set(ops._Tables(lens=P, free_pages=P, taken=P, tables=P, out_lens=P, out_taken=A, ld_tables=10, prompts=4, beams=2, page=16, table_width=10, room=5, free_count=100), kw)


@pytest.mark.parametrize("bad", [dict(lens=None), dict(free_pages=None), dict(taken=None), dict(tables=None), dict(out_lens=None), dict(out_taken=None), dict(out_taken=P),
                                 dict(ld_tables=9), dict(prompts=-1), dict(beams=0), dict(beams=65536), dict(page=0), dict(page=65537), dict(table_width=0),
                                 dict(room=-1), dict(room=(1 << 30) + 1), dict(free_count=-1), dict(table_width=1 << 20, ld_tables=1 << 20, page=2048),
                                 dict(prompts=1 << 20, beams=2048)])
def test_tables_refuses(bad):
    L, ops = _ops()
    assert L.tbs_page_tables(C.byref(_tables(ops, **bad)), None) == -1


def _slots(ops, **kw):
    return _set(ops._Slots(lens=P, tables=P, starts=P, positions=P, slots=P, ld_tables=10, prompts=4, tokens=50, page=16, table_width=10), kw)


@pytest.mark.parametrize("bad", [dict(lens=None), dict(tables=None), dict(starts=None), dict(positions=None), dict(slots=None), dict(ld_tables=9), dict(prompts=-1), dict(tokens=-1),
                                 dict(page=0), dict(page=65537), dict(table_width=0), dict(table_width=1 << 20, ld_tables=1 << 20, page=2048)])
def test_slots_refuses(bad):
    L, ops = _ops()
    assert L.tbs_page_slots(C.byref(_slots(ops, **bad)), None) == -1


# q [7, 8, 64], k and v [7, 2, 64] in bf16, each in memory of its own, a cache of 50 pages of 16 tokens
def _rotary(ops, **kw):
    return _set(ops._Rotary(q=A, k=B, v=D, positions=P, freqs=P, slots=P, q_out=E, k_out=E * 2, k_cache=E * 4, v_cache=E * 8, q_row=512, q_head=64, k_row=128, k_head=64, v_row=128,
                            v_head=64, q_out_row=512, q_out_head=64, k_out_row=128, k_out_head=64, k_cache_page=2048, k_cache_token=128, k_cache_head=64, v_cache_page=2048,
                            v_cache_token=128, v_cache_head=64, tokens=7, heads=8, kv_heads=2, dim=64, pairs=32, interleaved=0, pages=50, page=16, dtype=1), kw)


@pytest.mark.parametrize("bad", [dict(q=None), dict(k=None), dict(v=None), dict(positions=None), dict(freqs=None), dict(slots=None), dict(q_out=None), dict(k_out=None), dict(k_cache=None),
                                 dict(v_cache=None), dict(q=A + 1), dict(v_cache=E * 8 + 1), dict(tokens=-1), dict(heads=0), dict(heads=65536), dict(kv_heads=0), dict(dim=0),
                                 dict(dim=513), dict(pairs=-1), dict(pairs=33), dict(interleaved=2), dict(pages=0), dict(page=0), dict(page=65537), dict(dtype=3), dict(q_row=-1),
                                 dict(q_out_row=511), dict(q_out_head=63), dict(k_out_head=0), dict(k_cache_head=63), dict(v_cache_token=63), dict(k_cache_page=63),
                                 # results over what is read, or over each other
                                 dict(q_out=A, q_out_row=640), dict(q_out=A + 2), dict(q_out=B), dict(q_out=B - 7 * 1024 + 2), dict(q_out=D + 2), dict(k_out=A), dict(k_out=B + 2), dict(k_out=D), dict(k_out=E),
                                 dict(k_out=E + 7 * 1024 - 2),
                                 # a cache over what is read or written, over the other
                                 dict(k_cache=A), dict(k_cache=B + 7 * 256 - 2), dict(v_cache=D - 204800 + 2), dict(v_cache=E - 204800 + 2), dict(k_cache=E * 2), dict(k_cache=E * 8)])
def test_rotary_refuses(bad):
    L, ops = _ops()
    assert L.tbs_rotary(C.byref(_rotary(ops, **bad)), None) == -1


# q [7, 8, 64], k and v [7, 2, 64], out [7, 8, 64] in bf16
def _prompts(ops, **kw):
    return _set(ops._Prompts(q=A, k=B, v=D, starts=P, past=P, tables=P, k_cache=E * 4, v_cache=E * 8, out=E, workspace=P, workspace_bytes=1 << 40, q_row=512, q_head=64, k_row=128, k_head=64,
                             v_row=128, v_head=64, out_row=512, out_head=64, k_cache_page=2048, k_cache_token=128, k_cache_head=64, v_cache_page=2048, v_cache_token=128,
                             v_cache_head=64, ld_tables=10, tokens=7, prompts=3, heads=8, kv_heads=2, dim=64, page=16, pages=50, table_width=10, dtype=1), kw)


PLAIN = dict(past=None, tables=None, k_cache=None, v_cache=None)


@pytest.mark.parametrize("bad", [dict(q=None), dict(k=None), dict(v=None), dict(starts=None), dict(out=None), dict(past=None), dict(tables=None), dict(k_cache=None), dict(v_cache=None),
                                 dict(PLAIN, tables=P), dict(PLAIN, k_cache=P), dict(tokens=-1), dict(tokens=1 << 28), dict(prompts=-1), dict(heads=7), dict(heads=0), dict(kv_heads=0), dict(dim=0), dict(dim=12),
                                 dict(dim=264), dict(page=0), dict(page=65537), dict(pages=0), dict(table_width=0), dict(ld_tables=9), dict(table_width=1 << 20, page=2048, ld_tables=1 << 20),
                                 dict(dtype=3), dict(q=A + 1), dict(k_cache=P + 1), dict(q_row=-1), dict(out_row=511), dict(out_head=63), dict(out_head=0),
                                 dict(out=A, out_row=640), dict(out=A + 2), dict(out=A - 7 * 1024 + 2), dict(out=B), dict(out=B + 7 * 256 - 2), dict(out=D), dict(out=D - 7 * 1024 + 2), dict(k_cache=E),
                                 dict(v_cache=E - 204800 + 2), dict(out=E * 4 + 204800 - 2)])
def test_prompts_refuses(bad):
    L, ops = _ops()
    assert L.tbs_attend_prompts(C.byref(_prompts(ops, **bad)), None) == -1


def test_prompts_of_no_tokens_and_its_workspace():
    L, ops = _ops()
    assert L.tbs_attend_prompts(C.byref(_prompts(ops, tokens=0)), None) == 0
    assert L.tbs_attend_prompts(None, None) == -1 and L.tbs_attend_prompts_workspace(None) == -1
    assert L.tbs_attend_prompts_workspace(C.byref(_prompts(ops, dim=12))) == -1
    assert L.tbs_attend_prompts_workspace(C.byref(_prompts(ops, tokens=0))) == 0
    assert L.tbs_rotary(C.byref(_rotary(ops, tokens=0)), None) == 0
    for f in (L.tbs_rotary, L.tbs_page_tables, L.tbs_page_slots):
        assert f(None, None) == -1


def test_tensors_that_do_not_fit():
    import torch
    from paper_2302_14357_amd import attend_prompts, page_slots, page_tables, rotary
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)   # noqa: E731
    x, k, f = torch.zeros(5, 4, 8), torch.zeros(5, 2, 8), torch.zeros(4, dtype=torch.float64)
    calls = [lambda: attend_prompts(x, k, k, i32(2)), lambda: attend_prompts(x, k.half(), k, i32(2)), lambda: attend_prompts(x[0], k, k, i32(2)), lambda: attend_prompts(x, k, k, [0, 5]),
             lambda: attend_prompts(x, k, k, i32(2), past=i32(1)), lambda: rotary(x, k, i32(5), f), lambda: rotary(x, k, i32(5), f.float()), lambda: rotary(x, k, i32(5), f, v=k),
             lambda: rotary(x, k, i32(5), f, interleaved=torch.zeros(2)), lambda: page_tables(i32(3), page=4, width=2, free=i32(9), taken=i32(1)),
             lambda: page_slots(i32(3), i32(3, 2), page=4, tokens=9), lambda: rotary(x.int(), k.int(), i32(5), f)]
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_tensors_that_require_a_gradient():
    """None of the operators has a gradient, so a call that would lose one is refused; without grad mode it is a call like another (here: not on a GPU)."""
    import torch
    from paper_2302_14357_amd import attend_prompts, rotary
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)   # noqa: E731
    x, k, f, c, slots = torch.zeros(5, 4, 8), torch.zeros(5, 2, 8), torch.zeros(4, dtype=torch.float64), torch.zeros(3, 4, 2, 8), torch.zeros(5, dtype=torch.int64)
    leaf = lambda t: t.clone().requires_grad_()   # noqa: E731
    cached = dict(past=i32(1), tables=i32(1, 2))
    calls = [lambda g: attend_prompts(g(x), k, k, i32(2)), lambda g: attend_prompts(x, g(k), k, i32(2)), lambda g: attend_prompts(x, k, g(k), i32(2)),
             lambda g: attend_prompts(x, k, k, i32(2), out=g(x)), lambda g: attend_prompts(x, k, k, i32(2), k_cache=g(c), v_cache=c, **cached),
             lambda g: attend_prompts(x, k, k, i32(2), k_cache=c, v_cache=g(c), **cached), lambda g: rotary(g(x), k, i32(5), f), lambda g: rotary(x, g(k), i32(5), f),
             lambda g: rotary(x, k, i32(5), g(f)), lambda g: rotary(x, k, i32(5), f, v=g(k), k_cache=c, v_cache=c, slots=slots),
             lambda g: rotary(x, k, i32(5), f, v=k, k_cache=g(c), v_cache=c, slots=slots)]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call(leaf)
        for g in (leaf, lambda t: t):
            with torch.no_grad(), pytest.raises(ValueError) as e:
                call(g)
            assert "gradient" not in str(e.value)
