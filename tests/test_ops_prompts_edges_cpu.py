"""What the operators that bring prompts into the paged cache refuse besides, before they touch a GPU: memory that a call writes over what it reads or writes elsewhere."""

import ctypes as C

import pytest

from test_ops_prompts_cpu import A, E, P, _ops, _prompts, _rotary, _slots, _tables

K = E * 4                                                                        # the keys' cache of _rotary: 50 pages of 16 tokens, 2 heads of 64, 2 bytes a number
TURN = dict(k_cache_page=4096, k_cache_token=256, k_cache_head=128, v_cache_page=4096, v_cache_token=256, v_cache_head=128)   # (places between the heads for the other cache's)


@pytest.mark.parametrize("bad", [dict(v_cache=K + 2), dict(v_cache=K - 2), dict(v_cache=K + 128), dict(v_cache=K + 256), dict(v_cache=K + 4096), dict(v_cache=K + 4096 * 50 - 2), dict(v_cache=K - 4096 * 49),
                                 dict(TURN, v_cache=K + 126), dict(TURN, v_cache=K + 130), dict(TURN, v_cache=K + 256), dict(TURN, v_cache=K + 8192 * 49 + 254),
                                 dict(v_cache=K + 256, v_cache_token=64, v_cache_head=1024),   # heads' tokens together, in the keys' pages
                                 # a cache over itself: heads at the next token's, a token's at the next page's
                                 dict(k_cache_token=64), dict(v_cache_head=128), dict(k_cache_page=2047), dict(v_cache_page=128, v_cache_token=100)])
def test_rotary_refuses_caches_over_each_other(bad):
    L, ops = _ops()
    assert L.tbs_rotary(C.byref(_rotary(ops, **bad)), None) == -1


# lens [4], free_pages [100], taken [1], tables [8, 10], out_lens [8], out_taken [1], each in memory of its own
APART = dict(lens=P, free_pages=P + 1024, taken=P + 2048, tables=A, out_lens=A + 1024, out_taken=A + 2048)


@pytest.mark.parametrize("bad", [dict(out_lens=P), dict(out_lens=P - 28), dict(out_lens=P + 12), dict(tables=P), dict(tables=P - 316), dict(out_taken=P + 12), dict(out_taken=P), dict(tables=P + 1020),
                                 dict(out_lens=P + 1024 + 396), dict(out_taken=P + 1024 + 396), dict(out_lens=P + 2048), dict(tables=P + 2048 - 316), dict(out_taken=P + 2048), dict(out_lens=A),
                                 dict(out_lens=A + 316), dict(out_taken=A + 320 - 4), dict(out_taken=A + 1024 + 28), dict(beams=1, out_lens=P), dict(tables=P - 200, ld_tables=25, beams=1)])
def test_tables_refuses_results_over_what_is_read(bad):
    """Every workgroup reads the lengths of all prompts before its own: a result in their place would be one of those."""
    L, ops = _ops()
    assert L.tbs_page_tables(C.byref(_tables(ops, **dict(APART, **bad))), None) == -1


# lens [4], past [4], tables [4, 10], starts [5], positions [50], slots [50]
PLACES = dict(lens=P, past=P + 1024, tables=P + 2048, starts=A, positions=A + 1024, slots=A + 2048)


@pytest.mark.parametrize("bad", [dict(starts=P), dict(starts=P - 16), dict(starts=P + 1036), dict(positions=P - 196), dict(positions=P + 2048 + 156), dict(slots=P + 12), dict(slots=P + 1032), dict(slots=P + 2048 - 392),
                                 dict(positions=A), dict(slots=A + 1024 + 196), dict(starts=A + 2048 + 396), dict(starts=P + 2048, ld_tables=20), dict(past=None, starts=P)])
def test_slots_refuses_results_over_what_is_read(bad):
    L, ops = _ops()
    assert L.tbs_page_slots(C.byref(_slots(ops, **dict(PLACES, **bad))), None) == -1


@pytest.mark.parametrize("name", ["q_out", "k_out", "k_cache", "v_cache"])
@pytest.mark.parametrize("bad", [dict(positions=1022), dict(positions=-26), dict(freqs=1022), dict(freqs=-254), dict(slots=1022), dict(slots=-54)])
def test_rotary_refuses_results_over_positions_frequencies_and_slots(name, bad):
    """(addresses from the result's first byte: its first row is longer than that of any)"""
    L, ops = _ops()
    at = dict(q_out=E, k_out=E * 2, k_cache=K, v_cache=E * 8)[name]
    for k, v in bad.items():
        assert L.tbs_rotary(C.byref(_rotary(ops, **{k: at + min(v, 254 if name != "q_out" else v)})), None) == -1
    if name[1] == "_" and "cache" not in name:   # without a cache as well
        plain = dict(v=None, slots=None, k_cache=None, v_cache=None)
        for k, v in bad.items():
            if k != "slots":
                assert L.tbs_rotary(C.byref(_rotary(ops, **dict(plain, **{k: at + min(v, 254)}))), None) == -1


@pytest.mark.parametrize("bad", [dict(starts=E), dict(starts=E - 14), dict(starts=E + 7166), dict(past=E - 10), dict(past=E + 7166), dict(tables=E - 118), dict(tables=E + 7166), dict(tables=E - 1000, ld_tables=250)])
def test_prompts_refuses_results_over_starts_past_and_tables(bad):
    L, ops = _ops()
    assert L.tbs_attend_prompts(C.byref(_prompts(ops, **bad)), None) == -1


@pytest.mark.parametrize("call,most", [(dict(tokens=1, prompts=1, heads=32, kv_heads=8, dim=128, page=16, table_width=94, pages=94), 4 << 20),
                                       (dict(tokens=8, prompts=8, heads=8, kv_heads=8, dim=64, page=16, table_width=94, pages=800), 14 << 20),
                                       (dict(tokens=1000, prompts=1, heads=8, kv_heads=8, dim=64, past=None), 10 << 20),
                                       (dict(tokens=1, prompts=1, heads=1, kv_heads=1, dim=256, page=16, table_width=64, pages=64, dtype=0), 2 << 20),
                                       (dict(tokens=256, prompts=1, heads=8, kv_heads=8, dim=128, page=64, table_width=1600, pages=1600), 170 << 20)])
def test_prompts_workspace_is_as_large_as_the_call(call, most):
    """Pieces are four steps of 32 or 64 keys or more: a short table makes few of them, and a long one no more than the chip has places for."""
    L, ops = _ops()
    n = L.tbs_attend_prompts_workspace(C.byref(_prompts(ops, **call)))
    assert 0 < n <= most, n
