"""The operators that bring prompts into the paged cache, at calls that the other tests do not make: the largest values, results in the place of what is
read, strides of results, rows far apart, workspaces of short calls, empty lists."""

import os
import sys

import pytest
import torch

from test_ops_prompts import _close, _gen, _i32, _prompts_by, _prompts_case, _prompts_ref, _randn

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("size", [0.99, 1 / 300])
def test_prompts_of_the_largest_values(size, dim, dtype):
    """A mean of large values is no larger than they are, however large a sum of them is; next to them ordinary ones keep their digits.  (With scores of 0 and values of a 300th
    of the largest number the sums of a few keys are finite, those of all are not.)"""
    from paper_2302_14357_amd import attend_prompts
    g = _gen(dim)
    lens, past, page, heads, kv = [1, 70, 300], [0, 40, 900], 16, 4, 2
    q = _randn(g, sum(lens), heads, dim, dtype=dtype) if size > 0.5 else torch.zeros(sum(lens), heads, dim, dtype=dtype)
    k = _randn(g, sum(lens), kv, dim, dtype=dtype)
    width = 57
    tables = torch.arange(3 * width, dtype=torch.int32).view(3, width)
    kc = _randn(g, 3 * width, page, kv, dim, dtype=dtype)

    def values(*shape):
        x = (torch.rand(*shape, generator=g, dtype=torch.float64) * 0.25 + 0.75) * size * torch.finfo(dtype).max
        x[..., 1::4] *= torch.randint(0, 2, x[..., 1::4].shape, generator=g) * 2 - 1
        x[..., 2::4] = torch.randn(x[..., 2::4].shape, generator=g)
        return x.to(dtype)

    v, vc = values(sum(lens), kv, dim), values(3 * width, page, kv, dim)
    v[:, 1] = _randn(g, sum(lens), dim, dtype=dtype)   # (the other key head has ordinary ones)
    vc[:, :, 1] = _randn(g, 3 * width, page, dim, dtype=dtype)
    starts = _i32([0, 1, 71, 371])
    for cached in (False, True):
        kw = dict(past=_i32(past), k_cache=kc.cuda(), v_cache=vc.cuda(), tables=tables.cuda()) if cached else {}
        ref, tol = _prompts_ref(q, k, v, lens, past if cached else None, kc, vc, tables, page, None, dtype)
        for got in (attend_prompts(q.cuda(), k.cuda(), v.cuda(), starts, **kw), *(_prompts_by(f, q.cuda(), k.cuda(), v.cuda(), starts, **kw) for f in (1, 2))):
            _close(got, ref, tol)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [32, 64, 128, 256])
@pytest.mark.parametrize("lens,past", [([1], [127]), ([1], [255]), ([1], [256]), ([4], [1020]), ([1], [1504]), ([1] * 8, [1504, 3, 0, 700, 255, 256, 1023, 1]), ([130, 1], [896, 1024])])
def test_prompts_pieces_of_short_calls(lens, past, dim, dtype):
    """Keys shared out where the workspace has room for as many pieces of four steps as there may be, and none more (what lies behind it stays)."""
    _prompts_case(lens, past=past, heads=4, kv=2, dim=dim, dtype=dtype, pad=3, force=2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["halves", "halves_by_head", "heads", "tokens"])
def test_rotary_keys_and_values_in_one_tensor(layout, dtype):
    """Caches between each other's first and last number that share none: the same entries as in tensors of their own."""
    from paper_2302_14357_amd import rotary
    g = _gen(7)
    pages, page, kv, dim = 5, 4, 3, 24
    q, k, v = (_randn(g, 17, n, dim, dtype=dtype).cuda() for n in (6, kv, kv))
    at = torch.arange(17, dtype=torch.int32).cuda()
    freqs = 0.7 ** torch.arange(12, dtype=torch.float64).cuda()
    slots = torch.randperm(pages * page, generator=g)[:17].cuda()
    kw = dict(v=v, slots=slots)
    apart = [torch.full((pages, page, kv, dim), 77.0, dtype=dtype, device="cuda") for _ in range(2)]
    want = rotary(q, k, at, freqs, k_cache=apart[0], v_cache=apart[1], **kw)
    both = torch.full((pages * 2 * page * kv * dim,), 77.0, dtype=dtype, device="cuda")
    halves = both.view(pages, 2, page * kv * dim)
    kc, vc = {"halves": lambda: [halves[:, i].view(pages, page, kv, dim) for i in range(2)],
              "halves_by_head": lambda: [halves[:, 0].view(pages, page, kv, dim), halves[:, 1].view(pages, kv, page, dim).transpose(1, 2)],
              "heads": lambda: [both.view(pages, page, 2, kv, dim)[:, :, i] for i in range(2)],
              "tokens": lambda: [both.view(pages, page, kv, 2, dim)[:, :, :, i] for i in range(2)]}[layout]()
    got = rotary(q, k, at, freqs, k_cache=kc, v_cache=vc, **kw)
    for x, y in zip((*want, *apart), (*got, kc, vc)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs,shift", [(64, 32, 0), (64, 20, 0), (64, 32, 1), (40, 17, 3), (7, 3, 0)])
def test_rotary_tokens_with_one_slot_mix_whole_numbers(dim, pairs, shift, interleaved, dtype):
    """Of tokens that name one slot every number is one's, also where pieces of 16 bytes begin inside each other's; no neighbour of the slot is touched."""
    from paper_2302_14357_amd import rotary
    g = _gen(pairs)
    q, k, v = (_randn(g, 300, n, dim, dtype=dtype).cuda() for n in (2, 2, 2))
    kc, vc = (torch.full((shift + 12 * 2 * dim,), 77.0, dtype=dtype, device="cuda")[shift:].view(3, 4, 2, dim) for _ in range(2))
    slots = torch.full((300,), 5).cuda()
    slots[17] = 6
    _, turned = rotary(q, k, torch.arange(300, dtype=torch.int32).cuda(), 0.9 ** torch.arange(pairs, dtype=torch.float64).cuda(), interleaved=interleaved, v=v, k_cache=kc, v_cache=vc, slots=slots)
    for cache, new in ((kc.view(12, 2, dim), turned), (vc.view(12, 2, dim), v)):
        assert bool((cache[5] == new[slots == 5]).any(0).all())
        assert torch.equal(cache[6], new[17]) and bool((cache[[0, 1, 2, 3, 4, 7, 8, 9, 10, 11]] == 77.0).all())


def _rotary_call(q, k, v, at, freqs, slots, kc, vc, q_out, k_out, interleaved):
    """tbs_rotary itself, with outputs of the caller's."""
    import ctypes
    from paper_2302_14357_amd import ops
    L = ops.load_library()
    a = ops._Rotary(q=q.data_ptr(), k=k.data_ptr(), positions=at.data_ptr(), freqs=freqs.data_ptr(), q_out=q_out.data_ptr(), k_out=k_out.data_ptr(), tokens=q.shape[0], heads=q.shape[1],
                    kv_heads=k.shape[1], dim=q.shape[2], pairs=len(freqs), interleaved=int(interleaved), dtype=DTYPES.index(q.dtype))
    a.q_row, a.q_head, a.k_row, a.k_head = *q.stride()[:2], *k.stride()[:2]
    a.q_out_row, a.q_out_head, a.k_out_row, a.k_out_head = *q_out.stride()[:2], *k_out.stride()[:2]
    if slots is not None:
        a.v, a.slots, a.k_cache, a.v_cache, a.pages, a.page = v.data_ptr(), slots.data_ptr(), kc.data_ptr(), vc.data_ptr(), kc.shape[0], kc.shape[1]
        a.v_row, a.v_head = v.stride()[:2]
        a.k_cache_page, a.k_cache_token, a.k_cache_head = kc.stride()[:3]
        a.v_cache_page, a.v_cache_token, a.v_cache_head = vc.stride()[:3]
    assert L.tbs_rotary(ctypes.byref(a), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs", [(64, 32), (80, 16), (64, 20), (37, 17), (512, 256), (512, 255), (128, 64), (16, 0)])
@pytest.mark.parametrize("cached", [False, True])
def test_rotary_in_place_and_with_strides(cached, dim, pairs, interleaved, dtype):
    """Queries and keys turned where they are, beside their values in one tensor, and results with places between heads and tokens: bit for bit those of a call that makes its own."""
    from paper_2302_14357_amd import rotary
    g = _gen(dim + pairs)
    for tokens, heads, kv, shift in ((1, 1, 1, 0), (9, 4, 2, 0), (2100, 3, 1, 0), (70, 5, 5, 1)):
        x = _randn(g, tokens, heads + 2 * kv, dim, dtype=dtype)
        room = torch.empty(x.numel() + shift, dtype=dtype, device="cuda")[shift:].view(x.shape).copy_(x)
        q, k, v = room[:, :heads], room[:, heads:heads + kv], room[:, heads + kv:]
        at = torch.randint(0, 5000, (tokens,), generator=g, dtype=torch.int32).cuda()
        freqs = 10000.0 ** -(torch.arange(pairs, dtype=torch.float64) / max(pairs, 1)).cuda()
        slots = torch.randperm(tokens + 9, generator=g)[:tokens].cuda()
        caches = [[torch.full((tokens // 7 + 2, 7, kv, dim), 77.0, dtype=dtype, device="cuda") for _ in range(2)] for _ in range(3)]
        kw = dict(v=v, slots=slots, k_cache=caches[0][0], v_cache=caches[0][1]) if cached else {}
        want = rotary(q, k, at, freqs, interleaved=interleaved, **kw)
        # results with room around every head
        big = torch.full((tokens + 2, heads + kv + 1, dim + 3), 77.0, dtype=dtype, device="cuda")
        q2, k2 = big[1:tokens + 1, :heads, :dim], big[1:tokens + 1, heads:heads + kv, 1:dim + 1]
        _rotary_call(q, k, v, at, freqs, slots if cached else None, *caches[1], q2, k2, interleaved)
        assert torch.equal(q2, want[0]) and torch.equal(k2, want[1]) and torch.equal(room.cpu(), x)
        q2.fill_(77.0), k2.fill_(77.0)
        assert bool((big == 77.0).all())
        # in place
        _rotary_call(q, k, v, at, freqs, slots if cached else None, *caches[2], q, k, interleaved)
        assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v.cpu(), x[:, heads + kv:])
        for i in (1, 2):
            assert torch.equal(caches[i][0], caches[0][0]) and torch.equal(caches[i][1], caches[0][1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("which", ["k", "v", "both"])
def test_prompts_rows_far_apart(which, dtype):
    """New tokens' keys or values 32 MiB apart and more: the bits of a call on rows side by side."""
    from paper_2302_14357_amd import attend_prompts
    g = _gen(4)
    tokens, heads, kv, dim = 140, 4, 2, 64
    far = torch.empty(tokens, 2**25 // dtype.itemsize + 8, dtype=dtype, device="cuda")
    assert far.stride(0) * far.element_size() * 64 > 2**31
    q, k, v = (_randn(g, tokens, n, dim, dtype=dtype).cuda() for n in (heads, kv, kv))
    kf, vf = (far[:, i:i + kv * dim].view(tokens, kv, dim).copy_(x) if which in (n, "both") else x for i, n, x in ((0, "k", k), (kv * dim, "v", v)))
    starts = _i32([0, 7, tokens])
    kc, vc = (_randn(g, 12, 16, kv, dim, dtype=dtype).cuda() for _ in range(2))
    cached = dict(past=_i32([70, 30]), k_cache=kc, v_cache=vc, tables=_i32([[0, 1, 2, 3, 4, 5], [6, 7, 8, 9, 10, 11]]))
    for kw in ({}, cached):
        assert torch.equal(attend_prompts(q, kf, vf, starts, **kw), attend_prompts(q, k, v, starts, **kw))
        for force in (1, 2):
            assert torch.equal(_prompts_by(force, q, kf, vf, starts, **kw), _prompts_by(force, q, k, v, starts, **kw))


@pytest.mark.parametrize("together", [False, True])
def test_lists_that_are_all_empty(together):
    """No hypothesis of any utterance: nothing is read and nothing found."""
    from continue_nbest import Lm, continue_nbest
    lm = Lm(40, width=64, layers=1, heads=4, kv_heads=2, dtype=torch.float32, seed=3)
    assert continue_nbest(lm, [[], []], 4, 5, page=4, together=together) == ([[], []], 0)
    got, _ = continue_nbest(lm, [[], [((3, 5), -1.0)], []], 4, 5, page=4, together=together)
    assert got[0] == got[2] == [] and got[1]
