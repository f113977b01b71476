"""Operators of an autoregressive model against plain implementations in 64 bits.

Tolerances are sums of what can be lost: half a step of the output's type (eps / 2 relative), float32 sums of n terms (n 2^-24 of the sum of
their magnitudes), and what is named where it is used.  Whole numbers, written cache entries and copied pages are equal.
"""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def _half_step(ref, dtype):
    """Half a step of the type at ref (and of its smallest numbers)."""
    return ref.abs() * (torch.finfo(dtype).eps / 2) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def _close(got, ref, tol):
    off = (got.double().cpu() - ref).abs()
    assert torch.isfinite(got.float()).all()
    assert bool((off <= tol).all()), (float((off - tol).max()), float((off / tol.clamp(min=1e-300)).max()))


# ------------------------------------------------------------------ linear

ACTS = {"none": lambda y: y, "relu": lambda y: y.clamp(min=0), "tanh": torch.tanh, "gelu": lambda y: y * torch.special.ndtr(y), "silu": lambda y: y * torch.special.expit(y)}


def _linear_case(m, n, k, dtype, act, bias, residual, out_dtype=None, seed=0, pad=(0, 0, 0, 0), shift=0):
    """pad: elements between the rows of x, weight, residual and the result; shift: elements in front of them."""
    from paper_2302_14357_amd import linear
    g = _gen(seed + m * 7 + n * 3 + k)
    odt = out_dtype or dtype

    def place(rows, cols, kind, pad_):
        return torch.empty(shift + rows * (cols + pad_), dtype=kind, device="cuda")[shift:].as_strided((rows, cols), (cols + pad_, 1))
    x, w = _randn(g, m, k, dtype=dtype), _randn(g, n, k, dtype=dtype, scale=1 / math.sqrt(k))
    b = _randn(g, n) if bias else None
    r = _randn(g, m, n, dtype=odt) if residual else None
    xd, wd = place(m, k, dtype, pad[0]).copy_(x), place(n, k, dtype, pad[1]).copy_(w)
    rd = place(m, n, odt, pad[2]).copy_(r) if residual else None
    room = torch.full((shift + m * (n + pad[3]) + 64,), 77.0, dtype=odt, device="cuda")
    out = room[shift:shift + m * (n + pad[3])].as_strided((m, n), (n + pad[3], 1)) if m * (n + pad[3]) else room[:0].view(m, n)
    got = linear(xd, wd, b.cuda() if bias else None, act=act, residual=rd, out=out)
    assert got is out
    y = x.double() @ w.double().t()
    size = x.double().abs() @ w.double().abs().t()
    if bias:
        y, size = y + b.double(), size + b.double().abs()
    # a sum of k terms and the bias; slopes of the activations are at most 1.13, their own error a few units of float32, for outputs of 16 bits 1.5e-7 of y
    # from the error function's approximation
    loss = 1.13 * (k + 1) * 2.0**-24 * size + 4e-7 * (1 + y.abs())
    y = ACTS[act](y)
    if residual:
        y = y + r.double()
    _close(got, y, loss + 2.0**-24 * y.abs() + _half_step(y, odt) * (1 + 2.0**-10))
    written = torch.zeros_like(room, dtype=torch.bool)
    written[shift:shift + m * (n + pad[3])].as_strided((m, n), (n + pad[3], 1)).fill_(True)
    assert bool((room[~written] == 77.0).all()), "something beside the result was written"
    again = linear(xd, wd, b.cuda() if bias else None, act=act, residual=rd, out_dtype=odt)
    assert torch.equal(again, got)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 16, 8), (2, 100, 37), (5, 2560, 640), (16, 64, 4096), (17, 513, 257), (33, 31, 96), (64, 1000, 512), (65, 640, 72),
                                   (100, 1028, 1024), (129, 130, 520), (320, 512, 2048), (700, 2304, 64), (1000, 333, 200), (2049, 1024, 128)])
def test_linear_sizes(m, n, k, dtype):
    _linear_case(m, n, k, dtype, "none", True, False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("m,n,k", [(3, 640, 640), (130, 260, 256), (600, 1500, 320)])
def test_linear_epilogues(m, n, k, act, dtype):
    _linear_case(m, n, k, dtype, act, True, True)
    _linear_case(m, n, k, dtype, act, False, True, seed=1)
    _linear_case(m, n, k, dtype, act, False, False, out_dtype=torch.float32, seed=2)
    _linear_case(m, n, k, dtype, act, True, True, out_dtype=torch.float32, seed=3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(4, 200, 320), (40, 77, 64), (300, 520, 192), (1100, 1026, 256)])
@pytest.mark.parametrize("pad,shift", [((1, 0, 0, 0), 0), ((0, 3, 5, 7), 0), ((8, 8, 8, 8), 0), ((0, 0, 0, 0), 1), ((8, 16, 2, 4), 3), ((0, 0, 4, 4), 4)])
def test_linear_strides_and_alignment(m, n, k, pad, shift, dtype):
    _linear_case(m, n, k, dtype, "relu", True, True, pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_gelu_far_below_zero_in_float32(dtype):
    """Where 1 + erf has lost its digits: pre-activations from -10 to -4, exact, without a residual."""
    from paper_2302_14357_amd import linear
    y = torch.linspace(-10, -4, 4000).to(dtype).view(500, 8)
    got = linear(y.cuda(), torch.eye(8, dtype=dtype, device="cuda"), act="gelu", out_dtype=torch.float32)
    ref = 0.5 * y.double() * torch.special.erfc(-y.double() * math.sqrt(0.5))   # (torch's ndtr is 1 + erf, too)
    # erfc's argument is rounded twice, each worth y^2 half steps of the result; erfc is within 16 units, the products within one each
    _close(got, ref, ref.abs() * (2 * y.double() ** 2 + 32 + 2) * 2.0**-24)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_linear_gelu_far_below_zero_in_16_bits(dtype):
    """Half a step of the type and a quarter of one: pre-activations from -10 to -4, exact, without a residual; and 0 from where nothing is left."""
    from paper_2302_14357_amd import linear
    y = torch.linspace(-10, -4, 4000).to(dtype).view(500, 8)
    eye = torch.eye(8, dtype=dtype, device="cuda")
    ref = 0.5 * y.double() * torch.special.erfc(-y.double() * math.sqrt(0.5))
    _close(linear(y.cuda(), eye, act="gelu"), ref, 1.5 * _half_step(ref, dtype))
    far = linear(torch.full((3, 8), -20.0, dtype=dtype, device="cuda"), eye, act="gelu")
    assert bool((far == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act,low,high", [("gelu", -13.0, 100.0), ("silu", -80.0, 100.0), ("tanh", -100.0, 100.0)])
def test_linear_activations_in_16_bits(act, low, high, dtype):
    """All over their range, exact pre-activations of every size: half a step of the type and a quarter of one."""
    from paper_2302_14357_amd import linear
    g = _gen(41)
    y = torch.cat([torch.linspace(low, high, 4000), torch.linspace(-6, 6, 4000), torch.exp(torch.linspace(-14, 2.5, 2000)), -torch.exp(torch.linspace(-14, 2.5, 2000)), _randn(g, 2000)])
    y = y.to(dtype).view(-1, 8)
    x = y.double()
    ref = {"gelu": 0.5 * x * torch.special.erfc(-x * math.sqrt(0.5)), "silu": x / (1 + torch.exp(-x)), "tanh": torch.tanh(x)}[act]
    _close(linear(y.cuda(), torch.eye(8, dtype=dtype, device="cuda"), act=act), ref, 1.25 * _half_step(ref, dtype))


def _linear_by(kernel, x, w, b, act, r, out):
    import ctypes
    from paper_2302_14357_amd import ops
    L = ops.load_library()
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    a = ops._Linear(x=x.data_ptr(), w=w.data_ptr(), bias=b.data_ptr(), residual=r.data_ptr(), out=out.data_ptr(), ld_x=x.stride(0), ld_w=w.stride(0),
                    ld_residual=r.stride(0), ld_out=out.stride(0), m=x.shape[0], n=w.shape[0], k=x.shape[1], dtype=code[x.dtype], out_dtype=code[out.dtype], act=ops._ACTS[act])
    return L.linear_by(ctypes.byref(a), ctypes.c_int(kernel), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kernel", [1, 11, 22, 311, 312, 321, 322, 342, 121, 142, 164, 184])
def test_linear_every_kernel(kernel, dtype):
    """One, two, several and more K tiles than a kernel has stages, pieces behind K, one past and one short of whole tiles, one row, and the float32 result."""
    for m, n, k in [(1, 4, 8), (63, 66, 64), (65, 257, 72), (129, 250, 128), (193, 520, 200), (257, 254, 328), (300, 300, 1032), (30, 515, 640), (40, 70, 4104)]:
        for act, odt in (("gelu", dtype), ("none", torch.float32)):
            g = _gen(m + n + k)
            x, w, b, r = _randn(g, m, k, dtype=dtype), _randn(g, n, k, dtype=dtype, scale=1 / math.sqrt(k)), _randn(g, n), _randn(g, m, n, dtype=odt)
            room = torch.full((m + 1, n), 77.0, dtype=odt, device="cuda")
            assert _linear_by(kernel, x.cuda(), w.cuda(), b.cuda(), act, r.cuda(), room[:m]) == 0
            torch.cuda.synchronize()
            assert bool((room[m:] == 77.0).all())
            y = x.double() @ w.double().t() + b.double()
            loss = 1.13 * (k + 1) * 2.0**-24 * (x.double().abs() @ w.double().abs().t() + b.double().abs()) + 4e-7 * (1 + y.abs())
            y = ACTS[act](y) + r.double()
            _close(room[:m], y, loss + 2.0**-24 * y.abs() + _half_step(y, odt) * (1 + 2.0**-10))


@pytest.mark.parametrize("kernel", [121, 142, 164, 184, 311, 322, 342])
def test_linear_tiles_want_alignment(kernel):
    x, w, b = torch.zeros(70, 72, dtype=torch.bfloat16, device="cuda"), torch.zeros(80, 72, dtype=torch.bfloat16, device="cuda"), torch.zeros(80, device="cuda")
    out = torch.zeros(70, 80, dtype=torch.bfloat16, device="cuda")
    assert _linear_by(kernel, x[:, :71], w[:, :71], b, "none", out, out) == -1
    assert _linear_by(kernel, x[:, 1:65], w[:, 1:65], b, "none", out, out) == -1
    assert _linear_by(99, x, w, b, "none", out, out) == -1


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_in_place_residual_leading_dimensions_and_no_rows(dtype):
    from paper_2302_14357_amd import linear
    g = _gen(3)
    x, w, r = _randn(g, 2, 3, 64, dtype=dtype).cuda(), _randn(g, 48, 64, dtype=dtype).cuda(), _randn(g, 2, 3, 48, dtype=dtype).cuda()
    want = linear(x, w, residual=r)
    assert want.shape == (2, 3, 48)
    kept = r.clone()
    assert linear(x, w, residual=r, out=r) is r and torch.equal(r, want) and not torch.equal(r, kept)
    assert linear(x[:0], w).shape == (0, 3, 48)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 3, 70])
def test_linear_results_beside_what_is_read(m, dtype):
    """Slices of one tensor beside each other, rows between rows and memory end to end are no overlap; a result over x, the weights, the bias or another residual is refused."""
    from paper_2302_14357_amd import TbsError, linear
    g, n, k = _gen(m), 48, 64
    x, w, r = _randn(g, m, k, dtype=dtype).cuda(), _randn(g, n, k, dtype=dtype).cuda(), _randn(g, m, n, dtype=dtype).cuda()
    want = linear(x, w, residual=r)
    for order in ((0, 1, 2), (2, 0, 1), (1, 2, 0)):
        room = torch.zeros(m, n + k + n, dtype=dtype, device="cuda")
        parts = dict(zip(order, room.split([(k, n, n)[i] for i in order], 1)))
        parts[0].copy_(x), parts[2].copy_(r)
        assert torch.equal(linear(parts[0], w, residual=parts[2], out=parts[1]), want)
        assert torch.equal(parts[0], x) and torch.equal(parts[2], r)
    flat = torch.zeros(m * (k + n) + n * k, dtype=dtype, device="cuda")
    xs, out, ws = flat[:m * k].view(m, k), flat[m * k:m * (k + n)].view(m, n), flat[m * (k + n):].view(n, k)
    xs.copy_(x), ws.copy_(w)
    assert torch.equal(linear(xs, ws, residual=r, out=out), want) and torch.equal(ws, w)
    square = _randn(g, k, k, dtype=dtype).cuda()
    with pytest.raises(TbsError):
        linear(x, square, out=x)
    with pytest.raises(TbsError):
        linear(xs, ws, out=flat[m * k - 1:m * (k + n) - 1].view(m, n))
    with pytest.raises(TbsError):
        linear(square[:1], square, out=square[3:4])
    b = torch.zeros(max(m * n, n), device="cuda")
    with pytest.raises(TbsError):
        linear(x.float(), w.float(), b[-n:], out=b.view(-1, n))
    wide = torch.zeros(m * n + 1, dtype=dtype, device="cuda")
    with pytest.raises(TbsError):
        linear(x, w, residual=wide[1:].view(m, n), out=wide[:-1].view(m, n))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [2, 50, 900])
def test_linear_of_numbers_that_are_none(m, dtype):
    """A row with a NaN or an infinity is none of the other rows' business; an infinity of the bias or the residual comes through."""
    from paper_2302_14357_amd import linear
    g = _gen(5)
    x, w = _randn(g, m, 128, dtype=dtype).cuda(), _randn(g, 96, 128, dtype=dtype).cuda()
    want = linear(x, w, act="relu")
    bad = x.clone()
    bad[1, 7] = math.nan
    got = linear(bad, w, act="relu")
    assert torch.isnan(got[1]).all() and torch.equal(got[0], want[0]) and torch.equal(got[2:], want[2:])
    b = torch.zeros(96, device="cuda")
    b[3] = -math.inf
    got = linear(x, w, b)
    assert bool((got[:, 3] == -math.inf).all()) and torch.isfinite(got[:, :3]).all() and torch.isfinite(got[:, 4:]).all()


# ------------------------------------------------------------------ attention over a paged cache

def _attend_by(form, q, kc, vc, tables, lens, kn, vn, beams, scale):
    """attend_paged by one way of splitting its work: form = (1 row by row or 2 hypotheses together, tokens of a piece)."""
    import ctypes
    from paper_2302_14357_amd import ops
    rows, heads, dim = q.shape
    out = torch.empty(rows, heads, dim, dtype=q.dtype, device="cuda")
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    pieces = tables.shape[1] * kc.shape[1] // form[1] + 1 if form[1] else 1024
    work = torch.full((rows * heads * pieces * (dim + 2),), math.nan, device="cuda")
    a = ops._Attend(q=q.data_ptr(), k_cache=kc.data_ptr(), v_cache=vc.data_ptr(), tables=tables.data_ptr(), lens=lens.data_ptr(), out=out.data_ptr(),
                    workspace=work.data_ptr(), workspace_bytes=work.numel() * 4, q_row=q.stride(0), q_head=q.stride(1), out_row=heads * dim, out_head=dim,
                    k_page=kc.stride(0), k_token=kc.stride(1), k_head=kc.stride(2), v_page=vc.stride(0), v_token=vc.stride(1), v_head=vc.stride(2),
                    ld_tables=tables.stride(0), rows=rows, heads=heads, kv_heads=kc.shape[2], dim=dim, page=kc.shape[1], pages=kc.shape[0],
                    table_width=tables.shape[1], beams=beams, dtype=code[q.dtype], scale=scale or 0.0)
    if kn is not None:
        a.k_new, a.v_new = kn.data_ptr(), vn.data_ptr()
        a.k_new_row, a.k_new_head, a.v_new_row, a.v_new_head = kn.stride(0), kn.stride(1), vn.stride(0), vn.stride(1)
    assert ops.load_library().attend_by(ctypes.byref(a), ctypes.c_int(form[0]), ctypes.c_int(form[1]), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    return out


def _attend_case(lens, *, form=None, heads, kv, dim, page, dtype, beams=1, shared=0, new=True, layout="token", width=0, holes=(), seed=0, max_len=None, fused=False, scale=None,
                 garbage=True, q_scale=1.0):
    """lens: tokens of every row in the cache (negative: takes no part); shared: that many pages at the head of every group are one row's; holes:
    (row, place in its table) entries that name no page."""
    from paper_2302_14357_amd import attend_paged
    g, r = _gen(seed + dim + page), np.random.default_rng(seed + len(lens))
    rows = len(lens)
    width = max(width, max(max(n, ~n) for n in lens) // page + 1)
    pages = rows * width + 3
    tables = r.permutation(pages)[:rows * width].reshape(rows, width).astype(np.int32)
    for i in range(0, rows, beams):   # (only whole pages of everybody's are shared: nobody writes them)
        common = min(shared, min(max(n, ~n) for n in lens[i:i + beams]) // page)
        tables[i:i + beams, :common] = tables[i, :common]
    for i, j in holes:
        tables[i, j] = (-1, pages, -2**31, 2**31 - 1)[(i + j) % 4]
    kc, vc = _randn(g, pages, page, kv, dim, dtype=dtype), _randn(g, pages, page, kv, dim, dtype=dtype)
    qkv = _randn(g, rows, heads + 2 * kv, dim, dtype=dtype, scale=q_scale)
    q, kn, vn = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    # what no row may look at: places behind its last token (pages are read by the rows they belong to alone, or whole)
    if garbage:
        seen = np.zeros((pages, page), bool)
        for i, n in enumerate(lens):
            for t in range(max(n, 0)):
                p = tables[i, t // page]
                if 0 <= p < pages:
                    seen[p, t % page] = True
        off = torch.from_numpy(~seen)
        kc[off], vc[off] = math.nan, math.inf
    kd, vd = kc.cuda(), vc.cuda()
    if layout == "head":   # [pages, kv_heads, page, dim] in memory
        kd, vd = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (kd, vd))
    elif layout == "both":   # keys and values of a token side by side, one element further than a 16-byte boundary
        both = torch.empty(pages * page * kv * 2 * dim + 1, dtype=dtype, device="cuda")[1:].view(pages, page, kv, 2, dim)
        kd, vd = both[..., 0, :].copy_(kd), both[..., 1, :].copy_(vd)
    qd = qkv.cuda() if fused else None
    a, b, c = (qd[:, :heads], qd[:, heads:heads + kv], qd[:, heads + kv:]) if fused else (q.contiguous().cuda(), kn.contiguous().cuda(), vn.contiguous().cuda())
    ln = torch.tensor(lens, dtype=torch.int32).cuda()
    td = torch.from_numpy(tables).cuda()
    kw = dict(k_new=b, v_new=c) if new else {}
    k0, v0 = kd.clone(), vd.clone()
    if form:
        got = _attend_by(form, a, kd, vd, td, ln, kw.get("k_new"), kw.get("v_new"), beams, scale)
    else:
        got = attend_paged(a, kd, vd, td, ln, beams=beams, max_len=max_len, scale=scale, **kw)
    # the cache: the new tokens where they belong and nothing else
    for cache, before, fresh in ((kd, k0, b), (vd, v0, c)):
        want = before.clone()
        if new:
            for i, n in enumerate(lens):
                if n >= 0 and n < width * page and 0 <= tables[i, n // page] < pages:
                    want[tables[i, n // page], n % page] = fresh[i]
        assert torch.equal(cache.nan_to_num(nan=5e4), want.nan_to_num(nan=5e4))
    ref, tol = torch.zeros(rows, heads, dim, dtype=torch.float64), torch.zeros(rows, heads, dim, dtype=torch.float64)
    s = scale if scale is not None else 1 / math.sqrt(dim)
    for i, n in enumerate(lens):
        at = [(int(tables[i, t // page]), t % page) for t in range(min(max(n, 0), width * page)) if 0 <= tables[i, t // page] < pages]
        keys = [kc[p, o] for p, o in at] + ([kn[i]] if new and 0 <= n < width * page else [])
        vals = [vc[p, o] for p, o in at] + ([vn[i]] if new and 0 <= n < width * page else [])
        if not keys:
            continue
        k, v = torch.stack(keys).double().repeat_interleave(heads // kv, 1), torch.stack(vals).double().repeat_interleave(heads // kv, 1)   # [n, heads, dim]
        x = q[i].double()
        score = s * torch.einsum("hd,nhd->hn", x, k)
        p = torch.softmax(score, 1)
        # a score's error: a float32 sum of dim terms, its scaling (two units) and the exponential's argument; a weight's rounding: two 16-bit numbers
        e = (s * (dim + 2) * 2.0**-24 * torch.einsum("hd,nhd->hn", x.abs(), k.abs())).amax(1) + score.abs().amax(1) * 2.0**-21 + 2.0**-22
        size = torch.einsum("hn,nhd->hd", p, v.abs())
        ref[i] = torch.einsum("hn,nhd->hd", p, v)
        tol[i] = (2 * e + len(keys) * 2.0**-23 + (2.0**-15 if dtype != torch.float32 else 0))[:, None] * size
    _close(got, ref, tol + _half_step(ref, dtype) * (1 + 2.0**-7) + 1e-30)
    for i, n in enumerate(lens):
        if n < 0:
            assert bool((got[i] == 0).all())
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv,dim,page", [(1, 1, 64, 16), (8, 8, 64, 16), (8, 2, 128, 32), (32, 1, 128, 16), (20, 1, 40, 7), (6, 2, 80, 1), (4, 4, 8, 5), (3, 1, 96, 48),
                                               (2, 1, 32, 64), (4, 2, 256, 16), (2, 2, 136, 12), (40, 2, 64, 100), (5, 5, 24, 3)])
def test_attend_heads_and_pages(heads, kv, dim, page, dtype):
    _attend_case([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200], heads=heads, kv=kv, dim=dim, page=page, dtype=dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [True, False])
def test_attend_rows_without_tokens_and_rows_that_take_no_part(new, dtype):
    got = _attend_case([0, ~0, 5, ~40, 0, 77, ~16], heads=4, kv=2, dim=64, page=16, dtype=dtype, new=new)
    if not new:
        assert bool((got[0] == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["token", "head", "both"])
@pytest.mark.parametrize("fused", [False, True])
def test_attend_layouts(layout, fused, dtype):
    _attend_case([3, 100, 33, 250], heads=6, kv=3, dim=72, page=24, dtype=dtype, layout=layout, fused=fused)


@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_pages_that_do_not_exist(dtype):
    _attend_case([100, 100, 5, 64, 40], heads=4, kv=2, dim=64, page=16, dtype=dtype, holes=[(0, 2), (1, 0), (1, 6), (2, 0), (3, 0), (3, 1), (3, 2), (3, 3), (3, 4), (4, 1)])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,page,max_len", [([3000], 16, None), ([3000], 16, 5), ([2047, 2048, 1], 64, 4000), ([5000, 0, ~9], 48, 5001), ([4097], 1, None)])
def test_attend_split_over_the_length(lens, page, max_len, dtype):
    """Few rows: their tokens are dealt out to several workgroups; a bound that is too small loses nothing."""
    _attend_case(lens, heads=8, kv=2, dim=64, page=page, dtype=dtype, max_len=max_len)


@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_with_a_full_table(dtype):
    """No place for the new token: the row attends to what its table holds and writes nothing."""
    from paper_2302_14357_amd import attend_paged
    g = _gen(1)
    kc, vc = _randn(g, 4, 8, 1, 32, dtype=dtype).cuda(), _randn(g, 4, 8, 1, 32, dtype=dtype).cuda()
    q, kn = _randn(g, 2, 2, 32, dtype=dtype).cuda(), _randn(g, 2, 1, 32, dtype=dtype).cuda()
    t = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32).cuda()
    before = kc.clone()
    full = attend_paged(q, kc, vc, t, torch.tensor([16, 2**31 - 1], dtype=torch.int32).cuda(), k_new=kn, v_new=kn)
    assert torch.equal(kc, before)
    assert torch.equal(full, attend_paged(q, kc, vc, t, torch.tensor([16, 16], dtype=torch.int32).cuda()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("beams,heads,kv,lens,shared,page", [(5, 8, 8, 90, 4, 16), (8, 8, 2, 700, 40, 16), (4, 32, 2, 300, 9, 32), (32, 4, 1, 130, 8, 16), (3, 2, 2, 1000, 30, 32),
                                                             (2, 40, 2, 600, 17, 32)])
def test_attend_hypotheses_that_share_pages(beams, heads, kv, lens, shared, page, dtype):
    rows = [lens] * beams + [lens // 2 + 7] * beams
    rows[1] = ~rows[1]
    for form in (None, (2, 0), (2, 128), (2, 256), (2, 1 << 20), (1, 128)):
        _attend_case(rows, form=form, heads=heads, kv=kv, dim=64, page=page, dtype=dtype, beams=beams, shared=min(shared, (lens // 2 + 7) // page))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("form", [(2, 0), (2, 128), (2, 1 << 20)])
@pytest.mark.parametrize("heads,kv,dim,page", [(1, 1, 64, 16), (16, 2, 128, 32), (40, 2, 40, 7), (6, 2, 80, 1), (3, 1, 96, 48), (8, 4, 256, 16), (9, 3, 24, 3), (2, 1, 32, 64)])
def test_attend_hypotheses_together(heads, kv, dim, page, form, dtype):
    """Groups of four with common pages, with none, all finished, without tokens, of unequal lengths, with pages that do not exist in the common part and behind it."""
    lens = [150, 150, 150, 150] + [~20, ~3, ~0, ~100] + [0, 0, 0, 0] + [130, 33, 64, 5] + [300, ~300, 300, 299]
    for shared in (0, 1, 2):
        _attend_case(lens, form=form, heads=heads, kv=kv, dim=dim, page=page, dtype=dtype, beams=4, shared=min(shared, 5 // page))
    lens = [300, 300, 301, 290]
    _attend_case(lens, form=form, heads=heads, kv=kv, dim=dim, page=page, dtype=dtype, beams=4, shared=256 // page, holes=[(i, 0) for i in range(4)] + [(2, 260 // page), (1, 40 // page)])
    _attend_case(lens, form=form, heads=heads, kv=kv, dim=dim, page=page, dtype=dtype, beams=4, shared=256 // page, new=False)
    _attend_case(lens, form=form, heads=heads, kv=kv, dim=dim, page=page, dtype=dtype, beams=2, shared=100 // page)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,dim,beams,groups", [(4, 64, 2, 140), (16, 128, 5, 130), (4, 24, 3, 129)])
def test_attend_many_groups(heads, dim, beams, groups, dtype):
    """More groups and key heads than two workgroups a CU: few waves take a group."""
    lens = np.random.default_rng(groups).integers(0, 70, groups * beams)
    lens[::7] = ~lens[::7]
    for form in ((2, 0), (1, 0), None):
        _attend_case([int(x) for x in lens], form=form, heads=heads, kv=4, dim=dim, page=4, dtype=dtype, beams=beams, shared=6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("form", [(2, 0), (2, 512), (1, 0)])
def test_attend_more_pages_than_fit_at_a_time(form, dtype):
    """Pages of one token and of three, sixteen hypotheses: their table entries pass through LDS in several turns."""
    for page, n in ((1, 300), (3, 500)):
        _attend_case([n] * 15 + [n - 5], form=form, heads=4, kv=1, dim=32, page=page, dtype=dtype, beams=16, shared=200 // page)


@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_hypotheses_of_different_lengths_and_partly_shared_pages(dtype):
    """Two of a group share, two others do too, one has nothing in common, one is shorter than what they share."""
    from paper_2302_14357_amd import attend_paged
    g, page, kv, dim = _gen(9), 16, 2, 64
    lens = [400, 400, 390, 400, 400, 100]
    width = 26
    tables = np.arange(6 * width).reshape(6, width).astype(np.int32)
    tables[1, :20] = tables[0, :20]
    tables[4, :24] = tables[2, :24]
    tables[5, :6] = tables[0, :6]
    kc, vc = _randn(g, 6 * width, page, kv, dim, dtype=dtype).cuda(), _randn(g, 6 * width, page, kv, dim, dtype=dtype).cuda()
    q, kn, vn = (_randn(g, 6, h, dim, dtype=dtype).cuda() for h in (8, kv, kv))
    td, ln = torch.from_numpy(tables).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    for i, got in [(i, g) for g in (attend_paged(q, kc, vc, td, ln, k_new=kn, v_new=vn, beams=6), _attend_by((2, 0), q, kc, vc, td, ln, kn, vn, 6, None),
                                    _attend_by((2, 128), q, kc, vc, td, ln, kn, vn, 6, None)) for i in range(6)]:
        one = attend_paged(q[i:i + 1], kc, vc, td[i:i + 1], ln[i:i + 1], k_new=kn[i:i + 1], v_new=vn[i:i + 1])
        # (each is within its own error of the same result: float32 sums in another order, weights of two 16-bit numbers, and a rounding each)
        off = (got[i].double() - one[0].double()).abs()
        step = torch.finfo(dtype).eps * one[0].double().abs() + (2.0**-14 if dtype != torch.float32 else 2.0**-15) + 1e-7
        assert bool((off <= step).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv,dim,page,n", [(8, 8, 64, 16, 200), (32, 4, 128, 32, 500), (4, 2, 40, 7, 90), (4, 2, 256, 16, 150)])
def test_attend_numbers_that_are_none_are_their_own_hypothesis_business(heads, kv, dim, page, n, dtype):
    """A NaN or an infinity among one hypothesis' own tokens, its new one or its query: the others' outputs keep their bits, its own are those it has alone."""
    from paper_2302_14357_amd import attend_paged
    g, beams, rows, width = _gen(21), 4, 8, n // page + 1
    tables = np.random.default_rng(3).permutation(rows * width).reshape(rows, width).astype(np.int32)
    for i in range(0, rows, beams):
        tables[i:i + beams, :width // 2] = tables[i, :width // 2]
    k, v = (_randn(g, rows * width, page, kv, dim, dtype=dtype) for _ in range(2))
    q, kn, vn = (_randn(g, rows, h, dim, dtype=dtype) for h in (heads, kv, kv))
    td, ln = torch.from_numpy(tables).cuda(), torch.tensor([n, n, n - 3, n] * 2, dtype=torch.int32).cuda()
    own = [(int(tables[1, t // page]), t % page) for t in (width // 2 * page, n - page - 1, n - 1)]   # row 1's own: the first, one between, the last in the cache

    def run(form, **bad):
        x = {name: t.cuda().clone() for name, t in dict(q=q, k=k, v=v, kn=kn, vn=vn).items()}
        for name, (at, value) in bad.items():
            x[name][at] = value
        args = (x["q"], x["k"], x["v"], td, ln)
        if form:
            return _attend_by(form, *args, x["kn"], x["vn"], beams, None)
        return attend_paged(*args, k_new=x["kn"], v_new=x["vn"], beams=beams)
    others = [0, 2, 3, 4, 5, 6, 7]
    for form in (None, (1, 0), (2, 0), (2, 128)):
        want = run(form)
        assert torch.isfinite(want).all()
        for value in (math.nan, math.inf, -math.inf):
            for bad in [dict(v=(own[0], value)), dict(v=(own[1], value)), dict(v=(own[2] + (0,), value)), dict(k=(own[1], value)), dict(kn=(1, value)), dict(vn=(1, value)),
                        dict(vn=((1, kv - 1, dim - 1), value)), dict(q=(1, value)), dict(k=(own[0], value), v=(own[0], value), vn=(1, -value))]:
                got = run(form, **bad)
                assert torch.equal(got[others], want[others]), (form, bad)
                assert torch.equal(torch.isfinite(got[1]), torch.isfinite(run((1, 0), **bad)[1])), (form, bad)
                assert not torch.isfinite(got[1]).all() or "k" in bad or "kn" in bad


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("beams", [1, 4])
@pytest.mark.parametrize("n", [0, 1, 31, 32, 300])
def test_attend_an_infinity_comes_through(n, beams, dtype):
    """An infinite value of a token that a row attends to makes that dimension infinite, two of both signs or a NaN make it NaN: what the formula gives."""
    from paper_2302_14357_amd import attend_paged
    g, rows, heads, kv, dim, page = _gen(31), 4, 4, 2, 64, 16
    width = n // page + 1
    tables = torch.arange(rows * width, dtype=torch.int32).view(rows, width)
    k, v = (_randn(g, rows * width, page, kv, dim, dtype=dtype) for _ in range(2))
    q, kn, vn = (_randn(g, rows, h, dim, dtype=dtype) for h in (heads, kv, kv))
    vn[0] = math.inf
    vn[1, 0, 5], vn[1, 1, 6] = -math.inf, math.nan
    if n:
        v[tables[2, 0], 0, 1] = math.inf
        v[tables[3, (n - 1) // page], (n - 1) % page, :, 7:9] = torch.tensor([math.inf, -math.inf], dtype=dtype)
        vn[3, 1, 7] = -math.inf
    got = attend_paged(q.cuda(), k.cuda(), v.cuda(), tables.cuda(), torch.full((rows,), n, dtype=torch.int32).cuda(), k_new=kn.cuda(), v_new=vn.cuda(), beams=beams).cpu()
    for r in range(rows):
        keys, vals = (torch.cat([c[tables[r].long()].reshape(-1, kv, dim)[:n], x[r][None]]).double().repeat_interleave(heads // kv, 1) for c, x in ((k, kn), (v, vn)))
        p = torch.softmax((q[r].double() * keys).sum(2) / math.sqrt(dim), 0)
        want = (p[:, :, None] * vals).sum(0)
        assert torch.equal(torch.isnan(got[r]), torch.isnan(want)) and torch.equal(got[r] == math.inf, want == math.inf) and torch.equal(got[r] == -math.inf, want == -math.inf)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("beams,n", [(1, 40), (4, 40), (4, 3000)])
def test_attend_into_the_queries_place(beams, n, dtype):
    """The result may be q itself, also as a slice beside the new keys and values."""
    from paper_2302_14357_amd import attend_paged
    g, rows, heads, kv, dim, page = _gen(51), 4, 6, 2, 64, 16
    width = n // page + 1
    tables, lens = torch.randperm(rows * width, generator=g).int().view(rows, width).cuda(), torch.full((rows,), n, dtype=torch.int32).cuda()
    k, v = (_randn(g, rows * width, page, kv, dim, dtype=dtype).cuda() for _ in range(2))
    qkv = _randn(g, rows, heads + 2 * kv, dim, dtype=dtype).cuda()
    q, kn, vn = qkv.split((heads, kv, kv), 1)
    want = attend_paged(q, k, v, tables, lens, k_new=kn, v_new=vn, beams=beams)
    kept = qkv[:, heads:].clone()
    assert attend_paged(q, k, v, tables, lens, k_new=kn, v_new=vn, beams=beams, out=q) is q
    assert torch.equal(q, want) and torch.equal(qkv[:, heads:], kept)


@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_large_scores(dtype):
    """Weights of one token alone, of equal scores, and scores whose exponentials would overflow."""
    _attend_case([70, 130, 10], heads=4, kv=2, dim=64, page=16, dtype=dtype, q_scale=30.0)
    _attend_case([70, 130, 10], heads=4, kv=2, dim=64, page=16, dtype=dtype, q_scale=0.0)
    _attend_case([70, 130, 10], heads=4, kv=2, dim=64, page=16, dtype=dtype, scale=4.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_offsets_beyond_32_bits(dtype):
    """Pages whose place in the cache is more than 2^31 elements from its start."""
    from paper_2302_14357_amd import attend_paged
    g, page, kv, dim = _gen(11), 64, 1, 128
    pages = 2**31 // (page * kv * dim) + 1000
    small = [_randn(g, 8, page, kv, dim, dtype=dtype).cuda() for _ in range(2)]
    big = [torch.empty(pages, page, kv, dim, dtype=dtype, device="cuda") for _ in range(2)]
    place = torch.tensor([0, pages - 1, pages - 500, 3, pages - 999, pages - 2, 9, pages - 700])
    for b, s in zip(big, small):
        b[place.cuda()] = s
    q, kn = _randn(g, 1, 2, dim, dtype=dtype).cuda(), _randn(g, 1, 1, dim, dtype=dtype).cuda()
    ln = torch.tensor([8 * page - 3], dtype=torch.int32).cuda()
    want = attend_paged(q, *small, torch.arange(8, dtype=torch.int32)[None].cuda(), ln, k_new=kn, v_new=kn)
    got = attend_paged(q, *big, place.int()[None].cuda(), ln, k_new=kn, v_new=kn)
    assert torch.equal(got, want) and torch.equal(big[0][place[7], page - 3], kn[0])


# ------------------------------------------------------------------ selection

def _select_ref(logits, scores, finished, beams, eos):
    """The definition, in float64, with sorted lists."""
    out = []
    l = logits.double().numpy()
    for g in range(0, len(l), beams):
        cand = []
        for r in range(beams):
            s, x = float(scores[g + r]), l[g + r]
            if finished[g + r]:
                cand.append((s, r, 0, eos))
                continue
            if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any():
                continue
            top = x.max()
            lse = top + math.log(np.exp(x - top).sum())
            order = np.lexsort((np.arange(len(x)), -x))[:beams]
            cand += [(s + (float(x[v]) - lse), r, i, int(v)) for i, v in enumerate(order)]
        cand = sorted((c for c in cand if c[0] > -np.inf), key=lambda c: (-c[0], c[1], c[2]))[:beams]
        out += [(s, v, r, bool(v == eos or finished[g + r])) for s, r, _, v in cand] + [(-np.inf, -1, -1, True)] * (beams - len(cand))
    return out


def _select_check(logits, scores, finished, beams, eos, stride=None, shift=0):
    from paper_2302_14357_amd import beam_select
    rows, vocab = logits.shape
    stride = stride or vocab
    ld = torch.empty(shift + rows * stride, dtype=logits.dtype, device="cuda")[shift:].as_strided((rows, vocab), (stride, 1)).copy_(logits)
    fd = None if finished is None else finished.cuda()
    s, t, p, f = (x.cpu() for x in beam_select(ld, scores.cuda(), beams=beams, finished=fd, eos=eos))
    want = _select_ref(logits, scores, torch.zeros(rows, dtype=torch.bool) if finished is None else finished, beams, eos)
    assert t.tolist() == [w[1] for w in want]
    assert p.tolist() == [w[2] for w in want]
    assert f.tolist() == [w[3] for w in want]
    ref = np.array([w[0] for w in want])
    fine = np.isfinite(ref)
    assert np.array_equal(s.numpy()[~fine], ref[~fine])
    # the normaliser's exponentials are within 2e-12 of theirs, its sum and logarithm within a few units of float64
    assert np.all(np.abs(s.numpy()[fine] - ref[fine]) <= 4e-12 + 2.0**-50 * np.abs(ref[fine]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("groups,beams,vocab", [(1, 1, 1), (1, 1, 2), (3, 2, 3), (1, 5, 3), (2, 7, 2), (2, 5, 32), (4, 1, 1000), (3, 5, 1024), (2, 10, 1025), (1, 32, 31), (2, 32, 4096),
                                                (2, 16, 8191), (2, 16, 2048), (1, 17, 2048), (2, 16, 2049), (1, 1, 2047), (3, 16, 5), (2, 5, 8192), (2, 5, 8193), (1, 4, 50257), (40, 8, 9000), (1, 3, 262144), (130, 5, 700), (1, 32, 524288)])
def test_select_sizes(groups, beams, vocab, dtype):
    g = _gen(groups + beams + vocab)
    rows = groups * beams
    _select_check(_randn(g, rows, vocab, dtype=dtype, scale=3.0), -10 * torch.rand(rows, generator=g, dtype=torch.float64), None, beams, vocab - 1)


@pytest.mark.parametrize("dtype", DTYPES)
def test_select_equal_logits_and_scores(dtype):
    """All logits equal, a few values only, equal rows with equal scores: the lower row, then the lower token."""
    g = _gen(4)
    zero = torch.zeros(12, dtype=torch.float64)
    for vocab in (5, 300, 2048, 5000, 20000, 100000):
        _select_check(torch.full((12, vocab), 1.5, dtype=dtype), zero, None, 6, 0)
        _select_check(torch.randint(0, 3, (12, vocab), generator=g).to(dtype), zero - torch.arange(12), None, 6, 1)
        one = _randn(g, 1, vocab, dtype=dtype)
        _select_check(one.expand(12, vocab).contiguous(), zero, None, 4, 1)
        signed = torch.zeros(12, vocab, dtype=dtype)
        signed[:, ::2] = -0.0
        _select_check(signed, zero, None, 3, 1)
        rising = torch.arange(vocab).to(dtype).expand(12, vocab).contiguous()
        _select_check(rising, zero, None, 6, 1)
        _select_check(rising.flip(1).contiguous(), zero, None, 6, 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [40, 9001])
def test_select_finished_masked_and_absent(vocab, dtype):
    g = _gen(6)
    beams, rows = 5, 40
    l = _randn(g, rows, vocab, dtype=dtype, scale=4.0)
    s = -5 * torch.rand(rows, generator=g, dtype=torch.float64)
    f = torch.zeros(rows, dtype=torch.bool)
    f[[1, 2, 7, 8, 9]] = True
    f[10:15] = True                                   # a group that is done
    l[f] = math.nan                                   # (nobody looks at it)
    s[16:20] = -math.inf                              # a first step: one hypothesis
    s[20:25] = -math.inf                              # nothing at all
    s[12] = -math.inf                                 # finished, and not there
    l[25, 3:] = -math.inf                             # masks
    l[26, :] = -math.inf
    l[27, :] = torch.finfo(dtype).min                 # the type's lowest value: a candidate like another
    l[28, 1:] = torch.finfo(dtype).min
    l[29, 5] = math.nan
    l[30, 5] = math.inf
    l[31:35] = -math.inf
    l[31, vocab - 1] = 0.0                            # one candidate in its group but for row 30's
    s[36] = math.nan
    _select_check(l, s, f, beams, 2)
    _select_check(l, s, f, beams, -1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("stride,shift", [(1001, 0), (1008, 0), (1000, 1), (1003, 3), (1016, 8)])
def test_select_strides(stride, shift, dtype):
    g = _gen(8)
    _select_check(_randn(g, 9, 1000, dtype=dtype), -torch.rand(9, generator=g, dtype=torch.float64), None, 3, 5, stride=stride, shift=shift)


@pytest.mark.parametrize("dtype", DTYPES)
def test_select_peaked_and_wide_logits(dtype):
    """One token that has nearly everything, and logits from one end of the type to the other."""
    g = _gen(10)
    l = _randn(g, 6, 3000, dtype=dtype)
    l[:, 17] = 60.0
    l[3] = _randn(g, 3000, dtype=dtype, scale=1.0) * (0.1 * torch.finfo(dtype).max if dtype == torch.float16 else 1e4)
    l[4, :] = -torch.finfo(dtype).max
    l[4, 9] = torch.finfo(dtype).max
    _select_check(l, -torch.rand(6, generator=g, dtype=torch.float64), None, 3, 17)


# ------------------------------------------------------------------ reordering of paged states

def _reorder_ref(parents, tables, lens, finished, caches, beams, page, appended=1):
    """Plain loops over places."""
    rows, width = tables.shape
    t, n, drop = tables.copy(), lens.copy(), 0
    caches = [c.clone() for c in caches]
    old = [c.clone() for c in caches]
    now = np.minimum(np.where(lens >= 0, np.where(lens < width * page, lens + appended, width * page), ~lens), width * page)
    for g in range(0, rows, beams):
        ps = [int(p) if 0 <= p < beams else -1 for p in parents[g:g + beams]]
        left = [q for q in range(beams) if q not in ps]
        taken = set()
        for c, p in enumerate(ps):
            if p >= 0 and p not in taken:
                taken.add(p)
                t[g + c], n[g + c] = tables[g + p], now[g + p]
            else:
                q = left.pop(0)
                t[g + c], n[g + c] = tables[g + q], -1
                if p < 0:
                    continue
                whole = now[g + p] // page
                if any(tables[g + r, j] == tables[g + q, j] for j in range(whole, min(now[g + q] // page, width)) for r in range(beams) if r != q):
                    drop += 1
                    continue
                t[g + c, :whole] = tables[g + p, :whole]
                n[g + c] = now[g + p]
                k = now[g + p] % page
                if k and whole < width:
                    for x, y in zip(caches, old):
                        x[t[g + c, whole], :k] = y[tables[g + p, whole], :k]
            if finished is not None and finished[g + c] and n[g + c] >= 0:
                n[g + c] = ~n[g + c]
    return t, n, caches, drop


def _reorder_check(parents, lens, *, beams, page, width, kv=2, dim=16, dtype=torch.float32, layers=2, finished=None, appended=True, layout="token", seed=0, same=()):
    """same: (row, other, n): the first n pages of `row` are those of `other`."""
    from paper_2302_14357_amd import beam_reorder
    g, r = _gen(seed), np.random.default_rng(seed)
    parents, lens = np.asarray(parents, np.int32), np.asarray(lens, np.int32)
    rows = len(parents)
    tables = r.permutation(rows * width).reshape(rows, width).astype(np.int32)
    for row, other, n in same:
        tables[row, :n] = tables[other, :n]
    caches = [_randn(g, rows * width, page, kv, dim, dtype=dtype) for _ in range(2 * layers)]
    on = [c.cuda() for c in caches]
    if layout == "head":
        on = [c.transpose(1, 2).contiguous().transpose(1, 2) for c in on]
    elif layout == "odd":
        on = [torch.empty(rows * width, page, kv, dim + 3, dtype=dtype, device="cuda")[..., 1:dim + 1].copy_(c) for c in on]
    fd = None if finished is None else torch.tensor(finished).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    t, n = beam_reorder(torch.from_numpy(parents).cuda(), torch.from_numpy(tables).cuda(), torch.from_numpy(lens).cuda(), on, beams=beams, finished=fd, appended=appended,
                        status=status)
    wt, wn, wc, drop = _reorder_ref(parents, tables, lens, finished, caches, beams, page, int(appended))
    assert np.array_equal(n.cpu().numpy(), wn)
    assert np.array_equal(t.cpu().numpy(), wt)
    for x, y in zip(on, wc):
        assert torch.equal(x.cpu(), y)
    assert status.item() == drop
    return drop


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("beams,page,n", [(1, 4, 9), (2, 4, 0), (2, 1, 3), (5, 16, 50), (5, 16, 47), (5, 16, 48), (8, 7, 20), (16, 64, 100), (32, 3, 10)])
@pytest.mark.parametrize("layout", ["token", "head", "odd"])
def test_reorder(beams, page, n, layout, dtype):
    r = np.random.default_rng(beams * 100 + n)
    parents = np.concatenate([r.integers(0, beams, beams) for _ in range(3)] + [np.arange(beams), np.zeros(beams, int), np.arange(beams)[::-1]])
    _reorder_check(parents, [n] * len(parents), beams=beams, page=page, width=(n + 2) // page + 1, dtype=dtype, layout=layout)
    _reorder_check(parents, [n] * len(parents), beams=beams, page=page, width=(n + 2) // page + 1, dtype=dtype, layout=layout, appended=False)


def test_reorder_finished_absent_and_full():
    # a first step: one row, four that do not exist; then finished ones that move; a group whose places are all empty; parents out of range
    assert _reorder_check([0, 0, 0, 0, 0], [30, -1, -1, -1, -1], beams=5, page=8, width=5) == 0
    assert _reorder_check([2, 0, 0, 4, 1], [21, ~13, 21, ~8, 21], beams=5, page=8, width=4, finished=[False, True, False, False, True]) == 0
    assert _reorder_check([-1] * 5, [30, ~3, -1, 30, 30], beams=5, page=8, width=5, finished=[True] * 5) == 0
    assert _reorder_check([0, 7, -3, 0, 2**31 - 1], [30] * 5, beams=5, page=8, width=5) == 0
    # the table is full: nothing was appended, nothing is copied
    assert _reorder_check([0, 0, 1], [16, 16, 16], beams=3, page=8, width=2) == 0
    assert _reorder_check([0, 0, 1], [2**31 - 1, 16, ~(2**31 - 1)], beams=3, page=8, width=2) == 0
    # a row with two children that is shorter than the one without, whose pages are its own; shares them with another up to there; beyond that: dropped
    assert _reorder_check([0, 0, 1], [3, 3, 30], beams=3, page=8, width=5) == 0
    assert _reorder_check([0, 0, 1], [11, 30, 30], beams=3, page=8, width=5, same=[(2, 1, 1)]) == 0
    assert _reorder_check([0, 0, 1], [11, 30, 30], beams=3, page=8, width=5, same=[(2, 1, 2)]) == 1
    assert _reorder_check([1, 1, 1, 2], [30, 4, 12, 19], beams=4, page=8, width=5, same=[(3, 0, 1)]) == 2   # (both rows that give pages name the first)
    assert _reorder_check([0, 0, 0, 0], [0, 39, 39, 39], beams=4, page=8, width=5, same=[(2, 1, 3)]) == 2


def _reorder_many_steps(seed, *, groups, beams, page, steps, absent, heirs, ended=0.05):
    """Groups of hypotheses of different lengths, step by step with random parents, places that are empty (`absent` of them) and ones that end.  A cache's entries are
    the tokens themselves; every hypothesis' tokens are kept beside it in a list.  heirs: places of length -1 are parents as well.  Returns (dropped, empty)."""
    from paper_2302_14357_amd import beam_reorder
    r = np.random.default_rng(seed)
    rows, width = groups * beams, 16 // page + -(-steps // page) + 1
    tables = r.permutation(rows * width).reshape(rows, width).astype(np.int32)
    lens = np.where(r.random(rows) < 0.2, -1, r.integers(0, 14, rows)).astype(np.int32)
    cache = torch.full((rows * width, page, 1, 1), -7.0, device="cuda")
    said, count, status = [[] for _ in range(rows)], 0, torch.zeros(1, dtype=torch.int32, device="cuda")
    drops = empty = 0
    for step in range(-1, steps):
        # tokens to places of their rows: the given ones, then one a step for those that take part
        new = [(i, t) for i in range(rows) for t in (range(max(lens[i], 0)) if step < 0 else [lens[i]] * int(lens[i] >= 0))]
        for i, _ in new:
            count += 1
            said[i] = said[i] + [count]
        at = np.array([(tables[i, t // page], t % page) for i, t in new], np.int64).reshape(-1, 2)
        assert step < 0 or len({tuple(a) for a in at}) == len(at)
        cache[torch.from_numpy(at[:, 0]), torch.from_numpy(at[:, 1])] = torch.arange(count - len(new) + 1, count + 1, device="cuda")[:, None, None].float()
        if step < 0:
            continue
        parents = np.where(r.random(rows) < absent, -1, r.integers(0, beams, rows)).astype(np.int32)
        first = np.arange(rows) // beams * beams
        if not heirs:   # a place whose parent is without a hypothesis has none itself
            parents[(parents >= 0) & (lens[first + np.maximum(parents, 0)] == -1)] = -1
        done = r.random(rows) < ended
        t, n = beam_reorder(torch.from_numpy(parents).cuda(), torch.from_numpy(tables).cuda(), torch.from_numpy(lens).cuda(), [cache], beams=beams,
                            finished=torch.from_numpy(done).cuda(), status=status)
        before, tables, lens = lens, t.cpu().numpy(), n.cpu().numpy()
        said = [list(said[f + p]) if p >= 0 else [] for f, p in zip(first, parents)]
        lost = [i for i in range(rows) if lens[i] == -1 and parents[i] >= 0 and before[first[i] + parents[i]] != -1]
        drops, empty = drops + len(lost), empty + int((lens == -1).sum())
        assert status.item() == drops
        held = cache.cpu().numpy().reshape(-1, page)
        for i in range(rows):
            if parents[i] < 0 or (heirs and before[first[i] + parents[i]] == -1):
                assert lens[i] == -1
            if lens[i] == -1:
                said[i] = []
                continue
            k = max(lens[i], ~lens[i])
            assert k == len(said[i]) and held[tables[i, :-(-k // page)]].reshape(-1)[:k].tolist() == said[i], (step, i)
            own = set(tables[i, k // page:].tolist())   # what it goes on to write is no other hypothesis'
            for q in range(first[i], first[i] + beams):
                assert q == i or lens[q] == -1 or not own & set(tables[q].tolist()), (step, i, q)
    return drops, empty


@pytest.mark.parametrize("absent", [0.0, 0.1, 0.4])
@pytest.mark.parametrize("beams,page", [(2, 1), (3, 4), (4, 4), (8, 3)])
def test_reorder_step_by_step_overwrites_nobody(beams, page, absent):
    """Different lengths, empty places, dropped ones that give their pages on: every hypothesis that is there holds its tokens, and its pages to come are its own."""
    drops, empty = _reorder_many_steps(beams * 10 + page, groups=60, beams=beams, page=page, steps=20, absent=absent, heirs=False)
    assert empty > 0 and (drops > 0 or beams == 2 or absent > 0)   # (groups with empty places die out early)


@pytest.mark.parametrize("absent", [0.0, 0.1])
@pytest.mark.parametrize("beams,page", [(2, 1), (3, 4), (4, 4), (8, 3)])
def test_reorder_a_place_without_a_hypothesis_has_no_heirs(beams, page, absent):
    """Dropped and empty places as parents: their children have the length -1, and never a place in a living hypothesis' pages."""
    drops, empty = _reorder_many_steps(beams * 10 + page + 1, groups=60, beams=beams, page=page, steps=20, absent=absent, heirs=True)
    assert empty > 0


def test_reorder_children_of_no_hypothesis():
    from paper_2302_14357_amd import beam_reorder
    tables, lens = torch.arange(24, dtype=torch.int32).view(4, 6).cuda(), torch.tensor([20, -1, 7, ~9], dtype=torch.int32).cuda()
    for finished in (None, torch.tensor([False, True, False, True]).cuda()):
        for appended in (True, False):
            cache, status = torch.zeros(24, 4, 1, 8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
            t, n = beam_reorder(torch.tensor([1, 1, 0, 3], dtype=torch.int32).cuda(), tables, lens, [cache], beams=4, finished=finished, appended=appended, status=status)
            assert n.tolist() == [-1, -1, 20 + appended, 9 if finished is None else ~9] and status.item() == 0
            assert t[2].tolist() == tables[0].tolist() and t[3].tolist() == tables[3].tolist()
            assert sorted(t[:2].reshape(-1).tolist()) == tables[1:3].reshape(-1).tolist()   # (pages of the rows without children: nobody's get lost)


def test_reorder_gives_no_page_on_that_another_names():
    """Two steps: the first leaves a place that is dropped, or empty, with pages that a living hypothesis names; the second must not give them to another."""
    from paper_2302_14357_amd import beam_reorder
    for lens, first, second in (([11, 30, 30], [0, 0, 1], [0, 0, 2]), ([20, 20, 9], [0, -1, 2], [0, 2, 2])):
        page, width = 8, 6
        tables = np.arange(3 * width).reshape(3, width).astype(np.int32)
        if first[1] == 0:
            tables[2, :2] = tables[1, :2]
        else:
            tables[1, :2] = tables[0, :2]
        cache = torch.arange(3 * width * page, device="cuda").float().view(3 * width, page, 1, 1)
        t, n, status = torch.from_numpy(tables).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
        kept = 1 if first[1] == 0 else 0   # the hypothesis (its row at the start) that both steps keep
        length = lens[kept]
        want = cache[t[kept].long()].reshape(-1)[:length].tolist()
        for parents in (first, second):
            t, n = beam_reorder(torch.tensor(parents, dtype=torch.int32).cuda(), t, n, [cache], beams=3, status=status)
        place = 2 if kept == 1 else 0
        assert n[place].item() == length + 2
        assert cache[t[place].long()].reshape(-1)[:length].tolist() == want
        assert n[1 if kept == 1 else 2].item() == -1 or not set(t[1].tolist()) & set(t[place].tolist())


def test_reorder_many_caches():
    _reorder_check([0, 0, 1, 1], [5, 5, 9, 9], beams=2, page=4, width=4, layers=70)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_beam_decode_keeps_every_hypothesis(dtype):
    """Forty steps of attention, selection and reordering: every hypothesis' cache, read through its table, is the tokens it was made of, and its attention
    is that over a cache of its own."""
    from paper_2302_14357_amd import attend_paged, beam_reorder, beam_select
    g, beams, utts, page, kv, heads, dim, vocab, steps = _gen(12), 4, 3, 8, 2, 4, 32, 50, 40
    rows, width = beams * utts, steps // page + 2
    tables = torch.randperm(rows * width, generator=g).int().view(rows, width).cuda()
    kc, vc = (torch.full((rows * width, page, kv, dim), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    emb_k, emb_v = _randn(g, vocab, kv, dim, dtype=dtype).cuda(), _randn(g, vocab, kv, dim, dtype=dtype).cuda()
    table = _randn(g, vocab, vocab, scale=2.0)
    table[:, 0] -= 2.5                               # token 0 ends a hypothesis now and then
    table = table.cuda()
    lens = torch.full((rows,), -1, dtype=torch.int32)
    lens[::beams] = 0
    lens = lens.cuda()
    scores = torch.full((rows,), -math.inf, dtype=torch.float64)
    scores[::beams] = 0.0
    scores, done = scores.cuda(), torch.zeros(rows, dtype=torch.bool, device="cuda")
    last = torch.arange(rows).cuda() % vocab
    said = [[] for _ in range(rows)]
    for step in range(steps):
        q = _randn(g, rows, heads, dim, dtype=dtype).cuda()
        out = attend_paged(q, kc, vc, tables, lens, k_new=emb_k[last], v_new=emb_v[last], beams=beams)
        alive = [int(n) >= 0 for n in lens]
        for r in range(rows):
            if alive[r]:
                said[r] = said[r] + [int(last[r])]
                if step % 7 == 0:
                    mine = torch.tensor(said[r]).cuda()
                    n = len(said[r])
                    own = [torch.cat([e[mine], torch.zeros((-n) % page, kv, dim, dtype=dtype, device="cuda")]).view(-1, page, kv, dim) for e in (emb_k, emb_v)]
                    alone = attend_paged(q[r:r + 1], *own, torch.arange(own[0].shape[0], dtype=torch.int32)[None].cuda(), torch.tensor([n], dtype=torch.int32).cuda())
                    off = (alone[0].double() - out[r].double()).abs()
                    assert bool((off <= torch.finfo(dtype).eps * alone[0].double().abs() + (2.0**-14 if dtype != torch.float32 else 2.0**-15) + 1e-7).all())
        logits = table[last] + 0.01 * torch.randn(rows, vocab, generator=g).cuda()
        scores, tok, par, done = beam_select(logits, scores, beams=beams, finished=done, eos=0)
        tables, lens = beam_reorder(par, tables, lens, [kc, vc], beams=beams, finished=done)
        p = par.cpu()
        said = [list(said[r - r % beams + int(p[r])]) if p[r] >= 0 else [] for r in range(rows)]
        last = tok.long().clamp(min=0)
        for r in range(rows):
            n = int(lens[r])
            if n < 0:
                continue
            assert n == len(said[r])
            mine = torch.tensor(said[r]).cuda()
            pages = tables[r, :-(-n // page)].long()
            assert torch.equal(kc[pages].reshape(-1, kv, dim)[:n], emb_k[mine]) and torch.equal(vc[pages].reshape(-1, kv, dim)[:n], emb_v[mine])
        first = tables.cpu().numpy()
        for u in range(utts):   # own pages are nobody else's
            own = [set(first[r, (max(int(lens[r]), ~int(lens[r]))) // page:].tolist()) for r in range(u * beams, (u + 1) * beams) if int(lens[r]) >= 0]
            assert all(not a & b for i, a in enumerate(own) for b in own[:i])


def test_what_a_call_writes_has_a_new_version():
    """Autograd's count of writes goes up where a call writes a tensor of the caller's, and only there; tensors made in inference mode have none."""
    from paper_2302_14357_amd import attend_paged, beam_reorder, linear
    x, w, out = torch.zeros(3, 8, device="cuda"), torch.zeros(4, 8, device="cuda"), torch.zeros(3, 4, device="cuda")
    q, kn, k, v = torch.zeros(2, 2, 8, device="cuda"), torch.zeros(2, 1, 8, device="cuda"), torch.zeros(4, 4, 1, 8, device="cuda"), torch.zeros(4, 4, 1, 8, device="cuda")
    tables, lens, status = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2), torch.ones(2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    parents, layers = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 4, 4, 1, 8, device="cuda")
    o = torch.zeros(2, 2, 8, device="cuda")
    for call, changed in [(lambda: linear(x, w), []), (lambda: linear(x, w, residual=out, out=out), [out]), (lambda: attend_paged(q, k, v, tables, lens), []),
                          (lambda: attend_paged(q, k, v, tables, lens, k_new=kn, v_new=kn, out=o), [k, v, o]), (lambda: beam_reorder(parents, tables, lens, [k, v], beams=2, status=status), [k, v, status]),
                          (lambda: beam_reorder(parents, tables, lens, layers, beams=2), [layers])]:
        tensors = [x, w, out, q, kn, k, v, tables, lens, status, parents, layers, o]
        before = [t._version for t in tensors]
        call()
        assert [t._version - b for t, b in zip(tensors, before)] == [int(any(t is c for c in changed)) for t in tensors]
    with torch.inference_mode():
        k, v = torch.zeros(4, 4, 1, 8, device="cuda"), torch.zeros(4, 4, 1, 8, device="cuda")
        attend_paged(q, k, v, tables, lens, k_new=kn, v_new=kn)
    attend_paged(q, k, v, tables, lens, k_new=kn, v_new=kn)
    beam_reorder(parents, tables, lens, (k, v), beams=2)


# ------------------------------------------------------------------ streams and graphs

def _step(s):
    from paper_2302_14357_amd import attend_paged, beam_reorder, beam_select, linear
    x = linear(s["x"], s["w"], s["b"], act="gelu")
    qkv = linear(x, s["wq"]).view(s["rows"], -1, s["dim"])
    o = attend_paged(qkv[:, :8], s["k"], s["v"], s["tables"], s["lens"], k_new=qkv[:, 8:10], v_new=qkv[:, 10:], beams=s["beams"])
    logits = linear(linear(o.view(s["rows"], -1), s["wo"], residual=x), s["wl"], out_dtype=torch.float32)
    sel = beam_select(logits, s["scores"], beams=s["beams"], eos=3)
    return [o, logits, *sel, *beam_reorder(sel[2], s["tables"], s["lens"], [s["k"], s["v"]], beams=s["beams"], finished=sel[3])]


def _state(seed, dtype=torch.bfloat16, rows=20, beams=5, d=256, dim=32, page=16, n=3000):
    g = _gen(seed)
    width = n // page + 2
    c = lambda *s, scale=1.0, kind=dtype: _randn(g, *s, dtype=kind, scale=scale).cuda()   # noqa: E731
    return dict(rows=rows, beams=beams, dim=dim, x=c(rows, d), w=c(d, d, scale=0.06), b=c(d, kind=torch.float32), wq=c(12 * dim, d, scale=0.06), wo=c(d, 8 * dim, scale=0.06),
                wl=c(999, d, scale=0.06), k=c(rows * width, page, 2, dim), v=c(rows * width, page, 2, dim),
                tables=torch.randperm(rows * width, generator=g).int().view(rows, width).cuda(), lens=torch.full((rows,), n, dtype=torch.int32).cuda(),
                scores=-torch.rand(rows, generator=g, dtype=torch.float64).cuda())


def test_operators_on_another_stream():
    want = _step(_state(1))
    s = _state(1)   # (a step changes its state: pages of hypotheses that are gone are written)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _step(s)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_operators_in_a_graph():
    """One step captured and replayed on other inputs, with eager work in between: every replay gives what the eager step gives."""
    s = _state(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(s)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(s)
    for seed in (3, 4, 5):
        other = _state(seed)
        for k, v in other.items():
            if torch.is_tensor(v):
                s[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out] + [s["k"].clone(), s["v"].clone()]
        want = _step(other) + [other["k"], other["v"]]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
