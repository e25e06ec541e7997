"""Operators over a paged cache on the GPU against the plain 64-bit form (tests/paged_plain.py)."""
import ctypes as C
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2604_10900_amd as cask  # noqa: E402
from synth import caches  # noqa: E402
from tests import paged_plain as plain  # noqa: E402
from tests import parity  # noqa: E402

B = cask.binding


def _bytes(t):
    return t.contiguous().view(torch.uint8)


def _same(a, b):
    return torch.equal(_bytes(a), _bytes(b))


# ---------------------------------------------------------------- rows in and out

def _hard_rows(n, d, dtype, seed):
    """Rows of every magnitude, zeros, denormals, infinities and NaN, and rows whose quotients are ties."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, d, generator=g) * torch.exp2(torch.randint(-12, 12, (n, 1), generator=g).float())
    kind = torch.randint(0, 12, (n,), generator=g)
    x[kind == 0] = 0.0
    x[kind == 1] *= 2.0 ** -130
    x[kind == 2] *= 2.0 ** 110
    x[kind == 3, 5] = float("inf")
    x[kind == 4, 7] = float("nan")
    x[kind == 5] = -float("inf")
    tie = kind >= 8    # 448 x / a exactly between two values: a = 7 b, x = b m, m odd in 17 .. 31
    b = 2 * torch.randint(0, 4, (n, 1), generator=g).float() + 1
    m = 2 * torch.randint(8, 16, (n, d), generator=g).float() + 1
    ties = b * m * torch.exp2(torch.randint(-6, -1, (n, d), generator=g).float())
    ties[:, 0] = 7 * b[:, 0] * 8
    x[tie] = ties[tie]
    return x.to(plain.TORCH[dtype])


@pytest.mark.parametrize("dtype,cache,d,page_rows,interleaved", [
    ("bf16", "e4m3", 128, 64, False), ("bf16", "e4m3", 64, 16, True), ("f32", "e4m3", 128, 32, True), ("f32", "e4m3", 64, 64, False),
    ("bf16", "bf16", 128, 16, True), ("bf16", "bf16", 64, 128, False), ("f32", "f32", 64, 16, True), ("f32", "f32", 128, 64, False)])
def test_rows_written_and_read_back(dtype, cache, d, page_rows, interleaved):
    """Every row at its place with the definition's values, every other row as it was; read back, the values that a row
    stands for.  The rows of a unit start at any place, some beyond its capacity or in front of it, one of its pages is
    missing, one entry lies outside the pools, and one unit's rows lie partly outside the call's arrays."""
    pages = plain.make(dtype, cache, d, G=1, units=5, page_rows=page_rows, cap_pages=4, seed=d + page_rows, interleaved=interleaved)
    cap = 4 * page_rows
    pages.table[1, 1] = -1
    pages.table[1, 2] = pages.K.shape[0]
    n, start = [cap, cap - 3, 0, 7, 40], [0, 1, 5, cap - 4, -6]
    total = sum(n) + 9
    first = [0, n[0], 3, total - 4, n[0] + n[1]]     # (unit 3: its last rows are behind the arrays)
    n[3] = 6
    before = plain.host(pages)
    x = [_hard_rows(total, d, dtype, s) for s in (1, 2)]
    r = plain.rows(n, start, first)
    cask.cache_write(pages, r, x[0].cuda(), x[1].cuda())
    got = [torch.full((total, d), 3.0, dtype=plain.TORCH[dtype], device="cuda") for _ in range(2)]
    cask.cache_read(pages, r, *got)
    torch.cuda.synchronize()
    after, got = plain.host(pages), [t.cpu() for t in got]
    written = torch.zeros(after.K.shape[:2], dtype=torch.bool)
    read = torch.zeros(total, dtype=torch.bool)
    for u in range(5):
        for t in range(n[u]):
            at, where = first[u] + t, plain.place(before, u, start[u] + t)
            if at >= total:
                continue
            read[at] = True
            for i, (pool, scale) in enumerate(((after.K, after.K_scale), (after.V, after.V_scale))):
                if where is None:
                    assert (got[i][at] == 0).all()
                    continue
                written[where] = True
                val = pool.view(torch.uint8)[where].view(pool.dtype).double()
                if cache != "e4m3":
                    assert _same(pool[where], x[i][at]) and _same(got[i][at], x[i][at])
                    continue
                q, s, y = plain.quantise(x[i][at])
                assert abs(float(scale[where]) / float(s) - 1) <= 2.0 ** -24
                nan = torch.isnan(q)
                assert torch.equal(torch.isnan(val), nan)
                if dtype == "bf16":
                    assert torch.equal(val[~nan], q[~nan])
                else:   # 448 x rounded, its quotient to 2^-23 more: that much nearer to the border between two values
                    off, half = (val - y)[~nan & torch.isfinite(y)].abs(), (q - y)[~nan & torch.isfinite(y)].abs()
                    assert (off <= half + 2.0 ** -21 * y[~nan & torch.isfinite(y)].abs()).all()
                back = (val.float() * scale[where]).to(plain.TORCH[dtype])
                assert torch.equal(torch.isnan(got[i][at]), nan) and torch.equal(got[i][at][~nan], back[~nan])
    for i, k in enumerate(("K", "V", "K_scale", "V_scale")):
        a, b = getattr(after, k), getattr(before, k)
        if a is not None:
            a, b = (t.contiguous().view(torch.uint8).view(*t.shape[:2], -1) for t in (a, b))
            assert torch.equal(a[~written], b[~written]), k
    for t in got:
        assert (t[~read] == 3.0).all()


def test_rows_of_many_units_in_token_order():
    """Arrays [tokens, heads, d] of sequences of different length, and a cache without a table whose row stride is no
    power of two."""
    heads, new, d = 3, [5, 1, 33], 128
    pages = plain.make("bf16", "bf16", d, G=1, units=9, page_rows=77, table=False, seed=3)
    tokens = sum(new)
    x = [torch.randn(tokens, heads, d, generator=torch.Generator().manual_seed(s)).to(torch.bfloat16).cuda() for s in (1, 2)]
    begin = [0, 5, 6]
    r = plain.rows([n for n in new for _ in range(heads)], [36 + u for u in range(9)],
                   [b * heads + h for b in begin for h in range(heads)], pitch=heads)
    cask.cache_write(pages, r, *x)
    got = cask.cache_read(pages, r, torch.zeros_like(x[0]), torch.zeros_like(x[1]))
    torch.cuda.synchronize()
    assert _same(got[0], x[0]) and _same(got[1], x[1])
    for s in range(3):
        for h in range(heads):
            u = s * heads + h
            assert _same(pages.K[u, 36 + u: 36 + u + new[s]], x[0][begin[s]: begin[s] + new[s], h])
            assert _same(pages.V[u, 36 + u: 36 + u + new[s]], x[1][begin[s]: begin[s] + new[s], h])


def test_rows_behind_four_gigabytes():
    """Pools of more than 2^32 bytes: the last pages are as far away as they say."""
    d, page_rows = 128, 64
    n_pages = (1 << 32) // (d * page_rows) + 40
    p = plain.params("bf16", d, 2)
    K = torch.empty(n_pages, page_rows, d, dtype=torch.float8_e4m3fn, device="cuda")
    V = torch.empty_like(K)
    Ks, Vs = (torch.empty(n_pages, page_rows, dtype=torch.float32, device="cuda") for _ in range(2))
    table = torch.tensor([[n_pages - 1, n_pages - 7], [n_pages - 3, 0]], dtype=torch.int32, device="cuda")
    pages = cask.Pages(p, K, V, Ks, Vs, table=table)
    r = plain.rows([100, 128])
    x = [torch.randn(2, 128, d, generator=torch.Generator().manual_seed(s)).to(torch.bfloat16) for s in (1, 2)]
    cask.cache_write(pages, r, x[0].cuda(), x[1].cuda())
    q = torch.randn(2, 128, 2, d, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    out = cask.attend_paged(pages, r, q.cuda())
    torch.cuda.synchronize()
    small = cask.Pages.empty(p, 2, 128)     # the same rows in pools of their own
    cask.cache_write(small, r, x[0].cuda(), x[1].cuda())
    torch.cuda.synchronize()
    assert _same(out, cask.attend_paged(small, r, q.cuda()))
    assert _same(K[n_pages - 1], small.K[0]) and _same(K[n_pages - 3], small.K[2]) and _same(V[n_pages - 7, :36], small.V[1, :36])


# ---------------------------------------------------------------- attention

def _attend(pages, n, start, first, pitch, total, seed=0, max_rows=0, count=None, window=0, sinks=0, causal=True, one=None, q_gain=1.5,
            max_n=None):
    """The operator and the plain form; rows of `out` that no token has stay as they were."""
    p = pages.params
    dtype = "f32" if p.dtype == cask.F32 else "bf16"
    Q = (q_gain * torch.randn(total, p.q_per_kv, p.head_dim, generator=torch.Generator().manual_seed(seed))).to(plain.TORCH[dtype])
    out = torch.full_like(Q, 5.0).cuda()
    r = plain.rows(n, start, first, pitch, max_n=max_n)
    cask.attend_paged(pages, r, Q.cuda(), count=None if count is None else count.cuda(), window=window, sinks=sinks,
                      max_rows=max_rows, out=out)
    torch.cuda.synchronize()
    want = plain.attend(plain.host(pages), Q, n, start, first, pitch, causal=causal, count=count, window=window, sinks=sinks)
    rest = [i for i in range(total) if i not in want]
    assert (out[rest] == 5.0).all()
    return plain.check_attend(out, want, dtype, max(n) == 1 if one is None else one), out


TYPES = [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32"), ("f32", "e4m3")]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("G,page_rows", [(1, 16), (7, 64), (20, 32)])
def test_one_token(dtype, cache, d, G, page_rows):
    """A decode step over units from one row to thousands, at places around a tile and a page, with and without
    counts (fewer than the rows), a window and first rows; with the workspace's splits and without."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 300, 2000]
    pages = plain.make(dtype, cache, d, G, units=len(lens), page_rows=page_rows, cap_pages=-(-2000 // page_rows), seed=G)
    n, start = [1] * len(lens), [x - 1 for x in lens]
    first = list(range(len(lens)))[::-1]
    g = torch.Generator().manual_seed(9)
    count = torch.randint(-1, 30, (len(lens), 250), generator=g, dtype=torch.int32)
    for kw in (dict(), dict(count=count), dict(window=40, sinks=3), dict(window=1), dict(window=500, sinks=70, count=count), dict(window=7, sinks=5000)):
        _attend(pages, n, start, first, 1, len(lens), seed=G, **kw)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("units", [5, 300])
def test_one_token_of_caches_with_room_for_many_rows(dtype, cache, d, units):
    """Tables far wider than their units' rows, with nothing behind them: the call is dealt out, and its rows loaded,
    as for caches of many megabytes, unless it is told how many rows there are."""
    lens = [1 + 37 * u % 130 for u in range(units)]
    made = plain.make(dtype, cache, d, 3, units=units, page_rows=16, cap_pages=9, seed=units)
    table = torch.full((units, 8192), -1, dtype=torch.int32, device="cuda")
    table[:, :made.table.shape[1]] = made.table
    pages = cask.Pages(made.params, made.K, made.V, made.K_scale, made.V_scale, table)
    for kw in (dict(), dict(max_rows=130), dict(window=20, sinks=2)):
        _attend(pages, [1] * units, [x - 1 for x in lens], list(range(units)), 1, units, seed=2, **kw)


FORMS = [0, B.PATH_PAGED_FEW, B.PATH_PAGED_MANY]   # the library's choice, blocks of few query rows, blocks of many


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("G,page_rows", [(1, 64), (4, 16), (7, 32)])
def test_chunks(dtype, cache, d, G, page_rows, form):
    """Chunks of different length (none, one token, odd numbers, hundreds) behind caches of different length, in token
    order with several heads; causal, not causal, windows narrower and wider than chunk and tile."""
    if dtype == "f32" and form == B.PATH_PAGED_MANY:
        pytest.skip("blocks of many query rows are bf16's")
    heads, new, past = 2, [1, 0, 37, 130, 300], [50, 3, 0, 77, 500]
    pages = plain.make(dtype, cache, d, G, units=heads * len(new), page_rows=page_rows, cap_pages=-(-800 // page_rows), seed=G + d,
                       params_kw=dict(path_flags=form))
    begin = [sum(new[:i]) for i in range(len(new))]
    n, start = [x for x in new for _ in range(heads)], [x for x in past for _ in range(heads)]
    first = [b * heads + h for b in begin for h in range(heads)]
    count = torch.randint(1, 30, (len(n), 60), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    for kw in (dict(), dict(count=count), dict(window=33, sinks=4), dict(window=200, sinks=17, count=count), dict(window=1)):
        _attend(pages, n, start, first, heads, sum(new) * heads, seed=G, **kw)
    loose = plain.make(dtype, cache, d, G, units=heads * len(new), page_rows=page_rows, cap_pages=-(-800 // page_rows), seed=G + d,
                       params_kw=dict(causal=0, path_flags=form))
    _attend(loose, n, start, first, heads, sum(new) * heads, seed=G, causal=False)
    _attend(loose, n, start, first, heads, sum(new) * heads, seed=G, causal=False, window=50, sinks=2)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_few_units_many_rows_share_the_work(dtype, cache, form):
    """One unit of thousands of rows, one token and a short chunk: the splits' results together, and with no workspace
    or one a byte too small, a single workgroup's; the capacity in place of the rows' number gives the same."""
    if dtype == "f32" and form == B.PATH_PAGED_MANY:
        pytest.skip("blocks of many query rows are bf16's")
    for n, past in (([1], [5000]), ([9], [4001]), ([40], [6000])):
        pages = plain.make(dtype, cache, 128, 4, units=1, page_rows=64, cap_pages=96, seed=n[0], params_kw=dict(path_flags=form))
        p = pages.params
        one = n[0] == 1 and form != B.PATH_PAGED_MANY
        _attend(pages, n, past, [0], 1, n[0], max_rows=past[0] + n[0], one=one)
        _attend(pages, n, past, [0], 1, n[0], one=one)
        lib, r = cask.load(), plain.rows(n, past, [0])
        Q = torch.randn(n[0], 4, 128, generator=torch.Generator().manual_seed(0)).to(plain.TORCH[dtype])
        outs = [torch.zeros_like(Q).cuda() for _ in range(3)]
        cp, cr, Qd = p.c(), r.c(n[0]), Q.cuda()
        need = lib.cask_attend_paged_workspace_bytes(C.byref(cp), C.byref(pages._c), C.byref(cr), 0, 0, 0)
        assert need > 0
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        for o, w, b in ((outs[0], None, 0), (outs[1], ws.data_ptr(), need - 1), (outs[2], ws.data_ptr(), need)):
            assert lib.cask_attend_paged(C.byref(cp), C.byref(pages._c), C.byref(cr), Qd.data_ptr(), None, 0, 0, 0, 0, o.data_ptr(),
                                         w, b, torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        want = plain.attend(plain.host(pages), Q, n, past, [0], 1)
        for o in outs:
            plain.check_attend(o, want, dtype, n[0] == 1 and form != B.PATH_PAGED_MANY)
        assert _same(outs[0], outs[1])
        assert _same(outs[2], cask.attend_paged(pages, r, Qd))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n", [1, 60])
def test_rows_that_are_not_seen_may_hold_anything(dtype, cache, n, form):
    """NaN and infinities in rows behind the unit's last, in front of a window, behind a query, in the scales of pages
    and in pages of nobody: queries that do not see them give the same bits as over clean rows.  Queries that do
    see them get what they hold."""
    if dtype == "f32" and form == B.PATH_PAGED_MANY:
        pytest.skip("blocks of many query rows are bf16's")
    past, window, sinks = 200, 12, 3
    bad_rows = [5, 40, past - 20, past + 7, past + 30, past + n, past + n + 1]
    pages = plain.make(dtype, cache, 128, 4, units=2, page_rows=32, cap_pages=12, seed=4, params_kw=dict(path_flags=form))
    clean = plain.make(dtype, cache, 128, 4, units=2, page_rows=32, cap_pages=12, seed=4, params_kw=dict(path_flags=form))
    used = set(int(e) for e in pages.table.flatten())
    for c, fill in ((pages, float("nan")),):
        for pool in (c.K, c.V):
            for e in range(pool.shape[0]):
                if e not in used:
                    pool[e] = torch.full_like(pool[e].float(), fill).to(pool.dtype)
        for i, r in enumerate(bad_rows):
            e, w = plain.place(plain.host(c), 0, r)
            x = torch.full((128,), fill)
            if cache != "e4m3" and i % 2:
                x = torch.where(torch.arange(128) % 2 == 0, float("inf"), -float("inf"))
            c.K[e, w] = x.to(c.K.dtype).cuda()
            c.V[e, w] = x.to(c.V.dtype).cuda()
            if cache == "e4m3" and i % 2:
                c.K[e, w] = torch.ones(128).to(c.K.dtype).cuda()
                c.K_scale[e, w] = float("nan")
                c.V_scale[e, w] = float("inf")
    Q = torch.randn(2 * n, 4, 128, generator=torch.Generator().manual_seed(1)).to(plain.TORCH[dtype]).cuda()
    r = plain.rows([n, n], [past, past], [0, n])
    kw = dict(window=window, sinks=sinks)
    got, want = cask.attend_paged(pages, r, Q, **kw), cask.attend_paged(clean, r, Q, **kw)
    torch.cuda.synchronize()
    sees = [any(j <= past + t and (j > past + t - window or j < sinks) for j in bad_rows) for t in range(n)]
    assert _same(got[n:], want[n:])
    for t in range(n):
        if sees[t]:
            assert not torch.isfinite(got[t].float()).all(), t
        else:
            assert _same(got[t], want[t]), t
    assert n == 1 or (any(sees) and not all(sees))


def test_values_that_are_not_finite_reach_those_who_see_them():
    """A value that is not finite in one channel: not finite for the queries behind it, in that channel alone."""
    for dtype, form in (("bf16", 0), ("f32", 0), ("bf16", B.PATH_PAGED_MANY)):
        pages = plain.make(dtype, dtype, 64, 2, units=1, page_rows=16, cap_pages=8, seed=2, params_kw=dict(path_flags=form))
        for row, ch, x in ((10, 3, float("inf")), (20, 5, -float("inf")), (35, 60, float("nan"))):
            e, w = plain.place(plain.host(pages), 0, row)
            pages.V[e, w, ch] = x
        Q = torch.randn(60, 2, 64, generator=torch.Generator().manual_seed(1)).to(plain.TORCH[dtype]).cuda()
        fin = torch.isfinite(cask.attend_paged(pages, plain.rows([60]), Q).float().cpu())
        want = torch.ones_like(fin)
        want[10:, :, 3] = want[20:, :, 5] = want[35:, :, 60] = False
        assert torch.equal(fin, want)


def test_a_row_that_sees_nothing_is_zero():
    """Pages that are not there, a start in front of the cache, a start behind its capacity."""
    for dtype, cache, form in [(*t, 0) for t in TYPES] + [("bf16", "bf16", B.PATH_PAGED_MANY), ("bf16", "e4m3", B.PATH_PAGED_MANY)]:
        pages = plain.make(dtype, cache, 128, 3, units=4, page_rows=16, cap_pages=6, seed=1, params_kw=dict(path_flags=form))
        pages.table[0] = -1
        pages.table[1, 1:] = 1 << 30
        n, start = [20, 30, 30, 10], [10, 5, -12, 96]
        first = [0, 20, 50, 80]
        _, out = _attend(pages, n, start, first, 1, 90, window=10, sinks=0)
        assert (out[:20] == 0).all() and (out[20 + 21: 50] == 0).all() and (out[50:62] == 0).all()
        _attend(pages, n, start, first, 1, 90)
        one = [1, 1, 1, 1]
        _attend(pages, one, [3, 30, -1, 200], [0, 1, 2, 3], 1, 4, window=4, one=not form)


@pytest.mark.parametrize("form", FORMS)
def test_bounds_of_a_call(form):
    """n above max_n counts as max_n, a negative one as none; rows outside the arrays are neither read nor written."""
    pages = plain.make("bf16", "e4m3", 64, 2, units=4, page_rows=16, cap_pages=20, seed=8, params_kw=dict(path_flags=form))
    Q = torch.randn(100, 2, 64, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16)
    for dev_n, n, first in (([50, -4, 12, 30], [20, 0, 12, 20], [0, 10, 95, -3]), ([1 << 30, 1, 7, 9], [20, 1, 7, 9], [60, 99, 100, 1 << 45])):
        start = [9, 100, 31, 250]
        out = torch.full_like(Q, 5.0).cuda()
        r = plain.rows(dev_n, start, first, max_n=20)
        cask.attend_paged(pages, r, Q.cuda(), out=out)
        torch.cuda.synchronize()
        want = plain.attend(plain.host(pages), Q, n, start, [f if f >= 0 else 10 ** 9 for f in first], 1)
        plain.check_attend(out, want, "bf16", False)
        assert (out[[i for i in range(100) if i not in want]] == 5.0).all()


def test_dense_caches_of_an_event():
    """No table: the [n_units, stride, d] buffers of an event; one token against cask.attend, which does the same there."""
    for dtype in ("bf16", "f32"):
        pages = plain.make(dtype, dtype, 128, 7, units=6, page_rows=533, table=False, seed=3)
        lens = [533, 1, 100, 257, 384, 500]
        count = torch.randint(1, 9, (6, 384), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
        _, out = _attend(pages, [1] * 6, [x - 1 for x in lens], list(range(6)), 1, 6, count=count)
        Q = (1.5 * torch.randn(6, 7, 128, generator=torch.Generator().manual_seed(0))).to(plain.TORCH[dtype])
        other = cask.attend(pages.params, Q.cuda(), pages.K, pages.V, torch.tensor(lens, dtype=torch.int32, device="cuda"), count=count.cuda())
        want = plain.attend(plain.host(pages), Q, [1] * 6, [x - 1 for x in lens], list(range(6)), 1, count=count)
        plain.check_attend(other, want, dtype, True)
        _attend(pages, [90, 1, 3, 17, 5, 33], [443, 0, 97, 240, 379, 467], [0, 90, 91, 94, 111, 116], 1, 149, count=count)


def test_pages_given_back_behind_a_window():
    """Rows in front of the window, sinks apart, are not needed: their pages taken out of the table change no bit."""
    for n in (1, 70):
        pages = plain.make("bf16", "e4m3", 128, 4, units=3, page_rows=16, cap_pages=64, seed=5)
        start, window, sinks = [900, 500, 100], 130, 5
        Q = torch.randn(3 * n, 4, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        r = plain.rows([n] * 3, start, [0, n, 2 * n])
        want = cask.attend_paged(pages, r, Q, window=window, sinks=sinks)
        for u in range(3):
            gone = (start[u] - window + 1) // 16
            pages.table[u, 1: max(1, gone)] = -1
        torch.cuda.synchronize()
        assert _same(cask.attend_paged(pages, r, Q, window=window, sinks=sinks), want)


def test_same_bits_every_run_and_on_another_stream():
    pages = plain.make("bf16", "e4m3", 128, 7, units=3, page_rows=64, cap_pages=40, seed=6)
    for n in (1, 5, 150):
        Q = torch.randn(3 * n, 7, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        r = plain.rows([n] * 3, [2000, 1000, 17], [0, n, 2 * n])
        want = cask.attend_paged(pages, r, Q)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            got = cask.attend_paged(pages, r, Q)
        side.synchronize()
        assert _same(got, want) and _same(cask.attend_paged(pages, r, Q), want)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_long_caches_in_blocks_of_many_query_rows(cache):
    """More than 64 stages of 64 rows (the pages are looked up 64 at a time), counts that end in the middle of a stage,
    missing pages, a window that leaves a gap behind the first rows; few of the queries are compared."""
    past, n = 8500, 33
    pages = plain.make("bf16", cache, 64, 1, units=1, page_rows=16, cap_pages=540, seed=12, params_kw=dict(path_flags=B.PATH_PAGED_MANY))
    for e in (3, 77, 130, 262, 400, 401, 402, 403, 404):
        pages.table[0, e] = -1
    count = torch.randint(1, 5, (1, 4811), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    for kw in (dict(), dict(count=count), dict(window=5000, sinks=130, count=count), dict(window=64 * 64 + 5, sinks=1)):
        _attend(pages, [n], [past], [0], 1, n, one=False, **kw)


def test_references_that_have_to_follow():
    """Logits that grow by hundreds along the cache, and fall by as many: every sum is rescaled again and again, and what
    came before keeps its weight where that does not vanish."""
    for form in (B.PATH_PAGED_FEW, B.PATH_PAGED_MANY):
        for sign in (1.0, -1.0):
            pages = plain.make("bf16", "bf16", 64, 2, units=1, page_rows=16, cap_pages=20, seed=3, params_kw=dict(path_flags=form))
            ramp = sign * torch.linspace(-40, 40, 320)
            e = pages.table[0].long().cpu()
            K = pages.K.cpu().float()
            K[e, :, 0] = ramp.view(20, 16)
            pages.K.copy_(K.to(torch.bfloat16))
            Q = torch.randn(40, 2, 64, generator=torch.Generator().manual_seed(0))
            Q[..., 0] = 60.0
            Q = Q.to(torch.bfloat16)
            out = cask.attend_paged(pages, plain.rows([40], [280]), Q.cuda())
            torch.cuda.synchronize()
            plain.check_attend(out, plain.attend(plain.host(pages), Q, [40], [280], [0], 1), "bf16", False)


@pytest.mark.parametrize("form", FORMS[1:])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_large_values_stay_finite(cache, d, form):
    """Values of about 2^117 under logits that first are zero and then grow to 5.4 (2^7.8): no weight is larger than one, so that
    the sums of 300 rows stay finite, in one workgroup and in several that share the rows."""
    pages = plain.make("bf16", cache, d, 2, units=1, page_rows=16, cap_pages=20, seed=4, params_kw=dict(path_flags=form))
    p, n, past = pages.params, 40, 280
    g = torch.Generator().manual_seed(6)
    K, V = torch.zeros(1, 320, d), 2.0 ** 117 * (1 + torch.rand(1, 320, d, generator=g))
    K[0, 64:, 0] = 5.4 / 8.0 * math.sqrt(d)
    K[0, :64, 1] = torch.randn(64, generator=g)
    cask.cache_write(pages, plain.rows([320]), K.to(torch.bfloat16).cuda(), V.to(torch.bfloat16).cuda())
    Q = 0.1 * torch.randn(n, 2, d, generator=g)
    Q[..., 0] = 8.0
    Q = Q.to(torch.bfloat16)
    r = plain.rows([n], [past], [0])
    want = plain.attend(plain.host(pages), Q, [n], [past], [0], 1)
    plain.check_attend(cask.attend_paged(pages, r, Q.cuda()), want, "bf16", False)
    lib, cp, cr, Qd = cask.load(), p.c(), r.c(n), Q.cuda()
    out = torch.zeros_like(Qd)
    assert lib.cask_attend_paged(C.byref(cp), C.byref(pages._c), C.byref(cr), Qd.data_ptr(), None, 0, 0, 0, 0, out.data_ptr(), None, 0,
                                 torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    plain.check_attend(out, want, "bf16", False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("G,n", [(4, 2), (7, 3), (4, 8), (1, 33), (4, 40)])
def test_short_chunks_keep_two_terms(cache, d, G, n):
    """Several tokens in blocks of few query rows: the weights are two bf16 terms there as for one token (2^-16), also where
    several workgroups share the rows."""
    form = 0 if n * G <= 32 else B.PATH_PAGED_FEW
    for units, past in ((3, [77, 0, 300]), (1, [4000])):
        pages = plain.make("bf16", cache, d, G, units=units, page_rows=16, cap_pages=-(-(max(past) + n) // 16), seed=n + d, params_kw=dict(path_flags=form))
        first = [u * n for u in range(units)]
        for kw in (dict(), dict(window=50, sinks=5)):
            _attend(pages, [n] * units, past, first, 1, units * n, one=True, **kw)


@pytest.mark.parametrize("form", FORMS[1:])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [320, 4096])
def test_references_that_follow_in_every_kernel(cache, d, form, rows):
    """Logits that grow, or fall, by hundreds along the cache, for each type of rows and each width, also where several
    workgroups share the rows (4096 of them at least) and their references lie far apart; a page that is missing and counts."""
    n, past = 40, rows - 40
    for sign in (1.0, -1.0):
        pages = plain.make("bf16", cache, d, 2, units=1, page_rows=16, cap_pages=rows // 16, seed=3, params_kw=dict(path_flags=form))
        g = torch.Generator().manual_seed(8)
        K, V = torch.randn(1, rows, d, generator=g), torch.randn(1, rows, d, generator=g)
        K[0, :, 0] = sign * torch.linspace(-40, 40, rows)
        cask.cache_write(pages, plain.rows([rows]), K.to(torch.bfloat16).cuda(), V.to(torch.bfloat16).cuda())
        pages.table[0, 5] = -1
        Q = torch.randn(n, 2, d, generator=g)
        Q[..., 0] = 60.0
        Q = Q.to(torch.bfloat16)
        count = torch.randint(1, 9, (1, 100), generator=g, dtype=torch.int32)
        r, cp = plain.rows([n], [past], [0]), pages.params.c()
        need = cask.load().cask_attend_paged_workspace_bytes(C.byref(cp), C.byref(pages._c), C.byref(r.c(n)), 0, 0, 0)
        assert rows < 4096 or need > 0
        out = cask.attend_paged(pages, r, Q.cuda(), count=count.cuda())
        torch.cuda.synchronize()
        plain.check_attend(out, plain.attend(plain.host(pages), Q, [n], [past], [0], 1, count=count), "bf16", form == B.PATH_PAGED_FEW)


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_single_tokens_and_a_chunk_in_one_call(dtype, cache):
    """What a program does that takes new sequences in while others go on: one token for most units, hundreds for two,
    none for one, in token order; the units of a sequence group share the pages of their first rows."""
    G, d, units = 4, 128, 12
    new = [1, 1, 1, 250, 1, 0, 1, 1, 400, 1, 1, 1]
    past = [300, 17, 64, 64, 511, 30, 0, 128, 200, 1, 99, 640]
    pages = plain.make(dtype, cache, d, G, units=units, page_rows=32, cap_pages=21, seed=5)
    pages.table[1:8, :2] = pages.table[0, :2]     # (64 rows that eight units read)
    first = [sum(new[:u]) for u in range(units)]
    for kw in (dict(), dict(window=100, sinks=6)):
        _attend(pages, new, past, first, 1, sum(new), seed=3, **kw)


# ---------------------------------------------------------------- together

def test_a_step_replays_from_a_graph():
    """Write, attend and read back captured as one graph: replayed at other rows (the device's numbers change, the
    graph does not) it gives what the eager calls give."""
    dev = torch.device("cuda:0")
    d, G, units = 128, 4, 6
    p = plain.params("bf16", d, G)
    eager, cap = cask.Pages.empty(p, units, 1024), cask.Pages.empty(p, units, 1024)
    start = torch.zeros(units, dtype=torch.int32, device=dev)
    n = torch.ones(units, dtype=torch.int32, device=dev)
    r = cask.Rows(n, 20, start=start)
    K, V = (torch.zeros(units, 20, d, dtype=torch.bfloat16, device=dev) for _ in range(2))
    Q = torch.zeros(units, 20, G, d, dtype=torch.bfloat16, device=dev)

    def run(pages, out, back):
        cask.cache_write(pages, r, K, V)
        cask.attend_paged(pages, r, Q, window=300, sinks=2, out=out)
        cask.cache_read(pages, r, *back)

    def fresh():
        return torch.zeros_like(Q), (torch.zeros_like(K), torch.zeros_like(V))
    mine, captured = fresh(), fresh()
    run(cap, *captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(cap, *captured)
    g = torch.Generator().manual_seed(3)
    at = torch.zeros(units, dtype=torch.int32)
    for rep in range(5):
        n_now = torch.randint(0, 21, (units,), generator=g, dtype=torch.int32)
        for t in (K, V, Q):
            t.copy_(torch.randn(t.shape, generator=g).to(torch.bfloat16))
        n.copy_(n_now)
        start.copy_(at)
        for o in (mine, captured):
            o[0].zero_()
            o[1][0].zero_()
            o[1][1].zero_()
        torch.cuda.synchronize()
        graph.replay()
        run(eager, *mine)
        torch.cuda.synchronize()
        assert _same(cap.K, eager.K) and _same(cap.V, eager.V) and torch.equal(cap.K_scale, eager.K_scale) and torch.equal(cap.V_scale, eager.V_scale)
        assert _same(captured[0], mine[0]) and _same(captured[1][0], mine[1][0]) and _same(captured[1][1], mine[1][1])
        at += n_now + 100 * (rep == 2)


def test_a_loop_with_an_event():
    """As a serving program uses them together: a prompt and a trace written in chunks into e4m3 pages and attended to,
    the cache read back for an event when it is full, the event's rows written over it, and decode steps that go on
    with the counts.  Every attention against the plain form over what the pages hold."""
    dev = torch.device("cuda:0")
    w = caches.scaled(caches.WORKLOADS["cfg2"], n_layers=1, n_kv_heads=3, prefix=96, decode=416, budget=384)
    c = caches.make(w, seed=23)
    p = parity.params_of(w, sim_threshold=0.3)
    b = parity.to_device(c, p)
    units, N, d, G, Wn = b.n_units, b.max_unit_len, w.head_dim, w.q_per_kv, p.window
    K, V = b.K.view(units, N, d), b.V.view(units, N, d)
    pages = cask.Pages.empty(p, units, N + 64)
    g = torch.Generator().manual_seed(5)

    def attend(n, start, count=None):
        Q = torch.randn(units * n, G, d, generator=g).to(torch.bfloat16)
        r = plain.rows([n] * units, start)
        out = cask.attend_paged(pages, r, Q.cuda(), count=count, max_rows=N)
        torch.cuda.synchronize()
        want = plain.attend(plain.host(pages), Q, [n] * units, start, [u * n for u in range(units)], 1,
                            count=None if count is None else count.cpu())
        plain.check_attend(out, want, "bf16", n == 1)
    at = 0
    for n in (96, 200, 1, 215):
        cask.cache_write(pages, plain.rows([n] * units, [at] * units), K[:, at: at + n].contiguous(), V[:, at: at + n].contiguous())
        attend(n, [at] * units)
        at += n
    assert at == N
    full = plain.rows([N] * units)
    Kb, Vb = cask.cache_read(pages, full, torch.zeros(units, N, d, dtype=torch.bfloat16, device=dev), torch.zeros(units, N, d, dtype=torch.bfloat16, device=dev))
    assert float((Kb.float() - K.float()).norm() / K.float().norm()) < 2.0 ** -4    # half a step of e4m3 at the most
    b2 = cask.Batch(p, torch.arange(units + 1, dtype=torch.int64) * N, torch.full((units,), 96, dtype=torch.int32), Kb.view(-1, d), Vb.view(-1, d), b.Q)
    out = cask.Outputs(b2)
    K2, V2 = torch.zeros(units, p.budget, d, dtype=torch.bfloat16, device=dev), torch.zeros(units, p.budget, d, dtype=torch.bfloat16, device=dev)
    count = torch.zeros(units, p.budget, dtype=torch.int32, device=dev)
    cask.compress_step(b2, K2, V2, out, out_count=count)
    torch.cuda.synchronize()
    assert int(count.max()) > 1
    cask.cache_write(pages, cask.Rows(out.out_len, p.budget), K2, V2)       # the event's own row numbers, on the device
    at = out.out_len.cpu().tolist()
    for n in (1, 1, 30, 1):
        x = [torch.randn(units, n, d, generator=g).to(torch.bfloat16).to(dev) for _ in range(2)]
        cask.cache_write(pages, plain.rows([n] * units, at), *x)
        attend(n, at, count=count)
        at = [a + n for a in at]
