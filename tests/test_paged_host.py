"""Host side of the operators over a paged cache (CPU only): what a call refuses, the workspace it asks for, and the
plain form that the GPU tests compare with."""
import ctypes as C
import dataclasses
import math

import pytest
import torch

import paper_2604_10900_amd as cask
from tests import paged_plain as plain

B = cask.binding
FAKE = 256   # an address that is never looked at


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(B.LIB_PATH):
        from paper_2604_10900_amd.build import build_lib
        build_lib()
    return cask.load()


def _pages(**kw):
    f = dict(type=B.BF16, n_units=3, n_pages=30, page_rows=64, page_pitch=64, table_pitch=10, table=FAKE, K=FAKE, V=FAKE,
             K_scale=None, V_scale=None)
    f.update(kw)
    return B._Pages(*(f[k] for k, _ in B._Pages._fields_))


def _rows(**kw):
    f = dict(max_n=5, pitch=1, total=15, n=FAKE, start=None, first=None)
    f.update(kw)
    return B._Rows(*(f[k] for k, _ in B._Rows._fields_))


def _calls(lib, p=None, pages=None, rows=None, K=FAKE, V=FAKE, count=None, count_pitch=0, window=0, sinks=0, max_rows=0, ws=None):
    """Return codes of the three calls."""
    p = (p or cask.Params(q_per_kv=4, window=1, budget=2)).c()
    pages, rows = pages or _pages(), rows or _rows()
    a = (C.byref(p), C.byref(pages), C.byref(rows))
    return (lib.cask_cache_write(*a, K, V, None), lib.cask_cache_read(*a, K, V, None),
            lib.cask_attend_paged(*a, K, count, count_pitch, window, sinks, max_rows, V, ws, 0, None))


BAD_PAGES = [
    dict(type=B.F32), dict(type=3), dict(type=-1), dict(n_units=-1), dict(n_pages=-1), dict(page_rows=0), dict(page_rows=48),
    dict(page_rows=8), dict(page_rows=1 << 21, page_pitch=1 << 21), dict(page_pitch=63), dict(page_pitch=(1 << 40) + 1), dict(table_pitch=0),
    dict(table_pitch=1 << 25), dict(K=None), dict(V=None), dict(K=FAKE + 8), dict(V=FAKE + 4), dict(type=B.E4M3), dict(type=B.E4M3, K_scale=FAKE),
    dict(type=B.E4M3, V_scale=FAKE), dict(table=None, n_pages=2), dict(table=None, page_rows=(1 << 30) + 1, page_pitch=1 << 31),
    dict(type=B.E4M3, K_scale=FAKE, V_scale=FAKE, table=None, page_rows=72, page_pitch=80)]
BAD_ROWS = [dict(max_n=-1), dict(pitch=0), dict(total=-1), dict(total=(1 << 40) + 1), dict(n=None), dict(max_n=1 << 29)]


@pytest.mark.parametrize("bad", BAD_PAGES, ids=str)
def test_pages_that_are_refused(lib, bad):
    assert _calls(lib, pages=_pages(**bad)) == (B.EINVAL,) * 3


@pytest.mark.parametrize("bad", BAD_ROWS, ids=str)
def test_rows_that_are_refused(lib, bad):
    assert _calls(lib, rows=_rows(**bad)) == (B.EINVAL,) * 3


def test_places_that_would_leave_64_bits_are_refused(lib):
    """Rows of the arrays: t * pitch with t < 2^29 and pitch < total; places in the pools: entry * page_pitch rows of up to
    512 bytes.  The largest that fit are taken (as the size that is asked for shows)."""
    def need(**kw):
        p = cask.Params(q_per_kv=4, window=1, budget=2).c()
        pg, rw = dict(n_units=1, table_pitch=1 << 12), dict(max_n=1)
        for k, v in kw.items():
            (rw if k == "total" else pg)[k] = v
        return lib.cask_attend_paged_workspace_bytes(C.byref(p), C.byref(_pages(**pg)), C.byref(_rows(**rw)), 0, 0, 0)
    assert need(total=1 << 33) > 0
    assert need(total=(1 << 33) + 1) == 0 and _calls(lib, rows=_rows(total=(1 << 33) + 1)) == (B.EINVAL,) * 3
    most = (1 << 31) - 1   # pages
    for fits, too_many in ((dict(n_pages=1 << 13, page_pitch=1 << 40), dict(n_pages=(1 << 13) + 1, page_pitch=1 << 40)),
                           (dict(n_pages=most, page_pitch=1 << 22), dict(n_pages=most, page_pitch=(1 << 22) + 2))):
        assert need(**fits) > 0, fits
        assert need(**too_many) == 0 and _calls(lib, pages=_pages(**too_many)) == (B.EINVAL,) * 3, too_many


def test_arguments_that_are_refused(lib):
    assert _calls(lib, K=None) == (B.EINVAL,) * 3 and _calls(lib, V=None) == (B.EINVAL,) * 3
    assert _calls(lib, K=FAKE + 8) == (B.EINVAL,) * 3 and _calls(lib, V=FAKE + 2) == (B.EINVAL,) * 3
    for kw in (dict(window=-1), dict(sinks=-1), dict(max_rows=-1), dict(count=FAKE, count_pitch=0), dict(ws=FAKE + 4)):
        assert _calls(lib, **kw)[2] == B.EINVAL, kw
    ok, pg, rw = cask.Params(window=1, budget=2).c(), _pages(), _rows()
    for a in ((None, C.byref(pg), C.byref(rw)), (C.byref(ok), None, C.byref(rw)), (C.byref(ok), C.byref(pg), None)):
        assert lib.cask_cache_write(*a, FAKE, FAKE, None) == B.EINVAL
        assert lib.cask_attend_paged(*a, FAKE, None, 0, 0, 0, 0, FAKE, None, 0, None) == B.EINVAL
        assert lib.cask_attend_paged_workspace_bytes(*a, 0, 0, 0) == 0
    assert _calls(lib, p=cask.Params(head_dim=96, window=1, budget=2)) == (B.EINVAL,) * 3


def test_launches_that_would_have_too_many_threads(lib):
    """More query blocks than a launch may have: refused by the attention; fp32's blocks are the smaller ones."""
    big = dict(pages=_pages(n_units=1 << 15), rows=_rows(max_n=1 << 15, total=1 << 30))
    for G, dtype, bad in ((4, B.F32, True), (2, B.BF16, True), (1, B.BF16, False)):
        p = cask.Params(dtype=dtype, q_per_kv=G, window=1, budget=2)
        pages = _pages(n_units=1 << 15, type=dtype)
        need = lib.cask_attend_paged_workspace_bytes(C.byref(p.c()), C.byref(pages), C.byref(big["rows"]), 0, 0, 0)
        assert need == 0
        if bad:
            assert _calls(lib, p=p, pages=pages, rows=big["rows"])[2] == B.EINVAL


def test_nothing_to_do_touches_nothing(lib):
    """No units, no rows, no arrays: fine, whatever the pointers."""
    nothing = dict(K=None, V=None)
    for kw in (dict(pages=_pages(n_units=0, **nothing)), dict(rows=_rows(max_n=0, n=None)), dict(rows=_rows(total=0))):
        assert _calls(lib, K=None, V=None, **kw) == (B.OK,) * 3, kw


def test_workspace_of_the_attention(lib):
    """Nothing where the queries alone fill the chip or the rows are few; else partial results of every query row, at
    most 64 each; a window bounds the rows; device pointers play no part."""
    def need(units, n, rows, G=4, d=128, **kw):
        p = cask.Params(head_dim=d, q_per_kv=G, window=1, budget=2).c()
        pg = _pages(n_units=units, n_pages=1, table_pitch=1 << 12, K=None, V=None)
        rw = _rows(max_n=n, n=None)
        a = dict(window=0, sinks=0, max_rows=rows)
        a.update(kw)
        b = lib.cask_attend_paged_workspace_bytes(C.byref(p), C.byref(pg), C.byref(rw), a["window"], a["sinks"], a["max_rows"])
        per = units * n * G * (d + 2) * 4
        assert b % per == 0 and b // per <= 64
        return b // per
    assert need(4, 1, 32768) > 8 and need(1, 1, 1 << 18) > 8
    assert need(4, 1, 100) == 0 and need(4096, 1, 32768) == 0 and need(8, 4096, 32768) == 0
    assert need(4, 1, 32768, window=64, sinks=4) == 0
    assert need(4, 1, 0) == need(4, 1, 1 << 18) == need(4, 1, 1 << 30)   # 0 and more than the capacity: the capacity


def test_binding_refuses_what_does_not_fit():
    p = plain.params("bf16")
    K = torch.zeros(4, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):      # on the CPU
        cask.Pages(p, K, K)
    for bad in (K[:, :, :64], K[:, ::2], K.transpose(0, 1), K.view(-1, 128)):
        with pytest.raises(AssertionError):
            cask.Pages(p, bad, bad)
    q = K.to(torch.float8_e4m3fn)
    for s in ((None, None), (torch.ones(4, 16),) * 2, (torch.ones(4, 15),) * 2, (torch.ones(4, 16, dtype=torch.float64),) * 2):
        with pytest.raises(AssertionError):
            cask.Pages(p, q, q, *s)
    with pytest.raises(KeyError):
        cask.Pages(p, K.half(), K.half())
    n = torch.ones(3, dtype=torch.int32)
    with pytest.raises(AssertionError):
        cask.Rows(n, 1)


class _OnDevice(torch.Tensor):
    """A host tensor that says it is on the device: for checks that come before any call of the library."""
    is_cuda = True


@pytest.mark.parametrize("change", [dict(head_dim=128), dict(dtype=B.F32)], ids=str)
def test_parameters_changed_after_the_cache_was_made(monkeypatch, change):
    """A cache of other rows than the parameters speak of by now: refused before a kernel takes its pools for larger ones."""
    on = lambda t: t.as_subclass(_OnDevice)  # noqa: E731
    monkeypatch.setattr(B, "_current_device", lambda: None)
    p = cask.Params(dtype=B.BF16, head_dim=64, q_per_kv=1, window=1, budget=2)
    pool = on(torch.zeros(4, 16, 64).to(torch.float8_e4m3fn))
    scale = on(torch.ones(4, 16))
    pages = cask.Pages(p, pool, pool, scale, scale)
    rows = cask.Rows(on(torch.zeros(4, dtype=torch.int32)), 3)
    for k, v in change.items():
        setattr(p, k, v)
    dt = torch.float32 if p.dtype == B.F32 else torch.bfloat16
    for dtype in {dt, torch.bfloat16}:
        x = on(torch.zeros(12, p.head_dim, dtype=dtype))
        for call in (lambda: cask.cache_write(pages, rows, x, x), lambda: cask.cache_read(pages, rows, x, x),
                     lambda: cask.attend_paged(pages, rows, x[:, None], out=x[:, None])):
            with pytest.raises(AssertionError):
                call()


def test_a_table_without_pages_is_refused(monkeypatch):
    """A table of no pages a unit has no address: to the library it would be no table at all, where unit u owns page u."""
    monkeypatch.setattr(B, "_current_device", lambda: None)
    on = lambda t: t.as_subclass(_OnDevice)  # noqa: E731
    pool = on(torch.zeros(4, 16, 128, dtype=torch.bfloat16))
    p = plain.params("bf16")
    with pytest.raises(AssertionError):
        cask.Pages(p, pool, pool, table=on(torch.zeros(3, 0, dtype=torch.int32)))
    assert cask.Pages(p, pool, pool, table=on(torch.zeros(0, 2, dtype=torch.int32))).n_units == 0   # (no units: nothing to own)


def test_numbers_of_more_than_32_bits_are_refused(monkeypatch):
    """A window, a number of first rows or of rows that C would take for another one (its lowest 32 bits)."""
    on = lambda t: t.as_subclass(_OnDevice)  # noqa: E731
    monkeypatch.setattr(B, "_current_device", lambda: None)
    pool, n = on(torch.zeros(4, 16, 128, dtype=torch.bfloat16)), on(torch.zeros(4, dtype=torch.int32))
    pages, q = cask.Pages(plain.params("bf16"), pool, pool), on(torch.zeros(4, 1, 128, dtype=torch.bfloat16))
    rows = cask.Rows(n, 1)
    for kw in (dict(window=(1 << 32) + 5), dict(window=7, sinks=1 << 31), dict(max_rows=(1 << 32) + 1)):
        with pytest.raises(AssertionError):
            cask.attend_paged(pages, rows, q, out=q, **kw)
    with pytest.raises(AssertionError):
        cask.Rows(n, (1 << 32) + 1)
    with pytest.raises(AssertionError):
        cask.Rows(n, 1, pitch=(1 << 64) + 1)


def test_written_out_loads_wait_for_their_descriptor():
    """Between a vector instruction that writes a scalar register and a vector memory instruction that reads it lie five wait
    states; in front of a load in inline assembly the assembly itself has to give them (the compiler may put the
    descriptor there at the last moment, as when it brings spilled words back).  m0 needs one before a load to LDS."""
    import os
    import re
    from paper_2604_10900_amd import build
    found = 0
    for name in build.SOURCES:
        text = open(os.path.join(build.CSRC, name)).read()
        for asm in re.findall(r'asm volatile\(\s*"((?:[^"\\]|\\.)*buffer_load(?:[^"\\]|\\.)*)"', text):
            lines = [ln.split() for ln in asm.replace("\\t", "").split("\\n")]
            states, since_m0 = 0, None
            for i, ln in enumerate(lines):
                if ln[0].startswith("buffer_load"):
                    assert states >= 5 and (ln[-1] != "lds" or since_m0 >= 1), (name, asm)
                    found += 1
                n = int(ln[1], 0) + 1 if ln[0] == "s_nop" else 1
                states += n
                since_m0 = 0 if ln[:2] == ["s_mov_b32", "m0,"] else None if since_m0 is None else since_m0 + n
    assert found >= 4


# ---------------------------------------------------------------- the plain form itself

def _host_cache(**kw):
    """plain.make without a GPU: the tensors, no handle."""
    real, holder = cask.Pages, []

    class Fake:
        def __init__(self, p, K, V, K_scale=None, V_scale=None, table=None):
            self.params, self.K, self.V, self.K_scale, self.V_scale, self.table = p, K, V, K_scale, V_scale, table
            holder.append(self)
    cask.Pages = Fake
    try:
        return plain.make(device="cpu", **kw)
    finally:
        cask.Pages = real


def test_plain_quantiser_is_the_nearest_value():
    """Against all 256 e4m3 values: the nearest one, an even one in a tie; the row's largest value is 448 scales."""
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    code = {float(v): i for i, v in enumerate(every) if not math.isnan(v)}
    fin = every[~torch.isnan(every)].unique()
    g = torch.Generator().manual_seed(1)
    x = torch.randn(40, 64, generator=g, dtype=torch.float64)
    x[0] = 0.0
    x[1, :8] = torch.tensor([448., 17., 19., 21., 2.0 ** -10, 3 * 2.0 ** -10, 464., -17.])
    x[1, 6] = 448.0
    x[1, 8:] = 1.0
    q, s, y = plain.quantise(x)
    assert ((q[1, :6] - torch.tensor([448., 16., 20., 20., 0., 2.0 ** -8])).abs() == 0).all()
    for r in range(40):
        for c in range(64):
            d = (fin - y[r, c]).abs()
            near = fin[d == d.min()]
            assert float(q[r, c]) in near.tolist()
            if len(near) == 2:
                assert code[float(q[r, c])] % 2 == 0
        assert x[r].abs().max() == 0 or abs(float(s[r]) * 448 / float(x[r].abs().max()) - 1) < 1e-12
    odd = torch.tensor([[1.0, float("inf"), -float("inf"), float("nan"), 2.0]], dtype=torch.float64)
    q, s, _ = plain.quantise(odd)
    assert q[0, :3].tolist() == [224.0, 448.0, -448.0] and math.isnan(q[0, 3]) and float(s) == 2.0 / 448


def test_plain_attention_is_softmax_over_the_rows_a_query_sees():
    """Against torch's attention with a mask, counts as repeated rows, pages in order."""
    for cache in ("f32", "e4m3"):
        pages = _host_cache(dtype="f32", cache=cache, d=64, G=2, units=2, page_rows=16, cap_pages=4, seed=7)
        Q = torch.randn(14, 2, 64, generator=torch.Generator().manual_seed(1))
        count = torch.randint(1, 4, (2, 30), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
        got = plain.attend(pages, Q, [7, 7], [40, 3], [0, 7], 1, count=count, window=9, sinks=2)
        for u, past in ((0, 40), (1, 3)):
            K, V, there = plain.rows_of(pages, u, past + 7)
            assert there.all()
            rep = torch.repeat_interleave(torch.arange(past + 7), torch.cat([count[u], torch.ones(past + 7, dtype=torch.int32)])[: past + 7] if past + 7 >= 30
                                          else count[u, : past + 7])
            for t in range(7):
                i = past + t
                mask = (rep <= i) & ((rep > i - 9) | (rep < 2))
                want = torch.nn.functional.scaled_dot_product_attention(Q[u * 7 + t].double()[None], K[rep][None], V[rep][None], attn_mask=mask[None, None, :].expand(1, 2, -1))
                assert torch.allclose(got[u * 7 + t][0], want[0], rtol=1e-12, atol=1e-12)


def test_comparison_finds_a_planted_mistake():
    """check_attend passes the rounded result and fails one whose query sees a row too many or too few."""
    pages = _host_cache(dtype="bf16", cache="e4m3", d=128, G=2, units=1, page_rows=16, cap_pages=8, seed=3)
    Q = torch.randn(20, 2, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    want = plain.attend(pages, Q, [20], [60], [0], 1, window=30, sinks=2)
    out = torch.stack([want[i][0] for i in range(20)])
    for one in (True, False):
        assert plain.check_attend(out.to(torch.bfloat16), want, "bf16", one) <= 1.0
        for kw in (dict(window=31, sinks=2), dict(window=29, sinks=2), dict(window=30, sinks=3), dict(window=30, sinks=2, causal=False)):
            other = plain.attend(pages, Q, [20], [60], [0], 1, **kw)
            with pytest.raises(AssertionError):
                plain.check_attend(torch.stack([other[i][0] for i in range(20)]).to(torch.bfloat16), want, "bf16", one)


def test_params_are_left_as_they_were():
    """A paged call reads dtype, head_dim, q_per_kv, softmax_scale and causal alone: the struct has no new field."""
    assert [f.name for f in dataclasses.fields(cask.Params)][:3] == ["dtype", "head_dim", "q_per_kv"]
    assert C.sizeof(B._Pages) == 72 and C.sizeof(B._Rows) == 48
