"""Plain 64-bit form of the operators over a paged cache, on the CPU, and caches to try them on."""
import math

import torch

import paper_2604_10900_amd as cask

E4M3_MAX = 448.0
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


def params(dtype, d=128, G=1, **kw):
    return cask.Params(dtype=cask.F32 if dtype == "f32" else cask.BF16, head_dim=d, q_per_kv=G, window=1, budget=2, **kw)


def e4m3_of(x):
    """The e4m3 value next to each of x (float64, |x| <= 448), ties to the even significand."""
    _, e = torch.frexp(x.abs())
    step = torch.ldexp(torch.ones_like(x), (e - 4).clamp_min(-9).to(torch.int32))
    return torch.round(x / step) * step


def quantise(x):
    """(values as float64, scales as float64, quotients before rounding) of rows x [..., d]: the definition."""
    x = x.double()
    fin = torch.isfinite(x)
    a = torch.where(fin, x.abs(), torch.zeros_like(x)).amax(dim=-1).clamp_min(E4M3_MAX * 2.0 ** -126)
    y = x * E4M3_MAX / a[..., None]
    q = torch.where(fin, e4m3_of(torch.where(fin, y, torch.zeros_like(y))), y.clamp(-E4M3_MAX, E4M3_MAX))
    return q, a / E4M3_MAX, y


def place(pages, u, r):
    """(page, row of the page) of row r of unit u, None where no page is or outside the capacity."""
    n_pages, page_rows = pages.K.shape[:2]
    if pages.table is None:
        return (u, r) if 0 <= r < page_rows else None
    if not 0 <= r < pages.table.shape[1] * page_rows:
        return None
    e = int(pages.table[u, r // page_rows])
    return (e, r % page_rows) if 0 <= e < n_pages else None


def host(pages):
    """A copy of a cache with its tensors on the CPU (plain attributes, no handle)."""
    class H:
        pass
    h = H()
    for k in ("K", "V", "K_scale", "V_scale", "table"):
        t = getattr(pages, k)
        setattr(h, k, None if t is None else t.cpu())
    return h


def rows_of(h, u, n_rows):
    """(K, V float64 [n_rows, d], there [n_rows] bool) of a host copy's unit."""
    d = h.K.shape[2]
    K, V = torch.zeros(n_rows, d, dtype=torch.float64), torch.zeros(n_rows, d, dtype=torch.float64)
    there = torch.zeros(n_rows, dtype=torch.bool)
    at = [place(h, u, r) for r in range(n_rows)]
    ok = [r for r in range(n_rows) if at[r] is not None]
    if ok:
        pg, rw = torch.tensor([at[r][0] for r in ok]), torch.tensor([at[r][1] for r in ok])
        for out, pool, scale in ((K, h.K, h.K_scale), (V, h.V, h.V_scale)):
            x = pool.view(torch.uint8)[pg, rw].view(pool.dtype).double()
            out[ok] = x if scale is None else x * scale[pg, rw].double()[:, None]
        there[ok] = True
    return K, V, there


def attend(h, Q, n, start, first, pitch, scale=None, causal=True, count=None, window=0, sinks=0):
    """{array row: out [G, d]}, and beside it the bound's parts: A = sum p |v|, and the largest sum_c |q_c k_c| * scale
    that enters a softmax.  Q [total, G, d] on the CPU."""
    G, d = Q.shape[1:]
    scale = scale or 1.0 / math.sqrt(d)
    want = {}
    cap = h.K.shape[1] * (1 if h.table is None else h.table.shape[1])
    for u in range(len(n)):
        end = min(start[u] + n[u], cap)
        K, V, there = rows_of(h, u, max(end, 0))
        j = torch.arange(max(end, 0))
        w = torch.ones(max(end, 0), dtype=torch.float64)
        if count is not None:
            m = min(count.shape[1], max(end, 0))
            w[:m] = count[u, :m].clamp_min(1).double()
        for t in range(n[u]):
            at = first[u] + t * pitch
            if not 0 <= at < Q.shape[0]:
                continue
            i = start[u] + t
            see = there.clone()
            if causal:
                see &= j <= i
            if window:
                see &= (j > i - window) | (j < sinks)
            idx = see.nonzero()[:, 0]
            if len(idx) == 0:
                want[at] = (torch.zeros(G, d, dtype=torch.float64),) * 2 + (0.0, 0)
                continue
            q, k, v = Q[at].double(), K[idx], V[idx]
            x = q @ k.t() * scale + w[idx].log()
            p = torch.softmax(x, dim=1)
            want[at] = (p @ v, p @ v.abs(), float((q.abs() @ k.abs().t()).nan_to_num(0).max()) * scale, len(idx))
    return want


def check_attend(out, want, dtype, one_token):
    """Element by element: |error| <= half a step of the result's type * |want| + k * A, A = sum p |v|.
    k: a logit is a sum of d <= 128 products in fp32, off by at most (d + 2) 2^-24 * sum |q_c k_c| scale = delta, and so
    is the reference it meets: a weight is off by 2 * delta of itself, the normalised one by 4 * delta; exp2 and the
    weight's product with a scale 2^-22; a sum of N products N 2^-24 (N the rows seen, and as much again for the
    denominator).  bf16 weights: two terms, 2^-16, for one token; one term, half a step 2^-8, where there are more
    tokens.  Returns the largest error in units of its bound."""
    half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    worst = 0.0
    o = out.double().cpu().reshape(-1, *out.shape[-2:])
    for at, (y, A, logit, rows) in want.items():
        k = 4 * 130 * 2.0 ** -24 * logit + 2.0 ** -22 + 2 * rows * 2.0 ** -24
        if dtype != "f32":
            k += 2.0 ** -16 if one_token else 2.0 ** -8
        bound = half * y.abs() + k * A * (1 + half) + 1e-35
        err = (o[at] - y).abs()
        assert torch.isfinite(o[at]).all(), at
        worst = max(worst, float((err / bound).max()))
    assert worst <= 1.0, worst
    return worst


def make(dtype="bf16", cache="e4m3", d=128, G=4, units=3, page_rows=16, cap_pages=10, seed=0, interleaved=False, table=True,
         device="cuda", spare=3, params_kw=None):
    """A cache of random rows whose pages lie in any order."""
    g = torch.Generator().manual_seed(seed)
    p = params(dtype, d, G, **(params_kw or {}))
    n_pages = units * cap_pages + spare if table else units
    ct = TORCH[cache]
    gain = torch.ones(d)
    gain[torch.randperm(d, generator=g)[:4]] = 4.0
    x = [torch.randn(n_pages, page_rows, d, generator=g) * gain, torch.randn(n_pages, page_rows, d, generator=g)]
    kw = {}
    if cache == "e4m3":
        qs = [quantise(t) for t in x]
        x = [q[0].float() for q in qs]
        kw = dict(K_scale=qs[0][1].float(), V_scale=qs[1][1].float())
    pools = [t.to(ct) for t in x]
    if interleaved:   # one array [n_pages, 2, page_rows, d]
        both = torch.stack([t.view(torch.uint8) if cache == "e4m3" else t for t in pools], dim=1).to(device)
        pools = [(both[:, i].view(ct) if cache == "e4m3" else both[:, i]) for i in range(2)]
        if kw:
            s = torch.stack([kw["K_scale"], kw["V_scale"]], dim=1).to(device)
            kw = dict(K_scale=s[:, 0], V_scale=s[:, 1])
    else:
        pools = [t.to(device) for t in pools]
        kw = {k: v.to(device) for k, v in kw.items()}
    tab = None
    if table:
        tab = torch.randperm(n_pages, generator=g)[: units * cap_pages].view(units, cap_pages).to(torch.int32).contiguous().to(device)
    return cask.Pages(p, *pools, table=tab, **kw)


def rows(n, start=None, first=None, pitch=1, max_n=None, device="cuda"):
    t = lambda x, dt: None if x is None else torch.tensor(x, dtype=dt, device=device)  # noqa: E731
    return cask.Rows(t(n, torch.int32), max(n) if max_n is None else max_n, t(start, torch.int32), t(first, torch.int64), pitch)
