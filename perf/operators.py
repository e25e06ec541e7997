"""Operators over a paged KV cache: listed cases, drawn cases of the same ranges, how to prepare, run and
account for each, and what they compute from their definitions in 64 bits.

Kinds of call
  write   rows of new keys and values into the pages of a cache, quantised as they are written (e4m3, one
          scale a row) or as they are
  read    rows of a cache's pages back into plain arrays, as a compression event takes them
  attend  attention of the newest tokens of every sequence, one or a chunk of them, over the pages:
          causal, with token counts of folded rows, with a sliding window and first rows that stay visible

A case is a dict of plain values.  `seqs` sequences of `heads` units each (KV heads, or layers x KV heads);
a unit has a page table of its own, since units of one layer hold different numbers of rows after an event.
A sequence holds `past` rows and brings `new` ones (each up to `*_hi`, drawn per sequence, where that is set).
Arrays of a call are [tokens, heads, ...], the tokens of all sequences back to back.
"""
from __future__ import annotations

import math
import random

import torch

own = False   # False: the plain forms below; True: the framework's operators

E4M3_MAX = 448.0
SMALLEST = 2.0 ** -126   # the least scale of a row


def _case(name, kind, *, dtype="bf16", cache="e4m3", d=128, G=7, seqs=1, heads=4, page=64, past=0, past_hi=0, new=1,
          new_hi=0, window=0, sinks=0, counted=0):
    c = dict(kind=kind, dtype=dtype, cache=cache, d=d, G=G, seqs=seqs, heads=heads, page=page, past=past, past_hi=past_hi,
             new=new, new_hi=new_hi, window=window, sinks=sinks, counted=counted)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of a model of 28 layers x 4 KV heads: a row per unit, the smallest write
        _case("write_step", "write", heads=112, past=447),
        # a 2k chunk of a prompt, all layers, quantised
        _case("write_chunk", "write", heads=112, past=256, new=2048),
        # an event's outputs, fp32 as computed, of a batch of 17 sequences whose lengths fit no page
        _case("write_ragged", "write", dtype="f32", d=64, G=4, seqs=17, heads=8, page=16, past=0, past_hi=1900, new=301, new_hi=5077),
        # a whole trace of one sequence, all layers, back for the compression event that it is due
        _case("read_event", "read", heads=112, past=0, new=8448),
        # one layer of a few short caches
        _case("read_layer", "read", d=64, seqs=3, heads=8, page=16, past=0, new=200, new_hi=512),
        # one layer's decode step over a long trace: few units, many rows
        _case("decode_long", "attend", heads=4, past=32767),
        # a layer of a serving batch: 64 sequences over compressed caches with counts
        _case("decode_batch", "attend", G=4, seqs=64, heads=8, past=2047, past_hi=2175, counted=2048),
        # the same batch uncompressed under a sliding window: 4 first rows and 1024 last ones of up to 16k
        _case("decode_window", "attend", cache="bf16", G=4, seqs=64, heads=8, past=4096, past_hi=16384, window=1024, sinks=4),
        # a draft of 5 tokens verified at once, all layers, over fp32 caches
        _case("verify_f32", "attend", dtype="f32", cache="f32", d=64, G=4, heads=64, past=1500, new=5),
        # a 2k chunk of a 16k prompt, one layer
        _case("chunk_prompt", "attend", cache="bf16", past=16384, new=2048),
        # turns of different length over compressed and quantised caches, a layer of 8 sequences
        _case("chunk_turns", "attend", G=4, seqs=8, heads=8, past=384, past_hi=2048, new=100, new_hi=1000, counted=384),
        # a 4k chunk under a sliding window, 64 channels
        _case("chunk_window", "attend", cache="bf16", d=64, G=4, seqs=2, heads=8, page=32, past=301, new=4096, window=512, sinks=4),
    ]


# the most a drawn case may hold: elements written or read, elements of the caches attended to, logits
MOST_MOVED = 1.0e8
MOST_ELEMENTS = 1.3e8
MOST_LOGITS = 8.0e8
MOST_LOGITS_F32 = 1.0e8


def _log_int(rng: random.Random, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _units(rng: random.Random, most):
    """(seqs, heads) with seqs * heads spread over 1 .. most."""
    n = _log_int(rng, min(4, most), most) if most > 1 else 1
    seqs = rng.choice([1, 1, 2, 3, 8, 17, 64])
    while seqs > n:
        seqs = max(1, seqs // 2)
    return seqs, max(1, n // seqs)


def draw(rng: random.Random):
    kind = rng.choice(["write", "read", "decode", "decode", "chunk", "chunk", "chunk"])
    d = rng.choice([64, 128, 128])
    G = rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    dtype = rng.choice(["bf16"] * 5 + ["f32"])
    if kind in ("write", "read"):
        cache = rng.choice(["e4m3", "e4m3", "e4m3", dtype])
        new, past = _log_int(rng, 1, 9000), rng.randint(0, 2000)
        seqs, heads = _units(rng, max(1, min(512, int(MOST_MOVED / ((new + past) * d)))))
        return _case("", kind, dtype=dtype, cache=cache, d=d, G=G, seqs=seqs, heads=heads, page=page, past=past if kind == "write" else 0,
                     new=max(1, new // 3) if seqs > 1 else new, new_hi=new if seqs > 1 and new > 2 else 0)
    cache = dtype if dtype == "f32" else rng.choice(["e4m3", "e4m3", "bf16"])
    past = _log_int(rng, 16, 33000)
    new = 1 if kind == "decode" else _log_int(rng, 2, 4096)
    rows = past + new
    most = min(512, MOST_ELEMENTS / (rows * d), (MOST_LOGITS_F32 if dtype == "f32" else MOST_LOGITS) / (rows * new * G))
    while most < 1:
        new, past = max(1, new // 2), max(16, past // 2)
        rows = past + new
        most = min(512, MOST_ELEMENTS / (rows * d), (MOST_LOGITS_F32 if dtype == "f32" else MOST_LOGITS) / (rows * new * G))
    seqs, heads = _units(rng, int(most))
    window = rng.choice([0, 0, _log_int(rng, 16, 4096)])
    return _case("", "attend", dtype=dtype, cache=cache, d=d, G=G, seqs=seqs, heads=heads, page=page,
                 past=max(1, past // 2) if seqs > 1 else past, past_hi=past if seqs > 1 else 0,
                 new=max(1, new // 3) if seqs > 1 else new, new_hi=new if seqs > 1 and new > 2 else 0,
                 window=window, sinks=rng.choice([0, 1, 4, 16]) if window else 0, counted=rng.choice([0, min(past, 384)]))


# ---------------------------------------------------------------- inputs

def _lengths(c):
    """(rows held, rows brought) of every sequence: a property of the case."""
    r = random.Random(c["past"] * 7919 + c["new"] * 31 + c["past_hi"] + c["new_hi"])
    past = [r.randint(c["past"], c["past_hi"]) if c["past_hi"] else c["past"] for _ in range(c["seqs"])]
    new = [r.randint(c["new"], c["new_hi"]) if c["new_hi"] else c["new"] for _ in range(c["seqs"])]
    return past, new


_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


def _quantise(x):
    """(e4m3 values, scales) of rows x [..., d] in float32."""
    a = x.abs().amax(dim=-1).clamp_min(E4M3_MAX * SMALLEST)
    q = (x * E4M3_MAX / a[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q, a / E4M3_MAX


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 977)
    past, new = _lengths(c)
    d, G, heads, page = c["d"], c["G"], c["heads"], c["page"]
    units, tokens = c["seqs"] * heads, sum(new)
    dt, ct = _DTYPES[c["dtype"]], _DTYPES[c["cache"]]
    # pages in any order, with a few to spare; behind a sequence's last page its table has none (-1)
    per_seq = [(a + b + page - 1) // page for a, b in zip(past, new)]
    pitch = max(per_seq)
    n_pages = heads * sum(per_seq) + 5
    perm = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    held = torch.tensor(per_seq, device=dev).repeat_interleave(heads)
    slot = torch.arange(pitch, device=dev)
    at = (held.cumsum(0) - held)[:, None] + slot[None, :]
    table = torch.where(slot[None, :] < held[:, None], perm[at.clamp_max(n_pages - 1)], -1)
    s = dict(case=c, units=units, tokens=tokens, table=table.to(torch.int32).contiguous(), max_new=max(new),
             max_rows=max(a + b for a, b in zip(past, new)))
    s["past"] = torch.tensor(past, dtype=torch.int32, device=dev).repeat_interleave(heads)
    s["new"] = torch.tensor(new, dtype=torch.int32, device=dev).repeat_interleave(heads)
    begin = torch.tensor([sum(new[:i]) for i in range(c["seqs"])], dtype=torch.int64, device=dev)
    s["first"] = (begin[:, None] * heads + torch.arange(heads, device=dev)).reshape(-1).contiguous()
    scaled = c["cache"] == "e4m3"
    for name in ("K", "V"):
        pool = torch.empty(n_pages, page, d, dtype=ct, device=dev)
        scale = torch.ones(n_pages, page, dtype=torch.float32, device=dev) if scaled else None
        # keys: a few loud channels, as models have them, the same for all rows of a cache
        gain = torch.ones(d, device=dev)
        if name == "K":
            gain[torch.randperm(d, generator=g, device=dev)[:4]] = 8.0
        step = max(1, int(1.0e8 // (page * d)))
        for p0 in range(0, n_pages, step):
            x = torch.randn(min(step, n_pages - p0), page, d, generator=g, device=dev) * gain
            if scaled:
                pool[p0: p0 + step], scale[p0: p0 + step] = _quantise(x)
            else:
                pool[p0: p0 + step] = x.to(ct)
        s[name], s[name + "_scale"] = pool, scale
        if c["kind"] == "write":
            s[name + "_new"] = (torch.randn(tokens, heads, d, generator=g, device=dev) * gain).to(dt)
        elif c["kind"] == "read":
            s[name + "_out"] = torch.zeros(tokens, heads, d, dtype=dt, device=dev)
    if c["kind"] == "attend":
        q = torch.randn(tokens, heads, G, d, generator=g, device=dev) + torch.randn(1, heads, 1, d, generator=g, device=dev)
        s["Q"] = q.to(dt)
        s["out"] = torch.zeros_like(s["Q"])
        if c["counted"]:
            s["count"] = torch.ones(units, c["counted"], dtype=torch.int32, device=dev)
            folded = torch.rand(s["count"].shape, generator=g, device=dev) < 0.08
            s["count"] += folded * torch.randint(1, 24, s["count"].shape, generator=g, device=dev, dtype=torch.int32)
    return s


# ---------------------------------------------------------------- one pass

def _handle(s):
    """The cache and the rows of the call as the framework takes them: what a program keeps for as long as it
    keeps the cache and until it steps on, made in the first pass over a state."""
    if "handle" not in s:
        import paper_2604_10900_amd as cask
        c = s["case"]
        p = cask.Params(dtype=cask.F32 if c["dtype"] == "f32" else cask.BF16, head_dim=c["d"], q_per_kv=c["G"], window=1, budget=2)
        pages = cask.Pages(p, s["K"], s["V"], K_scale=s["K_scale"], V_scale=s["V_scale"], table=s["table"])
        rows = cask.Rows(s["new"], s["max_new"], start=s["past"], first=s["first"], pitch=c["heads"])
        s["handle"] = cask, pages, rows
    return s["handle"]


def _run_own(s):
    cask, pages, rows = _handle(s)
    c = s["case"]
    if c["kind"] == "write":
        cask.cache_write(pages, rows, s["K_new"], s["V_new"])
        return _pools(s)
    if c["kind"] == "read":
        return cask.cache_read(pages, rows, s["K_out"], s["V_out"])
    return cask.attend_paged(pages, rows, s["Q"], count=s.get("count"), window=c["window"], sinks=c["sinks"],
                             max_rows=s["max_rows"], out=s["out"])


def _pools(s):
    return {k: s[k] for k in ("K", "V", "K_scale", "V_scale") if s[k] is not None}


def _flat_rows(s):
    """Pool row of every row of the call, in the order of the call's arrays [tokens, heads]."""
    c = s["case"]
    heads, page = c["heads"], c["page"]
    new = s["new"][::heads].long()
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device=new.device), new, output_size=s["tokens"])
    t = torch.arange(s["tokens"], device=new.device) - (new.cumsum(0) - new)[seq]
    unit = seq[:, None] * heads + torch.arange(heads, device=new.device)[None, :]
    row = s["past"].long()[unit] + t[:, None]
    return s["table"][unit, row // page].long() * page + row % page


def _plain_write(s):
    at = _flat_rows(s).reshape(-1)
    for name in ("K", "V"):
        x = s[name + "_new"].reshape(-1, s["case"]["d"])
        pool = s[name].view(-1, x.shape[1])
        if s[name + "_scale"] is None:
            pool[at] = x.to(pool.dtype)
        else:
            q, scale = _quantise(x.float())
            pool.view(torch.uint8)[at] = q.view(torch.uint8)
            s[name + "_scale"].view(-1)[at] = scale
    return _pools(s)


def _plain_rows(s, name, at):
    """Rows `at` of a pool in float32."""
    x = s[name].view(torch.uint8).view(-1, s[name].shape[2] * s[name].element_size())[at].view(s[name].dtype).float()
    return x if s[name + "_scale"] is None else x * s[name + "_scale"].view(-1)[at][..., None]


def _plain_read(s):
    at = _flat_rows(s)
    for name in ("K", "V"):
        s[name + "_out"].copy_(_plain_rows(s, name, at))
    return s["K_out"], s["V_out"]


def _plain_attend(s):
    c = s["case"]
    d, G, heads, units, page = c["d"], c["G"], c["heads"], s["units"], c["page"]
    dev = s["Q"].device
    L, T = s["max_rows"], s["max_new"]
    j = torch.arange(L, device=dev)
    pages = s["table"].long()[:, j // page]                                     # [units, L]
    at = pages.clamp_min(0) * page + j % page
    K, V = _plain_rows(s, "K", at), _plain_rows(s, "V", at)                     # [units, L, d]
    t = torch.arange(T, device=dev)
    mine = (s["first"][:, None] + t * heads).clamp_max(s["tokens"] * heads - 1)  # rows of Q of every unit, padded to T
    q = s["Q"].view(-1, G, d)[mine].float().view(units, T * G, d)
    x = torch.matmul(q, K.transpose(1, 2)) * (1.0 / math.sqrt(d))               # [units, T G, L]
    if c["counted"]:
        bias = torch.zeros(units, L, device=dev)
        n = min(c["counted"], L)
        bias[:, :n] = s["count"][:, :n].float().log()
        x += bias[:, None, :]
    i = (s["past"].long()[:, None] + t)[:, :, None]                             # [units, T, 1]
    seen = (j <= i) & (pages >= 0)[:, None, :]
    if c["window"]:
        seen &= (j > i - c["window"]) | (j < c["sinks"])
    x = x.view(units, T, G, L).masked_fill_(~seen[:, :, None, :], -math.inf).view(units, T * G, L)
    top = x.amax(dim=-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    e = x.sub_(top).exp_()
    out = torch.matmul(e, V) / e.sum(dim=-1, keepdim=True).clamp_min(1e-30)
    # padded rows behind a unit's last token go to a spare row
    to = torch.where(t < s["new"][:, None], s["first"][:, None] + t * heads, s["tokens"] * heads)
    flat = torch.empty(s["tokens"] * heads + 1, G, d, dtype=s["out"].dtype, device=dev)
    flat[to.reshape(-1)] = out.view(units * T, G, d).to(flat.dtype)
    s["out"].view(-1, G, d).copy_(flat[:-1])
    return s["out"]


def run(s):
    if own:
        return _run_own(s)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[s["case"]["kind"]](s)


# ---------------------------------------------------------------- accounting

def _seen(i, window, sinks):
    """Rows that the token at row i sees."""
    if not window or window > i:
        return i + 1
    return window + min(sinks, i + 1 - window)


def work(case):
    """What a pass cannot do without: every row written or read once, with its scale; attention: every row that
    some token of its sequence sees once, and two products for every pair of a query and a row it sees."""
    c = case
    el = {"f32": 4, "bf16": 2, "e4m3": 1}
    d, G, heads = c["d"], c["G"], c["heads"]
    src = d * el[c["dtype"]]
    row = d * el[c["cache"]] + (4 if c["cache"] == "e4m3" else 0)
    past, new = _lengths(c)
    if c["kind"] != "attend":
        n = heads * sum(new)
        return {"bytes": 2.0 * n * (src + row), "flops": 2.0 * n * d * (3 if c["kind"] == "write" else 1) * (c["cache"] == "e4m3")}
    rows = pairs = 0
    for a, b in zip(past, new):
        first = max(0, a - c["window"] + 1) if c["window"] else 0     # the first row that the first token sees, sinks apart
        rows += a + b - first + min(c["sinks"], first)
        pairs += sum(_seen(i, c["window"], c["sinks"]) for i in range(a, a + b))
    return {"bytes": heads * (2.0 * rows * row + 4.0 * min(c["counted"], rows) + 2.0 * sum(new) * G * src),
            "flops": 4.0 * heads * pairs * G * d}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_e4m3(x):
    """The e4m3 value next to each of x (float64, within +-448), ties to the even significand."""
    _, e = torch.frexp(x.abs())
    step = torch.ldexp(torch.ones_like(x), (e - 4).clamp_min(-9).to(torch.int32))   # 3 bits behind the point; 2^-9 below 2^-6
    return torch.round(x / step) * step


def _exact_unit(s, u):
    """Rows past + new of unit u as pool rows, -1 where no page is."""
    c = s["case"]
    n = int(s["past"][u]) + int(s["new"][u])
    row = torch.arange(n, device=s["table"].device)
    entry = s["table"][u].long()[row // c["page"]]
    return torch.where(entry >= 0, entry * c["page"] + row % c["page"], -1)


def _exact_values(s, name, at):
    x = s[name].view(torch.uint8).view(-1, s[name].shape[2] * s[name].element_size())[at].view(s[name].dtype).double()
    return x * s[name + "_scale"].reshape(-1)[at].double()[:, None] if s[name + "_scale"] is not None else x


def exact(case, seed):
    c = dict(case)
    past, new = _lengths(c)
    if c["kind"] == "attend" and c["heads"] * c["G"] * sum(b * (a + b) for a, b in zip(past, new)) > 6.0e9:
        return None
    s = prepare(case, seed)
    heads, d, G = c["heads"], c["d"], c["G"]
    if c["kind"] == "write":
        out = {k: s[k].double() for k in ("K", "V", "K_scale", "V_scale") if s[k] is not None}
        for u in range(s["units"]):
            at = _exact_unit(s, u)[int(s["past"][u]):]
            mine = int(s["first"][u]) // heads + torch.arange(len(at), device=at.device)
            for name in ("K", "V"):
                x = s[name + "_new"][mine, u % heads].double()
                if s[name + "_scale"] is not None:
                    largest = x.abs().amax(dim=1).clamp_min(E4M3_MAX * SMALLEST)
                    x = _exact_e4m3(x * E4M3_MAX / largest[:, None])
                    out[name + "_scale"].view(-1)[at] = largest / E4M3_MAX
                out[name].view(-1, d)[at] = x
        return out
    if c["kind"] == "read":
        got = []
        for name in ("K", "V"):
            y = torch.empty(s["tokens"], heads, d, dtype=torch.float64, device=s["table"].device)
            for u in range(s["units"]):
                mine = int(s["first"][u]) // heads + torch.arange(int(s["new"][u]), device=y.device)
                y[mine, u % heads] = _exact_values(s, name, _exact_unit(s, u)[int(s["past"][u]):])
            got.append(y)
        return tuple(got)
    y = torch.empty(s["tokens"], heads, G, d, dtype=torch.float64, device=s["table"].device)
    for u in range(s["units"]):
        at = _exact_unit(s, u)
        here = (at >= 0).nonzero()[:, 0]
        k, v = _exact_values(s, "K", at[here]), _exact_values(s, "V", at[here])
        n, before, t0 = int(s["new"][u]), int(s["past"][u]), int(s["first"][u]) // heads
        w = torch.ones(len(at), dtype=torch.float64, device=y.device)
        if c["counted"]:
            m = min(c["counted"], len(at))
            w[:m] = s["count"][u, :m].double()
        for b0 in range(0, n, 512):
            b1 = min(n, b0 + 512)
            pos = before + torch.arange(b0, b1, device=y.device)[:, None]
            seen = here[None, :] <= pos
            if c["window"]:
                seen &= (pos - here[None, :] < c["window"]) | (here[None, :] < c["sinks"])
            q = s["Q"][t0 + b0: t0 + b1, u % heads].double()
            x = torch.matmul(q.reshape(-1, d), k.t().contiguous()).view(b1 - b0, G, len(here)) / math.sqrt(d)
            x = torch.where(seen[:, None, :], x, -math.inf)
            p = torch.exp(x - x.amax(dim=2, keepdim=True)) * w[here]
            p = p / p.sum(dim=2, keepdim=True)
            y[t0 + b0: t0 + b1, u % heads] = torch.matmul(p.view(-1, len(here)), v).view(b1 - b0, G, d)
    return y
