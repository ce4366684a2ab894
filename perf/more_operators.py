"""The paged K/V cache beside the d2Cache step, as timed cases: rows rotated by positions of several axes, rows appended to pages with the
rotation on the way, and the attention of new or selected rows over the pages.

  rotate     query or key rows [n, heads * head dimension] by positions of one axis (text) or three (time, height, width)
  append     new rows of a batch of sequences go into the sequences' pages, keys rotated, queries rotated beside them; read back as values
  attention  the packed rows of a batch against each sequence's pages: single tokens, chunks of a prompt, a chunk among single tokens, selected
             rows; causal, block-causal (semi-autoregressive blocks), with a window, without a mask; with or without the head average

Sequences lie in pages of one pool in no order, as a pool looks that has been in use.  Geometries are those of
paper_2509_23094_amd.workloads: LLaDA-8B shape (32 heads), Dream-7B shape (28 heads on 4), both with heads of 128 and bf16, and the small fp32 model
(4 heads of 64); "mid" has 12 heads of 64 on 2.
"""
import math

import torch

own = False

GEOMETRY = {"llada": (32, 32, 128), "dream": (28, 4, 128), "small": (4, 4, 64), "mid": (12, 2, 64)}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
THETA = 10000.0


def listed():
    return [
        # the queries of a single token: latency
        dict(name="rotate one row", kind="rotate", geo="dream", dtype="bf16", src="bf16", n=1, axes=1, ladder="shared", pairing="halves", part=1, far=1023),
        # 15 frames of 15 x 27 patches, as a projection leaves them (float), far into a long context
        dict(name="rotate video", kind="rotate", geo="llada", dtype="bf16", src="f32", n=6075, axes=3, ladder="shared", pairing="halves", part=1, far=200000),
        # a decode step of 64 sequences: one row each, straight from the projection
        dict(name="append decode", kind="append", geo="dream", dtype="bf16", src="f32", batch=64, m=1, others=1, L=4095, page=64, axes=1, ladder="shared",
             pairing="halves", part=1, far=0),
        # a prompt with an image in it fills its pages
        dict(name="append prompt", kind="append", geo="llada", dtype="bf16", src="bf16", batch=1, m=2500, others=1, L=2500, page=64, axes=3, ladder="shared",
             pairing="halves", part=1, far=5000),
        # the small fp32 model, odd chunks, half of each head rotated in neighbouring pairs, each axis with frequencies of its own
        dict(name="append small f32", kind="append", geo="small", dtype="f32", src="f32", batch=5, m=33, others=33, L=389, page=32, axes=3, ladder="own",
             pairing="neighbours", part=2, far=300),
        # one token against an odd cache length
        dict(name="attention one row", kind="attention", geo="dream", dtype="bf16", batch=1, m=1, others=1, L=1023, page=64, block=1, window=0, chosen=False,
             average=False),
        # a decode step of a serving batch, lengths from a few rows to thousands
        dict(name="attention decode batch", kind="attention", geo="dream", dtype="bf16", batch=64, m=1, others=1, L=8191, page=64, block=1, window=0,
             chosen=False, average=False),
        # one token behind a long document
        dict(name="attention decode long", kind="attention", geo="dream", dtype="bf16", batch=1, m=1, others=1, L=60001, page=128, block=1, window=0,
             chosen=False, average=False),
        # a chunk of a long prompt: every row up to its own index
        dict(name="attention chunk", kind="attention", geo="llada", dtype="bf16", batch=1, m=2500, others=1, L=7000, page=64, block=1, window=0, chosen=False,
             average=False),
        # a chunk of a prompt among the single tokens of 31 others
        dict(name="attention mixed", kind="attention", geo="dream", dtype="bf16", batch=32, m=777, others=1, L=4095, page=32, block=1, window=0, chosen=False,
             average=False),
        # the selected rows of a group of four sequences in the middle of their generations, average wanted for the selection
        dict(name="attention selected", kind="attention", geo="llada", dtype="bf16", batch=4, m=45, others=38, L=1823, page=64, block=0, window=0, chosen=True,
             average=True),
        # the small fp32 model in blocks of 32 that see each other in whole, no further back than 150 rows
        dict(name="attention small f32", kind="attention", geo="small", dtype="f32", batch=3, m=128, others=97, L=389, page=32, block=32, window=150,
             chosen=False, average=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _rotary(rng):
    return dict(axes=rng.choice([1, 1, 2, 3, 4]), ladder=rng.choice(["shared", "own"]), pairing=rng.choice(["halves", "halves", "neighbours"]),
                part=rng.choice([1, 1, 2]), far=rng.choice([0, 1000, 1000000]))


def draw(rng):
    kind = rng.choice(["rotate", "append", "append", "attention", "attention", "attention", "attention"])
    geo, dtype = rng.choice(list(GEOMETRY)), "f32" if rng.random() < 0.25 else "bf16"
    heads, kv_heads, dim = GEOMETRY[geo]
    src = rng.choice([dtype, "f32"])
    if kind == "rotate":
        return dict(kind=kind, geo=geo, dtype=dtype, src=src, n=_log(rng, 1, 6075)) | _rotary(rng)
    case = dict(kind=kind, geo=geo, dtype=dtype, page=rng.choice([32, 64, 128, 256]))
    if kind == "append":
        batch, m = _log(rng, 1, 64), _log(rng, 1, 2500)
        while batch * m > 2500:
            m = (m + 1) // 2
        return case | dict(src=src, batch=batch, m=m, others=rng.choice([1, m]), L=m + _log(rng, 1, 4096)) | _rotary(rng)
    batch, length, form = _log(rng, 1, 64), _log(rng, 1, 65536), rng.choice(["token", "chunk", "chunk", "mixed", "chosen"])
    m = 1 if form == "token" else min(length, _log(rng, 2, 2500))
    others = m if form in ("chunk", "chosen") else 1
    # no more keys in all than the decode batch has (28 heads on 4, bf16), no more products than the chunk has
    while batch * length * kv_heads * dim * (2 if dtype == "bf16" else 4) > 64 * 8192 * 4 * 128 * 2 or (m + (batch - 1) * others) * length * heads > 2500 * 7000 * 32 // 2:
        batch, length, m = (batch + 1) // 2, (length + 1) // 2, (m + 1) // 2
        m = min(m, length)
        others = m if form in ("chunk", "chosen") else 1
    average = form == "chosen" and (m * batch) * length <= 1 << 24 and rng.random() < 0.7
    return case | dict(batch=batch, m=m, others=others, L=length, block=0 if form == "chosen" else rng.choice([1, 1, 1, 32, 0]),
                       window=rng.choice([0, 0, 0, _log(rng, 16, 4096)]), chosen=form == "chosen", average=average)


def _sizes(case):
    """(rows, cache length) of each sequence: the case's own for the first; the others' lengths fall to about a twentieth, oddly."""
    n = case["batch"]
    lengths = [case["L"]] + [max(1, case["L"] - b * case["L"] * 19 // (20 * n) - 7 * (b % 5)) for b in range(1, n)]
    return [(min(case["m"] if b == 0 else case["others"], x), x) for b, x in enumerate(lengths)]


def _pairs(case):
    """Rotated pairs of a head on each axis: a quarter for the first of several, the rest spread."""
    n, axes = GEOMETRY[case["geo"]][2] // 2 // case["part"], case["axes"]
    if axes == 1:
        return [n]
    rest = n - n // 4
    return [n // 4] + [rest // (axes - 1) + (a < rest % (axes - 1)) for a in range(axes - 1)]


# ------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1) % (1 << 31))


def _rows(g, n, heads, dim, dtype):
    """Rows as projections of normed activations give them: standard deviation 0.02 sqrt(4096), some rows louder than others."""
    loud = torch.exp(0.3 * torch.randn((n, 1), generator=g, device="cuda"))
    return (torch.randn((n, heads * dim), generator=g, device="cuda") * 1.28 * loud).to(dtype)


def _positions(g, case, n):
    """Axis 0 counts frames, the others places in a picture; with one axis a count.  All of it behind a context of `far` rows."""
    at, axes = torch.arange(n, device="cuda"), case["axes"]
    far = int(torch.randint(0, case["far"] + 1, (1,), generator=g, device="cuda")) + case["far"]
    if axes == 1:
        return (at + far).to(torch.int32)[None]
    side = max(2, int(round(max(n, 4) ** (1 / 3))))
    each, left = [], at
    for _ in range(axes - 1):
        each.insert(0, left % side + far)
        left = left // side
    return torch.stack([left + far] + each).to(torch.int32)


def _inputs(case, seed):
    g, (heads, kv_heads, dim) = _generator(seed), GEOMETRY[case["geo"]]
    if case["kind"] == "rotate":
        return dict(x=_rows(g, case["n"], heads, dim, TYPES[case["src"]]), pos=_positions(g, case, case["n"]))
    sizes, page = _sizes(case), case["page"]
    rows = sum(m for m, _ in sizes)
    need = [-(-n // page) for _, n in sizes]
    s = dict(n_pages=sum(need) + 3, pages=torch.full((len(sizes), max(need)), -1, dtype=torch.int32, device="cuda"))
    free = torch.randperm(s["n_pages"], generator=g, device="cuda").to(torch.int32)
    for b, n in enumerate(need):
        s["pages"][b, :n] = free[sum(need[:b]): sum(need[:b]) + n]
    starts = [0]
    for m, _ in sizes:
        starts.append(starts[-1] + m)
    s["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["length"] = torch.tensor([n for _, n in sizes], dtype=torch.int32, device="cuda")
    if case["kind"] == "append":
        t = TYPES[case["src"]]
        s["q"], s["k"], s["v"] = _rows(g, rows, heads, dim, t), _rows(g, rows, kv_heads, dim, t), _rows(g, rows, kv_heads, dim, t)
        s["pos"] = _positions(g, case, rows) if case["far"] else None
        return s
    t = TYPES[case["dtype"]]
    s["q"] = _normal(g, (rows, heads * dim), t)
    s["k"], s["v"] = ([_rows(g, n, kv_heads, dim, t) for _, n in sizes] for _ in range(2))
    if case["chosen"]:
        s["at"] = torch.cat([torch.randperm(n, generator=g, device="cuda")[:m].sort().values for m, n in sizes]).to(torch.int32)
    return s


def _normal(g, shape, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * 1.28).to(dtype)


def prepare(case, seed):
    heads, kv_heads, dim = GEOMETRY[case["geo"]]
    s = dict(case=case, heads=heads, kv_heads=kv_heads, dim=dim, dtype=TYPES[case["dtype"]]) | _inputs(case, seed)
    if own:
        return s | _own(case, s)
    if case["kind"] != "rotate":
        sizes, page = _sizes(case), case["page"]
        s["sizes"], s["page"] = sizes, page
        s["kp"], s["vp"] = (torch.zeros((s["n_pages"], page, kv_heads, dim), dtype=s["dtype"], device="cuda") for _ in range(2))
        if case["kind"] == "attention":
            for c in "kv":
                for b, rows in enumerate(s.pop(c)):
                    at = torch.arange(rows.shape[0], device="cuda")
                    s[c + "p"][s["pages"][b, at // page].long(), at % page] = rows.view(-1, kv_heads, dim)
    if case["kind"] != "attention":
        s["freq"] = torch.tensor([THETA ** -e for e, _ in _ladder(case)], dtype=torch.float64, device="cuda")
        s["axis"] = torch.tensor([a for _, a in _ladder(case)], device="cuda")
    return s


def _ladder(case):
    """(exponent of the frequency, axis) of each rotated pair."""
    each, n, first = [], sum(_pairs(case)), 0
    for a, count in enumerate(_pairs(case)):
        each += [((first + i) / n if case["ladder"] == "shared" else i / count, a) for i in range(count)]
        first += count
    return each


# ------------------------------------------------------------------ the framework's calls

def _own(case, s):
    from paper_2509_23094_amd import binding as B
    rotary = None if case["kind"] == "attention" else B.Rotary(_pairs(case), THETA, ladder=case["ladder"], pairing=case["pairing"])
    rows = s["q"].shape[0] if case["kind"] == "attention" else 0
    ctx = B.PgContext(s["heads"], s["kv_heads"], s["dim"], case["dtype"], page_rows=case.get("page", 64), max_rows=rows, max_batch=case.get("batch", 1),
                      rotary=rotary)
    if case["kind"] == "rotate":
        return dict(ctx=ctx, out=torch.zeros(s["x"].shape, dtype=s["dtype"], device="cuda"))
    cache = B.PgCache(ctx, s["n_pages"])

    def values(n):
        return [torch.zeros((n, s["kv_heads"] * s["dim"]), dtype=s["dtype"], device="cuda") for _ in range(2)]

    if case["kind"] == "append":
        group = B.PgBatch(ctx, s["row_start"], s["length"], s["pages"], s["k"].shape[0])
        return dict(ctx=ctx, cache=cache, group=group, q_out=torch.zeros(s["q"].shape, dtype=s["dtype"], device="cuda"), rows=values(s["k"].shape[0]))
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), s["length"].long().cumsum(0)]).to(torch.int32)
    k, v = torch.cat(s.pop("k")), torch.cat(s.pop("v"))
    ctx.d2c_pg_append(cache, B.PgBatch(ctx, start, s["length"], s["pages"], k.shape[0]), k, v)
    group = B.PgBatch(ctx, s["row_start"], s["length"], s["pages"], rows, at=s.get("at"))
    average = torch.zeros((rows, case["L"]), device="cuda") if case["average"] else None
    return dict(ctx=ctx, cache=cache, group=group, out=torch.zeros_like(s["q"]), average=average)


def _run_own(s):
    ctx, case = s["ctx"], s["case"]
    if case["kind"] == "rotate":
        ctx.d2c_pg_rotate(s["x"], s["pos"], s["out"])
        return [s["out"]]
    if case["kind"] == "append":
        ctx.d2c_pg_append(s["cache"], s["group"], s["k"], s["v"], pos=s["pos"], q=s["q"], q_out=s["q_out"])
        ctx.d2c_pg_read(s["cache"], s["group"], *s["rows"])
        return [s["q_out"]] + s["rows"]
    ctx.d2c_pg_attention(s["cache"], s["group"], s["q"], s["out"], block=case["block"], window=case["window"], attn_avg=s["average"])
    return [s["out"]] + ([s["average"]] if case["average"] else [])


# ------------------------------------------------------------------ the plain forms

def _rotate(s, x, pos):
    """x [n, heads * dim], pos [axes, n]; angles in 64 bits, the rotation in 32."""
    n, dim, pairs = x.shape[0], s["dim"], s["freq"].shape[0]
    angle = pos.long()[s["axis"]].t().double() * s["freq"]
    c, d = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float().view(n, -1, dim)
    if s["case"]["pairing"] == "halves":
        a, b = x[..., :pairs], x[..., pairs: 2 * pairs]
        y = torch.cat([a * c - b * d, b * c + a * d, x[..., 2 * pairs:]], 2)
    else:
        a, b = x[..., 0: 2 * pairs: 2], x[..., 1: 2 * pairs: 2]
        y = torch.cat([torch.stack([a * c - b * d, b * c + a * d], 3).flatten(2), x[..., 2 * pairs:]], 2)
    return y.view(n, -1).to(s["dtype"])


def _append(s):
    index = torch.cat([torch.arange(n - m, n, device="cuda") for m, n in s["sizes"]])
    seq = torch.repeat_interleave(torch.arange(len(s["sizes"]), device="cuda"), (s["row_start"][1:] - s["row_start"][:-1]).long(), output_size=len(index))
    pos = index.expand(s["case"]["axes"], -1) if s["pos"] is None else s["pos"]
    page, row = s["pages"][seq, index // s["page"]].long(), index % s["page"]
    shape = (len(index), s["kv_heads"], s["dim"])
    s["kp"][page, row] = _rotate(s, s["k"], pos).view(shape)
    s["vp"][page, row] = s["v"].to(s["dtype"]).view(shape)
    return [_rotate(s, s["q"], pos), s["kp"][page, row].flatten(1), s["vp"][page, row].flatten(1)]


def _seen(i, n, block, window):
    """Which of n keys rows at the indices i see."""
    j, i = torch.arange(n, device="cuda")[None], i[:, None]
    ok = j < (i // block + 1) * block if block else torch.ones_like(i * j, dtype=torch.bool)
    if window:
        ok = ok & (j > i - window)
        if not block:
            ok = ok & (j < i + window)
    return ok


def _attention(s):
    case, heads, kv, dim = s["case"], s["heads"], s["kv_heads"], s["dim"]
    out, avg, first = torch.zeros_like(s["q"]), torch.zeros((s["q"].shape[0], case["L"]), device="cuda") if case["average"] else None, 0
    for b, (m, n) in enumerate(s["sizes"]):
        pages = s["pages"][b, : -(-n // s["page"])].long()
        k, v = (s[c][pages].flatten(0, 1)[:n].float().permute(1, 0, 2).contiguous() for c in ("kp", "vp"))
        rows = slice(first, first + m)
        q = s["q"][rows].float().view(m, kv, heads // kv, dim).permute(1, 2, 0, 3).reshape(kv, heads // kv * m, dim).contiguous()
        p = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(dim)
        i = s["at"][rows].long() if case["chosen"] else torch.arange(n - m, n, device="cuda")
        if case["block"] or case["window"]:
            p = torch.where(_seen(i, n, case["block"], case["window"]).repeat(heads // kv, 1), p, -math.inf)
        p = torch.exp(p - p.amax(2, keepdim=True))
        p = p / p.sum(2, keepdim=True)
        out[rows] = torch.matmul(p, v).view(heads, m, dim).transpose(0, 1).reshape(m, heads * dim).to(s["dtype"])
        if avg is not None:
            avg[rows, :n] = p.view(heads, m, n).mean(0)
        first += m
    return [out] + ([avg] if avg is not None else [])


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "rotate":
        return [_rotate(state, state["x"], state["pos"])]
    return _append(state) if kind == "append" else _attention(state)


def _visible(m, n, case):
    """Pairs of a row and a key that it sees."""
    block, window, total = case["block"], case["window"], 0
    if not (block or window):
        return m * n
    for i in (range(n - m, n) if not case["chosen"] else [(2 * r + 1) * n // (2 * m) for r in range(m)]):
        hi = min(n, (i // block + 1) * block) if block else min(n, i + window)
        total += hi - (max(0, i - window + 1) if window else 0)
    return total


def work(case):
    heads, kv_heads, dim = GEOMETRY[case["geo"]]
    t, src = 2 if case["dtype"] == "bf16" else 4, 2 if case.get("src", "f32") == "bf16" else 4
    if case["kind"] == "rotate":
        return dict(bytes=case["n"] * (heads * dim * (t + src) + 4 * case["axes"]), flops=3 * case["n"] * heads * dim // case["part"])
    sizes = _sizes(case)
    rows = sum(m for m, _ in sizes)
    if case["kind"] == "append":
        # rows in, queries out, keys and values into the pages and back out as values
        return dict(bytes=rows * (heads * dim * (t + src) + 2 * kv_heads * dim * (src + 3 * t) + (4 * case["axes"] if case["far"] else 0)),
                    flops=3 * rows * (heads + kv_heads) * dim // case["part"])
    keys = sum(min(n, m + case["window"]) if case["window"] and not case["chosen"] else n for m, n in sizes)
    return dict(bytes=2 * keys * kv_heads * dim * t + 2 * rows * heads * dim * t + (4 * sum(m * n for m, n in sizes) if case["average"] else 0),
                flops=4 * heads * dim * sum(_visible(m, n, case) for m, n in sizes))


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_rotate(case, x, pos):
    """Pairs as complex numbers, turned by exp(i angle)."""
    dim = GEOMETRY[case["geo"]][2]
    each, half = _ladder(case), len(_ladder(case))
    angle = torch.stack([pos[a].double() * THETA ** -e for e, a in each], 1)[:, None]
    x = x.double().unflatten(1, (-1, dim))
    turned, rest = x[..., : 2 * half], x[..., 2 * half:]
    z = turned.unflatten(2, (2, half)).transpose(2, 3) if case["pairing"] == "halves" else turned.unflatten(2, (half, 2))
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * torch.polar(torch.ones_like(angle), angle))
    return torch.cat([(z.transpose(2, 3) if case["pairing"] == "halves" else z).flatten(2), rest], 2).flatten(1)


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] == "rotate":
        return [_exact_rotate(case, x["x"], x["pos"])]
    sizes = _sizes(case)
    if case["kind"] == "append":
        pos = x["pos"] if x["pos"] is not None else torch.cat([torch.arange(n, device="cuda")[n - m:] for m, n in sizes]).repeat(case["axes"], 1)
        return [_exact_rotate(case, x["q"], pos), _exact_rotate(case, x["k"], pos), x["v"].double()]
    heads, kv_heads, dim = GEOMETRY[case["geo"]]
    out, avg = torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda"), torch.zeros((x["q"].shape[0], case["L"]), dtype=torch.float64, device="cuda")
    starts = x["row_start"].tolist()
    for b, (m, n) in enumerate(sizes):
        rows = slice(starts[b], starts[b] + m)
        at = x["at"][rows].double() if case["chosen"] else torch.arange(m, device="cuda").double() + (n - m)
        keys, hidden = torch.arange(n, device="cuda").double(), torch.zeros((m, n), dtype=torch.bool, device="cuda")
        if case["block"]:
            hidden |= (keys / case["block"]).floor() > (at / case["block"]).floor()[:, None]
        if case["window"]:
            hidden |= at[:, None] - keys >= case["window"]
            if not case["block"]:
                hidden |= keys - at[:, None] >= case["window"]
        for h in range(heads):
            g = h * kv_heads // heads * dim
            k, v = (x[c][b][:, g: g + dim].double() for c in "kv")
            score = x["q"][rows, h * dim: (h + 1) * dim].double() @ k.t() * dim ** -0.5
            p = torch.softmax(score.masked_fill(hidden, -math.inf), 1)
            out[rows, h * dim: (h + 1) * dim] = p @ v
            if case["average"]:
                avg[rows, :n] += p / heads
    return [out] + ([avg] if case["average"] else [])
