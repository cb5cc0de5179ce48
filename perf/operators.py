"""Performance cases of the operators of the 8-bit paged cache, with their plain forms.

A case is a dict of plain values.  `op` names the operator:

  map     kvd_q8_map: page table, rows and runs of a step from the lengths of its requests
  append  kvd_q8_append: the rows' keys and values into the pages, in 8 bits, and the pages' mean keys
  select  kvd_q8_select: the pages with the best scores for every row
  attn    kvd_q8_attn: attention of the rows over all their pages, or over `topk` selected ones

Sizes: `batch` sequences that hold `context` tokens each before the step (with `ragged` the later ones are shorter, down
to a sixteenth) and get `new` tokens in it (with `ragged` the earlier ones fewer), pages of `page` tokens of `kv_heads`
heads of 128 elements, `q_heads` query heads; buffers of a `map` hold `spare` rows more than the step has.
"""
import math

import torch

own = False

DEV = "cuda"
D = 128
TILE = 16                        # tokens of a tile of a page
EXP_MIN = -96                    # the least exponent of a scale


def _case(name, op, **kw):
    c = dict(name=name, op=op, batch=1, context=0, new=1, ragged=False, page=16, q_heads=32, kv_heads=8, dtype="bf16", topk=0,
             sink=0, recent=0, spare=0)
    c.update(kw)
    return c


def listed():
    return [
        # the bookkeeping of a decode step of a full serving batch: one token for each request
        _case("map_step", "map", batch=256, context=8192),
        # prompts of different lengths that are read in one step
        _case("map_prompts", "map", batch=96, context=0, new=1024, ragged=True, spare=13),
        # one token for each request into pages that are partly filled
        _case("append_step", "append", batch=64, context=1000, ragged=True),
        # the prompts of eight requests at once, nothing cached before
        _case("append_prompts", "append", batch=8, new=4096),
        # the next pieces of long prompts, seven query heads a KV head, large pages that begin and end inside a piece
        _case("append_pieces_page64", "append", dtype="f16", q_heads=28, kv_heads=4, batch=24, context=5000, new=777, ragged=True,
              page=64),
        # the pages of sixteen long contexts scored for one token each
        _case("select_step_128k", "select", batch=16, context=131071, topk=256, sink=1, recent=4),
        # several drafted tokens a request, each with pages of its own
        _case("select_drafts", "select", dtype="f16", q_heads=28, kv_heads=4, batch=12, context=30000, new=4, ragged=True, page=32,
              topk=64, recent=1),
        # interactive chat: few short contexts, launch latency counts
        _case("attn_step_1k", "attn", batch=4, context=1000, ragged=True),
        # the serving batch of ordinary contexts, bound by the memory
        _case("attn_step_32k", "attn", batch=16, context=32767),
        # contexts of very different lengths, drafted tokens, large pages
        _case("attn_drafts_ragged", "attn", dtype="f16", q_heads=28, kv_heads=4, batch=24, context=40000, new=3, ragged=True, page=32),
        # long contexts of which each head reads the pages selected for it
        _case("attn_selected_128k", "attn", batch=16, context=131071, topk=256),
        # pieces of prompts behind what was read before: bound by the matrix cores
        _case("attn_pieces_8k", "attn", batch=2, context=6144, new=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the ranges above: 1 to 512 sequences of up to a million tokens, steps of one token to 65536."""
    while True:
        c = _draw(rng)
        w, held = work(c), sum(-(-n // c["page"]) for n in _ends(c)) * c["page"] * c["kv_heads"] * 2 * D
        # the plain form's scores are the largest thing it makes
        scores = c["batch"] * max(_news(c)) * c["q_heads"] * (max(_ends(c)) if not c["topk"] else c["topk"] * c["page"])
        gathered = max(_ends(c)) * c["batch"] * c["kv_heads"] * D if c["op"] == "attn" and not c["topk"] else 0
        if c["op"] in ("append", "attn") and held > 2 << 30 or gathered > 1 << 29:
            continue
        if c["op"] == "attn" and c["topk"] and sum(_news(c)) * c["topk"] * c["page"] * c["kv_heads"] * D > 1 << 28:
            continue
        if c["op"] == "select" and sum(_news(c)) * max(_ends(c)) // c["page"] * c["kv_heads"] * D > 1 << 28:
            continue
        if w["flops"] <= 4.5e11 and w["bytes"] <= 1.0e9 and (c["op"] != "attn" or scores <= 1.1e9) and sum(_news(c)) <= 65536:
            return c


def _draw(rng):
    op = rng.choice(["map", "append", "select", "attn", "attn", "attn"])
    kv_heads = rng.choice([1, 2, 4, 8])
    q_heads = kv_heads * rng.choice([1, 2, 4, 4, 5, 7, 8])
    page = rng.choice([16, 16, 16, 32, 48, 64, 128])
    batch = _log(rng, 1, 512 if op in ("map", "append") else 64)
    step = rng.random() < 0.6
    new = 1 if step else _log(rng, 2, 8) if rng.random() < 0.4 else _log(rng, 9, 4096)
    context = _log(rng, 1 if rng.random() < 0.3 else 256, 1000000 if batch * kv_heads <= 4 else 131072)
    if new > 8 and rng.random() < 0.4:
        context = 0
    topk = 0
    if op == "select" or (op == "attn" and rng.random() < 0.35):
        topk = max(1, min(2048, _log(rng, 256, 8192) // page))
        new = min(new, 64)
    forced = topk // 16 if op == "select" and rng.random() < 0.5 else 0
    return _case("", op, batch=batch, context=context, new=new, ragged=rng.random() < 0.6, page=page, q_heads=q_heads,
                 kv_heads=kv_heads, dtype=rng.choice(["f16", "bf16"]), topk=topk, sink=forced, recent=forced,
                 spare=rng.choice([0, 0, rng.randint(1, 64)]) if op == "map" else 0)


# ---- sizes ---------------------------------------------------------------------------------------

def _lens(c):
    """Tokens of every sequence before the step."""
    n, B = c["context"], c["batch"]
    return [max(min(n, 1), n - (15 * n * b) // (16 * B) - 3 * b) if c["ragged"] else n for b in range(B)]


def _news(c):
    """New tokens of every sequence."""
    n, B = c["new"], c["batch"]
    return [max(1, n - (7 * n * (B - 1 - b)) // (8 * B)) if c["ragged"] else n for b in range(B)]


def _ends(c):
    return [a + n for a, n in zip(_lens(c), _news(c))]


def _pages(c):
    """Columns of the page table."""
    return max(-(-n // c["page"]) for n in _ends(c))


def work(c):
    P, H, Hq, lens, news, ends = c["page"], c["kv_heads"], c["q_heads"], _lens(c), _news(c), _ends(c)
    T, B = sum(news), c["batch"]
    runs = sum((e - 1) // P - a // P + 1 for a, e in zip(lens, ends))
    if c["op"] == "map":
        fresh = sum(-(-e // P) - -(-a // P) for a, e in zip(lens, ends))
        return {"bytes": 8 * B + 8 * fresh + 4 * runs + 8 * B + 8 * T + 16 * runs, "flops": 0}
    if c["op"] == "append":
        kept = sum(a % P for a in lens)                                  # tokens whose keys the mean is taken of once more
        return {"bytes": T * H * D * 6 + kept * H * D + runs * (16 + H * (4 + D + 4)), "flops": 4 * T * H * D}
    seen = [[a + i + 1 for i in range(n)] for a, n in zip(lens, news)]   # tokens that each row sees
    if c["op"] == "select":
        pages = sum(-(-x // P) for s in seen for x in s)
        read = sum(-(-e // P) for e in ends)
        return {"bytes": read * (H * (D + 4) + 4) + T * (Hq * D * 2 + H * c["topk"] * 4 + 8), "flops": 2 * pages * H * D}
    if c["topk"]:
        tokens = sum(min(x, c["topk"] * P) for s in seen for x in s)
        return {"bytes": tokens * H * 2 * D + T * H * c["topk"] * 4 + T * Hq * D * 4, "flops": 4 * tokens * Hq * D}
    tokens = sum(sum(s) for s in seen)
    return {"bytes": sum(ends) * H * 2 * D + sum(-(-e // P) for e in ends) * (4 + 2 * H) + T * Hq * (D * 4 + 4),
            "flops": 4 * tokens * Hq * D}


# ---- inputs --------------------------------------------------------------------------------------

def _dtype(c):
    return torch.float16 if c["dtype"] == "f16" else torch.bfloat16


def _gen(seed, *stream):
    g = torch.Generator(device=DEV)
    n = int(seed)
    for s in stream:
        n = (n * 1000003 + s + 1) % (1 << 62)
    g.manual_seed(n)
    return g


def _i32(values):
    return torch.tensor(values, dtype=torch.int32).to(DEV)


def _rows(c, seed):
    """The step as `map` leaves it: table, lengths, rows and runs, with the blocks of the pool dealt out at random."""
    lens, news, ends, P, NP = _lens(c), _news(c), _ends(c), c["page"], _pages(c)
    B, T = c["batch"], sum(news)
    a, n, e = (torch.tensor(v) for v in (lens, news, ends))
    have = -(-e // P)
    NB = int(have.sum()) + 7
    cpu = torch.Generator()
    cpu.manual_seed(int(seed) % (1 << 62))
    blocks = torch.randperm(NB, generator=cpu)
    used = torch.arange(NP)[None, :] < have[:, None]
    table = torch.full((B, NP), -1)
    table[used] = blocks[: int(have.sum())]
    start = torch.zeros(B + 1, dtype=torch.int64)
    start[1:] = n.cumsum(0)
    seq = torch.repeat_interleave(torch.arange(B), n)
    pos = a[seq] + torch.arange(T) - start[seq]
    first = a // P
    count = (e - 1) // P - first + 1
    rseq = torch.repeat_interleave(torch.arange(B), count)
    rpage = first[rseq] + torch.arange(len(rseq)) - (count.cumsum(0) - count)[rseq]
    lo, hi = torch.maximum(rpage * P, a[rseq]), torch.minimum((rpage + 1) * P, e[rseq])
    runs = torch.stack([table[rseq, rpage], start[rseq] + lo - a[rseq], lo - rpage * P, hi - lo], 1)
    to = lambda t: t.to(torch.int32).to(DEV)  # noqa: E731
    return dict(blocks=NB, n_rows=T, n_runs=len(rseq), table=to(table), kv_len=to(e), row_start=to(start), row_seq=to(seq), row_pos=to(pos), runs=to(runs),
                counts=torch.zeros(5, dtype=torch.int32, device=DEV))


def _keys(shape, g, dtype):
    """Keys as they come out of a projection: N(0, 1) with a few channels that are several times as large."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=dtype)
    x[..., 5::41] *= 6.0
    return x


def prepare(case, seed):
    c, g = case, _gen(seed, 0)
    H, P, T, dt = c["kv_heads"], c["page"], sum(_news(c)), _dtype(c)
    s = dict(case=c)
    if c["op"] == "map":
        lens, news = _lens(c), _news(c)
        NP, B = _pages(c), c["batch"]
        have = [-(-n // P) for n in lens]
        NB = sum(-(-e // P) for e in _ends(c)) + 100
        blocks = torch.randperm(NB, generator=g, device=DEV).to(torch.int32)
        used = torch.arange(NP, device=DEV)[None, :] < _i32(have)[:, None]
        table = torch.full((B, NP), -1, dtype=torch.int32, device=DEV)
        table[used] = blocks[: sum(have)]
        T += c["spare"]
        runs = min(T, T // P + 2 * B)
        s.update(blocks=NB, table=table, seq_len=_i32(lens), n_new=_i32(news), free=blocks[sum(have):].contiguous(),
                 free_count=_i32([NB - sum(have)]), n_rows=T, n_runs=runs)
        return s
    s.update(_rows(c, seed))
    NB = s["blocks"]
    if c["op"] == "select":
        s["means"] = (torch.randn((NB, H, D), generator=g, device=DEV) * 40.0).round().clamp(-127, 127).to(torch.int8)
        p2 = _two(torch.randint(-9, -5, (NB, H), generator=g, device=DEV)).float()
        s["mean_scales"] = p2 / torch.where(torch.rand((NB, H), generator=g, device=DEV) < 0.02, 7.0, float(P))
    else:
        # 8-bit pages as appending leaves them: the largest value of a page and head near the top of the range
        codes = torch.empty((NB, H, P // TILE, 2, TILE * D), dtype=torch.float8_e4m3fn, device=DEV)
        step = max(1, (1 << 28) // codes[0].numel())
        for i in range(0, NB, step):
            x = torch.randn(codes[i:i + step].shape, generator=g, device=DEV, dtype=torch.bfloat16)
            codes[i:i + step] = (x * 75.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
        s["pages"] = codes.view(torch.uint8)
        s["exps"] = torch.randint(-7, -4, (NB, H, 2), generator=g, device=DEV).to(torch.int8)
    if c["op"] == "append":
        s["means"] = torch.zeros((NB, H, D), dtype=torch.int8, device=DEV)
        s["mean_scales"] = torch.zeros((NB, H), device=DEV)
        s["k_new"] = _keys((T, H, D), g, dt)
        s["v_new"] = torch.randn((T, H, D), generator=g, device=DEV, dtype=dt)
        return s
    s["q"] = torch.randn((T, c["q_heads"], D), generator=g, device=DEV).to(dt)
    if c["op"] == "select":
        s["sel"] = torch.empty((T, H, c["topk"]), dtype=torch.int32, device=DEV)
        return s
    s["out"] = torch.empty((T, c["q_heads"], D), dtype=dt, device=DEV)
    s["lse"] = torch.empty((T, c["q_heads"]), dtype=torch.float32, device=DEV)
    if c["topk"]:
        seen = -(-(s["row_pos"] + 1) // P)
        key = torch.rand((T, H, _pages(c)), generator=g, device=DEV)
        at = torch.arange(_pages(c), device=DEV)
        key = torch.where(at < seen[:, None, None], key, torch.full_like(key, -1.0))
        key = torch.where(at == seen[:, None, None] - 1, torch.full_like(key, 2.0), key)   # the newest page is always read
        v, i = key.topk(min(c["topk"], _pages(c)), dim=-1)
        i = torch.where(v >= 0, i, torch.full_like(i, 1 << 40)).sort(dim=-1).values
        sel = torch.full((T, H, c["topk"]), -1, dtype=torch.int32, device=DEV)
        sel[..., : i.shape[-1]] = torch.where(i < 1 << 40, i, torch.full_like(i, -1)).to(torch.int32)
        s["sel"] = sel
    return s


# ---- one pass ------------------------------------------------------------------------------------

def _handle(s):
    """The framework's rows and cache over the state's buffers, kept with them."""
    if "rows" not in s:
        from paper_2605_18071_amd import kvd
        c = s["case"]
        names = () if c["op"] == "map" else ("kv_len", "row_start", "row_seq", "row_pos", "runs", "counts")
        s["rows"] = kvd.Q8Rows(s["table"], page_size=c["page"], n_blocks=s["blocks"], n_rows=s["n_rows"], max_runs=s["n_runs"],
                               **{n: s[n] for n in names})
        if c["op"] != "map":
            s["cache"] = kvd.Q8Cache(
                n_blocks=s["blocks"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], page_size=c["page"], kv_dtype=_dtype(c),
                sink_pages=c["sink"], recent_pages=c["recent"],
                buffers={n: s[n] for n in ("pages", "exps", "means", "mean_scales") if n in s})
            s["ws"] = s["cache"].workspace(s["rows"], select=c["op"] == "select")
    return s["rows"], s.get("cache")


def run(s):
    c = s["case"]
    if own:
        rows, cache = _handle(s)
        if c["op"] == "map":
            rows.map(s["seq_len"], s["n_new"], s["free"], s["free_count"])
            return dict(table=s["table"], kv_len=rows.kv_len, row_start=rows.row_start, row_seq=rows.row_seq, row_pos=rows.row_pos,
                        runs=rows.runs, counts=rows.counts)
        if c["op"] == "append":
            cache.append(rows, s["k_new"], s["v_new"])
            return dict(pages=s["pages"].view(torch.float8_e4m3fn), exps=s["exps"], means=s["means"], mean_scales=s["mean_scales"])
        if c["op"] == "select":
            cache.select(rows, s["q"], s["sel"], s["ws"])
            return dict(sel=s["sel"])
        cache.attend(rows, s["q"], s["out"], s["ws"], lse=s["lse"], sel_pages=s.get("sel"))
        return dict(out=s["out"], lse=s["lse"])
    return {"map": _map, "append": _append, "select": _select, "attn": _attend}[c["op"]](s)


# ---- the plain forms -----------------------------------------------------------------------------

def _map(s):
    P, T, R = s["case"]["page"], s["n_rows"], s["n_runs"]
    table, lens, news = s["table"], s["seq_len"], s["n_new"]
    B, NP = table.shape
    ends = lens + news
    start = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    start[1:] = news.cumsum(0)
    first, last = (lens + P - 1) // P, (ends + P - 1) // P
    fresh = last - first
    taken = fresh.cumsum(0).to(torch.int32)
    at = torch.arange(NP, device=DEV, dtype=torch.int32)[None, :]
    nth = (taken - fresh)[:, None] + at - first[:, None]
    is_new = (at >= first[:, None]) & (at < last[:, None])
    table.copy_(torch.where(is_new, s["free"][(s["free_count"] - 1 - nth).clamp(0, len(s["free"]) - 1).long()], table))
    none = torch.full((), -1, dtype=torch.int32, device=DEV)
    r = torch.arange(T, device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(start[1:].contiguous(), r, right=True).clamp(max=B - 1)
    real = r < start[-1]
    row_seq = torch.where(real, seq.to(torch.int32), none)
    row_pos = torch.where(real, lens[seq] + r - start[seq], none)
    page0 = lens // P
    n_runs = torch.where(news > 0, (ends - 1) // P - page0 + 1, torch.zeros_like(news))
    upto = n_runs.cumsum(0).to(torch.int32)
    i = torch.arange(R, device=DEV, dtype=torch.int32)
    b = torch.searchsorted(upto, i, right=True).clamp(max=B - 1)
    page = page0[b] + i - (upto - n_runs)[b]
    lo, hi = torch.maximum(page * P, lens[b]), torch.minimum((page + 1) * P, ends[b])
    one = torch.stack([table[b, page.clamp(0, NP - 1).long()], start[b] + lo - lens[b], lo - page * P, hi - lo], 1)
    pad = -(torch.arange(4, device=DEV, dtype=torch.int32) == 0).to(torch.int32)
    runs = torch.where((i < upto[-1])[:, None], one, pad)
    counts = torch.stack([start[-1], upto[-1], taken[-1], s["free_count"][0] - taken[-1], torch.zeros_like(taken[-1])])
    return dict(table=table, kv_len=ends, row_start=start, row_seq=row_seq, row_pos=row_pos, runs=runs, counts=counts)


def _natural(tiles):
    """Codes of the pages [..., tiles, 2, 2048] as keys and values [..., tokens, D] each.  A tile's keys lie in the order
    [half][8 dims of 32][token][32 dims of 64][dim], its values in [half][4 tokens][dim of 16][16 dims of 64][token]."""
    head = tiles.shape[:-3]
    n = len(head)
    k = tiles[..., 0, :].unflatten(-1, (2, 4, 16, 2, 8))
    v = tiles[..., 1, :].unflatten(-1, (2, 4, 16, 4, 4))
    lead = list(range(n + 1))
    k = k.permute(lead + [n + 3, n + 1, n + 4, n + 2, n + 5])            # tile, token | half, 32 dims, 8 dims, dim
    v = v.permute(lead + [n + 2, n + 5, n + 1, n + 4, n + 3])            # tile, 4 tokens, token | half, 16 dims, dim
    return k.reshape(head + (-1, D)), v.reshape(head + (-1, D))


def _tiled(k, v):
    """The other way: keys and values [..., P, D] as tiles [..., tiles, 2, 2048]."""
    n = k.dim() - 2
    lead = list(range(n + 1))
    k = k.unflatten(-2, (-1, 16)).unflatten(-1, (2, 2, 4, 8)).permute(lead + [n + 2, n + 4, n + 1, n + 3, n + 5])
    v = v.unflatten(-2, (-1, 4, 4)).unflatten(-1, (2, 4, 16)).permute(lead + [n + 3, n + 1, n + 5, n + 4, n + 2])
    return torch.stack([k.flatten(n + 1), v.flatten(n + 1)], n + 1)


def _two(e):
    """2^e of whole numbers, in 64 bits: the bits themselves, which no rounding of a power function can touch."""
    return ((e.to(torch.int64).clamp(-1022, 1023) + 1023) << 52).view(torch.float64)


def _append(s):
    P, runs = s["case"]["page"], s["runs"].long()
    block, row, off, count = (runs[:, i] for i in range(4))
    fp8 = s["pages"].view(torch.float8_e4m3fn)
    ok, ov = _natural(s["pages"][block])                                 # [runs][H][P][D] codes
    old = torch.stack([ok, ov], 2).view(torch.float8_e4m3fn).float()     # [runs][H][2][P][D]
    t = torch.arange(P, device=DEV)[None, :]
    fresh = ((t >= off[:, None]) & (t < (off + count)[:, None]))[:, None, None, :, None]
    kept = (t < off[:, None])[:, None, None, :, None]
    src = (row[:, None] + t - off[:, None]).clamp(0, s["k_new"].shape[0] - 1)
    new = torch.stack([s["k_new"][src], s["v_new"][src]], 1).float().permute(0, 3, 1, 2, 4)     # [runs][H][2][P][D]
    new = torch.where(fresh, new, torch.zeros((), device=DEV)).nan_to_num(0.0, math.inf, -math.inf)
    amax = torch.where(new.isinf(), torch.zeros((), device=DEV), new).abs().amax((-2, -1))
    m, x = torch.frexp(amax)                                             # m in [1/2, 1): 448 is 7/8 of 2^9
    need = torch.where(amax > 0, x - 9 + (m > 0.875).to(x.dtype), torch.full_like(x, EXP_MIN)).clamp(min=EXP_MIN)
    was, begins = s["exps"][block].to(x.dtype), (off == 0)[:, None, None]
    e = torch.where(begins, need, torch.maximum(was, need))
    up = lambda v: _two(v)[..., None, None].float()  # noqa: E731
    scaled = torch.where(fresh, (new * up(-e)).clamp(-448, 448), torch.where(kept, old * up(was - e), old))
    scaled = torch.where(begins[..., None, None] & ~fresh, torch.zeros((), device=DEV), scaled)
    codes = scaled.to(torch.float8_e4m3fn)
    s["pages"][block] = _tiled(codes[:, :, 0].view(torch.uint8), codes[:, :, 1].view(torch.uint8))
    s["exps"][block] = e.to(torch.int8)
    total = torch.where((fresh | kept)[:, :, 0], codes[:, :, 0].float() * 512.0, torch.zeros((), device=DEV)).double().sum(2)
    a = total.abs().amax(-1)
    m, x = torch.frexp(a)                                                # 127 is 127/128 of 2^7
    sh = (x - 7 + (m > 127.0 / 128.0).to(x.dtype)).clamp(min=0)
    s["means"][block] = (total * _two(-sh)[..., None]).round().to(torch.int8)
    s["mean_scales"][block] = (_two(sh + e[..., 0] - 9) / (off + count)[:, None]).float()
    return dict(pages=fp8, exps=s["exps"], means=s["means"], mean_scales=s["mean_scales"])


def _select(s):
    c, q = s["case"], s["q"]
    P, H, k = c["page"], c["kv_heads"], c["topk"]
    T, NP = q.shape[0], s["table"].shape[1]
    qs = q.unflatten(1, (H, -1)).double().sum(2)
    amax = qs.abs().amax(-1, keepdim=True)
    qi = (qs * torch.div(torch.full_like(amax, 127.0), amax)).round().float()
    blocks = s["table"][s["row_seq"].long()].clamp(min=0).long()         # [T][NP]
    dot = torch.matmul(s["means"][blocks].permute(0, 2, 1, 3).float(), qi[..., None])[..., 0]     # whole numbers below 2^24
    score = dot * s["mean_scales"][blocks].transpose(1, 2)
    seen = ((s["row_pos"] + P) // P)[:, None, None]
    at = torch.arange(NP, device=DEV)
    score = torch.where((at < c["sink"]) | (at >= seen - c["recent"]), torch.full_like(score, math.inf), score)
    score = torch.where(at < seen, score, torch.full_like(score, -math.inf))
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :k]
    best = torch.where(torch.arange(best.shape[-1], device=DEV) < seen, best, torch.full_like(best, 1 << 40)).sort(dim=-1).values
    s["sel"].fill_(-1)
    s["sel"][..., : best.shape[-1]] = torch.where(best < 1 << 40, best, torch.full_like(best, -1)).to(torch.int32)
    return dict(sel=s["sel"])


def _attend(s):
    c, q = s["case"], s["q"].float()
    P, H, B = c["page"], c["kv_heads"], c["batch"]
    T, G, scale = q.shape[0], c["q_heads"] // H, 1.0 / math.sqrt(D)
    table = s["table"].clamp(min=0).long()
    h = torch.arange(H, device=DEV)
    if c["topk"]:                                                        # every row and head its own pages
        page = s["sel"].long()                                           # [T][H][k]
        block = table[s["row_seq"].long()[:, None, None], page.clamp(min=0)]
        codes, exps = s["pages"][block, h[None, :, None]], s["exps"][block, h[None, :, None]]
        at = page[..., None] * P + torch.arange(P, device=DEV)
        at = torch.where(page[..., None] >= 0, at, torch.full_like(at, 1 << 40)).flatten(2)       # [T][H][tokens]
        seen = (at <= s["row_pos"][:, None, None])[:, :, None, :]
        query = q.unflatten(1, (H, G))                                   # [T][H][G][D]
    else:                                                                # the rows of a sequence together, as many as the longest has
        n = max(_news(c))
        lens, starts = s["kv_len"].long(), s["row_start"].long()
        count = starts[1:] - starts[:-1]
        i = torch.arange(n, device=DEV)
        row = (starts[:-1, None] + i).clamp(max=T - 1)                   # [B][n]
        block = table[:, None, :]
        codes, exps = s["pages"][block, h[None, :, None]], s["exps"][block, h[None, :, None]]
        at = torch.arange(table.shape[1] * P, device=DEV)
        last = lens[:, None] - count[:, None] + i                        # [B][n] positions
        seen = (at <= last[..., None])[:, None, :, None, :].expand(B, H, n, G, at.numel()).flatten(2, 3)
        query = q[row].unflatten(2, (H, G)).transpose(1, 2).flatten(2, 3)                        # [B][H][n G][D]
    k, v = _natural(codes)                                               # [..][pages][P][D] codes
    up = _two(exps).float()[..., None, None]
    k = (k.view(torch.float8_e4m3fn).float() * up[..., 0, :, :]).flatten(2, 3)
    logits = torch.matmul(query, k.transpose(-1, -2).contiguous()) * scale
    del k
    logits.masked_fill_(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = (logits - top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + top)[..., 0]
    out = torch.matmul(p, (v.view(torch.float8_e4m3fn).float() * up[..., 1, :, :]).flatten(2, 3)) / total
    if c["topk"]:
        s["out"].copy_(out.flatten(1, 2))
        s["lse"].copy_(lse.flatten(1, 2))
    else:
        seq, nth = s["row_seq"].long(), s["row_pos"].long()
        nth = nth - (lens - count)[seq]
        s["out"].copy_(out.unflatten(2, (n, G))[seq, :, nth].flatten(1, 2))
        s["lse"].copy_(lse.unflatten(2, (n, G))[seq, :, nth].flatten(1, 2))
    return dict(out=s["out"], lse=s["lse"])


# ---- the definitions, in 64 bits -----------------------------------------------------------------

def _power(e):
    """2^e: looked up among the powers that the CPU has."""
    return torch.tensor([math.ldexp(1.0, n) for n in range(-512, 512)], dtype=torch.float64, device=DEV)[e.long() + 512]


def _value(code, e):
    """The number that an 8-bit code of a scale 2^e stands for: sign, four bits of exponent, three of mantissa."""
    code = code.to(torch.int64)
    sign, ex, man = code >> 7, (code >> 3) & 15, code & 7
    mag = torch.where(ex == 0, man.double() * 2.0 ** -9, (8 + man).double() * _power(ex - 10))
    return torch.where(sign == 1, -mag, mag) * _power(e)


def _nearest(x):
    """x, at most 448, to the nearest value of 8 bits: eight steps an octave, steps of 2^-9 below 2^-6; halves to the even one."""
    _, ex = torch.frexp(x)
    step = _power(ex.clamp(min=-5) - 4)
    return (x / step).round() * step


def _page(pages, blocks, h, which):
    """Codes of one head's pages in the order of their tokens: [tokens][D] of keys (0) or values (1)."""
    P = pages.shape[2] * TILE
    t, d = torch.arange(P, device=DEV)[:, None], torch.arange(D, device=DEV)[None, :]
    i = t % TILE
    if which == 0:
        at = d // 64 * 1024 + (d // 8 % 4 * 16 + i) * 16 + d // 32 % 2 * 8 + d % 8
    else:
        at = d // 64 * 1024 + (i // 4 * 16 + d % 16) * 16 + d // 16 % 4 * 4 + i % 4
    flat = (t // TILE * 2 + which) * (TILE * D) + at
    return pages[blocks, h].flatten(1)[:, flat.flatten()].reshape(-1, D)


def exact(case, seed):
    c = case
    if c["op"] in ("map", "select"):
        return None                                                      # whole numbers
    s = prepare(case, seed)
    P, H = c["page"], c["kv_heads"]
    if c["op"] == "append":
        if s["runs"].shape[0] * H > 70000:
            return None
        values = torch.empty(s["pages"].shape, dtype=torch.float64, device=DEV)
        for i in range(0, s["blocks"], 256):
            values[i:i + 256] = _value(s["pages"][i:i + 256], torch.zeros(1, dtype=torch.int8, device=DEV))
        scales = s["mean_scales"].double()
        runs = s["runs"].long()
        t, d = torch.arange(P, device=DEV)[:, None], torch.arange(D, device=DEV)[None, :]
        i = t % TILE
        place = [(t // TILE * 2) * (TILE * D) + d // 64 * 1024 + (d // 8 % 4 * 16 + i) * 16 + d // 32 % 2 * 8 + d % 8,
                 (t // TILE * 2 + 1) * (TILE * D) + d // 64 * 1024 + (i // 4 * 16 + d % 16) * 16 + d // 16 % 4 * 4 + i % 4]
        for j in range(0, runs.shape[0], 1024):
            block, row, off, count = runs[j:j + 1024].T
            at = torch.arange(P, device=DEV)
            hi = (off + count)[:, None, None, None]
            tok = at[None, None, :, None]
            first = off[:, None, None, None]
            for which, x in enumerate((s["k_new"], s["v_new"])):
                src = (row[:, None] + at - off[:, None]).clamp(0, x.shape[0] - 1)
                fresh = (tok >= first) & (tok < hi)
                new = torch.where(fresh, x[src].double().transpose(1, 2), torch.zeros((), dtype=torch.float64, device=DEV))
                a = new.abs().amax((-2, -1))
                need = torch.ceil(torch.log2(a / 448.0))
                need = torch.where(448.0 * _power(need - 1) >= a, need - 1, need)
                need = torch.where(448.0 * _power(need) < a, need + 1, need)
                need = torch.where(a > 0, need, torch.full_like(need, EXP_MIN)).clamp(min=EXP_MIN)
                was = s["exps"][block, :, which].double()
                e = torch.where((off == 0)[:, None], need, torch.maximum(was, need))
                held = values[block].flatten(2)[..., place[which].flatten()].unflatten(-1, (P, D))
                kept = _nearest(held * _power(was - e)[..., None, None])
                got = torch.where(fresh, _nearest(new * _power(-e)[..., None, None]), torch.where(tok < first, kept, held))
                got = torch.where((first == 0) & ~fresh, torch.zeros((), dtype=torch.float64, device=DEV), got)
                whole = values[block].flatten(2)
                whole[..., place[which].flatten()] = got.flatten(2)
                values[block] = whole.unflatten(-1, (P // TILE, 2, TILE * D))
                if which == 0:
                    total = torch.where(tok < hi, got, torch.zeros((), dtype=torch.float64, device=DEV)).sum(2).abs().amax(-1) * 512.0
                    sh = torch.ceil(torch.log2(total.clamp(min=1.0) / 127.0)).clamp(min=0)
                    sh = torch.where((sh > 0) & (127.0 * _power(sh - 1) >= total), sh - 1, sh)
                    sh = torch.where(127.0 * _power(sh) < total, sh + 1, sh)
                    scales[block] = _power(sh + e - 9.0) / (off + count)[:, None]
        return dict(pages=values, exps=None, means=None, mean_scales=scales)
    if work(c)["flops"] > 6e11 or c["topk"] and s["row_seq"].numel() * H > 2000:
        return None                                                      # too long in a loop over rows and heads
    T, G, scale = s["q"].shape[0], c["q_heads"] // H, 1.0 / math.sqrt(D)
    out = torch.empty(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device=DEV)
    lens, news = _lens(c), _news(c)
    r0 = 0
    for b in range(c["batch"]):
        rows = [(r0 + i, lens[b] + i) for i in range(news[b])]
        for h in range(H):
            if c["topk"]:
                groups = [([r], s["sel"][r, h][s["sel"][r, h] >= 0].long()) for r, _ in rows]
            else:
                pages = torch.arange(-(-(lens[b] + news[b]) // P), device=DEV)
                groups = [([r for r, _ in rows[i:i + 512]], pages) for i in range(0, len(rows), 512)]
            for rs, pages in groups:
                blocks = s["table"][b, pages].long()
                ex = s["exps"][blocks, h].double().repeat_interleave(P, 0)
                k = _value(_page(s["pages"], blocks, h, 0), ex[:, :1])
                v = _value(_page(s["pages"], blocks, h, 1), ex[:, 1:])
                at = (pages[:, None] * P + torch.arange(P, device=DEV)).flatten()
                pos = s["row_pos"][rs[0]:rs[-1] + 1].long()
                x = s["q"][rs[0]:rs[-1] + 1, h * G:(h + 1) * G].double().flatten(0, 1) @ k.T * scale
                x = torch.where((at[None, :] <= pos[:, None]).repeat_interleave(G, 0), x, torch.full_like(x, -math.inf))
                total = torch.logsumexp(x, -1)
                out[rs[0]:rs[-1] + 1, h * G:(h + 1) * G] = (torch.exp(x - total[:, None]) @ v).unflatten(0, (len(rs), G))
                lse[rs[0]:rs[-1] + 1, h * G:(h + 1) * G] = total.unflatten(0, (len(rs), G))
        r0 += news[b]
    return dict(out=out, lse=lse)
