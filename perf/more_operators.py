"""Performance cases of the operators of the 4-bit paged cache and of the rotation before it, with their plain forms.

A case is a dict of plain values.  `op` names the operator:

  rotate  kvd_norm_rotate: the rows' query and key heads, normed and turned by their positions
  append  kvd_q4_append: the rows' keys and values into the pages, in 4 bits with a scale for each 32 elements
  read    kvd_q4_read: the rows' keys and values back out of the pages
  attn    kvd_q4_attn: attention of the rows over what they see of their pages

Sizes: `batch` sequences that hold `context` tokens each before the step (with `ragged` the later ones are shorter, down
to a sixteenth) and get `new` tokens in it (with `ragged` the earlier ones fewer), pages of `page` tokens of `kv_heads`
heads of 128 elements, `q_heads` query heads.

`rotate`: the first `rot` elements of a head in pairs (neighbours if `near`, else half of them apart), of `axes` positions,
`norm` or none.  `attn`: logits capped at `cap` (0: not), `slopes` of a bias by distance, a `window` of the last tokens,
documents of `docs` tokens that do not see each other, a `prefix` that every row sees whole (0: none).
"""
import math

import torch

own = False

DEV = "cuda"
D = 128
TILE = 16                        # tokens of a tile of a page
BLOCK = 32                       # elements of a scale
TILE_BYTES = 2176                # of a head's tile: codes of keys, codes of values, scales of keys, scales of values
K0, V0, KS0, VS0 = 0, 1024, 2048, 2112
EXP_MIN, EXP_MAX, BIAS = -96, 125, 127


def _case(name, op, **kw):
    c = dict(name=name, op=op, batch=1, context=0, new=1, ragged=False, page=16, q_heads=32, kv_heads=8, dtype="bf16", rot=D,
             near=False, axes=1, norm=True, cap=0.0, slopes=False, window=0, docs=0, prefix=0)
    c.update(kw)
    return c


def listed():
    return [
        # a decode step of an ordinary batch: launch latency counts
        _case("rotate_step", "rotate", batch=64, context=8000, ragged=True),
        # the prompts of eight requests at once, behind far positions
        _case("rotate_prompts", "rotate", batch=8, context=120000, new=4096),
        # images and text: time, height and width turn a part of the pairs each, an odd number of rows
        _case("rotate_axes", "rotate", dtype="f16", q_heads=28, kv_heads=4, batch=5, context=100, new=2047, near=True, axes=3),
        # one token for each request into pages that are partly filled
        _case("append_step", "append", batch=64, context=1000, ragged=True),
        # the prompts of eight requests at once, nothing cached before
        _case("append_prompts", "append", batch=8, new=4096),
        # the next pieces of long prompts, seven query heads a KV head, large pages that begin and end inside a piece
        _case("append_pieces_page64", "append", dtype="f16", q_heads=28, kv_heads=4, batch=24, context=5000, new=777, ragged=True,
              page=64),
        # a short piece of two requests, to be looked at by the caller
        _case("read_short", "read", batch=2, context=333, new=150),
        # whole contexts back in 16 bits, to be moved or written anew
        _case("read_contexts", "read", dtype="f16", batch=8, new=4096, ragged=True, page=32),
        # interactive chat: few short contexts, launch latency counts
        _case("attn_step_1k", "attn", batch=4, context=1000, ragged=True),
        # the serving batch of ordinary contexts, bound by the memory
        _case("attn_step_32k", "attn", batch=16, context=32767),
        # contexts of very different lengths, drafted tokens, large pages, capped scores that fall with the distance
        _case("attn_drafts_capped", "attn", dtype="f16", q_heads=28, kv_heads=4, batch=24, context=40000, new=3, ragged=True, page=32,
              cap=50.0, slopes=True),
        # pieces of prompts behind what was read before, many documents in each: bound by the matrix cores
        _case("attn_pieces_docs", "attn", batch=2, context=6144, new=2048, docs=5000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the ranges above: 1 to 512 sequences of up to a million tokens, steps of one token to 65536."""
    while True:
        c = _draw(rng)
        w, held = work(c), sum(-(-n // c["page"]) for n in _ends(c)) * c["page"] * c["kv_heads"] * 2 * D
        # the plain form's scores are the largest thing it makes
        scores = c["batch"] * max(_news(c)) * c["q_heads"] * max(_ends(c))
        gathered = max(_ends(c)) * c["batch"] * c["kv_heads"] * D if c["op"] == "attn" else 0
        if c["op"] != "rotate" and held > 2 << 30 or gathered > 1 << 29:
            continue
        if w["flops"] <= 1.4e11 and w["bytes"] <= 6.7e8 and (c["op"] != "attn" or scores <= 1.1e9) and sum(_news(c)) <= 65536:
            return c


def _draw(rng):
    op = rng.choice(["rotate", "append", "read", "attn", "attn", "attn"])
    kv_heads = rng.choice([1, 2, 4, 8])
    q_heads = kv_heads * rng.choice([1, 2, 4, 4, 5, 7, 8])
    page = rng.choice([16, 16, 16, 32, 48, 64, 128])
    batch = _log(rng, 1, 64 if op == "attn" else 512)
    step = rng.random() < 0.6
    new = 1 if step else _log(rng, 2, 8) if rng.random() < 0.4 else _log(rng, 9, 4096)
    context = _log(rng, 1 if rng.random() < 0.3 else 256, 1000000 if batch * kv_heads <= 4 else 131072)
    if new > 8 and rng.random() < 0.4:
        context = 0
    kw = {}
    if op == "rotate":
        kw = dict(rot=rng.choice([D, D, 96, 64, 32]), near=rng.random() < 0.4, axes=rng.choice([1, 1, 3]), norm=rng.random() < 0.7)
    if op == "attn":
        kw = dict(cap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.3)
        mask = rng.choice(["", "", "window", "docs", "prefix"])
        if mask:
            kw[mask] = _log(rng, 64, 16384)
    return _case("", op, batch=batch, context=context, new=new, ragged=rng.random() < 0.6, page=page, q_heads=q_heads,
                 kv_heads=kv_heads, dtype=rng.choice(["f16", "bf16"]), **kw)


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


def _sees(c, b, pos, end):
    """First and last position that sequence b's row at pos sees."""
    lo = max(0, pos - c["window"] + 1) if c["window"] else 0
    if c["docs"]:
        lo = max(lo, (pos + 17 * b) // c["docs"] * c["docs"] - 17 * b)
    return lo, max(pos, min(c["prefix"], end) - 1)


def _axis_pairs(c):
    """Pairs that turn by each axis."""
    n = c["rot"] // 2
    return [n] if c["axes"] == 1 else [n // 4, n // 2 - n // 8, n - n // 4 - (n // 2 - n // 8)]


def work(c):
    P, H, Hq, lens, news, ends = c["page"], c["kv_heads"], c["q_heads"], _lens(c), _news(c), _ends(c)
    T, entry = sum(news), H * (D + 2 * D // BLOCK)                       # bytes of a token: codes and scales
    if c["op"] == "rotate":
        return {"bytes": T * ((Hq + H) * D * 4 + c["axes"] * 4), "flops": T * (Hq + H) * (D * (3 if c["norm"] else 0) + 3 * c["rot"])}
    if c["op"] == "append":
        runs = sum((e - 1) // P - a // P + 1 for a, e in zip(lens, ends))
        return {"bytes": T * (H * D * 4 + entry) + runs * 16, "flops": 4 * T * H * D}
    if c["op"] == "read":
        return {"bytes": T * (H * D * 4 + entry + 8) + 4 * sum((e - 1) // P - a // P + 1 for a, e in zip(lens, ends)), "flops": 2 * T * H * D}
    pairs = tokens = 0
    for b, (a, n, e) in enumerate(zip(lens, news, ends)):
        sees = [_sees(c, b, a + i, e) for i in range(n)]
        pairs += sum(hi - lo + 1 for lo, hi in sees)
        tokens += max(hi for _, hi in sees) - min(lo for lo, _ in sees) + 1
    return {"bytes": tokens * entry + tokens // P * 4 + T * Hq * (D * 4 + 4), "flops": 4 * pairs * Hq * D}


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


def _rows(c, seed):
    """The step's table, lengths, rows and runs, with the blocks of the pool dealt out at random."""
    P, B = c["page"], c["batch"]
    a, n, e = (torch.tensor(v) for v in (_lens(c), _news(c), _ends(c)))
    T = int(n.sum())
    have = -(-e // P)
    NP, used_blocks = int(have.max()), int(have.sum())
    NB = used_blocks + 5
    cpu = torch.Generator()
    cpu.manual_seed(int(seed) % (1 << 62))
    blocks = torch.randperm(NB, generator=cpu)
    table = torch.full((B, NP), -1)
    table[torch.arange(NP)[None, :] < have[:, None]] = blocks[:used_blocks]
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
    return dict(blocks=NB, n_rows=T, n_runs=len(rseq), table=to(table), kv_len=to(e), row_start=to(start), row_seq=to(seq), row_pos=to(pos),
                runs=to(runs), counts=torch.zeros(5, dtype=torch.int32, device=DEV))


def _pool(NB, H, P, g):
    """Pages as appending leaves them: codes of N(0, 1) elements that a scale near a third of their largest was divided out of."""
    x = (torch.randn((1 << 17, 2), generator=g, device=DEV) * 2.0).clamp_(-6, 6)
    code = _code(x)
    pairs = code[:, 0] | code[:, 1] << 4
    pages = torch.empty((NB, H, P // TILE, TILE_BYTES), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 27) // pages[0].numel())
    for i in range(0, NB, step):
        n = pages[i:i + step]
        n[..., :KS0] = pairs[torch.randint(0, 1 << 17, n.shape[:-1] + (KS0,), generator=g, device=DEV, dtype=torch.int32)]
        n[..., KS0:] = torch.randint(BIAS - 2, BIAS + 1, n.shape[:-1] + (TILE_BYTES - KS0,), generator=g, device=DEV, dtype=torch.uint8)
    return pages


def prepare(case, seed):
    c, g = case, _gen(seed, 0)
    H, Hq, P, T, dt = c["kv_heads"], c["q_heads"], c["page"], sum(_news(c)), _dtype(c)
    s = dict(case=c)
    s.update(_rows(c, seed))
    if c["op"] == "rotate":
        s["q"] = torch.randn((T, Hq, D), generator=g, device=DEV, dtype=dt) * 3.0
        s["k"] = torch.randn((T, H, D), generator=g, device=DEV, dtype=dt) * 2.0
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        n = c["rot"] // 2
        s["inv_freq"] = (500000.0 ** (-torch.arange(n, dtype=torch.float64) / n)).float().to(DEV)
        pos = s["row_pos"]
        # an image's time, height and width: rows of 64 patches, 32 to an image
        s["positions"] = pos if c["axes"] == 1 else torch.stack([pos // 2048, pos // 64 % 32, pos % 64])
        for name in ("q_weight", "k_weight"):
            s[name] = (1.0 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(dt) if c["norm"] else None
        return s
    s["pages"] = _pool(s["blocks"], H, P, g)
    if c["op"] == "append":
        # keys as they come out of a projection: N(0, 1) with a few channels that are several times as large
        s["k_new"] = torch.randn((T, H, D), generator=g, device=DEV, dtype=dt)
        s["k_new"][..., 5::41] *= 6.0
        s["v_new"] = torch.randn((T, H, D), generator=g, device=DEV, dtype=dt)
        return s
    if c["op"] == "read":
        s["k"], s["v"] = (torch.empty((T, H, D), dtype=dt, device=DEV) for _ in range(2))
        return s
    s["q"] = torch.randn((T, Hq, D), generator=g, device=DEV).to(dt)
    s["out"] = torch.empty((T, Hq, D), dtype=dt, device=DEV)
    s["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=DEV)
    s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, Hq + 1) / Hq)).float().to(DEV) if c["slopes"] else None
    seq, pos = s["row_seq"], s["row_pos"]
    s["row_from"] = ((pos + 17 * seq) // c["docs"] * c["docs"] - 17 * seq).clamp(min=0).to(torch.int32) if c["docs"] else None
    s["prefix_len"] = torch.full((c["batch"],), c["prefix"], dtype=torch.int32, device=DEV) if c["prefix"] else None
    return s


# ---- one pass ------------------------------------------------------------------------------------

def _handle(s):
    """The framework's rows and cache (or rotation) over the state's buffers, kept with them."""
    if "handle" not in s:
        from paper_2605_18071_amd import kvd
        c = s["case"]
        if c["op"] == "rotate":
            s["handle"] = kvd.Rotary(s["inv_freq"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], kv_dtype=_dtype(c), interleaved=c["near"],
                                     axis_pairs=_axis_pairs(c), q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6)
        else:
            rows = kvd.Q8Rows(s["table"], page_size=c["page"], n_blocks=s["blocks"], n_rows=s["n_rows"], max_runs=s["n_runs"],
                              **{n: s[n] for n in ("kv_len", "row_start", "row_seq", "row_pos", "runs", "counts")})
            cache = kvd.Q4Cache(n_blocks=s["blocks"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], page_size=c["page"],
                                kv_dtype=_dtype(c), pages=s["pages"])
            s["handle"] = rows, cache, cache.workspace(rows) if c["op"] == "attn" else None
    return s["handle"]


def run(s):
    c = s["case"]
    if own:
        if c["op"] == "rotate":
            _handle(s).apply(s["positions"], s["q"], s["k"], q_out=s["q_out"], k_out=s["k_out"])
            return dict(q=s["q_out"], k=s["k_out"])
        rows, cache, ws = _handle(s)
        if c["op"] == "append":
            cache.append(rows, s["k_new"], s["v_new"])
            return dict(pages=s["pages"])
        if c["op"] == "read":
            cache.read(rows, s["k"], s["v"])
            return dict(k=s["k"], v=s["v"])
        cache.attend(rows, s["q"], s["out"], ws, lse=s["lse"], softcap=c["cap"], window=c["window"], slopes=s["slopes"],
                     row_from=s["row_from"], prefix_len=s["prefix_len"])
        return dict(out=s["out"], lse=s["lse"])
    return {"rotate": _rotate, "append": _append, "read": _read, "attn": _attend}[c["op"]](s)


# ---- the plain forms -----------------------------------------------------------------------------

def _rotate(s):
    c = s["case"]
    n = c["rot"] // 2
    axis = torch.repeat_interleave(torch.arange(c["axes"], device=DEV), torch.tensor(_axis_pairs(c), device=DEV), output_size=n)
    pos = s["positions"].reshape(c["axes"], -1).double()
    angle = pos[axis].T * s["inv_freq"].double()                         # [T][n], in 64 bits: positions are far
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    for name in ("q", "k"):
        x, w = s[name].float(), s[name + "_weight"]
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        turned, rest = x[..., : 2 * n], x[..., 2 * n:]
        a, b = (turned[..., 0::2], turned[..., 1::2]) if c["near"] else (turned[..., :n], turned[..., n:])
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1 if c["near"] else -2).flatten(-2)
        s[name + "_out"].copy_(torch.cat([y, rest], -1))
    return dict(q=s["q_out"], k=s["k_out"])


def _two(e):
    """2^e of whole numbers, in 64 bits: the bits themselves, which no rounding of a power function can touch."""
    return ((e.to(torch.int64).clamp(-1022, 1023) + 1023) << 52).view(torch.float64)


def _code(y):
    """4-bit codes of elements in -6..6, to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, halves to the even code."""
    a = y.abs()
    code = torch.where(a < 2, (2 * a).round(), torch.where(a < 4, a.round() + 2, (a / 2).round() + 4))
    return code.to(torch.uint8) | torch.signbit(y).to(torch.uint8) << 3


def _quantise(x):
    """Codes [..., D] and scales' bytes [..., D / BLOCK] of elements."""
    x = x.nan_to_num(0.0, math.inf, -math.inf).unflatten(-1, (-1, BLOCK))
    amax = torch.where(x.isinf(), torch.zeros((), device=DEV), x).abs().amax(-1)
    m, e = torch.frexp(amax)                                             # m in [1/2, 1): 7 is 7/8 of 2^3
    e = torch.where(amax > 0, e - 3 + (m > 0.875).to(e.dtype), torch.full_like(e, EXP_MIN)).clamp(EXP_MIN, EXP_MAX)
    y = (x * _two(-e)[..., None].float()).clamp(-6, 6)
    return _code(y).flatten(-2), (e + BIAS).to(torch.uint8)


def _split(b, dim):
    """Two codes from each byte, the lower bits first, along a new last dimension."""
    return torch.stack([b & 15, b >> 4], dim)


def _natural(pages):
    """Tiles [..., tiles, TILE_BYTES] as codes [..., tokens, D] of keys and of values, and scales [..., tokens, D / BLOCK] of both."""
    lead = list(range(pages.dim() - 1))
    n = len(lead)
    k = _split(pages[..., K0:V0].unflatten(-1, (TILE, D // 2)), -1).flatten(-2)
    v = _split(pages[..., V0:KS0].unflatten(-1, (4, 16, 2, 8)), -1)      # 32 dims, dim of 16, 16 dims, 2 tokens, token
    v = v.permute(lead + [n + 3, n + 4, n, n + 2, n + 1]).flatten(-3).flatten(-3, -2)
    ks = pages[..., KS0:VS0].unflatten(-1, (4, 4, 4)).permute(lead + [n + 2, n + 1, n]).flatten(-3, -2)
    vs = pages[..., VS0:].unflatten(-1, (4, TILE)).transpose(-1, -2)
    return [x.flatten(-3, -2) for x in (k, v, ks, vs)]


def _tiled(k, v, ks, vs):
    """The other way."""
    k, v, ks, vs = (x.unflatten(-2, (-1, TILE)) for x in (k, v, ks, vs))
    lead = list(range(k.dim() - 2))
    n = len(lead)
    k = (k[..., 0::2] | k[..., 1::2] << 4).flatten(-2)
    v = v.unflatten(-2, (8, 2)).unflatten(-1, (4, 2, 16))                # 2 tokens, token, 32 dims, 16 dims, dim
    v = v.permute(lead + [n + 2, n + 4, n + 3, n, n + 1])
    v = (v[..., 0] | v[..., 1] << 4).flatten(-4)
    ks = ks.unflatten(-2, (4, 4)).permute(lead + [n + 2, n + 1, n]).flatten(-3)
    return torch.cat([k, v, ks, vs.transpose(-1, -2).flatten(-2)], -1)


_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _value(code, scale):
    """Numbers of codes [..., D] and scales [..., D / BLOCK]."""
    t = torch.tensor(_VALUES, device=DEV)
    x = t[code.int()].unflatten(-1, (-1, BLOCK))
    return (x * _two(scale.int() - BIAS).float()[..., None]).flatten(-2)


def _append(s):
    P, runs = s["case"]["page"], s["runs"].long()
    block, row, off, count = (runs[:, i] for i in range(4))
    old = _natural(s["pages"][block])                                    # [runs][H][P][...] each
    t = torch.arange(P, device=DEV)[None, :]
    fresh = ((t >= off[:, None]) & (t < (off + count)[:, None]))[:, None, :, None]
    begins = (off == 0)[:, None, None, None]
    src = (row[:, None] + t - off[:, None]).clamp(0, s["k_new"].shape[0] - 1)
    (k, ks), (v, vs) = (_quantise(x.float()) for x in (s["k_new"], s["v_new"]))
    none = torch.zeros((), dtype=torch.uint8, device=DEV)
    empty = torch.full((), EXP_MIN + BIAS, dtype=torch.uint8, device=DEV)
    new = [torch.where(fresh, x[src].transpose(1, 2), torch.where(begins, z, o))
           for x, o, z in zip((k, v, ks, vs), old, (none, none, empty, empty))]
    s["pages"][block] = _tiled(*new)
    return dict(pages=s["pages"])                                        # codes and scales, byte for byte


def _read(s):
    c = s["case"]
    P, pos = c["page"], s["row_pos"].long()
    block = s["table"][s["row_seq"].long(), pos // P].long()[:, None]
    tile, t = (pos % P // TILE)[:, None], (pos % TILE)[:, None]
    h = torch.arange(c["kv_heads"], device=DEV)[None, :]
    pages, at = s["pages"], (block, h, tile)
    k = _split(pages[..., K0:V0].unflatten(-1, (TILE, D // 2))[at + (t,)], -1).flatten(-2)
    v = pages[..., V0:KS0].unflatten(-1, (4, 16, 2, 8))[at + (slice(None), slice(None), slice(None), t // 2)]
    v = (v >> (t % 2 * 4)[..., None, None, None].to(torch.uint8) & 15).transpose(-1, -2).flatten(-3)
    ks = pages[..., KS0:VS0].unflatten(-1, (4, 4, 4))[at + (slice(None), t % 4, t // 4)]
    vs = pages[..., VS0:].unflatten(-1, (4, TILE))[at + (slice(None), t)]
    s["k"].copy_(_value(k, ks))
    s["v"].copy_(_value(v, vs))
    return dict(k=s["k"], v=s["v"])


def _attend(s):
    c, q = s["case"], s["q"].float()
    P, H = c["page"], c["kv_heads"]
    T, G, scale = q.shape[0], c["q_heads"] // H, 1.0 / math.sqrt(D)
    n = max(_news(c))                                                    # the rows of a sequence together, as many as the longest has
    lens, starts = s["kv_len"].long(), s["row_start"].long()
    count = starts[1:] - starts[:-1]
    i = torch.arange(n, device=DEV)
    row = (starts[:-1, None] + i).clamp(max=T - 1)                       # [B][n]
    at = torch.arange(s["table"].shape[1] * P, device=DEV)
    pos = lens[:, None] - count[:, None] + i                             # [B][n] positions
    last, first = pos, torch.zeros_like(pos)
    if s["prefix_len"] is not None:
        last = torch.maximum(last, torch.minimum(s["prefix_len"].long(), lens)[:, None] - 1)
    if c["window"]:
        first = (pos - c["window"] + 1).clamp(min=0)
    if s["row_from"] is not None:
        first = torch.maximum(first, s["row_from"].long()[row])
    seen = (at >= first[..., None]) & (at <= last[..., None])            # [B][n][tokens]
    seen = seen[:, None, :, None, :].expand(-1, H, n, G, -1).flatten(2, 3)
    query = q[row].unflatten(2, (H, G)).transpose(1, 2).flatten(2, 3)    # [B][H][n G][D]
    h = torch.arange(H, device=DEV)
    k, v, ks, vs = _natural(s["pages"][s["table"].clamp(min=0).long()[:, None, :], h[None, :, None]])
    k, v = _value(k, ks).flatten(2, 3), _value(v, vs).flatten(2, 3)
    logits = torch.matmul(query, k.transpose(-1, -2).contiguous()) * scale
    del k
    if c["cap"]:
        logits = logits.div_(c["cap"]).tanh_().mul_(c["cap"])
    if s["slopes"] is not None:
        far = (pos[:, None, :, None, None] - at).abs().float()           # [B][1][n][1][tokens]
        logits.sub_((s["slopes"].view(H, 1, G, 1) * far).flatten(2, 3))
    logits.masked_fill_(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = (logits - top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + top)[..., 0]
    out = torch.matmul(p, v) / total
    seq, nth = s["row_seq"].long(), s["row_pos"].long()
    nth = nth - (lens - count)[seq]
    s["out"].copy_(out.unflatten(2, (n, G))[seq, :, nth].flatten(1, 2))
    s["lse"].copy_(lse.unflatten(2, (n, G))[seq, :, nth].flatten(1, 2))
    return dict(out=s["out"], lse=s["lse"])


# ---- the definitions, in 64 bits -----------------------------------------------------------------

def _number(code):
    """The number that a 4-bit code stands for: a sign, two bits of exponent, one of mantissa."""
    code = code.to(torch.int64)
    ex, man = code >> 1 & 3, (code & 1).double()
    mag = torch.where(ex == 0, 0.5 * man, torch.ldexp(1.0 + 0.5 * man, (ex - 1).double()))
    return torch.where(code >= 8, -mag, mag)


def _held(pages, block, h, t, which):
    """Values of the tokens t of the pages' blocks: [..., D] of keys (0) or values (1), block, h and t alike in shape."""
    d = torch.arange(D, device=DEV)
    block, h, t = block[..., None], h[..., None], t[..., None]
    i = t % TILE
    if which == 0:
        byte, high, scale = i * 64 + d // 2, d % 2, 2048 + d // 32 * 16 + i % 4 * 4 + i // 4
    else:
        byte, high, scale = 1024 + d // 32 * 256 + d % 16 * 16 + d // 16 % 2 * 8 + i // 2, i % 2, 2112 + d // 32 * 16 + i
    code = pages[block, h, t // TILE, byte].long() >> (4 * high) & 15
    return torch.ldexp(_number(code), pages[block, h, t // TILE, scale].double() - 127.0)


def exact(case, seed):
    c = case
    if c["op"] == "append":
        return None                                                      # whole numbers
    s = prepare(case, seed)
    P, H, G = c["page"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    if c["op"] == "rotate":
        n, pairs = c["rot"] // 2, _axis_pairs(c)
        pos = s["positions"].reshape(c["axes"], -1).double()
        turn = torch.cat([pos[a][:, None] * s["inv_freq"].double()[sum(pairs[:a]):sum(pairs[: a + 1])] for a in range(c["axes"])], 1)
        at = torch.arange(n, device=DEV)
        one, two = (2 * at, 2 * at + 1) if c["near"] else (at, at + n)
        got = {}
        for name in ("q", "k"):
            x = s[name].double()
            if s[name + "_weight"] is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + 1e-6) * s[name + "_weight"].double()
            z = torch.complex(x[..., one], x[..., two]) * torch.polar(torch.ones_like(turn), turn)[:, None]
            x[..., one], x[..., two] = z.real, z.imag
            got[name] = x
        return got
    if c["op"] == "read":
        pos, h = s["row_pos"].long()[:, None], torch.arange(H, device=DEV)[None, :]
        block = s["table"].long()[s["row_seq"].long()[:, None], pos // P]
        got = [[], []]
        for i in range(0, pos.shape[0], 4096):
            b, p = block[i:i + 4096], pos[i:i + 4096] % P
            b, p, hh = b.expand(-1, H), p.expand(-1, H), h.expand(b.shape[0], -1)
            for which in (0, 1):
                got[which].append(_held(s["pages"], b, hh, p, which))
        return dict(k=torch.cat(got[0]), v=torch.cat(got[1]))
    if work(c)["flops"] > 6e11:
        return None                                                      # too long in a loop over rows and heads
    out = torch.empty(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device=DEV)
    lens, news = _lens(c), _news(c)
    r0 = 0
    for b in range(c["batch"]):
        end = lens[b] + news[b]
        at = torch.arange(end, device=DEV)
        block = s["table"][b].long()[at // P]
        for h in range(H):
            hh = torch.full_like(at, h)
            k, v = (_held(s["pages"], block, hh, at % P, which) for which in (0, 1))
            for i in range(0, news[b], 512):
                n = min(512, news[b] - i)
                rs = slice(r0 + i, r0 + i + n)
                sees = torch.tensor([_sees(c, b, lens[b] + i + y, end) for y in range(n)], device=DEV)
                x = s["q"][rs, h * G:(h + 1) * G].double().flatten(0, 1) @ k.T / math.sqrt(D)
                x = x.unflatten(0, (n, G))
                if c["cap"]:
                    x = torch.tanh(x / c["cap"]) * c["cap"]
                if c["slopes"]:
                    far = (at[None, :] - (lens[b] + i + torch.arange(n, device=DEV))[:, None]).abs().double()
                    x = x - s["slopes"][h * G:(h + 1) * G].double()[None, :, None] * far[:, None, :]
                hidden = (at < sees[:, :1]) | (at > sees[:, 1:])
                x = torch.where(hidden[:, None, :], torch.full_like(x, -math.inf), x)
                total = torch.logsumexp(x, -1)
                out[rs, h * G:(h + 1) * G] = torch.exp(x - total[..., None]) @ v
                lse[rs, h * G:(h + 1) * G] = total
        r0 += news[b]
    return dict(out=out, lse=lse)
