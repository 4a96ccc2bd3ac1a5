"""More calls of a program that serves from compressed caches, and what they compute in elementary terms.

fp4     the cache in 4 bits: rows of 64 bytes of E2M1 codes with an E8M0 scale byte per 32 channels; new rows go in (append),
        a bf16 cache becomes one (store), rows come back (read), new tokens attend to it
rotate  what lies between a layer's projections and its cache: the norm of every query and key head, the rotation by position, the
        keys before it (which are scored) and after it (which are cached), and in one call with the append for single tokens
pages   room for new tokens, contexts that share pages and write to their own copies, reordered beams, pages given back,
        pools pushed together

Head shapes and lengths are those of the synthetic workloads (Llama-3.1-8B, Qwen-2.5-7B and Qwen-2.5-32B shapes, contexts of 4 K to
128 K tokens kept to 20 to 60 %), odd ones among them.  A cache: K and V pages seen as [page, layer, slot, head, channel],
tables[request][i] the page of logical page i, counts and seen [request, layer, head], mass, positions and the scales of 4-bit rows
[page, layer, head, slot]; refs[page]: how many table entries name it.
"""
import math
import random

import torch

own = False

D = 128
GAIN = 20.0                     # outlier channels of the keys
TINY, LARGEST = 2, 252          # scale bytes that are written: every value of theirs is a normal bf16 number


def _case(name, op, **kw):
    c = {"name": name, "op": op, "requests": 1, "layers": 1, "kv_heads": 8, "group": 4, "n_lo": 0, "n": 0, "new": 1,
         "ragged_new": False, "page": 16, "layout": "head", "ragged_heads": False, "accumulate": False, "cap": 0.0,
         "norm": True, "interleaved": False, "rotary": 128, "far": 0, "samples": 1, "own_all": False, "finished": 0,
         "free": 64, "shape_seed": 1}
    c.update(kw)
    return c


def listed():
    return [
        # the first steps behind a short context: one layer, one request, all latency
        _case("fp4_attention_short", "attention", n_lo=307, n=307),
        # one long context at 20 %, Qwen-2.5-7B heads: few heads, so the length has to be split
        _case("fp4_attention_one_128k", "attention", kv_heads=4, group=7, n_lo=26215, n=26215, page=64, accumulate=True),
        # drafted tokens to verify, some requests with fewer of them and some with none; pages of an odd size, heads side by side
        _case("fp4_attention_drafts", "attention", requests=12, new=5, ragged_new=True, n_lo=900, n=9831, page=24,
              layout="token", accumulate=True),
        # the largest: many long contexts, capped scores, eight query heads a kv head
        _case("fp4_attention_many_long", "attention", requests=48, group=8, n_lo=8192, n=32000, page=32, cap=30.0),
        # one token a request into one layer's pages
        _case("fp4_append_token", "append", requests=32, n_lo=500, n=9000),
        # the retained rows of a whole model's context, in pages of 16 bits so far, become a cache in 4 bits
        _case("fp4_store_model", "store", layers=32, n_lo=9831, n=9831),
        # a layer's queries and keys of a prompt: keys to score, keys to cache
        _case("rotate_prompt", "rotate", new=32768),
        # a step of 32 requests: queries rotated, keys rotated into the cache, far into long contexts, without norms
        _case("rotate_append_token", "rotate_append", requests=32, n_lo=300, n=2000, far=100000, norm=False),
        # a step's pages for 64 requests, a few of which need one
        _case("pages_step", "reserve", requests=64, n_lo=500, n=9000),
        # eight samples of each of 16 prompts go apart: the page that they all write to next is copied, all layers
        _case("pages_samples", "reserve", requests=128, samples=8, layers=32, n_lo=300, n=2000, free=512),
        # beams of 16 contexts are reordered
        _case("pages_beams", "fork", requests=64, samples=4, n_lo=4000, n=32000),
        # a third of the contexts has ended: their pages go back and the others' are pushed together
        _case("pages_compact", "compact", requests=48, layers=4, n_lo=900, n=9831, finished=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "append", "store", "rotate", "rotate_append", "reserve", "reserve",
                     "fork", "compact"])
    c = _case("", op, kv_heads=rng.choice([1, 2, 4, 8, 8]), page=rng.choice([16, 16, 32, 64, 128, 24, 7]),
              layout=rng.choice(["token", "head"]), requests=_log(rng, 1, 64), shape_seed=rng.randint(1, 10**6))
    most = {"attention": 48 * 8 * 16000, "append": 100000, "store": 32 * 8 * 9831, "rotate": 8 * 32768,
            "rotate_append": 100000, "reserve": 32 * 8 * 9000, "fork": 1 << 30, "compact": 48 * 8 * 16000}[op]    # rows
    c["n"] = _log(rng, 64, 65536)
    c["group"] = rng.choice([1, 2, 4, 4, 5, 7, 8])
    if op in ("append", "rotate_append"):
        c["new"] = rng.choice([1, 1, 1, 2, 5, _log(rng, 8, 600)])
        c["n"] = min(c["n"], 3000)
    if op == "attention":
        c["new"] = rng.choice([1, 1, 1, 1, 2, 4, 5])
        c["accumulate"] = rng.random() < 0.5
        c["cap"] = rng.choice([0.0, 0.0, 0.0, 30.0, 50.0])
    if op == "rotate":
        c["new"] = _log(rng, 1, 32768)
        c["n"] = 64
    if op in ("rotate", "rotate_append"):
        c["requests"] = _log(rng, 1, 32)
        c["norm"] = rng.random() < 0.7
        c["interleaved"] = rng.random() < 0.3
        c["rotary"] = rng.choice([128, 128, 128, 64, 32, 96])
        c["far"] = rng.choice([0, 1000, 100000])
    if op in ("reserve", "fork"):
        c["samples"] = rng.choice([1, 1, 2, 4, 8])
        c["new"] = rng.choice([1, 1, 5, 300])
        c["own_all"] = op == "reserve" and c["samples"] > 1 and rng.random() < 0.3
        c["n"] = min(c["n"], 2000 if c["own_all"] else 32000)
        c["free"] = rng.choice([64, 600])
    if op == "compact":
        c["n"] = min(c["n"], 20000)
    c["ragged_new"] = c["new"] > 1 and rng.random() < 0.5
    c["ragged_heads"] = op in ("attention", "store", "reserve", "compact") and rng.random() < 0.4
    c["n_lo"] = c["n"] if rng.random() < 0.3 else max(1, c["n"] // rng.choice([2, 4, 8]))
    per = c["kv_heads"] * (c["new"] if op in ("append", "rotate", "rotate_append") else c["n"])
    while c["requests"] > 1 and (c["requests"] * per > most or c["requests"] * c["kv_heads"] * c["n"] > 48 * 8 * 16000):
        c["requests"] -= 1
    layers = min(32, most / (c["requests"] * per), 48 * 8 * 16000 / (c["requests"] * c["kv_heads"] * c["n"]))
    c["layers"] = _log(rng, 1, layers) if layers > 1 and rng.random() < 0.4 else 1
    if op == "compact":
        c["finished"] = rng.randint(0, c["requests"] // 2)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------- shapes


def _lengths(case):
    """Tokens of every request; samples of one prompt have it in common."""
    r = random.Random(case["shape_seed"])
    got = [r.randint(case["n_lo"], case["n"]) for _ in range(case["requests"])]
    return [got[b - b % case["samples"]] for b in range(case["requests"])]


def _news(case):
    r = random.Random(case["shape_seed"] + 1)
    if not case["ragged_new"]:
        return [case["new"]] * case["requests"]
    return [r.randint(0, case["new"]) for _ in range(case["requests"])]


def _head_counts(case):
    """Cached tokens [request][layer][head] before the call."""
    r = random.Random(case["shape_seed"] + 2)
    L, H = case["layers"], case["kv_heads"]
    got = []
    for b, n in enumerate(_lengths(case)):
        if b % case["samples"]:
            got.append(got[-1])
        elif case["ragged_heads"]:      # heads of a layer that share H * n
            rows = []
            for _ in range(L):
                row = [n] * H
                for h in range(H // 2):
                    move = r.randint(0, n)
                    row[h] -= move
                    row[H - 1 - h] += move
                rows.append(row)
            got.append(rows)
        else:
            got.append([[n] * H for _ in range(L)])
    return got


def _written(case):
    """Logical pages of every request: the first that its new tokens go to (all that hold tokens: own_all), how many hold
    tokens, and how many there have to be."""
    page, got = case["page"], []
    for rows, new in zip(_head_counts(case), _news(case)):
        lo, top = min(min(r) for r in rows), max(max(r) for r in rows)
        holds = -(-top // page)
        first = 0 if case["own_all"] else lo // page if new > 0 else holds
        got.append((first, holds, -(-(top + new) // page)))
    return got


def _copies(case):
    """Pages that requests which share them get copies of.  Samples of a prompt write to the same ones; where all of them do, the last keeps
    what they had."""
    written, samples, got = _written(case), case["samples"], 0
    for b in range(0, case["requests"], samples):
        some = [hold - first for first, hold, _ in written[b:b + samples]]
        writers = sum(x > 0 for x in some)
        if len(some) > 1:
            got += max(some) * (writers if writers < len(some) else writers - 1)
    return got


def _news_room(case):
    return case["new"] if case["op"] in ("append", "rotate_append", "reserve", "fork", "attention") else 0


# ---------------------------------------------------------------------------------------- 4 bits, plain


def _encode(x):
    """bf16 [..., 128] -> codes uint8 [..., 64] (channel 2 i in the low half of byte i), scales uint8 [..., 4]."""
    g = x.reshape(*x.shape[:-1], 4, 32)
    top = (g.contiguous().view(torch.int16).to(torch.int32) & 0x7fff).amax(-1)
    s = ((top >> 7) + ((top & 127) >= 96).to(torch.int32) - 2).clamp(TINY, LARGEST)
    bad = top >= 0x7f80
    size = (g.float() * torch.ldexp(torch.ones_like(s, dtype=torch.float32), 127 - s).unsqueeze(-1)).abs()
    code = torch.zeros(g.shape, dtype=torch.uint8, device=x.device)
    for border, above in ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)):
        code += (size > border) if above else (size >= border)          # ties to the even code
    code |= (g.float() < 0).to(torch.uint8) << 3
    code = torch.where(bad.unsqueeze(-1), 0, code).reshape(*x.shape[:-1], 64, 2)
    s = torch.where(bad, 255, s)
    return code[..., 0] | code[..., 1] << 4, s.to(torch.uint8)


def _decode(codes, scales):
    """-> fp32 [..., 128]"""
    lut = torch.tensor([0., .5, 1., 1.5, 2., 3., 4., 6., -0., -.5, -1., -1.5, -2., -3., -4., -6.], device=codes.device)
    at = torch.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], 4, 32)
    s = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.to(torch.int32) - 127)
    s = torch.where(scales == 255, math.nan, s)
    return (lut[at.long()] * s.unsqueeze(-1)).reshape(*codes.shape[:-1], D)


# ---------------------------------------------------------------------------------------- inputs


def _rows(shape, g, dev, outliers):
    t = torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16)
    if outliers:
        t[..., torch.randperm(D, generator=g, device=dev)[:4]] *= GAIN
    return t


def _pool(pages, L, H, page, layout, g, dev):
    """K and V pages as [page, layer, slot, head, channel] views of how they lie in memory."""
    shape = (pages, L, page, H, D) if layout == "token" else (pages, L, H, page, D)
    got = [_rows(shape, g, dev, which == 0) for which in range(2)]
    return got if layout == "token" else [t.permute(0, 1, 3, 2, 4) for t in got]


def _pool4(pages, L, H, page, layout, g, dev, fill):
    """The same in 4 bits, and the scales as [page, layer, head, slot, group]."""
    shape = (pages, L, page, H) if layout == "token" else (pages, L, H, page)
    got = []
    for which in range(2):
        codes = torch.zeros(*shape, 64, dtype=torch.uint8, device=dev)
        scales = torch.zeros(pages, L, H, page, 4, dtype=torch.uint8, device=dev)
        at_once = max(1, (1 << 26) // (L * H * page * D))
        for p in range(0, pages, at_once) if fill else ():
            q = min(p + at_once, pages)
            codes[p:q], s = _encode(_rows((q - p, *shape[1:], D), g, dev, which == 0))
            scales[p:q] = s.transpose(2, 3) if layout == "token" else s
        got += [codes if layout == "token" else codes.permute(0, 1, 3, 2, 4), scales]
    return got


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 31)
    op, B, L, H, T, page = (case[k] for k in ("op", "requests", "layers", "kv_heads", "new", "page"))
    s = {"op": op, "case": case}
    lengths, news = _lengths(case), _news(case)
    s["new_tokens"] = torch.tensor(news, dtype=torch.int32, device=dev) if case["ragged_new"] else None
    Hq = H * case["group"]
    if op in ("attention", "rotate", "rotate_append"):
        s["q"] = torch.randn(B, L, T, Hq, D, generator=g, device=dev).mul_(
            0.5 + torch.rand(B, L, 1, Hq, 1, generator=g, device=dev)).to(torch.bfloat16)
    if op in ("append", "rotate", "rotate_append"):
        s["k"] = _rows((B, L, T, H, D), g, dev, True)
        s["v"] = _rows((B, L, T, H, D), g, dev, False)
    if op in ("rotate", "rotate_append"):
        half = case["rotary"] // 2
        s["freqs"] = 500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
        norm = [(0.5 + torch.rand(L, D, generator=g, device=dev)) if case["norm"] else None for _ in range(2)]
        s["q_norm"], s["k_norm"] = norm
    if op == "rotate":
        far = torch.randint(0, case["far"] + 1, (B, 1), generator=g, device=dev)
        s["positions"] = (far + torch.arange(T, device=dev)).to(torch.int32)
        if case["ragged_new"]:          # rows behind a request's tokens stay as they are
            s["q_out"], s["k_out"], s["k_plain"] = (torch.zeros_like(s[n]) for n in ("q", "k", "k"))
    if op != "rotate":
        _prepare_cache(s, case, seed, g, dev, lengths)
    if own:
        from paper_2507_08143_amd import compactor as C
        s["C"] = C
        if op in ("rotate", "rotate_append"):
            s["rotation"] = C.Rotation(s["freqs"], rotary_dim=case["rotary"], interleaved=case["interleaved"],
                                       q_norm=s["q_norm"], k_norm=s["k_norm"], eps=1e-6)
        if op != "rotate":
            state = s["tables"], s["counts"], s["seen"], s["mass"], s["positions"]
            if op in ("attention", "append", "store"):
                s["cache"] = C.Fp4Cache(s["k4"], s["v4"], s["k_scales"], s["v_scales"], *state)
            if op == "store":
                s["source"] = C.Cache(s["k_pages"], s["v_pages"], s["source_tables"], s["source_counts"], s["source_seen"],
                                      s["source_mass"], s["source_positions"])
            if op in ("rotate_append", "reserve", "fork", "compact"):
                s["cache"] = C.Cache(s["k_pages"], s["v_pages"], *state)
    return s


def _prepare_cache(s, case, seed, g, dev, lengths):
    op, B, L, H, page, samples = (case[k] for k in ("op", "requests", "layers", "kv_heads", "page", "samples"))
    counts = torch.tensor(_head_counts(case), dtype=torch.int32)
    most = int(counts.max()) + _news_room(case)
    per = -(-most // page)
    shares = op in ("reserve", "fork")
    own_pages = [-(-int(counts[b].max()) // page) if op in ("reserve", "fork", "compact") else per for b in range(B)]
    names = sum(own_pages[b] for b in range(B) if not shares or b % samples == 0)
    want = 0
    if op == "reserve":
        s["most"] = _copies(case)
        want = s["most"] + sum(need - hold for _, hold, need in _written(case))
    pages = names + want + (case["free"] if shares else 3) + 1            # the last one belongs to somebody else
    order = torch.randperm(pages - 1, generator=g, device=dev).to(torch.int32)
    tables = torch.full((B, per), -1, dtype=torch.int32, device=dev)
    at = 0
    for b in range(B):
        if shares and b % samples:
            tables[b] = tables[b - 1]
        else:
            tables[b, :own_pages[b]] = order[at:at + own_pages[b]]
            at += own_pages[b]
    s["tables"], s["start_tables"] = tables, tables.clone()
    s["state"] = torch.empty(2, B, L, H, dtype=torch.int32, device=dev)
    s["state"][0] = counts.to(dev)
    s["state"][1] = torch.tensor(lengths, device=dev).view(B, 1, 1) * 3 + case["far"]
    s["counts"], s["seen"] = s["state"][0], s["state"][1]
    s["start"] = s["state"].clone()
    s["max_tokens"] = per * page
    s["mass"] = torch.rand(pages, L, H, page, generator=g, device=dev)
    s["positions"] = torch.randint(0, 1 << 20, (pages, L, H, page), generator=g, device=dev, dtype=torch.int32)
    if op in ("attention", "append", "store"):
        s["k4"], s["k_scales"], s["v4"], s["v_scales"] = _pool4(pages, L, H, page, case["layout"], g, dev, op == "attention")
    if op in ("store", "rotate_append", "reserve", "fork", "compact"):
        s["k_pages"], s["v_pages"] = _pool(pages, L, H, page, case["layout"], g, dev)
    if op == "store":       # another pool's pages
        s["source_tables"] = torch.randperm(pages - 1, generator=g, device=dev).to(torch.int32)[:B * per].view(B, per)
        s["source_counts"], s["source_seen"] = s["start"][0], s["start"][1]
        s["source_mass"] = torch.rand(s["mass"].shape, generator=g, device=dev)
        s["source_positions"] = torch.randint(0, 1 << 20, s["mass"].shape, generator=g, device=dev, dtype=torch.int32)
    if op in ("reserve", "fork", "compact"):
        named = tables[tables >= 0].long()
        s["refs"] = torch.bincount(named, minlength=pages).to(torch.int32)
        s["refs"][pages - 1] = 1
        s["start_refs"] = s["refs"].clone()
    if op == "fork":
        b = torch.arange(B, device=dev)
        s["parents"] = (b - b % samples + torch.randint(0, samples, (B,), generator=g, device=dev)).clamp(max=B - 1).to(torch.int32)
    if op == "compact":
        ended = torch.randperm(B, generator=g, device=dev)[:case["finished"]]
        s["finished"] = torch.zeros(B, dtype=torch.int32, device=dev)
        s["finished"][ended] = 1
        left = s["refs"].clone()
        left[tables[ended][tables[ended] >= 0].long()] = 0
        s["most"] = int((left[int((left > 0).sum()):] > 0).sum())


# ---------------------------------------------------------------------------------------- plain forms


def _places(tables, page, slots):
    """(page, slot in the page) of the logical slots [request, ...]."""
    b = torch.arange(slots.shape[0], device=slots.device).view(-1, *[1] * (slots.dim() - 1))
    return tables.long()[b, slots.long() // page], slots.long() % page


def _new_of(s, B, T, dev):
    return s["new_tokens"] if s["new_tokens"] is not None else torch.full((B,), T, device=dev, dtype=torch.int32)


def _plain_attention(s):
    case, q = s["case"], s["q"]
    B, L, T, Hq, _ = q.shape
    G, n = case["group"], s["max_tokens"]
    H = Hq // G
    slots = torch.arange(n, device=q.device)
    page, at = _places(s["tables"], case["page"], slots.expand(B, -1))                          # [B, n]

    def rows(codes, scales):
        c = codes.transpose(1, 2)[page, at].permute(0, 2, 3, 1, 4)                               # [B, L, H, n, 64]
        return _decode(c, scales.permute(0, 3, 1, 2, 4)[page, at].permute(0, 2, 3, 1, 4))

    qf = q.view(B, L, T, H, G, D).permute(0, 1, 3, 2, 4, 5).reshape(B, L, H, T * G, D).float()
    k = rows(s["k4"], s["k_scales"])
    x = torch.matmul(qf, k.transpose(-1, -2).contiguous()) / math.sqrt(D)
    del k
    if case["cap"] > 0:
        x = case["cap"] * torch.tanh(x / case["cap"])
    t = torch.arange(T, device=q.device)
    new = _new_of(s, B, T, q.device)
    sees = s["counts"].unsqueeze(-1) - (new.view(B, 1, 1, 1) - 1 - t)
    sees = torch.where(t < new.view(B, 1, 1, 1), sees.clamp(min=0), 0)                          # [B, L, H, T]
    seen = (slots < sees.unsqueeze(-1)).unsqueeze(4).expand(B, L, H, T, G, n).reshape(B, L, H, T * G, n)
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    del x
    total = e.sum(-1, keepdim=True)
    lse = torch.log(total) + m
    e = e / torch.where(total == 0, 1.0, total)
    out = torch.matmul(e, rows(s["v4"], s["v_scales"]))
    if case["accumulate"]:
        mass = s["mass"].permute(0, 3, 1, 2)
        mass[page, at] = mass[page, at] + e.sum(3).permute(0, 3, 1, 2) / G
    out = out.view(B, L, H, T, G, D).permute(0, 1, 3, 2, 4, 5).reshape(B, L, T, Hq, D).to(torch.bfloat16)
    return out, lse.view(B, L, H, T, G).permute(0, 1, 3, 2, 4).reshape(B, L, T, Hq)


def _append_places(s):
    """Where the new rows go, [B, L, H, T]: (real, page, layer, slot in the page, head).  Tables hold every new row here, so a padding row
    rewrites what lies in a slot of its own."""
    B, L, T, H, _ = s["k"].shape
    dev = s["k"].device
    t = torch.arange(T, device=dev)
    new = _new_of(s, B, T, dev)
    real = (t < new.view(B, 1)).view(B, 1, 1, T)
    page, at = _places(s["tables"], s["case"]["page"], s["counts"].unsqueeze(-1) + t)
    return new, real, page, torch.arange(L, device=dev).view(1, L, 1, 1), at, torch.arange(H, device=dev).view(1, 1, H, 1)


def _plain_note(s, new, real, page, l, at, h):
    T = real.shape[3]
    s["mass"][page, l, h, at] = torch.where(real, 0.0, s["mass"][page, l, h, at])
    position = (s["seen"].unsqueeze(-1) + torch.arange(T, device=page.device)).to(torch.int32)
    s["positions"][page, l, h, at] = torch.where(real, position, s["positions"][page, l, h, at])
    s["state"].add_(new.view(1, -1, 1, 1).to(torch.int32))


def _plain_append(s):
    """-> the values of the new rows, as they are read back; zeros where there is no token"""
    new, real, page, l, at, h = _append_places(s)
    got = []
    for codes, scales, rows in ((s["k4"], s["k_scales"], s["k"]), (s["v4"], s["v_scales"], s["v"])):
        c, x = _encode(rows.transpose(2, 3))
        codes[page, l, at, h] = torch.where(real.unsqueeze(-1), c, codes[page, l, at, h])
        scales[page, l, h, at] = torch.where(real.unsqueeze(-1), x, scales[page, l, h, at])
        values = _decode(codes[page, l, at, h], scales[page, l, h, at])
        got.append(torch.where(real.unsqueeze(-1), values, 0.0).transpose(2, 3).to(torch.bfloat16))
    _plain_note(s, new, real, page, l, at, h)
    return got


def _plain_store(s):
    """-> the values of all rows"""
    case = s["case"]
    B, L, H = s["counts"].shape
    n = s["max_tokens"]
    slots = torch.arange(n, device=s["counts"].device)
    (p0, a0), (p1, a1) = (_places(t, case["page"], slots.expand(B, -1)) for t in (s["source_tables"], s["tables"]))
    s["state"].copy_(s["start"])
    held = (slots < s["counts"].unsqueeze(-1)).permute(0, 3, 1, 2)                              # [B, n, L, H]
    got = []
    for codes, scales, rows in ((s["k4"], s["k_scales"], s["k_pages"]), (s["v4"], s["v_scales"], s["v_pages"])):
        c, x = _encode(rows.transpose(1, 2)[p0, a0])                                            # [B, n, L, H, ..]
        to = codes.transpose(1, 2)
        to[p1, a1] = torch.where(held.unsqueeze(-1), c, to[p1, a1])
        to = scales.permute(0, 3, 1, 2, 4)
        to[p1, a1] = torch.where(held.unsqueeze(-1), x, to[p1, a1])
        got.append(torch.where(held.unsqueeze(-1), _decode(c, x), 0.0).to(torch.bfloat16).permute(0, 2, 1, 3, 4).contiguous())
    for name in ("mass", "positions"):
        to, value = s[name].permute(0, 3, 1, 2), s["source_" + name].permute(0, 3, 1, 2)[p0, a0]
        to[p1, a1] = torch.where(held, value, to[p1, a1])
    return got


def _plain_turn(s, x, weight, angle):
    """x [B, L, T, heads, 128] -> (normed, normed and turned by angle [B, L?, T, pairs] in 64 bits) in fp32"""
    case = s["case"]
    y = x.float()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * weight.view(-1, 1, 1, D)
    c, d = torch.cos(angle).float().unsqueeze(-2), torch.sin(angle).float().unsqueeze(-2)
    R = case["rotary"]
    turned = y.clone()
    a, b = (y[..., :R:2], y[..., 1:R:2]) if case["interleaved"] else (y[..., :R // 2], y[..., R // 2:R])
    first, second = a * c - b * d, b * c + a * d
    if case["interleaved"]:
        turned[..., :R:2], turned[..., 1:R:2] = first, second
    else:
        turned[..., :R // 2], turned[..., R // 2:R] = first, second
    return y, turned


def _plain_rotate(s):
    B, L, T, _, _ = s["q"].shape
    angle = (s["positions"].double().unsqueeze(-1) * s["freqs"]).unsqueeze(1)
    plain, k = _plain_turn(s, s["k"], s["k_norm"], angle)
    got = [_plain_turn(s, s["q"], s["q_norm"], angle)[1].to(torch.bfloat16), k.to(torch.bfloat16), plain.to(torch.bfloat16)]
    if s["new_tokens"] is None:
        return got
    real = (torch.arange(T, device=angle.device) < s["new_tokens"].view(B, 1)).view(B, 1, T, 1, 1)
    for to, x in zip((s["q_out"], s["k_out"], s["k_plain"]), got):
        to.copy_(torch.where(real, x, to))
    return s["q_out"], s["k_out"], s["k_plain"]


def _plain_rotate_append(s):
    new, real, page, l, at, h = _append_places(s)
    B, L, T, H, _ = s["k"].shape
    # heads have seen the same tokens
    position = s["seen"][:, :, :1] + torch.arange(T, device=page.device)
    angle = position.double().unsqueeze(-1) * s["freqs"]
    k = _plain_turn(s, s["k"], s["k_norm"], angle)[1].to(torch.bfloat16)
    q = _plain_turn(s, s["q"], s["q_norm"], angle)[1].to(torch.bfloat16)
    for pages, rows in ((s["k_pages"], k), (s["v_pages"], s["v"])):
        pages[page, l, at, h] = torch.where(real.unsqueeze(-1), rows.transpose(2, 3), pages[page, l, at, h])
    _plain_note(s, new, real, page, l, at, h)
    return torch.where(real.view(B, 1, T, 1, 1), q, 0.0)


def _plain_copies(s, frm, to):
    for t in (s["k_pages"], s["v_pages"], s["mass"], s["positions"]):
        t[to] = t[frm]


def _in_order(mask, frm, to, most, nobodys):
    """The pairs where mask is, in order, then pairs that change nothing: [most] each."""
    at = torch.where(mask, mask.cumsum(0) - 1, most).clamp(max=most)
    pairs = []
    for x in (frm, to):
        p = torch.full((most + 1,), nobodys, dtype=torch.int64, device=mask.device)
        pairs.append(p.scatter_(0, at, torch.where(mask, x, nobodys))[:most])
    return pairs


def _plain_reserve(s):
    case, tables, refs = s["case"], s["tables"], s["refs"]
    B, P = tables.shape
    N = refs.numel()
    dev = refs.device
    new = _new_of(s, B, case["new"], dev)
    top, low = s["counts"].amax((1, 2)), s["counts"].amin((1, 2))
    page = case["page"]
    holds = (top + page - 1) // page
    need = (torch.minimum(top + new, torch.full_like(top, P * page)) + page - 1) // page
    first = torch.zeros_like(low) if case["own_all"] else torch.where(new > 0, low // page, holds)
    i = torch.arange(P, device=dev)
    there = (tables >= 0) & (tables < N)
    named = torch.where(there, tables, 0).long()
    shared = (i >= first.unsqueeze(1)) & (i < holds.unsqueeze(1)) & there & (refs[named] > 1)
    fresh = (i >= holds.unsqueeze(1)) & (i < need.unsqueeze(1)) & ~there
    b = torch.arange(B, device=dev).unsqueeze(1).expand(B, P)
    tally = torch.zeros(N, dtype=torch.int64, device=dev).scatter_add_(0, named.flatten(), shared.flatten().long())
    last = torch.full((N,), -1, device=dev).scatter_reduce_(0, named.flatten(), torch.where(shared, b, -1).flatten(), "amax")
    copied = shared & ~((tally[named] == refs[named]) & (last[named] == b))      # the last of all that name a page keeps it
    wants = (copied | fresh).flatten()
    rank = wants.cumsum(0) - 1
    free = (refs != 0).to(torch.int8).sort(stable=True).indices
    lack = (wants.sum() - (refs == 0).sum()).clamp(min=0)
    wants = wants & (lack == 0)
    given = free[rank.clamp(min=0, max=N - 1)]
    old = named.flatten()
    copied = copied.flatten() & wants
    change = torch.zeros(N, dtype=torch.int64, device=dev)
    change.scatter_add_(0, given, wants.long())
    change.scatter_add_(0, old, -copied.long())
    tables.copy_(torch.where(wants, given, tables.flatten()).view(B, P))
    refs.add_(change)
    if s["most"]:
        _plain_copies(s, *_in_order(copied, old, given, s["most"], N - 1))
    return torch.stack((copied.sum(), lack)).to(torch.int32)


def _plain_fork(s):
    tables, refs = s["tables"], s["refs"]
    B, N = s["parents"].numel(), refs.numel()
    p = s["parents"].long()
    new = tables[p]
    change = torch.zeros(N + 1, dtype=torch.int64, device=refs.device)
    for t, by in ((new, 1), (tables, -1)):
        there = (t >= 0) & (t < N)
        change.index_add_(0, torch.where(there, t, N).flatten().long(), torch.full((t.numel(),), by, device=refs.device))
    refs.add_(change[:N])
    tables.copy_(new)
    s["state"].copy_(s["state"][:, p])


def _plain_compact(s):
    case, tables, refs = s["case"], s["tables"], s["refs"]
    B, P = tables.shape
    N, page, dev = refs.numel(), case["page"], refs.device
    s["state"].mul_(1 - s["finished"].view(1, B, 1, 1))
    keep = (s["counts"].amax((1, 2)) + page - 1) // page
    there = (tables >= 0) & (tables < N)
    back = there & (torch.arange(P, device=dev) >= keep.unsqueeze(1))
    change = torch.zeros(N + 1, dtype=torch.int64, device=dev)
    change.index_add_(0, torch.where(back, tables, N).flatten().long(), torch.full((B * P,), -1, device=dev))
    refs.add_(change[:N])
    tables.copy_(torch.where(back, -1, tables))
    live = refs > 0
    total = live.sum()
    before = live.cumsum(0) - live.long()
    p = torch.arange(N, device=dev)
    high, low = live & (p >= total), ~live & (p < total)
    to_of = torch.zeros(N + 1, dtype=torch.int64, device=dev)
    to_of.scatter_(0, torch.where(low, p - before, N), p)                 # the i-th lowest free page ..
    to = torch.where(high, to_of[(total - 1 - before).clamp(min=0)], p)   # .. takes the i-th highest that is not
    there = tables >= 0
    tables.copy_(torch.where(there, to[torch.where(there, tables, 0).long()], tables))
    if s["most"]:
        _plain_copies(s, *_in_order(high, p, to, s["most"], N - 1))
    moved = torch.zeros_like(refs).scatter_add_(0, to, refs)
    refs.copy_(moved)
    return high.sum().to(torch.int32)


def _restore(s):
    """What a pass starts from: these calls change what they find."""
    s["state"].copy_(s["start"])
    s["tables"].copy_(s["start_tables"])
    s["refs"].copy_(s["start_refs"])


def run(s):
    op, case = s["op"], s["case"]
    C, cache, new = s.get("C"), s.get("cache"), s["new_tokens"]
    if op == "attention":
        if own:
            out, lse = C.compactor_fp4_attention(cache, s["q"], new_tokens=new, softcap=case["cap"],
                                                 accumulate=case["accumulate"], want_lse=True)
        else:
            out, lse = _plain_attention(s)
        return {"out": out, "lse": lse, "mass": s["mass"] if case["accumulate"] else None}
    if op == "append":
        s["state"].copy_(s["start"])          # the rows are rewritten on every pass
        if own:
            C.compactor_fp4_append(cache, s["k"], s["v"], new_tokens=new)
            k, v = C.compactor_fp4_read(cache, case["new"], new_tokens=new)
        else:
            k, v = _plain_append(s)
        return {"k": k, "v": v, "mass": s["mass"], "positions": s["positions"], "counts": s["counts"], "seen": s["seen"]}
    if op == "store":
        if own:
            C.compactor_fp4_store(cache, s["source"])
            k, v = C.compactor_fp4_read(cache, s["max_tokens"], first=0)
        else:
            k, v = _plain_store(s)
        return {"k": k, "v": v, "mass": s["mass"], "positions": s["positions"], "counts": s["counts"], "seen": s["seen"]}
    if op == "rotate":
        if own:
            q, k, plain = C.compactor_rotate(s["rotation"], s["q"], s["k"], positions=s["positions"], new_tokens=new, want_plain=True,
                                             q_out=s.get("q_out"), k_out=s.get("k_out"), k_plain=s.get("k_plain"))
        else:
            q, k, plain = _plain_rotate(s)
        return {"q": q, "k": k, "k_plain": plain}
    if op == "rotate_append":
        s["state"].copy_(s["start"])
        if own:
            q = torch.zeros_like(s["q"]) if new is not None else None
            q = C.compactor_cache_append_rotated(cache, s["rotation"], s["k"], s["v"], s["q"], new_tokens=new, q_out=q)
        else:
            q = _plain_rotate_append(s)
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"].view(torch.int16), "positions": s["positions"],
                "mass": s["mass"], "counts": s["counts"], "seen": s["seen"]}
    _restore(s)
    got = {"tables": s["tables"], "refs": s["refs"]}
    if op == "reserve":
        if own:
            pairs, done = C.compactor_pages_reserve(cache, s["refs"], case["new"], new_tokens=new, own_all=case["own_all"])
            C.compactor_pages_copy(cache, pairs, done)
            got["done"] = done
        else:
            got["done"] = _plain_reserve(s)
    elif op == "fork":
        if own:
            C.compactor_pages_fork(cache, s["refs"], s["parents"])
        else:
            _plain_fork(s)
    else:
        if own:
            C.compactor_pages_release(cache, s["refs"], finished=s["finished"])
            pairs, done = C.compactor_pages_compact(cache, s["refs"])
            C.compactor_pages_copy(cache, pairs, done)
            got["moved"] = done[0]
        else:
            got["moved"] = _plain_compact(s)
    if op != "fork":      # rows are copies: compared bit by bit
        got.update(k_pages=s["k_pages"].view(torch.int16), v_pages=s["v_pages"].view(torch.int16), mass=s["mass"],
                   positions=s["positions"])
    got.update(counts=s["counts"], seen=s["seen"])
    return got


def work(case):
    B, L, H, G, T, page = (case[k] for k in ("requests", "layers", "kv_heads", "group", "new", "page"))
    op = case["op"]
    rows = sum(c for b in _head_counts(case) for l in b for c in l) if op != "rotate" else 0
    new = L * H * sum(_news(case))
    row4 = 2 * (D // 2 + 4)               # K and V of a token
    if op == "attention":
        state = 8 if case["accumulate"] else 0
        return {"bytes": rows * (row4 + state) + B * L * T * H * G * (4 * D + 4), "flops": rows * G * T * 4 * D}
    if op == "append":
        return {"bytes": new * (4 * D + 2 * row4 + 8 + 4 * D) + 16 * B * L * H, "flops": 0}
    if op == "store":
        return {"bytes": rows * (4 * D + 2 * row4 + 16 + 4 * D), "flops": 0}
    if op == "rotate":
        return {"bytes": new * D * (4 * G + 6), "flops": 0}
    if op == "rotate_append":
        return {"bytes": new * (D * (4 * G + 8) + 8) + 16 * B * L * H, "flops": 0}
    one = L * H * page * (4 * D + 8)      # bytes of a page
    heads = 8 * B * L * H
    if op == "fork":
        return {"bytes": 8 * sum(-(-max(max(r) for r in b) // page) for b in _head_counts(case)) + 2 * heads, "flops": 0}
    if op == "reserve":
        written = _written(case)
        return {"bytes": 2 * one * _copies(case) + heads // 2 + 8 * sum(need - min(first, hold) for first, hold, need in written), "flops": 0}
    held = [-(-max(max(r) for r in b) // page) for b in _head_counts(case)]
    gone = sum(held) * case["finished"] // B      # about a share `gone` of what stays lies in the part that is given up
    stay = sum(held) - gone
    return {"bytes": 2 * one * (stay * gone // max(1, stay + gone)) + 8 * sum(held) + heads, "flops": 0}


# ---------------------------------------------------------------------------------------- 64 bits


def _values64(x):
    """What a row's codes stand for, from the definition: bf16 [..., 128] -> 64 bits."""
    g = x.double().reshape(*x.shape[:-1], 4, 32)
    fraction, power = torch.frexp(g.abs().amax(-1, keepdim=True))               # fraction in [1/2, 1)
    power = torch.where(fraction >= 0.875, power, power - 1) - 2
    unit = torch.ldexp(torch.ones_like(fraction), power.clamp(TINY - 127, LARGEST - 127))
    size = (g / unit).abs().clamp(max=6.0)
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))          # of the numbers around it
    return (torch.round(size / step) * step * unit * torch.sign(g)).reshape(x.shape)


def _turned64(case, x, weight, angle):
    y = x.double()
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * weight.double()[:, None, None]
    R = case["rotary"]
    pairs = y[..., :R].unflatten(-1, (R // 2, 2) if case["interleaved"] else (2, R // 2))
    if not case["interleaved"]:
        pairs = pairs.transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), angle).unsqueeze(-2)
    z = torch.view_as_real(z)
    if not case["interleaved"]:
        z = z.transpose(-1, -2)
    return y, torch.cat((z.flatten(-2), y[..., R:]), -1)


def exact(case, seed):
    op = case["op"]
    if op in ("reserve", "fork", "compact"):
        return None            # copies and whole numbers
    s = prepare(case, seed)
    B, L, H, G, T, page = (case[k] for k in ("requests", "layers", "kv_heads", "group", "new", "page"))
    news, counts = _news(case), _head_counts(case)
    state = {"mass": None, "positions": None, "counts": None, "seen": None}
    if op == "append":
        got = {n: _values64(s[n]) for n in ("k", "v")}
        for b, n in enumerate(news):
            for t in got.values():
                t[b, :, n:] = 0.0
        return {**got, **state}
    if op == "store":
        got = {}
        for n in ("k", "v"):
            t = torch.zeros(B, L, s["max_tokens"], H, D, dtype=torch.float64, device=s["counts"].device)
            for b in range(B):
                rows = s[n + "_pages"][s["source_tables"][b].long()].permute(1, 0, 2, 3, 4).flatten(1, 2)      # [L, slots, H, D]
                for l in range(L):
                    for h in range(H):
                        c = counts[b][l][h]
                        t[b, l, :c, h] = _values64(rows[l, :c, h])
            got[n] = t
        return {**got, **state}
    if op == "rotate":
        angle = (s["positions"].double()[:, None, :, None] * s["freqs"])
        plain, k = _turned64(case, s["k"], s["k_norm"], angle)
        got = {"q": _turned64(case, s["q"], s["q_norm"], angle)[1], "k": k, "k_plain": plain}
        for b, n in enumerate(news):
            for t in got.values():
                t[b, :, n:] = 0.0
        return got
    if op == "rotate_append":
        seen = torch.tensor([3 * n + case["far"] for n in _lengths(case)], device=s["k"].device, dtype=torch.float64)
        angle = ((seen[:, None] + torch.arange(T, device=seen.device))[:, None, :, None] * s["freqs"])
        q, k = (_turned64(case, s[n], s[n + "_norm"], angle)[1] for n in ("q", "k"))
        pool = s["k_pages"].double()
        for b, n in enumerate(news):
            q[b, :, n:] = 0.0
            for l in range(L):
                for h in range(H):
                    slot = counts[b][l][h] + torch.arange(n, device=seen.device)
                    pool[s["tables"][b].long()[slot // page], l, slot % page, h] = k[b, l, :n, h]
        return {"q": q, "k_pages": pool, "v_pages": None, **state}
    # attention, head by head
    out = torch.zeros(B, L, T, H * G, D, dtype=torch.float64, device=s["q"].device)
    lse = torch.full((B, L, T, H * G), -math.inf, dtype=torch.float64, device=out.device)
    mass = s["mass"].double()
    numbers = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device=out.device) / 2

    def rows(codes, scales, c):
        byte = codes.reshape(-1, 64)[:c].long()
        code = torch.stack((byte % 16, byte // 16), 2).flatten(1)
        x = torch.where(code >= 8, -numbers[code % 8], numbers[code % 8])
        return x * torch.exp2(scales.reshape(-1, 4)[:c].double() - 127).repeat_interleave(32, 1)

    for b in range(B):
        pages = s["tables"][b].long()
        for l in range(L):
            for h in range(H):
                c = counts[b][l][h]
                k = rows(s["k4"][pages, l, :, h], s["k_scales"][pages, l, h], c)
                v = rows(s["v4"][pages, l, :, h], s["v_scales"][pages, l, h], c)
                weight = torch.zeros(pages.numel() * page, dtype=torch.float64, device=out.device)
                for t in range(news[b]):
                    see = c - (news[b] - 1 - t)
                    if see <= 0:
                        continue
                    at = slice(h * G, (h + 1) * G)
                    x = s["q"][b, l, t, at].double() @ k[:see].t() * D ** -0.5
                    if case["cap"] > 0:
                        x = torch.tanh(x / case["cap"]) * case["cap"]
                    lse[b, l, t, at] = torch.logsumexp(x, 1)
                    p = torch.softmax(x, 1)
                    out[b, l, t, at] = p @ v[:see]
                    weight[:see] += p.mean(0)
                if case["accumulate"]:
                    mass[pages, l, h] += weight.view(-1, page)
    return {"out": out, "lse": lse, "mass": mass if case["accumulate"] else None}
