"""A language model's reader beside the index, as measurable cases.

The passages that a search returns go through a model as one packed prompt,
their keys and values into a cache of 8-bit codes in pages, and the answers
are decoded from it.  A case is one pass through one of the operators of that
path: attention over whole prompts, appending to the cache, attention over the
cache, and the cache's pages (fork, resize, compact).

Cache layout: pages of 64 tokens, scale blocks of 16 tokens per head,

    k        [layers, pages, heads, 64, D]       int8 or e4m3
    v        [layers, pages, heads, 4, D, 16]    (tokens of a block innermost)
    k_scale  [layers, pages, heads, 4]           float32, v_scale likewise
    tables   [rows, width] int32 page ids (-1: none), lens [rows] int32,
    refs     [pages] int32: rows that hold a page (0: free)

`run` computes the operators in plain torch in 32 bits, or with own = True
calls the library's.
"""
import math
import random

import torch

own = False

PAGE, BLOCK = 64, 16
QMAX = {"int8": 127.0, "fp8": 448.0}
CODE = {"int8": torch.int8, "fp8": torch.float8_e4m3fn}
FLOAT = {"bf16": torch.bfloat16, "f16": torch.float16}
TINY = 2.0 ** -100   # amax below this is stored as zero


# ------------------------------------------------------------------- cases
def _prompt(name, rows, longest, shortest, heads, kv_heads, d, dtype, extra=0):
    """extra: keys before each row's queries (a prefix that is there already);
    negative: that many keys fewer than queries, so that the first see none."""
    return _named(name, op="prompt", rows=rows, longest=longest, shortest=shortest, heads=heads,
                  kv_heads=kv_heads, d=d, dtype=dtype, extra=extra)


def _append(name, rows, longest, shortest, new, kv_heads, d, kv, dtype):
    """new: new tokens of a row (0: all of them, the row was empty)."""
    return _named(name, op="append", rows=rows, longest=longest, shortest=shortest, new=new,
                  kv_heads=kv_heads, d=d, kv=kv, dtype=dtype)


def _attend(name, rows, longest, shortest, new, heads, kv_heads, d, kv, dtype, empty=0):
    """new: queries of a row, its last tokens (ragged where above 1); empty:
    rows of the batch that hold no token (slots of a server without a request)."""
    return _named(name, op="attend", rows=rows, longest=longest, shortest=shortest, new=new,
                  heads=heads, kv_heads=kv_heads, d=d, kv=kv, dtype=dtype, empty=empty)


def _pages(name, op, rows, longest, shortest, pages, layers, kv_heads, d, kv, more=0):
    """more: children of each parent (fork), tokens that rows grow and shrink
    by (resize); compact: unused."""
    return _named(name, op=op, rows=rows, longest=longest, shortest=shortest, pages=pages,
                  layers=layers, kv_heads=kv_heads, d=d, kv=kv, more=more)


def _named(name, **case):
    return dict(case, name=name) if name else case


def listed():
    return [
        # a handful of passages, each through a small encoder-sized model on its own
        _prompt("prompt_passages", 32, 200, 16, 12, 12, 64, "f16"),
        # the prompts of one scheduling step of a server, grouped heads
        _prompt("prompt_packed", 8, 2048, 130, 32, 8, 128, "bf16"),
        # one long context: many retrieved documents
        _prompt("prompt_long", 1, 16384, 16384, 16, 2, 128, "bf16"),
        # one decoded token of each of 64 running answers
        _append("append_step", 64, 4096, 300, 1, 8, 128, "int8", "bf16"),
        # whole prompts into empty rows
        _append("append_prompts", 16, 2000, 70, 0, 8, 128, "fp8", "f16"),
        # one user, one token: latency only
        _attend("attend_one", 1, 777, 777, 1, 32, 8, 128, "int8", "bf16"),
        # a decoding step of a full server, ragged contexts
        _attend("attend_batch", 64, 8192, 300, 1, 32, 8, 128, "int8", "bf16"),
        # few rows with very long contexts
        _attend("attend_long", 2, 131072, 100001, 1, 64, 8, 128, "fp8", "f16"),
        # chunks of later prompt parts against the cached earlier ones
        _attend("attend_chunk", 4, 8192, 2500, 256, 32, 8, 64, "fp8", "bf16"),
        # several answers from each of 24 contexts: the part-filled pages are copied
        _pages("fork_answers", "fork", 24, 4000, 100, 1400, 4, 8, 128, "int8", more=5),
        # a step's growth and the retreat after rejected drafts over many rows
        _pages("resize_rows", "resize", 512, 4000, 1, 40000, 1, 1, 64, "int8", more=70),
        # half-empty pool moved to its front, so that the rest can go
        _pages("compact_pool", "compact", 48, 3000, 50, 2400, 4, 8, 128, "fp8"),
    ]


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) if hi > lo else int(lo)
    return n | 1 if n > 1000 else n   # long ones are odd: no tile divides them


HEADS = [(32, 8), (12, 12), (64, 8), (16, 2), (24, 8), (8, 1), (14, 2), (5, 5)]


def draw(rng):
    op = rng.choice(["prompt", "prompt", "append", "attend", "attend", "attend", "fork", "resize", "compact"])
    heads, kv_heads = rng.choice(HEADS)
    d = rng.choice([64, 128, 128, 256])
    kv = rng.choice(["int8", "fp8"])
    dtype = rng.choice(["bf16", "f16"])
    if op == "prompt":
        longest = _log_int(rng, 3, min(8000, int((2 ** 39 / (2 * heads * d)) ** 0.5)))
        rows = _log_int(rng, 1, max(1, min(64, int(2 ** 31 / (heads * longest ** 2) / (d / 128)))))
        extra = rng.choice([0, 0, 0, rng.randint(1, 500), -rng.randint(1, 9)])
        return _prompt(None, rows, longest, max(1, longest // rng.randint(1, 12)), heads, kv_heads, d, dtype, extra)
    if op == "append":
        new = rng.choice([0, 1, 1, rng.randint(2, 40)])
        longest = _log_int(rng, max(new, 1), 6000)
        rows = _log_int(rng, 1, max(1, min(256, int(2 ** 25 / (longest * kv_heads * d)), 150000 // longest)))
        return _append(None, rows, longest, max(new, 1, longest // rng.randint(1, 12)), new, kv_heads, d, kv, dtype)
    if op == "attend":
        new = rng.choice([1, 1, 1, rng.randint(2, 9), _log_int(rng, 10, 400)])
        longest = _log_int(rng, max(new, 1), 120000)
        new = max(1, min(new, int(2 ** 37 / (4 * d * heads * longest))))
        most = min(256, 2 ** 28 / (longest * kv_heads * d), 2 ** 37 / (4 * d * heads * longest * new))
        rows = _log_int(rng, 1, max(1, int(most)))
        return _attend(None, rows, longest, max(new, longest // rng.randint(1, 12)), new, heads, kv_heads, d, kv, dtype,
                       rng.choice([0, 0, min(2, rows - 1)]))
    longest = _log_int(rng, 1, 5000)
    width = longest // PAGE + 1
    kv_heads = rng.choice([1, 2, 8])
    if op == "fork":
        rows, more, layers = _log_int(rng, 1, 32), rng.randint(1, 7), rng.randint(1, 4)
        pages = rows * width + 2 * rows * more + rng.randint(0, 100)
    elif op == "resize":
        rows, more, layers = _log_int(rng, 1, 400), rng.randint(1, 300), 1
        kv_heads, d = 1, 64
        pages = rows * (width + more // PAGE + 2) + rng.randint(0, 9000)
    else:
        rows, more, layers = _log_int(rng, 1, 48), 0, rng.randint(1, 4)
        pages = int(rows * width * rng.uniform(1.1, 2.5)) + 3
    return _pages(None, op, rows, longest, max(1, longest // rng.randint(1, 12)), min(pages, 2400) if op != "resize" else pages | 1,
                  layers, kv_heads, d, kv, more)


def _lens(case):
    """The rows' lengths: spread over the logarithm, the first one the longest."""
    r = random.Random("%d %d %d" % (case["rows"], case["longest"], case["shortest"]))
    lens = [case["longest"]] + [_log_int(r, case["shortest"], case["longest"]) for _ in range(case["rows"] - 1)]
    return lens[:len(lens) - case.get("empty", 0)] + [0] * case.get("empty", 0)


def _news(case, lens):
    if case["new"] <= 1:
        return [n if case["new"] == 0 else min(1, n) if case["op"] == "append" else 1 for n in lens]
    r = random.Random("new %d %d" % (case["rows"], case["new"]))
    return [min(n, case["new"] if i == 0 else r.randint((case["new"] + 1) // 2, case["new"])) for i, n in enumerate(lens)]


def _key_lens(case, lens):
    return [max(0, n + case["extra"]) for n in lens]


# ------------------------------------------------------------------ inputs
def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _cache(g, layers, pages, heads, d, kv):
    """Codes as quantised keys and values have them: normal, channels of
    different size, each block's largest near the end of the range."""
    spread = 0.12 + 0.2 * torch.rand(d, generator=g, device="cuda")
    spread[:: max(1, d // 4)] *= 2.5
    def codes(*shape):
        return torch.randn(layers, pages, heads, *shape, generator=g, device="cuda")
    def coded(x):
        x = x.mul_(QMAX[kv]).clamp_(-QMAX[kv], QMAX[kv])
        return x.round_().to(torch.int8) if kv == "int8" else x.to(torch.float8_e4m3fn)
    k = coded(codes(PAGE, d).mul_(spread))
    v = coded(codes(PAGE // BLOCK, d, BLOCK).mul_(0.3))
    def scales(mean):
        return (0.5 + torch.rand(layers, pages, heads, PAGE // BLOCK, generator=g, device="cuda")) * (mean / QMAX[kv])
    return {"k": k, "v": v, "k_scale": scales(5.0), "v_scale": scales(3.0),
            "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def _tables(g, lens, width, spare=3):
    """Page tables of rows that hold pages in no order; the pool's size."""
    counts = [-(-n // PAGE) for n in lens]
    total = sum(counts)
    order = torch.randperm(total + spare, generator=g, device="cuda")[:total].to(torch.int32)
    held = torch.arange(width, device="cuda")[None, :] < _ints(counts)[:, None]
    tables = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    tables[held] = order
    return tables, total + spare


def _held(case, seed, lens, width, taken=0):
    """Tables and reference counts of a pool in use: every second row shares
    the first whole pages of the row before it (a common context)."""
    r = random.Random(seed)
    counts = [-(-n // PAGE) for n in lens]
    free = list(range(case["pages"]))
    r.shuffle(free)
    keep = max(0, len(free) - taken)   # pages that stay free
    tables, refs, kept = [], [0] * case["pages"], []
    for i, n in enumerate(counts):
        whole = lens[i] // PAGE
        shared = tables[-1][:min(whole, lens[i - 1] // PAGE, len(tables[-1])) // 2] if i % 2 else []
        need = n - len(shared)
        if need > keep:                # a row that the pool has no room for holds nothing
            shared, need, n = [], 0, 0
        got = shared + [free.pop() for _ in range(need)]
        keep -= need
        for p in got:
            refs[p] += 1
        tables.append(got)
        kept.append(lens[i] if n else 0)
    full = [t + [-1] * (width - len(t)) for t in tables]
    return _ints(full).reshape(len(lens), width), _ints(kept), _ints(refs)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"op": case["op"]}
    lens = _lens(case)
    if case["op"] == "prompt":
        keys = _key_lens(case, lens)
        h, hk, dt = case["heads"], case["kv_heads"], FLOAT[case["dtype"]]
        s["starts"] = _ints(_starts(lens))
        if case["extra"] == 0:   # one fused projection: q, k and v are its parts
            qkv = torch.randn(sum(lens), h + 2 * hk, case["d"], generator=g, device="cuda").to(dt)
            s["q"], s["k"], s["v"], s["k_starts"] = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:], None
        else:
            s["q"] = torch.randn(sum(lens), h, case["d"], generator=g, device="cuda").to(dt)
            kv = torch.randn(2, sum(keys), hk, case["d"], generator=g, device="cuda").to(dt)
            s["k"], s["v"], s["k_starts"] = kv[0], kv[1], _ints(_starts(keys))
        s["longest"], s["longest_key"] = max(lens), max(keys)
        return s
    if case["op"] in ("append", "attend"):
        news = _news(case, lens)
        s["tables"], pages = _tables(g, lens, -(-max(lens) // PAGE))
        s["lens"], s["longest"], s["most_new"] = _ints(lens), max(lens), max(news)
        s.update(_cache(g, 1, pages, case["kv_heads"], case["d"], case["kv"]))
        s["starts"] = None if case["new"] == 1 and min(news) == 1 else _ints(_starts(news))
        dt, total = FLOAT[case["dtype"]], sum(news)
        if case["op"] == "attend":
            s["q"] = (1.5 * torch.randn(total, case["heads"], case["d"], generator=g, device="cuda")).to(dt)
        else:
            size = 0.5 + torch.rand(1, 2 * case["kv_heads"], case["d"], generator=g, device="cuda")
            size[..., ::max(1, case["d"] // 4)] *= 3.0
            kv = (size * torch.randn(total, 2 * case["kv_heads"], case["d"], generator=g, device="cuda")).to(dt)
            s["new_k"], s["new_v"] = kv[:, :case["kv_heads"]], kv[:, case["kv_heads"]:]
        return s
    more = case["more"]
    width = -(-(max(lens) + (more if case["op"] == "resize" else 0)) // PAGE) + 1
    s.update(_cache(g, case["layers"], case["pages"], case["kv_heads"], case["d"], case["kv"]))
    if case["op"] == "fork":
        rows = len(lens) * (1 + more)
        s["tables"], s["lens"], s["refs"] = _held(case, seed, lens + [0] * (rows - len(lens)), width, 2 * len(lens) * more)
        s["src"] = _ints([p for p in range(len(lens)) for _ in range(more)])
        s["dst"] = _ints(list(range(len(lens), rows)))
    elif case["op"] == "resize":
        r = random.Random(seed + 1)
        s["tables"], s["lens"], s["refs"] = _held(case, seed, lens, width, len(lens) * (more // PAGE + 2))
        kept = s["lens"].tolist()
        s["up"] = _ints([n + r.randint(0, more) for n in kept])
        s["down"] = _ints([max(0, n - r.randint(0, more)) if r.random() < 0.9 else -1 for n in kept])
    else:
        s["tables"], s["lens"], s["refs"] = _held(case, seed, lens, width)
    return s


# ------------------------------------------------------------- plain forms
def _places(starts, lens, total):
    """Row, index within the row and position of every new token."""
    t = torch.arange(total, device="cuda")
    if starts is None:
        return t, torch.zeros_like(t), lens.long() - 1
    at = starts.long()
    b = torch.searchsorted(at[1:], t, right=True)
    i = t - at[b]
    return b, i, lens.long()[b] - (at[1:] - at[:-1])[b] + i


def _softmax_product(q, k, v, seen):
    """q [.., m, d], k and v [.., n, d], seen [.., m, n] -> out, lse (natural)."""
    x = torch.matmul(q, k.transpose(-1, -2))
    x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True) if x.shape[-1] else x.new_full(x.shape[:-1] + (1,), -math.inf)
    base = torch.where(top == -math.inf, torch.zeros_like(top), top)
    x.sub_(base).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x, v) / torch.where(total == 0, torch.ones_like(total), total)
    return out, (base + total.log()).squeeze(-1)


def _plain_prompt(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    starts = s["starts"].long()
    k_starts = starts if s["k_starts"] is None else s["k_starts"].long()
    n, nk = starts[1:] - starts[:-1], k_starts[1:] - k_starts[:-1]
    rows, h, hk, d = n.numel(), q.shape[1], k.shape[1], q.shape[2]
    b, i, pos = _places(s["starts"], nk, q.shape[0])
    tk = torch.arange(k.shape[0], device="cuda")
    bk = torch.searchsorted(k_starts[1:], tk, right=True)
    qp = q.new_zeros(rows, s["longest"], h, d)
    qp[b, i] = q * (1.0 / math.sqrt(d))
    kp, vp = k.new_zeros(2, rows, s["longest_key"], hk, d)
    kp[bk, tk - k_starts[bk]] = k
    vp[bk, tk - k_starts[bk]] = v
    at = torch.full((rows, s["longest"]), -1, device="cuda")
    at[b, i] = pos
    seen = torch.arange(s["longest_key"], device="cuda") <= at[..., None]
    qp = qp.view(rows, s["longest"], hk, h // hk, d).permute(0, 2, 3, 1, 4)
    out, lse = _softmax_product(qp, kp.permute(0, 2, 1, 3)[:, :, None], vp.permute(0, 2, 1, 3)[:, :, None], seen[:, None, None])
    out, lse = out.reshape(rows, h, -1, d), lse.reshape(rows, h, -1)
    return {"out": out[b, :, i].to(s["q"].dtype), "lse": lse[b, :, i]}


def _coded(x, r, dtype):
    top = QMAX["int8" if dtype == torch.int8 else "fp8"]
    x = (x * r).clamp(-top, top)
    return x.round().to(torch.int8) if dtype == torch.int8 else x.to(dtype)


def _append_part(x, pages, scale, where, slot, inv, held, tokens_last):
    """One of the two stores: pages [pages, heads, 4, ...] codes, in place."""
    page, sub = where
    bits = pages.view(torch.int8)
    old = bits[page, :, sub].view(pages.dtype).float()                # [blocks, heads, 16, d]
    old = old.transpose(-1, -2) if tokens_last else old
    fresh = x.new_zeros(old.shape, dtype=torch.float32)
    fresh[inv, :, slot] = x.float()
    new = torch.zeros(old.shape[0], BLOCK, dtype=torch.bool, device="cuda")
    new[inv, slot] = True
    top = QMAX["int8" if pages.dtype == torch.int8 else "fp8"]
    amax = fresh.abs().amax((-1, -2))
    s0 = torch.where(held[:, None] > 0, scale[page, :, sub], torch.zeros_like(amax))
    s1 = torch.maximum(s0, torch.where(amax < TINY, torch.zeros_like(amax), amax / top))
    r = torch.where(s1 > 0, 1.0 / s1, torch.zeros_like(s1))[..., None, None]
    ratio = torch.where(s1 > 0, s0 / s1, torch.zeros_like(s1))[..., None, None]
    old = torch.where(held[:, None, None, None] > 0, old, torch.zeros_like(old))
    codes = torch.where(new[:, None, :, None], _coded(fresh, r, pages.dtype).float(),
                        _coded(old, ratio, pages.dtype).float()).to(pages.dtype)
    codes = codes.transpose(-1, -2).contiguous() if tokens_last else codes
    bits[page, :, sub] = codes.view(torch.int8)
    scale[page, :, sub] = s1


def _plain_append(s):
    b, i, pos = _places(s["starts"], s["lens"], s["new_k"].shape[0])
    first = pos - i                                       # of the row's new tokens
    wide = s["tables"].shape[1] * (PAGE // BLOCK)
    key, inv = torch.unique(b * wide + pos // BLOCK, return_inverse=True)
    row, blk = key // wide, key % wide
    begin = torch.zeros(s["lens"].numel(), dtype=torch.long, device="cuda").index_put_((b,), first)
    held = (begin[row] - blk * BLOCK).clamp(0, BLOCK)
    where = s["tables"].long()[row, blk // 4], blk % 4
    _, pages, heads, _, d = s["k"].shape
    _append_part(s["new_k"], s["k"][0].view(pages, heads, 4, BLOCK, d), s["k_scale"][0], where, pos % BLOCK, inv, held, False)
    _append_part(s["new_v"], s["v"][0], s["v_scale"][0], where, pos % BLOCK, inv, held, True)
    return {m: s[m] for m in ("k", "v", "k_scale", "v_scale")}


def _plain_attend(s):
    q, lens = s["q"].float(), s["lens"]
    _, _, hk, _, d = s["k"].shape
    h, rows, most = q.shape[1], lens.numel(), s["most_new"]
    pages = s["tables"][:, :-(-s["longest"] // PAGE)].long().clamp(min=0)
    n = pages.shape[1] * PAGE
    k = s["k"][0].view(torch.int8)[pages].view(s["k"].dtype).float().view(rows, -1, hk, 4, BLOCK, d)
    k = (k * s["k_scale"][0][pages][..., None, None]).permute(0, 2, 1, 3, 4, 5).reshape(rows, hk, n, d)
    v = s["v"][0].view(torch.int8)[pages].view(s["v"].dtype).float()
    v = (v * s["v_scale"][0][pages][..., None, None]).permute(0, 2, 1, 3, 5, 4).reshape(rows, hk, n, d)
    b, i, pos = _places(s["starts"], lens, q.shape[0])
    qp = q.new_zeros(rows, most, h, d)
    qp[b, i] = q * (1.0 / math.sqrt(d))
    at = torch.full((rows, most), -1, device="cuda")
    at[b, i] = pos
    seen = (torch.arange(n, device="cuda") <= at[..., None])[:, None].expand(rows, h // hk, most, n).reshape(rows, 1, -1, n)
    qp = qp.view(rows, most, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(rows, hk, -1, d)
    out, lse = _softmax_product(qp, k, v, seen)
    out, lse = out.reshape(rows, h, most, d), lse.reshape(rows, h, most)
    return {"out": out[b, :, i].to(s["q"].dtype), "lse": lse[b, :, i]}


def _copy_pages(s, src, dst):
    for m in ("k", "v", "k_scale", "v_scale"):
        t = s[m].view(torch.int8) if s[m].element_size() == 1 else s[m]
        t[:, dst] = t[:, src]


def _plain_fork(s):
    tables, lens, refs, src, dst = s["tables"], s["lens"], s["refs"], s["src"].long(), s["dst"].long()
    old, n = tables[src].clone(), lens[src].clone()
    part = (n % PAGE != 0) & (src != dst)
    free = (refs == 0).nonzero()[:, 0]
    last = part.long().cumsum(0)
    fits = ~part | (last <= free.numel())
    moved = src != dst
    away = tables[dst][moved]
    refs.index_add_(0, away[away >= 0].long(), -torch.ones_like(away[away >= 0]))
    whole = (torch.arange(tables.shape[1], device="cuda") < (n // PAGE)[:, None]) & (fits & moved)[:, None]
    refs.index_add_(0, old[whole].long(), torch.ones_like(old[whole]))
    took = (part & fits).nonzero()[:, 0]
    fresh = free[last[took] - 1]
    new = torch.where(whole, old, torch.full_like(old, -1))
    new[took, n[took] // PAGE] = fresh.to(torch.int32)
    refs[fresh] = 1
    _copy_pages(s, old[took, n[took] // PAGE].long(), fresh)
    tables[dst[moved]] = new[moved]
    lens[dst[moved]] = torch.where(fits, n, torch.zeros_like(n))[moved]


def _plain_resize(s, goal):
    tables, lens, refs = s["tables"], s["lens"], s["refs"]
    width, pages = tables.shape[1], (lens + PAGE - 1) // PAGE
    goal = torch.where((goal < 0) | (goal > width * PAGE), lens, goal)
    need = (goal + PAGE - 1) // PAGE
    col = torch.arange(width, device="cuda")
    drop = (col >= need[:, None]) & (col < pages[:, None])
    away = tables[drop]
    refs.index_add_(0, away.long(), -torch.ones_like(away))
    tables[drop] = -1
    grows = goal > lens
    last = (pages - 1).clamp(min=0).long()[:, None]
    held = tables.gather(1, last)[:, 0].clamp(min=0).long()
    part = grows & (lens % PAGE != 0) & (refs[held] > 1)
    more = torch.where(grows, need - pages + part.to(need.dtype), torch.zeros_like(need))
    end = more.long().cumsum(0)
    free = (refs == 0).nonzero()[:, 0]
    fits = (more == 0) | (end <= free.numel())
    first = pages - part.to(pages.dtype)
    put = (fits & grows)[:, None] & (col >= first[:, None]) & (col < need[:, None])
    index = ((end - more)[:, None] + col - first[:, None])[put]
    copied = part & fits
    source = held[copied]
    tables[put] = free[index].to(torch.int32)
    refs[free[index]] = 1
    refs.index_add_(0, source, -torch.ones_like(source, dtype=torch.int32))
    _copy_pages(s, source, tables.gather(1, last)[:, 0][copied].long())
    lens.copy_(torch.where(fits, goal, lens))


def _plain_compact(s, tables, refs):
    live = refs > 0
    count = live.sum()
    low = torch.arange(refs.numel(), device="cuda") < count
    src, dst = (live & ~low).nonzero()[:, 0], (~live & low).nonzero()[:, 0]
    to = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
    to[src] = dst.to(torch.int32)
    tables.copy_(torch.where(tables >= 0, to[tables.clamp(min=0).long()], tables))
    refs[dst] = refs[src]
    refs[src] = 0
    _copy_pages(s, src, dst)
    return count.to(torch.int32).reshape(1)


def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["op"] == "prompt":
        return _plain_prompt(s)
    if s["op"] == "append":
        return _plain_append(s)
    if s["op"] == "attend":
        return _plain_attend(s)
    said = {m: s[m] for m in ("k", "v", "k_scale", "v_scale", "tables", "lens", "refs")}
    if s["op"] == "fork":
        _plain_fork(s)
    elif s["op"] == "resize":
        _plain_resize(s, s["up"])
        _plain_resize(s, s["down"])
    else:   # the pool stays as it was, so that every pass has the same pages to move
        said["tables"], said["refs"] = s["tables"].clone(), s["refs"].clone()
        said["live"] = _plain_compact(s, said["tables"], said["refs"])
    return said


def _run_own(s):
    import paper_2607_16973_amd as tq
    if s["op"] == "prompt":
        out, lse = tq.attention(s["q"], s["k"], s["v"], s["starts"], s["k_starts"], longest=s["longest"], return_lse=True)
        return {"out": out, "lse": lse}
    cache = tq.KVCache.over(s["k"], s["v"], s["k_scale"], s["v_scale"], s["status"])
    if s["op"] == "append":
        cache.append(0, s["new_k"], s["new_v"], s["tables"], s["lens"], s["starts"])
        return {m: s[m] for m in ("k", "v", "k_scale", "v_scale")}
    if s["op"] == "attend":
        out, lse = cache.attend(0, s["q"], s["tables"], s["lens"], s["starts"], longest=s["longest"], return_lse=True)
        return {"out": out, "lse": lse}
    said = {m: s[m] for m in ("k", "v", "k_scale", "v_scale", "tables", "lens", "refs")}
    if s["op"] == "compact":
        said["tables"], said["refs"] = s["tables"].clone(), s["refs"].clone()
    rows = tq.KVPages.over(said["tables"], said["lens"], said["refs"])
    if s["op"] == "fork":
        rows.fork(s["src"], s["dst"], cache)
    elif s["op"] == "resize":
        rows.resize(s["up"], cache)
        rows.resize(s["down"], cache)
    else:
        said["live"] = rows.compact(cache)
    return said


# -------------------------------------------------------------------- work
def _seen_pairs(n, nk):
    """Pairs (query, key) of a row of n queries, the last ones of nk keys."""
    full = min(n, nk)
    return full * nk - full * (full - 1) // 2


def work(case):
    lens = _lens(case)
    if case["op"] == "prompt":
        keys, h, hk, d = _key_lens(case, lens), case["heads"], case["kv_heads"], case["d"]
        return {"bytes": 2 * d * (2 * h * sum(lens) + 2 * hk * sum(keys)) + 4 * h * sum(lens),
                "flops": 4 * d * h * sum(_seen_pairs(n, nk) for n, nk in zip(lens, keys))}
    if case["op"] == "append":
        news = _news(case, lens)
        blocks = sum((n - 1) // BLOCK - (n - m) // BLOCK + 1 for n, m in zip(lens, news) if m)
        hd = case["kv_heads"] * case["d"]
        return {"bytes": sum(news) * 2 * hd * 3 + blocks * case["kv_heads"] * 2 * 8, "flops": sum(news) * 2 * hd * 4}
    if case["op"] == "attend":
        news, h, hk, d = _news(case, lens), case["heads"], case["kv_heads"], case["d"]
        return {"bytes": sum(lens) * hk * (2 * d + 8 / BLOCK) + sum(news) * h * (4 * d + 4),
                "flops": 4 * d * h * sum(_seen_pairs(m, n) for m, n in zip(news, lens))}
    page = case["layers"] * case["kv_heads"] * (2 * PAGE * case["d"] + 2 * 4 * (PAGE // BLOCK))
    rows, pages = len(lens), sum(-(-n // PAGE) for n in lens)
    if case["op"] == "fork":
        forked = sum(1 for n in lens if n % PAGE) * case["more"]
        return {"bytes": 2 * page * forked + 4 * pages * (1 + 3 * case["more"]), "flops": 0}
    if case["op"] == "resize":   # up and down: counts read twice, the pages between taken and given back
        return {"bytes": 2 * 4 * (case["pages"] + 3 * rows) + 4 * 4 * rows * case["more"] // PAGE, "flops": 0}
    live = min(case["pages"], int(0.75 * pages))   # every second row shares about half of its pages
    return {"bytes": 2 * page * live * (case["pages"] - live) // case["pages"] + 4 * (2 * pages + 2 * case["pages"]), "flops": 0}


# ----------------------------------------------------- results in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("prompt", "attend"):
        return _exact_attention(case, s)
    if case["op"] == "append":
        return _exact_append(case, s)
    return None   # whole numbers and moved data


def _exact_attention(case, s):
    lens = _lens(case)
    keys = _key_lens(case, lens) if case["op"] == "prompt" else lens
    news = lens if case["op"] == "prompt" else _news(case, lens)
    h, hk, d = case["heads"], case["kv_heads"], case["d"]
    out = torch.zeros(sum(news), h, d, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(news), h), -math.inf, dtype=torch.float64, device="cuda")
    t0 = k0 = 0
    for b, (n, nk) in enumerate(zip(news, keys)):
        if case["op"] == "prompt":
            k, v = s["k"][k0:k0 + nk].double(), s["v"][k0:k0 + nk].double()
        else:
            held = s["tables"][b, :-(-nk // PAGE)].tolist()
            k = torch.cat([s["k"][0, p].double().reshape(hk, 4, BLOCK, d) * s["k_scale"][0, p].double()[:, :, None, None] for p in held]
                          or [torch.zeros(0, 4, BLOCK, d, dtype=torch.float64, device="cuda")])
            k = k.reshape(len(held), hk, PAGE, d).transpose(1, 2).reshape(-1, hk, d)[:nk]
            v = torch.cat([s["v"][0, p].double() * s["v_scale"][0, p].double()[:, :, None, None] for p in held]
                          or [torch.zeros(0, 4, d, BLOCK, dtype=torch.float64, device="cuda")])
            v = v.reshape(len(held), hk, 4, d, BLOCK).permute(0, 2, 4, 1, 3).reshape(-1, hk, d)[:nk]
        for i in range(0, n, 1024):
            m = min(1024, n - i)
            first = nk - n + i           # position of this part's first query
            see = min(nk, max(0, first + m))
            if see == 0:
                continue
            hidden = torch.arange(see, device="cuda")[None, :] > first + torch.arange(m, device="cuda")[:, None]
            for j in range(h):
                x = s["q"][t0 + i:t0 + i + m, j].double() @ k[:see, j // (h // hk)].T / math.sqrt(d)
                x[hidden] = -math.inf
                z = torch.logsumexp(x, -1)
                lse[t0 + i:t0 + i + m, j] = z
                out[t0 + i:t0 + i + m, j] = torch.where(z[:, None] > -math.inf, torch.exp(x - z[:, None]), 0.0) @ v[:see, j // (h // hk)]
        t0, k0 = t0 + n, k0 + nk
    return {"out": out, "lse": lse}


def _e4m3(x):
    """The nearest e4m3 value, ties to even mantissas (|x| <= 448)."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (x / step).round() * step


def _exact_append(case, s):
    lens, top = _lens(case), QMAX[case["kv"]]
    whole = case["kv"] == "int8"
    got = {m: s[m].double() for m in ("k", "v", "k_scale", "v_scale")}
    pages, hk, d = s["k"].shape[1], case["kv_heads"], case["d"]
    got["k"] = got["k"].view(1, pages, hk, 4, BLOCK, d)
    t0, tables = 0, s["tables"].tolist()
    for b, (n, m) in enumerate(zip(lens, _news(case, lens))):
        at = n - m
        while at < n:
            blk, to = at // BLOCK, min(n, (at // BLOCK + 1) * BLOCK)
            page, sub, c, u = tables[b][blk // 4], blk % 4, at % BLOCK, t0 + at - (n - m)
            for store, scales, new in (("k", "k_scale", "new_k"), ("v", "v_scale", "new_v")):
                x = s[new][u:u + to - at].double().transpose(0, 1)             # heads, tokens, d
                amax = x.abs().amax((1, 2))
                s0 = got[scales][0, page, :, sub] if c else torch.zeros_like(amax)
                s1 = torch.maximum(s0, torch.where(amax < TINY, 0.0, amax / top))
                z = got[store][0, page, :, sub] if store == "k" else got[store][0, page, :, sub].transpose(1, 2)
                z = z.clone() if c else torch.zeros_like(z)
                z = z * (s0 / s1)[:, None, None]
                z[:, c:c + to - at] = x / s1[:, None, None]
                z = torch.nan_to_num(z).clamp(-top, top)
                z = z.round() if whole else _e4m3(z)
                got[store][0, page, :, sub] = z if store == "k" else z.transpose(1, 2)
                got[scales][0, page, :, sub] = s1
            at = to
        t0 += m
    if whole:
        got["k"] = got["v"] = None
    else:
        got["k"] = got["k"].view(1, pages, hk, PAGE, d)
    return got
