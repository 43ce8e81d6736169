"""The paged token cache, operator by operator: what it computes, its plain form, and the calls a program makes.

Episodes of unlike length, and several answers or rollouts that go on from one history, share a pool of pages of bfloat16 rows for each
layer.  One table for all layers says which page holds an item's rows; a page may be held by several items.  Four operators work on it:

append     queries and keys rotated by their positions on one or three axes (time, row, column); keys and values into their rows' pages.
attention  softmax(scale q k) v of new rows over the whole history, causal, some keys masked: one token or a whole prompt.
step       items go on from other items' rows (forks), give rows up, and get pages for new ones: the free pages of lowest number, items
           in order.  Of a partly filled page that several items are about to write all but the last get copies, in every layer.  Where
           pages run out, an item is granted fewer rows.
compact    live pages move, in every layer, to the lowest numbers: the k-th live page behind the end to the k-th free page before it.

`run` computes them with elementary torch operations, or with `own` set through the package's calls.
"""
import math

import torch

own = False

# (query heads, key-value heads, head_dim, rotary pairs per axis): the layer of the episode benchmark, the toy layer of the tests, and
# other groupings that the layer kernels are built for
SHAPES = {
    "qwen": (28, 4, 128, (16, 24, 24)),
    "toy": (4, 4, 64, (8, 8, 16)),
    "mha": (4, 4, 128, (16, 24, 24)),
    "group4": (32, 8, 128, (16, 24, 24)),
    "group2": (8, 4, 64, (8, 8, 16)),
}
THETA = 1e6
TILE = 8            # rows of a page whose values lie together, by columns


def listed():
    return [
        # the token of an answer after one episode's frame: 128 text rows and a window of 8 frames of 256 held
        dict(name="attn token b1", op="attention", shape="qwen", B=1, n=1, lo=2176, hi=2176, page=64, shared=0, ragged=False, mask=False),
        # tokens of eight episodes of hundreds of frames
        dict(name="attn token long", op="attention", shape="qwen", B=8, n=1, lo=40001, hi=65535, page=64, shared=0, ragged=False, mask=False),
        # tokens of sixteen answers that go on from one history, in small pages, some rows masked
        dict(name="attn token forked", op="attention", shape="qwen", B=16, n=1, lo=2200, hi=2300, page=16, shared=2176, ragged=False, mask=True),
        # the 256 tokens of a new frame over seven frames and the text
        dict(name="attn frame b1", op="attention", shape="qwen", B=1, n=256, lo=1920, hi=1920, page=64, shared=0, ragged=False, mask=False),
        # frames of 1024 tokens of sixteen episodes, each with its own number of tokens and history
        dict(name="attn frames b16", op="attention", shape="qwen", B=16, n=1024, lo=2200, hi=3199, page=128, shared=0, ragged=True, mask=False),
        # a long prompt into an empty cache
        dict(name="attn prompt 8192", op="attention", shape="qwen", B=1, n=8192, lo=0, hi=0, page=64, shared=0, ragged=False, mask=False),
        # one token each of 64 episodes
        dict(name="append token b64", op="append", shape="qwen", B=64, n=1, lo=2000, hi=4100, page=64, ragged=False, axes=3),
        # a long prompt
        dict(name="append prompt 8192", op="append", shape="qwen", B=1, n=8192, lo=0, hi=0, page=64, ragged=False, axes=3),
        # pages for one answer's next token, in all layers' caches
        dict(name="step token b1", op="step", shape="qwen", B=1, fork=1, layers=28, n=1, lo=2176, hi=2176, page=64, spare=4, ragged=False),
        # sixteen answers each from the best of its four: 28 layers' partly filled pages copied
        dict(name="step fork b16", op="step", shape="qwen", B=16, fork=4, layers=28, n=8, lo=2205, hi=2230, page=64, spare=8, ragged=True),
        # three of six short episodes end, their pages are closed up, three others begin: the toy layer's caches
        dict(name="compact toy", op="compact", shape="toy", B=6, layers=2, lo=40, hi=100, page=16, spare=3),
        # eight of sixteen episodes of a thousand rows, 28 layers
        dict(name="compact b16", op="compact", shape="qwen", B=16, layers=28, lo=900, hi=1200, page=64, spare=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _most(op, key):
    return max(work(c)[key] for c in listed() if c["op"] == op)


def draw(rng):
    op = rng.choice(["attention", "attention", "append", "step", "compact"])
    shape, page = rng.choice(list(SHAPES)), rng.choice([16, 32, 64, 128, 256])
    while True:
        if op == "attention":
            # single tokens, a few rows, or a prompt, over histories of any length, their first rows shared or not
            n = rng.choice([1, _log(rng, 2, 16), _log(rng, 17, 8192)])
            B, hi = _log(rng, 1, 64), _log(rng, 1, 65000) if n < 17 else rng.choice([0, _log(rng, 1, 8000)])
            lo = int(hi * rng.uniform(0.3, 1.0))
            c = dict(op=op, shape=shape, B=B, n=n, lo=lo, hi=hi, page=page, shared=rng.choice([0, int(lo * rng.uniform(0.2, 1.0))]),
                     ragged=n > 1 and rng.random() < 0.5, mask=rng.random() < 0.3)
            square = B * SHAPES[shape][0] * n * (hi + n)   # what the plain form writes down
            rows = B * (hi + n) * SHAPES[shape][1] * SHAPES[shape][2]
            if work(c)["flops"] > _most(op, "flops") or square > 16 * 28 * 1024 * 4224 or rows > 8 * 65600 * 4 * 128:
                continue
        elif op == "append":
            B = _log(rng, 1, 64)
            n = rng.choice([1, _log(rng, 1, max(2, 8192 // B))])
            hi = rng.randint(0, 5000)
            c = dict(op=op, shape=shape, B=B, n=n, lo=int(hi * rng.uniform(0.2, 1.0)), hi=hi, page=page, ragged=n > 1 and rng.random() < 0.5,
                     axes=rng.choice([1, 3]))
        elif op == "step":
            fork = rng.choice([1, 2, 3, 4, 8])
            B, hi = fork * _log(rng, 1, 16), _log(rng, 1, 4000)
            c = dict(op=op, shape=shape, B=B, fork=fork, layers=_log(rng, 1, 28), n=_log(rng, 1, 300), lo=int(hi * rng.uniform(0.2, 1.0)),
                     hi=hi, page=page, spare=rng.choice([8, 2, -5]), ragged=rng.random() < 0.5)
        else:
            B, hi = 2 * _log(rng, 1, 16), _log(rng, 16, 4000)
            c = dict(op=op, shape=shape, B=B, layers=_log(rng, 1, 28), lo=int(hi * rng.uniform(0.3, 1.0)), hi=hi, page=page,
                     spare=rng.randint(0, 20))
        if op in ("step", "compact"):
            pages = _pages(c)
            H, KV, D, _ = SHAPES[shape]
            if pages * page * KV * D * c["layers"] > 600 * 64 * 4 * 128 * 28 // 2:
                continue
        if work(c)["bytes"] <= _most(op, "bytes"):
            return c


def _up(x, m):
    return (x + m - 1) // m


def _lens(c):
    """Rows held and rows new of each item: spread over the case's range; a ragged batch has items with fewer new rows, one with none.
    The items of a fork are as long as their first one, and in a compaction an item that ends as long as the one that takes its place."""
    B, f = c["B"], 2 if c["op"] == "compact" else c.get("fork", 1)
    held = [c["hi"] - (c["hi"] - c["lo"]) * (b // f) // max(1, B // f - 1) for b in range(B)]
    n = c.get("n", 0)
    new = [0 if c.get("ragged") and b % 5 == 3 else n - (b * n) // (3 * B) if c.get("ragged") else n for b in range(B)]
    return held, new


def _table_width(c):
    return _up(c["hi"] + c.get("n", 0), c["page"]) + 3


def _pages(c):
    """Pages of a pool: what the items need, and some to spare (step: or too few)."""
    held, new = _lens(c)
    R = c["page"]
    if c["op"] == "step":
        f = c["fork"]
        need = sum(_up(held[b], R) for b in range(0, c["B"], f))
        base = need
        for b in range(c["B"]):
            need += _up(held[b] + new[b], R) - _up(held[b], R) + (held[b] % R > 0 and new[b] > 0)
        return max(base + 1, need + c["spare"])
    shared = c.get("shared", 0) // R
    return shared + sum(_up(h + m, R) - shared for h, m in zip(held, new)) + c.get("spare", 5)


def _copies(c):
    """Rows copied by a step: of a partly filled page's writers all but the last, all of them if another item holds it besides."""
    held, new = _lens(c)
    R, f, rows = c["page"], c["fork"], 0
    for g in range(0, c["B"], f):
        writers = sum(m > 0 for m in new[g:g + f])
        if held[g] % R and f > 1:
            rows += min(writers, f - 1) * _up(held[g] % R, TILE) * TILE
    return rows


def _moves(c):
    """Pages that a compaction moves once the even items' pages, the lowest ones, are free."""
    held, _ = _lens(c)
    even = sum(_up(h, c["page"]) for h in held[::2])
    odd = sum(_up(h, c["page"]) for h in held[1::2])
    return min(even, odd)


def work(case):
    H, KV, D, _ = SHAPES[case["shape"]]
    held, new = _lens(case)
    row = 4 * KV * D                                            # a cached row of keys and values
    ints = 4 * case["B"] * (_table_width(case) + 3)
    if case["op"] == "append":
        return {"bytes": sum(new) * (4 * H * D + 2 * row) + 4 * sum(new), "flops": sum(new) * 6.0 * (H + KV) * D}
    if case["op"] == "attention":
        shared = case["shared"] // case["page"] * case["page"]
        live = [h + m - shared for h, m in zip(held, new) if m]
        seen = sum(live) + (shared if live else 0)
        pairs = sum(m * h + m * (m + 1) // 2 for h, m in zip(held, new))
        masks = sum(h + m for h, m in zip(held, new)) if case["mask"] else 0
        return {"bytes": seen * row + sum(new) * 4 * H * D + masks + ints, "flops": 4.0 * H * D * pairs}
    if case["op"] == "step":
        return {"bytes": 2 * case["layers"] * row * _copies(case) + 2 * ints + 4 * _pages(case), "flops": 0.0}
    return {"bytes": 2 * case["layers"] * row * case["page"] * _moves(case) + 4 * ints + 8 * _pages(case), "flops": 0.0}


# ---------------------------------------------------------------------------------------------- state
def prepare(case, seed):
    H, KV, D, section = SHAPES[case["shape"]]
    g = torch.Generator("cuda").manual_seed(seed)
    B, R, M, P = case["B"], case["page"], _table_width(case), _pages(case)
    lens, news = _lens(case)
    held, new = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (lens, news))
    s = dict(case, H=H, KV=KV, D=D, M=M, P=P, held=held, new=new)

    # which page holds what: numbers in no order, as after many episodes (compaction: the even items' first)
    order = torch.randperm(P, generator=torch.Generator().manual_seed(seed)).tolist()
    if case["op"] == "compact":
        order = sorted(order)
    table, taken = [[-1] * M for _ in range(B)], 0
    first = [] if case.get("shared", 0) < R else order[:case["shared"] // R]
    taken = len(first)
    for b in list(range(0, B, 2)) + list(range(1, B, 2)) if case["op"] == "compact" else range(B):
        if b % case.get("fork", 1):
            continue                                            # the others of a fork take its pages over
        rows = lens[b] + (news[b] if case["op"] in ("attention", "append") else 0)
        own_pages = _up(rows, R) - len(first)
        table[b][:len(first) + own_pages] = first + order[taken:taken + own_pages]
        taken += own_pages
    refs = [0] * P
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] += 1
    # the tables, rounded up to whole groups of four numbers, and the number of items that hold each page
    flat = [p for row in table for p in row]
    s["state"] = torch.tensor(flat + [0] * (-len(flat) % 4) + refs, dtype=torch.int32, device="cuda")
    s["table"] = s["state"][:B * M].view(B, M)
    s["refs"] = s["state"][-P:]

    s["k"], s["v"] = [], []
    for _ in range(case.get("layers", 1)):
        for name, shape in (("k", (P, KV, R, D)), ("v", (P, KV, R // TILE, D, TILE))):
            x = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
            # rows are not all of one size
            x *= (torch.rand(P, KV, 1, *[1] * (len(shape) - 3), device="cuda", generator=g) * 1.5 + 0.5).bfloat16()
            s[name].append(x)
    if case["op"] == "append":
        n = case["n"]
        # one projection's output: the rows q | k | v of each token
        s["rows"] = torch.randn(B, n, (H + 2 * KV) * D, device="cuda", generator=g).mul_(1.5).bfloat16()
        # a token's place in time and on the frame's grid of 16 x 16
        t = held[:, None] + torch.arange(n, dtype=torch.int32, device="cuda")
        s["pos"] = torch.stack([t // 16 * 16, t // 16 * 16 + t // 16 % 16, t // 16 * 16 + t % 16]).contiguous() if case["axes"] == 3 else t.contiguous()
        s["section"] = section if case["axes"] == 3 else (0, 0, 0)
        s["q_out"] = torch.zeros(B, n, H, D, dtype=torch.bfloat16, device="cuda")
    elif case["op"] == "attention":
        n = case["n"]
        s["q"] = torch.randn(B, n, H, D, device="cuda", generator=g).mul_(1.5).bfloat16()
        s["out"] = torch.zeros(B, n, H, D, dtype=torch.bfloat16, device="cuda")
        if case["mask"]:
            # a tenth of the keys dropped, and the first keys of every other item padded away
            m = torch.rand(B, M * R, device="cuda", generator=g) > 0.1
            pad = (held // 3 * (torch.arange(B, device="cuda") % 2))[:, None]
            s["key_mask"] = (m & (torch.arange(M * R, device="cuda") >= pad)).to(torch.uint8)
    else:
        s["granted"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        b = torch.arange(B, dtype=torch.int32, device="cuda")
        if case["op"] == "step":
            s["src"] = b // case["fork"] * case["fork"] if case["fork"] > 1 else None
        else:
            even = b % 2 == 0
            pair = torch.where(even, b + 1, b - 1)
            s["zero"] = torch.zeros_like(held)
            s["stay"] = torch.where(even, 0, held)              # the even items end
            s["swap"] = pair                                    # the odd ones' rows become theirs,
            s["taken"] = torch.where(even, held[pair.long()], 0)
            s["begin"] = torch.where(even, 0, held[pair.long()])    # and the odd ones begin anew
            s["n"] = case["hi"]
            s["live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:
        import paper_2604_24391_amd as fc
        s["fc"] = fc
        s["ctx"] = _context(fc)
        pages = fc.PageState(s["state"], B, M, P)
        s["caches"] = [fc.PCache(k, v, pages) for k, v in zip(s["k"], s["v"])]
        if case["op"] == "append":
            s["rope"] = fc.RopeAxes(THETA, s["section"])
    return s


_ctx = []


def _context(fc):
    """One context for the process, as a program keeps it, sized as the episode benchmark's."""
    if not _ctx:
        _ctx.append(fc.Context(fc.Caps(max_batch=64, max_tokens=256, max_seq=2176)))
    return _ctx[0]


# ---------------------------------------------------------------------------------------------- append
def _rotate(x, cos, sin):
    """Pairs (i, i + D / 2) of the last axis turned by their token's angles."""
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _append(s):
    B, n, H, KV, D, R, M = s["B"], s["n"], s["H"], s["KV"], s["D"], s["page"], s["M"]
    pair = torch.arange(D // 2, device="cuda")
    pos = s["pos"].view(-1, B, n)
    sec = s["section"]
    axis = (pair >= sec[0]).long() + (pair >= sec[0] + sec[1]).long() if sum(sec) else pair * 0
    angle = pos.double().index_select(0, axis).permute(1, 2, 0) * THETA ** (-2.0 * pair.double() / D)
    cos, sin = (f(angle).float()[:, :, None] for f in (torch.cos, torch.sin))
    q, k, v = s["rows"].view(B, n, H + 2 * KV, D).float().split([H, KV, KV], 2)
    live = torch.arange(n, device="cuda") < s["new"][:, None]
    s["q_out"].copy_(torch.where(live[..., None, None], _rotate(q, cos, sin).bfloat16(), s["q_out"]))
    # a token without a row of its own writes the first token's there is, again
    row = s["held"][:, None].long() + torch.arange(n, device="cuda")
    at = torch.where(live, torch.arange(B * n, device="cuda").view(B, n), int(s["B"] * n)).amin()
    pick = torch.where(live, torch.arange(B * n, device="cuda").view(B, n), at).flatten()
    row = row.flatten()[pick]
    page = s["table"].long()[pick // n, row // R]
    r = row % R
    s["k"][0][page, :, r] = _rotate(k, cos, sin).bfloat16().view(B * n, KV, D)[pick]
    s["v"][0][page, :, r // TILE, :, r % TILE] = v.bfloat16().reshape(B * n, KV, D)[pick]


# ---------------------------------------------------------------------------------------------- attention
def _attention(s):
    B, n, H, KV, D, R = s["B"], s["n"], s["H"], s["KV"], s["D"], s["page"]
    G, L = H // KV, s["hi"] + n
    there = s["table"][:, :_up(L, R)].clamp(min=0).long()
    k = s["k"][0][there].permute(0, 2, 1, 3, 4).reshape(B, KV, -1, D)[:, :, :L].float()
    v = s["v"][0][there].permute(0, 2, 1, 3, 5, 4).reshape(B, KV, -1, D)[:, :, :L].float()
    q = s["q"].float().view(B, n, KV, G, D).permute(0, 2, 1, 3, 4).reshape(B, KV, n * G, D)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(1 / math.sqrt(D)).view(B, KV, n, G, L)
    j, i = torch.arange(L, device="cuda"), torch.arange(n, device="cuda")
    seen = (j <= s["held"][:, None, None] + i[:, None]) & (i < s["new"][:, None])[..., None]
    if s["mask"]:
        seen = seen & (s["key_mask"][:, None, :L] != 0)
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    x = x.view(B, KV, n * G, L)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    x.div_(torch.where(total == 0, 1.0, total))
    o = torch.matmul(x, v).view(B, KV, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, H, D).bfloat16()
    s["out"].copy_(torch.where((i < s["new"][:, None])[..., None, None], o, s["out"]))


# ---------------------------------------------------------------------------------------------- step, compact
def _count(table, P):
    """Items that hold each page."""
    return torch.zeros(P + 1, dtype=torch.int32, device="cuda").index_add_(
        0, torch.where(table >= 0, table, P).flatten().long(), torch.ones(table.numel(), dtype=torch.int32, device="cuda"))[:P]


def _step(s, src, held, new, n):
    B, M, P, R = s["B"], s["M"], s["P"], s["page"]
    b, i = torch.arange(B, device="cuda"), torch.arange(M, device="cuda")
    kept = (held + R - 1) // R
    t = s["table"] if src is None else s["table"][src.long()]
    t = torch.where(i < kept[:, None], t, -1)
    refs = _count(t, P)
    m = torch.minimum(new.clamp(0, n), M * R - held)
    tail = (kept - 1).clamp(min=0).long()[:, None]
    page = t.gather(1, tail)[:, 0].long()
    writes = (held % R > 0) & (m > 0)
    shared = writes & (refs[page.clamp(min=0)] > 1)
    # the writers of one page before this one
    rank = ((page[:, None] == page) & shared[:, None] & shared & (b < b[:, None])).sum(1)
    copy = shared & (rank < refs[page.clamp(min=0)] - 1)
    more = (held + m + R - 1) // R - kept
    need = copy + more
    off = need.cumsum(0) - need
    free = torch.sort(torch.where(refs == 0, torch.arange(P, device="cuda"), P)).values      # P: none
    got = torch.minimum((((refs == 0).sum() - off).clamp(min=0)), need)
    copied = copy & (got > 0)
    fresh = free[off.clamp(max=P - 1)]
    # new pages go behind the kept ones, a copy in the last one's place
    j = i - kept[:, None] + copy[:, None].long()
    t = torch.where((i >= kept[:, None]) & (j < got[:, None]), free[(off[:, None] + j).clamp(0, P - 1)].int(), t)
    t = torch.where((i == tail) & copied[:, None], fresh[:, None].int(), t)
    s["table"].copy_(t)
    refs = _count(t, P)
    s["refs"].copy_(refs)
    stuck = shared & ~copied & (refs[page.clamp(min=0)] > 1)
    s["granted"].copy_(torch.where(stuck, 0, torch.minimum(m, (kept + got - copied.int()) * R - held)))
    # an item without a copy does the first one's again; without any, page 0 stays as it is
    pick = torch.where(copied, b, copied.int().argmax())
    some = copied.any()
    rows = torch.where(some, held[pick] % R, 0)
    tiles = (rows + TILE - 1) // TILE
    a, z = torch.where(some, page[pick], 0), torch.where(some, fresh[pick], 0)
    r = torch.arange(R // TILE, device="cuda") < tiles[:, None]
    for k, v in zip(s["k"], s["v"]):
        k, v = (x.view(P, s["KV"], R // TILE, -1) for x in (k, v))
        for x in (k, v):
            x[z] = torch.where(r[:, None, :, None], x[a], x[z])


def _compact(s):
    P, refs = s["P"], s["refs"]
    p = torch.arange(P, device="cuda")
    live = refs > 0
    L = live.sum()
    # the k-th live page behind the end and the k-th free page before it, P where there is none
    high = torch.sort(torch.where(live & (p >= L), p, P)).values
    low = torch.sort(torch.where(~live & (p < L), p, P)).values
    to = torch.arange(P + 1, device="cuda").scatter_(0, high, low)[:P]
    come = torch.arange(P + 1, device="cuda").scatter_(0, low, high)[:P]
    for k, v in zip(s["k"], s["v"]):
        k.copy_(k[come])
        v.copy_(v[come])
    s["refs"].copy_(torch.where(p < L, refs[come], 0))
    t = s["table"]
    t.copy_(torch.where(t >= 0, to[t.clamp(min=0).long()].int(), t))
    s["live"].copy_(L.int().view(1))


def run(s):
    op = s["op"]
    if op == "append":
        if own:
            H, KV, D = s["H"], s["KV"], s["D"]
            q, k, v = s["rows"].view(s["B"], s["n"], H + 2 * KV, D).split([H, KV, KV], 2)
            s["fc"].fc_pcache_append(s["ctx"], s["caches"][0], s["rope"], q, k, v, s["pos"], s["held"], s["new"], s["q_out"])
        else:
            _append(s)
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if op == "attention":
        if own:
            s["fc"].fc_pcache_attention(s["ctx"], s["caches"][0], s["q"], s["held"], s["new"], s["out"], key_mask=s.get("key_mask"))
        else:
            _attention(s)
        return s["out"]
    if op == "step":
        if own:
            s["fc"].fc_pcache_step(s["ctx"], s["caches"], s["held"], s["new"], s["n"], s["granted"], src=s["src"])
        else:
            _step(s, s["src"], s["held"], s["new"], s["n"])
        return {"state": s["state"], "granted": s["granted"], "k": s["k"], "v": s["v"]}
    # the even items end, the pool is closed up, the odd ones' rows become theirs and the odd ones begin anew, at the pool's end
    if own:
        s["fc"].fc_pcache_step(s["ctx"], s["caches"], s["stay"], s["zero"], s["n"], s["granted"])
        s["fc"].fc_pcache_compact(s["ctx"], s["caches"], s["live"])
        s["fc"].fc_pcache_step(s["ctx"], s["caches"], s["taken"], s["begin"], s["n"], s["granted"], src=s["swap"])
    else:
        _step(s, None, s["stay"], s["zero"], s["n"])
        _compact(s)
        _step(s, s["swap"], s["taken"], s["begin"], s["n"])
    return {"state": s["state"], "granted": s["granted"], "live": s["live"], "k": s["k"], "v": s["v"]}


# ---------------------------------------------------------------------------------------------- in 64 bits
def _rows64(s, name, b, L):
    """Item b's first L rows [L, KV, D]."""
    R = s["page"]
    x = s[name][0][s["table"][b, :_up(L, R)].long()].double()
    x = x.permute(0, 2, 4, 1, 3).flatten(1, 2) if name == "v" else x.transpose(1, 2)        # [pages, R, KV, D]
    return x.flatten(0, 1)[:L]


def _exact_append(s):
    H, KV, D, n, B, R = s["H"], s["KV"], s["D"], s["n"], s["B"], s["page"]
    held, new = _lens(s)
    sec = list(s["section"]) if sum(s["section"]) else [D // 2, 0, 0]
    pos = s["pos"].double().view(-1, B, n)
    turn = torch.cat([pos[min(a, pos.shape[0] - 1)][..., None].expand(-1, -1, m) for a, m in enumerate(sec)], -1)
    z = torch.polar(torch.ones_like(turn), turn * torch.pow(torch.tensor(THETA, dtype=torch.float64), -torch.arange(0, D, 2) / D).cuda())[:, :, None]
    rows = s["rows"].double().view(B, n, -1, D)
    q = torch.zeros(B, n, H, D, dtype=torch.float64, device="cuda")
    k, v = s["k"][0].double(), s["v"][0].double()
    table = s["table"].tolist()
    for b in range(B):
        m, h = new[b], held[b]
        w = torch.complex(rows[b, :m, :H + KV, :D // 2], rows[b, :m, :H + KV, D // 2:]) * z[b, :m]
        w = torch.cat([w.real, w.imag], -1)
        q[b, :m] = w[:, :H]
        for i0 in range(h // R, _up(h + m, R)):
            lo, hi = max(h, i0 * R), min(h + m, i0 * R + R)
            if hi <= lo:
                continue
            k[table[b][i0], :, lo - i0 * R:hi - i0 * R] = w[lo - h:hi - h, H:].transpose(0, 1)
            by_rows = v[table[b][i0]].transpose(-1, -2).reshape(KV, R, D)
            by_rows[:, lo - i0 * R:hi - i0 * R] = rows[b, lo - h:hi - h, H + KV:].transpose(0, 1)
            v[table[b][i0]] = by_rows.view(KV, R // TILE, TILE, D).transpose(-1, -2)
    return {"q": q, "k": [k], "v": [v]}


def _exact_attention(s):
    H, KV, D, n, B = s["H"], s["KV"], s["D"], s["n"], s["B"]
    held, new = _lens(s)
    out = torch.zeros(B, n, H, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        m, L = new[b], held[b] + new[b]
        if not m:
            continue
        k, v = (_rows64(s, x, b, L) for x in "kv")
        hidden = torch.arange(L, device="cuda") > held[b] + torch.arange(m, device="cuda")[:, None]
        if s["mask"]:
            hidden = hidden | (s["key_mask"][b, :L] == 0)
        for h in range(H):
            x = (s["q"][b, :m, h].double() @ k[:, h // (H // KV)].t()) / D ** 0.5
            p = torch.softmax(x.masked_fill_(hidden, -math.inf), -1).nan_to_num_(0.0)     # no key seen: no weight
            out[b, :m, h] = p @ v[:, h // (H // KV)]
    return out


class _Pages:
    """Tables and pools one item and one page after the other."""

    def __init__(self, s):
        self.R, self.P = s["page"], s["P"]
        self.t = [[p for p in row if p >= 0] for row in s["table"].tolist()]
        self.pools = [(x, name) for name in "kv" for x in s[name]]
        self.new = {name: [x.double() for x in s[name]] for name in "kv"}

    def copy(self, src, dst, rows):
        for name in "kv":
            for x in self.new[name]:
                if name == "k":
                    x[dst, :, :rows] = x[src, :, :rows].clone()
                else:
                    x[dst, :, :rows // TILE] = x[src, :, :rows // TILE].clone()

    def step(self, src, held, new):
        R = self.R
        self.t = [list(self.t[a][:_up(h, R)]) for a, h in zip(src, held)]
        holds = lambda p: sum(row.count(p) for row in self.t)
        free = sorted(set(range(self.P)) - {p for row in self.t for p in row})
        for b, (h, m) in enumerate(zip(held, new)):
            row = self.t[b]
            if m and h % R and holds(row[-1]) > 1:
                if not free:
                    continue
                to = free.pop(0)
                self.copy(row[-1], to, _up(h % R, TILE) * TILE)
                row[-1] = to
            for _ in range(_up(h + m, R) - _up(h, R)):
                if free:
                    row.append(free.pop(0))

    def compact(self):
        live = sorted({p for row in self.t for p in row})
        high = [p for p in live if p >= len(live)]
        low = sorted(set(range(len(live))) - set(live))
        for a, z in zip(high, low):
            self.copy(a, z, self.R)
        to = dict(zip(high, low))
        self.t = [[to.get(p, p) for p in row] for row in self.t]


def _exact_pages(s):
    held, new = _lens(s)
    p = _Pages(s)
    if s["op"] == "step":
        p.step([b // s["fork"] * s["fork"] for b in range(s["B"])], held, new)
        return {"state": None, "granted": None, **p.new}
    ids = list(range(s["B"]))
    p.step(ids, s["stay"].tolist(), [0] * len(ids))
    p.compact()
    p.step(s["swap"].tolist(), s["taken"].tolist(), s["begin"].tolist())
    return {"state": None, "granted": None, "live": None, **p.new}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention}.get(case["op"], _exact_pages)(s)
