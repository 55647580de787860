"""The paged MXFP4 cache in use: what a speculative step asks of it beside its linear layers.

A cache holds keys and values as MXFP4 (E2M1 codes, one E8M0 scale byte per 32 elements along the head dimension) in
pages of `page` tokens: `kq`, `vq` uint8 [pages, heads, page, dim / 2], `ks`, `vs` uint8 [pages, heads, page, dim / 32].
Row b of `table` lists the pages of sequence b, `lens[b]` counts its tokens, the last ones of them new in this call;
`starts` says which rows of the packed tensors are whose (None: the same number each).

Kinds of cases:

- "append"  a step's keys and values, fresh from the qkv product, are rotated, cast and put into their pages, the
            queries rotated beside them; the new tokens are then read back as the values that they stand for;
- "attend"  queries against the cache: one token, a draft tree, a piece of a prompt, a whole prompt;
- "fork"    sequences are forked into drafts, which get pages for their next tokens (a shared last page is copied);
            the last tokens that the drafts share are read back, and the next pass begins by dropping the drafts;
- "accept"  a draft tree's accepted tokens are moved together, the rest is given back, the accepted ones are read back.

Sizes: the head layouts of the 7B- and 70B-shaped stacks of `synth.py` (32 and 32 heads, 64 and 8 heads of 128) and
generic ones beside them.
"""
import math

import torch

own = False
DEV = "cuda"

# (query heads, key/value heads, head dimension)
HEADS_7B, HEADS_70B = (32, 32, 128), (64, 8, 128)


def _heads(h):
    return {"hq": h[0], "hkv": h[1], "dim": h[2]}


def _append(name, heads, page, rows, low, high, new, ragged=False, rotary=None):
    return {"name": name, "kind": "append", **_heads(heads), "page": page, "rows": rows, "low": low, "high": high, "new": new,
            "ragged": ragged, "rotary": heads[2] if rotary is None else rotary}


def _attend(name, heads, page, rows, low, high, new, ragged=False, tree=False, window=0, lse=False):
    return {"name": name, "kind": "attend", **_heads(heads), "page": page, "rows": rows, "low": low, "high": high, "new": new,
            "ragged": ragged, "tree": tree, "window": window, "lse": lse}


def _pages(name, kind, groups, dim, page, rows, low, high, new, branches=0):
    return {"name": name, "kind": kind, "groups": groups, "dim": dim, "page": page, "rows": rows, "low": low, "high": high,
            "new": new, "branches": branches}


def listed():
    return [
        # drafting: one token of one sequence goes into the cache (the smallest call: latency)
        _append("append_draft", HEADS_7B, 16, 1, 701, 701, 1),
        # verifying: a few tokens each of 24 sequences, the drafts' lengths differ
        _append("append_verify", HEADS_70B, 32, 24, 90, 6000, 9, ragged=True),
        # the prompts of three requests, 12 thousand tokens together
        _append("append_prompt", HEADS_7B, 64, 3, 2400, 6200, 6200, ragged=True),
        # drafting: one token against a short conversation (latency)
        _attend("attend_draft", HEADS_7B, 16, 1, 701, 701, 1),
        # drafting on a long document: few rows, a long axis
        _attend("attend_long", HEADS_70B, 64, 1, 131071, 131071, 1),
        # a server's batch of one token each, conversations of very different lengths
        _attend("attend_batch", HEADS_70B, 16, 64, 500, 16384, 1),
        # verifying a draft tree of 8 nodes for 8 sequences
        _attend("attend_tree", HEADS_70B, 32, 8, 1200, 7000, 8, tree=True, lse=True),
        # pieces of prompts behind a cached prefix, small heads, a sliding window
        _attend("attend_piece", (16, 2, 64), 32, 3, 5000, 9001, 1003, ragged=True, window=4096),
        # a whole prompt: every token against those before it
        _attend("attend_prompt", HEADS_7B, 64, 1, 5001, 5001, 5001),
        # two drafts each of four conversations, one layer's cache
        _pages("fork_drafts", "fork", 32, 128, 16, 4, 300, 1100, 5, branches=2),
        # eight samples each of 24 long prompts, eight layers of 8 heads in one page
        _pages("fork_samples", "fork", 64, 128, 32, 24, 1500, 8000, 40, branches=8),
        # the accepted paths of 48 draft trees, eight layers of 8 heads in one page
        _pages("accept_trees", "accept", 64, 128, 32, 48, 400, 6000, 24),
    ]


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    def log(low, high):
        return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))

    most = 0.9 * _cost(next(c for c in listed() if c["name"] == "attend_prompt"))
    heads = rng.choice([HEADS_7B, HEADS_70B, (16, 2, 64), (8, 1, 256), (32, 8, 64), (20, 4, 96), (10, 5, 192)])
    page = rng.choice([16, 32, 64, 128])
    while True:
        kind = rng.choice(["append", "attend one", "attend one", "attend some", "attend many", "fork", "accept"])
        rows, high = log(1, 96), log(40, 100000)
        low = max(1, int(high * rng.choice([0.05, 0.4, 1.0])))
        if kind == "append":
            new = log(1, 6000)
            case = _append("", heads, page, rows, max(low, new), max(high, new), new, rng.random() < 0.5, heads[2] if rng.random() < 0.7 else 32)
        elif kind == "attend one":
            case = _attend("", heads, page, rows, low, high, 1, window=rng.choice([0, 0, 0, 1024]), lse=rng.random() < 0.3)
        elif kind == "attend some":
            new = rng.randint(2, 32)
            tree = rng.random() < 0.5
            case = _attend("", heads, page, rows, max(low, new), max(high, new), new, not tree and rng.random() < 0.5, tree, lse=rng.random() < 0.3)
        elif kind == "attend many":
            new = log(33, 8000)
            case = _attend("", heads, page, max(1, rows // 12), max(low, new), max(high, new), new, rng.random() < 0.5, window=rng.choice([0, 0, 777]))
        else:
            new = rng.randint(2, 60) if kind == "fork" else rng.randint(4, 60)
            high = max(2 * page, min(high, 20000))
            case = _pages("", kind, rng.choice([8, 24, 64]), rng.choice([64, 128, 256]), page, max(1, rows // 2), max(2 * page, min(low, high)), high, new, rng.randint(1, 6) if kind == "fork" else 0)
        del case["name"]
        # what the plain form has to hold at once, in values
        wide = case["rows"] * (case["high"] + page) * (case.get("hkv", 1) * case["dim"] + (case.get("hq", 0) * case["new"] if case["kind"] == "attend" else 0))
        if _cost(case) <= most and wide <= 3e9 and (case["kind"] in ("append", "attend") or case["rows"] * (1 + case["branches"]) * (case["high"] + 2 * page + 60) * case["groups"] * case["dim"] <= 2e10):
            return case


# ---- lengths: they follow from the case alone, the seed says which row has which ------------------------------------

def _lengths(case):
    """(tokens, new tokens) of each row, in an order that the seed then shuffles."""
    got = []
    for b in range(case["rows"]):
        n = case["new"] if not case.get("ragged") else 1 + (b * 2 + 1) * (case["new"] - 1) // (2 * case["rows"])
        length = int(round(case["low"] * (case["high"] / case["low"]) ** ((b + 0.5) / case["rows"])))
        got.append((max(length, n), n))
    return got


def work(case):
    d, lens = case["dim"], _lengths(case)
    token = 2 * (d // 2 + d // 32)                                  # bytes of one token of one head: key and value
    if case["kind"] == "append":
        t = sum(n for _, n in lens)
        qkv = t * (case["hq"] + 2 * case["hkv"]) * d * 2
        return {"bytes": qkv + t * case["hq"] * d * 2 + 4 * t * case["rotary"] + t * case["hkv"] * (2 * token + 4 * d), "flops": 0}
    if case["kind"] == "attend":
        seen, pairs, t = 0, 0, 0
        for length, n in lens:
            w = case["window"] or length
            seen += min(length, w + n - 1)
            if case["tree"]:                                        # half of the other new tokens, about
                pairs += n * (length - n) + n * (n + 1) // 2
            else:
                pairs += sum(min(w, length - n + i + 1) for i in range(n))
            t += n
        moved = seen * case["hkv"] * token + 4 * t * case["hq"] * d + (4 * t * case["hq"] if case["lse"] else 0)
        return {"bytes": moved, "flops": 4 * pairs * case["hq"] * d}
    each = case["groups"] * token
    if case["kind"] == "fork":
        rows = case["rows"] * case["branches"]
        tables = 8 * sum(case["branches"] * -(-(n + case["new"]) // case["page"]) for n, _ in lens)
        copied = 2 * each * sum(case["branches"] * (n % case["page"]) for n, _ in lens)
        back = rows * case["page"] * (each + case["groups"] * 4 * d)
        return {"bytes": tables + copied + back, "flops": 0}
    kept = sum(_kept(case, b) for b in range(case["rows"]))
    return {"bytes": kept * (3 * each + case["groups"] * 4 * d), "flops": 0}


def _kept(case, b):
    """How many nodes of row b's draft tree are accepted."""
    return 1 + b % max(1, case["new"] // 2)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _numbers(shape, gen, large=8.0):
    """Projected hidden states: normal values, a few large channels, BF16."""
    x = torch.randn(shape, generator=gen, device=DEV)
    x[..., :: 37] *= large
    return x.to(torch.bfloat16)


def _cache(pages, groups, page, dim, gen):
    """A cache in use: every page holds cast numbers (a stock of up to 512 pages' worth, dealt out at random)."""
    got = []
    for _ in range(2):
        stock = max(1, min(pages, 512, (1 << 26) // (groups * page * dim)))
        code, scale = _cast(_numbers((stock, groups, page, dim), gen, 3.0))
        pick = torch.randint(stock, (pages,), generator=gen, device=DEV)
        got += [code[pick], scale[pick]]
    return got


def _order(case, seed):
    gen = torch.Generator().manual_seed(seed)
    at = torch.randperm(case["rows"], generator=gen).tolist()
    every = _lengths(case)
    return [every[i] for i in at], gen


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    lens, host = _order(case, seed)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    page, d, rows = case["page"], case["dim"], case["rows"]
    s = {"case": case}
    if case["kind"] in ("append", "attend"):
        width = max(n for n, _ in lens) // page + 2
        table = torch.randperm(rows * width, generator=gen, device=DEV).to(torch.int32).view(rows, width)
        s["cache"] = _cache(rows * width, case["hkv"], page, d, gen)
        s["table"], s["lens"] = table, _int([n for n, _ in lens])
        news = [n for _, n in lens]
        total, s["most"] = sum(news), max(news)
        s["starts"] = _int([sum(news[:i]) for i in range(rows + 1)]) if case["ragged"] else None
        s["total"] = total
        hq, hkv = case["hq"], case["hkv"]
        if case["kind"] == "append":
            qkv = _numbers((total, (hq + 2 * hkv) * d), gen)
            half = case["rotary"] // 2
            turn = 10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
            angle = torch.arange(max(n for n, _ in lens) + page, device=DEV, dtype=torch.float64)[:, None] * turn
            s["rope"] = (angle.cos().float(), angle.sin().float())
            s["q"], s["k"], s["v"] = (x.view(total, -1, d) for x in qkv.split([hq * d, hkv * d, hkv * d], dim=1))
        else:
            qkv = _numbers((total, (hq + 2 * hkv) * d), gen, 2.0)
            s["q"] = qkv[:, : hq * d].view(total, hq, d)
            s["tree"] = _tree(rows, case["new"], host) if case["tree"] else None
        return s
    groups, add = case["groups"], case["new"]
    forks = case["branches"]
    every = [n for n, _ in lens] + [0] * (rows * forks)
    width = (max(every) + add) // page + 2
    table = torch.full((len(every), width), -1, dtype=torch.int32)
    used = sum(-(-n // page) for n in every)
    pages = used + sum(-(-(n + add) // page) - n // page + 1 for n in every[:rows] for _ in range(max(1, forks))) + 8
    at, order = 0, torch.randperm(pages, generator=host).to(torch.int32)
    for b, n in enumerate(every):
        mine = -(-n // page)
        table[b, :mine] = order[at: at + mine]
        at += mine
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[order[:used].long()] = 1
    bits = torch.zeros(-(-pages // 32) * 32, dtype=torch.int64)
    bits[:pages] = refs == 0
    words = (bits.view(-1, 32) << torch.arange(32)).sum(1)
    s["free"] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).to(DEV)
    s["refs"], s["table"], s["lens"] = refs.to(DEV), table.to(DEV), _int(every)
    s["cache"] = _cache(pages, groups, page, d, gen)
    if case["kind"] == "fork":
        s["src"] = _int([b for b in range(rows) for _ in range(forks)])
        s["dst"] = _int([rows + i for i in range(rows * forks)])
        s["none"], s["add"] = _int([0] * (rows * forks)), _int([add] * (rows * forks))
        s["before"] = _int([n for n, _ in lens for _ in range(forks)])
        s["starts"], s["first"], s["total"] = None, rows, page * rows * forks
    else:
        s["rows"], s["base"], s["add"] = _int(list(range(rows))), _int([n for n, _ in lens]), _int([add] * rows)
        counts = [_kept(case, b) for b in range(rows)]
        keep = [[0] + sorted((1 + torch.randperm(add - 1, generator=host)[: c - 1]).tolist()) + [0] * (add - c) for c in counts]
        s["keep"], s["counts"] = _int(keep), _int(counts)
        s["after"] = s["base"] + s["counts"]
        s["starts"] = _int([sum(counts[:i]) for i in range(rows + 1)])
        s["total"], s["first"] = sum(counts), 0
    return s


def _tree(rows, new, host):
    """Draft trees: node i's word has a bit for itself and for each node above it."""
    words = []
    for _ in range(rows):
        mine = []
        for i in range(new):
            above = mine[int(torch.randint(i, (1,), generator=host))] if i else 0
            mine.append(above | 1 << i)
        words += mine
    return torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device=DEV)


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _cast(x):
    """BF16 [..., dim] -> (codes of two elements a byte [..., dim / 2], scale bytes [..., dim / 32])."""
    v = x.unflatten(-1, (-1, 32))
    most = (v.view(torch.int16) & 0x7FFF).amax(-1).to(torch.int32)
    bad = most >= 0x7F80
    scale = ((most >> 7) - 2).clamp(min=0)
    y = v.float().abs() * torch.exp2(127.0 - scale)[..., None]
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    r = (torch.round(y / step) * step).clamp(max=6)
    code = torch.where(r < 2, r * 2, torch.where(r < 4, r + 2, r / 2 + 4)).to(torch.uint8)
    code = code + (v.view(torch.int16) < 0) * 8
    code = torch.where(bad[..., None], 0, code).flatten(-2).to(torch.uint8)
    return code[..., 0::2] + code[..., 1::2] * 16, torch.where(bad, 255, scale).to(torch.uint8)


def _values(code, scale):
    """The 32-bit values that codes [..., dim / 2] and scale bytes [..., dim / 32] stand for."""
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    both = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], dim=1)
    x = both[code.int()].flatten(-2).unflatten(-1, (-1, 32))
    factor = torch.exp2(scale.float() - 127).masked_fill(scale == 255, math.nan)
    return (x * factor[..., None]).flatten(-2)


def _new(s, lens=None):
    """(row, position, number) of each packed token: the last tokens of the rows from s["first"] on."""
    lens = (s["lens"] if lens is None else lens).long()
    rows = lens.numel()
    t = torch.arange(s["total"], device=DEV)
    if s["starts"] is None:
        n = s["total"] // rows
        row, i, n = t // n, t % n, n
    else:
        row = torch.searchsorted(s["starts"][1:].long(), t, right=True)
        n = (s["starts"][1:] - s["starts"][:-1]).long()[row]
        i = t - s["starts"].long()[row]
    return row, lens[row] - n + i, i


def _place(s, row, at):
    """Page and slot of position `at` of the rows from s["first"] on."""
    page = s["case"]["page"]
    return s["table"][s.get("first", 0):][row, at // page].long(), at % page


def _read(s, lens=None):
    row, at, _ = _new(s, lens)
    p, o = _place(s, row, at)
    kq, ks, vq, vs = (x[p, :, o] for x in s["cache"])
    return _values(kq, ks).to(torch.bfloat16), _values(vq, vs).to(torch.bfloat16)


def _rotate(x, cos, sin):
    half = cos.shape[1]
    cos, sin, x = cos[:, None], sin[:, None], x.float()
    a, b = x[..., :half], x[..., half: 2 * half]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], dim=-1).to(torch.bfloat16)


def _plain_append(s):
    row, at, _ = _new(s)
    cos, sin = (x[at] for x in s["rope"])
    p, o = _place(s, row, at)
    for x, code, scale in ((_rotate(s["k"], cos, sin), 0, 1), (s["v"], 2, 3)):
        c, e = _cast(x)
        s["cache"][code][p, :, o] = c
        s["cache"][scale][p, :, o] = e
    return [_rotate(s["q"], cos, sin), *_read(s)]


def _plain_attend(s):
    case, q = s["case"], s["q"]
    rows, n, hq, hkv, d = case["rows"], s["most"], case["hq"], case["hkv"], case["dim"]
    lens, pages = s["lens"].long(), s["table"].long()
    row, at, i = _new(s)
    k, v = (_values(*(x[pages].transpose(1, 2).flatten(2, 3) for x in s["cache"][j: j + 2])) for j in (0, 2))
    padded = torch.zeros((rows, n, hq, d), device=DEV)
    padded[row, i] = q.float()
    padded = padded.view(rows, n, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).flatten(2, 3)      # rows, hkv, (group, n), d
    scores = torch.matmul(padded, k.transpose(2, 3)).mul_(d ** -0.5).unflatten(2, (-1, n))
    j = torch.arange(k.shape[2], device=DEV)
    limit = torch.full((rows, n), -1, dtype=torch.int64, device=DEV)
    limit[row, i] = at
    seen = j <= limit[..., None]
    if case["window"]:
        seen &= j > limit[..., None] - case["window"]
    if case["tree"]:
        node = j - (lens - n)[:, None, None]
        word = s["tree"].view(rows, n, 1)
        seen = (node < 0) | ((node < n) & ((word >> node.clamp(0, n - 1)) & 1 == 1))
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    scores = scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.flatten(2, 3), v).unflatten(2, (-1, n)) / total
    out = torch.where(total > 0, out, 0.0)
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)[row, i].to(torch.bfloat16)
    if not case["lse"]:
        return [out]
    return [out, (top + total.log())[..., 0].permute(0, 3, 1, 2).flatten(2, 3)[row, i]]


def _counted(s, rows, low, high):
    """Whether entry w of each of these table rows lies in [low, high)."""
    w = torch.arange(s["table"].shape[1], device=DEV)
    return (w >= low[:, None]) & (w < high[:, None])


def _plain_release(s, rows, keep):
    page, rows = s["case"]["page"], rows.long()
    old = s["lens"][rows].long()
    gone = _counted(s, rows, (torch.minimum(old, keep.long()) + page - 1) // page, (old + page - 1) // page)
    entries = s["table"][rows].long()
    s["refs"].index_add_(0, torch.where(gone, entries, 0).flatten(), -gone.flatten().to(torch.int32))
    s["table"][rows] = torch.where(gone, -1, entries).to(torch.int32)
    s["lens"][rows] = torch.minimum(old, keep.long()).to(torch.int32)


def _plain_fork(s, src, dst):
    page, src, dst = s["case"]["page"], src.long(), dst.long()
    n = s["lens"][src].long()
    has = _counted(s, src, torch.zeros_like(n), (n + page - 1) // page)
    entries = s["table"][src].long()
    s["refs"].index_add_(0, torch.where(has, entries, 0).flatten(), has.flatten().to(torch.int32))
    s["table"][dst] = torch.where(has, entries, -1).to(torch.int32)
    s["lens"][dst] = n.to(torch.int32)


def _plain_extend(s, rows, add):
    page, rows = s["case"]["page"], rows.long()
    n, table = s["lens"][rows].long(), s["table"]
    last = (n // page).clamp(max=table.shape[1] - 1)
    mine = table[rows, last].long()                                  # the page that the next token goes into, if one is begun
    open_ = (n % page != 0) & (add > 0)
    same = (mine[:, None] == mine) & open_[:, None] & open_
    before = same.tril(-1).sum(1)                                    # rows in front of this one that leave the same page
    copies = open_ & (s["refs"][mine.clamp(min=0)] - before > 1)
    w = torch.arange(table.shape[1], device=DEV)
    wants = _counted(s, rows, (n + page - 1) // page, (n + add.long() + page - 1) // page) | (copies[:, None] & (w == last[:, None]))
    order = torch.sort((s["refs"] != 0).to(torch.uint8), stable=True).indices      # free pages first, in their order
    got = order[(wants.flatten().cumsum(0) - 1).clamp(0, order.numel() - 1)].view(wants.shape)
    fresh = got.gather(1, last[:, None])[:, 0]
    there = torch.where(copies, fresh, mine)                         # a row that copies nothing copies its page onto itself
    at, to = mine[open_], there[open_]
    for x in s["cache"]:                                             # (slots behind the sequence's end hold nothing yet)
        x[to] = x[at]
    s["refs"].index_add_(0, mine.clamp(min=0), -copies.to(torch.int32))
    s["refs"].index_add_(0, torch.where(wants, got, 0).flatten(), wants.flatten().to(torch.int32))
    table[rows] = torch.where(wants, got, table[rows].long()).to(torch.int32)
    s["lens"][rows] = (n + add).to(torch.int32)


def _plain_compact(s):
    t = torch.arange(s["total"], device=DEV)
    row = torch.searchsorted(s["starts"][1:].long(), t, right=True)
    i = t - s["starts"].long()[row]
    base = s["base"].long()[row]
    p, o = _place(s, row, base + s["keep"].long()[row, i])
    p2, o2 = _place(s, row, base + i)
    for x in s["cache"]:
        x[p2, :, o2] = x[p, :, o]


def _plain_fork_case(s):
    _plain_release(s, s["dst"], s["none"])
    _plain_fork(s, s["src"], s["dst"])
    _plain_extend(s, s["dst"], s["add"])
    return [s["table"], s["lens"], s["refs"], *_read(s, s["before"])]


def _plain_accept(s):
    _plain_release(s, s["rows"], s["base"])
    _plain_extend(s, s["rows"], s["add"])
    _plain_compact(s)
    _plain_release(s, s["rows"], s["after"])
    return [s["table"], s["lens"], s["refs"], *_read(s)]


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _own(s):
    from paper_2503_13565_amd import binding
    kind, cache, first = s["case"]["kind"], binding.KvCache(*s["cache"]), s.get("first", 0)
    table, lens = s["table"], s["lens"]
    if kind == "attend":
        got = binding.mxfp4_kv_attention(s["q"], cache, table, lens, starts=s["starts"], window=s["case"]["window"], tree=s["tree"],
                                         return_lse=s["case"]["lse"])
        return list(got) if s["case"]["lse"] else [got]
    if kind == "append":
        q = binding.mxfp4_kv_append(cache, s["k"], s["v"], table, lens, starts=s["starts"], q=s["q"], rope=s["rope"])
        return [q, *binding.mxfp4_kv_read(cache, table, lens, s["total"], starts=s["starts"])]
    pool = binding.KvPool(s["refs"], s["free"])
    if kind == "fork":
        binding.mxfp4_kv_release(pool, cache, table, lens, s["dst"], s["none"])
        binding.mxfp4_kv_fork(pool, cache, table, lens, s["src"], s["dst"])
        binding.mxfp4_kv_extend(pool, cache, table, lens, s["dst"], s["add"])
        return [table, lens, s["refs"], *binding.mxfp4_kv_read(cache, table[first:], s["before"], s["total"])]
    else:
        binding.mxfp4_kv_release(pool, cache, table, lens, s["rows"], s["base"])
        binding.mxfp4_kv_extend(pool, cache, table, lens, s["rows"], s["add"])
        binding.mxfp4_kv_compact(cache, table, s["base"], s["keep"], s["counts"])
        binding.mxfp4_kv_release(pool, cache, table, lens, s["rows"], s["after"])
    return [table, lens, s["refs"], *binding.mxfp4_kv_read(cache, table, lens, s["total"], starts=s["starts"])]


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "attend": _plain_attend, "fork": _plain_fork_case, "accept": _plain_accept}[s["case"]["kind"]](s)


# ---- from the definitions, in 64 bits -------------------------------------------------------------------------------

def _meaning(code, scale):
    """Codes and scale bytes as 64-bit numbers, from the fields of an element: sign, two exponent bits, one mantissa bit."""
    c = torch.stack([code & 15, code >> 4], dim=-1).flatten(-2).double()
    sign, c = 1 - 2 * (c >= 8).double(), c % 8
    e, m = (c / 2).floor(), c % 2
    mag = torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e - 1))
    return sign * mag * (2.0 ** (scale.double() - 127)).repeat_interleave(32, dim=-1)


def _nearest(x):
    """BF16-representable 64-bit numbers -> the nearest numbers of each block's MXFP4 grid (ties to the even code), as 64-bit numbers."""
    v = x.unflatten(-1, (-1, 32))
    top = v.abs().amax(-1, keepdim=True)
    unit = 2.0 ** (torch.frexp(top).exponent.double() - 3).clamp(min=-127)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    even = torch.tensor([0, 1, 0, 1, 0, 1, 0, 1], dtype=torch.float64, device=x.device) * 1e-9
    y = (v / unit).abs()
    pick = torch.zeros_like(y)
    best = torch.full_like(y, math.inf)
    for g, odd in zip(grid, even):
        off = (y - g).abs() + odd
        pick, best = torch.where(off < best, g, pick), torch.minimum(best, off)
    return (torch.sign(v) * pick * unit).flatten(-2)


def _exact_append(case, s):
    lens, starts = s["lens"].tolist(), s["starts"]
    at = []
    for b, n in enumerate(lens):
        new = int(starts[b + 1] - starts[b]) if starts is not None else s["total"] // len(lens)
        at += list(range(n - new, n))
    at = torch.tensor(at, device=DEV)
    half = case["rotary"] // 2

    def turned(x):
        c, n = s["rope"][0].double()[at][:, None], s["rope"][1].double()[at][:, None]
        z = x.double()
        z1, z2 = z[..., :half].clone(), z[..., half: 2 * half].clone()
        z = z.clone()
        z[..., :half], z[..., half: 2 * half] = z1 * c - z2 * n, z2 * c + z1 * n
        return z

    return [turned(s["q"]), _nearest(turned(s["k"]).to(torch.bfloat16).double()), _nearest(s["v"].double())]


def _exact_attend(case, s):
    page, d, group = case["page"], case["dim"], case["hq"] // case["hkv"]
    outs, lses, at = [], [], 0
    for b, n in enumerate(s["lens"].tolist()):
        new = int(s["starts"][b + 1] - s["starts"][b]) if s["starts"] is not None else case["new"]
        mine = s["table"][b, : -(-n // page)].long()
        q = s["q"][at: at + new].double()
        i, j = torch.arange(new, device=DEV)[:, None], torch.arange(n, device=DEV)[None]
        sees = j <= n - new + i
        if case["window"]:
            sees &= j > n - new + i - case["window"]
        if case["tree"]:
            word = s["tree"][at: at + new][:, None]
            sees = (j < n - new) | ((word >> (j - (n - new)).clamp(min=0)) & 1).bool()
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float64, device=DEV)
        for h in range(case["hkv"]):
            kq, ks, vq, vs = (x[mine, h].flatten(0, 1)[:n] for x in s["cache"])
            k, v = _meaning(kq, ks), _meaning(vq, vs)
            for g in range(h * group, h * group + group):
                z = (q[:, g] @ k.T) / math.sqrt(d)
                z = torch.where(sees, z, -math.inf)
                lse[:, g] = torch.logsumexp(z, dim=1)
                out[:, g] = torch.exp(z - lse[:, g, None]) @ v
        outs.append(out)
        lses.append(lse)
        at += new
    return [torch.cat(outs)] + ([torch.cat(lses)] if case["lse"] else [])


def _exact_pages(case, s):
    """The values that the first pass reads back: moved as they were (table, lengths and counts are whole numbers)."""
    page, rows, free = case["page"], case["rows"], torch.nonzero(s["refs"] == 0).flatten().tolist()
    k, v = [], []
    for b, n in enumerate(s["lens"].tolist()[:rows]):
        mine = s["table"][b].tolist()
        if case["kind"] == "fork":
            at = list(range(n - page, n)) * case["branches"]
        else:
            for w in range(-(-n // page), -(-(n + case["new"]) // page)):
                mine[w] = free.pop(0)
            at = [n + i for i in s["keep"][b].tolist()[: _kept(case, b)]]
        p = torch.tensor([mine[i // page] for i in at], device=DEV)
        o = torch.tensor([i % page for i in at], device=DEV)
        kq, ks, vq, vs = (x[p, :, o] for x in s["cache"])
        k.append(_meaning(kq, ks))
        v.append(_meaning(vq, vs))
    return [None, None, None, torch.cat(k), torch.cat(v)]


def exact(case, seed):
    if case["kind"] in ("fork", "accept"):
        return _exact_pages(case, prepare(case, seed))
    if case["kind"] == "attend" and work(case)["flops"] * max(1, case["new"] / 64) > 3e14:
        return None
    s = prepare(case, seed)
    return (_exact_append if case["kind"] == "append" else _exact_attend)(case, s)
