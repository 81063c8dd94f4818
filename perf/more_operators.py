"""The operators of an 8-bit paged key/value cache, as timed cases.

  store   new keys and values of several requests into the cache, and the values that the codes stand for
  step    one token of each request: its key and value into the cache, and attention over it, through a window with first tokens that
          stay visible or over everything
  prompt  several tokens of each request: the same, causal among them
  serve   what happens to pages between two steps: those of finished requests are freed, new ones taken for growing requests, requests
          forked (their last, partly filled page is copied in all layers) and pages copied
  compact the pages in use are brought together at the cache's start, in all layers

`run` computes them in their plain form, from elementary operations in 32 bits, or, where `own` is true, with the library's calls.

Layout of the cache: a page of P tokens holds, for each key head, P / 16 cells of 32 D + 16 bytes, one to 16 tokens: the codes of their
keys [D/64][16][64], the codes of their values, the scale of the keys (32-bit), the scale of the values and 8 bytes of zeros.  A value of
token r (of the 16) and dimension d is byte 512 (d / 32) + 64 (d % 8) + 16 (r % 8 / 2) + 4 (d % 32 / 8) + 2 (r / 8) + r % 2.  A code is an
e4m3 number; it stands for itself times the cell's scale, 2^e, the lowest of 2^-15 and up with max |x| <= 448 * 2^e.  Values are
first brought between -61440 and 61440.  When a token joins a cell whose scale is too small for it, the scale grows and the other
tokens' codes are rounded again.
"""
import math
import random

import torch

own = False
CELL = 16


def listed():
    return [
        # users of a 70B model in the middle of their answers: a token each, into cells that hold some already
        dict(name="store_64_8x128", op="store", N=64, B=64, past=2000, kv_heads=8, dim=128, page=16, v="f16"),
        # prompts of several users at once behind what the cache holds of them, 32-bit values of the projection
        dict(name="store_16384_8x128", op="store", N=16384, B=7, past=777, kv_heads=8, dim=128, page=64, v="f32"),
        # one user at the start of a conversation, as many key heads as query heads
        dict(name="step_1_32x32x128_1003", op="step", B=1, q_heads=32, kv_heads=32, dim=128, page=16, longest=1003),
        # one user with a long document, scores capped
        dict(name="step_1_64x8x128_131072", op="step", B=1, q_heads=64, kv_heads=8, dim=128, page=64, longest=131072, cap=50.0),
        # many users, conversations of all lengths
        dict(name="step_48_64x8x128_16384", op="step", B=48, q_heads=64, kv_heads=8, dim=128, page=64, longest=16384, ragged=True),
        # endless conversations: a window and four first tokens
        dict(name="step_33_28x4x128_w4096", op="step", B=33, q_heads=28, kv_heads=4, dim=128, page=32, longest=20000, ragged=True, window=4096, sinks=4),
        # a short prompt of odd length on a small model with small heads
        dict(name="prompt_333_12x3x64", op="prompt", N=333, B=1, past=0, q_heads=12, kv_heads=3, dim=64, page=16),
        # the prompt of a 70B model: the most work of all
        dict(name="prompt_4096_64x8x128", op="prompt", N=4096, B=1, past=0, q_heads=64, kv_heads=8, dim=128, page=64),
        # pieces of several prompts, some behind long contexts, capped, through a window with first tokens
        dict(name="prompt_2045_32x8x128_w2048", op="prompt", N=2045, B=6, past=6000, q_heads=32, kv_heads=8, dim=128, page=32, window=2048, sinks=16, cap=30.0),
        # a few requests of a small model between two steps
        dict(name="serve_12x256", op="serve", rows=12, pages=256, tokens=300, page=16, page_bytes=16 * 2 * 129, layers=4, done=1, grow=8, fork=2, copies=1),
        # many requests, a question sampled several times
        dict(name="serve_256x6000", op="serve", rows=256, pages=6000, tokens=500, page=16, page_bytes=16 * 129 * 2, layers=24, done=32, grow=200, fork=48, copies=32),
        # a cache with as many holes as pages in use
        dict(name="compact_1536x12", op="compact", rows=64, pages=1536, tokens=400, page=16, page_bytes=16 * 8 * 129, layers=12, done=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "store", "step", "step", "step", "prompt", "prompt", "prompt", "serve", "compact"])
    if op in ("serve", "compact"):
        rows, tokens, page = _log_int(rng, 4, 256), _log_int(rng, 20, 600), rng.choice([16, 32, 64])
        page_bytes = page * rng.choice([1, 2, 4, 8]) * rng.choice([129, 257])
        pages = rows * -(-tokens // page) + rng.randint(rows, 3 * rows) + 8
        case = dict(op=op, rows=rows, pages=pages, tokens=tokens, page=page, page_bytes=page_bytes,
                    layers=max(1, min(_log_int(rng, 1, 32), 600_000_000 // (pages * page_bytes))), done=rng.randint(1, max(1, rows // 2)))
        if case["op"] == "serve":
            case.update(grow=rng.randint(0, rows - case["done"]), fork=rng.randint(1, case["done"]), copies=rng.randint(1, 8))
        return case
    dim = rng.choice([64, 128, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, rng.randint(1, 12)])
    page = rng.choice([16, 32, 64, 128])
    if op == "store":
        N = _log_int(rng, 1, min(16384, 16384 * 1024 // (kv_heads * dim)))
        return dict(op=op, N=N, B=min(N, _log_int(rng, 1, 64)), past=rng.choice([0, _log_int(rng, 1, 4000)]), kv_heads=kv_heads, dim=dim, page=page,
                    v=rng.choice(["f16", "f32"]))
    group = rng.choice([1, 4, 8, 8, rng.randint(1, 16)])
    case = dict(op=op, q_heads=group * kv_heads, kv_heads=kv_heads, dim=dim, page=page)
    if op == "step":
        case["B"] = _log_int(rng, 1, 64)
        case["longest"] = _log_int(rng, 1, max(1, min(131072, 48 * 16384 * 1024 // (case["B"] * max(kv_heads, 4) * max(dim, 128)) // 2)))
        if case["B"] > 1:
            case["ragged"] = True
    else:
        # scores of the largest listed prompt at most
        case["N"] = _log_int(rng, 2, 4096)
        case["B"] = min(case["N"], _log_int(rng, 1, 16))
        most = 64 * 4096 * 4096 * 128 // (2 * case["q_heads"] * max(dim, 64) * case["N"])
        case["N"] = min(case["N"], max(2, 2 * most))
        case["B"] = min(case["N"], case["B"])
        case["past"] = rng.choice([0, 0, _log_int(rng, 1, max(1, min(16384, most // 2)))])
    if rng.random() < 0.3:
        case["cap"] = rng.choice([20.0, 30.0, 50.0])
    if rng.random() < 0.4:
        case["window"] = _log_int(rng, 1, 4096)
        if rng.random() < 0.7:
            case["sinks"] = rng.choice([1, 4, 4, 16, rng.randint(1, 100)])
    return case


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _page_bytes(case):
    return case["page"] * case["kv_heads"] * (2 * case["dim"] + 1)


def _lengths(case, seed):
    """New tokens and keys in all of each request, on the host: what a program that schedules requests knows."""
    rng = random.Random(seed * 7919 + 11)
    B = case["B"]
    if case["op"] == "step":
        longest = case["longest"]
        return [1] * B, [longest] + [rng.randint(1, longest) if case.get("ragged") else longest for _ in range(B - 1)]
    N, past = case["N"], case["past"]
    cuts = sorted(rng.randint(0, N - B) for _ in range(B - 1))          # at least one token to a request
    new = [b - a + 1 for a, b in zip([0] + cuts, cuts + [N - B])]
    # the first has the longest past
    return new, [n + (past if i == 0 else rng.randint(0, past)) for i, n in enumerate(new)]


def _decode_table():
    c = torch.arange(256)
    e, m = c // 8 % 16, c % 8
    v = torch.where(e == 0, m / 8.0 * 2.0 ** -6, (1.0 + m / 8.0) * 2.0 ** (e - 7.0))
    return torch.where(c >= 128, -v, v).float().cuda()


def _places(dim):
    """Where in a cell the codes of token r and dimension d lie: keys and values, [16][dim]."""
    r, d = torch.arange(CELL).unsqueeze(1), torch.arange(dim).unsqueeze(0)
    k = d // 64 * 1024 + r * 64 + d % 64
    v = CELL * dim + 512 * (d // 32) + 64 * (d % 8) + 16 * (r % 8 // 2) + 4 * (d % 32 // 8) + 2 * (r // 8) + r % 2
    return k.cuda(), v.cuda()


def _need(top):
    """The scale that a largest value asks for."""
    m, e = torch.frexp(top)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.ldexp(torch.ones_like(top), e.clamp(min=-15))


def _round(x, s):
    """What the codes of x with scale s stand for, by s: e4m3 numbers."""
    y = x / s
    e = torch.frexp(y)[1]
    step = torch.ldexp(torch.ones_like(y), (e - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def _byte(q):
    """The codes of e4m3 numbers."""
    a = q.abs()
    e = torch.frexp(a)[1] - 1
    low = a < 2.0 ** -6
    mantissa = torch.where(low, a * 512.0, torch.ldexp(a, 3 - e) - 8.0)
    code = torch.where(low, 0, (e + 7) * 8) + mantissa.int()
    return (code + torch.where(torch.signbit(q), 128, 0)).to(torch.uint8)


def _limit(x):
    return x.float().clamp(-61440.0, 61440.0)


def _fill(cells, dim, gen, k_places, v_places):
    """Cells [n][bytes] as if 16 tokens had been stored in each: keys with a few large dimensions."""
    for i in range(0, cells.shape[0], 16384):
        part = cells[i:i + 16384]
        for side, places in enumerate((k_places, v_places)):
            x = _normal(gen, part.shape[0], CELL, dim)
            if side == 0:
                x = x * (1.0 + 3.0 * (torch.arange(dim, device="cuda") % 37 == 5))
            s = _need(x.abs().amax((1, 2)))
            part[:, places.flatten()] = _byte(_round(x, s.view(-1, 1, 1))).flatten(1)
            part[:, 2 * CELL * dim + 4 * side:2 * CELL * dim + 4 * side + 4] = s.view(-1, 1).view(torch.uint8)


def _prepare_cache(case, gen, seed):
    H, D, page = case["kv_heads"], case["dim"], case["page"]
    new, length = _lengths(case, seed)
    B, N = case["B"], sum(new)
    each = -(-max(length) // page)
    pages = B * each + 1
    cache = torch.zeros(pages, _page_bytes(case), dtype=torch.uint8, device="cuda")
    k_places, v_places = _places(D)
    if max(length) > max(new):
        _fill(cache.view(-1, 2 * CELL * D + CELL), D, gen, k_places, v_places)
    table = torch.randperm(pages, generator=gen, device="cuda")[:B * each].view(B, each).int()
    kv = _normal(gen, N, 2 * H * D)
    v = kv[:, H * D:] if case.get("v") == "f32" else kv[:, H * D:].half()
    first = [sum(new[:i]) for i in range(B + 1)]
    return dict(k=kv[:, :H * D].half().contiguous().view(N, H, D), v=v.unflatten(-1, (H, D)), cache=cache, table=table,
                first=torch.tensor(first, dtype=torch.int32, device="cuda"), length=torch.tensor(length, dtype=torch.int32, device="cuda"),
                host_first=first, host_length=length, k_places=k_places, v_places=v_places, decode=_decode_table(),
                k_values=torch.empty(N, H, D, dtype=torch.float16, device="cuda"), v_values=torch.empty(N, H, D, dtype=torch.float16, device="cuda"))


def _prepare_attention(case, gen, seed):
    s = _prepare_cache(case, gen, seed)
    N, hq, D = s["k"].shape[0], case["q_heads"], case["dim"]
    return dict(s, q=_normal(gen, N, hq, D).half(), y=torch.empty(N, hq * D, dtype=torch.float16, device="cuda"), scale=1.0 / math.sqrt(D),
                cap=float(case.get("cap", 0.0)), window=int(case.get("window", 0)), sinks=int(case.get("sinks", 0)))


def _prepare_pages(case, gen, seed):
    rng = random.Random(seed * 104729 + 5)
    rows, pages, page, layers, done = (case[k] for k in ("rows", "pages", "page", "layers", "done"))
    tokens = [rng.randint(1, case["tokens"]) for _ in range(rows)]
    table_pages = -(-case["tokens"] // page) + 4
    # pages of requests that came and went: in no order, none used twice
    order = list(range(pages))
    rng.shuffle(order)
    table, ref = torch.full((rows, table_pages), -1, dtype=torch.int32), torch.zeros(pages, dtype=torch.int32)
    copies = [[order.pop() for _ in range(case.get("copies", 0))] for _ in range(2)]
    for p in copies[0] + copies[1]:                                     # kept for others, of no request
        ref[p] = 1
    finished = set(rng.sample(range(rows), done))
    for r in range(rows):
        for e in range(-(-tokens[r] // page)):
            p = order.pop()
            table[r, e], ref[p] = p, 1
    live = [r for r in range(rows) if r not in finished]
    grow = rng.sample(live, min(case.get("grow", 0), len(live)))
    # a finished request's row becomes that of a child
    children = rng.sample(sorted(finished), min(case.get("fork", 0), done)) if live else []
    parents = [rng.choice([r for r in live if r not in grow] or live) for _ in children]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    size = lambda r: -(-tokens[r] // page)
    s = dict(table0=table.cuda(), ref0=ref.cuda(), table=table.cuda(), ref=ref.cuda(), short=torch.zeros(1, dtype=torch.int32, device="cuda"),
             fork_short=torch.zeros(1, dtype=torch.int32, device="cuda"), live=torch.zeros(1, dtype=torch.int32, device="cuda"),
             done=ints(sorted(finished)), zeros=ints([0] * done), ends=ints([table_pages] * done), grow=ints(grow), grow_from=ints([size(r) for r in grow]),
             grow_to=ints([min(table_pages, size(r) + rng.randint(0, 2)) for r in grow]), parent=ints(parents), child=ints(children),
             fork_length=ints([tokens[r] for r in parents]), src=ints(copies[0]), dst=ints(copies[1]),
             cache=torch.randint(0, 256, (layers, pages, case["page_bytes"] // 16, 16), generator=gen, device="cuda", dtype=torch.uint8).view(layers, pages, -1))
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    make = dict(store=_prepare_cache, step=_prepare_attention, prompt=_prepare_attention, serve=_prepare_pages, compact=_prepare_pages)[case["op"]]
    return dict(make(case, gen, int(seed)), case=dict(case))


# ---- plain forms

def _cells(s):
    """[pages][heads][P/16][bytes]"""
    case = s["case"]
    return s["cache"].view(s["cache"].shape[0], case["kv_heads"], case["page"] // CELL, -1)


def _scales(cells, dim, side):
    at = 2 * CELL * dim + 4 * side
    return cells[..., at:at + 4].contiguous().view(torch.float32).squeeze(-1)


def _plain_store(s):
    case, dim = s["case"], s["case"]["dim"]
    N, H, _ = s["k"].shape
    B, page = case["B"], case["page"]
    # the cells that get tokens, request by request, and behind them some that do not exist
    new = (s["first"][1:] - s["first"][:-1]).long()
    length, first = s["length"].long(), s["first"].long()
    start = length - new
    count = (length + CELL - 1) // CELL - start // CELL
    ends = count.cumsum(0)
    c = torch.arange(N // CELL + 2 * B, device="cuda")
    exists = c < ends[-1]
    b = torch.searchsorted(ends, c, right=True).clamp(max=B - 1)
    block = start[b] // CELL + c - (ends - count)[b]
    position = block.unsqueeze(1) * CELL + torch.arange(CELL, device="cuda")               # [cells][16]
    is_new = (position >= start[b].unsqueeze(1)) & (position < length[b].unsqueeze(1)) & exists.unsqueeze(1)
    is_old = (position < start[b].unsqueeze(1)) & exists.unsqueeze(1)
    token = torch.where(is_new, first[b].unsqueeze(1) + position - start[b].unsqueeze(1), N)
    at = torch.where(exists, block, 0) * CELL
    # the last page is nobody's: cells that do not exist land there
    spare = torch.ones(s["cache"].shape[0], dtype=torch.bool, device="cuda").scatter(0, s["table"].flatten().long(), False).int().argmax()
    where = (torch.where(exists, s["table"][b, at // page].long(), spare), torch.arange(H, device="cuda").view(H, 1), at // CELL % (page // CELL))
    cells = _cells(s)
    mine = cells[where[0], :, where[2]]                                                    # [cells][heads][bytes]
    out = []
    for side, (x, places) in enumerate(((s["k"], s["k_places"]), (s["v"], s["v_places"]))):
        x = torch.cat([_limit(x.half()), torch.zeros(1, H, dim, device="cuda")])
        x = x[token].transpose(1, 2)                                                       # [cells][heads][16][dim]
        old_scale = torch.where(is_old.any(1).unsqueeze(1), _scales(mine, dim, side), 0.0)
        old = s["decode"][mine[..., places.flatten()].int()].unflatten(-1, (CELL, dim)) * old_scale.view(-1, H, 1, 1)
        old = torch.where(is_old.view(-1, 1, CELL, 1), old, 0.0)
        scale = torch.maximum(_need(x.abs().amax((2, 3))), old_scale).view(-1, H, 1, 1)
        q = _round(x + old, scale)
        mine[..., places.flatten()] = _byte(q).flatten(2)
        at = 2 * CELL * dim + 4 * side
        mine[..., at:at + 4] = scale.contiguous().view(-1, H, 1).view(torch.uint8)
        values = torch.empty(N + 1, H, dim, dtype=torch.float16, device="cuda")
        values[token] = (q * scale).half().transpose(1, 2)
        out.append(values[:N])
    cells[where[0], :, where[2]] = mine
    return dict(k=out[0], v=out[1])


def _plain_attention(s):
    case, dim = s["case"], s["case"]["dim"]
    stored = _plain_store(s)
    cells = _cells(s)
    H, hq = case["kv_heads"], case["q_heads"]
    y = torch.empty_like(s["y"])
    for b in range(case["B"]):
        n0, n1, T = s["host_first"][b], s["host_first"][b + 1], s["host_length"][b]
        mine = cells[s["table"][b, :-(-T // case["page"])].long()].transpose(0, 1).flatten(1, 2)      # [heads][cells][bytes]

        def side(i, places):
            x = s["decode"][mine[..., places.flatten()].int()].unflatten(-1, (CELL, dim)) * _scales(mine, dim, i)[..., None, None]
            return x.flatten(1, 2)[:, :T]
        k, v = side(0, s["k_places"]), side(1, s["v_places"])
        n = torch.arange(T, device="cuda")
        for m0 in range(n0, n1, 512):
            m1 = min(n1, m0 + 512)
            q = s["q"][m0:m1].float().view(m1 - m0, H, hq // H, dim).permute(1, 2, 0, 3).flatten(1, 2)
            score = (q @ k.transpose(1, 2)) * s["scale"]
            if s["cap"] > 0.0:
                score = s["cap"] * torch.tanh(score / s["cap"])
            at = (T - n1 + torch.arange(m0, m1, device="cuda")).unsqueeze(1)
            out = n > at
            if s["window"] > 0:
                out = out | ((n <= at - s["window"]) & (n >= s["sinks"]))
            score = score.view(H, hq // H, m1 - m0, T).masked_fill(out, -math.inf)
            p = torch.exp(score - score.amax(-1, keepdim=True))
            o = (p.flatten(1, 2) @ v).view(H, hq // H, m1 - m0, dim) / p.sum(-1, keepdim=True)
            y[m0:m1] = o.permute(2, 0, 1, 3).reshape(m1 - m0, -1).half()
    return dict(stored, y=y)


def _give(ref, wanted):
    """Pages for the wanted places (a mask, in its order): the free ones, lowest first, or -1."""
    free = ref <= 0
    pages = ref.numel()
    order = torch.full((pages + 1,), -1, dtype=torch.int64, device="cuda")
    order[torch.where(free, free.cumsum(0) - 1, pages)] = torch.arange(pages, device="cuda")
    total = free.sum()
    rank = wanted.flatten().cumsum(0).view(wanted.shape) - 1
    return torch.where(wanted & (rank < total), order[rank.clamp(min=0, max=pages - 1)], -1), (wanted.sum() - total).clamp(min=0)


def _add(ref, which, by):
    """ref[which] += by where which is a page."""
    padded = torch.cat([ref, ref.new_zeros(1)])
    padded.index_add_(0, torch.where(which >= 0, which, ref.numel()).flatten().long(), torch.full((which.numel(),), by, dtype=ref.dtype, device="cuda"))
    ref.copy_(padded[:-1])


def _plain_free(s):
    table, ref = s["table"], s["ref"]
    e = torch.arange(table.shape[1], device="cuda")
    mine = table[s["done"].long()]
    out = (e >= s["zeros"].unsqueeze(1)) & (e < s["ends"].unsqueeze(1))
    _add(ref, torch.where(out, mine, -1), -1)
    table[s["done"].long()] = torch.where(out, -1, mine)


def _plain_serve(s):
    case, table, ref = s["case"], s["table"], s["ref"]
    table.copy_(s["table0"]), ref.copy_(s["ref0"])
    s["cache"][:, s["dst"].long()] = s["cache"][:, s["src"].long()]
    _plain_free(s)
    e = torch.arange(table.shape[1], device="cuda")
    wanted = (e >= s["grow_from"].unsqueeze(1)) & (e < s["grow_to"].unsqueeze(1))
    given, short = _give(ref, wanted)
    table[s["grow"].long()] = torch.where(wanted, given.int(), table[s["grow"].long()])
    _add(ref, given, 1)
    full = (s["fork_length"] // case["page"]).unsqueeze(1)
    part = (e == full) & (s["fork_length"] % case["page"] > 0).unsqueeze(1)
    given, fork_short = _give(ref, part)
    theirs, mine = table[s["parent"].long()], table[s["child"].long()]
    _add(ref, torch.where(e < full, theirs, -1), 1)
    _add(ref, given, 1)
    table[s["child"].long()] = torch.where(e < full, theirs, torch.where(part, given.int(), mine))
    copy = part & (given >= 0)
    # a child without a partly filled page repeats another's copy, or copies a page onto itself
    from_, to = torch.where(copy, theirs, -1).amax(1), torch.where(copy, given.int(), -1).amax(1)
    any_ = (to >= 0).int().argmax()
    from_, to = (torch.where(to >= 0, x, x[any_]).clamp(min=0).long() for x in (from_, to))
    s["cache"][:, to] = s["cache"][:, from_]
    return dict(table=table, ref=ref, short=short, fork_short=fork_short, cache=s["cache"])


def _plain_compact(s):
    table, ref = s["table"], s["ref"]
    table.copy_(s["table0"]), ref.copy_(s["ref0"])
    _plain_free(s)
    pages = ref.numel()
    used = ref > 0
    live = used.sum()
    n = torch.arange(pages, device="cuda")
    hole, mover = (n < live) & ~used, (n >= live) & used
    holes = torch.zeros(pages + 1, dtype=torch.int64, device="cuda")
    holes[torch.where(hole, hole.cumsum(0) - 1, pages)] = n
    to = torch.where(mover, holes[(mover.cumsum(0) - 1).clamp(min=0)], n)                  # of each page its new place
    source = torch.arange(pages + 1, device="cuda")                                        # and of each place where it comes from
    source[torch.where(mover, to, pages)] = n
    source = source[:pages]
    for layer in s["cache"]:
        layer.copy_(layer[source])
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    ref.copy_(torch.where(n < live, ref[source], 0))
    return dict(table=table, ref=ref, live=live, cache=s["cache"])


# ---- the library's calls

def _own(s):
    from paper_2607_21985_b200 import spdp
    case = s["case"]
    op = case["op"]
    if op in ("serve", "compact"):
        table, ref = s["table"], s["ref"]
        if "numbers" not in s:                              # the calls write 32-bit numbers, the plain form's are 64-bit ones: these have them in their lower halves
            s["numbers"] = torch.zeros(2, dtype=torch.int64, device="cuda")
            s["halves"] = [n.view(torch.int32)[:1] for n in s["numbers"].split(1)]
            s["wholes"] = list(s["numbers"].unbind())
        table.copy_(s["table0"]), ref.copy_(s["ref0"])
        if op == "compact":
            spdp.spdp_kv_pages_free(ref, table, s["done"], s["zeros"], s["ends"])
            spdp.spdp_kv_pages_compact(s["cache"], ref, table, s["halves"][0])
            return dict(table=table, ref=ref, live=s["wholes"][0], cache=s["cache"])
        spdp.spdp_kv_pages_copy(s["cache"], s["src"], s["dst"])
        spdp.spdp_kv_pages_free(ref, table, s["done"], s["zeros"], s["ends"])
        spdp.spdp_kv_pages_take(ref, table, s["grow"], s["grow_from"], s["grow_to"], s["halves"][0])
        spdp.spdp_kv_pages_fork(s["cache"], ref, table, case["page"], s["parent"], s["child"], s["fork_length"], s["halves"][1])
        return dict(table=table, ref=ref, short=s["wholes"][0], fork_short=s["wholes"][1], cache=s["cache"])
    first = None if op == "step" else s["first"]
    spdp.spdp_kv8_store(s["k"], s["v"], s["cache"], case["page"], s["table"], s["length"], first=first, k_values=s["k_values"], v_values=s["v_values"])
    stored = dict(k=s["k_values"], v=s["v_values"])
    if op == "store":
        return stored
    spdp.spdp_attn_kv8(s["q"], s["cache"], case["page"], case["kv_heads"], s["table"], s["length"], s["y"], s["scale"], first=first, cap=s["cap"],
                       window=s["window"], sinks=s["sinks"])
    return dict(stored, y=s["y"])


def run(state):
    if own:
        return _own(state)
    return dict(store=_plain_store, step=_plain_attention, prompt=_plain_attention, serve=_plain_serve, compact=_plain_compact)[state["case"]["op"]](state)


# ---- what cannot be done without

def _visible(new, length, window, sinks):
    """Keys that the tokens of a request see in all, and those that any of them sees."""
    pairs = 0
    for at in range(length - new, length):
        low = max(0, at + 1 - window) if window else 0
        pairs += at + 1 - low + min(sinks, low)
    low = max(0, length - new + 1 - window) if window else 0
    return pairs, length - low + min(sinks, low)


def work(case):
    """Every input once, every output once; of the cache what the tokens see, for requests of the average length."""
    op = case["op"]
    if op in ("serve", "compact"):
        tokens, rows, page = case["tokens"], case["rows"], case["page"]
        mean = (-(-tokens // page) + 1) / 2.0
        tables = 8.0 * rows * (-(-tokens // page) + 4) + 8.0 * case["pages"]
        if op == "serve":
            moved = case["copies"] + min(case["fork"], case["done"]) * (1.0 - 1.0 / page)
        else:
            used = (rows - case["done"]) * mean
            moved = used * (1.0 - used / case["pages"])
        return dict(bytes=2.0 * moved * case["layers"] * case["page_bytes"] + tables, flops=0.0)
    H, D, B = case["kv_heads"], case["dim"], case["B"]
    row = H * D
    if op == "store":
        N = case["N"]
        return dict(bytes=N * (row * ((4 if case["v"] == "f32" else 2) + 2 + 4 + 2) + 4.0) + B * 16.0, flops=8.0 * N * row)
    window, sinks = case.get("window", 0), case.get("sinks", 0)
    if op == "step":
        N, lengths = B, [case["longest"]] + [(case["longest"] + 1) // 2 if case.get("ragged") else case["longest"]] * (B - 1)
        new = [1] * B
    else:
        N = case["N"]
        new = [N // B + (1 if b < N % B else 0) for b in range(B)]
        lengths = [n + (case["past"] if b == 0 else case["past"] // 2) for b, n in enumerate(new)]
    seen = [_visible(n, t, window, sinks) for n, t in zip(new, lengths)]
    pairs, keys = sum(p for p, _ in seen), sum(k for _, k in seen)
    return dict(bytes=keys * row * (2 + 2.0 / D) + N * (row * (2 + 2 + 4 + 2) + case["q_heads"] * D * 4.0) + B * 12.0 + keys / case["page"] * 4.0,
                flops=4.0 * pairs * case["q_heads"] * D)


# ---- from the definitions, in 64 bits

def _exact_codes(x):
    """The e4m3 numbers nearest to x, ties to the even one: by comparison with all of them."""
    numbers = torch.tensor([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8) if (e, m) != (15, 7)],
                           dtype=torch.float64, device="cuda")
    a = x.abs().contiguous()
    high = torch.searchsorted(numbers, a).clamp(max=126)
    low = (high - 1).clamp(min=0)
    up, down = numbers[high] - a, a - numbers[low]
    return torch.where((up < down) | ((up == down) & (high % 2 == 0)), numbers[high], numbers[low]) * torch.sign(x)


def _exact_scale(top):
    e = -15
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def _exact_cells(s, b):
    """The cells of a request after the store, as values [heads][tokens][dim] of keys and of values; None in place of what it does not need."""
    case, D, H, P = s["case"], s["case"]["dim"], s["case"]["kv_heads"], s["case"]["page"]
    n0, n1, T = s["host_first"][b], s["host_first"][b + 1], s["host_length"][b]
    start = T - (n1 - n0)
    numbers = torch.tensor([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** (max(e, 1) - 7) * sign for sign in (1, -1) for e in range(16) for m in range(8)],
                           dtype=torch.float64, device="cuda")
    used = s["cache"][s["table"][b, :-(-T // P)].long()].view(-1, H, P // 16, 32 * D + 16).permute(1, 0, 2, 3).reshape(H, -1, 32 * D + 16)
    r, d = torch.arange(16, device="cuda"), torch.arange(D, device="cuda")
    key_at = (d // 64 * 1024 + d % 64).unsqueeze(0) + 64 * r.unsqueeze(1)
    value_at = 16 * D + (512 * (d // 32) + 64 * (d % 8) + 4 * (d // 8 % 4)).unsqueeze(0) + (16 * (r // 2 % 4) + 2 * (r // 8) + r % 2).unsqueeze(1)
    result = []
    for side, (x, at) in enumerate(((s["k"], key_at), (s["v"], value_at))):
        scale = used[..., 32 * D + 4 * side:32 * D + 4 * side + 4].contiguous().view(torch.float32).double()       # [heads][cells][1]
        x = x[n0:n1].half().double().clamp(-61440, 61440).transpose(0, 1)                                          # [heads][new][dim]
        old = (numbers[used[..., at.flatten()].long()] * scale).view(H, -1, 16, D).flatten(1, 2)[:, :start]
        whole = torch.cat([old, x], 1)
        whole = torch.cat([whole, whole.new_zeros(H, -T % 16, D)], 1).view(H, -1, 16, D)
        first = start // 16                                              # cells before it stay as they are
        touched = whole[:, first:]
        fresh = touched.clone().flatten(1, 2)
        fresh[:, :start % 16] = 0.0
        top = fresh.view(touched.shape).abs().amax((2, 3))
        want = torch.tensor([_exact_scale(v) for v in top.flatten().tolist()], dtype=torch.float64, device="cuda").view(top.shape)
        if start % 16:
            want[:, 0] = torch.maximum(want[:, 0], scale[:, first, 0])
        want = want[..., None, None]
        whole[:, first:] = _exact_codes(touched / want) * want
        result.append(whole.flatten(1, 2)[:, :T])
    return result


def _exact_cache(s):
    case = s["case"]
    D, H, attention = case["dim"], case["kv_heads"], case["op"] != "store"
    k, v = (torch.empty(s["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    y = torch.empty(s["y"].shape, dtype=torch.float64, device="cuda") if attention else None
    for b in range(case["B"]):
        n0, n1, T = s["host_first"][b], s["host_first"][b + 1], s["host_length"][b]
        keys, values = _exact_cells(s, b)
        k[n0:n1], v[n0:n1] = keys[:, T - (n1 - n0):].transpose(0, 1), values[:, T - (n1 - n0):].transpose(0, 1)
        for m0 in range(n0, n1, 256) if attention else ():
            m1 = min(n1, m0 + 256)
            z = torch.einsum("nhgd,htd->hgnt", s["q"][m0:m1].double().view(m1 - m0, H, -1, D), keys) * s["scale"]
            if s["cap"] > 0.0:
                z = s["cap"] * torch.tanh(z / s["cap"])
            i, j = torch.arange(T - n1 + m0, T - n1 + m1, device="cuda").unsqueeze(1), torch.arange(T, device="cuda")
            seen = j <= i
            if s["window"] > 0:
                seen = seen & ((i - j < s["window"]) | (j < s["sinks"]))
            z = torch.where(seen, z, -math.inf)
            y[m0:m1] = torch.einsum("hgnt,htd->nhgd", torch.softmax(z, -1), values).reshape(m1 - m0, -1)
    return dict(k=k, v=v, y=y) if attention else dict(k=k, v=v)


def _exact_pages(s):
    case = s["case"]
    table, ref, page = s["table0"].tolist(), s["ref0"].tolist(), case["page"]
    cache = s["cache"]

    def lowest():
        for p, n in enumerate(ref):
            if n <= 0:
                ref[p] = 1
                return p
        return -1

    def result(**more):
        tensor = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        return dict(table=tensor(table), ref=tensor(ref), **{k: torch.tensor(v, device="cuda") for k, v in more.items()}, cache=cache)

    if case["op"] == "serve":
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            cache[:, b] = cache[:, a]
    for r in s["done"].tolist():
        for e, p in enumerate(table[r]):
            if p >= 0:
                ref[p] -= 1
                table[r][e] = -1
    if case["op"] == "compact":
        live = sum(n > 0 for n in ref)
        holes = [p for p in range(live) if ref[p] <= 0]
        movers = [p for p in range(live, len(ref)) if ref[p] > 0]
        new = dict(zip(movers, holes))
        for a, b in new.items():
            cache[:, b] = cache[:, a]
            ref[b], ref[a] = ref[a], 0
        table = [[new.get(p, p) for p in row] for row in table]
        return result(live=live)
    short = fork_short = 0
    for r, a, b in zip(s["grow"].tolist(), s["grow_from"].tolist(), s["grow_to"].tolist()):
        for e in range(a, b):
            table[r][e] = lowest()
            short += table[r][e] < 0
    for a, b, n in zip(s["parent"].tolist(), s["child"].tolist(), s["fork_length"].tolist()):
        for e in range(n // page):
            table[b][e] = table[a][e]
            ref[table[a][e]] += 1
        if n % page:
            p = table[b][n // page] = lowest()
            if p >= 0:
                cache[:, p] = cache[:, table[a][n // page]]
            else:
                fork_short += 1
    return result(short=short, fork_short=fork_short)


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_pages(s) if case["op"] in ("serve", "compact") else _exact_cache(s)
