"""The operators around the packed projections of a decoder layer, as timed cases.

  lora    adapters of many requests beside a shared projection: y_n = base_n + s_a B_a A_a x_n, a the adapter of token n
  norm    norms of the query and key heads and their rotation by positions with one or several axes, in one pass
  store   new keys and values into a paged cache of 4-bit codes, and the values that the codes stand for
  step    one token of each request: its key and value into that cache, and attention over it

`run` computes them in their plain form, from elementary operations in 32 bits, or, where `own` is true, with the
library's calls.  Weights are N(0, 1/K) and N(0, 0.02^2), activations N(0, 1).

Layout of the 4-bit cache: a page holds, for each key head, the codes of its P tokens' keys [P][D/2], of their values
[P][D/2], the scales of the keys fp16 [P][D/32] and of the values [P][D/32].  A row's dimension 32 g + 8 c + j is
the j-th nibble (from the lowest) of the 32-bit word c D/32 + g.  A code is one of 1..15 and stands for (code - 8) * scale,
one scale to 32 dimensions: fp16(max |x| / 7).
"""
import math

import torch

own = False


def listed():
    return [
        # the smallest call: one token of one user through an attention projection of a 7B model
        dict(name="lora_1x4096x4096_r16", op="lora", N=1, K=4096, M=4096, rank=16, adapters=4, y="f16"),
        # eight users with adapters of their own, up-projection of a 70B model
        dict(name="lora_8x28672x8192_r64", op="lora", N=8, K=8192, M=28672, rank=64, adapters=16, y="f16"),
        # nothing a multiple of a tile, adapters of different ranks, some tokens without one, 32-bit results
        dict(name="lora_300x4001x4098_r20", op="lora", N=300, K=4098, M=4001, rank=20, adapters=5, ranks=True, run=37, y="f32"),
        # prompts of several users on the largest layer
        dict(name="lora_1024x28672x8192_r16", op="lora", N=1024, K=8192, M=28672, rank=16, adapters=8, run=200, y="f16"),
        # one token of a 7B model
        dict(name="norm_1_32x32x128", op="norm", N=1, q_heads=32, kv_heads=32, dim=128, rot=128, axes=1, x="f16"),
        # no power of two, heads of 64 rotated in part and by neighbours, 16-bit results of the projection
        dict(name="norm_333_12x3x64", op="norm", N=333, q_heads=12, kv_heads=3, dim=64, rot=40, axes=2, adjacent=True, x="f16"),
        # frames of a video behind a 70B model's projections, positions in time, height and width, 32-bit results of the projection
        dict(name="norm_4096_64x8x128", op="norm", N=4096, q_heads=64, kv_heads=8, dim=128, rot=128, axes=3, x="f32"),
        # a prompt of odd length
        dict(name="store_1021_8x128", op="store", N=1021, kv_heads=8, dim=128, page=16, v="f16"),
        # several prompts at once, 32-bit values of the projection
        dict(name="store_16384_8x128", op="store", N=16384, kv_heads=8, dim=128, page=64, v="f32"),
        # one user at the start of a conversation, as many key heads as query heads
        dict(name="step_1_32x32x128_1003", op="step", B=1, q_heads=32, kv_heads=32, dim=128, page=16, longest=1003),
        # one user with a long document, scores capped
        dict(name="step_1_64x8x128_131072", op="step", B=1, q_heads=64, kv_heads=8, dim=128, page=64, longest=131072, cap=50.0),
        # many users, conversations of all lengths: the most work of all
        dict(name="step_48_64x8x128_16384", op="step", B=48, q_heads=64, kv_heads=8, dim=128, page=64, longest=16384, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lora", "lora", "lora", "norm", "norm", "store", "step", "step", "step"])
    if op == "lora":
        step = 1 if rng.random() < 0.4 else 128           # layers of real models are multiples of 128; others are not
        M, K = (max(step, _log_int(rng, 512, 28672) // step * step), max(step, _log_int(rng, 512, 11008) // step * step))
        case = dict(op=op, N=_log_int(rng, 1, 1024), K=K, M=M, rank=rng.choice([4, 8, 16, 16, 32, 64, 128, rng.randint(1, 96)]),
                    adapters=rng.randint(1, 16), y=rng.choice(["f16", "f16", "f32"]))
        if case["y"] == "f32":
            case["N"] = min(case["N"], 512)
        if rng.random() < 0.3:
            case["ranks"] = True
        if case["N"] > 16 and rng.random() < 0.8:         # else every token draws its adapter
            case["run"] = _log_int(rng, 4, case["N"])
        return case
    dim = rng.choice([64, 128, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, rng.randint(1, 12)])
    if op == "norm":
        group = rng.choice([1, 2, 4, 8, rng.randint(1, 12)])
        case = dict(op=op, N=_log_int(rng, 1, max(1, min(8192, (4096 * 72 * 128) // ((group + 1) * kv_heads * dim)))), q_heads=group * kv_heads, kv_heads=kv_heads,
                    dim=dim, rot=rng.choice([dim, dim, dim // 2, 2 * rng.randint(3, dim // 2)]), axes=rng.randint(1, 3), x=rng.choice(["f16", "f32"]))
        if rng.random() < 0.4:
            case["adjacent"] = True
        return case
    page = rng.choice([16, 32, 64, 128])
    if op == "store":
        return dict(op=op, N=_log_int(rng, 1, min(16384, 16384 * 1024 // (kv_heads * dim))), kv_heads=kv_heads, dim=dim, page=page, v=rng.choice(["f16", "f32"]))
    group = rng.choice([1, 4, 8, 8, rng.randint(1, 16)])
    B = _log_int(rng, 1, 64)
    longest = _log_int(rng, 1, max(1, min(131072, 48 * 16384 * 1024 // (B * max(kv_heads, 4) * max(dim, 128)) // 2)))
    case = dict(op=op, B=B, q_heads=group * kv_heads, kv_heads=kv_heads, dim=dim, page=page, longest=longest)
    if B > 1:
        case["ragged"] = True
    if rng.random() < 0.3:
        case["cap"] = rng.choice([20.0, 30.0, 50.0])
    if rng.random() < 0.3:
        case["window"] = _log_int(rng, 1, 4096)
    return case


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda")


def _pages(case):
    """Pages of the longest request of a step, or of all tokens of a store."""
    return -(-case.get("longest", case.get("N")) // case["page"])


def _page_bytes(case):
    return case["kv_heads"] * case["page"] * case["dim"] * 9 // 8


def _prepare_lora(case, gen):
    N, K, M, rank, L = case["N"], case["K"], case["M"], case["rank"], case["adapters"]
    run = case.get("run", 1)
    # the tokens of a request stand together and share its adapter; one request in eight has none
    each = (_uniform(gen, -(-N // run)) * (L * 8 / 7)).int()
    each = torch.where(each < L, each, -1)
    ld = (K + 7) // 8 * 8                                   # a token's row starts on a 16-byte boundary
    X = torch.zeros(N, ld, dtype=torch.float16, device="cuda")
    X[:, :K] = _normal(gen, N, K).half()
    ydt = torch.float32 if case["y"] == "f32" else torch.float16
    ranks = torch.full((L,), rank, dtype=torch.int32, device="cuda")
    if case.get("ranks"):
        ranks = (1 + (_uniform(gen, L) * rank).int()).clamp(max=rank)
    return dict(X=X[:, :K], adapter=(each if L > 1 else each.clamp(min=0)).repeat_interleave(run)[:N].contiguous(),
                A=(_normal(gen, L, rank, K) / math.sqrt(K)).half(), B=(_normal(gen, L, M, rank) * 0.02).half(),
                scales=0.5 + _uniform(gen, L) * 2.0, ranks=ranks, base=_normal(gen, N, M).to(ydt),
                Y=torch.empty(N, M, dtype=ydt, device="cuda"))


def _sections(case):
    """Frequency pairs of each axis: the first gets the most."""
    half, axes = case["rot"] // 2, case["axes"]
    rest = half // (axes + 1)
    return [half - rest * (axes - 1)] + [rest] * (axes - 1)


def _prepare_norm(case, gen):
    N, hq, hk, D, rot, axes = (case[k] for k in ("N", "q_heads", "kv_heads", "dim", "rot", "axes"))
    dt = torch.float32 if case["x"] == "f32" else torch.float16
    qkv = _normal(gen, N, (hq + 2 * hk) * D).to(dt)         # what one projection for all three leaves
    start = int(1e6 * float(_uniform(gen, 1).cpu()) ** 4)   # short and long contexts
    n = torch.arange(N, device="cuda")
    pos = torch.stack([start + (n if axes == 1 else n // 256), n // 16 % 16, n % 16][:axes]).int()
    half = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    return dict(q=qkv[:, :hq * D].view(N, hq, D), k=qkv[:, hq * D:(hq + hk) * D].view(N, hk, D), pos=pos.contiguous(),
                inv_freq=(500000.0 ** (-2.0 * half / rot)).float(), sections=_sections(case),
                axis=torch.tensor([a for a, m in enumerate(_sections(case)) for _ in range(m)], device="cuda"), adjacent=bool(case.get("adjacent")), eps=1e-6,
                q_weight=(1.0 + 0.1 * _normal(gen, D)).half(), k_weight=(1.0 + 0.1 * _normal(gen, D)).half(),
                q_out=torch.empty(N, hq, D, dtype=torch.float16, device="cuda"), k_out=torch.empty(N, hk, D, dtype=torch.float16, device="cuda"))


def _codes(x):
    """fp16 [..., D] -> codes uint8 [..., D] and scales fp16 [..., D/32]."""
    f = x.float().unflatten(-1, (-1, 32))
    scale = (f.abs().amax(-1) / 7.0).half()
    s = scale.float().unsqueeze(-1)
    code = torch.where(s > 0, torch.round(f / torch.where(s > 0, s, 1.0)).clamp(-7, 7), 0.0) + 8.0
    return code.flatten(-2).to(torch.uint8), scale


def _rows(codes):
    """Codes [..., D] in the order of a row's bytes [..., D/2]."""
    by = codes.unflatten(-1, (-1, 4, 8)).transpose(-3, -2).flatten(-3)     # (group, c, j) -> (c, group, j)
    return by[..., 0::2] | (by[..., 1::2] << 4)


def _values(rows, scales):
    """The fp32 values that rows [..., D/2] with scales [..., D/32] stand for."""
    codes = torch.stack([rows & 15, rows >> 4], -1).flatten(-2)
    f = codes.unflatten(-1, (4, -1, 8)).transpose(-3, -2).flatten(-2).float() - 8.0
    return (f * scales.float().unsqueeze(-1)).flatten(-2)


def _parts(cache, case):
    """Views of a cache [pages][page_bytes]: key rows, value rows [pages][heads][P][D/2], key and value scales [..][P][D/32]."""
    H, P, D = case["kv_heads"], case["page"], case["dim"]
    head = cache.view(-1, H, P * D * 9 // 8)
    n, m = P * D // 2, P * D // 16
    return (head[..., :n].unflatten(-1, (P, -1)), head[..., n:2 * n].unflatten(-1, (P, -1)),
            head[..., 2 * n:2 * n + m].view(torch.float16).unflatten(-1, (P, -1)), head[..., 2 * n + m:].view(torch.float16).unflatten(-1, (P, -1)))


def _prepare_store(case, gen):
    N, H, D, page = case["N"], case["kv_heads"], case["dim"], case["page"]
    pages = _pages(case) + 2
    kv = _normal(gen, N, 2 * H * D)
    v = kv[:, H * D:] if case["v"] == "f32" else kv[:, H * D:].half()
    order = torch.randperm(pages, generator=gen, device="cuda")
    n = torch.arange(N, device="cuda")
    return dict(k=kv[:, :H * D].half().contiguous().view(N, H, D), v=v.unflatten(-1, (H, D)), slot=order[n // page] * page + n % page,
                cache=torch.zeros(pages, _page_bytes(case), dtype=torch.uint8, device="cuda"),
                k_values=torch.empty(N, H, D, dtype=torch.float16, device="cuda"), v_values=torch.empty(N, H, D, dtype=torch.float16, device="cuda"))


def _prepare_step(case, gen):
    B, hq, H, D, page, longest = (case[k] for k in ("B", "q_heads", "kv_heads", "dim", "page", "longest"))
    length = torch.full((B,), longest, dtype=torch.int32, device="cuda")
    if case.get("ragged"):                                  # the longest first, the others spread over all lengths
        length[1:] = torch.ceil(_uniform(gen, B - 1) * longest).int().clamp(1, longest)
    each = _pages(case)
    pages = B * each
    cache = torch.zeros(pages, _page_bytes(case), dtype=torch.uint8, device="cuda")
    for rows, scales in zip(_parts(cache, case)[:2], _parts(cache, case)[2:]):
        for p in range(0, pages, 1024):
            codes, s = _codes(_normal(gen, min(1024, pages - p), H, page, D).half())
            rows[p:p + 1024], scales[p:p + 1024] = _rows(codes), s
    table = torch.randperm(pages, generator=gen, device="cuda").view(B, each).int()
    last = (length - 1).long()
    slot = table.gather(1, (last // page).unsqueeze(1)).squeeze(1).long() * page + last % page
    kv = _normal(gen, B, 2 * H * D).half()
    return dict(q=_normal(gen, B, hq, D).half(), k=kv[:, :H * D].view(B, H, D), v=kv[:, H * D:].view(B, H, D), slot=slot, cache=cache, table=table,
                length=length, scale=1.5 / math.sqrt(D), cap=float(case.get("cap", 0.0)), window=int(case.get("window", 0)),
                k_values=torch.empty(B, H, D, dtype=torch.float16, device="cuda"), v_values=torch.empty(B, H, D, dtype=torch.float16, device="cuda"),
                y=torch.empty(B, hq * D, dtype=torch.float16, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    make = dict(lora=_prepare_lora, norm=_prepare_norm, store=_prepare_store, step=_prepare_step)[case["op"]]
    return dict(make(case, gen), case=dict(case))


def _plain_lora(s):
    A, B = s["A"].float(), s["B"].float()
    L, rank, K = A.shape
    # the products with all adapters side by side, then only the token's own: two matrix products
    mine = (s["adapter"].unsqueeze(1) == torch.arange(L, device="cuda")) * s["scales"]
    keep = torch.arange(rank, device="cuda") < s["ranks"].unsqueeze(1)
    t = (s["X"].float() @ A.view(L * rank, K).T).view(-1, L, rank) * (mine.unsqueeze(2) * keep)
    return (s["base"].float() + t.view(-1, L * rank) @ B.transpose(1, 2).reshape(L * rank, -1)).to(s["Y"].dtype)


def _plain_norm(s):
    half = s["inv_freq"].numel()
    angle = s["pos"].double()[s["axis"]].T * s["inv_freq"].double()          # [N][half], in 64 bits: positions go far
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)

    def one(x, weight):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * weight.float()
        turn, rest = x[..., :2 * half], x[..., 2 * half:]
        if s["adjacent"]:
            a, b = turn[..., 0::2], turn[..., 1::2]
            turn = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = turn[..., :half], turn[..., half:]
            turn = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([turn, rest], -1).half()
    return dict(q=one(s["q"], s["q_weight"]), k=one(s["k"], s["k_weight"]))


def _plain_store(s):
    case = s["case"]
    k_rows, v_rows, k_scales, v_scales = _parts(s["cache"], case)
    page, at = s["slot"] // case["page"], s["slot"] % case["page"]
    (kc, ks), (vc, vs) = _codes(s["k"]), _codes(s["v"].half())
    k_rows[page, :, at], v_rows[page, :, at] = _rows(kc), _rows(vc)
    k_scales[page, :, at], v_scales[page, :, at] = ks, vs
    return dict(k=_values(_rows(kc), ks).half(), v=_values(_rows(vc), vs).half())


def _plain_step(s):
    stored = _plain_store(s)
    k_rows, v_rows, k_scales, v_scales = _parts(s["cache"], s["case"])
    at = s["table"].long()

    def gather(rows, scales):                               # [B][heads][tokens][D]
        return _values(rows[at], scales[at]).transpose(1, 2).flatten(2, 3)
    k, v = gather(k_rows, k_scales), gather(v_rows, v_scales)
    B, H, T, D = k.shape
    score = (s["q"].float().view(B, H, -1, D) @ k.transpose(2, 3)) * s["scale"]
    if s["cap"] > 0.0:
        score = s["cap"] * torch.tanh(score / s["cap"])
    n = torch.arange(T, device="cuda")
    length = s["length"].unsqueeze(1)
    out = n >= length
    if s["window"] > 0:
        out = out | (n < length - s["window"])
    score = score.masked_fill(out.view(B, 1, 1, T), -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    y = (p @ v) / p.sum(-1, keepdim=True)
    return dict(stored, y=y.view(B, -1).half())


def _own(s):
    from paper_2607_21985_b200 import spdp
    op, page = s["case"]["op"], s["case"].get("page")
    if op == "lora":
        spdp.spdp_lora(s["X"], s["adapter"], s["A"], s["B"], s["Y"], base=s["base"], scales=s["scales"], ranks=s["ranks"])
        return s["Y"]
    if op == "norm":
        spdp.spdp_qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["pos"], s["inv_freq"], sections=s["sections"], q_weight=s["q_weight"],
                               k_weight=s["k_weight"], eps=s["eps"], adjacent=s["adjacent"])
        return dict(q=s["q_out"], k=s["k_out"])
    spdp.spdp_kv4_store(s["k"], s["v"], s["slot"], s["cache"], page, k_values=s["k_values"], v_values=s["v_values"])
    stored = dict(k=s["k_values"], v=s["v_values"])
    if op == "store":
        return stored
    spdp.spdp_attn_kv4(s["q"], s["cache"], page, s["k"].shape[1], s["table"], s["length"], s["y"], s["scale"], cap=s["cap"], window=s["window"])
    return dict(stored, y=s["y"])


def run(state):
    if own:
        return _own(state)
    return dict(lora=_plain_lora, norm=_plain_norm, store=_plain_store, step=_plain_step)[state["case"]["op"]](state)


def work(case):
    """Every input once, every output once; of adapters and of the cache what the tokens and lengths ask for on average."""
    op = case["op"]
    if op == "lora":
        N, K, M, rank = case["N"], case["K"], case["M"], case["rank"]
        requests = -(-N // case.get("run", 1))
        used = case["adapters"] * (1.0 - (1.0 - 7.0 / 8.0 / case["adapters"]) ** requests)
        rank = (rank + 1) / 2.0 if case.get("ranks") else rank
        return dict(bytes=2.0 * N * K + 2.0 * used * rank * (K + M) + 2.0 * N * M * (4 if case["y"] == "f32" else 2) + 4.0 * N,
                    flops=2.0 * N * 7.0 / 8.0 * rank * (K + M))
    if op == "norm":
        values = float(case["N"]) * (case["q_heads"] + case["kv_heads"]) * case["dim"]
        return dict(bytes=values * (6 if case["x"] == "f32" else 4) + 4.0 * case["N"] * case["axes"], flops=8.0 * values)
    row = case["kv_heads"] * case["dim"]
    if op == "store":
        return dict(bytes=case["N"] * (row * ((8 if case["v"] == "f32" else 6) + 4 + 9 / 8.0 - 2) + 8.0), flops=8.0 * case["N"] * row)
    keys = float(case["longest"])
    if case.get("ragged"):
        keys = (keys + (case["B"] - 1) * (keys + 1) / 2.0) / case["B"]
    if case.get("window"):
        keys = min(keys, float(case["window"]))
    B = case["B"]
    return dict(bytes=B * (keys * row * 9 / 8.0 + row * (4 + 4 + 9 / 8.0) + case["q_heads"] * case["dim"] * 4.0 + keys / case["page"] * 4.0 + 12.0),
                flops=B * 4.0 * keys * case["q_heads"] * case["dim"])


def _exact_lora(s):
    out = s["base"].double().clone()
    for a in range(s["A"].shape[0]):
        r = int(s["ranks"][a])
        at = (s["adapter"] == a).nonzero().squeeze(1)
        t = torch.einsum("nk,rk->nr", s["X"][at].double(), s["A"][a, :r].double())
        out[at] += float(s["scales"][a].double()) * torch.einsum("nr,mr->nm", t, s["B"][a, :, :r].double())
    return out


def _exact_norm(s):
    half = s["inv_freq"].numel()
    axis = [a for a, n in enumerate(s["sections"]) for _ in range(n)]
    angle = torch.stack([s["pos"][a].double() * s["inv_freq"][i].double() for i, a in enumerate(axis)], 1).unsqueeze(1)
    turn = torch.polar(torch.ones_like(angle), angle)

    def one(x, weight):
        x = x.double()
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]).sqrt() * weight.double()
        first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["adjacent"] else (slice(0, half), slice(half, 2 * half))
        z = torch.complex(x[..., first], x[..., second]) * turn
        x = x.clone()
        x[..., first], x[..., second] = z.real, z.imag
        return x
    return dict(q=one(s["q"], s["q_weight"]), k=one(s["k"], s["k_weight"]))


def _exact_values(x):
    x = x.half().double()
    g = x.view(*x.shape[:-1], x.shape[-1] // 32, 32)
    scale = (g.abs().max(-1, keepdim=True).values / 7).half().double()
    steps = torch.where(scale == 0, torch.zeros_like(g), (g / scale).round().clamp(-7, 7))
    return (steps * scale).view(x.shape)


def _exact_step(s):
    case = s["case"]
    P, D, H = case["page"], case["dim"], case["kv_heads"]
    DG, n = D // 32, P * D // 2
    dims = torch.arange(D, device="cuda")
    nibble = ((dims % 32 // 8) * DG + dims // 32) * 8 + dims % 8         # where in the row a dimension's code is
    new_k, new_v = _exact_values(s["k"]), _exact_values(s["v"])
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        T = int(s["length"][b])
        lo = max(0, T - s["window"]) if s["window"] else 0
        used = s["cache"][s["table"][b, :-(-T // P)].long()].view(-1, H, P * D * 9 // 8)

        def side(first, scales, new):
            byte = used[..., first:first + n].reshape(-1, H, P, D // 2)[..., nibble // 2].int()
            code = ((byte >> (4 * (nibble % 2)).int()) & 15).double() - 8.0
            sc = used[..., scales:scales + P * DG * 2].contiguous().view(torch.float16).view(-1, H, P, DG)[..., dims // 32].double()
            x = (code * sc).permute(1, 0, 2, 3).reshape(H, -1, D)[:, :T].clone()
            x[:, T - 1] = new[b]
            return x[:, lo:]
        k, v = side(0, 2 * n, new_k), side(n, 2 * n + P * DG * 2, new_v)
        z = torch.einsum("hgd,htd->hgt", s["q"][b].double().view(H, -1, D), k) * s["scale"]
        if s["cap"] > 0.0:
            z = s["cap"] * torch.tanh(z / s["cap"])
        out[b] = torch.einsum("hgt,htd->hgd", torch.softmax(z, -1), v).reshape(-1, D)
    return dict(k=new_k, v=new_v, y=out.view(case["B"], -1))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "store":
        return dict(k=_exact_values(s["k"]), v=_exact_values(s["v"]))
    return dict(lora=_exact_lora, norm=_exact_norm, step=_exact_step)[op](s)
