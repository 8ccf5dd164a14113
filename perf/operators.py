"""The operators of a decode step over a paged key-value cache as measured calls: in a plain form made of
elementary torch operations, in the form a program calls them in (``own``), and from their definitions in 64 bits.

* plan: ``nm_page_plan``, block tables and slots from the requests' lengths;
* rope: ``nm_qk_norm_rope``, norms and rotation of queries and keys, which leave for the cache with the values;
* attn: ``nm_paged_attention``, attention of one new token per request over that cache;
* w4:   ``nm_gemv_w4``, products of a few rows with 4-bit weights.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1}


# ---- cases ------------------------------------------------------------------------------------

def listed():
    return [
        # the next token of a few requests: what a small server plans before every step
        {"name": "plan_step_8", "op": "plan", "B": 8, "page": 16, "longest": 2048, "tokens": 8},
        # prompts of 500 requests that enter together, ragged
        {"name": "plan_prompts_500", "op": "plan", "B": 500, "page": 16, "longest": 8192, "tokens": 500000},
        # one request, one token, heads of a base encoder's size, fp32 rows as nm_gemm_pwl writes them
        {"name": "rope_1_token", "op": "rope", "T": 1, "hq": 12, "hk": 12, "d": 64, "rot": 64, "norm": False, "pairs": "half",
         "x": "f32", "y": "f32", "cache": "bf16", "page": 16, "by_head": False, "far": 4096},
        # a batch's step into an int8 cache, far positions, grouped heads
        {"name": "rope_step_i8", "op": "rope", "T": 96, "hq": 16, "hk": 4, "d": 128, "rot": 64, "norm": True, "pairs": "interleaved",
         "x": "f32", "y": "bf16", "cache": "i8", "page": 32, "by_head": True, "far": 1000000},
        # prompts: the same pass over many tokens, where memory counts
        {"name": "rope_prompts", "op": "rope", "T": 16397, "hq": 32, "hk": 8, "d": 128, "rot": 128, "norm": True, "pairs": "half",
         "x": "bf16", "y": "bf16", "cache": "bf16", "page": 16, "by_head": False, "far": 32768},
        # one short conversation: latency
        {"name": "attn_1_short", "op": "attn", "B": 1, "longest": 300, "hq": 12, "hk": 12, "d": 64, "window": 0,
         "q": "f32", "cache": "bf16", "y": "f32", "page": 16, "by_head": False},
        # one request over a very long cache: few rows, split over the length
        {"name": "attn_1_long", "op": "attn", "B": 1, "longest": 131071, "hq": 32, "hk": 8, "d": 128, "window": 0,
         "q": "bf16", "cache": "bf16", "y": "bf16", "page": 16, "by_head": False},
        # a full batch of ragged lengths
        {"name": "attn_48_ragged", "op": "attn", "B": 48, "longest": 8192, "hq": 32, "hk": 8, "d": 128, "window": 0,
         "q": "bf16", "cache": "bf16", "y": "bf16", "page": 64, "by_head": True},
        # an int8 cache, as many key heads as query heads
        {"name": "attn_64_i8", "op": "attn", "B": 64, "longest": 4097, "hq": 16, "hk": 16, "d": 64, "window": 0,
         "q": "f16", "cache": "i8", "y": "f16", "page": 32, "by_head": False},
        # a projection of one row of int8 codes at a base encoder's width: latency
        {"name": "w4_1x768x768_i8", "op": "w4", "M": 1, "N": 768, "K": 768, "group": 128, "x": "i8", "s": "f32", "y": "f32"},
        # one token through a wide layer: memory
        {"name": "w4_1x14336x4096", "op": "w4", "M": 1, "N": 14336, "K": 4096, "group": 128, "x": "bf16", "s": "bf16", "y": "bf16"},
        # a batch's step through a large projection
        {"name": "w4_33x8192x8192", "op": "w4", "M": 33, "N": 8192, "K": 8192, "group": 64, "x": "bf16", "s": "f16", "y": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "rope", "attn", "w4"])
    if op == "plan":
        B = _log(rng, 1, 4096)
        return {"op": op, "B": B, "page": rng.choice([8, 16, 32, 64, 128]), "longest": _log(rng, 256, 32768),
                "tokens": _log(rng, B, max(B, 500000))}
    if op == "rope":
        d, group = rng.choice([32, 64, 80, 96, 128, 256]), rng.choice([1, 2, 4, 8])
        hk = rng.choice([1, 2, 4, 8]) if group > 1 else rng.choice([4, 8, 12, 16])
        x = rng.choice(["f32", "bf16", "f16"])
        T = _log(rng, 1, 16397 * 48 * 128 / ((group + 2) * hk * d * SIZE[x] / 2 + 1))
        return {"op": op, "T": max(1, min(T, 40000)), "hq": hk * group, "hk": hk, "d": d, "rot": rng.choice([d, d, d // 2]), "norm": rng.random() < 0.6,
                "pairs": rng.choice(["half", "interleaved"]), "x": x, "y": x, "cache": rng.choice([x, x, "i8"]),
                "page": rng.choice([8, 16, 32, 64]), "by_head": rng.random() < 0.5, "far": _log(rng, 512, 1000000)}
    if op == "attn":
        d, group = rng.choice([32, 64, 80, 96, 128, 256]), rng.choice([1, 2, 4, 5, 8, 16, 24])
        hk = rng.choice([1, 2, 4, 8]) if group > 1 else rng.choice([4, 8, 12, 16])
        q = rng.choice(["f32", "bf16", "f16"])
        cache = rng.choice(["i8", "bf16" if q == "f32" else q])
        B = _log(rng, 1, 128)
        most = 48 * 8192 * 8 * 128 * 2 / (B * hk * d * SIZE[cache])  # no more bytes of cache than the largest listed one
        most = min(most, 48 * 8192 * 32 * 128 / (B * hk * group * d))
        return {"op": op, "B": B, "longest": _log(rng, 1, max(2, min(131072, most))), "hq": hk * group, "hk": hk, "d": d,
                "window": rng.choice([0, 0, 0, 512]), "q": q, "cache": cache, "y": q, "page": rng.choice([8, 16, 32, 64, 128]),
                "by_head": rng.random() < 0.5}
    x = rng.choice(["i8", "bf16", "f16"])
    group = rng.choice([32, 64, 128, 256])
    K = group * max(1, _log(rng, 256, 16384) // group)
    N = _log(rng, 200, 8192 * 8192 / K)
    return {"op": op, "M": _log(rng, 1, 64), "N": N, "K": K, "group": group, "x": x, "s": rng.choice(["f32", "bf16", "f16"]),
            "y": "f32" if x == "i8" else x}


def _lengths(case):
    """The lengths of a case's requests, in order: none among many, one of the longest, the others spread between."""
    B, top = case["B"], case["longest"]
    if B == 1:
        return [top]
    a = [int(round(top * (i / (B - 1)) ** 1.5)) for i in range(B)]
    return a


def _fresh(case):
    """New tokens of a plan's requests: shares of the tokens there are, no request beyond its longest."""
    B = case["B"]
    a = [2 * (i + 1) * case["tokens"] // (B * (B + 1)) for i in range(B)]
    if case["tokens"] < 4 * B:
        a = [case["tokens"] // B] * B
    return [min(v, case["longest"]) for v in a]


# ---- inputs -----------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0):
    if dtype == torch.int8:
        return (torch.randn(shape, generator=g, device=DEV) * (scale * 32)).round_().clamp_(-127, 127).to(torch.int8)
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32 if dtype == torch.float32 else torch.bfloat16 if dtype == torch.bfloat16 else torch.float16)
            * scale).to(dtype)


def _pool(g, case, pages, page, hk, d, dtype, scale=1.0):
    """A cache of `pages` pages as [pages, page, hk, d], its memory by tokens or by heads, with what earlier requests left in it."""
    if case["by_head"]:
        return _normal(g, (pages, hk, page, d), dtype, scale).permute(0, 2, 1, 3)
    return _normal(g, (pages, page, hk, d), dtype, scale)


def prepare(case, seed):
    return {"plan": _prepare_plan, "rope": _prepare_rope, "attn": _prepare_attn, "w4": _prepare_w4}[case["op"]](case, seed)


def _prepare_plan(case, seed):
    g, B, page = _gen(seed), case["B"], case["page"]
    i32 = dict(dtype=torch.int32, device=DEV)
    order = torch.randperm(B, generator=g, device=DEV)
    fresh = torch.tensor(_fresh(case), **i32)[order]
    room = case["longest"] - fresh
    cached = (torch.rand(B, generator=g, device=DEV) * (room + 1)).to(torch.int32).clamp_(max=case["longest"])
    cached = torch.minimum(cached, room)
    columns = -(-case["longest"] // page)
    held = (cached + page - 1) // page
    total = B * columns + 64
    pages = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    column = torch.arange(columns, **i32)
    table = torch.where(column < held[:, None], pages[:B * columns].reshape(B, columns), torch.full((), -1, **i32)).contiguous()
    free = pages[:B * columns].reshape(B, columns)[column.expand(B, columns) >= held[:, None]]
    free = torch.cat([free[torch.randperm(free.numel(), generator=g, device=DEV)], pages[B * columns:]]).contiguous()
    T = case["tokens"]
    return {"case": case, "cached": cached, "fresh": fresh, "free": free, "begin": torch.full((1,), 7, **i32), "table": table, "num_pages": total,
            "end": torch.zeros(1, **i32), "lens": torch.zeros(B, **i32), "row_start": torch.zeros(B + 1, **i32),
            "slots": torch.zeros(T, **i32), "positions": torch.zeros(T, **i32), "requests": torch.zeros(T, **i32), "status": torch.zeros(4, **i32)}


def _prepare_rope(case, seed):
    g, T, hq, hk, d = _gen(seed), case["T"], case["hq"], case["hk"], case["d"]
    x = _normal(g, (T, hq + 2 * hk, d), DTYPE[case["x"]])  # one row holds a token's queries, keys and values, as a fused projection leaves them
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    pages = -(-(T + T // 8 + 40) // case["page"])
    slots = torch.randperm(pages * case["page"], generator=g, device=DEV)[:T].to(torch.int32)
    if T > 8:
        slots[5::97] = -1  # a padded batch's rows have no slot
    both = torch.stack([_pool(g, case, pages, case["page"], hk, d, DTYPE[case["cache"]]) for _ in range(2)])
    if case["by_head"]:
        both = both.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
    s = {"case": case, "q": q, "k": k, "v": v, "slots": slots, "cache": both,
         "positions": torch.randint(0, case["far"], (T,), generator=g, device=DEV, dtype=torch.int32),
         "inv_freq": (10000.0 ** (-torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float64) / max(case["rot"], 1))).float(),
         "q_gamma": 1 + 0.1 * torch.randn(d, generator=g, device=DEV) if case["norm"] else None,
         "k_gamma": 1 + 0.1 * torch.randn(d, generator=g, device=DEV) if case["norm"] else None,
         "q_out": torch.empty((T, hq, d), dtype=DTYPE[case["y"]], device=DEV), "inv_scale": None, "scale": None}
    if case["cache"] == "i8":
        s["scale"] = (3.5 + torch.rand((2, hk), generator=g, device=DEV)) / 127
        s["inv_scale"] = 1 / s["scale"]
    return s


def _prepare_attn(case, seed):
    g, B, hq, hk, d, page = _gen(seed), case["B"], case["hq"], case["hk"], case["d"], case["page"]
    order = torch.randperm(B, generator=g, device=DEV)
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)[order]
    columns = -(-case["longest"] // page)
    held = [-(-n // page) for n in _lengths(case)]
    pages = sum(held) + 16
    used = torch.arange(columns, device=DEV) < ((lens + page - 1) // page)[:, None]
    table = torch.full((B, columns), -1, dtype=torch.int32, device=DEV)
    table[used] = torch.randperm(pages, generator=g, device=DEV)[:sum(held)].to(torch.int32)
    cache = DTYPE[case["cache"]]
    s = {"case": case, "q": _normal(g, (B, hq, d), DTYPE[case["q"]]), "lens": lens, "table": table,
         "k": _pool(g, case, pages, page, hk, d, cache), "v": _pool(g, case, pages, page, hk, d, cache),
         "scale": d ** -0.5, "k_scale": None, "v_scale": None,
         "out": torch.empty((B, hq, d), dtype=DTYPE[case["y"]], device=DEV), "lse": torch.empty((B, hq), dtype=torch.float32, device=DEV)}
    if case["cache"] == "i8":
        s["k_scale"], s["v_scale"] = ((3.5 + torch.rand(hk, generator=g, device=DEV)) / 127 for _ in range(2))
    return s


def _prepare_w4(case, seed):
    g, M, N, K = _gen(seed), case["M"], case["N"], case["K"]
    code = torch.randn((N, K), generator=g, device=DEV, dtype=torch.float16).mul_(2.5).round_().clamp_(-8, 7).to(torch.int8)
    W = ((code[:, 0::2] & 15) | (code[:, 1::2] << 4)).view(torch.uint8)
    scales = (0.02 * (0.5 + torch.rand((N, K // case["group"]), generator=g, device=DEV))).to(DTYPE[case["s"]])
    return {"case": case, "x": _normal(g, (M, K), DTYPE[case["x"]]), "W": W.contiguous(), "scales": scales, "alpha": 0.03 if case["x"] == "i8" else 1.0,
            "bias": torch.randn(N, generator=g, device=DEV), "out": torch.empty((M, N), dtype=DTYPE[case["y"]], device=DEV)}


# ---- one pass ---------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"plan": _own_plan, "rope": _own_rope, "attn": _own_attn, "w4": _own_w4}[op](state)
    return {"plan": _plain_plan, "rope": _plain_rope, "attn": _plain_attn, "w4": _plain_w4}[op](state)


def _own_plan(s):
    from paper_2305_14405_amd import binding as nm
    nm.nm_page_plan(s["cached"], s["fresh"], s["free"], s["begin"], s["table"], page_size=s["case"]["page"], num_pages=s["num_pages"],
                    free_end=s["end"], lens=s["lens"], row_start=s["row_start"], slots=s["slots"], positions=s["positions"],
                    requests=s["requests"], status=s["status"])
    return [s[n] for n in ("table", "end", "lens", "row_start", "slots", "positions", "requests", "status")]


def _own_rope(s):
    from paper_2305_14405_amd import binding as nm
    c, cache, inv = s["case"], s["cache"], s["inv_scale"]
    nm.nm_qk_norm_rope(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["q_out"], interleaved=c["pairs"] == "interleaved",
                       norm=c["norm"], q_gamma=s["q_gamma"], k_gamma=s["k_gamma"], eps=1e-6, k_cache=cache[0], v_cache=cache[1],
                       slots=s["slots"], k_inv_scale=None if inv is None else inv[0], v_inv_scale=None if inv is None else inv[1])
    return [s["q_out"], _values(s)]


def _own_attn(s):
    from paper_2305_14405_amd import binding as nm
    c = s["case"]
    args = (s["q"], s["k"], s["v"], s["table"], s["lens"], s["out"])
    more = dict(scale=s["scale"], window=c["window"], k_scale=s["k_scale"], v_scale=s["v_scale"], lse=s["lse"])
    if "ws" not in s:  # kept by the program, as the other calls' workspaces are
        s["ws"] = torch.empty(nm.nm_paged_attention_workspace(*args, **more), dtype=torch.uint8, device=DEV)
    nm.nm_paged_attention(*args, ws=s["ws"], **more)
    return [s["out"], s["lse"]]


def _own_w4(s):
    from paper_2305_14405_amd import binding as nm
    nm.nm_gemv_w4(s["x"], s["W"], s["scales"], s["out"], group=s["case"]["group"], alpha=s["alpha"], bias=s["bias"])
    return s["out"]


def _plain_plan(s):
    c, page = s["case"], s["case"]["page"]
    cached, fresh, free, table = s["cached"].long(), s["fresh"].long(), s["free"].long(), s["table"].long()
    columns, tokens, begin = table.shape[1], c["tokens"], s["begin"].long()
    after = cached + fresh
    have, want = (cached + page - 1) // page, (after + page - 1) // page
    need = torch.where(fresh > 0, want - have, 0)
    page_end, row_end = need.cumsum(0), fresh.cumsum(0)
    n_pages, n_tokens = page_end[-1], row_end[-1]
    flags = ((begin[0] + n_pages > free.numel()) * 1 + (want > columns).any() * 2 + (n_tokens > tokens) * 4 + ((cached < 0) | (fresh < 0)).any() * 8)
    ok = flags == 0
    column = torch.arange(columns, device=table.device)
    at = (begin + page_end - need)[:, None] + column - have[:, None]
    new = (column >= have[:, None]) & (column < (have + need)[:, None]) & ok
    table = torch.where(new, free[at.clamp(0, free.numel() - 1)], table)
    t = torch.arange(tokens, device=table.device)
    row = torch.searchsorted(row_end, t, right=True)
    real = (t < n_tokens) & ok
    row = row.clamp(max=c["B"] - 1)
    position = cached[row] + t - (row_end - fresh)[row]
    held = table[row, (position // page).clamp(0, columns - 1)]
    good = real & (held >= 0) & (held < s["num_pages"])
    s["table"].copy_(table)
    i32 = torch.int32
    start = torch.cat([torch.zeros_like(row_end[:1]), row_end]) * ok
    return [s["table"], (begin + n_pages * ok).to(i32), torch.where(ok, after, cached).to(i32), start.to(i32),
            torch.where(good, held * page + position % page, -1).to(i32), torch.where(real, position, 0).to(i32), torch.where(real, row, -1).to(i32),
            torch.stack([flags, n_tokens, n_pages, after.max()]).to(i32)]


def _values(s):
    """What the cache holds: codes as the values they stand for."""
    if s["scale"] is None:
        return s["cache"]
    if "values" not in s:
        s["values"] = torch.empty(s["cache"].shape, dtype=torch.bfloat16, device=DEV)
    return torch.mul(s["cache"], s["scale"][:, None, None, :, None], out=s["values"])


def _plain_turn(x, s, gamma):
    c = s["case"]
    x = x.float()
    if c["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gamma
    if c["rot"] == 0:
        return x
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    r = x[..., :c["rot"]]
    if c["pairs"] == "half":
        a, b = r[..., :c["rot"] // 2], r[..., c["rot"] // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., c["rot"]:]], -1)


def _plain_rope(s):
    q, k, v = _plain_turn(s["q"], s, s["q_gamma"]), _plain_turn(s["k"], s, s["k_gamma"]), s["v"].float()
    new, cache = torch.stack([k, v]), s["cache"]
    _, pages, page, hk, d = cache.shape
    if s["inv_scale"] is not None:
        new = (new * s["inv_scale"][:, None, :, None]).round().clamp(-127, 127)
    slots, n = s["slots"].long(), pages * page
    writer = torch.full((n + 1,), -1, device=DEV).index_copy(0, torch.where(slots < 0, n, slots), torch.arange(slots.numel(), device=DEV))[:n].view(pages, page)
    cache.copy_(torch.where((writer >= 0)[None, :, :, None, None], new.to(cache.dtype)[:, writer.clamp(min=0)], cache))
    return [q.to(DTYPE[s["case"]["y"]]), _values(s)]


def _plain_attn(s):
    c, q, lens = s["case"], s["q"].float(), s["lens"]
    B, hq, d = q.shape
    hk, page, L = c["hk"], c["page"], c["longest"]
    j = torch.arange(L, device=DEV)
    seen = j < lens[:, None]
    if c["window"]:
        seen = seen & (j >= lens[:, None] - c["window"])
    held = s["table"].long()[:, j // page].clamp(min=0)
    k, v = s["k"][held, j % page].permute(0, 2, 3, 1).float().contiguous(), s["v"][held, j % page].permute(0, 2, 1, 3).float().contiguous()
    v = v * seen[:, None, :, None]
    if s["k_scale"] is not None:
        k, v = k * s["k_scale"][:, None, None], v * s["v_scale"][:, None, None]
    scores = torch.matmul(q.view(B, hk, hq // hk, d), k) * s["scale"]
    scores = torch.where(seen[:, None, None], scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
    return [out.view(B, hq, d).to(DTYPE[c["y"]]), (top + total.log()).view(B, hq)]


def _plain_w4(s):
    c = s["case"]
    code = s["W"].view(torch.int8)
    w = torch.stack([(code << 4) >> 4, code >> 4], -1).view(c["N"], c["K"] // c["group"], c["group"])  # arithmetic shifts of signed bytes
    w = (w.float() * s["scales"].float()[:, :, None]).view(c["N"], c["K"])
    return (torch.matmul(s["x"].float(), w.t()) * s["alpha"] + s["bias"]).to(DTYPE[c["y"]])


# ---- what one pass cannot do without ------------------------------------------------------------

def work(case):
    if case["op"] == "plan":
        pages = sum(_fresh(case)) // case["page"]
        return {"bytes": 16 * case["B"] + 12 * case["tokens"] + 8 * pages + 32, "flops": 4 * case["tokens"]}
    if case["op"] == "rope":
        T, hq, hk, d = (case[n] for n in ("T", "hq", "hk", "d"))
        moved = (hq + 2 * hk) * SIZE[case["x"]] + hq * SIZE[case["y"]] + 2 * hk * SIZE[case["cache"]]
        return {"bytes": T * d * moved + 8 * T, "flops": 8 * T * (hq + hk) * d}
    if case["op"] == "attn":
        n = sum(min(v, case["window"] or v) for v in _lengths(case))
        B, hq, hk, d = (case[n] for n in ("B", "hq", "hk", "d"))
        return {"bytes": 2 * n * hk * d * SIZE[case["cache"]] + 4 * n // case["page"] + B * hq * (d * (SIZE[case["q"]] + SIZE[case["y"]]) + 4),
                "flops": 4 * n * hq * d}
    M, N, K = case["M"], case["N"], case["K"]
    return {"bytes": N * K // 2 + N * (K // case["group"]) * SIZE[case["s"]] + M * K * SIZE[case["x"]] + M * N * SIZE[case["y"]] + 4 * N, "flops": 2 * M * N * K}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "plan":
        return None  # whole numbers
    if case["op"] == "rope":
        return _exact_rope(case, s)
    if case["op"] == "attn":
        return _exact_attn(case, s)
    out = torch.empty((case["M"], case["N"]), dtype=torch.float64, device=DEV)
    x, G = s["x"].double(), case["group"]
    for n0 in range(0, case["N"], 1024):
        rows = s["W"][n0:n0 + 1024].long()
        w = torch.empty((rows.shape[0], case["K"]), dtype=torch.float64, device=DEV)
        for half in (0, 1):
            u = (rows // 16 if half else rows % 16)
            w[:, half::2] = torch.where(u >= 8, u - 16, u).double()
        w *= s["scales"][n0:n0 + 1024].double().repeat_interleave(G, 1)
        out[:, n0:n0 + 1024] = x @ w.T.contiguous()
    return out * s["alpha"] + s["bias"].double()


def _exact_rope(case, s):
    def turned(x, gamma):
        y = x.double().clone()
        if case["norm"]:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / case["d"] + 1e-6) * gamma.double()
        out, half = y.clone(), case["rot"] // 2
        for i in range(half):
            a, b = (i, i + half) if case["pairs"] == "half" else (2 * i, 2 * i + 1)
            phase = (s["positions"].double() * s["inv_freq"][i].double())[:, None]
            out[..., a] = y[..., a] * torch.cos(phase) - y[..., b] * torch.sin(phase)
            out[..., b] = y[..., a] * torch.sin(phase) + y[..., b] * torch.cos(phase)
        return out

    page, there = case["page"], s["slots"] >= 0
    at = s["slots"][there].long()
    cache = s["cache"].double()
    for n, x in enumerate((turned(s["k"], s["k_gamma"]), s["v"].double())):
        x = x[there]
        if s["inv_scale"] is not None:
            x = torch.clamp(torch.round(x * s["inv_scale"][n].double()[:, None]), -127, 127)
        cache[n, at // page, at % page] = x
    if s["scale"] is not None:
        cache = cache * s["scale"].double()[:, None, None, :, None]
    return [turned(s["q"], s["q_gamma"]), cache]


def _exact_attn(case, s):
    B, hq, hk, d, page = (case[n] for n in ("B", "hq", "hk", "d", "page"))
    out = torch.zeros((B, hq, d), dtype=torch.float64, device=DEV)
    lse = torch.full((B, hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        where = torch.arange(max(0, n - case["window"]) if case["window"] else 0, n, device=DEV)
        rows = s["table"][b].long()[where // page]
        k, v = (s[name][rows, where % page].double() for name in ("k", "v"))
        if case["cache"] == "i8":
            k, v = k * s["k_scale"].double()[:, None], v * s["v_scale"].double()[:, None]
        for h in range(hk):
            group = slice(h * (hq // hk), (h + 1) * (hq // hk))
            z = s["q"][b, group].double() @ k[:, h].T.contiguous() * s["scale"]
            lse[b, group] = torch.logsumexp(z, -1)
            out[b, group] = torch.softmax(z, -1) @ v[:, h].contiguous()
    return [out, lse]
