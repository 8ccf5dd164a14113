"""The operators of decoding with several hypotheses per request, over a paged key-value cache, as measured calls: in a plain form
made of elementary torch operations, in the form a program calls them in (``own``), and from their definitions in 64 bits.

* beam: ``nm_beam_select``, the next hypotheses of every request from its hypotheses' logits, and their histories;
* fork: ``nm_page_fork``, block tables of the next hypotheses from those of their parents: pages shared, copied on write, freed;
* copy: ``nm_page_copy``, the copies of pages that this asks for, in every layer's caches;
* attn: ``nm_shared_attention``, attention of one new token per row where groups of rows share a prefix.
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
        # four hypotheses of one request, fp32 logits as nm_gemm_pwl writes them: latency
        {"name": "beam_1x4", "op": "beam", "R": 1, "W": 4, "K": 4, "V": 32000, "x": "f32", "done": 0.0, "weight": False, "banned": 0.0, "history": 0},
        # an odd vocabulary, some hypotheses finished, ranked by their lengths, histories that follow
        {"name": "beam_24x6_finished", "op": "beam", "R": 24, "W": 6, "K": 6, "V": 50001, "x": "f16", "done": 0.25, "weight": True, "banned": 0.02,
         "history": 700},
        # a batch that keeps twice as many candidates as it has hypotheses, a large vocabulary: memory
        {"name": "beam_32x8_large", "op": "beam", "R": 32, "W": 8, "K": 16, "V": 131072, "x": "bf16", "done": 0.0, "weight": False, "banned": 0.0, "history": 0},
        # many requests with narrow beams and long histories
        {"name": "beam_300x2_histories", "op": "beam", "R": 300, "W": 2, "K": 2, "V": 32003, "x": "bf16", "done": 0.1, "weight": True, "banned": 0.0,
         "history": 4000},
        # four requests of four hypotheses: what a small server does after every step
        {"name": "fork_4x4", "op": "fork", "R": 4, "W": 4, "page": 16, "longest": 2048, "tail": 100, "keep": False, "gone": 0.0},
        # as many rows as a plan takes, prompts that a prefix cache keeps, some hypotheses given up
        {"name": "fork_512x8", "op": "fork", "R": 512, "W": 8, "page": 16, "longest": 8192, "tail": 200, "keep": True, "gone": 0.1},
        # a small model's twelve layers, the copies of four requests of four hypotheses
        {"name": "copy_16_of_24", "op": "copy", "n": 16, "caches": 24, "hk": 12, "d": 64, "x": "bf16", "page": 16, "by_head": False, "share": 0.5},
        # 256 rows through 32 layers
        {"name": "copy_256_of_64", "op": "copy", "n": 256, "caches": 64, "hk": 8, "d": 128, "x": "bf16", "page": 32, "by_head": True, "share": 0.6},
        # four hypotheses of one short conversation: latency
        {"name": "attn_1x4_short", "op": "attn", "G": 1, "W": 4, "prefix": 600, "tail": 40, "even": True, "hq": 12, "hk": 12, "d": 64,
         "q": "f32", "cache": "bf16", "y": "f32", "page": 16, "by_head": False},
        # hypotheses of a batch of ragged prompts, int8 caches
        {"name": "attn_16x8_i8", "op": "attn", "G": 16, "W": 8, "prefix": 8192, "tail": 130, "even": True, "hq": 16, "hk": 16, "d": 64,
         "q": "f16", "cache": "i8", "y": "f16", "page": 32, "by_head": False},
        # 64 answers sampled about one long document
        {"name": "attn_1x64_document", "op": "attn", "G": 1, "W": 64, "prefix": 32768, "tail": 512, "even": False, "hq": 32, "hk": 8, "d": 128,
         "q": "bf16", "cache": "bf16", "y": "bf16", "page": 16, "by_head": False},
        # a server's requests behind common instructions, each with a conversation of its own
        {"name": "attn_1x96_instructions", "op": "attn", "G": 1, "W": 96, "prefix": 4097, "tail": 4096, "even": False, "hq": 32, "hk": 8, "d": 128,
         "q": "bf16", "cache": "bf16", "y": "bf16", "page": 64, "by_head": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["beam", "beam", "fork", "copy", "attn", "attn"])
    if op == "beam":
        x = rng.choice(["f32", "bf16", "f16"])
        V, W = _log(rng, 1000, 262144), rng.choice([1, 2, 3, 4, 5, 8, 10, 16, 32])
        R = _log(rng, 1, min(512, 32 * 8 * 131072 * 2 / (V * W * SIZE[x])))
        return {"op": op, "R": R, "W": W, "K": rng.choice([W, W, min(64, 2 * W)]), "V": V, "x": x, "done": rng.choice([0.0, 0.2]),
                "weight": rng.random() < 0.5, "banned": rng.choice([0.0, 0.01]), "history": _log(rng, 1, 4000) if rng.random() < 0.5 else 0}
    if op == "fork":
        W = rng.choice([1, 2, 3, 4, 5, 8, 12])
        return {"op": op, "R": _log(rng, 1, 4096 // W), "W": W, "page": rng.choice([8, 16, 32, 64, 128]), "longest": _log(rng, 64, 4096), "tail": _log(rng, 1, 200),
                "keep": rng.random() < 0.5, "gone": rng.choice([0.0, 0.0, 0.2])}
    if op == "copy":
        d, x = rng.choice([32, 64, 80, 96, 128, 256]), rng.choice(["f32", "bf16", "f16"])
        hk, page, caches = rng.choice([1, 2, 4, 8, 12, 16]), rng.choice([8, 16, 32, 64]), rng.choice([2, 12, 24, 48, 64, 80])
        n = _log(rng, 1, 256 * 64 * 32 * 8 * 128 * 2 / (caches * page * hk * d * SIZE[x]))
        return {"op": op, "n": min(n, 1024), "caches": caches, "hk": hk, "d": d, "x": x, "page": page, "by_head": rng.random() < 0.5,
                "share": rng.choice([0.2, 0.5, 0.8, 1.0])}
    d, group = rng.choice([32, 64, 80, 96, 128, 256]), rng.choice([1, 2, 4, 5, 8, 16])
    hk = rng.choice([1, 2, 4, 8]) if group > 1 else rng.choice([4, 8, 12, 16])
    q = rng.choice(["f32", "bf16", "f16"])
    cache = rng.choice(["i8", "bf16" if q == "f32" else q])
    G, W = _log(rng, 1, 32), _log(rng, 2, 64)
    rows = 64 * 32768 * 32 * 128 / (G * W * hk * group * d)                   # no more products than the largest listed one
    held = 96 * 2048 * 8 * 128 * 2 / (hk * d * SIZE[cache])                   # nor bytes of cache
    tail = _log(rng, 1, max(2, min(4096, rows / 2, held / (G * W))))
    return {"op": op, "G": G, "W": W, "prefix": _log(rng, 16, max(32, min(32768, rows / 2, held / G))), "tail": tail, "even": rng.random() < 0.5, "hq": hk * group,
            "hk": hk, "d": d, "q": q, "cache": cache, "y": q, "page": rng.choice([8, 16, 32, 64, 128]), "by_head": rng.random() < 0.5}


def _spread(n, top, least=1):
    """n lengths up to top, in order: the longest last, none below least."""
    if n == 1:
        return [top]
    return [max(least, int(round(top * ((i + 1) / n) ** 1.5))) for i in range(n)]


# ---- inputs -----------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0):
    if dtype == torch.int8:
        return (torch.randn(shape, generator=g, device=DEV) * (scale * 32)).round_().clamp_(-127, 127).to(torch.int8)
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype) * scale


def _pool(g, case, lead, pages, page, hk, d, dtype):
    """Caches of `pages` pages as [*lead, pages, page, hk, d], their memory by tokens or by heads, with what earlier requests left in it."""
    if case["by_head"]:
        return _normal(g, (*lead, pages, hk, page, d), dtype).transpose(-2, -3)
    return _normal(g, (*lead, pages, page, hk, d), dtype)


def _order(seed, n):
    c = torch.Generator()
    c.manual_seed(seed)
    return torch.randperm(n, generator=c).tolist()


def prepare(case, seed):
    return {"beam": _prepare_beam, "fork": _prepare_fork, "copy": _prepare_copy, "attn": _prepare_attn}[case["op"]](case, seed)


def _prepare_beam(case, seed):
    g, R, W, K, V = _gen(seed), case["R"], case["W"], case["K"], case["V"]
    i32 = dict(dtype=torch.int32, device=DEV)
    x = _normal(g, (R * W, V), DTYPE[case["x"]], 2.5)
    if case["banned"]:
        x.masked_fill_(torch.rand(V, generator=g, device=DEV) < case["banned"], -math.inf)   # tokens that no one may take
    # the hypotheses of a request lie some units apart; in a first step only one is alive
    scores = -20 * torch.rand((R, 1), generator=g, device=DEV) - 4 * torch.rand((R, W), generator=g, device=DEV)
    if W > 1 and R > 2:
        scores[1, 1:] = -math.inf
    s = {"case": case, "x": x, "scores": scores, "done": None, "weight": None, "end": 2,
         "parents": torch.empty((R, K), **i32), "tokens": torch.empty((R, K), **i32), "totals": torch.empty((R, K), device=DEV),
         "done_out": torch.empty((R, K), **i32), "history": None}
    if case["done"]:
        s["done"] = (torch.rand((R, W), generator=g, device=DEV) < case["done"]).to(torch.int32)
    if case["weight"]:
        s["weight"] = 1 / (5 + 20 * torch.rand((R, W), generator=g, device=DEV)) ** 0.6
    if case["history"]:
        n = case["history"]
        s["history"] = torch.randint(0, V, (R * W, n + 1), generator=g, **i32)
        s["held"] = torch.randint(n // 2, n + 1, (R * W,), generator=g, **i32)
        s["history_out"], s["held_out"] = torch.zeros((R * K, n + 1), **i32), torch.empty(R * K, **i32)
    return s


def _prepare_fork(case, seed):
    g, R, W, page = _gen(seed), case["R"], case["W"], case["page"]
    i32 = dict(dtype=torch.int32, device=DEV)
    B, order = R * W, _order(seed, R)
    prompt = torch.tensor(_spread(R, case["longest"]), device=DEV)[torch.tensor(order, device=DEV)].repeat_interleave(W)
    lens = prompt + torch.randint(1, case["tail"] + 1, (R,), generator=g, device=DEV).repeat_interleave(W)
    columns, tail = -(-(case["longest"] + case["tail"]) // page), -(-case["tail"] // page) + 1
    col = torch.arange(columns, device=DEV)
    row = torch.arange(B, device=DEV)
    whole = (prompt // page)[:, None]
    # behind the prompt's whole pages a hypothesis has pages of its own, but for those that it shares with the one in front of it
    older = torch.where((row % W > 0) & (row % W % 2 == 1), torch.rand(B, generator=g, device=DEV) * (lens // page - prompt // page + 1), 0).long()[:, None]
    shared = torch.div(row, W, rounding_mode="floor")[:, None] * columns + col
    of = torch.where(col - whole < older, row[:, None] - 1, row[:, None])
    mine = R * columns + of * tail + (col - whole).clamp(0, tail - 1)
    total = R * columns + B * tail + B + 64
    pages = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    held = col < (lens[:, None] + page - 1) // page
    table = torch.where(held, pages[torch.where(col < whole, shared, mine)], -1).contiguous()
    used = torch.zeros(total + 1, dtype=torch.bool, device=DEV)
    used[torch.where(held, table, total).long().flatten()] = True
    used[total] = False
    parents = (row // W * W + torch.randint(0, W, (B,), generator=g, device=DEV)).to(torch.int32)
    if case["gone"]:
        parents[torch.rand(B, generator=g, device=DEV) < case["gone"]] = -1
    keep = None
    if case["keep"]:
        keep = torch.zeros(total, **i32)
        keep[table[:, 0].long()[lens >= page]] = 1
    free = pages[~used[pages.long()]]
    begin = total - free.numel()
    return {"case": case, "table": table, "lens": lens.to(torch.int32), "parents": parents, "pages": total, "keep": keep,
            "free": torch.cat([torch.zeros(begin, **i32), free]).contiguous(), "begin": torch.full((1,), begin, **i32),
            "table_out": torch.full((B, columns), -1, **i32), "lens_out": torch.zeros(B, **i32), "free_out": torch.zeros(total, **i32), "end": torch.zeros(1, **i32),
            "src": torch.zeros(B, **i32), "dst": torch.zeros(B, **i32), "slots": torch.zeros(B, **i32), "status": torch.zeros(4, **i32)}


def _prepare_copy(case, seed):
    g, n, page = _gen(seed), case["n"], case["page"]
    pages = 2 * n + 9
    perm = 1 + torch.randperm(pages - 1, generator=g, device=DEV).to(torch.int32)   # page 0 is in no copy
    src, dst = perm[:n].clone(), perm[n:2 * n].clone()
    if n > 1:
        none = torch.rand(n, generator=g, device=DEV) >= case["share"]       # rows that keep their last page
        src[none], dst[none] = -1, -1
    slots = torch.randint(1, page, (n,), generator=g, device=DEV).to(torch.int32)
    slots[src < 0] = 0
    return {"case": case, "src": src, "dst": dst, "slots": slots,
            "cache": _pool(g, case, (case["caches"],), pages, page, case["hk"], case["d"], DTYPE[case["x"]])}


def _lengths(case):
    """Of each group, in order: its prefix, and the rows' own positions behind its whole pages."""
    G, W, tail = case["G"], case["W"], case["tail"]
    prompts = _spread(G, case["prefix"])
    steps = _spread(G, tail)
    out = []
    for i in range(G):
        rest = prompts[i] % case["page"]                                     # a page that is not full is every row's own
        out.append((prompts[i] - rest, [rest + (steps[i] if case["even"] else n) for n in _spread(W, tail)]))
    return out


def _prepare_attn(case, seed):
    g, G, W, hq, hk, d, page = _gen(seed), case["G"], case["W"], case["hq"], case["hk"], case["d"], case["page"]
    i32 = dict(dtype=torch.int32, device=DEV)
    groups = [_lengths(case)[i] for i in _order(seed, G)]
    groups = [(p, [tails[j] for j in _order(seed + 1 + i, W)]) for i, (p, tails) in enumerate(groups)]
    lens = [p + n for p, tails in groups for n in tails]
    columns = -(-max(lens) // page)
    pages = sum(p // page + sum(-(-n // page) for n in tails) for p, tails in groups) + 16
    perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table, at = torch.full((G * W, columns), -1, **i32), 0
    for i, (p, tails) in enumerate(groups):
        first = p // page
        table[i * W:(i + 1) * W, :first] = perm[at:at + first]
        at += first
        for j, n in enumerate(tails):
            more = -(-n // page)
            table[i * W + j, first:first + more] = perm[at:at + more]
            at += more
    cache = DTYPE[case["cache"]]
    s = {"case": case, "q": _normal(g, (G * W, hq, d), DTYPE[case["q"]]), "table": table, "groups": groups, "lens": torch.tensor(lens, **i32),
         "start": torch.arange(0, G * W + 1, W, **i32), "shared": torch.tensor([p for p, _ in groups], **i32),
         "k": _pool(g, case, (), pages, page, hk, d, cache), "v": _pool(g, case, (), pages, page, hk, d, cache), "scale": d ** -0.5, "k_scale": None, "v_scale": None,
         "out": torch.empty((G * W, hq, d), dtype=DTYPE[case["y"]], device=DEV), "lse": torch.empty((G * W, hq), dtype=torch.float32, device=DEV)}
    if case["cache"] == "i8":
        s["k_scale"], s["v_scale"] = ((3.5 + torch.rand(hk, generator=g, device=DEV)) / 127 for _ in range(2))
    return s


# ---- one pass ---------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"beam": _own_beam, "fork": _own_fork, "copy": _own_copy, "attn": _own_attn}[op](state)
    return {"beam": _plain_beam, "fork": _plain_fork, "copy": _plain_copy, "attn": _plain_attn}[op](state)


def _workspace(s, bytes_of, *args, **more):
    """Kept by the program, as the other calls' workspaces are."""
    if "ws" not in s:
        s["ws"] = torch.empty(bytes_of(*args, **more), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _own_beam(s):
    from paper_2305_14405_amd import binding as nm
    args = (s["x"], s["scores"], s["parents"], s["tokens"], s["totals"])
    more = dict(done=s["done"], weight=s["weight"], end_token=s["end"], done_out=s["done_out"])
    if s["history"] is not None:
        more.update(history=s["history"], history_lens=s["held"], history_out=s["history_out"], history_lens_out=s["held_out"])
    nm.nm_beam_select(*args, ws=_workspace(s, nm.nm_beam_select_workspace, *args, **more), **more)
    return [s["parents"], s["tokens"], s["totals"], s["done_out"]] + ([] if s["history"] is None else [s["history_out"], s["held_out"]])


def _own_fork(s):
    from paper_2305_14405_amd import binding as nm
    args = (s["table"], s["lens"], s["parents"], s["free"], s["begin"], s["table_out"])
    more = dict(page_size=s["case"]["page"], num_pages=s["pages"], keep=s["keep"], lens_out=s["lens_out"], free_out=s["free_out"], free_end=s["end"],
                copy_src=s["src"], copy_dst=s["dst"], copy_slots=s["slots"], status=s["status"])
    nm.nm_page_fork(*args, ws=_workspace(s, nm.nm_page_fork_workspace, *args, **more), **more)
    return [s[n] for n in ("table_out", "lens_out", "free_out", "end", "src", "dst", "slots", "status")]


def _own_copy(s):
    from paper_2305_14405_amd import binding as nm
    if "desc" not in s:  # a program's caches stay where they are
        s["desc"] = nm.make_copy_desc(s["cache"], s["src"], s["dst"], s["slots"])
    nm.nm_page_copy(s["desc"])
    return s["cache"]


def _own_attn(s):
    from paper_2305_14405_amd import binding as nm
    args = (s["q"], s["k"], s["v"], s["table"], s["lens"], s["start"], s["shared"], s["out"])
    more = dict(scale=s["scale"], k_scale=s["k_scale"], v_scale=s["v_scale"], lse=s["lse"])
    nm.nm_shared_attention(*args, ws=_workspace(s, nm.nm_shared_attention_workspace, *args, **more), **more)
    return [s["out"], s["lse"]]


def _plain_beam(s):
    c = s["case"]
    R, W, K, V = (c[n] for n in ("R", "W", "K", "V"))
    x = s["x"].float() + 0.0                                                  # zeros of either sign are one value
    top = x.amax(-1, keepdim=True)
    lse = top[:, 0].double() + torch.exp(x - top).double().sum(-1).log()
    bits = x.view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7fffffff)).long()                       # as whole numbers, in the order of the values
    key = order * (1 << 32) + (V - 1 - torch.arange(V, device=DEV))          # of equal ones the lowest token first
    n = min(K, V)
    key = torch.topk(key, n, -1).values
    token = V - 1 - (key & 0xffffffff)
    best = torch.gather(x, 1, token).double()
    total = s["scores"].double()[:, :, None] + (best - lse[:, None]).view(R, W, n)
    token = token.view(R, W, n)
    if s["done"] is not None:
        over = (s["done"] != 0)[:, :, None]
        first = torch.arange(n, device=DEV) == 0
        total = torch.where(over, torch.where(first, s["scores"].double()[:, :, None], -math.inf), total)
        token = torch.where(over, s["end"], token)
    rank = total if s["weight"] is None else torch.where(total == -math.inf, total, total * s["weight"].double()[:, :, None])
    n = min(K, W * n)
    rank, at = torch.sort(rank.view(R, -1), dim=-1, descending=True, stable=True)
    rank, at = rank[:, :n], at[:, :n]
    there = rank > -math.inf
    total, token = torch.gather(total.view(R, -1), 1, at), torch.gather(token.view(R, -1), 1, at)
    parent = at // min(K, V) + torch.arange(R, device=DEV)[:, None] * W
    pad = K - n
    parent = torch.nn.functional.pad(torch.where(there, parent, -1), (0, pad), value=-1)
    token = torch.nn.functional.pad(torch.where(there, token, -1), (0, pad), value=-1)
    total = torch.nn.functional.pad(torch.where(there, total, -math.inf), (0, pad), value=-math.inf)
    was = torch.zeros_like(parent, dtype=torch.bool) if s["done"] is None else (s["done"] != 0).view(-1)[parent.clamp(min=0)] & (parent >= 0)
    i32 = torch.int32
    out = [parent.to(i32), token.to(i32), total.float(), (was | (token == s["end"])).to(i32)]
    if s["history"] is not None:
        row = parent.view(-1).clamp(min=0)
        held = torch.where(parent.view(-1) >= 0, s["held"].long()[row], 0)
        place = torch.arange(s["history"].shape[1], device=DEV)
        grows = (parent.view(-1) >= 0) & ~was.view(-1) & (held < place.numel())
        new = torch.where(place < held[:, None], s["history"][row].long(), s["history_out"].long())
        new = torch.where((place == held[:, None]) & grows[:, None], token.view(-1)[:, None], new)
        s["history_out"].copy_(new)
        out += [s["history_out"], (held + grows).to(i32)]
    return out


def _plain_fork(s):
    page, total = s["case"]["page"], s["pages"]
    table, lens, free, begin = s["table"].long(), s["lens"].long(), s["free"].long(), s["begin"].long()
    B, columns = table.shape
    col, row = torch.arange(columns, device=DEV), torch.arange(B, device=DEV)
    parent = s["parents"].long()
    lives = (parent >= 0) & (parent < B)
    p = torch.where(lives, parent, 0)
    first = torch.full((B + 1,), B, device=DEV).scatter_reduce_(0, torch.where(lives, parent, B), row, "amin")[:B]   # lowest child
    held = (lens + page - 1) // page
    whole = lens // page
    is_page = (table >= 0) & (table < total)
    # marks: anybody's, a living row's in front of its last page where that is not full, that page
    def marked(where):
        return torch.zeros(total + 1, dtype=torch.long, device=DEV).index_add_(0, torch.where(where & is_page, table, total).flatten(),
                                                                              torch.ones_like(table).flatten())[:total]
    living = (first < B)[:, None]
    old, full = marked(col < held[:, None]) > 0, marked((col < whole[:, None]) & living) > 0
    part = marked((col >= whole[:, None]) & (col < held[:, None]) & living)
    kept = torch.zeros_like(old) if s["keep"] is None else s["keep"] != 0
    last = table.gather(1, whole.clamp(max=columns - 1)[:, None])[:, 0]
    partial = (lens % page != 0) & (last >= 0) & (last < total)
    at = last.clamp(0, total - 1)
    apart = (part[at] > 1) | full[at] | kept[at]
    need = lives & partial[p] & (apart[p] | (first[p] != row))
    ends = need.long().cumsum(0)
    taken = ends[-1]
    gone = old & ~full & (part != 1) & ~kept
    freed = gone.long().cumsum(0)
    flags = (begin[0] + taken > free.numel()) * 1 + (begin[0] + taken - freed[-1] < 0) * 16
    ok = flags == 0
    need, gone, lives = need & ok, gone & ok, lives & ok
    dst = torch.where(need, free[(begin + ends - 1).clamp(0, free.numel() - 1)], -1)
    new = torch.where((col == whole[p][:, None]) & need[:, None], dst[:, None], table[p])
    s["table_out"].copy_(torch.where(lives[:, None] & (col < held[p][:, None]), new, s["table_out"].long()))
    end = begin + (taken - freed[-1]) * ok
    place = torch.arange(free.numel(), device=DEV)
    rest = torch.where(place >= begin + taken * ok, free, s["free_out"].long())
    rest = torch.cat([rest, rest[:1]]).index_copy(0, torch.where(gone, end + freed - 1, free.numel()), torch.arange(total, device=DEV))[:-1]
    s["free_out"].copy_(rest)
    i32 = torch.int32
    return [s["table_out"], torch.where(lives, lens[p], 0).to(i32), s["free_out"], end.to(i32), torch.where(need, last[p], -1).to(i32), dst.to(i32),
            torch.where(need, lens[p] % page, 0).to(i32), torch.stack([flags, taken, freed[-1], lives.sum()]).to(i32)]


def _plain_copy(s):
    cache = s["cache"]
    there = s["src"] >= 0
    src, dst = (torch.where(there, s[n], 0).long() for n in ("src", "dst"))  # page 0 onto itself
    moved = (torch.arange(cache.shape[2], device=DEV) < s["slots"][:, None])[:, :, None, None]
    for layer in cache:
        layer[dst] = torch.where(moved, layer[src], layer[dst])
    return cache


def _plain_attn(s):
    """Group by group: all its rows' queries against the prefix once, each row's against its own positions, joined as softmax joins."""
    c = s["case"]
    W, hq, hk, d, page = (c[n] for n in ("W", "hq", "hk", "d", "page"))
    out, lse = [], []
    for i, (p, tails) in enumerate(s["groups"]):
        rows = slice(i * W, (i + 1) * W)
        q = s["q"][rows].float().view(W, hk, hq // hk, d).permute(1, 0, 2, 3)
        first, n = p // page, max(tails)
        table = s["table"][rows].long()

        def read(cache, scale, pages):                                       # [hk, (rows,) positions, d] in 32 bits
            x = cache[pages].flatten(-4, -3).movedim(-2, 0).float()
            return x if scale is None else x * scale.view(-1, *[1] * (x.dim() - 1))
        own_pages = table[:, first:first + -(-n // page)].clamp(min=0)
        j = torch.arange(own_pages.shape[1] * page, device=DEV)
        seen = j < (s["lens"][rows] - p)[:, None]
        k, v = read(s["k"], s["k_scale"], own_pages), read(s["v"], s["v_scale"], own_pages) * seen[:, :, None]
        z = torch.matmul(q, k.transpose(-1, -2).contiguous()) * s["scale"]
        z = torch.where(seen[:, None, :], z, -math.inf)
        top = z.amax(-1, keepdim=True)
        if p:
            pk, pv = read(s["k"], s["k_scale"], table[0, :first]), read(s["v"], s["v_scale"], table[0, :first])
            pz = torch.matmul(q.reshape(hk, -1, d), pk.transpose(-1, -2).contiguous()).view(hk, W, hq // hk, p) * s["scale"]
            top = torch.maximum(top, pz.amax(-1, keepdim=True))
        e = torch.exp(z - top)
        total, acc = e.sum(-1, keepdim=True), torch.matmul(e, v)
        if p:
            e = torch.exp(pz - top)
            total = total + e.sum(-1, keepdim=True)
            acc = acc + torch.matmul(e.view(hk, -1, p), pv).view(acc.shape)
        out.append((acc / total).permute(1, 0, 2, 3).reshape(W, hq, d))
        lse.append((top + total.log()).permute(1, 0, 2, 3).reshape(W, hq))
    return [torch.cat(out).to(DTYPE[c["y"]]), torch.cat(lse)]


# ---- what one pass cannot do without ------------------------------------------------------------

def work(case):
    if case["op"] == "beam":
        n, moved = case["R"] * case["W"] * case["V"], case["R"] * case["K"] * (16 + 8 * case["history"])
        return {"bytes": n * SIZE[case["x"]] + moved, "flops": 3 * n}
    if case["op"] == "fork":
        entries = sum(-(-n // case["page"]) for n in _spread(case["R"], case["longest"])) * case["W"]
        return {"bytes": 8 * entries + 28 * case["R"] * case["W"], "flops": 4 * entries}
    if case["op"] == "copy":
        slots = case["n"] * case["share"] * case["page"] / 2 * case["caches"]
        return {"bytes": int(2 * slots * case["hk"] * case["d"] * SIZE[case["x"]]) + 12 * case["n"], "flops": int(slots)}
    G, W, hq, hk, d = (case[n] for n in ("G", "W", "hq", "hk", "d"))
    groups = _lengths(case)
    held = sum(p + sum(tails) for p, tails in groups)
    seen = sum(p * W + sum(tails) for p, tails in groups)
    return {"bytes": 2 * held * hk * d * SIZE[case["cache"]] + 4 * held // case["page"] + G * W * hq * (d * (SIZE[case["q"]] + SIZE[case["y"]]) + 4),
            "flops": 4 * seen * hq * d}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "fork":
        return None                                                          # whole numbers
    s = prepare(case, seed)
    if case["op"] == "beam":
        return _exact_beam(case, s)
    if case["op"] == "copy":
        cache = s["cache"].double() if s["cache"].numel() < 1 << 30 else s["cache"].clone()
        at, n = s["src"].tolist(), s["slots"].tolist()
        for i, to in enumerate(s["dst"].tolist()):
            if to >= 0:
                cache[:, to, :n[i]] = cache[:, at[i], :n[i]].clone()
        return cache
    return _exact_attn(case, s)


def _exact_beam(case, s):
    R, W, K, V = (case[n] for n in ("R", "W", "K", "V"))
    totals = torch.full((R, K), -math.inf, dtype=torch.float64, device=DEV)
    for r in range(R):
        logits = s["x"][r * W:(r + 1) * W].double()
        t = torch.log_softmax(logits, -1) + s["scores"][r].double()[:, None]
        if s["done"] is not None:
            for w in torch.nonzero(s["done"][r]).flatten().tolist():
                t[w] = -math.inf
                t[w, s["end"]] = s["scores"][r, w].double()
        if s["weight"] is None:
            best = torch.topk(t.flatten(), min(K, W * V)).values
        else:
            ranked = torch.topk((t * s["weight"][r].double()[:, None]).flatten(), min(K, W * V)).indices
            best = t.flatten()[ranked]
        totals[r, :best.numel()] = best
    return [None, None, totals, None] + ([None, None] if s["history"] is not None else [])


def _exact_attn(case, s):
    W, hq, hk, d, page = (case[n] for n in ("W", "hq", "hk", "d", "page"))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["q"].shape[0], hq), dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        where = torch.arange(n, device=DEV)
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
