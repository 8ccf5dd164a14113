"""nm_shared_attention against attention in 64 bits row by row (the definition: what nm_paged_attention computes), over caches whose rows share
prefixes, and a run of the calls for several hypotheses together."""
import math

import pytest
import torch

from test_gpu_decode import DEV, TYPES, assert_rounded, attention_64, gen, i32
from paper_2305_14405_amd import binding as nm

pytestmark = pytest.mark.gpu


def shared_case(seed, groups, hq, hk, d, q_dtype, cache_dtype, page=16, by_head=False, columns=None, size=1.0):
    """groups: (shared, [lengths of the rows]); shared None: rows of no group.  Rows with fewer positions than shared have pages of their own.  A
    prefix that ends inside a page has that page's slots in a page of every row.  Free slots, and pages that no row owns, hold NaN (codes: -128)."""
    g = gen(seed)
    lens = [n for _, rows in groups for n in rows]
    if columns is None:                                                      # wide enough that the rows are not taken one by one
        columns = max([-(-max(n, 0) // page) for n in lens] + [-(-1100 // (len(lens) * hk)) * 128 // page + 1])
    most = sum(-(-max(n, 0) // page) for n in lens) + 9
    B = len(lens)
    shape = (2, most, hk, page, d) if by_head else (2, most, page, hk, d)
    cache = torch.randn(shape, generator=g)
    cache = (cache * 32).round().clamp(-127, 127).to(torch.int8) if cache_dtype == torch.int8 else (cache * size).to(cache_dtype)
    cache = cache.transpose(2, 3) if by_head else cache
    order, at, b = torch.randperm(most, generator=g).tolist(), 0, 0
    table, used = torch.full((B, columns), -1, dtype=torch.int32), torch.zeros((most, page), dtype=torch.bool)
    start, shared = [], []
    for p, rows in groups:
        prefix = None
        if p is not None:
            start.append(b)
            shared.append(p)
        for n in rows:
            whole = p // page if p is not None and n >= p > 0 else 0
            if whole and prefix is None:
                prefix = b
            for i in range(-(-max(n, 0) // page)):
                if i < whole and prefix != b:
                    table[b, i] = table[prefix, i]
                    continue
                table[b, i] = order[at]
                used[order[at], :max(0, min(page, n - i * page))] = True
                if p is not None and n >= p > 0 and i == p // page and p % page:
                    if prefix is None:
                        prefix = b
                    if prefix != b:
                        cache[:, order[at], :p % page] = cache[:, table[prefix, i], :p % page]
                at += 1
            b += 1
        if p is not None and groups.index((p, rows)) == len(groups) - 1:
            start.append(b)
    if len(start) == len(shared):
        start.append(start[-1] + len([r for p, r in groups if p is not None][-1]) if shared else 0)
    cache[:, ~used] = -128 if cache_dtype == torch.int8 else float("nan")
    scales = 0.02 * (1 + torch.rand((2, hk), generator=g)) if cache_dtype == torch.int8 else None
    cache = cache.to(DEV) if not by_head else cache.transpose(2, 3).contiguous().to(DEV).transpose(2, 3)
    return dict(q=(torch.randn((B, hq, d), generator=g) * size).to(q_dtype).to(DEV), cache=cache, table=table.to(DEV), lens=i32(lens), start=i32(start), shared=i32(shared),
                scales=None if scales is None else scales.to(DEV))


def attend(c, out_dtype, scale, lse=True, ws=None, stream=None, out=None, out_inv_scale=1.0):
    B, hq, d = c["q"].shape
    full = torch.full((B + 2, hq, d), 77, dtype=out_dtype, device=DEV)
    out = full[1:-1] if out is None else out
    wide = torch.full((B + 2, hq), 77.0, device=DEV) if lse else None
    lse = wide[1:-1] if lse else None
    s = (None, None) if c["scales"] is None else c["scales"]
    args = (c["q"], c["cache"][0], c["cache"][1], c["table"], c["lens"], c["start"], c["shared"], out)
    more = dict(scale=scale, k_scale=s[0], v_scale=s[1], lse=lse, out_inv_scale=out_inv_scale)
    size = nm.nm_shared_attention_workspace(*args, **more)
    if ws is None and size:
        ws = torch.full((size,), 0xff, dtype=torch.uint8, device=DEV)        # NaN, so that nothing unwritten is read
    nm.nm_shared_attention(*args, ws=ws, stream=stream, **more)
    torch.cuda.synchronize()
    assert bool((full[0] == 77).all()) and bool((full[-1] == 77).all())
    assert lse is None or (bool((wide[0] == 77).all()) and bool((wide[-1] == 77).all()))
    return out, lse


def check(c, out_dtype, scale=None):
    scale = c["q"].shape[2] ** -0.5 if scale is None else scale
    out, lse = attend(c, out_dtype, scale)
    want, wl, e_out, e_lse = attention_64(c, scale)
    nan = want.isnan().any(-1)                                               # rows that hold a NaN within their length have NaN alone
    assert bool(want[nan].isnan().all()) and bool(out[nan].isnan().all()) and bool(lse[nan].isnan().all())
    assert_rounded(out[~nan], want[~nan], e_out[~nan], "out")
    empty = wl == -math.inf
    assert bool((lse[empty] == -math.inf).all()) and bool((out[empty] == 0).all())
    assert bool(((lse.double() - wl)[~empty & ~nan].abs() <= e_lse[~empty & ~nan]).all())
    return out, lse


# a prefix shared by a few, by many, by one; ending inside a page; too short; rows shorter than it, empty ones, rows that end with it, rows of no group
MIXED = [(None, [5, 700]), (640, [641, 640, 900, 0, 100, 672]), (1000, [1001]), (333, [340] * 11), (20, [30, 25]), (0, [50, 3]), (256, [256] * 4), (-7, [44, 800]), (500, [0, 3, 499]),
         (130, [1300, 131]), (None, [0, 1, 129])]


@pytest.mark.parametrize("q_dtype,cache_dtype,out_dtype", [
    (torch.bfloat16, torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16, torch.float16), (torch.float32, torch.int8, torch.float32),
    (torch.float32, torch.bfloat16, torch.float32), (torch.bfloat16, torch.int8, torch.bfloat16), (torch.float16, torch.bfloat16, torch.float16),
    (torch.bfloat16, torch.float16, torch.float32), (torch.float32, torch.float16, torch.bfloat16), (torch.float16, torch.int8, torch.float16)])
@pytest.mark.parametrize("hq,hk,d", [(4, 4, 64), (8, 2, 128), (5, 1, 32), (24, 1, 96), (6, 3, 16), (16, 1, 256), (34, 2, 80), (70, 1, 64)])
def test_shared_attention(q_dtype, cache_dtype, out_dtype, hq, hk, d):
    c = shared_case(hq + d, MIXED[1:-1], hq, hk, d, q_dtype, cache_dtype, by_head=bool(d & 32))
    check(c, out_dtype)


@pytest.mark.parametrize("hq,hk,d", [(16, 16, 64), (8, 8, 32), (16, 8, 16), (12, 12, 48), (16, 16, 16), (6, 6, 64)])
@pytest.mark.parametrize("by_head", [False, True])
@pytest.mark.parametrize("q_dtype", TYPES)
def test_shared_attention_neighbouring_heads_of_codes(q_dtype, by_head, hq, hk, d):
    """int8 heads that lie next to each other are taken as one of up to 128 elements, where groups are small; some groups here are larger."""
    c = shared_case(hq * d, [(300, [310, 301]), (512, [700, 513, 600]), (0, [40]), (900, [901]), (256, [300] * 20), (140, [141, 0]), (0, [9]), (130, [131, 2000]), (64, [65, 70])], hq, hk, d, q_dtype,
                    torch.int8, page=32, by_head=by_head)
    c["q"][1, :, 0] *= 100.0
    check(c, q_dtype)


def test_shared_attention_rows_in_front_of_and_behind_the_groups():
    c = shared_case(3, MIXED, 8, 2, 64, torch.bfloat16, torch.bfloat16)
    assert int(c["start"][0]) == 2 and int(c["start"][-1]) == c["lens"].numel() - 3
    check(c, torch.bfloat16)


@pytest.mark.parametrize("page", [1, 2, 8, 64, 256, 4096])
@pytest.mark.parametrize("cache_dtype", [torch.bfloat16, torch.int8])
def test_shared_attention_page_sizes(page, cache_dtype):
    check(shared_case(page, [(300, [310, 0, 613, 300]), (129, [130] * 3), (512, [513, 2000])], 8, 2, 64, torch.bfloat16, cache_dtype, page=page), torch.bfloat16)


@pytest.mark.parametrize("groups,hq,hk,d", [([(20000, [20001 + 3 * i for i in range(9)])], 8, 2, 128), ([(5000, [5010] * 40), (7000, [7001] * 3)], 4, 1, 64), ([(1024, [1100] * 130)], 2, 2, 64),
                                            ([(600, [700] * 2)] * 60, 4, 4, 32), ([(3000, [3000 + 1000 * i for i in range(5)])], 48, 2, 96), ([(900, [1000] * 7)], 12, 12, 256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_shared_attention_long_many_and_wide(groups, hq, hk, d, dtype):
    c = shared_case(len(groups), [(p, list(r)) for p, r in groups], hq, hk, d, dtype, torch.bfloat16, page=32)
    B = c["lens"].numel()
    if len(groups) == 60:                                                    # equal groups: their starts by hand
        c["start"], c["shared"] = i32(list(range(0, B + 1, 2))), i32([600] * 60)
    check(c, dtype)


def test_shared_attention_short_tables_need_no_workspace():
    c = shared_case(2, [(200, [201, 300, 7]), (100, [150] * 3)], 6, 3, 64, torch.float16, torch.float16, columns=19)
    args = (c["q"], c["cache"][0], c["cache"][1], c["table"], c["lens"], c["start"], c["shared"], torch.empty_like(c["q"]))
    assert nm.nm_shared_attention_workspace(*args, scale=1.0) == 0
    check(c, torch.float16)


def test_shared_attention_of_few_units():
    """Rows that are divided, but too few for sharing: taken one by one."""
    check(shared_case(13, [(700, [701, 750, 800, 0])], 12, 12, 64, torch.float32, torch.bfloat16, columns=51), torch.float32)


def test_shared_attention_without_groups():
    c = shared_case(4, [(None, [5, 0, 1400, 333])], 8, 2, 128, torch.bfloat16, torch.bfloat16)
    c["start"], c["shared"] = i32([0]), i32([])
    check(c, torch.bfloat16)


@pytest.mark.parametrize("start", [[0, 9, 5, 12], [-1, 4, 8, 12], [0, 4, 8, 13], [5, 5, 4, 4], [2 ** 31 - 1, 0, 3, 4]])
def test_shared_attention_groups_that_are_none(start):
    """Starts that do not ascend within the rows: every row by itself, by its own table."""
    c = shared_case(5, [(600, [700] * 12)], 4, 1, 64, torch.bfloat16, torch.bfloat16)
    c["start"], c["shared"] = i32(start), i32([600, 600, 2 ** 31 - 1])
    check(c, torch.bfloat16)


def test_shared_attention_bad_tables_lengths_and_prefixes():
    """Entries that are no pages take no part, lengths beyond the table count as the table's; a prefix longer than its rows is no one's."""
    c = shared_case(6, [(400, [500, 600, 450]), (300, [301] * 4)], 4, 2, 64, torch.bfloat16, torch.bfloat16, columns=1200)
    for b in (0, 1, 2):
        c["table"][b, 3], c["table"][b, 7] = -5, 10 ** 6
    c["table"][1, 30] = 2 ** 31 - 1
    c["lens"][2] = 10 ** 9                                                   # columns behind are -1: no pages
    c["shared"][1] = 2 ** 31 - 1
    check(c, torch.bfloat16)
    c["table"][3:] = -1                                                      # nothing left
    out, lse = check(c, torch.bfloat16)
    assert bool((out[3:] == 0).all()) and bool((lse[3:] == -math.inf).all())


def test_shared_attention_infinities_stay_in_their_rows():
    """Values that are infinite behind the prefix reach only the rows that hold them; in the prefix, all of its group."""
    c = shared_case(7, [(512, [600] * 5), (512, [520] * 3)], 4, 2, 64, torch.bfloat16, torch.bfloat16)
    own, prefix = int(c["table"][2, 35]), int(c["table"][5, 10])
    c["cache"][1, own, 3, 1, 7] = math.inf
    c["cache"][1, prefix, 3, 0, 9] = -math.inf
    out, lse = attend(c, torch.bfloat16, 0.125)
    hit = torch.zeros((8, 4, 64), dtype=torch.bool, device=DEV)
    hit[2, 2:, 7], hit[5:, :2, 9] = True, True
    assert not bool(out[hit].isfinite().any()) and bool(out[~hit].isfinite().all()) and bool(lse.isfinite().all())


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_shared_attention_scales_and_large_scores(scale):
    check(shared_case(8, [(700, [701, 750, 800])], 8, 2, 64, torch.float32, torch.bfloat16, size=4.0), torch.float32, scale=scale)


def test_shared_attention_codes_in_place_and_strides():
    c = shared_case(9, [(600, [610, 900, 601]), (256, [300] * 2)], 8, 2, 64, torch.bfloat16, torch.bfloat16)
    want, lse = attend(c, torch.bfloat16, 0.125)
    codes, _ = attend(c, torch.int8, 0.125, out_inv_scale=90.0)
    f32, _ = attend(c, torch.float32, 0.125)
    assert bool(((codes.float() - (f32 * 90).round().clamp(-127, 127)).abs() <= 1).all()) and bool(codes.any())
    wide = torch.zeros((5, 8 * 64 + 40), dtype=torch.bfloat16, device=DEV)
    wide[:, :512] = c["q"].view(5, -1)
    q = wide[:, :512].unflatten(1, (8, 64))
    c["q"] = q
    got, _ = attend(c, torch.bfloat16, 0.125, out=q)                         # in place, rows apart
    assert torch.equal(got, want) and not bool(wide[:, 512:].any())
    c["q"] = want.clone()
    a, _ = attend(c, torch.bfloat16, 0.125, lse=False)
    b, _ = attend(c, torch.bfloat16, 0.125)
    assert torch.equal(a, b)


def test_shared_attention_is_what_paged_attention_gives():
    """Within both calls' rounding, at more rows than a group's columns hold."""
    c = shared_case(10, [(2048, [2100 + i for i in range(37)])], 16, 4, 128, torch.float32, torch.bfloat16)
    out, lse = attend(c, torch.float32, 0.09)
    o2, l2 = torch.empty_like(out), torch.empty((37, 16), device=DEV)
    args = (c["q"], c["cache"][0], c["cache"][1], c["table"], c["lens"], o2)
    ws = torch.empty(nm.nm_paged_attention_workspace(*args, scale=0.09, lse=l2), dtype=torch.uint8, device=DEV)
    nm.nm_paged_attention(*args, scale=0.09, lse=l2, ws=ws)
    torch.cuda.synchronize()
    _, _, e_out, e_lse = attention_64(c, 0.09)
    assert bool(((out - o2).abs() <= 2 * e_out + 2.0 ** -22 * out.abs()).all()) and bool(((lse - l2).abs() <= 2 * e_lse + 2.0 ** -22 * lse.abs()).all())


@pytest.mark.parametrize("groups,hq,hk,d,dtype", [([(700, [720 + i for i in range(12)]), (None, [900])], 8, 4, 64, torch.int8),
                                                  ([(1500, [1510 + i % 7 for i in range(160)]), (400, [450] * 40)], 4, 2, 128, torch.bfloat16)])
def test_shared_attention_beyond_2_32_elements(groups, hq, hk, d, dtype):
    """The bits of a cache whose pages are neighbours, with pages so far apart that offsets need more than 32 bits."""
    c = shared_case(13, groups, hq, hk, d, torch.bfloat16, dtype)
    want, wl = check(c, torch.bfloat16)
    _, pages, page, _, _ = c["cache"].shape
    apart = (3 << 31) // pages // 128 * 128
    assert (pages - 1) * apart > 1 << 32
    far = torch.empty(2 * pages * apart, dtype=dtype, device=DEV).as_strided((2, pages, page, hk, d), (pages * apart, apart, hk * d, d, 1))
    for i in range(2):
        for j in range(pages):
            far[i, j].copy_(c["cache"][i, j])
    out, lse = attend({**c, "cache": far}, torch.bfloat16, d ** -0.5)
    assert torch.equal(out, want) and torch.equal(lse, wl)


def test_shared_attention_twice_at_once_and_replayed():
    """Two calls on two streams with workspaces of their own; a captured call, replayed while lengths, groups and tables change, its workspace filled anew."""
    a = shared_case(11, [(600, [650] * 6), (300, [400] * 5)], 8, 2, 64, torch.bfloat16, torch.bfloat16, columns=900)
    b = shared_case(12, [(900, [950] * 3)], 8, 2, 64, torch.bfloat16, torch.bfloat16)
    wants = [attend(c, torch.bfloat16, 0.125) for c in (a, b)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    outs = []
    for c, stream in ((a, s), (b, None)):
        out, lse = torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device=DEV)
        args = (c["q"], c["cache"][0], c["cache"][1], c["table"], c["lens"], c["start"], c["shared"], out)
        ws = torch.empty(nm.nm_shared_attention_workspace(*args, scale=0.125, lse=lse), dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        outs.append((args, ws, out, lse, stream))
    for args, ws, out, lse, stream in outs:
        nm.nm_shared_attention(*args, scale=0.125, lse=lse, ws=ws, stream=stream)
    torch.cuda.synchronize()
    for (_, _, out, lse, _), (wo, wl) in zip(outs, wants):
        assert torch.equal(out, wo) and torch.equal(lse, wl)
    args, ws, out, lse, _ = outs[0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nm.nm_shared_attention(*args, scale=0.125, lse=lse, ws=ws)
    for lens, start, shared in (([650] * 6 + [400] * 5, [0, 6, 11], [600, 300]), ([620] * 6 + [0, 3, 400, 399, 398], [0, 3, 11], [600, 0]), ([600] * 6 + [300] * 5, [0, 6, 11], [592, 300])):
        a["lens"].copy_(torch.tensor(lens)), a["start"].copy_(torch.tensor(start)), a["shared"].copy_(torch.tensor(shared))
        ws.fill_(0xff), out.fill_(5), lse.fill_(5)
        g.replay()
        torch.cuda.synchronize()
        wo, wl = attend(a, torch.bfloat16, 0.125)
        assert torch.equal(out, wo) and torch.equal(lse, wl)
        want, wl, e_out, _ = attention_64(a, 0.125)
        assert_rounded(out, want, e_out, "replay")


@pytest.mark.parametrize("groups,hq,hk,d,dtype", [([(5000, [5010 + 9 * i for i in range(64)])], 32, 8, 128, torch.bfloat16), ([(3000, [3000 + i for i in range(96)])], 16, 4, 64, torch.float32),
                                                  ([(2000, [2001 + i for i in range(8)]), (900, [950 + 30 * i for i in range(8)])], 16, 16, 64, torch.int8)])
def test_shared_attention_gives_the_same_bits_every_time(groups, hq, hk, d, dtype):
    """Prefixes of few and of many queries: in new workspaces, in old ones, and behind calls that leave other numbers there."""
    q = torch.float16 if dtype == torch.int8 else dtype
    c = shared_case(41, groups, hq, hk, d, q, torch.int8 if dtype == torch.int8 else torch.bfloat16, page=32)
    other = {**c, "q": c["q"] * 1.7, "lens": torch.clamp(c["lens"] - 40, min=0)}
    want, lse = check(c, q)
    args = (c["q"], c["cache"][0], c["cache"][1], c["table"], c["lens"], c["start"], c["shared"], torch.empty_like(c["q"]))
    s = (None, None) if c["scales"] is None else c["scales"]
    ws = torch.full((nm.nm_shared_attention_workspace(*args, scale=1.0, k_scale=s[0], v_scale=s[1]),), 0xff, dtype=torch.uint8, device=DEV)
    for i in range(12):
        if i % 3 == 2:
            attend(other, q, d ** -0.5, ws=ws)
        got, l = attend(c, q, d ** -0.5, ws=ws if i % 2 else None)
        assert torch.equal(got, want) and torch.equal(l, lse), i


def test_shared_attention_as_many_rows_as_it_takes():
    """4096 rows in 1024 groups of four."""
    B, hk, d, page = 4096, 1, 16, 32
    g = gen(1)
    cache = torch.randn((2, 1024 * 20 + 4096, page, hk, d), generator=g).to(torch.bfloat16).to(DEV)
    table = torch.full((B, 21), -1, dtype=torch.int32)
    table[:, :20] = torch.arange(1024 * 20, dtype=torch.int32).view(1024, 20).repeat_interleave(4, 0)
    table[:, 20] = 1024 * 20 + torch.arange(B, dtype=torch.int32)
    lens = 640 + torch.randint(0, 33, (B,), generator=g)
    c = dict(q=torch.randn((B, 2, d), generator=g).to(torch.bfloat16).to(DEV), cache=cache, table=table.to(DEV), lens=i32(lens.tolist()), start=i32(list(range(0, B + 1, 4))),
             shared=i32([640] * 1024), scales=None)
    out, lse = attend(c, torch.bfloat16, 0.25)
    some = list(range(0, B, 61)) + [B - 1]
    part = {**c, "q": c["q"][some], "table": c["table"][some], "lens": c["lens"][some]}
    want, wl, e_out, e_lse = attention_64(part, 0.25)
    assert_rounded(out[some], want, e_out, "out")
    assert bool(((lse[some].double() - wl).abs() <= e_lse).all())


def test_beam_search_over_a_paged_cache():
    """The calls as they are used: a prompt, then steps of plan, keys and values into the cache, attention, logits, selection, fork and copy.  Each
    step's attention is compared with the hypotheses' whole histories, held outside of any page, in 64 bits, and its selection with the rules."""
    from test_gpu_hypotheses import NEAR, scratch
    R, W, hq, hk, d, V, page, steps = 3, 4, 4, 2, 64, 500, 16, 40
    B, prompts, g = R * W, [1000, 37, 513], gen(77)
    columns, pages, dt = 70, 400, torch.bfloat16
    embed = (torch.randn((V, (hq + 2 * hk) * d), generator=g)).to(dt).to(DEV)   # a token's queries, keys and values
    head = (torch.randn((V, hq * d), generator=g) * 0.2).to(DEV)
    cache = torch.full((2, pages, page, hk, d), float("nan"), dtype=dt, device=DEV)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    table, other = torch.full((B, columns), -1, dtype=torch.int32, device=DEV), torch.full((B, columns), -1, dtype=torch.int32, device=DEV)
    free, free2, begin, end = torch.arange(pages, dtype=torch.int32, device=DEV).flip(0).contiguous(), z(pages), z(1), z(1)
    inv_freq = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().to(DEV)
    # prompts: a row each, forked into W hypotheses below
    tokens = [torch.randint(0, V, (n,), generator=g) for n in prompts]
    fresh, T = i32(prompts), sum(prompts)
    slots, positions, status, lens = z(T), z(T), z(4), z(R)
    nm.nm_page_plan(z(R), fresh, free, begin, table[:R], page_size=page, num_pages=pages, free_end=end, slots=slots, positions=positions, status=status, lens=lens)
    x = embed[torch.cat(tokens).to(DEV)].view(T, hq + 2 * hk, d)
    q_out = torch.empty((T, hq, d), dtype=dt, device=DEV)
    nm.nm_qk_norm_rope(x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:], positions, inv_freq, q_out, k_cache=cache[0], v_cache=cache[1], slots=slots, norm=True)
    history = [t.tolist() for t in tokens]                                    # of every row, outside
    parents = torch.arange(R, dtype=torch.int32, device=DEV).repeat_interleave(W)
    lens_in, free_begin = lens, end
    copies, lens_out, end2 = [z(B) for _ in range(3)], z(B), z(1)

    def fork(rows_in, lens_in, parents, table, other, free, free2, at, to):
        args = (table[:rows_in], lens_in, parents, free, at, other)
        more = dict(page_size=page, num_pages=pages, lens_out=lens_out, free_out=free2, free_end=to, copy_src=copies[0], copy_dst=copies[1], copy_slots=copies[2], status=status)
        nm.nm_page_fork(*args, ws=scratch(nm.nm_page_fork_workspace(*args, **more)), **more)
        nm.nm_page_copy(cache, *copies)
        torch.cuda.synchronize()
        assert status.tolist()[0] == 0
    fork(R, lens_in, parents, table, other, free, free2, free_begin, end2)
    table, other, free, free2 = other, table, free2, free
    history = [list(history[p]) for p in parents.tolist()]
    start, shared = i32([0, 4, 8, 12]), i32([n // page * page for n in prompts])
    scores = torch.zeros((R, W), device=DEV)
    scores[:, 1:] = -math.inf                                                 # one hypothesis to begin with
    token, done = z(R, W), z(R, W)
    token.copy_(torch.tensor([[h[-1]] * W for h in history[::W]]))
    at, to, lens = end2.clone(), z(1), lens_out.clone()
    for step in range(steps):
        slots, positions, row = z(B), z(B), z(B)
        nm.nm_page_plan(lens, torch.ones_like(lens), free, at, table, page_size=page, num_pages=pages, free_end=to, slots=slots, positions=positions, status=status, lens=row)
        x = embed[token.view(-1).clamp(min=0).long()].view(B, hq + 2 * hk, d)
        q = torch.empty((B, hq, d), dtype=dt, device=DEV)
        nm.nm_qk_norm_rope(x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:], positions, inv_freq, q, k_cache=cache[0], v_cache=cache[1], slots=slots, norm=True)
        out = torch.empty((B, hq, d), dtype=torch.float32, device=DEV)
        args = (q, cache[0], cache[1], table, row, start, shared, out)
        nm.nm_shared_attention(*args, scale=0.125, ws=scratch(nm.nm_shared_attention_workspace(*args, scale=0.125)))
        history = [h + [t] for h, t in zip(history, token.view(-1).tolist())]
        torch.cuda.synchronize()
        assert status.tolist()[0] == 0 and row.tolist() == [len(h) for h in history]
        if step % 6 == 0 or step == steps - 1:                                # keys and values of the whole history, through no page
            flat = torch.tensor([t for h in history for t in h])
            place = torch.cat([torch.arange(len(h)) for h in history])
            y = embed[flat.to(DEV)].view(-1, hq + 2 * hk, d)
            k = torch.empty((flat.numel(), hk, d), dtype=dt, device=DEV)
            nm.nm_qk_norm_rope(y[:, :hq], y[:, hq:hq + hk], y[:, hq + hk:], i32(place), inv_freq, torch.empty((flat.numel(), hq, d), dtype=dt, device=DEV), k_out=k, norm=True)
            n = max(len(h) for h in history)
            whole = torch.full((2, B, n, hk, d), float("nan"), dtype=dt, device=DEV)
            i = 0
            for b, h in enumerate(history):
                whole[0, b, :len(h)], whole[1, b, :len(h)] = k[i:i + len(h)], y[i:i + len(h), hq + hk:]
                i += len(h)
            want, _, e_out, _ = attention_64(dict(q=q, cache=whole, table=torch.arange(B, dtype=torch.int32, device=DEV)[:, None], lens=row, scales=None), 0.125)
            assert_rounded(out, want, e_out, f"step {step}")
        logits = out.view(B, -1) @ head.t().contiguous()
        parents, token, totals, over = z(R, W), z(R, W), torch.zeros((R, W), device=DEV), z(R, W)
        args = (logits, scores, parents, token, totals)
        nm.nm_beam_select(*args, ws=scratch(nm.nm_beam_select_workspace(*args)), done_out=over)
        torch.cuda.synchronize()
        t = torch.log_softmax(logits.double(), -1).view(R, W, V) + scores.double()[:, :, None]
        best = torch.topk(t.view(R, -1), W).values
        assert bool(((totals - best).abs() <= NEAR + 2.0 ** -23 * best.abs()).all())
        fork(B, row, parents.view(-1), table, other, free, free2, to, end2)
        table, other, free, free2 = other, table, free2, free
        history = [list(history[p]) for p in parents.view(-1).tolist()]
        scores, at, lens = totals, end2.clone(), lens_out.clone()
        held = {int(e) for b in range(B) for e in table[b, :-(-int(lens[b]) // page)].tolist()}
        left = free[int(at):].tolist()
        assert len(held) + len(left) == pages and held.isdisjoint(left) and len(set(left)) == len(left)   # no page is lost, or twice
