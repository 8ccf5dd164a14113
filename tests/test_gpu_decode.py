"""The calls of a decode step (plan, norms and rotation, attention over the cache, 4-bit products) against plain
implementations in 64 bits, and a run of them together."""
import math

import numpy as np
import pytest
import torch

from paper_2305_14405_amd import binding as nm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24                                                               # half a step of binary32, relative
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return g


def i32(*a, **k):
    return torch.tensor(*a, dtype=torch.int32, **k).to(DEV)


# ---- plan ---------------------------------------------------------------------------------------

def plan_in_python(cached, fresh, free, begin, table, page, num_pages, T):
    """The documented rules, one request after the other."""
    B, columns = table.shape
    up = lambda n: -(-n // page)  # noqa: E731
    need = [up(c + f) - up(c) if f > 0 else 0 for c, f in zip(cached, fresh)]
    flags = (1 if begin + sum(need) > len(free) else 0) | (2 if any(up(c + f) > columns for c, f in zip(cached, fresh)) else 0) | \
            (4 if sum(fresh) > T else 0) | (8 if min([0, begin, *cached, *fresh]) < 0 else 0)
    out = {"status": [flags, sum(fresh), sum(need), max([0] + [c + f for c, f in zip(cached, fresh)])], "table": table.copy(), "lens": list(cached),
           "row_start": [0] * (B + 1), "end": begin, "slots": [-1] * T, "positions": [0] * T, "requests": [-1] * T}
    if flags:
        return out
    t = 0
    for b in range(B):
        for j in range(need[b]):
            out["table"][b, up(cached[b]) + j] = free[out["end"]]
            out["end"] += 1
        for i in range(fresh[b]):
            p = cached[b] + i
            entry = out["table"][b, p // page]
            out["slots"][t] = entry * page + p % page if 0 <= entry < num_pages else -1
            out["positions"][t], out["requests"][t] = p, b
            t += 1
        out["lens"][b] = cached[b] + fresh[b]
        out["row_start"][b + 1] = t
    return out


def run_plan(cached, fresh, free, begin, table, page, num_pages, T, some=False, stride=None):
    B, columns = table.shape
    wide = torch.full((B, stride or columns), -77, dtype=torch.int32)
    wide[:, :columns] = torch.from_numpy(table)
    wide = wide.to(DEV)
    o = {"end": i32([-5]), "lens": i32([-5] * B), "row_start": i32([-5] * (B + 1)), "slots": i32([-5] * T), "positions": i32([-5] * T),
         "requests": i32([-5] * T), "status": i32([-5] * 4)}
    optional = {} if some else {n: o[n] for n in ("lens", "row_start", "positions", "requests")}
    nm.nm_page_plan(i32(cached), i32(fresh), i32(free), i32([begin]), wide[:, :columns], page_size=page, num_pages=num_pages, free_end=o["end"],
                    slots=o["slots"], status=o["status"], **optional)
    torch.cuda.synchronize()
    got = {n: v.cpu().tolist() for n, v in o.items()}
    wide = wide.cpu().numpy()
    assert (wide[:, columns:] == -77).all()
    got["table"] = wide[:, :columns]
    return got


def check_plan(got, want, names=("status", "lens", "row_start", "slots", "positions", "requests")):
    for n in names:
        assert got[n] == want[n], n
    assert got["end"] == [want["end"]]
    assert np.array_equal(got["table"], want["table"])


def random_plan(seed, B, page, longest, most_new, idle=0.3):
    r = np.random.default_rng(seed)
    cached = r.integers(0, longest + 1, B).tolist()
    fresh = [0 if r.random() < idle else int(r.integers(1, most_new + 1)) for _ in range(B)]
    columns = -(-(longest + most_new) // page)
    pages = r.permutation(B * columns + 50)
    table = np.full((B, columns), -1, np.int32)
    at = 0
    for b in range(B):
        n = -(-cached[b] // page)
        table[b, :n] = pages[at:at + n]
        at += n
    return cached, fresh, pages[at:].tolist(), table, len(pages)


@pytest.mark.parametrize("B,page,longest,most_new,extra", [
    (1, 16, 0, 1, 0), (1, 1, 5, 3, 2), (8, 16, 300, 1, 0), (255, 16, 100, 1, 7), (256, 8, 64, 40, 0), (257, 32, 200, 33, 1),
    (1000, 16, 50, 2, 100), (4096, 64, 300, 1, 0), (3, 128, 1000, 5000, 777), (40, 65536, 3, 100, 0), (2, 16, 10, 300000, 5)])
def test_page_plan_matches_python(B, page, longest, most_new, extra):
    cached, fresh, free, table, pages = random_plan(B + page, B, page, longest, most_new)
    args = (cached, fresh, free, 0 if len(free) < 60 else 9, table, page, pages, sum(fresh) + extra)
    check_plan(run_plan(*args, stride=table.shape[1] + 3), plan_in_python(*args))


def test_page_plan_optional_outputs_and_empty_batches():
    cached, fresh, free, table, pages = random_plan(3, 20, 16, 100, 9)
    args = (cached, fresh, free, 2, table, 16, pages, sum(fresh))
    check_plan(run_plan(*args, some=True), plan_in_python(*args), ("status", "slots"))
    check_plan(run_plan([], [], [5], 1, np.zeros((0, 4), np.int32), 16, 10, 6), plan_in_python([], [], [5], 1, np.zeros((0, 4), np.int32), 16, 10, 6))
    idle = ([3, 0], [0, 0], [], 0, np.array([[2, -1], [-1, -1]], np.int32), 16, 10, 0)
    check_plan(run_plan(*idle), plan_in_python(*idle))


@pytest.mark.parametrize("what", ["pages", "table", "rows", "cached", "fresh", "begin", "several"])
def test_page_plan_assigns_nothing_that_does_not_fit(what):
    cached, fresh, free, table, pages = random_plan(11, 300, 16, 100, 30, idle=0.1)
    need = plan_in_python(cached, fresh, free, 0, table, 16, pages, sum(fresh))["status"][2]
    begin, T = 4, sum(fresh) + 5
    free = free[:need + begin]
    if what in ("pages", "several"):
        free = free[:-1]
    if what in ("rows", "several"):
        T = sum(fresh) - 1
    if what == "table":
        fresh[150] += 100
        free, T = free + list(range(10)), T + 100
    if what == "cached":
        cached[299] = -1
    if what == "fresh":
        fresh[0] = -3
    if what == "begin":
        begin = -1
    args = (cached, fresh, free, begin, table, 16, pages, T)
    want, got = plan_in_python(*args), run_plan(*args)
    assert want["status"][0] != 0
    if what in ("cached", "fresh", "begin"):        # the numbers beside the flag are of no use then
        assert got["status"][0] & nm.NM_PLAN_BAD_LENGTH
        check_plan(got, want, ("lens", "row_start", "slots", "positions", "requests"))
    else:
        check_plan(got, want)


def test_page_plan_sums_beyond_31_bits():
    B, big = 3000, 2 ** 31 - 1
    table = np.full((B, 2), -1, np.int32)
    got = run_plan([0] * B, [big] * B, [1, 2], 0, table, 16, 100, 4)
    assert got["status"] == [nm.NM_PLAN_NO_PAGES | nm.NM_PLAN_TABLE_FULL | nm.NM_PLAN_NO_ROWS, big, big, big]
    assert got["slots"] == [-1] * 4 and got["lens"] == [0] * B and (got["table"] == -1).all()


def test_page_plan_entries_that_are_no_pages():
    table = np.array([[7, -1, -1], [-3, -1, -1], [99, -1, -1]], np.int32)
    args = ([3, 5, 6], [20, 2, 1], [50, 51], 0, table, 16, 51, 23)   # list entry 50 is the last page, 51 is none; rows 1 and 2 hold none
    got = run_plan(*args)
    check_plan(got, plan_in_python(*args))
    assert got["slots"][20:] == [-1, -1, -1] and got["slots"][13] == 50 * 16


# ---- norms and rotation ---------------------------------------------------------------------------

def rotate_64(x, positions, inv_freq, gamma, norm, interleaved, eps=1e-6):
    """(result, bound of a 32-bit evaluation's error) in binary64.  Rounding errors, in units of U relative to the operands: the mean of
    at most 256 squares 16 (a chain of 8 and a butterfly of 6, and the squares), halved by the root; the root, the quotient and two
    products 5; together 13 on y.  A turn adds two products and a sum, 3, and the sine and cosine: their angle is rounded
    to 32 bits once (pi U) and the functions are taken to be within 4 U: 8 U of either partner.  25 are granted, on the sum of the partners'
    absolute values."""
    y = x.double()
    if norm:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * (1 if gamma is None else gamma.double())
    out, size = y.clone(), y.abs().clone()
    rot = 2 * inv_freq.numel()
    if rot:
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        phase = positions.double()[:, None, None] * inv_freq.double()
        c, s = torch.cos(phase), torch.sin(phase)
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return out, 25 * U * size


def assert_rounded(got, want, error, what):
    """got is want, wrong by no more than error, rounded to its type (at most half a step of the result, or of the smallest normal number)."""
    bound = error + HALF_STEP[got.dtype] * ((want.abs() + error) + torch.finfo(got.dtype).tiny)
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"{what}: {float((off / bound).max()):.3g} of the bound"


def qk_case(seed, T, hq, hk, d, rot, dtype, cache_dtype, page=16, by_head=False, far=5000, pad=0):
    g = gen(seed)
    row = (hq + 2 * hk) * d + pad
    x = torch.randn((T, row), generator=g).to(dtype).to(DEV)
    q, k, v = (x[:, a * d:b * d].view(T, -1, d) for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    pages = -(-(T + 20) // page)
    shape = (2, pages, hk, page, d) if by_head else (2, pages, page, hk, d)
    cache = (torch.randn(shape, generator=g) * 30).to(cache_dtype).to(DEV)
    cache = cache.transpose(2, 3) if by_head else cache
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    if T > 2:
        slots[1], slots[T - 1] = -1, pages * page   # neither is a slot
    return dict(x=x, q=q, k=k, v=v, cache=cache, slots=slots.to(DEV), positions=torch.randint(0, far, (T,), generator=g, dtype=torch.int32).to(DEV),
                inv_freq=(10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().to(DEV),
                q_gamma=(1 + 0.2 * torch.randn(d, generator=g)).to(DEV), k_gamma=(1 + 0.2 * torch.randn(d, generator=g)).to(DEV),
                inv_scale=(20 + 10 * torch.rand((2, hk), generator=g)).to(DEV))


def check_qk(c, dtype_out, norm=True, interleaved=False, gammas=True, k_out=True, cached=True):
    T, hq, d = c["q"].shape
    hk = c["k"].shape[1]
    q_out = torch.full((T, hq, d), float("nan"), dtype=dtype_out, device=DEV)
    key = torch.full((T, hk, d), float("nan"), dtype=dtype_out, device=DEV) if k_out else None
    before, x = c["cache"].clone(), c["x"].clone()
    codes = before.dtype == torch.int8
    g = (c["q_gamma"], c["k_gamma"]) if gammas else (None, None)
    inv_freq = c["inv_freq"] if c["inv_freq"].numel() else None
    more = dict(k_cache=c["cache"][0], v_cache=c["cache"][1], slots=c["slots"]) if cached else {}
    if codes and cached:
        more.update(k_inv_scale=c["inv_scale"][0], v_inv_scale=c["inv_scale"][1])
    nm.nm_qk_norm_rope(c["q"], c["k"], c["v"], c["positions"], inv_freq, q_out, k_out=key, norm=norm, q_gamma=g[0], k_gamma=g[1],
                       interleaved=interleaved, **more)
    torch.cuda.synchronize()
    assert torch.equal(c["x"], x)
    wq, eq = rotate_64(c["q"], c["positions"], c["inv_freq"], g[0], norm, interleaved)
    wk, ek = rotate_64(c["k"], c["positions"], c["inv_freq"], g[1], norm, interleaved)
    assert_rounded(q_out, wq, eq, "q")
    if k_out:
        assert_rounded(key, wk, ek, "k")
    _, pages, page, _, _ = before.shape
    there = (c["slots"] >= 0) & (c["slots"] < pages * page) & cached
    at = c["slots"][there].long()
    written = torch.zeros((pages, page), dtype=torch.bool, device=DEV)
    written[at // page, at % page] = True
    assert torch.equal(c["cache"][:, ~written], before[:, ~written])             # nothing but the tokens' slots is touched
    for n, (want, error) in enumerate(((wk, ek), (c["v"].double(), torch.zeros_like(wk)))):
        got, want, error = c["cache"][n][at // page, at % page], want[there], error[there]
        if codes:
            inv = c["inv_scale"][n].double()[:, None]
            real = (want * inv).clamp(-127, 127)
            off = (got.double() - real).abs() - 0.5 - error * inv - 2 * U * real.abs()   # the product's rounding, and that to a code
            assert bool((off <= 0).all()), float(off.max())
        else:
            assert_rounded(got, want, error, "cache")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,hq,hk,d,rot", [(1, 1, 1, 64, 64), (1, 32, 8, 128, 128), (3, 12, 12, 64, 32), (70, 5, 1, 96, 48), (33, 4, 2, 80, 40),
                                           (9, 24, 3, 32, 32), (17, 2, 2, 256, 256), (5, 3, 3, 192, 64), (1030, 2, 1, 16, 16), (2, 7, 2, 8, 0)])
def test_qk_norm_rope(dtype, interleaved, T, hq, hk, d, rot):
    check_qk(qk_case(T + d, T, hq, hk, d, rot, dtype, dtype), dtype, interleaved=interleaved)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,hq,hk,d,rot,pad", [(4, 3, 2, 7, 4, 0), (5, 2, 1, 1, 0, 0), (6, 2, 2, 100, 50, 1), (3, 2, 1, 250, 250, 0), (1100, 1, 1, 66, 2, 3),
                                               (4, 2, 2, 64, 64, 1), (4, 2, 2, 64, 12, 0)])
def test_qk_norm_rope_odd_sizes_and_alignment(dtype, interleaved, T, hq, hk, d, rot, pad):
    check_qk(qk_case(T + d, T, hq, hk, d, rot, dtype, dtype, pad=pad), dtype, interleaved=interleaved)


@pytest.mark.parametrize("cache_dtype", [torch.float32, torch.bfloat16, torch.float16, torch.int8])
@pytest.mark.parametrize("by_head", [False, True])
@pytest.mark.parametrize("d", [64, 30])
@pytest.mark.parametrize("dtype,dtype_out", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float16), (torch.float16, torch.float32)])
def test_qk_norm_rope_types_and_layouts_of_the_cache(cache_dtype, by_head, d, dtype, dtype_out):
    check_qk(qk_case(d, 40, 4, 2, d, d, dtype, cache_dtype, page=8, by_head=by_head), dtype_out)


@pytest.mark.parametrize("d", [64, 22])
@pytest.mark.parametrize("norm,gammas,k_out,cached", [(False, False, True, True), (True, False, False, True), (True, True, True, False), (False, False, True, False)])
def test_qk_norm_rope_options(d, norm, gammas, k_out, cached):
    check_qk(qk_case(d, 21, 4, 2, d, d, torch.float32, torch.int8), torch.float32, norm=norm, gammas=gammas, k_out=k_out, cached=cached)


@pytest.mark.parametrize("d", [128, 126])
def test_qk_norm_rope_far_positions(d):
    c = qk_case(5, 64, 2, 1, d, d, torch.float32, torch.float32, far=2 ** 31 - 1)
    c["positions"][0] = 2 ** 31 - 1
    c["positions"][1] = -7
    check_qk(c, torch.float32)


@pytest.mark.parametrize("d", [64, 66])
def test_qk_norm_rope_in_place_and_on_a_stream(d):
    a, b = (qk_case(8, 50, 4, 2, d, d, torch.bfloat16, torch.bfloat16) for _ in range(2))
    q_out, k_out = torch.empty_like(a["q"]), torch.empty_like(a["k"])
    nm.nm_qk_norm_rope(a["q"], a["k"], a["v"], a["positions"], a["inv_freq"], q_out, k_out=k_out, norm=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    nm.nm_qk_norm_rope(b["q"], b["k"], b["v"], b["positions"], b["inv_freq"], b["q"], k_out=b["k"], norm=True, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(b["q"], q_out) and torch.equal(b["k"], k_out) and torch.equal(a["v"], b["v"])


def test_qk_norm_rope_special_values():
    """Zeros stay zeros under the norm, a NaN or an infinity stays in its own head, and codes saturate (NaN: -127)."""
    c = qk_case(2, 4, 2, 2, 64, 64, torch.float32, torch.int8)
    c["slots"] = i32([0, 1, 2, 3])
    c["q"][0], c["k"][0] = 0, 0
    c["q"][1, 1, 5] = float("nan")
    c["k"][2, 0, 7] = float("inf")
    c["v"][3, 1, :3] = torch.tensor([float("nan"), 1e30, -float("inf")], device=DEV)
    q_out = torch.empty((4, 2, 64), device=DEV)
    nm.nm_qk_norm_rope(c["q"], c["k"], c["v"], c["positions"], c["inv_freq"], q_out, norm=True, k_cache=c["cache"][0], v_cache=c["cache"][1],
                       slots=c["slots"], k_inv_scale=c["inv_scale"][0], v_inv_scale=c["inv_scale"][1])
    torch.cuda.synchronize()
    assert bool((q_out[0] == 0).all()) and bool((c["cache"][0, 0, 0] == 0).all())
    assert bool(q_out[1, 1].isnan().all()) and bool(q_out[1, 0].isfinite().all()) and bool(q_out[2:].isfinite().all())
    assert c["cache"][1, 0, 3, 1, :3].tolist() == [-127, 127, -127]


def test_decode_binding_refuses():
    c = qk_case(1, 4, 2, 2, 64, 64, torch.float32, torch.int8)
    q_out = torch.empty((4, 2, 64), device=DEV)
    good = dict(k_cache=c["cache"][0], v_cache=c["cache"][1], slots=c["slots"], k_inv_scale=c["inv_scale"][0], v_inv_scale=c["inv_scale"][1])
    args = [c["q"], c["k"], c["v"], c["positions"], c["inv_freq"], q_out]
    for at, bad in ((0, c["q"].transpose(1, 2)), (0, c["q"][..., ::2]), (1, c["k"].half()), (2, c["v"][:3]), (3, c["positions"].long()),
                    (3, c["positions"][:2]), (4, c["inv_freq"].double()), (5, q_out[:, :1]), (5, q_out.double()), (2, c["v"].cpu())):
        changed = list(args)
        changed[at] = bad
        with pytest.raises(nm.NmError):
            nm.nm_qk_norm_rope(*changed, **good)
    for change in (dict(slots=None), dict(v_cache=None), dict(k_cache=c["cache"][0][:, :, :1]), dict(v_cache=c["cache"][1].half()),
                   dict(k_inv_scale=None), dict(v_inv_scale=c["inv_scale"][1][:1]), dict(slots=c["slots"].long()), dict(q_gamma=c["q_gamma"][:3])):
        with pytest.raises(nm.NmError):
            nm.nm_qk_norm_rope(*args, **{**good, **change})


# ---- attention over the cache -----------------------------------------------------------------------

def paged_case(seed, lens, hq, hk, d, q_dtype, cache_dtype, page=16, by_head=False, columns=None, extra_pages=5, size=1.0):
    """A pool whose free slots, and pages that no request owns, hold NaN (codes: -128): what is behind a length does not matter."""
    g = gen(seed)
    B = len(lens)
    held = [-(-max(n, 0) // page) for n in lens]
    columns = max(held + [1]) if columns is None else columns
    pages = sum(held) + extra_pages
    shape = (2, pages, hk, page, d) if by_head else (2, pages, page, hk, d)
    cache = torch.randn(shape, generator=g)
    cache = (cache * 32).round().clamp(-127, 127).to(torch.int8) if cache_dtype == torch.int8 else (cache * size).to(cache_dtype)
    cache = cache.transpose(2, 3) if by_head else cache
    order = torch.randperm(pages, generator=g).tolist()
    table = torch.full((B, columns), -1, dtype=torch.int32)
    used, at = torch.zeros((pages, page), dtype=torch.bool), 0
    for b, n in enumerate(lens):
        for i in range(held[b]):
            table[b, i] = order[at]
            used[order[at], :max(0, min(page, n - i * page))] = True
            at += 1
    cache[:, ~used] = -128 if cache_dtype == torch.int8 else float("nan")
    scales = 0.02 * (1 + torch.rand((2, hk), generator=g)) if cache_dtype == torch.int8 else None
    cache = cache.to(DEV) if not by_head else cache.transpose(2, 3).contiguous().to(DEV).transpose(2, 3)
    return dict(q=(torch.randn((B, hq, d), generator=g) * size).to(q_dtype).to(DEV), cache=cache, table=table.to(DEV), lens=i32(lens),
                scales=None if scales is None else scales.to(DEV))


def attend(c, out_dtype, scale, window=0, lse=True, ws=None, stream=None, out=None, out_inv_scale=1.0):
    B, hq, d = c["q"].shape
    out = torch.full((B, hq, d), 77, dtype=out_dtype, device=DEV) if out is None else out
    lse = torch.full((B, hq), 77.0, device=DEV) if lse else None
    args = (c["q"], c["cache"][0], c["cache"][1], c["table"], c["lens"], out)
    s = (None, None) if c["scales"] is None else c["scales"]
    more = dict(scale=scale, window=window, k_scale=s[0], v_scale=s[1], lse=lse, out_inv_scale=out_inv_scale)
    size = nm.nm_paged_attention_workspace(*args, **more)
    if ws is None and size:
        ws = torch.full((size,), 0xff, dtype=torch.uint8, device=DEV)     # NaN, so that nothing unwritten is read
    nm.nm_paged_attention(*args, ws=ws, stream=stream, **more)
    return out, lse


def attention_64(c, scale, window=0):
    """(out, lse, bound of out's error, bound of lse's) in binary64, request by request.  A score is a sum of d products in
    binary32: at most (d + 4) U of the absolute products (the matrix instruction adds 32 at a time; 4: the factor, and the scales); its
    difference from the maximum, the exponential (2 steps of the result) and the sums add |s| 4 U, 4 U and, chain of n / 128 additions
    a wavefront, then of pieces and wavefronts, (n / 128 + 64) U; weights in two terms of 8 bits each: 2^-16.  Everything
    is relative to the weighted mean of |v|, twice (numerator and sum)."""
    B, hq, d = c["q"].shape
    _, pages, page, hk, _ = c["cache"].shape
    out = torch.zeros((B, hq, d), dtype=torch.float64, device=DEV)
    lse = torch.full((B, hq), -math.inf, dtype=torch.float64, device=DEV)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    top = c["table"].shape[1] * page
    for b, n in enumerate(c["lens"].tolist()):
        n = min(max(n, 0), top)
        where = torch.arange(max(0, n - window) if window else 0, n, device=DEV)
        entry = c["table"][b].long()[where // page]
        good = (entry >= 0) & (entry < pages)
        where, entry = where[good], entry[good]
        if not where.numel():
            continue
        k, v = (c["cache"][i][entry, where % page].double() for i in (0, 1))
        if c["scales"] is not None:
            k, v = k * c["scales"][0].double()[:, None], v * c["scales"][1].double()[:, None]
        k, v = (x.repeat_interleave(hq // hk, 1).transpose(0, 1) for x in (k, v))         # [hq, n, d]
        q = c["q"][b].double()
        s = (k * q[:, None]).sum(-1) * scale
        size = (k.abs() * q.abs()[:, None]).sum(-1) * abs(scale)
        w = torch.softmax(s, -1)
        out[b], lse[b] = (w[:, :, None] * v).sum(1), torch.logsumexp(s, -1)
        span = (s - s.amax(-1, keepdim=True)).abs()
        err = ((d + 4) * size + 4 * span + n / 128 + 72) * U
        mean = (w * err).sum(-1) + err[torch.arange(hq), s.argmax(-1)]
        e_out[b] = ((w * (err + 2.0 ** -16))[:, :, None] * v.abs()).sum(1) + (mean + 2.0 ** -16)[:, None] * (w[:, :, None] * v.abs()).sum(1)
        e_lse[b] = mean + 4 * U * lse[b].abs()
    return out, lse, e_out, e_lse


def check_attention(c, out_dtype, scale=None, window=0):
    scale = c["q"].shape[2] ** -0.5 if scale is None else scale
    out, lse = attend(c, out_dtype, scale, window)
    torch.cuda.synchronize()
    want, wl, e_out, e_lse = attention_64(c, scale, window)
    assert_rounded(out, want, e_out, "out")
    empty = wl == -math.inf
    assert bool((lse[empty] == -math.inf).all()) and bool((out[empty] == 0).all())
    assert bool(((lse.double() - wl)[~empty].abs() <= e_lse[~empty]).all())
    return out, lse


LENGTHS = [0, 1, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 300, 1000]


@pytest.mark.parametrize("q_dtype,cache_dtype,out_dtype", [
    (torch.bfloat16, torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16, torch.float16), (torch.float32, torch.int8, torch.float32),
    (torch.float32, torch.bfloat16, torch.float32), (torch.bfloat16, torch.int8, torch.bfloat16), (torch.float16, torch.bfloat16, torch.float16),
    (torch.bfloat16, torch.float16, torch.float32), (torch.float32, torch.float16, torch.bfloat16), (torch.float16, torch.int8, torch.float16)])
@pytest.mark.parametrize("hq,hk,d", [(4, 4, 64), (8, 2, 128), (5, 1, 32), (24, 1, 96), (6, 3, 16), (16, 1, 256), (34, 2, 80)])
def test_paged_attention(q_dtype, cache_dtype, out_dtype, hq, hk, d):
    check_attention(paged_case(hq + d, LENGTHS, hq, hk, d, q_dtype, cache_dtype, by_head=bool(d & 32)), out_dtype)


@pytest.mark.parametrize("page", [1, 2, 8, 32, 64, 256, 4096])
@pytest.mark.parametrize("cache_dtype", [torch.bfloat16, torch.int8])
def test_paged_attention_page_sizes(page, cache_dtype):
    check_attention(paged_case(page, [100, 0, 513, 1, 260], 8, 2, 64, torch.bfloat16, cache_dtype, page=page), torch.bfloat16)


@pytest.mark.parametrize("window", [1, 16, 31, 100, 128, 500, 5000])
def test_paged_attention_window(window):
    check_attention(paged_case(window, [0, 1, 90, 128, 700, 1500], 6, 2, 64, torch.float16, torch.float16), torch.float16, window=window)


@pytest.mark.parametrize("lens,hk,columns", [([70000], 2, None), ([40000, 3, 0, 17000], 1, None), ([5, 200], 4, 3000), ([129] * 70, 8, 100)])
def test_paged_attention_long_and_split(lens, hk, columns):
    check_attention(paged_case(len(lens), lens, hk * 4, hk, 128, torch.bfloat16, torch.bfloat16, page=64, columns=columns), torch.bfloat16)


@pytest.mark.parametrize("lens,hq,hk,d,columns", [([1023, 0, 1, 129, 256, 257, 640], 5, 5, 64, 64), ([300], 12, 12, 48, 19), ([140, 7], 34, 2, 16, 9), ([1000] * 3, 8, 2, 64, 63),
                                                  ([900, 3] * 45, 3, 3, 64, 64), ([1024, 130, 0, 700] * 10, 8, 4, 96, 64), ([1025, 1024, 1], 4, 4, 32, 65)])
@pytest.mark.parametrize("q_dtype,cache_dtype,window", [(torch.float32, torch.bfloat16, 0), (torch.bfloat16, torch.int8, 0), (torch.float16, torch.float16, 200)])
def test_paged_attention_rows_whole_or_divided(q_dtype, cache_dtype, window, lens, hq, hk, d, columns):
    """Tables of up to 1024 positions and a little more: a row to a workgroup of four or eight wavefronts, or divided."""
    check_attention(paged_case(hk + d, lens, hq, hk, d, q_dtype, cache_dtype, columns=columns), q_dtype, window=window)


@pytest.mark.parametrize("B,hq,hk,d,by_head,window", [(48, 16, 16, 64, False, 0), (48, 16, 16, 64, True, 0), (40, 32, 16, 32, False, 0), (130, 24, 6, 48, False, 333), (100, 8, 8, 16, False, 0),
                                                       (100, 64, 8, 64, False, 1000), (99, 128, 8, 64, False, 0), (60, 14, 14, 64, False, 0), (9, 96, 96, 16, False, 0), (130, 16, 16, 16, False, 2000)])
@pytest.mark.parametrize("q_dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_paged_attention_many_heads_of_codes(q_dtype, B, hq, hk, d, by_head, window):
    """Enough rows and columns of the table that neighbouring key heads are taken as one, where they lie next to each other; ragged lengths."""
    lens = [(i * i * 37) % 700 if i % 5 else 4000 * (i % 10 == 5) for i in range(B)]
    c = paged_case(B + d, lens, hq, hk, d, q_dtype, torch.int8, page=32, by_head=by_head, columns=130)
    c["q"][1, :, 0] *= 100.0
    check_attention(c, q_dtype, window=window)


def test_paged_attention_bad_tables_and_lengths():
    """Entries that are no pages take no part, lengths beyond the table count as the table's, negative ones as none."""
    c = paged_case(3, [100, 200, 64, 33, 50], 4, 2, 64, torch.bfloat16, torch.bfloat16, columns=13)
    c["table"][0, 2], c["table"][0, 6], c["table"][2, :] = -5, 10 ** 6, 2 ** 31 - 1
    c["table"][1, 3] = c["cache"].shape[1]
    c["lens"][3], c["lens"][1] = -4, 5000
    c["cache"] = torch.nan_to_num(c["cache"], nan=0.25)
    out, lse = check_attention(c, torch.bfloat16)
    assert bool((out[2:4] == 0).all()) and bool((lse[2:4] == -math.inf).all())


def test_paged_attention_large_scores_and_sizes():
    """Scores of thousands (one weight is 1), queries near the types' ends, and a row whose own values are infinite or NaN."""
    c = paged_case(9, [300, 300, 300, 300], 4, 2, 64, torch.float32, torch.float16, size=30.0)
    check_attention(c, torch.float32, scale=1.0)
    c["q"] *= 1e30
    check_attention(c, torch.float32, scale=1e-30)
    c["q"] *= 1e-55
    check_attention(c, torch.float32, scale=1e25)
    c["cache"][0, c["table"][1, 3], 5, 0, 1] = float("inf")
    c["cache"][1, c["table"][2, 3], 5, 1, 7] = float("nan")
    out, _ = attend(c, torch.float32, 1e25)
    torch.cuda.synchronize()
    assert bool(out[0].isfinite().all()) and bool(out[3].isfinite().all()) and bool(out[1, 2:].isfinite().all())
    assert bool(out[2, 2:, 7].isnan().all()) and bool(out[2, :2].isfinite().all()) and bool(out[2, 2:, :7].isfinite().all())


def test_paged_attention_codes_strides_and_stream():
    """int8 results are the codes of the fp32 ones; requests may be strided; another stream gives the same; no lse."""
    c = paged_case(4, [77, 500, 1200], 8, 2, 64, torch.bfloat16, torch.int8)
    f, _ = attend(c, torch.float32, 0.125)
    codes, _ = attend(c, torch.int8, 0.125, out_inv_scale=50.0)
    torch.cuda.synchronize()
    assert int((codes.double() - (f.double() * 50).clamp(-127, 127)).abs().gt(0.5 + 127 * 2.0 ** -15).sum()) == 0
    wide = torch.full((3, 12, 64), 5.0, dtype=torch.bfloat16, device=DEV)
    qw = torch.zeros((3, 24, 64), dtype=torch.bfloat16, device=DEV)
    qw[:, 8:16] = c["q"]
    want, _ = attend(c, torch.bfloat16, 0.125)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    attend({**c, "q": qw[:, 8:16]}, torch.bfloat16, 0.125, lse=False, stream=s, out=wide[:, 2:10])
    torch.cuda.synchronize()
    assert torch.equal(wide[:, 2:10], want) and bool((wide[:, :2] == 5).all()) and bool((wide[:, 10:] == 5).all())


@pytest.mark.parametrize("lens", [[300, 1, 0, 77], [5000, 2, 0, 1999, 640]])
def test_paged_attention_in_place(lens):
    c = paged_case(12, lens, 8, 2, 64, torch.bfloat16, torch.bfloat16)
    want, _ = attend(c, torch.bfloat16, 0.125)
    want = want.clone()
    q = c["q"].clone()
    got, _ = attend({**c, "q": q}, torch.bfloat16, 0.125, out=q)
    torch.cuda.synchronize()
    assert torch.equal(q, want)


def test_paged_attention_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes (and elements): the last pages of the pool."""
    pages, page, d = (1 << 32) // (16 * 64) + 40, 16, 64
    cache = torch.zeros((2, pages, page, 1, d), dtype=torch.int8, device=DEV)
    g = gen(1)
    own = [pages - 1, 3, pages - 2, pages // 2 + 7]
    for p in own:
        cache[:, p] = torch.randint(-127, 128, (2, page, 1, d), generator=g, dtype=torch.int8).to(DEV)
    c = dict(q=torch.randn((1, 4, d), generator=g).to(torch.bfloat16).to(DEV), cache=cache, table=i32([own]), lens=i32([61]), scales=torch.full((2, 1), 0.02, device=DEV))
    check_attention(c, torch.bfloat16)
    k, v = (torch.randn((1, 1, d), generator=g).to(DEV) for _ in range(2))
    q_out = torch.empty((1, 1, d), device=DEV)
    nm.nm_qk_norm_rope(k, k, v, None, None, q_out, k_cache=cache[0], v_cache=cache[1], slots=i32([(pages - 1) * page + 3]),
                       k_inv_scale=torch.full((1,), 40.0, device=DEV), v_inv_scale=torch.full((1,), 40.0, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(cache[1, pages - 1, 3], (v[0] * 40).round().clamp(-127, 127).to(torch.int8))


# ---- products with 4-bit weights ----------------------------------------------------------------------

def w4_case(seed, M, N, K, group, x_dtype, scale_dtype, pad=0):
    g = gen(seed)
    x = torch.randn((M, K + pad), generator=g)
    x = (x * 32).round().clamp(-128, 127).to(torch.int8) if x_dtype == torch.int8 else x.to(x_dtype)
    w = torch.randint(-8, 8, (N, K), generator=g)
    packed = ((w[:, 0::2] & 15) | ((w[:, 1::2] & 15) << 4)).to(torch.uint8)
    scales = (0.02 * (0.5 + torch.rand((N, K // group), generator=g))).to(scale_dtype)
    return dict(x=x.to(DEV)[:, :K], w=w.to(DEV), W=packed.to(DEV), scales=scales.to(DEV), group=group,
                bias=torch.randn(N, generator=g).to(DEV), alpha=0.03 if x_dtype == torch.int8 else 0.7)


def product_64(c, bias=True):
    """(result, bound of the 32-bit evaluation's error).  int8: sums within 128 weights are exact, then at most K / 1024 + 8 additions and 3 more
    roundings: (K / 1024 + 11) U of sum |x w| s.  bf16, fp16: within 128 weights eight matrix instructions of weights (at most 31) and
    offsets (24) add, each a tree of five levels and the accumulator, 48 roundings, 96 where they truncate: 96 U of sum |x| 55 s more."""
    s = c["scales"].double().repeat_interleave(c["group"], 1)
    w, x, a = c["w"].double() * s, c["x"].double(), c["alpha"]
    K = x.shape[1]
    y = x @ w.t().contiguous() * a + (c["bias"].double() if bias else 0)
    e = (K / 1024 + 11) * U * (x.abs() @ w.abs().t().contiguous()) * abs(a) + 2 * U * (y.abs() + (c["bias"].double().abs() if bias else 0))
    if c["x"].dtype != torch.int8:
        e = e + 96 * 55 * U * (x.abs() @ s.t().contiguous()) * abs(a)
    return y, e


def check_w4(c, out_dtype, bias=True):
    M, N = c["x"].shape[0], c["W"].shape[0]
    wide = torch.full((M, N + 3), 55.0, dtype=out_dtype, device=DEV)
    nm.nm_gemv_w4(c["x"], c["W"], c["scales"], wide[:, :N], group=c["group"], alpha=c["alpha"], bias=c["bias"] if bias else None)
    torch.cuda.synchronize()
    want, error = product_64(c, bias)
    assert_rounded(wide[:, :N], want, error, "product")
    assert bool((wide[:, N:] == 55).all())
    return wide[:, :N]


@pytest.mark.parametrize("x_dtype,scale_dtype,out_dtype", [(torch.int8, torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16, torch.bfloat16),
                                                           (torch.float16, torch.float16, torch.float16), (torch.bfloat16, torch.float32, torch.float32),
                                                           (torch.int8, torch.float16, torch.bfloat16)])
@pytest.mark.parametrize("M,N,K,group", [(1, 1, 32, 32), (1, 16, 128, 128), (2, 17, 160, 32), (3, 100, 192, 64), (7, 33, 1024, 256), (1, 768, 768, 128),
                                         (16, 40, 4096, 64), (17, 50, 2048, 512), (33, 31, 1120, 32), (64, 130, 896, 128), (65, 20, 384, 384),
                                         (1, 5, 65536, 128), (200, 9, 320, 64)])
def test_gemv_w4(x_dtype, scale_dtype, out_dtype, M, N, K, group):
    check_w4(w4_case(M + K, M, N, K, group, x_dtype, scale_dtype), out_dtype, bias=N % 2 == 0)


@pytest.mark.parametrize("x_dtype,scale_dtype,out_dtype", [(torch.int8, torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16, torch.bfloat16),
                                                           (torch.float16, torch.float32, torch.float32)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(1, 70, 2304), (16, 50, 11008), (33, 100, 2432), (2, 4100, 384), (16, 4097, 4224), (17, 2100, 896), (32, 2070, 4992), (40, 3001, 2176),
                                   (41, 8193, 1152), (48, 8200, 2560), (130, 1031, 2304)])
def test_gemv_w4_shares_of_the_work(x_dtype, scale_dtype, out_dtype, group, M, N, K):
    """Either side of 256 workgroups and of 2048 columns of x, with one, two and three tiles of rows."""
    check_w4(w4_case(M + N, M, N, K, group, x_dtype, scale_dtype), out_dtype)


@pytest.mark.parametrize("x_dtype", [torch.int8, torch.bfloat16, torch.float16])
def test_gemv_w4_every_weight_in_every_place(x_dtype):
    """Rows of x with a single one read one weight each: exact, so every place of a word and every one of the 16 weights is seen."""
    K = 256
    c = w4_case(3, 64, 48, K, 32, x_dtype, torch.float32)
    c["scales"].fill_(1.0)
    got = torch.empty((64, 48), device=DEV)
    for first in range(0, K, 64):
        x = torch.zeros((64, K), dtype=x_dtype, device=DEV)
        x[torch.arange(64), first + torch.arange(64)] = 1
        nm.nm_gemv_w4(x, c["W"], c["scales"], got, group=32)
        torch.cuda.synchronize()
        assert torch.equal(got, c["w"][:, first:first + 64].t().float())


def test_gemv_w4_strides_stream_and_codes():
    c = w4_case(5, 9, 70, 512, 64, torch.int8, torch.float32, pad=16)
    y = check_w4(c, torch.float32)
    codes = torch.empty((9, 70), dtype=torch.int8, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    nm.nm_gemv_w4(c["x"], c["W"], c["scales"], codes, group=64, alpha=c["alpha"], bias=c["bias"], out_inv_scale=20.0, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(codes, (y * 20.0).clamp(-127, 127).round().to(torch.int8))


@pytest.mark.parametrize("spec", [("gelu", -8.0, 8.0, 64, 0), ("relu", -8.0, 8.0, 2, 0), ("gelu", -4.0, 4.0, 1000, nm.NM_TABLE_CLAMP_INPUT),
                                  ("exp", -8.0, 0.0, 64, nm.NM_TABLE_MERGE | nm.NM_TABLE_COMPACT, 0.0, 0.05)])
def test_gemv_w4_table(spec):
    """The table of the result: the same values as nm_pwl_apply of the product without it."""
    c = w4_case(8, 5, 90, 256, 128, torch.int8, torch.float32)
    tables = nm.nm_build_tables([spec])
    y, z, want = (torch.empty((5, 90), device=DEV) for _ in range(3))
    args = dict(group=128, alpha=c["alpha"], bias=c["bias"])
    nm.nm_gemv_w4(c["x"], c["W"], c["scales"], y, **args)
    nm.nm_gemv_w4(c["x"], c["W"], c["scales"], z, tables=tables, table_idx=0, **args)
    nm.nm_pwl_apply(y, 1.0, tables, 0, 1.0, out_f32=want)
    torch.cuda.synchronize()
    assert torch.equal(z, want)


def test_gemv_w4_infinities_stay_in_their_rows():
    c = w4_case(6, 20, 33, 256, 64, torch.bfloat16, torch.float32)
    want, _ = product_64(c)
    clean = check_w4(c, torch.float32).clone()
    c["x"][4, 100], c["x"][17, 3] = float("inf"), float("nan")
    got = torch.empty((20, 33), device=DEV)
    nm.nm_gemv_w4(c["x"], c["W"], c["scales"], got, group=64, alpha=c["alpha"], bias=c["bias"])
    torch.cuda.synchronize()
    rest = [m for m in range(20) if m not in (4, 17)]
    assert torch.equal(got[rest], clean[rest]) and not bool(got[[4, 17]].isfinite().any())


def test_gemv_w4_binding_refuses():
    c = w4_case(1, 2, 16, 128, 64, torch.bfloat16, torch.float32)
    out = torch.empty((2, 16), device=DEV)
    good = [c["x"], c["W"], c["scales"], out]
    for at, bad, group in ((0, c["x"].double(), 64), (0, c["x"].cpu(), 64), (1, c["W"].to(torch.int8), 64), (1, c["W"][:, :32], 64), (2, c["scales"][:, :1], 64),
                           (2, c["scales"].t().contiguous().t(), 64), (3, out[:, :15], 64), (3, out.t(), 64), (0, c["x"], 48), (0, c["x"], 0), (0, c["x"], 32)):
        changed = list(good)
        changed[at] = bad
        with pytest.raises(nm.NmError):
            nm.nm_gemv_w4(*changed, group=group)


# ---- a step as it is used: plan, QKV product, norms and rotation into the cache, attention, output product -----------------

def step_64(x_codes, weights, s, table, positions, lens, page, cache, hq, hk, d):
    """A decoder's attention block for one token a request, in binary64 on the given (rounded) weights and cache."""
    qkv = x_codes.double() @ weights["qkv"].double().t().contiguous() * s["alpha_qkv"] + weights["bqkv"].double()
    B = x_codes.shape[0]
    q, k, v = (qkv[:, a * d:b * d].view(B, -1, d) for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    q, _ = rotate_64(q, positions, s["inv_freq"], s["gq"], True, False)
    k, _ = rotate_64(k, positions, s["inv_freq"], s["gk"], True, False)
    out = torch.zeros((B, hq, d), dtype=torch.float64, device=DEV)
    cache = cache.clone()
    for b in range(B):
        n = int(lens[b])
        where = torch.arange(n, device=DEV)
        row = table[b].long()[where // page]
        cache[0, row[-1], (n - 1) % page], cache[1, row[-1], (n - 1) % page] = k[b], v[b]
        kk, vv = (cache[i][row, where % page].repeat_interleave(hq // hk, 1).transpose(0, 1) for i in (0, 1))
        w = torch.softmax((kk * q[b][:, None]).sum(-1) * d ** -0.5, -1)
        out[b] = (w[:, :, None] * vv).sum(1)
    return out, cache


@pytest.mark.parametrize("graph", [False, True])
def test_a_decoder_step(graph):
    """Three steps one after the other on one set of buffers, eager or captured once and replayed (twice each: a step is idempotent): the
    framework's int8 product writes q, k, v in fp32; attention writes int8 codes, which a 4-bit product reads.  Every step against binary64."""
    B, hq, hk, d, H, page, columns = 5, 8, 2, 64, 256, 16, 40
    g, cached = gen(77), [0, 15, 16, 300, 627]
    pages = B * columns + 3
    s = dict(alpha_qkv=2e-4, inv_freq=(10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().to(DEV),
             gq=(1 + 0.1 * torch.randn(d, generator=g)).to(DEV), gk=(1 + 0.1 * torch.randn(d, generator=g)).to(DEV))
    weights = dict(qkv=torch.randint(-127, 128, ((hq + 2 * hk) * d, H), generator=g, dtype=torch.int8).to(DEV), bqkv=(0.1 * torch.randn((hq + 2 * hk) * d, generator=g)).to(DEV))
    wo = torch.randint(-8, 8, (H, hq * d), generator=g)
    wo_packed, wo_scales = ((wo[:, 0::2] & 15) | ((wo[:, 1::2] & 15) << 4)).to(torch.uint8).to(DEV), (0.01 + 0.01 * torch.rand((H, hq * d // 64), generator=g)).to(DEV)
    cache = torch.randn((2, pages, page, hk, d), generator=g).to(torch.bfloat16).to(DEV)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((B, columns), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(cached):
        held = -(-n // page)
        table[b, :held] = order[at:at + held]
        at += held
    table, free = table.to(DEV), order[at:].to(DEV)
    x = torch.empty((B, H), dtype=torch.int8, device=DEV)
    now, fresh, begin, end, lens, status = i32(cached), i32([1] * B), i32([0]), i32([0]), i32([0] * B), i32([9] * 4)
    slots, positions = i32([0] * (B + 2)), i32([0] * (B + 2))               # two rows more than there are tokens: a padded batch
    qkv = torch.zeros((B + 2, (hq + 2 * hk) * d), device=DEV)
    q = torch.zeros((B + 2, hq, d), dtype=torch.bfloat16, device=DEV)
    ctx = torch.empty((B, hq, d), dtype=torch.int8, device=DEV)
    y, lse = torch.empty((B, H), device=DEV), torch.empty((B, hq), device=DEV)
    third = lambda a, b: qkv[:, a * d:b * d].view(B + 2, -1, d)  # noqa: E731
    paged = nm.make_paged_desc(q[:B], cache[0], cache[1], table, lens, ctx, scale=d ** -0.5, out_inv_scale=60.0, lse=lse)
    ws = torch.empty(nm.nm_paged_attention_workspace(paged), dtype=torch.uint8, device=DEV)

    def step():
        nm.nm_page_plan(now, fresh, free, begin, table, page_size=page, num_pages=pages, free_end=end, lens=lens, slots=slots, positions=positions, status=status)
        nm.nm_gemm_pwl(x, weights["qkv"], bias=weights["bqkv"], alpha=s["alpha_qkv"], out_f32=qkv[:B])
        nm.nm_qk_norm_rope(third(0, hq), third(hq, hq + hk), third(hq + hk, hq + 2 * hk), positions, s["inv_freq"], q, norm=True, q_gamma=s["gq"],
                           k_gamma=s["gk"], k_cache=cache[0], v_cache=cache[1], slots=slots)
        nm.nm_paged_attention(paged, ws=ws)
        nm.nm_gemv_w4(ctx.view(B, hq * d), wo_packed, wo_scales, y, group=64, alpha=1 / 60.0)

    captured = None
    for _ in range(3):
        x.copy_(torch.randint(-127, 128, (B, H), generator=g, dtype=torch.int8))
        before = cache.double()
        if graph and captured is None:
            step()
            torch.cuda.synchronize()
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                step()
        for _ in range(2):
            (captured.replay if graph else step)()
            torch.cuda.synchronize()
        assert status.tolist()[0] == 0 and lens.tolist() == [n + 1 for n in now.tolist()] and slots.tolist()[B:] == [-1, -1]
        want, full = step_64(x, weights, s, table, positions[:B], lens, page, before, hq, hk, d)
        # q and the new keys and values are rounded to bf16 (2^-8 relative: |score| / 8 at most sqrt(d) gammas, so 8 * 2^-7 * 1.4^2 / 2 on a score, which
        # is that on a weight, twice; 2^-8 on a value of some 4), then the context to codes of 1 / 60
        off = (ctx.double() / 60 - want.clamp(-127 / 60, 127 / 60)).abs()
        assert float(off.max()) <= 0.5 / 60 + 4 * (2 * 8 * 2.0 ** -7 + 2.0 ** -8), float(off.max())
        assert float(off.mean()) < 0.01                                       # half a code is 0.0083
        w = wo.to(DEV).double() * wo_scales.double().repeat_interleave(64, 1)
        product = ctx.view(B, -1).double() @ w.t().contiguous() / 60
        bound = (hq * d / 1024 + 13) * U * (ctx.view(B, -1).double().abs() @ w.abs().t().contiguous()) / 60 + 2 * U * product.abs()
        assert bool(((y.double() - product).abs() <= bound).all())
        assert float((cache.double() - full).abs().max()) <= 2.0 ** -8 * float(full.abs().max()) + 1e-4
        now.copy_(lens)
        begin.copy_(end)


def test_two_calls_at_once_and_replays():
    """Each call twice at once on two streams, with outputs (and workspaces) of their own, and captured and replayed: the same bits every time."""
    a = paged_case(31, [3000, 17, 900, 0, 2500], 8, 2, 128, torch.bfloat16, torch.bfloat16, page=64)
    w = w4_case(32, 20, 200, 2048, 128, torch.bfloat16, torch.bfloat16)
    qk = [qk_case(33, 300, 8, 2, 128, 128, torch.bfloat16, torch.bfloat16) for _ in range(2)]
    outs = [dict(o=torch.zeros((5, 8, 128), dtype=torch.bfloat16, device=DEV), y=torch.zeros((20, 200), dtype=torch.bfloat16, device=DEV),
                 q=torch.zeros((300, 8, 128), dtype=torch.bfloat16, device=DEV)) for _ in range(2)]
    descs = [nm.make_paged_desc(a["q"], a["cache"][0], a["cache"][1], a["table"], a["lens"], o["o"], scale=0.1) for o in outs]
    wss = [torch.empty(nm.nm_paged_attention_workspace(x), dtype=torch.uint8, device=DEV) for x in descs]

    def calls(i):
        nm.nm_paged_attention(descs[i], ws=wss[i])
        nm.nm_gemv_w4(w["x"], w["W"], w["scales"], outs[i]["y"], group=128, bias=w["bias"])
        c = qk[i]
        nm.nm_qk_norm_rope(c["q"], c["k"], c["v"], c["positions"], c["inv_freq"], outs[i]["q"], norm=True, k_cache=c["cache"][0], v_cache=c["cache"][1], slots=c["slots"])

    calls(0)
    torch.cuda.synchronize()
    want = {n: t.clone() for n, t in outs[0].items()}
    want_cache = qk[0]["cache"].clone()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for o in outs:
            for t in o.values():
                t.zero_()
        torch.cuda.synchronize()
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                calls(i)
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(outs[i][n], want[n]) for n in want) and torch.equal(qk[i]["cache"], want_cache)
    graphs = []
    for i in (0, 1):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls(i)
        graphs.append(graph)
    for _ in range(4):
        for o in outs:
            for t in o.values():
                t.zero_()
        torch.cuda.synchronize()
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                graphs[i].replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(outs[i][n], want[n]) for n in want) and torch.equal(qk[i]["cache"], want_cache)


def test_a_graph_follows_the_lengths():
    """A captured call reads lengths and tables when it is replayed: other lengths, and back."""
    c = paged_case(41, [5, 700, 3000, 64], 8, 2, 64, torch.bfloat16, torch.int8)
    out = torch.zeros((4, 8, 64), dtype=torch.bfloat16, device=DEV)
    desc = nm.make_paged_desc(c["q"], c["cache"][0], c["cache"][1], c["table"], c["lens"], out, scale=0.125, k_scale=c["scales"][0], v_scale=c["scales"][1])
    ws = torch.empty(nm.nm_paged_attention_workspace(desc), dtype=torch.uint8, device=DEV)
    nm.nm_paged_attention(desc, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nm.nm_paged_attention(desc, ws=ws)
    for lens in ([5, 700, 3000, 64], [1, 0, 2999, 63], [0, 0, 0, 0], [5, 700, 1, 64], [5, 700, 3000, 64]):
        c["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        want, _, error, _ = attention_64(c, 0.125)
        assert_rounded(out, want, error, str(lens))


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-3])
@pytest.mark.parametrize("q_dtype,cache_dtype", [(torch.float32, torch.float16), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.int8)])
def test_paged_attention_scales(scale, q_dtype, cache_dtype):
    check_attention(paged_case(12, [1, 40, 900, 0], 4, 2, 64, q_dtype, cache_dtype), torch.float32, scale=scale)


@pytest.mark.parametrize("hq,hk,d,cache_dtype,by_head", [(16, 8, 16, torch.int8, False), (8, 8, 32, torch.int8, False), (40, 2, 32, torch.bfloat16, False),
                                                         (6, 6, 16, torch.float16, True), (64, 4, 32, torch.int8, False)])
@pytest.mark.parametrize("lens", [[2000, 1, 0, 700, 129], [0, 0, 0], [3], [130] * 40])
def test_paged_attention_heads_that_share_lines(hq, hk, d, cache_dtype, by_head, lens):
    check_attention(paged_case(13, lens, hq, hk, d, torch.float32, cache_dtype, page=32, by_head=by_head, columns=64), torch.float32)


def test_paged_attention_many_short_requests():
    r = np.random.default_rng(5)
    lens = [int(n) if n > 3 else 0 for n in r.integers(0, 60, 700)]
    lens[350] = 2500
    check_attention(paged_case(14, lens, 2, 1, 64, torch.bfloat16, torch.bfloat16, columns=200), torch.bfloat16)


def test_page_plan_outputs_at_odd_addresses():
    cached, fresh, free, table, pages = random_plan(21, 30, 16, 100, 9)
    T = sum(fresh) + 3
    want = plan_in_python(cached, fresh, free, 0, table, 16, pages, T)
    a = torch.full((3, T + 9), -5, dtype=torch.int32, device=DEV)
    o = [a[i, i + 1:i + 1 + T] for i in range(3)]
    nm.nm_page_plan(i32(cached), i32(fresh), i32(free), i32([0]), torch.from_numpy(table).to(DEV), page_size=16, num_pages=pages, free_end=i32([0]), slots=o[0],
                    positions=o[1], requests=o[2], status=i32([0] * 4))
    torch.cuda.synchronize()
    assert [x.cpu().tolist() for x in o] == [want["slots"], want["positions"], want["requests"]]
    for i in range(3):
        assert bool((a[i, :i + 1] == -5).all()) and bool((a[i, i + 1 + T:] == -5).all())
