"""CPU-only checks of the calls of a decode step: what they refuse, before anything reaches the GPU."""
import ctypes as C

import pytest

from paper_2305_14405_amd import binding as nm

Z = C.c_void_p(0)
P = 4096  # a non-null dummy address; never dereferenced because validation fails first


@pytest.fixture(scope="module")
def lib():
    return nm.load(preload_torch=False)


def refused(call, desc, wanted, **changes):
    """The call's status with some fields of a good description changed."""
    keep = {n: getattr(desc, n) for n in changes}
    for n, v in changes.items():
        setattr(desc, n, v)
    rc = call(C.byref(desc), Z)
    for n, v in keep.items():
        setattr(desc, n, v)
    assert rc == wanted, (changes, rc, nm.nm_last_error())
    assert nm.nm_last_error() != ""


def plan():
    d = nm.PlanDesc()
    d.B, d.page_size, d.num_pages, d.max_pages, d.n_free, d.max_tokens, d.table_stride = 4, 16, 64, 8, 10, 100, 8
    for i, n in enumerate(("cached", "fresh", "free_pages", "free_begin", "free_end", "block_table", "lens", "row_start", "slots",
                           "positions", "requests", "status")):
        setattr(d, n, P * (i + 1))
    return d


@pytest.mark.parametrize("changes", [
    dict(B=-1), dict(num_pages=-1), dict(max_pages=-1), dict(n_free=-1), dict(max_tokens=-1), dict(table_stride=7),
    dict(free_begin=None), dict(free_end=None), dict(status=None), dict(slots=None), dict(cached=None), dict(fresh=None),
    dict(block_table=None), dict(free_pages=None), dict(lens=P), dict(free_end=P * 4), dict(row_start=2 * P)])
def test_page_plan_refuses(lib, changes):
    refused(lib.nm_page_plan, plan(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.mark.parametrize("changes", [dict(B=nm.NM_PLAN_MAX_REQUESTS + 1), dict(page_size=0), dict(page_size=24), dict(page_size=1 << 17),
                                     dict(num_pages=1 << 27),
                                     dict(max_tokens=(1 << 30) + 1), dict(n_free=(1 << 30) + 1)])
def test_page_plan_does_not_cover(lib, changes):
    refused(lib.nm_page_plan, plan(), nm.NM_ERR_UNSUPPORTED, **changes)


def test_page_plan_positions_of_31_bits(lib):
    refused(lib.nm_page_plan, plan(), nm.NM_ERR_UNSUPPORTED, page_size=1 << 16, max_pages=1 << 15, table_stride=1 << 15)


def test_page_plan_null(lib):
    assert lib.nm_page_plan(None, Z) == nm.NM_ERR_INVALID_ARG


def qk():
    d = nm.QkDesc()
    d.T, d.hq, d.hk, d.d, d.rot, d.flags = 3, 4, 2, 64, 32, nm.NM_QK_NORM
    d.in_dtype, d.out_dtype, d.cache_dtype, d.num_pages, d.page_size = nm.NM_DT_BF16, nm.NM_DT_F32, nm.NM_DT_I8, 8, 16
    for i, n in enumerate(("q", "k", "v", "q_gamma", "k_gamma", "positions", "inv_freq", "q_out", "k_out", "k_cache", "v_cache", "slots",
                           "k_inv_scale", "v_inv_scale")):
        setattr(d, n, P * (i + 1))
    d.q_stride, d.k_stride, d.v_stride, d.q_out_stride, d.k_out_stride, d.eps = 512, 512, 512, 256, 128, 1e-6
    d.page_stride, d.slot_stride, d.head_stride = 2048, 128, 64
    return d


@pytest.mark.parametrize("changes", [
    dict(T=-1), dict(hq=0), dict(hk=0), dict(d=0), dict(rot=-2), dict(rot=31), dict(rot=66), dict(flags=4), dict(in_dtype=nm.NM_DT_I8),
    dict(out_dtype=nm.NM_DT_I8), dict(cache_dtype=nm.NM_DT_I32), dict(eps=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(k_cache=None),
    dict(v_cache=None), dict(q_stride=255), dict(k_stride=127), dict(v_stride=127), dict(q_out_stride=255), dict(k_out_stride=127),
    dict(num_pages=-1), dict(page_stride=-1), dict(slot_stride=-1), dict(head_stride=-1), dict(k_inv_scale=None), dict(v_inv_scale=None),
    dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(slots=None), dict(positions=None), dict(inv_freq=None),
    dict(q_out=P), dict(k_out=2 * P), dict(q_out=P, out_dtype=nm.NM_DT_BF16)])
def test_qk_norm_rope_refuses(lib, changes):
    refused(lib.nm_qk_norm_rope, qk(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.mark.parametrize("changes", [dict(d=258, q_stride=2000, k_stride=2000, v_stride=2000, q_out_stride=2000, k_out_stride=2000),
                                     dict(page_size=12), dict(num_pages=1 << 27), dict(T=(1 << 23) + 1), dict(hq=1 << 16)])
def test_qk_norm_rope_does_not_cover(lib, changes):
    refused(lib.nm_qk_norm_rope, qk(), nm.NM_ERR_UNSUPPORTED, **changes)


def test_qk_norm_rope_null_and_empty(lib):
    assert lib.nm_qk_norm_rope(None, Z) == nm.NM_ERR_INVALID_ARG
    d = qk()
    d.T, d.q, d.k, d.v, d.q_out, d.slots, d.positions = 0, None, None, None, None, None, None
    assert lib.nm_qk_norm_rope(C.byref(d), Z) == nm.NM_OK  # nothing to do


def paged():
    d = nm.PagedDesc()
    d.B, d.hq, d.hk, d.d, d.q_dtype, d.cache_dtype, d.out_dtype = 2, 8, 2, 64, nm.NM_DT_F32, nm.NM_DT_I8, nm.NM_DT_BF16
    d.page_size, d.num_pages, d.max_pages, d.q_stride, d.out_stride, d.table_stride = 16, 100, 40, 512, 512, 40
    for i, n in enumerate(("q", "k_cache", "v_cache", "k_scale", "v_scale", "block_table", "lens", "out", "lse")):
        setattr(d, n, P * (i + 1))
    d.page_stride, d.slot_stride, d.head_stride, d.scale, d.out_inv_scale = 2048, 128, 64, 0.125, 1.0
    return d


def attend(lib):
    return lambda desc, stream: lib.nm_paged_attention(desc, C.c_void_p(P), 1 << 40, stream)


@pytest.mark.parametrize("changes", [
    dict(B=-1), dict(hq=0), dict(hk=0), dict(hq=9), dict(d=0), dict(max_pages=-1), dict(num_pages=-1), dict(window=-1), dict(q_dtype=nm.NM_DT_I8),
    dict(cache_dtype=nm.NM_DT_F32), dict(out_dtype=nm.NM_DT_I32), dict(q_stride=511), dict(out_stride=511), dict(table_stride=39), dict(page_stride=-16),
    dict(slot_stride=-16), dict(head_stride=-16), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(lens=None), dict(out=None),
    dict(block_table=None), dict(k_cache=None), dict(v_cache=None), dict(k_scale=None), dict(v_scale=None)])
def test_paged_attention_refuses(lib, changes):
    refused(attend(lib), paged(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.mark.parametrize("changes", [
    dict(d=72), dict(d=272, q_stride=4000, out_stride=4000), dict(page_size=3), dict(num_pages=1 << 27), dict(max_pages=1 << 26, table_stride=1 << 26),
    dict(k_cache=P + 8), dict(v_cache=P + 4), dict(page_stride=2056), dict(slot_stride=136), dict(head_stride=72), dict(B=1 << 23, hq=2), dict(num_pages=1 << 20, page_stride=1 << 15), dict(num_pages=1 << 20, page_stride=1 << 14, cache_dtype=nm.NM_DT_BF16)])
def test_paged_attention_does_not_cover(lib, changes):
    refused(attend(lib), paged(), nm.NM_ERR_UNSUPPORTED, **changes)


def test_paged_attention_workspace(lib):
    n, d = C.c_size_t(), paged()
    assert lib.nm_paged_attention_workspace(None, C.byref(n)) == nm.NM_ERR_INVALID_ARG
    assert lib.nm_paged_attention_workspace(C.byref(d), None) == nm.NM_ERR_INVALID_ARG
    assert lib.nm_paged_attention_workspace(C.byref(d), C.byref(n)) == nm.NM_OK and n.value > 0
    for ws, size in ((None, n.value), (P, n.value - 1), (P + 128, n.value)):
        assert lib.nm_paged_attention(C.byref(d), C.c_void_p(ws), size, Z) == nm.NM_ERR_WORKSPACE
        assert "workspace" in nm.nm_last_error()
    d.max_pages = d.table_stride = 1
    assert lib.nm_paged_attention_workspace(C.byref(d), C.byref(n)) == nm.NM_OK and n.value == 0   # one piece needs none
    d.B, d.q, d.out, d.lens = 0, None, None, None
    assert lib.nm_paged_attention(C.byref(d), None, 0, Z) == nm.NM_OK


def w4():
    d = nm.W4Desc()
    d.M, d.N, d.K, d.group, d.x_dtype, d.scale_dtype, d.out_dtype = 3, 20, 256, 64, nm.NM_DT_BF16, nm.NM_DT_F32, nm.NM_DT_I8
    d.x, d.W, d.scales, d.bias, d.out = P, 2 * P, 3 * P, 4 * P, 5 * P
    d.x_stride, d.out_stride, d.alpha, d.table_idx, d.out_inv_scale = 256, 20, 1.0, -1, 1.0
    return d


@pytest.mark.parametrize("changes", [
    dict(M=-1), dict(N=0), dict(K=0), dict(group=0), dict(group=-64), dict(x_dtype=nm.NM_DT_F32), dict(scale_dtype=nm.NM_DT_I8), dict(out_dtype=nm.NM_DT_I32),
    dict(K=288), dict(group=128, K=192), dict(x_stride=255), dict(out_stride=19), dict(alpha=float("nan")), dict(alpha=float("inf")), dict(table_idx=0),
    dict(x=None), dict(W=None), dict(scales=None), dict(out=None)])
def test_gemv_w4_refuses(lib, changes):
    refused(lib.nm_gemv_w4, w4(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.mark.parametrize("changes", [dict(group=16), dict(group=96, K=192), dict(K=65536 + 64, x_stride=1 << 17), dict(M=(1 << 20) + 1), dict(N=1 << 26, out_stride=1 << 26),
                                     dict(x=P + 8), dict(W=P + 8), dict(x_stride=260), dict(M=1 << 20, N=1 << 13, out_stride=1 << 13)])
def test_gemv_w4_does_not_cover(lib, changes):
    refused(lib.nm_gemv_w4, w4(), nm.NM_ERR_UNSUPPORTED, **changes)


def test_gemv_w4_null_and_empty(lib):
    assert lib.nm_gemv_w4(None, Z) == nm.NM_ERR_INVALID_ARG
    d = w4()
    d.M, d.x, d.out = 0, None, None
    assert lib.nm_gemv_w4(C.byref(d), Z) == nm.NM_OK


def test_outputs_that_are_inputs(lib):
    for n, at in (("x", P), ("W", 2 * P), ("scales", 3 * P)):
        refused(lib.nm_gemv_w4, w4(), nm.NM_ERR_INVALID_ARG, out=at)
    refused(attend(lib), paged(), nm.NM_ERR_INVALID_ARG, out=P)
    refused(attend(lib), paged(), nm.NM_ERR_INVALID_ARG, out=P, out_dtype=nm.NM_DT_F32, out_stride=520)


@pytest.mark.parametrize("packed,desc", [(nm._PLAN, nm.PlanDesc), (nm._QK, nm.QkDesc), (nm._PAGED, nm.PagedDesc), (nm._W4, nm.W4Desc)])
def test_packed_descriptions_lie_as_the_structures(packed, desc):
    values = [float(i + 1) if t is C.c_float else i + 1 for i, (_, t) in enumerate(desc._fields_)]
    assert packed.size == C.sizeof(desc)
    d = desc.from_buffer_copy(packed.pack(*values))
    assert [getattr(d, n) for n, _ in desc._fields_] == values


def test_binding_refuses_host_tensors():
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(nm.NmError) as e:
        nm.nm_page_plan(i, i, i, i[:1], i.view(4, 1), page_size=16, num_pages=4, free_end=i[:1], slots=i, status=i)
    assert e.value.status == nm.NM_ERR_INVALID_ARG
    x = torch.zeros((2, 4, 64))
    with pytest.raises(nm.NmError):
        nm.nm_qk_norm_rope(x, x, x, i, None, x)
    with pytest.raises(nm.NmError):
        nm.nm_paged_attention(x, x.view(2, 1, 4, 64), x.view(2, 1, 4, 64), i.view(2, 2), i[:2], x, scale=1.0)


@pytest.mark.parametrize("changes", [dict(out=4 * P)])
def test_gemv_w4_out_is_the_bias(lib, changes):
    refused(lib.nm_gemv_w4, w4(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.mark.parametrize("changes", [*(dict(out=n * P) for n in range(2, 8)), *(dict(lse=n * P) for n in range(1, 9))])
def test_paged_attention_outputs_are_no_inputs(lib, changes):
    """Caches, scales, table and lengths are read while results are written; out may be q, but lse neither of them."""
    refused(attend(lib), paged(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.mark.parametrize("changes", [*(dict(q_out=n * P) for n in (2, 3, 4, 5, 6, 7, 9, 10, 11, 12, 13, 14)), *(dict(k_out=n * P) for n in (1, 3, 4, 5, 6, 7, 10, 11, 12, 13, 14)),
                                     *(dict(k_cache=n * P) for n in (1, 2, 3, 6, 11, 12, 13)), *(dict(v_cache=n * P) for n in (1, 2, 3, 6, 12, 14))])
def test_qk_norm_rope_outputs_are_no_inputs(lib, changes):
    """q_out may be q and k_out k; nothing else that is written may be read, or be written twice."""
    refused(lib.nm_qk_norm_rope, qk(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.fixture
def host_tensors(monkeypatch):
    """Descriptions of tensors in host memory can be made (none is given to a call that would run)."""
    import torch
    nm._here()
    monkeypatch.setattr(nm, "_current", lambda: -1)
    i, x = torch.zeros(8, dtype=torch.int32), torch.zeros((2, 4, 64))
    cache = torch.zeros((3, 16, 4, 64), dtype=torch.bfloat16)
    w = torch.zeros((2, 64), dtype=torch.bfloat16)
    return {
        nm.make_plan_desc: dict(cached=i[:2], fresh=i[:2], free_pages=i, free_begin=i[:1], block_table=i.view(2, 4), page_size=16, num_pages=4, free_end=i[:1],
                                slots=i, status=i[:4]),
        nm.make_qk_desc: dict(q=x, k=x, v=x, positions=i[:2], inv_freq=torch.zeros(32), q_out=x, k_cache=cache, v_cache=cache, slots=i[:2]),
        nm.make_paged_desc: dict(q=x, k_cache=cache, v_cache=cache, block_table=i.view(2, 4), lens=i[:2], out=x, scale=1.0),
        nm.make_w4_desc: dict(x=w, W=torch.zeros((5, 32), dtype=torch.uint8), scales=torch.zeros((5, 2)), out=torch.zeros((2, 5)), group=32)}


def test_calls_refuse_what_is_missing_or_misshapen(host_tensors):
    """A wanted tensor that is None or a number, or one of another rank, is refused as everything else is."""
    calls = {nm.make_plan_desc: nm.nm_page_plan, nm.make_qk_desc: nm.nm_qk_norm_rope, nm.make_paged_desc: nm.nm_paged_attention, nm.make_w4_desc: nm.nm_gemv_w4}
    for make, good in host_tensors.items():
        assert len(make(**good)) > 0
        for name, value in good.items():
            if name in ("inv_freq", "positions", "free_pages") or (make is nm.make_plan_desc and name == "slots"):
                continue                                                      # may be None, or of any length
            for bad in [None, "3"] + ([value[0], value[None], 3] if hasattr(value, "shape") else []):
                if hasattr(bad, "shape") and value.dim() == 1 and bad.numel() == value.numel():
                    continue                                                  # a list of numbers may have any shape
                with pytest.raises(nm.NmError) as e:
                    calls[make](make(**{**good, name: bad}), stream=0)
                assert e.value.status == nm.NM_ERR_INVALID_ARG and str(e.value), (make.__name__, name)


def test_calls_refuse_numbers_that_do_not_fit(host_tensors):
    calls = {nm.make_plan_desc: nm.nm_page_plan, nm.make_qk_desc: nm.nm_qk_norm_rope, nm.make_paged_desc: nm.nm_paged_attention, nm.make_w4_desc: nm.nm_gemv_w4}
    for make, name, value in ((nm.make_plan_desc, "page_size", 1 << 31), (nm.make_plan_desc, "num_pages", 1 << 40), (nm.make_plan_desc, "page_size", 16.5), (nm.make_qk_desc, "eps", 1e300),
                              (nm.make_paged_desc, "window", 1 << 31), (nm.make_paged_desc, "scale", 1e300), (nm.make_w4_desc, "alpha", 1e300), (nm.make_w4_desc, "table_idx", 1 << 31)):
        with pytest.raises(nm.NmError) as e:
            calls[make](make(**{**host_tensors[make], **dict.fromkeys(("norm",) if name == "eps" else (), True), name: value}), stream=0)
        assert e.value.status == nm.NM_ERR_INVALID_ARG, name


def test_calls_refuse_missing_arguments_and_other_calls_descriptions(host_tensors):
    descs = [make(**good) for make, good in host_tensors.items()]
    calls = [nm.nm_page_plan, nm.nm_qk_norm_rope, nm.nm_paged_attention, nm.nm_gemv_w4]
    for i, call in enumerate(calls):
        for bad in [None, 3, b""] + [d for j, d in enumerate(descs) if j != i]:
            with pytest.raises(nm.NmError) as e:
                call(bad, stream=0)
            assert e.value.status == nm.NM_ERR_INVALID_ARG
    with pytest.raises(nm.NmError):
        nm.nm_paged_attention_workspace(descs[0])
    with pytest.raises(nm.NmError):
        nm.nm_paged_attention_workspace()
    assert nm.nm_paged_attention_workspace(descs[2]) >= 0
