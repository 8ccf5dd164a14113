"""CPU-only checks of the calls for several hypotheses per request: what they refuse, before anything reaches the GPU."""
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
    for n, v in changes.items():
        setattr(desc, n, v)
    rc = call(C.byref(desc))
    assert rc == wanted, (changes, rc, nm.nm_last_error())
    assert nm.nm_last_error() != ""


def fill(desc, names):
    for i, n in enumerate(names):
        setattr(desc, n, P * (i + 1))
    return desc


def with_workspace(call):
    return lambda desc: call(desc, C.c_void_p(P * 100), 1 << 50, Z)


# ---- selection --------------------------------------------------------------------------------------

def beam():
    d = fill(nm.BeamDesc(), ("logits", "scores", "weight", "done", "history", "history_lens", "parents", "tokens", "scores_out", "done_out", "history_out",
                             "history_lens_out"))
    d.R, d.W, d.K, d.V, d.logits_dtype, d.end_token, d.max_history = 3, 4, 5, 1000, nm.NM_DT_BF16, 7, 20
    d.logits_stride, d.history_stride, d.history_out_stride = 1000, 20, 20
    return d


BEAM_IN, BEAM_OUT = ("logits", "scores", "weight", "done", "history", "history_lens"), ("parents", "tokens", "scores_out", "done_out", "history_out", "history_lens_out")


@pytest.mark.parametrize("changes", [
    dict(R=-1), dict(W=0), dict(K=0), dict(V=0), dict(logits_dtype=nm.NM_DT_I8), dict(end_token=-2), dict(end_token=1000), dict(end_token=-1), dict(logits_stride=999),
    dict(max_history=0), dict(history_stride=19), dict(history_out_stride=19), dict(logits=None), dict(scores=None), dict(parents=None), dict(tokens=None),
    dict(scores_out=None), dict(history_lens=None), dict(history_out=None), dict(history_lens_out=None), dict(history=None)]
    + [{o: P * (i + 1)} for o in BEAM_OUT for i in range(6)] + [{o: P * (7 + i)} for j, o in enumerate(BEAM_OUT) for i in range(6) if i != j])
def test_beam_select_refuses(lib, changes):
    refused(with_workspace(lib.nm_beam_select), beam(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.mark.parametrize("changes", [dict(W=65), dict(K=65), dict(R=1 << 19), dict(R=(1 << 17) + 1, K=64, W=1), dict(max_history=(1 << 30) + 1, history_stride=1 << 31, history_out_stride=1 << 31),
                                     dict(V=(1 << 26) + 1, logits_stride=1 << 27), dict(logits=P + 1)])
def test_beam_select_does_not_cover(lib, changes):
    refused(with_workspace(lib.nm_beam_select), beam(), nm.NM_ERR_UNSUPPORTED, **changes)


def workspace_checks(lib, name, d):
    n = C.c_size_t()
    ask, call = getattr(lib, name + "_workspace"), getattr(lib, name)
    assert ask(None, C.byref(n)) == nm.NM_ERR_INVALID_ARG and call(None, None, 0, Z) == nm.NM_ERR_INVALID_ARG
    assert ask(C.byref(d), None) == nm.NM_ERR_INVALID_ARG
    assert ask(C.byref(d), C.byref(n)) == nm.NM_OK and n.value > 0
    for ws, size in ((None, n.value), (P, n.value - 1), (P + 128, n.value)):
        assert call(C.byref(d), C.c_void_p(ws), size, Z) == nm.NM_ERR_WORKSPACE
        assert "workspace" in nm.nm_last_error()


def test_beam_select_workspace_null_and_empty(lib):
    d = beam()
    workspace_checks(lib, "nm_beam_select", d)
    d.R = 0
    for n in BEAM_IN + BEAM_OUT:
        setattr(d, n, None)
    d.end_token = -1
    assert lib.nm_beam_select(C.byref(d), None, 0, Z) == nm.NM_OK


# ---- fork -----------------------------------------------------------------------------------------------

FORK_IN, FORK_OUT = ("block_table", "lens", "parents", "keep", "free_begin", "free_pages"), ("table_out", "lens_out", "free_end", "copy_src", "copy_dst", "copy_slots", "status", "free_out")


def fork():
    d = fill(nm.ForkDesc(), FORK_IN + FORK_OUT)
    d.B_in, d.B_out, d.page_size, d.num_pages, d.max_pages, d.n_free, d.table_stride, d.table_out_stride = 3, 4, 16, 100, 9, 100, 9, 10
    return d


@pytest.mark.parametrize("changes", [
    dict(B_in=-1), dict(B_out=-1), dict(num_pages=-1), dict(max_pages=-1), dict(n_free=-1), dict(table_stride=8), dict(table_out_stride=8)]
    + [{n: None} for n in FORK_IN + FORK_OUT if n != "keep"]
    + [{o: P * (i + 1)} for o in FORK_OUT for i, n in enumerate(FORK_IN) if (o, n) != ("free_out", "free_pages")]
    + [{o: P * (7 + i)} for j, o in enumerate(FORK_OUT) for i in range(8) if i != j])
def test_page_fork_refuses(lib, changes):
    refused(with_workspace(lib.nm_page_fork), fork(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.mark.parametrize("changes", [dict(B_in=nm.NM_PLAN_MAX_REQUESTS + 1), dict(B_out=nm.NM_PLAN_MAX_REQUESTS + 1), dict(page_size=0), dict(page_size=24), dict(page_size=1 << 17),
                                     dict(num_pages=1 << 27), dict(max_pages=1 << 27, table_stride=1 << 27, table_out_stride=1 << 27), dict(n_free=(1 << 30) + 1),
                                     dict(num_pages=(1 << 30) + 1, page_size=1), dict(max_pages=(1 << 30) + 1, page_size=1, table_stride=1 << 31, table_out_stride=1 << 31)])
def test_page_fork_does_not_cover(lib, changes):
    refused(with_workspace(lib.nm_page_fork), fork(), nm.NM_ERR_UNSUPPORTED, **changes)


def test_page_fork_workspace_and_null(lib):
    workspace_checks(lib, "nm_page_fork", fork())


# ---- copy -----------------------------------------------------------------------------------------------

def copy(caches=(P * 4, P * 5)):
    d = fill(nm.CopyDesc(), ("src", "dst", "slots"))
    d.keep = (C.c_void_p * len(caches))(*caches)
    d.caches = C.addressof(d.keep)
    d.n, d.n_caches, d.hk, d.d, d.dtype, d.num_pages, d.page_size = 3, len(caches), 2, 64, nm.NM_DT_BF16, 10, 16
    d.page_stride, d.slot_stride, d.head_stride = 2048, 128, 64
    return d


def do_copy(lib):
    return lambda desc: lib.nm_page_copy(desc, Z)


@pytest.mark.parametrize("changes", [dict(n=-1), dict(n_caches=-1), dict(hk=0), dict(d=0), dict(num_pages=-1), dict(dtype=nm.NM_DT_I32), dict(page_stride=-1),
                                     dict(slot_stride=-1), dict(head_stride=-1), dict(caches=None), dict(src=None), dict(dst=None)])
def test_page_copy_refuses(lib, changes):
    refused(do_copy(lib), copy(), nm.NM_ERR_INVALID_ARG, **changes)


@pytest.mark.parametrize("caches", [(P * 4, None), (P,), (P * 4, P * 2), (P * 3,)])
def test_page_copy_refuses_caches(lib, caches):
    refused(do_copy(lib), copy(caches), nm.NM_ERR_INVALID_ARG)


@pytest.mark.parametrize("changes", [dict(n=(1 << 20) + 1), dict(n_caches=nm.NM_COPY_MAX_CACHES + 1), dict(page_size=12), dict(num_pages=1 << 27),
                                     dict(hk=1 << 14, d=1 << 14), dict(n=1 << 20, hk=1 << 12, d=1 << 14), dict(n=1 << 20, hk=128, d=128)])
def test_page_copy_does_not_cover(lib, changes):
    refused(do_copy(lib), copy(), nm.NM_ERR_UNSUPPORTED, **changes)


def test_page_copy_misaligned_null_and_empty(lib):
    refused(do_copy(lib), copy((P * 4 + 1,)), nm.NM_ERR_UNSUPPORTED)
    assert lib.nm_page_copy(None, Z) == nm.NM_ERR_INVALID_ARG
    for n in ("n", "n_caches", "num_pages"):
        d = copy()
        setattr(d, n, 0)
        d.src = d.dst = d.caches = None
        assert lib.nm_page_copy(C.byref(d), Z) == nm.NM_OK  # nothing to do


# ---- attention over shared prefixes -------------------------------------------------------------------

def shared():
    d = nm.SharedDesc()
    d.p.B, d.p.hq, d.p.hk, d.p.d, d.p.q_dtype, d.p.cache_dtype, d.p.out_dtype = 3, 8, 2, 64, nm.NM_DT_F32, nm.NM_DT_I8, nm.NM_DT_BF16
    d.p.page_size, d.p.num_pages, d.p.max_pages, d.p.q_stride, d.p.out_stride, d.p.table_stride = 16, 100, 80, 512, 512, 80
    fill(d.p, ("q", "k_cache", "v_cache", "k_scale", "v_scale", "block_table", "lens", "out", "lse"))
    d.p.page_stride, d.p.slot_stride, d.p.head_stride, d.p.scale, d.p.out_inv_scale = 2048, 128, 64, 0.125, 1.0
    d.G, d.group_start, d.shared = 2, P * 20, P * 21
    return d


def attend(lib, desc):
    return lib.nm_shared_attention(C.byref(desc), C.c_void_p(P * 100), 1 << 50, Z)


@pytest.mark.parametrize("changes", [
    dict(B=-1), dict(hq=0), dict(hk=0), dict(hq=9), dict(d=0), dict(max_pages=-1), dict(num_pages=-1), dict(window=-1), dict(q_dtype=nm.NM_DT_I8),
    dict(cache_dtype=nm.NM_DT_F32), dict(out_dtype=nm.NM_DT_I32), dict(q_stride=511), dict(out_stride=511), dict(table_stride=79), dict(page_stride=-16),
    dict(slot_stride=-16), dict(head_stride=-16), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(lens=None), dict(out=None),
    dict(block_table=None), dict(k_cache=None), dict(v_cache=None), dict(k_scale=None), dict(v_scale=None), dict(G=-1), dict(group_start=None), dict(shared=None),
    *(dict(out=n * P) for n in (1, 2, 3, 4, 5, 6, 7, 20, 21)), *(dict(lse=n * P) for n in (1, 2, 3, 4, 5, 6, 7, 8, 20, 21))])
def test_shared_attention_refuses(lib, changes):
    d = shared()
    for n, v in changes.items():
        setattr(d if n in ("G", "group_start", "shared") else d.p, n, v)
    assert attend(lib, d) == nm.NM_ERR_INVALID_ARG and "nm_shared_attention" in nm.nm_last_error()


@pytest.mark.parametrize("changes", [
    dict(d=72), dict(d=272, q_stride=4000, out_stride=4000), dict(page_size=3), dict(num_pages=1 << 27), dict(max_pages=1 << 26, table_stride=1 << 26),
    dict(k_cache=P + 8), dict(v_cache=P + 4), dict(page_stride=2056), dict(slot_stride=136), dict(head_stride=72), dict(num_pages=1 << 20, page_stride=1 << 15),
    dict(window=5), dict(B=nm.NM_PLAN_MAX_REQUESTS + 1), dict(G=nm.NM_PLAN_MAX_REQUESTS + 1)])
def test_shared_attention_does_not_cover(lib, changes):
    d = shared()
    for n, v in changes.items():
        setattr(d if n == "G" else d.p, n, v)
    assert attend(lib, d) == nm.NM_ERR_UNSUPPORTED and "nm_shared_attention" in nm.nm_last_error()


def test_shared_attention_workspace_null_and_empty(lib):
    workspace_checks(lib, "nm_shared_attention", shared())
    d, n = shared(), C.c_size_t()
    d.p.max_pages = d.p.table_stride = 20                                     # rows that are not divided need none
    assert lib.nm_shared_attention_workspace(C.byref(d), C.byref(n)) == nm.NM_OK and n.value == 0
    d.p.B, d.p.q, d.p.out, d.p.lens, d.group_start = 0, None, None, None, None
    assert lib.nm_shared_attention(C.byref(d), None, 0, Z) == nm.NM_OK


# ---- binding ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("packed,desc", [(nm._BEAM, nm.BeamDesc), (nm._FORK, nm.ForkDesc), (nm._COPY, nm.CopyDesc)])
def test_packed_descriptions_lie_as_the_structures(packed, desc):
    values = [float(i + 1) if t is C.c_float else i + 1 for i, (_, t) in enumerate(desc._fields_)]
    assert packed.size == C.sizeof(desc)
    d = desc.from_buffer_copy(packed.pack(*values))
    assert [getattr(d, n) for n, _ in desc._fields_] == values


def test_packed_description_of_shared_attention_lies_as_the_structure():
    values = [float(i + 1) if t is C.c_float else i + 1 for i, (_, t) in enumerate(nm.PagedDesc._fields_)]
    d = nm.SharedDesc.from_buffer_copy(nm._PAGED.pack(*values) + nm._GROUPS.pack(901, 902, 903))
    assert nm._SHARED.size == C.sizeof(d) and (d.G, d.group_start, d.shared) == (901, 902, 903)
    assert [getattr(d.p, n) for n, _ in nm.PagedDesc._fields_] == values


@pytest.fixture
def host_tensors(monkeypatch):
    """Descriptions of tensors in host memory can be made (none is given to a call that would run)."""
    import torch
    nm._here()
    monkeypatch.setattr(nm, "_current", lambda: -1)
    i = torch.zeros(8, dtype=torch.int32)
    o = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    return {
        nm.make_beam_desc: dict(logits=torch.zeros((6, 50)), scores=torch.zeros((2, 3)), parents=o(2, 4), tokens=o(2, 4), scores_out=torch.zeros((2, 4)), done=o(2, 3),
                                end_token=3, done_out=o(2, 4), history=o(6, 9), history_lens=o(6), history_out=o(8, 9), history_lens_out=o(8)),
        nm.make_fork_desc: dict(block_table=o(2, 4), lens=i[:2], parents=i[:3], free_pages=o(9), free_begin=i[:1], table_out=o(3, 4), page_size=16, num_pages=9, lens_out=o(3),
                                free_out=o(9), free_end=o(1), copy_src=o(3), copy_dst=o(3), copy_slots=o(3), status=o(4)),
        nm.make_shared_desc: dict(q=torch.zeros((2, 4, 64)), k_cache=torch.zeros((3, 16, 4, 64), dtype=torch.bfloat16), v_cache=torch.zeros((3, 16, 4, 64), dtype=torch.bfloat16),
                                  block_table=o(2, 4), lens=i[:2], group_start=i[:2], shared=i[:1], out=torch.zeros((2, 4, 64)), scale=1.0),
        nm.make_copy_desc: dict(caches=torch.zeros((2, 5, 16, 2, 64)), src=o(3), dst=o(3), slots=o(3))}


CALLS = {nm.make_beam_desc: nm.nm_beam_select, nm.make_fork_desc: nm.nm_page_fork, nm.make_copy_desc: nm.nm_page_copy, nm.make_shared_desc: nm.nm_shared_attention}
MAY_BE_NONE = ("done", "done_out", "slots", "keep")
ANY_LENGTH = ("src",)


def test_calls_refuse_what_is_missing_or_misshapen(host_tensors):
    """A wanted tensor that is None or a number, or one of another rank or type, is refused as everything else is."""
    import torch
    for make, good in host_tensors.items():
        assert len(make(**good)) > 0
        for name, value in good.items():
            bad = ["3"] if name in MAY_BE_NONE else [None, "3"]
            if hasattr(value, "shape"):
                bad += [3] if name in ("q", "out") else [3, value.double()]
                bad += [value[0]] if value.dim() > 1 or (value.numel() > 1 and name not in ANY_LENGTH) else []
                bad += [value[None]] if value.dim() > 1 and name not in ("parents", "tokens", "scores_out", "done", "scores") else []
            for b in bad:
                if make is nm.make_copy_desc and name == "caches" and isinstance(b, torch.Tensor) and b.dtype == torch.float64 and b.dim() != 5:
                    continue
                with pytest.raises(nm.NmError) as e:
                    CALLS[make](make(**{**good, name: b}), stream=0)
                assert e.value.status == nm.NM_ERR_INVALID_ARG and str(e.value), (make.__name__, name, b)


def test_calls_refuse_numbers_that_do_not_fit(host_tensors):
    for make, name, value in ((nm.make_beam_desc, "end_token", 1 << 31), (nm.make_fork_desc, "page_size", 1 << 31), (nm.make_fork_desc, "num_pages", 16.5),
                              (nm.make_fork_desc, "num_pages", 1 << 40)):
        with pytest.raises(nm.NmError) as e:
            make(**{**host_tensors[make], name: value})
        assert e.value.status == nm.NM_ERR_INVALID_ARG, name


def test_calls_refuse_missing_arguments_and_other_calls_descriptions(host_tensors):
    descs = {make: make(**good) for make, good in host_tensors.items()}
    for make, call in CALLS.items():
        for bad in [None, 3, b""] + [d for m, d in descs.items() if m is not make]:
            with pytest.raises(nm.NmError) as e:
                call(bad, stream=0)
            assert e.value.status == nm.NM_ERR_INVALID_ARG
    for ask, good, bad in ((nm.nm_beam_select_workspace, nm.make_beam_desc, nm.make_fork_desc), (nm.nm_page_fork_workspace, nm.make_fork_desc, nm.make_copy_desc),
                           (nm.nm_shared_attention_workspace, nm.make_shared_desc, nm.make_copy_desc)):
        assert ask(descs[good]) >= 0
        with pytest.raises(nm.NmError):
            ask(descs[bad])
        with pytest.raises(nm.NmError):
            ask()


def test_copies_of_a_list_of_caches_and_of_one_tensor_are_described_alike(host_tensors):
    import torch
    x, i = torch.zeros((3, 5, 16, 2, 64), dtype=torch.float16).transpose(2, 3).contiguous().transpose(2, 3), torch.zeros(4, dtype=torch.int32)
    a, b = (nm.CopyDesc.from_buffer_copy(nm.make_copy_desc(c, i, i)) for c in (x, list(x)))
    for d, keep in ((a, nm.make_copy_desc(x, i, i)), (b, nm.make_copy_desc(list(x), i, i))):
        assert list(keep.addresses) == [t.data_ptr() for t in x]
        assert (d.n, d.n_caches, d.hk, d.d, d.num_pages, d.page_size) == (4, 3, 2, 64, 5, 16)
        assert (d.page_stride, d.slot_stride, d.head_stride) == x.stride()[1:4]
    for bad in ([], [x[0], x[1].float()], [x[0], x[1][:4]], [x[0], x[1].contiguous()], x[0], x[..., ::2]):
        with pytest.raises(nm.NmError):
            nm.make_copy_desc(bad, i, i)


def test_beam_select_refuses_hypotheses_numbers_of_another_shape(host_tensors):
    """done and weight are [R, W], as scores are: their transposes, which have as many elements, and their elements in a row are refused."""
    import torch
    good = {**host_tensors[nm.make_beam_desc], "weight": torch.ones((2, 3))}
    assert len(nm.make_beam_desc(**good)) > 0
    for name in ("done", "weight"):
        for bad in (good[name].t().contiguous(), good[name].view(-1), good[name][None], good[name][:, :2].contiguous()):
            with pytest.raises(nm.NmError) as e:
                nm.make_beam_desc(**{**good, name: bad})
            assert e.value.status == nm.NM_ERR_INVALID_ARG and name in str(e.value)
    for name, fits in (("history_lens", (2, 3)), ("history_lens_out", (2, 4))):
        assert len(nm.make_beam_desc(**{**good, name: good[name].view(fits)})) > 0
        with pytest.raises(nm.NmError) as e:
            nm.make_beam_desc(**{**good, name: good[name].view(fits[::-1])})
        assert e.value.status == nm.NM_ERR_INVALID_ARG and name in str(e.value)
