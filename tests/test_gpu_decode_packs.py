"""nm_paged_attention over int8 caches whose neighbouring key heads may be taken as one: cases that are, by two, four and eight, and cases
where that ends at 64 elements or fewer and must not be (tests/test_paged_choice.py holds which is which)."""
import math

import pytest
import torch

from test_gpu_decode import DEV, assert_rounded, attention_64, paged_case
from paper_2305_14405_amd import binding as nm

# requests, query heads, key heads, elements, window, pages of 32 in the table; key heads that are taken as one
PACK_CASES = [(64, 64, 8, 32, 0, 256, 1), (200, 4, 2, 32, 0, 256, 1), (96, 12, 6, 32, 0, 256, 1), (100, 40, 8, 32, 5000, 256, 1), (130, 8, 4, 16, 0, 256, 1),
              (200, 2, 2, 16, 0, 256, 1), (64, 24, 8, 16, 0, 256, 1), (64, 16, 16, 32, 0, 128, 4), (96, 32, 8, 32, 5000, 256, 4), (64, 16, 16, 16, 0, 128, 8),
              (64, 12, 12, 48, 0, 128, 2), (64, 24, 12, 48, 4100, 256, 2), (64, 64, 8, 64, 0, 256, 2), (64, 6, 6, 64, 0, 256, 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("q_dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,hq,hk,d,window,columns,pack", PACK_CASES)
def test_heads_taken_as_one_or_not(q_dtype, B, hq, hk, d, window, columns, pack):
    lens = [(i * i * 37) % 300 if i % 11 else (0, 1, 127, 4000, 3500)[i // 11 % 5] for i in range(B)]
    lens[5 * (B // 5) - 1], lens[B // 2] = 4096, 129
    lens[7] = 6000 if columns == 256 else 4095                                # beyond the windows
    c = paged_case(B + d, lens, hq, hk, d, q_dtype, torch.int8, page=32, columns=columns)
    c["q"][1, :, 0] *= 100.0
    out = torch.full((B + 2, hq, d), 55.0, dtype=q_dtype, device=DEV)       # two requests' rows in front and behind are nobody's
    lse = torch.full((B + 2, hq), 55.0, device=DEV)
    args = (c["q"], c["cache"][0], c["cache"][1], c["table"], c["lens"], out[1:B + 1])
    more = dict(scale=d ** -0.5, window=window, k_scale=c["scales"][0], v_scale=c["scales"][1], lse=lse[1:B + 1])
    ws = torch.full((nm.nm_paged_attention_workspace(*args, **more),), 0xff, dtype=torch.uint8, device=DEV)
    nm.nm_paged_attention(*args, ws=ws, **more)
    torch.cuda.synchronize()
    for t in (out, lse):
        assert bool((t[0] == 55).all()) and bool((t[-1] == 55).all())
    want, wl, e_out, e_lse = attention_64(c, d ** -0.5, window)
    assert_rounded(out[1:-1], want, e_out, "out")
    got, empty = lse[1:-1].double(), wl == -math.inf
    assert bool((got[empty] == -math.inf).all()) and bool((out[1:-1][empty] == 0).all())
    assert bool(((got - wl)[~empty].abs() <= e_lse[~empty]).all())
