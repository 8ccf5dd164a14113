"""nm_gemv_w4 where the values of x differ much in size: errors against what the weights let through, not against x alone."""
import pytest
import torch

from test_gpu_decode import DEV, U, assert_rounded, w4_case
from paper_2305_14405_amd import binding as nm

pytestmark = pytest.mark.gpu


def product_of_weights(c):
    """(result, bound) in binary64.  A product of a 16-bit number and a weight is exact in binary32; within 128 weights four matrix instructions add, each
    a tree of five levels and the accumulator: 24 roundings, 48 where they truncate; then K / 1024 + 8 additions at most, and the scale, alpha and the
    bias 5 roundings more.  All on the sum of |x w| s: a weight of zero lets nothing through."""
    s = c["scales"].double().repeat_interleave(c["group"], 1)
    w, x, a = c["w"].double() * s, c["x"].double(), c["alpha"]
    y = x @ w.t().contiguous() * a + c["bias"].double()
    return y, (48 + x.shape[1] / 1024 + 13) * U * (x.abs() @ w.abs().t().contiguous()) * abs(a) + 2 * U * (y.abs() + c["bias"].double().abs())


def packed(w):
    return ((w[:, 0::2] & 15) | ((w[:, 1::2] & 15) << 4)).to(torch.uint8)


def call(c, out_dtype=torch.float32):
    out = torch.empty((c["x"].shape[0], c["W"].shape[0]), dtype=out_dtype, device=DEV)
    nm.nm_gemv_w4(c["x"], c["W"], c["scales"], out, group=c["group"], alpha=c["alpha"], bias=c["bias"])
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(1, 40, 512), (3, 16, 11008), (16, 4200, 640), (17, 50, 1152), (33, 4100, 384), (50, 8200, 256)])
def test_large_values_that_meet_zero_weights(x_dtype, group, M, N, K):
    """One value in 100 is some 30000 times the others, and most of its weights are zero, as are all weights of some columns."""
    c = w4_case(M + N, M, N, K, group, x_dtype, torch.float32)
    large = torch.arange(7, K, 100, device=DEV)
    c["x"] = (c["x"] * 0.01).to(x_dtype).contiguous()
    c["x"][:, large] = (c["x"][:, large].float() * 30000).to(x_dtype)
    c["w"][: N // 2, large] = 0
    c["w"][1] = 0
    c["W"] = packed(c["w"].cpu()).to(DEV)
    c["bias"] = c["bias"] * 0
    want, error = product_of_weights(c)
    assert_rounded(call(c), want, error, "product")


@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K,group", [(1, 33, 4096, 128), (20, 100, 2304, 64), (48, 70, 1024, 32)])
def test_values_of_one_sign(x_dtype, M, N, K, group):
    c = w4_case(M, M, N, K, group, x_dtype, torch.float32)
    c["x"] = c["x"].abs()
    want, error = product_of_weights(c)
    assert_rounded(call(c), want, error, "product")


@pytest.mark.parametrize("M", [1, 17])
def test_values_near_the_types_end(M):
    """2^126 times any weight and a small scale is finite, and exact."""
    c = w4_case(4, M, 48, 256, 64, torch.bfloat16, torch.float32)
    c["x"].zero_()
    c["x"][:, 37], c["alpha"], c["bias"] = 2.0 ** 126, 1.0, c["bias"] * 0
    c["scales"].fill_(2.0 ** -10)
    assert torch.equal(call(c).double(), (2.0 ** 116 * c["w"][:, 37].double()).expand(M, -1))


@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M", [1, 20, 40])
def test_infinities_follow_the_formula(x_dtype, M):
    """An infinity comes out as one where its weight is not zero, with its sign, and as NaN where it is; a NaN is a NaN everywhere."""
    c = w4_case(6, M, 130, 256, 64, x_dtype, torch.float32)
    row, clean = M // 2, call(c)
    c["x"][row, 100] = -float("inf")
    got, w = call(c), c["w"][:, 100].double()
    assert torch.equal(got[row].double().nan_to_num(nan=5.0), torch.where(w == 0, 5.0, -w.sign() * float("inf")).nan_to_num(nan=5.0))
    c["x"][row, 100] = float("nan")
    got = call(c)
    rest = torch.arange(M, device=DEV) != row
    assert bool(got[row].isnan().all()) and torch.equal(got[rest], clean[rest])
