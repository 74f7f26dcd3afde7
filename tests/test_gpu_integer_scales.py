"""The integer product where its scales are far apart: the smallest and the largest that integer rows come with, sums of zero, of one and
of many products, in each of its kernels."""
import pytest
import torch

from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_scaled import U32, UB, count

pytestmark = pytest.mark.gpu

LEAST = 2.0 ** -100 / 127                        # of a row whose largest magnitude is 2^-100
ROW_SCALES = (LEAST, 1.3 * 2.0 ** -75, 1.7 * 2.0 ** -20, 1.0, 1.1 * 2.0 ** 60, 3.3895313892515355e38 / 127)
COLUMN_SCALES = (LEAST, 1.7 * 2.0 ** -70, 1.5 / 127, 1.6 * 2.0 ** 66, 1.9 * 2.0 ** 97)


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


# few rows, in one and in two column fragments; tiles of split K-blocks; 64 x 128, 128 x 128 alone and two a CU; 256 x 256
@pytest.mark.parametrize("M,N,K", [(11, 64, 144), (40, 4624, 272), (33, 528, 1552), (250, 1040, 4112), (500, 1552, 1808), (600, 1040, 400), (1664, 1536, 1104),
                                   (4100, 1040, 272), (8190, 2032, 1040)])
@pytest.mark.parametrize("wide", [False, True])
def test_scales_far_apart(M, N, K, wide):
    """y = sum * w_scale * a_scale + bias: the sum's conversion and its product with w_scale are a rounding each, of a normal number
    or of zero whatever the scales; the second product and the bias are one more, of the result.  So neither an infinity nor a loss of bits
    comes from what lies between; only a result past the type's range, or below its normal numbers, is rounded there."""
    gh.say(f"scales {M}x{N}x{K} wide={wide}")
    g = torch.Generator(device="cuda")
    g.manual_seed(M + K)
    a, w = (torch.randint(-127, 128, (n, K), generator=g, device="cuda", dtype=torch.int32).to(torch.int8) for n in (M, N))
    a[::5] = 0                                   # sums of zero
    a[1::5] = 0
    a[1::5, K - 1] = 1                           # sums of one weight
    sa, sw = (torch.tensor([s[i % len(s)] for i in range(n)], device="cuda") for n, s in ((M, ROW_SCALES), (N, COLUMN_SCALES)))
    bias = torch.randint(-8, 9, (N,), generator=g, device="cuda").float() / 4
    p = (a.double() @ w.double().t()) * sw.double() * sa.double()[:, None]
    for b, m in ((bias, None), (None, count(M))):
        y = torch.full((M, N), 7.0, dtype=torch.float32 if wide else torch.bfloat16, device="cuda")
        fdl.fd_int_linear(a, sa, w, sw, y, bias=b, m=m)
        z = p if b is None else p + b.double()
        err = 2.0001 * U32 * p.abs() + U32 * z.abs() + 2.0 ** -149
        last = 2.0 ** 128                        # where rounding to the type may reach the infinity
        if not wide:
            err, last = err + UB * (z.abs() + err) + 2.0 ** -134, 2.0 ** 128 * (1 - 2.0 ** -8)
        past, inside = z.abs() >= 2.0 ** 128 * (1 + 2.0 ** -20), z.abs() <= last * (1 - 2.0 ** -20)
        got = y.double()
        assert bool((got[past] == torch.sign(z[past]) * float("inf")).all())
        assert bool(((got - z).abs() <= err)[inside].all()), (got - z)[inside].abs().max()
        assert bool((got[a.eq(0).all(1)] == (0 if b is None else b.double())).all())
