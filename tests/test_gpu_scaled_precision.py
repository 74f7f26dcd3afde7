"""How near the 8-bit products' sums, codes and scale bytes come to the 64-bit ones: in the size of their errors, where
test_gpu_scaled.py holds each value to the bound of the worst operands."""
import numpy as np
import pytest
import torch

from oracle import scaled as ref
from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_scaled import U32, check_codes, linear_case, run_linear

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


def check_same_codes(q, s, want, err, least):
    """check_codes, and each code is the nearest one to `want` wherever +- err leaves no choice (at least the share
    `least` of them)."""
    check_codes(q, s, want, err)
    r, c = want.shape
    lo, hi = (ref.scale_bytes(ref.block_tops(np.maximum(np.abs(want) + e, 0), 1)) for e in (-err, err))
    p = ref.spread(ref.powers(s[:, :lo.shape[1]]), r, c, 1)
    below, above = (ref.encode(np.clip((want + e) / p, -448, 448)) for e in (-err, err))
    sure = ref.spread(lo == hi, r, c, 1) & (below == above)
    assert np.mean(sure) >= least
    np.testing.assert_array_equal(q[sure], below[sure])


SIZES = [(8, 1536, 1536), (200, 1600, 1536), (3000, 1536, 512), (8190, 2032, 512)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_bf16_sums(M, N, K):
    """The sums before their rounding to bf16 are off by 3e-5 of a row's size at most (root mean square), seen in how many
    results are not the nearest value: a sum off by d has another nearest value with a probability of d over the step.  Cutting
    each group of 8 products at 2^-13 of the largest one's leading bit gives 2.1e-5 on these operands (computed in 64 bits);
    fp32's own additions, 2^-24 sqrt(K), a tenth of that.  Five standard deviations of the count on top."""
    gh.say(f"bf16 sums M={M} N={N} K={K}")
    a, sa, w, sw, _ = linear_case(M, N, K, 7)
    y, _ = run_linear(a, sa, w, sw, None, False, "bf16", M, None)
    want = ref.values(a, sa) @ ref.values(w, sw, 128).T
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(want), 1e-30))) - 7)
    most = np.minimum(1, 3e-5 * np.sqrt(np.mean(want * want, 1, keepdims=True)) / step).sum()
    off = np.abs(y.double().numpy() - torch.from_numpy(want).to(torch.bfloat16).double().numpy())
    assert np.count_nonzero(off) <= most + 5 * np.sqrt(most) + 1


@pytest.mark.parametrize("M,N,K", SIZES)
def test_fp32_sums(M, N, K):
    """K additions that round by half a step of the partial sum at most, in all directions: 2^-24 sqrt(K) of a row's size, root
    mean square, and the result's own rounding."""
    gh.say(f"fp32 sums M={M} N={N} K={K}")
    a, sa, w, sw, _ = linear_case(M, N, K, 7)
    y, _ = run_linear(a, sa, w, sw, None, False, "f32", M, None)
    want = ref.values(a, sa) @ ref.values(w, sw, 128).T
    size = np.sqrt(np.mean(want * want, 1))
    off = np.sqrt(np.mean((y.double().numpy() - want) ** 2, 1))
    assert np.max(off / size) <= (np.sqrt(K) + 1) * U32


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("M,N,K", [(700, 1040, 1552), (3000, 1536, 512), (3500, 4112, 2896)])
def test_product_codes_are_the_nearest(M, N, K, gelu):
    """Codes and scale bytes of a product are those of the sums in 64 bits wherever 3e-4 of a row's size (14 times the error
    above) leaves no choice: truncated codes would not be."""
    gh.say(f"product codes M={M} N={N} K={K} gelu={gelu}")
    a, sa, w, sw, _ = linear_case(M, N, K, 8)
    y, ys = run_linear(a, sa, w, sw, None, gelu, "8", M, None)
    z = ref.values(a, sa) @ ref.values(w, sw, 128).T
    err = np.broadcast_to(3e-4 * np.sqrt(np.mean(z * z, 1, keepdims=True)), z.shape)
    want, err = (ref.gelu(z), 1.13 * err + 2.0 ** -21 * np.abs(z)) if gelu else (z, err)
    check_same_codes(y.numpy(), ys, want, err, 0.4 if gelu else 0.9)   # GELU of far negative sums is near no code but zero
