"""The integer product in every one of its kernels, to bf16 and to fp32: each shape is listed with the kernel that it runs, which
tests/test_integer_dispatch.py holds to the compiled rule."""
import pytest
import torch

from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_scaled import count

pytestmark = pytest.mark.gpu

CUS = 256
# (kernel, whether the row count is on the device, M, N, K).  few A x B: A fragments of 16 rows and B of 16 columns a workgroup.  Sizes that
# end inside a fragment, a tile and a K-block; 256 x 256 tiles with one, two and three tiles a workgroup; "both" with the count
# that picks the larger tiles at capacity.
LISTED = [
    ("few1x1", False, 11, 64, 144), ("few1x1", True, 16, 4096, 1088), ("few1x2", False, 9, 4624, 1088), ("few1x2", True, 16, 8208, 16),
    ("few2x1", True, 20, 528, 272), ("few2x1", False, 32, 4096, 1040),
    ("few2x2", False, 20, 4624, 1280), ("few2x2", True, 31, 8176, 144), ("few2x2", True, 17, 4608, 1088), ("few2x2", False, 32, 4112, 16),
    ("few4x1", False, 50, 528, 272), ("few4x1", True, 64, 1536, 1088),
    ("few4x2", False, 33, 4624, 272), ("few4x2", True, 64, 4608, 1088), ("few4x2", True, 63, 8176, 144), ("few4x2", False, 48, 4112, 1264),
    ("split32", True, 33, 528, 1552), ("split32", False, 224, 1040, 1408), ("split32x64", False, 250, 1040, 4112), ("split32x64", True, 300, 1552, 1296),
    ("split64", True, 500, 1552, 1808), ("split64", False, 513, 1536, 2064),
    ("64x128", False, 600, 1040, 400), ("64x128", True, 129, 4096, 144), ("alone", True, 1664, 1536, 1104), ("alone", False, 1300, 2064, 400),
    ("128x128", False, 4100, 1040, 272), ("128x128", True, 3000, 1536, 400), ("128x128", True, 8190, 2032, 1040),
    ("256x256", False, 8190, 2032, 1040), ("256x256", False, 8190, 2048, 1168), ("256x256", False, 4606, 6384, 624), ("256x256", False, 12030, 3824, 752),
    ("both", True, 8190, 4080, 1296), ("both", True, 9828, 1536, 6144),
]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


@pytest.mark.parametrize("kernel,counted,M,N,K", LISTED)
@pytest.mark.parametrize("wide", [False, True])
def test_kernel(kernel, counted, M, N, K, wide):
    """Integer operands of few bits, so that the sum times scales of powers of two, and its bias, are exact in fp32 (at most 24 bits from
    2^-12 on): every element's place."""
    gh.say(f"{kernel} {M}x{N}x{K} counted={counted} wide={wide}")
    g = torch.Generator(device="cuda")
    g.manual_seed(M + N + K)
    a, w = (torch.randint(-7, 8, (n, K), generator=g, device="cuda", dtype=torch.int32).to(torch.int8) for n in (M, N))
    sa, sw = (2.0 ** torch.randint(-6, -3, (n,), generator=g, device="cuda").float() for n in (M, N))
    bias = torch.randint(-8, 9, (N,), generator=g, device="cuda").float() / 4
    z = (a.double() @ w.double().t()) * sa.double()[:, None] * sw.double()
    for m in (M, max(M - 3, 0), M // 3) if counted else (None,):
        for b in (None, bias):
            y = torch.full((M, N), 7.0, dtype=torch.float32 if wide else torch.bfloat16, device="cuda")
            fdl.fd_int_linear(a, sa, w, sw, y, bias=b, m=None if m is None else count(m))
            n = M if m is None else m
            assert torch.equal(y[:n], (z[:n] if b is None else z[:n] + b.double()).to(y.dtype)), (m, b is None)
            assert bool((y[n:] == 7).all())
