"""The attention over an 8-bit cache of the least scales: values around bf16's smallest."""
import numpy as np
import pytest
import torch

from oracle import scaled
from paper_2607_12121_amd import flashdiff as fdl
from tests.test_gpu_cache import run_attention
from tests.test_gpu_scaled import UB, bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


@pytest.mark.parametrize("dh", [16, 64, 128])
@pytest.mark.parametrize("rows", [1, 300])
def test_values_of_the_least_scales(rows, dh):
    """Keys of zero average equal values, which are the result but for its rounding (a bf16 one, of multiples of 2^-133) and, where a scale is 1
    or 2, the value's own to such a multiple.  The average of 512 equal values of weight one is exact."""
    tokens = 512
    zeros, ones = np.zeros((tokens, dh), np.uint8), np.full((1, tokens), 127, np.uint8)
    codes = np.tile(np.arange(dh, dtype=np.uint8) % 127 + 128 * (np.arange(dh) % 2).astype(np.uint8), (tokens, 1))
    q = bf16(np.random.default_rng(dh).standard_normal((rows, dh)))
    for byte in (1, 2, 3, 4, 10):
        want = scaled.CODES[codes[0]] * 2.0 ** (byte - 127)
        got = run_attention(q, zeros, ones, codes, np.full((1, tokens), byte, np.uint8), np.array([0, rows], np.int32), np.array([0, tokens], np.int32), 1, 1, dh)
        err = UB * np.abs(want) * (np.abs(want) >= 2.0 ** -126) + (2.0 ** -134 if byte < 3 else 0.0)
        assert np.all(np.abs(got[:, 0] - want) <= err), byte
