"""Which kernel an integer product runs, by the rule that the launch goes by: each shape of the GPU tests lands in the kernel that it is
listed for, and each kernel has shapes."""
import ctypes
import subprocess

import numpy as np
import pytest

from paper_2607_12121_amd import build
from tests.test_gpu_integer_kernels import CUS, LISTED

TILES = ["split32", "split32x64", "split64", "64x128", "alone", "128x128", "256x256", "both"]


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "r.cpp").write_text("""#include "fd_int_rules.h"
extern "C" int kernel(int M, int N, int K, int wide, int counted, int cus) { return fd::int_kernel(M, N, K, wide, counted, cus); }
extern "C" int large(int M, int N, int K, int wide, int cus) { return fd::int_large(M, N, K, wide, cus); }
extern "C" int frags(int M) { return fd::scaled_few_frags(M); }
extern "C" int two(int N, int cus) { return fd::scaled_few_wide(N, cus); }
""")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{build.CSRC}", str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    return ctypes.CDLL(str(d / "r.so"))


def kernel(rules, M, N, K, wide, counted):
    n = rules.kernel(M, N, K, wide, counted, CUS)
    return f"few{rules.frags(M)}x{1 + rules.two(N, CUS)}" if n == 0 else TILES[n - 1]


@pytest.mark.parametrize("wide", [0, 1])
def test_listed_shapes_run_their_kernels(rules, wide):
    for name, counted, M, N, K in LISTED:
        assert kernel(rules, M, N, K, wide, int(counted)) == name, (M, N, K)
        if name == "both":          # the count at capacity picks the large tiles, a third of it the small ones
            assert rules.large(M, N, K, wide, CUS) and not rules.large(M // 3, N, K, wide, CUS)
    assert {name for name, *_ in LISTED} == {f"few{a}x{b}" for a in (1, 2, 4) for b in (1, 2)} | set(TILES)
    tiles = [-(-M // 256) * -(-N // 256) for name, _, M, N, _ in LISTED if name == "256x256"]
    assert min(tiles) <= CUS and any(CUS < t <= 2 * CUS for t in tiles) and any(t > 2 * CUS for t in tiles)


def test_kernels_of_drawn_sizes(rules):
    """Two kernels are launched only where the count is on the device, and the 256 x 256 tiles by themselves only where it is not; few
    rows are few either way."""
    rng = np.random.default_rng(1)
    for M, N, K in zip(*(np.exp(rng.uniform(0, np.log(t), 3000)).astype(int) for t in (40000, 600, 600))):
        M, N, K = int(M), 16 * int(N), 16 * int(K)
        for wide in (0, 1):
            assert kernel(rules, M, N, K, wide, 0) != "both" and kernel(rules, M, N, K, wide, 1) != "256x256"
            assert kernel(rules, M, N, K, wide, 0).startswith("few") == kernel(rules, M, N, K, wide, 1).startswith("few")
