"""CPU tests of the 8-bit entry points: refusals before any launch, the scale stride, and the 64-bit
reference against torch's e4m3 conversion."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import scaled as ref
from paper_2607_12121_amd import build
from paper_2607_12121_amd import flashdiff as fdl
from tests.test_abi import no_gpu
from tests.test_isa_hazards import _hazards

P = 0x1000


def test_reference_codes_equal_torch():
    """Every e4m3 byte decodes as torch's, and a dense set of values, ties among them, rounds as torch's."""
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ref.CODES, t)
    fine = ref.CODES[np.isfinite(ref.CODES)]
    mids = (np.sort(fine)[1:] + np.sort(fine)[:-1]) / 2
    v = np.concatenate([fine, mids, mids * (1 + 1e-6), mids * (1 - 1e-6), np.linspace(-448, 448, 4001)]).astype(np.float32)
    got = ref.encode(v)
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("top,power", [(448.0, 0), (449.0, 1), (224.0, -1), (224.5, 0), (1.75, -8), (1.76, -7), (0.0, -126),
                                       (2.0 ** -140, -126), (3.0e38, 120), (np.inf, 128), (np.nan, 128)])
def test_reference_scale(top, power):
    assert ref.scale_bytes(np.array([top]))[0] == power + 127


def test_reference_rope_is_a_rotation():
    """Norms of pairs are kept, and equal shifts of q's and k's position leave their product."""
    rng = np.random.default_rng(0)
    x, z = rng.standard_normal((2, 5, 3, 64))
    pos = rng.integers(0, 1000, (5, 2))
    for halves in (False, True):
        kw = dict(dims=[24, 30], theta=[1e4, 100.0], step=[1.0, 0.5], halves=halves)
        r = ref.rope(x, pos, **kw)
        np.testing.assert_allclose(np.sum(r * r, -1), np.sum(x * x, -1), rtol=1e-12)
        np.testing.assert_array_equal(r[..., 54:], x[..., 54:])
        s = np.sum(r * ref.rope(z, pos + 7, **kw), -1)
        np.testing.assert_allclose(s, np.sum(ref.rope(x, pos + 40, **kw) * ref.rope(z, pos + 47, **kw), -1), rtol=0, atol=1e-10)


def test_scale_stride():
    for cols in (-1, 0, 1, 16, 128, 129, 512, 513, 1536, 6144):
        assert fdl.fd_scale_stride(cols) == (ref.stride(cols) if cols > 0 else 0)


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(rows=0), 1), (dict(cols=0), 1), (dict(cols=24), 3), (dict(block=64), 1), (dict(x=None), 1), (dict(q=None), 1),
    (dict(scale=None), 1), (dict(x=P + 8), 1), (dict(q=P + 4), 1), (dict(block=128, m=P), 1)])
def test_quant_blocks_refuses(change, status):
    a = dict(rows=4, cols=64, block=1, x=P, m=P, q=P, scale=P)
    a.update(change)
    st = fdl.lib().fd_quant_blocks(a["rows"], a["cols"], a["block"], a["x"], a["m"], a["q"], a["scale"], None)
    assert st == status, fdl.lib().fd_last_error()


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(rows=0), 1), (dict(D=72), 3), (dict(D=12304), 3), (dict(B=0), 1), (dict(h=None), 1), (dict(m=None), 1), (dict(q=None), 1),
    (dict(q_scale=None), 1), (dict(B=2, cu_q=None), 1), (dict(y=None, q=None, q_scale=None), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
    (dict(stride=-4), 1), (dict(stride=6), 1), (dict(h=P + 4), 1), (dict(y=P + 8), 1), (dict(gate=P + 4), 1), (dict(weight=P + 4), 1),
    (dict(shift=P + 4), 1), (dict(scale=P + 4), 1), (dict(q=P + 8), 1)])
def test_rms_quant_refuses(change, status):
    a = dict(rows=4, D=64, B=1, h=P, y=P, gate=P, weight=P, shift=P, scale=P, stride=192, eps=1e-6, cu_q=P, m=P, q=P, q_scale=P)
    a.update(change)
    assert fdl.lib().fd_rms_quant(*a.values(), None) == status, fdl.lib().fd_last_error()


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(rows=0), 1), (dict(rows=9), 1), (dict(rope=None), 1), (dict(hq=0), 1), (dict(hk=0), 1), (dict(hq=5000), 3), (dict(dh=32), 3),
    (dict(coord=None), 1), (dict(qkv=None), 1), (dict(m=None), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1),
    (dict(qkv=P + 8), 1), (dict(q=P + 8), 1), (dict(k=P + 8), 1), (dict(v=P + 8), 1)])
def test_rope_axes_refuses(change, status):
    a = dict(rows=4, tokens=8, rope=ctypes.byref(fdl.rope_axes([64])), hq=2, hk=1, dh=64, coord=P, qkv=P, idx=P, m=P, q=P, k=P, v=P)
    a.update(change)
    assert fdl.lib().fd_rope_axes(*a.values(), None) == status, fdl.lib().fd_last_error()


@no_gpu
@pytest.mark.parametrize("field,value", [("n_axes", 0), ("n_axes", 5), ("pairing", 2), ("dim", (3, 0, 0, 0)), ("dim", (0, 0, 0, 0)),
                                         ("dim", (66, 0, 0, 0)), ("dim", (-2, 0, 0, 0)), ("theta", (0.0,) * 4), ("theta", (float("nan"),) * 4),
                                         ("theta", (float("inf"),) * 4), ("step", (float("inf"),) * 4)])
def test_rope_descriptor_refused(field, value):
    r = fdl.rope_axes([64])
    if isinstance(value, tuple):
        for i, v in enumerate(value):
            getattr(r, field)[i] = v
    else:
        setattr(r, field, value)
    assert fdl.lib().fd_rope_axes(4, 8, ctypes.byref(r), 2, 1, 64, *([P] * 7), None) == 1
    two = fdl.rope_axes([40, 26])   # together more than the head
    assert fdl.lib().fd_rope_axes(4, 8, ctypes.byref(two), 2, 1, 64, *([P] * 7), None) == 1


@no_gpu
def test_sizes_beyond_32_bits_refused():
    """Rows whose numbers would pass 32 bits, and angles with no fraction left."""
    lib, n = fdl.lib(), (1 << 30) + 1
    assert lib.fd_quant_blocks(n, 64, 1, P, P, P, P, None) == 3
    assert lib.fd_rms_quant(n, 64, 1, P, None, None, None, None, None, 0, 1e-6, None, P, P, P, None) == 3
    assert lib.fd_rope_axes(n, n, ctypes.byref(fdl.rope_axes([64])), 2, 1, 64, *([P] * 7), None) == 3
    assert lib.fd_scaled_linear(n, 64, 64, P, P, P, P, None, 0, P, P, None, None, None, None) == 3
    for kw in (dict(step=7e6), dict(step=-7e6), dict(step=1e300, theta=1e-300), dict(theta=1e-8)):
        assert lib.fd_rope_axes(4, 8, ctypes.byref(fdl.rope_axes([64], **kw)), 2, 1, 64, *([P] * 7), None) == 1, kw


def test_bindings_refuse_wide_shapes():
    """Shapes whose sizes a 32-bit argument would cut; expanded, so that they hold one element."""
    one = torch.zeros(1, 1, dtype=torch.float8_e4m3fn)
    big, s = one.expand((1 << 32) + 4, 16), torch.zeros(4, 4, dtype=torch.uint8)
    i, h = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1)
    for call in (lambda: fdl.fd_quant_blocks(big, 1, big, s), lambda: fdl.fd_rms_quant(h.expand((1 << 32) + 4, 16), None, None, None, i),
                 lambda: fdl.fd_rope_axes(big, i.view(1, 1), None, i, h, h, h, 1, 1, 16, dims=[16]),
                 lambda: fdl.fd_scaled_linear(big, s, one, s, h)):
        with pytest.raises(fdl.FlashDiffError, match="at most 2"):
            call()


def test_rope_binding_refuses():
    for kw in (dict(dims=[]), dict(dims=[2] * 5), dict(dims=[8, 8], theta=[1e4]), dict(dims=[8], step=[1.0, 2.0])):
        with pytest.raises(fdl.FlashDiffError):
            fdl.rope_axes(**kw)


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(rows=0), 1), (dict(n=0), 1), (dict(k=0), 1), (dict(n=40), 3), (dict(k=72), 3), (dict(a=None), 1), (dict(sa=None), 1), (dict(w=None), 1),
    (dict(sw=None), 1), (dict(yb=None), 1), (dict(yf=P), 1), (dict(yq=P, ys=P), 1), (dict(ys=P), 1), (dict(yb=None, yq=P), 1),
    (dict(gelu=2), 1), (dict(a=P + 8), 1), (dict(w=P + 8), 1), (dict(sa=P + 2), 1), (dict(sw=P + 2), 1), (dict(bias=P + 4), 1), (dict(yb=P + 8), 1),
    (dict(yb=None, yf=P + 8), 1), (dict(yb=None, yq=P + 8, ys=P), 1), (dict(n=1 << 17, k=1 << 14), 3)])
def test_scaled_linear_refuses(change, status):
    a = dict(rows=4, n=64, k=64, a=P, sa=P, w=P, sw=P, bias=P, gelu=0, m=P, yb=P, yf=None, yq=None, ys=None)
    a.update(change)
    assert fdl.lib().fd_scaled_linear(*a.values(), None) == status, fdl.lib().fd_last_error()


def test_bindings_refuse_host_tensors():
    x, q = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.float8_e4m3fn)
    s, h = torch.zeros(4, 4, dtype=torch.uint8), torch.zeros(4, 64)
    i = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: fdl.fd_quant_blocks(x, 1, q, s), lambda: fdl.fd_rms_quant(h, q, s, i, i),
                 lambda: fdl.fd_rope_axes(x, i.view(1, 2), None, i, x, x, x, 1, 1, 16, dims=[8, 8]),
                 lambda: fdl.fd_scaled_linear(q, s, q, s, h)):
        with pytest.raises(fdl.FlashDiffError):
            call()


def test_product_rules(tmp_path):
    """The kernels of measured shapes, and that a call which launches both tile kernels can meet either row count."""
    src = tmp_path / "r.cpp"
    src.write_text('''
#include <cstdio>
#include "fd_scaled_rules.h"
int main(int, char**) {
  int n, N, K, c;
  while (std::scanf("%d %d %d %d", &n, &N, &K, &c) == 4)
    std::printf("%d %d %d %d %d\\n", (int)fd::scaled_few(n, N, K, c, false, 256) + 2 * (int)fd::scaled_few(n, N, K, c, true, 256), (int)fd::scaled_large(n, N, K, c, 256), (int)fd::scaled_both(n, N, K, c, 256), (int)fd::scaled_small(n, N, 256), (int)fd::scaled_few_wide(N, 256));
}
''')
    exe = tmp_path / "r"
    subprocess.run(["g++", "-std=c++17", f"-I{build.CSRC}", str(src), "-o", str(exe)], check=True)
    # (M, N, K, codes): few rows (1: to bf16, 2: to fp32), 256-row tiles, both, 64-row tiles
    cases = [((9828, 1536, 6144, 0), (0, 1, 1, 0)), ((5000, 1536, 6144, 0), (0, 0, 0, 0)), ((9828, 6144, 1536, 1), (0, 0, 0, 0)),
             ((32760, 1536, 6144, 0), (0, 1, 1, 0)), ((9828, 1536, 1536, 0), (0, 1, 0, 0)), ((1664, 1536, 6144, 0), (0, 0, 0, 0)),
             ((14280, 4096, 1024, 1), (0, 0, 0, 0)), ((1, 64, 64, 0), (3, 0, 0, 1)), ((1 << 30, 16, 16, 0), (0, 1, 1, 0)), ((9828, 4608, 1536, 0), (0, 1, 0, 0)),
             ((4096, 6144, 1536, 0), (0, 0, 0, 0)), ((1312, 1024, 4096, 0), (0, 0, 0, 1)), ((1366, 1536, 400, 0), (0, 0, 0, 0)), ((1344, 1536, 384, 0), (0, 0, 0, 1)),
             ((1, 1 << 20, 1024, 0), (3, 1, 0, 0)), ((1, 6144, 1536, 1), (0, 0, 0, 1)), ((32, 12288, 4096, 0), (0, 0, 0, 1)), ((32, 8192, 4096, 0), (3, 0, 0, 1)), ((64, 6144, 1536, 0), (3, 0, 0, 1)), ((128, 1536, 6144, 0), (2, 0, 0, 1)), ((128, 1536, 1536, 0), (3, 0, 0, 1)), ((128, 4608, 6144, 0), (0, 0, 0, 1)),
             ((200, 1536, 6144, 0), (0, 0, 0, 1)), ((400, 1536, 6144, 0), (0, 0, 0, 1))]
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c, _ in cases), capture_output=True, text=True, check=True).stdout
    for line, (case, want) in zip(out.splitlines(), cases):
        assert tuple(map(int, line.split())) == want + (int(case[1] > 4096),), case


def test_no_vector_memory_read_of_a_fresh_scalar(tmp_path):
    """The product's loads in inline assembly, searched as those of the bf16 products are."""
    out = tmp_path / "k.s"
    subprocess.run([build.hipcc(), *[f for f in build.HIPCC_FLAGS if f != "-Wall"], "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, "k_scaled_gemm.hip"), "-o", str(out)], check=True, capture_output=True)
    seen, bad = _hazards(out.read_text().splitlines())
    assert seen > 300
    assert not bad, bad[:3]


@no_gpu
def test_scaled_block_refuses():
    lib = fdl.lib()
    plan, d = fdl.FdPlan(16, 4, 1, 4, 16, *([P] * 6)), fdl.FdDims(16, 128, 2, 64, 256)
    need = lib.fd_scaled_block_ws_size(ctypes.byref(plan), ctypes.byref(d))
    assert need > lib.fd_block_ws_size(ctypes.byref(plan), ctypes.byref(d)) > 0
    assert lib.fd_scaled_block_ws_size(None, None) == 0
    ok = dict(plan=plan, dims=d, w=[P] * 15, rope=None, coord=None, h=P, idx=P, cu=P, m=P, k=P, v=P, ws=P, n=need)

    def call(**change):
        a = dict(ok, **change)
        w = a["w"] and fdl.FdScaledWeights(*a["w"])
        return lib.fd_scaled_block_forward(ctypes.byref(a["plan"]), ctypes.byref(a["dims"]), ctypes.byref(w) if w else None,
                                           ctypes.byref(a["rope"]) if a["rope"] else None, a["coord"], *(a[x] for x in ("h", "idx", "cu", "m", "k", "v", "ws", "n")), None)

    for x in ("w", "h", "idx", "cu", "m", "k", "v", "ws"):
        assert call(**{x: None}) == 1, x
    for i in range(15):
        w = [P] * 15
        w[i] = None
        assert i in (12, 13) or call(w=w) == 1          # the norms' weights may be absent
        w[i] = P + 2
        assert call(w=w) == 1, i
    assert call(n=need - 1) == 2 and b"workspace" in lib.fd_last_error()
    assert call(rope=fdl.rope_axes([64])) == 1          # no coordinates
    assert call(rope=fdl.rope_axes([66]), coord=P) == 1
    assert call(dims=fdl.FdDims(16, 96, 2, 48, 256)) == 3 and call(dims=fdl.FdDims(16, 128, 4, 64, 256)) == 2
    assert call(plan=fdl.FdPlan(2050, 1025, 1025, 2, 2, *([P] * 6))) == 3
    assert call(dims=fdl.FdDims(64, 4096, 32, 128, 1 << 19)) == 3   # 2 GiB of MLP weights
    for x in ("h", "k", "v", "ws"):
        assert call(**{x: P + 8}) == 1


def test_large_tile_cases_run_large_tiles(tmp_path):
    """The GPU tests of the 256 x 256 tiles have shapes that the rules send there, two tiles a workgroup among them; the
    one whose row count the device picks by launches both kernels."""
    from tests.test_gpu_scaled_paths import LARGE_CODES, LARGE_WIDE
    src = tmp_path / "r.cpp"
    src.write_text('''
#include <cstdio>
#include "fd_scaled_rules.h"
int main(int, char**) {
  int n, N, K, c;
  while (std::scanf("%d %d %d %d", &n, &N, &K, &c) == 4)
    std::printf("%d %d %d\\n", (int)(fd::scaled_few(n, N, K, c, false, 256) || fd::scaled_small(n, N, 256)), (int)fd::scaled_large(n, N, K, c, 256), (int)fd::scaled_both(n, N, K, c, 256));
}
''')
    exe = tmp_path / "r"
    subprocess.run(["g++", "-std=c++17", f"-I{build.CSRC}", str(src), "-o", str(exe)], check=True)
    cases = [(*s, 0) for s in LARGE_WIDE] + [(*s, 1) for s in LARGE_CODES] + [(3000, *LARGE_CODES[1][1:], 1)]
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, check=True).stdout
    got = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert all(few_or_small == 0 for few_or_small, _, _ in got)
    assert [large for _, large, _ in got] == [1] * (len(cases) - 1) + [0]
    assert got[-2][2] == 1
    tiles = [-(-M // 256) * -(-N // 256) for M, N, _, _ in cases[:-1]]
    assert max(tiles[:len(LARGE_WIDE)]) > 256 and max(tiles[len(LARGE_WIDE):]) > 256


@no_gpu
def test_scaled_block_refuses_rows_beyond_its_steps():
    """More tokens than the steps' row numbers hold: refused before the first of them is enqueued."""
    n = (1 << 30) + 1
    plan, d, w = fdl.FdPlan(n, 1025, 1024, 1 << 20, 1 << 20, *([P] * 6)), fdl.FdDims(16, 128, 2, 64, 256), fdl.FdScaledWeights(*[P] * 15)
    st = fdl.lib().fd_scaled_block_forward(ctypes.byref(plan), ctypes.byref(d), ctypes.byref(w), None, None, *([P] * 7), 1 << 62, None)
    assert st == 3 and b"rows" in fdl.lib().fd_last_error()


def test_scale_stride_to_the_last_column_count():
    for cols in ((1 << 30) + 1, 2 ** 31 - 129, 2 ** 31 - 128, 2 ** 31 - 127, 2 ** 31 - 1):
        assert fdl.fd_scale_stride(cols) == ref.stride(cols)


@no_gpu
def test_columns_beyond_32_bits_refused():
    lib = fdl.lib()
    for cols in ((1 << 30) + 16, 2 ** 31 - 128, 2 ** 31 - 16):
        assert lib.fd_quant_blocks(1, cols, 1, P, None, P, P, None) == 3 and b"columns" in lib.fd_last_error()
        assert lib.fd_quant_blocks(1, cols, 128, P, None, P, P, None) == 3
        assert lib.fd_rms_quant(1, cols, 1, P, None, None, None, None, None, 0, 1e-6, None, P, P, P, None) == 3
        assert lib.fd_scaled_linear(1, 64, cols, P, P, P, P, None, 0, None, P, None, None, None, None) == 3


def test_step_refuses_half_of_the_rotary_positions():
    """A descriptor without positions would fail in the first step, after the gate has moved on; positions without a
    descriptor would be ignored; positions laid out the other way round would turn by the wrong ones."""
    plan = fdl.make_plan(np.zeros(6, np.int32), np.array([0, 6]), 1, device="cpu")
    d, r, pos = fdl.dims(16, 64, 1, 64, 256), fdl.rope_axes([32, 32]), torch.zeros(6, 2, dtype=torch.int32)
    for rope, coord, why in ((r, None, "both"), (None, pos, "both"), (r, pos.t().contiguous(), "6, 2"), (r, pos[:5], "6, 2"), (r, pos[:, :1], "6, 2"), (r, pos, "coord must be a device tensor")):
        with pytest.raises(fdl.FlashDiffError, match=why):
            fdl.SparseStep(plan, d, {}, 1, device="cpu", scaled={}, rope=rope, coord=coord)


def test_bindings_name_what_is_absent():
    q, s, h, i = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8), torch.zeros(4, 64), torch.zeros(2, dtype=torch.int32)
    for call, what in ((lambda: fdl.fd_quant_blocks(None, 1, q, s), "x is"), (lambda: fdl.fd_rms_quant(None, q, s, i, i), "h is"),
                       (lambda: fdl.fd_rope_axes(None, i, None, i, h, h, h, 1, 1, 16, dims=[16]), "qkv is"),
                       (lambda: fdl.fd_rope_axes(h, None, None, i, h, h, h, 2, 1, 16, dims=[16]), "coord is"),
                       (lambda: fdl.fd_rope_axes(h, i.view(1, 2), None, i, h, h, h, 2, 1, 16), "axes are"),
                       (lambda: fdl.fd_scaled_linear(None, s, q, s, h), "a is"), (lambda: fdl.fd_scaled_linear(q, s, None, s, h), "w is"),
                       (lambda: fdl.fd_scaled_linear(q, s, q, s, None), "y is")):
        with pytest.raises(fdl.FlashDiffError, match=what):
            call()
