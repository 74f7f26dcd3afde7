"""The 8-bit operators where their kernels take another path: products in 256 x 256 tiles with a bias, GELU, 8-bit
results and short or ragged sums, blocks of NaN and far scale bytes through every kind of result, and norms of more rows than waves, whose requests change inside a run."""
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

from oracle import scaled as ref
from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_scaled import U32, check_linear, linear_case, rms_case, run_linear, run_rms
from tests.test_gpu_scaled_block import make
from tests.test_gpu_scaled_precision import check_same_codes

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


# ------------------------------------------------------------------ product

# (M, N, K): 256 x 256 tiles where the row count is the host's (test_scaled_host.py holds the rule to it).  Short sums, last
# blocks of 16 and of 112 columns, tiles that rows and columns leave part of, one tile a workgroup and two.
LARGE_WIDE = [(8192, 2048, 16), (8190, 2032, 240), (8190, 2048, 512), (14999, 2032, 144)]
LARGE_CODES = [(3500, 4112, 2896), (6800, 4368, 2832)]


@pytest.mark.parametrize("M,N,K", LARGE_WIDE)
@pytest.mark.parametrize("to,gelu", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
def test_large_tiles(M, N, K, to, gelu):
    gh.say(f"linear M={M} N={N} K={K} to={to} gelu={gelu}")
    case = linear_case(M, N, K, 5)
    y, ys = run_linear(*case, gelu, to, M, None)
    check_linear(y, ys, *case, gelu, to, M)


@pytest.mark.parametrize("M,N,K", LARGE_CODES)
@pytest.mark.parametrize("gelu", [False, True])
def test_large_tiles_to_codes(M, N, K, gelu):
    gh.say(f"linear M={M} N={N} K={K} to codes, gelu={gelu}")
    case = linear_case(M, N, K, 5)
    y, ys = run_linear(*case, gelu, "8", M, None)
    check_linear(y, ys, *case, gelu, "8", M)


@pytest.mark.parametrize("m", [6800, 3000, 77, 0])
def test_codes_with_the_row_count_on_the_device(m):
    """A capacity at which both tiles of 8-bit results are launched and the row count picks: codes and scale bytes of the
    call with just those rows where the host picks the same tiles (6800 and 3000), else within the bound of check_linear; rows
    past them stay."""
    M, N, K = LARGE_CODES[1]
    gh.say(f"linear capacity {M} N={N} K={K} to codes, m={m}")
    a, sa, w, sw, bias = linear_case(M, N, K, 6)
    y, ys = run_linear(a, sa, w, sw, bias, True, "8", M, m)
    if m in (6800, 3000):
        y2, ys2 = run_linear(a[:m], sa[:m], w, sw, bias, True, "8", m, None)
        assert torch.equal(y[:m], y2) and np.array_equal(ys[:m], ys2)
    some = np.unique(np.r_[:min(m, 40), max(0, m - 40):m].astype(int))
    if len(some):
        check_linear(y[some], ys[some], a[some], sa[some], w, sw, bias, True, "8", len(some))
    nk = -(-N // 128)
    assert (y[m:] == 0x55).all() and np.all(ys[m:] == 0x55) and np.all(ys[:, nk:] == 0x55)


@pytest.mark.parametrize("to", ["bf16", "8"])
@pytest.mark.parametrize("M,N,K", [(5, 400, 400), (200, 400, 400), (3000, 1536, 400), (8190, 2048, 400), (3500, 4112, 2896)])
def test_bad_blocks(M, N, K, to):
    """A NaN block of a row makes that row NaN, one of the weights its 128 columns, as values and as 8-bit blocks; the rest
    has the bits that it has without them."""
    gh.say(f"NaN blocks M={M} N={N} K={K} to={to}")
    case = linear_case(M, N, K)
    a, sa, w, sw, bias = (x.copy() for x in case)
    a[3, 128:256], sa[3, 1] = 0x7f, 255
    w[128:256, 384:512], sw[1, 3] = 0x7f, 255
    (y, ys), (clean, cs) = run_linear(a, sa, w, sw, bias, False, to, M, None), run_linear(*case, False, to, M, None)
    bad = np.zeros((M, N), bool)
    bad[3], bad[:, 128:256] = True, True
    if to == "8":
        y, clean, nk = y.numpy(), clean.numpy(), -(-N // 128)
        assert np.all((y[bad] & 127) == 127) and np.array_equal(ys[:, :nk] == 255, bad[:, ::128])
        assert np.array_equal(ys[:, :nk][~bad[:, ::128]], cs[:, :nk][~bad[:, ::128]])
    else:
        assert np.array_equal(torch.isnan(y).numpy(), bad)
        y, clean = y.view(torch.int16).numpy(), clean.view(torch.int16).numpy()
    assert np.array_equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("s", [0, 1, 2, 60, 127, 200, 246, 253, 254])
@pytest.mark.parametrize("to", ["bf16", "f32", "8"])
@pytest.mark.parametrize("M", [5, 200])
def test_every_finite_scale_byte(M, to, s):
    """Rows' scale bytes from 0 (2^-127, which fd_quant_blocks does not write) to 254, against weights that bring the product
    back towards ordinary size.  Codes are cut to values that are normal in fp32: 2 or more, or zero, beside the smallest
    scales, 1 or less beside the largest."""
    gh.say(f"scale byte {s} M={M} to={to}")
    a, sa, w, sw, _ = linear_case(M, 144, 256, 9)
    sa[:, :2], sw[:, :2] = s, np.clip(250 - s, 1, 246)
    mag = a & 0x7f
    if s < 3:
        a = np.where(mag >= 0x40, a, 0).astype(np.uint8)
    if s > 246:
        a = ((a & 0x80) | np.minimum(mag, 0x38)).astype(np.uint8)
    if sw[0, 0] < 20:
        w = np.where((w & 0x7f) >= 0x40, w, 0).astype(np.uint8)
    y, ys = run_linear(a, sa, w, sw, None, False, to, M, None)
    check_linear(y, ys, a, sa, w, sw, None, False, to, M)


# ------------------------------------------------------------------ residual and norm

@pytest.mark.parametrize("parts", ["ygwm", "m", "yg"])
@pytest.mark.parametrize("rows,D,B,m", [
    (9001, 320, 40, 8999), (5000, 768, 5, 5000), (4099, 1024, 9, 4099), (2100, 1088, 30, 2099), (3200, 1536, 2, 3200), (1500, 2064, 7, 1500),
    (1300, 6144, 4, 1290), (1100, 8192, 6, 1100), (1100, 12288, 3, 1030),
    (33, 528, 3, 30), (7, 1024, 2, 7), (5, 4112, 2, 5), (3, 6144, 3, 2)])
def test_rms_runs(rows, D, B, m, parts):
    """Runs of several rows a team of one, two and four waves, whose requests begin inside a run, one or more of them empty; and
    the widths between the forms.  fp32 errors as in test_rms_quant of test_gpu_scaled.py."""
    gh.say(f"rms {rows}x{D} B={B} m={m} parts={parts!r}")
    h, y, mod, weight, cu = rms_case(rows, D, B, m, parts, 1)
    if B > 2:
        cu[2] = cu[1]   # an empty request between two others
    got, q, s = run_rms(h, y, mod, weight, cu, m, parts)
    of_row = np.repeat(np.arange(B), np.diff(cu))
    pick = lambda i, on: mod[of_row, i * D:(i + 1) * D].astype(np.float64) if on in parts else None  # noqa: E731
    y64 = None if y is None else y.double().numpy()[:m]
    gate, shift, scale = pick(2, "g"), pick(0, "m"), pick(1, "m")
    wh, wa = ref.rms(h[:m], y64, gate, None if weight is None else weight.astype(np.float64), shift, scale, 1e-6)
    add = 0.0 if y64 is None else np.abs(y64) * (1.0 if gate is None else np.abs(gate))
    assert np.all(np.abs(got[:m] - wh) <= 2 * U32 * (np.abs(wh) + add))
    np.testing.assert_array_equal(got[m:], h[m:])
    base = np.abs(wa - (0 if shift is None else shift))
    h_err = 2 * U32 * (np.abs(wh) + add) / np.sqrt(np.mean(wh * wh, 1, keepdims=True))
    w_abs = (1.0 if weight is None else np.abs(weight)) * (1.0 if scale is None else np.abs(1 + scale))
    err = (28 + 8 + 2) * U32 * base + h_err * w_abs + 2 * U32 * np.abs(wa)
    check_same_codes(q[:m], s[:m], wa, err, 0.99)
    assert np.all(q[m:] == 0x55) and np.all(s[m:] == 0x55)


def test_residual_alone_in_runs():
    """h's update without codes, more rows than teams: the bits of the call that writes codes too."""
    h, y, mod, _, cu = rms_case(5000, 1088, 6, 4990, "yg", 2)
    want, _, _ = run_rms(h, y, mod, None, cu, 4990, "yg")
    x, d_mod = torch.from_numpy(h).cuda(), torch.from_numpy(mod).cuda()
    fdl.fd_rms_quant(x, None, None, torch.from_numpy(cu).cuda(), torch.tensor([4990], dtype=torch.int32, device="cuda"), y=y.cuda(), gate=d_mod[:, 2176:])
    assert np.array_equal(x.cpu().numpy(), want)


@pytest.mark.parametrize("D", [16, 768, 1536, 12288])
def test_rms_on_both_sides_of_the_overflow(D):
    """Rows of one magnitude, 2% below and above 2^64 / sqrt(D): their squares add up to 0.96 and 1.04 times 2^128.  Below, the
    norm is 1 (within the 38 half steps of test_rms_quant, so its code is 1's), above it is zero, as the header says; an
    ordinary row between them is as ever."""
    v = 2.0 ** 64 / np.sqrt(D)
    sign = np.where(np.arange(D) % 3 == 0, -1.0, 1.0)
    h = np.stack([0.98 * v * sign, sign, 1.02 * v * sign]).astype(np.float32)
    _, q, s = run_rms(h, None, np.zeros((1, 3 * D), np.float32), None, np.array([0, 3], np.int32), 3, "")
    got = ref.values(q, s)
    assert np.array_equal(got[0], sign) and np.array_equal(got[1], sign) and np.all(got[2] == 0)


# ------------------------------------------------------------------ rotary positions

def test_rope_of_more_rows_than_a_launch_has():
    """2^26 + 5 rows of 3 x 16, 64 threads a row: rows at both ends and where one launch meets the next, against the same rows
    in a call of their own."""
    rows, dh = (1 << 26) + 5, 16
    gh.say(f"rope of {rows} rows")
    pick = torch.cat([torch.arange(a, b) for a, b in ((0, 50), ((1 << 25) - 50, (1 << 25) + 50), ((1 << 26) - 50, rows))]).cuda()
    x = torch.zeros((rows, 3 * dh), dtype=torch.bfloat16, device="cuda")
    part = torch.randn((len(pick), 3 * dh), device="cuda").to(torch.bfloat16)
    x[pick] = part
    coord = torch.zeros((rows, 1), dtype=torch.int32, device="cuda")
    coord[pick] = torch.arange(1, len(pick) + 1, dtype=torch.int32, device="cuda")[:, None]
    m = torch.tensor([rows], dtype=torch.int32, device="cuda")
    (q, k, v), (q2, k2, v2) = ([torch.zeros((n, dh), dtype=torch.bfloat16, device="cuda") for _ in range(3)] for n in (rows, len(pick)))
    kw = dict(heads=1, kv_heads=1, head_dim=dh, dims=[16])
    fdl.fd_rope_axes(x, coord, None, m, q, k, v, **kw)
    fdl.fd_rope_axes(part, coord[pick].contiguous(), None, m, q2, k2, v2, **kw)
    assert torch.equal(q[pick], q2) and torch.equal(k[pick], k2) and torch.equal(v[pick], v2)
    assert not torch.equal(q2, part[:, :dh])


def rest_of_turns(pos, dim, theta, step):
    """pos * step * theta^(-2j / dim) / 2 pi without its whole turns, from 70 digits: [len(pos)][dim / 2], and the turns per
    position [dim / 2]."""
    with localcontext() as c:
        c.prec = 70
        two_pi = 2 * Decimal("3.1415926535897932384626433832795028841971693993751058209749445923078164")
        rate = [Decimal(step) * Decimal(theta) ** (Decimal(-2 * j) / Decimal(dim)) / two_pi for j in range(dim // 2)]
        turns = [[int(p) * r for r in rate] for p in pos]
        return np.array([[float(t - t.to_integral_value()) for t in row] for row in turns]), np.array([abs(float(r)) for r in rate])


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("theta,step", [(1e4, 1.0), (1e4, 6.5e6), (100.0, -40.0), (0.25, 3.0), (1e4, 1e5)])
def test_rope_of_far_positions(theta, step, halves):
    """Positions to the ends of int32 and pairs that turn up to a million times per position, against angles from 70 digits,
    within the error that the header states: 2^-26 + |pos| (2^-48 + 2^-58 r) of a turn, as radians times the pair's length; cosine,
    sine and products as in test_rope of test_gpu_scaled.py."""
    gh.say(f"rope theta={theta} step={step} halves={halves}")
    pos = np.array([0, 1, -1, 12345, 1_000_003, -99_999_999, 100_000_000, 1_234_567_891, 2 ** 31 - 1, -2 ** 31], np.int64)
    rows, dh = len(pos), 64
    x = torch.from_numpy(np.random.default_rng(11).standard_normal((rows, 3 * dh)).astype(np.float32)).to(torch.bfloat16)
    q, k, v = (torch.zeros((rows, dh), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    fdl.fd_rope_axes(x.cuda(), torch.from_numpy(pos.astype(np.int32))[:, None].cuda(), None, torch.tensor([rows], dtype=torch.int32, device="cuda"),
                     q, k, v, heads=1, kv_heads=1, head_dim=dh, dims=[dh], theta=theta, step=step, halves=halves)
    rest, rate = rest_of_turns(pos, dh, theta, step)
    c, n = np.cos(2 * np.pi * rest), np.sin(2 * np.pi * rest)
    err = 2 * np.pi * (2.0 ** -26 + np.abs(pos)[:, None] * (2.0 ** -48 + 2.0 ** -58 * rate))
    for got, at in ((q, 0), (k, dh)):
        x64, got = x.double().numpy()[:, at:at + dh], got.double().cpu().numpy()
        a, b = (slice(0, dh // 2), slice(dh // 2, dh)) if halves else (slice(0, dh, 2), slice(1, dh, 2))
        u, w = x64[:, a], x64[:, b]
        for part, want in ((a, u * c - w * n), (b, u * n + w * c)):
            far = err * np.hypot(u, w) + 2.0 ** -21 * (np.abs(u) + np.abs(w))
            assert np.all(np.abs(got[:, part] - want) <= 2.0 ** -8 * np.abs(want) + (1 + 2.0 ** -8) * far)


# ------------------------------------------------------------------ refusals

def test_block_weights_of_another_type_or_size_refused():
    """The block reads its parameters by address: what does not hold what it reads raises."""
    case, scaled, _, _ = make("tiny")
    mod = torch.zeros((case.w.B, 6 * case.w.D), device="cuda")
    fdl.scaled_weights(scaled, 0, mod)
    fdl.scaled_weights({k: t for k, t in scaled.items() if not k.startswith("norm")}, 0, mod)
    change = dict(norm_1=lambda t: t.bfloat16(), norm_2=lambda t: t[:, :-16].contiguous(), b_qkv=lambda t: t.bfloat16(), b_1=lambda t: t[:, :-64].contiguous(),
                  s_2=lambda t: t[..., :-4].contiguous(), w_1=lambda t: t.to(torch.float32), s_qkv=lambda t: t.cpu(), w_2=lambda t: t[:, :-64].contiguous())
    for name, f in change.items():
        with pytest.raises(fdl.FlashDiffError, match=name):
            fdl.scaled_weights(dict(scaled, **{name: f(scaled[name])}), 0, mod)
    with pytest.raises(fdl.FlashDiffError, match="mod"):
        fdl.scaled_weights(scaled, 0, mod[:, :-1].contiguous())


def test_step_refuses_positions_that_its_blocks_would():
    """Positions of another type, or with strides, raise when the step is made, not in it after the gate has moved on."""
    case, scaled, rope, pos = make("tiny")
    r, c = fdl.rope_axes(**rope), torch.from_numpy(pos).cuda()
    kw = dict(k_cache=case.k_cache.cuda(), v_cache=case.v_cache.cuda(), scaled=scaled, rope=r)
    fdl.SparseStep(case.plan, case.dims, case.params_gpu, case.w.L, coord=c, **kw)
    for bad in (c.long(), c.float(), c.t().contiguous().t(), c.cpu()):
        with pytest.raises(fdl.FlashDiffError):
            fdl.SparseStep(case.plan, case.dims, case.params_gpu, case.w.L, coord=bad, **kw)
