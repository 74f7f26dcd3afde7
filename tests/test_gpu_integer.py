"""8-bit integer rows, their product and the norms on both sides of a branch against the 64-bit reference: sizes around
their waves and tiles, no rows, rows past the count, zeros, infinities and NaN, every output type."""
import numpy as np
import pytest
import torch

from oracle import integer as ref
from oracle import scaled
from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_scaled import U32, UB, bf16, check_codes, count, dev

pytestmark = pytest.mark.gpu

FILL = 0x55


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


def ints(rows, cols):
    return torch.full((rows, cols), FILL, dtype=torch.int8, device="cuda"), torch.full((rows,), -7.0, device="cuda")


# ------------------------------------------------------------------ rows

@pytest.mark.parametrize("rows,cols,m", [(1, 16, None), (1, 512, 1), (5, 528, 4), (3, 1024, None), (9, 1040, 9), (4, 1536, 0), (3, 2064, 2),
                                         (2, 4112, None), (2, 6160, 2), (2, 8208, 1), (1, 32784, None), (2, 65536, 2), (20000, 32, 19999)])
def test_rows_exact(rows, cols, m):
    """Every step of the definition is one rounding of fp32, so the bits are the definition's."""
    gh.say(f"int8 rows {rows}x{cols} m={m}")
    rng = np.random.default_rng([rows, cols])
    x = bf16(rng.standard_normal((rows, cols)) * np.exp(3 * rng.standard_normal((rows, 1))))
    q, s = ints(rows, cols)
    fdl.fd_int_rows(x.cuda(), q, s, m=None if m is None else count(m))
    n = rows if m is None else m
    wq, ws = ref.int_rows(x.float().numpy())
    np.testing.assert_array_equal(q.cpu().numpy()[:n], wq[:n])
    np.testing.assert_array_equal(s.cpu().numpy()[:n], ws[:n])
    assert (q[n:] == FILL).all() and (s[n:] == -7).all()


def test_rows_edges():
    """Zeros, subnormals, the limit of a row of zeros and its neighbours, the largest values, ties; a bad row is NaN and its neighbours
    are as ever."""
    vals = [0.0, 1e-40, 1e-38, 2.0 ** -101, 2.0 ** -100, 2.0 ** -99, 1e-20, 1.0, 127.0, 254.0, 3e38, np.inf, -np.inf, np.nan]
    x = np.zeros((len(vals), 32), np.float32)
    for i, v in enumerate(vals):
        x[i] = (v if np.isfinite(v) else 1.0) * np.linspace(-1, 1, 32, dtype=np.float32)
        x[i, 7] = v
    x[9, :16] = 2 * (np.arange(16) - 7.5)       # of 254: every value a tie
    x = bf16(x)
    q, s = ints(*x.shape)
    fdl.fd_int_rows(x.cuda(), q, s)
    wq, ws = ref.int_rows(x.float().numpy())
    np.testing.assert_array_equal(s.cpu().numpy(), ws)
    np.testing.assert_array_equal(q.cpu().numpy(), wq)


# ------------------------------------------------------------------ product

def gelu_err(z):
    """What the kernel's GELU may be off for an exact argument: its exponent t has three roundings, then the
    exponent, one sum, the reciprocal (an ulp each) and a product."""
    t = np.abs(2 * np.sqrt(2 / np.pi) * np.log2(np.e) * (z + 0.044715 * z ** 3))
    return np.abs(scaled.gelu(z)) * (t * 2.0 ** -22 + 2.0 ** -21) + 2.0 ** -126


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("rows,n,k,m", [(1, 16, 16, None), (1, 4608, 1536, 1), (2, 48, 144, 1), (16, 144, 1088, 16), (17, 16, 128, 17), (33, 272, 112, 30),
                                        (64, 1536, 64, None), (65, 128, 4112, 65), (100, 1040, 528, 0), (129, 130 * 16, 16, 128), (257, 528, 1104, 257),
                                        (300, 4288, 1088, 299), (1021, 1536, 640, 1021), (1300, 4608, 144, 1299), (4100, 1040, 272, None)])
def test_linear(rows, n, k, m, wide, gelu):
    """The sum is exact; its conversion, the scales' product, the product with it and the bias are a rounding each."""
    gh.say(f"int8 linear {rows}x{n}x{k} m={m} wide={wide} gelu={gelu}")
    rng = np.random.default_rng([rows, n, k])
    a, w = rng.integers(-128, 128, (rows, k)).astype(np.int8), rng.integers(-128, 128, (n, k)).astype(np.int8)
    sa, sw = np.exp(rng.standard_normal(rows)).astype(np.float32) / 127, np.exp(rng.standard_normal(n)).astype(np.float32) / 127 / np.sqrt(k).astype(np.float32)
    bias = None if m is None else rng.standard_normal(n).astype(np.float32)
    y = torch.full((rows, n), 7.0, dtype=torch.float32 if wide else torch.bfloat16, device="cuda")
    fdl.fd_int_linear(dev(a), dev(sa), dev(w), dev(sw), y, bias=None if bias is None else dev(bias), gelu=gelu, m=None if m is None else count(m))
    cnt = rows if m is None else m
    got = y.double().cpu().numpy()
    z, size = ref.linear(a[:cnt], sa[:cnt], w, sw, bias)
    err = 4 * U32 * size + U32 * np.abs(z)
    want = z
    if gelu:
        want, err = scaled.gelu(z), 1.13 * err + gelu_err(z)       # GELU's slope is at most 1.129
    if not wide:
        err = err + UB * (np.abs(want) + err)
    worst = np.max(np.abs(got[:cnt] - want) - err, initial=-np.inf)
    assert worst <= 0, f"off by {worst} more than allowed"
    assert np.all(got[cnt:] == 7)


def test_linear_largest_sums():
    """Sums at the limits of the accumulator, +-2^30 at the most columns, are exact; scales of zero and NaN."""
    k = 65536
    a, w = np.full((3, k), -128, np.int8), np.full((32, k), -128, np.int8)
    a[1], w[5] = 127, 127
    sa, sw = np.array([1.0, 2.0, np.nan], np.float32), np.ones(32, np.float32)
    sw[7] = 0
    y = torch.zeros((3, 32), device="cuda")
    fdl.fd_int_linear(dev(a), dev(sa), dev(w), dev(sw), y)
    want = (a.astype(np.int64) @ w.astype(np.int64).T).astype(np.float32) * sa[:, None] * sw
    np.testing.assert_array_equal(y.cpu().numpy(), want)


# ------------------------------------------------------------------ norms

@pytest.mark.parametrize("parts,to", [(p, t) for p in ("", "y", "ypg", "pgm", "wm", "ypgwmr", "yr") for t in ("bf16", "codes", "ints", None)
                                      if t or "y" in p])
@pytest.mark.parametrize("rows,D,B,m", [(1, 16, 1, 1), (5, 64, 1, 3), (9, 1088, 4, 9), (33, 1536, 7, 30), (6, 2048, 2, 6), (5, 528, 2, 5),
                                        (5, 2064, 3, 4), (3, 6160, 2, 3), (2, 12288, 1, 2), (4, 128, 3, 0), (3, 4112, 1, 3)])
def test_norm_residual(rows, D, B, m, parts, to):
    """fp32 error: a sum of squares has at most 48 terms per lane and a tree of 8 levels (relative error 56 half steps,
    halved by the root), then the root, the quotients and the products, 8 roundings more."""
    gh.say(f"norm {rows}x{D} B={B} m={m} parts={parts!r} to={to}")
    rng = np.random.default_rng([rows, D, B])
    h = (rng.standard_normal((rows, D)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)
    y = bf16(rng.standard_normal((rows, D)) * np.exp(2 * rng.standard_normal((rows, 1)))) if "y" in parts else None
    mod = (0.3 * rng.standard_normal((B, 3 * D))).astype(np.float32)
    post, weight = ((1 + 0.1 * rng.standard_normal(D)).astype(np.float32) if on in parts else None for on in "pw")
    cuts = np.sort(rng.integers(0, m + 1, B - 1))
    cu = np.concatenate([[0], cuts, [m]]).astype(np.int32)
    residual = -0.625 if "r" in parts else 1.0
    d_h, d_mod = dev(h), dev(mod)
    piece = lambda i, on: d_mod[:, i * D:(i + 1) * D] if on in parts else None  # noqa: E731
    a, scale = None, None
    if to == "bf16":
        a = torch.full((rows, D), 7.0, dtype=torch.bfloat16, device="cuda")
    elif to == "codes":
        a, scale = (torch.full((rows, c), FILL, dtype=torch.uint8, device="cuda") for c in (D, scaled.stride(D)))
    elif to == "ints":
        a, scale = ints(rows, D)
    fdl.fd_norm_residual(d_h, a, dev(cu), count(m), y=None if y is None else y.cuda(), post_weight=None if post is None else dev(post),
                         gate=piece(2, "g"), residual=residual, weight=None if weight is None else dev(weight), shift=piece(0, "m"),
                         mod_scale=piece(1, "m"), a_scale=scale)
    of_row = np.repeat(np.arange(B), np.diff(cu))
    pick = lambda i, on: mod[of_row, i * D:(i + 1) * D].astype(np.float64) if on in parts else None  # noqa: E731
    y64 = None if y is None else y.double().numpy()[:m]
    shift, sc = pick(0, "m"), pick(1, "m")
    wh, add, wa = ref.norm_residual(h[:m], y64, post, pick(2, "g"), residual, weight, shift, sc, 1e-6)
    got_h = d_h.cpu().numpy()
    h_err = 0.0 if y is None else 2 * U32 * (np.abs(wh) + np.abs(residual * h[:m])) + (28 + 8 + 4) * U32 * np.abs(add)
    assert np.all(np.abs(got_h[:m] - wh) <= h_err)
    np.testing.assert_array_equal(got_h[m:], h[m:])
    if to is None or not m:
        return
    # an error of h reaches a through h itself and through its norm
    rms = np.sqrt(np.mean(wh * wh, 1, keepdims=True) + 1e-6)
    w_abs = (1.0 if weight is None else np.abs(weight)) * (1.0 if sc is None else np.abs(1 + sc))
    base = np.abs(wa - (0 if shift is None else shift))
    through = np.sqrt(np.mean(np.square(h_err * np.ones_like(wh)), 1, keepdims=True)) / rms
    err = ((28 + 8 + 2) * U32 + through) * base + h_err / rms * w_abs + 2 * U32 * np.abs(wa)
    got = a.cpu()
    if to == "bf16":
        assert np.all(np.abs(got.double().numpy()[:m] - wa) <= err + UB * (np.abs(wa) + err)) and (got[m:] == 7).all()
    elif to == "codes":
        check_codes(got.numpy()[:m], scale.cpu().numpy()[:m], wa, err)
        assert (got[m:] == FILL).all() and (scale[m:] == FILL).all()
    else:
        s = scale.double().cpu().numpy()[:m, None]
        top, top_err = np.max(np.abs(wa), 1, keepdims=True), np.max(err, 1, keepdims=True)
        assert np.all(np.abs(s - top / 127) <= top_err / 127 + U32 * s)
        q = got.numpy().astype(np.float64)[:m]
        # half a step, three roundings of a value of up to 127 steps, and the error of the value
        assert np.all(np.abs(q * s - wa) <= s * (0.5 + 127 * 3 * U32) + err) and np.max(np.abs(q)) == 127
        assert (got[m:] == FILL).all() and (scale[m:] == -7).all()


@pytest.mark.parametrize("D", [192, 1536])
def test_norm_residual_zero_and_bad_rows(D):
    """A branch or a stream of zeros (eps 0: 0 * inf is NaN, as the formula says; eps > 0: zeros), rows with an infinity or a NaN
    in the branch or in the stream: those rows alone are NaN."""
    rng = np.random.default_rng(5)
    for eps in (1e-6, 0.0):
        h = rng.standard_normal((7, D)).astype(np.float32)
        y = rng.standard_normal((7, D)).astype(np.float32)
        h[1] = y[1] = y[2] = 0
        h[3, 100], y[4, 3], y[5, 17] = np.inf, np.nan, np.inf
        a, s = ints(7, D)
        d_h = dev(h)
        fdl.fd_norm_residual(d_h, a, None, count(7), y=bf16(y).cuda(), a_scale=s, eps=eps)
        got, gh_ = a.double().cpu().numpy() * s.double().cpu().numpy()[:, None], d_h.cpu().numpy()
        assert np.all(np.isfinite(got[[0, 6]])) and np.all(np.isfinite(gh_[[0, 6]]))
        assert np.all(np.isnan(got[[3, 4, 5]])) and np.all(np.isnan(gh_[4])) and np.isnan(gh_[5, 17])
        if eps:
            assert np.all(got[1] == 0) and np.all(gh_[1] == 0) and np.array_equal(gh_[2], h[2]) and np.all(np.isfinite(got[2]))
        else:
            assert np.all(np.isnan(got[[1, 2]])) and np.all(np.isnan(gh_[[1, 2]]))


def test_norm_residual_strides():
    """A modulation of equal rows (stride 0) and one request without offsets: the bits of the plain calls."""
    rng = np.random.default_rng(8)
    h, y = dev(rng.standard_normal((7, 144)).astype(np.float32)), bf16(rng.standard_normal((7, 144))).cuda()
    mod = dev(rng.standard_normal((1, 432)).astype(np.float32))
    out = []
    for cu, g in ((None, mod), (dev(np.array([0, 7], np.int32)), mod), (dev(np.array([0, 2, 7], np.int32)), mod.expand(2, 432))):
        x, a = h.clone(), torch.zeros((7, 144), dtype=torch.bfloat16, device="cuda")
        fdl.fd_norm_residual(x, a, cu, count(7), y=y, gate=g[:, :144], shift=g[:, 144:288], mod_scale=g[:, 288:], residual=0.5)
        out.append((x.cpu(), a.cpu()))
    assert all(torch.equal(a, b) for o in out[1:] for a, b in zip(out[0], o))
