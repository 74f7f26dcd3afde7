"""The 8-bit cache and its attention against the 64-bit reference: head dims, shared key heads, lengths from none to many
tiles, rows and tokens outside the requests, bad values, and the calls of a block together."""
import numpy as np
import pytest
import torch

from oracle import integer as ref
from oracle import scaled
from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_scaled import U8, U32, UB, bf16, count, dev

pytestmark = pytest.mark.gpu

FILL = 0x55


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


# ------------------------------------------------------------------ writing

@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dh,dims,hq,hk,rows,tokens,m", [
    (16, [16], 1, 1, 1, 1, 1), (16, [4, 6, 6], 4, 4, 9, 12, 7), (16, [16], 3, 5, 4, 5, 4), (64, [64], 6, 2, 5, 5, 5), (64, [32, 32], 24, 8, 33, 40, 33),
    (64, [2, 14, 20], 3, 1, 6, 9, 6), (128, [44, 42, 42], 12, 12, 17, 50, 16), (128, [32, 32, 32, 32], 1, 1, 3, 8, 0),
    (128, [16, 32, 32], 2, 1, 5, 7, 5), (64, None, 5, 3, 7, 9, 7), (128, None, 3, 3, 3, 3, 2), (16, None, 7, 1, 5, 6, 5)])
def test_cache_write(dh, dims, hq, hk, rows, tokens, m, halves):
    """q as fd_rope_axes writes it; k and v within half a code step and the turn's error, 2^-21 of a pair's magnitudes; cache rows
    of other tokens stay."""
    gh.say(f"cache write dh={dh} dims={dims} heads={hq}/{hk} rows={rows} m={m} halves={halves}")
    rng = np.random.default_rng([dh, rows, hq])
    qkv = bf16(rng.standard_normal((rows, (hq + 2 * hk) * dh)) * np.exp(rng.standard_normal((rows, 1))))
    idx = np.sort(rng.permutation(tokens)[:rows]).astype(np.int32)
    n = 1 if dims is None else len(dims)
    theta, step = [1e4, 100.0, 1e6, 10.0][:n], [1.0, 0.25, 3.0, 1.0][:n]
    pos = rng.integers(-1000, 1 << 20, (tokens, n)).astype(np.int32)
    new = lambda *shape: torch.full(shape, FILL, dtype=torch.uint8, device="cuda")  # noqa: E731
    k, ks, v, vs = new(tokens, hk * dh), new(hk, tokens), new(tokens, hk * dh), new(hk, tokens)
    q = torch.full((rows, hq * dh), 7.0, dtype=torch.bfloat16, device="cuda")
    r = None if dims is None else fdl.rope_axes(dims, theta, step, halves)
    fdl.fd_cache_write(qkv.cuda(), None if dims is None else dev(pos), dev(idx), count(m), q, k, ks, v, vs, hq, hk, dh, rope=r)
    x = qkv.double().numpy().reshape(rows, -1, dh)[:m]
    want = x if dims is None else np.concatenate([scaled.rope(x[:, :hq + hk], pos[idx[:m]], dims, theta, step, halves), x[:, hq + hk:]], 1)
    half_width = np.zeros_like(x)
    if dims is not None:      # a turned value is made of its pair
        pair = np.abs(x[:, :hq + hk])
        top = np.max(pair, axis=2, keepdims=True) * np.ones_like(pair)
        half_width[:, :hq + hk] = 2.0 ** -20 * top
    got_q = q.double().cpu().numpy()
    assert np.all(np.abs(got_q[:m].reshape(m, hq, dh) - want[:, :hq]) <= half_width[:, :hq] + UB * (np.abs(want[:, :hq]) + half_width[:, :hq]))
    assert np.all(got_q[m:] == 7)
    others = np.setdiff1d(np.arange(tokens), idx[:m])
    for codes, sc, first in ((k, ks, hq), (v, vs, hq + hk)):
        codes, sc = codes.cpu().numpy().reshape(tokens, hk, dh), sc.cpu().numpy()
        w, e = want[:, first:first + hk], half_width[:, first:first + hk]
        top = np.max(np.abs(w), 2, initial=0)
        lo, hi = scaled.scale_bytes(np.maximum(top - np.max(e, 2, initial=0), 0)), scaled.scale_bytes(top + np.max(e, 2, initial=0))
        s = sc[:, idx[:m]].T
        assert np.all((lo <= s) & (s <= hi))
        got = ref.cache_values(codes, sc)[idx[:m]]
        assert np.all(np.abs(got - w) <= np.maximum(U8 * (np.abs(w) + e), 2.0 ** -10 * scaled.powers(s)[..., None]) + e)
        assert np.all(codes[others] == FILL) and np.all(sc[:, others] == FILL)
        if dims is None or first > hq:   # unturned values are exact: so are their codes
            wc, wsb = ref.head_codes(w)
            np.testing.assert_array_equal(s, wsb)
            np.testing.assert_array_equal(codes[idx[:m]], wc)


def test_cache_write_bad_values():
    """A head that holds an infinity or a NaN is NaN as a whole; heads of zeros, and the others, are as ever."""
    x = np.ones((3, 5 * 64), np.float32)
    x[0, 3 * 64 - 1], x[1, 3 * 64 + 5], x[2, 4 * 64:] = np.inf, np.nan, 0
    k, v = (torch.zeros((3, 128), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((2, 3), dtype=torch.uint8, device="cuda") for _ in range(2))
    q = torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda")
    fdl.fd_cache_write(bf16(x).cuda(), None, None, count(3), q, k, ks, v, vs, 1, 2, 64)
    for codes, sc, first in ((k, ks, 1), (v, vs, 3)):
        wc, wsb = ref.head_codes(x.reshape(3, 5, 64)[:, first:first + 2].astype(np.float64))
        np.testing.assert_array_equal(sc.cpu().numpy().T, wsb)
        got = codes.cpu().numpy().reshape(3, 2, 64)
        assert np.all((got[wsb == 255] & 127) == 127)
        np.testing.assert_array_equal(got[wsb != 255], wc[wsb != 255])


# ------------------------------------------------------------------ attention

def cache(rng, tokens, hk, dh, spread=0.3):
    x = rng.standard_normal((tokens, hk, dh)) * np.exp(spread * rng.standard_normal((tokens, hk, 1)))
    codes, s = ref.head_codes(x)
    return codes.reshape(tokens, hk * dh), np.ascontiguousarray(s.T)


def run_attention(q, k, ks, v, vs, cu, off, hq, hk, dh, scale=None, longest=None, stream=None):
    rows = q.shape[0]
    o = torch.full((rows, hq * dh), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((fdl.fd_cache_attention_ws_size(rows, hq, hk, dh),), 0xFF, dtype=torch.uint8, device="cuda")    # NaN
    fdl.fd_cache_attention(q.cuda(), dev(k), dev(ks), dev(v), dev(vs), o, dev(cu), dev(off), hq, hk, dh, ws, max_request_tokens=longest, scale=scale)
    return o.double().cpu().numpy().reshape(rows, hq, dh)


def check_attention(got, q, k, ks, v, vs, cu, off, hq, hk, dh, scale=None):
    """Weights w_j = p_j / sum p: the p are off by a rounding to bf16 and by the exponent's error (the scores' sums of dh
    products and their scaling in fp32), and both enter twice, through the product and through the sum; then the result's rounding."""
    rows = q.shape[0]
    want, size, score = ref.attention(q.double().numpy().reshape(rows, hq, dh), ref.cache_values(k.reshape(-1, hk, dh), ks),
                                      ref.cache_values(v.reshape(-1, hk, dh), vs), cu, off, dh ** -0.5 if scale is None else scale)
    rel = UB + (dh + 8) * 2 * U32 * score + 2.0 ** -20
    err = 2 * rel * size + UB * np.abs(want) + 2.0 ** -100
    inside = slice(cu[0], cu[-1])
    worst = np.max(np.abs(got[inside] - want[inside]) - err[inside], initial=-np.inf)
    assert worst <= 0, f"off by {worst} more than allowed"
    assert np.all(got[:cu[0]] == 7) and np.all(got[cu[-1]:] == 7)


SHAPES = [([1], [1]), ([1], [64]), ([1], [65]), ([2], [130]), ([1], [5000]), ([33], [63]), ([5, 0, 3], [70, 64, 129]), ([0, 0, 1], [5, 0, 1]),
          ([3, 4, 2], [40, 0, 300]), ([300, 0, 257, 1], [129, 64, 700, 1]), ([31, 32, 33, 64, 65], [64, 65, 127, 128, 1]), ([520], [1000])]


@pytest.mark.parametrize("dh,hq,hk", [(16, 2, 2), (64, 3, 3), (64, 6, 2), (128, 2, 2), (128, 8, 1), (16, 10, 2)])
@pytest.mark.parametrize("q_len,k_len", SHAPES, ids=lambda v: "-".join(map(str, v)))
def test_attention(q_len, k_len, dh, hq, hk):
    gh.say(f"cache attention dh={dh} heads={hq}/{hk} rows={q_len} keys={k_len}")
    rng = np.random.default_rng([dh, hq, sum(q_len), sum(k_len)])
    lead, rows, tokens = 3, 2 + sum(q_len) + 3, 3 + sum(k_len) + 70
    cu, off = (np.concatenate([[0], np.cumsum(v)]).astype(np.int32) for v in (q_len, k_len))
    off += lead
    k, ks = cache(rng, tokens, hk, dh)
    v, vs = cache(rng, tokens, hk, dh)
    for c, s in ((k, ks), (v, vs)):          # tokens of no request are NaN
        c[:lead], c[off[-1]:], s[:, :lead], s[:, off[-1]:] = 0x7f, 0x7f, 255, 255
    q = bf16(rng.standard_normal((rows, hq * dh)) * np.exp(0.5 * rng.standard_normal((rows, 1))))
    q[cu[-1]:] = float("nan")
    got = run_attention(q, k, ks, v, vs, cu, off, hq, hk, dh, longest=max(k_len))
    check_attention(got, q, k, ks, v, vs, cu, off, hq, hk, dh)


@pytest.mark.parametrize("dh", [16, 64, 128])
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_attention_extremes(rows, dh):
    """Scores that grow by hundreds from tile to tile and fall again, equal scores, scales far from one, a head of zeros."""
    rng = np.random.default_rng([rows, dh, 7])
    tokens, hq, hk = 700, 4, 4
    x = rng.standard_normal((tokens, hk, dh))
    x[:, 0] *= np.linspace(-40, 60, tokens)[:, None]      # head 0: larger and larger keys
    x[:, 1] = 1.0                                         # head 1: equal keys
    x[:, 2] *= 2.0 ** -60                                 # head 2: tiny keys
    k, ks = ref.head_codes(x)
    y = rng.standard_normal((tokens, hk, dh))
    y[:, 1] *= 2.0 ** 90
    y[:, 2] *= 2.0 ** -90
    y[:, 3] = 0
    v, vs = ref.head_codes(y)
    k, v, ks, vs = k.reshape(tokens, -1), v.reshape(tokens, -1), np.ascontiguousarray(ks.T), np.ascontiguousarray(vs.T)
    q = bf16(4 * rng.standard_normal((rows, hq * dh)))
    cu, off = np.array([0, rows], np.int32), np.array([0, tokens], np.int32)
    for scale in (None, 0.01):
        got = run_attention(q, k, ks, v, vs, cu, off, hq, hk, dh, scale=scale)
        check_attention(got, q, k, ks, v, vs, cu, off, hq, hk, dh, scale)


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_attention_bad_values(rows):
    """A NaN key or value makes its head's rows of its request NaN, and no others."""
    rng = np.random.default_rng(rows)
    q_len, k_len, hk, dh = [rows, rows], [200, 333], 2, 64
    cu, off = (np.concatenate([[0], np.cumsum(v)]).astype(np.int32) for v in (q_len, k_len))
    k, ks = cache(rng, 533, hk, dh)
    v, vs = cache(rng, 533, hk, dh)
    q = bf16(rng.standard_normal((2 * rows, 2 * dh)))
    clean = run_attention(q, k, ks, v, vs, cu, off, 2, hk, dh)
    k[150, :dh], ks[0, 150] = 0x7f, 255                  # request 0, head 0
    v[500, dh:], vs[1, 500] = 0x7f, 255                  # request 1, head 1
    got = run_attention(q, k, ks, v, vs, cu, off, 2, hk, dh)
    assert np.all(np.isnan(got[:rows, 0])) and np.all(np.isnan(got[rows:, 1]))
    np.testing.assert_array_equal(got[:rows, 1], clean[:rows, 1])
    np.testing.assert_array_equal(got[rows:, 0], clean[rows:, 0])


def test_attention_repeats():
    """The same call again gives the same bits, whatever the workspace holds."""
    rng = np.random.default_rng(3)
    cu, off = np.array([0, 1, 200], np.int32), np.array([0, 3000, 5000], np.int32)
    k, ks = cache(rng, 5000, 2, 128)
    v, vs = cache(rng, 5000, 2, 128)
    q = bf16(rng.standard_normal((200, 4 * 128)))
    runs = [run_attention(q, k, ks, v, vs, cu, off, 4, 2, 128) for _ in range(3)]
    np.testing.assert_array_equal(runs[0], runs[1])
    np.testing.assert_array_equal(runs[0], runs[2])
