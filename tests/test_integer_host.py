"""CPU tests of the integer rows, their product, the norms on both sides of a branch and the 8-bit cache: refusals before any
launch, the 64-bit reference, and the schedule of the attention over the cache."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import integer as ref
from oracle import scaled
from paper_2607_12121_amd import build
from paper_2607_12121_amd import flashdiff as fdl
from tests.test_abi import no_gpu
from tests.test_isa_hazards import _hazards

P = 0x1000
BIG = (1 << 30) + 1


# ------------------------------------------------------------------ the reference

def test_reference_rows():
    """Values within half a step (three roundings of up to 127 steps beside it), the largest one 127, ties to even."""
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((50, 96)) * np.exp(4 * rng.standard_normal((50, 1)))).astype(np.float32)
    q, s = ref.int_rows(x)
    assert np.all(np.max(np.abs(q.astype(int)), 1) == 127)
    assert np.all(np.abs(q * s.astype(np.float64)[:, None] - x) <= s[:, None] * (0.5 + 127 * 3 * 2.0 ** -24))
    q, s = ref.int_rows(np.array([[254, 1, 3, 5, -1, -3]], np.float32))
    assert q.tolist() == [[127, 0, 2, 2, 0, -2]] and s[0] == 2
    q, s = ref.int_rows(np.array([[0, 0], [1e-38, 0], [np.inf, 1], [np.nan, 1]], np.float32))
    assert not q.any() and s[0] == s[1] == 0 and np.isnan(s[2:]).all()


def test_reference_attention():
    """Equal keys average the values; a row's weights do not change with a shift of its scores; shared key heads."""
    rng = np.random.default_rng(1)
    k, v, q = rng.standard_normal((7, 2, 16)), rng.standard_normal((7, 2, 16)), rng.standard_normal((3, 6, 16))
    o, _, _ = ref.attention(q, np.ones_like(k), v, [0, 2, 3], [0, 4, 7], 0.25)
    np.testing.assert_allclose(o[0, 4], v[:4, 1].mean(0))
    np.testing.assert_allclose(o[2, 2], v[4:, 0].mean(0))
    o, size, score = ref.attention(q, k, v, [0, 0, 2], [0, 0, 7], 0.25)
    w = np.exp(0.25 * k[:, 1] @ q[1, 3])
    np.testing.assert_allclose(o[1, 3], w @ v[:, 1] / w.sum())
    assert np.isnan(o[2]).all() and (size >= np.abs(np.nan_to_num(o)) - 1e-12).all() and (score[:2] > 0).all()


def test_reference_head_codes():
    x = np.random.default_rng(2).standard_normal((5, 3, 64))
    c, s = ref.head_codes(x)
    want, ws = scaled.quant(np.concatenate([x, np.zeros_like(x)], 2).reshape(5, -1))     # a block of 128 columns a head
    np.testing.assert_array_equal(c, want.reshape(5, 3, 128)[..., :64])
    np.testing.assert_array_equal(s, ws)


# ------------------------------------------------------------------ refusals

@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(rows=0), 1), (dict(cols=0), 1), (dict(cols=24), 3), (dict(cols=65552), 3), (dict(rows=BIG), 3), (dict(x=None), 1), (dict(q=None), 1),
    (dict(scale=None), 1), (dict(x=P + 8), 1), (dict(q=P + 8), 1), (dict(scale=P + 2), 1)])
def test_int_rows_refuses(change, status):
    a = dict(rows=4, cols=64, x=P, m=P, q=P, scale=P)
    a.update(change)
    assert fdl.lib().fd_int_rows(*a.values(), None) == status, fdl.lib().fd_last_error()


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(rows=0), 1), (dict(n=0), 1), (dict(k=0), 1), (dict(n=40), 3), (dict(k=72), 3), (dict(k=65552), 3), (dict(n=(1 << 20) + 16), 3), (dict(rows=BIG), 3),
    (dict(n=1 << 16, k=1 << 15), 3), (dict(a=None), 1), (dict(sa=None), 1), (dict(w=None), 1), (dict(sw=None), 1), (dict(yb=None), 1), (dict(yf=P), 1),
    (dict(gelu=2), 1), (dict(a=P + 8), 1), (dict(w=P + 8), 1), (dict(sa=P + 2), 1), (dict(sw=P + 4), 1), (dict(bias=P + 4), 1), (dict(yb=P + 8), 1),
    (dict(yb=None, yf=P + 8), 1)])
def test_int_linear_refuses(change, status):
    a = dict(rows=4, n=64, k=64, a=P, sa=P, w=P, sw=P, bias=P, gelu=0, m=P, yb=P, yf=None)
    a.update(change)
    assert fdl.lib().fd_int_linear(*a.values(), None) == status, fdl.lib().fd_last_error()


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(rows=0), 1), (dict(D=0), 1), (dict(D=72), 3), (dict(D=12304), 3), (dict(B=0), 1), (dict(rows=BIG), 3), (dict(h=None), 1), (dict(m=None), 1),
    (dict(B=2, cu_q=None), 1), (dict(y=None, ab=None), 1), (dict(ac=P, sc=P), 1), (dict(ab=None, ac=P), 1), (dict(ab=None, sc=P), 1),
    (dict(ab=None, ai=P), 1), (dict(ab=None, si=P), 1), (dict(ab=None, ac=P, sc=P, ai=P, si=P), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
    (dict(residual=float("inf")), 1), (dict(residual=float("nan")), 1), (dict(stride=-4), 1), (dict(stride=6), 1), (dict(h=P + 4), 1), (dict(y=P + 8), 1),
    (dict(post=P + 4), 1), (dict(gate=P + 4), 1), (dict(weight=P + 4), 1), (dict(shift=P + 4), 1), (dict(scale=P + 4), 1), (dict(ab=P + 8), 1),
    (dict(ab=None, ac=P + 8, sc=P), 1), (dict(ab=None, ai=P + 8, si=P), 1), (dict(ab=None, ai=P, si=P + 2), 1)])
def test_norm_residual_refuses(change, status):
    a = dict(rows=4, D=64, B=1, h=P, y=P, residual=1.0, post=P, gate=P, weight=P, shift=P, scale=P, stride=192, eps=1e-6, cu_q=P, m=P,
             ab=P, ac=None, sc=None, ai=None, si=None)
    a.update(change)
    assert fdl.lib().fd_norm_residual(*a.values(), None) == status, fdl.lib().fd_last_error()


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(rows=0), 1), (dict(rows=9), 1), (dict(rows=BIG, tokens=BIG), 3), (dict(hq=0), 1), (dict(hk=0), 1), (dict(hq=5000), 3), (dict(hk=5000), 3), (dict(dh=32), 3), (dict(coord=None), 1),
    (dict(qkv=None), 1), (dict(m=None), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(ks=None), 1), (dict(v=None), 1), (dict(vs=None), 1),
    (dict(qkv=P + 8), 1), (dict(q=P + 8), 1), (dict(k=P + 8), 1), (dict(v=P + 8), 1), (dict(rope=ctypes.byref(fdl.rope_axes([66]))), 1)])
def test_cache_write_refuses(change, status):
    a = dict(rows=4, tokens=8, rope=ctypes.byref(fdl.rope_axes([64])), hq=2, hk=1, dh=64, coord=P, qkv=P, idx=P, m=P, q=P, k=P, ks=P, v=P, vs=P)
    a.update(change)
    assert fdl.lib().fd_cache_write(*a.values(), None) == status, fdl.lib().fd_last_error()


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(rows=0), 1), (dict(tokens=0), 1), (dict(B=0), 1), (dict(longest=-1), 1), (dict(longest=9), 1), (dict(B=1025), 3), (dict(rows=BIG), 3), (dict(tokens=BIG), 3),
    (dict(hq=0), 1), (dict(hk=0), 1), (dict(hq=3), 1), (dict(dh=32), 3), (dict(hq=5000), 3), (dict(rows=1 << 26, hq=64), 3), (dict(scale=0.0), 1), (dict(scale=-1.0), 1),
    (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(ks=None), 1), (dict(v=None), 1), (dict(vs=None), 1),
    (dict(cu=None), 1), (dict(off=None), 1), (dict(o=None), 1), (dict(ws=None), 1), (dict(q=P + 8), 1), (dict(k=P + 8), 1), (dict(v=P + 8), 1), (dict(o=P + 8), 1),
    (dict(ws=P + 16), 1), (dict(n=100), 2)])
def test_cache_attention_refuses(change, status):
    a = dict(rows=4, tokens=8, B=1, longest=8, hq=4, hk=2, dh=64, scale=0.125, q=P, k=P, ks=P, v=P, vs=P, cu=P, off=P, o=P, ws=P, n=1 << 40)
    a.update(change)
    assert fdl.lib().fd_cache_attention(*a.values(), None) == status, fdl.lib().fd_last_error()


def test_attention_workspace():
    size = fdl.fd_cache_attention_ws_size
    for bad in ((0, 2, 2, 64), (4, 0, 1, 64), (4, 3, 2, 64), (4, 2, 0, 64), (4, 2, 2, 32)):
        assert size(*bad) == 0
    # calls that only run with few rows need less
    assert 0 < size(96, 2, 2, 128) < size(97, 2, 2, 128) == size(1 << 20, 2, 2, 128)
    assert size(16, 8, 2, 64) < size(17, 8, 2, 64)


def test_bindings_refuse():
    """Absent, host, wide and mismatched tensors raise with the argument's name."""
    x, q8, f, i = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4), torch.zeros(2, dtype=torch.int32)
    c, ks, h, ws = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(1, 4, dtype=torch.uint8), torch.zeros(4, 64), torch.zeros(256, dtype=torch.uint8)
    wide = torch.zeros(1, 1, dtype=torch.int8).expand((1 << 32) + 4, 16)
    qkv = torch.zeros(4, 192, dtype=torch.bfloat16)
    write = lambda **kw: fdl.fd_cache_write(**{**dict(qkv=qkv, coord=None, idx=None, m=i, q=x, k=c, k_scale=ks, v=c, v_scale=ks, heads=1, kv_heads=1, head_dim=64), **kw})  # noqa: E731
    attn = lambda **kw: fdl.fd_cache_attention(**{**dict(q=x, k=c, k_scale=ks, v=c, v_scale=ks, o=x, cu_q=i, req_tok_off=i, heads=1, kv_heads=1, head_dim=64, ws=ws), **kw})  # noqa: E731
    for call, what in [
            (lambda: fdl.fd_int_rows(None, q8, f), "x is"), (lambda: fdl.fd_int_rows(x, q8, f), "x must be a device"), (lambda: fdl.fd_int_rows(wide, q8, f), "at most 2"),
            (lambda: fdl.fd_int_linear(None, f, q8, f, h), "a is"), (lambda: fdl.fd_int_linear(q8, f, None, f, h), "w is"), (lambda: fdl.fd_int_linear(q8, f, q8, f, None), "y is"),
            (lambda: fdl.fd_int_linear(q8, f, q8[:, :32], f, h), "64 columns, w 32"), (lambda: fdl.fd_int_linear(q8, f, q8, f, h), "a must be a device"),
            (lambda: fdl.fd_norm_residual(None, x, i, i), "h is"), (lambda: fdl.fd_norm_residual(h, x, i, i), "h must be a device"),
            (lambda: fdl.fd_norm_residual(h, x, i, i, a_scale=f), "a_scale belongs"), (lambda: fdl.fd_norm_residual(h, None, i, i, a_scale=f), "a_scale belongs"),
            (lambda: fdl.fd_norm_residual(h, x, i, i, gate=h), "gate, shift and mod_scale"),
            (lambda: write(qkv=None), "qkv is"), (lambda: write(k=None), "k is"), (lambda: write(k_scale=None), "k_scale is"), (lambda: write(heads=2), "qkv has 192"),
            (lambda: write(k=c[:, :32]), "k has 32"), (lambda: write(v_scale=ks.t()), "v_scale must be"), (lambda: write(v=c[:3], v_scale=ks[:, :3]), "same tokens"),
            (lambda: write(coord=i.view(2, 1)), "both coord and the axes"), (lambda: write(dims=[64]), "both coord and the axes"), (lambda: write(coord=i.view(2, 1), dims=[64]), "coord must be"),
            (lambda: write(), "must be a device"),
            (lambda: attn(q=None), "q is"), (lambda: attn(heads=2), "q has 64"), (lambda: attn(k=c[:, :32]), "k has 32"), (lambda: attn(v=c[:3], v_scale=ks[:, :3]), "same tokens"),
            (lambda: attn(cu_q=i[:1]), "requests"), (lambda: attn(req_tok_off=None), "requests"), (lambda: attn(cu_q=torch.zeros(3, dtype=torch.int32)), "requests"),
            (lambda: attn(ws=None), "ws"), (lambda: attn(), "must be a device|ws must")]:
        with pytest.raises(fdl.FlashDiffError, match=what):
            call()


# ------------------------------------------------------------------ the attention's schedule

SHIM = r"""
#include "fd_cache_sched.h"
template <int DH>
int pieces(int few, int may_cut, const int32_t* cu, const int32_t* tok, int B, int group, int H, int G, int nkv_max, int* out, int cap) {
  static fd::SchedTables t;
  const int qb = few ? fd::kFewRows : fd::cache_tile_rows(DH), kb = few ? fd::cache_few_keys(DH) : 64;
  long long tiles = 0;
  for (int b = 0; b < B; ++b) {
    const int rows = (cu[b + 1] - cu[b]) * group, keys = tok[b + 1] - tok[b];
    if (rows > 0 && keys > 0) tiles += (rows + qb - 1) / qb;
  }
  const int start = few ? 0 : fd::cache_item_steps(tiles * H, G);
  t.tpre[0] = 0; t.wpre[0] = 0;
  for (int b = 0; b < B; ++b) {
    const int rows = (cu[b + 1] - cu[b]) * group, keys = tok[b + 1] - tok[b], n = rows > 0 && keys > 0 ? (rows + qb - 1) / qb : 0;
    t.tpre[b + 1] = t.tpre[b] + n;
    t.wpre[b + 1] = t.wpre[b] + static_cast<long long>(n) * ((keys + kb - 1) / kb + start);
  }
  const fd::CacheSched<DH> s(&t, cu, tok, B, H, G, nkv_max, few, may_cut, start);
  int n = 0;
  if (s.work == 0) return 0;
  for (int blk = 0; blk < G; ++blk) {
    const int w = s.share(blk);
    long long p = s.bound(w);
    const long long p_end = s.bound(w + 1);
    while (p < p_end) {
      long long i0;
      int len, head, b, first, tau;
      s.locate(p, i0, len, head, b, first, tau);
      const int s0 = static_cast<int>(p - i0), s1 = static_cast<int>((p_end < i0 + len ? p_end : i0 + len) - i0);
      const int slot = s.cut ? s.slot_of(w, s0, s1, len) : -1;
      if (n == cap) return -1;
      const int row[9] = {w, head, b, tau - first, s.tile(s0), s.tile(s1), slot, slot >= 0 && s0 == 0 ? s.last_share(i0 + len) : -1, s.cut};
      for (int k = 0; k < 9; ++k) out[9 * n + k] = row[k];
      ++n;
      p = i0 + s1;
    }
  }
  return n;
}
extern "C" {
int cache_pieces(int dh, int few, int may_cut, const int32_t* cu, const int32_t* tok, int B, int group, int H, int G, int nkv_max, int* out, int cap) {
  return dh == 16 ? pieces<16>(few, may_cut, cu, tok, B, group, H, G, nkv_max, out, cap) : dh == 64 ? pieces<64>(few, may_cut, cu, tok, B, group, H, G, nkv_max, out, cap)
                                                                                                  : pieces<128>(few, may_cut, cu, tok, B, group, H, G, nkv_max, out, cap);
}
int slot_at(int x, int j) { return fd::CacheSched<64>::slot_at(x, j); }
int few_rows(int dh, int few, int tiles) { return fd::cache_few_rows(dh, few, tiles); }
int always_few(int dh, long long rows) { return fd::cache_always_few(dh, rows); }
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("sched")
    (d / "s.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{build.CSRC}", str(d / "s.cpp"), "-o", str(d / "s.so")], check=True)
    return ctypes.CDLL(str(d / "s.so"))


def check_schedule(shim, dh, few, may_cut, q_len, k_len, group, H, G):
    """Every key step of every item once and in order, no piece without keys; the pieces of a cut item lie in one share after the
    other, in the slots that the join reads, and the first one's share knows the last."""
    cu, tok = (np.concatenate([[0], np.cumsum(v)]).astype(np.int32) for v in (q_len, k_len))
    out = np.zeros((200000, 9), np.int32)
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    n = shim.cache_pieces(dh, few, may_cut, p(cu), p(tok), len(q_len), group, H, G, int(max(k_len) + 63) // 64, p(out), len(out))
    assert n >= 0
    qb, kb = (32, 512 if dh >= 64 else 256) if few else (256 if dh >= 64 else 128, 64)
    items = {(h, b, t): -(-k // kb) for h in range(H) for b, (q, k) in enumerate(zip(q_len, k_len)) if k for t in range(-(-q * group // qb))}
    got = {}
    for w, h, b, t, k0, k1, slot, last, cut in out[:n].tolist():
        assert 0 <= k0 < k1 and slot < 2 * G
        got.setdefault((h, b, t), []).append((k0, k1, w, slot, last))
    assert set(got) == set(items)
    used = set()
    for key, ps in got.items():
        ps.sort()
        assert [a[0] for a in ps] == [0] + [a[1] for a in ps[:-1]] and ps[-1][1] == items[key]
        if len(ps) == 1:
            assert ps[0][3] == -1
            continue
        assert may_cut
        first = ps[0][2]
        assert [a[2] for a in ps] == list(range(first, first + len(ps)))
        assert ps[0][4] == first + len(ps) - 1 and all(a[4] == -1 for a in ps[1:])
        assert [a[3] for a in ps] == [shim.slot_at(first, j) for j in range(len(ps))]
        assert not used & {a[3] for a in ps}
        used |= {a[3] for a in ps}
    return out[:n]


@pytest.mark.parametrize("dh", [16, 64, 128])
def test_schedule_runs_every_step_once(shim, dh):
    rng = np.random.default_rng(dh)
    cuts = 0
    for trial in range(400):
        B = int(rng.choice([1, 1, 2, 3, 8, 70]))
        few, may_cut = bool(rng.integers(2)), bool(rng.integers(4))
        k_len = np.where(rng.random(B) < 0.1, 0, np.exp(rng.uniform(0, 10.4 if B < 8 else 8, B)).astype(int))
        most = 200 if few else 3000
        q_len = np.where(rng.random(B) < 0.1, 0, np.exp(rng.uniform(0, np.log(most), B)).astype(int))
        group, H, G = int(rng.choice([1, 1, 2, 3, 8])), int(rng.integers(1, 25)), int(rng.choice([256, 512, 8]))
        rows = check_schedule(shim, dh, few, may_cut, q_len, np.maximum(k_len, 0), group, H, G)
        cuts += int(len(rows) and rows[0, 8])
    assert cuts > 50


def test_schedule_of_a_video_row(shim):
    """One row of 12 heads over 32760 keys: 768 steps, three a workgroup."""
    rows = check_schedule(shim, 128, True, True, [1], [32760], 1, 12, 256)
    assert np.all(np.bincount(rows[:, 0], weights=rows[:, 5] - rows[:, 4]) == 3)


@pytest.mark.parametrize("dh,most", [(16, 3), (64, 2), (128, 3)])
def test_few_rows_rule(shim, dh, most):
    assert shim.few_rows(dh, most, 1) and not shim.few_rows(dh, most + 1, 1)
    assert shim.always_few(dh, ctypes.c_longlong(32 * most)) and not shim.always_few(dh, ctypes.c_longlong(32 * most + 1))
    for rows in range(1, 200):      # always_few: however the rows are spread over requests
        for parts in (1, 2, 5):
            q = [rows // parts + (i < rows % parts) for i in range(parts)]
            few, tiles = sum(-(-n // 32) for n in q), sum(-(-n // (256 if dh >= 64 else 128)) for n in q)
            assert not shim.always_few(dh, ctypes.c_longlong(rows)) or shim.few_rows(dh, few, tiles)


def test_product_rules(tmp_path):
    """Which kernel a product runs: few rows, tiles of split K-blocks where each has a CU, or neither."""
    (tmp_path / "r.cpp").write_text("""#include "fd_int_rules.h"
extern "C" int way(int M, int N, int K, int cus) { return fd::int_few(M, N, K, cus) ? -1 : fd::int_split(M, N, K, cus); }
extern "C" int large(int M, int N, int K, int wide, int cus) { return fd::int_large(M, N, K, wide, cus); }
""")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", f"-I{build.CSRC}", str(tmp_path / "r.cpp"), "-o", str(tmp_path / "r.so")], check=True)
    lib = ctypes.CDLL(str(tmp_path / "r.so"))
    way = lib.way
    for M, N, K, wide, want in ((5000, 1600, 6400, 0, 1), (2048, 6400, 6400, 0, 1), (2600, 6400, 6400, 0, 0), (9828, 6144, 1536, 0, 1), (9828, 1536, 6144, 0, 1),
                                (5000, 1536, 6144, 0, 0), (6000, 4608, 1536, 1, 0), (32760, 1536, 6144, 1, 1), (1664, 1536, 6144, 0, 0), (1 << 30, 1 << 20, 65536, 1, 1)):
        assert lib.large(M, N, K, wide, 256) == want, (M, N, K)
    few, none, split32, split32x64, split64 = -1, 0, 1, 2, 3
    for M, N, K, want in ((1, 4608, 1536, few), (1, 4608, 6144, split32), (1, 1536, 6144, few), (16, 1536, 6144, split32), (1, 65536, 4096, few),
                          (16, 8208, 4096, few), (17, 1536, 1088, few), (17, 1536, 1536, split32), (64, 1536, 1088, few), (64, 1536, 6144, split32),
                          (129, 1536, 6144, split32), (171, 1536, 6144, split32x64), (256, 1536, 6144, split32x64), (512, 1536, 6144, split64),
                          (512, 1536, 1536, none), (700, 1536, 6144, none), (1021, 4288, 1088, none), (9828, 6144, 1536, none)):
        assert way(M, N, K, 256) == want, (M, N, K)
    rng = np.random.default_rng(0)
    for M, N, K in zip(*(np.exp(rng.uniform(0, np.log(t), 3000)).astype(int) for t in (40000, 4000, 4000))):
        M, N, K = int(M), 16 * int(N), 16 * int(K)
        w = way(M, N, K, 256)
        if w > 0:      # a round of workgroups
            bm, bn = {split32: (32, 32), split32x64: (32, 64), split64: (64, 64)}[w]
            assert -(-M // bm) * -(-N // bn) <= 256


def test_no_vector_memory_read_of_a_fresh_scalar(tmp_path):
    """The integer product's loads in inline assembly, searched as those of the bf16 products are."""
    out = tmp_path / "k.s"
    subprocess.run([build.hipcc(), *[f for f in build.HIPCC_FLAGS if f != "-Wall"], "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, "k_int_gemm.hip"), "-o", str(out)], check=True, capture_output=True)
    seen, bad = _hazards(out.read_text().splitlines())
    assert seen > 300
    assert not bad, bad[:3]
