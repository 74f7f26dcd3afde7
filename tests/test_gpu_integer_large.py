"""The integer rows, the norms, the product and the 8-bit cache where offsets pass 2 and 4 GiB: rows at both ends of buffers that
long, against the same rows in buffers of their own (whose numerics the other tests hold to the 64-bit reference)."""
import pytest
import torch

from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_scaled_large import count, ends, filled

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


def test_rows_and_product():
    """2.2 million rows of 1024: 4.5 GB of bf16, 2.25 GB of integers; results of 4.5 GB."""
    rows, cols = 2_200_000, 1024
    pick = ends(rows)
    gh.say(f"integer rows and product of {rows} x {cols}")
    x, part = filled(pick, rows, cols, torch.bfloat16)
    (q, s), (q2, s2) = ((torch.empty((n, cols), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")) for n in (rows, len(pick)))
    fdl.fd_int_rows(x, q, s)
    fdl.fd_int_rows(part, q2, s2)
    assert torch.equal(q[pick], q2) and torch.equal(s[pick], s2)
    del x
    w, sw = torch.randint(-127, 128, (528, cols), device="cuda", dtype=torch.int32).to(torch.int8), torch.rand(528, device="cuda")
    for m in (None, count(rows)):
        y, y2 = (torch.zeros((n, 528), dtype=torch.float32, device="cuda") for n in (rows, len(pick)))
        fdl.fd_int_linear(q, s, w, sw, y, m=m)
        fdl.fd_int_linear(q2, s2, w, sw, y2)
        assert torch.equal(y[pick], y2)


def test_norm_residual():
    """1.2 million rows of 1024: 4.9 GB of h."""
    rows, D = 1_200_000, 1024
    pick = ends(rows)
    gh.say(f"norms of {rows} x {D}")
    h, part = filled(pick, rows, D, torch.float32)
    y, y_part = filled(pick, rows, D, torch.bfloat16)
    (a, s), (a2, s2) = ((torch.empty((n, D), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")) for n in (rows, len(pick)))
    fdl.fd_norm_residual(h, a, None, count(rows), y=y, a_scale=s)
    fdl.fd_norm_residual(part, a2, None, count(len(pick)), y=y_part, a_scale=s2)
    assert torch.equal(h[pick], part) and torch.equal(a[pick], a2) and torch.equal(s[pick], s2)


def test_cache():
    """2.2 million tokens of 16 heads of 128: 4.5 GB of codes each; a request at each end and a long one between."""
    tokens, hk, dh = 2_200_000, 16, 128
    gh.say(f"cache of {tokens} tokens")
    pick = ends(tokens, 700)
    n = len(pick)
    qkv = torch.randn((n, 3 * hk * dh), device="cuda").to(torch.bfloat16)
    k, v = (torch.zeros((tokens, hk * dh), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((hk, tokens), 1, dtype=torch.uint8, device="cuda") for _ in range(2))
    k2, v2 = (torch.zeros((n, hk * dh), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks2, vs2 = (torch.zeros((hk, n), dtype=torch.uint8, device="cuda") for _ in range(2))
    q, q2, o, o2 = (torch.zeros((n, hk * dh), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    fdl.fd_cache_write(qkv, None, pick.to(torch.int32), count(n), q, k, ks, v, vs, hk, hk, dh)
    fdl.fd_cache_write(qkv, None, None, count(n), q2, k2, ks2, v2, vs2, hk, hk, dh)
    assert torch.equal(q, q2) and torch.equal(k[pick], k2) and torch.equal(v[pick], v2)
    assert torch.equal(ks[:, pick], ks2) and torch.equal(vs[:, pick], vs2)
    cu = torch.tensor([0, 700, 700, 1400], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 700, tokens - 700, tokens], dtype=torch.int32, device="cuda")
    off2 = torch.tensor([0, 700, 700, 1400], dtype=torch.int32, device="cuda")
    ws = torch.empty(fdl.fd_cache_attention_ws_size(n, hk, hk, dh), dtype=torch.uint8, device="cuda")
    fdl.fd_cache_attention(q, k, ks, v, vs, o, cu, off, hk, hk, dh, ws, max_request_tokens=700)
    fdl.fd_cache_attention(q2, k2, ks2, v2, vs2, o2, cu, off2, hk, hk, dh, ws, max_request_tokens=700)
    assert torch.equal(o, o2)
    # a row over all 2.2 million keys: zeros but for the two ends, whose scores' softmax the plain form in 64 bits gives
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for rows in (1, 300):      # few rows, tiles
        cu1 = one * rows
        off1 = torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
        got = torch.zeros((300, hk * dh), dtype=torch.bfloat16, device="cuda")
        fdl.fd_cache_attention(q[:300].contiguous(), k, ks, v, vs, got, cu1, off1, hk, hk, dh, ws)
        for r in {0, rows - 1}:
            for h in (0, hk - 1):
                c = slice(h * dh, (h + 1) * dh)
                val = lambda t, s: t[:, c].view(torch.float8_e4m3fn).double() * torch.exp2(s[h].double() - 127)[:, None]  # noqa: E731
                kk, vv = val(k2, ks2), val(v2, vs2)
                s = (kk @ q2[r, c].double()) * dh ** -0.5
                top = torch.clamp(s.max(), min=0)
                e = torch.exp(s - top)
                l = e.sum() + (tokens - n) * torch.exp(-top)
                want, size = (e @ vv) / l, (e @ vv.abs()) / l
                # weights off by a rounding to bf16 twice and by the exponent's error; every zero key's weight in the sum
                score = (kk.abs() @ q2[r, c].double().abs()).max() * dh ** -0.5
                rel = 2.0 ** -8 + (dh + 8) * 2.0 ** -23 * score + 2.0 ** -20
                err = 2 * rel * size + 2.0 ** -8 * want.abs() + 2.0 ** -100
                assert bool(((got[r, c].double() - want).abs() <= err).all()), (rows, r, h)
