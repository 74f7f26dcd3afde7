"""The 8-bit operators where offsets pass 2 and 4 GiB: rows at both ends of buffers that long, against the same rows in
buffers of their own (whose numerics test_gpu_scaled.py holds to the 64-bit reference)."""
import pytest
import torch

from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


def count(m):
    return torch.tensor([m], dtype=torch.int32, device="cuda")


def code(rows, cols, lead=None):
    return (torch.empty((rows, cols), dtype=torch.uint8, device="cuda"),
            torch.empty((rows if lead is None else lead, fdl.fd_scale_stride(cols)), dtype=torch.uint8, device="cuda"))


def ends(rows, n=200):
    return torch.cat([torch.arange(n), torch.arange(rows - n, rows)]).cuda()


def filled(pick, rows, cols, dtype):
    """[rows][cols] of zeros with random values in the rows `pick`, and those rows alone."""
    part = torch.randn((len(pick), cols), device="cuda").to(dtype)
    x = torch.zeros((rows, cols), dtype=dtype, device="cuda")
    x[pick] = part
    return x, part


def test_quant_and_product_rows():
    """2.2 million rows of 1024: 4.5 GB of bf16, 2.25 GB of codes."""
    rows, cols = 2_200_000, 1024
    pick = ends(rows)
    gh.say(f"quant and product of {rows} x {cols}")
    x, part = filled(pick, rows, cols, torch.bfloat16)
    (q, s), (q2, s2) = code(rows, cols), code(len(pick), cols)
    fdl.fd_quant_blocks(x, 1, q, s)
    fdl.fd_quant_blocks(part, 1, q2, s2)
    nk = cols // 128
    assert torch.equal(q[pick], q2) and torch.equal(s[pick][:, :nk], s2[:, :nk])
    del x
    w16 = torch.randn((64, cols), device="cuda").to(torch.bfloat16)
    w, sw = code(64, cols, 1)
    fdl.fd_quant_blocks(w16, 128, w, sw)
    for m in (None, count(rows)):
        y, y2 = (torch.zeros((n, 64), dtype=torch.bfloat16, device="cuda") for n in (rows, len(pick)))
        fdl.fd_scaled_linear(q, s, w, sw, y, m=m)
        fdl.fd_scaled_linear(q2, s2, w, sw, y2)
        assert torch.equal(y[pick], y2)


@pytest.mark.parametrize("to", ["f32", "8"])
def test_product_results(to):
    """300000 x 4096 results: 4.9 GB in fp32, 1.2 GB of codes."""
    rows, n, k = 300_000, 4096, 384
    pick = ends(rows)
    gh.say(f"product of {rows} x {n} to {to}")
    x, part = filled(pick, rows, k, torch.bfloat16)
    (q, s), (q2, s2), (w, sw) = code(rows, k), code(len(pick), k), code(n, k, n // 128)
    fdl.fd_quant_blocks(x, 1, q, s)
    fdl.fd_quant_blocks(part, 1, q2, s2)
    fdl.fd_quant_blocks(torch.randn((n, k), device="cuda").to(torch.bfloat16), 128, w, sw)
    if to == "8":
        (y, ys), (y2, ys2) = code(rows, n), code(len(pick), n)
    else:
        (y, ys), (y2, ys2) = ((torch.zeros((r, n), device="cuda"), None) for r in (rows, len(pick)))
    fdl.fd_scaled_linear(q, s, w, sw, y, ys)
    fdl.fd_scaled_linear(q2, s2, w, sw, y2, ys2)
    assert torch.equal(y[pick], y2)
    if to == "8":
        assert torch.equal(ys[pick], ys2)


def test_rms_rows():
    """1.1 million rows of 1024: 4.5 GB of the residual stream."""
    rows, cols = 1_100_000, 1024
    pick = ends(rows)
    gh.say(f"rms of {rows} x {cols}")
    h, part = filled(pick, rows, cols, torch.float32)
    y, ypart = filled(pick, rows, cols, torch.bfloat16)
    (q, s), (q2, s2) = code(rows, cols), code(len(pick), cols)
    fdl.fd_rms_quant(h, q, s, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), count(rows), y=y)
    fdl.fd_rms_quant(part, q2, s2, torch.tensor([0, len(pick)], dtype=torch.int32, device="cuda"), count(len(pick)), y=ypart)
    assert torch.equal(h[pick], part) and torch.equal(q[pick], q2) and torch.equal(s[pick][:, :8], s2[:, :8])


def test_rope_rows():
    """750000 rows of 3 x 1024: 4.6 GB in, caches past 1.5 GB; tokens in reverse, so that first rows meet last tokens."""
    rows, heads, dh = 750_000, 8, 128
    pick = ends(rows)
    gh.say(f"rope of {rows} rows")
    x, part = filled(pick, rows, 3 * heads * dh, torch.bfloat16)
    coord = torch.randint(0, 5000, (rows, 2), dtype=torch.int32, device="cuda")
    idx = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((rows, heads * dh), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    kw = dict(heads=heads, kv_heads=heads, head_dim=dh, dims=[64, 64])
    fdl.fd_rope_axes(x, coord, idx, count(rows), q, k, v, **kw)
    q2, k2, v2 = (torch.zeros((len(pick), heads * dh), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    tok = idx[pick].long()
    fdl.fd_rope_axes(part, coord[tok].contiguous(), None, count(len(pick)), q2, k2, v2, **kw)
    assert torch.equal(q[pick], q2) and torch.equal(k[tok], k2) and torch.equal(v[tok], v2)
